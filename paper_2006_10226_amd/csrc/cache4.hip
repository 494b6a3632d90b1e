// Writing and reading the 4-bit cache of include/qnn.h: one group of DP / 8
// neighbouring lanes per vector (a token's K or V of one head), eight channels
// a lane. The range of a vector comes from shuffles inside its group, so each
// input is read once and each code written once. 16384 tokens of 8 heads of 128 in
// f16, 85 MB moved: read back 18.7 us, a copy's rate (4.6 TB/s); written 22.6 us (3.8
// TB/s; with every eighth token skipped 21.8), bound by vector instructions (25 a
// value: conversion, range, quotient, rounding, addresses): its 13.1 million wave
// instructions are 21.3 us of issue at 2.4 GHz. 8-bit rows have half the bytes to
// read and as many instructions, 24.5 us.
#include "cache4.h"

#include <algorithm>

namespace qnn {
namespace {

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));

struct VecArgs {
    Cache4Args c;
    const void *k, *v;         // append: inputs
    void *ko, *vo;             // read: outputs
    int64_t k_ld, v_ld;
    const int32_t *slots;
    int32_t tokens;
    float ks, vs;              // 8-bit inputs
    int32_t kz, vz;
};

// Eight values of element type DT (qnn_dtype) at p, as f32.
template <int DT>
__device__ __forceinline__ void load8(const void *p, float s, int z, float (&x)[8])
{
    if constexpr (DT == QNN_FLOAT16) {
        const h8 h = *(const h8 *)p;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            x[i] = (float)h[i];
    } else if constexpr (DT == QNN_BFLOAT16) {
        const u4 w = *(const u4 *)p;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __builtin_bit_cast(float, w[i] << 16);
            x[2 * i + 1] = __builtin_bit_cast(float, w[i] & 0xffff0000u);
        }
    } else {
        const u2 w = *(const u2 *)p;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t b = (w[i >> 2] >> (8 * (i & 3))) & 0xffu;
            x[i] = (float)((DT == QNN_INT8 ? (int)(int8_t)b : (int)b) - z) * s;
        }
    }
}

// The value of another lane of the same 16 (a DPP control).
template <int CTRL>
__device__ __forceinline__ uint32_t lane_move(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 15, 15, true);
}

__device__ __forceinline__ uint32_t as_bits(float v) { return __builtin_bit_cast(uint32_t, v); }

// Thread -> vector: the workgroup's 256 threads take eight consecutive tokens
// of one head (16 for DP 64, four for 256), K and V, so that the tokens of a V
// tile are written together.
template <int DP>
struct Map {
    static constexpr int kLanes = DP / 8;                // per vector
    static constexpr int kVectors = 256 / kLanes;        // per workgroup
    static constexpr int kTokens = kVectors / 2;         // K and V
};

// V's two-byte units lie 16 bytes apart for one token and side by side for the
// eight of a tile: they go through LDS, so that neighbouring lanes store
// neighbouring tokens'.
template <int DP, int DT>
__global__ void __launch_bounds__(256) append_kernel(VecArgs a)
{
    using M = Map<DP>;
    __shared__ uint16_t unit[M::kTokens][DP / 4];
    const int lane = threadIdx.x % M::kLanes, vec = threadIdx.x / M::kLanes;
    const bool is_v = vec >= M::kTokens;
    const int head = blockIdx.x % a.c.heads;
    const int64_t tok0 = (int64_t)(blockIdx.x / a.c.heads) * M::kTokens, tok = tok0 + vec % M::kTokens;
    const int P = 1 << a.c.shift;
    // the head's block of a slot's page, nullptr for a slot outside the cache
    auto block_of = [&](int slot) -> uint8_t * {
        const int page = slot >> a.c.shift;
        return slot < 0 || page >= a.c.pages
                   ? nullptr
                   : a.c.data + (size_t)page * a.c.page_bytes + (size_t)head * a.c.head_bytes;
    };
    // the token whose V unit this thread stores in the end
    constexpr int kSide = M::kTokens < 8 ? M::kTokens : 8;
    const int my = threadIdx.x % kSide + threadIdx.x / (kSide * DP / 4) * kSide, my_unit = threadIdx.x / kSide % (DP / 4);
    const int my_slot = tok0 + my < a.tokens ? a.slots[tok0 + my] : -1;
    const int slot = tok < a.tokens ? a.slots[tok] : -1;
    uint8_t *const base = block_of(slot);
    // a skipped token's rows may not exist: nothing is loaded before its slot is known
    const int ch = lane * 8;
    float x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (base && ch < a.c.dim) {
        const int64_t off = tok * (is_v ? a.v_ld : a.k_ld) + head * a.c.dim + ch;
        constexpr int size = DT == QNN_UINT8 || DT == QNN_INT8 ? 1 : 2;
        load8<DT>((const uint8_t *)(is_v ? a.v : a.k) + off * size, is_v ? a.vs : a.ks, is_v ? a.vz : a.kz, x);
    }
    if (base) {   // a whole group: the shuffles below stay inside one
        const int at = slot & (P - 1);
        constexpr bool kHalf = DT == QNN_FLOAT16, kReal = kHalf || DT == QNN_BFLOAT16;
        constexpr float kMost = 0x1p126f;
        if constexpr (kReal) {
            float sum = 0.0f;   // NaN, or beyond kMost, where any of the eight is
#pragma unroll
            for (int i = 0; i < 8; ++i)
                sum += __builtin_fabsf(x[i]);
            if (!(sum <= kMost)) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    x[i] = x[i] == x[i] ? __builtin_amdgcn_fmed3f(x[i], -kMost, kMost) : 0.0f;
            }
        } else if ((is_v ? a.vs : a.ks) > kMost / 256.0f) {   // of 255 steps at most
#pragma unroll
            for (int i = 0; i < 8; ++i)
                x[i] = __builtin_amdgcn_fmed3f(x[i], -kMost, kMost);
        }
        float lo = 0.0f, hi = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            lo = fminf(lo, x[i]);
            hi = fmaxf(hi, x[i]);
        }
        // Over the group: neighbours, pairs, then mirrored eights and sixteens. -lo and
        // hi are +0 or more, so their bits compare as integers, one instruction a step
        // (as floats, three).
        uint32_t down = as_bits(0.0f - lo), up = as_bits(hi + 0.0f);
        down = max(down, lane_move<0xb1>(down));
        up = max(up, lane_move<0xb1>(up));
        down = max(down, lane_move<0x4e>(down));
        up = max(up, lane_move<0x4e>(up));
        down = max(down, lane_move<0x141>(down));
        up = max(up, lane_move<0x141>(up));
        if constexpr (M::kLanes >= 16) {
            down = max(down, lane_move<0x140>(down));
            up = max(up, lane_move<0x140>(up));
        }
        if constexpr (M::kLanes >= 32) {
            down = max(down, (uint32_t)__shfl_xor((int)down, 16));
            up = max(up, (uint32_t)__shfl_xor((int)up, 16));
        }
        float below = __builtin_bit_cast(float, down);
        const float range = __builtin_bit_cast(float, up) + below;
        float step;
        if constexpr (kHalf) {   // 0, or 2^-24 and more: the remainder is exact, the quotient the correctly rounded one
            const float q = range * (1.0f / 15.0f);
            step = __builtin_fmaf(__builtin_fmaf(-q, 15.0f, range), 1.0f / 15.0f, q);
        } else {
            step = range / 15.0f;
        }
        // the scale keeps 16 significant bits, rounded up so that 15 steps span the range
        const uint32_t sb = (as_bits(step) + 0xffu) & 0xffffff00u;
        float s = sb ? __builtin_bit_cast(float, sb) : 1.0f;
        if constexpr (!kHalf) {
            if (s < 0x1p-100f) {   // the reciprocal below would overflow; exact
                s *= 0x1p100f;
                below *= 0x1p100f;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    x[i] *= 0x1p100f;
            }
        }
        // x / s by a reciprocal within 2^-23 and one step on the remainder: that is
        // exact (16 bits of s, and q's error is 2^-22 of it), so the result is the
        // quotient, off by 2^-44, rounded once: exact where the quotient is a whole
        // number and a half. Other quotients (of a 16-bit x or of a product's 24 bits, and
        // 16 bits of s) are at least 2^-41 of themselves from where a rounding changes,
        // so the rounding is that of x / s (divisions took three times the
        // instructions, which bound the kernel).
        const float inv = __builtin_amdgcn_rcpf(s);
        auto steps = [&](float v) {
            const float q = v * inv;
            return __builtin_rintf(__builtin_fmaf(__builtin_fmaf(-q, s, v), inv, q));
        };
        const float z = fminf(steps(below), 15.0f);
        float c[8];   // the codes less z
#pragma unroll
        for (int i = 0; i < 8; ++i)
            c[i] = __builtin_amdgcn_fmed3f(steps(x[i]), -z, 15.0f - z);
        // four codes as the digits of a number to base 16, exact in f32
        auto four = [&](float c0, float c1, float c2, float c3) {
            const float high = __builtin_fmaf(c3, 16.0f, c2), low = __builtin_fmaf(c1, 16.0f, c0);
            return (uint32_t)__builtin_fmaf(high, 256.0f, __builtin_fmaf(z, 0x1111, low));
        };
        if (!is_v) {
            *(uint32_t *)(base + at * (DP / 2) + lane * 4) =
                four(c[0], c[2], c[4], c[6]) | four(c[1], c[3], c[5], c[7]) << 16;
        } else {
#pragma unroll
            for (int u = 0; u < 2; ++u)
                unit[vec - M::kTokens][lane * 2 + u] =
                    (uint16_t)four(c[4 * u], c[4 * u + 1], c[4 * u + 2], c[4 * u + 3]);
        }
        if (lane == 0)
            *(uint32_t *)(base + P * DP + (is_v ? 4 * P : 0) + at * 4) = sb | (uint32_t)z;
    }
    __syncthreads();
    if (uint8_t *const mine = block_of(my_slot)) {
        const int at = my_slot & (P - 1);
        *(uint16_t *)(mine + P * (DP / 2) + (at >> 3) * (4 * DP) + my_unit * 16 + (at & 7) * 2) = unit[my][my_unit];
    }
}

template <int DP, int DT>
__global__ void __launch_bounds__(256) read_kernel(VecArgs a)
{
    using M = Map<DP>;
    const int lane = threadIdx.x % M::kLanes, vec = threadIdx.x / M::kLanes;
    const bool is_v = vec >= M::kTokens;
    const int head = blockIdx.x % a.c.heads;
    const int64_t tok = (int64_t)(blockIdx.x / a.c.heads) * M::kTokens + vec % M::kTokens;
    const int ch = lane * 8;
    void *const out = is_v ? a.vo : a.ko;
    if (tok >= a.tokens || ch >= a.c.dim || !out)
        return;
    const int slot = a.slots[tok];
    const int page = slot >> a.c.shift, at = slot & ((1 << a.c.shift) - 1);
    float x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (slot >= 0 && page < a.c.pages) {
        const uint8_t *base = a.c.data + (size_t)page * a.c.page_bytes + (size_t)head * a.c.head_bytes;
        const int P = 1 << a.c.shift;
        const uint32_t rec = *(const uint32_t *)(base + P * DP + (is_v ? 4 * P : 0) + at * 4);
        const float s = rec_scale(rec), z = rec_zero(rec);
        uint32_t c[8];
        if (!is_v) {
            const uint32_t w = *(const uint32_t *)(base + at * (DP / 2) + lane * 4);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                c[i] = w >> (i & 1 ? 16 + 2 * (i - 1) : 2 * i);
        } else {
            const uint8_t *tile = base + P * (DP / 2) + (at >> 3) * (4 * DP) + (at & 7) * 2;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                c[i] = (uint32_t)(*(const uint16_t *)(tile + (lane * 2 + (i >> 2)) * 16)) >> (4 * (i & 3));
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
            x[i] = s * ((float)(c[i] & 15u) - z);
    }
    const int64_t off = tok * (is_v ? a.v_ld : a.k_ld) + head * a.c.dim + ch;
    if constexpr (DT == QNN_FLOAT16) {
        h8 h;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            h[i] = (_Float16)x[i];
        *(h8 *)((uint8_t *)out + off * 2) = h;
    } else {
        u4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __bf16 p = (__bf16)x[2 * i], q = (__bf16)x[2 * i + 1];
            w[i] = (uint32_t)__builtin_bit_cast(uint16_t, p) | (uint32_t)__builtin_bit_cast(uint16_t, q) << 16;
        }
        *(u4 *)((uint8_t *)out + off * 2) = w;
    }
}

template <int DP>
int64_t vec_blocks(const VecArgs &a)
{
    return ((int64_t)a.tokens + Map<DP>::kTokens - 1) / Map<DP>::kTokens * a.c.heads;
}

template <int DP>
hipError_t launch_append(const VecArgs &a, int dt, hipStream_t st)
{
    const dim3 grid((unsigned)vec_blocks<DP>(a));
    switch (dt) {
    case QNN_UINT8: launch_main((append_kernel<DP, QNN_UINT8>), grid, dim3(256), 0, st, a); break;
    case QNN_INT8: launch_main((append_kernel<DP, QNN_INT8>), grid, dim3(256), 0, st, a); break;
    case QNN_FLOAT16: launch_main((append_kernel<DP, QNN_FLOAT16>), grid, dim3(256), 0, st, a); break;
    default: launch_main((append_kernel<DP, QNN_BFLOAT16>), grid, dim3(256), 0, st, a); break;
    }
    return hipGetLastError();
}

template <int DP>
hipError_t launch_read(const VecArgs &a, int dt, hipStream_t st)
{
    const dim3 grid((unsigned)vec_blocks<DP>(a));
    if (dt == QNN_FLOAT16)
        launch_main((read_kernel<DP, QNN_FLOAT16>), grid, dim3(256), 0, st, a);
    else
        launch_main((read_kernel<DP, QNN_BFLOAT16>), grid, dim3(256), 0, st, a);
    return hipGetLastError();
}

// The row strides and alignment of k or v.
qnn_status check_rows(const char *what, const void *p, int64_t ld, const Cache4Args &c, int size)
{
    if (ld < (int64_t)c.heads * c.dim)
        return fail(QNN_ERR_SHAPE, "%s: row stride %lld does not hold %d heads of %d", what, (long long)ld, c.heads,
                    c.dim);
    if (ld % 8 || ((uintptr_t)p & (8 * size - 1)))
        return fail(QNN_ERR_UNSUPPORTED, "%s: rows must be aligned to 8 elements", what);
    return QNN_OK;
}

// A launch takes fewer than 2^32 threads.
qnn_status check_grid(const char *what, int32_t tokens, const Cache4Args &c)
{
    const int per = 1024 / cache4_padded(c.dim);   // Map<DP>::kTokens
    if (((int64_t)tokens + per - 1) / per * c.heads >= (int64_t(1) << 32) / 256)
        return fail(QNN_ERR_UNSUPPORTED, "%s: too many vectors in one call", what);
    return QNN_OK;
}

}  // namespace

qnn_status check_cache4(const qnn_cache4 &c, const char *what, Cache4Args *out)
{
    if (qnn_cache4_page_bytes(c.page_size, c.heads, c.head_dim) == 0)
        return fail(QNN_ERR_SHAPE,
                    "%s: cache of page_size %d, %d heads of %d (page_size 16 to 256, a power of two; head_dim a "
                    "multiple of 8, 8 to 256)", what, c.page_size, c.heads, c.head_dim);
    if (c.pages < 1 || (int64_t)c.pages * c.page_size >= (int64_t(1) << 31))
        return fail(QNN_ERR_SHAPE, "%s: cache of %d pages of %d tokens", what, c.pages, c.page_size);
    if (!c.data)
        return fail(QNN_ERR_NULL, "%s: the cache's data is NULL", what);
    if ((uintptr_t)c.data & 15)
        return fail(QNN_ERR_UNSUPPORTED, "%s: the cache's data must be 16-byte aligned", what);
    Cache4Args a{};
    a.data = (uint8_t *)c.data;
    a.pages = c.pages;
    a.shift = __builtin_ctz((unsigned)c.page_size);
    a.heads = c.heads;
    a.dim = c.head_dim;
    a.head_bytes = (uint32_t)c.page_size * (cache4_padded(c.head_dim) + 8);
    a.page_bytes = (uint32_t)qnn_cache4_page_bytes(c.page_size, c.heads, c.head_dim);
    *out = a;
    return QNN_OK;
}

}  // namespace qnn

using namespace qnn;

extern "C" {

size_t qnn_cache4_page_bytes(int32_t page_size, int32_t heads, int32_t head_dim)
{
    if (page_size < 16 || page_size > 256 || (page_size & (page_size - 1)) || heads < 1 || heads > 4096 ||
        head_dim < 8 || head_dim > 256 || head_dim % 8)
        return 0;
    return (size_t)heads * page_size * (cache4_padded(head_dim) + 8);
}

qnn_status qnn_cache4_append(void *stream, qnn_cache4 cache, const void *k, const void *v, qnn_dtype dtype,
                             qnn_qparams k_q, qnn_qparams v_q, int32_t tokens, int64_t k_ld, int64_t v_ld,
                             const int32_t *slots)
{
    VecArgs a{};
    qnn_status s = check_cache4(cache, "cache4_append", &a.c);
    if (s != QNN_OK)
        return s;
    const bool whole = dtype == QNN_UINT8 || dtype == QNN_INT8;
    if (!whole && dtype != QNN_FLOAT16 && dtype != QNN_BFLOAT16)
        return fail(QNN_ERR_DTYPE, "cache4_append: k and v must be uint8, int8, float16 or bfloat16");
    if (tokens < 0)
        return fail(QNN_ERR_SHAPE, "cache4_append: tokens must be >= 0");
    if (whole) {
        if ((s = check_qparams(k_q, "k qparams", 1, dtype, false)) != QNN_OK ||
            (s = check_qparams(v_q, "v qparams", 1, dtype, false)) != QNN_OK)
            return s;
        a.ks = k_q.scale[0];
        a.kz = k_q.zero_point[0];
        a.vs = v_q.scale[0];
        a.vz = v_q.zero_point[0];
    }
    if (tokens == 0)
        return QNN_OK;
    if (!k || !v || !slots)
        return fail(QNN_ERR_NULL, "cache4_append: k, v or slots is NULL");
    const int size = whole ? 1 : 2;
    if ((s = check_rows("cache4_append: k", k, k_ld, a.c, size)) != QNN_OK ||
        (s = check_rows("cache4_append: v", v, v_ld, a.c, size)) != QNN_OK ||
        (s = check_grid("cache4_append", tokens, a.c)) != QNN_OK)
        return s;
    a.k = k;
    a.v = v;
    a.k_ld = k_ld;
    a.v_ld = v_ld;
    a.slots = slots;
    a.tokens = tokens;
    const int dp = cache4_padded(a.c.dim);
    const hipStream_t st = (hipStream_t)stream;
    const hipError_t e = dp == 64    ? launch_append<64>(a, dtype, st)
                         : dp == 128 ? launch_append<128>(a, dtype, st)
                                     : launch_append<256>(a, dtype, st);
    return e == hipSuccess ? QNN_OK : hip_fail(e, "cache4_append launch");
}

qnn_status qnn_cache4_read(void *stream, qnn_cache4 cache, const int32_t *slots, int32_t tokens, void *k, void *v,
                           qnn_dtype dtype, int64_t k_ld, int64_t v_ld)
{
    VecArgs a{};
    qnn_status s = check_cache4(cache, "cache4_read", &a.c);
    if (s != QNN_OK)
        return s;
    if (dtype != QNN_FLOAT16 && dtype != QNN_BFLOAT16)
        return fail(QNN_ERR_DTYPE, "cache4_read: k and v must be float16 or bfloat16");
    if (tokens < 0)
        return fail(QNN_ERR_SHAPE, "cache4_read: tokens must be >= 0");
    if (tokens == 0 || (!k && !v))
        return QNN_OK;
    if (!slots)
        return fail(QNN_ERR_NULL, "cache4_read: slots is NULL");
    if ((k && (s = check_rows("cache4_read: k", k, k_ld, a.c, 2)) != QNN_OK) ||
        (v && (s = check_rows("cache4_read: v", v, v_ld, a.c, 2)) != QNN_OK) ||
        (s = check_grid("cache4_read", tokens, a.c)) != QNN_OK)
        return s;
    a.ko = k;
    a.vo = v;
    a.k_ld = k_ld;
    a.v_ld = v_ld;
    a.slots = slots;
    a.tokens = tokens;
    const int dp = cache4_padded(a.c.dim);
    const hipStream_t st = (hipStream_t)stream;
    const hipError_t e = dp == 64    ? launch_read<64>(a, dtype, st)
                         : dp == 128 ? launch_read<128>(a, dtype, st)
                                     : launch_read<256>(a, dtype, st);
    return e == hipSuccess ? QNN_OK : hip_fail(e, "cache4_read launch");
}

}  // extern "C"
