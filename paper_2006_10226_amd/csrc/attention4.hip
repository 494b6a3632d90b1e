// Attention over the 4-bit cache (qnn_attention4; the cache's layout is in
// include/qnn.h).
//
// Mathematics.  K_t = s_t (c_t - z_t) and V_t = s'_t (c'_t - z'_t), so with
// y_t = scale log2(e) q . K_t
//   q . K_t = s_t (sum_d q_d c_td - z_t sum_d q_d)
//   o_d = (sum_t w_t c'_td - sum_t w_t z'_t) / sum_t p_t,
//         p_t = 2^(y_t - u), w_t = p_t s'_t
// for any u (the terms of Eq. (3): codes multiplied as they are, the zero
// points' parts taken off). Both products run on the f16 matrix cores, which
// take the codes without any conversion: a code c in bits 0 .. 3 of an f16 is
// the subnormal c * 2^-24, and at bits 4 .. 7 it is c * 2^-20. Eight codes cost
// seven instructions. The cores cut each product some 27 bits below the
// largest that its operands' exponent fields allow (measured: sums of 32 codes
// by weights up to 1 are off by up to 2^-12 with codes at bit 0, 2^-16.2 at bit
// 4, 2^-16.6 with codes as ordinary f16 numbers), so bits 4 .. 7 it is: as
// exact as f32 sums.
//
// A wave holds 16 R query rows (a request's queries times the heads that share
// a cache head) and walks the tokens 32 at a time:
//   scores^T [token][row] = K q^T: a lane then has eight neighbouring tokens of
//   one row, which is exactly the operand that
//   o^T [channel][row] += V^T p^T wants: the weights never leave the lane.
// The running offset u of a row is raised only when a weight would leave
// f16's or a sum f32's comfortable range (w > 2^15 or sum p > 2^98), and then
// so that the largest weight is 2^7: f16 holds weights down to 2^-31 of it, so
// that a token which outweighs a long tail takes little of the tail's sum. The
// output is linear in the weights, so any u gives the same quotient.
//
// The four waves of a workgroup take every fourth 32 tokens and are joined
// through LDS. Where few rows meet a long cache, its tokens are split over
// workgroups, whose sums (unscaled, with their offsets) a second kernel joins.
//
// What bounds it: single tokens read each code once, (DP + 8) bytes for a token's K
// and V of a head; a step of 32 tokens is about 250 vector instructions for one row
// block, just under the memory's rate (four requests of 131072 tokens, 8 heads of
// 128: 107 us, 5.3 TB/s). Prompts hold two row blocks a wave, which share the
// unpacking (112 of 350 instructions), and are bound by vector instructions, which
// issue in three quarters of the cycles (2048 queries on 4096 tokens, 32 heads of
// 128, causal: 182 us, 570 TFLOP/s, matrix cores 25% busy, once the clocks have
// settled after some 200 calls; 200 to 214 before). A short cache is neither: eight
// workgroups' chain of loads and eight steps (one request of 1000 tokens 11.6 us).
#include "cache4.h"

#include <algorithm>
#include <cmath>

namespace qnn {
namespace {

typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));

struct AttnArgs {
    Cache4Args c;
    const void *q;
    void *o;
    const int32_t *table, *ctx, *cu;
    int64_t q_ld, o_ld, table_ld;
    int32_t q_dt, o_dt;
    int32_t tokens, requests, q_heads, group;   // group: query heads of a cache head
    int32_t width, max_q, causal, window;
    int32_t tiles;          // row tiles of a request and cache head
    // a long cache in parts of `chunk` tokens, each a workgroup's: their sums
    // [part][query row][DP] and (offset, sum p) [part][query row], row = token *
    // q_heads + head, which a second kernel joins (parts == 1: neither)
    int32_t parts, chunk;
    float *part_o;
    float2 *part_p;
    int32_t stripes, unit_tiles;   // shares of a head's row tiles, and the tiles of one (tiles > 1)
    int32_t grid;
    float scale;            // scale * log2(e), times the query's own scale
    int32_t q_zp;
    float o_scale;
    int32_t o_zp, o_lo, o_hi;
};

constexpr int kWaves = 4;
constexpr uint32_t kCode = 0x00f000f0u;   // a code at bits 4 .. 7 of each half: c * 2^-20
constexpr float kNone = -0x1.fffffep127f;   // offset of a row without tokens yet: no score is below
constexpr float kMaxWeight = 0x1p15f, kMaxSum = 0x1p98f;
constexpr float kFar = 0x1p14f;      // offsets beyond it are rounded by up to 2^-10 and more

// Tokens [lo, hi) that rows first .. last - 1 of a request see between them; a
// row is a query (row / group) and one of the heads.
struct Span {
    int lo, hi;
};
__device__ __forceinline__ Span seen(const AttnArgs &a, int ctx, int nq, int query_first, int query_last)
{
    const int held = min(ctx, a.width << a.c.shift);
    const int p0 = ctx - nq + query_first, p1 = ctx - nq + query_last;   // positions
    Span s;
    s.hi = a.causal ? min(held, p1 + 1) : held;
    s.lo = a.window > 0 && p0 >= a.window ? p0 - a.window + 1 : 0;
    return s;
}

// The part of a span that workgroup `part` takes: whole steps of 32 tokens, the
// last part to the end whatever the host took for the longest.
__device__ __forceinline__ Span part_of(const AttnArgs &a, Span s, int part)
{
    const int64_t from = (s.lo & ~31) + (int64_t)part * a.chunk;
    if (part < a.parts - 1)
        s.hi = (int)min((int64_t)s.hi, from + a.chunk);
    if (part > 0)
        s.lo = (int)min(from, (int64_t)INT32_MAX);
    return s;
}

// A request's first query row, and its number of queries (of which the first
// max_q are computed).
__device__ __forceinline__ int queries(const AttnArgs &a, int b, int *nq)
{
    if (!a.cu) {
        *nq = 1;
        return b;
    }
    const int first = min(max(a.cu[b], 0), a.tokens);
    *nq = max(min(a.cu[b + 1], a.tokens) - first, 0);
    return first;
}

// max over the four lanes that hold a row's tokens
__device__ __forceinline__ float row_max(float v)
{
    v = fmaxf(v, __shfl_xor(v, 16));
    return fmaxf(v, __shfl_xor(v, 32));
}
__device__ __forceinline__ float row_sum(float v)
{
    v += __shfl_xor(v, 16);
    return v + __shfl_xor(v, 32);
}

__device__ __forceinline__ float as_float(uint32_t v) { return __builtin_bit_cast(float, v); }

// Eight query values of element type dt from their bytes (8-bit ones in the
// first two words).
__device__ __forceinline__ void unpack_q8(u4 w, int dt, int zp, float (&x)[8])
{
    if (dt == QNN_FLOAT16) {
        const h8 h = __builtin_bit_cast(h8, w);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            x[i] = (float)h[i];
    } else if (dt == QNN_BFLOAT16) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            x[i] = __builtin_bit_cast(float, i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t b = (w[i >> 2] >> (8 * (i & 3))) & 0xffu;
            x[i] = (float)((dt == QNN_INT8 ? (int)(int8_t)b : (int)b) - zp);
        }
    }
}

// Stores N = 4, 8 or 16 neighbouring output values at element offset `at`.
template <int N>
__device__ __forceinline__ void store_out(const AttnArgs &a, int64_t at, const float (&v)[N])
{
    if (a.o_dt == QNN_FLOAT16 || a.o_dt == QNN_BFLOAT16) {
        uint32_t w[N / 2];
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            if (a.o_dt == QNN_FLOAT16)
                w[i] = __builtin_bit_cast(uint32_t, h2{(_Float16)v[2 * i], (_Float16)v[2 * i + 1]});
            else
                w[i] = (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v[2 * i]) |
                       (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v[2 * i + 1]) << 16;
        }
        uint32_t *p = (uint32_t *)((uint8_t *)a.o + at * 2);
#pragma unroll
        for (int i = 0; i < N / 2; i += 2)
            *(u2 *)(p + i) = u2{w[i], w[i + 1]};
    } else {
        uint32_t w[N / 4];
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            w[i] = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                // beyond the clamp before the integer conversion; NaN gives the zero point
                const float t = fminf(fmaxf(__builtin_rintf(v[4 * i + e] / a.o_scale), -1024.0f), 1024.0f);
                const int code = v[4 * i + e] == v[4 * i + e] ? (int)t + a.o_zp : a.o_zp;
                w[i] |= ((uint32_t)min(max(code, a.o_lo), a.o_hi) & 0xffu) << (8 * e);
            }
        }
        uint32_t *p = (uint32_t *)((uint8_t *)a.o + at);
#pragma unroll
        for (int i = 0; i < N / 4; ++i)
            p[i] = w[i];
    }
}

// Waves per SIMD that the registers are held to: those that the kernel nearly
// fits by itself (DP 128, one row block: 3 waves 113 us, 2 waves 119 us for four
// requests of 131072 tokens).
template <int DP, int R>
constexpr int wave_target()
{
    return R == 1 ? (DP == 64 ? 4 : DP == 128 ? 3 : 2) : (DP == 256 ? 1 : 2);
}

// FINE: the weights enter the matrix cores as two f16, their rounding and the
// rest. 16-bit outputs are rounded as coarsely as one f16; of 8-bit ones about
// one in 100 would fall on the other side of a step.
template <int DP, int R, bool FINE>
__global__ void __launch_bounds__(kWaves * 64, (wave_target<DP, R>())) attention4_kernel(AttnArgs a)
{
    constexpr int KS = DP / 32;    // K-steps of a score; words of K of a lane and token
    constexpr int NV = DP / 16;    // 16-channel blocks of the output
    constexpr int NW = DP / 64;    // 16-byte pieces of V of a lane (eight tokens, four channels each)
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 15, g = lane >> 4;

    int tile = 0, part, kvh, b;
    if (a.tiles == 1) {
        // nothing is shared: the first parts of every request, then the second ones
        // (of the longer requests only), ..., dealt to the XCDs in turn
        kvh = blockIdx.x % a.c.heads;
        const int rest = blockIdx.x / a.c.heads;
        b = rest % a.requests;
        part = rest / a.requests;
        if (part >= a.parts)
            return;
    } else {
        // row tiles of one cache head read the same tokens: they follow each other on
        // one XCD, or, where the heads don't fill the XCDs evenly, are dealt to
        // `stripes` of them; the longest (causal) first
        const int unit = (int)(blockIdx.x & 7) + 8 * (int)(blockIdx.x / (8u * a.unit_tiles * a.parts));
        const int rest = (int)(blockIdx.x / 8u % ((unsigned)a.unit_tiles * a.parts));
        tile = unit % a.stripes + a.stripes * (a.unit_tiles - 1 - rest / a.parts);
        part = rest % a.parts;
        kvh = unit / a.stripes % a.c.heads;
        b = unit / a.stripes / a.c.heads;
        if (tile >= a.tiles || b >= a.requests)
            return;
    }
    const int ctx = max(a.ctx[b], 0);
    int nq;
    const int first = queries(a, b, &nq);
    const int rows = min(nq, a.max_q) * a.group, row0 = tile * 16 * R;
    if (row0 >= rows)
        return;
    const Span span = part_of(a, seen(a, ctx, nq, row0 / a.group, (min(row0 + 16 * R, rows) - 1) / a.group), part);
    if (part > 0 && span.lo >= span.hi)
        return;

    // ---- queries, as the second operand: lane (n, g) holds channels 8 (g KS +
    // k) .. + 7 of row n for step k. Their loads are issued here, in one go, and
    // used once the first step's are on their way too: a workgroup's few dependent
    // memory latencies are what a short part costs.
    u4 raw[R][KS];
    int lo_row[R], hi_row[R];
    const bool wide = a.q_dt == QNN_FLOAT16 || a.q_dt == QNN_BFLOAT16;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int row = min(row0 + r * 16 + n, rows - 1);
        const int i = row / a.group, h = row - i * a.group;
        const Span own = seen(a, ctx, nq, i, i);
        lo_row[r] = own.lo;
        hi_row[r] = own.hi;
        const uint8_t *p = (const uint8_t *)a.q + ((int64_t)(first + i) * a.q_ld + (int64_t)(kvh * a.group + h) * a.c.dim)
                                                      * (wide ? 2 : 1);
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            const int ch = 8 * (g * KS + k), at = ch < a.c.dim ? ch : 0;
            if (wide) {
                raw[r][k] = *(const u4 *)(p + at * 2);
            } else {
                const u2 w = *(const u2 *)(p + at);
                raw[r][k] = u4{w[0], w[1], 0, 0};
            }
        }
    }

    const int P = 1 << a.c.shift;
    const int32_t *const table = a.table + b * a.table_ld;
    // What a step reads. Lane (n, g): K of tokens 8 (n / 4) + n % 4 (+ 4), words g
    // KS on; V and records of tokens 8 g .. + 7, V's unit n. A step is two halves of
    // 16 tokens, each in one page: their addresses are scalars, which a lane picks
    // from and adds an offset of its own to.
    struct Step {
        uint32_t k[2][KS];
        u4 v[NW];
        u4 rk[2], rv[2];
        bool bad;   // some page is none (uniform), the lane's own
        bool mine;
    };
    struct Pages {
        int p[2];
    };
    const uint32_t off_k = ((n >> 2 & 1) * 8 + (n & 3)) * (DP / 2) + g * KS * 4;
    const uint32_t off_v = (g & 1) * (4 * DP) + n * NW * 16, off_r = (g & 1) * 32;
    // pages of the halves (past the last token: the last one's)
    auto pages = [&](int t0) __attribute__((always_inline)) {
        return Pages{{table[min(t0, span.hi - 1) >> a.c.shift], table[min(t0 + 16, span.hi - 1) >> a.c.shift]}};
    };
    auto fetch = [&](Step &d, int t0, Pages pg) __attribute__((always_inline)) {
        const uint8_t *half[2];
        bool ok[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            ok[h] = (unsigned)pg.p[h] < (unsigned)a.c.pages;
            half[h] = a.c.data + (size_t)kvh * a.c.head_bytes + (size_t)(ok[h] ? pg.p[h] : 0) * a.c.page_bytes;
        }
        d.bad = !(ok[0] && ok[1]);
        d.mine = g < 2 ? ok[0] : ok[1];
        const int in0 = t0 & (P - 1), in1 = (t0 + 16) & (P - 1);   // multiples of 16
        const uint8_t *const kp = (n < 8 ? half[0] + in0 * (DP / 2) : half[1] + in1 * (DP / 2)) + off_k;
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int k = 0; k < KS; ++k)
                d.k[s][k] = ((const uint32_t *)(kp + s * 4 * (DP / 2)))[k];
        const uint8_t *const vp =
            (g < 2 ? half[0] + (P + in0) * (DP / 2) : half[1] + (P + in1) * (DP / 2)) + off_v;
#pragma unroll
        for (int j = 0; j < NW; ++j)
            d.v[j] = ((const u4 *)vp)[j];
        const uint8_t *const rp = (g < 2 ? half[0] + P * DP + in0 * 4 : half[1] + P * DP + in1 * 4) + off_r;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            d.rk[j] = ((const u4 *)rp)[j];
            d.rv[j] = ((const u4 *)(rp + 4 * P))[j];
        }
    };
    // tokens that every row of the tile sees
    const int all_lo = seen(a, ctx, nq, (min(row0 + 16 * R, rows) - 1) / a.group, (min(row0 + 16 * R, rows) - 1) / a.group).lo;
    const int all_hi = min(span.hi, seen(a, ctx, nq, row0 / a.group, row0 / a.group).hi);
    constexpr int kNext = kWaves * 32;
    int t0 = (span.lo & ~31) + wave * 32;
    Step d0;
    Pages pg{{-1, -1}};
    if (t0 < span.hi) {
        fetch(d0, t0, pages(t0));
        pg = pages(t0 + kNext);
    }

    u4 q[R][KS];
    float qsum[R], fac[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const bool live = row0 + r * 16 + n < rows;
        float x[KS][8], most = 0.0f;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            unpack_q8(raw[r][k], a.q_dt, a.q_zp, x[k]);
            const bool held = live && 8 * (g * KS + k) < a.c.dim;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                x[k][e] = held ? x[k][e] : 0.0f;
                most = fmaxf(most, fabsf(x[k][e]));
            }
        }
        most = row_max(most);
        // a power of two brings the row's largest to 2^14 .. 2^15: exact for 8-bit
        // and f16 values, and values of any exponent fit f16
        const int ex = (int)(__builtin_bit_cast(uint32_t, most) >> 23);   // 255: not finite, stays as it is
        const float up = ex == 255 ? 1.0f : __builtin_bit_cast(float, (uint32_t)min(127 + 14 + 127 - ex, 253) << 23);
        const float sgn = a.scale < 0.0f ? -up : up;
        float sum = 0.0f;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            h8 h8v;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                h8v[e] = (_Float16)(x[k][e] * sgn);
                sum += (float)h8v[e];
            }
            q[r][k] = __builtin_bit_cast(u4, h8v);
        }
        qsum[r] = row_sum(sum) * 0x1p-20f;
        // above 0, so that a masked score (-inf) stays one, and finite, so that a score
        // of 0 does: the largest f32 stands for what a row of 2^121 and more (scale
        // included) would have
        fac[r] = fminf(fmaxf(fabsf(a.scale) * 0x1p20f / up, 0x1p-126f), 0x1.fffffep127f);
    }

    f4 acc[R][NV], zacc[R];
    float off[R], total[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
#pragma unroll
        for (int j = 0; j < NV; ++j)
            acc[r][j] = f4{0, 0, 0, 0};
        zacc[r] = f4{0, 0, 0, 0};
        off[r] = kNone;
        total[r] = 0.0f;
    }

    auto step = [&](const Step &d, int t0) __attribute__((always_inline)) {
        const int tv = t0 + g * 8;
        // ---- scores: sc[r][j] of token tv + j
        f4 sc[R][2];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
#pragma unroll
            for (int r = 0; r < R; ++r)
                sc[r][s] = f4{0, 0, 0, 0};
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                const uint32_t w = d.k[s][k];
                const u4 c = u4{w << 4 & kCode, w & kCode, w >> 4 & kCode, w >> 8 & kCode};
#pragma unroll
                for (int r = 0; r < R; ++r)
                    sc[r][s] = __builtin_amdgcn_mfma_f32_16x16x32_f16(
                        __builtin_bit_cast(h8, c), __builtin_bit_cast(h8, q[r][k]), sc[r][s], 0, 0, 0);
            }
        }
        float vs[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            // V's scale with the zero point in its lowest bits: 2^-19 of it at most, far
            // below the weight's own rounding to f16
            vs[j] = as_float(d.rv[j >> 2][j & 3]);
            const float ks = rec_scale(d.rk[j >> 2][j & 3]), kz = rec_zero(d.rk[j >> 2][j & 3]);
#pragma unroll
            for (int r = 0; r < R; ++r)
                sc[r][j >> 2][j & 3] = __builtin_fmaf(-kz, qsum[r], sc[r][j >> 2][j & 3]) * ks;
        }
        if (d.bad || t0 < all_lo || t0 + 32 > all_hi) {
            // some row doesn't see some token; one that no row sees, or of no page,
            // may hold anything
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const bool held = tv + j >= span.lo && tv + j < span.hi && d.mine;
                vs[j] = held ? vs[j] : 0.0f;
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const bool sees = held && tv + j >= lo_row[r] && tv + j < hi_row[r];
                    sc[r][j >> 2][j & 3] = sees ? sc[r][j >> 2][j & 3] : -INFINITY;
                }
            }
        }
        u4 pw[R], pl[FINE ? R : 1];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float w[8], sum = 0.0f, top = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[r][j >> 2][j & 3], fac[r], -off[r]));
                w[j] = p * vs[j];
                sum += p;
                top = fmaxf(top, w[j]);
            }
            if (__any(top > kMaxWeight || sum > kMaxSum || fabsf(off[r]) > kFar)) {
                // raise the offset: the largest weight becomes 2^7 (or, where V's scales
                // are below 2^-83, the largest p 2^90). The scores are rounded before the
                // offset, a rounded one, is taken off: the unrounded one above may differ
                // from it by half a step, which beside 2^27 is 2^3.
#pragma clang fp contract(off)
                float most = kNone;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float x = sc[r][j >> 2][j & 3] * fac[r];
                    most = fmaxf(most, fmaxf(x + (__builtin_amdgcn_logf(vs[j]) - 7.0f), x - 90.0f));
                }
                most = fmaxf(row_max(most), off[r]);
                const float down = __builtin_amdgcn_exp2f(off[r] - most);
                off[r] = most;
                total[r] *= down;
                zacc[r] *= down;
#pragma unroll
                for (int j = 0; j < NV; ++j)
                    acc[r][j] *= down;
                sum = 0.0f;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float p = __builtin_amdgcn_exp2f(sc[r][j >> 2][j & 3] * fac[r] - most);
                    w[j] = p * vs[j];
                    sum += p;
                }
            }
            total[r] += sum;
            h8 h;
#pragma unroll
            for (int j = 0; j < 8; ++j)
                h[j] = (_Float16)w[j];   // rounded to nearest: 2^-11 of each weight, or 2^-25, at most
            pw[r] = __builtin_bit_cast(u4, h);
            if constexpr (FINE) {
                h8 l;
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    l[j] = (_Float16)(w[j] - (float)h[j]);
                pl[r] = __builtin_bit_cast(u4, l);
            }
        }
        // ---- output: V's pieces hold pairs of tokens of four channels
#pragma unroll
        for (int v = 0; v < NW; ++v) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                u4 c;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    c[e] = (i == 0 ? d.v[v][e] << 4 : d.v[v][e] >> (4 * i - 4)) & kCode;
#pragma unroll
                for (int r = 0; r < R; ++r)
                    acc[r][v * 4 + i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(
                        __builtin_bit_cast(h8, c), __builtin_bit_cast(h8, pw[r]), acc[r][v * 4 + i], 0, 0, 0);
                if constexpr (FINE) {
#pragma unroll
                    for (int r = 0; r < R; ++r)
                        acc[r][v * 4 + i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(
                            __builtin_bit_cast(h8, c), __builtin_bit_cast(h8, pl[r]), acc[r][v * 4 + i], 0, 0, 0);
                }
            }
        }
        // sum w z by the same cores, every row of the operand z
        u4 z;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            z[e] = __builtin_amdgcn_perm(d.rv[e >> 1][2 * (e & 1) + 1], d.rv[e >> 1][2 * (e & 1)], 0x0c040c00u) << 4;   // low bytes
#pragma unroll
        for (int r = 0; r < R; ++r) {
            zacc[r] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, z), __builtin_bit_cast(h8, pw[r]),
                                                             zacc[r], 0, 0, 0);
            if constexpr (FINE)
                zacc[r] = __builtin_amdgcn_mfma_f32_16x16x32_f16(
                    __builtin_bit_cast(h8, z), __builtin_bit_cast(h8, pl[r]), zacc[r], 0, 0, 0);
        }
    };
    constexpr bool kTwo = R == 1 || DP <= 128;   // registers for two steps
    if (kTwo && t0 < span.hi) {
        // two steps in registers: one is fetched, its pages' numbers a step earlier
        // still, while the other is computed
        Step d1;
        while (true) {
            const bool second = t0 + kNext < span.hi;
            if (second) {
                fetch(d1, t0 + kNext, pg);
                pg = pages(t0 + 2 * kNext);
            }
            step(d0, t0);
            if (!second)
                break;
            t0 += kNext;
            const bool third = t0 + kNext < span.hi;
            if (third) {
                fetch(d0, t0 + kNext, pg);
                pg = pages(t0 + 2 * kNext);
            }
            step(d1, t0);
            if (!third)
                break;
            t0 += kNext;
        }
    }
    if (!kTwo && t0 < span.hi) {
        while (true) {
            step(d0, t0);
            t0 += kNext;
            if (t0 >= span.hi)
                break;
            fetch(d0, t0, pg);
            pg = pages(t0 + kNext);
        }
    }

    // ---- the waves' parts joined: common offset, sums through LDS
    __shared__ float offs[kWaves][R * 16];
    __shared__ float sums[2][R * (NV * 4 + 1)][64];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        total[r] = row_sum(total[r]);
        if (g == 0)
            offs[wave][r * 16 + n] = off[r];
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < R; ++r) {
        float most = kNone;
#pragma unroll
        for (int w = 0; w < kWaves; ++w)
            most = fmaxf(most, offs[w][r * 16 + n]);
        const float down = __builtin_amdgcn_exp2f(off[r] - most);
        off[r] = most;
        total[r] *= down;
#pragma unroll
        for (int j = 0; j < NV; ++j)
            acc[r][j] = (acc[r][j] - zacc[r]) * (down * 0x1p20f);
    }
    auto put = [&](int slot) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    sums[slot][r * (NV * 4 + 1) + j * 4 + e][lane] = acc[r][j][e];
            sums[slot][r * (NV * 4 + 1) + NV * 4][lane] = total[r];
        }
    };
    auto take = [&](int slot) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    acc[r][j][e] += sums[slot][r * (NV * 4 + 1) + j * 4 + e][lane];
            total[r] += sums[slot][r * (NV * 4 + 1) + NV * 4][lane];
        }
    };
    if (wave >= 2)
        put(wave - 2);
    __syncthreads();
    if (wave < 2)
        take(wave);
    __syncthreads();
    if (wave == 1)
        put(0);
    __syncthreads();
    if (wave != 0)
        return;
    take(0);

    // ---- lane (n, g) has channels (4 g + e) NV + j of row n
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int row = row0 + r * 16 + n;
        if (row >= rows)
            continue;
        const int i = row / a.group, h = row - i * a.group;
        if (a.parts > 1) {
            const size_t at = (size_t)part * a.tokens * a.q_heads + (size_t)(first + i) * a.q_heads +
                              (kvh * a.group + h);
            float *const p = a.part_o + at * DP;
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int j = 0; j < NV; j += 4)
                    *(f4 *)(p + (g * 4 + e) * NV + j) =
                        f4{acc[r][j][e], acc[r][j + 1][e], acc[r][j + 2][e], acc[r][j + 3][e]};
            if (g == 0)
                a.part_p[at] = float2{off[r], total[r]};
            continue;
        }
        const int64_t at = (int64_t)(first + i) * a.o_ld + (int64_t)(kvh * a.group + h) * a.c.dim;
        const float inv = total[r] == 0.0f ? 0.0f : 1.0f / total[r];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int ch = (g * 4 + e) * NV;
            if constexpr (NV == 16) {
                float v[8];
#pragma unroll
                for (int half = 0; half < 2; ++half) {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        v[j] = acc[r][half * 8 + j][e] * inv;
                    if (ch + half * 8 < a.c.dim)
                        store_out(a, at + ch + half * 8, v);
                }
            } else {
                float v[NV];
#pragma unroll
                for (int j = 0; j < NV; ++j)
                    v[j] = acc[r][j][e] * inv;
                if (ch < a.c.dim)
                    store_out(a, at + ch, v);
            }
        }
    }
}

// Joins the parts of every query row: DP / 4 lanes hold its channels, and `crews`
// (a power of two, up to 1024 / DP) of such lanes share the parts, whose sums meet
// in LDS: with one crew, 64 parts were 128 dependent memory latencies.
template <int DP>
__global__ void __launch_bounds__(256) join_kernel(AttnArgs a, int blocks, int crews)
{
    constexpr int kLanes = DP / 4;
    __shared__ f4 sums[256];
    __shared__ float sum_p[256 / kLanes];
    const int lane = threadIdx.x % kLanes, crew = threadIdx.x / kLanes % crews;
    const int64_t at = ((int64_t)blockIdx.x * 256 + threadIdx.x) / (kLanes * crews);   // (request, query, head)
    const int head = (int)(at % a.q_heads);
    const int64_t bi = at / a.q_heads;
    const int b = (int)(bi / a.max_q), i = (int)(bi % a.max_q);
    int nq = 0, first = 0;
    if (b < a.requests)
        first = queries(a, b, &nq);
    const bool live = i < nq;
    const size_t row = (size_t)(first + i) * a.q_heads + head, rows = (size_t)a.tokens * a.q_heads;
    f4 o = f4{0, 0, 0, 0};
    float total = 0.0f, most = kNone;
    int parts = 0;
    if (live) {
        // the parts that its tile's workgroups wrote
        const int row0 = (i * a.group + head % a.group) / (16 * blocks) * (16 * blocks);
        const Span span = seen(a, max(a.ctx[b], 0), nq, row0 / a.group,
                               (min(row0 + 16 * blocks, min(nq, a.max_q) * a.group) - 1) / a.group);
        parts = span.lo < span.hi
                    ? (int)min((int64_t)a.parts, ((int64_t)span.hi - (span.lo & ~31) + a.chunk - 1) / a.chunk)
                    : 1;
        // the offset of all parts, each lane looking at some (the row's lanes are in one
        // wave, or fill several that look at the same ones)
        for (int s = lane; s < parts; s += kLanes)
            most = fmaxf(most, a.part_p[s * rows + row].x);
    }
#pragma unroll
    for (int d = 1; d < kLanes; d <<= 1)
        most = fmaxf(most, __shfl_xor(most, d));
#pragma unroll 4
    for (int s = crew; s < parts; s += crews) {
        const float2 p = a.part_p[s * rows + row];
        const float down = __builtin_amdgcn_exp2f(p.x - most);
        o += *(const f4 *)(a.part_o + (s * rows + row) * DP + lane * 4) * down;
        total += p.y * down;
    }
    if (crews > 1) {
        sums[threadIdx.x] = o;
        if (lane == 0)
            sum_p[threadIdx.x / kLanes] = total;
        __syncthreads();
        if (crew == 0)
            for (int c = 1; c < crews; ++c) {
                o += sums[threadIdx.x + c * kLanes];
                total += sum_p[threadIdx.x / kLanes + c];
            }
    }
    if (!live || crew != 0 || lane * 4 >= a.c.dim)
        return;
    const float inv = total == 0.0f ? 0.0f : 1.0f / total;
    const float v[4] = {o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
    store_out(a, (int64_t)(first + i) * a.o_ld + (int64_t)head * a.c.dim + lane * 4, v);
}

// Least tokens of a part: below, the join's launch and latencies may cost more than
// the walk they save, above, more is walked in one part than a join takes. In us,
// single tokens, by least tokens:              192   384   768   1536
//   1 request of 1000, 8 x 4 heads of 128     10.4  12.0  11.6  11.6
//   1 of 1600                                 10.8  11.8  13.8  15.0
//   1 of 8000                                 11.4  12.4  14.8  18.2
//   1 of 16000                                14.8  13.0  15.5  19.7
//   8 of 1600                                 12.7  12.2  14.5  15.6
//   8 of 4000                                 19.0  16.3  17.4  22.8
//   48 of 1600, 12 x 1 heads of 64            25.2  25.2  23.7  21.5
//   48 of 4000                                39.0  38.8  38.7  39.5
// 768 is never the slowest; few requests would take 192 to 384.
constexpr int kLeastPart = 768;

struct Shape {
    int blocks;
    int64_t tiles;
    int parts, chunk;
};

// Grid of a call: parts of the cache where the row tiles alone would leave the
// device idle.
Shape shape_of(const qnn_attention_params &p, int group, int heads, int page_size, bool packed)
{
    Shape s;
    const int64_t max_q = packed ? p.max_q : 1;
    s.blocks = max_q * group <= 16 ? 1 : 2;
    s.tiles = (max_q * group + 16 * s.blocks - 1) / (16 * s.blocks);
    int64_t span = (int64_t)p.table_width * page_size;
    if (p.max_ctx > 0)
        span = std::min<int64_t>(span, p.max_ctx);
    if (p.window > 0)
        span = std::min<int64_t>(span, (int64_t)p.window + (16 * s.blocks + group - 1) / group + 32);
    const int64_t base = s.tiles * heads * std::max(p.requests, 1);
    const int64_t want = 8 * (int64_t)device_cus();
    int64_t parts = std::min<int64_t>((want + base - 1) / base, span / kLeastPart);
    parts = base >= want ? 1 : std::max<int64_t>(1, std::min<int64_t>(parts, 128));
    const int64_t chunk = ((span + parts - 1) / parts + 127) / 128 * 128;
    s.parts = (int)std::max<int64_t>(1, (span + chunk - 1) / chunk);
    s.chunk = (int)std::min<int64_t>(chunk, 1 << 30);
    return s;
}

// Whether 32 bits hold the rows of a call of at most max_q queries a request; the
// sums of shape_of and the join's row numbers rely on it.
bool countable(const qnn_attention_params &p, int64_t max_q)
{
    constexpr int64_t kMost = int64_t(1) << 31;
    return (int64_t)p.tokens * p.q_heads < kMost && max_q * p.q_heads < kMost &&
           max_q * p.q_heads * p.requests < kMost;
}

size_t parts_bytes(const Shape &s, const qnn_attention_params &p, int dp)
{
    return s.parts == 1 ? 0 : (size_t)s.parts * p.tokens * p.q_heads * (dp * sizeof(float) + sizeof(float2));
}

template <int DP>
hipError_t launch_attention(const AttnArgs &a, int blocks, hipStream_t st)
{
    const dim3 grid((unsigned)a.grid), block(kWaves * 64);
    const bool fine = a.o_dt == QNN_UINT8 || a.o_dt == QNN_INT8;
    if (blocks == 1 && fine)
        launch_main((attention4_kernel<DP, 1, true>), grid, block, 0, st, a);
    else if (blocks == 1)
        launch_main((attention4_kernel<DP, 1, false>), grid, block, 0, st, a);
    else if (fine)
        launch_main((attention4_kernel<DP, 2, true>), grid, block, 0, st, a);
    else
        launch_main((attention4_kernel<DP, 2, false>), grid, block, 0, st, a);
    if (a.parts > 1) {
        int crews = 1;
        while (crews < 1024 / DP && crews * 4 < a.parts)
            crews *= 2;
        const int64_t rows = (int64_t)a.requests * a.max_q * a.q_heads, per = 1024 / DP / crews;
        join_kernel<DP><<<dim3((unsigned)((rows + per - 1) / per)), dim3(256), 0, st>>>(a, blocks, crews);
    }
    return hipGetLastError();
}

}  // namespace
}  // namespace qnn

using namespace qnn;

extern "C" {

size_t qnn_attention4_workspace_size(qnn_cache4 cache, qnn_attention_params p)
{
    // sizes that qnn_attention4 refuses need none
    if (qnn_cache4_page_bytes(cache.page_size, cache.heads, cache.head_dim) == 0 || p.q_heads < cache.heads ||
        p.q_heads % cache.heads || p.tokens <= 0 || p.requests <= 0 || p.max_q < 1 || p.table_width < 1)
        return 0;
    // the same for calls with cu_q and without (one query each): the larger
    const int group = p.q_heads / cache.heads, dp = cache4_padded(cache.head_dim);
    size_t most = 0;
    for (const bool packed : {true, false})
        if (countable(p, packed ? p.max_q : 1))
            most = std::max(most, parts_bytes(shape_of(p, group, cache.heads, cache.page_size, packed), p, dp));
    return most;
}

qnn_status qnn_attention4(void *stream, const void *q, qnn_dtype q_dtype, qnn_qparams q_q, qnn_cache4 cache,
                          const int32_t *table, const int32_t *ctx, const int32_t *cu_q, qnn_attention_params p,
                          void *o, qnn_dtype o_dtype, qnn_qparams o_q, void *workspace, size_t workspace_bytes)
{
    AttnArgs a{};
    qnn_status s = check_cache4(cache, "attention4", &a.c);
    if (s != QNN_OK)
        return s;
    auto whole = [](qnn_dtype t) { return t == QNN_UINT8 || t == QNN_INT8; };
    auto known = [&](qnn_dtype t) { return whole(t) || t == QNN_FLOAT16 || t == QNN_BFLOAT16; };
    if (!known(q_dtype) || !known(o_dtype))
        return fail(QNN_ERR_DTYPE, "attention4: q and o must be uint8, int8, float16 or bfloat16");
    if (p.tokens < 0 || p.requests < 0 || p.q_heads < 1 || p.max_q < 1 || p.max_ctx < 0 || p.window < 0)
        return fail(QNN_ERR_SHAPE, "attention4: tokens %d, requests %d, q_heads %d, max_q %d, max_ctx %d, window %d",
                    p.tokens, p.requests, p.q_heads, p.max_q, p.max_ctx, p.window);
    if (p.q_heads % a.c.heads)
        return fail(QNN_ERR_SHAPE, "attention4: %d query heads over %d cache heads", p.q_heads, a.c.heads);
    if (p.table_width < 1 || p.table_ld < p.table_width || (int64_t)p.table_width * cache.page_size > (int64_t(1) << 30))
        return fail(QNN_ERR_SHAPE, "attention4: table_width %d, table_ld %lld", p.table_width, (long long)p.table_ld);
    const int64_t row = (int64_t)p.q_heads * a.c.dim;
    if (p.q_ld < row || p.o_ld < row)
        return fail(QNN_ERR_SHAPE, "attention4: row strides %lld and %lld do not hold %d heads of %d", (long long)p.q_ld,
                    (long long)p.o_ld, p.q_heads, a.c.dim);
    if (!cu_q && p.tokens != p.requests)
        return fail(QNN_ERR_SHAPE, "attention4: %d tokens of %d requests need cu_q", p.tokens, p.requests);
    if (!std::isfinite(p.scale))
        return fail(QNN_ERR_QPARAM, "attention4: scale is not finite");
    if (whole(q_dtype) && (s = check_qparams(q_q, "q qparams", 1, q_dtype, false)) != QNN_OK)
        return s;
    if (whole(o_dtype) && (s = check_qparams(o_q, "o qparams", 1, o_dtype, false)) != QNN_OK)
        return s;
    if (p.tokens == 0 || p.requests == 0)
        return QNN_OK;
    if (!q || !o || !table || !ctx)
        return fail(QNN_ERR_NULL, "attention4: q, o, table or ctx is NULL");
    const int q_size = whole(q_dtype) ? 1 : 2, o_size = whole(o_dtype) ? 1 : 2;
    if (p.q_ld % 8 || p.o_ld % 8 || ((uintptr_t)q & (8 * q_size - 1)) || ((uintptr_t)o & (8 * o_size - 1)))
        return fail(QNN_ERR_UNSUPPORTED, "attention4: rows of q and o must be aligned to 8 elements");
    if (!countable(p, cu_q ? p.max_q : 1))
        return fail(QNN_ERR_UNSUPPORTED, "attention4: too many row tiles");
    if (qnn_attention4_workspace_size(cache, p) > workspace_bytes)
        return fail(QNN_ERR_SHAPE, "attention4: the workspace is smaller than qnn_attention4_workspace_size()");
    a.q = q;
    a.o = o;
    a.table = table;
    a.ctx = ctx;
    a.cu = cu_q;
    a.q_ld = p.q_ld;
    a.o_ld = p.o_ld;
    a.table_ld = p.table_ld;
    a.q_dt = q_dtype;
    a.o_dt = o_dtype;
    a.tokens = p.tokens;
    a.requests = p.requests;
    a.q_heads = p.q_heads;
    a.group = p.q_heads / a.c.heads;
    a.width = p.table_width;
    a.max_q = cu_q ? p.max_q : 1;
    a.causal = p.causal != 0;
    a.window = p.window;
    a.scale = p.scale * 1.44269504088896340736f * (whole(q_dtype) ? q_q.scale[0] : 1.0f);
    if (!std::isfinite(a.scale))
        return fail(QNN_ERR_QPARAM, "attention4: scale times q's scale is not finite");
    a.q_zp = whole(q_dtype) ? q_q.zero_point[0] : 0;
    if (whole(o_dtype)) {
        Range r;
        dtype_range(o_dtype, &r);
        a.o_scale = o_q.scale[0];
        a.o_zp = o_q.zero_point[0];
        a.o_lo = (int32_t)r.lo;
        a.o_hi = (int32_t)r.hi;
    }
    const Shape g = shape_of(p, a.group, a.c.heads, cache.page_size, cu_q != nullptr);
    // heads of requests, dealt to eight XCDs
    const int64_t heads = (int64_t)a.c.heads * p.requests;
    a.stripes = g.tiles == 1 ? 1 : heads % 8 == 0 ? 1 : heads % 4 == 0 ? 2 : heads % 2 == 0 ? 4 : 8;
    const int64_t unit_tiles = (g.tiles + a.stripes - 1) / a.stripes;
    const int64_t grid = g.tiles == 1 ? heads * g.parts : (heads * a.stripes + 7) / 8 * 8 * unit_tiles * g.parts;
    // a launch takes fewer than 2^32 threads (the join's are far fewer: it follows grids
    // below shape_of's `want` only)
    if (grid >= (int64_t(1) << 32) / (kWaves * 64))
        return fail(QNN_ERR_UNSUPPORTED, "attention4: too many row tiles");
    a.tiles = (int32_t)g.tiles;
    a.unit_tiles = (int32_t)unit_tiles;
    a.grid = (int32_t)grid;
    a.parts = g.parts;
    a.chunk = g.chunk;
    const int blocks = g.blocks;
    const int dp = cache4_padded(a.c.dim);
    if (a.parts > 1) {
        if (!workspace)
            return fail(QNN_ERR_NULL, "attention4: the call needs a workspace");
        if ((uintptr_t)workspace & 15)
            return fail(QNN_ERR_UNSUPPORTED, "attention4: the workspace must be 16-byte aligned");
        a.part_o = (float *)workspace;
        a.part_p = (float2 *)(a.part_o + (size_t)a.parts * a.tokens * a.q_heads * dp);
    }
    const hipStream_t st = (hipStream_t)stream;
    const hipError_t e = dp == 64    ? launch_attention<64>(a, blocks, st)
                         : dp == 128 ? launch_attention<128>(a, blocks, st)
                                     : launch_attention<256>(a, blocks, st);
    return e == hipSuccess ? QNN_OK : hip_fail(e, "attention4 launch");
}

}  // extern "C"
