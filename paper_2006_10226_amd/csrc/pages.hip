// Block tables and slots of a paged cache from the requests' lengths
// (qnn_pages_resize): three running sums over the requests (pages given
// back, pages taken, new tokens), then one element of work per page given
// back and per new token.
//
// The sums are one workgroup's work; what they give (offsets in the
// workspace and cu) lets every later element find its request by bisection
// and its page on the stack by its own number, so that nothing depends on an
// order of execution and no atomics are needed. A few kilobytes: what bounds it is
// dependent memory latencies (lengths, sums, bisection, page), 5.0 us for 64
// requests of a token each, 16.5 us in three kernels for 1000 requests with 55000 new
// tokens.
#include "qnn_host.h"
#include "qnn_internal.h"

#include <algorithm>

namespace qnn {
namespace {

struct Head;
struct PagesArgs {
    int32_t requests, shift;   // page size 1 << shift
    int32_t *lens;
    const int32_t *new_lens;
    int32_t *table;
    int32_t width;
    int64_t ld;
    int32_t *free_pages;
    int32_t capacity;
    int32_t *free_count;
    int32_t *cu, *slots, *positions;
    int32_t tokens;
    int32_t *status;
    // workspace: head, the old lengths, the running counts of pages given
    // back and taken (requests + 1 each)
    Head *head;
    int32_t *old, *gone, *got;
};

constexpr int kSumThreads = 1024;

// Pages of n tokens.
__device__ __forceinline__ int pages_of(int n, int shift) { return (int)(((int64_t)n + (1 << shift) - 1) >> shift); }

// What the sums say: whether anything is done, the stack's count with the pages
// given back on it, those, and the new tokens.
struct Head {
    int go, count, gone, tokens;
};

// Largest i with at[i] <= v, at[0 .. n] ascending with at[0] <= v < at[n].
template <typename A>
__device__ __forceinline__ int find(const A &at, int n, int v)
{
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (at[mid] <= v)
            lo = mid;
        else
            hi = mid;
    }
    return lo;
}

// T: int where no sum of a call can pass 32 bits, else long long.
template <typename T>
struct Sums {
    T gone, got, add;
};

// Running sums over the workgroup's threads, exclusive, and their totals.
template <typename T>
__device__ __forceinline__ Sums<T> block_scan(Sums<T> v, Sums<T> *total)
{
    __shared__ Sums<T> wave_sum[kSumThreads / 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    Sums<T> s = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const T a = __shfl_up(s.gone, d), b = __shfl_up(s.got, d), c = __shfl_up(s.add, d);
        if (lane >= d) {
            s.gone += a;
            s.got += b;
            s.add += c;
        }
    }
    __syncthreads();   // the last call's sums have been read
    if (lane == 63)
        wave_sum[wave] = s;
    __syncthreads();
    Sums<T> before{0, 0, 0}, all{0, 0, 0};
#pragma unroll 4
    for (int w = 0; w < kSumThreads / 64; ++w) {
        const Sums<T> t = wave_sum[w];
        if (w < wave) {
            before.gone += t.gone;
            before.got += t.got;
            before.add += t.add;
        }
        all.gone += t.gone;
        all.got += t.got;
        all.add += t.add;
    }
    *total = all;
    return Sums<T>{before.gone + s.gone - v.gone, before.got + s.got - v.got, before.add + s.add - v.add};
}

// One workgroup of kSumThreads: the running sums (to the workspace and cu, and to
// `lists` where all requests fit it), the decision, the lengths.
struct Lists {
    int old[kSumThreads], now[kSumThreads], gone[kSumThreads], got[kSumThreads], cu[kSumThreads + 1];
};
template <typename T, bool LISTS>
__device__ __forceinline__ Head sum_requests(const PagesArgs &a, Lists *lists)
{
    const int tid = threadIdx.x;
    const int n = *a.free_count;
    const long long most = (long long)a.width << a.shift;
    T gone = 0, got = 0, add = 0;
    int bad = n < 0 || n > a.capacity, old = 0, now = 0;
    Sums<T> s{0, 0, 0};
    // (counts are below 2^31 and numbers unsigned, here and below: the one past the
    // last, by a stride, doesn't wrap)
    const uint32_t requests = (uint32_t)a.requests;
    for (uint32_t at = 0; at < requests; at += kSumThreads) {
        const uint32_t b = at + tid;
        Sums<T> v{0, 0, 0};
        if (b < requests) {
            old = a.lens[b];
            now = a.new_lens[b];
            if (old < 0 || now < 0 || old > most || now > most) {
                bad = 1;
            } else {
                const int have = pages_of(old, a.shift), want = pages_of(now, a.shift);
                v = Sums<T>{max(have - want, 0), max(want - have, 0), max(now - old, 0)};
            }
        }
        Sums<T> total;
        s = block_scan<T>(v, &total);
        if (!LISTS && b < requests) {
            // a sum beyond 32 bits is refused below, by its total
            a.old[b] = old;
            a.gone[b] = (int)(gone + s.gone);
            a.got[b] = (int)(got + s.got);
            a.cu[b] = (int)(add + s.add);
        }
        gone += total.gone;
        got += total.got;
        add += total.add;
    }
    bad = __syncthreads_or(bad);
    int status = 0;
    if (bad)
        status = -1;
    else if (add > a.tokens)
        status = -2;
    else if (n + (long long)gone > a.capacity)
        status = -3;
    else if (got > n + (long long)gone)
        status = (int)min((long long)got - n - gone, (long long)INT32_MAX);
    if constexpr (LISTS) {
        if (tid < a.requests) {
            lists->old[tid] = old;
            lists->now[tid] = now;
            lists->gone[tid] = s.gone;
            lists->got[tid] = s.got;
            lists->cu[tid] = s.add;
            a.cu[tid] = status ? 0 : s.add;
            if (!status)
                a.lens[tid] = now;
        }
    } else {
        for (uint32_t b = tid; b < requests; b += kSumThreads) {
            if (status)
                a.cu[b] = 0;
            else
                a.lens[b] = a.new_lens[b];
        }
    }
    const Head h{status == 0, (int)(n + (long long)gone), status ? 0 : (int)gone, status ? 0 : (int)add};
    if (tid == 0) {
        a.cu[a.requests] = h.tokens;
        *a.status = status;
        if (status == 0)
            *a.free_count = (int)(n + (long long)gone - got);
        if constexpr (LISTS) {
            lists->cu[a.requests] = h.tokens;
        } else {
            a.gone[a.requests] = (int)gone;
            *a.head = h;
        }
    }
    return h;
}

// Pages given back: element `at` on, by `stride`.
template <typename G, typename N>
__device__ __forceinline__ void give_back(const PagesArgs &a, const Head &h, const G &gone, const N &now, uint32_t at,
                                          uint32_t stride)
{
    for (uint32_t n = at; n < (uint32_t)h.gone; n += stride) {
        const int i = (int)n, b = find(gone, a.requests, i);
        int32_t *entry = a.table + b * a.ld + pages_of(now[b], a.shift) + (i - gone[b]);
        a.free_pages[h.count - 1 - i] = *entry;
        *entry = -1;
    }
}

// Slots, positions and new table entries: tokens `at` on, by `stride`.
template <typename C, typename O, typename G>
__device__ __forceinline__ void place_tokens(const PagesArgs &a, const Head &h, const C &cu, const O &olds, const G &got,
                                             uint32_t at, uint32_t stride)
{
    for (uint32_t n = at; n < (uint32_t)a.tokens; n += stride) {
        const int t = (int)n;
        int slot = -1, pos = 0;
        if (t < h.tokens) {
            const int b = find(cu, a.requests, t);
            const int old = olds[b];
            pos = old + t - cu[b];
            const int j = pos >> a.shift, have = pages_of(old, a.shift), off = pos & ((1 << a.shift) - 1);
            int page;
            if (j < have) {
                page = a.table[b * a.ld + j];
            } else {
                page = a.free_pages[h.count - 1 - (got[b] + j - have)];
                if (off == 0)   // a new page's first token is a new one
                    a.table[b * a.ld + j] = page;
            }
            slot = (int)(((uint32_t)page << a.shift) + (uint32_t)off);
        }
        a.slots[t] = slot;
        if (a.positions)
            a.positions[t] = pos;
    }
}

// Everything in one workgroup, the running sums in LDS: few requests and tokens.
template <typename T>
__global__ void __launch_bounds__(kSumThreads) resize_kernel(PagesArgs a)
{
    __shared__ Lists lists;
    const Head h = sum_requests<T, true>(a, &lists);
    __syncthreads();
    give_back(a, h, lists.gone, lists.now, threadIdx.x, kSumThreads);
    __syncthreads();   // the pages taken may be among those given back
    place_tokens(a, h, lists.cu, lists.old, lists.got, threadIdx.x, kSumThreads);
}

__global__ void __launch_bounds__(kSumThreads) sum_kernel(PagesArgs a) { sum_requests<long long, false>(a, nullptr); }

__global__ void __launch_bounds__(256) give_back_kernel(PagesArgs a)
{
    // (the lengths have been updated: lens holds the new ones)
    give_back(a, *a.head, a.gone, a.lens, blockIdx.x * 256 + threadIdx.x, gridDim.x * 256);
}

__global__ void __launch_bounds__(256) place_kernel(PagesArgs a)
{
    place_tokens(a, *a.head, a.cu, a.old, a.got, blockIdx.x * 256 + threadIdx.x, gridDim.x * 256);
}

size_t round16(size_t v) { return (v + 15) / 16 * 16; }

}  // namespace
}  // namespace qnn

using namespace qnn;

extern "C" {

size_t qnn_pages_workspace_size(int32_t requests)
{
    if (requests < 0)
        return 0;
    return sizeof(Head) + 3 * round16(((size_t)requests + 1) * sizeof(int32_t));
}

qnn_status qnn_pages_resize(void *stream, int32_t requests, int32_t page_size, int32_t *lens, const int32_t *new_lens,
                            int32_t *table, int32_t table_width, int64_t table_ld, int32_t *free_pages,
                            int32_t free_capacity, int32_t *free_count, int32_t *cu, int32_t *slots,
                            int32_t *positions, int32_t token_capacity, int32_t *status, void *workspace)
{
    if (requests < 0 || token_capacity < 0 || free_capacity < 0)
        return fail(QNN_ERR_SHAPE, "pages_resize: negative requests, token_capacity or free_capacity");
    if (page_size < 1 || page_size > 4096 || (page_size & (page_size - 1)))
        return fail(QNN_ERR_SHAPE, "pages_resize: page_size %d is not a power of two of 1 to 4096", page_size);
    if (table_width < 1 || table_ld < table_width)
        return fail(QNN_ERR_SHAPE, "pages_resize: table_width %d, table_ld %lld", table_width, (long long)table_ld);
    if ((int64_t)table_width * page_size >= (int64_t(1) << 31))
        return fail(QNN_ERR_UNSUPPORTED, "pages_resize: a request's pages hold 2^31 tokens or more");
    if (!free_count || !cu || !status || !workspace || (requests && (!lens || !new_lens || !table)) ||
        (free_capacity && !free_pages) || (token_capacity && !slots))
        return fail(QNN_ERR_NULL, "pages_resize: a required pointer is NULL");
    if ((uintptr_t)workspace & 15)
        return fail(QNN_ERR_UNSUPPORTED, "pages_resize: the workspace must be 16-byte aligned");
    PagesArgs a{};
    a.requests = requests;
    a.shift = __builtin_ctz((unsigned)page_size);
    a.lens = lens;
    a.new_lens = new_lens;
    a.table = table;
    a.width = table_width;
    a.ld = table_ld;
    a.free_pages = free_pages;
    a.capacity = free_capacity;
    a.free_count = free_count;
    a.cu = cu;
    a.slots = slots;
    a.positions = positions;
    a.tokens = token_capacity;
    a.status = status;
    const size_t row = round16(((size_t)requests + 1) * sizeof(int32_t));
    char *ws = (char *)workspace;
    a.head = (Head *)ws;
    a.old = (int32_t *)(ws + sizeof(Head));
    a.gone = (int32_t *)(ws + sizeof(Head) + row);
    a.got = (int32_t *)(ws + sizeof(Head) + 2 * row);
    const hipStream_t st = (hipStream_t)stream;
    // One launch where a workgroup can do the elements' work in about two passes. A
    // call of 64 or 1000 requests and the copies that set it up: 16.5 us in one launch,
    // 22.6 in three, up to 8000 new tokens; 22.9 or 27.0 and 22.7 at 16000.
    if (requests <= kSumThreads && token_capacity <= 2 * kSumThreads) {
        const int64_t most = (int64_t)requests * table_width * page_size;
        if (most < (int64_t(1) << 31))
            launch_main((resize_kernel<int>), dim3(1), dim3(kSumThreads), 0, st, a);
        else
            launch_main((resize_kernel<long long>), dim3(1), dim3(kSumThreads), 0, st, a);
        const hipError_t e = hipGetLastError();
        return e == hipSuccess ? QNN_OK : hip_fail(e, "pages_resize launch");
    }
    launch_main(sum_kernel, dim3(1), dim3(kSumThreads), 0, st, a);
    give_back_kernel<<<256, 256, 0, st>>>(a);
    place_kernel<<<std::max(1, std::min(2048, (int)(((int64_t)token_capacity + 255) / 256))), 256, 0, st>>>(a);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? QNN_OK : hip_fail(e, "pages_resize launch");
}

}  // extern "C"
