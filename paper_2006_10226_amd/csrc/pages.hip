// Block tables and slots of a paged cache from the requests' lengths
// (qnn_pages_resize): three running sums over the requests (pages given
// back, pages taken, new tokens), then one element of work per page given
// back and per new token.
//
// The sums are one workgroup's work; what they give (offsets in the
// workspace and cu) lets every later element find its request by bisection
// and its page on the stack by its own number, so that nothing depends on an
// order of execution and no atomics are needed.
#include "qnn_host.h"
#include "qnn_internal.h"

#include <algorithm>

namespace qnn {
namespace {

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
    int32_t *head, *old, *gone, *got;
};
enum { HEAD_GO = 0, HEAD_COUNT = 1, HEAD_GONE = 2, HEAD_INTS = 4 };

constexpr int kSumThreads = 1024;

// Pages of n tokens.
__device__ __forceinline__ int pages_of(int n, int shift) { return (int)(((int64_t)n + (1 << shift) - 1) >> shift); }

// Largest i with at[i] <= v, at[0 .. n] ascending with at[0] <= v < at[n].
__device__ __forceinline__ int find(const int32_t *at, int n, int v)
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

struct Sums {
    long long gone, got, add;
};

// Running sums over the workgroup's threads, exclusive, and their totals.
__device__ __forceinline__ Sums block_scan(Sums v, Sums *total)
{
    __shared__ Sums wave_sum[kSumThreads / 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    Sums s = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const long long a = __shfl_up(s.gone, d), b = __shfl_up(s.got, d), c = __shfl_up(s.add, d);
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
    Sums before{0, 0, 0}, all{0, 0, 0};
#pragma unroll
    for (int w = 0; w < kSumThreads / 64; ++w) {
        const Sums t = wave_sum[w];
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
    return Sums{before.gone + s.gone - v.gone, before.got + s.got - v.got, before.add + s.add - v.add};
}

// One workgroup of kSumThreads: the running sums, the decision, the lengths.
__device__ void sum_requests(const PagesArgs &a)
{
    const int tid = threadIdx.x;
    const long long most = (long long)a.width << a.shift;
    long long gone = 0, got = 0, add = 0;
    int bad = 0;
    for (int at = 0; at < a.requests; at += kSumThreads) {
        const int b = at + tid;
        Sums v{0, 0, 0};
        int old = 0;
        if (b < a.requests) {
            old = a.lens[b];
            const int now = a.new_lens[b];
            if (old < 0 || now < 0 || old > most || now > most) {
                bad = 1;
            } else {
                const int have = pages_of(old, a.shift), want = pages_of(now, a.shift);
                v = Sums{max(have - want, 0), max(want - have, 0), max(now - old, 0)};
            }
        }
        Sums total;
        const Sums s = block_scan(v, &total);
        // a sum beyond 32 bits is refused below, by its 64-bit total
        if (b < a.requests) {
            a.old[b] = old;
            a.gone[b] = (int)(gone + s.gone);
            a.got[b] = (int)(got + s.got);
            a.cu[b] = (int)(add + s.add);
        }
        gone += total.gone;
        got += total.got;
        add += total.add;
    }
    const int n = *a.free_count;
    bad = __syncthreads_or(bad) || n < 0 || n > a.capacity;
    int status = 0;
    if (bad)
        status = -1;
    else if (add > a.tokens)
        status = -2;
    else if (n + gone > a.capacity)
        status = -3;
    else if (got > n + gone)
        status = (int)min(got - n - gone, (long long)INT32_MAX);
    for (int b = tid; b < a.requests; b += kSumThreads) {
        if (status)
            a.cu[b] = 0;
        else
            a.lens[b] = a.new_lens[b];
    }
    if (tid == 0) {
        a.gone[a.requests] = (int)gone;
        a.got[a.requests] = (int)got;
        a.cu[a.requests] = status ? 0 : (int)add;
        a.head[HEAD_GO] = status == 0;
        a.head[HEAD_COUNT] = (int)(n + gone);
        a.head[HEAD_GONE] = status ? 0 : (int)gone;
        *a.status = status;
        if (status == 0)
            *a.free_count = (int)(n + gone - got);
    }
}

// Pages given back: element `at` on, by `stride`.
__device__ __forceinline__ void give_back(const PagesArgs &a, int at, int stride)
{
    const int n = a.head[HEAD_GONE], count = a.head[HEAD_COUNT];
    for (int i = at; i < n; i += stride) {
        const int b = find(a.gone, a.requests, i);
        // the lengths have been updated: lens[b] is the new one
        int32_t *entry = a.table + b * a.ld + pages_of(a.lens[b], a.shift) + (i - a.gone[b]);
        a.free_pages[count - 1 - i] = *entry;
        *entry = -1;
    }
}

// Slots, positions and new table entries: tokens `at` on, by `stride`.
__device__ __forceinline__ void place_tokens(const PagesArgs &a, int at, int stride)
{
    const int go = a.head[HEAD_GO], count = a.head[HEAD_COUNT];
    const int total = go ? a.cu[a.requests] : 0;
    for (int t = at; t < a.tokens; t += stride) {
        int slot = -1, pos = 0;
        if (t < total) {
            const int b = find(a.cu, a.requests, t);
            const int old = a.old[b];
            pos = old + t - a.cu[b];
            const int j = pos >> a.shift, have = pages_of(old, a.shift), off = pos & ((1 << a.shift) - 1);
            int page;
            if (j < have) {
                page = a.table[b * a.ld + j];
            } else {
                page = a.free_pages[count - 1 - (a.got[b] + j - have)];
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

__global__ void __launch_bounds__(kSumThreads) sum_kernel(PagesArgs a) { sum_requests(a); }

__global__ void __launch_bounds__(256) give_back_kernel(PagesArgs a)
{
    give_back(a, blockIdx.x * 256 + threadIdx.x, gridDim.x * 256);
}

__global__ void __launch_bounds__(256) place_kernel(PagesArgs a)
{
    place_tokens(a, blockIdx.x * 256 + threadIdx.x, gridDim.x * 256);
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
    return HEAD_INTS * sizeof(int32_t) + 3 * round16(((size_t)requests + 1) * sizeof(int32_t));
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
    a.head = (int32_t *)ws;
    a.old = (int32_t *)(ws + HEAD_INTS * sizeof(int32_t));
    a.gone = (int32_t *)(ws + HEAD_INTS * sizeof(int32_t) + row);
    a.got = (int32_t *)(ws + HEAD_INTS * sizeof(int32_t) + 2 * row);
    const hipStream_t st = (hipStream_t)stream;
    launch_main(sum_kernel, dim3(1), dim3(kSumThreads), 0, st, a);
    give_back_kernel<<<256, 256, 0, st>>>(a);
    place_kernel<<<std::max(1, std::min(2048, (int)(((int64_t)token_capacity + 255) / 256))), 256, 0, st>>>(a);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? QNN_OK : hip_fail(e, "pages_resize launch");
}

}  // extern "C"
