// gfx950 kernel of the cache plan (ciar_cache_plan in include/ciar.h): which pages and slots the next new tokens of every
// request get.
#include "ciar_device.h"
#include "ciar_step.h"

namespace ciar {
namespace {

// Three running sums decide the plan, each over the requests in order: of the new tokens (which request a token belongs to, and
// whether it lies within the step), of the pages that requests lack (who is granted, and which entries of the ring are whose),
// of the pages that come back (where in the ring they go).  They depend on each other, and everything else is element by
// element, so every workgroup makes the sums for itself, a chunk of as many requests as it has threads at a time, and then takes
// its share of the chunk's tokens, new pages and returned pages; no exchange between workgroups, one launch.  What a workgroup
// writes no other one reads: pages are taken from entries of the ring and of the table that no one writes in this step.
// Bound by latency: eight requests of eight tokens are one workgroup's three sums, a thousand requests of up to 64 a wave or two
// of tokens in each workgroup (figures at launch_plan).

// Sum of `v` over the workgroup's threads up to and with this one; `total` the sum over all.
template <int THREADS>
__device__ __forceinline__ int64_t block_scan(int64_t v, int64_t* sums, int64_t& total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int64_t u = __shfl_up(v, d);
        if (lane >= d) v += u;
    }
    __syncthreads();
    if (lane == 63) sums[wave] = v;
    __syncthreads();
    int64_t before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
        if (w == wave) before = total;
        total += sums[w];
    }
    return before + v;
}

__device__ __forceinline__ int clamp32(int64_t v) { return (int)(v < 0 ? 0 : v > 0x7fffffff ? 0x7fffffff : v); }

// First of `n` ascending numbers that is above `x` (n if none is).
__device__ __forceinline__ int first_above(const int* list, int n, int x)
{
    int lo = 0, hi = n;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (list[mid] > x) hi = mid; else lo = mid + 1;
    }
    return lo;
}

template <int THREADS>
__global__ __launch_bounds__(THREADS) void plan_kernel(const PlanArgs A)
{
    __shared__ int64_t sums[THREADS / 64];
    __shared__ int s_end[THREADS], s_taken[THREADS], s_given[THREADS];   // running sums at the end of each request of the chunk
    __shared__ int s_length[THREADS], s_held[THREADS], s_pages[THREADS]; // (s_held: -1 where not granted)
    const int tid = threadIdx.x;
    const int64_t head = A.ring_state[0], tail = A.ring_state[1];
    const uint32_t P = (uint32_t)A.P;
    int64_t hm = head % A.P, tm = tail % A.P;
    const uint32_t head_at = (uint32_t)(hm < 0 ? hm + A.P : hm), tail_at = (uint32_t)(tm < 0 ? tm + A.P : tm);
    // (a ring that claims more than it holds breaks the call's preconditions: no index below leaves it)
    const int64_t there = tail - head < 0 ? 0 : tail - head > A.P ? A.P : tail - head;
    auto ring_at = [&](uint32_t from, uint32_t i) { return (from + i % P) % P; };

    int64_t tokens = 0, lacked = 0, taken = 0, given = 0;                 // sums over the chunks before
    for (int first = 0; first < A.R; first += THREADS) {
        const int r = first + tid, n = min(THREADS, A.R - first);
        const bool mine = tid < n;
        int64_t length = 0, fresh = 0;
        int held = 0;
        if (mine) {
            length = (int64_t)max(A.lengths[r], 0) + (A.kept ? max(A.kept[r], 0) : 0);
            fresh = max(A.fresh[r], 0);
            held = min(max(A.held[r], 0), A.width);
        }
        int64_t all;
        const int64_t end = tokens + block_scan<THREADS>(fresh, sums, all);
        const int64_t before = tokens;
        tokens += all;
        const int64_t pages = (length + fresh + A.page - 1) / A.page;
        const bool fits = mine && pages <= A.width && end <= A.T;
        const int64_t lacks = fits && pages > held ? pages - held : 0;
        const int64_t upto = lacked + block_scan<THREADS>(lacks, sums, all);
        lacked += all;
        const bool granted = fits && (lacks == 0 || upto <= there);
        const int64_t taken_before = taken;
        const int64_t gives = granted && held > pages ? held - pages : 0;
        const int64_t gone = given + block_scan<THREADS>(gives, sums, all);
        const int64_t given_before = given;
        given += all;
        s_end[tid] = clamp32(end < A.T ? end : A.T);
        s_taken[tid] = clamp32(upto);
        s_given[tid] = clamp32(gone);
        s_length[tid] = clamp32(length);
        s_pages[tid] = clamp32(pages);
        s_held[tid] = granted ? held : -1;
        if (mine && blockIdx.x == 0) {
            A.out_lengths[r] = (int)length;
            A.kv_len[r] = granted ? (int)(length + fresh) : 0;
            A.cu_new[r + 1] = clamp32(end < A.T ? end : A.T);
            A.out_held[r] = granted ? (int)pages : held;
            A.granted[r] = granted ? 1 : 0;
        }
        __syncthreads();
        // Entries of the ring that are taken now: up to the first request whose running sum passes what is there.  (Whoever lacks
        // pages behind it gets none, so that the running sums of those who do get theirs are their entries.)
        const int denied = first_above(s_taken, n, (int)there);
        if (denied > 0) taken = s_taken[denied - 1];
        const int stride = (int)gridDim.x * THREADS, at = (int)blockIdx.x * THREADS + tid;
        // the tokens' slots
        const int token_end = clamp32(tokens < A.T ? tokens : A.T);
        for (int64_t i = before + at; i < token_end; i += stride) {
            const int q = first_above(s_end, n, (int)i);
            if (q >= n) continue;                                         // (cannot be: s_end[n - 1] = token_end)
            const int64_t start = q > 0 ? s_end[q - 1] : before;
            const int64_t pos = (int64_t)s_length[q] + (i - start);
            int slot = -1;
            if (s_held[q] >= 0) {
                const int col = (int)(pos / A.page), off = (int)(pos - (int64_t)col * A.page);
                int page;
                if (col < s_held[q]) page = A.table[(int64_t)(first + q) * A.table_stride + col];
                else {
                    const int64_t own = (int64_t)s_taken[q] - (s_pages[q] - s_held[q]);       // entries taken before it
                    page = A.ring[ring_at(head_at, (uint32_t)(own + (col - s_held[q])))];
                }
                slot = (int)((int64_t)page * A.page + off);
            }
            A.slots[i] = slot;
            A.positions[i] = (int)pos;
            A.requests[i] = first + q;
        }
        // new pages into the table
        for (int64_t i = taken_before + at; i < taken; i += stride) {
            const int q = first_above(s_taken, n, (int)i);
            if (q >= n) continue;
            const int64_t own = (int64_t)s_taken[q] - (s_pages[q] - s_held[q]);
            const int64_t col = s_held[q] + (i - own);
            A.table[(int64_t)(first + q) * A.table_stride + col] = A.ring[ring_at(head_at, (uint32_t)i)];
        }
        // pages that come back
        for (int64_t i = given_before + at; i < given; i += stride) {
            const int q = first_above(s_given, n, (int)i);
            if (q >= n) continue;
            const int64_t own = (int64_t)s_given[q] - (s_held[q] - s_pages[q]);
            const int64_t col = s_pages[q] + (i - own);
            A.ring[ring_at(tail_at, (uint32_t)i)] = A.table[(int64_t)(first + q) * A.table_stride + col];
        }
        __syncthreads();
    }
    // places of the step that no request has claimed
    const int64_t from = tokens < A.T ? tokens : A.T;
    for (int64_t i = from + (int64_t)blockIdx.x * THREADS + tid; i < A.T; i += (int64_t)gridDim.x * THREADS) {
        A.slots[i] = -1;
        A.positions[i] = 0;
        A.requests[i] = -1;
    }
    if (blockIdx.x == 0 && tid == 0) {
        A.cu_new[0] = 0;
        A.out_ring_state[0] = head + taken;
        A.out_ring_state[1] = tail + given;
    }
}

}  // namespace

hipError_t launch_plan(const PlanArgs& args, hipStream_t stream)
{
    // A workgroup for every thousand or so of tokens and requests; more than one per compute unit would only repeat the sums.
    const int64_t work = (int64_t)args.T + args.R;
    const int64_t g = (work + 1023) / 1024;
    const unsigned grid = (unsigned)(g < 1 ? 1 : g > 256 ? 256 : g);
    if (args.R <= 256) hipLaunchKernelGGL(plan_kernel<256>, dim3(grid), dim3(256), 0, stream, args);
    else hipLaunchKernelGGL(plan_kernel<1024>, dim3(grid), dim3(1024), 0, stream, args);
    return hipGetLastError();
}

}  // namespace ciar
