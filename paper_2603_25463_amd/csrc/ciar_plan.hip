// gfx950 kernel of the cache plan (ciar_cache_plan in include/ciar.h): which pages and slots the next new tokens of every
// request get.
#include "ciar_device.h"
#include "ciar_step.h"

namespace ciar {
namespace {

// Three running sums decide the plan, each over the requests in order: of the new tokens (which request a token belongs to, and
// whether it lies within the step), of the pages that requests lack (who is granted, and which entries of the ring are whose),
// of the pages that come back (where in the ring they go).  They depend on each other, and everything else is element by
// element, so every workgroup makes the sums for itself, a chunk of 256 or 1024 requests at a time, one or four to a thread, and then takes its
// share of the chunk: tokens 256 at a time, requests' pages a wave to a request.  No exchange between workgroups, one launch.  What a
// workgroup writes no other one reads: pages are taken from entries of the ring and of the table that no one writes in this step.
// Sums are doubles: whole numbers below 2^53, added across a wave by data movement between lanes without LDS.
// Bound by latency: two trips to memory (the requests' numbers, the pages) and the sums between them.  Eight requests of eight
// tokens 3.6 us of kernel (with four requests to a thread 5.5: more code to fetch), a thousand of up to 64 7.0 (with 64-bit sums
// through LDS and a search for each token's request 10.5).
constexpr int kPlanThreads = 256;

// Sum of `v` over the workgroup's threads before this one; `total` the sum over all.
__device__ __forceinline__ double block_before(double v, double* sums, double& total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const double upto = wave_scan(v);
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    const double s0 = sums[0], s1 = sums[1], s2 = sums[2], s3 = sums[3];
    total = (s0 + s1) + (s2 + s3);
    const double before = wave == 0 ? 0.0 : wave == 1 ? s0 : wave == 2 ? s0 + s1 : s0 + s1 + s2;
    return before + (upto - v);
}

template <int N>
__device__ __forceinline__ double sum_of(const double (&v)[N])
{
    double s = v[0];
#pragma unroll
    for (int k = 1; k < N; ++k) s += v[k];
    return s;
}

__device__ __forceinline__ int clamp32(double v) { return v < 2147483647.0 ? (int)v : 0x7fffffff; }

// Largest value of the lanes up to and with this one (values of at least -1).
__device__ __forceinline__ int wave_max_scan(int v)
{
    v = max(v, dpp_or<kRowShr1, 0xf>(-1, v));
    v = max(v, dpp_or<kRowShr2, 0xf>(-1, v));
    v = max(v, dpp_or<kRowShr4, 0xf>(-1, v));
    v = max(v, dpp_or<kRowShr8, 0xf>(-1, v));
    v = max(v, dpp_or<kRowBcast15, 0xa>(-1, v));
    return max(v, dpp_or<kRowBcast31, 0xc>(-1, v));
}

struct PlanRequest {
    int length, start;                 // tokens held, first of its new tokens in the step
    int held, pages;                   // pages before (-1: not granted) and after
    int taken, given;                  // the ring's entries that are its: first of those taken, first of those put back
};

// i % n for the ring's counters, which pass 32 bits only after a very long life
__device__ __forceinline__ uint32_t wrapped(int64_t i, int32_t n)
{
    if ((uint64_t)i <= 0xffffffffull) return (uint32_t)i % (uint32_t)n;
    const int64_t m = i % n;
    return (uint32_t)(m < 0 ? m + n : m);
}

template <int kPlanEach>
__global__ __launch_bounds__(kPlanThreads) void plan_kernel(const PlanArgs A)
{
    constexpr int kPlanChunk = kPlanThreads * kPlanEach;
    __shared__ double sums[3][4];
    __shared__ PlanRequest s_req[kPlanChunk];
    __shared__ int s_first[2][kPlanThreads], s_top[2][4];          // (two sets: one is read while the next is written)
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t head = A.ring_state[0], tail = A.ring_state[1];
    const uint32_t P = (uint32_t)A.P;
    const uint32_t head_at = wrapped(head, A.P), tail_at = wrapped(tail, A.P);
    // (a ring that claims more than it holds breaks the call's preconditions: no index below leaves it)
    const int64_t there = tail - head < 0 ? 0 : tail - head > A.P ? A.P : tail - head;
    auto ring_at = [&](uint32_t from, uint32_t i) { return (from + i) % P; };          // (from < P < 2^28, i < 2^31)

    double tokens = 0.0, lacked = 0.0, given = 0.0;                // sums over the chunks before
    int64_t taken = 0;                                             // entries of the ring that are taken
    int set = 0;
    for (int first = 0; first < A.R; first += kPlanChunk) {
        const int n = min(kPlanChunk, A.R - first), r0 = first + tid * kPlanEach;
        double length[kPlanEach], fresh[kPlanEach], end[kPlanEach];
        int held[kPlanEach], pages[kPlanEach];
        bool fits[kPlanEach];
#pragma unroll
        for (int k = 0; k < kPlanEach; ++k) {
            const bool mine = r0 + k < A.R;
            const int r = mine ? r0 + k : first;
            length[k] = (double)max(A.lengths[r], 0) + (A.kept ? (double)max(A.kept[r], 0) : 0.0);
            fresh[k] = mine ? (double)max(A.fresh[r], 0) : 0.0;
            held[k] = min(max(A.held[r], 0), A.width);
        }
        double all;
        double run = tokens + block_before(sum_of(fresh), sums[0], all);
        const double before = tokens;
        tokens += all;
        double lack[kPlanEach];
#pragma unroll
        for (int k = 0; k < kPlanEach; ++k) {
            run += fresh[k];
            end[k] = run;
            // (beyond 32 bits: more pages than any row of the table holds)
            const uint32_t total = (uint32_t)min(length[k] + fresh[k], 4294901760.0), whole = total / (uint32_t)A.page;
            pages[k] = (int)min(whole + (whole * (uint32_t)A.page != total ? 1u : 0u), 0x7fffffffu);
            fits[k] = r0 + k < A.R && pages[k] <= A.width && end[k] <= (double)A.T;
            lack[k] = fits[k] && pages[k] > held[k] ? (double)(pages[k] - held[k]) : 0.0;
        }
        run = lacked + block_before(sum_of(lack), sums[1], all);
        lacked += all;
        bool granted[kPlanEach];
        double gives[kPlanEach], upto[kPlanEach];
        double most = -1.0;                                        // largest running sum of a request that gets what it lacks
#pragma unroll
        for (int k = 0; k < kPlanEach; ++k) {
            run += lack[k];
            upto[k] = run;
            granted[k] = fits[k] && (lack[k] == 0.0 || upto[k] <= (double)there);
            gives[k] = granted[k] && held[k] > pages[k] ? (double)(held[k] - pages[k]) : 0.0;
            if (granted[k] && lack[k] > 0.0) most = upto[k];
        }
        run = given + block_before(sum_of(gives), sums[2], all);
        given += all;
#pragma unroll
        for (int k = 0; k < kPlanEach; ++k) {
            const int r = r0 + k, i = tid * kPlanEach + k;
            if (i >= n) break;
            PlanRequest q;
            q.length = clamp32(length[k]);
            q.start = clamp32(min(end[k] - fresh[k], (double)A.T));
            q.held = granted[k] ? held[k] : -1;
            q.pages = pages[k];
            q.taken = clamp32(upto[k] - lack[k]);
            q.given = clamp32(run);
            run += gives[k];
            s_req[i] = q;
            if (blockIdx.x == 0) {
                A.out_lengths[r] = clamp32(length[k]);
                A.kv_len[r] = granted[k] ? clamp32(length[k] + fresh[k]) : 0;
                A.cu_new[r + 1] = clamp32(min(end[k], (double)A.T));
                A.out_held[r] = granted[k] ? pages[k] : held[k];
                A.granted[r] = granted[k] ? 1 : 0;
            }
        }
        // (whoever lacks pages behind one that is denied gets none: what is taken is the last granted running sum)
        {
            const int top = wave_max_scan(clamp32(most < 0.0 ? -1.0 : most));
            if (lane == 63) s_top[set][wave] = top;
        }
        // the tokens' slots, 256 at a time: every request marks its first token there, and the marks spread to the next one
        const int token_end = clamp32(min(tokens, (double)A.T)), token_first = clamp32(min(before, (double)A.T));
        const int step = (int)gridDim.x * kPlanThreads;
        int mark_set = 0;
        bool joined = false;
        for (int t0 = token_first + (int)blockIdx.x * kPlanThreads; t0 < token_end; t0 += step, mark_set ^= 1) {
            s_first[mark_set][tid] = -1;
            __syncthreads();
            joined = true;
#pragma unroll
            for (int k = 0; k < kPlanEach; ++k) {
                const int i = tid * kPlanEach + k;
                const double from = end[k] - fresh[k];
                if (i < n && fresh[k] > 0.0 && from < (double)t0 + kPlanThreads && end[k] > (double)t0)
                    s_first[mark_set][max(clamp32(from) - t0, 0)] = i;
            }
            __syncthreads();
            int own = wave_max_scan(s_first[mark_set][tid]);
            // (a wave whose first token has no mark goes on with the last mark before it)
            int carry = -1;
            for (int w = 0; w < wave; ++w) {
                const int last = wave_max_scan(s_first[mark_set][w * 64 + lane]);
                carry = max(carry, __builtin_amdgcn_readlane(last, 63));
            }
            own = max(own, carry);
            const int t = t0 + tid;
            if (t >= token_end || own < 0) continue;
            const PlanRequest q = s_req[own];
            const int64_t pos = (int64_t)q.length + (t - q.start);
            int slot = -1;
            if (q.held >= 0) {
                const int col = (int)((uint32_t)pos / (uint32_t)A.page), off = (int)((uint32_t)pos - (uint32_t)col * (uint32_t)A.page);
                const int page = col < q.held ? A.table[(int64_t)(first + own) * A.table_stride + col]
                                              : A.ring[ring_at(head_at, (uint32_t)(q.taken + (col - q.held)))];
                slot = (int)((int64_t)page * A.page + off);
            }
            A.slots[t] = slot;
            A.positions[t] = (int)pos;
            A.requests[t] = first + own;
        }
        if (!joined) __syncthreads();
        taken = max(taken, (int64_t)max(max(s_top[set][0], s_top[set][1]), max(s_top[set][2], s_top[set][3])));
        set ^= 1;
        // pages into the table and back into the ring, a wave to a request
        for (int i = (int)blockIdx.x * 4 + wave; i < n; i += (int)gridDim.x * 4) {
            const PlanRequest q = s_req[i];
            if (q.held < 0) continue;
            int32_t* row = A.table + (int64_t)(first + i) * A.table_stride;
            for (int c = lane; c < q.pages - q.held; c += 64) row[q.held + c] = A.ring[ring_at(head_at, (uint32_t)(q.taken + c))];
            for (int c = lane; c < q.held - q.pages; c += 64) A.ring[ring_at(tail_at, (uint32_t)(q.given + c))] = row[q.pages + c];
        }
        __syncthreads();
    }
    // places of the step that no request has claimed
    const int64_t from = clamp32(min(tokens, (double)A.T));
    for (int64_t i = from + (int64_t)blockIdx.x * kPlanThreads + tid; i < A.T; i += (int64_t)gridDim.x * kPlanThreads) {
        A.slots[i] = -1;
        A.positions[i] = 0;
        A.requests[i] = -1;
    }
    if (blockIdx.x == 0 && tid == 0) {
        A.cu_new[0] = 0;
        A.out_ring_state[0] = head + taken;
        A.out_ring_state[1] = tail + (int64_t)given;
    }
}

}  // namespace

hipError_t launch_plan(const PlanArgs& args, hipStream_t stream)
{
    // A workgroup for every 256 tokens and every four requests; more than one per compute unit would only repeat the sums.
    const int64_t by_tokens = ((int64_t)args.T + kPlanThreads - 1) / kPlanThreads, by_requests = ((int64_t)args.R + 3) / 4;
    const int64_t g = by_tokens > by_requests / 8 ? by_tokens : by_requests / 8, most = compute_units();
    const unsigned grid = (unsigned)(g < 1 ? 1 : g > most ? most : g);
    if (args.R <= kPlanThreads) hipLaunchKernelGGL(plan_kernel<1>, dim3(grid), dim3(kPlanThreads), 0, stream, args);
    else hipLaunchKernelGGL(plan_kernel<4>, dim3(grid), dim3(kPlanThreads), 0, stream, args);
    return hipGetLastError();
}

}  // namespace ciar
