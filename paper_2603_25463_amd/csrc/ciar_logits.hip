// gfx950 kernel of the logits' adjustments (ciar_adjust_logits in include/ciar.h): penalties for tokens that have come before,
// biases, grammar masks.
#include "ciar_device.h"
#include "ciar_step.h"

namespace ciar {
namespace {

// A workgroup takes a slice of the vocabulary for rows of one window: what the window's rows share (its history, its biases) is
// counted once into two words of LDS per token of the slice, then the rows stream by.  Row n of a window sees the drafted tokens
// before it: they are added to the counts one by one between the rows, each by the lane whose vector the token lies in, so that no
// barrier separates rows.  Tokens that nothing concerns (most) go through as bits: only their mask bit is looked at.
constexpr int kLogitThreads = 256, kLogitVecs = 2;             // vectors of 16 bytes per lane: a slice is 2048 fp32 or 4096 bf16 tokens
constexpr int kLogitRows = 64;                                 // most rows of a workgroup
constexpr uint32_t kEver = 0x80000000u;                        // the token has come up; below: how often behind the prompt

// The words in which a row's slices meet: [32 tag | 8 slices | 24 finite logits].  True for the last slice, with the row's sum.
__device__ __forceinline__ bool left_arrive(uint64_t* p, uint32_t tag, int slices, uint32_t part, uint32_t& sum)
{
    const unsigned long long own = (unsigned long long)tag << 32;
    unsigned long long seen = own;                             // (a fresh word, as the first to arrive makes it)
    for (;;) {
        const unsigned long long cur = (seen >> 32) == tag ? seen : own;
        const unsigned long long next = cur + ((1ull << 24) | part);
        const unsigned long long prev = atomicCAS((unsigned long long*)p, seen, next);
        if (prev == seen) {
            if ((int)((next >> 24) & 0xffull) != slices) return false;
            sum = (uint32_t)(next & 0xffffffull);
            // complete: hand the word back (a replay of this launch from a captured graph carries the same tag)
            __hip_atomic_store((unsigned long long*)p, 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            return true;
        }
        seen = prev;
    }
}

template <typename T>
__global__ __launch_bounds__(kLogitThreads) void adjust_kernel(const LogitArgs A)
{
    using E = Elt<T>;
    constexpr int EPV = E::kPerVec, SLICE = kLogitThreads * kLogitVecs * EPV;
    __shared__ uint32_t words[SLICE];
    __shared__ float bias[SLICE];
    __shared__ uint32_t left[kLogitRows];
    const int tid = threadIdx.x, lane = tid & 63;
    const int slice = blockIdx.x % A.slices;
    const int64_t rest = blockIdx.x / A.slices;
    const int chunk = (int)(rest % A.chunks);
    const int64_t w = rest / A.chunks;
    const int64_t first = w * A.window, n0 = first + (int64_t)chunk * A.rows_per_wg;
    const int64_t n1 = min(min(n0 + A.rows_per_wg, first + A.window), A.N);
    if (n0 >= n1) return;
    const int base = slice * SLICE, V = A.V;
    for (int i = tid; i < SLICE; i += kLogitThreads) { words[i] = 0; bias[i] = 0.f; }
    if (tid < kLogitRows) left[tid] = 0;
    __syncthreads();
    const uint32_t span = (uint32_t)min(SLICE, V - base);
    if (A.history_start) {
        const int64_t a = min(max(A.history_start[w], (int64_t)0), A.history_len);
        const int64_t b = min(max(A.history_start[w + 1], a), A.history_len);
        const int64_t prompt = A.prompt_len ? A.prompt_len[w] : 0;
        for (int64_t i = a + tid; i < b; i += kLogitThreads) {
            const uint32_t t = (uint32_t)A.history[i] - (uint32_t)base;
            if (t < span) {
                if (i - a < prompt) atomicOr(&words[t], kEver);
                else atomicAdd(&words[t], 1u);
            }
        }
    }
    if (A.drafted)
        for (int64_t i = first + tid; i < n0; i += kLogitThreads) {
            const uint32_t t = (uint32_t)A.drafted[i] - (uint32_t)base;
            if (t < span) atomicAdd(&words[t], 1u);
        }
    if (A.bias_start) {
        const int64_t a = min(max(A.bias_start[w], (int64_t)0), A.bias_len);
        const int64_t b = min(max(A.bias_start[w + 1], a), A.bias_len);
        // (equal tokens lie together: the first of them adds them up, in their order)
        for (int64_t i = a + tid; i < b; i += kLogitThreads) {
            const int id = A.bias_ids[i];
            const uint32_t t = (uint32_t)id - (uint32_t)base;
            if (t < span && (i == a || A.bias_ids[i - 1] != id)) {
                float v = A.bias_values[i];
                for (int64_t k = i + 1; k < b && A.bias_ids[k] == id; ++k) v += A.bias_values[k];
                bias[t] = v;
            }
        }
    }
    __syncthreads();
    const float theta = A.repetition ? A.repetition[w] : 1.f, often = A.frequency ? A.frequency[w] : 0.f;
    const float once = A.presence ? A.presence[w] : 0.f;
    const char* in = static_cast<const char*>(A.logits);
    char* out = static_cast<char*>(A.out);
    constexpr int ELT = 16 / EPV;
    for (int64_t n = n0; n < n1; ++n) {
        const uint8_t* mask = nullptr;
        if (A.allowed) {
            const int m = A.allowed_row[n];
            if (m >= 0) mask = reinterpret_cast<const uint8_t*>(A.allowed + (int64_t)min(m, A.mask_rows - 1) * A.allowed_stride);
        }
        int finite = 0;
#pragma unroll
        for (int u = 0; u < kLogitVecs; ++u) {
            const int at = (u * kLogitThreads + tid) * EPV, t0 = base + at;
            if (t0 >= V) continue;
            u32x4 x = *reinterpret_cast<const u32x4*>(in + (n * A.stride + t0) * ELT);
            uint32_t may = 0xffu;
            if (mask) may = EPV == 8 ? mask[t0 >> 3] : mask[t0 >> 3] >> (t0 & 4);
            float f[EPV];
            E::unpack(x, f);
            uint32_t word[EPV];
            float plus[EPV];
            bool any = false;
#pragma unroll
            for (int e = 0; e < EPV; ++e) {
                word[e] = words[at + e];
                plus[e] = bias[at + e];
                any |= word[e] != 0 || plus[e] != 0.f;
            }
            if (any) {
#pragma unroll
                for (int e = 0; e < EPV; ++e) {
                    const uint32_t c = word[e] & ~kEver;
                    if (word[e]) {
                        f[e] = f[e] > 0.f ? f[e] / theta : f[e] * theta;
                        f[e] = f[e] - often * (float)c;
                        f[e] = f[e] - (c ? once : 0.f);
                    }
                    f[e] += plus[e];
                }
            }
#pragma unroll
            for (int e = 0; e < EPV; ++e) {
                if (!(may >> e & 1u)) f[e] = -INFINITY;
                finite += t0 + e < V && (__float_as_uint(f[e]) & 0x7f800000u) != 0x7f800000u;
            }
            char* o = out + (n * A.out_stride + t0) * ELT;
            if constexpr (EPV == 4) {
                if (t0 + 4 <= V) *reinterpret_cast<u32x4*>(o) = u32x4{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
                else for (int e = 0; t0 + e < V; ++e) reinterpret_cast<float*>(o)[e] = f[e];
            } else {
                typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
                bf16x8 y;
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = (__bf16)f[e];
                if (t0 + 8 <= V) *reinterpret_cast<bf16x8*>(o) = y;
                else {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (t0 + e < V) reinterpret_cast<__bf16*>(o)[e] = y[e];
                }
            }
        }
        if (A.left) {
            for (int d = 1; d < 64; d <<= 1) finite += __shfl_xor(finite, d);
            if (lane == 0) atomicAdd(&left[n - n0], (uint32_t)finite);
        }
        if (A.drafted && n + 1 < n1) {
            const uint32_t t = (uint32_t)A.drafted[n] - (uint32_t)base;
            if (t < span && (int)(t / EPV) % kLogitThreads == tid) words[t] += 1;
        }
    }
    if (!A.left) return;
    __syncthreads();
    if (tid < (int)(n1 - n0)) {
        uint32_t sum = left[tid];
        if (A.slices == 1 || left_arrive(A.left_words + n0 + tid, A.tag, A.slices, left[tid], sum)) A.left[n0 + tid] = (int)sum;
    }
}

}  // namespace

hipError_t launch_adjust(int dtype, LogitArgs args, hipStream_t stream)
{
    if (args.N <= 0) return hipSuccess;
    const int slice = kLogitThreads * kLogitVecs * (dtype == 0 ? 4 : 8);
    args.slices = (args.V + slice - 1) / slice;
    const int64_t windows = (args.N + args.window - 1) / args.window;
    const int64_t longest = args.window < args.N ? args.window : args.N;
    args.rows_per_wg = (int)(longest < 8 ? longest : 8);
    args.chunks = (int)((longest + args.rows_per_wg - 1) / args.rows_per_wg);
    const int64_t grid = windows * args.chunks * args.slices;
    if (grid > 0x7fffffffLL) return hipErrorInvalidConfiguration;
    if (dtype == 0) hipLaunchKernelGGL(adjust_kernel<float>, dim3((unsigned)grid), dim3(kLogitThreads), 0, stream, args);
    else hipLaunchKernelGGL(adjust_kernel<bf16_t>, dim3((unsigned)grid), dim3(kLogitThreads), 0, stream, args);
    return hipGetLastError();
}

}  // namespace ciar
