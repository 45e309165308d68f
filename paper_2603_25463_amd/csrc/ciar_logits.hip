// gfx950 kernel of the logits' adjustments (ciar_adjust_logits in include/ciar.h): penalties for tokens that have come before,
// biases, grammar masks.
#include "ciar_device.h"
#include "ciar_step.h"

namespace ciar {
namespace {

// A workgroup takes a slice of the vocabulary for rows of one window: what the window's rows share (its history, its biases) is
// counted once into two words of LDS per token of the slice, then the rows stream by, each requested while the one before it is worked
// on.  Row n of a window sees the drafted tokens before it: they are added to the counts one by one between the rows, each by the lane
// whose vector the token lies in, so that no barrier separates rows.  A lane knows which of its vectors hold a token that anything
// concerns (a bit each): the others, which are most, go through as bits, masked, with a look for values that are not finite.
constexpr int kLogitThreads = 256, kLogitVecs = 2;             // vectors of 16 bytes per lane: a slice is 2048 fp32 or 4096 bf16 tokens
constexpr int kLogitRows = 64;                                 // most rows of a workgroup
constexpr uint32_t kEver = 0x80000000u;                        // the token has come up; below: how often behind the prompt

__device__ __forceinline__ int wave_sum_int(int v)
{
    v += dpp_or<kRowShr1, 0xf>(0, v);
    v += dpp_or<kRowShr2, 0xf>(0, v);
    v += dpp_or<kRowShr4, 0xf>(0, v);
    v += dpp_or<kRowShr8, 0xf>(0, v);
    v += dpp_or<kRowBcast15, 0xa>(0, v);
    v += dpp_or<kRowBcast31, 0xc>(0, v);
    return __builtin_amdgcn_readlane(v, 63);
}

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

// What the kernel does with a vector's 16 bytes.
template <typename T> struct LogitVec;
template <> struct LogitVec<float> {
    static constexpr int kPerVec = 4;
    static __device__ __forceinline__ void unpack(const u32x4& r, float* f) { Elt<float>::unpack(r, f); }
    static __device__ __forceinline__ u32x4 pack(const float* f)
    {
        return {__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
    }
    static __device__ __forceinline__ u32x4 masked(u32x4 r, uint32_t bits)
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) r[e] = bits >> e & 1u ? r[e] : 0xff800000u;
        return r;
    }
    static __device__ __forceinline__ int count_finite(const u32x4& r)
    {
        int n = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) n += (r[e] & 0x7f800000u) != 0x7f800000u;
        return n;
    }
    static __device__ __forceinline__ bool any_not_finite(const u32x4& r) { return count_finite(r) != 4; }
    static __device__ __forceinline__ void store_some(char* o, const u32x4& r, int n)
    {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < n) reinterpret_cast<uint32_t*>(o)[e] = r[e];
    }
};
template <> struct LogitVec<bf16_t> {
    static constexpr int kPerVec = 8;
    static __device__ __forceinline__ void unpack(const u32x4& r, float* f) { Elt<bf16_t>::unpack(r, f); }
    static __device__ __forceinline__ u32x4 pack(const float* f)
    {
        typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
        bf16x8 y;
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = (__bf16)f[e];
        return __builtin_bit_cast(u32x4, y);
    }
    static __device__ __forceinline__ u32x4 masked(u32x4 r, uint32_t bits)
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t lo = bits >> (2 * e) & 1u ? 0xffffu : 0u, hi = bits >> (2 * e + 1) & 1u ? 0xffff0000u : 0u;
            r[e] = (r[e] & (lo | hi)) | (0xff80ff80u & ~(lo | hi));
        }
        return r;
    }
    static __device__ __forceinline__ int count_finite(const u32x4& r)
    {
        int n = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) n += ((r[e] & 0x7f80u) != 0x7f80u) + ((r[e] & 0x7f800000u) != 0x7f800000u);
        return n;
    }
    // (the exponents of a word's two values, plus one each: bit 15 and bit 31 come up where they were all ones)
    static __device__ __forceinline__ bool any_not_finite(const u32x4& r)
    {
        uint32_t any = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) any |= (r[e] & 0x7f807f80u) + 0x00800080u;
        return (any & 0x80008000u) != 0;
    }
    static __device__ __forceinline__ void store_some(char* o, const u32x4& r, int n)
    {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n) reinterpret_cast<uint16_t*>(o)[e] = (uint16_t)(r[e / 2] >> (16 * (e & 1)));
    }
};

template <typename T>
__global__ __launch_bounds__(kLogitThreads) void adjust_kernel(const LogitArgs A)
{
    using E = LogitVec<T>;
    constexpr int EPV = E::kPerVec, SLICE = kLogitThreads * kLogitVecs * EPV;
    __shared__ __attribute__((aligned(16))) uint32_t words[SLICE];
    __shared__ __attribute__((aligned(16))) float bias[SLICE];
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
    {
        const u32x4 none = {0, 0, 0, 0};
        for (int i = 4 * tid; i < SLICE; i += 4 * kLogitThreads) {
            *reinterpret_cast<u32x4*>(&words[i]) = none;
            *reinterpret_cast<u32x4*>(&bias[i]) = none;
        }
    }
    if (tid < kLogitRows) left[tid] = 0;
    const char* in = static_cast<const char*>(A.logits);
    char* out = static_cast<char*>(A.out);
    constexpr int ELT = 16 / EPV;
    int at[kLogitVecs];
    bool there[kLogitVecs];
#pragma unroll
    for (int u = 0; u < kLogitVecs; ++u) {
        at[u] = (u * kLogitThreads + tid) * EPV;
        there[u] = base + at[u] < V;
    }
    u32x4 x[kLogitVecs];
    uint32_t may[kLogitVecs];                                  // the vector's mask bits
    auto request = [&](int64_t n) {
        const uint8_t* mask = nullptr;
        if (A.allowed) {
            const int m = A.allowed_row[n];
            if (m >= 0) mask = reinterpret_cast<const uint8_t*>(A.allowed + (int64_t)min(m, A.mask_rows - 1) * A.allowed_stride);
        }
#pragma unroll
        for (int u = 0; u < kLogitVecs; ++u) {
            may[u] = ~0u;
            if (!there[u]) continue;
            const int t0 = base + at[u];
            x[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(in + (n * A.stride + t0) * ELT));
            if (mask) may[u] = EPV == 8 ? mask[t0 >> 3] : mask[t0 >> 3] >> (t0 & 4);
        }
    };
    request(n0);
    __syncthreads();
    const uint32_t span = (uint32_t)min(SLICE, V - base);
    if (A.history_start) {
        const int64_t a = min(max(A.history_start[w], (int64_t)0), A.history_len);
        const int64_t b = min(max(A.history_start[w + 1], a), A.history_len);
        const int64_t prompt = A.prompt_len ? A.prompt_len[w] : 0;
        constexpr int AT_ONCE = 8;
        for (int64_t i = a + tid; i < b; i += AT_ONCE * kLogitThreads) {
            int id[AT_ONCE];
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) id[k] = i + k * kLogitThreads < b ? A.history[i + k * kLogitThreads] : -1;
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) {
                const uint32_t t = (uint32_t)id[k] - (uint32_t)base;
                if (id[k] >= 0 && t < span) {
                    if (i + k * kLogitThreads - a < prompt) atomicOr(&words[t], kEver);
                    else atomicAdd(&words[t], 1u);
                }
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
    const float theta = A.repetition ? A.repetition[w] : 1.f, often = A.frequency ? A.frequency[w] : 0.f;
    const float once = A.presence ? A.presence[w] : 0.f;
    __syncthreads();
    uint32_t concerned = 0;                                    // bit u: vector u has tokens with a count or a bias
#pragma unroll
    for (int u = 0; u < kLogitVecs; ++u)
#pragma unroll
        for (int e = 0; e < EPV; ++e)
            if (words[at[u] + e] != 0 || bias[at[u] + e] != 0.f) concerned |= 1u << u;
    for (int64_t n = n0; n < n1; ++n) {
        int finite = 0;
        u32x4 y[kLogitVecs];
#pragma unroll
        for (int u = 0; u < kLogitVecs; ++u) {
            if (!there[u]) continue;
            const int t0 = base + at[u];
            const uint32_t valid = t0 + EPV <= V ? (1u << EPV) - 1u : (1u << (V - t0)) - 1u, bits = may[u] & valid;
            if (concerned >> u & 1u) {
                float f[EPV];
                E::unpack(x[u], f);
#pragma unroll
                for (int e = 0; e < EPV; ++e) {
                    const uint32_t word = words[at[u] + e], c = word & ~kEver;
                    if (word) {
                        f[e] = f[e] > 0.f ? f[e] / theta : f[e] * theta;
                        f[e] = f[e] - often * (float)c;
                        f[e] = f[e] - (c ? once : 0.f);
                    }
                    f[e] += bias[at[u] + e];
                    if (!(bits >> e & 1u)) f[e] = -INFINITY;
                    finite += (__float_as_uint(f[e]) & 0x7f800000u) != 0x7f800000u;
                }
                y[u] = E::pack(f);
            } else {
                y[u] = E::masked(x[u], bits);
                finite += E::any_not_finite(x[u]) ? E::count_finite(y[u]) : __popc(bits);
            }
        }
        if (n + 1 < n1) request(n + 1);
#pragma unroll
        for (int u = 0; u < kLogitVecs; ++u) {
            if (!there[u]) continue;
            const int t0 = base + at[u];
            char* o = out + (n * A.out_stride + t0) * ELT;
            if (t0 + EPV <= V) __builtin_nontemporal_store(y[u], reinterpret_cast<u32x4*>(o));
            else E::store_some(o, y[u], V - t0);
        }
        if (A.left) {
            finite = wave_sum_int(finite);
            if (lane == 0) atomicAdd(&left[n - n0], (uint32_t)finite);
        }
        if (A.drafted && n + 1 < n1) {
            const uint32_t t = (uint32_t)A.drafted[n] - (uint32_t)base;
            if (t < span && (int)(t / EPV) % kLogitThreads == tid) {
                words[t] += 1;
                concerned |= 1u << (t / EPV / kLogitThreads);
            }
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
    // Rows of a workgroup: a whole window (up to 64 rows: its history is counted once for all of them) where that still makes four
    // workgroups a compute unit, fewer where it does not.
    const int64_t wanted = windows * args.slices * longest / (4 * (int64_t)compute_units());
    const int64_t most = longest < kLogitRows ? longest : kLogitRows;
    args.rows_per_wg = (int)(wanted < 1 ? 1 : wanted < most ? wanted : most);
    args.chunks = (int)((longest + args.rows_per_wg - 1) / args.rows_per_wg);
    const int64_t grid = windows * args.chunks * args.slices;
    if (grid > 0x7fffffffLL) return hipErrorInvalidConfiguration;
    if (dtype == 0) hipLaunchKernelGGL(adjust_kernel<float>, dim3((unsigned)grid), dim3(kLogitThreads), 0, stream, args);
    else hipLaunchKernelGGL(adjust_kernel<bf16_t>, dim3((unsigned)grid), dim3(kLogitThreads), 0, stream, args);
    return hipGetLastError();
}

}  // namespace ciar
