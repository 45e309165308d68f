// gfx950 kernels of the attention over the paged cache (ciar_paged_attention in include/ciar.h).
#include "ciar_device.h"
#include "ciar_step.h"

namespace ciar {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2f = 0.69314718055994530942f;

// 16 bytes from anywhere (rows of q lie where the caller has them).
__device__ __forceinline__ u32x4 load16_any(const void* p)
{
    u32x4 v;
    __builtin_memcpy(&v, p, 16);
    return v;
}

// The new tokens of a request and what they see.
struct Request {
    int begin, n, base, len;           // first row, rows, position of the first new token (may be negative), tokens in the cache
};
__device__ __forceinline__ Request request_of(const AttentionArgs& A, int r)
{
    Request q;
    q.begin = min(max(A.cu_new[r], 0), A.T);
    const int end = min(max(A.cu_new[r + 1], q.begin), A.T);
    q.n = min(end - q.begin, A.max_new);
    q.len = min(max(A.kv_len[r], 0), A.max_len);
    q.base = q.len - q.n;
    return q;
}

// Rows that belong to no request: nothing seen.
__device__ void fill_unclaimed(const AttentionArgs& A, int64_t from, int64_t step)
{
    const int first = min(max(A.cu_new[0], 0), A.T), last = min(max(A.cu_new[A.R], first), A.T);
    const int64_t per = (int64_t)A.q_heads * A.D, rows = first + (A.T - last);
    for (int64_t i = from; i < rows * per; i += step) {
        const int64_t row = i / per, t = row < first ? row : row - first + last;
        const int h = (int)((i - row * per) / A.D), d = (int)(i - row * per - (int64_t)h * A.D);
        ((uint16_t*)A.out.p)[t * A.out.token + h * A.out.head + d] = 0;
        if (d == 0 && A.lse) A.lse[t * A.q_heads + h] = -INFINITY;
    }
}

// One wave per sixteen rows (a row: a new token and a query head of the key head's group; heads of a token side by side) and key head.
// Scores as S^T = K Q^T, so that a lane's accumulators belong to one row (l % 16): the running maximum and sum, and the rescaling of
// the output, stay in the lane, four lanes of a row meet in two shuffles.  Two products of 16 tokens make a step of 32, their tokens
// chosen so that a lane's eight weights are eight consecutive tokens, which is how the second product wants them: the first takes
// tokens 8 g .. 8 g + 3 as its rows 4 g ..., the second 8 g + 4 .. 8 g + 7.
template <int D>
__global__ __launch_bounds__(64) void attention_kernel(const AttentionArgs A, int tiles, int64_t work)
{
    const int lane = threadIdx.x, col = lane & 15, grp = lane >> 4;
    if ((int64_t)blockIdx.x >= work) {
        fill_unclaimed(A, ((int64_t)blockIdx.x - work) * 64 + lane, ((int64_t)gridDim.x - work) * 64);
        return;
    }
    const int tile = blockIdx.x % tiles, h = (blockIdx.x / tiles) % A.kv_heads, r = blockIdx.x / tiles / A.kv_heads;
    const int g = A.q_heads / A.kv_heads;
    const Request R = request_of(A, r);
    const int rows = R.n * g, m0 = tile * 16;
    if (m0 >= rows) return;
    const int m = min(m0 + col, rows - 1), j = m / g, head = h * g + (m - j * g);
    const int seen = min(max(R.base + j + 1, 0), R.len);                          // tokens that this lane's row sees
    const int most = min(max(R.base + min(m0 + 15, rows - 1) / g + 1, 0), R.len); // and the tile's last row
    const int least = min(max(R.base + m0 / g + 1, 0), R.len);
    bf16x8 q[D / 32];
    const uint16_t* qrow = static_cast<const uint16_t*>(A.q.p) + (int64_t)(R.begin + j) * A.q.token + (int64_t)head * A.q.head;
#pragma unroll
    for (int k = 0; k < D / 32; ++k) q[k] = __builtin_bit_cast(bf16x8, load16_any(qrow + 32 * k + 8 * grp));
    f32x4 acc[D / 16];
#pragma unroll
    for (int b = 0; b < D / 16; ++b) acc[b] = {0.f, 0.f, 0.f, 0.f};
    float top = -INFINITY, total = 0.f;
    const float scale = A.scale * kLog2e;
    const int64_t head_bytes = (int64_t)A.page * D * 2;
    auto atom_at = [&](int token) -> int64_t {                                    // byte offset of the atom that holds a token
        const int page = token / A.page;
        const int p = min(max(A.table[(int64_t)r * A.table_stride + page], 0), A.pages - 1);
        return ((int64_t)p * A.kv_heads + h) * head_bytes + (int64_t)(token - page * A.page) / kAtom * (kAtom * D * 2);
    };
    for (int t0 = 0; t0 < most; t0 += 32) {
        const int64_t a0 = atom_at(t0), a1 = t0 + 16 < most ? atom_at(t0 + 16) : a0;
        const char* kp = static_cast<const char*>(A.k_cache) + (col < 8 ? a0 : a1) + ((col >> 2 & 1) * 8 + (col & 3)) * 16;
        f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = s0;
#pragma unroll
        for (int k = 0; k < D / 32; ++k) {
            const char* p = kp + (4 * k + grp) * 256;
            s0 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*reinterpret_cast<const bf16x8*>(p), q[k], s0, 0, 0, 0);
            s1 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*reinterpret_cast<const bf16x8*>(p + 64), q[k], s1, 0, 0, 0);
        }
        float s[8];
        float high = -INFINITY;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            s[e] = t0 + 8 * grp + e < seen ? (e < 4 ? s0[e & 3] : s1[e & 3]) * scale : -INFINITY;
            high = fmaxf(high, s[e]);
        }
        high = fmaxf(high, __shfl_xor(high, 16));
        high = fmaxf(high, __shfl_xor(high, 32));
        const float now = fmaxf(top, high), ref = now == -INFINITY ? 0.f : now;
        const float keep = __builtin_amdgcn_exp2f(top - ref);
        top = now;
        float sum = 0.f;
        bf16x8 w;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float p = __builtin_amdgcn_exp2f(s[e] - ref);
            sum += p;
            w[e] = (__bf16)p;
        }
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        total = total * keep + sum;
#pragma unroll
        for (int b = 0; b < D / 16; ++b) acc[b] *= keep;
        const char* vp = static_cast<const char*>(A.v_cache) + (grp < 2 ? a0 : a1) + ((grp & 1) * D + col) * 16;
        const bool edge = t0 + 32 > least;
        if (!edge) {
#pragma unroll
            for (int b = 0; b < D / 16; ++b)
                acc[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*reinterpret_cast<const bf16x8*>(vp + b * 256), w, acc[b], 0, 0, 0);
            continue;
        }
        // Where rows see different tokens, a value that is no number must not reach the rows that do not see it (0 * inf).
        // Values that no row sees are taken as zeros; if one is left that is not finite, the tokens go in one by one.
        auto value = [&](int b) -> bf16x8 {
            u32x4 v = *reinterpret_cast<const u32x4*>(vp + b * 256);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (t0 + 8 * grp + e >= most) v[e / 2] &= e & 1 ? 0x0000ffffu : 0xffff0000u;
            return __builtin_bit_cast(bf16x8, v);
        };
        bool bad = false;
#pragma unroll
        for (int b = 0; b < D / 16; ++b) {
            const u32x4 v = __builtin_bit_cast(u32x4, value(b));
#pragma unroll
            for (int e = 0; e < 4; ++e) bad |= (v[e] & 0x7f80u) == 0x7f80u || (v[e] & 0x7f800000u) == 0x7f800000u;
        }
        if (!__any(bad)) {
#pragma unroll
            for (int b = 0; b < D / 16; ++b) acc[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(value(b), w, acc[b], 0, 0, 0);
        } else {
            for (int i = 0; i < 32 && t0 + i < most; ++i) {
                bf16x8 one = w;
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (i != 8 * grp + e) one[e] = (__bf16)0.f;
#pragma unroll
                for (int b = 0; b < D / 16; ++b) {
                    u32x4 v = __builtin_bit_cast(u32x4, value(b));
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (i != 8 * grp + e) v[e / 2] &= e & 1 ? 0x0000ffffu : 0xffff0000u;
                    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
                    const f32x4 x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v), one, zero, 0, 0, 0);
                    if (t0 + i < seen) acc[b] += x;
                }
            }
        }
    }
    if (m0 + col >= rows) return;
    const float inv = total == 0.f ? 0.f : 1.f / total;
    __bf16* orow = (__bf16*)A.out.p + (int64_t)(R.begin + j) * A.out.token + (int64_t)head * A.out.head;
#pragma unroll
    for (int b = 0; b < D / 16; ++b)
#pragma unroll
        for (int v = 0; v < 4; ++v) orow[16 * b + 4 * grp + v] = (__bf16)(acc[b][v] * inv);
    if (grp == 0 && A.lse)
        A.lse[(int64_t)(R.begin + j) * A.q_heads + head] = total == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(total)) * kLn2f;
}

}  // namespace

size_t attention_workspace(const AttentionArgs&) { return 0; }

hipError_t launch_attention(const AttentionArgs& args, void*, hipStream_t stream)
{
    if (args.T <= 0) return hipSuccess;
    const int g = args.q_heads / args.kv_heads;
    const int64_t tiles = ((int64_t)args.max_new * g + 15) / 16, work = tiles * args.kv_heads * args.R;
    const int64_t grid = work + 32;
    if (grid > 0x7fffffffLL) return hipErrorInvalidConfiguration;
    switch (args.D) {
#define CIAR_CASE(d) case d: hipLaunchKernelGGL(attention_kernel<d>, dim3((unsigned)grid), dim3(64), 0, stream, args, (int)(tiles > 0 ? tiles : 1), work); break;
        CIAR_CASE(32) CIAR_CASE(64) CIAR_CASE(96) CIAR_CASE(128) CIAR_CASE(160) CIAR_CASE(192) CIAR_CASE(224) CIAR_CASE(256)
#undef CIAR_CASE
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

}  // namespace ciar
