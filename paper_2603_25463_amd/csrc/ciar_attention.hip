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

// What a workgroup works on.
struct Unit {
    int r, h, block, split;            // request, key head, block of rows, part of the tokens
};

// Which page an atom of a request lies in: atom / (page / 16) for any page size, as a multiplication (2 atom < 2^32; the
// multiplier is 2^(31 + shift) / (page / 16) rounded up, with 2^shift >= page / 16, which is exact for every atom below 2^31).
struct Pages {
    uint32_t mul, shift, per;          // per: atoms of a page
};
Pages pages_of(int page)
{
    Pages p;
    p.per = (uint32_t)(page / kAtom);
    p.shift = 0;
    while ((1u << p.shift) < p.per) ++p.shift;
    p.mul = (uint32_t)(((1ull << (31 + p.shift)) + p.per - 1) / p.per);
    return p;
}

constexpr int kSteps = 32;             // tokens of a step: two atoms
constexpr float kSlack = 8.f;          // binary orders that a row's weights may grow beyond the reference before it is moved

// ---- few rows to a key head: the cache streams by once ----------------------------------------------------------------------
//
// A workgroup of four waves takes up to 16 RT rows (a row: a new token and a query head of the key head's group; heads of a token
// side by side) of one request and key head, and a part of its tokens.  The waves deal the part's steps of 32 tokens among
// themselves, each with all the rows and a softmax of its own; keys and values go from memory into the registers that the matrix
// instructions take them from (the cache is laid out for that), requested a step ahead, through no LDS and past no barrier: what
// bounds this kernel is memory.  At the end the waves' rows meet in LDS.
//
// Scores as S^T = K Q^T: a lane's accumulators belong to one row (l % 16), so that reference, sum and the rescaling of the output
// stay in the lane.  Two products of 16 tokens make a step, their tokens chosen so that a lane's eight weights are eight
// consecutive tokens, as the second product (O^T = V^T P^T) wants them: the first takes tokens 8 g .. 8 g + 3 of the step as its rows
// 4 g ..., the second 8 g + 4 ....  The reference of a row moves only where a score exceeds it by more than kSlack: a vote of
// the wave, where a maximum over the row's four lanes and a rescaling of the output would be made each time.
template <int D, int RT>
__global__ __launch_bounds__(256) void few_rows_kernel(const AttentionArgs A, const Pages P, int blocks, int splits, int64_t work,
                                                       float* __restrict__ part_o, float2* __restrict__ part_s)
{
    constexpr int ROWF = D + 4;                                    // floats of a row in LDS
    __shared__ float meet[4][16][ROWF];
    __shared__ float2 stats[4][RT * 16];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 15, grp = lane >> 4;
    if ((int64_t)blockIdx.x >= work) {
        fill_unclaimed(A, ((int64_t)blockIdx.x - work) * 256 + tid, ((int64_t)gridDim.x - work) * 256);
        return;
    }
    Unit u;
    {
        int i = blockIdx.x;
        u.split = i % splits; i /= splits;
        u.block = i % blocks; i /= blocks;
        u.h = i % A.kv_heads;
        u.r = i / A.kv_heads;
    }
    const int g = A.q_heads / A.kv_heads;
    const Request R = request_of(A, u.r);
    const int rows = R.n * g, m0 = u.block * 16 * RT;
    if (m0 >= rows) return;
    const int most = min(max(R.base + min(m0 + 16 * RT - 1, rows - 1) / g + 1, 0), R.len);        // what the last row sees
    const int least = min(max(R.base + m0 / g + 1, 0), R.len);                                    // and the first
    const int steps = (most + kSteps - 1) / kSteps, each = (steps + splits - 1) / splits;
    const int first = u.split * each, last = min(first + each, steps);
    if (first >= last && u.split > 0) return;                      // (a row that sees nothing is the first part's)

    bf16x8 q[RT][D / 32];
    f32x4 acc[RT][D / 16];
    float ref[RT], total[RT];
    int seen[RT];
#pragma unroll
    for (int i = 0; i < RT; ++i) {
        const int m = min(m0 + 16 * i + col, rows - 1), j = m / g, head = u.h * g + (m - j * g);
        seen[i] = min(max(R.base + j + 1, 0), R.len);
        const uint16_t* qrow = static_cast<const uint16_t*>(A.q.p) + (int64_t)(R.begin + j) * A.q.token + (int64_t)head * A.q.head;
#pragma unroll
        for (int k = 0; k < D / 32; ++k) q[i][k] = __builtin_bit_cast(bf16x8, load16_any(qrow + 32 * k + 8 * grp));
#pragma unroll
        for (int b = 0; b < D / 16; ++b) acc[i][b] = {0.f, 0.f, 0.f, 0.f};
        ref[i] = -INFINITY;
        total[i] = 0.f;
    }
    const float scale = A.scale * kLog2e;
    const int64_t head_bytes = (int64_t)A.page * D * 2;
    const int32_t* row = A.table + (int64_t)u.r * A.table_stride;
    const int atoms = (most + kAtom - 1) / kAtom;
    auto atom_at = [&](int atom) -> int64_t {                      // byte offset of an atom of the request
        const uint32_t a = (uint32_t)min(atom, atoms - 1), page = __umulhi(2 * a, P.mul) >> P.shift;
        const int p = min(max(row[page], 0), A.pages - 1);
        return ((int64_t)p * A.kv_heads + u.h) * head_bytes + (int64_t)(a - page * P.per) * (kAtom * D * 2);
    };
    // this lane's keys and values of a step
    const int koff = ((col >> 2 & 1) * 8 + (col & 3)) * 16 + grp * 256, voff = ((grp & 1) * D + col) * 16;
    bf16x8 k0[D / 32], k1[D / 32], v[D / 16];
    auto load_keys = [&](int64_t a0, int64_t a1) {
        const char* p = static_cast<const char*>(A.k_cache) + (col < 8 ? a0 : a1) + koff;
#pragma unroll
        for (int k = 0; k < D / 32; ++k) {
            k0[k] = *reinterpret_cast<const bf16x8*>(p + k * 1024);
            k1[k] = *reinterpret_cast<const bf16x8*>(p + k * 1024 + 64);
        }
    };
    auto load_values = [&](int64_t a0, int64_t a1) {
        const char* p = static_cast<const char*>(A.v_cache) + (grp < 2 ? a0 : a1) + voff;
#pragma unroll
        for (int b = 0; b < D / 16; ++b) v[b] = *reinterpret_cast<const bf16x8*>(p + b * 256);
    };
    if (first + wave < last) {
        int step = first + wave;
        int64_t a0 = atom_at(2 * step), a1 = atom_at(2 * step + 1);
        load_keys(a0, a1);
        load_values(a0, a1);
        int64_t n0 = atom_at(2 * (step + 4)), n1 = atom_at(2 * (step + 4) + 1);
        for (; step < last; step += 4) {
            const int t0 = step * kSteps;
            f32x4 s0[RT], s1[RT];
#pragma unroll
            for (int i = 0; i < RT; ++i) s0[i] = s1[i] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < D / 32; ++k)
#pragma unroll
                for (int i = 0; i < RT; ++i) {
                    s0[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k0[k], q[i][k], s0[i], 0, 0, 0);
                    s1[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k1[k], q[i][k], s1[i], 0, 0, 0);
                }
            // the next step's keys, into the registers that have just been read (past the part's end: the last atom's again)
            a0 = n0; a1 = n1;
            load_keys(a0, a1);
            n0 = atom_at(2 * (step + 8)); n1 = atom_at(2 * (step + 8) + 1);
            const bool edge = t0 + kSteps > least;
            bf16x8 w[RT];
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                float s[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) s[e] = (e < 4 ? s0[i][e & 3] : s1[i][e & 3]) * scale;
                if (edge) {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (t0 + 8 * grp + e >= seen[i]) s[e] = -INFINITY;
                }
                float high = fmaxf(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])), fmaxf(fmaxf(s[4], s[5]), fmaxf(s[6], s[7])));
                if (__any(high > ref[i] + kSlack)) {
                    high = fmaxf(high, __shfl_xor(high, 16));
                    high = fmaxf(high, __shfl_xor(high, 32));
                    const float now = fmaxf(ref[i], high);
                    const float keep = now == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(ref[i] - now);
                    ref[i] = now;
                    total[i] *= keep;
#pragma unroll
                    for (int b = 0; b < D / 16; ++b) acc[i][b] *= keep;
                }
                const float sub = ref[i] == -INFINITY ? 0.f : ref[i];
                float sum = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float p = __builtin_amdgcn_exp2f(s[e] - sub);
                    sum += p;
                    w[i][e] = (__bf16)p;
                }
                total[i] += sum;                                   // (of this lane's tokens; the row's lanes meet at the end)
            }
            if (edge) {
                // Where rows see different tokens, a value that is no number must not reach the rows that do not see it (0 * inf).
                // Values that no row sees are taken as zeros; if one is left that is not finite, the tokens go in one by one.
                bool bad = false;
#pragma unroll
                for (int b = 0; b < D / 16; ++b) {
                    u32x4 x = __builtin_bit_cast(u32x4, v[b]);
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (t0 + 8 * grp + e >= most) x[e / 2] &= e & 1 ? 0x0000ffffu : 0xffff0000u;
#pragma unroll
                    for (int e = 0; e < 4; ++e) bad |= (x[e] & 0x7f80u) == 0x7f80u || (x[e] & 0x7f800000u) == 0x7f800000u;
                    v[b] = __builtin_bit_cast(bf16x8, x);
                }
                if (__any(bad)) {
#pragma unroll 1
                    for (int t = 0; t < kSteps && t0 + t < most; ++t) {
#pragma unroll
                        for (int i = 0; i < RT; ++i) {
                            bf16x8 one = w[i];
#pragma unroll
                            for (int e = 0; e < 8; ++e)
                                if (t != 8 * grp + e) one[e] = (__bf16)0.f;
#pragma unroll
                            for (int b = 0; b < D / 16; ++b) {
                                u32x4 x = __builtin_bit_cast(u32x4, v[b]);
#pragma unroll
                                for (int e = 0; e < 8; ++e)
                                    if (t != 8 * grp + e) x[e / 2] &= e & 1 ? 0x0000ffffu : 0xffff0000u;
                                const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
                                const f32x4 y = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), one, zero, 0, 0, 0);
                                if (t0 + t < seen[i]) acc[i][b] += y;
                            }
                        }
                    }
                    load_values(a0, a1);
                    continue;
                }
            }
#pragma unroll
            for (int b = 0; b < D / 16; ++b)
#pragma unroll
                for (int i = 0; i < RT; ++i) acc[i][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[b], w[i], acc[i][b], 0, 0, 0);
            load_values(a0, a1);
        }
    }
    // the waves' rows meet, sixteen at a time
#pragma unroll
    for (int i = 0; i < RT; ++i) {
        total[i] += __shfl_xor(total[i], 16);
        total[i] += __shfl_xor(total[i], 32);
        if (grp == 0) stats[wave][16 * i + col] = {ref[i], total[i]};
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < RT; ++i) {
        if (m0 + 16 * i >= rows) break;                            // (uniform)
        float high = -INFINITY;
#pragma unroll
        for (int x = 0; x < 4; ++x) high = fmaxf(high, stats[x][16 * i + col].x);
        const float mine = high == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ref[i] - high);
#pragma unroll
        for (int b = 0; b < D / 16; ++b) *reinterpret_cast<f32x4*>(&meet[wave][col][16 * b + 4 * grp]) = acc[i][b] * mine;
        __syncthreads();
        const int mr = tid >> 4, m = m0 + 16 * i + mr;             // sixteen threads to a row
        if (m < rows) {
            float top = -INFINITY, sum = 0.f;
#pragma unroll
            for (int x = 0; x < 4; ++x) top = fmaxf(top, stats[x][16 * i + mr].x);
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const float2 s = stats[x][16 * i + mr];
                sum += top == -INFINITY ? s.y : s.y * __builtin_amdgcn_exp2f(s.x - top);
            }
            const int j = m / g, head = u.h * g + (m - j * g);
            const int64_t t = R.begin + j;
            if (splits == 1) {
                const float inv = sum == 0.f ? 0.f : 1.f / sum;
                __bf16* o = (__bf16*)A.out.p + t * A.out.token + (int64_t)head * A.out.head;
                for (int d = (tid & 15) * 2; d < D; d += 32) {
                    float x = 0.f, y = 0.f;
#pragma unroll
                    for (int z = 0; z < 4; ++z) { x += meet[z][mr][d]; y += meet[z][mr][d + 1]; }
                    o[d] = (__bf16)(x * inv);
                    o[d + 1] = (__bf16)(y * inv);
                }
                if ((tid & 15) == 0 && A.lse) A.lse[t * A.q_heads + head] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2f;
            } else {
                const int64_t at = ((int64_t)u.split * A.T + t) * A.q_heads + head;
                for (int d = (tid & 15) * 4; d < D; d += 64) {
                    f32x4 x = *reinterpret_cast<const f32x4*>(&meet[0][mr][d]);
#pragma unroll
                    for (int z = 1; z < 4; ++z) x += *reinterpret_cast<const f32x4*>(&meet[z][mr][d]);
                    *reinterpret_cast<f32x4*>(part_o + at * D + d) = x;
                }
                if ((tid & 15) == 0) part_s[at] = {top, sum};
            }
        }
        __syncthreads();
    }
}

// The parts' rows meet: one workgroup per row; D / 4 threads to a part.
template <int D>
__global__ __launch_bounds__(256) void join_kernel(const AttentionArgs A, int blocks, int rows_per_block, int splits,
                                                   const float* __restrict__ part_o, const float2* __restrict__ part_s)
{
    constexpr int TPR = D / 4, AT_ONCE = 256 / TPR;
    __shared__ f32x4 sums[AT_ONCE][TPR];
    __shared__ float wave_top[4], wave_sum[4];
    const int tid = threadIdx.x;
    int i = blockIdx.x;
    const int mr = i % rows_per_block; i /= rows_per_block;
    const int block = i % blocks; i /= blocks;
    const int h = i % A.kv_heads, r = i / A.kv_heads;
    const int g = A.q_heads / A.kv_heads;
    const Request R = request_of(A, r);
    const int rows = R.n * g, m0 = block * rows_per_block, m = m0 + mr;
    if (m >= rows) return;
    const int most = min(max(R.base + min(m0 + rows_per_block - 1, rows - 1) / g + 1, 0), R.len);
    const int steps = (most + kSteps - 1) / kSteps, each = (steps + splits - 1) / splits;
    const int parts = each > 0 ? (steps + each - 1) / each : 1;    // those that have written
    const int j = m / g, head = h * g + (m - j * g);
    const int64_t t = R.begin + j, at = t * A.q_heads + head, step = (int64_t)A.T * A.q_heads;
    float top = -INFINITY;
    for (int s = tid; s < parts; s += 256) top = fmaxf(top, part_s[at + s * step].x);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
    if ((tid & 63) == 0) wave_top[tid >> 6] = top;
    __syncthreads();
    top = fmaxf(fmaxf(wave_top[0], wave_top[1]), fmaxf(wave_top[2], wave_top[3]));
    float sum = 0.f;
    for (int s = tid; s < parts; s += 256) {
        const float2 x = part_s[at + s * step];
        sum += top == -INFINITY ? x.y : x.y * __builtin_amdgcn_exp2f(x.x - top);
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d);
    if ((tid & 63) == 0) wave_sum[tid >> 6] = sum;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    const int c = tid % TPR, s0 = tid / TPR;
    if (s0 < AT_ONCE)
        for (int s = s0; s < parts; s += AT_ONCE) {
            const float f = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(part_s[at + s * step].x - top);
            o += *reinterpret_cast<const f32x4*>(part_o + (at + s * step) * D + 4 * c) * f;
        }
    if (s0 < AT_ONCE) sums[s0][c] = o;
    __syncthreads();
    if (tid >= TPR) return;
    sum = (wave_sum[0] + wave_sum[1]) + (wave_sum[2] + wave_sum[3]);
    o = sums[0][tid];
    for (int s = 1; s < AT_ONCE; ++s) o += sums[s][tid];
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    __bf16* y = (__bf16*)A.out.p + t * A.out.token + (int64_t)head * A.out.head + 4 * tid;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = (__bf16)(o[e] * inv);
    if (tid == 0 && A.lse) A.lse[at] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2f;
}

// How a call is laid out: rows of a workgroup (16 rt), blocks of rows per request and key head, parts of the tokens.
struct Shape {
    int rt, blocks, splits;
};
Shape shape_of(const AttentionArgs& a)
{
    Shape s;
    const int64_t rows = (int64_t)a.max_new * (a.q_heads / a.kv_heads);
    const int widest = a.D <= 128 ? 4 : a.D <= 256 ? 2 : 1;
    s.rt = rows <= 16 ? 1 : rows <= 32 || widest == 2 ? 2 : 4;
    s.blocks = (int)((rows + 16 * s.rt - 1) / (16 * s.rt));
    if (s.blocks < 1) s.blocks = 1;
    const int64_t units = (int64_t)a.R * a.kv_heads * s.blocks;
    const int64_t wanted = 1024, longest = (a.max_len + 255) / 256;
    int64_t n = units > 0 ? (wanted + units - 1) / units : 1;
    if (n > longest) n = longest;
    if (n > 256) n = 256;
    s.splits = (int)(n < 1 ? 1 : n);
    return s;
}

template <int D>
hipError_t launch_few(const AttentionArgs& a, const Shape& s, void* workspace, hipStream_t stream)
{
    const int64_t work = (int64_t)a.R * a.kv_heads * s.blocks * s.splits, grid = work + 32;
    if (grid > 0x7fffffffLL) return hipErrorInvalidConfiguration;
    const int64_t rows = (int64_t)s.splits * a.T * a.q_heads;
    float* po = static_cast<float*>(workspace);
    float2* ps = s.splits > 1 ? reinterpret_cast<float2*>(po + rows * D) : nullptr;
    const Pages P = pages_of(a.page);
    const dim3 g((unsigned)grid), b(256);
    switch (s.rt) {
        case 1: hipLaunchKernelGGL((few_rows_kernel<D, 1>), g, b, 0, stream, a, P, s.blocks, s.splits, work, po, ps); break;
        case 2: hipLaunchKernelGGL((few_rows_kernel<D, 2>), g, b, 0, stream, a, P, s.blocks, s.splits, work, po, ps); break;
        default:
            if constexpr (D <= 128) hipLaunchKernelGGL((few_rows_kernel<D, 4>), g, b, 0, stream, a, P, s.blocks, s.splits, work, po, ps);
            else return hipErrorInvalidValue;
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || s.splits == 1) return e;
    const int64_t join = (int64_t)a.R * a.kv_heads * s.blocks * 16 * s.rt;
    if (join > 0x7fffffffLL) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL(join_kernel<D>, dim3((unsigned)join), b, 0, stream, a, s.blocks, 16 * s.rt, s.splits, po, ps);
    return hipGetLastError();
}

}  // namespace

size_t attention_workspace(const AttentionArgs& args)
{
    const Shape s = shape_of(args);
    return s.splits > 1 ? (size_t)s.splits * args.T * args.q_heads * (args.D * 4 + 8) : 0;
}

hipError_t launch_attention(const AttentionArgs& args, void* workspace, hipStream_t stream)
{
    if (args.T <= 0) return hipSuccess;
    const Shape s = shape_of(args);
    switch (args.D) {
        case 32: return launch_few<32>(args, s, workspace, stream);
        case 64: return launch_few<64>(args, s, workspace, stream);
        case 96: return launch_few<96>(args, s, workspace, stream);
        case 128: return launch_few<128>(args, s, workspace, stream);
        case 160: return launch_few<160>(args, s, workspace, stream);
        case 192: return launch_few<192>(args, s, workspace, stream);
        case 224: return launch_few<224>(args, s, workspace, stream);
        case 256: return launch_few<256>(args, s, workspace, stream);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace ciar
