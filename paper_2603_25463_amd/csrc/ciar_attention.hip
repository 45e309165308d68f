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

// The output's accumulators on the vector ALUs, where that is rare (a rescaling, a value that is not finite): element by element in the
// accumulation registers.  As ordinary code such a branch would claim vector registers for all of them at once (128 of a lane's 256
// with 64 rows of 128 to a wave, and the loop next to it would spill).  The asm hides its reads from the compiler, which would keep
// them 19 cycles behind a matrix instruction that writes the registers, and its writes 2 before one that reads them: waited for here.
__device__ __forceinline__ void acc_settled()
{
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_nop 15\n\ts_nop 7");
}
__device__ __forceinline__ void acc_written()
{
    asm volatile("s_nop 7");
    __builtin_amdgcn_sched_barrier(0);
}
template <typename V>
__device__ __forceinline__ void scale_acc(V& acc, float f)
{
    acc_settled();
#pragma unroll
    for (int v = 0; v < (int)(sizeof(V) / 4); ++v) {
        float x = acc[v], t;
        asm volatile("v_accvgpr_read_b32 %1, %0\n\tv_mul_f32_e32 %1, %2, %1\n\tv_accvgpr_write_b32 %0, %1" : "+a"(x), "=&v"(t) : "v"(f));
        acc[v] = x;
    }
    acc_written();
}
template <typename V>
__device__ __forceinline__ void add_acc(V& acc, const V& y, bool take)
{
    acc_settled();
#pragma unroll
    for (int v = 0; v < (int)(sizeof(V) / 4); ++v) {
        const float z = take ? y[v] : 0.f;
        float x = acc[v], t;
        asm volatile("v_accvgpr_read_b32 %1, %0\n\tv_add_f32_e32 %1, %2, %1\n\tv_accvgpr_write_b32 %0, %1" : "+a"(x), "=&v"(t) : "v"(z));
        acc[v] = x;
    }
    acc_written();
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

// A request's row of pages, read through the scalar cache: its loads are counted apart from those of keys and values, which
// would otherwise all be waited for with each page.
using table_row = const __attribute__((address_space(4))) int32_t*;

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
    const table_row row = (table_row)(A.table + (int64_t)u.r * A.table_stride);
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
                    for (int b = 0; b < D / 16; ++b) scale_acc(acc[i][b], keep);
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
                                add_acc(acc[i][b], y, t0 + t < seen[i]);
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

// ---- many rows to a key head: the matrix cores' work ------------------------------------------------------------------------
//
// A workgroup of four waves takes 128 QT rows of one request and key head (a wave 32 QT), and a part of the tokens.  Steps of 32
// tokens come into LDS as they lie in the cache (global_load_lds, a ring of slots, requested two or three steps ahead), and every wave
// reads all of a step as operands of v_mfma_f32_32x32x16_bf16: a lane's 16 bytes are consecutive lanes', without conflicts.
// With 64 rows to a wave an operand feeds two matrix instructions, and LDS is half as busy as they are (with 32, as busy).
//
// S^T = K Q^T: lane l holds row l % 32, and of a step's tokens the eight of each atom's half l / 32 (keys enter an atom's rows with
// bits 2 and 3 of the token swapped, which makes a lane's accumulators consecutive tokens): they are the second product's operand
// as they are.  A wave has its SIMD to itself, so its vector instructions have to run while its own matrix instructions do:
// the loop's body computes the weights of step s next to the scores of step s + 1 and the output of step s - 1, all independent.  The
// references are looked at between bodies, and a rescaling, which is rare (kSlack), waits until the output has taken step s - 1.
typedef float f32x16 __attribute__((ext_vector_type(16)));
using lds_ptr = __attribute__((address_space(3))) void*;
using mem_ptr = const __attribute__((address_space(1))) void*;

// `n` things in pairs over `groups`: how many each group takes.
constexpr int pairs_of(int n, int groups) { return ((n + groups - 1) / groups + 1) / 2 * 2; }

// A lane's weights of a step, as the second product takes them: eight consecutive tokens of each atom.
template <int QT>
struct Weights {
    uint32_t pair[QT][8];
    __device__ __forceinline__ bf16x8 at(int i, int atom) const
    {
        return __builtin_bit_cast(bf16x8, u32x4{pair[i][4 * atom], pair[i][4 * atom + 1], pair[i][4 * atom + 2], pair[i][4 * atom + 3]});
    }
    // (the empty asm keeps them where they are computed: they are used a step later, and would be computed there)
    __device__ __forceinline__ void put(int i, int v, float a, float b)
    {
        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
        pair[i][v / 2] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b});
        asm volatile("" : "+v"(pair[i][v / 2]));
    }
};

template <int D, int QT>
__global__ __launch_bounds__(256, 1) void many_rows_kernel(const AttentionArgs A, const Pages P, int blocks, int splits, int64_t work,
                                                           float* __restrict__ part_o, float2* __restrict__ part_s)
{
    constexpr int KS = D / 16, DB = D / 32;                        // slices of 16 dimensions, blocks of 32
    constexpr int ATOM = kAtom * D * 2, HALF = 2 * ATOM, SLOT = 2 * HALF;       // bytes: keys, then values of a step
    constexpr int SLOTS = D <= 128 ? 5 : 4, AHEAD = SLOTS - 2;
    constexpr int PIECES = HALF / 1024, MINE = (PIECES + 3) / 4;   // 1 KiB requests of a step's keys (and values), and a wave's
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 31, half = lane >> 5;
    if ((int64_t)blockIdx.x >= work) {
        fill_unclaimed(A, ((int64_t)blockIdx.x - work) * 256 + tid, ((int64_t)gridDim.x - work) * 256);
        return;
    }
    Unit u;
    {
        int i = blockIdx.x;
        u.h = i % A.kv_heads; i /= A.kv_heads;
        u.split = i % splits; i /= splits;
        u.block = blocks - 1 - i % blocks;                         // the blocks that see most come first
        u.r = i / blocks;
    }
    const int g = A.q_heads / A.kv_heads;
    const Request R = request_of(A, u.r);
    constexpr int ROWS = 128 * QT;
    const int rows = R.n * g, m0 = u.block * ROWS;
    if (m0 >= rows) return;
    const int most = min(max(R.base + min(m0 + ROWS - 1, rows - 1) / g + 1, 0), R.len);
    const int least = min(max(R.base + m0 / g + 1, 0), R.len);
    const int steps = (most + kSteps - 1) / kSteps, each = (steps + splits - 1) / splits;
    const int first = u.split * each, last = min(first + each, steps);
    if (first >= last && u.split > 0) return;
    const int full = min(max(least / kSteps, first), last);        // steps that every row sees whole: [first, full)

    bf16x8 q[QT][KS];
    f32x16 acc[QT][DB];
    float ref[QT], total[QT];
    int seen[QT];
    const uint32_t flip = A.scale < 0.f ? 0x80008000u : 0u;        // (a negative scale is the queries': largest scores stay largest)
    const float scale = fabsf(A.scale) * kLog2e;
    const int mw = m0 + wave * 32 * QT;                            // this wave's first row
#pragma unroll
    for (int i = 0; i < QT; ++i) {
        const int m = min(mw + 32 * i + col, rows - 1), j = m / g, head = u.h * g + (m - j * g);
        seen[i] = min(max(R.base + j + 1, 0), R.len);
        const uint16_t* qrow = static_cast<const uint16_t*>(A.q.p) + (int64_t)(R.begin + j) * A.q.token + (int64_t)head * A.q.head;
#pragma unroll
        for (int k = 0; k < KS; ++k) q[i][k] = __builtin_bit_cast(bf16x8, load16_any(qrow + 16 * k + 8 * half) ^ flip);
#pragma unroll
        for (int b = 0; b < DB; ++b)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][b][v] = 0.f;
        ref[i] = -INFINITY;
        total[i] = 0.f;
    }
    if (first < last) {
        const int64_t head_bytes = (int64_t)A.page * D * 2;
        const table_row row = (table_row)(A.table + (int64_t)u.r * A.table_stride);
        const int atoms = (most + kAtom - 1) / kAtom;
        auto atom_at = [&](int atom) -> int64_t {
            const uint32_t a = (uint32_t)min(atom, atoms - 1), page = __umulhi(2 * a, P.mul) >> P.shift;
            const int p = min(max(row[page], 0), A.pages - 1);
            return ((int64_t)p * A.kv_heads + u.h) * head_bytes + (int64_t)(a - page * P.per) * ATOM;
        };
        // requests of a step whose atoms lie at a0, a1
        auto request = [&](int64_t a0, int64_t a1, int slot) {
#pragma unroll
            for (int x = 0; x < MINE; ++x) {
                const int piece = min(wave + 4 * x, PIECES - 1);   // (a repeated request writes what is there)
                const int64_t from = (piece >= PIECES / 2 ? a1 + (piece - PIECES / 2) * 1024 : a0 + piece * 1024) + lane * 16;
                char* to = lds + slot * SLOT + piece * 1024;
                __builtin_amdgcn_global_load_lds((mem_ptr)(static_cast<const char*>(A.k_cache) + from), (lds_ptr)to, 16, 0, 0);
                __builtin_amdgcn_global_load_lds((mem_ptr)(static_cast<const char*>(A.v_cache) + from), (lds_ptr)(to + HALF), 16, 0, 0);
            }
        };
        const int kread = (col >> 4) * ATOM + half * 256 + ((col & 3) | (col >> 1 & 4) | (col << 1 & 8)) * 16;
        const int vread = HALF + (half * D + col) * 16;
        auto key = [&](int slot, int k) { return *reinterpret_cast<const bf16x8*>(lds + slot * SLOT + kread + k * 512); };
        auto value = [&](int slot, int a, int b) { return *reinterpret_cast<const bf16x8*>(lds + slot * SLOT + vread + a * ATOM + b * 512); };
        auto scores = [&](f32x16 (&s)[QT], int slot) {
#pragma unroll
            for (int i = 0; i < QT; ++i)
#pragma unroll
                for (int v = 0; v < 16; ++v) s[i][v] = 0.f;
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                const bf16x8 x = key(slot, k);
#pragma unroll
                for (int i = 0; i < QT; ++i) s[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, q[i][k], s[i], 0, 0, 0);
            }
        };
        auto output = [&](const Weights<QT>& w, int slot) {
#pragma unroll
            for (int a = 0; a < 2; ++a)
#pragma unroll
                for (int b = 0; b < DB; ++b) {
                    const bf16x8 x = value(slot, a, b);
#pragma unroll
                    for (int i = 0; i < QT; ++i) acc[i][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, w.at(i, a), acc[i][b], 0, 0, 0);
                }
        };
        auto largest = [&](const f32x16& s) {
            float h = fmaxf(s[0], s[1]);
#pragma unroll
            for (int v = 2; v < 16; v += 2) h = fmaxf(fmaxf(s[v], s[v + 1]), h);
            return h * scale;
        };
        // moves the references where scores exceed them; true if any has moved (the factors are in keep)
        auto look = [&](const float (&high)[QT], float (&keep)[QT]) {
            bool up = false;
#pragma unroll
            for (int i = 0; i < QT; ++i) up |= high[i] > ref[i] + kSlack;
            if (!__any(up)) return false;
#pragma unroll
            for (int i = 0; i < QT; ++i) {
                const float now = fmaxf(ref[i], fmaxf(high[i], __shfl_xor(high[i], 32)));
                keep[i] = now == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(ref[i] - now);
                ref[i] = now;
                total[i] *= keep[i];
            }
            return true;
        };
        auto rescale = [&](const float (&keep)[QT]) {
#pragma unroll
            for (int i = 0; i < QT; ++i)
#pragma unroll
                for (int b = 0; b < DB; ++b) scale_acc(acc[i][b], keep[i]);
        };
        // the ring: step s lies in slot (s - first) % SLOTS
        int64_t n0 = 0, n1 = 0;
#pragma unroll
        for (int x = 0; x < AHEAD; ++x) request(atom_at(2 * (first + x)), atom_at(2 * (first + x) + 1), x);
        n0 = atom_at(2 * (first + AHEAD));
        n1 = atom_at(2 * (first + AHEAD) + 1);
        int slot = 0, ahead = AHEAD % SLOTS;                       // of the step s of the body, and of the step that is requested in it
        // What opens step s: the steps up to s + 1 (the last AHEAD - 2 requested may be under way) have arrived, and every wave is done with s - 2
        auto open = [&](int s) {
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(2 * MINE * (AHEAD - 2)) : "memory");
            request(n0, n1, ahead);
            ahead = ahead + 1 == SLOTS ? 0 : ahead + 1;
            n0 = atom_at(2 * (s + AHEAD + 1));
            n1 = atom_at(2 * (s + AHEAD + 1) + 1);
        };
        int s = first;
        Weights<QT> wa, wb;
        if (first < full) {
            asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(2 * MINE * (AHEAD - 1)) : "memory");
            f32x16 sa[QT], sb[QT];
            float high[QT], keep[QT];
            scores(sa, 0);
#pragma unroll
            for (int i = 0; i < QT; ++i) high[i] = largest(sa[i]);
            int prev = 0;
            // The body of step s: its weights, the scores of the next step, the output of the one before (unless it is the first).
            // Written as groups of QT matrix instructions on one operand, each followed by its share of the vector work and by the
            // read of the operand that the group after the next one takes; nothing moves from group to group.  Two groups of the
            // output open the body: their operands have been there since the body before, while the next step's keys are on their way.
            constexpr int GROUPS = KS + 2 * DB, LEAD = 2;
            constexpr int SHARE = pairs_of(16 * QT, GROUPS), SHARE1 = pairs_of(16 * QT, KS);
            bf16x8 op[2];                                          // operands of the next two groups
            auto operand = [&](int n, int keys, int values) -> bf16x8 {        // of group n
                if (n >= LEAD && n < LEAD + KS) return key(keys, n - LEAD);
                const int o = n < LEAD ? n : n - KS;
                return value(values, o / DB, o % DB);
            };
            auto body = [&](f32x16 (&now)[QT], f32x16 (&next)[QT], Weights<QT>& w, const Weights<QT>& before, auto opening) {
                constexpr bool FIRST = decltype(opening)::value;
                open(s);
                const bool moved = look(high, keep);
                const int after = slot + 1 == SLOTS ? 0 : slot + 1;
                float sub[QT], top[QT];
#pragma unroll
                for (int i = 0; i < QT; ++i) {
                    sub[i] = ref[i] == -INFINITY ? 0.f : ref[i];
                    top[i] = -INFINITY;
#pragma unroll
                    for (int v = 0; v < 16; ++v) next[i][v] = 0.f;
                }
                if constexpr (FIRST) { op[0] = key(after, 0); op[1] = key(after, 1); }
#pragma unroll
                for (int n = FIRST ? LEAD : 0; n < GROUPS; ++n) {
                    const bool keys = n >= LEAD && n < LEAD + KS;
                    if (FIRST && !keys) {
                        // (no step before: only the vector work)
                    } else {
                        const bf16x8 x = op[n & 1];
                        const int o = n < LEAD ? n : n - KS;
#pragma unroll
                        for (int i = 0; i < QT; ++i) {
                            if (keys) next[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, q[i][keys ? n - LEAD : 0], next[i], 0, 0, 0);
                            else acc[i][keys ? 0 : o % DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, before.at(i, keys ? 0 : o / DB), acc[i][keys ? 0 : o % DB], 0, 0, 0);
                        }
                    }
                    // (the last two reads are the next body's first: this step's values)
                    if (n + 2 < GROUPS) op[n & 1] = operand(n + 2, after, prev);
                    else op[n & 1] = operand(n + 2 - GROUPS, after, slot);
                    const int e0 = FIRST ? (n - LEAD) * SHARE1 : n * SHARE, e1 = FIRST ? e0 + SHARE1 : e0 + SHARE;
#pragma unroll
                    for (int e = e0; e < e1; e += 2)
                        if (e < 16 * QT) {
                            const int i = e / 16 < QT ? e / 16 : 0, v = e % 16;
                            const float p0 = __builtin_amdgcn_exp2f(fmaf(now[i][v], scale, -sub[i]));
                            const float p1 = __builtin_amdgcn_exp2f(fmaf(now[i][v + 1], scale, -sub[i]));
                            total[i] += p0;
                            total[i] += p1;
                            w.put(i, v, p0, p1);
                        }
                    if (n >= LEAD + KS + 1) {                      // the scores are there: their largest, a piece at a time
                        constexpr int LEFT = 2 * DB - LEAD - 1, PIECE = (16 + LEFT - 1) / (LEFT > 0 ? LEFT : 1);
                        const int v0 = (n - LEAD - KS - 1) * PIECE;
#pragma unroll
                        for (int i = 0; i < QT; ++i)
#pragma unroll
                            for (int v = v0; v < v0 + PIECE; ++v)
                                if (v < 16) top[i] = fmaxf(top[i], next[i][v]);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                if constexpr (2 * DB - LEAD - 1 <= 0) {
#pragma unroll
                    for (int i = 0; i < QT; ++i)
#pragma unroll
                        for (int v = 0; v < 16; ++v) top[i] = fmaxf(top[i], next[i][v]);
                }
#pragma unroll
                for (int i = 0; i < QT; ++i) high[i] = top[i] * scale;
                if (moved) rescale(keep);
                prev = slot;
                slot = after;
                ++s;
            };
            body(sa, sb, wa, wb, std::true_type{});
            bool odd = true;                                       // the latest weights are in wa
            while (s + 1 < full) {
                body(sb, sa, wb, wa, std::false_type{});
                body(sa, sb, wa, wb, std::false_type{});
            }
            if (s < full) {
                body(sb, sa, wb, wa, std::false_type{});
                odd = false;
            }
            if (odd) output(wa, prev); else output(wb, prev);
        }
        // the steps that rows see in part, one after another
        for (; s < last; ++s) {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            open(s);
            const int t0 = s * kSteps;
            if (mw < rows) {
                f32x16 x[QT];
                float high[QT], keep[QT];
                scores(x, slot);
#pragma unroll
                for (int i = 0; i < QT; ++i) {
#pragma unroll
                    for (int v = 0; v < 16; ++v)
                        if (t0 + (v >> 3) * kAtom + 8 * half + (v & 7) >= seen[i]) x[i][v] = -INFINITY;
                    high[i] = largest(x[i]);
                    if (scale == 0.f && high[i] != high[i]) high[i] = 0.f;
                }
                if (look(high, keep)) rescale(keep);
#pragma unroll
                for (int i = 0; i < QT; ++i) {
                    const float sub = ref[i] == -INFINITY ? 0.f : ref[i];
                    float sum = 0.f;
#pragma unroll
                    for (int v = 0; v < 16; ++v) {
                        const bool sees = t0 + (v >> 3) * kAtom + 8 * half + (v & 7) < seen[i];
                        const float p = sees ? __builtin_amdgcn_exp2f(fmaf(x[i][v], scale, -sub)) : 0.f;
                        sum += p;
                        x[i][v] = p;
                    }
#pragma unroll
                    for (int v = 0; v < 16; v += 2) wa.put(i, v, x[i][v], x[i][v + 1]);
                    total[i] += sum;
                }
                // values that no row sees are zeros; one that is not finite must not reach the rows that do not see it (0 * inf)
#pragma unroll 1
                for (int a = 0; a < 2; ++a) {
                    bf16x8 val[DB];
                    bool bad = false;
#pragma unroll
                    for (int b = 0; b < DB; ++b) {
                        u32x4 y = __builtin_bit_cast(u32x4, value(slot, a, b));
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if (t0 + a * kAtom + 8 * half + e >= most) y[e / 2] &= e & 1 ? 0x0000ffffu : 0xffff0000u;
#pragma unroll
                        for (int e = 0; e < 4; ++e) bad |= (y[e] & 0x7f80u) == 0x7f80u || (y[e] & 0x7f800000u) == 0x7f800000u;
                        val[b] = __builtin_bit_cast(bf16x8, y);
                    }
                    if (!__any(bad)) {
#pragma unroll
                        for (int b = 0; b < DB; ++b)
#pragma unroll
                            for (int i = 0; i < QT; ++i) acc[i][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(val[b], a ? wa.at(i, 1) : wa.at(i, 0), acc[i][b], 0, 0, 0);
                        continue;
                    }
#pragma unroll 1
                    for (int t = 0; t < kAtom && t0 + a * kAtom + t < most; ++t) {
#pragma unroll
                        for (int i = 0; i < QT; ++i) {
                            bf16x8 one = a ? wa.at(i, 1) : wa.at(i, 0);
#pragma unroll
                            for (int e = 0; e < 8; ++e)
                                if (t != 8 * half + e) one[e] = (__bf16)0.f;
#pragma unroll
                            for (int b = 0; b < DB; ++b) {
                                u32x4 y = __builtin_bit_cast(u32x4, val[b]);
#pragma unroll
                                for (int e = 0; e < 8; ++e)
                                    if (t != 8 * half + e) y[e / 2] &= e & 1 ? 0x0000ffffu : 0xffff0000u;
                                f32x16 zero;
#pragma unroll
                                for (int v = 0; v < 16; ++v) zero[v] = 0.f;
                                const f32x16 z = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, y), one, zero, 0, 0, 0);
                                add_acc(acc[i][b], z, t0 + a * kAtom + t < seen[i]);
                            }
                        }
                    }
                }
            }
            slot = slot + 1 == SLOTS ? 0 : slot + 1;
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");           // (requests past the end: LDS is handed on when the workgroup ends)
    }
#pragma unroll
    for (int i = 0; i < QT; ++i) {
        const int m = mw + 32 * i + col;
        const float sum = total[i] + __shfl_xor(total[i], 32);
        if (m >= rows) continue;
        const int j = m / g, head = u.h * g + (m - j * g);
        const int64_t t = R.begin + j;
        if (splits == 1) {
            const float inv = sum == 0.f ? 0.f : 1.f / sum;
            char* o = (char*)A.out.p + (t * A.out.token + (int64_t)head * A.out.head) * 2;
#pragma unroll
            for (int b = 0; b < DB; ++b)
#pragma unroll
                for (int v = 0; v < 16; v += 4) {
                    bf16x4 y;
#pragma unroll
                    for (int e = 0; e < 4; ++e) y[e] = (__bf16)(acc[i][b][v + e] * inv);
                    __builtin_memcpy(o + (32 * b + 2 * v + 4 * half) * 2, &y, 8);
                }
            if (half == 0 && A.lse) A.lse[t * A.q_heads + head] = sum == 0.f ? -INFINITY : (ref[i] + __builtin_amdgcn_logf(sum)) * kLn2f;
        } else {
            const int64_t at = ((int64_t)u.split * A.T + t) * A.q_heads + head;
#pragma unroll
            for (int b = 0; b < DB; ++b)
#pragma unroll
                for (int v = 0; v < 16; v += 4)
                    *reinterpret_cast<f32x4*>(part_o + at * D + 32 * b + 2 * v + 4 * half) = f32x4{acc[i][b][v], acc[i][b][v + 1], acc[i][b][v + 2], acc[i][b][v + 3]};
            if (half == 0) part_s[at] = {ref[i], sum};
        }
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

// How a call is laid out: rows of a workgroup, blocks of rows per request and key head, parts of the tokens.
struct Shape {
    bool many;
    int rows, blocks, splits;
};
Shape shape_of(const AttentionArgs& a)
{
    Shape s;
    const int64_t rows = (int64_t)a.max_new * (a.q_heads / a.kv_heads);
    s.many = rows > 64;
    if (s.many) s.rows = a.D <= 128 && rows > 128 ? 256 : 128;
    else s.rows = rows <= 16 ? 16 : rows <= 32 || a.D > 128 ? 32 : 64;
    s.blocks = (int)((rows + s.rows - 1) / s.rows);
    if (s.blocks < 1) s.blocks = 1;
    const int64_t units = (int64_t)a.R * a.kv_heads * s.blocks;
    const int64_t wanted = s.many ? 512 : 1024, longest = (a.max_len + 255) / 256;
    int64_t n = units > 0 ? (wanted + units - 1) / units : 1;
    if (n > longest) n = longest;
    if (n > 256) n = 256;
    s.splits = (int)(n < 1 ? 1 : n);
    return s;
}

// Asks once per device for the dynamic LDS that a kernel needs.
hipError_t allow_lds(const void* kernel, int bytes)
{
    return hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
}

template <int D, int QT>
hipError_t launch_many(const AttentionArgs& a, const Shape& s, unsigned grid, int64_t work, float* po, float2* ps, hipStream_t stream)
{
    constexpr int bytes = (D <= 128 ? 5 : 4) * 4 * kAtom * D * 2;
    const hipError_t e = allow_lds(reinterpret_cast<const void*>(&many_rows_kernel<D, QT>), bytes);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((many_rows_kernel<D, QT>), dim3(grid), dim3(256), bytes, stream, a, pages_of(a.page), s.blocks, s.splits, work, po, ps);
    return hipGetLastError();
}

template <int D>
hipError_t launch_shape(const AttentionArgs& a, const Shape& s, void* workspace, hipStream_t stream)
{
    const int64_t work = (int64_t)a.R * a.kv_heads * s.blocks * s.splits, grid = work + 32;
    const int64_t join = (int64_t)a.R * a.kv_heads * s.blocks * s.rows;
    if (grid > 0x7fffffffLL || join > 0x7fffffffLL) return hipErrorInvalidConfiguration;
    const int64_t rows = (int64_t)s.splits * a.T * a.q_heads;
    float* po = static_cast<float*>(workspace);
    float2* ps = s.splits > 1 ? reinterpret_cast<float2*>(po + rows * D) : nullptr;
    const dim3 g((unsigned)grid), b(256);
    hipError_t e;
    if (s.many) {
        if constexpr (D <= 128) e = s.rows == 256 ? launch_many<D, 2>(a, s, (unsigned)grid, work, po, ps, stream) : launch_many<D, 1>(a, s, (unsigned)grid, work, po, ps, stream);
        else e = launch_many<D, 1>(a, s, (unsigned)grid, work, po, ps, stream);
    } else {
        const Pages P = pages_of(a.page);
        if (s.rows == 16) hipLaunchKernelGGL((few_rows_kernel<D, 1>), g, b, 0, stream, a, P, s.blocks, s.splits, work, po, ps);
        else if (s.rows == 32) hipLaunchKernelGGL((few_rows_kernel<D, 2>), g, b, 0, stream, a, P, s.blocks, s.splits, work, po, ps);
        else if constexpr (D <= 128) hipLaunchKernelGGL((few_rows_kernel<D, 4>), g, b, 0, stream, a, P, s.blocks, s.splits, work, po, ps);
        e = hipGetLastError();
    }
    if (e != hipSuccess || s.splits == 1) return e;
    hipLaunchKernelGGL(join_kernel<D>, dim3((unsigned)join), b, 0, stream, a, s.blocks, s.rows, s.splits, po, ps);
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
        case 32: return launch_shape<32>(args, s, workspace, stream);
        case 64: return launch_shape<64>(args, s, workspace, stream);
        case 96: return launch_shape<96>(args, s, workspace, stream);
        case 128: return launch_shape<128>(args, s, workspace, stream);
        case 160: return launch_shape<160>(args, s, workspace, stream);
        case 192: return launch_shape<192>(args, s, workspace, stream);
        case 224: return launch_shape<224>(args, s, workspace, stream);
        case 256: return launch_shape<256>(args, s, workspace, stream);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace ciar
