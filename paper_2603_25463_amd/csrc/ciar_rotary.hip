// gfx950 kernels of the rotary positions (ciar_rotary in include/ciar.h): queries and keys turned by their positions, keys and
// values laid into the pages of the cache.
#include "ciar_device.h"
#include "ciar_step.h"

namespace ciar {
namespace {

// The sine and cosine of an angle in radians, for angles of positions far into a context: the angle comes in 64 bits, its
// multiple of pi / 2 is taken off there (pi / 2 in two parts: the remainder is right to 1e-16 of the angle), and the remainder in
// [-pi / 4, pi / 4] goes through the Taylor polynomials of degree 11 and 10 in 32 bits (their next terms are below 7e-12 and
// 2e-10 there: the rounding of the result is what is left).
__device__ __forceinline__ void turn_of(double angle, float& c, float& s)
{
    const double k = rint(angle * 0.63661977236758134308);          // 2 / pi
    double r = fma(-k, 1.57079632679489661923, angle);              // pi / 2, and what its 64 bits leave out
    r = fma(-k, 6.123233995736766036e-17, r);
    const float x = (float)r, x2 = x * x;
    float ps = fmaf(x2, -1.f / 39916800.f, 1.f / 362880.f);
    ps = fmaf(x2, ps, -1.f / 5040.f);
    ps = fmaf(x2, ps, 1.f / 120.f);
    ps = fmaf(x2, ps, -1.f / 6.f);
    const float sn = fmaf(x * x2, ps, x);
    float pc = fmaf(x2, -1.f / 3628800.f, 1.f / 40320.f);
    pc = fmaf(x2, pc, -1.f / 720.f);
    pc = fmaf(x2, pc, 1.f / 24.f);
    pc = fmaf(x2, pc, -0.5f);
    const float cs = fmaf(x2, pc, 1.f);
    const int q = (int)(long long)k & 3;                            // quarter turns
    const float a = q & 1 ? sn : cs, b = q & 1 ? cs : sn;
    c = q == 1 || q == 2 ? -a : a;
    s = q >= 2 ? -b : b;
}

// Sixteen bytes of a row, from wherever it lies (rows start at any element; the hardware takes such loads and stores).
__device__ __forceinline__ u32x4 load16_any(const void* p)
{
    u32x4 v;
    __builtin_memcpy(&v, p, 16);
    return v;
}

template <typename T> struct Row;
template <> struct Row<float> {
    static constexpr int kPerVec = 4;
    static __device__ __forceinline__ float load(const char* p) { return *reinterpret_cast<const float*>(p); }
    static __device__ __forceinline__ void store(char* p, float v) { *reinterpret_cast<float*>(p) = v; }
    static __device__ __forceinline__ void unpack(const u32x4& r, float* f) { Elt<float>::unpack(r, f); }
    static __device__ __forceinline__ u32x4 pack(const float* f)
    {
        return {__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
    }
};
template <> struct Row<bf16_t> {
    static constexpr int kPerVec = 8;
    static __device__ __forceinline__ float load(const char* p) { return bits_f((uint32_t)*reinterpret_cast<const uint16_t*>(p) << 16); }
    static __device__ __forceinline__ void store(char* p, float v) { *reinterpret_cast<__bf16*>(p) = (__bf16)v; }
    static __device__ __forceinline__ void unpack(const u32x4& r, float* f) { Elt<bf16_t>::unpack(r, f); }
    static __device__ __forceinline__ u32x4 pack(const float* f)
    {
        typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
        bf16x8 y;
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = (__bf16)f[e];
        return __builtin_bit_cast(u32x4, y);
    }
};

constexpr int kRotaryTokens = 16;      // most tokens of a workgroup

// A workgroup takes up to 16 tokens and a range of their heads (queries, keys, values, in that order).  First the factors of every
// dimension of its tokens go into LDS: y[d] = c x[d] + s x[partner of d], with c = 1, s = -0 for dimensions that are only copied (a
// negative zero stays one).  Then every thread takes the same 16 bytes of one head row after another: its own vector, and for pairs of
// halves the partners' (a second load of what another thread has just loaded; any offset).  Values are turned round in LDS: the cache
// wants a dimension's eight tokens side by side.  Tiles begin where an atom of the cache begins if the tokens' slots are
// consecutive (the first token's slot says where): a dimension's eight tokens are then one store; runs that are cut off are stored
// element by element.  Bound by memory: 16 bytes in, 16 out, four multiply-adds to an 8-byte pair.
template <typename T, bool INTERLEAVED>
__global__ __launch_bounds__(256) void rotary_kernel(const RotaryArgs A, int tile, int heads_per_wg, int stage)
{
    using V = Row<T>;
    constexpr int E = sizeof(T), EPV = V::kPerVec;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    float2* turns = reinterpret_cast<float2*>(lds);                 // [tile][DP]
    __shared__ int s_slot[kRotaryTokens];
    const int tid = threadIdx.x, D = A.D, n = A.n, half = n / 2;
    const int DP = (D + EPV - 1) / EPV * EPV;
    const bool cached = A.k_cache != nullptr;
    int shift = 0;
    if (cached && tile == kRotaryTokens) {
        const int s = A.slots[0];
        shift = s > 0 ? s % kAtom : 0;
    }
    const int t_first = (int)blockIdx.x * tile - shift;             // (negative in the first tile)
    const int t0 = max(t_first, 0), tokens = min(t_first + tile, A.T) - t0;
    if (tokens <= 0) return;
    const int turned = A.q_heads + A.kv_heads, all = turned + (cached ? A.kv_heads : 0);
    const int h0 = (int)blockIdx.y * heads_per_wg, h1 = min(h0 + heads_per_wg, all);
    if (cached && tid < tokens) {
        const int s = A.slots[t0 + tid];
        s_slot[tid] = s >= 0 && s < A.slot_count ? s : -1;
    }
    if (h0 < turned) {
        for (int i = tid; i < tokens * half; i += 256) {
            const int t = i / half, p = i - t * half;
            float c, s;
            turn_of((double)A.positions[t0 + t] * A.sign * A.inv_freq[p], c, s);
            c = (float)(c * A.magnitude);
            s = (float)(s * A.magnitude);
            turns[t * DP + (INTERLEAVED ? 2 * p : p)] = {c, -s};
            turns[t * DP + (INTERLEAVED ? 2 * p + 1 : p + half)] = {c, s};
        }
        const int rest = DP - n;
        for (int i = tid; i < tokens * rest; i += 256) {
            const int t = i / rest;
            turns[t * DP + n + (i - t * rest)] = {1.f, -0.f};
        }
    }
    __syncthreads();
    const int vecs = DP / EPV, rows = 256 / vecs, row0 = tid / vecs, d0 = (tid - row0 * vecs) * EPV;
    const int hb = min(h1, turned), hc = hb - h0;                  // heads to turn
    if (hc > 0 && row0 < rows) {
        const bool whole = d0 + EPV <= D;
        // where the vector's partners are: one vector `away` elements further, or (0) here and there, or nowhere (the rest is copied)
        const bool none = INTERLEAVED || d0 >= n;
        const int away = none || !whole ? 0 : d0 + EPV <= half ? half : d0 >= half ? -half : 0;
        const int dt = rows / hc, dh = rows - dt * hc;
        int t = row0 / hc, h = row0 - t * hc;
        for (; t < tokens; t += dt, h += dh) {
            if (h >= hc) { h -= hc; ++t; if (t >= tokens) break; }
            const int head = h0 + h, token = t0 + t;
            const bool isq = head < A.q_heads;
            const Heads& src = isq ? A.q : A.k;
            const int sh = isq ? head : head - A.q_heads;
            const char* row = static_cast<const char*>(src.p) + (token * src.token + sh * src.head) * E;
            float x[EPV], y[EPV], f[EPV];
            if (whole) V::unpack(load16_any(row + d0 * E), x);
            else {
#pragma unroll
                for (int e = 0; e < EPV; ++e) x[e] = d0 + e < D ? V::load(row + (d0 + e) * E) : 0.f;
            }
            if constexpr (INTERLEAVED) {
#pragma unroll
                for (int e = 0; e < EPV; ++e) y[e] = d0 + e < n ? x[e ^ 1] : 0.f;
            } else {
                if (away != 0) {
                    V::unpack(load16_any(row + (d0 + away) * E), y);
#pragma unroll
                    for (int e = 0; e < EPV; ++e) y[e] = d0 + e < n ? y[e] : 0.f;
                } else {
#pragma unroll
                    for (int e = 0; e < EPV; ++e) {
                        const int d = d0 + e;
                        y[e] = none || d >= n ? 0.f : V::load(row + (d < half ? d + half : d - half) * E);
                    }
                }
            }
            const float2* w = turns + t * DP + d0;
#pragma unroll
            for (int e = 0; e < EPV; ++e) f[e] = fmaf(x[e], w[e].x, y[e] * w[e].y);
            if (isq || !cached) {
                const Heads& dst = isq ? A.q_out : A.k_out;
                char* o = (char*)dst.p + (token * dst.token + sh * dst.head + d0) * E;
                const u32x4 r = V::pack(f);
                if (whole) __builtin_memcpy(o, &r, 16);
                else {
#pragma unroll
                    for (int e = 0; e < EPV; ++e)
                        if (d0 + e < D) V::store(o + e * E, f[e]);
                }
            } else if (E == 2) {
                const int slot = s_slot[t];
                if (slot >= 0) {
                    const int page = slot / A.page, off = slot - page * A.page;
                    const int64_t atom = (((int64_t)page * A.kv_heads + sh) * (A.page / kAtom) + off / kAtom) * kAtom * D;
                    *reinterpret_cast<u32x4*>((char*)A.k_cache + (atom + (d0 * 2 + off % kAtom) * 8) * 2) = V::pack(f);
                }
            }
        }
    }
    if (!cached || E != 2) return;
    // the values
    const int v0 = max(h0, turned);
    if (stage == 0) {
        // (few tokens: element by element)
        for (int h = v0; h < h1; ++h)
            for (int i = tid; i < tokens * D; i += 256) {
                const int t = i / D, d = i - t * D, slot = s_slot[t];
                if (slot < 0) continue;
                const int page = slot / A.page, off = slot - page * A.page, at = off % kAtom;
                const int64_t atom = (((int64_t)page * A.kv_heads + h - turned) * (A.page / kAtom) + off / kAtom) * kAtom * D;
                reinterpret_cast<uint16_t*>(A.v_cache)[atom + (at / 8 * D + d) * 8 + at % 8] =
                    static_cast<const uint16_t*>(A.v.p)[(t0 + t) * A.v.token + (h - turned) * A.v.head + d];
            }
        return;
    }
    if (v0 >= h1) return;
    // runs of consecutive slots within eight: a thread takes a dimension of a run
    const int RS = D + 2;                                           // halves of a staged row (rows of a column in different banks)
    uint16_t* staged = reinterpret_cast<uint16_t*>(lds);
    const int ds = 256 / D > 0 ? 256 / D : 1;
    for (int h = v0; h < h1; ++h) {
        __syncthreads();
        for (int i = tid; i < tokens * (D / 8); i += 256) {
            const int t = i / (D / 8), d = (i - t * (D / 8)) * 8;
            const u32x4 r = load16_any(static_cast<const char*>(A.v.p) + ((t0 + t) * A.v.token + (h - turned) * A.v.head + d) * 2);
            uint32_t* to = reinterpret_cast<uint32_t*>(staged + t * RS + d);
#pragma unroll
            for (int e = 0; e < 4; ++e) to[e] = r[e];
        }
        __syncthreads();
        for (int run = 0, t = 0; t < tokens; ++run) {
            const int slot = s_slot[t];
            int len = 1;
            while (t + len < tokens && slot >= 0 && (slot + len) % 8 != 0 && s_slot[t + len] == slot + len) ++len;
            if (slot >= 0 && (ds == 1 || run % ds == tid / D)) {
                const int page = slot / A.page, off = slot - page * A.page, at = off % kAtom;
                const int64_t atom = (((int64_t)page * A.kv_heads + h - turned) * (A.page / kAtom) + off / kAtom) * kAtom * D;
                for (int d = ds == 1 ? tid : tid % D; d < D; d += ds == 1 ? 256 : D) {
                    uint16_t* to = reinterpret_cast<uint16_t*>(A.v_cache) + atom + (at / 8 * D + d) * 8 + at % 8;
                    const uint16_t* from = staged + t * RS + d;
                    if (len == 8) {
                        u32x4 r;
#pragma unroll
                        for (int e = 0; e < 4; ++e) r[e] = from[2 * e * RS] | (uint32_t)from[(2 * e + 1) * RS] << 16;
                        *reinterpret_cast<u32x4*>(to) = r;
                    } else
                        for (int e = 0; e < len; ++e) to[e] = from[e * RS];
                }
            }
            t += len;
        }
    }
}

}  // namespace

hipError_t launch_rotary(int dtype, bool interleaved, const RotaryArgs& args, hipStream_t stream)
{
    if (args.T <= 0) return hipSuccess;
    const bool cached = args.k_cache != nullptr;
    const int heads = args.q_heads + args.kv_heads + (cached ? args.kv_heads : 0), cus = compute_units();
    // Tokens of a workgroup: 16 where they still make a workgroup for every compute unit (the cache's atoms whole, the factors of a
    // token computed for many heads), 1 where they do not.  Heads: as many ranges as make eight workgroups a unit.
    int tile = args.T >= kRotaryTokens * (cus / 4) ? kRotaryTokens : 1;
    if (args.D > 256 && tile > 4) tile = 4;                         // (factors of 8 bytes a dimension: 32 KiB of LDS)
    const int per = dtype == 0 ? 4 : 8, DP = (args.D + per - 1) / per * per;
    const int64_t tiles = ((int64_t)args.T + tile - 1) / tile + (cached && tile == kRotaryTokens ? 1 : 0);
    int64_t ranges = (8 * (int64_t)cus + tiles - 1) / tiles;
    if (ranges > (heads + 1) / 2) ranges = (heads + 1) / 2;
    if (ranges < 1) ranges = 1;
    const int each = (int)((heads + ranges - 1) / ranges);
    const int stage = tile == kRotaryTokens ? tile * (args.D + 2) * 2 : 0;
    const int bytes = tile * DP * 8 > stage ? tile * DP * 8 : stage;
    const dim3 grid((unsigned)tiles, (unsigned)((heads + each - 1) / each)), block(256);
    if (dtype == 0) {
        if (interleaved) hipLaunchKernelGGL((rotary_kernel<float, true>), grid, block, bytes, stream, args, tile, each, stage);
        else hipLaunchKernelGGL((rotary_kernel<float, false>), grid, block, bytes, stream, args, tile, each, stage);
    } else {
        if (interleaved) hipLaunchKernelGGL((rotary_kernel<bf16_t, true>), grid, block, bytes, stream, args, tile, each, stage);
        else hipLaunchKernelGGL((rotary_kernel<bf16_t, false>), grid, block, bytes, stream, args, tile, each, stage);
    }
    return hipGetLastError();
}

}  // namespace ciar
