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

template <typename T> struct Row;
template <> struct Row<float> {
    static __device__ __forceinline__ float load(const char* p) { return *reinterpret_cast<const float*>(p); }
    static __device__ __forceinline__ void store(char* p, float v) { *reinterpret_cast<float*>(p) = v; }
};
template <> struct Row<bf16_t> {
    static __device__ __forceinline__ float load(const char* p) { return bits_f((uint32_t)*reinterpret_cast<const uint16_t*>(p) << 16); }
    static __device__ __forceinline__ void store(char* p, float v) { *reinterpret_cast<__bf16*>(p) = (__bf16)v; }
};

// One workgroup per token, one element at a time.
template <typename T, bool INTERLEAVED>
__global__ __launch_bounds__(256) void rotary_kernel(const RotaryArgs A)
{
    __shared__ float2 turns[512];
    constexpr int E = sizeof(T);
    const int t = blockIdx.x, tid = threadIdx.x, half = A.n / 2;
    const double pos = (double)A.positions[t] * A.sign;
    for (int p = tid; p < half; p += 256) {
        float c, s;
        turn_of(pos * A.inv_freq[p], c, s);
        turns[p] = {(float)(c * A.magnitude), (float)(s * A.magnitude)};
    }
    __syncthreads();
    auto turned = [&](const char* row, int d) -> float {
        const float x = Row<T>::load(row + (int64_t)d * E);
        if (d >= A.n) return x;
        const bool second = INTERLEAVED ? (d & 1) : d >= half;
        const int p = INTERLEAVED ? d >> 1 : second ? d - half : d;
        const int other = INTERLEAVED ? d ^ 1 : second ? d - half : d + half;
        const float y = Row<T>::load(row + (int64_t)other * E);
        const float2 w = turns[p];
        return second ? x * w.x + y * w.y : x * w.x - y * w.y;
    };
    const int Dq = A.q_heads * A.D, Dk = A.kv_heads * A.D;
    for (int i = tid; i < Dq; i += 256) {
        const int h = i / A.D, d = i - h * A.D;
        const char* row = static_cast<const char*>(A.q.p) + (t * A.q.token + h * A.q.head) * E;
        Row<T>::store((char*)A.q_out.p + (t * A.q_out.token + h * A.q_out.head + d) * E, turned(row, d));
    }
    const int slot = A.k_cache ? A.slots[t] : 0;
    if (A.k_cache && (slot < 0 || slot >= A.slot_count)) return;
    for (int i = tid; i < Dk; i += 256) {
        const int h = i / A.D, d = i - h * A.D;
        const char* row = static_cast<const char*>(A.k.p) + (t * A.k.token + h * A.k.head) * E;
        const float x = turned(row, d);
        if (!A.k_cache) {
            Row<T>::store((char*)A.k_out.p + (t * A.k_out.token + h * A.k_out.head + d) * E, x);
        } else {
            const int page = slot / A.page, off = slot - page * A.page, a = off / kAtom, at = off % kAtom;
            const int64_t atom = (((int64_t)page * A.kv_heads + h) * (A.page / kAtom) + a) * kAtom * A.D;
            Row<T>::store((char*)A.k_cache + (atom + (d / 8 * kAtom + at) * 8 + d % 8) * E, x);
            const char* vrow = static_cast<const char*>(A.v.p) + (t * A.v.token + h * A.v.head) * E;
            Row<T>::store((char*)A.v_cache + (atom + (at / 8 * A.D + d) * 8 + at % 8) * E, Row<T>::load(vrow + (int64_t)d * E));
        }
    }
}

}  // namespace

hipError_t launch_rotary(int dtype, bool interleaved, const RotaryArgs& args, hipStream_t stream)
{
    if (args.T <= 0) return hipSuccess;
    const dim3 grid((unsigned)args.T), block(256);
    if (dtype == 0) {
        if (interleaved) hipLaunchKernelGGL((rotary_kernel<float, true>), grid, block, 0, stream, args);
        else hipLaunchKernelGGL((rotary_kernel<float, false>), grid, block, 0, stream, args);
    } else {
        if (interleaved) hipLaunchKernelGGL((rotary_kernel<bf16_t, true>), grid, block, 0, stream, args);
        else hipLaunchKernelGGL((rotary_kernel<bf16_t, false>), grid, block, 0, stream, args);
    }
    return hipGetLastError();
}

}  // namespace ciar
