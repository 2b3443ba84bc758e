// Device code that the vocabulary operators share: rows of any alignment in 16-byte chunks, block-wide sums, exponentials.
#pragma once
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "vocab.h"

namespace collm {
namespace vocab {

constexpr int kWave = 64;
constexpr float kNegInf = -__builtin_huge_valf();

__device__ __forceinline__ float bf16_to_f32(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    typedef float floatx2 __attribute__((ext_vector_type(2)));
    floatx2 v = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}

template <bool BF16> struct Elem;
template <> struct Elem<true> {
    typedef uint16_t type;
    static constexpr int kPerChunk = 8;
    static __device__ __forceinline__ float load(const void *row, int64_t i) { return bf16_to_f32(((const uint16_t *)row)[i]); }
    static __device__ __forceinline__ void store(void *row, int64_t i, float v) { ((uint16_t *)row)[i] = (uint16_t)pack_bf16(v, 0.f); }
};
template <> struct Elem<false> {
    typedef float type;
    static constexpr int kPerChunk = 4;
    static __device__ __forceinline__ float load(const void *row, int64_t i) { return ((const float *)row)[i]; }
    static __device__ __forceinline__ void store(void *row, int64_t i, float v) { ((float *)row)[i] = v; }
};

// A row of logits as the whole 16-byte chunks of memory inside it and the few elements before and behind them, its edges
// (fewer than a chunk on either side).  Element e of chunk c is element lo + c E + e of the row; edge t, which thread t
// takes, is element t (t < lo) or whole E + t.
template <bool BF16> struct Row {
    static constexpr int E = Elem<BF16>::kPerChunk;
    const void *row;   // first element
    const uint4 *body; // first whole chunk
    int n, lo, whole, edges;

    __device__ __forceinline__ Row(const void *p, int vocab) : row(p), n(vocab)
    {
        const int head = (int)(((uintptr_t)p & 15u) / (16 / E));
        lo = (E - head) % E;
        if (lo > n) lo = n;
        whole = (n - lo) / E;
        edges = n - whole * E;
        body = (const uint4 *)((const char *)p + lo * (16 / E));
    }
    // the whole chunks as a buffer: reads beyond them give 0
    __device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer() const
    {
        return __builtin_amdgcn_make_buffer_rsrc((void *)body, 0, whole * 16, 0x00020000);
    }
    __device__ __forceinline__ int edge_index(int t) const { return t < lo ? t : whole * E + t; }
    __device__ __forceinline__ float edge(int t) const { return t < edges ? Elem<BF16>::load(row, edge_index(t)) : kNegInf; }
    // a number for each element: chunk by chunk, then the edges
    __device__ __forceinline__ int bit(int i) const
    {
        if (i < lo) return whole * E + i;
        return i < lo + whole * E ? i - lo : i;
    }
    // value of element e of a chunk
    static __device__ __forceinline__ float value(const uint4 &v, int e)
    {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        if (!BF16) return __uint_as_float(w[e]);
        return __uint_as_float((e & 1) ? (w[e >> 1] & 0xffff0000u) : (w[e >> 1] << 16));
    }
    static __device__ __forceinline__ uint4 chunk(const float (&g)[8])
    {
        if (!BF16) return make_uint4(__float_as_uint(g[0]), __float_as_uint(g[1]), __float_as_uint(g[2]), __float_as_uint(g[3]));
        return make_uint4(pack_bf16(g[0], g[1]), pack_bf16(g[2], g[3]), pack_bf16(g[4], g[5]), pack_bf16(g[6], g[7]));
    }
};

// first element of row i of a call; NULL where it is not there
__device__ __forceinline__ const void *row_of(const LogitRows &r, int i)
{
    const int64_t at = r.rows ? (int64_t)__builtin_amdgcn_readfirstlane(r.rows[i]) : i;
    if (at < 0 || at >= r.n_held) return nullptr;
    return (const char *)r.logits + at * r.ld * (r.bf16 ? 2 : 4);
}

// ---- block-wide reductions (every thread gets the result, in scalar registers); `s` holds one value a wave and is free again on return ----
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ float uniform(float v) { return __uint_as_float(uniform(__float_as_uint(v))); }
__device__ __forceinline__ unsigned long long uniform(unsigned long long v)
{
    return (unsigned long long)uniform((uint32_t)(v >> 32)) << 32 | uniform((uint32_t)v);
}
__device__ __forceinline__ double uniform(double v) { return __longlong_as_double((long long)uniform((unsigned long long)__double_as_longlong(v))); }

template <typename T, int THREADS, typename F> __device__ __forceinline__ T block_reduce(T v, T *s, F f)
{
    constexpr int W = THREADS / kWave;
#pragma unroll
    for (int o = kWave / 2; o > 0; o >>= 1) v = f(v, __shfl_xor(v, o));
    if (W == 1) return uniform(v);
    const int lane = threadIdx.x & (kWave - 1);
    if (lane == 0) s[threadIdx.x / kWave] = v;
    __syncthreads();
    v = s[lane & (W - 1)];
#pragma unroll
    for (int o = W / 2; o > 0; o >>= 1) v = f(v, __shfl_xor(v, o));
    __syncthreads();
    return uniform(v);
}
template <int THREADS> __device__ __forceinline__ float block_max(float v, double *s)
{
    return block_reduce<float, THREADS>(v, (float *)s, [](float a, float b) { return fmaxf(a, b); });
}
template <int THREADS> __device__ __forceinline__ double block_sum(double v, double *s)
{
    return block_reduce<double, THREADS>(v, s, [](double a, double b) { return a + b; });
}

// 2^t 2^scale as p 2^n, n the nearest integer to t; p(f) = 1 + f q(f) on |f| <= 1/2 with q of degree 7, its coefficients fitted to
// (2^f - 1) / f by least squares with weights raised until the relative error was the same at all its peaks: 8.2e-13.  0 for t below -1000.
__device__ __forceinline__ double exp2_neg(double t, int scale)
{
    const double n = __builtin_rint(t);
    const double f = t - n;
    double p = 1.3178929944324011e-06;
    p = __builtin_fma(p, f, 1.5309156437291593e-05);
    p = __builtin_fma(p, f, 0.00015403825481710473);
    p = __builtin_fma(p, f, 0.0013333454859321126);
    p = __builtin_fma(p, f, 0.00961812861609056);
    p = __builtin_fma(p, f, 0.05550410935267852);
    p = __builtin_fma(p, f, 0.24022650698110812);
    p = __builtin_fma(p, f, 0.6931471805482116);
    p = __builtin_fma(p, f, 1.0);
    return t < -1000.0 ? 0.0 : __builtin_ldexp(p, (int)n + scale);
}

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
constexpr float kLow = -3.402823466e+38f;  // the least finite value: a running maximum begins here, so that -inf adds nothing

// Between writes to shared memory by a wave's lanes and reads of them by other lanes of that wave (and the other way round)
__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
}

template <typename T, typename F> __device__ __forceinline__ T wave_reduce(T v, F f)
{
#pragma unroll
    for (int o = kWave / 2; o > 0; o >>= 1) v = f(v, __shfl_xor(v, o));
    return v;
}
template <typename T> __device__ __forceinline__ T wave_sum(T v)
{
    return wave_reduce(v, [](T a, T b) { return a + b; });
}
__device__ __forceinline__ float wave_max(float v)
{
    return wave_reduce(v, [](float a, float b) { return fmaxf(a, b); });
}

// Cache policy of loads and stores that nothing reads again before the last-level cache has lost them: past it.
constexpr int kOnce = 2;
template <bool ONCE> __device__ __forceinline__ uint4 load_chunk(__amdgpu_buffer_rsrc_t row, int c)
{
    return __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(row, c * 16, 0, ONCE ? kOnce : 0));
}

// exp((z - ref) / tau).  The rounding of c and of the argument are errors of |z - ref| / tau 2^-24 each, small where the result is not.
// near: 2^32 times that, for sums and gradients of a whole row; what is below 2^-126 is lost, 2^-158 here.  With bf16 logits it is exp2(z c + b), one
// operation an element fewer than from the difference, with b = 32 - ref c rounded beforehand: the same factor 2^drift in every term, taken out
// in 64 bits.  The argument is about 32 at the largest terms and rounded to 2^-20 there, an error of 7e-7: for fp32 logits it is the square
// of an exponential of half the difference.
template <bool BF16> struct Exp {
    float c, ref, b;
    __device__ __forceinline__ Exp(float tau, float r) : c(uniform((float)(1.44269504088896340736 / (double)tau))), ref(r), b(__builtin_fmaf(-r, c, 32.f)) {}
    __device__ __forceinline__ void refer(float r)  // to another reference
    {
        ref = r;
        b = __builtin_fmaf(-r, c, 32.f);
    }
    __device__ __forceinline__ float near(float z) const
    {
        if (BF16) return __builtin_amdgcn_exp2f(__builtin_fmaf(z, c, b));
        const float half = __builtin_amdgcn_exp2f((z - ref) * (0.5f * c));
        return half * 0x1p32f * half;
    }
    __device__ __forceinline__ float operator()(float z) const { return __builtin_amdgcn_exp2f((z - ref) * c); }
    __device__ __forceinline__ double drift() const { return BF16 ? (double)ref * (double)c + (double)b : 32.0; }  // 32, about
    __device__ __forceinline__ bool sound() const { return fabs(drift() - 32.0) < 1.0; }                            // no more than rounding
};

// A thread's running sums: exp((z - m) / tau) and exp(z - m) over the logits it has met, m the largest of them.  A chunk's terms are added in 32
// bits, chunks in 64: in 32 the roundings of a long sum of like terms all go one way (3e-5 after 4096 chunks).
struct Running {
    float m = kLow;
    double s = 0.0, ce = 0.0;
    // (to a larger reference)
    __device__ __forceinline__ void raise(float to, float c)
    {
        s *= (double)__builtin_amdgcn_exp2f((m - to) * c);
        ce *= (double)__builtin_amdgcn_exp2f((m - to) * 1.44269504f);
        m = to;
    }
    template <int N> __device__ __forceinline__ void add(const float (&z)[N], float c)
    {
        float top = m;
#pragma unroll
        for (int e = 0; e < N; ++e) top = fmaxf(top, z[e]);
        raise(top, c);
        float part = 0.f, part_ce = 0.f;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            part += __builtin_amdgcn_exp2f((z[e] - m) * c);
            part_ce += __builtin_amdgcn_exp2f((z[e] - m) * 1.44269504f);
        }
        s += (double)part;
        ce += (double)part_ce;
    }
};

}  // namespace vocab
}  // namespace collm
