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

// A row of logits as the 16-byte chunks of memory that hold it.  Element i of the row is element (i + head) % E of chunk
// (i + head) / E.  The first and the last chunk may hold only a few elements of the row: those are read one by one, as
// nothing outside the row may be.
template <bool BF16> struct Row {
    static constexpr int E = Elem<BF16>::kPerChunk;
    const void *row;  // first element
    int n, head, chunks;

    __device__ __forceinline__ Row(const void *p, int vocab) : row(p), n(vocab)
    {
        head = (int)(((uintptr_t)p & 15u) / (16 / E));
        chunks = (vocab + head + E - 1) / E;
    }
    __device__ __forceinline__ const uint4 *base() const { return (const uint4 *)((uintptr_t)row & ~(uintptr_t)15); }
    __device__ __forceinline__ bool whole(int c) const { return c * E >= head && (c + 1) * E <= n + head; }
    __device__ __forceinline__ uint4 edge(int c) const  // elements outside the row: -inf
    {
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (BF16) {
                const int i = c * E - head + 2 * j;
                uint32_t lo = 0xff80u, hi = 0xff80u;
                if (i >= 0 && i < n) lo = ((const uint16_t *)row)[i];
                if (i + 1 >= 0 && i + 1 < n) hi = ((const uint16_t *)row)[i + 1];
                w[j] = lo | (hi << 16);
            } else {
                const int i = c * E - head + j;
                w[j] = 0xff800000u;
                if (i >= 0 && i < n) w[j] = ((const uint32_t *)row)[i];
            }
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    __device__ __forceinline__ uint4 load(int c) const { return whole(c) ? base()[c] : edge(c); }
    // value of element e of a chunk
    static __device__ __forceinline__ float value(const uint4 &v, int e)
    {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        if (!BF16) return __uint_as_float(w[e]);
        return __uint_as_float((e & 1) ? (w[e >> 1] & 0xffff0000u) : (w[e >> 1] << 16));
    }
};

// first element of row i of a call; NULL where it is not there
__device__ __forceinline__ const void *row_of(const LogitRows &r, int i)
{
    const int64_t at = r.rows ? (int64_t)r.rows[i] : i;
    if (at < 0 || at >= r.n_held) return nullptr;
    return (const char *)r.logits + at * r.ld * (r.bf16 ? 2 : 4);
}

// ---- block-wide reductions (every thread gets the result); `s` holds one value a wave and is free again on return ----
template <typename T, int THREADS, typename F> __device__ __forceinline__ T block_reduce(T v, T *s, F f)
{
#pragma unroll
    for (int o = kWave / 2; o > 0; o >>= 1) v = f(v, __shfl_xor(v, o));
    if (THREADS == kWave) return v;
    if ((threadIdx.x & (kWave - 1)) == 0) s[threadIdx.x / kWave] = v;
    __syncthreads();
    T r = s[0];
#pragma unroll
    for (int w = 1; w < THREADS / kWave; ++w) r = f(r, s[w]);
    __syncthreads();
    return r;
}
template <int THREADS> __device__ __forceinline__ float block_max(float v, double *s)
{
    return block_reduce<float, THREADS>(v, (float *)s, [](float a, float b) { return fmaxf(a, b); });
}
template <int THREADS> __device__ __forceinline__ double block_sum(double v, double *s)
{
    return block_reduce<double, THREADS>(v, s, [](double a, double b) { return a + b; });
}

// 2^t for t <= 0 as p 2^n with the rounded-off fraction in a polynomial: the Taylor series of e^x at x = f ln 2, |f| <= 1/2,
// to the power 12 (next term 2.4e-16); 0 for t below -1000
__device__ __forceinline__ double exp2_neg(double t, int scale)
{
    const double n = __builtin_rint(t);
    const double x = (t - n) * 0.69314718055994530942;
    double p = 1.0 / 479001600.0;
    p = __builtin_fma(p, x, 1.0 / 39916800.0);
    p = __builtin_fma(p, x, 1.0 / 3628800.0);
    p = __builtin_fma(p, x, 1.0 / 362880.0);
    p = __builtin_fma(p, x, 1.0 / 40320.0);
    p = __builtin_fma(p, x, 1.0 / 5040.0);
    p = __builtin_fma(p, x, 1.0 / 720.0);
    p = __builtin_fma(p, x, 1.0 / 120.0);
    p = __builtin_fma(p, x, 1.0 / 24.0);
    p = __builtin_fma(p, x, 1.0 / 6.0);
    p = __builtin_fma(p, x, 0.5);
    p = __builtin_fma(p, x, 1.0);
    p = __builtin_fma(p, x, 1.0);
    return t < -1000.0 ? 0.0 : __builtin_ldexp(p, (int)n + scale);
}

}  // namespace vocab
}  // namespace collm
