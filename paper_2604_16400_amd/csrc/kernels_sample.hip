// Tokens and top logits from rows of logits: selection in the falling order of a row.
//   sample      one token a row from temperature, top-k, top-p, min-p and a given random number
//   top_logits  the K largest logits of a row in order, and the row's log-sum-exp
//
// The order of a row is (logit falling, index rising).  Whatever is asked of a row is a place in that order: the k-th
// logit (counting), the logit at which the weights exp((z - max z) / T) reach p times their sum, the one at which they
// pass u times the sum of those kept.  A place is found without sorting: the logit's bits, made to rise with the value,
// are taken digit by digit (11, 11, 10 bits); for each digit a histogram of what is counted, over the logits that agree
// with the digits found so far, and a running sum over its bins say which digit comes next.  Among equal logits the place is a
// division, and the lowest indices come first.
//
// The sums of weights decide by their last bits which token comes out, so they are exact and in no order: each weight is
// computed in 64 bits and rounded once to a whole multiple of 2^-45 (fewer bits for vocabularies from 2^17 on),
// and whole numbers are added.  Two runs, and any split of the work, give the same token.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernels.h"
#include "vocab_device.h"

namespace collm {

namespace {

using namespace vocab;

typedef unsigned long long u64;

constexpr int kBins = 2048;
constexpr uint32_t kKeyNone = 0x007fffffu;  // key of -inf: nothing at or below it is ever taken
constexpr int kTies = 1024;                 // equal logits that are listed at once

// bits that rise with the value; NaN counts as -inf, -0 as 0
__device__ __forceinline__ uint32_t key_of(float x)
{
    x = (x == x ? x : kNegInf) + 0.0f;
    const uint32_t u = __float_as_uint(x);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t key)
{
    return __uint_as_float(key ^ ((key & 0x80000000u) ? 0x80000000u : 0xffffffffu));
}

// weights of a row as whole numbers
struct Weight {
    double m, c;  // largest logit, log2(e) / T
    int scale;    // a weight of 1 is 2^scale
    bool top_inf;
    __device__ __forceinline__ double log2_of(uint32_t key) const { return ((double)value_of(key) - m) * c; }
    __device__ __forceinline__ u64 operator()(uint32_t key) const
    {
        if (top_inf) return value_of(key) == __builtin_huge_valf() ? (u64)1 << scale : 0;
        // (added to 2^52, the last bit of the sum's fraction is worth 1: the rounding of that sum is the rounding)
        const double w = exp2_neg(log2_of(key), scale) + 4503599627370496.0;
        return (u64)__double_as_longlong(w) & (((u64)1 << 52) - 1);
    }
};

template <int THREADS> struct Shared {
    u64 hist[2][kBins];
    u64 wave_sum[THREADS / kWave];
    double red[THREADS / kWave];
    u64 above;
    int bin;
    uint32_t count;
    uint32_t list[kTies];
};

// The first bin at which the running sum over the bins reaches `goal` (1 <= goal <= total), and the sum before it;
// returns the total.  goal 0: the total alone.
template <int THREADS> __device__ u64 find_bin(Shared<THREADS> &sh, const u64 *hist, u64 goal, int &bin, u64 &above)
{
    constexpr int B = kBins / THREADS;
    u64 own[B], sum = 0;
#pragma unroll
    for (int b = 0; b < B; ++b) sum += own[b] = hist[threadIdx.x * B + b];
    u64 incl = sum;
    const int lane = threadIdx.x & (kWave - 1);
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
        const u64 up = __shfl_up(incl, o);
        if (lane >= o) incl += up;
    }
    if (lane == kWave - 1) sh.wave_sum[threadIdx.x / kWave] = incl;
    __syncthreads();
    u64 total = 0;
#pragma unroll
    for (int w = 0; w < THREADS / kWave; ++w) {
        if (w == (int)(threadIdx.x / kWave)) incl += total;
        total += sh.wave_sum[w];
    }
    u64 run = incl - sum;
    if (goal > run && goal <= incl) {
#pragma unroll
        for (int b = 0; b < B; ++b) {
            if (goal > run && goal <= run + own[b]) {
                sh.bin = threadIdx.x * B + b;
                sh.above = run;
            }
            run += own[b];
        }
    }
    __syncthreads();
    bin = sh.bin;
    above = sh.above;
    __syncthreads();
    return total;
}

// A place in the falling order: the q-th lowest index (from 1) among the logits of this key; `above`: what is counted
// over all greater keys
struct Place {
    uint32_t key;
    uint32_t q;
    u64 above;
};

template <bool BF16, int THREADS> struct Picker {
    Shared<THREADS> &sh;
    const Row<BF16> row;

    __device__ __forceinline__ Picker(Shared<THREADS> &s, const void *p, int vocab) : sh(s), row(p, vocab) {}

    // f(key, index) over the row's logits
    template <typename F> __device__ __forceinline__ void each(F f) const
    {
        for (int c = threadIdx.x; c < row.whole; c += THREADS) {
            const uint4 v = row.body[c];
#pragma unroll
            for (int e = 0; e < Row<BF16>::E; ++e) f(key_of(Row<BF16>::value(v, e)), row.lo + c * Row<BF16>::E + e);
        }
        if ((int)threadIdx.x < row.edges) f(key_of(row.edge(threadIdx.x)), row.edge_index(threadIdx.x));
    }
    __device__ __forceinline__ void clear(u64 *hist) const
    {
        for (int b = threadIdx.x; b < kBins; b += THREADS) hist[b] = 0;
        __syncthreads();
    }
    static constexpr int kLevels = BF16 ? 2 : 3;  // (a bf16 has no bits below the second digit)
    static __device__ __forceinline__ int shift(int level) { return level == 0 ? 21 : level == 1 ? 10 : 0; }
    static __device__ __forceinline__ int bin_of(uint32_t key, int level) { return kBins - 1 - (int)((key >> shift(level)) & (kBins - 1)); }

    // histogram of one digit of the keys that agree with `prefix` above it: what measure(key) gives for each logit, and
    // `extra` once for the key `extra_key`
    template <typename M> __device__ __forceinline__ void histogram(u64 *hist, int level, uint32_t prefix, M measure, uint32_t extra_key, u64 extra) const
    {
        clear(hist);
        const uint32_t mask = level == 0 ? 0u : level == 1 ? 0xffe00000u : 0xfffffc00u;
        auto add = [&](uint32_t key, u64 x) { atomicAdd(&hist[level == 2 ? kBins - 1 - (key & 1023u) : bin_of(key, level)], x); };
        each([&](uint32_t key, int) {
            if (key > kKeyNone && (key & mask) == prefix) {
                const u64 x = measure(key);
                if (x) add(key, x);
            }
        });
        if (extra && threadIdx.x == 0 && (extra_key & mask) == prefix) add(extra_key, extra);
        __syncthreads();
    }
    // The place at which what is counted reaches `goal`.  first: the histogram of the first digit; measure, extra: as
    // there; one(key): what one logit of that key counts.
    template <typename M, typename One>
    __device__ Place find(const u64 *first, u64 goal, M measure, One one, uint32_t extra_key, u64 extra) const
    {
        int bin;
        u64 above, part;
        find_bin<THREADS>(sh, first, goal, bin, above);
        uint32_t prefix = (uint32_t)(kBins - 1 - bin) << 21;
#pragma unroll
        for (int level = 1; level < kLevels; ++level) {
            histogram(sh.hist[1], level, prefix, measure, extra_key, extra);
            find_bin<THREADS>(sh, sh.hist[1], goal - above, bin, part);
            above += part;
            prefix |= (uint32_t)(kBins - 1 - bin) << (level == 1 ? 10 : 0);
        }
        if (BF16 && !(prefix & 0x80000000u)) prefix |= 0x3ffu;
        const u64 w = one(prefix);
        return {prefix, (uint32_t)((goal - above + w - 1) / w), above};
    }
    // the index of the q-th lowest (from 1) of the logits of one key
    __device__ int locate(uint32_t key, uint32_t q) const
    {
        int lo = 0, width = row.n;  // the indices in question
        for (;;) {
            if (threadIdx.x == 0) sh.count = 0;
            __syncthreads();
            each([&](uint32_t k, int i) {
                if (k == key && i >= lo && i - lo < width) {
                    const uint32_t at = atomicAdd(&sh.count, 1u);
                    if (at < kTies) sh.list[at] = (uint32_t)i;
                }
            });
            __syncthreads();
            const uint32_t count = sh.count;
            if (count <= kTies) {
                for (uint32_t t = threadIdx.x; t < count; t += THREADS) {
                    const uint32_t mine = sh.list[t];
                    uint32_t before = 0;
                    for (uint32_t j = 0; j < count; ++j) before += sh.list[j] < mine;
                    if (before == q - 1) sh.bin = (int)mine;
                }
                __syncthreads();
                const int found = sh.bin;
                __syncthreads();
                return found;
            }
            // too many: count them by ranges of indices and go on with the range that holds the q-th
            clear(sh.hist[1]);
            const int step = (width + kBins - 1) / kBins;
            each([&](uint32_t k, int i) {
                if (k == key && i >= lo && i - lo < width) atomicAdd(&sh.hist[1][(i - lo) / step], (u64)1);
            });
            __syncthreads();
            int bin;
            u64 above;
            find_bin<THREADS>(sh, sh.hist[1], q, bin, above);
            q -= (uint32_t)above;
            lo += bin * step;
            width = step;
        }
    }
};

// One block a row.  What bounds it: the passes over the row (read anew in each, from the caches behind the first) and the
// 64-bit exponentials of one of them.
template <bool BF16, int THREADS> __global__ void __launch_bounds__(THREADS) sample_kernel(SampleArgs p)
{
    __shared__ Shared<THREADS> sh;
    const int i = blockIdx.x;
    const void *at = row_of(p.r, i);
    const Picker<BF16, THREADS> pick(sh, at, at ? p.r.vocab : 0);
    float m = kNegInf;
    pick.each([&](uint32_t key, int) { m = fmaxf(m, value_of(key)); });
    m = block_max<THREADS>(m, sh.red);
    int token = -1;
    float logprob = kNegInf;
    if (m > kNegInf) {  // (the same for the whole block, as is every choice below)
        const float T = p.temperature ? p.temperature[i] : 1.0f;
        const int k = p.top_k ? p.top_k[i] : 0;
        const float top_p = p.top_p ? p.top_p[i] : 1.0f;
        const float min_p = p.min_p && p.min_p[i] > 0.0f ? fminf(p.min_p[i], 1.0f) : 0.0f;
        if (!(T > 0.0f) || k == 1) {
            token = pick.locate(key_of(m), 1);
            logprob = 0.0f;
        } else {
            Weight w;
            w.top_inf = m == __builtin_huge_valf();
            w.m = m;
            w.c = 1.44269504088896340736 / (double)T;
            w.scale = 62 - (32 - __builtin_clz((uint32_t)p.r.vocab));
            if (w.scale > 45) w.scale = 45;
            int bin;
            u64 above;
            // top-k: of the key at its edge only the lowest indices count, so many of them that there are k logits
            Place edge = {kKeyNone, 0, 0};
            if (k > 0 && k < p.r.vocab) {
                auto one = [](uint32_t) { return (u64)1; };
                pick.histogram(sh.hist[0], 0, 0, one, 0, 0);
                if (find_bin<THREADS>(sh, sh.hist[0], 0, bin, above) > (u64)k) edge = pick.find(sh.hist[0], k, one, one, 0, 0);
            }
            const u64 extra = edge.q ? w(edge.key) * edge.q : 0;
            auto inside = [&](uint32_t key) { return key > edge.key ? w(key) : (u64)0; };
            // min-p: the least key whose weight it keeps, and the sum of the weights it keeps
            uint32_t key_min = 0;
            if (min_p > 0.0f && !w.top_inf) {
                const double low = w.m + (double)T * log((double)min_p);
                const float f = (float)low;
                key_min = key_of(f) + ((double)f < low ? 1 : 0);
            }
            u64 over = threadIdx.x == 0 && edge.key >= key_min ? extra : 0;
            pick.histogram(sh.hist[0], 0, 0, [&](uint32_t key) {
                const u64 x = inside(key);
                if (key >= key_min) over += x;
                return x;
            }, edge.key, extra);
            u64 kept = find_bin<THREADS>(sh, sh.hist[0], 0, bin, above);
            if (top_p < 1.0f) {
                const double goal = ceil((double)top_p * (double)kept);
                const u64 g = !(goal >= 1.0) ? 1 : goal >= (double)kept ? kept : (u64)goal;
                const Place last = pick.find(sh.hist[0], g, inside, w, edge.key, extra);
                kept = last.above + last.q * w(last.key);
            }
            if (key_min) {
                // (both keep a prefix of the order: the shorter one counts)
                over = block_reduce<u64, THREADS>(over, sh.wave_sum, [](u64 a, u64 b) { return a + b; });
                kept = over < kept ? over : kept;
            }
            const double goal = floor((double)p.u[i] * (double)kept);
            const u64 g = !(goal >= 0.0) ? 1 : goal >= (double)(kept - 1) ? kept : (u64)goal + 1;
            const Place drawn = pick.find(sh.hist[0], g, inside, w, edge.key, extra);
            token = pick.locate(drawn.key, drawn.q);
            logprob = (float)((w.top_inf ? 0.0 : w.log2_of(drawn.key) * 0.69314718055994530942) - log(__builtin_ldexp((double)kept, -w.scale)));
        }
    }
    if (threadIdx.x == 0) {
        p.token[i] = token;
        if (p.logprob) p.logprob[i] = logprob;
    }
}

// One block a row: the k-th place by counting, then the k logits up to it, put in order by counting for each how many
// are before it.
template <bool BF16, int THREADS> __global__ void __launch_bounds__(THREADS) top_kernel(TopArgs p)
{
    __shared__ Shared<THREADS> sh;
    __shared__ u64 taken[kMaxTop];
    const int i = blockIdx.x;
    const void *at = row_of(p.r, i);
    const Picker<BF16, THREADS> pick(sh, at, at ? p.r.vocab : 0);
    float m = kNegInf;
    pick.each([&](uint32_t key, int) { m = fmaxf(m, value_of(key)); });
    m = block_max<THREADS>(m, sh.red);
    if (p.lse) {
        const float inv = 1.0f / p.temperature, ref = m > kNegInf ? m : 0.0f;
        // (of the logits as they are: a NaN among them shows)
        float part = expf((pick.row.edge(threadIdx.x) - ref) * inv);
        for (int c = threadIdx.x; c < pick.row.whole; c += THREADS) {
            const uint4 v = pick.row.body[c];
#pragma unroll
            for (int e = 0; e < Row<BF16>::E; ++e) part += expf((Row<BF16>::value(v, e) - ref) * inv);
        }
        const double sum = block_sum<THREADS>((double)part, sh.red);
        if (threadIdx.x == 0) p.lse[i] = (float)((double)ref / (double)p.temperature + log(sum));
    }
    auto one = [](uint32_t) { return (u64)1; };
    pick.histogram(sh.hist[0], 0, 0, one, 0, 0);
    int bin;
    u64 above;
    const u64 finite = find_bin<THREADS>(sh, sh.hist[0], 0, bin, above);
    uint32_t edge = kKeyNone + 1;  // the least key taken, and its last index
    int last = p.r.vocab;
    if (finite > (u64)p.k) {
        const Place place = pick.find(sh.hist[0], p.k, one, one, 0, 0);
        edge = place.key;
        last = pick.locate(place.key, place.q);
    }
    if (threadIdx.x == 0) sh.count = 0;
    __syncthreads();
    pick.each([&](uint32_t key, int idx) {
        if (key > edge || (key == edge && idx <= last)) {
            const uint32_t to = atomicAdd(&sh.count, 1u);
            if (to < kMaxTop) taken[to] = ((u64)~key << 32) | (uint32_t)idx;
        }
    });
    __syncthreads();
    const int count = (int)sh.count;  // min(k, finite)
    float *values = p.values + (int64_t)i * p.k;
    int32_t *indices = p.indices + (int64_t)i * p.k;
    for (int t = threadIdx.x; t < p.k; t += THREADS) {
        if (t >= count) {
            values[t] = kNegInf;
            indices[t] = -1;
            continue;
        }
        const u64 mine = taken[t];
        int before = 0;
        for (int j = 0; j < count; ++j) before += taken[j] < mine;
        values[before] = value_of(~(uint32_t)(mine >> 32));
        indices[before] = (int32_t)(uint32_t)mine;
    }
}

}  // namespace

hipError_t launch_sample(const SampleArgs &a, hipStream_t st)
{
    if (a.r.bf16) COLLM_LAUNCH((sample_kernel<true, 512>), dim3(a.r.n_rows), dim3(512), 0, st, a);
    else COLLM_LAUNCH((sample_kernel<false, 512>), dim3(a.r.n_rows), dim3(512), 0, st, a);
    return hipGetLastError();
}

hipError_t launch_top_logits(const TopArgs &a, hipStream_t st)
{
    if (a.r.bf16) COLLM_LAUNCH((top_kernel<true, 512>), dim3(a.r.n_rows), dim3(512), 0, st, a);
    else COLLM_LAUNCH((top_kernel<false, 512>), dim3(a.r.n_rows), dim3(512), 0, st, a);
    return hipGetLastError();
}

}  // namespace collm
