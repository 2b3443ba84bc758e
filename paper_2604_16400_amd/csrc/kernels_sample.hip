// Tokens and top logits from rows of logits: selection in the falling order of a row.
//   sample      one token a row from temperature, top-k, top-p, min-p and a given random number
//   top_logits  the K largest logits of a row in order, and the row's log-sum-exp
//
// The order of a row is (logit falling, index rising), and whatever is asked of a row lies near its beginning: the k-th logit, the
// logit at which the weights exp((z - max z) / T) reach p times their sum, the one at which they pass u times the sum of those kept.
// One pass over the row lists its beginning and adds up the rest: a logit is listed if it is not below a bound which at least
// `want` logits reach, taken from the threads' largest logits so far (the least, over the waves, of the (want / waves)-th largest of
// a wave's 64).  The list, a few times `want`, is put in order by a counting sort over equal steps of the logit, and all
// that is asked is read off it in 64 bits.  The sum of the rest need only be near: where its error could change what comes out, and where the
// list does not reach far enough, the row is done by digits instead (below): exact for every row, in more passes.
//
// By digits: the logit's bits, made to rise with the value, are taken 11, 11 and 10 at a time; for each digit a
// histogram of what is counted (logits, or their weights), over the logits that agree with the digits found so far, and a running sum over its
// bins say which digit comes next.  Among equal logits the place is a division, and the lowest indices come first.
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

constexpr int kList = 4096;   // logits listed of a row
constexpr int kSteps = 1024;  // of the logit, in the counting sort

template <int THREADS> struct Shared {
    union {
        struct {  // by digits
            u64 hist[2][kBins];
            uint32_t list[kTies];
        };
        struct {  // by the list
            u64 listed[kList], binned[kList];  // ~key above, index below: rising is the order of the row
            int start[kSteps + 1], fill[kSteps];
        };
    };
    u64 wave_sum[THREADS / kWave];
    double red[THREADS / kWave];
    float low[2][THREADS / kWave], top[THREADS / kWave];
    u64 above;
    int bin;
    uint32_t count;
    int reach, cut_p[2], cut_m, drawn;
    u64 kept;
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

// Token and its log probability by digits: every row, whatever its logits.
template <bool BF16, int THREADS> __device__ void sample_by_digits(Shared<THREADS> &sh, const SampleArgs &p, int i, const void *at, int &token, float &logprob)
{
    const Picker<BF16, THREADS> pick(sh, at, p.r.vocab);
    float m = kNegInf;
    pick.each([&](uint32_t key, int) { m = fmaxf(m, value_of(key)); });
    m = block_max<THREADS>(m, sh.red);
    token = -1;
    logprob = kNegInf;
    if (!(m > kNegInf)) return;  // (the same for the whole block, as is every choice below)
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

// What the one pass found
struct Found {
    int count;    // listed
    float bound;  // everything from here on is listed (below it only some of the logits met early)
    bool whole;   // every logit above -inf is listed
    double rest;  // sum of exp((z - ref) / T) over what is not listed
    float ref;
    bool ok;      // the list is not too long (and what it is sorted by is a number)
    bool summed;  // `rest` is right but for 2^-17 of it
};

// The least value of which at least `rank` of the wave's lanes have as much, but for its last 16 bits (0: nothing above -inf)
__device__ __forceinline__ uint32_t rank_in_wave(float v, int rank)
{
    const uint32_t key = key_of(v) >> 16;
    uint32_t at = 0;
#pragma unroll
    for (int b = 15; b >= 0; --b) {
        const uint32_t next = at | 1u << b;
        if (__popcll(__ballot(key >= next)) >= rank) at = next;
    }
    return at << 16;
}

// Lists the beginning of the row, at least `want` logits where there are as many, and sums the rest (if `sums`).
template <bool BF16, int THREADS> __device__ Found list_row(Shared<THREADS> &sh, const Row<BF16> &row, int want, bool sums, float tau)
{
    constexpr int E = Row<BF16>::E, U = 4, W = THREADS / kWave, kRound = U * THREADS;
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int rank = (want + W - 1) / W < kWave ? (want + W - 1) / W : kWave;
    if (threadIdx.x == 0) sh.count = 0;
    const __amdgpu_buffer_rsrc_t from = row.buffer();
    const float edge_z = row.edge(threadIdx.x);
    uint4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = load_chunk<false>(from, u * THREADS + threadIdx.x);
    float top = fmaxf(edge_z, kNegInf), bound = kLow;
    double rest = 0.0;
    Exp by_T(tau, 0.f);
    auto take = [&](float z, int idx) {
        const uint32_t to = atomicAdd(&sh.count, 1u);
        if (to < kList) sh.listed[to] = ((u64)~key_of(z) << 32) | (uint32_t)idx;
    };
    for (int r = 0, c = threadIdx.x; r == 0 || r * kRound < row.whole; ++r, c += kRound) {
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (c + u * THREADS < row.whole) {
#pragma unroll
                for (int e = 0; e < E; ++e) top = fmaxf(top, Row<BF16>::value(v[u], e));
            }
        const uint32_t key = rank_in_wave(top, rank);
        if (lane == 0) sh.low[r & 1][wave] = key > kKeyNone ? value_of(key) : kLow;
        if (r == 0) {
            const float m = wave_max(top);
            if (lane == 0) sh.top[wave] = m;
        }
        __syncthreads();
        bound = uniform(-wave_max(-sh.low[r & 1][lane & (W - 1)]));
        bound = fmaxf(bound, kLow);
        if (r == 0) {
            const float m = uniform(wave_max(sh.top[lane & (W - 1)]));
            by_T = Exp(tau, m > kNegInf ? m : 0.f);
            float z = edge_z;
            if (z >= bound) {
                take(z, row.edge_index(threadIdx.x));
                z = kNegInf;
            }
            if (sums) rest += (double)by_T.near(z);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (c + u * THREADS < row.whole) {
                float z[E], m = kNegInf, s = 0.f;
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    z[e] = Row<BF16>::value(v[u], e);
                    m = fmaxf(m, z[e]);
                }
                if (m >= bound) {
                    const int first = row.lo + (c + u * THREADS) * E;
#pragma unroll
                    for (int e = 0; e < E; ++e)
                        if (z[e] >= bound) {
                            take(z[e], first + e);
                            z[e] = kNegInf;
                        }
                }
                if (sums) {
#pragma unroll
                    for (int e = 0; e < E; ++e) s += by_T.near(z[e]);
                    rest += (double)s;
                }
            }
            v[u] = load_chunk<false>(from, c + kRound + u * THREADS);
        }
    }
    rest = sums ? block_sum<THREADS>(rest, sh.red) : 0.0;
    __syncthreads();
    Found f;
    f.count = (int)uniform(sh.count);
    f.bound = bound;
    f.whole = bound == kLow;
    f.ref = by_T.ref;
    f.rest = rest * exp2_neg(-by_T.drift(), 0);
    f.ok = f.count <= kList;
    f.summed = rest < 1e30 && fabs(by_T.drift() - 32.0) < 1.0;
    return f;
}

// Puts the list in order: a counting sort by equal steps of the logit, then each entry behind those of its step that are before it.
template <int THREADS> __device__ bool sort_list(Shared<THREADS> &sh, int count)
{
    constexpr int W = THREADS / kWave, N = kList / THREADS, B = kSteps / THREADS;
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    auto z_of = [](u64 x) { return value_of(~(uint32_t)(x >> 32)); };
    u64 mine[N];
    float top = kNegInf, low = __builtin_huge_valf();
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const int e = n * THREADS + threadIdx.x;
        if (e < count) {
            mine[n] = sh.listed[e];
            top = fmaxf(top, z_of(mine[n]));
            low = fminf(low, z_of(mine[n]));
        }
    }
    top = wave_max(top);
    low = -wave_max(-low);
    if (lane == 0) {
        sh.top[wave] = top;
        sh.low[0][wave] = low;
    }
#pragma unroll
    for (int b = 0; b < B; ++b) sh.fill[b * THREADS + threadIdx.x] = 0;
    __syncthreads();
    top = uniform(wave_max(sh.top[lane & (W - 1)]));
    low = uniform(-wave_max(-sh.low[0][lane & (W - 1)]));
    const float width = top - low;
    if (!(width < __builtin_huge_valf())) return false;
    const float scale = width > 0.f ? (float)(kSteps - 1) / width : 0.f;
    if (!(scale < __builtin_huge_valf())) return false;
    auto step_of = [&](u64 x) { return (int)fminf((top - z_of(x)) * scale, (float)(kSteps - 1)); };
#pragma unroll
    for (int n = 0; n < N; ++n)
        if (n * THREADS + (int)threadIdx.x < count) atomicAdd(&sh.fill[step_of(mine[n])], 1);
    __syncthreads();
    int own[B], sum = 0;
#pragma unroll
    for (int b = 0; b < B; ++b) sum += own[b] = sh.fill[threadIdx.x * B + b];
    int incl = sum;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
        const int up = __shfl_up(incl, o);
        if (lane >= o) incl += up;
    }
    if (lane == kWave - 1) sh.wave_sum[wave] = (u64)incl;
    __syncthreads();
    int run = incl - sum;
#pragma unroll
    for (int w = 0; w < W; ++w)
        if (w < wave) run += (int)sh.wave_sum[w];
#pragma unroll
    for (int b = 0; b < B; ++b) {
        sh.start[threadIdx.x * B + b] = run;
        sh.fill[threadIdx.x * B + b] = run;
        run += own[b];
    }
    if (threadIdx.x == THREADS - 1) sh.start[kSteps] = run;
    __syncthreads();
#pragma unroll
    for (int n = 0; n < N; ++n)
        if (n * THREADS + (int)threadIdx.x < count) sh.binned[atomicAdd(&sh.fill[step_of(mine[n])], 1)] = mine[n];
    __syncthreads();
#pragma unroll
    for (int n = 0; n < N; ++n) {
        if (n * THREADS + (int)threadIdx.x < count) {
            const u64 x = mine[n];
            const int b = step_of(x), lo = sh.start[b], hi = sh.start[b + 1];
            int at = lo;
            for (int j = lo; j < hi; ++j) at += sh.binned[j] < x;
            sh.listed[at] = x;
        }
    }
    __syncthreads();
    return true;
}

// One block a row.  What bounds it: one pass over the row, and the latency of the steps behind it.
template <bool BF16, int THREADS> __global__ void __launch_bounds__(THREADS, 8) sample_kernel(SampleArgs p)
{
    constexpr int N = kList / THREADS, W = THREADS / kWave;
    __shared__ Shared<THREADS> sh;
    const int i = blockIdx.x, lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const void *at = row_of(p.r, i);
    const Row<BF16> row(at, at ? p.r.vocab : 0);
    const float T = uniform(p.temperature ? p.temperature[i] : 1.0f);
    int k = (int)uniform((uint32_t)(p.top_k ? p.top_k[i] : 0));
    const float top_p = uniform(p.top_p ? p.top_p[i] : 1.0f);
    float min_p = uniform(p.min_p ? p.min_p[i] : 0.0f);
    min_p = min_p > 0.0f ? fminf(min_p, 1.0f) : 0.0f;
    const bool greedy = !(T > 0.0f) || k == 1;
    if (k <= 0 || k >= p.r.vocab) k = 0;
    // (of a nucleus or a row that nothing cuts the beginning is 128 logits: where its weights leave too much to the rest, by digits)
    const int want = greedy ? 1 : k ? (k < kTies ? k : kTies) : 128;
    const bool sums = !greedy && !k;
    const Found f = list_row<BF16, THREADS>(sh, row, want, sums, greedy ? 1.0f : T);
    int token = -1;
    float logprob = kNegInf;
    bool done = f.ok && f.count == 0;  // nothing above -inf
    if (!done && f.ok && (!sums || f.summed) && (!k || f.count >= k || f.whole) && sort_list<THREADS>(sh, f.count)) {
        const float m = value_of(~(uint32_t)(sh.listed[0] >> 32));
        if (greedy) {
            token = (int)(uint32_t)sh.listed[0];
            logprob = 0.0f;
            done = true;
        } else if (m < __builtin_huge_valf()) {
            Weight w;
            w.top_inf = false;
            w.m = m;
            w.c = 1.44269504088896340736 / (double)T;
            w.scale = 62 - (32 - __builtin_clz((uint32_t)p.r.vocab));
            if (w.scale > 45) w.scale = 45;
            // weights of the list, and their running sum; thread t has entries N t .. N t + N - 1.  The list reaches as far as
            // the bound: what was listed below it belongs to the rest.
            if (threadIdx.x == 0) sh.reach = f.count;
            __syncthreads();
            u64 own[N], sum = 0, below = 0;
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const int e = threadIdx.x * N + n;
                const uint32_t key = e < f.count ? ~(uint32_t)(sh.listed[e] >> 32) : 0;
                if (e < f.count && value_of(key) < f.bound) atomicMin(&sh.reach, e);
            }
            __syncthreads();
            const int n_k = k && k < sh.reach ? k : sh.reach;
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const int e = threadIdx.x * N + n;
                const u64 x = e < (k ? n_k : f.count) ? w(~(uint32_t)(sh.listed[e] >> 32)) : 0;
                own[n] = e < n_k ? x : 0;
                below += e < n_k ? 0 : x;
                sum += own[n];
            }
            if (sums) below = block_reduce<u64, THREADS>(below, sh.wave_sum, [](u64 a, u64 b) { return a + b; });
            u64 incl = sum;
#pragma unroll
            for (int o = 1; o < kWave; o <<= 1) {
                const u64 up = __shfl_up(incl, o);
                if (lane >= o) incl += up;
            }
            if (lane == kWave - 1) sh.wave_sum[wave] = incl;
            if (threadIdx.x == 0) {
                sh.cut_p[0] = sh.cut_p[1] = sh.cut_m = n_k;
                sh.drawn = -1;
            }
            __syncthreads();
            u64 listed = 0;
#pragma unroll
            for (int j = 0; j < W; ++j) {
                if (j == wave) incl += listed;
                listed += sh.wave_sum[j];
            }
            const u64 first = incl - sum;
            // what the row's weights sum to, at least and at most
            const double rest = sums ? f.rest * exp2_neg(((double)f.ref - (double)m) * w.c, w.scale) + (double)below : 0.0;
            const double all[2] = {(double)listed + rest * (1.0 - 0x1p-17), (double)listed + rest * (1.0 + 0x1p-17)};
            const double low = (double)m + (double)T * log((double)min_p);
            if (top_p < 1.0f || min_p > 0.0f) {
                u64 before = first;
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    const int e = threadIdx.x * N + n;
                    if (e > 0 && e < n_k) {
#pragma unroll
                        for (int a = 0; a < 2; ++a)
                            if (top_p < 1.0f && (double)before >= (double)top_p * all[a]) atomicMin(&sh.cut_p[a], e);
                        if (min_p > 0.0f && (double)value_of(~(uint32_t)(sh.listed[e] >> 32)) < low) atomicMin(&sh.cut_m, e);
                    }
                    before += own[n];
                }
                __syncthreads();
            }
            const int cut_p = sh.cut_p[0], cut_m = sh.cut_m, n = cut_p < cut_m ? cut_p : cut_m;
            // the list has to reach the cut: as the end of the top-k, of the row, or because something cuts before its end (for certain)
            const bool ends = n < n_k || k || f.whole;
            const bool open = !ends && !(top_p < 1.0f) && !(min_p > 0.0f);  // nothing cuts at all
            if ((ends || open) && (sh.cut_p[0] == sh.cut_p[1] || n < cut_p)) {
                // the weights kept
                u64 before = first;
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    before += own[j];
                    if ((int)threadIdx.x * N + j == n - 1) sh.kept = before;
                }
                __syncthreads();
                const u64 kept = sh.kept;
                const double u = (double)p.u[i];
                // the draw: the first entry whose running sum passes `goal`, for both ends of what the sum may be
                int drawn[2];
#pragma unroll
                for (int a = 0; a < 2; ++a) {
                    const double of = ends ? (double)kept : all[a];
                    const double goal = u * of;
                    before = first;
                    if (a == 1) __syncthreads();
                    u64 g = !(goal >= 0.0) ? 0 : (u64)goal;  // (passes: more than that, whole)
                    if (ends && g >= kept) g = kept - 1;
#pragma unroll
                    for (int j = 0; j < N; ++j) {
                        if (before <= g && g < before + own[j]) sh.drawn = threadIdx.x * N + j;
                        before += own[j];
                    }
                    __syncthreads();
                    drawn[a] = sh.drawn;
                    if (g >= listed) drawn[a] = -1;  // beyond the list
                }
                if (drawn[0] >= 0 && drawn[0] == drawn[1]) {
                    const u64 x = sh.listed[drawn[0]];
                    token = (int)(uint32_t)x;
                    const double of = ends ? (double)kept : 0.5 * (all[0] + all[1]);
                    logprob = (float)(w.log2_of(~(uint32_t)(x >> 32)) * 0.69314718055994530942 - log(__builtin_ldexp(of, -w.scale)));
                    done = true;
                }
            }
        }
    }
    if (!done) {
        __syncthreads();
        sample_by_digits<BF16, THREADS>(sh, p, i, at, token, logprob);
    }
    if (threadIdx.x == 0) {
        p.token[i] = token;
        if (p.logprob) p.logprob[i] = logprob;
    }
}

// One block a row, as above; a list that is too long: by digits, the k-th place by counting, then the k logits up to it.
template <bool BF16, int THREADS> __global__ void __launch_bounds__(THREADS, 8) top_kernel(TopArgs p)
{
    __shared__ Shared<THREADS> sh;
    const int i = blockIdx.x;
    const void *at = row_of(p.r, i);
    const Row<BF16> row(at, at ? p.r.vocab : 0);
    Found f = list_row<BF16, THREADS>(sh, row, p.k, p.lse != nullptr, p.temperature);
    double sum = 0.0;  // of exp((z - ref) / temperature)
    bool sorted = f.ok && (f.count >= p.k || f.whole) && sort_list<THREADS>(sh, f.count);
    if (p.lse && f.ok && f.summed) {
        const double c = 1.44269504088896340736 / (double)p.temperature;
        for (int e = threadIdx.x; sorted && e < f.count; e += THREADS)
            sum += exp2_neg(((double)value_of(~(uint32_t)(sh.listed[e] >> 32)) - (double)f.ref) * c, 0);
    }
    if (p.lse && !(sorted && f.summed)) {
        // (relative to each thread's largest logit; of the logits as they are: a NaN among them shows)
        Running run;
        const float c = (float)(1.44269504088896340736 / (double)p.temperature), edge[1] = {row.edge(threadIdx.x)};
        run.add(edge, c);
        for (int k = threadIdx.x; k < row.whole; k += THREADS) {
            const uint4 v = row.body[k];
            float z[Row<BF16>::E];
#pragma unroll
            for (int e = 0; e < Row<BF16>::E; ++e) z[e] = Row<BF16>::value(v, e);
            run.add(z, c);
        }
        f.ref = block_max<THREADS>(run.m, sh.red);
        run.raise(f.ref, c);
        sum = (double)run.s;
        f.rest = 0.0;
    }
    if (p.lse) {
        sum = block_sum<THREADS>(sum, sh.red) + f.rest;
        if (threadIdx.x == 0) p.lse[i] = (float)((double)f.ref / (double)p.temperature + log(sum));
    }
    if (!sorted) {
        __syncthreads();
        const Picker<BF16, THREADS> pick(sh, at, row.n);
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
                if (to < kMaxTop) sh.binned[to] = ((u64)~key << 32) | (uint32_t)idx;
            }
        });
        __syncthreads();
        f.count = (int)sh.count;  // min(k, finite)
        for (int t = threadIdx.x; t < f.count; t += THREADS) {
            const u64 x = sh.binned[t];
            int before = 0;
            for (int j = 0; j < f.count; ++j) before += sh.binned[j] < x;
            sh.listed[before] = x;
        }
        __syncthreads();
    }
    float *values = p.values + (int64_t)i * p.k;
    int32_t *indices = p.indices + (int64_t)i * p.k;
    for (int t = threadIdx.x; t < p.k; t += THREADS) {
        const bool there = t < f.count;
        const u64 x = there ? sh.listed[t] : 0;
        values[t] = there ? value_of(~(uint32_t)(x >> 32)) : kNegInf;
        indices[t] = there ? (int32_t)(uint32_t)x : -1;
    }
}

}  // namespace

hipError_t launch_sample(const SampleArgs &a, hipStream_t st)
{
    if (a.r.bf16) COLLM_LAUNCH((sample_kernel<true, 1024>), dim3(a.r.n_rows), dim3(1024), 0, st, a);
    else COLLM_LAUNCH((sample_kernel<false, 1024>), dim3(a.r.n_rows), dim3(1024), 0, st, a);
    return hipGetLastError();
}

hipError_t launch_top_logits(const TopArgs &a, hipStream_t st)
{
    if (a.r.bf16) COLLM_LAUNCH((top_kernel<true, 1024>), dim3(a.r.n_rows), dim3(1024), 0, st, a);
    else COLLM_LAUNCH((top_kernel<false, 1024>), dim3(a.r.n_rows), dim3(1024), 0, st, a);
    return hipGetLastError();
}

}  // namespace collm
