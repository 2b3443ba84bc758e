// Tokens and top logits from rows of logits: selection in the falling order of a row.
//   sample      one token a row from temperature, top-k, top-p, min-p and a given random number
//   top_logits  the K largest logits of a row in order, and the row's log-sum-exp
//
// The order of a row is (logit falling, index rising), and whatever is asked of a row lies near its beginning: the k-th logit, the
// logit at which the weights exp((z - max z) / T) reach p times their sum, the one at which they pass u times the sum of those kept.
// One pass over the row lists its beginning and adds up the rest: a logit is listed if it is not below a bound which at least
// `want` logits reach, taken from the threads' largest logits so far (the least, over the waves, of the (want / waves)-th largest of
// a wave's 64).  The list, a few times `want`, is put in order by a counting sort over equal steps of the logit, and all
// that is asked is read off it in 64 bits.  The sum of the rest need only be near: where its error, with the rounding of every weight in it, could change
// what comes out, and where the list does not reach far enough, the row is done by steps instead: exact for every row, in more passes.
//
// Rows of bf16 that are cut by their weights are not listed: they have few different logits.  One pass counts each (of either sign those of
// 32 octaves, 2^-15 to 2^17; what lies nearer to 0 is listed), a weight is computed once for each that occurs, and a running sum
// over them gives every place.  Only the token's index needs the row again.
//
// By steps: a histogram of what is counted (logits, or their weights) over equal steps of the logit and a running sum over it say in
// which step a place lies; the logits of that step are listed, or, if they are too many, taken by smaller steps of their bits.
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

constexpr int kBins = 2048;                 // steps of a histogram
constexpr int kSlots = 8192;                // logits that are counted by value
constexpr uint32_t kKeyNone = 0x007fffffu;  // key of -inf: nothing at or below it is ever taken
constexpr int kList = 4096;                 // logits listed of a row
constexpr int kSteps = 1024;                // of the logit, in the counting sort
constexpr int kQueue = 1536;                // chunks with logits to list
constexpr int kMost = 256;                  // logits that a row is asked to list
constexpr int kShort = 192;                  // entries of a list that is put in order without steps
constexpr int kFew = 512;                   // logits of one step that are listed

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

// A logit of the row in 64 bits: rising is the order of the row
__device__ __forceinline__ u64 entry(uint32_t key, int index) { return (u64)~key << 32 | (uint32_t)index; }
__device__ __forceinline__ uint32_t key_in(u64 entry) { return ~(uint32_t)(entry >> 32); }
__device__ __forceinline__ float value_in(u64 entry) { return value_of(key_in(entry)); }
__device__ __forceinline__ int index_in(u64 entry) { return (int)(uint32_t)entry; }

// weights of a row as whole numbers
struct Weight {
    double m, c;  // largest logit, log2(e) / T
    int scale;    // a weight of 1 is 2^scale
    bool top_inf;
    __device__ __forceinline__ double log2_of(uint32_t key) const { return ((double)value_of(key) - m) * c; }
    __device__ __forceinline__ u64 operator()(uint32_t key) const { return of(value_of(key)); }
    // (of a logit above -inf)
    __device__ __forceinline__ u64 of(float z) const
    {
        if (top_inf) return z == __builtin_huge_valf() ? (u64)1 << scale : 0;
        return finite(z);
    }
    // (where the largest logit is finite)
    __device__ __forceinline__ u64 finite(float z) const
    {
        // (added to 2^52, the last bit of the sum's fraction is worth 1: the rounding of that sum is the rounding)
        const double w = exp2_neg(((double)z - m) * c, scale) + 4503599627370496.0;
        return (u64)__double_as_longlong(w) & (((u64)1 << 52) - 1);
    }
};

template <int THREADS> struct Shared {
    u64 listed[kList];
    union {
        u64 binned[kList];
        struct {
            uint4 chunk[kQueue];
            int chunk_at[kQueue];
        };
        u64 hist[2][kBins];
        uint32_t times[kSlots];
    };
    int start[kSteps + 1], fill[kSteps];
    u64 wave_sum[THREADS / kWave];
    double red[THREADS / kWave];
    float low[2][THREADS / kWave], top[THREADS / kWave], all[THREADS / kWave];
    u64 above, found, aboves[2];
    int bins[2];
    uint32_t key_min, key_max;
    int bin;
    int count, queued, beyond;
    int cut_m, drawn;
    float logprob;
    u64 kept;
};

// A histogram's running sum: thread t has bins B t .. B t + B - 1
template <int THREADS> struct Scan {
    static constexpr int B = kBins / THREADS;
    u64 begin, end, total;
    __device__ __forceinline__ Scan() {}
    __device__ __forceinline__ Scan(Shared<THREADS> &sh, const u64 *hist)
    {
        u64 sum = 0;
#pragma unroll
        for (int b = 0; b < B; ++b) sum += hist[threadIdx.x * B + b];
        end = sum;
        const int lane = threadIdx.x & (kWave - 1);
#pragma unroll
        for (int o = 1; o < kWave; o <<= 1) {
            const u64 up = __shfl_up(end, o);
            if (lane >= o) end += up;
        }
        if (lane == kWave - 1) sh.wave_sum[threadIdx.x / kWave] = end;
        __syncthreads();
        total = 0;
#pragma unroll
        for (int w = 0; w < THREADS / kWave; ++w) {
            if (w == (int)(threadIdx.x / kWave)) end += total;
            total += sh.wave_sum[w];
        }
        begin = end - sum;
        total = uniform(total);
        __syncthreads();
    }
    // The first bins at which the running sum reaches goal[0] and goal[1] (1 <= goal <= total), and the sums before them
    __device__ __forceinline__ void find(Shared<THREADS> &sh, const u64 *hist, const u64 (&goal)[2], int (&bin)[2], u64 (&above)[2]) const
    {
#pragma unroll
        for (int a = 0; a < 2; ++a) {
            if (goal[a] <= begin || goal[a] > end) continue;
            u64 run = begin;
#pragma unroll
            for (int b = 0; b < B; ++b) {
                const u64 own = hist[threadIdx.x * B + b];
                if (goal[a] > run && goal[a] <= run + own) {
                    sh.bins[a] = threadIdx.x * B + b;
                    sh.aboves[a] = run;
                }
                run += own;
            }
        }
        __syncthreads();
#pragma unroll
        for (int a = 0; a < 2; ++a) {
            bin[a] = (int)uniform((uint32_t)sh.bins[a]);
            above[a] = uniform(sh.aboves[a]);
        }
        __syncthreads();
    }
    __device__ __forceinline__ void find(Shared<THREADS> &sh, const u64 *hist, u64 goal, int &bin, u64 &above) const
    {
        int b[2];
        u64 a[2];
        find(sh, hist, {goal, 0}, b, a);
        bin = b[0];
        above = a[0];
    }
};
template <int THREADS> __device__ __forceinline__ void find_bin(Shared<THREADS> &sh, const u64 *hist, u64 goal, int &bin, u64 &above)
{
    Scan<THREADS>(sh, hist).find(sh, hist, goal, bin, above);
}

// What is found by steps: the entry at which a running sum over the order of the row reaches a goal, and the sum before it
struct Spot {
    u64 at, above;
};

template <bool BF16, int THREADS> struct Steps {
    Shared<THREADS> &sh;
    const Row<BF16> row;
    float hi, scale;      // the first histogram's steps
    Scan<THREADS> scan;  // and its running sum

    __device__ __forceinline__ Steps(Shared<THREADS> &s, const Row<BF16> &r) : sh(s), row(r) {}

    // f(key, index) over the row's logits
    template <typename F> __device__ __forceinline__ void each(F f) const
    {
        each_value([&](float z, int idx) { f(key_of(z), idx); });
    }
    // f(logit, index) over the row's logits
    template <typename F> __device__ __forceinline__ void each_value(F f) const
    {
        each_chunk([&](const auto &z, int first) {
#pragma unroll
            for (int e = 0; e < (int)(sizeof z / sizeof z[0]); ++e) f(z[e], first + e);
        });
    }
    // f(logits side by side, index of the first) over the row's chunks and, one by one, its edges; four loads on the way at any time
    template <typename F> __device__ __forceinline__ void each_chunk(F f) const
    {
        constexpr int E = Row<BF16>::E, U = 4;
        const __amdgpu_buffer_rsrc_t from = row.buffer();
        uint4 v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] = load_chunk<false>(from, u * THREADS + threadIdx.x);
        for (int c = threadIdx.x; c < row.whole; c += U * THREADS) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int at = c + u * THREADS;
                if (at < row.whole) {
                    float z[E];
#pragma unroll
                    for (int e = 0; e < E; ++e) z[e] = Row<BF16>::value(v[u], e);
                    f(z, row.lo + at * E);
                }
                v[u] = load_chunk<false>(from, at + U * THREADS);
            }
        }
        if ((int)threadIdx.x < row.edges) {
            const float z[1] = {row.edge(threadIdx.x)};
            f(z, row.edge_index(threadIdx.x));
        }
    }
    __device__ __forceinline__ void clear(u64 *hist) const
    {
        for (int b = threadIdx.x; b < kBins; b += THREADS) hist[b] = 0;
        __syncthreads();
    }
    // The first histogram: equal steps from the largest logit down to `lo` and all below it; measure(key, index): what a logit counts
    // (0: nothing).  Returns the total.
    template <typename M> __device__ __forceinline__ u64 first(float m, float lo, M measure)
    {
        begin(m, lo);
        each([&](uint32_t key, int idx) {
            if (key <= kKeyNone) return;
            const u64 x = measure(key, idx);
            if (x) atomicAdd(&sh.hist[0][step(key)], x);
        });
        __syncthreads();
        scan = Scan<THREADS>(sh, sh.hist[0]);
        return scan.total;
    }
    __device__ __forceinline__ void begin(float m, float lo)
    {
        hi = m;
        scale = fminf((float)(kBins - 1) / (m - lo), 1e30f);
        if (!(scale >= 0.f)) scale = 0.f;
        clear(sh.hist[0]);
    }
    // The same of the weights of all logits, the largest finite; of fp32 a chunk's are worked out side by
    // side, without a branch (46 us of 200 rows of 50257 instead of 50; rows of bf16 rarely come here, and their kernel has no registers for it).  over: the sum of those of logits from `low` on that this thread met
    __device__ __forceinline__ u64 first_of_weights(float m, float lo, const Weight &w, float low, u64 &over)
    {
        begin(m, lo);
        if constexpr (BF16) {
            each_value([&](float z, int) {
                if (!(z > kNegInf)) return;
                const u64 x = w.finite(z);
                if (z >= low) over += x;
                if (x) atomicAdd(&sh.hist[0][step_of(z)], x);
            });
        }
        else each_chunk([&](const auto &z, int) {
            constexpr int N = (int)(sizeof z / sizeof z[0]);
            u64 x[N], any = 0;
#pragma unroll
            for (int e = 0; e < N; ++e) {
                x[e] = w.finite(z[e]);
                if (!(z[e] > kNegInf)) x[e] = 0;
                over += z[e] >= low ? x[e] : 0;
                any |= x[e];
            }
            if (!any) return;
#pragma unroll
            for (int e = 0; e < N; ++e) atomicAdd(&sh.hist[0][step_of(z[e])], x[e]);
        });
        __syncthreads();
        scan = Scan<THREADS>(sh, sh.hist[0]);
        return scan.total;
    }
    __device__ __forceinline__ int step_of(float z) const { return (int)fminf(fmaxf((hi - z) * scale, 0.f), (float)(kBins - 1)); }
    __device__ __forceinline__ int step(uint32_t key) const { return step_of(value_of(key)); }
    // Bounds outside which no logit is of the steps from `from` to `to`: (hi - z) scale is rounded twice in step_of, by 2^-24 each
    __device__ __forceinline__ void bounds(int from, int to, float &least, float &most) const
    {
        least = kNegInf;
        most = __builtin_huge_valf();
        if (to < kBins - 1 && scale > 0.f) {
            const double z = (double)hi - (double)(to + 1) / (double)scale * (1.0 + 0x1p-20);
            least = (float)z;
            if ((double)least > z) least = nextafterf(least, kNegInf);
        }
        if (from > 0) {
            const double z = (double)hi - (double)from / (double)scale * (1.0 - 0x1p-20);
            most = (float)z;
            if ((double)most < z) most = nextafterf(most, __builtin_huge_valf());
        }
    }
    // The spot at which what `measure` counts, as in the first histogram, reaches `goal` (1 <= goal <= total)
    template <typename M> __device__ __forceinline__ Spot find(u64 goal, M measure) const
    {
        int bin;
        u64 above;
        scan.find(sh, sh.hist[0], goal, bin, above);
        uint32_t k_lo = kKeyNone + 1, k_hi = 0xffffffffu;  // the keys in question
        int shift = -1;                                    // steps of their bits (-1: those of the first histogram)
        for (;;) {
            // those of the step
            if (threadIdx.x == 0) {
                sh.count = 0;
                sh.key_min = 0xffffffffu;
                sh.key_max = 0;
            }
            __syncthreads();
            each([&](uint32_t key, int idx) {
                if (key < k_lo || key > k_hi || (shift < 0 ? step(key) : (int)((k_hi - key) >> shift)) != bin || !measure(key, idx)) return;
                const int to = atomicAdd(&sh.count, 1);
                if (to < kFew) sh.listed[to] = entry(key, idx);
                atomicMin(&sh.key_min, key);
                atomicMax(&sh.key_max, key);
            });
            __syncthreads();
            const int count = (int)uniform((uint32_t)sh.count);
            k_lo = uniform(sh.key_min);
            k_hi = uniform(sh.key_max);
            if (count <= kFew) return among(goal, above, count, measure);
            if (k_lo == k_hi) {
                // alike: a division says how many, the lowest indices come first
                const u64 w = measure(k_lo, -1), q = (goal - above + w - 1) / w;
                return {entry(k_lo, locate(k_lo, (uint32_t)q)), above + (q - 1) * w};
            }
            const int bits = 32 - __builtin_clz(k_hi - k_lo);
            shift = bits > 11 ? bits - 11 : 0;
            clear(sh.hist[1]);
            each([&](uint32_t key, int idx) {
                if (key < k_lo || key > k_hi) return;
                const u64 x = measure(key, idx);
                if (x) atomicAdd(&sh.hist[1][(k_hi - key) >> shift], x);
            });
            __syncthreads();
            u64 part;
            find_bin<THREADS>(sh, sh.hist[1], goal - above, bin, part);
            above += part;
        }
    }
    // the spot among the `count` <= kFew entries listed
    template <typename M> __device__ __forceinline__ Spot among(u64 goal, u64 above, int count, M measure) const
    {
        sort_few(count);
        u64 x = 0, own = 0;
        if ((int)threadIdx.x < count) {
            x = sh.listed[kFew + threadIdx.x];
            own = measure(key_in(x), index_in(x));
        }
        u64 incl = own;
        const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
#pragma unroll
        for (int o = 1; o < kWave; o <<= 1) {
            const u64 up = __shfl_up(incl, o);
            if (lane >= o) incl += up;
        }
        if (lane == kWave - 1) sh.wave_sum[wave] = incl;
        __syncthreads();
        for (int w = 0; w < wave; ++w) incl += sh.wave_sum[w];
        const u64 before = above + incl - own;
        if (goal > before && goal <= before + own) {
            sh.found = x;
            sh.above = before;
        }
        __syncthreads();
        const Spot out = {uniform(sh.found), uniform(sh.above)};
        __syncthreads();
        return out;
    }
    // listed[0 .. count) in order to listed[kFew .. ), each behind those before it
    __device__ __forceinline__ void sort_few(int count) const
    {
        for (int t = threadIdx.x; t < count; t += THREADS) {
            const u64 x = sh.listed[t];
            int at = 0;
            for (int j = 0; j < count; ++j) at += sh.listed[j] < x;
            sh.listed[kFew + at] = x;
        }
        __syncthreads();
    }
    // the index of the q-th lowest (from 1) of the logits of one key
    __device__ __forceinline__ int locate(uint32_t key, uint32_t q) const
    {
        int lo = 0, width = row.n;  // the indices in question
        for (;;) {
            // counted by ranges of indices, until a range is one index
            clear(sh.hist[1]);
            const int range = (width + kBins - 1) / kBins;
            each([&](uint32_t k, int i) {
                if (k == key && i >= lo && i - lo < width) atomicAdd(&sh.hist[1][(i - lo) / range], (u64)1);
            });
            __syncthreads();
            int bin;
            u64 above;
            find_bin<THREADS>(sh, sh.hist[1], q, bin, above);
            q -= (uint32_t)above;
            lo += bin * range;
            width = range;
            if (range == 1) return lo;
        }
    }
    // largest and least logit above -inf (-inf and inf without any)
    __device__ __forceinline__ void extremes(float &m, float &least) const
    {
        m = kNegInf;
        float neg = kNegInf;
        each([&](uint32_t key, int) {
            if (key <= kKeyNone) return;
            m = fmaxf(m, value_of(key));
            neg = fmaxf(neg, -value_of(key));
        });
        m = block_max<THREADS>(m, sh.red);
        least = -block_max<THREADS>(neg, sh.red);
    }
};

// A row's sampling parameters as they count: k = 0, top_p = 1, min_p = 0 are off
struct Params {
    float T, top_p, min_p;
    int k;
    bool greedy;
    __device__ __forceinline__ Params(const SampleArgs &p, int i)
    {
        T = uniform(p.temperature ? p.temperature[i] : 1.0f);
        k = (int)uniform((uint32_t)(p.top_k ? p.top_k[i] : 0));
        top_p = uniform(p.top_p ? p.top_p[i] : 1.0f);
        if (!(top_p < 1.0f)) top_p = 1.0f;
        min_p = uniform(p.min_p ? p.min_p[i] : 0.0f);
        min_p = min_p > 0.0f ? fminf(min_p, 1.0f) : 0.0f;
        greedy = !(T > 0.0f) || k == 1;
        if (k <= 0 || k >= p.r.vocab || greedy) k = 0;
    }
};

__device__ __forceinline__ Weight weight_of(float m, float T, int vocab)
{
    Weight w;
    w.top_inf = m == __builtin_huge_valf();
    w.m = m;
    w.c = 1.44269504088896340736 / (double)T;
    w.scale = 62 - (32 - __builtin_clz((uint32_t)vocab));
    if (w.scale > 45) w.scale = 45;
    return w;
}

// The least logit, in 64 bits, whose weight min-p keeps (-inf where all weights are alike: infinite temperature, also at min_p 1, where
// the product is no number)
__device__ __forceinline__ double min_p_logit(const Weight &w, const Params &par)
{
    return fmax(w.m + (double)par.T * log((double)par.min_p), (double)kNegInf);
}

// Puts the list in order (below)
template <int THREADS> __device__ __forceinline__ bool sort_list(Shared<THREADS> &sh, int count);

// Token and its log probability by steps: every row, whatever its logits.  m: the largest logit, if known (NaN: not)
template <bool BF16, int THREADS>
__device__ __forceinline__ void sample_by_steps(Shared<THREADS> &sh, const Row<BF16> &row, const Params &par, float u, float m, int &token, float &logprob)
{
    constexpr int N = kList / THREADS;
    Steps<BF16, THREADS> steps(sh, row);
    float least = kLow;
    if (!(m == m) || par.k) steps.extremes(m, least);
    token = -1;
    logprob = kNegInf;
    if (!(m > kNegInf)) return;  // (the same for the whole block, as is every choice below)
    auto one = [](uint32_t, int) { return (u64)1; };
    if (par.greedy) {
        token = steps.locate(key_of(m), 1);
        logprob = 0.0f;
        return;
    }
    const Weight w = weight_of(m, par.T, row.n);
    u64 last = ~(u64)0;  // the last entry of the top-k
    if (par.k && steps.first(m, least, one) > (u64)par.k) last = steps.find(par.k, one).at;
    auto inside = [&](uint32_t key, int idx) { return entry(key, idx < 0 ? 0 : idx) <= last ? w(key) : (u64)0; };
    // min-p: the least key whose weight it keeps, and the sum of the weights it keeps
    uint32_t key_min = 0;
    if (par.min_p > 0.0f && !w.top_inf) {
        const double low = min_p_logit(w, par);
        const float f = (float)low;
        key_min = key_of(f) + ((double)f < low ? 1 : 0);
    }
    u64 over = 0;
    const float end = fmaxf(least, m - 44.0f * par.T);
    const bool all = last == ~(u64)0 && !w.top_inf;
    u64 total;
    if (all) {
        total = steps.first_of_weights(m, end, w, key_min > kKeyNone ? value_of(key_min) : kNegInf, over);
    } else {
        total = steps.first(m, end, [&](uint32_t key, int idx) {
            const u64 x = inside(key, idx);
            if (key >= key_min) over += x;
            return x;
        });
    }
    if (key_min) over = block_reduce<u64, THREADS>(over, sh.wave_sum, [](u64 a, u64 b) { return a + b; });
    else over = total;
    const double p_goal = ceil((double)par.top_p * (double)total);
    const u64 cut_goal = !(p_goal >= 1.0) ? 1 : p_goal >= (double)total ? total : (u64)p_goal;
    auto draw_goal = [&](u64 kept) {
        const double goal = floor((double)u * (double)kept);
        return !(goal >= 0.0) ? (u64)1 : goal >= (double)(kept - 1) ? kept : (u64)goal + 1;
    };
    // The step of top-p's cut says what is kept but for that step's own weights, and so, nearly always, the step of the draw: both are
    // listed in one pass, and in order.
    int cut_bin = -1;
    u64 cut_above = 0, least_kept = over, most_kept = over;
    if (par.top_p < 1.0f) {
        steps.scan.find(sh, sh.hist[0], cut_goal, cut_bin, cut_above);
        const u64 with = cut_above + uniform(sh.hist[0][cut_bin]);
        least_kept = cut_above + 1 < over ? cut_above + 1 : over;
        most_kept = with < over ? with : over;
        if (least_kept == most_kept) cut_bin = -1;  // (min-p cuts before)
    }
    int draw_bin[2];
    u64 draw_above[2];
    steps.scan.find(sh, sh.hist[0], {draw_goal(least_kept), draw_goal(most_kept)}, draw_bin, draw_above);
    const int bin_1 = draw_bin[0], bin_2 = draw_bin[1];
    const u64 above_1 = draw_above[0];
    if (threadIdx.x == 0) sh.count = 0;
    __syncthreads();
    // (most logits are told from their value alone)
    float draw_least, draw_most, cut_least = __builtin_huge_valf(), cut_most = kNegInf;
    steps.bounds(bin_1, bin_2, draw_least, draw_most);
    if (cut_bin >= 0) steps.bounds(cut_bin, cut_bin, cut_least, cut_most);
    auto may_be = [&](float z) { return (z >= draw_least && z <= draw_most) || (z >= cut_least && z <= cut_most); };
    auto list = [&](float z, int idx) {
        if (!(z > kNegInf)) return;
        const uint32_t key = key_of(z);
        const int b = steps.step(key);
        if (((b < bin_1 || b > bin_2) && b != cut_bin) || entry(key, idx) > last) return;
        const int to = atomicAdd(&sh.count, 1);
        if (to < kList) sh.listed[to] = entry(key, idx);
    };
    if constexpr (BF16) {
        steps.each_value([&](float z, int idx) {
            if (may_be(z)) list(z, idx);
        });
    } else {
        steps.each_chunk([&](const auto &z, int first) {
            constexpr int N = (int)(sizeof z / sizeof z[0]);
            bool any = false, in[N];
#pragma unroll
            for (int e = 0; e < N; ++e) {
                in[e] = (z[e] >= draw_least & z[e] <= draw_most) | (z[e] >= cut_least & z[e] <= cut_most);
                any |= in[e];
            }
            if (!any) return;
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (in[e]) list(z[e], first + e);
        });
    }
    __syncthreads();
    const int count = (int)uniform((uint32_t)sh.count);
    if (count <= kList && sort_list<THREADS>(sh, count)) {
        const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
        u64 own[N], sum = 0, sum_draw = 0;
        int bin[N];
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int e = threadIdx.x * N + n;
            own[n] = 0;
            bin[n] = -2;
            if (e < count) {
                own[n] = w(key_in(sh.listed[e]));
                bin[n] = steps.step(key_in(sh.listed[e]));
            }
            sum += own[n];
            if (bin[n] <= bin_2) sum_draw += own[n];
        }
        u64 incl = sum;
#pragma unroll
        for (int o = 1; o < kWave; o <<= 1) {
            const u64 up = __shfl_up(incl, o);
            if (lane >= o) incl += up;
        }
        if (lane == kWave - 1) sh.wave_sum[wave] = incl;
        __syncthreads();
        for (int k = 0; k < wave; ++k) incl += sh.wave_sum[k];
        __syncthreads();
        const u64 draws = block_reduce<u64, THREADS>(sum_draw, sh.wave_sum, [](u64 a, u64 b) { return a + b; });
        // the running sum in front of an entry: those of the cut's step alone begin at cut_above
        auto entries = [&](auto f) {
            u64 run = incl - sum;
#pragma unroll
            for (int n = 0; n < N; ++n) {
                f(n, bin[n] <= bin_2 ? above_1 + run : cut_above + (run - draws));
                run += own[n];
            }
        };
        u64 kept = over;
        if (cut_bin >= 0) {
            entries([&](int n, u64 before) {
                if (bin[n] == cut_bin && before < cut_goal && cut_goal <= before + own[n]) sh.kept = before + own[n];
            });
            __syncthreads();
            kept = uniform(sh.kept);
            kept = kept < over ? kept : over;
        } else if (par.top_p < 1.0f) {
            kept = least_kept;
        }
        const u64 g = draw_goal(kept);
        entries([&](int n, u64 before) {
            if (bin[n] >= bin_1 && bin[n] <= bin_2 && before < g && g <= before + own[n]) sh.found = sh.listed[threadIdx.x * N + n];
        });
        __syncthreads();
        const u64 drawn = uniform(sh.found);
        token = index_in(drawn);
        logprob = (float)((w.top_inf ? 0.0 : w.log2_of(key_in(drawn)) * 0.69314718055994530942) - log(__builtin_ldexp((double)kept, -w.scale)));
        return;
    }
    // too many logits in a step: step by step
    __syncthreads();
    steps.first(m, end, inside);
    u64 kept = over;
    if (par.top_p < 1.0f) {
        const Spot cut = steps.find(cut_goal, inside);
        const u64 with = cut.above + w(key_in(cut.at));
        kept = with < over ? with : over;
    }
    const u64 drawn = steps.find(draw_goal(kept), inside).at;
    token = index_in(drawn);
    logprob = (float)((w.top_inf ? 0.0 : w.log2_of(key_in(drawn)) * 0.69314718055994530942) - log(__builtin_ldexp((double)kept, -w.scale)));
}

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ u16x2 halves(uint32_t w) { return __builtin_bit_cast(u16x2, w); }

// The index of the q-th lowest (from 1) of the logits whose bf16 bits are `bits` (not a zero's): counted by runs of 128 chunks,
// then within the run.  held: the row's chunks in registers (SLOTS of them a thread; 0: read again).
template <int THREADS, int SLOTS>
__device__ __forceinline__ int locate_bits(Shared<THREADS> &sh, const Row<true> &row, const uint4 (&held)[SLOTS ? SLOTS : 1], uint32_t bits, uint32_t q)
{
    constexpr int U = 4, kRun = 2 * kWave;
    const int lane = threadIdx.x & (kWave - 1), runs = (row.whole + kRun - 1) / kRun;
    const u16x2 both = {(uint16_t)bits, (uint16_t)bits};
    auto any_in_chunk = [&](const uint4 &v) {
        const u16x2 none = __builtin_elementwise_min(__builtin_elementwise_min(halves(v.x) ^ both, halves(v.y) ^ both),
                                                     __builtin_elementwise_min(halves(v.z) ^ both, halves(v.w) ^ both));
        return none.x == 0 || none.y == 0;
    };
    auto in_chunk = [&](const uint4 &v) {  // one bit an element
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        uint32_t m = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) m |= ((w[j] & 0xffffu) == bits ? 1u << (2 * j) : 0u) | ((w[j] >> 16) == bits ? 2u << (2 * j) : 0u);
        return m;
    };
    // bins: the edges in front, the runs, the edges behind
    u64 *const hist = sh.hist[0];
    for (int r = threadIdx.x; r < kBins; r += THREADS) hist[r] = 0;
    if (threadIdx.x == 0) sh.count = 0;
    __syncthreads();
    const bool at_edge = (int)threadIdx.x < row.edges && ((const uint16_t *)row.row)[row.edge_index(threadIdx.x)] == (uint16_t)bits;
    if (at_edge) atomicAdd(&hist[(int)threadIdx.x < row.lo ? 0 : 1 + runs], (u64)1);
    if (at_edge && (int)threadIdx.x < row.lo) atomicAdd(&sh.count, 1);
    if constexpr (SLOTS > 0) {
#pragma unroll
        for (int k = 0; k < SLOTS; ++k) {
            const int at = k * THREADS + (int)threadIdx.x;
            if (at < row.whole && any_in_chunk(held[k])) atomicAdd(&hist[1 + at / kRun], (u64)__popc(in_chunk(held[k])));
        }
        __syncthreads();
    } else {
        const __amdgpu_buffer_rsrc_t from = row.buffer();
        uint4 v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] = load_chunk<false>(from, u * THREADS + threadIdx.x);
        // (as far as the q-th: half the row, on average)
        for (int c = threadIdx.x, done = 0; done < row.whole; c += U * THREADS, done += U * THREADS) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int at = c + u * THREADS;
                if (at < row.whole && any_in_chunk(v[u])) {
                    const int n = __popc(in_chunk(v[u]));
                    atomicAdd(&hist[1 + at / kRun], (u64)n);
                    atomicAdd(&sh.count, n);
                }
                v[u] = load_chunk<false>(from, at + U * THREADS);
            }
            __syncthreads();
            const bool met = uniform((uint32_t)sh.count) >= q;
            __syncthreads();
            if (met) break;
        }
    }
    int bin;
    u64 above;
    find_bin<THREADS>(sh, hist, q, bin, above);
    const int nth = (int)(q - (uint32_t)above);  // in the bin, from 1
    if (threadIdx.x < kWave) {
        // (edges are the first wave's; of a run a lane has two chunks)
        const bool mine = at_edge && ((int)threadIdx.x < row.lo ? 0 : 1 + runs) == bin;
        const int c = (bin - 1) * kRun + 2 * lane;
        uint32_t m = mine ? 1 : 0;
        if (bin > 0 && bin <= runs) {
            m = c < row.whole ? in_chunk(row.body[c]) : 0;
            if (c + 1 < row.whole) m |= in_chunk(row.body[c + 1]) << 8;
        }
        int incl = __popc(m);
#pragma unroll
        for (int o = 1; o < kWave; o <<= 1) {
            const int up = __shfl_up(incl, o);
            if (lane >= o) incl += up;
        }
        const int before = incl - __popc(m);
        if (nth > before && nth <= incl) {
            for (int k = before + 1; k < nth; ++k) m &= m - 1;
            sh.bin = bin > 0 && bin <= runs ? row.lo + c * 8 + __ffs(m) - 1 : row.edge_index(threadIdx.x);
        }
    }
    __syncthreads();
    const int found = (int)uniform((uint32_t)sh.bin);
    __syncthreads();
    return found;
}

// Token and log probability of a row of bf16 by counting how often each logit occurs; false: not that kind of row (NaN, infinity or a
// logit from 2^17 on among its logits, or many near 0).
//   slot t + kSlots / 2 (if negative): magnitude kNearest + t in bf16 bits.  In the order of the row: positive logits, t falling; those nearer to 0 than any
//   slot, listed; negative ones, t rising
template <int THREADS, int SLOTS>
__device__ __forceinline__ bool sample_by_slots(Shared<THREADS> &sh, const Row<true> &row, const Params &par, float u, int &token, float &logprob)
{
    constexpr int U = 4, N = kSlots / THREADS, W = THREADS / kWave, kHalf = kSlots / 2, kMiddle = kHalf / N;
    constexpr uint32_t kNearest = 0x3800u;  // 2^-15
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const __amdgpu_buffer_rsrc_t from = row.buffer();
    constexpr int kHeld = SLOTS ? SLOTS : 1, kAhead = SLOTS ? 1 : U;
    uint4 held[kHeld], v[kAhead];
    if constexpr (SLOTS > 0) {
#pragma unroll
        for (int k = 0; k < SLOTS; ++k) held[k] = load_chunk<false>(from, k * THREADS + threadIdx.x);
    } else {
#pragma unroll
        for (int k = 0; k < U; ++k) v[k] = load_chunk<false>(from, k * THREADS + threadIdx.x);
    }
    for (int k = threadIdx.x; k < kSlots / 4; k += THREADS) ((uint4 *)sh.times)[k] = make_uint4(0, 0, 0, 0);
    if (threadIdx.x == 0) sh.count = sh.queued = 0;
    __syncthreads();
    // a logit that may have no slot
    auto count = [&](uint32_t h, int idx) {
        const uint32_t mag = h & 0x7fffu, t = mag - kNearest;
        if (t < (uint32_t)kHalf) {
            atomicAdd(&sh.times[t + (h >> 15) * kHalf], 1u);
        } else if (mag < kNearest) {
            const int to = atomicAdd(&sh.count, 1);
            if (to < kFew) sh.listed[to] = entry(key_of(bf16_to_f32(h)), idx);
        } else if (h != 0xff80u) {
            sh.queued = 1;
        }
    };
    if ((int)threadIdx.x < row.edges) count(((const uint16_t *)row.row)[row.edge_index(threadIdx.x)], row.edge_index(threadIdx.x));
    auto count_chunk = [&](const uint4 &c, int at) {
        if (at >= row.whole) return;
        const uint32_t w[4] = {c.x, c.y, c.z, c.w};
        // two logits at a time: the bits less kNearest have a slot where bits 12 to 14 are clear
        u16x2 x[4];
        uint32_t out = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            x[j] = halves(w[j]) - u16x2{(uint16_t)kNearest, (uint16_t)kNearest};
            out |= __builtin_bit_cast(uint32_t, x[j]) & 0x70007000u;
        }
        if (!out) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const u16x2 sign = x[j] >> u16x2{15, 15};
                const uint32_t to = __builtin_bit_cast(uint32_t, (u16x2)((x[j] << u16x2{2, 2}) + sign * u16x2{4 * kHalf, 4 * kHalf}));  // in bytes
                atomicAdd((uint32_t *)((char *)sh.times + (to & 0xffffu)), 1u);
                atomicAdd((uint32_t *)((char *)sh.times + (to >> 16)), 1u);
            }
        } else if constexpr (SLOTS > 0) {
            // (those above -inf: of a masked row, whose chunks all come here, few; in a loop, as this is compiled SLOTS times: unrolled, 256 rows of
            // 128256 take 42 us instead of 35)
            uint32_t left = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const u16x2 some = __builtin_elementwise_min((u16x2)(halves(w[j]) ^ u16x2{0xff80, 0xff80}), u16x2{1, 1});
                const uint32_t two = __builtin_bit_cast(uint32_t, some);
                left |= ((two | two >> 15) & 3u) << (2 * j);
            }
            for (; left; left &= left - 1) {
                const int e = __ffs(left) - 1;
                const uint32_t pair = e < 4 ? (e < 2 ? w[0] : w[1]) : (e < 6 ? w[2] : w[3]);
                count((e & 1) ? pair >> 16 : pair & 0xffffu, row.lo + at * 8 + e);
            }
        } else {
            // (pairs of -inf, as in most of a masked row's chunks, have none; the loop above would take registers that this has not: 1024 rows 102 -> 110 us)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (w[j] == 0xff80ff80u) continue;
                count(w[j] & 0xffffu, row.lo + at * 8 + 2 * j);
                count(w[j] >> 16, row.lo + at * 8 + 2 * j + 1);
            }
        }
    };
    if constexpr (SLOTS > 0) {
#pragma unroll
        for (int k = 0; k < SLOTS; ++k) {
            count_chunk(held[k], k * THREADS + (int)threadIdx.x);
            __builtin_amdgcn_sched_barrier(0);
        }
    } else {
        for (int c = threadIdx.x; c < row.whole; c += U * THREADS) {
#pragma unroll
            for (int k = 0; k < U; ++k) {
                const int at = c + k * THREADS;
                count_chunk(v[k], at);
                v[k] = load_chunk<false>(from, at + U * THREADS);
            }
        }
    }
    __syncthreads();
    const int near_zero = (int)uniform((uint32_t)sh.count);
    if (uniform((uint32_t)sh.queued) || near_zero > kFew) return false;
    if (near_zero) Steps<true, THREADS>(sh, row).sort_few(near_zero);
    // Thread t has slots N t .. N t + N - 1 in the order of the row; the logits near 0 are in front of thread kMiddle's.  What occurs is put side by
    // side, in order: entries of a key and how often.  Few slots are in use, and those are neighbours: so every thread gets its share.
    auto key_at = [&](int o) { return key_of(bf16_to_f32(o < kHalf ? kNearest + (kHalf - 1 - o) : 0x8000u + kNearest + (o - kHalf))); };
    const u64 *zeros = sh.listed + kFew;
    u64 *const entries = sh.binned;  // (in the place of the counters)
    uint32_t count_of[N];
    u64 both = 0;  // entries << 32 | logits
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const int o = threadIdx.x * N + n;
        count_of[n] = sh.times[o < kHalf ? kHalf - 1 - o : o];
        both += count_of[n] ? (u64)1 << 32 | count_of[n] : 0;
    }
    u64 up_to = both;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
        const u64 up = __shfl_up(up_to, o);
        if (lane >= o) up_to += up;
    }
    if (lane == kWave - 1) sh.wave_sum[wave] = up_to;
    __syncthreads();  // (every counter has been read)
    u64 in_all = 0, before_zeros = 0;
#pragma unroll
    for (int k = 0; k < W; ++k) {
        if (k == wave) up_to += in_all;
        if (k == kMiddle / kWave) before_zeros = in_all;
        in_all += sh.wave_sum[k];
    }
    const int n_entries = (int)uniform((uint32_t)(in_all >> 32)) + near_zero, zeros_at = (int)uniform((uint32_t)(before_zeros >> 32));
    const int n_logits = (int)uniform((uint32_t)in_all) + near_zero, zeros_run = (int)uniform((uint32_t)before_zeros);
    // (what is beyond the slots may be asked for; more different logits than a list holds)
    if (n_entries == 0 || n_entries > kList || (par.k && n_logits < par.k)) return false;
    {
        const bool behind = (int)threadIdx.x >= kMiddle;
        int at = (int)((up_to - both) >> 32) + (behind ? near_zero : 0), run = (int)(uint32_t)(up_to - both) + (behind ? near_zero : 0);
        // (how many the top-k keeps)
        auto kept_of = [&](int times, int before) { return !par.k || before + times <= par.k ? times : before < par.k ? par.k - before : 0; };
#pragma unroll
        for (int n = 0; n < N; ++n) {
            if (!count_of[n]) continue;
            entries[at++] = (u64)key_at(threadIdx.x * N + n) << 32 | (uint32_t)kept_of((int)count_of[n], run);
            run += (int)count_of[n];
        }
        if ((int)threadIdx.x < near_zero)
            entries[zeros_at + threadIdx.x] = (u64)key_in(zeros[threadIdx.x]) << 32 | (uint32_t)kept_of(1, zeros_run + (int)threadIdx.x);
    }
    __syncthreads();
    const float m = value_of((uint32_t)(entries[0] >> 32));
    const Weight w = weight_of(m, par.T, row.n);
    // weights, a thread those of `each` entries, and those that min-p keeps
    constexpr int kEach = kList / THREADS;
    const int each = (n_entries + THREADS - 1) / THREADS;
    const double low = par.min_p > 0.0f ? min_p_logit(w, par) : kNegInf;
    u64 one[kEach], sum = 0, over = 0;
    uint32_t times[kEach];
#pragma unroll
    for (int n = 0; n < kEach; ++n) {
        const int e = threadIdx.x * each + n;
        times[n] = 0;
        one[n] = 0;
        if (n < each && e < n_entries) {
            const uint32_t key = (uint32_t)(entries[e] >> 32);
            times[n] = (uint32_t)entries[e];
            one[n] = w(key);
            if ((double)value_of(key) >= low) over += one[n] * times[n];
        }
        sum += one[n] * times[n];
    }
    u64 incl = sum;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
        const u64 up = __shfl_up(incl, o);
        if (lane >= o) incl += up;
    }
    if (lane == kWave - 1) sh.wave_sum[wave] = incl;
    __syncthreads();
    u64 total = 0;
#pragma unroll
    for (int k = 0; k < W; ++k) {
        if (k == wave) incl += total;
        total += sh.wave_sum[k];
    }
    __syncthreads();
    const u64 begin = incl - sum;
    // where the running sum reaches `goal`: the entry, how many of it (from 1), and the sum with those
    auto find = [&](u64 goal, int &slot, uint32_t &q, u64 &with) {
        if (goal > begin && goal <= incl) {
            u64 run = begin;
#pragma unroll
            for (int n = 0; n < kEach; ++n) {
                const u64 all = one[n] * times[n];
                if (goal > run && goal <= run + all) {
                    const uint32_t many = (uint32_t)((goal - run + one[n] - 1) / one[n]);
                    sh.bin = threadIdx.x * each + n;
                    sh.drawn = (int)many;
                    sh.above = run + many * one[n];
                }
                run += all;
            }
        }
        __syncthreads();
        slot = (int)uniform((uint32_t)sh.bin);
        q = uniform((uint32_t)sh.drawn);
        with = uniform(sh.above);
        __syncthreads();
    };
    int slot;
    uint32_t q;
    u64 kept = total, with;
    if (par.top_p < 1.0f) {
        const double goal = ceil((double)par.top_p * (double)total);
        find(!(goal >= 1.0) ? 1 : goal >= (double)total ? total : (u64)goal, slot, q, kept);
    }
    if (par.min_p > 0.0f) {
        // (both keep a prefix of the order: the shorter one counts)
        over = block_reduce<u64, THREADS>(over, sh.wave_sum, [](u64 a, u64 b) { return a + b; });
        kept = over < kept ? over : kept;
    }
    const double goal = floor((double)u * (double)kept);
    find(!(goal >= 0.0) ? 1 : goal >= (double)(kept - 1) ? kept : (u64)goal + 1, slot, q, with);
    const uint32_t key = uniform((uint32_t)(entries[slot] >> 32));
    if (slot >= zeros_at && slot < zeros_at + near_zero) {
        token = index_in(zeros[slot - zeros_at]);
    } else {
        __syncthreads();  // (the counters of what follows take the entries' place)
        token = locate_bits<THREADS, SLOTS>(sh, row, held, __float_as_uint(value_of(key)) >> 16, q);
    }
    logprob = (float)(w.log2_of(key) * 0.69314718055994530942 - log(__builtin_ldexp((double)kept, -w.scale)));
    return true;
}

// What the one pass found
struct Found {
    int count;    // listed
    bool whole;   // every logit above -inf is listed
    double rest;  // sum of exp((z - ref) / T) over what is not listed
    float ref, top;  // what the sum is relative to, at most the largest logit (0 where all are -inf); the largest logit
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

// Lists the beginning of the row, at least `want` logits where there are as many, and sums the rest (if `sums`).  Chunks with a logit to
// list are put aside, for a thread each to look at later: among the others the pass does not branch.
template <bool BF16, int THREADS> __device__ __forceinline__ Found list_row(Shared<THREADS> &sh, const Row<BF16> &row, int want, bool sums, float tau)
{
    constexpr int E = Row<BF16>::E, U = 4, W = THREADS / kWave, kRound = U * THREADS;
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int rank = (want + W - 1) / W < kWave ? (want + W - 1) / W : kWave;
    const __amdgpu_buffer_rsrc_t from = row.buffer();
    const float edge_z = row.edge(threadIdx.x);
    uint4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = load_chunk<false>(from, u * THREADS + threadIdx.x);
    if (threadIdx.x == 0) sh.count = sh.queued = sh.beyond = 0;
    float top = fmaxf(edge_z, kNegInf), bound = kLow;
    double rest = 0.0;
    Exp<BF16> by_T(tau, 0.f);
    auto largest = [&](const uint4 &v) {
        float m = kNegInf;
#pragma unroll
        for (int e = 0; e < E; ++e) m = fmaxf(m, Row<BF16>::value(v, e));
        return m;
    };
    // the bound from the threads' largest logits so far; two sets of words in turn, so that the wait between a call's writes and reads also
    // keeps the next but one call's writes behind those reads
    int turn = 0;
    auto raise_bound = [&]() {
        const uint32_t key = rank_in_wave(top, rank);
        if (lane == 0) sh.low[turn][wave] = key > kKeyNone ? value_of(key) : kLow;
        __syncthreads();
        bound = uniform(fmaxf(-wave_max(-sh.low[turn][lane & (W - 1)]), kLow));
        turn ^= 1;
    };
    // What the sum is relative to: the largest of the first round that is not all -inf.  Rounds before that one (`none` of them) weigh nothing whatever
    // it is; a NaN in them shows in the sum.
    int none = 0;
    for (;; ++none) {
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (none * kRound + u * THREADS + (int)threadIdx.x < row.whole) top = fmaxf(top, largest(v[u]));
        const float m = wave_max(top);
        if (lane == 0) sh.top[wave] = m;
        raise_bound();
        const float first = uniform(wave_max(sh.top[lane & (W - 1)]));
        if (first > kNegInf) by_T.refer(first);
        if (first > kNegInf || !sums || (none + 1) * kRound >= row.whole) break;
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int e = 0; e < E; ++e) rest += (double)by_T.near(Row<BF16>::value(v[u], e));
            v[u] = load_chunk<false>(from, (none + 1) * kRound + u * THREADS + threadIdx.x);
        }
        __syncthreads();  // (sh.top has been read)
    }
    int r = none;
    for (int c = r * kRound + threadIdx.x; r * kRound < row.whole; ++r, c += kRound) {
        if (r > none + 1) raise_bound();  // (of the next round nothing is known yet)
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int at = c + u * THREADS;
            if (at < row.whole) {
                const float m = largest(v[u]);
                top = fmaxf(top, m);
                if (m >= bound) {
                    const int to = atomicAdd(&sh.queued, 1);
                    if (to < kQueue) {
                        sh.chunk[to] = v[u];
                        sh.chunk_at[to] = at;
                    }
                } else if (sums) {
                    float s = 0.f;
#pragma unroll
                    for (int e = 0; e < E; ++e) s += by_T.near(Row<BF16>::value(v[u], e));
                    rest += (double)s;
                }
            }
            v[u] = load_chunk<false>(from, at + kRound);
        }
    }
    {
        const float m = wave_max(top);
        if (lane == 0) sh.all[wave] = m;
    }
    if (r > none + 1) raise_bound();
    else __syncthreads();
    const float largest_logit = uniform(wave_max(sh.all[lane & (W - 1)]));
    // Everything from the last bound on is listed.  The rest is added up in whole units, 2^-41 or less of the largest it may hold: which thread looks at which of
    // the chunks put aside is a matter of the run, and whole numbers have the same sum in every order.  A thread has at most 2^10 logits, so
    // 2^51 units and their roundings; sh.beyond: somewhere it has more, or no number.
    const int power = (int)(__float_as_uint(fminf(fmaxf(by_T.near(bound), 0x1p-100f), 1e30f)) >> 23) - 126;  // (2 to it is above that)
    const double scale = __builtin_ldexp(1.0, 41 - power);
    u64 units = 0;
    auto add = [&](double sum) {
        const double x = sum * scale;
        if (x < 0x1.4p51) units += (u64)__double_as_longlong(x + 0x1p52) & (((u64)1 << 52) - 1);
        else sh.beyond = 1;
    };
    auto look_at = [&](float z, int idx, double &sum) {
        if (z >= bound) {
            const int to = atomicAdd(&sh.count, 1);
            if (to < kList) sh.listed[to] = entry(key_of(z), idx);
        } else if (sums) {
            sum += (double)by_T.near(z);
        }
    };
    look_at(edge_z, row.edge_index(threadIdx.x), rest);
    if (sums) add(rest);
    const int queued = (int)uniform((uint32_t)sh.queued);
    for (int q = threadIdx.x; q < (queued < kQueue ? queued : kQueue); q += THREADS) {
        const uint4 chunk = sh.chunk[q];
        const int first = row.lo + sh.chunk_at[q] * E;
        double part = 0.0;
#pragma unroll
        for (int e = 0; e < E; ++e) look_at(Row<BF16>::value(chunk, e), first + e, part);
        if (sums) add(part);
    }
    if (sums) rest = (double)block_reduce<u64, THREADS>(units, sh.wave_sum, [](u64 a, u64 b) { return a + b; }) * __builtin_ldexp(1.0, power - 41);
    else __syncthreads();
    Found f;
    f.count = (int)uniform((uint32_t)sh.count);
    f.whole = bound == kLow;
    f.ref = by_T.ref;
    f.top = largest_logit;
    f.rest = rest * exp2_neg(-by_T.drift(), 0);
    f.ok = f.count <= kList && queued <= kQueue;
    // (A term's exponent t is off by 3 2^-24 of itself at most, and terms so small that this matters are less than half a unit of the weights: up to t = 32, where
    // the sum is less than 2^64, the error stays below 5e-6 of it.)
    f.summed = !uniform((uint32_t)sh.beyond) && rest < 0x1p64 && by_T.sound() && f.top < __builtin_huge_valf();
    return f;
}

// Puts the list in order.  A long one: a counting sort by equal steps of the logit, then each entry behind those of its step that are before it.
template <int THREADS> __device__ __forceinline__ bool sort_list(Shared<THREADS> &sh, int count)
{
    constexpr int W = THREADS / kWave, N = kList / THREADS, B = kSteps / THREADS;
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    if (count <= kShort) {
        // (a short one: each entry behind those before it)
        u64 x = 0;
        int at = 0;
        if ((int)threadIdx.x < count) {
            x = sh.listed[threadIdx.x];
#pragma unroll 8
            for (int j = 0; j < count; ++j) at += sh.listed[j] < x;
        }
        __syncthreads();
        if ((int)threadIdx.x < count) sh.listed[at] = x;
        __syncthreads();
        return true;
    }
    u64 mine[N];
    float top = kNegInf, low = __builtin_huge_valf();
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const int e = n * THREADS + threadIdx.x;
        if (e < count) {
            mine[n] = sh.listed[e];
            top = fmaxf(top, value_in(mine[n]));
            low = fminf(low, value_in(mine[n]));
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
    auto step_of = [&](u64 x) { return (int)fminf((top - value_in(x)) * scale, (float)(kSteps - 1)); };
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

// What a list in order says, by one wave: sh.drawn whether it decides the row, sh.bin the token, sh.logprob.  rest: sum of the exponentials that are
// not listed, good to 2^-17 of it; unlisted: how many they are, at most (0: none).  The weights are whole numbers: each of those not listed is
// within half a unit of its exponential.  What comes out has to be the same for every sum in between.
template <int THREADS>
__device__ __forceinline__ void read_list(Shared<THREADS> &sh, const Params &par, float u, const Weight &w, int count, double rest, int unlisted)
{
    const int lane = threadIdx.x & (kWave - 1);
    // lane l has entries each * l ..; their weights beside them
    const int n_k = par.k && par.k < count ? par.k : count, each = (n_k + kWave - 1) / kWave;
    const int begin = lane * each < n_k ? lane * each : n_k, end = begin + each < n_k ? begin + each : n_k;
    u64 sum = 0;
#pragma nounroll
    for (int e = begin; e < end; ++e) {
        const u64 x = w(key_in(sh.listed[e]));
        sh.binned[e] = x;
        sum += x;
    }
    u64 incl = sum;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
        const u64 up = __shfl_up(incl, o);
        if (lane >= o) incl += up;
    }
    const u64 first = incl - sum, listed = uniform((u64)__shfl(incl, kWave - 1));
    // what all weights sum to, at least and at most (a few roundings of the sums here beside the rest's)
    double all[2] = {(double)listed, (double)listed};
    if (unlisted) {
        const double unit = 0.5 * (double)unlisted + 0x1p-50 * (all[0] + rest);
        all[0] = fmax(all[0], all[0] + rest * (1.0 - 0x1p-17) - unit);
        all[1] += rest * (1.0 + 0x1p-17) + unit;
    }
    // the first entries that the cuts leave out
    int cut[2] = {n_k, n_k}, cut_m = n_k;
    if (par.top_p < 1.0f || par.min_p > 0.0f) {
        const double low = min_p_logit(w, par);
        const u64 goal[2] = {(u64)ceil(fmax((double)par.top_p * all[0], 0.0)), (u64)ceil(fmax((double)par.top_p * all[1], 0.0))};
        u64 before = first;
#pragma nounroll
        for (int e = begin; e < end; ++e) {
            if (e > 0 && par.top_p < 1.0f) {
#pragma unroll
                for (int a = 0; a < 2; ++a)
                    if (e < cut[a] && before >= goal[a]) cut[a] = e;
            }
            if (e < cut_m && par.min_p > 0.0f && (double)value_in(sh.listed[e]) < low) cut_m = e;
            before += sh.binned[e];
        }
#pragma unroll
        for (int o = kWave / 2; o > 0; o >>= 1) {
            cut[0] = min(cut[0], __shfl_xor(cut[0], o));
            cut[1] = min(cut[1], __shfl_xor(cut[1], o));
            cut_m = min(cut_m, __shfl_xor(cut_m, o));
        }
    }
    const int n = cut[0] < cut_m ? cut[0] : cut_m;
    // the list has to reach the cut: as the end of the top-k, of the row, or because something cuts before its end (for certain)
    const bool ends = n < n_k || par.k || !unlisted;
    const bool open = !ends && !(par.top_p < 1.0f) && !(par.min_p > 0.0f);  // nothing cuts at all
    bool decides = (ends || open) && (cut[0] == cut[1] || n < cut[0]);
    u64 kept = 0;
    {
        u64 before = first;
#pragma nounroll
        for (int e = begin; e < end && e < n; ++e) before += sh.binned[e];
        kept = before - first;
#pragma unroll
        for (int o = kWave / 2; o > 0; o >>= 1) kept += __shfl_xor(kept, o);
        kept = uniform(kept);
    }
    // the draw: the first entry whose running sum passes u times the sum, for both ends of what that may be
    int drawn[2];
#pragma unroll
    for (int a = 0; a < 2; ++a) {
        const double goal = (double)u * (ends ? (double)kept : all[a]);
        u64 g = !(goal >= 0.0) ? 0 : (u64)goal;  // (passes: more than that, whole)
        if (ends && g >= kept) g = kept - 1;
        int at = -1;
        if (first <= g && g < incl) {
            u64 before = first;
            int e = begin;
            for (; before + sh.binned[e] <= g; ++e) before += sh.binned[e];
            at = e;
        }
        const u64 who = __ballot(at >= 0);
        drawn[a] = who ? (int)uniform((uint32_t)__shfl(at, __ffsll(who) - 1)) : -1;
    }
    decides = decides && drawn[0] >= 0 && drawn[0] == drawn[1];
    if (lane == 0) {
        sh.drawn = decides ? 1 : 0;
        if (decides) {
            const u64 x = sh.listed[drawn[0]];
            const double of = ends ? (double)kept : 0.5 * (all[0] + all[1]);
            sh.bin = index_in(x);
            sh.logprob = (float)(w.log2_of(key_in(x)) * 0.69314718055994530942 - log(__builtin_ldexp(of, -w.scale)));
        }
    }
}

// One block a row.  ALONE: with a compute unit's registers to itself; SLOTS: chunks of a row of bf16 that a thread then holds.  What bounds it: one pass over the row, and
// the latency of the steps behind it; by value, the counters (2.1 logits a cycle and compute unit; shared memory is at work 34 % of the cycles, half of that
// bank conflicts, the vector units 41 %) and a second reading of 0.85 of the row (rounds of 32768 logits, one ahead, up to the drawn one); by steps, 87 vector
// instructions a logit in three passes, 30 of them the listing's and most others the 64-bit weights' (half of the cycles).  Measured: 1024 x 128256 bf16 with top-k 20 55 us (4.8 TB/s),
// with top-p 0.9 102 (by value); 256 rows of them mixed 31; 200 x 50257 fp32 with top-p 0.5 23.5 us (off the list), 0.9 50 (by steps); one row of 32000 bf16 8.6
// greedy, 12.6 with top-k 50 and top-p, 14.5 with top-p alone.
template <bool BF16, int THREADS, bool ALONE, int SLOTS> __global__ void __launch_bounds__(THREADS, ALONE ? 4 : 8) sample_kernel(SampleArgs p)
{
    __shared__ Shared<THREADS> sh;
    const int i = blockIdx.x, wave = (int)uniform((uint32_t)threadIdx.x / kWave);
    const void *at = row_of(p.r, i);
    const Row<BF16> row(at, at ? p.r.vocab : 0);
    const Params par(p, i);
    const float u = uniform(p.u[i]);
    // (of a nucleus or a row that nothing cuts the beginning is 128 logits)
    const int want = par.greedy ? 1 : par.k ? par.k : 128;
    const bool sums = !par.greedy && !par.k;
    int token = -1;
    float logprob = kNegInf;
    bool done = false;
    if constexpr (BF16)
        if (!par.greedy && (!par.k || par.k > kMost)) done = sample_by_slots<THREADS, SLOTS>(sh, row, par, u, token, logprob);
    Found f;
    f.ok = false;
    f.top = __builtin_nanf("");
    if (!done && want <= kMost) {
        if (BF16 && sums) __syncthreads();
        f = list_row<BF16, THREADS>(sh, row, want, sums, par.greedy ? 1.0f : par.T);
        done = f.ok && f.count == 0;  // nothing above -inf
    }
    bool reaches = !done && f.ok && (!sums || f.summed) && (!par.k || f.count >= par.k || f.whole);
    if (reaches && sums && !f.whole) {
        // (what the list weighs, nearly, in whole units again: a list that cannot reach is not put in order)
        const Exp<BF16> by_T(par.T, f.top);
        u64 units = 0;
        for (int e = threadIdx.x; e < f.count; e += THREADS) units += (u64)(by_T(value_in(sh.listed[e])) * 0x1p40f);
        const double part = (double)block_reduce<u64, THREADS>(units, sh.wave_sum, [](u64 a, u64 b) { return a + b; }) * 0x1p-40;
        const double beside = f.rest * (double)by_T(f.ref);
        const float share = par.top_p < 1.0f ? par.top_p : par.min_p > 0.0f ? 0.0f : u;
        reaches = part * 1.001 >= (double)share * (part + beside);
    }
    if (reaches && sort_list<THREADS>(sh, f.count)) {
        const float m = value_in(sh.listed[0]);
        if (par.greedy) {
            token = index_in(sh.listed[0]);
            logprob = 0.0f;
            done = true;
        } else if (m < __builtin_huge_valf()) {
            const Weight w = weight_of(m, par.T, row.n);
            // what the row's weights beside the list sum to
            const double rest = sums ? f.rest * exp2_neg(((double)f.ref - (double)m) * w.c, w.scale) : 0.0;
            if (wave == 0) read_list(sh, par, u, w, f.count, rest, sums && !f.whole ? row.n - f.count : 0);
            __syncthreads();
            done = uniform((uint32_t)sh.drawn) != 0;
            token = sh.bin;
            logprob = sh.logprob;
        }
    }
    if (!done) {
        __syncthreads();
        sample_by_steps<BF16, THREADS>(sh, row, par, u, f.top, token, logprob);
    }
    if (threadIdx.x == 0) {
        p.token[i] = token;
        if (p.logprob) p.logprob[i] = logprob;
    }
}

// One block a row, two to a compute unit.  Bound by memory where there are many rows: 3277 x 128256 bf16, k 64, 180 us (4.7 TB/s), 1000 x 128256
// fp32 97 (5.3 TB/s); 205 x 50257 bf16, k 250, 17.5 us; 32 x 32000 fp32, k 20, 12.7 us (one pass and a dozen block-wide waits).  A list that is too long, and k above 256:
// by steps, the k-th place by counting, then the k logits up to it (205 x 50257 bf16, k 300 / 1024, 50 / 68 us).
template <bool BF16, int THREADS> __global__ void __launch_bounds__(THREADS, 8) top_kernel(TopArgs p)
{
    __shared__ Shared<THREADS> sh;
    const int i = blockIdx.x;
    const void *at = row_of(p.r, i);
    const Row<BF16> row(at, at ? p.r.vocab : 0);
    Found f;
    f.ok = f.summed = false;
    if (p.k <= kMost) f = list_row<BF16, THREADS>(sh, row, p.k, p.lse != nullptr, p.temperature);
    double sum = 0.0;  // of exp((z - ref) / temperature)
    bool sorted = f.ok && (f.count >= p.k || f.whole) && sort_list<THREADS>(sh, f.count);
    if (p.lse && sorted && f.summed) {
        // (relative to the row's largest logit where that lies so far above `ref` that the terms would leave the range)
        const double c = 1.44269504088896340736 / (double)p.temperature, above = ((double)f.top - (double)f.ref) * c;
        if (above > 512.0) {
            f.rest *= exp2_neg(-above, 0);
            f.ref = f.top;
        }
        for (int e = threadIdx.x; e < f.count; e += THREADS)
            sum += exp2_neg(((double)value_in(sh.listed[e]) - (double)f.ref) * c, 0);
    }
    if (p.lse && !(sorted && f.summed)) {
        // (relative to each thread's largest logit; of the logits as they are: a NaN among them shows, also beside +inf)
        Running run;
        const float c = (float)(1.44269504088896340736 / (double)p.temperature), edge[1] = {row.edge(threadIdx.x)};
        bool nan = edge[0] != edge[0];
        run.add(edge, c);
        for (int k = threadIdx.x; k < row.whole; k += THREADS) {
            const uint4 v = row.body[k];
            float z[Row<BF16>::E];
#pragma unroll
            for (int e = 0; e < Row<BF16>::E; ++e) {
                z[e] = Row<BF16>::value(v, e);
                nan |= z[e] != z[e];
            }
            run.add(z, c);
        }
        f.ref = block_max<THREADS>(run.m, sh.red);
        run.raise(f.ref, c);
        sum = f.ref < __builtin_huge_valf() ? run.s : nan ? __builtin_nan("") : __builtin_huge_val();
        f.rest = 0.0;
    }
    if (p.lse) {
        sum = block_sum<THREADS>(sum, sh.red) + f.rest;
        if (threadIdx.x == 0) p.lse[i] = (float)((double)f.ref / (double)p.temperature + log(sum));
    }
    if (!sorted) {
        __syncthreads();
        Steps<BF16, THREADS> steps(sh, row);
        float m, least;
        steps.extremes(m, least);
        auto one = [](uint32_t, int) { return (u64)1; };
        u64 last = ~(u64)0;
        if (steps.first(m, least, one) > (u64)p.k) last = steps.find(p.k, one).at;
        if (threadIdx.x == 0) sh.count = 0;
        __syncthreads();
        steps.each([&](uint32_t key, int idx) {
            const u64 x = entry(key, idx);
            if (key > kKeyNone && x <= last) {
                const int to = atomicAdd(&sh.count, 1);
                if (to < kMaxTop) sh.binned[to] = x;
            }
        });
        __syncthreads();
        f.count = (int)uniform((uint32_t)sh.count);  // min(k, logits above -inf)
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
        values[t] = there ? value_in(x) : kNegInf;
        indices[t] = there ? index_in(x) : -1;
    }
}

}  // namespace

hipError_t launch_sample(const SampleArgs &a, hipStream_t st)
{
    // Rows for which there is a compute unit each have its registers: of bf16 the block holds them (up to 4 or 16 chunks a thread) and finds the
    // drawn logit there, 256 rows of 128256 40 -> 35 us, one of 32000 16.6 -> 14.4; of fp32 nothing goes to scratch memory, 200 rows of 50257 by
    // steps 57.6 -> 54.8.  More rows go two to a compute unit: 1024 of 128256 with top-k 54 us, 73 with one.
    const int chunks = a.r.vocab / 8;
    const bool alone = a.r.n_rows <= a.compute_units;
    if (!a.r.bf16 && alone) COLLM_LAUNCH((sample_kernel<false, 1024, true, 0>), dim3(a.r.n_rows), dim3(1024), 0, st, a);
    else if (!a.r.bf16) COLLM_LAUNCH((sample_kernel<false, 1024, false, 0>), dim3(a.r.n_rows), dim3(1024), 0, st, a);
    else if (alone && chunks <= 4 * 1024) COLLM_LAUNCH((sample_kernel<true, 1024, true, 4>), dim3(a.r.n_rows), dim3(1024), 0, st, a);
    else if (alone && chunks <= 16 * 1024) COLLM_LAUNCH((sample_kernel<true, 1024, true, 16>), dim3(a.r.n_rows), dim3(1024), 0, st, a);
    else COLLM_LAUNCH((sample_kernel<true, 1024, false, 0>), dim3(a.r.n_rows), dim3(1024), 0, st, a);
    return hipGetLastError();
}

hipError_t launch_top_logits(const TopArgs &a, hipStream_t st)
{
    if (a.r.bf16) COLLM_LAUNCH((top_kernel<true, 1024>), dim3(a.r.n_rows), dim3(1024), 0, st, a);
    else COLLM_LAUNCH((top_kernel<false, 1024>), dim3(a.r.n_rows), dim3(1024), 0, st, a);
    return hipGetLastError();
}

}  // namespace collm
