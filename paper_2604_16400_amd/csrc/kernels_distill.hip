// Distillation from a teacher's top logits: the loss of a row of student logits z and its gradient.
//
// The teacher's record of a row is k logits t and their places.  With temperature tau, p = softmax(t / tau) over the
// record, or, with the teacher's own log-sum-exp, p = exp(t / tau - lse) and r = max(0, 1 - sum p) for all other places.
// With q = softmax(z / tau), P = sum p + r and `rest` = the places outside the record,
//   KD   = sum_k p_k (log p_k - log q_k) + r (log r - log sum_rest q)
//   loss = a tau^2 KD + b CE,   CE = -log softmax(z)[label]
//   dloss/dz_v = a tau (P q_v - p_v - [v in rest] r q_v / sum_rest q) + b (softmax(z)_v - [v = label]).
// Outside the record the gradient is one multiple of exp((z_v - ref) / tau) plus one of exp(z_v - ref): the row is two
// coefficients, and the places of the record and of the label are written again, behind the others, from sums in 64 bits.
// The sum over the rest is taken over the rest alone (a bitmap of the record in shared memory masks it): 1 - sum q would lose it
// where the record holds nearly all of the mass.
//
// The sums need no largest logit first.  They are taken relative to the student's largest logit in the record, which is near the
// row's where student and teacher agree, so that an exponential is one fused multiply-add and one exp2.  Where a sum then is not
// finite, or so small that terms may have vanished, the row is summed again, each thread relative to the largest logit that it
// has met.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "kernels.h"
#include "vocab_device.h"

namespace collm {

namespace {

using namespace vocab;

// What the waves of a block tell each other, and a teacher's record of a row, in shared memory
template <int THREADS> struct Shared {
    double sum[THREADS / kWave], sum_ce[THREADS / kWave];
    float max[THREADS / kWave];
    float coef[kDistillStats];
};
// (dynamic: k entries of each, the bitmap of the row behind them)
struct Record {
    double *p;       // probabilities (of a place named twice: their sum, at its first entry)
    float *t, *z;    // the teacher's and the student's logits
    int32_t *at;     // places; -1: not an entry
    uint32_t *bits;  // one bit an element of the row
    uint8_t *first;  // whether the entry is its place's first
    __device__ __forceinline__ Record(double *mem, int k, int vocab)
        : p(mem), t((float *)(mem + k)), z(t + k), at((int32_t *)(z + k)), bits((uint32_t *)(at + k)), first((uint8_t *)(bits + (vocab + 31) / 32))
    {
    }
    static size_t bytes(int k, int vocab) { return (size_t)k * 21 + ((size_t)vocab + 31) / 32 * 4; }
};

struct Entry {
    int at;
    float t, z;
};
// entry j of row i's record: place and teacher's logit, then, when they are there, the student's logit
__device__ __forceinline__ Entry load_place(const DistillArgs &p, int i, int j, bool there)
{
    Entry e = {-1, kNegInf, 0.f};
    if (j < p.k && there) {  // (a row that is not there has no record to read)
        e.at = p.t_indices[(int64_t)i * p.k + j];
        e.t = p.t_values[(int64_t)i * p.k + j];
    }
    return e;
}
template <bool BF16, typename S = void> __device__ __forceinline__ void load_logit(Entry &e, const Row<BF16> &row, const S *span = nullptr)
{
    if (e.at < 0 || e.at >= row.n || !(e.t > kNegInf)) {
        e.at = -1;
        return;
    }
    if constexpr (!std::is_void_v<S>)
        if (!span->has(row, e.at)) return;  // (another block's, which may have written there already)
    e.z = Elem<BF16>::load(row.row, e.at);
}
template <bool BF16> __device__ __forceinline__ void put_entry(const Record &rec, int j, const Entry &e, const Row<BF16> &row)
{
    rec.at[j] = e.at;
    rec.t[j] = e.t;
    rec.z[j] = e.z;
    bool first = false;
    if (e.at >= 0) {
        const int b = row.bit(e.at);
        first = !(atomicOr(&rec.bits[b >> 5], 1u << (b & 31)) >> (b & 31) & 1u);
    }
    rec.first[j] = first;
}

// Row i's record into shared memory, its places into the bitmap.  mine: the entry of this thread's index, loaded before.
template <bool BF16, int THREADS>
__device__ __forceinline__ void put_record(const Record &rec, const DistillArgs &p, int i, const Row<BF16> &row, const Entry &mine)
{
    for (int j = threadIdx.x; j < p.k; j += THREADS) {
        Entry e = mine;
        if (j >= THREADS) {
            e = load_place(p, i, j, row.n > 0);
            load_logit(e, row);
        }
        put_entry(rec, j, e, row);
    }
}
template <bool BF16, int THREADS>
__device__ __forceinline__ void take_record_off(const Record &rec, const DistillArgs &p, const Row<BF16> &row)
{
    for (int j = threadIdx.x; j < p.k; j += THREADS)
        if (rec.at[j] >= 0) rec.bits[row.bit(rec.at[j]) >> 5] = 0;
}

// What a row's loss and coefficients need of its record
struct Teacher {
    bool some;              // whether there is a valid entry
    double p_sum, entropy;  // sum p, sum p log p
    double r;               // mass outside the record (before the student's rest is looked at)
    float ref;              // the record's largest z
    double cross;           // sum p (z - ref) / tau
    double in, in_ce;       // over its places: sum exp((z - ref) / tau), sum exp(z - ref)
};

// The student's largest logit in the record (by any wave); -inf without one
__device__ __forceinline__ float largest_in_record(const Record &rec, int k)
{
    float z = kNegInf;
    for (int j = threadIdx.x & (kWave - 1); j < k; j += kWave)
        if (rec.at[j] >= 0) z = fmaxf(z, rec.z[j]);
    return uniform(wave_max(z));
}

// By one wave: probabilities (into shared memory) and sums of the record there.  z_max: largest_in_record
__device__ __forceinline__ Teacher read_record(const Record &rec, const DistillArgs &p, int i, float z_max, bool sums, bool two)
{
    const int lane = threadIdx.x & (kWave - 1);
    const double inv = 1.0 / (double)p.temperature, log2e = 1.44269504088896340736;
    float top = kNegInf;
    for (int j = lane; j < p.k; j += kWave)
        if (rec.at[j] >= 0) top = fmaxf(top, rec.t[j]);
    top = wave_max(top);
    Teacher out;
    out.some = top > kNegInf;
    out.ref = z_max > kNegInf ? z_max : 0.f;
    double ref = 0.0, log_sum;  // logarithm of what p is divided by, relative to `ref`
    if (p.t_lse) {
        log_sum = (double)p.t_lse[i];
    } else {
        ref = out.some ? (double)top : 0.0;
        double part = 0.0;
        for (int j = lane; j < p.k; j += kWave)
            if (rec.at[j] >= 0) part += exp2_neg(((double)rec.t[j] - ref) * (inv * log2e), 0);
        log_sum = log(wave_sum(part));
    }
    const Exp<true> by_tau(p.temperature, out.ref), plain(1.0f, out.ref);  // (from the difference, whatever the logits' type)
    double p_sum = 0.0, entropy = 0.0, cross = 0.0, in = 0.0, in_ce = 0.0;
    bool twice = false;
    for (int j = lane; j < p.k; j += kWave) {
        double q = 0.0;
        if (rec.at[j] >= 0) {
            const double log_p = ((double)rec.t[j] - ref) * inv - log_sum;
            q = exp2_neg(log_p * log2e, 0);
            const float d = rec.z[j] - out.ref;
            if (q > 0.0) {
                entropy += q * log_p;
                cross += q * ((double)d * inv);
            }
            if (rec.first[j]) {
                in += (double)by_tau(rec.z[j]);
                if (two) in_ce += (double)plain(rec.z[j]);
            } else {
                twice = true;
            }
        }
        p_sum += q;
        rec.p[j] = q;
    }
    // Places named twice: the lowest entry stands for them, whichever thread came first to the bitmap
    if (__any(twice)) {
        wave_sync();
        in = in_ce = 0.0;
        for (int j = lane; j < p.k; j += kWave) {
            rec.t[j] = 0.f;  // (the record's t is not needed any more)
            rec.first[j] = false;
            int l = 0;
            while (rec.at[l] != rec.at[j]) ++l;
            if (rec.at[j] < 0 || l < j) continue;
            rec.first[j] = true;
            double q = 0.0;
            for (; l < p.k; ++l)
                if (rec.at[l] == rec.at[j]) q += rec.p[l];
            rec.t[j] = (float)q;
            if (sums) {
                in += (double)by_tau(rec.z[j]);
                if (two) in_ce += (double)plain(rec.z[j]);
            }
        }
        wave_sync();
        for (int j = lane; j < p.k; j += kWave) rec.p[j] = (double)rec.t[j];
    }
    out.p_sum = wave_sum(p_sum);
    out.r = p.t_lse ? fmax(0.0, 1.0 - out.p_sum) : 0.0;
    if (sums) {
        out.entropy = wave_sum(entropy);
        out.cross = wave_sum(cross);
        out.in = wave_sum(in);
        out.in_ce = two ? wave_sum(in_ce) : out.in;
    }
    return out;
}

// A block's share of a row: chunks [begin, end), the first share's with the row's edges
struct Span {
    int begin, end;
    bool edges;
    __device__ __forceinline__ Span(int part, int parts, int whole) : edges(part == 0)
    {
        const int each = (whole + parts - 1) / parts;
        begin = part * each < whole ? part * each : whole;
        end = begin + each < whole ? begin + each : whole;
    }
    // whether element `at` of the row is of this share
    template <bool BF16> __device__ __forceinline__ bool has(const Row<BF16> &row, int at) const
    {
        const int b = row.bit(at);
        return b < row.whole * Row<BF16>::E ? b >= begin * Row<BF16>::E && b < end * Row<BF16>::E : edges;
    }
};

// What the gradient of a row is made of, for dloss = 1; kept for the backward call as kDistillStats floats.
//   outside the record  u (one + second u), u = exp((z - ref) / tau), at temperatures 1 and 2 (a label's term is a power of u);
//                       elsewhere one u + second exp(z - ref)
//   in the record       in exp((z - max) / tau) + ce exp(z - max) - kd p
//   at the label        - label, in addition
enum { kNear = 1, kHasKd = 2, kHasLabel = 4 };
struct Coef {
    float ref, one, second, max, in, ce, kd, label;
    int flags;
    __device__ __forceinline__ Coef(const float *s, const DistillArgs &p, float g)  // g: dloss
        : ref(uniform(s[0])), one(uniform(s[1] * g)), second(uniform(s[2] * g)), max(uniform(s[3])), in(uniform(s[4] * g)), ce(uniform(s[5] * g)),
          flags((int)uniform(__float_as_uint(s[6])))
    {
        kd = flags & kHasKd ? uniform(p.kd_weight * p.temperature * g) : 0.f;
        label = flags & kHasLabel ? uniform(p.ce_weight * g) : 0.f;
    }
};

// A row's coefficients and loss from its record and the sums over the rest of it.  rest, rest_ce: sums of exp((z - ref) / tau) and exp(z - ref), as
// they are times 2^drift and 2^drift_ce
struct Finish {
    const Teacher &t;
    float ref, max;
    double rest, inv, to_rest, to_in, rest_scale, sum, sum_ce, second_scale, mass, r, kd, ce_weight;
    int label;
    bool any, live, two;
    __device__ __forceinline__ Finish(const DistillArgs &p, const Teacher &teacher, float ref_, double rest_, double rest_ce, double drift, double drift_ce,
                                      int label_, bool tail, bool two_)
        : t(teacher), ref(ref_), rest(rest_), label(label_), two(two_)
    {
        const double log2e = 1.44269504088896340736;
        any = rest != 0.0;  // (NaN is something)
        const bool held_some = t.in != 0.0;
        max = held_some ? (any ? fmaxf(ref, t.ref) : t.ref) : ref;
        inv = 1.0 / (double)p.temperature;
        // what turns the sums into sums relative to `max`, as powers of 2
        to_rest = any ? ((double)ref - (double)max) * inv * log2e - drift : 0.0;
        const double to_rest_ce = any ? ((double)ref - (double)max) * log2e - drift_ce : 0.0;
        to_in = held_some ? (double)t.ref - (double)max : 0.0;
        rest_scale = exp2_neg(to_rest, 0);
        second_scale = two ? exp2_neg(to_rest_ce, 0) : rest_scale;
        sum = rest * rest_scale;
        if (tail) sum += t.in * exp2_neg(to_in * inv * log2e, 0);
        sum_ce = sum;
        if (two) {
            sum_ce = rest_ce * second_scale;
            if (tail) sum_ce += t.in_ce * exp2_neg(to_in * log2e, 0);
        }
        live = sum != 0.0;
        r = tail && any && t.some ? t.r : 0.0;
        mass = t.p_sum + r;
        kd = (double)p.kd_weight * (double)p.temperature;
        ce_weight = (double)p.ce_weight;
    }
    __device__ __forceinline__ void coefficients(float *coef, bool near) const
    {
        const double over = 1.0 / sum, ce = live && label >= 0 ? ce_weight / sum_ce : 0.0;
        double one = live && t.some ? kd * (mass * rest_scale * over - (r > 0.0 ? r / rest : 0.0)) : 0.0;
        if (!two) one += ce * rest_scale;  // (temperature 1: the same exponentials)
        coef[0] = any ? ref : 0.f;
        coef[1] = (float)one;
        coef[2] = two ? (float)(ce * second_scale) : 0.f;
        coef[3] = live ? max : 0.f;
        coef[4] = live && t.some ? (float)(kd * mass * over) : 0.f;
        coef[5] = (float)ce;
        coef[6] = __uint_as_float((near ? kNear : 0) | (live && t.some ? kHasKd : 0) | (live && label >= 0 ? kHasLabel : 0));
        coef[7] = 0.f;
    }
    __device__ __forceinline__ double loss(const DistillArgs &p, float label_z) const
    {
        double out = 0.0;
        if (!live) return out;
        const double log_sum = log(sum);
        if (t.some) {
            out = t.entropy - t.cross + t.p_sum * (log_sum - to_in * inv);
            if (r > 0.0) out += r * (log(r) - (log(rest) + to_rest * 0.69314718055994530942 - log_sum));
            out *= kd * (double)p.temperature;
        }
        if (label >= 0) out += ce_weight * (log(sum_ce) - ((double)label_z - (double)max));
        return out;
    }
};

// The gradient of one row, place by place
template <bool BF16, bool ONCE> struct Gradient {
    static constexpr int E = Row<BF16>::E;
    Coef c;
    Exp<BF16> by_tau, plain;
    bool near, power, other;  // forms of the exponentials; whether there is a second term: a power of the first, or one of its own
    void *grad;
    bool same;  // its chunks lie as those of the logits

    __device__ __forceinline__ Gradient(const Coef &coef, const DistillArgs &p, const Row<BF16> &row, int64_t at)
        : c(coef), by_tau(p.temperature, c.ref), plain(1.0f, c.ref), near(c.flags & kNear)
    {
        other = c.second != 0.0f && p.temperature != 2.0f;
        power = c.second != 0.0f && p.temperature == 2.0f;
        grad = (char *)p.dlogits + at * p.ld_grad * (BF16 ? 2 : 4);
        same = (((uintptr_t)grad ^ (uintptr_t)row.row) & 15u) == 0;
    }
    template <int N> __device__ __forceinline__ void outside(float (&g)[8], const float (&z)[N]) const
    {
        // (the choices are the row's)
        if (near) {
#pragma unroll
            for (int e = 0; e < N; ++e) g[e] = by_tau.near(z[e]);
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e) g[e] = by_tau(z[e]);
        }
        if (power) {
#pragma unroll
            for (int e = 0; e < N; ++e) g[e] *= __builtin_fmaf(c.second, g[e], c.one);
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e) g[e] *= c.one;
        }
        if (other) {
#pragma unroll
            for (int e = 0; e < N; ++e) g[e] = __builtin_fmaf(c.second, near ? plain.near(z[e]) : plain(z[e]), g[e]);
        }
    }
    __device__ __forceinline__ void chunk(const Row<BF16> &row, const uint4 &v, int k) const
    {
        float g[8], z[E];
#pragma unroll
        for (int e = 0; e < E; ++e) z[e] = Row<BF16>::value(v, e);
        outside(g, z);
        char *to = (char *)grad + row.lo * (16 / E);
        if (same) {
            if (ONCE) __builtin_nontemporal_store(__builtin_bit_cast(u32x4, Row<BF16>::chunk(g)), (u32x4 *)to + k);
            else ((uint4 *)to)[k] = Row<BF16>::chunk(g);
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) Elem<BF16>::store(grad, row.lo + (int64_t)k * E + e, g[e]);
        }
    }
    // behind all chunks of the row: the edges, the record's places and the label's.  edge_z: this thread's edge
    __device__ __forceinline__ void edges(const Row<BF16> &row, float edge_z) const
    {
        if ((int)threadIdx.x >= row.edges) return;
        float g[8];
        const float z[1] = {edge_z};
        outside(g, z);
        Elem<BF16>::store(grad, row.edge_index(threadIdx.x), g[0]);
    }
    template <int THREADS>
    __device__ __forceinline__ void corrections(const Record &rec, const DistillArgs &p, const Row<BF16> &row, const Span &span, int label,
                                                float label_z, bool label_in_record) const
    {
        for (int j = threadIdx.x; j < p.k; j += THREADS)
            if (rec.at[j] >= 0 && rec.first[j] && span.has(row, rec.at[j])) entry(rec.at[j], rec.z[j], rec.p[j], p, label);
        if (label >= 0 && !label_in_record && threadIdx.x == 0 && span.has(row, label)) at_label(label, label_z);
    }
    // at a place of the record: its logit, its probability
    __device__ __forceinline__ void entry(int at, float z, double prob, const DistillArgs &p, int label) const
    {
        const Exp<BF16> kd(p.temperature, c.max), ce(1.0f, c.max);
        double g = (double)(c.in * kd(z)) - (double)c.kd * prob;
        if (c.ce != 0.0f) g += (double)(c.ce * ce(z)) - (at == label ? (double)c.label : 0.0);
        Elem<BF16>::store(grad, at, (float)g);
    }
    // at the label, outside the record
    __device__ __forceinline__ void at_label(int label, float label_z) const
    {
        float g[8];
        const float z[1] = {label_z};
        outside(g, z);
        Elem<BF16>::store(grad, label, g[0] - c.label);
    }
};

// f(chunk, its number, that it is not held) over a row's chunks [begin, end), U loads on the way at any time; BACK: the last ones first
template <bool BF16, int THREADS, int U, bool ONCE, bool BACK, typename F> __device__ __forceinline__ void stream(const Row<BF16> &row, int begin, int end, F f)
{
    const __amdgpu_buffer_rsrc_t from = row.buffer();  // (reads outside the row, before it too, give 0)
    constexpr int kStep = U * THREADS;
    const int steps = (end - begin + kStep - 1) / kStep;
    int c = begin + (int)threadIdx.x + (BACK ? (steps - 1) * kStep : 0);
    uint4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = load_chunk<ONCE>(from, c + u * THREADS);
    for (int i = 0; i < steps; ++i) {
        const int next = BACK ? c - kStep : c + kStep;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (c + u * THREADS < end) f(v[u], c + u * THREADS, std::false_type());
            v[u] = load_chunk<ONCE>(from, next + u * THREADS);
            __builtin_amdgcn_sched_barrier(0);
        }
        c = next;
    }
}

// A row's chunks: the first SLOTS * THREADS of them held in registers (thread t has chunks t, t + THREADS, ..), read once; what is
// beyond them is read again in every pass.
template <bool BF16, int THREADS, int SLOTS, bool ONCE> struct Held {
    uint4 v[SLOTS > 0 ? SLOTS : 1];

    // f(chunk, its number, whether it is held) over `row`, which is held; the chunk may be changed: what is held keeps the
    // change.  then(s, t): behind chunk s THREADS + t.
    template <typename F, typename Then> __device__ __forceinline__ void each(const Row<BF16> &row, F f, Then then)
    {
        // (a chunk at a time, and nothing worked out about it in one pass kept for the next: the registers are the row's)
        int t = threadIdx.x;
        asm volatile("" : "+v"(t));
#pragma unroll
        for (int s = 0; s < SLOTS; ++s) {
            if (t < row.whole - s * THREADS) f(v[s], s * THREADS + t, std::true_type());
            then(s, t);
            __builtin_amdgcn_sched_barrier(0);
        }
        stream<BF16, THREADS, SLOTS ? 1 : 4, SLOTS == 0 && ONCE, false>(row, SLOTS * THREADS, row.whole, f);  // (beside what is held it is read again)
    }
    template <typename F> __device__ __forceinline__ void each(const Row<BF16> &row, F f)
    {
        each(row, f, [](int, int) {});
    }
    // (through a buffer descriptor: what is beyond the row's last whole chunk is not read, without a branch)
    __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t row, int s, int t)
    {
        v[s] = load_chunk<ONCE>(row, s * THREADS + t);
    }
};

// Takes the record's places out of a chunk (-inf)
template <bool BF16> __device__ __forceinline__ void mask_chunk(uint4 &v, const uint32_t *bits, int c)
{
    constexpr int E = Row<BF16>::E;
    uint32_t in = ((const uint8_t *)bits)[c * E >> 3];
    if (!BF16) in = (in >> (c * E & 7)) & 15u;
    if (in) {
        uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int e = 0; e < E; ++e) {
            if (!(in >> e & 1u)) continue;
            if (BF16) w[e >> 1] = (e & 1) ? (w[e >> 1] & 0xffffu) | 0xff800000u : (w[e >> 1] & 0xffff0000u) | 0xff80u;
            else w[e] = 0xff800000u;
        }
        v = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// A block takes rows blockIdx.x, + gridDim.x, ..: record, sums, loss, and with GRAD the gradient.  While a row's gradient is written, each
// chunk's registers take the next row's: the memory has work while the block computes, though a row of 128 Ki bf16
// leaves no registers for a second block beside it.  With 16 or 20 chunks a thread also has 160 to 260 bytes of scratch memory: addresses and constants that
// are read again between the sums and the gradient, not the row (3 % more bytes written than the gradient has).  Bound by memory: loss and gradient of 8192 x 128256
// bf16 975 us (4.3 TB/s), of 1000 x 128256 fp32 268 (3.8 TB/s), loss alone of 1792 x 32000 bf16 25 us (4.6 TB/s), of 1000 x 128256 fp32 82 (6.3 TB/s, in part from
// the last-level cache); 32 x 32000 in one call 11.3 us.  The first wave does the record's and the row's arithmetic in 64 bits.
template <bool BF16, int THREADS, int SLOTS, bool GRAD, bool ONCE> __global__ void __launch_bounds__(THREADS, SLOTS ? 4 : 8) distill_kernel(DistillArgs p)
{
    constexpr int E = Row<BF16>::E, W = THREADS / kWave;
    __shared__ Shared<THREADS> sh;
    extern __shared__ double mem[];
    const Record rec(mem, p.k, p.r.vocab);
    uint32_t *const bits = rec.bits;
    const bool tail = p.t_lse != nullptr;  // the rest of the row is a term of its own
    const int lane = threadIdx.x & (kWave - 1), wave = uniform((uint32_t)threadIdx.x / kWave);
    Held<BF16, THREADS, SLOTS, ONCE> held;
    auto row_at = [&](int i) {  // (a row that is not there has no logits)
        const void *at = i < p.r.n_rows ? row_of(p.r, i) : nullptr;
        return Row<BF16>(at, at ? p.r.vocab : 0);
    };
    // What a thread needs of a row beside its chunks is on its way before them, in two steps (loads arrive in order): places first,
    // then the logits there.
    struct {
        Entry entry;
        float edge_z, label_z, dloss;
        int label;
    } ahead;
    auto load_places = [&](int i, const Row<BF16> &row) {
        ahead.entry = load_place(p, i, threadIdx.x, row.n > 0);
        ahead.label = row.n > 0 && p.labels ? p.labels[i] : -1;
        ahead.dloss = row.n > 0 && GRAD ? p.dloss[i] : 0.f;
    };
    auto load_logits = [&](const Row<BF16> &row) {
        load_logit(ahead.entry, row);
        ahead.edge_z = row.edge(threadIdx.x);
        ahead.label = (int)uniform((uint32_t)ahead.label);
        if (ahead.label < 0 || ahead.label >= row.n) ahead.label = -1;
        ahead.label_z = ahead.label >= 0 ? Elem<BF16>::load(row.row, ahead.label) : 0.f;
    };
    int i = blockIdx.x;
    Row<BF16> row = row_at(i);
    load_places(i, row);
    load_logits(row);
    {
        const __amdgpu_buffer_rsrc_t from = row.buffer();
#pragma unroll
        for (int s = 0; s < SLOTS; ++s) held.load(from, s, threadIdx.x);
    }
    for (int w = threadIdx.x; w < (p.r.vocab + 31) / 32; w += THREADS) bits[w] = 0;
    __syncthreads();
    for (;;) {
        put_record<BF16, THREADS>(rec, p, i, row, ahead.entry);
        __syncthreads();
        const int label = ahead.label;
        const float label_z = ahead.label_z, edge_z = ahead.edge_z, dloss = ahead.dloss;
        const int next = SLOTS > 0 ? i + (int)gridDim.x : p.r.n_rows;  // (a block that holds nothing takes one row)
        const Row<BF16> next_row = row_at(next);
        load_places(next, next_row);
        const int b = label >= 0 ? row.bit(label) : 0;
        const bool label_in_record = label >= 0 && (bits[b >> 5] >> (b & 31) & 1u);
        const bool two = label >= 0 && p.temperature != 1.0f, other = two && p.temperature != 2.0f;  // a second softmax, of its own
        const float z_max = largest_in_record(rec, p.k);
        Teacher t;
        if (wave == 0) t = read_record(rec, p, i, z_max, true, two);
        float ref = z_max > kNegInf ? z_max : 0.f;
        const Exp<BF16> by_tau(p.temperature, ref), plain(1.0f, ref);
        float edge_out = edge_z;
        {
            const int e = row.whole * E + threadIdx.x;
            if (tail && (int)threadIdx.x < row.edges && (bits[e >> 5] >> (e & 31) & 1u)) edge_out = kNegInf;
        }
        // over the rest of the row: sums of exp((z - ref) / tau) and, for the label at another temperature, of exp(z - ref); at temperature
        // 2 the latter is the former's square
        double part, part_ce;  // (a chunk's terms in 32 bits, chunks in 64)
        {
            const float u = by_tau.near(edge_out);
            part = (double)u;
            part_ce = (double)(other ? plain.near(edge_out) : u * u);
        }
        held.each(row, [&](uint4 &v, int k, auto) {
            if (tail) mask_chunk<BF16>(v, bits, k);
            float s = 0.f, s_ce = 0.f;
            if (other) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    s += by_tau.near(Row<BF16>::value(v, e));
                    s_ce += plain.near(Row<BF16>::value(v, e));
                }
                part_ce += (double)s_ce;
            } else if (two) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float u = by_tau.near(Row<BF16>::value(v, e));
                    s += u;
                    s_ce = __builtin_fmaf(u, u, s_ce);
                }
                part_ce += (double)s_ce;
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e) s += by_tau.near(Row<BF16>::value(v, e));
            }
            part += (double)s;
        });
        load_logits(next_row);
        double rest = wave_sum(part), rest_ce = two ? wave_sum(part_ce) : 1.0;
        if (lane == 0) {
            sh.sum[wave] = rest;
            sh.sum_ce[wave] = rest_ce;
        }
        __syncthreads();
        rest = uniform(wave_sum(lane < W ? sh.sum[lane] : 0.0));
        rest_ce = uniform(wave_sum(lane < W ? sh.sum_ce[lane] : 0.0));
        double drift = by_tau.drift(), drift_ce = other ? plain.drift() : 2.0 * drift;
        // finite, drifts that are roundings, and a rest that is not so small that the gradient would miss what was lost (3e-11 of the
        // record's largest term, times 2^32: it then is less than 1e-37 of the rest)
        const bool near = rest > 0.125 && rest < 1e30 && rest_ce > 1e-15 && rest_ce < 1e30 && by_tau.sound() && plain.sound();
        if (!near) {
            Running run;
            const float z[1] = {edge_out};
            run.add(z, by_tau.c);
            held.each(row, [&](uint4 &v, int k, auto is_held) {
                if (!is_held && tail) mask_chunk<BF16>(v, bits, k);
                float z[E];
#pragma unroll
                for (int e = 0; e < E; ++e) z[e] = Row<BF16>::value(v, e);
                run.add(z, by_tau.c);
            });
            __syncthreads();
            const float m = wave_max(run.m);
            run.raise(m, by_tau.c);
            rest = wave_sum(run.s);
            rest_ce = wave_sum(run.ce);
            if (lane == 0) {
                sh.max[wave] = m;
                sh.sum[wave] = rest;
                sh.sum_ce[wave] = rest_ce;
            }
            __syncthreads();
            const float wave_ref = lane < W ? sh.max[lane] : kLow;
            ref = uniform(wave_max(wave_ref));
            rest = uniform(wave_sum(lane < W ? sh.sum[lane] * (double)__builtin_amdgcn_exp2f((wave_ref - ref) * by_tau.c) : 0.0));
            rest_ce = uniform(wave_sum(lane < W ? sh.sum_ce[lane] * (double)__builtin_amdgcn_exp2f((wave_ref - ref) * 1.44269504f) : 0.0));
            drift = drift_ce = 0.0;
        }
        take_record_off<BF16, THREADS>(rec, p, row);
        if (wave == 0) {
            const Finish end(p, t, ref, rest, rest_ce, drift, drift_ce, label, tail, two);
            if (lane == 0) end.coefficients(sh.coef, near);
            if (GRAD) __syncthreads();
            // (the loss itself while the other waves go on)
            const double loss = end.loss(p, label_z);
            if (lane == 0) p.loss[i] = (float)loss;
            if (p.stats) {
                if (!GRAD) wave_sync();
                if (lane < kDistillStats) p.stats[(int64_t)i * kDistillStats + lane] = sh.coef[lane];
            }
        } else if (GRAD) {
            __syncthreads();
        }
        const __amdgpu_buffer_rsrc_t from = next_row.buffer();
        if (GRAD) {
            const Gradient<BF16, ONCE> g(Coef(sh.coef, p, dloss), p, row, row.n > 0 && p.r.rows ? (int64_t)__builtin_amdgcn_readfirstlane(p.r.rows[i]) : i);
            held.each(row, [&](uint4 &v, int k, auto) { g.chunk(row, v, k); }, [&](int s, int t) { held.load(from, s, t); });
            g.edges(row, edge_z);
            __syncthreads();
            g.template corrections<THREADS>(rec, p, row, Span(0, 1, row.whole), label, label_z, label_in_record);
        } else {
#pragma unroll
            for (int s = 0; s < SLOTS; ++s) held.load(from, s, threadIdx.x);
            __syncthreads();
        }
        if (SLOTS == 0 || next >= p.r.n_rows) return;
        i = next;
        row = next_row;
    }
}

// The gradient from what the forward call kept.  Rows and their chunks go from the last to the first: the forward call left the last-read
// ones in the last-level cache.  A row is `parts` blocks', each reading of the logits what it writes the gradient of (which may lie in their
// place); the record's probabilities are worked out by each.  1024 x 128256 bf16 97 us (5.4 TB/s, in part from the cache), 205 x 50257 fp32 16 us.
template <bool BF16, int THREADS, bool ONCE> __global__ void __launch_bounds__(THREADS, 8) distill_bwd_kernel(DistillArgs p, int parts)
{
    extern __shared__ double mem[];
    const Record rec(mem, p.k, p.r.vocab);
    uint32_t *const bits = rec.bits;
    const int block = (int)blockIdx.x / parts, i = p.r.n_rows - 1 - block;
    const void *at = row_of(p.r, i);
    if (!at) return;
    const Row<BF16> row(at, p.r.vocab);
    const Span span((int)blockIdx.x - block * parts, parts, row.whole);
    for (int w = threadIdx.x; w < (row.n + 31) / 32; w += THREADS) bits[w] = 0;
    __syncthreads();
    for (int j = threadIdx.x; j < p.k; j += THREADS) {
        Entry e = load_place(p, i, j, true);
        load_logit(e, row, &span);
        put_entry(rec, j, e, row);
    }
    int label = p.labels ? p.labels[i] : -1;
    if (label >= row.n) label = -1;
    const float label_z = label >= 0 && span.has(row, label) ? Elem<BF16>::load(at, label) : 0.f, edge_z = row.edge(threadIdx.x);
    __syncthreads();  // (every thread has read what it needs beside its chunks: the gradient may lie in the place of the logits)
    const int b = label >= 0 ? row.bit(label) : 0;
    const bool label_in_record = label >= 0 && (bits[b >> 5] >> (b & 31) & 1u);
    if (threadIdx.x < kWave) read_record(rec, p, i, kNegInf, false, false);
    const Gradient<BF16, ONCE> g(Coef(p.stats + (int64_t)i * kDistillStats, p, p.dloss[i]), p, row, p.r.rows ? (int64_t)p.r.rows[i] : i);
    stream<BF16, THREADS, 4, false, true>(row, span.begin, span.end, [&](const uint4 &v, int k, auto) { g.chunk(row, v, k); });
    if (span.edges) g.edges(row, edge_z);
    __syncthreads();
    g.template corrections<THREADS>(rec, p, row, span, label, label_z, label_in_record);
}

// ---- few rows: loss and gradient by many blocks a row, in two launches ----
// What the first launch leaves of a row in the workspace: the record's part by a block of its own, the sums over the rest by `parts` blocks, each
// relative to the largest logit it met.
struct Head {
    Teacher t;
    int label;
    float label_z;
    bool label_in_record;
};
struct Part {
    double s, ce;
    float m;
};
struct Kept {
    Head *head;
    Part *parts;
    double *p;
    float *z;
    int32_t *at;  // -1: no entry, or not its place's first
    static __host__ __device__ int64_t bytes(int k, int parts) { return ((int64_t)sizeof(Head) + parts * (int64_t)sizeof(Part) + k * (int64_t)16 + 15) / 16 * 16; }
    __device__ __forceinline__ Kept(const DistillArgs &a, int i, int n_parts)
        : head((Head *)((char *)a.workspace + i * bytes(a.k, n_parts))), parts((Part *)(head + 1)), p((double *)(parts + n_parts)), z((float *)(p + a.k)),
          at((int32_t *)(z + a.k))
    {
    }
};
static_assert(sizeof(Head) % 8 == 0 && sizeof(Part) % 8 == 0, "what follows them is 8-byte aligned");

// Block (row, part), the row's last block its record's: its arithmetic in 64 bits, the longest chain here, runs beside the sums.  Both launches together: one
// row of 128256 bf16 11.2 us, of 160000 fp32 11.1, 64 rows of 128256 20.8.
template <bool BF16, int THREADS> __global__ void __launch_bounds__(THREADS) distill_parts_kernel(DistillArgs p, int parts)
{
    constexpr int E = Row<BF16>::E, U = 4, W = THREADS / kWave;
    extern __shared__ double mem[];
    __shared__ Shared<THREADS> sh;
    const int i = (int)blockIdx.x / (parts + 1), part = (int)blockIdx.x - i * (parts + 1);
    const int lane = threadIdx.x & (kWave - 1), wave = (int)uniform((uint32_t)threadIdx.x / kWave);
    const void *start = row_of(p.r, i);
    if (!start) return;
    const Row<BF16> row(start, p.r.vocab);
    const Kept kept(p, i, parts);
    const bool tail = p.t_lse != nullptr;
    int label = (int)uniform((uint32_t)(p.labels ? p.labels[i] : -1));
    if (label < 0 || label >= row.n) label = -1;
    const bool two = label >= 0 && p.temperature != 1.0f;
    if (part == parts) {
        const Record rec(mem, p.k, p.r.vocab);
        Entry mine = load_place(p, i, threadIdx.x, true);
        for (int w = threadIdx.x; w < (row.n + 31) / 32; w += THREADS) rec.bits[w] = 0;
        load_logit(mine, row);
        const float label_z = label >= 0 ? Elem<BF16>::load(start, label) : 0.f;
        __syncthreads();
        put_record<BF16, THREADS>(rec, p, i, row, mine);
        __syncthreads();
        const float z_max = largest_in_record(rec, p.k);
        if (wave == 0) {
            const Teacher t = read_record(rec, p, i, z_max, true, two);
            if (lane == 0) {
                const int b = label >= 0 ? row.bit(label) : 0;
                kept.head->t = t;
                kept.head->label = label;
                kept.head->label_z = label_z;
                kept.head->label_in_record = label >= 0 && (rec.bits[b >> 5] >> (b & 31) & 1u);
            }
        }
        __syncthreads();
        for (int j = threadIdx.x; j < p.k; j += THREADS) {
            kept.p[j] = rec.p[j];
            kept.z[j] = rec.z[j];
            kept.at[j] = rec.first[j] ? rec.at[j] : -1;
        }
        return;
    }
    // this part of the rest of the row; the bitmap is of its chunks and, behind them, of the edges
    const Span span(part, parts, row.whole);
    uint32_t *const bits = (uint32_t *)mem;
    const __amdgpu_buffer_rsrc_t from = row.buffer();
    uint4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = load_chunk<false>(from, span.begin + u * THREADS + (int)threadIdx.x);
    const int first = span.begin * E, here = (span.end - span.begin) * E;
    float edge_z = span.edges ? row.edge(threadIdx.x) : kNegInf;
    if (tail) {
        for (int w = threadIdx.x; w < (here + 2 * E + 31) / 32; w += THREADS) bits[w] = 0;
        __syncthreads();
        for (int j = threadIdx.x; j < p.k; j += THREADS) {
            const Entry e = load_place(p, i, j, true);
            if (e.at < 0 || e.at >= row.n || !(e.t > kNegInf) || !span.has(row, e.at)) continue;
            const int b = row.bit(e.at), to = b < row.whole * E ? b - first : here + (b - row.whole * E);
            atomicOr(&bits[to >> 5], 1u << (to & 31));
        }
        __syncthreads();
        const int e = here + (int)threadIdx.x;
        if (span.edges && (int)threadIdx.x < row.edges && (bits[e >> 5] >> (e & 31) & 1u)) edge_z = kNegInf;
    }
    const float c = (float)(1.44269504088896340736 / (double)p.temperature);
    Running run;
    {
        const float z[1] = {edge_z};
        run.add(z, c);
    }
    for (int k = span.begin + (int)threadIdx.x; k < span.end; k += U * THREADS) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int at = k + u * THREADS;
            if (at < span.end) {
                if (tail) mask_chunk<BF16>(v[u], bits, at - span.begin);
                float z[E];
#pragma unroll
                for (int e = 0; e < E; ++e) z[e] = Row<BF16>::value(v[u], e);
                run.add(z, c);
            }
            v[u] = load_chunk<false>(from, at + U * THREADS);
        }
    }
    const float m = wave_max(run.m);
    run.raise(m, c);
    const double s = wave_sum(run.s), ce = wave_sum(run.ce);
    if (lane == 0) {
        sh.max[wave] = m;
        sh.sum[wave] = s;
        sh.sum_ce[wave] = ce;
    }
    __syncthreads();
    if (wave == 0) {
        const float wave_m = lane < W ? sh.max[lane] : kLow, top = wave_max(wave_m);
        const double all = wave_sum(lane < W ? sh.sum[lane] * (double)__builtin_amdgcn_exp2f((wave_m - top) * c) : 0.0);
        const double all_ce = wave_sum(lane < W ? sh.sum_ce[lane] * (double)__builtin_amdgcn_exp2f((wave_m - top) * 1.44269504f) : 0.0);
        if (lane == 0) kept.parts[part] = {all, all_ce, top};
    }
}

// Block (row, part): every wave joins the sums; the gradient of the part, the loss by the first part's last wave.  Of the logits only the part's
// own are read, as the gradient may lie in their place.
template <bool BF16, int THREADS> __global__ void __launch_bounds__(THREADS) distill_join_kernel(DistillArgs p, int parts)
{
    const int i = (int)blockIdx.x / parts, part = (int)blockIdx.x - i * parts;
    const int lane = threadIdx.x & (kWave - 1);
    const void *start = row_of(p.r, i);
    if (!start) {
        if (part == 0 && threadIdx.x == 0) p.loss[i] = 0.0f;
        return;
    }
    const Row<BF16> row(start, p.r.vocab);
    const Span span(part, parts, row.whole);
    const Kept kept(p, i, parts);
    const float edge_z = row.edge(threadIdx.x);
    const Teacher t = kept.head->t;
    const int label = kept.head->label;
    const float label_z = kept.head->label_z, c = (float)(1.44269504088896340736 / (double)p.temperature);
    const Part mine = lane < parts ? kept.parts[lane] : Part{0.0, 0.0, kLow};
    const float ref = uniform(wave_max(mine.m));
    const double rest = uniform(wave_sum(mine.s * (double)__builtin_amdgcn_exp2f((mine.m - ref) * c)));
    const double rest_ce = uniform(wave_sum(mine.ce * (double)__builtin_amdgcn_exp2f((mine.m - ref) * 1.44269504f)));
    const bool two = label >= 0 && p.temperature != 1.0f;
    const Finish end(p, t, ref, rest, rest_ce, 0.0, 0.0, label, p.t_lse != nullptr, two);
    float coef[kDistillStats];
    end.coefficients(coef, false);
    const Gradient<BF16, false> g(Coef(coef, p, p.dloss[i]), p, row, p.r.rows ? (int64_t)__builtin_amdgcn_readfirstlane(p.r.rows[i]) : i);
    stream<BF16, THREADS, 4, false, false>(row, span.begin, span.end, [&](const uint4 &v, int k, auto) { g.chunk(row, v, k); });
    if (span.edges) g.edges(row, edge_z);
    __syncthreads();
    for (int j = threadIdx.x; j < p.k; j += THREADS) {
        const int at = kept.at[j];
        if (at >= 0 && span.has(row, at)) g.entry(at, kept.z[j], kept.p[j], p, label);
    }
    if (threadIdx.x == 0 && label >= 0 && !kept.head->label_in_record && span.has(row, label)) g.at_label(label, label_z);
    if (part == 0 && threadIdx.x == THREADS - 1) p.loss[i] = (float)end.loss(p, label_z);
}

// Shares of a row that together with those of the other rows make up to `blocks` blocks, none below 1024 chunks; rows of up to 4096, which one block
// reads in four loads a thread, are not shared.  (A share of 512 chunks takes no less time, and with twice the blocks every one waits for its record.)
constexpr int kMostParts = kWave;
int parts_of(const DistillArgs &a, int chunks, int blocks)
{
    if (chunks <= 4 * 1024) return 1;
    int parts = blocks / a.r.n_rows;
    if (parts > chunks / 1024) parts = chunks / 1024;
    return parts < 1 ? 1 : parts > kMostParts ? kMostParts : parts;
}

template <int THREADS, typename K, typename... More> hipError_t launch(K kernel, int blocks, const DistillArgs &a, hipStream_t st, More... more)
{
    const size_t bytes = Record::bytes(a.k, a.r.vocab);  // up to 150 KiB
    if (bytes + sizeof(Shared<THREADS>) > (64u << 10)) {
        const hipError_t e = hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
        if (e != hipSuccess) return e;
    }
    COLLM_LAUNCH(kernel, dim3(blocks), dim3(THREADS), bytes, st, a, more...);
    return hipGetLastError();
}

template <bool BF16, int THREADS, int SLOTS, bool ONCE> hipError_t launch_held(const DistillArgs &a, hipStream_t st)
{
    const int fit = a.compute_units * (1024 / THREADS);  // blocks at a time, by their registers
    return launch<THREADS>(distill_kernel<BF16, THREADS, SLOTS, true, ONCE>, a.r.n_rows < fit ? a.r.n_rows : fit, a, st);
}

// Whether a call's rows are more than the last-level cache (256 MiB) keeps beside their gradient until something reads them again
bool past_the_cache(const LogitRows &r) { return (int64_t)r.n_rows * r.vocab * (r.bf16 ? 2 : 4) > (int64_t)128 << 20; }

// With the gradient, the block that holds a row in registers: the smallest that does where there are rows for all compute units, one of 1024
// threads where there are fewer.  From 1024 threads with 20 chunks each on, the rest of a row is read again.
template <bool BF16, bool ONCE> hipError_t launch_many(const DistillArgs &a, int chunks, hipStream_t st)
{
    if (chunks <= 256 * 16) return launch_held<BF16, 256, 16, ONCE>(a, st);
    if (chunks <= 512 * 16) return launch_held<BF16, 512, 16, ONCE>(a, st);
    if (chunks <= 1024 * 16) return launch_held<BF16, 1024, 16, ONCE>(a, st);
    return launch_held<BF16, 1024, 20, ONCE>(a, st);
}
template <bool BF16> hipError_t launch_step(const DistillArgs &a, hipStream_t st)
{
    const int chunks = a.r.vocab / Row<BF16>::E, parts = parts_of(a, chunks, a.compute_units);
    // Shares of a quarter of a row or less: one / 32 / 64 rows of 128256 bf16 22.6 / 24.4 / 25.8 -> 11.2 / 15.5 / 20.8 us, one row of 160000 fp32
    // 33.8 -> 11.1 (bf16 64000: 14.5 -> 11.8).  Halves lose: the logits are read twice, in two launches (128 rows of 128256: 29.4 -> 31.3).
    if (parts >= 4 && a.workspace_bytes >= a.r.n_rows * Kept::bytes(a.k, parts)) {
        const hipError_t e = launch<512>(distill_parts_kernel<BF16, 512>, a.r.n_rows * (parts + 1), a, st, parts);
        if (e != hipSuccess) return e;
        COLLM_LAUNCH((distill_join_kernel<BF16, 512>), dim3(a.r.n_rows * parts), dim3(512), 0, st, a, parts);
        return hipGetLastError();
    }
    if (past_the_cache(a.r)) return launch_many<BF16, true>(a, chunks, st);
    if (a.r.n_rows <= a.compute_units) {
        if (chunks <= 1024 * 4) return launch_held<BF16, 1024, 4, false>(a, st);
        if (chunks <= 1024 * 8) return launch_held<BF16, 1024, 8, false>(a, st);
        if (chunks <= 1024 * 16) return launch_held<BF16, 1024, 16, false>(a, st);
    }
    return launch_many<BF16, false>(a, chunks, st);
}

// Without it a row is read once by any block, a block a row: as small as leaves every compute unit its 2048 threads.
template <bool BF16, bool ONCE> hipError_t launch_loss(const DistillArgs &a, hipStream_t st)
{
    if (a.r.n_rows >= 8 * a.compute_units) return launch<256>(distill_kernel<BF16, 256, 0, false, ONCE>, a.r.n_rows, a, st);
    if (a.r.n_rows >= 4 * a.compute_units) return launch<512>(distill_kernel<BF16, 512, 0, false, ONCE>, a.r.n_rows, a, st);
    return launch<1024>(distill_kernel<BF16, 1024, 0, false, ONCE>, a.r.n_rows, a, st);
}

template <bool BF16, bool ONCE> hipError_t launch_gradient(const DistillArgs &a, hipStream_t st)
{
    if (a.r.n_rows >= 4 * a.compute_units) return launch<256>(distill_bwd_kernel<BF16, 256, ONCE>, a.r.n_rows, a, st, 1);
    if (a.r.n_rows >= 2 * a.compute_units) return launch<512>(distill_bwd_kernel<BF16, 512, ONCE>, a.r.n_rows, a, st, 1);
    // (a block for every second compute unit: forward and backward of one / 64 rows of 128256 bf16 21.4 / 25.1 -> 16.7 / 22.0 us, one row of
    // 160000 fp32 27.8 -> 19; with a block for each 32 rows take 20.2 instead of 19.3)
    const int parts = parts_of(a, a.r.vocab / Row<BF16>::E, a.compute_units / 2);
    return launch<1024>(distill_bwd_kernel<BF16, 1024, ONCE>, a.r.n_rows * parts, a, st, parts);
}

}  // namespace

hipError_t launch_distill_fwd(const DistillArgs &a, hipStream_t st)
{
    // (a backward call, for which `stats` is kept, reads the logits again)
    if (!a.stats) return a.r.bf16 ? launch_loss<true, true>(a, st) : launch_loss<false, true>(a, st);
    return a.r.bf16 ? launch_loss<true, false>(a, st) : launch_loss<false, false>(a, st);
}
hipError_t launch_distill_bwd(const DistillArgs &a, hipStream_t st)
{
    if (past_the_cache(a.r)) return a.r.bf16 ? launch_gradient<true, true>(a, st) : launch_gradient<false, true>(a, st);
    return a.r.bf16 ? launch_gradient<true, false>(a, st) : launch_gradient<false, false>(a, st);
}
hipError_t launch_distill_fwd_bwd(const DistillArgs &a, hipStream_t st) { return a.r.bf16 ? launch_step<true>(a, st) : launch_step<false>(a, st); }

}  // namespace collm
