// Distillation from a teacher's top logits: the loss of a row of student logits z and its gradient.
//
// The teacher's record of a row is k logits t and their places.  With temperature tau, p = softmax(t / tau) over the
// record, or, with the teacher's own log-sum-exp, p = exp(t / tau - lse) and r = max(0, 1 - sum p) for all other places.
// With q = softmax(z / tau), P = sum p + r and `rest` = the places outside the record,
//   KD   = sum_k p_k (log p_k - log q_k) + r (log r - log sum_rest q)
//   loss = a tau^2 KD + b CE,   CE = -log softmax(z)[label]
//   dloss/dz_v = a tau (P q_v - p_v - [v in rest] r q_v / sum_rest q) + b (softmax(z)_v - [v = label]).
// Outside the record the gradient is one multiple of exp((z_v - ref) / tau) plus one of exp(z_v - max): the row is two
// coefficients, and the places of the record and of the label are written again, behind the others, from sums in 64 bits.
// The sum over the rest is taken over the rest alone (a bitmap of the record in shared memory masks it), relative to its own
// largest logit: 1 - sum q would lose it where the record holds nearly all of the mass.  Sums are taken in one pass, each thread
// relative to the largest logit that it has met.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "kernels.h"
#include "vocab_device.h"

namespace collm {

namespace {

using namespace vocab;

constexpr float kLow = -3.402823466e+38f;  // the least finite value: a running maximum begins here, so that -inf adds nothing

// exp(d / tau) for d <= 0: the rounding of the factor and of the product are errors of |d / tau| 2^-24 each, small where the result is not
struct Exp {
    float c;
    __device__ __forceinline__ explicit Exp(float tau) : c(uniform((float)(1.44269504088896340736 / (double)tau))) {}
    __device__ __forceinline__ float operator()(float d) const { return __builtin_amdgcn_exp2f(d * c); }
};

// A teacher's record of a row in shared memory, and what the waves of a block tell each other
template <int THREADS> struct Shared {
    double sum[THREADS / kWave], sum_ce[THREADS / kWave];
    float max[THREADS / kWave];
    float coef[8];
    double p[kMaxTop];       // probabilities (of a place named twice: their sum, at its first entry)
    float t[kMaxTop], z[kMaxTop];  // the teacher's and the student's logits
    int32_t at[kMaxTop];     // places; -1: not an entry
    uint8_t first[kMaxTop];  // whether the entry is its place's first
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
template <bool BF16> __device__ __forceinline__ void load_logit(Entry &e, const Row<BF16> &row)
{
    if (e.at < 0 || e.at >= row.n || !(e.t > kNegInf)) e.at = -1;
    else e.z = Elem<BF16>::load(row.row, e.at);
}

// Row i's record into shared memory, its places into the bitmap.  mine: the entry of this thread's index, loaded before.
template <bool BF16, int THREADS>
__device__ __forceinline__ void put_record(Shared<THREADS> &sh, uint32_t *bits, const DistillArgs &p, int i, const Row<BF16> &row, const Entry &mine)
{
    for (int j = threadIdx.x; j < p.k; j += THREADS) {
        Entry e = mine;
        if (j >= THREADS) {
            e = load_place(p, i, j, row.n > 0);
            load_logit(e, row);
        }
        sh.at[j] = e.at;
        sh.t[j] = e.t;
        sh.z[j] = e.z;
        bool first = false;
        if (e.at >= 0) {
            const int b = row.bit(e.at);
            first = !(atomicOr(&bits[b >> 5], 1u << (b & 31)) >> (b & 31) & 1u);
        }
        sh.first[j] = first;
    }
}
template <bool BF16, int THREADS>
__device__ __forceinline__ void take_record_off(const Shared<THREADS> &sh, uint32_t *bits, const DistillArgs &p, const Row<BF16> &row)
{
    for (int j = threadIdx.x; j < p.k; j += THREADS)
        if (sh.at[j] >= 0) bits[row.bit(sh.at[j]) >> 5] = 0;
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

// What a row's loss and coefficients need of its record
struct Teacher {
    bool some;              // whether there is a valid entry
    double p_sum, entropy;  // sum p, sum p log p
    double r;               // mass outside the record (before the student's rest is looked at)
    float ref;              // the record's largest z
    double cross;           // sum p (z - ref) / tau
    double in, in_ce;       // over its places: sum exp((z - ref) / tau), sum exp(z - ref)
};

// By one wave: probabilities (into shared memory) and sums of the record there
template <int THREADS> __device__ Teacher read_record(Shared<THREADS> &sh, const DistillArgs &p, int i, bool sums, bool two)
{
    const int lane = threadIdx.x & (kWave - 1);
    const double inv = 1.0 / (double)p.temperature, log2e = 1.44269504088896340736;
    float top = kNegInf, z_max = kNegInf;
    for (int j = lane; j < p.k; j += kWave)
        if (sh.at[j] >= 0) {
            top = fmaxf(top, sh.t[j]);
            z_max = fmaxf(z_max, sh.z[j]);
        }
    top = wave_max(top);
    z_max = wave_max(z_max);
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
            if (sh.at[j] >= 0) part += exp2_neg(((double)sh.t[j] - ref) * (inv * log2e), 0);
        log_sum = log(wave_sum(part));
    }
    const Exp by_tau(p.temperature), plain(1.0f);
    double p_sum = 0.0, entropy = 0.0, cross = 0.0, in = 0.0, in_ce = 0.0;
    bool twice = false;
    for (int j = lane; j < p.k; j += kWave) {
        double q = 0.0;
        if (sh.at[j] >= 0) {
            const double log_p = ((double)sh.t[j] - ref) * inv - log_sum;
            q = exp2_neg(log_p * log2e, 0);
            const float d = sh.z[j] - out.ref;
            if (q > 0.0) {
                entropy += q * log_p;
                cross += q * ((double)d * inv);
            }
            if (sh.first[j]) {
                in += (double)by_tau(d);
                if (two) in_ce += (double)plain(d);
            } else {
                twice = true;
            }
        }
        p_sum += q;
        sh.p[j] = q;
    }
    out.p_sum = wave_sum(p_sum);
    out.r = p.t_lse ? fmax(0.0, 1.0 - out.p_sum) : 0.0;
    if (sums) {
        out.entropy = wave_sum(entropy);
        out.cross = wave_sum(cross);
        out.in = wave_sum(in);
        out.in_ce = two ? wave_sum(in_ce) : out.in;
    }
    if (__any(twice)) {
        for (int j = lane; j < p.k; j += kWave) {
            double q = 0.0;
            if (sh.first[j])
                for (int l = 0; l < p.k; ++l)
                    if (sh.at[l] == sh.at[j]) q += sh.p[l];
            sh.t[j] = (float)q;  // (the record's t is not needed any more)
        }
        for (int j = lane; j < p.k; j += kWave) sh.p[j] = (double)sh.t[j];
    }
    return out;
}

// What the gradient of a row is made of, for dloss = 1:
//   outside the record  out * exp((z - ref) / tau) + ce * exp(z - max)
//   in the record       in * exp((z - max) / tau) + ce * exp(z - max) - kd * p
//   at the label        - label, in addition
struct Coef {
    float ref, out, max, in, ce, kd, label;
    __device__ __forceinline__ explicit Coef(const float *s)
        : ref(uniform(s[0])), out(uniform(s[1])), max(uniform(s[2])), in(uniform(s[3])), ce(uniform(s[4])), kd(uniform(s[5])), label(uniform(s[6]))
    {
    }
    __device__ __forceinline__ void scale(float g)
    {
        out = uniform(out * g);
        in = uniform(in * g);
        ce = uniform(ce * g);
        kd = uniform(kd * g);
        label = uniform(label * g);
    }
};

// The gradient of one row, place by place
template <bool BF16> struct Gradient {
    static constexpr int E = Row<BF16>::E;
    Coef c;
    Exp by_tau, plain;
    float one, square;  // a place outside the record: u (one + square u), u = exp((z - ref) / tau): the label's term is a power of u at
    bool other;         // temperatures 1 and 2, elsewhere (other) an exponential of its own
    void *grad;
    bool same;  // its chunks lie as those of the logits

    __device__ __forceinline__ Gradient(const Coef &coef, const DistillArgs &p, const Row<BF16> &row, int64_t at)
        : c(coef), by_tau(p.temperature), plain(1.0f)
    {
        const float to_ref = uniform(plain(c.ref - c.max));
        one = c.out + (p.temperature == 1.0f ? c.ce * to_ref : 0.f);
        square = p.temperature == 2.0f ? c.ce * to_ref : 0.f;
        other = c.ce != 0.0f && p.temperature != 1.0f && p.temperature != 2.0f;
        grad = (char *)p.dlogits + at * p.ld_grad * (BF16 ? 2 : 4);
        same = (((uintptr_t)grad ^ (uintptr_t)row.row) & 15u) == 0;
    }
    __device__ __forceinline__ float outside(float z) const
    {
        const float u = by_tau(z - c.ref);
        const float g = u * __builtin_fmaf(square, u, one);
        return other ? __builtin_fmaf(c.ce, plain(z - c.max), g) : g;
    }
    __device__ __forceinline__ void chunk(const Row<BF16> &row, const uint4 &v, int k) const
    {
        float g[8];
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float u = by_tau(Row<BF16>::value(v, e) - c.ref);
            g[e] = u * __builtin_fmaf(square, u, one);
        }
        if (other) {  // (the same for the whole row)
#pragma unroll
            for (int e = 0; e < E; ++e) g[e] = __builtin_fmaf(c.ce, plain(Row<BF16>::value(v, e) - c.max), g[e]);
        }
        char *to = (char *)grad + row.lo * (16 / E);
        if (same) {
            ((uint4 *)to)[k] = Row<BF16>::chunk(g);
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) Elem<BF16>::store(grad, row.lo + (int64_t)k * E + e, g[e]);
        }
    }
    // behind all chunks of the row: the edges, the record's places and the label's.  edge_z: this thread's edge
    template <int THREADS> __device__ __forceinline__ void edges(const Row<BF16> &row, float edge_z) const
    {
        if ((int)threadIdx.x < row.edges) Elem<BF16>::store(grad, row.edge_index(threadIdx.x), outside(edge_z));
    }
    template <int THREADS>
    __device__ __forceinline__ void corrections(const Shared<THREADS> &sh, const DistillArgs &p, const Row<BF16> &row, int label, float label_z,
                                                bool label_in_record) const
    {
        for (int j = threadIdx.x; j < p.k; j += THREADS) {
            const int at = sh.at[j];
            if (at < 0 || !sh.first[j]) continue;
            const float z = sh.z[j];
            double g = (double)(c.in * by_tau(z - c.max)) - (double)c.kd * sh.p[j];
            if (c.ce != 0.0f) g += (double)(c.ce * plain(z - c.max)) - (at == label ? (double)c.label : 0.0);
            Elem<BF16>::store(grad, at, (float)g);
        }
        if (label >= 0 && !label_in_record && threadIdx.x == 0) Elem<BF16>::store(grad, label, outside(label_z) - c.label);
    }
};

// A row's chunks: the first SLOTS * THREADS of them held in registers (thread t has chunks t, t + THREADS, ..), read once; what is
// beyond them is read again in every pass.
template <bool BF16, int THREADS, int SLOTS> struct Held {
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
        for (int c = SLOTS * THREADS + threadIdx.x; c < row.whole; c += THREADS) {
            uint4 w = row.body[c];
            f(w, c, std::false_type());
        }
    }
    template <typename F> __device__ __forceinline__ void each(const Row<BF16> &row, F f)
    {
        each(row, f, [](int, int) {});
    }
    // (through a buffer descriptor: what is beyond the row's last whole chunk is not read, without a branch)
    __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t row, int s, int t)
    {
        v[s] = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(row, (s * THREADS + t) * 16, 0, 0));
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

// A thread's running sums: exp((z - m) / tau) and exp(z - m) over the logits it has met, m the largest of them
struct Running {
    float m = kLow, s = 0.f, ce = 0.f;
    // (to a larger reference; the label's exponential is the square of the other at temperature 2)
    __device__ __forceinline__ void raise(float to, const Exp &by_tau, const Exp &plain, bool other)
    {
        const float u = by_tau(m - to);
        s *= u;
        ce *= other ? plain(m - to) : u * u;
        m = to;
    }
    template <int N> __device__ __forceinline__ void add(const float (&z)[N], const Exp &by_tau, const Exp &plain, bool other)
    {
        float top = m;
#pragma unroll
        for (int e = 0; e < N; ++e) top = fmaxf(top, z[e]);
        raise(top, by_tau, plain, other);
        if (other) {  // (the same for the whole row)
#pragma unroll
            for (int e = 0; e < N; ++e) {
                s += by_tau(z[e] - m);
                ce += plain(z[e] - m);
            }
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float u = by_tau(z[e] - m);
                s += u;
                ce = __builtin_fmaf(u, u, ce);
            }
        }
    }
};

// A block takes rows blockIdx.x, + gridDim.x, ..: record, sums, loss, and with GRAD the gradient.  While a row's gradient is written, each
// chunk's registers take the next row's: the memory has work while the block computes, though a row of 128 Ki bf16
// leaves no registers for a second block beside it.  The first wave does the record's and the row's arithmetic in 64 bits.
template <bool BF16, int THREADS, int SLOTS, bool GRAD> __global__ void __launch_bounds__(THREADS, 4) distill_kernel(DistillArgs p)
{
    constexpr int E = Row<BF16>::E, W = THREADS / kWave;
    __shared__ Shared<THREADS> sh;
    extern __shared__ uint32_t bits[];
    const bool tail = p.t_lse != nullptr;  // the rest of the row is a term of its own
    const Exp by_tau(p.temperature), plain(1.0f);
    const int lane = threadIdx.x & (kWave - 1), wave = uniform((uint32_t)threadIdx.x / kWave);
    Held<BF16, THREADS, SLOTS> held;
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
        put_record<BF16, THREADS>(sh, bits, p, i, row, ahead.entry);
        __syncthreads();
        const int label = ahead.label;
        const float label_z = ahead.label_z, edge_z = ahead.edge_z, dloss = ahead.dloss;
        const int next = i + gridDim.x;
        const Row<BF16> next_row = row_at(next);
        load_places(next, next_row);
        const int b = label >= 0 ? row.bit(label) : 0;
        const bool label_in_record = label >= 0 && (bits[b >> 5] >> (b & 31) & 1u);
        const bool two = label >= 0 && p.temperature != 1.0f, other = two && p.temperature != 2.0f;  // a second softmax, of its own
        Teacher t;
        if (wave == 0) t = read_record<THREADS>(sh, p, i, true, two);
        Running run;
        {
            float z[1] = {edge_z};
            const int e = row.whole * E + threadIdx.x;
            if (tail && (int)threadIdx.x < row.edges && (bits[e >> 5] >> (e & 31) & 1u)) z[0] = kNegInf;
            run.add(z, by_tau, plain, other);
        }
        held.each(row, [&](uint4 &v, int k, auto) {
            if (tail) mask_chunk<BF16>(v, bits, k);
            float z[E];
#pragma unroll
            for (int e = 0; e < E; ++e) z[e] = Row<BF16>::value(v, e);
            run.add(z, by_tau, plain, other);
        });
        load_logits(next_row);
        run.raise(wave_max(run.m), by_tau, plain, other);
        const double part = wave_sum((double)run.s), part_ce = two ? wave_sum((double)run.ce) : 0.0;
        if (lane == 0) {
            sh.max[wave] = run.m;
            sh.sum[wave] = part;
            sh.sum_ce[wave] = part_ce;
        }
        __syncthreads();
        take_record_off<BF16, THREADS>(sh, bits, p, row);
        if (wave == 0) {
            // over the waves
            const double inv = 1.0 / (double)p.temperature;
            const float m = lane < W ? sh.max[lane] : kLow, rest_max = wave_max(m);
            const float u = by_tau(m - rest_max);
            const double rest = wave_sum(lane < W ? sh.sum[lane] * (double)u : 0.0);
            const double rest_ce = two ? wave_sum(lane < W ? sh.sum_ce[lane] * (double)(other ? plain(m - rest_max) : u * u) : 0.0) : 0.0;
            // relative to the row's largest logit
            const bool any = rest != 0.0;  // (NaN is something)
            const float max = t.in != 0.0 ? (any ? fmaxf(rest_max, t.ref) : t.ref) : rest_max;
            const double to_rest = any ? (double)rest_max - (double)max : 0.0, to_in = t.in != 0.0 ? (double)t.ref - (double)max : 0.0;
            const double log2e = 1.44269504088896340736;
            const double rest_scale = exp2_neg(to_rest * inv * log2e, 0);
            double sum = rest * rest_scale;
            if (tail) sum += t.in * exp2_neg(to_in * inv * log2e, 0);
            double sum_ce = sum;
            if (two) {
                sum_ce = rest_ce * exp2_neg(to_rest * log2e, 0);
                if (tail) sum_ce += t.in_ce * exp2_neg(to_in * log2e, 0);
            }
            const double r = tail && any && t.some ? t.r : 0.0, mass = t.p_sum + r, kd = (double)p.kd_weight * (double)p.temperature;
            const bool live = sum != 0.0;
            const float ce = live && label >= 0 ? (float)((double)p.ce_weight / sum_ce) : 0.f;
            const double over = 1.0 / sum;
            if (lane == 0) {
                sh.coef[0] = any ? rest_max : 0.f;
                sh.coef[1] = live && t.some ? (float)(kd * (mass * rest_scale * over - (r > 0.0 ? r / rest : 0.0))) : 0.f;
                sh.coef[2] = live ? max : 0.f;
                sh.coef[3] = live && t.some ? (float)(kd * mass * over) : 0.f;
                sh.coef[4] = ce;
                sh.coef[5] = live && t.some ? (float)kd : 0.f;
                sh.coef[6] = live && label >= 0 ? p.ce_weight : 0.f;
                sh.coef[7] = 0.f;
            }
            if (GRAD) __syncthreads();
            // (the loss itself while the other waves go on)
            double loss = 0.0;
            if (live) {
                const double log_sum = log(sum);
                if (t.some) {
                    loss = t.entropy - t.cross + t.p_sum * (log_sum - ((double)t.ref - (double)max) * inv);
                    if (r > 0.0) loss += r * (log(r) - (log(rest) + to_rest * inv - log_sum));
                    loss *= kd * (double)p.temperature;
                }
                if (label >= 0) loss += (double)p.ce_weight * (log(sum_ce) - ((double)label_z - (double)max));
            }
            if (lane == 0) p.loss[i] = (float)loss;
            if (p.stats && lane < kDistillStats) p.stats[(int64_t)i * kDistillStats + lane] = sh.coef[lane];
        } else if (GRAD) {
            __syncthreads();
        }
        const __amdgpu_buffer_rsrc_t from = next_row.buffer();
        if (GRAD) {
            Coef c(sh.coef);
            c.scale(dloss);
            const Gradient<BF16> g(c, p, row, row.n > 0 && p.r.rows ? (int64_t)__builtin_amdgcn_readfirstlane(p.r.rows[i]) : i);
            held.each(row, [&](uint4 &v, int k, auto) { g.chunk(row, v, k); }, [&](int s, int t) { held.load(from, s, t); });
            g.template edges<THREADS>(row, edge_z);
            __syncthreads();
            g.template corrections<THREADS>(sh, p, row, label, label_z, label_in_record);
        } else {
#pragma unroll
            for (int s = 0; s < SLOTS; ++s) held.load(from, s, threadIdx.x);
            __syncthreads();
        }
        if (next >= p.r.n_rows) return;
        i = next;
        row = next_row;
    }
}

// The gradient from what the forward call kept.
template <bool BF16, int THREADS> __global__ void __launch_bounds__(THREADS) distill_bwd_kernel(DistillArgs p)
{
    __shared__ Shared<THREADS> sh;
    extern __shared__ uint32_t bits[];
    const int i = blockIdx.x;
    const void *at = row_of(p.r, i);
    if (!at) return;
    const Row<BF16> row(at, p.r.vocab);
    for (int w = threadIdx.x; w < (row.n + 31) / 32; w += THREADS) bits[w] = 0;
    __syncthreads();
    Entry mine = load_place(p, i, threadIdx.x, true);
    load_logit(mine, row);
    put_record<BF16, THREADS>(sh, bits, p, i, row, mine);
    int label = p.labels ? p.labels[i] : -1;
    if (label >= row.n) label = -1;
    const float label_z = label >= 0 ? Elem<BF16>::load(at, label) : 0.f, edge_z = row.edge(threadIdx.x);
    __syncthreads();  // (every thread has read what it needs beside its chunks: the gradient may lie in the place of the logits)
    const int b = label >= 0 ? row.bit(label) : 0;
    const bool label_in_record = label >= 0 && (bits[b >> 5] >> (b & 31) & 1u);
    if (threadIdx.x < kWave) read_record<THREADS>(sh, p, i, false, false);
    Coef c(p.stats + (int64_t)i * kDistillStats);
    c.scale(p.dloss[i]);
    const Gradient<BF16> g(c, p, row, p.r.rows ? (int64_t)p.r.rows[i] : i);
    for (int k = threadIdx.x; k < row.whole; k += THREADS) g.chunk(row, row.body[k], k);
    g.template edges<THREADS>(row, edge_z);
    __syncthreads();
    g.template corrections<THREADS>(sh, p, row, label, label_z, label_in_record);
}

template <int THREADS, typename K> hipError_t launch(K kernel, int blocks, const DistillArgs &a, hipStream_t st)
{
    const size_t bytes = ((size_t)a.r.vocab + 31) / 32 * 4;  // the bitmap: up to 128 KiB
    if (bytes + sizeof(Shared<THREADS>) > (64u << 10)) {
        const hipError_t e = hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
        if (e != hipSuccess) return e;
    }
    COLLM_LAUNCH(kernel, dim3(blocks), dim3(THREADS), bytes, st, a);
    return hipGetLastError();
}

template <bool BF16, int THREADS, int SLOTS, bool GRAD> hipError_t launch_held(const DistillArgs &a, hipStream_t st)
{
    const int fit = a.compute_units * (1024 / THREADS);  // blocks at a time, by their registers
    return launch<THREADS>(distill_kernel<BF16, THREADS, SLOTS, GRAD>, a.r.n_rows < fit ? a.r.n_rows : fit, a, st);
}

// The block that holds a row in registers: the smallest that does; from 1024 threads with 20 chunks each on, the rest of a row is read again.
template <bool BF16, bool GRAD> hipError_t launch_rows(const DistillArgs &a, hipStream_t st)
{
    const int chunks = a.r.vocab / Row<BF16>::E;
    if (chunks <= 256 * 16) return launch_held<BF16, 256, 16, GRAD>(a, st);
    if (chunks <= 512 * 16) return launch_held<BF16, 512, 16, GRAD>(a, st);
    if (chunks <= 1024 * 16) return launch_held<BF16, 1024, 16, GRAD>(a, st);
    return launch_held<BF16, 1024, 20, GRAD>(a, st);
}

}  // namespace

hipError_t launch_distill_fwd(const DistillArgs &a, hipStream_t st)
{
    return a.r.bf16 ? launch_rows<true, false>(a, st) : launch_rows<false, false>(a, st);
}
hipError_t launch_distill_bwd(const DistillArgs &a, hipStream_t st)
{
    return a.r.bf16 ? launch<512>(distill_bwd_kernel<true, 512>, a.r.n_rows, a, st) : launch<512>(distill_bwd_kernel<false, 512>, a.r.n_rows, a, st);
}
hipError_t launch_distill_fwd_bwd(const DistillArgs &a, hipStream_t st)
{
    return a.r.bf16 ? launch_rows<true, true>(a, st) : launch_rows<false, true>(a, st);
}

}  // namespace collm
