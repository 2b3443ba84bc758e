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
// largest logit: 1 - sum q would lose it where the record holds nearly all of the mass.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernels.h"
#include "vocab_device.h"

namespace collm {

namespace {

using namespace vocab;

// exp(d / tau) for d <= 0.  log2(e) / tau comes in two parts, so that its rounding is not in every term of a sum; both are
// positive, so that d = -inf gives 0.
struct Exp {
    float hi, lo;
    __device__ __forceinline__ explicit Exp(float tau)
    {
        const double c = 1.44269504088896340736 / (double)tau;
        hi = (float)c;
        if ((double)hi >= c) hi = __uint_as_float(__float_as_uint(hi) - 1);
        lo = fmaxf((float)(c - (double)hi), 1e-37f);
    }
    __device__ __forceinline__ float operator()(float d) const { return __builtin_amdgcn_exp2f(__builtin_fmaf(d, hi, d * lo)); }
};

template <int THREADS> struct Record {
    double red[THREADS / kWave];
    double p[kMaxTop];      // probabilities; of a place named twice, their sum at its first entry
    float z[kMaxTop];       // the student's logits
    int32_t at[kMaxTop];    // places; -1: not an entry
    uint8_t first[kMaxTop]; // whether the entry is its place's first
};

// What a row's coefficients and corrections need of its record
struct Teacher {
    double p_sum, entropy;  // sum p, sum p log p
    double r;               // mass outside the record (before the student's rest is looked at)
    bool some;              // whether there is a valid entry
};

// Reads row i's record: probabilities, the student's logits at its places, and the bitmap of its places (`bits`: one bit an element of the
// row's chunks, cleared here).
template <bool BF16, int THREADS>
__device__ Teacher read_record(Record<THREADS> &rec, uint32_t *bits, const DistillArgs &p, int i, const Row<BF16> &row)
{
    const float *t = p.t_values + (int64_t)i * p.k;
    const int32_t *at = p.t_indices + (int64_t)i * p.k;
    for (int w = threadIdx.x; w < (row.n + row.head + 31) / 32; w += THREADS) bits[w] = 0;
    float top = kNegInf;
    for (int j = threadIdx.x; j < p.k; j += THREADS) {
        const int v = at[j];
        const bool valid = v >= 0 && v < row.n && t[j] > kNegInf;
        rec.at[j] = valid ? v : -1;
        rec.z[j] = valid ? Elem<BF16>::load(row.row, v) : 0.f;
        if (valid) top = fmaxf(top, t[j]);
    }
    Teacher out;
    top = block_max<THREADS>(top, rec.red);
    out.some = top > kNegInf;
    const double inv = 1.0 / (double)p.temperature;
    // logarithm of the sum that p divides by, relative to `ref`
    double ref = 0.0, log_sum = 0.0;
    if (p.t_lse) {
        log_sum = (double)p.t_lse[i];
    } else {
        ref = out.some ? (double)top : 0.0;
        double part = 0.0;
        for (int j = threadIdx.x; j < p.k; j += THREADS)
            if (rec.at[j] >= 0) part += exp(((double)t[j] - ref) * inv);
        log_sum = log(block_sum<THREADS>(part, rec.red));
    }
    double sum = 0.0, entropy = 0.0;
    for (int j = threadIdx.x; j < p.k; j += THREADS) {
        double q = 0.0;
        bool first = false;
        if (rec.at[j] >= 0) {
            const double log_p = ((double)t[j] - ref) * inv - log_sum;
            q = exp(log_p);
            if (q > 0.0) entropy += q * log_p;
            const int b = rec.at[j] + row.head;
            first = !(atomicOr(&bits[b >> 5], 1u << (b & 31)) >> (b & 31) & 1u);
        }
        sum += q;
        rec.p[j] = q;
        rec.first[j] = first;
    }
    out.p_sum = block_sum<THREADS>(sum, rec.red);
    out.entropy = block_sum<THREADS>(entropy, rec.red);
    out.r = p.t_lse ? fmax(0.0, 1.0 - out.p_sum) : 0.0;
    return out;
}

// What the gradient of a row is made of, for dloss = 1:
//   outside the record  out * exp((z - ref) / tau) + ce * exp(z - max)
//   in the record       in * exp((z - max) / tau) + ce * exp(z - max) - kd * p
//   at the label        - label, in addition
struct Coef {
    float ref, out, max, in, ce, kd, label;
    __device__ __forceinline__ void scale(float g)
    {
        out *= g;
        in *= g;
        ce *= g;
        kd *= g;
        label *= g;
    }
};

// Writes the gradient of chunks lo .. hi of a row: every place as one outside the record, then the record's and the label's.
template <bool BF16, int THREADS>
__device__ void write_gradient(const Record<THREADS> &rec, const uint32_t *bits, const DistillArgs &p, const Row<BF16> &row, void *grad, const Coef &c,
                               int label, int lo, int hi)
{
    constexpr int E = Row<BF16>::E;
    const Exp by_tau(p.temperature), plain(1.0f);
    const bool same = (((uintptr_t)grad ^ (uintptr_t)row.row) & 15u) == 0;
    uint4 *to = (uint4 *)((uintptr_t)grad & ~(uintptr_t)15);
    auto outside = [&](float z) { return c.out * by_tau(z - c.ref) + (c.ce != 0.0f ? c.ce * plain(z - c.max) : 0.0f); };
    const int first = lo * E - row.head, end = hi * E - row.head;  // the places written here
    const bool has_label = label >= first && label < end && label >= 0 && label < row.n;
    const float label_z = has_label ? Elem<BF16>::load(row.row, label) : 0.f;
    __syncthreads();  // (the gradient may lie in the place of the logits)
    for (int k = lo + threadIdx.x; k < hi; k += THREADS) {
        const uint4 v = row.load(k);
        float g[8];
#pragma unroll
        for (int e = 0; e < E; ++e) g[e] = outside(Row<BF16>::value(v, e));
        if (same && row.whole(k)) {
            to[k] = BF16 ? make_uint4(pack_bf16(g[0], g[1]), pack_bf16(g[2], g[3]), pack_bf16(g[4], g[5]), pack_bf16(g[6], g[7]))
                         : make_uint4(__float_as_uint(g[0]), __float_as_uint(g[1]), __float_as_uint(g[2]), __float_as_uint(g[3]));
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int at = k * E - row.head + e;
                if (at >= 0 && at < row.n) Elem<BF16>::store(grad, at, g[e]);
            }
        }
    }
    __syncthreads();
    for (int j = threadIdx.x; j < p.k; j += THREADS) {
        const int at = rec.at[j];
        if (at < first || at >= end || !rec.first[j]) continue;
        double q = 0.0;
        for (int l = 0; l < p.k; ++l)
            if (rec.at[l] == at) q += rec.p[l];
        const float z = rec.z[j];
        double g = (double)(c.in * by_tau(z - c.max)) - (double)c.kd * q;
        if (c.ce != 0.0f) g += (double)(c.ce * plain(z - c.max)) - (at == label ? (double)c.label : 0.0);
        Elem<BF16>::store(grad, at, (float)g);
    }
    const int b = label + row.head;
    if (has_label && threadIdx.x == 0 && !(bits[b >> 5] >> (b & 31) & 1u))
        Elem<BF16>::store(grad, label, outside(label_z) - c.label);
}

// One block a row: record, largest logits, sums, loss, and with GRAD the gradient.
template <bool BF16, int THREADS, bool GRAD> __global__ void __launch_bounds__(THREADS) distill_kernel(DistillArgs p)
{
    constexpr int E = Row<BF16>::E;
    __shared__ Record<THREADS> rec;
    extern __shared__ uint32_t bits[];
    const int i = blockIdx.x;
    const void *at = row_of(p.r, i);
    Coef c = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    float loss = 0.f;
    if (at) {
        const Row<BF16> row(at, p.r.vocab);
        const Teacher t = read_record<BF16, THREADS>(rec, bits, p, i, row);
        const int label = p.labels && p.labels[i] >= 0 && p.labels[i] < row.n ? p.labels[i] : -1;
        const bool tail = p.t_lse != nullptr;  // the rest of the row is a term of its own
        const bool two = label >= 0 && p.temperature != 1.0f && p.ce_weight != 0.0f;  // softmaxes
        auto outside = [&](int k) { return tail ? ~((bits[k * E >> 5] >> (k * E & 31))) : 0xffffffffu; };
        float rest_max = kNegInf, max = kNegInf;
        for (int k = threadIdx.x; k < row.chunks; k += THREADS) {
            const uint4 v = row.load(k);
            const uint32_t o = outside(k);
#pragma unroll
            for (int e = 0; e < E; ++e) rest_max = fmaxf(rest_max, (o >> e & 1u) ? Row<BF16>::value(v, e) : kNegInf);
        }
        max = rest_max;
        for (int j = threadIdx.x; j < p.k; j += THREADS)
            if (rec.at[j] >= 0) max = fmaxf(max, rec.z[j]);
        rest_max = block_max<THREADS>(rest_max, rec.red);
        max = block_max<THREADS>(max, rec.red);
        c.ref = rest_max > kNegInf ? rest_max : 0.f;
        c.max = max > kNegInf ? max : 0.f;
        const Exp by_tau(p.temperature), plain(1.0f);
        float part = 0.f, part_ce = 0.f;
        for (int k = threadIdx.x; k < row.chunks; k += THREADS) {
            const uint4 v = row.load(k);
            const uint32_t o = outside(k);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float z = Row<BF16>::value(v, e);
                part += (o >> e & 1u) ? by_tau(z - c.ref) : 0.f;
                if (two) part_ce += plain(z - c.max);
            }
        }
        const double inv = 1.0 / (double)p.temperature;
        const double rest = block_sum<THREADS>((double)part, rec.red);
        double in_part = 0.0, cross = 0.0;
        for (int j = threadIdx.x; j < p.k; j += THREADS) {
            if (rec.at[j] < 0) continue;
            const double d = ((double)rec.z[j] - (double)c.max) * inv;
            if (tail && rec.first[j]) in_part += exp(d);
            if (rec.p[j] > 0.0) cross += rec.p[j] * d;
        }
        const double shift = ((double)c.ref - (double)c.max) * inv;
        double sum = block_sum<THREADS>(in_part, rec.red);
        if (rest_max > kNegInf || rest != 0.0) sum += rest * exp(shift);
        cross = block_sum<THREADS>(cross, rec.red);
        const double sum_ce = two ? block_sum<THREADS>((double)part_ce, rec.red) : sum;
        if (sum != 0.0) {
            double value = 0.0;
            if (t.some) {
                const double r = tail && rest != 0.0 ? t.r : 0.0;
                const double mass = t.p_sum + r, kd = (double)p.kd_weight * p.temperature;
                value = t.entropy - cross + t.p_sum * log(sum);
                if (r > 0.0) value += r * (log(r) - (log(rest) + shift - log(sum)));
                value *= kd * p.temperature;
                c.in = (float)(kd * mass / sum);
                c.out = (float)(kd * (mass * exp(shift) / sum - (r > 0.0 ? r / rest : 0.0)));
                c.kd = (float)kd;
            }
            if (label >= 0) {
                value += (double)p.ce_weight * (log(sum_ce) - ((double)Elem<BF16>::load(at, label) - (double)c.max));
                c.ce = (float)((double)p.ce_weight / sum_ce);
                c.label = p.ce_weight;
            }
            loss = (float)value;
        }
        if (GRAD) {
            c.scale(p.dloss[i]);
            const int64_t to = p.r.rows ? (int64_t)p.r.rows[i] : i;
            void *grad = (char *)p.dlogits + to * p.ld_grad * (BF16 ? 2 : 4);
            write_gradient<BF16, THREADS>(rec, bits, p, row, grad, c, label, 0, row.chunks);
        }
    }
    if (threadIdx.x == 0) {
        if (p.loss) p.loss[i] = loss;
        if (p.stats) {
            float *s = p.stats + (int64_t)i * kDistillStats;
            s[0] = c.ref;
            s[1] = c.out;
            s[2] = c.max;
            s[3] = c.in;
            s[4] = c.ce;
            s[5] = c.kd;
            s[6] = c.label;
            s[7] = 0.f;
        }
    }
}

// The gradient from what the forward call kept.
template <bool BF16, int THREADS> __global__ void __launch_bounds__(THREADS) distill_bwd_kernel(DistillArgs p)
{
    __shared__ Record<THREADS> rec;
    extern __shared__ uint32_t bits[];
    const int i = blockIdx.x;
    const void *at = row_of(p.r, i);
    if (!at) return;
    const Row<BF16> row(at, p.r.vocab);
    read_record<BF16, THREADS>(rec, bits, p, i, row);
    const float *s = p.stats + (int64_t)i * kDistillStats;
    Coef c = {s[0], s[1], s[2], s[3], s[4], s[5], s[6]};
    c.scale(p.dloss[i]);
    const int64_t to = p.r.rows ? (int64_t)p.r.rows[i] : i;
    void *grad = (char *)p.dlogits + to * p.ld_grad * (BF16 ? 2 : 4);
    write_gradient<BF16, THREADS>(rec, bits, p, row, grad, c, p.labels ? p.labels[i] : -1, 0, row.chunks);
}

template <typename K> hipError_t launch(K kernel, int threads, const DistillArgs &a, hipStream_t st)
{
    const size_t bytes = ((size_t)a.r.vocab + 8 + 31) / 32 * 4;  // the bitmap: up to 128 KiB
    if (bytes > (64u << 10) - sizeof(Record<512>)) {
        const hipError_t e = hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
        if (e != hipSuccess) return e;
    }
    COLLM_LAUNCH(kernel, dim3(a.r.n_rows), dim3(threads), bytes, st, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_distill_fwd(const DistillArgs &a, hipStream_t st)
{
    return a.r.bf16 ? launch(distill_kernel<true, 512, false>, 512, a, st) : launch(distill_kernel<false, 512, false>, 512, a, st);
}
hipError_t launch_distill_bwd(const DistillArgs &a, hipStream_t st)
{
    return a.r.bf16 ? launch(distill_bwd_kernel<true, 512>, 512, a, st) : launch(distill_bwd_kernel<false, 512>, 512, a, st);
}
hipError_t launch_distill_fwd_bwd(const DistillArgs &a, hipStream_t st)
{
    return a.r.bf16 ? launch(distill_kernel<true, 512, true>, 512, a, st) : launch(distill_kernel<false, 512, true>, 512, a, st);
}

}  // namespace collm
