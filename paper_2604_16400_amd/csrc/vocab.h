// Argument blocks and launchers of the vocabulary operators (kernels_sample.hip, kernels_distill.hip).  take(first, n) leaves `n` rows of a call, from row
// `first` on.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace collm {

constexpr int kMaxVocab = 1 << 20;  // columns of a row of logits (a bitmap of a row fits the LDS; fixed-point sums have 20 bits to grow)
constexpr int kMaxTop = 1024;       // entries of a teacher's record
constexpr int kDistillStats = 8;    // floats that a forward call keeps of a row for the backward call
constexpr float kLeastTemperature = 0x1p-127f;  // of a call: log2(e) over it is a number of 32 bits
constexpr int kLaunchRows = 1 << 21;  // rows of one launch at most: a block of up to 1024 threads each, and a grid has fewer than 2^32
static_assert((int64_t)kLaunchRows * 1024 < (int64_t)1 << 32, "threads of a grid");

// The rows of one call: row i of the call is row (rows ? rows[i] : i) of the logits; an entry of `rows` outside
// [0, n_held) is a row that is not there
struct LogitRows {
    const void *logits;
    int64_t ld;
    const int32_t *rows;
    int n_rows, n_held, vocab;
    bool bf16;
    void take(int first, int n)
    {
        n_rows = n;
        if (rows) {
            rows += first;
        } else {
            logits = (const char *)logits + first * ld * (bf16 ? 2 : 4);
            n_held -= first;
        }
    }
};

// past the entries of `rows` rows, `width` each, of an array (NULL: there is none)
template <typename T> void skip(T *&p, int64_t rows, int64_t width = 1)
{
    if (p) p += rows * width;
}

struct SampleArgs {
    LogitRows r;
    const float *u, *temperature;  // temperature NULL: 1
    const int32_t *top_k;          // NULL: off
    const float *top_p, *min_p;    // NULL: off
    int32_t *token;
    float *logprob;                // optional
    int compute_units;             // of the GPU
    void take(int first, int n)
    {
        r.take(first, n);
        skip(u, first), skip(temperature, first), skip(top_k, first), skip(top_p, first), skip(min_p, first), skip(token, first), skip(logprob, first);
    }
};

struct TopArgs {
    LogitRows r;
    int k;
    float temperature;
    float *values;     // [n_rows, k]
    int32_t *indices;  // [n_rows, k]
    float *lse;        // optional
    void take(int first, int n)
    {
        r.take(first, n);
        skip(values, first, k), skip(indices, first, k), skip(lse, first);
    }
};

struct DistillArgs {
    LogitRows r;
    int k;
    const float *t_values;    // [n_rows, k]
    const int32_t *t_indices;
    const float *t_lse;       // [n_rows] or NULL: the record's probabilities sum to one
    const int32_t *labels;    // [n_rows] or NULL
    float temperature, kd_weight, ce_weight;
    float *loss;              // forward
    float *stats;             // forward: written if not NULL; backward alone: read
    const float *dloss;       // gradient
    void *dlogits;
    int64_t ld_grad;
    int compute_units;        // of the GPU
    void *workspace;          // of the call that does both
    int64_t workspace_bytes;
    void take(int first, int n)
    {
        r.take(first, n);
        skip(t_values, first, k), skip(t_indices, first, k), skip(t_lse, first), skip(labels, first);
        skip(loss, first), skip(stats, first, kDistillStats), skip(dloss, first);
        if (dlogits && !r.rows) dlogits = (char *)dlogits + first * ld_grad * (r.bf16 ? 2 : 4);
    }
};

hipError_t launch_sample(const SampleArgs &a, hipStream_t st);
hipError_t launch_top_logits(const TopArgs &a, hipStream_t st);
hipError_t launch_distill_fwd(const DistillArgs &a, hipStream_t st);
hipError_t launch_distill_bwd(const DistillArgs &a, hipStream_t st);
hipError_t launch_distill_fwd_bwd(const DistillArgs &a, hipStream_t st);

}  // namespace collm
