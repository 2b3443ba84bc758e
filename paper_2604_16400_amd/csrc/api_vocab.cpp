// C ABI of the vocabulary operators: validation and launches.
#include <hip/hip_runtime.h>

#include <cmath>

#include "collm_lora.h"
#include "status.h"
#include "vocab.h"

using namespace collm;

namespace {

inline bool aligned(const void *p, unsigned n) { return ((uintptr_t)p & (n - 1)) == 0; }
inline int elem_bytes(const collm_logits *s) { return s->dtype == COLLM_BF16 ? 2 : 4; }

inline bool temperature_ok(float t) { return t >= kLeastTemperature && std::isfinite(t); }

// Everything that a call's rows can be refused for.  COLLM_OK with s->n_rows == 0: nothing to do.
int check_rows(const collm_logits *s, const void *logits, LogitRows &r)
{
    if (!s) return COLLM_E_NULL;
    if (s->dtype != COLLM_F32 && s->dtype != COLLM_BF16) return COLLM_E_DTYPE;
    if (s->n_rows < 0 || s->n_held < 0 || s->vocab < 1 || s->vocab > kMaxVocab || s->ld < s->vocab) return COLLM_E_SHAPE;
    if (!s->rows && s->n_rows > s->n_held) return COLLM_E_SHAPE;
    if (s->n_held > 1 && s->ld > (INT64_MAX / 8) / s->n_held) return COLLM_E_SHAPE;
    if (s->n_rows == 0) return COLLM_OK;
    if (!logits && s->n_held > 0) return COLLM_E_NULL;  // (of no held row there is no memory: the call's rows are not there)
    if (!aligned(logits, elem_bytes(s)) || !aligned(s->rows, 4)) return COLLM_E_ALIGN;
    r.logits = logits;
    r.ld = s->ld;
    r.rows = s->rows;
    r.n_rows = s->n_rows;
    r.n_held = s->n_held;
    r.vocab = s->vocab;
    r.bf16 = s->dtype == COLLM_BF16;
    return COLLM_OK;
}

int check_workspace(const void *workspace, int64_t bytes)
{
    if (bytes < 0) return COLLM_E_SHAPE;
    if (bytes > 0 && !workspace) return COLLM_E_NULL;
    return aligned(workspace, 16) ? COLLM_OK : COLLM_E_ALIGN;
}

int check_distill(const collm_logits *s, const void *logits, const collm_distill *d, DistillArgs &a)
{
    const int rc = check_rows(s, logits, a.r);
    if (rc != COLLM_OK) return rc;
    if (!d) return COLLM_E_NULL;
    if (d->k < 1 || d->k > kMaxTop || !temperature_ok(d->temperature)) return COLLM_E_SHAPE;
    if (!std::isfinite(d->kd_weight) || !std::isfinite(d->ce_weight)) return COLLM_E_SHAPE;
    if (s->n_rows == 0) return COLLM_OK;
    if (!d->values || !d->indices) return COLLM_E_NULL;
    if (!aligned(d->values, 4) || !aligned(d->indices, 4) || !aligned(d->lse, 4) || !aligned(d->labels, 4)) return COLLM_E_ALIGN;
    a.k = d->k;
    a.t_values = d->values;
    a.t_indices = d->indices;
    a.t_lse = d->lse;
    a.labels = d->labels;
    a.temperature = d->temperature;
    a.kd_weight = d->kd_weight;
    a.ce_weight = d->ce_weight;
    return COLLM_OK;
}

// the gradient's rows lie apart from the logits, or are the logits' own
int check_grad(const collm_logits *s, const void *logits, const float *dloss, const void *dlogits, int64_t ld_grad)
{
    if (ld_grad < s->vocab || (s->n_held > 1 && ld_grad > (INT64_MAX / 8) / s->n_held)) return COLLM_E_SHAPE;
    if (s->n_rows == 0) return COLLM_OK;
    if (!dloss || (!dlogits && s->n_held > 0)) return COLLM_E_NULL;
    if (!aligned(dloss, 4) || !aligned(dlogits, elem_bytes(s))) return COLLM_E_ALIGN;
    if (s->n_held == 0) return COLLM_OK;
    const uintptr_t z = (uintptr_t)logits, g = (uintptr_t)dlogits;
    const uint64_t z_bytes = ((uint64_t)(s->n_held - 1) * s->ld + s->vocab) * elem_bytes(s);
    const uint64_t g_bytes = ((uint64_t)(s->n_held - 1) * ld_grad + s->vocab) * elem_bytes(s);
    const bool apart = z + z_bytes <= g || g + g_bytes <= z;
    return apart || (z == g && s->ld == ld_grad) ? COLLM_OK : COLLM_E_SHAPE;
}

// the call's rows, as many at a time as a launch takes
template <typename Args> int launch_rows(const Args &a, hipError_t (*launch)(const Args &, hipStream_t), void *stream)
{
    for (int64_t first = 0; first < a.r.n_rows; first += kLaunchRows) {
        const int64_t left = a.r.n_rows - first;
        Args part = a;
        part.take((int)first, (int)(left < kLaunchRows ? left : kLaunchRows));
        HIP_TRY(launch(part, (hipStream_t)stream));
    }
    return COLLM_OK;
}

}  // namespace

extern "C" {

int collm_sample(int device, const collm_logits *shape, const void *logits, const float *u, const collm_sampling *params, int32_t *token,
                 float *logprob, void *workspace, int64_t workspace_bytes, void *stream)
{
    SampleArgs a{};
    int rc = check_rows(shape, logits, a.r);
    if (rc == COLLM_OK) rc = check_workspace(workspace, workspace_bytes);
    if (rc != COLLM_OK || shape->n_rows == 0) return rc;
    if (!u || !token) return COLLM_E_NULL;
    if (!aligned(u, 4) || !aligned(token, 4) || !aligned(logprob, 4)) return COLLM_E_ALIGN;
    a.u = u;
    if (params) {
        if (!aligned(params->temperature, 4) || !aligned(params->top_k, 4) || !aligned(params->top_p, 4) || !aligned(params->min_p, 4))
            return COLLM_E_ALIGN;
        a.temperature = params->temperature;
        a.top_k = params->top_k;
        a.top_p = params->top_p;
        a.min_p = params->min_p;
    }
    a.token = token;
    a.logprob = logprob;
    HIP_TRY(hipSetDevice(device));
    HIP_TRY(hipDeviceGetAttribute(&a.compute_units, hipDeviceAttributeMultiprocessorCount, device));
    return launch_rows(a, launch_sample, stream);
}

int collm_top_logits(int device, const collm_logits *shape, const void *logits, int32_t k, float temperature, float *values, int32_t *indices,
                     float *lse, void *workspace, int64_t workspace_bytes, void *stream)
{
    TopArgs a{};
    int rc = check_rows(shape, logits, a.r);
    if (rc == COLLM_OK) rc = check_workspace(workspace, workspace_bytes);
    if (rc != COLLM_OK) return rc;
    if (k < 1 || k > kMaxTop || !temperature_ok(temperature)) return COLLM_E_SHAPE;
    if (shape->n_rows == 0) return COLLM_OK;
    if (!values || !indices) return COLLM_E_NULL;
    if (!aligned(values, 4) || !aligned(indices, 4) || !aligned(lse, 4)) return COLLM_E_ALIGN;
    a.k = k;
    a.temperature = temperature;
    a.values = values;
    a.indices = indices;
    a.lse = lse;
    HIP_TRY(hipSetDevice(device));
    return launch_rows(a, launch_top_logits, stream);
}

int collm_distill_fwd(int device, const collm_logits *shape, const void *logits, const collm_distill *teacher, float *loss, float *stats,
                      void *workspace, int64_t workspace_bytes, void *stream)
{
    DistillArgs a{};
    int rc = check_distill(shape, logits, teacher, a);
    if (rc == COLLM_OK) rc = check_workspace(workspace, workspace_bytes);
    if (rc != COLLM_OK || shape->n_rows == 0) return rc;
    if (!loss) return COLLM_E_NULL;
    if (!aligned(loss, 4) || !aligned(stats, 4)) return COLLM_E_ALIGN;
    a.loss = loss;
    a.stats = stats;
    HIP_TRY(hipSetDevice(device));
    HIP_TRY(hipDeviceGetAttribute(&a.compute_units, hipDeviceAttributeMultiprocessorCount, device));
    return launch_rows(a, launch_distill_fwd, stream);
}

int collm_distill_bwd(int device, const collm_logits *shape, const void *logits, const collm_distill *teacher, const float *stats, const float *dloss,
                      void *dlogits, int64_t ld_grad, void *stream)
{
    DistillArgs a{};
    int rc = check_distill(shape, logits, teacher, a);
    if (rc == COLLM_OK) rc = check_grad(shape, logits, dloss, dlogits, ld_grad);
    if (rc != COLLM_OK || shape->n_rows == 0) return rc;
    if (!stats) return COLLM_E_NULL;
    if (!aligned(stats, 4)) return COLLM_E_ALIGN;
    a.stats = const_cast<float *>(stats);  // (read only)
    a.dloss = dloss;
    a.dlogits = dlogits;
    a.ld_grad = ld_grad;
    HIP_TRY(hipSetDevice(device));
    HIP_TRY(hipDeviceGetAttribute(&a.compute_units, hipDeviceAttributeMultiprocessorCount, device));
    return launch_rows(a, launch_distill_bwd, stream);
}

int collm_distill_fwd_bwd(int device, const collm_logits *shape, const void *logits, const collm_distill *teacher, const float *dloss, float *loss,
                          void *dlogits, int64_t ld_grad, void *workspace, int64_t workspace_bytes, void *stream)
{
    DistillArgs a{};
    int rc = check_distill(shape, logits, teacher, a);
    if (rc == COLLM_OK) rc = check_grad(shape, logits, dloss, dlogits, ld_grad);
    if (rc == COLLM_OK) rc = check_workspace(workspace, workspace_bytes);
    if (rc != COLLM_OK || shape->n_rows == 0) return rc;
    if (!loss) return COLLM_E_NULL;
    if (!aligned(loss, 4)) return COLLM_E_ALIGN;
    a.loss = loss;
    a.dloss = dloss;
    a.dlogits = dlogits;
    a.ld_grad = ld_grad;
    a.workspace = workspace;
    a.workspace_bytes = workspace_bytes;
    HIP_TRY(hipSetDevice(device));
    HIP_TRY(hipDeviceGetAttribute(&a.compute_units, hipDeviceAttributeMultiprocessorCount, device));
    return launch_rows(a, launch_distill_fwd_bwd, stream);
}

}  // extern "C"
