// The C boundary of the losses on logits: argument checks, then the kernels' launches.
#include <cfloat>
#include <cmath>
#include "zf_ops_check.h"

using namespace zf;

namespace {

int check_rows(const zf_loss_rows &r) {
    if (r.dtype != 0 && r.dtype != 1) return refuse("dtype must be 0 (fp32) or 1 (bf16)");
    if (r.V < 1 || r.V > VOCAB_MAX) return refuse("V must be 1..2^24");
    if (r.rows < 0 || r.rows > INT32_MAX) return refuse("rows must be 0..2^31-1");
    if (r.row_stride_elems < r.V) return refuse("the row stride is smaller than V");
    if (!(r.temperature >= FLT_MIN && r.temperature <= FLT_MAX)) return refuse("temperature must be finite, at least 2^-126");   // (its reciprocal is finite)
    if (!r.loss) return refuse("null argument");
    if (r.rows && !r.logits) return refuse("null argument");
    if (!element_aligned(r.logits, r.dtype)) return refuse("the logits are not aligned to an element");
    return ZF_OK;
}
int check_grad(const zf_loss_rows &r, const void *d_grad, int64_t stride, bool needed) {
    if (!d_grad) return needed && r.rows ? refuse("null argument") : ZF_OK;
    if (!element_aligned(d_grad, r.dtype)) return refuse("the gradient is not aligned to an element");
    if (stride < r.V) return refuse("the gradient's row stride is smaller than V");
    if (d_grad == r.logits) return refuse("the gradient may not be the logits");
    return ZF_OK;
}
bool is_id(int32_t bytes) { return bytes == 4 || bytes == 8; }

int check(const zf_distill_args *a) {
    if (!a) return refuse("null argument");
    if (const int rc = check_rows(a->r)) return rc;
    if (a->n_listed < 1 || a->n_listed > TEACHER_MAX) return refuse("n_listed must be 1..1024");
    if (!is_id(a->id_bytes)) return refuse("id_bytes must be 4 or 8");
    if (a->values_dtype != 0 && a->values_dtype != 1) return refuse("values_dtype must be 0 (fp32) or 1 (bf16)");
    if (a->r.rows && (!a->ids || !a->values || !a->r.losses)) return refuse("null argument");
    return ZF_OK;
}
int check(const zf_policy_args *a) {
    if (!a) return refuse("null argument");
    if (const int rc = check_rows(a->r)) return rc;
    if (!is_id(a->token_bytes)) return refuse("token_bytes must be 4 or 8");
    if (!(a->clip_low >= 0.0) || !(a->clip_high >= 0.0)) return refuse("clip_low and clip_high must not be negative");
    if (!std::isfinite(a->kl_weight) || !std::isfinite(a->entropy_weight)) return refuse("kl_weight and entropy_weight must be finite");
    if (a->r.rows && (!a->tokens || !a->old_logprobs || !a->advantages || !a->logprobs || !a->r.losses)) return refuse("null argument");
    return ZF_OK;
}
int check(const zf_preference_args *a) {
    if (!a) return refuse("null argument");
    if (const int rc = check_rows(a->r)) return rc;
    if (!is_id(a->token_bytes) || !is_id(a->offset_bytes)) return refuse("token_bytes and offset_bytes must be 4 or 8");
    if (a->pairs < 0 || a->pairs > INT32_MAX / 2) return refuse("pairs must be 0..2^30-1");
    if (!std::isfinite(a->beta)) return refuse("beta must be finite");
    if (!(a->label_smoothing >= 0.0 && a->label_smoothing <= 1.0)) return refuse("label_smoothing must be 0..1");
    if (a->r.rows && (!a->tokens || !a->stats)) return refuse("null argument");
    if ((uintptr_t)a->stats % 16) return refuse("stats must be aligned to 16 bytes");
    if (preference_blocks(*a) > BLOCKS_MAX) return refuse("more logits than a call takes: split the rows");
    if (!a->offsets || (a->pairs && (!a->r.losses || !a->chosen || !a->rejected || !a->slopes))) return refuse("null argument");
    return ZF_OK;
}

template <class ArgsT, class Launch>
int forward(const ArgsT *a, void *d_grad, int64_t stride, int32_t device, Launch launch) {
    return guarded([&]() -> int {
        if (const int rc = check(a)) return rc;
        if (const int rc = check_grad(a->r, d_grad, stride, false)) return rc;
        return on_device(device, [&]() { return launch(LossGrad{d_grad, stride, nullptr, 0}); });
    });
}
template <class ArgsT, class Launch>
int backward(const ArgsT *a, const float *d_g, int32_t held, void *d_grad, int64_t stride, int32_t device, Launch launch) {
    return guarded([&]() -> int {
        if (const int rc = check(a)) return rc;
        if (const int rc = check_grad(a->r, d_grad, stride, true)) return rc;
        if (!d_g) return refuse("null argument");
        if (a->r.rows == 0) return ZF_OK;
        return on_device(device, [&]() { return launch(LossGrad{d_grad, stride, d_g, held}); });
    });
}

}  // namespace

extern "C" {

int zf_distill_loss(const zf_distill_args *a, void *d_grad, int64_t stride, int32_t device, void *hip_stream) {
    return forward(a, d_grad, stride, device, [&](const LossGrad &g) { return launch_distill(*a, g, (hipStream_t)hip_stream); });
}
int zf_distill_loss_backward(const zf_distill_args *a, const float *d_g, int32_t held, void *d_grad, int64_t stride, int32_t device, void *hip_stream) {
    return backward(a, d_g, held, d_grad, stride, device, [&](const LossGrad &g) { return launch_distill(*a, g, (hipStream_t)hip_stream); });
}
int zf_policy_loss(const zf_policy_args *a, void *d_grad, int64_t stride, int32_t device, void *hip_stream) {
    return forward(a, d_grad, stride, device, [&](const LossGrad &g) { return launch_policy(*a, g, (hipStream_t)hip_stream); });
}
int zf_policy_loss_backward(const zf_policy_args *a, const float *d_g, int32_t held, void *d_grad, int64_t stride, int32_t device, void *hip_stream) {
    return backward(a, d_g, held, d_grad, stride, device, [&](const LossGrad &g) { return launch_policy(*a, g, (hipStream_t)hip_stream); });
}
int zf_preference_loss(const zf_preference_args *a, int32_t device, void *hip_stream) {
    return forward(a, nullptr, 0, device, [&](const LossGrad &) { return launch_preference(*a, (hipStream_t)hip_stream); });
}
int zf_preference_loss_backward(const zf_preference_args *a, const float *d_g, void *d_grad, int64_t stride, int32_t device, void *hip_stream) {
    return backward(a, d_g, 0, d_grad, stride, device, [&](const LossGrad &g) { return launch_preference_backward(*a, g, (hipStream_t)hip_stream); });
}

}  // extern "C"
