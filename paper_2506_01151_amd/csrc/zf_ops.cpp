// The C boundary of the calls at the two ends of a step's logits: argument checks, then the kernels' launches.
#include <cfloat>
#include <cmath>
#include <new>
#include <string>
#include "zf_internal.h"
#include "zf_ops.h"

using namespace zf;

namespace {

int refuse(const char *why) { set_error(why); return ZF_ERR_INVALID_ARG; }
template <class F>
int on_device(int32_t device, F launch) {     // launches on `device`, and leaves the thread's current device as it was
    int before = -1;
    hipError_t e = hipGetDevice(&before);
    const bool other = e == hipSuccess && before != device;
    if (e == hipSuccess && other) e = hipSetDevice(device);
    if (e == hipSuccess) {
        e = launch();
        if (other) { const hipError_t back = hipSetDevice(before); if (e == hipSuccess) e = back; }
    }
    if (e == hipSuccess) return ZF_OK;
    set_error(std::string("HIP: ") + hipGetErrorString(e));
    return ZF_ERR_DEVICE;
}
template <class F>
auto guarded(F f) -> decltype(f()) {          // nothing is thrown across the boundary (an error's text may find no memory)
    try { return f(); } catch (const std::bad_alloc &) { return ZF_ERR_OOM; }
}
bool element_aligned(const void *p, int32_t dtype) { return (uintptr_t)p % (dtype == 0 ? 4 : 2) == 0; }

int check_logprobs(const zf_logprobs_args *a, bool backward) {
    if (!a) return refuse("null argument");
    if (a->dtype != 0 && a->dtype != 1) return refuse("dtype must be 0 (fp32) or 1 (bf16)");
    if (a->V < 1 || a->V > VOCAB_MAX) return refuse("V must be 1..2^24");
    if (a->rows < 0 || a->rows > INT32_MAX) return refuse("rows must be 0..2^31-1");
    if (a->row_stride_elems < a->V) return refuse("the row stride is smaller than V");
    if (a->n_tokens < 0 || a->n_tokens > GIVEN_MAX) return refuse("n_tokens must be 0..1024");
    if (a->top < 0 || a->top > TOP_MAX) return refuse("top must be 0..64");
    if (a->n_tokens && a->token_bytes != 4 && a->token_bytes != 8) return refuse("token_bytes must be 4 or 8");
    if (!(a->temperature >= FLT_MIN) || !std::isfinite(a->temperature)) return refuse("temperature must be finite, at least 2^-126");   // (its reciprocal is finite)
    if (a->rows == 0) return ZF_OK;
    if (logprobs_blocks(*a) > BLOCKS_MAX) return refuse("more logits than a call takes: split the rows");
    if (!a->logits || (a->n_tokens && (!a->tokens || !a->logprobs)) || (a->top && (!a->top_ids || !a->top_logprobs))) return refuse("null argument");
    if (!element_aligned(a->logits, a->dtype)) return refuse("the logits are not aligned to an element");
    if (backward && !a->stats) return refuse("the gradient needs the stats that zf_token_logprobs wrote");
    return ZF_OK;
}

}  // namespace

extern "C" {

int zf_quantize_blocks(const void *d_x, int32_t dtype, int64_t rows, int32_t cols, int64_t row_stride_elems, int32_t block_rows,
                       uint8_t *d_q, float *d_scale, int32_t device, void *hip_stream) {
    return guarded([&]() -> int {
        if (dtype != 0 && dtype != 1) return refuse("dtype must be 0 (fp32) or 1 (bf16)");
        if (rows < 0 || rows > INT32_MAX || cols < 1 || cols > (1 << 24)) return refuse("rows must be 0..2^31-1, cols 1..2^24");
        if (row_stride_elems < cols) return refuse("the row stride is smaller than cols");
        if (block_rows != 1 && block_rows != SCALE_BLOCK) return refuse("block_rows must be 1 or 128");
        if (block_rows == SCALE_BLOCK && (rows + SCALE_BLOCK - 1) / SCALE_BLOCK * (((int64_t)cols + SCALE_BLOCK - 1) / SCALE_BLOCK) > BLOCKS_MAX) return refuse("more blocks than a call takes: split the rows");
        if (rows == 0) return ZF_OK;
        if (!d_x || !d_q || !d_scale) return refuse("null argument");
        if (!element_aligned(d_x, dtype) || (uintptr_t)d_q % 16) return refuse("x must be aligned to an element, q to 16 bytes");
        return on_device(device, [&]() { return launch_quantize(d_x, dtype, rows, cols, row_stride_elems, block_rows, d_q, d_scale, (hipStream_t)hip_stream); });
    });
}

int zf_head_logits(const uint8_t *d_x, int64_t x_row_stride, const float *d_x_scale, const uint8_t *d_w, int64_t w_row_stride, const float *d_w_scale,
                   int32_t batch, int32_t V, int32_t K, const uint32_t *d_mask, void *d_out, int32_t dtype, int64_t out_row_stride_elems,
                   int32_t device, void *hip_stream) {
    return guarded([&]() -> int {
        if (dtype != 0 && dtype != 1) return refuse("dtype must be 0 (fp32) or 1 (bf16)");
        if (batch < 0 || batch > (1 << 20) || V < 1 || V > VOCAB_MAX || K < SCALE_BLOCK || K > (1 << 24) || K % SCALE_BLOCK) return refuse("batch must be 0..2^20, V 1..2^24, K a multiple of 128 up to 2^24");
        if (x_row_stride < K || w_row_stride < K || x_row_stride % 16 || w_row_stride % 16) return refuse("rows of x and w are K bytes, at multiples of 16");
        if (out_row_stride_elems < V) return refuse("the row stride is smaller than V");
        if (batch == 0) return ZF_OK;
        if (!d_x || !d_x_scale || !d_w || !d_w_scale || !d_out) return refuse("null argument");
        if ((uintptr_t)d_x % 16 || (uintptr_t)d_w % 16) return refuse("x and w must be aligned to 16 bytes");
        if (!element_aligned(d_out, dtype)) return refuse("the logits are not aligned to an element");
        const HeadArgs a{d_x, d_w, d_x_scale, d_w_scale, x_row_stride, w_row_stride, out_row_stride_elems, batch, V, K, d_mask, d_out, dtype};
        return on_device(device, [&]() { return launch_head(a, (hipStream_t)hip_stream); });
    });
}

int64_t zf_token_logprobs_workspace(const zf_logprobs_args *a) {
    return guarded([&]() -> int64_t {
        const int rc = check_logprobs(a, false);
        return rc != ZF_OK ? rc : a->rows ? logprobs_workspace(*a) : 0;
    });
}

int zf_token_logprobs(const zf_logprobs_args *a, void *d_workspace, int64_t workspace_bytes, int32_t device, void *hip_stream) {
    return guarded([&]() -> int {
        const int rc = check_logprobs(a, false);
        if (rc != ZF_OK || a->rows == 0) return rc;
        if (workspace_bytes < logprobs_workspace(*a)) return refuse("the workspace is smaller than zf_token_logprobs_workspace says");
        if (workspace_bytes && (!d_workspace || (uintptr_t)d_workspace % 16)) return refuse("the workspace must be aligned to 16 bytes");
        return on_device(device, [&]() { return launch_logprobs(*a, d_workspace, (hipStream_t)hip_stream); });
    });
}

int zf_token_logprobs_backward(const zf_logprobs_args *a, const float *g_logprobs, const float *g_entropy, const float *g_top,
                               void *d_grad, int64_t grad_row_stride_elems, int32_t device, void *hip_stream) {
    return guarded([&]() -> int {
        const int rc = check_logprobs(a, true);
        if (rc != ZF_OK || a->rows == 0) return rc;
        if (!d_grad || !element_aligned(d_grad, a->dtype)) return refuse("the gradient must be there, aligned to an element");
        if (grad_row_stride_elems < a->V) return refuse("the gradient's row stride is smaller than V");
        if (g_entropy && !a->entropy) return refuse("a gradient of the entropy needs the entropy");
        const LogprobsGrad g{a->n_tokens ? g_logprobs : nullptr, g_entropy, a->top ? g_top : nullptr, d_grad, grad_row_stride_elems};
        return on_device(device, [&]() { return launch_logprobs_backward(*a, g, (hipStream_t)hip_stream); });
    });
}

}  // extern "C"
