// Interface between the calls at the two ends of a step's logits (zf_ops.cpp) and their kernels (zf_head.hip, zf_logprobs.hip).
#pragma once
#include <hip/hip_runtime_api.h>
#include <cstdint>
#include "../../include/zapformat.h"

namespace zf {

static const int SCALE_BLOCK = 128;            // elements of a row that share a scale, and rows of a weight that do
static const float E4M3_MAX = 448.0f;          // e4m3's largest number
static const float SCALE_MIN = 0x1p-126f;      // no scale is below it (the smallest normal number of 32 bits)
static const int TOP_MAX = 64;                 // alternatives a row: one per lane of the joining wavefront
static const int GIVEN_MAX = 1024;             // given tokens a row: what the gradient's blocks list in LDS
static const int VOCAB_MAX = 1 << 24;
static const int64_t BLOCKS_MAX = (1 << 24) - 1; // workgroups of 256 threads in a launch (2^32 threads at most)

struct HeadArgs {
    const uint8_t *x, *w;
    const float *xs, *ws;
    int64_t x_stride, w_stride, y_stride;
    int32_t M, V, K;
    const uint32_t *mask;
    void *y;
    int32_t dtype;
};
struct LogprobsGrad {
    const float *g_logprobs, *g_entropy, *g_top;
    void *grad;
    int64_t stride;
};

hipError_t launch_quantize(const void *x, int dtype, int64_t rows, int32_t cols, int64_t stride, int32_t block_rows, uint8_t *q, float *scale, hipStream_t s);
hipError_t launch_head(const HeadArgs &a, hipStream_t s);
int64_t logprobs_workspace(const zf_logprobs_args &a);
int64_t logprobs_blocks(const zf_logprobs_args &a);   // workgroups that a pass over the logits takes
hipError_t launch_logprobs(const zf_logprobs_args &a, void *workspace, hipStream_t s);
hipError_t launch_logprobs_backward(const zf_logprobs_args &a, const LogprobsGrad &g, hipStream_t s);

}  // namespace zf
