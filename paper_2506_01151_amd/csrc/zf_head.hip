// The head's product in 8-bit floating point, and what brings its operands to 8 bits.
//
//   q = e4m3(x / s),  s = max(amax / 448, 2^-126)                 amax over a block: 128 columns of one row, or of 128 rows
//   y[m][v] = sum_k xs[m][k] ws[v / 128][k] (sum over the 128 columns of block k of x[m][..] w[v][..])
//
// One v_mfma_f32_16x16x128_f8f6f4 takes 16 tokens, 16 rows of the batch and exactly one block of columns, so a block's inner sum
// is one instruction from zero and its scale one fused multiply-add for each of the four results that a lane holds.  Sums are held in 32 bits.  The order of
// the 128 columns within the instruction's operands does not matter as long as it is the same for both: a lane takes bytes 16 c .. 16 c + 15 and
// 64 + 16 c .. 64 + 16 c + 15 of a block, c = lane / 16, of the row that is its lane % 16.
//   The 8-bit instructions are not exact to 32 bits, whatever their shape: of eight neighbouring products they keep what lies less than about 2^-14
// below the largest (measured: blocks of normal numbers come out 1.3e-5 off relative to their norm, of numbers spread over e^2 5e-5).  For logits in bf16, which are
// rounded by up to 2^-9 anyway, that is nothing.  For fp32 logits the operands are brought to bf16, which holds every e4m3 number, and
// four v_mfma_f32_16x16x32_bf16 make the block's sum (1e-8 and 7e-8 off), at half the rate.
#include <hip/hip_runtime.h>
#include <algorithm>
#include "zf_ops.h"

namespace zf {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
// 16 bytes at any multiple of an element: the memory system takes them there
template <typename ElemT> struct Piece;
template <> struct Piece<uint32_t> { typedef u32x4 type __attribute__((aligned(4))); };
template <> struct Piece<uint16_t> { typedef u32x4 type __attribute__((aligned(2))); };

__device__ __forceinline__ float of_bits(uint32_t x) { return __uint_as_float(x); }
__device__ __forceinline__ float of_bits(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
__device__ __forceinline__ uint16_t bf16_of(float x) {             // to nearest, ties to even
    uint32_t u = __float_as_uint(x);
    if ((u & 0x7FFFFFFFu) > 0x7F800000u) return (uint16_t)((u >> 16) | 0x40u);
    return (uint16_t)((u + 0x7FFFu + ((u >> 16) & 1u)) >> 16);
}

// ---- to 8 bits ----

// Eight consecutive elements of a row from column c on; zero from `cols` on.
template <typename ElemT>
__device__ __forceinline__ void load8(const ElemT *row, int32_t c, int32_t cols, float (&x)[8]) {
    const int EPV = 16 / sizeof(ElemT);
    if (c + 8 <= cols) {
#pragma unroll
        for (int h = 0; h < 8 / EPV; h++) {
            const u32x4 v = *reinterpret_cast<const typename Piece<ElemT>::type *>(row + c + h * EPV);
#pragma unroll
            for (int k = 0; k < EPV; k++) x[h * EPV + k] = sizeof(ElemT) == 4 ? of_bits((uint32_t)v[k]) : of_bits((uint16_t)(v[k / 2] >> (16 * (k & 1))));
        }
    } else {
#pragma unroll
        for (int k = 0; k < 8; k++) x[k] = c + k < cols ? of_bits(row[c + k]) : 0.0f;
    }
}
__device__ __forceinline__ float amax8(const float (&x)[8]) {
    float m = 0.0f;
#pragma unroll
    for (int k = 0; k < 8; k++) m = fmaxf(m, fabsf(x[k]));
    return m;
}
// A quotient beyond 448 (by its rounding) is 448; a NaN stays one.
__device__ __forceinline__ float to_range(float x, float scale) {
    const float t = x / scale, c = fminf(fmaxf(t, -E4M3_MAX), E4M3_MAX);
    return t != t ? t : c;
}
__device__ __forceinline__ u32x2 quantize8(const float (&x)[8], float scale) {
    u32x2 q;
#pragma unroll
    for (int h = 0; h < 2; h++) {
        int p = __builtin_amdgcn_cvt_pk_fp8_f32(to_range(x[4 * h], scale), to_range(x[4 * h + 1], scale), 0, false);
        p = __builtin_amdgcn_cvt_pk_fp8_f32(to_range(x[4 * h + 2], scale), to_range(x[4 * h + 3], scale), p, true);
        q[h] = (uint32_t)p;
    }
    return q;
}
__device__ __forceinline__ float scale_of(float amax) { return fmaxf(amax / E4M3_MAX, SCALE_MIN); }

// Blocks of one row: 16 lanes a block, eight columns a lane.
template <typename ElemT>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const ElemT *__restrict__ x, int64_t stride, int64_t rows, int32_t cols, int32_t n_blocks,
                                                            uint8_t *__restrict__ q, float *__restrict__ scale) {
    const int32_t lane = threadIdx.x % 16;
    for (int64_t block = (int64_t)blockIdx.x * 16 + threadIdx.x / 16; block < rows * n_blocks; block += (int64_t)gridDim.x * 16) {   // whole groups of 16 lanes
        const int64_t r = block / n_blocks;
        const int32_t b = (int32_t)(block - r * n_blocks);
        float v[8];
        load8(x + r * stride, b * SCALE_BLOCK + lane * 8, cols, v);
        float m = amax8(v);
#pragma unroll
        for (int d = 1; d < 16; d *= 2) m = fmaxf(m, __shfl_xor(m, d, 16));
        const float s = scale_of(m);
        *reinterpret_cast<u32x2 *>(q + block * SCALE_BLOCK + lane * 8) = quantize8(v, s);
        if (lane == 0) scale[block] = s;
    }
}

// Blocks of 128 rows: a workgroup a block, its elements stay in registers between the largest and the quotients.
template <typename ElemT>
__global__ __launch_bounds__(256) void quantize_square_kernel(const ElemT *__restrict__ x, int64_t stride, int64_t rows, int32_t cols, int32_t n_blocks,
                                                              uint8_t *__restrict__ q, float *__restrict__ scale) {
    __shared__ float most[4];
    const int32_t b = blockIdx.x % n_blocks, lane = threadIdx.x % 16;
    const int64_t tall = blockIdx.x / n_blocks, r0 = tall * SCALE_BLOCK + threadIdx.x / 16;
    float v[8][8], m = 0.0f;
#pragma unroll
    for (int p = 0; p < 8; p++) {
        const int64_t r = r0 + p * 16;
        if (r < rows) load8(x + r * stride, b * SCALE_BLOCK + lane * 8, cols, v[p]);
        else
#pragma unroll
            for (int k = 0; k < 8; k++) v[p][k] = 0.0f;
    }
#pragma unroll
    for (int p = 0; p < 8; p++) m = fmaxf(m, amax8(v[p]));
#pragma unroll
    for (int d = 1; d < 64; d *= 2) m = fmaxf(m, __shfl_xor(m, d));
    if (threadIdx.x % 64 == 0) most[threadIdx.x / 64] = m;
    __syncthreads();
    const float s = scale_of(fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3])));
#pragma unroll
    for (int p = 0; p < 8; p++) {
        const int64_t r = r0 + p * 16;
        if (r < rows) *reinterpret_cast<u32x2 *>(q + (r * n_blocks + b) * SCALE_BLOCK + lane * 8) = quantize8(v[p], s);
    }
    if (threadIdx.x == 0) scale[tall * n_blocks + b] = s;
}

// ---- the product ----

// Sixteen tokens against sixteen rows over the block's columns that a lane holds of both, as the logits' type wants it.
template <typename ElemT> struct Operand;
template <> struct Operand<uint16_t> {
    i32x8 v;
    __device__ __forceinline__ void take(i32x4 a, i32x4 b) { v = i32x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]}; }
    __device__ __forceinline__ f32x4 times(const Operand &o) const { return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(v, o.v, f32x4{0, 0, 0, 0}, 0, 0, 0, 0, 0, 0); }
};
template <> struct Operand<uint32_t> {
    bf16x8 v[4];
    static __device__ __forceinline__ bf16x8 wide(int a, int b) {
        const bf16x2 p = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, false), q = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, true);
        const bf16x2 r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, false), t = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, true);
        return bf16x8{p[0], p[1], q[0], q[1], r[0], r[1], t[0], t[1]};
    }
    __device__ __forceinline__ void take(i32x4 a, i32x4 b) { v[0] = wide(a[0], a[1]); v[1] = wide(a[2], a[3]); v[2] = wide(b[0], b[1]); v[3] = wide(b[2], b[3]); }
    __device__ __forceinline__ f32x4 times(const Operand &o) const {
        f32x4 d{0, 0, 0, 0};
#pragma unroll
        for (int h = 0; h < 4; h++) d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[h], o.v[h], d, 0, 0, 0);
        return d;
    }
};

// A workgroup has the 128 tokens of one scale and up to 16 MT rows of the batch: it lists the tokens that some of its rows allows and
// its wavefronts take sixteen of them at a time through all columns, straight from memory.  Results gather in LDS, so that the
// logits go out in whole rows of the range, -inf where nothing was computed.
template <int MT, bool MASK, typename ElemT>
__global__ __launch_bounds__(256) void head_rows_kernel(HeadArgs a) {
    constexpr int ROWS = MT * 16, PITCH = SCALE_BLOCK + 4;
    __shared__ float tile[ROWS][PITCH];
    __shared__ uint32_t words[ROWS][4], need[4];
    __shared__ uint8_t list[SCALE_BLOCK];
    const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
    const int32_t v0 = blockIdx.x * SCALE_BLOCK, m0 = blockIdx.y * ROWS;
    const int32_t rows = a.M - m0 < ROWS ? a.M - m0 : ROWS, n_v = a.V - v0 < SCALE_BLOCK ? a.V - v0 : SCALE_BLOCK, n_k = a.K / SCALE_BLOCK;
    int32_t count = n_v;
    if (MASK) {
        const int32_t W = (a.V + 31) / 32;
        if (tid < 4) need[tid] = 0;
        for (int i = tid; i < ROWS * PITCH; i += 256) (&tile[0][0])[i] = -INFINITY;
        __syncthreads();
        for (int i = tid; i < rows * 4; i += 256) {
            const int32_t j = i & 3, left = n_v - 32 * j;                    // tokens of the word that there are
            uint32_t w = left > 0 ? a.mask[(size_t)(m0 + i / 4) * W + v0 / 32 + j] : 0;
            if (left < 32 && left > 0) w &= (1u << left) - 1;
            words[i / 4][j] = w;
            if (w) atomicOr(&need[j], w);                                    // the same in any order
        }
        __syncthreads();
        count = __popc(need[0]) + __popc(need[1]) + __popc(need[2]) + __popc(need[3]);
        if (tid < SCALE_BLOCK && ((need[tid / 32] >> (tid % 32)) & 1)) {
            int at = __popc(need[tid / 32] & ((1u << (tid % 32)) - 1));
            for (int j = 0; j < tid / 32; j++) at += __popc(need[j]);
            list[at] = (uint8_t)tid;
        }
        __syncthreads();
    }
    const float *const ws = a.ws + (size_t)blockIdx.x * n_k;
    for (int g = wave * 16; g < count; g += 64) {
        const int i = g + lane % 16 < count ? g + lane % 16 : count - 1;     // behind the last token: its row once more
        const uint8_t *const wp = a.w + (int64_t)(v0 + (MASK ? list[i] : i)) * a.w_stride + lane / 16 * 16;
        const uint8_t *xp[MT];
        const float *xs[MT];
        f32x4 acc[MT];
#pragma unroll
        for (int t = 0; t < MT; t++) {
            const int32_t m = m0 + t * 16 + lane % 16 < a.M ? m0 + t * 16 + lane % 16 : a.M - 1;
            xp[t] = a.x + m * a.x_stride + lane / 16 * 16;
            xs[t] = a.xs + (size_t)m * n_k;
            acc[t] = f32x4{0, 0, 0, 0};
        }
        for (int32_t k = 0; k < n_k; k++) {
            Operand<ElemT> w, x;
            w.take(*reinterpret_cast<const i32x4 *>(wp + (size_t)k * SCALE_BLOCK), *reinterpret_cast<const i32x4 *>(wp + (size_t)k * SCALE_BLOCK + 64));
            const float s_w = ws[k];
#pragma unroll
            for (int t = 0; t < MT; t++) {
                x.take(*reinterpret_cast<const i32x4 *>(xp[t] + (size_t)k * SCALE_BLOCK), *reinterpret_cast<const i32x4 *>(xp[t] + (size_t)k * SCALE_BLOCK + 64));
                const f32x4 part = w.times(x);
                const float s = xs[t][k] * s_w;
#pragma unroll
                for (int r = 0; r < 4; r++) acc[t][r] = fmaf(s, part[r], acc[t][r]);
            }
        }
#pragma unroll
        for (int t = 0; t < MT; t++) {
            const int m = t * 16 + lane % 16;
#pragma unroll
            for (int r = 0; r < 4; r++) {
                const int j = g + lane / 16 * 4 + r;
                if (j >= count || m >= rows) continue;
                const int v = MASK ? list[j] : j;
                if (!MASK || ((words[m][v / 32] >> (v % 32)) & 1)) tile[m][v] = acc[t][r];
            }
        }
    }
    __syncthreads();
    constexpr int EPV = 16 / sizeof(ElemT), PIECES = SCALE_BLOCK / EPV;
    ElemT *const y = (ElemT *)a.y + v0;
    for (int i = tid; i < rows * PIECES; i += 256) {
        const int m = i / PIECES, v = i % PIECES * EPV;
        ElemT *const to = y + (int64_t)(m0 + m) * a.y_stride + v;
        union { ElemT e[EPV]; u32x4 v; } o;
#pragma unroll
        for (int k = 0; k < EPV; k++) o.e[k] = sizeof(ElemT) == 4 ? (ElemT)__float_as_uint(tile[m][v + k]) : (ElemT)bf16_of(tile[m][v + k]);
        if (v + EPV <= n_v) *reinterpret_cast<typename Piece<ElemT>::type *>(to) = o.v;
        else {
#pragma unroll
            for (int k = 0; k < EPV; k++) if (v + k < n_v) to[k] = o.e[k];
        }
    }
}

template <int MT, bool MASK, typename ElemT>
void head_rows(const HeadArgs &a, hipStream_t s) {
    const dim3 grid((a.V + SCALE_BLOCK - 1) / SCALE_BLOCK, (a.M + MT * 16 - 1) / (MT * 16));
    hipLaunchKernelGGL((head_rows_kernel<MT, MASK, ElemT>), grid, dim3(256), 0, s, a);
}
template <bool MASK, typename ElemT>
void head(const HeadArgs &a, hipStream_t s) {
    if (a.M <= 16) head_rows<1, MASK, ElemT>(a, s);
    else if (a.M <= 32) head_rows<2, MASK, ElemT>(a, s);
    else head_rows<4, MASK, ElemT>(a, s);
}

template <typename ElemT>
void quantize(const ElemT *x, int64_t rows, int32_t cols, int64_t stride, int32_t block_rows, uint8_t *q, float *scale, hipStream_t s) {
    const int32_t n_blocks = (cols + SCALE_BLOCK - 1) / SCALE_BLOCK;
    if (block_rows == 1)
        hipLaunchKernelGGL((quantize_rows_kernel<ElemT>), dim3((uint32_t)std::min<int64_t>((rows * n_blocks + 15) / 16, BLOCKS_MAX)), dim3(256), 0, s, x, stride, rows, cols, n_blocks, q, scale);
    else
        hipLaunchKernelGGL((quantize_square_kernel<ElemT>), dim3((uint32_t)((rows + SCALE_BLOCK - 1) / SCALE_BLOCK * n_blocks)), dim3(256), 0, s, x, stride, rows, cols, n_blocks, q, scale);
}

}  // namespace

hipError_t launch_quantize(const void *x, int dtype, int64_t rows, int32_t cols, int64_t stride, int32_t block_rows, uint8_t *q, float *scale, hipStream_t s) {
    if (dtype == 0) quantize((const uint32_t *)x, rows, cols, stride, block_rows, q, scale, s);
    else quantize((const uint16_t *)x, rows, cols, stride, block_rows, q, scale, s);
    return hipGetLastError();
}

hipError_t launch_head(const HeadArgs &a, hipStream_t s) {
    if (a.mask) a.dtype == 0 ? head<true, uint32_t>(a, s) : head<true, uint16_t>(a, s);
    else a.dtype == 0 ? head<false, uint32_t>(a, s) : head<false, uint16_t>(a, s);
    return hipGetLastError();
}

}  // namespace zf
