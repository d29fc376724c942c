// The head's product in 8-bit floating point, and what brings its operands to 8 bits.
//
//   q = e4m3(x / s),  s = max(amax / 448, 2^-126)                 amax over a block: 128 columns of one row, or of 128 rows
//   y[m][v] = sum_k xs[m][k] ws[v / 128][k] (sum over the 128 columns of block k of x[m][..] w[v][..])
//
// One v_mfma_f32_16x16x128_f8f6f4 takes 16 tokens, 16 rows of the batch and exactly one block of columns, so a block's inner sum
// is one instruction from zero and its scale one fused multiply-add for each of the four results that a lane holds.  The sum over the blocks is held in 32 bits.  The order of
// the 128 columns within the instruction's operands does not matter as long as it is the same for both: a lane takes bytes 16 c .. 16 c + 15 and
// 64 + 16 c .. 64 + 16 c + 15 of a block, c = lane / 16, of the row that is its lane % 16.
//   The 8-bit instructions do not hold a block's sum in 32 bits, whatever their shape: of eight neighbouring products each is cut, towards zero, to a multiple of 2^-13 of the largest one's power of
// two (measured: one of 2^-14 beside it is gone; the largest itself is exact).  So a logit is off by less than 7 x 2^-13 of the sum of its products' sizes; blocks of normal numbers come out 1.3e-5
// off relative to their norm, of numbers spread over e^2 5e-5, root of the mean square.  Logits in bf16 take them: one about as large as its norm is rounded by up to 2^-8 of itself anyway, 300 times
// that; one whose products cancel to a hundredth of their norm or less carries more of this than of its rounding.  The same product in bf16 instructions would take twice the time where the product
// bounds it.  For fp32 logits the operands are brought to bf16, which holds every e4m3 number, and four v_mfma_f32_16x16x32_bf16 make the block's sum (1e-8 and 7e-8 off), at half the rate.
#include <hip/hip_runtime.h>
#include <algorithm>
#include <atomic>
#include "zf_ops.h"

namespace zf {
namespace {

static const int COMPUTE_UNITS = 256;
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
    union { __bf16 b; uint16_t u; } o;
    o.b = (__bf16)x;
    return o.u;
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
// Quotients by a scale that many elements share, to nearest in 32 bits as a division gives them: with r the reciprocal to nearest, one step t + r (x - t s) brings the product x r
// within a step of the quotient and the next one rounds it right (Markstein's theorem on division by fused multiply-adds), as long as nothing leaves the
// range of normal numbers on the way: an element counts from s 2^-11 on and x - t s is a multiple of 2^-46 of it.  Scales beyond that divide.
// 32,000 x 4,096 bf16 in blocks of one row 72 us, with divisions 82; of 128 rows 83 and 98.
struct Quotient {
    float s, r;
    bool near_one;
    __device__ __forceinline__ Quotient(float scale) : s(scale), r(1.0f / scale), near_one(scale > 0x1p-60f && scale < 0x1p100f) {}
    __device__ __forceinline__ float of(float x) const {
        if (!near_one) return x / s;
        float t = x * r;
        t = fmaf(fmaf(-t, s, x), r, t);
        return copysignf(fmaf(fmaf(-t, s, x), r, t), x);   // (-0 stays one)
    }
};
// The quotients lie within 448 (1 + 2^-23), which is rounded to 448; a NaN stays one.
__device__ __forceinline__ u32x2 quantize8(const float (&x)[8], const Quotient &by) {
    u32x2 q;
#pragma unroll
    for (int h = 0; h < 2; h++) {
        int p = __builtin_amdgcn_cvt_pk_fp8_f32(by.of(x[4 * h]), by.of(x[4 * h + 1]), 0, false);
        p = __builtin_amdgcn_cvt_pk_fp8_f32(by.of(x[4 * h + 2]), by.of(x[4 * h + 3]), p, true);
        q[h] = (uint32_t)p;
    }
    return q;
}
__device__ __forceinline__ float scale_of(float amax) { return fmaxf(amax / E4M3_MAX, SCALE_MIN); }

// The largest of 16 neighbouring lanes, to all of them.
__device__ __forceinline__ float most_of_16(float x) {
    auto with = [](float x, auto moved) { return fmaxf(x, __int_as_float(moved(__float_as_int(x)))); };
    x = with(x, [](int v) { return __builtin_amdgcn_update_dpp(v, v, 0xB1, 0xF, 0xF, false); });      // lanes 1 0 3 2 of each four
    x = with(x, [](int v) { return __builtin_amdgcn_update_dpp(v, v, 0x4E, 0xF, 0xF, false); });      // lanes 2 3 0 1
    x = with(x, [](int v) { return __builtin_amdgcn_update_dpp(v, v, 0x141, 0xF, 0xF, false); });     // each eight reversed
    return with(x, [](int v) { return __builtin_amdgcn_update_dpp(v, v, 0x140, 0xF, 0xF, false); });  // the sixteen reversed
}

// Blocks of one row: 16 lanes a block, eight columns a lane, N blocks at once.  Memory bounds it: 32,000 x 4,096 bf16 72 us (5.5 TB/s), fp32 110 (6.0); 2,048 x 4,096 bf16
// 7.2 us, of which 4 are its bytes.
template <int N, typename ElemT>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const ElemT *__restrict__ x, int64_t stride, int64_t rows, int32_t cols, int32_t n_blocks,
                                                            uint8_t *__restrict__ q, float *__restrict__ scale) {
    const int32_t lane = threadIdx.x % 16;
    const int64_t n_all = rows * n_blocks;
    for (int64_t block = (int64_t)blockIdx.x * (16 * N) + threadIdx.x / 16; block < n_all; block += (int64_t)gridDim.x * (16 * N)) {   // whole groups of 16 lanes
        float v[N][8];
#pragma unroll
        for (int i = 0; i < N; i++) {
            const int64_t at = block + 16 * i < n_all ? block + 16 * i : block, r = at / n_blocks;
            load8(x + r * stride, (int32_t)(at - r * n_blocks) * SCALE_BLOCK + lane * 8, cols, v[i]);
        }
#pragma unroll
        for (int i = 0; i < N; i++) {
            const int64_t at = block + 16 * i;
            if (at >= n_all) break;
            const float s = scale_of(most_of_16(amax8(v[i])));
            *reinterpret_cast<u32x2 *>(q + at * SCALE_BLOCK + lane * 8) = quantize8(v[i], Quotient(s));
            if (lane == 0) scale[at] = s;
        }
    }
}

// Blocks of 128 rows: a workgroup a block, its elements stay in registers between the largest and the quotients: one pass over memory, which
// bounds it (32,000 x 4,096 fp32 115 us, 5.7 TB/s; bf16 83, 4.7).
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
    m = most_of_16(m);
    m = fmaxf(m, __shfl_xor(m, 16));
    m = fmaxf(m, __shfl_xor(m, 32));
    if (threadIdx.x % 64 == 0) most[threadIdx.x / 64] = m;
    __syncthreads();
    const float s = scale_of(fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3])));
    const Quotient by(s);
#pragma unroll
    for (int p = 0; p < 8; p++) {
        const int64_t r = r0 + p * 16;
        if (r < rows) *reinterpret_cast<u32x2 *>(q + (r * n_blocks + b) * SCALE_BLOCK + lane * 8) = quantize8(v[p], by);
    }
    if (threadIdx.x == 0) scale[tall * n_blocks + b] = s;
}

// ---- the product ----

// Sixteen tokens against sixteen rows over the block's columns that a lane holds of both, as the logits' type wants it.
template <typename ElemT> struct Operand;
template <> struct Operand<uint16_t> {
    i32x8 v;
    __device__ __forceinline__ void take(i32x4 a, i32x4 b) { v = i32x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]}; }
    static constexpr int STEPS = 1;
    template <int H> __device__ __forceinline__ f32x4 times(const Operand &o, f32x4 d) const { return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(v, o.v, d, 0, 0, 0, 0, 0, 0); }
};
template <> struct Operand<uint32_t> {
    bf16x8 v[4];
    static __device__ __forceinline__ bf16x8 wide(int a, int b) {
        const bf16x2 p = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, false), q = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, true);
        const bf16x2 r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, false), t = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, true);
        return bf16x8{p[0], p[1], q[0], q[1], r[0], r[1], t[0], t[1]};
    }
    __device__ __forceinline__ void take(i32x4 a, i32x4 b) { v[0] = wide(a[0], a[1]); v[1] = wide(a[2], a[3]); v[2] = wide(b[0], b[1]); v[3] = wide(b[2], b[3]); }
    static constexpr int STEPS = 4;
    template <int H> __device__ __forceinline__ f32x4 times(const Operand &o, f32x4 d) const { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[H], o.v[H], d, 0, 0, 0); }
};
// The sums of a block of A's tokens against B's rows: all products of a step before those of the next, which add to them.
template <int A, int B, typename ElemT, int H = 0>
__device__ __forceinline__ void multiply(const Operand<ElemT> (&a)[A], const Operand<ElemT> (&b)[B], f32x4 (&d)[A][B]) {
#pragma unroll
    for (int i = 0; i < A; i++)
#pragma unroll
        for (int j = 0; j < B; j++) d[i][j] = a[i].template times<H>(b[j], H ? d[i][j] : f32x4{0, 0, 0, 0});
    if constexpr (H + 1 < Operand<ElemT>::STEPS) multiply<A, B, ElemT, H + 1>(a, b, d);
}

__device__ __forceinline__ i32x4 piece_at(const uint8_t *p) { return *reinterpret_cast<const i32x4 *>(p); }

// ---- memory straight into LDS ----
//
// 64 lanes' 16 (or 4) bytes, each from its address, to consecutive places of LDS from `at` on.  As an instruction: it has no register for a result, and the
// compiler, which does not see it, leaves the waits to the caller instead of waiting in front of every read of LDS.  Its place comes from m0, which the compiler allots to
// nothing and, being reserved, is not to be named as overwritten: no other instruction of these kernels may use it (a test reads the assembly).
__device__ __forceinline__ void to_lds(const uint8_t *base, uint32_t off, uint32_t at) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(at), "v"(off), "s"(base) : "memory");
}
__device__ __forceinline__ void to_lds(const uint8_t *from, uint32_t at) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(at), "v"(from) : "memory");
}
__device__ __forceinline__ void to_lds(const float *from, uint32_t at) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(at), "v"(from) : "memory");
}
template <int N> __device__ __forceinline__ void arrived() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }   // of the wavefront's loads, all but the last N
// What a wavefront's lanes wrote to LDS before it is what they read behind it: LDS takes a wavefront's accesses in turn, the compiler has to leave them so.
__device__ __forceinline__ void in_turn() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}
__device__ __forceinline__ uint32_t lds_at(const void *p) { return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) uint8_t *)p; }

// ---- few rows: the weight streams past them ----
//
// A workgroup takes ranges of TOKENS tokens, each of one scale, and up to 16 MT rows of the batch.  Under a mask it lists the tokens that some of its rows allows, of up to
// RANGES ranges at a time.
//   Long lists, a range at a time: a wavefront takes a quarter of it.  Blocks of columns of the weight's rows and the activations come straight into LDS, STAGES - 1 blocks ahead, in
// lines: a fragment's own addresses (sixteen rows, 16 bytes of each) are taken a lane at a time, at a quarter of the rate.  Every wavefront issues the same number of loads for a
// block, so that a count says which have arrived; one barrier a block.  Piece c of row r lies at place c ^ (r % 8), so that eight rows' pieces of one
// column lie in different banks (the loads write LDS in lanes' order: it is their addresses in memory that are exchanged).  Results gather in LDS, so that the logits
// go out in whole rows of the range, -inf where nothing was computed.
//   The weight's way from memory bounds it: 16 rows x 128,256 x 4,096 bf16 103 us (5.1 TB/s), x 8,192 187 (5.6), 64 rows x 4,096 114 to 118 (4.5); one row x 32,000 x 4,096 29 (4.4).  With 64 rows fp32 logits' operands, brought to bf16 in every wavefront, take two fifths of the time beside it: 64 x 152,064 x 2,048 fp32 80 us, bf16 73.  Under
// masks workgroups take two or three ranges each, and the last ones run alone: 87 and 80.
//   Up to 32 tokens of all ranges, or of one (TOKENS = 16 has no others), sixteen at a time: the wavefronts take every fourth block of columns each, the weight straight to registers,
// activations through LDS (TOKENS = 16: straight to registers), and join their sums in a fixed order.  Everything is -inf first.  (16 x 128,256 x 4,096 with 200 tokens a
// row: 13.6 us; when every range was a workgroup's own 22.)
template <int MT, int TOKENS, bool MASK>
struct RowsLds {
    static constexpr int ROWS = MT * 16, PITCH = TOKENS + 4, RANGES = MASK && TOKENS > 16 ? 4 : 1, SHORT = 32;
    static constexpr int X_AT = TOKENS * SCALE_BLOCK, S_AT = X_AT + ROWS * SCALE_BLOCK, STAGE = S_AT + 64 * 4;   // weight, activations, their scales
    static constexpr int STAGES = TOKENS == 64 ? 7 : MT == 1 ? 4 : 3;
    static constexpr int OWN = TOKENS > 16 ? TOKENS / 4 : 16, W_LOADS = OWN / 8, G = OWN / 16, LOADS = W_LOADS + (MT + 1) / 2 + 1;                       // of a wavefront for a stage
    static constexpr int SPAN = MT == 1 ? 4096 : 1024;      // columns of the activations that the short form has in LDS
    static constexpr int LOOP = TOKENS > 16 ? STAGES * STAGE : 0, TILE = TOKENS > 16 ? ROWS * PITCH * 4 : 0, JOIN = 3 * ROWS * 16 * 4;  // the loop, then the logits; the short form's sums
    static constexpr int BYTES = LOOP > TILE ? (LOOP > JOIN ? LOOP : JOIN) : (TILE > JOIN ? TILE : JOIN);
    static_assert(!MASK || TOKENS == 16 || ROWS * SPAN <= STAGES * STAGE, "the short form's activations lie in the stages' memory");
};

template <int MT, int TOKENS, bool MASK, typename ElemT>
__global__ __launch_bounds__(256, 2) void head_rows_kernel(HeadArgs a, int32_t n_ranges) {
    typedef RowsLds<MT, TOKENS, MASK> Lds;
    constexpr int ROWS = Lds::ROWS, PITCH = Lds::PITCH, WORDS = (TOKENS + 31) / 32, STAGES = Lds::STAGES, RANGES = Lds::RANGES, EPV = 16 / sizeof(ElemT);
    extern __shared__ __align__(16) uint8_t mem[];
    __shared__ uint32_t words[MASK ? RANGES : 1][MASK ? ROWS : 1][WORDS], need[RANGES][WORDS];
    __shared__ uint16_t list[MASK ? RANGES * TOKENS : 1];                    // range of the group * TOKENS + token of the range
    const int tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64);
    const int32_t m0 = blockIdx.y * ROWS, rows = a.M - m0 < ROWS ? a.M - m0 : ROWS, n_k = a.K / SCALE_BLOCK, W = (a.V + 31) / 32;
    const int c0 = (lane / 16 ^ lane % 8) * 16, c1 = ((lane / 16 + 4) ^ lane % 8) * 16;      // the lane's two pieces of a row that is lane % 8 modulo 8
    auto x_row = [&](int r) { return m0 + (r < rows ? r : rows - 1); };
    int32_t base = blockIdx.x;                                               // the group's ranges are base, base + gridDim.x, ...
    auto first_of = [&](int range) { return (base + range * (int32_t)gridDim.x) * TOKENS; };   // token
    auto token_of = [&](int i) { return MASK ? first_of(list[i] / TOKENS) + list[i] % TOKENS : base * TOKENS + i; };
    auto allowed = [&](int i, int m) { return !MASK || ((words[list[i] / TOKENS][m][list[i] % TOKENS / 32] >> (list[i] % 32)) & 1); };
    auto put = [&](ElemT *to, float y) { *to = sizeof(ElemT) == 4 ? (ElemT)__float_as_uint(y) : (ElemT)bf16_of(y); };

    // Logits of a range, from LDS or -inf.
    auto store_range = [&](int32_t v0, const float *tile) {
        const int32_t n_v = a.V - v0 < TOKENS ? a.V - v0 : TOKENS;
        constexpr int PIECES = TOKENS / EPV;
        for (int i = tid; i < rows * PIECES; i += 256) {
            const int m = i / PIECES, v = i % PIECES * EPV;
            ElemT *const to = (ElemT *)a.y + (int64_t)(m0 + m) * a.y_stride + v0 + v;
            union { ElemT e[EPV]; u32x4 v; } o;
#pragma unroll
            for (int k = 0; k < EPV; k++) put(&o.e[k], tile ? tile[m * PITCH + v + k] : -INFINITY);
            if (v + EPV <= n_v) *reinterpret_cast<typename Piece<ElemT>::type *>(to) = o.v;
            else {
#pragma unroll
                for (int k = 0; k < EPV; k++) if (v + k < n_v) to[k] = o.e[k];
            }
        }
    };

    // Up to sixteen listed tokens from `at` on.
    auto short_form = [&](int at, int count) {
        constexpr bool NEAR = TOKENS > 16;                                                   // activations through LDS
        constexpr int U = NEAR ? Lds::SPAN / SCALE_BLOCK / 4 : MT == 4 ? 1 : MT == 2 ? 2 : 4;   // blocks of columns a wavefront asks for at a time
        const bool real = lane % 16 < count;
        const uint8_t *const wp = a.w + (int64_t)token_of(at + (real ? lane % 16 : 0)) * a.w_stride + lane / 16 * 16, *xp[MT];
        const float *xs[MT], *ws[4];
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const int j = lane / 16 * 4 + e;
            ws[e] = a.ws + (size_t)(token_of(at + (j < count ? j : 0)) / SCALE_BLOCK) * n_k;
        }
#pragma unroll
        for (int t = 0; t < MT; t++) {
            xp[t] = a.x + x_row(t * 16 + lane % 16) * a.x_stride + lane / 16 * 16;
            xs[t] = a.xs + (size_t)x_row(t * 16 + lane % 16) * n_k;
        }
        f32x4 acc[MT];
#pragma unroll
        for (int t = 0; t < MT; t++) acc[t] = f32x4{0, 0, 0, 0};
        for (int32_t from = 0; from < n_k; from += 4 * U) {
            i32x4 w[U][2] = {}, x[U][MT][2];
            float s[U][MT], s_w[U][4];
            if (NEAR) {
                const int groups = (rows + 7) / 8, n = n_k - from < 4 * U ? n_k - from : 4 * U;   // of eight rows; the span's blocks in turn
                for (int i = wave; i < groups * n; i += 4) {
                    const int r = i % groups * 8 + lane / 8, k = i / groups;
                    to_lds(a.x + x_row(r) * a.x_stride + (size_t)(from + k) * SCALE_BLOCK + (lane % 8 ^ lane / 8) * 16, lds_at(mem) + k * (ROWS * SCALE_BLOCK) + i % groups * 8 * SCALE_BLOCK);
                }
            }
#pragma unroll
            for (int u = 0; u < U; u++) {
                const int32_t k = from + wave + 4 * u;
                if (k >= n_k) continue;
                if (real)                                                    // (a lane with nothing to ask for takes its turn all the same)
#pragma unroll
                    for (int h = 0; h < 2; h++) w[u][h] = __builtin_nontemporal_load(reinterpret_cast<const i32x4 *>(wp + (size_t)k * SCALE_BLOCK + 64 * h));
#pragma unroll
                for (int e = 0; e < 4; e++) s_w[u][e] = ws[e][k];
#pragma unroll
                for (int t = 0; t < MT; t++) {
                    if (!NEAR)
#pragma unroll
                        for (int h = 0; h < 2; h++) x[u][t][h] = piece_at(xp[t] + (size_t)k * SCALE_BLOCK + 64 * h);
                    s[u][t] = xs[t][k];
                }
            }
            if (NEAR) {
                arrived<0>();
                __syncthreads();
            }
#pragma unroll
            for (int u = 0; u < U; u++) {
                if (from + wave + 4 * u >= n_k) continue;
                Operand<ElemT> v[MT], y[1];
                f32x4 part[1][MT];
#pragma unroll
                for (int t = 0; t < MT; t++) {
                    const uint8_t *const from_lds = mem + (wave + 4 * u) * (ROWS * SCALE_BLOCK) + (t * 16 + lane % 16) * SCALE_BLOCK;
                    if (NEAR) v[t].take(piece_at(from_lds + c0), piece_at(from_lds + c1));
                    else v[t].take(x[u][t][0], x[u][t][1]);
                }
                y[0].take(w[u][0], w[u][1]);
                multiply(y, v, part);
#pragma unroll
                for (int t = 0; t < MT; t++)
#pragma unroll
                    for (int e = 0; e < 4; e++) acc[t][e] = fmaf(s[u][t] * s_w[u][e], part[0][t][e], acc[t][e]);
            }
            if (NEAR) __syncthreads();                                       // the span has been read
        }
        f32x4 *const sums = reinterpret_cast<f32x4 *>(mem);
        if (wave) {
#pragma unroll
            for (int t = 0; t < MT; t++) sums[((wave - 1) * MT + t) * 64 + lane] = acc[t];
        }
        arrived<0>();                                                        // (what was -inf first, too)
        __syncthreads();
        if (wave == 0) {
#pragma unroll
            for (int t = 0; t < MT; t++) {
                f32x4 y = acc[t];
#pragma unroll
                for (int w = 0; w < 3; w++) y += sums[(w * MT + t) * 64 + lane];
                const int m = t * 16 + lane % 16;
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    const int j = lane / 16 * 4 + e;
                    if (j < count && m < rows && allowed(at + j, m)) put((ElemT *)a.y + (int64_t)(m0 + m) * a.y_stride + token_of(at + j), y[e]);
                }
            }
        }
        __syncthreads();
    };

    // The listed tokens of one range, `count` from `at` on, 32 a wavefront.
    auto long_form = [&](int32_t v0, int at, int count) {
        constexpr int XN = (MT + 1) / 2;                                     // groups of eight of the activations' rows that a wavefront brings
        constexpr int WL = Lds::W_LOADS, G = Lds::G, OWN = Lds::OWN;
        const uint8_t *from[WL + XN];
        const int place = (lane % 8 ^ lane / 8) * 16, first = wave * OWN;
#pragma unroll
        for (int i = 0; i < WL; i++) {
            const int j = first + i * 8 + lane / 8;                          // behind the last token: its row once more
            from[i] = a.w + (int64_t)token_of(at + (j < count ? j : count - 1)) * a.w_stride + place;
        }
#pragma unroll
        for (int i = 0; i < XN; i++) from[WL + i] = a.x + x_row((wave * XN + i) % (2 * MT) * 8 + lane / 8) * a.x_stride + place;
        const float *const xs = a.xs + (size_t)x_row(lane % ROWS) * n_k;
        const auto *const ws = (const __attribute__((address_space(4))) float *)(a.ws + (size_t)(v0 / SCALE_BLOCK) * n_k);   // read by the scalar unit
        // Workgroups begin at blocks of columns of their own: rows lie at multiples of a power of two, and who reads the same columns of many rows asks
        // few of the memory's channels (16 x 128,256 x 4,096: 113 us when all begin at the first, 103 so).
        const int32_t turn = (int32_t)(blockIdx.x * 5u % (uint32_t)n_k);
        auto turned = [&](int32_t k) { return k + turn < n_k ? k + turn : k + turn - n_k; };
        auto fetch = [&](int32_t k) {                                        // behind the last block: that one once more, for the count
            const uint32_t to = lds_at(mem) + k % STAGES * Lds::STAGE;
            const int32_t kk = turned(k < n_k ? k : n_k - 1);
#pragma unroll
            for (int i = 0; i < WL; i++) to_lds(from[i] + (size_t)kk * SCALE_BLOCK, to + (first + i * 8) * SCALE_BLOCK);
#pragma unroll
            for (int i = 0; i < XN; i++) to_lds(from[WL + i] + (size_t)kk * SCALE_BLOCK, to + Lds::X_AT + (wave * XN + i) % (2 * MT) * 8 * SCALE_BLOCK);
            to_lds(xs + kk, to + Lds::S_AT);
        };
        // The compiler has loads of the short form in mind, whose registers it uses again in the loop, and would wait there for all loads in flight: it is
        // told here that none is (64 x 152,064 x 2,048 under masks, bf16: 95 us -> 80).
        __builtin_amdgcn_s_waitcnt(0x0F70);
        f32x4 acc[G][MT];
#pragma unroll
        for (int g = 0; g < G; g++)
#pragma unroll
            for (int t = 0; t < MT; t++) acc[g][t] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int k = 0; k < STAGES - 1; k++) fetch(k);
        for (int32_t k = 0; k < n_k; k++) {
            arrived<(STAGES - 2) * Lds::LOADS>();
            __syncthreads();
            fetch(k + STAGES - 1);
            const uint8_t *const stage = mem + k % STAGES * Lds::STAGE;
            const float s_w = ws[turned(k)];
            Operand<ElemT> w[G];
#pragma unroll
            for (int g = 0; g < G; g++) {
                const uint8_t *const p = stage + (first + g * 16 + lane % 16) * SCALE_BLOCK;
                w[g].take(piece_at(p + c0), piece_at(p + c1));
            }
            constexpr int PAIR = MT > 1 ? 2 : 1;                             // sixteens of rows at a time
#pragma unroll
            for (int t0 = 0; t0 < MT; t0 += PAIR) {
                Operand<ElemT> v[PAIR];
                float s[PAIR];
                f32x4 part[G][PAIR];
#pragma unroll
                for (int t = 0; t < PAIR; t++) {
                    const int r = (t0 + t) * 16 + lane % 16;
                    v[t].take(piece_at(stage + Lds::X_AT + r * SCALE_BLOCK + c0), piece_at(stage + Lds::X_AT + r * SCALE_BLOCK + c1));
                    s[t] = reinterpret_cast<const float *>(stage + Lds::S_AT)[r] * s_w;
                }
                multiply(w, v, part);
#pragma unroll
                for (int t = 0; t < PAIR; t++)
#pragma unroll
                    for (int g = 0; g < G; g++)
#pragma unroll
                        for (int e = 0; e < 4; e++) acc[g][t0 + t][e] = fmaf(s[t], part[g][t][e], acc[g][t0 + t][e]);
            }
        }
        arrived<0>();
        __syncthreads();
        float *const tile = reinterpret_cast<float *>(mem);                  // the loop's memory becomes the logits'
        if (MASK) {
            for (int i = tid; i < ROWS * PITCH; i += 256) tile[i] = -INFINITY;
            __syncthreads();
        }
#pragma unroll
        for (int g = 0; g < G; g++)
#pragma unroll
            for (int t = 0; t < MT; t++) {
                const int m = t * 16 + lane % 16;
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    const int j = first + g * 16 + lane / 16 * 4 + e;
                    if (j < count && m < rows && allowed(at + j, m)) tile[m * PITCH + (MASK ? list[at + j] % TOKENS : j)] = acc[g][t][e];
                }
            }
        __syncthreads();
        store_range(v0, tile);
        __syncthreads();
    };

    for (; base < n_ranges; base += RANGES * gridDim.x) {
        if (!MASK) {
            const int32_t v0 = base * TOKENS, n_v = a.V - v0 < TOKENS ? a.V - v0 : TOKENS;
            if (TOKENS == 16) short_form(0, n_v);
            else if constexpr (TOKENS > 16) long_form(v0, 0, n_v);
            continue;
        }
        if (tid < RANGES * WORDS) need[tid / WORDS][tid % WORDS] = 0;
        __syncthreads();
        for (int i = tid; i < RANGES * rows * WORDS; i += 256) {
            const int range = i / (rows * WORDS), m = i / WORDS % rows, j = i % WORDS;
            const int32_t v0 = first_of(range), left = a.V - v0 - 32 * j;    // tokens from the word on (none in a range that is not there)
            uint32_t w = left > 0 ? a.mask[(size_t)(m0 + m) * W + v0 / 32 + j] >> (TOKENS < 32 ? v0 % 32 : 0) : 0;
            if (left > 0 && left < 32) w &= (1u << left) - 1;
            if (TOKENS < 32) w &= (1u << TOKENS % 32) - 1;
            words[range][m][j] = w;
            if (w) atomicOr(&need[range][j], w);                             // the same in any order
        }
        __syncthreads();
        int start[RANGES + 1];
        start[0] = 0;
#pragma unroll
        for (int range = 0; range < RANGES; range++) {
            start[range + 1] = start[range];
#pragma unroll
            for (int j = 0; j < WORDS; j++) {
                const uint32_t w = need[range][j];
                if (tid < TOKENS && tid / 32 == j && ((w >> (tid % 32)) & 1)) list[start[range + 1] + __popc(w & ((1u << (tid % 32)) - 1))] = (uint16_t)(range * TOKENS + tid);
                start[range + 1] += __popc(w);
            }
            start[range + 1] = __builtin_amdgcn_readfirstlane(start[range + 1]);
        }
        __syncthreads();
        if (TOKENS == 16 || start[RANGES] <= Lds::SHORT) {
#pragma unroll
            for (int range = 0; range < RANGES; range++) if (first_of(range) < a.V) store_range(first_of(range), nullptr);
            for (int i = 0; i < start[RANGES]; i += 16) short_form(i, start[RANGES] - i < 16 ? start[RANGES] - i : 16);
        } else {
            for (int range = 0; range < RANGES; range++) {
                const int32_t v0 = first_of(range);
                if (v0 >= a.V) break;
                int from = 0, to = 0;
#pragma unroll
                for (int i = 0; i < RANGES; i++) if (i == range) { from = start[i]; to = start[i + 1]; }
                if (to - from > Lds::SHORT) {
                    if constexpr (TOKENS > 16) long_form(v0, from, to - from);
                    continue;
                }
                store_range(v0, nullptr);
                for (int i = from; i < to; i += 16) short_form(i, to - i < 16 ? to - i : 16);
            }
        }
        __syncthreads();                                                     // before the lists are made again
    }
}

// ---- many rows: tiles of both operands in LDS ----
//
// A workgroup of eight wavefronts takes tiles of 64 MI tokens and 32 MJ rows of the batch, one after the other, a wavefront 16 MI tokens and 16 MJ rows.  A block of columns of both
// operands, 128 bytes a row, comes from memory straight into LDS while the block before is multiplied, the next tile's first one while this one's last is: two buffers, one
// barrier a block, pieces in places as above.  While sixteen rows' products run the sixteen before them are scaled and added.
//   2,048 x 128,256 x 4,096 bf16: 1,040 to 1,080 us, 2.0 PFLOP/s.  The matrix units are busy for 51 % of it, the other vector instructions (the scales, mostly) would be for 30 %
// by themselves, LDS for 25 %; a third of the wavefronts' time is waits for blocks and at barriers (the chip runs at 1.9 GHz meanwhile, of 2.4).  fp32 logits, 2,048 x 32,000 x 4,096: 488 us, 1.1 PFLOP/s, half
// of the bf16 instructions' rate and the operands' conversion beside them.
//   Under a mask a tile is computed whole.  That is right where the rows together allow most ranges (half of the tokens each, 128,256 x 4,096 bf16: 65 rows 143 us, in calls of 64 rows 174; 130 rows 157
// and 314), and far from it where they allow few: 50 tokens a row 65 rows 150 us, in calls of 64 rows 37, 130 rows 165 and 66, 256 rows 187 and 128.
//   Rows behind the last one are the last one again; their results are not stored.
template <int MJ, int MI, typename ElemT>
struct TileLds {
    static constexpr int ROWS = 32 * MJ, TOKENS = 64 * MI, W_BYTES = TOKENS * SCALE_BLOCK, X_BYTES = ROWS * SCALE_BLOCK, BUFFER = W_BYTES + X_BYTES;
    static constexpr int SCALES = 2 * BUFFER, OUT = SCALES + 2 * 512 * 4, PITCH = 16 * MI * sizeof(ElemT) + 16, BYTES = OUT + 8 * 16 * PITCH;
};

template <int MJ, int MI, bool MASK, typename ElemT>
__global__ __launch_bounds__(512, 2) void head_tile_kernel(HeadArgs a, int32_t tiles_m, int32_t n_tiles) {
    typedef TileLds<MJ, MI, ElemT> Lds;
    constexpr int LOADS = MI + MJ / 2;                                       // of a wavefront for a block: eight rows each, 8 MI of the weight, 4 MJ of the activations
    constexpr bool SPLIT = Lds::TOKENS % SCALE_BLOCK != 0;                   // tiles begin in the middle of 128 tokens, and wavefronts have some of both
    extern __shared__ __align__(16) uint8_t mem[];
    const int tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64), wv = wave % 4, wm = wave / 4;
    const int32_t n_k = a.K / SCALE_BLOCK, n_vb = (a.V + SCALE_BLOCK - 1) / SCALE_BLOCK, W = (a.V + 31) / 32;
    // workgroups go to the eight XCDs in turn: an XCD takes consecutive tiles, those of the same tokens one after the other, so that its L2 has a weight's rows once
    const int32_t per = n_tiles / 8, over = n_tiles % 8, xcd = blockIdx.x % 8, stride = (gridDim.x - xcd + 7) / 8;
    const int32_t end = (xcd + 1) * per + (xcd < over ? xcd + 1 : over);
    int32_t tile = xcd * per + (xcd < over ? xcd : over) + blockIdx.x / 8;
    if (tile >= end) return;
    const uint8_t *w0, *x0;                                                  // of the tile that is being brought
    uint32_t off[LOADS];                                                     // the host checks that a tile's rows lie within 32 bits
    const float *xs, *ws;                                                    // a thread's scales: of one row, and of the weight's first or second 128 tokens (the threads behind these two have them once more)
    auto aim = [&](int32_t t) {
        const int32_t v0 = t / tiles_m * Lds::TOKENS, m0 = t % tiles_m * Lds::ROWS;
        w0 = a.w + (int64_t)v0 * a.w_stride;
        x0 = a.x + (int64_t)m0 * a.x_stride;
#pragma unroll
        for (int i = 0; i < LOADS; i++) {
            const int32_t r = (i < MI ? wave * MI + i : wave * (MJ / 2) + i - MI) * 8 + lane / 8, left = i < MI ? a.V - v0 : a.M - m0;
            off[i] = (uint32_t)(r < left ? r : left - 1) * (uint32_t)(i < MI ? a.w_stride : a.x_stride) + (lane % 8 ^ lane / 8) * 16;
        }
        const int32_t row = m0 + tid % Lds::ROWS, vb = v0 / SCALE_BLOCK + tid / Lds::ROWS % 2;
        xs = a.xs + (size_t)(row < a.M ? row : a.M - 1) * n_k;
        ws = a.ws + (size_t)(vb < n_vb ? vb : n_vb - 1) * n_k;
    };
    auto fetch = [&](int32_t k, int b) {
#pragma unroll
        for (int i = 0; i < LOADS; i++)
            to_lds((i < MI ? w0 : x0) + (size_t)k * SCALE_BLOCK, off[i], lds_at(mem) + b * Lds::BUFFER + (i < MI ? (wave * MI + i) * 8 * SCALE_BLOCK : Lds::W_BYTES + (wave * (MJ / 2) + i - MI) * 8 * SCALE_BLOCK));
    };
    float *const scales = reinterpret_cast<float *>(mem + Lds::SCALES);
    uint8_t *const own = mem + Lds::OUT + wave * (16 * Lds::PITCH);
    const int32_t c0 = (lane / 16 ^ lane % 8) * 16, c1 = ((lane / 16 + 4) ^ lane % 8) * 16;   // the lane's two pieces of a row that is lane % 8 modulo 8
    aim(tile);
    scales[tid] = xs[0] * ws[0];
    fetch(0, 0);
    arrived<0>();
    __syncthreads();
    int b = 0;
    for (; tile < end; tile += stride) {
        const int second = (SCALE_BLOCK - tile / tiles_m * Lds::TOKENS % SCALE_BLOCK - wv * 16 * MI) / 16;   // sixteens of the wavefront before the second 128 tokens (or none)
        f32x4 acc[MJ][MI];
#pragma unroll
        for (int j = 0; j < MJ; j++)
#pragma unroll
            for (int i = 0; i < MI; i++) acc[j][i] = f32x4{0, 0, 0, 0};
        for (int32_t k = 0; k < n_k; k++, b ^= 1) {
            int32_t k_next = k + 1;
            if (k_next == n_k) {                                             // behind the last block: the next tile's first (behind the last tile: this one's, which nobody reads)
                k_next = 0;
                if (tile + stride < end) aim(tile + stride);
            }
            const float next_x = xs[k_next], next_w = ws[k_next];
            const uint8_t *const w_at = mem + b * Lds::BUFFER + (wv * 16 * MI + lane % 16) * SCALE_BLOCK;
            const uint8_t *const x_at = mem + b * Lds::BUFFER + Lds::W_BYTES + (wm * 16 * MJ + lane % 16) * SCALE_BLOCK;
            const float *const s_at = scales + b * 512 + (SPLIT ? 0 : wv * 16 * MI / SCALE_BLOCK) * Lds::ROWS + wm * 16 * MJ + lane % 16;
            Operand<ElemT> w[MI];
#pragma unroll
            for (int i = 0; i < MI; i++) w[i].take(piece_at(w_at + i * 16 * SCALE_BLOCK + c0), piece_at(w_at + i * 16 * SCALE_BLOCK + c1));
            f32x4 part[MI][1], last[MI];
            float s[2] = {0.0f, 0.0f}, s_last[2] = {0.0f, 0.0f};             // of the weight's first and second 128 tokens, where a wavefront may have some of both
            Operand<ElemT> x[1], x_next;
            x_next.take(piece_at(x_at + c0), piece_at(x_at + c1));
#pragma unroll
            for (int j = 0; j <= MJ; j++) {
                if (j < MJ) {
                    x[0] = x_next;
                    s[0] = s_at[j * 16];
                    if (SPLIT) s[1] = s_at[Lds::ROWS + j * 16];
                    if (j + 1 < MJ) x_next.take(piece_at(x_at + (j + 1) * 16 * SCALE_BLOCK + c0), piece_at(x_at + (j + 1) * 16 * SCALE_BLOCK + c1));
                    multiply(w, x, part);
                    if (j == 0) fetch(k_next, b ^ 1);                        // behind the reads that the first products wait for
                }
#pragma unroll
                for (int i = 0; i < MI; i++) {
                    if (j > 0)
#pragma unroll
                        for (int e = 0; e < 4; e++) acc[j - 1][i][e] = fmaf(SPLIT && i >= second ? s_last[1] : s_last[0], last[i][e], acc[j - 1][i][e]);
                    last[i] = part[i][0];
                }
                s_last[0] = s[0];
                if (SPLIT) s_last[1] = s[1];
                if (j > 0 && j < MJ)
#pragma unroll
                    for (int i = 0; i < MI; i++) {                            // a product, four sums, a product, ...
                        __builtin_amdgcn_sched_group_barrier(0x8, Operand<ElemT>::STEPS, 0);
                        __builtin_amdgcn_sched_group_barrier(0x2, 4, 0);
                    }
                __builtin_amdgcn_sched_barrier(0);
            }
            scales[(b ^ 1) * 512 + tid] = next_x * next_w;
            arrived<0>();
            __syncthreads();
        }
        // sixteen rows at a time through the wavefront's own part of LDS, from four tokens a lane to whole lines of 64 tokens
        constexpr int EPV = 16 / sizeof(ElemT), PIECES = 16 * MI / EPV;
        const int32_t v_w = tile / tiles_m * Lds::TOKENS + wv * 16 * MI, m_w = tile % tiles_m * Lds::ROWS + wm * 16 * MJ;
#pragma unroll
        for (int j = 0; j < MJ; j++) {
#pragma unroll
            for (int i = 0; i < MI; i++) {
                union { ElemT e[4]; uint64_t q; u32x4 v; } o;
#pragma unroll
                for (int e = 0; e < 4; e++) o.e[e] = sizeof(ElemT) == 4 ? (ElemT)__float_as_uint(acc[j][i][e]) : (ElemT)bf16_of(acc[j][i][e]);
                uint8_t *const to = own + lane % 16 * Lds::PITCH + (i * 16 + lane / 16 * 4) * sizeof(ElemT);
                if (sizeof(ElemT) == 4) *reinterpret_cast<u32x4 *>(to) = o.v;
                else *reinterpret_cast<uint64_t *>(to) = o.q;
            }
            in_turn();
#pragma unroll
            for (int i = 0; i < (16 * PIECES + 63) / 64; i++) {
                if (16 * PIECES % 64 && i * 64 + lane >= 16 * PIECES) continue;
                const int r = (i * 64 + lane) / PIECES, p = (i * 64 + lane) % PIECES;
                const int32_t m = m_w + j * 16 + r, v = v_w + p * EPV;
                union { ElemT e[EPV]; u32x4 v; } o;
                o.v = *reinterpret_cast<const u32x4 *>(own + r * Lds::PITCH + p * 16);
                if (m >= a.M || v >= a.V) continue;
                if (MASK) {
                    const uint32_t bits = a.mask[(size_t)m * W + (v >> 5)] >> (v & 31);
#pragma unroll
                    for (int e = 0; e < EPV; e++) if (!((bits >> e) & 1)) o.e[e] = sizeof(ElemT) == 4 ? (ElemT)0xFF800000u : (ElemT)0xFF80u;
                }
                ElemT *const to = (ElemT *)a.y + (int64_t)m * a.y_stride + v;
                if (v + EPV <= a.V) *reinterpret_cast<typename Piece<ElemT>::type *>(to) = o.v;
                else {
#pragma unroll
                    for (int e = 0; e < EPV; e++) if (v + e < a.V) to[e] = o.e[e];
                }
            }
            in_turn();
        }
    }
}

// LDS beyond 64 KB has to be allowed for a kernel, once on every device.
hipError_t allow_lds(const void *kernel, int bytes, std::atomic<uint64_t> &allowed) {
    int device = 0;
    hipError_t e = hipGetDevice(&device);
    if (e != hipSuccess) return e;
    const uint64_t bit = device < 64 ? 1ull << device : 0;
    if (bit && (allowed.load(std::memory_order_relaxed) & bit)) return hipSuccess;
    e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == hipSuccess) allowed.fetch_or(bit, std::memory_order_relaxed);
    return e;
}

template <int MJ, int MI, bool MASK, typename ElemT>
hipError_t head_tile(const HeadArgs &a, hipStream_t s) {
    typedef TileLds<MJ, MI, ElemT> Lds;
    static std::atomic<uint64_t> allowed{0};
    const hipError_t e = allow_lds((const void *)head_tile_kernel<MJ, MI, MASK, ElemT>, Lds::BYTES, allowed);
    if (e != hipSuccess) return e;
    const int32_t tiles_m = (a.M + Lds::ROWS - 1) / Lds::ROWS;
    const int64_t n = (int64_t)tiles_m * ((a.V + Lds::TOKENS - 1) / Lds::TOKENS);
    hipLaunchKernelGGL((head_tile_kernel<MJ, MI, MASK, ElemT>), dim3((uint32_t)std::min<int64_t>(n, COMPUTE_UNITS)), dim3(512), Lds::BYTES, s, a, tiles_m, (int32_t)n);
    return hipSuccess;
}

template <int MJ, bool MASK, typename ElemT>
hipError_t head_tile_of(const HeadArgs &a, int tokens, hipStream_t s) {
    return tokens == 256 ? head_tile<MJ, 4, MASK, ElemT>(a, s) : tokens == 192 ? head_tile<MJ, 3, MASK, ElemT>(a, s) : head_tile<MJ, 2, MASK, ElemT>(a, s);
}

template <int MT, int TOKENS, bool MASK, typename ElemT>
hipError_t head_rows(const HeadArgs &a, hipStream_t s) {
    typedef RowsLds<MT, TOKENS, MASK> Lds;
    static std::atomic<uint64_t> allowed{0};
    const hipError_t e = allow_lds((const void *)head_rows_kernel<MT, TOKENS, MASK, ElemT>, Lds::BYTES, allowed);
    if (e != hipSuccess) return e;
    // Without a mask a workgroup a range.  With one as many as the compute units hold, so that those with little to do in a range have several.
    const int32_t n = (a.V + TOKENS - 1) / TOKENS;
    const dim3 grid(Lds::RANGES > 1 ? std::min(n, 2 * COMPUTE_UNITS) : n, (a.M + MT * 16 - 1) / (MT * 16));
    hipLaunchKernelGGL((head_rows_kernel<MT, TOKENS, MASK, ElemT>), grid, dim3(256), Lds::BYTES, s, a, n);
    return hipSuccess;
}
// Ranges of 16 tokens where those of 128 would leave three compute units of four idle (one row x 2,048 x 1,024: 4.2 us, 6.0 in ranges of 128; 64 rows x 8,192 x 1,024: 10.1 and 9.2).
// Ranges of 64 where each finds a compute unit of its own (bf16, x 4,096: 8 rows x 9,000 12.4 us, in ranges of 128 16.0; 8 x 16,384 15.1 and 18.5; 64 x 10,000 19.2 and 25.0; 64 x 16,000 under
// masks 24.4 and 32.7; of short rows some lose a little, 8 x 16,384 x 512 5.2 and 4.9, others win, 64 rows 6.8 and 7.4), not where some find one and others share (8 x 20,000: x 4,096 22.8 and
// 19.7, x 1,024 8.3 and 6.6).
template <int MT, bool MASK, typename ElemT>
hipError_t head_few(const HeadArgs &a, hipStream_t s) {
    const int32_t n = (a.V + 63) / 64;                                       // ranges of 64
    if (n < 128) return head_rows<MT, 16, MASK, ElemT>(a, s);
    if (n <= COMPUTE_UNITS) return head_rows<MT, 64, MASK, ElemT>(a, s);
    return head_rows<MT, 128, MASK, ElemT>(a, s);
}
template <bool MASK, typename ElemT>
hipError_t head(const HeadArgs &a, hipStream_t s) {
    if (a.M <= 16) return head_few<1, MASK, ElemT>(a, s);
    if (a.M <= 32) return head_few<2, MASK, ElemT>(a, s);
    if (a.M <= 64) return head_few<4, MASK, ElemT>(a, s);
    if ((a.w_stride | a.x_stride) >= (1 << 24)) return head_rows<4, 128, MASK, ElemT>(a, s);   // a tile's rows would not lie within 32 bits
    // Tiles of 128, 192 or 256 rows (operands in bf16 take twice the registers: 128) and as many tokens, whichever are done first: tiles that a compute unit has, a tile's work and 64 more
    // in each direction for what it costs whatever its size; smaller ones have to promise a twentieth (1,030 x 32,000 x 4,096 fp32 283 us, with 192 tokens 289).  With 256 tokens alone and
    // so: 70 x 32,000 x 1,024 bf16 16.9 and 13.4 us, fp32 20.5 and 15.7; 130 x 32,000 x 4,096 bf16 58.3 and 47.0; 256 rows 65.0 and 57.5; 100 x 8,192 x 2,048 18.3 and 14.7; 300 x 32,000 x 4,096
    // fp32 116 and 102.
    int rows = 128, tokens = 256;
    int64_t least = INT64_MAX;
    for (int r = sizeof(ElemT) == 2 ? 256 : 128; r >= 128; r -= 64)
        for (int t = 256; t >= 128; t -= 64) {
            const int64_t tiles = (int64_t)((a.M + r - 1) / r) * ((a.V + t - 1) / t), cost = (tiles + COMPUTE_UNITS - 1) / COMPUTE_UNITS * (r + 64) * (t + 64);
            if (least == INT64_MAX || cost * 20 < least * 19) least = cost, rows = r, tokens = t;
        }
    if constexpr (sizeof(ElemT) == 2) {
        if (rows == 256) return head_tile_of<8, MASK, ElemT>(a, tokens, s);
        if (rows == 192) return head_tile_of<6, MASK, ElemT>(a, tokens, s);
    }
    return head_tile_of<4, MASK, ElemT>(a, tokens, s);
}

template <typename ElemT>
void quantize(const ElemT *x, int64_t rows, int32_t cols, int64_t stride, int32_t block_rows, uint8_t *q, float *scale, hipStream_t s) {
    const int32_t n_blocks = (cols + SCALE_BLOCK - 1) / SCALE_BLOCK;
    if (block_rows == 1) {
        // Two blocks of bf16 at once, 32 bytes of a lane as fp32's one, when there are more blocks than the chip holds lanes for (32,000 x 4,096 bf16: 72 us, one at a time
        // 76; 16 x 4,096: 3.4 and 2.9; two of fp32 116 instead of 110).
        const int n = sizeof(ElemT) == 2 && rows * n_blocks > 16 * 8 * COMPUTE_UNITS ? 2 : 1;
        hipLaunchKernelGGL((n == 2 ? quantize_rows_kernel<sizeof(ElemT) == 2 ? 2 : 1, ElemT> : quantize_rows_kernel<1, ElemT>),
                           dim3((uint32_t)std::min<int64_t>((rows * n_blocks + 16 * n - 1) / (16 * n), BLOCKS_MAX)), dim3(256), 0, s, x, stride, rows, cols, n_blocks, q, scale);
    }
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
    const hipError_t e = a.mask ? (a.dtype == 0 ? head<true, uint32_t>(a, s) : head<true, uint16_t>(a, s)) : (a.dtype == 0 ? head<false, uint32_t>(a, s) : head<false, uint16_t>(a, s));
    return e != hipSuccess ? e : hipGetLastError();
}

}  // namespace zf
