// Log probabilities of given tokens under a mask, with entropy and alternatives, and their gradient.
//
// Of a row's allowed logits x, with c = log2(e) / temperature, m their largest and z = x c - m c:
//   S = sum 2^z,  T = sum 2^z z
//   logprob of t = (x_t - m) / temperature - ln S        entropy = ln S - ln 2 T / S
//   d logits_v = 1 / temperature (p_v (-G - g_H (ln p_v + H)) + sum of g_j where token j is v),   G = sum of all g_j
// All of it is held in 32 bits, and sums that were taken around another m join by the factor 2^(m' c - m c).  z is one fused multiply-add to the rounded
// product R = m c: as a reference any number near it does, so long as everything that is compared was taken against the same, and all who need it
// work it out from m.  Far out, where m c - R would be more than a sixteenth (or R infinite: logits at the type's lowest value that a program masked with), z is (x - m) c.
//   A row is read once, in segments, a workgroup each; a second launch joins a row's segments and looks its given tokens up.
#include <hip/hip_runtime.h>
#include <algorithm>
#include <cfloat>
#include "zf_ops.h"

namespace zf {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
template <typename ElemT> struct Piece;       // 16 bytes at any multiple of an element: the memory system takes them there
template <> struct Piece<uint32_t> { typedef u32x4 type __attribute__((aligned(4))); };
template <> struct Piece<uint16_t> { typedef u32x4 type __attribute__((aligned(2))); };

static const float LOG2_E = 1.44269504088896340736f, LN_2 = 0.69314718055994530942f;
static const int THREADS = 256, ROWS_JOINED = 4;  // rows a workgroup of the joining kernel takes, a wavefront each
static const int PIECES = 4;                                             // 16-byte pieces of a segment that a thread holds; one where that leaves the chip half empty

struct Part { float m, S, T, pad; };          // of one segment of a row
// What is largest first, among equals the lowest token: the logit's bits in the order of their values, then the token's complement.  0: none.
typedef unsigned long long Key;

struct LogprobsArgs {
    zf_logprobs_args a;
    int32_t W, n_seg;
    float c, inv_t;                            // log2(e) / temperature, 1 / temperature
    Part *parts;                               // [rows][n_seg]
    Key *keys;                                 // [rows][n_seg][top]
};
struct GradArgs {
    LogprobsArgs l;
    LogprobsGrad g;
};

__device__ __forceinline__ float of_bits(uint32_t x) { return __uint_as_float(x); }
__device__ __forceinline__ float of_bits(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
// What z is taken against.
struct Reference {
    float m, R, c;
    bool far;                                  // the reference is m c itself, not R
    __device__ __forceinline__ Reference(float m_, float c_) : m(m_), R(m_ * c_), c(c_), far(!(fabsf(R) < 0x1p20f)) {}
};
__device__ __forceinline__ uint32_t in_order(float x) {                  // bits that compare as the values do; NaN and -inf: 0
    const uint32_t u = __float_as_uint(x + 0.0f);
    return x > -INFINITY ? u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u) : 0u;
}
__device__ __forceinline__ Key key_of(float x, uint32_t v) {
    const uint32_t o = in_order(x);
    return o ? (Key)o << 32 | (uint32_t)~v : 0;
}
__device__ __forceinline__ float logit_of(Key k) {
    const uint32_t o = (uint32_t)(k >> 32);
    return __uint_as_float(o ^ ((o >> 31) ? 0x80000000u : 0xFFFFFFFFu));
}
// Over a wavefront, to all lanes, by moves between lanes of 1, 2, 4, 8, 16 and 32; sums in this order, whatever the timing.
template <int CTRL, int ROWS = 0xF> __device__ __forceinline__ uint32_t moved(uint32_t none, uint32_t x) { return (uint32_t)__builtin_amdgcn_update_dpp((int)none, (int)x, CTRL, ROWS, 0xF, false); }
template <class F>
__device__ __forceinline__ uint32_t over_wave(uint32_t x, uint32_t none, F f) {
    x = f(x, moved<0x111>(none, x));           // the lane one below, of the same sixteen
    x = f(x, moved<0x112>(none, x));
    x = f(x, moved<0x114>(none, x));
    x = f(x, moved<0x118>(none, x));
    x = f(x, moved<0x142, 0xA>(none, x));      // lane 15 of each sixteen to the next
    x = f(x, moved<0x143, 0xC>(none, x));      // lane 31 to the upper half
    return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}
__device__ __forceinline__ float wave_max(float x) {
    return __uint_as_float(over_wave(__float_as_uint(x), 0xFF800000u, [](uint32_t a, uint32_t b) { return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b))); }));
}
__device__ __forceinline__ float wave_sum(float x) {
    return __uint_as_float(over_wave(__float_as_uint(x), 0u, [](uint32_t a, uint32_t b) { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); }));
}
__device__ __forceinline__ uint32_t wave_max(uint32_t x) { return over_wave(x, 0u, [](uint32_t a, uint32_t b) { return a > b ? a : b; }); }
__device__ __forceinline__ Key wave_max(Key k) {
    const uint32_t high = wave_max((uint32_t)(k >> 32));
    return (Key)high << 32 | wave_max((uint32_t)(k >> 32) == high ? (uint32_t)k : 0u);
}
__device__ __forceinline__ int four_sum(int x) {           // over four neighbouring lanes, to all of them
    x += (int)moved<0xB1>(0, x);                           // lanes 1 0 3 2 of each four
    return x + (int)moved<0x4E>(0, x);                     // lanes 2 3 0 1
}
__device__ __forceinline__ int sum_up_to(int x) {          // of sixteen lanes, each with those below it
    x += (int)moved<0x111>(0, x);
    x += (int)moved<0x112>(0, x);
    x += (int)moved<0x114>(0, x);
    return x + (int)moved<0x118>(0, x);
}
__device__ __forceinline__ float two_to(float x) { return __builtin_amdgcn_exp2f(x); }   // below 2^-126 nothing
// How far the reference of a part lies below the whole's: nothing times -inf is nothing, so -inf is a large number here.
__device__ __forceinline__ float below(float m, const Reference &whole) {
    if (m == whole.m) return 0.0f;
    const Reference part(m, whole.c);
    const float d = part.far ? (whole.far ? (m - whole.m) * whole.c : fmaf(m, whole.c, -whole.R)) : whole.far ? -fmaf(whole.m, whole.c, -part.R) : part.R - whole.R;
    return fmaxf(d, -1e4f);
}
// b joins a.  A side without anything has m = -inf and sums of zero (or NaN, where it has nothing but NaN).
__device__ __forceinline__ void join(Part &a, const Part &b, float c) {
    const Reference whole(fmaxf(a.m, b.m), c);
    const float da = below(a.m, whole), db = below(b.m, whole), fa = two_to(da), fb = two_to(db);
    a.T = fa * (a.T + a.S * da) + fb * (b.T + b.S * db);
    a.S = fa * a.S + fb * b.S;
    a.m = whole.m;
}
// The parts that the lanes of a wavefront hold (m = -inf, S = T = 0 in the others), joined, and what follows from the whole of a row.
struct RowEnd {
    Reference ref;
    float S, T, log2_S, ln_S;                  // ln_S: of the sum around m itself
    bool nothing;
    __device__ __forceinline__ RowEnd() : ref(0.0f, 0.0f) {}
    __device__ __forceinline__ RowEnd(const Part &mine, float c) : ref(wave_max(mine.m), c) {
        const float d = below(mine.m, ref), f = two_to(d);
        T = wave_sum(f * (mine.T + mine.S * d));
        S = wave_sum(f * mine.S);
        nothing = ref.m == -INFINITY && S == 0.0f;
        log2_S = nothing ? 0.0f : log2f(S);
        ln_S = LN_2 * (ref.far ? log2_S : log2_S - fmaf(ref.m, ref.c, -ref.R));
    }
    __device__ __forceinline__ float entropy() const { return nothing ? 0.0f : LN_2 * (log2_S - T / S); }
    // A finite logit has a finite log probability (the type's lowest value divided by a temperature below one is beyond 32 bits).
    __device__ __forceinline__ float logprob(float x, float temperature) const {
        const float lp = (x - ref.m) / temperature - ln_S;
        return lp < -FLT_MAX && x > -INFINITY ? -FLT_MAX : lp;
    }
    // Of a given token whose logit is x, -inf where the mask does not allow it.
    __device__ __forceinline__ float given(int64_t t, float x, const zf_logprobs_args &a) const {
        return t >= a.V ? NAN : t < 0 ? 0.0f : S != S ? S : x == -INFINITY ? -INFINITY : logprob(x, a.temperature);
    }
    __device__ __forceinline__ void store_row(const zf_logprobs_args &a, int64_t row) const {
        if (a.entropy) a.entropy[row] = entropy();
        if (a.stats) { a.stats[2 * row] = ref.m; a.stats[2 * row + 1] = log2_S; }
    }
    __device__ __forceinline__ void store_top(const zf_logprobs_args &a, int64_t row, int i, Key k) const {
        a.top_ids[row * a.top + i] = k ? (int32_t)~(uint32_t)k : -1;
        a.top_logprobs[row * a.top + i] = k ? logprob(logit_of(k), a.temperature) : -INFINITY;
    }
};
__device__ __forceinline__ bool allowed(const uint32_t *mask, int64_t row, int32_t W, uint32_t v) {
    return !mask || ((mask[row * W + (v >> 5)] >> (v & 31)) & 1u);
}

// A row's given token j: the token, and its logit (-inf where the mask does not allow it, or there is none such).
template <typename ElemT>
__device__ __forceinline__ void look_up(const LogprobsArgs &A, int64_t row, int j, int64_t *t, float *x) {
    const int64_t at = row * A.a.n_tokens + j;
    *t = A.a.token_bytes == 8 ? ((const int64_t *)A.a.tokens)[at] : ((const int32_t *)A.a.tokens)[at];
    *x = -INFINITY;
    if (*t >= 0 && *t < A.a.V) {
        const float logit = of_bits(((const ElemT *)A.a.logits)[row * A.a.row_stride_elems + *t]);
        if (allowed(A.a.mask, row, A.W, (uint32_t)*t)) *x = logit;
    }
}

// A thread's pieces of a row's segment, PIECES at a distance of THREADS pieces from token v on: their logits, -inf where there is no token or none that is
// allowed.  `whole`: the segment ends before the row does.  All loads are issued before the first is looked at.
template <int THREADS, int PIECES, int EPV, bool ONCE, typename ElemT>
__device__ __forceinline__ void load_pieces(const ElemT *row, const uint32_t *mask_row, int32_t v, int32_t V, bool whole, float (&x)[PIECES][EPV]) {
    constexpr uint32_t FULL = (1u << EPV) - 1u;
    u32x4 raw[PIECES];
    uint32_t bits[PIECES];
#pragma unroll
    for (int p = 0; p < PIECES; p++) {
        const int32_t at = v + p * (THREADS * EPV), left = V - at;
        bits[p] = FULL;
        const typename Piece<ElemT>::type *const from = reinterpret_cast<const typename Piece<ElemT>::type *>(row + at);
        if (whole || left >= EPV) raw[p] = ONCE ? __builtin_nontemporal_load(from) : *from;
        else {
            bits[p] = left > 0 ? (1u << left) - 1u : 0u;
            union { u32x4 v; ElemT e[EPV]; } o;
            o.v = u32x4{0, 0, 0, 0};
#pragma unroll
            for (int k = 0; k < EPV; k++) if (k < left) o.e[k] = row[at + k];
            raw[p] = o.v;
        }
        if (mask_row && (whole || left > 0)) bits[p] &= mask_row[at >> 5] >> (at & 31);
    }
#pragma unroll
    for (int p = 0; p < PIECES; p++) {
#pragma unroll
        for (int k = 0; k < EPV; k++) x[p][k] = __uint_as_float(sizeof(ElemT) == 4 ? raw[p][k] : k & 1 ? raw[p][k / 2] & 0xFFFF0000u : raw[p][k / 2] << 16);
        if (__any(bits[p] != FULL)) {
#pragma unroll
            for (int k = 0; k < EPV; k++) {
                const uint32_t yes = (uint32_t)__builtin_amdgcn_sbfe((int)bits[p], k, 1);
                x[p][k] = __uint_as_float((__float_as_uint(x[p][k]) & yes) | (0xFF800000u & ~yes));
            }
        }
    }
}

// The `top` largest of many keys.  A line is found that at least `top` of them reach (the upper sixteen bits of the `top`-th largest, a bit a step, with a
// ballot), what reaches it is listed -- little else does -- and a listed key's rank is the number of keys above it.  A list that overflows (many equal
// logits) is left to the caller, which takes the keys one by one, each the largest below the last.
static const int LISTED = 128;                             // keys that a wavefront lists

// The largest multiples of 2^16 that so many lanes reach, but at least 1 (0 stands for no logit).
template <int N>
__device__ __forceinline__ void lines_of(uint32_t o, const int (&lanes)[N], uint32_t (&line)[N]) {
#pragma unroll
    for (int i = 0; i < N; i++) line[i] = 0;
#pragma unroll
    for (int bit = 31; bit >= 16; bit--) {
#pragma unroll
        for (int i = 0; i < N; i++) {
            const uint32_t up = line[i] | 1u << bit;
            if (__popcll(__ballot(o >= up)) >= lanes[i]) line[i] = up;
        }
    }
#pragma unroll
    for (int i = 0; i < N; i++) line[i] = line[i] ? line[i] : 1;
}
// How many of a list's keys are above `mine`, which four neighbouring lanes have: each looks at a quarter of the list, which is padded with 32 zeros.
__device__ __forceinline__ int rank_of(Key mine, const Key *list, int n, int lane) {
    int rank = 0;
    for (int j = lane % 4; j < n; j += 32) {
#pragma unroll
        for (int u = 0; u < 8; u++) rank += list[j + 4 * u] > mine;
    }
    return four_sum(rank);
}

// A segment of a row, or (n_seg = 1) the whole of it, to the end.
//   Large inputs are bound by memory: 4,096 x 128,256 bf16 with entropy 179 us in a row of such calls (5.9 TB/s), 161 to 223 one by one under a trace, 202 at the median; 1,030 x 40,037 bf16 at odd
// elements 15.6 (5.3).  Alternatives are not hidden behind the memory's time: with 20 of them the former takes 314, the latter with the joining launch 34 (with 5 31, with 64 48, without 19), 2,048 x 32,000 bf16 under masks 78 (without
// 35).  Small inputs are bound by
// what follows in turn: 64 x 128,256 bf16 6.0 us without alternatives, of which 2.7 are its bytes; with 20 of them 10.5, with 64 12.3; one row of 32,000 fp32 4.5 without, with 5 7.0, with 64 8.2
// (of the 2.5 a fifth is the lines, a half the lists and the waits for the slowest wavefront's, the rest ranks and stores); 64 x 32,000 bf16 5.1, with 20 9.0.
template <int THREADS, int PIECES, bool ONCE, bool ENT, bool TOP, typename ElemT>
__global__ __launch_bounds__(THREADS) void logprobs_part_kernel(LogprobsArgs A) {
    constexpr int EPV = 16 / sizeof(ElemT), WAVES = THREADS / 64;
    __shared__ Part part[WAVES];
    __shared__ Key best[WAVES];
    __shared__ Key listed[TOP ? WAVES : 1][LISTED], all[TOP ? WAVES * LISTED + 32 : 1];
    __shared__ uint32_t lines[2][WAVES];
    __shared__ int n_listed[WAVES];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / 64), lane = tid % 64;
    const int64_t row = blockIdx.x / (uint32_t)A.n_seg;
    const int32_t seg = blockIdx.x % (uint32_t)A.n_seg, V = A.a.V, v0 = seg * (THREADS * PIECES * EPV) + tid * EPV;
    const ElemT *const logits = (const ElemT *)A.a.logits + row * A.a.row_stride_elems;
    const uint32_t *const mask = A.a.mask ? A.a.mask + row * A.W : nullptr;
    float x[PIECES][EPV], most = -INFINITY;
    load_pieces<THREADS, PIECES, EPV, ONCE>(logits, mask, v0, V, (seg + 1) * (THREADS * PIECES * EPV) <= V, x);
    const bool row_ends = A.n_seg == 1;                    // here; the last wavefront looks the given tokens up
    int64_t given = -1;
    float given_x = -INFINITY;
    if (row_ends && wave == WAVES - 1 && lane < A.a.n_tokens) look_up<ElemT>(A, row, lane, &given, &given_x);
#pragma unroll
    for (int p = 0; p < PIECES; p++)
#pragma unroll
        for (int k = 0; k < EPV; k++) most = fmaxf(most, x[p][k]);
    const float m = wave_max(most);
    const Reference ref(m, A.c);
    float S = 0.0f, T = 0.0f;
    if (!ref.far) {
#pragma unroll
        for (int p = 0; p < PIECES; p++)
#pragma unroll
            for (int k = 0; k < EPV; k++) {
                const float z = fmaf(x[p][k], ref.c, -ref.R), e = two_to(z);
                S += e;
                if (ENT) T = fmaf(e, fmaxf(z, -1e4f), T);  // nothing times -inf is nothing
            }
    } else if (m > -INFINITY) {
#pragma unroll
        for (int p = 0; p < PIECES; p++)
#pragma unroll
            for (int k = 0; k < EPV; k++) {
                const float z = (x[p][k] - m) * ref.c, e = two_to(z);
                S += e;
                if (ENT) T = fmaf(e, fmaxf(z, -1e4f), T);
            }
    } else {
#pragma unroll
        for (int p = 0; p < PIECES; p++)
#pragma unroll
            for (int k = 0; k < EPV; k++) if (x[p][k] != x[p][k]) S = T = x[p][k];
    }
    S = wave_sum(S);
    if (ENT) T = wave_sum(T);
    if (tid % 64 == 0) part[wave] = Part{m, S, T, 0.0f};
    if (TOP) {
        const uint32_t mine = in_order(most);              // as many lanes as reach a line have a logit that does
        uint32_t line[2];
        lines_of<2>(mine, {A.a.top, (A.a.top + WAVES - 1) / WAVES}, line);
        if (lane < 2) lines[lane][wave] = lane ? line[1] : line[0];
    }
    __syncthreads();
    const Part mine = lane < WAVES ? part[lane] : Part{-INFINITY, 0.0f, 0.0f, 0.0f};
    auto finish = [&](const RowEnd &end) {                 // (of the segment)
        if (!row_ends) {
            if (lane == 0) A.parts[blockIdx.x] = Part{end.ref.m, end.S, end.T, 0.0f};
            return;
        }
        if (lane == 0) end.store_row(A.a, row);
        for (int j = lane; j < A.a.n_tokens; j += 64) {
            if (j != lane) look_up<ElemT>(A, row, j, &given, &given_x);
            A.a.logprobs[row * A.a.n_tokens + j] = end.given(given, given_x, A.a);
        }
    };
    if (!TOP) {
        if (wave == WAVES - 1) finish(RowEnd(mine, A.c));
        return;
    }
    // `top` logits of a single wavefront reach the one, a share of them in each wavefront the other: the higher of the two
    const uint32_t line = max(wave_max(lines[0][lane % WAVES]), ~wave_max(~lines[1][lane % WAVES]));
    const float from = line <= 0x007FFFFFu ? -FLT_MAX : logit_of((Key)line << 32);
    int n = 0;
#pragma unroll
    for (int p = 0; p < PIECES; p++) {
        float largest = x[p][0];
#pragma unroll
        for (int k = 1; k < EPV; k++) largest = fmaxf(largest, x[p][k]);
        if (!__any(largest >= from)) continue;             // most often
#pragma unroll
        for (int k = 0; k < EPV; k++) {
            const unsigned long long who = __ballot(x[p][k] >= from);
            if (!who) continue;                            // most often
            const int at = n + __builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0));
            if (x[p][k] >= from && at < LISTED) listed[wave][at] = key_of(x[p][k], (uint32_t)(v0 + p * (THREADS * EPV) + k));
            n += __popcll(who);
        }
    }
    if (tid % 64 == 0) n_listed[wave] = n;
    __syncthreads();
    RowEnd end;
    if (row_ends || wave == WAVES - 1) end = RowEnd(mine, A.c);
    auto store = [&](int i, Key k) {
        if (row_ends) end.store_top(A.a, row, i, k);
        else A.keys[(int64_t)blockIdx.x * A.a.top + i] = k;
    };
    const int counts = lane < WAVES ? n_listed[lane] : 0, up_to = sum_up_to(counts);
    if (!__any(counts > LISTED)) {
        // All lists become one, and each key's rank the sum of what four lanes find above it, each in a quarter of the list: all wavefronts take part (64 x 32,000 bf16 with 20
        // alternatives 9.0 us; by the first wavefront alone, or by each against the others' lists in turn, 16.2).
        const int n_all = __builtin_amdgcn_readlane(up_to, WAVES - 1), before = __builtin_amdgcn_readlane(up_to, wave) - n;
        for (int i = lane; i < n; i += 64) all[before + i] = listed[wave][i];
        if (tid < 32) all[n_all + tid] = 0;                // nothing is below it: the list is taken 32 at a time
        __syncthreads();
        if (wave == WAVES - 1) finish(end);
        for (int i0 = wave * 16; i0 < n_all; i0 += THREADS / 4) {
            const int i = i0 + lane / 4;
            const Key mine = all[i < n_all ? i : 0];
            const int rank = rank_of(mine, all, n_all, lane);
            if (lane % 4 == 0 && i < n_all && rank < A.a.top) store(rank, mine);
        }
        for (int i = n_all + tid; i < A.a.top; i += THREADS) store(i, 0);
        return;
    }
    if (wave == WAVES - 1) finish(end);
    Key last = ~(Key)0;
    for (int i = 0; i < A.a.top; i++) {                    // the largest below the last one
        Key k0 = 0;
#pragma unroll
        for (int p = 0; p < PIECES; p++)
#pragma unroll
            for (int k = 0; k < EPV; k++) {
                const Key key = key_of(x[p][k], (uint32_t)(v0 + p * (THREADS * EPV) + k));
                if (key < last && key > k0) k0 = key;
            }
        k0 = wave_max(k0);
        if (tid % 64 == 0) best[wave] = k0;
        __syncthreads();
        k0 = best[0];
        for (int w = 1; w < WAVES; w++) if (best[w] > k0) k0 = best[w];
        if (tid == 0) store(i, k0);
        last = k0 ? k0 : 1;                                // none left: no key is below 1 but 0
        __syncthreads();
    }
}

// A row's parts, by one wavefront: 3.1 to 5 us, a launch's and two memory accesses' time (4,096 rows 5).  Its segments' alternatives are listed and ranked as a segment's are, up to JOINED_LANE in a lane; with more of them, or
// more equal ones than the list takes, they are merged from the segments' sorted lists, a lane at the head of each.
static const int JOINED_LANE = 16, JOINED = 256;           // keys of a lane, of the list

template <typename ElemT>
__global__ __launch_bounds__(ROWS_JOINED * 64) void logprobs_join_kernel(LogprobsArgs A) {
    __shared__ Key listed[ROWS_JOINED][JOINED + 32];
    extern __shared__ uint8_t taken[];                     // [ROWS_JOINED][n_seg]: keys of a segment that are out
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t row = (int64_t)blockIdx.x * ROWS_JOINED + wave;
    if (row >= A.a.rows) return;                           // whole wavefronts, and no barrier below
    // everything that has to come from memory is asked for first
    const int32_t n_keys = A.n_seg * A.a.top;
    const Key *const keys = A.keys + row * n_keys;
    const bool listable = A.a.top && n_keys <= JOINED_LANE * 64;
    Key own[JOINED_LANE];
    // A segment's keys lie sorted.  Each 64 of them go to the lanes from another one on, so that every lane has some of the first and the line, which a lane's
    // largest stands for, is not that of the last of a segment (64 alternatives of 16 segments: all would reach it;
    // 64 x 128,256 bf16: the whole kernel 42 us then).
    const int turn = 64 / ((n_keys + 63) / 64 + !n_keys);
    if (listable)
#pragma unroll
        for (int j = 0; j < JOINED_LANE; j++) {
            const int i = j * 64 + ((lane + j * turn) & 63);
            own[j] = 0;
            if (i < n_keys) own[j] = keys[i];
        }
    int64_t t = -1;
    float x = -INFINITY;
    if (lane < A.a.n_tokens) look_up<ElemT>(A, row, lane, &t, &x);
    Part mine_part{-INFINITY, 0.0f, 0.0f, 0.0f};
    for (int s = lane; s < A.n_seg; s += 64) join(mine_part, A.parts[row * A.n_seg + s], A.c);
    const RowEnd end(mine_part, A.c);
    if (lane == 0) end.store_row(A.a, row);
    for (int j = lane; j < A.a.n_tokens; j += 64) {
        if (j != lane) look_up<ElemT>(A, row, j, &t, &x);
        A.a.logprobs[row * A.a.n_tokens + j] = end.given(t, x, A.a);
    }
    if (!A.a.top) return;
    auto store = [&](int i, Key k) { end.store_top(A.a, row, i, k); };
    if (listable) {
        uint32_t most = 0;
#pragma unroll
        for (int j = 0; j < JOINED_LANE; j++) most = max(most, (uint32_t)(own[j] >> 32));
        uint32_t line[1];
        lines_of<1>(most, {A.a.top}, line);
        // With nearly as many alternatives as lanes that is what the poorest lane reaches; the line is then found among all keys (64 x 128,256 bf16 with 64 alternatives:
        // the kernel 15.2 us without, 10.7 so).
        auto reach = [&](uint32_t from) {
            int n = 0;
#pragma unroll
            for (int j = 0; j < JOINED_LANE; j++) n += __popcll(__ballot((uint32_t)(own[j] >> 32) >= from));
            return n;
        };
        if (reach(line[0]) > 128) {
            uint32_t found = 0;
#pragma unroll 1
            for (int bit = 31; bit >= 16; bit--) if (reach(found | 1u << bit) >= A.a.top) found |= 1u << bit;
            line[0] = max(found, line[0]);
        }
        Key *const list = listed[wave];
        int n = 0;
#pragma unroll
        for (int j = 0; j < JOINED_LANE; j++) {
            const bool in = (uint32_t)(own[j] >> 32) >= line[0];
            const unsigned long long who = __ballot(in);
            if (!who) continue;
            const int at = n + __popcll(who & ((1ull << lane) - 1));
            if (in && at < JOINED) list[at] = own[j];
            n += __popcll(who);
        }
        if (n <= JOINED) {
            if (lane < 32) list[n + lane] = 0;
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
            for (int i0 = 0; i0 < n; i0 += 16) {
                const int i = i0 + lane / 4;
                const Key mine = list[i < n ? i : 0];
                const int rank = rank_of(mine, list, n, lane);
                if (lane % 4 == 0 && i < n && rank < A.a.top) store(rank, mine);
            }
            for (int i = n + lane; i < A.a.top; i += 64) store(i, 0);
            return;
        }
    }
    uint8_t *const out = taken + wave * A.n_seg;
    for (int s = lane; s < A.n_seg; s += 64) out[s] = 0;   // a lane reads what it wrote itself
    Key mine = 0;
    int from = -1;
    bool look = true;
    for (int i = 0; i < A.a.top; i++) {
        if (look) {                                        // the largest key that is left of the lane's segments
            mine = 0;
            for (int s = lane; s < A.n_seg; s += 64) {
                const Key k = out[s] < A.a.top ? keys[(int64_t)s * A.a.top + out[s]] : 0;
                if (k > mine) { mine = k; from = s; }
            }
        }
        const Key k = wave_max(mine);
        look = k && k == mine;
        if (look) out[from]++;
        if (lane == 0) store(i, k);
    }
}

// The gradient: every thread reads a piece before it writes it, so the two may be the same memory.  4,096 x 128,256 bf16 345 us (6.1 TB/s), 300 x 32,000 fp32 15.5 (5.0).
// Every thread compares its elements with every token listed for the segment: 256 x 32,000 fp32 19 to 23 us a backward pass with one token a row, 23 with 64 (45 if they are the same one), 44 with 256, 127 with 1,024 (572); bf16 33 with 64 (67),
// 299 with 1,024 (972).
template <int PIECES, bool ONCE, typename ElemT>
__global__ __launch_bounds__(THREADS) void logprobs_grad_kernel(GradArgs A) {
    constexpr int EPV = 16 / sizeof(ElemT);
    __shared__ float sum;
    __shared__ int n_mine;
    __shared__ int32_t mine_v[GIVEN_MAX + TOP_MAX];        // tokens of the segment that have a gradient of their own
    __shared__ float mine_g[GIVEN_MAX + TOP_MAX];
    const zf_logprobs_args &a = A.l.a;
    const int tid = threadIdx.x, wave = tid / 64, lane = tid % 64;
    const int64_t row = blockIdx.x / (uint32_t)A.l.n_seg;
    const int32_t seg = blockIdx.x % (uint32_t)A.l.n_seg, V = a.V, first = seg * (THREADS * PIECES * EPV), v0 = first + tid * EPV;
    const ElemT *const logits = (const ElemT *)a.logits + row * a.row_stride_elems;
    const uint32_t *const mask = a.mask ? a.mask + row * A.l.W : nullptr;
    const bool whole = first + THREADS * PIECES * EPV <= V;
    float x[PIECES][EPV];
    load_pieces<THREADS, PIECES, EPV, ONCE>(logits, mask, v0, V, whole, x);
    float G = 0.0f;
    const int n_given = A.g.g_logprobs ? a.n_tokens : 0, n_all = n_given + (A.g.g_top ? a.top : 0);
    if (wave == 0) {                                       // the first wavefront lists them, in order
        int n = 0;
        for (int j0 = 0; j0 < n_all; j0 += 64) {
            const int j = j0 + lane;
            int64_t t = -1;
            float g = 0.0f, lp = -INFINITY;
            if (j < n_given) {
                const int64_t at = row * n_given + j;
                t = a.token_bytes == 8 ? ((const int64_t *)a.tokens)[at] : ((const int32_t *)a.tokens)[at];
                g = A.g.g_logprobs[at]; lp = a.logprobs[at];
            } else if (j < n_all) {
                const int64_t at = row * a.top + j - n_given;
                t = a.top_ids[at]; g = A.g.g_top[at]; lp = a.top_logprobs[at];
            }
            if (t < 0 || t >= V || !(lp > -INFINITY)) g = 0.0f, t = -1;      // (in a row with a NaN every token that is allowed has NaN anyway)
            G += g;
            const bool here = t >= first && t < first + THREADS * PIECES * EPV;
            const unsigned long long who = __ballot(here);
            if (here) { const int at = n + __popcll(who & ((1ull << lane) - 1)); mine_v[at] = (int32_t)t; mine_g[at] = g * A.l.inv_t; }
            n += __popcll(who);
        }
        G = wave_sum(G);
        if (lane == 0) { sum = G; n_mine = n; }
    }
    __syncthreads();
    G = sum;
    const Reference ref(a.stats[2 * row], A.l.c);
    const float log2_S = a.stats[2 * row + 1], inv_t = A.l.inv_t;
    const float gh = A.g.g_entropy ? A.g.g_entropy[row] : 0.0f, H = A.g.g_entropy ? a.entropy[row] : 0.0f;
    // d = p (base + slope log2 p), p = 2^y, y = log2 p
    const float base = inv_t * (-G - gh * H), slope = -inv_t * gh * LN_2;
    const int n = n_mine;
    // p may be 0, and 0 times what is not finite is NaN: rows with a NaN, infinite gradients, factors near 32 bits' limit (y is -1e4 at least, less log2 S).
    // There, and far out, where there may be nothing but -inf, every element is looked at.
    const bool look = ref.far || !(fabsf(base) + 2e4f * fabsf(slope) + fabsf(log2_S) < INFINITY);
    ElemT *const grad = (ElemT *)A.g.grad + row * A.g.stride;
#pragma unroll
    for (int p = 0; p < PIECES; p++) {
        const int32_t v = v0 + p * (THREADS * EPV);
        float d[EPV];
        if (!look) {
#pragma unroll
            for (int k = 0; k < EPV; k++) {
                const float y = fmaxf(fmaf(x[p][k], ref.c, -ref.R), -1e4f) - log2_S;
                d[k] = two_to(y) * fmaf(slope, y, base);
            }
        } else {
#pragma unroll
            for (int k = 0; k < EPV; k++) {
                const float y = fmaxf(ref.far ? (x[p][k] - ref.m) * ref.c : fmaf(x[p][k], ref.c, -ref.R), -1e4f) - log2_S, e = two_to(y);
                d[k] = x[p][k] == -INFINITY ? 0.0f : fmaf(e * y, slope, e * base);
            }
        }
        for (int j = 0; j < n; j++) {
#pragma unroll
            for (int k = 0; k < EPV; k++) if (mine_v[j] == v + k) d[k] += mine_g[j];
        }
        union { u32x4 v; ElemT e[EPV]; bf16x2 b[4]; } o;
#pragma unroll
        for (int k = 0; k < EPV; k += 2) {
            if (sizeof(ElemT) == 4) { o.v[k % 4] = __float_as_uint(d[k]); o.v[k % 4 + 1] = __float_as_uint(d[k + 1]); }
            else o.b[k / 2 % 4] = bf16x2{(__bf16)d[k], (__bf16)d[k + 1]};
        }
        typename Piece<ElemT>::type *const to = reinterpret_cast<typename Piece<ElemT>::type *>(grad + v);
        if (whole || v + EPV <= V) {
            if (ONCE) __builtin_nontemporal_store(o.v, to);
            else *to = o.v;
        } else {
#pragma unroll
            for (int k = 0; k < EPV; k++) if (v + k < V) grad[v + k] = o.e[k];
        }
    }
}

int64_t blocks_of(const zf_logprobs_args &a, int threads, int pieces) {
    const int32_t n = threads * pieces * (a.dtype == 0 ? 4 : 8);
    return a.rows * ((a.V + n - 1) / n);
}
// Threads of a workgroup and 16-byte pieces that each holds.  A row of up to 32,768 logits is one workgroup's, which ends it: no second launch, no workspace
// (300 x 32,000 fp32 12.2 us, in segments 14.8; one such row 9.7 and 8.9, but its call 7 us of the host and 11).  Longer rows are cut into segments of four pieces a thread, or of one where that would be fewer than two workgroups a compute unit and the joining
// wavefronts' lists hold the alternatives of so many.
struct Plan { int threads, pieces; int32_t n_seg; };
Plan plan_of(const zf_logprobs_args &a) {
    const int epv = a.dtype == 0 ? 4 : 8;
    const Plan whole[] = {{256, 1, 1}, {256, 4, 1}, {1024, 4, 1}, {1024, 8, 1}};
    for (const Plan &p : whole) if (a.V <= p.threads * p.pieces * epv && (a.dtype == 0 || p.pieces < 8)) return p;
    int pieces = PIECES;
    if (blocks_of(a, THREADS, PIECES) < 512 && blocks_of(a, THREADS, 1) / a.rows * a.top <= JOINED_LANE * 64) pieces = 1;
    return Plan{THREADS, pieces, (int32_t)(blocks_of(a, THREADS, pieces) / a.rows)};
}
LogprobsArgs args_of(const zf_logprobs_args &a, int32_t n_seg, void *workspace) {
    LogprobsArgs A{};
    A.a = a;
    A.W = (a.V + 31) / 32;
    A.n_seg = n_seg;
    A.c = LOG2_E / a.temperature;
    A.inv_t = 1.0f / a.temperature;
    A.parts = (Part *)workspace;
    A.keys = (Key *)(A.parts + a.rows * A.n_seg);
    return A;
}

// Rows that the last-level cache (256 MB) cannot hold until somebody reads them again pass it by.  4,096 x 128,256 bf16: the sums 187 us without, 181 so, the
// gradient 399 and 352; 2,000 x 128,256 fp32 177 and 162, 394 and 372; but 300 x 32,000 fp32 14.8 and 15.1, 16.5 and 17.4, and rows at odd
// elements (1,030 x 40,037 bf16) 19.5 and 21.0.
bool once(const zf_logprobs_args &a) {
    const int64_t size = a.dtype == 0 ? 4 : 2;
    return a.rows * a.V * size > (256ll << 20) && (uintptr_t)a.logits % 16 == 0 && a.row_stride_elems * size % 16 == 0;
}
template <int THREADS, int PIECES, bool ONCE, typename ElemT>
void parts(const LogprobsArgs &A, hipStream_t s) {
    const bool entropy = A.a.entropy != nullptr;
    auto *const part = A.a.top ? (entropy ? logprobs_part_kernel<THREADS, PIECES, ONCE, true, true, ElemT> : logprobs_part_kernel<THREADS, PIECES, ONCE, false, true, ElemT>)
                               : (entropy ? logprobs_part_kernel<THREADS, PIECES, ONCE, true, false, ElemT> : logprobs_part_kernel<THREADS, PIECES, ONCE, false, false, ElemT>);
    hipLaunchKernelGGL(part, dim3((uint32_t)(A.a.rows * A.n_seg)), dim3(THREADS), 0, s, A);
}
template <typename ElemT>
void forward(const LogprobsArgs &A, const Plan &p, hipStream_t s) {
    const bool pass = once(A.a);
    if (p.threads == 1024) {
        if constexpr (sizeof(ElemT) == 4) { if (p.pieces == 8) return pass ? parts<1024, 8, true, ElemT>(A, s) : parts<1024, 8, false, ElemT>(A, s); }
        return pass ? parts<1024, 4, true, ElemT>(A, s) : parts<1024, 4, false, ElemT>(A, s);
    }
    if (p.pieces == 1) parts<THREADS, 1, false, ElemT>(A, s);
    else if (pass) parts<THREADS, PIECES, true, ElemT>(A, s);
    else parts<THREADS, PIECES, false, ElemT>(A, s);
    if (A.n_seg > 1)
        hipLaunchKernelGGL((logprobs_join_kernel<ElemT>), dim3((uint32_t)((A.a.rows + ROWS_JOINED - 1) / ROWS_JOINED)), dim3(ROWS_JOINED * 64),
                           A.a.top ? ROWS_JOINED * A.n_seg : 0, s, A);
}

}  // namespace

int64_t logprobs_workspace(const zf_logprobs_args &a) {
    const int64_t n = plan_of(a).n_seg;
    return n > 1 ? a.rows * n * (int64_t)(sizeof(Part) + a.top * sizeof(Key)) : 0;
}
int64_t logprobs_blocks(const zf_logprobs_args &a) { return blocks_of(a, THREADS, 1); }   // at most

hipError_t launch_logprobs(const zf_logprobs_args &a, void *workspace, hipStream_t s) {
    const Plan p = plan_of(a);
    const LogprobsArgs A = args_of(a, p.n_seg, workspace);
    if (a.dtype == 0) forward<uint32_t>(A, p, s);
    else forward<uint16_t>(A, p, s);
    return hipGetLastError();
}

hipError_t launch_logprobs_backward(const zf_logprobs_args &a, const LogprobsGrad &g, hipStream_t s) {
    const int n = blocks_of(a, THREADS, PIECES) < 512 ? 1 : PIECES;       // pieces
    const GradArgs A{args_of(a, (int32_t)(blocks_of(a, THREADS, n) / a.rows), nullptr), g};
    const bool pass = once(a) && (uintptr_t)g.grad % 16 == 0 && g.stride * (a.dtype == 0 ? 4 : 2) % 16 == 0;
    auto *const kernel = n == 1 ? (a.dtype == 0 ? logprobs_grad_kernel<1, false, uint32_t> : logprobs_grad_kernel<1, false, uint16_t>)
                         : pass         ? (a.dtype == 0 ? logprobs_grad_kernel<PIECES, true, uint32_t> : logprobs_grad_kernel<PIECES, true, uint16_t>)
                                        : (a.dtype == 0 ? logprobs_grad_kernel<PIECES, false, uint32_t> : logprobs_grad_kernel<PIECES, false, uint16_t>);
    hipLaunchKernelGGL(kernel, dim3((uint32_t)(a.rows * A.l.n_seg)), dim3(THREADS), 0, s, A);
    return hipGetLastError();
}

}  // namespace zf
