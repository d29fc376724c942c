// Log probabilities of given tokens under a mask, with entropy and alternatives, and their gradient.
//
// Of a row's allowed logits x, with c = log2(e) / temperature and m their largest:
//   S = sum 2^((x - m) c),  T = sum 2^((x - m) c) (x - m) c
//   logprob of t = (x_t - m) / temperature - ln S        entropy = ln S - ln 2 T / S
//   d logits_v = 1 / temperature (p_v (-G - g_H (ln p_v + H)) + sum of g_j where token j is v),   G = sum of all g_j
// m, S and T are held in 32 bits, and sums that were taken around another m join by the factor 2^((m' - m) c).  x - m is taken before it is multiplied:
// logits at the type's lowest value stay finite then, and equal ones equally probable.
//   A row is read once, in segments, a workgroup each; a second launch joins a row's segments and looks its given tokens up.
#include <hip/hip_runtime.h>
#include <algorithm>
#include <cfloat>
#include "zf_ops.h"

namespace zf {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
template <typename ElemT> struct Piece;       // 16 bytes at any multiple of an element: the memory system takes them there
template <> struct Piece<uint32_t> { typedef u32x4 type __attribute__((aligned(4))); };
template <> struct Piece<uint16_t> { typedef u32x4 type __attribute__((aligned(2))); };

static const float LOG2_E = 1.44269504088896340736f, LN_2 = 0.69314718055994530942f;
static const int THREADS = 256, WAVES = THREADS / 64, ROWS_JOINED = 4;   // rows a workgroup of the joining kernel takes, a wavefront each
static const int PIECES = 4;                                             // 16-byte pieces of a segment that a thread holds

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
__device__ __forceinline__ void to_bits(float x, uint32_t *out) { *out = __float_as_uint(x); }
__device__ __forceinline__ void to_bits(float x, uint16_t *out) {       // to nearest, ties to even
    const uint32_t u = __float_as_uint(x);
    *out = (u & 0x7FFFFFFFu) > 0x7F800000u ? (uint16_t)((u >> 16) | 0x40u) : (uint16_t)((u + 0x7FFFu + ((u >> 16) & 1u)) >> 16);
}
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
__device__ __forceinline__ float two_to(float x) { return __builtin_amdgcn_exp2f(x); }   // below 2^-126 nothing
// A finite logit has a finite log probability (the type's lowest value divided by a temperature below one is beyond 32 bits).
__device__ __forceinline__ float logprob_of(float x, float m, float temperature, float ln_S) {
    const float lp = (x - m) / temperature - ln_S;
    return lp < -FLT_MAX && x > -INFINITY ? -FLT_MAX : lp;
}
// b joins a.  A side without anything has m = -inf and sums of zero (or NaN, where it has nothing but NaN).
__device__ __forceinline__ void join(Part &a, const Part &b, float c) {
    const float m = fmaxf(a.m, b.m);
    const float da = a.m == m ? 0.0f : fmaxf((a.m - m) * c, -1e4f), db = b.m == m ? 0.0f : fmaxf((b.m - m) * c, -1e4f);
    const float fa = two_to(da), fb = two_to(db);
    a.T = fa * (a.T + a.S * da) + fb * (b.T + b.S * db);
    a.S = fa * a.S + fb * b.S;
    a.m = m;
}
__device__ __forceinline__ bool allowed(const uint32_t *mask, int64_t row, int32_t W, uint32_t v) {
    return !mask || ((mask[row * W + (v >> 5)] >> (v & 31)) & 1u);
}

// Piece of a row from token v on: its logits, -inf where there is no token or none that is allowed.
template <typename ElemT, int EPV>
__device__ __forceinline__ void load_piece(const ElemT *row, const uint32_t *mask_row, int32_t v, int32_t V, float (&x)[EPV]) {
    constexpr uint32_t FULL = (1u << EPV) - 1u;
    const int32_t left = V - v;
    uint32_t bits = left >= EPV ? FULL : left > 0 ? (1u << left) - 1u : 0u;
    if (mask_row && left > 0) bits &= mask_row[v >> 5] >> (v & 31);
    if (left >= EPV) {
        const u32x4 p = *reinterpret_cast<const typename Piece<ElemT>::type *>(row + v);
#pragma unroll
        for (int k = 0; k < EPV; k++) x[k] = __uint_as_float(sizeof(ElemT) == 4 ? p[k] : k & 1 ? p[k / 2] & 0xFFFF0000u : p[k / 2] << 16);
    } else {
#pragma unroll
        for (int k = 0; k < EPV; k++) x[k] = k < left ? of_bits(row[v + k]) : 0.0f;
    }
    if (__any(bits != FULL)) {
#pragma unroll
        for (int k = 0; k < EPV; k++) {
            const uint32_t yes = (uint32_t)__builtin_amdgcn_sbfe((int)bits, k, 1);
            x[k] = __uint_as_float((__float_as_uint(x[k]) & yes) | (0xFF800000u & ~yes));
        }
    }
}

// The alternatives of a segment.  Every wavefront takes the `top`-th largest of its lanes' largest logits (by their bits in order, the upper sixteen of them): its
// part of the segment's alternatives lies at or above it, and little else does.  What does is listed, and of all lists together the rank of each is the number of keys above it.  When a list
// overflows (many equal logits) the keys are found one by one, each the largest below the last.
static const int LISTED = 128;                // keys a wavefront lists

template <bool ENT, bool TOP, typename ElemT>
__global__ __launch_bounds__(THREADS) void logprobs_part_kernel(LogprobsArgs A) {
    constexpr int EPV = 16 / sizeof(ElemT);
    __shared__ Part part[WAVES];
    __shared__ Key best[WAVES], listed[TOP ? WAVES * LISTED : 1];
    __shared__ int n_listed[WAVES];
    const int tid = threadIdx.x, wave = tid / 64;
    const int64_t row = blockIdx.x / (uint32_t)A.n_seg;
    const int32_t seg = blockIdx.x % (uint32_t)A.n_seg, V = A.a.V, v0 = seg * (THREADS * PIECES * EPV) + tid * EPV;
    const ElemT *const logits = (const ElemT *)A.a.logits + row * A.a.row_stride_elems;
    const uint32_t *const mask = A.a.mask ? A.a.mask + row * A.W : nullptr;
    float x[PIECES][EPV], most = -INFINITY;
#pragma unroll
    for (int p = 0; p < PIECES; p++) load_piece<ElemT, EPV>(logits, mask, v0 + p * (THREADS * EPV), V, x[p]);
#pragma unroll
    for (int p = 0; p < PIECES; p++)
#pragma unroll
        for (int k = 0; k < EPV; k++) most = fmaxf(most, x[p][k]);
    const float m = wave_max(most);
    float S = 0.0f, T = 0.0f;
    if (m > -INFINITY) {
#pragma unroll
        for (int p = 0; p < PIECES; p++)
#pragma unroll
            for (int k = 0; k < EPV; k++) {
                const float z = (x[p][k] - m) * A.c, e = two_to(z);
                S += e;
                if (ENT) T = fmaf(e, fmaxf(z, -1e4f), T);  // nothing times -inf is nothing
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
        const uint32_t mine = in_order(most);
        uint32_t line = 0;                                 // the largest multiple of 2^16 that `top` lanes reach
#pragma unroll
        for (int bit = 31; bit >= 16; bit--) {
            const uint32_t up = line | 1u << bit;
            if (__popcll(__ballot(mine >= up)) >= A.a.top) line = up;
        }
        if (line == 0) line = 1;                           // 0 stands for no logit
        int n = 0;
#pragma unroll
        for (int p = 0; p < PIECES; p++)
#pragma unroll
            for (int k = 0; k < EPV; k++) {
                const uint32_t o = in_order(x[p][k]);
                const unsigned long long who = __ballot(o >= line);
                if (!who) continue;
                const int at = n + __popcll(who & ((1ull << (tid % 64)) - 1));
                if (o >= line && at < LISTED) listed[wave * LISTED + at] = (Key)o << 32 | (uint32_t)~(uint32_t)(v0 + p * (THREADS * EPV) + k);
                n += __popcll(who);
            }
        if (tid % 64 == 0) n_listed[wave] = n;
    }
    __syncthreads();
    if (tid == 0) {
        Part all = part[0];
#pragma unroll
        for (int w = 1; w < WAVES; w++) join(all, part[w], A.c);
        A.parts[blockIdx.x] = all;
    }
    if (!TOP) return;
    Key *const out = A.keys + (int64_t)blockIdx.x * A.a.top;
    int n_all = 0;
    bool fits = true;
#pragma unroll
    for (int w = 0; w < WAVES; w++) { n_all += n_listed[w]; fits = fits && n_listed[w] <= LISTED; }
    if (fits) {
        for (int i = tid; i < WAVES * LISTED; i += THREADS) {
            if (i % LISTED >= n_listed[i / LISTED]) continue;
            const Key mine = listed[i];
            int rank = 0;
            for (int w = 0; w < WAVES; w++)
                for (int j = 0; j < n_listed[w]; j++) rank += listed[w * LISTED + j] > mine;
            if (rank < A.a.top) out[rank] = mine;
        }
        if (tid < A.a.top && tid >= n_all) out[tid] = 0;
        return;
    }
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
        if (tid == 0) out[i] = k0;
        last = k0 ? k0 : 1;                                // none left: no key is below 1 but 0
        __syncthreads();
    }
}

// A row's parts, by one wavefront; the alternatives are merged from the segments' sorted lists, a lane at the head of each.
static const int JOINED_KEYS = 1024;                       // so many of a row are brought to LDS (a step to the next of a list in memory takes ten times as long)
__host__ __device__ __forceinline__ int32_t join_bytes(int32_t n_seg, int32_t top) {
    return ((top && n_seg * top <= JOINED_KEYS ? n_seg * top * (int32_t)sizeof(Key) : 0) + n_seg + 7) / 8 * 8;
}

template <typename ElemT>
__global__ __launch_bounds__(ROWS_JOINED * 64) void logprobs_join_kernel(LogprobsArgs A) {
    extern __shared__ __align__(8) uint8_t lds[];          // of each row: its segments' keys where they fit, then how many of each are out
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t row = (int64_t)blockIdx.x * ROWS_JOINED + wave;
    if (row >= A.a.rows) return;                           // whole wavefronts, and no barrier below
    Part all{-INFINITY, 0.0f, 0.0f, 0.0f};
    for (int s = lane; s < A.n_seg; s += 64) join(all, A.parts[row * A.n_seg + s], A.c);
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const Part o{__shfl_xor(all.m, d), __shfl_xor(all.S, d), __shfl_xor(all.T, d), 0.0f};
        join(all, o, A.c);
    }
    const bool nothing = all.m == -INFINITY && all.S == 0.0f;
    const float ln_S = nothing ? 0.0f : logf(all.S);
    if (lane == 0) {
        if (A.a.entropy) A.a.entropy[row] = nothing ? 0.0f : ln_S - LN_2 * all.T / all.S;
        if (A.a.stats) { A.a.stats[2 * row] = all.m; A.a.stats[2 * row + 1] = ln_S; }
    }
    const ElemT *const logits = (const ElemT *)A.a.logits + row * A.a.row_stride_elems;
    for (int j = lane; j < A.a.n_tokens; j += 64) {
        const int64_t at = row * A.a.n_tokens + j;
        const int64_t t = A.a.token_bytes == 8 ? ((const int64_t *)A.a.tokens)[at] : ((const int32_t *)A.a.tokens)[at];
        float lp = 0.0f;
        if (t >= A.a.V) lp = NAN;
        else if (t >= 0) {
            lp = -INFINITY;
            if (!nothing && allowed(A.a.mask, row, A.W, (uint32_t)t)) lp = logprob_of(of_bits(logits[t]), all.m, A.a.temperature, ln_S);
            else if (all.S != all.S) lp = all.S;
        }
        A.a.logprobs[at] = lp;
    }
    if (!A.a.top) return;
    const int32_t n_keys = A.n_seg * A.a.top;
    const bool near = n_keys <= JOINED_KEYS;
    uint8_t *const own = lds + wave * join_bytes(A.n_seg, A.a.top), *const out = own + (near ? n_keys * sizeof(Key) : 0);
    const Key *keys = A.keys + row * n_keys;
    if (near) {
        Key *const copy = reinterpret_cast<Key *>(own);
        for (int i = lane; i < n_keys; i += 64) copy[i] = keys[i];
        keys = copy;
    }
    for (int s = lane; s < A.n_seg; s += 64) out[s] = 0;
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
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
        if (lane == 0) {
            A.a.top_ids[row * A.a.top + i] = k ? (int32_t)~(uint32_t)k : -1;
            A.a.top_logprobs[row * A.a.top + i] = k ? logprob_of(logit_of(k), all.m, A.a.temperature, ln_S) : -INFINITY;
        }
    }
}

// The gradient: every thread reads a piece before it writes it, so the two may be the same memory.
template <typename ElemT>
__global__ __launch_bounds__(THREADS) void logprobs_grad_kernel(GradArgs A) {
    constexpr int EPV = 16 / sizeof(ElemT);
    __shared__ float sums[WAVES];
    __shared__ int n_mine;
    __shared__ int32_t mine_v[GIVEN_MAX + TOP_MAX];        // tokens of the segment that have a gradient of their own
    __shared__ float mine_g[GIVEN_MAX + TOP_MAX];
    const zf_logprobs_args &a = A.l.a;
    const int tid = threadIdx.x, wave = tid / 64, lane = tid % 64;
    const int64_t row = blockIdx.x / (uint32_t)A.l.n_seg;
    const int32_t seg = blockIdx.x % (uint32_t)A.l.n_seg, V = a.V, first = seg * (THREADS * PIECES * EPV), v0 = first + tid * EPV;
    const ElemT *const logits = (const ElemT *)a.logits + row * a.row_stride_elems;
    const uint32_t *const mask = a.mask ? a.mask + row * A.l.W : nullptr;
    float x[PIECES][EPV];
#pragma unroll
    for (int p = 0; p < PIECES; p++) load_piece<ElemT, EPV>(logits, mask, v0 + p * (THREADS * EPV), V, x[p]);
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
            if (t < 0 || t >= V || lp == -INFINITY) g = 0.0f, t = -1;
            G += g;
            const bool here = t >= first && t < first + THREADS * PIECES * EPV;
            const unsigned long long who = __ballot(here);
            if (here) { const int at = n + __popcll(who & ((1ull << lane) - 1)); mine_v[at] = (int32_t)t; mine_g[at] = g; }
            n += __popcll(who);
        }
        G = wave_sum(G);
        if (lane == 0) { sums[0] = G; n_mine = n; }
    }
    __syncthreads();
    G = sums[0];
    const float m = a.stats[2 * row], ln_S = a.stats[2 * row + 1], inv_t = A.l.inv_t;
    const float gh = A.g.g_entropy ? A.g.g_entropy[row] : 0.0f, H = A.g.g_entropy ? a.entropy[row] : 0.0f;
    const bool nothing = m == -INFINITY;
    const float log2_S = ln_S * LOG2_E;
    const int n = n_mine;
    ElemT *const grad = (ElemT *)A.g.grad + row * A.g.stride;
#pragma unroll
    for (int p = 0; p < PIECES; p++) {
        const int32_t v = v0 + p * (THREADS * EPV);
        float d[EPV];
#pragma unroll
        for (int k = 0; k < EPV; k++) {
            const float y = fmaxf((x[p][k] - m) * A.l.c, -1e4f) - log2_S, e = two_to(y);
            d[k] = nothing || x[p][k] == -INFINITY ? 0.0f : e * (-G - gh * (y * LN_2 + H));
            if (x[p][k] != x[p][k]) d[k] = x[p][k];
        }
        for (int j = 0; j < n; j++) {
#pragma unroll
            for (int k = 0; k < EPV; k++) if (mine_v[j] == v + k) d[k] += mine_g[j];
        }
        union { u32x4 v; ElemT e[EPV]; } o;
#pragma unroll
        for (int k = 0; k < EPV; k++) to_bits(d[k] * inv_t, &o.e[k]);
        if (v + EPV <= V) *reinterpret_cast<typename Piece<ElemT>::type *>(grad + v) = o.v;
        else {
#pragma unroll
            for (int k = 0; k < EPV; k++) if (v + k < V) grad[v + k] = o.e[k];
        }
    }
}

int32_t segments(const zf_logprobs_args &a) {
    const int32_t n = THREADS * PIECES * (a.dtype == 0 ? 4 : 8);
    return (a.V + n - 1) / n;
}
LogprobsArgs with_plan(const zf_logprobs_args &a, void *workspace) {
    LogprobsArgs A{};
    A.a = a;
    A.W = (a.V + 31) / 32;
    A.n_seg = segments(a);
    A.c = LOG2_E / a.temperature;
    A.inv_t = 1.0f / a.temperature;
    A.parts = (Part *)workspace;
    A.keys = (Key *)(A.parts + a.rows * A.n_seg);
    return A;
}

template <typename ElemT>
void forward(const LogprobsArgs &A, hipStream_t s) {
    const dim3 grid((uint32_t)(A.a.rows * A.n_seg));
    const bool entropy = A.a.entropy != nullptr;
    auto *const part = A.a.top ? (entropy ? logprobs_part_kernel<true, true, ElemT> : logprobs_part_kernel<false, true, ElemT>)
                               : (entropy ? logprobs_part_kernel<true, false, ElemT> : logprobs_part_kernel<false, false, ElemT>);
    hipLaunchKernelGGL(part, grid, dim3(THREADS), 0, s, A);
    hipLaunchKernelGGL((logprobs_join_kernel<ElemT>), dim3((uint32_t)((A.a.rows + ROWS_JOINED - 1) / ROWS_JOINED)), dim3(ROWS_JOINED * 64),
                       A.a.top ? ROWS_JOINED * join_bytes(A.n_seg, A.a.top) : 0, s, A);
}

}  // namespace

int64_t logprobs_workspace(const zf_logprobs_args &a) { return a.rows * segments(a) * (int64_t)(sizeof(Part) + a.top * sizeof(Key)); }
int64_t logprobs_blocks(const zf_logprobs_args &a) { return a.rows * segments(a); }

hipError_t launch_logprobs(const zf_logprobs_args &a, void *workspace, hipStream_t s) {
    const LogprobsArgs A = with_plan(a, workspace);
    if (a.dtype == 0) forward<uint32_t>(A, s);
    else forward<uint16_t>(A, s);
    return hipGetLastError();
}

hipError_t launch_logprobs_backward(const zf_logprobs_args &a, const LogprobsGrad &g, hipStream_t s) {
    const GradArgs A{with_plan(a, nullptr), g};
    const dim3 grid((uint32_t)(a.rows * A.l.n_seg));
    if (a.dtype == 0) hipLaunchKernelGGL((logprobs_grad_kernel<uint32_t>), grid, dim3(THREADS), 0, s, A);
    else hipLaunchKernelGGL((logprobs_grad_kernel<uint16_t>), grid, dim3(THREADS), 0, s, A);
    return hipGetLastError();
}

}  // namespace zf
