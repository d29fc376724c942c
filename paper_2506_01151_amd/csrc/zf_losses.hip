// Losses that a learner takes on logits under masks, with the logits' gradient.
//
// Of a row's logits x that its mask allows and that are not -inf, with c = log2(e) / temperature, m their largest and y = (x - m) c:
//   S = sum 2^y,  T = sum 2^y y,  p = 2^y / S,  ln p = ln 2 y - ln S,  H = ln S - ln 2 T / S
// A row's loss is a function of a few log probabilities (of the teacher's listed tokens, of the token that was drawn), and of H; with f_k its derivatives for the
// former, -b that for H,
//   d loss / d x_v = 1 / temperature (p_v (-sum f + b (ln p_v + H)) + sum of f_k where token k is v)
// The distillation's outcome "another token" has p_R = S_R / S, S_R the sum over what is not listed, taken as such: 1 - sum of the listed would be
// nothing but rounding where a row is sure of itself.  Its derivative adds f_R p_v / p_R to the tokens outside the list and -f_R p_v to all.
//   Elements are taken in 32 bits, a row's few numbers in 64: ratios next to a border of the clipping, differences of nearly equal log probabilities.
#include <hip/hip_runtime.h>
#include <algorithm>
#include <cfloat>
#include "zf_logit_rows.h"
#include "zf_ops.h"

namespace zf {
namespace {

enum Kind { POLICY, DISTILL, LOGPROB };       // LOGPROB: of the given tokens alone, and what a gradient needs (preferences)

static const int CHUNK = 1 << 17;             // tokens whose bits LDS holds: which of them a row's teacher listed

struct Args {
    zf_loss_rows r;
    int32_t W, K;
    float c;                                   // log2(e) / temperature
    int32_t id_bytes, values_dtype, rest;
    const void *ids, *values;
    void *grad;
    int64_t grad_stride;
    const float *g;                            // the loss's own gradient, or null: one
    int32_t held;                              // the gradient for g = 1 is in place
    int32_t results;                           // the losses are wanted
    const float *old_logprobs, *advantages, *ref;
    double lowest, highest, kl_weight, entropy_weight;
    float *logprobs, *entropy, *stats;
};

struct Part { float m, S, T, pad; };
struct Ends {                                  // what the gradient of a row is made from
    float m, base, slope, at_token;            // d = 2^((x - m) c) (base + slope y); the given token's own
    int32_t nothing;                           // a gradient of zeros
};

__device__ __forceinline__ double wave_sum(double x) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) x += __shfl_xor(x, d);
    return x;
}
__device__ __forceinline__ double wave_max(double x) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) x = fmax(x, __shfl_xor(x, d));
    return x;
}
__device__ __forceinline__ int64_t id_at(const Args &A, int64_t i) { return A.id_bytes == 8 ? ((const int64_t *)A.ids)[i] : ((const int32_t *)A.ids)[i]; }
__device__ __forceinline__ bool allowed(const uint32_t *mask_row, int64_t v) { return !mask_row || ((mask_row[v >> 5] >> (v & 31)) & 1u); }

// Sums around another reference join by 2^((m' - m) c).  The references are finite (a part without anything has -FLT_MAX and sums of zero) or +inf
// (whose sum is NaN), and nothing times -inf is nothing: 1e4 stands for all that is below 2^-126.
__device__ __forceinline__ float apart(float m, float whole, float c) { return m == whole ? 0.0f : fmaxf((m - whole) * c, -1e4f); }
__device__ __forceinline__ Part join_wave(Part a, float c) {
    const float m = wave_max(a.m), d = apart(a.m, m, c), f = two_to(d);
    return Part{m, wave_sum(f * a.S), wave_sum(f * fmaf(a.S, d, a.T)), 0.0f};
}

// 16 bytes of a row from element v on as numbers: -inf where `bits` has none, where nothing is read either.
template <int EPV, typename ElemT>
__device__ __forceinline__ void load_piece(const ElemT *row, int64_t v, int32_t V, uint32_t bits, float (&x)[EPV]) {
    constexpr uint32_t FULL = (1u << EPV) - 1u;
    union { u32x4 v; ElemT e[EPV]; } o;
    o.v = u32x4{0, 0, 0, 0};
    if (V - v >= EPV) {
        if (bits) o.v = *reinterpret_cast<const typename Piece<ElemT>::type *>(row + v);
    } else {
#pragma unroll
        for (int k = 0; k < EPV; k++) if (v + k < V) o.e[k] = row[v + k];
    }
#pragma unroll
    for (int k = 0; k < EPV; k++) x[k] = __uint_as_float(sizeof(ElemT) == 4 ? o.v[k % 4] : k & 1 ? o.v[k / 2] & 0xFFFF0000u : o.v[k / 2] << 16);
    if (bits != FULL) {
#pragma unroll
        for (int k = 0; k < EPV; k++) x[k] = (bits >> k) & 1u ? x[k] : -INFINITY;
    }
}
template <int EPV>
__device__ __forceinline__ uint32_t bits_of(const uint32_t *mask_row, int64_t v, int32_t V) {
    constexpr uint32_t FULL = (1u << EPV) - 1u;
    const uint32_t inside = V - v >= EPV ? FULL : (1u << (int)(V - v)) - 1u;
    return mask_row ? (mask_row[v >> 5] >> (v & 31)) & inside : inside;
}
template <int EPV, typename ElemT>
__device__ __forceinline__ void store_piece(ElemT *grad, int64_t v, int32_t V, const float (&d)[EPV]) {
    union { u32x4 v; ElemT e[EPV]; bf16x2 b[4]; } o;
#pragma unroll
    for (int k = 0; k < EPV; k += 2) {
        if (sizeof(ElemT) == 4) { o.v[k % 4] = __float_as_uint(d[k]); o.v[k % 4 + 1] = __float_as_uint(d[k + 1]); }
        else o.b[k / 2 % 4] = bf16x2{(__bf16)d[k], (__bf16)d[k + 1]};
    }
    if (V - v >= EPV) *reinterpret_cast<typename Piece<ElemT>::type *>(grad + v) = o.v;
    else
#pragma unroll
        for (int k = 0; k < EPV; k++) if (v + k < V) grad[v + k] = o.e[k];
}
template <typename ElemT>
__device__ __forceinline__ void store_element(ElemT *to, float x) {
    if (sizeof(ElemT) == 4) *(float *)to = x;
    else *(__bf16 *)to = (__bf16)x;
}

// What a policy's loss makes of a row, by every lane of a wavefront alike.  Returns the row's loss.
__device__ __forceinline__ double policy_row(const Args &A, const Part &sum, int64_t row, int64_t t, float x, float wg, Ends *ends, float *logprob, float *entropy) {
    const double lnS = log((double)sum.S);
    const bool nan = t >= A.r.V || sum.S != sum.S;
    const bool counts = nan || x != -INFINITY;
    *entropy = nan ? NAN : sum.S == 0.0f ? 0.0f : (float)(lnS - (double)LN_2 * sum.T / sum.S);
    *ends = Ends{0.0f, 0.0f, 0.0f, 0.0f, 1};
    *logprob = -INFINITY;
    if (!counts) return 0.0;
    const double lp = nan ? (double)NAN : ((double)x - sum.m) / A.r.temperature - lnS;
    *logprob = lp < -FLT_MAX ? -FLT_MAX : (float)lp;
    const double a = A.advantages[row], ratio = exp(lp - A.old_logprobs[row]);
    const double kept = ratio < A.lowest ? A.lowest : ratio > A.highest ? A.highest : ratio;
    const bool clipped = kept * a < ratio * a;
    double loss = -(clipped ? kept * a : ratio * a), f = clipped ? 0.0 : -ratio * a;
    if (A.ref) {
        const double d = A.ref[row] - lp, up = expm1(d);
        loss += A.kl_weight * (up - d);
        f -= A.kl_weight * up;
    }
    const double b = A.entropy ? A.entropy_weight : 0.0, H = *entropy;
    loss -= b * H;
    // p (-f + b (ln p + H)), ln p = ln 2 y - ln S; for the token itself f more
    const double scale = (double)wg / A.r.temperature, toS = scale / sum.S;
    ends->m = sum.m;
    ends->base = (float)(toS * (b * (H - lnS) - f));
    ends->slope = (float)(toS * b * LN_2);
    ends->at_token = (float)(scale * (f + exp(lp) * (b * (lp + H) - f)));
    ends->nothing = 0;
    return loss;
}

// A row a workgroup, read twice where its gradient is wanted: for the sums, and for the gradient.
template <int TH, int KIND, bool ENT, typename ElemT>
__global__ __launch_bounds__(TH) void loss_rows_kernel(const Args A) {
    constexpr int EPV = 16 / sizeof(ElemT), WAVES = TH / 64;
    constexpr bool LIST = KIND == DISTILL;
    __shared__ Part part[WAVES];
    __shared__ Ends ends;
    __shared__ uint32_t listed[LIST ? CHUNK / 32 : 1];
    __shared__ int32_t entry_id[LIST ? TEACHER_MAX : 1];
    __shared__ float entry_x[LIST ? TEACHER_MAX : 1], entry_f[LIST ? TEACHER_MAX : 1];
    __shared__ uint32_t flags;                             // 1: an entry counts, 2: an id is beyond V, 4: an id is listed twice
    __shared__ float to_listed;                            // a listed token's gradient: its 2^y times this, and the entries' own
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / 64), lane = tid % 64;
    const int32_t V = A.r.V, n_pieces = (V + EPV - 1) / EPV;
    float g = 1.0f;
    if (A.g) {
        g = *A.g;
        if (A.held && g == 1.0f) return;
    }
    if (LIST) {
        for (int i = tid; i < CHUNK / 32; i += TH) listed[i] = 0;
        if (tid == 0) flags = 0;
        __syncthreads();
    }
    for (int64_t row = blockIdx.x; row < A.r.rows; row += gridDim.x) {
        const ElemT *const logits = (const ElemT *)A.r.logits + row * A.r.row_stride_elems;
        const uint32_t *const mask = A.r.mask ? A.r.mask + row * A.W : nullptr;
        ElemT *const grad = (ElemT *)A.grad + row * A.grad_stride;
        const float w = A.r.weight && KIND != LOGPROB ? A.r.weight[row] : 1.0f, wg = w * g;
        int64_t t = -1;
        float x_t = -INFINITY;
        bool looked = true;                                // the row is read
        if (LIST) {
            for (int k = tid; k < A.K; k += TH) {
                const int64_t id = id_at(A, row * A.K + k);
                float x = -INFINITY;
                if (id >= 0 && id < V && allowed(mask, id)) x = of_bits(logits[id]);
                const bool counts = x != -INFINITY;
                entry_id[k] = counts ? (int32_t)id : -1;
                entry_x[k] = x;
                if (counts || id >= V) atomicOr(&flags, id >= V ? 2u : 1u);
            }
            __syncthreads();
            looked = flags != 0;
        } else {
            t = id_at(A, row);
            looked = t >= 0;
            if (looked && t < V && allowed(mask, t)) x_t = of_bits(logits[t]);
        }
        if (!looked) {                                     // (alike in the whole workgroup)
            if (tid == 0 && A.results) {
                if (KIND != LOGPROB) A.r.losses[row] = 0.0f;
                if (KIND != DISTILL) A.logprobs[row] = 0.0f;
                if (KIND == LOGPROB) A.stats[2 * row] = A.stats[2 * row + 1] = 0.0f;
                if (ENT) A.entropy[row] = 0.0f;
            }
            if (A.grad) {
                const float zeros[EPV] = {};
                for (int j = tid; j < n_pieces; j += TH) store_piece<EPV>(grad, (int64_t)j * EPV, V, zeros);
            }
            if (LIST) __syncthreads();                     // before the lists are written again
            continue;
        }
        Part mine{-FLT_MAX, 0.0f, 0.0f, 0.0f};
        for (int32_t from = 0; from < V; from += CHUNK) {  // (one turn, unless bits of listed tokens are wanted of more than CHUNK of them)
            const int32_t to = LIST ? min(V, from + CHUNK) : V;
            if (LIST) {
                if (from) {
                    __syncthreads();
                    for (int i = tid; i < CHUNK / 32; i += TH) listed[i] = 0;
                    __syncthreads();
                }
                for (int k = tid; k < A.K; k += TH) {
                    const int32_t id = entry_id[k];
                    if (id < from || id >= to) continue;
                    const uint32_t bit = 1u << (id & 31), was = atomicOr(&listed[(id - from) >> 5], bit);
                    if (was & bit) atomicOr(&flags, 4u);
                }
                __syncthreads();
            }
            for (int32_t j = from / EPV + tid; j < (to + EPV - 1) / EPV; j += TH) {
                const int64_t v = (int64_t)j * EPV;
                uint32_t bits = bits_of<EPV>(mask, v, V);
                if (LIST) bits &= ~(listed[(v - from) >> 5] >> (v & 31));
                float x[EPV], most = mine.m;
                load_piece<EPV>(logits, v, V, bits, x);
#pragma unroll
                for (int k = 0; k < EPV; k++) most = fmaxf(most, x[k]);
                if (most > mine.m) {
                    const float d = apart(mine.m, most, A.c), f = two_to(d);
                    if (ENT) mine.T = f * fmaf(mine.S, d, mine.T);
                    mine.S *= f;
                    mine.m = most;
                }
                float S = 0.0f, T = 0.0f;
#pragma unroll
                for (int k = 0; k < EPV; k++) {
                    const float y = (x[k] - mine.m) * A.c, e = two_to(y);
                    S += e;
                    if (ENT) T = fmaf(e, fmaxf(y, -1e4f), T);
                }
                mine.S += S;
                if (ENT) mine.T += T;
            }
            if (!LIST) break;
        }
        mine = join_wave(mine, A.c);
        if (lane == 0) part[wave] = mine;
        __syncthreads();
        if (wave == 0) {
            const Part sum = join_wave(lane < WAVES ? part[lane] : Part{-FLT_MAX, 0.0f, 0.0f, 0.0f}, A.c);
            if (KIND == POLICY) {
                Ends e;
                float logprob, entropy;
                const double loss = policy_row(A, sum, row, t, x_t, wg, &e, &logprob, &entropy);
                if (lane == 0) {
                    ends = e;
                    if (A.results) {
                        A.r.losses[row] = (float)loss;
                        A.logprobs[row] = logprob;
                        if (ENT) A.entropy[row] = entropy;
                    }
                }
            } else if (KIND == LOGPROB) {
                const bool nan = t >= V || sum.S != sum.S;
                const double lp = nan ? (double)NAN : x_t == -INFINITY ? -INFINITY : ((double)x_t - sum.m) / A.r.temperature - log((double)sum.S);
                if (lane == 0) {
                    A.logprobs[row] = lp < -FLT_MAX && x_t != -INFINITY ? -FLT_MAX : (float)lp;
                    A.stats[2 * row] = sum.m;
                    A.stats[2 * row + 1] = sum.S == 0.0f ? 0.0f : 1.0f / sum.S;
                }
            } else {
                // the teacher's side
                double most = -INFINITY, total = 0.0;
                auto value = [&](int k) { const int64_t i = row * A.K + k; return (double)(A.values_dtype == 0 ? ((const float *)A.values)[i] : of_bits(((const uint16_t *)A.values)[i])); };
                const double T = A.r.temperature;
                float x_most = sum.m;
                for (int k = lane; k < A.K; k += 64) {
                    if (entry_id[k] < 0) continue;
                    x_most = fmaxf(x_most, entry_x[k]);
                    most = fmax(most, value(k));
                }
                x_most = zf::wave_max(x_most);
                most = A.rest ? 0.0 : wave_max(most);
                auto first = [&](int k) {                  // of the entries of one token
                    if (flags & 4u) for (int i = 0; i < k; i++) if (entry_id[i] == entry_id[k]) return false;
                    return true;
                };
                double S_listed = 0.0;
                for (int k = lane; k < A.K; k += 64) {
                    if (entry_id[k] < 0) continue;
                    const double v = value(k);
                    total += v == -INFINITY ? 0.0 : exp(A.rest ? v : (v - most) / T);
                    if (first(k)) S_listed += two_to((entry_x[k] - x_most) * A.c);
                }
                total = wave_sum(total);
                const double S_rest = sum.S, rest_down = ((double)sum.m - x_most) / T;       // ln of what brings S_rest to the same reference
                const double S = wave_sum(S_listed) + (S_rest == 0.0 ? 0.0 : S_rest * exp(rest_down)), lnS = log(S);
                const double inv = A.rest || total == 0.0 ? 1.0 : 1.0 / total, ln_total = A.rest || total == 0.0 ? 0.0 : log(total);
                double loss = 0.0, all = 0.0;
                const double scale = (double)wg / T;
                for (int k = lane; k < A.K; k += 64) {
                    if (entry_id[k] < 0) continue;
                    const double v = value(k), ln_q = A.rest ? v : (v - most) / T - ln_total, q = v == -INFINITY ? 0.0 : exp(A.rest ? v : (v - most) / T) * inv;
                    if (q != 0.0) loss += q * (ln_q - (((double)entry_x[k] - x_most) / T - lnS));
                    all += q;
                    entry_f[k] = (float)(-q * scale);
                }
                loss = wave_sum(loss);
                all = wave_sum(all);
                double q_rest = A.rest ? 1.0 - all : 0.0;
                if (q_rest < 0.0 || S_rest == 0.0) q_rest = 0.0;
                const double ln_rest = log(S_rest) + rest_down - lnS, p_rest = S_rest == 0.0 ? 0.0 : exp(ln_rest);
                if (q_rest != 0.0) loss += q_rest * (log(q_rest) - ln_rest);
                const bool nan = (flags & 2u) || S != S;
                all += q_rest;
                if (lane == 0) {
                    ends.m = sum.m;
                    ends.base = nan ? NAN : S_rest == 0.0 ? 0.0f : (float)(scale * (all * p_rest - q_rest) / S_rest);
                    ends.slope = 0.0f;
                    ends.nothing = 0;
                    ends.at_token = x_most;
                    to_listed = nan ? NAN : (float)(scale * all / S);
                    if (A.results) A.r.losses[row] = nan ? NAN : (float)loss;
                }
            }
        }
        if (KIND == LOGPROB) {
            __syncthreads();                               // before part is written again
            continue;
        }
        __syncthreads();
        if (A.grad) {
            const float m = ends.m, base = ends.base, slope = ends.slope;
            const bool zero = ends.nothing, look = !(fabsf(base) + 2e4f * fabsf(slope) < INFINITY);   // 0 times what is not finite is not 0
            for (int32_t j = tid; j < n_pieces; j += TH) {
                const int64_t v = (int64_t)j * EPV;
                float x[EPV], d[EPV];
                load_piece<EPV>(logits, v, V, zero ? 0u : bits_of<EPV>(mask, v, V), x);
#pragma unroll
                for (int k = 0; k < EPV; k++) {
                    const float y = (x[k] - m) * A.c, e = two_to(y), near = fmaxf(y, -1e4f);
                    d[k] = ENT ? (look ? fmaf(e * near, slope, e * base) : e * fmaf(slope, near, base)) : e * base;
                    if (zero || (look && x[k] == -INFINITY)) d[k] = 0.0f;
                }
                store_piece<EPV>(grad, v, V, d);
            }
            if (!LIST) {                                   // by the thread that has just written the token's piece
                if (x_t != -INFINITY && tid == (int)(t / EPV % TH) && t < V) store_element(grad + t, ends.at_token);
            } else {
                __syncthreads();
                const float x_most = ends.at_token;
                for (int k = tid; k < A.K; k += TH) {
                    const int32_t id = entry_id[k];
                    if (id < 0) continue;
                    float f = entry_f[k];
                    if (flags & 4u) {                      // the entries of the same token in order, by the first
                        bool first = true;
                        for (int i = 0; i < k; i++) first &= entry_id[i] != id;
                        if (!first) continue;
                        for (int i = k + 1; i < A.K; i++) if (entry_id[i] == id) f += entry_f[i];
                    }
                    store_element(grad + id, fmaf(two_to((entry_x[k] - x_most) * A.c), to_listed, f));
                }
            }
        }
        if (LIST) {
            __syncthreads();
            if (V <= CHUNK) for (int k = tid; k < A.K; k += TH) { if (entry_id[k] >= 0) listed[entry_id[k] >> 5] = 0; }
            else for (int i = tid; i < CHUNK / 32; i += TH) listed[i] = 0;
            if (tid == 0) flags = 0;
            __syncthreads();
        }
    }
}

// loss = sum of weight x losses, in 64 bits and one order.
__device__ __forceinline__ void sum_losses(const float *losses, const float *weight, int64_t n, float *loss, double *of_wave) {
    double sum = 0.0;
    for (int64_t i = threadIdx.x; i < n; i += blockDim.x) sum += (weight ? (double)weight[i] : 1.0) * losses[i];
    sum = wave_sum(sum);
    if (threadIdx.x % 64 == 0) of_wave[threadIdx.x / 64] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        sum = 0.0;
        for (int w = 0; w < (int)blockDim.x / 64; w++) sum += of_wave[w];
        *loss = (float)sum;
    }
}
__global__ __launch_bounds__(1024) void total_kernel(const float *losses, const float *weight, int64_t n, float *loss) {
    __shared__ double of_wave[16];
    sum_losses(losses, weight, n, loss, of_wave);
}

// ---- preferences ----
__device__ __forceinline__ int64_t offset_at(const zf_preference_args &p, int64_t s) { return p.offset_bytes == 8 ? ((const int64_t *)p.offsets)[s] : ((const int32_t *)p.offsets)[s]; }
__device__ __forceinline__ int64_t token_at(const zf_preference_args &p, int64_t row) { return p.token_bytes == 8 ? ((const int64_t *)p.tokens)[row] : ((const int32_t *)p.tokens)[row]; }

// A pair a workgroup: the rows' log ratios in 64 bits, in one order; the first half of the wavefronts takes the one sequence, the second the other.
__global__ __launch_bounds__(256) void pairs_kernel(const zf_preference_args p) {
    __shared__ double sums[4], counts[4];
    const int half = threadIdx.x / 128, lane = threadIdx.x % 128;
    for (int64_t pair = blockIdx.x; pair < p.pairs; pair += gridDim.x) {
        const int64_t o0 = offset_at(p, 2 * pair), o1 = offset_at(p, 2 * pair + 1), o2 = offset_at(p, 2 * pair + 2);
        const bool fits = 0 <= o0 && o0 <= o1 && o1 <= o2 && o2 <= p.r.rows;
        const int64_t begin = half ? o1 : o0, end = fits ? (half ? o2 : o1) : begin;
        double sum = 0.0, n = 0.0;
        for (int64_t row = begin + lane; row < end; row += 128) {
            if (token_at(p, row) < 0) continue;
            sum += p.ref_logprobs ? (double)p.logprobs[row] - p.ref_logprobs[row] : (double)p.logprobs[row];
            n += 1.0;
        }
        sum = wave_sum(sum);
        n = wave_sum(n);
        if (threadIdx.x % 64 == 0) { sums[threadIdx.x / 64] = sum; counts[threadIdx.x / 64] = n; }
        __syncthreads();
        if (threadIdx.x == 0) {
            double chosen = sums[0] + sums[1], rejected = sums[2] + sums[3];
            double n0 = 1.0, n1 = 1.0;
            if (p.average) { n0 = fmax(counts[0] + counts[1], 1.0); n1 = fmax(counts[2] + counts[3], 1.0); }
            chosen *= p.beta / n0;
            rejected *= p.beta / n1;
            const double h = chosen - rejected, s = p.label_smoothing;
            // -ln sigma(h) = max(-h, 0) + ln(1 + e^-|h|)
            const double tail = log1p(exp(-fabs(h)));
            double loss = (1.0 - s) * (fmax(-h, 0.0) + tail), slope = -(1.0 - s) / (1.0 + exp(h));
            if (s != 0.0) { loss += s * (fmax(h, 0.0) + tail); slope += s / (1.0 + exp(-h)); }
            const bool nan = !fits || h != h;
            p.r.losses[pair] = nan ? NAN : (float)loss;
            p.chosen[pair] = fits ? (float)chosen : NAN;
            p.rejected[pair] = fits ? (float)rejected : NAN;
            const double c = nan ? (double)NAN : slope * p.beta * (p.r.weight ? p.r.weight[pair] : 1.0);
            p.slopes[2 * pair] = (float)(c / n0);
            p.slopes[2 * pair + 1] = (float)(-c / n1);
        }
        __syncthreads();
    }
}

// The gradient of preferences: a row's slope is its sequence's.
template <int TH, typename ElemT>
__global__ __launch_bounds__(TH) void preference_grad_kernel(const zf_preference_args p, const float *g, float c, int32_t W, void *grad_, int64_t grad_stride) {
    constexpr int EPV = 16 / sizeof(ElemT);
    const int tid = threadIdx.x;
    const int32_t V = p.r.V, n_pieces = (V + EPV - 1) / EPV;
    for (int64_t row = blockIdx.x; row < p.r.rows; row += gridDim.x) {
        const ElemT *const logits = (const ElemT *)p.r.logits + row * p.r.row_stride_elems;
        ElemT *const grad = (ElemT *)grad_ + row * grad_stride;
        const uint32_t *const mask = p.r.mask ? p.r.mask + row * W : nullptr;
        int64_t low = 0, high = 2 * p.pairs;               // the last sequence that begins at or before the row
        while (low < high) {
            const int64_t mid = (low + high + 1) / 2;
            if (offset_at(p, mid) <= row) low = mid; else high = mid - 1;
        }
        const int64_t t = token_at(p, row);
        const bool counts = t >= 0 && low < 2 * p.pairs && offset_at(p, low) <= row && row < offset_at(p, low + 1) && p.logprobs[row] != -INFINITY;
        const float m = p.stats[2 * row], inv_S = p.stats[2 * row + 1], f = counts ? (float)((double)p.slopes[low] * *g / p.r.temperature) : 0.0f;
        const float base = -f * inv_S;
        const bool look = !(fabsf(base) < INFINITY);
        for (int32_t j = tid; j < n_pieces; j += TH) {
            const int64_t v = (int64_t)j * EPV;
            float x[EPV], d[EPV];
            load_piece<EPV>(logits, v, V, counts ? bits_of<EPV>(mask, v, V) : 0u, x);
#pragma unroll
            for (int k = 0; k < EPV; k++) {
                d[k] = two_to((x[k] - m) * c) * base;
                if (!counts || (look && x[k] == -INFINITY)) d[k] = 0.0f;
            }
            if (counts && t / EPV == j) {
#pragma unroll
                for (int k = 0; k < EPV; k++) if (t % EPV == k) d[k] += f;
            }
            store_piece<EPV>(grad, v, V, d);
        }
    }
}

int grid_of(int64_t n) { return (int)std::min<int64_t>(n, 1 << 16); }
template <int KIND, bool ENT>
void rows_of(const Args &A, hipStream_t s) {
    const bool small = A.r.V * (A.r.dtype == 0 ? 4 : 2) <= 32768;
    const dim3 grid(grid_of(A.r.rows));
    if (A.r.dtype == 0) {
        if (small) hipLaunchKernelGGL((loss_rows_kernel<256, KIND, ENT, uint32_t>), grid, dim3(256), 0, s, A);
        else hipLaunchKernelGGL((loss_rows_kernel<1024, KIND, ENT, uint32_t>), grid, dim3(1024), 0, s, A);
    } else {
        if (small) hipLaunchKernelGGL((loss_rows_kernel<256, KIND, ENT, uint16_t>), grid, dim3(256), 0, s, A);
        else hipLaunchKernelGGL((loss_rows_kernel<1024, KIND, ENT, uint16_t>), grid, dim3(1024), 0, s, A);
    }
}
Args common(const zf_loss_rows &r, const LossGrad &g) {
    Args A{};
    A.r = r;
    A.W = (r.V + 31) / 32;
    A.c = (float)(1.4426950408889634 / r.temperature);
    A.grad = g.grad; A.grad_stride = g.stride; A.g = g.g; A.held = g.held; A.results = !g.g;
    return A;
}
void total(const zf_loss_rows &r, int64_t n, hipStream_t s) { hipLaunchKernelGGL(total_kernel, dim3(1), dim3(1024), 0, s, r.losses, r.weight, n, r.loss); }

}  // namespace

hipError_t launch_distill(const zf_distill_args &a, const LossGrad &g, hipStream_t s) {
    Args A = common(a.r, g);
    A.K = a.n_listed; A.ids = a.ids; A.id_bytes = a.id_bytes; A.values = a.values; A.values_dtype = a.values_dtype; A.rest = a.rest;
    if (a.r.rows) rows_of<DISTILL, false>(A, s);
    if (A.results) total(a.r, a.r.rows, s);
    return hipGetLastError();
}

hipError_t launch_policy(const zf_policy_args &a, const LossGrad &g, hipStream_t s) {
    Args A = common(a.r, g);
    A.ids = a.tokens; A.id_bytes = a.token_bytes; A.old_logprobs = a.old_logprobs; A.advantages = a.advantages; A.ref = a.kl_weight != 0.0 ? a.ref_logprobs : nullptr;
    A.lowest = 1.0 - a.clip_low; A.highest = 1.0 + a.clip_high; A.kl_weight = a.kl_weight; A.entropy_weight = a.entropy_weight;
    A.logprobs = a.logprobs; A.entropy = a.entropy;
    if (a.r.rows) { if (a.entropy) rows_of<POLICY, true>(A, s); else rows_of<POLICY, false>(A, s); }
    if (A.results) total(a.r, a.r.rows, s);
    return hipGetLastError();
}

hipError_t launch_preference(const zf_preference_args &a, hipStream_t s) {
    Args A = common(a.r, LossGrad{});
    A.ids = a.tokens; A.id_bytes = a.token_bytes; A.logprobs = a.logprobs; A.stats = a.stats;
    if (a.r.rows) rows_of<LOGPROB, false>(A, s);
    if (a.pairs) hipLaunchKernelGGL(pairs_kernel, dim3(grid_of(a.pairs)), dim3(256), 0, s, a);
    total(a.r, a.pairs, s);
    return hipGetLastError();
}

hipError_t launch_preference_backward(const zf_preference_args &a, const LossGrad &g, hipStream_t s) {
    const int32_t W = (a.r.V + 31) / 32;
    const float c = (float)(1.4426950408889634 / a.r.temperature);
    if (a.r.rows == 0) return hipSuccess;
    if (a.r.dtype == 0) hipLaunchKernelGGL((preference_grad_kernel<1024, uint32_t>), dim3(grid_of(a.r.rows)), dim3(1024), 0, s, a, g.g, c, W, g.grad, g.stride);
    else hipLaunchKernelGGL((preference_grad_kernel<1024, uint16_t>), dim3(grid_of(a.r.rows)), dim3(1024), 0, s, a, g.g, c, W, g.grad, g.stride);
    return hipGetLastError();
}

}  // namespace zf
