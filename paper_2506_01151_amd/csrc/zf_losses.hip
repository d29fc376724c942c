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

__host__ __device__ constexpr int own_words_of(int pieces, int epv) { return (pieces * epv + 31) / 32; }      // words of a row's mask that a thread brings
__host__ __device__ constexpr int early_of(int pieces) { return pieces <= 16 ? 3 : 0; }                       // (more pieces leave no registers)
enum Kind { POLICY, DISTILL, LOGPROB };       // LOGPROB: of preferences' tokens alone, and what their gradient needs

static const int THREADS_MAX = 1024;
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
    int32_t once;                              // logits and gradient are larger than the last-level cache: they pass it by
    const float *old_logprobs, *advantages, *ref;
    double lowest, highest, kl_weight, entropy_weight;
    float *logprobs, *entropy;
    const void *offsets;                       // preferences: [sequences + 1]
    int64_t sequences;
    int32_t offset_bytes;
    float4 *found;                             // [rows], of preferences
};

struct Part { float m, S, T, pad; };
struct Ends {                                  // what the gradient of a row is made from
    float m, base, slope, at_token;            // d = 2^((x - m) c) (base + slope y); the given token's own
};

// Over a wavefront, to all lanes, by moves between lanes as zf_logit_rows.h has them for 32 bits.
__device__ __forceinline__ double from_lane(double x, int lane) {
    const uint64_t b = __double_as_longlong(x);
    return __longlong_as_double((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)b, lane) | (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(b >> 32), lane) << 32);
}
template <int CTRL, int ROWS = 0xF> __device__ __forceinline__ double plus_moved(double x) {
    const uint64_t b = __double_as_longlong(x);
    return x + __longlong_as_double((uint64_t)moved<CTRL, ROWS>(0u, (uint32_t)b) | (uint64_t)moved<CTRL, ROWS>(0u, (uint32_t)(b >> 32)) << 32);
}
__device__ __forceinline__ double wave_sum(double x) {
    x = plus_moved<0x111>(x);
    x = plus_moved<0x112>(x);
    x = plus_moved<0x114>(x);
    x = plus_moved<0x118>(x);
    x = plus_moved<0x142, 0xA>(x);
    x = plus_moved<0x143, 0xC>(x);
    return from_lane(x, 63);
}
// What is alike in the whole workgroup and not written by the kernel comes through the scalar unit, whose loads are waited for apart from a row's pieces: a vector load behind them would make everything that is
// asked for and written before it be waited for.
#define CONSTANT __attribute__((address_space(4)))
template <typename T> __device__ __forceinline__ T alike(const T *p) { return *(const CONSTANT T *)(uintptr_t)p; }
__device__ __forceinline__ int64_t token_at(const Args &A, int64_t row) { return A.id_bytes == 8 ? alike((const int64_t *)A.ids + row) : alike((const int32_t *)A.ids + row); }
__device__ __forceinline__ int64_t id_at(const Args &A, int64_t i) { return A.id_bytes == 8 ? ((const int64_t *)A.ids)[i] : ((const int32_t *)A.ids)[i]; }
__device__ __forceinline__ bool allowed(const uint32_t *mask_row, int64_t v) { return !mask_row || ((mask_row[v >> 5] >> (v & 31)) & 1u); }

// Sums around another reference join by 2^((m' - m) c).  The references are finite (a part without anything has -FLT_MAX and sums of zero) or +inf
// (whose sum is NaN), and nothing times -inf is nothing: 1e4 stands for all that is below 2^-126.
__device__ __forceinline__ float apart(float m, float whole, float c) { return m == whole ? 0.0f : fmaxf((m - whole) * c, -1e4f); }
__device__ __forceinline__ Part join_wave(Part a, float c) {
    const float m = wave_max(a.m), d = apart(a.m, m, c), f = two_to(d);
    return Part{m, wave_sum(f * a.S), wave_sum(f * fmaf(a.S, d, a.T)), 0.0f};
}

// A row is whole pieces of 16 bytes, and its last V % EPV elements, which the first threads take one each.
template <int EPV, typename ElemT>
__device__ __forceinline__ void numbers(const u32x4 &r, float (&x)[EPV]) {
#pragma unroll
    for (int k = 0; k < EPV; k++) x[k] = __uint_as_float(sizeof(ElemT) == 4 ? r[k % 4] : k & 1 ? r[k / 2] & 0xFFFF0000u : r[k / 2] << 16);
}
// -inf in the places of a piece that `bits` has none of
template <int EPV, typename ElemT>
__device__ __forceinline__ void forbid(u32x4 &r, uint32_t bits) {
    constexpr uint32_t NONE = sizeof(ElemT) == 4 ? 0xFF800000u : 0xFF80FF80u;
#pragma unroll
    for (int k = 0; k < 4; k++) {
        uint32_t yes;
        if (sizeof(ElemT) == 4) yes = (uint32_t)__builtin_amdgcn_sbfe((int)bits, k, 1);
        else {
            const uint32_t low = (uint32_t)__builtin_amdgcn_sbfe((int)bits, 2 * k, 1), high = (uint32_t)__builtin_amdgcn_sbfe((int)bits, 2 * k + 1, 1);
            yes = (low & 0xFFFFu) | (high & 0xFFFF0000u);
        }
        r[k] = (r[k] & yes) | (NONE & ~yes);
    }
}
#define GLOBAL __attribute__((address_space(1)))
// (Statements of nothing at either end of a branch: else the compiler makes the two accesses one, an ordinary one.)
template <typename ElemT>
__device__ __forceinline__ void store_raw(GLOBAL char *to, u32x4 v, bool once) {
    GLOBAL typename Piece<ElemT>::type *const at = (GLOBAL typename Piece<ElemT>::type *)to;
    if (once) {
        asm volatile("");
        __builtin_nontemporal_store(v, at);
        asm volatile("");
    } else *at = v;
}
template <typename ElemT>
__device__ __forceinline__ void store_raw(ElemT *to, u32x4 v, bool once) { store_raw<ElemT>((GLOBAL char *)to, v, once); }
template <typename ElemT>
__device__ __forceinline__ void store_element(ElemT *to, float x) {
    if (sizeof(ElemT) == 4) *(float *)to = x;
    else *(__bf16 *)to = (__bf16)x;
}
// U pieces from memory at a distance of TH, of whose places `bits` are wanted: all are asked for before the first is looked at, and nothing is where there are none.
template <int U, int EPV, typename ElemT>
__device__ __forceinline__ void load_pieces(const int TH, const ElemT *at, const uint32_t (&bits)[U], bool once, u32x4 (&r)[U]) {
    constexpr uint32_t NONE = sizeof(ElemT) == 4 ? 0xFF800000u : 0xFF80FF80u;
#pragma unroll
    for (int u = 0; u < U; u++) r[u] = u32x4{NONE, NONE, NONE, NONE};
    if (once) {
        asm volatile("");
#pragma unroll
        for (int u = 0; u < U; u++) if (bits[u]) r[u] = __builtin_nontemporal_load(reinterpret_cast<const typename Piece<ElemT>::type *>(at + u * TH * EPV));
        asm volatile("");
    } else {
#pragma unroll
        for (int u = 0; u < U; u++) if (bits[u]) r[u] = *reinterpret_cast<const typename Piece<ElemT>::type *>(at + u * TH * EPV);
    }
}
template <int EPV>
__device__ __forceinline__ uint32_t bits_of(const uint32_t *mask_row, int64_t v) {
    constexpr uint32_t FULL = (1u << EPV) - 1u;
    return mask_row ? (mask_row[v >> 5] >> (v & 31)) & FULL : FULL;
}

// What is known of a row beside its logits, asked for ahead of its turn.
struct Head {
    int64_t t;                                 // the given token
    float x, weight, old_logprob, advantage, ref;          // its logit, -inf where it is not allowed
    uint32_t raw, word, shift;                 // the four bytes that hold the logit, and where; of the mask
    int32_t sequence;                          // of preferences: the row's; PADDING, or NOWHERE: it has a token and no sequence
};
static const int32_t PADDING = -1, NOWHERE = -2;
// What a policy's loss makes of a row, by every lane of a wavefront alike.  Returns the row's loss.
__device__ __forceinline__ double policy_row(const Args &A, const Part &sum, const Head &h, float wg, Ends *ends, float *logprob, float *entropy) {
    const double lnS = log((double)sum.S);
    const bool nan = h.t >= A.r.V || sum.S != sum.S;
    const bool counts = nan || h.x != -INFINITY;
    *entropy = nan ? NAN : sum.S == 0.0f ? 0.0f : (float)(lnS - (double)LN_2 * sum.T / sum.S);
    *ends = Ends{sum.m, 0.0f, 0.0f, 0.0f};
    *logprob = -INFINITY;
    if (!counts) return 0.0;
    const double lp = nan ? (double)NAN : ((double)h.x - sum.m) / A.r.temperature - lnS;
    *logprob = lp < -FLT_MAX ? -FLT_MAX : (float)lp;
    const double a = h.advantage, ratio = exp(lp - h.old_logprob);
    const double kept = ratio < A.lowest ? A.lowest : ratio > A.highest ? A.highest : ratio;
    const bool clipped = kept * a < ratio * a;
    double loss = -(clipped ? kept * a : ratio * a), f = clipped ? 0.0 : -ratio * a;
    if (A.ref) {
        const double d = h.ref - lp, up = expm1(d);
        loss += A.kl_weight * (up - d);
        f -= A.kl_weight * up;
    }
    const double b = A.entropy ? A.entropy_weight : 0.0, H = *entropy;
    loss -= b * H;
    // p (-f + b (ln p + H)), ln p = ln 2 y - ln S; for the token itself f more
    const double scale = (double)wg / A.r.temperature, toS = scale / sum.S;
    ends->base = (float)(toS * (b * (H - lnS) - f));
    ends->slope = (float)(toS * b * LN_2);
    ends->at_token = (float)(scale * (f + (double)two_to((h.x - sum.m) * A.c) / sum.S * (b * (lp + H) - f)));
    return loss;
}

// ---- a teacher's listed tokens ----
// Each wavefront sums 64 entries around its own largest logit x_most and value v_most (with `rest` 0); the sums join as those of a row do.
struct Teacher {
    double total, mixed, S;                    // of e = e^((v - v_most) / T):  sum e,  sum e ((v - v_most) / T - (x - x_most) / T);  sum 2^((x - x_most) c) over different tokens
    double v_most;
    float x_most;
    int32_t some;
    double to_shares;                          // the call's factor and what makes e the entry's share of the whole
};
struct EntriesEnd {
    float x_most, to_listed;                   // a listed token's gradient: its 2^((x - x_most) c) times this, and the entries' own
    uint32_t flags;                            // 1: an entry counts, 2: an id is beyond V, 4: a token is listed twice
    uint32_t pad;
};
struct Entries {                               // in LDS, room for the call's n_listed
    Teacher *part;                             // [n / 64]
    EntriesEnd *end;
    int32_t *id;                               // [n]; -1: does not count
    float *x, *v;                              // v: the teacher's value, then e (rounded by u: it makes the entry's gradient, which is 32 bits at most; sums are of what it was made from)
    __device__ __forceinline__ Entries(char *at, int K) {
        part = (Teacher *)at;
        end = (EntriesEnd *)(part + (K + 63) / 64);
        id = (int32_t *)(end + 1);
        x = (float *)(id + K);
        v = x + K;
    }
};
__host__ __device__ __forceinline__ int entries_bytes(int K) { return ((K + 63) / 64 * (int)sizeof(Teacher) + (int)sizeof(EntriesEnd) + 12 * K + 15) / 16 * 16; }

// An entry as memory has it, asked for ahead of its turn.
struct Entry {
    int32_t id;                                // -1: none, V: beyond the vocabulary
    float v, x;                                // x: the token's logit, whether it is allowed or not
    uint32_t word;                             // of the mask
};
__device__ __forceinline__ void ask_id(const Args &A, int64_t row, int k, Entry &e) {
    const int64_t at = row * A.K + k;
    const int64_t id = id_at(A, at);
    e.id = id < 0 ? -1 : id < A.r.V ? (int32_t)id : A.r.V;
    e.v = A.values_dtype == 0 ? ((const float *)A.values)[at] : of_bits(((const uint16_t *)A.values)[at]);
}
template <typename ElemT>
__device__ __forceinline__ void ask_logit(const Args &A, const ElemT *logits, const uint32_t *mask, Entry &e) {
    e.x = -INFINITY;
    e.word = ~0u;
    if (e.id < 0 || e.id >= A.r.V) return;
    e.x = of_bits(logits[e.id]);
    if (mask) e.word = mask[e.id >> 5];
}
// Whether it counts
__device__ __forceinline__ bool list_entry(const Args &A, const Entry &e, int k, const Entries &E) {
    const bool inside = e.id >= 0 && e.id < A.r.V && ((e.word >> (e.id & 31)) & 1u), counts = inside && e.x != -INFINITY;
    E.id[k] = counts ? (int32_t)e.id : -1;
    E.x[k] = inside ? e.x : -INFINITY;
    E.v[k] = e.v;
    if (counts || e.id >= A.r.V) atomicOr(&E.end->flags, e.id >= A.r.V ? 2u : 1u);
    return counts;
}
__device__ __forceinline__ bool first_of(const Entries &E, int k) {      // of the entries of one token
    if (E.end->flags & 4u) for (int i = 0; i < k; i++) if (E.id[i] == E.id[k]) return false;
    return true;
}
// Entries 64 wave .. 64 wave + 63, by one wavefront; every entry has been read.
__device__ __forceinline__ void sum_entries(const Args &A, int wave, int lane, const Entries &E) {
    const int k = wave * 64 + lane;
    const bool counts = k < A.K && E.id[k] >= 0;
    const float x = counts ? E.x[k] : -INFINITY, x_most = wave_max(x);
    const double v = counts ? (double)E.v[k] : -INFINITY, T = A.r.temperature;
    const double v_most = A.rest ? 0.0 : (double)wave_max((float)v);
    double ln = 0.0, e = 0.0, S = 0.0;
    if (v != -INFINITY) {
        ln = A.rest ? v : (v - v_most) / T;
        e = exp(ln);
    }
    if (k < A.K) E.v[k] = (float)e;
    const double mixed = e == 0.0 ? 0.0 : e * (ln - ((double)x - x_most) / T);
    if (counts && first_of(E, k)) S = two_to((x - x_most) * A.c);
    const Teacher t{wave_sum(e), wave_sum(mixed), wave_sum(S), v_most, x_most, __any(counts), 0.0};
    if (lane == 0) E.part[wave] = t;
}
// A row's end, from the sums over what is not listed; by every lane of one wavefront alike.  Returns the row's loss.
__device__ __forceinline__ double distill_row(const Args &A, const Part &sum, float wg, const Entries &E, Ends *ends) {
    const double T = A.r.temperature;
    const int lane = threadIdx.x % 64;
    Teacher t{0.0, 0.0, 0.0, -INFINITY, -INFINITY, 0, 0.0};
    for (int w = 0; w < (A.K + 63) / 64; w++) {
        const Teacher u = E.part[w];
        if (!u.some) continue;
        if (!t.some) { t = u; continue; }
        const double v = A.rest ? 0.0 : fmax(t.v_most, u.v_most);
        const float x = fmaxf(t.x_most, u.x_most);
        const double vt = t.v_most == v ? 0.0 : (t.v_most - v) / T, vu = u.v_most == v ? 0.0 : (u.v_most - v) / T, ft = exp(vt), fu = exp(vu);
        const double xt = ((double)t.x_most - x) / T, xu = ((double)u.x_most - x) / T;
        t.mixed = (ft == 0.0 ? 0.0 : ft * (t.mixed + t.total * (vt - xt))) + (fu == 0.0 ? 0.0 : fu * (u.mixed + u.total * (vu - xu)));
        t.total = ft * t.total + fu * u.total;
        t.S = exp(xt) * t.S + exp(xu) * u.S;
        t.v_most = v;
        t.x_most = x;
    }
    const bool none = sum.S == 0.0f;                       // nothing that is not listed
    const float x_most = none ? t.x_most : fmaxf(t.x_most, sum.m);
    auto power = [](double ln) { return ln == 0.0 ? 1.0 : exp(ln); };
    const double S_rest = sum.S, down = none ? 0.0 : ((double)sum.m - x_most) / T, listed_down = t.some ? ((double)t.x_most - x_most) / T : 0.0;
    const double rest_to_S = power(down), S = S_rest * rest_to_S + t.S * power(listed_down);
    double q_rest = A.rest ? fmax(1.0 - t.total, 0.0) : 0.0;
    if (t.total != t.total) q_rest = NAN;
    if (none) q_rest = 0.0;
    // The whole workgroup waits here: lanes 0 to 3 take a logarithm and a reciprocal each at once, of S, S_R, sum e and q_R.
    const double of = lane == 0 ? S : lane == 1 ? S_rest : lane == 2 ? t.total : q_rest, ln = log(of), once = 1.0 / of;
    const double lnS = from_lane(ln, 0), by_S = from_lane(once, 0), by_rest = from_lane(once, 1);
    const double share = A.rest ? 1.0 : t.total == 0.0 ? 0.0 : from_lane(once, 2);
    double all = t.total * share;                          // sum of q
    double loss = t.total == 0.0 ? 0.0 : (A.rest ? t.mixed : t.mixed * share - from_lane(ln, 2)) + all * (lnS - listed_down);
    if (q_rest != 0.0) loss += q_rest * (from_lane(ln, 3) - (from_lane(ln, 1) + down - lnS));        // (ln p_R, also where p_R is 0 in 64 bits)
    const bool nan = (E.end->flags & 2u) || S != S;
    all += q_rest;
    const double scale = (double)wg / T;
    ends->m = sum.m;
    ends->base = nan ? NAN : none ? 0.0f : (float)(scale * (all * rest_to_S * by_S - q_rest * by_rest));
    ends->slope = 0.0f;
    ends->at_token = 0.0f;
    E.end->x_most = x_most;
    E.end->to_listed = nan ? NAN : (float)(scale * all * by_S);
    // (Equal also where both are -inf: entries that count, and none with a share.  Their difference would be NaN.)
    for (int w = 0; w < (A.K + 63) / 64; w++) E.part[w].to_shares = scale * share * (A.rest || !E.part[w].some || E.part[w].v_most == t.v_most ? 1.0 : exp((E.part[w].v_most - t.v_most) / T));
    return nan ? NAN : loss;
}
// The gradient of listed tokens, over what the row's own pass wrote there.
template <typename ElemT>
__device__ __forceinline__ void store_entries(const int TH, const Args &A, const Entries &E, ElemT *grad) {
    for (int k = threadIdx.x; k < A.K; k += TH) {
        const int32_t id = E.id[k];
        if (id < 0) continue;
        auto q = [&](int i) { return (float)(E.v[i] * E.part[i / 64].to_shares); };
        float f = q(k);
        if (E.end->flags & 4u) {                                // the entries of the same token in order, by the first
            if (!first_of(E, k)) continue;
            for (int i = k + 1; i < A.K; i++) if (E.id[i] == id) f += q(i);
        }
        store_element(grad + id, fmaf(two_to((E.x[k] - E.end->x_most) * A.c), E.end->to_listed, -f));
    }
}

// ---- preferences' sequences ----
__device__ __forceinline__ int64_t offset_at(const void *offsets, int32_t bytes, int64_t s) { return bytes == 8 ? ((const int64_t *)offsets)[s] : ((const int32_t *)offsets)[s]; }
// The sequence that a row belongs to, by one wavefront: the last that begins at or before it, if it ends behind it; -1: none.  64 offsets are looked at at a time.
__device__ __forceinline__ int32_t sequence_of(const Args &A, int64_t row, int lane) {
    int64_t first = 0, n = A.sequences;
    while (n > 0) {
        const int64_t step = (n + 63) / 64;
        const int64_t at = first + lane * step;
        const int64_t before = __popcll(__ballot(at < first + n && offset_at(A.offsets, A.offset_bytes, at < A.sequences ? at : 0) <= row));
        if (before == 0) return -1;
        const int64_t end = first + n;
        first += (before - 1) * step;
        if (step == 1) break;
        n = min(step, end - first);
    }
    return n > 0 && offset_at(A.offsets, A.offset_bytes, first) <= row && row < offset_at(A.offsets, A.offset_bytes, first + 1) ? (int32_t)first : -1;
}

// ---- a row's results ----
// The call's sum, where there is no other row; of more, total_kernel makes it.
__device__ __forceinline__ void store_loss(const Args &A, int64_t row, float loss, float weight) {
    A.r.losses[row] = loss;
    if (A.r.rows == 1) *A.r.loss = (float)((double)weight * loss);
}
template <int KIND>
__device__ __forceinline__ void ask_head(const Args &A, int64_t row, Head &h) {
    h.weight = A.r.weight && KIND != LOGPROB ? alike(A.r.weight + row) : 1.0f;
    if (KIND == POLICY) {
        h.old_logprob = alike(A.old_logprobs + row);
        h.advantage = alike(A.advantages + row);
        h.ref = A.ref ? alike(A.ref + row) : 0.0f;
    }
}
// The token's logit and its word of the mask, whether they will be wanted or not: neither waits for the other.
template <typename ElemT>
__device__ __forceinline__ void ask_token(const Args &A, const ElemT *logits, const uint32_t *mask, Head &h) {
    const int64_t at = h.t < 0 ? 0 : h.t < A.r.V ? h.t : A.r.V - 1;
    const uintptr_t place = (uintptr_t)(logits + at);
    h.raw = alike((const uint32_t *)(place & ~(uintptr_t)3));
    h.shift = sizeof(ElemT) == 4 ? 0 : place & 2 ? 0 : 16;
    h.word = mask ? alike(mask + (at >> 5)) : ~0u;
}
template <typename ElemT>
__device__ __forceinline__ void see_token(const Args &A, Head &h) {
    const uint32_t bits = h.raw << h.shift;
    h.x = h.t >= 0 && h.t < A.r.V && ((h.word >> (h.t & 31)) & 1u) ? of_bits(sizeof(ElemT) == 4 ? bits : bits & 0xFFFF0000u) : -INFINITY;
}
template <int KIND, bool ENT>
__device__ __forceinline__ void no_row(const Args &A, int64_t row, bool padding = true) {       // by one thread: a row that does not count
    if (!A.results) return;
    if (KIND != LOGPROB) store_loss(A, row, 0.0f, 0.0f);
    if (KIND == POLICY) A.logprobs[row] = 0.0f;
    if (KIND == LOGPROB) A.found[row] = float4{0.0f, 0.0f, 0.0f, __int_as_float(padding ? PADDING : NOWHERE)};
    if (ENT) A.entropy[row] = 0.0f;
}
// By one wavefront: what the sums over a row lead to.
template <int KIND, bool ENT>
__device__ __forceinline__ void finish_row(const Args &A, const Part &sum, int64_t row, const Head &h, float wg, int lane, const Entries &E, Ends &ends) {
    Ends e{};
    if (KIND == POLICY) {
        float logprob, entropy;
        const double loss = policy_row(A, sum, h, wg, &e, &logprob, &entropy);
        if (lane != 0) return;
        ends = e;
        if (!A.results) return;
        store_loss(A, row, (float)loss, h.weight);
        A.logprobs[row] = logprob;
        if (ENT) A.entropy[row] = entropy;
    } else if (KIND == LOGPROB) {
        const bool nan = h.t >= A.r.V || sum.S != sum.S;
        const double lp = nan ? (double)NAN : h.x == -INFINITY ? -INFINITY : ((double)h.x - sum.m) / A.r.temperature - log((double)sum.S);
        const float logprob = lp < -FLT_MAX && h.x != -INFINITY ? -FLT_MAX : (float)lp;
        if (lane == 0) A.found[row] = float4{sum.m, sum.S == 0.0f ? 0.0f : 1.0f / sum.S, logprob, __int_as_float(h.sequence)};
    } else {
        const double loss = distill_row(A, sum, wg, E, &e);
        if (lane != 0) return;
        ends = e;
        if (A.results) store_loss(A, row, (float)loss, h.weight);
    }
}

// ---- pieces of a row ----
template <bool ENT, int EPV>
__device__ __forceinline__ void add_piece(const float (&x)[EPV], float c, Part &sum) {
    float most = sum.m;
#pragma unroll
    for (int k = 0; k < EPV; k++) most = fmaxf(most, x[k]);
    if (most > sum.m) {
        const float d = apart(sum.m, most, c), f = two_to(d);
        if (ENT) sum.T = f * fmaf(sum.S, d, sum.T);
        sum.S *= f;
        sum.m = most;
    }
    float S = 0.0f, T = 0.0f;
#pragma unroll
    for (int k = 0; k < EPV; k++) {
        const float y = (x[k] - sum.m) * c, e = two_to(y);
        S += e;
        if (ENT) T = fmaf(e, fmaxf(y, -1e4f), T);
    }
    sum.S += S;
    if (ENT) sum.T += T;
}
// d = 2^y (base + slope y), y = (x - m) c.  For bf16 without the entropy's slope it is sign 2^(x c - K), K = m c - log2 |base|, in one multiply-add and the instruction that makes 2^: K is off by u |K|,
// d by as much, which is below a thousandth of its rounding to bf16 for |K| up to 100 or so (rows further out than 4,096 are taken the other way, see wild()).
struct Slope {
    float m, base, slope, K;
    uint32_t sign;                             // of two bf16 numbers
    __device__ __forceinline__ Slope(const Ends &e, float c) : m(e.m), base(e.base), slope(e.slope), K(fmaf(e.m, c, -__builtin_amdgcn_logf(fabsf(e.base)))), sign(e.base < 0.0f ? 0x80008000u : 0u) {}
    // What grad_of() makes of -inf: nothing times a factor, a zero with the factor's sign
    template <bool ENT, typename ElemT> __device__ __forceinline__ uint32_t zeros() const {
        if (sizeof(ElemT) == 2 && !ENT) return sign;
        const uint32_t of_factor = __float_as_uint(ENT ? fmaf(slope, -1e4f, base) : base) & 0x80000000u;
        return sizeof(ElemT) == 4 ? of_factor : of_factor | of_factor >> 16;
    }
};
template <bool ENT, int EPV, typename ElemT>
__device__ __forceinline__ u32x4 grad_of(const u32x4 &raw, const Slope &s, float c) {
    float x[EPV];
    numbers<EPV, ElemT>(raw, x);
    union { u32x4 v; bf16x2 b[4]; } o;
#pragma unroll
    for (int k = 0; k < EPV; k++) {
        if (EPV == 8 && !ENT) {
            x[k] = two_to(fmaf(x[k], c, -s.K));
            continue;
        }
        const float y = (x[k] - s.m) * c, e = two_to(y);
        x[k] = ENT ? e * fmaf(s.slope, fmaxf(y, -1e4f), s.base) : e * s.base;
    }
#pragma unroll
    for (int k = 0; k < EPV; k += 2) {
        if (EPV == 4) { o.v[k % 4] = __float_as_uint(x[k]); o.v[k % 4 + 1] = __float_as_uint(x[k + 1]); }
        else {
            o.b[k / 2 % 4] = bf16x2{(__bf16)x[k], (__bf16)x[k + 1]};
            if (!ENT) o.v[k / 2 % 4] |= s.sign;
        }
    }
    return o.v;
}
// Where factors are not finite, or near it -- 0 times them is not 0, and what is forbidden is to have 0 --, and where K would lose too much.
template <bool ENT, typename ElemT>
__device__ __forceinline__ bool wild(const Ends &e, float c) {
    return !(fabsf(e.base) + 2e4f * fabsf(e.slope) < INFINITY) || (sizeof(ElemT) == 2 && !ENT && e.base != 0.0f && !(fabsf(e.m * c) < 4096.0f));      // (of 0 K is infinite, and all d are 0)
}
template <bool ENT, int EPV>
__device__ __forceinline__ void grad_of_wild(const float (&x)[EPV], const Ends &ends, float c, float (&d)[EPV]) {
#pragma unroll
    for (int k = 0; k < EPV; k++) {
        const float y = (x[k] - ends.m) * c, e = two_to(y);
        d[k] = x[k] == -INFINITY ? 0.0f : ENT ? fmaf(e * fmaxf(y, -1e4f), ends.slope, e * ends.base) : e * ends.base;
    }
}
template <int EPV, typename ElemT>
__device__ __forceinline__ void store_zeros(const int TH, ElemT *grad, int32_t V, bool once) {
    for (int32_t j = threadIdx.x; j < V / EPV; j += TH) store_raw<ElemT>(grad + (int64_t)j * EPV, u32x4{0, 0, 0, 0}, once);
    if ((int)threadIdx.x < V % EPV) store_element(grad + V - V % EPV + threadIdx.x, 0.0f);
}

template <bool ENT, int EPV, typename ElemT>
__device__ __forceinline__ u32x4 wild_grad_of(const u32x4 &raw, const Ends &ends, float c) {
    float x[EPV], d[EPV];
    numbers<EPV, ElemT>(raw, x);
    grad_of_wild<ENT>(x, ends, c, d);
    union { u32x4 v; bf16x2 b[4]; } o;
#pragma unroll
    for (int k = 0; k < EPV; k += 2) {
        if (EPV == 4) { o.v[k % 4] = __float_as_uint(d[k]); o.v[k % 4 + 1] = __float_as_uint(d[k + 1]); }
        else o.b[k / 2 % 4] = bf16x2{(__bf16)d[k], (__bf16)d[k + 1]};
    }
    return o.v;
}
// A row's gradient, from memory, where wild() says so.
template <bool ENT, int EPV, typename ElemT>
__device__ __forceinline__ void wild_row(const int TH, const ElemT *logits, const uint32_t *mask, ElemT *grad, int32_t V, const Ends &ends, float c) {
    for (int32_t j = threadIdx.x; j < V / EPV; j += TH) {
        const uint32_t bits[1] = {bits_of<EPV>(mask, (int64_t)j * EPV)};
        u32x4 raw[1];
        load_pieces<1, EPV>(TH, logits + (int64_t)j * EPV, bits, false, raw);
        forbid<EPV, ElemT>(raw[0], bits[0]);
        store_raw<ElemT>(grad + (int64_t)j * EPV, wild_grad_of<ENT, EPV, ElemT>(raw[0], ends, c), false);
    }
}

template <int EPV>
__device__ __forceinline__ int writer_of(const int TH, int64_t v, int32_t V) { return v >= V - V % EPV ? (int)(v % EPV) : (int)(v / EPV % TH); }

// A row a workgroup, from memory: read for the sums, and again where its gradient is wanted.  For rows that do not fit a compute unit's registers, and calls without a gradient.  Bound by
// memory: log probabilities of 4,096 x 128,256 bf16, a quarter of them padding, 129 to 138 us (788 MB, 5.7 to 6.1 TB/s), of 501 x 152,064 fp32 40 (229 MB, 5.7); gradients under masks that
// leave 300 tokens, 1,024 x 152,064 fp32, 142: 623 MB are written, pieces without an allowed token are not read.
template <int KIND, bool ENT, typename ElemT>
__global__ __launch_bounds__(THREADS_MAX, 8) void loss_rows_kernel(const Args A) {
    constexpr int EPV = 16 / sizeof(ElemT), U = 4;
    const int TH = blockDim.x, WAVES = TH / 64;
    constexpr uint32_t FULL = (1u << EPV) - 1u;
    constexpr bool LIST = KIND == DISTILL;
    __shared__ Part part[THREADS_MAX / 64];
    __shared__ Ends shared_ends;
    __shared__ uint32_t listed[LIST ? CHUNK / 32 : 1];
    extern __shared__ __align__(16) char entries[];
    const Entries E(entries, A.K);
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / 64), lane = tid % 64;
    const int32_t V = A.r.V, n_pieces = V / EPV;
    float g = 1.0f;
    if (A.g) {
        g = *A.g;
        if (A.held && g == 1.0f) return;
    }
    if (LIST) {
        for (int i = tid; i < CHUNK / 32; i += TH) listed[i] = 0;
        if (tid == 0) E.end->flags = 0;
        __syncthreads();
    }
    for (int64_t row = blockIdx.x; row < A.r.rows; row += gridDim.x) {
        const ElemT *const logits = (const ElemT *)A.r.logits + row * A.r.row_stride_elems;
        const uint32_t *const mask = A.r.mask ? A.r.mask + row * A.W : nullptr;
        ElemT *const grad = (ElemT *)A.grad + row * A.grad_stride;
        Head h{-1, -INFINITY, 1.0f, 0.0f, 0.0f, 0.0f, 0, 0, 0, PADDING};
        ask_head<KIND>(A, row, h);
        const float wg = h.weight * g;
        bool looked;                                       // the row is read
        if (LIST) {
            for (int k = tid; k < A.K; k += TH) {
                Entry e;
                ask_id(A, row, k, e);
                ask_logit(A, logits, mask, e);
                list_entry(A, e, k, E);
            }
            __syncthreads();
            looked = E.end->flags != 0;
        } else {
            h.t = token_at(A, row);
            if (KIND == LOGPROB && h.t >= 0) h.sequence = sequence_of(A, row, lane);
            looked = h.t >= 0 && (KIND != LOGPROB || h.sequence >= 0);
            ask_token(A, logits, mask, h);
            see_token<ElemT>(A, h);
        }
        if (!looked) {                                     // (alike in the whole workgroup)
            if (tid == 0) no_row<KIND, ENT>(A, row, h.t < 0);
            if (A.grad) store_zeros<EPV>(TH, grad, V, A.once);
            if (LIST) __syncthreads();                     // before the lists are written again
            continue;
        }
        auto ask_words = [&](int32_t j, uint32_t (&words)[U]) {              // the mask's words that pieces j, j + TH .. lie in, a batch ahead of them
#pragma unroll
            for (int u = 0; u < U; u++) words[u] = mask ? mask[min(((int64_t)j + u * TH) * EPV, (int64_t)V - 1) >> 5] : ~0u;
        };
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
                    const int32_t id = E.id[k];
                    if (id < from || id >= to) continue;
                    const uint32_t bit = 1u << (id & 31), was = atomicOr(&listed[(id - from) >> 5], bit);
                    if (was & bit) atomicOr(&E.end->flags, 4u);
                }
                __syncthreads();
            }
            uint32_t words[U];
            ask_words(from / EPV + tid, words);
            for (int32_t j = from / EPV + tid; j < to / EPV; j += U * TH) {
                uint32_t bits[U];
                u32x4 raw[U];
#pragma unroll
                for (int u = 0; u < U; u++) {
                    const int64_t v = (int64_t)(j + u * TH) * EPV;
                    bits[u] = j + u * TH < to / EPV ? (words[u] >> (v & 31)) & FULL : 0u;
                    if (LIST && bits[u]) bits[u] &= ~(listed[(v - from) >> 5] >> (v & 31));
                }
                load_pieces<U, EPV>(TH, logits + (int64_t)j * EPV, bits, KIND == LOGPROB && A.once, raw);
                ask_words(j + U * TH, words);
#pragma unroll
                for (int u = 0; u < U; u++) {
                    if (!__any(bits[u] != 0)) continue;
                    if (__any(bits[u] != FULL)) forbid<EPV, ElemT>(raw[u], bits[u]);
                    float x[EPV];
                    numbers<EPV, ElemT>(raw[u], x);
                    add_piece<ENT>(x, A.c, mine);
                }
            }
            if (to == V && tid < V % EPV) {
                const int32_t v = V - V % EPV + tid;
                const bool mine_to_add = allowed(mask, v) && !(LIST && ((listed[(v - from) >> 5] >> (v & 31)) & 1u));
                const float x[1] = {mine_to_add ? of_bits(logits[v]) : -INFINITY};
                add_piece<ENT>(x, A.c, mine);
            }
            if (!LIST) break;
        }
        mine = join_wave(mine, A.c);
        if (lane == 0) part[wave] = mine;
        if (LIST) for (int u = wave; u < (A.K + 63) / 64; u += WAVES) sum_entries(A, u, lane, E);
        __syncthreads();
        if (wave == 0) finish_row<KIND, ENT>(A, join_wave(lane < WAVES ? part[lane] : Part{-FLT_MAX, 0.0f, 0.0f, 0.0f}, A.c), row, h, wg, lane, E, shared_ends);
        __syncthreads();
        if (KIND != LOGPROB && A.grad) {
            const Ends ends = shared_ends;
            const Slope slope(ends, A.c);
            const bool all = wild<ENT, ElemT>(ends, A.c);
            if (all) wild_row<ENT, EPV>(TH, logits, mask, grad, V, ends, A.c);
            uint32_t words[U];
            ask_words(tid, words);
            for (int32_t j = tid; j < n_pieces && !all; j += U * TH) {
                uint32_t bits[U];
                u32x4 raw[U];
#pragma unroll
                for (int u = 0; u < U; u++) bits[u] = j + u * TH < n_pieces ? (words[u] >> ((j + u * TH) * EPV & 31)) & FULL : 0u;
                load_pieces<U, EPV>(TH, logits + (int64_t)j * EPV, bits, A.once, raw);
                ask_words(j + U * TH, words);
#pragma unroll
                for (int u = 0; u < U; u++) {
                    u32x4 d{0, 0, 0, 0};
                    if (__any(bits[u] != 0)) {
                        if (__any(bits[u] != FULL)) forbid<EPV, ElemT>(raw[u], bits[u]);
                        d = grad_of<ENT, EPV, ElemT>(raw[u], slope, A.c);
                    }
                    if (j + u * TH < n_pieces) store_raw<ElemT>(grad + (int64_t)(j + u * TH) * EPV, d, A.once);
                }
            }
            if (tid < V % EPV) {
                const int32_t v = V - V % EPV + tid;
                const float x[1] = {allowed(mask, v) ? of_bits(logits[v]) : -INFINITY};
                float d[1];
                grad_of_wild<ENT>(x, ends, A.c, d);
                store_element(grad + v, d[0]);
            }
            if (!LIST) {                                   // by the thread that has just written the token's piece
                if (h.x != -INFINITY && tid == writer_of<EPV>(TH, h.t, V)) store_element(grad + h.t, ends.at_token);
            } else {
                __syncthreads();
                store_entries(TH, A, E, grad);
            }
        }
        if (LIST) {
            __syncthreads();
            if (V <= CHUNK) for (int k = tid; k < A.K; k += TH) { if (E.id[k] >= 0) listed[E.id[k] >> 5] = 0; }
            else for (int i = tid; i < CHUNK / 32; i += TH) listed[i] = 0;
            if (tid == 0) E.end->flags = 0;
            __syncthreads();
        }
    }
}

// A row a workgroup, held in registers between its sums and its gradient: NP pieces of 16 bytes a thread.  Workgroups stay.  As soon as the gradient of a piece is on
// the way its registers take the next row's piece, which is added to that row's sums LAG pieces later: memory is asked for, written and waited for all along the
// arithmetic of both.  Bound by memory: 4,096 x 128,256 bf16 under masks 402 to 417 us (2.1 GB, 5.1 TB/s; vector units busy for 60 %), 64 listed tokens and the rest 427 to 450; 8,192 x 32,000
// fp32 375 to 390 (5.4 TB/s).  loss_rows_kernel, which reads a row again for its
// gradient, in its place: distillation 438 -> 539, policy without masks 415 -> 468, under them 411 -> 416, 8,192 x 32,000 fp32 alike.  20 pieces leave too few registers for a row's state under a mask or with a
// list: 104 to 196 bytes of it a thread lie in memory (16 pieces with a list: 36 to 60).  2,000 x 152,064 bf16: policy 252, under masks 262, distillation 299; 1,024 x 80,000 fp32: policy 140, distillation 176.  A row's mask lies in LDS, without the tokens that a teacher listed: their sums and their gradient are taken from the list.
// PASS: 1: rows begin at multiples of 16 bytes, 2: and the gradient passes the cache by (Args::once; a branch for it at each store would have the compiler wait for stores with the loads).
template <int NP, int KIND, bool MASKED, bool ENT, int PASS, typename ElemT>
__global__ __launch_bounds__(THREADS_MAX, 4) void loss_resident_kernel(const Args A) {
    constexpr int EPV = 16 / sizeof(ElemT), OWN_WORDS = own_words_of(NP, EPV), LAG = 4, EARLY = early_of(NP), SPARE = NP == 16 ? 0 : 3;
    const int TH = blockDim.x, WAVES = TH / 64;
    constexpr uint32_t FULL = (1u << EPV) - 1u;
    constexpr bool LIST = KIND == DISTILL;
    static_assert(!LIST || MASKED, "listed tokens are taken out of the mask");
    __shared__ Part part[THREADS_MAX / 64];
    __shared__ Ends shared_ends;
    extern __shared__ __align__(16) char entries[];         // two rows' entries, a row's mask
    uint32_t *const bits_lds = (uint32_t *)(entries + (LIST ? 2 * entries_bytes(A.K) : 0));
    int tid = threadIdx.x;
    const int wave = __builtin_amdgcn_readfirstlane(tid / 64), lane = tid % 64;
    const int32_t V = A.r.V;
    int32_t n_pieces = V / EPV;
    float g = 1.0f;
    if (A.g) {
        g = *A.g;
        if (A.held && g == 1.0f) return;
    }
    auto logits_of = [&](int64_t row) { return (const ElemT *)A.r.logits + row * A.r.row_stride_elems; };
    auto mask_of = [&](int64_t row) { return A.r.mask ? A.r.mask + row * A.W : nullptr; };
    u32x4 raw[NP];
    uint32_t own_words[OWN_WORDS];
    auto read_words = [&](int64_t row) {                   // a row's mask, without what lies behind V
        const uint32_t *const m = mask_of(row);
#pragma unroll
        for (int i = 0; i < OWN_WORDS; i++) {
            const int32_t at = tid + i * TH, left = V - at * 32;
            own_words[i] = left <= 0 ? 0u : m ? m[at] : ~0u;
            if (left > 0 && left < 32) own_words[i] &= (1u << left) - 1u;
        }
    };
    auto store_words = [&]() {
#pragma unroll
        for (int i = 0; i < OWN_WORDS; i++) bits_lds[tid + i * TH] = own_words[i];
    };
    // The last SPARE pieces may be none of the row's and are left out then; of 16, one or two at most can be so, and leaving none out lets the last waits be for single pieces too
    // (4,096 x 128,256 bf16 with 64 listed tokens 448 -> 434 us; of 8 8,000 x 9,000 bf16 73 -> 80).
    // Every access to memory in the loop over pieces is made by all lanes and whatever the row: the wait for a piece can then leave those that were asked for after it on their way (a
    // piece that may or may not have been asked for would have to be waited for as the last one).  Pieces beyond the row's last are that one once more, written with the same bytes;
    // what is not wanted is asked for from one place.
    uint32_t top;                                          // bytes from a row's start to its last piece
    auto place_of = [&](int i) { return min(((uint32_t)tid + (uint32_t)(i * TH)) * 16u, top); };
    auto bits_at = [&](uint32_t place) -> uint32_t {
        const uint32_t byte = ((const uint8_t *)bits_lds)[place / (EPV == 8 ? 16u : 32u)];
        return EPV == 8 ? byte : (byte >> ((place / 16u & 1u) * 4u)) & FULL;
    };
    // (Rows that begin at multiples of 16 bytes pass the cache by, whatever their number: 32,768 x 2,048 fp32 111 us, else 135; others share lines with their neighbours: 1,030 x 40,037 bf16 50 and 58.)
    auto load = [&](const ElemT *from, uint32_t place) {
        const GLOBAL typename Piece<ElemT>::type *const at = (const GLOBAL typename Piece<ElemT>::type *)((const GLOBAL char *)(uintptr_t)from + place);
        return PASS ? __builtin_nontemporal_load(at) : *at;
    };
    auto fetch = [&](const ElemT *from, int i, bool wanted) {            // piece i of the thread; none is read of which the mask allows nothing
        uint32_t place = place_of(i);
        if (MASKED) place = bits_at(place) ? place : 0u;
        raw[i] = load(from, wanted ? place : 0u);
    };
    // The last EARLY pieces of the row after the next are asked for before the next row's sums come to an end: while a row's end is worked out, memory has them to bring,
    // and the sums do not wait for what was asked for last.  (Nobody knows yet which of them the mask allows, or whether the row counts.)
    u32x4 early[EARLY ? EARLY : 1];
    const bool last = tid < V % EPV;                       // the thread has one of the elements behind the whole pieces
    const int32_t v_last = V - V % EPV + tid;
    ElemT raw_last = 0;                                    // (not looked at before its turn)
    bool last_allowed = false;
    Part mine;
    uint32_t live, next_live = 0;                          // pieces with an allowed token
    auto add = [&](int i) {                                // what is not allowed becomes -inf
        uint32_t bits = FULL;
        if (MASKED) {
            bits = bits_at(place_of(i));
            next_live |= (bits ? 1u : 0u) << i;
            if (__any(bits != FULL)) forbid<EPV, ElemT>(raw[i], bits);
        }
        if (!MASKED || __any(bits != 0)) {
            float x[EPV];
            numbers<EPV, ElemT>(raw[i], x);
            const Part before = mine;
            add_piece<ENT>(x, A.c, mine);
            if ((i + 1) * TH > n_pieces && tid + i * TH >= n_pieces) mine = before;      // the last piece once more
        }
        asm volatile("" : "+v"(raw[i]));                   // (the numbers are made from their 16 bits again: kept, they would be twice the registers)
    };
    auto fetch_last = [&](const ElemT *from) {
        raw_last = from[last ? v_last : 0];
        last_allowed = !MASKED || (last && ((bits_lds[v_last >> 5] >> (v_last & 31)) & 1u));
    };
    auto add_last = [&]() {
        if (!last) return;
        const float x[1] = {last_allowed ? of_bits(raw_last) : -INFINITY};
        add_piece<ENT>(x, A.c, mine);
    };
    // A row's entries: ids and values are asked for two rows ahead, logits and masks one, up to TH of them; further ones when their row is listed.
    Entry ahead{}, after{};
    auto ask_entry = [&](int64_t row, Entry &e) { if (LIST && tid < A.K && row < A.r.rows) ask_id(A, row, tid, e); };
    auto ask_entry_logit = [&](int64_t row, Entry &e) { if (LIST && tid < A.K && row < A.r.rows) ask_logit(A, logits_of(row), mask_of(row), e); };
    auto list_row = [&](int64_t row, const Entries &E) {   // with the tokens' bits in LDS
        for (int k = tid; k < A.K; k += TH) {
            Entry e = ahead;
            if (k >= TH) {
                ask_id(A, row, k, e);
                ask_logit(A, logits_of(row), mask_of(row), e);
            }
            if (list_entry(A, e, k, E) && !((atomicAnd(&bits_lds[e.id >> 5], ~(1u << (e.id & 31))) >> (e.id & 31)) & 1u)) atomicOr(&E.end->flags, 4u);
        }
    };
    const int size = LIST ? entries_bytes(A.K) : 0;
    int64_t row = blockIdx.x;
    int turn = 0;
    Head head{-1, -INFINITY, 1.0f, 0.0f, 0.0f, 0.0f, 0, 0, 0, PADDING}, next_head = head;
    bool counts;
    // The first row
    ask_head<KIND>(A, row, head);
    if (!LIST) {
        head.t = token_at(A, row);
        ask_token(A, logits_of(row), mask_of(row), head);
        see_token<ElemT>(A, head);
        counts = head.t >= 0;
    }
    if (MASKED) {
        read_words(row);
        store_words();
        if (LIST && tid < 2) Entries(entries + tid * size, A.K).end->flags = 0;
        __syncthreads();
        if (LIST) {
            ask_entry(row, ahead);
            ask_entry_logit(row, ahead);
            list_row(row, Entries(entries, A.K));
            ask_entry(row + gridDim.x, ahead);
            ask_entry_logit(row + gridDim.x, ahead);
            ask_entry(row + 2 * (int64_t)gridDim.x, after);
            __syncthreads();
            counts = Entries(entries, A.K).end->flags != 0;
        }
    }
    // (The last wavefronts' work, beside the pieces: the first one's comes at the row's end.)
    auto sum_listed = [&](const Entries &E) { for (int u = WAVES - 1 - wave; u < (A.K + 63) / 64; u += WAVES) sum_entries(A, u, lane, E); };
    if (LIST && counts) sum_listed(Entries(entries, A.K));
    mine = Part{-FLT_MAX, 0.0f, 0.0f, 0.0f};
    top = (uint32_t)(n_pieces - 1) * 16u;
    if (counts) {
#pragma unroll
        for (int i = 0; i < NP; i++) fetch(logits_of(row), i, true);
#pragma unroll
        for (int i = 0; i < NP; i++) if (i < NP - SPARE || i * TH < n_pieces) add(i);
        fetch_last(logits_of(row));
        add_last();
    }
    if (!LIST && row + gridDim.x < A.r.rows) next_head.t = token_at(A, row + gridDim.x);
    if (MASKED && row + gridDim.x < A.r.rows) read_words(row + gridDim.x);
    if (row + gridDim.x < A.r.rows)
#pragma unroll
        for (int i = NP - EARLY; i < NP; i++) early[i - (NP - EARLY)] = load(logits_of(row + gridDim.x), place_of(i));
    for (;;) {
        n_pieces = __builtin_amdgcn_readfirstlane(n_pieces);
        asm volatile("" : "+v"(tid), "+s"(n_pieces));      // (whether a thread has its i-th piece is found anew for each row: kept, that would be registers of every i)
        const Entries E(entries + turn * size, A.K), next_E(entries + (turn ^ 1) * size, A.K);
        const int64_t next = row + gridDim.x;
        const bool more = next < A.r.rows;
        ElemT *const grad = (ElemT *)A.grad + row * A.grad_stride;
        live = next_live;
        next_live = 0;
        mine = join_wave(mine, A.c);
        if (lane == 0) part[wave] = mine;
        __syncthreads();
        if (MASKED && more) store_words();
        if (LIST) {
            if (tid == 0) next_E.end->flags = 0;
            __syncthreads();
            if (more) list_row(next, next_E);
        }
        // (A teacher's entries are listed by the first wavefronts at the same time: with what comes in the loop's middle 4,096 x 128,256 bf16 with 64 listed 479 -> 451 us.)
        if (wave == (LIST ? WAVES - 1 : 0)) {
            if (counts) finish_row<KIND, ENT>(A, join_wave(lane < WAVES ? part[lane] : Part{-FLT_MAX, 0.0f, 0.0f, 0.0f}, A.c), row, head, head.weight * g, lane, E, shared_ends);
            else if (lane == 0) no_row<KIND, ENT>(A, row);
        }
        __syncthreads();
        const Ends ends = shared_ends;
        const bool next_counts = more && (LIST ? next_E.end->flags != 0 : next_head.t >= 0);
        const Slope slope(ends, A.c);
        // Pieces of which nothing is allowed get the zeros that a forbidden token has in others: the row's last piece is written by wavefronts that have such pieces alone and by one that may have more.
        const uint32_t nothing = MASKED && counts ? slope.template zeros<ENT, ElemT>() : 0u;
        if (LIST) {
            if (next_counts) sum_listed(next_E);
            ahead = after;
            ask_entry_logit(next + gridDim.x, ahead);
            ask_entry(next + 2 * (int64_t)gridDim.x, after);
        }
        int64_t next_t = -1;
        const bool third = next + gridDim.x < A.r.rows;    // there is a row after the next
        const ElemT *const next_logits = logits_of(next_counts ? next : row), *const third_logits = logits_of(third ? next + gridDim.x : row);
        mine = Part{-FLT_MAX, 0.0f, 0.0f, 0.0f};
        const float x_of_row[1] = {last && last_allowed ? of_bits(raw_last) : -INFINITY};
        fetch_last(next_logits);
#pragma unroll
        for (int i = 0; i < NP + LAG; i++) {
            // What is alike in the workgroup comes in the loop's middle, while there is much on its way: at a row's end everything would wait for it.  (Never read beyond the rows.)
            if (i == NP / 2) {
                ask_head<KIND>(A, more ? next : row, next_head);
                if (!LIST) {
                    ask_token(A, logits_of(more ? next : row), mask_of(more ? next : row), next_head);
                    next_t = token_at(A, third ? next + gridDim.x : row);
                }
            }
            if (i == NP - 2) {                             // (and is there before the loop ends)
                if (!LIST) asm volatile("" : "+s"(next_head.raw), "+s"(next_head.word), "+s"(next_t));
                if (KIND == POLICY) asm volatile("" : "+s"(next_head.old_logprob), "+s"(next_head.advantage), "+s"(next_head.ref));
                asm volatile("" : "+s"(next_head.weight));
            }
            if (MASKED && i == NP - EARLY - 2) read_words(third ? next + gridDim.x : row);     // (here, so that they are there when the loop is done)
            if (i < NP && (i < NP - SPARE || i * TH < n_pieces)) {
                u32x4 d{nothing, nothing, nothing, nothing};
                if (counts && (!MASKED || __any((live >> i) & 1u))) d = grad_of<ENT, EPV, ElemT>(raw[i], slope, A.c);
                store_raw<ElemT>((GLOBAL char *)(uintptr_t)grad + place_of(i), d, PASS == 2);
                if (i < NP - EARLY) fetch(next_logits, i, next_counts);
                else {
                    // (Moves that the compiler does not see through: it would have the load bring its piece elsewhere, wait for it at once and move it here.)
#pragma unroll
                    for (int k = 0; k < 4; k++) {
                        uint32_t x;
                        asm volatile("v_mov_b32 %0, %1" : "=v"(x) : "v"(early[i - (NP - EARLY)][k]));
                        raw[i][k] = x;
                    }
                    early[i - (NP - EARLY)] = load(third_logits, third ? place_of(i) : 0u);
                }
            }
            if (i >= LAG && next_counts && (i - LAG < NP - SPARE || (i - LAG) * TH < n_pieces)) add(i - LAG);
        }
        if (counts && wild<ENT, ElemT>(ends, A.c)) {
            __syncthreads();                               // the last piece may have been written by several
            wild_row<ENT, EPV>(TH, logits_of(row), mask_of(row), grad, V, ends, A.c);
        }
        if (last) {
            float d[1] = {0.0f};
            if (counts) grad_of_wild<ENT>(x_of_row, ends, A.c, d);
            store_element(grad + v_last, d[0]);
        }
        if (next_counts) add_last();
        if (!LIST) {                                       // by the thread that has just written the token's piece
            const int passes = max(NP - SPARE, (n_pieces + TH - 1) / TH);
            const bool wrote = tid == writer_of<EPV>(TH, head.t, V) || (head.t / EPV == n_pieces - 1 && tid + (passes - 1) * TH >= n_pieces);      // (the last piece: each that did)
            if (counts && head.x != -INFINITY && wrote) store_element(grad + head.t, ends.at_token);
        } else {
            __syncthreads();
            if (counts) store_entries(TH, A, E, grad);
        }
        if (!more) return;
        row = next;
        turn ^= 1;
        counts = next_counts;
        head = next_head;
        if (!LIST) see_token<ElemT>(A, head);
        next_head.t = next_t;
    }
}

// loss = sum of weight x losses, in 64 bits and one order.
__device__ __forceinline__ void sum_losses(const float *losses, const float *weight, int64_t n, float *loss, double *of_wave) {
    constexpr int U = 4;                                   // asked for together
    double sum = 0.0;
    for (int64_t from = threadIdx.x; from < n; from += (int64_t)U * blockDim.x) {
        float l[U], w[U];
#pragma unroll
        for (int u = 0; u < U; u++) {
            const int64_t i = from + (int64_t)u * blockDim.x;
            l[u] = losses[i < n ? i : 0];
            w[u] = weight ? weight[i < n ? i : 0] : 1.0f;
        }
#pragma unroll
        for (int u = 0; u < U; u++) if (from + (int64_t)u * blockDim.x < n) sum += (double)w[u] * l[u];
    }
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
__device__ __forceinline__ int64_t offset_at(const zf_preference_args &p, int64_t s) { return offset_at(p.offsets, p.offset_bytes, s); }

// A sequence a wavefront: its rows' log ratios in 64 bits, in one order.  A workgroup has 8 pairs at a time; a call of a single workgroup sums the losses too.  Bound by the latency of offsets,
// rows, logarithms and the sum in turn: one pair of 12 rows each 4.4 us, 8 of 256 rows 8 to 12.
static const int PAIRS = 8;
__global__ __launch_bounds__(PAIRS * 128) void pairs_kernel(const zf_preference_args p) {
    __shared__ double sums[2 * PAIRS], counts[2 * PAIRS], of_wave[2 * PAIRS];
    const int wave = threadIdx.x / 64, lane = threadIdx.x % 64;
    const float4 *const found = (const float4 *)p.stats;
    for (int64_t first = (int64_t)blockIdx.x * PAIRS; first < p.pairs; first += (int64_t)gridDim.x * PAIRS) {
        const int64_t pair = first + wave / 2;
        bool fits = false;
        if (pair < p.pairs) {
            const int64_t o0 = offset_at(p, 2 * pair), o1 = offset_at(p, 2 * pair + 1), o2 = offset_at(p, 2 * pair + 2);
            fits = 0 <= o0 && o0 <= o1 && o1 <= o2 && o2 <= p.r.rows;
            const int64_t begin = wave % 2 ? o1 : o0, end = fits ? (wave % 2 ? o2 : o1) : begin;
            double sum = 0.0, n = 0.0;
            bool shared = false;                           // the offsets say that a row is in this sequence, and the row was found in another or in none: they descend elsewhere
            constexpr int U = 4;                           // asked for together
            for (int64_t from = begin + lane; from < end; from += U * 64) {
                float lp[U], ref[U];
                int32_t of[U];
#pragma unroll
                for (int u = 0; u < U; u++) {
                    const int64_t row = from + u * 64 < end ? from + u * 64 : from;
                    const float4 f = found[row];
                    lp[u] = f.z;
                    of[u] = __float_as_int(f.w);
                    ref[u] = p.ref_logprobs ? p.ref_logprobs[row] : 0.0f;
                }
#pragma unroll
                for (int u = 0; u < U; u++) {
                    if (from + u * 64 >= end || of[u] == PADDING) continue;
                    shared |= of[u] != 2 * pair + wave % 2;
                    sum += (double)lp[u] - ref[u];
                    n += 1.0;
                }
            }
            sum = wave_sum(sum);
            n = wave_sum(n);
            if (__any(shared)) n = -1.0;
            if (lane == 0) { sums[wave] = sum; counts[wave] = n; }
        }
        __syncthreads();
        if (pair < p.pairs && wave % 2 == 0 && lane == 0) {
            fits = fits && counts[wave] >= 0.0 && counts[wave + 1] >= 0.0;
            double chosen = sums[wave], rejected = sums[wave + 1], n0 = 1.0, n1 = 1.0;
            if (p.average) { n0 = fmax(counts[wave], 1.0); n1 = fmax(counts[wave + 1], 1.0); }
            chosen *= p.beta / n0;
            rejected *= p.beta / n1;
            const double h = chosen - rejected, s = p.label_smoothing;
            // -ln sigma(h) = max(-h, 0) + ln(1 + e^-|h|)
            const double tail = log1p(exp(-fabs(h)));
            double loss = 0.0, slope = 0.0;                // (a share of zero of an infinite term is none)
            if (s != 1.0) { loss = (1.0 - s) * (fmax(-h, 0.0) + tail); slope = -(1.0 - s) / (1.0 + exp(h)); }
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
    if (gridDim.x == 1) sum_losses(p.r.losses, p.r.weight, p.pairs, p.r.loss, of_wave);
}

// The gradient of preferences: a row's slope is its sequence's.  A workgroup has a segment of a row, U pieces of 16 bytes a thread.  Bound by memory: 4,096 x 128,256 bf16, a quarter of
// the rows padding, 319 to 335 us (1.84 GB, 5.6 TB/s).
template <int TH, int U, typename ElemT>
__global__ __launch_bounds__(TH) void preference_grad_kernel(const zf_preference_args p, const float *g, float c, int32_t W, ElemT *grad_, int64_t grad_stride, int32_t segments, int32_t once) {
    constexpr int EPV = 16 / sizeof(ElemT);
    constexpr uint32_t FULL = (1u << EPV) - 1u;
    const int tid = threadIdx.x;
    const int32_t V = p.r.V, n_pieces = V / EPV, segment = blockIdx.x % (uint32_t)segments, j = segment * (U * TH) + tid;
    const int64_t row = blockIdx.x / (uint32_t)segments;
    const ElemT *const logits = (const ElemT *)p.r.logits + row * p.r.row_stride_elems;
    ElemT *const grad = grad_ + row * grad_stride;
    const uint32_t *const mask = p.r.mask ? p.r.mask + row * W : nullptr;
    typedef float f32x4 __attribute__((ext_vector_type(4)));
    const f32x4 found = alike((const f32x4 *)p.stats + row);
    const int32_t sequence = __float_as_int(found.w);
    const bool counts = sequence >= 0 && found.z != -INFINITY;
    uint32_t bits[U];
    u32x4 raw[U];
#pragma unroll
    for (int u = 0; u < U; u++) bits[u] = counts && j + u * TH < n_pieces ? bits_of<EPV>(mask, (int64_t)(j + u * TH) * EPV) : 0u;
    load_pieces<U, EPV>(TH, logits + (int64_t)j * EPV, bits, once, raw);
    const int64_t t = p.token_bytes == 8 ? alike((const int64_t *)p.tokens + row) : alike((const int32_t *)p.tokens + row);
    const float f = counts ? (float)((double)alike(p.slopes + sequence) * alike(g) / p.r.temperature) : 0.0f, base = -f * found.y;
    const Ends ends{found.x, base, 0.0f, 0.0f};
    const Slope slope(ends, c);
    const bool all = wild<false, ElemT>(ends, c);
#pragma unroll
    for (int u = 0; u < U; u++) {
        u32x4 d{0, 0, 0, 0};
        if (__any(bits[u] != 0)) {
            if (__any(bits[u] != FULL)) forbid<EPV, ElemT>(raw[u], bits[u]);
            if (!all) d = grad_of<false, EPV, ElemT>(raw[u], slope, c);
            else d = wild_grad_of<false, EPV, ElemT>(raw[u], ends, c);
        }
        if (j + u * TH < n_pieces) store_raw<ElemT>(grad + (int64_t)(j + u * TH) * EPV, d, once);
    }
    if (counts && t < V - V % EPV && t / EPV % TH == tid && t / EPV >= segment * (U * TH) && t / EPV < (segment + 1) * (U * TH)) {   // the token's own element, by the thread that has just written its piece
        const float x[1] = {of_bits(logits[t])};
        float d[1];
        grad_of_wild<false>(x, ends, c, d);
        store_element(grad + t, d[0] + f);
    }
    if (segment == 0 && tid < V % EPV) {
        const int32_t v = V - V % EPV + tid;
        float d[1] = {0.0f};
        if (counts) {
            const float x[1] = {allowed(mask, v) ? of_bits(logits[v]) : -INFINITY};
            grad_of_wild<false>(x, ends, c, d);
            if (t == v) d[0] += f;
        }
        store_element(grad + v, d[0]);
    }
}

// Rows that the last-level cache (256 MB) cannot hold until somebody reads them again pass it by; not those at odd elements, whose lines are written in two parts.
bool whole(const zf_loss_rows &r, const void *p, int64_t stride) { return !p || ((uintptr_t)p % 16 == 0 && stride * (r.dtype == 0 ? 4 : 2) % 16 == 0); }
bool passes(const zf_loss_rows &r, const LossGrad &g) {
    return r.rows * r.V * (r.dtype == 0 ? 4 : 2) > (256ll << 20) && whole(r, r.logits, r.row_stride_elems) && whole(r, g.grad, g.stride);
}
static const int COMPUTE_UNITS = 256, GRAD_PIECES = 4;
int grid_of(int64_t n) { return (int)std::min<int64_t>(n, 1 << 16); }
// `threads` take a row, NP pieces each at most; as many workgroups as the compute units' registers hold (128 of a thread).  Without a gradient a row is read from memory by as many
// threads, in the same order, to the same bits.
template <int NP, int KIND, bool ENT, typename ElemT>
void rows_by(const Args &A, int threads, hipStream_t s) {
    const int lds = KIND == DISTILL ? entries_bytes(A.K) : 0;
    if constexpr (KIND != LOGPROB && NP > 0) {
        if (A.grad && A.r.V >= 16 / (int)sizeof(ElemT)) {
            // Where a workgroup has a compute unit to itself all take the same number of rows, on fewer compute units: the others' share of the memory is worth more than their time
            // (600 x 128,256 bf16 77.5 -> 73.3 us, 300 under masks 56.8 -> 54.1); of several on one some are done early either way (1,030 x 40,037 61 -> 63).
            const int64_t most = THREADS_MAX / threads * COMPUTE_UNITS, turns = most == COMPUTE_UNITS ? (A.r.rows + most - 1) / most : 1;
            const dim3 grid((int)std::min(most, (A.r.rows + turns - 1) / turns));
            const int pass = A.once ? 2 : whole(A.r, A.r.logits, A.r.row_stride_elems);
            const int words = own_words_of(NP, 16 / (int)sizeof(ElemT)) * threads * 4;
            auto launch = [&](auto *kernel, int bytes) { hipLaunchKernelGGL(kernel, grid, dim3(threads), bytes, s, A); };
            auto choose = [&](auto *k0, auto *k1, auto *k2, int bytes) { launch(pass == 0 ? k0 : pass == 1 ? k1 : k2, bytes); };
#define KERNEL(MASKED, PASS) loss_resident_kernel<NP, KIND, MASKED, ENT, PASS, ElemT>
            if (KIND == DISTILL || A.r.mask) choose(KERNEL(true, 0), KERNEL(true, 1), KERNEL(true, 2), 2 * lds + words);
            else if constexpr (KIND != DISTILL) choose(KERNEL(false, 0), KERNEL(false, 1), KERNEL(false, 2), 0);
#undef KERNEL
            return;
        }
    }
    // Rows that are read twice should still be in the last-level cache the second time: without masks one a compute unit (608 KB each, 256 MB of cache).
    const int64_t most = A.grad && !A.r.mask ? COMPUTE_UNITS : 1 << 16;
    hipLaunchKernelGGL((loss_rows_kernel<KIND, ENT, ElemT>), dim3((int)std::min(A.r.rows, most)), dim3(threads), lds, s, A);
}
template <int KIND, bool ENT, typename ElemT>
void rows_of(const Args &A, hipStream_t s) {
    const int32_t n = (A.r.V + (int)(16 / sizeof(ElemT)) - 1) / (int)(16 / sizeof(ElemT));    // pieces of a row
    // Preferences' log probabilities of many long rows: 256 threads a row, several rows a compute unit, whose starts and ends lie beside others' middles.  The kernel with 1,024 threads (or as many as below)
    // -> with 256: 4,096 x 100,001 bf16 under masks 152 -> 127 us, 20,000 x 17,000 fp32 203 -> 192, 4,096 x 128,256 bf16 with its gradient 139 -> 134; but without it, so that the cache has rows of the call
    // before, 140 -> 152, and 2,048 x 152,064 fp32 172 -> 186, 2,048 x 32,000 45 -> 48.  Fewer or shorter rows: 1,024 x 152,064 fp32 105 -> 111 a call, 8,000 x 4,000 bf16 29.5 -> 34.
    if (KIND == LOGPROB && A.r.rows >= 2048 && n > 16 * 64) return rows_by<0, KIND, ENT, ElemT>(A, 256, s);
    // A thread has all its pieces but the last three at least, or does some again: 16 of them where that fits, else 8.  A workgroup of its own on a compute unit takes a row in the shorter
    // time with twice the threads.  With 8 and with 16 pieces, policy steps: where 16 would have 3 or more again (n <= 13 by_16), 8,000 x 9,000 bf16 73 and 85 us, under masks 82 and 97, 6,000 x 12,000 73 and
    // 79, 32,768 x 2,000 fp32 115 and 127; near the border alike or a little better with 16 (5,000 x 13,300 bf16 73 and 69, 20,000 x 3,400 fp32 129 and 132); beyond, 8,192 x 20,000 fp32 273 and 266,
    // x 32,000 392 and 375, 2,400 x 32,000 bf16 79 and 70.
    const int by_16 = (n + 16 * 64 - 1) / (16 * 64) * 64, by_8 = (n + 8 * 64 - 1) / (8 * 64) * 64;
    if (by_8 <= THREADS_MAX && (A.r.rows <= COMPUTE_UNITS || n <= 13 * by_16)) return rows_by<8, KIND, ENT, ElemT>(A, by_8, s);
    if (n <= 16 * THREADS_MAX) return rows_by<16, KIND, ENT, ElemT>(A, by_16, s);
    if (n <= 20 * THREADS_MAX) return rows_by<20, KIND, ENT, ElemT>(A, THREADS_MAX, s);
    rows_by<0, KIND, ENT, ElemT>(A, THREADS_MAX, s);
}
template <int KIND, bool ENT>
void rows_of(const Args &A, hipStream_t s) {
    if (A.r.dtype == 0) rows_of<KIND, ENT, uint32_t>(A, s);
    else rows_of<KIND, ENT, uint16_t>(A, s);
}
Args common(const zf_loss_rows &r, const LossGrad &g) {
    Args A{};
    A.r = r;
    A.W = (r.V + 31) / 32;
    A.c = (float)(1.4426950408889634 / r.temperature);      // (off by u: an element's exponent y by u |y|, as by its difference and its product each)
    A.grad = g.grad; A.grad_stride = g.stride; A.g = g.g; A.held = g.held; A.results = !g.g;
    A.once = passes(r, g);
    return A;
}
void total(const zf_loss_rows &r, int64_t n, hipStream_t s) { hipLaunchKernelGGL(total_kernel, dim3(1), dim3(1024), 0, s, r.losses, r.weight, n, r.loss); }

}  // namespace

hipError_t launch_distill(const zf_distill_args &a, const LossGrad &g, hipStream_t s) {
    Args A = common(a.r, g);
    A.K = a.n_listed; A.ids = a.ids; A.id_bytes = a.id_bytes; A.values = a.values; A.values_dtype = a.values_dtype; A.rest = a.rest;
    if (a.r.rows) rows_of<DISTILL, false>(A, s);
    if (A.results && a.r.rows != 1) total(a.r, a.r.rows, s);
    return hipGetLastError();
}

hipError_t launch_policy(const zf_policy_args &a, const LossGrad &g, hipStream_t s) {
    Args A = common(a.r, g);
    A.ids = a.tokens; A.id_bytes = a.token_bytes; A.old_logprobs = a.old_logprobs; A.advantages = a.advantages; A.ref = a.kl_weight != 0.0 ? a.ref_logprobs : nullptr;
    A.lowest = 1.0 - a.clip_low; A.highest = 1.0 + a.clip_high; A.kl_weight = a.kl_weight; A.entropy_weight = a.entropy_weight;
    A.logprobs = a.logprobs; A.entropy = a.entropy;
    if (a.r.rows) { if (a.entropy) rows_of<POLICY, true>(A, s); else rows_of<POLICY, false>(A, s); }
    if (A.results && a.r.rows != 1) total(a.r, a.r.rows, s);
    return hipGetLastError();
}

hipError_t launch_preference(const zf_preference_args &a, hipStream_t s) {
    Args A = common(a.r, LossGrad{});
    A.ids = a.tokens; A.id_bytes = a.token_bytes; A.found = (float4 *)a.stats;
    A.offsets = a.offsets; A.offset_bytes = a.offset_bytes; A.sequences = 2 * a.pairs;
    if (a.r.rows) rows_of<LOGPROB, false>(A, s);
    // One workgroup has the pairs of a few thousand rows in a few microseconds, and the sum with them
    const int grid = a.pairs <= 4 * PAIRS && a.r.rows <= 32768 ? 1 : grid_of((a.pairs + PAIRS - 1) / PAIRS);
    hipLaunchKernelGGL(pairs_kernel, dim3(std::max(grid, 1)), dim3(PAIRS * 128), 0, s, a);
    if (grid > 1) total(a.r, a.pairs, s);
    return hipGetLastError();
}

int64_t preference_blocks(const zf_preference_args &a) {
    const int32_t n = a.r.V / (a.r.dtype == 0 ? 4 : 8);
    return a.r.rows * std::max(1, (n + GRAD_PIECES * 256 - 1) / (GRAD_PIECES * 256));
}
hipError_t launch_preference_backward(const zf_preference_args &a, const LossGrad &g, hipStream_t s) {
    if (a.r.rows == 0) return hipSuccess;
    const int64_t blocks = preference_blocks(a);
    const int32_t W = (a.r.V + 31) / 32, segments = (int32_t)(blocks / a.r.rows);
    const float c = (float)(1.4426950408889634 / a.r.temperature);
    if (a.r.dtype == 0) hipLaunchKernelGGL((preference_grad_kernel<256, GRAD_PIECES, uint32_t>), dim3((uint32_t)blocks), dim3(256), 0, s, a, g.g, c, W, (uint32_t *)g.grad, g.stride, segments, passes(a.r, g));
    else hipLaunchKernelGGL((preference_grad_kernel<256, GRAD_PIECES, uint16_t>), dim3((uint32_t)blocks), dim3(256), 0, s, a, g.g, c, W, (uint16_t *)g.grad, g.stride, segments, passes(a.r, g));
    return hipGetLastError();
}

}  // namespace zf
