// Log-probabilities of tokens and the losses on them (cc.h: cc_token_logprob, cc_token_logprob_backward, cc_policy_loss,
// cc_preference_loss).
//
// For a row of V logits l_j, its candidates j, m the largest of their logits, k the row's token:
//   e_j = exp(scale * (l_j - m)),  rest = sum over j != k of e_j,  total = rest + e_k
//   logprob = scale * (l_k - m) - log(total),  p_j = e_j / total,  1 - p_k = rest / total
//   d loss / d logits_j = scale * slope * ([j = k] - p_j),  slope = d loss / d logprob
// rest is summed without the token's own term, so that 1 - p_k keeps its relative precision for a token that is all but
// certain, and the log-probability is then -log1p(rest / e_k).  Logits are subtracted before they are scaled: equal ones
// of any size then have equal terms.
//
// `placed` leaves out the nodes that an earlier position of the order has: a workgroup first writes for every node the
// earliest position that has it, and a logit is a candidate if that position is not before its own.
//
// All of this reads a row once and writes a row at most: the kernels are bound by memory, so rows are read in vectors of
// 16 bytes whatever their alignment, and every lane reduces what it holds before lanes are reduced.
//   rows of up to 1024 logits: kept in the registers of a group of 1 to 64 lanes; loss and gradient in the same pass.
//   longer rows: a workgroup per row.
#include <hip/hip_runtime.h>

#include <cmath>

#include "cc_internal.h"
#include "cc_model.h"

namespace cc {
namespace {

using namespace ccm;

constexpr int kShortRow = 1024;       // cc.h: CC_MAX_N, the longest row with nodes left out
constexpr int kThreads = 256;
constexpr float kInf = __builtin_inff();

struct Args {
    const void* logits;
    void* grad;
    int64_t B, T, sb, st, gsb, gst;
    int V;
    const int32_t* tokens;
    const uint8_t* mask;
    float scale, grad_scale;
    float scale2, scale2_rest;        // scale * log2(e) as a float, and what that leaves out
    float* logprob;
    float2* rows;                     // {m, rest}
    double* gaps;                     // logprob - ref in 64 bits, for the margins
    const float* slope;
    int slope_per_token;              // else one per order
    const float *old_lp, *ref, *advantage;
    int advantage_per_token, mean_of_orders;
    float clip_low, clip_high, kl_coef;
    const int* counts;                // positions that count, per order
    const int2* parts;                // {positions, orders with any} per workgroup of the counting kernel
    int part_count;
    double* partial;                  // [workgroups][3]
    int row_slots, order_slots;       // short rows: a workgroup's rows of an order, and orders
    int chunks;                       // workgroups per order
    int64_t units;                    // workgroups that have rows
};

// A launch's first dimension holds fewer than 2^32 threads: workgroups beyond kAcross go to the second.
constexpr int64_t kAcross = 1 << 20;
__device__ __forceinline__ int64_t workgroup() { return (int64_t)blockIdx.y * kAcross + blockIdx.x; }
dim3 grid_of(int64_t units) {
    return units <= kAcross ? dim3((unsigned)units) : dim3((unsigned)kAcross, (unsigned)((units + kAcross - 1) / kAcross));
}

// Row statistics of a row and its token, in the form that loss and gradient need.
struct Row {
    float m, rest, own, total;        // own: e_k
    bool none;                        // no candidate
    double logprob;
};

// m, rest and the token's logit make the row's log-probability, in 64 bits: sums of log-probabilities are compared with
// sums of others, and 2^-24 of each term's size would be what is left of a difference.
//
// With d = scale * (l_k - m): logprob = -log(1 + x), x = rest / e_k, where the token has most of the sum; else d - log(total), total =
// f 2^e.  Both logarithms are log((1 + s) / (1 - s)) = 2 (s + s^3 / 3 + s^5 / 5 + ...) with s = x / (2 + x) or (f - 1) / (f + 1),
// |s| <= 1/5: what follows s^15 / 15 is below 5e-13.  Neither loses what is small in a sum with 1.
__device__ __forceinline__ Row finish_row(float m, float rest, float token_logit, float scale) {
    Row r;
    r.m = m;
    // The largest logit passes NaN over: nothing is a candidate only if the sum and the token's logit say so too.
    r.none = m == -kInf && rest == 0.0f && token_logit == -kInf;
    if (r.none) {                     // nothing is probable and nothing has a gradient
        r.own = 0.0f;
        r.total = 1.0f;
        r.rest = 0.0f;
        r.logprob = -(double)kInf;
        return r;
    }
    const double d = (double)scale * ((double)token_logit - (double)m);
    r.rest = rest;
    r.own = exp_fast((float)d);
    r.total = rest + r.own;
    const bool most = 2.0f * rest < r.own;
    int e = 0;
    float f = __builtin_frexpf(r.total, &e);          // 1/2 <= f < 1
    if (f < 0.75f) {
        f *= 2.0f;
        e -= 1;
    }
    const double top = most ? (double)rest : (double)f - 1.0, bottom = most ? 2.0 * (double)r.own + (double)rest : (double)f + 1.0;
    // the quotient: a reciprocal of 32 bits, made exact in two steps
    double inverse = (double)__builtin_amdgcn_rcpf((float)bottom);
    inverse = inverse * (2.0 - bottom * inverse);
    const double s = top * inverse * (2.0 - bottom * inverse), q = s * s;
    double series = 1.0 / 15;
    series = series * q + 1.0 / 13;
    series = series * q + 1.0 / 11;
    series = series * q + 1.0 / 9;
    series = series * q + 1.0 / 7;
    series = series * q + 1.0 / 5;
    series = series * q + 1.0 / 3;
    const double log = 2.0 * (s + s * q * series);
    r.logprob = most ? -log : d - ((double)e * kLn2 + log);
    if (!(r.total < kInf)) r.logprob = __builtin_nan("");             // an infinite or undefined logit among the candidates
    return r;
}

// exp(scale * x) for a difference x of two logits.  With the rest of the scale: what its rounding leaves out would make every term
// of every row too small or every term too large, and sums of log-probabilities would show it.  The scale is rounded
// towards zero and the rest is positive: for x = -infinity both products are.
__device__ __forceinline__ float term(const Args& a, float x) { return __builtin_amdgcn_exp2f(fmaf(x, a.scale2, x * a.scale2_rest)); }

// exp(x) - 1 in 64 bits, so that x can be taken from it: x = n ln 2 + r with |r| <= ln 2 / 2 and a little, exp(r) - 1 = r + r^2 (1/2! + r (1/3! + r/4!
// + ... + r^6/9!)).  What the series leaves out is below 3e-10 of the sum; its inner sum is at most an eighth of 1/2 and is taken in 32 bits,
// as constants of 64 bits would take registers from other wavefronts: both results are off by less than 2^-25 of themselves.
// Below -100 it is -1, and where n is held it is more than 32 bits hold.
__device__ __forceinline__ double grown_by(double x) {
    const double y = x < -100.0 ? -100.0 : x;             // NaN stays
    const float n = fminf(rintf((float)y * kLog2e), 250.0f);
    const double r = y - (double)n * kLn2;
    const float f = (float)r;
    float p = 1.0f / 362880;
    p = fmaf(p, f, 1.0f / 40320);
    p = fmaf(p, f, 1.0f / 5040);
    p = fmaf(p, f, 1.0f / 720);
    p = fmaf(p, f, 1.0f / 120);
    p = fmaf(p, f, 1.0f / 24);
    p = fmaf(p, f, 1.0f / 6);
    const double power = ldexp(1.0, (int)n);
    return power * (r + r * r * (0.5 + (double)(p * f))) + (power - 1.0);
}

// What a policy row adds to the loss, the divergence and the clipped share, and its slope.
struct PolicyTerms {
    float loss, kl, clipped, slope;
};
// What it needs of its position beside the logits.
struct PolicyInputs {
    float old_lp, ref, advantage;
    int order_count;
};
__device__ __forceinline__ PolicyInputs policy_inputs(const Args& a, int64_t at, int64_t order) {
    PolicyInputs r;
    r.old_lp = a.old_lp[at];
    r.ref = a.ref ? a.ref[at] : 0.0f;
    r.advantage = a.advantage[a.advantage_per_token ? at : order];
    r.order_count = a.mean_of_orders ? a.counts[order] : 1;
    return r;
}
__device__ __forceinline__ PolicyTerms policy_terms(const Args& a, double lp, const PolicyInputs& in) {
    PolicyTerms r;
    // of a difference x in 64 bits, rounded: off by |x| 2^-24 and the function's last bit, the result's own rounding where a ratio counts
    // (|x| < 1; in 64 bits throughout, 8192 rows of 65536 bf16 took 1 % longer)
    const float ratio = expf((float)(lp - (double)in.old_lp));
    // a ratio that 32 bits do not hold still has no part where there is no advantage, nor a divergence that counts for nothing; that
    // of an undefined log-probability makes the loss undefined
    const float free_gain = in.advantage == 0.0f && lp == lp ? 0.0f : ratio * in.advantage;
    const float held = fminf(fmaxf(ratio, 1.0f - a.clip_low), 1.0f + a.clip_high) * in.advantage;
    const bool clipped = held < free_gain;
    r.clipped = clipped ? 1.0f : 0.0f;
    r.loss = -(clipped ? held : free_gain);
    r.slope = clipped ? 0.0f : -free_gain;
    r.kl = 0.0f;
    if (a.ref) {
        // x = ref - lp is small where the policy is near the one to stay near to, and exp(x) - 1 - x then the square of it, halved: in 64
        // bits, since the difference loses what 32 bits hold of it.  That of an impossible token is infinite.
        const double away = (double)in.ref - lp, full = grown_by(away);
        const float grown = (float)full;
        r.kl = away == (double)kInf ? kInf : (float)(full - away);
        if (a.kl_coef != 0.0f) {
            r.loss += a.kl_coef * r.kl;
            r.slope -= a.kl_coef * grown;
        }
    }
    return r;
}

// Positions and orders that count, from the counting kernel's parts, one a lane.  Every wavefront adds them for itself.
__device__ __forceinline__ int2 all_counts(const Args& a) {
    const int lane = threadIdx.x & 63;
    const int2 p = lane < a.part_count ? a.parts[lane] : make_int2(0, 0);
    return make_int2(group_sum<64>(p.x), group_sum<64>(p.y));
}
__device__ __forceinline__ float weight_of(const Args& a, const int2& all, int order_count) {
    if (!a.mean_of_orders) return all.x > 0 ? 1.0f / (float)all.x : 0.0f;
    return order_count > 0 ? 1.0f / ((float)order_count * (float)all.y) : 0.0f;
}

__device__ __forceinline__ bool counts_here(const Args& a, int64_t at, int token) {
    return (uint32_t)token < (uint32_t)a.V && (!a.mask || a.mask[at] != 0);
}

// A workgroup's three sums, added in one order.
template <int THREADS>
__device__ __forceinline__ void store_partial(double* out, double s0, double s1, double s2, double* lds) {
    s0 = wave_sum_f64(s0);
    s1 = wave_sum_f64(s1);
    s2 = wave_sum_f64(s2);
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) {
        lds[wave * 3] = s0;
        lds[wave * 3 + 1] = s1;
        lds[wave * 3 + 2] = s2;
    }
    __syncthreads();
    if (threadIdx.x < 3) {
        double s = 0.0;
        for (int w = 0; w < THREADS / 64; ++w) s += lds[w * 3 + threadIdx.x];
        out[threadIdx.x] = s;
    }
}

// ------------------------------------------------------------------------------------------------------ short rows

// G lanes per row, K vectors of VEC logits per lane.  A workgroup has order_slots orders, row_slots rows of each; its wavefronts take
// batches of (64 / G) * ITER of these rows:
//   0. a lane per row: token and mask, what the loss needs of the position
//   1. G lanes per row, ITER rows each: all their vectors in flight, largest logit, exponentials (kept in registers), sum
//   2. a lane per row: log-probability and loss, in 64 bits and coalesced; G lanes would do that work G times
//   3. G lanes per row: the gradient
// with a wavefront's own words of LDS between the phases and no barrier.
//
// A lane's vector starts at element j; one that would end beyond the row is moved back to end with it.  It then repeats elements of
// the lane before it: these are left out of the sum, and their gradient is written twice, with the same value.  Every
// lane so has a whole vector to load and store.
//
// What it takes: 64000 rows of 1000 bf16 39 us forward (3.3 TB/s, some 17 vector operations per logit, exponentials and 64-bit ends of
// rows included) and 44 us for the gradient (5.8 TB/s of 256 MB); fewer or more rows a wavefront, and more wavefronts of fewer
// registers, are slower.
//
// The next batch's vectors are loaded before this one is worked, and the tokens of the one after it, which say what to load; the
// first batch's before the order's nodes are looked up.
struct RowInfo {
    int k, t, o, real;                // token (-1: the position does not count), position, order within the workgroup, whether there is a row
    int64_t in, out;                  // the row's place in the logits and in the gradient
};

template <class S, int VEC, int G, int K, int ITER, int KIND, bool PLACED>
__global__ __launch_bounds__(kThreads, KIND == kTokenPolicy ? 3 : 4) void short_rows_kernel(Args a) {
    constexpr int WAVES = kThreads / 64, PER = 64 / G, BATCH = PER * ITER;
    extern __shared__ int first_at[];                 // PLACED: [order_slots][stride] earliest position of each node
    __shared__ RowInfo infos[2][WAVES][BATCH];
    __shared__ float2 sums[WAVES][BATCH];             // {m, rest}
    __shared__ float own[WAVES][BATCH];               // the token's logit
    __shared__ float2 pulls[WAVES][BATCH];            // what multiplies the other terms, and the token's gradient
    __shared__ double sum_lds[3 * WAVES];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wlane = threadIdx.x & 63, group = wlane / G, lane = wlane % G, V = a.V;
    const int stride = (V + 7) & ~7;
    int64_t unit = workgroup();
    if (unit >= a.units) return;
    if (KIND == kTokenBackward) unit = a.units - 1 - unit;
    const int64_t first_order = a.order_slots > 1 ? unit * a.order_slots : unit / a.chunks;
    const int64_t first_row = a.order_slots > 1 ? 0 : (unit - first_order * a.chunks) * a.row_slots;
    const int orders = (int)min((int64_t)a.order_slots, a.B - first_order);
    const int rows = (int)min((int64_t)a.row_slots, a.T - first_row);
    const int slots = orders * rows;

    // 0. in two parts: the token of the lane's row, then what it decides.
    struct Position {
        int64_t order, at;
        int t, o, k;
        bool mine, masked;
    };
    const auto position = [&](int base) {
        Position p;
        const int slot = base + wlane;
        p.mine = wlane < BATCH && slot < slots;
        p.o = p.mine && orders > 1 ? slot / rows : 0;
        p.t = p.mine ? (int)first_row + slot - p.o * rows : 0;
        p.order = first_order + p.o;
        p.at = p.order * a.T + p.t;
        p.k = p.mine ? a.tokens[p.at] : -1;
        p.masked = p.mine && a.mask && a.mask[p.at] == 0;
        return p;
    };
    struct Batch {
        Pack<S, VEC> packs[ITER][K];
        PolicyInputs in;
        float2 saved;
        float slope, ref, token_logit;
        int64_t at;
        bool mine, valid;
    };
    const auto stage = [&](const Position& p, int base, RowInfo* info) {
        Batch r;                                      // of a row that does not count the vectors are zero, of none they are not looked at
        r.in = {};
        r.saved = {};
        r.slope = r.ref = r.token_logit = 0.0f;
        r.mine = p.mine;
        r.at = p.at;
        r.valid = p.mine && !p.masked && (uint32_t)p.k < (uint32_t)V;
        if (wlane < BATCH) {
            RowInfo row;
            row.k = r.valid ? p.k : -1;
            row.t = p.t;
            row.o = p.o;
            row.real = p.mine ? 1 : 0;
            row.in = p.order * a.sb + (int64_t)p.t * a.st;
            row.out = p.order * a.gsb + (int64_t)p.t * a.gst;
            info[wlane] = row;
        }
        wave_order();
#pragma unroll
        for (int it = 0; it < ITER; ++it) {
            if (base + it * PER >= slots) break;
            const RowInfo row = info[it * PER + group];
            if (row.k < 0) {
#pragma unroll
                for (int c = 0; c < K; ++c) r.packs[it][c] = Pack<S, VEC>();
                continue;
            }
#pragma unroll
            for (int c = 0; c < K; ++c) r.packs[it][c] = load_pack<VEC>((const S*)a.logits + row.in + min((c * G + lane) * VEC, V - VEC));
        }
        if (r.valid) {
            r.token_logit = widen(((const S*)a.logits)[p.order * a.sb + (int64_t)p.t * a.st + p.k]);
            if (KIND == kTokenPolicy) r.in = policy_inputs(a, p.at, p.order);
            if (KIND == kTokenForward && a.gaps && a.ref) r.ref = a.ref[p.at];
            if (KIND == kTokenBackward) {
                r.saved = a.rows[p.at];
                r.slope = a.slope[a.slope_per_token ? p.at : p.order];
            }
        }
        return r;
    };
    constexpr int STEP = WAVES * BATCH;
    const int start = wave * BATCH;
    Position coming = position(start);
    Batch next = stage(coming, start, infos[0][wave]);
    coming = position(start + STEP);
    int2 all = {0, 0};
    if (KIND == kTokenPolicy) all = all_counts(a);
    if (PLACED) {
        for (int i = threadIdx.x; i < orders * stride; i += kThreads) first_at[i] = 0x7fffffff;
        __syncthreads();
        const int upto = (int)first_row + rows;       // positions up to the last row's
        for (int i = threadIdx.x; i < orders * upto; i += kThreads) {
            const int o = i / upto, t = i - o * upto;
            const int k = a.tokens[(first_order + o) * a.T + t];
            if ((uint32_t)k < (uint32_t)V) atomicMin(&first_at[o * stride + k], t);
        }
        __syncthreads();
    }
    // The positions of the nodes that a lane's vectors hold: the same for all rows of one order.
    int first[PLACED ? K * VEC : 1];
    const auto look_up = [&](int o) {
#pragma unroll
        for (int c = 0; c < K; ++c)
#pragma unroll
            for (int i = 0; i < VEC; ++i) first[c * VEC + i] = first_at[o * stride + min((c * G + lane) * VEC, V - VEC) + i];
    };
    if (PLACED && orders == 1) look_up(0);
    double sum_loss = 0.0, sum_kl = 0.0, sum_clipped = 0.0;
    int parity = 0;
    for (int base = start; base < slots; base += STEP, parity ^= 1) {
        const Batch now = next;
        const RowInfo* const info = infos[parity][wave];
        if (base + STEP < slots) {
            next = stage(coming, base + STEP, infos[parity ^ 1][wave]);
            coming = position(base + 2 * STEP);
        }
        if (wlane < BATCH) {
            own[wave][wlane] = now.token_logit;
            if (KIND == kTokenBackward) sums[wave][wlane] = now.saved;
        }
        wave_order();
        // 1.
        float e[ITER][K * VEC];
#pragma unroll
        for (int it = 0; it < ITER; ++it) {
            const int at_row = it * PER + group;
            const RowInfo r = info[at_row];
            if (!__any(r.k >= 0)) {                   // none of the groups has a row that counts
#pragma unroll
                for (int i = 0; i < K * VEC; ++i) e[it][i] = 0.0f;
                continue;
            }
            if (PLACED && orders > 1) look_up(r.o);
            const float token_logit = own[wave][at_row];
            float m = token_logit;
            // What is no candidate becomes minus infinity, before it is looked at, and so does the token: its own term is no part of
            // the sum.  Where nodes are left out that is one comparison: the token stands at this position or before.
#pragma unroll
            for (int c = 0; c < K; ++c) {
                const int j0 = min((c * G + lane) * VEC, V - VEC);
                float* const z = e[it] + c * VEC;
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    z[i] = now.packs[it][c].get(i);
                    if (PLACED) z[i] = first[c * VEC + i] > r.t ? z[i] : -kInf;
                }
                if (!PLACED && (uint32_t)(r.k - j0) < (uint32_t)VEC) {
#pragma unroll
                    for (int i = 0; i < VEC; ++i) z[i] = j0 + i == r.k ? -kInf : z[i];
                }
#pragma unroll
                for (int i = 0; i < VEC; ++i) m = fmaxf(m, z[i]);
            }
            m = KIND == kTokenBackward ? sums[wave][at_row].x : group_max<G>(m);
            const float low = m == -kInf ? 0.0f : m;
            float rest = 0.0f;
#pragma unroll
            for (int c = 0; c < K; ++c) {
                const int j = (c * G + lane) * VEC, j0 = min(j, V - VEC);
                float* const z = e[it] + c * VEC;
#pragma unroll
                for (int i = 0; i < VEC; ++i) z[i] = term(a, z[i] - low);
                if (KIND == kTokenBackward) continue;
                float sum = 0.0f;
#pragma unroll
                for (int i = 0; i < VEC; ++i) sum += z[i];
                if (j0 != j && j < V) {               // without what the lane before it has
                    sum = 0.0f;
#pragma unroll
                    for (int i = 0; i < VEC; ++i) sum += j0 + i >= j ? z[i] : 0.0f;
                }
                rest += j < V ? sum : 0.0f;
            }
            if (KIND != kTokenBackward) {
                rest = group_sum<G>(rest);
                if (lane == 0) sums[wave][at_row] = make_float2(m, rest);
            }
        }
        wave_order();
        // 2.
        if (now.mine) {
            Row r = {};
            float slope = now.slope;
            if (now.valid) {
                const float2 s = KIND == kTokenBackward ? now.saved : sums[wave][wlane];
                r = finish_row(s.x, s.y, now.token_logit, a.scale);
                if (KIND == kTokenPolicy) {
                    const PolicyTerms p = policy_terms(a, r.logprob, now.in);
                    const float w = weight_of(a, all, now.in.order_count);
                    slope = w * p.slope;
                    sum_loss += (double)w * p.loss;
                    sum_kl += (double)w * p.kl;
                    sum_clipped += (double)w * p.clipped;
                }
            }
            if (KIND != kTokenBackward) {
                a.logprob[now.at] = (float)r.logprob;
                if (a.rows) a.rows[now.at] = make_float2(r.m, r.rest);
                if (KIND == kTokenForward && a.gaps) a.gaps[now.at] = now.valid ? r.logprob - (double)now.ref : 0.0;
            }
            if (KIND != kTokenForward) {
                const float pull = now.valid && !r.none ? slope * a.scale * a.grad_scale / r.total : 0.0f;
                pulls[wave][wlane] = make_float2(-pull, pull * r.rest);
            }
        }
        if (KIND == kTokenForward || !a.grad) continue;
        wave_order();
        // 3.
#pragma unroll
        for (int it = 0; it < ITER; ++it) {
            if (base + it * PER >= slots) break;
            const RowInfo r = info[it * PER + group];
            const float2 pull = pulls[wave][it * PER + group];
            S* const out = (S*)a.grad + r.out;
#pragma unroll
            for (int c = 0; c < K; ++c) {
                const int j = (c * G + lane) * VEC, j0 = min(j, V - VEC);
                float g[VEC];
#pragma unroll
                for (int i = 0; i < VEC; ++i) g[i] = e[it][c * VEC + i] * pull.x;
                if (PLACED && !(fabsf(pull.x) < kInf)) {
                    // what is no candidate has no gradient, whatever the row's others have: a term of 0, or in an undefined row a place
                    // that an earlier position has
#pragma unroll
                    for (int i = 0; i < VEC; ++i) {
                        const bool out_of_play = pull.x == pull.x ? e[it][c * VEC + i] == 0.0f : first_at[r.o * stride + j0 + i] <= r.t;
                        g[i] = out_of_play ? 0.0f : g[i];
                    }
                }
                if ((uint32_t)(r.k - j0) < (uint32_t)VEC) {
#pragma unroll
                    for (int i = 0; i < VEC; ++i) g[i] = j0 + i == r.k ? pull.y : g[i];
                }
                if ((int)(j < V) & r.real) store_pack(out + j0, Pack<S, VEC>::from(g));
            }
        }
    }
    if (KIND == kTokenPolicy) store_partial<kThreads>(a.partial + unit * 3, sum_loss, sum_kl, sum_clipped, sum_lds);
}

// ------------------------------------------------------------------------------------------------------- long rows

// A workgroup per row.  K > 0: the row, up to THREADS * K vectors, stays in registers as it was loaded, so that it is read once
// for log-probability, loss and gradient; its exponentials are taken twice, since 32 bits of each would not fit.  K = 0: rows
// longer than that are read twice.  As for short rows, a vector that would end beyond the row is moved back.
//
// Bound by memory: 8192 rows of 65536 bf16, loss and gradient, 340 us, 6.3 TB/s of 2.15 GB.
//
// The token's own term and repeated elements are taken out of the sum where they are, by the lane that has them, in a branch
// that other wavefronts skip.
//
// The backward pass goes through the rows from the last one: the last level of cache still holds some of what the forward
// pass read last (6216 rows of 50001 f16: 215 us in the forward pass's order, 204 us from the last row).
template <class S, int VEC>
__device__ __forceinline__ void widen_row(const Pack<S, VEC>& p, float z[VEC]) {
#pragma unroll
    for (int i = 0; i < VEC; ++i) z[i] = p.get(i);
}

// What was widened is not kept: the row stays in registers as it was loaded.
template <class S, int VEC, int N>
__device__ __forceinline__ void forget_all(Pack<S, VEC> (&p)[N]) {
#pragma unroll
    for (int c = 0; c < N; ++c) forget(p[c]);
}

template <class S, int THREADS, int K, int KIND>
__global__ __launch_bounds__(THREADS, K > 8 || (K == 0 && KIND != kTokenBackward) ? 5 - K / 16 : 8) void long_rows_kernel(Args a) {
    constexpr int VEC = 16 / sizeof(S), WAVES = THREADS / 64, STEP = THREADS * VEC, KEPT = K > 0 ? K : 4;
    __shared__ float2 wave_sums[WAVES];               // {m, rest}
    __shared__ float2 shared_pull;
    const int V = a.V, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t at = workgroup();
    if (at >= a.B * a.T) return;
    if (KIND == kTokenBackward) at = a.B * a.T - 1 - at;
    const int64_t order = at / a.T, t = at - order * a.T;
    const int k = a.tokens[at];
    const bool valid = counts_here(a, at, k);
    const S* const row = (const S*)a.logits + order * a.sb + t * a.st;
    S* const out = (S*)a.grad + order * a.gsb + t * a.gst;
    int mine = threadIdx.x * VEC;
    if (!valid) {
        if (KIND != kTokenBackward && threadIdx.x == 0) {
            a.logprob[at] = 0.0f;
            if (a.rows) a.rows[at] = make_float2(0.0f, 0.0f);
            if (a.gaps) a.gaps[at] = 0.0;
        }
        if (KIND == kTokenPolicy && threadIdx.x < 3) a.partial[at * 3 + threadIdx.x] = 0.0;
        if (KIND == kTokenForward || !a.grad) return;
        const float zero[VEC] = {};
        const Pack<S, VEC> p = Pack<S, VEC>::from(zero);
        for (int j = mine; j < V; j += STEP) store_pack(out + min(j, V - VEC), p);
        return;
    }
    Pack<S, VEC> kept[KEPT];
    if (K > 0) {
#pragma unroll
        for (int c = 0; c < K; ++c)
            if (c * STEP < V) kept[c] = load_pack<VEC>(row + min(c * STEP + mine, V - VEC));
    }
    const float token_logit = widen(row[k]);
    int2 all = {0, 0};
    PolicyInputs in = {};
    if (KIND == kTokenPolicy && wave == 0) {
        all = all_counts(a);
        in = policy_inputs(a, at, order);
    }
    float m = -kInf, rest = 0.0f;
    if (KIND == kTokenBackward) {
        const float2 saved = a.rows[at];
        m = saved.x;
        rest = saved.y;
        __syncthreads();                              // the gradient may take the logits' place: the token's has been read by all
    } else {
        // Elements of the vector at j that are not summed: the token, and those that the vector before it has.
        const auto leave_out = [&](int j, float z[VEC]) {
            const int j0 = min(j, V - VEC);
            if ((uint32_t)(k - j0) < (uint32_t)VEC || j0 != j) {
#pragma unroll
                for (int i = 0; i < VEC; ++i) z[i] = j0 + i == k || j0 + i < j ? -kInf : z[i];
            }
        };
        if (K > 0) {
            // The lane's largest logit, the token's among them, then its sum.
#pragma unroll
            for (int c = 0; c < K; ++c)
                if (c * STEP < V) m = fmaxf(m, largest(kept[c]));
            const float low = m == -kInf ? 0.0f : m;
            forget_all(kept);
            asm("" : "+v"(mine));                     // and places in the row are made again
#pragma unroll
            for (int c = 0; c < K; ++c)
                if (c * STEP < V) {
                    float z[VEC];
                    widen_row(kept[c], z);
                    leave_out(c * STEP + mine, z);
#pragma unroll
                    for (int i = 0; i < VEC; ++i) rest += term(a, z[i] - low);
                    __builtin_amdgcn_sched_barrier(0);    // one vector's values at a time: registers are for the row
                }
        } else {
            // KEPT vectors at a time, with a running maximum, the next ones on their way.
            const auto load = [&](int c0, Pack<S, VEC> (&to)[KEPT]) {
#pragma unroll
                for (int c = 0; c < KEPT; ++c)
                    if (c0 + c * STEP < V) to[c] = load_pack<VEC>(row + min(c0 + c * STEP + mine, V - VEC));
            };
            Pack<S, VEC> next[KEPT];
            load(0, next);
            for (int c0 = 0; c0 < V; c0 += KEPT * STEP) {
#pragma unroll
                for (int c = 0; c < KEPT; ++c) kept[c] = next[c];
                load(c0 + KEPT * STEP, next);
                float top = m;
#pragma unroll
                for (int c = 0; c < KEPT; ++c)
                    if (c0 + c * STEP < V) top = fmaxf(top, largest(kept[c]));
                const float low = top == -kInf ? 0.0f : top;
                rest *= term(a, m - low);
#pragma unroll
                for (int c = 0; c < KEPT; ++c)
                    if (c0 + c * STEP < V) {
                        float z[VEC];
                        widen_row(kept[c], z);
                        leave_out(c0 + c * STEP + mine, z);
#pragma unroll
                        for (int i = 0; i < VEC; ++i) rest += term(a, z[i] - low);
                    }
                m = top;
            }
        }
        const float lane_m = m;
        m = group_max<64>(m);
        float low = m == -kInf ? 0.0f : m;
        rest = group_sum<64>(rest * term(a, lane_m - low));
        if (lane == 0) wave_sums[wave] = make_float2(m, rest);
        __syncthreads();
        // every wavefront joins the wavefronts' pairs, one a lane
        const float2 w = lane < WAVES ? wave_sums[lane] : make_float2(-kInf, 0.0f);
        m = group_max<64>(w.x);
        low = m == -kInf ? 0.0f : m;
        rest = group_sum<64>(w.y * term(a, w.x - low));
    }
    if (wave == 0) {
        const Row r = finish_row(m, rest, token_logit, a.scale);
        float slope = 0.0f;
        if (KIND == kTokenPolicy) {
            const PolicyTerms p = policy_terms(a, r.logprob, in);
            const float w = weight_of(a, all, in.order_count);
            slope = w * p.slope;
            if (threadIdx.x == 0) {
                a.partial[at * 3] = (double)w * p.loss;
                a.partial[at * 3 + 1] = (double)w * p.kl;
                a.partial[at * 3 + 2] = (double)w * p.clipped;
            }
        } else if (KIND == kTokenBackward) {
            slope = a.slope[a.slope_per_token ? at : order];
        }
        if (KIND != kTokenBackward && threadIdx.x == 0) {
            a.logprob[at] = (float)r.logprob;
            if (a.rows) a.rows[at] = make_float2(r.m, r.rest);
            if (a.gaps) a.gaps[at] = r.logprob - (a.ref ? (double)a.ref[at] : 0.0);
        }
        if (KIND != kTokenForward && threadIdx.x == 0) {
            const float pull = r.none ? 0.0f : slope * a.scale * a.grad_scale / r.total;
            shared_pull = make_float2(-pull, pull * r.rest);
        }
    }
    if (KIND == kTokenForward || !a.grad) return;
    __syncthreads();
    const float2 pull = shared_pull;
    const float low = m == -kInf ? 0.0f : m;
    const auto gradient = [&](int j, const Pack<S, VEC>& p) {
        const int j0 = min(j, V - VEC);
        float z[VEC];
        widen_row(p, z);
#pragma unroll
        for (int i = 0; i < VEC; ++i) z[i] = term(a, z[i] - low) * pull.x;
        if ((uint32_t)(k - j0) < (uint32_t)VEC) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) z[i] = j0 + i == k ? pull.y : z[i];
        }
        const Pack<S, VEC> g = Pack<S, VEC>::from(z);
        if (K == 0 && j0 != j) {
            // Read again, in place perhaps: what this vector repeats may hold its gradient by now.  Only its own elements are stored.
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                if (j0 + i >= j) out[j0 + i] = g.element(i);
        } else if (j < V) {
            store_pack(out + j0, g);
        }
    };
    if (K > 0) {
        forget_all(kept);
        asm("" : "+v"(mine));
#pragma unroll
        for (int c = 0; c < K; ++c)
            if (c * STEP < V) {
                gradient(c * STEP + mine, kept[c]);
                __builtin_amdgcn_sched_barrier(0);
            }
    } else {
        for (int c0 = 0; c0 < V; c0 += KEPT * STEP) {
#pragma unroll
            for (int c = 0; c < KEPT; ++c)
                if (c0 + c * STEP < V) kept[c] = load_pack<VEC>(row + min(c0 + c * STEP + mine, V - VEC));
#pragma unroll
            for (int c = 0; c < KEPT; ++c)
                if (c0 + c * STEP < V) gradient(c0 + c * STEP + mine, kept[c]);
        }
    }
}

// ---------------------------------------------------------------------------------------------------- small kernels

// counts[b]: positions of order b that count; parts[workgroup]: positions and orders with any.
constexpr int kCountBlocks = 64, kCountThreads = 1024;
__global__ __launch_bounds__(kCountThreads) void count_kernel(const int32_t* __restrict__ tokens, const uint8_t* __restrict__ mask, int64_t B,
                                                              int64_t T, int V, int* __restrict__ counts, int2* __restrict__ parts) {
    constexpr int WAVES = kCountThreads / 64;
    __shared__ int2 lds[WAVES];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    int2 sum = {0, 0};
    for (int64_t b = (int64_t)blockIdx.x * WAVES + wave; b < B; b += (int64_t)gridDim.x * WAVES) {
        int n = 0;
#pragma unroll 4
        for (int64_t t = lane; t < T; t += 64)
            n += (int)((uint32_t)tokens[b * T + t] < (uint32_t)V) & (int)(!mask || mask[b * T + t] != 0);
        n = group_sum<64>(n);
        if (lane == 0) counts[b] = n;
        sum.x += n;
        sum.y += n > 0 ? 1 : 0;
    }
    if (lane == 0) lds[wave] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < WAVES; ++w) {
            sum.x += lds[w].x;
            sum.y += lds[w].y;
        }
        parts[blockIdx.x] = sum;
    }
}

constexpr int kSumThreads = 1024;

// The policy loss's three sums over the workgroups' partial sums, in one order.
__global__ __launch_bounds__(kSumThreads) void policy_sum_kernel(const double* __restrict__ partial, int64_t count, float* __restrict__ stats) {
    __shared__ double lds[3][kSumThreads / 64];
    double s[3] = {0.0, 0.0, 0.0};
#pragma unroll 8
    for (int64_t i = threadIdx.x; i < count; i += kSumThreads)
#pragma unroll
        for (int q = 0; q < 3; ++q) s[q] += partial[i * 3 + q];
#pragma unroll
    for (int q = 0; q < 3; ++q) {
        s[q] = wave_sum_f64(s[q]);
        if ((threadIdx.x & 63) == 0) lds[q][threadIdx.x >> 6] = s[q];
    }
    __syncthreads();
    if (threadIdx.x < 3) {
        double sum = 0.0;
        for (int w = 0; w < kSumThreads / 64; ++w) sum += lds[threadIdx.x][w];
        stats[threadIdx.x] = (float)sum;
    }
}

// A pair: its margin, its share of the loss, and the slope of its two sequences' log-probabilities.
__device__ __forceinline__ double finish_pair(double gap, int64_t p, int64_t pairs, float beta, float smoothing, float* __restrict__ margin,
                                              float* __restrict__ slope) {
    // A sequence that holds an impossible token makes the margin infinite: what is multiplied by zero then still has no part.
    const double m = beta == 0.0f && gap == gap ? 0.0 : (double)beta * gap;
    // softplus(x) = max(x, 0) + log1p(exp(-|x|))
    const double small = exp(-fabs(m)), tail = log1p(small), part = small / (1.0 + small);
    const double away = m >= 0.0 ? part : 1.0 - part, by = m >= 0.0 ? 1.0 - part : part;       // sigmoid(-m), sigmoid(m)
    const float s = (float)((double)beta / (double)pairs * ((double)smoothing * by - (1.0 - (double)smoothing) * away));
    margin[p] = (float)m;
    slope[p] = s;
    slope[p + pairs] = -s;
    const double against = smoothing == 1.0f ? 0.0 * tail : (1.0 - (double)smoothing) * (fmax(-m, 0.0) + tail);
    const double towards = smoothing == 0.0f ? 0.0 * tail : (double)smoothing * (fmax(m, 0.0) + tail);
    return (against + towards) / (double)pairs;
}

// TEAM threads share a pair's positions: one where they are few (a pair's 64-bit functions are then taken for 64 pairs at once), a
// workgroup's wavefronts or all of it where they are many.  Where one workgroup has all pairs it also adds their shares up; else
// pair_sum_kernel does.
template <int THREADS, int TEAM>
__global__ __launch_bounds__(THREADS) void pair_kernel(const double* __restrict__ gaps, int64_t pairs, int64_t T, float beta, float smoothing,
                                                       float* __restrict__ margin, float* __restrict__ slope, double* __restrict__ losses,
                                                       float* __restrict__ loss) {
    constexpr int TEAMS = THREADS / TEAM;
    __shared__ double lds[THREADS / 64];
    const int wave = threadIdx.x >> 6, team = threadIdx.x / TEAM, member = threadIdx.x % TEAM;
    double sum = 0.0;
    for (int64_t p0 = (int64_t)blockIdx.x * TEAMS; p0 < pairs; p0 += (int64_t)gridDim.x * TEAMS) {
        const int64_t p = p0 + team;
        double gap = 0.0;
        if (p < pairs) {
#pragma unroll 4
            for (int64_t t = member; t < T; t += TEAM) gap += gaps[p * T + t] - gaps[(p + pairs) * T + t];
        }
        if (TEAM >= 64) gap = wave_sum_f64(gap);
        if (TEAM > 64) {
            if ((threadIdx.x & 63) == 0) lds[wave] = gap;
            __syncthreads();
            gap = 0.0;
            for (int w = 0; w < TEAM / 64; ++w) gap += lds[team * (TEAM / 64) + w];
            __syncthreads();
        }
        if (member == 0 && p < pairs) {
            const double share = finish_pair(gap, p, pairs, beta, smoothing, margin, slope);
            if (loss) sum += share;
            else losses[p] = share;
        }
    }
    if (!loss) return;
    sum = wave_sum_f64(sum);
    if ((threadIdx.x & 63) == 0) lds[wave] = sum;
    __syncthreads();
    if (threadIdx.x != 0) return;
    sum = 0.0;
    for (int w = 0; w < THREADS / 64; ++w) sum += lds[w];
    *loss = (float)sum;
}

__global__ __launch_bounds__(kSumThreads) void pair_sum_kernel(const double* __restrict__ losses, int64_t pairs, float* __restrict__ loss) {
    __shared__ double lds[kSumThreads / 64];
    double s = 0.0;
    for (int64_t i = threadIdx.x; i < pairs; i += kSumThreads) s += losses[i];
    s = wave_sum_f64(s);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        s = 0.0;
        for (int w = 0; w < kSumThreads / 64; ++w) s += lds[w];
        *loss = (float)s;
    }
}

// --------------------------------------------------------------------------------------------------------- launches

size_t up256(size_t x) { return (x + 255u) & ~(size_t)255u; }

// Workspace: [counts or slopes: 4 B][parts][gaps or partial sums: 24 BT + 24][row statistics: 8 BT][losses: 8 B]
struct Layout {
    size_t counts, parts, sums, rows, losses, total;
};
Layout layout(int64_t B, int64_t T) {
    const size_t b = (size_t)B, bt = (size_t)B * (size_t)T;
    Layout l;
    l.counts = 0;
    l.parts = l.counts + up256(4 * b);
    l.sums = l.parts + up256(sizeof(int2) * kCountBlocks);
    l.rows = l.sums + up256(24 * bt + 24);
    l.losses = l.rows + up256(8 * bt);
    l.total = l.losses + up256(8 * b);
    return l;
}

template <class S, int VEC, int G, int K, int KIND>
int64_t launch_short(Args& a, bool placed, hipStream_t s) {
    // Two batches' vectors and one's exponentials, of 32 bits each, in registers: 16 elements a lane and batch of 32 bits, 32 of 16.
    // The forward pass keeps no exponentials and takes twice the rows.
    constexpr int MOST = (sizeof(S) == 4 ? 16 : 32) / (K * VEC) * (KIND == kTokenForward ? 2 : 1), ITER = MOST < 4 ? MOST : 4, batch = 64 / G * ITER, rows_at_once = batch * (kThreads / 64);
    // A workgroup takes several orders where their positions do not fill its batches; else up to four batches a wavefront of one
    // order's positions (the more, the fewer times the order's nodes are looked up), fewer where that would leave compute units idle.
    const int64_t T = a.T;
    if (T * 2 <= rows_at_once) {
        int64_t orders = rows_at_once / T;
        const int64_t stride = (a.V + 7) & ~7;
        if (placed && orders * stride > 8192) orders = 8192 / stride;
        while (orders > 1 && (a.B + orders - 1) / orders < 512) orders = (orders + 1) / 2;
        a.order_slots = (int)orders;
        a.row_slots = (int)T;
        a.chunks = 1;
    } else {
        int64_t passes = 4;
        while (passes > 1 && a.B * ((T + rows_at_once * passes - 1) / (rows_at_once * passes)) < 1024) passes /= 2;
        a.order_slots = 1;
        a.row_slots = (int)(rows_at_once * passes < T ? rows_at_once * passes : T);
        a.chunks = (int)((T + a.row_slots - 1) / a.row_slots);
    }
    const int64_t blocks = a.order_slots > 1 ? (a.B + a.order_slots - 1) / a.order_slots : a.B * a.chunks;
    a.units = blocks;
    if (placed)
        hipLaunchKernelGGL((short_rows_kernel<S, VEC, G, K, ITER, KIND, true>), grid_of(blocks), dim3(kThreads),
                           sizeof(int) * a.order_slots * ((a.V + 7) & ~7), s, a);
    else
        hipLaunchKernelGGL((short_rows_kernel<S, VEC, G, K, ITER, KIND, false>), grid_of(blocks), dim3(kThreads), 0, s, a);
    return blocks;
}

template <class S, int THREADS, int K, int KIND>
int64_t launch_long(Args& a, hipStream_t s) {
    const int64_t rows = a.B * a.T;
    hipLaunchKernelGGL((long_rows_kernel<S, THREADS, K, KIND>), grid_of(rows), dim3(THREADS), 0, s, a);
    return rows;
}

// One pass over the rows; returns the number of workgroups, each of which leaves a partial sum of the loss.
template <class S, int KIND>
int64_t launch_rows(Args& a, bool placed, hipStream_t s) {
    constexpr int VEC = 16 / sizeof(S);
    const int V = a.V;
    if (V <= kShortRow) {
        if (V < VEC) return launch_short<S, 1, 8, 1, KIND>(a, placed, s);
        if (V <= 8 * VEC) return launch_short<S, VEC, 8, 1, KIND>(a, placed, s);
        if (V <= 16 * VEC) return launch_short<S, VEC, 16, 1, KIND>(a, placed, s);
        if (V <= 32 * VEC) return launch_short<S, VEC, 32, 1, KIND>(a, placed, s);
        if (V <= 64 * VEC) return launch_short<S, VEC, 64, 1, KIND>(a, placed, s);
        if (V <= 128 * VEC) return launch_short<S, VEC, 64, 2, KIND>(a, placed, s);
        if constexpr (VEC == 4) return launch_short<S, VEC, 64, 4, KIND>(a, placed, s);
    }
    // The policy loss needs a row twice: threads and vectors per thread enough to hold it.  One pass takes a few vectors at a time,
    // in workgroups small enough that one's sums overlap others' loads.
    if constexpr (KIND == kTokenPolicy) {
        if (V <= 256 * VEC * 2) return launch_long<S, 256, 2, KIND>(a, s);
        if (V <= 256 * VEC * 4) return launch_long<S, 256, 4, KIND>(a, s);
        if (V <= 256 * VEC * 8) return launch_long<S, 256, 8, KIND>(a, s);
        if (V <= 512 * VEC * 8) return launch_long<S, 512, 8, KIND>(a, s);
        if (V <= 1024 * VEC * 8) return launch_long<S, 1024, 8, KIND>(a, s);
        if (V <= 1024 * VEC * 16) return launch_long<S, 1024, 16, KIND>(a, s);
        return launch_long<S, 1024, 0, KIND>(a, s);
    } else {
        // 256 threads or 1024 a row, in us of the forward kernel: rows short of a turn of 1024 threads' vectors leave most of these
        // without one (4096 x 5000 bf16: 12.7, 26.4; 4096 x 8192: 14.6, 26.2); fewer rows than two workgroups a compute unit want all
        // threads they can get (256 x 16384: 4.8, 4.4; 256 x 65536: 10.9, 8.0; 256 x 300007: 40.7, 31.7; but 512 x 16384: 5.6, 6.1); longer
        // ones want them the sooner the fewer rows there are (1024 x 16384: 8.3, 9.8; 1024 x 32768: 15.1, 15.4; 1024 x 65536: 27.9, 26.5;
        // 2048 x 33000: 28.2, 33.1; 4096 x 50001: 96, 95; 4096 x 65536: 107, 94).
        const int64_t rows = a.B * a.T, most = rows < 512 ? 1024 * VEC : rows < 2048 ? 4096 * VEC : 8192 * VEC - 1;
        if (V <= most) return launch_long<S, 256, 0, KIND>(a, s);
        return launch_long<S, 1024, 0, KIND>(a, s);
    }
}

template <class S>
hipError_t run(TokenKind kind, const TokenCall& c, hipStream_t s) {
    Args a = {};
    a.logits = c.logits;
    a.grad = c.grad;
    a.B = c.B; a.T = c.T; a.V = (int)c.V;
    a.sb = c.stride_b; a.st = c.stride_t;
    a.gsb = c.grad_stride_b; a.gst = c.grad_stride_t;
    a.tokens = c.tokens;
    a.mask = c.mask;
    a.scale = c.scale;
    const double scale2 = (double)c.scale * 1.4426950408889634074;
    a.scale2 = (float)scale2;
    if ((double)a.scale2 >= scale2) a.scale2 = std::nextafterf(a.scale2, 0.0f);
    a.scale2_rest = (float)(scale2 - (double)a.scale2);
    a.grad_scale = c.grad_scale;
    a.logprob = c.logprob;
    a.rows = (float2*)c.rows;
    a.slope = c.slope;
    a.slope_per_token = 1;
    a.old_lp = c.old;
    a.ref = c.ref;
    a.advantage = c.advantage;
    a.advantage_per_token = c.advantage_per_token;
    a.mean_of_orders = c.mean_of_orders;
    a.clip_low = c.clip_low;
    a.clip_high = c.clip_high;
    a.kl_coef = c.kl_coef;
    const bool any = c.B > 0 && c.T > 0;
    if (kind == kTokenForward) {
        if (any) launch_rows<S, kTokenForward>(a, c.placed, s);
        return hipGetLastError();
    }
    if (kind == kTokenBackward) {
        if (any) launch_rows<S, kTokenBackward>(a, c.placed, s);
        return hipGetLastError();
    }
    const Layout l = layout(c.B, c.T);
    char* const w = (char*)c.workspace;
    if (kind == kTokenPolicy) {
        int64_t partials = 0;
        a.partial = (double*)(w + l.sums);
        if (any) {
            const int64_t need = (c.B + kCountThreads / 64 - 1) / (kCountThreads / 64);
            a.part_count = (int)(need < kCountBlocks ? need : kCountBlocks);
            a.counts = (const int*)(w + l.counts);
            a.parts = (const int2*)(w + l.parts);
            hipLaunchKernelGGL(count_kernel, dim3((unsigned)a.part_count), dim3(kCountThreads), 0, s, c.tokens, c.mask, c.B, c.T, a.V,
                               (int*)(w + l.counts), (int2*)(w + l.parts));
            partials = launch_rows<S, kTokenPolicy>(a, c.placed, s);
        }
        hipLaunchKernelGGL(policy_sum_kernel, dim3(1), dim3(kSumThreads), 0, s, a.partial, partials, c.stats);
        return hipGetLastError();
    }
    // preference: log-probabilities, pairs, gradient
    const int64_t pairs = c.B / 2;
    a.rows = (float2*)(w + l.rows);
    a.gaps = (double*)(w + l.sums);
    if (any) launch_rows<S, kTokenForward>(a, c.placed, s);
    double* const losses = (double*)(w + l.losses);
    float* const slopes = (float*)(w + l.counts);
    // One workgroup, and no second launch, where it is done in one turn: a thread per pair of few positions, or a quarter of it per
    // pair of more.  Pairs x positions, one workgroup against two launches: kernels in us, 64 x 64 10.2, 11.3; 256 x 64 15.6, 16.8;
    // 1024 x 8 9.5, 9.2; 512 x 32 15.8, 13.0; 1024 x 16 15.9, 10.9; 1024 x 64 43.9, 19.3; 1 x 777 8.3, 9.4; 4 x 65 8.8, 8.7; 4 x 2048
    // 11.0, 9.5; 8 x 65 11.3, 9.0.  A call made from Python is 2.3 us shorter with one launch less: the lines are where that is lost.
    if (c.T <= 64 && pairs <= 1024 && pairs * c.T <= 16384) {
        hipLaunchKernelGGL((pair_kernel<1024, 1>), dim3(1), dim3(1024), 0, s, a.gaps, pairs, c.T, c.beta, c.smoothing, c.margin, slopes, losses,
                           c.stats);
    } else if (pairs <= 4 && c.T <= 2048) {
        hipLaunchKernelGGL((pair_kernel<1024, 256>), dim3(1), dim3(1024), 0, s, a.gaps, pairs, c.T, c.beta, c.smoothing, c.margin, slopes, losses,
                           c.stats);
    } else {
        const int64_t teams = c.T <= 64 ? 256 : 1, blocks = (pairs + teams - 1) / teams;
        const auto kernel = c.T <= 64 ? pair_kernel<256, 1> : pair_kernel<256, 256>;
        if (pairs > 0)
            hipLaunchKernelGGL(kernel, dim3((unsigned)(blocks < 65536 ? blocks : 65536)), dim3(256), 0, s, a.gaps, pairs, c.T, c.beta, c.smoothing,
                               c.margin, slopes, losses, (float*)nullptr);
        hipLaunchKernelGGL(pair_sum_kernel, dim3(1), dim3(kSumThreads), 0, s, losses, pairs, c.stats);
    }
    if (any && c.grad) {
        a.slope = (const float*)(w + l.counts);
        a.slope_per_token = 0;
        launch_rows<S, kTokenBackward>(a, c.placed, s);
    }
    return hipGetLastError();
}

}  // namespace

size_t token_workspace_bytes(int64_t B, int64_t T) { return layout(B, T).total; }

hipError_t launch_token(TokenKind kind, const TokenCall& c, hipStream_t s) {
    if (c.dtype == kF32) return run<float>(kind, c, s);
    if (c.dtype == kF16) return run<_Float16>(kind, c, s);
    return run<__bf16>(kind, c, s);
}

}  // namespace cc
