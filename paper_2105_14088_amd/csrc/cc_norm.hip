// Root-mean-square norm with the residual's addition, its gradient, and rows in 8 bits (cc.h: cc_rms_norm,
// cc_rms_norm_backward, cc_quantize_rows).
//
//   h = x + residual (an element of the type),  s = 1 / sqrt(mean of h^2 + eps),  out = h s w
//   u = h w,  q = the whole number nearest to 127 u / max|u|,  scale = s max|u| / 127
//   g = grad_out w,  grad_h = s (g - h s mean(g h s)) + grad_sum,  grad_w = sum over rows of grad_out h s
//
// s is a factor of a whole row, so q does not depend on it: the quotient u / max|u| has the borders of its rounding where exact
// products put them.  It is computed in 32 bits, and again in 64 where 32 cannot tell on which side of a border it lies.
// Squares are summed in 64 bits (an fp32 square may lie beyond the range of 32), which costs nothing beside the memory.
//
// All of this reads a row once: it stays in the registers of a team of 8 to 1024 threads between the row's sum and what is
// made of it.  The kernels are bound by memory.  A team takes rows in turn, so that weights are read once, and the gradient of the
// weights is summed in registers over a team's rows.  Rows longer than a team holds are read twice.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "cc_internal.h"
#include "cc_model.h"

namespace cc {
namespace {

using namespace ccm;

constexpr int kBlock = 256;              // threads of a workgroup of several teams
constexpr int threads_of(int team) { return team > 64 ? team : kBlock; }
constexpr int kLongBlock = 1024;

struct Args {
    const void *x, *residual, *weight;   // residual and weight may be null
    int64_t n, x_stride, residual_stride, sum_stride, out_stride, q_stride;
    int D;
    double eps, per_element;             // 1 / D
    void *sum, *out;                     // either may be null
    int8_t* q;
    float *scale, *rstd;
};
struct GradArgs {
    const void *grad, *h, *weight, *grad_sum;
    const float* rstd;
    void* grad_h;
    float* partial;                      // [workgroups][D], or null: no gradient of weights
    int64_t n, grad_stride, h_stride, grad_sum_stride, grad_h_stride;
    int D;
};

struct Sum64 {
    __device__ __forceinline__ double operator()(double a, double b) const { return a + b; }
};
struct Max64 {
    __device__ __forceinline__ double operator()(double a, double b) const { return __builtin_fmax(a, b); }
};
struct MaxBits {
    __device__ __forceinline__ uint32_t operator()(uint32_t a, uint32_t b) const { return a > b ? a : b; }
};
template <int BIT>
__device__ __forceinline__ double other_lane64(double v) {
    const uint64_t w = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = other_lane<BIT>((uint32_t)w), hi = other_lane<BIT>((uint32_t)(w >> 32));
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double of_halves(uint32_t lo, uint32_t hi) { return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo); }
// As group_reduce, for 64 bits.
template <int G, class Op>
__device__ __forceinline__ double group_reduce64(double v, Op op) {
    if constexpr (G > 1) v = op(v, other_lane64<1>(v));
    if constexpr (G > 2) v = op(v, other_lane64<2>(v));
    if constexpr (G > 4) v = op(v, other_lane64<4>(v));
    if constexpr (G > 8) v = op(v, other_lane64<8>(v));
    if constexpr (G > 16) {
        const uint64_t w = __builtin_bit_cast(uint64_t, v);
        const auto lo = __builtin_amdgcn_permlane16_swap((uint32_t)w, (uint32_t)w, false, false);
        const auto hi = __builtin_amdgcn_permlane16_swap((uint32_t)(w >> 32), (uint32_t)(w >> 32), false, false);
        v = op(of_halves(lo[0], hi[0]), of_halves(lo[1], hi[1]));
    }
    if constexpr (G > 32) {
        const uint64_t w = __builtin_bit_cast(uint64_t, v);
        const auto lo = __builtin_amdgcn_permlane32_swap((uint32_t)w, (uint32_t)w, false, false);
        const auto hi = __builtin_amdgcn_permlane32_swap((uint32_t)(w >> 32), (uint32_t)(w >> 32), false, false);
        v = op(of_halves(lo[0], hi[0]), of_halves(lo[1], hi[1]));
    }
    return v;
}
// Over a team.  One of several wavefronts is the whole workgroup and uses LDS; `slot` alternates between calls, so that one barrier
// a call is enough: a wavefront that is a call ahead writes elsewhere.
template <int TEAM, class V, class Op>
__device__ __forceinline__ V team_reduce(V v, Op op, double (*lds)[TEAM > 64 ? TEAM / 64 : 1], int slot) {
    constexpr int G = TEAM < 64 ? TEAM : 64;
    if constexpr (sizeof(V) == 8) v = group_reduce64<G>(v, op);
    else v = group_reduce<G>(v, op);
    if constexpr (TEAM > 64) {
        V* const to = (V*)lds[slot];
        if (threadIdx.x % 64 == 0) to[threadIdx.x / 64] = v;
        __syncthreads();
        v = to[0];
#pragma unroll
        for (int i = 1; i < TEAM / 64; ++i) v = op(v, to[i]);
    }
    return v;
}

// 1 / sqrt(v) to some 2^-44: the instruction's 2^-23, made better in one step.
__device__ __forceinline__ double inverse_root(double v) {
    const double y = __builtin_amdgcn_rsq(v), e = __builtin_fma(-v * y, y, 1.0);
    return v == __builtin_inf() ? 0.0 : __builtin_fma(y * e, 0.5 + 0.375 * e, y);
}

// What a row's largest element says about it.
struct RowScale {
    double most;                         // 0: nothing to divide by
    float inverse;                       // 127 / most, or NaN where 32 bits might not hold it or its products
    bool defined;
    __device__ __forceinline__ RowScale(double largest, bool finite) : most(largest), defined(finite) {
        const float m = (float)largest;
        inverse = finite && m > 0x1p-100f && m < 0x1p100f ? 127.0f * __builtin_amdgcn_rcpf(m) : __builtin_nanf("");
    }
    // s: what the row was not multiplied by
    __device__ __forceinline__ float scale(double s) const { return defined ? (float)(most * s * (1.0 / 127.0)) : __builtin_nanf(""); }
    // The whole numbers nearest to 127 u / most, ties to even.  In 32 bits a quotient is off by at most 127 * 6 * 2^-24 = 2^-14.4 (u, most, its
    // reciprocal, 127 times that and the product are rounded, the reciprocal to a whole step).  Where that reaches a border, what 127 u has
    // beyond r most says on which side of it the quotient lies: one operation, exact as long as 127 u is, in 64 bits or, where u has at most
    // 16 (R is float then: 127 u and r most have 23, and no bit of either lies below 2^-24 most unless r = 0), in 32.  An element of some
    // 5000 is so near; of bf16 ones one of 500, since half of the largest is a border, and then half of all
    // vectors have one (65536 x 1024: 49 us with a division in 64 bits there, 43 with this in 64, 38 in 32).
    // LONG: u is a product of two 32-bit elements and 127 u may have 55 bits.  What its rounding to 53 leaves out is added last.  The rounded one
    // lies at most some half of most beyond r most, and near a border no bit of it lies below 2^-54 most, so that is exact, and so is how
    // far it is from half of most (fp32 rows of 65536 x 1024: as long as without).
    template <class R, bool LONG, int N, class Exact>
    __device__ __forceinline__ void nearest(const float (&u)[N], Exact exact, int (&q)[N]) const {
        float worst = 0.0f, r[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float t = u[i] * inverse;
            r[i] = __builtin_rintf(t);
            worst = fmaxf(worst, __builtin_fabsf(t - r[i]));
        }
        const auto settle = [&] {
            const R m = (R)most, half = (R)0.5 * m;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const R top = (R)127 * (R)exact(i), beyond = __builtin_elementwise_fma(-(R)r[i], m, top);
                R over = __builtin_elementwise_abs(beyond) - half;
                if constexpr (LONG) {
                    const R rest = __builtin_elementwise_fma((R)127, (R)exact(i), -top);
                    over += beyond > (R)0 ? rest : -rest;
                }
                if (over > (R)0 || (over == (R)0 && ((int)r[i] & 1))) r[i] += beyond > (R)0 ? 1.0f : -1.0f;
            }
        };
        if (__ballot(inverse != inverse) != 0) {
#pragma unroll
            for (int i = 0; i < N; ++i) r[i] = defined && most > 0.0 ? (float)__builtin_rint(127.0 * exact(i) / most) : 0.0f;
            // a quotient of at most 39 and 32 bits is as far from a border as its rounding
            if constexpr (LONG)
                if (defined && most > 0.0) settle();
        } else if (__ballot(!(worst < 0.4999f)) != 0) {
            settle();
        }
#pragma unroll
        for (int i = 0; i < N; ++i) q[i] = (int)r[i];
    }
};

template <int N>
__device__ __forceinline__ void store_bytes(int8_t* p, const int (&q)[N]) {
    if constexpr (N == 1) {
        *p = (int8_t)q[0];
    } else {
        uint32_t w[N / 4];
#pragma unroll
        for (int i = 0; i < N / 4; ++i)
            w[i] = (q[4 * i] & 255) | (q[4 * i + 1] & 255) << 8 | (q[4 * i + 2] & 255) << 16 | (uint32_t)q[4 * i + 3] << 24;
        __builtin_memcpy(p, w, sizeof(w));
    }
}

template <class S, int VEC>
__device__ __forceinline__ Pack<S, VEC> added(const Pack<S, VEC>& a, const Pack<S, VEC>& b) {
    float f[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) f[i] = a.get(i) + b.get(i);
    return Pack<S, VEC>::from(f);
}
template <class W, int VEC>
__device__ __forceinline__ Pack<W, VEC> weights(const void* weight, int64_t at) {
    if (weight) return load_pack<VEC>((const W*)weight + at);
    float one[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) one[i] = 1.0f;
    return Pack<W, VEC>::from(one);
}

// What is found out about a row on the way through it.
template <bool NORM, bool QUANT>
struct Sums {
    double squares = 0.0;                // of h: infinite where an element is, undefined where one is
    double most = 0.0;                   // |u|: a product of finite 32-bit elements is finite in 64
    uint32_t bits = 0;                   // without a norm: the largest |x| by its bits, which infinite and undefined ones exceed
    // Some elements; those before `skip` have been added by another thread.
    template <class S, class W, int VEC>
    __device__ __forceinline__ void add(const Pack<S, VEC>& h, const Pack<W, VEC>& w, int skip) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            if constexpr (NORM) {
                const double v = (double)h.get(i), own = i < skip ? 0.0 : v;     // zero times an infinite v would be undefined
                squares = __builtin_fma(own, own, squares);
                if constexpr (QUANT) most = __builtin_fmax(most, __builtin_fabs(v * (double)w.get(i)));
            } else {
                bits = max(bits, __builtin_bit_cast(uint32_t, h.get(i)) & 0x7fffffffu);
            }
        }
    }
    // The row's factor and scale, once all threads of a team have added theirs.
    template <int TEAM>
    __device__ __forceinline__ RowScale joined(const Args& a, double (*lds)[TEAM > 64 ? TEAM / 64 : 1], int slot, double& s) {
        s = 1.0;
        if constexpr (NORM) {
            squares = team_reduce<TEAM>(squares, Sum64(), lds, slot);
            s = inverse_root(__builtin_fma(squares, a.per_element, a.eps));
            if constexpr (QUANT) most = team_reduce<TEAM>(most, Max64(), lds, 2 + slot);
            return RowScale(most, squares < __builtin_inf() && most < __builtin_inf());
        } else {
            bits = team_reduce<TEAM>(bits, MaxBits(), lds, slot);
            return RowScale((double)__builtin_bit_cast(float, bits), bits < 0x7f800000u);
        }
    }
};
template <class W, int VEC>
__device__ __forceinline__ bool finite(const Pack<W, VEC>& w) {
    bool all = true;
#pragma unroll
    for (int i = 0; i < VEC; ++i) all = all && __builtin_fabsf(w.get(i)) < __builtin_inff();
    return all;
}
template <bool NORM, bool QUANT, class S, class W, int VEC>
__device__ __forceinline__ void store_row(const Args& a, int64_t row, int at, const Pack<S, VEC>& h, const Pack<W, VEC>& w, float s,
                                          const RowScale& r) {
    if constexpr (NORM) {
        if (a.sum) store_pack((S*)a.sum + row * a.sum_stride + at, h);
        if (a.out) {
            float f[VEC];
#pragma unroll
            for (int i = 0; i < VEC; ++i) f[i] = h.get(i) * s * w.get(i);
            store_pack((S*)a.out + row * a.out_stride + at, Pack<S, VEC>::from(f));
        }
    }
    if constexpr (QUANT) {
        int q[VEC];
        float u[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) u[i] = NORM ? h.get(i) * w.get(i) : h.get(i);
        using R = std::conditional_t<(sizeof(S) == 2 && !NORM) || (std::is_same_v<S, __bf16> && std::is_same_v<W, __bf16>), float, double>;
        constexpr bool LONG = NORM && sizeof(S) + sizeof(W) == 8;
        r.template nearest<R, LONG>(u, [&](int i) { return NORM ? (double)h.get(i) * (double)w.get(i) : (double)h.get(i); }, q);
        store_bytes(a.q + row * a.q_stride + at, q);
    }
}

// Where a thread's vectors of a row lie.  One that would end beyond the row is moved back to end with it: its first `skip` elements are
// another's too.  All are loaded, at any length, so that a row's loads are in flight together; one that has no elements of its own
// (skip = VEC) is not stored.
template <int VEC, int TEAM, int K>
struct Place {
    int at[K], skip[K];
    bool uneven[K];                      // of the wavefront: some lane has elements to skip
    __device__ __forceinline__ Place(int lane, int D) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int i = (k * TEAM + lane) * VEC;
            at[k] = min(i, D - VEC);
            skip[k] = min(i - at[k], VEC);
            uneven[k] = __ballot(skip[k] > 0) != 0;
        }
    }
};

// A row into a team's registers.  The teams of a wavefront that has several go on together: one without a row has zeros.
template <int TEAM, int VEC, int K, class S>
__device__ __forceinline__ void load_row(Pack<S, VEC> (&to)[K], const S* row, const Place<VEC, TEAM, K>& place, bool live) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
        if constexpr (TEAM < 64) {
            to[k] = Pack<S, VEC>();
            if (live) to[k] = load_pack<VEC>(row + place.at[k]);
        } else {
            to[k] = load_pack<VEC>(row + place.at[k]);
        }
    }
}

// Bound by memory: 65536 x 1024 bf16 with a residual 91 us in a training pass, 5.9 TB/s, and 102 by itself, 5.3; into 8 bits 94 us, 5.0; rows in 8 bits
// alone 37 us, 5.5.  A
// team per row, the smallest that holds it: with more than 16 elements a thread registers leave too few wavefronts (2048
// columns, four vectors of 64 threads or two of 128).  A thread holds K vectors of VEC elements.  Everything is stored behind the row's
// sums: by then all of the row has been read, and the sum may be stored where x was.
template <class S, class W, int VEC, int TEAM, int K, bool NORM, bool QUANT>
__global__ __launch_bounds__(threads_of(TEAM)) void norm_kernel(const Args a) {
    constexpr int TEAMS = threads_of(TEAM) / TEAM;
    __shared__ double lds[NORM && QUANT ? 4 : 2][TEAM > 64 ? TEAM / 64 : 1];
    const int lane = threadIdx.x % TEAM, team = threadIdx.x / TEAM;
    Place<VEC, TEAM, K> place(lane, a.D);
    Pack<W, VEC> w[K];
    if constexpr (NORM) {
#pragma unroll
        for (int k = 0; k < K; ++k) w[k] = weights<W, VEC>(a.weight, place.at[k]);
    }
    double least = 0.0;                  // an undefined weight makes every row's largest element infinite
    if constexpr (NORM && QUANT) {
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (!finite(w[k])) least = __builtin_inf();
    }
    int slot = 0;
    for (int64_t first = (int64_t)blockIdx.x * TEAMS; first < a.n; first += (int64_t)gridDim.x * TEAMS, slot ^= 1) {
        const int64_t row = first + team;
        const bool live = row < a.n;
        if (TEAM == 64 && !live) break;
        Pack<S, VEC> h[K];
        load_row<TEAM>(h, (const S*)a.x + row * a.x_stride, place, live);
        if constexpr (NORM)
            if (a.residual) {
                Pack<S, VEC> p[K];
                load_row<TEAM>(p, (const S*)a.residual + row * a.residual_stride, place, live);
#pragma unroll
                for (int k = 0; k < K; ++k) h[k] = added(h[k], p[k]);
            }
        Sums<NORM, QUANT> sums;
        sums.most = least;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (place.uneven[k]) sums.add(h[k], w[k], place.skip[k]);
            else sums.add(h[k], w[k], 0);
        }
        double s;
        const RowScale r = sums.template joined<TEAM>(a, lds, slot, s);
        if (live) {
            if (lane == 0) {
                if constexpr (QUANT) a.scale[row] = r.scale(s);
                if constexpr (NORM)
                    if (a.rstd) a.rstd[row] = (float)s;
            }
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (place.skip[k] < VEC) store_row<NORM, QUANT>(a, row, place.at[k], h[k], w[k], (float)s, r);
        }
    }
}

// Rows that a team's registers do not hold: a workgroup per row reads it twice, the second time out of the caches (8192 x 40000 bf16 with a
// residual 580 us, 4.5 TB/s of what is read and written once).  Every element is read and written by one thread,
// as the sum may be stored where x was.
template <class S, class W, int VEC, bool NORM, bool QUANT>
__global__ __launch_bounds__(kLongBlock) void norm_long_kernel(const Args a) {
    __shared__ double lds[NORM && QUANT ? 4 : 2][kLongBlock / 64];
    const int whole = a.D - a.D % VEC;
    int slot = 0;
    for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x, slot ^= 1) {
        const auto take = [&](auto width, int at) {
            constexpr int N = decltype(width)::value;
            Pack<S, N> h = load_pack<N>((const S*)a.x + row * a.x_stride + at);
            if constexpr (NORM)
                if (a.residual) h = added(h, load_pack<N>((const S*)a.residual + row * a.residual_stride + at));
            return h;
        };
        const auto each = [&](auto body) {
            for (int at = threadIdx.x * VEC; at < whole; at += kLongBlock * VEC) body(std::integral_constant<int, VEC>(), at);
            for (int at = whole + threadIdx.x; at < a.D; at += kLongBlock) body(std::integral_constant<int, 1>(), at);
        };
        Sums<NORM, QUANT> sums;
        each([&](auto width, int at) {
            constexpr int N = decltype(width)::value;
            const auto w = weights<W, N>(a.weight, at);
            sums.add(take(width, at), w, 0);
            if constexpr (NORM && QUANT)
                if (!finite(w)) sums.most = __builtin_inf();
        });
        double s;
        const RowScale r = sums.template joined<kLongBlock>(a, lds, slot, s);
        if (threadIdx.x == 0) {
            if constexpr (QUANT) a.scale[row] = r.scale(s);
            if constexpr (NORM)
                if (a.rstd) a.rstd[row] = (float)s;
        }
        each([&](auto width, int at) {
            constexpr int N = decltype(width)::value;
            store_row<NORM, QUANT>(a, row, at, take(width, at), weights<W, N>(a.weight, at), (float)s, r);
        });
    }
}

// The gradient of a row, by a team as above, bound by memory: 65536 x 1024 bf16 with the stream's gradient 103 us by
// itself, 5.2 TB/s, and 115 behind the forward call.  Where there is a gradient of weights, a thread sums its columns over the team's rows,
// then a workgroup's teams are added in their order; norm_weight_kernel adds the workgroups.
template <class S, class W, int VEC, int TEAM, int K>
__global__ __launch_bounds__(threads_of(TEAM)) void norm_backward_kernel(const GradArgs a) {
    constexpr int TEAMS = threads_of(TEAM) / TEAM, COLUMNS = TEAM * K * VEC;
    __shared__ double lds[2][TEAM > 64 ? TEAM / 64 : 1];
    __shared__ float sums[TEAMS > 1 ? TEAMS * COLUMNS : 1];
    const int lane = threadIdx.x % TEAM, team = threadIdx.x / TEAM;
    const Place<VEC, TEAM, K> place(lane, a.D);
    Pack<W, VEC> w[K];
    float dw[K][VEC];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        w[k] = weights<W, VEC>(a.weight, place.at[k]);
#pragma unroll
        for (int i = 0; i < VEC; ++i) dw[k][i] = 0.0f;
    }
    int slot = 0;
    for (int64_t first = (int64_t)blockIdx.x * TEAMS; first < a.n; first += (int64_t)gridDim.x * TEAMS, slot ^= 1) {
        const int64_t row = first + team;
        const bool live = row < a.n;
        if (TEAM == 64 && !live) break;
        const float s = live ? a.rstd[row] : 0.0f;
        Pack<S, VEC> h[K], g[K], more[K] = {};
        load_row<TEAM>(h, (const S*)a.h + row * a.h_stride, place, live);
        load_row<TEAM>(g, (const S*)a.grad + row * a.grad_stride, place, live);
        if (a.grad_sum) load_row<TEAM>(more, (const S*)a.grad_sum + row * a.grad_sum_stride, place, live);
        float along = 0.0f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            float part = 0.0f;
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const float normed = h[k].get(i) * s;
                float term = g[k].get(i) * normed;
                dw[k][i] += term;
                if (place.uneven[k] && i < place.skip[k]) term = 0.0f;
                part = __builtin_fmaf(term, w[k].get(i), part);
            }
            along += part;
        }
        const float mean = (float)(team_reduce<TEAM>((double)along, Sum64(), lds, slot) / a.D);
        if (live) {
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (place.skip[k] < VEC) {
                    float f[VEC];
#pragma unroll
                    for (int i = 0; i < VEC; ++i)
                        f[i] = __builtin_fmaf(s, __builtin_fmaf(-h[k].get(i) * s, mean, g[k].get(i) * w[k].get(i)), more[k].get(i));
                    store_pack((S*)a.grad_h + row * a.grad_h_stride + place.at[k], Pack<S, VEC>::from(f));
                }
        }
    }
    if (!a.partial) return;
    float* const to = a.partial + (int64_t)blockIdx.x * a.D;
    if constexpr (TEAMS > 1) {
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (place.skip[k] < VEC) __builtin_memcpy(&sums[team * COLUMNS + (k * TEAM + lane) * VEC], dw[k], sizeof(dw[k]));
        __syncthreads();
        // the last vector's place holds the row's last VEC columns, wherever they begin
        const int last = (a.D - 1) / VEC;
        for (int j = threadIdx.x; j < a.D; j += kBlock) {
            const int v = j >= a.D - VEC ? last : j / VEC, i = v == last ? j - (a.D - VEC) : j % VEC;
            float sum = 0.0f;
            for (int t = 0; t < TEAMS; ++t) sum += sums[t * COLUMNS + v * VEC + i];
            to[j] = sum;
        }
    } else {
        // columns that two threads hold have the same sum in both
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (place.skip[k] < VEC) __builtin_memcpy(to + place.at[k], dw[k], sizeof(dw[k]));
    }
}

// Rows that a team's registers do not hold: a row's sum and its gradient in two readings, every element by one thread (8192 x 40000 bf16: 562 us,
// 4.7 TB/s of what is read and written once).
template <class S, class W, int VEC>
__global__ __launch_bounds__(kLongBlock) void norm_backward_long_kernel(const GradArgs a) {
    __shared__ double lds[2][kLongBlock / 64];
    const int whole = a.D - a.D % VEC;
    int slot = 0;
    for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x, slot ^= 1) {
        const float s = a.rstd[row];
        const S *h = (const S*)a.h + row * a.h_stride, *g = (const S*)a.grad + row * a.grad_stride;
        const auto each = [&](auto body) {
            for (int at = threadIdx.x * VEC; at < whole; at += kLongBlock * VEC) body(std::integral_constant<int, VEC>(), at);
            for (int at = whole + threadIdx.x; at < a.D; at += kLongBlock) body(std::integral_constant<int, 1>(), at);
        };
        double along = 0;
        each([&](auto width, int at) {
            constexpr int N = decltype(width)::value;
            const auto hp = load_pack<N>(h + at), gp = load_pack<N>(g + at);
            const auto w = weights<W, N>(a.weight, at);
            float part = 0.0f;
#pragma unroll
            for (int i = 0; i < N; ++i) part = __builtin_fmaf(gp.get(i) * (hp.get(i) * s), w.get(i), part);
            along += part;
        });
        const float mean = (float)(team_reduce<kLongBlock>(along, Sum64(), lds, slot) / a.D);
        each([&](auto width, int at) {
            constexpr int N = decltype(width)::value;
            const auto hp = load_pack<N>(h + at), gp = load_pack<N>(g + at);
            const auto w = weights<W, N>(a.weight, at);
            Pack<S, N> more = {};
            if (a.grad_sum) more = load_pack<N>((const S*)a.grad_sum + row * a.grad_sum_stride + at);
            float f[N];
#pragma unroll
            for (int i = 0; i < N; ++i) f[i] = __builtin_fmaf(s, __builtin_fmaf(-hp.get(i) * s, mean, gp.get(i) * w.get(i)), more.get(i));
            store_pack((S*)a.grad_h + row * a.grad_h_stride + at, Pack<S, N>::from(f));
        });
    }
}

// The weights' gradient of such rows, before grad_h is stored where grad_out may be: a thread has 4 columns of some rows.  The last
// thread's are moved back to end with the row; the columns that it shares have the same sums in both.  8192 x 40000 bf16: 305 us, the third
// reading of g and h; beside the row's second reading it was not tried.
template <class S>
__global__ __launch_bounds__(kBlock) void norm_columns_kernel(const GradArgs a, int64_t rows) {
    constexpr int N = 4, U = 4;
    int j = (blockIdx.x * kBlock + threadIdx.x) * N;
    if (j >= a.D) return;
    j = min(j, a.D - N);
    const int64_t first = (int64_t)blockIdx.y * rows, end = min(first + rows, a.n);
    float sum[N] = {};
    for (int64_t row = first; row < end; row += U) {
        Pack<S, N> g[U], h[U];
        float s[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t r = min(row + u, end - 1);
            g[u] = load_pack<N>((const S*)a.grad + r * a.grad_stride + j);
            h[u] = load_pack<N>((const S*)a.h + r * a.h_stride + j);
            s[u] = a.rstd[r];
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (row + u < end) {
#pragma unroll
                for (int i = 0; i < N; ++i) sum[i] += g[u].get(i) * (h[u].get(i) * s[u]);
            }
    }
    __builtin_memcpy(a.partial + (int64_t)blockIdx.y * a.D + j, sum, sizeof(sum));
}

// grad_weight[j] = the sum of `count` partial sums.  16 columns a workgroup; 64 groups of 16 lanes take the sums in turn, eight loads
// in flight each, and are added in a fixed order.  1024 sums of 1024 columns: 4.6 us, of which the loads' latency is most.
template <class W>
__global__ __launch_bounds__(1024) void norm_weight_kernel(const float* __restrict__ partial, int count, int D, W* grad_weight, int accumulate) {
    __shared__ float lds[16][16];
    const int in = threadIdx.x % 16, group = threadIdx.x / 16, j = blockIdx.x * 16 + in;
    float sum = 0.0f;
    if (j < D) {
        int i = group;
        for (; i + 7 * 64 < count; i += 8 * 64) {
            float v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) v[u] = partial[(int64_t)(i + u * 64) * D + j];
#pragma unroll
            for (int u = 0; u < 8; ++u) sum += v[u];
        }
        for (; i < count; i += 64) sum += partial[(int64_t)i * D + j];
    }
    sum += __shfl_xor(sum, 16, 64);
    sum += __shfl_xor(sum, 32, 64);
    if (threadIdx.x % 64 < 16) lds[threadIdx.x / 64][in] = sum;
    __syncthreads();
    if (threadIdx.x < 16 && j < D) {
        sum = lds[0][in];
        for (int i = 1; i < 16; ++i) sum += lds[i][in];
        if (accumulate) sum += widen(grad_weight[j]);
        grad_weight[j] = narrow<W>(sum);
    }
}

constexpr int64_t kMostBlocks = 2048;    // of 256 threads: as many as the card holds at once

int64_t blocks_for(int64_t n, int teams, int threads) {
    const int64_t need = (n + teams - 1) / teams, most = kMostBlocks * kBlock / threads;
    return need < most ? need : most;
}

// Calls f with the team and the vectors a thread holds: the fewest that hold a row; f.long_row() where none do.
template <int VEC, class F>
void by_length(int64_t D, F f) {
    using std::integral_constant;
#define CC_TEAM(TEAM, K) \
    if (D <= TEAM * K * VEC) return f(integral_constant<int, TEAM>(), integral_constant<int, K>())
    CC_TEAM(8, 1);
    CC_TEAM(16, 1);
    CC_TEAM(32, 1);
    CC_TEAM(64, 1);
    CC_TEAM(64, 2);
    if constexpr (VEC == 8) {
        CC_TEAM(128, 2);
        CC_TEAM(256, 2);
        CC_TEAM(512, 2);
        CC_TEAM(1024, 2);
    } else {
        CC_TEAM(64, 4);
        CC_TEAM(128, 4);
        CC_TEAM(256, 4);
        CC_TEAM(512, 4);
        CC_TEAM(512, 8);
    }
#undef CC_TEAM
    f(integral_constant<int, 0>(), integral_constant<int, 0>());
}
template <class S>
constexpr int kVec = 16 / sizeof(S);

template <class S, class W, bool NORM, bool QUANT>
void launch_rows(const Args& a, hipStream_t s) {
    constexpr int VEC = kVec<S>;
    if (a.D < VEC) {
        hipLaunchKernelGGL((norm_kernel<S, W, 1, 8, 1, NORM, QUANT>), dim3((unsigned)blocks_for(a.n, kBlock / 8, kBlock)), dim3(kBlock), 0, s, a);
        return;
    }
    by_length<VEC>(a.D, [&](auto team, auto k) {
        constexpr int TEAM = decltype(team)::value, K = decltype(k)::value;
        if constexpr (TEAM == 0) {
            hipLaunchKernelGGL((norm_long_kernel<S, W, VEC, NORM, QUANT>), dim3((unsigned)blocks_for(a.n, 1, kLongBlock)), dim3(kLongBlock), 0, s, a);
        } else {
            constexpr int threads = threads_of(TEAM), teams = threads / TEAM;
            hipLaunchKernelGGL((norm_kernel<S, W, VEC, TEAM, K, NORM, QUANT>), dim3((unsigned)blocks_for(a.n, teams, threads)), dim3(threads), 0, s, a);
        }
    });
}

// Workgroups that sum columns: each leaves a row of partial sums.
constexpr int64_t kGradBlocks = 1024, kLongParts = 32;
int64_t grad_blocks(int64_t n, int teams, int threads) {
    const int64_t need = (n + teams - 1) / teams, most = kGradBlocks * kBlock / threads;
    return need < most ? need : most;
}
// Rows of each part of a long row's sums, so that no part is empty.
int64_t rows_of_part(int64_t n) { return (n + kLongParts - 1) / kLongParts; }
// How many partial sums there are of a column.
template <int VEC>
int64_t partial_rows(int64_t n, int64_t D) {
    if (n == 0) return 0;
    if (D < VEC) return grad_blocks(n, kBlock / 8, kBlock);
    int64_t count = 0;
    by_length<VEC>(D, [&](auto team, auto) {
        constexpr int TEAM = decltype(team)::value;
        if constexpr (TEAM == 0) count = (n + rows_of_part(n) - 1) / rows_of_part(n);
        else count = grad_blocks(n, threads_of(TEAM) / TEAM, threads_of(TEAM));
    });
    return count;
}

template <class S, class W>
void launch_backward(GradArgs a, const NormBackwardCall& c, hipStream_t s) {
    constexpr int VEC = kVec<S>;
    const int64_t count = partial_rows<VEC>(a.n, a.D);
    if (a.D < VEC) {
        hipLaunchKernelGGL((norm_backward_kernel<S, W, 1, 8, 1>), dim3((unsigned)count), dim3(kBlock), 0, s, a);
    } else {
        by_length<VEC>(a.D, [&](auto team, auto k) {
            constexpr int TEAM = decltype(team)::value, K = decltype(k)::value;
            if constexpr (TEAM == 0) {
                if (a.partial)
                    hipLaunchKernelGGL((norm_columns_kernel<S>), dim3((unsigned)((a.D + kBlock * 4 - 1) / (kBlock * 4)), (unsigned)count), dim3(kBlock), 0, s, a,
                                       rows_of_part(a.n));
                hipLaunchKernelGGL((norm_backward_long_kernel<S, W, VEC>), dim3((unsigned)blocks_for(a.n, 1, kLongBlock)), dim3(kLongBlock), 0, s, a);
            } else {
                hipLaunchKernelGGL((norm_backward_kernel<S, W, VEC, TEAM, K>), dim3((unsigned)count), dim3(threads_of(TEAM)), 0, s, a);
            }
        });
    }
    if (!a.partial) return;
    const dim3 grid((unsigned)((a.D + 15) / 16));
    if (c.grad_weight_dtype == kF32)
        hipLaunchKernelGGL((norm_weight_kernel<float>), grid, dim3(1024), 0, s, a.partial, (int)count, a.D, (float*)c.grad_weight, (int)c.accumulate);
    else
        hipLaunchKernelGGL((norm_weight_kernel<W>), grid, dim3(1024), 0, s, a.partial, (int)count, a.D, (W*)c.grad_weight, (int)c.accumulate);
}

template <class S>
void backward_by_weight(const GradArgs& a, const NormBackwardCall& c, hipStream_t s) {
    if (c.weight_dtype == kF32) launch_backward<S, float>(a, c, s);
    else launch_backward<S, S>(a, c, s);
}

template <class S>
void forward_by_weight(const Args& a, const NormCall& c, hipStream_t s) {
    if (c.weight_dtype == kF32) c.q ? launch_rows<S, float, true, true>(a, s) : launch_rows<S, float, true, false>(a, s);
    else c.q ? launch_rows<S, S, true, true>(a, s) : launch_rows<S, S, true, false>(a, s);
}

}  // namespace

hipError_t launch_norm(const NormCall& c, hipStream_t s) {
    if (c.n == 0) return hipSuccess;
    Args a = {};
    a.x = c.x;
    a.residual = c.residual;
    a.weight = c.weight;
    a.n = c.n;
    a.x_stride = c.x_stride;
    a.residual_stride = c.residual_stride;
    a.sum_stride = c.sum_stride;
    a.out_stride = c.out_stride;
    a.q_stride = c.q_stride;
    a.D = (int)c.D;
    a.eps = c.eps;
    a.per_element = 1.0 / (double)c.D;
    a.sum = c.sum;
    a.out = c.out;
    a.q = c.q;
    a.scale = c.scale;
    a.rstd = c.rstd;
    if (c.dtype == kF32) forward_by_weight<float>(a, c, s);
    else if (c.dtype == kF16) forward_by_weight<_Float16>(a, c, s);
    else forward_by_weight<__bf16>(a, c, s);
    return hipGetLastError();
}

hipError_t launch_quantize(const NormCall& c, hipStream_t s) {
    if (c.n == 0) return hipSuccess;
    Args a = {};
    a.x = c.x;
    a.n = c.n;
    a.x_stride = c.x_stride;
    a.q_stride = c.q_stride;
    a.D = (int)c.D;
    a.q = c.q;
    a.scale = c.scale;
    if (c.dtype == kF32) launch_rows<float, float, false, true>(a, s);
    else if (c.dtype == kF16) launch_rows<_Float16, _Float16, false, true>(a, s);
    else launch_rows<__bf16, __bf16, false, true>(a, s);
    return hipGetLastError();
}

// A row of partial sums for every workgroup that leaves one; the type is not known here, so for the one that has more.
size_t norm_workspace_bytes(int64_t n, int64_t D) {
    const int64_t wide = partial_rows<kVec<_Float16>>(n, D), narrow = partial_rows<kVec<float>>(n, D);
    return (size_t)(((wide > narrow ? wide : narrow) * D * 4 + 255) / 256 * 256);
}

hipError_t launch_norm_backward(const NormBackwardCall& c, hipStream_t s) {
    if (c.n == 0) {
        // nothing to sum: the weights' gradient is cleared
        const dim3 grid((unsigned)((c.D + 15) / 16));
        if (c.grad_weight_dtype == kF32)
            hipLaunchKernelGGL((norm_weight_kernel<float>), grid, dim3(1024), 0, s, nullptr, 0, (int)c.D, (float*)c.grad_weight, 0);
        else if (c.grad_weight_dtype == kF16)
            hipLaunchKernelGGL((norm_weight_kernel<_Float16>), grid, dim3(1024), 0, s, nullptr, 0, (int)c.D, (_Float16*)c.grad_weight, 0);
        else
            hipLaunchKernelGGL((norm_weight_kernel<__bf16>), grid, dim3(1024), 0, s, nullptr, 0, (int)c.D, (__bf16*)c.grad_weight, 0);
        return hipGetLastError();
    }
    GradArgs a = {};
    a.grad = c.grad;
    a.h = c.h;
    a.weight = c.weight;
    a.grad_sum = c.grad_sum;
    a.rstd = c.rstd;
    a.grad_h = c.grad_h;
    a.partial = c.grad_weight ? (float*)c.workspace : nullptr;
    a.n = c.n;
    a.grad_stride = c.grad_stride;
    a.h_stride = c.h_stride;
    a.grad_sum_stride = c.grad_sum_stride;
    a.grad_h_stride = c.grad_h_stride;
    a.D = (int)c.D;
    if (c.dtype == kF32) backward_by_weight<float>(a, c, s);
    else if (c.dtype == kF16) backward_by_weight<_Float16>(a, c, s);
    else backward_by_weight<__bf16>(a, c, s);
    return hipGetLastError();
}

}  // namespace cc
