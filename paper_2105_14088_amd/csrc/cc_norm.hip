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
// All of this reads a row once: it stays in the registers of a team of 8 to 512 threads between the row's sum and what is
// made of it.  The kernels are bound by memory.  A team takes rows in turn, so that weights are read once, and the gradient of the
// weights is summed in registers over a team's rows.  Rows longer than a team holds are read twice.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "cc_internal.h"
#include "cc_model.h"

namespace cc {
namespace {

using namespace ccm;

constexpr int kBlock = 256;              // threads of a workgroup whose teams are smaller than it
constexpr int kLongBlock = 1024;

struct Args {
    const void *x, *residual, *weight;   // residual and weight may be null
    int64_t n, x_stride, residual_stride, sum_stride, out_stride, q_stride;
    int D;
    double eps;
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
template <int TEAM, class Op>
__device__ __forceinline__ double team_reduce(double v, Op op, double (*lds)[TEAM > 64 ? TEAM / 64 : 1], int slot) {
    if constexpr (TEAM <= 64) {
        return group_reduce64<TEAM>(v, op);
    } else {
        v = group_reduce64<64>(v, op);
        if (threadIdx.x % 64 == 0) lds[slot][threadIdx.x / 64] = v;
        __syncthreads();
        v = lds[slot][0];
#pragma unroll
        for (int i = 1; i < TEAM / 64; ++i) v = op(v, lds[slot][i]);
        return v;
    }
}

// What a row's sums say about it.  `check` is the sum of 0 u: undefined if an element of u is infinite or undefined.
struct RowScale {
    double most;                         // 0: nothing to divide by
    float inverse;                       // 127 / most, where 32 bits hold it
    bool defined;
    __device__ __forceinline__ RowScale(double largest, double check) : most(largest), inverse((float)(127.0 / largest)), defined(check == 0.0) {}
    // s: what the row was not multiplied by
    __device__ __forceinline__ float scale(double s) const { return defined ? (float)(most * s / 127.0) : __builtin_nanf(""); }
    // The whole number nearest to 127 u / most, ties to even.  In 32 bits the quotient is off by less than 127 * 2^-22 (u,
    // the inverse and their product are rounded); where that reaches a border, and where 32 bits do not hold
    // the inverse, it is taken in 64.
    template <class U>
    __device__ __forceinline__ int nearest(float u, U exact) const {
        if (!defined || most == 0.0) return 0;
        const float t = u * inverse;
        float r = __builtin_rintf(t);
        if (!(__builtin_fabsf(t - r) < 0.4999f)) r = (float)__builtin_rint(127.0 * exact() / most);
        return (int)r;
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

// A row's sums over some of its elements, from the element `skip` on.
template <bool NORM, bool QUANT, class S, class W, int VEC>
__device__ __forceinline__ void add_sums(const Pack<S, VEC>& h, const Pack<W, VEC>& w, int skip, double& squares, double& most, double& check) {
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        const double v = (double)h.get(i);
        if constexpr (NORM) squares = __builtin_fma(i < skip ? 0.0 : v, v, squares);
        if constexpr (QUANT) {
            const double u = NORM ? v * (double)w.get(i) : v;
            most = __builtin_fmax(most, __builtin_fabs(u));
            check = __builtin_fma(u, 0.0, check);
        }
    }
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
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const float v = h.get(i), f = w.get(i);
            q[i] = r.nearest(NORM ? v * f : v, [=] { return NORM ? (double)v * (double)f : (double)v; });
        }
        store_bytes(a.q + row * a.q_stride + at, q);
    }
}

// A team per row.  A thread holds K vectors of VEC elements; a vector that would end beyond the row is moved back to end
// with it, and the elements that it then shares with the one before have no second part in the sum of squares.
// Everything is stored behind the row's sums: by then all of the row has been read, and the sum may be stored where x was.
template <class S, class W, int VEC, int TEAM, int K, bool NORM, bool QUANT>
__global__ __launch_bounds__(TEAM > kBlock ? TEAM : kBlock) void norm_kernel(const Args a) {
    constexpr int TEAMS = TEAM > kBlock ? 1 : kBlock / TEAM;
    __shared__ double lds[2 * (1 + QUANT * 2)][TEAM > 64 ? TEAM / 64 : 1];
    const int lane = threadIdx.x % TEAM, team = threadIdx.x / TEAM;
    int at[K], skip[K];
    Pack<W, VEC> w[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int i = (k * TEAM + lane) * VEC;
        at[k] = i < a.D ? min(i, a.D - VEC) : -1;
        skip[k] = i - at[k];
        if constexpr (NORM) w[k] = at[k] >= 0 ? weights<W, VEC>(a.weight, at[k]) : Pack<W, VEC>();
    }
    int slot = 0;
    for (int64_t first = (int64_t)blockIdx.x * TEAMS; first < a.n; first += (int64_t)gridDim.x * TEAMS, slot ^= 1) {
        const int64_t row = first + team;
        const bool live = row < a.n;
        Pack<S, VEC> h[K];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            h[k] = Pack<S, VEC>();
            if (live && at[k] >= 0) h[k] = load_pack<VEC>((const S*)a.x + row * a.x_stride + at[k]);
        }
        if constexpr (NORM)
            if (a.residual) {
                Pack<S, VEC> p[K];
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    p[k] = Pack<S, VEC>();
                    if (live && at[k] >= 0) p[k] = load_pack<VEC>((const S*)a.residual + row * a.residual_stride + at[k]);
                }
#pragma unroll
                for (int k = 0; k < K; ++k) h[k] = added(h[k], p[k]);
            }
        double squares = 0, most = 0, check = 0;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (at[k] >= 0 && skip[k] > 0) add_sums<NORM, QUANT>(h[k], w[k], skip[k], squares, most, check);
            else add_sums<NORM, QUANT>(h[k], w[k], 0, squares, most, check);
        }
        double s = 1.0;
        if constexpr (NORM) {
            squares = team_reduce<TEAM>(squares, Sum64(), lds, slot);
            s = 1.0 / __builtin_sqrt(squares / a.D + a.eps);
        }
        if constexpr (QUANT) {
            most = team_reduce<TEAM>(most, Max64(), lds, 2 + slot);
            check = team_reduce<TEAM>(check, Sum64(), lds, 4 + slot);
        }
        const RowScale r(most, check);
        if (live) {
            if (lane == 0) {
                if constexpr (QUANT) a.scale[row] = r.scale(s);
                if constexpr (NORM)
                    if (a.rstd) a.rstd[row] = (float)s;
            }
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (at[k] >= 0) store_row<NORM, QUANT>(a, row, at[k], h[k], w[k], (float)s, r);
        }
    }
}

// Rows that a team's registers do not hold: a workgroup per row reads it twice.  Every element is read and written by one thread,
// as the sum may be stored where x was.
template <class S, class W, int VEC, bool NORM, bool QUANT>
__global__ __launch_bounds__(kLongBlock) void norm_long_kernel(const Args a) {
    __shared__ double lds[2 * (1 + QUANT * 2)][kLongBlock / 64];
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
        double squares = 0, most = 0, check = 0;
        each([&](auto width, int at) {
            constexpr int N = decltype(width)::value;
            add_sums<NORM, QUANT>(take(width, at), weights<W, N>(a.weight, at), 0, squares, most, check);
        });
        double s = 1.0;
        if constexpr (NORM) {
            squares = team_reduce<kLongBlock>(squares, Sum64(), lds, slot);
            s = 1.0 / __builtin_sqrt(squares / a.D + a.eps);
        }
        if constexpr (QUANT) {
            most = team_reduce<kLongBlock>(most, Max64(), lds, 2 + slot);
            check = team_reduce<kLongBlock>(check, Sum64(), lds, 4 + slot);
        }
        const RowScale r(most, check);
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

// The gradient of a row, by a team as above.  Where there is a gradient of weights, a thread sums its columns over the team's rows,
// then a workgroup's teams are added in their order; norm_weight_kernel adds the workgroups.
template <class S, class W, int VEC, int TEAM, int K>
__global__ __launch_bounds__(TEAM > kBlock ? TEAM : kBlock) void norm_backward_kernel(const GradArgs a) {
    constexpr int TEAMS = TEAM > kBlock ? 1 : kBlock / TEAM, COLUMNS = TEAM * K * VEC;
    __shared__ double lds[2][TEAM > 64 ? TEAM / 64 : 1];
    __shared__ float sums[TEAMS > 1 ? TEAMS * COLUMNS : 1];
    const int lane = threadIdx.x % TEAM, team = threadIdx.x / TEAM;
    int at[K], skip[K];
    Pack<W, VEC> w[K];
    float dw[K][VEC];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int i = (k * TEAM + lane) * VEC;
        at[k] = i < a.D ? min(i, a.D - VEC) : -1;
        skip[k] = i - at[k];
        w[k] = at[k] >= 0 ? weights<W, VEC>(a.weight, at[k]) : Pack<W, VEC>();
#pragma unroll
        for (int i = 0; i < VEC; ++i) dw[k][i] = 0.0f;
    }
    int slot = 0;
    for (int64_t first = (int64_t)blockIdx.x * TEAMS; first < a.n; first += (int64_t)gridDim.x * TEAMS, slot ^= 1) {
        const int64_t row = first + team;
        const bool live = row < a.n;
        const float s = live ? a.rstd[row] : 0.0f;
        Pack<S, VEC> h[K], g[K], more[K];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            h[k] = Pack<S, VEC>();
            g[k] = Pack<S, VEC>();
            more[k] = Pack<S, VEC>();
            if (live && at[k] >= 0) {
                h[k] = load_pack<VEC>((const S*)a.h + row * a.h_stride + at[k]);
                g[k] = load_pack<VEC>((const S*)a.grad + row * a.grad_stride + at[k]);
                if (a.grad_sum) more[k] = load_pack<VEC>((const S*)a.grad_sum + row * a.grad_sum_stride + at[k]);
            }
        }
        float along = 0.0f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            float part = 0.0f, shared = 0.0f;
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const float normed = h[k].get(i) * s, term = g[k].get(i) * normed;
                dw[k][i] += term;
                part = __builtin_fmaf(term, w[k].get(i), part);
                if (at[k] >= 0 && i < skip[k]) shared = __builtin_fmaf(term, w[k].get(i), shared);
            }
            along += part - shared;
        }
        const float mean = (float)(team_reduce<TEAM>((double)along, Sum64(), lds, slot) / a.D);
        if (live) {
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (at[k] >= 0) {
                    float f[VEC];
#pragma unroll
                    for (int i = 0; i < VEC; ++i)
                        f[i] = __builtin_fmaf(s, __builtin_fmaf(-h[k].get(i) * s, mean, g[k].get(i) * w[k].get(i)), more[k].get(i));
                    store_pack((S*)a.grad_h + row * a.grad_h_stride + at[k], Pack<S, VEC>::from(f));
                }
        }
    }
    if (!a.partial) return;
    float* const to = a.partial + (int64_t)blockIdx.x * a.D;
    if constexpr (TEAMS > 1) {
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (at[k] >= 0) __builtin_memcpy(&sums[team * COLUMNS + (k * TEAM + lane) * VEC], dw[k], sizeof(dw[k]));
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
            if (at[k] >= 0) __builtin_memcpy(to + at[k], dw[k], sizeof(dw[k]));
    }
}

// Rows that a team's registers do not hold: a row's sum and its gradient in two readings, every element by one thread.
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

// The weights' gradient of such rows, before grad_h is stored where grad_out may be: a thread has a column of some rows.
template <class S>
__global__ __launch_bounds__(kBlock) void norm_columns_kernel(const GradArgs a, int64_t rows) {
    const int j = blockIdx.x * kBlock + threadIdx.x;
    if (j >= a.D) return;
    const int64_t first = (int64_t)blockIdx.y * rows, end = min(first + rows, a.n);
    float sum = 0.0f;
    for (int64_t row = first; row < end; ++row)
        sum += widen(((const S*)a.grad)[row * a.grad_stride + j]) * (widen(((const S*)a.h)[row * a.h_stride + j]) * a.rstd[row]);
    a.partial[(int64_t)blockIdx.y * a.D + j] = sum;
}

// grad_weight[j] = the sum of `count` partial sums: 64 columns a workgroup, its wavefronts share the sums and are added in order.
template <class W>
__global__ __launch_bounds__(1024) void norm_weight_kernel(const float* __restrict__ partial, int count, int D, W* grad_weight, int accumulate) {
    __shared__ float lds[16][64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, j = blockIdx.x * 64 + lane;
    float sum = 0.0f;
    if (j < D)
        for (int i = wave; i < count; i += 16) sum += partial[(int64_t)i * D + j];
    lds[wave][lane] = sum;
    __syncthreads();
    if (wave == 0 && j < D) {
        for (int i = 1; i < 16; ++i) sum += lds[i][lane];
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
    CC_TEAM(64, 4);
    CC_TEAM(256, 2);
    CC_TEAM(256, 4);
    CC_TEAM(512, 4);
    if constexpr (VEC == 4) CC_TEAM(512, 8);
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
            constexpr int threads = TEAM > kBlock ? TEAM : kBlock, teams = threads / TEAM;
            hipLaunchKernelGGL((norm_kernel<S, W, VEC, TEAM, K, NORM, QUANT>), dim3((unsigned)blocks_for(a.n, teams, threads)), dim3(threads), 0, s, a);
        }
    });
}

// Workgroups that sum columns: each leaves a row of partial sums.
constexpr int64_t kGradBlocks = 1024, kLongParts = 16;
int64_t grad_blocks(int64_t n, int teams, int threads) {
    const int64_t need = (n + teams - 1) / teams, most = kGradBlocks * kBlock / threads;
    return need < most ? need : most;
}

template <class S, class W>
void launch_backward(GradArgs a, const NormBackwardCall& c, hipStream_t s) {
    constexpr int VEC = kVec<S>;
    int64_t count = 0;
    if (a.D < VEC) {
        count = grad_blocks(a.n, kBlock / 8, kBlock);
        hipLaunchKernelGGL((norm_backward_kernel<S, W, 1, 8, 1>), dim3((unsigned)count), dim3(kBlock), 0, s, a);
    } else {
        by_length<VEC>(a.D, [&](auto team, auto k) {
            constexpr int TEAM = decltype(team)::value, K = decltype(k)::value;
            if constexpr (TEAM == 0) {
                count = a.n < kLongParts ? a.n : kLongParts;
                const int64_t rows = (a.n + count - 1) / count;
                if (a.partial)
                    hipLaunchKernelGGL((norm_columns_kernel<S>), dim3((unsigned)((a.D + kBlock - 1) / kBlock), (unsigned)count), dim3(kBlock), 0, s, a, rows);
                hipLaunchKernelGGL((norm_backward_long_kernel<S, W, VEC>), dim3((unsigned)blocks_for(a.n, 1, kLongBlock)), dim3(kLongBlock), 0, s, a);
            } else {
                constexpr int threads = TEAM > kBlock ? TEAM : kBlock, teams = threads / TEAM;
                count = grad_blocks(a.n, teams, threads);
                hipLaunchKernelGGL((norm_backward_kernel<S, W, VEC, TEAM, K>), dim3((unsigned)count), dim3(threads), 0, s, a);
            }
        });
    }
    if (!a.partial) return;
    const dim3 grid((unsigned)((a.D + 63) / 64));
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

// A row of partial sums for every workgroup that leaves one: fewer the longer the row, as by_length and grad_blocks have it for
// the type with the most.
size_t norm_workspace_bytes(int64_t n, int64_t D) {
    const int64_t most = D <= 256 * 4 * 8 ? kGradBlocks : D <= 512 * 4 * 8 ? kGradBlocks * kBlock / 512 : kLongParts;
    return (size_t)(((n < most ? n : most) * D * 4 + 255) / 256 * 256);
}

hipError_t launch_norm_backward(const NormBackwardCall& c, hipStream_t s) {
    if (c.n == 0) {
        // nothing to sum: the weights' gradient is cleared
        const dim3 grid((unsigned)((c.D + 63) / 64));
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
