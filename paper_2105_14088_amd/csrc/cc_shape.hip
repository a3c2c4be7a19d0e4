// Logits shaped before a token is drawn, and the gradient (cc.h: cc_shape_logits, cc_shape_logits_backward).
//
//   z_j > 0 ? z_j / r : z_j r  where j is seen,  less p + f count_j  where it counts,  plus bias_j;  minus infinity where forbidden
//
// Every logit is read once and written once: the kernels are bound by memory.  How often a token is looked back on is counted in
// LDS, a word for each: its top bit says that the token is seen, the others count it from the sequence's start on.  Counts are
// whole numbers, so the order in which they are added does not matter.
//   rows of up to 2048 logits: a wavefront takes consecutive rows of a sequence.  It counts what the first looks back on; each
//   further row looks back on one token more.
//   longer rows: a workgroup takes a stretch of a row and counts the tokens that fall into it.
// An element is read and written by one thread, since the result may be stored where the logits were.
#include <hip/hip_runtime.h>

#include "cc_internal.h"
#include "cc_model.h"

namespace cc {
namespace {

using namespace ccm;

constexpr float kInf = __builtin_inff();
constexpr uint32_t kSeen = 1u << 31;
constexpr int kShortRow = 2048;
constexpr int kThreads = 256, kStretch = 4096;

struct Args {
    const void *logits, *grad;           // grad: backward only
    void* out;
    int64_t T, sb, st, gsb, gst, osb, ost;
    int V;
    const int32_t* history;
    int64_t L, history_stride;
    const int32_t *lengths, *starts;
    const float *penalties, *bias;
    int64_t bias_stride;
    const uint32_t* allowed;
    int64_t allowed_sb, allowed_st;
    int rows;                            // short rows: of a wavefront
    int64_t units;                       // wavefronts or workgroups that have something to do
    int per_row;                         // long rows: stretches;  short rows: wavefronts per sequence
};

// A launch's first dimension holds fewer than 2^32 threads: workgroups beyond kAcross go to the second.
constexpr int64_t kAcross = 1 << 20;
__device__ __forceinline__ int64_t workgroup() { return (int64_t)blockIdx.y * kAcross + blockIdx.x; }
dim3 grid_of(int64_t units) {
    return units <= kAcross ? dim3((unsigned)units) : dim3((unsigned)kAcross, (unsigned)((units + kAcross - 1) / kAcross));
}

struct Penalties {
    float r, inverse, p, f;
    bool forbids;
    __device__ __forceinline__ Penalties(const float* at) : r(at[0]), inverse(1.0f / at[0]), p(at[1]), f(at[2]), forbids(at[1] == kInf || at[2] == kInf) {}
};

template <bool BACK, bool COUNT>
__device__ __forceinline__ float shaped(float z, float g, uint32_t count, const Penalties& pen, float bias, bool allowed) {
    const bool seen = COUNT && count != 0, times = COUNT && (count & ~kSeen) != 0;
    const bool gone = !allowed || bias == -kInf || (times && pen.forbids);
    float v = BACK ? g : z;
    if (seen) v *= z > 0.0f ? pen.inverse : pen.r;
    if constexpr (!BACK) {
        if (times) v = __builtin_fmaf(-pen.f, (float)(count & ~kSeen), v - pen.p);
        v += bias;
    }
    return gone ? (BACK ? 0.0f : -kInf) : v;
}

// N logits of row (b, t) from j on; `count` holds theirs.
template <class S, int N, bool BACK, bool COUNT>
__device__ __forceinline__ void shape_at(const Args& a, const S* z, const S* g, S* out, const float* bias, const uint32_t* allowed, int j,
                                         const uint32_t* count, const Penalties& pen) {
    const Pack<S, N> zp = load_pack<N>(z + j);
    Pack<S, N> gp = {};
    if constexpr (BACK) gp = load_pack<N>(g + j);
    Pack<float, N> bp = {};
    if (bias) bp = load_pack<N>(bias + j);
    const uint32_t bits = allowed ? allowed[j / 32] >> (j % 32) : ~0u;
    uint32_t c[N] = {};
    if constexpr (COUNT) __builtin_memcpy(c, count, sizeof(c));
    float f[N];
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = shaped<BACK, COUNT>(zp.get(i), BACK ? gp.get(i) : 0.0f, c[i], pen, bp.get(i), bits >> i & 1);
    store_pack(out + j, Pack<S, N>::from(f));
}
// Those of the vector at j that the row has.
template <class S, int N, bool BACK, bool COUNT>
__device__ __forceinline__ void shape_vector(const Args& a, const S* z, const S* g, S* out, const float* bias, const uint32_t* allowed, int j,
                                             const uint32_t* count, const Penalties& pen) {
    if (j + N <= a.V) {
        shape_at<S, N, BACK, COUNT>(a, z, g, out, bias, allowed, j, count, pen);
    } else {
        for (int i = 0; j + i < a.V; ++i) shape_at<S, 1, BACK, COUNT>(a, z, g, out, bias, allowed, j + i, count + i, pen);
    }
}

// Entries [0, n) of a history that fall into [from, from + width) are counted, by threads `thread`, `thread` + threads, ...
__device__ __forceinline__ void count_history(const int32_t* history, int64_t n, int64_t start, int from, int width, uint32_t* count, int thread,
                                              int threads) {
    const auto add = [&](int32_t token, int64_t i) {
        const uint32_t at = (uint32_t)token - (uint32_t)from;         // below `from`: beyond any width
        if (at < (uint32_t)width) {
            if (i >= start) atomicAdd(count + at, 1u);
            else atomicOr(count + at, kSeen);
        }
    };
    const int64_t whole = n - n % 4;
    for (int64_t i = 4 * (int64_t)thread; i < whole; i += 4 * (int64_t)threads) {
        const auto tokens = load_pack<4>(history + i);
#pragma unroll
        for (int k = 0; k < 4; ++k) add(tokens.v[k], i + k);
    }
    if (whole + thread < n) add(history[whole + thread], whole + thread);
}

template <class S, int K, bool BACK, bool COUNT>
__global__ __launch_bounds__(kThreads) void short_kernel(const Args a) {
    constexpr int VEC = 16 / sizeof(S), CAP = 64 * VEC * K, WAVES = kThreads / 64;
    __shared__ __attribute__((aligned(16))) uint32_t counts[COUNT ? WAVES : 1][COUNT ? CAP : 1];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t unit = workgroup() * WAVES + wave;
    if (unit >= a.units) return;
    const int64_t b = unit / a.per_row, t0 = unit % a.per_row * a.rows, t1 = min(t0 + a.rows, a.T);
    uint32_t* const count = counts[COUNT ? wave : 0];
    const float one[3] = {1.0f, 0.0f, 0.0f};
    const Penalties pen(COUNT ? a.penalties + 3 * b : one);
    const int32_t* const history = a.history + b * a.history_stride;
    const int64_t start = COUNT && a.starts ? a.starts[b] : 0, length = COUNT && a.lengths ? a.lengths[b] : 0;
    if constexpr (COUNT) {
#pragma unroll
        for (int k = 0; k < K * VEC / 4; ++k) *(Pack<float, 4>*)(count + (k * 64 + lane) * 4) = Pack<float, 4>();
        wave_order();
        count_history(history, min(max(length + t0, (int64_t)0), a.L), start, 0, a.V, count, lane, 64);
        wave_order();
    }
    const float* const bias = a.bias ? a.bias + b * a.bias_stride : nullptr;
    for (int64_t t = t0; t < t1; ++t) {
        const S* const z = (const S*)a.logits + b * a.sb + t * a.st;
        const S* const g = (const S*)a.grad + b * a.gsb + t * a.gst;
        S* const out = (S*)a.out + b * a.osb + t * a.ost;
        const uint32_t* const allowed = a.allowed ? a.allowed + b * a.allowed_sb + t * a.allowed_st : nullptr;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int j = (k * 64 + lane) * VEC;
            if (j < a.V) shape_vector<S, VEC, BACK, COUNT>(a, z, g, out, bias, allowed, j, count + (COUNT ? j : 0), pen);
        }
        if constexpr (COUNT) {
            // the next row looks back on one entry more
            wave_order();
            const int64_t at = length + t;
            if (lane == 0 && t + 1 < t1 && at >= 0 && at < a.L) {
                const int32_t token = history[at];
                if ((uint32_t)token < (uint32_t)a.V) count[token] = at >= start ? count[token] + 1 : count[token] | kSeen;
            }
            wave_order();
        }
    }
}

template <class S, bool BACK, bool COUNT>
__global__ __launch_bounds__(kThreads) void long_kernel(const Args a) {
    constexpr int VEC = 16 / sizeof(S);
    __shared__ __attribute__((aligned(16))) uint32_t count[COUNT ? kStretch : 1];
    const int64_t unit = workgroup();
    if (unit >= a.units) return;
    const int64_t row = unit / a.per_row, b = row / a.T, t = row % a.T;
    const int from = (int)(unit % a.per_row) * kStretch, width = min(kStretch, a.V - from);
    const float one[3] = {1.0f, 0.0f, 0.0f};
    const Penalties pen(COUNT ? a.penalties + 3 * b : one);
    if constexpr (COUNT) {
#pragma unroll
        for (int k = 0; k < kStretch / kThreads / 4; ++k) *(Pack<float, 4>*)(count + (k * kThreads + threadIdx.x) * 4) = Pack<float, 4>();
        __syncthreads();
        const int64_t n = (a.lengths ? a.lengths[b] : 0) + t;
        count_history(a.history + b * a.history_stride, min(max(n, (int64_t)0), a.L), a.starts ? a.starts[b] : 0, from, width, count, threadIdx.x, kThreads);
        __syncthreads();
    }
    const S* const z = (const S*)a.logits + b * a.sb + t * a.st;
    const S* const g = (const S*)a.grad + b * a.gsb + t * a.gst;
    S* const out = (S*)a.out + b * a.osb + t * a.ost;
    const float* const bias = a.bias ? a.bias + b * a.bias_stride : nullptr;
    const uint32_t* const allowed = a.allowed ? a.allowed + b * a.allowed_sb + t * a.allowed_st : nullptr;
#pragma unroll
    for (int k = 0; k < kStretch / kThreads / VEC; ++k) {
        const int in = (k * kThreads + threadIdx.x) * VEC;
        if (in < width) shape_vector<S, VEC, BACK, COUNT>(a, z, g, out, bias, allowed, from + in, count + (COUNT ? in : 0), pen);
    }
}

template <class S, bool BACK, bool COUNT>
void launch(Args a, int64_t B, hipStream_t s) {
    constexpr int VEC = 16 / sizeof(S);
    if (a.V <= kShortRow) {
        // rows of a wavefront: as many as leave 4096 wavefronts, at most 16
        const int64_t rows = COUNT ? B * a.T / 4096 : 1;
        a.rows = (int)(rows < 1 ? 1 : rows > 16 ? 16 : rows);
        a.per_row = (int)((a.T + a.rows - 1) / a.rows);
        a.units = B * a.per_row;
        const dim3 grid = grid_of((a.units + kThreads / 64 - 1) / (kThreads / 64));
        if (a.V <= 64 * VEC) hipLaunchKernelGGL((short_kernel<S, 1, BACK, COUNT>), grid, dim3(kThreads), 0, s, a);
        else if (a.V <= 128 * VEC) hipLaunchKernelGGL((short_kernel<S, 2, BACK, COUNT>), grid, dim3(kThreads), 0, s, a);
        else if (a.V <= 256 * VEC) hipLaunchKernelGGL((short_kernel<S, 4, BACK, COUNT>), grid, dim3(kThreads), 0, s, a);
        else if constexpr (VEC == 4) hipLaunchKernelGGL((short_kernel<S, 8, BACK, COUNT>), grid, dim3(kThreads), 0, s, a);
    } else {
        a.per_row = (a.V + kStretch - 1) / kStretch;
        a.units = B * a.T * a.per_row;
        hipLaunchKernelGGL((long_kernel<S, BACK, COUNT>), grid_of(a.units), dim3(kThreads), 0, s, a);
    }
}

template <class S>
void run(const Args& a, int64_t B, hipStream_t s) {
    const bool count = a.history && a.penalties;
    if (a.grad) count ? launch<S, true, true>(a, B, s) : launch<S, true, false>(a, B, s);
    else count ? launch<S, false, true>(a, B, s) : launch<S, false, false>(a, B, s);
}

}  // namespace

hipError_t launch_shape(const ShapeCall& c, hipStream_t s) {
    Args a = {};
    a.logits = c.logits;
    a.grad = c.grad;
    a.out = c.out;
    a.T = c.T;
    a.sb = c.stride_b;
    a.st = c.stride_t;
    a.gsb = c.grad_stride_b;
    a.gst = c.grad_stride_t;
    a.osb = c.out_stride_b;
    a.ost = c.out_stride_t;
    a.V = (int)c.V;
    a.history = c.history;
    a.L = c.L;
    a.history_stride = c.history_stride;
    a.lengths = c.lengths;
    a.starts = c.starts;
    a.penalties = c.penalties;
    a.bias = c.bias;
    a.bias_stride = c.bias_stride;
    a.allowed = c.allowed;
    a.allowed_sb = c.allowed_stride_b;
    a.allowed_st = c.allowed_stride_t;
    if (c.dtype == kF32) run<float>(a, c.B, s);
    else if (c.dtype == kF16) run<_Float16>(a, c.B, s);
    else run<__bf16>(a, c.B, s);
    return hipGetLastError();
}

}  // namespace cc
