// Logits shaped before a token is drawn, and the gradient (cc.h: cc_shape_logits, cc_shape_logits_backward).
//
//   z_j > 0 ? z_j / r : z_j r  where j is seen,  less p + f count_j  where it counts,  plus bias_j;  minus infinity where forbidden
//
// Every logit is read once and written once: the kernels are bound by memory, and the shorter the rows the more by what they do for an
// element.  How often a token is looked back on is counted in LDS, a word for each: its top bit says that the token is seen, the
// others count it from the sequence's start on.  Where penalties only forbid (r = 1, p or f infinite), a bit for each says
// enough; nothing is then done for an element but to add its bias, and the gradient needs no logits.  Counts are whole numbers, so
// the order in which they are added does not matter.
//   rows of up to 2048 logits: a wavefront takes consecutive rows of a sequence.  It counts what the first looks back on; each
//   further row looks back on one token more.
//   longer rows: a workgroup takes a stretch of a row and counts the tokens that fall into it.
// The result may be stored where the logits were: a wavefront reads all of a row before it stores any of it (what ends beyond the row is moved
// back and shares elements with another vector), in longer rows an element is read and written by one thread.
#include <hip/hip_runtime.h>

#include "cc_internal.h"
#include "cc_model.h"

namespace cc {
namespace {

using namespace ccm;

constexpr float kInf = __builtin_inff();
constexpr uint32_t kSeen = 1u << 31;
constexpr int kShortRow = 2048;
constexpr int kThreads = 256;
constexpr int kEach = 16;                // elements of a thread in a stretch of a long row

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

// A division of 64 bits takes some 100 operations: most calls need none.
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {
    return (uint64_t)(a | b) >> 32 ? a / b : (int64_t)((uint32_t)a / (uint32_t)b);
}

// A value that all lanes have, in a scalar register.
__device__ __forceinline__ float uniform(float v) { return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, v))); }
struct Penalties {
    float r, p, f;
    bool forbids, only;                  // forbids what counts, and does nothing else
    // 1 / r = (high + low) 2^-shift to some 2^-47; `inverse` is high + low, rounded.  Both parts are of r's sign, and low is zero only if high is:
    // their products with an infinity add up to one.  shift is 0 unless r or its reciprocal may not have all bits.
    float inverse, high, low;
    int shift;
    __device__ __forceinline__ Penalties(const float* at) : r(uniform(at[0])), p(uniform(at[1])), f(uniform(at[2])) {
        forbids = p == kInf || f == kInf;
        only = forbids && r == 1.0f;
        shift = __builtin_fabsf(r) >= 0x1p-100f && __builtin_fabsf(r) <= 0x1p100f ? 0 : __builtin_amdgcn_frexp_expf(r) - 1;
        const float d = __builtin_amdgcn_ldexpf(r, -shift);
        inverse = uniform(1.0f / d);
        const bool beyond = __builtin_fmaf(inverse, d, -1.0f) > 0.0f;
        high = uniform(__builtin_bit_cast(float, __builtin_bit_cast(uint32_t, inverse) - beyond));
        low = high == 0.0f ? 0.0f : uniform(__builtin_copysignf(__builtin_fmaxf(__builtin_fabsf(__builtin_fmaf(-high, d, 1.0f) * high), 0x1p-149f), r));
    }
};

// `count` words at an element's address; N bits of a mask from bit j on, which may lie in two words.
template <int N>
__device__ __forceinline__ uint32_t bits_at(const uint32_t* words, int j, int last) {
    const uint32_t low = words[j / 32] >> (j % 32);
    if constexpr (N == 1) return low;
    return j % 32 + N <= 32 ? low : low | words[min(j / 32 + 1, last)] << (32 - j % 32);
}
// The biases that forbid, as bits.
template <int N>
__device__ __forceinline__ uint32_t banned(const Pack<float, N>& bias) {
    uint32_t bits = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) bits |= (uint32_t)(bias.get(i) == -kInf) << i;
    return bits;
}

// Where penalties do nothing, or only forbid: `in` are the logits, or the gradient.
template <class S, int N, bool BACK>
__device__ __forceinline__ Pack<S, N> shaped_plainly(const Pack<S, N>& in, const Pack<float, N>& bias, uint32_t live) {
    float f[N];
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = live >> i & 1 ? (BACK ? in.get(i) : in.get(i) + bias.get(i)) : (BACK ? 0.0f : -kInf);
    return Pack<S, N>::from(f);
}
template <class S, int N, bool BACK>
__device__ __forceinline__ Pack<S, N> shaped(const Pack<S, N>& z, const Pack<S, N>& g, const uint32_t (&count)[N], const Penalties& pen,
                                             const Pack<float, N>& bias, uint32_t live) {
    uint32_t any = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) any |= count[i];
    if (__ballot(any != 0) == 0) return shaped_plainly<S, N, BACK>(BACK ? g : z, bias, live);
    // Quotients of 32 bits are rounded once, as a division's are, in two operations for some ten (32 x 500 x 2000 counted: forward 77 us, with a
    // division 87, with the product by a rounded reciprocal 75; backward 141, 161, 137).  What is rounded to 16 bits may be off by 2^-23.4 before:
    // there it is the product.
    float f[N];
    if constexpr (sizeof(S) == 4) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float from = z.get(i), v = BACK ? g.get(i) : from;
            f[i] = count[i] && from > 0.0f ? __builtin_fmaf(v, pen.high, v * pen.low) : v * (count[i] ? pen.r : 1.0f);
        }
        if (pen.shift) {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (count[i] && z.get(i) > 0.0f) f[i] = __builtin_amdgcn_ldexpf(f[i], -pen.shift);
        }
    } else if (pen.shift) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float from = z.get(i), v = BACK ? g.get(i) : from;
            f[i] = count[i] ? from > 0.0f ? __builtin_amdgcn_ldexpf(v * pen.inverse, -pen.shift) : v * pen.r : v;
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float from = z.get(i), v = BACK ? g.get(i) : from;
            f[i] = v * (count[i] ? from > 0.0f ? pen.inverse : pen.r : 1.0f);
        }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const uint32_t times = count[i] & ~kSeen;
        float v = f[i];
        if constexpr (!BACK) v = (times ? __builtin_fmaf(-pen.f, (float)times, v - pen.p) : v) + bias.get(i);
        f[i] = (live >> i & 1) && !(times && pen.forbids) ? v : (BACK ? 0.0f : -kInf);
    }
    return Pack<S, N>::from(f);
}

// What entries do to their token's word or, where penalties only forbid, to its bit.
__device__ __forceinline__ void note(uint32_t* counts, uint32_t at, bool only, bool counted, uint32_t times) {
    if (counted) {
        if (only) atomicOr(counts + at / 32, 1u << (at % 32));
        else atomicAdd(counts + at, times);
    } else if (!only) {
        atomicOr(counts + at, kSeen);
    }
}
// The first n entries of a history that fall into [from, from + width), those from `start` on counted: threads `thread`, `thread` + threads, ...
// take four each.  Every stretch of a row goes through all of its history, so little is done for an entry; where most lanes have one, a
// token that many of them have is added for all at once (4096 entries of one token, each by itself, took 50 us of a call's 62).
__device__ __forceinline__ void look_back(const int32_t* history, int n, int start, int from, int width, int thread, int threads, uint32_t* counts,
                                          bool only) {
    const auto place = [&](int32_t token) { return (uint32_t)token - (uint32_t)from; };     // below `from`: beyond any width
    const auto each = [&](uint32_t at, int i) {
        if (at < (uint32_t)width) note(counts, at, only, i >= start, 1u);
    };
    const auto crowd = [&](uint32_t at, int i) {
        bool mine = at < (uint32_t)width;
        const uint64_t here = __ballot(mine);
        if (here == 0) return;
        const uint32_t leader = __builtin_ctzll(here), first = __builtin_amdgcn_readlane(at, leader);
        const uint64_t same = __ballot(mine && at == first), counted = __ballot(mine && at == first && i >= start);
        if (__builtin_popcountll(same) > 4) {
            if (threadIdx.x % 64 == leader) note(counts, first, only, counted != 0, __builtin_popcountll(counted));
            mine = mine && at != first;
        }
        if (mine) note(counts, at, only, i >= start, 1u);
    };
    if (n < 4) {
        if (thread < n) each(place(history[thread]), thread);
        return;
    }
    // what would end beyond the history is moved back to end with it, and what another thread has there is no token (-1) in this one
    const auto load = [&](int64_t i) { return load_pack<4>(history + min(i, (int64_t)n - 4)); };
    int64_t i = 4 * (int64_t)thread;
    Pack<int32_t, 4> next = load(i);
    for (int64_t first = 0; first < n; first += 4 * threads, i += 4 * threads) {
        Pack<int32_t, 4> tokens = next;
        if (first + 4 * threads < n) next = load(i + 4 * threads);
        const int moved = (int)max(i - (n - 4), (int64_t)0);
        if (moved > 0) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (k < moved) tokens.v[k] = -1;
        }
        const int at = (int)i - moved;
        if (__builtin_popcountll(__ballot(place(tokens.v[0]) < (uint32_t)width)) <= 32) {
#pragma unroll
            for (int k = 0; k < 4; ++k) each(place(tokens.v[k]), at + k);
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) crowd(place(tokens.v[k]), at + k);
        }
    }
}

// 64 lanes, K vectors each, for a row.  The next row is on its way while one is worked on.  Bound by memory where penalties only forbid: 64 x
// 1000 x 1000 bf16 61 us, 4.2 TB/s; with counts forward 68 us (3.8 TB/s) and gradient 90 (4.3): their 22 and 19
// vector operations a logit keep the SIMDs busy for 36 and 31 us, and with four wavefronts on each they do not all hide behind the memory.
template <class S, int VEC, int K, bool BACK, bool COUNT>
__global__ __launch_bounds__(kThreads) void short_kernel(const Args a) {
    constexpr int CAP = 64 * VEC * K, WAVES = kThreads / 64;
    __shared__ __attribute__((aligned(16))) uint32_t counts[COUNT ? WAVES : 1][COUNT ? (CAP < 256 ? 256 : CAP) : 1];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int64_t unit = workgroup() * WAVES + wave;
    if (unit >= a.units) return;
    const int64_t b = quotient(unit, a.per_row), t0 = (unit - b * a.per_row) * a.rows, t1 = min(t0 + a.rows, a.T);
    uint32_t* const count = counts[COUNT ? wave : 0];
    const float one[3] = {1.0f, 0.0f, 0.0f};
    const Penalties pen(COUNT ? a.penalties + 3 * b : one);
    const bool plain = !COUNT || pen.only;
    int at[K];
#pragma unroll
    for (int k = 0; k < K; ++k) at[k] = min((k * 64 + lane) * VEC, a.V - VEC);

    Pack<S, VEC> z[K], g[K];
    const auto load = [&](int64_t t, Pack<S, VEC>(&zs)[K], Pack<S, VEC>(&gs)[K]) {
        const S* const zrow = (const S*)a.logits + b * a.sb + t * a.st;
        const S* const grow = (const S*)a.grad + b * a.gsb + t * a.gst;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (BACK) gs[k] = load_pack<VEC>(grow + at[k]);
            if (!BACK || !plain) zs[k] = load_pack<VEC>(zrow + at[k]);
        }
    };
    load(t0, z, g);
    Pack<float, VEC> bias[K] = {};
    uint32_t ban[K] = {};
    if (a.bias) {
#pragma unroll
        for (int k = 0; k < K; ++k) bias[k] = load_pack<VEC>(a.bias + b * a.bias_stride + at[k]);
#pragma unroll
        for (int k = 0; k < K; ++k) ban[k] = banned(bias[k]);
    }
    const int32_t* const history = a.history + b * a.history_stride;
    const int start = COUNT && a.starts ? a.starts[b] : 0;
    const int64_t length = COUNT && a.lengths ? a.lengths[b] : 0;
    const int last = (a.V - 1) / 32;
    uint32_t later = ~0u;                // a lane for each row: the entry that the next one looks back on as well
    if constexpr (COUNT) {
        const int64_t entry = length + t0 + lane;
        if (lane < a.rows && entry >= 0 && entry < a.L) later = (uint32_t)history[entry];
        for (int i = lane * 4; i < (plain ? last + 1 : a.V); i += 256) *(Pack<float, 4>*)(count + i) = Pack<float, 4>();
        wave_order();
        look_back(history, (int)min(max(length + t0, (int64_t)0), a.L), start, 0, a.V, lane, 64, count, plain);
        wave_order();
    }
    for (int64_t t = t0; t < t1; ++t) {
        Pack<S, VEC> z1[K], g1[K];
        if (t + 1 < t1) load(t + 1, z1, g1);
        const uint32_t* const allowed = a.allowed ? a.allowed + b * a.allowed_sb + t * a.allowed_st : nullptr;
        S* const out = (S*)a.out + b * a.osb + t * a.ost;
        uint32_t live[K];
#pragma unroll
        for (int k = 0; k < K; ++k) live[k] = (allowed ? bits_at<VEC>(allowed, at[k], last) : ~0u) & ~ban[k];
        Pack<S, VEC> r[K];
        if (plain) {
#pragma unroll
            for (int k = 0; k < K; ++k)
                r[k] = shaped_plainly<S, VEC, BACK>(BACK ? g[k] : z[k], bias[k], COUNT ? live[k] & ~bits_at<VEC>(count, at[k], last) : live[k]);
        } else {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                uint32_t c[VEC];
                __builtin_memcpy(c, count + at[k], sizeof(c));
                r[k] = shaped<S, VEC, BACK>(z[k], g[k], c, pen, bias[k], live[k]);
            }
        }
#pragma unroll
        for (int k = 0; k < K; ++k)
            if ((k * 64 + lane) * VEC < a.V) store_pack(out + at[k], r[k]);
        if constexpr (COUNT) {
            // the next row looks back on one entry more
            wave_order();
            const uint32_t token = __builtin_amdgcn_readlane(later, (int)(t - t0));
            if (token < (uint32_t)a.V && lane == 0) note(count, token, plain, length + t >= start, 1u);
            wave_order();
        }
#pragma unroll
        for (int k = 0; k < K; ++k) {
            z[k] = z1[k];
            g[k] = g1[k];
        }
    }
}

// A stretch of a row: 128 rows of 131072 bf16 12 us without a history (5.5 TB/s), 21 with some 2000 entries each, as unequal as words.
// Every row counts its history anew, also where it is one entry longer than the row before: 8 x 512 x 32000 bf16 157 us, 106 without a history.  A
// vector that would end beyond the row is taken element by element.
template <class S, int THREADS, bool BACK, bool COUNT>
__global__ __launch_bounds__(THREADS) void long_kernel(const Args a) {
    constexpr int VEC = 16 / sizeof(S), K = kEach / VEC, STRETCH = kEach * THREADS;
    __shared__ __attribute__((aligned(16))) uint32_t count[COUNT ? STRETCH : 1];
    const int64_t unit = workgroup();
    if (unit >= a.units) return;
    const int64_t row = quotient(unit, a.per_row), b = quotient(row, a.T), t = row - b * a.T;
    // Every eighth workgroup is on the same XCD, and the first stretch often has most of a history: rows begin at another each.
    int turned = (int)(unit - row * a.per_row) + (int)((uint32_t)row % (uint32_t)a.per_row);
    if (turned >= a.per_row) turned -= a.per_row;
    const int from = turned * STRETCH, width = min(STRETCH, a.V - from);
    const float one[3] = {1.0f, 0.0f, 0.0f};
    const Penalties pen(COUNT ? a.penalties + 3 * b : one);
    const bool plain = !COUNT || pen.only;
    const S* const zrow = (const S*)a.logits + b * a.sb + t * a.st + from;
    const S* const grow = (const S*)a.grad + b * a.gsb + t * a.gst + from;
    S* const out = (S*)a.out + b * a.osb + t * a.ost + from;
    const float* const biases = a.bias ? a.bias + b * a.bias_stride + from : nullptr;
    const uint32_t* const allowed = a.allowed ? a.allowed + b * a.allowed_sb + t * a.allowed_st + from / 32 : nullptr;

    if constexpr (COUNT) {
        const int words = plain ? STRETCH / 32 : STRETCH;
        for (int i = threadIdx.x * 4; i < words; i += THREADS * 4) *(Pack<float, 4>*)(count + i) = Pack<float, 4>();
        __syncthreads();
        const int64_t n = (a.lengths ? a.lengths[b] : 0) + t;
        const int start = a.starts ? a.starts[b] : 0;
        look_back(a.history + b * a.history_stride, (int)min(max(n, (int64_t)0), a.L), start, from, width, threadIdx.x, THREADS, count, plain);
        __syncthreads();
    }
    Pack<S, VEC> z[K] = {}, g[K] = {};
    Pack<float, VEC> bias[K] = {};
    uint32_t live[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int in = (k * THREADS + threadIdx.x) * VEC;
        live[k] = ~0u;
        if (in + VEC <= width) {
            if (BACK) g[k] = load_pack<VEC>(grow + in);
            if (!BACK || !plain) z[k] = load_pack<VEC>(zrow + in);
            if (biases) bias[k] = load_pack<VEC>(biases + in);
            if (allowed) live[k] = allowed[in / 32] >> (in % 32);
        }
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int in = (k * THREADS + threadIdx.x) * VEC;
        if (in + VEC <= width) {
            live[k] &= ~banned(bias[k]);
            if (plain) {
                if (COUNT) live[k] &= ~(count[in / 32] >> (in % 32));
                store_pack(out + in, shaped_plainly<S, VEC, BACK>(BACK ? g[k] : z[k], bias[k], live[k]));
            } else {
                uint32_t c[VEC];
                __builtin_memcpy(c, __builtin_assume_aligned(count + in, 16), sizeof(c));
                store_pack(out + in, shaped<S, VEC, BACK>(z[k], g[k], c, pen, bias[k], live[k]));
            }
        } else {
            for (int i = in; i < width; ++i) {
                Pack<float, 1> bias1 = {};
                if (biases) bias1 = load_pack<1>(biases + i);
                uint32_t live1 = (allowed ? allowed[i / 32] >> (i % 32) : 1u) & ~banned(bias1);
                Pack<S, 1> z1 = load_pack<1>(zrow + i), g1 = {};
                if (BACK) g1 = load_pack<1>(grow + i);
                if (plain) {
                    if (COUNT) live1 &= ~(count[i / 32] >> (i % 32));
                    store_pack(out + i, shaped_plainly<S, 1, BACK>(BACK ? g1 : z1, bias1, live1));
                } else {
                    const uint32_t c[1] = {count[i]};
                    store_pack(out + i, shaped<S, 1, BACK>(z1, g1, c, pen, bias1, live1));
                }
            }
        }
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
        if (a.V < VEC) hipLaunchKernelGGL((short_kernel<S, 1, 1, BACK, COUNT>), grid, dim3(kThreads), 0, s, a);
        else if (a.V <= 64 * VEC) hipLaunchKernelGGL((short_kernel<S, VEC, 1, BACK, COUNT>), grid, dim3(kThreads), 0, s, a);
        else if (a.V <= 128 * VEC) hipLaunchKernelGGL((short_kernel<S, VEC, 2, BACK, COUNT>), grid, dim3(kThreads), 0, s, a);
        else if (a.V <= 256 * VEC) hipLaunchKernelGGL((short_kernel<S, VEC, 4, BACK, COUNT>), grid, dim3(kThreads), 0, s, a);
        else if constexpr (VEC == 4) hipLaunchKernelGGL((short_kernel<S, VEC, 8, BACK, COUNT>), grid, dim3(kThreads), 0, s, a);
    } else {
        // Longer stretches go through the history less often, and are more for one workgroup to wait for: 128 rows of 131072 with 4096 entries
        // 22.3 us with 256 threads, 21.6 with 512, 24 to 28 with 1024.
        const int threads = COUNT && a.V > 16384 ? 512 : 256;
        a.per_row = (a.V + kEach * threads - 1) / (kEach * threads);
        a.units = B * a.T * a.per_row;
        if (threads == 512) {
            if constexpr (COUNT) hipLaunchKernelGGL((long_kernel<S, 512, BACK, COUNT>), grid_of(a.units), dim3(512), 0, s, a);
        } else {
            hipLaunchKernelGGL((long_kernel<S, 256, BACK, COUNT>), grid_of(a.units), dim3(256), 0, s, a);
        }
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
