// Embedding lookup with scaling and its gradient (cc.h: cc_embed, cc_embed_backward).
//
//   out[i] = scale * table[ids[i]],     grad_table[v] = scale * (sum of grad[i] over the i with ids[i] = v, in order of i)
//
// An id outside [0, V) is no token: its output row is zero and its gradient goes nowhere.
//
// The lookup moves bytes and nothing else.  The gradient is a sum over rows scattered in no order; adding them with atomics
// would add them in another order on every call.  Tokens are sorted by id instead (a stable counting sort, so equal ids keep
// their order), the sorted list is cut into segments of equal length, and each segment is summed by lanes that lie along
// a row: frequent tokens are then shared by many segments and rare ones share one, so no distribution of ids leaves a
// workgroup with more to do than the others.  A run of one id that crosses a border leaves a partial sum on each side of it;
// a last kernel adds those in order.  The order of additions depends on sizes and ids alone.
#include <hip/hip_runtime.h>

#include "cc_internal.h"
#include "cc_model.h"

namespace cc {
namespace {

using namespace ccm;

constexpr int kThreads = 256;

// ---------------------------------------------------------------------------------------------------------- lookup

// A workgroup takes `rows` tokens; its threads take vectors of their rows in turn, U of them at once.  A vector that would end beyond
// its row is moved back to end with it and repeats what the one before it writes, so that every thread loads and stores a whole one.
template <class S, int VEC>
__global__ __launch_bounds__(kThreads) void embed_kernel(const S* __restrict__ table, int V, int D, int64_t table_stride,
                                                         const int32_t* __restrict__ ids, int64_t n, float scale,
                                                         S* __restrict__ out, int64_t out_stride, int rows) {
    constexpr int U = 4;
    const uint32_t per_row = (uint32_t)(D + VEC - 1) / VEC;
    const int64_t first = (int64_t)blockIdx.x * rows;
    const int have = (int)min((int64_t)rows, n - first);
    const uint32_t count = (uint32_t)have * per_row;
    for (uint32_t i0 = threadIdx.x; i0 < count; i0 += U * kThreads) {
        uint32_t row[U];
        int at[U], id[U];
        Pack<S, VEC> p[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t i = min(i0 + u * kThreads, count - 1);
            row[u] = i / per_row;
            at[u] = min((int)(i - row[u] * per_row) * VEC, D - VEC);
            id[u] = ids[first + row[u]];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if ((uint32_t)id[u] < (uint32_t)V) p[u] = load_pack<VEC>(table + (int64_t)id[u] * table_stride + at[u]);
            else p[u] = Pack<S, VEC>();
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (i0 + u * kThreads >= count) break;
            float f[VEC];
#pragma unroll
            for (int k = 0; k < VEC; ++k) f[k] = (uint32_t)id[u] < (uint32_t)V ? p[u].get(k) * scale : 0.0f;
            store_pack(out + (first + row[u]) * out_stride + at[u], Pack<S, VEC>::from(f));
        }
    }
}

// ------------------------------------------------------------------------------------------------------------ sort

// One pass of a stable counting sort by `bits` bits from `shift` up.  Tiles of kTile tokens, kSortWaves wavefronts each,
// a wavefront's tokens consecutive.  Short tiles: what a tile takes is a chain of ballots and LDS words per 64 tokens, and a list
// is cut into as many tiles as there are compute units soon enough.
constexpr int kTile = 1024, kSortWaves = 4, kSortThreads = kSortWaves * 64, kPerThread = kTile / kSortThreads;
constexpr int kMaxBits = 11;

__device__ __forceinline__ uint32_t key_of(int32_t id, uint32_t V) { return (uint32_t)id < V ? (uint32_t)id : V; }

// hist[tile][digit]: how many tokens of the tile have the digit
__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(const int32_t* __restrict__ ids, int64_t n, uint32_t V, int shift,
                                                                  int bits, uint32_t* __restrict__ hist) {
    __shared__ uint32_t bins[1 << kMaxBits];
    const uint32_t mask = (1u << bits) - 1u;
    for (uint32_t d = threadIdx.x; d <= mask; d += kSortThreads) bins[d] = 0;
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * kTile;
#pragma unroll
    for (int k = 0; k < kPerThread; ++k) {
        const int64_t i = first + k * kSortThreads + threadIdx.x;
        if (i < n) atomicAdd(&bins[(key_of(ids[i], V) >> shift) & mask], 1u);
    }
    __syncthreads();
    for (uint32_t d = threadIdx.x; d <= mask; d += kSortThreads) hist[((int64_t)blockIdx.x << bits) + d] = bins[d];
}

// hist[tile][digit] becomes the number of tokens with the digit in earlier tiles, totals[digit] the number in all.
// 64 digits per workgroup, the tiles in kParts parts.
constexpr int kParts = 16;
__global__ __launch_bounds__(64 * kParts) void sort_columns_kernel(uint32_t* __restrict__ hist, int64_t tiles, int bits,
                                                                   uint32_t* __restrict__ totals) {
    __shared__ uint32_t sums[kParts][64];
    const int lane = threadIdx.x & 63, part = threadIdx.x >> 6;
    const uint32_t d = blockIdx.x * 64 + lane;
    const bool real = d < (1u << bits);
    const int64_t each = (tiles + kParts - 1) / kParts, from = min(tiles, part * each), to = min(tiles, from + each);
    uint32_t sum = 0;
    if (real)
        for (int64_t t = from; t < to; ++t) sum += hist[(t << bits) + d];
    sums[part][lane] = sum;
    __syncthreads();
    uint32_t before = 0;
    for (int p = 0; p < part; ++p) before += sums[p][lane];
    if (!real) return;
    if (part == kParts - 1) totals[d] = before + sum;
    for (int64_t t = from; t < to; ++t) {
        const uint32_t c = hist[(t << bits) + d];
        hist[(t << bits) + d] = before;
        before += c;
    }
}

// Places each token behind the tokens of smaller digits, of its digit in earlier tiles, earlier wavefronts of its tile and
// earlier lanes.  keys_in == ids of the call where pos_in is null (a token's position is then its index).  With one tile
// there is no hist and no totals: the tile's own counts are all there is.
template <bool ONE_TILE>
__global__ __launch_bounds__(kSortThreads) void sort_place_kernel(const int32_t* __restrict__ keys_in, const int32_t* __restrict__ pos_in,
                                                                  int64_t n, uint32_t V, int shift, int bits,
                                                                  const uint32_t* __restrict__ hist, const uint32_t* __restrict__ totals,
                                                                  int32_t* __restrict__ keys_out, int32_t* __restrict__ pos_out) {
    extern __shared__ uint32_t lds[];                 // [kSortWaves][digits] counts, then where each wavefront's tokens go; [digits] starts
    __shared__ uint32_t wave_total[kSortWaves];
    const int digits = 1 << bits;
    const uint32_t mask = (uint32_t)digits - 1u;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t* const mine = lds + wave * digits;
    uint32_t* const starts = lds + kSortWaves * digits;
    for (int d = threadIdx.x; d < kSortWaves * digits; d += kSortThreads) lds[d] = 0;
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * kTile + wave * (64 * kPerThread);
    uint32_t key[kPerThread], rank[kPerThread];
#pragma unroll
    for (int k = 0; k < kPerThread; ++k) {
        const int64_t i = first + k * 64 + lane;
        key[k] = i < n ? key_of(keys_in[i], V) : ~0u;
    }
#pragma unroll
    for (int k = 0; k < kPerThread; ++k) {
        const bool real = first + k * 64 + lane < n;
        const uint32_t d = (key[k] >> shift) & mask;
        unsigned long long same = __ballot(real);
        for (int b = 0; b < bits; ++b) {
            const unsigned long long ones = __ballot((d >> b) & 1u);
            same &= ((d >> b) & 1u) ? ones : ~ones;
        }
        const uint32_t earlier = __popcll(same & ((1ull << lane) - 1ull));
        // the wavefront's own counts: every lane reads before the first lane of each digit writes
        rank[k] = real ? mine[d] + earlier : 0u;
        wave_order();
        if (real && earlier == 0) mine[d] += __popcll(same);
        wave_order();
    }
    __syncthreads();
    // starts[d]: tokens of smaller digits (each thread sums a stretch of digits, then wavefronts and lanes are chained)
    const int stretch = (digits + kSortThreads - 1) / kSortThreads;
    uint32_t sum = 0;
    for (int q = 0; q < stretch; ++q) {
        const int d = threadIdx.x * stretch + q;
        if (d >= digits) break;
        uint32_t c = 0;
        if (ONE_TILE) {
            for (int w = 0; w < kSortWaves; ++w) c += lds[w * digits + d];
        } else {
            c = totals[d];
        }
        starts[d] = sum;
        sum += c;
    }
    uint32_t upto = sum;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        const uint32_t o = __shfl_up(upto, m, 64);
        if (lane >= m) upto += o;
    }
    if (lane == 63) wave_total[wave] = upto;
    __syncthreads();
    uint32_t base = upto - sum;
    for (int w = 0; w < wave; ++w) base += wave_total[w];
    for (int q = 0; q < stretch; ++q) {
        const int d = threadIdx.x * stretch + q;
        if (d >= digits) break;
        uint32_t at = starts[d] + base + (ONE_TILE ? 0u : hist[((int64_t)blockIdx.x << bits) + d]);
        for (int w = 0; w < kSortWaves; ++w) {
            const uint32_t c = lds[w * digits + d];
            lds[w * digits + d] = at;
            at += c;
        }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kPerThread; ++k) {
        const int64_t i = first + k * 64 + lane;
        if (i >= n) continue;
        const uint32_t at = mine[(key[k] >> shift) & mask] + rank[k];
        keys_out[at] = (int32_t)key[k];
        pos_out[at] = pos_in ? pos_in[i] : (int32_t)i;
    }
}

// ------------------------------------------------------------------------------------------------------------ sums

struct SumArgs {
    int64_t n;
    int V, D;
    int64_t grad_stride, out_stride;
    float scale;
    int accumulate;
    int segment;                  // sorted tokens per segment, a multiple of 8
    int64_t segments;
    float* partial;               // [segments][2][D]
    int64_t sum_blocks;           // workgroups that sum; those behind them clear the rows of absent ids
};

// A lane's vector of a row: where it starts, and from which element on it is the lane's own.  One that would end beyond the row is
// moved back to end with it; it is loaded as a whole and stored from its own elements on.
template <int VEC>
struct Part {
    int at, skip;
    bool real;
    __device__ __forceinline__ Part(int want, int D) : at(min(want, D - VEC)), skip(want - min(want, D - VEC)), real(want < D) {}
    template <class T>
    __device__ __forceinline__ void store(T* row, const Pack<T, VEC>& p) const {
        if (skip == 0) {
            store_pack(row + at, p);
            return;
        }
#pragma unroll
        for (int k = 0; k < VEC; ++k)
            if (k >= skip) row[at + k] = p.element(k);
    }
};

template <int VEC, class GT>
__device__ __forceinline__ void write_row(GT* row, const Part<VEC>& part, const float* acc, float scale, bool accumulate) {
    float f[VEC];
#pragma unroll
    for (int k = 0; k < VEC; ++k) f[k] = scale * acc[k];
    if (accumulate) {
        const Pack<GT, VEC> old = load_pack<VEC>(row + part.at);
#pragma unroll
        for (int k = 0; k < VEC; ++k) f[k] = old.get(k) + scale * acc[k];
    }
    part.store(row, Pack<GT, VEC>::from(f));
}

// First index from `lo` on whose key is at least v.
__device__ __forceinline__ int64_t lower_bound(const int32_t* keys, int64_t lo, int64_t hi, int v) {
    while (lo < hi) {
        const int64_t mid = (lo + hi) >> 1;
        if (keys[mid] < v) lo = mid + 1; else hi = mid;
    }
    return lo;
}

// Where the ids are looked for by many, a workgroup keeps every step-th key of the sorted list: most of a search is then in LDS.
constexpr int kSamples = 1024;

// The sums: G lanes along a row (and blockIdx.y where a row is longer), a segment each.  keys and pos: sorted, with 8 more than n that
// may be read.
template <class S, class GT, int VEC, int G>
__global__ __launch_bounds__(kThreads) void embed_sums_kernel(const S* __restrict__ grad, const int32_t* __restrict__ keys,
                                                              const int32_t* __restrict__ pos, GT* __restrict__ out, SumArgs a) {
    constexpr int U = 8;
    if ((int64_t)blockIdx.x >= a.sum_blocks) {
        // Rows of ids that do not occur: 64 of them a workgroup, a lane looks for one of them, then the wavefronts clear them in turn.
        __shared__ int32_t samples[kSamples];
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        const int64_t every = (a.n + kSamples - 1) / kSamples;
        const int count = every > 0 ? (int)((a.n + every - 1) / every) : 0;
        for (int i = threadIdx.x; i < count; i += kThreads) samples[i] = keys[i * every];
        __syncthreads();
        const int64_t step = ((int64_t)gridDim.x - a.sum_blocks) * 64;
        for (int64_t v0 = ((int64_t)blockIdx.x - a.sum_blocks) * 64; v0 < a.V; v0 += step) {
            const int64_t v = v0 + lane;
            bool absent = false;
            if (v < a.V) {
                // the first sample that is not smaller; the key itself is not before the sample before it
                const int64_t s = lower_bound(samples, 0, count, (int)v);
                const int64_t i = lower_bound(keys, s > 0 ? (s - 1) * every + 1 : 0, min(a.n, s * every), (int)v);
                absent = i >= a.n || keys[i] != (int)v;
            }
            unsigned long long rows = __ballot(absent);
            const float zero[VEC] = {};
            for (int k = 0; rows != 0; ++k) {
                const int r = __ffsll((long long)rows) - 1;
                rows &= rows - 1;
                if ((k & (kThreads / 64 - 1)) != wave) continue;
                GT* const row = out + (v0 + r) * a.out_stride;
                for (int want = lane * VEC; want < a.D; want += 64 * VEC) write_row(row, Part<VEC>(want, a.D), zero, 0.0f, false);
            }
        }
        return;
    }
    int group = threadIdx.x / G;
    if (G >= 64) group = __builtin_amdgcn_readfirstlane(group);       // a segment's list is then read by scalar loads
    const Part<VEC> part((blockIdx.y * G + threadIdx.x % G) * VEC, a.D);
    const int64_t seg = (int64_t)blockIdx.x * (kThreads / G) + group;
    if (seg >= a.segments || !part.real) return;
    const int64_t from = seg * a.segment, to = min(a.n, from + a.segment);
    const int before = from > 0 ? keys[from - 1] : -1, after = to < a.n ? keys[to] : -1;
    int current = keys[from];
    bool open = current == before;                    // the run began in an earlier segment
    float* const slot = a.partial + seg * 2 * a.D;
    float acc[VEC];
#pragma unroll
    for (int k = 0; k < VEC; ++k) acc[k] = 0.0f;
    const auto flush = [&](bool goes_on) {
        if (current >= a.V) return;                   // no token
        if (open || goes_on) part.store(open ? slot : slot + a.D, Pack<float, VEC>::from(acc));
        else write_row(out + (int64_t)current * a.out_stride, part, acc, a.scale, a.accumulate != 0);
    };
    for (int64_t i = from; i < to; i += U) {
        int key[U];
        Pack<S, VEC> row[U];
#pragma unroll
        for (int u = 0; u < U; ++u) key[u] = keys[i + u];
        // beyond the segment's end, and for what is no token, the segment's first row stands in
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int p = i + u < to ? pos[i + u] : pos[from];
            row[u] = load_pack<VEC>(grad + (int64_t)p * a.grad_stride + part.at);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (i + u >= to) break;
            if (key[u] != current) {
                flush(false);
                current = key[u];
                open = false;
#pragma unroll
                for (int k = 0; k < VEC; ++k) acc[k] = 0.0f;
            }
#pragma unroll
            for (int k = 0; k < VEC; ++k) acc[k] += row[u].get(k);
        }
    }
    flush(current == after);
}

// Runs that cross borders: the segment in which a run begins adds the partial sums of the segments that it reaches.  How far it
// reaches is looked for in steps that double.
template <class GT, int VEC>
__global__ __launch_bounds__(kThreads) void embed_join_kernel(const int32_t* __restrict__ keys, GT* __restrict__ out, SumArgs a) {
    for (int64_t seg = blockIdx.x; seg + 1 < a.segments; seg += gridDim.x) {
        const int64_t from = seg * a.segment, to = from + a.segment;
        const int key = keys[to - 1];
        if (key >= a.V || keys[to] != key) continue;                                   // ends here
        if (keys[from] == key && from > 0 && keys[from - 1] == key) continue;          // began earlier
        // the last segment whose first key is the run's
        int64_t last = seg + 1, step = 1;
        while (last + step < a.segments && keys[(last + step) * a.segment] == key) {
            last += step;
            step *= 2;
        }
        for (; step > 0; step /= 2)
            if (last + step < a.segments && keys[(last + step) * a.segment] == key) last += step;
        for (int want = threadIdx.x * VEC; want < a.D; want += kThreads * VEC) {
            const Part<VEC> part(want, a.D);
            float acc[VEC];
            Pack<float, VEC> p = load_pack<VEC>(a.partial + (seg * 2 + 1) * a.D + part.at);
#pragma unroll
            for (int k = 0; k < VEC; ++k) acc[k] = p.get(k);
#pragma unroll 8
            for (int64_t s = seg + 1; s <= last; ++s) {
                p = load_pack<VEC>(a.partial + s * 2 * a.D + part.at);
#pragma unroll
                for (int k = 0; k < VEC; ++k) acc[k] += p.get(k);
            }
            write_row(out + (int64_t)key * a.out_stride, part, acc, a.scale, a.accumulate != 0);
        }
    }
}

size_t up256(size_t x) { return (x + 255u) & ~(size_t)255u; }

// Workspace of cc_embed_backward: two lists of keys and positions (each with room to be read 8 past its end), counts per
// tile and digit, totals per digit, partial sums.
struct Layout {
    int passes, bits;
    int64_t tiles, segments;
    int segment;
    size_t keys[2], pos[2], hist, totals, partial, total;
};
Layout layout(int64_t V, int64_t D, int64_t n) {
    Layout l;
    int all = 1;
    while ((V >> all) != 0) ++all;                    // keys are 0 .. V
    l.passes = (all + kMaxBits - 1) / kMaxBits;
    l.bits = (all + l.passes - 1) / l.passes;
    l.tiles = (n + kTile - 1) / kTile;
    // Short segments where tokens are few, so that there are some thousand wavefronts (2^21 elements of 8 a lane make 4096 of them); no
    // more than 4096 segments, which bounds what a run over all of them costs to join.
    int64_t s = (n + 4095) / 4096;
    const int64_t even = n * D >> 21;
    if (even > s) s = even;
    if (s < 8) s = 8;
    if (s > 1 << 20) s = 1 << 20;
    l.segment = (int)((s + 7) & ~(int64_t)7);
    l.segments = (n + l.segment - 1) / l.segment;
    size_t at = 0;
    const auto take = [&](size_t bytes) {
        const size_t here = at;
        at += up256(bytes);
        return here;
    };
    for (int i = 0; i < 2; ++i) {
        l.keys[i] = take(sizeof(int32_t) * (size_t)(n + 8));
        l.pos[i] = take(sizeof(int32_t) * (size_t)(n + 8));
    }
    l.hist = take(sizeof(uint32_t) * ((size_t)l.tiles << l.bits));
    l.totals = take(sizeof(uint32_t) << l.bits);
    l.partial = take(sizeof(float) * 2 * (size_t)l.segments * (size_t)D);
    l.total = at;
    return l;
}

template <class S, int VEC>
void launch_lookup(const EmbedCall& c, hipStream_t s) {
    const int64_t per_row = (c.D + VEC - 1) / VEC;
    // rows per workgroup: four vectors a thread, fewer where that leaves compute units without a workgroup
    int64_t rows = (4 * kThreads + per_row - 1) / per_row;
    while (rows > 1 && (c.n + rows - 1) / rows < 1024) rows = (rows + 1) / 2;
    hipLaunchKernelGGL((embed_kernel<S, VEC>), dim3((unsigned)((c.n + rows - 1) / rows)), dim3(kThreads), 0, s, (const S*)c.table, (int)c.V,
                       (int)c.D, c.table_stride, c.ids, c.n, c.scale, (S*)c.out, c.out_stride, (int)rows);
}

// Vectors of 16 bytes where a row has one.
template <class S>
hipError_t embed(const EmbedCall& c, hipStream_t s) {
    constexpr int VEC = 16 / sizeof(S);
    if (c.D >= VEC) launch_lookup<S, VEC>(c, s);
    else launch_lookup<S, 1>(c, s);
    return hipGetLastError();
}

template <class S, class GT, int VEC, int G>
void launch_sums(const S* grad, const int32_t* keys, const int32_t* pos, GT* out, SumArgs& a, hipStream_t s) {
    constexpr int per_block = kThreads / G;
    a.sum_blocks = (a.segments + per_block - 1) / per_block;
    int64_t clear = a.accumulate ? 0 : ((int64_t)a.V + 63) / 64;
    if (clear > 65536) clear = 65536;
    const unsigned columns = (unsigned)((a.D + G * VEC - 1) / (G * VEC));
    hipLaunchKernelGGL((embed_sums_kernel<S, GT, VEC, G>), dim3((unsigned)(a.sum_blocks + clear), columns), dim3(kThreads), 0, s, grad, keys,
                       pos, out, a);
}

template <class S, class GT>
hipError_t backward(const EmbedCall& c, hipStream_t s) {
    const Layout l = layout(c.V, c.D, c.n);
    char* const base = (char*)c.workspace;
    int32_t* keys[2] = {(int32_t*)(base + l.keys[0]), (int32_t*)(base + l.keys[1])};
    int32_t* pos[2] = {(int32_t*)(base + l.pos[0]), (int32_t*)(base + l.pos[1])};
    uint32_t *hist = (uint32_t*)(base + l.hist), *totals = (uint32_t*)(base + l.totals);
    const int digits = 1 << l.bits;                   // 40 KB of LDS for 2048 of them
    const size_t lds = sizeof(uint32_t) * (size_t)(kSortWaves + 1) * digits;
    const auto place = l.tiles <= 1 ? sort_place_kernel<true> : sort_place_kernel<false>;
    for (int p = 0; p < l.passes; ++p) {
        const int32_t* in = p == 0 ? c.ids : keys[(p + 1) & 1];
        const int32_t* pin = p == 0 ? nullptr : pos[(p + 1) & 1];
        const int shift = p * l.bits;
        if (l.tiles > 1) {
            hipLaunchKernelGGL(sort_count_kernel, dim3((unsigned)l.tiles), dim3(kSortThreads), 0, s, in, c.n, (uint32_t)c.V, shift, l.bits, hist);
            hipLaunchKernelGGL(sort_columns_kernel, dim3((unsigned)((digits + 63) / 64)), dim3(64 * kParts), 0, s, hist, l.tiles, l.bits, totals);
        }
        if (l.tiles > 0)
            hipLaunchKernelGGL(place, dim3((unsigned)l.tiles), dim3(kSortThreads), lds, s, in, pin, c.n, (uint32_t)c.V, shift, l.bits, hist,
                               totals, keys[p & 1], pos[p & 1]);
    }
    const int32_t *sorted = keys[(l.passes + 1) & 1], *places = pos[(l.passes + 1) & 1];
    SumArgs a;
    a.n = c.n;
    a.V = (int)c.V;
    a.D = (int)c.D;
    a.grad_stride = c.out_stride;
    a.out_stride = c.table_stride;
    a.scale = c.scale;
    a.accumulate = c.accumulate;
    a.segment = l.segment;
    a.segments = l.segments;
    a.partial = (float*)(base + l.partial);
    constexpr int VEC = 16 / sizeof(S);
    const int per_row = (int)((c.D + VEC - 1) / VEC);
    const S* grad = (const S*)c.out;
    GT* out = (GT*)c.grad_table;
    // lanes along a row: the power of two that covers it
    if (c.D < VEC) launch_sums<S, GT, 1, 8>(grad, sorted, places, out, a, s);
    else if (per_row <= 8) launch_sums<S, GT, VEC, 8>(grad, sorted, places, out, a, s);
    else if (per_row <= 16) launch_sums<S, GT, VEC, 16>(grad, sorted, places, out, a, s);
    else if (per_row <= 32) launch_sums<S, GT, VEC, 32>(grad, sorted, places, out, a, s);
    else if (per_row <= 64) launch_sums<S, GT, VEC, 64>(grad, sorted, places, out, a, s);
    else if (per_row <= 128) launch_sums<S, GT, VEC, 128>(grad, sorted, places, out, a, s);
    else launch_sums<S, GT, VEC, 256>(grad, sorted, places, out, a, s);
    if (l.segments > 1) {
        const unsigned blocks = (unsigned)(l.segments - 1 < 4096 ? l.segments - 1 : 4096);
        if (c.D < 4) hipLaunchKernelGGL((embed_join_kernel<GT, 1>), dim3(blocks), dim3(kThreads), 0, s, sorted, out, a);
        else hipLaunchKernelGGL((embed_join_kernel<GT, 4>), dim3(blocks), dim3(kThreads), 0, s, sorted, out, a);
    }
    return hipGetLastError();
}

}  // namespace

size_t embed_workspace_bytes(int64_t V, int64_t D, int64_t n) { return layout(V, D, n).total; }

hipError_t launch_embed(const EmbedCall& c, hipStream_t s) {
    if (c.dtype == kF32) return embed<float>(c, s);
    if (c.dtype == kF16) return embed<_Float16>(c, s);
    return embed<__bf16>(c, s);
}

hipError_t launch_embed_backward(const EmbedCall& c, hipStream_t s) {
    if (c.dtype == kF32) return backward<float, float>(c, s);
    if (c.dtype == kF16) return c.grad_dtype == kF32 ? backward<_Float16, float>(c, s) : backward<_Float16, _Float16>(c, s);
    return c.grad_dtype == kF32 ? backward<__bf16, float>(c, s) : backward<__bf16, __bf16>(c, s);
}

}  // namespace cc
