// Embedding lookup with scaling and its gradient (cc.h: cc_embed, cc_embed_backward).
//
//   out[i] = scale * table[ids[i]],     grad_table[v] = scale * (sum of grad[i] over the i with ids[i] = v)
//
// An id outside [0, V) is no token: its output row is zero and its gradient goes nowhere.
//
// The lookup moves bytes and nothing else.  The gradient is a sum over rows scattered in no order; adding them with atomics
// would add them in another order on every call.  Tokens are sorted by id instead, stably, so that equal ids keep their order (few
// by counting for each how many come before it, many by a counting sort).  The sorted list is cut into segments of equal length,
// and each segment is summed by lanes that lie along a row: frequent tokens are then shared by many segments and rare ones
// share one, so no distribution of ids leaves a workgroup with more to do than the others.  Within a segment an id's rows are added in
// the order of i.  A run of one id that crosses a border leaves a partial sum on each side of it; a last kernel adds those, every
// so many of them by a group of lanes and then the groups.  The order of additions depends on sizes and ids alone.
//
// Rows of ids that do not occur are zero.  All rows are cleared by additional workgroups of the kernels that sort: these wait for
// memory and leave its bandwidth unused, and to find the absent rows first took longer than to write the others twice.
#include <hip/hip_runtime.h>

#include "cc_internal.h"
#include "cc_model.h"

namespace cc {
namespace {

using namespace ccm;

constexpr int kThreads = 256;

// ---------------------------------------------------------------------------------------------------------- lookup

// Bound by memory: 65536 x 1024 bf16 out of 50001 rows 39 us, 6.0 TB/s of what it reads per token and writes.  A workgroup takes
// `rows` tokens; its threads take vectors of their rows in turn, U of them at once.  A vector that would end beyond
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

// A table that is cleared, in elements of two bytes: rows of `length`, `stride` apart, cut into units of about 64 KB: `rows` rows
// each or, of longer rows, one of `pieces` pieces.  A kernel's workgroups from `own` on clear the units from `first` on.
constexpr int kClearUnit = 1 << 15;
struct Clear {
    uint16_t* out;
    int64_t count, length, stride;
    int64_t rows, pieces, units, first, last;
    int64_t own;
    // Returns whether the workgroup was one of those that clear.
    __device__ __forceinline__ bool operator()() const {
        if ((int64_t)blockIdx.x < own) return false;
        for (int64_t u = first + ((int64_t)blockIdx.x - own); u < last; u += (int64_t)gridDim.x - own) {
            const int64_t row = pieces > 1 ? u / pieces : u * rows, at = pieces > 1 ? (u - row * pieces) * kClearUnit : 0;
            const int here = (int)min(rows, count - row), n = (int)min((int64_t)kClearUnit, length - at), vecs = (n + 7) / 8;
            for (int j = threadIdx.x; j < here * vecs; j += blockDim.x) {
                const int r = j / vecs, i = (j - r * vecs) * 8;
                uint16_t* const p = out + (row + r) * stride + at + i;
                const Pack<uint16_t, 8, false> zero = {};
                if (i + 8 <= n) __builtin_memcpy(p, &zero, sizeof(zero));
                else
                    for (int k = 0; k < n - i; ++k) p[k] = 0;
            }
        }
        return true;
    }
};
Clear clear_plan(void* out, int64_t count, int64_t length, int64_t stride) {
    Clear c = {};
    c.out = (uint16_t*)out;
    if (stride == length) {                           // one long row
        length *= count;
        count = 1;
    }
    c.count = count;
    c.length = length;
    c.stride = stride;
    c.rows = length < kClearUnit ? kClearUnit / length : 1;
    c.pieces = (length + kClearUnit - 1) / kClearUnit;
    c.units = c.pieces > 1 ? count * c.pieces : (count + c.rows - 1) / c.rows;
    return c;
}
// Share `part` of `parts` of what is to be cleared, in a launch with `own` other workgroups; returns how many workgroups that makes.
unsigned share(Clear& c, int part, int parts, int64_t own) {
    c.own = own;
    c.first = c.units * part / parts;
    c.last = c.units * (part + 1) / parts;
    const int64_t blocks = c.last - c.first;
    return (unsigned)(own + (blocks < 16384 ? blocks : 16384));
}

__device__ __forceinline__ uint32_t key_of(int32_t id, uint32_t V) { return (uint32_t)id < V ? (uint32_t)id : V; }

// Few tokens: a token's place is the number of smaller keys and of equal ones before it.  A workgroup has all keys in LDS and takes
// kRankTokens tokens; its groups of that many lanes look at keys in turn, the same four for all lanes of a group.  One launch
// instead of three or six (3000 tokens: 6 us, sorted in two passes 21; 12000: 17 against 24; sorted in one pass, 8192 and
// more tokens take 12).
constexpr int kRankMost = 12288, kRankMostOnePass = 8192, kRankTokens = 16, kRankThreads = 1024;
__global__ __launch_bounds__(kRankThreads) void rank_kernel(const int32_t* __restrict__ ids, int n, uint32_t V, int32_t* __restrict__ keys_out,
                                                            int32_t* __restrict__ pos_out, Clear clear) {
    constexpr int WAVES = kRankThreads / 64, GROUPS = kRankThreads / kRankTokens;
    __shared__ uint4 quads[kRankMost / 4];
    __shared__ uint32_t counts[WAVES][kRankTokens];
    if (clear()) return;
    uint32_t* const keys = (uint32_t*)quads;
    const int blocks = (n + kRankTokens - 1) / kRankTokens, block = blockIdx.x;
    for (int i = threadIdx.x; i < blocks * kRankTokens; i += kRankThreads) keys[i] = i < n ? key_of(ids[i], V) : ~0u;
    __syncthreads();
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, member = lane % kRankTokens, token = block * kRankTokens + member;
    const uint32_t key = keys[token];
    uint32_t count = 0;
    for (int b = threadIdx.x / kRankTokens; b < blocks; b += GROUPS) {
        const uint32_t bound = key + (b < block ? 1u : 0u);
#pragma unroll
        for (int q = 0; q < kRankTokens / 4; ++q) {
            const uint4 k = quads[b * (kRankTokens / 4) + q];
            count += (k.x < bound ? 1u : 0u) + (k.y < bound ? 1u : 0u) + (k.z < bound ? 1u : 0u) + (k.w < bound ? 1u : 0u);
        }
    }
    if (threadIdx.x < kRankTokens)                    // equal ones among the workgroup's own
        for (int e = 0; e < member; ++e) count += keys[block * kRankTokens + e] == key ? 1u : 0u;
    count += __shfl_xor(count, 16, 64);
    count += __shfl_xor(count, 32, 64);
    if (lane < kRankTokens) counts[wave][lane] = count;
    __syncthreads();
    if (threadIdx.x >= kRankTokens || token >= n) return;
    uint32_t at = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) at += counts[w][member];
    keys_out[at] = (int32_t)key;
    pos_out[at] = token;
}

// One pass of a stable counting sort by `bits` bits from `shift` up.  Tiles of kTile tokens, kSortWaves wavefronts each,
// a wavefront's tokens consecutive.  Short tiles: what a tile takes is a chain of ballots and LDS words per 64 tokens, and a list
// is cut into as many tiles as there are compute units soon enough.
constexpr int kTile = 1024, kSortWaves = 4, kSortThreads = kSortWaves * 64, kPerThread = kTile / kSortThreads;
constexpr int kMaxBits = 11;
constexpr int64_t kColumnsMost = 64, kColumnWordsMost = 16384;    // tiles, tiles times digits: see sort_place_kernel

// hist[tile][digit]: how many tokens of the tile have the digit
__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(const int32_t* __restrict__ ids, int64_t n, uint32_t V, int shift,
                                                                  int bits, uint32_t* __restrict__ hist, Clear clear) {
    __shared__ uint32_t bins[1 << kMaxBits];
    if (clear()) return;
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
                                                                   uint32_t* __restrict__ totals, Clear clear) {
    __shared__ uint32_t sums[kParts][64];
    if (clear()) return;
    const int lane = threadIdx.x & 63, part = threadIdx.x >> 6;
    const uint32_t d = blockIdx.x * 64 + lane;
    const bool real = d < (1u << bits);
    const int64_t each = (tiles + kParts - 1) / kParts, from = min(tiles, part * each), to = min(tiles, from + each);
    uint32_t sum = 0;
    if (real) {
#pragma unroll 8
        for (int64_t t = from; t < to; ++t) sum += hist[(t << bits) + d];
    }
    sums[part][lane] = sum;
    __syncthreads();
    uint32_t before = 0;
    for (int p = 0; p < part; ++p) before += sums[p][lane];
    if (!real) return;
    if (part == kParts - 1) totals[d] = before + sum;
#pragma unroll 8
    for (int64_t t = from; t < to; ++t) {
        const uint32_t c = hist[(t << bits) + d];
        hist[(t << bits) + d] = before;
        before += c;
    }
}

// Places each token behind the tokens of smaller digits, of its digit in earlier tiles, earlier wavefronts of its tile and
// earlier lanes.  keys_in == ids of the call where pos_in is null (a token's position is then its index).  COLUMNS: every workgroup adds
// the counts of all tiles itself, without sort_columns_kernel, where these are few.  What that takes grows with tiles times
// digits.  The whole gradient in us, with COLUMNS and without, by digits (twice as many passes for 256 of 50001 rows):
//   256:  16 tiles 34.1, 38.6    64 tiles 45.6, 48.9    111 tiles 59.5, 62.6    128 tiles 61.3, 60.0
//   512:  16 tiles 19.1, 20.6    31 tiles 20.1, 20.8     47 tiles 23.5, 23.2     64 tiles 24.7, 23.9
//   1024: 13 tiles 23.7, 24.1    16 tiles 23.7, 23.6     20 tiles 25.6, 23.7     64 tiles 31.2, 26.1
//   2048:  9 tiles 30.5, 28.1    64 tiles 43.4, 29.3
template <bool COLUMNS>
__global__ __launch_bounds__(kSortThreads) void sort_place_kernel(const int32_t* __restrict__ keys_in, const int32_t* __restrict__ pos_in,
                                                                  int64_t n, uint32_t V, int shift, int bits,
                                                                  const uint32_t* __restrict__ hist, const uint32_t* __restrict__ totals,
                                                                  int32_t* __restrict__ keys_out, int32_t* __restrict__ pos_out, Clear clear) {
    extern __shared__ uint32_t lds[];                 // [kSortWaves][digits] counts, then where each wavefront's tokens go
    __shared__ uint32_t wave_total[kSortWaves];
    if (clear()) return;
    const int digits = 1 << bits;
    const uint32_t mask = (uint32_t)digits - 1u;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t* const mine = lds + wave * digits;
    for (int d = threadIdx.x; d < kSortWaves * digits; d += kSortThreads) lds[d] = 0;
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * kTile + wave * (64 * kPerThread);
    uint32_t key[kPerThread], rank[kPerThread];
#pragma unroll
    for (int k = 0; k < kPerThread; ++k) {
        const int64_t i = first + k * 64 + lane;
        key[k] = i < n ? key_of(keys_in[i], V) : ~0u;
    }
    // each thread's stretch of digits: counts of all tiles and of the earlier ones, on their way while tokens are ranked
    constexpr int STRETCH = (1 << kMaxBits) / kSortThreads;
    const int stretch = (digits + kSortThreads - 1) / kSortThreads;
    uint32_t all[STRETCH], earlier_tiles[STRETCH];
    uint32_t* const column = lds + kSortWaves * digits;                  // COLUMNS: [digits] of all tiles, [digits] of the earlier ones
    if (COLUMNS) {
        const int tiles = (int)clear.own;
        for (int d = threadIdx.x; d < digits; d += kSortThreads) {
            uint32_t sum = 0, before = 0;
            // 16 at a time, the last of them too: one after the other, they would be waited for one by one
            for (int t0 = 0; t0 < tiles; t0 += 16) {
                uint32_t c[16];
#pragma unroll
                for (int u = 0; u < 16; ++u) c[u] = hist[((int64_t)min(t0 + u, tiles - 1) << bits) + d];
#pragma unroll
                for (int u = 0; u < 16; ++u) {
                    before += t0 + u < (int)blockIdx.x ? c[u] : 0u;
                    sum += t0 + u < tiles ? c[u] : 0u;
                }
            }
            column[d] = sum;
            column[digits + d] = before;
        }
    } else {
#pragma unroll
        for (int q = 0; q < STRETCH; ++q) {
            const int d = threadIdx.x * stretch + q;
            const bool real = q < stretch && d < digits;
            all[q] = real ? totals[d] : 0u;
            earlier_tiles[q] = real ? hist[((int64_t)blockIdx.x << bits) + d] : 0u;
        }
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
    if (COLUMNS) {
#pragma unroll
        for (int q = 0; q < STRETCH; ++q) {
            const int d = threadIdx.x * stretch + q;
            const bool real = q < stretch && d < digits;
            all[q] = real ? column[d] : 0u;
            earlier_tiles[q] = real ? column[digits + d] : 0u;
        }
    }
    // tokens of smaller digits: stretches are summed, then lanes and wavefronts are chained
    uint32_t sum = 0;
#pragma unroll
    for (int q = 0; q < STRETCH; ++q) sum += all[q];
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
#pragma unroll
    for (int q = 0; q < STRETCH; ++q) {
        const int d = threadIdx.x * stretch + q;
        if (q >= stretch || d >= digits) break;
        uint32_t at = base + earlier_tiles[q];
        base += all[q];
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

// The sums, bound by the latency of rows in no order (65536 x 1024 bf16, 2048 segments: 50 us, 3.6 TB/s; the next 8 rows on their
// way while 8 are summed took registers from other wavefronts: 52).  G lanes along a row (and blockIdx.y where a row is longer), a
// segment each.  keys and pos: sorted, with 8 more than n that may be read.
template <class S, class GT, int VEC, int G>
__global__ __launch_bounds__(kThreads) void embed_sums_kernel(const S* __restrict__ grad, const int32_t* __restrict__ keys,
                                                              const int32_t* __restrict__ pos, GT* __restrict__ out, SumArgs a) {
    constexpr int U = 8;
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
        // beyond the segment's end its first row stands in; the row of what is no token is loaded from its place and summed like others,
        // and the sum dropped
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

// Runs that cross borders: the partial sums of the segments that a run reaches are added up where it begins.  A workgroup looks at the
// ends of GROUPS segments, a wavefront each, and then adds for the runs it found: LANES lanes along a row, and GROUPS groups of them
// that take every GROUPS-th partial sum and are added up in their order.  (128000 x 250 over 1001 ids: 5.7 us, 8.0 us with a
// workgroup a segment and one group.)
constexpr int kJoinThreads = 512;
template <class GT, int VEC, int LANES>
__global__ __launch_bounds__(kJoinThreads) void embed_join_kernel(const int32_t* __restrict__ keys, GT* __restrict__ out, SumArgs a) {
    constexpr int GROUPS = kJoinThreads / LANES;
    __shared__ float sums[GROUPS > 1 ? kJoinThreads * VEC : 1];
    __shared__ int2 found[GROUPS];                    // {key, last segment} of the run that begins in a segment and goes on; key -1: none
    const int group = threadIdx.x / LANES, member = threadIdx.x % LANES, lane = threadIdx.x & 63;
    const int64_t seg0 = (int64_t)blockIdx.x * GROUPS;
    if ((int)(threadIdx.x >> 6) < GROUPS) {
        const int64_t seg = seg0 + (threadIdx.x >> 6);
        int2 run = {-1, 0};
        if (seg + 1 < a.segments) {
            const int64_t from = seg * a.segment, to = from + a.segment;
            const int key = keys[to - 1], after = keys[to], first = keys[from], before = from > 0 ? keys[from - 1] : -1;
            // it is a token, does not end here and did not begin earlier
            if (key < a.V && after == key && !(first == key && before == key)) {
                // The last segment whose first key is the run's: 64 looked at together, then every 64th and the 64 behind the last of these
                // (there are 4096 segments at most).
                const auto same_from = [&](int64_t s0, int64_t step) {
                    const int64_t s = s0 + lane * step;
                    const unsigned long long other = __ballot(!(s < a.segments && keys[s * a.segment] == key));
                    return other ? __ffsll((long long)other) - 1 : 64;
                };
                int64_t last = seg + same_from(seg + 1, 1);
                if (last == seg + 64) {
                    last += 64 * (int64_t)same_from(last + 64, 64);
                    last += same_from(last + 1, 1);
                }
                run = make_int2(key, (int)last);
            }
        }
        if (lane == 0) found[threadIdx.x >> 6] = run;
    }
    __syncthreads();
    for (int f = 0; f < GROUPS; ++f) {
        const int key = found[f].x;
        const int64_t seg = seg0 + f, last = found[f].y;
        if (key < 0) continue;
        for (int want = member * VEC; want - member * VEC < a.D; want += LANES * VEC) {
            const Part<VEC> part(want, a.D);
            float acc[VEC];
#pragma unroll
            for (int k = 0; k < VEC; ++k) acc[k] = 0.0f;
            if (part.real) {
#pragma unroll 8
                for (int64_t s = seg + group; s <= last; s += GROUPS) {
                    const Pack<float, VEC> p = load_pack<VEC>(a.partial + (s * 2 + (s == seg ? 1 : 0)) * a.D + part.at);
#pragma unroll
                    for (int k = 0; k < VEC; ++k) acc[k] += p.get(k);
                }
            }
            if (GROUPS > 1) {
#pragma unroll
                for (int k = 0; k < VEC; ++k) sums[threadIdx.x * VEC + k] = acc[k];
                __syncthreads();
                if (group == 0) {
#pragma unroll
                    for (int g = 1; g < GROUPS; ++g)
#pragma unroll
                        for (int k = 0; k < VEC; ++k) acc[k] += sums[(g * LANES + member) * VEC + k];
                }
                __syncthreads();
            }
            if (group == 0 && part.real) write_row(out + (int64_t)key * a.out_stride, part, acc, a.scale, a.accumulate != 0);
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
    const unsigned columns = (unsigned)((a.D + G * VEC - 1) / (G * VEC));
    if (a.segments > 0)
        hipLaunchKernelGGL((embed_sums_kernel<S, GT, VEC, G>), dim3((unsigned)((a.segments + per_block - 1) / per_block), columns), dim3(kThreads),
                           0, s, grad, keys, pos, out, a);
}

template <class GT, int VEC, int LANES>
void launch_join(const int32_t* keys, GT* out, const SumArgs& a, hipStream_t s) {
    constexpr int groups = kJoinThreads / LANES;
    hipLaunchKernelGGL((embed_join_kernel<GT, VEC, LANES>), dim3((unsigned)((a.segments - 1 + groups - 1) / groups)), dim3(kJoinThreads), 0, s, keys, out, a);
}

template <class S, class GT>
hipError_t backward(const EmbedCall& c, hipStream_t s) {
    const Layout l = layout(c.V, c.D, c.n);
    char* const base = (char*)c.workspace;
    int32_t* keys[2] = {(int32_t*)(base + l.keys[0]), (int32_t*)(base + l.keys[1])};
    int32_t* pos[2] = {(int32_t*)(base + l.pos[0]), (int32_t*)(base + l.pos[1])};
    uint32_t *hist = (uint32_t*)(base + l.hist), *totals = (uint32_t*)(base + l.totals);
    const int64_t unit = c.grad_dtype == kF32 ? 2 : 1;
    Clear clear = clear_plan(c.grad_table, c.V, c.D * unit, c.table_stride * unit);
    if (c.accumulate) clear.units = 0;
    int sorted_in = 0;
    if (c.n <= (l.passes > 1 ? kRankMost : kRankMostOnePass)) {
        const unsigned blocks = share(clear, 0, 1, (c.n + kRankTokens - 1) / kRankTokens);
        if (blocks > 0)
            hipLaunchKernelGGL(rank_kernel, dim3(blocks), dim3(kRankThreads), 0, s, c.ids, (int)c.n, (uint32_t)c.V, keys[0], pos[0], clear);
    } else {
        const bool columns = l.tiles <= kColumnsMost && l.tiles << l.bits <= kColumnWordsMost;
        const int digits = 1 << l.bits, each = columns ? 2 : 3, launches = each * l.passes;
        const size_t lds = sizeof(uint32_t) * (size_t)(kSortWaves + (columns ? 2 : 0)) * digits;   // 32 KB for 2048 of them; with columns 24 KB for 1024
        const auto place = columns ? sort_place_kernel<true> : sort_place_kernel<false>;
        for (int p = 0; p < l.passes; ++p) {
            const int32_t* in = p == 0 ? c.ids : keys[(p + 1) & 1];
            const int32_t* pin = p == 0 ? nullptr : pos[(p + 1) & 1];
            const int shift = p * l.bits;
            unsigned blocks = share(clear, each * p, launches, l.tiles);
            hipLaunchKernelGGL(sort_count_kernel, dim3(blocks), dim3(kSortThreads), 0, s, in, c.n, (uint32_t)c.V, shift, l.bits, hist, clear);
            if (!columns) {
                blocks = share(clear, each * p + 1, launches, (digits + 63) / 64);
                hipLaunchKernelGGL(sort_columns_kernel, dim3(blocks), dim3(64 * kParts), 0, s, hist, l.tiles, l.bits, totals, clear);
            }
            blocks = share(clear, each * p + each - 1, launches, l.tiles);
            hipLaunchKernelGGL(place, dim3(blocks), dim3(kSortThreads), lds, s, in, pin, c.n, (uint32_t)c.V, shift, l.bits, hist,
                               totals, keys[p & 1], pos[p & 1], clear);
        }
        sorted_in = (l.passes + 1) & 1;
    }
    const int32_t *sorted = keys[sorted_in], *places = pos[sorted_in];
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
        if (c.D < 4) launch_join<GT, 1, 64>(sorted, out, a, s);
        else if (c.D <= 256) launch_join<GT, 4, 64>(sorted, out, a, s);
        else if (c.D <= 512) launch_join<GT, 4, 128>(sorted, out, a, s);
        else if (c.D <= 1024) launch_join<GT, 4, 256>(sorted, out, a, s);
        else launch_join<GT, 4, 512>(sorted, out, a, s);
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
