// Product of rows in 8 bits with a scale for each row and each channel (cc.h: cc_product_i8).
//
//   out[m, n] = x_scale[m] w_scale[n] (sum over k of x[m, k] w[n, k]) + bias[n]
//
// The sum is one of whole numbers in 32 bits: at most 131071 terms of at most 2^14, so it is exact and does not depend on
// how it is cut.  Terms beyond K are zeros that are put where a tile ends inside a row; nothing beyond a row is read.
//
// tile_kernel: a workgroup has a tile of the result and goes along K in steps of 128 bytes.  Both operands come to LDS in pieces of 16
// bytes, straight from memory where all rows begin at words of 4 bytes (4096 x 4096 x 4004: 73 us; x 4001, through registers, 88), through
// registers else.  In LDS a row has 8 such pieces, and piece c lies at place c ^ (row / 2 % 8): the lanes that read the same piece of 16 rows then use all 64 banks once.  Two to
// four tiles are held: while one is multiplied, others are on their way.
//
// few_kernel: up to 32 rows, where reading the weights is what takes time: they go from memory to registers, each once; several
// wavefronts share a channel's K where there are few channels.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "cc_internal.h"
#include "cc_model.h"

namespace cc {
namespace {

using namespace ccm;

typedef int Int4 __attribute__((ext_vector_type(4)));
typedef int Int16 __attribute__((ext_vector_type(16)));

constexpr int kPiece = 16;

struct Args {
    const int8_t *x, *w;
    const float *x_scale, *w_scale, *bias;
    int64_t M, x_stride, w_stride, out_stride;
    int N, K;
    void* out;
    int tiles_m, tiles_n;
    bool bytes;                          // some row does not begin at a word of 4 bytes
};

// 16 bytes from k on of a row of fewer; what lies beyond it is zero and not read.
__device__ __forceinline__ Int4 load_short(const int8_t* row, int k, int K) {
    typedef uint64_t Long2 __attribute__((ext_vector_type(2)));
    Long2 v = {0, 0};
    for (int i = 0; k + i < K; ++i) {
        const uint64_t byte = (uint8_t)row[k + i];
        if (i < 8) v[0] |= byte << (8 * i);
        else v[1] |= byte << (8 * (i - 8));
    }
    return __builtin_bit_cast(Int4, v);
}

// A load of 16 bytes that does not begin at a word takes far longer than one that does (8 x 50001 x 1001: 22 us, x 1004 12): such a piece is read as
// the five words that it lies in, and `by` bytes of the first are shifted out (15 us).  At a row's ends, where a word has bytes that are not the row's, the piece is read as it lies, by = 0.
struct Whole {
    Int4 v;
    __device__ __forceinline__ Int4 get() const { return v; }
};
struct Words {
    Int4 v;
    uint32_t next, by;
    __device__ __forceinline__ Int4 get() const {
        return Int4{(int)__builtin_amdgcn_alignbyte(v[1], v[0], by), (int)__builtin_amdgcn_alignbyte(v[2], v[1], by),
                    (int)__builtin_amdgcn_alignbyte(v[3], v[2], by), (int)__builtin_amdgcn_alignbyte(next, v[3], by)};
    }
};
__device__ __forceinline__ uint32_t beyond_word(const void* p) { return (uint32_t)(uintptr_t)p & 3u; }
// The piece at p, of which `by` bytes are shifted out: 0, or as many as p is beyond a word.  `more`: there is a fifth word to read.
__device__ __forceinline__ Words load_words(const int8_t* p, uint32_t by, bool more) {
    Words w;
    p -= by;
    __builtin_memcpy(&w.v, p, kPiece);
    __builtin_memcpy(&w.next, p + (more ? kPiece : kPiece - 4), 4);
    w.by = by;
    return w;
}
// Any piece of a row of at least 16, without a branch: what lies beyond the row is zero, and where a piece ends beyond it, its last 16 bytes are read and
// shifted.
template <class Part>
struct Clipped {
    Part part;
    int beyond;                          // bytes before the piece, which are shifted out as well
    __device__ __forceinline__ Int4 get() const {
        typedef uint64_t Long2 __attribute__((ext_vector_type(2)));
        Long2 v = __builtin_bit_cast(Long2, part.get());
        const int shift = (beyond & 7) * 8;
        if (beyond & 8) v = Long2{v[1], 0};
        v = Long2{v[0] >> shift | v[1] << 1 << (63 - shift), v[1] >> shift};
        if (beyond >= kPiece) v = Long2{0, 0};
        return __builtin_bit_cast(Int4, v);
    }
};
__device__ __forceinline__ Whole load_whole(const int8_t* p) {
    Whole v;
    __builtin_memcpy(&v.v, p, kPiece);
    return v;
}
__device__ __forceinline__ Clipped<Whole> load_clipped(const int8_t* row, int k, int K) {
    const int at = min(k, K - kPiece);
    return {load_whole(row + at), min(k - at, kPiece)};
}
__device__ __forceinline__ Clipped<Words> load_clipped_words(const int8_t* row, int k, int K) {
    const int at = min(k, K - kPiece);
    const uint32_t by = beyond_word(row + at);
    const bool inside = at >= (int)by && at - (int)by + kPiece + 4 <= K;
    return {load_words(row + at, inside ? by : 0, inside), min(k - at, kPiece)};
}

// From the exact sum on in 32 bits: it is rounded, and so is each product and the sum with the bias.  Beyond 2^96 of xs a power of two is left to
// the last product, so that the first is not infinite where the result is not (that product takes 1 % of 8192 x 8192 x 4096; a choice of the order by
// row 2 %, and so does a branch around it).
__device__ __forceinline__ float scaled(int sum, float xs, float ws, float bias) {
    const bool far = __builtin_fabsf(xs) > 0x1p96f;
    return (float)sum * (far ? xs * 0x1p-64f : xs) * ws * (far ? 0x1p64f : 1.0f) + bias;
}

// An address that all lanes have, in scalar registers.
__device__ __forceinline__ const int8_t* scalar(const int8_t* p) {
    const uint64_t v = (uint64_t)p;
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
    return (const int8_t*)((uint64_t)hi << 32 | lo);
}

template <class S>
struct Elements {
    S v[16 / sizeof(S)];
};

// A launch's first dimension holds fewer than 2^32 threads: tiles beyond kAcross go to the third.
constexpr uint32_t kAcross = 1 << 20;

// Workgroups of one XCD (every eighth) get neighbouring tiles, and those in blocks of 8 rows of tiles, so that what they read at the
// same time is shared in its L2.
__device__ __forceinline__ void tile_of(uint32_t id, int tiles_m, int tiles_n, int& tm, int& tn) {
    const uint32_t count = (uint32_t)tiles_m * tiles_n, xcd = id % 8, each = count / 8, more = count % 8;
    const uint32_t at = xcd * each + min(xcd, more) + id / 8;
    constexpr uint32_t kGroup = 8;
    const uint32_t group = at / (kGroup * tiles_n), first = group * kGroup, rows = min(kGroup, (uint32_t)tiles_m - first);
    const uint32_t in = at - group * kGroup * tiles_n;
    tm = __builtin_amdgcn_readfirstlane((int)(first + in % rows));
    tn = __builtin_amdgcn_readfirstlane((int)(in / rows));
}

// How rows come to LDS: straight, through registers, or through registers from addresses that 32 bits do not reach from a tile's first.
enum RowMode { kRowsDirect, kRowsHeld, kRowsFar };

// Large products are bound by the matrix cores at the clock that the card's power leaves them: 8192 x 8192 x 4096 257 us, 2.14 POP/s (7 %
// less with neither loads nor LDS reads), x 16384 877 us, 2.51.  A wavefront of 128 x 128 reads a byte from LDS for 64 products; with four
// of them a compute unit's LDS is busy half of the time.  Smaller tiles: 2048 x 2048 x 2048 16 us, 1.1 POP/s; 1024 x 1024 x 1024 8 us, the call itself.
// RING tiles of the operands are held, so a tile has RING - 1 others' time to arrive.  With more than one workgroup to a tile (gridDim.y) each
// has a stretch of K, and S is int32: its sums go to a matrix of their own.
template <class S, int BM, int BN, int WM, int WN, int STEP, int RING, RowMode MODE>
__global__ __launch_bounds__((BM / WM) * (BN / WN) * 64) void tile_kernel(const Args a) {
    constexpr int THREADS = (BM / WM) * (BN / WN) * 64, WAVES = THREADS / 64;
    constexpr int MT = WM / 32, NT = WN / 32;
    constexpr int XBYTES = BM * STEP, WBYTES = BN * STEP, BYTES = XBYTES + WBYTES;
    constexpr int ROW = STEP / kPiece, SHARE = 256 / STEP;          // pieces of a row, rows that share the banks
    constexpr int PIECES = BYTES / (THREADS * kPiece), XPIECES = XBYTES / (THREADS * kPiece);
    static_assert(XBYTES % (THREADS * kPiece) == 0 && WBYTES % (THREADS * kPiece) == 0, "every load of a workgroup is of one operand");
    static_assert(THREADS / ROW % (SHARE * ROW) == 0, "a thread's pieces lie at the same place of their rows");
    static_assert(MODE == kRowsDirect || RING == 2, "registers hold one tile");
    constexpr int WIDE = WN * sizeof(S) <= 128 ? WN : 128 / sizeof(S);          // channels of the result that a wavefront has in LDS at once
    constexpr int STRIP = WIDE * (int)sizeof(S) + 16;               // a row of them
    static_assert(WAVES * WM * STRIP <= RING * BYTES, "they lie where the operands were");
    __shared__ __attribute__((aligned(128))) char lds[RING * BYTES];
    __shared__ __attribute__((aligned(16))) float channel[2][BN], row_scale[BM];    // channels' scales and biases, rows' scales

    const int thread = threadIdx.x, lane = thread % 64, wave = __builtin_amdgcn_readfirstlane(thread / 64);
    const int wm = wave / (BN / WN), wn = wave % (BN / WN);
    const uint32_t id = blockIdx.z * kAcross + blockIdx.x;
    if (id >= (uint32_t)a.tiles_m * a.tiles_n) return;
    int tm, tn;
    tile_of(id, a.tiles_m, a.tiles_n, tm, tn);
    const int64_t m0 = (int64_t)tm * BM;
    const int n0 = tn * BN;
    const int8_t* const xbase = a.x + m0 * a.x_stride;
    const int8_t* const wbase = a.w + (int64_t)n0 * a.w_stride;
    const int last_m = (int)min((int64_t)BM, a.M - m0) - 1, last_n = min(BN, a.N - n0) - 1;
    // Where this thread's pieces come from: rows beyond the last are the last again, their results are not stored.
    // Piece p of wavefront `wave` fills LDS from (p * THREADS + wave * 64) * 16 on.
    const int in_row = (lane % ROW) ^ (thread / ROW / SHARE % ROW);
    const auto row_of = [&](int p) {
        const int row = ((p < XPIECES ? p : p - XPIECES) * THREADS + thread) / ROW;
        return min(row, p < XPIECES ? last_m : last_n);
    };
    std::conditional_t<MODE == kRowsFar, int64_t, uint32_t> from[PIECES];
#pragma unroll
    for (int p = 0; p < PIECES; ++p)
        from[p] = (decltype(from[0] + 0))row_of(p) * (decltype(from[0] + 0))(p < XPIECES ? a.x_stride : a.w_stride) + in_row * kPiece;
    // Tiles on their way through registers: two where there is room, as a tile of LDS alone leaves loads too little time.
    constexpr int HOLD = MODE == kRowsDirect || PIECES > 8 ? 1 : 2;
    Int4 held[HOLD][MODE == kRowsDirect ? 1 : PIECES];
    const auto put = [&](int p, int buffer, const Int4& v) { *(Int4*)(lds + buffer * BYTES + (p * THREADS + thread) * kPiece) = v; };
    // The sum does not depend on the order of its terms: where K ends inside a tile, that tile is the first, so that only the start has to
    // look at where a row ends.
    const int whole = a.K / STEP, partial = a.K % STEP != 0, all = whole + partial;
    const int t0 = (int)((int64_t)all * blockIdx.y / gridDim.y), tiles = (int)((int64_t)all * (blockIdx.y + 1) / gridDim.y);
    const auto fetch = [&](int p, int t, int buffer, int set) {
        const int8_t* const base = (p < XPIECES ? xbase : wbase) + (int64_t)(t - partial) * STEP;
        if constexpr (MODE == kRowsDirect) {
            const uint32_t to = (uint32_t)(uintptr_t)lds + buffer * BYTES + wave * 1024 + p * THREADS * kPiece;
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                         :
                         : "s"(__builtin_amdgcn_readfirstlane(to)), "v"(from[p]), "s"(scalar(base)) : "memory", "m0");
        } else {
            __builtin_memcpy(&held[set][p], base + from[p], kPiece);
        }
    };
    const auto fetch_all = [&](int t, int buffer, int set) {
        if (t >= tiles) return;
#pragma unroll
        for (int p = 0; p < PIECES; ++p) fetch(p, t, buffer, set);
    };
    // The first tile, where K ends inside it: pieces that a row has all of come like others.
    const auto fetch_partial = [&] {
        const int k = whole * STEP + in_row * kPiece;
        constexpr int U = PIECES > 8 ? 4 : PIECES;
        if (MODE == kRowsDirect && k + kPiece <= a.K) {
#pragma unroll
            for (int p = 0; p < PIECES; ++p) fetch(p, all, 0, 0);
        } else if (MODE == kRowsDirect && k >= a.K) {
#pragma unroll
            for (int p = 0; p < PIECES; ++p) put(p, 0, Int4{0, 0, 0, 0});
        } else {
#pragma unroll
            for (int p = 0; p < PIECES; p += U) {
                const auto row = [&](int u) { return p + u < XPIECES ? xbase + row_of(p + u) * a.x_stride : wbase + row_of(p + u) * a.w_stride; };
                if (a.K < kPiece) {
#pragma unroll
                    for (int u = 0; u < U; ++u) put(p + u, 0, load_short(row(u), k, a.K));
                } else {
                    Clipped<Words> v[U];
#pragma unroll
                    for (int u = 0; u < U; ++u) v[u] = load_clipped_words(row(u), k, a.K);
#pragma unroll
                    for (int u = 0; u < U; ++u) put(p + u, 0, v[u].get());
                }
            }
        }
    };
    const auto put_held = [&](int buffer, int set) {
        if constexpr (MODE != kRowsDirect) {
#pragma unroll
            for (int p = 0; p < PIECES; ++p) put(p, buffer, held[set][p]);
        }
    };
    // Tile t + 1 is in LDS, for every wavefront, and nobody reads tile t there any more; the RING - 2 after it may still be on their way.
    const auto arrive = [&](bool later) {
        if (RING > 2 && later) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"((RING - 2) * PIECES) : "memory");
        else if (MODE == kRowsDirect) asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        else asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");       // held tiles stay on their way
    };

    Int16 sum[MT][NT];
    Int4 operand[2][MT + NT];
    const char* const xrow = lds + (wm * WM + lane % 32) * STEP;
    const char* const wrow = lds + XBYTES + (wn * WN + lane % 32) * STEP;
    // Operand o of part s of a tile (32 bytes of K), for the next multiplication.
    const auto read = [&](int o, int buffer, int s) {
        const int at = buffer * BYTES + ((2 * s + lane / 32) ^ (lane % 32 / SHARE % ROW)) * kPiece;
        operand[s & 1][o] = *(const Int4*)((o < MT ? xrow + o * 32 * STEP : wrow + (o - MT) * 32 * STEP) + at);
    };
    constexpr int PARTS = STEP / 32;
    static_assert(PARTS % 2 == 0, "the next tile's first part is read while this one's last is multiplied");
    // A part's products, and between them, in this order, what else is to be issued: a matrix core takes 32 cycles for a product.
    constexpr int PRODUCTS = MT * NT;
    const auto multiply = [&](int set, int q) {
        const int i = q / NT, j = q % NT;
        sum[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(operand[set][MT + j], operand[set][i], sum[i][j], 0, 0, 0);
    };

    // Tile t0 + r is fetched for buffer r, or into set (r - 1) % HOLD once tile t0 has been put from set 0.
    const bool starts_partial = t0 < partial;
    if (!starts_partial) {
        fetch_all(t0, 0, 0);
        put_held(0, 0);
    }
    constexpr int AHEAD = MODE == kRowsDirect ? RING : HOLD + 1;      // tiles that are in LDS or on their way
#pragma unroll
    for (int r = 1; r < AHEAD; ++r) fetch_all(t0 + r, r, (r - 1) % HOLD);
    if (starts_partial) fetch_partial();
    // behind the first tiles' loads, and not where they are used: each would be waited for by itself
    if constexpr (!std::is_same_v<S, int32_t>) {
        for (int i = thread; i < BN; i += THREADS) {
            const int n = n0 + min(i, last_n);
            channel[0][i] = a.w_scale[n];
            channel[1][i] = a.bias ? a.bias[n] : 0.0f;
        }
        for (int i = thread; i < BM; i += THREADS) row_scale[i] = a.x_scale[m0 + min(i, last_m)];
    }
    if (MODE == kRowsDirect && !starts_partial && t0 + RING - 1 < tiles)
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"((RING - 1) * PIECES) : "memory");
    else arrive(false);
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) sum[i][j][r] = 0;
    if (t0 < tiles) {
#pragma unroll
        for (int o = 0; o < MT + NT; ++o) read(o, 0, 0);
        // Tile t lies in buffer `now`, the next is put from set `set`.  `steady`: there are AHEAD more.  Asked at every tile, that would be a branch
        // behind which the compiler waits for all loads where some would do.
        const auto tile = [&](int t, int now, int set, auto steady) {
            constexpr bool STEADY = decltype(steady)::value;
            const int next = now + 1 == RING ? 0 : now + 1;
#pragma unroll
            for (int s = 0; s < PARTS - 1; ++s)
#pragma unroll
                for (int q = 0; q < PRODUCTS; ++q) {
                    multiply(s & 1, q);
#pragma unroll
                    for (int o = 0; o < MT + NT; ++o)
                        if (o * PRODUCTS / (MT + NT) == q) read(o, now, s + 1);
                    __builtin_amdgcn_sched_barrier(0);
                }
            // Behind the barrier this tile's place is free.  A quarter of the products goes before it, so that waiting for the others does not
            // stop the matrix core at once.
            constexpr int BEFORE = PRODUCTS / 4;
#pragma unroll
            for (int q = 0; q < BEFORE; ++q) multiply(1, q);
            __builtin_amdgcn_sched_barrier(0);
            if (STEADY || t + 1 < tiles) put_held(next, set);
            arrive(STEADY || t + RING - 1 < tiles);
            const bool more = STEADY || t + AHEAD < tiles;
#pragma unroll
            for (int q = BEFORE; q < PRODUCTS; ++q) {
                multiply(1, q);
                // read past the last tile too: what is read then is not used
#pragma unroll
                for (int o = 0; o < MT + NT; ++o)
                    if (BEFORE + o * (PRODUCTS - BEFORE) / (MT + NT) == q) read(o, next, 0);
                if (more) {
#pragma unroll
                    for (int p = 0; p < PIECES; ++p)
                        if (BEFORE + p * (PRODUCTS - BEFORE) / PIECES == q) fetch(p, t + AHEAD, now, set);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        int t = t0;
        if constexpr (HOLD == 2) {
            for (; t + 1 + AHEAD < tiles; t += 2) {
                tile(t, 0, 0, std::true_type());
                tile(t + 1, 1, 1, std::true_type());
            }
            for (; t < tiles; t += 2) {
                tile(t, 0, 0, std::false_type());
                if (t + 1 < tiles) tile(t + 1, 1, 1, std::false_type());
            }
        } else {
            int now = 0;
            for (; t + AHEAD < tiles; ++t) {
                tile(t, now, 0, std::true_type());
                now = now + 1 == RING ? 0 : now + 1;
            }
            for (; t < tiles; ++t) {
                tile(t, now, 0, std::false_type());
                now = now + 1 == RING ? 0 : now + 1;
            }
        }
    }

    // A lane has channels 8 g + 4 (lane / 32) .. + 3 of row lane % 32.  They go through LDS, each wavefront's its own, so that rows are stored in
    // vectors of 16 bytes side by side, 128 bytes of a row at a time.
    char* const strip = lds + wave * WM * STRIP;
    constexpr int VEC = 16 / sizeof(S), LANES = WIDE / VEC, ROWS = 64 / LANES;
    const int64_t mw = m0 + wm * WM;
    S* const out = (S*)a.out + (std::is_same_v<S, int32_t> ? blockIdx.y * a.M * a.out_stride : 0);
    float xs[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) xs[i] = std::is_same_v<S, int32_t> ? 0.0f : row_scale[wm * WM + i * 32 + lane % 32];
#pragma unroll
    for (int j0 = 0; j0 < NT; j0 += WIDE / 32) {
        const int nw = wn * WN + j0 * 32;
#pragma unroll
        for (int j = 0; j < WIDE / 32; ++j)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int in = j * 32 + 8 * g + 4 * (lane / 32);
                Pack<float, 4> ws = {}, bias = {};
                if constexpr (!std::is_same_v<S, int32_t>) {
                    ws = *(const Pack<float, 4>*)&channel[0][nw + in];
                    bias = *(const Pack<float, 4>*)&channel[1][nw + in];
                }
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    char* const to = strip + (i * 32 + lane % 32) * STRIP + in * sizeof(S);
                    const auto& part = sum[i][j0 + j];
                    if constexpr (std::is_same_v<S, int32_t>) {
                        *(Int4*)to = Int4{part[4 * g], part[4 * g + 1], part[4 * g + 2], part[4 * g + 3]};
                    } else {
                        float f[4];
#pragma unroll
                        for (int r = 0; r < 4; ++r) f[r] = scaled(part[4 * g + r], xs[i], ws.get(r), bias.get(r));
                        *(Pack<S, 4>*)to = Pack<S, 4>::from(f);
                    }
                }
            }
        wave_order();
#pragma unroll
        for (int r = 0; r < WM; r += ROWS) {
            const int row = r + lane / LANES, n = n0 + nw + lane % LANES * VEC;
            const int64_t m = mw + row;
            if (m < a.M && n < a.N) {
                const Int4 v = *(const Int4*)(strip + row * STRIP + lane % LANES * 16);
                S* const to = out + m * a.out_stride + n;
                if (n + VEC <= a.N) {
                    __builtin_memcpy(to, &v, sizeof(v));
                } else {
                    const auto each = __builtin_bit_cast(Elements<S>, v);
#pragma unroll
                    for (int e = 0; e < VEC; ++e)
                        if (n + e < a.N) to[e] = each.v[e];
                }
            }
        }
        wave_order();
    }
}

// The stretches' sums of an element, and what follows (64 x 8192, four stretches: 4 us): a thread has N channels of a row.  What would end beyond the row is moved back
// to end with it and stores what the thread before it stores as well.
template <class S, int N>
__global__ __launch_bounds__(256) void join_kernel(const Args a, const int32_t* __restrict__ sums, int stretches) {
    constexpr int U = 8;                 // loads in flight
    int n = (int)(blockIdx.x * 256 + threadIdx.x) * N;
    if (n >= a.N) return;
    n = min(n, a.N - N);
    float ws[N], bias[N];
#pragma unroll
    for (int r = 0; r < N; ++r) {
        ws[r] = a.w_scale[n + r];
        bias[r] = a.bias ? a.bias[n + r] : 0.0f;
    }
    for (int64_t m = blockIdx.y; m < a.M; m += gridDim.y) {
        const int32_t* const at = sums + m * a.N + n;
        int32_t sum[N] = {};
        for (int i = 0; i < stretches; i += U) {
            Pack<int32_t, N> v[U];
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = load_pack<N>(at + min(i + u, stretches - 1) * a.M * a.N);
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int r = 0; r < N; ++r) sum[r] += i + u < stretches ? v[u].v[r] : 0;
        }
        const float xs = a.x_scale[m];
        float f[N];
#pragma unroll
        for (int r = 0; r < N; ++r) f[r] = scaled(sum[r], xs, ws[r], bias[r]);
        store_pack((S*)a.out + m * a.out_stride + n, Pack<S, N>::from(f));
    }
}

// Bound by memory: 8 x 50001 x 1024 11.7 us, 4.4 TB/s; 8 x 8192 x 8192 14.4 us, 4.7; with rows at any byte 8 x 50001 x 1001 15 us, 3.4.  MT * 16 rows;
// NT * 16 channels to `share` wavefronts of a workgroup (8 at the most), each of which has a stretch of K.  Weights are read once, the rows
// of x once for every NT * 16 channels.
constexpr int kFewWaves = 8;
constexpr int64_t kFullCard = 256 * kFewWaves;
template <class S, int MT, int NT>
__global__ __launch_bounds__(kFewWaves * 64) void few_kernel(const Args a, int share) {
    extern __shared__ Int4 sums[];                // of wavefronts that share K
    auto* const parts = (Int4(*)[MT * NT][64])sums;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int64_t n0 = ((int64_t)blockIdx.x * (blockDim.x / 64 / share) + wave / share) * 16 * NT;
    const int steps = (a.K + 63) / 64, each = (steps + share - 1) / share;
    const int begin = min(wave % share * each, steps), end = min(begin + each, steps);
    Int4 sum[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) sum[i][j] = Int4{0, 0, 0, 0};
    // A lane has channels 4 (lane / 16) .. + 3 of row lane % 16.  Their scales are on their way while the sums are made.
    float ws[NT][4], bias[NT][4], xs[MT];
    if (n0 < a.N) {
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int64_t c = min(n0 + j * 16 + lane / 16 * 4 + r, (int64_t)a.N - 1);
                ws[j][r] = a.w_scale[c];
                bias[j][r] = a.bias ? a.bias[c] : 0.0f;
            }
#pragma unroll
        for (int i = 0; i < MT; ++i) xs[i] = a.x_scale[min((int64_t)i * 16 + lane % 16, a.M - 1)];
        const int8_t *wrow[NT], *xrow[MT];
#pragma unroll
        for (int j = 0; j < NT; ++j) wrow[j] = a.w + min(n0 + j * 16 + lane % 16, (int64_t)a.N - 1) * a.w_stride;
#pragma unroll
        for (int i = 0; i < MT; ++i) xrow[i] = a.x + min((int64_t)i * 16 + lane % 16, a.M - 1) * a.x_stride;
        const int in = lane / 16 * kPiece;
        constexpr int U = 8 / NT;
        // the loads of at most `most` steps in flight; `load` takes pieces that a row has all of, or any
        const auto batch = [&](auto most, int s, int count, auto load) __attribute__((always_inline)) {
            constexpr int U = decltype(most)::value;
            decltype(load(wrow[0], 0)) w[U][NT], x[U][MT];
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int j = 0; j < NT; ++j) w[u][j] = load(wrow[j], (s + min(u, count - 1)) * 64 + in);
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int i = 0; i < MT; ++i) x[u][i] = load(xrow[i], (s + min(u, count - 1)) * 64 + in);
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (u < count) {
                    Int4 wv[NT];
#pragma unroll
                    for (int j = 0; j < NT; ++j) wv[j] = w[u][j].get();
#pragma unroll
                    for (int i = 0; i < MT; ++i) {
                        const Int4 xv = x[u][i].get();
#pragma unroll
                        for (int j = 0; j < NT; ++j) sum[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wv[j], xv, sum[i][j], 0, 0, 0);
                    }
                }
        };
        int s = begin;
        if (a.K < kPiece) {
            if (s < end) batch(std::integral_constant<int, 1>(), s, 1, [&](const int8_t* row, int k) { return Whole{load_short(row, k, a.K)}; });
        } else {
            constexpr std::integral_constant<int, U> full;
            // a step too many costs its loads (20 x 1000 x 333, six steps: 12 us with the loads of eight, 8 with those of six)
            const auto some = [&](int s, int count, auto load) __attribute__((always_inline)) {
                if (count * 4 <= U) batch(std::integral_constant<int, U / 4>(), s, count, load);
                else if (count * 2 <= U) batch(std::integral_constant<int, U / 2>(), s, count, load);
                else if (count * 4 <= U * 3) batch(std::integral_constant<int, U * 3 / 4>(), s, count, load);
                else batch(full, s, min(count, U), load);
            };
            if (a.bytes) {
                const auto words = [&](const int8_t* row, int k) { return load_clipped_words(row, k, a.K); };
                if (s == 0) {
                    some(s, end, words);
                    s = U;
                }
                for (; s + U <= end && (s + U) * 64 + 4 <= a.K; s += U)
                    batch(full, s, U, [](const int8_t* row, int k) { return load_words(row + k, beyond_word(row), true); });
                for (; s < end; s += U) some(s, end - s, words);
            } else {
                for (; s + U <= end && (s + U) * 64 <= a.K; s += U) batch(full, s, U, [](const int8_t* row, int k) { return load_whole(row + k); });
                for (; s < end; s += U) some(s, end - s, [&](const int8_t* row, int k) { return load_clipped(row, k, a.K); });
            }
        }
    }
    if (share > 1) {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j) parts[wave][i * NT + j][lane] = sum[i][j];
        __syncthreads();
        if (wave % share != 0) return;
        for (int p = 1; p < share; ++p)
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) sum[i][j] += parts[wave + p][i * NT + j][lane];
    }
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const int64_t n = n0 + j * 16 + lane / 16 * 4;
        if (n >= a.N) continue;
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const int64_t m = i * 16 + lane % 16;
            if (m >= a.M) continue;
            S* const to = (S*)a.out + m * a.out_stride + n;
            float f[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) f[r] = scaled(sum[i][j][r], xs[i], ws[j][r], bias[j][r]);
            if (n + 4 <= a.N) {
                store_pack(to, Pack<S, 4>::from(f));
            } else {
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (n + r < a.N) to[r] = narrow<S>(f[r]);
            }
        }
    }
}

template <class S, int MT, int NT>
void launch_few(const Args& a, int64_t waves, hipStream_t s) {
    const int64_t places = (a.N + 16 * NT - 1) / (16 * NT);
    int share = 1;
    while (share < kFewWaves && places * share < waves && a.K > 512 / NT * share) share *= 2;
    // A compute unit has one workgroup of eight wavefronts or two: unless those nearly fill the card, wavefronts that share nothing go by
    // themselves (8 x 90000 x 1024: 18 us, 24 in eights; 1 x 131072 x 1024, where eights fill it twice: 27.7 and 27.4).
    const int64_t all = places * share, rounds = (all + kFullCard - 1) / kFullCard;
    const int64_t per = all * 10 >= rounds * kFullCard * 9 ? kFewWaves / share : 1;
    hipLaunchKernelGGL((few_kernel<S, MT, NT>), dim3((unsigned)((places + per - 1) / per)), dim3((unsigned)(per * share * 64)),
                       share > 1 ? (size_t)(per * share) * MT * NT * 64 * sizeof(Int4) : 0, s, a, share);
}

// Counts a result's tiles and gives the grid that has them.
dim3 tile_grid(Args& a, int bm, int bn, int stretches) {
    a.tiles_m = (int)((a.M + bm - 1) / bm);
    a.tiles_n = (a.N + bn - 1) / bn;
    const int64_t tiles = (int64_t)a.tiles_m * a.tiles_n;
    return dim3((unsigned)(tiles < kAcross ? tiles : kAcross), (unsigned)stretches, (unsigned)((tiles + kAcross - 1) / kAcross));
}

template <class S, int BM, int BN, int WM, int WN, int STEP, int RING>
void launch_tiles(Args a, bool direct, int stretches, hipStream_t s) {
    const dim3 grid = tile_grid(a, BM, BN, stretches), block((BM / WM) * (BN / WN) * 64);
    if (direct) hipLaunchKernelGGL((tile_kernel<S, BM, BN, WM, WN, STEP, RING, kRowsDirect>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((tile_kernel<S, BM, BN, WM, WN, 128, 2, kRowsHeld>), grid, block, 0, s, a);
}

int64_t tiles_of(int64_t M, int64_t N, int64_t side) { return ((M + side - 1) / side) * ((N + side - 1) / side); }

constexpr int64_t kFewRows = 32;
// A tile of 256 takes a compute unit, which has two of 128 at once; those take 0.6 of its time together (8192 x 8192 x 4096: 259 us in four
// rounds of the former, 305 in eight of the latter), but leave less of a last round unused (5000 x 5000 x 1024: 46 and 45 us).
bool large_tiles(int64_t M, int64_t N) {
    const double small = (double)tiles_of(M, N, 128) / 512;
    return (double)((tiles_of(M, N, 256) + 255) / 256) <= 0.6 * (small < 1.0 ? 1.0 : small);
}
// Stretches of K for tiles of 64: as many as give every compute unit two workgroups, none shorter than eight tiles of K.
int stretches_of(int64_t M, int64_t N, int64_t K) {
    if (M <= kFewRows || tiles_of(M, N, 128) >= 192) return 1;
    const int64_t most = K / 1024, want = 512 / tiles_of(M, N, 64);
    return (int)(want < 2 || most < 2 ? 1 : want < most ? want : most);
}

template <class S>
void run(const Args& a, void* workspace, hipStream_t s) {
    // of a tile's 256 rows the farthest is addressed by 31 bits from its first
    const bool far = a.x_stride >= 1 << 23 || a.w_stride >= 1 << 23;
    const bool direct = !far && !a.bytes;
    const int stretches = stretches_of(a.M, a.N, a.K);
    if (a.M <= kFewRows) {
        // 8 x 50001 x 1024: 11.9 us with 32 channels a wavefront, 13.4 with 16; 1 x 512 x 8192: 10.9 and 7.5 to 8.3
        if (a.N >= 16384) a.M <= 16 ? launch_few<S, 1, 2>(a, 1536, s) : launch_few<S, 2, 2>(a, 1536, s);
        else a.M <= 16 ? launch_few<S, 1, 1>(a, 2048, s) : launch_few<S, 2, 1>(a, 2048, s);
    } else if (far) {
        Args b = a;
        const dim3 grid = tile_grid(b, 64, 64, 1);
        hipLaunchKernelGGL((tile_kernel<S, 64, 64, 32, 32, 128, 2, kRowsFar>), grid, dim3(256), 0, s, b);
    } else if (stretches > 1) {
        Args b = a;
        b.out = workspace;
        b.out_stride = a.N;
        launch_tiles<int32_t, 64, 64, 32, 32, 128, 4>(b, direct, stretches, s);
        const unsigned rows = (unsigned)(a.M < 16384 ? a.M : 16384);
        if (a.N >= 4) hipLaunchKernelGGL((join_kernel<S, 4>), dim3((unsigned)((a.N + 1023) / 1024), rows), dim3(256), 0, s, a, (const int32_t*)workspace, stretches);
        else hipLaunchKernelGGL((join_kernel<S, 1>), dim3(1, rows), dim3(256), 0, s, a, (const int32_t*)workspace, stretches);
    } else if (tiles_of(a.M, a.N, 256) >= 128 && a.K > 512 && large_tiles(a.M, a.N)) {
        launch_tiles<S, 256, 256, 128, 128, 128, 2>(a, direct, 1, s);
    } else if (tiles_of(a.M, a.N, 128) >= 192) {
        launch_tiles<S, 128, 128, 64, 64, 128, 2>(a, direct, 1, s);
    } else {
        launch_tiles<S, 64, 64, 32, 32, 128, 4>(a, direct, 1, s);
    }
}

}  // namespace

size_t product_workspace_bytes(int64_t M, int64_t N, int64_t K) {
    if (M == 0 || N == 0) return 0;
    const int64_t stretches = stretches_of(M, N, K);
    return stretches > 1 ? (size_t)((stretches * M * N * 4 + 255) / 256 * 256) : 0;
}

hipError_t launch_product(const ProductCall& c, hipStream_t s) {
    Args a = {};
    a.x = c.x;
    a.w = c.w;
    a.x_scale = c.x_scale;
    a.w_scale = c.w_scale;
    a.bias = c.bias;
    a.M = c.M;
    a.N = (int)c.N;
    a.K = (int)c.K;
    a.x_stride = c.x_stride;
    a.w_stride = c.w_stride;
    a.out_stride = c.out_stride;
    a.out = c.out;
    a.bytes = (((uintptr_t)c.x | (uintptr_t)c.w | (uintptr_t)c.x_stride | (uintptr_t)c.w_stride) & 3) != 0;
    if (c.dtype == kF32) run<float>(a, c.workspace, s);
    else if (c.dtype == kF16) run<_Float16>(a, c.workspace, s);
    else run<__bf16>(a, c.workspace, s);
    return hipGetLastError();
}

}  // namespace cc
