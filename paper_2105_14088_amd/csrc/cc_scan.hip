// Gated linear recurrence over positions and its gradient (cc.h: cc_gated_scan, cc_gated_scan_backward).
//
//   keep = sigmoid(gate), take = 1 - keep = sigmoid(-gate)
//   h_t  = keep_t h_{t-1} + take_t x_t
//   With F_{t+1} what later positions ask of h_t (F_len = the last state's gradient):
//   lambda_t = dh_t + F_{t+1},  F_t = keep_t lambda_t
//   dx_t = take_t lambda_t,  dgate_t = lambda_t (h_{t-1} - x_t) keep_t take_t,  dh0 = F_0
//
// Channels are independent, so a thread owns two neighbouring channels of one sequence and walks along the positions,
// state in registers; a wavefront's lanes lie along the channels.  Where there are too few channels to fill the chip the
// positions are cut into segments: a first kernel reduces each segment to the pair (product of keeps, what it adds), a second
// chains the pairs, a third walks each segment from the state it found.
//
// The backward pass needs h_{t-1} in 32 bits, and h is stored rounded.  The forward pass keeps the state before every
// kScanChunk positions; the backward pass walks the chunks from the last one, makes a chunk's states again from x and the
// gate, which it has in registers anyway, and then goes back through them.  That reads less than h itself would take.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "cc_internal.h"
#include "cc_model.h"

// From the same state a position gives the same bits whichever walk it is worked in: products and sums are fused where fmaf says so and
// nowhere else.  (The state that a segment starts from is chained from rounded products of gates: T steps of one position give the
// bits of one call where its positions are not cut into segments.)
#pragma clang fp contract(off)

namespace cc {
namespace {

using namespace ccm;

constexpr int kThreads = 256, L = kScanChunk;

// keep and take from e = exp(-|gate|): 1 / (1 + e) and e / (1 + e), neither of them as one minus the other, so that both keep
// their relative precision.  In 32 bits: the exponential of a rounded product with log2 e (off by up to 1.5 |gate| 2^-24 and its last
// bit) and the reciprocal instruction (last bit) without a step to refine it: a step would take three operations of some twenty an
// element to win the last bit of a gate (1024 x 64 x 128 fp32, forward and backward: 1.40e-7 off the definition, elementary
// operations in 32 bits 1.24e-7).
//
// The smaller one is held as two factors, each with half of the exponential's argument.  What it multiplies is then rounded once
// where the product is subnormal, and the exponential instruction, which gives 0 for subnormal results, is never asked for
// one that matters.  MIXED: gates of up to kMild need none of that, and are the same as MildGates to the last bit, wherever a
// position is worked on: in a chunk, at its end or alone.
constexpr float kMild = 64.0f;
template <bool MIXED>
struct Gates {
    float keep1, keep2, take1, take2;
    __device__ __forceinline__ explicit Gates(float g) {
        const bool mild = MIXED && fabsf(g) <= kMild;
        const float q = exp_fast(mild ? -fabsf(g) : -0.5f * fabsf(g)), other = mild ? 1.0f : q;
        const float large = __builtin_amdgcn_rcpf(fmaf(q, other, 1.0f)), small2 = q * large;
        keep1 = g >= 0.0f ? 1.0f : other;
        keep2 = g >= 0.0f ? large : small2;
        take1 = g >= 0.0f ? other : 1.0f;
        take2 = g >= 0.0f ? small2 : large;
    }
    __device__ __forceinline__ float keep(float v) const { return v * keep1 * keep2; }
    __device__ __forceinline__ float take(float v) const { return v * take1 * take2; }
    __device__ __forceinline__ float step(float h, float x) const { return fmaf(h * keep1, keep2, take(x)); }
};
struct MildGates {
    float k, t;
    __device__ __forceinline__ explicit MildGates(float g) {
        const float e = exp_fast(-fabsf(g)), large = __builtin_amdgcn_rcpf(1.0f + e), small = e * large;
        k = g >= 0.0f ? large : small;
        t = g >= 0.0f ? small : large;
    }
    __device__ __forceinline__ float keep(float v) const { return v * k; }
    __device__ __forceinline__ float take(float v) const { return v * t; }
    __device__ __forceinline__ float step(float h, float x) const { return fmaf(h, k, take(x)); }
};

struct Args {
    const void *x, *gate, *h_in;      // h_in: gradient of h (backward)
    void *h, *grad_x, *grad_gate;
    int64_t xb, xt, gb, gt, hb, ht, dxb, dxt, dgb, dgt;
    int64_t B, T, D;
    int lanes;                        // threads per sequence
    const int32_t* lengths;
    const float* h0;
    float* last;
    const float* last_grad;
    float* states;
    float* grad_h0;
    int64_t chunks;                   // of kScanChunk positions in T
    int64_t segment;                  // positions per segment, a multiple of kScanChunk
    int segments;
    float *products, *sums;           // [segments][B * D]
    const float* starts;              // [segments][B * D], null with one segment
};

// What a thread owns: C neighbouring channels of one sequence.  Where the last thread of a row would reach beyond it, it is moved
// back to end with the row: it then computes a channel of the thread before it as well, and stores it again, the same value.  No load
// and no store depends on a lane's place in the row, and all of a chunk's are in flight together.
template <int C>
struct Lane {
    uint32_t b;
    int d;
    int64_t n;                        // positions that count
    bool real;
    __device__ __forceinline__ explicit Lane(const Args& a) {
        const uint32_t id = blockIdx.x * kThreads + threadIdx.x;
        b = id / (uint32_t)a.lanes;
        real = b < a.B;
        d = min(C * (int)(id - b * (uint32_t)a.lanes), (int)a.D - C);
        n = a.T;
        if (real && a.lengths) n = min(a.T, (int64_t)max(a.lengths[b], 0));
    }
};

// A tensor's rows as a thread sees them: a base that is the same in all lanes, kept in scalar registers and moved from chunk to
// row there, and a lane's offset in bytes of type Off.  With offsets of 32 bits (chosen where the tensor's sequences and a chunk's
// rows lie within them) a tensor takes one vector register for addresses; pointers of 64 bits to 16 rows of five tensors would
// take 160.
template <class S, int C, class Off>
struct Rows {
    S* base;
    int64_t stride;
    Off lane;
    __device__ __forceinline__ Rows(void* p, int64_t apart, int64_t stride_, const Lane<C>& l)
        : base((S*)p), stride(stride_), lane(((Off)l.b * (Off)apart + (Off)l.d) * (Off)sizeof(S)) {}
    // The base at position t, in scalar registers (the compiler would keep, and advance, one per lane).
    __device__ __forceinline__ S* at(int64_t t) const {
        const uint64_t v = (uint64_t)(base + t * stride);
        const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
        return (S*)(__attribute__((address_space(1))) S*)(((uint64_t)hi << 32) | lo);
    }
    __device__ __forceinline__ Pack<S, C> load(const S* p, int i) const {
        return load_pack<C>((const S*)((const char*)(p + i * stride) + lane));
    }
    __device__ __forceinline__ Pack<S, C> load_own(const S* p, int i) const {      // i differs between lanes
        return load_pack<C>((const S*)((const char*)p + (Off)(lane + (Off)i * ((Off)stride * (Off)sizeof(S)))));
    }
    // What is stored is a value of 32 bits that is rounded: an instruction that rounds a sum of products to f16 at once, where the
    // compiler finds its form, would store other bits in one walk than in another.
    __device__ __forceinline__ void store(S* p, int i, float v[C]) const {
        if (__is_same(S, _Float16)) {
#pragma unroll
            for (int c = 0; c < C; ++c) asm("" : "+v"(v[c]));
        }
        store_pack((S*)((char*)(p + i * stride) + lane), Pack<S, C>::from(v));
    }
    // A chunk's rows from position t on.  Of a chunk that does not count as a whole, the others' places hold the last row that does.
    template <bool FULL>
    __device__ __forceinline__ void load_chunk(int64_t t, int inside, Pack<S, C> rows[L]) const {
        const S* const p = at(t);
#pragma unroll
        for (int i = 0; i < L; ++i) rows[i] = FULL ? load(p, i) : load_own(p, min(i, inside - 1));
    }
};
template <int C, class Off>
__device__ __forceinline__ void read(const Rows<float, C, Off>& r, int64_t t, float v[C]) {
    const Pack<float, C> p = r.load(r.at(t), 0);
#pragma unroll
    for (int c = 0; c < C; ++c) v[c] = p.get(c);
}
template <int C, class Off>
__device__ __forceinline__ void write(const Rows<float, C, Off>& r, int64_t t, float v[C]) { r.store(r.at(t), 0, v); }

// MILD kernels ask whether a wavefront's gates of a chunk can be MildGates: five operations fewer each, for elements of 16 bits, whose
// walks wait for operations as much as for memory (32 x 1024 x 1024 bf16, forward and backward: 162 us with Gates alone, 152 so;
// of 32 bits there is no difference).
template <class S, int C>
__device__ __forceinline__ bool mild(const Pack<S, C> gs[L]) {
    float top = 0.0f;
#pragma unroll
    for (int i = 0; i < L; ++i)
#pragma unroll
        for (int c = 0; c < C; ++c) top = fmaxf(top, fabsf(gs[i].get(c)));
    return __all(top <= kMild);
}
// Nothing that was made of a chunk's rows before the ways part is kept beside them.
template <class S, int C>
__device__ __forceinline__ void forget_rows(Pack<S, C> rows[L]) {
#pragma unroll
    for (int i = 0; i < L; ++i) forget(rows[i]);
}

// What the length leaves of a chunk: all of it in all lanes, or something in some.
struct Part {
    int count, inside;                // positions of the segment, positions that count
    bool full;
    __device__ __forceinline__ Part(int64_t t0, int64_t to, int64_t end) {
        count = (int)min((int64_t)L, to - t0);
        inside = (int)max((int64_t)0, min((int64_t)L, end - t0));
        full = __all(inside >= L);
    }
};

// Forward walk.  Bound by memory (2 x 65536 x 1024 bf16: 149 us for 838 MB, 5.6 TB/s; SUMMARY reads 537 MB in 116 us).  SUMMARY: only the segment's product of keeps and what it adds; the last segment needs none.
template <class S, int C, class Off, bool MILD, bool SUMMARY>
__global__ __launch_bounds__(kThreads) void scan_kernel(Args a) {
    const Lane<C> l(a);
    if (!l.real) return;
    const int seg = blockIdx.y;
    const int64_t from = seg * a.segment, to = min(a.T, from + a.segment), end = min(to, l.n);
    const Rows<S, C, Off> x((void*)a.x, a.xb, a.xt, l), g((void*)a.gate, a.gb, a.gt, l), out(a.h, a.hb, a.ht, l);
    const Rows<float, C, Off> states(a.states, a.chunks * a.D, a.D, l), last(a.last, a.D, 0, l), h0((void*)a.h0, a.D, 0, l);
    const Rows<float, C, Off> starts((void*)a.starts, a.D, a.B * a.D, l), products(a.products, a.D, a.B * a.D, l), sums(a.sums, a.D, a.B * a.D, l);
    float h[C] = {}, product[C];
#pragma unroll
    for (int c = 0; c < C; ++c) product[c] = 1.0f;
    if (!SUMMARY) {
        if (a.starts) read<C>(starts, seg, h);
        else if (a.h0) read<C>(h0, 0, h);
    }
    struct Chunk {
        Pack<S, C> xs[L], gs[L];
    };
    const auto load = [&](auto whole, int64_t t0, int inside, Chunk& to) {
        constexpr bool FULL = decltype(whole)::value;
        x.template load_chunk<FULL>(t0, inside, to.xs);
        g.template load_chunk<FULL>(t0, inside, to.gs);
    };
    // FULL: the chunk counts as a whole and, in a MILD kernel, its gates are mild
    const auto walk = [&](auto whole, int64_t t0, const Part& part, const Chunk& loaded) {
        constexpr bool FULL = decltype(whole)::value;
        using Gate = std::conditional_t<FULL && MILD, MildGates, Gates<sizeof(S) == 2>>;
        Chunk own;
        if (!MILD && (FULL || part.inside > 0)) load(whole, t0, part.inside, own);
        const Chunk& rows = MILD ? loaded : own;
        S* const to_row = SUMMARY ? nullptr : out.at(t0);
#pragma unroll
        for (int i = 0; i < L; ++i) {
            const bool in = FULL || i < part.inside;
            float shown[C];
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const Gate gate(rows.gs[i].get(c));
                const float next = gate.step(h[c], rows.xs[i].get(c));
                h[c] = in ? next : h[c];
                if (SUMMARY) product[c] = in ? gate.keep(product[c]) : product[c];
                shown[c] = in ? next : 0.0f;
            }
            if (!SUMMARY && (FULL || i < part.count)) out.store(to_row, i, shown);
        }
    };
    for (int64_t t0 = from; t0 < to; t0 += L) {
        const Part part(t0, to, end);
        if (!SUMMARY && a.states) write<C>(states, t0 / L, h);
        bool whole = part.full;
        Chunk rows;
        if (MILD) {
            if (part.full) load(std::true_type(), t0, L, rows);
            else if (part.inside > 0) load(std::false_type(), t0, part.inside, rows);
            whole = part.full && mild<S, C>(rows.gs);
            forget_rows(rows.gs);
            forget_rows(rows.xs);
        }
        if (whole) walk(std::true_type(), t0, part, rows);
        else walk(std::false_type(), t0, part, rows);
    }
    if (SUMMARY) {
        write<C>(products, seg, product);
        write<C>(sums, seg, h);
    } else if (seg == a.segments - 1 && a.last) {
        write<C>(last, 0, h);
    }
}

// Backward walk.  (2 x 65536 x 1024 bf16: 256 us for 1.38 GB, 5.4 TB/s; SUMMARY 118 us.  A chunk's rows loaded while the one before is
// worked on: 210 registers and the same time.)  SUMMARY: only the segment's product of keeps and what it sends back; the first segment needs none.
template <class S, int C, class Off, bool MILD, bool SUMMARY>
__global__ __launch_bounds__(kThreads, SUMMARY ? 0 : sizeof(S) == 4 || MILD ? 3 : 4) void scan_backward_kernel(Args a) {
    const Lane<C> l(a);
    if (!l.real) return;
    const int seg = SUMMARY ? blockIdx.y + 1 : blockIdx.y;
    const int64_t from = seg * a.segment, to = min(a.T, from + a.segment), end = min(to, l.n);
    const Rows<S, C, Off> x((void*)a.x, a.xb, a.xt, l), g((void*)a.gate, a.gb, a.gt, l), dh((void*)a.h_in, a.hb, a.ht, l);
    const Rows<S, C, Off> dx_out(a.grad_x, a.dxb, a.dxt, l), dg_out(a.grad_gate, a.dgb, a.dgt, l);
    const Rows<float, C, Off> states(a.states, a.chunks * a.D, a.D, l), last_grad((void*)a.last_grad, a.D, 0, l), grad_h0(a.grad_h0, a.D, 0, l);
    const Rows<float, C, Off> starts((void*)a.starts, a.D, a.B * a.D, l), products(a.products, a.D, a.B * a.D, l), sums(a.sums, a.D, a.B * a.D, l);
    float f[C] = {}, product[C];
#pragma unroll
    for (int c = 0; c < C; ++c) product[c] = 1.0f;
    if (!SUMMARY) {
        if (a.starts) read<C>(starts, seg, f);
        else if (a.last_grad) read<C>(last_grad, 0, f);
    }
    struct Chunk {
        Pack<S, C> xs[L], gs[L], ds[L];
    };
    const auto load = [&](auto whole, int64_t t0, int inside, Chunk& to) {
        constexpr bool FULL = decltype(whole)::value;
        g.template load_chunk<FULL>(t0, inside, to.gs);
        dh.template load_chunk<FULL>(t0, inside, to.ds);
        if (!SUMMARY) x.template load_chunk<FULL>(t0, inside, to.xs);
    };
    const auto walk = [&](auto whole, int64_t t0, const Part& part, const Chunk& loaded) {
        constexpr bool FULL = decltype(whole)::value;
        using Gate = std::conditional_t<FULL && MILD, MildGates, Gates<sizeof(S) == 2>>;
        Chunk rows;
        float before[L][C], h[C] = {};
        if (MILD) rows = loaded;
        if (FULL || part.inside > 0) {
            if (!MILD) load(whole, t0, part.inside, rows);
            if (!SUMMARY) read<C>(states, t0 / L, h);
        }
        if (!SUMMARY) {
#pragma unroll
            for (int i = 0; i < L; ++i)
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    before[i][c] = h[c];
                    if (i + 1 < L) h[c] = Gate(rows.gs[i].get(c)).step(h[c], rows.xs[i].get(c));   // of use where position i + 1 counts
                }
        }
        // The gates are made again on the way back: kept, a chunk's would take 128 registers and three quarters of the wavefronts.
        if (!SUMMARY) {
#pragma unroll
            for (int i = 0; i < L; ++i) forget(rows.gs[i]);
        }
        S* const dx_row = SUMMARY ? nullptr : dx_out.at(t0);
        S* const dg_row = SUMMARY ? nullptr : dg_out.at(t0);
#pragma unroll
        for (int i = L - 1; i >= 0; --i) {
            const bool in = FULL || i < part.inside;
            float dx[C], dg[C];
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const Gate gate(rows.gs[i].get(c));
                const float lambda = rows.ds[i].get(c) + f[c];
                f[c] = in ? gate.keep(lambda) : f[c];
                if (SUMMARY) {
                    product[c] = in ? gate.keep(product[c]) : product[c];
                } else {
                    dx[c] = in ? gate.take(lambda) : 0.0f;
                    dg[c] = in ? gate.keep(gate.take(lambda * (before[i][c] - rows.xs[i].get(c)))) : 0.0f;
                }
            }
            if (!SUMMARY && (FULL || i < part.count)) {
                dx_out.store(dx_row, i, dx);
                dg_out.store(dg_row, i, dg);
            }
        }
    };
    for (int64_t t0 = to > from ? from + (to - from - 1) / L * L : from - L; t0 >= from; t0 -= L) {
        const Part part(t0, to, end);
        bool whole = part.full;
        Chunk rows;
        if (MILD) {
            if (part.full) load(std::true_type(), t0, L, rows);
            else if (part.inside > 0) load(std::false_type(), t0, part.inside, rows);
            whole = part.full && mild<S, C>(rows.gs);
            forget_rows(rows.gs);
            forget_rows(rows.ds);
            if (!SUMMARY) forget_rows(rows.xs);
            __builtin_amdgcn_sched_barrier(0);
        }
        if (whole) walk(std::true_type(), t0, part, rows);
        else walk(std::false_type(), t0, part, rows);
    }
    if (SUMMARY) {
        write<C>(products, seg, product);
        write<C>(sums, seg, f);
    } else if (seg == 0 && a.grad_h0) {
        write<C>(grad_h0, 0, f);
    }
}

// Chains the segments: what each starts from, left in the place of its product.  Forward from the first segment, backward from the
// last.  A workgroup has 64 channels and cuts the segments into kParts parts: each part's product and sum, then the parts in
// turn, then each part's segments from what it starts with.
constexpr int kParts = 16;
template <bool BACKWARD>
__global__ __launch_bounds__(64 * kParts) void scan_chain_kernel(float* products, const float* sums, const float* first, int segments, int64_t row) {
    __shared__ float part_product[kParts][64], part_sum[kParts][64];
    const int lane = threadIdx.x & 63, part = threadIdx.x >> 6;
    const int64_t i = (int64_t)blockIdx.x * 64 + lane;
    const bool real = i < row;
    const int each = (segments + kParts - 1) / kParts, from = min(segments, part * each), to = min(segments, from + each);
    const auto place = [&](int s) { return (int64_t)(BACKWARD ? segments - 1 - s : s) * row + i; };
    float product = 1.0f, sum = 0.0f;
    if (real) {
#pragma unroll 8
        for (int s = from; s < to; ++s) {
            if (s + 1 == segments) break;             // the last is not summed up
            const float p = products[place(s)];
            sum = fmaf(p, sum, sums[place(s)]);
            product *= p;
        }
    }
    part_product[part][lane] = product;
    part_sum[part][lane] = sum;
    __syncthreads();
    if (!real) return;
    float h = first ? first[i] : 0.0f;
    for (int p = 0; p < part; ++p) h = fmaf(part_product[p][lane], h, part_sum[p][lane]);
#pragma unroll 8
    for (int s = from; s < to; ++s) {
        const float p = s + 1 < segments ? products[place(s)] : 0.0f, q = s + 1 < segments ? sums[place(s)] : 0.0f;
        products[place(s)] = h;
        h = fmaf(p, h, q);
    }
}

// Segments for B sequences of T positions and D channels: as many as make 2^17 threads, of 32 positions at least; fewer than four
// cost more in launches and second readings than their threads bring.  Forward and backward in us, bf16, by segments:
//   8 x 4096 x 512     1: 490, 924   16: 68, 95    64: 41, 54   128: 41, 52
//   32 x 1024 x 1024   1: 126, 274    2: 126, 202   8: 62, 94    32: 63, 90
//   64 x 1024 x 1024   1: 150, 293    2: 152, 223   4: 126, 188  16: 136, 202
//   1024 x 64 x 64     1: 13, 22      2: 18, 23     4: 17, 21
struct Split {
    int64_t segment;
    int segments;
};
Split split(int64_t B, int64_t T, int64_t D) {
    const int64_t threads = B * ((D + 1) / 2);
    int64_t want = threads > 0 ? ((1 << 17) + threads - 1) / threads : 1;
    if (want > T / 32) want = T / 32;
    if (want < 4) want = 1;
    if (want > 16384) want = 16384;
    if (want < 1) want = 1;
    Split s;
    s.segment = (T + want - 1) / want;
    s.segment = (s.segment + L - 1) / L * L;
    if (s.segment < L) s.segment = L;
    s.segments = (int)((T + s.segment - 1) / s.segment);
    if (s.segments < 1) s.segments = 1;
    return s;
}

size_t up256(size_t x) { return (x + 255u) & ~(size_t)255u; }

Args arguments(const ScanCall& c, const Split& s, int channels) {
    Args a = {};
    a.x = c.x.p; a.xb = c.x.b; a.xt = c.x.t;
    a.gate = c.gate.p; a.gb = c.gate.b; a.gt = c.gate.t;
    a.hb = c.h.b; a.ht = c.h.t;
    a.B = c.B; a.T = c.T; a.D = c.D;
    a.lanes = (int)((c.D + channels - 1) / channels);
    a.lengths = c.lengths;
    a.states = c.states;
    a.chunks = (c.T + L - 1) / L;
    a.segment = s.segment;
    a.segments = s.segments;
    if (s.segments > 1) {
        a.products = (float*)c.workspace;
        a.sums = (float*)((char*)c.workspace + up256(sizeof(float) * (size_t)s.segments * (size_t)(c.B * c.D)));
        a.starts = a.products;
    }
    return a;
}

template <class S, int C, class Off, bool MILD>
hipError_t forward(const ScanCall& c, hipStream_t s) {
    const Split p = split(c.B, c.T, c.D);
    Args a = arguments(c, p, C);
    a.h = c.h.p;
    a.h0 = c.h0;
    a.last = c.last;
    const unsigned blocks = (unsigned)((c.B * a.lanes + kThreads - 1) / kThreads);
    const int64_t row = c.B * c.D;
    if (p.segments > 1) {
        hipLaunchKernelGGL((scan_kernel<S, C, Off, MILD, true>), dim3(blocks, p.segments - 1), dim3(kThreads), 0, s, a);
        hipLaunchKernelGGL((scan_chain_kernel<false>), dim3((unsigned)((row + 63) / 64)), dim3(64 * kParts), 0, s, a.products, a.sums, c.h0,
                           p.segments, row);
    }
    hipLaunchKernelGGL((scan_kernel<S, C, Off, MILD, false>), dim3(blocks, p.segments), dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

template <class S, int C, class Off, bool MILD>
hipError_t backward(const ScanCall& c, hipStream_t s) {
    const Split p = split(c.B, c.T, c.D);
    Args a = arguments(c, p, C);
    a.h_in = c.h.p;
    a.last_grad = c.last;
    a.grad_x = c.grad_x.p; a.dxb = c.grad_x.b; a.dxt = c.grad_x.t;
    a.grad_gate = c.grad_gate.p; a.dgb = c.grad_gate.b; a.dgt = c.grad_gate.t;
    a.grad_h0 = c.grad_h0;
    const unsigned blocks = (unsigned)((c.B * a.lanes + kThreads - 1) / kThreads);
    const int64_t row = c.B * c.D;
    if (p.segments > 1) {
        hipLaunchKernelGGL((scan_backward_kernel<S, C, Off, MILD, true>), dim3(blocks, p.segments - 1), dim3(kThreads), 0, s, a);
        hipLaunchKernelGGL((scan_chain_kernel<true>), dim3((unsigned)((row + 63) / 64)), dim3(64 * kParts), 0, s, a.products, a.sums,
                           (const float*)c.last, p.segments, row);
    }
    hipLaunchKernelGGL((scan_backward_kernel<S, C, Off, MILD, false>), dim3(blocks, p.segments), dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

// Whether a lane's offsets fit 32 bits: sequences and channels of a tensor, and a chunk's rows.  The first and the last state are bounded by
// themselves: without positions there are no kept states.
bool near(const Strided& t, const ScanCall& c, int64_t bytes) {
    return (double)bytes * ((double)(c.B > 0 ? c.B - 1 : 0) * (double)t.b + (double)c.D + (double)L * (double)t.t) < 4294967296.0;
}
bool all_near(const ScanCall& c, bool backward) {
    const int64_t e = c.dtype == kF32 ? 4 : 2, chunks = (c.T + L - 1) / L;
    const Strided states = {nullptr, chunks * c.D, c.D}, ends = {nullptr, c.D, 0};
    return near(c.x, c, e) && near(c.gate, c, e) && near(c.h, c, e) && near(states, c, 4) && near(ends, c, 4) &&
           (!backward || (near(c.grad_x, c, e) && near(c.grad_gate, c, e)));
}

template <class S, bool BACKWARD>
hipError_t choose(const ScanCall& c, hipStream_t s) {
    // A thread that is moved back reads the first state of a channel that another thread owns: not where that one may have
    // overwritten it with the last.
    const void *in = BACKWARD ? (const void*)c.last : (const void*)c.h0, *out = BACKWARD ? (const void*)c.grad_h0 : (const void*)c.last;
    const bool in_place = in && in == out;
    if (c.D == 1 || ((c.D & 1) && in_place)) return BACKWARD ? backward<S, 1, uint64_t, false>(c, s) : forward<S, 1, uint64_t, false>(c, s);
    if (!all_near(c, BACKWARD)) return BACKWARD ? backward<S, 2, uint64_t, false>(c, s) : forward<S, 2, uint64_t, false>(c, s);
    if constexpr (sizeof(S) == 2) return BACKWARD ? backward<S, 2, uint32_t, true>(c, s) : forward<S, 2, uint32_t, true>(c, s);
    else return BACKWARD ? backward<S, 2, uint32_t, false>(c, s) : forward<S, 2, uint32_t, false>(c, s);
}

}  // namespace

size_t scan_workspace_bytes(int64_t B, int64_t T, int64_t D) {
    const Split p = split(B, T, D);
    return p.segments > 1 ? 2 * up256(sizeof(float) * (size_t)p.segments * (size_t)(B * D)) : 0;
}

hipError_t launch_scan(const ScanCall& c, hipStream_t s) {
    if (c.dtype == kF32) return choose<float, false>(c, s);
    if (c.dtype == kF16) return choose<_Float16, false>(c, s);
    return choose<__bf16, false>(c, s);
}

hipError_t launch_scan_backward(const ScanCall& c, hipStream_t s) {
    if (c.dtype == kF32) return choose<float, true>(c, s);
    if (c.dtype == kF16) return choose<_Float16, true>(c, s);
    return choose<__bf16, true>(c, s);
}

}  // namespace cc
