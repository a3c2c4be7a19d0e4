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

#include "cc_internal.h"
#include "cc_model.h"

namespace cc {
namespace {

using namespace ccm;

constexpr int kThreads = 256, L = kScanChunk;

// keep and take from e = exp(-|gate|): 1 / (1 + e) and e / (1 + e), neither of them as one minus the other, so that both keep
// their relative precision.  The smaller one is held as two factors, each with half of the exponential's argument: what it
// multiplies is then rounded once where the product is subnormal, and the exponential instruction, which gives 0 for
// subnormal results, is never asked for one that matters.
struct Gates {
    float keep1, keep2, take1, take2;
    __device__ __forceinline__ explicit Gates(float g) {
        const float half = exp_fast(-0.5f * fabsf(g)), large = __builtin_amdgcn_rcpf(fmaf(half, half, 1.0f)), small2 = half * large;
        keep1 = g >= 0.0f ? 1.0f : half;
        keep2 = g >= 0.0f ? large : small2;
        take1 = g >= 0.0f ? half : 1.0f;
        take2 = g >= 0.0f ? small2 : large;
    }
    __device__ __forceinline__ float keep(float v) const { return v * keep1 * keep2; }
    __device__ __forceinline__ float take(float v) const { return v * take1 * take2; }
    __device__ __forceinline__ float step(float h, float x) const { return fmaf(h * keep1, keep2, take(x)); }
};

struct Args {
    const void *x, *gate, *h_in;      // h_in: gradient of h (backward)
    void *h, *grad_x, *grad_gate;
    int64_t xb, xt, gb, gt, hb, ht, dxb, dxt, dgb, dgt;
    int64_t B, T, D;
    int pairs;                        // threads per sequence: two channels each
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

// What a thread owns.
struct Lane {
    int64_t b, first, n;              // sequence; first channel's place in [B, D]; positions that count
    int d, have;                      // first channel, 1 or 2 of them
    bool real;
    __device__ __forceinline__ Lane(const Args& a) {
        const int64_t id = (int64_t)blockIdx.x * kThreads + threadIdx.x;
        b = id / a.pairs;
        real = b < a.B;
        d = 2 * (int)(id - b * a.pairs);
        have = min(2, (int)(a.D - d));
        first = b * a.D + d;
        n = a.T;
        if (real && a.lengths) n = min(a.T, (int64_t)max(a.lengths[b], 0));
    }
};

__device__ __forceinline__ void read2(const float* p, int have, float v[2]) {
    v[0] = p[0];
    v[1] = have > 1 ? p[1] : 0.0f;
}
__device__ __forceinline__ void write2(float* p, int have, const float v[2]) {
    p[0] = v[0];
    if (have > 1) p[1] = v[1];
}
template <class S>
__device__ __forceinline__ void write2(S* p, int have, float v0, float v1) {
    Pack<S, 2> r;
    r.v[0] = narrow<S>(v0);
    r.v[1] = narrow<S>(v1);
    store_some<2>(p, r, have);
}

// Forward walk.  SUMMARY: only the segment's product of keeps and what it adds; the last segment needs none.
template <class S, bool SUMMARY>
__global__ __launch_bounds__(kThreads) void scan_kernel(Args a) {
    const Lane l(a);
    if (!l.real) return;
    const int seg = blockIdx.y;
    const int64_t from = seg * a.segment, to = min(a.T, from + a.segment);
    const S* const x = (const S*)a.x + l.b * a.xb + l.d;
    const S* const g = (const S*)a.gate + l.b * a.gb + l.d;
    S* const out = SUMMARY ? nullptr : (S*)a.h + l.b * a.hb + l.d;
    const int64_t row = a.B * a.D;
    float h[2] = {0.0f, 0.0f}, product[2] = {1.0f, 1.0f};
    if (!SUMMARY) {
        if (a.starts) read2(a.starts + seg * row + l.first, l.have, h);
        else if (a.h0) read2(a.h0 + l.first, l.have, h);
    }
    for (int64_t t0 = from; t0 < to; t0 += L) {
        if (!SUMMARY && a.states) write2(a.states + (l.b * a.chunks + t0 / L) * a.D + l.d, l.have, h);
        const int count = (int)min((int64_t)L, to - t0), inside = (int)min((int64_t)L, l.n - t0);
        Pack<S, 2> xs[L], gs[L];
        if (inside >= L) {
#pragma unroll
            for (int i = 0; i < L; ++i) {
                xs[i] = load_some<2>(x + (t0 + i) * a.xt, l.have);
                gs[i] = load_some<2>(g + (t0 + i) * a.gt, l.have);
            }
        } else {
#pragma unroll
            for (int i = 0; i < L; ++i)
                if (i < inside) {
                    xs[i] = load_some<2>(x + (t0 + i) * a.xt, l.have);
                    gs[i] = load_some<2>(g + (t0 + i) * a.gt, l.have);
                }
        }
#pragma unroll
        for (int i = 0; i < L; ++i) {
            if (i < inside) {
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const Gates gate(widen(gs[i].v[c]));
                    h[c] = gate.step(h[c], widen(xs[i].v[c]));
                    if (SUMMARY) product[c] = gate.keep(product[c]);
                }
            }
            if (!SUMMARY && i < count) {
                const bool in = i < inside;
                write2(out + (t0 + i) * a.ht, l.have, in ? h[0] : 0.0f, in ? h[1] : 0.0f);
            }
        }
    }
    if (SUMMARY) {
        write2(a.products + seg * row + l.first, l.have, product);
        write2(a.sums + seg * row + l.first, l.have, h);
    } else if (seg == a.segments - 1 && a.last) {
        write2(a.last + l.first, l.have, h);
    }
}

// Backward walk.  SUMMARY: only the segment's product of keeps and what it sends back; the first segment needs none.
template <class S, bool SUMMARY>
__global__ __launch_bounds__(kThreads) void scan_backward_kernel(Args a) {
    const Lane l(a);
    if (!l.real) return;
    const int seg = SUMMARY ? blockIdx.y + 1 : blockIdx.y;
    const int64_t from = seg * a.segment, to = min(a.T, from + a.segment);
    const S* const x = (const S*)a.x + l.b * a.xb + l.d;
    const S* const g = (const S*)a.gate + l.b * a.gb + l.d;
    const S* const dh = (const S*)a.h_in + l.b * a.hb + l.d;
    const int64_t row = a.B * a.D;
    float f[2] = {0.0f, 0.0f}, product[2] = {1.0f, 1.0f};
    if (!SUMMARY) {
        if (a.starts) read2(a.starts + seg * row + l.first, l.have, f);
        else if (a.last_grad) read2(a.last_grad + l.first, l.have, f);
    }
    for (int64_t t0 = to > from ? from + (to - from - 1) / L * L : from - L; t0 >= from; t0 -= L) {
        const int count = (int)min((int64_t)L, to - t0), inside = (int)min((int64_t)L, l.n - t0);
        Pack<S, 2> xs[L], gs[L], ds[L];
#pragma unroll
        for (int i = 0; i < L; ++i)
            if (i < inside) {
                gs[i] = load_some<2>(g + (t0 + i) * a.gt, l.have);
                ds[i] = load_some<2>(dh + (t0 + i) * a.ht, l.have);
                if (!SUMMARY) xs[i] = load_some<2>(x + (t0 + i) * a.xt, l.have);
            }
        float before[L][2], h[2];
        if (!SUMMARY) {
            read2(a.states + (l.b * a.chunks + t0 / L) * a.D + l.d, l.have, h);
#pragma unroll
            for (int i = 0; i < L; ++i)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    before[i][c] = h[c];
                    if (i < inside) h[c] = Gates(widen(gs[i].v[c])).step(h[c], widen(xs[i].v[c]));
                }
        }
#pragma unroll
        for (int i = L - 1; i >= 0; --i) {
            float dx[2] = {0.0f, 0.0f}, dg[2] = {0.0f, 0.0f};
            if (i < inside) {
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const Gates gate(widen(gs[i].v[c]));
                    const float lambda = widen(ds[i].v[c]) + f[c];
                    f[c] = gate.keep(lambda);
                    if (SUMMARY) {
                        product[c] = gate.keep(product[c]);
                    } else {
                        dx[c] = gate.take(lambda);
                        dg[c] = gate.keep(gate.take(lambda * (before[i][c] - widen(xs[i].v[c]))));
                    }
                }
            }
            if (!SUMMARY && i < count) {
                write2((S*)a.grad_x + l.b * a.dxb + (t0 + i) * a.dxt + l.d, l.have, dx[0], dx[1]);
                write2((S*)a.grad_gate + l.b * a.dgb + (t0 + i) * a.dgt + l.d, l.have, dg[0], dg[1]);
            }
        }
    }
    if (SUMMARY) {
        write2(a.products + seg * row + l.first, l.have, product);
        write2(a.sums + seg * row + l.first, l.have, f);
    } else if (seg == 0 && a.grad_h0) {
        write2(a.grad_h0 + l.first, l.have, f);
    }
}

// Chains the segments: what each starts from, left in the place of its product.  Forward from the first segment, backward
// from the last.
template <bool BACKWARD>
__global__ __launch_bounds__(kThreads) void scan_chain_kernel(float* products, const float* sums, const float* first, int segments, int64_t row) {
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (i >= row) return;
    float h = first ? first[i] : 0.0f;
#pragma unroll 8
    for (int s = 0; s < segments; ++s) {
        const int64_t at = (BACKWARD ? segments - 1 - s : s) * row + i;
        const float p = s + 1 < segments ? products[at] : 0.0f, q = s + 1 < segments ? sums[at] : 0.0f;   // the last is not summed up
        products[at] = h;
        h = fmaf(p, h, q);
    }
}

// Segments for B sequences of T positions and D channels: as many as make 2^17 threads, of 64 positions at least.
struct Split {
    int64_t segment;
    int segments;
};
Split split(int64_t B, int64_t T, int64_t D) {
    const int64_t threads = B * ((D + 1) / 2);
    int64_t want = threads > 0 ? ((1 << 17) + threads - 1) / threads : 1;
    if (want > T / 64) want = T / 64;
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

Args arguments(const ScanCall& c, const Split& s) {
    Args a = {};
    a.x = c.x.p; a.xb = c.x.b; a.xt = c.x.t;
    a.gate = c.gate.p; a.gb = c.gate.b; a.gt = c.gate.t;
    a.hb = c.h.b; a.ht = c.h.t;
    a.B = c.B; a.T = c.T; a.D = c.D;
    a.pairs = (int)((c.D + 1) / 2);
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

template <class S>
hipError_t forward(const ScanCall& c, hipStream_t s) {
    const Split p = split(c.B, c.T, c.D);
    Args a = arguments(c, p);
    a.h = c.h.p;
    a.h0 = c.h0;
    a.last = c.last;
    const unsigned blocks = (unsigned)((c.B * a.pairs + kThreads - 1) / kThreads);
    const int64_t row = c.B * c.D;
    if (p.segments > 1) {
        hipLaunchKernelGGL((scan_kernel<S, true>), dim3(blocks, p.segments - 1), dim3(kThreads), 0, s, a);
        hipLaunchKernelGGL((scan_chain_kernel<false>), dim3((unsigned)((row + kThreads - 1) / kThreads)), dim3(kThreads), 0, s, a.products,
                           a.sums, c.h0, p.segments, row);
    }
    hipLaunchKernelGGL((scan_kernel<S, false>), dim3(blocks, p.segments), dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

template <class S>
hipError_t backward(const ScanCall& c, hipStream_t s) {
    const Split p = split(c.B, c.T, c.D);
    Args a = arguments(c, p);
    a.h_in = c.h.p;
    a.last_grad = c.last;
    a.grad_x = c.grad_x.p; a.dxb = c.grad_x.b; a.dxt = c.grad_x.t;
    a.grad_gate = c.grad_gate.p; a.dgb = c.grad_gate.b; a.dgt = c.grad_gate.t;
    a.grad_h0 = c.grad_h0;
    const unsigned blocks = (unsigned)((c.B * a.pairs + kThreads - 1) / kThreads);
    const int64_t row = c.B * c.D;
    if (p.segments > 1) {
        hipLaunchKernelGGL((scan_backward_kernel<S, true>), dim3(blocks, p.segments - 1), dim3(kThreads), 0, s, a);
        hipLaunchKernelGGL((scan_chain_kernel<true>), dim3((unsigned)((row + kThreads - 1) / kThreads)), dim3(kThreads), 0, s, a.products,
                           a.sums, (const float*)c.last, p.segments, row);
    }
    hipLaunchKernelGGL((scan_backward_kernel<S, false>), dim3(blocks, p.segments), dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

}  // namespace

size_t scan_workspace_bytes(int64_t B, int64_t T, int64_t D) {
    const Split p = split(B, T, D);
    return p.segments > 1 ? 2 * up256(sizeof(float) * (size_t)p.segments * (size_t)(B * D)) : 0;
}

hipError_t launch_scan(const ScanCall& c, hipStream_t s) {
    if (c.dtype == kF32) return forward<float>(c, s);
    if (c.dtype == kF16) return forward<_Float16>(c, s);
    return forward<__bf16>(c, s);
}

hipError_t launch_scan_backward(const ScanCall& c, hipStream_t s) {
    if (c.dtype == kF32) return backward<float>(c, s);
    if (c.dtype == kF16) return backward<_Float16>(c, s);
    return backward<__bf16>(c, s);
}

}  // namespace cc
