// Device-side helpers of the order-model kernels (cc_embed.hip, cc_scan.hip, cc_token.hip): element types, vectors of
// elements at any element's address, reductions over groups of lanes.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ccm {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr double kLn2 = 0.693147180559945309417;

// Element types in memory; every computation is in float.  Conversion to 16 bits rounds to nearest, ties to even.
__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(_Float16 v) { return (float)v; }
__device__ __forceinline__ float widen(__bf16 v) { return __builtin_bit_cast(float, (uint32_t)__builtin_bit_cast(uint16_t, v) << 16); }
template <class S>
__device__ __forceinline__ S narrow(float v) { return (S)v; }

// N elements that lie together, held as they lie in memory: pairs of 16-bit elements stay in one register, taken apart where they are
// used.  Their address need only be a multiple of the element's size: gfx950 loads and stores 16 bytes from any such address
// in one instruction, so a row of odd length needs no peeling.
template <class S, int N, bool PAIRS = sizeof(S) == 2 && N % 2 == 0>
struct Pack {
    S v[N];
    __device__ __forceinline__ float get(int i) const { return widen(v[i]); }
    __device__ __forceinline__ S element(int i) const { return v[i]; }
    __device__ __forceinline__ static Pack from(const float f[N]) {
        Pack r;
#pragma unroll
        for (int i = 0; i < N; ++i) r.v[i] = narrow<S>(f[i]);
        return r;
    }
};
template <class S, int N>
struct Pack<S, N, true> {
    uint32_t w[N / 2];
    __device__ __forceinline__ S element(int i) const { return __builtin_bit_cast(S, (uint16_t)(i & 1 ? w[i / 2] >> 16 : w[i / 2])); }
    __device__ __forceinline__ float get(int i) const {
        if constexpr (__is_same(S, __bf16)) return __builtin_bit_cast(float, i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
        return widen(element(i));
    }
    __device__ __forceinline__ static Pack from(const float f[N]) {
        typedef S Two __attribute__((ext_vector_type(2)));
        Pack r;
#pragma unroll
        for (int i = 0; i < N / 2; ++i) r.w[i] = __builtin_bit_cast(uint32_t, Two{narrow<S>(f[2 * i]), narrow<S>(f[2 * i + 1])});
        return r;
    }
};
template <int N, class S>
__device__ __forceinline__ Pack<S, N> load_pack(const S* p) {
    Pack<S, N> r;
    __builtin_memcpy(&r, p, sizeof(r));
    return r;
}
template <int N, class S>
__device__ __forceinline__ void store_pack(S* p, const Pack<S, N>& r) { __builtin_memcpy(p, &r, sizeof(r)); }

// The largest of N elements (a NaN among them is passed over).
template <class S, int N>
__device__ __forceinline__ float largest(const Pack<S, N>& p) {
    if constexpr (__is_same(S, _Float16) && N % 2 == 0) {
        typedef _Float16 Two __attribute__((ext_vector_type(2)));
        Two m = __builtin_bit_cast(Two, p.w[0]);
#pragma unroll
        for (int i = 1; i < N / 2; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(Two, p.w[i]));
        return fmaxf((float)m[0], (float)m[1]);
    } else {
        float m = p.get(0);
#pragma unroll
        for (int i = 1; i < N; ++i) m = fmaxf(m, p.get(i));
        return m;
    }
}

// Makes the compiler take a value as new, so that nothing computed from it before is kept.
template <class S, int N>
__device__ __forceinline__ void forget(Pack<S, N>& p) {
    if constexpr (sizeof(p) % 4 == 0) {
        uint32_t w[sizeof(p) / 4];
        __builtin_memcpy(w, &p, sizeof(p));
#pragma unroll
        for (unsigned k = 0; k < sizeof(p) / 4; ++k) asm("" : "+v"(w[k]));
        __builtin_memcpy(&p, w, sizeof(p));
    }
}

__device__ __forceinline__ float exp_fast(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

// The value (float or int) of the lane that differs in one bit of its number (1, 2, 4, 8), once the lanes below that bit agree.
template <int BIT, class V>
__device__ __forceinline__ V other_lane(V v) {
    constexpr int ctrl = BIT == 1 ? 0xB1 : BIT == 2 ? 0x4E : BIT == 4 ? 0x141 : 0x140;   // quad_perm, half mirror, mirror
    return __builtin_bit_cast(V, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), ctrl, 0xf, 0xf, true));
}
struct MaxOp {
    __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
};
struct SumOp {
    template <class V>
    __device__ __forceinline__ V operator()(V a, V b) const { return a + b; }
};
// Over each aligned group of G lanes; every lane ends with its group's result.  All 64 lanes are active.
template <int G, class V, class Op>
__device__ __forceinline__ V group_reduce(V v, Op op) {
    if constexpr (G > 1) v = op(v, other_lane<1>(v));
    if constexpr (G > 2) v = op(v, other_lane<2>(v));
    if constexpr (G > 4) v = op(v, other_lane<4>(v));
    if constexpr (G > 8) v = op(v, other_lane<8>(v));
    if constexpr (G > 16) {
        // exchanges the odd rows of 16 lanes of one register with the even rows of the other
        const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false);
        v = op(__builtin_bit_cast(V, (unsigned)r[0]), __builtin_bit_cast(V, (unsigned)r[1]));
    }
    if constexpr (G > 32) {
        const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false);
        v = op(__builtin_bit_cast(V, (unsigned)r[0]), __builtin_bit_cast(V, (unsigned)r[1]));
    }
    return v;
}
template <int G>
__device__ __forceinline__ float group_max(float v) { return group_reduce<G>(v, MaxOp()); }
template <int G, class V>
__device__ __forceinline__ V group_sum(V v) { return group_reduce<G>(v, SumOp()); }

__device__ __forceinline__ double wave_sum_f64(double v) {
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) v += __shfl_xor(v, m, 64);
    return v;
}
// Between accesses of a wavefront's lanes to each other's words of LDS: the hardware keeps their order, the compiler has to.
__device__ __forceinline__ void wave_order() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

}  // namespace ccm
