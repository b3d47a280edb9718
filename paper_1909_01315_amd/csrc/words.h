// Rows in words and sums over neighbouring lanes, shared by the attention
// kernels (dot products over edges, norms and rotations of their operands).
#pragma once

#include "device.h"

namespace gnnk {

// bf16 rows stay in their packed words until a column is needed: dot products
// of two bf16 rows take a pair of columns an instruction (v_dot2_f32_bf16: the
// exact products and the sum so far, off by at most 2.4 units of the last
// place of their sizes' sum; bf16 numbers below 2^-126 count as 0), which
// spares the widening and half the multiplications
struct bf16_pair_t {
    uint16_t x;
};

// vectors of words: VEC values of fp32, VEC / 2 pairs of bf16
template <int VEC>
struct IO<bf16_pair_t, VEC> {
    static __device__ __forceinline__ void load(const bf16_pair_t* p, float* w) {
        if constexpr (VEC == 8) {
            const u4_h x = *reinterpret_cast<const u4_h*>(p);
            w[0] = __uint_as_float(x.x); w[1] = __uint_as_float(x.y);
            w[2] = __uint_as_float(x.z); w[3] = __uint_as_float(x.w);
        } else if constexpr (VEC == 4) {
            const u2_h x = *reinterpret_cast<const u2_h*>(p);
            w[0] = __uint_as_float(x.x); w[1] = __uint_as_float(x.y);
        } else if constexpr (VEC == 2) {
            w[0] = __uint_as_float(*reinterpret_cast<const u1_h*>(p));
        } else {
            w[0] = __uint_as_float((uint32_t)p->x);
        }
    }
};

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ bf16x2 pair(float w) { return __builtin_bit_cast(bf16x2, w); }

// rows of T in words
template <typename T, int VEC>
struct Words {
    using type = float;
    static constexpr int N = VEC;
    static constexpr bool PAIRS = false;
    static __device__ __forceinline__ float at(const float* w, int i) { return w[i]; }
};
template <int VEC>
struct Words<bf16_t, VEC> {
    using type = bf16_pair_t;
    static constexpr int N = (VEC + 1) / 2;
    static constexpr bool PAIRS = true;
    static __device__ __forceinline__ float at(const float* w, int i) {
        const uint32_t x = __float_as_uint(w[i / 2]);
        return (i & 1) ? bf_hi(x) : bf_lo(x);
    }
};

template <int CTRL>
__device__ __forceinline__ float dpp_f(float x) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xF, 0xF, true));
}
constexpr int DPP_HALF_MIRROR = 0x141, DPP_MIRROR = 0x140;

// sums over the aligned run of `red` lanes (a power of two) that holds the
// lane, of N values at once; every lane gets the totals
template <int N>
__device__ __forceinline__ void run_totals(float* v, int red) {
    if (red >= 2)
#pragma unroll
        for (int u = 0; u < N; ++u) v[u] += dpp_f<DPP_QUAD_1032>(v[u]);
    if (red >= 4)
#pragma unroll
        for (int u = 0; u < N; ++u) v[u] += dpp_f<DPP_QUAD_2301>(v[u]);
    if (red >= 8)
#pragma unroll
        for (int u = 0; u < N; ++u) v[u] += dpp_f<DPP_HALF_MIRROR>(v[u]);
    if (red >= 16)
#pragma unroll
        for (int u = 0; u < N; ++u) v[u] += dpp_f<DPP_MIRROR>(v[u]);
    if (red >= 32)
#pragma unroll
        for (int u = 0; u < N; ++u) v[u] += __shfl_xor(v[u], 16, WAVE);
    if (red >= 64)
#pragma unroll
        for (int u = 0; u < N; ++u) v[u] += __shfl_xor(v[u], 32, WAVE);
}

// the value of lane X of each quad
template <int X>
__device__ __forceinline__ int32_t quad_lane(int32_t x) {
    return __builtin_amdgcn_update_dpp(0, x, X * 0x55, 0xF, 0xF, true);
}
template <int X>
__device__ __forceinline__ float quad_lane(float x) {
    return dpp_f<X * 0x55>(x);
}

// Sums over the aligned run of `red` >= 4 lanes of four groups of N values
// v[g N + n]: lane g of each quad gets the totals of group g (out[n]), a
// quarter of what every lane would get.
constexpr int DPP_QUAD_3210 = 0x1B;  // lane i reads lane 3 - i of its quad
template <int N>
__device__ __forceinline__ void quad_totals(const float* v, int red, float* out) {
    const bool b0 = __lane_id() & 1, b1 = __lane_id() & 2;
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const float v0 = v[n], v1 = v[N + n], v2 = v[2 * N + n], v3 = v[3 * N + n];
        const float lo = (b0 ? v1 : v0) + dpp_f<DPP_QUAD_1032>(b0 ? v0 : v1);  // groups 0 and 1 in lanes 0 and 1
        const float hi = (b0 ? v3 : v2) + dpp_f<DPP_QUAD_1032>(b0 ? v2 : v3);
        out[n] = (b1 ? hi : lo) + dpp_f<DPP_QUAD_2301>(b1 ? lo : hi);
    }
    // the lanes 4, 8, 16 and 32 apart (mirrors reverse a run: reversed twice)
    if (red >= 8)
#pragma unroll
        for (int n = 0; n < N; ++n) out[n] += dpp_f<DPP_HALF_MIRROR>(dpp_f<DPP_QUAD_3210>(out[n]));
    if (red >= 16)
#pragma unroll
        for (int n = 0; n < N; ++n) out[n] += dpp_f<DPP_MIRROR>(dpp_f<DPP_HALF_MIRROR>(out[n]));
    if (red >= 32)
#pragma unroll
        for (int n = 0; n < N; ++n) out[n] += __shfl_xor(out[n], 16, WAVE);
    if (red >= 64)
#pragma unroll
        for (int n = 0; n < N; ++n) out[n] += __shfl_xor(out[n], 32, WAVE);
}

}  // namespace gnnk
