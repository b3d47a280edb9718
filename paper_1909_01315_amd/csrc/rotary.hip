// Positions and norms of the attention's queries and keys: node_rotary turns
// pairs of columns of every head by angles made of the node's positions on
// several axes, node_norm_rotary divides each head by its root mean square
// first (with a weight per column), and the backward of the latter.
//
//   theta[n, i] = pos[n, axis(i)] * freq[i]
//   (a, b) -> (a cos theta - b sin theta, a sin theta + b cos theta)
//
// A pure stream: every head is read once and written once (backward: read
// twice, written once).  The angles depend on the row alone, so a block first
// computes the cosines and sines of its tile of rows into LDS, one per row
// and pair whatever the number of heads, and its lane groups then take one
// head each, neighbouring groups neighbouring heads, so that a wavefront's
// loads are contiguous.  A lane holds V pairs (2V columns): of the halves
// layout V columns of either half, of the interleaved one 2V columns side by
// side; columns past the last pair pass as they are, 2V a lane.
//
// Angles are products in fp64, reduced to turns there (a position of 10^6 at
// frequency 1 keeps its angle to 10^-10), and their sines and cosines fp32.
// Sums over a head (at most 2,048 columns) are fp32, weight gradients, sums
// over all rows, fp64.
#include "device.h"

namespace gnnk {

namespace {

constexpr double INV_2PI = 0.15915494309189533577;

// sum over the aligned run of `red` lanes (a power of two) that holds the
// lane; every lane gets the total.  All lanes must take part.
template <int CTRL>
__device__ __forceinline__ float dpp_f(float x) {
    return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), CTRL, 0xF, 0xF, false));
}
constexpr int DPP_HALF_MIRROR = 0x141, DPP_MIRROR = 0x140;
__device__ __forceinline__ float run_total(float v, int red) {
    if (red >= 2) v += dpp_f<DPP_QUAD_1032>(v);
    if (red >= 4) v += dpp_f<DPP_QUAD_2301>(v);
    if (red >= 8) v += dpp_f<DPP_HALF_MIRROR>(v);  // (the lanes of a quad hold one value)
    if (red >= 16) v += dpp_f<DPP_MIRROR>(v);
    if (red >= 32) v += __shfl_xor(v, 16, WAVE);
    if (red >= 64) v += __shfl_xor(v, 32, WAVE);
    return v;
}

enum : int { TURN = 0, NORM = 1, NORM_BWD = 2 };

// IL: the pairs are columns (2i, 2i + 1), else (i, i + P)
template <typename T, int V, bool IL, int MODE>
__global__ __launch_bounds__(256) void node_rotary_kernel(RotaryArgs A) {
    extern __shared__ float lds[];
    const bool second = blockIdx.x >= (unsigned)A.side[0].blocks;
    const RotarySide& S = A.side[second ? 1 : 0];
    int b = (int)blockIdx.x - (second ? A.side[0].blocks : 0);
    const int ch = b % A.nchunk;
    b /= A.nchunk;
    const int hb = b % S.hblocks, rb = b / S.hblocks;
    const int P = A.P, RT = S.tile_rows, tid = threadIdx.x;
    const int lig = tid & (A.L - 1), gid = tid >> A.log2L;
    const int rr = gid / S.HB, hl = gid - rr * S.HB, h = hb * S.HB + hl;
    const bool group_ok = rr < S.RB && h < S.H;
    const int vec = ch * A.L + lig;
    const bool act = group_ok && vec < A.NV;
    const int s0 = act ? vec * V : 0;          // first pair of the lane
    const bool turn = s0 < P;
    const int c0 = IL || !turn ? 2 * s0 : s0;
    const int c1 = IL || !turn ? 2 * s0 + V : P + s0;
    const bool has1 = V > 1 || c1 < A.F;       // (an odd width's last column has no partner)
    const int64_t head = (int64_t)(group_ok ? h : 0) * A.F;
    float* const cosv = lds;
    float* const sinv = lds + RT * P;

    float w[2 * V];
    if constexpr (MODE != TURN) {
#pragma unroll
        for (int i = 0; i < 2 * V; ++i) w[i] = 1.0f;
        if (S.w) {
            const T* p = reinterpret_cast<const T*>(S.w) + (S.w_per_head ? head : 0);
            IO<T, V>::load(p + c0, w);
            if (has1) IO<T, V>::load(p + c1, w + V);
        }
    }
    double dw[MODE == NORM_BWD ? 2 * V : 1];
#pragma unroll
    for (int i = 0; i < (MODE == NORM_BWD ? 2 * V : 1); ++i) dw[i] = 0.0;

    // 2V columns of a row's head, zeros for a lane outside it
    auto load = [&](const void* base, int64_t stride, int64_t n, bool ok, int at0, int at1, bool with1, float* t) {
#pragma unroll
        for (int i = 0; i < 2 * V; ++i) t[i] = 0.0f;
        if (ok) {
            const T* p = reinterpret_cast<const T*>(base) + n * stride + head;
            IO<T, V>::load(p + at0, t);
            if (with1) IO<T, V>::load(p + at1, t + V);
        }
    };
    auto rotate = [&](float* t, int r, float sgn) {
        if (!turn) return;
        float c[V], s[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            c[i] = cosv[r * P + s0 + i];
            s[i] = sgn * sinv[r * P + s0 + i];
        }
#pragma unroll
        for (int i = 0; i < V; ++i) {
            float& x = t[IL ? 2 * i : i];
            float& y = t[IL ? 2 * i + 1 : V + i];
            const float xr = x * c[i] - y * s[i], yr = x * s[i] + y * c[i];
            x = xr;
            y = yr;
        }
    };

    const int64_t tiles = (S.n + RT - 1) / RT;
    for (int64_t tile = rb; tile < tiles; tile += S.row_blocks) {
        const int64_t n0 = tile * RT;
        if (P > 0) {
            __syncthreads();  // (the tile before may still be read)
            for (int i = tid; i < RT * P; i += 256) {
                const int r = i / P, p = i - r * P;
                if (n0 + r < S.n) {
                    int axis = 0, end = A.pairs[0];
                    while (p >= end && axis < 3) end += A.pairs[++axis];
                    const int64_t at = (n0 + r) * S.pos_stride + axis;
                    const double x = S.pos_i32 ? (double)reinterpret_cast<const int32_t*>(S.pos)[at]
                                               : (double)reinterpret_cast<const float*>(S.pos)[at];
                    double turns = x * (double)S.freq[p] * INV_2PI;
                    turns -= rint(turns);
                    float sn, cs;
                    sincospif((float)(2.0 * turns), &sn, &cs);
                    cosv[i] = cs;
                    sinv[i] = sn;
                }
            }
            __syncthreads();
        }
        for (int r0 = 0; r0 < RT; r0 += S.RB) {
            const int r = r0 + rr;
            const int64_t n = n0 + r;
            const bool row_ok = group_ok && r < RT && n < S.n;
            const bool ok = act && row_ok;
            float t[2 * V];
            load(S.x, S.x_stride, n, ok, c0, c1, has1, t);
            if constexpr (MODE == TURN) {
                if (ok) rotate(t, r, A.sign);
            } else {
                float g[2 * V];
                float ss = 0.0f, dd = 0.0f;
#pragma unroll
                for (int i = 0; i < 2 * V; ++i) ss = fmaf(t[i], t[i], ss);
                if constexpr (MODE == NORM_BWD) {
                    load(S.g, S.g_stride, n, ok, c0, c1, has1, g);
                    if (ok) rotate(g, r, -1.0f);
#pragma unroll
                    for (int i = 0; i < 2 * V; ++i) dd = fmaf(g[i] * w[i], t[i], dd);
                }
                // a head wider than one pass: the sums of its other columns
                for (int o = 1; o < A.nchunk; ++o) {
                    const int ov = ((ch + o) % A.nchunk) * A.L + lig;
                    const bool ook = row_ok && ov < A.NV;
                    const int q0 = ook ? ov * V : 0;
                    const bool ot = q0 < P;
                    const int o0 = IL || !ot ? 2 * q0 : q0, o1 = IL || !ot ? 2 * q0 + V : P + q0;
                    const bool oh = V > 1 || o1 < A.F;
                    float y[2 * V];
                    load(S.x, S.x_stride, n, ook, o0, o1, oh, y);
#pragma unroll
                    for (int i = 0; i < 2 * V; ++i) ss = fmaf(y[i], y[i], ss);
                    if constexpr (MODE == NORM_BWD) {
                        // sum of (R^-1 g) w x
                        float z[2 * V], u[2 * V];
                        load(S.g, S.g_stride, n, ook, o0, o1, oh, z);
                        if (S.w) {
                            // (the weight has one row: a stride of 0)
                            const int64_t back = S.w_per_head ? 0 : -head;
                            load(reinterpret_cast<const T*>(S.w) + back, 0, 0, ook, o0, o1, oh, u);
                        } else {
#pragma unroll
                            for (int i = 0; i < 2 * V; ++i) u[i] = 1.0f;
                        }
#pragma unroll
                        for (int i = 0; i < V; ++i) {
                            const int ia = IL ? 2 * i : i, ib = IL ? 2 * i + 1 : V + i;
                            float za = z[ia], zb = z[ib];
                            if (ook && ot) {
                                const float c = cosv[r * P + q0 + i], s = sinv[r * P + q0 + i];
                                za = z[ia] * c + z[ib] * s;
                                zb = z[ib] * c - z[ia] * s;
                            }
                            dd = fmaf(za * u[ia], y[ia], dd);
                            dd = fmaf(zb * u[ib], y[ib], dd);
                        }
                    }
                }
                ss = run_total(ss, A.L);
                const float rn = 1.0f / sqrtf(ss * A.inv_F + A.eps);
                if constexpr (MODE == NORM) {
#pragma unroll
                    for (int i = 0; i < 2 * V; ++i) t[i] = t[i] * rn * w[i];
                    if (ok) rotate(t, r, 1.0f);
                } else {
                    dd = run_total(dd, A.L);
                    const float k = rn * rn * dd * A.inv_F;
#pragma unroll
                    for (int i = 0; i < 2 * V; ++i) {
                        // (a group without a row adds nothing: there rn may be infinite)
                        if (ok) dw[i] += (double)(g[i] * t[i] * rn);
                        t[i] = rn * (g[i] * w[i] - t[i] * k);
                    }
                }
            }
            if (ok && S.out) {
                T* p = reinterpret_cast<T*>(S.out) + n * S.out_stride + head;
                IO<T, V>::store(p + c0, t);
                if (has1) IO<T, V>::store(p + c1, t + V);
            }
        }
    }
    if constexpr (MODE == NORM_BWD) {
        if (!S.dw_part) return;
        // the block's sums: over its groups of one head, or of all heads, in
        // the order of the groups
        double* red = reinterpret_cast<double*>(lds);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 2 * V; ++i) red[i * 256 + tid] = act ? dw[i] : 0.0;
        __syncthreads();
        const int per = A.L * 2 * V;  // sums of one head
        const int heads = S.w_per_head ? S.HB : 1;
        for (int q = tid; q < per * heads; q += 256) {
            const int hq = q / per, x = q - hq * per;
            const int i = x / A.L, l = x - i * A.L;
            const int v = ch * A.L + l;
            if (v >= A.NV || hb * S.HB + hq >= S.H) continue;
            double sum = 0.0;
            if (S.w_per_head) {
                for (int k = 0; k < S.RB; ++k) sum += red[i * 256 + ((k * S.HB + hq) << A.log2L) + l];
            } else {
                for (int k = 0; k < S.RB * S.HB; ++k) sum += red[i * 256 + (k << A.log2L) + l];
            }
            const int sl = v * V;
            const bool tn = sl < P;
            const int d0 = IL || !tn ? 2 * sl : sl, d1 = IL || !tn ? 2 * sl + V : P + sl;
            const int col = i < V ? d0 + i : d1 + i - V;
            if (col >= A.F) continue;
            const int64_t part = S.w_per_head ? rb : (int64_t)rb * S.hblocks + hb;
            S.dw_part[part * S.dw_cols + (S.w_per_head ? (int64_t)(hb * S.HB + hq) * A.F : 0) + col] = sum;
        }
    }
}

// the weight gradients: the blocks' sums, 32 columns a workgroup, 32 runs of
// blocks side by side, each in order
template <typename T>
__global__ __launch_bounds__(1024) void node_rotary_dw_kernel(RotaryArgs A) {
    const RotarySide& S = A.side[blockIdx.y];
    if (!S.dw_part) return;
    __shared__ double red[32][33];
    const int c = threadIdx.x & 31, run = threadIdx.x >> 5;
    const int64_t col = (int64_t)blockIdx.x * 32 + c;
    const int64_t per = (S.dw_parts + 31) / 32;
    double sum = 0.0;
    if (col < S.dw_cols) {
        const int64_t end = (run + 1) * per < S.dw_parts ? (run + 1) * per : S.dw_parts;
        for (int64_t p = run * per; p < end; ++p) sum += S.dw_part[p * S.dw_cols + col];
    }
    red[run][c] = sum;
    __syncthreads();
    if (run == 0 && col < S.dw_cols) {
        for (int k = 1; k < 32; ++k) sum += red[k][c];
        IO<T, 1>::store1(reinterpret_cast<T*>(S.dw) + col, (float)sum);
    }
}

template <typename T, int V, int MODE>
void launch_v(const RotaryArgs& a, size_t lds, hipStream_t s) {
    const dim3 grid((unsigned)(a.side[0].blocks + a.side[1].blocks)), block(256);
    if (a.interleaved) hipLaunchKernelGGL((node_rotary_kernel<T, V, true, MODE>), grid, block, lds, s, a);
    else hipLaunchKernelGGL((node_rotary_kernel<T, V, false, MODE>), grid, block, lds, s, a);
}

template <typename T, int MODE>
void launch_mode(const RotaryArgs& a, int vec, size_t lds, hipStream_t s) {
    if constexpr (sizeof(T) == 2) {
        GNNK_VEC_DISPATCH_BF16(vec, launch_v<T, V, MODE>(a, lds, s))
    } else {
        GNNK_VEC_DISPATCH_F32(vec, launch_v<T, V, MODE>(a, lds, s))
    }
}

template <typename T>
void launch_t(const RotaryArgs& a, int vec, int mode, size_t lds, hipStream_t s) {
    if (mode == TURN) launch_mode<T, TURN>(a, vec, lds, s);
    else if (mode == NORM) launch_mode<T, NORM>(a, vec, lds, s);
    else launch_mode<T, NORM_BWD>(a, vec, lds, s);
    if (mode == NORM_BWD && (a.side[0].dw_part || a.side[1].dw_part)) {
        const int64_t c0 = a.side[0].dw_part ? a.side[0].dw_cols : 0, c1 = a.side[1].dw_part ? a.side[1].dw_cols : 0;
        const dim3 grid((unsigned)(((c0 > c1 ? c0 : c1) + 31) / 32), 2);
        hipLaunchKernelGGL((node_rotary_dw_kernel<T>), grid, dim3(1024), 0, s, a);
    }
}

}  // namespace

hipError_t launch_node_rotary(const RotaryArgs& a, int dtype, int vec, int mode, size_t lds, hipStream_t s) {
    if (a.side[0].blocks + a.side[1].blocks == 0) return hipSuccess;
    if (dtype == 0) launch_t<float>(a, vec, mode, lds, s);
    else launch_t<bf16_t>(a, vec, mode, lds, s);
    return hipGetLastError();
}

}  // namespace gnnk
