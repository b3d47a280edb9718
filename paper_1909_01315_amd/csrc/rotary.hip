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
// side; columns past the last pair pass as they are, 2V a lane.  Where V
// divides neither, the last lane of either kind reads whole vectors all the
// same, past its columns, and leaves the others alone.
//
// It is bound by the memory's streaming rate: 262,144 rows of 16 heads of 128
// bf16 turned in 365 us (5.9 TB/s read and written; a plain copy reaches 5.1;
// stores that bypass the caches take a third more), 8 and 8 heads of 32 fp32
// normed and turned in 184 (5.8), their backward in 309 and 5 for the blocks'
// weight gradients (5.1).  Odd widths are bound by instructions and a small
// call's latency: 20,011 rows of 6 and 3 heads of 47 bf16 23 us, backward 33
// and 4.  One row: 4 us.
//
// Angles are products in fp64, reduced to turns there (a position of 10^6 at
// frequency 1 keeps its angle to 10^-10), and their sines and cosines fp32, of
// the angle in half turns rounded to fp32 (which moves them by at most 2^-23,
// beside 2^-22 of their own).
// Sums over a head (at most 2,048 columns) are fp32, weight gradients, sums
// over all rows, fp64.
#include "words.h"

namespace gnnk {

namespace {

constexpr double INV_2PI = 0.15915494309189533577;

enum : int { TURN = 0, NORM = 1, NORM_BWD = 2 };

// the 2V columns of a lane's vector: V from c0 on and V from c1 on, of which
// the first n0 and n1 are its own
template <int V>
struct Lane {
    int s0;       // first pair
    int c0, c1;
    int n0, n1;
    bool turn;    // they are pairs, not columns after them
};
template <int V, bool IL, bool PART>
__device__ __forceinline__ Lane<V> lane_of(const RotaryArgs& A, int vec) {
    Lane<V> x;
    x.turn = vec < A.NA;
    x.s0 = x.turn ? vec * V : 0;
    x.c0 = x.turn ? (IL ? 2 * x.s0 : x.s0) : 2 * A.P + 2 * V * (vec - A.NA);
    x.c1 = x.turn && !IL ? A.P + x.s0 : x.c0 + V;
    if constexpr (PART) {
        const int m = x.turn ? 2 * (A.P - x.s0) : A.F - x.c0;  // columns from here on
        if (x.turn && !IL) {
            x.n0 = x.n1 = m < 2 * V ? m / 2 : V;
        } else {
            x.n0 = m < V ? m : V;
            x.n1 = m - V < 0 ? 0 : (m - V < V ? m - V : V);
        }
    } else {
        x.n0 = x.n1 = V;
    }
    return x;
}

// IL: the pairs are columns (2i, 2i + 1), else (i, i + P); PART: V divides
// neither the pairs nor what follows them
template <typename T, int V, bool IL, bool PART, int MODE>
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
    const Lane<V> me = lane_of<V, IL, PART>(A, act ? vec : 0);
    const int64_t head = (int64_t)(group_ok ? h : 0) * A.F;
    float* const cosv = lds;
    float* const sinv = lds + RT * P;

    auto load_w = [&](const Lane<V>& x, float* t) {
        if (S.w) {
            const T* p = reinterpret_cast<const T*>(S.w) + (S.w_per_head ? head : 0);
            if constexpr (PART) {
                // (one row, with nothing behind it that could be read past it)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    t[i] = IO<T, 1>::load1(p + x.c0 + (i < x.n0 ? i : 0));
                    t[V + i] = IO<T, 1>::load1(p + (i < x.n1 ? x.c1 + i : x.c0));
                }
            } else {
                IO<T, V>::load(p + x.c0, t);
                IO<T, V>::load(p + x.c1, t + V);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 2 * V; ++i) t[i] = 1.0f;
        }
    };
    float w[2 * V];
    if constexpr (MODE != TURN) load_w(me, w);
    double dw[MODE == NORM_BWD ? 2 * V : 1];
#pragma unroll
    for (int i = 0; i < (MODE == NORM_BWD ? 2 * V : 1); ++i) dw[i] = 0.0;

    // 2V columns of a row's head in words, zeros for a lane outside it; and
    // the words as values
    constexpr int N = Words<T, V>::N;
    auto get = [&](const void* base, int64_t stride, int64_t n, bool ok, const Lane<V>& x, float* raw) {
#pragma unroll
        for (int i = 0; i < 2 * N; ++i) raw[i] = 0.0f;
        if (ok) {
            const int64_t at = n * stride + head, room = (S.n - 1) * stride + (int64_t)S.H * A.F - at;
            const T* p = reinterpret_cast<const T*>(base) + at;
            fetch<T, V, PART>(p + x.c0, x.n0, room - x.c0, raw);
            fetch<T, V, PART>(p + x.c1, x.n1, room - x.c1, raw + N);
        }
    };
    auto values = [&](const Lane<V>& x, const float* raw, float* t) {
        widen<T, V, PART>(raw, x.n0, t);
        widen<T, V, PART>(raw + N, x.n1, t + V);
    };
    auto load = [&](const void* base, int64_t stride, int64_t n, bool ok, const Lane<V>& x, float* t) {
        float raw[2 * N];
        get(base, stride, n, ok, x, raw);
        values(x, raw, t);
    };
    auto rotate = [&](const Lane<V>& x, float* t, int r, float sgn) {
        if (!x.turn) return;
        float c[V], s[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const bool in = !PART || x.s0 + i < P;
            c[i] = in ? cosv[r * P + x.s0 + i] : 1.0f;
            s[i] = in ? sgn * sinv[r * P + x.s0 + i] : 0.0f;
        }
#pragma unroll
        for (int i = 0; i < V; ++i) {
            float& a = t[IL ? 2 * i : i];
            float& z = t[IL ? 2 * i + 1 : V + i];
            const float ar = a * c[i] - z * s[i], zr = a * s[i] + z * c[i];
            a = ar;
            z = zr;
        }
    };

    const int64_t tiles = (S.n + RT - 1) / RT;
    for (int64_t tile = rb; tile < tiles; tile += S.row_blocks) {
        const int64_t n0 = tile * RT;
        // forward: the first step's rows load while the angles are computed,
        // the next step's behind the arithmetic of one (the backward has no
        // registers to spare: 331 -> 364 us on 262,144 rows of 8 and 8 heads
        // of 32 fp32)
        constexpr bool AHEAD = MODE != NORM_BWD;
        float xr[2 * N];
        if constexpr (AHEAD)
            get(S.x, S.x_stride, n0 + rr, act && rr < RT && n0 + rr < S.n, me, xr);
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
            if constexpr (!AHEAD) get(S.x, S.x_stride, n, ok, me, xr);
            values(me, xr, t);
            if constexpr (AHEAD)
                get(S.x, S.x_stride, n + S.RB, act && r + S.RB < RT && n + S.RB < S.n, me, xr);
            if constexpr (MODE == TURN) {
                if (ok) rotate(me, t, r, A.sign);
            } else {
                float g[2 * V];
                float ss = 0.0f, dd = 0.0f;
#pragma unroll
                for (int i = 0; i < 2 * V; ++i) ss = fmaf(t[i], t[i], ss);
                if constexpr (MODE == NORM_BWD) {
                    load(S.g, S.g_stride, n, ok, me, g);
                    if (ok) rotate(me, g, r, -1.0f);
#pragma unroll
                    for (int i = 0; i < 2 * V; ++i) dd = fmaf(g[i] * w[i], t[i], dd);
                }
                // a head wider than one pass: the sums of its other columns
                for (int o = 1; o < A.nchunk; ++o) {
                    const int ov = ((ch + o) % A.nchunk) * A.L + lig;
                    const bool ook = row_ok && ov < A.NV;
                    const Lane<V> other = lane_of<V, IL, PART>(A, ook ? ov : 0);
                    float y[2 * V];
                    load(S.x, S.x_stride, n, ook, other, y);
#pragma unroll
                    for (int i = 0; i < 2 * V; ++i) ss = fmaf(y[i], y[i], ss);
                    if constexpr (MODE == NORM_BWD) {
                        float z[2 * V], u[2 * V];
                        load(S.g, S.g_stride, n, ook, other, z);
                        load_w(other, u);
                        if (ook) rotate(other, z, r, -1.0f);
#pragma unroll
                        for (int i = 0; i < 2 * V; ++i) dd = fmaf(z[i] * u[i], y[i], dd);
                    }
                }
                run_totals<1>(&ss, A.L);
                const float rn = 1.0f / sqrtf(ss * A.inv_F + A.eps);
                if constexpr (MODE == NORM) {
#pragma unroll
                    for (int i = 0; i < 2 * V; ++i) t[i] = t[i] * rn * w[i];
                    if (ok) rotate(me, t, r, 1.0f);
                } else {
                    run_totals<1>(&dd, A.L);
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
                store_part<T, V, PART>(p + me.c0, t, me.n0);
                store_part<T, V, PART>(p + me.c1, t + V, me.n1);
            }
        }
    }
    if constexpr (MODE == NORM_BWD) {
        if (!S.dw_part) return;
        // the block's sums: over its groups of one head, or of all heads, in
        // the order of the groups
        double* red = reinterpret_cast<double*>(lds);
        const int ld = 256 + A.L;  // (threads that differ in i meet in other banks)
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 2 * V; ++i) red[i * ld + tid] = act ? dw[i] : 0.0;
        __syncthreads();
        const int per = A.L * 2 * V;  // sums of one head
        const int heads = S.w_per_head ? S.HB : 1;
        for (int q = tid; q < per * heads; q += 256) {
            const int hq = q / per, x = q - hq * per;
            const int i = x / A.L, l = x - i * A.L;
            const int v = ch * A.L + l;
            if (v >= A.NV || hb * S.HB + hq >= S.H) continue;
            const Lane<V> at = lane_of<V, IL, PART>(A, v);
            if ((i < V ? i : i - V) >= (i < V ? at.n0 : at.n1)) continue;
            double sum = 0.0;
            if (S.w_per_head) {
                for (int k = 0; k < S.RB; ++k) sum += red[i * ld + ((k * S.HB + hq) << A.log2L) + l];
            } else {
                for (int k = 0; k < S.RB * S.HB; ++k) sum += red[i * ld + (k << A.log2L) + l];
            }
            const int col = i < V ? at.c0 + i : at.c1 + i - V;
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
        constexpr int U = 8;  // loads in flight
        for (int64_t p = run * per; p < end; p += U) {
            double x[U];
#pragma unroll
            for (int u = 0; u < U; ++u) x[u] = S.dw_part[(p + u < end ? p + u : p) * S.dw_cols + col];
#pragma unroll
            for (int u = 0; u < U; ++u) sum += p + u < end ? x[u] : 0.0;
        }
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
    if (a.part) {
        if (a.interleaved) hipLaunchKernelGGL((node_rotary_kernel<T, V, true, true, MODE>), grid, block, lds, s, a);
        else hipLaunchKernelGGL((node_rotary_kernel<T, V, false, true, MODE>), grid, block, lds, s, a);
    } else {
        if (a.interleaved) hipLaunchKernelGGL((node_rotary_kernel<T, V, true, false, MODE>), grid, block, lds, s, a);
        else hipLaunchKernelGGL((node_rotary_kernel<T, V, false, false, MODE>), grid, block, lds, s, a);
    }
}

template <typename T, int MODE>
void launch_mode(const RotaryArgs& a, int vec, size_t lds, hipStream_t s) {
    // (eight columns: bf16 forward only, see rotary_geo)
    if constexpr (sizeof(T) == 2 && MODE != NORM_BWD)
        if (vec == 8) return launch_v<T, 8, MODE>(a, lds, s);
    if (vec == 4) launch_v<T, 4, MODE>(a, lds, s);
    else if (vec == 2) launch_v<T, 2, MODE>(a, lds, s);
    else launch_v<T, 1, MODE>(a, lds, s);
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
