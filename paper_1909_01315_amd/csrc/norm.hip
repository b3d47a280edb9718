// The residual stream between attention layers: node_add_norm adds a layer's
// output to the stream and divides each row by its root mean square, its
// backward, and rows in 8 bits (after the norm, or as they are).
//
//   h = x + r,  rn = 1 / sqrt(mean(h^2) + eps),  y = h rn w
//   s = max |y| / 127,  q = round(127 y / max |y|)
//   dx = gh + rn (gy w - h rn^2 mean(gy w h)),  dw = sum over rows of gy h rn
//
// A pure stream: every row is read once and written once.  A row lies in the
// registers of a group of lanes, a wavefront at most or several wavefronts of
// one block, NPT vectors of 16 bytes a lane; its sums go over the lanes and
// then, by way of LDS, over the wavefronts.  Rows of odd widths are read by
// unaligned vectors, the last one past its columns, which are left aside.
//
// It is bound by the memory's streaming rate: 262,144 rows of 256 fp32 summed
// and normed in 178 us (6.0 TB/s read and written), 65,536 of 4,096 bf16 in 368
// (5.8), 232,965 of 512 bf16 with the norm in 8 bits in 139 (6.0), 100,000 of 376
// fp32 to 8 bits in 34 (5.6).  The backward reads three rows for one that it
// writes: 210 us and 11 for the weight's gradient on the first (5.1).  Rows of
// 282 bf16, which start on no vector, are slower: 300,000 of them 129 us (5.2
// TB/s), with the norm in 8 bits 127 (4.7), backward 165 (4.1).  What bounds them
// is not shown: 0.58, 0.76 and 0.92 vector instructions in a SIMD's four cycles,
// at 3.7, 3.6 and 2.8 wavefronts a SIMD, where rows of 288, whole vectors, issue
// 0.87, 0.70 and 1.23 at 7.2, 3.6 and 4.6.  20,011 of them, a short grid, 12 us,
// backward 17 and 5.  One row: 2.4 us.
//
// Sums over a row are fp32, over at most 32 terms a lane and then pairs of
// lanes; the gradient of the weight is a sum over all rows, fp32 within a lane's
// rows of a tile, fp64 from there on.  The norm is made of the sum in fp32, which
// is rounded for its own output alone; the backward reads that output, so in bf16
// its gradients carry one rounding of the sum.
#include "words.h"

namespace gnnk {

namespace {

// 8-bit values are stored at any address
typedef unsigned u2_b __attribute__((ext_vector_type(2), aligned(1)));
typedef unsigned u1_b __attribute__((aligned(1)));
typedef unsigned short u1s_b __attribute__((aligned(1)));

// the largest of x over the aligned run of `red` lanes; every lane gets it
__device__ __forceinline__ uint32_t run_most(uint32_t x, int red) {
    auto with = [&](uint32_t y) { x = x > y ? x : y; };
    if (red >= 2) with((uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, DPP_QUAD_1032, 0xF, 0xF, true));
    if (red >= 4) with((uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, DPP_QUAD_2301, 0xF, 0xF, true));
    if (red >= 8) with((uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, DPP_HALF_MIRROR, 0xF, 0xF, true));
    if (red >= 16) with((uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, DPP_MIRROR, 0xF, 0xF, true));
    if (red >= 32) with(__shfl_xor(x, 16, WAVE));
    if (red >= 64) with(__shfl_xor(x, 32, WAVE));
    return x;
}

// sums of N values over a row's lanes (and wavefronts); red: 16 * N floats of LDS
template <int N, bool WIDE>
__device__ __forceinline__ void row_totals(float* v, const AddNormArgs& A, float* red) {
    run_totals<N>(v, WIDE ? 64 : A.L);
    if constexpr (WIDE) {
        const int wave = threadIdx.x >> 6, first = wave & ~(A.waves - 1);
        __syncthreads();  // (the row before may still be read)
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int u = 0; u < N; ++u) red[wave * N + u] = v[u];
        __syncthreads();
#pragma unroll
        for (int u = 0; u < N; ++u) {
            v[u] = 0.0f;
            for (int k = 0; k < A.waves; ++k) v[u] += red[(first + k) * N + u];
        }
    }
}
template <bool WIDE>
__device__ __forceinline__ uint32_t row_most(uint32_t x, const AddNormArgs& A, uint32_t* red) {
    x = run_most(x, WIDE ? 64 : A.L);
    if constexpr (WIDE) {
        const int wave = threadIdx.x >> 6, first = wave & ~(A.waves - 1);
        __syncthreads();
        if ((threadIdx.x & 63) == 0) red[wave] = x;
        __syncthreads();
        x = 0;
        for (int k = 0; k < A.waves; ++k) x = red[first + k] > x ? red[first + k] : x;
    }
    return x;
}

// V values as 8-bit numbers, each the nearest to t * inv; inv 0: zeros,
// whatever t is
template <int V, bool PART>
__device__ __forceinline__ void put8(int8_t* p, const float* t, float inv, int n, int tail) {
    // beside 1.5 * 2^23 a float's last bit is 1: the sum is rounded to a whole number,
    // ties to even, whose lowest byte is its lowest byte (no magnitude passes 127
    // steps by more than what inv is off by, 2^-23 of it)
    uint32_t b[V], w[V / 4];
#pragma unroll
    for (int i = 0; i < V; ++i) b[i] = __float_as_uint(fmaf(t[i], inv, 12582912.0f));
#pragma unroll
    for (int i = 0; i < V / 4; ++i) {
        const uint32_t lo = __builtin_amdgcn_perm(b[i * 4 + 1], b[i * 4], 0x0C0C0400u);
        const uint32_t hi = __builtin_amdgcn_perm(b[i * 4 + 3], b[i * 4 + 2], 0x04000C0Cu);
        w[i] = inv == 0.0f ? 0u : lo | hi;
    }
    if (!PART || n == V) {
        if constexpr (V == 8) *reinterpret_cast<u2_b*>(p) = u2_b{w[0], w[1]};
        else *reinterpret_cast<u1_b*>(p) = w[0];
    } else {
        uint32_t x = w[0];
        if (V == 8 && (tail & 4)) {
            *reinterpret_cast<u1_b*>(p) = x;
            p += 4;
            x = w[V / 4 - 1];
        }
        if (tail & 2) {
            *reinterpret_cast<u1s_b*>(p) = (uint16_t)x;
            p += 2;
            x >>= 16;
        }
        if (tail & 1) *p = (int8_t)x;
    }
}
// a lane's vector of a row: its `n` columns, V or the last vector's, `tail`,
// the same in all lanes
template <typename T, int V, bool PART>
__device__ __forceinline__ void store_row(T* p, const float* t, int n, int tail) {
    if (!PART || n == V) put<T, V>(p, t);
    else if constexpr (PART) store_few<T, V / 2>(p, t, tail);
}

// NPT vectors of V values a lane, vector p of it being number p * lanes + lane
// of the row; PART: the last vector of a row holds fewer values than V.  The
// first `full_of` vectors of each lane are whole ones of the row (there are as
// many vectors a lane as it takes, but for eight, which stand for five to eight).
constexpr int full_of(int npt) { return npt <= 4 ? npt - 1 : 0; }

template <typename T, int NPT, bool PART, bool WIDE, int MODE>
__global__ __launch_bounds__(WIDE ? 512 : 256) void node_add_norm_kernel(AddNormArgs A) {
    constexpr int V = 16 / sizeof(T);
    constexpr int N = Words<T, V>::N;
    __shared__ float red[32];
    const int tid = threadIdx.x, TPR = WIDE ? A.waves * 64 : A.L;
    const int lig = tid & (TPR - 1), gid = tid / TPR, per = blockDim.x / TPR;
    const int C = A.C, tail = C & (V - 1);

    auto count = [&](int p) {  // columns of the lane's vector p
        if (p < full_of(NPT)) return V;
        const int left = C - (p * TPR + lig) * V;
        return left < 0 ? 0 : (left < V ? left : V);
    };
    auto get = [&](const void* base, int64_t stride, int64_t n, int p, bool ok, float* raw) {
#pragma unroll
        for (int i = 0; i < N; ++i) raw[i] = 0.0f;
        const int m = count(p), c = (p * TPR + lig) * V;
        if (ok && m > 0) {
            const int64_t at = n * stride + c;
            const T* const from = reinterpret_cast<const T*>(base) + at;
            if (p < full_of(NPT)) fetch<T, V, false>(from, V, 0, raw);
            else fetch<T, V, PART>(from, m, (A.n - 1) * stride + C - at, raw);
        }
    };
    float w[NPT][N];
    if constexpr (MODE != QUANT8) {
        if (A.w) {
#pragma unroll
            for (int p = 0; p < NPT; ++p) {
#pragma unroll
                for (int i = 0; i < N; ++i) w[p][i] = 0.0f;
                const int m = count(p), c = (p * TPR + lig) * V;
                if (m > 0) fetch<T, V, PART>(reinterpret_cast<const T*>(A.w) + c, m, C - c, w[p]);
            }
        }
    }
    const int64_t step = (int64_t)gridDim.x * per;
    float xr[NPT][N], rr[MODE == QUANT8 ? 1 : NPT][N];
    auto ahead = [&](int64_t n) {
#pragma unroll
        for (int p = 0; p < NPT; ++p) {
            get(A.x, A.x_stride, n, p, n < A.n, xr[p]);
            if constexpr (MODE != QUANT8)
                if (A.r) get(A.r, A.r_stride, n, p, n < A.n, rr[p]);
        }
    };
    ahead((int64_t)blockIdx.x * per + gid);
    for (int64_t n0 = (int64_t)blockIdx.x * per; n0 < A.n; n0 += step) {
        const int64_t n = n0 + gid;
        const bool ok = n < A.n;
        float h[NPT][V];
        float ss = 0.0f;
#pragma unroll
        for (int p = 0; p < NPT; ++p) {
            const int m = count(p);
            widen<T, V, PART>(xr[p], m, h[p]);
            if constexpr (MODE != QUANT8) {
                if (A.r) {
                    float t[V];
                    widen<T, V, PART>(rr[p], m, t);
#pragma unroll
                    for (int i = 0; i < V; ++i) h[p][i] += t[i];
                    if (ok && m > 0 && A.sum)
                        store_row<T, V, PART>(reinterpret_cast<T*>(A.sum) + n * A.sum_stride + (p * TPR + lig) * V,
                                              h[p], m, tail);
                }
#pragma unroll
                for (int i = 0; i < V; ++i) ss = fmaf(h[p][i], h[p][i], ss);
            }
        }
        ahead(n + step);
        if constexpr (MODE != QUANT8) {
            row_totals<1, WIDE>(&ss, A, red);
            const float rn = 1.0f / sqrtf(ss * A.inv_C + A.eps);
#pragma unroll
            for (int p = 0; p < NPT; ++p)
#pragma unroll
                for (int i = 0; i < V; ++i) h[p][i] *= A.w ? rn * Words<T, V>::at(w[p], i) : rn;
        }
        if constexpr (MODE == ADD_NORM) {
#pragma unroll
            for (int p = 0; p < NPT; ++p) {
                const int m = count(p);
                if (ok && m > 0)
                    store_row<T, V, PART>(reinterpret_cast<T*>(A.out) + n * A.out_stride + (p * TPR + lig) * V, h[p], m,
                                          tail);
            }
        } else {
            // the largest magnitude by its bits, where a NaN is the largest
            uint32_t most = 0;
#pragma unroll
            for (int p = 0; p < NPT; ++p) {
                const int m = count(p);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const uint32_t b = !PART || i < m ? __float_as_uint(h[p][i]) & 0x7FFFFFFFu : 0u;
                    most = b > most ? b : most;
                }
            }
            most = row_most<WIDE>(most, A, reinterpret_cast<uint32_t*>(red) + 16);
            // a row of zeros has scale 0; the scale is no subnormal, whose
            // inverse may be infinite; a row with a NaN or an infinity has
            // scale NaN and values 0, so that what is made of it is NaN
            const bool finite = most < 0x7F800000u;
            const float top = __uint_as_float(most);
            float s = fmaxf(top / 127.0f, 0x1p-126f);
            // values are rounded in one step from their product with the inverse, 127 / top.
            // It is off by at most 2^-23 of itself and never too small: half the largest
            // value, common in bf16, is a tie of 63.5 steps and goes to 64, the even one.
            // (1 / s, off either way, sent half of these to 63.)  Other ties among bf16
            // values are only where top is 127 times a power of two, whose inverse is exact
            float inv = 127.0f / top;
            if (fmaf(inv, top, -127.0f) < 0.0f) inv = __uint_as_float(__float_as_uint(inv) + 1);
            inv = finite ? fminf(inv, 0x1p126f) : 0.0f;
            s = !finite ? __uint_as_float(0x7FC00000u) : (most ? s : 0.0f);
#pragma unroll
            for (int p = 0; p < NPT; ++p) {
                const int m = count(p);
                if (ok && m > 0) put8<V, PART>(A.q + n * A.q_stride + (p * TPR + lig) * V, h[p], inv, m, tail);
            }
            if (ok && lig == 0) A.scale[n] = s;
        }
    }
}

// A block takes a tile of rows: gradients of the stream row by row, and the
// sum of gy h rn over the tile, which the next kernel adds up over the tiles.
// The next rows load before a row's gradients are stored: what waits for loads
// waits for all stores before them.  DENSE: every lane's vectors lie within the
// row, so that a set of rows is stored without a branch and the wait for the
// next rows leaves the stores out (there are some: DENSE asks for them).
template <typename T, int NPT, bool PART, bool WIDE, bool DENSE>
__global__ __launch_bounds__(WIDE ? 512 : 256) void node_add_norm_backward_kernel(AddNormArgs A) {
    constexpr int V = 16 / sizeof(T);
    constexpr int N = Words<T, V>::N;
    extern __shared__ float lds[];
    __shared__ float red[32];
    const int tid = threadIdx.x, TPR = WIDE ? A.waves * 64 : A.L;
    const int lig = tid & (TPR - 1), gid = tid / TPR, per = blockDim.x / TPR;
    const int C = A.C, tail = C & (V - 1);

    auto count = [&](int p) {
        if (DENSE || p < full_of(NPT)) return V;
        const int left = C - (p * TPR + lig) * V;
        return left < 0 ? 0 : (left < V ? left : V);
    };
    float w[NPT][N];
#pragma unroll
    for (int p = 0; p < NPT; ++p) {
#pragma unroll
        for (int i = 0; i < N; ++i) w[p][i] = 0.0f;
        const int m = count(p), c = (p * TPR + lig) * V;
        if (A.w && m > 0) fetch<T, V, PART>(reinterpret_cast<const T*>(A.w) + c, m, C - c, w[p]);
    }
    float hr[NPT][N], gr[NPT][N], sr[NPT][N];
    // (of no row past the last one: that one's again)
    auto load = [&](int64_t n) {
        n = n < A.n ? n : A.n - 1;
#pragma unroll
        for (int p = 0; p < NPT; ++p) {
            const int m = count(p), c = (p * TPR + lig) * V;
            if (!DENSE) {
#pragma unroll
                for (int i = 0; i < N; ++i) hr[p][i] = gr[p][i] = sr[p][i] = 0.0f;
            }
            if (DENSE || m > 0) {
                auto get = [&](const void* base, int64_t stride, float* raw) {
                    const int64_t at = n * stride + c;
                    const T* const from = reinterpret_cast<const T*>(base) + at;
                    if (p < full_of(NPT)) fetch<T, V, false>(from, V, 0, raw);
                    else fetch<T, V, PART>(from, m, (A.n - 1) * stride + C - at, raw);
                };
                get(A.x, A.x_stride, hr[p]);
                get(A.r, A.r_stride, gr[p]);
                if (A.gs) get(A.gs, A.gs_stride, sr[p]);
            }
        }
    };
    for (int64_t tile = blockIdx.x; tile < A.parts; tile += gridDim.x) {
        const int64_t first = tile * per * A.steps;
        float dw[NPT][V];
#pragma unroll
        for (int p = 0; p < NPT; ++p)
#pragma unroll
            for (int i = 0; i < V; ++i) dw[p][i] = 0.0f;

        if (A.n > 0) load(first + gid);
        for (int k = 0; k < A.steps; ++k) {
            const int64_t n0 = first + (int64_t)k * per, n = n0 + gid;
            if (n0 >= A.n) break;
            const bool ok = n < A.n;
            float h[NPT][V], g[NPT][V], s[NPT][V];
            float t[2] = {0.0f, 0.0f};  // sums of h^2 and of gy w h
#pragma unroll
            for (int p = 0; p < NPT; ++p) {
                const int m = count(p);
                widen<T, V, PART>(hr[p], m, h[p]);
                widen<T, V, PART>(gr[p], m, g[p]);
                if (A.gs) widen<T, V, PART>(sr[p], m, s[p]);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    t[0] = fmaf(h[p][i], h[p][i], t[0]);
                    t[1] = fmaf(A.w ? g[p][i] * Words<T, V>::at(w[p], i) : g[p][i], h[p][i], t[1]);
                }
            }
            if (k + 1 < A.steps && n0 + per < A.n) load(n + per);
            row_totals<2, WIDE>(t, A, red);
            const float rn = 1.0f / sqrtf(t[0] * A.inv_C + A.eps);
            const float mean = rn * rn * (t[1] * A.inv_C);
#pragma unroll
            for (int p = 0; p < NPT; ++p) {
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    // (a group without a row adds nothing)
                    if (ok) dw[p][i] = fmaf(g[p][i], h[p][i] * rn, dw[p][i]);
                    const float gw = A.w ? g[p][i] * Words<T, V>::at(w[p], i) : g[p][i];
                    const float d = rn * (gw - h[p][i] * mean);
                    h[p][i] = A.gs ? s[p][i] + d : d;
                }
            }
            if (!DENSE && !A.out) continue;
            T* const out = reinterpret_cast<T*>(A.out) + n * A.out_stride + lig * V;
            if (DENSE && n0 + per <= A.n) {
#pragma unroll
                for (int p = 0; p < NPT; ++p) put<T, V>(out + p * TPR * V, h[p]);
            } else {
#pragma unroll
                for (int p = 0; p < NPT; ++p) {
                    const int m = count(p);
                    if (ok && m > 0) store_row<T, V, PART>(out + p * TPR * V, h[p], m, tail);
                }
                if (DENSE) break;  // (they were the last rows)
            }
        }
        if (!A.part) continue;
        // the tile's sum over the block's rows side by side, in their order
        float* const part = A.part + tile * C;
#pragma unroll
        for (int p = 0; p < NPT; ++p) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < V; ++i) lds[i * blockDim.x + tid] = dw[p][i];
            __syncthreads();
            for (int q = tid; q < TPR * V; q += blockDim.x) {
                const int i = q / TPR, l = q - i * TPR, col = (p * TPR + l) * V + i;
                if (col >= C) continue;
                double sum = 0.0;
                for (int k = 0; k < per; ++k) sum += (double)lds[i * blockDim.x + k * TPR + l];
                part[col] = (float)sum;
            }
        }
    }
}

// the weight's gradient: the tiles' sums in fp64, COLS columns and a run of
// tiles a workgroup, 1,024 / COLS parts of it side by side, each in order, then
// the parts in order; of several runs their sums, which a second launch adds up.
// One launch where it can be: 1,250 tiles of 282 columns, 16 columns a workgroup,
// 6.6 us; in runs of 512 tiles, 64 columns a workgroup, and a second launch 10
template <typename T, typename P, int COLS>
__global__ __launch_bounds__(1024) void node_add_norm_dw_kernel(const P* part, int64_t parts, int C, double* sums, T* dw,
                                                                int runs) {
    constexpr int SUB = 1024 / COLS;
    __shared__ double red[SUB][COLS + 1];
    const int c = threadIdx.x % COLS, q = threadIdx.x / COLS;
    const int64_t col = (int64_t)(blockIdx.x / runs) * COLS + c, run = blockIdx.x % runs;
    const int64_t each = (parts + runs - 1) / runs, per = (each + SUB - 1) / SUB;
    const int64_t stop = (run + 1) * each < parts ? (run + 1) * each : parts;
    const int64_t first = run * each + q * per, end = first + per < stop ? first + per : stop;
    double sum = 0.0;
    if (col < C) {
        constexpr int U = 16;  // loads in flight
        for (int64_t p = first; p < end; p += U) {
            P x[U];
#pragma unroll
            for (int u = 0; u < U; ++u) x[u] = part[(p + u < end ? p + u : p) * C + col];
#pragma unroll
            for (int u = 0; u < U; ++u) sum += p + u < end ? (double)x[u] : 0.0;
        }
    }
    red[q][c] = sum;
    __syncthreads();
    if (q < 4) {
        for (int k = 1; k < SUB / 4; ++k) sum = (k == 1 ? red[q * (SUB / 4)][c] : sum) + red[q * (SUB / 4) + k][c];
    }
    __syncthreads();
    if (q < 4) red[q][c] = sum;
    __syncthreads();
    if (q == 0 && col < C) {
        sum = red[0][c] + red[1][c] + red[2][c] + red[3][c];
        if (sums) sums[run * C + col] = sum;
        else IO<T, 1>::store1(dw + col, (float)sum);
    }
}

template <typename T, int NPT, bool PART, bool WIDE>
void launch_n(const AddNormArgs& a, int mode, hipStream_t s) {
    const dim3 grid((unsigned)a.blocks), block((unsigned)a.threads);
    // a lane holds up to 2 MOST vectors, in the backward MOST; of several
    // wavefronts more than half of that, but for the widest rows of a backward
    constexpr int MOST = (int)sizeof(T);
    if constexpr (!WIDE || NPT > MOST) {
        if (mode == ADD_NORM)
            hipLaunchKernelGGL((node_add_norm_kernel<T, NPT, PART, WIDE, ADD_NORM>), grid, block, 0, s, a);
        else if (mode == ADD_NORM8)
            hipLaunchKernelGGL((node_add_norm_kernel<T, NPT, PART, WIDE, ADD_NORM8>), grid, block, 0, s, a);
        else if (mode == QUANT8)
            hipLaunchKernelGGL((node_add_norm_kernel<T, NPT, PART, WIDE, QUANT8>), grid, block, 0, s, a);
    }
    if constexpr (WIDE ? NPT > MOST / 2 : NPT <= MOST) {
        if (mode != ADD_NORM_BWD) return;
        const size_t lds = a.part ? a.threads * 64 / sizeof(T) : 0;
        if (!PART && a.out && a.C == (WIDE ? a.waves * 64 : a.L) * NPT * 16 / (int)sizeof(T))
            hipLaunchKernelGGL((node_add_norm_backward_kernel<T, NPT, false, WIDE, true>), grid, block, lds, s, a);
        else
            hipLaunchKernelGGL((node_add_norm_backward_kernel<T, NPT, PART, WIDE, false>), grid, block, lds, s, a);
    }
}

template <typename T, int NPT>
void launch_p(const AddNormArgs& a, int mode, hipStream_t s) {
    const bool part = a.C % (16 / (int)sizeof(T)) != 0;
    if (a.waves > 1) {
        if (part) launch_n<T, NPT, true, true>(a, mode, s);
        else launch_n<T, NPT, false, true>(a, mode, s);
    } else {
        if (part) launch_n<T, NPT, true, false>(a, mode, s);
        else launch_n<T, NPT, false, false>(a, mode, s);
    }
}

template <typename T>
void launch_t(const AddNormArgs& a, int npt, int mode, hipStream_t s) {
    if (a.blocks > 0) {
        if (npt == 1) launch_p<T, 1>(a, mode, s);
        else if (npt == 2) launch_p<T, 2>(a, mode, s);
        else if (npt == 3) launch_p<T, 3>(a, mode, s);
        else if (npt == 4) launch_p<T, 4>(a, mode, s);
        else if constexpr (sizeof(T) == 4) launch_p<T, 8>(a, mode, s);
    }
    if (mode == ADD_NORM_BWD && a.part) {
        const unsigned wide = (unsigned)((a.C + 63) / 64), narrow = (unsigned)((a.C + 15) / 16);
        T* const dw = reinterpret_cast<T*>(a.dw);
        if (a.runs > 1) {
            hipLaunchKernelGGL((node_add_norm_dw_kernel<T, float, 64>), dim3(wide * a.runs), dim3(1024), 0, s, a.part,
                               a.parts, a.C, a.sums, dw, a.runs);
            hipLaunchKernelGGL((node_add_norm_dw_kernel<T, double, 16>), dim3(narrow), dim3(1024), 0, s, a.sums,
                               (int64_t)a.runs, a.C, nullptr, dw, 1);
        } else {
            hipLaunchKernelGGL((node_add_norm_dw_kernel<T, float, 16>), dim3(narrow), dim3(1024), 0, s, a.part, a.parts,
                               a.C, nullptr, dw, 1);
        }
    }
}

}  // namespace

hipError_t launch_node_add_norm(const AddNormArgs& a, int dtype, int npt, int mode, hipStream_t s) {
    if (dtype == 0) launch_t<float>(a, npt, mode, s);
    else launch_t<bf16_t>(a, npt, mode, s);
    return hipGetLastError();
}

}  // namespace gnnk
