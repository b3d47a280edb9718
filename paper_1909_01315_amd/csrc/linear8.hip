// Products of rows in 8 bits with a weight in 8 bits that has a scale for each
// output column:
//
//   out[m, n] = xs[m] ws[n] sum_k x[m, k] w[n, k] + bias[n]
//
// The sum is one of whole numbers (v_mfma_i32_16x16x64_i8: exact up to 65,536
// columns), so neither its order nor how it is split shows in the result.
//
// The weight is laid out once, in the order in which the matrix instructions
// take it: blocks of 64 output columns and 128 of k, in them 2 steps of 64 of
// k, 4 fragments of 16 output columns, and for each of 64 lanes 16 bytes
// (row lane % 16 of the fragment, k from lane / 16 * 16 on); zeros past N and
// K.  Row 4 a + i of fragment j is output column 32 (j / 2) + 8 a + 4 (j % 2) + i
// of the block: the weight being the instruction's first operand, a lane's
// results of fragments 2 j and 2 j + 1 are then 8 columns side by side of one
// row of the output, one store of bf16, and those of the four lanes of a row 32.
#include "words.h"

namespace gnnk {

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
// bytes at any address, and aligned
typedef int i4_b __attribute__((ext_vector_type(4), aligned(1)));

constexpr int KB = 128;             // bytes of k of a step
constexpr int WBLOCK = 64 * KB;     // bytes of 64 output columns of a step
constexpr int LDS_BYTES = 160 * 1024;

__device__ __forceinline__ i32x4 mfma(i32x4 a, i32x4 b, i32x4 c) {
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0);
}

// 16 bytes of a row from column k on; those past the row's end count for
// nothing (the weight is 0 there), but are read only within the tensor, whose
// last byte lies before `end`
template <bool TAIL>
__device__ __forceinline__ i32x4 load_x(const int8_t* row, int k, int K, const int8_t* end) {
    if constexpr (TAIL) {
        if (k >= K) return i32x4{0, 0, 0, 0};
        if (row + k + 16 > end) {
            uint32_t w[4] = {0, 0, 0, 0};
            for (int i = 0; i < 16; ++i)
                if (k + i < K) {
                    const uint32_t b = (uint32_t)(uint8_t)row[k + i] << (i % 4 * 8);
                    w[0] |= i / 4 == 0 ? b : 0;
                    w[1] |= i / 4 == 1 ? b : 0;
                    w[2] |= i / 4 == 2 ? b : 0;
                    w[3] |= i / 4 == 3 ? b : 0;
                }
            return i32x4{(int)w[0], (int)w[1], (int)w[2], (int)w[3]};
        }
    }
    const i4_b x = *reinterpret_cast<const i4_b*>(row + k);
    return i32x4{x.x, x.y, x.z, x.w};
}

// first of the four output columns that a lane holds of fragment j
__device__ __forceinline__ int column_of(int j, int lane) { return (j >> 1) * 32 + (lane >> 4) * 8 + (j & 1) * 4; }

// scales and biases of COUNT output columns from n on (those past the last one
// are not stored)
template <typename T, int COUNT>
struct Columns {
    float s[COUNT], b[COUNT];
    __device__ __forceinline__ void load(const Linear8Args& A, int n) {
        const T* const bias = reinterpret_cast<const T*>(A.bias);
        if (n + COUNT <= A.N) {
#pragma unroll
            for (int i = 0; i < COUNT; i += 4) IO<float, 4>::load(A.ws + n + i, s + i);
            if (bias)
#pragma unroll
                for (int i = 0; i < COUNT; i += 4) IO<T, 4>::load(bias + n + i, b + i);
        } else {
#pragma unroll
            for (int i = 0; i < COUNT; ++i) {
                const int c = n + i < A.N ? n + i : A.N - 1;
                s[i] = A.ws[c];
                if (bias) b[i] = IO<T, 1>::load1(bias + c);
            }
        }
        if (!bias)
#pragma unroll
            for (int i = 0; i < COUNT; ++i) b[i] = 0.0f;
    }
};

// COUNT columns of row m of the output from column n on
template <typename T, int COUNT>
__device__ __forceinline__ void put_out(const Linear8Args& A, int64_t m, int n, float xs, const Columns<T, COUNT>& c,
                                        const int* sum) {
    T* const p = reinterpret_cast<T*>(A.out) + m * A.out_stride + n;
    float t[COUNT];
#pragma unroll
    for (int i = 0; i < COUNT; ++i) t[i] = fmaf((float)sum[i] * xs, c.s[i], c.b[i]);
    constexpr int V = COUNT < 16 / (int)sizeof(T) ? COUNT : 16 / (int)sizeof(T);
#pragma unroll
    for (int i = 0; i < COUNT; i += V) {
        const int left = A.N - n - i;
        if (left >= V) put<T, V>(p + i, t + i);
        else if (left > 0) store_few<T, V / 2>(p + i, t + i, left);
    }
}

// the tiles of a product: tm by tn, `group` of rows side by side; padded to
// eight equal runs
struct TileArgs {
    int64_t tm, tiles, padded;
    int32_t tn, group;
};

// the panels of a weight: `width` blocks of 64 output columns each; `split`
// wavefronts share the panel's columns of the same rows
struct StreamArgs {
    int32_t panels, width, split;
};

// Few rows: a block forms MI * 16 rows of NJ * 16 output columns, its
// wavefronts taking steps of k in turn straight from memory, and adds their
// sums up through LDS.
template <typename T, int MI, int NJ>
__global__ __launch_bounds__(1024) void linear8_few_kernel(Linear8Args A, int waves) {
    extern __shared__ i32x4 sums[];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    constexpr int PER = 4 / NJ;  // blocks that share 64 output columns, NJ fragments each
    const unsigned nbs = (unsigned)((A.N + 63) / 64) * PER, b = blockIdx.x % nbs;
    const int nb = b / PER, j0 = b % PER * NJ;
    const int64_t m0 = (int64_t)(blockIdx.x / nbs) * MI * 16;
    const int KS = (A.K + KB - 1) / KB, full = A.K / KB;
    const int8_t* const wp = A.w + (int64_t)nb * KS * WBLOCK + j0 * 1024 + lane * 16;
    const int8_t* const end = A.x + (A.M - 1) * A.x_stride + A.K;
    const int8_t* row[MI];
#pragma unroll
    for (int i = 0; i < MI; ++i) {
        const int64_t m = m0 + i * 16 + (lane & 15);
        row[i] = A.x + (m < A.M ? m : A.M - 1) * A.x_stride;
    }
    i32x4 acc[MI][NJ] = {};
    auto step = [&](int ks, auto tail) {
        i32x4 w[2][NJ], x[2][MI];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
#pragma unroll
            for (int j = 0; j < NJ; ++j)
                w[k][j] = *reinterpret_cast<const i32x4*>(wp + (int64_t)ks * WBLOCK + k * 4096 + j * 1024);
#pragma unroll
            for (int i = 0; i < MI; ++i)
                x[k][i] = load_x<tail.value>(row[i], ks * KB + k * 64 + (lane >> 4) * 16, A.K, end);
        }
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int j = 0; j < NJ; ++j) acc[i][j] = mfma(w[k][j], x[k][i], acc[i][j]);
    };
    int ks = wave;
    for (; ks < full; ks += waves) step(ks, std::integral_constant<bool, false>());
    if (ks < KS) step(ks, std::integral_constant<bool, true>());
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j) sums[((wave * MI + i) * NJ + j) * 64 + lane] = acc[i][j];
    __syncthreads();
    for (int f = wave; f < MI * NJ; f += waves) {
        i32x4 t = sums[f * 64 + lane];
        for (int k = 1; k < waves; ++k) t += sums[(k * MI * NJ + f) * 64 + lane];
        const int64_t m = m0 + f / NJ * 16 + (lane & 15);
        const int n = nb * 64 + column_of(j0 + f % NJ, lane);
        const int r[4] = {t.x, t.y, t.z, t.w};
        if (m < A.M && n < A.N) {
            Columns<T, 4> c;
            c.load(A, n);
            put_out<T, 4>(A, m, n, A.xs[m], c, r);
        }
    }
}

// Many rows: a block of WM by WN wavefronts forms BM rows of BN output columns.
// A step of 128 bytes of k goes through registers into one of two LDS buffers
// while the one before it is multiplied.  In LDS a row is 128 bytes, its
// 16-byte pieces in the order piece ^ (row % 8), so that the 8 lanes that are
// served at once, 8 rows of one piece, meet in no bank; the weight keeps its
// order, in which a lane's piece is at 16 * lane.
template <typename T, int BM, int BN, int WM, int WN, int BLOCKS>
__global__ __launch_bounds__(WM * WN * 64, BLOCKS) void linear8_tile_kernel(Linear8Args A, TileArgs G) {
    constexpr int THREADS = WM * WN * 64;
    constexpr int MT = BM / WM / 16, NT = BN / WN / 16;
    constexpr int XC = BM * 8 / THREADS, WC = BN * 8 / THREADS;  // pieces of a thread
    static_assert(NT % 4 == 0 && BM * 8 % THREADS == 0 && BN * 8 % THREADS == 0, "");
    extern __shared__ int8_t lds[];
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const int wm = wave / WN * MT * 16, wn = wave % WN * NT / 4;  // first row, first block of 64 output columns
    const int KS = (A.K + KB - 1) / KB, full = A.K / KB, NB = (A.N + 63) / 64;
    const int8_t* const end = A.x + (A.M - 1) * A.x_stride + A.K;

    for (int64_t b = blockIdx.x; b < G.padded; b += gridDim.x) {
        // blocks are dealt to the eight dies in turn: each gets a run of
        // tiles, in groups of rows that go over the output columns together
        const int64_t t = (b & 7) * (G.padded >> 3) + (b >> 3);
        if (t >= G.tiles) continue;
        const int64_t group = t / ((int64_t)G.group * G.tn), in = t - group * G.group * G.tn;
        const int64_t left = G.tm - group * G.group, high = left < G.group ? left : G.group;
        const int64_t m0 = (group * G.group + in % high) * BM;
        const int nb0 = (int)(in / high) * (BN / 64);

        const int8_t* row[XC];
        int xl[XC], xk[XC];  // place in LDS, bytes of k
#pragma unroll
        for (int i = 0; i < XC; ++i) {
            const int c = tid + i * THREADS, r = c >> 3, ch = c & 7;
            const int64_t m = m0 + r;
            row[i] = A.x + (m < A.M ? m : A.M - 1) * A.x_stride;
            xl[i] = r * KB + ((ch ^ (r & 7)) << 4);
            xk[i] = ch * 16;
        }
        const int8_t* wp[WC];
#pragma unroll
        for (int i = 0; i < WC; ++i) {
            const int c = tid + i * THREADS, nb = nb0 + c / 512;
            wp[i] = A.w + (int64_t)(nb < NB ? nb : NB - 1) * KS * WBLOCK + c % 512 * 16;
        }
        i32x4 xr[XC], wr[WC];
        auto load = [&](int ks) {
#pragma unroll
            for (int i = 0; i < WC; ++i) wr[i] = *reinterpret_cast<const i32x4*>(wp[i] + (int64_t)ks * WBLOCK);
            if (ks < full) {
#pragma unroll
                for (int i = 0; i < XC; ++i) xr[i] = load_x<false>(row[i], ks * KB + xk[i], A.K, end);
            } else {
#pragma unroll
                for (int i = 0; i < XC; ++i) xr[i] = load_x<true>(row[i], ks * KB + xk[i], A.K, end);
            }
        };
        auto put = [&](int buf) {
            int8_t* const xb = lds + buf * (BM + BN) * KB;
            int8_t* const wb = xb + BM * KB;
#pragma unroll
            for (int i = 0; i < XC; ++i) *reinterpret_cast<i32x4*>(xb + xl[i]) = xr[i];
#pragma unroll
            for (int i = 0; i < WC; ++i) *reinterpret_cast<i32x4*>(wb + (tid + i * THREADS) * 16) = wr[i];
        };
        i32x4 acc[MT][NT] = {};
        load(0);
        __syncthreads();  // (the tile before may still be read)
        put(0);
        __syncthreads();
        for (int ks = 0; ks < KS; ++ks) {
            if (ks + 1 < KS) load(ks + 1);
            const int8_t* const xb = lds + (ks & 1) * (BM + BN) * KB;
            const int8_t* const wb = xb + BM * KB + wn * WBLOCK + lane * 16;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                i32x4 x[MT];
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    const int r = wm + i * 16 + (lane & 15), ch = k * 4 + (lane >> 4);
                    x[i] = *reinterpret_cast<const i32x4*>(xb + r * KB + ((ch ^ (r & 7)) << 4));
                }
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    const i32x4 w = *reinterpret_cast<const i32x4*>(wb + (j >> 2) * WBLOCK + k * 4096 + (j & 3) * 1024);
#pragma unroll
                    for (int i = 0; i < MT; ++i) acc[i][j] = mfma(w, x[i], acc[i][j]);
                }
            }
            if (ks + 1 < KS) put((ks + 1) & 1);
            __syncthreads();
        }
        float xs[MT];
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const int64_t m = m0 + wm + i * 16 + (lane & 15);
            xs[i] = A.xs[m < A.M ? m : A.M - 1];
        }
#pragma unroll
        for (int j = 0; j < NT; j += 2) {
            const int n = (nb0 + wn + (j >> 2)) * 64 + column_of(j & 3, lane);
            if (n >= A.N) continue;
            Columns<T, 8> c;
            c.load(A, n);
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                const int64_t m = m0 + wm + i * 16 + (lane & 15);
                const i32x4 u = acc[i][j], v = acc[i][j + 1];
                const int r[8] = {u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w};
                if (m < A.M) put_out<T, 8>(A, m, n, xs[i], c, r);
            }
        }
    }
}

// Many rows of at most KS * 128 columns: a block keeps a panel of the weight
// in LDS and its wavefronts stream rows past it, MI * 16 at a time, which they
// read straight into registers and hold there for all of the panel's columns.
// Nothing waits for another wavefront once the panel is there.
template <typename T, int KS, int MI>
__global__ __launch_bounds__(1024, 1) void linear8_stream_kernel(Linear8Args A, StreamArgs G) {
    extern __shared__ int8_t lds[];
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    // the blocks of one run of rows sit on one die, one for each panel
    const int die = blockIdx.x & 7, at = blockIdx.x >> 3;
    const int panel = at % G.panels;
    const int64_t run = (int64_t)(at / G.panels) * 8 + die, runs = (int64_t)(gridDim.x >> 3) / G.panels * 8;
    const int NB = (A.N + 63) / 64, nb0 = panel * G.width;
    const int nbs = NB - nb0 < G.width ? NB - nb0 : G.width;  // blocks of 64 output columns
    {
        const i32x4* const w = reinterpret_cast<const i32x4*>(A.w + (int64_t)nb0 * KS * WBLOCK);
        i32x4* const l = reinterpret_cast<i32x4*>(lds);
        const int pieces = nbs * KS * (WBLOCK / 16);
        for (int c = tid; c < pieces; c += 1024) l[c] = w[c];
    }
    __syncthreads();
    const int8_t* const end = A.x + (A.M - 1) * A.x_stride + A.K;
    const int64_t tiles = (A.M + MI * 16 - 1) / (MI * 16);
    const int part = wave % G.split, teams = 16 / G.split;
    for (int64_t tile = run + runs * (wave / G.split); tile < tiles; tile += runs * teams) {
        const int64_t m0 = tile * (MI * 16);
        const int8_t* row[MI];
        float xs[MI];
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            const int64_t m = m0 + i * 16 + (lane & 15), mc = m < A.M ? m : A.M - 1;
            row[i] = A.x + mc * A.x_stride;
            xs[i] = A.xs[mc];
        }
        i32x4 x[KS * 2][MI];
#pragma unroll
        for (int k = 0; k < KS * 2; ++k)
#pragma unroll
            for (int i = 0; i < MI; ++i) {
                const int at_k = k * 64 + (lane >> 4) * 16;
                x[k][i] = k < KS * 2 - 2 ? load_x<false>(row[i], at_k, A.K, end) : load_x<true>(row[i], at_k, A.K, end);
            }
        for (int nb = part; nb < nbs; nb += G.split) {
            const int8_t* const w = lds + nb * KS * WBLOCK + lane * 16;
#pragma unroll
            for (int j = 0; j < 4; j += 2) {
                i32x4 acc[2][MI] = {};
#pragma unroll
                for (int k = 0; k < KS * 2; ++k)
#pragma unroll
                    for (int f = 0; f < 2; ++f) {
                        const i32x4 b = *reinterpret_cast<const i32x4*>(w + k * 4096 + (j + f) * 1024);
#pragma unroll
                        for (int i = 0; i < MI; ++i) acc[f][i] = mfma(b, x[k][i], acc[f][i]);
                    }
                const int n = (nb0 + nb) * 64 + column_of(j, lane);
                if (n < A.N) {
                    Columns<T, 8> c;
                    c.load(A, n);
#pragma unroll
                    for (int i = 0; i < MI; ++i) {
                        const int64_t m = m0 + i * 16 + (lane & 15);
                        const i32x4 u = acc[0][i], v = acc[1][i];
                        const int r[8] = {u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w};
                        if (m < A.M) put_out<T, 8>(A, m, n, xs[i], c, r);
                    }
                }
            }
        }
    }
}

// the weight in the order described above, a thread 16 bytes
__global__ __launch_bounds__(256) void weight8_pack_kernel(const int8_t* w, int64_t stride, int32_t N, int32_t K,
                                                           int8_t* packed, int64_t chunks) {
    const int KS = (K + KB - 1) / KB;
    for (int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x; c < chunks; c += (int64_t)gridDim.x * 256) {
        const int lane = (int)(c & 63), j = (int)(c >> 6) & 3, half = (int)(c >> 8) & 1;
        const int64_t b = c >> 9;
        const int ks = (int)(b % KS);
        const int r = lane & 15, k = ks * KB + half * 64 + (lane >> 4) * 16;
        const int64_t n = b / KS * 64 + (j >> 1) * 32 + (r >> 2) * 8 + (j & 1) * 4 + (r & 3);
        uint32_t x[4] = {0, 0, 0, 0};
        if (n < N)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (k + i < K) x[i / 4] |= (uint32_t)(uint8_t)w[n * stride + k + i] << (i % 4 * 8);
        *reinterpret_cast<i32x4*>(packed + c * 16) = i32x4{(int)x[0], (int)x[1], (int)x[2], (int)x[3]};
    }
}

template <typename T, int BM, int BN, int WM, int WN, int BLOCKS>
void launch_tile(const Linear8Args& a, hipStream_t s) {
    TileArgs g;
    g.tm = (a.M + BM - 1) / BM;
    g.tn = (a.N + BN - 1) / BN;
    g.tiles = g.tm * g.tn;
    g.padded = (g.tiles + 7) / 8 * 8;
    g.group = 8;
    const int64_t blocks = g.padded < (1 << 20) ? g.padded : 1 << 20;
    hipLaunchKernelGGL((linear8_tile_kernel<T, BM, BN, WM, WN, BLOCKS>), dim3((unsigned)blocks), dim3(WM * WN * 64),
                       2 * (BM + BN) * KB, s, a, g);
}

template <typename T, int MI, int NJ>
void launch_few(const Linear8Args& a, int waves, hipStream_t s) {
    const int64_t blocks = ((a.M + MI * 16 - 1) / (MI * 16)) * ((a.N + 63) / 64 * (4 / NJ));
    hipLaunchKernelGGL((linear8_few_kernel<T, MI, NJ>), dim3((unsigned)blocks), dim3(waves * 64),
                       waves * MI * NJ * 1024, s, a, waves);
}

template <typename T, int KS>
void launch_stream(const Linear8Args& a, hipStream_t s) {
    constexpr int MI = 2, CUS = 32;  // of a die
    const int NB = (a.N + 63) / 64, most = LDS_BYTES / (KS * WBLOCK);
    StreamArgs g;
    g.panels = (NB + most - 1) / most;
    if (g.panels > CUS) g.panels = CUS;  // (not reached: see launch_t)
    g.width = (NB + g.panels - 1) / g.panels;
    const int runs = CUS / g.panels * 8;
    const int64_t tiles = (a.M + MI * 16 - 1) / (MI * 16);
    g.split = 1;
    while (g.split < 16 && g.split < g.width && tiles * g.split < runs * 8) g.split *= 2;
    hipLaunchKernelGGL((linear8_stream_kernel<T, KS, MI>), dim3((unsigned)(runs * g.panels)), dim3(1024),
                       g.width * KS * WBLOCK, s, a, g);
}

template <typename T>
void launch_t(const Linear8Args& a, int way, hipStream_t s) {
    const int KS = (a.K + KB - 1) / KB, waves = KS < 16 ? KS : 16;
    if (way ? way == 1 : a.M <= 64) return a.M > 16 ? launch_few<T, 4, 1>(a, waves, s) : launch_few<T, 1, 1>(a, waves, s);
    if (way == 2) return launch_tile<T, 64, 64, 2, 1, 2>(a, s);
    if (way == 3) return launch_tile<T, 128, 64, 4, 1, 2>(a, s);
    if (way == 4) return launch_tile<T, 128, 128, 2, 2, 2>(a, s);
    if (way == 5) return launch_tile<T, 256, 128, 4, 2, 1>(a, s);
    if (way == 6) return launch_tile<T, 256, 256, 2, 2, 1>(a, s);
    if (way == 8 && KS <= 4 && a.N <= 8192) {
        if (KS == 1) return launch_stream<T, 1>(a, s);
        if (KS == 2) return launch_stream<T, 2>(a, s);
        if (KS == 3) return launch_stream<T, 3>(a, s);
        return launch_stream<T, 4>(a, s);
    }
    if (way == 7) return launch_tile<T, 256, 256, 4, 2, 1>(a, s);
    launch_tile<T, 128, 128, 2, 2, 2>(a, s);
}

}  // namespace

hipError_t launch_linear8(const Linear8Args& a, int dtype, int tile, hipStream_t s) {
    if (a.M == 0) return hipSuccess;
    if (dtype == 0) launch_t<float>(a, tile, s);
    else launch_t<bf16_t>(a, tile, s);
    return hipGetLastError();
}

hipError_t launch_weight8_pack(const int8_t* w, int64_t stride, int32_t N, int32_t K, int8_t* packed, hipStream_t s) {
    const int64_t chunks = (int64_t)((N + 63) / 64) * ((K + KB - 1) / KB) * (WBLOCK / 16);
    const int64_t blocks = (chunks + 255) / 256;
    hipLaunchKernelGGL(weight8_pack_kernel, dim3((unsigned)(blocks < 65536 ? blocks : 65536)), dim3(256), 0, s, w, stride,
                       N, K, packed, chunks);
    return hipGetLastError();
}

}  // namespace gnnk
