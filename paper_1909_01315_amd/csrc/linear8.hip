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
// (column lane % 16 of the fragment, k from lane / 16 * 16 on); zeros past N
// and K.  Column c of fragment j is output column 4 c + j of the block: of the
// four fragments' results a lane then holds 4 columns side by side, of 4 rows,
// and the 16 lanes of a row write its 64 columns at once, whole lines of 128
// bytes in bf16.  (With 64 bytes of a row a store, 16 rows at once, 262,144 rows
// of 256 to 768 columns took 150 us, 127 of them for the stores alone.)
//
// Four kernels, for what bounds a product (choose() has the rule).  What they
// measured, rows x columns to outputs, results in bf16:
//   few     1 x 1,024 to 1,536 3.2 us, 37 x 2,048 to 2,048 6.4: a launch, one
//           chain of loads and the join of its wavefronts
//   stream  262,144 x 256 to 768 81 us (5.8 TB/s; a fill of the output alone 59),
//           232,965 x 512 to 512 83 (4.3 TB/s, rows read once a panel), 20,011 x
//           282 to 141 of fp32 8.4
//   deep    16,384 x 4,096 to 4,096 212 us (2.6 POP/s), 229 to 239 where rows lie
//           4,096 bytes apart; x 2,048 124, x 8,192 396: 1.4 us a tile and step,
//           of which the matrix instructions alone take 1.02 (4.2 POP/s on random
//           bytes, 4.9 on zeros), and 8 us a tile besides, its stores among them
//   tile    100,000 x 1,501 to 1,500 430 us (1.05 POP/s), at addresses that loads
//           into LDS do not take
#include "words.h"

namespace gnnk {

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
// bytes at any address, and aligned
typedef int i4_b __attribute__((ext_vector_type(4), aligned(1)));

constexpr int KB = 128;             // bytes of k of a step
constexpr int WBLOCK = 64 * KB;     // bytes of 64 output columns of a step
constexpr int LDS_BYTES = 160 * 1024;
// bytes of an output that is stored past the caches (the last one holds 256 MB):
// 262,144 rows of 768 columns of bf16, 403 MB, 101 -> 81 us; 100,000 rows of 600,
// 120 MB, 57 -> 76
constexpr int64_t PAST_CACHES = 192 << 20;

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

// The same of any address, from the five words that hold the 16 bytes: loads at
// addresses that are no multiple of 4 take twice as long (100,000 rows of 282 to
// 128 columns 18 -> 14 us, of 1,001 to 512 111 -> 90; through tiles they wait for
// less, 1,501 to 1,500 384 -> 505).  Reads up to 3 bytes before and 4 after.
__device__ __forceinline__ i32x4 load_shifted(const int8_t* p) {
    const uint32_t by = (uint32_t)(uintptr_t)p & 3;
    const uint32_t* const w = reinterpret_cast<const uint32_t*>(p - by);
    const i4_el a = *reinterpret_cast<const i4_el*>(w);
    const uint32_t b = w[4];
    return i32x4{(int)__builtin_amdgcn_alignbyte(a.y, a.x, by), (int)__builtin_amdgcn_alignbyte(a.z, a.y, by),
                 (int)__builtin_amdgcn_alignbyte(a.w, a.z, by), (int)__builtin_amdgcn_alignbyte(b, a.w, by)};
}

// four columns; NT: past the caches
template <typename T, bool NT>
__device__ __forceinline__ void put_four(T* p, const float* t) {
    if constexpr (!NT) {
        put<T, 4>(p, t);
    } else if constexpr (sizeof(T) == 2) {
        const bf16x2 a = {(__bf16)t[0], (__bf16)t[1]}, b = {(__bf16)t[2], (__bf16)t[3]};
        __builtin_nontemporal_store(u2_h{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b)},
                                    reinterpret_cast<u2_h*>(p));
    } else {
        __builtin_nontemporal_store(f4_el{t[0], t[1], t[2], t[3]}, reinterpret_cast<f4_el*>(p));
    }
}

// The results of 16 rows and 64 output columns that the lanes of a wavefront
// hold, four rows (lane / 16 * 4 and on) by four columns (lane % 16 * 4 and on)
// each: scales and biases of the columns, then the rows.
template <typename T>
struct Columns {
    float s[4], b[4];
    int n;  // the first column
    __device__ __forceinline__ void load(const Linear8Args& A, int first, int lane) {
        const T* const bias = reinterpret_cast<const T*>(A.bias);
        n = first + (lane & 15) * 4;
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] = b[i] = 0.0f;
        if (n + 4 <= A.N) {
            IO<float, 4>::load(A.ws + n, s);
            if (bias) IO<T, 4>::load(bias + n, b);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (n + i < A.N) {
                    s[i] = A.ws[n + i];
                    if (bias) b[i] = IO<T, 1>::load1(bias + n + i);
                }
        }
    }
    __device__ __forceinline__ void load_lds(const float* ls, const float* lb, int nb, int first, int lane) {
        n = first + (lane & 15) * 4;
        IO<float, 4>::load(ls + nb * 64 + (lane & 15) * 4, s);
        IO<float, 4>::load(lb + nb * 64 + (lane & 15) * 4, b);
    }
    // scales from LDS (those of the 64 columns at ls), biases from memory
    __device__ __forceinline__ void load_mixed(const Linear8Args& A, const float* ls, int first, int lane) {
        n = first + (lane & 15) * 4;
        IO<float, 4>::load(ls + (lane & 15) * 4, s);
#pragma unroll
        for (int i = 0; i < 4; ++i) b[i] = 0.0f;
        if (A.bias) {
            const T* const bias = reinterpret_cast<const T*>(A.bias);
            if (n + 4 <= A.N) {
                IO<T, 4>::load(bias + n, b);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (n + i < A.N) b[i] = IO<T, 1>::load1(bias + n + i);
            }
        }
    }
    // row r of the lane's four, of scale xs
    __device__ __forceinline__ void row(float xs, int r, i32x4 c0, i32x4 c1, i32x4 c2, i32x4 c3, float* t) const {
        t[0] = fmaf((float)c0[r] * xs, s[0], b[0]);
        t[1] = fmaf((float)c1[r] * xs, s[1], b[1]);
        t[2] = fmaf((float)c2[r] * xs, s[2], b[2]);
        t[3] = fmaf((float)c3[r] * xs, s[3], b[3]);
    }
    // rows m .. m + 3, with scales xs
    __device__ __forceinline__ void store(const Linear8Args& A, int64_t m, const float* xs, i32x4 c0, i32x4 c1, i32x4 c2,
                                          i32x4 c3) const {
        T* p = reinterpret_cast<T*>(A.out) + m * A.out_stride + n;
#pragma unroll
        for (int r = 0; r < 4; ++r, p += A.out_stride) {
            float t[4];
            row(xs[r], r, c0, c1, c2, c3, t);
            if (m + r < A.M) {
                if (n + 4 <= A.N) put<T, 4>(p, t);
                else if (n < A.N) store_few<T, 2>(p, t, A.N - n);
            }
        }
    }
};
// scales of rows m .. m + 3 (those past the last one are not stored)
__device__ __forceinline__ void load_scales(const Linear8Args& A, int64_t m, float* xs) {
    if (m + 4 <= A.M) {
        IO<float, 4>::load(A.xs + m, xs);
    } else {
#pragma unroll
        for (int r = 0; r < 4; ++r) xs[r] = m + r < A.M ? A.xs[m + r] : 0.0f;
    }
}

// 16 bytes a lane from memory, at `from` + `off`, into LDS at `to` + 16 * lane
// (one `from` and `to` for all lanes).  It counts as a load of the wavefront's
// (vmcnt) that the compiler does not see: waits for it are written out.  It
// writes m0, which the compiler reserves and so does not take as a clobber; its
// own code for these kernels has no instruction that reads or writes m0.
__device__ __forceinline__ void load_to_lds(const int8_t* from, uint32_t off, uint32_t to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(off), "s"(from)
                 : "memory");
}

// the same of 4 bytes a lane, at `to` + 4 * lane
__device__ __forceinline__ void load_word_to_lds(const void* from, uint32_t off, uint32_t to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(to), "v"(off), "s"(from)
                 : "memory");
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
    const unsigned nbs = (unsigned)((A.N + 63) / 64) * PER, at = blockIdx.x % nbs;
    const int nb = at / PER, j0 = at % PER * NJ;
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
    // a wavefront that joins the sums of a fragment reads its scales first, while it
    // waits for its rows (37 rows of 2,048 to 2,048 columns in a captured graph 5.7 ->
    // 5.5 us, one of 4,096 to 4,096 4.1 -> 3.7)
    const int f = wave, n = nb * 64 + (lane & 15) * 4 + j0 + f % NJ;
    const int64_t m = m0 + f / NJ * 16 + (lane >> 4) * 4;
    float xs[4], s = 0.0f, b = 0.0f;
    if (f < MI * NJ) {
        const int c = n < A.N ? n : A.N - 1;
        load_scales(A, m, xs);
        s = A.ws[c];
        if (A.bias) b = IO<T, 1>::load1(reinterpret_cast<const T*>(A.bias) + c);
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
                for (int j = 0; j < NJ; ++j) acc[i][j] = mfma(x[k][i], w[k][j], acc[i][j]);
    };
    int ks = wave;
    for (; ks < full; ks += waves) step(ks, std::integral_constant<bool, false>());
    if (ks < KS) step(ks, std::integral_constant<bool, true>());
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j) sums[((wave * MI + i) * NJ + j) * 64 + lane] = acc[i][j];
    __syncthreads();
    auto join = [&](int f, int64_t m, int n, const float* xs, float s, float b) {
        i32x4 t = sums[f * 64 + lane];
        for (int k = 1; k < waves; ++k) t += sums[(k * MI * NJ + f) * 64 + lane];
        if (n >= A.N) return;
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (m + r < A.M)
                IO<T, 1>::store1(reinterpret_cast<T*>(A.out) + (m + r) * A.out_stride + n, fmaf((float)t[r] * xs[r], s, b));
    };
    if (f < MI * NJ) join(f, m, n, xs, s, b);
    // (fewer wavefronts than fragments: short rows)
    for (int g = f + waves; g < MI * NJ; g += waves) {
        const int n = nb * 64 + (lane & 15) * 4 + j0 + g % NJ, c = n < A.N ? n : A.N - 1;
        const int64_t m = m0 + g / NJ * 16 + (lane >> 4) * 4;
        load_scales(A, m, xs);
        join(g, m, n, xs, A.ws[c], A.bias ? IO<T, 1>::load1(reinterpret_cast<const T*>(A.bias) + c) : 0.0f);
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
                    for (int i = 0; i < MT; ++i) acc[i][j] = mfma(x[i], w, acc[i][j]);
                }
            }
            if (ks + 1 < KS) put((ks + 1) & 1);
            __syncthreads();
        }
        float xs[MT][4];
#pragma unroll
        for (int i = 0; i < MT; ++i) load_scales(A, m0 + wm + i * 16 + (lane >> 4) * 4, xs[i]);
#pragma unroll
        for (int j = 0; j < NT; j += 4) {
            Columns<T> c;
            c.load(A, (nb0 + wn + j / 4) * 64, lane);
#pragma unroll
            for (int i = 0; i < MT; ++i)
                c.store(A, m0 + wm + i * 16 + (lane >> 4) * 4, xs[i], acc[i][j], acc[i][j + 1], acc[i][j + 2],
                        acc[i][j + 3]);
        }
    }
}

// Many rows, long sums: WM by two wavefronts form BM rows of BN output columns,
// one tile after another.  Steps of 128 bytes of k, whole lines, are loaded
// straight into one of two LDS buffers while the one before is multiplied; a
// wavefront reads the fragments of half a step while it multiplies those of the
// half before.  The next tile's first two steps load while a tile is stored.
template <typename T, int BM, int BN, int WM, int BLOCKS, bool RAGGED, bool PAST>
__global__ __launch_bounds__(WM * 128, BLOCKS) void linear8_deep_kernel(Linear8Args A, TileArgs G) {
    constexpr int MT = BM / WM / 16, NT = BN / 32;
    constexpr int STAGE = (BM + BN) * KB, XL = BM / 16 / WM, WL = BN / 16 / WM;  // bytes; loads of a wavefront
    static_assert(NT % 4 == 0 && MT * WM * 16 == BM && XL * WM * 16 == BM && WL * WM * 16 == BN, "");
    static_assert(BM == BN && BM + BN == WM * 128, "a lane loads one column's scale or one row's");
    extern __shared__ int8_t lds[];
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) int8_t*)lds;
    float* const scales = reinterpret_cast<float*>(lds + 2 * STAGE);  // of columns and rows, for tiles in turn
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int wm = (wave >> 1) * MT * 16, wn = (wave & 1) * NT / 4;  // first row, first block of 64 output columns
    const int S = (A.K + KB - 1) / KB, NB = (A.N + 63) / 64;

    // In LDS a row of a step is 128 bytes, its pieces in the order
    // piece ^ (row % 8): 8 rows of one piece meet in no bank
    const int piece = ((lane & 7) ^ (lane >> 3)) * 16;
    // (pieces past the row's end are any of its bytes: the weight is 0 there)
    const int past = (S - 1) * KB + piece < A.K ? 0 : piece;
    const int8_t* const end = A.x + (A.M - 1) * A.x_stride + A.K;
    const int xr = (wm + (lane & 15)) * KB, wr = BM * KB + wn * WBLOCK + lane * 16;

    struct Place {
        int64_t m0;
        int nb0;
        bool there;
    };
    // the place of tile number b; none past the last one
    auto place = [&](int64_t b) {
        // blocks are dealt to the eight dies in turn: each gets a run of tiles
        const int64_t t = (b & 7) * (G.padded >> 3) + (b >> 3);
        if (b >= G.padded || t >= G.tiles) return Place{0, 0, false};
        const int64_t group = t / ((int64_t)G.group * G.tn);
        const int in = (int)(t - group * G.group * G.tn);
        const int64_t left = G.tm - group * G.group;
        const int high = left < G.group ? (int)left : G.group;
        return Place{(group * G.group + in % high) * BM, in / high * (BN / 64), true};
    };
    int64_t m0;
    int nb0;
    const int8_t* xb;
    uint32_t xo[XL];
    // go on to the tile at p; its scales load into LDS
    auto begin = [&](const Place& p, int turn) {
        m0 = p.m0;
        nb0 = p.nb0;
        xb = A.x + m0 * A.x_stride;
#pragma unroll
        for (int i = 0; i < XL; ++i) {
            const int r = (wave * XL + i) * 8 + (lane >> 3);
            xo[i] = (uint32_t)(m0 + r < A.M ? r : (int)(A.M - 1 - m0)) * (uint32_t)A.x_stride + piece;
        }
        const uint32_t to = lds0 + 2 * STAGE + turn * (BM + BN) * 4 + wave * 256;
        if (wave < WM) {
            const int n = nb0 * 64 + tid;
            load_word_to_lds(A.ws, (n < A.N ? n : A.N - 1) * 4, to);
        } else {
            const int r = tid - BN;
            load_word_to_lds(A.xs + m0, (m0 + r < A.M ? r : (int)(A.M - 1 - m0)) * 4, to);
        }
    };
    // loads `first` to `last` of a wavefront's for step s
    auto fill = [&](int s, int first, int last) {
        const uint32_t to = lds0 + (s & 1) * STAGE;
        const int off = s + 1 < S ? 0 : past;
#pragma unroll
        for (int l = 0; l < XL + WL; ++l) {
            if (l < first || l >= last) continue;
            if (l < XL) {
                const uint32_t at = xo[l < XL ? l : 0] - off, place = to + (wave * XL + l) * 1024;
                if (!RAGGED || s + 1 < S) {
                    load_to_lds(xb + s * KB, at, place);
                } else {
                    // (the last row of all: its last piece may pass the tensor's end)
                    const int8_t* const from = xb + s * KB + at;
                    if (from + 16 <= end)
                        load_to_lds(xb + s * KB, at, place);
                    else
                        *reinterpret_cast<i32x4*>(lds + (place - lds0) + lane * 16) =
                            load_x<true>(from, 0, (int)(end - from), end);
                }
            } else {
                const int part = wave * WL + l - XL, nb = nb0 + part / 8;
                load_to_lds(A.w + ((int64_t)(nb < NB ? nb : NB - 1) * S + s) * WBLOCK + part % 8 * 1024, lane * 16,
                            to + BM * KB + part * 1024);
            }
        }
    };
    i32x4 x[2][MT], w[2][NT];
    i32x4 acc[MT][NT];
    // part of the fragments of half a step: four of the weight's, or the rows'
    constexpr int PARTS = NT / 4 + 1;
    auto read = [&](int s, int half, int part) {
        const int8_t* const at = lds + (s & 1) * STAGE;
        if (part < NT / 4) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                w[half][part * 4 + j] = *reinterpret_cast<const i32x4*>(at + wr + half * 4096 + part * WBLOCK + j * 1024);
        } else {
            const int p = ((half * 4 + (lane >> 4)) ^ (lane & 7)) << 4;
#pragma unroll
            for (int i = 0; i < MT; ++i) x[half][i] = *reinterpret_cast<const i32x4*>(at + xr + p + i * 16 * KB);
        }
    };
    // half a step; the fragments of the next half, of step `rs`, and the loads
    // of step `fs` (negative: none) are issued between its products, lest they
    // hold them up
    auto half_step = [&](int half, int rs, int fs) {
#pragma unroll
        for (int i = 0; i < MT; ++i) {
#pragma unroll
            for (int j = 0; j < NT; ++j) acc[i][j] = mfma(x[half][i], w[half][j], acc[i][j]);
            __builtin_amdgcn_sched_barrier(0);
            if (rs >= 0 && i < PARTS) read(rs, half ^ 1, i);
            if (fs >= 0) fill(fs, i * (XL + WL) / MT, (i + 1) * (XL + WL) / MT);
            __builtin_amdgcn_sched_barrier(0);
        }
    };

    int64_t b = blockIdx.x;
    Place at = place(b);
    if (!at.there) return;
    begin(at, 0);
    fill(0, 0, XL + WL);
    if (S > 1) fill(1, 0, XL + WL);
    bool drained = true;
    for (int turn = 0; at.there; turn ^= 1) {
        // the first step is there; what may be on its way: the second one, and
        // the stores of a whole tile before, one for each four sums.  (Of a last
        // step that load_x reads there may be fewer loads, but it waits for its
        // own, and so for all before them)
        if (drained || S == 1)
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        else
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(XL + WL + MT * NT < 63 ? XL + WL + MT * NT : 63) : "memory");
        b += gridDim.x;
        at = place(b);
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
#pragma unroll
        for (int p = 0; p < PARTS; ++p) read(0, 0, p);
        for (int s = 0; s + 1 < S; ++s) {
            half_step(0, s, -1);
            // the loads of step s + 1 are there, and step s is read to its end
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
            half_step(1, s + 1, s + 2 < S ? s + 2 : -1);
        }
        half_step(0, S - 1, -1);
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        const int64_t m = m0 + wm;
        const int nb = nb0 + wn;
        if (at.there) {
            begin(at, turn ^ 1);
            fill(0, 0, XL + WL);
            if (S > 1) fill(1, 0, XL + WL);
        }
        half_step(1, -1, -1);

        const float* const ls = scales + turn * (BM + BN);
        const uint32_t oo = ((uint32_t)(lane >> 4) * 4 * (uint32_t)A.out_stride + (lane & 15) * 4) * sizeof(T);
        float xs[MT][4];
#pragma unroll
        for (int i = 0; i < MT; ++i) IO<float, 4>::load(ls + BN + wm + i * 16 + (lane >> 4) * 4, xs[i]);
        Columns<T> cols[NT / 4];
#pragma unroll
        for (int j = 0; j < NT / 4; ++j) cols[j].load_mixed(A, ls + (wn + j) * 64, (nb + j) * 64, lane);
        // (of a whole tile: a store for each four sums)
        const bool whole = m + MT * 16 <= A.M && (nb + NT / 4) * 64 <= A.N;
        drained = !whole;
#pragma unroll
        for (int j = 0; j < NT; j += 4) {
            const Columns<T>& c = cols[j / 4];
            if (whole) {
                char* const base = reinterpret_cast<char*>(reinterpret_cast<T*>(A.out) + m * A.out_stride + (nb + j / 4) * 64);
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        float t[4];
                        c.row(xs[i][r], r, acc[i][j], acc[i][j + 1], acc[i][j + 2], acc[i][j + 3], t);
                        put_four<T, PAST>(reinterpret_cast<T*>(base + (i * 16 + r) * A.out_stride * (int64_t)sizeof(T) + oo), t);
                    }
            } else {
#pragma unroll
                for (int i = 0; i < MT; ++i)
                    c.store(A, m + i * 16 + (lane >> 4) * 4, xs[i], acc[i][j], acc[i][j + 1], acc[i][j + 2],
                            acc[i][j + 3]);
            }
        }
    }
}

// Many rows of at most KS * 128 columns: a block keeps a panel of the weight
// in LDS and its wavefronts stream rows past it, MI * 16 at a time, which they
// read straight into registers and hold there for all of the panel's columns.
// Nothing waits for another wavefront once the panel is there.
template <typename T, int KS, int MI, int WAVES, bool NT, bool SHIFT>
__global__ __launch_bounds__(WAVES * 64, 1) void linear8_stream_kernel(Linear8Args A, StreamArgs G) {
    extern __shared__ int8_t lds[];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    // the blocks of one run of rows sit on one die, one for each panel
    const int die = blockIdx.x & 7, at = blockIdx.x >> 3;
    const int panel = at % G.panels;
    const int64_t run = (int64_t)(at / G.panels) * 8 + die, runs = (int64_t)(gridDim.x >> 3) / G.panels * 8;
    const int NB = (A.N + 63) / 64, nb0 = panel * G.width;
    const int nbs = NB - nb0 < G.width ? NB - nb0 : G.width;  // blocks of 64 output columns
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) int8_t*)lds;
    for (int c = wave; c < nbs * KS * (WBLOCK / 1024); c += WAVES)
        load_to_lds(A.w + (int64_t)nb0 * KS * WBLOCK + c * 1024, lane * 16, lds0 + c * 1024);
    // scales and biases beside it: read from memory, a wavefront would wait for
    // its own stores each time
    float* const ls = reinterpret_cast<float*>(lds + G.width * KS * WBLOCK);
    float* const lb = ls + G.width * 64;
    for (int c = tid; c < nbs * 64; c += WAVES * 64) {
        const int n = nb0 * 64 + c;
        ls[c] = n < A.N ? A.ws[n] : 0.0f;
        lb[c] = n < A.N && A.bias ? IO<T, 1>::load1(reinterpret_cast<const T*>(A.bias) + n) : 0.0f;
    }
    // a lane's place in 16 rows, 32 bits beside an address that the lanes share
    const uint32_t xo = (uint32_t)(lane & 15) * (uint32_t)A.x_stride + (lane >> 4) * 16;
    const uint32_t oo = ((uint32_t)(lane >> 4) * 4 * (uint32_t)A.out_stride + (lane & 15) * 4) * sizeof(T);
    const int8_t* const end = A.x + (A.M - 1) * A.x_stride + A.K;
    const int64_t tiles = (A.M + MI * 16 - 1) / (MI * 16);
    const int part = wave % G.split, teams = WAVES / G.split;
    i32x4 x[KS * 2][MI];
    float xs[MI][4];
    auto load = [&](int64_t tile) {
        const int64_t m0 = tile * (MI * 16);
#pragma unroll
        for (int i = 0; i < MI; ++i) load_scales(A, m0 + i * 16 + (lane >> 4) * 4, xs[i]);
        const int8_t* const base = A.x + m0 * A.x_stride;
        if (base + (MI * 16 - 1) * A.x_stride + KS * KB + (SHIFT ? 4 : 0) <= end && (!SHIFT || tile > 0)) {
            // (what follows a row's end counts for nothing, and lies in the tensor)
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int k = 0; k < KS * 2; ++k)
                    x[k][i] = SHIFT ? load_shifted(base + i * 16 * A.x_stride + k * 64 + xo)
                                    : load_x<false>(base + i * 16 * A.x_stride + k * 64 + xo, 0, A.K, end);
        } else {
#pragma unroll
            for (int i = 0; i < MI; ++i) {
                const int64_t m = m0 + i * 16 + (lane & 15);
                const int8_t* const row = A.x + (m < A.M ? m : A.M - 1) * A.x_stride;
#pragma unroll
                for (int k = 0; k < KS * 2; ++k) {
                    const int at = k * 64 + (lane >> 4) * 16;
                    x[k][i] = k < KS * 2 - 2 ? load_x<false>(row, at, A.K, end) : load_x<true>(row, at, A.K, end);
                }
            }
        }
    };
    const int64_t step = runs * teams;
    int64_t tile = run + runs * (wave / G.split);
    if (tile < tiles) load(tile);
    // the panel is there
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    while (tile < tiles) {
        const int64_t m0 = tile * (MI * 16);
        for (int nb = part; nb < nbs; nb += G.split) {
            const int8_t* const w = lds + nb * KS * WBLOCK + lane * 16;
            i32x4 acc[4][MI] = {};
#pragma unroll
            for (int k = 0; k < KS * 2; ++k)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const i32x4 b = *reinterpret_cast<const i32x4*>(w + k * 4096 + j * 1024);
#pragma unroll
                    for (int i = 0; i < MI; ++i) acc[j][i] = mfma(x[k][i], b, acc[j][i]);
                }
            Columns<T> c;
            c.load_lds(ls, lb, nb, (nb0 + nb) * 64, lane);
            if (m0 + MI * 16 <= A.M && (nb0 + nb + 1) * 64 <= A.N) {
                char* const base = reinterpret_cast<char*>(reinterpret_cast<T*>(A.out) + m0 * A.out_stride + (nb0 + nb) * 64);
#pragma unroll
                for (int i = 0; i < MI; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        float t[4];
                        c.row(xs[i][r], r, acc[0][i], acc[1][i], acc[2][i], acc[3][i], t);
                        put_four<T, NT>(reinterpret_cast<T*>(base + (i * 16 + r) * A.out_stride * (int64_t)sizeof(T) + oo), t);
                    }
            } else {
#pragma unroll
                for (int i = 0; i < MI; ++i)
                    c.store(A, m0 + i * 16 + (lane >> 4) * 4, xs[i], acc[0][i], acc[1][i], acc[2][i], acc[3][i]);
            }
        }
        tile += step;
        if (tile < tiles) load(tile);
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
        const int64_t n = b / KS * 64 + r * 4 + j;
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

template <typename T, int BM, int BN, int WM, int BLOCKS, bool RAGGED, bool PAST>
void launch_deep_of(const Linear8Args& a, hipStream_t s) {
    TileArgs g;
    g.tm = (a.M + BM - 1) / BM;
    g.tn = (a.N + BN - 1) / BN;
    g.tiles = g.tm * g.tn;
    g.padded = (g.tiles + 7) / 8 * 8;
    g.group = 8;
    const int64_t blocks = g.padded < 256 * BLOCKS ? g.padded : 256 * BLOCKS;
    hipLaunchKernelGGL((linear8_deep_kernel<T, BM, BN, WM, BLOCKS, RAGGED, PAST>), dim3((unsigned)blocks), dim3(WM * 128),
                       2 * (BM + BN) * KB + 2 * (BM + BN) * 4, s, a, g);
}

template <typename T, int BM, int BN, int WM, int BLOCKS>
void launch_deep(const Linear8Args& a, hipStream_t s) {
    const bool past = a.M * a.N * (int64_t)sizeof(T) > PAST_CACHES;
    if (a.K % 16)
        return past ? launch_deep_of<T, BM, BN, WM, BLOCKS, true, true>(a, s)
                    : launch_deep_of<T, BM, BN, WM, BLOCKS, true, false>(a, s);
    return past ? launch_deep_of<T, BM, BN, WM, BLOCKS, false, true>(a, s)
                : launch_deep_of<T, BM, BN, WM, BLOCKS, false, false>(a, s);
}

template <typename T, int MI, int NJ>
void launch_few(const Linear8Args& a, int waves, hipStream_t s) {
    const int64_t blocks = ((a.M + MI * 16 - 1) / (MI * 16)) * ((a.N + 63) / 64 * (4 / NJ));
    hipLaunchKernelGGL((linear8_few_kernel<T, MI, NJ>), dim3((unsigned)blocks), dim3(waves * 64),
                       waves * MI * NJ * 1024, s, a, waves);
}

template <typename T, int KS, int MI, int WAVES, bool NT, bool SHIFT>
void launch_stream(const Linear8Args& a, hipStream_t s) {
    constexpr int CUS = 32;  // of a die
    const int NB = (a.N + 63) / 64, most = LDS_BYTES / (KS * WBLOCK + 512);
    StreamArgs g;
    g.panels = (NB + most - 1) / most;  // (at most CUS: of 64 blocks at least two a panel)
    g.width = (NB + g.panels - 1) / g.panels;
    const int runs = CUS / g.panels * 8;
    const int64_t tiles = (a.M + MI * 16 - 1) / (MI * 16);
    g.split = 1;
    while (WAVES % (g.split * 2) == 0 && g.split < g.width && tiles * g.split < runs * WAVES / 2) g.split *= 2;
    hipLaunchKernelGGL((linear8_stream_kernel<T, KS, MI, WAVES, NT, SHIFT>), dim3((unsigned)(runs * g.panels)),
                       dim3(WAVES * 64), g.width * (KS * WBLOCK + 512), s, a, g);
}

template <typename T, int MI, int WAVES, bool NT, bool SHIFT>
void launch_streams_of(const Linear8Args& a, hipStream_t s) {
    const int KS = (a.K + KB - 1) / KB;
    if (KS == 1) return launch_stream<T, 1, MI, WAVES, NT, SHIFT>(a, s);
    if (KS == 2) return launch_stream<T, 2, MI, WAVES, NT, SHIFT>(a, s);
    if (KS == 3) return launch_stream<T, 3, MI, WAVES, NT, SHIFT>(a, s);
    if (KS == 4) return launch_stream<T, 4, MI, WAVES, NT, SHIFT>(a, s);
    if (KS == 5) return launch_stream<T, 5, MI, WAVES, NT, SHIFT>(a, s);
    if (KS == 6) return launch_stream<T, 6, MI, WAVES, NT, SHIFT>(a, s);
    if (KS == 7) return launch_stream<T, 7, MI, WAVES, NT, SHIFT>(a, s);
    return launch_stream<T, 8, MI, WAVES, NT, SHIFT>(a, s);
}

template <typename T, int MI, int WAVES, bool NT>
void launch_streams(const Linear8Args& a, hipStream_t s) {
    if ((a.x_stride | (int64_t)(uintptr_t)a.x) & 3) return launch_streams_of<T, MI, WAVES, NT, true>(a, s);
    launch_streams_of<T, MI, WAVES, NT, false>(a, s);
}

enum Tile { AUTO, FEW, TILE64, TILE128, DEEP128, DEEP256, STREAM, STREAM_PAST };

// The kernel for a product, by what 10 to 300,000 rows of 128 to 4,096 columns
// measured (us; a call of few rows takes 6.5 on the host):
//  - few rows, or so few products for their depth that one block after another
//    would read long sums: FEW (2,048 to 2,048 columns, 130 rows 9.2, DEEP128
//    11.0, 300 rows 16.6 and 11.6; 4,096 to 1,024, 200 rows 11 and 18; at addresses
//    that are no whole words half as many: 3,001 to 1,000, 400 rows 31, TILE64 19)
//  - rows of up to 512 columns, and up to 1,024 where they do not start on 16
//    bytes: STREAM (100,000 rows, 512 to 512 columns 34, DEEP128 40, TILE128 60;
//    600 to 512 in rows of 600 bytes 47, 53, 72; 1,024 to 512 73, 68, 92)
//  - other rows that start on whole words: DEEP256 where sums are long and the last
//    round of tiles is not much shorter than the chip is wide (20,000 rows, 4,096
//    to 512 columns, 158 tiles 45, DEEP128 53; 1,000 rows, 64 tiles 38, 18.5;
//    20,000 rows, 1,024 to 1,024 columns 37, 27), else DEEP128
//  - what is left, wider rows at any address: tiles through registers, small
//    ones where those fill the chip (4,000 rows, 1,000 to 300 columns 11.3 and 14;
//    20,000 rows 23 and 19)
Tile choose(const Linear8Args& a, int es, int KS, bool words, bool lines, bool streams) {
    const int64_t macs = (a.M + 63) / 64 * 64 * a.N * a.K;
    if (a.M <= 64 || (KS > 4 && macs <= KS * (words ? 65000000ll : 30000000ll))) return FEW;
    if (streams && (KS <= 4 || !lines)) return a.M * a.N * es > PAST_CACHES ? STREAM_PAST : STREAM;
    if (!words) return ((a.M + 63) / 64) * ((a.N + 63) / 64) <= 512 ? TILE64 : TILE128;
    const int64_t big = ((a.M + 255) / 256) * ((a.N + 255) / 256);
    return KS >= 16 && a.N > 256 && big * 100 >= (big + 255) / 256 * 256 * 55 ? DEEP256 : DEEP128;
}

template <typename T>
void launch_t(const Linear8Args& a, int tile, hipStream_t s) {
    const int KS = (a.K + KB - 1) / KB, waves = KS < 16 ? KS : 16;
    // places within a tile of rows fit 32 bits; rows that start on whole words, as
    // loads into LDS take them, or on 16 bytes; rows that a wavefront's registers hold
    const bool near = a.x_stride < (1 << 24) && a.out_stride < (1 << 24);
    const int64_t place = a.x_stride | (int64_t)(uintptr_t)a.x;
    const bool words = near && place % 4 == 0, lines = place % 16 == 0, streams = near && KS <= 8 && a.N <= 4096;
    switch (tile ? tile : choose(a, sizeof(T), KS, words, lines, streams)) {
        case FEW: return a.M > 16 ? launch_few<T, 4, 1>(a, waves, s) : launch_few<T, 1, 1>(a, waves, s);
        case TILE64: return launch_tile<T, 64, 64, 2, 1, 2>(a, s);
        case DEEP128:
            if (words) return launch_deep<T, 128, 128, 2, 2>(a, s);
            break;
        case DEEP256:
            if (words) return launch_deep<T, 256, 256, 4, 1>(a, s);
            break;
        case STREAM:
            if (streams) return launch_streams<T, 1, 16, false>(a, s);
            break;
        case STREAM_PAST:
            if (streams) return launch_streams<T, 1, 16, true>(a, s);
            break;
        default: break;
    }
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
