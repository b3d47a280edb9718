// Dot-product attention over a graph's edges, forward and backward:
//
//   s_e = scale q[v, h] . k[u, j] + bias[e, h]     (j the key head of query head h)
//   out[v, h, :] = sum_e softmax(s)_e v[u, j, :]   over the in-edges e = (u, v)
//
// in one pass over each destination's in-edges, with the running maximum and
// sum of the softmax, so no score is written.  An edge gathers one row of keys
// and one of values; a lane holds VEC columns of a key head, the vectors of a
// head in a power of two of neighbouring lanes, so that a head's dot product
// is one reduction over them (cross-lane moves up to 16 lanes, shuffles beyond)
// and every lane of the head gets it.  Heads
// beyond one wavefront's lanes are slices of the grid.  Of the R query heads
// that share a key head, a lane takes RC at once in registers (each key and
// value row is then gathered and widened once for them), RL neighbouring runs
// of lanes take as many beside each other, and what is left takes turns; where
// R is no multiple, the last ones do the last head's work again and write
// nothing.
//
// Dot products and the sums over the edges of one wavefront's share of a
// row are fp32; the partial results of a long row's segments are joined in
// fp64 in segment order.
//
// What bounds it is the gathers, once the dot products are made of packed bf16
// pairs and the scores of a head are formed once:
//   232,965 rows, 114.6M edges sorted by destination, 8 heads of 16 bf16: 2.97
//     ms, 58 GB through L2 at 19.4 TB/s (13 GB past it);
//   232,965 rows, 14.3M edges, 8 heads of 16 fp32: forward 1.06 ms, backward
//     by destination 1.08, by source 1.20, 7.7 to 8.2 GB past L2 at 7.0 to 7.3
//     TB/s, as fast as rows at random come from there;
//   262,144 rows of 32 edges, 8 query and 2 key heads of 32 bf16, a bias per
//     head: forward 0.37 ms (2.6 GB past L2 at 7.0 TB/s), by destination 0.49
//     (5.7 TB/s, the vector units three quarters busy), by source 1.54 (12 GB
//     at 7.8 TB/s: four query heads' rows and a record an edge);
//   a row of 100,000 edges, 8 and 2 heads of 64 bf16: 15 us and 8 us to join;
//   20,000 rows, 109,170 edges, 8 heads of 8 fp32: 12 to 14 us a pass and 4 us
//     to join, latencies.
#include <type_traits>

#include "words.h"

namespace gnnk {

namespace {

// a lane's place in the row of heads (a slice of them)
struct Place {
    int j;     // key head
    int rl;    // which run of the key head's lanes
    int c;     // first column within the head
    int skip;  // columns that the vector before holds too
    bool own;  // the lane belongs to a head
    bool act;  // and holds a vector of it
    bool first;  // the first one
};
template <int VEC>
__device__ __forceinline__ Place place_of(const DotArgs& D, int lig) {
    const int x = lig >> D.log2HL, f = lig & ((1 << D.log2HL) - 1);
    const int hl = x >> D.log2RL;
    const int j = (D.slice0 + (int)blockIdx.y) * D.heads_slice + hl;
    Place p;
    p.own = hl < D.heads_slice && j < D.K;
    p.act = p.own && f < D.FV;
    p.j = p.own ? j : 0;
    p.rl = x & ((1 << D.log2RL) - 1);
    const int at = f * VEC, last = D.F - VEC;
    p.c = p.act ? (at < last ? at : last) : 0;
    p.skip = p.act && at > last ? at - last : 0;
    p.first = p.act && f == 0;
    return p;
}

// a lane's share of a dot product of two rows in words, without the columns
// it shares
template <typename T, int VEC, bool OV>
__device__ __forceinline__ float share(const float* x, const float* y, const Place& p) {
    using W = Words<T, VEC>;
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < W::N; ++i) {
        if constexpr (W::PAIRS) {
            float yi = y[i], xi = x[i];
            if constexpr (OV) {
                // (both, so that an infinite value of a shared column meets no 0)
                const uint32_t m = (2 * i < p.skip ? 0u : 0xFFFFu) | (2 * i + 1 < p.skip ? 0u : 0xFFFF0000u);
                yi = __uint_as_float(__float_as_uint(yi) & m);
                xi = __uint_as_float(__float_as_uint(xi) & m);
            }
            s = __builtin_amdgcn_fdot2_f32_bf16(pair(xi), pair(yi), s, false);
        } else if constexpr (OV) {
            s = i < p.skip ? s : fmaf(x[i], y[i], s);
        } else {
            s = fmaf(x[i], y[i], s);
        }
    }
    return p.act ? s : 0.0f;
}

// a row's own operand of the scores: fp32 scaled once, bf16 as it is (its
// totals are scaled instead)
template <typename T, int VEC>
__device__ __forceinline__ void own_row(const DotArgs& D, const void* base, int64_t at, float* w) {
    using W = Words<T, VEC>;
    IO<typename W::type, VEC>::load(reinterpret_cast<const typename W::type*>(base) + at, w);
    if constexpr (!W::PAIRS) {
#pragma unroll
        for (int i = 0; i < W::N; ++i) w[i] *= D.scale;
    }
}
template <typename T, int VEC>
__device__ __forceinline__ void row_words(const void* base, int64_t at, float* w) {
    using W = Words<T, VEC>;
    IO<typename W::type, VEC>::load(reinterpret_cast<const typename W::type*>(base) + at, w);
}

// ---------------------------------------------------------------------------
// the walk over a row's edges

constexpr int U = 4;  // edges in flight per lane group

// what U edges bring to a lane: words of the two gathered rows, the record of
// the source pass, the bias of RC query heads
template <int N, int RC>
struct Batch {
    float a[U][N], b[U][N];
    float4 rec[U];
    float bias[U][RC];
    int32_t ed[U];
    bool ok[U];
};

struct Ids {
    int32_t nb[U], ed[U];
};

__device__ __forceinline__ void spread_quad(int32_t x, int32_t* v) {
    v[0] = quad_lane<0>(x);
    v[1] = quad_lane<1>(x);
    v[2] = quad_lane<2>(x);
    v[3] = quad_lane<3>(x);
}

// Ids of the positions p .. p + U - 1 (those past e take p's): lane u of each
// quad loads one and hands it to the quad.  A load of all four in every lane
// took the loads' return path as long as a gather.
template <bool EDGES>
__device__ __forceinline__ void load_ids(const CsrDev& C, int32_t p, int32_t e, Ids& id) {
    static_assert(U == 4, "an id a lane of a quad");
    int32_t x = p + (__lane_id() & 3);
    x = x < e ? x : p;
    spread_quad(C.idx[x], id.nb);
    if constexpr (EDGES) {
        if (C.eid) {
            spread_quad(C.eid[x], id.ed);
        } else {
#pragma unroll
            for (int u = 0; u < U; ++u) id.ed[u] = p + u < e ? p + u : p;
        }
    }
}

// a row of a node table; FAST: byte offsets of 32 bits (the host checks)
template <typename T, int VEC, bool FAST>
__device__ __forceinline__ void gather(const OperandDev& o, int32_t nb, int col, float* w) {
    using W = typename Words<T, VEC>::type;
    if constexpr (FAST) {
        const uint32_t off = __umul24((uint32_t)nb, (uint32_t)o.stride * (uint32_t)sizeof(T)) +
                             (uint32_t)col * (uint32_t)sizeof(T);
        IO<W, VEC>::load(reinterpret_cast<const W*>(reinterpret_cast<const char*>(o.data) + off), w);
    } else {
        IO<W, VEC>::load(reinterpret_cast<const W*>(o.data) + (uint64_t)(uint32_t)nb * (uint32_t)o.stride + col, w);
    }
}

// The loads of a batch: columns col of the tables a and b, with REC the record
// of (neighbour, head hq), with BIAS the values of heads hq .. hq + RC - 1, RC
// being the heads whose scores the lane takes.
template <typename T, int VEC, int RC, bool FAST, bool BIAS, bool REC>
__device__ __forceinline__ void issue(const EngineArgs& A, const DotArgs& D, const Ids& id, int col, int hq,
                                      Batch<Words<T, VEC>::N, RC>& x) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
        gather<T, VEC, FAST>(A.a, id.nb[u], col, x.a[u]);
        gather<T, VEC, FAST>(A.b, id.nb[u], col, x.b[u]);
        if constexpr (REC && FAST)
            x.rec[u] = *reinterpret_cast<const float4*>(
                reinterpret_cast<const char*>(D.rec) +
                (__umul24((uint32_t)id.nb[u], (uint32_t)D.H * 16u) + (uint32_t)hq * 16u));
        else if constexpr (REC) x.rec[u] = D.rec[(uint64_t)(uint32_t)id.nb[u] * (uint32_t)D.H + (uint32_t)hq];
    }
    if constexpr (BIAS) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            x.ed[u] = id.ed[u];
            const T* b = reinterpret_cast<const T*>(D.bias) +
                         (uint64_t)(uint32_t)id.ed[u] * (uint32_t)D.bias_stride;
            if (D.bias_per_head) {
                if (RC <= 2 || D.R % (RC << D.log2RL) == 0) {  // (2: of key heads that two share)
                    IO<T, RC>::load(b + hq, x.bias[u]);
                } else {
#pragma unroll
                    for (int r = 0; r < RC; ++r) {
                        const int h = hq + r < D.H ? hq + r : D.H - 1;  // (past the key head's: not used)
                        x.bias[u][r] = IO<T, 1>::load1(b + h);
                    }
                }
            } else {
                x.bias[u][0] = IO<T, 1>::load1(b);
#pragma unroll
                for (int r = 1; r < RC; ++r) x.bias[u][r] = x.bias[u][0];
            }
        }
    }
}

// A lane group takes U edges at b + start, b + start + stride, ... of a row
// [b, e): the groups of a wavefront side by side (start U g, stride U G), or a
// group its own row (0, U).  The ids of a batch load behind the gathers of the
// one before it.  (The next batch's gathers in flight while one is summed
// took registers that wavefronts need: 8.4M edges, 8 query and 2 key heads of
// 32 bf16, forward 499 -> 533 us, source pass 1,537 -> 1,810.)
template <typename T, int VEC, int RC, bool FAST, bool BIAS, bool REC, class F>
__device__ __forceinline__ void walk(const EngineArgs& A, const DotArgs& D, int32_t b, int32_t e, int32_t start,
                                     int32_t stride, int col, int hq, F& sink) {
    int32_t p = b + start;
    if (p >= e) return;
    Ids id;
    Batch<Words<T, VEC>::N, RC> x;
    load_ids<BIAS>(A.csr, p, e, id);
    issue<T, VEC, RC, FAST, BIAS, REC>(A, D, id, col, hq, x);
    int32_t pn = p + stride;
    load_ids<BIAS>(A.csr, pn < e ? pn : p, e, id);
    while (pn < e) {
        sink.template take<true>(x);
        issue<T, VEC, RC, FAST, BIAS, REC>(A, D, id, col, hq, x);
        p = pn;
        pn += stride;
        load_ids<BIAS>(A.csr, pn < e ? pn : p, e, id);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) x.ok[u] = p + u < e;
    sink.template take<false>(x);
}

// scores of a batch for one query head from their totals; gone[u]: the slot
// lies outside the row or is masked
template <typename T, int RC, bool BIAS, bool ALL, class B>
__device__ __forceinline__ void scores(const DotArgs& D, const B& x, int r, float* s, bool* gone) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
        gone[u] = ALL ? false : !x.ok[u];
        if constexpr (Words<T, 2>::PAIRS) s[u] = BIAS ? fmaf(s[u], D.scale, x.bias[u][r]) : s[u] * D.scale;
        else if constexpr (BIAS) s[u] += x.bias[u][r];
        if constexpr (BIAS) gone[u] |= x.bias[u][r] == -INFINITY;
    }
}

// ---------------------------------------------------------------------------
// forward

// the RC query heads that a lane takes in one turn
template <int RC>
struct Heads {
    int first, last;  // and the last one of its key head
    __device__ __forceinline__ Heads(const DotArgs& D, const Place& p, int turn)
        : first(p.j * D.R + turn + p.rl * RC), last(p.j * D.R + D.R - 1) {}
    __device__ __forceinline__ bool has(int r) const { return first + r <= last; }
    __device__ __forceinline__ int at(int r) const { return has(r) ? first + r : last; }
};

// the weight of a slot that lies outside the row or is masked: a zero that no
// exponential gives
constexpr float GONE = -0.0f;
__device__ __forceinline__ bool is_gone(float w) { return __float_as_uint(w) == 0x80000000u; }

// Of four query heads in registers (SPLIT, heads of at least four lanes), the
// totals are shared out: lane r of each quad keeps the scores, maximum and sum
// of head r and hands its weights around, a quarter of the exponentials and
// comparisons that every lane would make for itself.
template <typename T, int VEC, int RC, bool SPLIT, bool OV, bool BIAS>
struct Forward {
    static constexpr int SC = SPLIT ? 1 : RC;  // heads whose scores a lane keeps
    const DotArgs& D;
    const Place& p;
    Heads<RC> hq;  // the lane's query heads
    using W = Words<T, VEC>;
    float q[RC][W::N];
    float m[SC], l[SC], acc[RC][VEC];

    __device__ __forceinline__ Forward(const DotArgs& D_, const Place& p_, int turn, int64_t row)
        : D(D_), p(p_), hq(D_, p_, turn) {
#pragma unroll
        for (int r = 0; r < RC; ++r) {
            own_row<T, VEC>(D, D.q, row * D.q_stride + (int64_t)hq.at(r) * D.F + p.c, q[r]);
#pragma unroll
            for (int i = 0; i < VEC; ++i) acc[r][i] = 0.0f;
        }
#pragma unroll
        for (int r = 0; r < SC; ++r) {
            m[r] = -INFINITY;
            l[r] = 0.0f;
        }
    }
    // the first head whose scores the lane keeps
    __device__ __forceinline__ int score_head() const { return SPLIT ? hq.at(__lane_id() & 3) : hq.at(0); }
    // a value that the lane of head r keeps
    template <int R>
    static __device__ __forceinline__ float of(const float* v) {
        if constexpr (SPLIT) return quad_lane<R>(v[0]);
        else return v[R];
    }
    template <bool ALL, class B>
    __device__ __forceinline__ void take(const B& x) {
        float s[RC * U];
#pragma unroll
        for (int r = 0; r < RC; ++r)
#pragma unroll
            for (int u = 0; u < U; ++u) s[r * U + u] = share<T, VEC, OV>(q[r], x.a[u], p);
        if constexpr (SPLIT) quad_totals<U>(s, 1 << D.log2HL, s);
        else run_totals<RC * U>(s, 1 << D.log2HL);
        bool gone[SC][U];
        float f[SC];
        bool grew = false;
#pragma unroll
        for (int r = 0; r < SC; ++r) {
            float* sr = s + r * U;
            scores<T, SC, BIAS, ALL>(D, x, r, sr, gone[r]);
            float mn = m[r];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                sr[u] = gone[r][u] ? -INFINITY : sr[u];
                mn = fmaxf(mn, sr[u]);
            }
            const float at = mn == -INFINITY ? 0.0f : mn;
            grew |= mn > m[r];
            f[r] = exp_le0(m[r] - at);
            m[r] = mn;
#pragma unroll
            for (int u = 0; u < U; ++u) sr[u] = gone[r][u] ? GONE : exp_le0(sr[u] - at);  // the weights
        }
        if (__ballot(grew) != 0ull) {
#pragma unroll
            for (int r = 0; r < SC; ++r) l[r] *= f[r];
            each([&](auto R) {
                const float g = of<R()>(f);
#pragma unroll
                for (int i = 0; i < VEC; ++i) acc[R()][i] *= g;
            });
        }
#pragma unroll
        for (int r = 0; r < SC; ++r)
#pragma unroll
            for (int u = 0; u < U; ++u) l[r] += s[r * U + u];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float v[VEC];
#pragma unroll
            for (int i = 0; i < VEC; ++i) v[i] = W::at(x.b[u], i);
            each([&](auto R) {
                float w;
                if constexpr (SPLIT) w = quad_lane<R()>(s[u]);
                else w = s[R() * U + u];
                // (a slot that is gone adds nothing, whatever value it holds)
                if ((BIAS || !ALL) && is_gone(w)) return;
#pragma unroll
                for (int i = 0; i < VEC; ++i) acc[R()][i] = fmaf(w, v[i], acc[R()][i]);
            });
        }
    }
    // fn(integral constant r) for each query head in registers
    template <class F>
    static __device__ __forceinline__ void each(F fn) {
        heads<0>(fn);
    }
    template <int R, class F>
    static __device__ __forceinline__ void heads(F& fn) {
        if constexpr (R < RC) {
            fn(std::integral_constant<int, R>{});
            heads<R + 1>(fn);
        }
    }
    // the states of the wavefront's lane groups, pairwise
    __device__ __forceinline__ void join_groups(int L) {
        for (int x = L; x < WAVE; x <<= 1) {
            float f[SC], g[SC];
#pragma unroll
            for (int r = 0; r < SC; ++r) {
                const float om = __shfl_xor(m[r], x, WAVE), ol = __shfl_xor(l[r], x, WAVE);
                const float mn = fmaxf(m[r], om), at = mn == -INFINITY ? 0.0f : mn;
                f[r] = exp_le0(m[r] - at);
                g[r] = exp_le0(om - at);
                l[r] = l[r] * f[r] + ol * g[r];
                m[r] = mn;
            }
            each([&](auto R) {
                const float fr = of<R()>(f), gr = of<R()>(g);
#pragma unroll
                for (int i = 0; i < VEC; ++i)
                    acc[R()][i] = acc[R()][i] * fr + __shfl_xor(acc[R()][i], x, WAVE) * gr;
            });
        }
    }
    // fn(head, maximum, sum) in one lane for each of the heads
    template <class F>
    __device__ __forceinline__ void each_score(F fn) const {
        if constexpr (SPLIT) {
            const int x = __lane_id() & ((1 << D.log2HL) - 1);
            if (x < 4 && hq.has(x)) fn(score_head(), m[0], l[0]);
        } else if (p.first) {
#pragma unroll
            for (int r = 0; r < RC; ++r)
                if (hq.has(r)) fn(hq.at(r), m[r], l[r]);
        }
    }
};

// the statistics of a row's head: the maximum and 1 / sum
__device__ __forceinline__ void write_stats(const DotArgs& D, int64_t row, int hq, float m, float l) {
    if (!D.stats) return;
    float* st = D.stats + row * D.stats_stride + 2 * hq;
    st[0] = l == 0.0f ? 0.0f : m;
    st[1] = l == 0.0f ? 0.0f : 1.0f / l;
}

// the row of a wavefront's hub segment or big row (slot: its segment), or of
// the lane group's small row
struct Work {
    int64_t r, b, e;
    int slot;
};
__device__ __forceinline__ Work wave_work(const EngineArgs& A, int w) {
    Work k;
    if (w < A.sch.n_seg) {
        const int4 s = A.csr.segw[w];
        k = Work{s.x, s.y, s.z, s.w};
    } else {
        const int4 t = A.csr.rowt[A.sch.n_hub + (w - A.sch.n_seg)];
        k = Work{t.x, t.y, t.z, -1};
    }
    return Work{uniform64(k.r), uniform64(k.b), uniform64(k.e), k.slot};
}
__device__ __forceinline__ Work lane_work(const EngineArgs& A, int w, int G, int g) {
    const int64_t k = A.sch.n_big + (int64_t)(w - A.sch.w_big_end) * G + g;
    if (k >= A.sch.n_nz) return Work{-1, 0, 0, -1};
    const int4 t = A.csr.rowt[k];
    return Work{t.x, t.y, t.z, -1};
}
// rows without edges: fn(row) for each row of this lane group
template <class F>
__device__ __forceinline__ void empty_rows(const EngineArgs& A, int w, int G, int g, F fn) {
    const int64_t k0 = A.sch.n_nz + ((int64_t)(w - A.sch.w_small_end) * G + g) * A.sch.fill_rows_per_group;
    for (int x = 0; x < A.sch.fill_rows_per_group; ++x)
        if (k0 + x < A.sch.n_rows) fn((int64_t)A.csr.perm[k0 + x]);
}

template <typename T, int VEC, int RC, bool SPLIT, bool OV, bool BIAS, bool FAST>
__global__ __launch_bounds__(256, 3) void dot_forward_kernel(EngineArgs A, DotArgs D) {
    const int w = wave_id();
    if (w >= A.sch.w_total) return;
    const Lanes ln = lanes_of(A.geo);
    const int G = A.geo.G, L = A.geo.L;
    const Place p = place_of<VEC>(D, ln.lig);
    const int kcol = p.j * D.F + p.c, step = RC << D.log2RL;
    using State = Forward<T, VEC, RC, SPLIT, OV, BIAS>;
    if (w < A.sch.w_small_end) {
        const bool wave = w < A.sch.w_big_end;
        const Work k = wave ? wave_work(A, w) : lane_work(A, w, G, ln.g);
        const int64_t self = k.r >= 0 ? k.r : 0;
        for (int r = 0; r < D.R; r += step) {
            State st(D, p, r, self);
            walk<T, VEC, State::SC, FAST, BIAS, false>(A, D, (int32_t)k.b, (int32_t)k.e, wave ? U * ln.g : 0,
                                                       wave ? U * G : U, kcol, st.score_head(), st);
            if (wave) st.join_groups(L);
            float il[State::SC];
#pragma unroll
            for (int x = 0; x < State::SC; ++x) il[x] = st.l[x] == 0.0f ? 0.0f : 1.0f / st.l[x];
            float ih[RC];  // (lanes read each other's: before any of them is done)
            State::each([&](auto x) { ih[x()] = State::template of<x()>(il); });
            if ((wave && ln.g != 0) || k.r < 0 || !(p.act || SPLIT)) continue;
            const int64_t W = (int64_t)D.H * D.F;
            const bool own = p.own;
            if (k.slot >= 0) {
                float* P = D.part + (int64_t)k.slot * D.part_stride;
                if (own)
                    st.each_score([&](int hq, float m, float l) {
                        P[W + 2 * hq] = m;
                        P[W + 2 * hq + 1] = l;
                    });
                if (!p.act) continue;
#pragma unroll
                for (int x = 0; x < RC; ++x)
                    if (st.hq.has(x))
#pragma unroll
                        for (int i = 0; i < VEC; ++i) P[(int64_t)st.hq.at(x) * D.F + p.c + i] = st.acc[x][i];
            } else {
                if (own) st.each_score([&](int hq, float m, float l) { write_stats(D, k.r, hq, m, l); });
                if (!p.act) continue;
#pragma unroll
                for (int x = 0; x < RC; ++x) {
#pragma unroll
                    for (int i = 0; i < VEC; ++i) st.acc[x][i] *= ih[x];
                    if (st.hq.has(x))
                        IO<T, VEC>::store(reinterpret_cast<T*>(D.out) + k.r * D.out_stride +
                                              (int64_t)st.hq.at(x) * D.F + p.c, st.acc[x]);
                }
            }
        }
    } else {
        empty_rows(A, w, G, ln.g, [&](int64_t row) {
            const float zero[VEC] = {};
            for (int r = p.rl; r < D.R && p.act; r += 1 << D.log2RL) {
                const int hq = p.j * D.R + r;
                IO<T, VEC>::store(reinterpret_cast<T*>(D.out) + row * D.out_stride + (int64_t)hq * D.F + p.c, zero);
                if (p.first) write_stats(D, row, hq, 0.0f, 0.0f);
            }
        });
    }
}

// Hub rows: the states of a row's segments joined.  A workgroup takes `cols`
// columns (a power of two up to 64) of one row, its threads the columns of
// every (threads / cols)-th segment, U loads in flight; join_runs then joins
// the runs, first those of a wavefront.  A few columns and many runs where
// rows have many segments (one node of 100,000 edges has 1,563).  30,900 hub
// rows of two segments and more of 128 columns: 78 us, with 8 or 16 loads in flight
// 91 and more; one row of 1,563 segments of 512 columns 8.5 us either way, of
// which 4 are any such kernel's.
template <int N, class Add>
__device__ __forceinline__ void join_runs(double (*red)[256], double* v, int cols, Add add) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6, c = lane & (cols - 1);
    auto lanes = [&] {
        for (int x = cols; x < WAVE; x <<= 1) {
            double o[N];
#pragma unroll
            for (int i = 0; i < N; ++i) o[i] = __shfl_xor(v[i], x, WAVE);
            add(v, o);
        }
    };
    lanes();
    if (lane < cols)
#pragma unroll
        for (int i = 0; i < N; ++i) red[i][wave * cols + c] = v[i];
    __syncthreads();
    if (wave != 0) return;
    for (int w = lane / cols, first = 1; w < waves; w += WAVE / cols, first = 0) {
        double o[N];
#pragma unroll
        for (int i = 0; i < N; ++i) o[i] = red[i][w * cols + c];
        if (first) {
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = o[i];
        } else {
            add(v, o);
        }
    }
    lanes();
}

template <typename T>
__global__ void dot_join_kernel(EngineArgs A, DotArgs D, int cols) {
    __shared__ double red[3][256];
    const int t = threadIdx.x, runs = blockDim.x / cols, run = t / cols, W = D.H * D.F;
    const int col = (int)blockIdx.y * cols + (t - run * cols);
    const int64_t row = A.csr.perm[blockIdx.x];
    const int s0 = A.csr.hub_off[blockIdx.x], s1 = A.csr.hub_off[blockIdx.x + 1];
    const bool ok = col < W;
    const int hq = ok ? col / D.F : 0;
    double v[3] = {-INFINITY, 0.0, 0.0};  // maximum, sum of weights, weighted sum
    auto raise = [&](double* x, float mn) {
        const double f = (double)exp_le0((float)x[0] - (mn == -INFINITY ? 0.0f : mn));
        x[0] = mn;
        x[1] *= f;
        x[2] *= f;
    };
    if (ok) {
        for (int s = s0 + run; s < s1; s += U * runs) {
            float pm[U], pl[U], pa[U], mn = (float)v[0];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int x = s + u * runs;
                const float* P = D.part + (uint64_t)(uint32_t)(x < s1 ? x : s) * (uint32_t)D.part_stride;
                pm[u] = P[W + 2 * hq];
                pl[u] = P[W + 2 * hq + 1];
                pa[u] = P[col];
            }
#pragma unroll
            for (int u = 0; u < U; ++u) mn = fmaxf(mn, pm[u]);
            raise(v, mn);
            const float at = mn == -INFINITY ? 0.0f : mn;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (s + u * runs < s1) {
                    const double g = (double)exp_le0(pm[u] - at);
                    v[1] = fma((double)pl[u], g, v[1]);
                    v[2] = fma((double)pa[u], g, v[2]);
                }
            }
        }
    }
    join_runs<3>(red, v, cols, [&](double* x, double* o) {
        const float mn = fmaxf((float)x[0], (float)o[0]);
        raise(x, mn);
        raise(o, mn);
        x[1] += o[1];
        x[2] += o[2];
    });
    if (t >= cols || !ok) return;
    IO<T, 1>::store1(reinterpret_cast<T*>(D.out) + row * D.out_stride + col, v[1] == 0.0 ? 0.0f : (float)(v[2] / v[1]));
    if (col % D.F == 0) write_stats(D, row, hq, (float)v[0], (float)v[1]);
}

// ---------------------------------------------------------------------------
// backward
//
//   da_e = dout[v] . v[u],  S = sum_in a_e da_e,  ds_e = a_e (da_e - S)
//   dq[v] = scale sum_in ds_e k[u]     dbias_e = ds_e
//   dk[u] = scale sum_out ds_e q[v]    dv[u] = sum_out a_e dout[v]
//
// a_e is recomputed from the forward's statistics.  The destination pass
// takes S0 = dout[v] . out[v], which is S but for the rounding of out, and
// sums w = a (da - S0), w k and a k; with delta = sum w, S = S0 + delta and
// dq = scale (sum w k - delta sum a k): what a bf16 out lost is put right, and
// no large values cancel.  It leaves a record {max, 1 / sum, S} per
// destination and head for the source pass, which walks the reverse graph's
// CSR and gathers q, dout and the record.

template <typename T, int VEC, int RC, bool SPLIT, bool OV, bool BIAS>
struct ToDst {
    using Fwd = Forward<T, VEC, RC, SPLIT, OV, BIAS>;
    static constexpr int SC = Fwd::SC;  // heads whose scores a lane keeps, as in the forward
    const DotArgs& D;
    const Place& p;
    Heads<RC> hq;  // the lane's query heads
    using W = Words<T, VEC>;
    float q[RC][W::N], dz[RC][W::N], m[SC], il[SC], S0[SC], delta[SC];
    float e1[RC][VEC], e2[RC][VEC];

    __device__ __forceinline__ ToDst(const DotArgs& D_, const Place& p_, int turn, int64_t row)
        : D(D_), p(p_), hq(D_, p_, turn) {
        float zo[RC];
#pragma unroll
        for (int r = 0; r < RC; ++r) {
            const int64_t c = (int64_t)hq.at(r) * D.F + p.c;
            float o[W::N];
            own_row<T, VEC>(D, D.q, row * D.q_stride + c, q[r]);
            row_words<T, VEC>(D.dz, row * D.dz_stride + c, dz[r]);
            row_words<T, VEC>(D.o, row * D.o_stride + c, o);
            zo[r] = share<T, VEC, OV>(dz[r], o, p);
#pragma unroll
            for (int i = 0; i < VEC; ++i) e1[r][i] = e2[r][i] = 0.0f;
        }
        if constexpr (SPLIT) quad_totals<1>(zo, 1 << D.log2HL, S0);
        else run_totals<RC>(zo, 1 << D.log2HL);
#pragma unroll
        for (int r = 0; r < SC; ++r) {
            if constexpr (!SPLIT) S0[r] = zo[r];
            const int h = SPLIT ? score_head() : hq.at(r);
            m[r] = D.stats[row * D.stats_stride + 2 * h];
            il[r] = D.stats[row * D.stats_stride + 2 * h + 1];
            delta[r] = 0.0f;
        }
    }
    __device__ __forceinline__ int score_head() const { return SPLIT ? hq.at(__lane_id() & 3) : hq.at(0); }
    template <bool ALL, class B>
    __device__ __forceinline__ void take(const B& x) {
        float s[RC * U], t[RC * U];
#pragma unroll
        for (int r = 0; r < RC; ++r)
#pragma unroll
            for (int u = 0; u < U; ++u) {
                s[r * U + u] = share<T, VEC, OV>(q[r], x.a[u], p);
                t[r * U + u] = share<T, VEC, OV>(dz[r], x.b[u], p);
            }
        if constexpr (SPLIT) {
            quad_totals<U>(s, 1 << D.log2HL, s);
            quad_totals<U>(t, 1 << D.log2HL, t);
        } else {
            run_totals<RC * U>(s, 1 << D.log2HL);
            run_totals<RC * U>(t, 1 << D.log2HL);
        }
#pragma unroll
        for (int r = 0; r < SC; ++r) {
            bool gone[U];
            float *sr = s + r * U, *tr = t + r * U;
            scores<T, SC, BIAS, ALL>(D, x, r, sr, gone);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                sr[u] = gone[u] ? GONE : exp_le0(sr[u] - m[r]) * il[r];  // the weight
                tr[u] = gone[u] ? 0.0f : sr[u] * (tr[u] - S0[r]);
                delta[r] += tr[u];
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float v[VEC];
#pragma unroll
            for (int i = 0; i < VEC; ++i) v[i] = W::at(x.a[u], i);
            Fwd::each([&](auto R) {
                float a, w;
                if constexpr (SPLIT) {
                    a = quad_lane<R()>(s[u]);
                    w = quad_lane<R()>(t[u]);
                } else {
                    a = s[R() * U + u];
                    w = t[R() * U + u];
                }
                if ((BIAS || !ALL) && is_gone(a)) return;
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    e1[R()][i] = fmaf(w, v[i], e1[R()][i]);
                    e2[R()][i] = fmaf(a, v[i], e2[R()][i]);
                }
            });
        }
    }
    __device__ __forceinline__ void join_groups(int L) {
        for (int x = L; x < WAVE; x <<= 1) {
#pragma unroll
            for (int r = 0; r < SC; ++r) delta[r] += __shfl_xor(delta[r], x, WAVE);
#pragma unroll
            for (int r = 0; r < RC; ++r)
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    e1[r][i] += __shfl_xor(e1[r][i], x, WAVE);
                    e2[r][i] += __shfl_xor(e2[r][i], x, WAVE);
                }
        }
    }
    // fn(head, index of its score) in one lane for each of the heads
    template <class F>
    __device__ __forceinline__ void each_score(F fn) const {
        if constexpr (SPLIT) {
            const int x = __lane_id() & ((1 << D.log2HL) - 1);
            if (x < 4 && hq.has(x)) fn(score_head(), 0);
        } else if (p.first) {
#pragma unroll
            for (int r = 0; r < RC; ++r)
                if (hq.has(r)) fn(hq.at(r), r);
        }
    }
};

// gradients of a bias that the heads share where they take several passes:
// the sum over this pass's heads, added to those of the passes before (their
// sums by edge id in D.edge_acc)
template <typename T, int VEC, bool OV, bool BIAS>
struct ToEdge {
    const DotArgs& D;
    const Place& p;
    int hq, L;
    using W = Words<T, VEC>;
    float q[W::N], dz[W::N];
    float4 rec;

    __device__ __forceinline__ ToEdge(const DotArgs& D_, const Place& p_, int hq_, int64_t row, int L_)
        : D(D_), p(p_), hq(hq_), L(L_) {
        const int64_t c = (int64_t)hq * D.F + p.c;
        own_row<T, VEC>(D, D.q, row * D.q_stride + c, q);
        row_words<T, VEC>(D.dz, row * D.dz_stride + c, dz);
        rec = D.rec[row * D.H + hq];
    }
    template <bool ALL, class B>
    __device__ __forceinline__ void take(const B& x) {
        float s[2 * U], ds[U];
        bool gone[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            s[u] = share<T, VEC, OV>(q, x.a[u], p);
            s[U + u] = share<T, VEC, OV>(dz, x.b[u], p);
        }
        run_totals<2 * U>(s, 1 << D.log2HL);
        scores<T, 1, BIAS, ALL>(D, x, 0, s, gone);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            ds[u] = exp_le0(s[u] - rec.x) * rec.y * (s[U + u] - rec.z);
            ds[u] = gone[u] ? 0.0f : ds[u];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) ds[u] = p.first ? ds[u] : 0.0f;
        run_totals<U>(ds, L);
        if (__lane_id() & (L - 1)) return;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (!ALL && !x.ok[u]) continue;
            float y = ds[u];
            if (!D.edge_first) y += D.edge_acc[(uint32_t)x.ed[u]];
            if (D.edge_last)
                IO<T, 1>::store1(reinterpret_cast<T*>(D.d_bias) +
                                     (uint64_t)(uint32_t)x.ed[u] * (uint32_t)D.d_bias_stride, y);
            else D.edge_acc[(uint32_t)x.ed[u]] = y;
        }
    }
};

template <typename T, int VEC, int RC, bool SPLIT, bool OV, bool BIAS, bool FAST>
__global__ __launch_bounds__(256, RC == 4 ? 2 : 3) void dot_backward_dst_kernel(EngineArgs A, DotArgs D) {
    const int w = wave_id();
    if (w >= A.sch.w_total) return;
    const Lanes ln = lanes_of(A.geo);
    const int G = A.geo.G, L = A.geo.L;
    const Place p = place_of<VEC>(D, ln.lig);
    const int kcol = p.j * D.F + p.c, step = RC << D.log2RL;
    using State = ToDst<T, VEC, RC, SPLIT, OV, BIAS>;
    if (w < A.sch.w_small_end) {
        const bool wave = w < A.sch.w_big_end;
        const Work k = wave ? wave_work(A, w) : lane_work(A, w, G, ln.g);
        const int64_t self = k.r >= 0 ? k.r : 0;
        for (int r = 0; r < D.R; r += step) {
            State st(D, p, r, self);
            walk<T, VEC, State::SC, FAST, BIAS, false>(A, D, (int32_t)k.b, (int32_t)k.e, wave ? U * ln.g : 0,
                                                       wave ? U * G : U, kcol, st.score_head(), st);
            if (wave) st.join_groups(L);
            float dh[RC];  // (lanes read each other's: before any of them is done)
            State::Fwd::each([&](auto x) { dh[x()] = State::Fwd::template of<x()>(st.delta); });
            if ((wave && ln.g != 0) || k.r < 0 || !(p.act || SPLIT)) continue;
            const int64_t W = (int64_t)D.H * D.F;
            if (k.slot >= 0) {
                float* P = D.part + (int64_t)k.slot * D.part_stride;
                if (p.own)
                    st.each_score([&](int hq, int x) {
                        P[2 * W + 2 * hq] = st.delta[x];
                        P[2 * W + 2 * hq + 1] = st.S0[x];
                    });
                if (!p.act) continue;
#pragma unroll
                for (int x = 0; x < RC; ++x) {
                    if (!st.hq.has(x)) break;
                    const int64_t c = (int64_t)st.hq.at(x) * D.F + p.c;
#pragma unroll
                    for (int i = 0; i < VEC; ++i) {
                        P[c + i] = st.e1[x][i];
                        P[W + c + i] = st.e2[x][i];
                    }
                }
            } else {
                if (p.own)
                    st.each_score([&](int hq, int x) {
                        D.rec[k.r * D.H + hq] = make_float4(st.m[x], st.il[x], st.S0[x] + st.delta[x], 0.0f);
                    });
                if (!p.act || !D.d_q) continue;
#pragma unroll
                for (int x = 0; x < RC; ++x) {
                    float v[VEC];
#pragma unroll
                    for (int i = 0; i < VEC; ++i) v[i] = D.scale * (st.e1[x][i] - dh[x] * st.e2[x][i]);
                    if (st.hq.has(x))
                        IO<T, VEC>::store(reinterpret_cast<T*>(D.d_q) + k.r * D.d_q_stride +
                                              (int64_t)st.hq.at(x) * D.F + p.c, v);
                }
            }
        }
    } else if (D.d_q) {
        empty_rows(A, w, G, ln.g, [&](int64_t row) {
            const float zero[VEC] = {};
            for (int r = p.rl; r < D.R && p.act; r += 1 << D.log2RL)
                IO<T, VEC>::store(reinterpret_cast<T*>(D.d_q) + row * D.d_q_stride +
                                      (int64_t)(p.j * D.R + r) * D.F + p.c, zero);
        });
    }
}

// the destination pass's hub rows, laid out as in dot_join_kernel
template <typename T>
__global__ void dot_join_dst_kernel(EngineArgs A, DotArgs D, int cols) {
    __shared__ double red[3][256];
    const int t = threadIdx.x, runs = blockDim.x / cols, run = t / cols, W = D.H * D.F;
    const int col = (int)blockIdx.y * cols + (t - run * cols);
    const int64_t row = A.csr.perm[blockIdx.x];
    const int s0 = A.csr.hub_off[blockIdx.x], s1 = A.csr.hub_off[blockIdx.x + 1];
    const bool ok = col < W;
    const int hq = ok ? col / D.F : 0;
    double v[3] = {};  // sums of w k and a k, delta
    if (ok) {
        for (int s = s0 + run; s < s1; s += U * runs) {
            float p1[U], p2[U], pd[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int x = s + u * runs;
                const float* P = D.part + (uint64_t)(uint32_t)(x < s1 ? x : s) * (uint32_t)D.part_stride;
                p1[u] = P[col];
                p2[u] = P[W + col];
                pd[u] = P[2 * W + 2 * hq];
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (s + u * runs < s1) {
                    v[0] += (double)p1[u];
                    v[1] += (double)p2[u];
                    v[2] += (double)pd[u];
                }
        }
    }
    join_runs<3>(red, v, cols, [](double* x, const double* o) {
#pragma unroll
        for (int i = 0; i < 3; ++i) x[i] += o[i];
    });
    if (t >= cols || !ok) return;
    if (D.d_q)
        IO<T, 1>::store1(reinterpret_cast<T*>(D.d_q) + row * D.d_q_stride + col,
                         (float)((double)D.scale * (v[0] - v[2] * v[1])));
    if (col % D.F == 0) {
        const float* st = D.stats + row * D.stats_stride + 2 * hq;
        const float S0 = D.part[(int64_t)s0 * D.part_stride + 2 * W + 2 * hq + 1];
        D.rec[row * D.H + hq] = make_float4(st[0], st[1], (float)((double)S0 + v[2]), 0.0f);
    }
}

// query head r0 of each key head of a slice
template <typename T, int VEC, bool OV, bool FAST>
__global__ __launch_bounds__(256) void dot_backward_edge_kernel(EngineArgs A, DotArgs D) {
    const int w = wave_id();
    if (w >= A.sch.w_small_end) return;
    const Lanes ln = lanes_of(A.geo);
    const int G = A.geo.G, L = A.geo.L;
    const Place p = place_of<VEC>(D, ln.lig);
    const bool wave = w < A.sch.w_big_end;
    const Work k = wave ? wave_work(A, w) : lane_work(A, w, G, ln.g);
    const int64_t self = k.r >= 0 ? k.r : A.csr.rowt[0].x;
    ToEdge<T, VEC, OV, true> st(D, p, p.j * D.R + D.r0, self, L);
    walk<T, VEC, 1, FAST, true, false>(A, D, (int32_t)k.b, (int32_t)k.e, wave ? U * ln.g : 0, wave ? U * G : U,
                                       p.j * D.F + p.c, st.hq, st);
}

// the source pass: dk and dv of a row over its out-edges, and the gradients of
// the bias where this pass sees what they take (a value per head, or all heads
// of a shared one side by side)
template <typename T, int VEC, bool OV, bool BIAS>
struct ToSrc {
    const DotArgs& D;
    const Place& p;
    int hq = 0, L;
    using W = Words<T, VEC>;
    float k[W::N], v[W::N];
    float dk[VEC], dv[VEC];

    __device__ __forceinline__ ToSrc(const DotArgs& D_, const Place& p_, int64_t row, int L_)
        : D(D_), p(p_), L(L_) {
        const int64_t c = (int64_t)p.j * D.F + p.c;
        own_row<T, VEC>(D, D.k, row * D.k_stride + c, k);
        row_words<T, VEC>(D.v, row * D.v_stride + c, v);
#pragma unroll
        for (int i = 0; i < VEC; ++i) dk[i] = dv[i] = 0.0f;
    }
    template <bool ALL, class B>
    __device__ __forceinline__ void take(const B& x) {
        float s[2 * U];
        bool gone[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            s[u] = share<T, VEC, OV>(k, x.a[u], p);
            s[U + u] = share<T, VEC, OV>(v, x.b[u], p);
        }
        run_totals<2 * U>(s, 1 << D.log2HL);
        scores<T, 1, BIAS, ALL>(D, x, 0, s, gone);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const float a = exp_le0(s[u] - x.rec[u].x) * x.rec[u].y;
            const float w = a * (s[U + u] - x.rec[u].z);
            if (!gone[u]) {
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    dk[i] = fmaf(w, W::at(x.a[u], i), dk[i]);
                    dv[i] = fmaf(a, W::at(x.b[u], i), dv[i]);
                }
            }
            s[u] = gone[u] ? 0.0f : w;
        }
        if (!BIAS || !D.src_bias) return;
        if (D.bias_per_head) {
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (p.first && (ALL || x.ok[u])) store_dbias(x.ed[u], hq, s[u]);
        } else {
#pragma unroll
            for (int u = 0; u < U; ++u) s[u] = p.first ? s[u] : 0.0f;
            run_totals<U>(s, L);
#pragma unroll
            for (int u = 0; u < U; ++u)
                if ((__lane_id() & (L - 1)) == 0 && (ALL || x.ok[u])) store_dbias(x.ed[u], 0, s[u]);
        }
    }
    __device__ __forceinline__ void store_dbias(int32_t ed, int h, float x) {
        IO<T, 1>::store1(reinterpret_cast<T*>(D.d_bias) + (uint64_t)(uint32_t)ed * (uint32_t)D.d_bias_stride + h, x);
    }
    // sums over the lanes that differ in the bits from .. to / 2 of their number
    __device__ __forceinline__ void join(int from, int to) {
        for (int x = from; x < to; x <<= 1)
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                dk[i] += __shfl_xor(dk[i], x, WAVE);
                dv[i] += __shfl_xor(dv[i], x, WAVE);
            }
    }
    // over the query heads of a key head, side by side
    __device__ __forceinline__ void join_heads() { join(1 << D.log2HL, 1 << (D.log2HL + D.log2RL)); }
    __device__ __forceinline__ void write(int64_t row) {
        const int64_t c = (int64_t)p.j * D.F + p.c;
#pragma unroll
        for (int i = 0; i < VEC; ++i) dk[i] *= D.scale;
        if (D.d_k) IO<T, VEC>::store(reinterpret_cast<T*>(D.d_k) + row * D.d_k_stride + c, dk);
        if (D.d_v) IO<T, VEC>::store(reinterpret_cast<T*>(D.d_v) + row * D.d_v_stride + c, dv);
    }
};

template <typename T, int VEC, bool OV, bool BIAS, bool FAST>
__global__ __launch_bounds__(256, 3) void dot_backward_src_kernel(EngineArgs A, DotArgs D) {
    const int w = wave_id();
    if (w >= A.sch.w_total) return;
    const Lanes ln = lanes_of(A.geo);
    const int G = A.geo.G, L = A.geo.L;
    const Place p = place_of<VEC>(D, ln.lig);
    if (w < A.sch.w_small_end) {
        const bool wave = w < A.sch.w_big_end;
        const Work k = wave ? wave_work(A, w) : lane_work(A, w, G, ln.g);
        const int64_t self = k.r >= 0 ? k.r : 0;
        ToSrc<T, VEC, OV, BIAS> st(D, p, self, L);
        for (int r = p.rl; r < D.R; r += 1 << D.log2RL) {
            st.hq = p.j * D.R + r;
            walk<T, VEC, 1, FAST, BIAS, true>(A, D, (int32_t)k.b, (int32_t)k.e, wave ? U * ln.g : 0,
                                              wave ? U * G : U, st.hq * D.F + p.c, st.hq, st);
        }
        if (wave) st.join(L, WAVE);
        st.join_heads();
        if ((wave && ln.g != 0) || k.r < 0 || !p.act || p.rl != 0) return;
        if (k.slot >= 0) {
            float* P = D.part + (int64_t)k.slot * D.part_stride;
            const int64_t W = (int64_t)D.K * D.F, c = (int64_t)p.j * D.F + p.c;
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                P[c + i] = st.dk[i];
                P[W + c + i] = st.dv[i];
            }
        } else {
            st.write(k.r);
        }
    } else {
        empty_rows(A, w, G, ln.g, [&](int64_t row) {
            const float zero[VEC] = {};
            const int64_t c = (int64_t)p.j * D.F + p.c;
            if (!p.act || p.rl != 0) return;
            if (D.d_k) IO<T, VEC>::store(reinterpret_cast<T*>(D.d_k) + row * D.d_k_stride + c, zero);
            if (D.d_v) IO<T, VEC>::store(reinterpret_cast<T*>(D.d_v) + row * D.d_v_stride + c, zero);
        });
    }
}

// the source pass's hub rows, laid out as in dot_join_kernel
template <typename T>
__global__ void dot_join_src_kernel(EngineArgs A, DotArgs D, int cols) {
    __shared__ double red[1][256];
    const int t = threadIdx.x, runs = blockDim.x / cols, run = t / cols, W = D.K * D.F;
    const int col = (int)blockIdx.y * cols + (t - run * cols);
    const int64_t row = A.csr.perm[blockIdx.x];
    const int s0 = A.csr.hub_off[blockIdx.x], s1 = A.csr.hub_off[blockIdx.x + 1];
    const bool ok = col < 2 * W;
    double x = 0.0;
    if (ok) {
        for (int s = s0 + run; s < s1; s += U * runs) {
            float y[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                y[u] = D.part[(uint64_t)(uint32_t)(s + u * runs < s1 ? s + u * runs : s) * (uint32_t)D.part_stride + col];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (s + u * runs < s1) x += (double)y[u];
        }
    }
    join_runs<1>(red, &x, cols, [](double* a, const double* b) { *a += *b; });
    if (t >= cols || !ok) return;
    if (col < W) {
        if (D.d_k)
            IO<T, 1>::store1(reinterpret_cast<T*>(D.d_k) + row * D.d_k_stride + col, (float)((double)D.scale * x));
    } else if (D.d_v) {
        IO<T, 1>::store1(reinterpret_cast<T*>(D.d_v) + row * D.d_v_stride + (col - W), (float)x);
    }
}

// ---------------------------------------------------------------------------

// columns and threads of a workgroup that joins segments
struct Join {
    int cols, threads;
    dim3 grid(const EngineArgs& a, int64_t width) const {
        return dim3((unsigned)a.sch.n_hub, (unsigned)((width + cols - 1) / cols));
    }
};
Join join_of(const EngineArgs& a) {
    const bool many = a.sch.n_seg > 64ll * a.sch.n_hub;
    return many ? Join{8, 1024} : Join{64, 256};
}

template <typename T, int V, int RC, bool OV, bool BIAS, bool FAST>
void dot_launch(const EngineArgs& a, const DotArgs& d, int pass, hipStream_t s) {
    const dim3 grid(blocks_for_waves(a.sch.w_total), (unsigned)d.slices), block(WAVE * WPB);
    const Join j = join_of(a);
    const int64_t HF = (int64_t)d.H * d.F, KF = (int64_t)d.K * d.F;
    const dim3 threads(j.threads);
    const bool split = RC == 4 && d.log2HL >= 2;
    if (pass == 0) {
        if constexpr (RC == 4)
            if (split) hipLaunchKernelGGL((dot_forward_kernel<T, V, RC, true, OV, BIAS, FAST>), grid, block, 0, s, a, d);
        if (!split) hipLaunchKernelGGL((dot_forward_kernel<T, V, RC, false, OV, BIAS, FAST>), grid, block, 0, s, a, d);
        if (a.sch.n_hub > 0) hipLaunchKernelGGL((dot_join_kernel<T>), j.grid(a, HF), threads, 0, s, a, d, j.cols);
    } else if (pass == 1) {
        if constexpr (RC == 4)
            if (split)
                hipLaunchKernelGGL((dot_backward_dst_kernel<T, V, RC, true, OV, BIAS, FAST>), grid, block, 0, s, a, d);
        if (!split)
            hipLaunchKernelGGL((dot_backward_dst_kernel<T, V, RC, false, OV, BIAS, FAST>), grid, block, 0, s, a, d);
        if (a.sch.n_hub > 0) hipLaunchKernelGGL((dot_join_dst_kernel<T>), j.grid(a, HF), threads, 0, s, a, d, j.cols);
    } else if (pass == 2) {
        hipLaunchKernelGGL((dot_backward_src_kernel<T, V, OV, BIAS, FAST>), grid, block, 0, s, a, d);
        if (a.sch.n_hub > 0)
            hipLaunchKernelGGL((dot_join_src_kernel<T>), j.grid(a, 2 * KF), threads, 0, s, a, d, j.cols);
    } else {
        const dim3 egrid(blocks_for_waves(a.sch.w_small_end), (unsigned)d.slices);
        hipLaunchKernelGGL((dot_backward_edge_kernel<T, V, OV, FAST>), egrid, block, 0, s, a, d);
    }
}

template <typename T, int V, int RC, bool OV, bool FAST>
void dot_bias(const EngineArgs& a, const DotArgs& d, int pass, hipStream_t s) {
    if (d.bias) dot_launch<T, V, RC, OV, true, FAST>(a, d, pass, s);
    else dot_launch<T, V, RC, OV, false, FAST>(a, d, pass, s);
}

// the widest vectors have kernels without shared columns and for several query
// heads in registers; narrower heads and tables past 32-bit offsets one each
template <typename T, int V>
void dot_t(const EngineArgs& a, const DotArgs& d, int pass, bool fast, hipStream_t s) {
    constexpr bool WIDE = V == (sizeof(T) == 4 ? 4 : 8);
    if (!fast) {
        dot_bias<T, V, 1, true, false>(a, d, pass, s);
    } else if constexpr (!WIDE) {
        dot_bias<T, V, 1, true, true>(a, d, pass, s);
    } else if (d.F % V != 0) {
        if (d.RC == 4) dot_bias<T, V, 4, true, true>(a, d, pass, s);
        else if (d.RC == 2) dot_bias<T, V, 2, true, true>(a, d, pass, s);
        else dot_bias<T, V, 1, true, true>(a, d, pass, s);
    } else {
        if (d.RC == 4) dot_bias<T, V, 4, false, true>(a, d, pass, s);
        else if (d.RC == 2) dot_bias<T, V, 2, false, true>(a, d, pass, s);
        else dot_bias<T, V, 1, false, true>(a, d, pass, s);
    }
}

}  // namespace

hipError_t launch_dot(const EngineArgs& a, const DotArgs& d, int pass, int dtype, int vec, bool fast, hipStream_t s) {
    if (a.sch.w_total <= 0 || (pass == 3 && a.sch.w_small_end <= 0)) return hipSuccess;
    if (dtype == 0) {
        GNNK_VEC_DISPATCH_F32(vec, dot_t<float, V>(a, d, pass, fast, s))
    } else {
        GNNK_VEC_DISPATCH_BF16(vec, dot_t<bf16_t, V>(a, d, pass, fast, s))
    }
    return hipGetLastError();
}

}  // namespace gnnk
