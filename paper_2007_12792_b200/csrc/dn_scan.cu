// The gated linear recurrence over the rows of a field, h_t = a_t h_{t-1} + w_t x_t, and its gradients.
//
// A span of rows acts on the state ahead of it as h -> P h + H (P the product of its a_t, H its result from a zero state), and spans
// compose: (P2, H2) after (P1, H1) is (P2 P1, P2 H1 + H2).  So the rows of a column are cut into pieces that are worked on at the
// same time: a thread runs over R consecutive rows of V adjacent columns and keeps their a and b = w x in registers, the pairs
// (P, H) of a block's row groups meet in shared memory, those of a cluster's blocks in each other's shared memory, and every
// thread runs over its registers once more from the state it then knows.  g and x are read once, h is written once, for any number
// of rows and columns: many columns are marched by a block each, few columns by a cluster of up to 16 blocks along the rows.
//
// Backward, the gradient mu_t = a_t (dh_t + mu_{t+1}) runs the other way with the same factors, so one exchange carries P, H (the
// states are formed again from one in 32 bits ahead of every 64 rows) and M (mu from zero).
#include "dn_eight.cuh"

#include <type_traits>

namespace dn {
namespace {

constexpr int SCAN_MOST_BLOCKS = 16;       // blocks per cluster

struct RowsOf { char* p; int64_t batch, row; };           // strides in bytes

struct ScanArgs {
    RowsOf g, x, h, dh, dg, dx;
    const float* start;          // h0, or dL/dh_last
    float* end;                  // h_last, or dL/dh0
    const int32_t* lengths;
    uint8_t *gq, *xq, *gs, *xs;
    float* states;
    int64_t rows_padded;
    int rows, cols, strips, blocks, nblk, nchunk;
    int mix, int8;               // int8: the input's format (the gate's always is)
};

template <class T, int V> using Raw = std::conditional_t<sizeof(T) * V == 4, uint32_t, uint16_t>;

template <class T, int V> __device__ __forceinline__ void expand(Raw<T, V> r, float (&f)[V]) {
    if constexpr (V == 1) {
        T t;
        memcpy(&t, &r, sizeof t);
        f[0] = as_float(t);
    } else {
        T t[2];
        memcpy(t, &r, sizeof t);
        f[0] = as_float(t[0]);
        f[1] = as_float(t[1]);
    }
}
template <class T, int V> __device__ __forceinline__ Raw<T, V> join(const float (&f)[V]) {
    T t[V];
#pragma unroll
    for (int v = 0; v < V; ++v) t[v] = rounded<T>(f[v]);
    Raw<T, V> r;
    memcpy(&r, t, sizeof r);
    return r;
}
template <class W> __device__ __forceinline__ W load_at(const char* p) { return *reinterpret_cast<const W*>(p); }
template <class W> __device__ __forceinline__ void store_at(char* p, W v) { *reinterpret_cast<W*>(p) = v; }

__device__ __forceinline__ unsigned cluster_address(const void* local, int rank) {
    unsigned r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"((unsigned)__cvta_generic_to_shared(local)), "r"(rank));
    return r;
}
__device__ __forceinline__ void cluster_store(unsigned at, float v) { asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at), "f"(v) : "memory"); }
__device__ __forceinline__ void cluster_barrier() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// Where a thread works: lanes LX across the columns (V each) and 32 / LX down the rows, warps WR down and WC across.
template <int V, int LX, int WR, int WC, int R> struct Place {
    static constexpr int NG = WR * (32 / LX), COLS = WC * LX * V, TILE = NG * R, THREADS = 32 * WR * WC;
    int b, rank, q, col, c, len;
    bool cv;
    __device__ Place(const ScanArgs& A) {
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        q = (warp % WR) * (32 / LX) + lane / LX;
        col = (warp / WR) * LX * V + (lane % LX) * V;
        const unsigned unit = blockIdx.x / A.blocks;
        rank = blockIdx.x % A.blocks;
        b = unit / A.strips;
        c = (int)(unit % A.strips) * COLS + col;
        cv = c < A.cols;
        len = A.rows;
    }
    __device__ void read_length(const ScanArgs& A) {
        if (A.lengths) len = min(max(A.lengths[b], 0), A.rows);
    }
};

// ---- forward -----------------------------------------------------------------------------------------------------------------
template <class T, int V, int LX, int WR, int WC, int R, bool SAVE8>
__global__ void __launch_bounds__(32 * WR * WC) scan_forward_kernel(const __grid_constant__ ScanArgs A) {
    static_assert(!SAVE8 || (LX == 32 && R == 16), "a row's 32 columns of a scale lie in one warp; 16 scale bytes are one store");
    using Pl = Place<V, LX, WR, WC, R>;
    using W = Raw<T, V>;
    constexpr int NG = Pl::NG, COLS = Pl::COLS, TILE = Pl::TILE;
    __shared__ float aggP[2][NG > 1 ? NG : 1][NG > 1 ? COLS : 1], aggH[2][NG > 1 ? NG : 1][NG > 1 ? COLS : 1];
    __shared__ float totP[2][SCAN_MOST_BLOCKS][NG > 1 ? COLS : 1], totH[2][SCAN_MOST_BLOCKS][NG > 1 ? COLS : 1];
    Pl at(A);
    const int q = at.q, col = at.col, c = at.c, rank = at.rank;
    const bool cv = at.cv;
    const int K = NG > 1 ? A.blocks : 1;
    dep_wait();
    at.read_length(A);
    const int len = at.len;
    const int span = K * TILE;
    const int steps = (int)(((int64_t)len + span - 1) / span);

    float carry[V];
#pragma unroll
    for (int v = 0; v < V; ++v) carry[v] = (A.start && cv) ? A.start[(int64_t)at.b * A.cols + c + v] : 0.0f;

    int t0 = rank * TILE + q * R;
    const char* pg = A.g.p + at.b * A.g.batch + t0 * A.g.row + c * (int64_t)sizeof(T);
    const char* px = A.x.p + at.b * A.x.batch + t0 * A.x.row + c * (int64_t)sizeof(T);
    char* ph = A.h.p + at.b * A.h.batch + t0 * A.h.row + c * (int64_t)sizeof(T);

    W rg[R], rx[R];
    auto fetch = [&](int first) {
        const int n = cv ? len - first : 0;
#pragma unroll
        for (int i = 0; i < R; ++i) {
            rg[i] = i < n ? load_at<W>(pg + i * A.g.row) : W(0);
            rx[i] = i < n ? load_at<W>(px + i * A.x.row) : W(0);
        }
    };
    if (steps > 0) fetch(t0);
    if (K > 1) cluster_barrier();                          // every block of the cluster runs before one writes to another

    for (int s = 0; s < steps; ++s) {
        const int n = cv ? len - t0 : 0;                   // rows i < n hold data; the others pass the state on
        float a[R][V], bb[R][V], P[V], H[V];
#pragma unroll
        for (int v = 0; v < V; ++v) { P[v] = 1.0f; H[v] = 0.0f; }
        uint32_t sg[SAVE8 ? 4 : 1] = {}, sx[SAVE8 ? 4 : 1] = {};
#pragma unroll
        for (int i = 0; i < R; ++i) {
            float g[V], x[V];
            expand<T, V>(rg[i], g);
            expand<T, V>(rx[i], x);
            if constexpr (SAVE8) {
                unsigned mg = magnitude_bits(g[0]), mx = magnitude_bits(x[0]);
                if constexpr (V == 2) {                    // two blocks of 32 columns in a warp's row
                    mg = max(mg, magnitude_bits(g[1]));
                    mx = max(mx, magnitude_bits(x[1]));
                    const bool low = (threadIdx.x & 16) == 0;
                    const unsigned g0 = __reduce_max_sync(~0u, low ? mg : 0u), g1 = __reduce_max_sync(~0u, low ? 0u : mg);
                    const unsigned x0 = __reduce_max_sync(~0u, low ? mx : 0u), x1 = __reduce_max_sync(~0u, low ? 0u : mx);
                    mg = low ? g0 : g1;
                    mx = low ? x0 : x1;
                } else {
                    mg = __reduce_max_sync(~0u, mg);
                    mx = __reduce_max_sync(~0u, mx);
                }
                const int bg = scale_byte(mg, true), bx = scale_byte(mx, A.int8);
                sg[i / 4] |= (uint32_t)bg << (8 * (i % 4));
                sx[i / 4] |= (uint32_t)bx << (8 * (i % 4));
                if (i < n) {
                    const float ig = inverse_scale_of(bg), ix = inverse_scale_of(bx);
                    const int64_t o = ((int64_t)at.b * A.rows + t0 + i) * A.cols + c;
                    if constexpr (V == 2) {
                        *reinterpret_cast<uint16_t*>(A.gq + o) = (uint16_t)(code_int8(g[0], ig) | code_int8(g[1], ig) << 8);
                        *reinterpret_cast<uint16_t*>(A.xq + o) = (uint16_t)(code8(x[0], ix, A.int8) | code8(x[1], ix, A.int8) << 8);
                    } else {
                        A.gq[o] = (uint8_t)code_int8(g[0], ig);
                        A.xq[o] = (uint8_t)code8(x[0], ix, A.int8);
                    }
                }
            }
#pragma unroll
            for (int v = 0; v < V; ++v) {
                float w;
                gates<sizeof(T) == 4>(g[v], a[i][v], w);
                bb[i][v] = A.mix ? w * x[v] : x[v];
                if (i >= n) { a[i][v] = 1.0f; bb[i][v] = 0.0f; }
                P[v] *= a[i][v];
                H[v] = fmaf(a[i][v], H[v], bb[i][v]);
            }
        }
        if constexpr (SAVE8) {
            if ((threadIdx.x & (V == 2 ? 15 : 31)) == 0 && cv && t0 < A.rows_padded) {
                const int64_t o = ((int64_t)at.b * A.nblk + c / kBlock8) * A.rows_padded + t0;
                *reinterpret_cast<uint4*>(A.gs + o) = make_uint4(sg[0], sg[1], sg[2], sg[3]);
                *reinterpret_cast<uint4*>(A.xs + o) = make_uint4(sx[0], sx[1], sx[2], sx[3]);
            }
        }
        pg += span * A.g.row;
        px += span * A.x.row;
        if (s + 1 < steps) fetch(t0 + span);               // in flight while the states of this step are found

        float hin[V];
        if constexpr (NG == 1) {
#pragma unroll
            for (int v = 0; v < V; ++v) { hin[v] = carry[v]; carry[v] = fmaf(P[v], carry[v], H[v]); }
        } else {
            const int buf = s & 1;
#pragma unroll
            for (int v = 0; v < V; ++v) { aggP[buf][q][col + v] = P[v]; aggH[buf][q][col + v] = H[v]; }
            __syncthreads();
            if (K == 1) {
#pragma unroll
                for (int j = 0; j < NG; ++j)
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        if (j == q) hin[v] = carry[v];
                        carry[v] = fmaf(aggP[buf][j][col + v], carry[v], aggH[buf][j][col + v]);
                    }
            } else {
                float Pb[V], Hb[V], Pt[V], Ht[V];          // of the groups ahead of this one; of all
#pragma unroll
                for (int v = 0; v < V; ++v) { Pb[v] = Pt[v] = 1.0f; Hb[v] = Ht[v] = 0.0f; }
#pragma unroll
                for (int j = 0; j < NG; ++j)
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        if (j == q) { Pb[v] = Pt[v]; Hb[v] = Ht[v]; }
                        const float p = aggP[buf][j][col + v];
                        Ht[v] = fmaf(p, Ht[v], aggH[buf][j][col + v]);
                        Pt[v] *= p;
                    }
                for (int peer = q; peer < K; peer += NG)
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        cluster_store(cluster_address(&totP[buf][rank][col + v], peer), Pt[v]);
                        cluster_store(cluster_address(&totH[buf][rank][col + v], peer), Ht[v]);
                    }
                cluster_barrier();
                float hc[V] = {};
                for (int peer = 0; peer < K; ++peer)
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        if (peer == rank) hc[v] = carry[v];
                        carry[v] = fmaf(totP[buf][peer][col + v], carry[v], totH[buf][peer][col + v]);
                    }
#pragma unroll
                for (int v = 0; v < V; ++v) hin[v] = fmaf(Pb[v], hc[v], Hb[v]);
            }
        }
        if (A.states && cv && t0 % kChunkRows == 0 && t0 < A.rows) {
            float* st = A.states + ((int64_t)at.b * A.nchunk + t0 / kChunkRows) * A.cols + c;
#pragma unroll
            for (int v = 0; v < V; ++v) st[v] = hin[v];
        }
        const int m = cv ? A.rows - t0 : 0;
#pragma unroll
        for (int i = 0; i < R; ++i) {
            float out[V];
#pragma unroll
            for (int v = 0; v < V; ++v) {
                hin[v] = fmaf(a[i][v], hin[v], bb[i][v]);
                out[v] = i < n ? hin[v] : 0.0f;
            }
            if (i < m) store_at<W>(ph + i * A.h.row, join<T, V>(out));
        }
        ph += span * A.h.row;
        t0 += span;
    }
    for (; t0 < A.rows; t0 += span, ph += span * A.h.row)  // rows behind a sequence
        for (int i = 0; i < R && i < A.rows - t0; ++i)
            if (cv) store_at<W>(ph + i * A.h.row, W(0));
    if (A.end && rank == 0 && q == 0 && cv) {
#pragma unroll
        for (int v = 0; v < V; ++v) A.end[(int64_t)at.b * A.cols + c + v] = carry[v];
    }
}

// ---- backward ----------------------------------------------------------------------------------------------------------------
template <class T, int V, int LX, int WR, int WC, bool SAVED8>
__global__ void __launch_bounds__(32 * WR * WC) scan_backward_kernel(const __grid_constant__ ScanArgs A) {
    constexpr int R = 8, GC = kChunkRows / R;              // 8 scale bytes are one load; groups of a chunk
    using Pl = Place<V, LX, WR, WC, R>;
    using W = Raw<T, V>;
    using Q = std::conditional_t<V == 2, uint16_t, uint8_t>;
    constexpr int NG = Pl::NG, COLS = Pl::COLS, TILE = Pl::TILE;
    static_assert(NG == 1 || TILE % kChunkRows == 0, "a tile holds whole chunks, or is the only one");
    constexpr int SG = NG > 1 ? NG : 1, SC = NG > 1 ? COLS : 1;
    __shared__ float aggP[2][SG][SC], aggH[2][SG][SC], aggM[2][SG][SC];
    __shared__ float totP[2][SCAN_MOST_BLOCKS][SC], totM[2][SCAN_MOST_BLOCKS][SC];
    Pl at(A);
    const int q = at.q, col = at.col, c = at.c, rank = at.rank;
    const bool cv = at.cv;
    const int K = NG > 1 ? A.blocks : 1;
    dep_wait();
    at.read_length(A);
    const int len = at.len;
    const int span = K * TILE;
    const int steps = (int)(((int64_t)len + span - 1) / span);

    float carry[V];                                        // mu of the row behind
#pragma unroll
    for (int v = 0; v < V; ++v) carry[v] = (A.start && cv) ? A.start[(int64_t)at.b * A.cols + c + v] : 0.0f;

    for (int t = steps * span + rank * TILE + q * R; t < A.rows; t += span)          // rows behind a sequence
        for (int i = 0; i < R && i < A.rows - t; ++i)
            if (cv) {
                store_at<W>(A.dg.p + at.b * A.dg.batch + (t + i) * A.dg.row + c * (int64_t)sizeof(T), W(0));
                store_at<W>(A.dx.p + at.b * A.dx.batch + (t + i) * A.dx.row + c * (int64_t)sizeof(T), W(0));
            }

    int t0 = (steps - 1) * span + rank * TILE + q * R;
    W rg[SAVED8 ? 1 : R], rx[SAVED8 ? 1 : R], rd[R];
    Q qg[SAVED8 ? R : 1], qx[SAVED8 ? R : 1];
    uint2 sg{}, sx{};
    float st[V];
    const int qc = NG > 1 ? q % GC : 0;                    // groups of the same chunk ahead of this one
    auto fetch = [&](int first) {
        const int n = cv ? len - first : 0;
        if constexpr (SAVED8) {
            const int64_t o = ((int64_t)at.b * A.rows + first) * A.cols + c;
            const int64_t os = ((int64_t)at.b * A.nblk + c / kBlock8) * A.rows_padded + first;
            if (n > 0) { sg = *reinterpret_cast<const uint2*>(A.gs + os); sx = *reinterpret_cast<const uint2*>(A.xs + os); }
#pragma unroll
            for (int i = 0; i < R; ++i) {
                qg[i] = i < n ? *reinterpret_cast<const Q*>(A.gq + o + (int64_t)i * A.cols) : Q(0);
                qx[i] = i < n ? *reinterpret_cast<const Q*>(A.xq + o + (int64_t)i * A.cols) : Q(0);
            }
        } else {
            const char* pg = A.g.p + at.b * A.g.batch + first * A.g.row + c * (int64_t)sizeof(T);
            const char* px = A.x.p + at.b * A.x.batch + first * A.x.row + c * (int64_t)sizeof(T);
#pragma unroll
            for (int i = 0; i < R; ++i) {
                rg[i] = i < n ? load_at<W>(pg + i * A.g.row) : W(0);
                rx[i] = i < n ? load_at<W>(px + i * A.x.row) : W(0);
            }
        }
        const char* pd = A.dh.p + at.b * A.dh.batch + first * A.dh.row + c * (int64_t)sizeof(T);
        const int nd = A.dh.p ? n : 0;
#pragma unroll
        for (int i = 0; i < R; ++i) rd[i] = i < nd ? load_at<W>(pd + i * A.dh.row) : W(0);
        const float* ps = A.states + ((int64_t)at.b * A.nchunk + first / kChunkRows) * A.cols + c;
#pragma unroll
        for (int v = 0; v < V; ++v) st[v] = n > 0 ? ps[v] : 0.0f;
    };
    if (steps > 0) fetch(t0);
    if (K > 1) cluster_barrier();

    for (int s = steps - 1; s >= 0; --s) {
        const int n = cv ? len - t0 : 0;
        float a[R][V], w[R][V], x[R][V], d[R][V], P[V], H[V], M[V], hin[V];
#pragma unroll
        for (int v = 0; v < V; ++v) { P[v] = 1.0f; H[v] = 0.0f; M[v] = 0.0f; hin[v] = st[v]; }
#pragma unroll
        for (int i = 0; i < R; ++i) {
            float g[V];
            if constexpr (SAVED8) {
                const float fg = scale_of(((i < 4 ? sg.x : sg.y) >> (8 * (i % 4))) & 255), fx = scale_of(((i < 4 ? sx.x : sx.y) >> (8 * (i % 4))) & 255);
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    g[v] = value_int8((qg[i] >> (8 * v)) & 255, fg);
                    x[i][v] = value8((qx[i] >> (8 * v)) & 255, fx, A.int8);
                }
            } else {
                expand<T, V>(rg[i], g);
                expand<T, V>(rx[i], x[i]);
            }
            expand<T, V>(rd[i], d[i]);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                gates<sizeof(T) == 4>(g[v], a[i][v], w[i][v]);
                if (i >= n) { a[i][v] = 1.0f; w[i][v] = 0.0f; x[i][v] = 0.0f; }
                P[v] *= a[i][v];
                H[v] = fmaf(a[i][v], H[v], A.mix ? w[i][v] * x[i][v] : x[i][v]);
            }
        }
#pragma unroll
        for (int i = R - 1; i >= 0; --i)
#pragma unroll
            for (int v = 0; v < V; ++v) M[v] = a[i][v] * (d[i][v] + M[v]);
        if (s > 0) fetch(t0 - span);

        float mu[V];
        if constexpr (NG == 1) {
#pragma unroll
            for (int v = 0; v < V; ++v) { mu[v] = carry[v]; carry[v] = fmaf(P[v], carry[v], M[v]); }
        } else {
            const int buf = s & 1;
#pragma unroll
            for (int v = 0; v < V; ++v) { aggP[buf][q][col + v] = P[v]; aggH[buf][q][col + v] = H[v]; aggM[buf][q][col + v] = M[v]; }
            __syncthreads();
            for (int j = q - qc; j < q; ++j)
#pragma unroll
                for (int v = 0; v < V; ++v) hin[v] = fmaf(aggP[buf][j][col + v], hin[v], aggH[buf][j][col + v]);
            if (K == 1) {
#pragma unroll
                for (int j = NG - 1; j >= 0; --j)
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        if (j == q) mu[v] = carry[v];
                        carry[v] = fmaf(aggP[buf][j][col + v], carry[v], aggM[buf][j][col + v]);
                    }
            } else {
                float Pb[V], Mb[V], Pt[V], Mt[V];
#pragma unroll
                for (int v = 0; v < V; ++v) { Pb[v] = Pt[v] = 1.0f; Mb[v] = Mt[v] = 0.0f; }
#pragma unroll
                for (int j = NG - 1; j >= 0; --j)
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        if (j == q) { Pb[v] = Pt[v]; Mb[v] = Mt[v]; }
                        const float p = aggP[buf][j][col + v];
                        Mt[v] = fmaf(p, Mt[v], aggM[buf][j][col + v]);
                        Pt[v] *= p;
                    }
                for (int peer = q; peer < K; peer += NG)
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        cluster_store(cluster_address(&totP[buf][rank][col + v], peer), Pt[v]);
                        cluster_store(cluster_address(&totM[buf][rank][col + v], peer), Mt[v]);
                    }
                cluster_barrier();
                float mc[V] = {};
                for (int peer = K - 1; peer >= 0; --peer)
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        if (peer == rank) mc[v] = carry[v];
                        carry[v] = fmaf(totP[buf][peer][col + v], carry[v], totM[buf][peer][col + v]);
                    }
#pragma unroll
                for (int v = 0; v < V; ++v) mu[v] = fmaf(Pb[v], mc[v], Mb[v]);
            }
        }
        // x <- a (1 - a) (h_{t-1} [- x]), the factor of dg
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float in = A.mix ? w[i][v] * x[i][v] : x[i][v];
                const float diff = A.mix ? hin[v] - x[i][v] : hin[v];
                hin[v] = fmaf(a[i][v], hin[v], in);
                x[i][v] = a[i][v] * w[i][v] * diff;
            }
        const int m = cv ? A.rows - t0 : 0;
        char* pdg = A.dg.p + at.b * A.dg.batch + t0 * A.dg.row + c * (int64_t)sizeof(T);
        char* pdx = A.dx.p + at.b * A.dx.batch + t0 * A.dx.row + c * (int64_t)sizeof(T);
#pragma unroll
        for (int i = R - 1; i >= 0; --i) {
            float og[V], ox[V];
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float lam = d[i][v] + mu[v];
                og[v] = i < n ? lam * x[i][v] : 0.0f;
                ox[v] = i < n ? (A.mix ? lam * w[i][v] : lam) : 0.0f;
                mu[v] = a[i][v] * lam;
            }
            if (i < m) {
                store_at<W>(pdg + i * A.dg.row, join<T, V>(og));
                store_at<W>(pdx + i * A.dx.row, join<T, V>(ox));
            }
        }
        t0 -= span;
    }
    if (A.end && rank == 0 && q == 0 && cv) {
#pragma unroll
        for (int v = 0; v < V; ++v) A.end[(int64_t)at.b * A.cols + c + v] = carry[v];
    }
}

// ---- launches ----------------------------------------------------------------------------------------------------------------
using Kernel = void (*)(ScanArgs);

struct Shape {                   // of a launch
    Kernel kernel;
    int cols, tile, threads;     // columns and rows of a block
    bool split;                  // a column's rows may be shared by the blocks of a cluster
};
template <int V, int LX, int WR, int WC, int R> Shape shape_of(Kernel k, bool split) {
    using Pl = Place<V, LX, WR, WC, R>;
    return Shape{k, Pl::COLS, Pl::TILE, Pl::THREADS, split};
}

enum Layout { ONE_ROW, SHORT, TALL, NARROW };

template <class T, int V> Shape forward_shape(Layout l, bool save8) {
    if (save8) return l == SHORT ? shape_of<V, 32, 1, 4, 16>(scan_forward_kernel<T, V, 32, 1, 4, 16, true>, false)
                                 : shape_of<V, 32, 4, 1, 16>(scan_forward_kernel<T, V, 32, 4, 1, 16, true>, true);
    switch (l) {
        case ONE_ROW: return shape_of<V, 32, 1, 4, 1>(scan_forward_kernel<T, V, 32, 1, 4, 1, false>, false);
        case SHORT: return shape_of<V, 32, 1, 4, 16>(scan_forward_kernel<T, V, 32, 1, 4, 16, false>, false);
        case TALL: return shape_of<V, 32, 4, 1, 16>(scan_forward_kernel<T, V, 32, 4, 1, 16, false>, true);
        default: return shape_of<V, 8, 4, 1, 16>(scan_forward_kernel<T, V, 8, 4, 1, 16, false>, true);
    }
}
template <class T, int V, bool SAVED8> Shape backward_shape(Layout l) {
    switch (l) {
        case ONE_ROW:
        case SHORT: return shape_of<V, 32, 1, 4, 8>(scan_backward_kernel<T, V, 32, 1, 4, SAVED8>, false);
        case TALL: return shape_of<V, 32, 8, 1, 8>(scan_backward_kernel<T, V, 32, 8, 1, SAVED8>, true);
        default: return shape_of<V, 8, 8, 1, 8>(scan_backward_kernel<T, V, 8, 8, 1, SAVED8>, true);
    }
}

Shape pick(const dn_scan& s, bool pairs, bool forward, bool save8, Layout l) {
    switch (s.type) {
        case DN_F32: return forward ? forward_shape<float, 1>(l, save8) : save8 ? backward_shape<float, 1, true>(l) : backward_shape<float, 1, false>(l);
        case DN_BF16:
            if (pairs) return forward ? forward_shape<__nv_bfloat16, 2>(l, save8) : save8 ? backward_shape<__nv_bfloat16, 2, true>(l) : backward_shape<__nv_bfloat16, 2, false>(l);
            return forward ? forward_shape<__nv_bfloat16, 1>(l, save8) : save8 ? backward_shape<__nv_bfloat16, 1, true>(l) : backward_shape<__nv_bfloat16, 1, false>(l);
        default:
            if (pairs) return forward ? forward_shape<__half, 2>(l, save8) : save8 ? backward_shape<__half, 2, true>(l) : backward_shape<__half, 2, false>(l);
            return forward ? forward_shape<__half, 1>(l, save8) : save8 ? backward_shape<__half, 1, true>(l) : backward_shape<__half, 1, false>(l);
    }
}

constexpr int64_t MOST_GRID = 0x7fffffff;

// Layout and blocks per cluster.  A sample's strip of columns is marched by one block where there are enough strips to fill the
// device, else by a cluster along the rows; where even clusters of 16 leave SMs idle, strips of 8 lanes.
dn_status launch(const dn_scan& s, bool pairs, bool forward, ScanArgs& A, cudaStream_t stream) {
    const bool save8 = s.format != DN_SAVE_FULL;
    const int sms = sm_count();
    auto units = [&](const Shape& f) { return (((int64_t)s.cols + f.cols - 1) / f.cols) * s.batch; };
    Layout l = s.rows <= (forward ? 16 : 8) ? (s.rows <= 1 && !save8 ? ONE_ROW : SHORT) : TALL;
    Shape f = pick(s, pairs, forward, save8, l);
    if (l == TALL && !(forward && save8) && units(f) * SCAN_MOST_BLOCKS < sms) f = pick(s, pairs, forward, save8, NARROW);
    int blocks = 1;
    const int64_t n = units(f);
    if (f.split)
        while (blocks < SCAN_MOST_BLOCKS && n * blocks < 4 * sms && (int64_t)blocks * f.tile < s.rows) blocks *= 2;
    if (n * blocks > MOST_GRID) return DN_ERR_SIZE;
    A.strips = (s.cols + f.cols - 1) / f.cols;
    A.blocks = blocks;
    if (blocks > 8 && cudaFuncSetAttribute(f.kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) { (void)cudaGetLastError(); return DN_ERR_CUDA; }
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(n * blocks)); cfg.blockDim = dim3(f.threads); cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)blocks; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr; cfg.numAttrs = blocks > 1 ? 2 : 1;
    if (cudaLaunchKernelEx(&cfg, f.kernel, A) != cudaSuccess) { (void)cudaGetLastError(); return DN_ERR_CUDA; }
    return DN_OK;
}

// ---- checks of arguments --------------------------------------------------------------------------------------------------------
int element_bytes(int type) { return type == DN_F32 ? 4 : 2; }

dn_status check(const dn_scan* s) {
    if (!s) return DN_ERR_NULL;
    if (s->batch < 1 || s->cols < 1 || s->rows < 0 || s->rows > (1 << 30) || s->cols > (1 << 30)) return DN_ERR_SIZE;
    if (s->type < DN_F32 || s->type > DN_F16 || (s->flags & ~DN_SCAN_MIX) || s->format < DN_SAVE_FULL || s->format > DN_E4M3) return DN_ERR_MODE;
    // the most rows that a call touches, in elements and bytes, stay far below 2^63
    if ((double)s->batch * s->rows * s->cols > 1e15) return DN_ERR_SIZE;
    if ((((int64_t)s->cols + 7) / 8) * s->batch * SCAN_MOST_BLOCKS > MOST_GRID && (((int64_t)s->cols + 31) / 32) * s->batch * 4 > MOST_GRID) return DN_ERR_SIZE;
    return DN_OK;
}

constexpr int64_t MOST_STRIDE = (int64_t)1 << 46;

dn_status check_rows(const dn_scan& s, const dn_rows& r, bool output) {
    if (r.batch_stride < 0 || r.row_stride < 0 || r.batch_stride > MOST_STRIDE || r.row_stride > MOST_STRIDE) return DN_ERR_LAYOUT;
    if (s.rows == 0) return DN_OK;
    if (!r.data) return DN_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(r.data) % element_bytes(s.type)) return DN_ERR_LAYOUT;
    if ((double)(s.batch - 1) * r.batch_stride + (double)(s.rows - 1) * r.row_stride + s.cols > 4e15) return DN_ERR_LAYOUT;
    if (output) {
        // samples of whole row sets, or (time-major) rows of whole sample sets
        const int64_t inner = s.cols, B = s.batch, T = s.rows;
        const bool by_sample = (T == 1 || r.row_stride >= inner) && (B == 1 || r.batch_stride >= (T - 1) * r.row_stride + inner);
        const bool by_row = (B == 1 || r.batch_stride >= inner) && (T == 1 || r.row_stride >= (B - 1) * r.batch_stride + inner);
        // batch strides shorter than a sample's rows, with rows far apart, would interleave: columns of one wide array
        if (!by_sample && !by_row) return DN_ERR_LAYOUT;
    }
    return DN_OK;
}

struct Span { uintptr_t lo, hi; };
Span span_of(const void* p, size_t bytes) { return Span{reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + bytes}; }
Span span_of(const dn_scan& s, const dn_rows& r) {
    if (s.rows == 0 || !r.data) return Span{0, 0};
    return span_of(r.data, (size_t)(((s.batch - 1) * r.batch_stride + (s.rows - 1) * r.row_stride + s.cols) * element_bytes(s.type)));
}
bool meet(Span a, Span b) { return a.lo < b.hi && b.lo < a.hi; }
// Two arrays share an element: their spans meet, unless they are columns of one wider array (same strides, side by side).
bool meet(const dn_scan& s, const dn_rows& a, const dn_rows& b) {
    if (!meet(span_of(s, a), span_of(s, b))) return false;
    const int64_t e = element_bytes(s.type), inner = s.cols;
    const bool same = (s.rows == 1 || a.row_stride == b.row_stride) && (s.batch == 1 || a.batch_stride == b.batch_stride);
    if (!same) return true;
    const int64_t unit = s.rows > 1 && s.batch > 1 ? (a.row_stride < a.batch_stride ? a.row_stride : a.batch_stride)
                         : s.rows > 1 ? a.row_stride : s.batch > 1 ? a.batch_stride : 0;
    if (unit < 2 * inner || (s.rows > 1 && a.row_stride % unit) || (s.batch > 1 && a.batch_stride % unit)) return true;
    const int64_t d = (int64_t)(reinterpret_cast<uintptr_t>(a.data) - reinterpret_cast<uintptr_t>(b.data));
    if (d % e) return true;
    const int64_t off = ((d / e) % unit + unit) % unit;
    return off < inner || off > unit - inner;
}
// adjacent columns of a 16-bit array in one access of 4 bytes
bool paired(const dn_scan& s, const dn_rows* r) {
    return !r || !r->data || s.rows == 0 || (reinterpret_cast<uintptr_t>(r->data) % 4 == 0 && r->batch_stride % 2 == 0 && r->row_stride % 2 == 0);
}
RowsOf rows_of(const dn_scan& s, const dn_rows* r) {
    if (!r || !r->data) return RowsOf{nullptr, 0, 0};
    const int64_t e = element_bytes(s.type);
    return RowsOf{static_cast<char*>(r->data), r->batch_stride * e, r->row_stride * e};
}
dn_status check_checkpoint(const dn_scan& s, const void* p, size_t bytes, ScanArgs& A) {
    const ScanSaved l = scan_saved(s.batch, s.rows, s.cols, s.format);
    if (l.total && (!p || reinterpret_cast<uintptr_t>(p) % kAlign || bytes < l.total)) return DN_ERR_WORKSPACE;
    uint8_t* at = static_cast<uint8_t*>(const_cast<void*>(p));
    A.gq = at + l.gq; A.xq = at + l.xq; A.gs = at + l.gs; A.xs = at + l.xs;
    A.states = reinterpret_cast<float*>(at + l.states);
    A.rows_padded = l.rows_padded; A.nblk = l.nblk; A.nchunk = l.nchunk;
    return DN_OK;
}
#define DN_CHECK(x) do { const dn_status st_ = (x); if (st_ != DN_OK) return st_; } while (0)

}  // namespace
}  // namespace dn

using namespace dn;

extern "C" {

size_t dn_scan_checkpoint_bytes(const dn_scan* s) {
    if (check(s) != DN_OK) return 0;
    const size_t n = scan_saved(s->batch, s->rows, s->cols, s->format).total;
    return n ? n : kAlign;
}

dn_status dn_scan_forward(const dn_scan* s, const dn_rows* g, const dn_rows* x, const float* h0, const dn_rows* h, float* h_last,
                          void* checkpoint, size_t checkpoint_bytes, void* stream) {
    DN_CHECK(check(s));
    if (!g || !x || !h) return DN_ERR_NULL;
    DN_CHECK(check_rows(*s, *g, false));
    DN_CHECK(check_rows(*s, *x, false));
    DN_CHECK(check_rows(*s, *h, true));
    const size_t edge = (size_t)s->batch * s->cols * sizeof(float);
    if (reinterpret_cast<uintptr_t>(h0) % 4 || reinterpret_cast<uintptr_t>(h_last) % 4 || reinterpret_cast<uintptr_t>(s->lengths) % 4) return DN_ERR_LAYOUT;
    ScanArgs A{};
    dn_scan q = *s;
    if (checkpoint) DN_CHECK(check_checkpoint(*s, checkpoint, checkpoint_bytes, A));
    else { q.format = DN_SAVE_FULL; A.rows_padded = 0; }
    const Span out = span_of(*s, *h), last = span_of(h_last, h_last ? edge : 0), first = span_of(h0, h0 ? edge : 0);
    const Span len = span_of(s->lengths, s->lengths ? (size_t)s->batch * 4 : 0);
    const Span keep = span_of(checkpoint, checkpoint ? scan_saved(s->batch, s->rows, s->cols, s->format).total : 0);
    if (meet(*s, *h, *g) || meet(*s, *h, *x) || meet(out, first) || meet(out, last) || meet(out, len) || meet(out, keep)) return DN_ERR_ALIAS;
    if (meet(keep, span_of(*s, *g)) || meet(keep, span_of(*s, *x)) || meet(keep, first) || meet(keep, last) || meet(keep, len)) return DN_ERR_ALIAS;
    if (meet(last, span_of(*s, *g)) || meet(last, span_of(*s, *x)) || meet(last, len) || (h_last != h0 && meet(last, first))) return DN_ERR_ALIAS;
    A.g = rows_of(*s, g); A.x = rows_of(*s, x); A.h = rows_of(*s, h);
    A.start = h0; A.end = h_last; A.lengths = s->lengths;
    A.rows = s->rows; A.cols = s->cols;
    A.mix = (s->flags & DN_SCAN_MIX) != 0; A.int8 = q.format == DN_INT8;
    const bool pairs = s->type != DN_F32 && s->cols % 2 == 0 && paired(*s, g) && paired(*s, x) && paired(*s, h);
    return launch(q, pairs, true, A, static_cast<cudaStream_t>(stream));
}

dn_status dn_scan_backward(const dn_scan* s, const dn_rows* g, const dn_rows* x, const void* checkpoint, size_t checkpoint_bytes,
                           const dn_rows* dh, const float* dh_last, const dn_rows* dg, const dn_rows* dx, float* dh0, void* stream) {
    DN_CHECK(check(s));
    const bool full = s->format == DN_SAVE_FULL;
    if ((full && (!g || !x)) || !dg || !dx) return DN_ERR_NULL;
    if (full) { DN_CHECK(check_rows(*s, *g, false)); DN_CHECK(check_rows(*s, *x, false)); }
    if (dh && dh->data) DN_CHECK(check_rows(*s, *dh, false));
    DN_CHECK(check_rows(*s, *dg, true));
    DN_CHECK(check_rows(*s, *dx, true));
    const size_t edge = (size_t)s->batch * s->cols * sizeof(float);
    if (reinterpret_cast<uintptr_t>(dh0) % 4 || reinterpret_cast<uintptr_t>(dh_last) % 4 || reinterpret_cast<uintptr_t>(s->lengths) % 4) return DN_ERR_LAYOUT;
    ScanArgs A{};
    DN_CHECK(check_checkpoint(*s, checkpoint, checkpoint_bytes, A));
    const Span first = span_of(dh0, dh0 ? edge : 0), last = span_of(dh_last, dh_last ? edge : 0);
    const Span len = span_of(s->lengths, s->lengths ? (size_t)s->batch * 4 : 0);
    const Span keep = span_of(checkpoint, scan_saved(s->batch, s->rows, s->cols, s->format).total);
    const dn_rows none{nullptr, 0, 0};
    const dn_rows &in_g = full ? *g : none, &in_x = full ? *x : none, &in_d = dh ? *dh : none;
    for (const dn_rows* out : {dg, dx}) {
        const Span o = span_of(*s, *out);
        if (meet(*s, *out, in_g) || meet(*s, *out, in_x) || meet(*s, *out, in_d) || meet(o, first) || meet(o, last) || meet(o, len) || meet(o, keep)) return DN_ERR_ALIAS;
    }
    if (meet(*s, *dg, *dx)) return DN_ERR_ALIAS;
    if (meet(first, span_of(*s, in_g)) || meet(first, span_of(*s, in_x)) || meet(first, span_of(*s, in_d)) || meet(first, len) || meet(first, keep) ||
        (dh0 != dh_last && meet(first, last))) return DN_ERR_ALIAS;
    A.g = rows_of(*s, &in_g); A.x = rows_of(*s, &in_x); A.dh = rows_of(*s, &in_d); A.dg = rows_of(*s, dg); A.dx = rows_of(*s, dx);
    A.start = dh_last; A.end = dh0; A.lengths = s->lengths;
    A.rows = s->rows; A.cols = s->cols;
    A.mix = (s->flags & DN_SCAN_MIX) != 0; A.int8 = s->format == DN_INT8;
    const bool pairs = s->type != DN_F32 && s->cols % 2 == 0 && paired(*s, &in_g) && paired(*s, &in_x) && paired(*s, &in_d) && paired(*s, dg) && paired(*s, dx);
    return launch(*s, pairs, false, A, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
