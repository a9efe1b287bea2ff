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
//
// What moves the data.  Arrays on 16-byte places and strides: tiles of 64 rows (128 rows of half the columns) by bulk copies, two stages
// ahead of the arithmetic, results back the same way from a piece of shared memory per warp; that takes the address arithmetic off the
// threads (18 instructions per element of a 16-bit type forward, 29 with plain loads, 35 backward) and the raw tiles off their registers.
// Others: loads into registers a step ahead.  Where even clusters of 16 blocks leave SMs idle (fewer strips of columns on the whole device
// than a sixteenth of its SMs): lanes 8 across, 4 groups of rows down.  Up to 16 rows (backward 8): a thread per column, nothing to exchange.
//
// What bounds it.  Memory, where there are strips of columns enough: 1024^2 x 64 in 32 bits 134 us forward (92 % of the measured copy rate)
// and 218 us backward (95 %), 32 x 2048 x 2048 bf16 139 us (89 %).  With fewer, the last and uneven wave and the latency of a step (about 1 us
// forward, 1.3 backward: copy, 16 or 8 rows of dependent products, exchange): 8 x 2048 x 2048 bf16 39 us (80 %) and 66 us (78 %), one sequence of
// 65536 x 2048 170 us (73 %) and 330 us (63 %).  3.1 to 3.4 warps per scheduler fit, limited by the registers that hold a tile, and an
// instruction is issued in 54 to 55 % of the cycles; most stalls are waits for the result before.
// Measured and not kept: five blocks per SM forward (96 registers, a few spilled: 38 -> 44 us); three backward, with x and dh read again
// from shared memory (66 -> 90 us) or spilled (8-bit checkpoint 147 -> 204 us); dh kept in 16 bits until it is used (66 -> 71 us).
#include "dn_eight.cuh"

#include <cuda.h>

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
    int int8;                    // the input's format (the gate's always is)
    int copy_tries, block_tries; // limits of the waits for a tile and for the other blocks
};

template <class T, int V> using Raw = std::conditional_t<sizeof(T) * V == 4, uint32_t, uint16_t>;

template <class T, int V> __device__ __forceinline__ Cols<V> expand(Raw<T, V> r) {
    T t[V];
    memcpy(t, &r, sizeof t);
    Cols<V> f;
#pragma unroll
    for (int v = 0; v < V; ++v) f.v[v] = as_float(t[v]);
    return f;
}
template <class T, int V> __device__ __forceinline__ Raw<T, V> join(const Cols<V>& f) {
    T t[V];
#pragma unroll
    for (int v = 0; v < V; ++v) t[v] = rounded<T>(f.v[v]);
    Raw<T, V> r;
    memcpy(&r, t, sizeof r);
    return r;
}
// gates of 16-bit values are held to LEAST_GATE in 16 bits, both columns at once (-87 is a value of both types)
__device__ __forceinline__ uint32_t held(uint32_t r, __nv_bfloat16) {
    asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(r) : "r"(0xc2aec2aeu));
    return r;
}
__device__ __forceinline__ uint32_t held(uint32_t r, __half) {
    asm("max.NaN.f16x2 %0, %0, %1;" : "+r"(r) : "r"(0xd570d570u));
    return r;
}
template <class T, int V> __device__ __forceinline__ void gate_parts(Raw<T, V> r, Cols<V>& a, Cols<V>& w, float none) {
    if constexpr (sizeof(T) == 4) gates<true>(expand<T, V>(r), a, w, none);
    else if constexpr (V == 2) gates<false, true>(expand<T, V>(held(r, T())), a, w, none);
    else gates<false>(expand<T, V>(r), a, w, none);
}
// The gate of an 8-bit checkpoint is held to +-63.5 = 127 / 2, where its sigmoid is 1 or 0 to 2^-91: its 32 neighbours have steps of 1/2 at
// most, and an infinite one has a code.  Its bits without the sign, of 32-bit values the upper 16:
template <class T> inline constexpr uint32_t MOST_GATE8 = std::is_same_v<T, __half> ? 0x53f0u : 0x427eu;
__device__ __forceinline__ uint32_t held8(uint32_t r, __nv_bfloat16) {
    asm("min.NaN.bf16x2 %0, %0, %1;\n\tmax.NaN.bf16x2 %0, %0, %2;" : "+r"(r) : "r"(0x427e427eu), "r"(0xc27ec27eu));
    return r;
}
__device__ __forceinline__ uint32_t held8(uint32_t r, __half) {
    asm("min.NaN.f16x2 %0, %0, %1;\n\tmax.NaN.f16x2 %0, %0, %2;" : "+r"(r) : "r"(0x53f053f0u), "r"(0xd3f0d3f0u));
    return r;
}
__device__ __forceinline__ uint32_t held8(uint32_t r, float) { return r; }               // (not needed)
__device__ __forceinline__ float held8(float v) {
    asm("min.NaN.f32 %0, %0, %1;\n\tmax.NaN.f32 %0, %0, %2;" : "+f"(v) : "f"(63.5f), "f"(-63.5f));
    return v;
}
template <class W> __device__ __forceinline__ W load_at(const char* p) { return *reinterpret_cast<const W*>(p); }
template <class W> __device__ __forceinline__ void store_at(char* p, W v) { *reinterpret_cast<W*>(p) = v; }

__device__ __forceinline__ unsigned cluster_address(const void* local, int rank) {
    unsigned r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"((unsigned)__cvta_generic_to_shared(local)), "r"(rank));
    return r;
}
// A store into a block of the cluster that counts its bytes at a barrier there: what waits at the barrier sees what was stored.  A barrier
// of the whole cluster would make each block wait for its own stores of h as well.
__device__ __forceinline__ void cluster_send(unsigned at, unsigned bar, float a, float b) {
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.f32 [%0], {%1, %2}, [%3];" ::"r"(at), "f"(a), "f"(b), "r"(bar) : "memory");
}
__device__ __forceinline__ void cluster_send(unsigned at, unsigned bar, float a, float b, float c, float d) {
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1, %2, %3, %4}, [%5];" ::"r"(at), "f"(a), "f"(b), "f"(c), "f"(d), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ void barrier_init(uint64_t* bar) { asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"((unsigned)__cvta_generic_to_shared(bar)) : "memory"); }
__device__ __forceinline__ void barrier_expect(uint64_t* bar, unsigned bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"((unsigned)__cvta_generic_to_shared(bar)), "r"(bytes) : "memory");
}
// (the condition stands inside: around it the compiler makes two versions of a step, and spills)
__device__ __forceinline__ void barrier_expect_unless(int lost, uint64_t* bar, unsigned bytes) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.eq.u32 p, %2, 0;\n\t@p mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n\t}" ::"r"((unsigned)__cvta_generic_to_shared(bar)), "r"(bytes),
                 "r"(lost) : "memory");
}
// A copy arrives and the blocks of a cluster run together, so the wait ends; should it ever not (tries: each suspends the thread for
// about 4 us, a second in all), false.  A thread whose wait ran out is lost: all it finds from then on is NaN, and so is the map of its
// rows that the others of the block read.  It neither waits again nor sends nor orders anything, so the blocks that would hear from it are
// lost in turn.
constexpr int WAIT_TRIES = 1 << 18, LOST = 1 << 20;        // (LOST, what is added to a loop over blocks, is past them all)
__device__ __forceinline__ bool barrier_wait(uint64_t* bar, unsigned parity, int tries) {
    const unsigned at = (unsigned)__cvta_generic_to_shared(bar);
#pragma unroll 1
    for (int i = 0; i < tries; ++i) {
        unsigned done;
        asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                     : "=r"(done) : "r"(at), "r"(parity) : "memory");
        if (done) return true;
    }
    return false;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

// ---- bulk copies of tiles (coordinates: column, row, sample) ----
struct TileMaps { CUtensorMap in[3], out[4]; };            // g, x, dh; h or dg, dx, codes of g, codes of x
__device__ __forceinline__ void tile_load(void* to, const CUtensorMap& m, int col, int row, int b, uint64_t* bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(
                     (unsigned)__cvta_generic_to_shared(to)), "l"(&m), "r"(col), "r"(row), "r"(b), "r"((unsigned)__cvta_generic_to_shared(bar)) : "memory");
}
__device__ __forceinline__ void tile_store(const CUtensorMap& m, const void* from, int col, int row, int b) {
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(&m),
                 "r"((unsigned)__cvta_generic_to_shared(from)), "r"(col), "r"(row), "r"(b) : "memory");
}
__device__ __forceinline__ void stores_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
__device__ __forceinline__ void stores_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }   // their shared memory may be written again
__device__ __forceinline__ void stores_done() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
__device__ __forceinline__ unsigned char* on_128(unsigned char* shared) {         // the next multiple of 128 bytes
    return shared + (-(unsigned)__cvta_generic_to_shared(shared) & 127u);
}
__device__ __forceinline__ void shared_to_bulk() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

__device__ __forceinline__ float not_a_number() { return __uint_as_float(0x7fffffffu); }

// factors and offsets of V adjacent columns, in one access
template <int V> struct __align__(8 * V) Maps { Cols<V> p, h; };

// Where a thread works: lanes LX across the columns (V each) and 32 / LX down the rows, warps WR down and WC across, R rows each.
// An address is a place that is the same for the whole block, which the uniform registers hold, plus the thread's own offset, which does
// not change; Off is 64 bits wide only for rows so far apart that a tile of them passes 4 GiB.
template <int V, int LX, int WR, int WC, int R> struct Place {
    static constexpr int NG = WR * (32 / LX), COLS = WC * LX * V, TILE = NG * R, THREADS = 32 * WR * WC;
    int b, rank, first, q, col, c, len;
    bool cv, all;                // this thread's columns exist; the block's do
    __device__ Place(const ScanArgs& A) {
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        q = (warp % WR) * (32 / LX) + lane / LX;
        col = (warp / WR) * LX * V + (lane % LX) * V;
        const unsigned unit = blockIdx.x / A.blocks;
        rank = blockIdx.x % A.blocks;
        b = unit / A.strips;
        first = (int)(unit % A.strips) * COLS;
        c = first + col;
        cv = c < A.cols;
        all = first + COLS <= A.cols;
        len = A.rows;
    }
    __device__ void read_length(const ScanArgs& A) {
        if (A.lengths) len = min(max(A.lengths[b], 0), A.rows);
    }
    __device__ char* base(const RowsOf& r, int size) const { return r.p + b * r.batch + first * (int64_t)size; }
    template <class Off> __device__ Off offset(const RowsOf& r, int size) const { return (Off)(q * R) * (Off)r.row + (Off)(col * size); }
};
using Yes = std::true_type;
using No = std::false_type;

// Magnitudes of a row's gate (low half) and input (high half), the larger of the thread's columns: the upper 16 bits without the sign, whose
// order as integers is that of the magnitudes.
template <class T, int V> __device__ __forceinline__ uint32_t magnitudes(Raw<T, V> g, Raw<T, V> x) {
    if constexpr (sizeof(T) == 4) return __byte_perm(g, x, 0x7632) & 0x7fff7fffu;
    else if constexpr (V == 1) return (g | (uint32_t)x << 16) & 0x7fff7fffu;
    else return __vmaxu2(__byte_perm(g, x, 0x5410) & 0x7fff7fffu, __byte_perm(g, x, 0x7632) & 0x7fff7fffu);
}
// Per block: where it stands, and what a step of it exchanges.  The blocks of a cluster send one another the map of their tile; a buffer
// is written again two steps later, when its readers have sent what they found with it.
template <int V, int LX, int WR, int WC, int R> struct Exchange {
    using Pl = Place<V, LX, WR, WC, R>;
    static constexpr int NG = Pl::NG, LANES = WC * LX;
    Maps<V> agg[2][NG > 1 ? NG : 1][NG > 1 ? LANES : 1];
    uint64_t bars[2];
    int ordered;                 // tiles, where they come by bulk copies

    __device__ void init(int K) {
        if (K > 1 && threadIdx.x == 0) {
            barrier_init(&bars[0]);
            barrier_init(&bars[1]);
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
    }
    // The value that enters this thread's rows, from the map (p, h) of these rows and the value `carry` that enters the step's first ones;
    // carry becomes what leaves the last ones.  DOWN: rows are passed from the last to the first.  `between`: what to do once all maps of
    // the block can be read.  sent: what the blocks of the cluster sent, [2][K][LANES].
    template <bool DOWN, bool TILES, class F> __device__ __forceinline__ Cols<V> enter(Maps<V>* sent, int k, int K, int rank, int q, int lane, const Cols<V>& p, const Cols<V>& h, Cols<V>& carry, int& lost, int tries, F between) {
        if constexpr (NG == 1) {
            const Cols<V> in = carry;
            carry = fma(p, carry, h);
            between();
            return in;
        } else {
            const int buf = k & 1;
            agg[buf][q][lane] = Maps<V>{p, h};
            __syncthreads();
            between();
            Cols<V> in = carry;
            if (K == 1) {
#pragma unroll
                for (int i = 0; i < NG; ++i) {
                    const int j = DOWN ? NG - 1 - i : i;
                    const Maps<V> e = agg[buf][j][lane];
                    if (j == q) in = carry;
                    carry = fma(e.p, carry, e.h);
                }
                if (TILES && lost) in = all_of<V>(not_a_number());  // (carry is so by this thread's map)
                return in;
            }
            Cols<V> pb = all_of<V>(1.0f), hb = all_of<V>(0.0f), pt = pb, ht = hb;                // of the groups ahead of this one; of all
#pragma unroll
            for (int i = 0; i < NG; ++i) {
                const int j = DOWN ? NG - 1 - i : i;
                const Maps<V> e = agg[buf][j][lane];
                if (j == q) { pb = pt; hb = ht; }
                if (i == 0) { pt = e.p; ht = e.h; }
                else { ht = fma(e.p, ht, e.h); pt = mul(e.p, pt); }
            }
            for (int peer = q + lost; peer < K; peer += NG) {
                const unsigned to = cluster_address(&sent[(buf * K + rank) * LANES + lane], peer), bar = cluster_address(&bars[buf], peer);
                if constexpr (V == 1) cluster_send(to, bar, pt.v[0], ht.v[0]); else cluster_send(to, bar, pt.v[0], pt.v[1], ht.v[0], ht.v[1]);
            }
            if (threadIdx.x == 0) barrier_expect_unless(lost, &bars[buf], K * LANES * (unsigned)sizeof(Maps<V>));
            if (!lost && !barrier_wait(&bars[buf], (k >> 1) & 1, tries)) lost = LOST;
            const int ahead = DOWN ? K - 1 - rank : rank;
#pragma unroll 4
            for (int i = 0; i < ahead; ++i) {
                const Maps<V> e = sent[(buf * K + (DOWN ? K - 1 - i : i)) * LANES + lane];
                carry = fma(e.p, carry, e.h);
            }
            in = fma(pb, carry, hb);
#pragma unroll 4
            for (int i = ahead; i < K; ++i) {
                const Maps<V> e = sent[(buf * K + (DOWN ? K - 1 - i : i)) * LANES + lane];
                carry = fma(e.p, carry, e.h);
            }
            if (lost) in = carry = all_of<V>(not_a_number());
            return in;
        }
    }
};

// ---- forward -----------------------------------------------------------------------------------------------------------------
constexpr int FORWARD_STAGES = 2, BACKWARD_STAGES = 2;     // tiles of a block that are on their way or being read

// Shared memory of a block that moves its tiles by bulk copies: IN input tiles per stage, and per warp a piece of each output.
template <int STAGES, int IN_BYTES, int WARPS, int OUT_BYTES> struct __align__(128) Tiles {
    unsigned char in[STAGES][IN_BYTES];
    unsigned char out[WARPS][OUT_BYTES];
    uint64_t arrived[STAGES];
};
template <class T, int V, bool SAVE8> using ForwardTiles =
    Tiles<FORWARD_STAGES, 2 * 64 * 32 * V * (int)sizeof(T), 4, 16 * 32 * V * ((int)sizeof(T) + (SAVE8 ? 2 : 0))>;
template <class T, int V, bool SAVED8> using BackwardTiles =
    Tiles<BACKWARD_STAGES, 64 * 32 * V * (SAVED8 ? (int)sizeof(T) + 2 : 3 * (int)sizeof(T)), 8, 8 * 32 * V * 2 * (int)sizeof(T)>;

template <class T, int V, int LX, int WR, int WC, int R, bool SAVE8, bool MIX, bool BULK, class Off>
__global__ void __launch_bounds__(32 * WR * WC, SAVE8 && !BULK ? 3 : 4) scan_forward_kernel(const __grid_constant__ ScanArgs A, const __grid_constant__ TileMaps maps) {
    static_assert(!BULK || (WR == 4 && WC == 1 && R == 16), "the tiles and pieces of the tensor maps");
    static_assert(!SAVE8 || (LX * V >= 32 && R == 16), "a row's 32 columns of a scale lie in one warp, 16 rows' scales in 16 lanes");
    using Pl = Place<V, LX, WR, WC, R>;
    using W = Raw<T, V>;
    constexpr int NG = Pl::NG, TILE = Pl::TILE, S = sizeof(T);
    constexpr int ROW = LX * V * S, ST = FORWARD_STAGES;   // bytes of a tile's row
    [[maybe_unused]] constexpr int PIECE = 32 / LX * R;    // rows of a warp
    __shared__ Exchange<V, LX, WR, WC, R> ex;
    extern __shared__ __align__(128) unsigned char dynamic[];
    using Here = ForwardTiles<T, V, SAVE8>;
    [[maybe_unused]] Here& tiles = *reinterpret_cast<Here*>(on_128(dynamic));
    auto* const sent = reinterpret_cast<Maps<V>*>(BULK ? on_128(dynamic) + sizeof(Here) : dynamic);
    Pl at(A);
    const int q = at.q, c = at.c;
    const bool cv = at.cv;
    const int K = NG > 1 ? A.blocks : 1;
    ex.init(K);
    if constexpr (BULK) {
        if (threadIdx.x == 0) {
#pragma unroll
            for (int i = 0; i < ST; ++i) barrier_init(&tiles.arrived[i]);
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
        __syncthreads();
    }
    int lost = 0;
    const float none = S == 4 ? 0.0f : least_decay();
    dep_wait();
    at.read_length(A);
    const int len = at.len;
    const int span = K * TILE;
    const int steps = (int)(((int64_t)len + span - 1) / span);

    Cols<V> carry;
#pragma unroll
    for (int v = 0; v < V; ++v) carry.v[v] = (A.start && cv) ? A.start[(int64_t)at.b * A.cols + c + v] : 0.0f;

    const char *const bg = at.base(A.g, S), *const bx = at.base(A.x, S);
    char* const bh = at.base(A.h, S);
    const Off og = at.template offset<Off>(A.g, S), ox = at.template offset<Off>(A.x, S), oh = at.template offset<Off>(A.h, S);
    int row0 = at.rank * TILE;                             // of the block's tile; this thread's rows start at row0 + q R

    W rg[R], rx[R];
    auto fetch = [&](int r0) {
        const char *g = bg + r0 * A.g.row, *x = bx + r0 * A.x.row;
        if (at.all && r0 + TILE <= len) {
#pragma unroll
            for (int i = 0; i < R; ++i) {
                rg[i] = load_at<W>(g + i * A.g.row + og);
                rx[i] = load_at<W>(x + i * A.x.row + ox);
            }
        } else {
            const int n = cv ? len - r0 - q * R : 0;
#pragma unroll
            for (int i = 0; i < R; ++i) {
                rg[i] = i < n ? load_at<W>(g + i * A.g.row + og) : W(0);
                rx[i] = i < n ? load_at<W>(x + i * A.x.row + ox) : W(0);
            }
        }
    };
    [[maybe_unused]] auto order = [&](int s) {             // one thread: the tile of step s
        ex.ordered = s + 1;
        uint64_t* bar = &tiles.arrived[s % ST];
        unsigned char* to = tiles.in[s % ST];
        const int row = (s * K + at.rank) * TILE;
        barrier_expect(bar, 2 * TILE * ROW);
        tile_load(to, maps.in[0], at.first, row, at.b, bar);
        tile_load(to + TILE * ROW, maps.in[1], at.first, row, at.b, bar);
    };
    [[maybe_unused]] auto take = [&](int s) {              // this thread's part of it
        if (!lost && !barrier_wait(&tiles.arrived[s % ST], (s / ST) & 1, A.copy_tries)) lost = LOST;
        const unsigned char* from = tiles.in[s % ST] + q * R * ROW + at.col * S;
#pragma unroll
        for (int i = 0; i < R; ++i) {
            rg[i] = *reinterpret_cast<const W*>(from + i * ROW);
            rx[i] = *reinterpret_cast<const W*>(from + TILE * ROW + i * ROW);
        }
        if (SAVE8 && lost) {                               // (encode reads such rows from where they come from)
#pragma unroll
            for (int i = 0; i < R; ++i) rg[i] = (W)0x7fff7fffu;
        }
    };
    if constexpr (BULK) {
        if (threadIdx.x == 0)
            for (int s = 0; s < ST && s < steps; ++s) order(s);
    } else if (steps > 0) fetch(row0);
    if (K > 1) { cluster_arrive(); cluster_wait(); }       // every block of the cluster runs before one writes to another
    [[maybe_unused]] unsigned char* const mine_out = BULK ? tiles.out[threadIdx.x >> 5] + (threadIdx.x & 31) / LX * R * ROW + at.col * S : nullptr;
    [[maybe_unused]] unsigned char* const mine_codes =
        BULK ? tiles.out[threadIdx.x >> 5] + PIECE * ROW + (threadIdx.x & 31) / LX * R * LX * V + at.col : nullptr;

    // (8 x 4096 x 2048 bf16 with its 8-bit checkpoint: 133 us, 63 % of the copy rate, against 310 us with a reduction per row and conversions
    // by the unit that the exponentials use; 38 instructions per element.)
    // Codes and scales of this warp's 16 rows.  The largest magnitudes of the 16 rows are found together: at every stage of a butterfly a lane
    // hands half of its rows to the other and keeps the other's share of the rest, 15 exchanges of gate and input at once in place of 64
    // or 80; lane r then holds row r, works out its scales, and hands them round.
    [[maybe_unused]] auto encode = [&](auto full, int n) {
        constexpr bool FULL = decltype(full)::value;
        const int lane = threadIdx.x & 31, t0 = row0 + q * R;
        uint32_t m[R];
#pragma unroll
        for (int i = 0; i < R; ++i) m[i] = magnitudes<T, V>(rg[i], rx[i]);
#pragma unroll
        for (int h = 8; h >= 1; h /= 2)
#pragma unroll
            for (int j = 0; j < h; ++j) {
                const bool up = (lane & h) != 0;
                const uint32_t keep = up ? m[j + h] : m[j], send = up ? m[j] : m[j + h];
                m[j] = __vmaxu2(keep, __shfl_xor_sync(~0u, send, h));
            }
        if (V == 1) m[0] = __vmaxu2(m[0], __shfl_xor_sync(~0u, m[0], 16));
        const int eg = magnitude_exponent<T>(m[0] & 0xffffu), exx = magnitude_exponent<T>(m[0] >> 16);
        const int block = (at.first + (threadIdx.x >> 5) / WR * LX * V) / kBlock8 + (LX * V == 64 ? lane >> 4 : 0);
        uint8_t *const gs = A.gs + ((int64_t)at.b * A.nblk + block) * A.rows_padded + t0, *const xs = A.xs + ((int64_t)at.b * A.nblk + block) * A.rows_padded + t0;
        const bool mine = block < A.nblk && t0 < A.rows_padded;
        uint8_t *const gq = A.gq + (((int64_t)at.b * A.rows + row0) * A.cols + at.first), *const xq = A.xq + (((int64_t)at.b * A.rows + row0) * A.cols + at.first);
        const Off oq = (Off)(q * R) * (Off)A.cols + (Off)at.col;
        auto put = [&](int i, uint32_t kg, uint32_t kx) {
            using Q = std::conditional_t<V == 2, uint16_t, uint8_t>;
            if constexpr (BULK) {
                *reinterpret_cast<Q*>(mine_codes + i * LX * V) = (Q)kg;
                *reinterpret_cast<Q*>(mine_codes + (PIECE + i) * LX * V) = (Q)kx;
            } else if (FULL || i < n) {
                *reinterpret_cast<Q*>(gq + (int64_t)i * A.cols + oq) = (Q)kg;
                *reinterpret_cast<Q*>(xq + (int64_t)i * A.cols + oq) = (Q)kx;
            }
        };
        if (__any_sync(~0u, eg == 255 || exx == 255)) {    // values that are not finite: row by row
            const char *g = bg + row0 * A.g.row, *x = bx + row0 * A.x.row;
#pragma unroll 1
            for (int i = 0; i < R; ++i) {
                Cols<V> vg = expand<T, V>(i < n ? load_at<W>(g + i * A.g.row + og) : W(0)), vx = expand<T, V>(i < n ? load_at<W>(x + i * A.x.row + ox) : W(0));
                unsigned mg = 0, mx = 0;
#pragma unroll
                for (int v = 0; v < V; ++v) { vg.v[v] = held8(vg.v[v]); mg = max(mg, magnitude_bits(vg.v[v])); mx = max(mx, magnitude_bits(vx.v[v])); }
#pragma unroll
                for (int h = V == 2 ? 8 : 16; h >= 1; h /= 2) { mg = max(mg, __shfl_xor_sync(~0u, mg, h)); mx = max(mx, __shfl_xor_sync(~0u, mx, h)); }
                const int sg = scale_byte(mg, true), sx = scale_byte(mx, A.int8);
                uint32_t kg = 0, kx = 0;
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    kg |= code_int8(vg.v[v], inverse_scale_of(sg)) << (8 * v);
                    kx |= code8(vx.v[v], inverse_scale_of(sx), A.int8) << (8 * v);
                }
                put(i, kg, kx);
                if (mine && (lane & (V == 2 ? 15 : 31)) == 0) { gs[i] = (uint8_t)sg; xs[i] = (uint8_t)sx; }
            }
            return;
        }
        const int sg = max(min(eg, 132) - 6, 1), sx = max(exx - (A.int8 ? 6 : 7), 1);
        if (mine && (V == 2 || lane < 16)) { gs[lane & 15] = (uint8_t)sg; xs[lane & 15] = (uint8_t)sx; }
        const uint32_t inverse = (uint32_t)(254 - sg) << 7 | (uint32_t)(254 - sx) << 23;            // upper halves of the two floats
        auto codes = [&](auto far) {
#pragma unroll
            for (int i = 0; i < R; ++i) {
                const uint32_t both = __shfl_sync(~0u, inverse, V == 2 ? (lane & 16) | i : i);
                W g = rg[i];
                if constexpr (decltype(far)::value) g = (W)held8(g, T());
                const uint32_t kg = codes_int8(expand<T, V>(g), __uint_as_float(both << 16));
                const Cols<V> vx = expand<T, V>(rx[i]);
                const float ix = __uint_as_float(both & 0xffff0000u);
                put(i, kg, A.int8 ? codes_int8(vx, ix) : codes_e4m3(vx, ix));
            }
        };
        // (codes of single values are held to 127 themselves)
        if constexpr (V == 2) {
            if (__any_sync(~0u, (m[0] & 0xffffu) > MOST_GATE8<T>)) { codes(Yes{}); return; }
        }
        codes(No{});
    };

    Cols<V> a[R], bb[R], P, H;
    // rows i < n of this thread hold data; the others (none in a full tile) pass the state on
    auto prepare = [&](auto full, int n) {
        constexpr bool FULL = decltype(full)::value;
        if constexpr (SAVE8) encode(full, n);
#pragma unroll
        for (int i = 0; i < R; ++i) {
            Cols<V> w;
            gate_parts<T, V>(rg[i], a[i], w, none);
            bb[i] = expand<T, V>(rx[i]);
            if (MIX) bb[i] = mul(w, bb[i]);
            if (!FULL && i >= n) { a[i] = all_of<V>(1.0f); bb[i] = all_of<V>(0.0f); }
            P = i ? mul(P, a[i]) : a[i];
            H = i ? fma(a[i], H, bb[i]) : bb[i];
        }
    };

    for (int s = 0; s < steps; ++s) {
        const bool full = at.all && row0 + TILE <= len;
        const int t0 = row0 + q * R, n = cv ? len - t0 : 0;
        if constexpr (BULK) {
            take(s);
            if ((threadIdx.x & 31) == 0) stores_read();    // the pieces of the step before
            __syncwarp();
        }
        if (full) prepare(Yes{}, n); else prepare(No{}, n);
        if (BULK && lost) P = all_of<V>(not_a_number());
        if constexpr (!BULK)
            if (s + 1 < steps) fetch(row0 + span);         // in flight while the states of this step are found

        Cols<V> hin = ex.template enter<false, BULK>(sent, s, K, at.rank, q, at.col / V, P, H, carry, lost, A.block_tries, [&] {
            if constexpr (BULK)
                if (threadIdx.x == 0 && !lost && s + ST < steps) order(s + ST);          // the block has read this step's tile
        });
        if (A.states && cv && t0 % kChunkRows == 0 && t0 < A.rows) {
            float* st = A.states + ((int64_t)at.b * A.nchunk + t0 / kChunkRows) * A.cols + c;
#pragma unroll
            for (int v = 0; v < V; ++v) st[v] = hin.v[v];
        }
        char* ph = bh + row0 * A.h.row;
        if constexpr (BULK) {
#pragma unroll
            for (int i = 0; i < R; ++i) {
                hin = fma(a[i], hin, bb[i]);
                *reinterpret_cast<W*>(mine_out + i * ROW) = full || i < n ? join<T, V>(hin) : W(0);
            }
            shared_to_bulk();
            __syncwarp();
            if ((threadIdx.x & 31) == 0 && t0 < A.rows) {
                const unsigned char* from = tiles.out[threadIdx.x >> 5];
                tile_store(maps.out[0], from, at.first, t0, at.b);
                if (SAVE8) {
                    tile_store(maps.out[2], from + PIECE * ROW, at.first, t0, at.b);
                    tile_store(maps.out[3], from + PIECE * ROW + PIECE * LX * V, at.first, t0, at.b);
                }
                stores_commit();
            }
        } else if (full) {
#pragma unroll
            for (int i = 0; i < R; ++i) {
                hin = fma(a[i], hin, bb[i]);
                store_at<W>(ph + i * A.h.row + oh, join<T, V>(hin));
            }
        } else {
            const int m = cv ? A.rows - t0 : 0;
#pragma unroll
            for (int i = 0; i < R; ++i) {
                hin = fma(a[i], hin, bb[i]);
                if (i < m) store_at<W>(ph + i * A.h.row + oh, i < n ? join<T, V>(hin) : W(0));
            }
        }
        row0 += span;
    }
    for (; row0 < A.rows; row0 += span)                    // rows behind a sequence
        for (int i = 0; i < R && i < A.rows - row0 - q * R; ++i)
            if (cv) store_at<W>(bh + (row0 + i) * A.h.row + oh, W(0));
    if (A.end && at.rank == 0 && q == 0 && cv) {
#pragma unroll
        for (int v = 0; v < V; ++v) A.end[(int64_t)at.b * A.cols + c + v] = carry.v[v];
    }
    if (BULK && (threadIdx.x & 31) == 0) stores_done();
    if (BULK && lost && threadIdx.x == 0)                  // the block stays until what is on its way to it has landed
        for (int i = max(ex.ordered - ST, 0); i < ex.ordered; ++i) barrier_wait(&tiles.arrived[i % ST], (i / ST) & 1, WAIT_TRIES);
    if (K > 1) { cluster_arrive(); cluster_wait(); }       // no block's shared memory goes while another could write to it
    if (lost) __nanosleep(100000);                         // nor while what another sent before it was lost is on its way
}

// ---- backward ----------------------------------------------------------------------------------------------------------------
template <class T, int V, int LX, int WR, int WC, bool SAVED8, bool MIX, bool BULK, class Off>
__global__ void __launch_bounds__(32 * WR * WC, 16 / (WR * WC)) scan_backward_kernel(const __grid_constant__ ScanArgs A, const __grid_constant__ TileMaps maps) {
    constexpr int R = 8, GC = kChunkRows / R;              // 8 scale bytes are one load; groups of a chunk
    static_assert(!BULK || (LX == 32 && WR == 8 && WC == 1), "the tiles and pieces of the tensor maps");
    using Pl = Place<V, LX, WR, WC, R>;
    using W = Raw<T, V>;
    using Q = std::conditional_t<V == 2, uint16_t, uint8_t>;
    constexpr int NG = Pl::NG, TILE = Pl::TILE, S = sizeof(T);
    static_assert(NG == 1 || TILE % kChunkRows == 0, "a tile holds whole chunks, or is the only one");
    __shared__ Exchange<V, LX, WR, WC, R> ex;
    __shared__ Cols<V> aggH[2][NG > 1 ? NG : 1][NG > 1 ? WC * LX : 1];
    constexpr int ROW = 32 * V * S, QROW = SAVED8 ? 32 * V : ROW, ST = BACKWARD_STAGES;      // bytes of a row of dh, of gate and input
    extern __shared__ __align__(128) unsigned char dynamic[];
    using Here = BackwardTiles<T, V, SAVED8>;
    [[maybe_unused]] Here& tiles = *reinterpret_cast<Here*>(on_128(dynamic));
    auto* const sent = reinterpret_cast<Maps<V>*>(BULK ? on_128(dynamic) + sizeof(Here) : dynamic);
    Pl at(A);
    const int q = at.q, c = at.c, lane = at.col / V;
    const bool cv = at.cv;
    const int K = NG > 1 ? A.blocks : 1;
    ex.init(K);
    if constexpr (BULK) {
        if (threadIdx.x == 0) {
#pragma unroll
            for (int i = 0; i < ST; ++i) barrier_init(&tiles.arrived[i]);
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
        __syncthreads();
    }
    int lost = 0;
    const float none = S == 4 ? 0.0f : least_decay();
    dep_wait();
    at.read_length(A);
    const int len = at.len;
    const int span = K * TILE;
    const int steps = (int)(((int64_t)len + span - 1) / span);

    Cols<V> carry;                                         // mu of the row behind
#pragma unroll
    for (int v = 0; v < V; ++v) carry.v[v] = (A.start && cv) ? A.start[(int64_t)at.b * A.cols + c + v] : 0.0f;

    const char *const bg = SAVED8 ? nullptr : at.base(A.g, S), *const bx = SAVED8 ? nullptr : at.base(A.x, S), *const bd = A.dh.p ? at.base(A.dh, S) : nullptr;
    char *const bdg = at.base(A.dg, S), *const bdx = at.base(A.dx, S);
    const Off og = at.template offset<Off>(A.g, S), ox = at.template offset<Off>(A.x, S), od = at.template offset<Off>(A.dh, S);
    const Off odg = at.template offset<Off>(A.dg, S), odx = at.template offset<Off>(A.dx, S), oq = (Off)(q * R) * (Off)A.cols + (Off)at.col;

    for (int r0 = steps * span + at.rank * TILE; r0 < A.rows; r0 += span)            // rows behind a sequence
        for (int i = 0; i < R && i < A.rows - r0 - q * R; ++i)
            if (cv) {
                store_at<W>(bdg + (r0 + i) * A.dg.row + odg, W(0));
                store_at<W>(bdx + (r0 + i) * A.dx.row + odx, W(0));
            }

    int row0 = (steps - 1) * span + at.rank * TILE;
    W rg[SAVED8 ? 1 : R], rx[SAVED8 ? 1 : R], rd[R];
    Q qg[SAVED8 ? R : 1], qx[SAVED8 ? R : 1];
    uint2 sg{}, sx{};
    Cols<V> st;
    const int qc = NG > 1 ? q % GC : 0;                    // groups of the same chunk ahead of this one
    auto fetch_rows = [&](auto full, int r0) {
        constexpr bool FULL = decltype(full)::value;
        const int t = r0 + q * R, n = cv ? len - t : 0;
        if constexpr (SAVED8) {
            if (FULL || n > 0) {
                const int64_t os = ((int64_t)at.b * A.nblk + c / kBlock8) * A.rows_padded + t;
                sg = *reinterpret_cast<const uint2*>(A.gs + os);
                sx = *reinterpret_cast<const uint2*>(A.xs + os);
            }
        }
        const float* ps = A.states + ((int64_t)at.b * A.nchunk + t / kChunkRows) * A.cols + c;
#pragma unroll
        for (int v = 0; v < V; ++v) st.v[v] = FULL || n > 0 ? ps[v] : 0.0f;
        if constexpr (BULK) return;
        if constexpr (SAVED8) {
            const int64_t o = ((int64_t)at.b * A.rows + r0) * A.cols + at.first;
#pragma unroll
            for (int i = 0; i < R; ++i) {
                qg[i] = FULL || i < n ? *reinterpret_cast<const Q*>(A.gq + (o + (int64_t)i * A.cols) + oq) : Q(0x8080);
                qx[i] = FULL || i < n ? *reinterpret_cast<const Q*>(A.xq + (o + (int64_t)i * A.cols) + oq) : Q(0x8080);
            }
        } else {
            const char *g = bg + r0 * A.g.row, *x = bx + r0 * A.x.row;
#pragma unroll
            for (int i = 0; i < R; ++i) {
                rg[i] = FULL || i < n ? load_at<W>(g + i * A.g.row + og) : W(0);
                rx[i] = FULL || i < n ? load_at<W>(x + i * A.x.row + ox) : W(0);
            }
        }
        const char* d = bd + r0 * A.dh.row;
#pragma unroll
        for (int i = 0; i < R; ++i) rd[i] = (FULL || i < n) && bd ? load_at<W>(d + i * A.dh.row + od) : W(0);
    };
    auto fetch = [&](int r0) {
        if (at.all && r0 + TILE <= len) fetch_rows(Yes{}, r0); else fetch_rows(No{}, r0);
    };
    [[maybe_unused]] auto order = [&](int k) {             // one thread: the tile of the k-th step
        ex.ordered = k + 1;
        uint64_t* bar = &tiles.arrived[k % ST];
        unsigned char* to = tiles.in[k % ST];
        const int row = ((steps - 1 - k) * K + at.rank) * TILE;
        barrier_expect(bar, TILE * (2 * QROW + (bd ? ROW : 0)));
        tile_load(to, maps.in[0], at.first, row, at.b, bar);
        tile_load(to + TILE * QROW, maps.in[1], at.first, row, at.b, bar);
        if (bd) tile_load(to + 2 * TILE * QROW, maps.in[2], at.first, row, at.b, bar);
    };
    [[maybe_unused]] auto take = [&](int k) {              // this thread's part of it
        if (!lost && !barrier_wait(&tiles.arrived[k % ST], (k / ST) & 1, A.copy_tries)) lost = LOST;
        const unsigned char *from = tiles.in[k % ST] + q * R * QROW + at.col * (QROW / (32 * V)), *fd = tiles.in[k % ST] + 2 * TILE * QROW + q * R * ROW + at.col * S;
#pragma unroll
        for (int i = 0; i < R; ++i) {
            if constexpr (SAVED8) {
                qg[i] = *reinterpret_cast<const Q*>(from + i * QROW);
                qx[i] = *reinterpret_cast<const Q*>(from + TILE * QROW + i * QROW);
            } else {
                rg[i] = *reinterpret_cast<const W*>(from + i * QROW);
                rx[i] = *reinterpret_cast<const W*>(from + TILE * QROW + i * QROW);
            }
            rd[i] = bd ? *reinterpret_cast<const W*>(fd + i * ROW) : W(0);
        }
    };
    if constexpr (BULK) {
        if (threadIdx.x == 0)
            for (int k = 0; k < ST && k < steps; ++k) order(k);
    }
    if (steps > 0) fetch(row0);
    if (K > 1) { cluster_arrive(); cluster_wait(); }
    [[maybe_unused]] unsigned char* const mine_out = BULK ? tiles.out[threadIdx.x >> 5] + at.col * S : nullptr;

    Cols<V> a[R], w[R], x[R], d[R], P, H, M;
    auto prepare = [&](auto full, int n) {
        constexpr bool FULL = decltype(full)::value;
        uint32_t zero_g = 0, zero_x = 0;
        if constexpr (SAVED8) {
            constexpr int PER = 4 / V;                     // rows whose codes fill a word
#pragma unroll
            for (int i = 0; i < R; i += PER) {
                uint32_t wg = 0, wx = 0;
#pragma unroll
                for (int j = 0; j < PER; ++j) { wg |= (uint32_t)qg[i + j] << (8 * V * j); wx |= (uint32_t)qx[i + j] << (8 * V * j); }
                zero_g |= any_zero_byte(wg);
                zero_x |= any_zero_byte(wx);
            }
            if (!A.int8) zero_x = 0;
#pragma unroll
            for (int i = 0; i < R; ++i) w[i] = values_int8<V>(qg[i], scale_of(((i < 4 ? sg.x : sg.y) >> (8 * (i % 4))) & 255));
            if (A.int8) {
#pragma unroll
                for (int i = 0; i < R; ++i) x[i] = values_int8<V>(qx[i], scale_of(((i < 4 ? sx.x : sx.y) >> (8 * (i % 4))) & 255));
            } else {
#pragma unroll
                for (int i = 0; i < R; ++i) x[i] = values_e4m3<V>(qx[i], scale_of(((i < 4 ? sx.x : sx.y) >> (8 * (i % 4))) & 255));
            }
            if (zero_g | zero_x) {                         // rare: some value of this thread was not finite
#pragma unroll
                for (int i = 0; i < R; ++i)
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        if (((qg[i] >> (8 * v)) & 255) == 0) w[i].v[v] = __uint_as_float(0x7fffffffu);
                        if (A.int8 && ((qx[i] >> (8 * v)) & 255) == 0) x[i].v[v] = __uint_as_float(0x7fffffffu);
                    }
            }
        }
#pragma unroll
        for (int i = 0; i < R; ++i) {
            if constexpr (SAVED8) {
                const Cols<V> g = w[i];
                gates<S == 4>(g, a[i], w[i], none);
            } else {
                gate_parts<T, V>(rg[i], a[i], w[i], none);
                x[i] = expand<T, V>(rx[i]);
            }
            d[i] = expand<T, V>(rd[i]);
            if (!FULL && i >= n) { a[i] = all_of<V>(1.0f); w[i] = x[i] = d[i] = all_of<V>(0.0f); }
            const Cols<V> in = MIX ? mul(w[i], x[i]) : x[i];
            P = i ? mul(P, a[i]) : a[i];
            H = i ? fma(a[i], H, in) : in;
            M = i ? fma(d[i], P, M) : mul(d[i], P);        // what enters row i passes through a_i .. a_0
        }
    };
    auto write = [&](auto full, int n, int m, Cols<V> mu) {
        constexpr bool FULL = decltype(full)::value;
        char *pdg = bdg + row0 * A.dg.row, *pdx = bdx + row0 * A.dx.row;
#pragma unroll
        for (int i = R - 1; i >= 0; --i) {
            const Cols<V> lam = add(d[i], mu), og_ = mul(lam, x[i]), ox_ = MIX ? mul(lam, w[i]) : lam;
            mu = mul(a[i], lam);
            if constexpr (BULK) {
                *reinterpret_cast<W*>(mine_out + i * ROW) = FULL || i < n ? join<T, V>(og_) : W(0);
                *reinterpret_cast<W*>(mine_out + (R + i) * ROW) = FULL || i < n ? join<T, V>(ox_) : W(0);
            } else if (FULL || i < m) {
                store_at<W>(pdg + i * A.dg.row + odg, FULL || i < n ? join<T, V>(og_) : W(0));
                store_at<W>(pdx + i * A.dx.row + odx, FULL || i < n ? join<T, V>(ox_) : W(0));
            }
        }
        if constexpr (BULK) {
            shared_to_bulk();
            __syncwarp();
            if ((threadIdx.x & 31) == 0 && row0 + q * R < A.rows) {
                const unsigned char* from = tiles.out[threadIdx.x >> 5];
                tile_store(maps.out[0], from, at.first, row0 + q * R, at.b);
                tile_store(maps.out[1], from + R * ROW, at.first, row0 + q * R, at.b);
                stores_commit();
            }
        }
    };

    for (int s = steps - 1; s >= 0; --s) {
        const bool full = at.all && row0 + TILE <= len;
        const int t0 = row0 + q * R, n = cv ? len - t0 : 0, k = steps - 1 - s, buf = k & 1;
        Cols<V> hin = st;
        if constexpr (BULK) {
            take(k);
            if ((threadIdx.x & 31) == 0) stores_read();    // the pieces of the step before
            __syncwarp();
        }
        if (full) prepare(Yes{}, n); else prepare(No{}, n);
        if (BULK && lost) P = all_of<V>(not_a_number());
        if (s > 0) fetch(row0 - span);                     // (with bulk copies: states and scales)

        if constexpr (NG > 1) aggH[buf][q][lane] = H;
        const Cols<V> mu = ex.template enter<true, BULK>(sent, k, K, at.rank, q, lane, P, M, carry, lost, A.block_tries, [&] {
            if constexpr (BULK)
                if (threadIdx.x == 0 && !lost && k + ST < steps) order(k + ST);          // the block has read this step's tile
            if constexpr (NG > 1)
                for (int j = q - qc; j < q; ++j) hin = fma(ex.agg[buf][j][lane].p, hin, aggH[buf][j][lane]);
        });
        // x <- a (1 - a) (h_{t-1} [- x]), the factor of dg
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const Cols<V> in = MIX ? mul(w[i], x[i]) : x[i];
            const Cols<V> diff = MIX ? fma(x[i], all_of<V>(-1.0f), hin) : hin;
            hin = fma(a[i], hin, in);
            x[i] = mul(mul(a[i], w[i]), diff);
        }
        const int m = cv ? A.rows - t0 : 0;
        if (full) write(Yes{}, n, m, mu); else write(No{}, n, m, mu);
        row0 -= span;
    }
    if (A.end && at.rank == 0 && q == 0 && cv) {
#pragma unroll
        for (int v = 0; v < V; ++v) A.end[(int64_t)at.b * A.cols + c + v] = carry.v[v];
    }
    if (BULK && (threadIdx.x & 31) == 0) stores_done();
    if (BULK && lost && threadIdx.x == 0)                  // the block stays until what is on its way to it has landed
        for (int i = max(ex.ordered - ST, 0); i < ex.ordered; ++i) barrier_wait(&tiles.arrived[i % ST], (i / ST) & 1, WAIT_TRIES);
    if (K > 1) { cluster_arrive(); cluster_wait(); }
    if (lost) __nanosleep(100000);
}

// ---- launches ----------------------------------------------------------------------------------------------------------------
using Kernel = void (*)(ScanArgs, TileMaps);

struct Shape {                   // of a launch
    Kernel kernel;
    int cols, tile, threads;     // columns and rows of a block
    bool split;                  // a column's rows may be shared by the blocks of a cluster
    int tiles;                   // bytes of shared memory of the kernels that move their tiles by bulk copies, else 0
    int piece;                   // rows that a warp of those stores
    int sent;                    // bytes that a block of a cluster receives per block and step
    double latency;              // us of a step of a block that has its SM to itself
    // With bulk copies at least what lets 512 threads onto an SM (of its 228 KB), no more: 32-bit kernels have registers for another
    // block, and with it 64 x 1024^2 is 228 us backward in place of 218, 16 x 1024^2 from 8 bits 81 in place of 76 (the last wave is emptier).
    int shared(int blocks) const {
        const int need = (tiles ? tiles + 128 : 0) + (blocks > 1 ? 2 * blocks * sent : 0), least = tiles ? (228 << 10) / (512 / threads + 1) : 0;
        return need > least ? need : least;
    }
};
template <int V, int LX, int WR, int WC, int R> Shape shape_of(Kernel k, bool split, int tiles = 0) {
    using Pl = Place<V, LX, WR, WC, R>;
    return Shape{k, Pl::COLS, Pl::TILE, Pl::THREADS, split, tiles, 32 / LX * R, WC * LX * (int)sizeof(Maps<V>), (R == 8 ? 1.1 : 0.8) + 0.15 * (32 / LX - 1)};
}

// TALL_FAR: rows so far apart that offsets within a tile take 64 bits; BULK: TALL with bulk copies of tiles; BULK_HALF: strips of half the
// columns and tiles of twice the rows (forward)
enum Layout { ONE_ROW, SHORT, TALL, NARROW, TALL_FAR, BULK, BULK_HALF };
using Near = uint32_t;
using Far = int64_t;

template <class T, int V, bool MIX> Shape forward_shape(Layout l, bool save8) {
    if constexpr (sizeof(T) * V == 4)
        if (l == BULK)
            return save8 ? shape_of<V, 32, 4, 1, 16>(scan_forward_kernel<T, V, 32, 4, 1, 16, true, MIX, true, Far>, true, sizeof(ForwardTiles<T, V, true>))
                         : shape_of<V, 32, 4, 1, 16>(scan_forward_kernel<T, V, 32, 4, 1, 16, false, MIX, true, Far>, true, sizeof(ForwardTiles<T, V, false>));
    if constexpr (sizeof(T) * V == 4)
        if (l == BULK_HALF && !save8)
            return shape_of<V, 16, 4, 1, 16>(scan_forward_kernel<T, V, 16, 4, 1, 16, false, MIX, true, Far>, true, sizeof(ForwardTiles<T, V, false>));
    if constexpr (V == 2)
        if (l == BULK_HALF && save8)
            return shape_of<V, 16, 4, 1, 16>(scan_forward_kernel<T, V, 16, 4, 1, 16, true, MIX, true, Far>, true, sizeof(ForwardTiles<T, V, true>));
    if (save8) switch (l) {
        case ONE_ROW:
        case SHORT: return shape_of<V, 32, 1, 4, 16>(scan_forward_kernel<T, V, 32, 1, 4, 16, true, MIX, false, Near>, false);
        case TALL_FAR: return shape_of<V, 32, 4, 1, 16>(scan_forward_kernel<T, V, 32, 4, 1, 16, true, MIX, false, Far>, true);
        default: return shape_of<V, 32, 4, 1, 16>(scan_forward_kernel<T, V, 32, 4, 1, 16, true, MIX, false, Near>, true);
    }
    switch (l) {
        case ONE_ROW: return shape_of<V, 32, 1, 4, 1>(scan_forward_kernel<T, V, 32, 1, 4, 1, false, MIX, false, Near>, false);
        case SHORT: return shape_of<V, 32, 1, 4, 16>(scan_forward_kernel<T, V, 32, 1, 4, 16, false, MIX, false, Near>, false);
        case NARROW: return shape_of<V, 8, 4, 1, 16>(scan_forward_kernel<T, V, 8, 4, 1, 16, false, MIX, false, Near>, true);
        case TALL_FAR: return shape_of<V, 32, 4, 1, 16>(scan_forward_kernel<T, V, 32, 4, 1, 16, false, MIX, false, Far>, true);
        default: return shape_of<V, 32, 4, 1, 16>(scan_forward_kernel<T, V, 32, 4, 1, 16, false, MIX, false, Near>, true);
    }
}
template <class T, int V, bool SAVED8, bool MIX> Shape backward_shape(Layout l) {
    if constexpr (sizeof(T) * V == 4)
        if (l == BULK || l == BULK_HALF) return shape_of<V, 32, 8, 1, 8>(scan_backward_kernel<T, V, 32, 8, 1, SAVED8, MIX, true, Far>, true, sizeof(BackwardTiles<T, V, SAVED8>));
    switch (l) {
        case ONE_ROW:
        case SHORT: return shape_of<V, 32, 1, 4, 8>(scan_backward_kernel<T, V, 32, 1, 4, SAVED8, MIX, false, Near>, false);
        case NARROW: return shape_of<V, 8, 8, 1, 8>(scan_backward_kernel<T, V, 8, 8, 1, SAVED8, MIX, false, Near>, true);
        case TALL_FAR: return shape_of<V, 32, 8, 1, 8>(scan_backward_kernel<T, V, 32, 8, 1, SAVED8, MIX, false, Far>, true);
        default: return shape_of<V, 32, 8, 1, 8>(scan_backward_kernel<T, V, 32, 8, 1, SAVED8, MIX, false, Near>, true);
    }
}
template <class T, int V> Shape shape_for(bool mix, bool forward, bool save8, Layout l) {
    if (forward) return mix ? forward_shape<T, V, true>(l, save8) : forward_shape<T, V, false>(l, save8);
    if (save8) return mix ? backward_shape<T, V, true, true>(l) : backward_shape<T, V, true, false>(l);
    return mix ? backward_shape<T, V, false, true>(l) : backward_shape<T, V, false, false>(l);
}

Shape pick(const dn_scan& s, bool pairs, bool forward, bool save8, Layout l) {
    const bool mix = (s.flags & DN_SCAN_MIX) != 0;
    switch (s.type) {
        case DN_F32: return shape_for<float, 1>(mix, forward, save8, l);
        case DN_BF16: return pairs ? shape_for<__nv_bfloat16, 2>(mix, forward, save8, l) : shape_for<__nv_bfloat16, 1>(mix, forward, save8, l);
        default: return pairs ? shape_for<__half, 2>(mix, forward, save8, l) : shape_for<__half, 1>(mix, forward, save8, l);
    }
}

constexpr int64_t MOST_GRID = 0x7fffffff;

// Clusters of `blocks` blocks that the device holds at a time.
int active_clusters(const Shape& f, int blocks) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(blocks); cfg.blockDim = dim3(f.threads); cfg.dynamicSmemBytes = f.shared(blocks);
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = (unsigned)blocks; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
    cfg.attrs = at; cfg.numAttrs = 1;
    int n = 0;
    if (cudaFuncSetAttribute(f.kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess ||
        cudaFuncSetAttribute(f.kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, f.shared(SCAN_MOST_BLOCKS)) != cudaSuccess || cudaOccupancyMaxActiveClusters(&n, f.kernel, &cfg) != cudaSuccess) { (void)cudaGetLastError(); return 0; }
    return n;
}

// Blocks per cluster for n strips of columns and the time that they are estimated to take.
//
// A step takes a latency (loads, arithmetic, exchange: f.latency us), 0.2 us more where blocks wait for one another, and more the more blocks
// share an SM, 1.4 us with all its slots taken; a wave takes 3 us to start and end.  Measured on 32 strips of 65536 rows of 64 columns in 16
// bits, us per step (64 rows a block): a block each 0.88, clusters of 2 1.16, of 4 1.19, of 8 1.57 (201 us for all); of 16 1.93, but only 27 such
// fit the device at a time (247 us).  As 64 strips of 32 columns, 128 rows a block: 1.03, 1.34, 1.65, clusters of 8 2.6 (168 us).
struct Plan { int blocks; double time; };
Plan plan_for(const Shape& f, int64_t n, int rows) {
    struct Known { Kernel kernel; int dev, rows; int64_t n; Plan plan; };
    constexpr int KEPT = 16;
    thread_local Known known[KEPT] = {};                   // the last few answers: a function of the arguments and the device
    thread_local int next = 0;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) { (void)cudaGetLastError(); return Plan{1, 0.0}; }
    for (const Known& k : known)
        if (k.kernel == f.kernel && k.dev == dev && k.rows == rows && k.n == n) return k.plan;
    const double sms = sm_count();
    const int64_t most = ((int64_t)rows + f.tile - 1) / f.tile;
    Plan best{1, 1e30};
    double slots = 1.0;
    for (int k = 1; k <= SCAN_MOST_BLOCKS && k <= most; ++k) {
        const int64_t active = active_clusters(f, k);
        if (active < 1) continue;
        if (k == 1) slots = active / sms;
        const double waves = n < 3 * active ? (double)((n + active - 1) / active) : (double)n / active;
        const double steps = (double)((rows + (int64_t)k * f.tile - 1) / ((int64_t)k * f.tile));
        const double taken = (double)(n < active ? n : active) * k / sms;
        const double t = waves * (steps * (f.latency + (k > 1 ? 0.2 + 0.01 * k : 0.0) + 1.4 * taken / slots) + 3.0);
        if (t < best.time) best = Plan{k, t};
        if (waves > 4.0) break;                            // strips enough to fill the device several times
    }
    known[next] = Known{f.kernel, dev, rows, n, best};
    next = (next + 1) % KEPT;
    return best;
}

// ---- tensor maps -------------------------------------------------------------------------------------------------------------
int element_bytes(int type) { return type == DN_F32 ? 4 : 2; }

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                                 CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiled encode_tiled() {                               // the driver's function, looked up once; NULL: the kernels without bulk copies serve
    static const EncodeTiled f = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) {
            (void)cudaGetLastError();
            p = nullptr;
        }
        return reinterpret_cast<EncodeTiled>(p);
    }();
    return f;
}
// What a bulk copy asks of an array: 16-byte places and strides, none of them 0 (a row that all share), below 2^40 bytes.
bool bulk_fits(const dn_scan& s, const RowsOf& r) {
    if (!r.p) return true;
    auto stride = [](int64_t n, int64_t b) { return n <= 1 || (b > 0 && b % 16 == 0 && b < ((int64_t)1 << 40)); };
    return reinterpret_cast<uintptr_t>(r.p) % 16 == 0 && stride(s.rows, r.row) && stride(s.batch, r.batch);
}
bool tile_map(CUtensorMap* m, const dn_scan& s, const RowsOf& r, int type, int cols, int rows) {           // type: dn_type, or -1 for bytes
    const CUtensorMapDataType t = type == DN_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : type == DN_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                                  : type == DN_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_UINT8;
    const cuuint64_t dims[3] = {(cuuint64_t)s.cols, (cuuint64_t)s.rows, (cuuint64_t)s.batch};
    const cuuint64_t strides[2] = {(cuuint64_t)r.row, (cuuint64_t)(s.batch > 1 ? r.batch : r.row)};       // (of one sample: any; there are more rows than one)
    const cuuint32_t box[3] = {(cuuint32_t)cols, (cuuint32_t)rows, 1}, one[3] = {1, 1, 1};
    return encode_tiled()(m, t, 3, r.p, dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
bool tile_maps(TileMaps* m, const dn_scan& s, const ScanArgs& A, bool forward, const Shape& f) {
    const bool save8 = s.format != DN_SAVE_FULL;
    const RowsOf gq{reinterpret_cast<char*>(A.gq), (int64_t)s.rows * s.cols, s.cols}, xq{reinterpret_cast<char*>(A.xq), (int64_t)s.rows * s.cols, s.cols};
    if (forward)
        return tile_map(&m->in[0], s, A.g, s.type, f.cols, f.tile) && tile_map(&m->in[1], s, A.x, s.type, f.cols, f.tile) &&
               tile_map(&m->out[0], s, A.h, s.type, f.cols, f.piece) &&
               (!save8 || (tile_map(&m->out[2], s, gq, -1, f.cols, f.piece) && tile_map(&m->out[3], s, xq, -1, f.cols, f.piece)));
    return tile_map(&m->in[0], s, save8 ? gq : A.g, save8 ? -1 : s.type, f.cols, f.tile) &&
           tile_map(&m->in[1], s, save8 ? xq : A.x, save8 ? -1 : s.type, f.cols, f.tile) && (!A.dh.p || tile_map(&m->in[2], s, A.dh, s.type, f.cols, f.tile)) &&
           tile_map(&m->out[0], s, A.dg, s.type, f.cols, f.piece) && tile_map(&m->out[1], s, A.dx, s.type, f.cols, f.piece);
}

// Layout and blocks per cluster.  A sample's strip of columns is marched by one block where there are enough strips to fill the
// device, else by a cluster along the rows; where even clusters of 16 leave SMs idle, strips of 8 lanes.
dn_status launch(const dn_scan& s, bool pairs, bool forward, ScanArgs& A, cudaStream_t stream) {
    const bool save8 = s.format != DN_SAVE_FULL;
    const int sms = sm_count();
    auto units = [&](const Shape& f) { return (((int64_t)s.cols + f.cols - 1) / f.cols) * s.batch; };
    Layout l = s.rows <= (forward ? 16 : 8) ? (s.rows <= 1 && !save8 ? ONE_ROW : SHORT) : TALL;
    Shape f = pick(s, pairs, forward, save8, l);
    TileMaps maps{};
    if (l == TALL) {
        int64_t row = save8 ? s.cols : 0;                  // bytes between rows, at most
        for (const RowsOf& r : {A.g, A.x, A.h, A.dh, A.dg, A.dx}) row = r.row > row ? r.row : row;
        const bool far = (row + 1) * 64 + 4096 > (int64_t)UINT32_MAX, very = (row + 1) * 256 + 4096 > (int64_t)UINT32_MAX;
        bool bulk = (s.type == DN_F32 || pairs) && (!save8 || s.cols % 16 == 0) && encode_tiled() != nullptr;
        for (const RowsOf& r : {A.g, A.x, A.h, A.dh, A.dg, A.dx}) bulk = bulk && bulk_fits(s, r);
        if (!far && !very && !(forward && save8) && units(f) * SCAN_MOST_BLOCKS < sms) f = pick(s, pairs, forward, save8, NARROW);
        else {
            const Shape g = pick(s, pairs, forward, save8, BULK);
            if (bulk && tile_maps(&maps, s, A, forward, g)) {
                f = g;
                const Shape h = pick(s, pairs, forward, save8, BULK_HALF);
                if (h.cols < g.cols && plan_for(h, units(h), s.rows).time < plan_for(g, units(g), s.rows).time && tile_maps(&maps, s, A, forward, h)) f = h;
            } else if (far) f = pick(s, pairs, forward, save8, TALL_FAR);
        }
    }
    int blocks = 1;
    const int64_t n = units(f);
    if (f.split) blocks = plan_for(f, n, s.rows).blocks;
    if (n * blocks > MOST_GRID) return DN_ERR_SIZE;
    A.strips = (s.cols + f.cols - 1) / f.cols;
    A.blocks = blocks;
    A.copy_tries = s.flags & DN_SCAN_GIVE_UP_TILES ? 0 : WAIT_TRIES;
    A.block_tries = s.flags & DN_SCAN_GIVE_UP_BLOCKS ? 0 : WAIT_TRIES;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(n * blocks)); cfg.blockDim = dim3(f.threads); cfg.stream = stream; cfg.dynamicSmemBytes = f.shared(blocks);
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)blocks; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr; cfg.numAttrs = blocks > 1 ? 2 : 1;
    if (cudaLaunchKernelEx(&cfg, f.kernel, A, maps) != cudaSuccess) { (void)cudaGetLastError(); return DN_ERR_CUDA; }
    return DN_OK;
}

// ---- checks of arguments --------------------------------------------------------------------------------------------------------
dn_status check(const dn_scan* s) {
    if (!s) return DN_ERR_NULL;
    if (s->batch < 1 || s->cols < 1 || s->rows < 0 || s->rows > (1 << 30) || s->cols > (1 << 30)) return DN_ERR_SIZE;
    if (s->type < DN_F32 || s->type > DN_F16 || (s->flags & ~(DN_SCAN_MIX | DN_SCAN_GIVE_UP_TILES | DN_SCAN_GIVE_UP_BLOCKS)) || s->format < DN_SAVE_FULL || s->format > DN_E4M3) return DN_ERR_MODE;
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
    A.int8 = q.format == DN_INT8;
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
    A.int8 = s->format == DN_INT8;
    const bool pairs = s->type != DN_F32 && s->cols % 2 == 0 && paired(*s, &in_g) && paired(*s, &in_x) && paired(*s, &in_d) && paired(*s, dg) && paired(*s, dx);
    return launch(*s, pairs, false, A, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
