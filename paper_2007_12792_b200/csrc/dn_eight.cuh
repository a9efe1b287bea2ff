// Values in 8 bits: blocks of 32 share a scale 2^e, one byte each.
//
//   A  = largest finite magnitude of the block, 2^k <= A < 2^(k+1)
//   int8:  e = max(k - 6, -126), code = rint(v / 2^e) held to [-127, 127]; stored + 128 (1 .. 255), 0 stands for "not finite"
//   e4m3:  e = max(k - 7, -126), code = e4m3 nearest to v / 2^e held to [-240, 240]; 0x7f stands for "not finite"
//
// A scale that is a power of two costs up to one bit of the code, and makes v / 2^e, code * 2^e and the scale itself exact: the code's
// rounding is the only one, every implementation of these lines finds the same values, and reading back takes a shift and a product.
// |value - v| <= 2^e / 2, for int8 < 2^e where |v| > 127.5 * 2^e (held to 127 instead of a coarser scale for the whole block: so
// nothing that is read back lies beyond the type it came from); e4m3: |value - v| <= 2^-4 |v|, or 2^e * 2^-10 for small v.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include <type_traits>

#include "dn_internal.cuh"

namespace dn {

constexpr int kBlock8 = 32;            // values that share a scale
constexpr int kChunkRows = DN_SCAN_CHUNK;  // rows between two states that a checkpoint of the scan keeps in 32 bits

// Where things live in a checkpoint of the scan (byte offsets, 256-byte aligned): codes [batch][rows][cols] of gate and input, their
// scales [batch][blocks of 32 columns][rows, padded to a multiple of 64] (rows innermost: a thread that owns consecutive rows of a
// column moves their scales in one access), and the state ahead of every 64th row, [batch][ceil(rows / 64)][cols] floats.
struct ScanSaved {
    size_t gq, xq, gs, xs, states, total;
    int nblk, nchunk;
    int64_t rows_padded;
};
inline ScanSaved scan_saved(int64_t batch, int64_t rows, int64_t cols, int format) {
    ScanSaved s{};
    s.nblk = (int)((cols + kBlock8 - 1) / kBlock8);
    s.nchunk = (int)((rows + kChunkRows - 1) / kChunkRows);
    s.rows_padded = (int64_t)s.nchunk * kChunkRows;
    size_t off = 0;
    const size_t codes = format ? align_up((size_t)batch * rows * cols) : 0;
    const size_t scales = format ? align_up((size_t)batch * s.nblk * s.rows_padded) : 0;
    s.gq = off; off += codes;
    s.xq = off; off += codes;
    s.gs = off; off += scales;
    s.xs = off; off += scales;
    s.states = off; off += align_up((size_t)batch * s.nchunk * cols * sizeof(float));
    s.total = off;
    return s;
}

#ifdef __CUDACC__
__device__ __forceinline__ float as_float(float v) { return v; }
__device__ __forceinline__ float as_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float as_float(__half v) { return __half2float(v); }
template <class T> __device__ __forceinline__ T rounded(float v);
template <> __device__ __forceinline__ float rounded<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 rounded<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half rounded<__half>(float v) { return __float2half_rn(v); }

// Values of V adjacent columns; two are worked on by one instruction where there is one for pairs.
template <int V> struct __align__(4 * V) Cols { float v[V]; };
template <int V> __device__ __forceinline__ Cols<V> all_of(float f) {
    Cols<V> r;
#pragma unroll
    for (int v = 0; v < V; ++v) r.v[v] = f;
    return r;
}
__device__ __forceinline__ unsigned long long pair_bits(const Cols<2>& c) {
    unsigned long long r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(c.v[0]), "f"(c.v[1]));
    return r;
}
__device__ __forceinline__ Cols<2> pair_of(unsigned long long b) {
    Cols<2> r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.v[0]), "=f"(r.v[1]) : "l"(b));
    return r;
}
__device__ __forceinline__ Cols<1> mul(Cols<1> a, Cols<1> b) { return Cols<1>{{a.v[0] * b.v[0]}}; }
__device__ __forceinline__ Cols<1> add(Cols<1> a, Cols<1> b) { return Cols<1>{{a.v[0] + b.v[0]}}; }
__device__ __forceinline__ Cols<1> fma(Cols<1> a, Cols<1> b, Cols<1> c) { return Cols<1>{{fmaf(a.v[0], b.v[0], c.v[0])}}; }
__device__ __forceinline__ Cols<2> mul(Cols<2> a, Cols<2> b) {
    unsigned long long r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(pair_bits(a)), "l"(pair_bits(b)));
    return pair_of(r);
}
__device__ __forceinline__ Cols<2> add(Cols<2> a, Cols<2> b) {
    unsigned long long r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(pair_bits(a)), "l"(pair_bits(b)));
    return pair_of(r);
}
__device__ __forceinline__ Cols<2> fma(Cols<2> a, Cols<2> b, Cols<2> c) {
    unsigned long long r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(pair_bits(a)), "l"(pair_bits(b)), "l"(pair_bits(c)));
    return pair_of(r);
}

// p = 1 / (1 + e^-z) and q = 1 / (1 + e^z), each to a few units in its own last place (one minus the other would have 10 bits left for
// z = 10): the smaller is e^-|z| / (1 + e^-|z|), the larger is one minus the smaller, which is rounded once: a quotient would be off by a
// unit of 2^-24, the same way row after row, and a decay near 1 multiplies hundreds of them.  Both are exactly 0 or 1 at z = +-inf.
// ACCURATE, for 32-bit results: expf; else the approximate exponential, whose relative error grows with |z| to 1e-6, which 16-bit
// results do not show.
template <bool ACCURATE> __device__ __forceinline__ void two_sided_gates(float z, float& p, float& q) {
    const float e = ACCURATE ? expf(-fabsf(z)) : __expf(-fabsf(z));
    const float less = __fdividef(e, 1.0f + e), more = 1.0f - less;
    const bool up = z >= 0.0f;
    p = up ? more : less;
    q = up ? less : more;
}

// The same as the decay and the input's weight of the recurrence.  For 16-bit types with z held to at least LEAST_GATE, so that e^-z cannot
// overflow, and what that leaves of p (2^-125) taken away, so that p is 0 there: 6 operations instead of some 16, 10 for two columns.
// Of p near 1 that is off by 2^-23 at most (1 + e^-z rounded, its reciprocal an ulp off), 3.5e-8 on average against 1.7e-8 for one minus the
// smaller part, which would take 5 more operations for two columns; neither keeps more than a few digits of 1 - p where p decays slowly.
// HELD: the caller has held z.  none: least_decay().
constexpr float LEAST_GATE = -87.0f;
__device__ __forceinline__ void exponential_gate(float t, float& e) { asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(t)); }
__device__ __forceinline__ void reciprocal_gate(float d, float& p) { asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(p) : "f"(d)); }
__device__ __forceinline__ float least_decay() {           // the operations of gates() below, at LEAST_GATE
    float e, p;
    exponential_gate(__fmul_rn(LEAST_GATE, -1.4426950408889634f), e);
    reciprocal_gate(__fadd_rn(e, 1.0f), p);
    return -p;
}
template <bool ACCURATE, bool HELD = false, int V>
__device__ __forceinline__ void gates(const Cols<V>& z, Cols<V>& p, Cols<V>& q, float none) {
    if constexpr (ACCURATE) {
#pragma unroll
        for (int v = 0; v < V; ++v) two_sided_gates<true>(z.v[v], p.v[v], q.v[v]);
    } else {
        Cols<V> t = z, e;
        if (!HELD)
#pragma unroll
            for (int v = 0; v < V; ++v) asm("max.NaN.f32 %0, %0, %1;" : "+f"(t.v[v]) : "f"(LEAST_GATE));
        t = mul(t, all_of<V>(-1.4426950408889634f));       // - log2 e
#pragma unroll
        for (int v = 0; v < V; ++v) exponential_gate(t.v[v], e.v[v]);
        const Cols<V> d = add(e, all_of<V>(1.0f));
#pragma unroll
        for (int v = 0; v < V; ++v) reciprocal_gate(d.v[v], p.v[v]);
        q = mul(e, p);
        p = add(p, all_of<V>(none));
    }
}
// |v| as bits, 0 where v is not finite: the order of these as integers is that of the magnitudes
__device__ __forceinline__ unsigned magnitude_bits(float v) {
    const unsigned m = __float_as_uint(v) & 0x7fffffffu;
    return m < 0x7f800000u ? m : 0u;
}
// the biased exponent (255: not finite) of a value whose upper 16 bits without the sign these are
template <class T> __device__ __forceinline__ int magnitude_exponent(uint32_t upper) {
    if constexpr (std::is_same_v<T, __half>) return (int)(__float_as_uint(__half2float(__ushort_as_half((unsigned short)upper))) >> 23);
    else return (int)(upper >> 7);
}
// the scale's byte (e + 127, 1 .. 248) for a block whose largest magnitude has these bits
__device__ __forceinline__ int scale_byte(unsigned bits, bool int8) {
    const int b = (int)(bits >> 23) - (int8 ? 6 : 7);
    return b > 1 ? b : 1;
}
__device__ __forceinline__ float scale_of(int byte) { return __uint_as_float((unsigned)byte << 23); }
__device__ __forceinline__ float inverse_scale_of(int byte) { return __uint_as_float((unsigned)(254 - byte) << 23); }

__device__ __forceinline__ unsigned code_int8(float v, float inverse) {
    const float q = fminf(fmaxf(rintf(v * inverse), -127.0f), 127.0f);
    return (__float_as_uint(v) & 0x7fffffffu) < 0x7f800000u ? (unsigned)(__float2int_rn(q) + 128) : 0u;
}
__device__ __forceinline__ unsigned code_e4m3(float v, float inverse) {
    const float q = fminf(fmaxf(v * inverse, -240.0f), 240.0f);            // rounding is monotonic and 240 is a value: held before or after
    return (__float_as_uint(v) & 0x7fffffffu) < 0x7f800000u ? (unsigned)__nv_cvt_float_to_fp8(q, __NV_SATFINITE, __NV_E4M3) : 0x7fu;
}
__device__ __forceinline__ unsigned code8(float v, float inverse, bool int8) { return int8 ? code_int8(v, inverse) : code_e4m3(v, inverse); }

__device__ __forceinline__ float value_e4m3(unsigned code, float scale) {
    return __half2float(__half(__nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)code, __NV_E4M3))) * scale;
}
// Codes of V adjacent columns, first column in the lowest byte.  v / 2^e + 2^23 + 2^22 + 128 is rounded to an integer by the sum itself
// (the quotient is exact, and inside a fused product and sum not even formed); the code then stands in the last bits.  The values are
// finite.
__device__ __forceinline__ uint32_t codes_int8(const Cols<1>& v, float inverse) {
    const int t = __float_as_int(fmaf(v.v[0], inverse, 12583040.0f));
    return (uint32_t)(min(max(t, 0x4b400001), 0x4b4000ff) & 255);
}
__device__ __forceinline__ uint32_t codes_int8(const Cols<2>& v, float inverse) {
    const Cols<2> t = fma(v, all_of<2>(inverse), all_of<2>(12583040.0f));
    const uint32_t w = __byte_perm(__float_as_uint(t.v[0]), __float_as_uint(t.v[1]), 0x5410);      // 0 .. 256 in either half
    return __byte_perm(__vmaxu2(__vminu2(w, 0x00ff00ffu), 0x00010001u), 0u, 0x4420);
}
__device__ __forceinline__ uint32_t codes_e4m3(const Cols<1>& v, float inverse) { return code_e4m3(v.v[0], inverse); }
__device__ __forceinline__ uint32_t codes_e4m3(const Cols<2>& v, float inverse) {
    const Cols<2> t = mul(v, all_of<2>(inverse));
    const float2 h = make_float2(fminf(fmaxf(t.v[0], -240.0f), 240.0f), fminf(fmaxf(t.v[1], -240.0f), 240.0f));
    return (uint32_t)__nv_cvt_float2_to_fp8x2(h, __NV_SATFINITE, __NV_E4M3);
}
// ... and back: a code set into the last bits of 2^23 is a float without the conversion unit, which the exponentials need.  A code 0, not a number, is read as -128 here: the caller looks for it (any_zero_byte).
template <int V> __device__ __forceinline__ Cols<V> values_int8(uint32_t codes, float scale) {
    Cols<V> f;
    f.v[0] = __uint_as_float(__byte_perm(codes, 0x4b000000u, 0x7440));
    if constexpr (V == 2) f.v[1] = __uint_as_float(__byte_perm(codes, 0x4b000000u, 0x7441));
    return mul(add(f, all_of<V>(-8388736.0f)), all_of<V>(scale));
}
template <int V> __device__ __forceinline__ Cols<V> values_e4m3(uint32_t codes, float scale) {
    if constexpr (V == 1) return Cols<1>{{value_e4m3(codes, scale)}};
    else {
        const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)codes, __NV_E4M3);
        return mul(Cols<2>{{__half2float(__half(__half_raw{h.x})), __half2float(__half(__half_raw{h.y}))}}, all_of<2>(scale));
    }
}
__device__ __forceinline__ uint32_t any_zero_byte(uint32_t w) { return (w - 0x01010101u) & ~w & 0x80808080u; }
#endif

}  // namespace dn
