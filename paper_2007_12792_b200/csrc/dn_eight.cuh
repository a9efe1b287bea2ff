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

#include "dn_internal.cuh"

namespace dn {

constexpr int kBlock8 = 32;            // values that share a scale
constexpr int kChunkRows = 64;         // rows between two states that a checkpoint of the scan keeps in 32 bits

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

// p = 1 / (1 + e^-z) and q = 1 / (1 + e^z).  The smaller is e^-|z| / (1 + e^-|z|), to a few units in its own last place (one minus the
// other would have 10 bits left for z = 10); the larger is one minus the smaller, which is rounded once: a quotient would be off by a few
// units of 2^-24, the same way row after row, and a decay near 1 multiplies hundreds of them.  e^-|z| cannot overflow, and both are
// exactly 0 or 1 at z = +-inf.  ACCURATE: expf instead of the approximate exponential, whose
// relative error grows with |z| to 1e-6; 16-bit results do not show that.
template <bool ACCURATE>
__device__ __forceinline__ void gates(float z, float& p, float& q) {
    const float e = ACCURATE ? expf(-fabsf(z)) : __expf(-fabsf(z));
    const float less = __fdividef(e, 1.0f + e), more = 1.0f - less;
    const bool up = z >= 0.0f;
    p = up ? more : less;
    q = up ? less : more;
}

// |v| as bits, 0 where v is not finite: the order of these as integers is that of the magnitudes
__device__ __forceinline__ unsigned magnitude_bits(float v) {
    const unsigned m = __float_as_uint(v) & 0x7fffffffu;
    return m < 0x7f800000u ? m : 0u;
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

// an integer 0 .. 255 set into the last bits of 2^23 becomes a float without the conversion unit, which the exponentials need
__device__ __forceinline__ float value_int8(unsigned code, float scale) {
    const float v = (__uint_as_float(0x4b000000u | code) - 8388736.0f) * scale;
    return code ? v : __uint_as_float(0x7fffffffu);
}
__device__ __forceinline__ float value_e4m3(unsigned code, float scale) {
    return __half2float(__half(__nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)code, __NV_E4M3))) * scale;
}
__device__ __forceinline__ float value8(unsigned code, float scale, bool int8) { return int8 ? value_int8(code, scale) : value_e4m3(code, scale); }
#endif

}  // namespace dn
