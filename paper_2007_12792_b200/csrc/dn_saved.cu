// Tensors saved in 8 bits, and pointwise activations whose backward pass reads their input in 8 bits.
//
// All four kernels are one pass over memory: a thread takes 8 adjacent values (16 bytes of a 16-bit type, twice that of a 32-bit one),
// four lanes share a block of 32 and its scale, and UNITS such loads of a thread are in flight at a time.  The activation's forward
// kernel writes y and the packed input from one read of x; its backward kernel reads the packed input and dy and writes dx: 10 bytes
// per element of a 16-bit type for both, 12 with the input kept as it is.
#include "dn_eight.cuh"

namespace dn {
namespace {

constexpr int SAVED_THREADS = 256, UNIT = 8, UNITS = 4;

__host__ __device__ constexpr int64_t scales_at(int64_t n) { return (n + 15) / 16 * 16; }

template <class T> __device__ __forceinline__ void load_unit(const T* p, int64_t i, int64_t n, bool wide, float (&f)[UNIT]) {
    if (wide && i + UNIT <= n) {
        T t[UNIT];
        constexpr int W = UNIT * sizeof(T) / 16;
        uint4 r[W];
#pragma unroll
        for (int k = 0; k < W; ++k) r[k] = reinterpret_cast<const uint4*>(p + i)[k];
        memcpy(t, r, sizeof t);
#pragma unroll
        for (int j = 0; j < UNIT; ++j) f[j] = as_float(t[j]);
    } else {
#pragma unroll
        for (int j = 0; j < UNIT; ++j) f[j] = i + j < n ? as_float(p[i + j]) : 0.0f;
    }
}
template <class T> __device__ __forceinline__ void store_unit(T* p, int64_t i, int64_t n, bool wide, const float (&f)[UNIT]) {
    if (wide && i + UNIT <= n) {
        T t[UNIT];
        constexpr int W = UNIT * sizeof(T) / 16;
        uint4 r[W];
#pragma unroll
        for (int j = 0; j < UNIT; ++j) t[j] = rounded<T>(f[j]);
        memcpy(r, t, sizeof t);
#pragma unroll
        for (int k = 0; k < W; ++k) reinterpret_cast<uint4*>(p + i)[k] = r[k];
    } else {
#pragma unroll
        for (int j = 0; j < UNIT; ++j)
            if (i + j < n) p[i + j] = rounded<T>(f[j]);
    }
}

// the codes and the scale of a block, from the four lanes that hold it (each warp calls this as a whole)
__device__ __forceinline__ void store_codes(uint8_t* packed, int64_t i, int64_t n, bool int8, const float (&f)[UNIT]) {
    unsigned m = 0;
#pragma unroll
    for (int j = 0; j < UNIT; ++j) m = max(m, magnitude_bits(f[j]));
    m = max(m, __shfl_xor_sync(~0u, m, 1));
    m = max(m, __shfl_xor_sync(~0u, m, 2));
    const int byte = scale_byte(m, int8);
    const float inverse = inverse_scale_of(byte);
    uint32_t c[2] = {};
#pragma unroll
    for (int j = 0; j < UNIT; ++j) c[j / 4] |= code8(f[j], inverse, int8) << (8 * (j % 4));
    if (i + UNIT <= n) {
        *reinterpret_cast<uint2*>(packed + i) = make_uint2(c[0], c[1]);
    } else {
#pragma unroll
        for (int j = 0; j < UNIT; ++j)
            if (i + j < n) packed[i + j] = (uint8_t)(c[j / 4] >> (8 * (j % 4)));
    }
    if (i % kBlock8 == 0 && i < n) packed[scales_at(n) + i / kBlock8] = (uint8_t)byte;
}
struct Codes { uint32_t c[2]; int byte; };
__device__ __forceinline__ Codes load_codes(const uint8_t* packed, int64_t i, int64_t n) {
    Codes r{};
    if (i + UNIT <= n) {
        const uint2 u = *reinterpret_cast<const uint2*>(packed + i);
        r.c[0] = u.x;
        r.c[1] = u.y;
    } else {
#pragma unroll
        for (int j = 0; j < UNIT; ++j)
            if (i + j < n) r.c[j / 4] |= (uint32_t)packed[i + j] << (8 * (j % 4));
    }
    if (i < n) r.byte = packed[scales_at(n) + i / kBlock8];
    return r;
}
__device__ __forceinline__ void values_of(const Codes& r, bool int8, float (&f)[UNIT]) {
    const float scale = scale_of(r.byte);
#pragma unroll
    for (int j = 0; j < UNIT; ++j) f[j] = value8((r.c[j / 4] >> (8 * (j % 4))) & 255, scale, int8);
}

// z of the gate s(z) and dz/dx; beyond |x| = 16 the gate is 0 or 1 to the last bit and x^3 could overflow
template <int KIND> __device__ __forceinline__ float gate_argument(float x, float& dz) {
    if (KIND == DN_SILU) { dz = 1.0f; return x; }
    constexpr float two_c = 1.5957691216057308f;           // 2 sqrt(2 / pi)
    const float t = fabsf(x) > 16.0f ? copysignf(16.0f, x) : x, t2 = t * t;
    dz = two_c * fmaf(3.0f * 0.044715f, t2, 1.0f);
    return two_c * t * fmaf(0.044715f, t2, 1.0f);
}
template <int KIND, bool ACCURATE> __device__ __forceinline__ float activation(float x) {
    if (KIND == DN_TANH) return tanhf(x);
    float dz, p, q;
    two_sided_gates<ACCURATE>(gate_argument<KIND>(x, dz), p, q);
    return x * p;
}
template <int KIND, bool ACCURATE> __device__ __forceinline__ float slope(float x) {
    float dz, p, q;
    if (KIND == DN_TANH) {                                 // 1 - tanh^2 = 4 s(2x) s(-2x), which keeps its digits where tanh is near 1
        two_sided_gates<ACCURATE>(2.0f * x, p, q);
        return 4.0f * p * q;
    }
    const float z = gate_argument<KIND>(x, dz);
    two_sided_gates<ACCURATE>(z, p, q);
    if (KIND == DN_GELU) x = fabsf(x) > 16.0f ? copysignf(16.0f, x) : x;
    return p * fmaf(x * q, dz, 1.0f);
}

template <class T> __global__ void __launch_bounds__(SAVED_THREADS) pack_kernel(int64_t n, const T* src, int int8, uint8_t* packed, bool wide) {
    dep_wait();
    const int64_t first = ((int64_t)blockIdx.x * SAVED_THREADS * UNITS + threadIdx.x) * UNIT;
    float f[UNITS][UNIT];
#pragma unroll
    for (int u = 0; u < UNITS; ++u) load_unit(src, first + (int64_t)u * SAVED_THREADS * UNIT, n, wide, f[u]);
#pragma unroll
    for (int u = 0; u < UNITS; ++u) store_codes(packed, first + (int64_t)u * SAVED_THREADS * UNIT, n, int8, f[u]);
}
template <class T> __global__ void __launch_bounds__(SAVED_THREADS) unpack_kernel(int64_t n, T* dst, int int8, const uint8_t* packed, bool wide) {
    dep_wait();
    const int64_t first = ((int64_t)blockIdx.x * SAVED_THREADS * UNITS + threadIdx.x) * UNIT;
    Codes r[UNITS];
#pragma unroll
    for (int u = 0; u < UNITS; ++u) r[u] = load_codes(packed, first + (int64_t)u * SAVED_THREADS * UNIT, n);
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
        float f[UNIT];
        values_of(r[u], int8, f);
        store_unit(dst, first + (int64_t)u * SAVED_THREADS * UNIT, n, wide, f);
    }
}
template <class T, int KIND>
__global__ void __launch_bounds__(SAVED_THREADS) activation_forward_kernel(int64_t n, const T* x, T* y, int int8, uint8_t* packed, bool wide) {
    dep_wait();
    const int64_t first = ((int64_t)blockIdx.x * SAVED_THREADS * UNITS + threadIdx.x) * UNIT;
    float f[UNITS][UNIT];
#pragma unroll
    for (int u = 0; u < UNITS; ++u) load_unit(x, first + (int64_t)u * SAVED_THREADS * UNIT, n, wide, f[u]);
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
        const int64_t i = first + (int64_t)u * SAVED_THREADS * UNIT;
        if (packed) store_codes(packed, i, n, int8, f[u]);
#pragma unroll
        for (int j = 0; j < UNIT; ++j) f[u][j] = activation<KIND, sizeof(T) == 4>(f[u][j]);
        store_unit(y, i, n, wide, f[u]);
    }
}
template <class T, int KIND>
__global__ void __launch_bounds__(SAVED_THREADS) activation_backward_kernel(int64_t n, const uint8_t* packed, int int8, const T* dy, T* dx, bool wide) {
    dep_wait();
    const int64_t first = ((int64_t)blockIdx.x * SAVED_THREADS * UNITS + threadIdx.x) * UNIT;
    float d[UNITS][UNIT];
    Codes r[UNITS];
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
        load_unit(dy, first + (int64_t)u * SAVED_THREADS * UNIT, n, wide, d[u]);
        r[u] = load_codes(packed, first + (int64_t)u * SAVED_THREADS * UNIT, n);
    }
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
        float f[UNIT];
        values_of(r[u], int8, f);
#pragma unroll
        for (int j = 0; j < UNIT; ++j) d[u][j] *= slope<KIND, sizeof(T) == 4>(f[j]);
        store_unit(dx, first + (int64_t)u * SAVED_THREADS * UNIT, n, wide, d[u]);
    }
}

constexpr int64_t MOST_VALUES = (int64_t)1 << 43;          // blocks of a launch stay below 2^31

dn_status check(int64_t n, int type, int format) {
    if (n < 1 || n > MOST_VALUES) return DN_ERR_SIZE;
    if (type < DN_F32 || type > DN_F16 || (format != DN_INT8 && format != DN_E4M3)) return DN_ERR_MODE;
    return DN_OK;
}
size_t bytes_of(int64_t n, int type) { return (size_t)n * (type == DN_F32 ? 4 : 2); }
bool off(const void* p, int type) { return reinterpret_cast<uintptr_t>(p) % (type == DN_F32 ? 4 : 2) != 0; }
bool off16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 != 0; }
bool meet(const void* a, size_t na, const void* b, size_t nb) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x < y + nb && y < x + na;
}
template <typename... KArgs, typename... Args> dn_status go(void (*kernel)(KArgs...), int64_t n, void* stream, Args... args) {
    const int64_t per = (int64_t)SAVED_THREADS * UNITS * UNIT;
    const cudaError_t e = launch_dependent(kernel, dim3((unsigned)((n + per - 1) / per)), dim3(SAVED_THREADS), 0, static_cast<cudaStream_t>(stream), args...);
    if (e == cudaSuccess) return DN_OK;
    (void)cudaGetLastError();
    return DN_ERR_CUDA;
}
template <class T> dn_status activate(int64_t n, int kind, const void* x, void* y, int int8, void* packed, bool wide, void* stream) {
    auto k = kind == DN_SILU ? activation_forward_kernel<T, DN_SILU> : kind == DN_GELU ? activation_forward_kernel<T, DN_GELU> : activation_forward_kernel<T, DN_TANH>;
    return go(k, n, stream, n, static_cast<const T*>(x), static_cast<T*>(y), int8, static_cast<uint8_t*>(packed), wide);
}
template <class T> dn_status differentiate(int64_t n, int kind, const void* packed, int int8, const void* dy, void* dx, bool wide, void* stream) {
    auto k = kind == DN_SILU ? activation_backward_kernel<T, DN_SILU> : kind == DN_GELU ? activation_backward_kernel<T, DN_GELU> : activation_backward_kernel<T, DN_TANH>;
    return go(k, n, stream, n, static_cast<const uint8_t*>(packed), int8, static_cast<const T*>(dy), static_cast<T*>(dx), wide);
}

}  // namespace
}  // namespace dn

using namespace dn;

#define DN_TRY(x) do { const dn_status st_ = (x); if (st_ != DN_OK) return st_; } while (0)

extern "C" {

size_t dn_packed_bytes(int64_t n) {
    if (n < 1 || n > MOST_VALUES) return 0;
    return (size_t)(scales_at(n) + (n + kBlock8 - 1) / kBlock8);
}

dn_status dn_pack(int64_t n, int32_t type, const void* src, int32_t format, void* packed, void* stream) {
    DN_TRY(check(n, type, format));
    if (!src || !packed) return DN_ERR_NULL;
    if (off(src, type) || off16(packed)) return DN_ERR_LAYOUT;
    if (meet(src, bytes_of(n, type), packed, dn_packed_bytes(n))) return DN_ERR_ALIAS;
    const int int8 = format == DN_INT8;
    const bool wide = !off16(src);
    uint8_t* q = static_cast<uint8_t*>(packed);
    if (type == DN_F32) return go(pack_kernel<float>, n, stream, n, static_cast<const float*>(src), int8, q, wide);
    if (type == DN_BF16) return go(pack_kernel<__nv_bfloat16>, n, stream, n, static_cast<const __nv_bfloat16*>(src), int8, q, wide);
    return go(pack_kernel<__half>, n, stream, n, static_cast<const __half*>(src), int8, q, wide);
}

dn_status dn_unpack(int64_t n, int32_t type, const void* packed, int32_t format, void* dst, void* stream) {
    DN_TRY(check(n, type, format));
    if (!dst || !packed) return DN_ERR_NULL;
    if (off(dst, type) || off16(packed)) return DN_ERR_LAYOUT;
    if (meet(dst, bytes_of(n, type), packed, dn_packed_bytes(n))) return DN_ERR_ALIAS;
    const int int8 = format == DN_INT8;
    const bool wide = !off16(dst);
    const uint8_t* q = static_cast<const uint8_t*>(packed);
    if (type == DN_F32) return go(unpack_kernel<float>, n, stream, n, static_cast<float*>(dst), int8, q, wide);
    if (type == DN_BF16) return go(unpack_kernel<__nv_bfloat16>, n, stream, n, static_cast<__nv_bfloat16*>(dst), int8, q, wide);
    return go(unpack_kernel<__half>, n, stream, n, static_cast<__half*>(dst), int8, q, wide);
}

dn_status dn_activation_forward(int64_t n, int32_t type, int32_t kind, const void* x, void* y, int32_t format, void* packed, void* stream) {
    DN_TRY(check(n, type, format));
    if (kind < DN_SILU || kind > DN_TANH) return DN_ERR_MODE;
    if (!x || !y) return DN_ERR_NULL;
    if (off(x, type) || off(y, type) || off16(packed)) return DN_ERR_LAYOUT;
    const size_t b = bytes_of(n, type), k = packed ? dn_packed_bytes(n) : 0;
    if (meet(x, b, y, b) || meet(x, b, packed, k) || meet(y, b, packed, k)) return DN_ERR_ALIAS;
    const int int8 = format == DN_INT8;
    const bool wide = !off16(x) && !off16(y);
    if (type == DN_F32) return activate<float>(n, kind, x, y, int8, packed, wide, stream);
    if (type == DN_BF16) return activate<__nv_bfloat16>(n, kind, x, y, int8, packed, wide, stream);
    return activate<__half>(n, kind, x, y, int8, packed, wide, stream);
}

dn_status dn_activation_backward(int64_t n, int32_t type, int32_t kind, const void* packed, int32_t format, const void* dy, void* dx, void* stream) {
    DN_TRY(check(n, type, format));
    if (kind < DN_SILU || kind > DN_TANH) return DN_ERR_MODE;
    if (!packed || !dy || !dx) return DN_ERR_NULL;
    if (off(dy, type) || off(dx, type) || off16(packed)) return DN_ERR_LAYOUT;
    const size_t b = bytes_of(n, type), k = dn_packed_bytes(n);
    if ((dx != dy && meet(dx, b, dy, b)) || meet(dx, b, packed, k)) return DN_ERR_ALIAS;
    const int int8 = format == DN_INT8;
    const bool wide = !off16(dy) && !off16(dx);
    if (type == DN_F32) return differentiate<float>(n, kind, packed, int8, dy, dx, wide, stream);
    if (type == DN_BF16) return differentiate<__nv_bfloat16>(n, kind, packed, int8, dy, dx, wide, stream);
    return differentiate<__half>(n, kind, packed, int8, dy, dx, wide, stream);
}

}  // extern "C"
