// Tensors saved in 8 bits, and pointwise activations whose backward pass reads their input in 8 bits.
//
// All four kernels are one pass over memory: a thread takes 8 adjacent values (16 bytes of a 16-bit type, 32 of a 32-bit one, in one
// access), four lanes share a block of 32 and its scale, and UNITS such loads of a thread are in flight at a time.  The activation's
// forward kernel writes y and the packed input from one read of x; its backward kernel reads the packed input and dy and writes dx: 10 bytes
// per element of a 16-bit type for both, 12 with the input kept as it is.
//
// What bounds them: memory in 32 bits (2^25 values: packing 27 us = 95 % of the measured copy rate, reading back 28 us = 91 %, silu and tanh
// 48 + 48 us = 96 %, gelu 48 + 52 us = 97 and 88 %).  In 16 bits the instructions show (how many per
// value, and in how many of the cycles a scheduler issued one):
//   packing  22 us = 72 %   13 instructions, 64 %      reading back  18 us = 84 %    9, 62 %
//   silu     31 us = 84 %   21, 75 %                   backward      36 us = 72 %   20, 61 % (42 warps per SM, 40 registers)
//   gelu     35 us = 74 %   26, 78 %                   backward      44 us = 58 %   27, 64 % (36 warps, 44 registers)
//   tanh     38 us = 68 %   31, 81 % (tanhf)           backward      38 us = 68 %   26, 74 %
// Measured: four units per thread are slower backward (44 us: fewer warps fit), 16-byte stores of 32-bit values 37 us for 29 (every
// sector in two halves), streaming hints on loads and stores no gain.
#include "dn_eight.cuh"

namespace dn {
namespace {

constexpr int SAVED_THREADS = 256, UNIT = 8, UNITS = 2, PAIRS = UNIT / 2;

__host__ __device__ constexpr int64_t scales_at(int64_t n) { return (n + 15) / 16 * 16; }

using Pair = Cols<2>;
template <class T> struct Unit { uint4 w[UNIT * sizeof(T) / 16]; };          // 8 values as they lie in memory

template <class T> __device__ __forceinline__ Unit<T> load_unit(const T* p, int64_t i, int64_t n, int wide) {
    Unit<T> u;
    if (sizeof(T) == 4 && wide == 32 && i + UNIT <= n) {
        constexpr int H = sizeof u / 16 - 1;               // (0, and not reached, for 16-bit types)
        asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
            : "=r"(u.w[0].x), "=r"(u.w[0].y), "=r"(u.w[0].z), "=r"(u.w[0].w), "=r"(u.w[H].x), "=r"(u.w[H].y), "=r"(u.w[H].z), "=r"(u.w[H].w) : "l"(p + i) : "memory");
    } else if (wide && i + UNIT <= n) {
#pragma unroll
        for (int k = 0; k < (int)(UNIT * sizeof(T) / 16); ++k) u.w[k] = reinterpret_cast<const uint4*>(p + i)[k];
    } else {
        T t[UNIT];
#pragma unroll
        for (int j = 0; j < UNIT; ++j) t[j] = i + j < n ? p[i + j] : rounded<T>(0.0f);
        memcpy(&u, t, sizeof u);
    }
    return u;
}
template <class T> __device__ __forceinline__ void values_in(const Unit<T>& u, Pair (&f)[PAIRS]) {
    T t[UNIT];
    memcpy(t, &u, sizeof t);
#pragma unroll
    for (int j = 0; j < PAIRS; ++j) f[j] = Pair{{as_float(t[2 * j]), as_float(t[2 * j + 1])}};
}
template <class T> __device__ __forceinline__ void store_unit(T* p, int64_t i, int64_t n, int wide, const Pair (&f)[PAIRS]) {
    T t[UNIT];
#pragma unroll
    for (int j = 0; j < UNIT; ++j) t[j] = rounded<T>(f[j / 2].v[j % 2]);
    if (wide && i + UNIT <= n) {
        Unit<T> u;
        memcpy(&u, t, sizeof u);
        if (sizeof(T) == 4 && wide == 32) {
            constexpr int H = sizeof u / 16 - 1;
            asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p + i), "r"(u.w[0].x), "r"(u.w[0].y), "r"(u.w[0].z), "r"(u.w[0].w),
                         "r"(u.w[H].x), "r"(u.w[H].y), "r"(u.w[H].z), "r"(u.w[H].w) : "memory");
        } else {
#pragma unroll
            for (int k = 0; k < (int)(UNIT * sizeof(T) / 16); ++k) reinterpret_cast<uint4*>(p + i)[k] = u.w[k];
        }
    } else {
#pragma unroll
        for (int j = 0; j < UNIT; ++j)
            if (i + j < n) p[i + j] = t[j];
    }
}

// The exponent (biased; 255: not finite) of the largest magnitude of a block, from the four lanes that hold it.  Of 16-bit values two
// are compared at a time, as integers without their signs.
template <class T> __device__ __forceinline__ int largest_exponent(const Unit<T>& u) {
    if constexpr (sizeof(T) == 4) {
        unsigned m = 0;
#pragma unroll
        for (int k = 0; k < 2; ++k) m = max(max(m, max(u.w[k].x & 0x7fffffffu, u.w[k].y & 0x7fffffffu)), max(u.w[k].z & 0x7fffffffu, u.w[k].w & 0x7fffffffu));
        m = max(m, __shfl_xor_sync(~0u, m, 1));
        m = max(m, __shfl_xor_sync(~0u, m, 2));
        return (int)(m >> 23);
    } else {
        unsigned m = __vmaxu2(__vmaxu2(u.w[0].x & 0x7fff7fffu, u.w[0].y & 0x7fff7fffu), __vmaxu2(u.w[0].z & 0x7fff7fffu, u.w[0].w & 0x7fff7fffu));
        m = __vmaxu2(m, __shfl_xor_sync(~0u, m, 1));
        m = __vmaxu2(m, __shfl_xor_sync(~0u, m, 2));
        return magnitude_exponent<T>(max(m & 0xffffu, m >> 16));
    }
}

// the codes and the scale of a block, from the four lanes that hold it (each warp calls this as a whole)
template <class T> __device__ __forceinline__ void store_codes(uint8_t* packed, int64_t i, int64_t n, bool int8, const Unit<T>& u, const Pair (&f)[PAIRS]) {
    const int e = largest_exponent(u);
    uint32_t c[2] = {};
    int byte = max(e - (int8 ? 6 : 7), 1);
    if (__any_sync(~0u, e == 255)) {                       // values that are not finite
        unsigned m = 0;
#pragma unroll
        for (int j = 0; j < UNIT; ++j) m = max(m, magnitude_bits(f[j / 2].v[j % 2]));
        m = max(m, __shfl_xor_sync(~0u, m, 1));
        m = max(m, __shfl_xor_sync(~0u, m, 2));
        byte = scale_byte(m, int8);
#pragma unroll
        for (int j = 0; j < UNIT; ++j) c[j / 4] |= code8(f[j / 2].v[j % 2], inverse_scale_of(byte), int8) << (8 * (j % 4));
    } else {
        const float inverse = inverse_scale_of(byte);
        uint32_t k[PAIRS];
        if (int8) {
#pragma unroll
            for (int j = 0; j < PAIRS; ++j) k[j] = codes_int8(f[j], inverse);
        } else {
#pragma unroll
            for (int j = 0; j < PAIRS; ++j) k[j] = codes_e4m3(f[j], inverse);
        }
        c[0] = __byte_perm(k[0], k[1], 0x5410);
        c[1] = __byte_perm(k[2], k[3], 0x5410);
    }
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
        for (int j = 0; j < UNIT; ++j) r.c[j / 4] |= (i + j < n ? (uint32_t)packed[i + j] : 128u) << (8 * (j % 4));
    }
    if (i < n) r.byte = packed[scales_at(n) + i / kBlock8];
    return r;
}
__device__ __forceinline__ void values_of(const Codes& r, bool int8, Pair (&f)[PAIRS]) {
    const float scale = scale_of(r.byte);
    if (int8) {
#pragma unroll
        for (int j = 0; j < PAIRS; ++j) f[j] = values_int8<2>(r.c[j / 2] >> (16 * (j % 2)), scale);
        if (any_zero_byte(r.c[0]) | any_zero_byte(r.c[1])) {
#pragma unroll
            for (int j = 0; j < UNIT; ++j)
                if (((r.c[j / 4] >> (8 * (j % 4))) & 255) == 0) f[j / 2].v[j % 2] = __uint_as_float(0x7fffffffu);
        }
    } else {
#pragma unroll
        for (int j = 0; j < PAIRS; ++j) f[j] = values_e4m3<2>((r.c[j / 2] >> (16 * (j % 2))) & 0xffff, scale);
    }
}

// z of the gate s(z) and dz/dx; beyond |x| = 16 the gate is 0 or 1 to the last bit and x^3 could overflow
__device__ __forceinline__ Pair held16(const Pair& x) {
    Pair t = x;
#pragma unroll
    for (int v = 0; v < 2; ++v)
        if (fabsf(x.v[v]) > 16.0f) t.v[v] = copysignf(16.0f, x.v[v]);
    return t;
}
constexpr float TWO_C = 1.5957691216057308f;               // 2 sqrt(2 / pi)
// s(z) and s(-z) of a pair.  With 16-bit results e^-|z| is the square of an approximate exponential of half the argument: the product is
// also right below the smallest normal number, where z multiplies s(z) back up into the type's range.
template <bool ACCURATE> __device__ __forceinline__ void pair_gates(const Pair& z, Pair& p, Pair& q) {
    if constexpr (ACCURATE) {
#pragma unroll
        for (int v = 0; v < 2; ++v) two_sided_gates<true>(z.v[v], p.v[v], q.v[v]);
    } else {
        const Pair t = mul(z, all_of<2>(0.7213475204444817f));       // log2 e / 2
        Pair e, r;
#pragma unroll
        for (int v = 0; v < 2; ++v) exponential_gate(-fabsf(t.v[v]), e.v[v]);
        e = mul(e, e);
        const Pair d = add(e, all_of<2>(1.0f));
#pragma unroll
        for (int v = 0; v < 2; ++v) reciprocal_gate(d.v[v], r.v[v]);
        const Pair less = mul(e, r);
#pragma unroll
        for (int v = 0; v < 2; ++v) {
            p.v[v] = z.v[v] >= 0.0f ? r.v[v] : less.v[v];
            q.v[v] = z.v[v] >= 0.0f ? less.v[v] : r.v[v];
        }
    }
}
template <int KIND, bool ACCURATE> __device__ __forceinline__ Pair activation(const Pair& x) {
    if constexpr (KIND == DN_TANH) return Pair{{tanhf(x.v[0]), tanhf(x.v[1])}};
    else {
        Pair p, q, z = x;
        if constexpr (KIND == DN_GELU) {
            const Pair t = held16(x);
            z = mul(mul(t, all_of<2>(TWO_C)), fma(mul(t, t), all_of<2>(0.044715f), all_of<2>(1.0f)));
        }
        pair_gates<ACCURATE>(z, p, q);
        return mul(x, p);
    }
}
template <int KIND, bool ACCURATE> __device__ __forceinline__ Pair slope(Pair x) {
    Pair p, q;
    if constexpr (KIND == DN_TANH) {                       // 1 - tanh^2 = 4 s(2x) s(-2x), which keeps its digits where tanh is near 1
#pragma unroll
        for (int v = 0; v < 2; ++v) two_sided_gates<ACCURATE>(2.0f * x.v[v], p.v[v], q.v[v]);
        return mul(mul(p, all_of<2>(4.0f)), q);
    } else if constexpr (KIND == DN_SILU) {
        pair_gates<ACCURATE>(x, p, q);
        return fma(mul(x, q), p, p);
    } else {
        x = held16(x);
        const Pair x2 = mul(x, x);
        const Pair z = mul(mul(x, all_of<2>(TWO_C)), fma(x2, all_of<2>(0.044715f), all_of<2>(1.0f)));
        const Pair dz = fma(x2, all_of<2>(TWO_C * 3.0f * 0.044715f), all_of<2>(TWO_C));
        pair_gates<ACCURATE>(z, p, q);
        return fma(mul(mul(x, q), dz), p, p);
    }
}

template <class T> __global__ void __launch_bounds__(SAVED_THREADS) pack_kernel(int64_t n, const T* src, int int8, uint8_t* packed, int wide) {
    dep_wait();
    const int64_t first = ((int64_t)blockIdx.x * SAVED_THREADS * UNITS + threadIdx.x) * UNIT;
    Unit<T> w[UNITS];
#pragma unroll
    for (int u = 0; u < UNITS; ++u) w[u] = load_unit(src, first + (int64_t)u * SAVED_THREADS * UNIT, n, wide);
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
        Pair f[PAIRS];
        values_in(w[u], f);
        store_codes(packed, first + (int64_t)u * SAVED_THREADS * UNIT, n, int8, w[u], f);
    }
}
template <class T> __global__ void __launch_bounds__(SAVED_THREADS) unpack_kernel(int64_t n, T* dst, int int8, const uint8_t* packed, int wide) {
    dep_wait();
    const int64_t first = ((int64_t)blockIdx.x * SAVED_THREADS * UNITS + threadIdx.x) * UNIT;
    Codes r[UNITS];
#pragma unroll
    for (int u = 0; u < UNITS; ++u) r[u] = load_codes(packed, first + (int64_t)u * SAVED_THREADS * UNIT, n);
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
        Pair f[PAIRS];
        values_of(r[u], int8, f);
        store_unit(dst, first + (int64_t)u * SAVED_THREADS * UNIT, n, wide, f);
    }
}
template <class T, int KIND>
__global__ void __launch_bounds__(SAVED_THREADS) activation_forward_kernel(int64_t n, const T* x, T* y, int int8, uint8_t* packed, int wide) {
    dep_wait();
    const int64_t first = ((int64_t)blockIdx.x * SAVED_THREADS * UNITS + threadIdx.x) * UNIT;
    Unit<T> w[UNITS];
#pragma unroll
    for (int u = 0; u < UNITS; ++u) w[u] = load_unit(x, first + (int64_t)u * SAVED_THREADS * UNIT, n, wide);
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
        const int64_t i = first + (int64_t)u * SAVED_THREADS * UNIT;
        Pair f[PAIRS];
        values_in(w[u], f);
        if (packed) store_codes(packed, i, n, int8, w[u], f);
#pragma unroll
        for (int j = 0; j < PAIRS; ++j) f[j] = activation<KIND, sizeof(T) == 4>(f[j]);
        store_unit(y, i, n, wide, f);
    }
}
template <class T, int KIND>
__global__ void __launch_bounds__(SAVED_THREADS) activation_backward_kernel(int64_t n, const uint8_t* packed, int int8, const T* dy, T* dx, int wide) {
    dep_wait();
    const int64_t first = ((int64_t)blockIdx.x * SAVED_THREADS * UNITS + threadIdx.x) * UNIT;
    Unit<T> w[UNITS];
    Codes r[UNITS];
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
        w[u] = load_unit(dy, first + (int64_t)u * SAVED_THREADS * UNIT, n, wide);
        r[u] = load_codes(packed, first + (int64_t)u * SAVED_THREADS * UNIT, n);
    }
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
        Pair f[PAIRS], d[PAIRS];
        values_of(r[u], int8, f);
        values_in(w[u], d);
#pragma unroll
        for (int j = 0; j < PAIRS; ++j) d[j] = mul(d[j], slope<KIND, sizeof(T) == 4>(f[j]));
        store_unit(dx, first + (int64_t)u * SAVED_THREADS * UNIT, n, wide, d);
    }
}

constexpr int64_t MOST_VALUES = (int64_t)1 << 42;          // blocks of a launch stay below 2^31
static_assert(MOST_VALUES / (SAVED_THREADS * UNITS * UNIT) < 0x7fffffff, "");

dn_status check(int64_t n, int type, int format) {
    if (n < 1 || n > MOST_VALUES) return DN_ERR_SIZE;
    if (type < DN_F32 || type > DN_F16 || (format != DN_INT8 && format != DN_E4M3)) return DN_ERR_MODE;
    return DN_OK;
}
size_t bytes_of(int64_t n, int type) { return (size_t)n * (type == DN_F32 ? 4 : 2); }
bool off(const void* p, int type) { return reinterpret_cast<uintptr_t>(p) % (type == DN_F32 ? 4 : 2) != 0; }
bool off16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 != 0; }
// bytes of an access: 32 (32-bit types), 16, or element by element (0)
int width(const void* a, const void* b) {
    const uintptr_t both = reinterpret_cast<uintptr_t>(a) | reinterpret_cast<uintptr_t>(b);
    return both % 32 == 0 ? 32 : both % 16 == 0 ? 16 : 0;
}
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
template <class T> dn_status activate(int64_t n, int kind, const void* x, void* y, int int8, void* packed, int wide, void* stream) {
    auto k = kind == DN_SILU ? activation_forward_kernel<T, DN_SILU> : kind == DN_GELU ? activation_forward_kernel<T, DN_GELU> : activation_forward_kernel<T, DN_TANH>;
    return go(k, n, stream, n, static_cast<const T*>(x), static_cast<T*>(y), int8, static_cast<uint8_t*>(packed), wide);
}
template <class T> dn_status differentiate(int64_t n, int kind, const void* packed, int int8, const void* dy, void* dx, int wide, void* stream) {
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
    const int wide = width(src, src);
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
    const int wide = width(dst, dst);
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
    const int wide = width(x, y);
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
    const int wide = width(dy, dx);
    if (type == DN_F32) return differentiate<float>(n, kind, packed, int8, dy, dx, wide, stream);
    if (type == DN_BF16) return differentiate<__nv_bfloat16>(n, kind, packed, int8, dy, dx, wide, stream);
    return differentiate<__half>(n, kind, packed, int8, dy, dx, wide, stream);
}

}  // extern "C"
