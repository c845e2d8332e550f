// Storage types of the output-head kernels (4-bit product, sampling,
// distillation): loads and stores of binary32, binary16 and bfloat16 values
// as binary32, one at a time or eight (16 or 32 bytes) at a time.
#pragma once

#include "lrc_device.h"
#include "lrc_internal.h"

namespace lrc {

typedef __bf16 bhalf_t;
typedef __bf16 bhalf2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bhalf8_t __attribute__((ext_vector_type(8)));
typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef unsigned uint4v_t __attribute__((ext_vector_type(4)));
typedef unsigned uint2v_t __attribute__((ext_vector_type(2)));

constexpr float kLog2e = 1.4426950408889634f;

// Conversions round to nearest even; bfloat16 keeps subnormals and NaN.
template <typename T> __device__ __forceinline__ T from_f32(float x) { return (T)x; }

// Element i of an array whose type is known at run time only.
__device__ __forceinline__ float load_as_f32(const void* p, int64_t i, int prec) {
    if (prec == P32) return static_cast<const float*>(p)[i];
    if (prec == P16) return (float)static_cast<const half_t*>(p)[i];
    return (float)static_cast<const bhalf_t*>(p)[i];
}
__device__ __forceinline__ void store_from_f32(void* p, int64_t i, int prec, float v) {
    if (prec == P32) static_cast<float*>(p)[i] = v;
    else if (prec == P16) static_cast<half_t*>(p)[i] = (half_t)v;
    else static_cast<bhalf_t*>(p)[i] = (bhalf_t)v;
}

// 16 bytes of elements from any address that is aligned to the element (one
// wide access; the hardware takes unaligned global addresses).
template <typename T> inline constexpr int kVec = 16 / sizeof(T);
template <typename T> __device__ __forceinline__ uint4v_t load16(const T* p) {
    uint4v_t v;
    __builtin_memcpy(&v, p, 16);
    return v;
}
template <typename T> __device__ __forceinline__ void store16(T* p, uint4v_t v) { __builtin_memcpy(p, &v, 16); }
// The same for data that is not used again soon.
typedef uint4v_t uint4u_t __attribute__((aligned(2)));
template <typename T> __device__ __forceinline__ uint4v_t load16_once(const T* p) {
    return __builtin_nontemporal_load(reinterpret_cast<const uint4u_t*>(p));
}
template <typename T> __device__ __forceinline__ void store16_once(T* p, uint4v_t v) {
    __builtin_nontemporal_store(v, reinterpret_cast<uint4u_t*>(p));
}

// Element e of 16 loaded bytes, widened.
template <typename T> __device__ __forceinline__ float elem(const uint4v_t& v, int e);
template <> __device__ __forceinline__ float elem<float>(const uint4v_t& v, int e) { return __uint_as_float(v[e]); }
template <> __device__ __forceinline__ float elem<bhalf_t>(const uint4v_t& v, int e) {
    return __uint_as_float(e & 1 ? v[e >> 1] & 0xFFFF0000u : v[e >> 1] << 16);
}
template <> __device__ __forceinline__ float elem<half_t>(const uint4v_t& v, int e) {
    const unsigned u = v[e >> 1];   // a copy: a bit cast of a vector's element reads its first one
    const half2_t h = __builtin_bit_cast(half2_t, u);
    return (float)h[e & 1];
}

// -infinity in the storage type T, as bits.
template <typename T> inline constexpr unsigned kNegInfBits = 0xFF800000u;
template <> inline constexpr unsigned kNegInfBits<bhalf_t> = 0xFF80u;
template <> inline constexpr unsigned kNegInfBits<half_t> = 0xFC00u;
template <typename T>
inline constexpr unsigned kNegInfPair = sizeof(T) == 4 ? kNegInfBits<T> : kNegInfBits<T> << 16 | kNegInfBits<T>;
template <typename T> __device__ __forceinline__ void set_bits(uint4v_t& v, int e, unsigned bits) {
    if (sizeof(T) == 4) v[e] = bits;
    else v[e >> 1] = e & 1 ? (v[e >> 1] & 0x0000FFFFu) | bits << 16 : (v[e >> 1] & 0xFFFF0000u) | bits;
}

// The vector at element i of a row of V: -infinity past the row's end.
template <typename T> __device__ __forceinline__ uint4v_t load_row16(const T* row, int64_t i, int64_t V) {
    if (i + kVec<T> <= V) return load16(row + i);
    uint4v_t v = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < kVec<T>; ++e) {
        unsigned b = kNegInfBits<T>;
        if (i + e < V) {
            if constexpr (sizeof(T) == 4) b = __builtin_bit_cast(unsigned, row[i + e]);
            else b = __builtin_bit_cast(unsigned short, row[i + e]);
        }
        set_bits<T>(v, e, b);
    }
    return v;
}

// Two values as storage bits of T in one word (T of 16 bits), rounded to nearest even.
template <typename T> __device__ __forceinline__ unsigned pack2(float a, float b);
template <> __device__ __forceinline__ unsigned pack2<half_t>(float a, float b) {
    return __builtin_bit_cast(unsigned, half2_t{(half_t)a, (half_t)b});
}
template <> __device__ __forceinline__ unsigned pack2<bhalf_t>(float a, float b) {
    return __builtin_bit_cast(unsigned, bhalf2_t{(bhalf_t)a, (bhalf_t)b});
}
template <typename T> __device__ __forceinline__ uint4v_t pack16(const float (&g)[kVec<T>]) {
    uint4v_t v;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        if constexpr (sizeof(T) == 4) v[q] = __float_as_uint(g[q]);
        else v[q] = pack2<T>(g[2 * q], g[2 * q + 1]);
    }
    return v;
}

}  // namespace lrc
