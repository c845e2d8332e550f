// Storage types of the output-head kernels (4-bit product, sampling, distillation,
// norm, adapters, verification): loads and stores of binary32, binary16 and bfloat16
// values as binary32, one at a time or eight (16 or 32 bytes) at a time, and sums and
// maxima over a workgroup.
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

__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) x = __builtin_fmaxf(x, __shfl_xor(x, off, 64));
    return x;
}
// Over the workgroup's NT / 64 waves, in a fixed order; one barrier, so each use
// has a `red` of its own.
template <int NT> __device__ __forceinline__ float block_add(float x, float* red) {
    x = wave_sum(x);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
    __syncthreads();
    float t = 0.0f;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) t += red[w];
    return t;
}
template <int NT> __device__ __forceinline__ float block_max(float x, float* red) {
    x = wave_max(x);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
    __syncthreads();
    float t = -__builtin_inff();
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) t = __builtin_fmaxf(t, red[w]);
    return t;
}

// Keeps the packed form in the registers: without it the widened values of one
// pass over the row are kept for the next (210 against 114 registers).
template <int N> __device__ __forceinline__ void stay(uint4v_t (&v)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) asm volatile("" : "+v"(v[i][q]));
}

// One 16-byte operand a lane: 32 K values of an instruction for 16-bit types, four
// instructions of 4 K values for binary32.
template <typename T> __device__ __forceinline__ float4_t mma16(const uint4v_t& a, const uint4v_t& b, float4_t c);
template <> __device__ __forceinline__ float4_t mma16<half_t>(const uint4v_t& a, const uint4v_t& b, float4_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8_t, a), __builtin_bit_cast(half8_t, b), c, 0, 0, 0);
}
template <> __device__ __forceinline__ float4_t mma16<bhalf_t>(const uint4v_t& a, const uint4v_t& b, float4_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bhalf8_t, a), __builtin_bit_cast(bhalf8_t, b), c, 0, 0, 0);
}
template <> __device__ __forceinline__ float4_t mma16<float>(const uint4v_t& a, const uint4v_t& b, float4_t c) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
        c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[e]), __uint_as_float(b[e]), c, 0, 0, 0);
    return c;
}

// The vector at column c of a row of L, zeros past the end.
template <typename T> __device__ __forceinline__ uint4v_t load_zero16(const T* row, int64_t c, int64_t L) {
    if (c + kVec<T> <= L) return load16(row + c);
    uint4v_t v = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < kVec<T>; ++e)
        if (c + e < L) {
            unsigned b;
            if constexpr (sizeof(T) == 4) b = __builtin_bit_cast(unsigned, row[c + e]);
            else b = __builtin_bit_cast(unsigned short, row[c + e]);
            set_bits<T>(v, e, b);
        }
    return v;
}

// The operand of this lane from a tile in LDS whose rows (pitch `pitch`, 8-byte aligned)
// are the K axis: K values k0 + E (lane / 16) .., column c0 + lane % 16.  The transposing
// read gives lane i of 16 column i of four rows.
template <typename T> __device__ __forceinline__ uint4v_t turned(const T* tile, int pitch, int k0, int c0) {
    const int lr = threadIdx.x & 15, lg = (threadIdx.x & 63) >> 4;
    if constexpr (sizeof(T) == 4) {
        uint4v_t x;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = __float_as_uint(tile[(k0 + 4 * lg + e) * pitch + c0 + lr]);
        return x;
    } else {
        typedef short s4_t __attribute__((ext_vector_type(4)));
        const T* p = tile + (k0 + 8 * lg + (lr >> 2)) * pitch + c0 + 4 * (lr & 3);
        const s4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4_t*)(p));
        const s4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4_t*)(p + 4 * pitch));
        return __builtin_bit_cast(uint4v_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
}

// The power of two that brings a largest magnitude (as bits) to [2^14, 2^15), where
// binary16 pairs are to hold it; 1 for other types, zeros, infinities and NaN.
template <typename T> __device__ __forceinline__ float range_scale(unsigned amax) {
    if constexpr (!__is_same(T, half_t)) return 1.0f;
    if (amax == 0 || amax >= 0x7F800000u) return 1.0f;
    const int e = std::max((int)(amax >> 23), 1) - 127;          // floor(log2), subnormals as 2^-126
    return __uint_as_float((unsigned)(std::min(14 - e, 126) + 127) << 23);
}

}  // namespace lrc
