// 4-bit weights: quantization, and the product with a batch of activations
// plus a rank-k compensation.
//
// Format.  Row i of W is ceil(n / 32) * 16 bytes of E2M1 codes (sign, two
// exponent bits, one mantissa bit: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their
// negatives), the code of column j in nibble j & 1 of byte j / 2, zeros past
// n; scales are m x ceil(n / group).  w_ij = code_ij scale_i,(j / group).  The
// compute units widen a pair of codes to binary16 or bfloat16 exactly in one
// instruction (v_cvt_scalef32_pk_*_fp4).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "head_device.h"

namespace lrc {

// ------------------------------------------------------------ quantization --
// scale = max |w| over the group times the rounded 1/6 (rounded to binary32,
// then to the scale's type); the code is the E2M1 value nearest to w / scale (the quotient rounded
// to binary32, binary64 for binary64 weights), ties to the even code, beyond 6
// saturating.  A group with a NaN or an infinity, or whose scale overflows,
// gets the scale NaN and codes 0.
//
// A lane takes 8 consecutive weights (one 32-bit word of codes), so a group is
// group / 8 neighbouring lanes, and a wave 512 weights of one row.

// code of a finite quotient a >= 0
template <typename Q>
__device__ __forceinline__ unsigned e2m1_of(Q a) {
    return (unsigned)(a > (Q)0.25) + (a >= (Q)0.75) + (a > (Q)1.25) + (a >= (Q)1.75) + (a > (Q)2.5) + (a >= (Q)3.5) +
           (a > (Q)5.0);
}
__device__ __forceinline__ float e2m1_value(unsigned c) {
    // 0, 0.5, then binary32 with the code's exponent and mantissa bits
    const float v = __uint_as_float((c + (126u << 1)) << 22);
    return c < 2 ? 0.5f * (float)c : v;
}

template <typename T> struct QuotientOf { using type = float; };
template <> struct QuotientOf<double> { using type = double; };

template <typename T, bool VEC>
__global__ __launch_bounds__(256) void k_q4_quantize(const T* __restrict__ W, int64_t ldw, int64_t m, int64_t n,
                                                     int lanes, int chunks, unsigned* __restrict__ codes, int64_t wpr,
                                                     void* __restrict__ scales, int64_t G, int sprec,
                                                     T* __restrict__ values, unsigned long long* __restrict__ nbad) {
    using Q = typename QuotientOf<T>::type;
    const int lane = threadIdx.x & 63;
    const int64_t wid = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int64_t i = wid / chunks;
    if (i >= m) return;
    const int64_t word = (wid % chunks) * 64 + lane, j0 = word * 8;
    const T* src = W + i * ldw;
    Q w[8];
    if (VEC && j0 + 8 <= n) {
        typedef T vec_t __attribute__((ext_vector_type(16 / sizeof(T))));
#pragma unroll
        for (int h = 0; h < (int)(8 * sizeof(T) / 16); ++h) {
            const vec_t v = __builtin_nontemporal_load(reinterpret_cast<const vec_t*>(src + j0) + h);
#pragma unroll
            for (int q = 0; q < (int)(16 / sizeof(T)); ++q) w[h * (16 / sizeof(T)) + q] = (Q)v[q];
        }
    } else {
#pragma unroll
        for (int q = 0; q < 8; ++q) w[q] = j0 + q < n ? (Q)src[j0 + q] : (Q)0;
    }
    // NaN and infinity have the largest bits
    Q amax = 0;
    bool bad = false;
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        const Q a = __builtin_elementwise_abs(w[q]);
        bad |= !(a <= (sizeof(Q) == 8 ? (Q)1.7976931348623157e308 : (Q)3.4028234663852886e38f));
        amax = a > amax ? a : amax;
    }
    for (int off = 1; off < lanes; off <<= 1) {
        const Q o = __shfl_xor(amax, off, 64);
        amax = o > amax ? o : amax;
        bad |= (bool)__shfl_xor((int)bad, off, 64);
    }
    float sc = (float)(amax * ((Q)1 / (Q)6));
    if (sprec == P16) sc = (float)(half_t)sc;
    else if (sprec == PB16) sc = (float)(bhalf_t)sc;
    bad |= !(sc <= 3.4028234663852886e38f);
    if (bad) sc = __builtin_nanf("");
    unsigned out = 0;
    Q val[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        const Q a = __builtin_elementwise_abs(w[q]);
        const unsigned c = sc > 0.0f ? e2m1_of<Q>(a / (Q)sc) : 0u;
        const bool neg = sizeof(Q) == 8 ? __double_as_longlong((double)w[q]) < 0 : __float_as_int((float)w[q]) < 0;
        const bool sign = neg && !bad;
        out |= (c | (sign ? 8u : 0u)) << (4 * q);
        const Q v = (Q)e2m1_value(c) * (Q)sc;
        val[q] = sign ? -v : v;
    }
    if (word < wpr) codes[i * wpr + word] = out;
    if (word % lanes == 0 && j0 < n) {
        store_from_f32(scales, i * G + word / lanes, sprec, sc);
        if (bad && nbad) atomicAdd(nbad, 1ull);
    }
    if (values) {
        T* dst = values + i * n;
        if (VEC && j0 + 8 <= n) {
            typedef T vec_t __attribute__((ext_vector_type(16 / sizeof(T))));
#pragma unroll
            for (int h = 0; h < (int)(8 * sizeof(T) / 16); ++h) {
                vec_t v;
#pragma unroll
                for (int q = 0; q < (int)(16 / sizeof(T)); ++q) v[q] = (T)val[h * (16 / sizeof(T)) + q];
                __builtin_nontemporal_store(v, reinterpret_cast<vec_t*>(dst + j0) + h);
            }
        } else {
#pragma unroll
            for (int q = 0; q < 8; ++q)
                if (j0 + q < n) dst[j0 + q] = (T)val[q];
        }
    }
}

static __global__ void k_q4_zero(unsigned long long* p) { *p = 0ull; }

constexpr int64_t kQ4Waves = (int64_t)1 << 25;        // of one launch: 2^31 threads

template <typename T>
static void quantize_t(const void* W, int64_t ldw, int64_t m, int64_t n, int64_t group, void* codes, void* scales,
                       int sprec, void* values, unsigned long long* nbad, hipStream_t st) {
    const int64_t wpr = q4_row_bytes(n) / 4, chunks = (wpr + 63) / 64, G = (n + group - 1) / group;
    const bool vec = reinterpret_cast<uintptr_t>(W) % 16 == 0 && ldw * sizeof(T) % 16 == 0 &&
                     (!values || (reinterpret_cast<uintptr_t>(values) % 16 == 0 && n * sizeof(T) % 16 == 0));
    auto* kern = vec ? k_q4_quantize<T, true> : k_q4_quantize<T, false>;
    (void)in_panels(m, std::max<int64_t>(1, kQ4Waves / chunks), [&](int64_t i, int64_t rows) {
        hipLaunchKernelGGL(kern, dim3((unsigned)((rows * chunks + 3) / 4)), dim3(256), 0, st, (const T*)W + i * ldw, ldw, rows,
                           n, (int)(group / 8), (int)chunks, (unsigned*)codes + i * wpr, wpr,
                           static_cast<char*>(scales) + i * G * elem_bytes(sprec), G, sprec,
                           values ? (T*)values + i * n : nullptr, nbad);
        return hipSuccess;
    });
}

hipError_t launch_q4_quantize(const void* W, int64_t ldw, int prec, int64_t m, int64_t n, int64_t group, void* codes,
                              void* scales, int sprec, void* values, unsigned long long* nbad, hipStream_t st) {
    if (nbad) hipLaunchKernelGGL(k_q4_zero, dim3(1), dim3(1), 0, st, nbad);
    KernelTimer t("q4_quantize", st);
    if (prec == P64) quantize_t<double>(W, ldw, m, n, group, codes, scales, sprec, values, nbad, st);
    else if (prec == P32) quantize_t<float>(W, ldw, m, n, group, codes, scales, sprec, values, nbad, st);
    else if (prec == P16) quantize_t<half_t>(W, ldw, m, n, group, codes, scales, sprec, values, nbad, st);
    else quantize_t<bhalf_t>(W, ldw, m, n, group, codes, scales, sprec, values, nbad, st);
    return hipGetLastError();
}

// ------------------------------------------------------------------ product --
// Y[b][i] = sum_J scale_iJ sum_{j in J} code_ij x_bj + sum_r U_ir T'_br with
// T'_br = s_r sum_j V_jr x_bj.
//
// The codes widen exactly, so the matrix cores form sum code x with exact
// products and FP32 sums, and the scale enters once per group in FP32.  An MFMA
// takes 32 columns; a lane's 16 bytes of codes (32 columns of one row) are
// transposed between the four lanes of that row, so that each MFMA meets 32
// consecutive columns, which lie in one group whatever its size.
// Binary32 activations are the exact sum of three bfloat16 values (8 + 8 + 8
// bits, truncated) and take three MFMAs.  The compensation runs in FP32 on
// v_mfma_f32_16x16x4_f32: T' and the factors are not rounded further.

struct Q4Args {
    const unsigned char* codes;
    const void* scales;
    int64_t rb, G;
    int sprec, gshift;
    const void* U;
    const float* Tm;      // T' [batch][kp], kp = k rounded up to 16, zero past k; or tsplits
    int tsplits;          // partial sums [tsplits][batch][k] without the factor s
    int64_t kp;
    const void* s;
    int64_t k;
    int fprec;
    const void* X;
    int64_t ldx, plane;   // k_q4_tile: 16-bit planes, `plane` elements apart
    void* Y;
    int64_t ldy;
    int yprec;
    int64_t m, n, b;
    float* part;          // k_q4_tile: partial sums [split][batch][m], or null
    int splits;
};

// Activations as MFMA operands: P planes of 8 values.
template <typename T> struct ActTraits;
template <> struct ActTraits<half_t> {
    static constexpr int P = 1;
    using plane_t = half_t;
    using frag = half8_t;
    static __device__ __forceinline__ float4_t mfma(frag a, frag b, float4_t c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
    }
    static __device__ __forceinline__ frag widen(unsigned w) {
        const half2_t p0 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 0);
        const half2_t p1 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 1);
        const half2_t p2 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 2);
        const half2_t p3 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 3);
        return frag{p0[0], p0[1], p1[0], p1[1], p2[0], p2[1], p3[0], p3[1]};
    }
};
template <> struct ActTraits<bhalf_t> {
    static constexpr int P = 1;
    using plane_t = bhalf_t;
    using frag = bhalf8_t;
    static __device__ __forceinline__ float4_t mfma(frag a, frag b, float4_t c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    }
    static __device__ __forceinline__ frag widen(unsigned w) {
        const bhalf2_t p0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 0);
        const bhalf2_t p1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 1);
        const bhalf2_t p2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 2);
        const bhalf2_t p3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 3);
        return frag{p0[0], p0[1], p1[0], p1[1], p2[0], p2[1], p3[0], p3[1]};
    }
};
template <> struct ActTraits<float> : ActTraits<bhalf_t> {
    static constexpr int P = 3;
};

// x = h + m + l exactly, each with 8 significant bits, as bits of bfloat16; an
// infinity keeps its sign in h alone, NaN stays NaN.
__device__ __forceinline__ void split3(float x, unsigned (&p)[3]) {
    const unsigned ux = __float_as_uint(x);
    const bool special = (ux & 0x7F800000u) == 0x7F800000u;
    const float r = special ? 0.0f : x - __uint_as_float(ux & 0xFFFF0000u);
    const unsigned um = __float_as_uint(r);
    p[0] = x != x ? 0x7FC0u : ux >> 16;
    p[1] = um >> 16;
    p[2] = __float_as_uint(r - __uint_as_float(um & 0xFFFF0000u)) >> 16;
}

// The 8 values x[j .. j + 8) of one row of n as MFMA operands; zero past n.
template <typename T>
__device__ __forceinline__ void load_act(const T* x, int64_t j, int64_t n,
                                         typename ActTraits<T>::frag (&f)[ActTraits<T>::P]) {
    uint4v_t v[sizeof(T) / 2];
    if (j + 8 <= n) {
#pragma unroll
        for (int h = 0; h < (int)sizeof(T) / 2; ++h) v[h] = load16(x + j + h * kVec<T>);
    } else {
#pragma unroll
        for (int h = 0; h < (int)sizeof(T) / 2; ++h) {
            v[h] = uint4v_t{0, 0, 0, 0};
#pragma unroll
            for (int e = 0; e < kVec<T>; ++e) {
                const int64_t q = j + h * kVec<T> + e;
                if (q < n) {
                    unsigned b;
                    if constexpr (sizeof(T) == 4) b = __builtin_bit_cast(unsigned, x[q]);
                    else b = __builtin_bit_cast(unsigned short, x[q]);
                    set_bits<T>(v[h], e, b);
                }
            }
        }
    }
    if constexpr (sizeof(T) == 4) {
        uint4v_t o[3];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            unsigned lo[3], hi[3];
            split3(elem<float>(v[q >> 1], 2 * (q & 1)), lo);
            split3(elem<float>(v[q >> 1], 2 * (q & 1) + 1), hi);
#pragma unroll
            for (int t = 0; t < 3; ++t) o[t][q] = lo[t] | hi[t] << 16;
        }
#pragma unroll
        for (int t = 0; t < 3; ++t) f[t] = __builtin_bit_cast(bhalf8_t, o[t]);
    } else {
        f[0] = __builtin_bit_cast(typename ActTraits<T>::frag, v[0]);
    }
}

// Transposes the 4 x 4 words (lane group, register): register t of lane group
// j becomes what register j of lane group t was.
__device__ __forceinline__ void transpose4(unsigned (&w)[4]) {
    auto a = __builtin_amdgcn_permlane16_swap(w[0], w[1], false, false);
    auto b = __builtin_amdgcn_permlane16_swap(w[2], w[3], false, false);
    auto c = __builtin_amdgcn_permlane32_swap(a[0], b[0], false, false);
    auto d = __builtin_amdgcn_permlane32_swap(a[1], b[1], false, false);
    w[0] = c[0];
    w[1] = d[0];
    w[2] = c[1];
    w[3] = d[1];
}

// Four ranks of a row of U (as stored; zero past k) from rank c on, widened by
// the caller: loading and converting apart lets all loads of a step overlap.
__device__ __forceinline__ uint4v_t load_ranks(const Q4Args& a, int64_t row, int64_t c, bool whole) {
    uint4v_t v = {0, 0, 0, 0};
    const int64_t at = row * a.k + c;
    if (a.fprec == P32) {
        const unsigned* u = static_cast<const unsigned*>(a.U) + at;
        if (whole) return load16(u);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (c + e < a.k) v[e] = u[e];
    } else {
        const unsigned short* u = static_cast<const unsigned short*>(a.U) + at;
        if (whole) {
            uint2v_t h;
            __builtin_memcpy(&h, u, 8);
            v[0] = h[0];
            v[1] = h[1];
        } else {
            unsigned w[4] = {0, 0, 0, 0};
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (c + e < a.k) w[e] = u[e];
            v[0] = w[0] | w[1] << 16;
            v[1] = w[2] | w[3] << 16;
        }
    }
    return v;
}

// Adds T' U^T, 16 ranks at a time from rank q0 in steps of `step`, to FA x FB
// result blocks: tm[f] points at T' of this lane's batch row in block f (a pitch
// of whole 16 ranks, zero past k), row[r] is its row of U in block r.
template <int FA, int FB>
__device__ __forceinline__ void add_ranks(const Q4Args& a, const float* const (&tm)[FA], const int64_t (&row)[FB],
                                          int64_t q0, int64_t step, float4_t (&acc)[FB][FA]) {
    const int lg = (threadIdx.x & 63) >> 4;
    for (int64_t q = q0; q < a.k; q += step) {
        const int64_t c = q + lg * 4;
        const bool whole = q + 16 <= a.k;
        uint4v_t ur[FB];
        float4_t tv[FA];
#pragma unroll
        for (int r = 0; r < FB; ++r) ur[r] = load_ranks(a, row[r], c, whole);
#pragma unroll
        for (int f = 0; f < FA; ++f) tv[f] = *reinterpret_cast<const float4_t*>(tm[f] + c);
        float4_t uv[FB];
        if (a.fprec == P32) {
#pragma unroll
            for (int r = 0; r < FB; ++r) uv[r] = __builtin_bit_cast(float4_t, ur[r]);
        } else if (a.fprec == P16) {
#pragma unroll
            for (int r = 0; r < FB; ++r)
#pragma unroll
                for (int e = 0; e < 4; ++e) uv[r][e] = elem<half_t>(ur[r], e);
        } else {
#pragma unroll
            for (int r = 0; r < FB; ++r)
#pragma unroll
                for (int e = 0; e < 4; ++e) uv[r][e] = elem<bhalf_t>(ur[r], e);
        }
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int r = 0; r < FB; ++r)
#pragma unroll
                for (int f = 0; f < FA; ++f) acc[r][f] = mfma(tv[f][t], uv[r][t], acc[r][f]);
    }
}

// Sum of `count` values `step` apart, in order, 16 loads at a time.
__device__ __forceinline__ float sum_splits(const float* from, int count, int64_t step) {
    float t = 0.0f;
    for (int q = 0; q < count; q += 16) {
        float v[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] = q + e < count ? from[(q + e) * step] : 0.0f;
#pragma unroll
        for (int e = 0; e < 16; ++e) t += v[e];
    }
    return t;
}

// ---- few rows: the weights' bytes bound it --------------------------------
// One workgroup of NW waves: 16 RT rows of W for up to 16 rows of X.  The waves
// take steps of 128 columns in turn (so a workgroup streams whole rows) and add
// up through LDS in a fixed order.  Only codes come from memory inside the loop,
// four steps ahead: activations (as 16-bit planes), scales and T' are in LDS, a
// chunk of KC columns (a multiple of 512 NW) at a time.  FL: MFMAs (32 columns)
// per scale group, 4 for groups of 128 and more, whose words need no transpose.
constexpr int kRowsTm = 4096;         // T' values kept in LDS

template <typename T, int RT, int FL, int NW>
__global__ __launch_bounds__(64 * NW) void k_q4_rows(Q4Args a, int KC) {
    using Tr = ActTraits<T>;
    using P16 = typename Tr::plane_t;
    constexpr int P = Tr::P, NT = 64 * NW;
    extern __shared__ uint4v_t lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, lr = lane & 15, lg = lane >> 4;
    const int b = (int)a.b, pitch = KC + 8, GC = KC >> a.gshift;
    P16* xs = reinterpret_cast<P16*>(lds);                                   // [P][b][pitch]
    float* ss = reinterpret_cast<float*>(xs + P * b * pitch);                // [16 RT][GC + 1]
    float* tm = ss + ((16 * RT * (GC + 1) + 3) & ~3);                        // [b][kp]
    const int64_t i0 = (int64_t)blockIdx.x * 16 * RT;
    int64_t row[RT], tok[1] = {std::min(lr, b - 1)};
    const unsigned char* src[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        row[r] = std::min(i0 + 16 * r + lr, a.m - 1);
        src[r] = a.codes + row[r] * a.rb + lg * 16;
    }
    const int64_t blocks = (a.n + 127) / 128;
    uint4v_t w[4][RT];
    auto load = [&](int q, int64_t kb) {
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            w[q][r] = uint4v_t{0, 0, 0, 0};
            if (kb * 64 + lg * 16 < a.rb)
                w[q][r] = __builtin_nontemporal_load(reinterpret_cast<const uint4v_t*>(src[r] + kb * 64));
        }
    };
#pragma unroll
    for (int q = 0; q < 4; ++q) load(q, q * NW + wave);

    auto stage = [&](int64_t j0) {
        for (int e = tid; e < b * (KC / 8); e += NT) {
            const int t = e / (KC / 8), c = e % (KC / 8) * 8;
            typename Tr::frag f[P];
            load_act<T>(static_cast<const T*>(a.X) + t * a.ldx, j0 + c, a.n, f);
#pragma unroll
            for (int p = 0; p < P; ++p) *reinterpret_cast<typename Tr::frag*>(xs + (p * b + t) * pitch + c) = f[p];
        }
        const int64_t g0 = j0 >> a.gshift;
        for (int e = tid; e < 16 * RT * GC; e += NT) {
            const int r = e / GC, g = e % GC;
            ss[r * (GC + 1) + g] =
                g0 + g < a.G ? load_as_f32(a.scales, std::min(i0 + r, a.m - 1) * a.G + g0 + g, a.sprec) : 0.0f;
        }
    };
    stage(0);
    const bool held = a.k > 0 && a.b * a.kp <= kRowsTm;
    if (held)
        for (int e = tid; e < b * (int)a.kp; e += NT) {
            float x = 0.0f;
            if (!a.tsplits) {
                x = a.Tm[e];
            } else {
                const int t = e / (int)a.kp, c = e % (int)a.kp;
                if (c < a.k) {
                    const float* from = a.Tm + t * a.k + c;
                    x = sum_splits(from, a.tsplits, a.b * a.k) * load_as_f32(a.s, c, a.fprec);
                }
            }
            tm[e] = x;
        }
    __syncthreads();

    float4_t acc[RT][1];
#pragma unroll
    for (int r = 0; r < RT; ++r) acc[r][0] = zero_accv<float4_t>();
    const P16* xl = xs + (int)tok[0] * pitch + (FL == 4 ? lg * 32 : lg * 8);
    const float* sl = ss + lr * (GC + 1);
    int64_t c0 = 0;                                     // first step of the chunk
    for (int64_t kb0 = wave; kb0 - wave < blocks; kb0 += 4 * NW) {
        if ((kb0 - wave - c0) * 128 == KC) {
            c0 = kb0 - wave;
            __syncthreads();
            stage(c0 * 128);
            __syncthreads();
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int64_t kb = kb0 + q * NW;
            if (kb < blocks) {
                const int col = (int)(kb - c0) * 128;
                unsigned ww[RT][4];
#pragma unroll
                for (int r = 0; r < RT; ++r) {
#pragma unroll
                    for (int t = 0; t < 4; ++t) ww[r][t] = w[q][r][t];
                    if (FL != 4) transpose4(ww[r]);
                }
                load(q, kb + 4 * NW);
                float4_t d[RT];
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    typename Tr::frag x[P];
#pragma unroll
                    for (int p = 0; p < P; ++p)
                        x[p] = *reinterpret_cast<const typename Tr::frag*>(xl + p * b * pitch + col + (FL == 4 ? t * 8 : t * 32));
#pragma unroll
                    for (int r = 0; r < RT; ++r) {
                        const typename Tr::frag wf = Tr::widen(ww[r][t]);
                        if (t % FL == 0) d[r] = zero_accv<float4_t>();
#pragma unroll
                        for (int p = P - 1; p >= 0; --p) d[r] = Tr::mfma(x[p], wf, d[r]);
                        if (t % FL == FL - 1) {
                            const float sc = sl[16 * r * (GC + 1) + ((col + (t / FL) * 32 * FL) >> a.gshift)];
#pragma unroll
                            for (int v = 0; v < 4; ++v) acc[r][0][v] += sc * d[r][v];
                        }
                    }
                }
            }
        }
    }
    if (a.k) {
        const float* const at[1] = {(held ? tm : a.Tm) + tok[0] * a.kp};
        add_ranks(a, at, row, 16 * wave, 16 * NW, acc);
    }
    __syncthreads();
    float* red = reinterpret_cast<float*>(lds);                              // [NW][16][16 RT + 1]
    constexpr int RP = 16 * RT + 1;
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int v = 0; v < 4; ++v) red[(wave * 16 + 4 * lg + v) * RP + 16 * r + lr] = acc[r][0][v];
    __syncthreads();
    for (int e = tid; e < 16 * RT * b; e += NT) {
        const int i = e % (16 * RT), t = e / (16 * RT);
        if (i0 + i < a.m) {
            float y = red[t * RP + i];
#pragma unroll
            for (int q = 1; q < NW; ++q) y += red[(q * 16 + t) * RP + i];
            store_from_f32(a.Y, t * a.ldy + i0 + i, a.yprec, y);
        }
    }
}

// ---- many rows: tiles --------------------------------------------------------
// One workgroup of WX x WR waves: BM = 16 NR WR rows of W for BT = 16 NX WX rows of
// X, a wave 16 NR x 16 NX results.  Steps of 128 columns
// move codes and activations straight into one of D LDS buffers, D - 1 steps
// ahead.  Rows of X (256 bytes a step) have their 16-byte chunks XOR-swizzled by
// the row on the global side; rows of codes are 64 bytes, a wave's 16 of them one
// contiguous load.  Codes are widened in registers, once for NX MFMAs.  X: 16-bit
// planes, 16-byte aligned rows, zero from n on to the next multiple of 128 (codes
// read past a row's end meet these zeros).
template <typename T, int WX, int NX, int WR> struct TileCfg {
    static constexpr int P = ActTraits<T>::P, NW = WX * WR, NR = WR == 4 && WX == 1 ? 2 : 4;
    static constexpr int BM = 16 * NR * WR, BT = 16 * NX * WX;                   // rows of W and of X
    static constexpr int XB = P * BT * 256, BUF = XB + BM * 64;                  // bytes of a step
    static constexpr int D = BUF <= 20480 ? 4 : BUF <= 24576 || (BUF <= 49152 && NW == 8) ? 3 : 2;
    static constexpr int EU = NW == 8 || D * BUF <= 81920 ? 2 : 1;
    static constexpr int XL = BT / 4 / NW, WL = BM / 16 / NW;                    // loads of a wave in a step
    static constexpr int LOADS = P * XL + WL;
};

// SB: bytes of a scale.  The two 16-bit types are told apart by a mask, without a branch.
template <int SB> __device__ __forceinline__ float scale_of_bits(unsigned u, unsigned bf16_mask) {
    if (SB == 4) return __uint_as_float(u);
    const unsigned short h = (unsigned short)u;
    const unsigned x = __float_as_uint((float)__builtin_bit_cast(half_t, h));
    return __uint_as_float((u << 16 & bf16_mask) | (x & ~bf16_mask));
}

template <typename T, int WX, int NX, int WR, int FL, int SB>
__global__ __launch_bounds__(64 * WX * WR, (TileCfg<T, WX, NX, WR>::EU)) void k_q4_tile(Q4Args a, int tiles_m, int tiles_b) {
    using Tr = ActTraits<T>;
    using C = TileCfg<T, WX, NX, WR>;
    constexpr int P = C::P, NR = C::NR, BT = C::BT, BM = C::BM, D = C::D, XL = C::XL, WL = C::WL;
    __shared__ alignas(16) char S[D * C::BUF];
    const int tid = threadIdx.x, lane = tid & 63, lr = lane & 15, lg = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wx = wave % WX, wr = wave / WX;
    // an XCD's consecutive workgroups take 8 row tiles for one tile of X after another
    const int64_t lt = xcd_tile((int64_t)tiles_m * tiles_b * a.splits);
    if (lt >= (int64_t)tiles_m * tiles_b * a.splits) return;
    const int64_t split = lt / ((int64_t)tiles_m * tiles_b), q = lt % ((int64_t)tiles_m * tiles_b);
    const int64_t g = q / (8 * tiles_b), gs = std::min<int64_t>(8, tiles_m - 8 * g), in = q - g * 8 * tiles_b;
    const int64_t i0 = (8 * g + in % gs) * BM, b0 = in / gs * BT;

    float4_t acc[NR][NX];
#pragma unroll
    for (int r = 0; r < NR; ++r)
#pragma unroll
        for (int f = 0; f < NX; ++f) acc[r][f] = zero_accv<float4_t>();

    const int64_t blocks = (a.n + 127) / 128;
    const int64_t k0 = blocks * split / a.splits, k1 = blocks * (split + 1) / a.splits;
    // a wave moves 4 XL rows of every plane, 4 a load, and 16 WL rows of codes, 16 a load
    const char* xs[XL];
#pragma unroll
    for (int h = 0; h < XL; ++h) {
        const int r = (wave * XL + h) * 4 + lg;
        xs[h] = static_cast<const char*>(a.X) + (std::min(b0 + r, a.b - 1) * a.ldx + ((lr ^ (r & 15)) * 8)) * 2;
    }
    const unsigned char* cs[WL];
#pragma unroll
    for (int h = 0; h < WL; ++h) cs[h] = a.codes + std::min(i0 + (wave * WL + h) * 16 + (lane >> 2), a.m - 1) * a.rb;
    auto move = [&](int64_t kb, int buf) {
        char* to = S + buf * C::BUF;
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int h = 0; h < XL; ++h)
                __builtin_amdgcn_global_load_lds(
                    (const __attribute__((address_space(1))) void*)(xs[h] + p * a.plane * 2 + kb * 256),
                    (__attribute__((address_space(3))) void*)(to + p * BT * 256 + (wave * XL + h) * 1024), 16, 0, 0);
        const int64_t off = std::min(kb * 64 + (lane & 3) * 16, a.rb - 16);
#pragma unroll
        for (int h = 0; h < WL; ++h)
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(cs[h] + off),
                                             (__attribute__((address_space(3))) void*)(to + C::XB + (wave * WL + h) * 1024), 16, 0,
                                             0);
    };
    int64_t srow[NR];                                   // where a row's scales begin
#pragma unroll
    for (int r = 0; r < NR; ++r) srow[r] = std::min(i0 + wr * 16 * NR + 16 * r + lr, a.m - 1) * a.G;
    unsigned sn[NR][4 / FL];
    auto fetch = [&](int64_t kb) {                      // bits only: converting here would wait for the load
        int64_t at[4 / FL];
#pragma unroll
        for (int t = 0; t < 4 / FL; ++t) at[t] = std::min(kb * 128 + t * 32 * FL, a.n - 1) >> a.gshift;
#pragma unroll
        for (int r = 0; r < NR; ++r)
#pragma unroll
            for (int t = 0; t < 4 / FL; ++t)
                sn[r][t] = SB == 4 ? static_cast<const unsigned*>(a.scales)[srow[r] + at[t]]
                                   : static_cast<const unsigned short*>(a.scales)[srow[r] + at[t]];
    };
    const unsigned bf16_mask = a.sprec == PB16 ? ~0u : 0u;
    if (k0 < k1) fetch(k0);
#pragma unroll
    for (int d = 0; d < D - 1; ++d)
        if (k0 + d < k1) move(k0 + d, d);
    // A group's products d join acc with its scale, each block of them one block
    // of products later, the last one in the next step (scale `carry`).
    float4_t d[NR][NX];
#pragma unroll
    for (int f = 0; f < NX; ++f) d[NR - 1][f] = zero_accv<float4_t>();
    float carry = 0.0f;
    auto flush = [&](int r, float scale) {
#pragma unroll
        for (int f = 0; f < NX; ++f)
#pragma unroll
            for (int v = 0; v < 4; ++v) acc[r][f][v] += scale * d[r][f][v];
    };
    int buf = 0;
    for (int64_t kb = k0; kb < k1; ++kb) {
        // this step has landed when no more than the loads of the D - 2 later ones are on their way
        if (kb + D - 2 < k1) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((D - 2) * C::LOADS) : "memory");
        else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        float sc[NR][4 / FL];
#pragma unroll
        for (int r = 0; r < NR; ++r)
#pragma unroll
            for (int t = 0; t < 4 / FL; ++t) sc[r][t] = scale_of_bits<SB>(sn[r][t], bf16_mask);
        if (kb + 1 < k1) fetch(kb + 1);
        if (kb + D - 1 < k1) move(kb + D - 1, buf == 0 ? D - 1 : buf - 1);
        const char* from = S + buf * C::BUF;
        unsigned ww[NR][4];
#pragma unroll
        for (int r = 0; r < NR; ++r) {
            const uint4v_t w = *reinterpret_cast<const uint4v_t*>(from + C::XB + (wr * 16 * NR + 16 * r + lr) * 64 + lg * 16);
#pragma unroll
            for (int t = 0; t < 4; ++t) ww[r][t] = w[t];
            if (FL != 4) transpose4(ww[r]);
        }
        typename Tr::frag x[2][NX][P];
        auto read = [&](int t) {
#pragma unroll
            for (int f = 0; f < NX; ++f) {
                const int r = wx * 16 * NX + 16 * f + lr, ch = (FL == 4 ? lg * 4 + t : t * 4 + lg) ^ (r & 15);
#pragma unroll
                for (int p = 0; p < P; ++p)
                    x[t & 1][f][p] = *reinterpret_cast<const typename Tr::frag*>(from + p * BT * 256 + r * 256 + ch * 16);
            }
        };
        read(0);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            if (t < 3) read(t + 1);
#pragma unroll
            for (int r = 0; r < NR; ++r) {
                const typename Tr::frag wf = Tr::widen(ww[r][t]);
#pragma unroll
                for (int f = 0; f < NX; ++f) {
                    if (t % FL == 0) d[r][f] = zero_accv<float4_t>();
#pragma unroll
                    for (int p = P - 1; p >= 0; --p) d[r][f] = Tr::mfma(x[t & 1][f][p], wf, d[r][f]);
                }
                // the block before this one, whose products are done by now
                if (r == 0 && t % FL == 0) flush(NR - 1, t == 0 ? carry : sc[NR - 1][(t - 1) / FL]);
                if (r > 0 && t % FL == FL - 1) flush(r - 1, sc[r - 1][t / FL]);
            }
        }
        carry = sc[NR - 1][4 / FL - 1];
        buf = buf == D - 1 ? 0 : buf + 1;
    }
    flush(NR - 1, carry);
    if (split == 0 && a.k) {
        int64_t row[NR];
        const float* tm[NX];
#pragma unroll
        for (int r = 0; r < NR; ++r) row[r] = std::min(i0 + wr * 16 * NR + 16 * r + lr, a.m - 1);
#pragma unroll
        for (int f = 0; f < NX; ++f) tm[f] = a.Tm + std::min(b0 + wx * 16 * NX + 16 * f + lr, a.b - 1) * a.kp;
        add_ranks(a, tm, row, 0, 16, acc);
    }
#pragma unroll
    for (int r = 0; r < NR; ++r)
#pragma unroll
        for (int f = 0; f < NX; ++f)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const int64_t i = i0 + wr * 16 * NR + 16 * r + lr, b = b0 + wx * 16 * NX + 16 * f + 4 * lg + v;
                if (i < a.m && b < a.b) {
                    if (a.part) a.part[(split * a.b + b) * a.m + i] = acc[r][f][v];
                    else store_from_f32(a.Y, b * a.ldy + i, a.yprec, acc[r][f][v]);
                }
            }
}

// Y = the sum of the splits, in their order.
__global__ __launch_bounds__(256) void k_q4_join(const float* __restrict__ part, int splits, int64_t m, int64_t b,
                                                 void* __restrict__ Y, int64_t ldy, int yprec) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, t = blockIdx.y;
    if (i >= m) return;
    float y = 0.0f;
    for (int q = 0; q < splits; ++q) y += part[(q * b + t) * m + i];
    store_from_f32(Y, t * ldy + i, yprec, y);
}

// Activations as 16-bit planes of padded rows (pitch ldp, zero from n on).
template <typename T>
__global__ __launch_bounds__(256) void k_q4_pack(const T* __restrict__ X, int64_t ldx, int64_t n, int64_t b,
                                                 unsigned short* __restrict__ out, int64_t ldp) {
    const int64_t per = ldp / 8, step = (int64_t)gridDim.x * 256;
    for (int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x; c < b * per; c += step) {
        typename ActTraits<T>::frag f[ActTraits<T>::P];
        load_act<T>(X + c / per * ldx, c % per * 8, n, f);
#pragma unroll
        for (int p = 0; p < ActTraits<T>::P; ++p)
            *reinterpret_cast<typename ActTraits<T>::frag*>(out + p * b * ldp + c * 8) = f[p];
    }
}

// ---- T' = diag(s) V^T x -----------------------------------------------------
// Partial sums of V^T x over a range of columns: part[split][batch][k].  A
// workgroup of 4 waves takes 16 TW batch rows and up to 16 F ranks; steps of 128
// rows of V go through LDS in binary32 (as they lie in memory when the tile holds
// all ranks: no index arithmetic per value).  TW = 4: a wave per 16 batch rows;
// TW = 1: the waves share the columns and add up in order.
template <typename T, int F, int TW>
__global__ __launch_bounds__(256) void k_q4_mid(const T* __restrict__ X, int64_t ldx, const void* __restrict__ V,
                                                int fprec, int64_t n, int64_t k, int64_t b, int64_t chunk,
                                                float* __restrict__ part) {
    extern __shared__ float lv[];
    const int tid = threadIdx.x, lane = tid & 63, lr = lane & 15, lg = lane >> 4, wave = tid >> 6;
    const int64_t r0 = (int64_t)blockIdx.x * 16 * F, s = blockIdx.y, b0 = (int64_t)blockIdx.z * 16 * TW;
    const int w = (int)std::min<int64_t>(k - r0, 16 * F);
    const int64_t j0 = s * chunk, j1 = std::min(n, j0 + chunk);
    const T* x = X + std::min(b0 + (TW == 4 ? 16 * wave : 0) + lr, b - 1) * ldx;
    float4_t acc[F];
#pragma unroll
    for (int f = 0; f < F; ++f) acc[f] = zero_accv<float4_t>();
    for (int64_t j = j0; j < j1; j += 128) {
        const int rows = (int)std::min<int64_t>(128, j1 - j);
        __syncthreads();
        if (w == k) {
            const int64_t at = j * k;
            const int count = rows * w;
            if (fprec == P32) {
                for (int e = tid; e < 128 * w; e += 256) lv[e] = e < count ? static_cast<const float*>(V)[at + e] : 0.0f;
            } else {
                const unsigned short* src = static_cast<const unsigned short*>(V) + at;
                for (int e = tid * 8; e < 128 * w; e += 2048) {
                    if (e + 8 <= count) {
                        const uint4v_t v = load16(src + e);
#pragma unroll
                        for (int h = 0; h < 8; ++h) lv[e + h] = fprec == P16 ? elem<half_t>(v, h) : elem<bhalf_t>(v, h);
                    } else {
#pragma unroll
                        for (int h = 0; h < 8; ++h)
                            if (e + h < 128 * w) lv[e + h] = e + h < count ? load_as_f32(V, at + e + h, fprec) : 0.0f;
                    }
                }
            }
        } else {
            for (int e = tid; e < 128 * 16 * F; e += 256) {
                const int c = e % (16 * F), r = e / (16 * F);
                if (c < w) lv[r * w + c] = r < rows ? load_as_f32(V, (j + r) * k + r0 + c, fprec) : 0.0f;
            }
        }
        __syncthreads();
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            const int hh = TW == 4 ? h : wave;
            if (TW == 4 || h == 0) {
                const int64_t c = j + hh * 32 + lg * 8;
                float xv[8];
                if (c + 8 <= j1) {
#pragma unroll
                    for (int q = 0; q < (int)sizeof(T) / 2; ++q) {
                        const uint4v_t v = load16(x + c + q * kVec<T>);
#pragma unroll
                        for (int e = 0; e < kVec<T>; ++e) xv[q * kVec<T> + e] = elem<T>(v, e);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) xv[e] = c + e < j1 ? (float)x[c + e] : 0.0f;
                }
#pragma unroll
                for (int e = 0; e < 8; ++e)
#pragma unroll
                    for (int f = 0; f < F; ++f) {
                        const int r = 16 * f + lr;
                        acc[f] = mfma(xv[e], r < w ? lv[(hh * 32 + lg * 8 + e) * w + r] : 0.0f, acc[f]);
                    }
            }
        }
    }
    if (TW == 4) {
#pragma unroll
        for (int f = 0; f < F; ++f)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const int64_t bb = b0 + 16 * wave + 4 * lg + v, r = 16 * f + lr;
                if (bb < b && r < w) part[(s * b + bb) * k + r0 + r] = acc[f][v];
            }
    } else {
        __syncthreads();
#pragma unroll
        for (int f = 0; f < F; ++f)
#pragma unroll
            for (int v = 0; v < 4; ++v) lv[(wave * 16 + 4 * lg + v) * 16 * F + 16 * f + lr] = acc[f][v];
        __syncthreads();
        for (int e = tid; e < 256 * F; e += 256) {
            const int r = e % (16 * F), t = e / (16 * F);
            float y = lv[t * 16 * F + r];
#pragma unroll
            for (int q = 1; q < 4; ++q) y += lv[(q * 16 + t) * 16 * F + r];
            if (b0 + t < b && r < w) part[(s * b + b0 + t) * k + r0 + r] = y;
        }
    }
}

// The same for 16-bit activations and factors, on the 16-bit matrix cores with
// exact products: both binary16, or bfloat16 with the one of the two that is
// binary16 as the sum of two bfloat16 values (8 + 3 bits; an infinity of the other
// meets the first alone, as the second may be 0).  Steps of 128 rows of V
// lie transposed in LDS ([rank][column], PV planes).  FV: V is binary16.
// 4096 rows of 8192, k = 65: 53 us, k_q4_mid 86.
template <typename T, bool FV, int F, int TW>
__global__ __launch_bounds__(256) void k_q4_mid16(const T* __restrict__ X, int64_t ldx,
                                                  const unsigned short* __restrict__ V, int64_t n, int64_t k, int64_t b,
                                                  int64_t chunk, float* __restrict__ part) {
    constexpr bool XH = std::is_same_v<T, half_t>;
    constexpr bool HALF = XH && FV;                       // else bfloat16 products
    constexpr int PX = XH && !FV ? 2 : 1, PV = !XH && FV ? 2 : 1, PITCH = 136;
    using M = ActTraits<std::conditional_t<HALF, half_t, bhalf_t>>;
    using frag = typename M::frag;
    extern __shared__ uint4v_t lds16[];
    unsigned short* lv = reinterpret_cast<unsigned short*>(lds16);                // [PV][16 F][PITCH]
    const int tid = threadIdx.x, lane = tid & 63, lr = lane & 15, lg = lane >> 4, wave = tid >> 6;
    const int64_t r0 = (int64_t)blockIdx.x * 16 * F, s = blockIdx.y, b0 = (int64_t)blockIdx.z * 16 * TW;
    const int w = (int)std::min<int64_t>(k - r0, 16 * F);
    const int64_t j0 = s * chunk, j1 = std::min(n, j0 + chunk);
    const T* x = X + std::min(b0 + (TW == 4 ? 16 * wave : 0) + lr, b - 1) * ldx;
    // x for the low plane of V: infinities and NaN, which the high plane takes, as 0
    auto finite = [](frag f) {
        uint4v_t v = __builtin_bit_cast(uint4v_t, f);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const unsigned top = ((v[q] & 0x7F807F80u) + 0x00800080u) & 0x80008000u;    // a bit per special half
            v[q] &= ~((top << 1) - (top >> 15));
        }
        return __builtin_bit_cast(frag, v);
    };
    auto put = [&](int r, int j, unsigned h) {
        if (PV == 1) {
            lv[r * PITCH + j] = (unsigned short)h;
        } else {
            const unsigned short hh = (unsigned short)h;
            const float f = (float)__builtin_bit_cast(half_t, hh);
            const unsigned u = __float_as_uint(f);
            const bool special = (u & 0x7F800000u) == 0x7F800000u;
            const float lo = special ? 0.0f : f - __uint_as_float(u & 0xFFFF0000u);
            lv[r * PITCH + j] = (unsigned short)(f != f ? 0x7FC0u : u >> 16);
            lv[(16 * F + r) * PITCH + j] = (unsigned short)(__float_as_uint(lo) >> 16);
        }
    };
    float4_t acc[F];
#pragma unroll
    for (int f = 0; f < F; ++f) acc[f] = zero_accv<float4_t>();
    for (int64_t j = j0; j < j1; j += 128) {
        const int rows = (int)std::min<int64_t>(128, j1 - j);
        frag xa[TW == 4 ? 4 : 1][PX];
#pragma unroll
        for (int h = 0; h < (TW == 4 ? 4 : 1); ++h) {
            typename ActTraits<T>::frag raw[1];
            load_act<T>(x, j + (TW == 4 ? h : wave) * 32 + lg * 8, j1, raw);
            if constexpr (PX == 1) {
                xa[h][0] = __builtin_bit_cast(frag, raw[0]);
            } else {
                const uint4v_t v = __builtin_bit_cast(uint4v_t, raw[0]);
                uint4v_t hi, lo;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    unsigned p[2][3];
                    split3(elem<half_t>(v, 2 * q), p[0]);
                    split3(elem<half_t>(v, 2 * q + 1), p[1]);
                    hi[q] = p[0][0] | p[1][0] << 16;
                    lo[q] = p[0][1] | p[1][1] << 16;
                }
                xa[h][0] = __builtin_bit_cast(frag, hi);
                xa[h][PX - 1] = __builtin_bit_cast(frag, lo);
            }
        }
        __syncthreads();
        if (rows < 128) {                                 // columns past the end meet zeros of x: no NaN here
            for (int e = tid; e < PV * 16 * F * PITCH / 8; e += 256) lds16[e] = uint4v_t{0, 0, 0, 0};
            __syncthreads();
        }
        if (w == k) {
            const unsigned short* src = V + j * k;
            const int count = rows * w;
#pragma unroll 2
            for (int e = tid * 8; e < count; e += 2048) {
                uint4v_t v = {0, 0, 0, 0};
                if (e + 8 <= count) {
                    v = load16(src + e);
                } else {
#pragma unroll
                    for (int h = 0; h < 8; ++h)
                        if (e + h < count) set_bits<half_t>(v, h, src[e + h]);
                }
                int jj = e / w, r = e % w;
#pragma unroll
                for (int h = 0; h < 8; ++h) {
                    if (e + h < count) put(r, jj, h & 1 ? v[h >> 1] >> 16 : v[h >> 1] & 0xFFFFu);
                    if (++r == w) {
                        r = 0;
                        ++jj;
                    }
                }
            }
        } else {
            for (int e = tid; e < rows * 16 * F; e += 256) {
                const int r = e % (16 * F), jj = e / (16 * F);
                if (r < w) put(r, jj, V[(j + jj) * k + r0 + r]);
            }
        }
        __syncthreads();
#pragma unroll
        for (int h = 0; h < (TW == 4 ? 4 : 1); ++h) {
            const frag xl = PV == 2 ? finite(xa[h][0]) : xa[h][0];
#pragma unroll
            for (int f = 0; f < F; ++f) {
                const int at = (16 * f + lr) * PITCH + (TW == 4 ? h : wave) * 32 + lg * 8;
                if constexpr (PV == 2)
                    acc[f] = M::mfma(xl, *reinterpret_cast<const frag*>(lv + 16 * F * PITCH + at), acc[f]);
                const frag vf = *reinterpret_cast<const frag*>(lv + at);
#pragma unroll
                for (int p = PX - 1; p >= 0; --p) acc[f] = M::mfma(xa[h][p], vf, acc[f]);
            }
        }
    }
    if (TW == 4) {
#pragma unroll
        for (int f = 0; f < F; ++f)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const int64_t bb = b0 + 16 * wave + 4 * lg + v;
                const int r = 16 * f + lr;
                if (bb < b && r < w) part[(s * b + bb) * k + r0 + r] = acc[f][v];
            }
    } else {
        float* red = reinterpret_cast<float*>(lds16);     // [4][16][16 F]
        __syncthreads();
#pragma unroll
        for (int f = 0; f < F; ++f)
#pragma unroll
            for (int v = 0; v < 4; ++v) red[(wave * 16 + 4 * lg + v) * 16 * F + 16 * f + lr] = acc[f][v];
        __syncthreads();
        for (int e = tid; e < 256 * F; e += 256) {
            const int r = e % (16 * F), t = e / (16 * F);
            float y = red[t * 16 * F + r];
#pragma unroll
            for (int q = 1; q < 4; ++q) y += red[(q * 16 + t) * 16 * F + r];
            if (b0 + t < b && r < w) part[(s * b + b0 + t) * k + r0 + r] = y;
        }
    }
}

// T'[b][r] = s_r times the sum of the partials, in split order; rows of kp, zero
// past k.
__global__ __launch_bounds__(256) void k_q4_mid_finish(const float* __restrict__ part, int splits,
                                                       const void* __restrict__ s, int fprec, int64_t k, int64_t kp,
                                                       int64_t b, float* __restrict__ Tm) {
    const int64_t step = (int64_t)gridDim.x * 256;
    for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < b * kp; e += step) {
        const int64_t r = e % kp;
        float t = 0.0f;
        if (r < k) t = sum_splits(part + e / kp * k + r, splits, b * k) * load_as_f32(s, r, fprec);
        Tm[e] = t;
    }
}

// ------------------------------------------------------------------ plan --
namespace {

// Workgroups of the strided kernels above for `items`, one a thread up to 2^24.
unsigned strided_grid(int64_t items) { return (unsigned)std::min<int64_t>((items + 255) / 256, 65536); }

struct Q4Plan {
    bool tile;            // k_q4_tile, else k_q4_rows
    int wx, nx, wr;       // tile: waves along X, 16-row blocks of X per wave, waves along W
    int splits;           // tile: parts of the columns
    bool pack;            // tile: activations copied to padded planes
    int64_t ldp;
    int kc, nw, rt;       // rows: columns in LDS at a time, waves, row blocks per wave
    size_t lds;
    int mid_splits, mid_tw;
    int64_t mid_chunk;
    bool mid_finish;      // T' finished by a kernel of its own
    size_t tm, mid_part, planes, part;
};

// 8192 x 8192 bfloat16, a call with k = 65: 8 rows 29.5 us here, 34.6 on the tiles;
// 9 rows 36.9 against 34.6, 16 rows 42.9 against 35.1.  k = 0: 8 rows 14.6 against
// 15.1, 9 rows 21.7 against 15.1.
constexpr int64_t kRowsMax = 8;
// k_q4_rows for few rows whose activations leave room in LDS: false when
// the tile kernel is to be taken.
bool plan_rows(Q4Plan& p, const Q4Weights& w, int64_t b, int prec) {
    if (b > kRowsMax) return false;
    const int64_t planes = prec == P32 ? 3 : 1, tiles = (w.m + 15) / 16;
    p.rt = tiles >= 1024 ? 2 : 1;
    p.nw = tiles <= 512 && b * planes <= 8 ? 8 : 4;
    // 64 KB of activations, and no more than the columns there are
    const int64_t unit = 512 * p.nw, most = std::min<int64_t>(65536 / (2 * b * planes), 8192) / unit * unit;
    if (most < unit) return false;
    p.kc = (int)std::min<int64_t>(most, round_up(w.n, unit));
    const size_t x = (size_t)planes * b * (p.kc + 8) * 2, s = (size_t)16 * p.rt * (p.kc / w.group + 1) * 4;
    const int64_t kp = round_up(w.k, 16);
    const size_t t = w.k && b * kp <= kRowsTm ? (size_t)b * kp * 4 + 16 : 0;
    p.lds = std::max(x + s + t, (size_t)p.nw * 16 * (16 * p.rt + 1) * 4);
    return true;
}

Q4Plan plan_q4(const Q4Weights& w, const void* X, int64_t ldx, int64_t b, int prec) {
    Q4Plan p{};
    const int64_t blocks = (w.n + 127) / 128;
    p.tile = !plan_rows(p, w, b, prec);
    if (p.tile) {
        p.wx = prec == P32 || b <= 64 ? 1 : 2;
        p.nx = b <= 16 ? 1 : b <= 32 ? 2 : 4;
        p.wr = p.wx == 1 ? 4 : 2;
        if (p.wx == 2 && (w.m + 255) / 256 * ((b + 127) / 128) >= 256) p.wr = 4;
        const int64_t tiles = (w.m + 127) / 128 * ((b + 16 * p.nx * p.wx - 1) / (16 * p.nx * p.wx));
        p.splits = (int)std::min<int64_t>(std::max<int64_t>(1, 512 / tiles), std::max<int64_t>(1, blocks / 4));
        const int e = elem_bytes(prec);
        p.ldp = blocks * 128;
        p.pack = prec == P32 || w.n % 128 || reinterpret_cast<uintptr_t>(X) % 16 || ldx * e % 16;
        if (p.pack) p.planes = (size_t)(prec == P32 ? 3 : 1) * b * p.ldp * 2;
        if (p.splits > 1) p.part = (size_t)p.splits * b * w.m * 4;
    }
    if (w.k) {
        const int64_t kp = round_up(w.k, 16);
        p.mid_tw = b <= 16 ? 1 : 4;
        const int64_t groups = (w.k + 127) / 128 * ((b + 16 * p.mid_tw - 1) / (16 * p.mid_tw));
        // enough workgroups for the chip, few partials for their readers (one row of
        // 8192 columns, k = 65: 64 parts 6.4 us, 32 parts 9.5, their reader 1 us longer)
        int64_t s = std::min<int64_t>(blocks, std::max<int64_t>(1, 512 / groups));
        s = std::min<int64_t>(s, b == 1 ? 64 : b <= 16 ? 32 : 64);
        p.mid_chunk = (blocks + s - 1) / s * 128;
        p.mid_splits = (int)((w.n + p.mid_chunk - 1) / p.mid_chunk);
        p.mid_finish = p.tile || b * p.mid_splits > 64 || b * kp > kRowsTm;
        p.mid_part = (size_t)p.mid_splits * b * w.k * 4;
        if (p.mid_finish) p.tm = (size_t)b * kp * 4;
    }
    return p;
}

size_t plan_bytes(const Q4Plan& p) {
    auto r = [](size_t x) { return (size_t)round_up((int64_t)x, 256); };
    return r(p.tm) + r(p.mid_part) + r(p.planes) + r(p.part);
}

template <typename T, int RT, int FL, int NW>
hipError_t launch_rows(const Q4Plan& p, const Q4Args& a, hipStream_t st) {
    auto* kern = k_q4_rows<T, RT, FL, NW>;
    if (p.lds > 65536) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kern),
                                                 hipFuncAttributeMaxDynamicSharedMemorySize, (int)p.lds);
        if (e != hipSuccess) return e;
    }
    KernelTimer t("q4_rows", st);
    hipLaunchKernelGGL(kern, dim3((unsigned)((a.m + 16 * RT - 1) / (16 * RT))), dim3(64 * NW), p.lds, st, a, p.kc);
    return hipGetLastError();
}
template <typename T, int FL>
hipError_t rows_t(const Q4Plan& p, const Q4Args& a, hipStream_t st) {
    if (p.rt == 2) return launch_rows<T, 2, FL, 4>(p, a, st);
    return p.nw == 8 ? launch_rows<T, 1, FL, 8>(p, a, st) : launch_rows<T, 1, FL, 4>(p, a, st);
}

template <typename T, int WX, int NX, int WR, int FL, int SB>
void launch_tile(const Q4Args& a, hipStream_t st) {
    using C = TileCfg<T, WX, NX, WR>;
    const int tm = (int)((a.m + C::BM - 1) / C::BM), tb = (int)((a.b + C::BT - 1) / C::BT);
    KernelTimer t("q4_tile", st);
    hipLaunchKernelGGL((k_q4_tile<T, WX, NX, WR, FL, SB>), dim3(xcd_grid((int64_t)tm * tb * a.splits)),
                       dim3(64 * C::NW), 0, st, a, tm, tb);
}
template <typename T, int FL, int SB>
void tile_sb(const Q4Plan& p, const Q4Args& a, hipStream_t st) {
    if constexpr (sizeof(T) == 2) {
        if (p.wx == 2 && p.wr == 4) return launch_tile<T, 2, 4, 4, FL, SB>(a, st);
        if (p.wx == 2) return launch_tile<T, 2, 4, 2, FL, SB>(a, st);
    }
    if (p.nx == 1) return launch_tile<T, 1, 1, 4, FL, SB>(a, st);
    if (p.nx == 2) return launch_tile<T, 1, 2, 4, FL, SB>(a, st);
    launch_tile<T, 1, 4, 4, FL, SB>(a, st);
}
template <typename T, int FL>
void tile_t(const Q4Plan& p, const Q4Args& a, hipStream_t st) {
    if (a.sprec == P32) tile_sb<T, FL, 4>(p, a, st);
    else tile_sb<T, FL, 2>(p, a, st);
}

template <typename T, int F>
void mid_f(const Q4Plan& p, const Q4Weights& w, const Q4Args& a, float* part, hipStream_t st) {
    KernelTimer t("q4_mid", st);
    const dim3 grid((unsigned)((w.k + 16 * F - 1) / (16 * F)), p.mid_splits,
                    (unsigned)((a.b + 16 * p.mid_tw - 1) / (16 * p.mid_tw)));
    const T* x = static_cast<const T*>(a.X);
    const size_t red = (size_t)4 * 16 * 16 * F * 4;
    if constexpr (sizeof(T) == 2) {
        if (w.fprec != P32) {
            const bool fv = w.fprec == P16;
            const size_t lds = std::max<size_t>((size_t)(fv && !std::is_same_v<T, half_t> ? 2 : 1) * 16 * F * 136 * 2, red);
            auto* kern = p.mid_tw == 4 ? (fv ? k_q4_mid16<T, true, F, 4> : k_q4_mid16<T, false, F, 4>)
                                       : (fv ? k_q4_mid16<T, true, F, 1> : k_q4_mid16<T, false, F, 1>);
            hipLaunchKernelGGL(kern, grid, dim3(256), lds, st, x, a.ldx, static_cast<const unsigned short*>(w.V), w.n, w.k,
                               a.b, p.mid_chunk, part);
            return;
        }
    }
    const int64_t wide = std::min<int64_t>(w.k, 16 * F);
    const size_t lds = std::max<size_t>((size_t)128 * wide * 4, red);
    auto* kern = p.mid_tw == 4 ? k_q4_mid<T, F, 4> : k_q4_mid<T, F, 1>;
    hipLaunchKernelGGL(kern, grid, dim3(256), lds, st, x, a.ldx, w.V, w.fprec, w.n, w.k, a.b, p.mid_chunk, part);
}

template <typename T>
hipError_t apply_t(const Q4Weights& w, Q4Args& a, int prec, Workspace& ws, hipStream_t st) {
    const Q4Plan p = plan_q4(w, a.X, a.ldx, a.b, prec);
    float* Tm = static_cast<float*>(ws.take(p.tm));
    float* mid = static_cast<float*>(ws.take(p.mid_part));
    unsigned short* planes = static_cast<unsigned short*>(ws.take(p.planes));
    a.part = static_cast<float*>(ws.take(p.part));
    if (ws.overrun) return hipErrorOutOfMemory;
    if (w.k) {
        if (w.k <= 32) mid_f<T, 2>(p, w, a, mid, st);
        else if (w.k <= 80) mid_f<T, 5>(p, w, a, mid, st);
        else mid_f<T, 8>(p, w, a, mid, st);
        if (p.mid_finish) {
            KernelTimer t("q4_mid_finish", st);
            hipLaunchKernelGGL(k_q4_mid_finish, dim3(strided_grid(a.b * a.kp)), dim3(256), 0, st, mid,
                               p.mid_splits, w.s, w.fprec, w.k, a.kp, a.b, Tm);
            a.Tm = Tm;
        } else {
            a.Tm = mid;
            a.tsplits = p.mid_splits;
        }
    }
    if (!p.tile) {
        if (a.gshift == 5) return rows_t<T, 1>(p, a, st);
        if (a.gshift == 6) return rows_t<T, 2>(p, a, st);
        return rows_t<T, 4>(p, a, st);
    }
    a.splits = p.splits;
    if (p.pack) {
        KernelTimer t("q4_pack", st);
        hipLaunchKernelGGL(k_q4_pack<T>, dim3(strided_grid(a.b * (p.ldp / 8))), dim3(256), 0, st,
                           static_cast<const T*>(a.X), a.ldx, w.n, a.b, planes, p.ldp);
        a.X = planes;
        a.ldx = p.ldp;
        a.plane = a.b * p.ldp;
    }
    if (a.gshift == 5) tile_t<T, 1>(p, a, st);
    else if (a.gshift == 6) tile_t<T, 2>(p, a, st);
    else tile_t<T, 4>(p, a, st);
    if (p.splits > 1) {
        KernelTimer t("q4_join", st);
        hipLaunchKernelGGL(k_q4_join, dim3((unsigned)((w.m + 255) / 256), (unsigned)a.b), dim3(256), 0, st, a.part, p.splits,
                           w.m, a.b, a.Y, a.ldy, a.yprec);
    }
    return hipGetLastError();
}

}  // namespace

// Larger calls run in panels of X (the grids' third dimension ends at 2^16) and of W
// (the tiles' grids: a thread for 32 outputs or more, for 8 or 16 in batches up to 32;
// the row kernel's: 8 threads a row of W; so at most 2^31 and a half).
constexpr int64_t kQ4Panel = 1 << 20;
int64_t weight_panel(int64_t batch) { return std::min<int64_t>(1 << 28, ((int64_t)1 << 36) / batch); }

size_t q4_apply_workspace_bytes(const Q4Weights& w, const void* X, int64_t ldx, int64_t batch, int prec) {
    size_t bytes = 0;
    auto panel = [&](int64_t m, int64_t b) {
        Q4Weights part = w;
        part.m = m;
        if (m && b) bytes = std::max(bytes, plan_bytes(plan_q4(part, X, ldx, b, prec)));
    };
    const int64_t b = std::min(batch, kQ4Panel), m = std::min(w.m, weight_panel(b));
    for (int64_t rows : {b, batch % b}) {
        panel(m, rows);
        panel(w.m % m, rows);
    }
    return bytes;
}

hipError_t launch_q4_apply(const Q4Weights& w, const void* X, int64_t ldx, void* Y, int64_t ldy, int64_t batch,
                           int prec, int yprec, Workspace& ws, hipStream_t st) {
    const int64_t rb = q4_row_bytes(w.n), G = (w.n + w.group - 1) / w.group;
    auto panel = [&](int64_t i0, int64_t rows, int64_t b0, int64_t b) {
        Q4Weights part = w;
        part.m = rows;
        Q4Args a{};
        a.codes = static_cast<const unsigned char*>(w.codes) + i0 * rb;
        a.scales = static_cast<const char*>(w.scales) + i0 * G * elem_bytes(w.sprec);
        a.rb = rb;
        a.G = G;
        a.sprec = w.sprec;
        a.gshift = __builtin_ctzll((unsigned long long)w.group);
        a.U = w.k ? static_cast<const char*>(w.U) + i0 * w.k * elem_bytes(w.fprec) : nullptr;
        a.s = w.s;
        a.k = w.k;
        a.kp = round_up(w.k, 16);
        a.fprec = w.fprec;
        a.X = static_cast<const char*>(X) + b0 * ldx * elem_bytes(prec);
        a.ldx = ldx;
        a.Y = static_cast<char*>(Y) + (b0 * ldy + i0) * elem_bytes(yprec);
        a.ldy = ldy;
        a.yprec = yprec;
        a.m = rows;
        a.n = w.n;
        a.b = b;
        ws.reset();
        return prec == P32   ? apply_t<float>(part, a, prec, ws, st)
               : prec == P16 ? apply_t<half_t>(part, a, prec, ws, st)
                             : apply_t<bhalf_t>(part, a, prec, ws, st);
    };
    const int64_t most = weight_panel(std::min(batch, kQ4Panel));
    return in_panels(batch, kQ4Panel, [&](int64_t b0, int64_t b) {
        return in_panels(w.m, most, [&](int64_t i0, int64_t rows) { return panel(i0, rows, b0, b); });
    });
}

}  // namespace lrc
