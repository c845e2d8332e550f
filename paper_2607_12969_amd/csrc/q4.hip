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

template <typename T>
static void quantize_t(const void* W, int64_t ldw, int64_t m, int64_t n, int64_t group, void* codes, void* scales,
                       int sprec, void* values, unsigned long long* nbad, hipStream_t st) {
    const int64_t wpr = q4_row_bytes(n) / 4, chunks = (wpr + 63) / 64, G = (n + group - 1) / group;
    const bool vec = reinterpret_cast<uintptr_t>(W) % 16 == 0 && ldw * sizeof(T) % 16 == 0 &&
                     (!values || (reinterpret_cast<uintptr_t>(values) % 16 == 0 && n * sizeof(T) % 16 == 0));
    const unsigned grid = (unsigned)((m * chunks + 3) / 4);
    auto* kern = vec ? k_q4_quantize<T, true> : k_q4_quantize<T, false>;
    hipLaunchKernelGGL(kern, dim3(grid), dim3(256), 0, st, (const T*)W, ldw, m, n, (int)(group / 8), (int)chunks,
                       (unsigned*)codes, wpr, scales, G, sprec, (T*)values, nbad);
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
    const float* Tm;     // T' [batch][k]
    int64_t k;
    int fprec;
    const void* X;
    int64_t ldx;
    void* Y;
    int64_t ldy;
    int yprec;
    int64_t m, n, b;
};

// Activations as MFMA operands: P planes of 8 values.
template <typename T> struct ActTraits;
template <> struct ActTraits<half_t> {
    static constexpr int P = 1;
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

// x = h + m + l exactly, each with 8 significant bits; an infinity keeps its
// sign in h alone, NaN stays NaN.
__device__ __forceinline__ void split3(float x, unsigned short (&p)[3]) {
    const unsigned ux = __float_as_uint(x);
    unsigned hi = ux & 0xFFFF0000u;
    float r = x - __uint_as_float(hi);
    if ((ux & 0x7FFFFFFFu) == 0x7F800000u) r = 0.0f;
    if (x != x) hi = 0x7FC00000u;
    const unsigned um = __float_as_uint(r);
    const float l = (r != r) ? 0.0f : r - __uint_as_float(um & 0xFFFF0000u);
    p[0] = (unsigned short)(hi >> 16);
    p[1] = (unsigned short)((r != r) ? 0u : um >> 16);
    p[2] = (unsigned short)(__float_as_uint(l) >> 16);
}

// The 8 values x[j .. j + 8) of one row of n as MFMA operands; zero past n.
template <typename T, bool VEC>
__device__ __forceinline__ void load_act(const T* x, int64_t j, int64_t n, typename ActTraits<T>::frag (&f)[ActTraits<T>::P]) {
    T v[8];
    if (VEC && j + 8 <= n) {
        typedef T vec_t __attribute__((ext_vector_type(16 / sizeof(T))));
#pragma unroll
        for (int h = 0; h < (int)(8 * sizeof(T) / 16); ++h) {
            const vec_t w = reinterpret_cast<const vec_t*>(x + j)[h];
#pragma unroll
            for (int q = 0; q < (int)(16 / sizeof(T)); ++q) v[h * (16 / sizeof(T)) + q] = w[q];
        }
    } else {
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] = j + q < n ? x[j + q] : (T)0.0f;
    }
    if constexpr (sizeof(T) == 4) {
        unsigned short s[3][8];
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            unsigned short p[3];
            split3(v[q], p);
#pragma unroll
            for (int t = 0; t < 3; ++t) s[t][q] = p[t];
        }
#pragma unroll
        for (int t = 0; t < 3; ++t) f[t] = __builtin_bit_cast(bhalf8_t, s[t]);
    } else {
        f[0] = __builtin_bit_cast(typename ActTraits<T>::frag, v);
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

// One workgroup of 4 waves: 16 RT rows of W for 16 NB rows of X; the waves
// split the columns in steps of 128 and add up through LDS in a fixed order.
template <typename T, int NB, int RT, bool VEC>
__global__ __launch_bounds__(256) void k_q4_rows(Q4Args a) {
    using Tr = ActTraits<T>;
    __shared__ float red[4][16 * NB][16 * RT + 1];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int lr = lane & 15, lg = lane >> 4;
    const int64_t i0 = (int64_t)blockIdx.x * 16 * RT, b0 = (int64_t)blockIdx.y * 16 * NB;
    int64_t row[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) row[r] = std::min(i0 + 16 * r + lr, a.m - 1);
    const T* x[NB];
#pragma unroll
    for (int f = 0; f < NB; ++f) x[f] = static_cast<const T*>(a.X) + std::min(b0 + 16 * f + lr, a.b - 1) * a.ldx;
    float4_t acc[RT][NB];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int f = 0; f < NB; ++f) acc[r][f] = zero_accv<float4_t>();
    const int64_t blocks = (a.n + 127) / 128;
    for (int64_t kb = wave; kb < blocks; kb += 4) {
        unsigned w[RT][4];
        const int64_t off = kb * 64 + lg * 16;
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            uint4v_t c = {0, 0, 0, 0};
            if (off < a.rb) c = *reinterpret_cast<const uint4v_t*>(a.codes + row[r] * a.rb + off);
#pragma unroll
            for (int t = 0; t < 4; ++t) w[r][t] = c[t];
            transpose4(w[r]);
        }
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int64_t j = kb * 128 + t * 32;
            if (j >= a.n) break;
            typename Tr::frag xa[NB][Tr::P];
#pragma unroll
            for (int f = 0; f < NB; ++f) load_act<T, VEC>(x[f], j + lg * 8, a.n, xa[f]);
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const float sc = load_as_f32(a.scales, row[r] * a.G + (j >> a.gshift), a.sprec);
                const typename Tr::frag wf = Tr::widen(w[r][t]);
#pragma unroll
                for (int f = 0; f < NB; ++f) {
                    float4_t d = zero_accv<float4_t>();
#pragma unroll
                    for (int p = Tr::P - 1; p >= 0; --p) d = Tr::mfma(xa[f][p], wf, d);
#pragma unroll
                    for (int v = 0; v < 4; ++v) acc[r][f][v] += sc * d[v];
                }
            }
        }
    }
    // compensation: T' (rows of the batch) against U (rows of W), 16 ranks a step
    for (int64_t q = wave * 16; q < a.k; q += 64) {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int64_t c = q + lg * 4 + t;
            float tv[NB], uv[RT];
#pragma unroll
            for (int f = 0; f < NB; ++f) tv[f] = c < a.k ? a.Tm[std::min(b0 + 16 * f + lr, a.b - 1) * a.k + c] : 0.0f;
#pragma unroll
            for (int r = 0; r < RT; ++r) uv[r] = c < a.k ? load_as_f32(a.U, row[r] * a.k + c, a.fprec) : 0.0f;
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int f = 0; f < NB; ++f) acc[r][f] = mfma(tv[f], uv[r], acc[r][f]);
        }
    }
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int f = 0; f < NB; ++f)
#pragma unroll
            for (int v = 0; v < 4; ++v) red[wave][16 * f + 4 * lg + v][16 * r + lr] = acc[r][f][v];
    __syncthreads();
    for (int e = threadIdx.x; e < 256 * NB * RT; e += 256) {
        const int i = e % (16 * RT), f = e / (16 * RT);
        if (i0 + i < a.m && b0 + f < a.b) {
            float y = red[0][f][i];
            y += red[1][f][i];
            y += red[2][f][i];
            y += red[3][f][i];
            store_from_f32(a.Y, (b0 + f) * a.ldy + i0 + i, a.yprec, y);
        }
    }
}

// Partial sums of V^T x: part[split][batch][k], one wave per 16 ranks x 16
// batch rows x split of the columns.
template <typename T, bool VEC>
__global__ __launch_bounds__(64) void k_q4_mid(const T* __restrict__ X, int64_t ldx, const void* __restrict__ V,
                                               int fprec, int64_t n, int64_t k, int64_t b, int64_t chunk,
                                               float* __restrict__ part) {
    const int lane = threadIdx.x, lr = lane & 15, lg = lane >> 4;
    const int64_t r0 = (int64_t)blockIdx.x * 16, b0 = (int64_t)blockIdx.y * 16, s = blockIdx.z;
    const int64_t j0 = s * chunk, j1 = std::min(n, j0 + chunk);
    const T* x = X + std::min(b0 + lr, b - 1) * ldx;
    const int64_t r = std::min(r0 + lr, k - 1);
    float4_t acc = zero_accv<float4_t>();
    for (int64_t j = j0 + lg * 8; j - lg * 8 < j1; j += 32) {
        float xv[8];
        if (VEC && j + 8 <= j1) {
            typedef T vec_t __attribute__((ext_vector_type(16 / sizeof(T))));
#pragma unroll
            for (int h = 0; h < (int)(8 * sizeof(T) / 16); ++h) {
                const vec_t w = reinterpret_cast<const vec_t*>(x + j)[h];
#pragma unroll
                for (int q = 0; q < (int)(16 / sizeof(T)); ++q) xv[h * (16 / sizeof(T)) + q] = (float)w[q];
            }
        } else {
#pragma unroll
            for (int q = 0; q < 8; ++q) xv[q] = j + q < j1 ? (float)x[j + q] : 0.0f;
        }
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            const float v = j + q < j1 ? load_as_f32(V, (j + q) * k + r, fprec) : 0.0f;
            acc = mfma(xv[q], v, acc);
        }
    }
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        const int64_t bb = b0 + 4 * lg + v;
        if (bb < b && r0 + lr < k) part[(s * b + bb) * k + r0 + lr] = acc[v];
    }
}

// T'[b][r] = s_r times the sum of the partials, in split order.
__global__ __launch_bounds__(256) void k_q4_mid_finish(const float* __restrict__ part, int splits,
                                                       const void* __restrict__ s, int fprec, int64_t k, int64_t count,
                                                       float* __restrict__ Tm) {
    const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (e >= count) return;
    float t = 0.0f;
    for (int q = 0; q < splits; ++q) t += part[q * count + e];
    Tm[e] = t * load_as_f32(s, e % k, fprec);
}

namespace {
struct MidPlan {
    int splits;
    int64_t chunk;
};
// About four waves per compute unit, each at least 64 columns deep.
MidPlan plan_mid(int64_t n, int64_t k, int64_t b) {
    const int64_t tiles = (k + 15) / 16 * ((b + 15) / 16);
    int64_t s = std::max<int64_t>(1, std::min<int64_t>(1024 / std::max<int64_t>(tiles, 1), (n + 63) / 64));
    const int64_t chunk = round_up((n + s - 1) / s, 32);
    s = (n + chunk - 1) / chunk;
    return {(int)s, chunk};
}
}  // namespace

size_t q4_apply_workspace_bytes(const Q4Weights& w, int64_t batch, int) {
    if (!w.k) return 0;
    const size_t t = (size_t)batch * w.k * 4;
    return (size_t)round_up((int64_t)t, 256) + (size_t)round_up((int64_t)(t * plan_mid(w.n, w.k, batch).splits), 256);
}

template <typename T, int NB, int RT>
static void launch_rows(const Q4Args& a, bool vec, hipStream_t st) {
    KernelTimer t("q4_rows", st);
    auto* kern = vec ? k_q4_rows<T, NB, RT, true> : k_q4_rows<T, NB, RT, false>;
    hipLaunchKernelGGL(kern, dim3((unsigned)((a.m + 16 * RT - 1) / (16 * RT)), (unsigned)((a.b + 16 * NB - 1) / (16 * NB))),
                       dim3(256), 0, st, a);
}

template <typename T>
static hipError_t apply_t(const Q4Weights& w, Q4Args& a, Workspace& ws, hipStream_t st) {
    const bool vec = reinterpret_cast<uintptr_t>(a.X) % 16 == 0 && a.ldx * sizeof(T) % 16 == 0;
    if (w.k) {
        const MidPlan p = plan_mid(w.n, w.k, a.b);
        float* Tm = static_cast<float*>(ws.take((size_t)a.b * w.k * 4));
        float* part = static_cast<float*>(ws.take((size_t)p.splits * a.b * w.k * 4));
        if (ws.overrun) return hipErrorOutOfMemory;
        {
            KernelTimer t("q4_mid", st);
            auto* kern = vec ? k_q4_mid<T, true> : k_q4_mid<T, false>;
            hipLaunchKernelGGL(kern, dim3((unsigned)((w.k + 15) / 16), (unsigned)((a.b + 15) / 16), p.splits), dim3(64),
                               0, st, (const T*)a.X, a.ldx, w.V, w.fprec, w.n, w.k, a.b, p.chunk, part);
        }
        KernelTimer t("q4_mid_finish", st);
        const int64_t count = a.b * w.k;
        hipLaunchKernelGGL(k_q4_mid_finish, dim3((unsigned)((count + 255) / 256)), dim3(256), 0, st, part, p.splits,
                           w.s, w.fprec, w.k, count, Tm);
        a.Tm = Tm;
    }
    if (a.b <= 16) launch_rows<T, 1, 1>(a, vec, st);
    else if (a.b <= 32) launch_rows<T, 2, 2>(a, vec, st);
    else launch_rows<T, 4, 2>(a, vec, st);
    return hipGetLastError();
}

hipError_t launch_q4_apply(const Q4Weights& w, const void* X, int64_t ldx, void* Y, int64_t ldy, int64_t batch,
                           int prec, int yprec, Workspace& ws, hipStream_t st) {
    Q4Args a{};
    a.codes = static_cast<const unsigned char*>(w.codes);
    a.scales = w.scales;
    a.rb = q4_row_bytes(w.n);
    a.G = (w.n + w.group - 1) / w.group;
    a.sprec = w.sprec;
    a.gshift = __builtin_ctzll((unsigned long long)w.group);
    a.U = w.U;
    a.k = w.k;
    a.fprec = w.fprec;
    a.X = X;
    a.ldx = ldx;
    a.Y = Y;
    a.ldy = ldy;
    a.yprec = yprec;
    a.m = w.m;
    a.n = w.n;
    a.b = batch;
    if (prec == P32) return apply_t<float>(w, a, ws, st);
    if (prec == P16) return apply_t<half_t>(w, a, ws, st);
    return apply_t<bhalf_t>(w, a, ws, st);
}

}  // namespace lrc
