// Root-mean-square norm of rows, with the residual's addition in front and, if
// asked for, an 8-bit output behind; and its gradient.
//
//   h = x + r (rounded once to the storage type), rstd = (mean h^2 + eps)^(-1/2),
//   y = h rstd w;   in 8 bits: t = max |y| / 448, y8 = the e4m3 value nearest to the binary32 y / t.
//   dh = rstd (w dy - h rstd mean(w dy h rstd)) + dsum,   dw = sum_rows dy h rstd.
//
// Bound by memory: every array is read or written once.  A row stays in the
// registers of its workgroup between its sum, its maximum and its output (up to NV
// vectors of 16 bytes a thread); longer rows are read again.  Thread t of NT takes
// the row's whole vectors t, t + NT, .. and the n % kVec last elements one a thread.
// 4096 rows of 8192 in bfloat16 with a residual, to e4m3: 50 us, 4.7 TB/s (a large copy
// 4.7); 2047 rows of 5003 (odd rows begin off 16 bytes) 21 us, their gradient 25 us and 5 for
// the sum of dw: 3.9 and 3.3 TB/s.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "head_device.h"

namespace lrc {

namespace {

constexpr float kE4m3Max = 448.0f;
constexpr unsigned kE4m3NaN = 0x7F7F7F7Fu;

// kVec<T> weights from element i on (1 without weights), whatever their type.
template <int E> __device__ __forceinline__ void load_weights(const void* w, int prec, int64_t i, float (&out)[E]) {
    if (!w) {
#pragma unroll
        for (int e = 0; e < E; ++e) out[e] = 1.0f;
    } else if (prec == P32) {
        const float* p = static_cast<const float*>(w) + i;
#pragma unroll
        for (int h = 0; h < E / 4; ++h) {
            const uint4v_t v = load16(p + 4 * h);
#pragma unroll
            for (int e = 0; e < 4; ++e) out[4 * h + e] = elem<float>(v, e);
        }
    } else {
        const unsigned short* p = static_cast<const unsigned short*>(w) + i;
        uint4v_t v = {0, 0, 0, 0};
        if (E == 8) {
            v = load16(p);
        } else {
            uint2v_t h;
            __builtin_memcpy(&h, p, 8);
            v[0] = h[0];
            v[1] = h[1];
        }
#pragma unroll
        for (int e = 0; e < E; ++e) out[e] = prec == P16 ? elem<half_t>(v, e) : elem<bhalf_t>(v, e);
    }
}
__device__ __forceinline__ float load_weight(const void* w, int prec, int64_t i) {
    return w ? load_as_f32(w, i, prec) : 1.0f;
}

__device__ __forceinline__ unsigned abs_bits(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

// Largest of the workgroup's values, with a barrier.
template <int NT> __device__ __forceinline__ unsigned block_umax(unsigned x, unsigned* red) {
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) x = std::max(x, (unsigned)__shfl_xor((int)x, off, 64));
    if (NT == 64) return x;
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) x = std::max(x, red[w]);
    return x;
}
template <int NT> __device__ __forceinline__ float block_total(float x, float* red) {
    if constexpr (NT == 64) return wave_sum(x);
    else return block_add<NT>(x, red);
}

// The 8-bit codes of a row: the values nearest to the binary32 quotients y / t, t its scale, ties to
// even.  A quotient is y (1 / t) corrected by its remainder twice: the first time leaves it less than
// a step from y / t, the second the nearest binary32 value.  (y (1 / t) alone is off by a step or two, which
// takes the other neighbour where y / t lies there beside the middle of two codes; products of bfloat16 values
// and weights meet such middles in one place of ten thousand.)  4096 rows of 8192: 51 us with
// the corrections, 50.5 without (shortest calls).
struct ToE4m3 {
    float t, up, d, inv;         // d = t up, a power of two that keeps the remainders of tiny scales in range
    bool nan;
    __device__ __forceinline__ explicit ToE4m3(unsigned amax_bits) {
        nan = amax_bits >= 0x7F800000u;                     // a NaN or an infinity among the y
        t = nan ? __builtin_nanf("") : __uint_as_float(amax_bits) / kE4m3Max;
        up = t < 0x1p-60f ? 0x1p80f : 1.0f;
        d = t * up;
        inv = d > 0.0f ? 1.0f / d : 0.0f;                   // a scale of 0: codes 0
    }
    // the clamp meets scales that rounding made too small
    __device__ __forceinline__ float scaled(float y) const {
        const float a = y * up;
        float q = a * inv;
        q = __builtin_fmaf(__builtin_fmaf(-q, d, a), inv, q);
        q = __builtin_fmaf(__builtin_fmaf(-q, d, a), inv, q);
        return __builtin_copysignf(__builtin_fminf(__builtin_fabsf(q), kE4m3Max), y);     // the corrections lose the sign of 0
    }
    __device__ __forceinline__ unsigned pack4(const float* y) const {
        if (nan) return kE4m3NaN;
        int v = __builtin_amdgcn_cvt_pk_fp8_f32(scaled(y[0]), scaled(y[1]), 0, false);
        return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(scaled(y[2]), scaled(y[3]), v, true);
    }
    __device__ __forceinline__ unsigned char one(float y) const {
        const float v[4] = {y, 0.0f, 0.0f, 0.0f};
        return (unsigned char)pack4(v);
    }
};

}  // namespace

// Q8: y in e4m3 with the scale of each row; else in T.
template <typename T, bool Q8, int NV, int NT>
__global__ __launch_bounds__(NT) void k_rms_norm(NormArgs a, int64_t row0) {
    constexpr int E = kVec<T>;
    __shared__ float red[NT / 64];
    __shared__ unsigned redm[NT / 64];
    const int t = threadIdx.x;
    const int64_t r = row0 + blockIdx.x;
    const T* x = static_cast<const T*>(a.x) + r * a.ldx;
    const T* res = a.residual ? static_cast<const T*>(a.residual) + r * a.ldr : nullptr;
    T* sum = a.sum ? static_cast<T*>(a.sum) + r * a.lds : nullptr;
    const int64_t full = a.n / E, tail = full * E + t;
    const bool has_tail = tail < a.n;

    uint4v_t v[NV > 0 ? NV : 1];
    float ss = 0.0f, last = 0.0f;
    // h of vector q, also stored
    auto take = [&](int64_t q) {
        uint4v_t h = load16_once(x + q * E);
        if (res) {
            const uint4v_t o = load16_once(res + q * E);
            float f[E];
#pragma unroll
            for (int e = 0; e < E; ++e) f[e] = elem<T>(h, e) + elem<T>(o, e);
            h = pack16<T>(f);
            if (sum) store16_once(sum + q * E, h);
        }
#pragma unroll
        for (int e = 0; e < E; ++e) ss += elem<T>(h, e) * elem<T>(h, e);
        return h;
    };
    if (has_tail) {
        T h = x[tail];
        if (res) {
            h = from_f32<T>((float)h + (float)res[tail]);
            if (sum) sum[tail] = h;
        }
        last = (float)h;
        ss += last * last;
    }
    if constexpr (NV > 0) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int64_t q = t + (int64_t)i * NT;
            v[i] = uint4v_t{0, 0, 0, 0};
            if (q < full) v[i] = take(q);
        }
    } else {
        for (int64_t q = t; q < full; q += NT) (void)take(q);
    }
    const float rstd = 1.0f / sqrtf(block_total<NT>(ss, red) / (float)a.n + a.eps);
    if (a.rstd && t == 0) a.rstd[r] = rstd;
    if constexpr (NV > 0) stay(v);

    // y of a vector held in h
    auto scaled = [&](const uint4v_t& h, int64_t q, float (&y)[E]) {
        float w[E];
        load_weights<E>(a.weight, a.wprec, q * E, w);
#pragma unroll
        for (int e = 0; e < E; ++e) y[e] = elem<T>(h, e) * rstd * w[e];
    };
    auto again = [&](int64_t q) {                           // h of a row that the registers do not hold
        if (!res) return load16(x + q * E);
        if (sum) return load16(sum + q * E);
        const uint4v_t h = load16(x + q * E), o = load16(res + q * E);
        float f[E];
#pragma unroll
        for (int e = 0; e < E; ++e) f[e] = elem<T>(h, e) + elem<T>(o, e);
        return pack16<T>(f);
    };
    auto each = [&](auto&& f) {
        if constexpr (NV > 0) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int64_t q = t + (int64_t)i * NT;
                if (q < full) f(q, v[i]);
            }
        } else {
            for (int64_t q = t; q < full; q += NT) f(q, again(q));
        }
    };
    const float ylast = has_tail ? last * rstd * load_weight(a.weight, a.wprec, tail) : 0.0f;
    if constexpr (Q8) {
        unsigned amax = abs_bits(ylast);
        each([&](int64_t q, const uint4v_t& h) {
            float y[E];
            scaled(h, q, y);
#pragma unroll
            for (int e = 0; e < E; ++e) amax = std::max(amax, abs_bits(y[e]));
        });
        const ToE4m3 to(block_umax<NT>(amax, redm));
        if (t == 0) a.scales[r] = to.t;
        unsigned char* out = static_cast<unsigned char*>(a.y) + r * a.ldy;
        each([&](int64_t q, const uint4v_t& h) {
            float y[E];
            scaled(h, q, y);
            unsigned c[E / 4];
#pragma unroll
            for (int e = 0; e < E / 4; ++e) c[e] = to.pack4(y + 4 * e);
            __builtin_memcpy(out + q * E, c, E);
        });
        if (has_tail) out[tail] = to.one(ylast);
    } else {
        T* out = static_cast<T*>(a.y) + r * a.ldy;
        each([&](int64_t q, const uint4v_t& h) {
            float y[E];
            scaled(h, q, y);
            store16_once(out + q * E, pack16<T>(y));
        });
        if (has_tail) out[tail] = from_f32<T>(ylast);
    }
}

// A workgroup takes the rows g, g + G, .. and adds up their part of dw, each thread
// for the columns that are its own: part[g][n].  NV <= 2: the next row is on its way
// while this one is reduced, and the weights stay in registers; threads past the row's
// vectors load and store the last one again, the same bits, without a branch (a branch around
// stores would make the next row's loads wait for them).  NV = 0: rows of any
// length, read twice, and dw through the partial sums in memory.
template <typename T, int NV, int NT>
__global__ __launch_bounds__(NT, 4) void k_rms_norm_backward(NormGradArgs a, float* __restrict__ part) {
    constexpr int E = kVec<T>, H = NV > 0 ? NV : 1;
    constexpr bool kAhead = NV == 1 || NV == 2;
    __shared__ float red[2][NT / 64];
    const int t = threadIdx.x, nt = blockDim.x;             // whole waves, at most NT
    const int64_t full = a.n / E, tail = full * E + t;
    const bool has_tail = tail < a.n;
    float dw[H][E], dwlast = 0.0f;
#pragma unroll
    for (int i = 0; i < H; ++i)
#pragma unroll
        for (int e = 0; e < E; ++e) dw[i][e] = 0.0f;
    float* mine = part ? part + (int64_t)blockIdx.x * a.n : nullptr;
    const float wlast = has_tail ? load_weight(a.weight, a.wprec, tail) : 0.0f;
    float wv[H][E];
    if constexpr (kAhead) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
#pragma unroll
            for (int e = 0; e < E; ++e) wv[i][e] = 0.0f;
            load_weights<E>(a.weight, a.wprec, std::min(t + (int64_t)i * nt, full - 1) * E, wv[i]);
        }
    }
    uint4v_t vd[H], vh[H], vs[H], nd[H], nh[H];
    float rstd = 0.0f, nrstd = 0.0f;
    T td{}, th{}, ts{}, ntd{}, nth{};                       // the tail's element
    auto fetch = [&](int64_t r, uint4v_t (&d)[H], uint4v_t (&x)[H], float& rs, T& dl, T& xl) {
        const T* dy = static_cast<const T*>(a.dy) + r * a.lddy;
        const T* h = static_cast<const T*>(a.h) + r * a.ldh;
        rs = a.rstd[r];
        if (has_tail) {
            dl = dy[tail];
            xl = h[tail];
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int64_t q = std::min(t + (int64_t)i * nt, full - 1);
            d[i] = load16_once(dy + q * E);
            x[i] = load16_once(h + q * E);
        }
    };
    int parity = 0;
    if constexpr (kAhead)
        if ((int64_t)blockIdx.x < a.rows) fetch(blockIdx.x, nd, nh, nrstd, ntd, nth);
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x, parity ^= 1) {
        const T* dy = static_cast<const T*>(a.dy) + r * a.lddy;
        const T* h = static_cast<const T*>(a.h) + r * a.ldh;
        const T* ds = a.dsum ? static_cast<const T*>(a.dsum) + r * a.ldd : nullptr;
        T* dx = static_cast<T*>(a.dx) + r * a.ldx;
        // asked for before the next row, and needed after the sum
        if (ds && has_tail) ts = ds[tail];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int64_t q = std::min(t + (int64_t)i * nt, full - 1);
            vs[i] = uint4v_t{0, 0, 0, 0};
            if (ds) vs[i] = load16_once(ds + q * E);
        }
        if constexpr (kAhead) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                vd[i] = nd[i];
                vh[i] = nh[i];
            }
            rstd = nrstd;
            td = ntd;
            th = nth;
            if (r + gridDim.x < a.rows) fetch(r + gridDim.x, nd, nh, nrstd, ntd, nth);
        } else {
            fetch(r, vd, vh, rstd, td, th);
        }
        float s = 0.0f;
        auto weights = [&](int i, int64_t q, float (&w)[E]) {
            if constexpr (kAhead) {
#pragma unroll
                for (int e = 0; e < E; ++e) w[e] = wv[i][e];
            } else {
                load_weights<E>(a.weight, a.wprec, q * E, w);
            }
        };
        auto along = [&](int i, int64_t q, const uint4v_t& d, const uint4v_t& x) {
            float w[E];
            weights(i, q, w);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float g = elem<T>(d, e), xh = elem<T>(x, e) * rstd;
                s += g * w[e] * xh;
                if (NV > 0) dw[i][e] += g * xh;
            }
        };
        float gl = 0.0f, xl = 0.0f;
        if (has_tail) {
            gl = (float)td;
            xl = (float)th * rstd;
            s += gl * wlast * xl;
            dwlast += gl * xl;
        }
        if constexpr (NV > 0) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (t + (int64_t)i * nt < full) along(i, t + (int64_t)i * nt, vd[i], vh[i]);
        } else {
            for (int64_t q = t; q < full; q += nt) along(0, q, load16(dy + q * E), load16(h + q * E));
        }
        // Where dx is dy or dsum, several threads load a row's last vector and several store it: it has
        // to be here in each of them before the barrier, behind which the first may store.
        if constexpr (NV > 0) {
            stay(vd);
            stay(vs);
        }
        // the sum of the row; two sets of places, so that one barrier a row is enough
        float total = wave_sum(s);
        if (NT > 64 && nt > 64) {
            if ((t & 63) == 0) red[parity][t >> 6] = total;
            __syncthreads();
            total = 0.0f;
            for (int w = 0; w < nt / 64; ++w) total += red[parity][w];
        }
        const float mean = total / (float)a.n;
        auto store = [&](int i, int64_t q, const uint4v_t& d, const uint4v_t& x, const uint4v_t& o) {
            float w[E], g[E];
            weights(i, q, w);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float y = rstd * (elem<T>(d, e) * w[e] - elem<T>(x, e) * rstd * mean);
                g[e] = ds ? y + elem<T>(o, e) : y;
            }
            store16_once(dx + q * E, pack16<T>(g));
        };
        if constexpr (NV > 0) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
                store(i, std::min(t + (int64_t)i * nt, full - 1), vd[i], vh[i], vs[i]);
        } else {
            for (int64_t q = t; q < full; q += nt) {
                const uint4v_t d = load16(dy + q * E), x = load16(h + q * E);
                if (mine) {
                    const bool first = r == blockIdx.x;
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        const float g = elem<T>(d, e) * (elem<T>(x, e) * rstd);
                        mine[q * E + e] = first ? g : mine[q * E + e] + g;
                    }
                }
                store(0, q, d, x, ds ? load16(ds + q * E) : uint4v_t{0, 0, 0, 0});
            }
        }
        if (has_tail) {
            const float y = rstd * (gl * wlast - xl * mean);
            dx[tail] = from_f32<T>(ds ? y + (float)ts : y);
        }
    }
    if (!mine) return;
    if constexpr (NV > 0) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int64_t q = t + (int64_t)i * nt;
            if (q < full)
#pragma unroll
                for (int h = 0; h < E / 4; ++h) {
                    const float4_t o = {dw[i][4 * h], dw[i][4 * h + 1], dw[i][4 * h + 2], dw[i][4 * h + 3]};
                    __builtin_memcpy(mine + q * E + 4 * h, &o, 16);
                }
        }
    }
    if (has_tail) mine[tail] = dwlast;
}

// dw = the sum of the workgroups' parts: 64 columns a workgroup, its 16 waves a run of
// the parts each, added up in wave order.
__global__ __launch_bounds__(1024) void k_rms_norm_dw(const float* __restrict__ part, int64_t groups, int64_t n,
                                                      void* __restrict__ dw, int wprec) {
    __shared__ float red[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t c = (int64_t)blockIdx.x * 64 + lane;
    float s = 0.0f;
    if (c < n) {
        const int64_t end = groups * (wave + 1) / 16;
        for (int64_t g = groups * wave / 16; g < end; g += 8) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = g + e < end ? part[(g + e) * n + c] : 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) s += v[e];
        }
    }
    red[wave][lane] = s;
    __syncthreads();
    if (wave == 0 && c < n) {
#pragma unroll
        for (int w = 1; w < 16; ++w) s += red[w][lane];
        store_from_f32(dw, c, wprec, s);
    }
}

namespace {

// Threads of a row: with many rows as few as hold it in four vectors each, so that a compute
// unit holds several rows, with few rows one vector each.  bfloat16, rows of 5003, four vectors against
// one: 512 rows 11.6 and 9.2 us, 1024 rows 14.2 and 15.5, 4096 rows 40 and 48 (rows of 8192, which
// fill 1024 threads: 12.6 and 9.3, 16.7 and 16.4, 52 and 49).  nv = 0: the row is read again.
struct NormPlan {
    int nt, nv;
};
NormPlan plan_norm(int64_t rows, int64_t n, int prec) {
    const int64_t vecs = n / (prec == P32 ? 4 : 8), want = rows >= 1024 ? 4 : 1;
    NormPlan p{vecs <= 64 * want ? 64 : vecs <= 256 * want ? 256 : 1024, 0};
    const int64_t nv = (vecs + p.nt - 1) / p.nt;
    p.nv = nv <= 1 ? 1 : nv <= 2 ? 2 : nv <= 4 ? 4 : 0;
    return p;
}

template <typename T, bool Q8, int NV, int NT>
hipError_t norm_launch(const NormArgs& a, hipStream_t st) {
    return in_panels(a.rows, kRowPanel, [&](int64_t r, int64_t rows) {
        KernelTimer t("rms_norm", st);
        hipLaunchKernelGGL((k_rms_norm<T, Q8, NV, NT>), dim3((unsigned)rows), dim3(NT), 0, st, a, r);
        return hipGetLastError();
    });
}
template <typename T, bool Q8>
hipError_t norm_t(const NormArgs& a, hipStream_t st) {
    const NormPlan p = plan_norm(a.rows, a.n, a.prec);
#define LRC_NORM(NV, NT) \
    if (p.nv == NV && p.nt == NT) return norm_launch<T, Q8, NV, NT>(a, st);
    LRC_NORM(1, 64) LRC_NORM(2, 64) LRC_NORM(4, 64) LRC_NORM(1, 256) LRC_NORM(2, 256) LRC_NORM(4, 256)
    LRC_NORM(1, 1024) LRC_NORM(2, 1024) LRC_NORM(4, 1024)
#undef LRC_NORM
    return norm_launch<T, Q8, 0, 1024>(a, st);
}

struct NormGradPlan {
    int nt, nv;
    int64_t groups;
};
NormGradPlan plan_norm_grad(int64_t rows, int64_t n, int prec) {
    const int64_t vecs = n / (prec == P32 ? 4 : 8);
    NormGradPlan p;
    // waves that hold the row in two vectors a thread, four past 2 x 1024
    p.nv = vecs < 1 ? 0 : vecs <= 64 ? 1 : vecs <= 2048 ? 2 : vecs <= 4096 ? 4 : 0;
    p.nt = p.nv == 0 ? 1024 : (int)std::max<int64_t>(1, (vecs + 64 * p.nv - 1) / (64 * p.nv)) * 64;
    // as many workgroups as the compute units hold at once, with the same number of rows each
    const int64_t most = 256 * std::max(1, 1024 / p.nt), rounds = std::max<int64_t>(1, (rows + most - 1) / most);
    p.groups = (rows + rounds - 1) / rounds;
    return p;
}

template <typename T, int NV, int NT>
hipError_t grad_launch(const NormGradArgs& a, float* part, const NormGradPlan& p, hipStream_t st) {
    KernelTimer t("rms_norm_backward", st);
    hipLaunchKernelGGL((k_rms_norm_backward<T, NV, NT>), dim3((unsigned)p.groups), dim3(p.nt), 0, st, a, part);
    return hipGetLastError();
}
template <typename T> hipError_t grad_t(const NormGradArgs& a, Workspace& ws, hipStream_t st) {
    const NormGradPlan p = plan_norm_grad(a.rows, a.n, a.prec);
    float* part = nullptr;
    if (a.dw && a.rows) {
        part = static_cast<float*>(ws.take((size_t)p.groups * a.n * 4));
        if (ws.overrun) return hipErrorOutOfMemory;
    }
    hipError_t e = hipSuccess;
    if (a.rows) {
        if (p.nv == 1) e = grad_launch<T, 1, 64>(a, part, p, st);
        else if (p.nv == 2 && p.nt <= 512) e = grad_launch<T, 2, 512>(a, part, p, st);
        else if (p.nv == 2) e = grad_launch<T, 2, 1024>(a, part, p, st);
        else if (p.nv == 4) e = grad_launch<T, 4, 1024>(a, part, p, st);
        else e = grad_launch<T, 0, 1024>(a, part, p, st);
    }
    if (e != hipSuccess || !a.dw) return e;
    KernelTimer t("rms_norm_dw", st);
    hipLaunchKernelGGL(k_rms_norm_dw, dim3((unsigned)((a.n + 63) / 64)), dim3(1024), 0, st, part, a.rows ? p.groups : 0, a.n,
                       a.dw, a.wprec);
    return hipGetLastError();
}

}  // namespace

size_t norm_grad_workspace_bytes(const NormGradArgs& a) {
    return a.dw && a.rows ? (size_t)plan_norm_grad(a.rows, a.n, a.prec).groups * a.n * 4 + 256 : 0;
}

hipError_t launch_rms_norm(const NormArgs& a, hipStream_t st) {
    if (a.scales)
        return a.prec == P32   ? norm_t<float, true>(a, st)
               : a.prec == P16 ? norm_t<half_t, true>(a, st)
                               : norm_t<bhalf_t, true>(a, st);
    return a.prec == P32   ? norm_t<float, false>(a, st)
           : a.prec == P16 ? norm_t<half_t, false>(a, st)
                           : norm_t<bhalf_t, false>(a, st);
}

hipError_t launch_rms_norm_backward(const NormGradArgs& a, Workspace& ws, hipStream_t st) {
    return a.prec == P32   ? grad_t<float>(a, ws, st)
           : a.prec == P16 ? grad_t<half_t>(a, ws, st)
                           : grad_t<bhalf_t>(a, ws, st);
}

}  // namespace lrc
