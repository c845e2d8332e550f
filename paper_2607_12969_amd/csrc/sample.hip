// One token per row of logits, from a given uniform number.
//
// With M the row's largest logit, c = log2(e) / T and z = (l - M) c (one
// rounding each), a token weighs w = 2^z, held as the whole number
// q = floor(2^31 w).  Sums of q are exact in any order, so the result does not
// depend on how a row is split, and a token lighter than 2^-31 of the likeliest
// (128 times finer than a 24-bit uniform number resolves) is never drawn.
//   top-k  the k first tokens by logit, ties by index;
//   top-p  of those, the tokens before which less than p of their mass lies;
//   min-p  of those, w >= min_p (the likeliest always stays);
//   draw   the first index at which the running sum of the kept q passes u S.
// top-k and top-p keep a prefix of the order by logit: every logit above some
// v, and the first r of those equal to v.  v and r come from histograms of
// counts and masses: 2048 bins over z in (-32, 0], then over the bits of the
// logits inside the bin that holds the cut.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "head_device.h"

namespace lrc {

namespace {

constexpr int kBins = 2048;
constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr float kNegInf = -__builtin_inff();

// Order of binary32 values as unsigned integers (no NaN; -0 just below 0 is
// folded onto 0 by the caller).
__device__ __forceinline__ unsigned key_of(float x) {
    const unsigned u = __float_as_uint(x);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float of_key(unsigned k) {
    return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k);
}



// A logit as the draw sees it: NaN counts as -infinity, -0 as 0.
__device__ __forceinline__ float logit(float x) { return x != x ? kNegInf : x + 0.0f; }

// kVec consecutive logits from index i on; -infinity past the row's end.
template <typename T, bool VEC>
__device__ __forceinline__ void load_logits(const T* row, int64_t i, int64_t V, float (&l)[kVec<T>]) {
    if (VEC && i + kVec<T> <= V) {
        typedef T vec_t __attribute__((ext_vector_type(kVec<T>)));
        const vec_t v = *reinterpret_cast<const vec_t*>(row + i);
#pragma unroll
        for (int e = 0; e < kVec<T>; ++e) l[e] = logit((float)v[e]);
    } else {
#pragma unroll
        for (int e = 0; e < kVec<T>; ++e) l[e] = i + e < V ? logit((float)row[i + e]) : kNegInf;
    }
}

struct Weigh {
    float M, c;
    __device__ __forceinline__ float z(float l) const { return l == M ? 0.0f : (l - M) * c; }
    __device__ __forceinline__ float w(float l) const { return __builtin_amdgcn_exp2f(z(l)); }
    static __device__ __forceinline__ unsigned q(float w) { return (unsigned)(w * 2147483648.0f); }
};

__device__ __forceinline__ float scale_of(float T) {
    return __builtin_fminf(__builtin_fmaxf((1.0f / T) * 1.4426950408889634f, 1.17549435e-38f), 3.4028234663852886e38f);
}

typedef unsigned long long u64;

__device__ __forceinline__ u64 wave_add(u64 x) {
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) x += __shfl_xor(x, off, 64);
    return x;
}

struct Shared {
    unsigned count[kBins];
    u64 mass[kBins];
    u64 red[kWaves];
    unsigned redc[kWaves];
    float redf[kWaves];
    int bin;
    u64 before;
    unsigned beforec;
    unsigned kmin, kmax;
};

// The first bin at which the running count (by_count) or mass reaches
// `target` (>= 1), and the running count and mass before it.  Every thread
// takes 2 bins.  bin = -1 when the total stays below the target.
__device__ __forceinline__ void find_bin(Shared& s, bool by_count, u64 target, int& bin, u64& before, unsigned& beforec) {
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const u64 m0 = s.mass[2 * t], m1 = s.mass[2 * t + 1];
    const unsigned c0 = s.count[2 * t], c1 = s.count[2 * t + 1];
    u64 m = m0 + m1;
    unsigned c = c0 + c1;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const u64 om = __shfl_up(m, off, 64);
        const unsigned oc = __shfl_up(c, off, 64);
        if (lane >= off) {
            m += om;
            c += oc;
        }
    }
    if (lane == 63) {
        s.red[wave] = m;
        s.redc[wave] = c;
    }
    if (t == 0) s.bin = -1;
    __syncthreads();
    for (int w = 0; w < wave; ++w) {
        m += s.red[w];
        c += s.redc[w];
    }
    const u64 e0 = by_count ? c - c0 - c1 : m - m0 - m1;          // before bin 2t
    const u64 e1 = e0 + (by_count ? c0 : m0), e2 = e1 + (by_count ? c1 : m1);
    if (e0 < target && e2 >= target) {
        const bool first = e1 >= target;
        s.bin = 2 * t + !first;
        s.before = first ? m - m0 - m1 : m - m1;
        s.beforec = first ? c - c0 - c1 : c - c1;
    }
    __syncthreads();
    bin = s.bin;
    before = s.before;
    beforec = s.beforec;
    __syncthreads();
}

// Visits the row: wave w takes the contiguous part [w L, (w + 1) L), blocks of
// 64 kVec logits, a lane kVec consecutive ones.
template <typename T, bool VEC, typename F>
__device__ __forceinline__ void visit(const T* row, int64_t V, int64_t L, F&& f) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t end = std::min(V, (wave + 1) * L);
    for (int64_t i = wave * L; i < end; i += 64 * kVec<T>) {
        float l[kVec<T>];
        load_logits<T, VEC>(row, i + lane * kVec<T>, V, l);
        f(i, l);
    }
}

// The cut at `target` in the order by logit: all logits above v, and of those
// equal to v as many as reach the target.  above: mass above v.  qv: weight of
// v, ties: tokens equal to v.  false when the row does not reach the target.
template <typename T, bool VEC>
__device__ bool select(Shared& s, const T* row, int64_t V, int64_t L, const Weigh& wt, bool by_count, u64 target,
                       float& v, u64& above, unsigned& countabove) {
    const int t = threadIdx.x;
    auto clear = [&] {
        for (int b = t; b < kBins; b += kThreads) {
            s.count[b] = 0;
            s.mass[b] = 0;
        }
        if (t == 0) {
            s.kmin = ~0u;
            s.kmax = 0u;
        }
        __syncthreads();
    };
    auto zbin = [](float z) { return std::min((int)(z * -64.0f), kBins - 1); };
    clear();
    visit<T, VEC>(row, V, L, [&](int64_t, const float (&l)[kVec<T>]) {
#pragma unroll
        for (int e = 0; e < kVec<T>; ++e) {
            const float z = wt.z(l[e]);
            if (z >= -31.0f) {
                const int b = zbin(z);
                atomicAdd(&s.count[b], 1u);
                atomicAdd(&s.mass[b], (u64)Weigh::q(__builtin_amdgcn_exp2f(z)));
            }
        }
    });
    __syncthreads();
    int bin;
    u64 before;
    unsigned beforec;
    find_bin(s, by_count, target, bin, before, beforec);
    if (bin < 0) return false;
    const int zb = bin;
    // range of keys inside the bin
    auto inside = [&](float l) {
        const float z = wt.z(l);
        return z >= -31.0f && zbin(z) == zb;
    };
    unsigned lo = ~0u, hi = 0u;
    visit<T, VEC>(row, V, L, [&](int64_t, const float (&l)[kVec<T>]) {
#pragma unroll
        for (int e = 0; e < kVec<T>; ++e)
            if (inside(l[e])) {
                const unsigned k = key_of(l[e]);
                lo = std::min(lo, k);
                hi = std::max(hi, k);
            }
    });
    if (t == 0) {
        s.kmin = ~0u;
        s.kmax = 0u;
    }
    __syncthreads();
    atomicMin(&s.kmin, lo);
    atomicMax(&s.kmax, hi);
    __syncthreads();
    lo = s.kmin;
    hi = s.kmax;
    __syncthreads();
    u64 base = before;
    unsigned basec = beforec;
    while (lo < hi) {
        // bins of 2^sh keys from the top
        int sh = 0;
        while (((hi - lo) >> sh) >= (unsigned)kBins) ++sh;
        clear();
        visit<T, VEC>(row, V, L, [&](int64_t, const float (&l)[kVec<T>]) {
#pragma unroll
            for (int e = 0; e < kVec<T>; ++e) {
                const unsigned k = key_of(l[e]);
                if (k >= lo && k <= hi) {
                    const unsigned b = (hi - k) >> sh;
                    atomicAdd(&s.count[b], 1u);
                    atomicAdd(&s.mass[b], (u64)Weigh::q(wt.w(l[e])));
                }
            }
        });
        __syncthreads();
        find_bin(s, by_count, target - (by_count ? basec : base), bin, before, beforec);
        if (bin < 0) break;
        base += before;
        basec += beforec;
        const unsigned top = hi - ((unsigned)bin << sh);
        lo = std::max(lo, top - ((1u << sh) - 1u));
        hi = top;
    }
    v = of_key(hi);
    above = base;
    countabove = basec;
    return true;
}

}  // namespace

template <typename T, bool VEC>
__global__ __launch_bounds__(kThreads) void k_sample_row(SampleArgs a, int64_t L) {
    __shared__ Shared s;
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const int64_t r = blockIdx.x, V = a.vocab;
    const T* row = static_cast<const T*>(a.logits) + r * a.ld;

    float M = kNegInf;
    visit<T, VEC>(row, V, L, [&](int64_t, const float (&l)[kVec<T>]) {
#pragma unroll
        for (int e = 0; e < kVec<T>; ++e) M = __builtin_fmaxf(M, l[e]);
    });
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) M = __builtin_fmaxf(M, __shfl_xor(M, off, 64));
    if (lane == 0) s.redf[wave] = M;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) M = __builtin_fmaxf(M, s.redf[w]);
    if (M == kNegInf) {          // nothing to draw from
        if (t == 0) a.tokens[r] = -1;
        return;
    }
    const float temp = a.temperature ? a.temperature[r] : 1.0f;
    const bool greedy = !(temp > 0.0f);
    Weigh wt{M, greedy ? 1.0f : scale_of(temp)};
    float v = kNegInf, floor_w = 0.0f;
    u64 ties = ~0ull;            // kept tokens equal to v
    if (greedy) {
        v = M;
        ties = 1;
    } else {
        const int64_t k = a.top_k ? a.top_k[r] : 0;
        const float p = a.top_p ? a.top_p[r] : 1.0f, mp = a.min_p ? a.min_p[r] : 0.0f;
        if (mp > 0.0f) floor_w = std::min(mp, 1.0f);
        u64 mass = 0;
        bool have = false;
        if (k > 0 && k < V) {
            float vk;
            u64 above;
            unsigned ca;
            if (select<T, VEC>(s, row, V, L, wt, true, (u64)k, vk, above, ca)) {
                v = vk;
                ties = (u64)k - ca;
                mass = above + ties * Weigh::q(wt.w(vk));
                have = true;
            }
        }
        if (p < 1.0f) {
            if (!have) {
                u64 m = 0;
                visit<T, VEC>(row, V, L, [&](int64_t, const float (&l)[kVec<T>]) {
#pragma unroll
                    for (int e = 0; e < kVec<T>; ++e) m += Weigh::q(wt.w(l[e]));
                });
                m = wave_add(m);
                if (lane == 0) s.red[wave] = m;
                __syncthreads();
                for (int w = 0; w < kWaves; ++w) mass += s.red[w];
                __syncthreads();
            }
            const double P = __builtin_ceil((double)p * (double)mass);
            const u64 target = P >= 1.0 ? (u64)P : 1ull;
            float vp;
            u64 above;
            unsigned ca;
            if (select<T, VEC>(s, row, V, L, wt, false, target, vp, above, ca)) {
                const u64 q = Weigh::q(wt.w(vp));
                v = vp;
                ties = (target - above + q - 1) / q;
            }
        }
    }
    // kept mass of each wave's part
    u64 sum = 0;
    unsigned eq = 0;
    const u64 qv = v == kNegInf ? 0 : Weigh::q(wt.w(v)) * (u64)(wt.w(v) >= floor_w);
    auto kept_above = [&](float l) {
        const float w = wt.w(l);
        return l > v && w >= floor_w ? Weigh::q(w) : 0u;
    };
    visit<T, VEC>(row, V, L, [&](int64_t, const float (&l)[kVec<T>]) {
#pragma unroll
        for (int e = 0; e < kVec<T>; ++e) {
            sum += kept_above(l[e]);
            eq += l[e] == v && v != kNegInf;
        }
    });
    sum = wave_add(sum);
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) eq += __shfl_xor(eq, off, 64);
    __syncthreads();
    if (lane == 0) {
        s.red[wave] = sum;
        s.redc[wave] = eq;
    }
    __syncthreads();
    u64 S = 0, before = 0, eqb = 0, mine = 0, eqmine = 0;
    for (int w = 0; w < kWaves; ++w) {
        const u64 c = s.redc[w], left = ties > eqb ? ties - eqb : 0;
        const u64 add = s.red[w] + qv * std::min(c, left);
        if (w < wave) before += add;
        if (w == wave) {
            mine = add;
            eqmine = eqb;
        }
        S += add;
        eqb += c;
    }
    const float u = greedy || !(a.u[r] > 0.0f) ? 0.0f : a.u[r];
    const double td = (double)u * (double)S;
    const u64 target = td >= (double)S ? S - 1 : (u64)td;
    if (target < before || target >= before + mine) return;
    // this wave's part holds the token: block by block, then lane by lane
    u64 run = before, run_eq = eqmine;
    const int64_t end = std::min(V, (wave + 1) * L);
    for (int64_t i = wave * L; i < end; i += 64 * kVec<T>) {
        float l[kVec<T>];
        load_logits<T, VEC>(row, i + lane * kVec<T>, V, l);
        u64 ps = 0;
        unsigned pe = 0;
#pragma unroll
        for (int e = 0; e < kVec<T>; ++e) {
            ps += kept_above(l[e]);
            pe += l[e] == v && v != kNegInf;
        }
        u64 is = ps;
        unsigned ie = pe;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const u64 os = __shfl_up(is, off, 64);
            const unsigned oe = __shfl_up(ie, off, 64);
            if (lane >= off) {
                is += os;
                ie += oe;
            }
        }
        auto kept_eq = [&](u64 from, u64 count) {      // of `count` ties after `from` earlier ones
            return from >= ties ? 0ull : std::min(count, ties - from);
        };
        const u64 total = __shfl(is, 63, 64), totale = __shfl(ie, 63, 64);
        const u64 block = total + qv * kept_eq(run_eq, totale);
        if (target < run + block) {
            u64 at = run + is - ps + qv * kept_eq(run_eq, ie - pe);
            u64 ne = run_eq + ie - pe;
#pragma unroll
            for (int e = 0; e < kVec<T>; ++e) {
                u64 add = kept_above(l[e]);
                if (l[e] == v && v != kNegInf) {
                    if (ne < ties) add += qv;
                    ++ne;
                }
                if (target >= at && target < at + add) a.tokens[r] = i + lane * kVec<T> + e;
                at += add;
            }
            return;
        }
        run += block;
        run_eq += totale;
    }
}

size_t sample_workspace_bytes(const SampleArgs&) { return 0; }

template <typename T>
static void launch_rows(const SampleArgs& a, hipStream_t st) {
    const bool vec = reinterpret_cast<uintptr_t>(a.logits) % 16 == 0 && a.ld * sizeof(T) % 16 == 0;
    const int64_t L = round_up((a.vocab + kWaves - 1) / kWaves, 64 * kVec<T>);
    auto* kern = vec ? k_sample_row<T, true> : k_sample_row<T, false>;
    hipLaunchKernelGGL(kern, dim3((unsigned)a.rows), dim3(kThreads), 0, st, a, L);
}

hipError_t launch_sample(const SampleArgs& a, Workspace&, hipStream_t st) {
    KernelTimer t("sample_row", st);
    if (a.prec == P32) launch_rows<float>(a, st);
    else if (a.prec == P16) launch_rows<half_t>(a, st);
    else launch_rows<bhalf_t>(a, st);
    return hipGetLastError();
}

}  // namespace lrc
