// Order and weight of the logits of a row, shared by the draw of a token
// (sample.hip) and the verification of drafted ones (verify.hip): which tokens
// top-k, top-p and min-p keep, and the draw among them.  The rules stand at the top
// of sample.hip.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>

#include "head_device.h"

namespace lrc {

namespace {

typedef unsigned long long u64;
constexpr int kBins = 2048;
constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kPart = 512;               // list entries of a wave
constexpr int kRanked = kThreads;        // values of a bin that are ranked one against all
constexpr float kNegInf = -__builtin_inff();

// Order of binary32 values as unsigned integers (no NaN; -0 counts as 0).
__device__ __forceinline__ unsigned key_of(float x) {
    const unsigned u = __float_as_uint(x + 0.0f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float of_key(unsigned k) {
    return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k);
}

// NaN logits fail every comparison below and weigh (unsigned)NaN = 0.
struct Weigh {
    float M, c;
    __device__ __forceinline__ float z(float l) const { return (l - M) * c; }
    __device__ __forceinline__ float w(float l) const { return __builtin_amdgcn_exp2f(z(l)); }
    static __device__ __forceinline__ unsigned q(float w) { return (unsigned)(w * 2147483648.0f); }
};
// The row whose maximum is +infinity: only that logit weighs.
struct WeighInf {
    __device__ __forceinline__ float z(float l) const { return l == __builtin_inff() ? 0.0f : kNegInf; }
    __device__ __forceinline__ float w(float l) const { return l == __builtin_inff() ? 1.0f : 0.0f; }
};
__device__ __forceinline__ int bin_of(float z) { return (int)(z * -64.0f); }       // z in [-31, 0]

__device__ __forceinline__ float scale_of(float T) {
    return __builtin_fminf(__builtin_fmaxf((1.0f / T) * kLog2e, 1.17549435e-38f), 3.4028234663852886e38f);
}

template <typename X> __device__ __forceinline__ X wave_add(X x) {
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) x += __shfl_xor(x, off, 64);
    return x;
}

struct Shared {
    unsigned count[kBins];
    u64 mass[kBins];
    float lv[kWaves * kPart];            // list: logits ...
    unsigned li[kWaves * kPart];              // ... and, for top-k, indices
    int ln[kWaves];                      // entries of each wave
    int n;                               // entries without order
    u64 red[kWaves];
    unsigned redc[kWaves];
    float redf[kWaves];
    int bin;
    u64 before;
    unsigned beforec;
    unsigned kmin, kmax;
    int nb;                              // values in the bin of the cut
    unsigned eq;                         // values equal to the cut
};

__device__ __forceinline__ void clear_bins(Shared& s) {
    for (int b = threadIdx.x; b < kBins; b += kThreads) {
        s.count[b] = 0;
        s.mass[b] = 0;
    }
    __syncthreads();
}

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

struct Cut {
    float v;             // all logits above v ...
    u64 above;           // ... their mass ...
    unsigned count;      // ... and number
    unsigned eq;         // logits equal to v; 0: not counted
};

// A row in memory, or the 16 L logits of it from `base` on: wave w takes the
// contiguous part [base + w L, base + (w + 1) L) in blocks of 64 vectors, a lane
// kVec consecutive logits of each.
template <typename T> struct Row {
    static constexpr int E = kVec<T>, B = 64 * E;
    const T* row;
    unsigned V, L, base;
    // f(index of the lane's first logit, logits) for the blocks of [begin, end), in
    // order; four loads at a time
    template <typename F> __device__ __forceinline__ void visit(unsigned begin, unsigned end, F&& f) const {
        const unsigned lane = (threadIdx.x & 63) * E;
        unsigned i = begin;
        for (; i + 4 * B <= end; i += 4 * B) {
            uint4v_t v[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] = load16(row + (size_t)i + q * B + lane);
#pragma unroll
            for (int q = 0; q < 4; ++q) f(i + q * B + lane, v[q]);
        }
#pragma unroll 1
        for (; i < end; i += B) f(i + lane, load_row16(row, (int64_t)i + lane, (int64_t)V));
    }
    __device__ __forceinline__ unsigned begin(int wave) const {
        return (unsigned)std::min<uint64_t>(V, (uint64_t)base + (uint64_t)wave * L);
    }
    // the blocks of this wave's part, and every logit of it
    template <typename F> __device__ __forceinline__ void part(F&& f) const {
        const int wave = threadIdx.x >> 6;
        visit(begin(wave), begin(wave + 1), f);
    }
    template <typename F> __device__ __forceinline__ void each(F&& f) const {
        part([&](unsigned, const uint4v_t& v) {
#pragma unroll
            for (int e = 0; e < E; ++e) f(elem<T>(v, e));
        });
    }
};

// Entries begin, begin + step, .. below end of the list in LDS.
struct List {
    const float* lv;
    int begin, end, step;
    template <typename F> __device__ __forceinline__ void each(F&& f) const {
        for (int e = begin; e < end; e += step) f(lv[e]);
    }
};

// The cut inside bin `zb`, with `before` mass and `beforec` tokens in the bins
// above it; `from` holds every logit of the bin, and may hold others.
template <typename W, typename From>
__device__ __noinline__ Cut refine(Shared& s, W wt, bool by_count, u64 target, int zb, u64 before, unsigned beforec,
                                   From from) {
    const int t = threadIdx.x;
    unsigned lo = ~0u, hi = 0u;
    if (t == 0) {
        s.kmin = ~0u;
        s.kmax = 0u;
        s.eq = 0u;
        s.nb = 0;
        s.before = before;
        s.beforec = beforec;
    }
    __syncthreads();
    from.each([&](float l) {
        const float z = wt.z(l);
        if (z >= -31.0f && bin_of(z) == zb) {
            const unsigned k = key_of(l);
            lo = std::min(lo, k);
            hi = std::max(hi, k);
            const int at = atomicAdd(&s.nb, 1);
            if (at < kRanked) s.mass[at] = (u64)k << 32 | Weigh::q(wt.w(l));
        }
    });
    if (lo <= hi) {
        atomicMin(&s.kmin, lo);
        atomicMax(&s.kmax, hi);
    }
    __syncthreads();
    const int n = s.nb;
    if (n <= kRanked) {
        // each value against all: what lies above it and how often it occurs
        if (t < n) {
            const u64 mine = s.mass[t];
            const unsigned key = (unsigned)(mine >> 32);
            u64 above = before;
            unsigned c = beforec, eq = 0;
#pragma unroll 8
            for (int j = 0; j < n; ++j) {
                const u64 o = s.mass[j];
                const unsigned ok = (unsigned)(o >> 32);
                above += ok > key ? (unsigned)o : 0u;
                c += ok > key;
                eq += ok == key;
            }
            const u64 prior = by_count ? c : above, reached = prior + (by_count ? eq : (u64)eq * (unsigned)mine);
            if (prior < target && reached >= target) {      // equal values write the same
                s.kmin = key;
                s.before = above;
                s.beforec = c;
                s.eq = eq;
            }
        }
        __syncthreads();
        const Cut cut{of_key(s.kmin), s.before, s.beforec, s.eq};
        __syncthreads();
        return cut;
    }
    lo = s.kmin;
    hi = s.kmax;
    while (lo < hi) {
        // bins of 2^sh keys from the top
        int sh = 0;
        while (((hi - lo) >> sh) >= (unsigned)kBins) ++sh;
        __syncthreads();
        clear_bins(s);
        from.each([&](float l) {
            const unsigned k = key_of(l);
            if (l == l && k >= lo && k <= hi) {
                const unsigned b = (hi - k) >> sh;
                atomicAdd(&s.count[b], 1u);
                if (!by_count) atomicAdd(&s.mass[b], (u64)Weigh::q(wt.w(l)));
            }
        });
        __syncthreads();
        int bin;
        u64 m;
        unsigned c;
        find_bin(s, by_count, target - (by_count ? beforec : before), bin, m, c);
        if (bin < 0) break;
        before += m;
        beforec += c;
        const unsigned top = hi - ((unsigned)bin << sh);
        lo = std::max(lo, top - ((1u << sh) - 1u));
        hi = top;
    }
    __syncthreads();
    return Cut{of_key(hi), before, beforec, 0u};
}

// Kept tokens: logits above v and the first `ties` equal to v, of weight at least
// floor_w.
template <typename W> struct Kept {
    W wt;
    float v, floor_w;
    u64 ties, qv;        // qv: weight of a tie
    bool all;            // no cut
    __device__ __forceinline__ void cut(float at, u64 t) {
        v = at;
        ties = t;
        all = false;
        const float w = wt.w(at);
        qv = w >= floor_w ? Weigh::q(w) : 0u;
    }
    __device__ __forceinline__ unsigned above(float l) const {
        const float w = wt.w(l);
        return (all || l > v) && w >= floor_w ? Weigh::q(w) : 0u;
    }
    __device__ __forceinline__ bool tied(float l) const { return !all && l == v; }
    // mass of `count` ties after `from` earlier ones
    __device__ __forceinline__ u64 of_ties(u64 from, u64 count) const {
        return from >= ties ? 0ull : qv * std::min(count, ties - from);
    }
};

// Which wave's part holds the draw.  sum, eq: this lane's kept mass above v and
// ties.  FIRST: the target is u times the total; else it is given, with the mass
// and the ties before the parts in run and run_eq.  Leaves in run and run_eq those
// before the part it returns (-1: none).
template <bool FIRST, typename W>
__device__ __forceinline__ int find_part(Shared& s, const Kept<W>& k, u64 sum, unsigned eq, float u, u64& target, u64& run,
                                         u64& run_eq) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    sum = wave_add(sum);
    eq = wave_add(eq);
    __syncthreads();
    if (lane == 0) {
        s.red[wave] = sum;
        s.redc[wave] = eq;
    }
    __syncthreads();
    if (FIRST) {
        u64 S = 0, c = 0;
        for (int w = 0; w < kWaves; ++w) {
            S += s.red[w] + k.of_ties(c, s.redc[w]);
            c += s.redc[w];
        }
        const double td = (double)(u > 0.0f ? u : 0.0f) * (double)S;
        target = td >= (double)S ? S - 1 : (u64)td;
        run = run_eq = 0;
    }
    for (int w = 0; w < kWaves; ++w) {
        const u64 add = s.red[w] + k.of_ties(run_eq, s.redc[w]);
        if (target < run + add) return w;
        run += add;
        run_eq += s.redc[w];
    }
    return -1;
}

// Writes the token if it is among this wave's E logits a lane; else moves run and
// run_eq past them and returns true.
template <int E, typename W>
__device__ __forceinline__ bool find_lane(const Kept<W>& k, u64 target, u64& run, u64& run_eq, const float (&l)[E],
                                          const unsigned (&at)[E], int64_t* token) {
    const int lane = threadIdx.x & 63;
    u64 is = 0;
    unsigned ie = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        is += k.above(l[e]);
        ie += k.tied(l[e]);
    }
    const u64 ps = is;
    const unsigned pe = ie;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const u64 os = __shfl_up(is, off, 64);
        const unsigned oe = __shfl_up(ie, off, 64);
        if (lane >= off) {
            is += os;
            ie += oe;
        }
    }
    const u64 total = __shfl(is, 63, 64), totale = __shfl(ie, 63, 64);
    const u64 block = total + k.of_ties(run_eq, totale);
    if (target >= run + block) {
        run += block;
        run_eq += totale;
        return true;
    }
    u64 ne = run_eq + ie - pe, here = run + is - ps + k.of_ties(run_eq, ie - pe);
#pragma unroll
    for (int e = 0; e < E; ++e) {
        u64 add = k.above(l[e]);
        if (k.tied(l[e])) {
            if (ne < k.ties) add += k.qv;
            ++ne;
        }
        if (target >= here && target < here + add) *token = at[e];
        here += add;
    }
    return false;
}

// The draw inside [from, to), which holds the token: kept mass of 16 parts of it,
// then the part that holds the token.  run, run_eq: kept mass and ties before it.
template <typename T, typename W>
__device__ __forceinline__ void draw_range(Shared& s, const Row<T>& row, const Kept<W>& k, float u, u64 target, u64 run,
                                           u64 run_eq, unsigned from, unsigned to, int64_t* token) {
    constexpr int E = kVec<T>;
    const int wave = threadIdx.x >> 6;
    u64 sum = 0;
    unsigned eq = 0;
    const unsigned sub = ((to - from + kWaves * row.B - 1) / (kWaves * row.B)) * row.B;
    auto sub_begin = [&](int w) { return (unsigned)std::min<uint64_t>(to, (uint64_t)from + (uint64_t)w * sub); };
    row.visit(sub_begin(wave), sub_begin(wave + 1), [&](unsigned, const uint4v_t& v) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            sum += k.above(elem<T>(v, e));
            eq += k.tied(elem<T>(v, e));
        }
    });
    const int w = find_part<false>(s, k, sum, eq, u, target, run, run_eq);
    if (wave != w) return;
    const unsigned lane = (threadIdx.x & 63) * E, end = sub_begin(w + 1);
#pragma unroll 1
    for (unsigned i = sub_begin(w); i < end; i += row.B) {
        const uint4v_t v = load_row16(row.row, (int64_t)i + lane, (int64_t)row.V);
        float l[E];
        unsigned at[E];
#pragma unroll
        for (int e = 0; e < E; ++e) {
            l[e] = elem<T>(v, e);
            at[e] = i + lane + e;
        }
        if (!find_lane<E>(k, target, run, run_eq, l, at, token)) return;
    }
}

// The draw over the row: kept mass of each wave's part, then inside the one that
// holds the token.
template <typename T, typename W>
__device__ __forceinline__ void draw_row(Shared& s, const Row<T>& row, const Kept<W>& k, float u, int64_t* token) {
    u64 target = 0, run, run_eq, sum = 0;
    unsigned eq = 0;
    row.each([&](float l) {
        sum += k.above(l);
        eq += k.tied(l);
    });
    const int part = find_part<true>(s, k, sum, eq, u, target, run, run_eq);
    if (part < 0) return;
    draw_range(s, row, k, u, target, run, run_eq, row.begin(part), row.begin(part + 1), token);
}

// Number of smallest weights that reach `target` from `above`.
__device__ __forceinline__ u64 ties_to(u64 target, u64 above, u64 q) { return (target - above + q - 1) / q; }
__device__ __forceinline__ u64 mass_target(float p, u64 mass) {
    const double P = __builtin_ceil((double)p * (double)mass);
    return P >= 1.0 ? (u64)P : 1ull;
}

// What any filters keep, by passes over the row.
template <typename T, typename W>
__device__ __forceinline__ Kept<W> cut_any(Shared& s, const Row<T>& row, W wt, int64_t k, float p, float floor_w) {
    Kept<W> kept{wt, 0.0f, floor_w, 0, 0, true};
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    Cut cut;
    auto select = [&](bool by_count, u64 target) {
        __syncthreads();
        clear_bins(s);
        row.each([&](float l) {
            const float z = wt.z(l);
            if (z >= -31.0f) {
                atomicAdd(&s.count[bin_of(z)], 1u);
                atomicAdd(&s.mass[bin_of(z)], (u64)Weigh::q(wt.w(l)));
            }
        });
        __syncthreads();
        int bin;
        u64 before;
        unsigned beforec;
        find_bin(s, by_count, target, bin, before, beforec);
        if (bin < 0) return false;
        cut = refine(s, wt, by_count, target, bin, before, beforec, row);
        return true;
    };
    if (k > 0 && k < (int64_t)row.V && select(true, (u64)k)) kept.cut(cut.v, (u64)k - cut.count);
    if (p < 1.0f) {
        // mass of what top-k keeps
        u64 m = 0;
        row.each([&](float l) {
            if (kept.all || l > kept.v) m += Weigh::q(wt.w(l));
        });
        m = wave_add(m);
        __syncthreads();
        if (lane == 0) s.red[wave] = m;
        __syncthreads();
        u64 mass = kept.all ? 0 : kept.ties * Weigh::q(wt.w(kept.v));
        for (int w = 0; w < kWaves; ++w) mass += s.red[w];
        const u64 target = mass_target(p, mass);
        if (select(false, target)) kept.cut(cut.v, ties_to(target, cut.above, Weigh::q(wt.w(cut.v))));
    }
    return kept;
}

// Any filters and the draw, all passes over the row.
template <typename T, typename W>
__device__ __noinline__ void sample_any(Shared& s, Row<T> row, W wt, int64_t k, float p, float floor_w, float u,
                                        int64_t* token) {
    const Kept<W> kept = cut_any(s, row, wt, k, p, floor_w);
    draw_row(s, row, kept, u, token);
}

// The tokens of this wave's part down to bin `last`, in index order, to its list in
// LDS; their number, which may pass the list's kPart entries.
template <typename T, typename R>
__device__ __forceinline__ int gather_down_to(Shared& s, const R& row, const Weigh& wt, int last) {
    constexpr int E = kVec<T>;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int n = 0;
    row.part([&](unsigned i, const uint4v_t& v) {
        unsigned mask = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float z = wt.z(elem<T>(v, e));
            if (z >= -31.0f && bin_of(z) <= last) mask |= 1u << e;
        }
        if (__builtin_amdgcn_ballot_w64(mask != 0)) {
            const int c = __builtin_popcount(mask);
            int at = c;
#pragma unroll
            for (int off = 1; off < 64; off <<= 1) {
                const int o = __shfl_up(at, off, 64);
                if (lane >= off) at += o;
            }
            const int total = __shfl(at, 63, 64);
            at += n - c;
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (mask >> e & 1u) {
                    if (at < kPart) {
                        s.lv[wave * kPart + at] = elem<T>(v, e);
                        s.li[wave * kPart + at] = i + e;
                    }
                    ++at;
                }
            n += total;
        }
    });
    return n;
}

// What top-k and top-p keep of the waves' lists (`list`: this wave's), which hold every
// token down to the bin of the k-th (bin < 0: every token that weighs anything).
__device__ __forceinline__ void cut_list(Shared& s, Kept<Weigh>& kept, const List& list, int64_t k, int bin,
                                         unsigned beforec, bool topp, float p) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const Weigh wt = kept.wt;
    u64 before;
    if (bin >= 0) {
        const Cut cut = refine(s, wt, true, (u64)k, bin, 0, beforec, list);
        kept.cut(cut.v, (u64)k - cut.count);
    }
    if (topp) {
        u64 m = 0;
        list.each([&](float l) {
            if (kept.all || l > kept.v) m += Weigh::q(wt.w(l));
        });
        m = wave_add(m);
        __syncthreads();
        if (lane == 0) s.red[wave] = m;
        clear_bins(s);
        u64 mass = kept.all ? 0 : kept.ties * Weigh::q(wt.w(kept.v));
        for (int w = 0; w < kWaves; ++w) mass += s.red[w];
        const u64 target = mass_target(p, mass);
        list.each([&](float l) { atomicAdd(&s.mass[bin_of(wt.z(l))], (u64)Weigh::q(wt.w(l))); });
        __syncthreads();
        find_bin(s, false, target, bin, before, beforec);
        if (bin >= 0) {
            const Cut cut = refine(s, wt, false, target, bin, before, 0u, list);
            kept.cut(cut.v, ties_to(target, cut.above, Weigh::q(wt.w(cut.v))));
        }
    }
}

// The same, min-p and the draw (n entries of this wave).
__device__ __forceinline__ void finish_topk(Shared& s, Kept<Weigh>& kept, int64_t k, int bin, unsigned beforec, int n,
                                            bool topp, float p, float u, int64_t* token) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const List list{s.lv, wave * kPart + lane, wave * kPart + n, 64};
    cut_list(s, kept, list, k, bin, beforec, topp, p);
    u64 target = 0, run, run_eq, sum = 0;
    unsigned eq = 0;
    list.each([&](float l) {
        sum += kept.above(l);
        eq += kept.tied(l);
    });
    if (find_part<true>(s, kept, sum, eq, u, target, run, run_eq) != wave) return;
    for (int e0 = 0; e0 < n; e0 += 64) {
        const int e = wave * kPart + e0 + lane;
        const float l[1] = {e0 + lane < n ? s.lv[e] : __builtin_nanf("")};
        const unsigned at[1] = {e0 + lane < n ? s.li[e] : 0u};
        if (!find_lane<1>(kept, target, run, run_eq, l, at, token)) return;
    }
}

}  // namespace

}  // namespace lrc
