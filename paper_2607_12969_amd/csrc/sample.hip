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
// v, and the first r of those equal to v.
//
// One workgroup of 16 waves per row, wave w the w-th part of it.  The vector units
// bound it (131072 logits: 0.9 us per instruction and element on one compute
// unit), so a row is passed as few times as its filters allow, in loops short
// enough to stay in the instruction cache (a row held in registers, its passes
// unrolled, ran three times slower), with the row coming from L2 after the first
// pass:
//   top-k        maximum; counts over 2048 bins of z in (-32, 0]; the tokens down
//                to the bin that holds the cut go, in index order, to a list in
//                LDS, where the rest happens;
//   top-p alone  maximum; masses over the bins; the values in the bin of the cut
//                to LDS, where v and r are found; kept mass of each part; the draw
//                inside one part;
//   neither      maximum; kept mass; draw.
// Inside a bin, v comes from ranking its values one against all, or, above kRanked of
// them, from histograms over their bits.  What does not
// fit its list (thousands of equal logits, say), and rows with an infinite
// maximum, find v by histograms over the row itself.
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
    // every logit of this wave's part
    template <typename F> __device__ __forceinline__ void each(F&& f) const {
        const int wave = threadIdx.x >> 6;
        visit(begin(wave), begin(wave + 1), [&](unsigned, const uint4v_t& v) {
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
            }
        }
        __syncthreads();
        const Cut cut{of_key(s.kmin), s.before, s.beforec};
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
    return Cut{of_key(hi), before, beforec};
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

// Any filters, all passes over the row.
template <typename T, typename W>
__device__ __noinline__ void sample_any(Shared& s, Row<T> row, W wt, int64_t k, float p, float floor_w, float u,
                                        int64_t* token) {
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
    draw_row(s, row, kept, u, token);
}

// The tokens of this wave's part down to bin `last`, in index order, to its list in
// LDS; their number, which may pass the list's kPart entries.
template <typename T>
__device__ __forceinline__ int gather_down_to(Shared& s, const Row<T>& row, const Weigh& wt, int last) {
    constexpr int E = kVec<T>;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int n = 0;
    row.visit(row.begin(wave), row.begin(wave + 1), [&](unsigned i, const uint4v_t& v) {
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

// top-k, top-p, min-p and the draw over the waves' lists (n entries of this wave),
// which hold every token down to the bin of the k-th (bin < 0: every token that
// weighs anything).
__device__ __forceinline__ void finish_topk(Shared& s, Kept<Weigh>& kept, int64_t k, int bin, unsigned beforec, int n,
                                            bool topp, float p, float u, int64_t* token) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const Weigh wt = kept.wt;
    u64 before;
    const List list{s.lv, wave * kPart + lane, wave * kPart + n, 64};
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

template <typename T>
__global__ __launch_bounds__(kThreads) void k_sample_row(SampleArgs a, unsigned L) {
    __shared__ Shared s;
    constexpr int E = kVec<T>;
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const int64_t r = blockIdx.x;
    const unsigned V = (unsigned)a.vocab;
    const Row<T> row{static_cast<const T*>(a.logits) + r * a.ld, V, L, 0};
    const float temp = a.temperature ? a.temperature[r] : 1.0f, u = a.u[r];
    const int64_t k = a.top_k ? a.top_k[r] : 0;
    const float p = a.top_p ? a.top_p[r] : 1.0f, mp = a.min_p ? a.min_p[r] : 0.0f;
    for (int b = t; b < kBins; b += kThreads) {
        s.count[b] = 0;
        s.mass[b] = 0;
    }
    if (t == 0) s.n = 0;

    float M = kNegInf;
    row.each([&](float l) { M = __builtin_fmaxf(M, l); });
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) M = __builtin_fmaxf(M, __shfl_xor(M, off, 64));
    if (lane == 0) s.redf[wave] = M;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) M = __builtin_fmaxf(M, s.redf[w]);
    int64_t* token = a.tokens + r;
    if (M == kNegInf) {          // nothing to draw from
        if (t == 0) *token = -1;
        return;
    }
    if (!(temp > 0.0f)) {        // the first logit equal to the maximum
        unsigned at = V;
        row.visit(row.begin(wave), row.begin(wave + 1), [&](unsigned i, const uint4v_t& v) {
#pragma unroll
            for (int e = E - 1; e >= 0; --e)
                if (elem<T>(v, e) == M) at = std::min(at, i + e);
        });
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) at = std::min(at, __shfl_xor(at, off, 64));
        if (lane == 0) s.redc[wave] = at;
        __syncthreads();
        if (t == 0) {
            for (int w = 1; w < kWaves; ++w) at = std::min(at, s.redc[w]);
            *token = at;
        }
        return;
    }
    const float floor_w = mp > 0.0f ? std::min(mp, 1.0f) : 0.0f;
    if (M == __builtin_inff()) {
        sample_any(s, row, WeighInf{}, k, p, floor_w, u, token);
        return;
    }
    const Weigh wt{M, scale_of(temp)};
    Kept<Weigh> kept{wt, 0.0f, floor_w, 0, 0, true};
    const bool topk = k > 0 && k < (int64_t)V, topp = p < 1.0f;
    int bin;
    u64 before;
    unsigned beforec;
    if (!topk) {
        if (topp) {
            // masses; their total is the mass that p is of
            row.each([&](float l) {
                const float z = wt.z(l);
                if (z >= -31.0f) atomicAdd(&s.mass[bin_of(z)], (u64)Weigh::q(__builtin_amdgcn_exp2f(z)));
            });
            __syncthreads();
            const u64 m = wave_add(s.mass[2 * t] + s.mass[2 * t + 1]);
            if (lane == 0) s.red[wave] = m;
            __syncthreads();
            u64 mass = 0;
            for (int w = 0; w < kWaves; ++w) mass += s.red[w];
            __syncthreads();
            const u64 target = mass_target(p, mass);
            find_bin(s, false, target, bin, before, beforec);
            // the values in that bin, in any order
            row.each([&](float l) {
                const float z = wt.z(l);
                if (z >= -31.0f && bin_of(z) == bin) {
                    const int at = atomicAdd(&s.n, 1);
                    if (at < kWaves * kPart) s.lv[at] = l;
                }
            });
            __syncthreads();
            const int n = s.n;
            if (bin < 0 || n > kWaves * kPart) {
                sample_any(s, row, wt, 0, p, floor_w, u, token);
                return;
            }
            const Cut cut = refine(s, wt, false, target, bin, before, 0u, List{s.lv, t, n, kThreads});
            kept.cut(cut.v, ties_to(target, cut.above, Weigh::q(wt.w(cut.v))));
        }
        draw_row(s, row, kept, u, token);
        return;
    }
    // top-k: counts, then the tokens down to the bin of the k-th, in index order
    row.each([&](float l) {
        const float z = wt.z(l);
        if (z >= -31.0f) atomicAdd(&s.count[bin_of(z)], 1u);
    });
    __syncthreads();
    find_bin(s, true, (u64)k, bin, before, beforec);
    const int last = bin < 0 ? kBins : bin;          // fewer than k tokens weigh anything: all of them
    const int n = gather_down_to(s, row, wt, last);
    if (lane == 0) s.ln[wave] = n;
    __syncthreads();
    bool fits = true;
    for (int w = 0; w < kWaves; ++w) fits &= s.ln[w] <= kPart;
    if (!fits) {
        sample_any(s, row, wt, k, p, floor_w, u, token);
        return;
    }
    finish_topk(s, kept, k, bin, beforec, n, topp, p, u, token);
}

// ---- few rows: a row on several workgroups ------------------------------------
// The passes over a row become launches, each on `parts` workgroups a row (16 L
// logits each), joined through memory; the last one, a workgroup a row, does what
// concerns the lists and draws inside one part.  Four launches cost more than the
// passes save until few rows are long, and from 17 rows the parts of all rows no
// longer fit the 256 compute units at once.  FP32, us, one workgroup a row against
// this, no filter / top-p / top-k / both / a batch of all four:
//     1 x 65536     16 34 22 27       18 31 25 31
//     1 x 131072    22 55 29 34       19 36 25 30
//     8 x 131072    25 56 32 36 55    22 38 29 34 37
//     16 x 98304    20 45 27 32 45    21 37 28 33 37
//     16 x 131072   25 56 32 37 56    22 40 31 36 39
//     24 x 131072   26 57 32 37 56    27 50 39 44 48
//     48 x 131072   25 57 33 38 56    33 63 52 57 61
namespace {

struct SplitBuffers {
    float* max;          // [rows][parts]: maximum ...
    unsigned* first;     // ... and the first index that holds it
    u64* hist;           // [rows][kBins]: counts (top-k) or masses (top-p alone)
    u64* mass;           // [rows][parts]: kept mass (above the bin of the cut)
    int* n;              // [rows][parts]: entries of the list; above kPart: does not fit
    float* lv;           // [rows][parts][kPart]
    unsigned* li;
};

// What a row asks for.
struct Asked {
    float temp, u, p, mp, M;
    int64_t k;
    bool topk, topp;
    __device__ __forceinline__ Asked(const SampleArgs& a, const SplitBuffers& b, int64_t r, int parts) {
        temp = a.temperature ? a.temperature[r] : 1.0f;
        u = a.u[r];
        k = a.top_k ? a.top_k[r] : 0;
        p = a.top_p ? a.top_p[r] : 1.0f;
        mp = a.min_p ? a.min_p[r] : 0.0f;
        topk = k > 0 && k < a.vocab;
        topp = p < 1.0f;
        M = kNegInf;
        for (int q = 0; q < parts; ++q) M = __builtin_fmaxf(M, b.max[r * parts + q]);
    }
    // a draw by weights of finite logits
    __device__ __forceinline__ bool weighs() const { return temp > 0.0f && M != kNegInf && M != __builtin_inff(); }
    __device__ __forceinline__ float floor_w() const { return mp > 0.0f ? std::min(mp, 1.0f) : 0.0f; }
};

}  // namespace

template <typename T>
__global__ __launch_bounds__(kThreads) void k_sample_max(SampleArgs a, SplitBuffers b, unsigned L, int parts) {
    __shared__ float redf[kWaves];
    __shared__ unsigned redc[kWaves];
    constexpr int E = kVec<T>;
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6, part = blockIdx.x;
    const int64_t r = blockIdx.y;
    const Row<T> row{static_cast<const T*>(a.logits) + r * a.ld, (unsigned)a.vocab, L, (unsigned)part * kWaves * L};
    for (int q = part * kThreads + t; q < kBins; q += parts * kThreads) b.hist[r * kBins + q] = 0;
    float M = kNegInf;
    unsigned at = ~0u;
    row.visit(row.begin(wave), row.begin(wave + 1), [&](unsigned i, const uint4v_t& v) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float l = elem<T>(v, e);
            if (l > M) {
                M = l;
                at = i + e;
            }
        }
    });
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) {
        const float m = __shfl_xor(M, off, 64);
        const unsigned o = __shfl_xor(at, off, 64);
        if (m > M || (m == M && o < at)) {
            M = m;
            at = o;
        }
    }
    if (lane == 0) {
        redf[wave] = M;
        redc[wave] = at;
    }
    __syncthreads();
    if (t == 0) {
        for (int w = 1; w < kWaves; ++w)
            if (redf[w] > M) {
                M = redf[w];
                at = redc[w];
            }
        b.max[r * parts + part] = M;
        b.first[r * parts + part] = at;
    }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_sample_hist(SampleArgs a, SplitBuffers b, unsigned L, int parts) {
    __shared__ u64 mass[kBins];
    const int64_t r = blockIdx.y;
    const Asked q(a, b, r, parts);
    if (!q.weighs() || !(q.topk || q.topp)) return;
    const Row<T> row{static_cast<const T*>(a.logits) + r * a.ld, (unsigned)a.vocab, L, blockIdx.x * kWaves * L};
    for (int e = threadIdx.x; e < kBins; e += kThreads) mass[e] = 0;
    __syncthreads();
    const Weigh wt{q.M, scale_of(q.temp)};
    if (q.topk) {
        row.each([&](float l) {
            const float z = wt.z(l);
            if (z >= -31.0f) atomicAdd(reinterpret_cast<unsigned*>(&mass[bin_of(z)]), 1u);
        });
    } else {
        row.each([&](float l) {
            const float z = wt.z(l);
            if (z >= -31.0f) atomicAdd(&mass[bin_of(z)], (u64)Weigh::q(__builtin_amdgcn_exp2f(z)));
        });
    }
    __syncthreads();
    for (int e = threadIdx.x; e < kBins; e += kThreads)
        if (mass[e]) atomicAdd(&b.hist[r * kBins + e], mass[e]);
}

namespace {

// The bin of the cut from the row's histogram.
__device__ __forceinline__ void find_cut_bin(Shared& s, const Asked& q, const u64* hist, u64& target, int& bin, u64& before,
                                             unsigned& beforec) {
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    u64 h[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        h[e] = hist[2 * t + e];
        s.count[2 * t + e] = q.topk ? (unsigned)h[e] : 0u;
        s.mass[2 * t + e] = q.topk ? 0ull : h[e];
    }
    target = (u64)q.k;
    if (!q.topk) {
        const u64 m = wave_add(h[0] + h[1]);
        if (lane == 0) s.red[wave] = m;
        __syncthreads();
        u64 mass = 0;
        for (int w = 0; w < kWaves; ++w) mass += s.red[w];
        target = mass_target(q.p, mass);
    }
    __syncthreads();
    find_bin(s, q.topk, target, bin, before, beforec);
}

}  // namespace

template <typename T>
__global__ __launch_bounds__(kThreads) void k_sample_gather(SampleArgs a, SplitBuffers b, unsigned L, int parts) {
    __shared__ Shared s;
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const int64_t r = blockIdx.y, at = r * parts + blockIdx.x;
    const Asked q(a, b, r, parts);
    if (!q.weighs()) return;
    const Row<T> row{static_cast<const T*>(a.logits) + r * a.ld, (unsigned)a.vocab, L, blockIdx.x * kWaves * L};
    const Weigh wt{q.M, scale_of(q.temp)};
    const float floor_w = q.floor_w();
    u64 target, before;
    int bin = kBins;
    unsigned beforec;
    if (t == 0) s.n = 0;
    if (q.topk || q.topp) find_cut_bin(s, q, b.hist + r * kBins, target, bin, before, beforec);
    if (q.topk) {
        // in index order: the waves' lists one after another
        const int n = gather_down_to(s, row, wt, bin < 0 ? kBins : bin);
        if (lane == 0) s.ln[wave] = n;
        __syncthreads();
        int from = 0, total = 0;
        bool fits = true;
        for (int w = 0; w < kWaves; ++w) {
            if (w < wave) from += s.ln[w];
            total += s.ln[w];
            fits &= s.ln[w] <= kPart;
        }
        fits &= total <= kPart;
        if (fits)
            for (int e = lane; e < n; e += 64) {
                b.lv[at * kPart + from + e] = s.lv[wave * kPart + e];
                b.li[at * kPart + from + e] = s.li[wave * kPart + e];
            }
        if (t == 0) b.n[at] = fits ? total : kPart + 1;
        return;
    }
    // kept mass above the bin of the cut (all, without one); the values in it, in any order
    u64 sum = 0;
    row.each([&](float l) {
        const float z = wt.z(l);
        if (z >= -31.0f) {
            const int zb = bin_of(z);
            if (zb < bin) {
                const float w = wt.w(l);
                sum += w >= floor_w ? Weigh::q(w) : 0u;
            } else if (zb == bin) {
                const int e = atomicAdd(&s.n, 1);
                if (e < kPart) b.lv[at * kPart + e] = l;
            }
        }
    });
    sum = wave_add(sum);
    if (lane == 0) s.red[wave] = sum;
    __syncthreads();
    if (t == 0) {
        u64 m = 0;
        for (int w = 0; w < kWaves; ++w) m += s.red[w];
        b.mass[at] = m;
        b.n[at] = bin < 0 ? kPart + 1 : s.n;
    }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_sample_pick(SampleArgs a, SplitBuffers b, unsigned L, int parts,
                                                          unsigned whole) {
    __shared__ Shared s;
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const int64_t r = blockIdx.x;
    const Asked q(a, b, r, parts);
    int64_t* token = a.tokens + r;
    const Row<T> row{static_cast<const T*>(a.logits) + r * a.ld, (unsigned)a.vocab, whole, 0};
    if (q.M == kNegInf) {
        if (t == 0) *token = -1;
        return;
    }
    if (!(q.temp > 0.0f)) {
        if (t == 0) {
            int at = 0;
            while (b.max[r * parts + at] != q.M) ++at;
            *token = b.first[r * parts + at];
        }
        return;
    }
    const float floor_w = q.floor_w();
    if (q.M == __builtin_inff()) {
        sample_any(s, row, WeighInf{}, q.k, q.p, floor_w, q.u, token);
        return;
    }
    const Weigh wt{q.M, scale_of(q.temp)};
    Kept<Weigh> kept{wt, 0.0f, floor_w, 0, 0, true};
    u64 target = 0, before, run, run_eq, sum = 0;
    int bin = -1, n = 0;
    unsigned beforec, eq = 0;
    if (q.topk || q.topp) {
        bool fits = true;
        for (int w = 0; w < parts; ++w) fits &= b.n[r * parts + w] <= kPart;
        if (!fits) {
            sample_any(s, row, wt, q.k, q.p, floor_w, q.u, token);
            return;
        }
        if (wave < parts) {
            const int64_t at = r * parts + wave;
            n = b.n[at];
            for (int e = lane; e < n; e += 64) {
                s.lv[wave * kPart + e] = b.lv[at * kPart + e];
                s.li[wave * kPart + e] = q.topk ? b.li[at * kPart + e] : 0u;
            }
        }
        find_cut_bin(s, q, b.hist + r * kBins, target, bin, before, beforec);
    }
    if (q.topk) {
        finish_topk(s, kept, q.k, bin, beforec, n, q.topp, q.p, q.u, token);
        return;
    }
    if (q.topp) {
        const List list{s.lv, wave * kPart + lane, wave * kPart + n, 64};
        const Cut cut = refine(s, wt, false, target, bin, before, 0u, list);
        kept.cut(cut.v, ties_to(target, cut.above, Weigh::q(wt.w(cut.v))));
        list.each([&](float l) {
            sum += kept.above(l);
            eq += kept.tied(l);
        });
    }
    if (wave < parts && lane == 0) sum += b.mass[r * parts + wave];
    const int part = find_part<true>(s, kept, sum, eq, q.u, target, run, run_eq);
    if (part < 0) return;
    const unsigned from = (unsigned)part * kWaves * L;
    draw_range(s, row, kept, q.u, target, run, run_eq, from, std::min((unsigned)a.vocab, from + kWaves * L), token);
}

namespace {

// Parts of a row (at most one for each wave of k_sample_pick), or 1: k_sample_row.
struct SamplePlan {
    int parts;
    unsigned L, whole;   // logits of a wave: in a part, in the row
};
SamplePlan plan_sample(const SampleArgs& a) {
    const int64_t block = 64 * (a.prec == P32 ? kVec<float> : kVec<half_t>);
    SamplePlan p{1, 0, (unsigned)round_up((a.vocab + kWaves - 1) / kWaves, block)};
    if (a.rows > 16 || a.vocab < 98304) return p;    // measured above
    const int64_t want = kWaves;                      // 16 rows: 256 workgroups
    p.L = (unsigned)round_up((a.vocab + kWaves * want - 1) / (kWaves * want), block);
    p.parts = (int)((a.vocab + (int64_t)kWaves * p.L - 1) / ((int64_t)kWaves * p.L));
    return p;
}

SplitBuffers split_buffers(const SampleArgs& a, int parts, Workspace& ws) {
    const size_t rp = (size_t)a.rows * parts;
    SplitBuffers b;
    b.max = static_cast<float*>(ws.take(rp * 4));
    b.first = static_cast<unsigned*>(ws.take(rp * 4));
    b.hist = static_cast<u64*>(ws.take((size_t)a.rows * kBins * 8));
    b.mass = static_cast<u64*>(ws.take(rp * 8));
    b.n = static_cast<int*>(ws.take(rp * 4));
    b.lv = static_cast<float*>(ws.take(rp * kPart * 4));
    b.li = static_cast<unsigned*>(ws.take(rp * kPart * 4));
    return b;
}

template <typename T> hipError_t sample_t(const SampleArgs& a, Workspace& ws, hipStream_t st) {
    const SamplePlan p = plan_sample(a);
    const dim3 threads(kThreads);
    if (p.parts == 1)
        return in_panels(a.rows, kRowPanel, [&](int64_t r, int64_t count) {
            auto from = [&](auto* x) { return x ? x + r : x; };
            SampleArgs q = a;
            q.logits = static_cast<const T*>(a.logits) + r * a.ld;
            q.rows = count;
            q.u = a.u + r;
            q.temperature = from(a.temperature);
            q.top_k = from(a.top_k);
            q.top_p = from(a.top_p);
            q.min_p = from(a.min_p);
            q.tokens = a.tokens + r;
            KernelTimer t("sample_row", st);
            hipLaunchKernelGGL(k_sample_row<T>, dim3((unsigned)count), threads, 0, st, q, p.whole);
            return hipGetLastError();
        });
    const dim3 rows((unsigned)a.rows), split(p.parts, (unsigned)a.rows);      // 16 rows at most
    const SplitBuffers b = split_buffers(a, p.parts, ws);
    if (ws.overrun) return hipErrorOutOfMemory;
    KernelTimer t("sample_split", st);
    hipLaunchKernelGGL(k_sample_max<T>, split, threads, 0, st, a, b, p.L, p.parts);
    hipLaunchKernelGGL(k_sample_hist<T>, split, threads, 0, st, a, b, p.L, p.parts);
    hipLaunchKernelGGL(k_sample_gather<T>, split, threads, 0, st, a, b, p.L, p.parts);
    hipLaunchKernelGGL(k_sample_pick<T>, rows, threads, 0, st, a, b, p.L, p.parts, p.whole);
    return hipGetLastError();
}

}  // namespace

size_t sample_workspace_bytes(const SampleArgs& a) {
    const int parts = plan_sample(a).parts;
    if (parts == 1) return 0;
    const size_t rp = (size_t)a.rows * parts;
    return 7 * 256 + rp * (4 + 4 + 8 + 4 + 8 * kPart) + (size_t)a.rows * kBins * 8;
}

hipError_t launch_sample(const SampleArgs& a, Workspace& ws, hipStream_t st) {
    return a.prec == P32 ? sample_t<float>(a, ws, st) : a.prec == P16 ? sample_t<half_t>(a, ws, st) : sample_t<bhalf_t>(a, ws, st);
}

}  // namespace lrc
