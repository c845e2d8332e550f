// Drafted tokens checked against the target's logits, from given uniform numbers.
//
// Row j of a request holds the target's logits behind its first j drafts, row j of
// the draft model those that draft j was drawn from.  A token weighs the whole number
// W that the draw of a token gives it under the request's temperature and filters
// (sample_device.h); S is the sum of a row's weights.  Draft t of place j is taken if
//   u_j Wq(t) Sp < Wp(t) Sq          (p target, q draft; without draft logits q is sure of t)
// in binary64, one rounding a product.  At the first draft that is not taken the token
// is drawn from max(P - Q, 0), P = floor(Wp 2^52 / Sp), Q = floor(Wq 2^52 / Sq), or,
// where that is 0 throughout, from Wp; behind the last draft from Wp, which is the draw
// of sample.hip.  All sums are of whole numbers: the result does not depend on how
// the work is split.
//
// The rows come in rounds, a launch each: as many places of every request at first as fill the compute
// units, then twice as many each time; rows behind a rejected draft are left out (48 requests of 5
// drafts: two rounds, 140 of 8: four).  A workgroup passes its row as often as the filters need (maximum;
// bins, cut; sum) and leaves which tokens it keeps, their sum and the draft's weight.  Two more launches
// decide and draw: sums over parts of the row (or two) that a request draws from, then the part that
// holds the token (by one workgroup a request in one launch 48 requests of 65536 took 60 us, 14 + 10 in
// two).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "sample_device.h"

namespace lrc {

namespace {

constexpr int kHeld = 8;                 // vectors of a thread that stay in registers
enum : unsigned { NOTHING = 0, FINITE = 1, INFINITE = 2, GREEDY = 3 };

// What a row keeps: logits above v, and those equal to v up to index `last`, of weight
// floor_w or more.
struct RowLaw {
    float M, c, v, floor_w;
    unsigned last, mode;
    u64 S;       // sum of the weights
    u64 wt;      // weight of the draft of this place
    __device__ __forceinline__ unsigned weight(float l, unsigned i) const {
        if (mode == GREEDY) return i == last ? 1u << 31 : 0u;
        const float w = mode == FINITE ? __builtin_amdgcn_exp2f((l - M) * c) : l == __builtin_inff() ? 1.0f : 0.0f;
        const bool kept = mode != NOTHING && (l > v || (l == v && i <= last)) && w >= floor_w;
        return kept ? Weigh::q(w) : 0u;
    }
};

// Drafts of request r: those before the first that names no token.
__device__ __forceinline__ int drafts_of(const VerifyArgs& a, int64_t r) {
    const int D = (int)a.drafts, lane = threadIdx.x & 63;
    for (int n = 0; n < D; n += 64) {
        const bool none = n + lane < D && (uint64_t)a.draft[r * D + n + lane] >= (uint64_t)a.vocab;
        const u64 m = __builtin_amdgcn_ballot_w64(none);
        if (m) return n + __builtin_ctzll(m);
    }
    return D;
}

// How many of the first `limit` drafts of request r are taken; 64 at a time, a lane each,
// alike in every wave.
__device__ __forceinline__ int taken_of(const VerifyArgs& a, const RowLaw* lp, const RowLaw* lq, int64_t r, int limit) {
    const int lane = threadIdx.x & 63;
    const bool sure = !a.draft_logits;
    const float* u = a.u + r * (a.drafts + 1);
    for (int n = 0; n < limit; n += 64) {
        const int j = n + lane;
        bool no = false;
        if (j < limit) {
            const float x = u[j] > 0.0f ? std::min(u[j], 0.99999994f) : 0.0f;
            const double wq = sure ? 1.0 : (double)lq[j].wt, Sq = sure ? 1.0 : (double)lq[j].S;
            no = !(((double)x * wq) * (double)lp[j].S < (double)lp[j].wt * Sq);
        }
        const u64 m = __builtin_amdgcn_ballot_w64(no);
        if (m) return n + __builtin_ctzll(m);
    }
    return limit;
}

// Index of the entry with which the running number of ties reaches `ties` (>= 1), E
// entries a lane; moves `seen` past a block that does not reach it and returns false.
template <int E>
__device__ __forceinline__ bool find_tie(u64 ties, u64& seen, const bool (&tied)[E], const unsigned (&at)[E], int* out) {
    const int lane = threadIdx.x & 63;
    unsigned c = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) c += tied[e];
    unsigned run = c;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const unsigned o = __shfl_up(run, off, 64);
        if (lane >= off) run += o;
    }
    const unsigned total = __shfl(run, 63, 64);
    if (seen + total < ties) {
        seen += total;
        return false;
    }
    u64 n = seen + run - c;
#pragma unroll
    for (int e = 0; e < E; ++e)
        if (tied[e] && ++n == ties) *out = (int)at[e];
    return true;
}

// A row whose first NV blocks of each wave stay in registers between the passes (what
// 256 compute units pass at once does not fit L2: each further pass met the memory's rate).
template <typename T, int NV> struct HeldRow : Row<T> {
    using Base = Row<T>;
    static constexpr int E = Base::E, B = Base::B;
    uint4v_t v[NV];
    __device__ __forceinline__ HeldRow(const T* row, unsigned V, unsigned L) : Base{row, V, L, 0} {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const unsigned lane = (threadIdx.x & 63) * E, from = this->begin(wave), to = this->begin(wave + 1);
#pragma unroll
        for (int q = 0; q < NV; ++q) {
            v[q] = uint4v_t{kNegInfPair<T>, kNegInfPair<T>, kNegInfPair<T>, kNegInfPair<T>};
            if (from + q * B < to) v[q] = load_row16(row, (int64_t)from + q * B + lane, (int64_t)V);
        }
    }
    template <typename F> __device__ __forceinline__ void part(F&& f) const {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const unsigned lane = (threadIdx.x & 63) * E, from = this->begin(wave), to = this->begin(wave + 1);
#pragma unroll
        for (int q = 0; q < NV; ++q)
            if (from + q * B < to) f(from + q * B + lane, v[q]);
        if (from + NV * B < to) this->visit(from + NV * B, to, f);
    }
    template <typename F> __device__ __forceinline__ void each(F&& f) const {
        part([&](unsigned, const uint4v_t& x) {
#pragma unroll
            for (int e = 0; e < E; ++e) f(elem<T>(x, e));
        });
    }
};

// Kept mass of the waves' sums, and the last tie that is kept.  `walk(f)` calls
// f(tied, at), for each block of this wave's part in order, until it returns true.
template <typename W, typename Walk>
__device__ __forceinline__ void finish_law(Shared& s, const Kept<W>& k, u64 sum, unsigned eq, RowLaw& law, Walk&& walk) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    sum = wave_add(sum);
    eq = wave_add(eq);
    __syncthreads();
    if (lane == 0) {
        s.red[wave] = sum;
        s.redc[wave] = eq;
    }
    if (threadIdx.x == 0) s.bin = -1;
    __syncthreads();
    u64 S = 0, ties = 0, seen = 0;
    int part = -1;
    for (int w = 0; w < kWaves; ++w) {
        S += s.red[w];
        if (part < 0 && !k.all && ties + s.redc[w] >= k.ties) {
            part = w;
            seen = ties;
        }
        ties += s.redc[w];
    }
    law.S = S + (k.all ? 0 : k.of_ties(0, ties));
    law.v = k.all ? kNegInf : k.v;
    law.last = ~0u;
    if (!k.all && ties > k.ties) {
        if (wave == part) walk(k.ties, seen);
        __syncthreads();
        law.last = (unsigned)s.bin;
    }
}

template <typename T, typename R, typename W>
__device__ __forceinline__ void law_of_row(Shared& s, const R& row, const Kept<W>& k, RowLaw& law) {
    constexpr int E = kVec<T>;
    u64 sum = 0;
    unsigned eq = 0;
    row.each([&](float l) {
        sum += k.above(l);
        eq += k.tied(l);
    });
    finish_law(s, k, sum, eq, law, [&](u64 ties, u64 seen) {
        const int wave = threadIdx.x >> 6;
        const unsigned lane = (threadIdx.x & 63) * E, end = row.begin(wave + 1);
#pragma unroll 1
        for (unsigned i = row.begin(wave); i < end; i += row.B) {
            const uint4v_t v = load_row16(row.row, (int64_t)i + lane, (int64_t)row.V);
            bool tied[E];
            unsigned at[E];
#pragma unroll
            for (int e = 0; e < E; ++e) {
                tied[e] = elem<T>(v, e) == k.v && i + lane + e < row.V;
                at[e] = i + lane + e;
            }
            if (find_tie<E>(ties, seen, tied, at, &s.bin)) return;
        }
    });
}

// A cut with ties that are not all kept.
template <typename T>
__device__ __noinline__ void law_ties(Shared& s, Row<T> row, Kept<Weigh> kept, RowLaw* law) {
    RowLaw o = *law;
    law_of_row<T>(s, row, kept, o);
    *law = o;
}

// Rows whose cut the fast paths do not hold: every pass over the row.
template <typename T, typename W>
__device__ __noinline__ void law_any(Shared& s, Row<T> row, W wt, int64_t k, float p, float floor_w, RowLaw* law) {
    RowLaw o = *law;
    const Kept<W> kept = cut_any(s, row, wt, k, p, floor_w);
    law_of_row<T>(s, row, kept, o);
    *law = o;
}

template <typename T, int NV>
__device__ __forceinline__ RowLaw row_law(Shared& s, HeldRow<T, NV>& row, float temp, int64_t k, float p, float mp) {
    constexpr int E = kVec<T>;
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    RowLaw law{kNegInf, 0.0f, kNegInf, 0.0f, ~0u, NOTHING, 0, 0};
    for (int b = t; b < kBins; b += kThreads) {
        s.count[b] = 0;
        s.mass[b] = 0;
    }
    if (t == 0) s.n = 0;
    float M = kNegInf;
    row.each([&](float l) { M = __builtin_fmaxf(M, l); });
    stay(row.v);
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) M = __builtin_fmaxf(M, __shfl_xor(M, off, 64));
    if (lane == 0) s.redf[wave] = M;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) M = __builtin_fmaxf(M, s.redf[w]);
    law.M = M;
    if (M == kNegInf) return law;
    if (!(temp > 0.0f)) {        // the first logit equal to the maximum
        unsigned at = row.V;
        row.part([&](unsigned i, const uint4v_t& v) {
#pragma unroll
            for (int e = E - 1; e >= 0; --e)
                if (elem<T>(v, e) == M) at = std::min(at, i + e);
        });
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) at = std::min(at, (unsigned)__shfl_xor((int)at, off, 64));
        if (lane == 0) s.redc[wave] = at;
        __syncthreads();
        for (int w = 0; w < kWaves; ++w) at = std::min(at, s.redc[w]);
        law.mode = GREEDY;
        law.last = at;
        law.S = 1ull << 31;
        return law;
    }
    law.floor_w = mp > 0.0f ? std::min(mp, 1.0f) : 0.0f;
    if (M == __builtin_inff()) {
        law.mode = INFINITE;
        law_any(s, static_cast<const Row<T>&>(row), WeighInf{}, k, p, law.floor_w, &law);
        return law;
    }
    law.mode = FINITE;
    law.c = scale_of(temp);
    const Weigh wt{M, law.c};
    Kept<Weigh> kept{wt, 0.0f, law.floor_w, 0, 0, true};
    const bool topk = k > 0 && k < (int64_t)row.V, topp = p < 1.0f;
    int bin;
    u64 before;
    unsigned beforec;
    if (!topk) {
        if (topp) {
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
            stay(row.v);
            // the values in that bin, in any order, and the mass that min-p alone keeps
            auto take = [&](float l, float z) {
                if (z >= -31.0f && bin_of(z) == bin) {
                    const int at = atomicAdd(&s.n, 1);
                    if (at < kWaves * kPart) s.lv[at] = l;
                }
            };
            u64 least = 0;
            if (law.floor_w > 0.0f) {
                row.each([&](float l) {
                    const float z = wt.z(l), w = __builtin_amdgcn_exp2f(z);
                    take(l, z);
                    least += w >= law.floor_w ? Weigh::q(w) : 0u;
                });
                least = wave_add(least);
            } else {
                row.each([&](float l) { take(l, wt.z(l)); });
            }
            __syncthreads();
            const int n = s.n;
            if (bin < 0 || n > kWaves * kPart) {
                law_any(s, static_cast<const Row<T>&>(row), wt, 0, p, law.floor_w, &law);
                return law;
            }
            const Cut cut = refine(s, wt, false, target, bin, before, 0u, List{s.lv, t, n, kThreads});
            kept.cut(cut.v, ties_to(target, cut.above, Weigh::q(wt.w(cut.v))));
            if (cut.eq == 0 || cut.eq > kept.ties) {
                law_ties(s, static_cast<const Row<T>&>(row), kept, &law);
                return law;
            }
            law.v = cut.v;
            if (kept.qv) {                   // min-p keeps the cut, and so all above it
                law.S = cut.above + cut.eq * kept.qv;
                return law;
            }
            if (lane == 0) s.red[wave] = least;
            __syncthreads();
            for (int w = 0; w < kWaves; ++w) law.S += s.red[w];
            return law;
        }
        u64 sum = 0;                         // all, or what min-p keeps
        row.each([&](float l) {
            const float w = wt.w(l);
            sum += w >= law.floor_w ? Weigh::q(w) : 0u;
        });
        sum = wave_add(sum);
        if (lane == 0) s.red[wave] = sum;
        __syncthreads();
        for (int w = 0; w < kWaves; ++w) law.S += s.red[w];
        return law;
    }
    // top-k: counts, then the tokens down to the bin of the k-th, in index order
    row.each([&](float l) {
        const float z = wt.z(l);
        if (z >= -31.0f) atomicAdd(&s.count[bin_of(z)], 1u);
    });
    __syncthreads();
    find_bin(s, true, (u64)k, bin, before, beforec);
    stay(row.v);
    const int n = gather_down_to<T>(s, row, wt, bin < 0 ? kBins : bin);
    if (lane == 0) s.ln[wave] = n;
    __syncthreads();
    bool fits = true;
    for (int w = 0; w < kWaves; ++w) fits &= s.ln[w] <= kPart;
    if (!fits) {
        law_any(s, static_cast<const Row<T>&>(row), wt, k, p, law.floor_w, &law);
        return law;
    }
    const List list{s.lv, wave * kPart + lane, wave * kPart + n, 64};
    cut_list(s, kept, list, k, bin, beforec, topp, p);
    u64 sum = 0;
    unsigned eq = 0;
    list.each([&](float l) {
        sum += kept.above(l);
        eq += kept.tied(l);
    });
    finish_law(s, kept, sum, eq, law, [&](u64 ties, u64 seen) {
        for (int e0 = 0; e0 < n; e0 += 64) {
            const int e = wave * kPart + e0 + lane;
            const bool tied[1] = {e0 + lane < n && s.lv[e] == kept.v};
            const unsigned at[1] = {e0 + lane < n ? s.li[e] : 0u};
            if (find_tie<1>(ties, seen, tied, at, &s.bin)) return;
        }
    });
    return law;
}

}  // namespace

// One workgroup a row, for the places [j0, j1): the target's rows of a request, then the
// draft model's.  Rows that its drafts do not reach are left out, and so are all of a request
// that an earlier launch saw reject a draft.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_verify_rows(VerifyArgs a, RowLaw* __restrict__ laws, unsigned L, int j0, int j1) {
    __shared__ Shared s;
    const int D = (int)a.drafts, n = j1 - j0 + (a.draft_logits ? std::min(j1, D) - j0 : 0);
    const int64_t r = blockIdx.x / n;
    const int at = (int)(blockIdx.x % n);
    const bool target = at < j1 - j0;
    const int j = j0 + (target ? at : at - (j1 - j0));
    const int have = drafts_of(a, r);
    if (j > have || (!target && j == have)) return;
    RowLaw* mine = laws + r * (D + 1 + (a.draft_logits ? D : 0));
    if (j0 > 0 && taken_of(a, mine, mine + D + 1, r, j0) < j0) return;
    const T* logits = target ? static_cast<const T*>(a.logits) + r * a.lr + j * a.ld
                             : static_cast<const T*>(a.draft_logits) + r * a.lrq + j * a.ldq;
    HeldRow<T, kHeld> row(logits, (unsigned)a.vocab, L);
    RowLaw law = row_law(s, row, a.temperature ? a.temperature[r] : 1.0f, a.top_k ? a.top_k[r] : 0,
                         a.top_p ? a.top_p[r] : 1.0f, a.min_p ? a.min_p[r] : 0.0f);
    if (threadIdx.x == 0) {
        if (j < have) {
            const int64_t d = a.draft[r * a.drafts + j];
            law.wt = law.weight((float)logits[d], (unsigned)d);
        }
        mine[target ? j : D + 1 + j] = law;
    }
}

namespace {

// What a request draws its token from: the row behind its accepted drafts, or what that
// row has above the draft model's.
template <typename T> struct Source {
    RowLaw p, q;
    const T *prow, *qrow;
    double ap, aq;
    unsigned drafted, V;
    int taken;
    bool rest, sure;
    // weight in the row itself, and above the draft's
    __device__ __forceinline__ void weights(float lp, float lq, unsigned i, u64& plain, u64& above) const {
        const unsigned w = p.weight(lp, i);
        plain = w;
        above = 0;
        if (rest) {
            const u64 P = (u64)((double)w * ap);
            const u64 Q = sure ? (i == drafted ? 1ull << 52 : 0ull) : (u64)((double)q.weight(lq, i) * aq);
            above = P > Q ? P - Q : 0ull;
        }
    }
    __device__ __forceinline__ uint4v_t load_p(unsigned at) const { return load_row16(prow, (int64_t)at, (int64_t)V); }
    __device__ __forceinline__ uint4v_t load_q(unsigned at) const {
        return rest && !sure ? load_row16(qrow, (int64_t)at, (int64_t)V) : uint4v_t{0, 0, 0, 0};
    }
    __device__ __forceinline__ Source(const VerifyArgs& a, const RowLaw* laws, int64_t r) {
        const int64_t D = a.drafts;
        sure = !a.draft_logits;
        const RowLaw* lp = laws + r * (D + 1 + (sure ? 0 : D));
        const RowLaw* lq = lp + D + 1;
        const int have = drafts_of(a, r);
        taken = taken_of(a, lp, lq, r, have);
        rest = taken < have;
        p = lp[taken];
        q = rest && !sure ? lq[taken] : RowLaw{0.0f, 0.0f, 0.0f, 0.0f, 0u, NOTHING, 0, 0};
        drafted = rest ? (unsigned)a.draft[r * D + taken] : 0u;
        ap = 4503599627370496.0 / (double)p.S;
        aq = q.S ? 4503599627370496.0 / (double)q.S : 0.0;
        V = (unsigned)a.vocab;
        prow = static_cast<const T*>(a.logits) + r * a.lr + taken * a.ld;
        qrow = rest && !sure ? static_cast<const T*>(a.draft_logits) + r * a.lrq + taken * a.ldq : prow;
    }
};

}  // namespace

// Sums of a request's weights over its parts of `size` tokens: [request][part][2], of the row
// itself and of what it has above the draft model's.
template <typename T>
__global__ __launch_bounds__(256) void k_verify_sums(VerifyArgs a, const RowLaw* __restrict__ laws, u64* __restrict__ sums,
                                                     unsigned size) {
    constexpr int E = kVec<T>, B = 256 * E;
    __shared__ u64 red[4][2];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t r = blockIdx.y;
    const Source<T> s(a, laws, r);
    u64 plain = 0, above = 0;
    if (s.p.mode != NOTHING) {
        const unsigned from = blockIdx.x * size, to = (unsigned)std::min<uint64_t>(s.V, (uint64_t)from + size);
#pragma unroll 2
        for (unsigned i = from; i < to; i += B) {
            const unsigned at = i + threadIdx.x * E;
            const uint4v_t v = s.load_p(at), w = s.load_q(at);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                u64 x, y;
                s.weights(elem<T>(v, e), elem<T>(w, e), at + e, x, y);
                plain += x;
                above += y;
            }
        }
    }
    plain = wave_add(plain);
    above = wave_add(above);
    if (lane == 0) {
        red[wave][0] = plain;
        red[wave][1] = above;
    }
    __syncthreads();
    if (threadIdx.x < 2) {
        u64 t = 0;
        for (int w = 0; w < 4; ++w) t += red[w][threadIdx.x];
        sums[(r * gridDim.x + blockIdx.x) * 2 + threadIdx.x] = t;
    }
}

// One workgroup a request: its accepted drafts, and the token from the part that holds it.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_verify_draw(VerifyArgs a, const RowLaw* __restrict__ laws, const u64* __restrict__ sums,
                                                          int parts, unsigned size) {
    constexpr int E = kVec<T>, B = 64 * E;
    __shared__ u64 red[kWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t r = blockIdx.x, D = a.drafts;
    const Source<T> s(a, laws, r);
    const int c = s.taken;
    int64_t* out = a.tokens + r * (D + 1);
    for (int64_t j = threadIdx.x; j <= D; j += kThreads)
        if (j != c) out[j] = j < c ? a.draft[r * D + j] : -1;
    if (threadIdx.x == 0 && a.accepted) a.accepted[r] = c;
    // 64 parts at most: a lane each
    const u64* mine = sums + r * parts * 2;
    const u64 plain = lane < parts ? mine[2 * lane] : 0, above = lane < parts ? mine[2 * lane + 1] : 0;
    const u64 all = wave_add(above);
    const bool rest = all != 0;        // nothing above the draft model's: the target's own
    u64 run = rest ? above : plain;
    const u64 S = rest ? all : wave_add(plain);
    if (!S) {
        if (threadIdx.x == 0) out[c] = -1;
        return;
    }
    const float x = a.u[r * (D + 1) + D];
    const double td = (double)(x > 0.0f ? x : 0.0f) * (double)S;
    const u64 target = td >= (double)S ? S - 1 : (u64)td;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const u64 o = __shfl_up(run, off, 64);
        if (lane >= off) run += o;
    }
    const int part = __builtin_ctzll(__builtin_amdgcn_ballot_w64(target < run));
    u64 before = part ? __shfl(run, part - 1, 64) : 0;
    // inside the part: the sum of each wave's share, then the share that holds the token
    const unsigned from = part * size, to = (unsigned)std::min<uint64_t>(s.V, (uint64_t)from + size);
    const unsigned sub = ((to - from + kWaves * B - 1) / (kWaves * B)) * B;
    auto bound = [&](int w) { return (unsigned)std::min<uint64_t>(to, (uint64_t)from + (uint64_t)w * sub); };
    auto share = [&](unsigned at, u64 (&h)[E]) {
        const uint4v_t v = s.load_p(at), w = s.load_q(at);
        u64 t = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            u64 x, y;
            s.weights(elem<T>(v, e), elem<T>(w, e), at + e, x, y);
            h[e] = rest ? y : x;
            t += h[e];
        }
        return t;
    };
    u64 sum = 0, h[E];
#pragma unroll 1
    for (unsigned i = bound(wave); i < bound(wave + 1); i += B) sum += share(i + lane * E, h);
    sum = wave_add(sum);
    if (lane == 0) red[wave] = sum;
    __syncthreads();
    int w = 0;
    for (; w < kWaves - 1 && target >= before + red[w]; ++w) before += red[w];
    if (wave != w) return;
#pragma unroll 1
    for (unsigned i = bound(w); i < bound(w + 1); i += B) {
        const u64 own = share(i + lane * E, h);
        u64 scan = own;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const u64 o = __shfl_up(scan, off, 64);
            if (lane >= off) scan += o;
        }
        const u64 block = __shfl(scan, 63, 64);
        if (target >= before + block) {
            before += block;
            continue;
        }
        u64 here = before + scan - own;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            if (target >= here && target < here + h[e]) out[c] = i + lane * E + e;
            here += h[e];
        }
        return;
    }
}

namespace {

int64_t rows_per(const VerifyArgs& a) { return a.drafts + 1 + (a.draft_logits ? a.drafts : 0); }
int64_t requests_panel(const VerifyArgs& a) { return std::max<int64_t>(1, kRowPanel / rows_per(a)); }

// Parts of a row that the sums are taken of: about 1024 workgroups, 64 a row at most (a
// lane each of the next launch), whole steps of 256 vectors.
unsigned part_size(const VerifyArgs& a, int64_t requests, int e) {
    const int64_t step = 256 * (16 / e), steps = (a.vocab + step - 1) / step;
    const int64_t parts = std::min<int64_t>({64, steps, std::max<int64_t>(1, 1024 / requests)});
    return (unsigned)((steps + parts - 1) / parts * step);
}

template <typename T> hipError_t verify_t(const VerifyArgs& a, Workspace& ws, hipStream_t st) {
    const int64_t panel = requests_panel(a), most = std::min(a.requests, panel);
    RowLaw* laws = static_cast<RowLaw*>(ws.take((size_t)most * rows_per(a) * sizeof(RowLaw)));
    u64* sums = static_cast<u64*>(ws.take((size_t)most * 64 * 2 * sizeof(u64)));
    if (ws.overrun) return hipErrorOutOfMemory;
    const unsigned L = (unsigned)round_up((a.vocab + kWaves - 1) / kWaves, 64 * kVec<T>);
    return in_panels(a.requests, panel, [&](int64_t r, int64_t count) {
        auto from = [&](auto* x, int64_t per) { return x ? x + r * per : x; };
        VerifyArgs q = a;
        q.requests = count;
        q.logits = static_cast<const T*>(a.logits) + r * a.lr;
        q.draft_logits = a.draft_logits ? static_cast<const T*>(a.draft_logits) + r * a.lrq : nullptr;
        q.draft = from(a.draft, a.drafts);
        q.u = a.u + r * (a.drafts + 1);
        q.temperature = from(a.temperature, 1);
        q.top_k = from(a.top_k, 1);
        q.top_p = from(a.top_p, 1);
        q.min_p = from(a.min_p, 1);
        q.tokens = a.tokens + r * (a.drafts + 1);
        q.accepted = from(a.accepted, 1);
        // A round of one row a compute unit first, then twice as many places each time: rows
        // behind a rejected draft need not be looked at.  48 requests, 5 drafts, 65536 tokens,
        // top-p, rejections at random: 122 us in one launch of 528 rows, 2 x 38 in two.
        for (int64_t j0 = 0, some = std::max<int64_t>(1, 128 / count); j0 <= a.drafts; j0 += some, some *= 2) {
            if (j0) some = std::min(some, a.drafts + 1 - j0);
            const int64_t j1 = std::min(a.drafts + 1, j0 + some), n = j1 - j0 + (a.draft_logits ? std::min(j1, a.drafts) - j0 : 0);
            KernelTimer t("verify_rows", st);
            hipLaunchKernelGGL(k_verify_rows<T>, dim3((unsigned)(count * n)), dim3(kThreads), 0, st, q, laws, L, (int)j0, (int)j1);
        }
        const unsigned size = part_size(a, count, sizeof(T));
        const int parts = (int)((a.vocab + size - 1) / size);
        // the grid's second dimension ends at 65535
        return in_panels(count, 65535, [&](int64_t first, int64_t some) {
            VerifyArgs v = q;
            v.requests = some;
            v.logits = static_cast<const T*>(q.logits) + first * a.lr;
            v.draft_logits = a.draft_logits ? static_cast<const T*>(q.draft_logits) + first * a.lrq : nullptr;
            v.draft = q.draft ? q.draft + first * a.drafts : nullptr;
            v.u = q.u + first * (a.drafts + 1);
            v.tokens = q.tokens + first * (a.drafts + 1);
            v.accepted = q.accepted ? q.accepted + first : nullptr;
            const RowLaw* l = laws + first * rows_per(a);
            {
                KernelTimer t("verify_sums", st);
                hipLaunchKernelGGL(k_verify_sums<T>, dim3(parts, (unsigned)some), dim3(256), 0, st, v, l, sums, size);
            }
            KernelTimer t("verify_draw", st);
            hipLaunchKernelGGL(k_verify_draw<T>, dim3((unsigned)some), dim3(kThreads), 0, st, v, l, sums, parts, size);
            return hipGetLastError();
        });
    });
}

}  // namespace

size_t verify_workspace_bytes(const VerifyArgs& a) {
    return (size_t)std::min(a.requests, requests_panel(a)) * (rows_per(a) * sizeof(RowLaw) + 64 * 2 * sizeof(u64)) + 512;
}

hipError_t launch_verify(const VerifyArgs& a, Workspace& ws, hipStream_t st) {
    return a.prec == P32 ? verify_t<float>(a, ws, st) : a.prec == P16 ? verify_t<half_t>(a, ws, st) : verify_t<bhalf_t>(a, ws, st);
}

}  // namespace lrc
