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
// Two launches.  The first, one workgroup a row, passes each row as often as its
// filters need (maximum; bins, cut; sum) and leaves which tokens it keeps, their sum
// and the draft's weight; the vector units bound it, as they do the draw.  The second,
// one workgroup a request, decides and draws from one row or two.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "sample_device.h"

namespace lrc {

namespace {

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

template <typename T, typename W>
__device__ __forceinline__ void law_of_row(Shared& s, const Row<T>& row, const Kept<W>& k, RowLaw& law) {
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

// Rows whose cut the fast paths do not hold: every pass over the row.
template <typename T, typename W>
__device__ __noinline__ void law_any(Shared& s, Row<T> row, W wt, int64_t k, float p, float floor_w, RowLaw* law) {
    RowLaw o = *law;
    const Kept<W> kept = cut_any(s, row, wt, k, p, floor_w);
    law_of_row(s, row, kept, o);
    *law = o;
}

template <typename T>
__device__ __forceinline__ RowLaw row_law(Shared& s, const Row<T>& row, float temp, int64_t k, float p, float mp) {
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
        row.visit(row.begin(wave), row.begin(wave + 1), [&](unsigned i, const uint4v_t& v) {
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
        law_any(s, row, WeighInf{}, k, p, law.floor_w, &law);
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
                law_any(s, row, wt, 0, p, law.floor_w, &law);
                return law;
            }
            const Cut cut = refine(s, wt, false, target, bin, before, 0u, List{s.lv, t, n, kThreads});
            kept.cut(cut.v, ties_to(target, cut.above, Weigh::q(wt.w(cut.v))));
        }
        law_of_row(s, row, kept, law);
        return law;
    }
    // top-k: counts, then the tokens down to the bin of the k-th, in index order
    row.each([&](float l) {
        const float z = wt.z(l);
        if (z >= -31.0f) atomicAdd(&s.count[bin_of(z)], 1u);
    });
    __syncthreads();
    find_bin(s, true, (u64)k, bin, before, beforec);
    const int n = gather_down_to(s, row, wt, bin < 0 ? kBins : bin);
    if (lane == 0) s.ln[wave] = n;
    __syncthreads();
    bool fits = true;
    for (int w = 0; w < kWaves; ++w) fits &= s.ln[w] <= kPart;
    if (!fits) {
        law_any(s, row, wt, k, p, law.floor_w, &law);
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

// One workgroup a row: request r's rows are the target's 0 .. drafts, then the draft
// model's 0 .. drafts - 1.  Rows that its drafts do not reach are left out.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_verify_rows(VerifyArgs a, RowLaw* __restrict__ laws, unsigned L) {
    __shared__ Shared s;
    const int per = (int)a.drafts + 1 + (a.draft_logits ? (int)a.drafts : 0);
    const int64_t r = blockIdx.x / per;
    const int at = (int)(blockIdx.x % per);
    const bool target = at <= a.drafts;
    const int j = target ? at : at - (int)a.drafts - 1;
    const int have = drafts_of(a, r);
    if (j > have || (!target && j == have)) return;
    const T* logits = target ? static_cast<const T*>(a.logits) + r * a.lr + j * a.ld
                             : static_cast<const T*>(a.draft_logits) + r * a.lrq + j * a.ldq;
    const Row<T> row{logits, (unsigned)a.vocab, L, 0};
    RowLaw law = row_law(s, row, a.temperature ? a.temperature[r] : 1.0f, a.top_k ? a.top_k[r] : 0,
                         a.top_p ? a.top_p[r] : 1.0f, a.min_p ? a.min_p[r] : 0.0f);
    if (threadIdx.x == 0) {
        if (j < have) {
            const int64_t d = a.draft[r * a.drafts + j];
            law.wt = law.weight((float)logits[d], (unsigned)d);
        }
        laws[blockIdx.x] = law;
    }
}

// One workgroup a request: how many drafts are taken, and the token behind them.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_verify_draw(VerifyArgs a, const RowLaw* __restrict__ laws, unsigned L) {
    constexpr int E = kVec<T>, B = 64 * E;
    __shared__ u64 red[kWaves];
    __shared__ int taken;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t r = blockIdx.x, D = a.drafts;
    const int per = (int)D + 1 + (a.draft_logits ? (int)D : 0);
    const RowLaw* lp = laws + r * per;
    const RowLaw* lq = lp + D + 1;
    const int have = drafts_of(a, r);
    const float* u = a.u + r * (D + 1);
    if (wave == 0) {
        int n = 0;
        for (; n < have; n += 64) {
            const int j = n + lane;
            bool no = false;
            if (j < have) {
                const float x = u[j] > 0.0f ? std::min(u[j], 0.99999994f) : 0.0f;
                const double q = a.draft_logits ? (double)lq[j].wt : 1.0, Sq = a.draft_logits ? (double)lq[j].S : 1.0;
                no = !(((double)x * q) * (double)lp[j].S < (double)lp[j].wt * Sq);
            }
            const u64 m = __builtin_amdgcn_ballot_w64(no);
            if (m) {
                n += __builtin_ctzll(m);
                break;
            }
        }
        if (lane == 0) taken = std::min(n, have);
    }
    __syncthreads();
    const int c = taken;
    int64_t* out = a.tokens + r * (D + 1);
    for (int64_t j = threadIdx.x; j <= D; j += kThreads)
        if (j != c) out[j] = j < c ? a.draft[r * D + j] : -1;
    if (threadIdx.x == 0 && a.accepted) a.accepted[r] = c;
    const RowLaw p = lp[c];
    if (p.mode == NOTHING) {
        if (threadIdx.x == 0) out[c] = -1;
        return;
    }
    bool rest = c < have;
    const bool sure = !a.draft_logits;
    const RowLaw q = rest && !sure ? lq[c] : RowLaw{0.0f, 0.0f, 0.0f, 0.0f, 0u, NOTHING, 0, 0};
    const unsigned drafted = rest ? (unsigned)a.draft[r * D + c] : 0u;
    const double ap = 4503599627370496.0 / (double)p.S, aq = q.S ? 4503599627370496.0 / (double)q.S : 0.0;
    const T* prow = static_cast<const T*>(a.logits) + r * a.lr + c * a.ld;
    const T* qrow = rest && !sure ? static_cast<const T*>(a.draft_logits) + r * a.lrq + c * a.ldq : prow;
    auto share = [&](float l, float lq_, unsigned i) -> u64 {
        const unsigned w = p.weight(l, i);
        if (!rest) return w;
        const u64 P = (u64)((double)w * ap);
        const u64 Q = sure ? (i == drafted ? 1ull << 52 : 0ull) : (u64)((double)q.weight(lq_, i) * aq);
        return P > Q ? P - Q : 0ull;
    };
    const unsigned V = (unsigned)a.vocab;
    // this lane's sum over the blocks of [begin, end)
    auto sum_of = [&](unsigned begin, unsigned end) {
        u64 sum = 0;
#pragma unroll 1
        for (unsigned i = begin; i < end; i += B) {
            const unsigned at = i + lane * E;
            const uint4v_t v = load_row16(prow, (int64_t)at, (int64_t)V), w = load_row16(qrow, (int64_t)at, (int64_t)V);
#pragma unroll
            for (int e = 0; e < E; ++e) sum += share(elem<T>(v, e), elem<T>(w, e), at + e);
        }
        return wave_add(sum);
    };
    auto bound = [&](unsigned from, unsigned step, int w, unsigned to) {
        return (unsigned)std::min<uint64_t>(to, (uint64_t)from + (uint64_t)w * step);
    };
    // which of the waves' sums holds `target`; run: what lies before it
    auto find = [&](u64 target, u64& run) {
        for (int w = 0; w < kWaves; ++w) {
            if (target < run + red[w]) return w;
            run += red[w];
        }
        return -1;
    };
    u64 S = 0;
    for (;;) {
        const u64 sum = sum_of(bound(0, L, wave, V), bound(0, L, wave + 1, V));
        if (lane == 0) red[wave] = sum;
        __syncthreads();
        for (int w = 0; w < kWaves; ++w) S += red[w];
        if (S || !rest) break;
        rest = false;                  // nothing of the target above the draft: the target itself
        __syncthreads();
    }
    if (!S) {
        if (threadIdx.x == 0) out[c] = -1;
        return;
    }
    const float x = u[D];
    const double td = (double)(x > 0.0f ? x : 0.0f) * (double)S;
    const u64 target = td >= (double)S ? S - 1 : (u64)td;
    u64 run = 0;
    const int part = find(target, run);
    if (part < 0) return;
    // the same inside that part
    const unsigned from = bound(0, L, part, V), to = bound(0, L, part + 1, V);
    const unsigned sub = ((to - from + kWaves * B - 1) / (kWaves * B)) * B;
    __syncthreads();
    const u64 sum = sum_of(bound(from, sub, wave, to), bound(from, sub, wave + 1, to));
    if (lane == 0) red[wave] = sum;
    __syncthreads();
    const int w = find(target, run);
    if (wave != w) return;
    const unsigned end = bound(from, sub, w + 1, to);
#pragma unroll 1
    for (unsigned i = bound(from, sub, w, to); i < end; i += B) {
        const unsigned at = i + lane * E;
        const uint4v_t v = load_row16(prow, (int64_t)at, (int64_t)V), o = load_row16(qrow, (int64_t)at, (int64_t)V);
        u64 h[E], mine = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            h[e] = share(elem<T>(v, e), elem<T>(o, e), at + e);
            mine += h[e];
        }
        u64 scan = mine;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const u64 b = __shfl_up(scan, off, 64);
            if (lane >= off) scan += b;
        }
        const u64 block = __shfl(scan, 63, 64);
        if (target >= run + block) {
            run += block;
            continue;
        }
        u64 here = run + scan - mine;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            if (target >= here && target < here + h[e]) out[c] = at + e;
            here += h[e];
        }
        return;
    }
}

namespace {

int64_t rows_per(const VerifyArgs& a) { return a.drafts + 1 + (a.draft_logits ? a.drafts : 0); }
int64_t requests_panel(const VerifyArgs& a) { return std::max<int64_t>(1, kRowPanel / rows_per(a)); }

template <typename T> hipError_t verify_t(const VerifyArgs& a, Workspace& ws, hipStream_t st) {
    const int64_t panel = requests_panel(a);
    RowLaw* laws = static_cast<RowLaw*>(ws.take((size_t)std::min(a.requests, panel) * rows_per(a) * sizeof(RowLaw)));
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
        {
            KernelTimer t("verify_rows", st);
            hipLaunchKernelGGL(k_verify_rows<T>, dim3((unsigned)(count * rows_per(a))), dim3(kThreads), 0, st, q, laws, L);
        }
        KernelTimer t("verify_draw", st);
        hipLaunchKernelGGL(k_verify_draw<T>, dim3((unsigned)count), dim3(kThreads), 0, st, q, laws, L);
        return hipGetLastError();
    });
}

}  // namespace

size_t verify_workspace_bytes(const VerifyArgs& a) {
    return (size_t)std::min(a.requests, requests_panel(a)) * rows_per(a) * sizeof(RowLaw) + 256;
}

hipError_t launch_verify(const VerifyArgs& a, Workspace& ws, hipStream_t st) {
    return a.prec == P32 ? verify_t<float>(a, ws, st) : a.prec == P16 ? verify_t<half_t>(a, ws, st) : verify_t<bhalf_t>(a, ws, st);
}

}  // namespace lrc
