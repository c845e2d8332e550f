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

#include "sample_device.h"

namespace lrc {

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
    const int n = gather_down_to<T>(s, row, wt, last);
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
        const int n = gather_down_to<T>(s, row, wt, bin < 0 ? kBins : bin);
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
