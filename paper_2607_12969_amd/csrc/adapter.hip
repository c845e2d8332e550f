// Low-rank adapters of many requests beside a shared projection, and their gradient.
//
// Row i of X meets adapter a = ids_i of N (or none, where ids_i names none):
//   H_i  = X_i A_a^T                        A: N x k x n
//   Y_i  = base_i + c_a H_i B_a^T           B: N x m x k
//   dH_i = c_a dY_i B_a,  dX_i = base_i + dH_i A_a
//   dA_a = sum dH_i^T X_i,  dB_a = c_a sum dY_i^T H_i    over the rows of a, in row order.
//
// k is small, so all of it is bound by the bytes of X, Y and their gradients, and in
// batches of a few rows by those of the adapters and by launches.
//
// Few rows: a workgroup takes one row and a range of columns (down), then one row and a
// range of outputs (up); vector units, H in binary32.
//
// Many rows: one workgroup sorts the rows by adapter (stable radix sort), so that tiles of
// rows of one adapter go through the matrix cores: down (X read once, all k ranks a
// tile, columns split over workgroups, joined in order), up (H from LDS), outer (the
// gradients of A and B, long runs of rows split and joined in order).  H and dH stay in
// binary32; as an operand of the 16-bit matrix cores a value is the sum of two 16-bit ones
// (16 bits of a bfloat16 pair, 22 of a binary16 pair), which is well below the rounding
// of the 16-bit result.  (Three bfloat16 values, 24 bits, leave the results' errors against 64 bits
// as they are to four digits, 1.66e-3 by their own rounding, and cost, 4096 rows of 8192: k = 16 2 of 166 us,
// k = 64 2 of 67 in the product and 45 of 154 in the gradient, k = 96 18 of 82 and 63 of 274.)  Binary16 pairs are scaled by a power of two, of the row or, where rows
// are summed, of the column of the tile, so that their range does not matter.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "head_device.h"

namespace lrc {

namespace {

constexpr int kTile = 64;             // rows of a tile (down, up)
constexpr int kRun = 512;             // rows of a run (outer)

struct AdapterSort {
    const int64_t* ids;
    int64_t rows, count;
    int *key[2], *order[2];           // the sorted ones in [passes & 1]
    int4 *tiles, *runs;               // first position, rows, key, (runs) slot
    int2* runs_of;                    // per adapter: first slot (-1: one run, no slot), runs
    int* counts;
};
struct AdapterDown {
    const void *P, *Q;
    int64_t ldp, L, k, kp, rows, count;
    const int* order;
    const int4* tiles;
    const int* counts;
    int max_tiles, splits;
    float* part;
};
struct AdapterUp {
    const float *part, *inner, *scale;    // inner, scale: factors of each adapter on H and on H Q^T, or null
    float* Hout;                          // H in the rows' own order, or null
    const void *Q, *base;
    void* O;
    int64_t L, k, kp, rows, count, ldb, ldo;
    int splits;
    const int* order;
    const int4* tiles;
    const int* counts;
    int max_tiles, chunks;
};
struct AdapterRange {
    const float* H[2];
    float* scale[2];
    int64_t k, kp;
    const int* order;
    const int4* runs;
    const int* counts;
};
struct AdapterOuter {
    const void* P;
    const float *H, *scale, *range;   // scale: factor of each adapter, range: of each run and rank, or null
    int64_t ldp, L, k, kp;
    const int* order;
    const int4* runs;
    const int* counts;
    int max_runs, tiles_l;
    float* part;
    void* G;
};

template <typename T> inline constexpr int kParts = sizeof(T) == 4 ? 1 : 2;     // 16-bit values that stand for one of H
template <typename T> inline constexpr int kStep = 4 * kVec<T>;                 // K values of mma16

// Bits of the T value(s) that stand for x.
template <typename T> __device__ __forceinline__ void split_value(float x, unsigned (&p)[kParts<T>]);
template <> __device__ __forceinline__ void split_value<float>(float x, unsigned (&p)[1]) { p[0] = __float_as_uint(x); }
template <> __device__ __forceinline__ void split_value<bhalf_t>(float x, unsigned (&p)[2]) {
    const bhalf_t h = (bhalf_t)x;
    const float lo = x - (float)h;
    p[0] = __builtin_bit_cast(unsigned short, h);
    p[1] = __builtin_bit_cast(unsigned short, (bhalf_t)(__builtin_fabsf(lo) <= 3.4028234663852886e38f ? lo : 0.0f));
}
template <> __device__ __forceinline__ void split_value<half_t>(float x, unsigned (&p)[2]) {
    const half_t h = (half_t)x;
    const float lo = x - (float)h;
    p[0] = __builtin_bit_cast(unsigned short, h);
    p[1] = __builtin_bit_cast(unsigned short, (half_t)(__builtin_fabsf(lo) <= 3.4028234663852886e38f ? lo : 0.0f));
}
__device__ __forceinline__ bool named(int64_t id, int64_t count) { return (uint64_t)id < (uint64_t)count; }

}  // namespace

// ---- few rows -----------------------------------------------------------------
// part[split][row][k]: X_row A^T over 64 E columns.
template <typename T>
__global__ __launch_bounds__(256) void k_adapter_down_rows(AdapterArgs a, float* __restrict__ part) {
    constexpr int E = kVec<T>;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t r = blockIdx.y, id = a.ids[r];
    if (!named(id, a.count)) return;
    const int64_t c = ((int64_t)blockIdx.x * 64 + lane) * E;
    const T* A = static_cast<const T*>(a.A) + id * a.k * a.n;
    const uint4v_t x = load_zero16(static_cast<const T*>(a.X) + r * a.ldx, c, a.n);
    float* out = part + ((int64_t)blockIdx.x * a.rows + r) * a.k;
    for (int64_t j0 = wave * 4; j0 < a.k; j0 += 16) {
        float s[4];
        uint4v_t w[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) w[q] = load_zero16(A + std::min(j0 + q, a.k - 1) * a.n, c, a.n);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            s[q] = 0.0f;
#pragma unroll
            for (int e = 0; e < E; ++e) s[q] += elem<T>(x, e) * elem<T>(w[q], e);
            s[q] = wave_sum(s[q]);
        }
        if (lane < 4 && j0 + lane < a.k) out[j0 + lane] = lane == 0 ? s[0] : lane == 1 ? s[1] : lane == 2 ? s[2] : s[3];
    }
}

// Y_row = base + c H B^T for `per` outputs; a group of 2^shift lanes shares an output's k.
template <typename T>
__global__ __launch_bounds__(256) void k_adapter_up_rows(AdapterArgs a, const float* __restrict__ part, int splits, int per,
                                                         int shift) {
    constexpr int E = kVec<T>;
    __shared__ float h[kAdapterMaxRank + 8];
    const int64_t r = blockIdx.y, id = a.ids[r];
    const bool has = named(id, a.count);
    const int t = threadIdx.x, k = (int)a.k;
    if (t < k) {
        float s = 0.0f;
        if (has) {
            const float* from = part + r * k + t;
            for (int q = 0; q < splits; q += 8) {
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = q + e < splits ? from[(int64_t)(q + e) * a.rows * k] : 0.0f;
#pragma unroll
                for (int e = 0; e < 8; ++e) s += v[e];
            }
        }
        if (a.hidden && blockIdx.x == 0) a.hidden[r * k + t] = s;
        h[t] = s;
    }
    if (t < 8) h[k + t] = 0.0f;
    __syncthreads();
    const float c = has && a.scale ? a.scale[id] : 1.0f;
    const int64_t i0 = (int64_t)blockIdx.x * per, i1 = std::min(a.m, i0 + per);
    const int sub = t & ((1 << shift) - 1), group = t >> shift, groups = 256 >> shift;
    const T* base = a.base ? static_cast<const T*>(a.base) + r * a.ldb : nullptr;
    T* y = static_cast<T*>(a.Y) + r * a.ldy;
    for (int64_t i = i0 + group; i - group < i1; i += groups) {
        float s = 0.0f;
        if (has && i < i1) {
            const T* B = static_cast<const T*>(a.B) + (id * a.m + i) * k;
            for (int j = sub * E; j < k; j += E << shift) {
                const uint4v_t w = load_zero16(B, j, k);
#pragma unroll
                for (int e = 0; e < E; ++e) s += h[j + e] * elem<T>(w, e);
            }
        }
        for (int off = 1; off < 1 << shift; off <<= 1) s += __shfl_xor(s, off, 64);
        if (sub == 0 && i < i1) {
            const float b = base ? (float)base[i] : 0.0f;
            y[i] = has ? from_f32<T>(b + c * s) : from_f32<T>(b);
        }
    }
}

// ---- rows in the order of their adapters -----------------------------------------
namespace {

constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;
constexpr int kLdsRows = 8192;        // rows that are sorted in LDS

// Exclusive sum over the workgroup (`total`: of all).
__device__ __forceinline__ unsigned block_scan(unsigned x, unsigned* red, unsigned& total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    unsigned s = x;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const unsigned o = __shfl_up(s, off, 64);
        if (lane >= off) s += o;
    }
    __syncthreads();
    if (lane == 63) red[wave] = s;
    __syncthreads();
    total = 0;
    unsigned before = 0;
    for (int w = 0; w < kSortWaves; ++w) {
        if (w < wave) before += red[w];
        total += red[w];
    }
    return before + s - x;
}
// Largest of the threads before this one (-1: none), and smallest of those behind it.
__device__ __forceinline__ int block_max_before(int x, int* red) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int s = x;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int o = __shfl_up(s, off, 64);
        if (lane >= off) s = std::max(s, o);
    }
    const int prev = __shfl_up(s, 1, 64);
    __syncthreads();
    if (lane == 63) red[wave] = s;
    __syncthreads();
    int m = lane ? prev : -1;
    for (int w = 0; w < wave; ++w) m = std::max(m, red[w]);
    return m;
}
__device__ __forceinline__ int block_min_behind(int x, int* red) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int s = x;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int o = __shfl_down(s, off, 64);
        if (lane + off < 64) s = std::min(s, o);
    }
    const int next = __shfl_down(s, 1, 64);
    __syncthreads();
    if (lane == 0) red[wave] = s;
    __syncthreads();
    int m = lane < 63 ? next : INT32_MAX;
    for (int w = wave + 1; w < kSortWaves; ++w) m = std::min(m, red[w]);
    return m;
}

}  // namespace

// Rows sorted by adapter, those without one last (key `count`): order, keys, the tiles
// of up to kTile rows of one key, the runs of up to kRun rows of one adapter (slot: where
// a run's partial sums go, -1 for an adapter's only run), and for each adapter its first
// slot and its number of runs.  counts: tiles, runs.  One workgroup, a stable radix sort of
// 4 bits a pass.
//
// Up to 8192 rows, in LDS: a wave takes consecutive positions, 64 at a time.  A position's
// rank among those of its digit is counted by ballots, lane d keeping the running number of
// digit d; only the waves' totals meet.  4096 rows of 8 adapters take 15 us, bound by the
// issue and the latency of one compute unit (counters of each thread and digit in LDS: 15 us
// too, through memory: 24 us; the loops unrolled over registers: 14 us, for four times the code).
__global__ __launch_bounds__(kSortThreads) void k_adapter_sort(AdapterSort s, int passes) {
    typedef unsigned long long u64;
    __shared__ int skey[2][kLdsRows];
    __shared__ unsigned short sorder[2][kLdsRows], srank[kLdsRows];
    __shared__ unsigned tot[kSortWaves][16];
    __shared__ u64 sbegins[kLdsRows / 64];
    __shared__ int firsts[kSortWaves], lasts[kSortWaves];
    __shared__ unsigned sums[kSortWaves][3];
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6, digit = lane & 15;
    const int rows = (int)s.rows, per = (rows + kSortThreads - 1) / kSortThreads;
    const int b = wave * per * 64, e = b + per * 64;        // positions of this wave; those past the rows stay last
    const u64 below = (1ull << lane) - 1, upto = below | 1ull << lane;
    for (int64_t q = t; q < s.count; q += kSortThreads) s.runs_of[q] = int2{0, 0};
    int64_t id[kLdsRows / kSortThreads] = {};               // all loads at once: one latency, not `per` of them
    if (rows > 0)
#pragma unroll
        for (int i = 0; i < kLdsRows / kSortThreads; ++i) id[i] = s.ids[std::min(t + i * kSortThreads, rows - 1)];
#pragma unroll
    for (int i = 0; i < kLdsRows / kSortThreads; ++i) {
        const int p = t + i * kSortThreads;
        if (i >= per) break;
        skey[0][p] = p >= rows ? INT32_MAX : named(id[i], s.count) ? (int)id[i] : (int)s.count;
        sorder[0][p] = (unsigned short)p;
    }
    __syncthreads();
    int which = 0;
    for (int pass = 0; pass < passes; ++pass, which ^= 1) {
        const int shift = 4 * pass;
        unsigned cnt = 0;
#pragma unroll 1
        for (int p = b + lane; p < e; p += 64) {
            const int d = skey[which][p] >> shift & 15;
            u64 same = ~0ull, mine = ~0ull;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const u64 m = __builtin_amdgcn_ballot_w64(d >> q & 1);
                same &= d >> q & 1 ? m : ~m;
                mine &= digit >> q & 1 ? m : ~m;
            }
            srank[p] = (unsigned short)(__shfl(cnt, d, 64) + __builtin_popcountll(same & below));
            cnt += __builtin_popcountll(mine);
        }
        if (lane < 16) tot[wave][lane] = cnt;
        __syncthreads();
        unsigned at = 0, total = 0;                         // of this lane's digit: before this wave, in all
#pragma unroll 4
        for (int w = 0; w < kSortWaves; ++w) {
            const unsigned v = tot[w][digit];
            at += w < wave ? v : 0u;
            total += v;
        }
        unsigned ex = total;
#pragma unroll
        for (int off = 1; off < 16; off <<= 1) {
            const unsigned v = __shfl_up(ex, off, 16);
            if (digit >= off) ex += v;
        }
        at += ex - total;
#pragma unroll 1
        for (int p = b + lane; p < e; p += 64) {
            const int k = skey[which][p];
            const unsigned to = __shfl(at, k >> shift & 15, 64) + srank[p];
            skey[which ^ 1][to] = k;
            sorder[which ^ 1][to] = sorder[which][p];
        }
        __syncthreads();
    }
    // segments of equal keys: a bit for each position that begins one
    const int* keys = skey[which];
    int* key = s.key[which];
    int* order = s.order[which];
    int first = rows, last = -1;
#pragma unroll 1
    for (int p = b + lane; p < e; p += 64) {
        const int k = keys[p];
        if (p < rows) {
            key[p] = k;
            order[p] = sorder[which][p];
        }
        const u64 m = __builtin_amdgcn_ballot_w64(p < rows && (p == 0 || k != keys[std::max(p - 1, 0)]));
        if (lane == 0) sbegins[p >> 6] = m;
        if (m) {
            first = std::min(first, p - lane + __builtin_ctzll(m));
            last = p - lane + 63 - __builtin_clzll(m);
        }
    }
    if (lane == 0) {
        firsts[wave] = first;
        lasts[wave] = last;
    }
    __syncthreads();
    int before = -1, behind = rows;                         // last begin before this wave, first one behind it
#pragma unroll 4
    for (int w = 0; w < kSortWaves; ++w) {
        before = std::max(before, w < wave ? lasts[w] : -1);
        behind = std::min(behind, w > wave ? firsts[w] : rows);
    }
    // twice over the positions: count tiles, runs and slots, then write them
    unsigned at[3] = {0, 0, 0};
#pragma unroll 1
    for (int walk = 0; walk < 2; ++walk) {
        int carry = before;
        unsigned n[3] = {at[0], at[1], at[2]};
#pragma unroll 1
        for (int p = b + lane; p < e; p += 64) {
            const u64 m = sbegins[p >> 6], m0 = m & upto;
            u64 m1 = m & ~upto;
            const int here = p - lane, start = m0 ? here + 63 - __builtin_clzll(m0) : carry;
            if (m) carry = here + 63 - __builtin_clzll(m);
            // where the segment ends: the next begin
            int end = m1 ? here + __builtin_ctzll(m1) : -1;
            for (int q = (p >> 6) + 1; q < e >> 6 && __builtin_amdgcn_ballot_w64(end < 0); ++q) {
                m1 = sbegins[q];
                if (end < 0 && m1) end = q * 64 + __builtin_ctzll(m1);
            }
            if (end < 0) end = behind;
            const int k = keys[p], in = p - start;
            const bool tile = p < rows && in % kTile == 0, run = p < rows && in % kRun == 0 && k < s.count;
            const u64 mt = __builtin_amdgcn_ballot_w64(tile), mr = __builtin_amdgcn_ballot_w64(run),
                      ms = __builtin_amdgcn_ballot_w64(run && end - start > kRun);
            if (walk) {
                if (tile) s.tiles[n[0] + __builtin_popcountll(mt & below)] = int4{p, std::min(kTile, end - p), k, 0};
                if (run) {
                    const int slot = end - start > kRun ? (int)n[2] + __builtin_popcountll(ms & below) : -1;
                    if (in == 0) s.runs_of[k] = int2{slot, (end - start + kRun - 1) / kRun};
                    s.runs[n[1] + __builtin_popcountll(mr & below)] = int4{p, std::min(kRun, end - p), k, slot};
                }
            }
            n[0] += __builtin_popcountll(mt);
            n[1] += __builtin_popcountll(mr);
            n[2] += __builtin_popcountll(ms);
        }
        if (walk) break;
        if (lane < 3) sums[wave][lane] = lane == 0 ? n[0] : lane == 1 ? n[1] : n[2];
        __syncthreads();
        unsigned run[3];                                    // lane w: the waves up to w
#pragma unroll
        for (int q = 0; q < 3; ++q) run[q] = sums[lane & 15][q];
#pragma unroll
        for (int off = 1; off < 16; off <<= 1)
#pragma unroll
            for (int q = 0; q < 3; ++q) {
                const unsigned v = __shfl_up(run[q], off, 16);
                if ((lane & 15) >= off) run[q] += v;
            }
#pragma unroll
        for (int q = 0; q < 3; ++q) at[q] = wave ? __shfl(run[q], wave - 1, 64) : 0u;
        if (t == 15) {
            s.counts[0] = (int)run[0];
            s.counts[1] = (int)run[1];
        }
    }
}

// The same for any number of rows, keys and order in memory: a thread takes consecutive
// rows, with counters of its own in LDS.
__global__ __launch_bounds__(kSortThreads) void k_adapter_sort_memory(AdapterSort s, int passes) {
    __shared__ unsigned cnt[16 * kSortThreads];
    __shared__ unsigned red[kSortWaves];
    __shared__ int redi[kSortWaves];
    const int t = threadIdx.x;
    const int rows = (int)s.rows, per = (rows + kSortThreads - 1) / kSortThreads;
    const int b = std::min(rows, t * per), e = std::min(rows, b + per);
    for (int64_t q = t; q < s.count; q += kSortThreads) s.runs_of[q] = int2{0, 0};
    int which = 0;
    auto key = [&](int p) -> int& { return s.key[which][p]; };
    auto order = [&](int p) -> int& { return s.order[which][p]; };
    // f(position, key, order) of this thread's positions in turn, those of 8 loaded at once: 65536
    // rows of 8 adapters 312 us (one after the other, each waiting for memory, 413 us)
    auto each = [&](auto with_order, auto&& f) {
        for (int p = b; p < e; p += 8) {
            int k[8], o[8] = {};
#pragma unroll
            for (int j = 0; j < 8; ++j) k[j] = key(std::min(p + j, e - 1));
            if constexpr (with_order)
#pragma unroll
                for (int j = 0; j < 8; ++j) o[j] = order(std::min(p + j, e - 1));
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (p + j < e) f(p + j, k[j], o[j]);
        }
    };
    const std::true_type yes;
    const std::false_type no;
    for (int p = t; p < rows; p += kSortThreads) {
        const int64_t id = s.ids[p];
        key(p) = named(id, s.count) ? (int)id : (int)s.count;
        order(p) = p;
    }
    __syncthreads();
    for (int pass = 0; pass < passes; ++pass) {
        const int shift = 4 * pass;
#pragma unroll
        for (int d = 0; d < 16; ++d) cnt[d * kSortThreads + t] = 0;
        each(no, [&](int, int k, int) { ++cnt[(k >> shift & 15) * kSortThreads + t]; });
        __syncthreads();
        // running count over (digit, thread): thread t's 16 entries are consecutive
        unsigned c[16], sum = 0, total;
#pragma unroll
        for (int d = 0; d < 16; ++d) {
            c[d] = cnt[16 * t + d];
            sum += c[d];
        }
        unsigned at = block_scan(sum, red, total);
#pragma unroll
        for (int d = 0; d < 16; ++d) {
            cnt[16 * t + d] = at;
            at += c[d];
        }
        __syncthreads();
        each(yes, [&](int, int k, int o) {
            const unsigned to = cnt[(k >> shift & 15) * kSortThreads + t]++;
            s.key[which ^ 1][to] = k;
            s.order[which ^ 1][to] = o;
        });
        which ^= 1;
        __syncthreads();
    }
    // segments of equal keys
    const int left = b > 0 && b < e ? key(b - 1) : -1;              // keys are not negative
    int first = -1, head = INT32_MAX, prev = left;                  // this thread's last and first segment start
    each(no, [&](int p, int k, int) {
        if (k != prev) {
            first = p;
            head = std::min(head, p);
        }
        prev = k;
    });
    const int before = block_max_before(first, redi);
    const int behind = block_min_behind(head, redi);
    // two walks over this thread's positions: count, then write
    unsigned tiles = 0, runs = 0, slots = 0, tile0 = 0, run0 = 0, slot0 = 0;
#pragma unroll 1
    for (int walk = 0; walk < 2; ++walk) {
        int start = before, end = -1;                               // end: of the segment, once it is known
        prev = left;
        each(no, [&](int p, int k, int) {
            if (k != prev) {
                start = p;
                end = -1;
            }
            prev = k;
            const int in = p - start;
            if (in % kTile) return;
            // the segment's end: the next start, here or behind this thread's part
            const bool run = in % kRun == 0 && k < s.count;
            if (end < 0) {
                end = std::min(behind, rows);
                for (int q = p + 1; q < e; ++q)
                    if (key(q) != k) {
                        end = q;
                        break;
                    }
            }
            const int n_runs = (end - start + kRun - 1) / kRun;
            if (walk) s.tiles[tile0 + tiles] = int4{p, std::min(kTile, end - p), k, 0};
            ++tiles;
            if (run) {
                if (walk) {
                    if (in == 0) s.runs_of[k] = int2{n_runs > 1 ? (int)(slot0 + slots) : -1, n_runs};
                    s.runs[run0 + runs] = int4{p, std::min(kRun, end - p), k, n_runs > 1 ? (int)(slot0 + slots) : -1};
                }
                ++runs;
                slots += n_runs > 1;
            }
        });
        if (!walk) {
            unsigned nt, nr, ns;
            tile0 = block_scan(tiles, red, nt);
            run0 = block_scan(runs, red, nr);
            slot0 = block_scan(slots, red, ns);
            if (t == 0) {
                s.counts[0] = (int)nt;
                s.counts[1] = (int)nr;
            }
            tiles = runs = slots = 0;
        }
    }
}

// ---- down: partial sums of P Q^T ----------------------------------------------------
// One workgroup of 4 waves: a tile of 64 rows of P (pitch ldp, L columns) and up to 16 F
// ranks of Q, over a range of columns; steps of 256 bytes a row go through registers to
// one of two LDS buffers, their loads issued three steps ahead (two for more than 64
// ranks: more would spill).  Q is N x k x L, or (TURN)
// N x L x k: then its part lies in LDS as it does in memory and the operands come by the
// transposing read.  16-byte chunks are XOR-swizzled by the row.  VEC: k in whole vectors
// (TURN).  part[split][position][kp].  4096 rows of 8192 (67 MB): k = 16 and 64 20 us, 3.3 TB/s;
// a workgroup has nine steps, and three dependent reads before the first.
template <typename T, int F, bool TURN, bool VEC>
__global__ __launch_bounds__(256, F <= 4 ? 2 : 1) void k_adapter_down(AdapterDown a) {
    constexpr int E = kVec<T>, S = 16 * E, QP = 16 * F + E;          // QP: pitch of turned rows
    constexpr int XB = kTile * 16, QB = TURN ? S * QP / E : 16 * F * 16;
    __shared__ uint4v_t lds[2][XB + QB];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, lr = lane & 15, lg = lane >> 4;
    const int64_t lt = xcd_tile((int64_t)a.max_tiles * a.splits);
    if (lt >= (int64_t)a.max_tiles * a.splits) return;
    const int split = (int)((unsigned)lt / (unsigned)a.max_tiles), tile = (int)lt - split * a.max_tiles;
    const int4 td = a.tiles[tile];                             // on its way together with the count
    if (tile >= a.counts[0]) return;
    if (td.z >= a.count) return;
    const int64_t j0 = (int64_t)blockIdx.y * 128;              // ranks j0 .. j0 + 16 F
    const unsigned steps = (unsigned)((a.L + S - 1) / S), each = steps / (unsigned)a.splits, more = steps - each * a.splits;
    const int64_t s0 = each * split + std::min<unsigned>(split, more), s1 = s0 + each + ((unsigned)split < more);
    const int ch = tid & 15, rr = tid >> 4;
    const T *px[4], *qx[F];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        px[i] = static_cast<const T*>(a.P) + (int64_t)a.order[td.x + std::min(rr + 16 * i, td.y - 1)] * a.ldp + ch * E;
    // a row of Q, or (TURN) the vector rc of its row qr + S / F i
    constexpr int RC = 16 * F / E;
    const int rc = tid % RC, qr = tid / RC;
    const T* Q = static_cast<const T*>(a.Q) + (int64_t)td.z * a.k * a.L;
#pragma unroll
    for (int i = 0; i < F; ++i)
        qx[i] = TURN ? Q + (int64_t)(qr + S / F * i) * a.k + (VEC ? std::min<int64_t>(j0 + rc * E, a.k - E) : 0)
                     : Q + std::min(j0 + rr + 16 * i, a.k - 1) * a.L + ch * E;
    // Whole steps run in a loop without branches between the loads, the row's partial
    // last step follows.
    constexpr int ST = F <= 4 ? 3 : 2;                         // steps on their way from memory
    uint4v_t vp[ST][4], vq[ST][F];
    auto load = [&](int64_t s, uint4v_t (&p)[4], uint4v_t (&q)[F]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) p[i] = load16(px[i] + s * S);
#pragma unroll
        for (int i = 0; i < F; ++i) {
            if constexpr (!TURN) q[i] = load16(qx[i] + s * S);
            else if constexpr (VEC) q[i] = load16(qx[i] + s * S * a.k);
            else q[i] = load_zero16(qx[i] + s * S * a.k, j0 + rc * E, a.k);
        }
    };
    auto put = [&](int buf, const uint4v_t (&p)[4], const uint4v_t (&q)[F]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) lds[buf][(rr + 16 * i) * 16 + (ch ^ rr)] = p[i];
#pragma unroll
        for (int i = 0; i < F; ++i) lds[buf][XB + (TURN ? (qr + S / F * i) * (QP / E) + rc : (rr + 16 * i) * 16 + (ch ^ rr))] = q[i];
    };
    float4_t acc[F];
#pragma unroll
    for (int f = 0; f < F; ++f) acc[f] = zero_accv<float4_t>();
    auto product = [&](int buf) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint4v_t x = lds[buf][(16 * wave + lr) * 16 + ((4 * q + lg) ^ lr)];
#pragma unroll
            for (int f = 0; f < F; ++f) {
                uint4v_t w;
                if constexpr (!TURN) w = lds[buf][XB + (16 * f + lr) * 16 + ((4 * q + lg) ^ lr)];
                else w = turned<T>(reinterpret_cast<const T*>(&lds[buf][XB]), QP, kStep<T> * q, 16 * f);
                acc[f] = mma16<T>(w, x, acc[f]);
            }
        }
    };
    const int64_t whole = std::min(s1, a.L / S);
    int buf = 0;
    if (s0 < whole) {
#pragma unroll
        for (int i = 0; i < ST; ++i) load(std::min(s0 + i, whole - 1), vp[i], vq[i]);
        put(0, vp[0], vq[0]);
        __syncthreads();
        auto step = [&](int i) {
            product(buf);
            put(buf ^ 1, vp[(i + 1) % ST], vq[(i + 1) % ST]);
            __syncthreads();
            buf ^= 1;
        };
        int64_t s = s0;
        // no branch between the loads: each wait is for its own (more than 64 ranks would spill)
        for (; F <= 4 && s + 2 * ST <= whole; s += ST)
#pragma unroll
            for (int i = 0; i < ST; ++i) {
                load(s + i + ST, vp[i], vq[i]);
                step(i);
            }
        for (; s < whole; s += ST) {
#pragma unroll
            for (int i = 0; i < ST; ++i) {
                if (s + i >= whole) break;
                if (s + i + ST < whole) load(s + i + ST, vp[i], vq[i]);
                step(i);
            }
        }
    }
    if (whole < s1) {
        const int64_t c = whole * S;
#pragma unroll
        for (int i = 0; i < 4; ++i) vp[0][i] = load_zero16(px[i], c, a.L - ch * E);
#pragma unroll
        for (int i = 0; i < F; ++i) {
            vq[0][i] = uint4v_t{0, 0, 0, 0};
            if constexpr (!TURN) vq[0][i] = load_zero16(qx[i], c, a.L - ch * E);
            else if (c + qr + S / F * i < a.L)
                vq[0][i] = VEC ? load16(qx[i] + c * a.k) : load_zero16(qx[i] + c * a.k, j0 + rc * E, a.k);
        }
        __syncthreads();
        put(buf, vp[0], vq[0]);
        __syncthreads();
        product(buf);
    }
    const int row = 16 * wave + lr;
    if (row < td.y) {
        float* out = a.part + ((int64_t)split * a.rows + td.x + row) * a.kp + j0;
#pragma unroll
        for (int f = 0; f < F; ++f)
            if (j0 + 16 * f + 4 * lg < a.kp) *reinterpret_cast<float4_t*>(out + 16 * f + 4 * lg) = acc[f];
    }
}

// H of a row: the sum of its splits, in order, times the adapter's factor; 0 without
// an adapter.  A workgroup takes 256 / k2 rows, k2 = k rounded up to a power of two.
__global__ __launch_bounds__(256) void k_adapter_join(AdapterDown a, const int* __restrict__ key, const float* __restrict__ scale,
                                                      float* __restrict__ H, int shift) {
    const int64_t p = ((int64_t)blockIdx.x << (8 - shift)) + (threadIdx.x >> shift);
    const int j = threadIdx.x & ((1 << shift) - 1);
    if (p >= a.rows || j >= a.k) return;
    const int id = key[p], row = a.order[p];
    float s = 0.0f;
    if (id < a.count) {
        const float* from = a.part + p * a.kp + j;
        const int64_t step = a.rows * a.kp;
        for (int q = 0; q < a.splits; q += 8) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = q + e < a.splits ? from[(q + e) * step] : 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) s += v[e];
        }
        if (scale) s *= scale[id];
    }
    H[(int64_t)row * a.k + j] = s;
}

// ---- up: O = base + c H Q^T ------------------------------------------------------------
// One workgroup of 4 waves: a tile of 64 rows and every `chunks`-th 128 columns, of them
// 32 a wave's: workgroups that run together write together what lies together.  H is the
// sum of down's parts, in order (times the adapter's factor where `inner` is given); it
// lies in LDS as kParts values, and the tile's first workgroup stores it.  Q (N x L x k)
// comes straight from L2 as operands, or (TURN: N x k x L) through LDS of the wave and
// the transposing read, the base straight from memory, all of it one step ahead.  A wave
// works alone, without a barrier: its results cross LDS, 32 rows at a time, so that
// neighbouring lanes load and store neighbouring 16 bytes of a row.  4096 rows of 8192 with a
// base (134 MB): k = 16 34 us, k = 64 45 (51 with the operands' own layout, 16 rows apart from
// lane to lane).
// KS: steps of the K axis (k rounded up), 0: any number.  VEC: k in whole vectors, so
// that operands are loaded without a branch.
template <typename T, int KS, bool VEC, bool TURN>
__global__ __launch_bounds__(256, sizeof(T) == 2 && (KS == 1 || KS == 2) ? 3 : 2) void k_adapter_up(AdapterUp a, int ks) {
    constexpr int E = kVec<T>, P = kParts<T>, KN = KS ? KS : 1, KV = kStep<T>;
    constexpr int CH = 32 / E, RS = 64 / CH, NI = kTile / RS, OP = 36;     // pieces of a row, rows a store, stores
    constexpr int TP = 32 + E;                                             // pitch of Q's tile
    __shared__ float cross[4][32 * OP];
    __shared__ alignas(16) T qt[TURN ? 4 : 1][TURN ? KV * TP : 1];
    extern __shared__ uint4v_t dyn[];
    __shared__ float factor[kTile];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lr = lane & 15, lg = lane >> 4;
    const int64_t lt = xcd_tile((int64_t)a.max_tiles * a.chunks);
    if (lt >= (int64_t)a.max_tiles * a.chunks) return;
    const int tile = (int)((unsigned)lt / (unsigned)a.chunks), chunk = (int)lt - tile * a.chunks;
    const int4 td = a.tiles[tile];                                  // on its way together with the count
    if (tile >= a.counts[0]) return;
    const int64_t stride = (int64_t)a.chunks * 128;
    const bool has = td.z < a.count;
    const int steps = KS ? KS : ks, pitch = 4 * steps + 1;          // chunks of a row of H
    // this lane's pieces: rows lane / CH + RS i, 16 bytes from column ch E on
    const int ch = lane % CH, r0 = lane / CH;
    const T* base[NI];
    T* out[NI];
    bool live[NI];
#pragma unroll
    for (int i = 0; i < NI; ++i) {
        const int row = a.order[td.x + std::min(r0 + RS * i, td.y - 1)];
        live[i] = r0 + RS * i < td.y;
        out[i] = static_cast<T*>(a.O) + row * a.ldo;
        base[i] = a.base ? static_cast<const T*>(a.base) + row * a.ldb : nullptr;
    }
    int64_t c = chunk * 128 + 32 * wave;
    if (!has) {                                                     // the base alone
        if (a.Hout && chunk == 0)
            for (int e = tid; e < td.y * (int)a.k; e += 256) a.Hout[(int64_t)a.order[td.x + e / (int)a.k] * a.k + e % (int)a.k] = 0.0f;
        if (a.base == a.O && a.ldb == a.ldo) return;
        for (; c < a.L; c += stride) {
            const int64_t cc = c + ch * E;
            uint4v_t v[NI];
#pragma unroll
            for (int i = 0; i < NI; ++i) v[i] = a.base ? load_zero16(base[i], cc, a.L) : uint4v_t{0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                if (!live[i]) continue;
                if (cc + E <= a.L) {
                    store16(out[i] + cc, v[i]);
                } else {
#pragma unroll
                    for (int e = 0; e < E; ++e)
                        if (cc + e < a.L) out[i][cc + e] = from_f32<T>(elem<T>(v[i], e));
                }
            }
        }
        return;
    }
    const T* Q = static_cast<const T*>(a.Q) + (int64_t)td.z * a.L * a.k;
    uint4v_t bn[NI], qn[KN][2];
    // `edge`: the columns may pass L.  What lies past k (another rank's values, from a clamped
    // place) becomes 0 where it is used: here it would make the fetch wait for itself.
    auto past = [&](int s, int f) {
        return TURN ? s * KV + f * (KV / 2) + lane / CH >= (int)a.k : VEC && s * KV + lg * E >= (int)a.k;
    };
    auto fetch_q = [&](int64_t c, int s, uint4v_t (&q)[2], auto edge) {
#pragma unroll
        for (int f = 0; f < 2; ++f) {
            if constexpr (TURN) {
                const int64_t j = (int64_t)s * KV + f * (KV / 2) + lane / CH;
                const T* row = Q + std::min(j, a.k - 1) * a.L;
                if constexpr (edge) q[f] = load_zero16(row, c + ch * E, a.L);
                else q[f] = load16(row + c + ch * E);
            } else {
                const int64_t j = (int64_t)s * KV + lg * E;
                const T* row = Q + std::min(c + 16 * f + lr, a.L - 1) * a.k;
                if constexpr (VEC) {
                    q[f] = load16(row + std::min<int64_t>(j, a.k - E));
                } else {
                    q[f] = load_zero16(row, j, a.k);
                }
            }
        }
    };
    auto fetch = [&](int64_t c, auto edge) {
        if (a.base)
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                if constexpr (edge) bn[i] = load_zero16(base[i], c + ch * E, a.L);
                else bn[i] = load16(base[i] + c + ch * E);
            }
        if constexpr (KS > 0)
#pragma unroll
            for (int s = 0; s < KN; ++s) fetch_q(c, s, qn[s], edge);
    };
    const std::true_type yes;
    const std::false_type no;
#pragma unroll
    for (int i = 0; i < NI; ++i) bn[i] = uint4v_t{0, 0, 0, 0};
    if (c + 32 <= a.L) fetch(c, no);
    // H: four threads a row
    {
        const int row = tid >> 2, sub = tid & 3, pos = td.x + std::min(row, td.y - 1);
        const float* from = a.part + (int64_t)pos * a.kp;
        const int64_t step = a.rows * a.kp;
        const float inner = a.inner ? a.inner[td.z] : 1.0f;
        // E values of vector q, zeros past kp (and, as the parts hold them, rounded from garbage past k)
        // (eight parts of all of it at once: the sum waits for memory once or twice)
        auto values = [&](int q, float (&x)[E]) {
            constexpr int N4 = E / 4;
            float4_t v[N4];
#pragma unroll
            for (int e = 0; e < N4; ++e) v[e] = zero_accv<float4_t>();
            for (int p = 0; p < a.splits; p += 8) {
                float4_t w[8][N4];
#pragma unroll
                for (int h = 0; h < 8; ++h)
#pragma unroll
                    for (int e = 0; e < N4; ++e)
                        w[h][e] = *reinterpret_cast<const float4_t*>(from + std::min<int64_t>((int64_t)q * E + 4 * e, a.kp - 4) +
                                                                     std::min(p + h, a.splits - 1) * step);
#pragma unroll
                for (int h = 0; h < 8; ++h)
                    if (p + h < a.splits)
#pragma unroll
                        for (int e = 0; e < N4; ++e) v[e] += w[h][e];
            }
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] = (int64_t)q * E + e < a.k ? v[e >> 2][e & 3] * inner : 0.0f;
        };
        unsigned amax = 0;
        for (int q = sub; q < 4 * steps; q += 4) {
            float x[E];
            values(q, x);
            if (chunk == 0 && a.Hout && row < td.y) {
                float* h = a.Hout + (int64_t)a.order[pos] * a.k + (int64_t)q * E;
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if ((int64_t)q * E + e < a.k) h[e] = x[e];
            }
            if constexpr (__is_same(T, half_t)) {
                // kept in binary32 until the row's range is known
#pragma unroll
                for (int e = 0; e < E; ++e) amax = std::max(amax, __float_as_uint(x[e]) & 0x7FFFFFFFu);
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    const float4_t v = {x[4 * p], x[4 * p + 1], x[4 * p + 2], x[4 * p + 3]};
                    dyn[(p * kTile + row) * pitch + q] = __builtin_bit_cast(uint4v_t, v);
                }
            } else {
                uint4v_t v[P];
#pragma unroll
                for (int p = 0; p < P; ++p) v[p] = uint4v_t{0, 0, 0, 0};
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    unsigned b[P];
                    split_value<T>(x[e], b);
#pragma unroll
                    for (int p = 0; p < P; ++p) set_bits<T>(v[p], e, b[p]);
                }
#pragma unroll
                for (int p = 0; p < P; ++p) dyn[(p * kTile + row) * pitch + q] = v[p];
            }
        }
        float sc = 1.0f;
        if constexpr (__is_same(T, half_t)) {
            amax = std::max(amax, (unsigned)__shfl_xor((int)amax, 1, 64));
            amax = std::max(amax, (unsigned)__shfl_xor((int)amax, 2, 64));
            sc = range_scale<T>(amax);
            for (int q = sub; q < 4 * steps; q += 4) {
                float4_t x[2];
                uint4v_t v[2];
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    x[p] = __builtin_bit_cast(float4_t, dyn[(p * kTile + row) * pitch + q]);
                    v[p] = uint4v_t{0, 0, 0, 0};
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    unsigned b[2];
                    split_value<half_t>(x[e >> 2][e & 3] * sc, b);
#pragma unroll
                    for (int p = 0; p < 2; ++p) set_bits<half_t>(v[p], e, b[p]);
                }
#pragma unroll
                for (int p = 0; p < 2; ++p) dyn[(p * kTile + row) * pitch + q] = v[p];
            }
        }
        if (sub == 0) factor[row] = (a.scale ? a.scale[td.z] : 1.0f) / sc;
    }
    __syncthreads();
    float fac[NI];
#pragma unroll
    for (int i = 0; i < NI; ++i) fac[i] = factor[r0 + RS * i];
    uint4v_t b[NI], q[KN][2];
    auto product = [&](float4_t (&acc)[2][4], int s, const uint4v_t (&w)[2]) {
        uint4v_t x[2];
#pragma unroll
        for (int f = 0; f < 2; ++f) x[f] = past(s, f) ? uint4v_t{0, 0, 0, 0} : w[f];
        if constexpr (TURN) {
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int f = 0; f < 2; ++f)
                *reinterpret_cast<uint4v_t*>(&qt[wave][(f * (KV / 2) + lane / CH) * TP + ch * E]) = x[f];
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int f = 0; f < 2; ++f) x[f] = turned<T>(qt[wave], TP, 0, 16 * f);
        }
#pragma unroll
        for (int g = 0; g < 4; ++g)
#pragma unroll
            for (int p = P - 1; p >= 0; --p) {
                const uint4v_t h = dyn[(p * kTile + 16 * g + lr) * pitch + 4 * s + lg];
                acc[0][g] = mma16<T>(x[0], h, acc[0][g]);
                acc[1][g] = mma16<T>(x[1], h, acc[1][g]);
            }
    };
    auto results = [&](int64_t c, auto edge) {
        float4_t acc[2][4];
#pragma unroll
        for (int f = 0; f < 2; ++f)
#pragma unroll
            for (int g = 0; g < 4; ++g) acc[f][g] = zero_accv<float4_t>();
        if constexpr (KS > 0) {
#pragma unroll
            for (int s = 0; s < KS; ++s) product(acc, s, q[s]);
        } else {
#pragma unroll 2
            for (int s = 0; s < steps; ++s) {
                uint4v_t w[2];
                fetch_q(c, s, w, edge);
                product(acc, s, w);
            }
        }
        const int64_t cc = c + ch * E;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int f = 0; f < 2; ++f)
#pragma unroll
                for (int g = 0; g < 2; ++g)
                    *reinterpret_cast<float4_t*>(&cross[wave][(16 * g + lr) * OP + 16 * f + 4 * lg]) = acc[f][2 * half + g];
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int i = half * NI / 2; i < (half + 1) * NI / 2; ++i) {
                const float* x = &cross[wave][(r0 + RS * i - 32 * half) * OP + ch * E];
                float y[E];
#pragma unroll
                for (int e = 0; e < E; e += 4) {
                    const float4_t v = *reinterpret_cast<const float4_t*>(x + e);
#pragma unroll
                    for (int h = 0; h < 4; ++h) y[e + h] = elem<T>(b[i], e + h) + fac[i] * v[h];
                }
                // rows past the tile's are its last row once more, bit for bit: stored without a
                // branch, so that the next step's loads can be waited for without these stores
                if constexpr (edge) {
#pragma unroll
                    for (int e = 0; e < E; ++e)
                        if (live[i] && cc + e < a.L) out[i][cc + e] = from_f32<T>(y[e]);
                } else {
                    store16(out[i] + cc, pack16<T>(y));
                }
            }
        }
    };
    auto take = [&]() {
#pragma unroll
        for (int i = 0; i < NI; ++i) b[i] = bn[i];
#pragma unroll
        for (int s = 0; s < KN; ++s) {
            q[s][0] = qn[s][0];
            q[s][1] = qn[s][1];
        }
    };
    for (; c + 32 <= a.L; c += stride) {
        take();
        if (c + stride + 32 <= a.L) fetch(c + stride, no);
        results(c, no);
    }
    if (c < a.L) {
        fetch(c, yes);
        take();
        results(c, yes);
    }
}

// ---- outer: sums over rows -------------------------------------------------------------
// The power of two by which the values of a rank are scaled in a run (binary16 pairs), and
// its inverse: scale[run][rank] of two sources.
__global__ __launch_bounds__(256) void k_adapter_range(AdapterRange a) {
    __shared__ unsigned red[16][16];
    const int run = blockIdx.x, tid = threadIdx.x;
    if (run >= a.counts[1]) return;
    const int4 rd = a.runs[run];
    const int j = tid & 15, g = tid >> 4, rank = blockIdx.y * 16 + j;
    const float* H = blockIdx.z ? a.H[1] : a.H[0];
    unsigned amax = 0;
    if (rank < a.k && H)
#pragma unroll 8
        for (int p = g; p < rd.y; p += 16)
            amax = std::max(amax, __float_as_uint(H[(int64_t)a.order[rd.x + p] * a.k + rank]) & 0x7FFFFFFFu);
    red[g][j] = amax;
    __syncthreads();
    if (g == 0) {
#pragma unroll
        for (int q = 1; q < 16; ++q) amax = std::max(amax, red[q][j]);
        (blockIdx.z ? a.scale[1] : a.scale[0])[(int64_t)run * a.kp + rank] = range_scale<half_t>(amax);
    }
}

// Ranks of a workgroup of `outer`: more would spill (and in 16-bit types a build of 128 gave
// wrong gradients of B, for a reason that was not found).
template <typename T> inline constexpr int kOuterRanks = sizeof(T) == 4 ? 32 : 64;

// G = sum over a run's rows of P_row x H_row.  One workgroup of 4 waves: 128 columns of P,
// of them 32 a wave's, and up to 16 F ranks; steps of 64 rows go through registers to one of
// two LDS buffers, H as kParts values, turned ([rank][row]).  COLS: G is k x L (else L x k).
// 4096 rows of 8192, k = 16, both gradients: 34 to 40 us for 134 MB.
template <typename T, int F> struct OuterLds {
    static constexpr int PITCH = 128 + (sizeof(T) == 4 ? 4 : 16), HP = 64 + kVec<T>;
    alignas(16) T p[2][64 * PITCH];
    alignas(16) T h[2][kParts<T> * 16 * F * HP];
    int order[kRun];
};
template <typename T, int F, bool COLS>
__device__ __forceinline__ void outer_product(const AdapterOuter& a, OuterLds<T, F>& m) {
    constexpr int E = kVec<T>, P = kParts<T>, CH = 128 / E, RS = 256 / CH, NI = 64 / RS, KV = kStep<T>;
    constexpr int PITCH = OuterLds<T, F>::PITCH, HP = OuterLds<T, F>::HP;
    auto& lds = m.p;
    auto& hs = m.h;
    auto& order = m.order;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, lr = lane & 15, lg = lane >> 4;
    const int64_t total = (int64_t)a.max_runs * a.tiles_l, lt = xcd_tile(total);
    if (blockIdx.x >= (total + 7) / 8 * 8 || lt >= total) return;       // the grid is the larger gradient's
    const int run = total <= UINT32_MAX ? (int)((unsigned)lt / (unsigned)a.tiles_l) : (int)(lt / a.tiles_l);
    const int4 rd = a.runs[run];                                        // on its way together with the count
    if (run >= a.counts[1]) return;
    const int64_t c0 = (lt - (int64_t)run * a.tiles_l) * 128, j0 = (int64_t)blockIdx.y * kOuterRanks<T>;
    const int ch = tid % CH, r0 = tid / CH, n = rd.y;
    for (int p = tid; p < n; p += 256) order[p] = a.order[rd.x + p];
    __syncthreads();
    const int hr = tid >> 2, hj = tid & 3;                // H: four threads a row, ranks hj + 4 i
    constexpr bool RANGED = __is_same(T, half_t);
    const float* range = RANGED ? a.range + (int64_t)run * a.kp : nullptr;
    float sc[RANGED ? 4 * F : 1] = {1.0f};
    if constexpr (RANGED)
#pragma unroll
        for (int i = 0; i < 4 * F; ++i) sc[i] = range[std::min(j0 + hj + 4 * i, a.k - 1)];
    constexpr int ST = 2;                                 // steps on their way from memory
    uint4v_t vr[ST][NI];
    float hr_[ST][4 * F];
    // without branches between the loads, from clamped places
    auto load = [&](int p0, uint4v_t (&v)[NI], float (&hv)[4 * F], auto whole) {
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const T* row = static_cast<const T*>(a.P) + (int64_t)order[std::min(p0 + r0 + RS * i, n - 1)] * a.ldp;
            if constexpr (whole) v[i] = load16(row + c0 + ch * E);
            else v[i] = load_zero16(row, c0 + ch * E, a.L);
        }
        const float* h = a.H + (int64_t)order[std::min(p0 + hr, n - 1)] * a.k;
#pragma unroll
        for (int i = 0; i < 4 * F; ++i) hv[i] = h[std::min(j0 + hj + 4 * i, a.k - 1)];
    };
    // rows past the run, whose loads met another row, as zeros
    auto put = [&](int p0, int buf, const uint4v_t (&v)[NI], const float (&hv)[4 * F]) {
#pragma unroll
        for (int i = 0; i < NI; ++i)
            *reinterpret_cast<uint4v_t*>(&lds[buf][(r0 + RS * i) * PITCH + ch * E]) =
                p0 + r0 + RS * i < n ? v[i] : uint4v_t{0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < 4 * F; ++i) {
            unsigned b[P];
            split_value<T>(p0 + hr < n && j0 + hj + 4 * i < a.k ? hv[i] * sc[RANGED ? i : 0] : 0.0f, b);
#pragma unroll
            for (int q = 0; q < P; ++q) {
                T* o = &hs[buf][(q * 16 * F + hj + 4 * i) * HP + hr];
                if constexpr (sizeof(T) == 4) *o = __uint_as_float(b[q]);
                else *o = __builtin_bit_cast(T, (unsigned short)b[q]);
            }
        }
    };
    float4_t acc[2][F];
#pragma unroll
    for (int f = 0; f < F; ++f) acc[0][f] = acc[1][f] = zero_accv<float4_t>();
    auto step = [&](int p0, int buf, uint4v_t (&v)[NI], float (&hv)[4 * F], const uint4v_t (&vn)[NI], const float (&hn)[4 * F],
                    auto whole) {
        load(std::min(p0 + 64 * ST, n - 1), v, hv, whole);        // past the end: the last row
#pragma unroll
        for (int s = 0; s < 64 / KV; ++s) {
            uint4v_t x[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) x[h] = turned<T>(lds[buf], PITCH, s * KV, 32 * wave + 16 * h);
#pragma unroll
            for (int f = 0; f < F; ++f)
#pragma unroll
                for (int q = P - 1; q >= 0; --q) {
                    const uint4v_t h = *reinterpret_cast<const uint4v_t*>(&hs[buf][(q * 16 * F + 16 * f + lr) * HP + s * KV + lg * E]);
#pragma unroll
                    for (int w = 0; w < 2; ++w) acc[w][f] = COLS ? mma16<T>(x[w], h, acc[w][f]) : mma16<T>(h, x[w], acc[w][f]);
                }
        }
        put(p0 + 64, buf ^ 1, vn, hn);
        __syncthreads();
    };
    auto run_all = [&](auto whole) {
        load(0, vr[0], hr_[0], whole);
        load(std::min(64, n - 1), vr[1], hr_[1], whole);
        put(0, 0, vr[0], hr_[0]);
        __syncthreads();
        for (int p0 = 0; p0 < n; p0 += 128) {
            step(p0, 0, vr[0], hr_[0], vr[1], hr_[1], whole);
            if (p0 + 64 < n) step(p0 + 64, 1, vr[1], hr_[1], vr[0], hr_[0], whole);
        }
    };
    if (c0 + 128 <= a.L) run_all(std::true_type());
    else run_all(std::false_type());
    const float c = a.scale ? a.scale[rd.z] : 1.0f;
    // a lane's four results are consecutive in G: along L (COLS) or along the ranks
    const int64_t row_len = COLS ? a.L : a.k;
#pragma unroll
    for (int w = 0; w < 2; ++w)
#pragma unroll
        for (int f = 0; f < F; ++f) {
            const int64_t l = c0 + 32 * wave + 16 * w, j = j0 + 16 * f;
            const int64_t row = COLS ? j + lr : l + lr, col = (COLS ? l : j) + 4 * lg;
            if (row >= (COLS ? a.k : a.L)) continue;
            float y[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int64_t rank = COLS ? row : col + e;
                y[e] = acc[w][f][e] * (RANGED ? c / range[std::min(rank, a.k - 1)] : c);
            }
            if (rd.w >= 0) {
                float* o = a.part + ((int64_t)rd.w * (COLS ? a.k : a.L) + row) * row_len + col;
                if (col + 4 <= row_len) __builtin_memcpy(o, y, 16);
                else
                    for (int e = 0; e < 4; ++e)
                        if (col + e < row_len) o[e] = y[e];
            } else {
                T* o = static_cast<T*>(a.G) + ((int64_t)rd.z * (COLS ? a.k : a.L) + row) * row_len + col;
                T z[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) z[e] = from_f32<T>(y[e]);
                if (col + 4 <= row_len) __builtin_memcpy(o, z, sizeof(z));
                else
                    for (int e = 0; e < 4; ++e)
                        if (col + e < row_len) o[e] = z[e];
            }
        }
}

// The gradients of A (0) and of B (1), each with a grid as large as the larger one.
template <typename T, int F>
__global__ __launch_bounds__(256, 2) void k_adapter_outer(AdapterOuter da, AdapterOuter db) {
    __shared__ OuterLds<T, F> m;
    if (blockIdx.z) outer_product<T, F, false>(db, m);
    else outer_product<T, F, true>(da, m);
}

// Gradients of adapters with several runs (their sum, in order) or none (0): of A and of B.
struct AdapterSum {
    const float* part[2];
    void* G[2];
    int64_t per[2], count;
    const int2* runs_of;
};
template <typename T> __global__ __launch_bounds__(256) void k_adapter_sum(AdapterSum a) {
    const int which = blockIdx.z;
    const int64_t per = which ? a.per[1] : a.per[0];
    const float* part = which ? a.part[1] : a.part[0];
    T* G = static_cast<T*>(which ? a.G[1] : a.G[0]);
    if (!G) return;
    for (int64_t id = blockIdx.y; id < a.count; id += gridDim.y) {
        const int2 r = a.runs_of[id];
        if (r.y == 1) continue;
        for (int64_t e = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; e < per; e += (int64_t)gridDim.x * 1024) {
            const int n = (int)std::min<int64_t>(4, per - e);
            float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            if (n == 4 && per % 4 == 0) {
#pragma unroll 4
                for (int q = 0; q < r.y; ++q) {
                    const float4_t v = *reinterpret_cast<const float4_t*>(part + (r.x + q) * per + e);
#pragma unroll
                    for (int h = 0; h < 4; ++h) s[h] += v[h];
                }
            } else {
                for (int q = 0; q < r.y; ++q)
                    for (int h = 0; h < n; ++h) s[h] += part[(r.x + q) * per + e + h];
            }
            for (int h = 0; h < n; ++h) G[id * per + e + h] = from_f32<T>(s[h]);
        }
    }
}

// ------------------------------------------------------------------ plan --
namespace {

int sort_passes(int64_t count) {
    int bits = 1;
    while (count >> bits) ++bits;
    return (bits + 3) / 4;
}

// Sizes and slices of the workspace for `rows` rows of `count` adapters.
struct AdapterPlan {
    int64_t rows, count, k, kp, max_tiles, max_runs, max_slots;
    AdapterPlan(int64_t rows_, int64_t count_, int64_t k_) : rows(rows_), count(count_), k(k_) {
        kp = round_up(k, 16);
        const int64_t segments = std::min(rows, count + 1);
        max_tiles = std::max<int64_t>(1, rows / kTile + segments);
        max_runs = std::max<int64_t>(1, rows / kRun + segments);
        // an adapter of r > kRun rows has at most (r + kRun - 1) / kRun runs
        max_slots = std::max<int64_t>(1, (rows + (kRun - 1) * std::min(count, rows / (kRun + 1))) / kRun);
    }
    // columns of `down` are split until about 512 workgroups share them
    int down_splits(int64_t L, int e) const {
        const int64_t steps = (L * e + 255) / 256, tiles = max_tiles * ((k + 127) / 128);
        return (int)std::max<int64_t>(1, std::min(steps, std::max<int64_t>(1, 512 / tiles)));
    }
};

struct Slices {
    Workspace* ws;
    size_t bytes = 0;
    template <typename X> X* take(int64_t n) {
        const size_t b = (size_t)round_up(std::max<int64_t>(n, 1) * (int64_t)sizeof(X), 256);
        bytes += b;
        return ws ? static_cast<X*>(ws->take(b)) : nullptr;
    }
};

AdapterSort take_sort(Slices& s, const AdapterPlan& p, const int64_t* ids) {
    AdapterSort a{};
    a.ids = ids;
    a.rows = p.rows;
    a.count = p.count;
    for (int q = 0; q < 2; ++q) {
        a.key[q] = s.take<int>(p.rows);
        a.order[q] = s.take<int>(p.rows);
    }
    a.tiles = s.take<int4>(p.max_tiles);
    a.runs = s.take<int4>(p.max_runs);
    a.runs_of = s.take<int2>(p.count);
    a.counts = s.take<int>(2);
    return a;
}

hipError_t run_sort(const AdapterSort& a, hipStream_t st) {
    KernelTimer t("adapter_sort", st);
    auto* kern = a.rows <= kLdsRows ? k_adapter_sort : k_adapter_sort_memory;
    hipLaunchKernelGGL(kern, dim3(1), dim3(kSortThreads), 0, st, a, sort_passes(a.count));
    return hipGetLastError();
}

template <typename T, int F> void down_f(const AdapterDown& a, bool turn, hipStream_t st) {
    auto* kern = !turn                 ? k_adapter_down<T, F, false, true>
                 : a.k % kVec<T> == 0 ? k_adapter_down<T, F, true, true>
                                       : k_adapter_down<T, F, true, false>;
    hipLaunchKernelGGL(kern, dim3(xcd_grid((int64_t)a.max_tiles * a.splits), (unsigned)((a.k + 127) / 128)), dim3(256), 0, st, a);
}
// Parts of P Q^T, Q N x k x L or (turn) N x L x k.
template <typename T>
AdapterDown run_down(const AdapterPlan& p, const AdapterSort& s, const void* P, int64_t ldp, int64_t L, const void* Q, bool turn,
                     float* part, hipStream_t st) {
    AdapterDown a{};
    a.P = P;
    a.ldp = ldp;
    a.L = L;
    a.Q = Q;
    a.k = p.k;
    a.kp = p.kp;
    a.rows = p.rows;
    a.count = p.count;
    a.order = s.order[sort_passes(p.count) & 1];
    a.tiles = s.tiles;
    a.counts = s.counts;
    a.max_tiles = (int)p.max_tiles;
    a.splits = p.down_splits(L, sizeof(T));
    a.part = part;
    KernelTimer t("adapter_down", st);
    const int64_t f = (std::min<int64_t>(p.k, 128) + 15) / 16;
    if (f <= 1) down_f<T, 1>(a, turn, st);
    else if (f <= 2) down_f<T, 2>(a, turn, st);
    else if (f <= 4) down_f<T, 4>(a, turn, st);
    else down_f<T, 8>(a, turn, st);
    return a;
}
// H alone, of the parts.
hipError_t run_join(const AdapterDown& d, const int* key, const float* scale, float* H, hipStream_t st) {
    int shift = 0;
    while (1 << shift < d.k) ++shift;
    const int64_t per = 256 >> shift;
    KernelTimer t("adapter_join", st);
    hipLaunchKernelGGL(k_adapter_join, dim3((unsigned)((std::max<int64_t>(d.rows, 1) + per - 1) / per)), dim3(256), 0, st, d, key,
                       scale, H, shift);
    return hipGetLastError();
}

// O = base + scale H Q^T, H = inner times the parts, stored at Hout.  Q N x L x k or (turn)
// N x k x L.
template <typename T, bool TURN> hipError_t up_t(const AdapterUp& a, hipStream_t st) {
    const int KS = (int)((a.k + kStep<T> - 1) / kStep<T>);
    const size_t lds = (size_t)kParts<T> * kTile * (4 * KS + 1) * 16;
    const bool vec = TURN || a.k % kVec<T> == 0;
    auto* kern = !vec      ? KS == 1   ? k_adapter_up<T, 1, TURN, TURN>
                             : KS == 2 ? k_adapter_up<T, 2, TURN, TURN>
                                       : k_adapter_up<T, 0, TURN, TURN>
                 : KS == 1 ? k_adapter_up<T, 1, true, TURN>
                 : KS == 2 ? k_adapter_up<T, 2, true, TURN>
                 : KS == 4 && sizeof(T) == 2 ? k_adapter_up<T, sizeof(T) == 2 ? 4 : 0, true, TURN>
                                             : k_adapter_up<T, 0, true, TURN>;
    if (lds > 65536) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kern),
                                                 hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return e;
    }
    KernelTimer t("adapter_up", st);
    hipLaunchKernelGGL(kern, dim3(xcd_grid((int64_t)a.max_tiles * a.chunks)), dim3(256), lds, st, a, KS);
    return hipGetLastError();
}
template <typename T>
hipError_t run_up(const AdapterPlan& p, const AdapterSort& s, const AdapterDown& d, const void* Q, bool turn, int64_t L,
                  const float* inner, const float* scale, float* Hout, const void* base, int64_t ldb, void* O, int64_t ldo,
                  hipStream_t st) {
    AdapterUp a{};
    a.part = d.part;
    a.inner = inner;
    a.scale = scale;
    a.Hout = Hout;
    a.Q = Q;
    a.base = base;
    a.O = O;
    a.L = L;
    a.k = p.k;
    a.kp = p.kp;
    a.rows = p.rows;
    a.count = p.count;
    a.ldb = ldb;
    a.ldo = ldo;
    a.splits = d.splits;
    a.order = d.order;
    a.tiles = s.tiles;
    a.counts = s.counts;
    a.max_tiles = (int)p.max_tiles;
    // one round of workgroups, three a compute unit: each begins with two dependent loads
    a.chunks = (int)std::min((L + 127) / 128, std::max<int64_t>(1, 768 / p.max_tiles));
    return turn ? up_t<T, true>(a, st) : up_t<T, false>(a, st);
}

template <typename T, int F> void outer_f(const AdapterOuter& a, const AdapterOuter& b, hipStream_t st) {
    const dim3 grid(xcd_grid((int64_t)a.max_runs * std::max(a.tiles_l, b.tiles_l)), (unsigned)((a.k + kOuterRanks<T> - 1) / kOuterRanks<T>), 2);
    hipLaunchKernelGGL((k_adapter_outer<T, F>), grid, dim3(256), 0, st, a, b);
}

// Few rows go one by one, each with its adapter's factors from L2 or beyond; more are sorted by
// adapter first, which costs three launches and the sort.  8192 x 8192 with a base, in us, row by
// row against sorted, of 4 and of 64 adapters: bfloat16, k = 16: 64 rows 13 and 14, 128 rows 13
// against 25 and 15 against 31, 256 rows 19 against 28 and 26 against 31; k = 64: 128 rows 35 against 37 and
// 48 against 45, 256 rows 63 against 46 and 85 against 45; FP32, k = 16: 128 rows 20 against 25 and 27
// against 54, 256 rows 38 against 32 and 45 against 54; k = 64: 128 rows 75 against 54 and 101 against 128.
bool few_rows(int64_t rows, int64_t k, int prec) {
    return rows <= 64 || (rows <= 256 && rows * k * elem_bytes(prec) <= 16384);
}

int64_t rows_splits(int64_t n, int prec) {
    const int64_t per = 64 * (prec == P32 ? 4 : 8);
    return (n + per - 1) / per;
}

// Where the parts of a call lie; ws == nullptr: their size alone.
struct ApplySlices {
    AdapterSort sort;
    float* part;
};
ApplySlices apply_slices(const AdapterArgs& a, Slices& s) {
    ApplySlices o{};
    if (few_rows(a.rows, a.k, a.prec)) {
        o.part = s.take<float>(rows_splits(a.n, a.prec) * a.rows * a.k);
        return o;
    }
    const AdapterPlan p(a.rows, a.count, a.k);
    o.sort = take_sort(s, p, a.ids);
    o.part = s.take<float>(p.down_splits(a.n, elem_bytes(a.prec)) * a.rows * p.kp);
    return o;
}

template <typename T> hipError_t apply_t(const AdapterArgs& a, Workspace& ws, hipStream_t st) {
    Slices s{&ws};
    const ApplySlices o = apply_slices(a, s);
    if (ws.overrun) return hipErrorOutOfMemory;
    if (few_rows(a.rows, a.k, a.prec)) {
        const int splits = (int)rows_splits(a.n, a.prec);
        {
            KernelTimer t("adapter_down_rows", st);
            hipLaunchKernelGGL(k_adapter_down_rows<T>, dim3(splits, (unsigned)a.rows), dim3(256), 0, st, a, o.part);
        }
        int shift = 0;
        while (shift < 4 && (kVec<T> << shift) < a.k) ++shift;
        const int64_t want = std::max<int64_t>(1, 1024 / a.rows);           // workgroups of a row
        const int64_t groups = 256 >> shift;
        const int64_t per = round_up((a.m + want - 1) / want, groups);
        KernelTimer t("adapter_up_rows", st);
        hipLaunchKernelGGL(k_adapter_up_rows<T>, dim3((unsigned)((a.m + per - 1) / per), (unsigned)a.rows), dim3(256), 0, st, a,
                           o.part, splits, (int)per, shift);
        return hipGetLastError();
    }
    const AdapterPlan p(a.rows, a.count, a.k);
    const hipError_t e = run_sort(o.sort, st);
    if (e != hipSuccess) return e;
    const AdapterDown d = run_down<T>(p, o.sort, a.X, a.ldx, a.n, a.A, false, o.part, st);
    return run_up<T>(p, o.sort, d, a.B, false, a.m, nullptr, a.scale, a.hidden, a.base, a.ldb, a.Y, a.ldy, st);
}

struct GradSlices {
    AdapterSort sort;
    float *part, *dH, *sums[2], *range[2];
};
GradSlices grad_slices(const AdapterGradArgs& a, Slices& s) {
    const AdapterPlan p(a.rows, a.count, a.k);
    GradSlices o{};
    o.sort = take_sort(s, p, a.ids);
    o.part = s.take<float>(p.down_splits(a.m, elem_bytes(a.prec)) * a.rows * p.kp);
    o.dH = s.take<float>(a.rows * a.k);
    if (a.prec == P16)
        for (int q = 0; q < 2; ++q) o.range[q] = s.take<float>(p.max_runs * p.kp);
    o.sums[0] = a.dA ? s.take<float>(p.max_slots * a.n * a.k) : nullptr;
    o.sums[1] = a.dB ? s.take<float>(p.max_slots * a.m * a.k) : nullptr;
    return o;
}

template <typename T> hipError_t grad_t(const AdapterGradArgs& a, Workspace& ws, hipStream_t st) {
    Slices sl{&ws};
    const GradSlices o = grad_slices(a, sl);
    if (ws.overrun) return hipErrorOutOfMemory;
    const AdapterPlan p(a.rows, a.count, a.k);
    const int odd = sort_passes(p.count) & 1;
    hipError_t e = run_sort(o.sort, st);
    if (e != hipSuccess) return e;
    if (a.dX || a.dA) {
        const AdapterDown d = run_down<T>(p, o.sort, a.dY, a.lddy, a.m, a.B, true, o.part, st);
        e = a.dX ? run_up<T>(p, o.sort, d, a.A, true, a.n, a.scale, nullptr, o.dH, a.base, a.ldb, a.dX, a.lddx, st)
                 : run_join(d, o.sort.key[odd], a.scale, o.dH, st);
    }
    if (e != hipSuccess || (!a.dA && !a.dB)) return e;
    const float* H[2] = {o.dH, a.hidden};
    if (o.range[0]) {
        const AdapterRange r{{a.dA ? H[0] : nullptr, a.dB ? H[1] : nullptr}, {o.range[0], o.range[1]}, a.k, p.kp,
                             o.sort.order[odd], o.sort.runs, o.sort.counts};
        KernelTimer t("adapter_range", st);
        hipLaunchKernelGGL(k_adapter_range, dim3((unsigned)p.max_runs, (unsigned)(p.kp / 16), 2), dim3(256), 0, st, r);
    }
    AdapterOuter w[2] = {};
    AdapterSum sum{};
    for (int q = 0; q < 2; ++q) {
        w[q].P = q ? a.dY : a.X;
        w[q].ldp = q ? a.lddy : a.ldx;
        w[q].L = q ? a.m : a.n;
        w[q].H = H[q];
        w[q].range = o.range[q];
        w[q].k = a.k;
        w[q].kp = p.kp;
        w[q].scale = q ? a.scale : nullptr;
        w[q].order = o.sort.order[odd];
        w[q].runs = o.sort.runs;
        w[q].counts = o.sort.counts;
        w[q].max_runs = (int)p.max_runs;
        w[q].G = q ? a.dB : a.dA;
        w[q].tiles_l = w[q].G ? (int)((w[q].L + 127) / 128) : 0;
        w[q].part = o.sums[q];
        sum.part[q] = o.sums[q];
        sum.G[q] = w[q].G;
        sum.per[q] = w[q].L * a.k;
    }
    {
        KernelTimer t("adapter_outer", st);
        if (a.k <= 16) outer_f<T, 1>(w[0], w[1], st);
        else if (a.k <= 32) outer_f<T, 2>(w[0], w[1], st);
        else outer_f<T, kOuterRanks<T> / 16>(w[0], w[1], st);
    }
    sum.count = a.count;
    sum.runs_of = o.sort.runs_of;
    KernelTimer t("adapter_sum", st);
    const int64_t per = std::max(sum.per[0], sum.per[1]);
    hipLaunchKernelGGL(k_adapter_sum<T>,
                       dim3((unsigned)std::min<int64_t>((per + 1023) / 1024, 1024), (unsigned)std::min<int64_t>(a.count, 65535), 2),
                       dim3(256), 0, st, sum);
    return hipGetLastError();
}

}  // namespace

size_t adapter_workspace_bytes(const AdapterArgs& a) {
    Slices s{nullptr};
    (void)apply_slices(a, s);
    return s.bytes;
}
size_t adapter_grad_workspace_bytes(const AdapterGradArgs& a) {
    Slices s{nullptr};
    (void)grad_slices(a, s);
    return s.bytes;
}
hipError_t launch_adapter(const AdapterArgs& a, Workspace& ws, hipStream_t st) {
    return a.prec == P32 ? apply_t<float>(a, ws, st) : a.prec == P16 ? apply_t<half_t>(a, ws, st) : apply_t<bhalf_t>(a, ws, st);
}
hipError_t launch_adapter_backward(const AdapterGradArgs& a, Workspace& ws, hipStream_t st) {
    return a.prec == P32 ? grad_t<float>(a, ws, st) : a.prec == P16 ? grad_t<half_t>(a, ws, st) : grad_t<bhalf_t>(a, ws, st);
}

}  // namespace lrc
