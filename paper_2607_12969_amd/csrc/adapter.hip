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
// of the 16-bit result.  Binary16 pairs are scaled by a power of two, of the row or, where rows
// are summed, of the column of the tile, so that their range does not matter.
#include <hip/hip_runtime.h>

#include <algorithm>

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
    const float *H, *scale;           // scale: factor of each adapter, or null
    const void *Q, *base;
    void* O;
    int64_t L, k, count, ldb, ldo, cols;
    const int* order;
    const int4* tiles;
    const int* counts;
    int max_tiles, chunks;
};
struct AdapterTurn {
    const float* H[2];
    void* out[2];
    float* inv[2];
    int64_t k, kp, ldt;
    const int* order;
    const int4* runs;
    const int* counts;
};
struct AdapterOuter {
    const void *P, *H;
    const float *inv, *scale;
    int64_t ldp, L, k, kp, ldt;
    const int* order;
    const int4* runs;
    const int* counts;
    int max_runs, tiles_l;
    float* part;
    void* G;
};

// One 16-byte operand a lane: 32 K values of an instruction for 16-bit types, four
// instructions of 4 K values for binary32.
template <typename T> __device__ __forceinline__ float4_t mma16(const uint4v_t& a, const uint4v_t& b, float4_t c);
template <> __device__ __forceinline__ float4_t mma16<half_t>(const uint4v_t& a, const uint4v_t& b, float4_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8_t, a), __builtin_bit_cast(half8_t, b), c, 0, 0, 0);
}
template <> __device__ __forceinline__ float4_t mma16<bhalf_t>(const uint4v_t& a, const uint4v_t& b, float4_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bhalf8_t, a), __builtin_bit_cast(bhalf8_t, b), c, 0, 0, 0);
}
template <> __device__ __forceinline__ float4_t mma16<float>(const uint4v_t& a, const uint4v_t& b, float4_t c) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
        c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[e]), __uint_as_float(b[e]), c, 0, 0, 0);
    return c;
}

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
// The power of two that brings a largest magnitude (as bits) to [2^14, 2^15), where
// binary16 pairs are to hold it; 1 for other types, zeros, infinities and NaN.
template <typename T> __device__ __forceinline__ float range_scale(unsigned amax) {
    if constexpr (!__is_same(T, half_t)) return 1.0f;
    if (amax == 0 || amax >= 0x7F800000u) return 1.0f;
    const int e = std::max((int)(amax >> 23), 1) - 127;          // floor(log2), subnormals as 2^-126
    return __uint_as_float((unsigned)(std::min(14 - e, 126) + 127) << 23);
}

// The vector at column c of a row of L, zeros past the end.
template <typename T> __device__ __forceinline__ uint4v_t load_zero16(const T* row, int64_t c, int64_t L) {
    if (c + kVec<T> <= L) return load16(row + c);
    uint4v_t v = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < kVec<T>; ++e)
        if (c + e < L) {
            unsigned b;
            if constexpr (sizeof(T) == 4) b = __builtin_bit_cast(unsigned, row[c + e]);
            else b = __builtin_bit_cast(unsigned short, row[c + e]);
            set_bits<T>(v, e, b);
        }
    return v;
}

__device__ __forceinline__ bool named(int64_t id, int64_t count) { return (uint64_t)id < (uint64_t)count; }

}  // namespace

// ---- few rows -----------------------------------------------------------------
// part[split][row][k]: X_row A^T over 64 E VX columns.
template <typename T, int VX>
__global__ __launch_bounds__(256) void k_adapter_down_rows(AdapterArgs a, float* __restrict__ part) {
    constexpr int E = kVec<T>;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t r = blockIdx.y, id = a.ids[r];
    if (!named(id, a.count)) return;
    const int64_t c0 = (int64_t)blockIdx.x * 64 * E * VX;
    const T* x = static_cast<const T*>(a.X) + r * a.ldx;
    const T* A = static_cast<const T*>(a.A) + id * a.k * a.n;
    float xv[VX][E];
#pragma unroll
    for (int v = 0; v < VX; ++v) {
        const uint4v_t w = load_zero16(x, c0 + (v * 64 + lane) * E, a.n);
#pragma unroll
        for (int e = 0; e < E; ++e) xv[v][e] = elem<T>(w, e);
    }
    float* out = part + ((int64_t)blockIdx.x * a.rows + r) * a.k;
    for (int64_t j0 = wave * 4; j0 < a.k; j0 += 16) {
        float s[4];
        uint4v_t w[4][VX];
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int v = 0; v < VX; ++v)
                w[q][v] = load_zero16(A + std::min(j0 + q, a.k - 1) * a.n, c0 + (v * 64 + lane) * E, a.n);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            s[q] = 0.0f;
#pragma unroll
            for (int v = 0; v < VX; ++v)
#pragma unroll
                for (int e = 0; e < E; ++e) s[q] += xv[v][e] * elem<T>(w[q][v], e);
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

constexpr int kSortThreads = 512, kSortWaves = kSortThreads / 64;

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
// slot and its number of runs.  counts: tiles, runs.
__global__ __launch_bounds__(kSortThreads) void k_adapter_sort(AdapterSort s, int passes) {
    __shared__ unsigned cnt[16 * kSortThreads];
    __shared__ unsigned red[kSortWaves];
    __shared__ int redi[kSortWaves];
    const int t = threadIdx.x;
    const int rows = (int)s.rows, per = (rows + kSortThreads - 1) / kSortThreads;
    const int b = std::min(rows, t * per), e = std::min(rows, b + per);
    for (int64_t q = t; q < s.count; q += kSortThreads) s.runs_of[q] = int2{0, 0};
    int* key = s.key[0];
    int* order = s.order[0];
    for (int p = b; p < e; ++p) {
        const int64_t id = s.ids[p];
        key[p] = named(id, s.count) ? (int)id : (int)s.count;
        order[p] = p;
    }
    for (int pass = 0; pass < passes; ++pass) {
        const int shift = 4 * pass;
        int* key2 = s.key[(pass + 1) & 1];
        int* order2 = s.order[(pass + 1) & 1];
#pragma unroll
        for (int d = 0; d < 16; ++d) cnt[d * kSortThreads + t] = 0;
        for (int p = b; p < e; ++p) ++cnt[(key[p] >> shift & 15) * kSortThreads + t];
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
        for (int p = b; p < e; ++p) {
            const unsigned to = cnt[(key[p] >> shift & 15) * kSortThreads + t]++;
            key2[to] = key[p];
            order2[to] = order[p];
        }
        __threadfence_block();
        __syncthreads();
        key = key2;
        order = order2;
    }
    // segments of equal keys
    int first = -1, head = INT32_MAX;        // this thread's last and first segment start
    for (int p = b; p < e; ++p)
        if (p == 0 || key[p] != key[p - 1]) {
            first = p;
            head = std::min(head, p);
        }
    const int before = block_max_before(first, redi);
    const int behind = block_min_behind(head, redi);
    // two walks over this thread's positions: count, then write
    unsigned tiles = 0, runs = 0, slots = 0, tile0 = 0, run0 = 0, slot0 = 0;
    for (int walk = 0; walk < 2; ++walk) {
        int start = before;
        for (int p = b; p < e; ++p) {
            if (p == 0 || key[p] != key[p - 1]) start = p;
            const int in = p - start;
            if (in % kTile) continue;
            // the segment's end: the next start, here or behind this thread's part
            const bool run = in % kRun == 0 && key[p] < s.count;
            int end = std::min(behind, rows);
            for (int q = p + 1; q < e; ++q)
                if (key[q] != key[q - 1]) {
                    end = q;
                    break;
                }
            const int n_runs = (end - start + kRun - 1) / kRun;
            if (walk) s.tiles[tile0 + tiles] = int4{p, std::min(kTile, end - p), key[p], 0};
            ++tiles;
            if (run) {
                if (walk) {
                    if (in == 0) s.runs_of[key[p]] = int2{n_runs > 1 ? (int)(slot0 + slots) : -1, n_runs};
                    s.runs[run0 + runs] = int4{p, std::min(kRun, end - p), key[p], n_runs > 1 ? (int)(slot0 + slots) : -1};
                }
                ++runs;
                slots += n_runs > 1;
            }
        }
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
// rows of Q (N x k x L), over a range of columns; steps of 256 bytes a row go through
// registers to one of two LDS buffers, the loads of a step issued before the products of
// the one before it.  A row's 16-byte chunks are XOR-swizzled by the row.
// part[split][position][kp].
template <typename T, int F>
__global__ __launch_bounds__(256) void k_adapter_down(AdapterDown a) {
    constexpr int E = kVec<T>, S = 16 * E, R = kTile + 16 * F;
    __shared__ uint4v_t lds[2][R * 16];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, lr = lane & 15, lg = lane >> 4;
    const int64_t lt = xcd_tile((int64_t)a.max_tiles * a.splits);
    if (lt >= (int64_t)a.max_tiles * a.splits) return;
    const int split = (int)(lt / a.max_tiles), tile = (int)(lt % a.max_tiles);
    if (tile >= a.counts[0]) return;
    const int4 td = a.tiles[tile];
    if (td.z >= a.count) return;
    const int64_t j0 = (int64_t)blockIdx.y * 128;              // ranks j0 .. j0 + 16 F
    const int64_t steps = (a.L + S - 1) / S, s0 = steps * split / a.splits, s1 = steps * (split + 1) / a.splits;
    const int ch = tid & 15, rr = tid >> 4;
    const T *px[4], *qx[F];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        px[i] = static_cast<const T*>(a.P) + (int64_t)a.order[td.x + std::min(rr + 16 * i, td.y - 1)] * a.ldp;
#pragma unroll
    for (int i = 0; i < F; ++i)
        qx[i] = static_cast<const T*>(a.Q) + ((int64_t)td.z * a.k + std::min(j0 + rr + 16 * i, a.k - 1)) * a.L;
    uint4v_t vp[4], vq[F];
    auto load = [&](int64_t s) {
        const int64_t c = s * S + ch * E;
#pragma unroll
        for (int i = 0; i < 4; ++i) vp[i] = load_zero16(px[i], c, a.L);
#pragma unroll
        for (int i = 0; i < F; ++i) vq[i] = load_zero16(qx[i], c, a.L);
    };
    auto put = [&](int buf) {
#pragma unroll
        for (int i = 0; i < 4; ++i) lds[buf][(rr + 16 * i) * 16 + (ch ^ rr)] = vp[i];
#pragma unroll
        for (int i = 0; i < F; ++i) lds[buf][(kTile + rr + 16 * i) * 16 + (ch ^ rr)] = vq[i];
    };
    float4_t acc[F];
#pragma unroll
    for (int f = 0; f < F; ++f) acc[f] = zero_accv<float4_t>();
    if (s0 < s1) {
        load(s0);
        put(0);
    }
    __syncthreads();
    for (int64_t s = s0; s < s1; ++s) {
        const int buf = (int)(s - s0) & 1;
        if (s + 1 < s1) load(s + 1);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint4v_t x = lds[buf][(16 * wave + lr) * 16 + ((4 * q + lg) ^ lr)];
#pragma unroll
            for (int f = 0; f < F; ++f)
                acc[f] = mma16<T>(lds[buf][(kTile + 16 * f + lr) * 16 + ((4 * q + lg) ^ lr)], x, acc[f]);
        }
        if (s + 1 < s1) put(buf ^ 1);
        __syncthreads();
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
// an adapter.
__global__ __launch_bounds__(256) void k_adapter_join(AdapterDown a, const int* __restrict__ key, const float* __restrict__ scale,
                                                      float* __restrict__ H) {
    const int64_t step = (int64_t)gridDim.x * 256;
    for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < a.rows * a.k; e += step) {
        const int64_t p = e / a.k, j = e % a.k;
        float s = 0.0f;
        const int id = key[p];
        if (id < a.count) {
            for (int q = 0; q < a.splits; ++q) s += a.part[(q * a.rows + p) * a.kp + j];
            if (scale) s *= scale[id];
        }
        H[(int64_t)a.order[p] * a.k + j] = s;
    }
}

// ---- up: O = base + c H Q^T ------------------------------------------------------------
// One workgroup of 4 waves: a tile of 64 rows and `cols` columns, 128 at a time, of them
// 32 a wave.  H (as kParts values) lies in LDS, rows of Q (N x L x k) come straight from
// L2 as operands; results cross LDS so that whole 16-byte pieces of rows are stored.
template <typename T>
__global__ __launch_bounds__(256) void k_adapter_up(AdapterUp a, int KS) {
    constexpr int E = kVec<T>, P = kParts<T>, OP = 132;
    extern __shared__ uint4v_t dyn[];
    __shared__ float out[kTile * OP];
    __shared__ float factor[kTile];
    __shared__ int rowof[kTile];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, lr = lane & 15, lg = lane >> 4;
    const int64_t lt = xcd_tile((int64_t)a.max_tiles * a.chunks);
    if (lt >= (int64_t)a.max_tiles * a.chunks) return;
    const int tile = (int)(lt / a.chunks);
    if (tile >= a.counts[0]) return;
    const int4 td = a.tiles[tile];
    const int64_t c0 = lt % a.chunks * a.cols, c1 = std::min(a.L, c0 + a.cols);
    const bool has = td.z < a.count;
    if (!has && a.base == a.O && a.ldb == a.ldo) return;
    const int pitch = 4 * KS + 1;                                   // chunks of a row of H
    if (tid < kTile) rowof[tid] = a.order[td.x + std::min(tid, td.y - 1)];
    if (has) {
        // four threads a row
        const int row = tid >> 2, part = tid & 3;
        const float* h = a.H + (int64_t)a.order[td.x + std::min(row, td.y - 1)] * a.k;
        unsigned amax = 0;
        if (__is_same(T, half_t)) {
            for (int64_t j = part; j < a.k; j += 4) amax = std::max(amax, __float_as_uint(h[j]) & 0x7FFFFFFFu);
            amax = std::max(amax, (unsigned)__shfl_xor((int)amax, 1, 64));
            amax = std::max(amax, (unsigned)__shfl_xor((int)amax, 2, 64));
        }
        const float sc = range_scale<T>(amax);
        if (part == 0) factor[row] = (a.scale ? a.scale[td.z] : 1.0f) / sc;
        for (int q = part; q < 4 * KS; q += 4) {
            uint4v_t v[P];
#pragma unroll
            for (int p = 0; p < P; ++p) v[p] = uint4v_t{0, 0, 0, 0};
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int64_t j = (int64_t)q * E + e;
                unsigned b[P];
                split_value<T>(j < a.k ? h[j] * sc : 0.0f, b);
#pragma unroll
                for (int p = 0; p < P; ++p) set_bits<T>(v[p], e, b[p]);
            }
#pragma unroll
            for (int p = 0; p < P; ++p) dyn[(p * kTile + row) * pitch + q] = v[p];
        }
    }
    __syncthreads();
    const T* Q = static_cast<const T*>(a.Q) + (int64_t)(has ? td.z : 0) * a.L * a.k;
    for (int64_t c = c0; c < c1; c += 128) {
        // the base of this thread's pieces: rows tid / (128 / E) + 2 E i
        constexpr int CH = 128 / E, RS = 256 / CH, NI = kTile / RS;
        const int ch = tid % CH, r0 = tid / CH;
        const int64_t cc = c + ch * E;
        uint4v_t b[NI];
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            b[i] = uint4v_t{0, 0, 0, 0};
            if (a.base && r0 + RS * i < td.y && cc < c1)
                b[i] = load_zero16(static_cast<const T*>(a.base) + rowof[r0 + RS * i] * a.ldb, cc, a.L);
        }
        float4_t acc[2][4];
        if (has) {
#pragma unroll
            for (int f = 0; f < 2; ++f)
#pragma unroll
                for (int g = 0; g < 4; ++g) acc[f][g] = zero_accv<float4_t>();
            for (int s = 0; s < KS; ++s) {
                uint4v_t q[2];
#pragma unroll
                for (int f = 0; f < 2; ++f)
                    q[f] = load_zero16(Q + std::min(c + 32 * wave + 16 * f + lr, a.L - 1) * a.k, (int64_t)s * kStep<T> + lg * E, a.k);
#pragma unroll
                for (int g = 0; g < 4; ++g)
#pragma unroll
                    for (int p = P - 1; p >= 0; --p) {
                        const uint4v_t h = dyn[(p * kTile + 16 * g + lr) * pitch + 4 * s + lg];
#pragma unroll
                        for (int f = 0; f < 2; ++f) acc[f][g] = mma16<T>(q[f], h, acc[f][g]);
                    }
            }
#pragma unroll
            for (int f = 0; f < 2; ++f)
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    *reinterpret_cast<float4_t*>(&out[(16 * g + lr) * OP + 32 * wave + 16 * f + 4 * lg]) = acc[f][g];
            __syncthreads();
        }
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const int row = r0 + RS * i;
            if (row < td.y && cc < c1) {
                if (has) {
                    float y[E];
#pragma unroll
                    for (int e = 0; e < E; ++e) y[e] = elem<T>(b[i], e) + factor[row] * out[row * OP + ch * E + e];
                    b[i] = pack16<T>(y);
                }
                T* o = static_cast<T*>(a.O) + rowof[row] * a.ldo + cc;
                if (cc + E <= a.L) {
                    store16_once(o, b[i]);
                } else {
#pragma unroll
                    for (int e = 0; e < E; ++e)
                        if (cc + e < a.L) o[e] = from_f32<T>(elem<T>(b[i], e));
                }
            }
        }
        if (has) __syncthreads();
    }
}

// ---- outer: sums over rows -------------------------------------------------------------
// H and dH turned for the outer products: [value][rank][position] per source, each run's
// ranks scaled by a power of two of their own (1 / scale[run][rank] undoes it).
template <typename T>
__global__ __launch_bounds__(256) void k_adapter_turn(AdapterTurn a) {
    constexpr int P = kParts<T>;
    __shared__ float tile[16][kRun + 1];
    __shared__ unsigned red[16][16];
    const int run = blockIdx.x, tid = threadIdx.x;
    if (run >= a.counts[1]) return;
    const int4 rd = a.runs[run];
    const int j0 = blockIdx.y * 16;
    const float* H = blockIdx.z ? a.H[1] : a.H[0];
    T* out = static_cast<T*>(blockIdx.z ? a.out[1] : a.out[0]);
    float* inv = blockIdx.z ? a.inv[1] : a.inv[0];
    const int j = tid & 15, g = tid >> 4;
    unsigned amax = 0;
    for (int p = g; p < rd.y; p += 16) {
        const float x = j0 + j < a.k ? H[(int64_t)a.order[rd.x + p] * a.k + j0 + j] : 0.0f;
        tile[j][p] = x;
        amax = std::max(amax, __float_as_uint(x) & 0x7FFFFFFFu);
    }
    red[g][j] = amax;
    __syncthreads();
    // 16 threads a rank
    const int jj = tid >> 4, l = tid & 15;
    amax = 0;
#pragma unroll
    for (int q = 0; q < 16; ++q) amax = std::max(amax, red[q][jj]);
    const float sc = range_scale<T>(amax);
    if (l == 0) inv[(int64_t)run * a.kp + j0 + jj] = 1.0f / sc;
    for (int p = l; p < rd.y; p += 16) {
        unsigned b[P];
        split_value<T>(tile[jj][p] * sc, b);
#pragma unroll
        for (int q = 0; q < P; ++q) {
            T* o = out + ((int64_t)q * a.kp + j0 + jj) * a.ldt + rd.x + p;
            if constexpr (sizeof(T) == 4) *o = __uint_as_float(b[q]);
            else *o = __builtin_bit_cast(T, (unsigned short)b[q]);
        }
    }
}

// G = sum over a run's rows of P_row x H_row.  One workgroup of 4 waves: 128 columns of P,
// of them 32 a wave, and up to 16 F ranks; steps of 64 rows of P go through
// registers to one of two LDS buffers.  COLS: G is k x L (else L x k).
template <typename T, int F, bool COLS>
__global__ __launch_bounds__(256) void k_adapter_outer(AdapterOuter a) {
    constexpr int E = kVec<T>, P = kParts<T>, CH = 128 / E, RS = 256 / CH, NI = 64 / RS, KV = kStep<T>;
    constexpr int PITCH = 128 + (sizeof(T) == 4 ? 4 : 16);
    __shared__ alignas(16) T lds[2][64 * PITCH];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, lr = lane & 15, lg = lane >> 4;
    const int64_t lt = xcd_tile((int64_t)a.max_runs * a.tiles_l);
    if (lt >= (int64_t)a.max_runs * a.tiles_l) return;
    const int run = (int)(lt / a.tiles_l);
    if (run >= a.counts[1]) return;
    const int4 rd = a.runs[run];
    const int64_t c0 = lt % a.tiles_l * 128, j0 = (int64_t)blockIdx.y * 128;
    const int ch = tid % CH, r0 = tid / CH, n = rd.y;
    uint4v_t v[NI];
    auto load = [&](int p0) {
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const int p = p0 + r0 + RS * i;
            v[i] = uint4v_t{0, 0, 0, 0};
            if (p < n && c0 + ch * E < a.L)
                v[i] = load_zero16(static_cast<const T*>(a.P) + (int64_t)a.order[rd.x + p] * a.ldp, c0 + ch * E, a.L);
        }
    };
    auto put = [&](int buf) {
#pragma unroll
        for (int i = 0; i < NI; ++i) *reinterpret_cast<uint4v_t*>(&lds[buf][(r0 + RS * i) * PITCH + ch * E]) = v[i];
    };
    float4_t acc[2][F];
#pragma unroll
    for (int f = 0; f < F; ++f) acc[0][f] = acc[1][f] = zero_accv<float4_t>();
    load(0);
    put(0);
    __syncthreads();
    for (int p0 = 0; p0 < n; p0 += 64) {
        const int buf = p0 / 64 & 1;
        if (p0 + 64 < n) load(p0 + 64);
#pragma unroll
        for (int s = 0; s < 64 / KV; ++s) {
            uint4v_t x[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int c = 32 * wave + 16 * h;
                if constexpr (sizeof(T) == 4) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[h][e] = __float_as_uint(lds[buf][(s * KV + 4 * lg + e) * PITCH + c + lr]);
                } else {
                    // the transposing read: lane i of 16 receives column i of four rows
                    typedef short s4_t __attribute__((ext_vector_type(4)));
                    const T* p = &lds[buf][(s * KV + 8 * lg + (lr >> 2)) * PITCH + c + 4 * (lr & 3)];
                    const s4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4_t*)(p));
                    const s4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4_t*)(p + 4 * PITCH));
                    x[h] = __builtin_bit_cast(uint4v_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
                }
            }
            const int64_t at = p0 + s * KV + lg * E;
#pragma unroll
            for (int f = 0; f < F; ++f)
#pragma unroll
                for (int q = P - 1; q >= 0; --q) {
                    // zero past the run: the positions behind it are another's
                    const T* row = static_cast<const T*>(a.H) + ((int64_t)q * a.kp + std::min<int64_t>(j0 + 16 * f + lr, a.kp - 1)) * a.ldt + rd.x;
                    const uint4v_t h = load_zero16(row, at, n);
#pragma unroll
                    for (int w = 0; w < 2; ++w) acc[w][f] = COLS ? mma16<T>(x[w], h, acc[w][f]) : mma16<T>(h, x[w], acc[w][f]);
                }
        }
        if (p0 + 64 < n) put(buf ^ 1);
        __syncthreads();
    }
    const float c = a.scale ? a.scale[rd.z] : 1.0f;
    const float* inv = a.inv + (int64_t)run * a.kp;
    auto store = [&](int64_t l, int64_t j, float y) {
        if (l >= a.L || j >= a.k) return;
        y *= c * inv[j];
        const int64_t at = COLS ? j * a.L + l : l * a.k + j;
        if (rd.w < 0) static_cast<T*>(a.G)[(int64_t)rd.z * a.L * a.k + at] = from_f32<T>(y);
        else a.part[(int64_t)rd.w * a.L * a.k + at] = y;
    };
#pragma unroll
    for (int w = 0; w < 2; ++w)
#pragma unroll
        for (int f = 0; f < F; ++f)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int64_t l = c0 + 32 * wave + 16 * w, j = j0 + 16 * f;
                if (COLS) store(l + 4 * lg + e, j + lr, acc[w][f][e]);
                else store(l + lr, j + 4 * lg + e, acc[w][f][e]);
            }
}

// Gradients of adapters with several runs (their sum, in order) or none (0).
template <typename T>
__global__ __launch_bounds__(256) void k_adapter_sum(const int2* __restrict__ runs_of, const float* __restrict__ part,
                                                     int64_t per, T* __restrict__ G, int64_t count) {
    for (int64_t id = blockIdx.y; id < count; id += gridDim.y) {
        const int2 r = runs_of[id];
        if (r.y == 1) continue;
        for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < per; e += (int64_t)gridDim.x * 256) {
            float s = 0.0f;
            for (int q = 0; q < r.y; ++q) s += part[(r.x + q) * per + e];
            G[id * per + e] = from_f32<T>(s);
        }
    }
}

// Used adapters transposed: N x R x C to N x C x R.
template <typename T>
__global__ __launch_bounds__(256) void k_adapter_flip(const int2* __restrict__ runs_of, const T* __restrict__ in, int64_t R, int64_t C,
                                                      T* __restrict__ out, int64_t count, int64_t tiles_c) {
    __shared__ T tile[64][65];
    const int64_t id = blockIdx.y;
    const int64_t r0 = blockIdx.x / tiles_c * 64, c0 = blockIdx.x % tiles_c * 64;
    const int x = threadIdx.x & 63, y = threadIdx.x >> 6;
    for (int64_t q = id; q < count; q += gridDim.y) {
        if (runs_of[q].y == 0) continue;
        __syncthreads();
        for (int i = y; i < 64 && r0 + i < R; i += 4)
            if (c0 + x < C) tile[i][x] = in[(q * R + r0 + i) * C + c0 + x];
        __syncthreads();
        for (int i = y; i < 64 && c0 + i < C; i += 4)
            if (r0 + x < R) out[(q * C + c0 + i) * R + r0 + x] = tile[x][i];
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
        max_slots = 2 * (rows / kRun) + 1;
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
    hipLaunchKernelGGL(k_adapter_sort, dim3(1), dim3(kSortThreads), 0, st, a, sort_passes(a.count));
    return hipGetLastError();
}

unsigned strided(int64_t items) { return (unsigned)std::max<int64_t>(1, std::min<int64_t>((items + 255) / 256, 65536)); }

template <typename T, int F> void down_f(const AdapterDown& a, hipStream_t st) {
    hipLaunchKernelGGL((k_adapter_down<T, F>), dim3(xcd_grid((int64_t)a.max_tiles * a.splits), (unsigned)((a.k + 127) / 128)),
                       dim3(256), 0, st, a);
}
// H = P Q^T, times the adapters' factors where `scale` is given.
template <typename T>
hipError_t run_down(const AdapterPlan& p, const AdapterSort& s, const void* P, int64_t ldp, int64_t L, const void* Q,
                    const float* scale, float* part, float* H, hipStream_t st) {
    AdapterDown a{};
    a.P = P;
    a.ldp = ldp;
    a.L = L;
    a.Q = Q;
    a.k = p.k;
    a.kp = p.kp;
    a.rows = p.rows;
    a.count = p.count;
    const int odd = sort_passes(p.count) & 1;
    a.order = s.order[odd];
    a.tiles = s.tiles;
    a.counts = s.counts;
    a.max_tiles = (int)p.max_tiles;
    a.splits = p.down_splits(L, sizeof(T));
    a.part = part;
    {
        KernelTimer t("adapter_down", st);
        const int64_t f = (std::min<int64_t>(p.k, 128) + 15) / 16;
        if (f <= 1) down_f<T, 1>(a, st);
        else if (f <= 2) down_f<T, 2>(a, st);
        else if (f <= 4) down_f<T, 4>(a, st);
        else down_f<T, 8>(a, st);
    }
    KernelTimer t("adapter_join", st);
    hipLaunchKernelGGL(k_adapter_join, dim3(strided(p.rows * p.k)), dim3(256), 0, st, a, s.key[odd], scale, H);
    return hipGetLastError();
}

template <typename T>
hipError_t run_up(const AdapterPlan& p, const AdapterSort& s, const float* H, const void* Q, int64_t L, const float* scale,
                  const void* base, int64_t ldb, void* O, int64_t ldo, hipStream_t st) {
    AdapterUp a{};
    a.H = H;
    a.Q = Q;
    a.L = L;
    a.k = p.k;
    a.count = p.count;
    a.scale = scale;
    a.base = base;
    a.ldb = ldb;
    a.O = O;
    a.ldo = ldo;
    a.order = s.order[sort_passes(p.count) & 1];
    a.tiles = s.tiles;
    a.counts = s.counts;
    a.max_tiles = (int)p.max_tiles;
    // about 1024 workgroups, whole steps of 128 columns each
    const int64_t steps = (L + 127) / 128;
    const int64_t chunks = std::min(steps, std::max<int64_t>(1, 1024 / p.max_tiles));
    a.cols = (steps + chunks - 1) / chunks * 128;
    a.chunks = (int)((L + a.cols - 1) / a.cols);
    const int KS = (int)((p.k + kStep<T> - 1) / kStep<T>);
    const size_t lds = (size_t)kParts<T> * kTile * (4 * KS + 1) * 16;
    auto* kern = k_adapter_up<T>;
    if (lds + sizeof(float) * kTile * 140 > 65536) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kern),
                                                 hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return e;
    }
    KernelTimer t("adapter_up", st);
    hipLaunchKernelGGL(kern, dim3(xcd_grid((int64_t)a.max_tiles * a.chunks)), dim3(256), lds, st, a, KS);
    return hipGetLastError();
}

template <typename T, bool COLS> void outer_f(const AdapterOuter& a, hipStream_t st) {
    const dim3 grid(xcd_grid((int64_t)a.max_runs * a.tiles_l), (unsigned)((a.k + 127) / 128));
    const int64_t f = (std::min<int64_t>(a.k, 128) + 15) / 16;
    if (f <= 1) hipLaunchKernelGGL((k_adapter_outer<T, 1, COLS>), grid, dim3(256), 0, st, a);
    else if (f <= 2) hipLaunchKernelGGL((k_adapter_outer<T, 2, COLS>), grid, dim3(256), 0, st, a);
    else if (f <= 4) hipLaunchKernelGGL((k_adapter_outer<T, 4, COLS>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((k_adapter_outer<T, 8, COLS>), grid, dim3(256), 0, st, a);
}

// Batches of this many rows and fewer go row by row.
constexpr int64_t kFewRows = 64;

int64_t rows_splits(int64_t n, int prec) {
    const int64_t per = 64 * (prec == P32 ? 4 : 8);
    return (n + per - 1) / per;
}

// Where the parts of a call lie; ws == nullptr: their size alone.
struct ApplySlices {
    AdapterSort sort;
    float *part, *H;
};
ApplySlices apply_slices(const AdapterArgs& a, Slices& s) {
    ApplySlices o{};
    if (a.rows <= kFewRows) {
        o.part = s.take<float>(rows_splits(a.n, a.prec) * a.rows * a.k);
        return o;
    }
    const AdapterPlan p(a.rows, a.count, a.k);
    o.sort = take_sort(s, p, a.ids);
    o.part = s.take<float>(p.down_splits(a.n, elem_bytes(a.prec)) * a.rows * p.kp);
    o.H = a.hidden ? a.hidden : s.take<float>(a.rows * a.k);
    return o;
}

template <typename T> hipError_t apply_t(const AdapterArgs& a, Workspace& ws, hipStream_t st) {
    Slices s{&ws};
    const ApplySlices o = apply_slices(a, s);
    if (ws.overrun) return hipErrorOutOfMemory;
    if (a.rows <= kFewRows) {
        const int splits = (int)rows_splits(a.n, a.prec);
        {
            KernelTimer t("adapter_down_rows", st);
            hipLaunchKernelGGL((k_adapter_down_rows<T, 1>), dim3(splits, (unsigned)a.rows), dim3(256), 0, st, a, o.part);
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
    hipError_t e = run_sort(o.sort, st);
    if (e == hipSuccess) e = run_down<T>(p, o.sort, a.X, a.ldx, a.n, a.A, nullptr, o.part, o.H, st);
    if (e == hipSuccess) e = run_up<T>(p, o.sort, o.H, a.B, a.m, a.scale, a.base, a.ldb, a.Y, a.ldy, st);
    return e;
}

struct GradSlices {
    AdapterSort sort;
    float *part, *dH, *sums, *inv[2];
    void *Bt, *At, *turned[2];
    int64_t ldt;
};
GradSlices grad_slices(const AdapterGradArgs& a, Slices& s) {
    const AdapterPlan p(a.rows, a.count, a.k);
    const int e = elem_bytes(a.prec), parts = e == 4 ? 1 : 2;
    GradSlices o{};
    o.sort = take_sort(s, p, a.ids);
    o.part = s.take<float>(p.down_splits(a.m, e) * a.rows * p.kp);
    o.dH = s.take<float>(a.rows * a.k);
    o.Bt = s.take<char>(a.count * a.m * a.k * e);
    o.At = a.dX ? s.take<char>(a.count * a.n * a.k * e) : nullptr;
    o.ldt = round_up(a.rows, 8) + 8;
    for (int q = 0; q < 2; ++q) {
        o.turned[q] = s.take<char>(parts * p.kp * o.ldt * e);
        o.inv[q] = s.take<float>(p.max_runs * p.kp);
    }
    o.sums = s.take<float>(p.max_slots * std::max(a.m, a.n) * a.k);
    return o;
}

template <typename T> hipError_t flip(const AdapterSort& s, const void* in, int64_t R, int64_t C, void* out, int64_t count, hipStream_t st) {
    const int64_t tc = (C + 63) / 64, tr = (R + 63) / 64;
    KernelTimer t("adapter_flip", st);
    hipLaunchKernelGGL(k_adapter_flip<T>, dim3((unsigned)(tc * tr), (unsigned)std::min<int64_t>(count, 65535)), dim3(256), 0, st,
                       s.runs_of, static_cast<const T*>(in), R, C, static_cast<T*>(out), count, tc);
    return hipGetLastError();
}

template <typename T> hipError_t grad_t(const AdapterGradArgs& a, Workspace& ws, hipStream_t st) {
    Slices sl{&ws};
    const GradSlices o = grad_slices(a, sl);
    if (ws.overrun) return hipErrorOutOfMemory;
    const AdapterPlan p(a.rows, a.count, a.k);
    hipError_t e = run_sort(o.sort, st);
    if (e == hipSuccess) e = flip<T>(o.sort, a.B, a.m, a.k, o.Bt, a.count, st);
    if (e == hipSuccess) e = run_down<T>(p, o.sort, a.dY, a.lddy, a.m, o.Bt, a.scale, o.part, o.dH, st);
    if (e == hipSuccess && a.dX) {
        e = flip<T>(o.sort, a.A, a.k, a.n, o.At, a.count, st);
        if (e == hipSuccess) e = run_up<T>(p, o.sort, o.dH, o.At, a.n, nullptr, a.base, a.ldb, a.dX, a.lddx, st);
    }
    if (e != hipSuccess || (!a.dA && !a.dB)) return e;
    AdapterTurn tn{};
    tn.H[0] = o.dH;
    tn.H[1] = a.hidden;
    for (int q = 0; q < 2; ++q) {
        tn.out[q] = o.turned[q];
        tn.inv[q] = o.inv[q];
    }
    tn.k = a.k;
    tn.kp = p.kp;
    tn.ldt = o.ldt;
    tn.order = o.sort.order[sort_passes(p.count) & 1];
    tn.runs = o.sort.runs;
    tn.counts = o.sort.counts;
    {
        KernelTimer t("adapter_turn", st);
        hipLaunchKernelGGL(k_adapter_turn<T>, dim3((unsigned)p.max_runs, (unsigned)(p.kp / 16), 2), dim3(256), 0, st, tn);
    }
    for (int q = 0; q < 2; ++q) {
        void* G = q ? a.dB : a.dA;
        if (!G) continue;
        AdapterOuter w{};
        w.P = q ? a.dY : a.X;
        w.ldp = q ? a.lddy : a.ldx;
        w.L = q ? a.m : a.n;
        w.H = o.turned[q];
        w.inv = o.inv[q];
        w.k = a.k;
        w.kp = p.kp;
        w.ldt = o.ldt;
        w.scale = q ? a.scale : nullptr;
        w.order = tn.order;
        w.runs = o.sort.runs;
        w.counts = o.sort.counts;
        w.max_runs = (int)p.max_runs;
        w.tiles_l = (int)((w.L + 127) / 128);
        w.part = o.sums;
        w.G = G;
        {
            KernelTimer t("adapter_outer", st);
            if (q) outer_f<T, false>(w, st);
            else outer_f<T, true>(w, st);
        }
        KernelTimer t("adapter_sum", st);
        const int64_t per = w.L * a.k;
        hipLaunchKernelGGL(k_adapter_sum<T>, dim3((unsigned)std::min<int64_t>((per + 255) / 256, 2048), (unsigned)std::min<int64_t>(a.count, 65535)),
                           dim3(256), 0, st, o.sort.runs_of, o.sums, per, static_cast<T*>(G), a.count);
    }
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
