// Distillation from a teacher's top logits: loss and gradient by the
// student's logits, one workgroup per row.
//
// With z the student's logits, q = softmax(z / T), and p the teacher's
// probabilities of its K named tokens (p_k = exp(t_k / T - lse)),
//   loss = w T^2 [ sum_k p_k (log p_k - log q_k) + r (log r - log Q) ],
//   dloss/dz_j = w T (P q_j - p_j)          for a named token j,
//                w T (P q_j - r q_j / Q)    for any other,   P = sum_k p_k + r.
// Without a given lse, lse = log sum_k exp(t_k / T), r = 0 and P = 1 (the teacher
// renormalized over the named tokens).  With the teacher's own lse, r =
// max(1 - sum_k p_k, 0) and Q = the student's mass outside the named tokens are
// one more class; P is above 1 where the named probabilities are (logits rounded
// after their lse was taken, a token named twice).  The row is then summed without
// the named tokens (a bitmap of them in LDS), relative to its own maximum: Q
// neither cancels nor underflows, and the K named ones are added to the whole sum
// afterwards.
//
// Bound by memory: the logits are read once and the gradient written once.  A
// row stays in registers between the maximum, the sum and the gradient (up to
// 16 vectors of 16 bytes a thread); longer rows are read again.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "head_device.h"

namespace lrc {

namespace {

constexpr int kSlab = 1 << 18;           // logits whose bitmap is held at a time
constexpr float kNegInf = -__builtin_inff();

enum { FORWARD = 0, BOTH = 1, BACKWARD = 2 };

// log x, to a few 2^-26: the logarithm of the significand alone is binary32 (one of x
// would carry half an ulp of its size, 2.4e-7 for sums of a few hundred).
__device__ __forceinline__ double log_of(double x) {
    int e;
    double m = frexp(x, &e);                // [0.5, 1)
    if (m < 0.70710678) {
        m *= 2.0;
        e -= 1;
    }
    if (!(m > 0.0 && m < 2.0)) return (double)logf((float)x);
    const float f = (float)m;
    return (double)e * 0.6931471805599453 + (double)logf(f) + (m - (double)f);
}
// exp x, to a few 2^-24 of itself: the argument's whole part stays out of binary32.
__device__ __forceinline__ double exp_of(double x) {
    const double y = x * 1.4426950408889634;
    if (!(y > -1000.0 && y < 1000.0)) return (double)__builtin_amdgcn_exp2f((float)y);
    const double n = rint(y);
    return ldexp((double)__builtin_amdgcn_exp2f((float)(y - n)), (int)n);
}

// A value that every lane of the wave holds, in scalar registers: the row keeps the others.
__device__ __forceinline__ double uniform(double x) {
    const long long u = __double_as_longlong(x);
    const unsigned lo = __builtin_amdgcn_readfirstlane((unsigned)u), hi = __builtin_amdgcn_readfirstlane((unsigned)(u >> 32));
    return __longlong_as_double((long long)((unsigned long long)hi << 32 | lo));
}

__device__ __forceinline__ float uniform(float x) {
    return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x)));
}

template <typename T>
__device__ void zero_row(T* out, int V, int nt) {
    const int full = V / kVec<T>;
    for (int q = threadIdx.x; q < full; q += nt) store16(out + (int64_t)q * kVec<T>, uint4v_t{0, 0, 0, 0});
    if ((int)threadIdx.x < V % kVec<T>) out[full * kVec<T> + threadIdx.x] = from_f32<T>(0.0f);
}

}  // namespace

// NV vectors a thread hold the row's vocab / kVec whole vectors (thread t of the
// workgroup those at t, t + NT, ..), or NV = 0: any length, read again for the
// gradient.  The vocab % kVec last logits are one a thread.  Dynamic LDS: the K
// ids, student and teacher logits, the bitmap.  What concerns the named tokens alone is
// done by every wave for itself: five barriers a row.
template <typename T, int MODE, int NV, int NT>
__global__ __launch_bounds__(NT, NV <= 4 ? 8 : NV <= 8 ? 7 : 4) void k_distill_row(DistillArgs a, float* __restrict__ loss, float* __restrict__ stats,
                                                    const float* __restrict__ dloss, T* grad, int64_t ldg) {
    extern __shared__ int lds[];
    __shared__ float red[2][NT / 64];
    __shared__ int dup;
    constexpr int E = kVec<T>;
    const int t = threadIdx.x, lane = t & 63;
    const int64_t i = blockIdx.x;
    const int V = (int)a.vocab, K = (int)a.K, full = V / E, over = V % E;
    int* ids = lds;
    float* zk = reinterpret_cast<float*>(ids + K);
    float* tk = zk + K;
    unsigned* named = reinterpret_cast<unsigned*>(tk + K);
    const T* row = static_cast<const T*>(a.logits) + i * a.ld;
    T* out = MODE == FORWARD ? nullptr : grad + i * ldg;
    const float w = a.weight ? a.weight[i] : 1.0f;
    const bool tail = a.teacher_lse != nullptr;
    auto nothing = [&] {
        if (MODE != BACKWARD && t == 0) loss[i] = 0.0f;
        if (MODE != BACKWARD && stats && t < 4) stats[i * 4 + t] = 0.0f;
        if (MODE != FORWARD) zero_row(out, V, NT);
    };
    if (w == 0.0f) {                        // a row that does not count
        nothing();
        return;
    }
    uint4v_t held[NV > 0 ? NV : 1];
    if (NV > 0) {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            held[v] = uint4v_t{kNegInfPair<T>, kNegInfPair<T>, kNegInfPair<T>, kNegInfPair<T>};
            if (v * NT + t < full) held[v] = load16_once(row + v * NT * E + t * E);
        }
    }
    float last = t < over ? (float)row[full * E + t] : kNegInf;
    // the named tokens: id, the student's logit; a bit for each
    if (t == 0) dup = 0;
    for (int k = t; k < K; k += NT) {
        const int64_t id = a.ids[i * K + k];
        const bool ok = id >= 0 && id < V;
        ids[k] = ok ? (int)id : -1;
        zk[k] = ok ? (float)row[id] : 0.0f;
        tk[k] = load_as_f32(a.top, i * K + k, a.tprec);
    }
    auto mark = [&](int j0, int j1) {
        for (int q = t; q < (j1 - j0 + 31) / 32; q += NT) named[q] = 0u;
        __syncthreads();
        for (int k = t; k < K; k += NT) {
            const int id = ids[k];
            if (id >= j0 && id < j1) {
                const unsigned bit = 1u << ((id - j0) & 31);
                if (atomicOr(&named[(id - j0) >> 5], bit) & bit) dup = 1;
            }
        }
        __syncthreads();
    };
    auto slab_end = [&](int j0) { return V - j0 > kSlab ? j0 + kSlab : V; };
    if (NV > 0) mark(0, V);
    else __syncthreads();

    // the teacher: differences of its logits in binary64, K values a row
    const double invT = uniform(1.0 / (double)a.temperature);
    auto teacher = [&](int k) { return (double)tk[k] * invT; };
    double lse;
    if (tail) {
        lse = (double)a.teacher_lse[i];
    } else {
        float mx = kNegInf;
        bool nan = false;
        for (int k = lane; k < K; k += 64)
            if (ids[k] >= 0) {
                mx = __builtin_fmaxf(mx, tk[k]);
                nan |= tk[k] != tk[k];
            }
        mx = wave_max(mx);
        nan = __builtin_amdgcn_ballot_w64(nan) != 0;
        if (mx == kNegInf && !nan) {        // the teacher names nothing
            nothing();
            return;
        }
        const double m = (double)mx * invT;
        double x = 0.0;
        for (int k = lane; k < K; k += 64)
            if (ids[k] >= 0) x += exp_of(teacher(k) - m);
        lse = uniform(m + log_of(wave_sum(x)));
    }
    auto prob = [&](int k) { return ids[k] >= 0 ? exp_of(teacher(k) - lse) : 0.0; };
    double r = 0.0, P = 1.0;
    if (tail) {
        double sp = 0.0;
        for (int k = lane; k < K; k += 64) sp += prob(k);
        sp = uniform(wave_sum(sp));
        r = uniform(sp < 1.0 ? 1.0 - sp : (sp != sp ? sp : 0.0));
        P = sp < 1.0 ? 1.0 : sp;
    }

    // m, s: maximum and sum of exp((z - m) / T) over the row, without the named
    // tokens when they are a class of their own (tail)
    const float c = uniform(kLog2e / a.temperature);
    float m = kNegInf, s = 0.0f;
    auto hide = [&](uint4v_t& v, int j, int j0) {       // named tokens of the vector at j to -infinity
        const unsigned bits = named[(j - j0) >> 5] >> ((j - j0) & 31) & ((1u << E) - 1u);
        if (bits) {
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (bits >> e & 1u) set_bits<T>(v, e, kNegInfBits<T>);
        }
    };
    auto hide_last = [&](int j0) {
        const int j = full * E + t - j0;
        if (tail && t < over && (named[j >> 5] >> (j & 31) & 1u)) last = kNegInf;
    };
    auto weigh = [&](float l) { return __builtin_amdgcn_exp2f((l - m) * c); };
    if (MODE == BACKWARD) {
        m = stats[i * 4 + 2];
        s = stats[i * 4 + 3];
    } else if (NV > 0) {
        hide_last(0);
        m = last;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            if (tail && v * NT + t < full) hide(held[v], (v * NT + t) * E, 0);
#pragma unroll
            for (int e = 0; e < E; ++e) m = __builtin_fmaxf(m, elem<T>(held[v], e));
        }
        m = uniform(block_max<NT>(m, red[0]));
        if (m == kNegInf) m = 0.0f;
        stay(held);
        s = weigh(last);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
#pragma unroll
            for (int e = 0; e < E; ++e) s += weigh(elem<T>(held[v], e));
        }
        s = uniform(block_add<NT>(s, red[1]));
        stay(held);
    } else {
        for (int j0 = 0; j0 < V; j0 = slab_end(j0)) {
            const int j1 = slab_end(j0);
            mark(j0, j1);
            if (j1 == V) {
                hide_last(j0);
                const float mx = __builtin_fmaxf(m, last);
                if (mx != kNegInf) {
                    s = s * __builtin_amdgcn_exp2f((m - mx) * c) + __builtin_amdgcn_exp2f((last - mx) * c);
                    m = mx;
                }
            }
            for (int x = t; x < (j1 - j0) / E; x += NT) {
                const int j = j0 + x * E;
                uint4v_t v = load16(row + j);
                if (tail) hide(v, j, j0);
                float mx = m;
#pragma unroll
                for (int e = 0; e < E; ++e) mx = __builtin_fmaxf(mx, elem<T>(v, e));
                if (mx > m) {
                    s *= __builtin_amdgcn_exp2f((m - mx) * c);
                    m = mx;
                }
                const float base = m == kNegInf ? 0.0f : m;
#pragma unroll
                for (int e = 0; e < E; ++e) s += __builtin_amdgcn_exp2f((elem<T>(v, e) - base) * c);
            }
            __syncthreads();
        }
        if (last != last) s = last;
        float mx = block_max<NT>(m, red[0]);
        if (mx == kNegInf) mx = 0.0f;
        if (m != kNegInf) s *= __builtin_amdgcn_exp2f((m - mx) * c);
        m = mx;
        s = block_add<NT>(s, red[1]);
    }

    // a token named twice counts once in the student's sum, and with both
    // probabilities in the gradient: `first` slots stand for their token
    auto first = [&](int k) {
        bool f = ids[k] >= 0;
        if (dup)
            for (int q = 0; q < k; ++q) f &= ids[q] != ids[k];
        return f;
    };
    // M, S: of the whole row; with tail S = rest + x, x the named tokens' part
    float M = m;
    double S = s, x = 0.0, rest = 0.0;
    if (MODE == BACKWARD) {
        if (NV == 0)
            for (int j0 = 0; j0 < V; j0 = slab_end(j0)) {
                mark(j0, slab_end(j0));
                __syncthreads();
            }
        M = stats[i * 4];
        (tail ? x : S) = stats[i * 4 + 1];
    } else if (tail) {
        float mx = s > 0.0f ? m : kNegInf;
        for (int k = lane; k < K; k += 64)
            if (ids[k] >= 0) mx = __builtin_fmaxf(mx, zk[k]);
        mx = wave_max(mx);
        M = uniform(mx == kNegInf ? 0.0f : mx);
        for (int k = lane; k < K; k += 64)
            if (first(k)) x += (double)__builtin_amdgcn_exp2f((zk[k] - M) * c);
        x = uniform(wave_sum(x));
    }
    if (tail) {
        rest = uniform(s == 0.0f ? 0.0 : (double)s * (double)__builtin_amdgcn_exp2f((m - M) * c));
        S = uniform(rest + x);
    }
    // The loss and the statistics, by the first wave while the others go on to the
    // gradient; at the end where a workgroup is short and many share a compute unit
    // (4096 x 8000 38.9 us against 39.7; 64 x 65536 17.0 against 16.5).
    constexpr bool kLast = MODE == BOTH && NV == 4;
    auto finish = [&] {
        // Where the rest is most of the student's mass, log Q = -log(1 + x / rest) and log S
        // = log rest - log Q: both terms of the loss share the error of log s, and do not
        // lose their small difference to two logarithms of the whole sum.
        const double logrest = uniform((double)(m - M) * invT + log_of((double)s));
        const bool most = tail && x < rest;
        const double l = uniform(log_of(most ? 1.0 + x * (double)__builtin_amdgcn_rcpf((float)rest) : S));
        const double logQ = most ? -l : logrest - l, logS = most ? logrest + l : l;
        double kl = 0.0;
        for (int k = lane; k < K; k += 64) {
            const double p = prob(k);
            if (!(p == 0.0)) kl += p * ((teacher(k) - lse) - ((double)(zk[k] - M) * invT - logS));
        }
        kl = wave_sum(kl);
        if (t == 0) {
            if (r != 0.0)
                kl += r * (log_of(r) - logQ);
            loss[i] = (float)((double)w * (double)a.temperature * (double)a.temperature * kl);
        }
        if (stats && t < 4) stats[i * 4 + t] = t == 0 ? M : t == 1 ? (float)(tail ? x : S) : t == 2 ? m : s;
    };
    if (MODE != BACKWARD && !kLast && t < 64) finish();
    if (MODE == FORWARD) return;

    const double scale = uniform((double)w * (double)a.temperature * (double)(MODE == BACKWARD && dloss ? dloss[i] : 1.0f));
    const bool sound = S > 0.0 && S <= 1e300;            // else the row holds NaN or nothing
    double coef = scale * P * (double)__builtin_amdgcn_exp2f((m - M) * c) / S;
    if (r != 0.0) coef -= s > 0.0f ? scale * r / (double)s : 0.0;
    const float cf = uniform(sound ? (float)coef : __builtin_nanf(""));
    auto put = [&](T* at, const uint4v_t& v) {
        float g[E];
#pragma unroll
        for (int e = 0; e < E; ++e) g[e] = weigh(elem<T>(v, e)) * cf;
        store16_once(at, pack16<T>(g));
    };
    if (t < over) out[full * E + t] = from_f32<T>(weigh(last) * cf);
    if (NV > 0) {
#pragma unroll
        for (int v = 0; v < NV; ++v)
            if (v * NT + t < full) put(out + v * NT * E + t * E, held[v]);
    } else {
        for (int q = t; q < full; q += NT) put(out + (int64_t)q * E, load16_once(row + (int64_t)q * E));
    }
    __syncthreads();
    // the named tokens over it
    for (int k = t; k < K; k += NT) {
        if (!first(k)) continue;
        double p = prob(k);
        if (dup)
            for (int q = k + 1; q < K; ++q) p += ids[q] == ids[k] ? prob(q) : 0.0;
        const double q = sound ? P * (double)__builtin_amdgcn_exp2f((zk[k] - M) * c) / S : (double)__builtin_nanf("");
        out[ids[k]] = from_f32<T>((float)(scale * (q - p)));
    }
    if (kLast && t < 64) finish();
}

namespace {
template <typename T, int MODE, int NV, int NT>
void launch_nv(const DistillArgs& a, float* loss, float* stats, const float* dloss, void* grad, int64_t ldg,
               hipStream_t st) {
    const size_t lds = (size_t)a.K * 12 + (size_t)((std::min<int64_t>(a.vocab, kSlab) + 31) / 32) * 4 + 8;
    hipLaunchKernelGGL((k_distill_row<T, MODE, NV, NT>), dim3((unsigned)a.rows), dim3(NT), lds, st, a, loss, stats,
                       dloss, (T*)grad, ldg);
}

// The step takes the smallest workgroup whose registers hold the row.  bfloat16, K =
// 64, both sides measured in turn: 4096 x 65536 215 us against 241 read twice, 2000 x
// 10007 30 against 45.  The forward and the backward pass read a row once and need
// no registers for it: workgroups of 256 run more rows at a time (4096 x 65536
// forward 97 us against 130 with 1024 threads, 2000 x 10007 16 against 37, backward
// 23 against 29), those of 1024 suit few rows (64 x 65536 12 against 15, backward 10
// against 15) and the backward pass of long ones (4096 x 65536 204 against 219).
template <typename T, int MODE>
void launch_t(const DistillArgs& a, float* loss, float* stats, const float* dloss, void* grad, int64_t ldg,
              hipStream_t st) {
    const int64_t vecs = a.vocab / kVec<T>;
    if constexpr (MODE == BOTH) {
        if (vecs <= 256 * 4) launch_nv<T, MODE, 4, 256>(a, loss, stats, dloss, grad, ldg, st);
        else if (vecs <= 256 * 8) launch_nv<T, MODE, 8, 256>(a, loss, stats, dloss, grad, ldg, st);
        else if (vecs <= 256 * 16) launch_nv<T, MODE, 16, 256>(a, loss, stats, dloss, grad, ldg, st);
        else if (vecs <= 512 * 16) launch_nv<T, MODE, 16, 512>(a, loss, stats, dloss, grad, ldg, st);
        else if (vecs <= 1024 * 16) launch_nv<T, MODE, 16, 1024>(a, loss, stats, dloss, grad, ldg, st);
        else launch_nv<T, MODE, 0, 1024>(a, loss, stats, dloss, grad, ldg, st);
    } else {
        if (vecs <= 512 || (a.rows >= 1024 && (MODE == FORWARD || vecs <= 4096)))
            launch_nv<T, MODE, 0, 256>(a, loss, stats, dloss, grad, ldg, st);
        else
            launch_nv<T, MODE, 0, 1024>(a, loss, stats, dloss, grad, ldg, st);
    }
}

template <int MODE>
hipError_t launch_mode(const DistillArgs& a, float* loss, float* stats, const float* dloss, void* grad, int64_t ldg,
                       hipStream_t st) {
    return in_panels(a.rows, kRowPanel, [&](int64_t r, int64_t count) {
        auto from = [&](auto* x, int64_t each = 1) { return x ? x + r * each : x; };
        DistillArgs p = a;
        p.logits = static_cast<const char*>(a.logits) + r * a.ld * elem_bytes(a.prec);
        p.rows = count;
        p.ids = a.ids + r * a.K;
        p.top = static_cast<const char*>(a.top) + r * a.K * elem_bytes(a.tprec);
        p.teacher_lse = from(a.teacher_lse);
        p.weight = from(a.weight);
        void* g = from(static_cast<char*>(grad), ldg * elem_bytes(a.prec));
        float *l = from(loss), *s = from(stats, 4);
        const float* d = from(dloss);
        if (a.prec == P32) launch_t<float, MODE>(p, l, s, d, g, ldg, st);
        else if (a.prec == P16) launch_t<half_t, MODE>(p, l, s, d, g, ldg, st);
        else launch_t<bhalf_t, MODE>(p, l, s, d, g, ldg, st);
        return hipGetLastError();
    });
}
}  // namespace

hipError_t launch_distill(const DistillArgs& a, float* loss, float* stats, void* grad, int64_t ldg, hipStream_t st) {
    KernelTimer t(grad ? "distill_step" : "distill_forward", st);
    return grad ? launch_mode<BOTH>(a, loss, stats, nullptr, grad, ldg, st)
                : launch_mode<FORWARD>(a, loss, stats, nullptr, nullptr, 0, st);
}

hipError_t launch_distill_backward(const DistillArgs& a, const float* stats, const float* dloss, void* grad,
                                   int64_t ldg, hipStream_t st) {
    KernelTimer t("distill_backward", st);
    return launch_mode<BACKWARD>(a, nullptr, const_cast<float*>(stats), dloss, grad, ldg, st);
}

}  // namespace lrc
