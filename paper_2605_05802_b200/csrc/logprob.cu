// Log-probabilities of taken tokens, their gradient, and the policy loss from logits with the gradient of the logits.
//
// A row of logits is one distribution over up to a few hundred thousand tokens; everything here is a pass over rows with a
// handful of operations an element, bound by HBM.  With M the largest logit of what a thread has seen so far and
// c = log2(e) / temperature it keeps
//     S = sum 2^((x - M) c),   U = sum 2^((x - M) c) (x - M) c
// (U for the entropy only), rescaled when M grows: one pass gives log p and H.  Exponentials and the sums of the 16 or 32
// elements that a thread takes at a time are fp32; what is carried from one such batch to the next, and between threads, is
// fp64, so that the many small terms beside a large one are not rounded off against it.  (x - M) is taken before the product
// with c: rows masked with the type's lowest value would overflow the other way round.
//
// A CTA takes a row, or, where there are too few rows for the GPU, a cluster of CTAs does and their sums meet in shared
// memory.  Loads are 16-byte vectors, four in flight a thread; elements before the first boundary of 16 bytes and behind the
// last are taken one by one.
#include <cooperative_groups.h>
#include <math_constants.h>

#include "policy.cuh"

namespace sr {
namespace {

constexpr int kRowThreads = 512;
constexpr int kUnroll = 4;
constexpr double kLn2 = 0.693147180559945309417232;

__device__ __forceinline__ float exp2_approx(float t) {        // 2^t within 2 ulp; 2^-inf = 0
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(t));
    return r;
}
__device__ __forceinline__ float minus_inf() { return __int_as_float(0xFF800000); }

// What is known of a row, or of a part of it.
struct RowSums {
    float m;
    double s, u;
};

// Takes N more elements.  A maximum of -inf (nothing but such logits so far) stands for 0 in the exponents, which gives
// terms of 0; NaN and +inf end up in s.
template <int N, bool kEntropy>
__device__ __forceinline__ void take(const float (&x)[N], float c, RowSums& r) {
    float top = x[0];
#pragma unroll
    for (int k = 1; k < N; ++k) top = fmaxf(top, x[k]);
    if (top > r.m) {
        const float shift = (r.m - top) * c;                    // -inf at first: factor 0
        const double f = (double)exp2_approx(shift);
        if (kEntropy) r.u = f * (r.u + (double)fmaxf(shift, -1000.0f) * r.s);
        r.s *= f;
        r.m = top;
    }
    const float m = r.m == minus_inf() ? 0.0f : r.m;
    float s[4] = {0.0f, 0.0f, 0.0f, 0.0f}, u[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const float t = (x[k] - m) * c;
        const float e = exp2_approx(t);
        s[k & 3] += e;
        if (kEntropy) u[k & 3] = fmaf(e, fmaxf(t, -1000.0f), u[k & 3]);      // 0 * -inf is 0 here; a NaN is in s already
    }
    r.s += (double)((s[0] + s[1]) + (s[2] + s[3]));
    if (kEntropy) r.u += (double)((u[0] + u[1]) + (u[2] + u[3]));
}

// r, seen from the maximum M of several parts.
template <bool kEntropy>
__device__ __forceinline__ void rescale(RowSums& r, float M, float c) {
    if (r.m == M) return;                                       // -inf among them: a part with nothing but such logits
    const float shift = (r.m - M) * c;
    const double f = (double)exp2_approx(shift);
    if (kEntropy) r.u = f * (r.u + (double)fmaxf(shift, -1000.0f) * r.s);
    r.s *= f;
    r.m = M;
}

// Sums of all threads' parts, in every thread.  kCluster: over the cluster.
template <bool kEntropy, bool kCluster>
__device__ __forceinline__ RowSums combine(RowSums r, float c) {
    __shared__ float s_m[32];
    __shared__ double s_s[32], s_u[32];
    __shared__ RowSums s_cta;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    float M = r.m;
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) M = fmaxf(M, __shfl_xor_sync(0xFFFFFFFFu, M, off));
    if (lane == 0) s_m[warp] = M;
    __syncthreads();
    M = s_m[0];
    for (int w = 1; w < warps; ++w) M = fmaxf(M, s_m[w]);
    rescale<kEntropy>(r, M, c);
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
        r.s += __shfl_xor_sync(0xFFFFFFFFu, r.s, off);
        if (kEntropy) r.u += __shfl_xor_sync(0xFFFFFFFFu, r.u, off);
    }
    if (lane == 0) {
        s_s[warp] = r.s;
        if (kEntropy) s_u[warp] = r.u;
    }
    __syncthreads();
    r.s = s_s[0];
    r.u = kEntropy ? s_u[0] : 0.0;
    for (int w = 1; w < warps; ++w) {
        r.s += s_s[w];
        if (kEntropy) r.u += s_u[w];
    }
    if (kCluster) {
        const auto cluster = cooperative_groups::this_cluster();
        if (threadIdx.x == 0) s_cta = r;
        cluster.sync();
        const unsigned n = cluster.num_blocks();
        float top = minus_inf();
        for (unsigned b = 0; b < n; ++b) top = fmaxf(top, cluster.map_shared_rank(&s_cta, b)->m);
        RowSums sum = {top, 0.0, 0.0};
        for (unsigned b = 0; b < n; ++b) {
            RowSums part = *cluster.map_shared_rank(&s_cta, b);
            rescale<kEntropy>(part, top, c);
            sum.s += part.s;
            if (kEntropy) sum.u += part.u;
        }
        cluster.sync();                        // nobody leaves while its sums are read
        r = sum;
    }
    if (r.m == minus_inf()) r.s = CUDART_NAN;  // no token can occur: there is no distribution
    return r;
}

// How a row falls into single elements before the first 16-byte boundary, vectors, and single elements behind them.
template <typename T>
struct RowParts {
    int head, vecs, tail;
    __device__ __forceinline__ RowParts(const T* row, int vocab) {
        const int off = (int)(reinterpret_cast<uintptr_t>(row) & 15) / (int)sizeof(T);
        head = min(vocab, off ? Vec<T>::kElems - off : 0);
        vecs = (vocab - head) / Vec<T>::kElems;
        tail = vocab - head - vecs * Vec<T>::kElems;
    }
    // place of the k-th single element
    __device__ __forceinline__ int single(int k) const { return k < head ? k : head + vecs * Vec<T>::kElems + (k - head); }
};

template <typename T>
__device__ __forceinline__ uint4 all_minus_inf() {
    const uint32_t w = sizeof(T) == 4 ? 0xFF800000u : std::is_same<T, __half>::value ? 0xFC00FC00u : 0xFF80FF80u;
    return make_uint4(w, w, w, w);
}

// Sums over the part of a row that thread `at` of `threads` has.
template <typename T, bool kEntropy>
__device__ __forceinline__ RowSums sum_row(const T* row, int vocab, int at, int threads, float c) {
    constexpr int E = Vec<T>::kElems;
    const RowParts<T> parts(row, vocab);
    RowSums r = {minus_inf(), 0.0, 0.0};
    if (at < parts.head + parts.tail) {
        const float x[1] = {to_float(row[parts.single(at)])};
        take<1, kEntropy>(x, c, r);
    }
    const uint4* body = reinterpret_cast<const uint4*>(row + parts.head);
    for (long long v = at; v < parts.vecs; v += (long long)threads * kUnroll) {
        uint4 q[kUnroll];
#pragma unroll
        for (int k = 0; k < kUnroll; ++k) {
            const long long i = v + (long long)k * threads;
            q[k] = i < parts.vecs ? body[i] : all_minus_inf<T>();
        }
        float x[kUnroll * E];
#pragma unroll
        for (int k = 0; k < kUnroll; ++k) {
            float y[E];
            unpack(q[k], y, T());
#pragma unroll
            for (int j = 0; j < E; ++j) x[k * E + j] = y[j];
        }
        take<kUnroll * E, kEntropy>(x, c, r);
    }
    return r;
}

// The gradient of a row: e (k0 + k1 t) with t = (x - M) c and e = 2^t, and `at_target` more at the target.
struct RowGradient {
    float M, c, k0, k1, at_target;
    int target;
};
template <bool kEntropy>
__device__ __forceinline__ float gradient(const RowGradient& g, float x) {
    const float t = (x - g.M) * g.c;
    const float e = exp2_approx(t);
    return kEntropy ? e * fmaf(g.k1, fmaxf(t, -1000.0f), g.k0) : e * g.k0;
}
// kZero: the row's gradient is 0 and its logits are not read.
template <typename T, bool kEntropy, bool kZero>
__device__ __forceinline__ void write_gradient(const T* row, T* out, int vocab, int at, int threads, const RowGradient& g) {
    constexpr int E = Vec<T>::kElems;
    const RowParts<T> parts(out, vocab);
    const bool vec = kZero || ((reinterpret_cast<uintptr_t>(row) ^ reinterpret_cast<uintptr_t>(out)) & 15) == 0;
    auto one = [&](int j) {
        float v = kZero ? 0.0f : gradient<kEntropy>(g, to_float(row[j]));
        if (!kZero && j == g.target) v += g.at_target;
        out[j] = from_float<T>(v);
    };
    if (!vec) {                                // the two rows lie differently against 16 bytes
        for (long long j = at; j < vocab; j += threads) one((int)j);
        return;
    }
    if (at < parts.head + parts.tail) one(parts.single(at));
    const uint4* body = reinterpret_cast<const uint4*>(row + parts.head);
    uint4* to = reinterpret_cast<uint4*>(out + parts.head);
    const int target_vec = kZero || g.target < parts.head ? -1 : (g.target - parts.head) / E;
    for (long long v = at; v < parts.vecs; v += (long long)threads * kUnroll) {
        uint4 q[kUnroll];
#pragma unroll
        for (int k = 0; k < kUnroll; ++k) {
            const long long i = v + (long long)k * threads;
            q[k] = kZero || i >= parts.vecs ? make_uint4(0u, 0u, 0u, 0u) : body[i];
        }
#pragma unroll
        for (int k = 0; k < kUnroll; ++k) {
            const long long i = v + (long long)k * threads;
            if (i >= parts.vecs) break;
            if (!kZero) {
                float x[E];
                unpack(q[k], x, T());
#pragma unroll
                for (int j = 0; j < E; ++j) x[j] = gradient<kEntropy>(g, x[j]);
                if (i == target_vec) {
                    const int at_j = (g.target - parts.head) % E;
#pragma unroll
                    for (int j = 0; j < E; ++j)
                        if (j == at_j) x[j] += g.at_target;
                }
                q[k] = pack(x, T());
            }
            to[i] = q[k];
        }
    }
}

__device__ __forceinline__ bool counts_as_target(int32_t y, int vocab, int32_t* status, bool report) {
    if (y >= vocab && report && status) atomicOr(status, SR_STATUS_BAD_TARGET);
    return y >= 0 && y < vocab;
}

template <typename T, bool kEntropy, bool kCluster>
__global__ void __launch_bounds__(kRowThreads)
token_logprob_kernel(const T* __restrict__ logits, int vocab, long long pitch, const int32_t* __restrict__ targets, double temperature, float c, int ctas,
                     float* __restrict__ logp, float* __restrict__ row_stats, float* __restrict__ entropy, int32_t* __restrict__ status) {
    grid_begin();
    const int t = kCluster ? blockIdx.x / ctas : blockIdx.x, part = kCluster ? blockIdx.x % ctas : 0;
    const int32_t y = targets[t];
    const bool first = part == 0 && threadIdx.x == 0;
    if (!counts_as_target(y, vocab, status, first)) {
        if (first) {
            logp[t] = 0.0f;
            if (row_stats) row_stats[2 * (size_t)t] = row_stats[2 * (size_t)t + 1] = 0.0f;
            if (kEntropy) entropy[t] = 0.0f;
        }
        return;
    }
    const T* row = logits + (size_t)t * pitch;
    RowSums r = sum_row<T, kEntropy>(row, vocab, part * kRowThreads + threadIdx.x, ctas * kRowThreads, c);
    r = combine<kEntropy, kCluster>(r, c);
    if (first) {
        const double log_S = log(r.s);
        logp[t] = (float)(((double)to_float(row[y]) - (double)r.m) / temperature - log_S);
        if (row_stats) {
            row_stats[2 * (size_t)t] = r.m;
            row_stats[2 * (size_t)t + 1] = (float)r.s;
        }
        if (kEntropy) entropy[t] = (float)(log_S - kLn2 * r.u / r.s);
    }
}

template <typename T, bool kEntropy>
__global__ void __launch_bounds__(kRowThreads)
token_logprob_backward_kernel(const T* logits, int vocab, long long pitch, const int32_t* __restrict__ targets, const float* __restrict__ row_stats,
                              const float* __restrict__ entropy, const float* __restrict__ d_logp, const float* __restrict__ d_entropy, double temperature, float c,
                              int parts, T* d_logits, long long d_pitch) {
    grid_begin();
    const int t = blockIdx.x / parts, part = blockIdx.x % parts;
    const int32_t y = targets[t];
    T* out = d_logits + (size_t)t * d_pitch;
    RowGradient g = {};
    if (y < 0 || y >= vocab) {
        write_gradient<T, false, true>(nullptr, out, vocab, part * kRowThreads + threadIdx.x, parts * kRowThreads, g);
        return;
    }
    const double S = (double)row_stats[2 * (size_t)t + 1], d = (double)d_logp[t];
    double k0 = -d;
    if (kEntropy) {
        const double dh = (double)d_entropy[t];
        k0 -= dh * ((double)entropy[t] - log(S));
        g.k1 = (float)(-dh * kLn2 / (S * temperature));
    }
    g.M = row_stats[2 * (size_t)t];
    g.c = c;
    g.k0 = (float)(k0 / (S * temperature));
    g.at_target = (float)(d / temperature);
    g.target = y;
    write_gradient<T, kEntropy, false>(logits + (size_t)t * pitch, out, vocab, part * kRowThreads + threadIdx.x, parts * kRowThreads, g);
}

// The rollout of every token that counts, -1 for the others, so that the rows of the next kernel start reading at once.
__global__ void __launch_bounds__(256)
token_rows_kernel(PolicyBatch b, const int32_t* __restrict__ targets, int vocab, int n, int32_t* __restrict__ row_of, int32_t* __restrict__ status) {
    grid_begin();
    const int t = blockIdx.x * 256 + threadIdx.x;
    if (t >= n) return;
    int r = -1;
    if (counts_as_target(targets[t], vocab, status, true) && !(b.mask && b.mask[t] == 0) && b.rows > 0 && t >= b.row_start[0] && t < b.row_start[b.rows]) {
        r = row_between(b.row_start, 0, b.rows, t);
        if (b.weight[r] == 0.0f) r = -1;
    }
    row_of[t] = r;
}

template <typename T, bool kCluster>
__global__ void __launch_bounds__(kRowThreads)
policy_loss_logits_kernel(PolicyBatch b, const T* logits, int vocab, long long pitch, const int32_t* __restrict__ targets, const int32_t* __restrict__ row_of,
                          double temperature, float c, int ctas, float* __restrict__ logp, PolicyTerms<float>* __restrict__ terms, T* d_logits, long long d_pitch) {
    grid_begin();
    const int t = kCluster ? blockIdx.x / ctas : blockIdx.x, part = kCluster ? blockIdx.x % ctas : 0;
    const int at = part * kRowThreads + threadIdx.x, threads = ctas * kRowThreads;
    const int rollout = row_of[t];
    const bool first = part == 0 && threadIdx.x == 0;
    T* out = d_logits + (size_t)t * d_pitch;
    RowGradient g = {};
    if (rollout < 0) {
        write_gradient<T, false, true>(nullptr, out, vocab, at, threads, g);
        if (first) {
            logp[t] = 0.0f;
            terms[t] = PolicyTerms<float>{0.0f, 0.0f, 0.0f, 0.0f};
        }
        return;
    }
    const T* row = logits + (size_t)t * pitch;
    const int32_t y = targets[t];
    const float A = b.adv[rollout], w = b.weight[rollout];
    const double x_y = (double)to_float(row[y]);               // before anyone writes: d_logits may be the logits
    RowSums r = sum_row<T, false>(row, vocab, at, threads, c);
    r = combine<false, kCluster>(r, c);
    __shared__ RowGradient s_g;
    if (threadIdx.x == 0) {
        const double lp = (x_y - (double)r.m) / temperature - log(r.s);
        PolicyTerms<float> term;
        const float d = policy_token(b, (size_t)t, lp, A, w, term);
        if (first) {
            logp[t] = (float)lp;
            terms[t] = term;
        }
        g.M = r.m;
        g.c = c;
        g.k0 = (float)(-(double)d / (r.s * temperature));
        g.at_target = (float)((double)d / temperature);
        g.target = y;
        s_g = g;
    }
    __syncthreads();
    g = s_g;
    write_gradient<T, false, false>(row, out, vocab, at, threads, g);
}

// CTAs to a row: one where the rows alone fill the GPU; else a power of two up to the portable cluster size, of which each
// still has a vector or two a thread.
int ctas_of_row(int n_tokens, int vocab, int elem) {
    int ctas = 1;
    while (ctas < 8 && (long long)n_tokens * ctas < 2 * 148 && (long long)vocab * elem > 2LL * ctas * kRowThreads * 16) ctas *= 2;
    return ctas;
}

template <typename T>
int launch_forward(const LogitsArgs& a, float* logp, float* row_stats, float* entropy, int32_t* status, cudaStream_t s) {
    const float c = (float)(1.0 / (kLn2 * a.temperature));
    const int ctas = ctas_of_row(a.n_tokens, a.vocab, (int)sizeof(T));
    const auto kernel = ctas > 1 ? (entropy ? token_logprob_kernel<T, true, true> : token_logprob_kernel<T, false, true>)
                                 : (entropy ? token_logprob_kernel<T, true, false> : token_logprob_kernel<T, false, false>);
    return launch_as(true, ctas, "token_logprob_kernel", kernel, a.n_tokens * ctas, kRowThreads, 0, s, static_cast<const T*>(a.logits), a.vocab, (long long)a.pitch, a.targets,
                     a.temperature, c, ctas, logp, row_stats, entropy, status);
}

template <typename T>
int launch_backward(const LogitsArgs& a, const float* row_stats, const float* entropy, const float* d_logp, const float* d_entropy, void* d_logits, int64_t d_pitch, cudaStream_t s) {
    const float c = (float)(1.0 / (kLn2 * a.temperature));
    const int parts = ctas_of_row(a.n_tokens, a.vocab, (int)sizeof(T));
    const auto kernel = d_entropy ? token_logprob_backward_kernel<T, true> : token_logprob_backward_kernel<T, false>;
    return launch("token_logprob_backward_kernel", kernel, a.n_tokens * parts, kRowThreads, 0, s, static_cast<const T*>(a.logits), a.vocab, (long long)a.pitch, a.targets, row_stats, entropy,
                  d_logp, d_entropy, a.temperature, c, parts, static_cast<T*>(d_logits), (long long)d_pitch);
}

template <typename T>
int launch_step(const LogitsArgs& a, const PolicyBatch& b, const int32_t* row_of, float* logp, PolicyTerms<float>* terms, void* d_logits, int64_t d_pitch, cudaStream_t s) {
    const float c = (float)(1.0 / (kLn2 * a.temperature));
    const int ctas = ctas_of_row(a.n_tokens, a.vocab, (int)sizeof(T));
    const auto kernel = ctas > 1 ? policy_loss_logits_kernel<T, true> : policy_loss_logits_kernel<T, false>;
    return launch_as(true, ctas, "policy_loss_logits_kernel", kernel, a.n_tokens * ctas, kRowThreads, 0, s, b, static_cast<const T*>(a.logits), a.vocab, (long long)a.pitch, a.targets, row_of,
                     a.temperature, c, ctas, logp, terms, static_cast<T*>(d_logits), (long long)d_pitch);
}

}  // namespace

int launch_token_logprob(const LogitsArgs& a, float* logp, float* row_stats, float* entropy, int32_t* status, cudaStream_t s) {
    if (a.n_tokens == 0) return SR_OK;
    switch (a.dtype) {
        case SR_DTYPE_F32: return launch_forward<float>(a, logp, row_stats, entropy, status, s);
        case SR_DTYPE_BF16: return launch_forward<__nv_bfloat16>(a, logp, row_stats, entropy, status, s);
        default: return launch_forward<__half>(a, logp, row_stats, entropy, status, s);
    }
}

int launch_token_logprob_backward(const LogitsArgs& a, const float* row_stats, const float* entropy, const float* d_logp, const float* d_entropy, void* d_logits,
                                  int64_t d_pitch, cudaStream_t s) {
    if (a.n_tokens == 0) return SR_OK;
    switch (a.dtype) {
        case SR_DTYPE_F32: return launch_backward<float>(a, row_stats, entropy, d_logp, d_entropy, d_logits, d_pitch, s);
        case SR_DTYPE_BF16: return launch_backward<__nv_bfloat16>(a, row_stats, entropy, d_logp, d_entropy, d_logits, d_pitch, s);
        default: return launch_backward<__half>(a, row_stats, entropy, d_logp, d_entropy, d_logits, d_pitch, s);
    }
}

int launch_policy_loss_logits(const LogitsArgs& a, const PolicyBatch& b, float* loss, float* logp, void* d_logits, int64_t d_pitch, float* stats, int32_t* status,
                              const StepScratch& ws, cudaStream_t s) {
    if (a.n_tokens > 0) {
        SR_LAUNCH("token_rows_kernel", token_rows_kernel, (int)(((long long)a.n_tokens + 255) / 256), 256, 0, s, b, a.targets, a.vocab, a.n_tokens, ws.row_of, status);
        int rc;
        switch (a.dtype) {
            case SR_DTYPE_F32: rc = launch_step<float>(a, b, ws.row_of, logp, ws.terms, d_logits, d_pitch, s); break;
            case SR_DTYPE_BF16: rc = launch_step<__nv_bfloat16>(a, b, ws.row_of, logp, ws.terms, d_logits, d_pitch, s); break;
            default: rc = launch_step<__half>(a, b, ws.row_of, logp, ws.terms, d_logits, d_pitch, s); break;
        }
        if (rc != SR_OK) return rc;
    }
    return launch_sum_terms(ws.terms, a.n_tokens, b.beta, loss, stats, ws.partial, s);
}

}  // namespace sr
