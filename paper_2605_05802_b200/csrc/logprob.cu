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
// How a row is taken, by its length and by how many there are (held_row, ctas_of_row, ring_ctas):
//   - up to 40 KB a CTA it is held in registers: all loads on their way together, nothing rescaled, and the loss writes the gradient
//     from them (1200 rows of 4096 fp32: 11 us of a step's 18.9, 39 MB);
//   - longer, it streams through the registers, a batch ahead (4096 rows of 151936 bf16, a quarter masked: 152 to 163 us, 5.7 to 6.1 TB/s);
//   - the loss, which needs it twice, holds it in the shared memory of a cluster (the ring below: the same rows and zeros for those masked
//     409 to 416 us, 2.2 GB; from memory twice 536).
// Where rows alone do not fill the GPU (fewer than two CTAs an SM), a cluster takes one and its sums meet in shared memory: 8 rows
// of 151936 take 4.4 us.  Where they do, more CTAs a row cost more than the shorter last wave gives (4096 rows, two a row: 189 us).
#include <cooperative_groups.h>
#include <math_constants.h>

#include "policy.cuh"
#include "ring.cuh"

namespace sr {
namespace {

constexpr int kRowThreads = 256;          // sums: rows of CTAs that end at other times fill each other's gaps (512 threads, 4096 rows of 151936 bf16, a quarter masked: 188 us, 256: 173)
constexpr int kWriteThreads = 512;        // gradients alone: nobody waits for anybody (256 threads, 2048 such rows: 181 us, 512: 175)
constexpr int kUnroll = 4;
constexpr int kHeldThreads = 256, kMostVecs = 10;
constexpr int kMaxCtas = 8;              // to a row: the portable cluster size
constexpr double kLn2 = 0.693147180559945309417232;

__device__ __forceinline__ float exp2_approx(float t) {        // 2^t within 2 ulp; 2^-inf = 0
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(t));
    return r;
}
__device__ __forceinline__ float minus_inf() { return __int_as_float(0xFF800000); }

// log S of a sum that is at least 1, to 2^-24 of itself or 2^-24, whichever is more: S = 2^e m, and only log m, below 1, is
// taken in fp32.  (A logarithm in fp64 is a chain of a hundred instructions and more that the whole row waits for.)
__device__ __forceinline__ double log_sum(double S) {
    const int hi = __double2hiint(S), e = ((hi >> 20) & 0x7FF) - 1023;
    const float m = (float)__hiloint2double((hi & 0x000FFFFF) | 0x3FF00000, __double2loint(S));
    return e < 1024 ? fma((double)e, kLn2, (double)logf(m)) : S;         // NaN and inf stay what they are
}

// Largest of a warp's numbers, in every lane; NaN only where all are.
__device__ __forceinline__ float warp_max(float x) {
    float r;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
    return r;
}

// What is known of a row, or of a part of it.
struct RowSums {
    float m;
    double s, u;
};

// fp32 sums of the terms of a few elements, four of each side by side.
template <bool kEntropy>
struct TermSums {
    f32x2 s[2] = {0ull, 0ull}, u[2] = {0ull, 0ull};

    // N (an even number of) elements, none of them above m (or NaN, or +inf: these end up in s).
    template <int N>
    __device__ __forceinline__ void add(const float (&x)[N], float m, float c) {
        const f32x2 minus_m = two(-m), cc = two(c);
#pragma unroll
        for (int k = 0; k < N; k += 2) {
            const f32x2 t = mul2(add2(two(x[k], x[k + 1]), minus_m), cc);
            const float t0 = low_of(t), t1 = high_of(t);
            const f32x2 e = two(exp2_approx(t0), exp2_approx(t1));
            s[(k >> 1) & 1] = add2(s[(k >> 1) & 1], e);
            // 0 * -inf is to be 0 here; a NaN is in s already
            if (kEntropy) u[(k >> 1) & 1] = fma2(e, two(fmaxf(t0, -1000.0f), fmaxf(t1, -1000.0f)), u[(k >> 1) & 1]);
        }
    }
    static __device__ __forceinline__ double total(const f32x2 (&v)[2]) {
        const f32x2 both = add2(v[0], v[1]);
        return (double)(low_of(both) + high_of(both));
    }
    // Moves the sums into r.
    __device__ __forceinline__ void flush(RowSums& r) {
        r.s += total(s);
        s[0] = s[1] = 0ull;
        if (kEntropy) {
            r.u += total(u);
            u[0] = u[1] = 0ull;
        }
    }
};

// Makes `top` the maximum where it is larger.
template <bool kEntropy>
__device__ __forceinline__ void grow(float top, float c, RowSums& r) {
    if (!(top > r.m)) return;
    const float shift = (r.m - top) * c;                        // -inf at first: factor 0
    const double f = (double)exp2_approx(shift);
    if (kEntropy) r.u = f * (r.u + (double)fmaxf(shift, -1000.0f) * r.s);
    r.s *= f;
    r.m = top;
}
// Takes one more element.  A maximum of -inf (nothing but such logits so far) stands for 0 in the exponents, which gives terms
// of 0.
template <bool kEntropy>
__device__ __forceinline__ void take(float x, float c, RowSums& r) {
    grow<kEntropy>(x, c, r);
    const float t = (x - (r.m == minus_inf() ? 0.0f : r.m)) * c, e = exp2_approx(t);
    r.s += (double)e;
    if (kEntropy) r.u += (double)(e * fmaxf(t, -1000.0f));
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

// Sum of a warp's parts, in every lane.  kLanes: only the first so many have one that is not empty.
template <bool kEntropy, int kLanes>
__device__ __forceinline__ RowSums warp_sum(RowSums r, float c) {
    rescale<kEntropy>(r, warp_max(r.m), c);
#pragma unroll
    for (int off = kLanes / 2; off > 0; off >>= 1) {
        r.s += __shfl_xor_sync(0xFFFFFFFFu, r.s, off);
        if (kEntropy) r.u += __shfl_xor_sync(0xFFFFFFFFu, r.u, off);
    }
    if (kLanes < 32) {
        r.s = __shfl_sync(0xFFFFFFFFu, r.s, 0);
        if (kEntropy) r.u = __shfl_sync(0xFFFFFFFFu, r.u, 0);
    }
    return r;
}
// Sums of all threads' parts (up to eight warps), in every thread; over the cluster where it has several CTAs, whose threads have
// arrived at its barrier.
template <bool kEntropy>
__device__ __forceinline__ RowSums combine(RowSums r, float c, int ctas) {
    static_assert(kMaxCtas == 8 && kRowThreads <= 256 && kHeldThreads <= 256, "eight parts of the later sums");
    __shared__ RowSums s_warp[8], s_cta[kMaxCtas];
    const RowSums none = {minus_inf(), 0.0, 0.0};
    const int lane = threadIdx.x & 31;
    r = warp_sum<kEntropy, 32>(r, c);
    if (lane == 0) s_warp[threadIdx.x >> 5] = r;
    __syncthreads();
    r = warp_sum<kEntropy, 8>(lane < (int)(blockDim.x >> 5) ? s_warp[lane] : none, c);
    if (ctas > 1) {
        // every CTA writes its sums to all the others: after the barrier each reads its own memory, and may leave
        const auto cluster = cooperative_groups::this_cluster();
        cluster_wait();
        if ((int)threadIdx.x < ctas) *cluster.map_shared_rank(&s_cta[cluster.block_rank()], threadIdx.x) = r;
        cluster.sync();
        r = warp_sum<kEntropy, 8>(lane < ctas ? s_cta[lane] : none, c);
    }
    if (r.m == minus_inf()) r.s = CUDART_NAN;  // no token can occur: there is no distribution
    return r;
}

// Unpacks a vector; the compiler is kept from holding on to elements that it has unpacked before, which would take twice the
// registers.
template <int E, typename T>
__device__ __forceinline__ void unpack_again(uint4 v, float (&x)[E], T) {
    asm volatile("" : "+r"(v.x), "+r"(v.y), "+r"(v.z), "+r"(v.w));
    unpack(v, x, T());
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

// Takes the elements of N vectors.
template <typename T, bool kEntropy, int N>
__device__ __forceinline__ void take_vectors(const uint4 (&q)[N], float c, RowSums& r) {
    VecMax<T> top(minus_inf());
#pragma unroll
    for (int k = 0; k < N; ++k) top.take(q[k]);
    grow<kEntropy>(top.value(), c, r);
    const float m = r.m == minus_inf() ? 0.0f : r.m;
    TermSums<kEntropy> sums;
#pragma unroll
    for (int k = 0; k < N; ++k) {
        float x[Vec<T>::kElems];
        unpack_again(q[k], x, T());
        sums.add(x, m, c);
    }
    sums.flush(r);
}

// Sums over the part of a row that thread `at` of `threads` has.  kThreads: their number where it is known, or 0.  kAgain: the row is
// read again soon, and may stay in L2.
template <typename T, bool kEntropy, bool kAgain, int kThreads>
__device__ __forceinline__ RowSums sum_row(const T* row, int vocab, int at, int some_threads, float c) {
    const int threads = kThreads ? kThreads : some_threads;
    const RowParts<T> parts(row, vocab);
    RowSums r = {minus_inf(), 0.0, 0.0};
    if (at < parts.head + parts.tail) take<kEntropy>(to_float(row[parts.single(at)]), c, r);
    // The batch after the one at hand is on its way while that is summed up.  Batches that are whole are told apart: looking at the
    // end of the row for every vector takes a sixth of all instructions.
    const uint4* body = reinterpret_cast<const uint4*>(row + parts.head) + at;
    int left = parts.vecs - at;                // vectors from `body` on, this thread's at 0, threads, 2 threads, ...
    const int step = threads * kUnroll, whole = step - threads;
    uint4 next[kUnroll];
    const auto load = [&](const uint4* from) {
#pragma unroll
        for (int k = 0; k < kUnroll; ++k) next[k] = kAgain ? from[k * threads] : load_once(from + k * threads);
    };
    const auto load_rest = [&](const uint4* from, int have) {
#pragma unroll
        for (int k = 0; k < kUnroll; ++k) next[k] = k * threads >= have ? all_minus_inf<T>() : kAgain ? from[k * threads] : load_once(from + k * threads);
    };
    const auto take_next = [&](auto load_more) {
        uint4 q[kUnroll];
#pragma unroll
        for (int k = 0; k < kUnroll; ++k) q[k] = next[k];
        load_more();
        take_vectors<T, kEntropy>(q, c, r);
        body += step;
        left -= step;
    };
    if (left > whole) {
        load(body);
        while (left > step + whole) take_next([&] { load(body + step); });
        take_next([&] {
            if (left > step) load_rest(body + step, left - step);
        });
    } else if (left > 0) {
        load_rest(body, left);
    }
    if (left > 0) take_next([] {});
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
// Of a vector's elements, in place.
template <bool kEntropy, int E>
__device__ __forceinline__ void gradients(const RowGradient& g, float (&x)[E]) {
    const f32x2 minus_m = two(-g.M), cc = two(g.c), k0 = two(g.k0), k1 = two(g.k1);
#pragma unroll
    for (int k = 0; k < E; k += 2) {
        const f32x2 t = mul2(add2(two(x[k], x[k + 1]), minus_m), cc);
        const float t0 = low_of(t), t1 = high_of(t);
        const f32x2 e = two(exp2_approx(t0), exp2_approx(t1));
        const f32x2 d = kEntropy ? mul2(e, fma2(k1, two(fmaxf(t0, -1000.0f), fmaxf(t1, -1000.0f)), k0)) : mul2(e, k0);
        x[k] = low_of(d);
        x[k + 1] = high_of(d);
    }
}
// A row spread over the registers of a cluster: kVecs vectors a thread, and a single element where the row has some.  It is read
// once, whatever is made of it, and all of a thread's loads are on their way together.
template <typename T, int kVecs>
struct HeldRow {
    static constexpr int E = Vec<T>::kElems;
    uint4 q[kVecs];
    float x1;
    int single;                      // place of x1, or -1

    // kWhole: rows are many, and most threads have all of their vectors: those do not look at each (16384 rows of 4096 bf16 46 -> 35 us).
    template <bool kWhole>
    __device__ __forceinline__ void load(const T* row, const RowParts<T>& parts, int at, int threads) {
        const uint4* body = reinterpret_cast<const uint4*>(row + parts.head);
        if (kWhole && at + (kVecs - 1) * threads < parts.vecs) {
#pragma unroll
            for (int k = 0; k < kVecs; ++k) q[k] = load_once(body + at + k * threads);
        } else {
#pragma unroll
            for (int k = 0; k < kVecs; ++k) {
                const int i = at + k * threads;
                q[k] = i < parts.vecs ? load_once(body + i) : all_minus_inf<T>();
            }
        }
        single = at < parts.head + parts.tail ? parts.single(at) : -1;
        x1 = single >= 0 ? to_float(row[single]) : minus_inf();
    }
    // The thread's own maximum first, then the terms: nothing is rescaled.
    template <bool kEntropy>
    __device__ __forceinline__ RowSums sums(float c) const {
        VecMax<T> top(x1);                                     // x1 is an element: exact in its type
#pragma unroll
        for (int k = 0; k < kVecs; ++k) top.take(q[k]);
        RowSums r = {top.value(), 0.0, 0.0};
        if (!(r.m > minus_inf())) r.m = minus_inf();           // a NaN alone is no maximum
        take<kEntropy>(x1, c, r);
        const float m = r.m == minus_inf() ? 0.0f : r.m;
        TermSums<kEntropy> sums;
#pragma unroll
        for (int k = 0; k < kVecs; ++k) {
            float x[E];
            unpack_again(q[k], x, T());
            sums.add(x, m, c);
            if (k % 4 == 3 || k == kVecs - 1) sums.flush(r);
        }
        return r;
    }
    __device__ __forceinline__ void write_gradient(T* out, const RowParts<T>& parts, int at, int threads, const RowGradient& g) const {
        uint4* to = reinterpret_cast<uint4*>(out + parts.head);
        const int target_vec = g.target < parts.head ? -1 : (g.target - parts.head) / E;
#pragma unroll
        for (int k = 0; k < kVecs; ++k) {
            const int i = at + k * threads;
            if (i >= parts.vecs) break;
            float x[E];
            unpack_again(q[k], x, T());
            gradients<false>(g, x);
            if (i == target_vec) {
                const int at_j = (g.target - parts.head) % E;
#pragma unroll
                for (int j = 0; j < E; ++j)
                    if (j == at_j) x[j] += g.at_target;
            }
            store_once(to + i, pack(x, T()));
        }
        if (single >= 0) {
            float v = gradient<false>(g, x1);
            if (single == g.target) v += g.at_target;
            out[single] = from_float<T>(v);
        }
    }
};

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
                gradients<kEntropy>(g, x);
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

// kAlone: one CTA to a row.
template <typename T, bool kEntropy, bool kAlone>
__global__ void __launch_bounds__(kRowThreads, 4)
token_logprob_kernel(const T* logits, int vocab, long long pitch, const int32_t* targets, double inv_temperature, float c, int some_ctas,
                     float* logp, float* row_stats, float* entropy, int32_t* status) {
    grid_begin();
    const int ctas = kAlone ? 1 : some_ctas, t = blockIdx.x / ctas, part = blockIdx.x % ctas;
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
    if (!kAlone) cluster_arrive();
    const T* row = logits + (size_t)t * pitch;
    const float x_y = first ? to_float(row[y]) : 0.0f;        // on its way meanwhile
    RowSums r = sum_row<T, kEntropy, false, kAlone ? kRowThreads : 0>(row, vocab, part * kRowThreads + threadIdx.x, ctas * kRowThreads, c);
    r = combine<kEntropy>(r, c, ctas);
    if (first) {
        const double log_S = log_sum(r.s);
        logp[t] = (float)(((double)x_y - (double)r.m) * inv_temperature - log_S);
        if (row_stats) {
            row_stats[2 * (size_t)t] = r.m;
            row_stats[2 * (size_t)t + 1] = (float)r.s;
        }
        if (kEntropy) entropy[t] = (float)(log_S - kLn2 * r.u / r.s);
    }
}

template <typename T, int kVecs, bool kEntropy, bool kAlone>
__global__ void __launch_bounds__(kHeldThreads, kVecs > 7 ? 3 : 4)
held_logprob_kernel(const T* logits, int vocab, long long pitch, const int32_t* targets, double inv_temperature, float c, int some_ctas,
                    float* logp, float* row_stats, float* entropy, int32_t* status) {
    grid_begin();
    const int ctas = kAlone ? 1 : some_ctas;
    const int t = blockIdx.x / ctas, part = blockIdx.x % ctas;
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
    if (!kAlone) cluster_arrive();
    const T* row = logits + (size_t)t * pitch;
    HeldRow<T, kVecs> held;
    held.template load<kAlone>(row, RowParts<T>(row, vocab), part * kHeldThreads + threadIdx.x, ctas * kHeldThreads);
    const float x_y = first ? to_float(row[y]) : 0.0f;        // on its way meanwhile
    const RowSums r = combine<kEntropy>(held.template sums<kEntropy>(c), c, ctas);
    if (first) {
        const double log_S = log_sum(r.s);
        logp[t] = (float)(((double)x_y - (double)r.m) * inv_temperature - log_S);
        if (row_stats) {
            row_stats[2 * (size_t)t] = r.m;
            row_stats[2 * (size_t)t + 1] = (float)r.s;
        }
        if (kEntropy) entropy[t] = (float)(log_S - kLn2 * r.u / r.s);
    }
}

// Element by element: as many CTAs as there are, nobody waits (2048 rows of 151936 bf16, a quarter zeros: 176 us, 6.2 TB/s).
template <typename T, bool kEntropy>
__global__ void __launch_bounds__(kWriteThreads)
token_logprob_backward_kernel(const T* logits, int vocab, long long pitch, const int32_t* targets, const float* row_stats,
                              const float* entropy, const float* d_logp, const float* d_entropy, double temperature, float c,
                              int parts, T* d_logits, long long d_pitch) {
    grid_begin();
    const int t = blockIdx.x / parts, part = blockIdx.x % parts;
    const int32_t y = targets[t];
    T* out = d_logits + (size_t)t * d_pitch;
    RowGradient g = {};
    if (y < 0 || y >= vocab) {
        write_gradient<T, false, true>(nullptr, out, vocab, part * blockDim.x + threadIdx.x, parts * blockDim.x, g);
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
    write_gradient<T, kEntropy, false>(logits + (size_t)t * pitch, out, vocab, part * blockDim.x + threadIdx.x, parts * blockDim.x, g);
}

// The rollout of every token that counts, -1 for the others, so that the rows of the next kernel start reading at once.
__global__ void __launch_bounds__(256)
token_rows_kernel(PolicyBatch b, const int32_t* targets, int vocab, int n, int32_t* row_of, int32_t* status) {
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

// By one thread: the token's terms of the loss and the gradient of its row.  A function of its own, so that the registers of a
// held row are put aside for it in that thread alone.
__device__ __noinline__ void token_gradient(const PolicyBatch& b, const PolicyToken& k, int t, float x_y, float m, double S, double inv_temperature, float* logp,
                                            PolicyTerms* terms, RowGradient* g) {
    const double lp = ((double)x_y - (double)m) * inv_temperature - log_sum(S);
    PolicyParts parts;
    const float d = policy_gradient(b, k, lp, parts) * (float)inv_temperature;
    g->k0 = -d / (float)S;
    g->at_target = d;
    if (logp) {
        logp[t] = (float)lp;
        terms[t] = policy_terms(b, k, parts);
    }
}
__device__ __forceinline__ PolicyToken load_token(const PolicyBatch& b, int t, int rollout) {
    return PolicyToken{b.old_logp ? b.old_logp[t] : 0.0f, b.ref_logp ? b.ref_logp[t] : 0.0f, b.adv[rollout], b.weight[rollout]};
}
// The gradient of a row, in every thread of the CTA; `first` writes down the token's figures.
__device__ __forceinline__ RowGradient loss_gradient(const PolicyBatch& b, const PolicyToken& k, int t, float x_y, int y, const RowSums& r, double inv_temperature, float c, bool first,
                                                     float* logp, PolicyTerms* terms) {
    __shared__ RowGradient s_g;
    if (threadIdx.x == 0) token_gradient(b, k, t, x_y, r.m, r.s, inv_temperature, first ? logp : nullptr, terms, &s_g);
    __syncthreads();
    RowGradient g = s_g;
    g.M = r.m;
    g.c = c;
    g.k1 = 0.0f;
    g.target = y;
    return g;
}

// Rows that are read twice: those that lie differently in logits and gradient, too long or too few for the ring, and batches of
// more tokens than its list has.
template <typename T>
__global__ void __launch_bounds__(kRowThreads, 4)
policy_loss_logits_kernel(PolicyBatch b, const T* logits, int vocab, long long pitch, const int32_t* targets, const int32_t* row_of,
                          double inv_temperature, float c, int ctas, float* logp, PolicyTerms* terms, T* d_logits, long long d_pitch) {
    grid_begin();
    const int t = blockIdx.x / ctas, part = blockIdx.x % ctas;
    const int at = part * kRowThreads + threadIdx.x, threads = ctas * kRowThreads;
    const int rollout = row_of[t];
    const bool first = part == 0 && threadIdx.x == 0;
    T* out = d_logits + (size_t)t * d_pitch;
    RowGradient g = {};
    if (rollout < 0) {
        write_gradient<T, false, true>(nullptr, out, vocab, at, threads, g);
        if (first) {
            logp[t] = 0.0f;
            terms[t] = PolicyTerms{0.0, 0.0f, 0.0f, 0.0f};
        }
        return;
    }
    if (ctas > 1) cluster_arrive();
    const T* row = logits + (size_t)t * pitch;
    const int32_t y = targets[t];
    const float x_y = to_float(row[y]);                        // before anyone writes: d_logits may be the logits
    const PolicyToken token = threadIdx.x == 0 ? load_token(b, t, rollout) : PolicyToken{};      // on its way meanwhile
    RowSums r = sum_row<T, false, true, 0>(row, vocab, at, threads, c);
    r = combine<false>(r, c, ctas);
    g = loss_gradient(b, token, t, x_y, y, r, inv_temperature, c, first, logp, terms);
    write_gradient<T, false, false>(row, out, vocab, at, threads, g);
}

// Bound by how many rows are under way: one takes 4 to 5 us from its CTA's start to its end.  Seven CTAs an SM for one or two vectors a
// thread (16384 rows of 4096 bf16: 96 us, with five 114); for four vectors six gain 3 % where rows are thousands and lose as much at 1200.
template <typename T, int kVecs, bool kAlone>
__global__ void __launch_bounds__(kHeldThreads, kVecs > 7 ? 3 : kVecs > 4 ? 4 : kVecs > 2 ? 5 : 7)
held_policy_loss_kernel(PolicyBatch b, const T* logits, int vocab, long long pitch, const int32_t* targets, const int32_t* row_of,
                        double inv_temperature, float c, int some_ctas, float* logp, PolicyTerms* terms, T* d_logits, long long d_pitch) {
    grid_begin();
    const int ctas = kAlone ? 1 : some_ctas, t = blockIdx.x / ctas, part = blockIdx.x % ctas;
    const int at = part * kHeldThreads + threadIdx.x, threads = ctas * kHeldThreads;
    const int rollout = row_of[t];
    const bool first = part == 0 && threadIdx.x == 0;
    T* out = d_logits + (size_t)t * d_pitch;
    if (rollout < 0) {
        write_gradient<T, false, true>(nullptr, out, vocab, at, threads, RowGradient());
        if (first) {
            logp[t] = 0.0f;
            terms[t] = PolicyTerms{0.0, 0.0f, 0.0f, 0.0f};
        }
        return;
    }
    if (!kAlone) cluster_arrive();
    const T* row = logits + (size_t)t * pitch;
    const RowParts<T> parts(row, vocab);
    HeldRow<T, kVecs> held;
    held.template load<kAlone>(row, parts, at, threads);
    const int32_t y = targets[t];
    const float x_y = to_float(row[y]);                        // before anyone writes: d_logits may be the logits
    const PolicyToken token = threadIdx.x == 0 ? load_token(b, t, rollout) : PolicyToken{};      // on its way meanwhile
    const RowSums r = combine<false>(held.template sums<false>(c), c, ctas);
    const RowGradient g = loss_gradient(b, token, t, x_y, y, r, inv_temperature, c, first, logp, terms);
    held.write_gradient(out, parts, at, threads, g);
}

// ---- long rows, held in shared memory
//
// A row of 150000 tokens does not fit the registers or the shared memory of one SM, and read twice it comes from HBM twice (the
// second pass found 3 % of it in L2).  So a cluster holds it, a slice a CTA, in a ring of chunks: one thread has them copied in
// (bulk copies that count their bytes at a barrier); eight warps add them up as they come and send their sums to every CTA of
// the cluster; one warp turns these into the row's gradient and finds out about the row to come; and the eight write the
// gradient from the same chunks, each of which is then free for the next row.  CTAs stay and take row after row: the copies never
// wait for the sums of a row, and two CTAs an SM take turns at computing and at waiting.
// Read once, written once, but not at the rate of a copy (2048 rows of 32000 bf16 62 us, 4.2 TB/s; fp32 93, 5.6): 15 instructions an
// element (54 % of the issue slots), two of them ex2 (64 % of its rate), and two microseconds a row in which its sums meet.
constexpr int kRingThreads = 256, kRingWarps = kRingThreads / 32;
constexpr int kChunkVecs = 2 * kRingThreads;       // two vectors a thread: with one, more instructions went into finding them than into the terms
constexpr int kChunk = kChunkVecs * 16;            // bytes
constexpr int kRingSlots = 13;                     // 104 KB: two CTAs an SM
constexpr int kRingRow = 10;                       // chunks of a slice at most: three slots and more are ahead
constexpr int kZeros = 4096;                       // bytes of zeros that gradients of tokens that do not count are copied from

// A slot, and the parity of the phase that its use is.
struct RingPlace {
    uint32_t slot = 0, phase = 0;
    __device__ __forceinline__ void step() {
        if (++slot == kRingSlots) {
            slot = 0;
            phase ^= 1u;
        }
    }
};
struct RingPart {
    double s;
    float m, unused;
};
// A row to come.  Its target's logit stands here too: written, it has been read.
struct RingRow {
    int t, y;                        // t < 0: there is none
    float x_y;
};
constexpr int kRingQueue = 8;        // rows that a CTA may know of
// Counters: tokens that count; the next row of them to be taken; the next slice of the others; whether a CTA has given up a wait.
enum { kLive, kNextLive, kNextOther, kGaveUp };

// kAlone: one CTA to a row.  It is no cluster, and nothing is sent: what would be is written here, and its writers arrive.
template <typename T, bool kAlone>
__global__ void __launch_bounds__(kRingThreads + 64, 2)
ring_policy_loss_kernel(const __grid_constant__ PolicyBatch b, const T* logits, int vocab, long long pitch, const int4* list, int32_t* counters, int n_tokens, double inv_temperature,
                        float c, int ctas, float* logp, PolicyTerms* terms, T* d_logits, long long d_pitch, int32_t* status) {
    constexpr int E = Vec<T>::kElems;
    extern __shared__ __align__(128) unsigned char s_ring[];
    __shared__ uint64_t s_full[kRingSlots], s_empty[kRingSlots];                  // chunks that are there, and that are done with
    __shared__ uint64_t s_got[kRingQueue], s_known[2], s_met[2], s_ready[2];      // by row: its number, what it is, the cluster's sums, the gradient
    __shared__ __align__(16) RingPart s_part[2][kMaxCtas * kRingWarps];
    __shared__ __align__(16) int4 s_number[kRingQueue];
    __shared__ RingRow s_row[2];
    __shared__ RowGradient s_gradient[2];
    __shared__ int s_gave_up;
    __shared__ __align__(16) uint4 s_zeros[kZeros / 16];
    const int rank = kAlone ? 0 : blockIdx.x % ctas;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) {
        for (int k = 0; k < kRingSlots; ++k) {
            barrier_init(&s_full[k], 1);
            barrier_init(&s_empty[k], kRingWarps);
        }
        for (int k = 0; k < kRingQueue; ++k) barrier_init(&s_got[k], 1);
        for (int k = 0; k < 2; ++k) {
            barrier_init(&s_known[k], 1);
            barrier_init(&s_met[k], kAlone ? kRingWarps : 1);
            barrier_init(&s_ready[k], 1);
        }
        s_gave_up = 0;
        barriers_ready();
    }
    if (threadIdx.x < kZeros / 16) s_zeros[threadIdx.x] = make_uint4(0u, 0u, 0u, 0u);
    shared_written();
    // barriers of every CTA are there before anyone writes to it
    if (kAlone) __syncthreads();
    else cooperative_groups::this_cluster().sync();
    grid_begin();
    volatile int* const gave_up = &s_gave_up;
    const int live = counters[kLive];
    // this CTA's vectors of a row
    const int log_ctas = kAlone ? 0 : 31 - __clz(ctas);     // a power of two
    const auto slice = [&](const RowParts<T>& parts, int& begin, int& end) {
        begin = (int)(((long long)parts.vecs * rank) >> log_ctas);
        end = (int)(((long long)parts.vecs * (rank + 1)) >> log_ctas);
    };
    // The list's entry of the cluster's turn-th row; none: x < 0.
    const auto entry = [&](int turn) {
        const int at = turn & (kRingQueue - 1);
        barrier_wait(&s_got[at], (turn / kRingQueue) & 1, gave_up);
        const int number = *reinterpret_cast<volatile int*>(&s_number[at].x);
        return number < live && !*gave_up ? list[number] : make_int4(-1, 0, 0, 0);
    };

    // Rows are dealt out as clusters ask for them: some may have started late.  The first CTA's copying thread asks, and tells
    // the others.  It is at most five rows ahead of its own consumers (a slice has three chunks at least), and those are never two
    // ahead of anyone's: a place in the queue has been read by all long before it is used again.
    if (warp == kRingWarps) {                  // has chunks copied in, by one thread
        RingPlace place;
        uint32_t n = 0;
        const auto tell = [&](int turn, int number) {
            const int at = turn & (kRingQueue - 1);
            if (kAlone) {
                s_number[at].x = number;
                barrier_arrive(&s_got[at]);
            } else {
                for (int k = 0; k < ctas; ++k) store_at(&s_number[at], (uint32_t)number, 0ull, &s_got[at], k);
            }
        };
        // The gradients of tokens that do not count are zeros, copied from shared memory without a thread's help, a slice of a row
        // for every slice of a row that counts: they fill what the sums leave of the bandwidth.
        const int others = (n_tokens - live) << log_ctas;
        const auto clear = [&](int number) {
            const RowParts<T> parts(d_logits + (size_t)list[live + (number >> log_ctas)].x * d_pitch, vocab);
            T* const out = d_logits + (size_t)list[live + (number >> log_ctas)].x * d_pitch;
            const int part = number & (ctas - 1);
            const long long begin = ((long long)parts.vecs * part) >> log_ctas, end = ((long long)parts.vecs * (part + 1)) >> log_ctas;
            uint4* to = reinterpret_cast<uint4*>(out + parts.head);
            for (long long v = begin; v < end; v += kZeros / 16) bulk_store(to + v, s_zeros, (uint32_t)min((long long)(kZeros / 16), end - v) * 16u);
            if (part == 0)
                for (int k = 0; k < parts.head + parts.tail; ++k) out[parts.single(k)] = from_float<T>(0.0f);
        };
        if (lane == 0) {
            if (rank == 0) tell(0, atomicAdd(&counters[kNextLive], 1));
            for (int turn = 0;; ++turn) {
                if (!kAlone) barrier_expect(&s_got[turn & (kRingQueue - 1)], 16);
                const int4 row_of = entry(turn);
                if (row_of.x < 0) break;
                int number = 0;
                if (rank == 0) number = atomicAdd(&counters[kNextLive], 1);
                const int other = atomicAdd(&counters[kNextOther], 1);
                const T* row = logits + (size_t)row_of.x * pitch;
                const RowParts<T> parts(row, vocab);
                int begin, end;
                slice(parts, begin, end);
                const uint4* body = reinterpret_cast<const uint4*>(row + parts.head);
                for (int v = begin; v < end; v += kChunkVecs, ++n) {
                    if (n >= kRingSlots) barrier_wait(&s_empty[place.slot], place.phase ^ 1u, gave_up);
                    if (*gave_up) break;
                    const uint32_t bytes = (uint32_t)min(kChunkVecs, end - v) * 16u;
                    barrier_expect(&s_full[place.slot], bytes);
                    bulk_load(s_ring + place.slot * kChunk, body + v, bytes, &s_full[place.slot]);
                    place.step();
                }
                if (rank == 0) tell(turn + 1, number);
                if (other < others) clear(other);
            }
            for (;;) {
                const int other = atomicAdd(&counters[kNextOther], 1);
                if (other >= others) break;
                clear(other);
            }
            bulk_stores_done();
            // no copy is in flight when the CTA ends
            int ignored = 0;
            for (uint32_t k = n > kRingSlots ? n - kRingSlots : 0; k < n; ++k) barrier_wait(&s_full[k % kRingSlots], (k / kRingSlots) & 1, &ignored);
        }
    } else if (warp == kRingWarps + 1) {       // says which row comes next, and turns the cluster's sums into its gradient
        int4 row = make_int4(-1, 0, 0, 0), next = row;
        PolicyToken token = {}, next_token = {};
        float x_y = 0.0f;
        T next_x = from_float<T>(0.0f);
        const auto look_ahead = [&](int turn) {    // its target's logit is read before anyone can write: d_logits may be the logits
            next = entry(turn);
            if (next.x >= 0) {
                next_x = logits[(size_t)next.x * pitch + next.y];
                next_token = load_token(b, next.x, next.z);
            }
        };
        const auto announce = [&](int side) {
            row = next;
            token = next_token;
            x_y = to_float(next_x);
            if (lane == 0) {
                s_row[side] = RingRow{row.x, row.y, x_y};
                barrier_arrive(&s_known[side]);
            }
        };
        look_ahead(0);
        announce(0);
        for (int turn = 0; row.x >= 0; ++turn) {
            const int side = turn & 1;
            if (!kAlone && lane == 0) barrier_expect(&s_met[side], (uint32_t)(sizeof(RingPart) * kRingWarps) * (uint32_t)ctas);
            look_ahead(turn + 1);              // on its way while this row is summed up
            barrier_wait(&s_met[side], (turn >> 1) & 1, gave_up);
            // The cluster waits for k0 and at_target.  They come from the log p in fp64 that is written down of the token: every CTA
            // works it out alike, and gradient and figures take the same side of the clip range.
            constexpr int kParts = kAlone ? 1 : (kMaxCtas * kRingWarps + 31) / 32;
            const int parts = kRingWarps << log_ctas;          // fewer than the lanes: several have the same one, and sum them up in fewer steps
            RingPart part[kParts];
            float M = minus_inf();
            double S = 0.0;
#pragma unroll
            for (int k = 0; k < kParts; ++k) {
                part[k] = 32 * k < parts ? s_part[side][(lane & (parts - 1)) + 32 * k] : RingPart{0.0, minus_inf(), 0.0f};
                M = fmaxf(M, part[k].m);
            }
            M = warp_max(M);
#pragma unroll
            for (int k = 0; k < kParts; ++k) S += part[k].s * (double)(part[k].m == M ? 1.0f : exp2_approx((part[k].m - M) * c));
#pragma unroll
            for (int off = 16; off > 0; off >>= 1)
                if (off < parts) S += __shfl_xor_sync(0xFFFFFFFFu, S, off);
            if (M == minus_inf()) S = CUDART_NAN;      // no token can occur: there is no distribution
            const double lp = ((double)x_y - (double)M) * inv_temperature - log_sum(S);
            PolicyParts loss_parts;
            const float d = policy_gradient(b, token, lp, loss_parts) * (float)inv_temperature;
            if (lane == 0) {
                RowGradient& g = s_gradient[side];
                g.M = M;
                g.k0 = -d / (float)S;
                g.at_target = d;
                barrier_arrive(&s_ready[side]);
            }
            const int t = row.x;
            const PolicyToken token_t = token;
            __syncwarp();
            announce(side ^ 1);
            if (rank == 0 && lane == 0) {
                logp[t] = (float)lp;
                terms[t] = policy_terms(b, token_t, loss_parts);
            }
            __syncwarp();
        }
    } else {
        RingPlace place;                       // of the row's first chunk
        for (int turn = 0;; ++turn) {
            const int side = turn & 1;
            barrier_wait(&s_known[side], (turn >> 1) & 1, gave_up);
            const int t = s_row[side].t, y = s_row[side].y;
            if (t < 0 || *gave_up) break;
            const T* row = logits + (size_t)t * pitch;
            T* out = d_logits + (size_t)t * d_pitch;
            const RowParts<T> parts(row, vocab);
            int begin, end;
            slice(parts, begin, end);
            const int chunks = (end - begin + kChunkVecs - 1) / kChunkVecs, whole = (end - begin) / kChunkVecs;
            const unsigned char* const from = s_ring + threadIdx.x * 16;
            const int single = rank == 0 && (int)threadIdx.x < parts.head + parts.tail ? parts.single(threadIdx.x) : -1;
            const float x1 = single >= 0 ? to_float(row[single]) : minus_inf();

            RowSums r = {minus_inf(), 0.0, 0.0};
            RingPlace at = place;
            int k = 0;
            for (; k + 2 <= whole; k += 2) {
                uint4 v[4];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    barrier_wait(&s_full[at.slot], at.phase, gave_up);
                    v[2 * h] = *reinterpret_cast<const uint4*>(from + at.slot * kChunk);
                    v[2 * h + 1] = *reinterpret_cast<const uint4*>(from + at.slot * kChunk + kChunk / 2);
                    at.step();
                }
                take_vectors<T, false>(v, c, r);
            }
            if (k < chunks) {                              // what is left: a whole chunk, the beginning of one, or both
                uint4 v[4] = {all_minus_inf<T>(), all_minus_inf<T>(), all_minus_inf<T>(), all_minus_inf<T>()};
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if (k + h >= chunks) break;
                    barrier_wait(&s_full[at.slot], at.phase, gave_up);
                    const int have = end - begin - (k + h) * kChunkVecs;
                    if ((int)threadIdx.x < have) v[2 * h] = *reinterpret_cast<const uint4*>(from + at.slot * kChunk);
                    if ((int)threadIdx.x + kRingThreads < have) v[2 * h + 1] = *reinterpret_cast<const uint4*>(from + at.slot * kChunk + kChunk / 2);
                    at.step();
                }
                take_vectors<T, false>(v, c, r);
            }
            if (single >= 0) take<false>(x1, c, r);
            // every warp of the cluster leaves its sums with every CTA
            const float M = warp_max(r.m);
            rescale<false>(r, M, c);
#pragma unroll
            for (int off = 16; off > 0; off >>= 1) r.s += __shfl_xor_sync(0xFFFFFFFFu, r.s, off);
            if (kAlone) {
                if (lane == 0) {
                    s_part[side][warp] = RingPart{r.s, M, 0.0f};
                    barrier_arrive(&s_met[side]);
                }
            } else if (lane < ctas) {
                store_at(&s_part[side][rank * kRingWarps + warp], (unsigned long long)__double_as_longlong(r.s), (unsigned long long)__float_as_uint(M), &s_met[side], lane);
            }

            barrier_wait(&s_ready[side], (turn >> 1) & 1, gave_up);
            RowGradient g = s_gradient[side];
            g.c = c;
            g.k1 = 0.0f;
            g.target = y;
            uint4* to = reinterpret_cast<uint4*>(out + parts.head) + begin + threadIdx.x;
            const auto write = [&](uint4 v, uint4* at) {
                float x[E];
                unpack(v, x, T());
                gradients<false>(g, x);
                store_once(at, pack(x, T()));
            };
            for (k = 0; k + 2 <= whole; k += 2, to += 2 * kChunkVecs) {
                uint4 v[4];
                RingPlace second = place;
                second.step();
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    v[h] = *reinterpret_cast<const uint4*>(from + place.slot * kChunk + h * (kChunk / 2));
                    v[2 + h] = *reinterpret_cast<const uint4*>(from + second.slot * kChunk + h * (kChunk / 2));
                }
                __syncwarp();
                if (lane == 0) {
                    barrier_arrive(&s_empty[place.slot]);
                    barrier_arrive(&s_empty[second.slot]);
                }
                place = second;
                place.step();
#pragma unroll
                for (int h = 0; h < 4; ++h) write(v[h], to + h * kRingThreads);
            }
            for (; k < chunks; ++k, to += kChunkVecs) {
                const int have = end - begin - k * kChunkVecs;
                uint4 v[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) v[h] = *reinterpret_cast<const uint4*>(from + place.slot * kChunk + h * (kChunk / 2));   // behind the end: an older row's, not used
                __syncwarp();
                if (lane == 0) barrier_arrive(&s_empty[place.slot]);
                place.step();
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    if ((int)threadIdx.x + h * kRingThreads < have) write(v[h], to + h * kRingThreads);
            }
            // The target once more, by the thread that has just written it: looking for it in every vector costs more.
            const int target_vec = y < parts.head ? -1 : (y - parts.head) / E - begin;
            if (target_vec >= 0 && target_vec < end - begin && target_vec % kRingThreads == (int)threadIdx.x) out[y] = from_float<T>(gradient<false>(g, s_row[side].x_y) + g.at_target);
            if (single >= 0) {
                float v = gradient<false>(g, x1);
                if (single == y) v += g.at_target;
                out[single] = from_float<T>(v);
            }
        }
    }
    __syncwarp();
    // Nobody leaves while its memory may be written to; and whoever gave up has said so.  A row that was dropped for it, on whichever
    // CTA, is missing from the loss, which the sum over the tokens then makes NaN.
    if (kAlone) __syncthreads();
    else cooperative_groups::this_cluster().sync();
    if (threadIdx.x == 0 && *gave_up) {
        atomicExch(&counters[kGaveUp], 1);
        if (status) atomicOr(status, SR_STATUS_TIMEOUT);
    }
}

// What token_rows_kernel says of every token, as a list: token, target and rollout of those that count, in order, and then the
// others, whose figures are written here; and the ring's counters.  One cluster.
constexpr int kListThreads = 1024, kListTokens = 65536;
__global__ void __launch_bounds__(kListThreads)
token_list_kernel(const __grid_constant__ PolicyBatch b, const int32_t* targets, int vocab, int n, int4* list, int32_t* counters, float* logp, PolicyTerms* terms, int32_t* status) {
    grid_begin();
    cluster_arrive();
    __shared__ int s_warp[32], s_cta[8];
    const auto cluster = cooperative_groups::this_cluster();
    const int ctas = gridDim.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int first = (int)((long long)n * blockIdx.x / ctas), last = (int)((long long)n * (blockIdx.x + 1) / ctas);
    // rollout and target of token t, a lane, of the 32 from t0 on; -1: it does not count
    const auto look_up = [&](int t0, bool report) {
        const int t = t0 + lane;
        const int y = t < last ? targets[t] : -1;
        int r = -1;
        const bool is = counts_as_target(y, vocab, status, report);
        if (b.rows > 0) {
            const int r_first = warp_row_between(b.row_start, 0, b.rows, t0), r_last = warp_row_between(b.row_start, r_first, b.rows, min(t0 + 31, last - 1));
            if (is && !(b.mask && b.mask[t] == 0) && t >= b.row_start[0] && t < b.row_start[b.rows]) {
                r = row_between(b.row_start, r_first, r_last + 1, t);
                if (b.weight[r] == 0.0f) r = -1;
            }
        }
        return make_int2(r, y);
    };
    int2 own = make_int2(-1, -1);              // of the first sweep: mostly there is no other
    int mine = 0;
    for (int t0 = first + 32 * warp; t0 < last; t0 += kListThreads) {
        const int2 found = look_up(t0, true);
        if (t0 == first + 32 * warp) own = found;
        mine += __popc(__ballot_sync(0xFFFFFFFFu, found.x >= 0));
    }
    if (lane == 0) s_warp[warp] = mine;
    __syncthreads();
    cluster_wait();
    if (warp == 0) {
        const int total = __reduce_add_sync(0xFFFFFFFFu, s_warp[lane]);
        if (lane < ctas) *cluster.map_shared_rank(&s_cta[blockIdx.x], lane) = total;
    }
    cluster.sync();
    int before = 0, all = 0;                   // tokens that count in the CTAs before this, and in all
    for (int k = 0; k < ctas; ++k) {
        if (k < (int)blockIdx.x) before += s_cta[k];
        all += s_cta[k];
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        counters[kLive] = all;
        counters[kNextLive] = counters[kNextOther] = counters[kGaveUp] = 0;
    }
    for (int base = first; base < last; base += kListThreads) {
        const int t0 = base + 32 * warp, t = t0 + lane;
        if (base != first && t0 < last) own = look_up(t0, false);
        const bool counts = t < last && own.x >= 0;
        const unsigned bits = __ballot_sync(0xFFFFFFFFu, counts);
        __syncthreads();
        if (lane == 0) s_warp[warp] = __popc(bits);
        __syncthreads();
        const int of_warp = s_warp[lane], total = __reduce_add_sync(0xFFFFFFFFu, of_warp), in_warps = __reduce_add_sync(0xFFFFFFFFu, lane < warp ? of_warp : 0);
        const int at = before + in_warps + __popc(bits & low_mask(lane));       // tokens that count before t
        if (t < last) {
            list[counts ? at : all + (t - at)] = make_int4(t, own.y, own.x, 0);
            if (!counts) {
                logp[t] = 0.0f;
                terms[t] = PolicyTerms{0.0, 0.0f, 0.0f, 0.0f};
            }
        }
        before += total;
    }
}

// How a row is held: CTAs to a row and vectors a thread, or no way to.  One CTA, or, where the rows alone do not fill the GPU, a
// cluster as long as each thread still has a vector.  More vectors than ten a thread leave too few CTAs an SM.
struct Held {
    int ctas, vecs;
};
Held held_row(int n_tokens, int vocab, int elem) {
    const long long need = ((long long)vocab * elem + 15) / 16;
    Held h = {1, 0};
    while (h.ctas < kMaxCtas && (long long)n_tokens * h.ctas < 2 * 148 && need > (long long)h.ctas * kHeldThreads) h.ctas *= 2;
    const long long least = (need + (long long)h.ctas * kHeldThreads - 1) / ((long long)h.ctas * kHeldThreads);
    h.vecs = least > kMostVecs ? 0 : least <= 1 ? 1 : least <= 2 ? 2 : least <= 4 ? 4 : least <= 7 ? 7 : kMostVecs;
    return h;
}
template <typename F>
int with_vecs(int vecs, F f) {
    switch (vecs) {
        case 1: return f(std::integral_constant<int, 1>());
        case 2: return f(std::integral_constant<int, 2>());
        case 4: return f(std::integral_constant<int, 4>());
        case 7: return f(std::integral_constant<int, 7>());
        default: return f(std::integral_constant<int, kMostVecs>());
    }
}

// CTAs to a row: one where the rows alone fill the GPU; else a power of two up to the portable cluster size, of which each
// still has a vector or two a thread.
int ctas_of_row(int n_tokens, int vocab, int elem) {
    int ctas = 1;
    while (ctas < kMaxCtas && (long long)n_tokens * ctas < 2 * 148 && (long long)vocab * elem > 2LL * ctas * kRowThreads * 16) ctas *= 2;
    return ctas;
}

template <typename T>
int launch_forward(const LogitsArgs& a, float* logp, float* row_stats, float* entropy, int32_t* status, cudaStream_t s) {
    const float c = (float)(1.0 / (kLn2 * a.temperature));
    const Held held = held_row(a.n_tokens, a.vocab, (int)sizeof(T));
    if (held.vecs)
        return with_vecs(held.vecs, [&](auto vecs) {
            const auto kernel = held.ctas == 1 ? (entropy ? held_logprob_kernel<T, vecs(), true, true> : held_logprob_kernel<T, vecs(), false, true>)
                                               : (entropy ? held_logprob_kernel<T, vecs(), true, false> : held_logprob_kernel<T, vecs(), false, false>);
            return launch_as(true, held.ctas, "held_logprob_kernel", kernel, a.n_tokens * held.ctas, kHeldThreads, 0, s, static_cast<const T*>(a.logits), a.vocab, (long long)a.pitch, a.targets,
                             1.0 / a.temperature, c, held.ctas, logp, row_stats, entropy, status);
        });
    const int ctas = ctas_of_row(a.n_tokens, a.vocab, (int)sizeof(T));
    const auto kernel = ctas == 1 ? (entropy ? token_logprob_kernel<T, true, true> : token_logprob_kernel<T, false, true>)
                                  : (entropy ? token_logprob_kernel<T, true, false> : token_logprob_kernel<T, false, false>);
    return launch_as(true, ctas, "token_logprob_kernel", kernel, a.n_tokens * ctas, kRowThreads, 0, s, static_cast<const T*>(a.logits), a.vocab, (long long)a.pitch, a.targets,
                     1.0 / a.temperature, c, ctas, logp, row_stats, entropy, status);
}

template <typename T>
int launch_backward(const LogitsArgs& a, const float* row_stats, const float* entropy, const float* d_logp, const float* d_entropy, void* d_logits, int64_t d_pitch, cudaStream_t s) {
    const float c = (float)(1.0 / (kLn2 * a.temperature));
    const int parts = ctas_of_row(a.n_tokens, a.vocab, (int)sizeof(T));
    const int threads = (long long)a.vocab * (int)sizeof(T) > 4LL * kWriteThreads * 16 ? kWriteThreads : kWriteThreads / 2;     // four vectors a thread and more, or fewer threads
    const auto kernel = d_entropy ? token_logprob_backward_kernel<T, true> : token_logprob_backward_kernel<T, false>;
    return launch("token_logprob_backward_kernel", kernel, a.n_tokens * parts, threads, 0, s, static_cast<const T*>(a.logits), a.vocab, (long long)a.pitch, a.targets, row_stats, entropy,
                  d_logp, d_entropy, a.temperature, c, parts, static_cast<T*>(d_logits), (long long)d_pitch);
}

// Whether rows that are held can be written as they were read: logits and gradient lie alike against 16 bytes in every row.
bool alike(const LogitsArgs& a, const void* d_logits, int64_t d_pitch) {
    const uintptr_t apart = reinterpret_cast<uintptr_t>(a.logits) ^ reinterpret_cast<uintptr_t>(d_logits);
    return (apart & 15) == 0 && (a.n_tokens == 1 || ((a.pitch - d_pitch) * dtype_bytes(a.dtype)) % 16 == 0);
}

// CTAs to a row of the ring kernel, or 0: rows too long for it, short enough to be held in registers, or too few for its CTAs, which
// stay.  Held, 1200 rows of 20000 bf16 take 31 us, through the ring 36.  160 rows of 50021 in clusters of two are a row and a bit for
// each: 23 us, and 20 from memory twice; 300 of them 27, and 31.  Where rows ask for clusters of eight (above 163840 numbers of 16 bits)
// slices are short and the sums meet as often, which still pays: 1024 rows of 200000 216 us, from memory twice 233; 256000 234, and
// 285 (of 163840 in clusters of four 139, and 187).  Rows of more than eight slices have no ring: 600 of 327680 169 us, of 327696 258.
// Its list is one cluster's work, kept to 65536 tokens: so many rows of 20600 take 1141 us, from memory twice 1189; twice as many take
// 2403, and with a longer list would take 2265.
int ring_ctas(int n_tokens, int vocab, int elem) {
    const long long vecs = ((long long)vocab * elem + 15) / 16;
    if (n_tokens > kListTokens || vecs <= kHeldThreads * kMostVecs) return 0;
    int ctas = 1;
    while (ctas < kMaxCtas && vecs > (long long)ctas * kChunkVecs * kRingRow) ctas *= 2;
    return vecs > (long long)ctas * kChunkVecs * kRingRow || (long long)n_tokens * ctas < 3 * 148 ? 0 : ctas;
}
template <typename T>
int launch_ring(const LogitsArgs& a, const PolicyBatch& b, const StepScratch& ws, int ctas, float* logp, void* d_logits, int64_t d_pitch, int32_t* status, cudaStream_t s) {
    const float c = (float)(1.0 / (kLn2 * a.temperature));
    const auto kernel = ctas == 1 ? ring_policy_loss_kernel<T, true> : ring_policy_loss_kernel<T, false>;
    constexpr int kBytes = kRingSlots * kChunk;
    SR_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kBytes));
    const int list_ctas = min(8, (a.n_tokens + kListThreads - 1) / kListThreads * 2);
    int rc = launch_as(true, list_ctas, "token_list_kernel", token_list_kernel, list_ctas, kListThreads, 0, s, b, a.targets, a.vocab, a.n_tokens, ws.list, ws.counters, logp, ws.terms, status);
    if (rc != SR_OK) return rc;
    const int clusters = min(a.n_tokens, 2 * 148 / ctas);      // those that find no room at first take what rows are left
    return launch_as(true, ctas, "ring_policy_loss_kernel", kernel, clusters * ctas, kRingThreads + 64, kBytes, s, b, static_cast<const T*>(a.logits), a.vocab, (long long)a.pitch,
                     ws.list, ws.counters, a.n_tokens, 1.0 / a.temperature, c, ctas, logp, ws.terms, static_cast<T*>(d_logits), (long long)d_pitch, status);
}
template <typename T>
int launch_step(const LogitsArgs& a, const PolicyBatch& b, const int32_t* row_of, float* logp, PolicyTerms* terms, void* d_logits, int64_t d_pitch, cudaStream_t s) {
    const float c = (float)(1.0 / (kLn2 * a.temperature));
    const Held held = held_row(a.n_tokens, a.vocab, (int)sizeof(T));
    if (held.vecs && alike(a, d_logits, d_pitch))
        return with_vecs(held.vecs, [&](auto vecs) {
            const auto kernel = held.ctas == 1 ? held_policy_loss_kernel<T, vecs(), true> : held_policy_loss_kernel<T, vecs(), false>;
            return launch_as(true, held.ctas, "held_policy_loss_kernel", kernel, a.n_tokens * held.ctas, kHeldThreads, 0, s, b, static_cast<const T*>(a.logits),
                             a.vocab, (long long)a.pitch, a.targets, row_of, 1.0 / a.temperature, c, held.ctas, logp, terms, static_cast<T*>(d_logits), (long long)d_pitch);
        });
    const int ctas = ctas_of_row(a.n_tokens, a.vocab, (int)sizeof(T));
    return launch_as(true, ctas, "policy_loss_logits_kernel", policy_loss_logits_kernel<T>, a.n_tokens * ctas, kRowThreads, 0, s, b, static_cast<const T*>(a.logits), a.vocab, (long long)a.pitch, a.targets, row_of,
                     1.0 / a.temperature, c, ctas, logp, terms, static_cast<T*>(d_logits), (long long)d_pitch);
}

// gave_up: where the kernels say so if they give up, or NULL where none can.
template <typename T>
int launch_rows(const LogitsArgs& a, const PolicyBatch& b, const StepScratch& ws, float* logp, void* d_logits, int64_t d_pitch, int32_t* status, const int32_t** gave_up, cudaStream_t s) {
    const int ring = alike(a, d_logits, d_pitch) ? ring_ctas(a.n_tokens, a.vocab, (int)sizeof(T)) : 0;
    *gave_up = ring ? ws.counters + kGaveUp : nullptr;
    if (ring) return launch_ring<T>(a, b, ws, ring, logp, d_logits, d_pitch, status, s);
    SR_LAUNCH("token_rows_kernel", token_rows_kernel, (int)(((long long)a.n_tokens + 255) / 256), 256, 0, s, b, a.targets, a.vocab, a.n_tokens, ws.row_of, status);
    return launch_step<T>(a, b, ws.row_of, logp, ws.terms, d_logits, d_pitch, s);
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
    const int32_t* gave_up = nullptr;
    if (a.n_tokens > 0) {
        int rc;
        switch (a.dtype) {
            case SR_DTYPE_F32: rc = launch_rows<float>(a, b, ws, logp, d_logits, d_pitch, status, &gave_up, s); break;
            case SR_DTYPE_BF16: rc = launch_rows<__nv_bfloat16>(a, b, ws, logp, d_logits, d_pitch, status, &gave_up, s); break;
            default: rc = launch_rows<__half>(a, b, ws, logp, d_logits, d_pitch, status, &gave_up, s); break;
        }
        if (rc != SR_OK) return rc;
    }
    return launch_sum_terms(ws.terms, a.n_tokens, b.beta, gave_up, loss, stats, ws.partial, s);
}

}  // namespace sr
