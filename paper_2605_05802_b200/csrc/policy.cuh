// What a token contributes to the clipped policy loss, and which rollout it belongs to (policy.cu, logprob.cu).
#pragma once

#include "logits.cuh"

namespace sr {

// The batch that a loss is computed over, as sr_policy_loss documents it.
struct PolicyBatch {
    const float* old_logp;           // NULL: rho = 1
    const float* ref_logp;           // NULL: no KL term
    const float* adv;
    const float* weight;
    const int64_t* row_start;
    const uint8_t* mask;
    int rows;
    double clip_low, clip_high, beta;
    float low, high, beta32;         // 1 - clip_low, 1 + clip_high, beta
    float less_low, less_high;       // -clip_low, clip_high: the borders less 1
};
// What the loss reads of one token beside its log-probability.
struct PolicyToken {
    float old_logp, ref_logp, adv, weight;
};

// Weighted terms of one token.  Advantages of a group add up to 0, so that the loss is a small difference of large gains: these
// are not rounded to fp32.
struct PolicyTerms {
    double gain;
    float kl, clipped, rho;
};
// Sums of them.
template <typename F>
struct PolicySums {
    F gain, kl, clipped, rho;
};

// Largest r in [lo, hi) with start[r] <= t, by one thread; lo where there is none.  Whatever the array holds, the result lies in
// the range.
__device__ __forceinline__ int row_between(const int64_t* start, int lo, int hi, long long t) {
    while (hi - lo > 1) {
        const int mid = lo + ((hi - lo) >> 1);
        if (start[mid] <= t) lo = mid;
        else hi = mid;
    }
    return lo;
}

// The same by a whole warp, 32 places at a time: three dependent loads for 30000 rollouts.
__device__ __forceinline__ int warp_row_between(const int64_t* start, int lo, int hi, long long t) {
    const int lane = threadIdx.x & 31;
    while (hi - lo > 1) {
        const int step = (hi - lo + 31) >> 5;              // below hi - lo: the range shrinks
        const long long at = lo + (long long)lane * step;
        const bool below = lane == 0 || (at < hi && start[at] <= t);
        lo += (31 - __clz(__ballot_sync(0xFFFFFFFFu, below))) * step;
        hi = min(hi, lo + step);
    }
    return lo;
}

// The rollouts of the tokens that a warp passes through in ascending order, 128 at a time, four a lane: starts, weights and
// advantages of 32 rollouts at once, a rollout a lane, so that most lots of 128 need no loads.
struct RowWalk {
    const PolicyBatch* b;
    uint32_t begin, end;             // tokens that lie in a rollout
    int base;                        // the rollout before the lanes'
    float weight, adv;               // its
    uint32_t lane_start;             // of rollout base + 1 + lane; none: never reached
    float lane_weight, lane_adv;
    uint32_t until;                  // the rollout at hand goes on up to there: its
    float here_weight, here_adv;

    // Tokens are fewer than 2^31: where a start lies before or behind them all is enough.
    static __device__ __forceinline__ uint32_t place(long long start) { return (uint32_t)min(max(start, 0LL), 0xFFFFFFFFLL); }
    __device__ __forceinline__ void fill(int row) {
        const int at = row + 1 + (threadIdx.x & 31);
        const bool is = at < b->rows;
        base = row;
        lane_start = is ? place(b->row_start[at]) : 0xFFFFFFFFu;
        lane_weight = is ? b->weight[at] : 0.0f;
        lane_adv = lane_weight != 0.0f ? b->adv[at] : 0.0f;      // what a rollout without weight has is not used
        weight = b->weight[row];
        adv = weight != 0.0f ? b->adv[row] : 0.0f;
        until = 0;
    }
    __device__ __forceinline__ void find(const PolicyBatch& batch, uint32_t first) {
        b = &batch;
        begin = place(b->row_start[0]);
        end = place(b->row_start[b->rows]);
        fill(warp_row_between(b->row_start, 0, b->rows, first));
    }
    // Whether the 128 tokens from w0 on lie in one rollout (or before the first, or behind the last); then w and a are its weight
    // and advantage.
    __device__ __forceinline__ bool one_rollout(uint32_t w0, float& w, float& a) {
        w = here_weight;
        a = here_adv;
        if (w0 + 127 < until) return true;
        unsigned in = __ballot_sync(0xFFFFFFFFu, lane_start <= w0 + 127);
        if (in == 0xFFFFFFFFu) {                                 // more starts than the lanes hold: move on to the rollout of w0
            const int passed = __popc(__ballot_sync(0xFFFFFFFFu, lane_start <= w0));
            fill(passed < 32 ? base + passed : warp_row_between(b->row_start, base + 32, b->rows, w0));
            in = __ballot_sync(0xFFFFFFFFu, lane_start <= w0 + 127);
        }
        const unsigned passed = __ballot_sync(0xFFFFFFFFu, lane_start <= w0);
        const int last = 31 - __clz(passed);                     // starts ascend; -1: none is passed
        w = __shfl_sync(0xFFFFFFFFu, lane_weight, last & 31);
        a = __shfl_sync(0xFFFFFFFFu, lane_adv, last & 31);
        if (last < 0) {
            w = weight;
            a = adv;
        }
        here_weight = w;
        here_adv = a;
        until = last < 31 ? __shfl_sync(0xFFFFFFFFu, lane_start, last + 1) : 0;
        return passed == in;
    }
    // Weight and advantage of this lane's tokens t0 .. t0 + 3 where the 128 from w0 on lie in several.
    __device__ __forceinline__ void several_rollouts(uint32_t w0, uint32_t t0, float (&w)[4], float (&a)[4]) {
        if (__any_sync(0xFFFFFFFFu, lane_start > w0 + 127)) {
            int before = 0;                                      // starts that are not behind t0: they ascend
#pragma unroll
            for (int step = 16; step > 0; step >>= 1) {
                const uint32_t probe = __shfl_sync(0xFFFFFFFFu, lane_start, before + step - 1);
                if (probe <= t0) before += step;
            }
            uint32_t until = __shfl_sync(0xFFFFFFFFu, lane_start, before);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                while (__any_sync(0xFFFFFFFFu, until <= t0 + j)) {       // lane 31's start is behind the lot: `before` stays below 32
                    before += until <= t0 + j;
                    until = __shfl_sync(0xFFFFFFFFu, lane_start, before);
                }
                const float ws = __shfl_sync(0xFFFFFFFFu, lane_weight, (before - 1) & 31), as = __shfl_sync(0xFFFFFFFFu, lane_adv, (before - 1) & 31);
                w[j] = before ? ws : weight;
                a[j] = before ? as : adv;
            }
        } else {                                                 // 33 rollouts and more in 128 tokens
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int row = row_between(b->row_start, base, b->rows, t0 + j);
                w[j] = b->weight[row];
                a[j] = w[j] != 0.0f ? b->adv[row] : 0.0f;
            }
        }
    }
};

static __device__ __noinline__ float far_expm1(float d) { return expm1f(d); }       // rare: kept out of the loops

// e^d - 1 and e^d - 1 - d.  With d = n ln 2 + r and |r| <= ln(2) / 2, e^r - 1 = r + q with q = r^2 times the Taylor series of
// (e^r - 1 - r) / r^2, cut where the next term is below 2^-27 of the sum (ln 2 in two parts is Cody and Waite's); then
//     e^d - 1 - d = 2^n q + (2^n r + (2^n - 1) - d),
// whose second part is exactly 0 for n = 0: policies that nearly agree lose nothing.
// For |d| <= 80, two numbers at a time: 2^n, r and q.
// kLast: with the last term, which e^d - 1 by itself does not need (2^-26 of r).
template <bool kLast>
__device__ __forceinline__ void exp_parts(f32x2 d, f32x2& s, f32x2& r, f32x2& q) {
    const f32x2 z = fma2(d, two(1.44269504f), two(12582912.0f));           // 1.5 * 2^23: n stands in the lowest bits
    const f32x2 n = add2(z, two(-12582912.0f));
    r = fma2(n, two(-0.693359375f), d);            // ln 2 in two parts, the first with few bits: this product is exact
    r = fma2(n, two(2.12194440054690583e-4f), r);
    f32x2 g = two(1.0f / 5040.0f);
    if (kLast) g = fma2(two(1.0f / 40320.0f), r, g);
    g = fma2(g, r, two(1.0f / 720.0f));
    g = fma2(g, r, two(1.0f / 120.0f));
    g = fma2(g, r, two(1.0f / 24.0f));
    g = fma2(g, r, two(1.0f / 6.0f));
    g = fma2(g, r, two(0.5f));
    q = mul2(mul2(g, r), r);
    const auto power = [](float z) { return __uint_as_float((__float_as_uint(z) << 23) + 0x3F800000u); };
    s = two(power(low_of(z)), power(high_of(z)));
}
// e^d and e^d - 1, each to its own size.
__device__ __forceinline__ void exp_near(f32x2 d, f32x2& e, f32x2& em1) {
    f32x2 s, r, q;
    exp_parts<false>(d, s, r, q);
    const f32x2 rest = add2(r, q);
    e = fma2(s, rest, s);
    em1 = fma2(s, rest, add2(s, two(-1.0f)));
}
__device__ __forceinline__ void exp_less_line_near(f32x2 d, f32x2& em1, f32x2& kl) {
    f32x2 s, r, q;
    exp_parts<true>(d, s, r, q);
    const f32x2 less = add2(s, two(-1.0f));
    kl = fma2(s, q, fma2(d, two(-1.0f), fma2(s, r, less)));
    em1 = fma2(s, add2(r, q), less);
}
__device__ __forceinline__ float exp_less_one(float d) {
    if (fabsf(d) > 80.0f) return far_expm1(d);
    f32x2 e, em1;
    exp_near(two(d, 0.0f), e, em1);
    return low_of(em1);
}
__device__ __forceinline__ void exp_less_line(float d, float& em1, float& kl) {
    if (fabsf(d) > 80.0f) {                        // 2^n r may overflow before the sum does
        em1 = far_expm1(d);
        kl = em1 - d;
    } else {
        f32x2 em1_2, kl_2;
        exp_less_line_near(two(d, 0.0f), em1_2, kl_2);
        em1 = low_of(em1_2);
        kl = low_of(kl_2);
    }
}

// The gradient of the log-probability of a token that counts, and what its terms are made of.  `lp` is fp32 where it came from memory,
// fp64 where it has just been computed.
//
// Whether rho is past a border of the clip range would be lost in 32 bits (and a token on the wrong side has a wholly wrong
// gradient): rho in fp32 is off by up to 2^-22 and |log rho| 2^-23 of itself, so within four and two times that of a border the
// comparison is made again in fp64.
constexpr float kMargin = 9.5367431640625e-7f, kMarginSlope = 2.384185791015625e-7f;
__device__ __forceinline__ float ratio_margin(float delta) { return fmaf(fabsf(delta), kMarginSlope, kMargin); }
static __device__ __noinline__ double exact_ratio(double lp, double old_logp) { return exp(lp - old_logp); }      // rare as well
struct PolicyParts {
    float rho, delta, kl;            // delta = log rho
    bool clipped;
};
template <typename F>
__device__ __forceinline__ float policy_gradient(const PolicyBatch& b, const PolicyToken& k, F lp, PolicyParts& out) {
    const float A = k.adv;
    float rho = lp == lp ? 1.0f : (float)lp, delta = rho - 1.0f;         // a NaN stays one
    bool clipped = false;
    if (b.old_logp) {
        const float border = A > 0.0f ? b.high : b.low;
        delta = (float)(lp - (F)k.old_logp);
        rho = expf(delta);
        clipped = A > 0.0f ? rho > border : A < 0.0f && rho < border;
        if (fabsf(rho - border) <= ratio_margin(delta) * border) {
            const double exact = exact_ratio((double)lp, (double)k.old_logp);
            clipped = A > 0.0f ? exact > 1.0 + b.clip_high : A < 0.0f && exact < 1.0 - b.clip_low;
        }
    }
    float d_lp = clipped || A == 0.0f ? 0.0f : -A * rho;
    float kl = 0.0f;
    if (b.ref_logp) {
        float em1;
        exp_less_line((float)((F)k.ref_logp - lp), em1, kl);
        if (b.beta != 0.0) d_lp = fmaf(-b.beta32, em1, d_lp);
    }
    out = PolicyParts{rho, delta, kl, clipped};
    return k.weight * d_lp;
}
// Its terms.  rho - 1 is taken to its own size: see PolicyTerms.
__device__ __forceinline__ PolicyTerms policy_terms(const PolicyBatch& b, const PolicyToken& k, const PolicyParts& p) {
    const float A = k.adv, w = k.weight;
    const double used = !p.clipped ? 1.0 + (double)exp_less_one(p.delta) : A > 0.0f ? 1.0 + b.clip_high : 1.0 - b.clip_low;
    return PolicyTerms{A == 0.0f ? 0.0 : (double)w * (double)A * used, w * p.kl, p.clipped ? w : 0.0f, w * p.rho};
}

// The loss from the sums over all tokens.
__device__ __forceinline__ void write_policy_loss(const PolicySums<double>& sum, double beta, float* loss, float* stats) {
    *loss = (float)(beta != 0.0 ? beta * sum.kl - sum.gain : -sum.gain);
    if (stats) {
        stats[0] = (float)sum.gain;
        stats[1] = (float)sum.kl;
        stats[2] = (float)sum.clipped;
        stats[3] = (float)sum.rho;
    }
}

__device__ __forceinline__ void add_terms(PolicySums<double>& a, const PolicySums<double>& b) {
    a.gain += b.gain;
    a.kl += b.kl;
    a.clipped += b.clipped;
    a.rho += b.rho;
}

// Sum over the threads of a CTA, in thread 0; every thread takes part.  The order depends on the thread count alone.
__device__ __forceinline__ PolicySums<double> block_sum(PolicySums<double> v) {
    __shared__ PolicySums<double> s_warp[32];
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
        PolicySums<double> o;
        o.gain = __shfl_xor_sync(0xFFFFFFFFu, v.gain, off);
        o.kl = __shfl_xor_sync(0xFFFFFFFFu, v.kl, off);
        o.clipped = __shfl_xor_sync(0xFFFFFFFFu, v.clipped, off);
        o.rho = __shfl_xor_sync(0xFFFFFFFFu, v.rho, off);
        add_terms(v, o);
    }
    if ((threadIdx.x & 31) == 0) s_warp[threadIdx.x >> 5] = v;
    __syncthreads();
    if (threadIdx.x == 0)
        for (unsigned w = 1; w < blockDim.x >> 5; ++w) add_terms(v, s_warp[w]);
    return v;
}

constexpr int kMaxPartials = 1184;   // CTAs that leave a sum each: eight on each of 148 SMs

// policy.cu
int launch_loss_weights(const int64_t* row_start, const uint8_t* mask, int32_t n_tokens, const uint8_t* drop_mask, int32_t n_groups, int32_t N, int32_t mode,
                        double scale, float* weight, int64_t* counts, void* ws, cudaStream_t s);
int launch_policy_loss(const PolicyBatch& b, const float* logp, int32_t n, float* loss, float* d_logp, float* stats, double* partial, cudaStream_t s);
// Sums the terms of n tokens into loss and stats; NaN where *gave_up is set (NULL: it cannot be).
int launch_sum_terms(const PolicyTerms* terms, int n, double beta, const int32_t* gave_up, float* loss, float* stats, double* partial, cudaStream_t s);

// logprob.cu
struct StepScratch {
    double* partial;                 // [kMaxPartials][4]
    PolicyTerms* terms;              // [n_tokens]
    int32_t* row_of;                 // [n_tokens], or the same memory as
    int4* list;                      // [n_tokens]
    int32_t* counters;               // [4]
};
int launch_policy_loss_logits(const LogitsArgs& a, const PolicyBatch& b, float* loss, float* logp, void* d_logits, int64_t d_pitch, float* stats, int32_t* status,
                              const StepScratch& ws, cudaStream_t s);

}  // namespace sr
