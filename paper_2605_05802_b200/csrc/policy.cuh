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
    float low, high;                 // 1 - clip_low, 1 + clip_high
};
// What the loss reads of one token beside its log-probability.
struct PolicyToken {
    float old_logp, ref_logp, adv, weight;
};

// Weighted terms of one token, or their sums.
template <typename F>
struct PolicyTerms {
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

// The rollouts of the tokens that a warp passes through in ascending order, 128 at a time, four a lane.
struct RowWalk {
    const int64_t* start;
    int rows, r;                     // r: the rollout of the first token of the 128 at hand, or the one before the first
    long long begin, end;            // tokens that lie in a rollout

    __device__ __forceinline__ void find(const int64_t* row_start, int n_rows, long long first) {
        start = row_start;
        rows = n_rows;
        begin = start[0];
        end = start[rows];
        r = warp_row_between(start, 0, rows, first);
    }
    // Row of token t0 (this lane's) of the 128 that begin at w0, and the token behind its last; moves on.  Lanes look at the
    // next 32 starts together; where the 128 tokens have more rollouts they search for themselves.
    __device__ __forceinline__ int row_of(long long w0, long long t0, long long& until) {
        const int lane = threadIdx.x & 31;
        const int at = r + 1 + lane;
        const long long next = at < rows ? start[at] : INT64_MAX;       // start of rollout r + 1 + lane
        const unsigned within = __ballot_sync(0xFFFFFFFFu, next <= w0 + 127);
        int row = r;
        if (within == 0u) {                                      // all in one rollout
            until = INT64_MAX;
        } else if (within != 0xFFFFFFFFu) {
            // as many of the (ascending) starts as are not behind t0
            int before = 0;
#pragma unroll
            for (int step = 16; step > 0; step >>= 1) {
                const long long probe = __shfl_sync(0xFFFFFFFFu, next, before + step - 1);
                if (probe <= t0) before += step;
            }
            row = r + before;
            until = __shfl_sync(0xFFFFFFFFu, next, before & 31);
            r += __popc(__ballot_sync(0xFFFFFFFFu, next <= w0 + 128));
        } else {
            const int last = warp_row_between(start, r, rows, w0 + 128);
            row = row_between(start, r, last + 1, t0);
            until = row + 1 < rows ? start[row + 1] : INT64_MAX;
            r = last;
        }
        return row;
    }
};

// Terms of a token that counts, and the gradient of its log-probability.  `lp` is fp32 where it came from memory, fp64
// where it has just been computed.
//
// Two differences decide what is lost in 32 bits.  Whether rho is past a border of the clip range: rho in fp32 is off by up
// to 2^-22 of itself, so within 2^-20 of a border the comparison is made again in fp64 (a token on the wrong side has a
// wholly wrong gradient).  And e^d - 1 - d of policies that nearly agree: below 1/2 it is d^2 times the Taylor series of
// (e^d - 1 - d) / d^2, cut where the next term is below 2^-29 of the sum.
template <typename F>
__device__ __forceinline__ float policy_token(const PolicyBatch& b, const PolicyToken& k, F lp, PolicyTerms<float>& out) {
    const float A = k.adv, w = k.weight;
    float rho = lp == lp ? 1.0f : (float)lp;        // a NaN stays one
    const float border = A > 0.0f ? b.high : b.low;
    bool clipped = false;
    if (b.old_logp) {
        const F delta = lp - (F)k.old_logp;
        rho = expf((float)delta);
        clipped = A > 0.0f ? rho > border : A < 0.0f && rho < border;
        if (fabsf(rho - border) <= 9.5367431640625e-7f * border) {
            const double exact = exp((double)lp - (double)k.old_logp);
            clipped = A > 0.0f ? exact > 1.0 + b.clip_high : A < 0.0f && exact < 1.0 - b.clip_low;
        }
    }
    const float gain = A == 0.0f ? 0.0f : A * (clipped ? border : rho);
    float d_lp = clipped || A == 0.0f ? 0.0f : -A * rho;
    float kl = 0.0f;
    if (b.ref_logp) {
        const float d = (float)((F)k.ref_logp - lp);
        float em1;
        if (fabsf(d) < 0.5f) {
            float s = 1.0f / 362880.0f;
            s = fmaf(s, d, 1.0f / 40320.0f);
            s = fmaf(s, d, 1.0f / 5040.0f);
            s = fmaf(s, d, 1.0f / 720.0f);
            s = fmaf(s, d, 1.0f / 120.0f);
            s = fmaf(s, d, 1.0f / 24.0f);
            s = fmaf(s, d, 1.0f / 6.0f);
            s = fmaf(s, d, 0.5f);
            kl = s * d * d;
            em1 = d + kl;
        } else {
            em1 = expm1f(d);
            kl = em1 - d;
        }
        if (b.beta != 0.0) d_lp = fmaf(-(float)b.beta, em1, d_lp);
    }
    out.gain = w * gain;
    out.kl = w * kl;
    out.clipped = clipped ? w : 0.0f;
    out.rho = w * rho;
    return w * d_lp;
}

// The loss from the sums over all tokens.
__device__ __forceinline__ void write_policy_loss(const PolicyTerms<double>& sum, double beta, float* loss, float* stats) {
    *loss = (float)(beta != 0.0 ? beta * sum.kl - sum.gain : -sum.gain);
    if (stats) {
        stats[0] = (float)sum.gain;
        stats[1] = (float)sum.kl;
        stats[2] = (float)sum.clipped;
        stats[3] = (float)sum.rho;
    }
}

__device__ __forceinline__ void add_terms(PolicyTerms<double>& a, const PolicyTerms<double>& b) {
    a.gain += b.gain;
    a.kl += b.kl;
    a.clipped += b.clipped;
    a.rho += b.rho;
}

// Sum over the threads of a CTA, in thread 0; every thread takes part.  The order depends on the thread count alone.
__device__ __forceinline__ PolicyTerms<double> block_sum(PolicyTerms<double> v) {
    __shared__ PolicyTerms<double> s_warp[32];
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
        PolicyTerms<double> o;
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
// Sums the terms of n tokens into loss and stats.
int launch_sum_terms(const PolicyTerms<float>* terms, int n, double beta, float* loss, float* stats, double* partial, cudaStream_t s);

// logprob.cu
struct StepScratch {
    double* partial;                 // [kMaxPartials][4]
    PolicyTerms<float>* terms;       // [n_tokens]
    int32_t* row_of;                 // [n_tokens]
};
int launch_policy_loss_logits(const LogitsArgs& a, const PolicyBatch& b, float* loss, float* logp, void* d_logits, int64_t d_pitch, float* stats, int32_t* status,
                              const StepScratch& ws, cudaStream_t s);

}  // namespace sr
