// Clipped policy loss over packed rollouts: the weights that share it out, the loss and its gradient.
//
// Weights.  weight[r] needs the tokens of r that count and their total over the batch.  A warp counts a rollout's mask bytes, 32 a
// lane; one cluster then sums up and divides.  A byte per token and 16 bytes per rollout: bound by the launches and by their chains
// of dependent loads (8192 rollouts, 5.2M tokens: 8 us; 80 rollouts in one launch: 3).
//
// Loss.  Four tokens a thread, 17 bytes a token.  A warp searches row_start once, for the first of its tokens, and moves on from
// there: 128 tokens mostly lie in one rollout or a few, whose starts the lanes look at together.  5.2M tokens take 28 us, 3.1 TB/s:
// bound by 97 instructions a token and their latency, with one or two lots of 128 ahead; with fewer registers three CTAs an SM took as
// long as two, four longer.
// With a search and branches for every token it took 60.
#include <cooperative_groups.h>
#include <math_constants.h>

#include "policy.cuh"

namespace sr {
namespace {

// Mask bytes of [a, e) that are not zero, among the 32 from `at` on, and 0 <= a, e <= n_tokens; `at` lies so that a vector may be
// loaded there.
__device__ __forceinline__ int count_32(const uint8_t* mask, int n_tokens, long long a, long long e, long long at) {
    const int lo = (int)max(0LL, min(32LL, a - at)), hi = (int)max(0LL, min(32LL, e - at));
    if (lo >= hi) return 0;
    if (at >= 0 && at + 32 <= n_tokens) {
        const uint4 x = reinterpret_cast<const uint4*>(mask + at)[0], y = reinterpret_cast<const uint4*>(mask + at)[1];
        const uint32_t w[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
        uint32_t bits = 0u;
#pragma unroll
        for (int q = 0; q < 8; ++q)      // one bit per byte, gathered by a product whose partial products do not meet
            bits |= (((__vminu4(w[q], 0x01010101u) * 0x00204081u) >> 21) & 0xFu) << (4 * q);
        return __popc(bits & low_mask(hi) & ~low_mask(lo));
    }
    int n = 0;
    for (int k = lo; k < hi; ++k) n += mask[at + k] != 0;
    return n;
}

constexpr int kLongRollout = 16384;      // mask bytes: a whole CTA counts them
constexpr int kRowsOfCta = 256;          // at most

// Tokens that count of rollouts first .. first + rows - 1, by a CTA: a warp to a rollout, and all of it to a long one.
// Rollouts of groups that are cut are not looked at.
__device__ __forceinline__ void count_rows(const int64_t* row_start, const uint8_t* mask, int n_tokens,
                                           const uint8_t* drop_mask, int N, int first, int rows, int32_t* s_count) {
    __shared__ int s_part[32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const int off = (int)((16 - (reinterpret_cast<uintptr_t>(mask) & 15)) & 15);         // positions off, off + 16, ... are aligned
    const auto begin_of = [&](long long a) { return a - ((a - off) & 15); };
    int any_long = 0;
    for (int i = warp; i < rows; i += warps) {
        long long a = 0, e = 0;
        if (!(drop_mask && drop_mask[(first + i) / N])) {
            a = min(max((long long)row_start[first + i], 0LL), (long long)n_tokens);
            e = min(max((long long)row_start[first + i + 1], a), (long long)n_tokens);
        }
        int n = 0;
        if (e - a > kLongRollout) {
            n = -1;
            any_long = 1;
        } else {
            for (long long at = begin_of(a) + 32 * lane; at < e; at += 1024) n += count_32(mask, n_tokens, a, e, at);
            n = __reduce_add_sync(0xFFFFFFFFu, n);
        }
        if (lane == 0) s_count[i] = n;
    }
    if (!__syncthreads_or(any_long)) return;
    for (int i = 0; i < rows; ++i) {
        if (s_count[i] >= 0) continue;
        const long long a = max((long long)row_start[first + i], 0LL), e = min((long long)row_start[first + i + 1], (long long)n_tokens);
        int n = 0;
        for (long long at = begin_of(a) + 32LL * threadIdx.x; at < e; at += 32LL * blockDim.x) n += count_32(mask, n_tokens, a, e, at);
        n = __reduce_add_sync(0xFFFFFFFFu, n);
        if (lane == 0) s_part[warp] = n;
        __syncthreads();
        if (threadIdx.x == 0) {
            for (int w = 1; w < warps; ++w) n += s_part[w];
            s_count[i] = n;
        }
        __syncthreads();
    }
}

__global__ void __launch_bounds__(256)
count_tokens_kernel(const int64_t* row_start, int rows, const uint8_t* mask, int n_tokens, const uint8_t* drop_mask, int N, int rows_of_cta,
                    int32_t* tokens) {
    grid_begin();
    __shared__ int32_t s_count[kRowsOfCta];
    const int first = blockIdx.x * rows_of_cta, have = min(rows_of_cta, rows - first);
    count_rows(row_start, mask, n_tokens, drop_mask, N, first, have, s_count);
    for (int i = threadIdx.x; i < have; i += 256) tokens[first + i] = s_count[i];
}

constexpr int kWeightThreads = 1024;

// One cluster.  kCount: its CTAs count the tokens of up to kRowsOfCta rollouts each; otherwise `tokens` holds the counts, or is
// NULL where every token counts (n_tokens is the mask's size, and not looked at then).
template <bool kCount>
__global__ void __launch_bounds__(kWeightThreads)
loss_weights_kernel(const int64_t* row_start, const uint8_t* mask, int n_tokens, const int32_t* tokens,
                    const uint8_t* drop_mask, int N, int rows, int mode, double scale, float* weight, int64_t* counts) {
    grid_begin();
    cluster_arrive();
    __shared__ long long s_tokens[32], s_total[8];
    __shared__ int s_live[32], s_rows[8];
    __shared__ int32_t s_count[kCount ? kRowsOfCta : 1];
    const auto cluster = cooperative_groups::this_cluster();
    const int ctas = gridDim.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const int first = (int)((long long)rows * blockIdx.x / ctas), last = (int)((long long)rows * (blockIdx.x + 1) / ctas);
    if (kCount) {
        count_rows(row_start, mask, n_tokens, drop_mask, N, first, last - first, s_count);
        __syncthreads();
    }
    const auto tokens_of = [&](int r) -> long long {
        if (kCount) return s_count[r - first];
        if (tokens) return tokens[r];
        if (drop_mask && drop_mask[r / N]) return 0;
        return max((long long)(row_start[r + 1] - row_start[r]), 0LL);
    };
    const int own = first + (int)threadIdx.x;                  // most batches have no more rollouts than threads
    const long long own_tokens = own < last ? tokens_of(own) : 0;
    long long sum = own_tokens;
    int live = own_tokens > 0;
    for (long long r = (long long)own + blockDim.x; r < last; r += blockDim.x) {
        const long long n = tokens_of((int)r);
        sum += n;
        live += n > 0;
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, off);
    live = __reduce_add_sync(0xFFFFFFFFu, live);
    if (lane == 0) { s_tokens[warp] = sum; s_live[warp] = live; }
    __syncthreads();
    cluster_wait();
    if (warp == 0) {
        sum = lane < warps ? s_tokens[lane] : 0;
        live = __reduce_add_sync(0xFFFFFFFFu, lane < warps ? s_live[lane] : 0);
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, off);
        if (lane < ctas) {                 // to every CTA's own memory: after the barrier nobody reads another's
            *cluster.map_shared_rank(&s_total[blockIdx.x], lane) = sum;
            *cluster.map_shared_rank(&s_rows[blockIdx.x], lane) = live;
        }
    }
    cluster.sync();
    sum = 0;
    live = 0;
    for (int c = 0; c < ctas; ++c) { sum += s_total[c]; live += s_rows[c]; }
    if (counts && blockIdx.x == 0 && threadIdx.x == 0) { counts[0] = sum; counts[1] = live; }
    const auto weigh = [&](long long r, long long n) {
        double w = scale;
        if (mode == SR_LOSS_TOKEN_MEAN) w /= (double)sum;
        if (mode == SR_LOSS_ROLLOUT_MEAN) w /= (double)live * (double)n;
        weight[r] = n > 0 ? (float)w : 0.0f;
    };
    if (own < last) weigh(own, own_tokens);
    for (long long r = (long long)own + blockDim.x; r < last; r += blockDim.x) weigh(r, tokens_of((int)r));
}

// What thread 0 of every CTA does with its sum.  kCluster: the grid is one cluster, whose sums meet in shared memory and become
// the loss; its threads have arrived at the cluster's barrier.  failed: terms are missing, loss and figures become NaN.
template <bool kCluster>
__device__ __forceinline__ void leave_sum(PolicySums<double> sum, double beta, bool failed, double* partial, float* loss, float* stats) {
    if (!kCluster) {
        if (threadIdx.x == 0) reinterpret_cast<PolicySums<double>*>(partial)[blockIdx.x] = sum;
        return;
    }
    __shared__ PolicySums<double> s_sum[8];
    const auto cluster = cooperative_groups::this_cluster();
    cluster_wait();
    if (threadIdx.x == 0) *cluster.map_shared_rank(&s_sum[blockIdx.x], 0) = sum;
    cluster.sync();                        // the first CTA's memory alone is read after it
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        for (unsigned c = 1; c < gridDim.x; ++c) add_terms(sum, s_sum[c]);
        if (failed) sum.gain = sum.kl = sum.clipped = sum.rho = CUDART_NAN;
        write_policy_loss(sum, beta, loss, stats);
    }
}

// Gradient and terms of the rare token that the code below leaves to this.
__device__ __noinline__ float one_token(const PolicyBatch& b, float old_logp, float ref_logp, float adv, float weight, float lp, PolicyTerms& out) {
    const PolicyToken token{old_logp, ref_logp, adv, weight};
    PolicyParts parts;
    const float gradient = policy_gradient(b, token, lp, parts);
    out = policy_terms(b, token, parts);
    return gradient;
}
// The same of four tokens side by side, two to an instruction and without branches: one that does not count (bit 8 j of
// `counts`) has policies that agree.  Lanes that need another look (a ratio at a border of the clip range, numbers near overflow, a NaN, which
// a factor of 0 would not take away here) take their tokens one by one.  kOne: they lie in one rollout, w[0] and a[0] are its.
//
// Advantages of a group add up to 0, and the loss is a small difference of large terms.  So what is added up in fp32 is w A (rho - 1), from
// the series that the KL term has, and w A by itself goes into sum_gain, in fp64.  A token that does not count has rho - 1 = 0 and adds
// nothing to the sums.
template <bool kOne>
__device__ __forceinline__ void four_tokens(const PolicyBatch& b, const float (&lp)[4], const float (&old_logp)[4], const float (&ref_logp)[4], const float (&w)[4],
                                            const float (&a)[4], uint32_t counts, float (&grad)[4], PolicySums<float>& sum, double& sum_gain) {
    const float inf = __int_as_float(0x7F800000);
    bool again = false, is[4], past[4];
    float A[4], rho[4], less[4], used[4], kl[4] = {0.0f, 0.0f, 0.0f, 0.0f}, delta[4] = {0.0f, 0.0f, 0.0f, 0.0f};      // less: rho - 1, to its own size; used: within the clip range
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        is[j] = (counts >> (8 * j)) & 1u;
        A[j] = kOne ? (counts != 0u ? a[0] : 0.0f) : is[j] ? a[j] : 0.0f;
    }
    if (!b.old_logp) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            less[j] = is[j] && !(lp[j] == lp[j]) ? lp[j] : 0.0f;    // a NaN stays one
            rho[j] = 1.0f + less[j];
        }
    } else {
#pragma unroll
        for (int j = 0; j < 4; j += 2) {
            if (is[j]) delta[j] = lp[j] - old_logp[j];
            if (is[j + 1]) delta[j + 1] = lp[j + 1] - old_logp[j + 1];
            again |= !(fabsf(delta[j]) <= 80.0f) || !(fabsf(delta[j + 1]) <= 80.0f);
            f32x2 e, em1;
            exp_near(two(delta[j], delta[j + 1]), e, em1);
            rho[j] = low_of(e);
            rho[j + 1] = high_of(e);
            less[j] = low_of(em1);
            less[j + 1] = high_of(em1);
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float border = A[j] > 0.0f ? b.high : b.low, less_border = A[j] > 0.0f ? b.less_high : b.less_low;
        used[j] = fminf(fmaxf(less[j], A[j] < 0.0f ? b.less_low : -inf), A[j] > 0.0f ? b.less_high : inf);
        past[j] = used[j] != less[j];
        grad[j] = -A[j] * (past[j] ? 0.0f : rho[j]);
        again |= !(fabsf(less[j] - less_border) > fmaf(fabsf(delta[j]), kMarginSlope * border, kMargin * border));      // also: NaN
    }
    if (b.ref_logp) {
#pragma unroll
        for (int j = 0; j < 4; j += 2) {
            const float d0 = is[j] ? ref_logp[j] - lp[j] : 0.0f, d1 = is[j + 1] ? ref_logp[j + 1] - lp[j + 1] : 0.0f;
            again |= !(fabsf(d0) <= 80.0f) || !(fabsf(d1) <= 80.0f);
            f32x2 em1, both;
            exp_less_line_near(two(d0, d1), em1, both);
            kl[j] = low_of(both);
            kl[j + 1] = high_of(both);
            grad[j] = fmaf(-b.beta32, low_of(em1), grad[j]);
            grad[j + 1] = fmaf(-b.beta32, high_of(em1), grad[j + 1]);
        }
    }
    if (again) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            PolicyTerms term = {0.0, 0.0f, 0.0f, 0.0f};
            grad[j] = is[j] ? one_token(b, old_logp[j], ref_logp[j], A[j], kOne ? w[0] : w[j], lp[j], term) : 0.0f;
            sum_gain += term.gain;
            sum.kl += term.kl;
            sum.clipped += term.clipped;
            sum.rho += term.rho;
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        rho[j] = is[j] ? rho[j] : 0.0f;
        grad[j] = is[j] ? (kOne ? w[0] : w[j]) * grad[j] : 0.0f;
    }
    const auto of = [&](int j) { return past[j] ? 1.0f : 0.0f; };
    if (kOne) {
        sum_gain += (double)__popc(counts) * ((double)w[0] * (double)A[0]);
        sum.gain = fmaf(w[0] * A[0], (used[0] + used[1]) + (used[2] + used[3]), sum.gain);
        sum.kl = fmaf(w[0], (kl[0] + kl[1]) + (kl[2] + kl[3]), sum.kl);
        sum.clipped = fmaf(w[0], (of(0) + of(1)) + (of(2) + of(3)), sum.clipped);
        sum.rho = fmaf(w[0], (rho[0] + rho[1]) + (rho[2] + rho[3]), sum.rho);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float weight = is[j] ? w[j] : 0.0f;
            sum_gain += (double)weight * (double)A[j];
            sum.gain = fmaf(weight * A[j], used[j], sum.gain);
            sum.kl = fmaf(weight, kl[j], sum.kl);
            sum.clipped = fmaf(weight, of(j), sum.clipped);
            sum.rho = fmaf(weight, rho[j], sum.rho);
        }
    }
}

// kCluster: one launch, see leave_sum.  A warp has a run of tokens, 128 at a time; the next lot is on its way while it works on
// one.
template <bool kVec, bool kCluster>
__global__ void __launch_bounds__(kCluster ? 512 : 256, kCluster ? 1 : 2)
policy_loss_kernel(const __grid_constant__ PolicyBatch b, const float* logp, float* d_logp, int n, double* partial, float* loss,
                   float* stats) {
    grid_begin();
    if (kCluster) cluster_arrive();
    const int lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    const int all = gridDim.x * warps, warp = blockIdx.x * warps + (threadIdx.x >> 5);
    const uint32_t tokens = (uint32_t)n;                       // token numbers are unsigned: the last lot may end behind 2^31
    const long long lots = ((long long)n + 127) >> 7;
    uint32_t lot = (uint32_t)(lots * warp / all);
    const uint32_t end = (uint32_t)(lots * (warp + 1) / all);
    PolicySums<double> sum = {0.0, 0.0, 0.0, 0.0};
    PolicySums<float> mine = {0.0f, 0.0f, 0.0f, 0.0f};
    struct Four {
        float lp[4], old_logp[4], ref_logp[4];
        uint32_t mask;
    } next;
    auto load = [&](uint32_t t0) {
        Four next;
        if (kVec && t0 + 4 <= tokens) {
            const float4 v = *reinterpret_cast<const float4*>(logp + t0);
            next.lp[0] = v.x; next.lp[1] = v.y; next.lp[2] = v.z; next.lp[3] = v.w;
            if (b.old_logp) {
                const float4 o = *reinterpret_cast<const float4*>(b.old_logp + t0);
                next.old_logp[0] = o.x; next.old_logp[1] = o.y; next.old_logp[2] = o.z; next.old_logp[3] = o.w;
            }
            if (b.ref_logp) {
                const float4 f = *reinterpret_cast<const float4*>(b.ref_logp + t0);
                next.ref_logp[0] = f.x; next.ref_logp[1] = f.y; next.ref_logp[2] = f.z; next.ref_logp[3] = f.w;
            }
            next.mask = b.mask ? *reinterpret_cast<const uint32_t*>(b.mask + t0) : 0xFFFFFFFFu;
            return next;
        }
        next.mask = 0u;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (t0 + k >= tokens) continue;
            next.lp[k] = logp[t0 + k];
            if (b.old_logp) next.old_logp[k] = b.old_logp[t0 + k];
            if (b.ref_logp) next.ref_logp[k] = b.ref_logp[t0 + k];
            next.mask |= (b.mask ? (uint32_t)b.mask[t0 + k] : 1u) << (8 * k);
        }
        return next;
    };
    if (lot < end) next = load((lot << 7) + 4 * lane);
    RowWalk walk;
    if (lot < end && b.rows > 0) walk.find(b, lot << 7);
    for (; lot < end; ++lot) {
        const Four four = next;
        const uint32_t w0 = lot << 7, t0 = w0 + 4 * lane;
        if (lot + 1 < end) next = load(t0 + 128);
        float grad[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        if (b.rows > 0) {
            uint32_t counts = four.mask;
            if (w0 < walk.begin || walk.end - w0 < 128u || w0 >= walk.end) {    // some lie in no rollout
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (t0 + j < walk.begin || t0 + j >= walk.end) counts &= ~(0xFFu << (8 * j));
            }
            counts = __vminu4(counts, 0x01010101u);
            float w[4], a[4];
            if (walk.one_rollout(w0, w[0], a[0])) {
                if (w[0] != 0.0f) four_tokens<true>(b, four.lp, four.old_logp, four.ref_logp, w, a, counts, grad, mine, sum.gain);
            } else {
                walk.several_rollouts(w0, t0, w, a);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (w[j] == 0.0f) counts &= ~(1u << (8 * j));
                four_tokens<false>(b, four.lp, four.old_logp, four.ref_logp, w, a, counts, grad, mine, sum.gain);
            }
        }
        if ((lot & 3u) == 3u || lot + 1 == end) {        // fp32 over up to 16 tokens, fp64 from there on
            sum.gain += (double)mine.gain;
            sum.kl += (double)mine.kl;
            sum.clipped += (double)mine.clipped;
            sum.rho += (double)mine.rho;
            mine = PolicySums<float>{0.0f, 0.0f, 0.0f, 0.0f};
        }
        if (d_logp) {
            if (kVec && t0 + 4 <= tokens) {
                *reinterpret_cast<float4*>(d_logp + t0) = make_float4(grad[0], grad[1], grad[2], grad[3]);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (t0 + j < tokens) d_logp[t0 + j] = grad[j];
            }
        }
    }
    leave_sum<kCluster>(block_sum(sum), b.beta, false, partial, loss, stats);
}

// Sums of terms: of the tokens (PolicyTerms), or of the CTAs before (PolicySums<double>).
template <typename Terms, bool kCluster>
__global__ void __launch_bounds__(1024)
sum_terms_kernel(const Terms* terms, int n, double beta, const int32_t* gave_up, double* partial, float* loss, float* stats) {
    grid_begin();
    if (kCluster) cluster_arrive();
    const bool failed = kCluster && gave_up != nullptr && *gave_up != 0;
    PolicySums<double> sum = {0.0, 0.0, 0.0, 0.0};
#pragma unroll 4
    for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (long long)gridDim.x * blockDim.x) {
        const Terms t = terms[i];
        add_terms(sum, PolicySums<double>{(double)t.gain, (double)t.kl, (double)t.clipped, (double)t.rho});
    }
    leave_sum<kCluster>(block_sum(sum), beta, failed, partial, loss, stats);
}

}  // namespace

int launch_loss_weights(const int64_t* row_start, const uint8_t* mask, int32_t n_tokens, const uint8_t* drop_mask, int32_t n_groups, int32_t N, int32_t mode,
                        double scale, float* weight, int64_t* counts, void* ws, cudaStream_t s) {
    const int rows = n_groups * N;
    if (rows == 0) {
        if (counts) SR_CUDA_TRY(cudaMemsetAsync(counts, 0, 2 * sizeof(int64_t), s));
        return SR_OK;
    }
    // Masked batches of up to 2048 rollouts and 65536 tokens are counted in the cluster itself, in one launch; eight SMs would take
    // 15 us for 770000 tokens, a launch of its own on all SMs 5.
    const bool here = mask != nullptr && rows <= 8 * kRowsOfCta && n_tokens <= 1 << 16;
    int32_t* const tokens = mask && !here ? static_cast<int32_t*>(ws) : nullptr;
    if (tokens) {
        const int of_cta = min(kRowsOfCta, max(8, rows / (148 * 8) & ~7));
        SR_LAUNCH("count_tokens_kernel", count_tokens_kernel, (rows + of_cta - 1) / of_cta, 256, 0, s, row_start, rows, mask, n_tokens, drop_mask, N, of_cta, tokens);
    }
    // up to the portable cluster size
    const int ctas = here ? min(8, (rows + 31) / 32) : min(8, (int)(((long long)rows + kWeightThreads - 1) / kWeightThreads));
    const int threads = here ? kWeightThreads : min(kWeightThreads, (rows + 31) & ~31);
    return launch_as(true, ctas, "loss_weights_kernel", here ? loss_weights_kernel<true> : loss_weights_kernel<false>, ctas, threads, 0, s, row_start, mask, n_tokens, tokens,
                     drop_mask, N, rows, mode, scale, weight, counts);
}

// Up to 32768 tokens, four a thread, and sums of up to 131072 are one cluster's work: one launch.
int launch_sum_terms(const PolicyTerms* terms, int n, double beta, const int32_t* gave_up, float* loss, float* stats, double* partial, cudaStream_t s) {
    if (n <= 1 << 17) {
        const int ctas = max(1, min(8, (n + 1023) / 1024)), threads = max(32, min(1024, (n + 31) & ~31));
        return launch_as(true, ctas, "sum_terms_kernel", sum_terms_kernel<PolicyTerms, true>, ctas, threads, 0, s, terms, n, beta, gave_up, partial, loss, stats);
    }
    const int blocks = (int)min((long long)kMaxPartials, ((long long)n + 4095) / 4096);
    SR_LAUNCH("sum_terms_kernel", sum_terms_kernel<PolicyTerms, false>, blocks, 1024, 0, s, terms, n, beta, gave_up, partial, loss, stats);
    SR_LAUNCH("sum_terms_kernel", sum_terms_kernel<PolicySums<double>, true>, 1, 1024, 0, s, reinterpret_cast<const PolicySums<double>*>(partial), blocks, beta, gave_up, partial, loss, stats);
    return SR_OK;
}

int launch_policy_loss(const PolicyBatch& b, const float* logp, int32_t n, float* loss, float* d_logp, float* stats, double* partial, cudaStream_t s) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(logp) | reinterpret_cast<uintptr_t>(d_logp) | reinterpret_cast<uintptr_t>(b.old_logp) | reinterpret_cast<uintptr_t>(b.ref_logp);
    const bool vec = (at & 15) == 0 && (reinterpret_cast<uintptr_t>(b.mask) & 3) == 0;
    if (n <= 8 * 1024 * 4) {
        const int lots = (n + 127) / 128, ctas = max(1, min(8, (lots + 15) / 16)), threads = max(1, min(16, (lots + ctas - 1) / ctas)) * 32;
        return launch_as(true, ctas, "policy_loss_kernel", vec ? policy_loss_kernel<true, true> : policy_loss_kernel<false, true>, ctas, threads, 0, s, b, logp, d_logp, n, partial, loss, stats);
    }
    const int blocks = (int)min((long long)(148 * 2), ((long long)n + 1023) / 1024);
    SR_LAUNCH("policy_loss_kernel", vec ? policy_loss_kernel<true, false> : policy_loss_kernel<false, false>, blocks, 256, 0, s, b, logp, d_logp, n, partial, loss, stats);
    SR_LAUNCH("sum_terms_kernel", sum_terms_kernel<PolicySums<double>, true>, 1, 1024, 0, s, reinterpret_cast<const PolicySums<double>*>(partial), blocks, b.beta, static_cast<const int32_t*>(nullptr), partial, loss, stats);
    return SR_OK;
}

}  // namespace sr
