// Clipped policy loss over packed rollouts: the weights that share it out, the loss and its gradient.
//
// Weights.  weight[r] needs the tokens of r that count and their total over the batch.  A warp takes 1024 mask bytes, 32 a
// lane, as bits with a prefix sum of their number; the rollouts that meet those bytes are then dealt to the lanes, each of
// which has its count from two look-ups, and one integer atomic adds it to the rollout's (whole numbers: any order gives the
// same).  One cluster then sums up and divides.  A byte per token and 16 bytes per rollout.
//
// Loss.  Four tokens a thread, 17 bytes a token, bound by HBM for large batches and by the launch for small ones.  Which
// rollout a token is in comes from a search of row_start by the warp for its first and last token; only where these differ
// do lanes search, between the two.
#include <cooperative_groups.h>

#include "policy.cuh"

namespace sr {
namespace {

// Bit k set iff byte k of the 32 from `at` on is non-zero and lies below `end`.
__device__ __forceinline__ uint32_t mask_bits(const uint8_t* __restrict__ mask, long long at, long long end) {
    uint32_t bits = 0u;
    if (at + 32 <= end && (reinterpret_cast<uintptr_t>(mask + at) & 15) == 0) {
        const uint4 a = __ldg(reinterpret_cast<const uint4*>(mask + at)), b = __ldg(reinterpret_cast<const uint4*>(mask + at) + 1);
        const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int q = 0; q < 8; ++q)      // one bit per byte, gathered by a product whose partial products do not meet
            bits |= (((__vminu4(w[q], 0x01010101u) * 0x00204081u) >> 21) & 0xFu) << (4 * q);
        return bits;
    }
    for (int k = 0; k < 32 && at + k < end; ++k) bits |= (mask[at + k] != 0 ? 1u : 0u) << k;
    return bits;
}

constexpr int kMaskTile = 1024;          // mask bytes a warp

__global__ void __launch_bounds__(256)
count_tokens_kernel(const int64_t* __restrict__ row_start, int rows, const uint8_t* __restrict__ mask, int n_tokens, int32_t* __restrict__ tokens) {
    grid_begin();
    const int lane = threadIdx.x & 31;
    const long long first = ((long long)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5)) * kMaskTile;
    if (first >= n_tokens) return;
    const long long last = min(first + kMaskTile, (long long)n_tokens);
    const uint32_t bits = mask_bits(mask, first + 32 * lane, last);
    const int own = __popc(bits);
    int before = own;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int up = __shfl_up_sync(0xFFFFFFFFu, before, d);
        if (lane >= d) before += up;
    }
    before -= own;
    // set bits below position `at` of the tile, 0 .. kMaskTile
    const int all = __shfl_sync(0xFFFFFFFFu, before + own, 31);
    auto below = [&](int at) {
        const uint32_t b = __shfl_sync(0xFFFFFFFFu, bits, (at >> 5) & 31);
        const int n = __shfl_sync(0xFFFFFFFFu, before, (at >> 5) & 31);
        return at >= kMaskTile ? all : n + __popc(b & low_mask(at & 31));
    };
    int r = warp_row_between(row_start, 0, rows, first) + lane;
    for (;; r += 32) {
        long long a = last, e = last;
        if (r < rows) {
            a = min(max((long long)__ldg(row_start + r), first), last);
            e = min(max((long long)__ldg(row_start + r + 1), a), last);
        }
        const int n = below((int)(e - first)) - below((int)(a - first));
        if (n > 0) atomicAdd(tokens + r, n);
        if (__all_sync(0xFFFFFFFFu, a >= last)) break;      // ascending starts: the rest lies behind the tile
        if (__shfl_sync(0xFFFFFFFFu, r, 31) >= rows - 1) break;
    }
}

constexpr int kWeightThreads = 1024;

// tokens: counts of the rollouts, or NULL where every token counts.
__global__ void __launch_bounds__(kWeightThreads)
loss_weights_kernel(const int64_t* __restrict__ row_start, const int32_t* __restrict__ tokens, const uint8_t* __restrict__ drop_mask, int N, int rows,
                    int mode, double scale, float* __restrict__ weight, int64_t* __restrict__ counts) {
    grid_begin();
    __shared__ long long s_tokens[32], s_total;
    __shared__ int s_live[32], s_rows;
    const int stride = gridDim.x * kWeightThreads, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    auto tokens_of = [&](int r) -> long long {
        if (drop_mask && drop_mask[r / N]) return 0;
        if (tokens) return tokens[r];
        return max((long long)(row_start[r + 1] - row_start[r]), 0LL);
    };
    long long sum = 0;
    int live = 0;
    for (long long r = blockIdx.x * kWeightThreads + threadIdx.x; r < rows; r += stride) {
        const long long n = tokens_of((int)r);
        sum += n;
        live += n > 0;
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
        sum += __shfl_xor_sync(0xFFFFFFFFu, sum, off);
        live += __shfl_xor_sync(0xFFFFFFFFu, live, off);
    }
    if (lane == 0) { s_tokens[warp] = sum; s_live[warp] = live; }
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kWeightThreads / 32; ++w) { sum += s_tokens[w]; live += s_live[w]; }
        s_total = sum;
        s_rows = live;
    }
    const auto cluster = cooperative_groups::this_cluster();
    cluster.sync();
    sum = 0;
    live = 0;
    for (unsigned b = 0; b < gridDim.x; ++b) {
        sum += *cluster.map_shared_rank(&s_total, b);
        live += *cluster.map_shared_rank(&s_rows, b);
    }
    cluster.sync();                        // nobody leaves while its sums are read
    if (counts && blockIdx.x == 0 && threadIdx.x == 0) { counts[0] = sum; counts[1] = live; }
    for (long long r = blockIdx.x * kWeightThreads + threadIdx.x; r < rows; r += stride) {
        const long long n = tokens_of((int)r);
        double w = scale;
        if (mode == SR_LOSS_TOKEN_MEAN) w /= (double)sum;
        if (mode == SR_LOSS_ROLLOUT_MEAN) w /= (double)live * (double)n;
        weight[r] = n > 0 ? (float)w : 0.0f;
    }
}

// kCluster: the grid is one cluster and its sums meet in shared memory: one launch.
template <bool kVec, bool kCluster>
__global__ void __launch_bounds__(kCluster ? 1024 : 256)
policy_loss_kernel(PolicyBatch b, const float* logp, float* d_logp, int n, double* __restrict__ partial, float* __restrict__ loss, float* __restrict__ stats) {
    grid_begin();
    const int lane = threadIdx.x & 31;
    PolicyTerms<double> sum = {0.0, 0.0, 0.0, 0.0};
    const long long rows_begin = b.rows > 0 ? __ldg(b.row_start) : 0, rows_end = b.rows > 0 ? __ldg(b.row_start + b.rows) : 0;
    for (long long t0 = ((long long)blockIdx.x * blockDim.x + threadIdx.x) * 4; t0 - 4 * lane < n; t0 += 4LL * gridDim.x * blockDim.x) {
        const long long w0 = t0 - 4 * lane;                     // the warp's tokens are w0 .. w0 + 127
        const int have = (int)max(0LL, min(4LL, n - t0));
        float lp[4] = {0.0f, 0.0f, 0.0f, 0.0f}, grad[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        if (kVec && have == 4) {
            const float4 v = *reinterpret_cast<const float4*>(logp + t0);
            lp[0] = v.x; lp[1] = v.y; lp[2] = v.z; lp[3] = v.w;
        } else {
            for (int k = 0; k < have; ++k) lp[k] = logp[t0 + k];
        }
        PolicyTerms<float> mine = {0.0f, 0.0f, 0.0f, 0.0f};
        if (b.rows > 0) {
            const int r_first = warp_row_between(b.row_start, 0, b.rows, w0);
            const int r_last = warp_row_between(b.row_start, r_first, b.rows, min(w0 + 127, (long long)n - 1));
            int r = r_first == r_last ? r_first : row_between(b.row_start, r_first, r_last + 1, t0);
            for (int k = 0; k < have; ++k) {
                const long long t = t0 + k;
                if (t < rows_begin || t >= rows_end || (b.mask && b.mask[t] == 0)) continue;
                while (r < r_last && __ldg(b.row_start + r + 1) <= t) ++r;
                const float w = __ldg(b.weight + r);
                if (w == 0.0f) continue;
                PolicyTerms<float> term;
                grad[k] = policy_token(b, (size_t)t, lp[k], __ldg(b.adv + r), w, term);
                mine.gain += term.gain;
                mine.kl += term.kl;
                mine.clipped += term.clipped;
                mine.rho += term.rho;
            }
        }
        sum.gain += (double)mine.gain;
        sum.kl += (double)mine.kl;
        sum.clipped += (double)mine.clipped;
        sum.rho += (double)mine.rho;
        if (d_logp) {
            if (kVec && have == 4) *reinterpret_cast<float4*>(d_logp + t0) = make_float4(grad[0], grad[1], grad[2], grad[3]);
            else
                for (int k = 0; k < have; ++k) d_logp[t0 + k] = grad[k];
        }
    }
    sum = block_sum(sum);
    if (kCluster) {
        __shared__ PolicyTerms<double> s_sum;
        const auto cluster = cooperative_groups::this_cluster();
        if (threadIdx.x == 0) s_sum = sum;
        cluster.sync();
        if (blockIdx.x == 0 && threadIdx.x == 0) {
            for (unsigned c = 1; c < gridDim.x; ++c) add_terms(sum, *cluster.map_shared_rank(&s_sum, c));
            write_policy_loss(sum, b.beta, loss, stats);
        }
        cluster.sync();                        // nobody leaves while its sums are read
    } else if (threadIdx.x == 0) {
        reinterpret_cast<PolicyTerms<double>*>(partial)[blockIdx.x] = sum;
    }
}

// Sums of terms: of the CTAs before (double), or of the tokens themselves (float).
template <typename F>
__global__ void __launch_bounds__(256)
sum_terms_kernel(const PolicyTerms<F>* __restrict__ terms, int n, double beta, PolicyTerms<double>* __restrict__ partial, float* __restrict__ loss, float* __restrict__ stats) {
    grid_begin();
    PolicyTerms<double> sum = {0.0, 0.0, 0.0, 0.0};
    for (long long i = blockIdx.x * 256 + threadIdx.x; i < n; i += gridDim.x * 256) {
        const PolicyTerms<F> t = terms[i];
        add_terms(sum, PolicyTerms<double>{(double)t.gain, (double)t.kl, (double)t.clipped, (double)t.rho});
    }
    sum = block_sum(sum);
    if (threadIdx.x != 0) return;
    if (gridDim.x == 1) write_policy_loss(sum, beta, loss, stats);
    else partial[blockIdx.x] = sum;
}

}  // namespace

int launch_loss_weights(const int64_t* row_start, const uint8_t* mask, int32_t n_tokens, const uint8_t* drop_mask, int32_t n_groups, int32_t N, int32_t mode,
                        double scale, float* weight, int64_t* counts, void* ws, cudaStream_t s) {
    const int rows = n_groups * N;
    if (rows == 0) {
        if (counts) SR_CUDA_TRY(cudaMemsetAsync(counts, 0, 2 * sizeof(int64_t), s));
        return SR_OK;
    }
    int32_t* const tokens = mask ? static_cast<int32_t*>(ws) : nullptr;
    if (mask) {
        SR_CUDA_TRY(cudaMemsetAsync(tokens, 0, (size_t)rows * sizeof(int32_t), s));
        const int tiles = (int)(((long long)n_tokens + kMaskTile - 1) / kMaskTile);
        if (tiles > 0) SR_LAUNCH("count_tokens_kernel", count_tokens_kernel, (tiles + 7) / 8, 256, 0, s, row_start, rows, mask, n_tokens, tokens);
    }
    int ctas = 1;                                  // up to the portable cluster size
    while (ctas < 8 && ctas * kWeightThreads < rows) ctas *= 2;
    return launch_as(true, ctas, "loss_weights_kernel", loss_weights_kernel, ctas, kWeightThreads, 0, s, row_start, tokens, drop_mask, N, rows, mode, scale, weight, counts);
}

int launch_sum_terms(const PolicyTerms<float>* terms, int n, double beta, float* loss, float* stats, double* partial, cudaStream_t s) {
    auto* const part = reinterpret_cast<PolicyTerms<double>*>(partial);
    const int blocks = n > 8192 ? min(kMaxPartials, (n + 2047) / 2048) : 1;
    SR_LAUNCH("sum_terms_kernel", sum_terms_kernel<float>, blocks, 256, 0, s, terms, n, beta, part, loss, stats);
    if (blocks > 1) SR_LAUNCH("sum_terms_kernel", sum_terms_kernel<double>, 1, 256, 0, s, part, blocks, beta, part, loss, stats);
    return SR_OK;
}

int launch_policy_loss(const PolicyBatch& b, const float* logp, int32_t n, float* loss, float* d_logp, float* stats, double* partial, cudaStream_t s) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(logp) | reinterpret_cast<uintptr_t>(d_logp);
    const bool vec = (at & 15) == 0;
    if (n <= 8 * 1024 * 4) {
        int ctas = 1;
        while (ctas < 8 && ctas * 1024 < n) ctas *= 2;
        const int threads = max(32, ((n + ctas * 4 - 1) / (ctas * 4) + 31) & ~31);
        return launch_as(true, ctas, "policy_loss_kernel", vec ? policy_loss_kernel<true, true> : policy_loss_kernel<false, true>, ctas, threads, 0, s, b, logp, d_logp, n, partial, loss, stats);
    }
    const int blocks = (int)min((long long)kMaxPartials, ((long long)n + 1023) / 1024);
    SR_LAUNCH("policy_loss_kernel", vec ? policy_loss_kernel<true, false> : policy_loss_kernel<false, false>, blocks, 256, 0, s, b, logp, d_logp, n, partial, loss, stats);
    auto* const part = reinterpret_cast<PolicyTerms<double>*>(partial);
    SR_LAUNCH("sum_terms_kernel", sum_terms_kernel<double>, 1, 256, 0, s, part, blocks, b.beta, part, loss, stats);
    return SR_OK;
}

}  // namespace sr
