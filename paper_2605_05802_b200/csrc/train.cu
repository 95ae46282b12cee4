// extern "C" boundary of the trainer's operators (sr_train.h): argument checks and dispatch.
#include <math.h>

#include <algorithm>
#include <new>

#include "checks.cuh"
#include "policy.cuh"

using namespace sr;

namespace {

// What every call on logits has in common.
int check_logits(const void* logits, int32_t dtype, int32_t n_tokens, int32_t vocab, int64_t pitch, const int32_t* targets, double temperature) {
    if (n_tokens < 0 || vocab < 1 || pitch < vocab || pitch > kMaxPitch) return SR_ERR_BAD_SIZE;
    if (dtype_bytes(dtype) == 0) return SR_ERR_BAD_DTYPE;
    // 1 / temperature and its product with log2(e) are ordinary fp32 numbers
    if (!(temperature >= 1e-30 && temperature <= 1e30)) return SR_ERR_BAD_VALUE;
    if (n_tokens > 0 && (logits == nullptr || targets == nullptr)) return SR_ERR_NULL;
    if (!aligned(logits, dtype_bytes(dtype)) || !aligned(targets, 4)) return SR_ERR_ALIGN;
    return SR_OK;
}

int check_policy(const float* adv, const float* weight, const int64_t* row_start, int32_t n_rollouts, double clip_low, double clip_high, double beta, const float* loss) {
    if (n_rollouts < 0 || n_rollouts > (1 << 30)) return SR_ERR_BAD_N;
    if (!(clip_low >= 0.0 && clip_high >= 0.0 && beta >= 0.0) || isinf(clip_low) || isinf(clip_high) || beta > kLargest) return SR_ERR_BAD_VALUE;
    if (loss == nullptr || (n_rollouts > 0 && (adv == nullptr || weight == nullptr || row_start == nullptr))) return SR_ERR_NULL;
    if (!aligned(row_start, 8) || !aligned_4(adv, weight, loss)) return SR_ERR_ALIGN;
    return SR_OK;
}

int check_grads(const void* const* grads, const int64_t* counts, const int32_t* dtypes, int32_t n_tensors) {
    if (n_tensors < 0) return SR_ERR_BAD_N;
    if (n_tensors > 0 && (grads == nullptr || counts == nullptr || dtypes == nullptr)) return SR_ERR_NULL;
    int64_t pieces = 0;
    for (int i = 0; i < n_tensors; ++i) {
        if (counts[i] < 0) return SR_ERR_BAD_SIZE;
        const int size = dtype_bytes(dtypes[i]);
        if (size == 0) return SR_ERR_BAD_DTYPE;
        pieces += grad_pieces(counts[i], dtypes[i]);                // of one tensor below 2^52
        if (pieces > INT32_MAX) return SR_ERR_BAD_SIZE;
        if (counts[i] > 0 && grads[i] == nullptr) return SR_ERR_NULL;
        if (!aligned(grads[i], size)) return SR_ERR_ALIGN;
    }
    return SR_OK;
}

struct Range {
    uintptr_t begin, end;
};
// Whether a range that is written reaches into another of them or into one that is read.  Sorts both lists, which mostly are (a
// program's gradients follow one another): together they would not be.
bool overlap(Range* written, size_t n_written, Range* read, size_t n_read) {
    const auto before = [](const Range& x, const Range& y) { return x.begin < y.begin; };
    if (!std::is_sorted(written, written + n_written, before)) std::sort(written, written + n_written, before);
    if (!std::is_sorted(read, read + n_read, before)) std::sort(read, read + n_read, before);
    for (size_t i = 1; i < n_written; ++i)
        if (written[i - 1].end > written[i].begin) return true;
    for (size_t i = 0, w = 0; i < n_read; ++i) {
        while (w < n_written && written[w].end <= read[i].begin) ++w;
        if (w < n_written && written[w].begin < read[i].end) return true;
    }
    return false;
}

constexpr size_t kPartialBytes = (size_t)kMaxPartials * 4 * sizeof(double);

}  // namespace

extern "C" {

int sr_token_logprob(const void* logits, int32_t dtype, int32_t n_tokens, int32_t vocab, int64_t pitch, const int32_t* targets, double temperature, float* logp,
                     float* row_stats, float* entropy, int32_t* status, void* stream) {
    const int rc = check_logits(logits, dtype, n_tokens, vocab, pitch, targets, temperature);
    if (rc != SR_OK) return rc;
    if (n_tokens > 0 && logp == nullptr) return SR_ERR_NULL;
    if (!aligned_4(logp, row_stats, entropy, status)) return SR_ERR_ALIGN;
    return launch_token_logprob(LogitsArgs{logits, dtype, n_tokens, vocab, pitch, targets, temperature}, logp, row_stats, entropy, status, static_cast<cudaStream_t>(stream));
}

int sr_token_logprob_backward(const void* logits, int32_t dtype, int32_t n_tokens, int32_t vocab, int64_t pitch, const int32_t* targets, const float* row_stats,
                              const float* entropy, const float* d_logp, const float* d_entropy, double temperature, void* d_logits, int64_t d_pitch, void* stream) {
    int rc = check_logits(logits, dtype, n_tokens, vocab, pitch, targets, temperature);
    if (rc != SR_OK) return rc;
    if (n_tokens > 0 && (row_stats == nullptr || d_logp == nullptr || (d_entropy != nullptr && entropy == nullptr))) return SR_ERR_NULL;
    if (!aligned_4(row_stats, entropy, d_logp, d_entropy)) return SR_ERR_ALIGN;
    rc = check_rows(logits, pitch, d_logits, d_pitch, dtype, n_tokens, vocab);
    if (rc != SR_OK) return rc;
    return launch_token_logprob_backward(LogitsArgs{logits, dtype, n_tokens, vocab, pitch, targets, temperature}, row_stats, entropy, d_logp, d_entropy, d_logits, d_pitch,
                                         static_cast<cudaStream_t>(stream));
}

size_t sr_loss_weights_workspace_bytes(int32_t n_rollouts) {
    return n_rollouts < 0 ? 0 : align_up((size_t)(n_rollouts > 0 ? n_rollouts : 1) * sizeof(int32_t), 256);
}

int sr_loss_weights(const int64_t* row_start, const uint8_t* mask, int32_t n_tokens, const uint8_t* drop_mask, int32_t n_groups, int32_t N, int32_t mode, double scale,
                    float* weight, int64_t* counts, void* workspace, size_t workspace_bytes, void* stream) {
    if (n_groups < 0 || N < 1 || (int64_t)n_groups * N > (1 << 30)) return SR_ERR_BAD_N;
    if (n_tokens < 0) return SR_ERR_BAD_SIZE;
    if (mode != SR_LOSS_SUM && mode != SR_LOSS_TOKEN_MEAN && mode != SR_LOSS_ROLLOUT_MEAN) return SR_ERR_BAD_MODE;
    if (!(fabs(scale) <= kLargest)) return SR_ERR_BAD_VALUE;
    if (n_groups > 0 && (row_start == nullptr || weight == nullptr)) return SR_ERR_NULL;
    if (!aligned(row_start, 8) || !aligned(counts, 8) || !aligned_4(weight)) return SR_ERR_ALIGN;
    if (n_groups > 0 && short_of(workspace, workspace_bytes, sr_loss_weights_workspace_bytes(n_groups * N))) return SR_ERR_WORKSPACE;
    return launch_loss_weights(row_start, mask, n_tokens, drop_mask, n_groups, N, mode, scale, weight, counts, workspace, static_cast<cudaStream_t>(stream));
}

size_t sr_policy_loss_workspace_bytes(int32_t n_tokens) { return n_tokens < 0 ? 0 : kPartialBytes; }

int sr_policy_loss(const float* logp, const float* logp_old, const float* logp_ref, const float* adv, const float* weight, const int64_t* row_start, int32_t n_rollouts,
                   const uint8_t* mask, int32_t n_tokens, double clip_low, double clip_high, double beta, float* loss, float* d_logp, float* stats, void* workspace,
                   size_t workspace_bytes, void* stream) {
    if (n_tokens < 0) return SR_ERR_BAD_SIZE;
    const int rc = check_policy(adv, weight, row_start, n_rollouts, clip_low, clip_high, beta, loss);
    if (rc != SR_OK) return rc;
    if (n_tokens > 0 && logp == nullptr) return SR_ERR_NULL;
    if (!aligned_4(logp, logp_old, logp_ref, d_logp, stats)) return SR_ERR_ALIGN;
    if (short_of(workspace, workspace_bytes, kPartialBytes)) return SR_ERR_WORKSPACE;
    const PolicyBatch b{logp_old, logp_ref, adv, weight, row_start, mask, n_rollouts, clip_low, clip_high, beta, (float)(1.0 - clip_low), (float)(1.0 + clip_high), (float)beta, (float)-clip_low, (float)clip_high};
    return launch_policy_loss(b, logp, n_tokens, loss, d_logp, stats, static_cast<double*>(workspace), static_cast<cudaStream_t>(stream));
}

size_t sr_policy_loss_logits_workspace_bytes(int32_t n_tokens) {
    return n_tokens < 0 ? 0 : kPartialBytes + align_up((size_t)n_tokens * (sizeof(PolicyTerms) + sizeof(int4)) + 4 * sizeof(int32_t), 256);
}

int sr_policy_loss_logits(const void* logits, int32_t dtype, int32_t n_tokens, int32_t vocab, int64_t pitch, const int32_t* targets, const float* logp_old,
                          const float* logp_ref, const float* adv, const float* weight, const int64_t* row_start, int32_t n_rollouts, const uint8_t* mask, double clip_low,
                          double clip_high, double beta, double temperature, float* loss, float* logp, void* d_logits, int64_t d_pitch, float* stats, int32_t* status,
                          void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_logits(logits, dtype, n_tokens, vocab, pitch, targets, temperature);
    if (rc != SR_OK) return rc;
    rc = check_policy(adv, weight, row_start, n_rollouts, clip_low, clip_high, beta, loss);
    if (rc != SR_OK) return rc;
    if (n_tokens > 0 && logp == nullptr) return SR_ERR_NULL;
    if (!aligned_4(logp, logp_old, logp_ref, stats, status)) return SR_ERR_ALIGN;
    rc = check_rows(logits, pitch, d_logits, d_pitch, dtype, n_tokens, vocab);
    if (rc != SR_OK) return rc;
    if (short_of(workspace, workspace_bytes, sr_policy_loss_logits_workspace_bytes(n_tokens))) return SR_ERR_WORKSPACE;
    const PolicyBatch b{logp_old, logp_ref, adv, weight, row_start, mask, n_rollouts, clip_low, clip_high, beta, (float)(1.0 - clip_low), (float)(1.0 + clip_high), (float)beta, (float)-clip_low, (float)clip_high};
    StepScratch ws;
    ws.partial = static_cast<double*>(workspace);
    ws.list = reinterpret_cast<int4*>(static_cast<char*>(workspace) + kPartialBytes);
    ws.row_of = reinterpret_cast<int32_t*>(ws.list);
    ws.terms = reinterpret_cast<PolicyTerms*>(ws.list + n_tokens);
    ws.counters = reinterpret_cast<int32_t*>(ws.terms + n_tokens);
    return launch_policy_loss_logits(LogitsArgs{logits, dtype, n_tokens, vocab, pitch, targets, temperature}, b, loss, logp, d_logits, d_pitch, stats, status, ws,
                                     static_cast<cudaStream_t>(stream));
}

size_t sr_grad_norm_workspace_bytes(int32_t n_tensors) { return n_tensors < 0 ? 0 : grad_norm_workspace_bytes(n_tensors); }

int sr_grad_norm(const void* const* grads, const int64_t* counts, const int32_t* dtypes, int32_t n_tensors, float* norm, void* workspace, size_t workspace_bytes, void* stream) {
    const int rc = check_grads(grads, counts, dtypes, n_tensors);
    if (rc != SR_OK) return rc;
    if (norm == nullptr) return SR_ERR_NULL;
    if (!aligned_4(norm)) return SR_ERR_ALIGN;
    if (short_of(workspace, workspace_bytes, grad_norm_workspace_bytes(n_tensors))) return SR_ERR_WORKSPACE;
    return launch_grad_norm(grads, counts, dtypes, n_tensors, norm, workspace, static_cast<cudaStream_t>(stream));
}

int sr_clip_grads(const void* const* grads, const int64_t* counts, const int32_t* dtypes, int32_t n_tensors, const float* norm, double max_norm, void* const* out,
                  int32_t* status, void* stream) {
    const int rc = check_grads(grads, counts, dtypes, n_tensors);
    if (rc != SR_OK) return rc;
    if (!(max_norm >= 0.0 && max_norm <= kLargest)) return SR_ERR_BAD_VALUE;
    if (norm == nullptr) return SR_ERR_NULL;
    if (!aligned_4(norm, status)) return SR_ERR_ALIGN;
    if (n_tensors == 0) return SR_OK;
    // every buffer that is written must lie apart from all the others
    Range* const written = new (std::nothrow) Range[2 * (size_t)n_tensors + 1];
    if (written == nullptr) return SR_ERR_WORKSPACE;
    Range* const read = written + n_tensors;
    size_t n_written = 0, n_read = 0;
    int bad = SR_OK;
    read[n_read++] = Range{reinterpret_cast<uintptr_t>(norm), reinterpret_cast<uintptr_t>(norm) + 4};
    for (int i = 0; i < n_tensors && bad == SR_OK; ++i) {
        if (counts[i] == 0) continue;
        const size_t bytes = (size_t)counts[i] * dtype_bytes(dtypes[i]);
        const void* to = out ? out[i] : grads[i];
        if (to == nullptr) bad = SR_ERR_NULL;
        else if (!aligned(to, dtype_bytes(dtypes[i]))) bad = SR_ERR_ALIGN;
        const uintptr_t a = reinterpret_cast<uintptr_t>(grads[i]), b = reinterpret_cast<uintptr_t>(to);
        written[n_written++] = Range{b, b + bytes};
        if (a != b) read[n_read++] = Range{a, a + bytes};
    }
    if (bad == SR_OK && overlap(written, n_written, read, n_read)) bad = SR_ERR_OVERLAP;
    delete[] written;
    if (bad != SR_OK) return bad;
    return launch_clip_grads(grads, counts, dtypes, n_tensors, norm, (float)max_norm, out, status, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
