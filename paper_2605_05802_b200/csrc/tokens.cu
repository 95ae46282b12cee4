// extern "C" boundary of the operators on token ids (sr_tokens.h): argument checks and dispatch.
#include <math.h>

#include "checks.cuh"
#include "tokens.cuh"

using namespace sr;

namespace {

// Histories (their arrays are used where a penalty is), masks and the rows that are written.
int check_rules(bool penalties, const int32_t* history, int64_t n_history, const int64_t* history_start, const int32_t* history_len, const uint32_t* allowed, int32_t n_masks,
                int64_t mask_pitch, const int32_t* mask_row, int32_t n_rows, int32_t vocab) {
    if (n_history < 0) return SR_ERR_BAD_SIZE;
    if (allowed != nullptr && (n_masks < 0 || mask_pitch < ((int64_t)vocab + 31) / 32 || mask_pitch > kMaxPitch || (mask_row == nullptr && n_masks < n_rows))) return SR_ERR_BAD_SIZE;
    if (penalties && n_rows > 0 && ((history == nullptr && n_history > 0) || history_start == nullptr || history_len == nullptr)) return SR_ERR_NULL;
    if (!aligned_4(history, history_len, allowed, mask_row) || !aligned(history_start, 8)) return SR_ERR_ALIGN;
    return SR_OK;
}

int check_in(const void* in, int32_t dtype, int32_t n_rows, int32_t vocab, int64_t pitch) {
    if (n_rows < 0 || vocab < 1 || pitch < vocab || pitch > kMaxPitch) return SR_ERR_BAD_SIZE;
    if (dtype_bytes(dtype) == 0) return SR_ERR_BAD_DTYPE;
    if (n_rows > 0 && in == nullptr) return SR_ERR_NULL;
    return aligned(in, dtype_bytes(dtype)) ? SR_OK : SR_ERR_ALIGN;
}

constexpr int32_t kMostWidth = 1 << 24;

// Rows of tokens and of a table: sizes, types, pointers.
int check_table(const void* table, int32_t table_dtype, int32_t vocab, int64_t table_pitch, const int32_t* tokens, int32_t n_tokens, const void* rows, int32_t dtype, int32_t width,
                int64_t pitch, double scale, const int32_t* status) {
    if (n_tokens < 0 || vocab < 1 || width < 1 || width > kMostWidth || pitch < width || pitch > kMaxPitch || table_pitch < width || table_pitch > kMaxPitch) return SR_ERR_BAD_SIZE;
    if (dtype_bytes(dtype) == 0 || dtype_bytes(table_dtype) == 0 || (table_dtype != dtype && table_dtype != SR_DTYPE_F32)) return SR_ERR_BAD_DTYPE;
    if (!(fabs(scale) <= kLargest)) return SR_ERR_BAD_VALUE;
    if (table == nullptr || (n_tokens > 0 && (tokens == nullptr || rows == nullptr))) return SR_ERR_NULL;
    if (!aligned(table, dtype_bytes(table_dtype)) || !aligned(rows, dtype_bytes(dtype)) || !aligned_4(tokens, status)) return SR_ERR_ALIGN;
    if (n_tokens == 0) return SR_OK;
    const uintptr_t a = reinterpret_cast<uintptr_t>(table), b = reinterpret_cast<uintptr_t>(rows);
    const uint64_t a_bytes = ((uint64_t)(vocab - 1) * table_pitch + width) * dtype_bytes(table_dtype), b_bytes = ((uint64_t)(n_tokens - 1) * pitch + width) * dtype_bytes(dtype);
    return a + a_bytes <= b || b + b_bytes <= a ? SR_OK : SR_ERR_OVERLAP;
}

}  // namespace

extern "C" {

int sr_adjust_logits(const void* logits, int32_t dtype, int32_t n_rows, int32_t vocab, int64_t pitch, const int32_t* history, int64_t n_history, const int64_t* history_start,
                     const int32_t* history_len, const int32_t* prompt_len, const float* repetition, const float* presence, const float* frequency, const int32_t* bias_token,
                     const float* bias_value, int64_t n_bias, const int64_t* bias_start, const int32_t* bias_len, const uint32_t* allowed, int32_t n_masks, int64_t mask_pitch,
                     const int32_t* mask_row, void* out, int64_t out_pitch, int32_t* status, void* stream) {
    int rc = check_in(logits, dtype, n_rows, vocab, pitch);
    if (rc != SR_OK) return rc;
    const bool penalties = repetition != nullptr || presence != nullptr || frequency != nullptr;
    rc = check_rules(penalties, history, n_history, history_start, history_len, allowed, n_masks, mask_pitch, mask_row, n_rows, vocab);
    if (rc != SR_OK) return rc;
    if (n_bias < 0) return SR_ERR_BAD_SIZE;
    if (bias_value != nullptr && n_rows > 0 && (bias_token == nullptr || bias_start == nullptr || bias_len == nullptr)) return SR_ERR_NULL;
    if (!aligned_4(prompt_len, repetition, presence, frequency, bias_token, bias_value, bias_len, status) || !aligned(bias_start, 8)) return SR_ERR_ALIGN;
    rc = check_rows(logits, pitch, out, out_pitch, dtype, n_rows, vocab);
    if (rc != SR_OK) return rc;
    AdjustArgs a = {};
    a.in = logits; a.out = out;
    a.pitch = pitch; a.out_pitch = out_pitch;
    a.dtype = dtype; a.n_rows = n_rows; a.vocab = vocab;
    if (penalties) { a.history = history; a.n_history = n_history; a.history_start = history_start; a.history_len = history_len; a.prompt_len = prompt_len; }
    a.repetition = repetition; a.presence = presence; a.frequency = frequency;
    if (bias_value) { a.bias_token = bias_token; a.bias_value = bias_value; a.n_bias = n_bias; a.bias_start = bias_start; a.bias_len = bias_len; }
    if (allowed) { a.allowed = allowed; a.n_masks = n_masks; a.mask_pitch = mask_pitch; a.mask_row = mask_row; }
    a.status = status;
    return launch_adjust(a, false, static_cast<cudaStream_t>(stream));
}

int sr_adjust_logits_backward(const void* d_out, int32_t dtype, int32_t n_rows, int32_t vocab, int64_t d_out_pitch, const void* logits, int64_t pitch, const int32_t* history,
                              int64_t n_history, const int64_t* history_start, const int32_t* history_len, const float* repetition, const uint32_t* allowed, int32_t n_masks,
                              int64_t mask_pitch, const int32_t* mask_row, void* d_logits, int64_t d_pitch, int32_t* status, void* stream) {
    int rc = check_in(d_out, dtype, n_rows, vocab, d_out_pitch);
    if (rc != SR_OK) return rc;
    rc = check_rules(repetition != nullptr, history, n_history, history_start, history_len, allowed, n_masks, mask_pitch, mask_row, n_rows, vocab);
    if (rc != SR_OK) return rc;
    if (!aligned_4(repetition, status)) return SR_ERR_ALIGN;
    if (repetition != nullptr) {
        rc = check_in(logits, dtype, n_rows, vocab, pitch);
        if (rc != SR_OK) return rc;
        rc = check_rows(logits, pitch, d_logits, d_pitch, dtype, n_rows, vocab);
        if (rc != SR_OK) return rc;
    }
    rc = check_rows(d_out, d_out_pitch, d_logits, d_pitch, dtype, n_rows, vocab);
    if (rc != SR_OK) return rc;
    AdjustArgs a = {};
    a.in = d_out; a.out = d_logits;
    a.pitch = d_out_pitch; a.out_pitch = d_pitch;
    a.dtype = dtype; a.n_rows = n_rows; a.vocab = vocab;
    if (repetition) {
        a.logits = logits; a.logits_pitch = pitch;
        a.history = history; a.n_history = n_history; a.history_start = history_start; a.history_len = history_len;
        a.repetition = repetition;
    }
    if (allowed) { a.allowed = allowed; a.n_masks = n_masks; a.mask_pitch = mask_pitch; a.mask_row = mask_row; }
    a.status = status;
    return launch_adjust(a, true, static_cast<cudaStream_t>(stream));
}

int sr_embed_tokens(const void* table, int32_t table_dtype, int32_t vocab, int32_t width, int64_t table_pitch, const int32_t* tokens, int32_t n_tokens, double scale, void* out,
                    int32_t dtype, int64_t pitch, int32_t* status, void* stream) {
    const int rc = check_table(table, table_dtype, vocab, table_pitch, tokens, n_tokens, out, dtype, width, pitch, scale, status);
    if (rc != SR_OK) return rc;
    return launch_embed(EmbedArgs{table, table_dtype, vocab, width, table_pitch, tokens, n_tokens, (float)scale, out, dtype, pitch, status}, static_cast<cudaStream_t>(stream));
}

size_t sr_embed_tokens_backward_workspace_bytes(int32_t n_tokens, int32_t vocab, int32_t width) {
    return n_tokens < 0 || vocab < 1 || width < 1 || width > kMostWidth ? 0 : embed_grad_workspace_bytes(n_tokens, vocab, width);
}

int sr_embed_tokens_backward(const void* d_out, int32_t dtype, int32_t n_tokens, int32_t width, int64_t pitch, const int32_t* tokens, int32_t vocab, double scale, void* d_table,
                             int32_t table_dtype, int64_t table_pitch, int32_t accumulate, int32_t* status, void* workspace, size_t workspace_bytes, void* stream) {
    const int rc = check_table(d_table, table_dtype, vocab, table_pitch, tokens, n_tokens, d_out, dtype, width, pitch, scale, status);
    if (rc != SR_OK) return rc;
    if (short_of(workspace, workspace_bytes, embed_grad_workspace_bytes(n_tokens, vocab, width))) return SR_ERR_WORKSPACE;
    return launch_embed_grad(EmbedGradArgs{d_out, dtype, n_tokens, width, pitch, tokens, vocab, (float)scale, d_table, table_dtype, table_pitch, accumulate != 0, status}, workspace,
                             static_cast<cudaStream_t>(stream));
}

}  // extern "C"
