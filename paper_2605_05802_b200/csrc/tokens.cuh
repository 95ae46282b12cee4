// The operators on token ids: what their C entry points hand to the kernels.
#pragma once

#include "logits.cuh"
#include "sr_tokens.h"

namespace sr {

// adjust.cu.  Forward: `in` are the logits.  Backward: `in` is the gradient of `out`, `logits` what the forward call had.
struct AdjustArgs {
    const void *in, *logits;
    void* out;
    int64_t pitch, logits_pitch, out_pitch;
    int32_t dtype, n_rows, vocab;
    const int32_t* history;              // of the next five all or none: what is NULL here is not used
    int64_t n_history;
    const int64_t* history_start;
    const int32_t *history_len, *prompt_len;
    const float *repetition, *presence, *frequency;
    const int32_t* bias_token;
    const float* bias_value;
    int64_t n_bias;
    const int64_t* bias_start;
    const int32_t* bias_len;
    const uint32_t* allowed;
    int32_t n_masks;
    int64_t mask_pitch;
    const int32_t* mask_row;
    int32_t* status;
};
int launch_adjust(const AdjustArgs& a, bool backward, cudaStream_t s);

// embed.cu
struct EmbedArgs {
    const void* table;
    int32_t table_dtype, vocab, width;
    int64_t table_pitch;
    const int32_t* tokens;
    int32_t n_tokens;
    float scale;
    void* out;
    int32_t dtype;
    int64_t pitch;
    int32_t* status;
};
int launch_embed(const EmbedArgs& a, cudaStream_t s);
struct EmbedGradArgs {
    const void* d_out;
    int32_t dtype, n_tokens, width;
    int64_t pitch;
    const int32_t* tokens;
    int32_t vocab;
    float scale;
    void* d_table;
    int32_t table_dtype;
    int64_t table_pitch;
    bool accumulate;
    int32_t* status;
};
size_t embed_grad_workspace_bytes(int32_t n_tokens, int32_t vocab, int32_t width);
int launch_embed_grad(const EmbedGradArgs& a, void* ws, cudaStream_t s);

}  // namespace sr
