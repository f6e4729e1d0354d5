// Attention under masks (mslt_op_attention_masked): what its kernels share.
#pragma once
#include "common.cuh"
#include "../../include/mslt.h"

namespace mslt {

// The mask and the scores' form, as the kernels read them.
struct AttnMask {
  int S, causal;
  float scale, cap;
  const float* slopes;
  const int32_t *prefix, *docs, *lens;
};

// fp32 (attn_masked_f32.cu) and bf16 (attn_masked_tc.cu); err: 256 bytes
int attn_masked_f32_fwd(const mslt_attention_desc& d, cudaStream_t st, char* err);
int attn_masked_f32_bwd(const mslt_attention_desc& d, float* delta, cudaStream_t st, char* err);
int attn_masked_tc_fwd(const mslt_attention_desc& d, int* status, cudaStream_t st, char* err);
int attn_masked_tc_bwd(const mslt_attention_desc& d, float* delta, int* status, cudaStream_t st, char* err);

}  // namespace mslt
