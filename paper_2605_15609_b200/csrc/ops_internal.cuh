// Internal declarations of the operators around the step (attention of the drafts, upkeep of the prefix's
// cache, confidences from logits).
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include "psd_internal.cuh"

namespace psd {

// draft_attention.cu
int launch_draft_attention(const void* q, const void* k_prefix, const void* v_prefix, const int32_t* prefix_len,
                           const void* k_own, const void* v_own, const int32_t* own_len, const psd_attention_t& a,
                           void* out, float* lse, void* workspace, int32_t* status_dev, cudaStream_t st);
const char* draft_attention_kernels(int B, int D, int M, int Hq, int Hkv, int Dh, int P, int S, int32_t* splits);
// bytes that a call writes, and what the public size function answers: that of this and of all smaller batches
size_t draft_attention_needs(int B, int D, int M, int Hq, int Hkv, int Dh, int P, int S);
size_t draft_attention_workspace(int B, int D, int M, int Hq, int Hkv, int Dh, int P, int S);

// prefix_weights.cu
int launch_prefix_weights(const void* q, const void* k_prefix, const int32_t* prefix_len, const float* lse,
                          const psd_attention_t& a, float beta, const float* acc_in, float* acc_out, void* workspace,
                          int32_t* status_dev, cudaStream_t st);
size_t prefix_weights_needs(int B, int D, int M, int Hq, int Hkv, int P);
size_t prefix_weights_workspace(int B, int D, int M, int Hq, int Hkv, int P);

// prefix_evict.cu
int launch_prefix_evict(const float* scores, const void* k, const void* v, const int32_t* prefix_len,
                        const psd_evict_t& e, void* k_out, void* v_out, int32_t* index, float* scores_out,
                        int32_t* len_out, cudaStream_t st);

// confidence_logits.cu
int launch_confidence_logits(const void* logits, int dtype, int64_t row_stride, int B, int D, int M, int V,
                             const psd_logits_edit_t& e, int32_t* out_token, float* out_conf, float* out_lse,
                             void* workspace, int32_t* status_dev, cudaStream_t st);
size_t confidence_logits_needs(int64_t n_rows, int M, int V, int bias_rows);      // bias_rows 0: no bias
size_t confidence_logits_workspace(int64_t n_rows, int V);

}  // namespace psd
