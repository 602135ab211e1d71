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
// the own keys, joined with `splits` partial results over the prefix (po, pl as launch_prefix_attention leaves them; splits <= 64)
int launch_own_and_join(const void* q, const void* k_own, const void* v_own, const int32_t* own_len, const psd_attention_t& a,
                        const float* po, const float* pl, int splits, void* out, float* lse, cudaStream_t st);
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

// argument checks that the entry points of these operators share (ops_api.cu)
bool attention_sizes_ok(int32_t B, int32_t D, int32_t M, int32_t Hq, int32_t Hkv, int32_t Dh, int32_t P, int32_t S);
int check_attention(const psd_attention_t& a, bool with_out);

// quantize.cu
int launch_quantize_rows(const void* x, int dtype, int64_t row_stride, int64_t n_rows, int H, int8_t* codes, int64_t code_stride,
                         float* scale, cudaStream_t st);
int launch_prefix_quantize(const void* k, const void* v, const int32_t* begin, const int32_t* end, const psd_quantize_t& q,
                           int8_t* k_codes, int8_t* v_codes, float* k_scale, float* v_scale, cudaStream_t st);

// rotate.cu
int launch_rotate(const void* q, const void* k, const void* v, const int32_t* position, const double* frequency, const void* q_norm,
                  const void* k_norm, const int32_t* slot, const psd_rotate_t& a, void* q_out, void* k_out, void* v_out, cudaStream_t st);

// confidence_q8.cu (x: memory for n_rows rounded up to 128 rows)
int launch_confidence_q8(const int8_t* x, const float* x_scale, const int8_t* w, const float* w_scale, int n_rows, int H, int V,
                         Partials part, int32_t* status_dev, cudaStream_t st, SplitPlan* plan);
int launch_join_triples(Partials part, const SplitPlan& plan, int n_rows, int32_t* out_token, float* out_conf, float* out_lse, int32_t* status_dev,
                        cudaStream_t st);

}  // namespace psd
