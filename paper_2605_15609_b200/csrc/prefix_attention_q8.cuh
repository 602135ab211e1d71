// The prefix part of the drafts' attention over an 8-bit cache, called by ops_q8_api.cu.
#pragma once
#include "ops_internal.cuh"

namespace psd {

struct PrefixQ8 {
    const int8_t *k, *v;             // codes
    const float *k_scale, *v_scale;  // [B, Hkv, ceil(P / block)]
    int block;                       // tokens per scale: 16, 32, 64 or 128
};

struct PrefixQ8Plan {
    int row_blocks;   // 16-row blocks of a warp: 1 or 2
    int units;        // CTAs along the rows of a key head
    int splits;       // partial results per row
    int dhp;          // floats per partial output row: 64 or 128
};
PrefixQ8Plan plan_prefix_q8(int B, int D, int M, int Hq, int Hkv, int Dh, int P);

// Partial results of every row over its sequence's prefix, as launch_prefix_attention leaves them: po [splits][rows][dhp], pl
// [splits][rows].
int launch_prefix_attention_q8(const void* q, const PrefixQ8& c, const int32_t* prefix_len, const psd_attention_t& a, const PrefixQ8Plan& p,
                               float* po, float* pl, int32_t* status_dev, cudaStream_t st);

}  // namespace psd
