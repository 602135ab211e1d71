// The prefix part of the drafts' attention (prefix_attention.cu), called by draft_attention.cu.
#pragma once
#include "psd_internal.cuh"

namespace psd {

constexpr int kMaxPrefixSplits = 64;   // two per lane of the warp that joins a row
constexpr int kMaxOwnTiles = 16;       // tiles of own keys that a query tile may have in the fused form

struct PrefixPlan {
    int tq;        // tokens per query tile (tq * Hq/Hkv <= 128 rows)
    int n_qt;      // query tiles per sequence and key head
    int units;     // CTAs along the query tiles
    int splits;    // partial results per row
    int dhp;       // floats per partial output row: 64 or 128
    bool fused;    // the kernel takes the own keys too and writes final outputs (splits == 1)
};
int drafts_per_tile(int M, int tq);     // drafts of M tokens that a query tile of tq tokens meets at most
bool fuses_own(int M, int tq, int S);   // whether a query tile's own keys can follow an unsplit prefix in the same kernel
PrefixPlan plan_prefix(int B, int D, int M, int Hq, int Hkv, int Dh, int P, int S);

// plan.fused: final outputs into out and lse (NULL: not wanted).  Otherwise partial results of every row over its sequence's
// prefix: po [splits][rows][dhp] normalised outputs (not written where the split holds no key), pl [splits][rows] base-2
// log-sum-exps (-inf there); row = token * Hq + head.
int launch_prefix_attention(const void* q, const void* k, const void* v, const int32_t* prefix_len, const void* k_own, const void* v_own,
                            const int32_t* own_len, const psd_attention_t& a, const PrefixPlan& p, float* po, float* pl, void* out,
                            float* lse, int32_t* status_dev, cudaStream_t st);

}  // namespace psd
