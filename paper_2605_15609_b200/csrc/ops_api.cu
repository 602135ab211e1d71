// extern "C" entry points of the operators around the step: argument checks, then the launches.  See psd.h.
#include <cmath>
#include "ops_internal.cuh"

namespace psd {
namespace {

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

bool heads_ok(int32_t Hq, int32_t Hkv, int32_t Dh) {
    return Hq >= 1 && Hkv >= 1 && Hq % Hkv == 0 && Hq / Hkv <= 128 && Dh >= 8 && Dh <= 128 && Dh % 8 == 0;
}
// Lengths that kernels walk in steps of thousands with 32-bit positions: a step past the end must not overflow.
constexpr int32_t kMostSteps = 1 << 30;

bool strides_ok(const psd_kv_strides_t& s) { return s.outer >= 0 && s.token > 0 && s.head >= 0; }
bool strides_aligned(const psd_kv_strides_t& s) { return s.outer % 8 == 0 && s.token % 8 == 0 && s.head % 8 == 0; }
// what a tensor map takes: strides below 2^40 bytes
bool strides_small(const psd_kv_strides_t& s) {
    const int64_t top = (int64_t)1 << 38;
    return s.outer < top && s.token < top && s.head < top;
}

}  // namespace

// Rows (tokens times heads) and head-blocks of the grids are indexed with 32 bits; everything that is
// multiplied by a stride is computed in 64.
bool attention_sizes_ok(int32_t B, int32_t D, int32_t M, int32_t Hq, int32_t Hkv, int32_t Dh, int32_t P, int32_t S) {
    if (B < 1 || D < 1 || M < 1 || P < 0 || S < 0 || !heads_ok(Hq, Hkv, Dh)) return false;
    if ((int64_t)B * D > INT32_MAX || (int64_t)B * D * M > INT32_MAX) return false;
    return (int64_t)B * D * M * Hq <= INT32_MAX / 2 && P <= INT32_MAX - 1024 && S <= INT32_MAX - 1024;
}
int check_attention(const psd_attention_t& a, bool with_out) {
    if (!attention_sizes_ok(a.B, a.D, a.M, a.Hq, a.Hkv, a.Dh, a.P, a.S)) return PSD_ERR_SHAPE;
    if (!(a.scale > 0.f) || !std::isfinite(a.scale)) return PSD_ERR_SHAPE;
    if ((a.dtype != PSD_BF16 && a.dtype != PSD_FP16) || a.reserved != 0) return PSD_ERR_UNSUPPORTED;
    if (a.q_token <= 0 || a.q_head <= 0 || !strides_ok(a.kp) || !strides_small(a.kp)) return PSD_ERR_SHAPE;
    if (a.q_token >= ((int64_t)1 << 38) || a.q_head >= ((int64_t)1 << 38)) return PSD_ERR_SHAPE;
    if (a.q_token % 8 || a.q_head % 8 || !strides_aligned(a.kp)) return PSD_ERR_ALIGN;
    if (with_out) {
        if (a.causal != 0 && a.causal != 1) return PSD_ERR_SHAPE;
        if (a.out_token <= 0 || a.out_head <= 0 || !strides_ok(a.vp) || !strides_ok(a.ko) || !strides_ok(a.vo) ||
            !strides_small(a.vp) || !strides_small(a.ko) || !strides_small(a.vo))
            return PSD_ERR_SHAPE;
        if (a.out_token % 8 || a.out_head % 8 || !strides_aligned(a.vp) || !strides_aligned(a.ko) || !strides_aligned(a.vo))
            return PSD_ERR_ALIGN;
    }
    return PSD_OK;
}

}  // namespace psd

using namespace psd;

extern "C" {

size_t psd_attention_workspace_bytes(int32_t B, int32_t D, int32_t M, int32_t Hq, int32_t Hkv, int32_t Dh, int32_t P,
                                     int32_t S) {
    if (!attention_sizes_ok(B, D, M, Hq, Hkv, Dh, P, S)) return 0;
    return draft_attention_workspace(B, D, M, Hq, Hkv, Dh, P, S);
}

const char* psd_attention_kernel_names(int32_t B, int32_t D, int32_t M, int32_t Hq, int32_t Hkv, int32_t Dh, int32_t P, int32_t S,
                                       int32_t* splits) {
    if (!attention_sizes_ok(B, D, M, Hq, Hkv, Dh, P, S)) return nullptr;
    return draft_attention_kernels(B, D, M, Hq, Hkv, Dh, P, S, splits);
}

int psd_draft_attention(const void* q, const void* k_prefix, const void* v_prefix, const int32_t* prefix_len,
                        const void* k_own, const void* v_own, const int32_t* own_len, const psd_attention_t* a,
                        void* out, float* lse, void* workspace, size_t workspace_bytes, int32_t* status_dev,
                        void* cuda_stream) {
    if (!q || !a || !out || !workspace) return PSD_ERR_NULL;
    if (const int e = check_attention(*a, true)) return e;
    if ((a->P > 0 && (!k_prefix || !v_prefix)) || (a->S > 0 && (!k_own || !v_own))) return PSD_ERR_NULL;
    if (!aligned(q, 16) || !aligned(k_prefix, 16) || !aligned(v_prefix, 16) || !aligned(k_own, 16) || !aligned(v_own, 16) ||
        !aligned(out, 16) || !aligned(workspace, 256) || !aligned(prefix_len, 4) || !aligned(own_len, 4) ||
        !aligned(lse, 4) || !aligned(status_dev, 4))
        return PSD_ERR_ALIGN;
    if (workspace_bytes < draft_attention_needs(a->B, a->D, a->M, a->Hq, a->Hkv, a->Dh, a->P, a->S))
        return PSD_ERR_WORKSPACE;
    return launch_draft_attention(q, k_prefix, v_prefix, prefix_len, k_own, v_own, own_len, *a, out, lse, workspace,
                                  status_dev, reinterpret_cast<cudaStream_t>(cuda_stream));
}

size_t psd_weights_workspace_bytes(int32_t B, int32_t D, int32_t M, int32_t Hq, int32_t Hkv, int32_t Dh, int32_t P) {
    if (!attention_sizes_ok(B, D, M, Hq, Hkv, Dh, P, 0) || P < 1) return 0;
    return prefix_weights_workspace(B, D, M, Hq, Hkv, P);
}

int psd_prefix_weights(const void* q, const void* k_prefix, const int32_t* prefix_len, const float* lse,
                       const psd_attention_t* a, float beta, const float* acc_in, float* acc_out, void* workspace,
                       size_t workspace_bytes, int32_t* status_dev, void* cuda_stream) {
    if (!q || !k_prefix || !lse || !a || !acc_out || !workspace) return PSD_ERR_NULL;
    if (const int e = check_attention(*a, false)) return e;
    if (a->P < 1 || !std::isfinite(beta)) return PSD_ERR_SHAPE;
    if (!aligned(q, 16) || !aligned(k_prefix, 16) || !aligned(workspace, 256) || !aligned(prefix_len, 4) ||
        !aligned(lse, 4) || !aligned(acc_in, 4) || !aligned(acc_out, 4) || !aligned(status_dev, 4))
        return PSD_ERR_ALIGN;
    if (workspace_bytes < prefix_weights_needs(a->B, a->D, a->M, a->Hq, a->Hkv, a->P)) return PSD_ERR_WORKSPACE;
    return launch_prefix_weights(q, k_prefix, prefix_len, lse, *a, beta, acc_in, acc_out, workspace, status_dev,
                                 reinterpret_cast<cudaStream_t>(cuda_stream));
}

int psd_prefix_evict(const float* scores, const void* k, const void* v, const int32_t* prefix_len, const psd_evict_t* e,
                     void* k_out, void* v_out, int32_t* index, float* scores_out, int32_t* len_out, void* cuda_stream) {
    if (!scores || !k || !v || !e || !k_out || !v_out || !index) return PSD_ERR_NULL;
    if (e->B < 1 || !heads_ok(e->Hkv, e->Hkv, e->Dh) || e->P < 1 || e->P > kMostSteps || e->keep < 1 || e->keep > kMostSteps ||
        e->n_sink < 0 || e->n_recent < 0 || (int64_t)e->n_sink + e->n_recent > e->keep ||
        (int64_t)e->B * e->Hkv > INT32_MAX / 2)
        return PSD_ERR_SHAPE;
    if (e->dtype != PSD_BF16 && e->dtype != PSD_FP16) return PSD_ERR_UNSUPPORTED;
    // a destination that shares one slot among several keys would be written by all of them
    const bool out_ok = (e->k_out.outer > 0 || e->B == 1) && (e->v_out.outer > 0 || e->B == 1) &&
                        (e->k_out.head > 0 || e->Hkv == 1) && (e->v_out.head > 0 || e->Hkv == 1);
    if (!strides_ok(e->k) || !strides_ok(e->v) || !strides_ok(e->k_out) || !strides_ok(e->v_out) || !out_ok)
        return PSD_ERR_SHAPE;
    if (!strides_aligned(e->k) || !strides_aligned(e->v) || !strides_aligned(e->k_out) || !strides_aligned(e->v_out) ||
        !aligned(k, 16) || !aligned(v, 16) || !aligned(k_out, 16) || !aligned(v_out, 16) || !aligned(scores, 4) ||
        !aligned(prefix_len, 4) || !aligned(index, 4) || !aligned(scores_out, 4) || !aligned(len_out, 4))
        return PSD_ERR_ALIGN;
    return launch_prefix_evict(scores, k, v, prefix_len, *e, k_out, v_out, index, scores_out, len_out,
                               reinterpret_cast<cudaStream_t>(cuda_stream));
}

size_t psd_logits_workspace_bytes(int32_t n_rows, int32_t V) {
    if (n_rows < 1 || V < 1 || n_rows > kMostSteps || V > kMostSteps) return 0;
    return confidence_logits_workspace(n_rows, V);
}

int psd_confidence_logits(const void* logits, int32_t dtype, int64_t row_stride, int32_t B, int32_t D, int32_t M, int32_t V,
                          const psd_logits_edit_t* edit, int32_t* out_token, float* out_conf, float* out_lse,
                          void* workspace, size_t workspace_bytes, int32_t* status_dev, void* cuda_stream) {
    if (!logits || !out_token || !out_conf || !workspace) return PSD_ERR_NULL;
    if (B < 1 || D < 1 || M < 1 || V < 1 || V > kMostSteps || row_stride < V) return PSD_ERR_SHAPE;
    if ((int64_t)B * D > kMostSteps || (int64_t)B * D * M > kMostSteps) return PSD_ERR_SHAPE;
    const int64_t n_rows = (int64_t)B * D * M;
    if (dtype != PSD_BF16 && dtype != PSD_FP16 && dtype != PSD_FP32) return PSD_ERR_UNSUPPORTED;
    psd_logits_edit_t e = {};
    e.repetition = 1.f;
    e.bias_rows = e.allow_rows = 1;
    if (edit) {
        e = *edit;
        if (e.reserved != 0) return PSD_ERR_UNSUPPORTED;
        if (!(e.repetition > 0.f) || !std::isfinite(e.repetition) || !std::isfinite(e.presence) || !std::isfinite(e.frequency))
            return PSD_ERR_SHAPE;
        if (e.history_cap < 0 || e.history_cap > kMostSteps || (e.bias && (e.bias_rows < 1 || n_rows % e.bias_rows)) ||
            (e.allow && (e.allow_rows < 1 || n_rows % e.allow_rows)))
            return PSD_ERR_SHAPE;
        if ((e.draft_tokens == nullptr) != (e.draft_mask == nullptr) || (e.history_cap > 0 && !e.history && e.history_len))
            return PSD_ERR_NULL;
        if (!e.bias) e.bias_rows = 1;
        if (!e.allow) e.allow_rows = 1;
    }
    if (!aligned(logits, dtype == PSD_FP32 ? 4 : 2) || !aligned(workspace, 256) || !aligned(out_token, 4) ||
        !aligned(out_conf, 4) || !aligned(out_lse, 4) || !aligned(status_dev, 4) || !aligned(e.history, 4) ||
        !aligned(e.history_len, 4) || !aligned(e.draft_tokens, 4) || !aligned(e.draft_mask, 4) || !aligned(e.bias, 4) ||
        !aligned(e.allow, 4))
        return PSD_ERR_ALIGN;
    if (workspace_bytes < confidence_logits_needs(n_rows, M, V, e.bias ? e.bias_rows : 0)) return PSD_ERR_WORKSPACE;
    return launch_confidence_logits(logits, dtype, row_stride, B, D, M, V, e, out_token, out_conf, out_lse, workspace,
                                    status_dev, reinterpret_cast<cudaStream_t>(cuda_stream));
}

}  // extern "C"
