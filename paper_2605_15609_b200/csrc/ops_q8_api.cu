// extern "C" entry points of the 8-bit step and the rotation: argument checks, then the launches.  See psd.h.
#include <cmath>
#include "ops_internal.cuh"
#include "prefix_attention_q8.cuh"

namespace psd {
namespace {

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
inline size_t round_up(size_t x) { return (x + 255) / 256 * 256; }
bool head_ok(int32_t Dh) { return Dh >= 8 && Dh <= 128 && Dh % 8 == 0; }
bool block_ok(int32_t n) { return n == 16 || n == 32 || n == 64 || n == 128; }
constexpr int32_t kMostSteps = 1 << 30;
bool eights(int64_t a, int64_t b, int64_t c) { return a % 8 == 0 && b % 8 == 0 && c % 8 == 0; }
// codes of the hidden rows: whole tiles of 128 rows (launch_confidence_q8)
size_t codes_bytes(int32_t n_rows, int32_t H) { return round_up((size_t)((n_rows + 127) / 128) * 128 * H); }
bool head_shape_ok(int32_t n_rows, int32_t H, int32_t V) {
    // sums of products of codes stay below 2^31: 127 * 127 * 131072
    return n_rows >= 1 && n_rows <= kMostSteps && H >= 64 && H % 64 == 0 && H <= 131072 && V >= 1 && V < 2147483647 - 256;
}

}  // namespace
}  // namespace psd

using namespace psd;

extern "C" {

int psd_rope_frequencies(int32_t rotary, double base, int32_t kind, double factor, double original, double low, double high,
                         double* frequency, float* gain) {
    if (!frequency) return PSD_ERR_NULL;
    if (rotary < 2 || rotary > 128 || rotary % 2 || !(base > 1.0) || !std::isfinite(base) || !(factor >= 1.0) || !std::isfinite(factor))
        return PSD_ERR_SHAPE;
    if (kind < PSD_ROPE_PLAIN || kind > PSD_ROPE_BY_PARTS) return PSD_ERR_UNSUPPORTED;
    if (kind == PSD_ROPE_STRETCHED && rotary == 2) return PSD_ERR_SHAPE;
    if (kind == PSD_ROPE_BY_PARTS && (!(original >= 1.0) || !std::isfinite(original) || !(low >= 0.0) || !(high > low) || !std::isfinite(high)))
        return PSD_ERR_SHAPE;
    if (kind == PSD_ROPE_STRETCHED) base *= std::pow(factor, (double)rotary / (rotary - 2));
    for (int j = 0; j < rotary / 2; ++j) {
        double f = std::pow(base, -2.0 * j / rotary);
        if (kind == PSD_ROPE_LINEAR) f /= factor;
        if (kind == PSD_ROPE_BY_PARTS) {
            double w = (original * f / 6.283185307179586477 - low) / (high - low);
            w = w < 0.0 ? 0.0 : w > 1.0 ? 1.0 : w;
            f = w * f + (1.0 - w) * f / factor;
        }
        frequency[j] = f;
    }
    if (gain) *gain = kind == PSD_ROPE_BY_PARTS ? (float)(0.1 * std::log(factor) + 1.0) : 1.0f;
    return PSD_OK;
}

int psd_rotate_qk(const void* q, const void* k, const void* v, const int32_t* position, const double* frequency,
                  const void* q_norm, const void* k_norm, const int32_t* slot, const psd_rotate_t* r, void* q_out, void* k_out,
                  void* v_out, void* cuda_stream) {
    if (!r) return PSD_ERR_NULL;
    if (r->n_tokens < 1 || r->n_tokens > kMostSteps || r->Hq < 0 || r->Hkv < 0 || r->Hq + (int64_t)r->Hkv < 1 ||
        r->Hq > 16384 || r->Hkv > 16384 || !head_ok(r->Dh) || r->rotary < 0 || r->rotary > r->Dh || r->rotary % 2)
        return PSD_ERR_SHAPE;
    if ((r->interleaved != 0 && r->interleaved != 1) || !(r->eps > 0.f) || !std::isfinite(r->eps) || !(r->gain > 0.f) ||
        !std::isfinite(r->gain) || (slot && r->n_slots < 0))
        return PSD_ERR_SHAPE;
    if (r->dtype != PSD_BF16 && r->dtype != PSD_FP16) return PSD_ERR_UNSUPPORTED;
    if ((r->Hq > 0 && (!q || !q_out)) || (r->Hkv > 0 && (!k || !k_out)) || (v && (!v_out || r->Hkv == 0)) ||
        (r->rotary > 0 && (!position || !frequency)))
        return PSD_ERR_NULL;
    const bool hq = r->Hq > 0, hk = r->Hkv > 0;
    if ((hq && (r->q_token <= 0 || r->q_head <= 0 || r->q_out_token <= 0 || r->q_out_head <= 0)) ||
        (hk && (r->k_token <= 0 || r->k_head <= 0 || r->k_out_token <= 0 || r->k_out_head <= 0)) ||
        (v && (r->v_token <= 0 || r->v_head <= 0 || r->v_out_token <= 0 || r->v_out_head <= 0)))
        return PSD_ERR_SHAPE;
    if ((hq && (!eights(r->q_token, r->q_head, r->q_out_token) || r->q_out_head % 8)) ||
        (hk && (!eights(r->k_token, r->k_head, r->k_out_token) || r->k_out_head % 8)) ||
        (v && (!eights(r->v_token, r->v_head, r->v_out_token) || r->v_out_head % 8)))
        return PSD_ERR_ALIGN;
    if ((hq && (!aligned(q, 16) || !aligned(q_out, 16))) || (hk && (!aligned(k, 16) || !aligned(k_out, 16))) ||
        (v && (!aligned(v, 16) || !aligned(v_out, 16))) || !aligned(q_norm, 16) || !aligned(k_norm, 16) || !aligned(position, 4) ||
        !aligned(slot, 4) || !aligned(frequency, 8))
        return PSD_ERR_ALIGN;
    return launch_rotate(q, k, v, position, frequency, q_norm, k_norm, slot, *r, q_out, k_out, v_out,
                         reinterpret_cast<cudaStream_t>(cuda_stream));
}

int psd_quantize_rows(const void* x, int32_t dtype, int64_t row_stride, int64_t n_rows, int32_t H, int8_t* codes,
                      int64_t code_stride, float* scale, void* cuda_stream) {
    if (!x || !codes || !scale) return PSD_ERR_NULL;
    if (n_rows < 1 || n_rows > kMostSteps || H < 8 || H % 8 || H > kMostSteps || row_stride < H || code_stride < H) return PSD_ERR_SHAPE;
    if (dtype != PSD_BF16 && dtype != PSD_FP16) return PSD_ERR_UNSUPPORTED;
    if (row_stride % 8 || code_stride % 8 || !aligned(x, 16) || !aligned(codes, 8) || !aligned(scale, 4)) return PSD_ERR_ALIGN;
    return launch_quantize_rows(x, dtype, row_stride, n_rows, H, codes, code_stride, scale, reinterpret_cast<cudaStream_t>(cuda_stream));
}

int psd_prefix_quantize(const void* k, const void* v, const int32_t* begin, const int32_t* end, const psd_quantize_t* q,
                        int8_t* k_codes, int8_t* v_codes, float* k_scale, float* v_scale, void* cuda_stream) {
    if (!k || !v || !q || !k_codes || !v_codes || !k_scale || !v_scale) return PSD_ERR_NULL;
    if (q->B < 1 || q->Hkv < 1 || !head_ok(q->Dh) || q->P < 1 || q->P > kMostSteps || !block_ok(q->block) || q->span < 0 ||
        (int64_t)q->B * q->Hkv > INT32_MAX / 2)
        return PSD_ERR_SHAPE;
    if ((q->dtype != PSD_BF16 && q->dtype != PSD_FP16) || q->reserved != 0) return PSD_ERR_UNSUPPORTED;
    for (const psd_kv_strides_t* s : {&q->k, &q->v, &q->k_codes, &q->v_codes})
        if (s->outer < 0 || s->token <= 0 || s->head < 0) return PSD_ERR_SHAPE;
    // a destination that shares one slot among several keys would be written by all of them
    for (const psd_kv_strides_t* s : {&q->k_codes, &q->v_codes})
        if ((s->outer == 0 && q->B > 1) || (s->head == 0 && q->Hkv > 1)) return PSD_ERR_SHAPE;
    for (const psd_kv_strides_t* s : {&q->k, &q->v, &q->k_codes, &q->v_codes})
        if (!eights(s->outer, s->token, s->head)) return PSD_ERR_ALIGN;
    if (!aligned(k, 16) || !aligned(v, 16) || !aligned(k_codes, 8) || !aligned(v_codes, 8) || !aligned(k_scale, 4) ||
        !aligned(v_scale, 4) || !aligned(begin, 4) || !aligned(end, 4))
        return PSD_ERR_ALIGN;
    return launch_prefix_quantize(k, v, begin, end, *q, k_codes, v_codes, k_scale, v_scale, reinterpret_cast<cudaStream_t>(cuda_stream));
}

size_t psd_attention_q8_workspace_bytes(int32_t B, int32_t D, int32_t M, int32_t Hq, int32_t Hkv, int32_t Dh, int32_t P, int32_t S) {
    if (!attention_sizes_ok(B, D, M, Hq, Hkv, Dh, P, S) || Dh % 16) return 0;
    return P == 0 ? 256 : prefix_q8_workspace(B, D, M, Hq, Hkv, Dh, P);
}

const char* psd_attention_q8_kernel_names(int32_t B, int32_t D, int32_t M, int32_t Hq, int32_t Hkv, int32_t Dh, int32_t P, int32_t S,
                                          int32_t* splits) {
    if (!attention_sizes_ok(B, D, M, Hq, Hkv, Dh, P, S) || Dh % 16) return nullptr;
    if (P == 0) return draft_attention_kernels(B, D, M, Hq, Hkv, Dh, P, S, splits);
    const PrefixQ8Plan p = plan_prefix_q8(B, D, M, Hq, Hkv, Dh, P, S);
    if (splits) *splits = p.one ? 0 : p.splits;
    if (p.one) return "draft_attention_kernel";
    return !p.tiles ? "prefix_rows_q8_kernel+draft_attention_kernel"
                    : p.final ? "prefix_tiles_q8_kernel" : "prefix_tiles_q8_kernel+draft_attention_kernel";
}

int psd_draft_attention_q8(const void* q, const int8_t* k_codes, const int8_t* v_codes, const float* k_scale,
                           const float* v_scale, int32_t block, const int32_t* prefix_len, const void* k_own,
                           const void* v_own, const int32_t* own_len, const psd_attention_t* a, void* out, float* lse,
                           void* workspace, size_t workspace_bytes, int32_t* status_dev, void* cuda_stream) {
    if (!q || !a || !out || !workspace) return PSD_ERR_NULL;
    if (const int e = check_attention(*a, true)) return e;
    if (a->Dh % 16 || !block_ok(block)) return PSD_ERR_SHAPE;
    if ((a->P > 0 && (!k_codes || !v_codes || !k_scale || !v_scale)) || (a->S > 0 && (!k_own || !v_own))) return PSD_ERR_NULL;
    for (const psd_kv_strides_t* s : {&a->kp, &a->vp})
        if (s->outer % 16 || s->token % 16 || s->head % 16) return PSD_ERR_ALIGN;
    if (!aligned(q, 16) || !aligned(k_codes, 16) || !aligned(v_codes, 16) || !aligned(k_scale, 4) || !aligned(v_scale, 4) ||
        !aligned(k_own, 16) || !aligned(v_own, 16) || !aligned(out, 16) || !aligned(workspace, 256) || !aligned(prefix_len, 4) ||
        !aligned(own_len, 4) || !aligned(lse, 4) || !aligned(status_dev, 4))
        return PSD_ERR_ALIGN;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
    if (a->P == 0) return launch_draft_attention(q, nullptr, nullptr, nullptr, k_own, v_own, own_len, *a, out, lse, workspace, status_dev, st);
    const PrefixQ8Plan plan = plan_prefix_q8(a->B, a->D, a->M, a->Hq, a->Hkv, a->Dh, a->P, a->S);
    const int64_t rows = (int64_t)a->B * a->D * a->M * a->Hq;
    if (workspace_bytes < prefix_q8_needs(a->B, a->D, a->M, a->Hq, a->Hkv, a->Dh, a->P, a->S)) return PSD_ERR_WORKSPACE;
    float* po = reinterpret_cast<float*>(workspace);
    float* pl = po + rows * plan.splits * plan.dhp;
    const PrefixQ8 c = {k_codes, v_codes, k_scale, v_scale, block};
    const int e = launch_prefix_attention_q8(q, c, prefix_len, k_own, v_own, own_len, *a, plan, po, pl, out, lse, status_dev, st);
    if (e != PSD_OK || plan.final) return e;
    return launch_own_and_join(q, k_own, v_own, own_len, *a, po, pl, plan.splits, out, lse, st);
}

size_t psd_confidence_q8_workspace_bytes(int32_t n_rows, int32_t H, int32_t V) {
    if (!head_shape_ok(n_rows, H, V)) return 0;
    return partial_bytes(n_rows, V) + codes_bytes(n_rows, H) + round_up((size_t)n_rows * 4);
}

int psd_confidence_q8(const void* hidden, int32_t dtype, const int8_t* w_codes, const float* w_scale, int32_t n_rows, int32_t H,
                      int32_t V, int32_t* out_token, float* out_conf, float* out_lse, void* workspace, size_t workspace_bytes,
                      int32_t* status_dev, void* cuda_stream) {
    if (!hidden || !w_codes || !w_scale || !out_token || !out_conf || !workspace) return PSD_ERR_NULL;
    if (!head_shape_ok(n_rows, H, V)) return PSD_ERR_SHAPE;
    if (dtype != PSD_BF16 && dtype != PSD_FP16) return PSD_ERR_UNSUPPORTED;
    if (!aligned(hidden, 16) || !aligned(w_codes, 16) || !aligned(w_scale, 4) || !aligned(workspace, 256) || !aligned(out_token, 4) ||
        !aligned(out_conf, 4) || !aligned(out_lse, 4) || !aligned(status_dev, 4))
        return PSD_ERR_ALIGN;
    if (workspace_bytes < psd_confidence_q8_workspace_bytes(n_rows, H, V)) return PSD_ERR_WORKSPACE;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
    const Partials part = carve_partials(workspace, n_rows, V);
    int8_t* codes = reinterpret_cast<int8_t*>(workspace) + partial_bytes(n_rows, V);
    float* scale = reinterpret_cast<float*>(codes + codes_bytes(n_rows, H));
    if (const int e = launch_quantize_rows(hidden, dtype, H, n_rows, H, codes, H, scale, st)) return e;
    SplitPlan plan;
    if (const int e = launch_confidence_q8(codes, scale, w_codes, w_scale, n_rows, H, V, part, status_dev, st, &plan)) return e;
    return launch_join_triples(part, plan, n_rows, out_token, out_conf, out_lse, status_dev, st);
}

}  // extern "C"
