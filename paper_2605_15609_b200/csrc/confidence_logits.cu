// Token, confidence and log-sum-exp of rows of logits under penalties, biases and grammar masks.
//
// One pass over the logits (the only large operand): a CTA takes a few rows that share one text (a draft) and one
// bias row, and a chunk of the vocabulary; a warp walks a row's columns with a running maximum and sum per lane,
//     m' = max(m, x),  s' = s * 2^((m - m') log2 e) + sum 2^((x - m') log2 e),
// and writes one (max, sum, lowest argmax) triple per row and chunk; a second kernel merges them.
//
// The edits touch few tokens.  The CTA counts the text's tokens of its chunk in shared memory once for all its rows
// and marks every token that has a count or a bias ("special").  The main loop treats special tokens as absent, like
// tokens that the grammar forbids; each lane then takes the special tokens of its words one by one, reads the logit
// again (from L1/L2) and edits it with separately rounded operations.  So the loop that streams the logits has no
// per-token edit in it, whatever the edits are.
//
// Differences are taken before the multiplication by log2 e: a row whose maximum is the type's lowest value would
// overflow a precomputed product, and its rounding would shift every term by the same relative error.
#include "combine.cuh"
#include "ops_internal.cuh"
#include "tc_common.cuh"

namespace psd {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMaxChunk = 16384;      // tokens per CTA: 64 KB of counts
constexpr int kMinWarpCols = 512;     // columns a warp takes at least (sets the number of triples per row)
constexpr int kRowsPerCta = 64;
constexpr float kLog2e = 1.4426950408889634f;

struct Part { float m, s; int32_t a, pad; };

struct LogitsArgs {
    const void* logits;
    int64_t stride;
    int M, V, D;
    int unit_rows, slices, rows_per_cta;   // rows of one node and one bias row; CTAs they are cut into; rows of each
    int chunk, n_chunks, wpr;              // columns per CTA; CTAs along the vocabulary; warps that share a row
    int rows_per_bias, rows_per_allow, words;
    psd_logits_edit_t e;
    Part* part;                            // [rows][n_chunks * wpr]
};

template <typename T> struct Vec;
template <> struct Vec<__nv_bfloat16> {
    static constexpr int E = 8;
    static __device__ __forceinline__ void unpack(const uint4& r, float (&x)[8]) {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ float one(const __nv_bfloat16* p) { return __bfloat162float(*p); }
};
template <> struct Vec<__half> {
    static constexpr int E = 8;
    static __device__ __forceinline__ void unpack(const uint4& r, float (&x)[8]) {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
            x[2 * i] = f.x;
            x[2 * i + 1] = f.y;
        }
    }
    static __device__ __forceinline__ float one(const __half* p) { return __half2float(*p); }
};
template <> struct Vec<float> {
    static constexpr int E = 4;
    static __device__ __forceinline__ void unpack(const uint4& r, float (&x)[4]) {
        x[0] = __uint_as_float(r.x); x[1] = __uint_as_float(r.y); x[2] = __uint_as_float(r.z); x[3] = __uint_as_float(r.w);
    }
    static __device__ __forceinline__ float one(const float* p) { return *p; }
};

// A sum relative to maximum m, moved to maximum M >= m (m = -inf: the sum is 0, or NaN from a NaN among the values).
__device__ __forceinline__ float rescaled(float s, float m, float M) {
    return m == -INFINITY ? s : s * ex2((m - M) * kLog2e);
}

// G values of one lane joined to its running maximum and sum; g names the group for the search of the argmax.
template <int G>
__device__ __forceinline__ void fold_group(const float (&x)[G], int g, float& m, float& s, int& best) {
    float gm = x[0];
#pragma unroll
    for (int j = 1; j < G; ++j) gm = fmaxf(gm, x[j]);
    best = gm > m ? g : best;
    const float mn = fmaxf(m, gm);
    const float base = mn == -INFINITY ? 0.f : mn;
    float t = s * ex2((m == mn ? 0.f : m - base) * kLog2e);     // m = -inf here means s = 0 (or NaN), factor 0 or 1
    float acc[2] = {0.f, 0.f};
#pragma unroll
    for (int j = 0; j < G; ++j) acc[j & 1] += ex2((x[j] - base) * kLog2e);
    s = t + (acc[0] + acc[1]);
    m = mn;
}

// VEC: 16-byte loads, lane l takes E neighbouring columns; otherwise (rows not 16-byte aligned) lane l takes columns
// l, l + 32, .. of a run of 256, one element per load.
template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads) logits_kernel(const LogitsArgs a) {
    constexpr int E = VEC ? Vec<T>::E : 8;     // columns of a lane per step
    constexpr int STEP = 32 * E;               // columns of a warp per step
    extern __shared__ int32_t sh[];
    int32_t* cnt = sh;                                             // [chunk]
    uint32_t* special = reinterpret_cast<uint32_t*>(sh + a.chunk);  // [chunk / 32]
    const int c = blockIdx.x % a.n_chunks;
    const int us = blockIdx.x / a.n_chunks;
    const int slice = us % a.slices;
    const int64_t unit0 = (int64_t)(us / a.slices) * a.unit_rows;      // first row of the unit
    const int64_t row0 = unit0 + (int64_t)slice * a.rows_per_cta;
    const int n_rows = min(a.rows_per_cta, a.unit_rows - slice * a.rows_per_cta);
    const int64_t node = unit0 / a.M;
    const int v0 = c * a.chunk, vw = min(a.chunk, a.V - v0);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const bool counts = a.e.history || a.e.draft_tokens;
    const float* bias = a.e.bias ? a.e.bias + (row0 / a.rows_per_bias) * (int64_t)a.V + v0 : nullptr;

    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (counts) {
        for (int i = threadIdx.x; i < a.chunk; i += kThreads) cnt[i] = 0;
        __syncthreads();
        if (a.e.history) {
            const int64_t b = node / a.D;
            const int n = a.e.history_len ? min(max(a.e.history_len[b], 0), a.e.history_cap) : a.e.history_cap;
            const int32_t* h = a.e.history + b * a.e.history_cap;
            for (int i = threadIdx.x; i < n; i += kThreads) {
                const unsigned t = (unsigned)h[i] - (unsigned)v0;
                if (t < (unsigned)vw && h[i] >= 0) atomicAdd(&cnt[t], 1);
            }
        }
        if (a.e.draft_tokens) {
            for (int i = threadIdx.x; i < a.M; i += kThreads) {
                const int id = a.e.draft_tokens[node * a.M + i];
                const unsigned t = (unsigned)id - (unsigned)v0;
                if (a.e.draft_mask[node * a.M + i] == 0 && id >= 0 && t < (unsigned)vw) atomicAdd(&cnt[t], 1);
            }
        }
        __syncthreads();
    }
    for (int w = warp; w < a.chunk / 32; w += kWarps) {
        const int i = w * 32 + lane;
        const bool sp = i < vw && ((counts && cnt[i] > 0) || (bias && bias[i] != 0.f));
        const uint32_t bits = __ballot_sync(0xffffffffu, sp);
        if (lane == 0) special[w] = bits;
    }
    __syncthreads();

    const int cols = a.chunk / a.wpr;                      // columns of one warp, a multiple of 512
    const int c0 = (warp % a.wpr) * cols;
    const int n_split = a.n_chunks * a.wpr;
    for (int rr = warp / a.wpr; rr < n_rows; rr += kWarps / a.wpr) {
        const int64_t row = row0 + rr;
        const T* lg = reinterpret_cast<const T*>(a.logits) + row * a.stride + v0;
        const uint32_t* allow = a.e.allow ? a.e.allow + (row / a.rows_per_allow) * (int64_t)a.words + v0 / 32 : nullptr;
        // bits of the 32 columns from column i (a multiple of 32) that the main loop takes
        auto open_word = [&](int i) -> uint32_t {
            const int left = vw - i;
            if (left <= 0) return 0u;
            uint32_t ok = allow ? allow[i >> 5] : 0xffffffffu;
            if (left < 32) ok &= (1u << left) - 1u;
            return ok;
        };
        // the E values of step k as the main loop sees them: -inf where absent
        auto load = [&](int k, float (&x)[E]) {
            if (VEC) {
                const int i = c0 + k * STEP + lane * E;
                const uint32_t w = i < vw ? open_word(i & ~31) & ~special[i >> 5] : 0u;
                const uint32_t b = w >> (i & 31);
                if (i + E <= vw) {
                    const uint4 r = __ldg(reinterpret_cast<const uint4*>(lg + i));
                    float y[Vec<T>::E];
                    Vec<T>::unpack(r, y);
#pragma unroll
                    for (int j = 0; j < E; ++j) x[j] = (b >> j) & 1u ? y[j < Vec<T>::E ? j : 0] : -INFINITY;
                } else {
#pragma unroll
                    for (int j = 0; j < E; ++j) x[j] = (i + j < vw && ((b >> j) & 1u)) ? Vec<T>::one(lg + i + j) : -INFINITY;
                }
            } else {
#pragma unroll
                for (int j = 0; j < E; ++j) {
                    const int i = c0 + k * STEP + j * 32;
                    const uint32_t w = i < vw ? open_word(i) & ~special[i >> 5] : 0u;
                    const float y = i + lane < vw ? Vec<T>::one(lg + i + lane) : 0.f;
                    x[j] = (w >> lane) & 1u ? y : -INFINITY;
                }
            }
        };
        float m = -INFINITY, s = 0.f;
        int best = -1;
        const int steps = min(cols, max(0, vw - c0) + STEP - 1) / STEP;
#pragma unroll 4
        for (int k = 0; k < steps; ++k) {
            float x[E];
            load(k, x);
            fold_group<E>(x, k, m, s, best);
        }
        // the special tokens of this warp's columns, in ascending order within a lane
        float sm = -INFINITY, ss = 0.f;
        int sa = INT32_MAX;
        for (int w = lane; w < cols / 32; w += 32) {
            const int i = c0 + w * 32;
            uint32_t bits = i < vw ? special[i >> 5] & open_word(i) : 0u;
            while (bits) {
                const int v = i + __ffs(bits) - 1;
                bits &= bits - 1;
                float x = Vec<T>::one(lg + v);
                const int n = counts ? cnt[v] : 0;
                if (n > 0) {
                    x = x > 0.f ? __fdiv_rn(x, a.e.repetition) : __fmul_rn(x, a.e.repetition);
                    x = __fsub_rn(x, __fadd_rn(__fmul_rn(a.e.frequency, (float)n), a.e.presence));
                }
                if (bias) x = __fadd_rn(x, bias[v]);
                const float mn = fmaxf(sm, x);
                if (x > sm) sa = v;
                ss = rescaled(ss, sm, mn) + (x == -INFINITY ? 0.f : ex2((x - mn) * kLog2e));
                sm = mn;
            }
        }
        // the warp's maximum; the lanes that hold it look up its column
        float M = fmaxf(m, sm);
#pragma unroll
        for (int o = 16; o; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
        float t = rescaled(s, m, M) + rescaled(ss, sm, M);
#pragma unroll
        for (int o = 16; o; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
        int at = INT32_MAX;
        if (M > -INFINITY) {
            if (sm == M) at = sa;
            if (m == M) {
                float x[E];
                load(best, x);
                int j = E - 1;
#pragma unroll
                for (int q = E - 2; q >= 0; --q) j = x[q] == M ? q : j;
                at = min(at, VEC ? c0 + best * STEP + lane * E + j : c0 + best * STEP + j * 32 + lane);
            }
        }
        at = __reduce_min_sync(0xffffffffu, at);
        if (lane == 0) {
            Part p = {M, t, at == INT32_MAX ? INT32_MAX : v0 + at, 0};
            a.part[row * n_split + c * a.wpr + warp % a.wpr] = p;
        }
    }
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

// One warp per row: the row's triples in a fixed order (lane by lane, then a fixed tree).
__global__ void __launch_bounds__(kThreads) logits_merge_kernel(const Part* __restrict__ part, int64_t n_rows, int n_split,
                                                                int32_t* __restrict__ out_token, float* __restrict__ out_conf,
                                                                float* __restrict__ out_lse, int32_t* status_dev) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int lane = threadIdx.x & 31;
    const int64_t row = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
    if (row >= n_rows) return;
    float m = -INFINITY, s = 0.f;
    int at = INT32_MAX;
    for (int i = lane; i < n_split; i += 32) {
        const Part p = part[row * n_split + i];
        const float mn = fmaxf(m, p.m);
        at = p.m > m ? p.a : p.m == m ? min(at, p.a) : at;
        s = rescaled(s, m, mn) + rescaled(p.s, p.m, mn);
        m = mn;
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        const float m2 = __shfl_xor_sync(0xffffffffu, m, o), s2 = __shfl_xor_sync(0xffffffffu, s, o);
        const int a2 = __shfl_xor_sync(0xffffffffu, at, o);
        const float mn = fmaxf(m, m2);
        at = m2 > m ? a2 : m2 == m ? min(at, a2) : at;
        s = rescaled(s, m, mn) + rescaled(s2, m2, mn);
        m = mn;
    }
    if (lane == 0) {
        const bool none = m == -INFINITY;          // nothing left, or only NaN (then s is NaN)
        const float sum = none && s == 0.f ? 0.f : s;
        out_token[row] = none || at == INT32_MAX ? -1 : at;
        out_conf[row] = none ? sum : 1.0f / sum;
        if (out_lse) out_lse[row] = none ? (sum == 0.f ? -INFINITY : sum) : m + logf(sum);
        if (status_dev && !(isfinite(sum) && m < INFINITY)) count_nonfinite_row(status_dev);
    }
}

// Columns per CTA and warps per row.  A warp should have a few thousand columns (the count of the text and the final
// reduction of a row are paid per CTA and per warp), and the grid at least two CTAs per SM.
void choose_chunk(int64_t units, int rows, int V, int& chunk, int& wpr) {
    wpr = rows >= 8 ? 1 : rows >= 4 ? 2 : rows >= 2 ? 4 : 8;
    chunk = 4096 * wpr < kMaxChunk ? 4096 * wpr : kMaxChunk;
    const int64_t want = 2 * (int64_t)sm_count();
    while (chunk / wpr > kMinWarpCols && units * ((V + chunk - 1) / chunk) < want) chunk /= 2;
}

template <typename T>
int launch(const LogitsArgs& a, int64_t grid, bool vec, cudaStream_t st) {
    const int smem = a.chunk * 4 + a.chunk / 8;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = pdl_enabled() ? 1 : 0;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    static std::atomic<unsigned long long> set_v{0}, set_s{0};
    constexpr int most = kMaxChunk * 4 + kMaxChunk / 8;
    cudaError_t e;
    if (vec) {
        if (!ensure_dynamic_smem(logits_kernel<T, true>, most, set_v)) return PSD_ERR_CUDA;
        e = cudaLaunchKernelEx(&cfg, logits_kernel<T, true>, a);
    } else {
        if (!ensure_dynamic_smem(logits_kernel<T, false>, most, set_s)) return PSD_ERR_CUDA;
        e = cudaLaunchKernelEx(&cfg, logits_kernel<T, false>, a);
    }
    count_launch();
    return e == cudaSuccess ? PSD_OK : PSD_ERR_CUDA;
}

}  // namespace

size_t confidence_logits_workspace(int64_t n_rows, int V) {
    // a chunk is a multiple of 512 columns and holds at least 512 per warp
    const int64_t n_split = (V + kMinWarpCols - 1) / kMinWarpCols + kMaxChunk / kMinWarpCols;
    return ((size_t)n_rows * n_split * sizeof(Part) + 255) / 256 * 256;
}

int launch_confidence_logits(const void* logits, int dtype, int64_t row_stride, int B, int D, int M, int V,
                             const psd_logits_edit_t& e, int32_t* out_token, float* out_conf, float* out_lse,
                             void* workspace, int32_t* status_dev, cudaStream_t st) {
    LogitsArgs a = {};
    const int64_t n_rows = (int64_t)B * D * M;
    a.logits = logits;
    a.stride = row_stride;
    a.M = M; a.V = V; a.D = D;
    a.e = e;
    const bool neutral = e.repetition == 1.f && e.presence == 0.f && e.frequency == 0.f;
    if (neutral || e.history_cap == 0) a.e.history = nullptr;
    if (neutral) a.e.draft_tokens = nullptr;
    a.rows_per_bias = (int)(n_rows / (e.bias ? e.bias_rows : 1));
    a.rows_per_allow = (int)(n_rows / (e.allow ? e.allow_rows : 1));
    a.words = (V + 31) / 32;
    a.unit_rows = e.bias ? gcd_int(M, a.rows_per_bias) : M;
    a.slices = (a.unit_rows + kRowsPerCta - 1) / kRowsPerCta;
    a.rows_per_cta = (a.unit_rows + a.slices - 1) / a.slices;
    a.slices = (a.unit_rows + a.rows_per_cta - 1) / a.rows_per_cta;
    const int64_t units = n_rows / a.unit_rows * a.slices;
    choose_chunk(units, a.rows_per_cta, V, a.chunk, a.wpr);
    a.n_chunks = (V + a.chunk - 1) / a.chunk;
    a.part = reinterpret_cast<Part*>(workspace);
    const int64_t grid = units * a.n_chunks;
    if (grid > INT32_MAX) return PSD_ERR_SHAPE;
    const int esize = dtype == PSD_FP32 ? 4 : 2;
    const bool vec = reinterpret_cast<uintptr_t>(logits) % 16 == 0 && (row_stride * esize) % 16 == 0;
    const int rc = dtype == PSD_BF16 ? launch<__nv_bfloat16>(a, grid, vec, st)
                 : dtype == PSD_FP16 ? launch<__half>(a, grid, vec, st) : launch<float>(a, grid, vec, st);
    if (rc != PSD_OK) return rc;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((n_rows + kWarps - 1) / kWarps));
    cfg.blockDim = dim3(kThreads);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = pdl_enabled() ? 1 : 0;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t err = cudaLaunchKernelEx(&cfg, logits_merge_kernel, (const Part*)a.part, n_rows, a.n_chunks * a.wpr,
                                               out_token, out_conf, out_lse, status_dev);
    count_launch();
    return err == cudaSuccess ? PSD_OK : PSD_ERR_CUDA;
}

}  // namespace psd
