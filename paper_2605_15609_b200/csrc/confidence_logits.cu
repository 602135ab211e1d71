// Token, confidence and log-sum-exp of rows of logits under penalties, biases and grammar masks.
//
// One pass over the logits (the only large operand): a CTA takes a few rows that share one text (a draft) and one
// bias row, and a chunk of the vocabulary; a warp walks a row's columns with a running maximum and sum per lane,
//     m' = max(m, x),  s' = s * 2^((m - m') log2 e) + sum 2^((x - m') log2 e),
// and writes one (max, sum, lowest argmax) triple per row and chunk; a second kernel merges them.
//
// The edits touch few tokens.  The CTA counts the text's tokens of its chunk in shared memory once for all its rows
// and marks every token that has a count or a bias ("special").  Per row, a warp first puts down one bit per column of
// its own: open = allowed, inside the vocabulary and not special; on the way each lane takes the special tokens of its words
// one by one, reads the logit and edits it with separately rounded operations.  The loop that streams the logits then
// knows nothing but those bits, whatever the edits are, and does not load 32 vectors of which no column is open.
//
// Differences are taken before the multiplication by log2 e: a row whose maximum is the type's lowest value would
// overflow a precomputed product, and its rounding would shift every term by the same relative error.
#include "combine.cuh"
#include "attn_tc.cuh"

namespace psd {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMaxChunk = 16384;      // tokens per CTA: 64 KB of counts
constexpr int kMinWarpCols = 256;     // columns a warp takes at least (sets the number of triples per row)
constexpr int kRowsPerCta = 64;

struct Part { float m, s; int32_t a, pad; };

struct LogitsArgs {
    const void* logits;
    int64_t stride;
    int M, V, D;
    int unit_rows, slices, rows_per_cta;   // rows of one node and one bias row; CTAs they are cut into; rows of each
    int chunk, n_chunks, wpr;              // columns per CTA; CTAs along the vocabulary; warps that share a row
    int rows_per_bias, rows_per_allow, words;
    int merge_early;                       // the merge's blocks are few: let them become resident at once
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

// The E values of a lane's vector, -inf where their bit is 0.
template <int E>
__device__ __forceinline__ void close_bits(float (&x)[E], uint32_t bits) {
#pragma unroll
    for (int j = 0; j < E; ++j) x[j] = bits & (1u << j) ? x[j] : -INFINITY;
}

// E values joined to a lane's running maximum and sum; g names the vector for the search of the argmax.
template <int E>
__device__ __forceinline__ void fold_vector(const float (&x)[E], int g, float& m, float& s, int& best) {
    float gm = max3(x[0], x[1], x[2]);
#pragma unroll
    for (int j = 3; j + 1 < E; j += 2) gm = max3(gm, x[j], x[j + 1]);
    if (E % 2 == 0) gm = fmaxf(gm, x[E - 1]);
    best = gm > m ? g : best;
    const float mn = fmaxf(m, gm);
    const float base = mn == -INFINITY ? 0.f : mn;
    const float f = ex2((m == mn ? 0.f : m - base) * kLog2e);   // m = -inf: s is 0 (or NaN), the factor 0 or 1
    const f32x2 nb = pack2(-base, -base), k = pack2(kLog2e, kLog2e);
    f32x2 acc = 0ull;
#pragma unroll
    for (int j = 0; j < E; j += 2) acc = add2(acc, ex2_pair(mul2(add2(pack2(x[j], x[j + 1]), nb), k)));
    float a0, a1;
    unpack2(acc, a0, a1);
    s = fmaf(s, f, a0 + a1);
    m = mn;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) logits_kernel(const LogitsArgs a) {
    constexpr int E = Vec<T>::E;               // columns of a lane's 16-byte vector
    constexpr int STEP = 32 * E;               // columns of a warp per step
    constexpr int U = 4;                       // vectors in flight per lane
    extern __shared__ int32_t sh[];
    int32_t* cnt = sh;                                              // [chunk]
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
    const int cols = a.chunk / a.wpr;                      // columns of one warp, a multiple of 256
    uint32_t* open = special + a.chunk / 32 + warp * (cols / 32 + 2) + 1;   // [cols / 32] and a closed word on either side

    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (a.merge_early) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (counts) {
        for (int i = threadIdx.x; i < a.chunk; i += kThreads) cnt[i] = 0;
        __syncthreads();
        if (a.e.history) {
            const int64_t b = node / a.D;
            const int n = a.e.history_len ? min(max(a.e.history_len[b], 0), a.e.history_cap) : a.e.history_cap;
            const int32_t* h = a.e.history + b * a.e.history_cap;
#pragma unroll 4
            for (int i = threadIdx.x; i < n; i += kThreads) {
                const int id = h[i];
                const unsigned t = (unsigned)id - (unsigned)v0;
                if (t < (unsigned)vw && id >= 0) atomicAdd(&cnt[t], 1);
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
#pragma unroll 4
    for (int w = warp; w < a.chunk / 32; w += kWarps) {
        const int i = w * 32 + lane;
        const bool sp = i < vw && ((counts && cnt[i] > 0) || (bias && bias[i] != 0.f));
        const uint32_t bits = __ballot_sync(0xffffffffu, sp);
        if (lane == 0) special[w] = bits;
    }
    if (lane == 0) open[-1] = open[cols / 32] = 0u;
    __syncthreads();

    const int c0 = (warp % a.wpr) * cols;
    const int len = max(0, min(cols, vw - c0));            // columns of this warp that exist
    const int n_split = a.n_chunks * a.wpr;
    for (int rr = warp / a.wpr; rr < n_rows; rr += kWarps / a.wpr) {
        const int64_t row = row0 + rr;
        const T* lg = reinterpret_cast<const T*>(a.logits) + row * a.stride + v0 + c0;    // this warp's column 0
        // Vectors are aligned in memory: with rows that are not, the first one starts `back` columns ahead of column 0.
        const int back = (int)((reinterpret_cast<uintptr_t>(lg) & 15) / sizeof(T));
        const uint32_t* allow = a.e.allow ? a.e.allow + (row / a.rows_per_allow) * (int64_t)a.words + (v0 + c0) / 32 : nullptr;
        float sm = -INFINITY, ss = 0.f;                    // the special tokens of this lane
        int sa = INT32_MAX;
        for (int w = lane; w < cols / 32; w += 32) {
            const int left = len - w * 32;
            uint32_t ok = 0u;
            if (left > 0) {
                ok = allow ? allow[w] : 0xffffffffu;
                if (left < 32) ok &= (1u << left) - 1u;
            }
            const uint32_t sp = special[c0 / 32 + w];
            open[w] = ok & ~sp;
            uint32_t bits = ok & sp;
            while (bits) {
                const int v = w * 32 + __ffs(bits) - 1;
                bits &= bits - 1;
                float x = Vec<T>::one(lg + v);
                const int n = counts ? cnt[c0 + v] : 0;
                if (n > 0) {
                    x = x > 0.f ? __fdiv_rn(x, a.e.repetition) : __fmul_rn(x, a.e.repetition);
                    x = __fsub_rn(x, __fadd_rn(__fmul_rn(a.e.frequency, (float)n), a.e.presence));
                }
                if (bias) x = __fadd_rn(x, bias[c0 + v]);
                const float mn = fmaxf(sm, x);
                if (x > sm) sa = v;
                ss = rescaled(ss, sm, mn) + (x == -INFINITY ? 0.f : ex2((x - mn) * kLog2e));
                sm = mn;
            }
        }
        __syncwarp();
        // bits of the vector that starts at column i (i >= -back, not a multiple of E when back != 0)
        auto bits_at = [&](int i) -> uint32_t {
            const uint32_t* w = open + (i >> 5);
            if (back == 0) return i < cols ? w[0] >> (i & 31) & ((1u << E) - 1u) : 0u;
            return i < cols ? __funnelshift_r(w[0], w[1], i & 31) & ((1u << E) - 1u) : 0u;
        };
        // first and last column of the row, as columns of this warp: a vector that reaches past them is read piece by piece
        const int lo = -(v0 + c0), hi = a.V - v0 - c0;
        auto fetch = [&](int i) -> uint4 {
            if (i >= lo && i + E <= hi) return __ldg(reinterpret_cast<const uint4*>(lg + i));
            uint4 r = make_uint4(0, 0, 0, 0);
            T* piece = reinterpret_cast<T*>(&r);
#pragma unroll
            for (int j = 0; j < E; ++j)
                if (i + j >= lo && i + j < hi) piece[j] = lg[i + j];
            return r;
        };
        float m = -INFINITY, s = 0.f;
        int best = -1;
        const int steps = len > 0 ? (len + back + STEP - 1) / STEP : 0;
        for (int k0 = 0; k0 < steps; k0 += U) {
            uint32_t bits[U];
            uint4 raw[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = (k0 + u) * STEP + lane * E - back;
                bits[u] = k0 + u < steps ? bits_at(i) : 0u;
                raw[u] = make_uint4(0, 0, 0, 0);
                if (bits[u]) raw[u] = fetch(i);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (!__any_sync(0xffffffffu, bits[u])) continue;
                float x[E];
                Vec<T>::unpack(raw[u], x);
                close_bits<E>(x, bits[u]);
                fold_vector<E>(x, k0 + u, m, s, best);
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
                const int i = best * STEP + lane * E - back;
                float x[E];
                Vec<T>::unpack(fetch(i), x);
                close_bits<E>(x, bits_at(i));
                int j = E - 1;
#pragma unroll
                for (int q = E - 2; q >= 0; --q) j = x[q] == M ? q : j;
                at = min(at, i + j);
            }
        }
        at = __reduce_min_sync(0xffffffffu, at);
        if (lane == 0) {
            Part p = {M, t, at == INT32_MAX ? INT32_MAX : v0 + c0 + at, 0};
            a.part[row * n_split + c * a.wpr + warp % a.wpr] = p;
        }
        __syncwarp();                                      // the row's bits have been read
    }
    if (!a.merge_early) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
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
#pragma unroll 8
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

int shared_bytes(int chunk, int wpr) { return chunk * 4 + chunk / 8 + kWarps * (chunk / wpr / 32 + 2) * 4; }

template <typename T>
int launch(const LogitsArgs& a, int64_t grid, cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = shared_bytes(a.chunk, a.wpr);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = pdl_enabled() ? 1 : 0;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    static std::atomic<unsigned long long> set{0};
    if (!ensure_dynamic_smem(logits_kernel<T>, shared_bytes(kMaxChunk, 1), set)) return PSD_ERR_CUDA;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, logits_kernel<T>, a);
    count_launch();
    return e == cudaSuccess ? PSD_OK : PSD_ERR_CUDA;
}

}  // namespace

size_t confidence_logits_workspace(int64_t n_rows, int V) {
    // a chunk holds at least kMinWarpCols columns per warp
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
    a.merge_early = n_rows <= 8 * kWarps;
    const int rc = dtype == PSD_BF16 ? launch<__nv_bfloat16>(a, grid, st)
                 : dtype == PSD_FP16 ? launch<__half>(a, grid, st) : launch<float>(a, grid, st);
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
