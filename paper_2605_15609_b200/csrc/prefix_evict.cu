// Eviction from the prefix's cache by accumulated attention weight.
//
// Kernel 1, one CTA per (sequence, key head): finds the n-th largest score among the positions that are not kept
// anyway by a radix select over order-preserving 32-bit keys (11, 11 and 10 bits; histograms in shared memory), then
// walks the positions in order and writes those above the threshold key, and the first of those equal to it.  The scores
// of up to kCached positions stay in shared memory after the first read.
// Kernel 2 copies the kept rows: 16 bytes per thread, consecutive threads along a row; this is the part that is bound
// by memory (two rows read and two written per kept position).
#include "ops_internal.cuh"
#include "tc_common.cuh"

namespace psd {
namespace {

constexpr int kSelThreads = 1024;
constexpr int kBins = 2048;
constexpr int kCached = 48 * 1024;   // keys held in shared memory (192 KB)

// Larger key = higher score; NaN is the lowest, -0 equals +0.
__device__ __forceinline__ uint32_t score_key(float x) {
    if (x != x) return 0u;
    const uint32_t u = __float_as_uint(x == 0.f ? 0.f : x);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

struct SelectArgs {
    const float* scores;
    const int32_t* prefix_len;
    int P, Hkv, keep, n_sink, n_recent, cached;
    int32_t* index;
    float* scores_out;
    int32_t* len_out;
};

__global__ void __launch_bounds__(kSelThreads) evict_select_kernel(const SelectArgs a) {
    extern __shared__ uint32_t keys[];             // [cached]
    __shared__ uint32_t hist[kBins];
    __shared__ uint32_t warp_sum[32];
    __shared__ uint32_t s_digit, s_left;
    const int bh = blockIdx.x, b = bh / a.Hkv, h = bh % a.Hkv;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int L = a.prefix_len ? min(max(a.prefix_len[b], 0), a.P) : a.P;
    const float* sc = a.scores + (int64_t)bh * a.P;
    int32_t* index = a.index + (int64_t)bh * a.keep;
    float* so = a.scores_out ? a.scores_out + (int64_t)bh * a.keep : nullptr;
    const int n_out = min(L, a.keep);
    if (h == 0 && tid == 0 && a.len_out) a.len_out[b] = n_out;
    for (int i = n_out + tid; i < a.keep; i += kSelThreads) {
        index[i] = -1;
        if (so) so[i] = 0.f;
    }
    // positions [lo, hi) compete for n_free places; the others are kept
    const int lo = min(a.n_sink, L), hi = max(lo, L - a.n_recent);
    uint32_t threshold = 0, n_equal = 0;            // keep keys > threshold, and the first n_equal equal to it
    if (L > a.keep) {
        const bool cached = L <= a.cached;
        uint32_t left = (uint32_t)(a.keep - lo - (L - hi));      // n_free < hi - lo here
        uint32_t prefix = 0, mask = 0;
        if (left > 0) {
#pragma unroll 1
            for (int pass = 0; pass < 3; ++pass) {
                const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
                const uint32_t digits = pass == 2 ? 1023u : 2047u;
                for (int i = tid; i < kBins; i += kSelThreads) hist[i] = 0;
                __syncthreads();
                for (int i = lo + tid; i < hi; i += kSelThreads) {
                    uint32_t k;
                    if (pass == 0 || !cached) {
                        k = score_key(sc[i]);
                        if (cached) keys[i] = k;
                    } else {
                        k = keys[i];
                    }
                    if ((k & mask) == prefix) atomicAdd(&hist[(k >> shift) & digits], 1u);
                }
                __syncthreads();
                // suffix sums: thread t owns bins 2t, 2t + 1, counted from the top
                const int b1 = kBins - 1 - 2 * tid, b0 = b1 - 1;
                const uint32_t c1 = hist[b1], c0 = hist[b0];
                uint32_t run = c0 + c1;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const uint32_t y = __shfl_up_sync(0xffffffffu, run, o);
                    if (lane >= o) run += y;
                }
                if (lane == 31) warp_sum[warp] = run;
                __syncthreads();
                if (warp == 0) {
                    uint32_t w = warp_sum[lane];
#pragma unroll
                    for (int o = 1; o < 32; o <<= 1) {
                        const uint32_t y = __shfl_up_sync(0xffffffffu, w, o);
                        if (lane >= o) w += y;
                    }
                    warp_sum[lane] = w;
                }
                __syncthreads();
                const uint32_t above = run - c0 - c1 + (warp ? warp_sum[warp - 1] : 0u);   // keys in higher bins
                if (above < left && above + c1 >= left) { s_digit = b1; s_left = left - above; }
                else if (above + c1 < left && above + c1 + c0 >= left) { s_digit = b0; s_left = left - above - c1; }
                __syncthreads();
                prefix |= s_digit << shift;
                mask |= digits << shift;
                left = s_left;
                __syncthreads();
            }
            threshold = prefix;
            n_equal = left;
        } else {
            threshold = 0xffffffffu;                 // no score is above this
        }
    }
    // ordered write: per tile of 1024 positions, counts of kept and of equal keys before each thread
    uint32_t base_above = 0, base_eq = 0;
    const bool all = L <= a.keep;
    for (int t0 = 0; t0 < L; t0 += kSelThreads) {
        const int i = t0 + tid;
        float x = 0.f;
        bool above = false, eq = false;
        if (i < L) {
            x = sc[i];
            const uint32_t k = score_key(x);
            const bool middle = i >= lo && i < hi;
            above = all || !middle || k > threshold;
            eq = !above && k == threshold && n_equal > 0;
        }
        const uint32_t ba = __ballot_sync(0xffffffffu, above), be = __ballot_sync(0xffffffffu, eq);
        if (lane == 0) warp_sum[warp] = __popc(ba) | (__popc(be) << 16);
        __syncthreads();
        if (warp == 0) {
            uint32_t w = warp_sum[lane];
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t y = __shfl_up_sync(0xffffffffu, w, o);
                if (lane >= o) w += y;
            }
            warp_sum[lane] = w;
        }
        __syncthreads();
        const uint32_t before = warp ? warp_sum[warp - 1] : 0u, total = warp_sum[31];
        const uint32_t lt = (1u << lane) - 1u;
        const uint32_t n_above = base_above + (before & 0xffffu) + __popc(ba & lt);
        const uint32_t eq_before = base_eq + (before >> 16) + __popc(be & lt);
        if (above || (eq && eq_before < n_equal)) {
            const uint32_t at = n_above + min(eq_before, n_equal);
            index[at] = i;
            if (so) so[at] = x;
        }
        base_above += total & 0xffffu;
        base_eq += total >> 16;
        __syncthreads();
    }
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

struct GatherArgs {
    const uint4 *k, *v;
    uint4 *k_out, *v_out;
    psd_kv_strides_t ks, vs, kos, vos;      // in units of 16 bytes
    const int32_t* index;
    int Hkv, keep, chunks;                   // chunks: 16-byte pieces per row
    int64_t pieces;                          // B * keep * Hkv * chunks
};

constexpr int kGatherThreads = 256, kGatherPer = 4;

__global__ void __launch_bounds__(kGatherThreads) evict_gather_kernel(const GatherArgs a) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int64_t base = (int64_t)blockIdx.x * (kGatherThreads * kGatherPer) + threadIdx.x;
    uint4 rk[kGatherPer], rv[kGatherPer];
    int64_t ok[kGatherPer], ov[kGatherPer];
#pragma unroll
    for (int u = 0; u < kGatherPer; ++u) {
        const int64_t p = base + (int64_t)u * kGatherThreads;
        ok[u] = -1;
        if (p >= a.pieces) continue;
        const int64_t row = p / a.chunks;
        const int ch = (int)(p - row * a.chunks);
        const int64_t bs = row / a.Hkv;
        const int h = (int)(row - bs * a.Hkv);
        const int64_t b = bs / a.keep;
        const int slot = (int)(bs - b * a.keep);
        const int j = a.index[(b * a.Hkv + h) * a.keep + slot];
        if (j < 0) continue;
        rk[u] = __ldcs(a.k + b * a.ks.outer + (int64_t)j * a.ks.token + h * a.ks.head + ch);
        rv[u] = __ldcs(a.v + b * a.vs.outer + (int64_t)j * a.vs.token + h * a.vs.head + ch);
        ok[u] = b * a.kos.outer + (int64_t)slot * a.kos.token + h * a.kos.head + ch;
        ov[u] = b * a.vos.outer + (int64_t)slot * a.vos.token + h * a.vos.head + ch;
    }
#pragma unroll
    for (int u = 0; u < kGatherPer; ++u)
        if (ok[u] >= 0) {
            a.k_out[ok[u]] = rk[u];
            a.v_out[ov[u]] = rv[u];
        }
}

psd_kv_strides_t pieces_of(const psd_kv_strides_t& s) { return {s.outer / 8, s.token / 8, s.head / 8}; }

}  // namespace

int launch_prefix_evict(const float* scores, const void* k, const void* v, const int32_t* prefix_len,
                        const psd_evict_t& e, void* k_out, void* v_out, int32_t* index, float* scores_out,
                        int32_t* len_out, cudaStream_t st) {
    SelectArgs s = {scores, prefix_len, e.P, e.Hkv, e.keep, e.n_sink, e.n_recent, e.P < kCached ? e.P : kCached,
                    index, scores_out, len_out};
    if (e.P > kCached) s.cached = 0;       // too long to hold: every pass reads the scores again (from L2)
    static std::atomic<unsigned long long> smem_set{0};
    if (!ensure_dynamic_smem(evict_select_kernel, kCached * 4, smem_set)) return PSD_ERR_CUDA;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(e.B * e.Hkv);
    cfg.blockDim = dim3(kSelThreads);
    cfg.dynamicSmemBytes = (size_t)s.cached * 4;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = pdl_enabled() ? 1 : 0;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    cudaError_t err = cudaLaunchKernelEx(&cfg, evict_select_kernel, s);
    count_launch();
    if (err != cudaSuccess) return PSD_ERR_CUDA;
    GatherArgs g = {};
    g.k = reinterpret_cast<const uint4*>(k);
    g.v = reinterpret_cast<const uint4*>(v);
    g.k_out = reinterpret_cast<uint4*>(k_out);
    g.v_out = reinterpret_cast<uint4*>(v_out);
    g.ks = pieces_of(e.k); g.vs = pieces_of(e.v); g.kos = pieces_of(e.k_out); g.vos = pieces_of(e.v_out);
    g.index = index;
    g.Hkv = e.Hkv; g.keep = e.keep; g.chunks = e.Dh / 8;
    g.pieces = (int64_t)e.B * e.keep * e.Hkv * g.chunks;
    const int64_t per = kGatherThreads * kGatherPer, blocks = (g.pieces + per - 1) / per;
    if (blocks > INT32_MAX) return PSD_ERR_SHAPE;
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3(kGatherThreads);
    cfg.dynamicSmemBytes = 0;
    err = cudaLaunchKernelEx(&cfg, evict_gather_kernel, g);
    count_launch();
    return err == cudaSuccess ? PSD_OK : PSD_ERR_CUDA;
}

}  // namespace psd
