// Eviction from the prefix's cache by accumulated attention weight.
//
// Kernel 1, a cluster of one to eight CTAs per (sequence, key head): finds the n-th largest score among the positions that are
// not kept anyway by a radix select over order-preserving 32-bit keys (11, 11 and 10 bits; four copies of the histogram in
// shared memory, since scores of one magnitude fall into few bins; the CTAs add up one another's counts over distributed
// shared memory and so all take the same digit), then every warp walks a run of positions, counts what it keeps, and, after
// one scan over the warps and CTAs, writes it in order.  The keys of up to kCached positions per CTA stay in shared memory.
// 64 heads of up to 32768 positions: 27 us with one CTA per head, 21 with two, 28 with four (two to an SM); each
// cluster barrier costs about 0.7 us.
// Kernel 2 copies the kept rows: 16 bytes per thread, consecutive threads along a row; this is the part that is bound
// by memory (two rows read and two written per kept position): 64 heads, 8192 of up to 32768 keys of 128 x 2 bytes, 537 MB, in 89
// us = 0.83-0.92 of the copy bandwidth.
#include "ops_internal.cuh"
#include "tc_common.cuh"

namespace psd {
namespace {

constexpr int kSelThreads = 1024;
constexpr int kBins = 2048;
constexpr int kCopies = 4;
constexpr int kPad = 8;              // words between copies beyond the bins: equal bins of different copies are in different banks
constexpr int kCached = 36 * 1024;   // keys of a CTA held in shared memory (144 KB)
constexpr int kMaxCluster = 8;

// Larger key = higher score; NaN is the lowest, -0 equals +0.
__device__ __forceinline__ uint32_t score_key(float x) {
    if (x != x) return 0u;
    const uint32_t u = __float_as_uint(x == 0.f ? 0.f : x);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

__device__ __forceinline__ void cluster_barrier() {
    asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}
// The sum of two neighbouring words (8-byte aligned) over the CTAs [0, n) of the cluster: all loads are in flight at once.
__device__ __forceinline__ uint2 sum_over_ctas(const uint32_t* p, int n) {
    uint2 v[kMaxCluster], sum = {0, 0};
#pragma unroll
    for (int r = 0; r < kMaxCluster; ++r) {
        v[r] = {0, 0};
        if (r >= n) continue;
        uint32_t at;
        asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(p)), "r"(r));
        asm volatile("ld.shared::cluster.v2.u32 {%0, %1}, [%2];" : "=r"(v[r].x), "=r"(v[r].y) : "r"(at) : "memory");
    }
#pragma unroll
    for (int r = 0; r < kMaxCluster; ++r) {
        sum.x += v[r].x;
        sum.y += v[r].y;
    }
    return sum;
}

struct SelectArgs {
    const float* scores;
    const int32_t* prefix_len;
    int P, Hkv, keep, n_sink, n_recent;
    int log_cta, own;             // a cluster of 1 << log_cta CTAs per head, `own` positions for each
    int32_t* index;
    float* scores_out;
    int32_t* len_out;
};

// CACHED: the keys stay in shared memory after the first pass; otherwise every pass makes them again.
template <bool CACHED>
__global__ void __launch_bounds__(kSelThreads) evict_select_kernel(const SelectArgs a) {
    // in a cluster: [2][kBins] this CTA's counts, read by the cluster, passes alternate; then, if CACHED, the keys of this CTA
    extern __shared__ __align__(8) uint32_t dynamic[];
    __shared__ uint32_t hist[kCopies][kBins + kPad];
    __shared__ __align__(8) uint32_t cta_sum[2];                // this CTA's keys above and equal to the threshold
    __shared__ uint32_t warp_sum[32], warp_eq[32];
    __shared__ uint32_t s_digit, s_left;
    const int n_cta = 1 << a.log_cta, rank = blockIdx.x & (n_cta - 1), bh = blockIdx.x >> a.log_cta, b = bh / a.Hkv, h = bh % a.Hkv;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    for (int i = tid; i < kCopies * (kBins + kPad); i += kSelThreads) (&hist[0][0])[i] = 0;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int L = a.prefix_len ? min(max(a.prefix_len[b], 0), a.P) : a.P;
    const float* sc = a.scores + (int64_t)bh * a.P;
    int32_t* index = a.index + (int64_t)bh * a.keep;
    float* so = a.scores_out ? a.scores_out + (int64_t)bh * a.keep : nullptr;
    const int n_out = min(L, a.keep);
    if (h == 0 && tid == 0 && rank == 0 && a.len_out) a.len_out[b] = n_out;
    for (int i = n_out + rank * kSelThreads + tid; i < a.keep; i += n_cta * kSelThreads) {
        index[i] = -1;
        if (so) so[i] = 0.f;
    }
    if (L <= a.keep) {
        for (int i = rank * kSelThreads + tid; i < L; i += n_cta * kSelThreads) {
            index[i] = i;
            if (so) so[i] = sc[i];
        }
        asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
        return;
    }
    // this CTA's positions [c0, c1); the whole cluster takes the same decisions, so it meets at every barrier
    const int c0 = min(L, rank * a.own), c1 = min(L, c0 + a.own);
    uint32_t* keys = dynamic + (n_cta > 1 ? 2 * kBins : 0);
    // positions [lo, hi) compete for n_free places; the others are kept: their keys are the largest there is (no score's)
    const int lo = min(a.n_sink, L), hi = max(lo, L - a.n_recent);
    auto make_key = [&](int i, float x) { return (unsigned)(i - lo) < (unsigned)(hi - lo) ? score_key(x) : 0xffffffffu; };
    auto key_at = [&](int i) { return CACHED ? keys[i - c0] : make_key(i, sc[i]); };
    uint32_t threshold = 0xfffffffeu, n_equal = 0;  // keep keys > threshold, and the first n_equal equal to it
    __syncthreads();
    {
        uint32_t left = (uint32_t)(a.keep - lo - (L - hi));      // n_free < hi - lo here
        uint32_t prefix = 0, mask = 0;
#pragma unroll 1
        for (int pass = 0; pass < 3; ++pass) {
            const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
            const uint32_t digits = pass == 2 ? 1023u : 2047u;
            uint32_t* mine = hist[lane & (kCopies - 1)];
            if (pass == 0) {
                // the scores once, eight loads in flight per thread
#pragma unroll 1
                for (int i0 = c0 + tid; i0 < c1; i0 += 8 * kSelThreads) {
                    float x[8];
#pragma unroll
                    for (int u = 0; u < 8; ++u) x[u] = i0 + u * kSelThreads < c1 ? sc[i0 + u * kSelThreads] : 0.f;
#pragma unroll
                    for (int u = 0; u < 8; ++u) {
                        const int i = i0 + u * kSelThreads;
                        if (i >= c1) break;
                        const uint32_t k = make_key(i, x[u]);
                        if (CACHED) keys[i - c0] = k;
                        if (k != 0xffffffffu) atomicAdd(&mine[k >> 21], 1u);
                    }
                }
            } else {
#pragma unroll 4
                for (int i = c0 + tid; i < c1; i += kSelThreads) {
                    const uint32_t k = key_at(i);
                    if ((k & mask) == prefix && k != 0xffffffffu) atomicAdd(&mine[(k >> shift) & digits], 1u);
                }
            }
            __syncthreads();
            if (left == 0) break;                                // every place is taken (the keys have been made)
            // suffix sums: thread t owns bins 2t, 2t + 1, counted from the top (and clears them for the next pass)
            const int b1 = kBins - 1 - 2 * tid, b0 = b1 - 1;
            uint32_t n1 = 0, n0 = 0;
#pragma unroll
            for (int q = 0; q < kCopies; ++q) {
                n1 += hist[q][b1];
                n0 += hist[q][b0];
                hist[q][b1] = hist[q][b0] = 0;
            }
            if (n_cta > 1) {
                uint32_t* mine_total = dynamic + (pass & 1) * kBins;
                *reinterpret_cast<uint2*>(mine_total + b0) = {n0, n1};
                cluster_barrier();
                const uint2 n = sum_over_ctas(mine_total + b0, n_cta);
                n0 = n.x;
                n1 = n.y;
            }
            uint32_t run = n0 + n1;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t y = __shfl_up_sync(0xffffffffu, run, o);
                if (lane >= o) run += y;
            }
            if (lane == 31) warp_sum[warp] = run;
            __syncthreads();
            uint32_t before = lane < warp ? warp_sum[lane] : 0u;
            before = __reduce_add_sync(0xffffffffu, before);
            const uint32_t above = run - n0 - n1 + before;       // keys in higher bins
            if (above < left && above + n1 >= left) { s_digit = b1; s_left = left - above; }
            else if (above + n1 < left && above + n1 + n0 >= left) { s_digit = b0; s_left = left - above - n1; }
            __syncthreads();
            prefix |= s_digit << shift;
            mask |= digits << shift;
            left = s_left;
        }
        if (left > 0) {
            threshold = prefix;
            n_equal = left;
        }
    }
    // ordered write: a warp takes a run of positions, in steps of 32; first counts, then places
    const int per = (c1 - c0 + 32 * 32 - 1) / (32 * 32) * 32, i0 = min(c1, c0 + warp * per), i1 = min(c1, i0 + per);
    uint32_t n_above = 0, n_eq = 0;
#pragma unroll 4
    for (int i = i0; i < i1; i += 32) {
        const uint32_t k = i + lane < i1 ? key_at(i + lane) : 0u;
        n_above += __popc(__ballot_sync(0xffffffffu, k > threshold));
        n_eq += __popc(__ballot_sync(0xffffffffu, k == threshold && i + lane < i1));
    }
    if (lane == 0) { warp_sum[warp] = n_above; warp_eq[warp] = n_eq; }
    __syncthreads();
    uint32_t base_above = __reduce_add_sync(0xffffffffu, lane < warp ? warp_sum[lane] : 0u);
    uint32_t base_eq = __reduce_add_sync(0xffffffffu, lane < warp ? warp_eq[lane] : 0u);
    if (n_cta > 1) {
        if (tid == kSelThreads - 1) {
            cta_sum[0] = base_above + warp_sum[31];
            cta_sum[1] = base_eq + warp_eq[31];
        }
        cluster_barrier();
        const uint2 n = sum_over_ctas(cta_sum, rank);
        base_above += n.x;
        base_eq += n.y;
    }
    const uint32_t lt = (1u << lane) - 1u;
    // (the scores are fetched for eight steps at once, kept or not: in the branch every step would wait for its own)
#pragma unroll 1
    for (int j0 = i0; j0 < i1; j0 += 8 * 32) {
        float x[8];
        if (so || !CACHED)
#pragma unroll
            for (int u = 0; u < 8; ++u)
                if (j0 + u * 32 < i1) x[u] = j0 + u * 32 + lane < i1 ? sc[j0 + u * 32 + lane] : 0.f;
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            if (j0 + u * 32 >= i1) break;
            const int i = j0 + u * 32 + lane;
            const uint32_t k = i < i1 ? (CACHED ? keys[i - c0] : make_key(i, x[u])) : 0u;
            const bool above = k > threshold, eq = k == threshold && i < i1;
            const uint32_t ba = __ballot_sync(0xffffffffu, above), be = __ballot_sync(0xffffffffu, eq);
            const uint32_t eq_before = base_eq + __popc(be & lt);
            if (above || (eq && eq_before < n_equal)) {
                const uint32_t at = base_above + __popc(ba & lt) + min(eq_before, n_equal);
                index[at] = i;
                if (so) so[at] = x[u];
            }
            base_above += __popc(ba);
            base_eq += __popc(be);
        }
    }
    if (n_cta > 1) cluster_barrier();              // no CTA's shared memory goes while another may read it
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
    // CTAs per head: as many as keep a wave of them on the SMs and 4096 positions to each (below that a barrier costs more than
    // the positions)
    int log_cta = 0;
    while ((2 << log_cta) <= kMaxCluster && ((int64_t)e.B * e.Hkv * 2 << log_cta) <= sm_count() && e.P >> (log_cta + 1) >= 4096) ++log_cta;
    const int n_cta = 1 << log_cta, own = (int)(((int64_t)e.P + n_cta * 32 - 1) / (n_cta * 32) * 32);
    SelectArgs s = {scores, prefix_len, e.P, e.Hkv, e.keep, e.n_sink, e.n_recent, log_cta, own, index, scores_out, len_out};
    const bool cached = own <= kCached;
    const int counts = n_cta > 1 ? 2 * kBins * 4 : 0;
    static std::atomic<unsigned long long> smem_set{0}, smem_set_far{0};
    if (!ensure_dynamic_smem(evict_select_kernel<true>, kCached * 4 + 2 * kBins * 4, smem_set) ||
        !ensure_dynamic_smem(evict_select_kernel<false>, 2 * kBins * 4, smem_set_far)) return PSD_ERR_CUDA;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(e.B * e.Hkv * n_cta);
    cfg.blockDim = dim3(kSelThreads);
    cfg.dynamicSmemBytes = counts + (cached ? (size_t)own * 4 : 0);
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = pdl_enabled() ? 1 : 0;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim = {(unsigned)n_cta, 1, 1};
    cfg.attrs = attr;
    cfg.numAttrs = n_cta > 1 ? 2 : 1;
    cudaError_t err = cached ? cudaLaunchKernelEx(&cfg, evict_select_kernel<true>, s) : cudaLaunchKernelEx(&cfg, evict_select_kernel<false>, s);
    cfg.numAttrs = 1;
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
