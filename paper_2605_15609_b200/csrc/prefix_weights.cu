// Attention weight drawn by every prefix key, summed over the rows that read it:
//   sum_r exp(scale * q_r . K_j - lse_r)  =  sum_r 2^(c * q_r . K_j - lse_r log2 e),   c = scale * log2 e.
//
// The scores are computed transposed, S^T = K Q^T: a tile of 128 keys is the M side of tcgen05.mma and 128 query rows are
// the N side, so a thread of the epilogue (one TMEM lane) owns one KEY and walks the query rows as columns.  The sum over
// rows is then a running sum in a register: no reduction between threads, no atomics, a fixed order.  A CTA keeps two key
// tiles in shared memory and streams the query rows of their key head past both (each query tile is fetched once per 256
// keys), so K is read once and nothing but the sums is written.
//
// Warps 0-3 and 4-7 take the two key tiles, warp 8 loads, warp 9 issues the products.  Accumulators are double-buffered per
// key tile (4 x 128 TMEM columns).  One exponential per score is what bounds the kernel (16 per clock and SM against 8192
// multiply-adds): see ex2_some.
#include "attn_tc.cuh"

namespace psd {
namespace {

constexpr int kKeysPerCta = 256;
constexpr int kQStages = 4;
constexpr int kEpilogue = 16;           // warps that sum: two per key tile and quarter, 64 columns of a query tile each
constexpr int kWThreads = (kEpilogue + 2) * 32;
constexpr int kMaxSplits = 16;

struct WeightsArgs {
    const int32_t* prefix_len;
    const float *lse, *acc_in;
    float *acc_out, *part;          // part: [splits][B * Hkv][P] when splits > 1
    int32_t* status_dev;
    int T, G, Hq, Hkv, Dh, P;       // T: tokens per sequence (D * M)
    int tq, n_qt, key_ctas, splits; // tokens per query tile, query tiles, CTAs along the keys, splits of the query tiles
    int k_outer, k_head;            // 0: that dimension of the cache is shared
    float c, beta;
    int bf16;
    long long wait_limit;
};

template <int SLABS>
__global__ void __launch_bounds__(kWThreads, 1)
weights_tc_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_q, const WeightsArgs a) {
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
    constexpr int TILE = SLABS * kSlabBytes;
    unsigned char* k_tiles = smem;                                   // [2][TILE]
    unsigned char* q_tiles = smem + 2 * TILE;                        // [kQStages][TILE]
    float* lse_buf = reinterpret_cast<float*>(smem + (2 + kQStages) * TILE);       // [kEpilogue][2][64]
    float* halves = lse_buf + kEpilogue * 2 * 64;                    // [2][128] sums of the second halves
    uint64_t* bars = reinterpret_cast<uint64_t*>(halves + 256);
    uint64_t *k_full = bars, *q_full = bars + 1, *q_empty = q_full + kQStages, *s_full = q_empty + kQStages /* [2][2] */,
             *s_empty = s_full + 4, *drain = s_empty + 4;
    uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(drain + 1);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_holder + 1);

    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    const int kc = blockIdx.x % a.key_ctas;
    const int rest = blockIdx.x / a.key_ctas, split = rest % a.splits, bh = rest / a.splits;
    const int b = bh / a.Hkv, h = bh % a.Hkv;
    const int key0 = kc * kKeysPerCta;

    if (threadIdx.x == 0) {
        mbar_init(k_full, 1);
        for (int s = 0; s < kQStages; ++s) { mbar_init(&q_full[s], 1); mbar_init(&q_empty[s], 1); }
        for (int s = 0; s < 4; ++s) { mbar_init(&s_full[s], 1); mbar_init(&s_empty[s], 8); }
        mbar_init(drain, 1);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kEpilogue && lane == 0) { tma_prefetch_desc(&map_k); tma_prefetch_desc(&map_q); }
    if (warp == kEpilogue + 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_holder)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, *tmem_holder, 0);
    asm volatile("griddepcontrol.wait;" ::: "memory");

    const WaitCtx wc = {abort_flag, a.status_dev, a.wait_limit, 0u};
    const int L = a.prefix_len ? min(max(a.prefix_len[b], 0), a.P) : a.P;
    // query tiles of this split; none when no key of this CTA is inside the prefix
    const int q_lo = key0 < L ? (int)((long long)a.n_qt * split / a.splits) : 0;
    const int q_hi = key0 < L ? (int)((long long)a.n_qt * (split + 1) / a.splits) : 0;
    const int n_it = q_hi - q_lo;
    const int n_kt = L - key0 > 128 ? 2 : 1;      // key tiles that hold keys

    float total = 0.f;
    if (warp == kEpilogue) {
        if (n_it > 0) {
            const bool leader = elect_one();
            if (leader) {
                mbar_arrive_expect_tx(k_full, n_kt * TILE);
                for (int t = 0; t < n_kt; ++t)
                    for (int s = 0; s < SLABS; ++s)
                        tma_load_4d(k_tiles + t * TILE + s * kSlabBytes, &map_k, k_full, s * kSlabElems, h * a.k_head, key0 + t * 128, b * a.k_outer);
            }
            const uint32_t q_bytes = (uint32_t)(SLABS * a.tq * a.G * 128);
            int it = 0;
            bool ok = true;
            for (; it < n_it; ++it) {
                const int s = it % kQStages;
                if (!mbar_wait_warp(&q_empty[s], ((it / kQStages) & 1) ^ 1, wc)) { ok = false; break; }
                if (leader) {
                    mbar_arrive_expect_tx(&q_full[s], q_bytes);
#pragma unroll
                    for (int c = 0; c < SLABS; ++c)
                        tma_load_3d(q_tiles + s * TILE + c * kSlabBytes, &map_q, &q_full[s], c * kSlabElems, h * a.G, b * a.T + (q_lo + it) * a.tq);
                }
            }
            if (!ok) {
                // giving up: no copy may be in flight when the CTA exits
                long long t0 = clock64();
                while (!mbar_try_wait(k_full, 0) && clock64() - t0 < WAIT_LIMIT_CYCLES) {}
                for (int i = it > kQStages ? it - kQStages : 0; i < it; ++i) {
                    t0 = clock64();
                    while (!mbar_try_wait(&q_full[i % kQStages], (i / kQStages) & 1) && clock64() - t0 < WAIT_LIMIT_CYCLES) {}
                }
            }
        }
    } else if (warp == kEpilogue + 1) {
        if (n_it > 0) {
            const bool leader = elect_one();
            const uint32_t idesc = umma_idesc16(128, a.bf16, false);
            const int k_steps = (a.Dh + 15) / 16;
            const uint64_t dk = umma_smem_desc(smem_u32(k_tiles)), dq = umma_smem_desc(smem_u32(q_tiles));
            bool ok = mbar_wait_warp(k_full, 0, wc);
            for (int it = 0; ok && it < n_it; ++it) {
                const int s = it % kQStages, buf = it & 1;
                if (!mbar_wait_warp(&q_full[s], (it / kQStages) & 1, wc)) { ok = false; break; }
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    if (!ok || t >= n_kt) continue;
                    if (!mbar_wait_warp(&s_empty[t * 2 + buf], ((it >> 1) & 1) ^ 1, wc)) { ok = false; continue; }
                    tc_fence_after();
                    if (leader) {
                        const uint64_t k = dk + (uint64_t)(t * (TILE >> 4)), q = dq + (uint64_t)(s * (TILE >> 4));
#pragma unroll
                        for (int i = 0; i < SLABS * 4; ++i)
                            if (i < k_steps) {
                                const uint64_t off = (i / 4) * (kSlabBytes >> 4) + (i % 4) * 2;
                                umma_f16(tmem + (t * 2 + buf) * 128, k + off, q + off, idesc, i != 0);
                            }
                        umma_commit(&s_full[t * 2 + buf]);
                    }
                }
                if (ok && leader) umma_commit(&q_empty[s]);
            }
            if (!ok) {
                if (leader) umma_commit(drain);
                const long long t0 = clock64();
                while (!mbar_try_wait(drain, 0) && clock64() - t0 < WAIT_LIMIT_CYCLES) {}
            }
        }
    } else {
        const int t = warp >> 3, half = (warp >> 2) & 1, quarter = warp & 3;
        float* lb = lse_buf + warp * 128;
        float s4[4] = {0.f, 0.f, 0.f, 0.f};
        // This lane's two columns of every query tile: where their lse is, and which token of the tile they belong to.
        const float* lp[2];
        int lt_tok[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int c = half * 64 + lane * 2 + u;
            lt_tok[u] = c < a.tq * a.G ? c / a.G : a.T;
            lp[u] = a.lse + ((int64_t)b * a.T + (int64_t)q_lo * a.tq + c / a.G) * a.Hq + h * a.G + c % a.G;
        }
        // -lse * log2 e of the columns of tile `it`; -inf marks a column that adds nothing
        auto fetch_lse = [&](int it, float (&v)[2]) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const float l = lt_tok[u] + (q_lo + it) * a.tq < a.T ? lp[u][(int64_t)it * a.tq * a.Hq] : -INFINITY;
                v[u] = l == -INFINITY ? -INFINITY : -l * kLog2e;
            }
        };
        // Two chunks of 32 columns per tile: while one is summed the next is on its way from tensor memory, across tiles too,
        // so that the exponentials never wait for a load.
        const uint32_t lane_at = tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(t * 256 + half * 64);
        uint32_t r[2][32];
        auto sum = [&](const uint32_t (&r)[32], const float* lt, bool all) {
            if (all) {
#pragma unroll
                for (int j = 0; j < 32; j += 4) {
                    const float4 l = *reinterpret_cast<const float4*>(lt + j);
                    const uint32_t* x = r + j;
                    s4[0] += ex2(fmaf(__uint_as_float(x[0]), a.c, l.x));
                    s4[1] += ex2(fmaf(__uint_as_float(x[1]), a.c, l.y));
                    s4[2] += ex2(fmaf(__uint_as_float(x[2]), a.c, l.z));
                    s4[3] += ex2(fmaf(__uint_as_float(x[3]), a.c, l.w));
                }
            } else {
                // some columns are absent (what the tile holds there is not used)
#pragma unroll
                for (int j = 0; j < 32; ++j) {
                    const float l = lt[j];
                    if (l != -INFINITY) s4[0] += ex2(fmaf(__uint_as_float(r[j]), a.c, l));
                }
            }
        };
        float nl[2];
        bool ok = t < n_kt && n_it > 0;
        if (ok) {
            fetch_lse(0, nl);
            ok = mbar_wait_warp(&s_full[t * 2], 0, wc);
            tc_fence_after();
            if (ok) tmem_ld32(lane_at, r[0]);
        }
        for (int it = 0; ok && it < n_it; ++it) {
            const int buf = it & 1;
            float* lt = lb + buf * 64;
            *reinterpret_cast<float2*>(lt + lane * 2) = make_float2(nl[0], nl[1]);
            const bool all = __all_sync(0xffffffffu, nl[0] > -INFINITY && nl[1] > -INFINITY);
            if (it + 1 < n_it) fetch_lse(it + 1, nl);
            __syncwarp();
            tmem_wait_ld(r[0]);
            tmem_ld32(lane_at + buf * 128 + 32, r[1]);
            sum(r[0], lt, all);
            tmem_wait_ld(r[1]);
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&s_empty[t * 2 + buf]);
            if (it + 1 < n_it) {
                ok = mbar_wait_warp(&s_full[t * 2 + (buf ^ 1)], ((it + 1) >> 1) & 1, wc);
                tc_fence_after();
                if (ok) tmem_ld32(lane_at + (buf ^ 1) * 128, r[0]);
            }
            sum(r[1], lt + 32, all);
        }
        total = (s4[0] + s4[1]) + (s4[2] + s4[3]);
        if (half) halves[t * 128 + quarter * 32 + lane] = total;
    }
    tc_fence_before();
    __syncthreads();
    if (warp < kEpilogue && !((warp >> 2) & 1) && !*abort_flag) {
        const int row = (warp >> 3) * 128 + (warp & 3) * 32 + lane, key = key0 + row;
        total += halves[row];
        if (key < a.P) {
            const int64_t o = (int64_t)bh * a.P + key;
            if (a.splits > 1)
                a.part[(int64_t)split * (gridDim.x / a.key_ctas / a.splits) * a.P + o] = total;
            else
                a.acc_out[o] = key < L ? (a.acc_in ? a.beta * a.acc_in[o] : 0.f) + total : 0.f;
        }
    }
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (warp == kEpilogue + 1) {
        __syncwarp();
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
    }
}

// Adds the splits' sums in order.
__global__ void __launch_bounds__(256) weights_join_kernel(const WeightsArgs a, int64_t n) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int64_t o = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (o >= n) return;
    const int j = (int)(o % a.P), b = (int)(o / a.P) / a.Hkv;
    const int L = a.prefix_len ? min(max(a.prefix_len[b], 0), a.P) : a.P;
    float s = 0.f;
    for (int i = 0; i < a.splits; ++i) s += a.part[(int64_t)i * n + o];
    a.acc_out[o] = j < L ? (a.acc_in ? a.beta * a.acc_in[o] : 0.f) + s : 0.f;
}

struct WeightsPlan { int tq, n_qt, key_ctas, splits; };

// Splits of the query rows: only when the key tiles alone leave SMs idle.
WeightsPlan plan_weights(int B, int D, int M, int Hq, int Hkv, int P) {
    WeightsPlan p;
    p.tq = 128 / (Hq / Hkv);
    const int64_t T = (int64_t)D * M;
    p.n_qt = (int)((T + p.tq - 1) / p.tq);
    p.key_ctas = (P + kKeysPerCta - 1) / kKeysPerCta;
    const int64_t ctas = (int64_t)B * Hkv * p.key_ctas;
    int64_t s = sm_count() / ctas;
    if (s > kMaxSplits) s = kMaxSplits;
    if (s > p.n_qt) s = p.n_qt;
    p.splits = s < 1 ? 1 : (int)s;
    return p;
}

template <int SLABS>
int launch_w(const CUtensorMap& mk, const CUtensorMap& mq, const WeightsArgs& a, int64_t grid, cudaStream_t st) {
    constexpr int smem = (2 + kQStages) * SLABS * kSlabBytes + kEpilogue * 2 * 64 * 4 + 1024 + 1024 + 256;
    static_assert(smem <= 227 * 1024, "shared memory of the weights kernel");
    static std::atomic<unsigned long long> set{0};
    if (!ensure_dynamic_smem(weights_tc_kernel<SLABS>, smem, set)) return PSD_ERR_CUDA;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3(kWThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = pdl_enabled() ? 1 : 0;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    cudaError_t e = cudaLaunchKernelEx(&cfg, weights_tc_kernel<SLABS>, mk, mq, a);
    count_launch();
    if (e != cudaSuccess) return PSD_ERR_CUDA;
    if (a.splits > 1) {
        const int64_t n = grid / a.splits / a.key_ctas * a.P;
        cfg.gridDim = dim3((unsigned)((n + 255) / 256));
        cfg.blockDim = dim3(256);
        cfg.dynamicSmemBytes = 0;
        e = cudaLaunchKernelEx(&cfg, weights_join_kernel, a, n);
        count_launch();
    }
    return e == cudaSuccess ? PSD_OK : PSD_ERR_CUDA;
}

}  // namespace

size_t prefix_weights_workspace(int B, int D, int M, int Hq, int Hkv, int Dh, int P) {
    const WeightsPlan p = plan_weights(B, D, M, Hq, Hkv, P);
    return p.splits > 1 ? ((size_t)p.splits * B * Hkv * P * 4 + 255) / 256 * 256 : 256;
}

int launch_prefix_weights(const void* q, const void* k_prefix, const int32_t* prefix_len, const float* lse,
                          const psd_attention_t& a, float beta, const float* acc_in, float* acc_out, void* workspace,
                          int32_t* status_dev, cudaStream_t st) {
    const WeightsPlan p = plan_weights(a.B, a.D, a.M, a.Hq, a.Hkv, a.P);
    const int64_t grid = (int64_t)p.key_ctas * p.splits * a.B * a.Hkv;
    if (grid > INT32_MAX) return PSD_ERR_SHAPE;
    CUtensorMap mk, mq;
    if (!make_cache_map(&mk, k_prefix, a.dtype, a.kp, a.B, a.P, a.Hkv, a.Dh, 128) || !make_query_map(&mq, q, a, p.tq))
        return PSD_ERR_CUDA;
    WeightsArgs w = {prefix_len, lse, acc_in, acc_out, reinterpret_cast<float*>(workspace), status_dev, a.D * a.M, a.Hq / a.Hkv, a.Hq,
                     a.Hkv, a.Dh, a.P, p.tq, p.n_qt, p.key_ctas, p.splits, a.kp.outer ? 1 : 0, a.kp.head ? 1 : 0,
                     a.scale * kLog2e, beta, a.dtype == PSD_BF16 ? 1 : 0, wait_limit_cycles()};
    return a.Dh <= 64 ? launch_w<1>(mk, mq, w, grid, st) : launch_w<2>(mk, mq, w, grid, st);
}

}  // namespace psd
