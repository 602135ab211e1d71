// Fused LM-head + confidence kernel over an 8-bit head: hidden rows in codes with a scale each, W in codes with a scale for
// each vocabulary row.
//
//   l[r, v] = fp32(fp32(fp32(sum_j x[r, j] w[v, j]) * w_scale[v]) * x_scale[r]),   x^ = argmax_v l, c = softmax(l)[x^]
//
// The integer sums are exact, so the logits and the token are one number for every order of summing.
//
// The kernel is built as the 16-bit one is (one CTA per SM over a list of tiles of 128 rows x up to 256 vocabulary rows, TMA
// ring, one issuing thread, epilogue out of tensor memory, carried triples); a K-slice is again one 128-byte swizzle row, which
// here is 128 codes, and the product is kind::i8 (M 128, N the tile's width, K 32, 32-bit integer accumulators).  The epilogue
// converts a sum, multiplies it by the column's and the row's scale and folds it as there; each epilogue warp keeps the
// columns' scales of its tile in shared memory.
//
// Bound: one pass over W for few rows (half the bytes of a 16-bit head), the tensor cores (twice the 16-bit rate) for many; as
// there, 94 bytes per clock and SM from L2 are what the products need.  Measured (V = 126464, H = 4096): 128 rows 85.8 us, 6.1 TB/s
// (the whole call 89), 8192 rows 3.07-3.1 ms, 2.77 POP/s at the board's power limit (the 16-bit head: 176 us, 6.2 ms).
#include <algorithm>
#include "attn_tc.cuh"
#include "combine.cuh"

namespace psd {
namespace {

constexpr int kSlice = 128;                                    // codes per K-slice
constexpr int kBarriers = 256;
constexpr int kCarry = kCarryEntries * BLOCK_M * 12;
constexpr int kScales = 4 * BLOCK_N * 4;                       // the columns' scales, a copy per epilogue warp
constexpr int kSmem = STAGES * STAGE_BYTES + 1024 + kBarriers + kCarry + kScales;
static_assert(kSmem <= 227 * 1024, "shared memory of the 8-bit kernel");

// kind::i8: signed 8-bit A and B, 32-bit integer accumulator, both K-major, M = 128, N = n
__device__ __forceinline__ uint32_t idesc_i8(int n) {
    return (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(BLOCK_M >> 4) << 24);
}
__device__ __forceinline__ void umma_i8(uint32_t tmem_d, uint64_t desc_a, uint64_t desc_b, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(tmem_d), "l"(desc_a), "l"(desc_b), "r"(idesc), "r"(accumulate) : "memory");
}

__global__ void __launch_bounds__(NUM_THREADS, 1)
confidence_q8_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b_wide,
                     const __grid_constant__ CUtensorMap map_b_narrow, const TileGeometry geo, int n_rows, int H, int V,
                     const float* __restrict__ x_scale, const float* __restrict__ w_scale, float* __restrict__ pm,
                     float* __restrict__ ps, int32_t* __restrict__ pa, int32_t* status_dev, size_t part_cap) {
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + STAGES * STAGE_BYTES);
    uint64_t *full_bar = bars, *empty_bar = bars + STAGES, *acc_full_bar = bars + 2 * STAGES, *acc_empty_bar = acc_full_bar + 2,
             *drain_bar = acc_empty_bar + 2, *never_bar = drain_bar + 1;
    uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(never_bar + 1);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_holder + 1);
    float* carry_m = reinterpret_cast<float*>(smem + STAGES * STAGE_BYTES + kBarriers);
    float* carry_s = carry_m + kCarryEntries * BLOCK_M;
    int32_t* carry_a = reinterpret_cast<int32_t*>(carry_s + kCarryEntries * BLOCK_M);
    float* scales = reinterpret_cast<float*>(carry_a + kCarryEntries * BLOCK_M);     // [4][BLOCK_N]

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int k_blocks = (H + kSlice - 1) / kSlice;          // (the last slice may be half: TMA fills zeros)
    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) { mbar_init(&full_bar[s], 1); mbar_init(&empty_bar[s], 1); }
        for (int a = 0; a < 2; ++a) { mbar_init(&acc_full_bar[a], 1); mbar_init(&acc_empty_bar[a], 4); }
        mbar_init(drain_bar, 1);
        mbar_init(never_bar, 1);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0 && lane == 0) { tma_prefetch_desc(&map_a); tma_prefetch_desc(&map_b_wide); tma_prefetch_desc(&map_b_narrow); }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_holder)), "r"(TMEM_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_holder;
    asm volatile("griddepcontrol.wait;" ::: "memory");        // the rows' codes come from the kernel ahead

    const int n_mt = geo.n_mt;
    const WaitCtx wc = {abort_flag, status_dev, geo.wait_limit, 0u};
    TileCursor cur;
    cur.begin(geo, blockIdx.x, gridDim.x, n_mt);

    if (warp == 0) {
        if (lane == 0) {
            // L2: W passes once for one row tile and leaves first; otherwise both operands are read again within a band
            const uint64_t pol_w = geo.n_mt == 1 ? l2_policy_evict_first() : l2_policy_evict_last();
            const uint64_t pol_h = l2_policy_evict_last();
            // One row tile: the CTAs begin at different slices (integer sums: any order), since a slice of few rows is a few lines of memory, for
            // which all of them would ask at once.
            const int turn = geo.n_mt == 1 ? (int)((long long)blockIdx.x * k_blocks / gridDim.x) : 0;
            int q = 0;
            bool ok = true;
            for (int ev; ok && (ev = cur.next(geo)) != TileCursor::DONE;) {
                if (ev != TileCursor::TILE) continue;
                const CUtensorMap* mb = cur.v_tile < geo.rem || geo.rem == 0 ? &map_b_wide : &map_b_narrow;
                const uint32_t bytes = A_BYTES + (uint32_t)cur.ncols * kSlice;
                for (int kb = 0; kb < k_blocks; ++kb, ++q) {
                    const int s = q % STAGES;
                    if (!mbar_wait(&empty_bar[s], ((q / STAGES) & 1) ^ 1, wc)) { ok = false; break; }
                    unsigned char* sa = smem + s * STAGE_BYTES;
                    const int k0 = (kb + turn < k_blocks ? kb + turn : kb + turn - k_blocks) * kSlice;
                    mbar_arrive_expect_tx(&full_bar[s], bytes);
                    tma_load_2d(sa, &map_a, &full_bar[s], k0, cur.m_tile * BLOCK_M, pol_h);
                    tma_load_2d(sa + A_BYTES, mb, &full_bar[s], k0, cur.v0, pol_w);
                    if (geo.stall_test && q == 0 && !mbar_wait(never_bar, 0, wc)) { ok = false; ++q; break; }
                }
            }
            if (!ok)        // giving up: no copy may be in flight when the CTA exits
                for (int i = q > STAGES ? q - STAGES : 0; i < q; ++i) {
                    const long long t0 = clock64();
                    while (!mbar_try_wait(&full_bar[i % STAGES], (i / STAGES) & 1) && clock64() - t0 < WAIT_LIMIT_CYCLES) {}
                }
        }
    } else if (warp == 1) {
        if (lane == 0) {
            int q = 0, it = 0;
            bool ok = true;
            for (int ev; ok && (ev = cur.next(geo)) != TileCursor::DONE;) {
                if (ev != TileCursor::TILE) continue;
                const int acc = it & 1;
                if (!mbar_wait(&acc_empty_bar[acc], ((it >> 1) & 1) ^ 1, wc)) { ok = false; break; }
                tc_fence_after();
                const uint32_t idesc = idesc_i8(cur.ncols), tmem_d = tmem_base + (uint32_t)(acc * BLOCK_N);
                for (int kb = 0; kb < k_blocks; ++kb, ++q) {
                    const int s = q % STAGES;
                    if (!mbar_wait(&full_bar[s], (q / STAGES) & 1, wc)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t a_addr = smem_u32(smem + s * STAGE_BYTES);
                    const uint64_t da = umma_smem_desc(a_addr), db = umma_smem_desc(a_addr + A_BYTES);
#pragma unroll
                    for (int k = 0; k < 4; ++k)      // 32 codes = 32 bytes inside the swizzle row: +2 in 16-byte units
                        umma_i8(tmem_d, da + (uint64_t)(k * 2), db + (uint64_t)(k * 2), idesc, (kb | k) != 0);
                    umma_commit(&empty_bar[s]);
                }
                if (ok) umma_commit(&acc_full_bar[acc]);
                ++it;
            }
            if (!ok) {
                umma_commit(drain_bar);
                const long long t0 = clock64();
                while (!mbar_try_wait(drain_bar, 0) && clock64() - t0 < WAIT_LIMIT_CYCLES) {}
            }
        }
    } else {
        const int quarter = warp & 3, row_in_tile = quarter * 32 + lane;
        float* ws = scales + quarter * BLOCK_N;
        int it = 0;
        bool ok = true;
        auto reset_carry = [&]() {
#pragma unroll
            for (int e = 0; e < kCarryEntries; ++e) {
                carry_m[e * BLOCK_M + row_in_tile] = -INFINITY;
                carry_s[e * BLOCK_M + row_in_tile] = 0.f;
                carry_a[e * BLOCK_M + row_in_tile] = 0;
            }
        };
        if (geo.carry) reset_carry();
        for (int ev; ok && (ev = cur.next(geo)) != TileCursor::DONE;) {
            if (ev == TileCursor::BAND_END) {
                const int entries = cur.end_h / cur.end_gcd;
                const int slot = (int)blockIdx.x / cur.end_gcd, base = (int)blockIdx.x % cur.end_gcd;
                for (int e = 0; e < entries; ++e) {
                    const int row = (cur.end_m0 + base + e * cur.end_gcd) * BLOCK_M + row_in_tile;
                    if (row < n_rows && PSD_DEBUG_OK((size_t)slot * n_rows + row < part_cap && e < kCarryEntries, status_dev)) {
                        const size_t o = (size_t)slot * n_rows + row;
                        pm[o] = carry_m[e * BLOCK_M + row_in_tile];
                        ps[o] = carry_s[e * BLOCK_M + row_in_tile];
                        pa[o] = carry_a[e * BLOCK_M + row_in_tile];
                    }
                }
                reset_carry();
                continue;
            }
            const int v0 = cur.v0, ncols = cur.ncols, acc = it & 1, row = cur.m_tile * BLOCK_M + row_in_tile;
            __syncwarp();                                 // the warp is done with the last tile's scales
            for (int c = lane; c < ncols; c += 32) ws[c] = v0 + c < V ? w_scale[v0 + c] : 0.f;
            const float xs = row < n_rows ? x_scale[row] : 0.f;
            __syncwarp();
            if (!mbar_wait(&acc_full_bar[acc], (it >> 1) & 1, wc)) ok = false;
            if (!(ok = __all_sync(0xffffffffu, ok))) break;
            tc_fence_after();
            const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(acc * BLOCK_N);
            const int entry = geo.carry ? ((cur.m_tile - cur.m0) / cur.gcd) * BLOCK_M + row_in_tile : 0;
            if (!PSD_DEBUG_OK(cur.m_tile >= 0 && cur.m_tile < n_mt && v0 >= 0 && v0 < V && ncols > 0 && ncols <= BLOCK_N &&
                                  entry >= 0 && entry < kCarryEntries * BLOCK_M, status_dev)) { ok = false; break; }
            float run_m = -INFINITY, run_s = 0.f;
            int run_a = 0;
            if (geo.carry) { run_m = carry_m[entry]; run_s = carry_s[entry]; run_a = carry_a[entry]; }
            const bool ragged = v0 + ncols > V;
            for (int c = 0; c < ncols; c += 32) {
                uint32_t r[32];
                float x[32];
                const bool whole = ncols - c >= 32;
                if (whole) {
                    tmem_ld32(taddr + c, r);
                    tmem_wait_ld(r);
                } else {
                    uint32_t h[16];
                    tmem_ld16(taddr + c, h);
                    tmem_wait_ld16(h);
#pragma unroll
                    for (int j = 0; j < 16; ++j) { r[j] = h[j]; r[16 + j] = 0; }
                }
#pragma unroll
                for (int j = 0; j < 32; ++j) x[j] = __fmul_rn(__fmul_rn(__int2float_rn((int)r[j]), ws[(c + j) & (BLOCK_N - 1)]), xs);
                if (ragged || !whole) {
#pragma unroll
                    for (int j = 0; j < 32; ++j)
                        if (v0 + c + j >= V || c + j >= ncols) x[j] = -INFINITY;     // no logits
                }
                fold_chunk(x, v0 + c, run_m, run_s, run_a);
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&acc_empty_bar[acc]);
            if (geo.carry) {
                carry_m[entry] = run_m; carry_s[entry] = run_s; carry_a[entry] = run_a;
            } else if (row < n_rows && PSD_DEBUG_OK((size_t)cur.v_tile * n_rows + row < part_cap, status_dev)) {
                const size_t o = (size_t)cur.v_tile * n_rows + row;
                pm[o] = run_m;
                ps[o] = run_s;
                pa[o] = run_a;
            }
            ++it;
        }
    }
    tc_fence_before();
    __syncthreads();
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (warp == 1) {
        __syncwarp();
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(TMEM_COLS) : "memory");
    }
}

// Joins the triples of few rows, a warp per row and lanes along the splits, all loads issued together: combine_kernel's 8 threads per row
// would walk 19 of 148 splits each, one after the other (10 us for 128 rows, against 5).  Equal maxima keep the lower index, sums that hold a NaN stay NaN.
constexpr int kJoinRows = 2048;
__global__ void __launch_bounds__(128) join_triples_kernel(const float* __restrict__ pm, const float* __restrict__ ps, const int32_t* __restrict__ pa,
                                                           const SplitPlan plan, int n_rows, int32_t* __restrict__ out_token, float* __restrict__ out_conf,
                                                           float* __restrict__ out_lse, int32_t* status_dev) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int row = blockIdx.x * 4 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (row >= n_rows) return;
    const int n = plan.uniform > 0 ? plan.uniform : carried_splits(plan.G, plan.hb, (n_rows + plan.tile_rows - 1) / plan.tile_rows, row / plan.tile_rows);
    constexpr int kBatch = 5;
    float m = -INFINITY, s = 0.f;
    int32_t a = INT32_MAX;
    for (int j0 = lane; j0 < n; j0 += 32 * kBatch) {
        float bm[kBatch], bs[kBatch];
        int32_t ba[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const int j = j0 + 32 * u;
            const size_t o = (size_t)j * n_rows + row;
            bm[u] = j < n ? pm[o] : -INFINITY;
            bs[u] = j < n ? ps[o] : 0.f;
            ba[u] = j < n ? pa[o] : INT32_MAX;
        }
        float top = m;
#pragma unroll
        for (int u = 0; u < kBatch; ++u) top = fmaxf(top, bm[u]);
        const float base = top == -INFINITY ? 0.f : top;
        s *= expf(m - base);
        if (m != top) a = INT32_MAX;
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            s = fmaf(bs[u], expf(bm[u] - base), s);
            if (bm[u] == top) a = min(a, ba[u]);
        }
        m = top;
    }
    float top = m;
#pragma unroll
    for (int x = 16; x; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
    s *= expf(m - (top == -INFINITY ? 0.f : top));
    if (m != top) a = INT32_MAX;
#pragma unroll
    for (int x = 16; x; x >>= 1) {
        s += __shfl_xor_sync(0xffffffffu, s, x);
        a = min(a, __shfl_xor_sync(0xffffffffu, a, x));
    }
    if (lane == 0) {
        out_token[row] = a;
        out_conf[row] = 1.0f / s;
        if (out_lse) out_lse[row] = top + logf(s);
        if (status_dev && !(isfinite(top) && isfinite(s))) count_nonfinite_row(status_dev);
    }
}

// A [rows, H] matrix of codes, boxes of 128 x box_rows, 128-byte swizzle, zeros outside.
bool make_codes_map(CUtensorMap* m, const void* base, int rows, int H, int box_rows) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    cuuint64_t dims[2] = {(cuuint64_t)H, (cuuint64_t)rows};
    cuuint64_t strides[1] = {(cuuint64_t)H};
    cuuint32_t box[2] = {(cuuint32_t)kSlice, (cuuint32_t)box_rows};
    cuuint32_t estr[2] = {1, 1};
    return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace

int launch_confidence_q8(const int8_t* x, const float* x_scale, const int8_t* w, const float* w_scale, int n_rows, int H, int V,
                         Partials part, int32_t* status_dev, cudaStream_t st, SplitPlan* plan) {
    static std::atomic<unsigned long long> smem_set{0};
    if (!ensure_dynamic_smem(confidence_q8_kernel, kSmem, smem_set)) return PSD_ERR_CUDA;
    const int sms = sm_count();
    TileGeometry g = choose_geometry(n_rows, V, sms, max_splits(V), BLOCK_M, 16);
    choose_order(g, n_rows, (H + 1) / 2, V, BLOCK_M, band_bytes(), tile_order());     // (rows of H bytes)
    if (g.n_mt == 1) { g.row_bands = 1; g.band = 1; }
    const int wide_rows = (g.rem ? g.base_units + 1 : g.base_units) * 16;
    const int narrow_rows = g.base_units > 0 ? g.base_units * 16 : wide_rows;
    CUtensorMap map_a, map_bw, map_bn;
    // (whole row tiles: x has memory for them.  Rows behind the last are read, whatever they hold, and not used: with the map ending at the last row
    // the pass took 131 us instead of 85 for 4 rows, 98 instead of 88 for 16, V = 126464, H = 4096)
    if (!make_codes_map(&map_a, x, (n_rows + BLOCK_M - 1) / BLOCK_M * BLOCK_M, H, BLOCK_M) || !make_codes_map(&map_bw, w, V, H, wide_rows) ||
        !make_codes_map(&map_bn, w, V, H, narrow_rows))
        return PSD_ERR_CUDA;
    const int n_tiles = g.n_mt * g.n_vt, grid = n_tiles < sms ? n_tiles : sms;
    int most_splits = 0;
    for (int m0 = 0; m0 < g.n_mt;) {
        const int h = band_height(grid, g.band, g.n_mt - m0);
        most_splits = std::max(most_splits, grid / gcd_int(grid, h));
        m0 += h;
    }
    // carried triples: where they leave fewer than one per vocabulary tile (which the workspace is sized for)
    g.carry = (g.row_bands && most_splits <= g.n_vt) ? 1 : 0;
    if (g.carry) *plan = SplitPlan{0, grid, g.band, BLOCK_M, n_rows, nullptr};
    else *plan = uniform_splits(g.n_vt);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(NUM_THREADS);
    cfg.dynamicSmemBytes = kSmem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = pdl_enabled() ? 1 : 0;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, confidence_q8_kernel, map_a, map_bw, map_bn, g, n_rows, H, V, x_scale, w_scale, part.m,
                                             part.s, part.a, status_dev, part.cap);
    count_launch();
    return e == cudaSuccess ? PSD_OK : PSD_ERR_CUDA;
}

int launch_join_triples(Partials part, const SplitPlan& plan, int n_rows, int32_t* out_token, float* out_conf, float* out_lse, int32_t* status_dev,
                        cudaStream_t st) {
    if (n_rows > kJoinRows) return launch_combine(part, plan, n_rows, out_token, out_conf, out_lse, st, nullptr, nullptr, 0, status_dev);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((n_rows + 3) / 4);
    cfg.blockDim = dim3(128);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = pdl_enabled() ? 1 : 0;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, join_triples_kernel, (const float*)part.m, (const float*)part.s, (const int32_t*)part.a, plan, n_rows,
                                             out_token, out_conf, out_lse, status_dev);
    count_launch();
    return e == cudaSuccess ? PSD_OK : PSD_ERR_CUDA;
}

}  // namespace psd
