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
// converts a sum, multiplies it by the column's and the row's scale and folds it; each epilogue warp keeps the columns' scales of its
// tile in shared memory, loaded a tile ahead.  A tile's columns are shared by two groups of four warps: the products of a tile of 128 x 256 take 0.25 us
// for every 128 of H, and the epilogue, a chain of latencies, 7 us with four warps, 2.9 with eight and 2.8 with sixteen, which slow the
// products down (8192 rows, H = 1024: 1.47 ms, 0.79, 0.85; 3537 rows, H = 256: 652 us, 283, 269; 512 rows, H = 4096: 200, 196, 200).
//
// Bound: one pass over W for few rows (half the bytes of a 16-bit head), the tensor cores (twice the 16-bit rate) for many; as
// there, 94 bytes per clock and SM from L2 are what the products need.  Measured (V = 126464, H = 4096): 128 rows 85.8 us, 6.1 TB/s
// (the whole call 89), 8192 rows 3.07-3.15 ms, 2.77 POP/s at the board's power limit (the 16-bit head: 176 us, 6.2 ms).
#include <algorithm>
#include "attn_tc.cuh"
#include "combine.cuh"

namespace psd {
namespace {

constexpr int kSlice = 128;                                    // codes per K-slice
constexpr int kBarriers = 256;
constexpr int kCarry = kCarryEntries * BLOCK_M * 12;
constexpr int kGroups = 2;                                     // of four epilogue warps, each with a share of a tile's columns
constexpr int kThreads = 64 + kGroups * 128;                   // warp 0: TMA, warp 1: MMA and tensor memory
constexpr int kShare = BLOCK_N / kGroups;
constexpr int kScales = 4 * BLOCK_N * 4;                       // the columns' scales, each epilogue warp's
constexpr int kHanded = (kGroups - 1) * BLOCK_M * 12;          // triples of the other groups' shares
constexpr int kSmem = STAGES * STAGE_BYTES + 1024 + kBarriers + kCarry + kScales + kHanded;
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

// A CTA's tiles in the order of TileCursor.  Within a band the next one is found without a division, which each of the epilogue's warps would else wait for
// between tiles (`entry`: which of the band's row tiles that the CTA meets).
struct TileWalk : TileCursor {
    int entry, v, m, e, step_v, step_m, step_e, entries;
    __device__ __forceinline__ void band_begins() {
        if (h <= 0) return;
        v = c / h; m = c - v * h; e = m / gcd;
        step_v = G / h; step_m = G - step_v * h; step_e = step_m / gcd;
        entries = h / gcd;
    }
    __device__ __forceinline__ void begin(const TileGeometry& g, int c_, int G_, int n_mt_) {
        TileCursor::begin(g, c_, G_, n_mt_);
        entry = 0;
        if (g.carry) band_begins();
    }
    __device__ __forceinline__ int next(const TileGeometry& g) {
        if (!g.carry || m0 >= n_mt) return TileCursor::next(g);
        if (v < g.n_vt) {
            v_tile = v; m_tile = m0 + m; entry = e;
            tile_columns(g, v_tile, v0, ncols);
            v += step_v; m += step_m; e += step_e;
            if (m >= h) { m -= h; e -= entries; ++v; }
            return TILE;
        }
        r = h * g.n_vt;
        const int ev = TileCursor::next(g);
        band_begins();
        return ev;
    }
};

// 32 sums of a row, columns col0 .. col0 + n - 1 of them, to logits and into the running triple.  The column of a maximum is not looked for if it is
// no larger than `known`.
__device__ __forceinline__ void fold_sums(const uint32_t (&r)[32], const float* ws, float xs, int col0, int n, float known, float& run_m, float& run_s,
                                          int& run_a) {
    constexpr float LOG2E = 1.4426950408889634f;
    float x[32];
    const f32x2 xs2 = pack2(xs, xs);
#pragma unroll
    for (int j = 0; j < 32; j += 4) {
        const float4 w = *reinterpret_cast<const float4*>(ws + j);
        unpack2(mul2(mul2(pack2(__int2float_rn((int)r[j]), __int2float_rn((int)r[j + 1])), pack2(w.x, w.y)), xs2), x[j], x[j + 1]);
        unpack2(mul2(mul2(pack2(__int2float_rn((int)r[j + 2]), __int2float_rn((int)r[j + 3])), pack2(w.z, w.w)), xs2), x[j + 2], x[j + 3]);
    }
    if (n < 32) {
#pragma unroll
        for (int j = 0; j < 32; ++j)
            if (j >= n) x[j] = -INFINITY;                          // no logits
    }
    float top[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        top[u] = max3(x[8 * u], x[8 * u + 1], x[8 * u + 2]);
        top[u] = max3(top[u], x[8 * u + 3], x[8 * u + 4]);
        top[u] = max3(top[u], x[8 * u + 5], x[8 * u + 6]);
        top[u] = fmaxf(top[u], x[8 * u + 7]);
    }
    const float cm = fmaxf(max3(top[0], top[1], top[2]), top[3]);
    if (cm > run_m) {
        if (cm > known) {
            int at[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                at[u] = 32;
#pragma unroll
                for (int j = 7; j >= 0; --j) at[u] = x[8 * u + j] == cm ? 8 * u + j : at[u];
            }
            run_a = col0 + min(min(at[0], at[1]), min(at[2], at[3]));
        }
        run_s *= ex2((run_m - cm) * LOG2E);
        run_m = cm;
    }
    const f32x2 neg = pack2(-run_m * LOG2E, -run_m * LOG2E), log2e = pack2(LOG2E, LOG2E);
    f32x2 acc[2] = {0ull, 0ull};
#pragma unroll
    for (int j = 0; j < 32; j += 2) acc[j / 2 & 1] = add2(acc[j / 2 & 1], ex2_pair(fma2(pack2(x[j], x[j + 1]), log2e, neg)));
    float a, b;
    unpack2(add2(acc[0], acc[1]), a, b);
    run_s += a + b;
}

__global__ void __launch_bounds__(kThreads, 1)
confidence_q8_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b_wide,
                     const __grid_constant__ CUtensorMap map_b_narrow, const TileGeometry geo, int n_rows, int H, int V,
                     const float* __restrict__ x_scale, const float* __restrict__ w_scale, float* __restrict__ pm,
                     float* __restrict__ ps, int32_t* __restrict__ pa, int32_t* status_dev, size_t part_cap) {
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + STAGES * STAGE_BYTES);
    uint64_t *full_bar = bars, *empty_bar = bars + STAGES, *acc_full_bar = bars + 2 * STAGES, *acc_empty_bar = acc_full_bar + 2,
             *drain_bar = acc_empty_bar + 2, *never_bar = drain_bar + 1, *handed_bar = never_bar + 1, *taken_bar = handed_bar + 4;      // [4]: a quarter of the rows each
    uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(taken_bar + 4);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_holder + 1);
    float* carry_m = reinterpret_cast<float*>(smem + STAGES * STAGE_BYTES + kBarriers);
    float* carry_s = carry_m + kCarryEntries * BLOCK_M;
    int32_t* carry_a = reinterpret_cast<int32_t*>(carry_s + kCarryEntries * BLOCK_M);
    float* scales = reinterpret_cast<float*>(carry_a + kCarryEntries * BLOCK_M);     // [kGroups][4][kShare]
    float* handed_m = scales + 4 * BLOCK_N;                                          // [kGroups - 1][BLOCK_M]
    float* handed_s = handed_m + (kGroups - 1) * BLOCK_M;
    int32_t* handed_a = reinterpret_cast<int32_t*>(handed_s + (kGroups - 1) * BLOCK_M);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int k_blocks = (H + kSlice - 1) / kSlice;          // (the last slice may be half: TMA fills zeros)
    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) { mbar_init(&full_bar[s], 1); mbar_init(&empty_bar[s], 1); }
        for (int a = 0; a < 2; ++a) { mbar_init(&acc_full_bar[a], 1); mbar_init(&acc_empty_bar[a], 4 * kGroups); }
        for (int a = 0; a < 4; ++a) { mbar_init(&handed_bar[a], kGroups - 1); mbar_init(&taken_bar[a], 1); }
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
    TileWalk cur;
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
        // Group g takes the columns from g * share(ncols) on.  Group 0 carries what was before; the others start anew with every tile and hand
        // their triples to group 0.
        const int quarter = warp & 3, row_in_tile = quarter * 32 + lane, group = (warp - 2) >> 2;
        float* ws = scales + (warp - 2) * kShare;
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
        if (geo.carry && group == 0) reset_carry();
        // the next tile's scales come while this one is folded
        auto share = [](int ncols) { return (ncols / kGroups + 31) / 32 * 32; };
        float next_w[kShare / 32], next_x = 0.f;
        auto load_scales = [&]() {
            const int v = cur.v0 + group * share(cur.ncols) + lane, row = cur.m_tile * BLOCK_M + row_in_tile;
#pragma unroll
            for (int u = 0; u < kShare / 32; ++u) next_w[u] = v + u * 32 < V ? w_scale[v + u * 32] : 0.f;
            next_x = row < n_rows ? x_scale[row] : 0.f;
        };
        int in_band = 0;                                  // tiles of this band so far
        int ev = cur.next(geo);
        bool loaded = false;
        while (ev != TileCursor::DONE) {
            if (ev == TileCursor::BAND_END) {
                if (group == 0) {
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
                }
                in_band = 0;
                ev = cur.next(geo);
                continue;
            }
            if (!loaded) load_scales();
            const int v0 = cur.v0, ncols = cur.ncols, acc = it & 1, v_tile = cur.v_tile, row = cur.m_tile * BLOCK_M + row_in_tile;
            const int limit = min(ncols, V - v0), c0 = group * share(ncols), c1 = min(c0 + share(ncols), limit);
            const int entry = cur.entry * BLOCK_M + row_in_tile;
            if (!PSD_DEBUG_OK(cur.m_tile >= 0 && cur.m_tile < n_mt && v0 >= 0 && v0 < V && ncols > 0 && ncols <= BLOCK_N && c1 - c0 <= kShare &&
                                  entry >= 0 && entry < kCarryEntries * BLOCK_M, status_dev)) { ok = false; break; }
            __syncwarp();                                 // the warp is done with the last tile's scales
#pragma unroll
            for (int u = 0; u < kShare / 32; ++u) ws[u * 32 + lane] = next_w[u];
            const float xs = next_x;
            __syncwarp();
            ev = cur.next(geo);
            if ((loaded = ev == TileCursor::TILE)) load_scales();
            if (!mbar_wait(&acc_full_bar[acc], (it >> 1) & 1, wc)) ok = false;
            if (!(ok = __all_sync(0xffffffffu, ok))) break;
            tc_fence_after();
            const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(acc * BLOCK_N);
            float run_m = -INFINITY, run_s = 0.f;
            int run_a = 0;
            if (geo.carry && group == 0) { run_m = carry_m[entry]; run_s = carry_s[entry]; run_a = carry_a[entry]; }
            // What group 0 has carried by now only spares the search for the column of a maximum that will not be one.  It may be as it was two tiles ago, which
            // this accumulator's round trip bears out, and must be of this band.
            const float known = geo.carry && group && in_band >= 2 ? reinterpret_cast<volatile float*>(carry_m)[entry] : -INFINITY;
            ++in_band;
            // (a chunk of 32 columns stays inside the accumulator; what lies behind the tile's columns is masked)
            for (int c = c0; c < c1; c += 32) {
                uint32_t r[32];
                tmem_ld32(taddr + c, r);
                tmem_wait_ld(r);
                fold_sums(r, ws + c - c0, xs, v0 + c, limit - c, known, run_m, run_s, run_a);
            }
            tc_fence_before();
            if (group) {
                const int hand = (group - 1) * BLOCK_M + row_in_tile;
                if (!mbar_wait(&taken_bar[quarter], (it & 1) ^ 1, wc)) ok = false;
                if (!(ok = __all_sync(0xffffffffu, ok))) break;
                handed_m[hand] = run_m; handed_s[hand] = run_s; handed_a[hand] = run_a;
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(&handed_bar[quarter]);
                    mbar_arrive(&acc_empty_bar[acc]);
                }
                ++it;
                continue;
            }
            if (!mbar_wait(&handed_bar[quarter], it & 1, wc)) ok = false;
            if (!(ok = __all_sync(0xffffffffu, ok))) break;
            float other[kGroups - 1], top = run_m;
#pragma unroll
            for (int u = 0; u < kGroups - 1; ++u) {
                other[u] = handed_m[u * BLOCK_M + row_in_tile];
                if (other[u] > top) {                     // (equal maxima: the lower column)
                    top = other[u];
                    run_a = handed_a[u * BLOCK_M + row_in_tile];
                }
            }
            if (run_m != top) run_s *= ex2((run_m - top) * kLog2e);
#pragma unroll
            for (int u = 0; u < kGroups - 1; ++u)
                run_s = fmaf(handed_s[u * BLOCK_M + row_in_tile], other[u] == top ? 1.f : ex2((other[u] - top) * kLog2e), run_s);
            run_m = top;
            if (geo.carry) { carry_m[entry] = run_m; carry_s[entry] = run_s; carry_a[entry] = run_a; }
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(&taken_bar[quarter]);
                mbar_arrive(&acc_empty_bar[acc]);
            }
            if (!geo.carry && row < n_rows && PSD_DEBUG_OK((size_t)v_tile * n_rows + row < part_cap, status_dev)) {
                const size_t o = (size_t)v_tile * n_rows + row;
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
    // Rows that fit a band are read once in either order; in this one they are carried over the vocabulary.
    if (g.n_mt == 1 || (tile_order() == 0 && (long long)g.n_mt * BLOCK_M * H <= band_bytes())) { g.row_bands = 1; g.band = g.n_mt; }
    const int n_tiles = g.n_mt * g.n_vt, grid = n_tiles < sms ? n_tiles : sms;
    // (the height that such bands get: looked for once here, it is at hand for each thread that asks)
    if (g.row_bands) g.band = band_height(grid, g.band, g.band);
    const int wide_rows = (g.rem ? g.base_units + 1 : g.base_units) * 16;
    const int narrow_rows = g.base_units > 0 ? g.base_units * 16 : wide_rows;
    CUtensorMap map_a, map_bw, map_bn;
    // (whole row tiles: x has memory for them.  Rows behind the last are read, whatever they hold, and not used: with the map ending at the last row
    // the pass took 131 us instead of 85 for 4 rows, 98 instead of 88 for 16, V = 126464, H = 4096)
    if (!make_codes_map(&map_a, x, (n_rows + BLOCK_M - 1) / BLOCK_M * BLOCK_M, H, BLOCK_M) || !make_codes_map(&map_bw, w, V, H, wide_rows) ||
        !make_codes_map(&map_bn, w, V, H, narrow_rows))
        return PSD_ERR_CUDA;
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
    cfg.blockDim = dim3(kThreads);
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
