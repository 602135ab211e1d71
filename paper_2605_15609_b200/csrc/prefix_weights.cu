// Attention weight drawn by every prefix key, summed over the rows that read it:
//   sum_r exp(scale * q_r . K_j - lse_r)  =  sum_r 2^(c * q_r . K_j - lse_r log2 e),   c = scale * log2 e.
// The exponent is one FMA in base 2 over the rounded lse_r log2 e and c: a weight's relative error is 2^-24 (|lse_r| + |score|) and
// that of the ex2 instruction, 3e-7 measured where fp32 that subtracts before it scales gives 0.6e-7, at one more
// instruction per score.
//
// The scores are computed transposed, S^T = K Q^T: a tile of 128 keys is the M side of tcgen05.mma and 128 query rows are
// the N side, so a thread of the epilogue (one TMEM lane) owns one KEY and walks the query rows as columns.  The sum over
// rows is then a running sum in a register: no reduction between threads, no atomics, a fixed order.  A CTA keeps two key
// tiles in shared memory and streams the query rows of their key head past both (each query tile is fetched once per 256
// keys), so K is read once and nothing but the sums is written.
//
// CTAs are persistent and take every gridDim-th unit of (256 keys, split of the query rows); tensor memory, barriers and the
// query ring are set up once.  Units are numbered through the sequences' own lengths, so that every CTA gets the same number
// (deep sweep: one CTA per unit 534 us, equal shares of all units 582 us, of the units with keys 448 us).
//
// Warps 0-15 sum: eight per key tile, two per quarter, each with 64 columns of every query tile; warp 16 loads, warp 17
// issues the products.  Accumulators are double-buffered per key tile (4 x 128
// TMEM columns).  One exponential per score is
// what bounds the kernel: 16 per clock and SM, 8 cycles of a scheduler per 32 scores.  (A polynomial in place of part of them
// was measured slower at every share: packed fp32 runs at half the rate of single, so the polynomial costs 10 cycles.)
#include "attn_tc.cuh"

namespace psd {
namespace {

constexpr int kKeysPerCta = 256;
constexpr int kQStages = 4;
constexpr int kEpilogue = 16;           // warps that sum: two per key tile and quarter, 64 columns of a query tile each
constexpr int kWThreads = (kEpilogue + 4) * 32;   // (two idle: register shares go by four warps)
constexpr int kMaxSplits = 16;
constexpr int kMaxSeqs = 256;           // sequences whose keys are counted up front, so that only units with keys are dealt out

struct WeightsArgs {
    const int32_t* prefix_len;
    const float *lse, *acc_in;
    float *acc_out, *part;          // part: [splits][B * Hkv][P] when splits > 1
    int32_t* status_dev;
    int T, G, Hq, Hkv, Dh, P;       // T: tokens per sequence (D * M)
    int tq, n_qt, key_ctas, splits; // tokens per query tile, query tiles, units along the keys, splits of the query tiles
    int bh, units;                  // B * Hkv; all units
    int k_outer, k_head;            // 0: that dimension of the cache is shared
    float c, beta;
    int bf16;
    long long wait_limit;
    int stall_test;                 // PSD_TUNE_SELFTEST_STALL
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
    uint64_t *k_full = bars, *k_empty = k_full + 1, *q_full = k_empty + 1, *q_empty = q_full + kQStages,
             *s_full = q_empty + kQStages /* [2][2] */, *s_empty = s_full + 4, *x_full = s_empty + 4 /* [8] */, *x_empty = x_full + 8 /* [8] */,
             *drain = x_empty + 8, *never = drain + 1 /* nothing arrives on it: self-test of the give-up path */;
    uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(never + 1);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_holder + 1);
    int* ends = const_cast<int*>(abort_flag) + 1;                    // [kMaxSeqs] key units of the sequences up to and with b

    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        mbar_init(k_full, 1);
        mbar_init(k_empty, 1);
        for (int s = 0; s < kQStages; ++s) { mbar_init(&q_full[s], 1); mbar_init(&q_empty[s], 1); }
        for (int s = 0; s < 4; ++s) { mbar_init(&s_full[s], 1); mbar_init(&s_empty[s], 8); }
        for (int s = 0; s < 8; ++s) { mbar_init(&x_full[s], 1); mbar_init(&x_empty[s], 1); }
        mbar_init(drain, 1);
        mbar_init(never, 1);
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

    // a unit: 256 keys from key0 of (b, h), query tiles [q_lo, q_lo + n_it); n_it = 0 when none of its keys is in the prefix
    struct Unit { int b, h, bh, split, key0, L, q_lo, n_it, n_kt; };
    auto length = [&](int b) { return a.prefix_len ? min(max(a.prefix_len[b], 0), a.P) : a.P; };
    // With lengths of their own the sequences' key units are numbered through: unit u = (key unit of all sequences, head, split),
    // and CTAs share out units that have keys, which all cost the same.
    const int n_seq = a.bh / a.Hkv;
    const bool counted = a.prefix_len && n_seq <= kMaxSeqs;
    int n_units = a.units;
    if (counted) {
        for (int i = threadIdx.x; i < n_seq; i += kWThreads) ends[i] = (length(i) + kKeysPerCta - 1) / kKeysPerCta;
        __syncthreads();
        if (warp == 0) {
            int sum = 0;
            for (int i0 = 0; i0 < n_seq; i0 += 32) {
                int run = i0 + lane < n_seq ? ends[i0 + lane] : 0;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int y = __shfl_up_sync(0xffffffffu, run, o);
                    if (lane >= o) run += y;
                }
                if (i0 + lane < n_seq) ends[i0 + lane] = sum + run;
                sum += __shfl_sync(0xffffffffu, run, 31);
            }
        }
        __syncthreads();
        n_units = ends[n_seq - 1] * a.Hkv * a.splits;
    }
    auto unit_at = [&](int u) {
        Unit x;
        int kc;
        if (counted) {
            // key units of a sequence next to each other, then heads, then splits
            const int per = a.Hkv * a.splits, at = u / per;       // (rough place: sequence by key units)
            int lo = 0, hi = n_seq - 1;
            while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                if (ends[mid] > at) hi = mid;
                else lo = mid + 1;
            }
            x.b = lo;
            const int before = lo ? ends[lo - 1] : 0, n = ends[lo] - before, in = u - before * per;
            kc = in % n;
            x.h = in / n % a.Hkv;
            x.split = in / n / a.Hkv;
            x.bh = x.b * a.Hkv + x.h;
        } else {
            kc = u % a.key_ctas;
            const int rest = u / a.key_ctas;
            x.split = rest % a.splits;
            x.bh = rest / a.splits;
            x.b = x.bh / a.Hkv;
            x.h = x.bh - x.b * a.Hkv;
        }
        x.key0 = kc * kKeysPerCta;
        x.L = length(x.b);
        x.q_lo = (int)((long long)a.n_qt * x.split / a.splits);
        x.n_it = x.key0 < x.L ? (int)((long long)a.n_qt * (x.split + 1) / a.splits) - x.q_lo : 0;
        x.n_kt = x.L - x.key0 > 128 ? 2 : 1;
        return x;
    };

    if (warp >= kEpilogue) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
    if (warp == kEpilogue) {
        const bool leader = elect_one();
        const uint32_t q_bytes = (uint32_t)(SLABS * a.tq * a.G * 128);
        int work = 0, qi = 0;                // units with work, and query tiles, so far
        bool ok = true;
#pragma unroll 1
        for (int u = blockIdx.x; ok && u < n_units; u += gridDim.x) {
            const Unit x = unit_at(u);
            if (x.n_it == 0) continue;
            if (!mbar_wait_warp(k_empty, (work & 1) ^ 1, wc)) { ok = false; break; }
            if (leader) {
                mbar_arrive_expect_tx(k_full, x.n_kt * TILE);
                for (int t = 0; t < x.n_kt; ++t)
#pragma unroll
                    for (int s = 0; s < SLABS; ++s)
                        tma_load_4d(k_tiles + t * TILE + s * kSlabBytes, &map_k, k_full, s * kSlabElems, x.h * a.k_head,
                                    x.key0 + t * 128, x.b * a.k_outer);
            }
            ++work;
#pragma unroll 1
            for (int it = 0; it < x.n_it; ++it, ++qi) {
                const int s = qi % kQStages;
                if (!mbar_wait_warp(&q_empty[s], ((qi / kQStages) & 1) ^ 1, wc)) { ok = false; break; }
                if (leader) {
                    mbar_arrive_expect_tx(&q_full[s], q_bytes);
#pragma unroll
                    for (int c = 0; c < SLABS; ++c)
                        tma_load_3d(q_tiles + s * TILE + c * kSlabBytes, &map_q, &q_full[s], c * kSlabElems, x.h * a.G, x.b * a.T + (x.q_lo + it) * a.tq);
                }
                if (a.stall_test && qi == 0 && !mbar_wait_warp(never, 0, wc)) { ok = false; ++qi; break; }
            }
        }
        if (!ok) {
            // giving up: no copy may be in flight when the CTA exits
            for (int i = work > 0 ? work - 1 : 0; i < work; ++i) {
                const long long t0 = clock64();
                while (!mbar_try_wait(k_full, i & 1) && clock64() - t0 < WAIT_LIMIT_CYCLES) {}
            }
            for (int i = qi > kQStages ? qi - kQStages : 0; i < qi; ++i) {
                const long long t0 = clock64();
                while (!mbar_try_wait(&q_full[i % kQStages], (i / kQStages) & 1) && clock64() - t0 < WAIT_LIMIT_CYCLES) {}
            }
        }
    } else if (warp == kEpilogue + 1) {
        const bool leader = elect_one();
        const uint32_t idesc = umma_idesc16(128, a.bf16, false);
        const int k_steps = (a.Dh + 15) / 16;
        const uint64_t dk = umma_smem_desc(smem_u32(k_tiles)), dq = umma_smem_desc(smem_u32(q_tiles));
        int work = 0, qi = 0, done[2] = {0, 0};          // done[t]: accumulators of key tile t filled so far
        bool ok = true;
#pragma unroll 1
        for (int u = blockIdx.x; ok && u < n_units; u += gridDim.x) {
            const Unit x = unit_at(u);
            if (x.n_it == 0) continue;
            if (!(ok = mbar_wait_warp(k_full, work & 1, wc))) break;
            ++work;
#pragma unroll 1
            for (int it = 0; ok && it < x.n_it; ++it, ++qi) {
                const int s = qi % kQStages;
                if (!(ok = mbar_wait_warp(&q_full[s], (qi / kQStages) & 1, wc))) break;
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    if (!ok || t >= x.n_kt) continue;
                    const int buf = done[t] & 1;
                    if (!(ok = mbar_wait_warp(&s_empty[t * 2 + buf], ((done[t] >> 1) & 1) ^ 1, wc))) continue;
                    ++done[t];
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
            if (ok && leader) umma_commit(k_empty);
        }
        if (!ok) {
            if (leader) umma_commit(drain);
            const long long t0 = clock64();
            while (!mbar_try_wait(drain, 0) && clock64() - t0 < WAIT_LIMIT_CYCLES) {}
        }
    }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 104;");
        const int t = warp >> 3, half = (warp >> 2) & 1, quarter = warp & 3, row = quarter * 32 + lane;
        float* lb = lse_buf + warp * 128;
        const uint32_t lane_at = tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(t * 256 + half * 64);
        // This lane's two columns of every query tile: token of the tile (T: none) and offset of its lse.
        int col_tok[2], col_off[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int c = half * 64 + lane * 2 + u;
            col_tok[u] = c < a.tq * a.G ? c / a.G : a.T;
            col_off[u] = c / a.G * a.Hq + c % a.G;
        }
        float s4[4];
        uint32_t r[2][16];
        // Four chunks of 16 columns per tile: while one is summed the next is on its way from tensor memory, across tiles too,
        // so that the exponentials never wait for a load.
        auto sum = [&](const uint32_t (&r)[16], const float* lt, bool all) {
            if (all) {
#pragma unroll
                for (int j = 0; j < 16; j += 4) {
                    const float4 l = *reinterpret_cast<const float4*>(lt + j);
                    s4[0] += ex2(fmaf(__uint_as_float(r[j]), a.c, l.x));
                    s4[1] += ex2(fmaf(__uint_as_float(r[j + 1]), a.c, l.y));
                    s4[2] += ex2(fmaf(__uint_as_float(r[j + 2]), a.c, l.z));
                    s4[3] += ex2(fmaf(__uint_as_float(r[j + 3]), a.c, l.w));
                }
            } else {
                // some columns are absent (what the tile holds there is not used)
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const float l = lt[j];
                    if (l != -INFINITY) s4[0] += ex2(fmaf(__uint_as_float(r[j]), a.c, l));
                }
            }
        };
        if (counted) {
            // keys past a sequence's last unit belong to no unit: 0 (a split's partial sums there are not read)
            for (int64_t o = (int64_t)blockIdx.x * (kEpilogue * 32) + threadIdx.x; o < (int64_t)a.bh * a.P; o += (int64_t)gridDim.x * (kEpilogue * 32)) {
                const int j = (int)(o % a.P), bb = (int)(o / a.P) / a.Hkv;
                if (j >= (ends[bb] - (bb ? ends[bb - 1] : 0)) * kKeysPerCta) a.acc_out[o] = 0.f;
            }
        }
        int done = 0, passed = 0;            // accumulators of this key tile read so far; sums passed between the halves
        bool ok = true;
#pragma unroll 1
        for (int u = blockIdx.x; ok && u < n_units; u += gridDim.x) {
            const Unit x = unit_at(u);
            float total = 0.f;
            if (x.n_it > 0) {
                if (t < x.n_kt) {
                    // -lse * log2 e of the columns of tile `it`; -inf marks a column that adds nothing
                    const float* lse = a.lse + ((int64_t)x.b * a.T + (int64_t)x.q_lo * a.tq) * a.Hq + x.h * a.G;
                    auto fetch_lse = [&](int it, float (&v)[2]) {
#pragma unroll
                        for (int q = 0; q < 2; ++q) {
                            const float l = col_tok[q] + (x.q_lo + it) * a.tq < a.T ? lse[(int64_t)it * a.tq * a.Hq + col_off[q]] : -INFINITY;
                            v[q] = l == -INFINITY ? -INFINITY : -l * kLog2e;
                        }
                    };
                    float nl[2];
                    fetch_lse(0, nl);
                    s4[0] = s4[1] = s4[2] = s4[3] = 0.f;
                    ok = mbar_wait_warp(&s_full[t * 2 + (done & 1)], (done >> 1) & 1, wc);
                    tc_fence_after();
                    if (ok) tmem_ld16(lane_at + (done & 1) * 128, r[0]);
                    for (int it = 0; ok && it < x.n_it; ++it) {
                        const int buf = done & 1;
                        float* lt = lb + buf * 64;
                        *reinterpret_cast<float2*>(lt + lane * 2) = make_float2(nl[0], nl[1]);
                        const bool all = __all_sync(0xffffffffu, nl[0] > -INFINITY && nl[1] > -INFINITY);
                        if (it + 1 < x.n_it) fetch_lse(it + 1, nl);
                        __syncwarp();
                        tmem_wait_ld16(r[0]);
                        tmem_ld16(lane_at + buf * 128 + 16, r[1]);
                        sum(r[0], lt, all);
                        tmem_wait_ld16(r[1]);
                        tmem_ld16(lane_at + buf * 128 + 32, r[0]);
                        sum(r[1], lt + 16, all);
                        tmem_wait_ld16(r[0]);
                        tmem_ld16(lane_at + buf * 128 + 48, r[1]);
                        sum(r[0], lt + 32, all);
                        tmem_wait_ld16(r[1]);
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&s_empty[t * 2 + buf]);
                        ++done;
                        if (it + 1 < x.n_it) {
                            ok = mbar_wait_warp(&s_full[t * 2 + (buf ^ 1)], (done >> 1) & 1, wc);
                            tc_fence_after();
                            if (ok) tmem_ld16(lane_at + (buf ^ 1) * 128, r[0]);
                        }
                        sum(r[1], lt + 48, all);
                    }
                    total = (s4[0] + s4[1]) + (s4[2] + s4[3]);
                }
                // the two halves of a key's columns: the second half hands its sum to the first
                if (ok && t < x.n_kt) {
                    if (half) {
                        ok = mbar_wait_warp(&x_empty[t * 4 + quarter], (passed & 1) ^ 1, wc);
                        halves[t * 128 + row] = total;
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&x_full[t * 4 + quarter]);
                    } else {
                        ok = mbar_wait_warp(&x_full[t * 4 + quarter], passed & 1, wc);
                        total += halves[t * 128 + row];
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&x_empty[t * 4 + quarter]);
                    }
                    ++passed;
                }
            }
            const int key = x.key0 + t * 128 + row;
            if (ok && !half && key < a.P) {
                const int64_t o = (int64_t)x.bh * a.P + key;
                if (a.splits > 1) a.part[(int64_t)x.split * a.bh * a.P + o] = total;
                else a.acc_out[o] = key < x.L ? (a.acc_in ? a.beta * a.acc_in[o] : 0.f) + total : 0.f;
            }
        }
    }
    tc_fence_before();
    __syncthreads();
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
    for (int i = 0; j < L && i < a.splits; ++i) s += a.part[(int64_t)i * n + o];
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
int launch_w(const CUtensorMap& mk, const CUtensorMap& mq, const WeightsArgs& a, cudaStream_t st) {
    constexpr int smem = (2 + kQStages) * SLABS * kSlabBytes + kEpilogue * 2 * 64 * 4 + 1024 + 1024 + 512 + kMaxSeqs * 4;
    static_assert(smem <= 227 * 1024, "shared memory of the weights kernel");
    static std::atomic<unsigned long long> set{0};
    if (!ensure_dynamic_smem(weights_tc_kernel<SLABS>, smem, set)) return PSD_ERR_CUDA;
    static std::atomic<int> regs{0};      // 16 warps of 104 and 4 of 64 registers a thread
    if (!launched_with(weights_tc_kernel<SLABS>, (kEpilogue * 32 * 104 + 128 * 64) / kWThreads, regs)) return PSD_ERR_CUDA;
    cudaLaunchConfig_t cfg = {};
    const int sms = sm_count();
    cfg.gridDim = dim3(a.units < sms ? a.units : sms);
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
        const int64_t n = (int64_t)a.bh * a.P;
        cfg.gridDim = dim3((unsigned)((n + 255) / 256));
        cfg.blockDim = dim3(256);
        cfg.dynamicSmemBytes = 0;
        e = cudaLaunchKernelEx(&cfg, weights_join_kernel, a, n);
        count_launch();
    }
    return e == cudaSuccess ? PSD_OK : PSD_ERR_CUDA;
}

}  // namespace

size_t prefix_weights_needs(int B, int D, int M, int Hq, int Hkv, int P) {
    const WeightsPlan p = plan_weights(B, D, M, Hq, Hkv, P);
    return p.splits > 1 ? ((size_t)p.splits * B * Hkv * P * 4 + 255) / 256 * 256 : 256;
}

// What these sizes and all with smaller B, D, M and P need at most: units of 256 keys are split only while the splits of all of them
// fit the SMs, so a large batch may need nothing where a small one does.
size_t prefix_weights_workspace(int B, int D, int M, int Hq, int Hkv, int P) {
    const int n_qt = plan_weights(B, D, M, Hq, Hkv, P).n_qt;
    if (n_qt == 1) return 256;
    const int64_t most = (int64_t)B * Hkv * P * (n_qt < kMaxSplits ? n_qt : kMaxSplits), once = (int64_t)sm_count() * kKeysPerCta;
    return ((size_t)(most < once ? most : once) * 4 + 255) / 256 * 256;
}

int launch_prefix_weights(const void* q, const void* k_prefix, const int32_t* prefix_len, const float* lse,
                          const psd_attention_t& a, float beta, const float* acc_in, float* acc_out, void* workspace,
                          int32_t* status_dev, cudaStream_t st) {
    const WeightsPlan p = plan_weights(a.B, a.D, a.M, a.Hq, a.Hkv, a.P);
    const int64_t units = (int64_t)p.key_ctas * p.splits * a.B * a.Hkv;
    if (units > INT32_MAX - 1024) return PSD_ERR_SHAPE;
    CUtensorMap mk, mq;
    if (!make_cache_map(&mk, k_prefix, a.dtype, a.kp, a.B, a.P, a.Hkv, a.Dh, 128) || !make_query_map(&mq, q, a, p.tq))
        return PSD_ERR_CUDA;
    WeightsArgs w = {prefix_len, lse, acc_in, acc_out, reinterpret_cast<float*>(workspace), status_dev, a.D * a.M, a.Hq / a.Hkv, a.Hq,
                     a.Hkv, a.Dh, a.P, p.tq, p.n_qt, p.key_ctas, p.splits, a.B * a.Hkv, (int)units, a.kp.outer ? 1 : 0, a.kp.head ? 1 : 0,
                     a.scale * kLog2e, beta, a.dtype == PSD_BF16 ? 1 : 0, wait_limit_cycles(), selftest_stall()};
    return a.Dh <= 64 ? launch_w<1>(mk, mq, w, st) : launch_w<2>(mk, mq, w, st);
}

}  // namespace psd
