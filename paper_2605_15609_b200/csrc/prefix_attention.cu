// Attention of query tiles over the shared prefix, on tcgen05: partial outputs and log-sum-exps, joined with the drafts'
// own keys by draft_attention_kernel.
//
// All query rows of a sequence that share a key head (tokens of all its drafts times the heads of the group) are cut into
// tiles of up to 128 rows; a CTA runs two STREAMS, each with its own tile S of scores (128 rows x 128 keys) and output O
// in tensor memory (4 x 128 columns: all of it).  With two or more tiles the streams take two query tiles over the same
// keys, so every K and V tile in shared memory serves 256 rows; with one tile they take the two halves of the CTA's
// keys.  One warp loads K and V tiles by TMA into a ring, one issues the products, and four warps per stream do the
// softmax: a thread owns a row (TMEM lane), so maxima and sums need no other thread.  While one stream's softmax runs, the tensor cores work on the other stream:
//   .. PV0(j) S0(j+1) | PV1(j) S1(j+1) | PV0(j+1) ..      (S0(j+1) overwrites the scores whose weights PV0(j) just read)
// The weights P overwrite the scores in tensor memory as packed 16-bit pairs and are the A operand of PV, which starts on
// the first half of the weights while the others are computed.
//
// The running maximum is only raised, and O rescaled, when a row's maximum grew by more than 2^8: weights may then be as
// large as 2^8, which costs no accuracy in a floating type, and rescaling O (reading and writing 128 x Dh of tensor
// memory) becomes rare.
//
// Keys past the prefix's end are masked in the scores, and their V rows are zeroed in shared memory before the product,
// since 0 * NaN would spoil a row.
#include "attn_tc.cuh"
#include "prefix_attention.cuh"

namespace psd {
namespace {

constexpr int kPThreads = 384;              // warps 0-3, 4-7: softmax of stream 0, 1; 8: TMA; 9: MMA; 10, 11 idle
constexpr float kRaise = 8.0f;              // growth of a row's maximum (log2) that triggers a rescale

constexpr int kMaxSorted = 128;             // sequences that are put in order of length

template <int SLABS> struct Ring { static constexpr int N = SLABS == 2 ? 5 : 8; };

struct PrefixArgs {
    const int32_t* prefix_len;
    float* po;                 // [splits][R * Hq][DHP] normalised outputs
    float* pl;                 // [splits][R * Hq] log2-sum-exp2
    int32_t* status_dev;
    int64_t rows;              // R * Hq
    int T, G, Hq, Hkv, Dh, P;
    int tq, n_qt, units, splits;   // tokens per tile, tiles per (sequence, key head), CTAs along them, splits written
    int k_outer, k_head, v_outer, v_head;
    int B, longest_first;      // longest_first: CTAs take the sequences by falling length
    float c;                   // scale * log2 e
    int bf16;
    long long wait_limit;
};

__device__ __forceinline__ uint32_t pack16(float lo, float hi, bool bf16) {
    uint32_t r;
    if (bf16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

template <int SLABS, bool BF16>
__global__ void __launch_bounds__(kPThreads, 1)
prefix_attention_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                        const __grid_constant__ CUtensorMap map_v, const PrefixArgs a) {
    extern __shared__ __align__(1024) unsigned char smem[];          // the 128-byte swizzle repeats every 1024 bytes
    constexpr int TILE = SLABS * kSlabBytes, NS = Ring<SLABS>::N, DHP = SLABS * 64;
    unsigned char* q_tiles = smem;                                   // [2][TILE]
    unsigned char* ring = smem + 2 * TILE;                           // [NS][TILE]
    uint64_t* bars = reinterpret_cast<uint64_t*>(ring + NS * TILE);
    uint64_t *q_full = bars, *full = bars + 1, *empty = full + NS, *s_full = empty + NS /* [2] */, *p_half = s_full + 2, *p_ready = p_half + 2,
             *o_done = p_ready + 2 /* [2] */, *drain = o_done + 2;
    uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(drain + 1);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_holder + 1);
    volatile int* sequence = abort_flag + 1;

    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    const bool shared_keys = a.n_qt > 1;          // two query tiles over the same keys
    const int unit = blockIdx.x % a.units;
    const int rest = blockIdx.x / a.units;
    const int n_cs = shared_keys ? a.splits : a.splits / 2;          // CTAs along the keys
    const int cs = rest % n_cs, bh = rest / n_cs;
    const int h = bh % a.Hkv;
    int b = bh / a.Hkv;
    const int qt0 = shared_keys ? unit * 2 : 0;
    const int n_streams = shared_keys ? min(2, a.n_qt - qt0) : 2;

    if (threadIdx.x == 0) {
        mbar_init(q_full, 1);
        for (int s = 0; s < NS; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 1); }
        for (int s = 0; s < 2; ++s) { mbar_init(&s_full[s], 1); mbar_init(&p_half[s], 4); mbar_init(&p_ready[s], 4); mbar_init(&o_done[s], 1); }
        mbar_init(drain, 1);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 8 && lane == 0) { tma_prefetch_desc(&map_q); tma_prefetch_desc(&map_k); tma_prefetch_desc(&map_v); }
    if (warp == 9) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_holder)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, *tmem_holder, 0);
    asm volatile("griddepcontrol.wait;" ::: "memory");

    const WaitCtx wc = {abort_flag, a.status_dev, a.wait_limit, 0u};
    auto length = [&](int i) { return a.prefix_len ? min(max(a.prefix_len[i], 0), a.P) : a.P; };
    if (a.longest_first) {
        // the sequences in order of length, so that the last CTAs to start are short ones
        const int i = threadIdx.x;
        if (i < a.B) {
            const int mine = length(i);
            int rank = 0;
            for (int x = 0; x < a.B; ++x) {
                const int y = length(x);
                rank += y > mine || (y == mine && x < i);
            }
            if (rank == b) *sequence = i;
        }
        __syncthreads();
        b = *sequence;
    }
    const int L = length(b);
    const int tiles = (L + 127) / 128;
    // key tiles [t0, t0 + nt) of each stream: split s of a.splits even shares
    auto share = [&](int x) { return (int)((long long)tiles * x / a.splits); };
    const int sp0 = shared_keys ? cs : cs * 2, sp1 = shared_keys ? cs : cs * 2 + 1;
    const int t00 = share(sp0), t01 = share(sp1);
    const int nt0 = share(sp0 + 1) - t00, nt1 = n_streams > 1 ? share(sp1 + 1) - t01 : 0;
    const int most = max(nt0, nt1);
    const int n_q = shared_keys ? n_streams : 1;                     // query tiles of this CTA

    if (warp >= 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 80;");
        if (warp == 8 && most > 0) {
            // ---------------------------------------------------------------- loader
            const bool leader = elect_one();
            if (leader) {
                mbar_arrive_expect_tx(q_full, (uint32_t)(n_q * SLABS * a.tq * a.G * 128));
                for (int t = 0; t < n_q; ++t)
                    for (int c = 0; c < SLABS; ++c)
                        tma_load_3d(q_tiles + t * TILE + c * kSlabBytes, &map_q, q_full, c * kSlabElems, h * a.G, b * a.T + (qt0 + t) * a.tq);
            }
            int item = 0;
            bool ok = true;
            // per round and list: V of tile j, then K of tile j + 1 (shared keys: stream 0's list serves both streams)
            const int lists = shared_keys ? 1 : 2;
#pragma unroll 1
            for (int x = 0; ok && x < 2 * lists * (most + 1); ++x) {
                const bool is_k = x & 1;
                const int s = lists == 2 ? (x >> 1) & 1 : 0, j = (lists == 2 ? x >> 2 : x >> 1) - (is_k ? 0 : 1);
                if (j < 0 || j >= (s ? nt1 : nt0)) continue;
                const int slot = item % NS;
                if (!mbar_wait_warp(&empty[slot], ((item / NS) & 1) ^ 1, wc)) { ok = false; break; }
                if (leader) {
                    const CUtensorMap* map = is_k ? &map_k : &map_v;
                    const int tile = (s ? t01 : t00) + j;
                    mbar_arrive_expect_tx(&full[slot], TILE);
#pragma unroll
                    for (int c = 0; c < SLABS; ++c)
                        tma_load_4d(ring + slot * TILE + c * kSlabBytes, map, &full[slot], c * kSlabElems,
                                    h * (is_k ? a.k_head : a.v_head), tile * 128, b * (is_k ? a.k_outer : a.v_outer));
                }
                ++item;
            }
            if (!ok) {
                // giving up: no copy may be in flight when the CTA exits
                long long c0 = clock64();
                while (!mbar_try_wait(q_full, 0) && clock64() - c0 < WAIT_LIMIT_CYCLES) {}
                for (int i = item > NS ? item - NS : 0; i < item; ++i) {
                    c0 = clock64();
                    while (!mbar_try_wait(&full[i % NS], (i / NS) & 1) && clock64() - c0 < WAIT_LIMIT_CYCLES) {}
                }
            }
        } else if (warp == 9 && most > 0) {
            // ---------------------------------------------------------------- products
            // One warp issues both streams' products in turn: left to themselves (a warp each) the streams fall into step, and
            // their softmaxes and their products each wait for one another.
            const bool leader = elect_one();
            const uint32_t id_s = umma_idesc16(128, BF16, false);
            const uint32_t id_o = umma_idesc16((a.Dh + 15) / 16 * 16, BF16, true);
            const int k_steps = (a.Dh + 15) / 16;
            const uint64_t dq = umma_smem_desc(smem_u32(q_tiles)), dk = umma_smem_desc(smem_u32(ring));
            const uint64_t dv = umma_smem_desc_mn(smem_u32(ring), kSlabBytes);
            auto wait_item = [&](int item) { return mbar_wait_warp(&full[item % NS], (item / NS) & 1, wc); };
            auto scores = [&](int s, int item, bool release) {
                const uint64_t q = dq + (uint64_t)((shared_keys ? s : 0) * (TILE >> 4)), k = dk + (uint64_t)((item % NS) * (TILE >> 4));
#pragma unroll
                for (int i = 0; i < SLABS * 4; ++i)
                    if (i < k_steps) {
                        const uint64_t off = (i / 4) * (kSlabBytes >> 4) + (i % 4) * 2;
                        umma_f16(tmem + s * 128, q + off, k + off, id_s, i != 0);
                    }
                umma_commit(&s_full[s]);
                if (release) umma_commit(&empty[item % NS]);
            };
            int next = 0;      // ring items, in the loader's order
            bool ok = mbar_wait_warp(q_full, 0, wc);
            int k_of[2] = {-1, -1};
            if (nt0 > 0) k_of[0] = next++;
            if (nt1 > 0) k_of[1] = shared_keys ? 0 : next++;
#pragma unroll
            for (int s = 0; s < 2; ++s)
                if (ok && k_of[s] >= 0 && (ok = wait_item(k_of[s]))) {
                    tc_fence_after();
                    if (leader) scores(s, k_of[s], !shared_keys || s == n_streams - 1);
                }
            int v = 0, k = 0;
#pragma unroll 1
            for (int j = 0; ok && j < most; ++j) {
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    const int n = s ? nt1 : nt0;
                    if (!ok || j >= n) continue;
                    const bool first = !shared_keys || s == 0, last = !shared_keys || s == n_streams - 1, more = j + 1 < n;
                    if (first) {
                        v = next++;
                        k = more ? next++ : v;
                        // the tiles have usually landed long before the weights are ready
                        if (!(ok = wait_item(v) && wait_item(k))) continue;
                    }
                    if (!(ok = mbar_wait_warp(&p_half[s], j & 1, wc))) continue;
                    tc_fence_after();
                    // keys of this tile in steps of 16 (the last tile may hold fewer)
                    const int left = L - ((s ? t01 : t00) + j) * 128, steps = left >= 128 ? 8 : (left + 15) / 16;
                    const uint64_t vd = dv + (uint64_t)((v % NS) * (TILE >> 4));
                    const uint32_t t_s = tmem + s * 128, t_o = t_s + 256;
                    auto pv = [&](int i) {
                        if (i < steps) umma_f16_ts(t_o, t_s + i * 8, vd + (uint64_t)(i * (2048 >> 4)), id_o, (j | i) != 0);
                    };
                    if (leader) { pv(0); pv(1); pv(2); pv(3); }
                    if (!(ok = mbar_wait_warp(&p_ready[s], j & 1, wc))) continue;
                    tc_fence_after();
                    if (leader) {
                        pv(4); pv(5); pv(6); pv(7);
                        // the scores of the next tile overwrite the weights just read; their commit covers PV as well
                        if (more) scores(s, k, last);
                        else umma_commit(&o_done[s]);
                        if (last) umma_commit(&empty[v % NS]);
                    }
                }
            }
            if (!ok) {
                if (leader) umma_commit(drain);
                const long long c0 = clock64();
                while (!mbar_try_wait(drain, 0) && clock64() - c0 < WAIT_LIMIT_CYCLES) {}
            }
        }
        __syncwarp();
    } else {
        // -------------------------------------------------------------------- softmax: stream s, keys [64 half, 64 half + 64), row = lane
        asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
        const int s = warp >> 2, quarter = warp & 3, row = quarter * 32 + lane;
        const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
        const uint32_t t_s = tmem + lanes + s * 128, t_o = tmem + lanes + 256 + s * 128;
        const f32x2 cc = pack2(a.c, a.c);
        float m = 0.f, l = 0.f;
        bool ok = true;
        const int n = s ? nt1 : nt0, first_tile = s ? t01 : t00;
        for (int j = 0; j < n; ++j) {
            if (!(ok = mbar_wait_warp(&s_full[s], j & 1, wc))) break;
            tc_fence_after();
            const int left = L - (first_tile + j) * 128;
            uint32_t r[4][32];
#pragma unroll
            for (int c = 0; c < 4; ++c) tmem_ld32(t_s + c * 32, r[c]);
#pragma unroll
            for (int c = 0; c < 4; ++c) tmem_wait_ld(r[c]);
            if (left < 128) {
#pragma unroll
                for (int c = 0; c < 4; ++c)
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        if (c * 32 + i >= left) r[c][i] = 0xff800000u;
            }
            float u[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                auto x = [&](int i) { return __uint_as_float(r[c][i]); };
                u[c] = max3(x(0), x(1), x(2));
#pragma unroll
                for (int i = 3; i < 31; i += 2) u[c] = max3(u[c], x(i), x(i + 1));
                u[c] = fmaxf(u[c], x(31));
            }
            const float top = fmaxf(max3(u[0], u[1], u[2]), u[3]) * a.c;
            if (j == 0) {
                m = top == -INFINITY ? 0.f : top;
            } else if (__any_sync(0xffffffffu, top > m + kRaise)) {
                const float mn = top > m + kRaise ? top : m;
                const float f = ex2(m - mn);
                m = mn;
                l *= f;
#pragma unroll 1
                for (int c = 0; c < a.Dh; c += 8) {
                    uint32_t o[8];
                    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                                 : "=r"(o[0]), "=r"(o[1]), "=r"(o[2]), "=r"(o[3]), "=r"(o[4]), "=r"(o[5]), "=r"(o[6]), "=r"(o[7])
                                 : "r"(t_o + c));
                    asm volatile("tcgen05.wait::ld.sync.aligned;"
                                 : "+r"(o[0]), "+r"(o[1]), "+r"(o[2]), "+r"(o[3]), "+r"(o[4]), "+r"(o[5]), "+r"(o[6]), "+r"(o[7]) :: "memory");
#pragma unroll
                    for (int i = 0; i < 8; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};"
                                 ::"r"(o[0]), "r"(o[1]), "r"(o[2]), "r"(o[3]), "r"(o[4]), "r"(o[5]), "r"(o[6]), "r"(o[7]), "r"(t_o + c)
                                 : "memory");
                }
            }
            if (left < 128) {
                // V rows past the end that the product's last step of 16 keys reads: zero, whatever the cache holds there (all
                // that share the tile do it: the same zeros)
                int item;
                if (shared_keys) item = 1 + 2 * j;
                else {
                    // items before this V: the first K tiles of both streams, then per round V and next K of each stream
                    item = (nt0 > 0) + (nt1 > 0);
                    for (int q = 0; q < j; ++q) item += (q < nt0) + (q + 1 < nt0) + (q < nt1) + (q + 1 < nt1);
                    if (s == 1) item += (j < nt0) + (j + 1 < nt0);
                }
                if (!(ok = mbar_wait_warp(&full[item % NS], (item / NS) & 1, wc))) break;
                const int stop = (left + 15) / 16 * 16;
                unsigned char* v = ring + (item % NS) * TILE;
                for (int x = left * 8 * SLABS + row; x < stop * 8 * SLABS; x += 128) {
                    const int key = x / (8 * SLABS), ch = x % (8 * SLABS);
                    *reinterpret_cast<uint4*>(v + (ch / 8) * kSlabBytes + key * 128 + (ch % 8) * 16) = make_uint4(0, 0, 0, 0);
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            }
            const f32x2 nm = pack2(-m, -m);
            f32x2 acc[2] = {0ull, 0ull};
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                uint32_t p[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const f32x2 x = fma2(pack2(__uint_as_float(r[c][2 * i]), __uint_as_float(r[c][2 * i + 1])), cc, nm);
                    const f32x2 e = ex2_pair(x);
                    acc[i & 1] = add2(acc[i & 1], e);
                    float y, z;
                    unpack2(e, y, z);
                    p[i] = pack16(y, z, BF16);
                }
                tmem_st16(t_s + c * 16, p);
                if (c == 1 || c == 3) {
                    tmem_wait_st();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(c == 1 ? &p_half[s] : &p_ready[s]);
                }
            }
            float l0, l1;
            unpack2(add2(acc[0], acc[1]), l0, l1);
            l += l0 + l1;
        }
        if (s < n_streams) {
            const int64_t tok0 = (int64_t)b * a.T + (int64_t)(qt0 + (shared_keys ? s : 0)) * a.tq;
            const int64_t tok = tok0 + row / a.G;
            const bool live = row < a.tq * a.G && tok < (int64_t)(b + 1) * a.T;
            const int64_t at = (int64_t)(s ? sp1 : sp0) * a.rows + tok * a.Hq + h * a.G + row % a.G;
            if (ok && n > 0) {
                ok = mbar_wait_warp(&o_done[s], 0, wc);
                tc_fence_after();
                if (ok) {
                    const float inv = 1.0f / l;
                    float* o = a.po + at * DHP;
#pragma unroll 1
                    for (int c = 0; c < a.Dh; c += 32) {
                        uint32_t x[32];
                        tmem_ld32(t_o + c, x);
                        tmem_wait_ld(x);
                        if (live) {
#pragma unroll
                            for (int i = 0; i < 32; i += 8)
                                asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(o + c + i),
                                             "f"(__uint_as_float(x[i]) * inv), "f"(__uint_as_float(x[i + 1]) * inv),
                                             "f"(__uint_as_float(x[i + 2]) * inv), "f"(__uint_as_float(x[i + 3]) * inv),
                                             "f"(__uint_as_float(x[i + 4]) * inv), "f"(__uint_as_float(x[i + 5]) * inv),
                                             "f"(__uint_as_float(x[i + 6]) * inv), "f"(__uint_as_float(x[i + 7]) * inv) : "memory");
                        }
                    }
                }
            }
            if (live && ok) a.pl[at] = n > 0 ? m + log2f(l) : -INFINITY;
        }
    }
    tc_fence_before();
    __syncthreads();
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (warp == 9) {
        __syncwarp();
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
    }
}

template <int SLABS, bool BF16>
int launch_p(const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv, const PrefixArgs& a, int64_t grid, cudaStream_t st) {
    constexpr int smem = (2 + Ring<SLABS>::N) * SLABS * kSlabBytes + 256;
    static_assert(smem <= 227 * 1024, "shared memory of the prefix kernel");
    static std::atomic<unsigned long long> set{0};
    if (!ensure_dynamic_smem(prefix_attention_kernel<SLABS, BF16>, smem, set)) return PSD_ERR_CUDA;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3(kPThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = pdl_enabled() ? 1 : 0;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, prefix_attention_kernel<SLABS, BF16>, mq, mk, mv, a);
    count_launch();
    return e == cudaSuccess ? PSD_OK : PSD_ERR_CUDA;
}

}  // namespace

// How the prefix's keys are split.  A CTA takes two query tiles (or the only one twice, over two ranges of keys); when
// (sequence, key head, tile pair) alone leaves SMs idle the keys are split, down to kMinTiles tiles of 128 keys per split.
PrefixPlan plan_prefix(int B, int D, int M, int Hq, int Hkv, int Dh, int P) {
    constexpr int kMinTiles = 2;
    PrefixPlan p = {};
    p.tq = 128 / (Hq / Hkv);
    p.n_qt = (int)(((int64_t)D * M + p.tq - 1) / p.tq);
    p.units = p.n_qt > 1 ? (p.n_qt + 1) / 2 : 1;
    const int tiles = (P + 127) / 128;
    const int64_t ctas = (int64_t)B * Hkv * p.units;
    int64_t s = sm_count() / ctas;
    const int per = p.n_qt > 1 ? 1 : 2;                 // splits a CTA writes
    if (s * per > tiles / kMinTiles) s = tiles / kMinTiles / per;
    if (s * per > kMaxPrefixSplits) s = kMaxPrefixSplits / per;
    if (s < 1) s = 1;
    p.splits = (int)s * per;
    p.dhp = Dh <= 64 ? 64 : 128;
    return p;
}

int launch_prefix_attention(const void* q, const void* k, const void* v, const int32_t* prefix_len, const psd_attention_t& a,
                            const PrefixPlan& p, float* po, float* pl, int32_t* status_dev, cudaStream_t st) {
    CUtensorMap mq, mk, mv;
    if (!make_query_map(&mq, q, a, p.tq) || !make_cache_map(&mk, k, a.dtype, a.kp, a.B, a.P, a.Hkv, a.Dh, 128) ||
        !make_cache_map(&mv, v, a.dtype, a.vp, a.B, a.P, a.Hkv, a.Dh, 128))
        return PSD_ERR_CUDA;
    const int64_t grid = (int64_t)a.B * a.Hkv * p.units * (p.n_qt > 1 ? p.splits : p.splits / 2);
    if (grid > INT32_MAX) return PSD_ERR_SHAPE;
    const bool bf16 = a.dtype == PSD_BF16;
    PrefixArgs x = {prefix_len, po, pl, status_dev, (int64_t)a.B * a.D * a.M * a.Hq, a.D * a.M, a.Hq / a.Hkv, a.Hq, a.Hkv, a.Dh, a.P,
                    p.tq, p.n_qt, p.units, p.splits, a.kp.outer ? 1 : 0, a.kp.head ? 1 : 0, a.vp.outer ? 1 : 0, a.vp.head ? 1 : 0,
                    a.B, prefix_len && a.B > 1 && a.B <= kMaxSorted && grid > sm_count() ? 1 : 0,
                    a.scale * kLog2e, bf16 ? 1 : 0, wait_limit_cycles()};
    if (p.dhp == 64) return bf16 ? launch_p<1, true>(mq, mk, mv, x, grid, st) : launch_p<1, false>(mq, mk, mv, x, grid, st);
    return bf16 ? launch_p<2, true>(mq, mk, mv, x, grid, st) : launch_p<2, false>(mq, mk, mv, x, grid, st);
}

}  // namespace psd
