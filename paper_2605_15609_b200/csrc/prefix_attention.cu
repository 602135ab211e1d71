// Attention of query tiles over the shared prefix (and, with many rows, the drafts' own keys), on tcgen05.
//
// All query rows of a sequence that share a key head (tokens of all its drafts times the heads of the group) are cut into
// tiles of up to 128 rows; a CTA runs two STREAMS, each with its own tile S of scores (128 rows x 128 keys) and output O
// in tensor memory (4 x 128 columns: all of it).  With two or more tiles the streams take two query tiles over the same
// keys, so every K and V tile in shared memory serves 256 rows; with one tile they take the two halves of the CTA's
// keys.  One warp loads K and V tiles by TMA into a ring, one issues the products, and four warps per stream do the
// softmax: a thread owns a row (TMEM lane), so maxima and sums need no other thread.  While one stream's softmax runs, the
// tensor cores work on the other stream:
//   .. PV0(j) S0(j+1) | PV1(j) S1(j+1) | PV0(j+1) ..      (S0(j+1) overwrites the scores whose weights PV0(j) just read)
// The weights P overwrite the scores in tensor memory as packed 16-bit pairs and are the A operand of PV, which starts on
// the first half of the weights while the others are computed.
//
// The running maximum is only raised, and O rescaled, when a row's maximum grew by more than 2^8: weights may then be as
// large as 2^8, which costs no accuracy in a floating type, and rescaling O (reading and writing 128 x Dh of tensor
// memory) becomes rare.  In fp16 weights are kept 2^7 larger still, up to 2^15 of its 2^16: it holds nothing below 2^-25,
// and thousands of keys that far below a row's maximum count together (4000 keys 2^-26.7 below it were nearly all lost otherwise,
// 3.7e-5 of the output); a weight is then off by 2^-32 of the maximum at most.
//
// Where the prefix is not split (many rows), the drafts' own keys follow it in the same kernel as further tiles of the list,
// one draft at a time: its products leave the rows of other drafts as they are (a mask of tensor-memory rows), so what one
// draft's keys and values hold cannot reach another, and the CTA writes final outputs.  Otherwise partial results go to
// draft_attention_kernel, which takes the own keys and joins.
//
// Bound, for Dh = 128, by products and exponentials alike (2048 cycles each per 256 rows x 128 keys); measured 3500 cycles, the
// chain scores -> softmax -> weights -> product of a stream: 16 sequences x 8 key heads x 2048 rows over up to 8192 keys (mean 0.63
// of that, 705 GFLOP) in 705 us, 1.0 PFLOP/s (0.96-1.0 over seeds of mean 0.56-0.66, 635-760 us), where the board's power limit
// already holds the clock at 1840-1900 MHz.
//
// Keys past the prefix's end are masked in the scores, and their V rows are zeroed in shared memory before the product,
// since 0 * NaN would spoil a row.
#include "attn_tc.cuh"
#include "prefix_attention.cuh"

namespace psd {
namespace {

constexpr int kPThreads = 384;              // warps 0-3, 4-7: softmax of stream 0, 1; 8: TMA; 9: MMA; 10, 11 idle
constexpr float kRaise = 8.0f;              // growth of a row's maximum (log2) that triggers a rescale
constexpr float kHalfRoom = 7.0f;           // fp16: how far (log2) the reference is set below the maximum

constexpr int kMaxSorted = 128;             // sequences that are put in order of length
constexpr int kBarBytes = 1024;             // barriers, flags and the lists of own tiles

struct OwnTile { int node, key0, len; };    // a tile of own keys: draft of the sequence, first key, the draft's length

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
    // own keys and final outputs (fused == 1); else partial results
    int fused, D, M, S, causal, own_box;
    int ko_outer, ko_head, vo_outer, vo_head;
    const int32_t* own_len;
    void* out;
    float* lse;
    int64_t out_token, out_head;
    float c;                   // scale * log2 e
    long long wait_limit;
    int stall_test;            // PSD_TUNE_SELFTEST_STALL
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
                        const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CUtensorMap map_ko,
                        const __grid_constant__ CUtensorMap map_vo, const PrefixArgs a) {
    extern __shared__ __align__(1024) unsigned char smem[];          // the 128-byte swizzle repeats every 1024 bytes
    constexpr int TILE = SLABS * kSlabBytes, NS = Ring<SLABS>::N, DHP = SLABS * 64;
    unsigned char* q_tiles = smem;                                   // [2][TILE]
    unsigned char* ring = smem + 2 * TILE;                           // [NS][TILE]
    uint64_t* bars = reinterpret_cast<uint64_t*>(ring + NS * TILE);
    uint64_t *q_full = bars, *full = bars + 1, *empty = full + NS, *s_full = empty + NS /* [2] */, *p_half = s_full + 2, *p_ready = p_half + 2,
             *o_done = p_ready + 2 /* [2] */, *drain = o_done + 2,
             *never = drain + 1 /* nothing arrives on it: self-test of the give-up path */;
    uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(never + 1);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_holder + 1);
    volatile int* sequence = abort_flag + 1;
    int* n_own = const_cast<int*>(abort_flag) + 2;                  // [2] own tiles of the streams
    OwnTile* own = reinterpret_cast<OwnTile*>(n_own + 2);            // [2][kMaxOwnTiles]

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
        mbar_init(never, 1);
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
    if (a.fused) {
        if (threadIdx.x < 2) {
            // thread s lists the own tiles of stream s: the drafts whose tokens are in its query tile
            const int s = threadIdx.x, first = (qt0 + s) * a.tq, last = min(a.T, first + a.tq) - 1;
            int n = 0;
            if (s < n_streams && a.S > 0)
                for (int d = first / a.M; d <= last / a.M; ++d) {
                    const int len = a.own_len ? min(max(a.own_len[(int64_t)b * a.D + d], 0), a.S) : a.S;
                    for (int k0 = 0; k0 < len && n < kMaxOwnTiles; k0 += 128) own[s * kMaxOwnTiles + n++] = OwnTile{d, k0, len};
                }
            n_own[s] = n;
        }
        __syncthreads();
    }
    const int tiles = (L + 127) / 128;
    // key tiles [t0, t0 + nt) of the prefix for each stream: split s of a.splits even shares; then the stream's own tiles
    auto share = [&](int x) { return (int)((long long)tiles * x / a.splits); };
    const int sp0 = shared_keys ? cs : cs * 2, sp1 = shared_keys ? cs : cs * 2 + 1;
    const int t00 = share(sp0), t01 = share(sp1);
    const int np0 = share(sp0 + 1) - t00, np1 = n_streams > 1 ? share(sp1 + 1) - t01 : 0;
    const int nt0 = np0 + (a.fused ? n_own[0] : 0), nt1 = np1 + (a.fused ? n_own[1] : 0);
    const int most = max(nt0, nt1);
    // Tiles come through one ring, in the order: per round j = -1, 0, ..: V of tile j, K of tile j + 1 for stream 0, then for
    // stream 1.  Tiles below `common` are one for both streams and listed for stream 0 only.
    const int common = shared_keys ? np0 : 0;
    auto listed = [&](int s, int j) { return j >= 0 && j < (s ? nt1 : nt0) && (s == 0 || j >= common); };
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
#pragma unroll 1
            for (int x = 0; ok && x < 4 * (most + 1); ++x) {
                const bool is_k = x & 1;
                const int s = (x >> 1) & 1, j = (x >> 2) - (is_k ? 0 : 1);
                if (!listed(s, j)) continue;
                const int slot = item % NS, np = s ? np1 : np0;
                if (!mbar_wait_warp(&empty[slot], ((item / NS) & 1) ^ 1, wc)) { ok = false; break; }
                if (leader) {
                    unsigned char* to = ring + slot * TILE;
                    if (j < np) {
                        const CUtensorMap* map = is_k ? &map_k : &map_v;
                        mbar_arrive_expect_tx(&full[slot], TILE);
#pragma unroll
                        for (int c = 0; c < SLABS; ++c)
                            tma_load_4d(to + c * kSlabBytes, map, &full[slot], c * kSlabElems, h * (is_k ? a.k_head : a.v_head),
                                        ((s ? t01 : t00) + j) * 128, b * (is_k ? a.k_outer : a.v_outer));
                    } else {
                        const OwnTile o = own[s * kMaxOwnTiles + j - np];
                        const CUtensorMap* map = is_k ? &map_ko : &map_vo;
                        mbar_arrive_expect_tx(&full[slot], (uint32_t)(SLABS * a.own_box * 128));
#pragma unroll
                        for (int c = 0; c < SLABS; ++c)
                            tma_load_4d(to + c * kSlabBytes, map, &full[slot], c * kSlabElems, h * (is_k ? a.ko_head : a.vo_head), o.key0,
                                        (b * a.D + o.node) * (is_k ? a.ko_outer : a.vo_outer));
                    }
                }
                ++item;
                if (a.stall_test && item == 1 && !mbar_wait_warp(never, 0, wc)) ok = false;
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
            const uint32_t id_own = umma_idesc16(a.own_box, BF16, false);
            auto wait_item = [&](int item) { return mbar_wait_warp(&full[item % NS], (item / NS) & 1, wc); };
            auto scores = [&](int s, int item, bool own_tile, bool release) {
                const uint64_t q = dq + (uint64_t)((shared_keys ? s : 0) * (TILE >> 4)), k = dk + (uint64_t)((item % NS) * (TILE >> 4));
                const uint32_t id = own_tile ? id_own : id_s;
#pragma unroll
                for (int i = 0; i < SLABS * 4; ++i)
                    if (i < k_steps) {
                        const uint64_t off = (i / 4) * (kSlabBytes >> 4) + (i % 4) * 2;
                        umma_f16(tmem + s * 128, q + off, k + off, id, i != 0);
                    }
                umma_commit(&s_full[s]);
                if (release) umma_commit(&empty[item % NS]);
            };
            int next = 0;                    // ring items, in the loader's order
            bool ok = mbar_wait_warp(q_full, 0, wc);
            int v = 0, k = 0;
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                if (!ok || (s ? nt1 : nt0) == 0) continue;
                if (listed(s, 0)) {
                    k = next++;
                    if (!(ok = wait_item(k))) continue;
                }
                tc_fence_after();
                if (leader) scores(s, k, (s ? np1 : np0) == 0, common == 0 || s == n_streams - 1);
            }
#pragma unroll 1
            for (int j = 0; ok && j < most; ++j) {
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    const int n = s ? nt1 : nt0, np = s ? np1 : np0;
                    if (!ok || j >= n) continue;
                    const bool more = j + 1 < n;
                    // (the tiles have usually landed long before the weights are ready)
                    if (listed(s, j)) { v = next++; ok = wait_item(v); }
                    if (ok && listed(s, j + 1)) { k = next++; ok = wait_item(k); }
                    if (!ok || !(ok = mbar_wait_warp(&p_half[s], j & 1, wc))) continue;
                    tc_fence_after();
                    // keys of this tile in steps of 16 (the last tile of a list may hold fewer); rows of other drafts stay
                    int left = L - ((s ? t01 : t00) + j) * 128;
                    uint32_t off[4] = {0u, 0u, 0u, 0u};
                    if (j >= np) {
                        const OwnTile o = own[s * kMaxOwnTiles + j - np];
                        left = o.len - o.key0;
                        const int lo = (o.node * a.M - (qt0 + s) * a.tq) * a.G, hi = lo + a.M * a.G;
#pragma unroll
                        for (int w = 0; w < 4; ++w) {
                            const int l0 = min(max(lo - w * 32, 0), 32), h0 = min(max(hi - w * 32, 0), 32);     // active rows [l0, h0)
                            const uint32_t below_h = h0 == 32 ? 0xffffffffu : (1u << h0) - 1u, below_l = l0 == 32 ? 0xffffffffu : (1u << l0) - 1u;
                            off[w] = ~(below_h & ~below_l);
                        }
                    }
                    const int steps = left >= 128 ? 8 : (left + 15) / 16;
                    const uint64_t vd = dv + (uint64_t)((v % NS) * (TILE >> 4));
                    const uint32_t t_s = tmem + s * 128, t_o = t_s + 256;
                    auto pv = [&](int i) {
                        if (i >= steps) return;
                        if (j < np) umma_f16_ts(t_o, t_s + i * 8, vd + (uint64_t)(i * (2048 >> 4)), id_o, (j | i) != 0);
                        else umma_f16_ts_rows(t_o, t_s + i * 8, vd + (uint64_t)(i * (2048 >> 4)), id_o, off, 1);     // (O was set to 0 if np == 0)
                    };
                    if (leader) { pv(0); pv(1); pv(2); pv(3); }
                    if (!(ok = mbar_wait_warp(&p_ready[s], j & 1, wc))) continue;
                    tc_fence_after();
                    if (leader) {
                        pv(4); pv(5); pv(6); pv(7);
                        // the scores of the next tile overwrite the weights just read; their commit covers PV as well
                        if (more) scores(s, k, j + 1 >= np, j + 1 >= common || s == n_streams - 1);
                        else umma_commit(&o_done[s]);
                        if (j >= common || s == n_streams - 1) umma_commit(&empty[v % NS]);
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
        float m = 0.f, l = 0.f;          // reference (scaled by c) and sum relative to it
        bool fresh = true;               // no score seen yet
        bool ok = true;
        const int n = s ? nt1 : nt0, np = s ? np1 : np0, first_tile = s ? t01 : t00;
        const int my_tok = (qt0 + (shared_keys ? s : 0)) * a.tq + row / a.G;                    // this row's token of the sequence,
        const int my_node = a.fused ? my_tok / a.M : 0, my_i = a.fused ? my_tok % a.M : 0;       // its draft and place in it
        if (n > 0 && np == 0) {
            // only own tiles, each for some of the rows: O begins at 0
            uint32_t zero[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) zero[i] = 0u;
            for (int c = 0; c < a.Dh; c += 32) tmem_st32(t_o + c, zero);
            tmem_wait_st();
        }
        int base = listed(0, 0) + listed(1, 0);      // ring items ahead of round j
        for (int j = 0; j < n; ++j) {
            if (!(ok = mbar_wait_warp(&s_full[s], j & 1, wc))) break;
            tc_fence_after();
            int left = L - (first_tile + j) * 128;   // keys of this tile,
            int lim = left;                          // and those that this row sees
            if (j >= np) {
                const OwnTile o = own[s * kMaxOwnTiles + j - np];
                left = o.len - o.key0;
                lim = my_node != o.node ? 0 : a.causal ? min(left, left - a.M + 1 + my_i) : left;
            }
            uint32_t r[4][32];
#pragma unroll
            for (int c = 0; c < 4; ++c) tmem_ld32(t_s + c * 32, r[c]);
#pragma unroll
            for (int c = 0; c < 4; ++c) tmem_wait_ld(r[c]);
            if (left < 128 || j >= np) {
#pragma unroll
                for (int c = 0; c < 4; ++c)
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        if (c * 32 + i >= lim) r[c][i] = 0xff800000u;
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
            // the reference that this tile's maximum asks for
            const float high = fmaxf(max3(u[0], u[1], u[2]), u[3]), top = BF16 ? high * a.c : fmaf(high, a.c, -kHalfRoom);
            const bool raise = top > (fresh ? -INFINITY : m + kRaise);
            if (__any_sync(0xffffffffu, raise)) {
                // the first scores of a row, or (rare) a much higher maximum: set the reference and rescale what has been summed
                // (PV of the tile before is done: these scores were committed after it)
                const bool rescale = raise && !fresh;
                const float f = rescale ? ex2(m - top) : 1.f;
                if (raise) { m = top; fresh = false; }
                l *= f;
                if (__any_sync(0xffffffffu, rescale))
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
                const int item = base + (s && j >= common ? listed(0, j) + listed(0, j + 1) : 0);
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
            base += listed(0, j) + listed(0, j + 1) + listed(1, j) + listed(1, j + 1);
        }
        if (s < n_streams) {
            const bool live = row < a.tq * a.G && my_tok < a.T;
            const int64_t tok = (int64_t)b * a.T + my_tok;
            const int head = h * a.G + row % a.G;
            if (n > 0 && ok) {
                ok = mbar_wait_warp(&o_done[s], 0, wc);
                tc_fence_after();
            }
            const bool none = fresh && l == 0.f;             // no key seen
            const float inv = none ? 0.f : 1.0f / l;
            if (ok && a.fused) {
                uint16_t* o = reinterpret_cast<uint16_t*>(a.out) + tok * a.out_token + (int64_t)head * a.out_head;
#pragma unroll 1
                for (int c = 0; c < a.Dh; c += 32) {
                    uint32_t x[32];
                    if (n > 0) {
                        tmem_ld32(t_o + c, x);
                        tmem_wait_ld(x);
                    }
#pragma unroll
                    for (int i = 0; i < 32; i += 8)
                        if (live && c + i < a.Dh) {
                            uint32_t y[4];
#pragma unroll
                            for (int q = 0; q < 4; ++q)
                                y[q] = none ? 0u : pack16(__uint_as_float(x[i + 2 * q]) * inv, __uint_as_float(x[i + 2 * q + 1]) * inv, BF16);
                            *reinterpret_cast<uint4*>(o + c + i) = make_uint4(y[0], y[1], y[2], y[3]);
                        }
                }
                if (live && a.lse) a.lse[tok * a.Hq + head] = none ? -INFINITY : m * kLn2 + logf(l);
            } else if (ok) {
                const int64_t at = (int64_t)(s ? sp1 : sp0) * a.rows + tok * a.Hq + head;
                float* o = a.po + at * DHP;
#pragma unroll 1
                for (int c = 0; n > 0 && c < a.Dh; c += 32) {
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
                if (live) a.pl[at] = n > 0 ? m + log2f(l) : -INFINITY;
            }
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
int launch_p(const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv, const CUtensorMap& mko, const CUtensorMap& mvo, const PrefixArgs& a, int64_t grid, cudaStream_t st) {
    constexpr int smem = (2 + Ring<SLABS>::N) * SLABS * kSlabBytes + kBarBytes;
    static_assert(smem <= 227 * 1024, "shared memory of the prefix kernel");
    static std::atomic<unsigned long long> set{0};
    if (!ensure_dynamic_smem(prefix_attention_kernel<SLABS, BF16>, smem, set)) return PSD_ERR_CUDA;
    static std::atomic<int> regs{0};      // 8 warps of 208 and 4 of 80 registers a thread
    if (!launched_with(prefix_attention_kernel<SLABS, BF16>, (256 * 208 + 128 * 80 + kPThreads - 1) / kPThreads, regs)) return PSD_ERR_CUDA;
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
    const cudaError_t e = cudaLaunchKernelEx(&cfg, prefix_attention_kernel<SLABS, BF16>, mq, mk, mv, mko, mvo, a);
    count_launch();
    return e == cudaSuccess ? PSD_OK : PSD_ERR_CUDA;
}

}  // namespace

int drafts_per_tile(int M, int tq) { return (tq + M - 2) / M + 1; }

// Own keys in the same kernel: when nothing is split (one result per row) and the drafts of a query tile are few.  A draft
// costs a tile however few keys it has, which a kernel of their own does not.  Measured, 32 own keys, in this kernel against two: 16
// sequences of 16 drafts, 32 heads of 128 over 8, prefix 1024, 3 drafts to a tile 116 against 198 us, 5: 71 against 111, 9: 47
// against 61, 12: 50 against 56; 32 drafts, 16 heads of 64, prefix 2048, 5: 304 against 423, 9: 209 against 229, prefix 1024, 10: 170
// against 170, 12: 177 against 158.
bool fuses_own(int M, int tq, int S) {
    const int drafts = drafts_per_tile(M, tq);
    return (int64_t)drafts * ((S + 127) / 128) <= kMaxOwnTiles && drafts <= 9;
}

// How the prefix's keys are split.  A CTA takes two query tiles (or the only one twice, over two ranges of keys); when
// (sequence, key head, tile pair) alone leaves SMs idle the keys are split, down to kMinTiles tiles of 128 keys per split.
PrefixPlan plan_prefix(int B, int D, int M, int Hq, int Hkv, int Dh, int P, int S) {
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
    p.fused = p.n_qt > 1 && p.splits == 1 && fuses_own(M, p.tq, S);
    return p;
}

int launch_prefix_attention(const void* q, const void* k, const void* v, const int32_t* prefix_len, const void* k_own, const void* v_own,
                            const int32_t* own_len, const psd_attention_t& a, const PrefixPlan& p, float* po, float* pl, void* out,
                            float* lse, int32_t* status_dev, cudaStream_t st) {
    CUtensorMap mq, mk, mv, mko, mvo;
    if (!make_query_map(&mq, q, a, p.tq) || !make_cache_map(&mk, k, a.dtype, a.kp, a.B, a.P, a.Hkv, a.Dh, 128) ||
        !make_cache_map(&mv, v, a.dtype, a.vp, a.B, a.P, a.Hkv, a.Dh, 128))
        return PSD_ERR_CUDA;
    const int own_box = a.S >= 128 ? 128 : (a.S + 15) / 16 * 16;
    if (p.fused && a.S > 0) {
        if (!make_cache_map(&mko, k_own, a.dtype, a.ko, a.B * a.D, a.S, a.Hkv, a.Dh, own_box) ||
            !make_cache_map(&mvo, v_own, a.dtype, a.vo, a.B * a.D, a.S, a.Hkv, a.Dh, own_box))
            return PSD_ERR_CUDA;
    } else {
        mko = mk;
        mvo = mv;
    }
    const int64_t grid = (int64_t)a.B * a.Hkv * p.units * (p.n_qt > 1 ? p.splits : p.splits / 2);
    if (grid > INT32_MAX) return PSD_ERR_SHAPE;
    const bool bf16 = a.dtype == PSD_BF16;
    PrefixArgs x = {};
    x.prefix_len = prefix_len;
    x.po = po; x.pl = pl;
    x.status_dev = status_dev;
    x.rows = (int64_t)a.B * a.D * a.M * a.Hq;
    x.T = a.D * a.M; x.G = a.Hq / a.Hkv; x.Hq = a.Hq; x.Hkv = a.Hkv; x.Dh = a.Dh; x.P = a.P;
    x.tq = p.tq; x.n_qt = p.n_qt; x.units = p.units; x.splits = p.splits;
    x.k_outer = a.kp.outer ? 1 : 0; x.k_head = a.kp.head ? 1 : 0;
    x.v_outer = a.vp.outer ? 1 : 0; x.v_head = a.vp.head ? 1 : 0;
    x.B = a.B;
    x.longest_first = prefix_len && a.B > 1 && a.B <= kMaxSorted && grid > sm_count() ? 1 : 0;
    x.fused = p.fused ? 1 : 0;
    x.D = a.D; x.M = a.M; x.S = a.S; x.causal = a.causal; x.own_box = own_box > 0 ? own_box : 16;
    x.ko_outer = a.ko.outer ? 1 : 0; x.ko_head = a.ko.head ? 1 : 0;
    x.vo_outer = a.vo.outer ? 1 : 0; x.vo_head = a.vo.head ? 1 : 0;
    x.own_len = own_len;
    x.out = out; x.lse = lse;
    x.out_token = a.out_token; x.out_head = a.out_head;
    x.c = a.scale * kLog2e;
    x.wait_limit = wait_limit_cycles();
    x.stall_test = selftest_stall();
    if (p.dhp == 64) return bf16 ? launch_p<1, true>(mq, mk, mv, mko, mvo, x, grid, st) : launch_p<1, false>(mq, mk, mv, mko, mvo, x, grid, st);
    return bf16 ? launch_p<2, true>(mq, mk, mv, mko, mvo, x, grid, st) : launch_p<2, false>(mq, mk, mv, mko, mvo, x, grid, st);
}

}  // namespace psd
