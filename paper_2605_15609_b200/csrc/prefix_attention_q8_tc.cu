// Attention of many query rows over a prefix in 8-bit codes, on tcgen05: prefix_attention_kernel's two streams (see there: query
// tiles of up to 128 rows, scores and outputs in tensor memory, weights overwriting scores, a thread per row in the softmax) with
// a stage in front of the products that widens the codes.
//
// TMA brings tiles of 128 keys in codes (16 KB) into a small ring; six warps widen them into a second ring of 16-bit tiles in the
// swizzled layout that the products read.  Codes are exact in 16 bits, so nothing is rounded there: keys become the queries' type, values
// fp16.  The keys' scale of each 16 columns is the factor of their scores in the exponent (in place of the one factor of the 16-bit kernel),
// the values' scale multiplies the weights, and these products go to tensor memory in fp16, up to 2^15 relative to a reference of the row's own (w) beside
// the one of its weights (m): a row may attend to none of the blocks whose values are large.  That is a product's maximum per 16 columns and 8 factors more
// a tile, 2% of the time below.
// Keys past the end are masked in the scores; their codes are finite, so their weights of 0 need no further care.
//
// Where the prefix is not split, the drafts' own 16-bit keys follow it as further tiles, as there: TMA brings them into the wide ring
// directly, and before a stream's first of them its output is multiplied by the reference of the value scales, so that both kinds add up.  The own
// weights of bf16 are kept below 1 (kOwnRoom), or sums of large values would leave fp32's range where their mean does not.
//
// Where the keys are split over up to eight CTAs, these are a cluster and join their results themselves: the own tiles are dealt out to
// them, each leaves its outputs, maxima and sums in its shared memory, and each reads and writes a share of the rows.  Nothing goes through
// memory, and no second kernel starts.
//
// Bound: for Dh = 128 products and exponentials as there (2048 cycles each per 256 rows x 128 keys), in the latency chain of scores, softmax
// and products; widening takes about 650 issue slots per scheduler of the same round, the values' scales 64 more per warp.  Measured: 16 sequences x 8 key
// heads x 2048 rows over up to 8192 keys (the seed's 667 GFLOP) 759-790 us, 0.85-0.88 PFLOP/s (16-bit cache: 665 us; without widening, and with one reference a row, 690).  The
// instruction cache is the next bound: with full and last tiles in one piece of straight code beside unrolled widening and issuing
// the same call took 1064 us.
#include "attn_tc.cuh"
#include "prefix_attention.cuh"
#include "prefix_attention_q8.cuh"

namespace psd {
namespace {

constexpr int kQThreads = 512;              // warps 0-3, 4-7: softmax of stream 0, 1; 8: TMA; 9: MMA; 10-15: widening
constexpr int kWideners = 192;
constexpr float kRaise = 8.0f;              // growth of a row's maximum (log2) that triggers a rescale
constexpr float kHalfRoom = 7.0f;           // how far (log2) the reference is set below the maximum: weights go up to 2^15
constexpr float kOwnRoom = -8.0f;           // the same for the own keys of bf16: weights up to 1
constexpr int kMaxSorted = 128;             // sequences that are put in order of length
constexpr int kBarBytes = 1024;
constexpr int kParts = 16;                  // results of a row that a cluster joins, at most

struct OwnTile { int node, key0, len; };    // a tile of own keys: draft of the sequence, first key, the draft's length

// Tiles in flight: codes (RAW; with a single query tile the other's memory holds as many again, since a cache that is read for few rows comes from
// HBM at the rate that the copies in flight allow) and widened ones.
template <int SLABS> struct Rings {
    static constexpr int RAW = SLABS == 2 ? 2 : 8, MOST = SLABS == 2 ? 4 : 8, WIDE = SLABS == 2 ? 4 : 8;
    static_assert(MOST < 2 * WIDE, "the loader is less than two items of a wide slot ahead of the widening");
};

struct TcArgs {
    const float *k_scale, *v_scale;
    const int32_t* prefix_len;
    float *po, *pl;
    int32_t* status_dev;
    int64_t rows;
    int T, G, Hq, Hkv, Dh, P, nb, shift;
    int tq, n_qt, units, splits;
    int k_outer, k_head, v_outer, v_head;
    int B, longest_first;
    // own keys and final outputs (fused == 1: one CTA has all keys of a row; 2: a cluster of n_cs joins); else partial results
    int fused, n_cs, D, M, S, causal, own_box;
    int ko_outer, ko_head, vo_outer, vo_head;
    const int32_t* own_len;
    void* out;
    float* lse;
    int64_t out_token, out_head;
    float c;
    long long wait_limit;
    int stall_test;
    uint32_t f16_codes, bf16_codes;
};

__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}
__device__ __forceinline__ uint32_t peer(uint32_t addr, int rank) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}

// The codes in bytes (b, b + 1) of x as two 16-bit numbers; sel spreads them over bytes 0 and 2.
template <bool BF16>
__device__ __forceinline__ uint32_t widen_pair(uint32_t x, uint32_t sel, uint32_t pattern) {
    const uint32_t t = __byte_perm(x, 0u, sel);
    return BF16 ? codes_bf16(t, pattern) : codes_f16(t, pattern);
}
// One tile of 128 keys x SLABS * 64 codes (rows dense) into SLABS swizzled slabs, by kWideners threads, 8 codes at a time.  A thread's
// place in a key's row is the same in every turn; its key moves by 12 (or 24), so the swizzle of its place takes two values: addresses are
// three registers and constants.
template <int SLABS, bool BF16>
__device__ __forceinline__ void widen_tile(uint32_t raw, uint32_t to, int tid, uint32_t pattern) {
    constexpr int CH = SLABS * 8, KEYS = kWideners / CH, BATCH = 5, TURNS = 128 / KEYS, REST = 128 - TURNS * KEYS;
    static_assert(KEYS % 4 == 0 && TURNS % BATCH == 0 && REST > 0 && REST < KEYS, "turns of a tile");
    constexpr uint32_t FLIP = KEYS % 8 ? 64u : 0u;         // what a turn changes in the swizzle of this thread's place
    const int key = tid / CH, ch = tid % CH;
    uint32_t src = raw + tid * 8, row = to + (ch / 8) * kSlabBytes + key * 128, at = ((ch % 8) ^ (key & 7)) << 4;
    uint32_t w[BATCH][2];
    auto load = [&](int i) { asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(w[i][0]), "=r"(w[i][1]) : "r"(src + i * (kWideners * 8))); };
    auto store = [&](int i) {
        asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(row + (i & 1 ? at ^ FLIP : at) + i * KEYS * 128), "r"(widen_pair<BF16>(w[i][0], 0x1100, pattern)),
                     "r"(widen_pair<BF16>(w[i][0], 0x3322, pattern)), "r"(widen_pair<BF16>(w[i][1], 0x1100, pattern)), "r"(widen_pair<BF16>(w[i][1], 0x3322, pattern)) : "memory");
    };
    // (a loop, not straight code: the kernel's instructions have to stay in the SM's cache beside the softmax)
#pragma unroll 1
    for (int i0 = 0; i0 < TURNS; i0 += BATCH) {
#pragma unroll
        for (int i = 0; i < BATCH; ++i) load(i);
#pragma unroll
        for (int i = 0; i < BATCH; ++i) store(i);
        src += BATCH * kWideners * 8;
        row += BATCH * KEYS * 128;
        at ^= BATCH & 1 ? FLIP : 0u;
    }
    if (key < REST) {
        load(0);
        store(0);
    }
}

template <int SLABS, bool BF16, bool JOINED>
__global__ void __launch_bounds__(kQThreads, 1)
prefix_tiles_q8_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                       const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CUtensorMap map_ko,
                       const __grid_constant__ CUtensorMap map_vo, const TcArgs a) {
    extern __shared__ __align__(1024) unsigned char smem[];
    constexpr int TILE = SLABS * kSlabBytes, RAW = TILE / 2, MOST = Rings<SLABS>::MOST, NS = Rings<SLABS>::WIDE, DHP = SLABS * 64;
    unsigned char* q_tiles = smem;                                   // [2][TILE]
    unsigned char* ring = smem + 2 * TILE;                           // [NS][TILE]
    unsigned char* raw = ring + NS * TILE;                           // [Rings::RAW][RAW]
    uint64_t* bars = reinterpret_cast<uint64_t*>(raw + Rings<SLABS>::RAW * RAW);
    uint64_t *q_full = bars, *raw_full = bars + 1, *raw_empty = raw_full + MOST, *full = raw_empty + MOST, *empty = full + NS, *s_full = empty + NS /* [2] */,
             *p_half = s_full + 2, *p_ready = p_half + 2, *o_done = p_ready + 2, *drain = o_done + 2, *never = drain + 1;
    uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(never + 1);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_holder + 1);
    volatile int* sequence = abort_flag + 1;
    int* n_own = const_cast<int*>(abort_flag) + 2;                  // [2] own tiles of the streams
    OwnTile* own = reinterpret_cast<OwnTile*>(n_own + 2);            // [2][kMaxOwnTiles]

    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    const bool shared_keys = a.n_qt > 1;
    const uint32_t NR = shared_keys ? Rings<SLABS>::RAW : MOST;      // (powers of 2)
    auto raw_slot = [&](int in) {
        const uint32_t slot = (uint32_t)in & (NR - 1);
        return slot < Rings<SLABS>::RAW ? raw + slot * RAW : q_tiles + TILE + (slot - Rings<SLABS>::RAW) * RAW;
    };
    auto raw_bar = [&](uint64_t* b, int in) { return b + ((uint32_t)in & (NR - 1)); };
    auto raw_turn = [&](int in) { return (uint32_t)in / NR & 1u; };
    const int n_cs = a.n_cs;                      // CTAs along the keys; joined: neighbours (a cluster)
    constexpr bool joined = JOINED;               // (compiled apart: the other form is a few percent faster without this one's code)
    const int rest = joined ? blockIdx.x / n_cs : blockIdx.x / a.units, unit = joined ? rest % a.units : blockIdx.x % a.units;
    const int cs = joined ? blockIdx.x % n_cs : rest % n_cs, bh = rest / (joined ? a.units : n_cs), h = bh % a.Hkv;
    int b = bh / a.Hkv;
    const int qt0 = shared_keys ? unit * 2 : 0;
    const int n_streams = shared_keys ? min(2, a.n_qt - qt0) : 2;

    if (threadIdx.x == 0) {
        mbar_init(q_full, 1);
        for (int s = 0; s < MOST; ++s) { mbar_init(&raw_full[s], 1); mbar_init(&raw_empty[s], kWideners / 32); }
        for (int s = 0; s < NS; ++s) { mbar_init(&full[s], kWideners / 32); mbar_init(&empty[s], 1); }
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
    const int L = length(b), tiles = (L + 127) / 128;
    if (a.fused) {
        if (warp < 2) {
            // warp s lists the own tiles of stream s, the drafts whose tokens are in its query tile, a lane per draft (joined: every n_cs-th tile, or with
            // one query tile every 2 n_cs-th)
            const int s = warp, first = (qt0 + (shared_keys ? s : 0)) * a.tq, last = min(a.T, first + a.tq) - 1;
            const int deal = !joined ? 1 : shared_keys ? n_cs : 2 * n_cs, mine = !joined ? 0 : shared_keys ? cs : 2 * cs + s;
            int before = 0;
            if (s < n_streams && a.S > 0)
                for (int d0 = first / a.M; d0 <= last / a.M; d0 += 32) {
                    const int d = d0 + lane;
                    const int len = d > last / a.M ? 0 : a.own_len ? min(max(a.own_len[(int64_t)b * a.D + d], 0), a.S) : a.S;
                    int upto = (len + 127) / 128;
                    const int n = upto;
#pragma unroll
                    for (int x = 1; x < 32; x *= 2) {
                        const int y = __shfl_up_sync(0xffffffffu, upto, x);
                        if (lane >= x) upto += y;
                    }
                    for (int k = 0; k < n; ++k) {
                        const int i = before + upto - n + k;
                        if (i % deal == mine && i / deal < kMaxOwnTiles) own[s * kMaxOwnTiles + i / deal] = OwnTile{d, k * 128, len};
                    }
                    before += __shfl_sync(0xffffffffu, upto, 31);
                }
            if (lane == 0) n_own[s] = min(before > mine ? (before - mine + deal - 1) / deal : 0, kMaxOwnTiles);
        }
        __syncthreads();
    }
    auto share = [&](int x) { return (int)((long long)tiles * x / a.splits); };
    const int sp0 = shared_keys ? cs : cs * 2, sp1 = shared_keys ? cs : cs * 2 + 1;
    const int t00 = share(sp0), t01 = share(sp1);
    const int np0 = share(sp0 + 1) - t00, np1 = n_streams > 1 ? share(sp1 + 1) - t01 : 0;      // tiles of the prefix,
    const int nt0 = np0 + (a.fused ? n_own[0] : 0), nt1 = np1 + (a.fused ? n_own[1] : 0);      // and with the stream's own
    const int most = max(nt0, nt1);
    // Tiles in the order: per round j = -1, 0, ..: V of tile j, K of tile j + 1 for stream 0, then for stream 1; those
    // below `common` are one for both streams and listed for stream 0 only.
    const int common = shared_keys ? np0 : 0;
    auto listed = [&](int s, int j) { return j >= 0 && j < (s ? nt1 : nt0) && (s == 0 || j >= common); };
    const int n_q = shared_keys ? n_streams : 1;

    if (warp >= 8) asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
    if (warp >= 10) {
        // -------------------------------------------------------------------- widening
        const int tid = threadIdx.x - 10 * 32;
        int item = 0, in = 0;               // ring items, and those that come in codes
        bool ok = true;
#pragma unroll 1
        for (int x = 0; ok && x < 4 * (most + 1); ++x) {
            const bool is_k = x & 1;
            const int s = (x >> 1) & 1, j = (x >> 2) - (is_k ? 0 : 1);
            if (!listed(s, j)) continue;
            if (j >= (s ? np1 : np0)) { ++item; continue; }
            if (!(ok = mbar_wait_warp(&empty[item % NS], ((item / NS) & 1) ^ 1, wc))) break;
            if (!(ok = mbar_wait_warp(raw_bar(raw_full, in), raw_turn(in), wc))) break;
            const uint32_t from = smem_u32(raw_slot(in)), to = smem_u32(ring + (item % NS) * TILE);
            if (BF16 && is_k) widen_tile<SLABS, true>(from, to, tid, a.bf16_codes);
            else widen_tile<SLABS, false>(from, to, tid, a.f16_codes);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(raw_bar(raw_empty, in));
                mbar_arrive(&full[item % NS]);
            }
            ++item;
            ++in;
        }
    } else if (warp >= 8) {
        if (warp == 8 && most > 0) {
            // ---------------------------------------------------------------- loader
            const bool leader = elect_one();
            if (leader) {
                mbar_arrive_expect_tx(q_full, (uint32_t)(n_q * SLABS * a.tq * a.G * 128));
                for (int t = 0; t < n_q; ++t)
                    for (int c = 0; c < SLABS; ++c)
                        tma_load_3d(q_tiles + t * TILE + c * kSlabBytes, &map_q, q_full, c * kSlabElems, h * a.G, b * a.T + (qt0 + t) * a.tq);
            }
            int item = 0, in = 0, first_own = -1;
            bool ok = true;
#pragma unroll 1
            for (int x = 0; ok && x < 4 * (most + 1); ++x) {
                const bool is_k = x & 1;
                const int s = (x >> 1) & 1, j = (x >> 2) - (is_k ? 0 : 1), np = s ? np1 : np0;
                if (!listed(s, j)) continue;
                if (j < np) {
                    if (!mbar_wait_warp(raw_bar(raw_empty, in), raw_turn(in) ^ 1, wc)) { ok = false; break; }
                    if (leader) {
                        mbar_arrive_expect_tx(raw_bar(raw_full, in), RAW);
                        tma_load_4d(raw_slot(in), is_k ? &map_k : &map_v, raw_bar(raw_full, in), 0, h * (is_k ? a.k_head : a.v_head),
                                    ((s ? t01 : t00) + j) * 128, b * (is_k ? a.k_outer : a.v_outer));
                    }
                    ++in;
                } else {
                    const int slot = item % NS;
                    // The slot's last item must have come and gone.  Up to here this warp has only seen the codes' ring, which lets it be two items of a
                    // slot ahead of the widening; a wait by parity tells one from the other only once the slot's last item is known to be there.
                    if (item >= NS && !mbar_wait_warp(&full[slot], ((item / NS) & 1) ^ 1, wc)) { ok = false; break; }
                    if (!mbar_wait_warp(&empty[slot], ((item / NS) & 1) ^ 1, wc)) { ok = false; break; }
                    if (leader) {
                        const OwnTile o = own[s * kMaxOwnTiles + j - np];
                        const CUtensorMap* map = is_k ? &map_ko : &map_vo;
                        // (this warp stands in for the widening ones)
                        mbar_arrive_expect_tx(&full[slot], (uint32_t)(SLABS * a.own_box * 128));
                        for (int i = 1; i < kWideners / 32; ++i) mbar_arrive(&full[slot]);
#pragma unroll
                        for (int c = 0; c < SLABS; ++c)
                            tma_load_4d(ring + slot * TILE + c * kSlabBytes, map, &full[slot], c * kSlabElems, h * (is_k ? a.ko_head : a.vo_head),
                                        o.key0, (b * a.D + o.node) * (is_k ? a.ko_outer : a.vo_outer));
                    }
                    if (first_own < 0) first_own = item;
                }
                ++item;
                if (a.stall_test && item == 1 && !mbar_wait_warp(never, 0, wc)) ok = false;
            }
            if (!ok) {
                // giving up: no copy may be in flight when the CTA exits
                long long c0 = clock64();
                while (!mbar_try_wait(q_full, 0) && clock64() - c0 < WAIT_LIMIT_CYCLES) {}
                for (int i = max(in - (int)NR, 0); i < in; ++i) {
                    c0 = clock64();
                    while (!mbar_try_wait(raw_bar(raw_full, i), raw_turn(i)) && clock64() - c0 < WAIT_LIMIT_CYCLES) {}
                }
                for (int i = max(first_own, item - NS); first_own >= 0 && i < item; ++i) {
                    c0 = clock64();
                    while (!mbar_try_wait(&full[i % NS], (i / NS) & 1) && clock64() - c0 < WAIT_LIMIT_CYCLES) {}
                }
            }
        } else if (warp == 9 && most > 0) {
            // ---------------------------------------------------------------- products (one warp, both streams in turn)
            const bool leader = elect_one();
            const uint32_t id_s = umma_idesc16(128, BF16, false), id_o = umma_idesc16((a.Dh + 15) / 16 * 16, false, true);
            const uint32_t id_s_own = umma_idesc16(a.own_box, BF16, false), id_o_own = umma_idesc16((a.Dh + 15) / 16 * 16, BF16, true);
            const int k_steps = (a.Dh + 15) / 16;
            const uint64_t dq = umma_smem_desc(smem_u32(q_tiles)), dk = umma_smem_desc(smem_u32(ring));
            const uint64_t dv = umma_smem_desc_mn(smem_u32(ring), kSlabBytes);
            auto wait_item = [&](int item) { return mbar_wait_warp(&full[item % NS], (item / NS) & 1, wc); };
            auto scores = [&](int s, int item, bool own_tile, bool release) {
                const uint64_t q = dq + (uint64_t)((shared_keys ? s : 0) * (TILE >> 4)), k = dk + (uint64_t)((item % NS) * (TILE >> 4));
                const uint32_t id = own_tile ? id_s_own : id_s;
#pragma unroll
                for (int i = 0; i < SLABS * 4; ++i)
                    if (i < k_steps) {
                        const uint64_t off = (i / 4) * (kSlabBytes >> 4) + (i % 4) * 2;
                        umma_f16(tmem + s * 128, q + off, k + off, id, i != 0);
                    }
                umma_commit(&s_full[s]);
                if (release) umma_commit(&empty[item % NS]);
            };
            int next = 0;
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
#pragma unroll 1
                for (int s = 0; s < 2; ++s) {
                    const int n = s ? nt1 : nt0, np = s ? np1 : np0;
                    if (!ok || j >= n) continue;
                    const bool more = j + 1 < n;
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
                        const int lo = (o.node * a.M - (qt0 + (shared_keys ? s : 0)) * a.tq) * a.G, hi = lo + a.M * a.G;
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
                        // (O was set to 0 if np == 0)
                        umma_f16_ts_rows(t_o, t_s + i * 8, vd + (uint64_t)(i * (2048 >> 4)), j < np ? id_o : id_o_own, off, j >= np || (j | i) != 0);
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
        // -------------------------------------------------------------------- softmax: a row per thread
        asm volatile("setmaxnreg.inc.sync.aligned.u32 192;");
        const int s = warp >> 2, quarter = warp & 3, row = quarter * 32 + lane;
        const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
        const uint32_t t_s = tmem + lanes + s * 128, t_o = tmem + lanes + 256 + s * 128;
        float m = 0.f, l = 0.f;          // reference (in the exponent's units) and sum relative to it
        float w = -INFINITY;             // reference of weight times value scale, which the output is relative to (own keys: m)
        bool fresh = true;               // no score seen yet
        bool ok = true;
        const int n = s ? nt1 : nt0, np = s ? np1 : np0, first_tile = s ? t01 : t00;
        const int my_tok = (qt0 + (shared_keys ? s : 0)) * a.tq + row / a.G;                     // this row's token of the sequence,
        const int my_node = a.fused ? my_tok / a.M : 0, my_i = a.fused ? my_tok % a.M : 0;       // its draft and place in it
        // Scales of a tile: lane i holds the keys' of columns 16 i .., lane 8 + i the values', relative to the largest of this stream's
        // keys, lane 16 + i their logarithms.  They are loaded a round ahead.
        const float* ks = a.k_scale + ((int64_t)b * a.Hkv + h) * a.nb;
        const float* vs = a.v_scale + ((int64_t)b * a.Hkv + h) * a.nb;
        float vref = 1.17549435e-38f;
        if (np > 0) {
            const int j1 = min(((first_tile + np) * 128 - 1) >> a.shift, (L - 1) >> a.shift);
            for (int j = ((first_tile * 128) >> a.shift) + lane; j <= j1; j += 32) vref = fmaxf(vref, vs[j]);
#pragma unroll
            for (int x = 16; x; x >>= 1) vref = fmaxf(vref, __shfl_xor_sync(0xffffffffu, vref, x));
        }
        const float vinv = 1.f / vref;
        auto scale_of = [&](int j) {
            if (j >= np) return lane & 8 ? 1.f : a.c;       // own keys
            const int key = (first_tile + j) * 128 + (lane & 7) * 16;
            if (key >= L) return 0.f;                   // (what stands there was never written)
            const float x = lane & 24 ? vs[key >> a.shift] * vinv : ks[key >> a.shift] * a.c;
            if (lane & 16) return lg2(x);
            return lane & 8 || x != 0.f ? x : 1.17549435e-38f;      // masked scores are -inf times this
        };
        float next_scale = n > 0 ? scale_of(0) : 0.f;
        if (n > 0 && np == 0) {
            // only own tiles, each for some of the rows: O begins at 0
            uint32_t zero[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) zero[i] = 0u;
            for (int c = 0; c < a.Dh; c += 32) tmem_st32(t_o + c, zero);
            tmem_wait_st();
        }
        int base = listed(0, 0) + listed(1, 0);      // ring items ahead of round j
        // One tile.  FULL: 128 keys of the prefix, seen by every row; else the prefix's last keys or own ones.  The two are compiled apart:
        // the walk over full tiles is most of the time, and its instructions have to stay in the SM's cache beside the other warps'.
        auto tile = [&](int j, auto full_tile) {
            constexpr bool FULL = decltype(full_tile)::value;
            const bool own_tile = !FULL && j >= np;
            const float sc = next_scale;
            if (j + 1 < n) next_scale = scale_of(j + 1);
            if (!mbar_wait_warp(&s_full[s], j & 1, wc)) return false;
            tc_fence_after();
            int left = L - (first_tile + j) * 128;   // keys of this tile,
            int lim = left;                          // and those that this row sees
            if (own_tile) {
                const OwnTile o = own[s * kMaxOwnTiles + j - np];
                left = o.len - o.key0;
                lim = my_node != o.node ? 0 : a.causal ? min(left, left - a.M + 1 + my_i) : left;
            }
            uint32_t r[4][32];
#pragma unroll
            for (int c = 0; c < 4; ++c) tmem_ld32(t_s + c * 32, r[c]);
#pragma unroll
            for (int c = 0; c < 4; ++c) tmem_wait_ld(r[c]);
            if (!FULL) {
#pragma unroll
                for (int c = 0; c < 4; ++c)
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        if (c * 32 + i >= lim) r[c][i] = 0xff800000u;
            }
            float high = -INFINITY, high_w = -INFINITY;
#pragma unroll
            for (int g = 0; g < 8; ++g) {
                auto x = [&](int i) { return __uint_as_float(r[g >> 1][(g & 1) * 16 + i]); };
                float u = max3(x(0), x(1), x(2));
#pragma unroll
                for (int i = 3; i < 15; i += 2) u = max3(u, x(i), x(i + 1));
                u = fmaxf(u, x(15));
                // (columns past the end have the scale 0 where their 16 hold no key: -inf * 0 is no number and drops out)
                u *= __shfl_sync(0xffffffffu, sc, g);
                high = fmaxf(high, u);
                high_w = fmaxf(high_w, u + __shfl_sync(0xffffffffu, sc, 16 + g));
            }
            // the references that this tile's maxima ask for
            const float top = high - (BF16 && own_tile ? kOwnRoom : kHalfRoom);
            const bool raise = top > (fresh ? -INFINITY : m + kRaise);
            const float top_w = high_w - kHalfRoom;
            const bool raise_w = !own_tile && top_w > w + kRaise;
            const bool unit = own_tile && j == np && j > 0;        // from here on outputs are relative to 1, not to vref
            if (unit || __any_sync(0xffffffffu, raise || raise_w)) {
                const float m0 = m, w0 = w;
                float f = 1.f;
                if (raise) m = top;
                if (unit && BF16 && !fresh) m = fmaxf(m, m0 + (kHalfRoom - kOwnRoom));
                w = own_tile ? m : fmaxf(raise_w ? top_w : w, m - kFar);
                if (!fresh) {
                    l *= ex2(m0 - m);
                    f = unit ? times_ex2(vref, w0 - w) : ex2(w0 - w);
                }
                fresh = fresh && !raise;
                if (__any_sync(0xffffffffu, f != 1.f))
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
            if (own_tile && left < 128) {
                // own values past the end that the product's last step of 16 keys reads: zero, whatever stands there
                const int item = base + (s && j >= common ? listed(0, j) + listed(0, j + 1) : 0);
                if (!mbar_wait_warp(&full[item % NS], (item / NS) & 1, wc)) return false;
                const int stop = (left + 15) / 16 * 16;
                unsigned char* v = ring + (item % NS) * TILE;
                for (int x = left * 8 * SLABS + row; x < stop * 8 * SLABS; x += 128) {
                    const int key = x / (8 * SLABS), ch = x % (8 * SLABS);
                    *reinterpret_cast<uint4*>(v + (ch / 8) * kSlabBytes + key * 128 + (ch % 8) * 16) = make_uint4(0, 0, 0, 0);
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            }
            const f32x2 nm = pack2(-m, -m);
            const float gain = ex2(fminf(m - w, kFar));
            f32x2 acc[2] = {0ull, 0ull};
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                uint32_t p[16];
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    float kf = __shfl_sync(0xffffffffu, sc, 2 * c + g);
                    const float vf = __shfl_sync(0xffffffffu, sc, 8 + 2 * c + g) * gain;
                    if (!FULL && kf == 0.f) kf = 1.f;      // no key among these 16: their scores are -inf
                    const f32x2 kk = pack2(kf, kf), vv = pack2(vf, vf);
#pragma unroll
                    for (int i = g * 8; i < g * 8 + 8; ++i) {
                        const f32x2 e = ex2_pair(fma2(pack2(__uint_as_float(r[c][2 * i]), __uint_as_float(r[c][2 * i + 1])), kk, nm));
                        acc[i & 1] = add2(acc[i & 1], e);
                        float y, z;
                        unpack2(mul2(e, vv), y, z);
                        // (own values are of the queries' type)
                        if (!FULL && BF16 && own_tile) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(p[i]) : "f"(z), "f"(y));
                        else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(p[i]) : "f"(z), "f"(y));
                    }
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
            return true;
        };
        int j = 0;
#pragma unroll 1
        for (const int n_full = min(np, L / 128 - first_tile); ok && j < n_full; ++j) ok = tile(j, std::true_type());
#pragma unroll 1
        for (; ok && j < n; ++j) ok = tile(j, std::false_type());
        const float out_unit = np < n ? 1.f : times_ex2(vref, w - m);       // of the outputs
        if (joined) {
            // outputs by the sum of weights (of a row: 16-byte pieces, rotated by the row so that a quarter of a warp writes all banks) and (reference, sum)
            // into the ring, which is free once both streams' products are done
            for (int x = 0; ok && x < 2; ++x)
                if ((x ? nt1 : nt0) > 0) ok = mbar_wait_warp(&o_done[x], 0, wc);
            tc_fence_after();
            const bool none = n == 0 || (fresh && l == 0.f);
            const float u = none ? 0.f : out_unit / l;
            const uint32_t to = smem_u32(ring) + (s * 128 + row) * DHP * 4;
#pragma unroll 1
            for (int c = 0; ok && n > 0 && c < a.Dh; c += 32) {
                uint32_t x[32];
                tmem_ld32(t_o + c, x);
                tmem_wait_ld(x);
#pragma unroll
                for (int i = 0; i < 32; i += 4)
                    asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(to + ((((c + i) / 4) ^ (row & 7)) << 4)), "f"(__uint_as_float(x[i]) * u),
                                 "f"(__uint_as_float(x[i + 1]) * u), "f"(__uint_as_float(x[i + 2]) * u), "f"(__uint_as_float(x[i + 3]) * u) : "memory");
            }
            reinterpret_cast<float2*>(raw)[s * 128 + row] = none ? make_float2(-INFINITY, 0.f) : make_float2(m, l);
        } else if (s < n_streams) {
            const bool live = row < a.tq * a.G && my_tok < a.T;
            if (n > 0 && ok) {
                ok = mbar_wait_warp(&o_done[s], 0, wc);
                tc_fence_after();
            }
            const bool none = fresh && l == 0.f;             // no key seen
            const float inv = none ? 0.f : out_unit / l;
            const int64_t tok = (int64_t)b * a.T + my_tok;
            const int head = h * a.G + row % a.G;
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
                            for (int q = 0; q < 4; ++q) {
                                const float lo = __uint_as_float(x[i + 2 * q]) * inv, hi = __uint_as_float(x[i + 2 * q + 1]) * inv;
                                if (BF16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(y[q]) : "f"(hi), "f"(lo));
                                else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(y[q]) : "f"(hi), "f"(lo));
                                if (none) y[q] = 0u;
                            }
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
    __syncwarp();
    tc_fence_before();
    if (joined) {
        cluster_sync();
        if (warp < 8 && !*abort_flag) {
            // A share of the rows; part p of a row is CTA p's (one query tile: stream p % 2 of CTA p / 2).  First the parts' weights, a thread per row,
            // then the outputs, a thread per row and four columns.
            const int n_rows = shared_keys ? n_streams * 128 : 128, parts = shared_keys ? n_cs : 2 * n_cs;
            const int lo = n_rows * cs / n_cs, n_mine = n_rows * (cs + 1) / n_cs - lo;
            const uint32_t so = smem_u32(ring), stats = smem_u32(raw);
            float* weights = reinterpret_cast<float*>(raw + 2048);               // [128][kParts]
            auto place = [&](int x, int q) { return shared_keys ? x : (q & 1) * 128 + x; };        // of row x in part q
            auto owner = [&](int q) { return shared_keys ? q : q / 2; };
            auto token = [&](int x) {                                              // -1: no row
                const int r = x & 127, t = (qt0 + (x >> 7)) * a.tq + r / a.G;
                return r < a.tq * a.G && t < a.T ? t : -1;
            };
            if ((int)threadIdx.x < n_mine) {
                const int x = lo + threadIdx.x, t = token(x);
                float mm[kParts], ll[kParts], top = -INFINITY, sum = 0.f;
#pragma unroll
                for (int q = 0; q < kParts; ++q) {
                    mm[q] = -INFINITY;
                    ll[q] = 0.f;
                    if (q < parts && t >= 0)
                        asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(mm[q]), "=f"(ll[q]) : "r"(peer(stats + place(x, q) * 8, owner(q))) : "memory");
                }
#pragma unroll
                for (int q = 0; q < kParts; ++q) top = fmaxf(top, mm[q]);
                const float base = top == -INFINITY ? 0.f : top;
                bool some = false;
#pragma unroll
                for (int q = 0; q < kParts; ++q)
                    if (mm[q] != -INFINITY) {                                    // (others hold no outputs)
                        some = true;
                        mm[q] = ex2(mm[q] - base) * ll[q];
                        sum += mm[q];
                    } else {
                        mm[q] = 0.f;
                    }
                const float inv = some ? 1.f / sum : 0.f;
#pragma unroll
                for (int q = 0; q < kParts; ++q) weights[threadIdx.x * kParts + q] = mm[q] * inv;
                if (a.lse && t >= 0) a.lse[((int64_t)b * a.T + t) * a.Hq + h * a.G + (x & 127) % a.G] = some ? top * kLn2 + logf(sum) : -INFINITY;
            }
            asm volatile("bar.sync 1, 256;" ::: "memory");
#pragma unroll 1
            for (int i = threadIdx.x; i < n_mine * (DHP / 4); i += 256) {
                const int y = i / (DHP / 4), col = i % (DHP / 4) * 4, x = lo + y, r = x & 127, t = token(x);
                if (t < 0 || col >= a.Dh) continue;
                const float* w = weights + y * kParts;
                float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
                for (int q0 = 0; q0 < parts; q0 += 8) {
                    float4 z[8];
#pragma unroll
                    for (int q = 0; q < 8; ++q) {
                        z[q] = make_float4(0.f, 0.f, 0.f, 0.f);
                        if (q0 + q < parts && w[q0 + q] != 0.f)
                            asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(z[q].x), "=f"(z[q].y), "=f"(z[q].z), "=f"(z[q].w)
                                         : "r"(peer(so + place(x, q0 + q) * DHP * 4 + (((col >> 2) ^ (r & 7)) << 4), owner(q0 + q))) : "memory");
                    }
#pragma unroll
                    for (int q = 0; q < 8; ++q) {
                        const float f = q0 + q < parts ? w[q0 + q] : 0.f;
                        acc[0] = fmaf(f, z[q].x, acc[0]); acc[1] = fmaf(f, z[q].y, acc[1]);
                        acc[2] = fmaf(f, z[q].z, acc[2]); acc[3] = fmaf(f, z[q].w, acc[3]);
                    }
                }
                uint32_t y0, y1;
                if (BF16) {
                    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(y0) : "f"(acc[1]), "f"(acc[0]));
                    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(y1) : "f"(acc[3]), "f"(acc[2]));
                } else {
                    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(y0) : "f"(acc[1]), "f"(acc[0]));
                    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(y1) : "f"(acc[3]), "f"(acc[2]));
                }
                *reinterpret_cast<uint2*>(reinterpret_cast<uint16_t*>(a.out) + ((int64_t)b * a.T + t) * a.out_token + (int64_t)(h * a.G + r % a.G) * a.out_head + col) =
                    make_uint2(y0, y1);
            }
        }
        __syncwarp();
        cluster_sync();                                  // no CTA leaves while another reads its shared memory
    } else {
        __syncthreads();
    }
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (warp == 9) {
        __syncwarp();
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
    }
}

// A cache of codes, boxes of 128 tokens of one head, rows of dhp bytes.
bool make_tile_map(CUtensorMap* m, const void* base, const psd_kv_strides_t& s, int outer, int tokens, int heads, int Dh, int dhp) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    cuuint64_t dims[4] = {(cuuint64_t)Dh, (cuuint64_t)(s.head ? heads : 1), (cuuint64_t)tokens, (cuuint64_t)(s.outer ? outer : 1)};
    cuuint64_t strides[3] = {(cuuint64_t)(s.head ? s.head : 16), (cuuint64_t)s.token, (cuuint64_t)(s.outer ? s.outer : 16)};
    cuuint32_t b[4] = {(cuuint32_t)dhp, 1, 128, 1};
    cuuint32_t estr[4] = {1, 1, 1, 1};
    return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, const_cast<void*>(base), dims, strides, b, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int SLABS, bool BF16, bool JOINED>
int launch_j(const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv, const CUtensorMap& mko, const CUtensorMap& mvo, const TcArgs& a, int64_t grid,
             cudaStream_t st) {
    constexpr int TILE = SLABS * kSlabBytes;
    constexpr int smem = (2 + Rings<SLABS>::WIDE) * TILE + Rings<SLABS>::RAW * (TILE / 2) + kBarBytes;
    static_assert(smem <= 227 * 1024, "shared memory of the 8-bit tile kernel");
    static_assert(Rings<SLABS>::WIDE * TILE >= 2 * 128 * SLABS * 64 * 4 && Rings<SLABS>::RAW * (TILE / 2) >= 2 * 128 * 8 + 128 * kParts * 4, "outputs and sums that a cluster joins");
    static std::atomic<unsigned long long> set{0};
    if (!ensure_dynamic_smem(prefix_tiles_q8_kernel<SLABS, BF16, JOINED>, smem, set)) return PSD_ERR_CUDA;
    static std::atomic<int> regs{0};      // 8 warps of 192 and 8 of 64 registers a thread
    if (!launched_with(prefix_tiles_q8_kernel<SLABS, BF16, JOINED>, (256 * 192 + 256 * 64) / kQThreads, regs)) return PSD_ERR_CUDA;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3(kQThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = pdl_enabled() ? 1 : 0;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim = {JOINED ? (unsigned)a.n_cs : 1u, 1u, 1u};
    cfg.attrs = attr;
    cfg.numAttrs = JOINED ? 2 : 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, prefix_tiles_q8_kernel<SLABS, BF16, JOINED>, mq, mk, mv, mko, mvo, a);
    count_launch();
    return e == cudaSuccess ? PSD_OK : PSD_ERR_CUDA;
}

template <int SLABS, bool BF16>
int launch_t(const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv, const CUtensorMap& mko, const CUtensorMap& mvo, const TcArgs& a, int64_t grid,
             cudaStream_t st) {
    return a.fused == 2 ? launch_j<SLABS, BF16, true>(mq, mk, mv, mko, mvo, a, grid, st) : launch_j<SLABS, BF16, false>(mq, mk, mv, mko, mvo, a, grid, st);
}

}  // namespace

// Clusters of n CTAs of this kernel that the device holds at once (asked once per device; without a device: a B200 whose processor clusters leave
// 15 clusters of 8).
int q8_clusters(int n) {
    static const int usual[9] = {0, 148, 74, 45, 33, 26, 22, 15, 15};
    static std::atomic<int> seen[64][9];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return usual[n];
    int v = seen[dev][n].load(std::memory_order_relaxed);
    if (v > 0) return v;
    constexpr int smem = (2 + Rings<2>::WIDE) * 2 * kSlabBytes + Rings<2>::RAW * kSlabBytes + kBarBytes;
    static std::atomic<unsigned long long> set{0};
    if (!ensure_dynamic_smem(prefix_tiles_q8_kernel<2, true, true>, smem, set)) return usual[n];
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)n * 64);
    cfg.blockDim = dim3(kQThreads);
    cfg.dynamicSmemBytes = smem;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim = {(unsigned)n, 1u, 1u};
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaOccupancyMaxActiveClusters(&v, prefix_tiles_q8_kernel<2, true, true>, &cfg) != cudaSuccess || v < 1) {
        cudaGetLastError();
        v = usual[n];
    }
    seen[dev][n].store(v, std::memory_order_relaxed);
    return v;
}

int launch_prefix_tiles_q8(const void* q, const PrefixQ8& c, const int32_t* prefix_len, const void* k_own, const void* v_own,
                           const int32_t* own_len, const psd_attention_t& a, const PrefixPlan& p, bool joined, float* po, float* pl, void* out,
                           float* lse, int32_t* status_dev, cudaStream_t st) {
    CUtensorMap mq, mk, mv, mko, mvo;
    if (!make_query_map(&mq, q, a, p.tq) || !make_tile_map(&mk, c.k, a.kp, a.B, a.P, a.Hkv, a.Dh, p.dhp) ||
        !make_tile_map(&mv, c.v, a.vp, a.B, a.P, a.Hkv, a.Dh, p.dhp))
        return PSD_ERR_CUDA;
    const int own_box = a.S >= 128 ? 128 : (a.S + 15) / 16 * 16;
    if ((p.fused || joined) && a.S > 0) {
        if (!make_cache_map(&mko, k_own, a.dtype, a.ko, a.B * a.D, a.S, a.Hkv, a.Dh, own_box) ||
            !make_cache_map(&mvo, v_own, a.dtype, a.vo, a.B * a.D, a.S, a.Hkv, a.Dh, own_box))
            return PSD_ERR_CUDA;
    } else {
        mko = mk;
        mvo = mv;
    }
    const int64_t grid = (int64_t)a.B * a.Hkv * p.units * (p.n_qt > 1 ? p.splits : p.splits / 2);
    if (grid > INT32_MAX) return PSD_ERR_SHAPE;
    TcArgs x = {};
    x.k_scale = c.k_scale; x.v_scale = c.v_scale;
    x.prefix_len = prefix_len;
    x.po = po; x.pl = pl;
    x.status_dev = status_dev;
    x.rows = (int64_t)a.B * a.D * a.M * a.Hq;
    x.T = a.D * a.M; x.G = a.Hq / a.Hkv; x.Hq = a.Hq; x.Hkv = a.Hkv; x.Dh = a.Dh; x.P = a.P;
    x.nb = (a.P + c.block - 1) / c.block;
    x.shift = c.block == 16 ? 4 : c.block == 32 ? 5 : c.block == 64 ? 6 : 7;
    x.tq = p.tq; x.n_qt = p.n_qt; x.units = p.units; x.splits = p.splits;
    x.k_outer = a.kp.outer ? 1 : 0; x.k_head = a.kp.head ? 1 : 0;
    x.v_outer = a.vp.outer ? 1 : 0; x.v_head = a.vp.head ? 1 : 0;
    x.B = a.B;
    x.longest_first = prefix_len && a.B > 1 && a.B <= kMaxSorted && grid > sm_count() ? 1 : 0;
    x.fused = joined ? 2 : p.fused ? 1 : 0;
    x.n_cs = p.n_qt > 1 ? p.splits : p.splits / 2;
    x.D = a.D; x.M = a.M; x.S = a.S; x.causal = a.causal; x.own_box = own_box > 0 ? own_box : 16;
    x.ko_outer = a.ko.outer ? 1 : 0; x.ko_head = a.ko.head ? 1 : 0;
    x.vo_outer = a.vo.outer ? 1 : 0; x.vo_head = a.vo.head ? 1 : 0;
    x.own_len = own_len;
    x.out = out; x.lse = lse;
    x.out_token = a.out_token; x.out_head = a.out_head;
    x.c = a.scale * kLog2e;
    x.wait_limit = wait_limit_cycles();
    x.stall_test = selftest_stall();
    x.f16_codes = kF16Codes;
    x.bf16_codes = kBf16Codes;
    const bool bf16 = a.dtype == PSD_BF16;
    if (p.dhp == 64) return bf16 ? launch_t<1, true>(mq, mk, mv, mko, mvo, x, grid, st) : launch_t<1, false>(mq, mk, mv, mko, mvo, x, grid, st);
    return bf16 ? launch_t<2, true>(mq, mk, mv, mko, mvo, x, grid, st) : launch_t<2, false>(mq, mk, mv, mko, mvo, x, grid, st);
}

}  // namespace psd
