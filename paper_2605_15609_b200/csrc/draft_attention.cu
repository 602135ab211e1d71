// Attention of the drafts over the shared prefix and over each draft's own keys.
//
// One CTA takes up to 16 * WM rows (query tokens times the heads of one key head) of one draft and walks the keys in
// tiles of 64 with a running maximum and sum per row; WK = 4 / WM warps share a 16-row block and take 64 / WK keys of
// every tile each.  Products are m16n8k16 tensor instructions with fp32 accumulation: a draft has few keys of its own (a
// block of 32 or 64), and tiles of 128 keys shared with other drafts would let one draft's NaN reach another's rows.  K and
// V tiles are double-buffered by asynchronous copies that fill what lies past a length (or past Dh) with zeros, so nothing
// that was never written is multiplied.
//
// CODES: the prefix is a cache of 8-bit codes (prefix_attention_q8.cu), short enough to be walked here.  Its tiles are widened on their way to
// shared memory (keys to T, values to fp16; registers hold the next tile's codes meanwhile), scores are multiplied by their key's scale, weights by the
// value's, in fp16 and relative to the row's largest such product (w); outputs are relative to that until the first own tile.  While the value scales are
// close together (not `wide`) the largest weight and scale serve instead: 9.9 us against 10.4 (4 drafts of 32 tokens, 4 heads of 64, 257 keys).
//
// What the warps of a row block hold and the partial results over the prefix are then joined row by row, a warp per row
// and all lanes along Dh: the kernel's time is the traffic of those partial results (4 bytes per output element and split
// against 2 written), and this order reads and writes whole lines.
#include "attn_tc.cuh"
#include "prefix_attention.cuh"
#include "prefix_attention_q8.cuh"

namespace psd {
namespace {

constexpr int kKeys = 64;        // keys per tile
constexpr int kThreads = 128;

// ROOM: weights are kept 2^ROOM larger than relative to the row's maximum.  fp16 holds nothing below 2^-25, and thousands of keys
// that far below a maximum count together; with the largest weight at 2^15 nothing above 2^-40 of it is lost.
template <typename T> struct Mma;
template <> struct Mma<__nv_bfloat16> {
    static constexpr bool BF16 = true;
    static constexpr float ROOM = 0.f;
    static __device__ __forceinline__ void run(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    }
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        uint32_t r;
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
        return r;
    }
};
template <> struct Mma<__half> {
    static constexpr bool BF16 = false;
    static constexpr float ROOM = 15.f;
    static __device__ __forceinline__ void run(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    }
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        uint32_t r;
        asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
        return r;
    }
};

__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ void ldsm4_t(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ void cp16(uint32_t dst, const void* src, bool ok) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(ok ? 16 : 0) : "memory");
}

struct OwnArgs {
    const void *q, *kp, *vp, *ko, *vo;
    const int32_t *prefix_len, *own_len;
    void* out;
    float* lse;
    psd_attention_t a;
    int row_blocks;      // CTAs per (node, key head)
    int stages;          // tiles of keys in shared memory: 2 (the next one is loaded ahead) or 1
    // partial results over the prefix (prefix_attention.cu), or NULL: this kernel walks the prefix's keys itself
    const float *po, *pl;
    int splits;          // <= kMaxPrefixSplits
    int64_t rows;
    PrefixQ8 q8;         // CODES: the prefix
    int nb, shift;
    uint32_t f16_codes, bf16_codes;
};

// Joins the rows warp, warp + 4, .. of a CTA: WK warps' results in shared memory and the splits' in global memory, RB rows
// and SP splits at a time.  A warp per row, lanes along Dh.
template <typename T, int DHP, int WK, int RB, int SP>
__device__ __forceinline__ void join_rows(const OwnArgs& p, const float* so, const float* sm, int row0, int row_end, int node, int h,
                                          int warp, int lane) {
    constexpr int E = DHP / 32;                              // elements per lane: 2 or 4
    constexpr int OLD = DHP + 8;
    const psd_attention_t& a = p.a;
    const int G = a.Hq / a.Hkv;
    const bool in = lane * E < a.Dh;                         // columns past Dh were not written
    for (int r0 = warp; r0 < row_end; r0 += 4 * RB) {
        int64_t at[RB], t[RB];
        float z[RB][2], y[RB][SP][E];                        // log2-sums of splits lane, lane + 32; outputs of SP splits
        auto fetch = [&](int k, int x0) {
#pragma unroll
            for (int u = 0; u < SP; ++u) {
#pragma unroll
                for (int e = 0; e < E; ++e) y[k][u][e] = 0.f;
                if (in && x0 + u < p.splits) {
                    const float* po = p.po + ((x0 + u) * p.rows + at[k]) * DHP + lane * E;
                    if (E == 4) *reinterpret_cast<float4*>(y[k][u]) = __ldcs(reinterpret_cast<const float4*>(po));
                    else *reinterpret_cast<float2*>(y[k][u]) = __ldcs(reinterpret_cast<const float2*>(po));
                }
            }
        };
        int hh[RB];
#pragma unroll
        for (int k = 0; k < RB; ++k) {
            const int rr = row0 + min(r0 + 4 * k, row_end - 1), i = rr / G;
            hh[k] = h * G + rr % G;
            t[k] = (int64_t)node * a.M + i;
            at[k] = t[k] * a.Hq + hh[k];
#pragma unroll
            for (int q = 0; q < 2; ++q) z[k][q] = lane + 32 * q < p.splits ? p.pl[(lane + 32 * q) * p.rows + at[k]] : -INFINITY;
            fetch(k, 0);
        }
#pragma unroll
        for (int k = 0; k < RB; ++k) {
            const int r = r0 + 4 * k;
            if (r >= row_end) break;
            float top = fmaxf(z[k][0], z[k][1]);
#pragma unroll
            for (int x = 16; x; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
            const int r16 = (r / 16) * WK * 16 + r % 16;     // this row in the first of its warps
#pragma unroll
            for (int w = 0; w < WK; ++w) top = fmaxf(top, sm[r16 + w * 16]);
            const float base = top == -INFINITY ? 0.f : top;
            float acc[E], sum = 0.f;
#pragma unroll
            for (int e = 0; e < E; ++e) acc[e] = 0.f;
#pragma unroll
            for (int w = 0; w < WK; ++w) {
                const float f = ex2(sm[r16 + w * 16] - base);
                sum = fmaf(f, sm[64 + r16 + w * 16], sum);
#pragma unroll
                for (int e = 0; e < E; ++e) acc[e] = fmaf(f, so[(r16 + w * 16) * OLD + lane * E + e], acc[e]);
            }
#pragma unroll 1
            for (int x0 = 0; x0 < p.splits; x0 += SP) {
                if (x0) fetch(k, x0);
#pragma unroll
                for (int u = 0; u < SP; ++u) {
                    const int x = x0 + u;
                    const float zx = __shfl_sync(0xffffffffu, x < 32 ? z[k][0] : z[k][1], x & 31);
                    if (x < p.splits && zx != -INFINITY) {
                        const float wt = ex2(zx - base);
                        sum += wt;
#pragma unroll
                        for (int e = 0; e < E; ++e) acc[e] = fmaf(wt, y[k][u][e], acc[e]);
                    }
                }
            }
            const bool none = top == -INFINITY && sum == 0.f;
            const float inv = none ? 0.f : 1.f / sum;
            if (in) {
                uint32_t pk[E / 2];
#pragma unroll
                for (int e = 0; e < E / 2; ++e) pk[e] = Mma<T>::pack(acc[2 * e] * inv, acc[2 * e + 1] * inv);
                T* out = reinterpret_cast<T*>(p.out) + t[k] * a.out_token + (int64_t)hh[k] * a.out_head + lane * E;
                if (E == 4) *reinterpret_cast<uint2*>(out) = make_uint2(pk[0], pk[E / 2 - 1]);
                else *reinterpret_cast<uint32_t*>(out) = pk[0];
            }
            if (p.lse && lane == 0) p.lse[at[k]] = none ? -INFINITY : top * kLn2 + logf(sum);
        }
    }
}

template <typename T, int DHP, int WM, bool CODES>
__global__ void __launch_bounds__(kThreads, WM == 1 && !CODES ? 4 : 3) draft_attention_kernel(const OwnArgs p) {
    constexpr bool BF16 = Mma<T>::BF16;
    constexpr float OWN_ROOM = Mma<T>::ROOM, ROOM = CODES ? 15.f : OWN_ROOM;         // (weights over codes are fp16)
    constexpr int WK = 4 / WM, KPW = kKeys / WK;      // warps per row block, keys per warp and tile
    constexpr int LD = DHP + 8;                        // padded row of a tile (bank-conflict-free ldmatrix)
    constexpr int NQ = DHP / 16, NO = DHP / 8, NS = KPW / 8;
    extern __shared__ __align__(16) unsigned char smem[];
    T* tiles = reinterpret_cast<T*>(smem);             // [2 stages][K, V][kKeys][LD]
    const psd_attention_t& a = p.a;
    const int G = a.Hq / a.Hkv, rows = a.M * G;
    const int rb = blockIdx.x % p.row_blocks;
    const int nh = blockIdx.x / p.row_blocks, h = nh % a.Hkv, node = nh / a.Hkv, b = node / a.D;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int wm = warp / WK, wk = warp % WK;
    const int r0 = rb * 16 * WM + wm * 16 + (lane >> 2);       // this thread's rows: r0 and r0 + 8
    // With partial results the kernel before this one is the prefix's, which has itself waited for whatever wrote the
    // inputs; only its results are waited for, below.
    if (!p.po) asm volatile("griddepcontrol.wait;" ::: "memory");
    const int Lp = a.P == 0 || p.po ? 0 : p.prefix_len ? min(max(p.prefix_len[b], 0), a.P) : a.P;
    const int Lo = a.S == 0 ? 0 : p.own_len ? min(max(p.own_len[node], 0), a.S) : a.S;

    // query fragments straight from global memory
    uint32_t qf[NQ][4];
    int64_t q_at[2];
    bool live[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int r = r0 + 8 * u;
        live[u] = r < rows;
        const int i = live[u] ? r / G : 0, g = live[u] ? r % G : 0;
        q_at[u] = ((int64_t)node * a.M + i) * a.q_token + (int64_t)(h * G + g) * a.q_head;
    }
#pragma unroll
    for (int kk = 0; kk < NQ; ++kk)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int u = e & 1, d = kk * 16 + (lane & 3) * 2 + (e >> 1) * 8;
            qf[kk][e] = live[u] && d < a.Dh ? *reinterpret_cast<const uint32_t*>(reinterpret_cast<const T*>(p.q) + q_at[u] + d) : 0u;
        }
    float o[NO][4];
#pragma unroll
    for (int n = 0; n < NO; ++n) o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.f;
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
    float w[2] = {-INFINITY, -INFINITY};               // CODES: maximum of scores plus log2 of their value's scale relative to vref (not `wide`: m)
    const float scale2 = a.scale * kLog2e;
    // own keys visible to this thread's rows
    int own_seen[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int i = (r0 + 8 * u) / G;
        own_seen[u] = a.causal ? min(Lo, Lo - a.M + 1 + i) : Lo;
    }

    const int tp = (Lp + kKeys - 1) / kKeys, tiles_n = tp + (Lo + kKeys - 1) / kKeys;
    auto fetch = [&](int t, int stage) {
        const bool own = t >= tp;
        const int j0 = (own ? t - tp : t) * kKeys, len = own ? Lo : Lp;
        const psd_kv_strides_t &sk = own ? a.ko : a.kp, &sv = own ? a.vo : a.vp;
        const T* kb = reinterpret_cast<const T*>(own ? p.ko : p.kp) + (own ? node : b) * sk.outer + h * sk.head;
        const T* vb = reinterpret_cast<const T*>(own ? p.vo : p.vp) + (own ? node : b) * sv.outer + h * sv.head;
        T* dk = tiles + stage * 2 * kKeys * LD;
        constexpr int C = DHP / 8;
#pragma unroll
        for (int x = threadIdx.x; x < kKeys * C; x += kThreads) {
            const int r = x / C, c = (x % C) * 8, j = j0 + r;
            const bool ok = j < len && c < a.Dh;
            const int64_t jj = ok ? j : 0;
            cp16(smem_u32(dk + r * LD + c), kb + jj * sk.token + (ok ? c : 0), ok);
            cp16(smem_u32(dk + (kKeys + r) * LD + c), vb + jj * sv.token + (ok ? c : 0), ok);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    const bool ahead = p.stages == 2;
    if (ahead && tiles_n > 0 && (!CODES || tp == 0)) fetch(0, 0);
    // CODES: a tile's codes and scales, between memory and shared memory
    constexpr int PIECES = kKeys * (DHP / 8) / kThreads;                      // of 8 codes, a thread's, of keys and as many of values
    // (a scale serves 16 keys at least: [0] the keys', [1] the values', [2] its logarithm)
    __shared__ float scales[3][CODES ? kKeys / 16 : 1];
    uint2 codes[CODES ? 2 * PIECES : 1];
    float scale_kv = 0.f, vref = 1.17549435e-38f, vlow = INFINITY, vinv = 0.f;
    bool wide = false;
    const float *ks = nullptr, *vs = nullptr;
    auto load_codes = [&](int t) {
        const int8_t* kb = p.q8.k + b * a.kp.outer + h * a.kp.head;
        const int8_t* vb = p.q8.v + b * a.vp.outer + h * a.vp.head;
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int x = threadIdx.x + i * kThreads, c = x % (DHP / 8) * 8, j = t * kKeys + x / (DHP / 8);
            const bool ok = j < Lp && c < a.Dh;
            codes[i] = ok ? *reinterpret_cast<const uint2*>(kb + j * a.kp.token + c) : make_uint2(0u, 0u);
            codes[PIECES + i] = ok ? *reinterpret_cast<const uint2*>(vb + j * a.vp.token + c) : make_uint2(0u, 0u);
        }
        // threads 0 .. 3: the keys' scales, 4 .. 11: the values'; those of keys past the end were never written
        const int j = t * kKeys + threadIdx.x % 4 * 16;
        scale_kv = 0.f;
        if (threadIdx.x < 12 && j < Lp) {
            scale_kv = threadIdx.x < 4 ? ks[j >> p.shift] * scale2 : vs[j >> p.shift] * vinv;
            if (threadIdx.x < 4 && scale_kv == 0.f) scale_kv = 1.17549435e-38f;
        }
    };
    auto store_codes = [&](int stage) {
        T* dk = tiles + stage * 2 * kKeys * LD;
        auto pair = [&](uint32_t w, uint32_t sel, bool bf16) {
            const uint32_t x = __byte_perm(w, 0u, sel);
            return bf16 ? codes_bf16(x, p.bf16_codes) : codes_f16(x, p.f16_codes);
        };
#pragma unroll
        for (int i = 0; i < 2 * PIECES; ++i) {
            const int x = threadIdx.x + i % PIECES * kThreads, c = x % (DHP / 8) * 8, r = x / (DHP / 8) + (i < PIECES ? 0 : kKeys);
            const bool bf16 = BF16 && i < PIECES;
            *reinterpret_cast<uint4*>(dk + r * LD + c) = make_uint4(pair(codes[i].x, 0x1100, bf16), pair(codes[i].x, 0x3322, bf16),
                                                                     pair(codes[i].y, 0x1100, bf16), pair(codes[i].y, 0x3322, bf16));
        }
        if (threadIdx.x < 12) scales[threadIdx.x / 4][threadIdx.x % 4] = threadIdx.x < 8 ? scale_kv : lg2(scale_kv);
    };
    if (CODES && Lp > 0) {
        ks = p.q8.k_scale + ((int64_t)b * a.Hkv + h) * p.nb;
        vs = p.q8.v_scale + ((int64_t)b * a.Hkv + h) * p.nb;
        for (int j = lane; j <= (Lp - 1) >> p.shift; j += 32) {
            const float x = vs[j];
            vref = fmaxf(vref, x);
            vlow = fminf(vlow, x);
        }
#pragma unroll
        for (int x = 16; x; x >>= 1) vref = fmaxf(vref, __shfl_xor_sync(0xffffffffu, vref, x));
        wide = __any_sync(0xffffffffu, vlow < vref * kNear);
        vinv = 1.f / vref;
        load_codes(0);
    }
    for (int t = 0; t < tiles_n; ++t) {
        const bool coded = CODES && t < tp;
        if (coded) {
            store_codes(ahead ? t & 1 : 0);
            if (t + 1 < tp) load_codes(t + 1);
        } else if (!ahead) {
            fetch(t, 0);
        }
        if (ahead && t + 1 < tiles_n && !(CODES && t + 1 < tp)) {
            fetch(t + 1, (t + 1) & 1);
            asm volatile("cp.async.wait_group 1;" ::: "memory");
        } else {
            asm volatile("cp.async.wait_group 0;" ::: "memory");
        }
        __syncthreads();
        const T* kt = tiles + (ahead ? t & 1 : 0) * 2 * kKeys * LD + wk * KPW * LD;
        const T* vt = kt + kKeys * LD;
        float s[NS][4];
#pragma unroll
        for (int n = 0; n < NS; ++n) s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.f;
#pragma unroll
        for (int kk = 0; kk < NQ; kk += 2)
#pragma unroll
            for (int n = 0; n < NS; ++n) {
                uint32_t r[4];
                ldsm4(r, smem_u32(kt + (n * 8 + (lane & 7)) * LD + kk * 16 + (lane >> 3) * 8));
                Mma<T>::run(s[n], qf[kk], r[0], r[1]);
                Mma<T>::run(s[n], qf[kk + 1], r[2], r[3]);
            }
        // masks: keys past the length, and own keys that this row does not see
        const bool own = t >= tp;
        const int j0 = (own ? t - tp : t) * kKeys + wk * KPW + (lane & 3) * 2;
        float mx[2] = {m[0], m[1]}, mw[2] = {w[0], w[1]};
        auto scale_at = [&](int which, int n) { return scales[which][(wk * KPW + n * 8) / 16 % (CODES ? kKeys / 16 : 1)]; };
#pragma unroll
        for (int n = 0; n < NS; ++n) {
            const float by = coded ? scale_at(0, n) : scale2;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int j = j0 + n * 8 + (e & 1);
                s[n][e] = j < (own ? own_seen[e >> 1] : Lp) ? s[n][e] * by : -INFINITY;
                mx[e >> 1] = fmaxf(mx[e >> 1], s[n][e]);
            }
            if (n % 2 && coded && wide) {
                const float log = scale_at(2, n);
#pragma unroll
                for (int u = 0; u < 2; ++u)
                    mw[u] = fmaxf(mw[u], fmaxf(max3(s[n - 1][2 * u], s[n - 1][2 * u + 1], s[n][2 * u]), s[n][2 * u + 1]) + log);
            }
        }
        float f[2], base[2], gain[2] = {1.f, 1.f};
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            mx[u] = fmaxf(mx[u], __shfl_xor_sync(0xffffffffu, mx[u], 1));
            mx[u] = fmaxf(mx[u], __shfl_xor_sync(0xffffffffu, mx[u], 2));
            f[u] = m[u] == mx[u] ? 1.f : ex2(m[u] - mx[u]);
            base[u] = mx[u] == -INFINITY ? 0.f : mx[u] - (own ? OWN_ROOM : ROOM);
            m[u] = mx[u];
            l[u] *= f[u];
            if (coded && !wide) {
                w[u] = m[u];
            } else if (coded) {
                mw[u] = fmaxf(mw[u], __shfl_xor_sync(0xffffffffu, mw[u], 1));
                mw[u] = fmaxf(mw[u], __shfl_xor_sync(0xffffffffu, mw[u], 2));
                mw[u] = fmaxf(mw[u], m[u] - kFar);
                f[u] = mw[u] == w[u] ? 1.f : ex2(w[u] - mw[u]);
                w[u] = mw[u];
                gain[u] = ex2(fminf(m[u] - w[u], kFar));
            } else if (CODES && t == tp && t > 0) {                // the first own tile: from here on outputs are relative to m and 1
                l[u] *= ex2(OWN_ROOM - ROOM);
                f[u] = w[u] == -INFINITY ? 1.f : times_ex2(vref, w[u] - m[u] + (OWN_ROOM - ROOM));
            }
        }
#pragma unroll
        for (int n = 0; n < NO; ++n) {
            o[n][0] *= f[0]; o[n][1] *= f[0]; o[n][2] *= f[1]; o[n][3] *= f[1];
        }
#pragma unroll
        for (int n = 0; n < NS; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                s[n][e] = ex2(s[n][e] - base[e >> 1]);
                l[e >> 1] += s[n][e];
                if (coded) s[n][e] *= scale_at(1, n) * gain[e >> 1];
            }
#pragma unroll
        for (int kb = 0; kb < KPW / 16; ++kb) {
            if (coded) {
                const uint32_t pa[4] = {Mma<__half>::pack(s[2 * kb][0], s[2 * kb][1]), Mma<__half>::pack(s[2 * kb][2], s[2 * kb][3]),
                                        Mma<__half>::pack(s[2 * kb + 1][0], s[2 * kb + 1][1]), Mma<__half>::pack(s[2 * kb + 1][2], s[2 * kb + 1][3])};
#pragma unroll
                for (int n = 0; n < NO; n += 2) {
                    uint32_t r[4];
                    ldsm4_t(r, smem_u32(vt + (kb * 16 + (lane & 15)) * LD + n * 8 + (lane >> 4) * 8));
                    Mma<__half>::run(o[n], pa, r[0], r[1]);
                    Mma<__half>::run(o[n + 1], pa, r[2], r[3]);
                }
                continue;
            }
            const uint32_t pa[4] = {Mma<T>::pack(s[2 * kb][0], s[2 * kb][1]), Mma<T>::pack(s[2 * kb][2], s[2 * kb][3]),
                                    Mma<T>::pack(s[2 * kb + 1][0], s[2 * kb + 1][1]), Mma<T>::pack(s[2 * kb + 1][2], s[2 * kb + 1][3])};
#pragma unroll
            for (int n = 0; n < NO; n += 2) {
                uint32_t r[4];
                ldsm4_t(r, smem_u32(vt + (kb * 16 + (lane & 15)) * LD + n * 8 + (lane >> 4) * 8));
                Mma<T>::run(o[n], pa, r[0], r[1]);
                Mma<T>::run(o[n + 1], pa, r[2], r[3]);
            }
        }
        __syncthreads();
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        l[u] += __shfl_xor_sync(0xffffffffu, l[u], 1);
        l[u] += __shfl_xor_sync(0xffffffffu, l[u], 2);
    }
    const bool only_codes = CODES && tiles_n == tp;          // no own tile came: relative to m and 1 now
    if (only_codes) {
        float f[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            f[u] = w[u] == -INFINITY ? 1.f : times_ex2(vref, w[u] - m[u] - ROOM);
            l[u] *= ex2(-ROOM);
        }
#pragma unroll
        for (int n = 0; n < NO; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[n][e] *= f[e >> 1];
    }
    // every warp's rows to shared memory (the tiles are no longer needed: the loop ends with a barrier)
    constexpr int OLD = DHP + 8;                             // padded row: the float2 stores of 8 rows hit different banks
    float* so = reinterpret_cast<float*>(smem);              // [4 warps][16][OLD]
    float* sm = so + 4 * 16 * OLD;                           // [4 warps][16] references, then sums
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int r = warp * 16 + (lane >> 2) + 8 * u;
#pragma unroll
        for (int n = 0; n < NO; ++n)
            *reinterpret_cast<float2*>(&so[r * OLD + n * 8 + (lane & 3) * 2]) = make_float2(o[n][2 * u], o[n][2 * u + 1]);
        if ((lane & 3) == 0) {
            sm[r] = m[u] - (only_codes ? 0.f : OWN_ROOM);      // what outputs and sums are relative to
            sm[64 + r] = l[u];
        }
    }
    __syncthreads();
    if (p.po) asm volatile("griddepcontrol.wait;" ::: "memory");
    // out = (sum_w 2^(m_w-T) O_w + sum_x 2^(z_x-T) P_x) / (sum_w 2^(m_w-T) l_w + sum_x 2^(z_x-T)), in this order
    const int row_end = min(16 * WM, rows - rb * 16 * WM);
    // Few splits: several rows at a time, their loads issued together and before it is known which splits hold keys
    // (what a split without keys did not write is loaded and dropped).  Many splits: eight splits at a time.
    if (p.splits <= 2) join_rows<T, DHP, WK, 4, 2>(p, so, sm, rb * 16 * WM, row_end, node, h, warp, lane);
    else join_rows<T, DHP, WK, 1, 8>(p, so, sm, rb * 16 * WM, row_end, node, h, warp, lane);
}

template <typename T, int DHP, int WM, bool CODES>
int launch_rows(OwnArgs& p, cudaStream_t st) {
    const psd_attention_t& a = p.a;
    const int rows = a.M * (a.Hq / a.Hkv);
    p.row_blocks = (rows + 16 * WM - 1) / (16 * WM);
    const int64_t grid = (int64_t)a.B * a.D * a.Hkv * p.row_blocks;
    if (grid > INT32_MAX) return PSD_ERR_SHAPE;
    const int64_t tiles = (int64_t)(p.po ? 0 : (a.P + kKeys - 1) / kKeys) + (a.S + kKeys - 1) / kKeys;
    // one stage where more CTAs than fit with two want to be resident: the others' arithmetic then hides a CTA's loads
    p.stages = tiles > 1 && grid <= 3 * sm_count() ? 2 : 1;
    constexpr int tile_bytes = 2 * kKeys * (DHP + 8) * 2, join_bytes = (4 * 16 * (DHP + 8) + 4 * 16 * 2) * 4;
    const int smem = p.stages * tile_bytes > join_bytes ? p.stages * tile_bytes : join_bytes;
    static std::atomic<unsigned long long> set{0};
    if (!ensure_dynamic_smem(draft_attention_kernel<T, DHP, WM, CODES>, 2 * tile_bytes, set)) return PSD_ERR_CUDA;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = pdl_enabled() ? 1 : 0;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, draft_attention_kernel<T, DHP, WM, CODES>, (const OwnArgs)p);
    count_launch();
    return e == cudaSuccess ? PSD_OK : PSD_ERR_CUDA;
}
// Rows per CTA, in blocks of 16: 64 where that still gives every SM two CTAs, fewer otherwise (then four warps share the keys
// and the join of a row block).
int row_blocks_per_cta(int64_t nodes_heads, int rows) {
    const int64_t want = 2 * sm_count();
    if (rows > 32 && nodes_heads * ((rows + 63) / 64) >= want) return 4;
    if (rows > 16 && nodes_heads * ((rows + 31) / 32) >= want) return 2;
    return 1;
}

// Whether this kernel walks the prefix too, in one launch: it reads the prefix once per draft instead of once per sequence, but
// saves a launch and the join.  It does while a wave of its CTAs (three per SM) has few tiles of 64 keys to walk: measured, one
// launch against two, 4 drafts of 32 tokens: 4 heads of 64, prefix 257: 7 against 15 us, 1024: 14 against 17, 1536: 18 against
// 17, 2048: 23 against 17; 32 heads of 128 over 8 key heads, prefix 257: 14 against 16 us, 512: 18 against 20, 768: 24 against 22;
// the same heads, drafts of 2 tokens, 257: 11 against 14, 512: 14 against 14, 1024: 24 against 15; 16 sequences of one token, 512:
// 14 against 17, 1024: 24 against 22.
// Where the tensor-core kernel can take the own keys as well, it is one launch too and wins with rows for a third of the SMs (a CTA
// has up to 256; 8 sequences of 8 drafts of 4 tokens, 16 heads of 128 over 2, prefix 257, 16 CTAs: 24 against 14 us): 32 heads of 128 over 8, 4
// drafts of 32 tokens, prefix 128: 4 sequences 13 against 26 us, 16 sequences 28 against 63, 32 sequences 50 against 109; 8
// sequences, 32 heads of 64 over 4, prefix 512: 17 against 50.  It then loses only while the prefix is short and its tiles hold
// several drafts, each a tile of own keys: 5 sequences of 4 drafts of 33 tokens, 16 heads of 64, prefix 64: 17 against 11, 257: 21
// against 19, 512: 22 against 25, heads of 128, prefix 64: 18 against 17, 128: 18 against 20, 257: 23 against 30.
int one_launch_tiles(int Dh) { return Dh <= 64 ? 16 : 8; }
bool one_launch(int B, int D, int M, int Hq, int Hkv, int Dh, int P, int S) {
    const PrefixPlan plan = plan_prefix(B, D, M, Hq, Hkv, Dh, P, S);
    if (P > 0 && plan.fused && 3 * (int64_t)B * Hkv * plan.units >= sm_count() &&
        (P > (Dh <= 64 ? 320 : 128) || drafts_per_tile(M, plan.tq) < 4))
        return false;
    const int rows = M * (Hq / Hkv);
    const int64_t nh = (int64_t)B * D * Hkv;
    const int r = 16 * row_blocks_per_cta(nh, rows);
    const int64_t ctas = nh * ((rows + r - 1) / r), waves = (ctas + 3 * sm_count() - 1) / (3 * sm_count());
    return waves * ((P + kKeys - 1) / kKeys) <= one_launch_tiles(Dh);
}

template <typename T, int DHP, bool CODES = false>
int launch_dh(OwnArgs& p, cudaStream_t st) {
    switch (row_blocks_per_cta((int64_t)p.a.B * p.a.D * p.a.Hkv, p.a.M * (p.a.Hq / p.a.Hkv))) {
        case 4: return launch_rows<T, DHP, 4, CODES>(p, st);
        case 2: return launch_rows<T, DHP, 2, CODES>(p, st);
        default: return launch_rows<T, DHP, 1, CODES>(p, st);
    }
}

}  // namespace

// Bytes of `rows` partial results, rounded up.
static size_t partial_bytes(int64_t rows, int dhp) { return rows == 0 ? 256 : ((size_t)rows * (dhp + 1) * 4 + 255) / 256 * 256; }

size_t draft_attention_needs(int B, int D, int M, int Hq, int Hkv, int Dh, int P, int S) {
    if (one_launch(B, D, M, Hq, Hkv, Dh, P, S)) return 256;
    const PrefixPlan p = plan_prefix(B, D, M, Hq, Hkv, Dh, P, S);
    return partial_bytes(p.fused ? 0 : (int64_t)B * D * M * Hq * p.splits, p.dhp);
}

// What these sizes and all with smaller B, D, P and S need at most: a large batch may need nothing where a small one splits its
// keys, and a caller whose batch shrinks keeps its workspace.  Two bounds on the partial results of a split form: its CTAs fill the
// SMs once (2 * 128 rows each), and the splits are bounded by the prefix.
size_t draft_attention_workspace(int B, int D, int M, int Hq, int Hkv, int Dh, int P, int S) {
    const int64_t sms = sm_count(), G = Hq / Hkv, tq = 128 / G, T = (int64_t)D * M, tiles = (P + 127) / 128;
    const int64_t once = 2 * sms * tq * G, rows = (int64_t)B * T * Hq;
    const int dhp = Dh <= 64 ? 64 : 128;
    // One launch (or no partial results) at every smaller size: smaller batches use smaller blocks of rows, but then at most 4 CTAs per SM, two waves.
    const int most = M * (int)G > 32 ? 64 : M * (int)G > 16 ? 32 : 16;
    const int64_t ctas = (int64_t)B * D * Hkv * ((M * G + most - 1) / most), waves = (ctas + 3 * sms - 1) / (3 * sms);
    if ((waves < 2 ? 2 : waves) * ((P + kKeys - 1) / kKeys) <= one_launch_tiles(Dh)) return 256;
    auto least = [](int64_t a, int64_t b) { return a < b ? a : b; };
    auto larger = [](int64_t a, int64_t b) { return a > b ? a : b; };
    int64_t partial = 0;
    if (M <= tq) {
        // one query tile, at least two splits
        const int64_t r = (int64_t)B * least(T, tq) * Hq;
        partial = least(r * larger(2, least(tiles / 2, kMaxPrefixSplits)), larger(2 * r, once));
    }
    if (T > tq) {
        if (!fuses_own(M, (int)tq, S)) partial = larger(partial, rows);
        if (tiles >= 4) partial = larger(partial, least(rows * least(tiles / 2, kMaxPrefixSplits), once));
    }
    const size_t all = partial_bytes(partial, dhp), here = draft_attention_needs(B, D, M, Hq, Hkv, Dh, P, S);
    return all > here ? all : here;
}

const char* draft_attention_kernels(int B, int D, int M, int Hq, int Hkv, int Dh, int P, int S, int32_t* splits) {
    if (one_launch(B, D, M, Hq, Hkv, Dh, P, S)) {
        if (splits) *splits = 0;
        return "draft_attention_kernel";
    }
    const PrefixPlan p = plan_prefix(B, D, M, Hq, Hkv, Dh, P, S);
    if (splits) *splits = p.splits;
    return p.fused ? "prefix_attention_kernel" : "prefix_attention_kernel+draft_attention_kernel";
}

// Whether this kernel walks a prefix in codes too: while it is short (a tile takes 1.6 us of a CTA, 0.8 with heads of 64, and more the more CTAs share an
// SM), against what else there is: two launches for few rows of a key head, else the tcgen05 kernel.  Measured in us, this against that, 32 heads of 128 over 8:
// one token, prefix 128: 8.1, 8.4; 257: 13.0, 10.7; 4 drafts of 32 tokens, 64: 9.7, 13.1; 257: 17.7, 17.5; 768: 32.2, 23.0.
// Beyond four CTAs per SM (drafts in the hundreds over a few keys) the forms' times follow their waves of CTAs, and the lower estimate wins: fitted to
// 240 drawn shapes of up to 700 keys, 5 to 250 us, which each estimate meets within 15%.  Over 81 other shapes the rule takes 12.8 us on average (geometric),
// always the better form 12.7.
bool one_launch_codes(int B, int D, int M, int Hq, int Hkv, int Dh, int P, int S) {
    const PrefixPlan plan = plan_prefix(B, D, M, Hq, Hkv, Dh, P, S);
    const int rows = M * (Hq / Hkv), sms = sm_count(), steps = (P + kKeys - 1) / kKeys, own = (S + kKeys - 1) / kKeys;
    const bool few = (int64_t)D * rows <= 32;
    const int64_t nh = (int64_t)B * D * Hkv;
    const int blocks = row_blocks_per_cta(nh, rows), r = 16 * blocks;
    const int64_t ctas = nh * ((rows + r - 1) / r);
    if (ctas > 4 * sms) {
        const double half = Dh <= 64 ? 0.5 : 1, x = half * ctas * blocks / sms, y = half * ctas / sms;      // (blocks of rows, CTAs) per SM
        const double one = 3.8 + 0.7 * y + x * (0.55 + 0.6 * (steps + own)) + 0.37 * half * (steps + own);
        if (few) {
            const double z = (double)B * Hkv / sms;
            return one < 6.8 + z * (D * rows > 16 ? 1.36 + 2 * half * (1.9 + 0.26 * steps) : half * (1.9 + 0.26 * steps)) + 0.6 * x * (1 + own);
        }
        const double waves = (double)(((int64_t)B * Hkv * plan.units + sms - 1) / sms), tiles = (P + 127) / 128;
        const int met = plan.tq / M < 1 ? 1 : plan.tq / M < D ? plan.tq / M : D;
        return one < (plan.fused ? 1.5 + waves * (9 + 2.3 * tiles + 1.6 * met * ((S + 127) / 128)) : 5.1 + waves * (6.5 + 1.55 * tiles) + 0.8 * x * (1 + own));
    }
    if (plan.fused && 3 * (int64_t)B * Hkv * plan.units >= sms && (P > (Dh <= 64 ? 320 : 128) || drafts_per_tile(M, plan.tq) < 4)) return false;
    const int crowd = ctas <= 2 * sms ? 1 : ctas <= 3 * sms ? 2 : 4;
    return (int64_t)crowd * steps <= (Dh <= 64 ? few ? 6 : 8 : few ? 4 : 5);
}

int launch_codes_and_own(const void* q, const PrefixQ8& c, const int32_t* prefix_len, const void* k_own, const void* v_own, const int32_t* own_len,
                         const psd_attention_t& a, void* out, float* lse, cudaStream_t st) {
    OwnArgs p = {q, nullptr, nullptr, k_own, v_own, prefix_len, own_len, out, lse, a, 0, 1, nullptr, nullptr, 0, 0, c, (a.P + c.block - 1) / c.block,
                 c.block == 16 ? 4 : c.block == 32 ? 5 : c.block == 64 ? 6 : 7, kF16Codes, kBf16Codes};
    if (a.dtype == PSD_BF16) return a.Dh <= 64 ? launch_dh<__nv_bfloat16, 64, true>(p, st) : launch_dh<__nv_bfloat16, 128, true>(p, st);
    return a.Dh <= 64 ? launch_dh<__half, 64, true>(p, st) : launch_dh<__half, 128, true>(p, st);
}

int launch_own_and_join(const void* q, const void* k_own, const void* v_own, const int32_t* own_len, const psd_attention_t& a,
                        const float* po, const float* pl, int splits, void* out, float* lse, cudaStream_t st) {
    OwnArgs p = {q, nullptr, nullptr, k_own, v_own, nullptr, own_len, out, lse, a, 0, 1, po, pl, splits, (int64_t)a.B * a.D * a.M * a.Hq, {}, 0, 0, 0, 0};
    if (a.dtype == PSD_BF16) return a.Dh <= 64 ? launch_dh<__nv_bfloat16, 64>(p, st) : launch_dh<__nv_bfloat16, 128>(p, st);
    return a.Dh <= 64 ? launch_dh<__half, 64>(p, st) : launch_dh<__half, 128>(p, st);
}

int launch_draft_attention(const void* q, const void* k_prefix, const void* v_prefix, const int32_t* prefix_len,
                           const void* k_own, const void* v_own, const int32_t* own_len, const psd_attention_t& a,
                           void* out, float* lse, void* workspace, int32_t* status_dev, cudaStream_t st) {
    OwnArgs p = {q, k_prefix, v_prefix, k_own, v_own, prefix_len, own_len, out, lse, a, 0, 1, nullptr, nullptr, 0, 0, {}, 0, 0, 0, 0};
    if (!one_launch(a.B, a.D, a.M, a.Hq, a.Hkv, a.Dh, a.P, a.S)) {
        const PrefixPlan plan = plan_prefix(a.B, a.D, a.M, a.Hq, a.Hkv, a.Dh, a.P, a.S);
        p.rows = (int64_t)a.B * a.D * a.M * a.Hq;
        float* po = reinterpret_cast<float*>(workspace);
        float* pl = po + p.rows * plan.splits * plan.dhp;
        const int e = launch_prefix_attention(q, k_prefix, v_prefix, prefix_len, k_own, v_own, own_len, a, plan, po, pl, out, lse,
                                              status_dev, st);
        if (e != PSD_OK || plan.fused) return e;
        p.po = po;
        p.pl = pl;
        p.splits = plan.splits;
    }
    if (a.dtype == PSD_BF16) return a.Dh <= 64 ? launch_dh<__nv_bfloat16, 64>(p, st) : launch_dh<__nv_bfloat16, 128>(p, st);
    return a.Dh <= 64 ? launch_dh<__half, 64>(p, st) : launch_dh<__half, 128>(p, st);
}

}  // namespace psd
