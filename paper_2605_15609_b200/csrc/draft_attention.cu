// Attention of the drafts over the shared prefix and over each draft's own keys.
//
// One CTA takes up to 16 * WM rows (query tokens times the heads of one key head) of one draft and walks the keys in
// tiles of 64 with a running maximum and sum per row; WK = 4 / WM warps share a 16-row block and take 64 / WK keys of
// every tile each, and join their maxima, sums and outputs at the end.  Products are m16n8k16 tensor instructions with
// fp32 accumulation; K and V tiles are double-buffered by asynchronous copies that fill what lies past a length (or past
// Dh) with zeros, so nothing that was never written is multiplied, and a CTA only ever reads its own draft's keys.
#include "attn_tc.cuh"
#include "prefix_attention.cuh"

namespace psd {
namespace {

constexpr int kKeys = 64;        // keys per tile
constexpr int kThreads = 128;

template <typename T> struct Mma;
template <> struct Mma<__nv_bfloat16> {
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
    // partial results over the prefix (prefix_attention.cu), or NULL: this kernel walks the prefix's keys itself
    const float *po, *pl;
    int splits, dhp;
    int64_t rows;
};

template <typename T, int DHP, int WM>
__global__ void __launch_bounds__(kThreads) draft_attention_kernel(const OwnArgs p) {
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
    if (tiles_n > 0) fetch(0, 0);
    for (int t = 0; t < tiles_n; ++t) {
        if (t + 1 < tiles_n) {
            fetch(t + 1, (t + 1) & 1);
            asm volatile("cp.async.wait_group 1;" ::: "memory");
        } else {
            asm volatile("cp.async.wait_group 0;" ::: "memory");
        }
        __syncthreads();
        const T* kt = tiles + (t & 1) * 2 * kKeys * LD + wk * KPW * LD;
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
        float mx[2] = {m[0], m[1]};
#pragma unroll
        for (int n = 0; n < NS; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int j = j0 + n * 8 + (e & 1);
                s[n][e] = j < (own ? own_seen[e >> 1] : Lp) ? s[n][e] * scale2 : -INFINITY;
                mx[e >> 1] = fmaxf(mx[e >> 1], s[n][e]);
            }
        float f[2], base[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            mx[u] = fmaxf(mx[u], __shfl_xor_sync(0xffffffffu, mx[u], 1));
            mx[u] = fmaxf(mx[u], __shfl_xor_sync(0xffffffffu, mx[u], 2));
            base[u] = mx[u] == -INFINITY ? 0.f : mx[u];
            f[u] = m[u] == mx[u] ? 1.f : ex2(m[u] - base[u]);
            m[u] = mx[u];
            l[u] *= f[u];
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
            }
#pragma unroll
        for (int kb = 0; kb < KPW / 16; ++kb) {
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
    if (WK > 1) {
        // join the warps of a row block: maxima and sums first, then the outputs, in warp order
        float* sm = reinterpret_cast<float*>(smem);             // [4 warps][16] max, then sum
        float* so = sm + 4 * 16 * 2;                             // [4 warps][16][DHP]
        const int row = lane >> 2;
        if ((lane & 3) == 0) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                sm[warp * 16 + row + 8 * u] = m[u];
                sm[64 + warp * 16 + row + 8 * u] = l[u];
            }
        }
#pragma unroll
        for (int n = 0; n < NO; ++n)
#pragma unroll
            for (int u = 0; u < 2; ++u)
                *reinterpret_cast<float2*>(&so[(warp * 16 + row + 8 * u) * DHP + n * 8 + (lane & 3) * 2]) =
                    make_float2(o[n][2 * u], o[n][2 * u + 1]);
        __syncthreads();
        if (wk != 0) return;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            float f[WK], mj = -INFINITY;
#pragma unroll
            for (int w = 0; w < WK; ++w) mj = fmaxf(mj, sm[(warp + w) * 16 + row + 8 * u]);
            const float base = mj == -INFINITY ? 0.f : mj;
            l[u] = 0.f;
#pragma unroll
            for (int w = 0; w < WK; ++w) {
                f[w] = ex2(sm[(warp + w) * 16 + row + 8 * u] - base);
                l[u] += f[w] * sm[64 + (warp + w) * 16 + row + 8 * u];
            }
            m[u] = mj;
#pragma unroll
            for (int n = 0; n < NO; ++n) {
                float x = 0.f, y = 0.f;
#pragma unroll
                for (int w = 0; w < WK; ++w) {
                    const float2 z = *reinterpret_cast<const float2*>(&so[((warp + w) * 16 + row + 8 * u) * DHP + n * 8 + (lane & 3) * 2]);
                    x += f[w] * z.x;
                    y += f[w] * z.y;
                }
                o[n][2 * u] = x;
                o[n][2 * u + 1] = y;
            }
        }
    }
    if (p.po) asm volatile("griddepcontrol.wait;" ::: "memory");
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        if (!live[u]) continue;
        const int r = r0 + 8 * u, i = r / G, g = r % G;
        const int64_t t = (int64_t)node * a.M + i;
        if (p.po) {
            // join the prefix's partial results, in order: out = (2^(m-T) o + sum_i 2^(z_i-T) O_i) / (2^(m-T) l + sum_i 2^(z_i-T))
            const int64_t at = t * a.Hq + h * G + g;
            float T2 = m[u];
            for (int x = 0; x < p.splits; ++x) T2 = fmaxf(T2, p.pl[x * p.rows + at]);
            const float f = m[u] == -INFINITY ? 1.f : ex2(m[u] - T2);
            l[u] *= f;
#pragma unroll
            for (int n = 0; n < NO; ++n) { o[n][2 * u] *= f; o[n][2 * u + 1] *= f; }
            for (int x = 0; x < p.splits; ++x) {
                const float z = p.pl[x * p.rows + at];
                if (z == -INFINITY) continue;                    // the split held no key: its output was not written
                const float w = ex2(z - T2);
                const float* po = p.po + (x * p.rows + at) * p.dhp + (lane & 3) * 2;
                l[u] += w;
#pragma unroll
                for (int n = 0; n < NO; ++n) {
                    if (n * 8 >= a.Dh) break;
                    const float2 y = *reinterpret_cast<const float2*>(po + n * 8);
                    o[n][2 * u] = fmaf(w, y.x, o[n][2 * u]);
                    o[n][2 * u + 1] = fmaf(w, y.y, o[n][2 * u + 1]);
                }
            }
            m[u] = T2;
        }
        const bool none = m[u] == -INFINITY && l[u] == 0.f;
        const float inv = none ? 0.f : 1.f / l[u];
        T* out = reinterpret_cast<T*>(p.out) + t * a.out_token + (int64_t)(h * G + g) * a.out_head;
#pragma unroll
        for (int n = 0; n < NO; ++n) {
            const int d = n * 8 + (lane & 3) * 2;
            if (d < a.Dh) *reinterpret_cast<uint32_t*>(out + d) = Mma<T>::pack(o[n][2 * u] * inv, o[n][2 * u + 1] * inv);
        }
        if (p.lse && (lane & 3) == 0) p.lse[t * a.Hq + h * G + g] = none ? -INFINITY : m[u] * kLn2 + logf(l[u]);
    }
}

template <typename T, int DHP, int WM>
int launch_rows(OwnArgs& p, cudaStream_t st) {
    const psd_attention_t& a = p.a;
    const int rows = a.M * (a.Hq / a.Hkv);
    p.row_blocks = (rows + 16 * WM - 1) / (16 * WM);
    const int64_t grid = (int64_t)a.B * a.D * a.Hkv * p.row_blocks;
    if (grid > INT32_MAX) return PSD_ERR_SHAPE;
    constexpr int tile_bytes = 2 * 2 * kKeys * (DHP + 8) * 2, join_bytes = (4 * 16 * 2 + 4 * 16 * DHP) * 4;
    constexpr int smem = tile_bytes > join_bytes ? tile_bytes : join_bytes;
    static std::atomic<unsigned long long> set{0};
    if (!ensure_dynamic_smem(draft_attention_kernel<T, DHP, WM>, smem, set)) return PSD_ERR_CUDA;
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
    const cudaError_t e = cudaLaunchKernelEx(&cfg, draft_attention_kernel<T, DHP, WM>, (const OwnArgs)p);
    count_launch();
    return e == cudaSuccess ? PSD_OK : PSD_ERR_CUDA;
}
template <typename T, int DHP>
int launch_dh(OwnArgs& p, cudaStream_t st) {
    const int rows = p.a.M * (p.a.Hq / p.a.Hkv);
    return rows <= 16 ? launch_rows<T, DHP, 1>(p, st) : rows <= 32 ? launch_rows<T, DHP, 2>(p, st)
                                                                   : launch_rows<T, DHP, 4>(p, st);
}

}  // namespace

size_t draft_attention_workspace(int B, int D, int M, int Hq, int Hkv, int Dh, int P, int S) {
    if (P == 0) return 256;
    const PrefixPlan p = plan_prefix(B, D, M, Hq, Hkv, Dh, P);
    return ((size_t)B * D * M * Hq * p.splits * (p.dhp + 1) * 4 + 255) / 256 * 256;
}

int launch_draft_attention(const void* q, const void* k_prefix, const void* v_prefix, const int32_t* prefix_len,
                           const void* k_own, const void* v_own, const int32_t* own_len, const psd_attention_t& a,
                           void* out, float* lse, void* workspace, int32_t* status_dev, cudaStream_t st) {
    OwnArgs p = {q, k_prefix, v_prefix, k_own, v_own, prefix_len, own_len, out, lse, a, 0, nullptr, nullptr, 0, 0, 0};
    if (a.P > 0) {
        const PrefixPlan plan = plan_prefix(a.B, a.D, a.M, a.Hq, a.Hkv, a.Dh, a.P);
        p.rows = (int64_t)a.B * a.D * a.M * a.Hq;
        float* po = reinterpret_cast<float*>(workspace);
        float* pl = po + p.rows * plan.splits * plan.dhp;
        if (const int e = launch_prefix_attention(q, k_prefix, v_prefix, prefix_len, a, plan, po, pl, status_dev, st)) return e;
        p.po = po;
        p.pl = pl;
        p.splits = plan.splits;
        p.dhp = plan.dhp;
    }
    if (a.dtype == PSD_BF16) return a.Dh <= 64 ? launch_dh<__nv_bfloat16, 64>(p, st) : launch_dh<__nv_bfloat16, 128>(p, st);
    return a.Dh <= 64 ? launch_dh<__half, 64>(p, st) : launch_dh<__half, 128>(p, st);
}

}  // namespace psd
