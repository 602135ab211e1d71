// Attention of query rows over the shared prefix whose cache holds 8-bit codes, with a scale for each block of tokens and key head.
//
//   s_j = scale * k_scale[block of j] * (q . kc_j),   out = sum_j p_j * v_scale[block of j] * vc_j / sum_j p_j,  p_j = 2^(s_j log2 e - m)
//
// Codes are whole numbers up to 127 and so exact in either 16-bit type: they are widened on the way to the tensor instructions, with
// nothing rounded, the keys' scale multiplies a score and the values' scale a weight.  Weights times value scale go to the product in fp16 whatever
// the queries' type (their rounding is 2^-11 then), 2^7 to 2^15 times as large as relative to the row's largest such product, so that none is off by
// more than 2^-32 of that beside its rounding: a row keeps two references, one of its weights for their sum and one of these products for its outputs.
// (With one reference and the largest value scale a row lost what it attends to beside a block of larger values that it does not.)
//
// A CTA takes 16 or 32 rows (query tokens times the heads of one key head) and a range of keys; its four warps go through slices of 32 keys
// by themselves, each with a ring of its own that TMA fills, a running maximum and sums, and are joined at the end.  No barrier
// of the CTA stands in the loop.  Bytes go from shared memory to the operands of m16n8k16 without a transposition: the order of a
// product's inner dimension is free, so a thread takes the 16 or 32 neighbouring bytes of a key that are its share of every step (queries are
// laid out to match), and for the values the bytes of four keys at 16 neighbouring dimensions, which are paired key by key.
//
// Bound for few rows: the cache's bytes, 2 Dh per key; widening takes 3 to 4 instructions for two codes, about 40% of the issue
// slots that the bytes' time offers.  Measured, single tokens of 32 heads of 128 over 8: 64 sequences of 16384 keys 363-381 us, 5.9 TB/s of
// codes and scales; of 3300 to 16384 keys 233-244 us, 5.6-5.7 TB/s; 32 sequences x 5 tokens (20 rows) 197-211 us, 2.7 TB/s (two CTAs per SM, whose
// warps' chains use 38% of the issue slots).
#include <cmath>
#include "attn_tc.cuh"
#include "prefix_attention_q8.cuh"

namespace psd {
namespace {

constexpr int kThreads = 128;
constexpr int kSlice = 32;           // keys a warp takes at a time
constexpr int kStages = 2;           // slices in a warp's ring
constexpr float kRaise = 8.f;        // growth of a row's maximum (log2) that raises its reference
constexpr float kRoom = 7.f;         // how far (log2) weights are kept above the reference: up to 2^15

struct Q8Args {
    const void* q;
    const float *k_scale, *v_scale;
    const int32_t* prefix_len;
    float *po, *pl;
    int32_t* status_dev;
    int64_t rows, q_token, q_head;   // rows: B * D * M * Hq
    int T, G, Hq, Hkv, Dh, P, nb, shift, splits;
    int k_outer, k_head, v_outer, v_head;
    int B, longest_first;            // longest_first: CTAs take the sequences by falling length
    float c;                         // scale * log2 e
    long long wait_limit;
    int stall_test;
    uint32_t f16_codes, bf16_codes;  // kF16Codes, kBf16Codes
};

__device__ __forceinline__ void mma_bf16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_f16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <int DHP, int RB, bool BF16>
// (heads of 64: a fourth CTA per SM, 64 single tokens over 128 keys 10.7 us, without it 13.1)
__global__ void __launch_bounds__(kThreads, RB == 1 ? (DHP == 64 ? 4 : 3) : 2)
prefix_rows_q8_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const Q8Args a) {
    extern __shared__ __align__(1024) unsigned char smem[];
    constexpr int SLICE = kSlice * DHP, STAGE = 2 * SLICE, KS = DHP / 16, NO = DHP / 8;
    __shared__ uint64_t bars[4 * kStages + 1];
    __shared__ int abort_word, sequence;
    volatile int* abort_flag = &abort_word;
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    unsigned char* ring = smem + warp * kStages * STAGE;
    uint64_t *full = bars + warp * kStages, *never = bars + 4 * kStages;
    if (threadIdx.x == 0) {
        for (int i = 0; i <= 4 * kStages; ++i) mbar_init(&bars[i], 1);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        tma_prefetch_desc(&map_k);
        tma_prefetch_desc(&map_v);
    }
    __syncthreads();
    asm volatile("griddepcontrol.wait;" ::: "memory");

    const int cs = blockIdx.x % a.splits, bh = blockIdx.x / a.splits;
    const int h = bh % a.Hkv;
    int b = bh / a.Hkv;
    if (a.longest_first) {
        // the sequences in order of length, so that the last CTAs to start are short ones
        if (threadIdx.x < a.B) {
            const int mine = a.prefix_len[threadIdx.x];
            int rank = 0;
            for (int x = 0; x < a.B; ++x) {
                const int y = a.prefix_len[x];
                rank += y > mine || (y == mine && x < (int)threadIdx.x);
            }
            if (rank == b) sequence = threadIdx.x;
        }
        __syncthreads();
        b = sequence;
    }
    const WaitCtx wc = {abort_flag, a.status_dev, a.wait_limit, 0u};
    const int L = a.prefix_len ? min(max(a.prefix_len[b], 0), a.P) : a.P;
    const int slices = (L + kSlice - 1) / kSlice;
    const int s0 = (int)((long long)slices * cs / a.splits), s1 = (int)((long long)slices * (cs + 1) / a.splits);
    auto load = [&](int slice, int stage) {
        unsigned char* to = ring + stage * STAGE;
        mbar_arrive_expect_tx(&full[stage], STAGE);
        tma_load_4d(to, &map_k, &full[stage], 0, h * a.k_head, slice * kSlice, b * a.k_outer);
        tma_load_4d(to + SLICE, &map_v, &full[stage], 0, h * a.v_head, slice * kSlice, b * a.v_outer);
    };
    const int first = s0 + warp, mine = first < s1 ? (s1 - first + 3) / 4 : 0;     // slices first, first + 4, ..
    int issued = min(kStages, mine);
    if (lane == 0)
        for (int i = 0; i < issued; ++i) load(first + 4 * i, i);

    // scales: lane i holds what scores of the slice's keys 16 i .. 16 i + 15 are multiplied by, lane 2 + i the same for weights, lane 4 + i its logarithm
    const float* scales = (lane & 6 ? a.v_scale : a.k_scale) + ((int64_t)b * a.Hkv + h) * a.nb;
    float vref = 1.17549435e-38f;                       // one for the CTA: its warps are joined
    if (s1 > s0) {
        const float* vs = a.v_scale + ((int64_t)b * a.Hkv + h) * a.nb;
        const int j1 = min((s1 * kSlice - 1) >> a.shift, (L - 1) >> a.shift);
        for (int j = ((s0 * kSlice) >> a.shift) + lane; j <= j1; j += 32) vref = fmaxf(vref, vs[j]);
#pragma unroll
        for (int x = 16; x; x >>= 1) vref = fmaxf(vref, __shfl_xor_sync(0xffffffffu, vref, x));
    }
    const float vinv = 1.f / vref;
    auto scale_of = [&](int slice) {
        const int key = slice * kSlice + (lane & 1) * 16;
        if (key >= L) return 0.f;                       // (what stands there was never written)
        const float x = scales[key >> a.shift] * (lane & 6 ? vinv : a.c);
        if (lane & 4) return lg2(x);
        return lane & 2 || x != 0.f ? x : 1.17549435e-38f;      // masked scores are -inf times this
    };
    float next_scale = mine > 0 ? scale_of(first) : 0.f;

    // queries: in step s of the product over dimensions this thread's share is 4 neighbouring ones from `base(s)`
    const int rows = a.T * a.G;                          // 16 RB at most
    uint32_t qf[RB][KS][4];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int r = rb * 16 + g + 8 * u;
            const bool live = r < rows;
            const int64_t tok = (int64_t)b * a.T + (live ? r / a.G : 0);
            const uint16_t* q = reinterpret_cast<const uint16_t*>(a.q) + tok * a.q_token + (int64_t)(h * a.G + (live ? r % a.G : 0)) * a.q_head;
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const int d = t * (DHP / 4) + s * 4;
                uint2 w = make_uint2(0u, 0u);
                if (live && d < a.Dh) w = *reinterpret_cast<const uint2*>(q + d);
                qf[rb][s][u] = __byte_perm(w.x, w.y, 0x5410);
                qf[rb][s][2 + u] = __byte_perm(w.x, w.y, 0x7632);
            }
        }
    // m: the scores' reference, which l is relative to; w: that of scores plus log2 of their value's scale, which o is relative to
    float o[RB][NO][4], m[RB][2], w[RB][2], l[RB][2];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
#pragma unroll
        for (int n = 0; n < NO; ++n) o[rb][n][0] = o[rb][n][1] = o[rb][n][2] = o[rb][n][3] = 0.f;
        m[rb][0] = m[rb][1] = w[rb][0] = w[rb][1] = -INFINITY;
        l[rb][0] = l[rb][1] = 0.f;
    }
    const uint32_t f16_codes = a.f16_codes, bf16_codes = a.bf16_codes;
    bool ok = true;
    int i = 0;
#pragma unroll 1
    for (; i < mine; ++i) {
        const int stage = i % kStages, slice = first + 4 * i;
        const float sc = next_scale;
        if (i + 1 < mine) next_scale = scale_of(slice + 4);
        if (!(ok = mbar_wait_warp(&full[stage], (i / kStages) & 1, wc))) break;
        if (a.stall_test && !(ok = mbar_wait_warp(never, 0, wc))) { ++i; break; }
        const unsigned char *kt = ring + stage * STAGE, *vt = kt + SLICE;
        float s[RB][4][4];
#pragma unroll
        for (int nt = 0; nt < 4; ++nt) {
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) s[rb][nt][0] = s[rb][nt][1] = s[rb][nt][2] = s[rb][nt][3] = 0.f;
#pragma unroll
            for (int c = 0; c < KS / 4; ++c) {
                const int at = DHP == 128 ? (nt * 8 + g) * 128 + (((2 * t + c) ^ g) << 4) : (nt * 8 + g) * 64 + ((t ^ (g >> 1)) << 4);
                const uint4 w4 = *reinterpret_cast<const uint4*>(kt + at);
                const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const uint32_t b0 = BF16 ? codes_bf16(w[x], bf16_codes) : codes_f16(w[x], f16_codes);
                    const uint32_t b1 = BF16 ? codes_bf16(w[x] >> 8, bf16_codes) : codes_f16(w[x] >> 8, f16_codes);
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb) {
                        if (BF16) mma_bf16(s[rb][nt], qf[rb][c * 4 + x], b0, b1);
                        else mma_f16(s[rb][nt], qf[rb][c * 4 + x], b0, b1);
                    }
                }
            }
        }
        const int left = L - slice * kSlice;
        float vn[2], vlog[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float ks = __shfl_sync(0xffffffffu, sc, i);
            vn[i] = __shfl_sync(0xffffffffu, sc, 2 + i);
            vlog[i] = __shfl_sync(0xffffffffu, sc, 4 + i);
#pragma unroll
            for (int rb = 0; rb < RB; ++rb)
#pragma unroll
                for (int e = 0; e < 8; ++e) s[rb][2 * i + e / 4][e % 4] *= ks;
        }
        if (left < kSlice) {
#pragma unroll
            for (int rb = 0; rb < RB; ++rb)
#pragma unroll
                for (int nt = 0; nt < 4; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (nt * 8 + 2 * t + (e & 1) >= left) s[rb][nt][e] = -INFINITY;
        }
        // a reference of a row is raised, and what has been summed rescaled, only when its maximum grew by 2^kRaise (which one of the row's lanes sees)
        bool higher = false;
        auto maxima = [&](int rb, int u, float& x, float& y) {
            auto of16 = [&](int i) { return fmaxf(max3(s[rb][2 * i][2 * u], s[rb][2 * i][2 * u + 1], s[rb][2 * i + 1][2 * u]), s[rb][2 * i + 1][2 * u + 1]); };
            const float x0 = of16(0), x1 = of16(1);
            x = fmaxf(x0, x1);
            y = fmaxf(x0 + vlog[0], x1 + vlog[1]);
        };
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                float x, y;
                maxima(rb, u, x, y);
                higher |= x > m[rb][u] + kRaise || y > w[rb][u] + kRaise;
            }
        if (__any_sync(0xffffffffu, higher)) {
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
                float f[2];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    float x, y;
                    maxima(rb, u, x, y);
#pragma unroll
                    for (int i = 1; i < 4; i *= 2) {
                        x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, i));
                        y = fmaxf(y, __shfl_xor_sync(0xffffffffu, y, i));
                    }
                    if (x > m[rb][u] + kRaise) {
                        l[rb][u] *= ex2(m[rb][u] - x);
                        m[rb][u] = x;
                    }
                    y = fmaxf(y > w[rb][u] + kRaise ? y : w[rb][u], m[rb][u] - kFar);
                    f[u] = y == w[rb][u] ? 1.f : ex2(w[rb][u] - y);
                    w[rb][u] = y;
                }
#pragma unroll
                for (int n = 0; n < NO; ++n) { o[rb][n][0] *= f[0]; o[rb][n][1] *= f[0]; o[rb][n][2] *= f[1]; o[rb][n][3] *= f[1]; }
            }
        }
        uint32_t pa[RB][2][4];
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            const float base[2] = {m[rb][0] == -INFINITY ? 0.f : m[rb][0] - kRoom, m[rb][1] == -INFINITY ? 0.f : m[rb][1] - kRoom};
            float vg[2][2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const float gain = ex2(fminf(m[rb][u] - w[rb][u], kFar));
                vg[u][0] = vn[0] * gain;
                vg[u][1] = vn[1] * gain;
            }
#pragma unroll
            for (int nt = 0; nt < 4; ++nt) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float p = ex2(s[rb][nt][e] - base[e >> 1]);
                    l[rb][e >> 1] += p;
                    s[rb][nt][e] = p * vg[e >> 1][nt >> 1];
                }
#pragma unroll
                for (int u = 0; u < 2; ++u)
                    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(pa[rb][nt >> 1][(nt & 1) * 2 + u]) : "f"(s[rb][nt][2 * u + 1]), "f"(s[rb][nt][2 * u]));
            }
        }
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            constexpr int NW = DHP / 32;                         // words of a key that this thread takes: 16 or 8 dimensions
            uint32_t w[4][NW];
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int key = kb * 16 + 2 * t + (x & 1) + (x >> 1) * 8;
                if (DHP == 128) {
                    *reinterpret_cast<uint4*>(w[x]) = *reinterpret_cast<const uint4*>(vt + key * 128 + ((g ^ (key & 7)) << 4));
                } else {
                    *reinterpret_cast<uint2*>(w[x]) = *reinterpret_cast<const uint2*>(vt + key * 64 + (((g >> 1) ^ ((key >> 1) & 3)) << 4) + (g & 1) * 8);
                }
            }
#pragma unroll
            for (int x = 0; x < NW; ++x)
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    const int sel = y | y << 4 | (4 + y) << 8 | (4 + y) << 12;
                    const uint32_t b0 = codes_f16(__byte_perm(w[0][x], w[1][x], sel), f16_codes);
                    const uint32_t b1 = codes_f16(__byte_perm(w[2][x], w[3][x], sel), f16_codes);
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb) mma_f16(o[rb][x * 4 + y], pa[rb][kb], b0, b1);
                }
        }
        __syncwarp();
        if (issued < mine) {
            if (lane == 0) load(first + 4 * issued, stage);
            ++issued;
        }
    }
    if (!ok) {
        // giving up: no copy may be in flight when the CTA goes on
        for (int x = i; x < issued; ++x) {
            const long long c0 = clock64();
            while (!mbar_try_wait(&full[x % kStages], (x / kStages) & 1) && clock64() - c0 < WAIT_LIMIT_CYCLES) {}
        }
    }
    // join the warps, 16 rows at a time
    constexpr int OLD = DHP + 4;
    float *so = reinterpret_cast<float*>(smem), *sm = so + 4 * 16 * OLD, *sl = sm + 64;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        __syncthreads();
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            float sum = l[rb][u];
            sum += __shfl_xor_sync(0xffffffffu, sum, 1);
            sum += __shfl_xor_sync(0xffffffffu, sum, 2);
            const int r = warp * 16 + g + 8 * u;
            const float by = m[rb][u] == -INFINITY ? 1.f : ex2(w[rb][u] - m[rb][u]);      // outputs relative to m and vref, as the other warps'
            if (t == 0) { sm[r] = m[rb][u]; sl[r] = sum; }
            // column 2 t + e of tile n is dimension (2 t + e) * NO + n
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int n = 0; n < NO; n += 4)
                    *reinterpret_cast<float4*>(&so[r * OLD + (2 * t + e) * NO + n]) =
                        make_float4(o[rb][n][2 * u + e] * by, o[rb][n + 1][2 * u + e] * by, o[rb][n + 2][2 * u + e] * by, o[rb][n + 3][2 * u + e] * by);
        }
        __syncthreads();
        const int x = threadIdx.x >> 3, part = threadIdx.x & 7, r = rb * 16 + x;
        if (r < rows && ok) {
            float top = -INFINITY, sum = 0.f, f[4];
#pragma unroll
            for (int w = 0; w < 4; ++w) top = fmaxf(top, sm[w * 16 + x]);
            const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                f[w] = ex2(sm[w * 16 + x] - base);
                sum = fmaf(f[w], sl[w * 16 + x], sum);
            }
            const bool none = top == -INFINITY && sum == 0.f;
            const int64_t at = (int64_t)cs * a.rows + ((int64_t)b * a.T + r / a.G) * a.Hq + h * a.G + r % a.G;
            if (part == 0) a.pl[at] = none ? -INFINITY : base - kRoom + log2f(sum);
            const float inv = vref / sum;
            if (!none)
#pragma unroll
                for (int d = 0; d < DHP / 8; d += 4) {
                    const int col = part * 4 + d * 8;
                    if (col >= a.Dh) break;
                    float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const float4 z = *reinterpret_cast<const float4*>(&so[(w * 16 + x) * OLD + col]);
                        y.x = fmaf(f[w], z.x, y.x); y.y = fmaf(f[w], z.y, y.y); y.z = fmaf(f[w], z.z, y.z); y.w = fmaf(f[w], z.w, y.w);
                    }
                    *reinterpret_cast<float4*>(a.po + at * DHP + col) = make_float4(y.x * inv, y.y * inv, y.z * inv, y.w * inv);
                }
        }
    }
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

// A cache of codes [outer, tokens, heads, Dh], boxes of `box` tokens of one head: all its bytes (DHP), swizzled by their width.
bool make_codes_map(CUtensorMap* m, const void* base, const psd_kv_strides_t& s, int outer, int tokens, int heads, int Dh, int dhp, int box) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    cuuint64_t dims[4] = {(cuuint64_t)Dh, (cuuint64_t)(s.head ? heads : 1), (cuuint64_t)tokens, (cuuint64_t)(s.outer ? outer : 1)};
    cuuint64_t strides[3] = {(cuuint64_t)(s.head ? s.head : 16), (cuuint64_t)s.token, (cuuint64_t)(s.outer ? s.outer : 16)};
    cuuint32_t b[4] = {(cuuint32_t)dhp, 1, (cuuint32_t)box, 1};
    cuuint32_t estr[4] = {1, 1, 1, 1};
    return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, const_cast<void*>(base), dims, strides, b, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              dhp == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int DHP, int RB, bool BF16>
int launch_r(const CUtensorMap& mk, const CUtensorMap& mv, const Q8Args& a, int64_t grid, cudaStream_t st) {
    constexpr int ring = 4 * kStages * 2 * kSlice * DHP, join = (4 * 16 * (DHP + 4) + 128) * 4, smem = ring > join ? ring : join;
    static std::atomic<unsigned long long> set{0};
    if (!ensure_dynamic_smem(prefix_rows_q8_kernel<DHP, RB, BF16>, smem, set)) return PSD_ERR_CUDA;
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
    const cudaError_t e = cudaLaunchKernelEx(&cfg, prefix_rows_q8_kernel<DHP, RB, BF16>, mk, mv, a);
    count_launch();
    return e == cudaSuccess ? PSD_OK : PSD_ERR_CUDA;
}

}  // namespace

// How the keys of the few-rows kernel are split.  At least what fills the SMs (a partial wave of CTAs else); beyond that, a CTA costs about as
// much as kCost keys beside its own: split into s, all CTAs' costs take ctas * kCost * s / slots of the time, and the last one to finish P / s
// keys, least together at s = sqrt(P * slots / (ctas * kCost)).  Measured, single tokens, 32 heads of 128 over 8: 64 sequences of up to 16384
// keys: 2 waves of CTAs 241 us, s = 4 or 5 234, 8 waves 245; 16 sequences: s = 3 104, 7 74, 14 85.  No fewer than kLeast keys: one sequence of 16384
// keys in 55 splits 22.8, in 32 19.5 (the join reads less).
constexpr double kCost = 1500;
constexpr int kLeast = 512;

PrefixQ8Plan plan_prefix_q8(int B, int D, int M, int Hq, int Hkv, int Dh, int P, int S) {
    const int64_t rows = (int64_t)D * M * (Hq / Hkv);
    PrefixQ8Plan p = {};
    p.dhp = Dh <= 64 ? 64 : 128;
    if (one_launch_codes(B, D, M, Hq, Hkv, Dh, P, S)) {
        p.one = p.final = true;
        p.splits = 1;
        return p;
    }
    p.tiles = rows > 32;
    if (p.tiles) {
        p.tile = plan_prefix(B, D, M, Hq, Hkv, Dh, P, S);
        if (!p.tile.fused) {
            // Up to eight CTAs along the keys are a cluster that joins by itself: as many as let all clusters run at once, if that leaves no stream more
            // than three rounds (about 2 us each) longer than more splits and a second kernel (about 10 us) would, and the drafts (a tile of own keys
            // each) are few.  Measured, 32 heads of 128 over 8, against a second kernel: one draft of 32 tokens, prefix 2000: 20.0 against 23.9 us, four:
            // 22.3 against 24.7, prefix 1000: 21.5 against 23.7; 16 drafts of one token, prefix 4000: 21.5 against 18.6.
            const int per = p.tile.n_qt > 1 ? 1 : 2, met = drafts_per_tile(M, p.tile.tq), tiles = (P + 127) / 128;
            int n = p.tile.splits / per < 8 ? p.tile.splits / per : 8;
            while (n > 1 && (int64_t)B * Hkv * p.tile.units > q8_clusters(n)) --n;
            const int64_t own = (int64_t)(D < met ? D : met) * ((S + 127) / 128);
            if (n > 1 && (tiles + n * per - 1) / (n * per) <= (tiles + p.tile.splits - 1) / p.tile.splits + 3 && own <= 4) {
                p.joined = true;
                p.tile.splits = n * per;
            }
        }
        p.final = p.tile.fused || p.joined;
        p.splits = p.tile.splits;
        return p;
    }
    p.row_blocks = rows > 16 ? 2 : 1;
    const int64_t ctas = (int64_t)B * Hkv, slots = (int64_t)sm_count() * (p.row_blocks == 1 ? 3 : 2);
    int64_t s = (int64_t)(std::sqrt((double)P * slots / (ctas * kCost)) + 0.5);
    if (s < slots / ctas) s = slots / ctas;
    if (s > (P + kLeast - 1) / kLeast) s = (P + kLeast - 1) / kLeast;
    if (s > kMaxPrefixSplits) s = kMaxPrefixSplits;
    p.splits = s < 1 ? 1 : (int)s;
    return p;
}

static size_t partial_bytes_q8(int64_t rows, int dhp) { return ((size_t)rows * (dhp + 1) * 4 + 255) / 256 * 256; }

size_t prefix_q8_needs(int B, int D, int M, int Hq, int Hkv, int Dh, int P, int S) {
    const PrefixQ8Plan p = plan_prefix_q8(B, D, M, Hq, Hkv, Dh, P, S);
    if (p.final) return 256;
    return partial_bytes_q8((int64_t)B * D * M * Hq * p.splits, p.dhp);
}

// An upper bound of what this call and all with smaller B, D and P need.  Rows are split while their CTAs fill the SMs once (256 rows each at
// most), in the few-rows kernel as plan_prefix_q8 says (32 rows each at most), and no further than the prefix allows; a single query tile of
// the tcgen05 kernel is always split in two.
size_t prefix_q8_workspace(int B, int D, int M, int Hq, int Hkv, int Dh, int P) {
    const int64_t rows = (int64_t)B * D * M * Hq, T = (int64_t)D * M, G = Hq / Hkv, tq = 128 / G, sms = sm_count();
    const int64_t pairs = 2 * (int64_t)B * Hq * (T < tq ? T : tq);
    const double few = 2.0 * B * Hkv;                               // the few-rows kernel's CTAs ahead of the splits, twice over
    int64_t n = (rows > pairs ? rows : pairs) + 256 * sms + (int64_t)(32.0 * (std::sqrt(3.0 * sms * few * P / kCost) + few));
    int64_t most = ((int64_t)P + 255) / 256;
    if (most > kMaxPrefixSplits) most = kMaxPrefixSplits;
    if (most < 2) most = 2;
    if (n > rows * most) n = rows * most;
    return partial_bytes_q8(n, Dh <= 64 ? 64 : 128);
}

int launch_prefix_attention_q8(const void* q, const PrefixQ8& c, const int32_t* prefix_len, const void* k_own, const void* v_own,
                               const int32_t* own_len, const psd_attention_t& a, const PrefixQ8Plan& p, float* po, float* pl, void* out,
                               float* lse, int32_t* status_dev, cudaStream_t st) {
    if (p.one) return launch_codes_and_own(q, c, prefix_len, k_own, v_own, own_len, a, out, lse, st);
    if (p.tiles) return launch_prefix_tiles_q8(q, c, prefix_len, k_own, v_own, own_len, a, p.tile, p.joined, po, pl, out, lse, status_dev, st);
    CUtensorMap mk, mv;
    if (!make_codes_map(&mk, c.k, a.kp, a.B, a.P, a.Hkv, a.Dh, p.dhp, kSlice) || !make_codes_map(&mv, c.v, a.vp, a.B, a.P, a.Hkv, a.Dh, p.dhp, kSlice))
        return PSD_ERR_CUDA;
    const int64_t grid = (int64_t)a.B * a.Hkv * p.splits;
    if (grid > INT32_MAX) return PSD_ERR_SHAPE;
    Q8Args x = {};
    x.q = q;
    x.k_scale = c.k_scale; x.v_scale = c.v_scale;
    x.prefix_len = prefix_len;
    x.po = po; x.pl = pl;
    x.status_dev = status_dev;
    x.rows = (int64_t)a.B * a.D * a.M * a.Hq;
    x.q_token = a.q_token; x.q_head = a.q_head;
    x.T = a.D * a.M; x.G = a.Hq / a.Hkv; x.Hq = a.Hq; x.Hkv = a.Hkv; x.Dh = a.Dh; x.P = a.P;
    x.nb = (a.P + c.block - 1) / c.block;
    x.shift = c.block == 16 ? 4 : c.block == 32 ? 5 : c.block == 64 ? 6 : 7;
    x.splits = p.splits;
    x.k_outer = a.kp.outer ? 1 : 0; x.k_head = a.kp.head ? 1 : 0;
    x.v_outer = a.vp.outer ? 1 : 0; x.v_head = a.vp.head ? 1 : 0;
    x.B = a.B;
    x.longest_first = prefix_len && a.B > 1 && a.B <= kThreads && grid > 3 * (int64_t)sm_count() ? 1 : 0;
    x.c = a.scale * kLog2e;
    x.wait_limit = wait_limit_cycles();
    x.stall_test = selftest_stall();
    x.f16_codes = kF16Codes;
    x.bf16_codes = kBf16Codes;
    const bool bf16 = a.dtype == PSD_BF16;
    auto go = [&](auto dhp, auto rb) {
        return bf16 ? launch_r<decltype(dhp)::value, decltype(rb)::value, true>(mk, mv, x, grid, st)
                    : launch_r<decltype(dhp)::value, decltype(rb)::value, false>(mk, mv, x, grid, st);
    };
    using std::integral_constant;
    if (p.dhp == 64) return p.row_blocks == 1 ? go(integral_constant<int, 64>(), integral_constant<int, 1>()) : go(integral_constant<int, 64>(), integral_constant<int, 2>());
    return p.row_blocks == 1 ? go(integral_constant<int, 128>(), integral_constant<int, 1>()) : go(integral_constant<int, 128>(), integral_constant<int, 2>());
}

}  // namespace psd
