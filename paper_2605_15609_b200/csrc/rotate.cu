// Norms of queries and keys per head, their position rotation, and the filing of keys and values in cache slots, in one pass.
//
//   y = x * w / sqrt(mean(x^2) + eps)   (where a weight is given),
//   (z_a, z_b) = gain * (y_a cos t - y_b sin t, y_b cos t + y_a sin t),   t = position * frequency[j],
// for the pairs (a, b) = (j, j + R/2) ("halves") or (2j, 2j + 1) ("interleaved") of the first R numbers of a head.
//
// Bound: memory, each head read and written once.  4 or 8 lanes take a head, 16 numbers a lane, laid out so that both numbers of a
// pair sit in one lane (two pieces of 8: halves R/2 apart, or neighbours); a warp takes 4 or 8 heads of one token at a time
// and up to kHeads such groups, whose loads are all issued before the angles are computed.  The angle is the
// 64-bit product, reduced to a fraction of a turn before it is rounded to fp32 (far positions keep their
// accuracy); a warp's groups of lanes share the sines of their token, each computing some of them.
#include "ops_internal.cuh"
#include "tc_common.cuh"

namespace psd {
namespace {

constexpr int kThreads = 128;

struct RotateArgs {
    const void *q, *k, *v, *q_norm, *k_norm;
    void *q_out, *k_out, *v_out;
    const int32_t *position, *slot;
    const double* frequency;
    psd_rotate_t a;
    int heads;            // Hq + Hkv (+ Hkv values)
    int warps;            // warps per token
};

template <bool BF16>
__device__ __forceinline__ void widen8(const uint4& v, float (&x)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (BF16) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        } else {
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
            x[2 * i] = f.x;
            x[2 * i + 1] = f.y;
        }
    }
}
template <bool BF16>
__device__ __forceinline__ uint4 narrow8(const float (&x)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (BF16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(x[2 * i + 1]), "f"(x[2 * i]));
        else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(x[2 * i + 1]), "f"(x[2 * i]));
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// sin and cos of 2 pi * (position * frequency / 2 pi): the turn's whole part is dropped in 64 bits
__device__ __forceinline__ float2 turn(int position, double frequency, float gain) {
    double t = (double)position * frequency * 0.15915494309189533577;
    t -= rint(t);
    float s, c;
    sincospif(2.0f * (float)t, &s, &c);
    return make_float2(c * gain, s * gain);
}

// LANES lanes per head (4: Dh <= 64, 8: Dh <= 128); N groups of 32 / LANES heads per warp.  PAIRED: both numbers of
// every pair are in one lane (interleaved, or R a multiple of 16); else they meet in shared memory.
template <bool BF16, int LANES, int N, bool PAIRED>
__global__ void __launch_bounds__(kThreads) rotate_kernel(const RotateArgs p) {
    constexpr int HPW = 32 / LANES;                                 // heads a warp takes at a time
    __shared__ float row[PAIRED ? 1 : kThreads / 32][PAIRED ? 1 : HPW][PAIRED ? 1 : LANES * 16 + 1];
    const psd_rotate_t& a = p.a;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t w = (int64_t)blockIdx.x * (kThreads / 32) + warp;
    const int t = (int)(w / p.warps), part = (int)(w % p.warps);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (t >= a.n_tokens) return;
    const int l = lane % LANES, grp = lane / LANES, R = a.rotary, pieces = a.Dh / 8;
    // this lane's two pieces of a head
    int c0 = 2 * l, c1 = 2 * l + 1;
    if (PAIRED && !a.interleaved && R > 0) {
        if (l < R / 16) { c0 = l; c1 = l + R / 16; }
        // (the others: the pieces behind the rotated part, two by two)
    }
    const bool has0 = c0 < pieces, has1 = c1 < pieces;
    const int64_t at_k = p.slot ? p.slot[t] : t;
    const bool filed = at_k >= 0 && (!p.slot || at_k < a.n_slots);
    uint4 x0[N], x1[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int h = (part * N + i) * HPW + grp;
        x0[i] = x1[i] = make_uint4(0, 0, 0, 0);
        if (h < p.heads) {
            const uint16_t* s = h < a.Hq ? reinterpret_cast<const uint16_t*>(p.q) + t * a.q_token + h * a.q_head
                              : h < a.Hq + a.Hkv ? reinterpret_cast<const uint16_t*>(p.k) + t * a.k_token + (h - a.Hq) * a.k_head
                                                 : reinterpret_cast<const uint16_t*>(p.v) + t * a.v_token + (h - a.Hq - a.Hkv) * a.v_head;
            if (has0) x0[i] = *reinterpret_cast<const uint4*>(s + c0 * 8);
            if (has1) x1[i] = *reinterpret_cast<const uint4*>(s + c1 * 8);
        }
    }
    // sines and cosines of this lane's 8 pairs (first of them: pair j0 of the head); not PAIRED: of its 16 numbers
    constexpr int NC = PAIRED ? 8 : 16;
    float cs[NC], sn[NC];
    {
        const int pos = R > 0 ? p.position[t] : 0;
        const int half = R / 2;
        if (PAIRED) {
            const int j0 = a.interleaved ? 8 * l : 8 * c0;
            const bool rotated = a.interleaved ? j0 < half : l < R / 16;
            constexpr int EACH = 8 / HPW;                           // pairs that each group of lanes computes
            float2 mine[EACH];
#pragma unroll
            for (int e = 0; e < EACH; ++e) {
                const int j = j0 + grp * EACH + e;
                mine[e] = rotated && j < half ? turn(pos, p.frequency[j], a.gain) : make_float2(1.f, 0.f);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                cs[j] = __shfl_sync(0xffffffffu, mine[j % EACH].x, (j / EACH) * LANES + l);
                sn[j] = __shfl_sync(0xffffffffu, mine[j % EACH].y, (j / EACH) * LANES + l);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const int d = 16 * l + j;
                const float2 z = d < R ? turn(pos, p.frequency[d % half], a.gain) : make_float2(1.f, 0.f);
                cs[j] = z.x;
                sn[j] = d < half ? -z.y : z.y;
            }
        }
    }
    float wq0[8], wq1[8];                                            // the weight of the heads at hand
    int have = -1;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int h = (part * N + i) * HPW + grp;
        const int kind = h < a.Hq ? 0 : h < a.Hq + a.Hkv ? 1 : 2;
        float f0[8], f1[8];
        if (kind < 2) {
            widen8<BF16>(x0[i], f0);
            widen8<BF16>(x1[i], f1);
        }
        const void* weight = kind == 0 ? p.q_norm : kind == 1 ? p.k_norm : nullptr;
        float sum = 0.f;
        if (kind < 2 && weight) {
#pragma unroll
            for (int j = 0; j < 8; ++j) sum = fmaf(f0[j], f0[j], fmaf(f1[j], f1[j], sum));
        }
#pragma unroll
        for (int d = 1; d < LANES; d *= 2) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        if (kind < 2 && weight) {
            if (have != kind) {
                const uint16_t* wt = reinterpret_cast<const uint16_t*>(weight);
                widen8<BF16>(has0 ? *reinterpret_cast<const uint4*>(wt + c0 * 8) : make_uint4(0, 0, 0, 0), wq0);
                widen8<BF16>(has1 ? *reinterpret_cast<const uint4*>(wt + c1 * 8) : make_uint4(0, 0, 0, 0), wq1);
                have = kind;
            }
            const float inv = rsqrtf(sum / (float)a.Dh + a.eps);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                f0[j] *= inv * wq0[j];
                f1[j] *= inv * wq1[j];
            }
        }
        uint4 y0 = x0[i], y1 = x1[i];
        if (PAIRED) {
            if (kind < 2) {
                if (a.interleaved) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        if (16 * l + 2 * j >= R) break;
                        const float u0 = f0[2 * j], u1 = f0[2 * j + 1];
                        f0[2 * j] = u0 * cs[j] - u1 * sn[j];
                        f0[2 * j + 1] = u1 * cs[j] + u0 * sn[j];
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        if (16 * l + 8 + 2 * j >= R) break;
                        const float v0 = f1[2 * j], v1 = f1[2 * j + 1];
                        f1[2 * j] = v0 * cs[4 + j] - v1 * sn[4 + j];
                        f1[2 * j + 1] = v1 * cs[4 + j] + v0 * sn[4 + j];
                    }
                } else if (l < R / 16) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float u = f0[j], v = f1[j];
                        f0[j] = u * cs[j] - v * sn[j];
                        f1[j] = v * cs[j] + u * sn[j];
                    }
                }
            }
        } else {
            float* r = row[warp][grp];
            __syncwarp();
            if (kind < 2) {
#pragma unroll
                for (int j = 0; j < 8; ++j) { r[16 * l + j] = f0[j]; r[16 * l + 8 + j] = f1[j]; }
            }
            __syncwarp();
            if (kind < 2) {
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const int d = 16 * l + j;
                    float& f = j < 8 ? f0[j & 7] : f1[j & 7];
                    if (d < R) f = f * cs[j] + r[d < R / 2 ? d + R / 2 : d - R / 2] * sn[j];
                }
            }
        }
        if (kind < 2) {
            y0 = narrow8<BF16>(f0);
            y1 = narrow8<BF16>(f1);
        }
        if (h < p.heads && (kind == 0 || filed)) {
            uint16_t* d = kind == 0 ? reinterpret_cast<uint16_t*>(p.q_out) + t * a.q_out_token + h * a.q_out_head
                        : kind == 1 ? reinterpret_cast<uint16_t*>(p.k_out) + at_k * a.k_out_token + (h - a.Hq) * a.k_out_head
                                    : reinterpret_cast<uint16_t*>(p.v_out) + at_k * a.v_out_token + (h - a.Hq - a.Hkv) * a.v_out_head;
            if (has0) *reinterpret_cast<uint4*>(d + c0 * 8) = y0;
            if (has1) *reinterpret_cast<uint4*>(d + c1 * 8) = y1;
        }
    }
}

template <bool BF16, int LANES, int N, bool PAIRED>
int launch_n(RotateArgs& p, cudaStream_t st) {
    constexpr int HPW = 32 / LANES;
    p.warps = (p.heads + HPW * N - 1) / (HPW * N);
    const int64_t grid = ((int64_t)p.a.n_tokens * p.warps + kThreads / 32 - 1) / (kThreads / 32);
    if (grid > INT32_MAX) return PSD_ERR_SHAPE;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3(kThreads);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = pdl_enabled() ? 1 : 0;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, rotate_kernel<BF16, LANES, N, PAIRED>, (const RotateArgs)p);
    count_launch();
    return e == cudaSuccess ? PSD_OK : PSD_ERR_CUDA;
}
template <bool BF16, int LANES, bool PAIRED>
int launch_l(RotateArgs& p, cudaStream_t st) {
    // several groups of heads per warp once the warps fill the SMs anyway
    constexpr int HPW = 32 / LANES;
    const int64_t groups = (int64_t)p.a.n_tokens * ((p.heads + HPW - 1) / HPW);
    return groups >= 4 * 64 * (int64_t)sm_count() ? launch_n<BF16, LANES, 4, PAIRED>(p, st) : launch_n<BF16, LANES, 1, PAIRED>(p, st);
}
template <bool BF16>
int launch_t(RotateArgs& p, cudaStream_t st) {
    const bool paired = p.a.interleaved || p.a.rotary % 16 == 0;
    if (p.a.Dh <= 64) return paired ? launch_l<BF16, 4, true>(p, st) : launch_l<BF16, 4, false>(p, st);
    return paired ? launch_l<BF16, 8, true>(p, st) : launch_l<BF16, 8, false>(p, st);
}

}  // namespace

int launch_rotate(const void* q, const void* k, const void* v, const int32_t* position, const double* frequency, const void* q_norm,
                  const void* k_norm, const int32_t* slot, const psd_rotate_t& a, void* q_out, void* k_out, void* v_out, cudaStream_t st) {
    RotateArgs p = {q, k, v, q_norm, k_norm, q_out, k_out, v_out, position, slot, frequency, a, a.Hq + a.Hkv + (v ? a.Hkv : 0), 0};
    return a.dtype == PSD_BF16 ? launch_t<true>(p, st) : launch_t<false>(p, st);
}

}  // namespace psd
