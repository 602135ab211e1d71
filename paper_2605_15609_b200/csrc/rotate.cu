// Norms of queries and keys per head, their position rotation, and the filing of keys and values in cache slots, in one pass.
//
//   y = x * w / sqrt(mean(x^2) + eps)   (where a weight is given),
//   (z_a, z_b) = gain * (y_a cos t - y_b sin t, y_b cos t + y_a sin t),   t = position * frequency[j],
// for the pairs (a, b) = (j, j + R/2) ("halves") or (2j, 2j + 1) ("interleaved") of the first R numbers of a head.
//
// Bound: memory, each head read and written once.  4 or 8 lanes take a head, 16 numbers a lane, laid out so that both numbers of a
// pair sit in one lane (two pieces of 8: halves R/2 apart, or neighbours; other halves meet in shared memory).  A CTA takes four
// tokens' heads of one kind (q, k or v: the kind, its strides and its weight are uniform), a warp all of a token's, two groups
// of 4 or 8 heads in flight.  The weight is folded into sines and cosines, and arithmetic is on pairs (fp32x2): one group per launch slot, a kind chosen per
// lane and scalar arithmetic took 58 us where this takes 38 (8192 tokens, 32 + 8 + 8 heads of 128, 201 MB: 5.3 TB/s; four groups in flight
// 41 us, 64 registers 41, 256 threads 39).  The angle is the 64-bit product, reduced to a fraction of a turn before it is rounded to
// fp32 (far positions keep their accuracy); a warp's groups of lanes share the sines of their token, each computing some of them.
#include "ops_internal.cuh"
#include "attn_tc.cuh"

namespace psd {
namespace {

constexpr int kThreads = 128;

struct RotateArgs {
    const void *q, *k, *v, *q_norm, *k_norm;
    void *q_out, *k_out, *v_out;
    const int32_t *position, *slot;
    const double* frequency;
    psd_rotate_t a;
    int per;              // heads that a warp takes
    int parts_q, parts_k; // CTAs along the heads of q, and of k (the rest: of v)
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
// sin and cos of 2 pi * (position * frequency / 2 pi): the turn's whole part is dropped in 64 bits
__device__ __forceinline__ float2 turn(int position, double frequency, float gain) {
    double t = (double)position * frequency * 0.15915494309189533577;
    t -= rint(t);
    float s, c;
    sincospif(2.0f * (float)t, &s, &c);
    return make_float2(c * gain, s * gain);
}

// Two words of 16-bit pairs as pairs of fp32: their low halves and their high halves.
template <bool BF16>
__device__ __forceinline__ void widen_apart(uint32_t a, uint32_t b, f32x2& lo, f32x2& hi) {
    if (BF16) {
        lo = pack2(__uint_as_float(a << 16), __uint_as_float(b << 16));
        hi = pack2(__uint_as_float(a & 0xffff0000u), __uint_as_float(b & 0xffff0000u));
    } else {
        const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&a)), y = __half22float2(*reinterpret_cast<const __half2*>(&b));
        lo = pack2(x.x, y.x);
        hi = pack2(x.y, y.y);
    }
}
template <bool BF16>
__device__ __forceinline__ f32x2 widen_word(uint32_t a) {
    if (BF16) return pack2(__uint_as_float(a << 16), __uint_as_float(a & 0xffff0000u));
    const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&a));
    return pack2(x.x, x.y);
}
template <bool BF16>
__device__ __forceinline__ uint32_t narrow2(float lo, float hi) {
    uint32_t w;
    if (BF16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(hi), "f"(lo));
    else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(hi), "f"(lo));
    return w;
}

// A lane's 16 numbers as the first and the second ones of its 8 pairs, two pairs to a register pair.
template <bool BF16, bool INTER>
__device__ __forceinline__ void split_pairs(const uint4& u, const uint4& v, f32x2 (&x)[4], f32x2 (&y)[4]) {
    const uint32_t a[4] = {u.x, u.y, u.z, u.w}, b[4] = {v.x, v.y, v.z, v.w};
    if (INTER) {
        widen_apart<BF16>(a[0], a[1], x[0], y[0]);
        widen_apart<BF16>(a[2], a[3], x[1], y[1]);
        widen_apart<BF16>(b[0], b[1], x[2], y[2]);
        widen_apart<BF16>(b[2], b[3], x[3], y[3]);
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) { x[k] = widen_word<BF16>(a[k]); y[k] = widen_word<BF16>(b[k]); }
    }
}
template <bool BF16, bool INTER>
__device__ __forceinline__ void join_pairs(const f32x2 (&x)[4], const f32x2 (&y)[4], uint4& u, uint4& v) {
    uint32_t a[4], b[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        float x0, x1, y0, y1;
        unpack2(x[k], x0, x1);
        unpack2(y[k], y0, y1);
        uint32_t& p = INTER ? (k < 2 ? a[2 * k] : b[2 * k - 4]) : a[k];
        uint32_t& q = INTER ? (k < 2 ? a[2 * k + 1] : b[2 * k - 3]) : b[k];
        p = INTER ? narrow2<BF16>(x0, y0) : narrow2<BF16>(x0, x1);
        q = INTER ? narrow2<BF16>(x1, y1) : narrow2<BF16>(y0, y1);
    }
    u = make_uint4(a[0], a[1], a[2], a[3]);
    v = make_uint4(b[0], b[1], b[2], b[3]);
}

// How a lane holds a head: both numbers of every pair in its two pieces (halves whose R is a multiple of 16; interleaved), or, for other
// halves, 16 neighbouring numbers, whose partners are read from shared memory.
enum { kHalves = 0, kInterleaved = 1, kAnyHalves = 2 };

// LANES lanes per head (4: Dh <= 64, 8: Dh <= 128); N groups of 32 / LANES heads per warp.
template <bool BF16, int LANES, int N, int MODE>
__global__ void __launch_bounds__(kThreads) rotate_kernel(const RotateArgs p) {
    constexpr int HPW = 32 / LANES;                                 // heads a warp takes at a time
    constexpr bool PAIRED = MODE != kAnyHalves, INTER = MODE == kInterleaved;
    __shared__ float row[PAIRED ? 1 : kThreads / 32][PAIRED ? 1 : HPW][PAIRED ? 1 : LANES * 16 + 1];
    __shared__ float2 turns[PAIRED ? 1 : kThreads / 32][PAIRED ? 1 : 64];
    const psd_rotate_t& a = p.a;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    // blockIdx.x: four tokens, one per warp; blockIdx.y: up to `per` heads of q, of k or of v
    const int t = blockIdx.x * (kThreads / 32) + warp;
    const int kind = (int)blockIdx.y < p.parts_q ? 0 : (int)blockIdx.y < p.parts_q + p.parts_k ? 1 : 2;
    const int h0 = ((int)blockIdx.y - (kind == 0 ? 0 : kind == 1 ? p.parts_q : p.parts_q + p.parts_k)) * p.per, H = min(kind == 0 ? a.Hq : a.Hkv, h0 + p.per);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (t >= a.n_tokens) return;
    const int l = lane % LANES, grp = lane / LANES, R = a.rotary, half = R / 2, pieces = a.Dh / 8;
    // this lane's two pieces of a head
    const bool low = MODE == kHalves && l < R / 16;                 // (the other lanes: the pieces behind the rotated part, two by two)
    const int c0 = low ? l : 2 * l, c1 = low ? l + R / 16 : 2 * l + 1;
    const bool has0 = c0 < pieces, has1 = c1 < pieces;
    const int64_t at = kind > 0 && p.slot ? p.slot[t] : t;
    const bool filed = kind == 0 || !p.slot || (at >= 0 && at < a.n_slots);
    const int64_t in_head = kind == 0 ? a.q_head : kind == 1 ? a.k_head : a.v_head;
    const int64_t out_head = kind == 0 ? a.q_out_head : kind == 1 ? a.k_out_head : a.v_out_head;
    const uint16_t* src = reinterpret_cast<const uint16_t*>(kind == 0 ? p.q : kind == 1 ? p.k : p.v) +
                          t * (kind == 0 ? a.q_token : kind == 1 ? a.k_token : a.v_token) + (h0 + grp) * in_head;
    uint16_t* dst = reinterpret_cast<uint16_t*>(kind == 0 ? p.q_out : kind == 1 ? p.k_out : p.v_out) +
                    at * (kind == 0 ? a.q_out_token : kind == 1 ? a.k_out_token : a.v_out_token) + (h0 + grp) * out_head;
    // N groups of heads are in flight: each is loaded again as soon as it has been stored
    const int64_t in_step = HPW * in_head, out_step = HPW * out_head;
    uint4 x0[N], x1[N];
    auto load = [&](int i, int h) {
        x0[i] = x1[i] = make_uint4(0, 0, 0, 0);
        if (h + grp < H) {
            if (has0) x0[i] = *reinterpret_cast<const uint4*>(src + c0 * 8);
            if (has1) x1[i] = *reinterpret_cast<const uint4*>(src + c1 * 8);
        }
        src += in_step;
    };
    auto store = [&](int h, const uint4& u, const uint4& v) {
        if (filed && h + grp < H) {
            if (has0) *reinterpret_cast<uint4*>(dst + c0 * 8) = u;
            if (has1) *reinterpret_cast<uint4*>(dst + c1 * 8) = v;
        }
        dst += out_step;
    };
#pragma unroll
    for (int i = 0; i < N; ++i) load(i, h0 + i * HPW);
    if (kind == 2) {
#pragma unroll 1
        for (int h = h0; h < H; h += N * HPW) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                store(h + i * HPW, x0[i], x1[i]);
                load(i, h + (N + i) * HPW);
            }
        }
        return;
    }
    // sines and cosines of this lane's 8 pairs (first of them: pair j0 of the head); kAnyHalves: of its 16 numbers
    constexpr int NC = PAIRED ? 8 : 16;
    float cs[NC], sn[NC];
    const int pos = R > 0 ? p.position[t] : 0, j0 = 8 * l;
    const int turned = MODE == kHalves ? (low ? 8 : 0) : min(max(half - j0, 0), 8);    // of its 8 pairs, the first that are rotated
    if (PAIRED) {
        constexpr int EACH = 8 / HPW;                               // pairs that each group of lanes computes
        float2 mine[EACH];
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int j = grp * EACH + e;
            mine[e] = j < turned ? turn(pos, p.frequency[j0 + j], a.gain) : make_float2(1.f, 0.f);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            cs[j] = __shfl_sync(0xffffffffu, mine[j % EACH].x, (j / EACH) * LANES + l);
            sn[j] = __shfl_sync(0xffffffffu, mine[j % EACH].y, (j / EACH) * LANES + l);
        }
    } else {
        for (int j = lane; j < half; j += 32) turns[warp][j] = turn(pos, p.frequency[j], a.gain);
        __syncwarp();
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const int d = 16 * l + j;
            const float2 z = d < R ? turns[warp][d < half ? d : d - half] : make_float2(1.f, 0.f);
            cs[j] = z.x;
            sn[j] = d < half ? -z.y : z.y;
        }
    }
    // PAIRED: with the weights w of the heads at hand, x' = x (w_x cos) - y (w_y sin), y' = y (w_y cos) + x (w_x sin)
    f32x2 xx[4], yx[4], yy[4], xy[4];
    float wt[16];                                                    // kAnyHalves
    const uint16_t* weight = reinterpret_cast<const uint16_t*>(kind == 0 ? p.q_norm : p.k_norm);
    {
        const uint32_t one = BF16 ? 0x3f803f80u : 0x3c003c00u;
        uint4 u = make_uint4(one, one, one, one), v = u;
        if (weight && has0) u = *reinterpret_cast<const uint4*>(weight + c0 * 8);
        if (weight && has1) v = *reinterpret_cast<const uint4*>(weight + c1 * 8);
        if (PAIRED) {
            f32x2 wx[4], wy[4];
            split_pairs<BF16, INTER>(u, v, wx, wy);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const f32x2 c = pack2(cs[2 * k], cs[2 * k + 1]), s = pack2(sn[2 * k], sn[2 * k + 1]), ns = pack2(-sn[2 * k], -sn[2 * k + 1]);
                xx[k] = mul2(wx[k], c);
                yx[k] = mul2(wy[k], ns);
                yy[k] = mul2(wy[k], c);
                xy[k] = mul2(wx[k], s);
            }
        } else {
            float f[8];
            widen8<BF16>(u, f);
#pragma unroll
            for (int j = 0; j < 8; ++j) wt[j] = f[j];
            widen8<BF16>(v, f);
#pragma unroll
            for (int j = 0; j < 8; ++j) wt[8 + j] = f[j];
        }
    }
    const float per = 1.f / (float)a.Dh;
#pragma unroll 1
    for (int h = h0; h < H; h += N * HPW)
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (h + i * HPW >= H) break;
        uint4 y0 = x0[i], y1 = x1[i];
        f32x2 x[4], y[4];
        split_pairs<BF16, INTER>(x0[i], x1[i], x, y);
        float inv = 1.f;
        if (weight) {
            f32x2 sum2 = mul2(x[0], x[0]);
#pragma unroll
            for (int k = 1; k < 4; ++k) sum2 = fma2(x[k], x[k], sum2);
#pragma unroll
            for (int k = 0; k < 4; ++k) sum2 = fma2(y[k], y[k], sum2);
            float s0, s1;
            unpack2(sum2, s0, s1);
            float sum = s0 + s1;
#pragma unroll
            for (int d = 1; d < LANES; d *= 2) sum += __shfl_xor_sync(0xffffffffu, sum, d);
            inv = rsqrtf(fmaf(sum, per, a.eps));
        }
        if (PAIRED) {
            {
                const f32x2 ii = pack2(inv, inv);
                f32x2 ox[4], oy[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    x[k] = mul2(x[k], ii);
                    y[k] = mul2(y[k], ii);
                    ox[k] = mul2(x[k], xx[k]);
                    oy[k] = mul2(y[k], yy[k]);
                    // (numbers that are not rotated stay apart from their neighbours, which may be infinite)
                    if (2 * k < turned) {
                        f32x2 bx = fma2(y[k], yx[k], ox[k]), by = fma2(x[k], xy[k], oy[k]);
                        if (INTER && 2 * k + 1 >= turned) {
                            float e0, e1, r0, r1;
                            unpack2(bx, r0, r1); unpack2(ox[k], e0, e1);
                            bx = pack2(r0, e1);
                            unpack2(by, r0, r1); unpack2(oy[k], e0, e1);
                            by = pack2(r0, e1);
                        }
                        ox[k] = bx;
                        oy[k] = by;
                    }
                }
                join_pairs<BF16, INTER>(ox, oy, y0, y1);
            }
        } else {
            float f[16];
#pragma unroll
            for (int k = 0; k < 4; ++k) { unpack2(x[k], f[2 * k], f[2 * k + 1]); unpack2(y[k], f[8 + 2 * k], f[9 + 2 * k]); }
            float* r = row[warp][grp];
            __syncwarp();
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                f[j] *= inv * wt[j];
                r[16 * l + j] = f[j];
            }
            __syncwarp();
            uint32_t o[8];
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const int d = 16 * l + j;
                if (d < R) f[j] = f[j] * cs[j] + r[d < half ? d + half : d - half] * sn[j];
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] = narrow2<BF16>(f[2 * j], f[2 * j + 1]);
            y0 = make_uint4(o[0], o[1], o[2], o[3]);
            y1 = make_uint4(o[4], o[5], o[6], o[7]);
        }
        store(h + i * HPW, y0, y1);
        load(i, h + (N + i) * HPW);
    }
}

template <bool BF16, int LANES, int N, int MODE>
int launch_n(RotateArgs& p, cudaStream_t st) {
    auto parts = [&](int heads) { return (heads + p.per - 1) / p.per; };
    p.parts_q = parts(p.a.Hq);
    p.parts_k = parts(p.a.Hkv);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((p.a.n_tokens + kThreads / 32 - 1) / (kThreads / 32)), (unsigned)(p.parts_q + p.parts_k * (p.v ? 2 : 1)));
    cfg.blockDim = dim3(kThreads);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = pdl_enabled() ? 1 : 0;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, rotate_kernel<BF16, LANES, N, MODE>, (const RotateArgs)p);
    count_launch();
    return e == cudaSuccess ? PSD_OK : PSD_ERR_CUDA;
}
template <bool BF16, int LANES, int MODE>
int launch_l(RotateArgs& p, cudaStream_t st) {
    // A warp takes all heads of a token's queries (keys, values) once the tokens alone fill the SMs, one group at a time of few tokens; with one group of
    // heads a second one in flight only costs registers (16384 tokens, 8 + 8 + 8 heads of 64: 27.7 against 24.5 us).
    constexpr int HPW = 32 / LANES;
    if (p.a.n_tokens >= 8 * sm_count() && (p.a.Hq > HPW || p.a.Hkv > HPW)) {
        p.per = 16 * HPW;
        return launch_n<BF16, LANES, 2, MODE>(p, st);
    }
    p.per = HPW;
    return launch_n<BF16, LANES, 1, MODE>(p, st);
}
template <bool BF16, int LANES>
int launch_m(RotateArgs& p, cudaStream_t st) {
    if (p.a.interleaved) return launch_l<BF16, LANES, kInterleaved>(p, st);
    return p.a.rotary % 16 == 0 ? launch_l<BF16, LANES, kHalves>(p, st) : launch_l<BF16, LANES, kAnyHalves>(p, st);
}
template <bool BF16>
int launch_t(RotateArgs& p, cudaStream_t st) {
    return p.a.Dh <= 64 ? launch_m<BF16, 4>(p, st) : launch_m<BF16, 8>(p, st);
}

}  // namespace

int launch_rotate(const void* q, const void* k, const void* v, const int32_t* position, const double* frequency, const void* q_norm,
                  const void* k_norm, const int32_t* slot, const psd_rotate_t& a, void* q_out, void* k_out, void* v_out, cudaStream_t st) {
    RotateArgs p = {q, k, v, q_norm, k_norm, q_out, k_out, v_out, position, slot, frequency, a, 0, 0, 0};
    return a.dtype == PSD_BF16 ? launch_t<true>(p, st) : launch_t<false>(p, st);
}

}  // namespace psd
