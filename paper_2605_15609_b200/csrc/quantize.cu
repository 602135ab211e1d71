// 8-bit integer forms of 16-bit numbers: rows of a matrix (one scale a row) and the caches of a prefix (one scale for each
// block of tokens and key head).
//
//   scale = max(fp32(amax * fp32(1/127)), 2^-126),   r = fp32(1 / scale),   code = rint(fp32(x * r))
//
// in fp32, each operation rounded by itself, so the codes are one number for every implementation of these lines (no
// operation here may be contracted with the next); |x * r| <= 127 (1 + 2^-22), so no code passes 127.  A unit that holds a
// NaN or an infinity gets the scale NaN and codes 0: all of it stands for NaN.
//
// Bound: memory, 2 bytes read and 1 written per element.  A UNIT (one row, or the tokens of a block of one head) is read once
// into registers by 1, 2, 4 or 8 warps, 8 pieces of 8 numbers per lane at most (all loads in flight together: 4 KB a warp; with 16
// pieces fewer warps fit: 16 tokens a block 169 against 110 us, 64 a block 109 against 104, with 4 129 us),
// reduced, and written from the registers; longer rows are read twice.  Absolute values are compared as 16-bit integers, two
// at a time, which also finds NaN and infinity (the largest patterns).
#include "ops_internal.cuh"
#include "tc_common.cuh"

namespace psd {
namespace {

constexpr int kPieces = 8;           // pieces of 8 numbers that a lane holds
template <int WPU> constexpr int kWarps = WPU < 4 ? 4 : WPU;         // of a CTA

struct QuantArgs {
    const void* x[2];                // rows: x[0]; caches: keys, values
    int8_t* codes[2];
    float* scale[2];
    const int32_t *begin, *end;
    int64_t n_units;
    int64_t outer[2], token[2], head[2], code_outer[2], code_token[2], code_head[2];
    int pieces;                      // per unit
    int per_token;                   // pieces of one token (caches), 1 .. 16
    int magic;                       // p / per_token = p * magic >> 16 for p < 2048: ceil(65536 / per_token)
    int P, Hkv, T, nb, nb_call;      // caches: capacity, heads, tokens per block, blocks, blocks per sequence of this call
    int span;
};

template <bool BF16>
__device__ __forceinline__ void widen(uint32_t w, float& lo, float& hi) {
    if (BF16) {
        lo = __uint_as_float(w << 16);
        hi = __uint_as_float(w & 0xffff0000u);
    } else {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
        lo = f.x;
        hi = f.y;
    }
}

// CACHE: units are (sequence, block, head, keys or values); else rows.  WPU warps share a unit.
template <bool CACHE, bool BF16, int WPU>
__global__ void __launch_bounds__(kWarps<WPU> * 32) quantize_kernel(const QuantArgs a) {
    __shared__ uint32_t top[kWarps<WPU>];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t unit = (int64_t)blockIdx.x * (kWarps<WPU> / WPU) + warp / WPU;
    const int lane_u = (warp % WPU) * 32 + lane;                  // lane among the unit's
    constexpr int LANES = WPU * 32;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const uint16_t* x = nullptr;
    int8_t* codes = nullptr;
    float* scale = nullptr;
    int64_t step_in = 0, step_out = 0;                             // between tokens
    int pieces = 0;
    if (unit < a.n_units) {
        if (CACHE) {
            // heads next to each other: a CTA's warps read neighbouring memory
            int64_t u = unit;
            const int h = (int)(u % a.Hkv);
            u /= a.Hkv;
            const int kv = (int)(u & 1);
            u >>= 1;
            const int b = (int)(u / a.nb_call);
            const int begin = a.begin ? min(max(a.begin[b], 0), a.P) : 0;
            int end = a.end ? min(max(a.end[b], 0), a.P) : a.P;
            if (end - begin > a.span) end = begin + a.span;
            const int j = begin / a.T + (int)(u % a.nb_call);
            const int64_t t0 = (int64_t)j * a.T;
            if (begin < end && t0 < end) {
                pieces = (int)min((int64_t)a.T, end - t0) * a.per_token;
                x = reinterpret_cast<const uint16_t*>(a.x[kv]) + b * a.outer[kv] + t0 * a.token[kv] + h * a.head[kv];
                codes = a.codes[kv] + b * a.code_outer[kv] + t0 * a.code_token[kv] + h * a.code_head[kv];
                scale = a.scale[kv] + ((int64_t)b * a.Hkv + h) * a.nb + j;
                step_in = a.token[kv];
                step_out = a.code_token[kv];
            }
        } else {
            pieces = a.pieces;
            x = reinterpret_cast<const uint16_t*>(a.x[0]) + unit * a.outer[0];
            codes = a.codes[0] + unit * a.code_outer[0];
            scale = a.scale[0] + unit;
        }
    }
    uint4 v[kPieces];
    auto load = [&](int p0) {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int p = p0 + i * LANES + lane_u;
            v[i] = make_uint4(0, 0, 0, 0);
            if (p < pieces) {
                const int tok = CACHE ? p * a.magic >> 16 : 0;
                const uint16_t* at = CACHE ? x + tok * step_in + (p - tok * a.per_token) * 8 : x + (int64_t)p * 8;
                v[i] = __ldcs(reinterpret_cast<const uint4*>(at));
            }
        }
    };
    uint32_t m = 0;                  // two 16-bit maxima
    for (int p0 = 0; p0 < pieces || p0 == 0; p0 += kPieces * LANES) {
        load(p0);
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            m = __vmaxu2(m, v[i].x & 0x7fff7fffu);
            m = __vmaxu2(m, v[i].y & 0x7fff7fffu);
            m = __vmaxu2(m, v[i].z & 0x7fff7fffu);
            m = __vmaxu2(m, v[i].w & 0x7fff7fffu);
        }
    }
    m = max(m & 0xffffu, m >> 16);
    m = __reduce_max_sync(0xffffffffu, m);
    if (WPU > 1) {
        if (lane == 0) top[warp] = m;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < WPU; ++i) m = max(m, top[warp / WPU * WPU + i]);
    }
    const bool fine = m < (BF16 ? 0x7f80u : 0x7c00u);
    float amax, unused;
    widen<BF16>(m, amax, unused);
    const float s = fmaxf(__fmul_rn(amax, 1.0f / 127.0f), 1.17549435e-38f);
    const float r = fine ? __frcp_rn(s) : 0.f;
    if (scale && lane_u == 0) *scale = fine ? s : __int_as_float(0x7fc00000);
    const bool again = pieces > kPieces * LANES;
    for (int p0 = 0; p0 < pieces; p0 += kPieces * LANES) {
        if (again) load(p0);
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int p = p0 + i * LANES + lane_u;
            if (p >= pieces) break;
            const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
            uint32_t n[8];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                float lo, hi;
                widen<BF16>(w[k], lo, hi);
                // rint by adding 1.5 * 2^23: the low byte is then the code.  (0 * infinity in a unit that is not fine: masked)
                n[2 * k] = __float_as_uint(__fadd_rn(__fmul_rn(lo, r), 12582912.f));
                n[2 * k + 1] = __float_as_uint(__fadd_rn(__fmul_rn(hi, r), 12582912.f));
            }
            uint2 o;
            o.x = __byte_perm(__byte_perm(n[0], n[1], 0x0040), __byte_perm(n[2], n[3], 0x0040), 0x5410);
            o.y = __byte_perm(__byte_perm(n[4], n[5], 0x0040), __byte_perm(n[6], n[7], 0x0040), 0x5410);
            if (!fine) o = make_uint2(0, 0);
            const int tok = CACHE ? p * a.magic >> 16 : 0;
            int8_t* at = CACHE ? codes + tok * step_out + (p - tok * a.per_token) * 8 : codes + (int64_t)p * 8;
            *reinterpret_cast<uint2*>(at) = o;
        }
    }
}

template <bool CACHE, bool BF16, int WPU>
int launch_w(const QuantArgs& a, cudaStream_t st) {
    constexpr int per_cta = kWarps<WPU> / WPU;
    const int64_t grid = (a.n_units + per_cta - 1) / per_cta;
    if (grid > INT32_MAX) return PSD_ERR_SHAPE;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3(kWarps<WPU> * 32);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = pdl_enabled() ? 1 : 0;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, quantize_kernel<CACHE, BF16, WPU>, a);
    count_launch();
    return e == cudaSuccess ? PSD_OK : PSD_ERR_CUDA;
}

template <bool CACHE>
int launch_q(const QuantArgs& a, bool bf16, cudaStream_t st) {
    // Warps per unit: what holds it in registers; four where the units alone leave most warps of the SMs without work.  Eight against four that
    // read twice: 128 tokens a block of 128, 140 against 201 us for 8 x 16384 tokens; 4096 rows of 16384, 37 against 54, of 20000 (read twice either way) 62 against 69.
    int w = a.pieces <= kPieces * 32 ? 1 : a.pieces <= kPieces * 64 ? 2 : a.pieces <= kPieces * 128 ? 4 : 8;
    if (w < 4 && a.n_units * w < 16 * (int64_t)sm_count() && a.pieces > 64) w = 4;
    if (w == 1) return bf16 ? launch_w<CACHE, true, 1>(a, st) : launch_w<CACHE, false, 1>(a, st);
    if (w == 2) return bf16 ? launch_w<CACHE, true, 2>(a, st) : launch_w<CACHE, false, 2>(a, st);
    if (w == 4) return bf16 ? launch_w<CACHE, true, 4>(a, st) : launch_w<CACHE, false, 4>(a, st);
    return bf16 ? launch_w<CACHE, true, 8>(a, st) : launch_w<CACHE, false, 8>(a, st);
}

}  // namespace

int launch_quantize_rows(const void* x, int dtype, int64_t row_stride, int64_t n_rows, int H, int8_t* codes, int64_t code_stride,
                         float* scale, cudaStream_t st) {
    QuantArgs a = {};
    a.x[0] = x;
    a.codes[0] = codes;
    a.scale[0] = scale;
    a.n_units = n_rows;
    a.outer[0] = row_stride;
    a.code_outer[0] = code_stride;
    a.pieces = H / 8;
    return launch_q<false>(a, dtype == PSD_BF16, st);
}

int launch_prefix_quantize(const void* k, const void* v, const int32_t* begin, const int32_t* end, const psd_quantize_t& q,
                           int8_t* k_codes, int8_t* v_codes, float* k_scale, float* v_scale, cudaStream_t st) {
    QuantArgs a = {};
    a.x[0] = k; a.x[1] = v;
    a.codes[0] = k_codes; a.codes[1] = v_codes;
    a.scale[0] = k_scale; a.scale[1] = v_scale;
    a.begin = begin; a.end = end;
    const psd_kv_strides_t in[2] = {q.k, q.v}, out[2] = {q.k_codes, q.v_codes};
    for (int i = 0; i < 2; ++i) {
        a.outer[i] = in[i].outer; a.token[i] = in[i].token; a.head[i] = in[i].head;
        a.code_outer[i] = out[i].outer; a.code_token[i] = out[i].token; a.code_head[i] = out[i].head;
    }
    a.P = q.P; a.Hkv = q.Hkv; a.T = q.block;
    a.nb = (q.P + q.block - 1) / q.block;
    a.span = q.span > 0 && q.span < q.P ? q.span : q.P;
    // a range of `span` tokens touches at most this many blocks, wherever it begins
    const int most = (a.span + q.block - 1) / q.block + (begin ? 1 : 0);
    a.nb_call = most < a.nb ? most : a.nb;
    a.n_units = (int64_t)q.B * a.nb_call * q.Hkv * 2;
    a.per_token = q.Dh / 8;
    a.magic = (65536 + a.per_token - 1) / a.per_token;
    a.pieces = q.block * a.per_token;
    return launch_q<true>(a, q.dtype == PSD_BF16, st);
}

}  // namespace psd
