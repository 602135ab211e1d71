// Token, confidence and log-sum-exp of rows of logits under penalties, biases and grammar masks.
//
// One pass over the logits (the only large operand): a CTA takes a few rows that share one text (a draft) and one
// bias row, and a chunk of the vocabulary; a warp walks a row's columns with a running maximum m and sum s per lane, four
// 16-byte vectors at a time, and writes one (max, sum, where) record per row and chunk; a second kernel merges them.
//
// The edits touch few tokens.  The CTA counts the text's tokens of its chunk in shared memory once for all its rows and
// lists every token that has a count or a bias ("special"), in order.  Per row, a warp puts down one bit per column of
// its own: open = allowed, inside the vocabulary and not special; the special tokens are then edited 32 at a time, with
// separately rounded operations.  The loop that streams the logits knows nothing but the bits, whatever the edits are (a
// table in shared memory turns the bits of a 16-byte vector into the mask of its words), and does not load a group of
// vectors of which no column is open.  What bounds it is the instructions per column (about 9, two of them at an eighth and a
// half of the issue rate) and how many warps hide each other's loads: four CTAs per SM of 64 registers a thread beat three of
// 80 (8192 x 126464 bf16, before the prefetch: 592 against 667 us), and chunks of 4096 columns beat 2048 (the set-up per CTA) and 8192.
//
// Sums are kept relative to 2^r, r = the rounded product m * log2 e, so that a term is one FMA and one exponential,
// 2^(x log2 e - r), and the rounding of r is the same in every term, the maximum's own included: it cancels in
// confidence = (the maximum's term) / sum.  Maxima beyond 1e37 (a row of the type's lowest values, infinities) would overflow
// that product: their terms are 2^((x - m) log2 e).
//
// The column of a maximum is looked up only where it counts: a record says which lane's group of 32 columns held the
// maximum, and the merge searches the one group of each row that won.
#include "combine.cuh"
#include "attn_tc.cuh"

namespace psd {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMaxChunk = 16384;      // tokens per CTA: 64 KB of counts
constexpr int kMinWarpCols = 256;     // columns a warp takes at least (sets the number of records per row)
constexpr int kRowsPerCta = 64;
constexpr int kBaseCols = 4096;       // columns of a row that a warp takes at most
constexpr int kCtas = 4;              // resident CTAs per SM that registers and shared memory are kept to
constexpr int kGuard = 36;            // closed words behind a warp's open bits: a group of 1024 columns may reach past them
constexpr int U = 4;                  // vectors of a group and lane
constexpr float kHuge = 1e37f;

// A warp's record of its columns of a row.  bits == 0: `at` is the column itself (INT32_MAX: none).  Otherwise the maximum is
// in the group of columns (one lane's four vectors) that starts at column `at`, and those with a bit are open.
struct Part { float m, s; int32_t at; uint32_t bits; };

struct LogitsArgs {
    const void* logits;
    int64_t stride;
    int M, V, D;
    int unit_rows, slices, rows_per_cta;   // rows of one node and one bias row; CTAs they are cut into; rows of each
    int chunk, n_chunks, wpr;              // columns per CTA; CTAs along the vocabulary; warps that share a row
    int rows_per_bias, rows_per_allow, words;
    int merge_early;                       // the merge's blocks are few: let them become resident at once
    psd_logits_edit_t e;
    Part* part;                            // [rows][n_chunks * wpr]
};

template <typename T> struct Vec;
template <> struct Vec<__nv_bfloat16> {
    static constexpr int E = 8;
    static constexpr uint32_t NEG = 0xff80ff80u;           // two times -inf
    static __device__ __forceinline__ float one(const __nv_bfloat16* p) { return __bfloat162float(*p); }
    // two columns, and the larger of two words' columns (exact: a maximum needs no wider type)
    static __device__ __forceinline__ f32x2 pair(const uint32_t* w, int i) { return pack2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u)); }
    static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) {
        uint32_t d;
        asm("max.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
        return d;
    }
    static __device__ __forceinline__ float top(uint32_t w) { return fmaxf(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
};
template <> struct Vec<__half> {
    static constexpr int E = 8;
    static constexpr uint32_t NEG = 0xfc00fc00u;
    static __device__ __forceinline__ float one(const __half* p) { return __half2float(*p); }
    static __device__ __forceinline__ f32x2 pair(const uint32_t* w, int i) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
        return pack2(f.x, f.y);
    }
    static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) {
        uint32_t d;
        asm("max.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
        return d;
    }
    static __device__ __forceinline__ float top(uint32_t w) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
        return fmaxf(f.x, f.y);
    }
};
template <> struct Vec<float> {
    static constexpr int E = 4;
    static constexpr uint32_t NEG = 0xff800000u;
    static __device__ __forceinline__ float one(const float* p) { return *p; }
    static __device__ __forceinline__ f32x2 pair(const uint32_t* w, int i) { return pack2(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1])); }
    static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) { return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b))); }
    static __device__ __forceinline__ float top(uint32_t w) { return __uint_as_float(w); }
};

// Term of x in a sum with maximum m >= x.
__device__ __forceinline__ float term(float x, float m) {
    if (fabsf(m) > kHuge) return ex2((x - m) * kLog2e);
    return ex2(fmaf(x, kLog2e, -__fmul_rn(m, kLog2e)));
}
// A sum kept for maximum m, moved to maximum M >= m (m = -inf: the sum is 0, or NaN from a NaN among the values).
__device__ __forceinline__ float rescaled(float s, float m, float M) {
    if (m == -INFINITY || m == M) return s;
    if (fabsf(m) > kHuge || fabsf(M) > kHuge) return s * ex2((m - M) * kLog2e);
    return s * ex2(__fmul_rn(m, kLog2e) - __fmul_rn(M, kLog2e));      // (not contracted: r is the rounded product)
}

template <typename T>
__global__ void __launch_bounds__(kThreads, kCtas) logits_kernel(const LogitsArgs a) {
    constexpr int E = Vec<T>::E;               // columns of a 16-byte vector
    constexpr int STEP = 32 * E;               // columns of a warp per vector and lane
    constexpr int GC = U * STEP, GW = GC / 32; // columns of a group (1024, or 512 of 4 bytes), and their words of open bits
    constexpr int TABLE = 1 << E;
    extern __shared__ __align__(16) int32_t sh[];
    uint4* table = reinterpret_cast<uint4*>(sh);                    // [TABLE] masks of a vector's words
    int32_t* cnt = sh + TABLE * 4;                                  // [chunk] occurrences in the text
    uint32_t* special = reinterpret_cast<uint32_t*>(cnt + a.chunk);  // [chunk / 32] bits
    const int words = a.chunk / 32;
    uint16_t* first = reinterpret_cast<uint16_t*>(special + words);  // [words + 2] special tokens ahead of a word
    uint16_t* list = first + words + 2;                             // [chunk] special tokens in order
    const int c = blockIdx.x % a.n_chunks;
    const int us = blockIdx.x / a.n_chunks;
    const int slice = us % a.slices;
    const int64_t unit0 = (int64_t)(us / a.slices) * a.unit_rows;      // first row of the unit
    const int64_t row0 = unit0 + (int64_t)slice * a.rows_per_cta;
    const int n_rows = min(a.rows_per_cta, a.unit_rows - slice * a.rows_per_cta);
    const int64_t node = unit0 / a.M;
    const int v0 = c * a.chunk, vw = min(a.chunk, a.V - v0);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const bool counts = a.e.history || a.e.draft_tokens;
    const float* bias = a.e.bias ? a.e.bias + (row0 / a.rows_per_bias) * (int64_t)a.V + v0 : nullptr;
    const int cols = a.chunk / a.wpr;                      // columns of one warp, a multiple of 256
    // [cols / 32] open bits of this warp's columns, one closed word ahead and kGuard behind
    uint32_t* open = reinterpret_cast<uint32_t*>(list + a.chunk) + warp * (cols / 32 + 1 + kGuard) + 1;

    if (threadIdx.x < TABLE) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (E == 4) w[i] = threadIdx.x >> i & 1 ? 0xffffffffu : 0u;
            else w[i] = (threadIdx.x >> (2 * i) & 1 ? 0xffffu : 0u) | (threadIdx.x >> (2 * i + 1) & 1 ? 0xffff0000u : 0u);
        }
        table[threadIdx.x] = make_uint4(w[0], w[1], w[2], w[3]);
    }
    for (int i = lane; i < kGuard + 1; i += 32) open[i ? cols / 32 + i - 1 : -1] = 0u;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (a.merge_early) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    // A row's chunk starts on its way into L2 while the row before is worked on (whole 16-byte granules; 590 against 564 us with
    // it.  The first row's as well, under the set-up: 553, but 128 rows of 4 bytes, one per warp, then lose 2 of 27 us).
    const int c0 = (warp % a.wpr) * cols;
    const int len = max(0, min(cols, vw - c0));            // columns of this warp that exist
    auto row_at = [&](int rr) { return reinterpret_cast<const T*>(a.logits) + (row0 + rr) * a.stride + v0 + c0; };   // column 0
    auto prefetch = [&](int rr) {
        if (lane == 0 && rr < n_rows && len > 0) {
            const T* lg = row_at(rr);
            const int back = (int)((reinterpret_cast<uintptr_t>(lg) & 15) / sizeof(T)), bytes = ((len + back) * (int)sizeof(T) + 15) / 16 * 16;
            asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(lg - back), "r"(bytes) : "memory");
        }
    };
    if (counts) {
        for (int i = threadIdx.x; i < a.chunk; i += kThreads) cnt[i] = 0;
        __syncthreads();
        if (a.e.history) {
            const int64_t b = node / a.D;
            const int n = a.e.history_len ? min(max(a.e.history_len[b], 0), a.e.history_cap) : a.e.history_cap;
            const int32_t* h = a.e.history + b * a.e.history_cap;
#pragma unroll 4
            for (int i = threadIdx.x; i < n; i += kThreads) {
                const int id = h[i];
                const unsigned t = (unsigned)id - (unsigned)v0;
                if (t < (unsigned)vw && id >= 0) atomicAdd(&cnt[t], 1);
            }
        }
        if (a.e.draft_tokens) {
            for (int i = threadIdx.x; i < a.M; i += kThreads) {
                const int id = a.e.draft_tokens[node * a.M + i];
                const unsigned t = (unsigned)id - (unsigned)v0;
                if (a.e.draft_mask[node * a.M + i] == 0 && id >= 0 && t < (unsigned)vw) atomicAdd(&cnt[t], 1);
            }
        }
        __syncthreads();
    }
#pragma unroll 16
    for (int w = warp; w < words; w += kWarps) {
        const int i = w * 32 + lane;
        const bool sp = i < vw && ((counts && cnt[i] > 0) || (bias && bias[i] != 0.f));
        const uint32_t bits = __ballot_sync(0xffffffffu, sp);
        if (lane == 0) special[w] = bits;
    }
    __syncthreads();
    if (warp == 0) {
        int total = 0;
        for (int w0 = 0; w0 < words; w0 += 32) {
            const int n = w0 + lane < words ? __popc(special[w0 + lane]) : 0;
            int run = n;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int y = __shfl_up_sync(0xffffffffu, run, o);
                if (lane >= o) run += y;
            }
            if (w0 + lane < words) first[w0 + lane] = (uint16_t)(total + run - n);
            total += __shfl_sync(0xffffffffu, run, 31);
        }
        if (lane == 0) first[words] = (uint16_t)total;
    }
    __syncthreads();
    for (int w = threadIdx.x; w < words; w += kThreads) {
        uint32_t bits = special[w];
        for (int n = first[w]; bits; ++n) {
            list[n] = (uint16_t)(w * 32 + __ffs(bits) - 1);
            bits &= bits - 1;
        }
    }
    __syncthreads();

    const int n_split = a.n_chunks * a.wpr;
    const int sp0 = first[c0 / 32], sp1 = first[(c0 + cols) / 32];
    for (int rr = warp / a.wpr; rr < n_rows; rr += kWarps / a.wpr) {
        const int64_t row = row0 + rr;
        const T* lg = row_at(rr);
        prefetch(rr + kWarps / a.wpr);
        // Vectors are aligned in memory: with rows that are not, the first one starts `back` columns ahead of column 0.
        const int back = (int)((reinterpret_cast<uintptr_t>(lg) & 15) / sizeof(T));
        const uint32_t* allow = a.e.allow ? a.e.allow + (row / a.rows_per_allow) * (int64_t)a.words + (v0 + c0) / 32 : nullptr;
        if (allow) {
#pragma unroll 4
            for (int w = lane; w < cols / 32; w += 32) {
                const int left = len - w * 32;
                const uint32_t inside = left >= 32 ? 0xffffffffu : left > 0 ? (1u << left) - 1u : 0u;
                open[w] = (left > 0 ? allow[w] : 0u) & inside & ~special[c0 / 32 + w];
            }
        } else {
            for (int w = lane; w < cols / 32; w += 32) {
                const int left = len - w * 32;
                open[w] = (left >= 32 ? 0xffffffffu : left > 0 ? (1u << left) - 1u : 0u) & ~special[c0 / 32 + w];
            }
        }
        // the special tokens, ascending within a lane
        float sm = -INFINITY, ss = 0.f;
        int sa = INT32_MAX;
        for (int e = sp0 + lane; e < sp1; e += 32) {
            const int v = list[e] - c0;
            float x = Vec<T>::one(lg + v);
            const int n = counts ? cnt[c0 + v] : 0;
            if (n > 0) {
                x = x > 0.f ? __fdiv_rn(x, a.e.repetition) : __fmul_rn(x, a.e.repetition);
                x = __fsub_rn(x, __fadd_rn(__fmul_rn(a.e.frequency, (float)n), a.e.presence));
            }
            if (bias) x = __fadd_rn(x, bias[c0 + v]);
            if (allow && !(allow[v >> 5] >> (v & 31) & 1u)) continue;
            const float mn = fmaxf(sm, x);
            if (x > sm) sa = v;
            ss = rescaled(ss, sm, mn) + (x == -INFINITY ? 0.f : term(x, mn));
            sm = mn;
        }
        __syncwarp();
        // first and last column of the row, as columns of this warp: a vector that reaches past them is read piece by piece
        const int lo = -(v0 + c0), hi = a.V - v0 - c0;
        const int shift = (lane * E - back) & 31;
        const uint32_t* my_open = open + ((lane * E - back) >> 5);
        const T* my = lg + lane * E - back;
        float m = -INFINITY, s = 0.f;
        int best = -1;
        uint32_t best_bits = 0u;
        const int groups = len > 0 ? (len + back + GC - 1) / GC : 0;
#pragma unroll 1
        for (int g = 0; g < groups; ++g) {
            uint32_t bits = 0u;                            // of this lane's 32 columns
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const uint32_t* w = my_open + g * GW + u * (STEP / 32);
                const uint32_t b = back ? __funnelshift_r(w[0], w[1], shift) : w[0] >> shift;
                bits |= (b & (TABLE - 1)) << (u * E);
            }
            if (!__any_sync(0xffffffffu, bits)) continue;
            uint4 raw[U];
            if (g * GC - back >= lo && (g + 1) * GC - back <= hi) {
#pragma unroll
                for (int u = 0; u < U; ++u) raw[u] = __ldcs(reinterpret_cast<const uint4*>(my + g * GC + u * STEP));
            } else {
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int i = g * GC + u * STEP + lane * E - back;
                    raw[u] = make_uint4(0, 0, 0, 0);
                    if (i >= lo && i + E <= hi) {
                        raw[u] = __ldcs(reinterpret_cast<const uint4*>(lg + i));
                    } else {
                        T* piece = reinterpret_cast<T*>(&raw[u]);
#pragma unroll
                        for (int j = 0; j < E; ++j)
                            if (i + j >= lo && i + j < hi) piece[j] = lg[i + j];
                    }
                }
            }
            uint32_t w[4 * U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const uint4 k = table[bits >> (u * E) & (TABLE - 1)];
                constexpr uint32_t N = Vec<T>::NEG;
                w[4 * u] = (raw[u].x & k.x) | (N & ~k.x);
                w[4 * u + 1] = (raw[u].y & k.y) | (N & ~k.y);
                w[4 * u + 2] = (raw[u].z & k.z) | (N & ~k.z);
                w[4 * u + 3] = (raw[u].w & k.w) | (N & ~k.w);
            }
            uint32_t q[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                q[i] = w[i];
#pragma unroll
                for (int k = 4; k < 4 * U; k += 4) q[i] = Vec<T>::larger(q[i], w[i + k]);
            }
            const float gm = Vec<T>::top(Vec<T>::larger(Vec<T>::larger(q[0], q[1]), Vec<T>::larger(q[2], q[3])));
            if (gm > m) {
                s = rescaled(s, m, gm);
                best = g;
                best_bits = bits;
                m = gm;
            }
            f32x2 acc[2] = {0ull, 0ull};
            if (fabsf(m) <= kHuge || m == -INFINITY) {
                const float r = m == -INFINITY ? 0.f : __fmul_rn(m, kLog2e);
                const f32x2 l2 = pack2(kLog2e, kLog2e), nr = pack2(-r, -r);
#pragma unroll
                for (int i = 0; i < U * E / 2; ++i) acc[i & 1] = add2(acc[i & 1], ex2_pair(fma2(Vec<T>::pair(w, i), l2, nr)));
            } else {
#pragma unroll
                for (int i = 0; i < U * E / 2; ++i) {
                    float x, y;
                    unpack2(Vec<T>::pair(w, i), x, y);
                    acc[0] = add2(acc[0], pack2(ex2((x - m) * kLog2e), ex2((y - m) * kLog2e)));
                }
            }
            float a0, a1;
            unpack2(add2(acc[0], acc[1]), a0, a1);
            s += a0 + a1;
        }
        // the warp's maximum and sum
        float top = fmaxf(m, sm);
#pragma unroll
        for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        float t = rescaled(s, m, top) + rescaled(ss, sm, top);
#pragma unroll
        for (int o = 16; o; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
        const uint32_t in_group = __ballot_sync(0xffffffffu, m == top && best >= 0), in_special = __ballot_sync(0xffffffffu, sm == top && sa != INT32_MAX);
        Part p = {top, t, INT32_MAX, 0u};
        if (__popc(in_group) == 1 && in_special == 0u) {
            // one lane's group holds it: the merge looks the column up if this record wins
            const int l = __ffs(in_group) - 1;
            p.at = v0 + c0 + __shfl_sync(0xffffffffu, best, l) * GC + l * E - back;
            p.bits = __shfl_sync(0xffffffffu, best_bits, l);
        } else if (in_group | in_special) {
            int at = sm == top ? sa : INT32_MAX;
            if (m == top && best >= 0) {
                for (int k = 0; k < U * E; ++k) {          // a group's columns ascend with k
                    const int i = best * GC + (k / E) * STEP + lane * E + k % E - back;
                    if (best_bits >> k & 1u && Vec<T>::one(lg + i) == top) { at = min(at, i); break; }
                }
            }
            at = __reduce_min_sync(0xffffffffu, at);
            p.at = at == INT32_MAX ? INT32_MAX : v0 + c0 + at;
        }
        if (lane == 0) a.part[row * n_split + c * a.wpr + warp % a.wpr] = p;
        __syncwarp();                                      // the row's bits have been read
    }
    if (!a.merge_early) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

// One warp per row: the row's records in a fixed order (lane by lane, then a fixed tree); of equal maxima the first record's.
template <typename T>
__global__ void __launch_bounds__(kThreads) logits_merge_kernel(const Part* __restrict__ part, const T* __restrict__ logits,
                                                                int64_t stride, int64_t n_rows, int n_split,
                                                                int32_t* __restrict__ out_token, float* __restrict__ out_conf,
                                                                float* __restrict__ out_lse, int32_t* status_dev) {
    constexpr int E = Vec<T>::E, STEP = 32 * E;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int lane = threadIdx.x & 31;
    const int64_t row = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
    if (row >= n_rows) return;
    float m = -INFINITY, s = 0.f;
    int from = INT32_MAX;                          // the first record with this maximum
#pragma unroll 8
    for (int i = lane; i < n_split; i += 32) {
        const float2 p = *reinterpret_cast<const float2*>(&part[row * n_split + i]);
        const float mn = fmaxf(m, p.x);
        if (p.x > m) from = i;
        s = rescaled(s, m, mn) + rescaled(p.y, p.x, mn);
        m = mn;
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        const float m2 = __shfl_xor_sync(0xffffffffu, m, o), s2 = __shfl_xor_sync(0xffffffffu, s, o);
        const int f2 = __shfl_xor_sync(0xffffffffu, from, o);
        const float mn = fmaxf(m, m2);
        from = m2 > m ? f2 : m2 == m ? min(from, f2) : from;
        s = rescaled(s, m, mn) + rescaled(s2, m2, mn);
        m = mn;
    }
    int token = -1;
    if (from != INT32_MAX) {
        const Part p = part[row * n_split + from];
        token = p.at;
        if (p.bits) {
            // lane k looks at the k-th column of the group
            const int v = p.at + (lane / E) * STEP + lane % E;
            const bool hit = (p.bits >> lane & 1u) && Vec<T>::one(logits + row * stride + v) == m;
            const uint32_t hits = __ballot_sync(0xffffffffu, hit);
            token = __shfl_sync(0xffffffffu, v, hits ? __ffs(hits) - 1 : 0);
        }
    }
    if (lane == 0) {
        const bool none = m == -INFINITY;          // nothing left, or only NaN (then s is NaN)
        const float sum = none ? s : s / term(m, m);
        out_token[row] = none || token == INT32_MAX ? -1 : token;
        out_conf[row] = none ? sum : 1.0f / sum;
        if (out_lse) out_lse[row] = none ? (sum == 0.f ? -INFINITY : sum) : m + logf(sum);
        if (status_dev && !(isfinite(sum) && m < INFINITY)) count_nonfinite_row(status_dev);
    }
}

// Rows and columns per CTA, warps per row.  A warp should have a row of kBaseCols columns or several, since the set-up of the
// special tokens is paid per CTA and the reduction per row and chunk; a small batch is spread over the SMs first by rows (128
// x 126465 fp32, 496 CTAs either way: 8 rows x 4096 columns 27 us, 32 rows x 1024 columns 34 us), then by columns.
void choose_shape(int64_t units, int unit_rows, int V, int& rows, int& chunk, int& wpr) {
    const int64_t want = 3 * (int64_t)sm_count();
    rows = unit_rows < kRowsPerCta ? unit_rows : kRowsPerCta;
    const int64_t chunks = (V + kBaseCols - 1) / kBaseCols;
    while (rows > kWarps && units * ((unit_rows + rows - 1) / rows) * chunks < want) rows = (rows + 1) / 2;
    wpr = rows >= 8 ? 1 : rows >= 4 ? 2 : rows >= 2 ? 4 : 8;
    chunk = kBaseCols * wpr < kMaxChunk ? kBaseCols * wpr : kMaxChunk;
    units *= (unit_rows + rows - 1) / rows;
    while (chunk / wpr > kMinWarpCols && units * ((V + chunk - 1) / chunk) < 2 * (int64_t)sm_count()) chunk /= 2;
}

int shared_bytes(int chunk, int wpr, int E) {
    return (16 << E) + chunk * 4 + chunk / 8 + (chunk / 32 + 2) * 2 + chunk * 2 + kWarps * (chunk / wpr / 32 + 1 + kGuard) * 4;
}

template <typename T>
int launch(const LogitsArgs& a, int64_t grid, int64_t n_rows, int32_t* out_token, float* out_conf, float* out_lse, int32_t* status_dev,
           cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = shared_bytes(a.chunk, a.wpr, Vec<T>::E);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = pdl_enabled() ? 1 : 0;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    static std::atomic<unsigned long long> set{0};
    if (!ensure_dynamic_smem(logits_kernel<T>, shared_bytes(kMaxChunk, 1, 8), set)) return PSD_ERR_CUDA;
    cudaError_t e = cudaLaunchKernelEx(&cfg, logits_kernel<T>, a);
    count_launch();
    if (e != cudaSuccess) return PSD_ERR_CUDA;
    cfg.gridDim = dim3((unsigned)((n_rows + kWarps - 1) / kWarps));
    cfg.dynamicSmemBytes = 0;
    e = cudaLaunchKernelEx(&cfg, logits_merge_kernel<T>, (const Part*)a.part, reinterpret_cast<const T*>(a.logits), a.stride, n_rows,
                           a.n_chunks * a.wpr, out_token, out_conf, out_lse, status_dev);
    count_launch();
    return e == cudaSuccess ? PSD_OK : PSD_ERR_CUDA;
}

}  // namespace

// Rows of a unit: of one draft, and of one bias row where there are several.
static int rows_per_unit(int64_t n_rows, int M, int bias_rows) { return bias_rows > 0 ? gcd_int(M, (int)(n_rows / bias_rows)) : M; }

size_t confidence_logits_needs(int64_t n_rows, int M, int V, int bias_rows) {
    const int unit_rows = rows_per_unit(n_rows, M, bias_rows);
    int rows, chunk, wpr;
    choose_shape(n_rows / unit_rows, unit_rows, V, rows, chunk, wpr);
    return (size_t)n_rows * ((V + chunk - 1) / chunk * wpr) * sizeof(Part);
}

// The most records that n_rows rows of V columns or fewer can have, however they are cut into units.  Warps begin with kBaseCols
// columns, or 2048 where eight share a row, and the last chunk's may have none.  They get fewer, kMinWarpCols at least, only
// while the CTAs do not fill the SMs twice, so then there are fewer than 4 CTAs per SM, of rows x warps per row <= kRowsPerCta.
size_t confidence_logits_workspace(int64_t n_rows, int V) {
    const int64_t wide = n_rows * (V / (kMaxChunk / kWarps) + 1 + kWarps);
    const int64_t narrow = n_rows * ((V + kMinWarpCols - 1) / kMinWarpCols + kWarps), few = 4 * (int64_t)sm_count() * kRowsPerCta;
    const int64_t spread = narrow < few ? narrow : few;
    return ((size_t)(wide > spread ? wide : spread) * sizeof(Part) + 255) / 256 * 256;
}

int launch_confidence_logits(const void* logits, int dtype, int64_t row_stride, int B, int D, int M, int V,
                             const psd_logits_edit_t& e, int32_t* out_token, float* out_conf, float* out_lse,
                             void* workspace, int32_t* status_dev, cudaStream_t st) {
    LogitsArgs a = {};
    const int64_t n_rows = (int64_t)B * D * M;
    a.logits = logits;
    a.stride = row_stride;
    a.M = M; a.V = V; a.D = D;
    a.e = e;
    const bool neutral = e.repetition == 1.f && e.presence == 0.f && e.frequency == 0.f;
    if (neutral || e.history_cap == 0) a.e.history = nullptr;
    if (neutral) a.e.draft_tokens = nullptr;
    a.rows_per_bias = (int)(n_rows / (e.bias ? e.bias_rows : 1));
    a.rows_per_allow = (int)(n_rows / (e.allow ? e.allow_rows : 1));
    a.words = (V + 31) / 32;
    a.unit_rows = rows_per_unit(n_rows, M, e.bias ? e.bias_rows : 0);
    choose_shape(n_rows / a.unit_rows, a.unit_rows, V, a.rows_per_cta, a.chunk, a.wpr);
    a.slices = (a.unit_rows + a.rows_per_cta - 1) / a.rows_per_cta;
    const int64_t units = n_rows / a.unit_rows * a.slices;
    a.n_chunks = (V + a.chunk - 1) / a.chunk;
    a.part = reinterpret_cast<Part*>(workspace);
    const int64_t grid = units * a.n_chunks;
    if (grid > INT32_MAX) return PSD_ERR_SHAPE;
    a.merge_early = n_rows <= 8 * kWarps;
    if (dtype == PSD_BF16) return launch<__nv_bfloat16>(a, grid, n_rows, out_token, out_conf, out_lse, status_dev, st);
    if (dtype == PSD_FP16) return launch<__half>(a, grid, n_rows, out_token, out_conf, out_lse, status_dev, st);
    return launch<float>(a, grid, n_rows, out_token, out_conf, out_lse, status_dev, st);
}

}  // namespace psd
