// The prefix part of the drafts' attention over an 8-bit cache, called by ops_q8_api.cu.
#pragma once
#include "ops_internal.cuh"
#include "prefix_attention.cuh"

namespace psd {

// Widening of codes, two at a time.  `pattern` holds kF16Codes or kBf16Codes in a register (it comes with the kernel's arguments): with two
// constants the compiler makes two instructions of "and, then xor".
constexpr uint32_t kF16Codes = 0x64806480u, kBf16Codes = 0x43004300u;
// The codes in bytes 0 and 2 of x as two fp16 numbers: 1024 + (code + 128) is the pattern 0x6400 + (byte ^ 0x80); minus 1152.
__device__ __forceinline__ uint32_t codes_f16(uint32_t x, uint32_t pattern) {
    uint32_t t, r;
    asm("lop3.b32 %0, %1, %2, %3, 0x6a;" : "=r"(t) : "r"(x), "n"(0x00ff00ff), "r"(pattern));      // (x & mask) ^ pattern
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(t), "r"(pattern));
    return r;
}
// The same in bf16, whose 7 bits of fraction hold 128 + the code's low 7 bits: minus 128, or 256 where the sign bit is set.
__device__ __forceinline__ uint32_t codes_bf16(uint32_t x, uint32_t pattern) {
    uint32_t t, u, r;
    asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(t) : "r"(x), "n"(0x007f007f), "r"(pattern));      // (x & mask) | pattern
    asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(u) : "r"(x), "n"(0x00800080), "r"(pattern));
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(t), "r"(u));
    return r;
}

// Kernels whose time is instructions keep one reference for a row while no value scale at hand is below kNear of the largest.
constexpr float kNear = 1.f / 16.f;
// How far (log2) a row's reference of weight times value scale (relative to the largest scale at hand) may lie below that of its weights: the factor between
// the two, and weights times it, stay inside fp32's range.
constexpr float kFar = 110.f;

struct PrefixQ8 {
    const int8_t *k, *v;             // codes
    const float *k_scale, *v_scale;  // [B, Hkv, ceil(P / block)]
    int block;                       // tokens per scale: 16, 32, 64 or 128
};

// draft_attention.cu: the prefix in codes and the own keys in one launch, and whether that is the form of these sizes
int launch_codes_and_own(const void* q, const PrefixQ8& c, const int32_t* prefix_len, const void* k_own, const void* v_own, const int32_t* own_len,
                         const psd_attention_t& a, void* out, float* lse, cudaStream_t st);
bool one_launch_codes(int B, int D, int M, int Hq, int Hkv, int Dh, int P, int S);

// Which kernel takes the prefix, and how its work is cut.
struct PrefixQ8Plan {
    bool one;           // draft_attention_kernel walks it (final outputs); else:
    bool tiles;         // prefix_tiles_q8_kernel (tcgen05), cut as `tile` says; else prefix_rows_q8_kernel: row_blocks
    bool joined;        // ..with splits that a cluster joins
    bool final;         // the kernel takes the own keys too and writes final outputs; else partial results
    int row_blocks;     // 16-row blocks of a warp: 1 or 2
    PrefixPlan tile;
    int splits;         // partial results per row
    int dhp;            // floats per partial output row: 64 or 128
};
PrefixQ8Plan plan_prefix_q8(int B, int D, int M, int Hq, int Hkv, int Dh, int P, int S);
// bytes of the partial results of a call, and of all calls with smaller B, D and P
size_t prefix_q8_needs(int B, int D, int M, int Hq, int Hkv, int Dh, int P, int S);
size_t prefix_q8_workspace(int B, int D, int M, int Hq, int Hkv, int Dh, int P);

// plan.final: final outputs into out and lse.  Otherwise partial results of every row over its sequence's prefix, as
// launch_prefix_attention leaves them: po [splits][rows][dhp], pl [splits][rows].
int launch_prefix_attention_q8(const void* q, const PrefixQ8& c, const int32_t* prefix_len, const void* k_own, const void* v_own,
                               const int32_t* own_len, const psd_attention_t& a, const PrefixQ8Plan& p, float* po, float* pl, void* out,
                               float* lse, int32_t* status_dev, cudaStream_t st);
// prefix_attention_q8_tc.cu
int q8_clusters(int n);      // clusters of n CTAs of the tcgen05 kernel that the device holds at once
int launch_prefix_tiles_q8(const void* q, const PrefixQ8& c, const int32_t* prefix_len, const void* k_own, const void* v_own,
                           const int32_t* own_len, const psd_attention_t& a, const PrefixPlan& p, bool joined, float* po, float* pl, void* out,
                           float* lse, int32_t* status_dev, cudaStream_t st);

}  // namespace psd
