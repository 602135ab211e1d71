// Device and host helpers of the tensor-core kernels that read the prefix's cache: tensor maps of strided caches and of
// query rows, TMA loads in three and four dimensions, operand descriptors, packed fp32 arithmetic, base-2 exponentials.
#pragma once
#include "ops_internal.cuh"
#include "tc_common.cuh"

namespace psd {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kSlabBytes = 128 * 128;     // 128 rows x 64 elements of 2 bytes: one swizzled slab
constexpr int kSlabElems = 64;

// ---- TMA ----------------------------------------------------------------------------------------
__device__ __forceinline__ void tma_load_3d(void* dst, const CUtensorMap* map, uint64_t* bar, int x, int y, int z) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                 ::"r"(smem_u32(dst)), "l"(reinterpret_cast<uint64_t>(map)), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z)
                 : "memory");
}
__device__ __forceinline__ void tma_load_4d(void* dst, const CUtensorMap* map, uint64_t* bar, int x, int y, int z, int w) {
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
                 ::"r"(smem_u32(dst)), "l"(reinterpret_cast<uint64_t>(map)), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z), "r"(w)
                 : "memory");
}

// A bounded wait of a whole warp: every lane gets the same answer, so that warp-wide instructions may follow.  The loop must
// not be unrolled: hundreds of tries in a row at every wait would make most of a kernel's code out of waits.
__device__ __forceinline__ bool mbar_wait_warp(uint64_t* bar, uint32_t parity, const WaitCtx& w) {
    bool r = mbar_try_wait(bar, parity);
    if (!r) {
        const long long t0 = clock64();
#pragma unroll 1
        for (int i = 1;; ++i) {
            r = mbar_try_wait(bar, parity);
            if (r) break;
            if (i & 63) continue;
            if (*w.abort_flag) break;
            if (clock64() - t0 > w.limit) {
                raise_abort(w);
                break;
            }
        }
    }
    return __all_sync(0xffffffffu, r);
}

// One lane of a converged warp.  The issuing warps run their loops with all lanes and let the elected one issue: addresses
// and descriptors then stay in uniform registers.  (With the whole loop under `if (lane == 0)` every operand of every
// tcgen05.mma is moved there first: eight products took 900 cycles to issue instead of 512 to run.)
__device__ __forceinline__ bool elect_one() {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r != 0;
}

// ---- tcgen05 --------------------------------------------------------------------------------------
// Instruction descriptor, kind::f16: fp32 accumulator, M = 128, N = n; A and B of one 16-bit type; b_mn: B is stored
// with its N dimension contiguous (as a tile of V is: keys down, head dimension along).
__device__ __forceinline__ uint32_t umma_idesc16(int n, bool bf16, bool b_mn) {
    const uint32_t t = bf16 ? 1u : 0u;
    return (1u << 4) | (t << 7) | (t << 10) | ((b_mn ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
}
// Operand whose N dimension is contiguous: slabs of 64 elements x rows (K), 128-byte swizzle.  The leading byte offset
// is the distance of the next 64 elements along N (the next slab), the stride byte offset that of the next 8 rows of K.
__device__ __forceinline__ uint64_t umma_smem_desc_mn(uint32_t addr, uint32_t slab_bytes) {
    uint64_t d = 0;
    d |= (uint64_t)((addr & 0x3FFFF) >> 4);
    d |= (uint64_t)(slab_bytes >> 4) << 16;
    d |= (uint64_t)(1024 >> 4) << 32;
    d |= (uint64_t)1 << 46;
    d |= (uint64_t)2 << 61;
    return d;
}
// A operand in tensor memory (packed 16-bit pairs, two per column), B in shared memory.
__device__ __forceinline__ void umma_f16_ts(uint32_t tmem_d, uint32_t tmem_a, uint64_t desc_b, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                 ::"r"(tmem_d), "r"(tmem_a), "l"(desc_b), "r"(idesc), "r"(accumulate) : "memory");
}

// The same with the rows of tensor memory whose bit is set in off[] left as they are.
__device__ __forceinline__ void umma_f16_ts_rows(uint32_t tmem_d, uint32_t tmem_a, uint64_t desc_b, uint32_t idesc, const uint32_t (&off)[4],
                                                 uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %8, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, {%4, %5, %6, %7}, p;\n\t}"
                 ::"r"(tmem_d), "r"(tmem_a), "l"(desc_b), "r"(idesc), "r"(off[0]), "r"(off[1]), "r"(off[2]), "r"(off[3]), "r"(accumulate)
                 : "memory");
}

// 32 lanes x 32 columns without the wait: the caller waits (tmem_wait_ld) before it uses the values.
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
          "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
          "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr));
}
// Every load issued so far has arrived.  The registers pass through, so that no use of them moves above the wait.
__device__ __forceinline__ void tmem_wait_ld(uint32_t (&r)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                   "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]),
                   "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]),
                   "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
                 :: "memory");
}

__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr));
}
__device__ __forceinline__ void tmem_wait_ld16(uint32_t (&r)[16]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                   "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])
                 :: "memory");
}

// 16 packed columns written back by each lane.
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
        ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
          "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};"
        ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
          "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
          "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]),
          "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]), "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// ---- packed fp32 ------------------------------------------------------------------------------------
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pack2(float a, float b) {
    f32x2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void unpack2(f32x2 x, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x)); }
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
    f32x2 d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
    f32x2 d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
    f32x2 d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

__device__ __forceinline__ float lg2(float x) {
    float y;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// x * 2^e where 2^e alone may leave fp32's range
__device__ __forceinline__ float times_ex2(float x, float e) {
    const float h = ex2(0.5f * e);
    return x * h * h;
}
// (2^x stays with ex2: a polynomial on the fp32 pipes takes 10 cycles of a scheduler per 32 results, ex2 takes 8.)
__device__ __forceinline__ f32x2 ex2_pair(f32x2 x) {
    float a, b;
    unpack2(x, a, b);
    return pack2(ex2(a), ex2(b));
}

// ---- host: register shares --------------------------------------------------------------------------------
// A kernel whose warps trade registers (setmaxnreg) waits forever if its shares add up to more than it was launched with:
// the launch is refused unless the compiler gave it at least `need` registers a thread.
template <typename Kernel>
bool launched_with(Kernel kernel, int need, std::atomic<int>& seen) {
    int n = seen.load(std::memory_order_relaxed);
    if (n == 0) {
        cudaFuncAttributes f;
        if (cudaFuncGetAttributes(&f, kernel) != cudaSuccess) return false;
        n = f.numRegs;
        seen.store(n, std::memory_order_relaxed);
    }
    return n >= need;
}

// ---- host: tensor maps --------------------------------------------------------------------------------
CUtensorMapDataType map_type(int dtype) {
    return dtype == PSD_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
}

// A cache [outer, tokens, heads, Dh] with strides s (elements), boxes of `box` tokens x 64 elements of one head.  A
// dimension with stride 0 is shared: its extent becomes 1 and the kernel's coordinate is multiplied by 0.
bool make_cache_map(CUtensorMap* m, const void* base, int dtype, const psd_kv_strides_t& s, int outer, int tokens, int heads, int Dh,
                    int box) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    cuuint64_t dims[4] = {(cuuint64_t)Dh, (cuuint64_t)(s.head ? heads : 1), (cuuint64_t)tokens, (cuuint64_t)(s.outer ? outer : 1)};
    cuuint64_t strides[3] = {(cuuint64_t)(s.head ? s.head : 8) * 2, (cuuint64_t)s.token * 2, (cuuint64_t)(s.outer ? s.outer : 8) * 2};
    cuuint32_t b[4] = {(cuuint32_t)kSlabElems, 1, (cuuint32_t)box, 1};
    cuuint32_t estr[4] = {1, 1, 1, 1};
    return fn(m, map_type(dtype), 4, const_cast<void*>(base), dims, strides, b, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// Query rows [tokens, heads, Dh], boxes of `tq` tokens x the G heads of one key head x 64 elements: tile row = token * G + head.
bool make_query_map(CUtensorMap* m, const void* base, const psd_attention_t& a, int tq) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    cuuint64_t dims[3] = {(cuuint64_t)a.Dh, (cuuint64_t)a.Hq, (cuuint64_t)a.B * a.D * a.M};
    cuuint64_t strides[2] = {(cuuint64_t)a.q_head * 2, (cuuint64_t)a.q_token * 2};
    cuuint32_t b[3] = {(cuuint32_t)kSlabElems, (cuuint32_t)(a.Hq / a.Hkv), (cuuint32_t)tq};
    cuuint32_t estr[3] = {1, 1, 1};
    return fn(m, map_type(a.dtype), 3, const_cast<void*>(base), dims, strides, b, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace
}  // namespace psd
