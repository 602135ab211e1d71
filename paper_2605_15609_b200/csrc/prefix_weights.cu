// Attention weight drawn by every prefix key, summed over the rows that read it.
//
// One thread per key: the key stays in registers, the queries of the key head pass by in shared memory (every thread
// reads the same query element), and the thread adds exp2(s * scale * log2 e - lse * log2 e) of its own column of scores.
// No reduction between threads and a fixed order of the sum.
#include "ops_internal.cuh"
#include "tc_common.cuh"

namespace psd {
namespace {

constexpr int kKeys = 128, kRows = 8;

template <typename T> __device__ __forceinline__ float to_f(T x);
template <> __device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
template <> __device__ __forceinline__ float to_f(__half x) { return __half2float(x); }

template <typename T, int DHP>
__global__ void __launch_bounds__(kKeys) weights_kernel(const T* __restrict__ q, const T* __restrict__ k,
                                                        const int32_t* __restrict__ prefix_len, const float* __restrict__ lse,
                                                        const psd_attention_t a, float beta, const float* acc_in, float* acc_out) {
    __shared__ float4 qs[kRows][DHP / 4];
    __shared__ float ls[kRows];
    const int b = blockIdx.y / a.Hkv, h = blockIdx.y % a.Hkv, G = a.Hq / a.Hkv;
    const int L = prefix_len ? min(max(prefix_len[b], 0), a.P) : a.P;
    const int j = blockIdx.x * kKeys + threadIdx.x;
    float kr[DHP];
#pragma unroll
    for (int d = 0; d < DHP; ++d)
        kr[d] = j < L && d < a.Dh ? to_f(k[b * a.kp.outer + j * a.kp.token + h * a.kp.head + d]) : 0.f;
    float sum = 0.f;
    const int n = a.D * a.M * G;
    if (blockIdx.x * kKeys < L) {
        for (int r0 = 0; r0 < n; r0 += kRows) {
            __syncthreads();
            for (int i = threadIdx.x; i < kRows * DHP; i += kKeys) {
                const int r = r0 + i / DHP, d = i % DHP;
                float x = 0.f;
                if (r < n && d < a.Dh)
                    x = to_f(q[((int64_t)b * a.D * a.M + r / G) * a.q_token + (int64_t)(h * G + r % G) * a.q_head + d]);
                reinterpret_cast<float*>(qs[i / DHP])[d] = x;
            }
            if (threadIdx.x < kRows) {
                const int r = r0 + threadIdx.x;
                const float l = r < n ? lse[((int64_t)b * a.D * a.M + r / G) * a.Hq + h * G + r % G] : -INFINITY;
                ls[threadIdx.x] = l == -INFINITY ? INFINITY : l;
            }
            __syncthreads();
            for (int r = 0; r < kRows; ++r) {
                float s = 0.f;
#pragma unroll
                for (int d = 0; d < DHP / 4; ++d) {
                    const float4 x = qs[r][d];
                    s = fmaf(x.x, kr[4 * d], s); s = fmaf(x.y, kr[4 * d + 1], s);
                    s = fmaf(x.z, kr[4 * d + 2], s); s = fmaf(x.w, kr[4 * d + 3], s);
                }
                sum += ex2((s * a.scale - ls[r]) * 1.4426950408889634f);
            }
        }
    }
    if (j < a.P) {
        const int64_t o = (int64_t)blockIdx.y * a.P + j;
        acc_out[o] = j < L ? (acc_in ? beta * acc_in[o] : 0.f) + sum : 0.f;
    }
}

template <typename T>
void run(const void* q, const void* k, const int32_t* prefix_len, const float* lse, const psd_attention_t& a, float beta,
         const float* acc_in, float* acc_out, cudaStream_t st) {
    const dim3 grid((a.P + kKeys - 1) / kKeys, a.B * a.Hkv);
    if (a.Dh <= 64)
        weights_kernel<T, 64><<<grid, kKeys, 0, st>>>((const T*)q, (const T*)k, prefix_len, lse, a, beta, acc_in, acc_out);
    else
        weights_kernel<T, 128><<<grid, kKeys, 0, st>>>((const T*)q, (const T*)k, prefix_len, lse, a, beta, acc_in, acc_out);
}

}  // namespace

size_t prefix_weights_workspace(int, int, int, int, int, int, int) { return 256; }

int launch_prefix_weights(const void* q, const void* k_prefix, const int32_t* prefix_len, const float* lse,
                          const psd_attention_t& a, float beta, const float* acc_in, float* acc_out, void*, int32_t*,
                          cudaStream_t st) {
    if (a.dtype == PSD_BF16) run<__nv_bfloat16>(q, k_prefix, prefix_len, lse, a, beta, acc_in, acc_out, st);
    else run<__half>(q, k_prefix, prefix_len, lse, a, beta, acc_in, acc_out, st);
    count_launch();
    return cudaGetLastError() == cudaSuccess ? PSD_OK : PSD_ERR_CUDA;
}

}  // namespace psd
