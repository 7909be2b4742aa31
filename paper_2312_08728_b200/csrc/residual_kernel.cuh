// Softmax loss with its gradient for rows of logits (bmgd_softmax_residual), and the gather of a mini-batch
// (bmgd_gather_batch).
//
//     R_ic = scale (exp(z_ic - lse_i) - [c = y_i]),   loss_i = lse_i - z_{i, y_i},   lse_i = log sum_c exp(z_ic)
//
// lse comes from one pass that keeps the running maximum and the sum relative to it.  A row whose label is outside
// [0, C), or whose logits are all -inf (a mask that leaves nothing), has no gradient: zeros, loss 0.
#pragma once
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "shuffle.cuh"

namespace bmgdk {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

template <typename T> __device__ __forceinline__ float to_f32(T x);
template <> __device__ __forceinline__ float to_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }
template <> __device__ __forceinline__ float to_f32<__half>(__half x) { return __half2float(x); }
template <typename T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_f32<__half>(float x) { return __float2half_rn(x); }

// running maximum and sum of 2^((z - max) log2 e); NaN sticks to the sum
struct MaxSum {
    float m, s;
};
__device__ __forceinline__ float exp_to(float z, float m) { return exp2f((z - m) * kLog2e); }
__device__ __forceinline__ void take(MaxSum& a, float z) {
    const float m = fmaxf(a.m, z);
    if (m == -INFINITY) return;  // nothing but -inf so far (a NaN in z makes the maximum the other value; it enters the sum below)
    a.s = (a.m == -INFINITY ? 0.f : a.s * exp_to(a.m, m)) + exp_to(z, m);
    a.m = m;
}
__device__ __forceinline__ MaxSum join(const MaxSum& a, const MaxSum& b) {
    MaxSum r;
    r.m = fmaxf(a.m, b.m);
    if (r.m == -INFINITY) { r.s = a.s + b.s; return r; }
    r.s = (a.m == -INFINITY ? a.s : a.s * exp_to(a.m, r.m)) + (b.m == -INFINITY ? b.s : b.s * exp_to(b.m, r.m));
    return r;
}

// One block per row, the row read twice (the second time mostly from L2).
template <typename T>
__global__ void __launch_bounds__(256) residual_rows_kernel(const T* __restrict__ z, long long ldz, const int* __restrict__ y,
                                                            T* __restrict__ out, long long ldo, float* __restrict__ loss,
                                                            long long rows, int C, float scale) {
    __shared__ MaxSum part[8];
    for (long long i = blockIdx.x; i < rows; i += gridDim.x) {
        const T* zi = z + i * ldz;
        T* oi = out + i * ldo;
        MaxSum a{-INFINITY, 0.f};
        for (int c = threadIdx.x; c < C; c += blockDim.x) {
            const float x = to_f32(zi[c]);
            if (isnan(x)) a.s = x; else take(a, x);
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            MaxSum b{__shfl_xor_sync(0xFFFFFFFFu, a.m, o), __shfl_xor_sync(0xFFFFFFFFu, a.s, o)};
            a = join(a, b);
        }
        __syncthreads();  // the row before this one has read its sums
        if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = a;
        __syncthreads();
        a = part[0];
        for (int w = 1; w < (int)blockDim.x / 32; ++w) a = join(a, part[w]);
        const int label = y[i];
        const bool counts = label >= 0 && label < C && !(a.m == -INFINITY && !isnan(a.s));
        const float inv = scale / a.s;
        for (int c = threadIdx.x; c < C; c += blockDim.x) {
            float r = 0.f;
            if (counts) {
                r = exp_to(to_f32(zi[c]), a.m) * inv;
                if (c == label) r -= scale;
            }
            oi[c] = from_f32<T>(r);
        }
        if (threadIdx.x == 0 && loss) loss[i] = counts ? (a.m - to_f32(zi[label])) + logf(a.s) : 0.f;
    }
}

// Rows pi(first), pi(first + 1), ... of a buffer, pi the shuffle of one round: the mini-batch as contiguous rows.  A warp
// copies a row at a time, in the widest pieces that all rows are aligned to.
template <typename V>
__global__ void __launch_bounds__(256) gather_batch_kernel(const unsigned char* __restrict__ x, long long row_bytes,
                                                           const int* __restrict__ y, uint32_t N0, unsigned long long seed,
                                                           uint32_t chain, uint32_t round, uint32_t first, uint32_t count,
                                                           unsigned char* __restrict__ out_x, int* __restrict__ out_y) {
    const FeistelDomain dom = make_domain(N0);
    const RoundKeys rk = round_keys(seed, chain, round);
    const int lane = threadIdx.x & 31;
    const long long pieces = row_bytes / (long long)sizeof(V);
    for (uint32_t j = blockIdx.x * 8u + (threadIdx.x >> 5); j < count; j += gridDim.x * 8u) {
        const uint32_t r = perm_index(first + j, dom, rk);
        const V* src = reinterpret_cast<const V*>(x + (long long)r * row_bytes);
        V* dst = reinterpret_cast<V*>(out_x + (long long)j * row_bytes);
        for (long long k = lane; k < pieces; k += 32) dst[k] = src[k];
        if (lane == 0 && y) out_y[j] = y[r];
    }
}

}  // namespace bmgdk
