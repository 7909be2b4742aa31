// Softmax loss with its gradient for rows of logits (bmgd_softmax_residual), and the gather of a mini-batch
// (bmgd_gather_batch).
//
//     R_ic = scale (exp(z_ic - lse_i) - [c = y_i]),   loss_i = lse_i - z_{i, y_i},   lse_i = log sum_c exp(z_ic)
//
// The sum is taken relative to the largest logit, pieces of a row joined by their maxima and sums.  A row whose label is outside
// [0, C), or whose logits are all -inf (a mask that leaves nothing), has no gradient: zeros, loss 0.
#pragma once
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "shuffle.cuh"

namespace bmgdk {

constexpr float kLog2e = 1.4426950408889634f;

template <typename T> __device__ __forceinline__ float to_f32(T x);
template <> __device__ __forceinline__ float to_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }
template <> __device__ __forceinline__ float to_f32<__half>(__half x) { return __half2float(x); }
template <typename T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_f32<__half>(float x) { return __float2half_rn(x); }

// Maximum and sum of exp(z - maximum) of some of a row's logits.  NaN enters the sum, not the maximum; while the maximum is
// -inf the sum is taken relative to 0, so that -inf counts for nothing and NaN still shows.
struct MaxSum {
    float m, s;
};
__device__ __forceinline__ float exp_fast(float x) {  // exp for x <= 0 within 2^-22 + |x| 2^-23 of itself; below 2^-126 zero
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x * kLog2e));
    return r;
}
// (the difference is taken first: next to the type's lowest value a product with log2 e would overflow)
__device__ __forceinline__ float against(float m) { return m == -INFINITY ? 0.f : m; }
__device__ __forceinline__ MaxSum join(const MaxSum& a, const MaxSum& b) {
    const float m = fmaxf(a.m, b.m), to = against(m);
    return MaxSum{m, a.s * exp_fast(against(a.m) - to) + b.s * exp_fast(against(b.m) - to)};
}
__device__ __forceinline__ MaxSum join_lanes(MaxSum a, int lanes) {
    for (int o = lanes / 2; o > 0; o >>= 1) a = join(a, MaxSum{__shfl_xor_sync(0xFFFFFFFFu, a.m, o), __shfl_xor_sync(0xFFFFFFFFu, a.s, o)});
    return a;
}
// what a row's sums say: whether it has a gradient, and the factor of its exponentials
__device__ __forceinline__ bool row_counts(const MaxSum& a, int label, int C) {
    return label >= 0 && label < C && !(a.m == -INFINITY && !isnan(a.s));
}
__device__ __forceinline__ float row_loss(const MaxSum& a, float z_label) { return (against(a.m) - z_label) + logf(a.s); }

// ---- up to 256 classes: LANES lanes of a warp hold a row, up to eight logits each
template <typename T, int LANES>
__global__ void __launch_bounds__(256) residual_short_kernel(const T* __restrict__ z, long long ldz, const int* __restrict__ y,
                                                             T* __restrict__ out, long long ldo, float* __restrict__ loss,
                                                             long long rows, int C, float scale) {
    const int lane = threadIdx.x & (LANES - 1);
    const long long stride = (long long)gridDim.x * (256 / LANES);
    for (long long first = (long long)blockIdx.x * (256 / LANES); first < rows; first += stride) {  // (whole warps: they join by shuffles)
        const long long i = first + threadIdx.x / LANES;
        const bool in = i < rows;
        float x[8];
        MaxSum a{-INFINITY, 0.f};
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int c = lane + k * LANES;
            x[k] = in && c < C ? to_f32(z[i * ldz + c]) : -INFINITY;
            a.m = fmaxf(a.m, x[k]);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) a.s += exp_fast(x[k] - against(a.m));
        a = join_lanes(a, LANES);
        if (!in) continue;
        const int label = y[i];
        const bool counts = row_counts(a, label, C);
        const float m = against(a.m), factor = scale / a.s;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int c = lane + k * LANES;
            if (c >= C) break;
            float r = 0.f;
            if (counts) {
                r = exp_fast(x[k] - m) * factor;
                if (c == label) {
                    r -= scale;
                    if (loss) loss[i] = row_loss(a, x[k]);
                }
            }
            out[i * ldo + c] = from_f32<T>(r);
        }
        if (!counts && lane == 0 && loss) loss[i] = 0.f;
    }
}

// ---- longer rows, held in registers: read once, written once
// R blocks (a cluster) of TH threads share a row (TH = 32: a warp has one, eight to a block).  A thread holds up to NV pieces
// of 16 bytes; the logits before the first 16-byte boundary and behind the last go one each to the first threads.  All
// of a thread's loads are in flight together, which is what keeps memory busy: bound by the one pass over the data.
template <typename T> struct Piece {
    static constexpr int kValues = 16 / (int)sizeof(T);
};
template <typename T>
__device__ __forceinline__ void unpack_piece(const uint4& w, float (&x)[Piece<T>::kValues]) {
    const T* p = reinterpret_cast<const T*>(&w);
#pragma unroll
    for (int i = 0; i < Piece<T>::kValues; ++i) x[i] = to_f32(p[i]);
}
__device__ __forceinline__ uint32_t residual_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}

template <typename T, int TH, int NV>
__global__ void __launch_bounds__(TH == 32 ? 256 : TH) residual_row_kernel(const T* __restrict__ z, long long ldz, const int* __restrict__ y,
                                                                           T* __restrict__ out, long long ldo, float* __restrict__ loss,
                                                                           long long rows, int C, float scale, int R) {
    constexpr int VE = Piece<T>::kValues;
    __shared__ MaxSum part[TH / 32];
    __shared__ MaxSum total;
    const int tid = TH == 32 ? (int)threadIdx.x & 31 : (int)threadIdx.x;
    const int rank = R > 1 ? (int)residual_rank() : 0;
    const long long i = TH == 32 ? blockIdx.x * 8ll + (threadIdx.x >> 5) : (long long)blockIdx.x / R;
    if (i >= rows) return;  // (a whole warp; otherwise the grid has exactly the rows)
    const T* zi = z + i * ldz;
    T* oi = out + i * ldo;
    const int label = y[i];
    const int head = min(C, (int)(((16u - ((uintptr_t)zi & 15u)) & 15u) / sizeof(T)));
    const int pieces = (C - head) / VE, edges = C - pieces * VE;
    const int per = (pieces + R - 1) / R, begin = rank * per, count = min(per, pieces - begin);
    const uint4* src = reinterpret_cast<const uint4*>(zi + head) + begin;
    uint4 w[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k)
        if (tid + k * TH < count) w[k] = __ldcs(src + tid + k * TH);
    // place of this thread's odd logit: before the pieces or behind them
    const bool odd = rank == 0 && tid < edges;
    const int at = tid < head ? tid : tid + pieces * VE;
    const float edge = odd ? to_f32(zi[at]) : -INFINITY;

    MaxSum a{edge, 0.f};
#pragma unroll
    for (int k = 0; k < NV; ++k)
        if (tid + k * TH < count) {
            float x[VE];
            unpack_piece<T>(w[k], x);
#pragma unroll
            for (int e = 0; e < VE; ++e) a.m = fmaxf(a.m, x[e]);
        }
    if (isnan(a.m)) a.m = -INFINITY;  // (the odd logit is NaN and there is no other)
    a.s = exp_fast(edge - against(a.m));
#pragma unroll
    for (int k = 0; k < NV; ++k)
        if (tid + k * TH < count) {
            float x[VE];
            unpack_piece<T>(w[k], x);
#pragma unroll
            for (int e = 0; e < VE; ++e) a.s += exp_fast(x[e] - against(a.m));
        }
    a = join_lanes(a, 32);
    if constexpr (TH > 32) {
        if ((tid & 31) == 0) part[tid >> 5] = a;
        __syncthreads();
        a = part[0];
        for (int k = 1; k < TH / 32; ++k) a = join(a, part[k]);
        if (R > 1) {  // the row's other blocks, in their order
            if (tid == 0) total = a;
            asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
            const uint32_t mine = (uint32_t)__cvta_generic_to_shared(&total);
            MaxSum b[8];
#pragma unroll
            for (int c = 0; c < 8; ++c) {
                if (c >= R) break;
                uint32_t p;
                asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(p) : "r"(mine), "r"(c));
                asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(b[c].m), "=f"(b[c].s) : "r"(p) : "memory");
            }
            a = b[0];
#pragma unroll
            for (int c = 1; c < 8; ++c) {
                if (c >= R) break;
                a = join(a, b[c]);
            }
            asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");  // (waited for at the end)
        }
    }
    const bool counts = row_counts(a, label, C);
    const float m = against(a.m), factor = counts ? scale / a.s : 0.f, minus = counts ? scale : 0.f;
    const int in_pieces = label - head;  // the label's place among the pieces
    const bool same = (((uintptr_t)zi ^ (uintptr_t)oi) & 15u) == 0;
    T* dst = oi + head + (long long)begin * VE;
#pragma unroll
    for (int k = 0; k < NV; ++k)
        if (tid + k * TH < count) {
            float x[VE];
            unpack_piece<T>(w[k], x);
            const int v = tid + k * TH, first = (begin + v) * VE;
#pragma unroll
            for (int e = 0; e < VE; ++e) {
                float r = exp_fast(x[e] - m) * factor;
                if (!counts) r = 0.f;
                x[e] = first + e == in_pieces ? r - minus : r;
            }
            if (same) {
                uint4 q;
                T* t = reinterpret_cast<T*>(&q);
#pragma unroll
                for (int e = 0; e < VE; ++e) t[e] = from_f32<T>(x[e]);
                __stcs(reinterpret_cast<uint4*>(dst) + v, q);
            } else {
#pragma unroll
                for (int e = 0; e < VE; ++e) dst[(long long)v * VE + e] = from_f32<T>(x[e]);
            }
        }
    if (odd) {
        float r = counts ? exp_fast(edge - m) * factor : 0.f;
        if (at == label) r -= minus;
        oi[at] = from_f32<T>(r);
    }
    if (rank == 0 && tid == 0 && loss) loss[i] = counts ? row_loss(a, to_f32(zi[label])) : 0.f;
    if (TH > 32 && R > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// ---- rows too long for that: a block per row, the row read twice (the second time mostly from L2)
template <typename T>
__global__ void __launch_bounds__(1024) residual_long_kernel(const T* __restrict__ z, long long ldz, const int* __restrict__ y,
                                                             T* __restrict__ out, long long ldo, float* __restrict__ loss,
                                                             long long rows, int C, float scale) {
    __shared__ MaxSum part[32];
    for (long long i = blockIdx.x; i < rows; i += gridDim.x) {
        const T* zi = z + i * ldz;
        T* oi = out + i * ldo;
        MaxSum a{-INFINITY, 0.f};
        for (int c0 = threadIdx.x; c0 < C; c0 += 8 * 1024) {
            float x[8], top = -INFINITY;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                x[k] = c0 + k * 1024 < C ? to_f32(zi[c0 + k * 1024]) : -INFINITY;
                top = fmaxf(top, x[k]);
            }
            MaxSum b{top, 0.f};
#pragma unroll
            for (int k = 0; k < 8; ++k) b.s += exp_fast(x[k] - against(top));
            a = join(a, b);
        }
        a = join_lanes(a, 32);
        __syncthreads();  // the row before this one has read its sums
        if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = a;
        __syncthreads();
        a = part[0];
        for (int w = 1; w < 32; ++w) a = join(a, part[w]);
        const int label = y[i];
        const bool counts = row_counts(a, label, C);
        const float m = against(a.m), factor = scale / a.s;
        for (int c = threadIdx.x; c < C; c += 1024) {
            float r = 0.f;
            if (counts) {
                r = exp_fast(to_f32(zi[c]) - m) * factor;
                if (c == label) r -= scale;
            }
            oi[c] = from_f32<T>(r);
        }
        if (threadIdx.x == 0 && loss) loss[i] = counts ? row_loss(a, to_f32(zi[label])) : 0.f;
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
