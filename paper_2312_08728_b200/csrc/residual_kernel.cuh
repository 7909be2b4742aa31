// Softmax loss with its gradient for rows of logits (bmgd_softmax_residual), and the gather of a mini-batch
// (bmgd_gather_batch).
//
//     R_ic = scale (exp(z_ic - lse_i) - [c = y_i]),   loss_i = lse_i - z_{i, y_i},   lse_i = log sum_c exp(z_ic)
//
// The sum is taken relative to the largest logit, pieces of a row joined by their maxima and sums.  A row whose label is outside
// [0, C), or whose logits are all -inf (a mask that leaves nothing), has no gradient: zeros, loss 0.
#pragma once
#include <cstdint>
#include <cuda_runtime.h>

#include "shuffle.cuh"
#include "values.cuh"

namespace bmgdk {

// Maximum and sum of exp(z - maximum) of some of a row's logits.  NaN enters the sum, not the maximum; while the maximum is
// -inf the sum is taken relative to 0, so that -inf counts for nothing and NaN still shows.
struct MaxSum {
    float m, s;
};
// (the difference is taken first: next to the type's lowest value a product with log2 e would overflow)
__device__ __forceinline__ float against(float m) { return m == -INFINITY ? 0.f : m; }
// factor that takes a sum to a larger maximum; a sum without one is 0 or NaN and stays so (0 times the exponential of what
// lies between 0 and a row of very negative logits would be NaN)
__device__ __forceinline__ float carry(float from, float to) { return from == -INFINITY ? 1.f : exp_fast(from - against(to)); }
__device__ __forceinline__ MaxSum join(const MaxSum& a, const MaxSum& b) {
    const float m = fmaxf(a.m, b.m);
    return MaxSum{m, a.s * carry(a.m, m) + b.s * carry(b.m, m)};
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

// ---- up to 64 classes: LANES lanes of a warp hold a row, up to eight logits each
template <typename T, int LANES>
__global__ void __launch_bounds__(256, 6) residual_short_kernel(const T* __restrict__ z, long long ldz, const int* __restrict__ y,
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
__device__ __forceinline__ uint32_t residual_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}

// (in pairs, because the exponentials' arithmetic competes with memory in the 16-bit types)
// the exponentials of a piece against a maximum, two at a time: exp_fast(x - m)
template <typename T, typename F>
__device__ __forceinline__ void piece_powers(const uint4& w, const Pair& minus_m, const Pair& log2e, F&& take) {
    constexpr int VE = Piece<T>::kValues;
    float x[VE];
    unpack_piece<T>(w, x);
#pragma unroll
    for (int e = 0; e < VE; e += 2) {
        float2 p = ((Pair(x[e], x[e + 1]) + minus_m) * log2e).both();
        asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(p.x));
        asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(p.y));
        take(e, Pair(p.x, p.y));
    }
}
// largest of a piece's values and `top`, NaN left aside
__device__ __forceinline__ float piece_max(float top, const uint4& w, float) {
    float x[4];
    unpack_piece<float>(w, x);
    return fmaxf(fmaxf(top, fmaxf(x[0], x[1])), fmaxf(x[2], x[3]));
}
__device__ __forceinline__ float piece_max(float top, const uint4& w, __nv_bfloat16) {
    const __nv_bfloat162* p = reinterpret_cast<const __nv_bfloat162*>(&w);
    const float2 m = __bfloat1622float2(__hmax2(__hmax2(p[0], p[1]), __hmax2(p[2], p[3])));
    return fmaxf(top, fmaxf(m.x, m.y));
}
__device__ __forceinline__ float piece_max(float top, const uint4& w, __half) {
    const __half2* p = reinterpret_cast<const __half2*>(&w);
    const float2 m = __half22float2(__hmax2(__hmax2(p[0], p[1]), __hmax2(p[2], p[3])));
    return fmaxf(top, fmaxf(m.x, m.y));
}
// A value joined over the threads of a block and the R blocks of its cluster, in a fixed order; `cells` is this use's own.
template <int TH, bool MAX>
__device__ __forceinline__ float row_join(float v, float* cells, int tid, int R) {
    auto op = [](float a, float b) { return MAX ? fmaxf(a, b) : a + b; };
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = op(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
    if constexpr (TH > 32) {
        if ((tid & 31) == 0) cells[tid >> 5] = v;
        __syncthreads();
        v = cells[0];
#pragma unroll
        for (int k = 1; k < TH / 32; ++k) v = op(v, cells[k]);
        if (R > 1) {
            float* mine = cells + TH / 32;
            if (tid == 0) *mine = v;
            asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
            const uint32_t at = (uint32_t)__cvta_generic_to_shared(mine);
            float b[8];
#pragma unroll
            for (int c = 0; c < 8; ++c) {
                if (c >= R) break;
                uint32_t p;
                asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(p) : "r"(at), "r"(c));
                asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(b[c]) : "r"(p) : "memory");
            }
            v = b[0];
#pragma unroll
            for (int c = 1; c < 8; ++c) {
                if (c >= R) break;
                v = op(v, b[c]);
            }
        }
    }
    return v;
}

// Two of these blocks' worth of registers fit an SM at least; the pieces are unpacked anew in each of the three passes over
// them (the compiler would rather keep twice as many registers of unpacked values, and one block to an SM: 706 us
// instead of 443 at 8191 x 50257 in bf16).
template <typename T, int TH, int NV>
__global__ void __launch_bounds__(TH == 32 ? 256 : TH, TH == 32 ? (NV <= 2 ? 6 : 4) : 1024 / TH) residual_row_kernel(
    const T* __restrict__ z, long long ldz, const int* __restrict__ y, T* __restrict__ out, long long ldo, float* __restrict__ loss,
    long long rows, int C, float scale, int R) {
    constexpr int VE = Piece<T>::kValues;
    __shared__ float cells[2][TH / 32 + 1];
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

    float top = fmaxf(edge, -INFINITY);  // (NaN left aside)
#pragma unroll
    for (int k = 0; k < NV; ++k)
        if (tid + k * TH < count) top = piece_max(top, w[k], T());
    top = row_join<TH, true>(top, cells[0], tid, R);
    // (the difference by itself, not folded into a multiply-add: it is exact next to the largest logit, so that a row with one
    // class left has probability one and no gradient, and it cannot overflow)
    const float m = against(top);
    auto power = [&](float x) { return exp_fast(x - m); };
    const Pair minus_m(-m, -m), log2e(kLog2e, kLog2e);
    Pair sums(power(edge), 0.f);  // (-inf gives zero)
#pragma unroll
    for (int k = 0; k < NV; ++k)
        if (tid + k * TH < count) piece_powers<T>(w[k], minus_m, log2e, [&](int, const Pair& p) { sums = sums + p; });
    const float sum = row_join<TH, false>(sums.both().x + sums.both().y, cells[1], tid, R);
    if (TH > 32 && R > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");  // this block has read the others' cells
    const bool counts = row_counts(MaxSum{top, sum}, label, C);
    const float factor = scale / sum;
    const bool same = (((uintptr_t)zi ^ (uintptr_t)oi) & 15u) == 0;
    T* dst = oi + head + (long long)begin * VE;
#pragma unroll
    for (int k = 0; k < NV; ++k)
        if (tid + k * TH < count) {
            const int v = tid + k * TH;
            uint4 q = make_uint4(0, 0, 0, 0);
            T* t = reinterpret_cast<T*>(&q);
            if (counts) piece_powers<T>(w[k], minus_m, log2e, [&](int e, const Pair& p) { put_pair<T>(t + e, p * Pair(factor, factor)); });
            if (same) {
                __stcs(reinterpret_cast<uint4*>(dst) + v, q);
            } else {
#pragma unroll
                for (int e = 0; e < VE; ++e) dst[(long long)v * VE + e] = t[e];
            }
        }
    if (odd) oi[at] = from_f32<T>(counts ? power(edge) * factor : 0.f);
    // the label's own value is put right by the thread that has just written it
    const int piece = (label - head) / VE - begin;
    const bool mine = label >= head && label < head + pieces * VE ? piece >= 0 && piece < count && piece % TH == tid : odd && at == label;
    if (counts && mine) {
        const float x = to_f32(zi[label]);
        oi[label] = from_f32<T>(power(x) * factor - scale);
        if (loss) loss[i] = logf(sum) + (m - x);
    }
    if (!counts && rank == 0 && tid == 0 && loss) loss[i] = 0.f;
    if (TH > 32 && R > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// ---- longer rows than a block's registers hold: a block per row, the row read twice.  The second time it comes from L2, so that
// memory sees one read and one write, as long as the rows under way fit there: 1024 / TH blocks to an SM, TH growing
// with the row.  Measured: 8191 x 50257 in bf16 (100 KB a row) with 256 threads 326 us (5.05 TB/s), with 512 threads 370,
// held in the registers of clusters of two blocks 443; 4096 x 50257 in fp32 (200 KB) 356 with 256 threads, 295 with 512.
template <typename T, int TH>
__global__ void __launch_bounds__(TH, 1024 / TH) residual_long_kernel(const T* __restrict__ z, long long ldz, const int* __restrict__ y,
                                                                        T* __restrict__ out, long long ldo, float* __restrict__ loss,
                                                                        long long rows, int C, float scale) {
    constexpr int VE = Piece<T>::kValues, kAhead = 4;  // pieces a thread has under way
    __shared__ MaxSum part[TH / 32];
    const Pair log2e(kLog2e, kLog2e);
    const int tid = threadIdx.x;
    for (long long i = blockIdx.x; i < rows; i += gridDim.x) {
        const T* zi = z + i * ldz;
        T* oi = out + i * ldo;
        const int head = min(C, (int)(((16u - ((uintptr_t)zi & 15u)) & 15u) / sizeof(T)));
        const int pieces = (C - head) / VE, edges = C - pieces * VE;
        const uint4* src = reinterpret_cast<const uint4*>(zi + head);
        const bool odd = tid < edges;
        const int at = tid < head ? tid : tid + pieces * VE;
        const float edge = odd ? to_f32(zi[at]) : -INFINITY;
        MaxSum a{fmaxf(edge, -INFINITY), 0.f};
        a.s = exp_fast(edge - against(a.m));
        uint4 w[kAhead], next[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (tid + k * TH < pieces) next[k] = src[tid + k * TH];
        for (int k0 = tid; k0 < pieces; k0 += kAhead * TH) {
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                w[k] = next[k];
                if (k0 + (kAhead + k) * TH < pieces) next[k] = src[k0 + (kAhead + k) * TH];
            }
            float top = a.m;
#pragma unroll
            for (int k = 0; k < kAhead; ++k)
                if (k0 + k * TH < pieces) top = piece_max(top, w[k], T());
            const float m = against(top);
            Pair sums(a.s * carry(a.m, top), 0.f);
            a.m = top;
#pragma unroll
            for (int k = 0; k < kAhead; ++k)
                if (k0 + k * TH < pieces) piece_powers<T>(w[k], Pair(-m, -m), log2e, [&](int, const Pair& p) { sums = sums + p; });
            a.s = sums.both().x + sums.both().y;
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k)  // the second reading begins while the sums are joined
            if (tid + k * TH < pieces) next[k] = __ldcs(src + tid + k * TH);
        a = join_lanes(a, 32);
        __syncthreads();  // the row before this one has read its sums
        if ((tid & 31) == 0) part[tid >> 5] = a;
        __syncthreads();
        a = part[0];
#pragma unroll
        for (int k = 1; k < TH / 32; ++k) a = join(a, part[k]);
        const int label = y[i];
        const bool counts = row_counts(a, label, C), same = (((uintptr_t)zi ^ (uintptr_t)oi) & 15u) == 0;
        const float m = against(a.m), factor = scale / a.s;
        T* dst = oi + head;
        for (int k0 = tid; k0 < pieces; k0 += kAhead * TH) {
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                w[k] = next[k];
                if (k0 + (kAhead + k) * TH < pieces) next[k] = __ldcs(src + k0 + (kAhead + k) * TH);
            }
#pragma unroll
            for (int k = 0; k < kAhead; ++k)
                if (k0 + k * TH < pieces) {
                    const int v = k0 + k * TH;
                    uint4 q = make_uint4(0, 0, 0, 0);
                    T* t = reinterpret_cast<T*>(&q);
                    if (counts) piece_powers<T>(w[k], Pair(-m, -m), log2e, [&](int e, const Pair& p) { put_pair<T>(t + e, p * Pair(factor, factor)); });
                    if (same) {
                        __stcs(reinterpret_cast<uint4*>(dst) + v, q);
                    } else {
#pragma unroll
                        for (int e = 0; e < VE; ++e) dst[(long long)v * VE + e] = t[e];
                    }
                }
        }
        if (odd) oi[at] = from_f32<T>(counts ? exp_fast(edge - m) * factor : 0.f);
        // the label's own value is put right by the thread that has just written it
        const int piece = (label - head) / VE;
        if (counts && (label >= head && label < head + pieces * VE ? piece % TH == tid : odd && at == label)) {
            const float x = to_f32(zi[label]);
            oi[label] = from_f32<T>(exp_fast(x - m) * factor - scale);
            if (loss) loss[i] = row_loss(a, x);
        }
        if (!counts && tid == 0 && loss) loss[i] = 0.f;
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
