// Tensor-core contractions of the gated feed-forward block (bmgd_gated_ffn_forward, bmgd_gated_ffn_backward).
//
//   forward    G = X Wg, U = X Wu, H = act(G) * U      one kernel: a tile holds the same columns of G and U side by side,
//              Y = H Wd                                 so the product is taken where the accumulators are read out
//   backward   dH = dY Wd^T, dU = dH act(G), dG = dH (U act'(G))  one kernel; the two factors come from the forward pass
//              dX = dG Wg^T + dU Wu^T                   one accumulator, the second product continues the first
//              dWg = X^T dG, dWu = X^T dU               one launch over both
//              dWd = H^T dY
// Rows of every matrix are contiguous.  Both ways of reading a tile exist for each operand: "K-major", the contraction
// index along the rows, or "MN-major", across them; nothing is transposed in memory.  H, dG and dU are rounded to the type
// of the rows between the kernels (they are the operands of the next contraction, which takes no other type); sums are fp32
// in tensor memory, and act(G) and U act'(G) are kept in fp32 for the backward pass: rounded to 16 bits they would add as much
// to the gradients' error as both other roundings together, and their traffic hides behind the arithmetic.
//
// What bounds it: the tensor cores, from a few hundred rows on.  Warp 0 copies tiles of 64 along the contraction by TMA
// into a ring of stages with the 128-byte swizzle, warp 1 issues tcgen05.mma, warps 4 to 7 read accumulators out of
// tensor memory; two accumulators take turns, so that reading one out overlaps the next tile's arithmetic.  With
// CG = 2 two CTAs of a cluster work on one tile of 256 rows: each fetches its 128 rows of A and half of B, and the
// even one issues for both.
#pragma once
#include <cstdint>
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "softmax_kernel.cuh"

namespace bmgdk {

enum { kActSilu = 0, kActGelu = 1, kActRelu = 2, kActSigmoid = 3 };
enum { kEpiGated = 0, kEpiPlain = 1, kEpiBackward = 2 };

constexpr int kFfnThreads = 256;
constexpr int kFfnBK = 64;
constexpr int kTurnPitch = 36;  // words per row there: 32 and four, so that eight lanes' 16-byte accesses meet no bank twice
constexpr int kFfnGroup = 8;  // tiles along M that are worked on together: their rows of A stay in L2 while B passes

struct FfnParams {
    CUtensorMap a[2], b[2];  // second pair: the second half of the contraction (segments = 2) or of the launch (problems = 2)
    void* out[2];            // plain: D of problem 0 and 1.  gated: H.  backward: dG, dU
    long long ld_out;
    float* value;            // act(G) and U act'(G): written by the gated form (null: not wanted), read by the backward one
    float* slope;
    long long ld_save;
    long long M;
    int N, K;
    int segments, problems;
    int tiles_m, tiles_n;
    int type, act;
    int vec;                 // plain: all rows of the outputs start on 16-byte boundaries
    int* status;
    unsigned long long timeout_ns;
};

struct FfnWait {
    int* status;
    unsigned long long timeout_ns;
    bool aborted;
};
__device__ __forceinline__ void ffn_wait(uint32_t bar, uint32_t parity, FfnWait& w) {
    if (w.aborted || mbar_try_wait(bar, parity)) return;
    const unsigned long long t0 = global_ns();
    uint32_t spins = 0;
    while (!mbar_try_wait(bar, parity)) {
        if ((++spins & 0xFFu) == 0u && (global_ns() - t0 >= w.timeout_ns || ((volatile int*)w.status)[0] != 0)) {
            atomicCAS(w.status, 0, kStatusTimeout);
            w.aborted = true;
            return;
        }
    }
}

__device__ __forceinline__ uint32_t leader_addr(uint32_t addr) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(addr));
    return r;
}
template <int CG>
__device__ __forceinline__ void ffn_tma(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
    if constexpr (CG == 1)
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                     ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3}], [%4];"
                     ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
template <int CG>
__device__ __forceinline__ void ffn_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    if constexpr (CG == 1)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
// one arrival on `bar` (of both CTAs with CG = 2) once everything issued so far has finished
template <int CG>
__device__ __forceinline__ void ffn_commit(uint32_t bar) {
    if constexpr (CG == 1)
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                     ::"r"(bar), "h"((uint16_t)3) : "memory");
}
template <int CG>
__device__ __forceinline__ void ffn_tmem_alloc(uint32_t dst, uint32_t cols) {
    if constexpr (CG == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dst), "r"(cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    } else {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dst), "r"(cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
}
template <int CG>
__device__ __forceinline__ void ffn_tmem_free(uint32_t addr, uint32_t cols) {
    if constexpr (CG == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(cols));
    else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(cols));
}
// 16 or 32 consecutive fp32 columns of this thread's lane; the caller waits with tmem_wait before it uses them
__device__ __forceinline__ void tmem_load16(uint32_t addr, uint32_t* r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(addr) : "memory");
}
__device__ __forceinline__ void tmem_load32(uint32_t addr, uint32_t* r) {
    tmem_load16(addr, r);
    tmem_load16(addr + 16, r + 16);
}
__device__ __forceinline__ void tmem_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

// ---------------------------------------------------------------- activation
// act(g) and act'(g) in fp32 (silu g s, gelu g Phi(g), relu, sigmoid s; s = 1 / (1 + exp(-g)))
__device__ __forceinline__ float act_value(int act, float g) {
    if (act == kActRelu) return g > 0.f ? g : g * 0.f;  // (0 times NaN stays NaN)
    if (act == kActGelu) return 0.5f * g * (1.f + erff(g * 0.70710678118654752f));
    const float s = __fdividef(1.f, 1.f + __expf(-g));
    return act == kActSigmoid ? s : g * s;
}
__device__ __forceinline__ void act_both(int act, float g, float& value, float& slope) {
    if (act == kActRelu) {
        value = g > 0.f ? g : g * 0.f;
        slope = g > 0.f ? 1.f : g * 0.f;
    } else if (act == kActGelu) {
        const float cdf = 0.5f * (1.f + erff(g * 0.70710678118654752f));
        value = g * cdf;
        slope = cdf + g * __expf(-0.5f * g * g) * 0.3989422804014327f;
    } else {
        const float s = __fdividef(1.f, 1.f + __expf(-g));
        if (act == kActSigmoid) { value = s; slope = s * (1.f - s); }
        else { value = g * s; slope = s * (1.f + g * (1.f - s)); }
    }
}

__device__ __forceinline__ uint32_t pack2(int type, float a, float b) {
    if (type == BMGD_TYPE_BF16) {
        const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&v);
    }
    const __half2 v = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
}
// ---------------------------------------------------------------- shapes
template <int CG, int BN>
struct FfnShape {
    static constexpr int kA = 128 * kFfnBK * 2;            // bytes of A per stage and CTA
    static constexpr int kB = BN / CG * kFfnBK * 2;        // bytes of B per stage and CTA
    static constexpr int kStage = kA + kB;
    static constexpr int kStages = kStage > 40960 ? 4 : 6;
    static constexpr int kBars = kStages * kStage;         // mbarriers and the tensor-memory address behind the ring
    static constexpr int kTurn = kBars + 256;              // where a warp turns rows per lane into pieces of rows per lane
    static constexpr int kSmem = kTurn + 4 * 32 * kTurnPitch * 4 + 1024;  // (1024: the ring starts on a 1024-byte boundary)
};

// fetch `ROWS` rows (K-major) or columns (MN-major) of an operand, from `mn` on, 64 along the contraction from `k` on
template <int CG, bool MN_MAJOR, int ROWS>
__device__ __forceinline__ void ffn_fetch(uint32_t dst, const CUtensorMap* map, int mn, int k, uint32_t bar) {
    if constexpr (MN_MAJOR) {
#pragma unroll
        for (int i = 0; i < ROWS / 64; ++i) ffn_tma<CG>(dst + (uint32_t)(i * 64 * 128), map, mn + i * 64, k, bar);
    } else {
        ffn_tma<CG>(dst, map, k, mn, bar);  // the map's box has ROWS rows
    }
}

// ---------------------------------------------------------------- the kernel
// EPI: what is done with a tile.  A_MN, B_MN: the operand is read across its rows.  BN: columns of a tile (gated: BN / 2
// of G and as many of U).
template <int CG, int BN, int EPI, bool A_MN, bool B_MN>
__global__ void __launch_bounds__(kFfnThreads, 1) ffn_kernel(const __grid_constant__ FfnParams P) {
    using S = FfnShape<CG, BN>;
    extern __shared__ unsigned char ffn_smem[];
    const uint32_t ring = (smem_u32(ffn_smem) + 1023u) & ~1023u;
    const uint32_t full = ring + S::kBars, empty = full + 8 * S::kStages, acc_full = empty + 8 * S::kStages, acc_empty = acc_full + 16;
    const uint32_t slot = acc_empty + 16;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = CG == 2 ? cluster_ctarank() : 0u;
    const int pair = (int)blockIdx.x / CG, pairs = (int)gridDim.x / CG;
    constexpr int kCols = EPI == kEpiGated ? BN / 2 : BN;   // columns of the output that a tile covers
    constexpr uint32_t kTmemCols = 2 * BN;

    if (threadIdx.x == 0) {
        for (int s = 0; s < S::kStages; ++s) { mbar_init(full + 8 * s, 1); mbar_init(empty + 8 * s, 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(acc_full + 8 * i, 1); mbar_init(acc_empty + 8 * i, 4 * CG); }
        fence_barrier_init();
    }
    if (warp == 2) ffn_tmem_alloc<CG>(slot, kTmemCols);
    tc_fence_before();
    __syncthreads();
    if constexpr (CG == 2) { cluster_arrive_release(); cluster_wait_acquire(); }
    tc_fence_after();
    uint32_t tmem;
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(tmem) : "r"(slot));

    const long long per_problem = (long long)P.tiles_m * P.tiles_n;
    const long long tiles = per_problem * P.problems;
    const int kblocks = (P.K + kFfnBK - 1) / kFfnBK, steps = kblocks * P.segments;
    auto place = [&](long long t, int& which, long long& m0, int& n0) {
        which = (int)(t / per_problem);
        const long long r = t - which * per_problem, g = r / ((long long)kFfnGroup * P.tiles_n);
        const int first = (int)g * kFfnGroup, gm = min(kFfnGroup, P.tiles_m - first);
        const int r2 = (int)(r - g * kFfnGroup * P.tiles_n);
        m0 = (long long)(first + r2 % gm) * (128 * CG);
        n0 = (r2 / gm) * kCols;
    };
    FfnWait w{P.status, P.timeout_ns, false};

    if (warp == 0) {
        if (lane == 0) {
            int s = 0;
            uint32_t phase = 0;
            for (long long t = pair; t < tiles && !w.aborted; t += pairs) {
                int which, n0;
                long long m0;
                place(t, which, m0, n0);
                const int am = (int)m0 + (int)rank * 128;
                for (int k = 0; k < steps; ++k) {
                    ffn_wait(empty + 8 * s, phase ^ 1u, w);
                    if (w.aborted) break;
                    const int seg = k >= kblocks ? 1 : 0, k0 = (k - seg * kblocks) * kFfnBK;
                    uint32_t bar = full + 8 * s;
                    if (rank == 0) mbar_arrive_expect_tx(bar, S::kStage * CG);
                    if constexpr (CG == 2) bar = leader_addr(bar);
                    const uint32_t sa = ring + s * S::kStage, sb = sa + S::kA;
                    ffn_fetch<CG, A_MN, 128>(sa, &P.a[seg], am, k0, bar);
                    if constexpr (EPI == kEpiGated) {
                        // the first half of the tile's columns is G, the second U; with two CTAs one fetches each
                        if constexpr (CG == 2) ffn_fetch<CG, B_MN, BN / 2>(sb, &P.b[rank], n0, k0, bar);
                        else {
                            ffn_fetch<CG, B_MN, BN / 2>(sb, &P.b[0], n0, k0, bar);
                            ffn_fetch<CG, B_MN, BN / 2>(sb + S::kB / 2, &P.b[1], n0, k0, bar);
                        }
                    } else {
                        ffn_fetch<CG, B_MN, BN / CG>(sb, &P.b[seg + which], n0 + (int)rank * (BN / CG), k0, bar);
                    }
                    if (++s == S::kStages) { s = 0; phase ^= 1u; }
                }
            }
        }
    } else if (warp == 1) {
        if (lane == 0 && rank == 0) {
            const uint32_t fmt = P.type == BMGD_TYPE_BF16 ? 1u : 0u;
            const uint32_t idesc = (1u << 4) | (fmt << 7) | (fmt << 10) | ((A_MN ? 1u : 0u) << 15) | ((B_MN ? 1u : 0u) << 16) |
                                   ((uint32_t)(BN >> 3) << 17) | ((uint32_t)(128 * CG >> 4) << 24);
            int s = 0, acc = 0;
            uint32_t phase = 0, acc_phase = 0;
            for (long long t = pair; t < tiles && !w.aborted; t += pairs) {
                ffn_wait(acc_empty + 8 * acc, acc_phase ^ 1u, w);
                tc_fence_after();
                for (int k = 0; k < steps && !w.aborted; ++k) {
                    ffn_wait(full + 8 * s, phase, w);
                    if (w.aborted) break;
                    tc_fence_after();
                    const uint32_t sa = ring + s * S::kStage, sb = sa + S::kA;
#pragma unroll
                    for (int i = 0; i < kFfnBK / 16; ++i) {
                        const uint64_t da = A_MN ? tc_smem_desc(sa + i * 2048, 64 * 128, 1024) : tc_smem_desc(sa + i * 32, 16, 1024);
                        const uint64_t db = B_MN ? tc_smem_desc(sb + i * 2048, 64 * 128, 1024) : tc_smem_desc(sb + i * 32, 16, 1024);
                        ffn_mma<CG>(tmem + (uint32_t)(acc * BN), da, db, idesc, (k | i) != 0 ? 1u : 0u);
                    }
                    ffn_commit<CG>(empty + 8 * s);
                    if (++s == S::kStages) { s = 0; phase ^= 1u; }
                }
                if (w.aborted) break;
                ffn_commit<CG>(acc_full + 8 * acc);
                if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
            }
        }
    } else if (warp >= 4) {
        // A lane reads a row out of tensor memory; what a warp writes to (or reads from) global memory at a time should be
        // pieces of rows.  In between the values take turns through shared memory, 32 to a row.
        int acc = 0;
        uint32_t acc_phase = 0;
        const int quarter = warp & 3;
        float* const turn = reinterpret_cast<float*>(ffn_smem + (ring - smem_u32(ffn_smem)) + S::kTurn) + quarter * 32 * kTurnPitch;
        for (long long t = pair; t < tiles; t += pairs) {
            int which, n0;
            long long m0;
            place(t, which, m0, n0);
            ffn_wait(acc_full + 8 * acc, acc_phase, w);
            w.aborted = __any_sync(0xFFFFFFFFu, w.aborted);
            if (w.aborted) break;
            tc_fence_after();
            const long long row0 = m0 + (long long)rank * 128 + quarter * 32;
            const int rows = (int)min(32ll, P.M - row0);  // (may be negative)
            const uint32_t ta = tmem + (uint32_t)(acc * BN) + ((uint32_t)(quarter * 32) << 16);
            if constexpr (EPI == kEpiGated) {
                // 16 columns of G and 16 of U at a time; then a lane has four columns of rows lane / 4, lane / 4 + 8, ...
                const int sub = (lane & 3) * 4;
#pragma unroll 1
                for (int c = 0; c < kCols; c += 16) {
                    const int col = n0 + c;
                    if (col >= P.N) break;
                    uint32_t r[32];
                    tmem_load16(ta + (uint32_t)c, r);
                    tmem_load16(ta + (uint32_t)(BN / 2 + c), r + 16);
                    tmem_wait();
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        *reinterpret_cast<uint4*>(turn + lane * kTurnPitch + 4 * i) = make_uint4(r[4 * i], r[4 * i + 1], r[4 * i + 2], r[4 * i + 3]);
                    __syncwarp();
#pragma unroll
                    for (int it = 0; it < 4; ++it) {
                        const int i = it * 8 + (lane >> 2);
                        if (i < rows && col + sub < P.N) {  // (rows of H, act(G) and U act'(G) are padded to multiples of 8)
                            const float4 g = *reinterpret_cast<const float4*>(turn + i * kTurnPitch + sub);
                            const float4 u = *reinterpret_cast<const float4*>(turn + i * kTurnPitch + 16 + sub);
                            float4 v, s;
                            if (P.value) {
                                act_both(P.act, g.x, v.x, s.x); act_both(P.act, g.y, v.y, s.y);
                                act_both(P.act, g.z, v.z, s.z); act_both(P.act, g.w, v.w, s.w);
                                const long long at = (row0 + i) * P.ld_save + col + sub;
                                *reinterpret_cast<float4*>(P.value + at) = v;
                                *reinterpret_cast<float4*>(P.slope + at) = make_float4(u.x * s.x, u.y * s.y, u.z * s.z, u.w * s.w);
                            } else {
                                v = make_float4(act_value(P.act, g.x), act_value(P.act, g.y), act_value(P.act, g.z), act_value(P.act, g.w));
                            }
                            *reinterpret_cast<uint2*>(static_cast<uint16_t*>(P.out[0]) + (row0 + i) * P.ld_out + col + sub) =
                                make_uint2(pack2(P.type, v.x * u.x, v.y * u.y), pack2(P.type, v.z * u.z, v.w * u.w));
                        }
                    }
                    __syncwarp();
                }
            } else if constexpr (EPI == kEpiBackward) {
                const int sub = (lane & 7) * 4;
#pragma unroll 1
                for (int c = 0; c < kCols; c += 32) {
                    const int col = n0 + c;
                    if (col >= P.N) break;
                    float4 v[8], s[8];
#pragma unroll
                    for (int it = 0; it < 8; ++it) {
                        const int i = it * 4 + (lane >> 3);
                        const long long at = (row0 + i) * P.ld_save + col + sub;
                        if (i < rows && col + sub < P.N) {
                            v[it] = __ldcs(reinterpret_cast<const float4*>(P.value + at));
                            s[it] = __ldcs(reinterpret_cast<const float4*>(P.slope + at));
                        }
                    }
                    uint32_t r[32];
                    tmem_load32(ta + (uint32_t)c, r);
                    tmem_wait();
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        *reinterpret_cast<uint4*>(turn + lane * kTurnPitch + 4 * i) = make_uint4(r[4 * i], r[4 * i + 1], r[4 * i + 2], r[4 * i + 3]);
                    __syncwarp();
#pragma unroll
                    for (int it = 0; it < 8; ++it) {
                        const int i = it * 4 + (lane >> 3);
                        if (i < rows && col + sub < P.N) {
                            const float4 d = *reinterpret_cast<const float4*>(turn + i * kTurnPitch + sub);
                            const long long at = (row0 + i) * P.ld_out + col + sub;
                            *reinterpret_cast<uint2*>(static_cast<uint16_t*>(P.out[0]) + at) =
                                make_uint2(pack2(P.type, d.x * s[it].x, d.y * s[it].y), pack2(P.type, d.z * s[it].z, d.w * s[it].w));
                            *reinterpret_cast<uint2*>(static_cast<uint16_t*>(P.out[1]) + at) =
                                make_uint2(pack2(P.type, d.x * v[it].x, d.y * v[it].y), pack2(P.type, d.z * v[it].z, d.w * v[it].w));
                        }
                    }
                    __syncwarp();
                }
            } else {
                uint16_t* const out = static_cast<uint16_t*>(P.out[which]);
                uint16_t* const half = reinterpret_cast<uint16_t*>(turn);  // 32 16-bit values to a row here, 40 apart
#pragma unroll 1
                for (int c = 0; c < kCols; c += 32) {
                    const int col = n0 + c;
                    if (col >= P.N) break;
                    uint32_t r[32];
                    tmem_load32(ta + (uint32_t)c, r);
                    tmem_wait();
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        uint32_t q[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) q[j] = pack2(P.type, __uint_as_float(r[8 * i + 2 * j]), __uint_as_float(r[8 * i + 2 * j + 1]));
                        *reinterpret_cast<uint4*>(half + lane * 40 + 8 * i) = make_uint4(q[0], q[1], q[2], q[3]);
                    }
                    __syncwarp();
                    if (P.vec && col + 32 <= P.N) {
#pragma unroll
                        for (int it = 0; it < 4; ++it) {
                            const int i = it * 8 + (lane >> 2), sub = (lane & 3) * 8;
                            if (i < rows)
                                *reinterpret_cast<uint4*>(out + (row0 + i) * P.ld_out + col + sub) = *reinterpret_cast<const uint4*>(half + i * 40 + sub);
                        }
                    } else if (col + lane < P.N) {
#pragma unroll 8
                        for (int i = 0; i < rows; ++i) out[(row0 + i) * P.ld_out + col + lane] = half[i * 40 + lane];
                    }
                    __syncwarp();
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if constexpr (CG == 2)
                    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(leader_addr(acc_empty + 8 * acc)) : "memory");
                else mbar_arrive(acc_empty + 8 * acc);
            }
            if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
        }
    }
    __syncwarp();
    if (__any_sync(0xFFFFFFFFu, w.aborted)) {  // given up: copies and products may still be in flight
        const unsigned long long t0 = global_ns();
        while (global_ns() - t0 < kSmxLingerNs) __nanosleep(1000);
    }
    tc_fence_before();
    __syncthreads();
    if constexpr (CG == 2) { cluster_arrive_release(); cluster_wait_acquire(); }
    tc_fence_after();
    if (warp == 2) ffn_tmem_free<CG>(tmem, kTmemCols);
}

// rows of `cols` 16-bit values from stride ld to stride ld_out >= cols, the rest of each row zero: for operands whose
// rows do not start on 16-byte boundaries, which TMA cannot read
__global__ void __launch_bounds__(256) ffn_align_kernel(const uint16_t* __restrict__ in, long long ld, uint16_t* __restrict__ out,
                                                        long long ld_out, long long rows, int cols) {
    const long long total = rows * ld_out;
    for (long long i = blockIdx.x * 256ll + threadIdx.x; i < total; i += gridDim.x * 256ll) {
        const long long r = i / ld_out;
        const int c = (int)(i - r * ld_out);
        out[i] = c < cols ? in[r * ld + c] : (uint16_t)0;
    }
}

}  // namespace bmgdk
