// Tensor-core contractions of the gated feed-forward block (bmgd_gated_ffn_forward, bmgd_gated_ffn_backward).
//
//   forward    G = X Wg, U = X Wu, H = act(G) * U      one kernel: a tile holds the same columns of G and U side by side,
//              Y = H Wd                                 so the product is taken where the accumulators are read out
//   backward   dH = dY Wd^T, dU = dH act(G), dG = dH U act'(G)   one kernel; H is formed again on the way
//              dX = dG Wg^T + dU Wu^T                   one accumulator, the second product continues the first
//              dWg = X^T dG, dWu = X^T dU               one launch over both
//              dWd = H^T dY
// Rows of every matrix are contiguous.  Both ways of reading a tile exist for each operand: "K-major", the contraction
// index along the rows, or "MN-major", across them; nothing is transposed in memory.  G, U, dG, dU and H are rounded to
// the type of the rows between the kernels (they are the operands of the next contraction, which takes no other type);
// sums are fp32 in tensor memory.
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
constexpr int kFfnGroup = 8;  // tiles along M that are worked on together: their rows of A stay in L2 while B passes

struct FfnParams {
    CUtensorMap a[2], b[2];  // second pair: the second half of the contraction (segments = 2) or of the launch (problems = 2)
    void* out[2];            // plain: D of problem 0 and 1.  gated: H.  backward: dG, dU
    long long ld_out;
    void* gate;              // gated: G and U to save (null: not saved).  backward: read
    void* up;
    long long ld_save;
    void* h;                 // backward: H
    long long ld_h;
    long long M;
    int N, K;
    int segments, problems;
    int tiles_m, tiles_n;
    int type, act;
    int vec;                 // all rows of the outputs (and of G and U) start on 16-byte boundaries
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
// 32 consecutive fp32 columns of this thread's lane; the caller waits with tmem_wait before it uses them
__device__ __forceinline__ void tmem_load32(uint32_t addr, uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, "
        "%18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
          "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
          "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr) : "memory");
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
        slope = g > 0.f ? 1.f : 0.f;
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
__device__ __forceinline__ float2 unpack2(int type, uint32_t w) {
    if (type == BMGD_TYPE_BF16) return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
    return __half22float2(*reinterpret_cast<__half2*>(&w));
}
// 32 columns of one row: columns from N on are left alone
__device__ __forceinline__ void store32(void* base, long long ld, long long row, int col, int N, int type, bool vec, const float (&x)[32]) {
    uint16_t* p = static_cast<uint16_t*>(base) + row * ld + col;
    if (vec && col + 32 <= N) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            reinterpret_cast<uint4*>(p)[i] = make_uint4(pack2(type, x[8 * i], x[8 * i + 1]), pack2(type, x[8 * i + 2], x[8 * i + 3]),
                                                        pack2(type, x[8 * i + 4], x[8 * i + 5]), pack2(type, x[8 * i + 6], x[8 * i + 7]));
    } else {
#pragma unroll
        for (int i = 0; i < 32; ++i)
            if (col + i < N) p[i] = (uint16_t)pack2(type, x[i], 0.f);
    }
}
__device__ __forceinline__ void load32(const void* base, long long ld, long long row, int col, int N, bool vec, uint32_t (&w)[16]) {
    const uint16_t* p = static_cast<const uint16_t*>(base) + row * ld + col;
    if (vec && col + 32 <= N) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint4 v = reinterpret_cast<const uint4*>(p)[i];
            w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const uint32_t lo = col + 2 * i < N ? p[2 * i] : 0u, hi = col + 2 * i + 1 < N ? p[2 * i + 1] : 0u;
            w[i] = lo | (hi << 16);
        }
    }
}

// ---------------------------------------------------------------- shapes
template <int CG, int BN>
struct FfnShape {
    static constexpr int kA = 128 * kFfnBK * 2;            // bytes of A per stage and CTA
    static constexpr int kB = BN / CG * kFfnBK * 2;        // bytes of B per stage and CTA
    static constexpr int kStage = kA + kB;
    static constexpr int kStages = kStage > 40960 ? 4 : 6;
    static constexpr int kBars = kStages * kStage;         // mbarriers and the tensor-memory address behind the ring
    static constexpr int kSmem = kBars + 256 + 1024;       // (1024: the ring starts on a 1024-byte boundary)
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
        int acc = 0;
        uint32_t acc_phase = 0;
        const int quarter = warp & 3;
        const bool vec = P.vec != 0;
        for (long long t = pair; t < tiles; t += pairs) {
            int which, n0;
            long long m0;
            place(t, which, m0, n0);
            ffn_wait(acc_full + 8 * acc, acc_phase, w);
            w.aborted = __any_sync(0xFFFFFFFFu, w.aborted);
            if (w.aborted) break;
            tc_fence_after();
            const long long row = m0 + (long long)rank * 128 + quarter * 32 + lane;
            const bool in = row < P.M;
            const uint32_t ta = tmem + (uint32_t)(acc * BN) + ((uint32_t)(quarter * 32) << 16);
#pragma unroll 1
            for (int c = 0; c < kCols; c += 32) {
                const int col = n0 + c;
                if (col >= P.N) break;
                if constexpr (EPI == kEpiGated) {
                    uint32_t rg[32], ru[32];
                    tmem_load32(ta + (uint32_t)c, rg);
                    tmem_load32(ta + (uint32_t)(BN / 2 + c), ru);
                    tmem_wait();
                    if (in) {
                        float g[32], u[32];
#pragma unroll
                        for (int i = 0; i < 32; ++i) { g[i] = __uint_as_float(rg[i]); u[i] = __uint_as_float(ru[i]); }
                        if (P.gate) {
                            store32(P.gate, P.ld_save, row, col, P.N, P.type, vec, g);
                            store32(P.up, P.ld_save, row, col, P.N, P.type, vec, u);
                        }
#pragma unroll
                        for (int i = 0; i < 32; ++i) g[i] = act_value(P.act, g[i]) * u[i];
                        store32(P.out[0], P.ld_out, row, col, P.N, P.type, vec, g);
                    }
                } else if constexpr (EPI == kEpiPlain) {
                    uint32_t r[32];
                    tmem_load32(ta + (uint32_t)c, r);
                    tmem_wait();
                    if (in) {
                        float x[32];
#pragma unroll
                        for (int i = 0; i < 32; ++i) x[i] = __uint_as_float(r[i]);
                        store32(P.out[which], P.ld_out, row, col, P.N, P.type, vec, x);
                    }
                } else {
                    uint32_t r[32], wg[16], wu[16];
                    tmem_load32(ta + (uint32_t)c, r);
                    if (in) {
                        load32(P.gate, P.ld_save, row, col, P.N, vec, wg);
                        load32(P.up, P.ld_save, row, col, P.N, vec, wu);
                    }
                    tmem_wait();
                    if (in) {
                        float dg[32], du[32], h[32];
#pragma unroll
                        for (int i = 0; i < 32; ++i) {
                            const float2 g2 = unpack2(P.type, wg[i >> 1]), u2 = unpack2(P.type, wu[i >> 1]);
                            const float g = i & 1 ? g2.y : g2.x, u = i & 1 ? u2.y : u2.x, d = __uint_as_float(r[i]);
                            float value, slope;
                            act_both(P.act, g, value, slope);
                            h[i] = value * u;
                            du[i] = d * value;
                            dg[i] = d * u * slope;
                        }
                        store32(P.out[0], P.ld_out, row, col, P.N, P.type, vec, dg);
                        store32(P.out[1], P.ld_out, row, col, P.N, P.type, vec, du);
                        store32(P.h, P.ld_h, row, col, P.N, P.type, vec, h);
                    }
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
