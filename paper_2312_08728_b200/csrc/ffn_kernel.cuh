// Tensor-core contractions of the gated feed-forward block (bmgd_gated_ffn_forward, bmgd_gated_ffn_backward).
//
//   forward    G = X Wg, U = X Wu, H = act(G) * U      one kernel: a tile holds the same columns of G and U side by side,
//              Y = H Wd                                 so the product is taken where the accumulators are read out
//   backward   dH = dY Wd^T, dU = dH act(G), dG = dH (U act'(G))  one kernel; the two factors come from the forward pass
//              dX = dG Wg^T + dU Wu^T                   one accumulator, the second product continues the first
//              dWg = X^T dG, dWu = X^T dU, dWd = H^T dY  one launch over the three
// Rows of every matrix are contiguous.  Both ways of reading a tile exist for each operand: "K-major", the contraction
// index along the rows, or "MN-major", across them; nothing is transposed in memory.  H, dG and dU are rounded to the type
// of the rows between the kernels (they are the operands of the next contraction, which takes no other type; in fp16 values
// above 65,504 become Inf there); sums are fp32
// in tensor memory, and act(G) and U act'(G) are kept in fp32 for the backward pass: rounded to 16 bits they would add as much
// to the gradients' error as both other roundings together, and their traffic hides behind the arithmetic.
//
// What bounds it: the tensor cores, from a few hundred rows on (ffn_kernel); below, reading the weights once
// (ffn_few_kernel).
#pragma once
#include <cstdint>
#include <cuda.h>
#include <cuda_runtime.h>

#include "activation.cuh"
#include "contract.cuh"

namespace bmgdk {

enum { kEpiGated = 0, kEpiPlain = 1, kEpiBackward = 2 };

constexpr int kFfnBK = 64;
constexpr int kFfnGroup = 8;  // tiles along M that are worked on together: their rows of A stay in L2 while B passes
constexpr int kFfnProblems = 3;

// D [M][N] = sum over segments of A_s B_s
struct FfnProblem {
    CUtensorMap a[2], b[2];  // one per segment (gated: b[0] is Wg, b[1] is Wu)
    void* out;               // D, or H
    long long ld_out;
    long long first_tile;    // tiles of all problems before this one
    int M, N, K;
    int segments;
    int tiles_m, tiles_n;
    int a_mn;                // few rows: the weights are read across their rows
    int vec;                 // rows of D start on 16-byte boundaries
};

struct FfnParams {
    FfnProblem p[kFfnProblems];
    int problems;
    long long tiles;
    void* out_up;            // backward: dU beside dG
    float* value;            // act(G) and U act'(G): written by the gated form (null: not wanted), read by the backward one
    float* slope;
    long long ld_save;
    int type, act;
    int early;               // many rows: this launch needs nothing of the one before it, only of those before that
    unsigned fills;          // stages of its ring that a CTA fills: as many as there are, fewer only to test how waits run out
    unsigned* gave_up;       // counts waits that ran out of time
    unsigned long long timeout_ns;
};

template <int CG>
__device__ __forceinline__ void ffn_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    if constexpr (CG == 1)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
// ---------------------------------------------------------------- shapes
// Read-out: eight warps (with four the gated form that saves its factors kept the tensor cores waiting at 2048 inputs: 64 %
// active, and one stage of the ring less costs nothing there).  Each turns its values through a buffer of its own in shared
// memory, rows of kWords words.  The 16-byte pieces of a row stand in an order of the row's own (turn32), so that eight lanes meet no bank twice,
// neither those of eight rows that write the same piece nor those of two rows that read four pieces each.
template <int EPI>
struct FfnReadOut {
    static constexpr int kWarps = 8;
    static constexpr int kRows = EPI == kEpiBackward ? 16 : 32;
    static constexpr int kWords = 32;                           // plain: 64 values of 16 bits
    static constexpr int kCols = EPI == kEpiGated ? 16 : EPI == kEpiPlain ? 64 : 32;  // columns of the tile taken at a time
    static constexpr int kBytes = kWarps * kRows * kWords * 4;
    static constexpr int kThreads = 128 + kWarps * 32;
};
template <int CG, int BN, int EPI>
struct FfnShape {
    static constexpr int kA = 128 * kFfnBK * 2;            // bytes of A per stage and CTA
    static constexpr int kB = BN / CG * kFfnBK * 2;        // bytes of B per stage and CTA
    static constexpr int kStage = kA + kB;
    static constexpr int kStages = EPI == kEpiGated ? 5 : 6;
    static constexpr int kBars = kStages * kStage;         // mbarriers and the tensor-memory address behind the ring
    static constexpr int kTurn = kBars + 256;              // where a warp turns rows per lane into pieces of rows per lane
    static constexpr int kSmem = kTurn + FfnReadOut<EPI>::kBytes + 1024;  // (1024: the ring starts on a 1024-byte boundary)
};

// fetch `rows` rows (K-major) or columns (MN-major) of an operand, from `mn` on, 64 along the contraction from `k` on
template <int CG>
__device__ __forceinline__ void ffn_fetch(uint32_t dst, const CUtensorMap* map, bool mn_major, int rows, int mn, int k, uint32_t bar) {
    if (mn_major) {
#pragma unroll
        for (int i = 0; i < rows; i += 64) ffn_tma<CG>(dst + (uint32_t)(i * 128), map, mn + i, k, bar);
    } else {
        ffn_tma<CG>(dst, map, k, mn, bar);  // the map's box has that many rows
    }
}
// Descriptor of such a tile at address 0, and what one instruction's 16 along the contraction add to it.  One thread issues
// everything: whatever it computes between two instructions the tensor core may have to wait for.
struct FfnDesc {
    uint64_t base;
    uint32_t step;
    __device__ __forceinline__ explicit FfnDesc(bool mn_major)
        : base(mn_major ? tc_smem_desc(0, 64 * 128, 1024) : tc_smem_desc(0, 16, 1024)), step(mn_major ? 2048u >> 4 : 32u >> 4) {}
    // (a shared-memory address carries the CTA's rank in its cluster in the bits above the offset)
    __device__ __forceinline__ uint64_t at(uint32_t tile) const { return base + ((tile >> 4) & 0x3FFFu); }
};
__device__ __forceinline__ uint32_t ffn_idesc(int type, bool a_mn, bool b_mn, int m, int n) {
    const uint32_t fmt = type == BMGD_TYPE_BF16 ? 1u : 0u;
    return (1u << 4) | (fmt << 7) | (fmt << 10) | ((a_mn ? 1u : 0u) << 15) | ((b_mn ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) |
           ((uint32_t)(m >> 4) << 24);
}

// ---------------------------------------------------------------- many rows
// Warp 0 copies tiles of 64 along the contraction by TMA into a ring of stages with the 128-byte swizzle, warp 1 issues
// tcgen05.mma, warps 4 to 11 read accumulators out of tensor memory; two accumulators take turns, so that reading one out
// overlaps the next tile's arithmetic.  With CG = 2 two CTAs of a cluster work on one tile of 256 rows: each fetches its 128
// rows of A and half of B, and the even one issues for both.  The gradients of the three weights are problems of one
// launch: their tiles fill the GPU together.
// EPI: what is done with a tile.  BN: columns of a tile (gated: BN / 2 of G and as many of U).  A_MN, B_MN: an operand is
// read across its rows.  They are known when the kernel is compiled because one thread fetches and one thread issues for the whole
// tile: choosing at run time cost 5 % of the forward pass at 4096 rows and 13 % of the backward pass.
template <int CG, int BN, int EPI, bool A_MN, bool B_MN>
__global__ void __launch_bounds__(FfnReadOut<EPI>::kThreads, 1) ffn_kernel(const __grid_constant__ FfnParams P) {
    using S = FfnShape<CG, BN, EPI>;
    using R = FfnReadOut<EPI>;
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
        for (int i = 0; i < 2; ++i) { mbar_init(acc_full + 8 * i, 1); mbar_init(acc_empty + 8 * i, R::kWarps * CG); }
        fence_barrier_init();
    }
    if (threadIdx.x == 32) {
        prefetch_map(&P.p[0].a[0]);
        prefetch_map(&P.p[0].b[EPI == kEpiGated ? rank : 0]);
    }
    if (warp == 2) ffn_tmem_alloc<CG>(slot, kTmemCols);
    tc_fence_before();
    __syncthreads();
    if constexpr (CG == 2) { cluster_arrive_release(); cluster_wait_acquire(); }
    tc_fence_after();
    uint32_t tmem;
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(tmem) : "r"(slot));
    // early: the kernel before this one is ours, and let this one start only when everything before it had finished.  The two
    // share no memory that either writes, so they may run side by side; this one still ends after that one.
    if (!P.early) wait_for_previous_kernel();
    let_next_kernel_start();

    const long long tiles = P.tiles;
    auto place = [&](long long t, int& which, int& m0, int& n0) {
        which = 0;
        while (which + 1 < P.problems && P.p[which + 1].first_tile <= t) ++which;
        const FfnProblem& q = P.p[which];
        const unsigned r = (unsigned)(t - q.first_tile), per = (unsigned)(kFfnGroup * q.tiles_n), g = r / per;
        const unsigned first = g * kFfnGroup, gm = min((unsigned)kFfnGroup, (unsigned)q.tiles_m - first), r2 = r - g * per;
        m0 = (int)(first + r2 % gm) * (128 * CG);
        n0 = (int)(r2 / gm) * kCols;
    };
    FfnWait w{P.gave_up, P.timeout_ns, false};

    if (warp == 0) {
        if (lane == 0) {
            int s = 0;
            uint32_t phase = 0;
            unsigned left = P.fills;
            for (long long t = pair; t < tiles && !w.aborted && left != 0; t += pairs) {
                int which, m0, n0;
                place(t, which, m0, n0);
                const FfnProblem& q = P.p[which];
                const int am = m0 + (int)rank * 128, K = q.K, segments = q.segments;
                for (int seg = 0; seg < segments && !w.aborted && left != 0; ++seg) {
                    const CUtensorMap* const map_a = &q.a[seg];
                    const CUtensorMap* const map_b = EPI == kEpiGated ? &q.b[rank] : &q.b[seg];
                    for (int k0 = 0; k0 < K && left != 0; k0 += kFfnBK, --left) {
                        ffn_wait(empty + 8 * s, phase ^ 1u, w);
                        if (w.aborted) break;
                        uint32_t bar = full + 8 * s;
                        if (rank == 0) mbar_arrive_expect_tx(bar, S::kStage * CG);
                        if constexpr (CG == 2) bar = leader_addr(bar);
                        const uint32_t sa = ring + s * S::kStage, sb = sa + S::kA;
                        ffn_fetch<CG>(sa, map_a, A_MN, 128, am, k0, bar);
                        if constexpr (EPI == kEpiGated) {
                            // the first half of the tile's columns is G, the second U; with two CTAs one fetches each
                            if constexpr (CG == 2) ffn_fetch<CG>(sb, map_b, B_MN, BN / 2, n0, k0, bar);
                            else {
                                ffn_fetch<CG>(sb, map_b, B_MN, BN / 2, n0, k0, bar);
                                ffn_fetch<CG>(sb + S::kB / 2, map_b + 1, B_MN, BN / 2, n0, k0, bar);
                            }
                        } else {
                            ffn_fetch<CG>(sb, map_b, B_MN, BN / CG, n0 + (int)rank * (BN / CG), k0, bar);
                        }
                        if (++s == S::kStages) { s = 0; phase ^= 1u; }
                    }
                }
            }
            if (rank == 0) ffn_drain(full, S::kStages, s, phase, w);  // (copies of both CTAs: the other one waits for this one below)
        }
    } else if (warp == 1) {
        if (lane == 0 && rank == 0) {
            const uint32_t idesc = ffn_idesc(P.type, A_MN, B_MN, 128 * CG, BN);
            const FfnDesc ad(A_MN), bd(B_MN);
            int s = 0, acc = 0;
            uint32_t phase = 0, acc_phase = 0;
            for (long long t = pair; t < tiles && !w.aborted; t += pairs) {
                int which, m0, n0;
                place(t, which, m0, n0);
                const FfnProblem& q = P.p[which];
                const int steps = q.segments * ((q.K + kFfnBK - 1) / kFfnBK);
                ffn_wait(acc_empty + 8 * acc, acc_phase ^ 1u, w);
                tc_fence_after();
                for (int k = 0; k < steps && !w.aborted; ++k) {
                    ffn_wait(full + 8 * s, phase, w);
                    if (w.aborted) break;
                    tc_fence_after();
                    uint64_t da = ad.at(ring + s * S::kStage), db = bd.at(ring + s * S::kStage + S::kA);
#pragma unroll
                    for (int i = 0; i < kFfnBK / 16; ++i, da += ad.step, db += bd.step)
                        ffn_mma<CG>(tmem + (uint32_t)(acc * BN), da, db, idesc, (k | i) != 0 ? 1u : 0u);
                    ffn_commit<CG>(empty + 8 * s);
                    if (++s == S::kStages) { s = 0; phase ^= 1u; }
                }
                if (w.aborted) break;
                ffn_commit<CG>(acc_full + 8 * acc);
                if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
            }
            ffn_drain(empty, S::kStages, s, phase, w);
        }
    } else if (warp >= 4) {
        // A lane reads a row out of tensor memory; what a warp writes to (or reads from) global memory at a time should be
        // pieces of rows: in between the values go through shared memory.
        int acc = 0;
        uint32_t acc_phase = 0;
        const int quarter = warp & 3, part = (warp - 4) >> 2;  // two warps share a quarter of the rows: one takes the even pieces
        float* const turn = reinterpret_cast<float*>(ffn_smem + (ring - smem_u32(ffn_smem)) + S::kTurn) + (warp - 4) * R::kRows * R::kWords;
        for (long long t = pair; t < tiles; t += pairs) {
            int which, m0, n0;
            place(t, which, m0, n0);
            const FfnProblem& q = P.p[which];
            const int N = q.N;
            const long long ld_out = q.ld_out;
            uint16_t* const out = static_cast<uint16_t*>(q.out);
            ffn_wait(acc_full + 8 * acc, acc_phase, w);
            w.aborted = __any_sync(0xFFFFFFFFu, w.aborted);
            const long long row0 = (long long)m0 + rank * 128 + quarter * 32;
            const int rows = (int)min(32ll, q.M - row0);  // (may be negative)
            if (w.aborted) {  // this warp's part of this tile, and of those that follow, has not been computed: NaN
                for (int c = part * R::kCols; c < kCols; c += 2 * R::kCols)
#pragma unroll 1
                    for (int k = lane; k < rows * R::kCols; k += 32) {
                        const int col = n0 + c + k % R::kCols;
                        const long long row = row0 + k / R::kCols;
                        if (col >= N) continue;
                        out[row * ld_out + col] = 0x7FFFu;  // (in either 16-bit type)
                        if constexpr (EPI == kEpiBackward) static_cast<uint16_t*>(P.out_up)[row * ld_out + col] = 0x7FFFu;
                        if (EPI == kEpiGated && P.value) P.value[row * P.ld_save + col] = P.slope[row * P.ld_save + col] = __uint_as_float(0x7FC00000u);
                    }
                continue;
            }
            tc_fence_after();
            const uint32_t ta = tmem + (uint32_t)(acc * BN) + ((uint32_t)(quarter * 32) << 16);
            if constexpr (EPI == kEpiGated) {
                // 16 columns of G and 16 of U at a time; then a lane has four columns of rows lane / 4, lane / 4 + 8, ...
                const int sub = (lane & 3) * 4;
#pragma unroll 1
                for (int c = part * R::kCols; c < kCols; c += 2 * R::kCols) {
                    const int col = n0 + c;
                    if (col >= N) break;
                    uint32_t r[32];
                    tmem_load16(ta + (uint32_t)c, r);
                    tmem_load16(ta + (uint32_t)(BN / 2 + c), r + 16);
                    tmem_wait();
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        *reinterpret_cast<uint4*>(turn + turn32(lane, i)) = make_uint4(r[4 * i], r[4 * i + 1], r[4 * i + 2], r[4 * i + 3]);
                    __syncwarp();
#pragma unroll
                    for (int it = 0; it < 4; ++it) {
                        const int i = it * 8 + (lane >> 2);
                        if (i < rows && col + sub < N) {  // (rows of H, act(G) and U act'(G) are padded to multiples of 8)
                            const float4 g = *reinterpret_cast<const float4*>(turn + turn32(i, lane & 3));
                            const float4 u = *reinterpret_cast<const float4*>(turn + turn32(i, 4 + (lane & 3)));
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
                            *reinterpret_cast<uint2*>(out + (row0 + i) * ld_out + col + sub) =
                                make_uint2(pack2(P.type, v.x * u.x, v.y * u.y), pack2(P.type, v.z * u.z, v.w * u.w));
                        }
                    }
                    __syncwarp();
                }
            } else if constexpr (EPI == kEpiBackward) {
                // 32 columns of the factors at a time, a lane four columns of rows lane / 8, lane / 8 + 4, ...: pieces of 128 bytes
                // (4096 x 5632 values from 2048 outputs: 92 us, with pieces of 64 bytes 112); the sums come through shared memory 16
                // rows at a time.
                const int sub = (lane & 7) * 4;
#pragma unroll 1
                for (int c = part * R::kCols; c < kCols; c += 2 * R::kCols) {
                    const int col = n0 + c;
                    if (col >= N) break;
                    float4 v[8], s[8];
#pragma unroll
                    for (int it = 0; it < 8; ++it) {
                        const int i = it * 4 + (lane >> 3);
                        const long long at = (row0 + i) * P.ld_save + col + sub;
                        if (i < rows && col + sub < N) {
                            v[it] = __ldcs(reinterpret_cast<const float4*>(P.value + at));
                            s[it] = __ldcs(reinterpret_cast<const float4*>(P.slope + at));
                        }
                    }
                    uint32_t r[32];
                    tmem_load32(ta + (uint32_t)c, r);
                    tmem_wait();
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        if ((lane >> 4) == half) {
#pragma unroll
                            for (int i = 0; i < 8; ++i)
                                *reinterpret_cast<uint4*>(turn + turn32(lane & 15, i)) = make_uint4(r[4 * i], r[4 * i + 1], r[4 * i + 2], r[4 * i + 3]);
                        }
                        __syncwarp();
#pragma unroll
                        for (int it = 4 * half; it < 4 * half + 4; ++it) {
                            const int i = it * 4 + (lane >> 3);
                            if (i < rows && col + sub < N) {
                                const float4 d = *reinterpret_cast<const float4*>(turn + turn32(i & 15, lane & 7));
                                const long long at = (row0 + i) * ld_out + col + sub;
                                *reinterpret_cast<uint2*>(out + at) =
                                    make_uint2(pack2(P.type, d.x * s[it].x, d.y * s[it].y), pack2(P.type, d.z * s[it].z, d.w * s[it].w));
                                *reinterpret_cast<uint2*>(static_cast<uint16_t*>(P.out_up) + at) =
                                    make_uint2(pack2(P.type, d.x * v[it].x, d.y * v[it].y), pack2(P.type, d.z * v[it].z, d.w * v[it].w));
                            }
                        }
                        __syncwarp();
                    }
                }
            } else {
                // 64 columns at a time: rows of 128 bytes
                const uint16_t* const half = reinterpret_cast<const uint16_t*>(turn);
                const bool vec = q.vec != 0;
#pragma unroll 1
                for (int c = part * R::kCols; c < kCols; c += 2 * R::kCols) {
                    const int col = n0 + c;
                    if (col >= N) break;
                    uint32_t r[64];
                    tmem_load32(ta + (uint32_t)c, r);
                    tmem_load32(ta + (uint32_t)(c + 32), r + 32);
                    tmem_wait();
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        uint32_t p[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) p[j] = pack2(P.type, __uint_as_float(r[8 * i + 2 * j]), __uint_as_float(r[8 * i + 2 * j + 1]));
                        *reinterpret_cast<uint4*>(turn + turn32(lane, i)) = make_uint4(p[0], p[1], p[2], p[3]);
                    }
                    __syncwarp();
                    if (vec && col + 64 <= N) {
#pragma unroll
                        for (int it = 0; it < 8; ++it) {
                            const int i = it * 4 + (lane >> 3);
                            if (i < rows)
                                *reinterpret_cast<uint4*>(out + (row0 + i) * ld_out + col + (lane & 7) * 8) = *reinterpret_cast<const uint4*>(turn + turn32(i, lane & 7));
                        }
                    } else {
#pragma unroll
                        for (int h = 0; h < 64; h += 32) {
                            if (col + h + lane < N) {
#pragma unroll 8
                                for (int i = 0; i < rows; ++i) out[(row0 + i) * ld_out + col + h + lane] = half[2 * turn32(i, (h + lane) >> 3) + (lane & 7)];
                            }
                        }
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
    if (__any_sync(0xFFFFFFFFu, w.aborted)) ffn_linger();
    tc_fence_before();
    __syncthreads();
    if constexpr (CG == 2) { cluster_arrive_release(); cluster_wait_acquire(); }
    tc_fence_after();
    if (warp == 2) ffn_tmem_free<CG>(tmem, kTmemCols);
    if (P.early) wait_for_previous_kernel();
}

// ---------------------------------------------------------------- few rows, and everything small
// The same contractions where the tiles of the form above would leave SMs without work, with the roles exchanged: 128
// features (columns of the weights) are the rows of a tile, and NR rows of X its columns, so that the tensor core wastes nothing
// on missing rows and a stage of the ring is nearly all weights.  The contraction is split over the S CTAs of a cluster, as many
// as give each SM something to read; their partial sums are added through distributed shared memory in the order of
// the CTAs.  What bounds it: reading the weights (4 MB and more), or the latency of one pass through copy, product and sum.
constexpr int kFewThreads = 256;
constexpr int kFewPart = 128;  // features of a tile

template <int NR, int EPI>
struct FewShape {
    static constexpr int kTiles = EPI == kEpiGated ? 2 : 1;       // tiles of weights per stage: Wg and Wu
    static constexpr int kA = 128 * kFfnBK * 2;
    static constexpr int kStage = kTiles * kA + NR * kFfnBK * 2;
    static constexpr int kCtasPerSm = 2;                          // one's arithmetic and read-out overlap the other's copies
    static constexpr int kStages = 110 * 1024 / kStage > 10 ? 10 : 110 * 1024 / kStage;
    static constexpr int kRing = kStages * kStage;
    static constexpr int kPassRows = NR < 64 ? NR : 64;            // rows whose partial sums are exchanged at a time
    static constexpr int kParts = kTiles * kPassRows * kFewPart * 4;  // they take the ring's place once it is done with
    static_assert(kParts <= kRing, "partial sums");
    static constexpr int kBars = kRing;
    static constexpr int kSmem = kBars + 256 + 1024;
    static constexpr uint32_t kTmemCols = kTiles * NR < 32 ? 32 : kTiles * NR;
};

__device__ __forceinline__ void store4_any(uint16_t* p, int type, bool vec, int left, float4 v) {
    const uint32_t lo = pack2(type, v.x, v.y), hi = pack2(type, v.z, v.w);
    if (vec && left >= 4) { *reinterpret_cast<uint2*>(p) = make_uint2(lo, hi); return; }
    if (left > 0) p[0] = (uint16_t)lo;
    if (left > 1) p[1] = (uint16_t)(lo >> 16);
    if (left > 2) p[2] = (uint16_t)hi;
    if (left > 3) p[3] = (uint16_t)(hi >> 16);
}

// A CTA's share of `some` rows whose partial sums stand in the shared memory of S <= SP CTAs: a warp takes rows S * 8 apart, four
// features per lane, and as many rows at once as make eight loads: each takes the time of a trip to another SM.
template <int SP, int PASS_ROWS, int EPI>
__device__ __forceinline__ void few_finish(const FfnParams& P, const FfnProblem& q, uint32_t sums, int S, int part, int warp, int lane,
                                           int f, int first_row, int some) {
    constexpr int kRows = EPI == kEpiGated ? (SP < 4 ? 4 / SP : 1) : 8 / SP;
    const int left = q.N - f, step = S * (kFewThreads / 32);
    uint16_t* const out = static_cast<uint16_t*>(q.out);
    for (int i0 = part * (kFewThreads / 32) + warp; i0 < some; i0 += step * kRows) {
        float4 y[kRows][SP], z[kRows][SP];
#pragma unroll
        for (int b = 0; b < kRows; ++b) {
            const uint32_t at = sums + (uint32_t)(((i0 + b * step) * kFewPart + lane * 4) * 4);
            if (b > 0 && i0 + b * step >= some) continue;
#pragma unroll
            for (int c = 0; c < SP; ++c) {
                if (c >= S) continue;
                y[b][c] = ld_cluster4(at, c);
                if constexpr (EPI == kEpiGated) z[b][c] = ld_cluster4(at + PASS_ROWS * kFewPart * 4, c);
            }
        }
        if (left <= 0) continue;
#pragma unroll
        for (int b = 0; b < kRows; ++b) {
            if (b > 0 && i0 + b * step >= some) continue;
            float4 x = y[b][0], u = z[b][0];
#pragma unroll
            for (int c = 1; c < SP; ++c) {
                if (c >= S) continue;
                x.x += y[b][c].x; x.y += y[b][c].y; x.z += y[b][c].z; x.w += y[b][c].w;
                if constexpr (EPI == kEpiGated) { u.x += z[b][c].x; u.y += z[b][c].y; u.z += z[b][c].z; u.w += z[b][c].w; }
            }
            const long long row = first_row + i0 + b * step;
            if constexpr (EPI == kEpiGated) {
                float4 v, s;
                act_both(P.act, x.x, v.x, s.x); act_both(P.act, x.y, v.y, s.y);
                act_both(P.act, x.z, v.z, s.z); act_both(P.act, x.w, v.w, s.w);
                if (P.value) {
                    *reinterpret_cast<float4*>(P.value + row * P.ld_save + f) = v;
                    *reinterpret_cast<float4*>(P.slope + row * P.ld_save + f) = make_float4(u.x * s.x, u.y * s.y, u.z * s.z, u.w * s.w);
                }
                store4_any(out + row * q.ld_out + f, P.type, true, 4, make_float4(v.x * u.x, v.y * u.y, v.z * u.z, v.w * u.w));
            } else if constexpr (EPI == kEpiBackward) {
                const float4 v = *reinterpret_cast<const float4*>(P.value + row * P.ld_save + f);
                const float4 s = *reinterpret_cast<const float4*>(P.slope + row * P.ld_save + f);
                store4_any(out + row * q.ld_out + f, P.type, true, 4, make_float4(x.x * s.x, x.y * s.y, x.z * s.z, x.w * s.w));
                store4_any(static_cast<uint16_t*>(P.out_up) + row * q.ld_out + f, P.type, true, 4, make_float4(x.x * v.x, x.y * v.y, x.z * v.z, x.w * v.w));
            } else {
                store4_any(out + row * q.ld_out + f, P.type, q.vec, left, x);
            }
        }
    }
}

// Grid: S CTAs (one cluster) per tile.  a: the weights, b: the rows; tiles_m and tiles_n count tiles of NR rows and of 128
// features.  early: the kernel before this one is ours and started after everything before it had finished, so the
// weights, which it does not write, may be fetched while it still runs.
template <int NR, int EPI>
__global__ void __launch_bounds__(kFewThreads, FewShape<NR, EPI>::kCtasPerSm) ffn_few_kernel(const __grid_constant__ FfnParams P, const int S, const int early) {
    using F = FewShape<NR, EPI>;
    extern __shared__ unsigned char ffn_smem[];
    const uint32_t ring = (smem_u32(ffn_smem) + 1023u) & ~1023u;
    const uint32_t full = ring + F::kBars, empty = full + 8 * F::kStages, done = empty + 8 * F::kStages, slot = done + 8;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const FfnProblem& q = P.p[0];
    const int part = (int)blockIdx.x % S, tile = (int)blockIdx.x / S;
    const int f0 = tile / q.tiles_m * kFewPart, r0 = tile % q.tiles_m * NR;

    if (threadIdx.x == 0) {
        for (int s = 0; s < F::kStages; ++s) { mbar_init(full + 8 * s, 1); mbar_init(empty + 8 * s, 1); }
        mbar_init(done, 1);
        fence_barrier_init();
    }
    if (threadIdx.x == 32) {
        prefetch_map(&q.a[0]);
        prefetch_map(&q.b[0]);
        if (EPI == kEpiGated || q.segments > 1) prefetch_map(&q.a[1]);
    }
    if (warp == 2) ffn_tmem_alloc<1>(slot, F::kTmemCols);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    uint32_t tmem;
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(tmem) : "r"(slot));
    // (all but the warp that fetches: the bounded waits below must not count the time of the kernel before)
    if (!early || warp != 0) wait_for_previous_kernel();

    const int kblocks = (q.K + kFfnBK - 1) / kFfnBK, steps = kblocks * q.segments;
    const int first = (int)((long long)steps * part / S), last = (int)((long long)steps * (part + 1) / S);
    FfnWait w{P.gave_up, P.timeout_ns, false};
    if (warp == 0) {
        if (lane == 0) {
            const bool a_mn = q.a_mn;
            const int fill_to = (int)min((long long)last, (long long)first + P.fills);
            auto weights = [&](int k, int s) {
                const int seg = k >= kblocks ? 1 : 0, k0 = (k - seg * kblocks) * kFfnBK;
                const uint32_t bar = full + 8 * s, sa = ring + s * F::kStage;
                mbar_arrive_expect_tx(bar, F::kStage);
                ffn_fetch<1>(sa, &q.a[seg], a_mn, 128, f0, k0, bar);
                if constexpr (EPI == kEpiGated) ffn_fetch<1>(sa + F::kA, &q.a[1], a_mn, 128, f0, k0, bar);
            };
            auto rows = [&](int k, int s) {
                const int seg = k >= kblocks ? 1 : 0, k0 = (k - seg * kblocks) * kFfnBK;
                ffn_fetch<1>(ring + s * F::kStage + F::kTiles * F::kA, &q.b[seg], false, NR, r0, k0, full + 8 * s);
            };
            int ahead = 0;
            if (early) {
                for (; ahead < F::kStages && first + ahead < fill_to; ++ahead) weights(first + ahead, ahead);
                wait_for_previous_kernel();
            }
            int s = 0;
            uint32_t phase = 0;
            for (int k = first; k < fill_to; ++k) {
                if (k - first >= ahead) {
                    ffn_wait(empty + 8 * s, phase ^ 1u, w);
                    if (w.aborted) break;
                    weights(k, s);
                }
                rows(k, s);
                if (++s == F::kStages) { s = 0; phase ^= 1u; }
            }
            ffn_drain(full, F::kStages, s, phase, w);
        }
    } else if (warp == 1) {
        if (lane == 0) {
            const uint32_t idesc = ffn_idesc(P.type, q.a_mn, false, 128, NR);
            const FfnDesc ad(q.a_mn), bd(false);
            int s = 0;
            uint32_t phase = 0;
            for (int k = first; k < last; ++k) {
                ffn_wait(full + 8 * s, phase, w);
                if (w.aborted) break;
                tc_fence_after();
                uint64_t da = ad.at(ring + s * F::kStage), db = bd.at(ring + s * F::kStage + F::kTiles * F::kA);
#pragma unroll
                for (int i = 0; i < kFfnBK / 16; ++i, da += ad.step, db += bd.step) {
#pragma unroll
                    for (int h = 0; h < F::kTiles; ++h)
                        ffn_mma<1>(tmem + (uint32_t)(h * NR), da + (uint64_t)(h * (F::kA >> 4)), db, idesc, (k != first || i != 0) ? 1u : 0u);
                }
                ffn_commit<1>(empty + 8 * s);
                if (++s == F::kStages) { s = 0; phase ^= 1u; }
            }
            if (!w.aborted) ffn_commit<1>(done);  // (waited for below)
            else ffn_drain(empty, F::kStages, s, phase, w);
        }
    }
    __syncwarp();
    if (early && warp == 0) wait_for_previous_kernel();
    // after the last product the ring's memory is free for the partial sums [row][128 features]
    ffn_wait(done, 0, w);
    tc_fence_after();
    let_next_kernel_start();
    const bool given_up = __syncthreads_or(w.aborted ? 1 : 0) != 0;

    const int f = f0 + lane * 4;
    const int rows = min(NR, q.M - r0);
    const uint32_t ta = tmem + ((uint32_t)((warp & 3) * 32) << 16);
#pragma unroll 1
    for (int base = 0; base < rows; base += F::kPassRows) {
        if (base > 0) {  // the sums of the pass before have been read
            __syncthreads();
            if (S > 1) { cluster_arrive_release(); cluster_wait_acquire(); }
        }
        // two warps share a quarter of the features: they take turns at 16 rows
        const uint32_t to = ring + (uint32_t)(((warp & 3) * 32 + lane) * 4);
#pragma unroll 1
        for (int c = (warp >> 2) * 16; c < F::kTiles * F::kPassRows; c += 32) {
            const int h = c / F::kPassRows, col = c - h * F::kPassRows;
            if (base + col >= rows) continue;
            uint32_t r[16];
            tmem_load16(ta + (uint32_t)(h * NR + base + col), r);
            tmem_wait();
            if (given_up) fill_nan(r);  // (every CTA of the cluster adds them, so all of the tile's outputs are NaN)
#pragma unroll
            for (int i = 0; i < 16; ++i) asm volatile("st.shared.b32 [%0], %1;" ::"r"(to + (uint32_t)((c + i) * kFewPart * 4)), "r"(r[i]) : "memory");
        }
        tc_fence_before();
        __syncthreads();
        if (S > 1) { cluster_arrive_release(); cluster_wait_acquire(); }
        // each CTA finishes its share of the rows
        const int some = min(F::kPassRows, rows - base);
        if (S == 1) few_finish<1, F::kPassRows, EPI>(P, q, ring, S, part, warp, lane, f, r0 + base, some);
        else if (S == 2) few_finish<2, F::kPassRows, EPI>(P, q, ring, S, part, warp, lane, f, r0 + base, some);
        else if (S <= 4) few_finish<4, F::kPassRows, EPI>(P, q, ring, S, part, warp, lane, f, r0 + base, some);
        else few_finish<8, F::kPassRows, EPI>(P, q, ring, S, part, warp, lane, f, r0 + base, some);
    }
    if (given_up) ffn_linger();
    __syncthreads();
    if (S > 1) { cluster_arrive_release(); cluster_wait_acquire(); }  // peers have read this CTA's sums
    tc_fence_after();
    if (warp == 2) ffn_tmem_free<1>(tmem, F::kTmemCols);
}

// ---------------------------------------------------------------- operands that TMA cannot read
// Rows of `cols` 16-bit values from stride ld to stride ld_out (a multiple of 8, at least cols), the rest of each row zero.
struct AlignJob {
    const uint16_t* in;
    uint16_t* out;
    long long ld, rows;
    int ld_out, cols;
};
struct AlignParams {
    AlignJob job[5];
};
__global__ void __launch_bounds__(256) ffn_align_kernel(const __grid_constant__ AlignParams P) {
    wait_for_previous_kernel();
    let_next_kernel_start();
    const AlignJob& j = P.job[blockIdx.y];
    const unsigned per = (unsigned)j.ld_out / 8;
    const long long total = j.rows * per;
    for (long long i = blockIdx.x * 256ll + threadIdx.x; i < total; i += gridDim.x * 256ll) {
        const long long r = i / per;
        const int c = (int)(i - r * per) * 8;
        const uint16_t* in = j.in + r * j.ld + c;
        uint32_t v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t lo = c + 2 * k < j.cols ? in[2 * k] : 0u, hi = c + 2 * k + 1 < j.cols ? in[2 * k + 1] : 0u;
            v[k] = lo | (hi << 16);
        }
        *reinterpret_cast<uint4*>(j.out + r * j.ld_out + c) = make_uint4(v[0], v[1], v[2], v[3]);
    }
}

}  // namespace bmgdk
