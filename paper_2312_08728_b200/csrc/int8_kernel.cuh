// Product in 8-bit integers with a scale for each token and each channel (bmgd_quantized_linear).
//
//     y_ij = (sum_k q_ik w_jk) qs_i ws_j + bias_j       q [rows][inputs], w [outputs][inputs], sums in 32-bit integers (exact)
//
// Both operands stand along the contraction ("K-major"): the weights are laid out once, by channels.  What bounds it: the tensor cores
// from a few hundred tokens on (int8_kernel), reading the weights once below (int8_few_kernel).  The ring of stages is in bytes that
// of the 16-bit contractions, 128 along the contraction and 128 or 256 rows, but a stage is 128 values deep.
#pragma once
#include <cstdint>
#include <cuda.h>
#include <cuda_runtime.h>

#include "contract.cuh"

namespace bmgdk {

constexpr int kInt8BK = 128;
constexpr int kInt8Group = 8;   // tiles along the tokens that are worked on together: their rows stay in L2 while the weights pass
constexpr int kInt8None = (int)0x80000000u;  // no sum of up to 131,071 products of 8 bits: stands for one that was not computed

struct Int8Params {
    CUtensorMap q, w;
    const signed char *q_rows, *w_rows;     // the same memory, for rows on any boundary (int8_few_kernel)
    long long ld_q, ld_w;
    const float *q_scale, *w_scale, *bias;  // bias: null for none
    void* out;
    long long ld_out, tiles;
    int M, N, K;
    int tiles_m, tiles_n;
    int type, vec;              // vec: rows of the output start on 16-byte boundaries
    unsigned fills;             // as FfnParams
    unsigned* gave_up;
    unsigned long long timeout_ns;
};

template <int CG>
__device__ __forceinline__ void int8_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    if constexpr (CG == 1)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
// signed 8-bit operands, 32-bit integer sums
__device__ __forceinline__ uint32_t int8_idesc(int m, int n) {
    return (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
__device__ __forceinline__ float int8_nan() { return __uint_as_float(0x7FC00000u); }
__device__ __forceinline__ void int8_store1(void* out, int type, long long at, float v) {
    if (type == BMGD_TYPE_F32) static_cast<float*>(out)[at] = v;
    else static_cast<uint16_t*>(out)[at] = (uint16_t)pack2(type, v, 0.f);
}

// ---------------------------------------------------------------- many tokens
// As ffn_kernel: warp 0 copies tiles into the ring, warp 1 issues the products, warps 4 to 11 read accumulators out, which take
// turns.  CG = 2: pairs of CTAs, 256 tokens by 192 or 256 channels (128 channels took as long a tile as 256).  The tokens are the tile's rows; a channel's scale and bias come from shared memory,
// where the read-out warps put those of the next tile before they wait for its products.
constexpr int kInt8Threads = 128 + 8 * 32;
template <int CG, int BN>
struct Int8Shape {
    static constexpr int kA = 128 * kInt8BK;
    static constexpr int kB = BN / CG * kInt8BK;
    static constexpr int kStage = kA + kB;
    static constexpr int kStages = kStage <= 28672 ? 6 : 5;
    static constexpr int kBars = kStages * kStage;
    static constexpr int kScale = kBars + 256;                   // [2][2][BN] fp32: scale and bias of a tile's channels
    static constexpr int kTurn = kScale + 2 * 2 * BN * 4;
    static constexpr int kSmem = kTurn + 8 * 32 * 32 * 4 + 1024;
};

template <int CG, int BN>
__global__ void __launch_bounds__(kInt8Threads, 1) int8_kernel(const __grid_constant__ Int8Params P) {
    using S = Int8Shape<CG, BN>;
    extern __shared__ unsigned char int8_smem[];
    const uint32_t ring = (smem_u32(int8_smem) + 1023u) & ~1023u;
    unsigned char* const base = int8_smem + (ring - smem_u32(int8_smem));
    const uint32_t full = ring + S::kBars, empty = full + 8 * S::kStages, acc_full = empty + 8 * S::kStages, acc_empty = acc_full + 16;
    const uint32_t slot = acc_empty + 16;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = CG == 2 ? cluster_ctarank() : 0u;
    const int pair = (int)blockIdx.x / CG, pairs = (int)gridDim.x / CG;
    constexpr uint32_t kTmemCols = BN <= 128 ? 256 : 512;  // (two accumulators, in a power of two)

    if (threadIdx.x == 0) {
        for (int s = 0; s < S::kStages; ++s) { mbar_init(full + 8 * s, 1); mbar_init(empty + 8 * s, 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(acc_full + 8 * i, 1); mbar_init(acc_empty + 8 * i, 8 * CG); }
        fence_barrier_init();
    }
    if (threadIdx.x == 32) {
        prefetch_map(&P.q);
        prefetch_map(&P.w);
    }
    if (warp == 2) ffn_tmem_alloc<CG>(slot, kTmemCols);
    tc_fence_before();
    __syncthreads();
    if constexpr (CG == 2) { cluster_arrive_release(); cluster_wait_acquire(); }
    tc_fence_after();
    uint32_t tmem;
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(tmem) : "r"(slot));
    wait_for_previous_kernel();
    let_next_kernel_start();

    const long long tiles = P.tiles;
    auto place = [&](long long t, int& m0, int& n0) {
        const unsigned r = (unsigned)t, per = (unsigned)(kInt8Group * P.tiles_n), g = r / per;
        const unsigned first = g * kInt8Group, gm = min((unsigned)kInt8Group, (unsigned)P.tiles_m - first), r2 = r - g * per;
        m0 = (int)(first + r2 % gm) * (128 * CG);
        n0 = (int)(r2 / gm) * BN;
    };
    FfnWait w{P.gave_up, P.timeout_ns, false};

    if (warp == 0) {
        if (lane == 0) {
            int s = 0;
            uint32_t phase = 0;
            unsigned left = P.fills;
            for (long long t = pair; t < tiles && !w.aborted && left != 0; t += pairs) {
                int m0, n0;
                place(t, m0, n0);
                const int am = m0 + (int)rank * 128, bn = n0 + (int)rank * (BN / CG);
                for (int k0 = 0; k0 < P.K && left != 0; k0 += kInt8BK, --left) {
                    ffn_wait(empty + 8 * s, phase ^ 1u, w);
                    if (w.aborted) break;
                    uint32_t bar = full + 8 * s;
                    if (rank == 0) mbar_arrive_expect_tx(bar, S::kStage * CG);
                    if constexpr (CG == 2) bar = leader_addr(bar);
                    const uint32_t sa = ring + s * S::kStage, sb = sa + S::kA;
                    ffn_tma<CG>(sa, &P.q, k0, am, bar);
                    ffn_tma<CG>(sb, &P.w, k0, bn, bar);
                    if (++s == S::kStages) { s = 0; phase ^= 1u; }
                }
            }
            if (rank == 0) ffn_drain(full, S::kStages, s, phase, w);  // (copies of both CTAs: the other one waits for this one below)
        }
    } else if (warp == 1) {
        if (lane == 0 && rank == 0) {
            const uint32_t idesc = int8_idesc(128 * CG, BN);
            const uint64_t desc = tc_smem_desc(0, 16, 1024);
            int s = 0, acc = 0;
            uint32_t phase = 0, acc_phase = 0;
            const int steps = (P.K + kInt8BK - 1) / kInt8BK;
            for (long long t = pair; t < tiles && !w.aborted; t += pairs) {
                ffn_wait(acc_empty + 8 * acc, acc_phase ^ 1u, w);
                tc_fence_after();
                for (int k = 0; k < steps && !w.aborted; ++k) {
                    ffn_wait(full + 8 * s, phase, w);
                    if (w.aborted) break;
                    tc_fence_after();
                    const uint32_t at = ring + s * S::kStage;
                    uint64_t da = desc + ((at >> 4) & 0x3FFFu), db = desc + (((at + S::kA) >> 4) & 0x3FFFu);
#pragma unroll
                    for (int i = 0; i < kInt8BK / 32; ++i, da += 2, db += 2)
                        int8_mma<CG>(tmem + (uint32_t)(acc * BN), da, db, idesc, (k | i) != 0 ? 1u : 0u);
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
        int acc = 0;
        uint32_t acc_phase = 0;
        const int quarter = warp & 3, part = (warp - 4) >> 2;  // two warps share a quarter of the rows: one takes the even pieces
        float* const scales = reinterpret_cast<float*>(base + S::kScale);
        float* const turn = reinterpret_cast<float*>(base + S::kTurn) + (warp - 4) * 32 * 32;
        for (long long t = pair; t < tiles; t += pairs) {
            int m0, n0;
            place(t, m0, n0);
            // (the buffer of the tile before last: the barrier behind it says that all warps are done with it)
            float* const ws = scales + acc * 2 * BN;
            const int own = (int)threadIdx.x - 128;
            if (own < BN) {
                const int col = n0 + own;
                ws[own] = col < P.N ? __ldca(P.w_scale + col) : 0.f;
                ws[BN + own] = P.bias && col < P.N ? __ldca(P.bias + col) : 0.f;
            }
            asm volatile("bar.sync 1, 256;" ::: "memory");
            const long long row0 = (long long)m0 + rank * 128 + quarter * 32;
            const int rows = (int)max(0ll, min(32ll, P.M - row0));
            const float qs = lane < rows ? __ldca(P.q_scale + row0 + lane) : 0.f;
            ffn_wait(acc_full + 8 * acc, acc_phase, w);
            w.aborted = __any_sync(0xFFFFFFFFu, w.aborted);
            if (w.aborted) {  // this warp's part of this tile, and of those that follow, has not been computed: NaN
                for (int c = part * 64; c < BN; c += 128)
#pragma unroll 1
                    for (int k = lane; k < rows * 64; k += 32) {
                        const int col = n0 + c + k % 64;
                        if (col < P.N) int8_store1(P.out, P.type, (row0 + k / 64) * P.ld_out + col, int8_nan());
                    }
                if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
                continue;
            }
            tc_fence_after();
            const uint32_t ta = tmem + (uint32_t)(acc * BN) + ((uint32_t)(quarter * 32) << 16);
            // a lane reads 32 columns of its row at a time; through shared memory they become pieces of rows
            auto scaled = [&](const uint32_t (&r)[32], int c, float (&v)[32]) {
#pragma unroll
                for (int i = 0; i < 32; i += 4) {
                    const float4 f = *reinterpret_cast<const float4*>(ws + c + i), b = *reinterpret_cast<const float4*>(ws + BN + c + i);
                    v[i] = (float)(int)r[i] * qs * f.x + b.x;
                    v[i + 1] = (float)(int)r[i + 1] * qs * f.y + b.y;
                    v[i + 2] = (float)(int)r[i + 2] * qs * f.z + b.z;
                    v[i + 3] = (float)(int)r[i + 3] * qs * f.w + b.w;
                }
            };
#pragma unroll 1
            for (int c = part * 64; c < BN; c += 128) {
                const int col = n0 + c;
                if (col >= P.N) break;
                if (P.type == BMGD_TYPE_F32) {
                    float* const out = static_cast<float*>(P.out);
#pragma unroll 1
                    for (int h = 0; h < 64; h += 32) {
                        uint32_t r[32];
                        float v[32];
                        tmem_load32(ta + (uint32_t)(c + h), r);
                        tmem_wait();
                        scaled(r, c + h, v);
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            *reinterpret_cast<float4*>(turn + turn32(lane, i)) = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
                        __syncwarp();
                        if (P.vec && col + h + 32 <= P.N) {
#pragma unroll
                            for (int it = 0; it < 8; ++it) {
                                const int i = it * 4 + (lane >> 3);
                                if (i < rows)
                                    *reinterpret_cast<float4*>(out + (row0 + i) * P.ld_out + col + h + (lane & 7) * 4) = *reinterpret_cast<const float4*>(turn + turn32(i, lane & 7));
                            }
                        } else if (col + h + lane < P.N) {
#pragma unroll 8
                            for (int i = 0; i < rows; ++i) out[(row0 + i) * P.ld_out + col + h + lane] = turn[turn32(i, lane >> 2) + (lane & 3)];
                        }
                        __syncwarp();
                    }
                } else {
                    uint16_t* const out = static_cast<uint16_t*>(P.out);
                    const uint16_t* const half = reinterpret_cast<const uint16_t*>(turn);
#pragma unroll
                    for (int h = 0; h < 64; h += 32) {
                        uint32_t r[32];
                        float v[32];
                        tmem_load32(ta + (uint32_t)(c + h), r);
                        tmem_wait();
                        scaled(r, c + h, v);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            uint32_t p[4];
#pragma unroll
                            for (int j = 0; j < 4; ++j) p[j] = pack2(P.type, v[8 * i + 2 * j], v[8 * i + 2 * j + 1]);
                            *reinterpret_cast<uint4*>(turn + turn32(lane, h / 8 + i)) = make_uint4(p[0], p[1], p[2], p[3]);
                        }
                    }
                    __syncwarp();
                    if (P.vec && col + 64 <= P.N) {
#pragma unroll
                        for (int it = 0; it < 8; ++it) {
                            const int i = it * 4 + (lane >> 3);
                            if (i < rows)
                                *reinterpret_cast<uint4*>(out + (row0 + i) * P.ld_out + col + (lane & 7) * 8) = *reinterpret_cast<const uint4*>(turn + turn32(i, lane & 7));
                        }
                    } else {
#pragma unroll
                        for (int h = 0; h < 64; h += 32)
                            if (col + h + lane < P.N) {
#pragma unroll 8
                                for (int i = 0; i < rows; ++i) out[(row0 + i) * P.ld_out + col + h + lane] = half[2 * turn32(i, (h + lane) >> 3) + (lane & 7)];
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
}

// ---------------------------------------------------------------- few tokens, and everything small
// As ffn_few_kernel, with the roles exchanged: 128 channels are the rows of a tile, NR tokens its columns, so that a stage of the ring is
// nearly all weights; the contraction is split over the S CTAs of a cluster.  Sums of integers are exact in any order.
constexpr int kInt8FewThreads = 256;
constexpr int kInt8Part = 128;  // channels of a tile

template <int NR>
struct Int8FewShape {
    static constexpr int kA = kInt8Part * kInt8BK;
    static constexpr int kStage = kA + NR * kInt8BK;
    static constexpr int kStages = 110 * 1024 / kStage > 10 ? 10 : 110 * 1024 / kStage;
    static constexpr int kRing = kStages * kStage;
    static constexpr int kPassRows = NR < 64 ? NR : 64;        // tokens whose partial sums are exchanged at a time
    static_assert(kPassRows * kInt8Part * 4 <= kRing, "partial sums take the ring's place once it is done with");
    static constexpr int kBars = kRing;
    static constexpr int kSmem = kBars + 256 + 1024;
    static constexpr uint32_t kTmemCols = NR < 32 ? 32 : NR;
};

__device__ __forceinline__ int4 ld_cluster_ints(uint32_t addr, int cta) {
    const float4 v = ld_cluster4(addr, cta);
    return make_int4(__float_as_int(v.x), __float_as_int(v.y), __float_as_int(v.z), __float_as_int(v.w));
}
// A CTA's share of `some` tokens: a warp takes tokens S * 8 apart, a lane four channels, and as many tokens at once as make eight loads
template <int SP>
__device__ __forceinline__ void int8_few_finish(const Int8Params& P, uint32_t sums, int S, int part, int warp, int lane, int f, int first_row, int some) {
    constexpr int kRows = 8 / SP;
    const int left = P.N - f, step = S * (kInt8FewThreads / 32);
    float ws[4], b[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        ws[e] = e < left ? __ldca(P.w_scale + f + e) : 0.f;
        b[e] = e < left && P.bias ? __ldca(P.bias + f + e) : 0.f;
    }
    for (int i0 = part * (kInt8FewThreads / 32) + warp; i0 < some; i0 += step * kRows) {
        int4 y[kRows][SP];
        float qs[kRows];
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            if (r > 0 && i0 + r * step >= some) continue;
            const uint32_t at = sums + (uint32_t)(((i0 + r * step) * kInt8Part + lane * 4) * 4);
            qs[r] = __ldca(P.q_scale + first_row + i0 + r * step);
#pragma unroll
            for (int c = 0; c < SP; ++c)
                if (c < S) y[r][c] = ld_cluster_ints(at, c);
        }
        if (left <= 0) continue;
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            if (r > 0 && i0 + r * step >= some) continue;
            int4 x = y[r][0];
            bool none = x.x == kInt8None;
#pragma unroll
            for (int c = 1; c < SP; ++c) {
                if (c >= S) continue;
                none |= y[r][c].x == kInt8None;
                x.x += y[r][c].x; x.y += y[r][c].y; x.z += y[r][c].z; x.w += y[r][c].w;
            }
            float v[4] = {(float)x.x * qs[r] * ws[0] + b[0], (float)x.y * qs[r] * ws[1] + b[1], (float)x.z * qs[r] * ws[2] + b[2], (float)x.w * qs[r] * ws[3] + b[3]};
            if (none) v[0] = v[1] = v[2] = v[3] = int8_nan();
            const long long at = (first_row + i0 + r * step) * P.ld_out + f;
            if (P.vec && left >= 4) {
                if (P.type == BMGD_TYPE_F32) *reinterpret_cast<float4*>(static_cast<float*>(P.out) + at) = make_float4(v[0], v[1], v[2], v[3]);
                else *reinterpret_cast<uint2*>(static_cast<uint16_t*>(P.out) + at) = make_uint2(pack2(P.type, v[0], v[1]), pack2(P.type, v[2], v[3]));
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (e < left) int8_store1(P.out, P.type, at + e, v[e]);
            }
        }
    }
}

// Stages filled by the block's own threads where the rows of an operand do not start on 16-byte boundaries.  A thread keeps to its pieces' rows and columns of
// a stage, reads the two aligned pieces that hold each of its own and shifts them against one another.  They may reach into the neighbouring rows, never beyond the matrix:
// its ends, and rows of fewer than 48 values, are read byte by byte.  With a copy of both operands in front of the kernel
// instead: 29 x 1371 -> 2501 8.5 us and 3.5 more on the host, now 8.7; 60 x 4099 -> 4097 17.3, now 15.8; 16 x 11009 -> 4096 26.7, now 22.7 (with strides of 11008 13).
// Pieces stand where TMA would put them (128-byte swizzle); rows and columns beyond the matrix are zeros.
constexpr int kInt8Fillers = kInt8FewThreads - 32;
template <int NR>
struct Int8FewFill {
    static constexpr int kPieces = (kInt8Part + NR) * 8, kEach = (kPieces + kInt8Fillers - 1) / kInt8Fillers, kBatch = kEach <= 7 ? kEach : (kEach + 1) / 2;
    static_assert(kInt8Fillers % 8 == 0, "a thread keeps to its columns");
    const signed char* row[kEach];  // at this thread's columns
    unsigned some, first, last;     // a bit for each: not beyond the matrix; the matrix's first row, its last
    int thread, c;

    __device__ __forceinline__ static const signed char* place(const Int8Params& P, int f0, int r0, int i, int& r, int& rows) {  // of row i of a stage
        const bool token = i >= kInt8Part;
        r = token ? r0 + i - kInt8Part : f0 + i;
        rows = token ? P.M : P.N;
        return token ? P.q_rows + r * P.ld_q : P.w_rows + r * P.ld_w;
    }
    __device__ __forceinline__ void start(const Int8Params& P, int f0, int r0, int thread_) {
        some = first = last = 0;
        thread = thread_;
        c = (thread & 7) * 16;
#pragma unroll
        for (int u = 0; u < kEach; ++u) {
            int r, rows;
            row[u] = place(P, f0, r0, (thread + u * kInt8Fillers) >> 3, r, rows) + c;
            if (thread + u * kInt8Fillers >= kPieces || r >= rows) continue;
            some |= 1u << u;
            if (r == 0 || P.K < 48) first |= 1u << u;
            if (r == rows - 1 || P.K < 48) last |= 1u << u;
        }
    }
    // A stage's rows on their way to L2, two stages ahead (16 x 11009 -> 4096: 28 us to 24).  It reads nothing, so it may come before the wait for the kernel in front.
    __device__ __forceinline__ void fetch(const Int8Params& P, int k) const {
        if (c != 0 || k * kInt8BK >= P.K) return;
#pragma unroll
        for (int u = 0; u < kEach; ++u)
            if (some >> u & 1u) asm volatile("prefetch.global.L2 [%0];" ::"l"(row[u] + k * kInt8BK));
    }
    __device__ __forceinline__ static void put(uint32_t stage, int i, const uint32_t (&x)[4]) {
        const int r = i >> 3;
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(stage + (uint32_t)(r * kInt8BK + (((i ^ r) & 7) << 4))), "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]) : "memory");
    }
    __device__ __forceinline__ void operator()(const Int8Params& P, int f0, int r0, uint32_t stage, int k) const {
        const int at = k * kInt8BK + c, count = P.K - at;  // values from here to the rows' ends
        const unsigned here = count > 0 ? some : 0u, ends = here & ((at == 0 ? first : 0u) | (count < 32 ? last : 0u)), pieces = here & ~ends;
#pragma unroll
        for (int u0 = 0; u0 < kEach; u0 += kBatch) {
            uint4 v[kBatch][2];
#pragma unroll
            for (int u = u0; u < min(kEach, u0 + kBatch); ++u) {
                const uint4* two = reinterpret_cast<const uint4*>(row[u] + k * kInt8BK - ((uintptr_t)row[u] & 15u));
#pragma unroll
                for (int e = 0; e < 2; ++e) v[u - u0][e] = pieces >> u & 1u ? __ldca(two + e) : make_uint4(0, 0, 0, 0);
            }
#pragma unroll
            for (int u = u0; u < min(kEach, u0 + kBatch); ++u) {
                const uint4 &l = v[u - u0][0], &h = v[u - u0][1];
                const unsigned shift = (unsigned)((uintptr_t)row[u] & 15u);
                const bool by8 = shift & 8u, by4 = shift & 4u;
                const uint32_t w[6] = {by8 ? l.z : l.x, by8 ? l.w : l.y, by8 ? h.x : l.z, by8 ? h.y : l.w, by8 ? h.z : h.x, by8 ? h.w : h.y};
                uint32_t y[5], x[4];
#pragma unroll
                for (int e = 0; e < 5; ++e) y[e] = by4 ? w[e + 1] : w[e];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    x[e] = __funnelshift_r(y[e], y[e + 1], 8 * (shift & 3u));
                    if (count < 16) x[e] &= count >= 4 * e + 4 ? ~0u : count <= 4 * e ? 0u : ~0u >> (32 - 8 * (count - 4 * e));
                }
                if (thread + u * kInt8Fillers < kPieces) put(stage, thread + u * kInt8Fillers, x);
            }
        }
#pragma unroll 1
        for (unsigned left = ends; left != 0; left &= left - 1) {
            const int i = thread + (__ffs((int)left) - 1) * kInt8Fillers;
            int r, rows;
            const signed char* p = place(P, f0, r0, i >> 3, r, rows) + at;
            uint32_t byte[16], x[4] = {0u, 0u, 0u, 0u};
#pragma unroll
            for (int b = 0; b < 16; ++b) byte[b] = b < count ? (uint32_t)(unsigned char)__ldca(p + b) : 0u;
#pragma unroll
            for (int b = 0; b < 16; ++b) x[b / 4] |= byte[b] << (8 * (b % 4));
            put(stage, i, x);
        }
        fence_async_proxy();  // (the products read shared memory by the other way)
    }
};
template <>
struct Int8FewFill<0> {};

// Grid: S CTAs (one cluster) per tile; tiles_m and tiles_n count tiles of NR tokens and of 128 channels.  ANY: rows on any boundary, filled by all
// warps but the one that issues the products.
template <int NR, bool ANY>
__global__ void __launch_bounds__(kInt8FewThreads, 2) int8_few_kernel(const __grid_constant__ Int8Params P, const int S) {
    using F = Int8FewShape<NR>;
    extern __shared__ unsigned char int8_smem[];
    const uint32_t ring = (smem_u32(int8_smem) + 1023u) & ~1023u;
    const uint32_t full = ring + F::kBars, empty = full + 8 * F::kStages, done = empty + 8 * F::kStages, slot = done + 8;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int part = (int)blockIdx.x % S, tile = (int)blockIdx.x / S;
    const int f0 = tile / P.tiles_m * kInt8Part, r0 = tile % P.tiles_m * NR;

    if (threadIdx.x == 0) {
        for (int s = 0; s < F::kStages; ++s) { mbar_init(full + 8 * s, ANY ? kInt8Fillers / 32 : 1); mbar_init(empty + 8 * s, 1); }
        mbar_init(done, 1);
        fence_barrier_init();
    }
    if (!ANY && threadIdx.x == 32) {
        prefetch_map(&P.w);
        prefetch_map(&P.q);
    }
    if (warp == 2) ffn_tmem_alloc<1>(slot, F::kTmemCols);
    const int steps = (P.K + kInt8BK - 1) / kInt8BK;
    const int first = (int)((long long)steps * part / S), last = (int)((long long)steps * (part + 1) / S);
    Int8FewFill<ANY ? NR : 0> fill;
    if constexpr (ANY) {
        fill.start(P, f0, r0, (int)threadIdx.x - (warp > 1 ? 32 : 0));
        if (warp != 1) {
            fill.fetch(P, first);
            if (first + 1 < last) fill.fetch(P, first + 1);
        }
    } else if (warp == 3 && first + lane < min(last, first + 8)) {  // weights on their way to L2 while the kernel in front still runs (norm, product 4096 -> 22016, gate, product: 8 tokens 38.5 us to 33.4)
        asm volatile("cp.async.bulk.prefetch.tensor.2d.L2.global.tile [%0, {%1, %2}];" ::"l"(&P.w), "r"((first + lane) * kInt8BK), "r"(f0) : "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    uint32_t tmem;
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(tmem) : "r"(slot));
    wait_for_previous_kernel();
    let_next_kernel_start();

    FfnWait w{P.gave_up, P.timeout_ns, false};
    const int fill_to = (int)min((long long)last, (long long)first + P.fills);
    if (ANY && warp != 1) {
        int s = 0;
        uint32_t phase = 0;
        for (int k = first; k < fill_to; ++k) {
            ffn_wait(empty + 8 * s, phase ^ 1u, w);
            w.aborted = __any_sync(0xFFFFFFFFu, w.aborted);
            if (w.aborted) break;
            if constexpr (ANY) {
                if (k + 2 < fill_to) fill.fetch(P, k + 2);
                fill(P, f0, r0, ring + s * F::kStage, k);
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(full + 8 * s);
            if (++s == F::kStages) { s = 0; phase ^= 1u; }
        }
    } else if (!ANY && warp == 0) {
        if (lane == 0) {
            int s = 0;
            uint32_t phase = 0;
            for (int k = first; k < fill_to; ++k) {
                ffn_wait(empty + 8 * s, phase ^ 1u, w);
                if (w.aborted) break;
                const uint32_t bar = full + 8 * s, sa = ring + s * F::kStage;
                mbar_arrive_expect_tx(bar, F::kStage);
                ffn_tma<1>(sa, &P.w, k * kInt8BK, f0, bar);
                ffn_tma<1>(sa + F::kA, &P.q, k * kInt8BK, r0, bar);
                if (++s == F::kStages) { s = 0; phase ^= 1u; }
            }
            ffn_drain(full, F::kStages, s, phase, w);
        }
    } else if (warp == 1) {
        if (lane == 0) {
            const uint32_t idesc = int8_idesc(128, NR);
            const uint64_t desc = tc_smem_desc(0, 16, 1024);
            int s = 0;
            uint32_t phase = 0;
            for (int k = first; k < last; ++k) {
                ffn_wait(full + 8 * s, phase, w);
                if (w.aborted) break;
                tc_fence_after();
                const uint32_t at = ring + s * F::kStage;
                uint64_t da = desc + ((at >> 4) & 0x3FFFu), db = desc + (((at + F::kA) >> 4) & 0x3FFFu);
#pragma unroll
                for (int i = 0; i < kInt8BK / 32; ++i, da += 2, db += 2) int8_mma<1>(tmem, da, db, idesc, (k != first || i != 0) ? 1u : 0u);
                ffn_commit<1>(empty + 8 * s);
                if (++s == F::kStages) { s = 0; phase ^= 1u; }
            }
            if (!w.aborted) ffn_commit<1>(done);  // (waited for below)
            else ffn_drain(empty, F::kStages, s, phase, w);
        }
    }
    __syncwarp();
    // after the last product the ring's memory is free for the partial sums [token][128 channels]
    ffn_wait(done, 0, w);
    tc_fence_after();
    const bool given_up = __syncthreads_or(w.aborted ? 1 : 0) != 0;

    const int f = f0 + lane * 4;
    const int rows = min(NR, P.M - r0);
    const uint32_t ta = tmem + ((uint32_t)((warp & 3) * 32) << 16);
#pragma unroll 1
    for (int at = 0; at < rows; at += F::kPassRows) {
        if (at > 0) {  // the sums of the pass before have been read
            __syncthreads();
            if (S > 1) { cluster_arrive_release(); cluster_wait_acquire(); }
        }
        // two warps share a quarter of the channels: they take turns at 16 tokens
        const uint32_t to = ring + (uint32_t)(((warp & 3) * 32 + lane) * 4);
#pragma unroll 1
        for (int c = (warp >> 2) * 16; c < F::kPassRows; c += 32) {
            if (at + c >= rows) continue;
            uint32_t r[16];
            tmem_load16(ta + (uint32_t)(at + c), r);
            tmem_wait();
#pragma unroll
            for (int i = 0; i < 16; ++i)
                asm volatile("st.shared.b32 [%0], %1;" ::"r"(to + (uint32_t)((c + i) * kInt8Part * 4)), "r"(given_up ? (uint32_t)kInt8None : r[i]) : "memory");
        }
        tc_fence_before();
        __syncthreads();
        if (S > 1) { cluster_arrive_release(); cluster_wait_acquire(); }
        const int some = min(F::kPassRows, rows - at);
        if (S == 1) int8_few_finish<1>(P, ring, S, part, warp, lane, f, r0 + at, some);
        else if (S == 2) int8_few_finish<2>(P, ring, S, part, warp, lane, f, r0 + at, some);
        else if (S <= 4) int8_few_finish<4>(P, ring, S, part, warp, lane, f, r0 + at, some);
        else int8_few_finish<8>(P, ring, S, part, warp, lane, f, r0 + at, some);
    }
    if (given_up) ffn_linger();
    __syncthreads();
    if (S > 1) { cluster_arrive_release(); cluster_wait_acquire(); }  // peers have read this CTA's sums
    tc_fence_after();
    if (warp == 2) ffn_tmem_free<1>(tmem, F::kTmemCols);
}

// ---------------------------------------------------------------- one or two tokens
// A warp to a channel, its row of weights read in batches of 32 x 4 pieces of 16 bytes, the next batch (or channel) under way while this
// one is multiplied on the integer dot-product units; the tokens stand in shared memory.  Bound by reading the weights once.  No tensor maps, barriers or
// tensor memory to set up, and no split along the contraction: 1 x 4096 -> 11008 8.7 us where int8_few_kernel took 11.8 (a launch by itself 2.3,
// reading the weights at the copy rate 6.9); in batches of 8 pieces with half as many warps 10.9.  Four tokens took 16.0 that way where int8_few_kernel
// takes 12.0: each is read from shared memory as often as the weights from memory.
constexpr int kInt8Vec = 4;
// Weights that all warps together bring to L2 before they wait for the kernel in front, in lines of 128 bytes: a quarter of L2, so that none is gone again when it is read.  1 x 4096 ->
// 11008 9.9 us without any, 8.7 with 32 MB, 9.1 with 64 or without a bound (45 MB); 1 x 16384 -> 4096 13.5, 11.6, 13.3; 1 x 65552 -> 11008 117, 117, 119, 127 without a bound (310 MB).
constexpr long long kInt8Ahead = (32ll << 20) / 128;
constexpr __host__ __device__ int int8_ahead(long long warps) { return (int)(kInt8Ahead / warps); }
// of the next row, `left` being a warp's share that is left
constexpr __host__ __device__ int int8_ahead_lines(int inputs, int left) { return (inputs + 127) / 128 < left ? (inputs + 127) / 128 : left; }
constexpr bool int8_ahead_holds() {
    for (int inputs : {1, 127, 128, 129, 4096, 11008, 16000, 65552, 102400})
        for (int warps : {1, 37, 296 * 8, 296 * 13, 296 * 16}) {
            long long all = 0;
            for (int left = int8_ahead(warps), rows = 0; rows < 4 && left > 0; left -= int8_ahead_lines(inputs, left), ++rows) all += warps * (long long)int8_ahead_lines(inputs, left);
            if (all > kInt8Ahead) return false;
        }
    return true;
}
static_assert(int8_ahead_holds(), "all warps' lines together stay within the bound");
struct Int8VecParams {
    const signed char *q, *w;               // rows of w on 16-byte boundaries
    const float *q_scale, *w_scale, *bias;
    void* out;
    long long ld_q, ld_w, ld_out;
    int N, K, type;
    int ahead;                              // lines of weights that a warp brings to L2 before it waits
};
template <int M>
__global__ void __launch_bounds__(512, 2) int8_vec_kernel(const __grid_constant__ Int8VecParams P) {
    extern __shared__ uint4 int8_tokens[];  // [M][pieces], zeros behind the last value
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    const int pieces = (P.K + 15) / 16, full = P.K / 16, batches = (full + 32 * kInt8Vec - 1) / (32 * kInt8Vec), step = (int)gridDim.x * warps;
    int n = (int)blockIdx.x * warps + warp;
    // weights on their way to L2 while the kernel in front still runs; it reads nothing
    for (int c = n, left = P.ahead; c < P.N && left > 0; c += step, left -= int8_ahead_lines(P.K, left))
        for (int b = lane; b < int8_ahead_lines(P.K, left); b += 32) asm volatile("prefetch.global.L2 [%0];" ::"l"(P.w + c * P.ld_w + b * 128));
    wait_for_previous_kernel();
    let_next_kernel_start();
    uint4 v[kInt8Vec];
    auto fetch = [&](int channel, int batch) {
        const uint4* row = reinterpret_cast<const uint4*>(P.w + channel * P.ld_w);
#pragma unroll
        for (int u = 0; u < kInt8Vec; ++u) {
            const int p = (batch * kInt8Vec + u) * 32 + lane;
            v[u] = p < full ? __ldcs(row + p) : make_uint4(0, 0, 0, 0);
        }
    };
    if (n < P.N) fetch(n, 0);
    for (int m = 0; m < M; ++m) {
        signed char* to = reinterpret_cast<signed char*>(int8_tokens + m * pieces);
        const signed char* from = P.q + m * P.ld_q;
        if (((uintptr_t)from & 15u) == 0) {
            for (int p = threadIdx.x; p < full; p += blockDim.x) int8_tokens[m * pieces + p] = *reinterpret_cast<const uint4*>(from + 16 * p);
            if (threadIdx.x < 16 && full < pieces) to[full * 16 + threadIdx.x] = full * 16 + (int)threadIdx.x < P.K ? from[full * 16 + threadIdx.x] : (signed char)0;
        } else {
            for (int c = threadIdx.x; c < pieces * 16; c += blockDim.x) to[c] = c < P.K ? from[c] : (signed char)0;
        }
    }
    __syncthreads();
    for (; n < P.N; n += step) {
        int sum[M] = {};
        for (int b = 0; b < batches; ++b) {
            uint4 now[kInt8Vec];
#pragma unroll
            for (int u = 0; u < kInt8Vec; ++u) now[u] = v[u];
            if (b + 1 < batches) fetch(n, b + 1);
            else if (n + step < P.N) fetch(n + step, 0);
#pragma unroll
            for (int u = 0; u < kInt8Vec; ++u) {
                const int p = (b * kInt8Vec + u) * 32 + lane;
                if (p >= full) continue;
#pragma unroll
                for (int m = 0; m < M; ++m) {
                    const uint4 t = int8_tokens[m * pieces + p];
                    sum[m] = __dp4a((int)now[u].x, (int)t.x, sum[m]);
                    sum[m] = __dp4a((int)now[u].y, (int)t.y, sum[m]);
                    sum[m] = __dp4a((int)now[u].z, (int)t.z, sum[m]);
                    sum[m] = __dp4a((int)now[u].w, (int)t.w, sum[m]);
                }
            }
        }
        if (batches == 0 && n + step < P.N) fetch(n + step, 0);
        // what is left of the row, fewer than 16 values
        if (full * 16 + lane < P.K) {
            const int c = full * 16 + lane, x = P.w[n * P.ld_w + c];
#pragma unroll
            for (int m = 0; m < M; ++m) sum[m] += x * reinterpret_cast<const signed char*>(int8_tokens + m * pieces)[c];
        }
        const float ws = __ldca(P.w_scale + n), bias = P.bias ? __ldca(P.bias + n) : 0.f;
#pragma unroll
        for (int m = 0; m < M; ++m) {
            const int total = __reduce_add_sync(0xFFFFFFFFu, sum[m]);
            if (lane == m) int8_store1(P.out, P.type, m * P.ld_out + n, (float)total * __ldca(P.q_scale + m) * ws + bias);
        }
    }
}

// ---------------------------------------------------------------- operands that TMA cannot read
// Rows of `cols` bytes from stride ld to stride ld_out (a multiple of 16, at least cols), the rest of each row zero.
struct Int8AlignJob {
    const signed char* in;
    signed char* out;
    long long ld, ld_out, rows;
    int cols;
};
struct Int8AlignParams {
    Int8AlignJob job[2];
};
__device__ __forceinline__ void int8_align_one(const Int8AlignJob& j) {
    const unsigned per = (unsigned)(j.ld_out / 16);
    const long long total = j.rows * per;
    for (long long i = blockIdx.x * 256ll + threadIdx.x; i < total; i += gridDim.x * 256ll) {
        const long long r = i / per;
        const int c = (int)(i - r * per) * 16;
        const signed char* in = j.in + r * j.ld + c;
        uint32_t v[4];
        const unsigned shift = (unsigned)((uintptr_t)in & 3u);
        // inside the row: words, shifted; next to its ends byte by byte
        if (c >= 4 && c + 20 <= j.cols) {
            const uint32_t* word = reinterpret_cast<const uint32_t*>(in - shift);
            uint32_t lo = word[0];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t hi = word[k + 1];
                v[k] = __funnelshift_r(lo, hi, 8 * shift);
                lo = hi;
            }
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                v[k] = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (c + 4 * k + e < j.cols) v[k] |= (uint32_t)(unsigned char)in[4 * k + e] << (8 * e);
            }
        }
        *reinterpret_cast<uint4*>(j.out + r * j.ld_out + c) = make_uint4(v[0], v[1], v[2], v[3]);
    }
}
template <int JOBS>  // (a template, so that every file may hold it)
__global__ void __launch_bounds__(256) int8_align_kernel(const __grid_constant__ Int8AlignParams P) {
    wait_for_previous_kernel();
    let_next_kernel_start();
    int8_align_one(P.job[blockIdx.y]);
}

}  // namespace bmgdk
