// What the contractions on the tensor cores share: bounded waits, copies by TMA, accumulators in tensor memory, the way of
// a row's values through shared memory.
#pragma once
#include <cstdint>
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "glm_kernel.cuh"  // barriers, clusters, the clock: its kernels are made in the tables that ask for them
#include "launch.cuh"
#include "tensor_core.cuh"

namespace bmgdk {

// A wait with a limit of its own: that one kernel gave up says nothing about the others, on this stream or another.
struct FfnWait {
    unsigned* gave_up;
    unsigned long long timeout_ns;
    bool aborted;
};
__device__ __forceinline__ void ffn_wait(uint32_t bar, uint32_t parity, FfnWait& w) {
    if (w.aborted || mbar_try_wait(bar, parity)) return;
    const unsigned long long t0 = global_ns();
    uint32_t spins = 0;
    while (!mbar_try_wait(bar, parity)) {
        if ((++spins & 0xFFu) == 0u && global_ns() - t0 >= w.timeout_ns) {
            atomicAdd(w.gave_up, 1u);
            w.aborted = true;
            return;
        }
    }
}

// Parity of the last round of stage `i` of a ring, `s` and `phase` being the stage and the round's parity that come next; 1
// for a stage without a round, which a barrier takes for completed.
constexpr __host__ __device__ uint32_t ffn_last_round(int i, int s, uint32_t phase) { return i < s ? phase : phase ^ 1u; }
constexpr bool ffn_last_round_holds() {
    for (int stages = 1; stages <= 10; ++stages)
        for (int fills = 0; fills <= 35; ++fills) {
            int s = 0;
            uint32_t phase = 0;
            for (int k = 0; k < fills; ++k)
                if (++s == stages) { s = 0; phase ^= 1u; }
            for (int i = 0; i < stages; ++i) {
                const int rounds = fills / stages + (i < fills % stages ? 1 : 0);
                if (ffn_last_round(i, s, phase) != (rounds == 0 ? 1u : (uint32_t)(rounds - 1) & 1u)) return false;
            }
        }
    return true;
}
static_assert(ffn_last_round_holds(), "a drained ring waits for the last round of every stage");
// A block leaves only when its copies have landed and its products are done, whoever of its warps gave up: the thread that
// issued them waits for the last round of every stage (in a launch that went well they are complete), with a limit again.
constexpr unsigned long long kFfnDrainNs = 1000000000ull;
__device__ __forceinline__ void ffn_drain(uint32_t bars, int stages, int s, uint32_t phase, const FfnWait& w) {
    FfnWait d{w.gave_up, kFfnDrainNs, false};
    for (int i = 0; i < stages; ++i) ffn_wait(bars + 8 * i, ffn_last_round(i, s, phase), d);
}
// What ffn_drain does not see after a wait was given up, it leaves time for: copies of a pair's second CTA that the first
// one, stopped earlier, had not announced, and arrivals on their way to the other CTA's barriers.
constexpr unsigned long long kFfnLingerNs = 1000000ull;
__device__ __forceinline__ void ffn_linger() {
    const unsigned long long t0 = global_ns();
    while (global_ns() - t0 < kFfnLingerNs) __nanosleep(1000);
}

__device__ __forceinline__ void prefetch_map(const CUtensorMap* map) { asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory"); }
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
template <int N> __device__ __forceinline__ void fill_nan(uint32_t (&r)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) r[i] = 0x7FC00000u;
}

__device__ __forceinline__ uint32_t pack2(int type, float a, float b) {
    if (type == BMGD_TYPE_BF16) {
        const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&v);
    }
    const __half2 v = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
}
// word of piece `c` (16 bytes) of row `r`
__device__ __forceinline__ int turn32(int r, int c) { return r * 32 + ((c ^ (((r & 1) << 2) | ((r >> 1) & 3))) << 2); }
__device__ __forceinline__ float4 ld_cluster4(uint32_t addr, int cta) {
    uint32_t a;
    float4 v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(addr), "r"(cta));
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(a) : "memory");
    return v;
}

}  // namespace bmgdk
