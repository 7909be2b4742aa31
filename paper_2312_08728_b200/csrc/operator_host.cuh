// Host side that the operators' launches share: facts of the device, tensor maps, workspaces.
#pragma once
#include <atomic>
#include <cstdint>
#include <cuda.h>
#include <cuda_runtime.h>
#include <mutex>

#include "../../include/bmgd.h"

namespace bmgdk {

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
inline EncodeTiledFn encode_tiled() {
    static std::once_flag once;
    static EncodeTiledFn fn = nullptr;
    std::call_once(once, [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) == cudaSuccess && q == cudaDriverEntryPointSuccess)
            fn = reinterpret_cast<EncodeTiledFn>(p);
        else
            cudaGetLastError();
    });
    return fn;
}

// What a launch needs to know of the current device.  Looked up once per device: a call of a small block takes less time on
// the GPU than these queries take on the host.
constexpr int kMaxDevices = 64;
struct Device {
    int index, sms, smem;
    unsigned* gave_up;
    unsigned fills;                // see FfnParams
    unsigned long long budget_ns;  // of any single wait inside a kernel; 0: wait_bound
};
int current_device(Device* d);

// A kernel's dynamic shared memory, allowed once per device; `done` holds a bit per device and belongs to the kernel.
template <typename K>
inline int allow_smem(K* fn, int bytes, const Device& dev, std::atomic<unsigned long long>& done) {
    const unsigned long long bit = 1ull << (dev.index & 63);
    if (done.load(std::memory_order_relaxed) & bit) return BMGD_OK;
    if (bytes > dev.smem) return BMGD_ERR_LAUNCH;
    if (cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) { cudaGetLastError(); return BMGD_ERR_CUDA; }
    if (dev.index < kMaxDevices) done.fetch_or(bit, std::memory_order_relaxed);
    return BMGD_OK;
}

// Bound on any single wait inside a kernel: two seconds, and more than a step of the contraction ever takes for each step.
inline unsigned long long wait_bound(const Device& dev, int64_t steps) { return dev.budget_ns ? dev.budget_ns : 2000000000ull + 10000ull * (unsigned long long)steps; }

inline void launch_config(cudaLaunchConfig_t* lc, cudaLaunchAttribute (&at)[2], dim3 grid, int threads, int smem, int cluster, cudaStream_t s) {
    lc->gridDim = grid;
    lc->blockDim = dim3((unsigned)threads);
    lc->dynamicSmemBytes = smem;
    lc->stream = s;
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = cluster; at[1].val.clusterDim.y = 1; at[1].val.clusterDim.z = 1;
    lc->attrs = at;
    lc->numAttrs = cluster > 1 ? 2 : 1;
}

inline int64_t up256(int64_t x) { return (x + 255) / 256 * 256; }

// Workspace in the order it is used: copies of operands whose rows TMA cannot read, then the intermediates.
struct Space {
    unsigned char* base;
    int64_t used;
    void* take(int64_t bytes) {
        void* p = base ? base + used : nullptr;
        used += up256(bytes);
        return p;
    }
};

}  // namespace bmgdk
