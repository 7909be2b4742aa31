// Host side of bmgd_dropout.
#include <cmath>

#include "../../include/bmgd.h"
#include "dropout_kernel.cuh"

namespace {

using namespace bmgdk;

template <typename T, bool RES>
int dropout(const DropoutParams& P, cudaStream_t s) {
    constexpr int kAhead = 2;
    const bool flat = P.rows == 1 && ((uintptr_t)P.x | (uintptr_t)P.y | (uintptr_t)P.residual) % 16 == 0;
    const int64_t blocks = flat ? (P.width / 8 + 1 + 256 * kAhead - 1) / (256 * kAhead) : (P.rows * ((P.width + 7) / 8 + 1) + 255) / 256;
    if (blocks > 0x7FFFFFFFll) return BMGD_ERR_ARG;
    if (flat) dropout_flat_kernel<T, RES, kAhead><<<(unsigned)blocks, 256, 0, s>>>(P);
    else dropout_rows_kernel<T, RES><<<(unsigned)blocks, 256, 0, s>>>(P);
    return cudaGetLastError() == cudaSuccess ? BMGD_OK : BMGD_ERR_CUDA;
}

// [rows][width] of strides lp and lq (in bytes w a row): the same memory value for value, or none of it
bool apart_or_same(const void* p, int64_t lp, const void* q, int64_t lq, int64_t w, int64_t rows) {
    if (p == q && (lp == lq || rows == 1)) return true;
    const uintptr_t a = (uintptr_t)p, b = (uintptr_t)q;
    return a >= b + (uintptr_t)((rows - 1) * lq + w) || b >= a + (uintptr_t)((rows - 1) * lp + w);
}

}  // namespace

extern "C" {

int bmgd_dropout(const void* dev_x, int64_t ld_x, const void* dev_residual, int64_t ld_residual, int64_t rows, int64_t width, int32_t type,
                 double rate, uint64_t seed, const int64_t* dev_step, int32_t layer, void* dev_y, int64_t ld_y, void* stream) {
    if (rows < 0 || rows > 0x7FFFFFFFll || width < 1 || width > (1ll << 40) || type < BMGD_TYPE_F32 || type > BMGD_TYPE_F16) return BMGD_ERR_ARG;
    if (!(rate >= 0.0) || !(rate < 1.0) || layer < 0 || layer > 0xFFFF) return BMGD_ERR_ARG;
    const uint32_t threshold = (uint32_t)std::nearbyint(rate * 65536.0);
    if (threshold > 65535u) return BMGD_ERR_ARG;  // (nothing would be kept)
    if (rows == 0) return BMGD_OK;
    if (width > (1ll << 60) / rows) return BMGD_ERR_ARG;
    const int64_t eb = type == BMGD_TYPE_F32 ? 4 : 2;
    if (!dev_x || !dev_y || ld_x < width || ld_y < width || (dev_residual && ld_residual < width)) return BMGD_ERR_ARG;
    if ((uintptr_t)dev_x % eb || (uintptr_t)dev_y % eb || (uintptr_t)dev_residual % eb || (uintptr_t)dev_step % 8) return BMGD_ERR_ARG;
    if (!apart_or_same(dev_y, ld_y * eb, dev_x, ld_x * eb, width * eb, rows)) return BMGD_ERR_ARG;
    if (dev_residual && !apart_or_same(dev_y, ld_y * eb, dev_residual, ld_residual * eb, width * eb, rows)) return BMGD_ERR_ARG;
    DropoutParams P{};
    P.x = dev_x; P.residual = dev_residual; P.y = dev_y; P.step = reinterpret_cast<const long long*>(dev_step);
    P.ld_x = ld_x; P.ld_residual = ld_residual; P.ld_y = ld_y; P.rows = rows; P.width = width;
    for (uint32_t r = 0; r < 10; ++r) {
        P.key[r][0] = (uint32_t)seed + r * 0x9E3779B9u;
        P.key[r][1] = (uint32_t)(seed >> 32) + r * 0xBB67AE85u;
    }
    P.threshold = threshold; P.tag = kDropTag + (uint32_t)layer;
    P.factor = (float)(65536.0 / (65536.0 - threshold));
    if (ld_x == width && ld_y == width && (!dev_residual || ld_residual == width)) { P.width *= rows; P.rows = 1; }
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (type == BMGD_TYPE_F32) return dev_residual ? dropout<float, true>(P, s) : dropout<float, false>(P, s);
    if (type == BMGD_TYPE_BF16) return dev_residual ? dropout<__nv_bfloat16, true>(P, s) : dropout<__nv_bfloat16, false>(P, s);
    return dev_residual ? dropout<__half, true>(P, s) : dropout<__half, false>(P, s);
}

}  // extern "C"
