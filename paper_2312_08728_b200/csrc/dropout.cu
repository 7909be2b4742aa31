// Host side of bmgd_dropout.
#include <cmath>

#include "../../include/bmgd.h"
#include "dropout_kernel.cuh"

namespace {

using namespace bmgdk;

template <typename T, bool ONE_ROW, bool RES>
int dropout_as(const DropoutParams& P, cudaStream_t s) {
    constexpr int kAhead = 2;
    const int64_t units = ONE_ROW ? (P.width + 7) / 8 : P.rows * ((P.width + 7) / 8 + 1);
    const int64_t blocks = (units + 256 * kAhead - 1) / (256 * kAhead);
    if (blocks > 0x7FFFFFFFll) return BMGD_ERR_ARG;
    dropout_kernel<T, ONE_ROW, RES, kAhead><<<(unsigned)blocks, 256, 0, s>>>(P);
    return cudaGetLastError() == cudaSuccess ? BMGD_OK : BMGD_ERR_CUDA;
}
template <typename T>
int dropout(const DropoutParams& P, cudaStream_t s) {
    if (P.rows == 1) return P.residual ? dropout_as<T, true, true>(P, s) : dropout_as<T, true, false>(P, s);
    return P.residual ? dropout_as<T, false, true>(P, s) : dropout_as<T, false, false>(P, s);
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
    DropoutParams P{dev_x, dev_residual, dev_y, reinterpret_cast<const long long*>(dev_step), ld_x, ld_residual, ld_y, rows, width, seed, threshold,
                    kDropTag + (uint32_t)layer, (float)(65536.0 / (65536.0 - threshold))};
    if (ld_x == width && ld_y == width && (!dev_residual || ld_residual == width)) { P.width *= rows; P.rows = 1; }
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (type == BMGD_TYPE_F32) return dropout<float>(P, s);
    if (type == BMGD_TYPE_BF16) return dropout<__nv_bfloat16>(P, s);
    return dropout<__half>(P, s);
}

}  // extern "C"
