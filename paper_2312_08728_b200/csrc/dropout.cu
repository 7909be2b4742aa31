// Host side of bmgd_dropout.
#include <cmath>

#include "../../include/bmgd.h"
#include "dropout_kernel.cuh"
#include "overlap.cuh"

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

}  // namespace

extern "C" {

int bmgd_dropout(const bmgd_dropout_args* a, void* stream) {
    if (!a || a->rows < 0 || a->rows > 0x7FFFFFFFll || a->width < 1 || a->width > (1ll << 40) || a->type < BMGD_TYPE_F32 || a->type > BMGD_TYPE_F16) return BMGD_ERR_ARG;
    if (!(a->rate >= 0.0) || !(a->rate < 1.0) || a->layer < 0 || a->layer > 0xFFFF) return BMGD_ERR_ARG;
    const uint32_t threshold = (uint32_t)std::nearbyint(a->rate * 65536.0);
    if (threshold > 65535u) return BMGD_ERR_ARG;  // (nothing would be kept)
    if (a->rows == 0) return BMGD_OK;
    if (a->width > (1ll << 60) / a->rows) return BMGD_ERR_ARG;
    const int64_t eb = a->type == BMGD_TYPE_F32 ? 4 : 2;
    if (!a->x || !a->y || a->ld_x < a->width || a->ld_y < a->width || (a->residual && a->ld_residual < a->width)) return BMGD_ERR_ARG;
    if ((uintptr_t)a->x % eb || (uintptr_t)a->y % eb || (uintptr_t)a->residual % eb || (uintptr_t)a->step % 8) return BMGD_ERR_ARG;
    const Region y{a->y, a->rows, a->width * eb, a->ld_y * eb};
    if (share_memory(y, vector_region(a->step, 8))) return BMGD_ERR_ARG;
    if (!same_or_apart(y, {a->x, a->rows, a->width * eb, a->ld_x * eb}) || !same_or_apart(y, {a->residual, a->rows, a->width * eb, a->ld_residual * eb})) return BMGD_ERR_ARG;
    DropoutParams P{};
    P.x = a->x; P.residual = a->residual; P.y = a->y; P.step = reinterpret_cast<const long long*>(a->step);
    P.ld_x = a->ld_x; P.ld_residual = a->ld_residual; P.ld_y = a->ld_y; P.rows = a->rows; P.width = a->width;
    for (uint32_t r = 0; r < 10; ++r) {
        P.key[r][0] = (uint32_t)a->seed + r * 0x9E3779B9u;
        P.key[r][1] = (uint32_t)(a->seed >> 32) + r * 0xBB67AE85u;
    }
    P.threshold = threshold; P.tag = kDropTag + (uint32_t)a->layer;
    P.factor = (float)(65536.0 / (65536.0 - threshold));
    if (a->ld_x == a->width && a->ld_y == a->width && (!a->residual || a->ld_residual == a->width)) { P.width *= a->rows; P.rows = 1; }
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (a->type == BMGD_TYPE_F32) return a->residual ? dropout<float, true>(P, s) : dropout<float, false>(P, s);
    if (a->type == BMGD_TYPE_BF16) return a->residual ? dropout<__nv_bfloat16, true>(P, s) : dropout<__nv_bfloat16, false>(P, s);
    return a->residual ? dropout<__half, true>(P, s) : dropout<__half, false>(P, s);
}

}  // extern "C"
