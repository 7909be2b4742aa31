// Host side of bmgd_softmax_residual and bmgd_gather_batch.
#include <algorithm>
#include <cmath>

#include "../../include/bmgd.h"
#include "residual_kernel.cuh"

namespace {

using namespace bmgdk;

int launched() { return cudaGetLastError() == cudaSuccess ? BMGD_OK : BMGD_ERR_CUDA; }

template <typename T, int TH, int NV>
int residual_rows(const T* z, int64_t ldz, const int32_t* y, T* out, int64_t ldo, float* loss, int64_t rows, int32_t C, float scale, int R, cudaStream_t s) {
    cudaLaunchConfig_t lc{};
    lc.gridDim = dim3((unsigned)(TH == 32 ? (rows + 7) / 8 : rows * R));
    lc.blockDim = dim3(TH == 32 ? 256 : TH);
    lc.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = R; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
    lc.attrs = at;
    lc.numAttrs = R > 1 ? 1 : 0;
    if (cudaLaunchKernelEx(&lc, residual_row_kernel<T, TH, NV>, z, (long long)ldz, y, out, (long long)ldo, loss, (long long)rows, C, scale, R) != cudaSuccess) {
        cudaGetLastError();
        return BMGD_ERR_CUDA;
    }
    return BMGD_OK;
}

// By the row's length in pieces of 16 bytes: a warp to a row up to 256 pieces, then blocks of 128 to 512 threads with eight
// pieces each, then the form that reads a row twice, or for a few rows clusters of blocks of 512.
template <typename T>
int residual(const void* logits, int64_t ldz, const int32_t* y, void* residual, int64_t ldo, float* loss, int64_t rows, int32_t C, float scale, cudaStream_t s) {
    const T* z = static_cast<const T*>(logits);
    T* out = static_cast<T*>(residual);
    if (C <= 64) {
        const unsigned grid = (unsigned)std::min<int64_t>((rows * (C <= 16 ? 2 : C <= 32 ? 4 : 8) + 255) / 256, 148 * 32);
        if (C <= 16) residual_short_kernel<T, 2><<<grid, 256, 0, s>>>(z, ldz, y, out, ldo, loss, rows, C, scale);
        else if (C <= 32) residual_short_kernel<T, 4><<<grid, 256, 0, s>>>(z, ldz, y, out, ldo, loss, rows, C, scale);
        else residual_short_kernel<T, 8><<<grid, 256, 0, s>>>(z, ldz, y, out, ldo, loss, rows, C, scale);
        return launched();
    }
    const int64_t pieces = ((int64_t)C * (int64_t)sizeof(T) + 15) / 16;
    if (pieces <= 32) return residual_rows<T, 32, 1>(z, ldz, y, out, ldo, loss, rows, C, scale, 1, s);
    if (pieces <= 64) return residual_rows<T, 32, 2>(z, ldz, y, out, ldo, loss, rows, C, scale, 1, s);
    if (pieces <= 128) return residual_rows<T, 32, 4>(z, ldz, y, out, ldo, loss, rows, C, scale, 1, s);
    if (pieces <= 256) return residual_rows<T, 32, 8>(z, ldz, y, out, ldo, loss, rows, C, scale, 1, s);
    if (pieces <= 512) return residual_rows<T, 128, 4>(z, ldz, y, out, ldo, loss, rows, C, scale, 1, s);
    if (pieces <= 1024) return residual_rows<T, 128, 8>(z, ldz, y, out, ldo, loss, rows, C, scale, 1, s);
    if (pieces <= 2048) return residual_rows<T, 256, 8>(z, ldz, y, out, ldo, loss, rows, C, scale, 1, s);
    if (pieces <= 4096) return residual_rows<T, 512, 8>(z, ldz, y, out, ldo, loss, rows, C, scale, 1, s);
    if (rows * 8 <= 148 * 2 && pieces <= 4096 * 8) return residual_rows<T, 512, 8>(z, ldz, y, out, ldo, loss, rows, C, scale, 8, s);
    if (pieces <= 8192) residual_long_kernel<T, 256><<<(unsigned)std::min<int64_t>(rows, 148 * 4), 256, 0, s>>>(z, ldz, y, out, ldo, loss, rows, C, scale);
    else if (pieces <= 20480) residual_long_kernel<T, 512><<<(unsigned)std::min<int64_t>(rows, 148 * 2), 512, 0, s>>>(z, ldz, y, out, ldo, loss, rows, C, scale);
    else residual_long_kernel<T, 1024><<<(unsigned)std::min<int64_t>(rows, 148), 1024, 0, s>>>(z, ldz, y, out, ldo, loss, rows, C, scale);
    return launched();
}

}  // namespace

extern "C" {

int bmgd_softmax_residual(const void* dev_logits, int64_t ld_logits, const int32_t* dev_y, int64_t rows, int32_t C, int32_t type,
                          double scale, void* dev_residual, int64_t ld_residual, float* dev_loss, void* stream) {
    if (rows < 0 || rows > 0x7FFFFFFFll || C < 1 || type < BMGD_TYPE_F32 || type > BMGD_TYPE_F16 || !std::isfinite((float)scale)) return BMGD_ERR_ARG;
    if (rows == 0) return BMGD_OK;
    if (!dev_logits || !dev_y || !dev_residual || ld_logits < C || ld_residual < C) return BMGD_ERR_ARG;
    const int eb = type == BMGD_TYPE_F32 ? 4 : 2;
    if ((uintptr_t)dev_logits % eb || (uintptr_t)dev_residual % eb || (uintptr_t)dev_y % 4 || (uintptr_t)dev_loss % 4) return BMGD_ERR_ARG;
    const uintptr_t z = (uintptr_t)dev_logits, o = (uintptr_t)dev_residual;  // the label's logit is read after its row is written
    if (z < o + (uintptr_t)(((rows - 1) * ld_residual + C) * eb) && o < z + (uintptr_t)(((rows - 1) * ld_logits + C) * eb)) return BMGD_ERR_ARG;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const float f = (float)scale;
    if (type == BMGD_TYPE_F32) return residual<float>(dev_logits, ld_logits, dev_y, dev_residual, ld_residual, dev_loss, rows, C, f, s);
    if (type == BMGD_TYPE_BF16) return residual<__nv_bfloat16>(dev_logits, ld_logits, dev_y, dev_residual, ld_residual, dev_loss, rows, C, f, s);
    return residual<__half>(dev_logits, ld_logits, dev_y, dev_residual, ld_residual, dev_loss, rows, C, f, s);
}

int bmgd_gather_batch(const void* dev_x, int64_t row_bytes, const int32_t* dev_y, int64_t rows, uint64_t seed, uint32_t chain,
                      uint32_t round, int64_t first, int64_t count, void* dev_out_x, int32_t* dev_out_y, void* stream) {
    if (rows < 1 || rows > 0x7FFFFFFFll || row_bytes < 1 || first < 0 || count < 0 || first > rows || count > rows - first) return BMGD_ERR_ARG;
    if (count == 0) return BMGD_OK;
    if (!dev_x || !dev_out_x || (dev_y && !dev_out_y) || (uintptr_t)dev_y % 4 || (uintptr_t)dev_out_y % 4) return BMGD_ERR_ARG;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const int grid = (int)std::min<int64_t>((count + 7) / 8, 148 * 8);
    const unsigned char* x = static_cast<const unsigned char*>(dev_x);
    unsigned char* o = static_cast<unsigned char*>(dev_out_x);
    const uintptr_t low = (uintptr_t)dev_x | (uintptr_t)dev_out_x | (uintptr_t)row_bytes;
    const uint32_t n0 = (uint32_t)rows, a = (uint32_t)first, n = (uint32_t)count;
    if (low % 16 == 0) gather_batch_kernel<uint4><<<grid, 256, 0, s>>>(x, row_bytes, dev_y, n0, seed, chain, round, a, n, o, dev_out_y);
    else if (low % 4 == 0) gather_batch_kernel<uint32_t><<<grid, 256, 0, s>>>(x, row_bytes, dev_y, n0, seed, chain, round, a, n, o, dev_out_y);
    else if (low % 2 == 0) gather_batch_kernel<uint16_t><<<grid, 256, 0, s>>>(x, row_bytes, dev_y, n0, seed, chain, round, a, n, o, dev_out_y);
    else gather_batch_kernel<unsigned char><<<grid, 256, 0, s>>>(x, row_bytes, dev_y, n0, seed, chain, round, a, n, o, dev_out_y);
    return launched();
}

}  // extern "C"
