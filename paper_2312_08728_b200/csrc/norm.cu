// Host side of bmgd_rms_norm_forward, bmgd_rms_norm_backward, bmgd_quantize_rows and bmgd_quantize_weight.
#include <algorithm>
#include <cmath>
#include <limits>

#include "../../include/bmgd.h"
#include "norm_kernel.cuh"
#include "operator_host.cuh"
#include "overlap.cuh"

namespace {

using namespace bmgdk;

int launched() { return cudaGetLastError() == cudaSuccess ? BMGD_OK : BMGD_ERR_CUDA; }
// As a dependent of the kernel before it, and letting the next one start beside it: a token's way through a layer is a row of short kernels, and a product brings its
// weights to L2 meanwhile.
template <typename P>
int start(void (*fn)(P), unsigned grid, int threads, const P& params, cudaStream_t s) {
    cudaLaunchConfig_t lc{};
    cudaLaunchAttribute at[2];
    launch_config(&lc, at, dim3(grid), threads, 0, 1, s);
    if (cudaLaunchKernelEx(&lc, fn, params) != cudaSuccess) { cudaGetLastError(); return BMGD_ERR_CUDA; }
    return BMGD_OK;
}
int value_bytes(int type) { return type == BMGD_TYPE_F32 ? 4 : 2; }
bool off(const void* p, int bytes) { return (uintptr_t)p % (unsigned)bytes != 0; }
// whether rows of that stride in bytes all start on 16-byte boundaries
bool on16(const void* p, int64_t stride) { return ((uintptr_t)p | (uintptr_t)stride) % 16 == 0; }

// Threads of a row of `count` pieces: a warp up to 64 (two each), then two pieces a thread up to 1024, four up to 2048, eight.
struct Threads {
    int pieces, threads;  // of a thread; 32: a warp, eight rows to a block
};
Threads threads_for(int64_t count) {
    if (count <= 32) return {1, 32};
    if (count <= 64) return {2, 32};
    const int nv = count <= 1024 ? 2 : count <= 2048 ? 4 : 8;
    return {nv, (int)((count + nv * 32 - 1) / (nv * 32)) * 32};
}
// Blocks that go through the rows: as many as the registers of an SM hold (64 a thread, with four pieces 128), and a multiple of eight where they come
// round again: eight rows on, every tensor's rows start at the same place within 16 bytes.
unsigned flow_grid(const Threads& t, int64_t rows, int per_sm_threads) {
    if (t.threads == 32) return (unsigned)std::min<int64_t>((rows + 7) / 8, 148 * (per_sm_threads / 256));
    const int64_t most = 148 * std::max(1, per_sm_threads / t.threads) / 8 * 8;
    return (unsigned)std::min<int64_t>(rows, most);
}

template <typename T, bool RES, bool CODES, bool ANY>
int forward_flow(const NormParams& P, cudaStream_t s) {
    const Threads t = threads_for((P.width + Piece<T>::kValues - 1) / Piece<T>::kValues);
    const unsigned grid = flow_grid(t, P.rows, t.pieces >= 4 ? 512 : 1024);
    if (t.threads == 32 && t.pieces == 1) return start(norm_flow_kernel<T, 1, true, RES, CODES, ANY>, grid, 256, P, s);
    if (t.threads == 32) return start(norm_flow_kernel<T, 2, true, RES, CODES, ANY>, grid, 256, P, s);
    if (t.pieces == 2) return start(norm_flow_kernel<T, 2, false, RES, CODES, ANY>, grid, t.threads, P, s);
    if (t.pieces == 4) return start(norm_flow_kernel<T, 4, false, RES, CODES, ANY>, grid, t.threads, P, s);
    return start(norm_flow_kernel<T, 8, false, RES, CODES, ANY>, grid, t.threads, P, s);
}
// Rows of up to 4096 pieces; longer ones are read more than once.
template <typename T, bool CODES>
int forward(const NormParams& P, bool aligned, cudaStream_t s) {
    const int64_t pieces = ((int64_t)P.width * (int64_t)sizeof(T) + 15) / 16;
    if (pieces > 4096) return start(norm_long_kernel<T, CODES>, (unsigned)P.rows, 1024, P, s);
    if (aligned) return P.residual ? forward_flow<T, true, CODES, false>(P, s) : forward_flow<T, false, CODES, false>(P, s);
    return P.residual ? forward_flow<T, true, CODES, true>(P, s) : forward_flow<T, false, CODES, true>(P, s);
}

// How the backward pass takes a row: in pieces of 16 bytes where every row of every tensor starts on such a boundary; on any boundary; long rows
// in pieces or single values.
struct BackShape {
    bool aligned;
    Threads of;           // threads 0: the form for long rows
    int blocks;
};
BackShape back_shape(const bmgd_rms_norm* a) {
    const int eb = value_bytes(a->type), ve = 16 / eb;
    const uintptr_t low = (uintptr_t)a->total | (uintptr_t)a->dy | (uintptr_t)a->dtotal | (uintptr_t)a->dx |
                          (uintptr_t)((a->ld_total | a->ld_dy | (a->dtotal ? a->ld_dtotal : 0) | a->ld_dx) * eb);
    BackShape b{};
    b.aligned = low % 16 == 0 && a->width % ve == 0;
    const int pieces = (a->width + ve - 1) / ve;
    if (pieces > 2048) {
        b.blocks = (int)std::min<int64_t>(a->rows, 148);
    } else {
        b.of = threads_for(pieces);
        b.blocks = (int)flow_grid(b.of, a->rows, 512);
    }
    return b;
}
constexpr int kMostSums = 50 * 1024;  // columns whose sums fit shared memory
template <typename T, int VE>
int backward_long(const NormParams& P, unsigned grid, cudaStream_t s) {
    if (!P.part || P.width > kMostSums) {
        norm_back_long_kernel<T, VE, false><<<grid, 1024, 0, s>>>(P);
        return launched();
    }
    Device dev{};
    int rc = current_device(&dev);
    static std::atomic<unsigned long long> allowed{0};
    if (rc == BMGD_OK) rc = allow_smem(norm_back_long_kernel<T, VE, true>, kMostSums * 4, dev, allowed);
    if (rc != BMGD_OK) return rc;
    norm_back_long_kernel<T, VE, true><<<grid, 1024, (size_t)P.width * 4, s>>>(P);
    return launched();
}
template <typename T, bool ANY>
int backward_flow(const NormParams& P, const BackShape& b, cudaStream_t s) {
    const unsigned grid = (unsigned)b.blocks;
    if (b.of.threads == 32 && b.of.pieces == 1) norm_back_kernel<T, 1, true, ANY><<<grid, 256, 0, s>>>(P);
    else if (b.of.threads == 32) norm_back_kernel<T, 2, true, ANY><<<grid, 256, 0, s>>>(P);
    else if (b.of.pieces == 2) norm_back_kernel<T, 2, false, ANY><<<grid, b.of.threads, 0, s>>>(P);
    else norm_back_kernel<T, 4, false, ANY><<<grid, b.of.threads, 0, s>>>(P);
    return launched();
}
template <typename T>
int backward(const NormParams& P, const BackShape& b, cudaStream_t s) {
    if (b.of.threads == 0) return b.aligned ? backward_long<T, Piece<T>::kValues>(P, (unsigned)b.blocks, s) : backward_long<T, 1>(P, (unsigned)b.blocks, s);
    return b.aligned ? backward_flow<T, false>(P, b, s) : backward_flow<T, true>(P, b, s);
}
template <typename T>
int backward_all(const NormParams& P, const BackShape& b, cudaStream_t s) {
    const int rc = backward<T>(P, b, s);
    if (rc != BMGD_OK || !P.dweight) return rc;
    cudaLaunchConfig_t lc{};
    cudaLaunchAttribute at[2];
    launch_config(&lc, at, dim3((unsigned)((P.width + 31) / 32)), 1024, 0, 1, s);
    if (cudaLaunchKernelEx(&lc, norm_weight_kernel<T>, (const float*)P.part, b.blocks, P.width, P.dweight, P.weight_f32) != cudaSuccess) { cudaGetLastError(); return BMGD_ERR_CUDA; }
    return BMGD_OK;
}

int64_t weight_bytes(const bmgd_rms_norm* a) { return (int64_t)a->width * (a->weight_type == BMGD_TYPE_F32 ? 4 : value_bytes(a->type)); }
int check(const bmgd_rms_norm* a) {
    if (!a || a->rows < 0 || a->rows > 0x7FFFFFFFll || a->width < 1 || a->width > (1 << 24) || a->reserved != 0) return BMGD_ERR_ARG;
    if (a->type < BMGD_TYPE_F32 || a->type > BMGD_TYPE_F16) return BMGD_ERR_ARG;
    if (a->weight && a->weight_type != a->type && a->weight_type != BMGD_TYPE_F32) return BMGD_ERR_ARG;
    if (!(a->eps >= 0.0) || !std::isfinite((float)a->eps)) return BMGD_ERR_ARG;
    return off(a->weight, a->weight_type == BMGD_TYPE_F32 ? 4 : value_bytes(a->type)) ? BMGD_ERR_ARG : BMGD_OK;
}
NormParams shared_params(const bmgd_rms_norm* a) {
    NormParams P{};
    P.weight = a->weight;
    P.weight_f32 = a->weight_type == BMGD_TYPE_F32;
    P.rows = a->rows; P.width = a->width; P.eps = a->eps > 0.0 ? std::max((float)a->eps, std::numeric_limits<float>::denorm_min()) : 0.f; P.per_width = 1.f / (float)a->width;
    P.rstd = a->rstd;
    P.far = a->rows * a->width * value_bytes(a->type) > kFarBytes;
    return P;
}

int check_backward(const bmgd_rms_norm* a) {
    const int rc = check(a);
    if (rc != BMGD_OK) return rc;
    const int eb = value_bytes(a->type);
    if (a->ld_total < a->width || a->ld_dy < a->width || a->ld_dx < a->width || (a->dtotal && a->ld_dtotal < a->width)) return BMGD_ERR_ARG;
    if ((a->dweight != nullptr) != (a->weight != nullptr) || off(a->dweight, a->weight_type == BMGD_TYPE_F32 ? 4 : eb)) return BMGD_ERR_ARG;
    if (a->rows == 0) return BMGD_OK;
    if (!a->total || !a->dy || !a->dx || !a->rstd) return BMGD_ERR_ARG;
    if (off(a->total, eb) || off(a->dy, eb) || off(a->dx, eb) || off(a->dtotal, eb) || off(a->rstd, 4)) return BMGD_ERR_ARG;
    const int64_t w = (int64_t)a->width * eb;  // a row of dx may be written before another thread has read the same row
    const Region dx{a->dx, a->rows, w, a->ld_dx * eb};
    const int64_t weights = weight_bytes(a);
    return writes_apart({dx, vector_region(a->dweight, weights)}, {{a->total, a->rows, w, a->ld_total * eb}, {a->dy, a->rows, w, a->ld_dy * eb}, {a->dtotal, a->rows, w, a->ld_dtotal * eb},
                        vector_region(a->weight, weights), vector_region(a->rstd, a->rows * 4)}) ? BMGD_OK : BMGD_ERR_ARG;
}

// Up to 384 threads with two, four or six pieces: a row's values are held in fp32, and two blocks of four pieces a thread (85 registers) fit an SM.
template <typename T, bool GATE, bool ANY>
int codes_flow(const CodesParams& P, cudaStream_t s) {
    const int64_t count = (P.width + Piece<T>::kValues - 1) / Piece<T>::kValues;
    Threads t = threads_for(count);
    if (t.threads > 32) {
        t.pieces = count <= 768 ? 2 : count <= 1536 ? 4 : 6;
        t.threads = (int)((count + t.pieces * 32 - 1) / (t.pieces * 32)) * 32;
    }
    const unsigned grid = flow_grid(t, P.rows, t.pieces == 6 ? 384 : t.pieces == 4 ? 768 : 1024);
    if (t.threads == 32 && t.pieces == 1) return start(codes_flow_kernel<T, 1, true, GATE, ANY>, grid, 256, P, s);
    if (t.threads == 32) return start(codes_flow_kernel<T, 2, true, GATE, ANY>, grid, 256, P, s);
    if (t.pieces == 2) return start(codes_flow_kernel<T, 2, false, GATE, ANY>, grid, t.threads, P, s);
    if (t.pieces == 4) return start(codes_flow_kernel<T, 4, false, GATE, ANY>, grid, t.threads, P, s);
    return start(codes_flow_kernel<T, 6, false, GATE, ANY>, grid, t.threads, P, s);
}
template <typename T>
int codes(const CodesParams& P, bool aligned, cudaStream_t s) {
    if (((int64_t)P.width * (int64_t)sizeof(T) + 15) / 16 > 6 * 384) return start(codes_long_kernel<T>, (unsigned)P.rows, 1024, P, s);
    if (aligned) return P.gate ? codes_flow<T, true, false>(P, s) : codes_flow<T, false, false>(P, s);
    return P.gate ? codes_flow<T, true, true>(P, s) : codes_flow<T, false, true>(P, s);
}

template <typename T>
int weight_codes(const void* w, int64_t ld_w, int inputs, int outputs, signed char* codes, int64_t ld_codes, float* scale, cudaStream_t s) {
    codes_weight_kernel<T><<<(unsigned)((outputs + 31) / 32), 1024, 0, s>>>(static_cast<const T*>(w), ld_w, inputs, outputs, codes, ld_codes, scale);
    return launched();
}

}  // namespace

extern "C" {

int bmgd_rms_norm_forward(const bmgd_rms_norm* a, void* stream) {
    const int rc = check(a);
    if (rc != BMGD_OK) return rc;
    if (a->rows == 0) return BMGD_OK;
    const int eb = value_bytes(a->type);
    const int64_t w = (int64_t)a->width * eb;
    if (!a->x || a->ld_x < a->width || off(a->x, eb) || off(a->residual, eb) || off(a->total, eb) || off(a->y, eb) || off(a->rstd, 4) || off(a->scale, 4)) return BMGD_ERR_ARG;
    if ((a->y == nullptr) == (a->codes == nullptr) || (a->codes != nullptr) != (a->scale != nullptr)) return BMGD_ERR_ARG;
    if (a->y ? a->ld_y < a->width : a->ld_codes < a->width) return BMGD_ERR_ARG;
    if ((a->residual != nullptr) != (a->total != nullptr) || (a->residual && (a->ld_residual < a->width || a->ld_total < a->width))) return BMGD_ERR_ARG;
    // (rows are read more than once where they are long)
    const Region x{a->x, a->rows, w, a->ld_x * eb}, r{a->residual, a->rows, w, a->ld_residual * eb}, total{a->total, a->rows, w, a->ld_total * eb},
        y = a->y ? Region{a->y, a->rows, w, a->ld_y * eb} : Region{a->codes, a->rows, a->width, a->ld_codes};
    if (!writes_apart({total, y, vector_region(a->scale, a->rows * 4), vector_region(a->rstd, a->rows * 4)}, {x, r, vector_region(a->weight, weight_bytes(a))})) return BMGD_ERR_ARG;
    NormParams P = shared_params(a);
    P.x = a->x; P.ld_x = a->ld_x;
    P.residual = a->residual; P.ld_residual = a->ld_residual;
    P.total = a->total; P.ld_total = a->ld_total;
    P.y = a->y; P.ld_y = a->ld_y;
    P.codes = reinterpret_cast<signed char*>(a->codes); P.ld_codes = a->ld_codes; P.scale = a->scale;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool aligned = w % 16 == 0 && on16(a->x, a->ld_x * eb) && on16(a->residual, a->residual ? a->ld_residual * eb : 0) &&
                         on16(a->total, a->total ? a->ld_total * eb : 0) && (a->y ? on16(a->y, a->ld_y * eb) : on16(a->codes, a->ld_codes));
    if (a->type == BMGD_TYPE_F32) return a->y ? forward<float, false>(P, aligned, s) : forward<float, true>(P, aligned, s);
    if (a->type == BMGD_TYPE_BF16) return a->y ? forward<__nv_bfloat16, false>(P, aligned, s) : forward<__nv_bfloat16, true>(P, aligned, s);
    return a->y ? forward<__half, false>(P, aligned, s) : forward<__half, true>(P, aligned, s);
}

int bmgd_rms_norm_workspace_bytes(const bmgd_rms_norm* a, int64_t* bytes) {
    if (!bytes) return BMGD_ERR_ARG;
    const int rc = check(a);
    if (rc != BMGD_OK) return rc;
    *bytes = a->weight && a->rows > 0 ? up256(back_shape(a).blocks * (int64_t)a->width * 4) : 0;
    return BMGD_OK;
}

int bmgd_rms_norm_backward(const bmgd_rms_norm* a, void* workspace, int64_t workspace_bytes, void* stream) {
    int rc = check_backward(a);
    if (rc != BMGD_OK) return rc;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (a->rows == 0) {
        if (a->dweight && cudaMemsetAsync(a->dweight, 0, (size_t)a->width * (a->weight_type == BMGD_TYPE_F32 ? 4 : 2), s) != cudaSuccess) { cudaGetLastError(); return BMGD_ERR_CUDA; }
        return BMGD_OK;
    }
    int64_t need = 0;
    rc = bmgd_rms_norm_workspace_bytes(a, &need);
    if (rc != BMGD_OK) return rc;
    if (need > 0 && (!workspace || (uintptr_t)workspace % 256 != 0)) return BMGD_ERR_ARG;
    if (workspace_bytes < need) return BMGD_ERR_CAPACITY;
    const BackShape b = back_shape(a);
    NormParams P = shared_params(a);
    P.x = a->total; P.ld_x = a->ld_total;
    P.dy = a->dy; P.ld_dy = a->ld_dy;
    P.dtotal = a->dtotal; P.ld_dtotal = a->ld_dtotal;
    P.dx = a->dx; P.ld_dx = a->ld_dx;
    P.dweight = a->dweight;
    P.part = a->weight ? static_cast<float*>(workspace) : nullptr;
    if (a->type == BMGD_TYPE_F32) return backward_all<float>(P, b, s);
    if (a->type == BMGD_TYPE_BF16) return backward_all<__nv_bfloat16>(P, b, s);
    return backward_all<__half>(P, b, s);
}

int bmgd_quantize_rows(const bmgd_quantize_rows_args* a, void* stream) {
    if (!a || a->rows < 0 || a->rows > 0x7FFFFFFFll || a->width < 1 || a->width > (1 << 24) || a->type < BMGD_TYPE_F32 || a->type > BMGD_TYPE_F16) return BMGD_ERR_ARG;
    if (a->activation < BMGD_ACT_SILU || a->activation > BMGD_ACT_SIGMOID || a->reserved != 0) return BMGD_ERR_ARG;
    if (a->rows == 0) return BMGD_OK;
    const int eb = value_bytes(a->type);
    if (!a->x || !a->codes || !a->scale || a->ld_x < a->width || a->ld_codes < a->width || (a->gate && a->ld_gate < a->width)) return BMGD_ERR_ARG;
    if (off(a->x, eb) || off(a->gate, eb) || off(a->scale, 4)) return BMGD_ERR_ARG;
    const int64_t w = (int64_t)a->width * eb;
    const Region q{a->codes, a->rows, a->width, a->ld_codes};
    if (!writes_apart({q, vector_region(a->scale, a->rows * 4)}, {{a->x, a->rows, w, a->ld_x * eb}, {a->gate, a->rows, w, a->ld_gate * eb}})) return BMGD_ERR_ARG;
    const CodesParams P{a->x, a->gate, reinterpret_cast<signed char*>(a->codes), a->scale, a->ld_x, a->ld_gate, a->ld_codes, a->rows, a->width, a->activation};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool aligned = w % 16 == 0 && on16(a->x, a->ld_x * eb) && on16(a->gate, a->gate ? a->ld_gate * eb : 0) && on16(a->codes, a->ld_codes);
    if (a->type == BMGD_TYPE_F32) return codes<float>(P, aligned, s);
    if (a->type == BMGD_TYPE_BF16) return codes<__nv_bfloat16>(P, aligned, s);
    return codes<__half>(P, aligned, s);
}

int bmgd_quantize_weight(const void* dev_w, int64_t ld_w, int32_t inputs, int32_t outputs, int32_t type, int8_t* dev_codes,
                         int64_t ld_codes, float* dev_scale, void* stream) {
    if (inputs < 1 || outputs < 1 || inputs > (1 << 24) || outputs > (1 << 24) || type < BMGD_TYPE_F32 || type > BMGD_TYPE_F16) return BMGD_ERR_ARG;
    if (!dev_w || !dev_codes || !dev_scale || ld_w < outputs || ld_codes < inputs || off(dev_w, value_bytes(type)) || off(dev_scale, 4)) return BMGD_ERR_ARG;
    const int eb = value_bytes(type);
    if (!writes_apart({{dev_codes, outputs, inputs, ld_codes}, vector_region(dev_scale, outputs * 4ll)}, {{dev_w, inputs, (int64_t)outputs * eb, ld_w * eb}})) return BMGD_ERR_ARG;
    signed char* q = reinterpret_cast<signed char*>(dev_codes);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (type == BMGD_TYPE_F32) return weight_codes<float>(dev_w, ld_w, inputs, outputs, q, ld_codes, dev_scale, s);
    if (type == BMGD_TYPE_BF16) return weight_codes<__nv_bfloat16>(dev_w, ld_w, inputs, outputs, q, ld_codes, dev_scale, s);
    return weight_codes<__half>(dev_w, ld_w, inputs, outputs, q, ld_codes, dev_scale, s);
}

}  // extern "C"
