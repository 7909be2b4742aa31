// Host side of the gated feed-forward block: checks, tensor maps, choice of tile, launches.
#include <algorithm>
#include <cstring>
#include <mutex>

#include "../../include/bmgd.h"
#include "ffn_kernel.cuh"

namespace {

using namespace bmgdk;

// Set by a kernel whose wait ran out of time; read and cleared by bmgd_stream_check.
__device__ int g_ffn_status[2];

int* status_address() {
    void* p = nullptr;
    if (cudaGetSymbolAddress(&p, g_ffn_status) != cudaSuccess) { cudaGetLastError(); return nullptr; }
    return static_cast<int*>(p);
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiledFn encode_tiled() {
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

// A matrix of 16-bit values as the kernels read it.
struct Matrix {
    const void* base;
    int64_t rows, cols, ld;
};

int make_map(const Matrix& m, int type, int box_rows, CUtensorMap* out) {
    EncodeTiledFn enc = encode_tiled();
    if (!enc) return BMGD_ERR_CUDA;
    const cuuint64_t dims[2] = {(cuuint64_t)m.cols, (cuuint64_t)m.rows};
    const cuuint64_t strides[1] = {(cuuint64_t)m.ld * 2u};
    const cuuint32_t box[2] = {64u, (cuuint32_t)box_rows};
    const cuuint32_t step[2] = {1u, 1u};
    const CUresult r = enc(out, type == BMGD_TYPE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2,
                           const_cast<void*>(m.base), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                           CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? BMGD_OK : BMGD_ERR_CUDA;
}

struct Device {
    int sms, smem;
};
int current_device(Device* d) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&d->sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&d->smem, cudaDevAttrMaxSharedMemoryPerBlockOptin, dev) != cudaSuccess) {
        cudaGetLastError();
        return BMGD_ERR_CUDA;
    }
    return BMGD_OK;
}

template <int CG, int BN, int EPI, bool A_MN, bool B_MN>
int launch(FfnParams& P, const Matrix (&a)[2], const Matrix (&b)[2], const Device& dev, cudaStream_t s) {
    using S = FfnShape<CG, BN>;
    constexpr int kCols = EPI == kEpiGated ? BN / 2 : BN;
    const int pairs_b = EPI == kEpiGated ? 2 : std::max(P.segments, P.problems);
    for (int i = 0; i < 2; ++i) {
        const int ka = i < P.segments ? i : 0, kb = i < pairs_b ? i : 0;
        int rc = make_map(a[ka], P.type, A_MN ? 64 : 128, &P.a[i]);
        if (rc == BMGD_OK) rc = make_map(b[kb], P.type, B_MN ? 64 : (EPI == kEpiGated ? BN / 2 : BN / CG), &P.b[i]);
        if (rc != BMGD_OK) return rc;
    }
    P.tiles_m = (int)((P.M + 128 * CG - 1) / (128 * CG));
    P.tiles_n = (P.N + kCols - 1) / kCols;
    const int64_t tiles = (int64_t)P.tiles_m * P.tiles_n * P.problems;
    if (S::kSmem > dev.smem) return BMGD_ERR_LAUNCH;
    auto* fn = ffn_kernel<CG, BN, EPI, A_MN, B_MN>;
    if (cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem) != cudaSuccess) { cudaGetLastError(); return BMGD_ERR_CUDA; }
    cudaLaunchConfig_t lc{};
    lc.gridDim = dim3((unsigned)std::min<int64_t>(tiles, dev.sms / CG) * CG);
    lc.blockDim = dim3(kFfnThreads);
    lc.dynamicSmemBytes = S::kSmem;
    lc.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = CG; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
    lc.attrs = at; lc.numAttrs = CG > 1 ? 1 : 0;
    if (cudaLaunchKernelEx(&lc, fn, P) != cudaSuccess) { cudaGetLastError(); return BMGD_ERR_CUDA; }
    return BMGD_OK;
}

// Tiles of 256 rows x 256 columns for two CTAs wherever they fill half the GPU; otherwise tiles of 128 x 128 for one.
template <int EPI, bool A_MN, bool B_MN>
int contract(FfnParams& P, const Matrix (&a)[2], const Matrix (&b)[2], const Device& dev, cudaStream_t s) {
    constexpr int kCols = EPI == kEpiGated ? 128 : 256;
    const int64_t large = ((P.M + 255) / 256) * ((P.N + kCols - 1) / kCols) * P.problems;
    if (large * 4 >= dev.sms) return launch<2, 256, EPI, A_MN, B_MN>(P, a, b, dev, s);
    return launch<1, 128, EPI, A_MN, B_MN>(P, a, b, dev, s);
}

int64_t up8(int64_t x) { return (x + 7) / 8 * 8; }
int64_t up256(int64_t x) { return (x + 255) / 256 * 256; }
bool tma_ready(const Matrix& m) { return (uintptr_t)m.base % 16 == 0 && m.ld % 8 == 0; }

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

int align_matrix(Matrix* m, Space* space, bool run, cudaStream_t s) {
    if (tma_ready(*m)) return BMGD_OK;
    Matrix to = *m;
    to.ld = up8(m->cols);
    to.base = space->take(to.rows * to.ld * 2);
    if (run) {
        const int64_t total = to.rows * to.ld;
        ffn_align_kernel<<<(unsigned)std::min<int64_t>((total + 255) / 256, 148 * 16), 256, 0, s>>>(
            static_cast<const uint16_t*>(m->base), m->ld, static_cast<uint16_t*>(const_cast<void*>(to.base)), to.ld, to.rows, (int)to.cols);
        if (cudaGetLastError() != cudaSuccess) return BMGD_ERR_CUDA;
    }
    *m = to;
    return BMGD_OK;
}

bool bad_pointer(const void* p) { return !p || (uintptr_t)p % 2 != 0; }

int check(const bmgd_gated_ffn* g, int pass, bool pointers) {
    if (!g || (pass != BMGD_FFN_FORWARD && pass != BMGD_FFN_BACKWARD)) return BMGD_ERR_ARG;
    if (g->rows < 0 || g->rows > 0x7FFFFF00ll || g->inputs < 1 || g->hidden < 1 || g->outputs < 1) return BMGD_ERR_ARG;
    if (g->inputs > (1 << 24) || g->hidden > (1 << 24) || g->outputs > (1 << 24)) return BMGD_ERR_ARG;
    if (g->type == BMGD_TYPE_F32) return BMGD_ERR_UNIMPLEMENTED;
    if (g->type != BMGD_TYPE_BF16 && g->type != BMGD_TYPE_F16) return BMGD_ERR_ARG;
    if (g->activation < BMGD_ACT_SILU || g->activation > BMGD_ACT_SIGMOID || g->reserved != 0) return BMGD_ERR_ARG;
    if (g->ld_x < g->inputs || g->ld_gate < g->hidden || g->ld_up < g->hidden || g->ld_down < g->outputs) return BMGD_ERR_ARG;
    if (pass == BMGD_FFN_BACKWARD && g->ld_dy < g->outputs) return BMGD_ERR_ARG;
    if (pass == BMGD_FFN_FORWARD && g->ld_y < g->outputs) return BMGD_ERR_ARG;
    if ((pass == BMGD_FFN_BACKWARD || g->saved_value) && (g->ld_saved < g->hidden || g->ld_saved % 8 != 0)) return BMGD_ERR_ARG;
    if (!pointers || g->rows == 0) return BMGD_OK;
    if (bad_pointer(g->x) || bad_pointer(g->w_gate) || bad_pointer(g->w_up) || bad_pointer(g->w_down)) return BMGD_ERR_ARG;
    if ((g->saved_value == nullptr) != (g->saved_slope == nullptr) || (g->saved_value == nullptr) != (g->saved_hidden == nullptr)) return BMGD_ERR_ARG;
    if ((uintptr_t)g->saved_value % 16 || (uintptr_t)g->saved_slope % 16 || (uintptr_t)g->saved_hidden % 16) return BMGD_ERR_ARG;
    if (pass == BMGD_FFN_FORWARD) return bad_pointer(g->y) ? BMGD_ERR_ARG : BMGD_OK;
    if (!g->saved_value || bad_pointer(g->dy) || bad_pointer(g->dx) || bad_pointer(g->dw_gate) || bad_pointer(g->dw_up) || bad_pointer(g->dw_down))
        return BMGD_ERR_ARG;
    return BMGD_OK;
}

bool wide(const void* p, int64_t ld) { return (uintptr_t)p % 16 == 0 && ld % 8 == 0; }

// run = false: only counts the workspace
int forward(const bmgd_gated_ffn* g, Space* space, bool run, const Device& dev, int* status, cudaStream_t s) {
    Matrix x{g->x, g->rows, g->inputs, g->ld_x}, wg{g->w_gate, g->inputs, g->hidden, g->ld_gate},
        wu{g->w_up, g->inputs, g->hidden, g->ld_up}, wd{g->w_down, g->hidden, g->outputs, g->ld_down};
    for (Matrix* m : {&x, &wg, &wu, &wd}) {
        const int rc = align_matrix(m, space, run, s);
        if (rc != BMGD_OK) return rc;
    }
    const int64_t ldh = g->saved_hidden ? g->ld_saved : up8(g->hidden);
    void* h = g->saved_hidden ? g->saved_hidden : space->take(g->rows * ldh * 2);
    if (!run) return BMGD_OK;
    FfnParams P{};
    P.type = g->type; P.act = g->activation; P.status = status; P.timeout_ns = 2000000000ull;
    P.M = g->rows;
    P.segments = P.problems = 1;
    P.N = g->hidden; P.K = g->inputs;
    P.out[0] = h; P.ld_out = ldh;
    P.value = g->saved_value; P.slope = g->saved_slope; P.ld_save = g->ld_saved;
    {
        const Matrix a[2] = {x, x}, b[2] = {wg, wu};
        const int rc = contract<kEpiGated, false, true>(P, a, b, dev, s);
        if (rc != BMGD_OK) return rc;
    }
    P.N = g->outputs; P.K = g->hidden;
    P.out[0] = g->y; P.ld_out = g->ld_y;
    P.vec = wide(g->y, g->ld_y);
    const Matrix hm{h, g->rows, g->hidden, ldh};
    const Matrix a[2] = {hm, hm}, b[2] = {wd, wd};
    return contract<kEpiPlain, false, true>(P, a, b, dev, s);
}

int backward(const bmgd_gated_ffn* g, Space* space, bool run, const Device& dev, int* status, cudaStream_t s) {
    Matrix x{g->x, g->rows, g->inputs, g->ld_x}, wg{g->w_gate, g->inputs, g->hidden, g->ld_gate},
        wu{g->w_up, g->inputs, g->hidden, g->ld_up}, wd{g->w_down, g->hidden, g->outputs, g->ld_down},
        dy{g->dy, g->rows, g->outputs, g->ld_dy};
    for (Matrix* m : {&x, &wg, &wu, &wd, &dy}) {
        const int rc = align_matrix(m, space, run, s);
        if (rc != BMGD_OK) return rc;
    }
    const int64_t ldh = up8(g->hidden);
    const Matrix h{g->saved_hidden, g->rows, g->hidden, g->ld_saved}, dg{space->take(g->rows * ldh * 2), g->rows, g->hidden, ldh},
        du{space->take(g->rows * ldh * 2), g->rows, g->hidden, ldh};
    if (!run) return BMGD_OK;
    FfnParams P{};
    P.type = g->type; P.act = g->activation; P.status = status; P.timeout_ns = 2000000000ull;
    int rc;
    {   // dH, and from it dG and dU
        P.M = g->rows; P.N = g->hidden; P.K = g->outputs;
        P.segments = P.problems = 1;
        P.out[0] = const_cast<void*>(dg.base); P.out[1] = const_cast<void*>(du.base); P.ld_out = ldh;
        P.value = g->saved_value; P.slope = g->saved_slope; P.ld_save = g->ld_saved;
        const Matrix a[2] = {dy, dy}, b[2] = {wd, wd};
        rc = contract<kEpiBackward, false, false>(P, a, b, dev, s);
        if (rc != BMGD_OK) return rc;
    }
    {   // dX
        P.N = g->inputs; P.K = g->hidden; P.segments = 2;
        P.out[0] = g->dx; P.ld_out = g->inputs;
        P.vec = wide(g->dx, g->inputs);
        const Matrix a[2] = {dg, du}, b[2] = {wg, wu};
        rc = contract<kEpiPlain, false, false>(P, a, b, dev, s);
        if (rc != BMGD_OK) return rc;
    }
    {   // dWg and dWu
        P.M = g->inputs; P.N = g->hidden; P.K = (int)g->rows; P.segments = 1; P.problems = 2;
        P.out[0] = g->dw_gate; P.out[1] = g->dw_up; P.ld_out = g->hidden;
        P.vec = wide(g->dw_gate, g->hidden) && wide(g->dw_up, g->hidden);
        const Matrix a[2] = {x, x}, b[2] = {dg, du};
        rc = contract<kEpiPlain, true, true>(P, a, b, dev, s);
        if (rc != BMGD_OK) return rc;
    }
    P.M = g->hidden; P.N = g->outputs; P.problems = 1;
    P.out[0] = g->dw_down; P.ld_out = g->outputs;
    P.vec = wide(g->dw_down, g->outputs);
    const Matrix a[2] = {h, h}, b[2] = {dy, dy};
    return contract<kEpiPlain, true, true>(P, a, b, dev, s);
}

int run_pass(const bmgd_gated_ffn* g, int pass, void* workspace, int64_t workspace_bytes, void* stream) {
    int rc = check(g, pass, true);
    if (rc != BMGD_OK) return rc;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (g->rows == 0) {
        if (pass == BMGD_FFN_FORWARD) return BMGD_OK;
        if (bad_pointer(g->dw_gate) || bad_pointer(g->dw_up) || bad_pointer(g->dw_down)) return BMGD_ERR_ARG;
        const size_t wb = (size_t)g->inputs * g->hidden * 2, db = (size_t)g->hidden * g->outputs * 2;
        if (cudaMemsetAsync(g->dw_gate, 0, wb, s) != cudaSuccess || cudaMemsetAsync(g->dw_up, 0, wb, s) != cudaSuccess ||
            cudaMemsetAsync(g->dw_down, 0, db, s) != cudaSuccess) { cudaGetLastError(); return BMGD_ERR_CUDA; }
        return BMGD_OK;
    }
    Device dev{};
    Space need{nullptr, 0};
    rc = pass == BMGD_FFN_FORWARD ? forward(g, &need, false, dev, nullptr, s) : backward(g, &need, false, dev, nullptr, s);
    if (rc != BMGD_OK) return rc;
    if (!workspace || (uintptr_t)workspace % 256 != 0) return BMGD_ERR_ARG;
    if (workspace_bytes < need.used) return BMGD_ERR_CAPACITY;
    rc = current_device(&dev);
    if (rc != BMGD_OK) return rc;
    int* status = status_address();
    if (!status) return BMGD_ERR_CUDA;
    Space space{static_cast<unsigned char*>(workspace), 0};
    return pass == BMGD_FFN_FORWARD ? forward(g, &space, true, dev, status, s) : backward(g, &space, true, dev, status, s);
}

}  // namespace

extern "C" {

int bmgd_gated_ffn_workspace_bytes(const bmgd_gated_ffn* g, int32_t pass, int64_t* bytes) {
    if (!bytes) return BMGD_ERR_ARG;
    const int rc = check(g, pass, false);
    if (rc != BMGD_OK) return rc;
    Device dev{};
    Space need{nullptr, 0};
    const int r = pass == BMGD_FFN_FORWARD ? forward(g, &need, false, dev, nullptr, nullptr) : backward(g, &need, false, dev, nullptr, nullptr);
    *bytes = std::max<int64_t>(need.used, 256);
    return r;
}

int bmgd_gated_ffn_forward(const bmgd_gated_ffn* g, void* workspace, int64_t workspace_bytes, void* stream) {
    return run_pass(g, BMGD_FFN_FORWARD, workspace, workspace_bytes, stream);
}

int bmgd_gated_ffn_backward(const bmgd_gated_ffn* g, void* workspace, int64_t workspace_bytes, void* stream) {
    return run_pass(g, BMGD_FFN_BACKWARD, workspace, workspace_bytes, stream);
}

int bmgd_stream_check(void* stream) {
    if (cudaStreamSynchronize(static_cast<cudaStream_t>(stream)) != cudaSuccess) { cudaGetLastError(); return BMGD_ERR_CUDA; }
    int st[2] = {0, 0};
    if (cudaMemcpyFromSymbol(st, g_ffn_status, sizeof st) != cudaSuccess) { cudaGetLastError(); return BMGD_ERR_CUDA; }
    if (st[0] == 0) return BMGD_OK;
    const int zero[2] = {0, 0};
    cudaMemcpyToSymbol(g_ffn_status, zero, sizeof zero);
    return st[0];
}

}  // extern "C"
