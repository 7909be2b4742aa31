// Host side of the gated feed-forward block: checks, tensor maps, choice of tile, launches.
#include <algorithm>
#include <atomic>
#include <cstring>
#include <mutex>

#include "../../include/bmgd.h"
#include "ffn_kernel.cuh"

namespace {

using namespace bmgdk;

// Waits that ran out of time on this device, ever.  Only counted up: what bmgd_stream_check has reported is kept on the host,
// so that no report can wipe out another.
__device__ unsigned g_ffn_gave_up;

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

// What a launch needs to know of the current device.  Looked up once per device: a call of a small block takes less time on
// the GPU than these queries take on the host.
constexpr int kMaxDevices = 64;
struct Device {
    int index, sms, smem;
    unsigned* gave_up;
    unsigned fills;                // see FfnParams
    unsigned long long budget_ns;  // of any single wait inside a kernel; 0: wait_bound
};
int current_device(Device* d) {
    static Device known[kMaxDevices];
    static std::atomic<bool> ready[kMaxDevices];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); return BMGD_ERR_CUDA; }
    if (dev >= 0 && dev < kMaxDevices && ready[dev].load(std::memory_order_acquire)) { *d = known[dev]; return BMGD_OK; }
    void* p = nullptr;
    d->index = dev;
    if (cudaDeviceGetAttribute(&d->sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&d->smem, cudaDevAttrMaxSharedMemoryPerBlockOptin, dev) != cudaSuccess ||
        cudaGetSymbolAddress(&p, g_ffn_gave_up) != cudaSuccess) {
        cudaGetLastError();
        return BMGD_ERR_CUDA;
    }
    d->gave_up = static_cast<unsigned*>(p);
    d->fills = ~0u;
    d->budget_ns = 0;
    static std::mutex one;
    std::lock_guard<std::mutex> hold(one);
    if (dev >= 0 && dev < kMaxDevices && !ready[dev].load(std::memory_order_relaxed)) {
        known[dev] = *d;
        ready[dev].store(true, std::memory_order_release);
    }
    return BMGD_OK;
}
// A kernel's dynamic shared memory, allowed once per device; `done` holds a bit per device and belongs to the kernel.
template <typename K>
int allow_smem(K* fn, int bytes, const Device& dev, std::atomic<unsigned long long>& done) {
    const unsigned long long bit = 1ull << (dev.index & 63);
    if (done.load(std::memory_order_relaxed) & bit) return BMGD_OK;
    if (bytes > dev.smem) return BMGD_ERR_LAUNCH;
    if (cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) { cudaGetLastError(); return BMGD_ERR_CUDA; }
    if (dev.index < kMaxDevices) done.fetch_or(bit, std::memory_order_relaxed);
    return BMGD_OK;
}

// Bound on any single wait inside a kernel: two seconds, and more than a step of the contraction ever takes for each step.
unsigned long long wait_bound(const Device& dev, int64_t steps) { return dev.budget_ns ? dev.budget_ns : 2000000000ull + 10000ull * (unsigned long long)steps; }

// One contraction as the host describes it: out [M][N] = sum over segments of a[s] b[s].
struct Problem {
    Matrix a[2], b[2];
    void* out;
    int64_t ld_out;
    int64_t M;
    int N, K, segments;
    bool vec;
};

void launch_config(cudaLaunchConfig_t* lc, cudaLaunchAttribute (&at)[2], dim3 grid, int threads, int smem, int cluster, cudaStream_t s) {
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

template <int CG, int BN, int EPI, bool A_MN, bool B_MN>
int launch(FfnParams& P, const Problem* problems, int count, const Device& dev, cudaStream_t s) {
    using S = FfnShape<CG, BN, EPI>;
    constexpr int kCols = EPI == kEpiGated ? BN / 2 : BN;
    int64_t tiles = 0, steps = 0;
    for (int k = 0; k < count; ++k) {
        const Problem& x = problems[k];
        FfnProblem& q = P.p[k];
        steps = std::max(steps, (int64_t)x.segments * x.K / kFfnBK);
        for (int i = 0; i < 2; ++i) {
            int rc = BMGD_OK;
            if (i < x.segments) rc = make_map(x.a[i], P.type, A_MN ? 64 : 128, &q.a[i]);
            if (rc == BMGD_OK && (i < x.segments || EPI == kEpiGated)) rc = make_map(x.b[i], P.type, B_MN ? 64 : BN / CG, &q.b[i]);
            if (rc != BMGD_OK) return rc;
        }
        q.out = x.out; q.ld_out = x.ld_out;
        q.M = (int)x.M; q.N = x.N; q.K = x.K; q.segments = x.segments;
        q.vec = x.vec;
        q.tiles_m = (int)((x.M + 128 * CG - 1) / (128 * CG));
        q.tiles_n = (x.N + kCols - 1) / kCols;
        q.first_tile = tiles;
        tiles += (int64_t)q.tiles_m * q.tiles_n;
    }
    P.problems = count;
    P.tiles = tiles;
    P.timeout_ns = wait_bound(dev, steps);
    auto* fn = ffn_kernel<CG, BN, EPI, A_MN, B_MN>;
    static std::atomic<unsigned long long> allowed{0};
    const int rc = allow_smem(fn, S::kSmem, dev, allowed);
    if (rc != BMGD_OK) return rc;
    cudaLaunchConfig_t lc{};
    cudaLaunchAttribute at[2];
    launch_config(&lc, at, dim3((unsigned)std::min<int64_t>(tiles, dev.sms / CG) * CG), FfnReadOut<EPI>::kThreads, S::kSmem, CG, s);
    if (cudaLaunchKernelEx(&lc, fn, P) != cudaSuccess) { cudaGetLastError(); return BMGD_ERR_CUDA; }
    return BMGD_OK;
}

template <int NR, int EPI, bool W_MN>
int launch_few(FfnParams& P, const Problem& x, int split, bool early, const Device& dev, cudaStream_t s) {
    using F = FewShape<NR, EPI>;
    FfnProblem& q = P.p[0];
    // exchanged roles: the weights are the kernel's a
    for (int i = 0; i < 2; ++i) {
        int rc = BMGD_OK;
        if (i < x.segments || EPI == kEpiGated) rc = make_map(x.b[i], P.type, W_MN ? 64 : 128, &q.a[i]);
        if (rc == BMGD_OK && i < x.segments) rc = make_map(x.a[i], P.type, NR, &q.b[i]);
        if (rc != BMGD_OK) return rc;
    }
    q.out = x.out; q.ld_out = x.ld_out;
    q.M = (int)x.M; q.N = x.N; q.K = x.K; q.segments = x.segments;
    q.a_mn = W_MN; q.vec = x.vec;
    q.tiles_m = (int)((x.M + NR - 1) / NR);
    q.tiles_n = (x.N + kFewPart - 1) / kFewPart;
    P.timeout_ns = wait_bound(dev, (int64_t)x.segments * x.K / kFfnBK);
    auto* fn = ffn_few_kernel<NR, EPI>;
    static std::atomic<unsigned long long> allowed{0};
    const int rc = allow_smem(fn, F::kSmem, dev, allowed);
    if (rc != BMGD_OK) return rc;
    cudaLaunchConfig_t lc{};
    cudaLaunchAttribute at[2];
    launch_config(&lc, at, dim3((unsigned)(q.tiles_m * q.tiles_n * split)), kFewThreads, F::kSmem, split, s);
    if (cudaLaunchKernelEx(&lc, fn, P, split, early ? 1 : 0) != cudaSuccess) { cudaGetLastError(); return BMGD_ERR_CUDA; }
    return BMGD_OK;
}

// Rows per tile and split of the contraction for the form with exchanged roles, by an estimate in microseconds fitted to a
// sweep on B200 over rows 1 to 2000, widths 256 to 11008: a CTA takes in 80 KB a microsecond (its stages in flight over the
// latency of a copy), all of them together no more than 24 MB; reading out a row's sums takes 0.015 (backward 0.02) and
// exchanging them 0.006 (0.01) more per CTA of the cluster, a cluster about 1.  Its choice is within 3 us of the best of the
// sweep throughout; always taking 128 rows and the largest split that fits cost up to 9 us of 30 there.  (Splits of 5 to 7 were
// not part of the sweep.)
struct FewChoice {
    int rows, split;
};
template <int EPI>
FewChoice choose_few(const Problem& x, const Device& dev) {
    const double read_out = EPI == kEpiBackward ? 0.02 : 0.015, exchange = EPI == kEpiBackward ? 0.01 : 0.006;
    const int kinds = EPI == kEpiGated ? 2 : 1, steps = x.segments * ((x.K + kFfnBK - 1) / kFfnBK);
    FewChoice best{16, 1};
    double least = 1e30;
    for (int nr = 16; nr <= 128; nr *= 2) {
        if (nr > 16 && nr / 2 >= x.M) break;
        const int64_t tiles = ((x.M + nr - 1) / nr) * ((x.N + kFewPart - 1) / kFewPart), slots = 2 * (int64_t)dev.sms;
        const double stage = kinds * 16384 + nr * 128, rows = (double)std::min<int64_t>(nr, x.M) * kinds;
        for (int split : {1, 2, 3, 4, 8}) {
            if (split > 1 && (tiles * split > slots || split * 2 > steps)) break;
            const double turns = (double)((tiles * split + slots - 1) / slots);
            const double copies = std::max(turns * ((steps + split - 1) / split) * stage / 80e3, (double)tiles * steps * stage / 24e6);
            const double t = copies + turns * rows * (read_out + exchange * (split - 1)) + (split > 1 ? 1.0 : 0.0);
            if (t < least) { least = t; best = FewChoice{nr, split}; }
        }
    }
    return best;
}
template <int EPI, bool W_MN>
int contract_few(FfnParams& P, const Problem& x, bool early, const Device& dev, cudaStream_t s) {
    const FewChoice c = choose_few<EPI>(x, dev);
    if (c.rows == 16) return launch_few<16, EPI, W_MN>(P, x, c.split, early, dev, s);
    if (c.rows == 32) return launch_few<32, EPI, W_MN>(P, x, c.split, early, dev, s);
    if (c.rows == 64) return launch_few<64, EPI, W_MN>(P, x, c.split, early, dev, s);
    return launch_few<128, EPI, W_MN>(P, x, c.split, early, dev, s);
}

// Rows by weights.  The form with exchanged roles for few rows, and wherever tiles of 128 x 128 do not fill the GPU once (not
// for the gated kind, whose exchange is twice as long: 250 rows 1024 -> 4096 took 7 us more of 30 that way).  Otherwise tiles
// of 256 rows x 256 columns for two CTAs from 0.4 of them per SM on, or of 128 x 128: measured on the gated kind, 777 rows
// 504 -> 1376 (44 large tiles) 3 us more with the large ones, 300 rows 2048 -> 4096 (64) 4 us more with the small ones.
template <int EPI, bool ROWS_MN, bool W_MN>
int contract_many(FfnParams& P, const Problem* problems, int count, const Device& dev, cudaStream_t s) {
    constexpr int kCols = EPI == kEpiGated ? 128 : 256;
    int64_t large = 0;
    for (int k = 0; k < count; ++k) large += ((problems[k].M + 255) / 256) * ((problems[k].N + kCols - 1) / kCols);
    // a contraction of a few steps (the weights' gradients of few rows) is all read-out, which pairs of CTAs do not speed up:
    // one row 4096 -> 11008 -> 4096 took 11 us more of 84 with them
    const bool short_sum = problems[0].segments * (int64_t)problems[0].K <= 256;
    if (large * 5 >= dev.sms * 2 && !short_sum) return launch<2, 256, EPI, ROWS_MN, W_MN>(P, problems, count, dev, s);
    return launch<1, 128, EPI, ROWS_MN, W_MN>(P, problems, count, dev, s);
}
template <int EPI, bool W_MN>
int contract(FfnParams& P, const Problem& x, bool early, const Device& dev, cudaStream_t s) {
    const int64_t tiles = ((x.M + 127) / 128) * ((x.N + 127) / 128);
    const bool few = EPI == kEpiGated ? x.M <= 128 : x.M <= 256 || tiles <= dev.sms;
    return few ? contract_few<EPI, W_MN>(P, x, early, dev, s) : contract_many<EPI, false, W_MN>(P, &x, 1, dev, s);
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

// Operands that TMA cannot read are copied, all of them in one launch.
int align_matrices(Matrix* const* list, int count, Space* space, bool run, cudaStream_t s) {
    AlignParams P{};
    int jobs = 0;
    int64_t most = 0;
    for (int i = 0; i < count; ++i) {
        Matrix* m = list[i];
        if (tma_ready(*m)) continue;
        Matrix to = *m;
        to.ld = up8(m->cols);
        to.base = space->take(to.rows * to.ld * 2);
        P.job[jobs++] = AlignJob{static_cast<const uint16_t*>(m->base), static_cast<uint16_t*>(const_cast<void*>(to.base)), m->ld, m->rows, (int)to.ld, (int)m->cols};
        most = std::max(most, to.rows * (to.ld / 8));
        *m = to;
    }
    if (!run || jobs == 0) return BMGD_OK;
    cudaLaunchConfig_t lc{};
    cudaLaunchAttribute at[2];
    launch_config(&lc, at, dim3((unsigned)std::min<int64_t>((most + 255) / 256, 148 * 8), (unsigned)jobs), 256, 0, 1, s);
    if (cudaLaunchKernelEx(&lc, ffn_align_kernel, P) != cudaSuccess) { cudaGetLastError(); return BMGD_ERR_CUDA; }
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
    if (!g->saved_value || bad_pointer(g->dy) || (uintptr_t)g->dx % 2 != 0 || bad_pointer(g->dw_gate) || bad_pointer(g->dw_up) || bad_pointer(g->dw_down))
        return BMGD_ERR_ARG;
    return BMGD_OK;
}

bool wide(const void* p, int64_t ld) { return (uintptr_t)p % 16 == 0 && ld % 8 == 0; }

// run = false: only counts the workspace
int forward(const bmgd_gated_ffn* g, Space* space, bool run, const Device& dev, cudaStream_t s) {
    Matrix x{g->x, g->rows, g->inputs, g->ld_x}, wg{g->w_gate, g->inputs, g->hidden, g->ld_gate},
        wu{g->w_up, g->inputs, g->hidden, g->ld_up}, wd{g->w_down, g->hidden, g->outputs, g->ld_down};
    Matrix* const operands[4] = {&x, &wg, &wu, &wd};
    int rc = align_matrices(operands, 4, space, run, s);
    if (rc != BMGD_OK) return rc;
    const int64_t ldh = g->saved_hidden ? g->ld_saved : up8(g->hidden);
    void* h = g->saved_hidden ? g->saved_hidden : space->take(g->rows * ldh * 2);
    if (!run) return BMGD_OK;
    FfnParams P{};
    P.type = g->type; P.act = g->activation; P.gave_up = dev.gave_up; P.fills = dev.fills;
    P.value = g->saved_value; P.slope = g->saved_slope; P.ld_save = g->ld_saved;
    const Problem gated{{x, x}, {wg, wu}, h, ldh, g->rows, g->hidden, g->inputs, 1, true};
    rc = contract<kEpiGated, true>(P, gated, false, dev, s);
    if (rc != BMGD_OK) return rc;
    const Matrix hm{h, g->rows, g->hidden, ldh};
    const Problem down{{hm, hm}, {wd, wd}, g->y, g->ld_y, g->rows, g->outputs, g->hidden, 1, wide(g->y, g->ld_y)};
    return contract<kEpiPlain, true>(P, down, true, dev, s);
}

int backward(const bmgd_gated_ffn* g, Space* space, bool run, const Device& dev, cudaStream_t s) {
    Matrix x{g->x, g->rows, g->inputs, g->ld_x}, wg{g->w_gate, g->inputs, g->hidden, g->ld_gate},
        wu{g->w_up, g->inputs, g->hidden, g->ld_up}, wd{g->w_down, g->hidden, g->outputs, g->ld_down},
        dy{g->dy, g->rows, g->outputs, g->ld_dy};
    Matrix* const operands[5] = {&x, &wg, &wu, &wd, &dy};
    int rc = align_matrices(operands, 5, space, run, s);
    if (rc != BMGD_OK) return rc;
    const int64_t ldh = up8(g->hidden), n = g->rows;
    const Matrix h{g->saved_hidden, n, g->hidden, g->ld_saved}, dg{space->take(n * ldh * 2), n, g->hidden, ldh}, du{space->take(n * ldh * 2), n, g->hidden, ldh};
    if (!run) return BMGD_OK;
    FfnParams P{};
    P.type = g->type; P.act = g->activation; P.gave_up = dev.gave_up; P.fills = dev.fills;
    P.value = g->saved_value; P.slope = g->saved_slope; P.ld_save = g->ld_saved;
    P.out_up = const_cast<void*>(du.base);
    // dH, and from it dG and dU
    const Problem factors{{dy, dy}, {wd, wd}, const_cast<void*>(dg.base), ldh, n, g->hidden, g->outputs, 1, true};
    rc = contract<kEpiBackward, false>(P, factors, false, dev, s);
    if (rc != BMGD_OK) return rc;
    if (g->dx) {
        const Problem dx{{dg, du}, {wg, wu}, g->dx, g->inputs, n, g->inputs, g->hidden, 2, wide(g->dx, g->inputs)};
        rc = contract<kEpiPlain, false>(P, dx, true, dev, s);
        if (rc != BMGD_OK) return rc;
    }
    const Problem weights[3] = {
        {{x, x}, {dg, dg}, g->dw_gate, g->hidden, g->inputs, g->hidden, (int)n, 1, wide(g->dw_gate, g->hidden)},
        {{x, x}, {du, du}, g->dw_up, g->hidden, g->inputs, g->hidden, (int)n, 1, wide(g->dw_up, g->hidden)},
        {{h, h}, {dy, dy}, g->dw_down, g->outputs, g->hidden, g->outputs, (int)n, 1, wide(g->dw_down, g->outputs)}};
    P.early = g->dx != nullptr;  // dX and the weights' gradients need nothing of one another
    return contract_many<kEpiPlain, true, true>(P, weights, 3, dev, s);
}

int run_pass(const bmgd_gated_ffn* g, int pass, void* workspace, int64_t workspace_bytes, void* stream, unsigned fills = ~0u,
             unsigned long long budget_ns = 0) {
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
    rc = pass == BMGD_FFN_FORWARD ? forward(g, &need, false, dev, s) : backward(g, &need, false, dev, s);
    if (rc != BMGD_OK) return rc;
    if (need.used > 0 && (!workspace || (uintptr_t)workspace % 256 != 0)) return BMGD_ERR_ARG;
    if (workspace_bytes < need.used) return BMGD_ERR_CAPACITY;
    rc = current_device(&dev);
    if (rc != BMGD_OK) return rc;
    dev.fills = fills;
    dev.budget_ns = budget_ns;
    Space space{static_cast<unsigned char*>(workspace), 0};
    return pass == BMGD_FFN_FORWARD ? forward(g, &space, true, dev, s) : backward(g, &space, true, dev, s);
}

}  // namespace

extern "C" {

int bmgd_gated_ffn_workspace_bytes(const bmgd_gated_ffn* g, int32_t pass, int64_t* bytes) {
    if (!bytes) return BMGD_ERR_ARG;
    const int rc = check(g, pass, false);
    if (rc != BMGD_OK) return rc;
    Device dev{};
    Space need{nullptr, 0};
    const int r = pass == BMGD_FFN_FORWARD ? forward(g, &need, false, dev, nullptr) : backward(g, &need, false, dev, nullptr);
    *bytes = need.used;
    return r;
}

int bmgd_gated_ffn_forward(const bmgd_gated_ffn* g, void* workspace, int64_t workspace_bytes, void* stream) {
    return run_pass(g, BMGD_FFN_FORWARD, workspace, workspace_bytes, stream);
}

int bmgd_gated_ffn_backward(const bmgd_gated_ffn* g, void* workspace, int64_t workspace_bytes, void* stream) {
    return run_pass(g, BMGD_FFN_BACKWARD, workspace, workspace_bytes, stream);
}

int bmgd_debug_gated_ffn_timeout(const bmgd_gated_ffn* g, int32_t pass, void* workspace, int64_t workspace_bytes, int32_t fills,
                                 double budget_ms, void* stream) {
    if (fills < 0 || !(budget_ms > 0.0) || budget_ms > 1000.0) return BMGD_ERR_ARG;
    return run_pass(g, pass, workspace, workspace_bytes, stream, (unsigned)fills, (unsigned long long)(budget_ms * 1e6));
}

int bmgd_stream_check(void* stream) {
    static std::mutex one;
    static unsigned reported[kMaxDevices];
    Device dev{};
    const int rc = current_device(&dev);
    if (rc != BMGD_OK) return rc;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    unsigned count = 0;
    if (cudaMemcpyAsync(&count, dev.gave_up, sizeof count, cudaMemcpyDeviceToHost, s) != cudaSuccess || cudaStreamSynchronize(s) != cudaSuccess) {
        cudaGetLastError();
        return BMGD_ERR_CUDA;
    }
    std::lock_guard<std::mutex> hold(one);
    unsigned& known = reported[dev.index & (kMaxDevices - 1)];
    if ((int)(count - known) <= 0) return BMGD_OK;  // (another thread may have read, and reported, a later count)
    known = count;
    return BMGD_ERR_TIMEOUT;
}

}  // extern "C"
