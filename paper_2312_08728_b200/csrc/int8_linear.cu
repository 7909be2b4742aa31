// Host side of the product in 8-bit integers: checks, tensor maps, choice of tile, launches.
#include <algorithm>
#include <atomic>

#include "../../include/bmgd.h"
#include "int8_kernel.cuh"
#include "operator_host.cuh"
#include "overlap.cuh"

namespace {

using namespace bmgdk;

// A matrix of bytes as the kernels read it.
struct Bytes {
    const void* base;
    int64_t rows, cols, ld;
};

int make_map(const Bytes& m, int box_rows, CUtensorMap* out) {
    EncodeTiledFn enc = encode_tiled();
    if (!enc) return BMGD_ERR_CUDA;
    const cuuint64_t dims[2] = {(cuuint64_t)m.cols, (cuuint64_t)m.rows};
    const cuuint64_t strides[1] = {(cuuint64_t)m.ld};
    const cuuint32_t box[2] = {(cuuint32_t)kInt8BK, (cuuint32_t)box_rows};
    const cuuint32_t step[2] = {1u, 1u};
    const CUresult r = enc(out, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(m.base), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                           CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? BMGD_OK : BMGD_ERR_CUDA;
}

template <int CG, int BN>
int launch(Int8Params& P, const Bytes& q, const Bytes& w, const Device& dev, cudaStream_t s) {
    using S = Int8Shape<CG, BN>;
    int rc = make_map(q, 128, &P.q);
    if (rc == BMGD_OK) rc = make_map(w, BN / CG, &P.w);
    if (rc != BMGD_OK) return rc;
    P.tiles_m = (P.M + 128 * CG - 1) / (128 * CG);
    P.tiles_n = (P.N + BN - 1) / BN;
    P.tiles = (int64_t)P.tiles_m * P.tiles_n;
    auto* fn = int8_kernel<CG, BN>;
    static std::atomic<unsigned long long> allowed{0};
    rc = allow_smem(fn, S::kSmem, dev, allowed);
    if (rc != BMGD_OK) return rc;
    cudaLaunchConfig_t lc{};
    cudaLaunchAttribute at[2];
    launch_config(&lc, at, dim3((unsigned)std::min<int64_t>(P.tiles, dev.sms / CG) * CG), kInt8Threads, S::kSmem, CG, s);
    if (cudaLaunchKernelEx(&lc, fn, P) != cudaSuccess) { cudaGetLastError(); return BMGD_ERR_CUDA; }
    return BMGD_OK;
}

bool tma_ready(const Bytes& m) { return (uintptr_t)m.base % 16 == 0 && m.ld % 16 == 0; }

template <int NR, bool ANY>
int launch_few(Int8Params& P, const Bytes& q, const Bytes& w, int split, const Device& dev, cudaStream_t s) {
    using F = Int8FewShape<NR>;
    int rc = BMGD_OK;
    if constexpr (ANY) {
        P.q_rows = static_cast<const signed char*>(q.base); P.ld_q = q.ld;
        P.w_rows = static_cast<const signed char*>(w.base); P.ld_w = w.ld;
    } else {
        rc = make_map(q, NR, &P.q);
        if (rc == BMGD_OK) rc = make_map(w, kInt8Part, &P.w);
    }
    if (rc != BMGD_OK) return rc;
    P.tiles_m = (P.M + NR - 1) / NR;
    P.tiles_n = (P.N + kInt8Part - 1) / kInt8Part;
    auto* fn = int8_few_kernel<NR, ANY>;
    static std::atomic<unsigned long long> allowed{0};
    rc = allow_smem(fn, F::kSmem, dev, allowed);
    if (rc != BMGD_OK) return rc;
    cudaLaunchConfig_t lc{};
    cudaLaunchAttribute at[2];
    launch_config(&lc, at, dim3((unsigned)(P.tiles_m * P.tiles_n * split)), kInt8FewThreads, F::kSmem, split, s);
    if (cudaLaunchKernelEx(&lc, fn, P, split) != cudaSuccess) { cudaGetLastError(); return BMGD_ERR_CUDA; }
    return BMGD_OK;
}

// Tokens per tile and split of the contraction for the form with exchanged roles: the estimate of the 16-bit contractions, whose
// stages have the same bytes.  any: stages filled by threads, about 1.2 us each, so that single ones are worth a CTA.
struct FewChoice {
    int rows, split;
};
FewChoice choose_few(const Int8Params& P, bool any, const Device& dev) {
    const int steps = (P.K + kInt8BK - 1) / kInt8BK;
    FewChoice best{16, 1};
    double least = 1e30;
    for (int nr = 16; nr <= 128; nr *= 2) {
        if (nr > 16 && nr / 2 >= P.M) break;
        const int64_t tiles = (int64_t)((P.M + nr - 1) / nr) * ((P.N + kInt8Part - 1) / kInt8Part), slots = 2 * (int64_t)dev.sms;
        const double stage = 16384 + nr * 128, rows = (double)std::min(nr, P.M);
        for (int split : {1, 2, 3, 4, 8}) {
            if (split > 1 && (tiles * split > slots || split * (any ? 1 : 2) > steps)) break;
            const double turns = (double)((tiles * split + slots - 1) / slots);
            const double copies = std::max(turns * ((steps + split - 1) / split) * (any ? 1.2 : stage / 80e3), (double)tiles * steps * stage / 24e6);
            const double t = copies + turns * rows * (0.015 + 0.006 * (split - 1)) + (split > 1 ? 1.0 : 0.0);
            if (t < least) { least = t; best = FewChoice{nr, split}; }
        }
    }
    return best;
}

constexpr int kSms = 148;               // (the workspace's size follows from it, with or without a device)
constexpr int kVecBytes = 100 * 1024;  // of tokens in shared memory, for each of two blocks to an SM

int64_t up16(int64_t x) { return (x + 15) / 16 * 16; }

// Operands that TMA cannot read are copied, both in one launch.
int align_operands(Bytes* const (&list)[2], Space* space, bool run, cudaStream_t s) {
    Int8AlignParams A{};
    int jobs = 0;
    int64_t most = 0;
    for (Bytes* m : list) {
        if (tma_ready(*m)) continue;
        Bytes to = *m;
        to.ld = up16(m->cols);
        to.base = space->take(to.rows * to.ld);
        A.job[jobs++] = Int8AlignJob{static_cast<const signed char*>(m->base), static_cast<signed char*>(const_cast<void*>(to.base)), m->ld, to.ld, m->rows, (int)m->cols};
        most = std::max(most, to.rows * (to.ld / 16));
        *m = to;
    }
    if (!run || jobs == 0) return BMGD_OK;
    cudaLaunchConfig_t lc{};
    cudaLaunchAttribute at[2];
    launch_config(&lc, at, dim3((unsigned)std::min<int64_t>((most + 255) / 256, 148 * 8), (unsigned)jobs), 256, 0, 1, s);
    if (cudaLaunchKernelEx(&lc, int8_align_kernel<2>, A) != cudaSuccess) { cudaGetLastError(); return BMGD_ERR_CUDA; }
    return BMGD_OK;
}

int check(const bmgd_quantized_linear_args* a, bool pointers) {
    if (!a || a->rows < 0 || a->rows > 0x7FFFFF00ll || a->inputs < 1 || a->inputs > 131071 || a->outputs < 1 || a->outputs > (1 << 24)) return BMGD_ERR_ARG;
    if (a->type < BMGD_TYPE_F32 || a->type > BMGD_TYPE_F16 || a->reserved != 0) return BMGD_ERR_ARG;
    if (a->ld_codes < a->inputs || a->ld_weight < a->inputs || a->ld_y < a->outputs) return BMGD_ERR_ARG;
    if (!pointers || a->rows == 0) return BMGD_OK;
    if (!a->codes || !a->scale || !a->weight || !a->weight_scale || !a->y) return BMGD_ERR_ARG;
    if ((uintptr_t)a->scale % 4 || (uintptr_t)a->weight_scale % 4 || (uintptr_t)a->bias % 4 || (uintptr_t)a->y % (a->type == BMGD_TYPE_F32 ? 4 : 2)) return BMGD_ERR_ARG;
    const int64_t eb = a->type == BMGD_TYPE_F32 ? 4 : 2;
    const Region y{a->y, a->rows, a->outputs * eb, a->ld_y * eb};
    return writes_apart({y}, {{a->codes, a->rows, a->inputs, a->ld_codes}, {a->weight, a->outputs, a->inputs, a->ld_weight}, vector_region(a->scale, a->rows * 4),
                              vector_region(a->weight_scale, a->outputs * 4ll), vector_region(a->bias, a->outputs * 4ll)}) ? BMGD_OK : BMGD_ERR_ARG;
}

// One or two tokens: two blocks to an SM, with as many warps each (8 to 16) as let the channels come out most evenly, 2 x 148 x W of them at a
// time.  (11008 channels: 13 warps, three each; 4096: 14, one each.)
template <int M>
int launch_vec(Int8VecParams P, const Device& dev, cudaStream_t s) {
    const int blocks = 2 * dev.sms;
    int best = 8;
    if (P.N <= blocks * 8) {
        best = std::max(1, (P.N + blocks - 1) / blocks);
    } else {
        int64_t least = INT64_MAX;
        for (int w = 8; w <= 16; ++w) {
            const int64_t span = (int64_t)blocks * w, reached = (P.N + span - 1) / span * span;
            if (reached <= least) { least = reached; best = w; }
        }
    }
    const int bytes = M * ((P.K + 15) / 16) * 16;
    auto* fn = int8_vec_kernel<M>;
    if (bytes > 48 * 1024) {
        static std::atomic<unsigned long long> allowed{0};
        const int rc = allow_smem(fn, kVecBytes, dev, allowed);
        if (rc != BMGD_OK) return rc;
    }
    cudaLaunchConfig_t lc{};
    cudaLaunchAttribute at[2];
    const int grid = std::min((P.N + best - 1) / best, blocks);
    P.ahead = int8_ahead(grid * best);
    launch_config(&lc, at, dim3((unsigned)grid), best * 32, bytes, 1, s);
    if (cudaLaunchKernelEx(&lc, fn, P) != cudaSuccess) { cudaGetLastError(); return BMGD_ERR_CUDA; }
    return BMGD_OK;
}
// whether the form for one or two tokens takes it
bool few_enough(const bmgd_quantized_linear_args* a) {
    return a->rows <= 2 && (uintptr_t)a->weight % 16 == 0 && (a->ld_weight % 16 == 0 || a->outputs == 1) && a->rows * ((a->inputs + 15) / 16 * 16) <= kVecBytes;
}

// run = false: only counts the workspace
int product(const bmgd_quantized_linear_args* a, Space* space, bool run, const Device& dev, cudaStream_t s) {
    Bytes q{a->codes, a->rows, a->inputs, a->ld_codes}, w{a->weight, a->outputs, a->inputs, a->ld_weight};
    if (few_enough(a) && dev.budget_ns == 0) {  // (the others' waits are what a budget is given to test)
        if (!run) return BMGD_OK;
        const Int8VecParams V{reinterpret_cast<const signed char*>(a->codes), reinterpret_cast<const signed char*>(a->weight), a->scale, a->weight_scale, a->bias, a->y,
                              a->ld_codes, a->ld_weight, a->ld_y, a->outputs, a->inputs, a->type, 0};
        return a->rows == 1 ? launch_vec<1>(V, dev, s) : launch_vec<2>(V, dev, s);
    }
    const int64_t small = ((a->rows + 127) / 128) * ((a->outputs + 127ll) / 128);
    const bool few = a->rows <= 64 || small * 2 < kSms, ready = tma_ready(q) && tma_ready(w);
    if (!few) {
        Bytes* const operands[2] = {&q, &w};
        const int rc = align_operands(operands, space, run, s);
        if (rc != BMGD_OK) return rc;
    }
    if (!run) return BMGD_OK;
    Int8Params P{};
    P.q_scale = a->scale; P.w_scale = a->weight_scale; P.bias = a->bias;
    P.out = a->y; P.ld_out = a->ld_y;
    P.M = (int)a->rows; P.N = a->outputs; P.K = a->inputs;
    P.type = a->type;
    const int eb = a->type == BMGD_TYPE_F32 ? 4 : 2;
    P.vec = (uintptr_t)a->y % 16 == 0 && a->ld_y * eb % 16 == 0;
    P.fills = dev.fills; P.gave_up = dev.gave_up;
    P.timeout_ns = wait_bound(dev, P.K / kInt8BK);
    // Exchanged roles up to 64 tokens, and where tiles of 128 x 128 do not fill half the GPU; otherwise the tiles that take least turns, a turn of
    // 128 x 128, of 256 x 192 and of 256 x 256 for a pair being as 0.30 to 0.33 to 0.38 (microseconds for 128 inputs).  Measured on 4096 -> 11008: 128 tokens
    // 18.0 with exchanged roles, 14.4, 15.6, 17.3 with the three; 256: 23.7, 22.8, 16.0, 17.7; 512: 27.1 with the third, 24.0 with the second; 1024: 44.7, 38.5.
    if (few) {
        const FewChoice c = choose_few(P, !ready, dev);
        if (c.rows == 16) return ready ? launch_few<16, false>(P, q, w, c.split, dev, s) : launch_few<16, true>(P, q, w, c.split, dev, s);
        if (c.rows == 32) return ready ? launch_few<32, false>(P, q, w, c.split, dev, s) : launch_few<32, true>(P, q, w, c.split, dev, s);
        if (c.rows == 64) return ready ? launch_few<64, false>(P, q, w, c.split, dev, s) : launch_few<64, true>(P, q, w, c.split, dev, s);
        return ready ? launch_few<128, false>(P, q, w, c.split, dev, s) : launch_few<128, true>(P, q, w, c.split, dev, s);
    }
    const int64_t pairs = dev.sms / 2, tall = (a->rows + 255) / 256;
    auto turns = [](int64_t tiles, int64_t units) { return (double)((tiles + units - 1) / units); };
    const double t128 = 0.30 * turns(small, dev.sms), t192 = 0.33 * turns(tall * ((a->outputs + 191ll) / 192), pairs), t256 = 0.38 * turns(tall * ((a->outputs + 255ll) / 256), pairs);
    if (t128 <= t192 && t128 <= t256) return launch<1, 128>(P, q, w, dev, s);
    return t192 <= t256 ? launch<2, 192>(P, q, w, dev, s) : launch<2, 256>(P, q, w, dev, s);
}

int run_product(const bmgd_quantized_linear_args* a, void* workspace, int64_t workspace_bytes, void* stream, unsigned fills = ~0u, unsigned long long budget_ns = 0) {
    int rc = check(a, true);
    if (rc != BMGD_OK || a->rows == 0) return rc;
    Device dev{};
    dev.budget_ns = budget_ns;
    Space need{nullptr, 0};
    rc = product(a, &need, false, dev, nullptr);
    if (rc != BMGD_OK) return rc;
    if (need.used > 0 && (!workspace || (uintptr_t)workspace % 256 != 0)) return BMGD_ERR_ARG;
    if (workspace_bytes < need.used) return BMGD_ERR_CAPACITY;
    rc = current_device(&dev);
    if (rc != BMGD_OK) return rc;
    dev.fills = fills;
    dev.budget_ns = budget_ns;
    Space space{static_cast<unsigned char*>(workspace), 0};
    return product(a, &space, true, dev, static_cast<cudaStream_t>(stream));
}

}  // namespace

extern "C" {

int bmgd_quantized_linear_workspace_bytes(const bmgd_quantized_linear_args* a, int64_t* bytes) {
    if (!bytes) return BMGD_ERR_ARG;
    int rc = check(a, false);
    if (rc != BMGD_OK) return rc;
    Device dev{};
    Space need{nullptr, 0};
    rc = product(a, &need, false, dev, nullptr);
    *bytes = need.used;
    return rc;
}

int bmgd_quantized_linear(const bmgd_quantized_linear_args* a, void* workspace, int64_t workspace_bytes, void* stream) {
    return run_product(a, workspace, workspace_bytes, stream);
}

int bmgd_debug_quantized_linear_timeout(const bmgd_quantized_linear_args* a, void* workspace, int64_t workspace_bytes, int32_t fills,
                                        double budget_ms, void* stream) {
    if (fills < 0 || !(budget_ms > 0.0) || budget_ms > 1000.0) return BMGD_ERR_ARG;
    return run_product(a, workspace, workspace_bytes, stream, (unsigned)fills, (unsigned long long)(budget_ms * 1e6));
}

}  // extern "C"
