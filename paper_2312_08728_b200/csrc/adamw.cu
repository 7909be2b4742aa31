// Host side of bmgd_adamw_step: checks, the table of tensors, launches.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>

#include "../../include/bmgd.h"
#include "adamw_kernel.cuh"

namespace {

using namespace bmgdk;

constexpr int kSmallTable = 12;   // about 1 KB of kernel parameters
constexpr int kLargeTable = 360;  // just below the 32,764 bytes that a launch may take
static_assert(sizeof(AdamwTable<kLargeTable>) <= 32764, "kernel parameters");

int type_bytes(int t) { return t == BMGD_TYPE_F32 ? 4 : 2; }

struct Range { uintptr_t lo, hi; int written; };

// Tensors that an update writes must not share memory with anything else it touches.
int check_overlap(const bmgd_adamw_tensor* t, int32_t count) {
    Range* r = new (std::nothrow) Range[(size_t)count * 7];
    if (!r) return BMGD_ERR_ALLOC;
    size_t k = 0;
    auto add = [&](const void* p, int64_t bytes, int written) {
        if (p && bytes > 0) r[k++] = Range{(uintptr_t)p, (uintptr_t)p + (uintptr_t)bytes, written};
    };
    for (int32_t i = 0; i < count; ++i) {
        const bmgd_adamw_tensor& e = t[i];
        const int64_t sb = e.state_bits == 8 ? 1 : 4, blocks = (e.count + kAdamwUnit - 1) / kAdamwUnit;
        add(e.param, e.count * type_bytes(e.param_type), 1);
        add(e.grad, e.count * type_bytes(e.grad_type), 0);
        add(e.m, e.count * sb, 1);
        add(e.v, e.count * sb, 1);
        add(e.master, e.count * 4, 1);
        if (e.state_bits == 8) { add(e.m_scale, blocks, 1); add(e.v_scale, blocks, 1); }
    }
    std::sort(r, r + k, [](const Range& x, const Range& y) { return x.lo < y.lo; });
    uintptr_t top = 0, top_written = 0;
    int rc = BMGD_OK;
    for (size_t i = 0; i < k && rc == BMGD_OK; ++i) {
        if (r[i].lo < top_written || (r[i].written && r[i].lo < top)) rc = BMGD_ERR_ARG;
        top = std::max(top, r[i].hi);
        if (r[i].written) top_written = std::max(top_written, r[i].hi);
    }
    delete[] r;
    return rc;
}

bool in_unit(double x) { return x >= 0.0 && x < 1.0; }

// Sum of squares (bits = 0: all tensors), or the update of the tensors whose moments are held in `bits` bits.
template <int CAP>
int launch(const bmgd_adamw_tensor* t, int32_t count, const AdamwHead& head, int bits, int blocks, double* partial, cudaStream_t s) {
    AdamwTable<CAP>* T = new (std::nothrow) AdamwTable<CAP>;
    if (!T) return BMGD_ERR_ALLOC;
    T->h = head;
    const long long per_chunk = (long long)head.units * kAdamwUnit * (kAdamwThreads / 32);
    long long chunks = 0;
    int k = 0;
    for (int32_t i = 0; i < count; ++i) {
        const bmgd_adamw_tensor& x = t[i];
        if (x.count == 0 || (bits != 0 && x.state_bits != bits)) continue;
        AdamwEntry& e = T->e[k++];
        e.param = x.param; e.grad = x.grad; e.m = x.m; e.v = x.v;
        e.m_scale = static_cast<uint8_t*>(x.m_scale); e.v_scale = static_cast<uint8_t*>(x.v_scale);
        e.master = static_cast<float*>(x.master);
        e.n = x.count;
        e.first_chunk = chunks;
        e.keep = (float)(1.0 - head.lr * x.weight_decay);
        e.index = (uint32_t)x.index;
        e.ptype = (uint8_t)x.param_type; e.gtype = (uint8_t)x.grad_type;
        const int sb = x.state_bits == 8 ? 1 : 4;
        e.aligned = (uintptr_t)x.param % (4 * type_bytes(x.param_type)) == 0 && (uintptr_t)x.grad % (4 * type_bytes(x.grad_type)) == 0 &&
                    (uintptr_t)x.m % (4 * sb) == 0 && (uintptr_t)x.v % (4 * sb) == 0 && (uintptr_t)x.master % 16 == 0;
        chunks += (x.count + per_chunk - 1) / per_chunk;
    }
    T->h.count = k;
    T->h.chunks = chunks;
    if (k == 0) { T->h.count = 1; std::memset(&T->e[0], 0, sizeof T->e[0]); }  // nothing to update, but the step counts
    const int grid = (int)std::max<long long>(1, std::min<long long>(chunks, blocks));
    if (bits == 0) adamw_norm_kernel<CAP><<<blocks, kAdamwThreads, 0, s>>>(*T, partial);
    else if (bits == 8) adamw_kernel<CAP, 8><<<grid, kAdamwThreads, 0, s>>>(*T);
    else adamw_kernel<CAP, 32><<<grid, kAdamwThreads, 0, s>>>(*T);
    delete T;
    return cudaGetLastError() == cudaSuccess ? BMGD_OK : BMGD_ERR_CUDA;
}

}  // namespace

extern "C" {

int bmgd_adamw_step(const bmgd_adamw_tensor* tensors, int32_t count, const bmgd_adamw_config* cfg, void* dev_control,
                    void* dev_scratch, int64_t scratch_bytes, void* stream) {
    if (!cfg || !dev_control || count < 0 || (count > 0 && !tensors)) return BMGD_ERR_ARG;
    if ((uintptr_t)dev_control % 8 != 0) return BMGD_ERR_ARG;
    // (lr, the decay and the gradients' factor are fp32 in the kernel: what overflows there would be Inf)
    if (!std::isfinite((float)cfg->lr) || !in_unit(cfg->a) || !in_unit(cfg->b) || !(cfg->eps >= 0.0) || !std::isfinite(cfg->eps) ||
        !std::isfinite((float)cfg->grad_scale) || !(cfg->max_norm >= 0.0) || !std::isfinite(cfg->max_norm))
        return BMGD_ERR_ARG;
    int64_t total = 0;
    for (int32_t i = 0; i < count; ++i) {
        const bmgd_adamw_tensor& e = tensors[i];
        if (e.count < 0 || e.count > ((int64_t)1 << 40)) return BMGD_ERR_ARG;
        if (e.param_type < BMGD_TYPE_F32 || e.param_type > BMGD_TYPE_F16 || e.grad_type < BMGD_TYPE_F32 || e.grad_type > BMGD_TYPE_F16)
            return BMGD_ERR_ARG;
        if ((e.state_bits != 8 && e.state_bits != 32) || !std::isfinite((float)(cfg->lr * e.weight_decay))) return BMGD_ERR_ARG;
        if (e.count == 0) continue;
        if (!e.param || !e.grad || !e.m || !e.v || (e.state_bits == 8 && (!e.m_scale || !e.v_scale))) return BMGD_ERR_ARG;
        if ((uintptr_t)e.param % type_bytes(e.param_type) || (uintptr_t)e.grad % type_bytes(e.grad_type) || (uintptr_t)e.master % 4 ||
            (e.state_bits == 32 && ((uintptr_t)e.m % 4 || (uintptr_t)e.v % 4)))
            return BMGD_ERR_ARG;
        // fp16 has too few bits for the sum of many small steps, and no room below for random rounding: it needs the copy
        if (e.param_type == BMGD_TYPE_F16 && !e.master) return BMGD_ERR_UNIMPLEMENTED;
        if (e.param_type == BMGD_TYPE_F32 && e.master) return BMGD_ERR_ARG;
        total += e.count;
    }
    const int rc = check_overlap(tensors, count);
    if (rc != BMGD_OK) return rc;
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
        return BMGD_ERR_CUDA;
    // as many blocks as fit an SM: of the sum of squares, and of the update of moments in 32 and in 8 bits
    const int sum_blocks = std::min(kAdamwMaxBlocks, sms * 8), blocks = std::min(kAdamwMaxBlocks, sms * 3), blocks8 = std::min(kAdamwMaxBlocks, sms * 4);
    const bool clip = cfg->max_norm > 0.0;
    AdamwHead h{};
    h.control = static_cast<long long*>(dev_control);
    h.lr = cfg->lr; h.a = cfg->a; h.b = cfg->b; h.grad_scale = cfg->grad_scale; h.max_norm = cfg->max_norm;
    h.eps = std::max((float)cfg->eps, 0x1p-63f);
    h.seed_lo = (uint32_t)cfg->seed; h.seed_hi = (uint32_t)(cfg->seed >> 32);
    // a warp takes up to four units of a tensor in a row, fewer where that would leave SMs without work
    const int64_t per_unit = (int64_t)blocks * (kAdamwThreads / 32) * kAdamwUnit;
    h.units = (int)std::max<int64_t>(1, std::min<int64_t>(4, total / per_unit));
    const int launches = std::max(1, (count + kLargeTable - 1) / kLargeTable);
    const bool small = count <= kSmallTable;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    double* partial = static_cast<double*>(dev_scratch);
    auto part = [&](int l, int bits, double* sums) {
        const int32_t first = l * kLargeTable, some = std::min(count - first, kLargeTable);
        return small ? launch<kSmallTable>(tensors + first, some, h, bits, bits == 0 ? sum_blocks : bits == 8 ? blocks8 : blocks, sums, s)
                     : launch<kLargeTable>(tensors + first, some, h, bits, bits == 0 ? sum_blocks : bits == 8 ? blocks8 : blocks, sums, s);
    };
    if (clip) {
        if (!partial || (uintptr_t)partial % 8 != 0) return BMGD_ERR_ARG;
        if (scratch_bytes < (int64_t)launches * sum_blocks * 8) return BMGD_ERR_CAPACITY;
        for (int l = 0; l < launches; ++l) {
            const int e = part(l, 0, partial + (int64_t)l * sum_blocks);
            if (e != BMGD_OK) return e;
        }
        h.partial = partial;
        h.npartial = launches * sum_blocks;
    }
    int held[2] = {0, 0};  // tensors with moments in 32 and in 8 bits
    for (int32_t i = 0; i < count; ++i)
        if (tensors[i].count > 0) ++held[tensors[i].state_bits == 8];
    const int last = held[1] ? 8 : 32;  // a width without tensors is launched only where there is nothing else to count the update
    for (int bits = 32; bits >= 8; bits -= 24) {
        if (bits == 32 && !held[0] && last == 8) continue;
        if (bits == 8 && !held[1]) continue;
        for (int l = 0; l < launches; ++l) {
            h.final = bits == last && l == launches - 1;
            const int e = part(l, bits, nullptr);
            if (e != BMGD_OK) return e;
        }
    }
    return BMGD_OK;
}

}  // extern "C"
