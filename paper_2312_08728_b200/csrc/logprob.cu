// Host side of bmgd_log_probs and bmgd_log_probs_backward.
#include <algorithm>

#include "../../include/bmgd.h"
#include "logprob_kernel.cuh"
#include "overlap.cuh"

namespace {

using namespace bmgdk;

int launched() { return cudaGetLastError() == cudaSuccess ? BMGD_OK : BMGD_ERR_CUDA; }

// By the row's length in pieces of 16 bytes: a warp to a row up to 128, then blocks of 64 threads, or of 512 where the rows are too few to give
// every SM some.  As many blocks as an SM holds.
template <typename T, bool TOP>
int forward(const LogProbParams& P, cudaStream_t s) {
    const int64_t pieces = ((int64_t)P.C * (int64_t)sizeof(T) + 15) / 16;
    if (pieces <= 128) logprob_kernel<T, 32, TOP><<<(unsigned)std::min<int64_t>((P.rows + 7) / 8, 148 * 3), 256, 0, s>>>(P);
    else if (pieces <= 512 || P.rows > 148 * 4) logprob_kernel<T, 64, TOP><<<(unsigned)std::min<int64_t>(P.rows, 148 * 12), 64, 0, s>>>(P);
    else logprob_kernel<T, 512, TOP><<<(unsigned)std::min<int64_t>(P.rows, 148), 512, 0, s>>>(P);
    return launched();
}
// A warp to a row up to 128 pieces, else blocks of 256 threads, from 2048 pieces on 512 (8191 x 50257: 265 and 255 us), several to a row where the
// rows alone do not fill the GPU.
template <typename T>
int backward(const LogProbParams& P, cudaStream_t s) {
    const int64_t pieces = ((int64_t)P.C * (int64_t)sizeof(T) + 15) / 16;
    const unsigned rows = (unsigned)P.rows;
    const unsigned share = (unsigned)std::max<int64_t>(1, std::min<int64_t>((pieces + 1023) / 1024, 148 * 4 / P.rows));
    if (pieces <= 128) logprob_back_kernel<T, 32><<<(rows + 7) / 8, 256, 0, s>>>(P);
    else if (pieces < 2048 || share > 1) logprob_back_kernel<T, 256><<<dim3(rows, share), 256, 0, s>>>(P);
    else logprob_back_kernel<T, 512><<<rows, 512, 0, s>>>(P);
    return launched();
}

int check(const bmgd_log_probs_args* a) {
    if (!a || a->rows < 0 || a->rows > 0x7FFFFFFFll || a->C < 1 || a->C > (1 << 30) || a->type < BMGD_TYPE_F32 || a->type > BMGD_TYPE_F16) return BMGD_ERR_ARG;
    if (a->top < 0 || a->top > kMostAlternatives || a->top > a->C || a->reserved != 0) return BMGD_ERR_ARG;
    if (a->rows == 0) return BMGD_OK;
    const int eb = a->type == BMGD_TYPE_F32 ? 4 : 2;
    if (!a->logits || a->ld_logits < a->C || (uintptr_t)a->logits % eb) return BMGD_ERR_ARG;
    const uintptr_t words = (uintptr_t)a->y | (uintptr_t)a->logprob | (uintptr_t)a->entropy | (uintptr_t)a->saved | (uintptr_t)a->top_class |
                            (uintptr_t)a->top_logprob | (uintptr_t)a->dlogprob | (uintptr_t)a->dentropy;
    return words % 4 == 0 ? BMGD_OK : BMGD_ERR_ARG;
}
LogProbParams params(const bmgd_log_probs_args* a) {
    LogProbParams P{};
    P.z = a->logits; P.ld = a->ld_logits;
    P.y = a->y;
    P.logprob = a->logprob; P.entropy = a->entropy; P.saved = a->saved;
    P.index = a->top_class; P.value = a->top_logprob;
    P.dlogprob = a->dlogprob; P.dentropy = a->dentropy;
    P.dz = a->dlogits; P.ld_dz = a->ld_dlogits;
    P.rows = a->rows; P.C = a->C; P.top = a->top;
    P.far = a->rows * a->C * (a->type == BMGD_TYPE_F32 ? 4 : 2) > kFarBytes;
    return P;
}

}  // namespace

extern "C" {

int bmgd_log_probs(const bmgd_log_probs_args* a, void* stream) {
    const int rc = check(a);
    if (rc != BMGD_OK) return rc;
    if (a->rows == 0) return BMGD_OK;
    if (a->top > 0 && (!a->top_class || !a->top_logprob)) return BMGD_ERR_ARG;
    const int64_t eb = a->type == BMGD_TYPE_F32 ? 4 : 2, words = a->rows * 4;
    if (!writes_apart({vector_region(a->logprob, words), vector_region(a->entropy, words), vector_region(a->saved, words * 3), vector_region(a->top_class, words * a->top),
                       vector_region(a->top_logprob, words * a->top)}, {{a->logits, a->rows, a->C * eb, a->ld_logits * eb}, vector_region(a->y, words)})) return BMGD_ERR_ARG;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const LogProbParams P = params(a);
    const bool top = a->top > 0;
    if (a->type == BMGD_TYPE_F32) return top ? forward<float, true>(P, s) : forward<float, false>(P, s);
    if (a->type == BMGD_TYPE_BF16) return top ? forward<__nv_bfloat16, true>(P, s) : forward<__nv_bfloat16, false>(P, s);
    return top ? forward<__half, true>(P, s) : forward<__half, false>(P, s);
}

int bmgd_log_probs_backward(const bmgd_log_probs_args* a, void* stream) {
    const int rc = check(a);
    if (rc != BMGD_OK) return rc;
    if (a->rows == 0) return BMGD_OK;
    const int64_t eb = a->type == BMGD_TYPE_F32 ? 4 : 2;
    if (!a->saved || !a->dlogits || a->ld_dlogits < a->C || (uintptr_t)a->dlogits % eb) return BMGD_ERR_ARG;
    // the gradient may take the logits' place, value for value
    const int64_t words = a->rows * 4;
    if (!same_or_apart({a->dlogits, a->rows, a->C * eb, a->ld_dlogits * eb}, {a->logits, a->rows, a->C * eb, a->ld_logits * eb})) return BMGD_ERR_ARG;
    if (!writes_apart({{a->dlogits, a->rows, a->C * eb, a->ld_dlogits * eb}}, {vector_region(a->y, words), vector_region(a->saved, words * 3), vector_region(a->dlogprob, words),
                       vector_region(a->dentropy, words)})) return BMGD_ERR_ARG;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const LogProbParams P = params(a);
    if (a->type == BMGD_TYPE_F32) return backward<float>(P, s);
    if (a->type == BMGD_TYPE_BF16) return backward<__nv_bfloat16>(P, s);
    return backward<__half>(P, s);
}

}  // extern "C"
