// Dropout from a counter-based generator (bmgd_dropout): the mask is drawn again wherever it is needed and stored nowhere.
//
//     y_j = residual_j + (u_j >= threshold ? x_j 65536 / (65536 - threshold) : 0),   threshold = rate 2^16 to the nearest
//
// j counts the values row by row; the eight numbers u of 16 bits of values 8 b .. 8 b + 7 are the words of one block of Philox4x32-10
// with counter (b, b >> 32, step, 'DROP' + layer) and key seed, low half first.  (The rounds' shuffle has another third word with each of its
// counters' fourth words 0 and 1, so one seed serves both.)  16 bits are enough: the factor is that of the threshold, so the mean is
// kept exactly, and a rate is met within 2^-17.  With 32 bits a value the generator would take twice the instructions.  What bounds it: memory, each value read
// and written once, with the generator's ten rounds (about 8 instructions a value) beside it.
#pragma once
#include <cstdint>
#include <cuda_runtime.h>

#include "values.cuh"

namespace bmgdk {

constexpr uint32_t kDropTag = 0x44524F50u;

struct DropoutParams {
    const void *x, *residual;  // residual: null for none
    void* y;
    const long long* step;     // null: 0
    long long ld_x, ld_residual, ld_y, rows, width;
    uint32_t key[10][2];       // of the ten rounds
    uint32_t threshold, tag;
    float factor;
};

// Which of the eight values of a block are kept.  A 32 x 32 multiplication gives both halves of its product in one instruction.
__device__ __forceinline__ void drop_block(const DropoutParams& P, long long block, uint32_t step, bool (&keep)[8]) {
    uint32_t c0 = (uint32_t)block, c1 = (uint32_t)((unsigned long long)block >> 32), c2 = step, c3 = P.tag;
    const uint32_t limit = P.threshold << 16;
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const unsigned long long a = 0xD2511F53ull * c0, b = 0xCD9E8D57ull * c2;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ P.key[r][0];
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ P.key[r][1];
        c3 = (uint32_t)a;
    }
    const uint32_t w[4] = {c0, c1, c2, c3};
#pragma unroll
    for (int e = 0; e < 4; ++e) {  // (limit: the threshold in the upper half; what stands below a number's 16 bits decides nothing)
        keep[2 * e] = w[e] << 16 >= limit;
        keep[2 * e + 1] = w[e] >= limit;
    }
}
template <typename T, bool RES, int VE>
__device__ __forceinline__ uint4 drop_piece(const uint4& v, const uint4& r, const bool* keep, float factor) {
    float f[VE], g[VE];
    unpack_piece<T>(v, f);
    if constexpr (RES) unpack_piece<T>(r, g);
#pragma unroll
    for (int e = 0; e < VE; ++e) {
        f[e] = keep[e] ? f[e] * factor : 0.f;
        if constexpr (RES) f[e] += g[e];
    }
    return pack_piece<T>(f);
}

// Contiguous tensors on 16-byte boundaries: `count` values, AHEAD blocks of eight to a thread.
template <typename T, bool RES, int AHEAD>
__global__ void __launch_bounds__(256) dropout_flat_kernel(const __grid_constant__ DropoutParams P) {
    constexpr int VE = Piece<T>::kValues, kParts = 8 / VE;
    const uint32_t step = P.step ? (uint32_t)__ldg(P.step) : 0u;
    const long long begin = (long long)blockIdx.x * (256 * AHEAD), full = P.width / 8;
    const int left = (int)min((long long)(256 * AHEAD), full - begin);  // whole blocks here (may be negative)
    const uint4* x = static_cast<const uint4*>(P.x) + begin * kParts;
    const uint4* z = static_cast<const uint4*>(P.residual) + begin * kParts;
    uint4* y = static_cast<uint4*>(P.y) + begin * kParts;
    uint4 v[AHEAD][kParts], r[AHEAD][kParts];
#pragma unroll
    for (int a = 0; a < AHEAD; ++a)
        if ((int)threadIdx.x + a * 256 < left) {
#pragma unroll
            for (int p = 0; p < kParts; ++p) {
                v[a][p] = __ldcs(x + (threadIdx.x + a * 256) * kParts + p);
                if constexpr (RES) r[a][p] = __ldcs(z + (threadIdx.x + a * 256) * kParts + p);
            }
        }
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) {
        const int u = (int)threadIdx.x + a * 256;
        bool keep[8];
        if (u < left) {
            drop_block(P, begin + u, step, keep);
#pragma unroll
            for (int p = 0; p < kParts; ++p) y[u * kParts + p] = drop_piece<T, RES, VE>(v[a][p], r[a][p], keep + p * VE, P.factor);
        } else if (begin + u == full && full * 8 < P.width) {  // the last values, fewer than eight
            drop_block(P, full, step, keep);
            const T *xs = static_cast<const T*>(P.x) + full * 8, *zs = static_cast<const T*>(P.residual) + full * 8;
            T* ys = static_cast<T*>(P.y) + full * 8;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (full * 8 + e < P.width) ys[e] = from_f32<T>((keep[e] ? to_f32(xs[e]) * P.factor : 0.f) + (RES ? to_f32(zs[e]) : 0.f));
        }
    }
}

// Rows of any stride on any boundary: a row's values lie in blocks (i width) / 8 to ((i + 1) width - 1) / 8, the first and the last of which it may share
// with its neighbours.  A thread takes a block of a row at a time.
template <typename T, bool RES>
__global__ void __launch_bounds__(256) dropout_rows_kernel(const __grid_constant__ DropoutParams P) {
    constexpr int VE = Piece<T>::kValues, kParts = 8 / VE;
    const uint32_t step = P.step ? (uint32_t)__ldg(P.step) : 0u;
    const long long per = (P.width + 7) / 8 + 1, u = (long long)blockIdx.x * 256 + threadIdx.x;
    const long long row = u < 0xFFFFFFFFll && per < 0xFFFFFFFFll ? (long long)((uint32_t)u / (uint32_t)per) : u / per;
    if (row >= P.rows) return;
    const long long start = row * P.width, block = start / 8 + (u - row * per), at = block * 8 - start;
    const int first = at < 0 ? (int)-at : 0, last = (int)min(8ll, P.width - at);  // values of the block that belong to the row
    if (last <= first) return;
    const T* x = static_cast<const T*>(P.x) + row * P.ld_x + at;
    const T* z = static_cast<const T*>(P.residual) + row * P.ld_residual + at;
    T* y = static_cast<T*>(P.y) + row * P.ld_y + at;
    const bool whole = first == 0 && last == 8;
    uint4 v[kParts], r[kParts];
    if (whole) {
#pragma unroll
        for (int p = 0; p < kParts; ++p) {
            v[p] = load_piece(x + p * VE);
            if constexpr (RES) r[p] = load_piece(z + p * VE);
        }
    }
    bool keep[8];
    drop_block(P, block, step, keep);
    if (whole) {
#pragma unroll
        for (int p = 0; p < kParts; ++p) store_piece(y + p * VE, drop_piece<T, RES, VE>(v[p], r[p], keep + p * VE, P.factor));
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e >= first && e < last) y[e] = from_f32<T>((keep[e] ? to_f32(x[e]) * P.factor : 0.f) + (RES ? to_f32(z[e]) : 0.f));
    }
}

}  // namespace bmgdk
