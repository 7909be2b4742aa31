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

#include "shuffle.cuh"
#include "values.cuh"

namespace bmgdk {

constexpr uint32_t kDropTag = 0x44524F50u;

struct DropoutParams {
    const void *x, *residual;  // residual: null for none
    void* y;
    const long long* step;     // null: 0
    long long ld_x, ld_residual, ld_y, rows, width;
    unsigned long long seed;
    uint32_t threshold, tag;
    float factor;
};

// Rows of `width` values; contiguous tensors come as one row.  A row's values lie in blocks (i width) / 8 to ((i + 1) width - 1) / 8,
// the first and the last of which it may share with its neighbours.  AHEAD: blocks of eight values that a thread has under way.
template <typename T, bool ONE_ROW, bool RES, int AHEAD>
__global__ void __launch_bounds__(256) dropout_kernel(const __grid_constant__ DropoutParams P) {
    constexpr int VE = Piece<T>::kValues, kParts = 8 / VE;
    const uint32_t step = P.step ? (uint32_t)__ldg(P.step) : 0u;
    const uint32_t k0 = (uint32_t)P.seed, k1 = (uint32_t)(P.seed >> 32);
    const uint32_t limits = P.threshold | P.threshold << 16;
    const long long per = ONE_ROW ? (P.width + 7) / 8 : (P.width + 7) / 8 + 1, units = ONE_ROW ? per : per * P.rows;
    const long long chunk = (long long)blockIdx.x * (256 * AHEAD);
    uint4 v[AHEAD][kParts], r[AHEAD][kParts];
    const T *x[AHEAD], *z[AHEAD];
    T* y[AHEAD];
    long long block[AHEAD];
    int first[AHEAD], last[AHEAD];  // values of the block that belong to the row
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) {
        const long long u = chunk + (int)threadIdx.x + a * 256;
        long long row = 0, at = u * 8;
        block[a] = u;
        if constexpr (!ONE_ROW) {
            row = u < 0xFFFFFFFFll && per < 0xFFFFFFFFll ? (long long)((uint32_t)u / (uint32_t)per) : u / per;
            const long long start = row * P.width;
            block[a] = start / 8 + (u - row * per);
            at = block[a] * 8 - start;
        }
        first[a] = at < 0 ? (int)-at : 0;
        last[a] = u >= units ? 0 : (int)min(8ll, P.width - at);  // (may be negative)
        x[a] = static_cast<const T*>(P.x) + row * P.ld_x + at;
        z[a] = static_cast<const T*>(P.residual) + row * P.ld_residual + at;
        y[a] = static_cast<T*>(P.y) + row * P.ld_y + at;
        if (first[a] > 0 || last[a] < 8) continue;
#pragma unroll
        for (int p = 0; p < kParts; ++p) {
            v[a][p] = load_piece(x[a] + p * VE);
            if constexpr (RES) r[a][p] = load_piece(z[a] + p * VE);
        }
    }
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) {
        if (last[a] <= first[a]) continue;
        uint32_t w[4];
        philox4x32_10((uint32_t)block[a], (uint32_t)(block[a] >> 32), step, P.tag, k0, k1, w);
        bool keep[8];
#pragma unroll
        for (int e = 0; e < 8; e += 2) __vibmax_u16x2(w[e >> 1], limits, &keep[e + 1], &keep[e]);  // (both halves at once: whether a half is at least its limit)
        if (first[a] == 0 && last[a] == 8) {
#pragma unroll
            for (int p = 0; p < kParts; ++p) {
                float f[VE], g[VE];
                unpack_piece<T>(v[a][p], f);
                if constexpr (RES) unpack_piece<T>(r[a][p], g);
#pragma unroll
                for (int e = 0; e < VE; ++e) {
                    f[e] = keep[p * VE + e] ? f[e] * P.factor : 0.f;
                    if constexpr (RES) f[e] += g[e];
                }
                store_piece(y[a] + p * VE, pack_piece<T>(f));
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e >= first[a] && e < last[a]) y[a][e] = from_f32<T>((keep[e] ? to_f32(x[a][e]) * P.factor : 0.f) + (RES ? to_f32(z[a][e]) : 0.f));
        }
    }
}

}  // namespace bmgdk
