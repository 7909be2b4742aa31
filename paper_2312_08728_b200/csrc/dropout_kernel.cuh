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

constexpr int kDropAhead = 4;  // blocks of eight values that a thread has under way

// rows of `width` values; contiguous tensors come as one row.  A row's values lie in blocks (i width) / 8 to ((i + 1) width - 1) / 8,
// the first and the last of which it may share with its neighbours.
template <typename T, bool ONE_ROW>
__global__ void __launch_bounds__(256) dropout_kernel(const __grid_constant__ DropoutParams P) {
    constexpr int VE = Piece<T>::kValues, kParts = 8 / VE;
    const uint32_t step = P.step ? (uint32_t)__ldg(P.step) : 0u;
    const uint32_t k0 = (uint32_t)P.seed, k1 = (uint32_t)(P.seed >> 32);
    const long long per = ONE_ROW ? (P.width + 7) / 8 : (P.width + 7) / 8 + 1, units = ONE_ROW ? per : per * P.rows;
    const long long first = (long long)blockIdx.x * (256 * kDropAhead) + threadIdx.x;
    uint4 v[kDropAhead][kParts], r[kDropAhead][kParts];
    long long at[kDropAhead], row[kDropAhead];  // first value of the block in its row (may be negative), row
#pragma unroll
    for (int a = 0; a < kDropAhead; ++a) {
        const long long u = first + a * 256;
        row[a] = ONE_ROW ? 0 : u / per;
        const long long start = ONE_ROW ? 0 : row[a] * P.width;
        at[a] = u < units ? (start / 8 + (ONE_ROW ? u : u - row[a] * per)) * 8 - start : P.width;
        if (at[a] < 0 || at[a] + 8 > P.width) continue;
        const T* x = static_cast<const T*>(P.x) + row[a] * P.ld_x + at[a];
        const T* z = static_cast<const T*>(P.residual) + row[a] * P.ld_residual + at[a];
#pragma unroll
        for (int p = 0; p < kParts; ++p) {
            v[a][p] = load_piece(x + p * VE);
            if (P.residual) r[a][p] = load_piece(z + p * VE);
        }
    }
#pragma unroll
    for (int a = 0; a < kDropAhead; ++a) {
        if (at[a] >= P.width) continue;
        const long long block = ((ONE_ROW ? 0 : row[a] * P.width) + at[a]) / 8;
        uint32_t w[4];
        philox4x32_10((uint32_t)block, (uint32_t)(block >> 32), step, P.tag, k0, k1, w);
        auto kept = [&](int e, float x) { return ((w[e >> 1] >> (16 * (e & 1))) & 0xFFFFu) >= P.threshold ? x * P.factor : 0.f; };
        T* y = static_cast<T*>(P.y) + row[a] * P.ld_y + at[a];
        if (at[a] >= 0 && at[a] + 8 <= P.width) {
#pragma unroll
            for (int p = 0; p < kParts; ++p) {
                float x[VE], z[VE];
                unpack_piece<T>(v[a][p], x);
                if (P.residual) unpack_piece<T>(r[a][p], z);
#pragma unroll
                for (int e = 0; e < VE; ++e) x[e] = kept(p * VE + e, x[e]) + (P.residual ? z[e] : 0.f);
                store_piece(y + p * VE, pack_piece<T>(x));
            }
        } else {
            const T* x = static_cast<const T*>(P.x) + row[a] * P.ld_x + at[a];
            const T* z = static_cast<const T*>(P.residual) + row[a] * P.ld_residual + at[a];
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (at[a] + e >= 0 && at[a] + e < P.width) y[e] = from_f32<T>(kept(e, to_f32(x[e])) + (P.residual ? to_f32(z[e]) : 0.f));
        }
    }
}

}  // namespace bmgdk
