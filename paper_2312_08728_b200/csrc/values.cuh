// Values of the three element types in fp32 and back, and rows of them in pieces of 16 bytes.
#pragma once
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <type_traits>

#include "pair.cuh"

namespace bmgdk {

constexpr float kLog2e = 1.4426950408889634f;

template <typename T> __device__ __forceinline__ float to_f32(T x);
template <> __device__ __forceinline__ float to_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }
template <> __device__ __forceinline__ float to_f32<__half>(__half x) { return __half2float(x); }
template <typename T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_f32<__half>(float x) { return __float2half_rn(x); }

__device__ __forceinline__ float exp_fast(float x) {  // exp for x <= 0 within 2^-22 + |x| 2^-23 of itself; below 2^-126 zero
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x * kLog2e));
    return r;
}
template <typename T> struct Piece {
    static constexpr int kValues = 16 / (int)sizeof(T);
};
template <typename T>
__device__ __forceinline__ void unpack_piece(const uint4& w, float (&x)[Piece<T>::kValues]);
template <>
__device__ __forceinline__ void unpack_piece<float>(const uint4& w, float (&x)[4]) {
    x[0] = __uint_as_float(w.x); x[1] = __uint_as_float(w.y); x[2] = __uint_as_float(w.z); x[3] = __uint_as_float(w.w);
}
template <>
__device__ __forceinline__ void unpack_piece<__nv_bfloat16>(const uint4& w, float (&x)[8]) {  // (bf16 is the upper half of fp32)
    const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(v[i] << 16);
        x[2 * i + 1] = __uint_as_float(v[i] & 0xFFFF0000u);
    }
}
template <>
__device__ __forceinline__ void unpack_piece<__half>(const uint4& w, float (&x)[8]) {
    const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&v[i]));
        x[2 * i] = f.x;
        x[2 * i + 1] = f.y;
    }
}
template <typename T> __device__ __forceinline__ void put_pair(T* t, const Pair& p);
template <> __device__ __forceinline__ void put_pair<float>(float* t, const Pair& p) { const float2 x = p.both(); t[0] = x.x; t[1] = x.y; }
template <> __device__ __forceinline__ void put_pair<__nv_bfloat16>(__nv_bfloat16* t, const Pair& p) {
    *reinterpret_cast<__nv_bfloat162*>(t) = __float22bfloat162_rn(p.both());
}
template <> __device__ __forceinline__ void put_pair<__half>(__half* t, const Pair& p) { *reinterpret_cast<__half2*>(t) = __float22half2_rn(p.both()); }

// A piece at p, at once where it stands on a 16-byte boundary, value by value elsewhere.  What is read once and what is
// written for a later kernel passes the caches as data that is not wanted again.
template <typename T>
__device__ __forceinline__ uint4 load_piece(const T* p) {
    if (((uintptr_t)p & 15u) == 0) return __ldcs(reinterpret_cast<const uint4*>(p));
    uint4 w;
    T* t = reinterpret_cast<T*>(&w);
#pragma unroll
    for (int i = 0; i < Piece<T>::kValues; ++i) t[i] = p[i];
    return w;
}
// Results larger than this many bytes are written as data that is not wanted again (the gradient of 8191 x 50257 bf16 logits: 275 us to 258); smaller ones stay
// in L2 for the kernel that reads them.
constexpr long long kFarBytes = 48ll << 20;
__device__ __forceinline__ void store16(uint4* p, const uint4& w, bool far) {
    if (far) __stcs(p, w);
    else *p = w;
}
template <typename T>
__device__ __forceinline__ void store_piece(T* p, const uint4& w, bool far = false) {
    if (((uintptr_t)p & 15u) == 0) {
        store16(reinterpret_cast<uint4*>(p), w, far);
        return;
    }
    const T* t = reinterpret_cast<const T*>(&w);
#pragma unroll
    for (int i = 0; i < Piece<T>::kValues; ++i) p[i] = t[i];
}
template <typename T>
__device__ __forceinline__ uint32_t pack_pair(float a, float b) {  // two 16-bit values
    if constexpr (std::is_same<T, __half>::value) {
        const __half2 h = __floats2half2_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&h);
    } else {
        const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
}
template <typename T>
__device__ __forceinline__ uint4 pack_piece(const float (&x)[Piece<T>::kValues]) {
    if constexpr (sizeof(T) == 4) return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    else return make_uint4(pack_pair<T>(x[0], x[1]), pack_pair<T>(x[2], x[3]), pack_pair<T>(x[4], x[5]), pack_pair<T>(x[6], x[7]));
}
// How a row of `width` values at p falls into pieces: `head` values before the first 16-byte boundary, `pieces`, the rest.
// (head + rest < 2 * 16 / sizeof(T) <= 16 values, one each for the first threads.)
template <typename T>
struct RowPieces {
    int head, pieces, edges;
    __device__ __forceinline__ RowPieces(const T* p, int width) {
        head = min(width, (int)(((16u - ((uintptr_t)p & 15u)) & 15u) / sizeof(T)));
        pieces = (width - head) / Piece<T>::kValues;
        edges = width - pieces * Piece<T>::kValues;
    }
    __device__ __forceinline__ int edge(int i) const { return i < head ? i : i + pieces * Piece<T>::kValues; }  // column of edge i
    __device__ __forceinline__ int column(int piece) const { return head + piece * Piece<T>::kValues; }
};

// A value joined over the threads of a row, in a fixed order: a warp (TH = 32) or a block of TH threads.  `cells` (TH / 32
// values) is this use's own until the next barrier of the block.
enum { kJoinSum, kJoinMax };
__device__ __forceinline__ float nan_max(float a, float b) {  // NaN wins
    float m;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(a), "f"(b));
    return m;
}
template <int TH, int OP, typename V>
__device__ __forceinline__ V join_row(V v, V* cells) {
    auto op = [](V a, V b) { if constexpr (OP == kJoinSum) return a + b; else return nan_max(a, b); };
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = op(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
    if constexpr (TH > 32) {
        if ((threadIdx.x & 31) == 0) cells[threadIdx.x >> 5] = v;
        __syncthreads();
        v = cells[0];
#pragma unroll
        for (int k = 1; k < TH / 32; ++k) v = op(v, cells[k]);
    }
    return v;
}

}  // namespace bmgdk
