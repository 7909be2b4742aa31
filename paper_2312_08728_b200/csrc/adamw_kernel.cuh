// One AdamW update of many tensors in one launch (bmgd_adamw_step), and the sum of squares of their gradients.
//
// Per value, with t the number of this update, g the gradient times grad_scale and the clipping factor:
//     m <- a m + (1-a) g;   v <- b v + ((1-b) g) g
//     theta <- theta (1 - lr wd) - (lr / (1-a^t)) (m / (sqrt(v) / sqrt(1-b^t) + eps))
// Every product and sum is rounded to fp32 by itself (no contraction), so the moments do not depend on how the compiler
// schedules them, and their codes can be checked bit for bit.
//
// What bounds it: memory (200 million fp32 values: 898 us, 6.2 TB/s; bf16 with fp32 copies 929 us, 6.5 TB/s), and where moments
// have 8 bits the 77 instructions a value and the wait for a unit's loads (see adamw_unit8).  Each value of theta, the gradient and
// the moments is read once and written once.  A warp takes units of 256 consecutive values of one tensor: lane l holds values
// 4l..4l+3 and 128+4l..128+4l+3, so that every access of the warp is one contiguous piece, and the 256 values that share a scale
// in the 8-bit form sit in one warp.
//
// Moments in 8 bits.  256 consecutive values share one byte s, the biased fp32 exponent of their largest magnitude:
//   m: code in e4m3, value code * 2^(s-134): the largest magnitude lies in [128, 256) before scaling;
//   v: five exponent and three mantissa bits without a sign, value 2^((c>>3)-30) (1 + (c&7)/8) 2^(s-127), code 0 is zero.
//      v spans twice the exponents of m; 31 octaves with eight steps each are as fine as 16 steps per octave of sqrt(v).
// Powers of two as scales: scaling is exact, the only rounding is the one to the code.  That one is at random, by bits
// hashed from (seed, t, tensor, place): the change of v in one step is about 1-b of it, far below half a code step, so
// rounding to nearest would leave v where it is for ever (and the step length wrong by a factor), while random
// rounding keeps the mean.  A nonzero v below the smallest code becomes that code, not zero: theta must never be
// divided by eps alone where m has a value.  theta in bf16 without an fp32 copy is rounded at random for the same
// reason: lr times one step is mostly below half a bf16 step.
#pragma once
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>

#include "pair.cuh"

namespace bmgdk {

constexpr int kAdamwThreads = 256;
constexpr int kAdamwUnit = 256;        // values a warp holds at a time; values that share a scale
constexpr int kAdamwMaxBlocks = 1184;  // blocks of the sum of squares: partial sums in the scratch

enum { kTypeF32 = 0, kTypeBF16 = 1, kTypeF16 = 2 };

struct AdamwEntry {
    void* param;
    const void* grad;
    void* m;
    void* v;
    uint8_t* m_scale;
    uint8_t* v_scale;
    float* master;
    long long n;
    long long first_chunk;  // chunks of all entries before this one
    float keep;             // 1 - lr wd
    uint32_t index;         // place of the tensor in the caller's list: part of the random key
    uint8_t ptype, gtype, aligned;
};

struct AdamwHead {
    long long* control;   // [0] updates taken, [1] updates left out, [2] blocks that have finished, [3] norm (fp64 bits)
    const double* partial;
    int npartial;         // partial sums of squares; 0: no clipping
    int count;
    long long chunks;
    int units;            // units a warp takes per chunk
    int final;            // the last launch of the update: counts it
    double lr, a, b, grad_scale, max_norm;
    float eps;
    uint32_t seed_lo, seed_hi;
};

template <int CAP>
struct AdamwTable {
    AdamwHead h;
    AdamwEntry e[CAP];
};

// 32-bit mixing function (two xor-shift-multiply rounds; Appleby's published finaliser)
__host__ __device__ __forceinline__ uint32_t mix32(uint32_t x) {
    x ^= x >> 16; x *= 0x85EBCA6Bu;
    x ^= x >> 13; x *= 0xC2B2AE35u;
    return x ^ (x >> 16);
}

template <int CAP>
__device__ __forceinline__ int adamw_find(const AdamwTable<CAP>& T, long long chunk) {
    int lo = 0, hi = T.h.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (T.e[mid].first_chunk <= chunk) lo = mid; else hi = mid - 1;
    }
    return lo;
}

__device__ __forceinline__ float2 unpack_bf16(uint32_t w) {
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}
__device__ __forceinline__ float2 unpack_f16(uint32_t w) {
    return __half22float2(*reinterpret_cast<__half2*>(&w));
}

// four consecutive values from `at` on; values from `n` on read as zero
__device__ __forceinline__ float4 load4(const void* base, int type, long long at, long long n, bool aligned) {
    if (aligned && at + 4 <= n) {
        if (type == kTypeF32) return __ldcs(reinterpret_cast<const float4*>(static_cast<const float*>(base) + at));
        const uint2 w = __ldcs(reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(base) + at));
        const float2 lo = type == kTypeBF16 ? unpack_bf16(w.x) : unpack_f16(w.x);
        const float2 hi = type == kTypeBF16 ? unpack_bf16(w.y) : unpack_f16(w.y);
        return make_float4(lo.x, lo.y, hi.x, hi.y);
    }
    float x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[i] = 0.f;
        if (at + i < n)
            x[i] = type == kTypeF32    ? static_cast<const float*>(base)[at + i]
                   : type == kTypeBF16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(base)[at + i])
                                       : __half2float(static_cast<const __half*>(base)[at + i]);
    }
    return make_float4(x[0], x[1], x[2], x[3]);
}
__device__ __forceinline__ void store4(void* base, int type, long long at, long long n, bool aligned, const float (&x)[4]) {
    if (aligned && at + 4 <= n) {
        if (type == kTypeF32) {
            __stcs(reinterpret_cast<float4*>(static_cast<float*>(base) + at), make_float4(x[0], x[1], x[2], x[3]));
        } else {
            uint2 w;
            if (type == kTypeBF16) {
                const __nv_bfloat162 a = __floats2bfloat162_rn(x[0], x[1]), b = __floats2bfloat162_rn(x[2], x[3]);
                w = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
            } else {
                const __half2 a = __floats2half2_rn(x[0], x[1]), b = __floats2half2_rn(x[2], x[3]);
                w = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
            }
            __stcs(reinterpret_cast<uint2*>(static_cast<uint16_t*>(base) + at), w);
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (at + i >= n) break;
        if (type == kTypeF32) static_cast<float*>(base)[at + i] = x[i];
        else if (type == kTypeBF16) static_cast<__nv_bfloat16*>(base)[at + i] = __float2bfloat16_rn(x[i]);
        else static_cast<__half*>(base)[at + i] = __float2half_rn(x[i]);
    }
}
__device__ __forceinline__ uint32_t load_codes(const void* base, long long at, long long n, bool aligned) {
    const uint8_t* p = static_cast<const uint8_t*>(base);
    if (aligned && at + 4 <= n) return __ldcs(reinterpret_cast<const uint32_t*>(p + at));
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (at + i < n) w |= (uint32_t)p[at + i] << (8 * i);
    return w;
}
__device__ __forceinline__ void store_codes(void* base, long long at, long long n, bool aligned, uint32_t w) {
    uint8_t* p = static_cast<uint8_t*>(base);
    if (aligned && at + 4 <= n) { __stcs(reinterpret_cast<uint32_t*>(p + at), w); return; }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (at + i < n) p[at + i] = (uint8_t)(w >> (8 * i));
}

__device__ __forceinline__ float power_of_two(int biased) { return __uint_as_float((uint32_t)biased << 23); }
__device__ __forceinline__ bool finite_bits(uint32_t b) { return (b & 0x7F800000u) != 0x7F800000u; }

// ---- codes of 8 bits, four to a word
// e4m3 values before scaling, by way of fp16, which holds all of them (0x7F and 0xFF give NaN)
__device__ __forceinline__ void decode_m4(uint32_t w, float (&x)[4]) {
    const __half2_raw lo = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w & 0xFFFFu), __NV_E4M3);
    const __half2_raw hi = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w >> 16), __NV_E4M3);
    const float2 a = __half22float2(__half2(lo)), b = __half22float2(__half2(hi));
    x[0] = a.x; x[1] = a.y; x[2] = b.x; x[3] = b.y;
}
// x scaled to |x| < 256 and finite.  From 2^-6 on the upper bits of x count code steps, 2^20 units of the last place each;
// below, steps are 2^-9 throughout, which the last places of |x| + 2^-6 count.  Rounding that sum towards zero is exact for the
// purpose: the draw has 16 bits, so every threshold is a multiple of 16 units.
__device__ __forceinline__ uint32_t encode_m(float x, uint32_t r16) {
    const uint32_t mag = __float_as_uint(x) & 0x7FFFFFFFu;
    const uint32_t low = __float_as_uint(__fadd_rz(__uint_as_float(mag), 0x1p-6f)) - (121u << 23);
    const uint32_t y = mag >= (121u << 23) ? mag - (120u << 23) : low;
    return ((y + (r16 << 4)) >> 20) | ((__float_as_uint(x) >> 24) & 0x80u);
}
__device__ __forceinline__ void decode_v4(uint32_t w, int s, float (&x)[4]) {
    const uint32_t base = (uint32_t)(s - 30) << 23;  // exponent and mantissa bits of a code are those of the value, shifted
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t c = (w >> (8 * i)) & 0xFFu;
        x[i] = c == 0u ? 0.f : __uint_as_float((c << 20) + base);
    }
    if (__vcmpeq4(w, 0xFFFFFFFFu)) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (((w >> (8 * i)) & 0xFFu) == 0xFFu) x[i] = __uint_as_float(0x7FC00000u);
    }
}
__device__ __forceinline__ uint32_t encode_v(float v, int s, uint32_t r16) {  // v finite
    const int y = (int)(__float_as_uint(v) - ((uint32_t)(s - 30) << 23) + (r16 << 4));
    return v == 0.f ? 0u : (uint32_t)max(y >> 20, 1);
}

// x^n for an integer n >= 0
__device__ __forceinline__ double int_pow(double x, long long n) {
    double r = 1.0;
    while (n > 0) {
        if (n & 1) r *= x;
        x *= x;
        n >>= 1;
    }
    return r;
}

// ---------------------------------------------------------------- sum of squares of all gradients
// Every block sums its chunks in fp64 (a square of an fp32 value cannot overflow there, and the order of the sum does not
// show in the fp32 clipping factor); the partial sums are added in a fixed order by the update's blocks.
template <int CAP>
__global__ void __launch_bounds__(kAdamwThreads) adamw_norm_kernel(const __grid_constant__ AdamwTable<CAP> T, double* partial) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    double sum = 0.0;
    for (long long chunk = blockIdx.x; chunk < T.h.chunks; chunk += gridDim.x) {
        const AdamwEntry& e = T.e[adamw_find(T, chunk)];
        const long long unit0 = ((chunk - e.first_chunk) * (kAdamwThreads / 32) + warp) * T.h.units;
        for (int u = 0; u < T.h.units; ++u) {
            const long long at = (unit0 + u) * kAdamwUnit + lane * 4;
            if ((unit0 + u) * kAdamwUnit >= e.n) break;
            const float4 x = load4(e.grad, e.gtype, at, e.n, e.aligned), y = load4(e.grad, e.gtype, at + 128, e.n, e.aligned);
            const float g[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
#pragma unroll
            for (int i = 0; i < 8; ++i) { const double d = (double)g[i]; sum = fma(d, d, sum); }
        }
    }
    __shared__ double part[kAdamwThreads / 32];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
    if (lane == 0) part[warp] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        double s = 0.0;
        for (int w = 0; w < kAdamwThreads / 32; ++w) s += part[w];
        partial[blockIdx.x] = s;
    }
}

// ---------------------------------------------------------------- the update
// m / (sqrt(v) root + eps) with the root and the reciprocal each within 2^-23 of their values: they move theta by lr at most, and
// the exact forms cost as many instructions as the rest of the formula.  The square root takes subnormal v for what they are: in
// the first updates root = 1 / sqrt(1-b^t) is 30 or more, and sqrt(v) root counts beside the smallest eps (2^-63) although v is below
// 2^-126.  The sum is at least 2^-63, so the reciprocal needs no subnormals.
__device__ __forceinline__ float sqrt_near(float x) {
    float r;
    asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// the same for x = 0 or x >= 2^-126, with fewer instructions (about 3 % of the update with moments in 8 bits)
__device__ __forceinline__ float sqrt_normal(float x) {
    float r;
    asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float reciprocal_near(float x) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

struct AdamwFactors {
    float gscale, step, root, a, a1, b, b1, eps;
    int fine;
    uint32_t key;
    double norm;
};

template <int TYPE> __device__ __forceinline__ void load4_wide(const void* base, long long at, float (&x)[4]) {
    const float4 v = load4(base, TYPE, at, at + 4, true);
    x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
}
template <int TYPE, bool WIDE> __device__ __forceinline__ void load4_any(const void* base, long long at, long long n, float (&x)[4]) {
    if constexpr (WIDE) { load4_wide<TYPE>(base, at, x); return; }
    const float4 v = load4(base, TYPE, at, n, false);
    x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
}

// One unit of a tensor.  WIDE: it lies within the tensor and every array allows vector accesses.  (Other units, and those with
// infinities or NaN where moments have 8 bits, are few: their code is kept out of the way.)
template <int PT, bool MASTER, int GT, int BITS, bool WIDE>
__device__ __forceinline__ void adamw_unit_body(const AdamwEntry& e, long long unit, int lane, const AdamwFactors& F, float keep, uint32_t key) {
    const long long n = e.n;
    const long long at[2] = {unit * kAdamwUnit + lane * 4, unit * kAdamwUnit + lane * 4 + 128};
    constexpr bool kRandomTheta = PT == kTypeBF16 && !MASTER;
    float p[2][4], g[2][4], m[2][4], v[2][4];
    uint32_t cm[2], cv[2];
    int sm = 0, sv = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        load4_any<GT, WIDE>(e.grad, at[h], n, g[h]);
        if constexpr (MASTER) load4_any<kTypeF32, WIDE>(e.master, at[h], n, p[h]);
        else load4_any<PT, WIDE>(e.param, at[h], n, p[h]);
        if constexpr (BITS == 8) {
            cm[h] = load_codes(e.m, at[h], n, WIDE);
            cv[h] = load_codes(e.v, at[h], n, WIDE);
        } else {
            load4_any<kTypeF32, WIDE>(e.m, at[h], n, m[h]);
            load4_any<kTypeF32, WIDE>(e.v, at[h], n, v[h]);
        }
    }
    if constexpr (BITS == 8) {
        sm = e.m_scale[unit];
        sv = e.v_scale[unit];
        const float unscale = power_of_two(sm - 7);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            decode_m4(cm[h], m[h]);
            decode_v4(cv[h], sv, v[h]);
#pragma unroll
            for (int i = 0; i < 4; ++i) m[h][i] *= unscale;
        }
    }
    uint32_t top_m = 0, top_v = 0;  // largest magnitudes of the new moments, infinities and NaN among them
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float gi = __fmul_rn(g[h][i], F.gscale);
            m[h][i] = __fadd_rn(__fmul_rn(m[h][i], F.a), __fmul_rn(gi, F.a1));
            v[h][i] = __fadd_rn(__fmul_rn(v[h][i], F.b), __fmul_rn(__fmul_rn(gi, F.b1), gi));
            const float denom = __fadd_rn(__fmul_rn(sqrt_near(v[h][i]), F.root), F.eps);
            p[h][i] = __fsub_rn(__fmul_rn(p[h][i], keep), __fmul_rn(__fmul_rn(m[h][i], reciprocal_near(denom)), F.step));
            if constexpr (BITS == 8) {
                top_m = max(top_m, __float_as_uint(m[h][i]) & 0x7FFFFFFFu);
                top_v = max(top_v, __float_as_uint(v[h][i]) & 0x7FFFFFFFu);
            }
        }
    }
    // the unit starts at a multiple of 256, so all its places share the upper 32 bits
    const uint32_t k = key + (uint32_t)((unsigned long long)at[0] >> 32) * 0x85EBCA6Bu;
    uint32_t wm[2] = {0, 0}, wv[2] = {0, 0};
    if constexpr (BITS == 8) {
        top_m = __reduce_max_sync(0xFFFFFFFFu, top_m);
        top_v = __reduce_max_sync(0xFFFFFFFFu, top_v);
        if (max(top_m, top_v) >= 0x7F800000u) {  // some value is infinite or NaN: the scales go by the others
            top_m = top_v = 0;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t bm = __float_as_uint(m[h][i]) & 0x7FFFFFFFu, bv = __float_as_uint(v[h][i]) & 0x7FFFFFFFu;
                    if (bm < 0x7F800000u) top_m = max(top_m, bm);
                    else { wm[h] |= 0xFFu << (8 * i); m[h][i] = 0.f; }  // the code of NaN
                    if (bv < 0x7F800000u) top_v = max(top_v, bv);
                    else { wv[h] |= 0xFFu << (8 * i); v[h][i] = 0.f; }
                }
            top_m = __reduce_max_sync(0xFFFFFFFFu, top_m);
            top_v = __reduce_max_sync(0xFFFFFFFFu, top_v);
        }
        sm = max((int)(top_m >> 23), 16);
        sv = max((int)(top_v >> 23), 40);
    }
    const float scale = power_of_two(261 - sm);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        if constexpr (BITS == 32) {
            store4(e.m, kTypeF32, at[h], n, WIDE, m[h]);
            store4(e.v, kTypeF32, at[h], n, WIDE, v[h]);
        }
        if constexpr (MASTER) store4(e.master, kTypeF32, at[h], n, WIDE, p[h]);
        if constexpr (BITS == 8 || kRandomTheta) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t r = mix32(((uint32_t)at[h] + i) ^ k);
                if constexpr (BITS == 8) {
                    wm[h] |= encode_m(m[h][i] * scale, r & 0xFFFFu) << (8 * i);
                    wv[h] |= encode_v(v[h][i], sv, r >> 16) << (8 * i);
                }
                if constexpr (kRandomTheta) {
                    const uint32_t b = __float_as_uint(p[h][i]);
                    const uint32_t up = (b + (mix32(r ^ 0x9E3779B9u) & 0xFFFFu)) & 0xFFFF0000u;
                    if (finite_bits(b)) p[h][i] = __uint_as_float(up);
                }
            }
        }
        if constexpr (BITS == 8) {
            store_codes(e.m, at[h], n, WIDE, wm[h]);
            store_codes(e.v, at[h], n, WIDE, wv[h]);
        }
        store4(e.param, PT, at[h], n, WIDE, p[h]);
    }
    if (BITS == 8 && lane == 0) { e.m_scale[unit] = (uint8_t)sm; e.v_scale[unit] = (uint8_t)sv; }
}

template <int PT, bool MASTER, int GT, int BITS>
__device__ __noinline__ void adamw_unit_any(const AdamwEntry& e, long long unit, int lane, const AdamwFactors& F, float keep, uint32_t key) {
    adamw_unit_body<PT, MASTER, GT, BITS, false>(e, unit, lane, F, keep, key);
}

// largest magnitude and smallest value of three; NaN wins the first
__device__ __forceinline__ float top3(float a, float b, float c) {
    float r;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ float low3(float a, float b, float c) {
    float r;
    asm("min.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
// the uppermost bytes of four words, in order
__device__ __forceinline__ uint32_t top_bytes(const uint32_t (&x)[4]) {
    return __byte_perm(__byte_perm(x[0], x[1], 0x0073), __byte_perm(x[2], x[3], 0x0073), 0x5410);
}

// A full unit with moments in 8 bits.  Instructions and the latency of a unit's loads bound this form, not memory (200 million
// values in bf16: 1079 us value by value, 741 in this way with three blocks to an SM, 664 with four, whose 64 registers
// spill 132 bytes over all combinations of types; their traffic needs 310; issue slots 56 % and memory 28 % busy),
// hence: two values to an instruction wherever the formula allows; the largest and
// smallest of several values in one; four codes at a time through bytes.
// A code is the upper bits of y, the value's exponent and mantissa counted from the format's smallest, plus the draw: for m
// y is the larger of the magnitude's bits and those of (magnitude + 2^-6) less 2^23, which count in constant steps below
// 2^-6 (there the second is the larger, above it the first); for v it is at least one code.  y * 16 + draw * 256 then has the code
// in its uppermost byte, for m plus 0xC0 (120 << 23, times 16), which (b ^ 0xC0) & 0x7F takes off.
template <int PT, bool MASTER, int GT>
__device__ __forceinline__ void adamw_unit8(const AdamwEntry& e, long long unit, int lane, const AdamwFactors& F, float keep, uint32_t key) {
    const long long at = unit * kAdamwUnit + lane * 4;
    constexpr bool kRandomTheta = PT == kTypeBF16 && !MASTER;
    float p[8], g[8], m[8], v[8];
    uint32_t cm[2], cv[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        load4_wide<GT>(e.grad, at + 128 * h, *reinterpret_cast<float(*)[4]>(g + 4 * h));
        if constexpr (MASTER) load4_wide<kTypeF32>(e.master, at + 128 * h, *reinterpret_cast<float(*)[4]>(p + 4 * h));
        else load4_wide<PT>(e.param, at + 128 * h, *reinterpret_cast<float(*)[4]>(p + 4 * h));
        cm[h] = load_codes(e.m, at + 128 * h, e.n, true);
        cv[h] = load_codes(e.v, at + 128 * h, e.n, true);
    }
    const int old_m = e.m_scale[unit], old_v = e.v_scale[unit];
    const uint32_t base = (uint32_t)(old_v - 30) << 23;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        decode_m4(cm[h], *reinterpret_cast<float(*)[4]>(m + 4 * h));
#pragma unroll
        for (int i = 0; i < 4; ++i) v[4 * h + i] = __uint_as_float(__byte_perm(cv[h], 0, 0x4440 + i) * (1u << 20) + base);
        // a byte of zeros (no moment yet) or of ones (NaN) among the four
        if (((cv[h] - 0x01010101u) & ~cv[h] & 0x80808080u) | ((~cv[h] - 0x01010101u) & cv[h] & 0x80808080u)) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t c = (cv[h] >> (8 * i)) & 0xFFu;
                if (c == 0u) v[4 * h + i] = 0.f;
                if (c == 0xFFu) v[4 * h + i] = __uint_as_float(0x7FC00000u);
            }
        }
    }
    const Pair unscale(power_of_two(old_m - 7)), gscale(F.gscale), a(F.a), a1(F.a1), b(F.b), b1(F.b1), root(F.root), eps(F.eps), kept(keep), step(-F.step);
    float top_m = 0.f, top_v = 0.f, top_p = 0.f, low_v = __uint_as_float(0x7F7FFFFFu);
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        // (the sums one by one: a sum of products in pairs comes out as one rounding, and the moments' codes are defined by two)
        const Pair gi = Pair(g[i], g[i + 1]) * gscale;
        const float2 ma = ((Pair(m[i], m[i + 1]) * unscale) * a).both(), mb = (gi * a1).both();
        const float2 va = (Pair(v[i], v[i + 1]) * b).both(), vb = ((gi * b1) * gi).both();
        const Pair mi(__fadd_rn(ma.x, mb.x), __fadd_rn(ma.y, mb.y));
        const float2 vi = make_float2(__fadd_rn(va.x, vb.x), __fadd_rn(va.y, vb.y));
        const float2 denom = (Pair(sqrt_normal(vi.x), sqrt_normal(vi.y)) * root + eps).both();
        const Pair quotient = mi * Pair(reciprocal_near(denom.x), reciprocal_near(denom.y));
        const float2 pi = (Pair(p[i], p[i + 1]) * kept + quotient * step).both(), mm = mi.both();
        m[i] = mm.x; m[i + 1] = mm.y;
        v[i] = vi.x; v[i + 1] = vi.y;
        p[i] = pi.x; p[i + 1] = pi.y;
        top_m = top3(top_m, mm.x, mm.y);
        top_v = top3(top_v, vi.x, vi.y);
        top_p = top3(top_p, pi.x, pi.y);
        low_v = low3(low_v, vi.x, vi.y);
    }
    // infinities, NaN and subnormal v are the other form's; nothing has been written yet
    if (__any_sync(0xFFFFFFFFu, !(top3(top_m, top_v, top_p) < INFINITY) || low_v < 0x1p-126f)) {
        bool other = !(top3(top_m, top_v, top_p) < INFINITY);
#pragma unroll
        for (int i = 0; i < 8; ++i) other = other || (v[i] > 0.f && v[i] < 0x1p-126f);
        if (__any_sync(0xFFFFFFFFu, other)) {
            adamw_unit_any<PT, MASTER, GT, 8>(e, unit, lane, F, keep, key);
            return;
        }
    }
    const int new_m = max((int)(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(top_m)) >> 23), 16);
    const int new_v = max((int)(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(top_v)) >> 23), 40);
    const Pair scale(power_of_two(261 - new_m));
    const uint32_t from = (uint32_t)(new_v - 30) << 23;
    const uint32_t k = key + (uint32_t)((unsigned long long)at >> 32) * 0x85EBCA6Bu;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t place = (uint32_t)(at + 128 * h) ^ k;  // (a multiple of four before the key: i sets its lowest bits)
        uint32_t xm[4], um[4], uv[4], theta[4];
#pragma unroll
        for (int i = 0; i < 4; i += 2) {
            const float2 x = (Pair(m[4 * h + i], m[4 * h + i + 1]) * scale).both();
            xm[i] = __float_as_uint(x.x);
            xm[i + 1] = __float_as_uint(x.y);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t r = mix32(place ^ (uint32_t)i), mag = xm[i] & 0x7FFFFFFFu;
            const uint32_t small = __float_as_uint(__fadd_rz(__uint_as_float(mag), 0x1p-6f)) - (1u << 23);
            um[i] = max(mag, small) * 16u + __byte_perm(r, 0, 0x4104);
            uv[i] = (uint32_t)max((int)(__float_as_uint(v[4 * h + i]) - from), 1 << 20) * 16u + __byte_perm(r, 0, 0x4324);
            if constexpr (kRandomTheta) theta[i] = __float_as_uint(p[4 * h + i]) + (mix32(r ^ 0x9E3779B9u) & 0xFFFFu);
        }
        uint32_t wv = top_bytes(uv);
        if (low_v == 0.f) {  // (v is never negative)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (v[4 * h + i] == 0.f) wv &= ~(0xFFu << (8 * i));
        }
        store_codes(e.m, at + 128 * h, e.n, true, ((top_bytes(um) ^ 0xC0C0C0C0u) & 0x7F7F7F7Fu) | (top_bytes(xm) & 0x80808080u));
        store_codes(e.v, at + 128 * h, e.n, true, wv);
        if constexpr (MASTER) store4(e.master, kTypeF32, at + 128 * h, e.n, true, *reinterpret_cast<float(*)[4]>(p + 4 * h));
        if constexpr (kRandomTheta)
            __stcs(reinterpret_cast<uint2*>(static_cast<uint16_t*>(e.param) + at + 128 * h),
                   make_uint2(__byte_perm(theta[0], theta[1], 0x7632), __byte_perm(theta[2], theta[3], 0x7632)));
        else store4(e.param, PT, at + 128 * h, e.n, true, *reinterpret_cast<float(*)[4]>(p + 4 * h));
    }
    if (lane == 0) { e.m_scale[unit] = (uint8_t)new_m; e.v_scale[unit] = (uint8_t)new_v; }
}

template <int PT, bool MASTER, int GT, int BITS>
__device__ __forceinline__ void adamw_units(const AdamwEntry& e, long long unit0, int units, int lane, const AdamwFactors& F, uint32_t key) {
    const float keep = e.keep;
    for (int u = 0; u < units; ++u) {
        const long long unit = unit0 + u;
        if (unit * kAdamwUnit >= e.n) break;
        if (e.aligned && (unit + 1) * kAdamwUnit <= e.n) {
            if constexpr (BITS == 8) adamw_unit8<PT, MASTER, GT>(e, unit, lane, F, keep, key);
            else adamw_unit_body<PT, MASTER, GT, BITS, true>(e, unit, lane, F, keep, key);
        } else {
            adamw_unit_any<PT, MASTER, GT, BITS>(e, unit, lane, F, keep, key);
        }
    }
}

// BITS: how the moments of all tensors of this launch are held.  Their types differ from tensor to tensor; the code for
// each combination is chosen once for a warp's units.
template <int CAP, int BITS>
__global__ void __launch_bounds__(kAdamwThreads, BITS == 8 ? 4 : 3) adamw_kernel(const __grid_constant__ AdamwTable<CAP> T) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    __shared__ AdamwFactors shared_factors;
    __shared__ double part[kAdamwThreads / 32];
    if (T.h.npartial > 0) {
        double s = 0.0;
        for (int i = threadIdx.x; i < T.h.npartial; i += kAdamwThreads) s += T.h.partial[i];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
        if (lane == 0) part[warp] = s;
        __syncthreads();
    }
    if (threadIdx.x == 0) {
        AdamwFactors& F = shared_factors;
        const long long t = T.h.control[0] + 1;
        double scale = T.h.grad_scale;
        F.fine = 1;
        F.norm = 0.0;
        if (T.h.npartial > 0) {
            double s = 0.0;
            for (int w = 0; w < kAdamwThreads / 32; ++w) s += part[w];
            const double norm = sqrt(s) * fabs(T.h.grad_scale);
            F.norm = norm;
            F.fine = isfinite(norm) ? 1 : 0;
            scale *= fmin(T.h.max_norm / (norm + 1e-6), 1.0);
        }
        const double c1 = 1.0 - int_pow(T.h.a, t), c2 = 1.0 - int_pow(T.h.b, t);
        F.gscale = (float)scale;
        F.step = (float)(T.h.lr / c1);
        F.root = (float)(1.0 / sqrt(c2));
        F.a = (float)T.h.a; F.a1 = (float)(1.0 - T.h.a);
        F.b = (float)T.h.b; F.b1 = (float)(1.0 - T.h.b);
        F.eps = T.h.eps;
        F.key = mix32(T.h.seed_lo + (uint32_t)t * 0x9E3779B9u);
    }
    __syncthreads();
    const AdamwFactors& F = shared_factors;
    if (F.fine) {
        for (long long chunk = blockIdx.x; chunk < T.h.chunks; chunk += gridDim.x) {
            const AdamwEntry& e = T.e[adamw_find(T, chunk)];
            const uint32_t key = mix32(F.key ^ (T.h.seed_hi + e.index * 0x9E3779B9u));
            const long long unit0 = ((chunk - e.first_chunk) * (kAdamwThreads / 32) + warp) * T.h.units;
            const int units = T.h.units;
#define BMGD_ADAMW_GRADS(PT, MASTER)                                                                          \
    if (e.gtype == kTypeF32) adamw_units<PT, MASTER, kTypeF32, BITS>(e, unit0, units, lane, F, key);          \
    else if (e.gtype == kTypeBF16) adamw_units<PT, MASTER, kTypeBF16, BITS>(e, unit0, units, lane, F, key);   \
    else adamw_units<PT, MASTER, kTypeF16, BITS>(e, unit0, units, lane, F, key)
            if (e.ptype == kTypeF32) { BMGD_ADAMW_GRADS(kTypeF32, false); }
            else if (e.ptype == kTypeF16) { BMGD_ADAMW_GRADS(kTypeF16, true); }
            else if (e.master) { BMGD_ADAMW_GRADS(kTypeBF16, true); }
            else { BMGD_ADAMW_GRADS(kTypeBF16, false); }
#undef BMGD_ADAMW_GRADS
        }
    }
    if (T.h.final) {  // the last block to finish counts the update: every block has read the count by then
        __syncthreads();
        if (threadIdx.x == 0) {
            unsigned int* ticket = reinterpret_cast<unsigned int*>(T.h.control + 2);
            if (atomicAdd(ticket, 1u) == gridDim.x - 1) {
                *ticket = 0u;
                if (F.fine) T.h.control[0] += 1;
                else T.h.control[1] += 1;
                if (T.h.npartial > 0) T.h.control[3] = __double_as_longlong(F.norm);
            }
        }
    }
}

}  // namespace bmgdk
