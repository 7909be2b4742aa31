// One AdamW update of many tensors in one launch (bmgd_adamw_step), and the sum of squares of their gradients.
//
// Per value, with t the number of this update, g the gradient times grad_scale and the clipping factor:
//     m <- a m + (1-a) g;   v <- b v + ((1-b) g) g
//     theta <- theta (1 - lr wd) - (lr / (1-a^t)) (m / (sqrt(v) / sqrt(1-b^t) + eps))
// Every product and sum is rounded to fp32 by itself (no contraction), so the result does not depend on how the
// compiler schedules it: two kernels that process the same value in different places agree bit for bit.
//
// What bounds it: memory.  Each value of theta, the gradient and the moments is read once and written once.  A warp
// takes units of 256 consecutive values of one tensor: lane l holds values 4l..4l+3 and 128+4l..128+4l+3, so that every
// access of the warp is one contiguous piece, and the 256 values that share a scale in the 8-bit form sit in one warp.
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
#include <cuda_runtime.h>

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
    uint8_t ptype, gtype, bits, aligned;
    uint32_t reserved;
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

// value of an e4m3 code before scaling: exact
__device__ __forceinline__ float decode_m(uint32_t c) {
    const uint32_t mag = c & 0x7Fu;
    // exponent field 0 counts in steps of 2^-9
    float x = mag >= 8u ? __uint_as_float((mag << 20) + (120u << 23)) : (float)mag * 0x1p-9f;
    if (mag == 0x7Fu) x = __uint_as_float(0x7FC00000u);
    return __uint_as_float(__float_as_uint(x) | ((c & 0x80u) << 24));
}
__device__ __forceinline__ uint32_t encode_m(float x, uint32_t r16) {  // x scaled to |x| < 256
    const uint32_t bits = __float_as_uint(x), mag = bits & 0x7FFFFFFFu;
    uint32_t c;
    if (mag >= 0x3C800000u) c = (mag - (120u << 23) + (r16 << 4)) >> 20;  // |x| >= 2^-6
    else c = min((uint32_t)__fadd_rn(__uint_as_float(mag) * 512.f, (float)r16 * 0x1p-16f), 8u);
    if (!finite_bits(bits)) c = 0x7Fu;
    return c | ((bits >> 24) & 0x80u);
}
__device__ __forceinline__ float decode_v(uint32_t c, int s) {
    const uint32_t e = (c >> 3) + (uint32_t)(s - 30);
    float x = __uint_as_float((e << 23) | ((c & 7u) << 20));
    if (c == 0u) x = 0.f;
    if (c == 255u) x = __uint_as_float(0x7FC00000u);
    return x;
}
__device__ __forceinline__ uint32_t encode_v(float v, int s, uint32_t r16) {
    const int y = (int)(__float_as_uint(v) - ((uint32_t)(s - 30) << 23));
    uint32_t c = y >= (1 << 20) ? (uint32_t)(y + (int)(r16 << 4)) >> 20 : 1u;
    if (v == 0.f) c = 0u;
    if (!finite_bits(__float_as_uint(v))) c = 255u;
    return c;
}
// biased exponent of the largest finite magnitude of the warp's unit
__device__ __forceinline__ int unit_exponent(const float (&x)[8], int least) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t mag = __float_as_uint(x[i]) & 0x7FFFFFFFu;
        if (mag < 0x7F800000u) top = max(top, mag);
    }
    top = __reduce_max_sync(0xFFFFFFFFu, top);
    return max((int)(top >> 23), least);
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
struct AdamwFactors {
    float gscale, step, root, a, a1, b, b1, eps;
    int fine;
    uint32_t key;
    double norm;
};

template <int CAP>
__global__ void __launch_bounds__(kAdamwThreads) adamw_kernel(const __grid_constant__ AdamwTable<CAP> T) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    __shared__ AdamwFactors F;
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
        const long long t = T.h.control[0] + 1;
        double scale = T.h.grad_scale;
        F.fine = 1;
        F.norm = 0.0;
        if (T.h.npartial > 0) {
            double s = 0.0;
            for (int w = 0; w < kAdamwThreads / 32; ++w) s += part[w];
            const double norm = sqrt(s) * T.h.grad_scale;
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
    if (F.fine) {
        const float gscale = F.gscale, step = F.step, root = F.root, fa = F.a, fa1 = F.a1, fb = F.b, fb1 = F.b1, eps = F.eps;
        for (long long chunk = blockIdx.x; chunk < T.h.chunks; chunk += gridDim.x) {
            const AdamwEntry& e = T.e[adamw_find(T, chunk)];
            const long long n = e.n;
            const bool al = e.aligned, eight = e.bits == 8;
            const float keep = e.keep;
            const bool random_theta = e.ptype == kTypeBF16 && e.master == nullptr;
            const uint32_t key = mix32(F.key ^ (T.h.seed_hi + e.index * 0x9E3779B9u));
            const long long unit0 = ((chunk - e.first_chunk) * (kAdamwThreads / 32) + warp) * T.h.units;
            for (int u = 0; u < T.h.units; ++u) {
                const long long unit = unit0 + u;
                if (unit * kAdamwUnit >= n) break;
                const long long at[2] = {unit * kAdamwUnit + lane * 4, unit * kAdamwUnit + lane * 4 + 128};
                float p[8], g[8], m[8], v[8];
                uint32_t cm[2] = {0, 0}, cv[2] = {0, 0};
                int sm = 0, sv = 0;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float4 x = load4(e.grad, e.gtype, at[h], n, al);
                    const float4 y = e.master ? load4(e.master, kTypeF32, at[h], n, al) : load4(e.param, e.ptype, at[h], n, al);
                    g[4 * h] = x.x; g[4 * h + 1] = x.y; g[4 * h + 2] = x.z; g[4 * h + 3] = x.w;
                    p[4 * h] = y.x; p[4 * h + 1] = y.y; p[4 * h + 2] = y.z; p[4 * h + 3] = y.w;
                    if (eight) {
                        cm[h] = load_codes(e.m, at[h], n, al);
                        cv[h] = load_codes(e.v, at[h], n, al);
                    } else {
                        const float4 a4 = load4(e.m, kTypeF32, at[h], n, al), b4 = load4(e.v, kTypeF32, at[h], n, al);
                        m[4 * h] = a4.x; m[4 * h + 1] = a4.y; m[4 * h + 2] = a4.z; m[4 * h + 3] = a4.w;
                        v[4 * h] = b4.x; v[4 * h + 1] = b4.y; v[4 * h + 2] = b4.z; v[4 * h + 3] = b4.w;
                    }
                }
                if (eight) {
                    sm = e.m_scale[unit];
                    sv = e.v_scale[unit];
                    const float unscale = power_of_two(sm - 7);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        m[i] = decode_m((cm[i >> 2] >> (8 * (i & 3))) & 0xFFu) * unscale;
                        v[i] = decode_v((cv[i >> 2] >> (8 * (i & 3))) & 0xFFu, sv);
                    }
                }
                float q[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float gi = __fmul_rn(g[i], gscale);
                    m[i] = __fadd_rn(__fmul_rn(m[i], fa), __fmul_rn(gi, fa1));
                    v[i] = __fadd_rn(__fmul_rn(v[i], fb), __fmul_rn(__fmul_rn(gi, fb1), gi));
                    const float denom = __fadd_rn(__fmul_rn(__fsqrt_rn(v[i]), root), eps);
                    q[i] = __fsub_rn(__fmul_rn(p[i], keep), __fmul_rn(__fdiv_rn(m[i], denom), step));
                }
                uint32_t r[8];
                if (eight || random_theta) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const long long place = at[i >> 2] + (i & 3);
                        r[i] = mix32((uint32_t)place ^ (key + (uint32_t)(place >> 32) * 0x85EBCA6Bu));
                    }
                }
                if (eight) {
                    const int tm = unit_exponent(m, 16), tv = unit_exponent(v, 40);
                    const float scale = power_of_two(261 - tm);
                    uint32_t wm[2] = {0, 0}, wv[2] = {0, 0};
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        wm[i >> 2] |= encode_m(m[i] * scale, r[i] & 0xFFFFu) << (8 * (i & 3));
                        wv[i >> 2] |= encode_v(v[i], tv, r[i] >> 16) << (8 * (i & 3));
                    }
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        store_codes(e.m, at[h], n, al, wm[h]);
                        store_codes(e.v, at[h], n, al, wv[h]);
                    }
                    if (lane == 0) { e.m_scale[unit] = (uint8_t)tm; e.v_scale[unit] = (uint8_t)tv; }
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float x[4] = {q[4 * h], q[4 * h + 1], q[4 * h + 2], q[4 * h + 3]};
                    if (!eight) {
                        const float mm[4] = {m[4 * h], m[4 * h + 1], m[4 * h + 2], m[4 * h + 3]};
                        const float vv[4] = {v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]};
                        store4(e.m, kTypeF32, at[h], n, al, mm);
                        store4(e.v, kTypeF32, at[h], n, al, vv);
                    }
                    if (e.master) store4(e.master, kTypeF32, at[h], n, al, x);
                    if (random_theta) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const uint32_t b = __float_as_uint(x[i]);
                            const uint32_t up = (b + (mix32(r[4 * h + i] ^ 0x9E3779B9u) & 0xFFFFu)) & 0xFFFF0000u;
                            if (finite_bits(b)) x[i] = __uint_as_float(up);
                        }
                    }
                    store4(e.param, e.ptype, at[h], n, al, x);
                }
            }
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
