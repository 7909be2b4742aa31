// Two fp32 values in a 64-bit register: one instruction adds or multiplies both, each rounded to nearest by itself.
#pragma once
#include <cuda_runtime.h>

namespace bmgdk {

struct Pair {
    unsigned long long v;
    __device__ __forceinline__ Pair(float a, float b) { asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b)); }
    __device__ __forceinline__ explicit Pair(float a) : Pair(a, a) {}
    __device__ __forceinline__ float2 both() const {
        float2 r;
        asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
        return r;
    }
};
__device__ __forceinline__ Pair operator+(Pair a, const Pair& b) { asm("add.rn.f32x2 %0, %0, %1;" : "+l"(a.v) : "l"(b.v)); return a; }
__device__ __forceinline__ Pair operator*(Pair a, const Pair& b) { asm("mul.rn.f32x2 %0, %0, %1;" : "+l"(a.v) : "l"(b.v)); return a; }
__device__ __forceinline__ Pair multiply_add(const Pair& a, const Pair& b, Pair c) {  // one rounding
    asm("fma.rn.f32x2 %0, %1, %2, %0;" : "+l"(c.v) : "l"(a.v), "l"(b.v));
    return c;
}

}  // namespace bmgdk
