// pairs.cuh -- two floats in one instruction (add, mul .f32x2), each rounded as by itself.
#pragma once

namespace quan {

// A pair in an aligned register pair, as the instructions take it.
__device__ __forceinline__ unsigned long long pair_of(float2 v) {
    unsigned long long r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(v.x), "f"(v.y));
    return r;
}
__device__ __forceinline__ float2 of_pair(unsigned long long v) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
    return r;
}
__device__ __forceinline__ unsigned long long add2(unsigned long long a, unsigned long long b) {
    unsigned long long r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ unsigned long long mul2(unsigned long long a, unsigned long long b) {
    unsigned long long r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    return of_pair(add2(pair_of(a), pair_of(b)));
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    return of_pair(mul2(pair_of(a), pair_of(b)));
}

}  // namespace quan
