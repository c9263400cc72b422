// Paired f32 arithmetic.
#pragma once
#include <stdint.h>

namespace tw {

// Two f32 operations in one instruction, each rounded by itself.
struct Two { uint64_t b; };
__device__ __forceinline__ Two two(float x, float y) {
    Two t;
    asm("mov.b64 %0, {%1, %2};" : "=l"(t.b) : "f"(x), "f"(y));
    return t;
}
__device__ __forceinline__ void apart(Two t, float &x, float &y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(t.b)); }
__device__ __forceinline__ Two mul2(Two a, Two b) {
    Two t;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(t.b) : "l"(a.b), "l"(b.b));
    return t;
}
__device__ __forceinline__ Two fma2(Two a, Two b, Two c) {
    Two t;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(t.b) : "l"(a.b), "l"(b.b), "l"(c.b));
    return t;
}
__device__ __forceinline__ Two add2(Two a, Two b) {
    Two t;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(t.b) : "l"(a.b), "l"(b.b));
    return t;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float m;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(m) : "f"(a), "f"(b), "f"(c));
    return m;
}

}  // namespace tw
