// Two fp32 values in a pair of registers, and packed operations on such pairs (one instruction for both).
#pragma once
#include <stdint.h>

namespace slide_attn {

using pair = unsigned long long;

// A pair of one value twice is best built once, outside of the loops.
__device__ __forceinline__ pair make_pair(float x, float y) {
    pair p;
    asm("mov.b64 %0, {%1, %2};" : "=l"(p) : "f"(x), "f"(y));
    return p;
}
__device__ __forceinline__ pair both(float x) { return make_pair(x, x); }
__device__ __forceinline__ void split_pair(pair p, float& x, float& y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(p)); }
__device__ __forceinline__ pair fma2(pair a, pair b, pair c) {
    pair d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ pair add2(pair a, pair b) {
    pair d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ pair mul2(pair a, pair b) {
    pair d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}

}  // namespace slide_attn
