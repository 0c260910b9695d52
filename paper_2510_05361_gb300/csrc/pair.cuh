// pair.cuh -- fp32 arithmetic two values at a time.
#pragma once

#include <cuda_runtime.h>
#include <cstdint>

namespace mtdao {

// Two fp32 operations in one instruction, each rounded as the single ones are.
struct Pair {
    uint64_t bits;
    __device__ __forceinline__ Pair() {}
    __device__ __forceinline__ Pair(float lo, float hi) { asm("mov.b64 %0, {%1, %2};" : "=l"(bits) : "f"(lo), "f"(hi)); }
    __device__ __forceinline__ explicit Pair(float both) : Pair(both, both) {}
    __device__ __forceinline__ void get(float &lo, float &hi) const {
        asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(bits));
    }
    __device__ __forceinline__ float lo() const { float a, b; get(a, b); return a; }
    __device__ __forceinline__ float hi() const { float a, b; get(a, b); return b; }
};
__device__ __forceinline__ Pair operator*(Pair a, Pair b) {
    Pair r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.bits) : "l"(a.bits), "l"(b.bits));
    return r;
}
__device__ __forceinline__ Pair operator+(Pair a, Pair b) {
    Pair r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.bits) : "l"(a.bits), "l"(b.bits));
    return r;
}
__device__ __forceinline__ Pair minus(Pair a, Pair b) {           // rounded once: -b is exact
    float lo, hi;
    b.get(lo, hi);
    return a + Pair(-lo, -hi);
}
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) {
    Pair r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.bits) : "l"(a.bits), "l"(b.bits), "l"(c.bits));
    return r;
}

// a b, rounded, also where it is added to something next: the assembler fuses a packed
// product and sum (seen in a result's last bit), but not this.
__device__ __forceinline__ Pair product(Pair a, Pair b) { return fma2(a, b, Pair(0.0f)); }

}  // namespace mtdao
