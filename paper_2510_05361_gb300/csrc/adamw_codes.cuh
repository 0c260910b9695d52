// adamw_codes.cuh -- how AdamW's states are held in 8 bits, and the random
// numbers of their rounding (stated with the AdamW calls in mtdao.h).
#pragma once

#include <cuda_runtime.h>
#include <cstdint>

namespace mtdao {

__host__ __device__ __forceinline__ uint64_t splitmix64(uint64_t z) {
    z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
    z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
    return z ^ (z >> 31);
}
constexpr uint64_t kGolden = 0x9E3779B97F4A7C15ull;

// Odd constant of place i in a group of 8: 0x9E3779B1^(i + 1) mod 2^32.  Powers of a
// large odd number, so that the places' random numbers are near independent of
// one another (multiples of one number by 1, 3, 5, ... would correlate by 1/3).
__host__ __device__ constexpr uint32_t place_odd(int i) {
    uint32_t r = 1;
    for (int k = 0; k <= i; ++k) r *= 0x9E3779B1u;
    return r;
}

// m is e4m3, v is e5m2.  kTop: the block's largest magnitude is scaled to [2^kTop,
// 2^(kTop + 1)), which no rounding can take past the largest code; kDrop: bits of an
// fp32 mantissa that a code does not keep.
struct CodeM {
    static constexpr int kTop = 7, kDrop = 20;
};
struct CodeV {
    static constexpr int kTop = 14, kDrop = 21;
};

// The scale of a block of a given largest magnitude, and its inverse: powers of two, so that
// scaling rounds nothing.
template <typename Code>
__device__ __forceinline__ void block_scale(float largest, float &scale, float &inverse) {
    const uint32_t e = __float_as_uint(largest) >> 23;
    scale = __uint_as_float((e - Code::kTop) << 23);
    inverse = __uint_as_float((254u - e + Code::kTop) << 23);
    if (e < 17u) scale = inverse = 0.0f;                                      // below 2^-110
    if (e >= 255u) scale = inverse = __uint_as_float(0x7fffffffu);            // an infinity or a NaN
}

// The largest magnitude of eight values of every lane of the warp; a NaN where there is one.
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ float block_max(const float *x) {
    const float lane = max3(max3(x[0], x[1], x[2]), max3(x[3], x[4], x[5]), max3(x[6], x[7], 0.0f));
    float r;
    asm("redux.sync.max.NaN.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(lane));
    return r;
}

// y, moved within half a code step either way by the given random word: the nearest code of
// the result is y rounded stochastically.  (Among the subnormal codes the step
// is larger than the move, and rounding tends to the nearest.)
template <typename Code>
__device__ __forceinline__ float moved(float y, uint32_t word) {
    const uint32_t by = (word >> (32 - Code::kDrop)) - (1u << (Code::kDrop - 1));
    return __uint_as_float(__float_as_uint(y) + by);
}

__device__ __forceinline__ uint32_t pack_e4m3(float a, float b) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(b), "f"(a));
    return r;
}
__device__ __forceinline__ uint32_t pack_e5m2(float a, float b) {
    uint16_t r;
    asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(r) : "f"(b), "f"(a));
    return r;
}
__device__ __forceinline__ float2 half2_to_float2(uint32_t h) {
    float2 r;
    asm("{\n .reg .b16 l, h;\n mov.b32 {l, h}, %2;\n cvt.f32.f16 %0, l;\n cvt.f32.f16 %1, h;\n}"
        : "=f"(r.x), "=f"(r.y) : "r"(h));
    return r;
}
__device__ __forceinline__ float2 unpack_e4m3(uint32_t two) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(static_cast<uint16_t>(two)));
    return half2_to_float2(h);
}
__device__ __forceinline__ float2 unpack_e5m2(uint32_t four, int upper) {        // e5m2 is fp16's upper half
    return half2_to_float2(__byte_perm(four, 0u, upper ? 0x3424 : 0x1404));
}

// Eight codes of a lane to values: the codes times scale.
__device__ __forceinline__ void decode_m(uint2 c, float scale, float *m) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 t = unpack_e4m3((i < 2 ? c.x : c.y) >> (16 * (i & 1)));
        m[2 * i] = t.x * scale;
        m[2 * i + 1] = t.y * scale;
    }
}
__device__ __forceinline__ void decode_v(uint2 c, float scale, float *v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 t = unpack_e5m2((i < 2 ? c.x : c.y), i & 1);
        v[2 * i] = t.x * scale;
        v[2 * i + 1] = t.y * scale;
    }
}

// A block's eight values in each lane to codes and the block's scale.  RANDOM: rounded with the
// random word times each place's constant, else to nearest.  The whole warp calls it.
template <bool RANDOM>
__device__ __forceinline__ uint2 encode_m(const float *m, uint32_t word, float &scale) {
    float inverse, y[8];
    block_scale<CodeM>(block_max(m), scale, inverse);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        y[i] = m[i] * inverse;
        // what is too small to count must not meet the move: it would borrow from the sign
        if (RANDOM && fabsf(y[i]) >= 0x1p-30f) y[i] = moved<CodeM>(y[i], word * place_odd(i));
    }
    return make_uint2(pack_e4m3(y[0], y[1]) | pack_e4m3(y[2], y[3]) << 16,
                      pack_e4m3(y[4], y[5]) | pack_e4m3(y[6], y[7]) << 16);
}
template <bool RANDOM>
__device__ __forceinline__ uint2 encode_v(const float *v, uint32_t word, float &scale) {
    float inverse, y[8];
    block_scale<CodeV>(block_max(v), scale, inverse);
    if (inverse == 0.0f) return make_uint2(0u, 0u);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        y[i] = fmaxf(v[i] * inverse, 0x1p-16f);
        if (RANDOM) y[i] = moved<CodeV>(y[i], word * place_odd(i));
    }
    return make_uint2(pack_e5m2(y[0], y[1]) | pack_e5m2(y[2], y[3]) << 16,
                      pack_e5m2(y[4], y[5]) | pack_e5m2(y[6], y[7]) << 16);
}

}  // namespace mtdao
