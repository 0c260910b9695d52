// adamw.cu -- AdamW over lists of tensors (the formulas and the format of the states are in
// mtdao.h): the step, the gradients' norms, the replicas' average.
//
// Every kernel walks the list by records of up to 2048 elements of one tensor
// (AdamwChunk), a thread block each; a warp of it takes 256 elements, which is
// the block of elements that shares a scale in 8 bits, eight consecutive ones a lane: the
// block's largest magnitude is then one warp reduction, and a step reads and
// writes each quantity once.
#include "adamw.h"
#include "adamw_codes.cuh"
#include "kahan.cuh"
#include "replica_mean.cuh"

namespace mtdao {
namespace {

__device__ __forceinline__ AdamwChunk load_chunk(const AdamwChunk *c) {
    union {
        AdamwChunk chunk;
        uint4 w[2];
    } u;
    u.w[0] = __ldg(reinterpret_cast<const uint4 *>(c));
    u.w[1] = __ldg(reinterpret_cast<const uint4 *>(c) + 1);
    return u.chunk;
}

__device__ __forceinline__ float bf16_to_float(uint16_t b) { return __uint_as_float(static_cast<uint32_t>(b) << 16); }

// Eight values of a tensor from element at on, zeros past n.
__device__ __forceinline__ void load8(const void *p, bool bf16, int at, int n, float *out) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        out[i] = 0.0f;
        if (at + i < n)
            out[i] = bf16 ? bf16_to_float(static_cast<const uint16_t *>(p)[at + i]) : static_cast<const float *>(p)[at + i];
    }
}

// bf16 bits of x with a random 16-bit word added below them; a NaN stays one.
__device__ __forceinline__ uint16_t bf16_random(float x, uint32_t word) {
    const uint32_t bits = __float_as_uint(x);
    return static_cast<uint16_t>((x != x ? bits | 0x400000u : bits + (word & 0xffffu)) >> 16);
}
__device__ __forceinline__ uint16_t bf16_nearest(float x) {
    const uint32_t bits = __float_as_uint(x);
    return static_cast<uint16_t>((x != x ? bits | 0x400000u : bits + 0x7fffu + ((bits >> 16) & 1u)) >> 16);
}

__device__ __forceinline__ float sqrt_approx(float x) {
    float r;
    asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// m and v are formed with a rounding after each operation in 8 bits: what the
// formula gives then does not depend on the compiler's choice of fused operations.
// In 32 bits the products stay unrounded (one rounding less for each).
template <int BITS>
__device__ __forceinline__ float ema(float b, float c, float s, float target) {
    if constexpr (BITS == 8) return __fadd_rn(__fmul_rn(s, b), __fmul_rn(target, c));
    return isinf(s) && c < 1.0f ? fmaf(c, target, s) : fmaf(c, target, fmaf(-c, s, s));
}

template <int BITS>
__global__ void __launch_bounds__(kAdamwThreads) adamw_step_kernel(const AdamwList a, const AdamwScalars sc,
                                                                   const float *clip_scale) {
    const AdamwChunk c = load_chunk(a.chunks + blockIdx.x);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (warp * kAdamwBlock >= c.n) return;
    const int at = warp * kAdamwBlock + 8 * lane;
    const uint32_t block = c.block + warp;
    const int64_t e = static_cast<int64_t>(block) * kAdamwBlock + 8 * lane;
    const uint32_t replica = static_cast<uint32_t>(blockIdx.x / a.n_chunks);
    const bool p16 = (c.flags & kAdamwParamBf16) != 0;

    float g[8], p[8], m[8], v[8];
    load8(c.g, (c.flags & kAdamwGradBf16) != 0, at, c.n, g);
    load8(c.p, p16, at, c.n, p);
    if constexpr (BITS == 8) {
        decode_m(reinterpret_cast<const uint2 *>(a.m)[e / 8], a.m_scale[block], m);
        decode_v(reinterpret_cast<const uint2 *>(a.v)[e / 8], a.v_scale[block], v);
    } else {
        load8(static_cast<const float *>(a.m) + e, false, 0, 8, m);
        load8(static_cast<const float *>(a.v) + e, false, 0, 8, v);
    }
    const float s = clip_scale ? clip_scale[replica] : 1.0f;
    const float keep = fmaf(-sc.decay, c.decay, 1.0f);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float gi = __fmul_rn(g[i], s);
        m[i] = ema<BITS>(sc.b1, sc.c1, m[i], gi);
        v[i] = ema<BITS>(sc.b2, sc.c2, v[i], __fmul_rn(gi, gi));
        p[i] = fmaf(-sc.step, __fdividef(m[i], fmaf(sqrt_approx(v[i]), sc.root, sc.eps)), p[i] * keep);
    }
    uint32_t low = 0, high = 0;
    if (BITS == 8 || p16) {
        const uint64_t blocks = static_cast<uint64_t>(a.n_state) / kAdamwBlock;
        const uint64_t group = (block - replica * blocks) * (kAdamwBlock / 8) + lane;
        const uint64_t z = splitmix64(sc.key + ((static_cast<uint64_t>(replica) << 32) + group) * kGolden);
        low = static_cast<uint32_t>(z);
        high = static_cast<uint32_t>(z >> 32);
    }
    if constexpr (BITS == 8) {
        float scale;
        const uint2 cm = encode_m<true>(m, low, scale);
        reinterpret_cast<uint2 *>(a.m)[e / 8] = cm;
        if (lane == 0) a.m_scale[block] = scale;
        const uint2 cv = encode_v<true>(v, high, scale);
        reinterpret_cast<uint2 *>(a.v)[e / 8] = cv;
        if (lane == 0) a.v_scale[block] = scale;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            static_cast<float *>(a.m)[e + i] = m[i];
            static_cast<float *>(a.v)[e + i] = v[i];
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (at + i >= c.n) break;
        if (p16)
            static_cast<uint16_t *>(c.p)[at + i] = bf16_random(p[i], low * place_odd(i));
        else
            static_cast<float *>(c.p)[at + i] = p[i];
    }
}

// ---------------------------------------------------------------- gradient norms

__global__ void __launch_bounds__(kAdamwThreads) adamw_norm_kernel(const AdamwList a, double *partial) {
    const int replica = blockIdx.y;
    const AdamwChunk *chunks = a.chunks + replica * a.n_chunks;
    Kahan sum;
    double wide = 0.0;
    for (int64_t k = blockIdx.x; k < a.n_chunks; k += gridDim.x) {
        const AdamwChunk c = load_chunk(chunks + k);
        float g[8];
        load8(c.g, (c.flags & kAdamwGradBf16) != 0, 8 * threadIdx.x, c.n, g);
        float q = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) q = fmaf(g[i], g[i], q);
        if (q >= 0x1p-90f && q <= 0x1p100f) {
            sum.add(q);
        } else {                                     // zeros, or squares that fp32 does not hold
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (g[i] != 0.0f) wide = fma(static_cast<double>(g[i]), static_cast<double>(g[i]), wide);
        }
    }
    __shared__ double sums[kAdamwThreads / 32];
    const double w = warp_sum(sum.value() + wide);
    if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = w;
    __syncthreads();
    if (threadIdx.x == 0) {
        double t = 0.0;
        for (int i = 0; i < kAdamwThreads / 32; ++i) t += sums[i];
        partial[static_cast<int64_t>(replica) * gridDim.x + blockIdx.x] = t;
    }
}

__global__ void __launch_bounds__(32) adamw_norm_last_kernel(const double *partial, int blocks, double *sums, float *scale,
                                                             double max_norm) {
    double t = 0.0;
    for (int i = threadIdx.x; i < blocks; i += 32) t += partial[static_cast<int64_t>(blockIdx.x) * blocks + i];
    t = warp_sum(t);
    if (threadIdx.x != 0) return;
    if (sums) sums[blockIdx.x] = t;
    if (scale) {
        const double s = max_norm / (sqrt(t) + 1e-6);
        scale[blockIdx.x] = static_cast<float>(s > 1.0 ? 1.0 : s);       // a NaN stays one
    }
}

// ---------------------------------------------------------------- average

// The mean over the replicas of what get(r) gives; see replica_mean.cuh.
template <typename Get>
__device__ __forceinline__ void mean8(int M, Get get, float *out) {
    float s[8];
    get(0, s);
    DiffSum sum[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[i] = DiffSum(s[i]);
    for (int r = 1; r < M; ++r) {
        get(r, s);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i].add(s[i]);
    }
    bool odd = false;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float q = sum[i].partial() / static_cast<float>(M);
        out[i] = q == 0.0f ? sum[i].s0 : sum[i].s0 + q;
        odd |= out[i] != out[i];
    }
    if (!odd) return;
    float plain[8] = {};
    for (int r = 0; r < M; ++r) {
        get(r, s);
#pragma unroll
        for (int i = 0; i < 8; ++i) plain[i] += s[i];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) out[i] = mean_or_plain(out[i], plain[i], static_cast<float>(M));
}

template <int BITS>
__global__ void __launch_bounds__(kAdamwThreads) adamw_average_kernel(const AdamwList a, uint32_t mask) {
    const AdamwChunk c = load_chunk(a.chunks + blockIdx.x);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (warp * kAdamwBlock >= c.n) return;
    const int at = warp * kAdamwBlock + 8 * lane;
    const int64_t blocks = a.n_state / kAdamwBlock;
    const int64_t block = c.block + warp;
    const int64_t e = block * kAdamwBlock + 8 * lane;
    float mean[8];
    if (mask & 1u) {
        const bool p16 = (c.flags & kAdamwParamBf16) != 0;
        mean8(a.M, [&](int r, float *s) { load8(load_chunk(a.chunks + r * a.n_chunks + blockIdx.x).p, p16, at, c.n, s); },
              mean);
        for (int r = 0; r < a.M; ++r) {
            void *p = load_chunk(a.chunks + r * a.n_chunks + blockIdx.x).p;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (at + i >= c.n) break;
                if (p16)
                    static_cast<uint16_t *>(p)[at + i] = bf16_nearest(mean[i]);
                else
                    static_cast<float *>(p)[at + i] = mean[i];
            }
        }
    }
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        if (!(mask & (2u << q))) continue;
        void *held = q == 0 ? a.m : a.v;
        float *scales = q == 0 ? a.m_scale : a.v_scale;
        if constexpr (BITS == 8) {
            mean8(a.M, [&](int r, float *s) {
                const uint2 codes = static_cast<const uint2 *>(held)[(r * a.n_state + e) / 8];
                const float scale = scales[r * blocks + block];
                if (q == 0) decode_m(codes, scale, s); else decode_v(codes, scale, s);
            }, mean);
            float scale;
            const uint2 codes = q == 0 ? encode_m<false>(mean, 0, scale) : encode_v<false>(mean, 0, scale);
            for (int r = 0; r < a.M; ++r) {
                static_cast<uint2 *>(held)[(r * a.n_state + e) / 8] = codes;
                if (lane == 0) scales[r * blocks + block] = scale;
            }
        } else {
            float *s32 = static_cast<float *>(held);
            mean8(a.M, [&](int r, float *s) { load8(s32 + r * a.n_state + e, false, 0, 8, s); }, mean);
            for (int r = 0; r < a.M; ++r)
#pragma unroll
                for (int i = 0; i < 8; ++i) s32[r * a.n_state + e + i] = mean[i];
        }
    }
}

// ---------------------------------------------------------------- records

__global__ void __launch_bounds__(kAdamwThreads) adamw_bind_kernel(AdamwChunk *chunks, const AdamwTensor *tensors,
                                                                   int32_t n_tensors, void *const *table,
                                                                   const int32_t *dtype, bool grads, int64_t n_chunks,
                                                                   int64_t n_blocks) {
    const int64_t k = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x;
    if (k >= n_chunks) return;
    int32_t lo = 0, hi = n_tensors;                  // the last tensor whose first chunk is at most k: an empty
    while (hi - lo > 1) {                            // tensor has its successor's, so the found one holds k
        const int32_t mid = (lo + hi) / 2;
        if (tensors[mid].first_chunk <= k) lo = mid; else hi = mid;
    }
    const AdamwTensor t = tensors[lo];
    const int64_t first = (k - t.first_chunk) * kAdamwChunk;
    const bool bf16 = dtype[lo] == MTDAO_BF16;
    AdamwChunk &c = chunks[blockIdx.y * n_chunks + k];
    char *p = static_cast<char *>(table[static_cast<int64_t>(blockIdx.y) * n_tensors + lo]) + first * (bf16 ? 2 : 4);
    if (grads) {
        c.g = p;
        c.flags = (c.flags & ~kAdamwGradBf16) | (bf16 ? kAdamwGradBf16 : 0u);
        return;
    }
    const int64_t left = t.numel - first;
    c.p = p;
    c.block = static_cast<uint32_t>(blockIdx.y * n_blocks + t.first_block + first / kAdamwBlock);
    c.n = static_cast<int32_t>(left < kAdamwChunk ? left : kAdamwChunk);
    c.flags = (c.flags & ~kAdamwParamBf16) | (bf16 ? kAdamwParamBf16 : 0u);
    c.decay = t.decay;
}

}  // namespace

cudaError_t launch_adamw_bind(AdamwChunk *chunks, const AdamwTensor *tensors, int32_t n_tensors, void *const *table,
                              const int32_t *dtype, bool grads, int64_t n_chunks, int64_t n_blocks, int32_t M,
                              cudaStream_t stream) {
    const dim3 grid(static_cast<unsigned>((n_chunks + kAdamwThreads - 1) / kAdamwThreads), M);
    adamw_bind_kernel<<<grid, kAdamwThreads, 0, stream>>>(chunks, tensors, n_tensors, table, dtype, grads, n_chunks,
                                                          n_blocks);
    return cudaGetLastError();
}

cudaError_t launch_adamw_step(const AdamwList &a, const AdamwScalars &sc, const float *clip_scale, cudaStream_t stream) {
    const unsigned grid = static_cast<unsigned>(a.n_chunks * a.M);
    if (a.bits == 8)
        adamw_step_kernel<8><<<grid, kAdamwThreads, 0, stream>>>(a, sc, clip_scale);
    else
        adamw_step_kernel<32><<<grid, kAdamwThreads, 0, stream>>>(a, sc, clip_scale);
    return cudaGetLastError();
}

int adamw_norm_blocks(int num_sms, int M, int64_t n_chunks) {
    const int64_t want = (8 * static_cast<int64_t>(num_sms) + M - 1) / M;
    return static_cast<int>(n_chunks < want ? n_chunks : want);
}

cudaError_t launch_adamw_norm(const AdamwList &a, int blocks, double *partial, double *sums, float *scale,
                              double max_norm, cudaStream_t stream) {
    adamw_norm_kernel<<<dim3(blocks, a.M), kAdamwThreads, 0, stream>>>(a, partial);
    adamw_norm_last_kernel<<<a.M, 32, 0, stream>>>(partial, blocks, sums, scale, max_norm);
    return cudaGetLastError();
}

cudaError_t launch_adamw_average(const AdamwList &a, uint32_t mask, cudaStream_t stream) {
    const unsigned grid = static_cast<unsigned>(a.n_chunks);
    if (a.bits == 8)
        adamw_average_kernel<8><<<grid, kAdamwThreads, 0, stream>>>(a, mask);
    else
        adamw_average_kernel<32><<<grid, kAdamwThreads, 0, stream>>>(a, mask);
    return cudaGetLastError();
}

}  // namespace mtdao
