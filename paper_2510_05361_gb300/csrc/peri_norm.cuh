// peri_norm.cuh -- what the Peri-LN residual update's kernels share: the arguments, and how a
// row's columns lie over threads.
#pragma once

#include <cuda_runtime.h>
#include <cstdint>

#include "mtdao.h"
#include "mtdao_internal.h"
#include "pair.cuh"

namespace mtdao {

struct Bf16 {
    uint16_t bits;
};
__device__ __forceinline__ float value(float x) { return x; }
__device__ __forceinline__ float value(Bf16 x) { return __uint_as_float(static_cast<uint32_t>(x.bits) << 16); }
template <typename T>
__device__ __forceinline__ T rounded(float x);
template <>
__device__ __forceinline__ float rounded<float>(float x) { return x; }
template <>
__device__ __forceinline__ Bf16 rounded<Bf16>(float x) {
    uint16_t r;
    asm("cvt.rn.bf16.f32 %0, %1;" : "=h"(r) : "f"(x));
    return Bf16{r};
}
__device__ __forceinline__ uint32_t bf16x2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// Copies to shared memory that run while the thread goes on.
__device__ __forceinline__ void copy_async16(void *to, const void *from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;"
                 :: "r"(static_cast<uint32_t>(__cvta_generic_to_shared(to))), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LATER>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" :: "n"(LATER) : "memory"); }

// Eight elements of a row as they lie in memory: one access of 16 (bf16) or 32 bytes (fp32).
template <typename T>
struct Eight;
template <>
struct Eight<Bf16> {
    uint32_t w[4];
    __device__ __forceinline__ float get(int i) const {
        return __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
    }
    __device__ __forceinline__ Pair pair(int i) const {
        return Pair(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
    }
    __device__ __forceinline__ void set(const float *x) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = bf16x2(x[2 * i], x[2 * i + 1]);
    }
    __device__ __forceinline__ void zero() { w[0] = w[1] = w[2] = w[3] = 0; }
    __device__ __forceinline__ void from_shared(const char *at) {
        const uint4 q = *reinterpret_cast<const uint4 *>(at);
        w[0] = q.x, w[1] = q.y, w[2] = q.z, w[3] = q.w;
    }
    __device__ __forceinline__ void put(int i, Bf16 x) {
        w[i / 2] |= static_cast<uint32_t>(x.bits) << (16 * (i & 1));
    }
    __device__ __forceinline__ void load(const Bf16 *p) {
        const uint4 q = __ldcs(reinterpret_cast<const uint4 *>(p));
        w[0] = q.x, w[1] = q.y, w[2] = q.z, w[3] = q.w;
    }
    __device__ __forceinline__ void load_kept(const Bf16 *p) {
        const uint4 q = __ldg(reinterpret_cast<const uint4 *>(p));
        w[0] = q.x, w[1] = q.y, w[2] = q.z, w[3] = q.w;
    }
    __device__ __forceinline__ void store(Bf16 *p) const {
        __stcs(reinterpret_cast<uint4 *>(p), make_uint4(w[0], w[1], w[2], w[3]));
    }
};
template <>
struct Eight<float> {
    float w[8];
    __device__ __forceinline__ float get(int i) const { return w[i]; }
    __device__ __forceinline__ Pair pair(int i) const { return Pair(w[2 * i], w[2 * i + 1]); }
    __device__ __forceinline__ void set(const float *x) {
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = x[i];
    }
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = 0.0f;
    }
    __device__ __forceinline__ void put(int i, float x) { w[i] = x; }
    __device__ __forceinline__ void from_shared(const char *at) {
        const float4 a = *reinterpret_cast<const float4 *>(at), b = *reinterpret_cast<const float4 *>(at + 16);
        w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w, w[4] = b.x, w[5] = b.y, w[6] = b.z, w[7] = b.w;
    }
    __device__ __forceinline__ void load(const float *p) {
        asm volatile("ld.global.cs.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=f"(w[0]), "=f"(w[1]), "=f"(w[2]), "=f"(w[3]), "=f"(w[4]), "=f"(w[5]), "=f"(w[6]), "=f"(w[7])
                     : "l"(p));
    }
    __device__ __forceinline__ void load_kept(const float *p) {
        const float4 a = __ldg(reinterpret_cast<const float4 *>(p)), b = __ldg(reinterpret_cast<const float4 *>(p) + 1);
        w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w, w[4] = b.x, w[5] = b.y, w[6] = b.z, w[7] = b.w;
    }
    __device__ __forceinline__ void store(float *p) const {
        asm volatile("st.global.cs.v8.f32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};"
                     :: "f"(w[0]), "f"(w[1]), "f"(w[2]), "f"(w[3]), "f"(w[4]), "f"(w[5]), "f"(w[6]), "f"(w[7]), "l"(p)
                     : "memory");
    }
};

// The columns of a row over `threads` threads, in groups of eight: thread t's q-th group holds eight consecutive
// columns where the row can be read in whole groups (VEC: d a multiple of 8, every address of 8 elements),
// else eight columns `threads` apart, so that neighbours read neighbours.
template <bool VEC>
struct Columns {
    int t, threads, d;
    __device__ __forceinline__ int at(int q, int i) const {
        return VEC ? (q * threads + t) * 8 + i : t + threads * (q * 8 + i);
    }
    __device__ __forceinline__ bool valid(int q, int i) const { return at(q, VEC ? 0 : i) < d; }
    template <typename T>
    __device__ __forceinline__ void load(const T *row, int q, Eight<T> &e) const {
        if constexpr (VEC) {
            if (valid(q, 0)) e.load(row + at(q, 0)); else e.zero();
        } else {
            e.zero();
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (valid(q, i)) e.put(i, row[at(q, i)]);
        }
    }
    template <typename T>
    __device__ __forceinline__ void store(T *row, int q, const Pair *x) const {
        float y[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i].get(y[2 * i], y[2 * i + 1]);
        store(row, q, y);
    }
    template <typename T>
    __device__ __forceinline__ void store(T *row, int q, const float *x) const {
        if constexpr (VEC) {
            Eight<T> e;
            e.set(x);
            if (valid(q, 0)) e.store(row + at(q, 0));
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (valid(q, i)) row[at(q, i)] = rounded<T>(x[i]);
        }
    }
};

// A vector whose type is known at the launch only: weights, gate and their gradients.  Read by
// every row, and kept in the first-level cache.
struct Vector {
    void *p;
    int32_t bf16;
    __device__ __forceinline__ float get(int64_t i) const {
        return bf16 ? value(static_cast<const Bf16 *>(p)[i]) : static_cast<const float *>(p)[i];
    }
    __device__ __forceinline__ void set(int64_t i, float x) const {
        if (bf16) static_cast<Bf16 *>(p)[i] = rounded<Bf16>(x);
        else static_cast<float *>(p)[i] = x;
    }
    template <bool VEC>
    __device__ __forceinline__ void load(const Columns<VEC> &c, int64_t row, int q, Pair *x) const {
        float y[8];
        load(c, row, q, y);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = Pair(y[2 * i], y[2 * i + 1]);
    }
    template <bool VEC>
    __device__ __forceinline__ void load(const Columns<VEC> &c, int64_t row, int q, float *x) const {
        if (bf16) {
            Eight<Bf16> e;
            if constexpr (!VEC) c.load(static_cast<const Bf16 *>(p) + row, q, e);
            else if (c.valid(q, 0)) e.load_kept(static_cast<const Bf16 *>(p) + row + c.at(q, 0));
            else e.zero();
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = e.get(i);
        } else {
            Eight<float> e;
            if constexpr (!VEC) c.load(static_cast<const float *>(p) + row, q, e);
            else if (c.valid(q, 0)) e.load_kept(static_cast<const float *>(p) + row + c.at(q, 0));
            else e.zero();
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = e.get(i);
        }
    }
};

struct NormArgs {
    int64_t rows, gate_rows, per_gate;      // per_gate: rows of one gate row
    int32_t d, layer;
    int32_t wide;                           // all rows are fp32
    float eps, residual_scale;
    int64_t ld_x, ld_f, ld_y, ld_h, ld_dy, ld_dh, ld_dx, ld_df;
    const void *x, *f, *dy, *dh;
    void *y, *h, *dx, *df;
    Vector post_w, post_b, pre_w, pre_b, gate;
    Vector d_post_w, d_post_b, d_pre_w, d_pre_b, d_gate;
    float2 *stats;                          // [2][rows]
    float *partial;                         // workspace of backward: see peri_norm_backward.cuh
    int32_t contiguous;                     // backward: a worker's rows are neighbours
    int32_t split;                          // backward: a gate row's rows may belong to several workers
};

// The rows' gate, as the kernels tell them apart.
enum { kGateNone, kGateChannel, kGateRows, kGateElement };
__host__ __device__ __forceinline__ int gate_kind(const NormArgs &a) {
    return a.gate.p == nullptr ? kGateNone : a.gate_rows == 1 ? kGateChannel : a.per_gate == 1 ? kGateElement : kGateRows;
}

// Index of the first element of row r's gate row.
__device__ __forceinline__ int64_t gate_row(const NormArgs &a, int64_t r) {
    if (a.gate_rows == 1) return 0;
    if (a.per_gate == 1) return r * a.d;
    const int64_t g = a.rows <= 0xffffffffll ? static_cast<uint32_t>(r) / static_cast<uint32_t>(a.per_gate)
                                             : r / a.per_gate;
    return g * a.d;
}

// vec: d is a multiple of 8 and every row starts at a multiple of 8 elements.
template <typename S, typename B>
cudaError_t launch_peri_forward(const NormArgs &a, bool vec, cudaStream_t stream);
template <typename S, typename B>
cudaError_t launch_peri_backward(const NormArgs &a, bool vec, cudaStream_t stream);

// Workspace of the backward pass, in floats, and how its rows are dealt out.
struct BackwardPlan {
    int groups_of_eight;                    // columns of a thread
    int lanes;                              // of a row, where it has one warp or less
    int warps;                              // of a row, in one thread block
    int cluster;                            // thread blocks of a row
    int groups;                             // rows that a thread block works on at a time
    int64_t blocks;                         // thread blocks, or clusters of them
    bool contiguous, split, full;
    int64_t floats;
};
constexpr int kPeriSms = 152;               // of the device that this is written for: sizes grids, no more
BackwardPlan plan_backward(const NormArgs &a, bool vec);

}  // namespace mtdao
