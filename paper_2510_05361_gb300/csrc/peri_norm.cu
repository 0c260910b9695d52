// peri_norm.cu -- the Peri-LN residual update and its gradients (formulas in mtdao.h).
#include <cuda_runtime.h>

#include <cmath>
#include <cstdint>
#include <cstdio>

#include <nvtx3/nvToolsExt.h>

#include "mtdao.h"
#include "mtdao_internal.h"

namespace mtdao {
namespace {

constexpr int kRowThreads = 256;

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

// Eight elements of a row as they lie in memory: one access of 16 (bf16) or 32 bytes (fp32).
template <typename T>
struct Eight;
template <>
struct Eight<Bf16> {
    uint32_t w[4];
    __device__ __forceinline__ float get(int i) const {
        return __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
    }
    __device__ __forceinline__ void set(const float *x) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = bf16x2(x[2 * i], x[2 * i + 1]);
    }
    __device__ __forceinline__ void zero() { w[0] = w[1] = w[2] = w[3] = 0; }
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
    __device__ __forceinline__ void set(const float *x) {
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = x[i];
    }
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = 0.0f;
    }
    __device__ __forceinline__ void put(int i, float x) { w[i] = x; }
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
    __device__ __forceinline__ void load(const Columns<VEC> &c, int64_t row, int q, float *x) const {
        if (VEC && c.valid(q, 0)) {
            if (bf16) {
                Eight<Bf16> e;
                e.load_kept(static_cast<const Bf16 *>(p) + row + c.at(q, 0));
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = e.get(i);
            } else {
                Eight<float> e;
                e.load_kept(static_cast<const float *>(p) + row + c.at(q, 0));
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = e.get(i);
            }
            return;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = !VEC && c.valid(q, i) ? get(row + c.at(q, i)) : 0.0f;
    }
};

struct NormArgs {
    int64_t rows, gate_rows, per_gate;      // per_gate: rows of one gate row
    int32_t d, layer;
    float eps, residual_scale;
    int64_t ld_x, ld_f, ld_y, ld_h, ld_dy, ld_dh, ld_dx, ld_df;
    const void *x, *f, *dy, *dh;
    void *y, *h, *dx, *df;
    Vector post_w, post_b, pre_w, pre_b, gate;
    Vector d_post_w, d_post_b, d_pre_w, d_pre_b, d_gate;
    float2 *stats;                          // [2][rows]
    float2 *row_sums;                       // [rows], workspace
};

// The sum over a row's W warps, the same in each of its threads.  parts: W floats of the row's,
// not read by anyone since the last barrier but one.
template <int W>
__device__ __forceinline__ float row_sum(float v, float *parts) {
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
    if constexpr (W == 1) return v;
    if ((threadIdx.x & 31) == 0) parts[threadIdx.x >> 5] = v;
    __syncthreads();
    float t = 0.0f;
#pragma unroll
    for (int i = 0; i < W; ++i) t += parts[i];
    return t;
}

// Gate row of row r.
__device__ __forceinline__ int64_t gate_row(const NormArgs &a, int64_t r) {
    if (a.gate_rows == 1) return 0;
    if (a.per_gate == 1) return r * a.d;
    const int64_t g = a.rows <= 0xffffffffll ? static_cast<uint32_t>(r) / static_cast<uint32_t>(a.per_gate) : r / a.per_gate;
    return g * a.d;
}

// Rows of up to 32 W * 8 V columns, W warps a row; a block holds one row (W > 1) or four (W = 1).
// A row's loads go out together and the row stays in registers: it is read and written once.  The
// weights come from the first-level cache each time: a thread has no room for its columns' (up to five
// vectors) beside the row.
template <typename S, typename B, int V, int W, bool VEC, bool LAYER>
__global__ void __launch_bounds__(W == 1 ? 128 : 32 * W) peri_forward_kernel(const NormArgs a) {
    __shared__ float parts[4][W];
    constexpr int kRows = W == 1 ? 4 : 1;
    const Columns<VEC> cols{static_cast<int>(threadIdx.x) & (32 * W - 1), 32 * W, a.d};
    const float inv_d = 1.0f / static_cast<float>(a.d);
    for (int64_t r = static_cast<int64_t>(blockIdx.x) * kRows + (W == 1 ? threadIdx.x >> 5 : 0); r < a.rows;
         r += static_cast<int64_t>(gridDim.x) * kRows) {
        Eight<S> x[V];
        Eight<B> f[V];
#pragma unroll
        for (int q = 0; q < V; ++q) cols.load(static_cast<const B *>(a.f) + r * a.ld_f, q, f[q]);
#pragma unroll
        for (int q = 0; q < V; ++q) cols.load(static_cast<const S *>(a.x) + r * a.ld_x, q, x[q]);
        float y[V][8];
        float2 sf = make_float2(0.0f, 0.0f), sy = make_float2(0.0f, 0.0f);
        float sum = 0.0f;
        if constexpr (LAYER) {
#pragma unroll
            for (int q = 0; q < V; ++q)
#pragma unroll
                for (int i = 0; i < 8; ++i) sum += f[q].get(i);
            sf.x = row_sum<W>(sum, parts[0]) * inv_d;
        }
        sum = 0.0f;
#pragma unroll
        for (int q = 0; q < V; ++q)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float z = f[q].get(i) - sf.x;
                if (!LAYER || cols.valid(q, i)) sum = fmaf(z, z, sum);
            }
        sf.y = rsqrtf(fmaf(row_sum<W>(sum, parts[1]), inv_d, a.eps));
        const int64_t gate = a.gate.p ? gate_row(a, r) : 0;
        sum = 0.0f;
#pragma unroll
        for (int q = 0; q < V; ++q) {
            float w[8], t[8];
            a.post_w.load(cols, 0, q, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) t[i] = (f[q].get(i) - sf.x) * sf.y * w[i];
            if (a.post_b.p) {
                a.post_b.load(cols, 0, q, w);
#pragma unroll
                for (int i = 0; i < 8; ++i) t[i] += w[i];
            }
            if (a.gate.p) {
                a.gate.load(cols, gate, q, w);
#pragma unroll
                for (int i = 0; i < 8; ++i) t[i] *= w[i];
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                y[q][i] = fmaf(a.residual_scale, x[q].get(i), t[i]);
                if (LAYER) sum += y[q][i];
            }
            cols.store(static_cast<S *>(a.y) + r * a.ld_y, q, y[q]);
        }
        if constexpr (LAYER) sy.x = row_sum<W>(sum, parts[2]) * inv_d;
        sum = 0.0f;
#pragma unroll
        for (int q = 0; q < V; ++q)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float z = y[q][i] - sy.x;
                if (!LAYER || cols.valid(q, i)) sum = fmaf(z, z, sum);
            }
        sy.y = rsqrtf(fmaf(row_sum<W>(sum, parts[3]), inv_d, a.eps));
#pragma unroll
        for (int q = 0; q < V; ++q) {
            float w[8], h[8];
            a.pre_w.load(cols, 0, q, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) h[i] = (y[q][i] - sy.x) * sy.y * w[i];
            if (a.pre_b.p) {
                a.pre_b.load(cols, 0, q, w);
#pragma unroll
                for (int i = 0; i < 8; ++i) h[i] += w[i];
            }
            cols.store(static_cast<B *>(a.h) + r * a.ld_h, q, h);
        }
        if (a.stats && cols.t == 0) {
            a.stats[r] = sf;
            a.stats[a.rows + r] = sy;
        }
        if (W > 1) __syncthreads();                    // the next row writes parts again
    }
}

template <typename S, typename B, int V, int W, bool VEC>
cudaError_t launch_forward_rows(const NormArgs &a, cudaStream_t stream) {
    constexpr int kRows = W == 1 ? 4 : 1;
    const int64_t blocks = (a.rows + kRows - 1) / kRows;
    const unsigned grid = static_cast<unsigned>(blocks < 0x7fffffff ? blocks : 0x7fffffff);
    auto kernel = a.layer ? peri_forward_kernel<S, B, V, W, VEC, true> : peri_forward_kernel<S, B, V, W, VEC, false>;
    kernel<<<grid, W == 1 ? 128 : 32 * W, 0, stream>>>(a);
    return cudaGetLastError();
}

// As few warps as hold a row at four groups of eight columns a thread.
template <typename S, typename B>
cudaError_t launch_forward(const NormArgs &a, bool vec, cudaStream_t stream) {
    const int groups = (a.d + 255) / 256;              // of a warp's 256 columns
    if (!vec) {
        if (groups <= 1) return launch_forward_rows<S, B, 1, 1, false>(a, stream);
        if (groups <= 4) return launch_forward_rows<S, B, 4, 1, false>(a, stream);
        if (groups <= 16) return launch_forward_rows<S, B, 4, 4, false>(a, stream);
        return launch_forward_rows<S, B, 4, 16, false>(a, stream);
    }
    if (groups <= 1) return launch_forward_rows<S, B, 1, 1, true>(a, stream);
    if (groups <= 2) return launch_forward_rows<S, B, 2, 1, true>(a, stream);
    if (groups <= 3) return launch_forward_rows<S, B, 3, 1, true>(a, stream);
    if (groups <= 4) return launch_forward_rows<S, B, 4, 1, true>(a, stream);
    if (groups <= 8) return launch_forward_rows<S, B, 4, 2, true>(a, stream);
    if (groups <= 16) return launch_forward_rows<S, B, 4, 4, true>(a, stream);
    if (groups <= 32) return launch_forward_rows<S, B, 4, 8, true>(a, stream);
    return launch_forward_rows<S, B, 4, 16, true>(a, stream);
}

__device__ float block_sum(float v) {
    __shared__ float sums[kRowThreads / 32];
    for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = v;
    __syncthreads();
    float t = 0.0f;
    for (int i = 0; i < kRowThreads / 32; ++i) t += sums[i];
    return t;
}

// What backward recomputes of an element of row r.
template <typename S, typename B>
struct Back {
    const NormArgs &a;
    int64_t r;
    const S *y, *dy;
    const B *f, *dh;
    float2 sf, sy;
    __device__ Back(const NormArgs &args, int64_t row) : a(args), r(row) {
        y = static_cast<const S *>(a.y) + r * a.ld_y;
        dy = a.dy ? static_cast<const S *>(a.dy) + r * a.ld_dy : nullptr;
        f = static_cast<const B *>(a.f) + r * a.ld_f;
        dh = static_cast<const B *>(a.dh) + r * a.ld_dh;
        sf = a.stats[r];
        sy = a.stats[a.rows + r];
    }
    __device__ float n_y(int c) const { return (value(y[c]) - sy.x) * sy.y; }
    __device__ float n_f(int c) const { return (value(f[c]) - sf.x) * sf.y; }
    __device__ float q(int c) const { return value(dh[c]) * a.pre_w.get(c); }
    __device__ float gate(int c) const { return a.gate.p ? a.gate.get(r / a.per_gate * a.d + c) : 1.0f; }
    // the gradient of y; means: of q n_y and (layer) of q
    __device__ float total(int c, float2 means) const {
        return (dy ? value(dy[c]) : 0.0f) + sy.y * (q(c) - n_y(c) * means.x - means.y);
    }
};

template <typename S, typename B>
__global__ void __launch_bounds__(kRowThreads) peri_backward_rows_kernel(const NormArgs a) {
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const Back<S, B> k(a, r);
        float qn = 0.0f, q = 0.0f;
        for (int c = threadIdx.x; c < a.d; c += kRowThreads) {
            qn = fmaf(k.q(c), k.n_y(c), qn);
            q += k.q(c);
        }
        const float2 means = make_float2(block_sum(qn) / a.d, a.layer ? block_sum(q) / a.d : 0.0f);
        if (threadIdx.x == 0) a.row_sums[r] = means;
        float un = 0.0f, u = 0.0f;
        for (int c = threadIdx.x; c < a.d; c += kRowThreads) {
            const float t = k.total(c, means);
            const float uc = t * k.gate(c) * a.post_w.get(c);
            un = fmaf(uc, k.n_f(c), un);
            u += uc;
        }
        un = block_sum(un) / a.d;
        u = a.layer ? block_sum(u) / a.d : 0.0f;
        for (int c = threadIdx.x; c < a.d; c += kRowThreads) {
            const float t = k.total(c, means);
            const float uc = t * k.gate(c) * a.post_w.get(c);
            (static_cast<S *>(a.dx) + r * a.ld_dx)[c] = rounded<S>(a.residual_scale * t);
            (static_cast<B *>(a.df) + r * a.ld_df)[c] = rounded<B>(k.sf.y * (uc - k.n_f(c) * un - u));
        }
    }
}

template <typename S, typename B>
__global__ void __launch_bounds__(kRowThreads) peri_backward_columns_kernel(const NormArgs a) {
    const int c = blockIdx.x * kRowThreads + threadIdx.x;
    if (c >= a.d) return;
    float pre_w = 0.0f, pre_b = 0.0f, post_w = 0.0f, post_b = 0.0f, gate = 0.0f;
    for (int64_t r = 0; r < a.rows; ++r) {
        const Back<S, B> k(a, r);
        const float t = k.total(c, a.row_sums[r]), dz = t * k.gate(c), n = k.n_f(c), dh = value(k.dh[c]);
        pre_w = fmaf(dh, k.n_y(c), pre_w);
        pre_b += dh;
        post_w = fmaf(dz, n, post_w);
        post_b += dz;
        if (a.gate.p) {
            gate = fmaf(t, fmaf(n, a.post_w.get(c), a.post_b.p ? a.post_b.get(c) : 0.0f), gate);
            if ((r + 1) % a.per_gate == 0) {
                a.d_gate.set(r / a.per_gate * a.d + c, gate);
                gate = 0.0f;
            }
        }
    }
    a.d_pre_w.set(c, pre_w);
    a.d_post_w.set(c, post_w);
    if (a.post_b.p) {
        a.d_pre_b.set(c, pre_b);
        a.d_post_b.set(c, post_b);
    }
}

template <typename S, typename B>
cudaError_t launch_backward(const NormArgs &a, cudaStream_t stream) {
    const unsigned grid = static_cast<unsigned>(a.rows < 65536 ? a.rows : 65536);
    if (a.rows > 0) peri_backward_rows_kernel<S, B><<<grid, kRowThreads, 0, stream>>>(a);
    peri_backward_columns_kernel<S, B><<<(a.d + kRowThreads - 1) / kRowThreads, kRowThreads, 0, stream>>>(a);
    return cudaGetLastError();
}

// ---------------------------------------------------------------- arguments

struct Range {
    explicit Range(const char *name) { nvtxRangePushA(name); }
    ~Range() { nvtxRangePop(); }
    Range(const Range &) = delete;
    Range &operator=(const Range &) = delete;
};

int invalid(const char *what) {
    char msg[128];
    snprintf(msg, sizeof msg, "peri_norm: %s", what);
    return set_thread_error(MTDAO_ERR_INVALID, msg);
}

bool is_type(int32_t t) { return t == MTDAO_F32 || t == MTDAO_BF16; }
uintptr_t size_of(int32_t t) { return t == MTDAO_BF16 ? 2 : 4; }
bool aligned(const void *p, int32_t type) { return reinterpret_cast<uintptr_t>(p) % size_of(type) == 0; }

// Whether every row starts at a multiple of eight elements.
bool by_eight(const void *p, int64_t ld, int32_t type) {
    return reinterpret_cast<uintptr_t>(p) % (8 * size_of(type)) == 0 && ld % 8 == 0;
}

int check_shape(const mtdao_peri_norm *s, bool backward) {
    if (s == nullptr) return invalid("the description is NULL");
    if (s->rows < 0 || s->rows > (int64_t(1) << 40)) return invalid("rows outside 0 .. 2^40");
    if (s->d < 1 || s->d > MTDAO_PERI_NORM_MAX_D) return invalid("d outside 1 .. MTDAO_PERI_NORM_MAX_D");
    if (s->norm != MTDAO_NORM_RMS && s->norm != MTDAO_NORM_LAYER) return invalid("unknown norm");
    if (!is_type(s->stream_dtype) || !is_type(s->branch_dtype) || !is_type(s->weight_dtype) ||
        (s->gate_rows != 0 && !is_type(s->gate_dtype)))
        return invalid("unknown type");
    if (s->stream_dtype == MTDAO_BF16 && s->branch_dtype != MTDAO_BF16)
        return invalid("a bf16 stream takes a bf16 branch");
    if (!(std::isfinite(s->eps) && s->eps >= 0.0) || !std::isfinite(s->residual_scale))
        return invalid("eps and residual_scale must be finite, eps not negative");
    if (s->gate_rows < 0 || s->gate_rows > (int64_t(1) << 40) || (s->gate_rows > 0 && s->rows > 0 && s->rows % s->gate_rows != 0))
        return invalid("gate_rows must divide rows");
    const int64_t lds[] = {s->ld_f, s->ld_y, backward ? s->ld_dy : s->ld_x, backward ? s->ld_dh : s->ld_h,
                           backward ? s->ld_dx : s->ld_x, backward ? s->ld_df : s->ld_h};
    for (int64_t ld : lds)
        if (ld < s->d || ld > (int64_t(1) << 40)) return invalid("a row stride is smaller than d, or over 2^40");
    return MTDAO_OK;
}

NormArgs arguments(const mtdao_peri_norm *s) {
    NormArgs a = {};
    a.rows = s->rows;
    a.gate_rows = s->gate_rows;
    a.per_gate = s->gate_rows > 0 && s->rows > 0 ? s->rows / s->gate_rows : 1;
    a.d = s->d;
    a.layer = s->norm == MTDAO_NORM_LAYER;
    a.eps = static_cast<float>(s->eps);
    a.residual_scale = static_cast<float>(s->residual_scale);
    a.ld_x = s->ld_x, a.ld_f = s->ld_f, a.ld_y = s->ld_y, a.ld_h = s->ld_h;
    a.ld_dy = s->ld_dy, a.ld_dh = s->ld_dh, a.ld_dx = s->ld_dx, a.ld_df = s->ld_df;
    return a;
}

Vector vector_of(const void *p, int32_t type) { return Vector{const_cast<void *>(p), type == MTDAO_BF16}; }

int done(cudaError_t e, const char *what) {
    if (e == cudaSuccess) return MTDAO_OK;
    char msg[256];
    snprintf(msg, sizeof msg, "%s: %s", what, cudaGetErrorString(e));
    return set_thread_error(MTDAO_ERR_CUDA, msg);
}

}  // namespace
}  // namespace mtdao

using namespace mtdao;

extern "C" int mtdao_peri_norm_forward(const mtdao_peri_norm *s, const void *x, const void *f, const void *post_w,
                                       const void *post_b, const void *pre_w, const void *pre_b, const void *gate,
                                       void *y, void *h, float *stats, void *cuda_stream) {
    if (int rc = check_shape(s, false)) return rc;
    if ((post_b == nullptr) != (pre_b == nullptr)) return invalid("post_b and pre_b come together");
    if ((gate == nullptr) != (s->gate_rows == 0)) return invalid("a gate needs gate_rows, and none without it");
    if (s->rows == 0) return MTDAO_OK;
    if (!x || !f || !post_w || !pre_w || !y || !h) return invalid("a pointer is NULL");
    if (!aligned(x, s->stream_dtype) || !aligned(y, s->stream_dtype) || !aligned(f, s->branch_dtype) ||
        !aligned(h, s->branch_dtype) || !aligned(post_w, s->weight_dtype) || !aligned(post_b, s->weight_dtype) ||
        !aligned(pre_w, s->weight_dtype) || !aligned(pre_b, s->weight_dtype) || (gate && !aligned(gate, s->gate_dtype)) ||
        reinterpret_cast<uintptr_t>(stats) % 8)
        return set_thread_error(MTDAO_ERR_ALIGN, "peri_norm: a pointer is not aligned to its type (stats: 8 bytes)");
    Range range("mtdao_peri_norm_forward");
    NormArgs a = arguments(s);
    a.x = x, a.f = f, a.y = y, a.h = h;
    a.post_w = vector_of(post_w, s->weight_dtype);
    a.post_b = vector_of(post_b, s->weight_dtype);
    a.pre_w = vector_of(pre_w, s->weight_dtype);
    a.pre_b = vector_of(pre_b, s->weight_dtype);
    a.gate = vector_of(gate, s->gate_dtype);
    a.stats = reinterpret_cast<float2 *>(stats);
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const int32_t st = s->stream_dtype, br = s->branch_dtype, wt = s->weight_dtype;
    const bool vec = s->d % 8 == 0 && by_eight(x, s->ld_x, st) && by_eight(y, s->ld_y, st) && by_eight(f, s->ld_f, br) &&
                     by_eight(h, s->ld_h, br) && by_eight(post_w, 8, wt) && by_eight(post_b, 8, wt) &&
                     by_eight(pre_w, 8, wt) && by_eight(pre_b, 8, wt) && (!gate || by_eight(gate, 8, s->gate_dtype));
    const cudaError_t e = st == MTDAO_BF16   ? launch_forward<Bf16, Bf16>(a, vec, stream)
                          : br == MTDAO_BF16 ? launch_forward<float, Bf16>(a, vec, stream)
                                             : launch_forward<float, float>(a, vec, stream);
    return done(e, "peri_norm forward");
}

extern "C" int64_t mtdao_peri_norm_workspace(const mtdao_peri_norm *s) {
    if (check_shape(s, true)) return -1;
    return s->rows * 8;
}

extern "C" int mtdao_peri_norm_backward(const mtdao_peri_norm *s, const void *dh, const void *dy, const void *y,
                                        const void *f, const float *stats, const void *post_w, const void *post_b,
                                        const void *pre_w, const void *gate, void *dx, void *df, void *d_post_w,
                                        void *d_post_b, void *d_pre_w, void *d_pre_b, void *d_gate, void *workspace,
                                        int64_t workspace_bytes, void *cuda_stream) {
    if (int rc = check_shape(s, true)) return rc;
    if ((post_b == nullptr) != (d_post_b == nullptr) || (post_b == nullptr) != (d_pre_b == nullptr))
        return invalid("post_b, d_post_b and d_pre_b come together");
    if ((gate == nullptr) != (s->gate_rows == 0) || (gate == nullptr) != (d_gate == nullptr))
        return invalid("gate, d_gate and gate_rows come together");
    if (!post_w || !pre_w || !d_post_w || !d_pre_w) return invalid("a pointer is NULL");
    if (s->rows > 0 && (!dh || !y || !f || !stats || !dx || !df)) return invalid("a pointer is NULL");
    const int32_t st = s->stream_dtype, br = s->branch_dtype, wt = s->weight_dtype;
    if (!aligned(dy, st) || !aligned(y, st) || !aligned(dx, st) || !aligned(dh, br) || !aligned(f, br) ||
        !aligned(df, br) || !aligned(post_w, wt) || !aligned(post_b, wt) || !aligned(pre_w, wt) ||
        !aligned(d_post_w, wt) || !aligned(d_post_b, wt) || !aligned(d_pre_w, wt) || !aligned(d_pre_b, wt) ||
        (gate && (!aligned(gate, s->gate_dtype) || !aligned(d_gate, s->gate_dtype))) ||
        reinterpret_cast<uintptr_t>(stats) % 8 || reinterpret_cast<uintptr_t>(workspace) % 16)
        return set_thread_error(MTDAO_ERR_ALIGN,
                                "peri_norm: a pointer is not aligned to its type (stats: 8 bytes, workspace: 16)");
    const int64_t need = mtdao_peri_norm_workspace(s);
    if (workspace_bytes < need || (need > 0 && workspace == nullptr)) return invalid("the workspace is too small");
    Range range("mtdao_peri_norm_backward");
    NormArgs a = arguments(s);
    a.dh = dh, a.dy = dy, a.y = const_cast<void *>(y), a.f = f, a.dx = dx, a.df = df;
    a.stats = reinterpret_cast<float2 *>(const_cast<float *>(stats));
    a.post_w = vector_of(post_w, wt), a.post_b = vector_of(post_b, wt), a.pre_w = vector_of(pre_w, wt);
    a.gate = vector_of(gate, s->gate_dtype);
    a.d_post_w = vector_of(d_post_w, wt), a.d_post_b = vector_of(d_post_b, wt);
    a.d_pre_w = vector_of(d_pre_w, wt), a.d_pre_b = vector_of(d_pre_b, wt);
    a.d_gate = vector_of(d_gate, s->gate_dtype);
    a.row_sums = static_cast<float2 *>(workspace);
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (s->rows == 0 && gate) {
        const cudaError_t e = cudaMemsetAsync(d_gate, 0, static_cast<size_t>(s->gate_rows) * s->d * size_of(s->gate_dtype), stream);
        if (e != cudaSuccess) return done(e, "peri_norm backward");
    }
    const cudaError_t e = st == MTDAO_BF16   ? launch_backward<Bf16, Bf16>(a, stream)
                          : br == MTDAO_BF16 ? launch_backward<float, Bf16>(a, stream)
                                             : launch_backward<float, float>(a, stream);
    return done(e, "peri_norm backward");
}
