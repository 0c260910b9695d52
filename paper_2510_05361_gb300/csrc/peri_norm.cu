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

// A vector whose type is known at the launch only: weights, gate and their gradients.
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

// Mean and reciprocal deviation of the row whose column c get(c) gives.
template <typename Get>
__device__ float2 row_stats(const NormArgs &a, Get get) {
    float mean = 0.0f, q = 0.0f;
    if (a.layer) {
        for (int c = threadIdx.x; c < a.d; c += kRowThreads) mean += get(c);
        mean = block_sum(mean) / a.d;
    }
    for (int c = threadIdx.x; c < a.d; c += kRowThreads) {
        const float z = get(c) - mean;
        q = fmaf(z, z, q);
    }
    return make_float2(mean, 1.0f / sqrtf(block_sum(q) / a.d + a.eps));
}

template <typename S, typename B>
__global__ void __launch_bounds__(kRowThreads) peri_forward_kernel(const NormArgs a) {
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const S *x = static_cast<const S *>(a.x) + r * a.ld_x;
        const B *f = static_cast<const B *>(a.f) + r * a.ld_f;
        const float2 sf = row_stats(a, [&](int c) { return value(f[c]); });
        auto y_of = [&](int c) {
            float z = (value(f[c]) - sf.x) * sf.y * a.post_w.get(c);
            if (a.post_b.p) z += a.post_b.get(c);
            if (a.gate.p) z *= a.gate.get(r / a.per_gate * a.d + c);
            return fmaf(a.residual_scale, value(x[c]), z);
        };
        const float2 sy = row_stats(a, y_of);
        for (int c = threadIdx.x; c < a.d; c += kRowThreads) {
            const float y = y_of(c);
            float h = (y - sy.x) * sy.y * a.pre_w.get(c);
            if (a.pre_b.p) h += a.pre_b.get(c);
            (static_cast<S *>(a.y) + r * a.ld_y)[c] = rounded<S>(y);
            (static_cast<B *>(a.h) + r * a.ld_h)[c] = rounded<B>(h);
        }
        if (a.stats && threadIdx.x == 0) {
            a.stats[r] = sf;
            a.stats[a.rows + r] = sy;
        }
    }
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
cudaError_t launch_forward(const NormArgs &a, cudaStream_t stream) {
    const unsigned grid = static_cast<unsigned>(a.rows < 65536 ? a.rows : 65536);
    peri_forward_kernel<S, B><<<grid, kRowThreads, 0, stream>>>(a);
    return cudaGetLastError();
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
    const cudaError_t e = s->stream_dtype == MTDAO_BF16   ? launch_forward<Bf16, Bf16>(a, stream)
                          : s->branch_dtype == MTDAO_BF16 ? launch_forward<float, Bf16>(a, stream)
                                                          : launch_forward<float, float>(a, stream);
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
