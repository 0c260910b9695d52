// peri_norm_forward.cuh -- the Peri-LN residual update (formulas in mtdao.h).
#pragma once

#include "peri_norm.cuh"

namespace mtdao {
namespace {

// The sum over a row's L lanes (W = 1) or W warps, the same in each of its threads.  parts: W floats of the
// row's, not read by anyone since the last barrier but one.
template <int W, int L>
__device__ __forceinline__ float row_sum(float v, float *parts) {
#pragma unroll
    for (int off = L / 2; off > 0; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
    if constexpr (W == 1) return v;
    if ((threadIdx.x & 31) == 0) parts[threadIdx.x >> 5] = v;
    __syncthreads();
    float t = 0.0f;
#pragma unroll
    for (int i = 0; i < W; ++i) t += parts[i];
    return t;
}

// Rows of up to 8 V columns a thread, over L lanes (W = 1: d <= 64 and 128 take 8 and 16, 21 -> 92 %
// of the memory's rate at d = 64) or W warps; a thread block holds one row (W > 1) or 128 / L.
// A row's loads go out together and the row stays in registers: it is read and written once.  The
// weights come from the first-level cache each time: a thread has no room for its columns' (up to five
// vectors) beside the row.  (Asynchronous copies to shared memory, one to four rows ahead, were slower, 50 to 80 % of the
// memory's rate against 78 to 91: they leave the first-level cache no room for the weights.)
template <typename S, typename B, int V, int W, int L, bool VEC, bool LAYER>
__global__ void __launch_bounds__(W == 1 ? 128 : 32 * W) peri_forward_kernel(const NormArgs a) {
    __shared__ float parts[4][W];
    constexpr int kThreads = W == 1 ? L : 32 * W, kRows = W == 1 ? 128 / L : 1;
    const Columns<VEC> cols{static_cast<int>(threadIdx.x) % kThreads, kThreads, a.d};
    const float inv_d = 1.0f / static_cast<float>(a.d);
    // a warp's lanes stay together: rows past the last are worked on as zeros, and not written
    const int64_t step = static_cast<int64_t>(gridDim.x) * kRows;
    for (int64_t base = static_cast<int64_t>(blockIdx.x) * kRows; base < a.rows; base += step) {
        const int64_t r = base + threadIdx.x / kThreads;
        const bool live = kRows == 1 || r < a.rows;
        Eight<S> x[V];
        Eight<B> f[V];
#pragma unroll
        for (int q = 0; q < V; ++q)
            if (live) cols.load(static_cast<const B *>(a.f) + r * a.ld_f, q, f[q]); else f[q].zero();
#pragma unroll
        for (int q = 0; q < V; ++q)
            if (live) cols.load(static_cast<const S *>(a.x) + r * a.ld_x, q, x[q]); else x[q].zero();
        float y[V][8];
        float2 sf = make_float2(0.0f, 0.0f), sy = make_float2(0.0f, 0.0f);
        float sum = 0.0f;
        if constexpr (LAYER) {
#pragma unroll
            for (int q = 0; q < V; ++q)
#pragma unroll
                for (int i = 0; i < 8; ++i) sum += f[q].get(i);
            sf.x = row_sum<W, L>(sum, parts[0]) * inv_d;
        }
        sum = 0.0f;
#pragma unroll
        for (int q = 0; q < V; ++q)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float z = f[q].get(i) - sf.x;
                if (!LAYER || cols.valid(q, i)) sum = fmaf(z, z, sum);
            }
        sf.y = rsqrtf(fmaf(row_sum<W, L>(sum, parts[1]), inv_d, a.eps));
        const int64_t gate = a.gate.p && live ? gate_row(a, r) : 0;
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
            if (live) cols.store(static_cast<S *>(a.y) + r * a.ld_y, q, y[q]);
        }
        if constexpr (LAYER) sy.x = row_sum<W, L>(sum, parts[2]) * inv_d;
        sum = 0.0f;
#pragma unroll
        for (int q = 0; q < V; ++q)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float z = y[q][i] - sy.x;
                if (!LAYER || cols.valid(q, i)) sum = fmaf(z, z, sum);
            }
        sy.y = rsqrtf(fmaf(row_sum<W, L>(sum, parts[3]), inv_d, a.eps));
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
            if (live) cols.store(static_cast<B *>(a.h) + r * a.ld_h, q, h);
        }
        if (a.stats && live && cols.t == 0) {
            a.stats[r] = sf;
            a.stats[a.rows + r] = sy;
        }
        if (W > 1) __syncthreads();                    // the next row writes parts again
    }
}

template <typename S, typename B, int V, int W, int L, bool VEC>
cudaError_t launch_forward_rows(const NormArgs &a, cudaStream_t stream) {
    constexpr int kRows = W == 1 ? 128 / L : 1;
    const int64_t blocks = (a.rows + kRows - 1) / kRows;
    const unsigned grid = static_cast<unsigned>(blocks < 0x7fffffff ? blocks : 0x7fffffff);
    auto kernel = a.layer ? peri_forward_kernel<S, B, V, W, L, VEC, true> : peri_forward_kernel<S, B, V, W, L, VEC, false>;
    kernel<<<grid, W == 1 ? 128 : 32 * W, 0, stream>>>(a);
    return cudaGetLastError();
}

}  // namespace

// As few warps as hold a row at four groups of eight columns a thread: more threads a row wait for one
// another more (d = 2048, bf16: four groups 6050 GB/s, two 5151, one 4143).
template <typename S, typename B>
cudaError_t launch_peri_forward(const NormArgs &a, bool vec, cudaStream_t stream) {
    const int groups = (a.d + 255) / 256;              // of a warp's 256 columns
    if (!vec) {
        if (groups <= 1) return launch_forward_rows<S, B, 1, 1, 32, false>(a, stream);
        if (groups <= 4) return launch_forward_rows<S, B, 4, 1, 32, false>(a, stream);
        if (groups <= 16) return launch_forward_rows<S, B, 4, 4, 32, false>(a, stream);
        return launch_forward_rows<S, B, 4, 16, 32, false>(a, stream);
    }
    if (a.d <= 64) return launch_forward_rows<S, B, 1, 1, 8, true>(a, stream);
    if (a.d <= 128) return launch_forward_rows<S, B, 1, 1, 16, true>(a, stream);
    if (groups <= 1) return launch_forward_rows<S, B, 1, 1, 32, true>(a, stream);
    if (groups <= 2) return launch_forward_rows<S, B, 2, 1, 32, true>(a, stream);
    if (groups <= 3) return launch_forward_rows<S, B, 3, 1, 32, true>(a, stream);
    if (groups <= 4) return launch_forward_rows<S, B, 4, 1, 32, true>(a, stream);
    if (groups <= 6) return launch_forward_rows<S, B, 3, 2, 32, true>(a, stream);
    if (groups <= 8) return launch_forward_rows<S, B, 4, 2, 32, true>(a, stream);
    if (groups <= 16) return launch_forward_rows<S, B, 4, 4, 32, true>(a, stream);
    if (groups <= 32) return launch_forward_rows<S, B, 4, 8, 32, true>(a, stream);
    return launch_forward_rows<S, B, 4, 16, 32, true>(a, stream);
}

}  // namespace mtdao
