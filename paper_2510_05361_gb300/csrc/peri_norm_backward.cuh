// peri_norm_backward.cuh -- the gradients of the Peri-LN residual update (formulas in mtdao.h).
//
// One pass over the rows.  A thread has the same eight columns of every row that its worker takes (a
// worker: the warps of one row, in one thread block or a cluster of them), so that the sums over rows which
// the weights' gradients are stay in its registers; a row's own two sums (of the norm before the
// block, then of the one after it) go over the worker's warps.  The next row is on its way while one is worked on.
// Four sums a column: of dh n_y, dh, dY n_f, dY, from which a gate that is the
// same for the rows summed gives its own gradient and the norm's (post_w S is the gate's, gate S the weight's).
//
// Workspace: [blocks][d] for the first two sums each, then for the other two the same.  Where several
// rows share a gate row and there are many gate rows, a worker takes whole ones, writes their gradients itself
// and keeps the weight's sums, [workers][d].  Where there are few (split), a gate row's sums come
// from several workers: [workers + gate rows][d], a worker's part of gate row g at worker +
// g, which no other pair of the two shares, as both only grow along the rows.  A second kernel adds in order.
#pragma once

#include <cooperative_groups.h>

#include "peri_norm.cuh"

namespace mtdao {
namespace {

template <typename S, typename B>
struct BackRow {
    Eight<S> y, dy;
    Eight<B> dh, f;
    float2 sf, sy;
};

template <int W, int G, int C>
struct RowSums {
    float parts[G][2][2][W * C];                       // worker's row, use, value
    static constexpr int kWarps = W * C;

    // Sums of N values over the worker's warps; use: 0 and 1 in turn, so that one barrier each is enough.
    template <int N>
    __device__ __forceinline__ void add(float (&v)[N], int use) {
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int off = 16; off > 0; off >>= 1) v[n] += __shfl_xor_sync(0xffffffffu, v[n], off);
        if constexpr (kWarps > 1) {
            const int lane = threadIdx.x & 31, group = threadIdx.x / (32 * W), warp = threadIdx.x / 32 % W;
            if constexpr (C > 1) {
                auto cluster = cooperative_groups::this_cluster();
                const int rank = static_cast<int>(cluster.block_rank());
#pragma unroll
                for (int n = 0; n < N; ++n)
                    if (lane < C) *cluster.map_shared_rank(&parts[group][use][n][rank * W + warp], lane) = v[n];
                cluster.sync();
            } else {
                if (lane == 0) {
#pragma unroll
                    for (int n = 0; n < N; ++n) parts[group][use][n][warp] = v[n];
                }
                if constexpr (G == 1)
                    __syncthreads();
                else
                    asm volatile("bar.sync %0, %1;" :: "r"(group + 1), "n"(32 * W) : "memory");
            }
#pragma unroll
            for (int n = 0; n < N; ++n) {
                if constexpr (kWarps <= 8) {
                    v[n] = 0.0f;
#pragma unroll
                    for (int i = 0; i < kWarps; ++i) v[n] += parts[group][use][n][i];
                } else {
                    v[n] = 0.0f;
#pragma unroll
                    for (int i = 0; i < kWarps; i += 32)
                        if (i + lane < kWarps) v[n] += parts[group][use][n][i + lane];
#pragma unroll
                    for (int off = 16; off > 0; off >>= 1) v[n] += __shfl_xor_sync(0xffffffffu, v[n], off);
                }
            }
        }
    }
};

// FULL: "layer" norm or biases; else the sums of dh and dY and the means are left out.
template <typename S, typename B, int W, int G, int C, bool VEC, bool FULL>
__global__ void __launch_bounds__(32 * W * G, W == 16 ? 1 : 2) peri_backward_kernel(const NormArgs a) {
    constexpr int kSums = FULL ? 4 : 2;                 // A, S or A, S, B, D
    __shared__ RowSums<W, G, C> sums;
    __shared__ float joined[G > 1 ? 32 * W * G * 8 : 1];
    const int group = threadIdx.x / (32 * W);
    const int rank = C > 1 ? static_cast<int>(cooperative_groups::this_cluster().block_rank()) : 0;
    const int64_t block = blockIdx.x / C, worker = block * G + group, workers = static_cast<int64_t>(gridDim.x / C) * G;
    const Columns<VEC> cols{rank * 32 * W + static_cast<int>(threadIdx.x) % (32 * W), 32 * W * C, a.d};
    const float inv_d = 1.0f / static_cast<float>(a.d);
    const int kind = gate_kind(a);

    int64_t r = worker, end = a.rows, step = workers;
    if (a.contiguous) {
        const int64_t unit = a.split ? 1 : a.per_gate, units = a.rows / unit, most = (units + workers - 1) / workers;
        r = min(units, worker * most) * unit;
        end = min(units, (worker + 1) * most) * unit;
        step = 1;
    }
    float pre_w[8], through[8], sum[kSums][8];           // through: post_w times the gate of the rows
    a.pre_w.load(cols, 0, 0, pre_w);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
#pragma unroll
        for (int k = 0; k < kSums; ++k) sum[k][i] = 0.0f;
    }
    auto set_gate = [&](int64_t row) {
        a.post_w.load(cols, 0, 0, through);
        if (kind == kGateNone || kind == kGateElement) return;
        float g[8];
        a.gate.load(cols, gate_row(a, row), 0, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) through[i] *= g[i];
    };
    auto load = [&](int64_t row, BackRow<S, B> &in) {
        cols.load(static_cast<const B *>(a.dh) + row * a.ld_dh, 0, in.dh);
        cols.load(static_cast<const S *>(a.y) + row * a.ld_y, 0, in.y);
        if (a.dy) cols.load(static_cast<const S *>(a.dy) + row * a.ld_dy, 0, in.dy); else in.dy.zero();
        cols.load(static_cast<const B *>(a.f) + row * a.ld_f, 0, in.f);
        in.sf = __ldg(a.stats + row);
        in.sy = __ldg(a.stats + a.rows + row);
    };
    // row k of the workspace's array n (0: A, 1: B, then S and D)
    auto place = [&](int n, int64_t k) {
        const int64_t blocks = gridDim.x / C, rows = kind != kGateRows ? blocks : a.split ? workers + a.gate_rows : workers;
        return a.partial + (n < 2 ? n * blocks + k : 2 * blocks + (n - 2) * rows + k) * a.d;
    };
    // what S and D hold at the end of gate row g
    auto end_gate = [&](int64_t g) {
        float gate[8], w[8], b[8], out[8];
        if (a.split) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (cols.valid(0, i)) {
                    place(2, worker + g)[cols.at(0, i)] = sum[1][i];
                    if (FULL) place(3, worker + g)[cols.at(0, i)] = sum[FULL ? 3 : 0][i];
                }
        } else {
            a.gate.load(cols, g * a.d, 0, gate);
            a.post_w.load(cols, 0, 0, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) out[i] = w[i] * sum[1][i], b[i] = 0.0f;
            if (FULL && a.post_b.p) {
                a.post_b.load(cols, 0, 0, b);
#pragma unroll
                for (int i = 0; i < 8; ++i) out[i] = fmaf(b[i], sum[FULL ? 3 : 0][i], out[i]);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (cols.valid(0, i)) {
                    a.d_gate.set(g * a.d + cols.at(0, i), out[i]);
                    // the weight's and the bias's sums go on in the worker's place
                    place(2, worker)[cols.at(0, i)] += gate[i] * sum[1][i];
                    if (FULL) place(3, worker)[cols.at(0, i)] += gate[i] * sum[FULL ? 3 : 0][i];
                }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            sum[1][i] = 0.0f;
            if (FULL) sum[FULL ? 3 : 0][i] = 0.0f;
        }
    };

    if constexpr (C > 1) cooperative_groups::this_cluster().sync();   // every block of the cluster runs
    set_gate(min(r, a.rows - 1));
    int64_t g = kind == kGateRows ? r / a.per_gate : 0, g_end = (g + 1) * a.per_gate;
    BackRow<S, B> now, next;
    if (r < end) load(r, now);
    for (; r < end; r += step) {
        if (r + step < end) load(r + step, next);
        float each[8], w[8], b[8];
        if (kind == kGateElement) a.gate.load(cols, r * a.d, 0, each);
        float q[8], t[8], v1[FULL ? 2 : 1] = {};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float dh = now.dh.get(i), n = (now.y.get(i) - now.sy.x) * now.sy.y;
            q[i] = dh * pre_w[i];
            t[i] = n;
            v1[0] = fmaf(q[i], n, v1[0]);
            sum[0][i] = fmaf(dh, n, sum[0][i]);
            if (FULL) {
                v1[FULL ? 1 : 0] += q[i];
                sum[FULL ? 2 : 0][i] += dh;
            }
        }
        sums.add(v1, 0);
        const float m1 = v1[0] * inv_d, m2 = FULL && a.layer ? v1[FULL ? 1 : 0] * inv_d : 0.0f;
        float out[8], v2[FULL ? 2 : 1] = {};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            t[i] = fmaf(now.sy.y, q[i] - t[i] * m1 - m2, now.dy.get(i));              // dY
            out[i] = a.residual_scale * t[i];
        }
        cols.store(static_cast<S *>(a.dx) + r * a.ld_dx, 0, out);
        if (kind == kGateElement) {
            a.post_w.load(cols, 0, 0, w);
            if (FULL && a.post_b.p) a.post_b.load(cols, 0, 0, b);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float z = (now.f.get(i) - now.sf.x) * now.sf.y * w[i];
                if (FULL && a.post_b.p) z += b[i];
                out[i] = t[i] * z;
                t[i] *= each[i];                                                     // dz
            }
            if (VEC) {
                if (a.d_gate.bf16) cols.store(static_cast<Bf16 *>(a.d_gate.p) + r * a.d, 0, out);
                else cols.store(static_cast<float *>(a.d_gate.p) + r * a.d, 0, out);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (cols.valid(0, i)) a.d_gate.set(r * a.d + cols.at(0, i), out[i]);
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float n = (now.f.get(i) - now.sf.x) * now.sf.y;
            sum[1][i] = fmaf(t[i], n, sum[1][i]);
            if (FULL) sum[FULL ? 3 : 0][i] += t[i];
            q[i] = t[i] * through[i];
            v2[0] = fmaf(q[i], n, v2[0]);
            if (FULL) v2[FULL ? 1 : 0] += q[i];
        }
        sums.add(v2, 1);
        const float m3 = v2[0] * inv_d, m4 = FULL && a.layer ? v2[FULL ? 1 : 0] * inv_d : 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float n = (now.f.get(i) - now.sf.x) * now.sf.y;
            out[i] = now.sf.y * (q[i] - n * m3 - m4);
        }
        cols.store(static_cast<B *>(a.df) + r * a.ld_df, 0, out);
        if (kind == kGateRows) {
            const bool last = r + 1 == end;
            if (last || r + 1 == g_end) {
                end_gate(g);
                ++g, g_end += a.per_gate;
                if (!last) set_gate(r + 1);
            }
        }
        now = next;
    }

    // the block's rows of the workspace: its groups' sums, added in their order
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kSums; ++k) {
        if (k % 2 == 1 && kind == kGateRows) continue;             // S and D are there already
        const int array = kSums == 2 ? 2 * k : k % 2 * 2 + k / 2;    // A 0, B 1, S 2, D 3
        if constexpr (G > 1) {
#pragma unroll
            for (int i = 0; i < 8; ++i) joined[threadIdx.x * 8 + i] = sum[k][i];
            __syncthreads();
            if (group == 0) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    float v = 0.0f;
#pragma unroll
                    for (int g = 0; g < G; ++g) v += joined[(g * 32 * W + threadIdx.x) * 8 + i];
                    if (cols.valid(0, i)) place(array, block)[cols.at(0, i)] = v;
                }
            }
            __syncthreads();
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (cols.valid(0, i)) place(array, block)[cols.at(0, i)] = sum[k][i];
        }
    }
    if constexpr (C > 1) cooperative_groups::this_cluster().sync();   // nobody's shared memory goes while it may be written
}

// The sums over the workspace's rows, 32 columns a thread block, eight threads a column.
template <typename S>
__global__ void __launch_bounds__(256) peri_backward_sums_kernel(const NormArgs a, int64_t blocks, int64_t workers, bool full) {
    __shared__ float parts[8][33];
    const int c = blockIdx.x * 32 + (threadIdx.x & 31), part = threadIdx.x >> 5;
    const bool valid = c < a.d;
    const int kind = gate_kind(a);
    auto reduce = [&](float v) {
        __syncthreads();
        parts[part][threadIdx.x & 31] = v;
        __syncthreads();
        float t = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) t += parts[i][threadIdx.x & 31];
        return t;
    };
    auto column = [&](const float *p, int64_t lo, int64_t hi) {
        float v = 0.0f;
        if (valid)
            for (int64_t k = lo + part; k < hi; k += 8) v += p[k * a.d + c];
        return reduce(v);
    };
    const float *A = a.partial, *Bs = A + blocks * a.d, *Ss = Bs + blocks * a.d;
    const int64_t rows = kind == kGateRows ? (a.split ? workers + a.gate_rows : workers) : blocks;
    const float *Ds = Ss + rows * a.d;
    const float pre_w = column(A, 0, blocks), pre_b = full ? column(Bs, 0, blocks) : 0.0f;
    float post_w = 0.0f, post_b = 0.0f;
    if (kind == kGateRows && a.split) {
        const float w = valid ? a.post_w.get(c) : 0.0f, b = valid && a.post_b.p ? a.post_b.get(c) : 0.0f;
        const int64_t most = (a.rows + workers - 1) / workers;         // rows of a worker
        for (int64_t g = part; valid && g < a.gate_rows; g += 8) {      // gate rows over the column's threads
            const int64_t lo = g * a.per_gate / most + g, hi = ((g + 1) * a.per_gate - 1) / most + g + 1;
            float s = 0.0f, d = 0.0f;
            for (int64_t k = lo; k < hi; ++k) {
                s += Ss[k * a.d + c];
                if (full) d += Ds[k * a.d + c];
            }
            const float gate = a.gate.get(g * a.d + c);
            post_w = fmaf(gate, s, post_w);
            post_b = fmaf(gate, d, post_b);
            a.d_gate.set(g * a.d + c, fmaf(w, s, b * d));
        }
        post_w = reduce(post_w);
        post_b = reduce(post_b);
    } else {
        post_w = column(Ss, 0, rows);
        post_b = full ? column(Ds, 0, rows) : 0.0f;
        if (kind == kGateChannel && valid) {
            const float gate = a.gate.get(c), b = a.post_b.p ? a.post_b.get(c) : 0.0f;
            if (part == 0) a.d_gate.set(c, fmaf(a.post_w.get(c), post_w, b * post_b));
            post_w *= gate;
            post_b *= gate;
        }
    }
    if (!valid || part != 0) return;
    a.d_pre_w.set(c, pre_w);
    a.d_post_w.set(c, post_w);
    if (a.post_b.p) {
        a.d_pre_b.set(c, pre_b);
        a.d_post_b.set(c, post_b);
    }
}

template <typename S, typename B, int W, int C, bool VEC>
cudaError_t launch_backward_rows(const NormArgs &a, const BackwardPlan &p, cudaStream_t stream) {
    constexpr int G = W == 1 ? 8 : W == 2 ? 4 : W <= 4 ? 2 : 1;
    auto kernel = a.layer || a.post_b.p ? peri_backward_kernel<S, B, W, G, C, VEC, true> : peri_backward_kernel<S, B, W, G, C, VEC, false>;
    cudaLaunchConfig_t config = {};
    config.gridDim = dim3(static_cast<unsigned>(p.blocks * C));
    config.blockDim = dim3(32 * W * G);
    config.stream = stream;
    cudaLaunchAttribute cluster;
    cluster.id = cudaLaunchAttributeClusterDimension;
    cluster.val.clusterDim.x = C;
    cluster.val.clusterDim.y = cluster.val.clusterDim.z = 1;
    config.attrs = &cluster;
    config.numAttrs = C > 1 ? 1 : 0;
    return cudaLaunchKernelEx(&config, kernel, a);
}

}  // namespace

template <typename S, typename B>
cudaError_t launch_peri_backward(const NormArgs &args, bool vec, cudaStream_t stream) {
    NormArgs a = args;
    const BackwardPlan p = plan_backward(a, vec);
    a.contiguous = p.contiguous, a.split = p.split;
    const bool full = a.layer || a.post_b.p;
    const int64_t workers = p.blocks * p.groups;
    cudaError_t e = cudaSuccess;
    if (a.rows == 0 || (p.contiguous && !p.split)) {   // nothing writes the sums, or they grow in place
        e = cudaMemsetAsync(a.partial, 0, static_cast<size_t>(p.floats) * sizeof(float), stream);
        if (e != cudaSuccess) return e;
    }
    if (a.rows > 0) {
        if (p.cluster > 1) {
            e = vec ? (p.cluster == 2 ? launch_backward_rows<S, B, 16, 2, true>(a, p, stream)
                                      : launch_backward_rows<S, B, 16, 4, true>(a, p, stream))
                    : launch_backward_rows<S, B, 16, 4, false>(a, p, stream);
        } else if (!vec) {
            e = p.warps == 1   ? launch_backward_rows<S, B, 1, 1, false>(a, p, stream)
                : p.warps == 4 ? launch_backward_rows<S, B, 4, 1, false>(a, p, stream)
                               : launch_backward_rows<S, B, 16, 1, false>(a, p, stream);
        } else {
            switch (p.warps) {
                case 1: e = launch_backward_rows<S, B, 1, 1, true>(a, p, stream); break;
                case 2: e = launch_backward_rows<S, B, 2, 1, true>(a, p, stream); break;
                case 3: e = launch_backward_rows<S, B, 3, 1, true>(a, p, stream); break;
                case 4: e = launch_backward_rows<S, B, 4, 1, true>(a, p, stream); break;
                case 8: e = launch_backward_rows<S, B, 8, 1, true>(a, p, stream); break;
                default: e = launch_backward_rows<S, B, 16, 1, true>(a, p, stream); break;
            }
        }
        if (e != cudaSuccess) return e;
    }
    peri_backward_sums_kernel<S><<<(a.d + 31) / 32, 256, 0, stream>>>(a, p.blocks, workers, full);
    return cudaGetLastError();
}

}  // namespace mtdao
