// peri_norm_api.cu -- the C calls of the Peri-LN residual update: checks of arguments, and how
// the backward pass deals out its rows.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstdio>

#include <nvtx3/nvToolsExt.h>

#include "peri_norm.cuh"

namespace mtdao {

// A thread has sixteen columns of a long row where it keeps two sums for each, else eight (four sums of sixteen are more
// than its registers hold); rows too long for one thread block are spread over a cluster of them.  512 threads an
// SM; fewer where rows run out.
BackwardPlan plan_backward(const NormArgs &a, bool vec) {
    BackwardPlan p = {};
    p.full = a.layer || a.post_b.p || !vec;            // rows of odd columns have one kernel for both
    p.cluster = p.warps = p.groups_of_eight = 1;
    p.lanes = 32;
    if (!vec) {
        // by the columns: rows of 509 in four warps took 228 us for 144 (bf16), of 2001 in sixteen 621 for 290
        p.warps = a.d <= 256 ? 1 : a.d <= 512 ? 2 : a.d <= 1024 ? 4 : a.d <= 2048 ? 8 : 16;
        p.cluster = a.d <= 4096 ? 1 : 4;
    } else if (a.d <= 256) {
        p.lanes = a.d <= 64 ? 8 : a.d <= 128 ? 16 : 32;
    } else if (a.d > 4096 && !a.wide && !p.full) {     // 16 warps and shared memory for two rows of 8192
        p.groups_of_eight = 2;
        p.warps = a.d <= 6144 ? 12 : 16;
        while (8192 * p.cluster < a.d) p.cluster *= 2;
    } else if (p.full || a.d <= 1024) {
        const int need = (a.d + 255) / 256;
        p.warps = need <= 4 ? need : need <= 8 ? 8 : need > 16 && need <= 24 ? 12 : 16;
        while (4096 * p.cluster < a.d) p.cluster *= 2;
    } else {
        p.groups_of_eight = 2;
        while (512 * p.warps < a.d && p.warps < 8) p.warps *= 2;
        while (4096 * p.cluster < a.d) p.cluster *= 2;
    }
    const int threads = p.warps == 3 ? 96 : p.warps <= 4 ? 128 : 32 * p.warps;
    p.groups = threads / (p.warps == 1 ? p.lanes : 32 * p.warps);
    // A cluster's thread blocks run in one group of SMs: of four on an SM each no 38 fit, but 36 (more would wait for the
    // others' end: 4096 fp32 rows of 16384 in 759 us for 465).
    const int64_t most = (p.cluster == 4 ? 36 : kPeriSms / p.cluster) * (512 / threads);
    p.blocks = std::max<int64_t>(1, std::min(most, (a.rows + p.groups - 1) / p.groups));
    const int64_t workers = p.blocks * p.groups;
    const bool rows_gate = gate_kind(a) == kGateRows;
    p.contiguous = rows_gate;
    p.split = rows_gate && a.gate_rows < 4 * workers;       // else each worker takes whole gate rows
    const int64_t second = p.split ? workers + a.gate_rows : rows_gate ? workers : p.blocks;
    p.floats = 2 * (p.blocks + second) * static_cast<int64_t>(a.d);
    return p;
}

namespace {

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
    if (s->gate_rows < 0 || s->gate_rows > (int64_t(1) << 40) ||
        (s->gate_rows > 0 && s->rows > 0 && s->rows % s->gate_rows != 0))
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
    a.wide = s->branch_dtype == MTDAO_F32;
    a.eps = static_cast<float>(s->eps);
    a.residual_scale = static_cast<float>(s->residual_scale);
    a.ld_x = s->ld_x, a.ld_f = s->ld_f, a.ld_y = s->ld_y, a.ld_h = s->ld_h;
    a.ld_dy = s->ld_dy, a.ld_dh = s->ld_dh, a.ld_dx = s->ld_dx, a.ld_df = s->ld_df;
    return a;
}

Vector vector_of(const void *p, int32_t type) { return Vector{const_cast<void *>(p), type == MTDAO_BF16}; }

int done(cudaError_t e, const char *what) {
    if (e == cudaSuccess) return MTDAO_OK;
    cudaGetLastError();                                // reported here, not by the next launch
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
    const cudaError_t e = st == MTDAO_BF16   ? launch_peri_forward<Bf16, Bf16>(a, vec, stream)
                          : br == MTDAO_BF16 ? launch_peri_forward<float, Bf16>(a, vec, stream)
                                             : launch_peri_forward<float, float>(a, vec, stream);
    return done(e, "peri_norm forward");
}

extern "C" int64_t mtdao_peri_norm_workspace(const mtdao_peri_norm *s) {
    if (check_shape(s, true)) return -1;
    // whatever the addresses and the biases turn out to be: the most that a plan can need
    NormArgs a = arguments(s);
    a.gate.p = s->gate_rows > 0 ? const_cast<mtdao_peri_norm *>(s) : nullptr;      // any address: there is a gate
    int64_t floats = plan_backward(a, false).floats;
    if (s->d % 8 == 0) {
        floats = std::max(floats, plan_backward(a, true).floats);
        a.post_b.p = const_cast<mtdao_peri_norm *>(s);
        floats = std::max(floats, plan_backward(a, true).floats);
    }
    return floats * static_cast<int64_t>(sizeof(float));
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
    a.partial = static_cast<float *>(workspace);
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (s->rows == 0 && gate) {
        const size_t bytes = static_cast<size_t>(s->gate_rows) * s->d * size_of(s->gate_dtype);
        const cudaError_t e = cudaMemsetAsync(d_gate, 0, bytes, stream);
        if (e != cudaSuccess) return done(e, "peri_norm backward");
    }
    const bool vec = s->d % 8 == 0 && (!dy || by_eight(dy, s->ld_dy, st)) && by_eight(y, s->ld_y, st) &&
                     by_eight(dx, s->ld_dx, st) && by_eight(dh, s->ld_dh, br) && by_eight(f, s->ld_f, br) &&
                     by_eight(df, s->ld_df, br) && by_eight(post_w, 8, wt) && by_eight(post_b, 8, wt) &&
                     by_eight(pre_w, 8, wt) &&
                     (!gate || (by_eight(gate, 8, s->gate_dtype) && by_eight(d_gate, 8, s->gate_dtype)));
    const cudaError_t e = st == MTDAO_BF16   ? launch_peri_backward<Bf16, Bf16>(a, vec, stream)
                          : br == MTDAO_BF16 ? launch_peri_backward<float, Bf16>(a, vec, stream)
                                             : launch_peri_backward<float, float>(a, vec, stream);
    return done(e, "peri_norm backward");
}
