// C ABI of the calls that train the layer around a program's own expert products: argument checks and launches.  Declarations and
// contracts live in include/moe.h.
#include <hip/hip_runtime.h>

#include "gate_grad.hpp"
#include "problem.hpp"
#include "swiglu8.hpp"
#include "unsort.hpp"

using namespace moe;

static int launched() { return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP; }
static bool aligned16(const void *p) { return ((uintptr_t)p & 15) == 0; }
static int rows_of(const moe_problem_t *p) { return p->capacity > 0 ? p->E * p->capacity : p->T * p->k; }
static int elem_bytes(const moe_problem_t *p) { return p->dtype == MOE_DT_F32 ? 4 : 2; }
// Workgroups for `n` pieces of work, `each` of them per workgroup; the kernels take more in strides of the grid.
static unsigned grid_for(size_t n, size_t each) {
    const size_t g = (n + each - 1) / each;
    return (unsigned)(g < (1u << 20) ? g : (1u << 20));
}

static size_t gate_grad_stride(const moe_problem_t *p) { return ((size_t)p->d * p->E + p->E + 63) / 64 * 64; }  // floats of a part

// How the gate's gradient is cut: blocks of tokens, and parts of the tokens for tasks of dWg and of dx.
static void gate_grad_plan(const moe_problem_t *p, GateGradArgs *a) {
    const int cols = kChunkBytes / elem_bytes(p);
    a->T = p->T; a->d = p->d; a->E = p->E; a->k = p->k;
    a->block = p->k <= 8 ? 256 : p->k <= 16 ? 128 : 64;
    a->chunks = (p->d + cols - 1) / cols;
    const int blocks = (p->T + a->block - 1) / a->block;
    int want = 256 / a->chunks;
    if (want < 1) want = 1;
    if (want > blocks) want = blocks;
    a->dw_blocks = a->dx_blocks = (blocks + want - 1) / want;
    a->dw_parts = a->dx_parts = (blocks + a->dw_blocks - 1) / a->dw_blocks;
}

template <typename ET>
static int launch_gate_grad(const GateGradArgs &a, hipStream_t st) {
    const size_t rows = (size_t)(a.dw_parts && a.x ? a.block : 0), columns = a.dx_parts ? a.E : 0;
    size_t smem = sizeof(GateGradLds) + (rows > columns ? rows : columns) * kChunkBytes;
    const size_t turn = (size_t)32 * (a.E + 1) * 4;
    if (smem < turn) smem = turn;
    const dim3 grid(a.dw_chunks * a.dw_parts + a.chunks * a.dx_parts), block(kGateGradThreads);
    auto go = [&](auto kern) {
        if (const int rc = allow_lds((const void *)kern, smem)) return rc;
        hipLaunchKernelGGL(kern, grid, block, smem, st, a);
        return launched();
    };
    const int per_wave = (a.E + kGateGradWaves - 1) / kGateGradWaves;
    if (per_wave <= 1) return go(k_gate_grad<ET, 1>);
    if (per_wave <= 4) return go(k_gate_grad<ET, 4>);
    if (per_wave <= 8) return go(k_gate_grad<ET, 8>);
    return go(k_gate_grad<ET, 16>);
}

extern "C" {

int moe_unsort(const moe_problem_t *p, const void *rows, const int32_t *inv_perm, const float *topk_w, const void *addend, void *out,
               int32_t *status_dev, void *stream) {
    const int rc = check_problem(p);
    if (rc) return rc;
    if (!rows || !inv_perm || !out) return MOE_ERR_INVALID_ARG;
    if (!aligned16(rows) || !aligned16(addend) || !aligned16(out)) return MOE_ERR_INVALID_ARG;
    UnsortArgs a = {};
    a.T = p->T; a.d = p->d; a.k = p->k; a.rows = rows_of(p);
    a.sorted = rows; a.inv_perm = inv_perm; a.w = topk_w; a.addend = addend; a.out = out; a.status = status_dev;
    const dim3 grid(grid_for(p->T, 4));
    hipStream_t st = (hipStream_t)stream;
    if (p->dtype == MOE_DT_F32)
        hipLaunchKernelGGL(k_unsort<float>, grid, dim3(kThreads), 0, st, a);
    else
        hipLaunchKernelGGL(k_unsort<bf16_t>, grid, dim3(kThreads), 0, st, a);
    return launched();
}

int moe_unsort_backward(const moe_problem_t *p, const void *dout, const void *rows, const int32_t *inv_perm, const float *topk_w,
                        const int32_t *counts, void *drows, float *dtopk_w, int32_t *status_dev, void *stream) {
    int rc = check_problem(p);
    if (rc) return rc;
    if (!dout || !inv_perm || (!drows && !dtopk_w) || (dtopk_w && !rows)) return MOE_ERR_INVALID_ARG;
    if (p->capacity > 0 && !counts) return MOE_ERR_INVALID_ARG;
    if (!aligned16(dout) || !aligned16(rows) || !aligned16(drows)) return MOE_ERR_INVALID_ARG;
    UnsortArgs a = {};
    a.T = p->T; a.d = p->d; a.k = p->k; a.rows = rows_of(p); a.capacity = p->capacity; a.E = p->E;
    a.dout = dout; a.sorted = rows; a.inv_perm = inv_perm; a.w = topk_w; a.counts = counts; a.drows = drows; a.dw = dtopk_w;
    a.status = status_dev;
    hipStream_t st = (hipStream_t)stream;
    const dim3 grid(grid_for(p->T, 4));
    if (p->dtype == MOE_DT_F32)
        hipLaunchKernelGGL(k_unsort_backward<float>, grid, dim3(kThreads), 0, st, a);
    else
        hipLaunchKernelGGL(k_unsort_backward<bf16_t>, grid, dim3(kThreads), 0, st, a);
    if ((rc = launched())) return rc;
    if (p->capacity > 0 && drows) {
        hipLaunchKernelGGL(k_zero_unused, dim3(grid_for(a.rows, 4)), dim3(kThreads), 0, st, counts, a.rows, p->capacity,
                           (size_t)p->d * elem_bytes(p), drows);
        rc = launched();
    }
    return rc;
}

size_t moe_backward_workspace_bytes(const moe_problem_t *p) {
    if (check_problem(p) != MOE_OK) return 0;
    GateGradArgs a;
    gate_grad_plan(p, &a);
    return a.dw_parts * gate_grad_stride(p) * 4;
}

int moe_route_backward(const moe_problem_t *p, const void *x, const void *Wg, const int32_t *topk_idx, const float *topk_w,
                       const float *dtopk_w, void *dx, float *dWg, float *dgate_bias, int32_t *status_dev, void *workspace, void *stream) {
    int rc = check_problem(p);
    if (rc) return rc;
    if (!topk_idx || !topk_w || !dtopk_w || (!dx && !dWg && !dgate_bias)) return MOE_ERR_INVALID_ARG;
    if ((dx && !Wg) || (dWg && !x)) return MOE_ERR_INVALID_ARG;
    if (!aligned16(x) || !aligned16(Wg) || !aligned16(dx) || !aligned16(dWg)) return MOE_ERR_INVALID_ARG;
    const bool sums = dWg || dgate_bias;
    if (sums && (!workspace || ((uintptr_t)workspace & 255) != 0)) return MOE_ERR_WORKSPACE;
    GateGradArgs a = {};
    gate_grad_plan(p, &a);
    a.x = dWg ? x : nullptr; a.Wg = Wg; a.idx = topk_idx; a.w = topk_w; a.dw = dtopk_w; a.dx = dx; a.dWg = dWg; a.dbias = dgate_bias;
    a.status = status_dev;
    a.dw_chunks = dWg ? a.chunks : 1;
    if (!sums) a.dw_parts = 0;
    if (!dx) a.dx_parts = 0;
    const size_t n_w = (size_t)p->d * p->E;
    if (a.dw_parts > 1) {
        a.part_stride = gate_grad_stride(p);
        if (dWg) a.dWg = (float *)workspace;
        if (dgate_bias) a.dbias = (float *)workspace + n_w;
    }
    hipStream_t st = (hipStream_t)stream;
    rc = p->dtype == MOE_DT_F32 ? launch_gate_grad<float>(a, st) : launch_gate_grad<bf16_t>(a, st);
    if (rc || a.dw_parts <= 1) return rc;
    const size_t from = dWg ? 0 : n_w, n = dgate_bias ? n_w + p->E : n_w;
    hipLaunchKernelGGL(k_gate_grad_join, dim3(grid_for(n - from, kThreads)), dim3(kThreads), 0, st, (const float *)workspace, a.part_stride,
                       a.dw_parts, from, n_w, n, dWg, dgate_bias);
    return launched();
}

static int check_swiglu(const moe_problem_t *p, int64_t ld, const int32_t *counts, const void *codes, const void *scales) {
    if (p->capacity > 0 && !counts) return MOE_ERR_INVALID_ARG;
    if (ld < p->f || ld * elem_bytes(p) % 16 != 0) return MOE_ERR_INVALID_ARG;
    if (!codes != !scales || !aligned16(codes)) return MOE_ERR_INVALID_ARG;
    return MOE_OK;
}

int moe_swiglu(const moe_problem_t *p, const void *g, const void *u, int64_t ld, const int32_t *counts, void *h, uint8_t *codes,
               uint8_t *scales, void *stream) {
    int rc = check_problem(p);
    if (rc) return rc;
    if (!g || !u || (!h && !codes)) return MOE_ERR_INVALID_ARG;
    if ((rc = check_swiglu(p, ld, counts, codes, scales))) return rc;
    if (!aligned16(g) || !aligned16(u) || !aligned16(h)) return MOE_ERR_INVALID_ARG;
    SwigluArgs a = {};
    a.rows = rows_of(p); a.f = p->f; a.capacity = p->capacity; a.ld = ld;
    a.g = g; a.u = u; a.counts = counts; a.h = h; a.codes = codes; a.scales = scales;
    const dim3 grid(grid_for((size_t)a.rows * ((p->f + kScaleBlock - 1) / kScaleBlock * 4), kThreads));
    hipStream_t st = (hipStream_t)stream;
    if (p->dtype == MOE_DT_F32)
        hipLaunchKernelGGL(k_swiglu<float>, grid, dim3(kThreads), 0, st, a);
    else
        hipLaunchKernelGGL(k_swiglu<bf16_t>, grid, dim3(kThreads), 0, st, a);
    return launched();
}

int moe_swiglu_backward(const moe_problem_t *p, const void *dh, const uint8_t *codes, const uint8_t *scales, const int32_t *counts,
                        void *dg, void *du, int64_t ld, void *h, void *stream) {
    int rc = check_problem(p);
    if (rc) return rc;
    if (!dh || !codes || !dg || !du) return MOE_ERR_INVALID_ARG;
    if ((rc = check_swiglu(p, ld, counts, codes, scales))) return rc;
    if (!aligned16(dh) || !aligned16(dg) || !aligned16(du) || !aligned16(h)) return MOE_ERR_INVALID_ARG;
    SwigluArgs a = {};
    a.rows = rows_of(p); a.f = p->f; a.capacity = p->capacity; a.ld = ld;
    a.dh = dh; a.counts = counts; a.dg = dg; a.du = du; a.h = h;
    a.codes = const_cast<uint8_t *>(codes); a.scales = const_cast<uint8_t *>(scales);
    const dim3 grid(grid_for((size_t)a.rows * (p->f / kLaneValues), kThreads));
    hipStream_t st = (hipStream_t)stream;
    if (p->dtype == MOE_DT_F32)
        hipLaunchKernelGGL(k_swiglu_backward<float>, grid, dim3(kThreads), 0, st, a);
    else
        hipLaunchKernelGGL(k_swiglu_backward<bf16_t>, grid, dim3(kThreads), 0, st, a);
    return launched();
}

}  // extern "C"
