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

// Few tokens: below the first number a token's slots are several workgroups (the gradient of 17 x 16 rows of 3968 9.7 -> 6.9 us, 500 x 32 of 512
// 15.3 -> 8.8; 1000 x 16 of 2048 24.1 -> 24.9), up to the second a long row a workgroup of 1024 threads (fp32 8 x 8 rows of 2368 8.5 -> 7.5;
// bf16 64 x 8 of 7168 9.0 -> 9.1, 500 x 8 22.3 -> 25.8).
constexpr int kFewTokens = 512, kVeryFewTokens = 32;
template <typename ET>
static bool stream_rows(const UnsortArgs &a) {
    return (size_t)a.rows * a.d * sizeof(ET) > kStreamBytes;
}
template <typename ET, int KB, int U, int G>
static int launch_unsort(UnsortArgs &a, hipStream_t st) {
    a.parts = (a.d / Piece<ET>::N + G * U - 1) / (G * U);
    const dim3 grid(grid_for((size_t)a.T * a.parts, kThreads / G));
    if (G == 64 && stream_rows<ET>(a))
        hipLaunchKernelGGL((k_unsort<ET, KB, U, G, G == 64>), grid, dim3(kThreads), 0, st, a);
    else
        hipLaunchKernelGGL((k_unsort<ET, KB, U, G, false>), grid, dim3(kThreads), 0, st, a);
    return launched();
}
// Rows in flight (the k of a token, up to 8), pieces per lane so that about 8 loads are, and lanes by the row's length: 16384 x 8 rows of 64
// with 8 / 64 lanes 6.1 / 13.4 us, 8192 x 1 of 512 with 1 / 4 pieces per lane 4.8 / 7.6.
template <typename ET>
static int pick_unsort(UnsortArgs &a, hipStream_t st) {
    const int pieces = a.d / Piece<ET>::N;
    if (pieces <= 32) {
        if (pieces <= 8) return a.k <= 2 ? launch_unsort<ET, 2, 1, 8>(a, st) : launch_unsort<ET, 8, 1, 8>(a, st);
        if (pieces <= 16) return a.k <= 2 ? launch_unsort<ET, 2, 1, 16>(a, st) : launch_unsort<ET, 8, 1, 16>(a, st);
        return a.k <= 2 ? launch_unsort<ET, 2, 1, 32>(a, st) : launch_unsort<ET, 8, 1, 32>(a, st);
    }
    if (a.k <= 2) return pieces <= 64 ? launch_unsort<ET, 2, 1, 64>(a, st) : pieces <= 128 ? launch_unsort<ET, 2, 2, 64>(a, st) : launch_unsort<ET, 2, 4, 64>(a, st);
    if (a.k <= 4) return pieces <= 64 ? launch_unsort<ET, 4, 1, 64>(a, st) : launch_unsort<ET, 4, 2, 64>(a, st);
    return launch_unsort<ET, 8, 1, 64>(a, st);
}

template <typename ET, int KB, int L>
static int launch_unsort_backward(UnsortArgs &a, hipStream_t st) {
    constexpr int NT = unsort_backward_threads(L);
    a.batches = a.T < kFewTokens ? (a.k + KB - 1) / KB : 1;
    a.token_groups = (int)grid_for(a.T, NT / L) * a.batches;
    const unsigned zero_groups = a.capacity > 0 && a.drows ? grid_for(a.rows, NT / 16) : 0u;
    const dim3 grid(a.token_groups + zero_groups);
    if (L >= 64 && stream_rows<ET>(a))
        hipLaunchKernelGGL((k_unsort_backward<ET, KB, L, (L >= 64)>), grid, dim3(NT), 0, st, a);
    else
        hipLaunchKernelGGL((k_unsort_backward<ET, KB, L, false>), grid, dim3(NT), 0, st, a);
    return launched();
}
template <typename ET, int L>
static int pick_unsort_backward(UnsortArgs &a, hipStream_t st) {
    return a.k <= 2 ? launch_unsort_backward<ET, 2, L>(a, st) : a.k <= 4 ? launch_unsort_backward<ET, 4, L>(a, st) : launch_unsort_backward<ET, 8, L>(a, st);
}
// Lanes per token by the row's length: 4096 x 8 rows of 2048 with 64 / 128 / 256 lanes 71 / 65 / 59 us.
template <typename ET>
static int pick_unsort_backward(UnsortArgs &a, hipStream_t st) {
    const int pieces = a.d / Piece<ET>::N;
    if (pieces <= 8) return pick_unsort_backward<ET, 8>(a, st);
    if (pieces <= 16) return pick_unsort_backward<ET, 16>(a, st);
    if (pieces <= 32) return pick_unsort_backward<ET, 32>(a, st);
    if (pieces <= 64) return pick_unsort_backward<ET, 64>(a, st);
    if (pieces <= 128) return pick_unsort_backward<ET, 128>(a, st);
    return pieces <= 256 || a.T > kVeryFewTokens ? pick_unsort_backward<ET, 256>(a, st) : pick_unsort_backward<ET, 1024>(a, st);
}

// How the gate's gradient is cut.
static void gate_grad_plan(const moe_problem_t *p, GateGradArgs *a) {
    const int cols = kChunkBytes / elem_bytes(p);
    a->T = p->T; a->d = p->d; a->E = p->E; a->k = p->k;
    a->dx_chunks = (p->d + cols - 1) / cols;
    a->block = p->k <= 8 ? 128 : p->k <= 16 ? 64 : 32;
    const auto parts_of = [](int tasks, int chunks) { return tasks > chunks ? tasks / chunks : 1; };
    const int blocks = (p->T + a->block - 1) / a->block, dx_want = parts_of(512, a->dx_chunks);
    a->dx_blocks = (blocks + dx_want - 1) / dx_want;
    a->dx_parts = (blocks + a->dx_blocks - 1) / a->dx_blocks;
    // Parts of dWg's tokens: 64 of them take a task 0.85 us (1.3 to 1.75 in fp32), a part's sums 0.8 us per MB to write and read again, and
    // the launch that adds them up 3 us.  At most three tasks for four CUs: dx's, which share the CUs, would wait for them.  us, with dx, by
    // parts: 4096 x 8 of 128 of 2048 4 / 6 / 8 / 16: 23.0 / 20.7 / 22.8 / 24.1, 1024 tokens 1 / 4 / 16: 18.2 / 11.9 / 19.9; 2048 x 8 of 256
    // of 7168 1 / 2 / 4: 35.3 / 40.9 / 44.8; 16384 x 4 of 32 of 64 16 / 64 / 256: 17.9 / 9.8 / 13.4; 9683 x 3 of 3 of 720 (fp32) 16 / 21:
    // 19.8 / 18.5.  (By the problem alone, whichever gradients are wanted: their bits are the same alone and together.)
    constexpr int kReduction = 64;  // tokens, a multiple of every shape's
    a->dw_chunks = (p->d + kGateDwCols - 1) / kGateDwCols;
    a->dw_groups = (p->E + kGateDwExperts - 1) / kGateDwExperts;
    a->dw_experts = ((p->E + a->dw_groups - 1) / a->dw_groups + 3) / 4 * 4;
    const int units = (p->T + kReduction - 1) / kReduction, most = parts_of(192, a->dw_chunks * a->dw_groups);
    const double unit_us = p->dtype == MOE_DT_F32 ? (p->E <= 64 ? 1.3 : 1.75) : 0.85, part_us = 0.8e-6 * 4.0 * p->d * p->E;
    double best = 0.0;
    int each = units;
    for (int n = 1; n <= most && n <= units; ++n) {
        const int per = (units + n - 1) / n;
        const double us = per * unit_us + n * part_us + (n > 1 ? 3.0 + 0.05 * n : 0.0);
        if (n == 1 || us < best) best = us, each = per;
    }
    a->dw_tokens = each * kReduction;
    a->dw_parts = (p->T + a->dw_tokens - 1) / a->dw_tokens;
    a->part_stride = ((size_t)p->d * p->E + p->E + 63) / 64 * 64;
}

template <class C>
static int launch_gate_grad(const GateGradArgs &a, hipStream_t st) {
    const size_t dx = a.dx_parts ? sizeof(GateDxLds) + (size_t)(a.E + 1) * kChunkBytes : 0;
    const size_t dw = a.dw_chunks ? (size_t)C::LDS : 0, db = a.dbias ? (size_t)kGateGradThreads / 8 * a.E * 4 : 0;
    const size_t smem = dx > dw ? (dx > db ? dx : db) : (dw > db ? dw : db);
    if (const int rc = allow_lds((const void *)k_gate_grad<C>, smem)) return rc;
    hipLaunchKernelGGL(k_gate_grad<C>, dim3((a.dw_chunks * a.dw_groups + (a.dbias ? 1 : 0)) * a.dw_parts + a.dx_chunks * a.dx_parts), dim3(kGateGradThreads), smem, st, a);
    if (const int rc = launched()) return rc;
    if (a.dw_parts <= 1) return MOE_OK;
    const size_t pieces = (size_t)a.d * a.E / 4 + (a.E + 3) / 4;
    hipLaunchKernelGGL(k_gate_grad_join, dim3((unsigned)((pieces + 63) / 64)), dim3(kThreads), 0, st, a);
    return launched();
}

template <typename ET, int WE, int KT>
static int pick_gate_grad(const GateGradArgs &a, hipStream_t st) {
    return a.k <= 8 ? launch_gate_grad<GateDwShape<ET, WE, KT, true>>(a, st) : launch_gate_grad<GateDwShape<ET, WE, KT, false>>(a, st);
}
// Up to 64 experts take shapes of their own: half as much of dl's LDS, and for fp32 twice as many tokens per block.  us, with the shapes of
// 128 / their own: bf16 16384 x 4 of 64 of 512 16.9 / 15.5; fp32 9683 x 3 of 3 of 720 21.2 / 18.5, 256 x 2 of 8 of 512 10.6 / 8.5.
template <typename ET>
static int pick_gate_grad(const GateGradArgs &a, hipStream_t st) {
    if (a.E <= 64) return pick_gate_grad<ET, 2, 64>(a, st);
    return pick_gate_grad<ET, 4, sizeof(ET) == 2 ? 64 : 32>(a, st);
}

// Workgroups for all pieces of the rows.  (A grid has less than 2^32 threads; rows of so many pieces are more than the memory holds.)
template <typename ET>
static int swiglu_grid(const SwigluArgs &a, dim3 *grid) {
    const size_t pieces = (size_t)a.rows * ((a.f + kScaleBlock - 1) / kScaleBlock * (kScaleBlock / Piece<ET>::N));
    const size_t n = (pieces + kSwigluPieces * kThreads - 1) / (kSwigluPieces * kThreads);
    if (n >= (1u << 24)) return MOE_ERR_UNSUPPORTED;
    *grid = dim3((unsigned)n);
    return MOE_OK;
}
template <typename ET>
static int launch_swiglu(const SwigluArgs &a, hipStream_t st) {
    dim3 grid;
    if (const int rc = swiglu_grid<ET>(a, &grid)) return rc;
    if ((size_t)a.rows * a.f * 2 * sizeof(ET) > kStreamBytes)
        hipLaunchKernelGGL((k_swiglu<ET, true>), grid, dim3(kThreads), 0, st, a);
    else
        hipLaunchKernelGGL((k_swiglu<ET, false>), grid, dim3(kThreads), 0, st, a);
    return launched();
}
template <typename ET>
static int launch_swiglu_backward(const SwigluArgs &a, hipStream_t st) {
    dim3 grid;
    if (const int rc = swiglu_grid<ET>(a, &grid)) return rc;
    if ((size_t)a.rows * a.f * (2 + sizeof(ET)) > kStreamBytes)
        hipLaunchKernelGGL((k_swiglu_backward<ET, true>), grid, dim3(kThreads), 0, st, a);
    else
        hipLaunchKernelGGL((k_swiglu_backward<ET, false>), grid, dim3(kThreads), 0, st, a);
    return launched();
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
    return p->dtype == MOE_DT_F32 ? pick_unsort<float>(a, (hipStream_t)stream) : pick_unsort<bf16_t>(a, (hipStream_t)stream);
}

int moe_unsort_backward(const moe_problem_t *p, const void *dout, const void *rows, const int32_t *inv_perm, const float *topk_w,
                        const int32_t *counts, void *drows, float *dtopk_w, int32_t *status_dev, void *stream) {
    const int rc = check_problem(p);
    if (rc) return rc;
    if (!dout || !inv_perm || (!drows && !dtopk_w) || (dtopk_w && !rows)) return MOE_ERR_INVALID_ARG;
    if (p->capacity > 0 && !counts) return MOE_ERR_INVALID_ARG;
    if (!aligned16(dout) || !aligned16(rows) || !aligned16(drows)) return MOE_ERR_INVALID_ARG;
    UnsortArgs a = {};
    a.T = p->T; a.d = p->d; a.k = p->k; a.rows = rows_of(p); a.capacity = p->capacity;
    a.dout = dout; a.sorted = rows; a.inv_perm = inv_perm; a.w = topk_w; a.counts = counts; a.drows = drows; a.dw = dtopk_w;
    a.status = status_dev;
    return p->dtype == MOE_DT_F32 ? pick_unsort_backward<float>(a, (hipStream_t)stream) : pick_unsort_backward<bf16_t>(a, (hipStream_t)stream);
}

size_t moe_backward_workspace_bytes(const moe_problem_t *p) {
    if (check_problem(p) != MOE_OK) return 0;
    GateGradArgs a;
    gate_grad_plan(p, &a);
    return a.dw_parts > 1 ? a.dw_parts * a.part_stride * 4 : 256;  // (one part's sums go straight to dWg and dgate_bias)
}

int moe_route_backward(const moe_problem_t *p, const void *x, const void *Wg, const int32_t *topk_idx, const float *topk_w,
                       const float *dtopk_w, void *dx, float *dWg, float *dgate_bias, int32_t *status_dev, void *workspace, void *stream) {
    const int rc = check_problem(p);
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
    if (!dWg) a.dw_chunks = 0;
    if (!sums) a.dw_parts = 0;
    if (!dx) a.dx_parts = 0;
    a.parts = (float *)workspace;
    hipStream_t st = (hipStream_t)stream;
    return p->dtype == MOE_DT_F32 ? pick_gate_grad<float>(a, st) : pick_gate_grad<bf16_t>(a, st);
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
    return p->dtype == MOE_DT_F32 ? launch_swiglu<float>(a, (hipStream_t)stream) : launch_swiglu<bf16_t>(a, (hipStream_t)stream);
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
    return p->dtype == MOE_DT_F32 ? launch_swiglu_backward<float>(a, (hipStream_t)stream) : launch_swiglu_backward<bf16_t>(a, (hipStream_t)stream);
}

}  // extern "C"
