// C ABI of the experts' products as calls of their own: argument checks and launches.  Declarations and contracts live in include/moe.h.
#include <hip/hip_runtime.h>

#include "ffn.hpp"
#include "problem.hpp"

using namespace moe;

static bool aligned16(const void *p) { return ((uintptr_t)p & 15) == 0; }
static int rows_of(const moe_problem_t *p) { return p->capacity > 0 ? p->E * p->capacity : p->T * p->k; }
static int elem_bytes(const moe_problem_t *p) { return p->dtype == MOE_DT_F32 ? 4 : 2; }
static bool bad_stride(const moe_problem_t *p, int64_t ld, int cols) { return ld < cols || ld * elem_bytes(p) % 16 != 0; }

// Of the current device, asked of the runtime once.
static int compute_units(int *n) {
    constexpr int kDevices = 64;
    static int known[kDevices];  // (whoever writes, writes the same)
    int device = 0;
    if (hipGetDevice(&device) != hipSuccess) return MOE_ERR_HIP;
    int cus = device < kDevices ? __atomic_load_n(&known[device], __ATOMIC_RELAXED) : 0;
    if (!cus) {
        if (hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, device) != hipSuccess) return MOE_ERR_HIP;
        if (device < kDevices) __atomic_store_n(&known[device], cus, __ATOMIC_RELAXED);
    }
    *n = (cus + kTileQueues - 1) / kTileQueues * kTileQueues;
    return MOE_OK;
}

// How a product is launched: workgroups, and whether their tiles are planned.
struct Launch {
    const void *kernel;
    unsigned groups, smem;
    int bm;
    bool planned;
};
// Tiles per workgroup from which on they are handed out by a plan, which is a launch of its own.
constexpr int kPlannedTiles = 2;

template <class T, FfnOp OP>
static int prepare(FfnArgs &a, Launch *l) {
    constexpr int COLS = OP == kFfnUp ? T::BN / 2 : T::BN;
    a.nt = (a.N + COLS - 1) / COLS * (OP == kFfnDw && a.o1 ? 2 : 1);
    a.mt = (a.M + T::BM - 1) / T::BM;
    // row blocks, at most: one per BM rows and one more per expert (ragged: and for the rows behind the last one)
    size_t blocks;
    if (OP == kFfnDw)
        blocks = (size_t)a.E * a.mt;
    else if (a.capacity)
        blocks = (size_t)a.E * ((a.capacity + T::BM - 1) / T::BM);
    else
        blocks = (size_t)a.rows / T::BM + (size_t)(a.E < a.rows ? a.E : a.rows) + 1;
    if (blocks * a.nt >= (size_t)1 << 30) return MOE_ERR_UNSUPPORTED;  // (tiles are counted in 32 bits)
    int cus = 0;
    if (const int rc = compute_units(&cus)) return rc;
    if (const int rc = allow_lds((const void *)k_ffn<T, OP>, T::SMEM)) return rc;
    const size_t tiles = (blocks * a.nt + kTileQueues - 1) / kTileQueues * kTileQueues, room = (size_t)cus * T::OCC;
    l->kernel = (const void *)k_ffn<T, OP>;
    l->groups = (unsigned)(tiles < room ? tiles : room);
    l->smem = T::SMEM;
    l->bm = T::BM;
    l->planned = tiles >= kPlannedTiles * room;
    return MOE_OK;
}

template <typename ET, FfnOp OP>
static int pick(FfnArgs &a, int slots, Launch *l) {
    if constexpr (sizeof(ET) == 4) {
        return slots / a.E > 48 ? prepare<FfnTile<ET, 2, 2, 2, 2, 64, 2>, OP>(a, l) : prepare<FfnTile<ET, 1, 2, 1, 4, 64, 2>, OP>(a, l);
    } else {
#ifndef V256
#define V256 4, 4, 2, 2, 64, 1
#endif
#ifndef V128
#define V128 4, 4, 2, 2, 64, 1
#endif
#ifndef V32
#define V32 1, 2, 1, 4, 128, 1
#endif
        if (slots / a.E > 160) return prepare<FfnTile<ET, V256>, OP>(a, l);
        return slots / a.E > 48 ? prepare<FfnTile<ET, V128>, OP>(a, l) : prepare<FfnTile<ET, V32>, OP>(a, l);
    }
}
template <typename ET>
static int pick_dw(FfnArgs &a, Launch *l) {
    if constexpr (sizeof(ET) == 4)
        return prepare<FfnTile<ET, 2, 2, 2, 2, 64, 2>, kFfnDw>(a, l);
    else
#ifndef VDW
#define VDW 4, 4, 2, 2, 64, 1
#endif
        return prepare<FfnTile<ET, VDW>, kFfnDw>(a, l);
}
template <FfnOp OP>
static int pick(const moe_problem_t *p, FfnArgs &a, Launch *l) {
    if constexpr (OP == kFfnDw)
        return p->dtype == MOE_DT_F32 ? pick_dw<float>(a, l) : pick_dw<bf16_t>(a, l);
    else
        return p->dtype == MOE_DT_F32 ? pick<float, OP>(a, p->T * p->k, l) : pick<bf16_t, OP>(a, p->T * p->k, l);
}
// A call's launches: a product of rows (any but dw), dw, or both.
template <FfnOp OP>
static int launch(const moe_problem_t *p, FfnArgs *rows, FfnArgs *dw, void *workspace, void *stream) {
    hipStream_t st = (hipStream_t)stream;
    Launch l[2] = {};
    FfnArgs *a[2] = {rows, dw};
    if (rows)
        if (const int rc = pick<OP>(p, *rows, &l[0])) return rc;
    if (dw)
        if (const int rc = pick<kFfnDw>(p, *dw, &l[1])) return rc;
    FfnPlan *plans = (FfnPlan *)workspace;
    if (l[0].planned || l[1].planned) {
        FfnPlanArgs plan = {};
        if (l[0].planned) plan.rows = *rows, plan.rows_plan = plans, plan.bm = l[0].bm, rows->plan = plans;
        if (l[1].planned) plan.dw = *dw, plan.dw_plan = plans + 1, dw->plan = plans + 1;
        hipLaunchKernelGGL(k_ffn_plan, dim3(1), dim3(kThreads), 0, st, plan);
        if (hipGetLastError() != hipSuccess) return MOE_ERR_HIP;
    }
    for (int i = 0; i < 2; ++i) {
        if (!a[i]) continue;
        void *args[] = {a[i]};
        if (hipLaunchKernel(l[i].kernel, dim3(l[i].groups), dim3(kThreads), args, l[i].smem, st) != hipSuccess) return MOE_ERR_HIP;
    }
    return MOE_OK;
}
static FfnArgs args_of(const moe_problem_t *p, const int32_t *counts) {
    FfnArgs a = {};
    a.E = p->E; a.rows = rows_of(p); a.capacity = p->capacity; a.counts = counts;
    return a;
}

extern "C" {

size_t moe_ffn_workspace_bytes(const moe_problem_t *p) { return check_problem(p) == MOE_OK ? (2 * sizeof(FfnPlan) + 255) / 256 * 256 : 0; }

static int check_workspace(const void *ws) { return !ws || ((uintptr_t)ws & 255) != 0 ? MOE_ERR_WORKSPACE : MOE_OK; }

int moe_ffn_up(const moe_problem_t *p, const void *x_perm, const void *W1, const void *W3, int64_t ldw, const int32_t *counts, void *g, void *u,
               int64_t ld, void *h, void *workspace, void *stream) {
    int rc = check_problem(p);
    if (rc) return rc;
    if (!x_perm || !W1 || !W3 || !counts || !g != !u || (!g && !h)) return MOE_ERR_INVALID_ARG;
    if (bad_stride(p, ldw, p->f) || (g && bad_stride(p, ld, p->f))) return MOE_ERR_INVALID_ARG;
    if (!aligned16(x_perm) || !aligned16(W1) || !aligned16(W3) || !aligned16(g) || !aligned16(u) || !aligned16(h)) return MOE_ERR_INVALID_ARG;
    if ((rc = check_workspace(workspace))) return rc;
    FfnArgs a = args_of(p, counts);
    a.N = p->f; a.K = p->d;
    a.A0 = x_perm; a.lda = p->d;
    a.B0 = W1; a.B1 = W3; a.ldb = ldw; a.eb = (long long)p->d * ldw;
    a.o0 = g; a.o1 = u; a.ldo = ld; a.o2 = h;
    return launch<kFfnUp>(p, &a, nullptr, workspace, stream);
}

int moe_ffn_down(const moe_problem_t *p, const void *h, const void *W2, const int32_t *counts, void *y, void *workspace, void *stream) {
    int rc = check_problem(p);
    if (rc) return rc;
    if (!h || !W2 || !counts || !y) return MOE_ERR_INVALID_ARG;
    if (!aligned16(h) || !aligned16(W2) || !aligned16(y)) return MOE_ERR_INVALID_ARG;
    if ((rc = check_workspace(workspace))) return rc;
    FfnArgs a = args_of(p, counts);
    a.N = p->d; a.K = p->f;
    a.A0 = h; a.lda = p->f;
    a.B0 = W2; a.ldb = p->d; a.eb = (long long)p->f * p->d;
    a.o0 = y;
    return launch<kFfnDown>(p, &a, nullptr, workspace, stream);
}

int moe_ffn_down_backward(const moe_problem_t *p, const void *dy, const void *W2, const void *h, const void *g, const void *u, const int32_t *counts,
                          void *dh, void *dg, void *du, int64_t ld, void *dW2, void *workspace, void *stream) {
    int rc = check_problem(p);
    if (rc) return rc;
    if (!dy || !counts || !dg != !du || (!dh && !dg && !dW2)) return MOE_ERR_INVALID_ARG;
    if (((dh || dg) && !W2) || (dg && (!g || !u)) || (dW2 && !h)) return MOE_ERR_INVALID_ARG;
    if (dg && bad_stride(p, ld, p->f)) return MOE_ERR_INVALID_ARG;
    if (!aligned16(dy) || !aligned16(W2) || !aligned16(h) || !aligned16(g) || !aligned16(u) || !aligned16(dh) || !aligned16(dg) || !aligned16(du) ||
        !aligned16(dW2))
        return MOE_ERR_INVALID_ARG;
    if ((rc = check_workspace(workspace))) return rc;
    FfnArgs rows = args_of(p, counts), dw = rows;
    {
        FfnArgs &a = rows;
        a.N = p->f; a.K = p->d;
        a.A0 = dy; a.lda = p->d;
        a.B0 = W2; a.ldb = p->d; a.eb = (long long)p->f * p->d;
        a.g = g; a.u = u; a.ldg = ld;
        a.o0 = dg; a.o1 = du; a.ldo = ld; a.o2 = dh;
    }
    {
        FfnArgs &a = dw;
        a.M = p->f; a.N = p->d;
        a.A0 = h; a.lda = p->f;
        a.B0 = dy; a.ldb = p->d;
        a.o0 = dW2; a.ldo = p->d; a.eo = (long long)p->f * p->d;
    }
    return launch<kFfnDh>(p, dh || dg ? &rows : nullptr, dW2 ? &dw : nullptr, workspace, stream);
}

int moe_ffn_up_backward(const moe_problem_t *p, const void *x_perm, const void *W1, const void *W3, int64_t ldw, const void *dg, const void *du,
                        int64_t ld, const int32_t *counts, void *dx, void *dW1, void *dW3, void *workspace, void *stream) {
    int rc = check_problem(p);
    if (rc) return rc;
    if (!counts || (!dx && !dW1 && !dW3)) return MOE_ERR_INVALID_ARG;
    if ((dx && (!W1 || !W3)) || ((dx || dW1) && !dg) || ((dx || dW3) && !du) || ((dW1 || dW3) && !x_perm)) return MOE_ERR_INVALID_ARG;
    if (bad_stride(p, ldw, p->f) || bad_stride(p, ld, p->f)) return MOE_ERR_INVALID_ARG;
    if (!aligned16(x_perm) || !aligned16(W1) || !aligned16(W3) || !aligned16(dg) || !aligned16(du) || !aligned16(dx) || !aligned16(dW1) || !aligned16(dW3))
        return MOE_ERR_INVALID_ARG;
    if ((rc = check_workspace(workspace))) return rc;
    FfnArgs rows = args_of(p, counts), dw = rows;
    {
        FfnArgs &a = rows;
        a.N = p->d; a.K = p->f;
        a.A0 = dg; a.A1 = du; a.lda = ld;
        a.B0 = W1; a.B1 = W3; a.ldb = ldw; a.eb = (long long)p->d * ldw;
        a.o0 = dx;
    }
    {
        FfnArgs &a = dw;
        a.M = p->d; a.N = p->f;
        a.A0 = x_perm; a.lda = p->d;
        a.B0 = dW1 ? dg : du; a.B1 = du; a.ldb = ld;
        a.o0 = dW1 ? dW1 : dW3; a.o1 = dW1 ? dW3 : nullptr; a.ldo = ldw; a.eo = (long long)p->d * ldw;
    }
    return launch<kFfnDx>(p, dx ? &rows : nullptr, dW1 || dW3 ? &dw : nullptr, workspace, stream);
}

}  // extern "C"
