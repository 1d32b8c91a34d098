// C ABI of the experts' products as calls of their own: argument checks and launches.  Declarations and contracts live in include/moe.h.
#include <hip/hip_runtime.h>

#include <math.h>

#include <algorithm>

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

// How a product is launched: workgroups, whether their tiles are planned, and what joins the parts of a reduction that is cut.
struct Launch {
    const void *kernel, *join;
    unsigned groups, smem;
    size_t part_bytes;
    int kind, bm;
    bool planned;
};
// Tiles per workgroup from which on they are handed out by a plan, which is a launch of its own (5 us; what it gains: see ffn()).  Tiles of 32 rows take
// the same each: 128 x 8 of 128 of 2048 x 768 down 73 us, with a plan 76.
constexpr int kPlannedTiles = 2;

// The tiles there are to choose from, and what they take where all CUs have them: us for 64 bytes of the reduction, at the start and end, and
// (256 rows) for 64 rows that a block lacks.  Measured, 16384 rows x 2048 x 2048 on 8 experts, 1.55 to 1.75 GHz: bf16 256 x 256 0.80 us a stage with
// 256 rows, 0.38 with 64; 128 x 128, two of them per CU, 0.55; 32 x 256 0.26 and 32 x 128 0.14 (more where the weights come from memory:
// 128 tokens x 8 of 128 of 2048 x 768 0.47); fp32 128 x 128 1.58, 64 x 128 1.02 (and 4 % more since numbers are scaled as they are cut, in both).
struct Kind {
    int bm, bn, occ;
    double stage_us, more_us, less_us;
};
constexpr int kKinds = 4;
constexpr Kind kKindsBf16[kKinds] = {{256, 256, 1, 0.82, 12, 0.14}, {128, 128, 2, 0.56, 7, 0}, {32, 256, 1, 0.35, 6, 0}, {32, 128, 1, 0.18, 5, 0}};
constexpr Kind kKindsF32[2] = {{128, 128, 2, 1.6, 7, 0}, {64, 128, 2, 1.02, 5, 0}};
template <typename ET, int KIND> struct TileOf;
template <> struct TileOf<bf16_t, 0> { typedef FfnTile<bf16_t, 4, 4, 2, 2, 1, 64, 1> type; };
template <> struct TileOf<bf16_t, 1> { typedef FfnTile<bf16_t, 2, 2, 2, 2, 1, 64, 2> type; };
template <> struct TileOf<bf16_t, 2> { typedef FfnTile<bf16_t, 1, 2, 1, 4, 1, 128, 1> type; };
template <> struct TileOf<bf16_t, 3> { typedef FfnTile<bf16_t, 1, 2, 1, 2, 2, 128, 1> type; };
template <> struct TileOf<float, 0> { typedef FfnTile<float, 2, 2, 2, 2, 1, 64, 2> type; };
template <> struct TileOf<float, 1> { typedef FfnTile<float, 1, 2, 2, 2, 1, 64, 2> type; };

// The tile, and the parts of the reduction, that take least by what they are worth.  (256 CUs, whatever the card, for the same bits.)
// Measured, us, * what is taken.  By tile, 256 x 256 / 128 x 128 / 32 x 256 / 32 x 128: one token of 8 of 128 of 2048 x 768 up - / 18.6 / 19.2 / 14.4*; 128 x
// 8 down 80 / 82 / 73* / 82; 4096 x 8 up 306* / 390 / 536 / 667; 4096 x 4 of 128 of 2880 x 2880 down 530* / 624 / 817 / 907; 4096 x 8 dh and dW2, by
// dW2's tile, 403* / 483.  fp32, 1001 x 6 of 48 of 1040 x 368, 128 rows / 64: by dx's 219 / 215*, by dw's 217* / 233.  By parts, 1 / 2 / 4 / 8 / 16 /
// 32: a token of 2 of 8 of 4096 x 14336 down 91 / 58 / 52* / 52 / 56 / 69; 16384 rows of 2 experts of 256 x 256 dx, dW1 and dW3, by dw's, 121 / 74 / 48 / 37 / 34* /
// 43; fp32 one row of 2048 x 512 down 91 / 51 / 30 / 21 / 18* / 19; where the model errs: 64 x 2 of 8 of 1024 x 2816 dx, dW1 and dW3, by dx's, 61 / 59 /
// 67*.
constexpr int kCus = 256, kMostParts = 32;
constexpr size_t kPartBytes = (size_t)32 << 20;  // of parts' sums, at most
// fp32: stages that the tile of 128 rows may add up in one sum (1024 steps).  Of 3584 steps the 2-norm of the error was 1.0e-6 of the result's, that of
// an fp32 product of the library's; what is longer, and dw where an expert could have more rows, is left to 64 rows and their sums of sums, 4e-7 of
// 16384 steps (growing with the root of their number), for 1.25 times the time.
constexpr int kOneSum = 64;
constexpr double kLeastStages = 8;                // of a part
struct Choice {
    int kind, split;
    size_t part_bytes;
};
static int matrices_of(FfnOp op, const FfnArgs &a) { return op == kFfnUp || (op == kFfnDw && !a.down) ? 2 : 1; }  // (dW1 and dW3: alone as together, for the same bits)
static double rows_per_expert(const moe_problem_t *p) {  // of one that has any, about
    const int slots = p->T * p->k;
    return (double)slots / (p->E < slots ? p->E : slots);
}
static double stages_of(const moe_problem_t *p, FfnOp op, const FfnArgs &a) {
    return op == kFfnDw ? rows_per_expert(p) * elem_bytes(p) / 64 : (op == kFfnDx ? 2.0 : 1.0) * a.K * elem_bytes(p) / 64;
}
static size_t sums_of(const moe_problem_t *p, FfnOp op, const FfnArgs &a) {  // bytes of a part's
    return (op == kFfnDw ? (size_t)p->E * a.M : (size_t)a.rows) * a.N * matrices_of(op, a) * 4;
}
// Room for the sums of whatever parts the product is cut into, with these rows or with fewer: a product of rows may be cut into more parts where there are
// fewer rows (their tiles leave CUs idle, and their sums fit kPartBytes), and a program asks once, for the most rows it has.
static size_t room_of(const moe_problem_t *p, FfnOp op, const FfnArgs &a) {
    int s = 1;
    while (2 * s <= kMostParts && stages_of(p, op, a) / (2 * s) >= kLeastStages) s *= 2;  // (not more of them with fewer rows)
    const size_t sums = sums_of(p, op, a);
    if (op == kFfnDw)  // the sums are of the same size whatever the rows
        while (s > 1 && s * sums > kPartBytes) s /= 2;
    return s == 1 ? 0 : std::min(s * sums, kPartBytes);
}
static Choice choose(const moe_problem_t *p, FfnOp op, const FfnArgs &a) {
    const int slots = p->T * p->k, experts = p->E < slots ? p->E : slots, sz = elem_bytes(p), mats = matrices_of(op, a);
    const double rows = rows_per_expert(p);
    Choice best = {0, 1, 0};
    double best_us = 0;
    for (int k = 0; k < (sz == 4 || op == kFfnDw ? 2 : kKinds); ++k) {
        const Kind &t = sz == 2 ? kKindsBf16[k] : kKindsF32[k];
        const int cols = op == kFfnUp ? t.bn / 2 : t.bn;
        const double nt = (double)((a.N + cols - 1) / cols) * (op == kFfnDw ? mats : 1);
        // row blocks, half a one more per expert than its rows fill, and how many times 64 rows one lacks
        const double per_expert = rows / t.bm + 0.5 > 1 ? rows / t.bm + 0.5 : 1;
        const double blocks = op == kFfnDw ? (double)p->E * ((a.M + t.bm - 1) / t.bm) : experts * per_expert;
        const double lacks = op == kFfnDw ? 0 : floor((t.bm - rows / per_expert) / 64);
        const double stages = stages_of(p, op, a);
        const double longest = op == kFfnDw ? p->T * sz / 64. : stages;
        for (int s = 1; s <= kMostParts; s *= 2) {
            if (sz == 4 && k == 0 && longest / s > kOneSum) continue;
            if (s > 1 && stages / s < kLeastStages) break;
            const size_t bytes = s == 1 ? 0 : s * sums_of(p, op, a);
            if (bytes > kPartBytes) break;
            const double per = blocks * nt * s / (kCus * t.occ), rounds = per <= 1 ? 1 : per + 0.5;
            const double us = rounds * (stages / s * (t.stage_us - lacks * t.less_us) + t.more_us) + (s > 1 ? 6 + bytes / 2e6 : 0);
            if (best_us == 0 || us < best_us) best_us = us, best = {k, s, bytes};
        }
    }
    return best;
}

template <class T, FfnOp OP>
static int prepare(FfnArgs &a, Launch *l) {
    constexpr int COLS = OP == kFfnUp ? T::BN / 2 : T::BN;
    a.nt = (a.N + COLS - 1) / COLS * (OP == kFfnDw && a.o1 ? 2 : 1) * a.split;
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
    const size_t tiles = (blocks * a.nt + kTileQueues - 1) / kTileQueues * kTileQueues, room = (size_t)cus * T::OCC;
    l->kernel = (const void *)k_ffn<T, OP>;
    l->join = a.split > 1 ? (const void *)k_ffn_join<typename T::ET, OP> : nullptr;
    l->groups = (unsigned)(tiles < room ? tiles : room);
    l->smem = T::SMEM;
    l->bm = T::BM;
    l->planned = T::BM >= 64 && tiles >= kPlannedTiles * room;
    return MOE_OK;
}
template <typename ET, FfnOp OP>
static int prepare(int kind, FfnArgs &a, Launch *l) {
    if (kind == 0) return prepare<typename TileOf<ET, 0>::type, OP>(a, l);
    if (kind == 1) return prepare<typename TileOf<ET, 1>::type, OP>(a, l);
    if constexpr (OP != kFfnDw && sizeof(ET) == 2) {
        if (kind == 2) return prepare<typename TileOf<ET, 2>::type, OP>(a, l);
        return prepare<typename TileOf<ET, 3>::type, OP>(a, l);
    }
    return MOE_ERR_UNSUPPORTED;  // (no such kind)
}
// The kernel of both products of a backward call, NULL where their workgroups need different room.
template <typename ET, FfnOp OP, int KIND, int DW>
static const void *both_of() {
    typedef typename TileOf<ET, KIND>::type T;
    typedef typename TileOf<ET, DW>::type TDW;
    if constexpr ((OP == kFfnDh || OP == kFfnDx) && T::OCC == TDW::OCC)
        return (const void *)k_ffn_both<T, OP, TDW>;
    else
        return nullptr;
}
template <typename ET, FfnOp OP>
static const void *both_of(int kind, int dw) {
    if (kind == 0) return dw ? both_of<ET, OP, 0, 1>() : both_of<ET, OP, 0, 0>();
    if (kind == 1) return dw ? both_of<ET, OP, 1, 1>() : both_of<ET, OP, 1, 0>();
    if constexpr (sizeof(ET) == 2) {
        if (!dw) return kind == 2 ? both_of<ET, OP, 2, 0>() : both_of<ET, OP, 3, 0>();
    }
    return nullptr;
}
template <FfnOp OP>
static int prepare(const moe_problem_t *p, FfnArgs &a, float *part, Launch *l) {
    const Choice c = choose(p, OP, a);
    a.split = c.split, a.part = part, l->kind = c.kind, l->part_bytes = (c.part_bytes + 255) / 256 * 256;
    return p->dtype == MOE_DT_F32 ? prepare<float, OP>(c.kind, a, l) : prepare<bf16_t, OP>(c.kind, a, l);
}
// The workspace: two plans, then the parts' sums of a call's products.
static FfnPlan *plans_of(void *workspace) { return (FfnPlan *)workspace; }
static float *parts_of(void *workspace) { return (float *)((char *)workspace + (2 * sizeof(FfnPlan) + 255) / 256 * 256); }

// A call's launches: a product of rows (any but dw), dw, or both.
template <FfnOp OP>
static int launch(const moe_problem_t *p, FfnArgs *rows, FfnArgs *dw, void *workspace, void *stream) {
    hipStream_t st = (hipStream_t)stream;
    Launch l[2] = {};
    FfnArgs *a[2] = {rows, dw};
    float *parts = parts_of(workspace);
    if (rows)
        if (const int rc = prepare<OP>(p, *rows, parts, &l[0])) return rc;
    if (dw)
        if (const int rc = prepare<kFfnDw>(p, *dw, parts + (rows ? l[0].part_bytes / 4 : 0), &l[1])) return rc;
    const void *both = nullptr;
    if (rows && dw) both = p->dtype == MOE_DT_F32 ? both_of<float, OP>(l[0].kind, l[1].kind) : both_of<bf16_t, OP>(l[0].kind, l[1].kind);
    for (int i = 0; i < 2; ++i)
        if (a[i])
            if (const int rc = allow_lds(both ? both : l[i].kernel, l[i].smem)) return rc;
    FfnPlan *plans = plans_of(workspace);
    if (l[0].planned || l[1].planned) {
        FfnPlanArgs plan = {};
        if (l[0].planned) plan.rows = *rows, plan.rows_plan = plans, plan.bm = l[0].bm, rows->plan = plans;
        if (l[1].planned) plan.dw = *dw, plan.dw_plan = plans + 1, dw->plan = plans + 1;
        hipLaunchKernelGGL(k_ffn_plan, dim3(2), dim3(kThreads), 0, st, plan);
        if (hipGetLastError() != hipSuccess) return MOE_ERR_HIP;
    }
    if (both) {
        unsigned first = l[0].groups;
        void *args[] = {rows, dw, &first};
        if (hipLaunchKernel(both, dim3(l[0].groups + l[1].groups), dim3(kThreads), args, l[0].smem, st) != hipSuccess) return MOE_ERR_HIP;
    }
    for (int i = 0; i < 2; ++i) {
        if (!a[i]) continue;
        void *args[] = {a[i]};
        if (!both && hipLaunchKernel(l[i].kernel, dim3(l[i].groups), dim3(kThreads), args, l[i].smem, st) != hipSuccess) return MOE_ERR_HIP;
        if (!l[i].join) continue;
        const size_t pieces = (i ? (size_t)a[i]->E * a[i]->M * (a[i]->o1 ? 2 : 1) : (size_t)a[i]->rows) * (a[i]->N / 8), groups = (pieces + kThreads - 1) / kThreads;
        if (hipLaunchKernel(l[i].join, dim3((unsigned)(groups < 4096 ? groups : 4096)), dim3(kThreads), args, 0, st) != hipSuccess) return MOE_ERR_HIP;
    }
    return MOE_OK;
}
static FfnArgs args_of(const moe_problem_t *p, const int32_t *counts) {
    FfnArgs a = {};
    a.E = p->E; a.rows = rows_of(p); a.capacity = p->capacity; a.counts = counts; a.split = 1;
    return a;
}

extern "C" {

size_t moe_ffn_workspace_bytes(const moe_problem_t *p) {
    if (check_problem(p) != MOE_OK) return 0;
    size_t parts[6];  // up, down, dh, dx, dW2, dW1 and dW3
    for (int i = 0; i < 6; ++i) {
        FfnArgs a = args_of(p, nullptr);
        const FfnOp op = (FfnOp)(i < kFfnDw ? i : kFfnDw);
        const bool down = i == kFfnDw;
        a.down = down, a.M = down ? p->f : p->d, a.N = op == kFfnDw ? (down ? p->d : p->f) : op == kFfnUp || op == kFfnDh ? p->f : p->d;
        a.K = op == kFfnUp || op == kFfnDh ? p->d : p->f;
        parts[i] = (room_of(p, op, a) + 255) / 256 * 256;
    }
    const size_t down_backward = parts[kFfnDh] + parts[4], up_backward = parts[kFfnDx] + parts[5];
    return (size_t)((char *)parts_of(nullptr) - (char *)nullptr) + std::max({parts[kFfnUp], parts[kFfnDown], down_backward, up_backward});
}

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
        a.down = true; a.M = p->f; a.N = p->d;
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
