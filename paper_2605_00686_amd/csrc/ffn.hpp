// The experts' products as calls of their own, forward and backward: rows sorted by expert times the expert's weights, with the
// activation (or its gradient) taken from the fp32 sums before they are rounded.
//
//   up       g = x W1[e], u = x W3[e], h = silu(g) u        rows x d  times d x f, twice
//   down     y = h W2[e]                                    rows x f  times f x d
//   dh       dh = dy W2[e]^T, taken on to dg and du         rows x d  times (f x d)^T
//   dx       dx = dg W1[e]^T + du W3[e]^T                   rows x 2f times (d x 2f)^T: one reduction over both
//   dw       dW[e] = a^T b over the rows of e               (rows x M)^T times rows x N
//
// All are tiles of C[m,n] = sum over k of A(m,k) B(k,n) on the matrix cores; what differs is which of an operand's indices is contiguous
// in memory, k ("KC" below) or the other one, and what is done with a tile's sums.  Sums are fp32, outputs are rounded once.
//
// What bounds them: with hundreds of rows per expert the matrix cores (2 operations per multiply, 1.2 PFLOP/s of bf16 in a large product of the
// library's on this card, whose clock falls to 1.55 GHz under that load); with dozens and fewer the weights, read once (5 to 6 TB/s).  Reached:
// 16384 x 2 of 8 experts of 4096 x 14336 up 1.15 PFLOP/s, dx and dw 1.14 together; 128 x 8 of 128 of 2048 x 768 down 5.9 TB/s; 4096 x 8 of 128 of 2048 x
// 768, where both take about the same, up 300 us, of which its bytes take 222 in a copy.  What is left of the matrix cores' time: a stage
// of 256 x 256 x 32 takes 1400 cycles, 1024 of them products; the rest is 24 to 40 LDS reads and 8 loads per wavefront, a barrier, and dx's
// rows of 64 bytes, half a cache line each, which ask the L2 twice.  One workgroup of 4 wavefronts per CU with 128 x 128 sums each reads LDS
// least; 8 wavefronts, two workgroups of 128 x 256, stages of 128 bytes and starts that are staggered were level or slower.
//
// Figures here and of the choices in moe_ffn.hip are of one build: calls one after another in a graph, with two sets of inputs in turn, median on one card
// ("kernel": of a kernel trace).  The same case is 2 % away on another card or day, and a row of calls from a program up to 6 %.
#pragma once
#include <type_traits>

#include "gemm_bf16.hpp"
#include "pieces.hpp"
#include "swiglu8.hpp"
#include "tile_lists.hpp"

namespace moe {

typedef long long i64;

enum FfnOp { kFfnUp, kFfnDown, kFfnDh, kFfnDx, kFfnDw };

struct FfnArgs {
    int E, rows, capacity;
    const int32_t *counts;
    int M, N, K;     // N columns per matrix; K reduction steps per pair of operands; dw: M x N per matrix, reduction over the rows
    bool down;       // dw: it is dW2
    int mt, nt;      // column tiles of all matrices; dw: row tiles
    long long lda, ldb, ldo, ldg;  // elements from one row to the next: operands, outputs, g and u
    long long eb, eo;              // elements from one expert's matrix to the next: weights; dw: outputs
    const void *A0, *A1, *B0, *B1;
    const void *g, *u;  // dh: the activation's inputs
    void *o0, *o1, *o2;
    int split;    // parts that the reduction is cut into; their sums go to `part`, and k_ffn_join makes the outputs of them
    float *part;  // [split][rows][N] (up: g then u for each part); dw: [split][matrix][E][M][N]
    const struct FfnPlan *plan;  // of k_ffn_plan, NULL: every workgroup makes its own tables and takes every n-th tile
};

// One operand's stage: R indices x KB bytes of the reduction (64: 32 steps of bf16, 16 of fp32), R * KB bytes of LDS.
//   KC:     [R][KB bytes]
//   not KC: [steps][R]
// A load instruction moves 64 x 16 bytes into consecutive LDS, so a lane's place there says which piece of 16 bytes it fetches: pieces are
// placed so that the reads below meet no bank twice.
template <typename ET, int R, bool KC_, int KB, int WAVES>
struct Operand {
    static constexpr bool KC = KC_;
    static constexpr int SZ = sizeof(ET), STEPS = KB / SZ, BYTES = R * KB;
    static constexpr int INSTR = BYTES / 1024, PER_WAVE = (INSTR + WAVES - 1) / WAVES;
    static constexpr int ROW = KC ? KB : R * SZ;  // bytes of a row in LDS
    static constexpr int PIECES = ROW / 16, ROWS_PER_INSTR = 64 / PIECES;
    static constexpr int READS = KC ? 1 : SZ == 2 ? 2 : 4;  // LDS instructions per fragment
    static_assert(KC || SZ * R >= 128, "rows the placement is made for");
    static __device__ __forceinline__ int place(int row, int c) {  // (its own inverse)
        if (KC) return c ^ (KB == 64 ? (row >> 2) & 3 : (row >> 1) & 7);
        if (SZ == 4) return c ^ (((row >> 2) & 1) << 3);
        return R >= 128 ? c ^ ((row & 3) << 2) : c ^ (((row >> 1) & 1) << 2);
    }
    // (where there are fewer instructions than wavefronts the upper ones repeat the lower ones': the same bytes to the same place)
    static __device__ __forceinline__ int instr(int wave, int i) { return (i * WAVES + wave) % INSTR; }
    static __device__ __forceinline__ int row_of(int instr, int lane) { return instr * ROWS_PER_INSTR + lane / PIECES; }
    static __device__ __forceinline__ int piece_of(int instr, int lane) { return place(row_of(instr, lane), lane % PIECES); }
};

// Asynchronous load of 64 x 16 bytes to LDS.  Inline assembly: the compiler would wait for its own in front of every LDS read.
__device__ __forceinline__ void load_to_lds(const char *src, u32 lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" : : "s"(__builtin_amdgcn_readfirstlane(lds)), "v"(src) : "m0");
}

// A workgroup's row block, or dw's expert: rows [begin, begin + used) are expert e's, those up to begin + extent nobody's.
struct Segment {
    int e, begin, used, extent, block;
};
// Where every expert's rows lie, and which tiles each XCD takes.
struct FfnTables {
    __align__(16) int used[kMaxExperts];
    int begin[kMaxExperts + 1];  // begin[E]: behind the last one's (ragged)
    int first[kMaxExperts + 1];  // first row block of an expert, of the rows of nobody behind the last (ragged); dw: rows before, and kDwStart for each expert
    int order[kMaxExperts];      // dw's plan: the tiles are in this order of experts
    int edge[kTileQueues + 1];   // tiles [edge[x], edge[x + 1]) are XCD x's
    int next;                    // in a workgroup's copy: the tile it takes next
    u64 sum[8];                  // scratch
};
struct FfnPlan {
    FfnTables tables;
    mutable Counter taken[kTileQueues];  // tiles handed out of an XCD's list, beyond the first ones
};

// MB x NB blocks of 32 x 32 per wavefront, WM x WN wavefronts (row blocks go round those of a column) and KW of each, which share a stage's steps;
// stages of KB bytes of the reduction, as many as fit the LDS of OCC workgroups per CU.
template <typename ET_, int MB_, int NB_, int WM_, int WN_, int KW_, int KB_, int OCC_>
struct FfnTile {
    typedef ET_ ET;
    static constexpr int MB = MB_, NB = NB_, WM = WM_, WN = WN_, KW = KW_, KB = KB_, OCC = OCC_, WAVES = WM * WN * KW;
    static constexpr int BM = 32 * MB * WM, BN = 32 * NB * WN;
    static constexpr int ROOM = (160 * 1024 / OCC - (int)sizeof(FfnTables)) / 1024 * 1024, SMEM = ROOM + (int)sizeof(FfnTables);
    static constexpr int stage_bytes(int live) { return (BN + BM / MB * live) * KB; }  // of a tile with `live` row blocks per wavefront
    static constexpr int stages(int live) { return ROOM / stage_bytes(live) < 7 ? ROOM / stage_bytes(live) : 7; }
    // fp32: sums of this many stages are added up apart, where there are registers for them (64 rows; 128 rows would spill 100 of them and more).
    // A sum's roundings, six per 16 steps, are those of its length.  512 x 2 of 8 experts of 8192 x 2048, dx, 2-norm of the error against 64 bits:
    // one sum of 16384 steps 1.1e-6, sums of 32 stages 4e-7.
    static constexpr int SUM_STAGES = sizeof(ET) == 4 && MB * NB <= 2 ? 32 : 0;
    static_assert(WAVES * 64 == kThreads, "threads");
};

__device__ __forceinline__ u64 scan_workgroup(u64 v, u64 *lds, u64 *total) {  // inclusive, kThreads threads
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const u64 o = __shfl_up(v, d);
        if (lane >= d) v += o;
    }
    if (lane == 63) lds[wave] = v;
    __syncthreads();
    u64 before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) {
        if (w < wave) before += lds[w];
        all += lds[w];
    }
    *total = all;
    return v + before;
}

// The last of the E + 1 ascending numbers that is `v` or less (the first one is).
__device__ __forceinline__ int last_up_to(const int *list, int n, int v) {
    int found = 0;
    for (int i = threadIdx.x & 63; i - (int)(threadIdx.x & 63) < n; i += 64) found += __popcll(__ballot(i < n && list[i] <= v));
    return uniform(found) - 1;
}

// Tiles of an expert in groups of kTileGroup rows of tiles, column by column inside a group: the 32 that an XCD works on at a time share operands in its
// L2.  16384 x 2 of 8 experts of 4096 x 14336 up, ms, by 1 / 2 / 3 / 4 / 6 / 8: 8.05 / 7.11 / 6.90 / 6.74 / 6.67 / 6.74; 4096 x 8 of 128 of 2048 x 768 the same
// by all.  Groups that go over experts' ends took 6 % longer for 4096 x 4 of 128 of 2880 x 2880 down.
constexpr int kTileGroup = 6;
__device__ __forceinline__ void tile_in_groups(int t, int rows, int cols, int *r, int *c) {
    const int group = t / (kTileGroup * cols), in = t - group * kTileGroup * cols, first = group * kTileGroup;
    const int n = min(kTileGroup, rows - first);
    *r = first + in % n, *c = in / n;
}

// The tables (in LDS), by kThreads threads; thread i has expert i.  Workgroups go round the eight XCDs, and each XCD takes a stretch of the tiles,
// whose neighbours read the same operands, from its own L2.
template <bool DW>
__device__ __forceinline__ void make_tables(const FfnArgs &a, int bm, FfnTables *t) {
    const int tid = threadIdx.x;
    static_assert(kThreads >= kMaxExperts, "a thread per expert");
    const int n = tid < a.E ? min(max(a.counts[tid], 0), a.rows) : 0;
    int begin = tid * a.capacity, used = min(n, a.capacity), first, total, last = a.rows;
    u64 all;
    if (a.capacity) {
        if (DW) {
            const int to = (int)scan_workgroup((u64)(tid < a.E ? used + kDwStart : 0), t->sum, &all);
            first = to - used - kDwStart, total = (int)all;
        } else {
            const int blocks = (a.capacity + bm - 1) / bm;
            first = tid * blocks, total = a.E * blocks;
        }
    } else {
        // rows and blocks in one scan, 39 and 25 bits
        constexpr u64 kRows = ((u64)1 << 39) - 1;
        const u64 end = scan_workgroup((u64)((n + bm - 1) / bm) << 39 | (u64)n, t->sum, &all), rows_end = end & kRows;
        last = (int)min(all & kRows, (u64)a.rows);
        begin = (int)min(rows_end - n, (u64)a.rows), used = (int)min(rows_end, (u64)a.rows) - begin;
        if (DW) {
            first = begin + tid * kDwStart, total = last + a.E * kDwStart;
        } else if ((all & kRows) <= (u64)a.rows && a.rows <= 1 << 29) {
            first = (int)(end >> 39) - (n + bm - 1) / bm, total = (int)(all >> 39);
        } else {  // counts that are cut, or more blocks than 25 bits hold
            const int blocks = (used + bm - 1) / bm;
            first = (int)scan_workgroup((u64)blocks, t->sum + 4, &all) - blocks, total = (int)all;
        }
    }
    if (tid < a.E) t->begin[tid] = begin, t->used[tid] = used, t->first[tid] = first;
    if (tid == 0) t->begin[a.E] = last, t->first[a.E] = total;
    if (!DW && tid <= kTileQueues) {
        const int row_blocks = total + (a.capacity ? 0 : (a.rows - last + bm - 1) / bm);
        t->edge[tid] = (int)((i64)row_blocks * a.nt * tid / kTileQueues);
    }
    __syncthreads();
    if (DW) {
        static_assert(kDwLists == kTileQueues && kMaxExperts <= 256, "as dw_edge has them");
        if (tid <= kTileQueues) t->edge[tid] = dw_edge(tid, a.E, a.mt * a.nt, total, t->first, t->used);
        __syncthreads();
    }
}

// dw: a plan deals the experts out to the XCDs by their rows, from the largest to the smallest and back again, and each XCD begins with its largest.
// (For fewer experts, stretches of the same work are more even.)  us, in the experts' order / by rows: 4096 x 8 of 128 of 2048 x 768 dW2 217 / 210,
// dW1 and dW3 400 / 390.  The products of rows stay in the experts' order: their short tiles, which wait for weights, side by side at the end
// take longer than mixed with the others, by 7 % (up) and 6 % (dx).
constexpr int kDealtExperts = 32;
__device__ __forceinline__ void deal_experts(const FfnArgs &a, FfnTables *t) {
    const int tid = threadIdx.x, mine = tid < a.E ? t->used[tid] : 0;
    if (a.E < kDealtExperts) {
        if (tid < a.E) t->order[tid] = tid;
        __syncthreads();
        return;
    }
    int rank = 0;
    for (int e = 0; e < a.E; e += 4) {
        const int4 n = *(const int4 *)&t->used[e];  // (the last ones may be of no expert)
        const int four[4] = {n.x, n.y, n.z, n.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) rank += e + j < a.E && (four[j] > mine || (four[j] == mine && e + j < tid));
    }
    // rank r is number r / 8 of its XCD
    const int rounds = a.E / kTileQueues, rest = a.E % kTileQueues;
    auto before = [&](int x) {  // experts of the XCDs before x
        return x * rounds + (rounds & 1 ? max(x - (kTileQueues - rest), 0) : min(x, rest));
    };
    if (tid < a.E) {
        const int round = rank / kTileQueues, x = round & 1 ? kTileQueues - 1 - rank % kTileQueues : rank % kTileQueues;
        t->order[before(x) + round] = tid;
    }
    if (tid <= kTileQueues) t->edge[tid] = before(tid) * a.mt * a.nt;
    __syncthreads();
}

// The tables of a call's products, a workgroup each.
struct FfnPlanArgs {
    FfnArgs rows, dw;  // the launches'
    FfnPlan *rows_plan, *dw_plan;  // NULL: there is none
    int bm;
};
__global__ __launch_bounds__(kThreads) void k_ffn_plan(FfnPlanArgs a) {
    __shared__ FfnTables t;
    const int tid = threadIdx.x;
    auto out = [&](FfnPlan *p) {
        for (int i = tid; i < (int)(sizeof(FfnTables) / 4); i += kThreads) ((u32 *)&p->tables)[i] = ((const u32 *)&t)[i];
        if (tid < kTileQueues) p->taken[tid].v = 0;
        __syncthreads();
    };
    if (blockIdx.x == 0) {
        if (a.rows_plan) make_tables<false>(a.rows, a.bm, &t), out(a.rows_plan);
    } else if (a.dw_plan) {
        make_tables<true>(a.dw, 1, &t), deal_experts(a.dw, &t), out(a.dw_plan);
    }
}

// The fragments of N blocks of an operand for step `kk` (32 bytes of the reduction) of a stage: lane l has index l & 31 of a block and the
// steps of its half, l >> 5: 8 of bf16, 4 of fp32.
template <class O, int N, int M>
__device__ __forceinline__ void read_frags(const char *stage, int kk, const int (&at)[M], int lane, u32x4_t (&f)[N]) {
    static_assert(N <= M, "blocks");
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if constexpr (O::KC) {
            const int r = at[i] + (lane & 31);
            f[i] = *(const u32x4_t *)(stage + r * O::ROW + O::place(r, kk * 2 + (lane >> 5)) * 16);
        } else if constexpr (O::SZ == 2) {
            // (each 16 lanes read 4 steps x 16 indices and hand them out transposed)
            const int c = at[i] + 16 * ((lane >> 4) & 1) + 4 * (lane & 3), k = 8 * (lane >> 5) + ((lane & 15) >> 2);
            const char *p = stage + (kk * 16 + k) * O::ROW + O::place(k, c >> 3) * 16 + (c & 7) * 2;
            typedef s16x4_t __attribute__((address_space(3))) *At;
            const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((At)p), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((At)(p + 4 * O::ROW));
            f[i] = __builtin_bit_cast(u32x4_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            const int c = at[i] + (lane & 31), k = 4 * (lane >> 5);
            const char *p = stage + (kk * 8 + k) * O::ROW + O::place(k, c >> 2) * 16 + (c & 3) * 4;
#pragma unroll
            for (int j = 0; j < 4; ++j) f[i][j] = *(const u32 *)(p + j * O::ROW);
        }
    }
}
// Until no more than the loads of `behind` stages, LPS each, are in flight.
template <int MOST, int LPS>
__device__ __forceinline__ void wait_behind(int behind) {
    if constexpr (MOST <= 0) {
        wait_vmcnt<0>();
    } else {
        static_assert(MOST * LPS <= 63, "vmcnt range");
        if (behind >= MOST)
            wait_vmcnt<MOST * LPS>();
        else
            wait_behind<MOST - 1, LPS>(behind);
    }
}

template <typename ET>
__device__ __forceinline__ void multiply(const u32x4_t &b, const u32x4_t &a, f32x16_t &acc) {
    if constexpr (sizeof(ET) == 2) {
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, b), __builtin_bit_cast(bf16x8_t, a), acc, 0, 0, 0);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(b[j]), __uint_as_float(a[j]), acc, 0, 0, 0);
    }
}

// Eight fp32 numbers as three bf16 numbers each: 2^24 x = p0 + p1 + p2 with |p1| and |p2| up to 2^-8 and 2^-17 of that, and nothing left, since at that
// scale every bit that an fp32 number can have is one of a normal bf16 number.  (As they are, numbers below 2^-110 would lose bits and those
// below 2^-133 all of them, whatever they are multiplied by; the scaling costs 1 to 4 % of a call.)  Of the nine products of two numbers the six
// largest are taken; the others come to 2^-24 of the whole at most, half a step of fp32.  On the matrix cores those six take 192 cycles for 32 x 32
// x 16, the fp32 instructions 512.  Sums are 2^48 times as large until their tile's end: a number of 2^104 and more, or one that is not finite,
// and a sum of 2^80 and more come out infinite or as NaN.
constexpr float kCutScale = 0x1p24f;
struct Cut {
    u32x4_t part[3];
};
__device__ __forceinline__ Cut cut_f32(const u32x4_t &lo, const u32x4_t &hi) {
    Cut c;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float x = __uint_as_float(i < 2 ? lo[2 * i] : hi[2 * i - 4]) * kCutScale, y = __uint_as_float(i < 2 ? lo[2 * i + 1] : hi[2 * i - 3]) * kCutScale;
#pragma unroll
        for (int j = 0; j < 3; ++j) {
            const u32 p = pack_bf16x2(x, y);
            c.part[j][i] = p;
            x -= __uint_as_float(p << 16), y -= __uint_as_float(p & 0xffff0000u);
        }
    }
    return c;
}

// Workgroup `group` of `groups`.
template <class T, FfnOp OP>
__device__ __forceinline__ void ffn(const FfnArgs &a, u32 group, u32 groups) {
    typedef typename T::ET ET;
    constexpr bool DW = OP == kFfnDw, AK = !DW, BK = OP == kFfnDh || OP == kFfnDx, GATED = OP == kFfnUp;
    typedef Operand<ET, T::BM, AK, T::KB, T::WAVES> OA;
    typedef Operand<ET, T::BN, BK, T::KB, T::WAVES> OB;
    constexpr int LPS = OA::PER_WAVE + OB::PER_WAVE, SZ = sizeof(ET), STEPS = OA::STEPS, PIECE = 16 / SZ;
    constexpr int COLS = GATED ? T::BN / 2 : T::BN;  // columns of a matrix per tile
    static_assert(!GATED || T::NB % 2 == 0, "g and u of the same columns");
    extern __shared__ __align__(128) char smem[];
    char *stages = smem;
    FfnTables *tables = (FfnTables *)(smem + T::ROOM);
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), wn = wave % T::WN, wm = wave / T::WN % T::WM, wk = wave / (T::WN * T::WM);
    if (a.plan) {
        for (int i = tid; i < (int)(sizeof(FfnTables) / 4); i += kThreads) ((u32 *)tables)[i] = ((const u32 *)&a.plan->tables)[i];
        __syncthreads();
    } else {
        make_tables<DW>(a, T::BM, tables);
    }
    const int row_blocks = uniform(tables->edge[kTileQueues]) / a.nt;  // (dw: of tiles)
    // The tile after this one.  Where there is a plan, tiles are handed out as workgroups come for them, first of the own XCD's list, then of
    // the others': experts' last row blocks, and dw's experts, differ in what they take.  (Without / with a plan: 4096 x 4 of 128 of 2880 x 2880 down
    // 568 / 530 us, 16384 x 2 of 8 of 4096 x 14336 dx and dw 14.5 / 13.6 ms.)
    int list = group % kTileQueues;
    const int mine = group / kTileQueues, per_list = groups / kTileQueues;
    int taken = 0;  // thread 0: what it was given of `list`
    auto ask = [&]() __attribute__((always_inline)) {
        if (a.plan && tid == 0) taken = (int)atomicAdd(&a.plan->taken[list].v, 1u);
    };
    auto answer = [&]() __attribute__((always_inline)) {  // thread 0; the others read it behind a barrier
        // (Waited for here by everybody, asked or not: the compiler would do so where it next needs the register, which may be in the loops below, and
        // for all of a tile's loads in flight: a fifth more time for 4096 x 4 of 128 of 2880 x 2880 down.)
        asm volatile("" : "+v"(taken));
        if (!a.plan || tid) return;
        int t = tables->edge[list] + per_list + taken;
        for (int tries = 1; t >= tables->edge[list + 1] && tries < kTileQueues; ++tries) {
            list = (list + 1) % kTileQueues;
            t = tables->edge[list] + per_list + (int)atomicAdd(&a.plan->taken[list].v, 1u);
        }
        tables->next = t < tables->edge[list + 1] ? t : -1;
    };
    int tile = uniform(tables->edge[list]) + mine;
    if (tile >= uniform(tables->edge[list + 1])) {
        if (!a.plan) return;
        ask();
        answer();
        __syncthreads();
        tile = uniform(tables->next);
        if (tile < 0) return;
    }

    const int half = a.K / STEPS;  // stages of a pair of operands
    const int per_matrix = (a.N + COLS - 1) / COLS;  // dw: column tiles of the second matrix lie behind those of the first
    struct Tile {
        Segment s;
        int row0, n0, matrix;  // first row (of the segment's; dw: of the matrix) and column
        int part, k0, nk, end;  // part of the reduction: its first stage and how many; stages of the whole
    };
    auto tile_at = [&](int t) __attribute__((always_inline)) {
        Tile w;
        int r, c;
        if (DW) {
            const int per = a.mt * a.nt;
            const int at = t / per;
            w.s.e = a.plan ? uniform(tables->order[at]) : at, w.s.block = 0;
            tile_in_groups(t - at * per, a.mt, a.nt, &r, &c);
            w.s.begin = uniform(tables->begin[w.s.e]), w.s.used = w.s.extent = uniform(tables->used[w.s.e]);
            w.row0 = r * T::BM;
            w.end = (w.s.used + STEPS - 1) / STEPS;
        } else {
            const int e = last_up_to(tables->first, a.E + 1, t / a.nt), first = uniform(tables->first[e]);
            tile_in_groups(t - first * a.nt, (e < a.E ? uniform(tables->first[e + 1]) : row_blocks) - first, a.nt, &r, &c);
            w.s.e = e, w.s.block = r;
            w.s.begin = uniform(a.capacity ? e * a.capacity : tables->begin[e]);
            w.s.used = e < a.E ? uniform(tables->used[e]) : 0;
            w.s.extent = a.capacity ? a.capacity : e < a.E ? w.s.used : a.rows - w.s.begin;
            w.row0 = w.s.block * T::BM;
            w.end = w.row0 >= w.s.used ? 0 : OP == kFfnDx ? 2 * half : half;
        }
        w.part = c % a.split, c /= a.split;
        w.k0 = (int)((i64)w.end * w.part / a.split), w.nk = (int)((i64)w.end * (w.part + 1) / a.split) - w.k0;
        w.matrix = DW ? c / per_matrix : 0;
        w.n0 = (c - w.matrix * per_matrix) * COLS;
        return w;
    };

    // Row blocks that are not full have loops of their own, for a quarter, a half and three quarters of the rows, and more stages in flight: 0.38 us
    // a stage for 64 rows, 0.82 for 256 (16384 rows x 2048 x 2048 on 8 experts, kernel).
    constexpr bool SHORT = !DW && SZ == 2 && T::MB % 4 == 0;
    auto loads_of_a = [](int live) __attribute__((always_inline)) { return (OA::INSTR * live / T::MB + T::WAVES - 1) / T::WAVES; };

    // ---- loads.  A lane's places in the operands; they go on from stage to stage.
    const char *ap[OA::PER_WAVE], *bp[OB::PER_WAVE];
    const size_t lda = (size_t)a.lda * SZ, ldb = (size_t)a.ldb * SZ;
    const size_t a_step = AK ? T::KB : STEPS * lda, b_step = BK ? T::KB : STEPS * ldb;
    const u32 lds = lds_offset(stages);
    int next, k0, nk, end, used;  // the stage to load; stages and rows of the tile that is loaded
    int live, a_loads;   // row blocks per wavefront it has, loads of A per wavefront
    u32 stage_bytes, to_end;
    u32 to;              // where it goes
    // before a stage's loads: on to the second pair of operands; rows past the expert's last one are that one again
    auto begin_stage = [&]() __attribute__((always_inline)) {
        if (OP == kFfnDx && next == half && k0 < half) {
            const long long da = (const char *)a.A1 - (const char *)a.A0 - (long long)half * T::KB, db = (const char *)a.B1 - (const char *)a.B0 - (long long)half * T::KB;
#pragma unroll
            for (int i = 0; i < OA::PER_WAVE; ++i) ap[i] += da;
#pragma unroll
            for (int i = 0; i < OB::PER_WAVE; ++i) bp[i] += db;
        }
        if (OP == kFfnDw && next == end - 1) {
            const int left = used - 1 - next * STEPS;
#pragma unroll
            for (int i = 0; i < OA::PER_WAVE; ++i) ap[i] -= (size_t)max(OA::row_of(OA::instr(wave, i), lane) - left, 0) * lda;
#pragma unroll
            for (int i = 0; i < OB::PER_WAVE; ++i) bp[i] -= (size_t)max(OB::row_of(OB::instr(wave, i), lane) - left, 0) * ldb;
        }
    };
    auto load_one = [&](int i) __attribute__((always_inline)) {
        if (i < OA::PER_WAVE) {
            load_to_lds(ap[i], to + OB::BYTES + OA::instr(wave, i) * 1024);
            ap[i] += a_step;
        } else {
            const int j = i - OA::PER_WAVE;
            load_to_lds(bp[j], to + OB::instr(wave, j) * 1024);
            bp[j] += b_step;
        }
    };
    auto end_stage = [&]() __attribute__((always_inline)) {
        ++next;
        to += stage_bytes;
        if (to == to_end) to = lds;
    };
    auto load_stage = [&]() __attribute__((always_inline)) {
        begin_stage();
#pragma unroll
        for (int i = 0; i < LPS; ++i)
            if (i >= a_loads && i < OA::PER_WAVE)
                continue;
            else
                load_one(i);
        end_stage();
    };
    // The first stages of a tile: nobody may be reading the stages any more.  up: dealt out among the blocks of the last tile's results, of which it has
    // three times as many bytes as down.  All first / dealt out, us: 4096 x 8 of 128 of 2048 x 768 up 310 / 307, 16384 x 2 of 8 of 4096 x 14336 up
    // 6735 / 6670; dealt out for the gradients too, kernel, 722 / 722 and 13600 / 13670.
    constexpr bool DEAL = GATED && T::KW == 1;
    int until = 0;  // the stage behind them
    auto start = [&](const Tile &w) __attribute__((always_inline)) {
        next = k0 = w.k0, nk = w.nk, end = w.end, used = w.s.used, to = lds;
        if (DEAL) until = k0;
        if (!nk) return;
        const int rows = used - w.row0;
        live = !SHORT || rows > T::BM / 4 * 3 ? T::MB : rows > T::BM / 2 ? T::MB / 4 * 3 : rows > T::BM / 4 ? T::MB / 2 : T::MB / 4;
        a_loads = loads_of_a(live), stage_bytes = T::stage_bytes(live);
        const int ns = live == T::MB ? T::stages(T::MB) : live == T::MB / 4 * 3 ? T::stages(T::MB / 4 * 3) : live == T::MB / 2 ? T::stages(T::MB / 2) : T::stages(T::MB / 4);
        to_end = lds + ns * stage_bytes;
        const bool second = OP == kFfnDx && k0 >= half;  // of the pairs of operands
        const char *A = (const char *)(second ? a.A1 : a.A0) + (size_t)(second ? k0 - half : k0) * a_step;
        const char *B = (const char *)((DW && w.matrix) || second ? a.B1 : a.B0) + (size_t)(second ? k0 - half : k0) * b_step;
#pragma unroll
        for (int i = 0; i < OA::PER_WAVE; ++i) {
            const int in = OA::instr(wave, i), r = OA::row_of(in, lane), c = OA::piece_of(in, lane);
            if constexpr (AK) {
                ap[i] = A + (size_t)(w.s.begin + min(w.row0 + r, used - 1)) * lda + c * 16;
            } else {
                const int m = w.row0 + c * PIECE;
                ap[i] = A + (size_t)(w.s.begin + r) * lda + (size_t)(m < a.M ? m : 0) * SZ;
            }
        }
#pragma unroll
        for (int i = 0; i < OB::PER_WAVE; ++i) {
            const int in = OB::instr(wave, i), r = OB::row_of(in, lane), c = OB::piece_of(in, lane);
            if constexpr (BK) {
                bp[i] = B + (size_t)w.s.e * a.eb * SZ + (size_t)min(w.n0 + r, a.N - 1) * ldb + c * 16;
            } else {
                int n = c * PIECE;
                const char *from = B;
                if (GATED && n >= COLS) from += (const char *)a.B1 - (const char *)a.B0, n -= COLS;
                n += w.n0;
                const size_t first = DW ? (size_t)w.s.begin * ldb : (size_t)w.s.e * a.eb * SZ;
                bp[i] = from + first + (size_t)r * ldb + (size_t)(n < a.N ? n : 0) * SZ;
            }
        }
        const int ahead = min(nk, ns);
        if constexpr (DEAL)
            until = k0 + ahead;
        else
            for (int i = 0; i < ahead; ++i) load_stage();
    };
    auto load_first = [&]() __attribute__((always_inline)) {
        while (DEAL && next < until) load_stage();
    };

    // ---- products
    f32x16_t acc[T::MB][T::NB];
    int a_at[T::MB], b_at[T::NB];
#pragma unroll
    for (int mb = 0; mb < T::MB; ++mb) a_at[mb] = (mb * T::WM + wm) * 32;
#pragma unroll
    for (int nb = 0; nb < T::NB; ++nb)
        b_at[nb] = !GATED ? (wn * T::NB + nb) * 32 : nb < T::NB / 2 ? (wn * T::NB / 2 + nb) * 32 : COLS + (wn * T::NB / 2 + nb - T::NB / 2) * 32;

    // Fragments are read a step ahead of the products that take them; a stage's buffer is free when everybody has read its last
    // fragments, and the loads of the stage that goes there are dealt out over the steps that follow.
    constexpr int KK = T::KB / 32 / T::KW;  // a wavefront's steps per stage
    static_assert(KK % 2 == 0, "two sets of fragments in turn");
    auto products = [&](auto blocks, auto cut) __attribute__((always_inline)) {
        constexpr bool CUT = decltype(cut)::value, ASK = SZ == 2 || CUT;  // (once per tile)
        constexpr int LIVE = decltype(blocks)::value, NS = T::stages(LIVE), STAGE = T::stage_bytes(LIVE);
        static_assert(NS >= 2, "stages");
        constexpr int AL = (OA::INSTR * LIVE / T::MB + T::WAVES - 1) / T::WAVES, LPS = AL + OB::PER_WAVE;  // loads per wavefront and stage
        constexpr int LPK = (LPS + KK - 1) / KK;
        constexpr int NREAD = LIVE * OA::READS + T::NB * OB::READS, NMUL = LIVE * T::NB, NMFMA = NMUL * (SZ == 2 ? 1 : 4);
        struct Frags {
            u32x4_t a[LIVE], b[T::NB];
        };
        Frags f0, f1;
        auto read = [&](const char *stage, int kk, Frags &f) __attribute__((always_inline)) {
            read_frags<OA>(stage + OB::BYTES, wk * KK + kk, a_at, lane, f.a);
            read_frags<OB>(stage, wk * KK + kk, b_at, lane, f.b);
        };
        // products of `cur`, with the reads of `nxt` and, if LOADS, share `part` of a stage's loads in between
        auto step = [&](const char *stage, int kk, Frags &nxt, const Frags &cur, auto loads, int part) __attribute__((always_inline)) {
            constexpr bool LOADS = decltype(loads)::value;
            read(stage, kk, nxt);
#pragma unroll
            for (int mb = 0; mb < LIVE; ++mb)
#pragma unroll
                for (int nb = 0; nb < T::NB; ++nb) {
                    const int i = mb * T::NB + nb;
                    if (LOADS) {
#pragma unroll
                        for (int j = 0; j < LPK; ++j)
                            if (j * NMUL / LPK == i && part * LPK + j < LPS) load_one(part * LPK + j < AL ? part * LPK + j : part * LPK + j - AL + OA::PER_WAVE);
                    }
                    multiply<ET>(cur.b[nb], cur.a[mb], acc[mb][nb]);
                }
#pragma unroll
            for (int i = 0; i < NMFMA; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // a product ...
                if (i < NREAD) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);  // ... an LDS read
            }
            if (NREAD > NMFMA) __builtin_amdgcn_sched_group_barrier(0x100, NREAD - NMFMA, 0);
        };
        // stage kt has landed, and everybody has read what the next loads replace
        auto landed = [&](int kt, int behind) __attribute__((always_inline)) {
            wait_behind<NS - 1, LPS>(behind);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            __syncthreads();
            if (OP == kFfnDw && k0 + kt == end - 1 && used % STEPS) {
                // the steps past the expert's last row: zeros in both operands, whatever lies there
                char *stage = stages + kt % NS * STAGE;
                const int from = used % STEPS;
                for (int i = tid; i < (STEPS - from) * (T::BM * SZ / 16); i += kThreads) *(u32x4_t *)(stage + OB::BYTES + from * T::BM * SZ + i * 16) = u32x4_t{0, 0, 0, 0};
                for (int i = tid; i < (STEPS - from) * (T::BN * SZ / 16); i += kThreads)
                    *(u32x4_t *)(stage + from * T::BN * SZ + i * 16) = u32x4_t{0, 0, 0, 0};
                __syncthreads();
            }
        };
        landed(0, min(nk, NS) - 1);
        char *stage = stages;
        auto first_steps = [&](auto loads) __attribute__((always_inline)) {  // of a stage: all but the last
#pragma unroll
            for (int kk = 0; kk + 1 < KK; ++kk) {
                if (kk & 1)
                    step(stage, kk + 1, f0, f1, loads, kk + 1);
                else
                    step(stage, kk + 1, f1, f0, loads, kk + 1);
            }
        };
        auto on = [&]() __attribute__((always_inline)) {
            stage += STAGE;
            if (stage == stages + NS * STAGE) stage = stages;
        };
        if constexpr (CUT) {
            // (two workgroups per CU: while one reads and cuts, the other multiplies)
            Cut ca[LIVE], cb[T::NB];
            auto read_cut = [&]() __attribute__((always_inline)) {
                Frags lo, hi;
                read(stage, 0, lo);
                read(stage, 1, hi);
#pragma unroll
                for (int i = 0; i < LIVE; ++i) ca[i] = cut_f32(lo.a[i], hi.a[i]);
#pragma unroll
                for (int i = 0; i < T::NB; ++i) cb[i] = cut_f32(lo.b[i], hi.b[i]);
            };
            auto multiply_cut = [&]() __attribute__((always_inline)) {
                constexpr int kTerms[6][2] = {{2, 0}, {0, 2}, {1, 1}, {1, 0}, {0, 1}, {0, 0}};  // (the smallest first)
#pragma unroll
                for (int t = 0; t < 6; ++t)
#pragma unroll
                    for (int mb = 0; mb < LIVE; ++mb)
#pragma unroll
                        for (int nb = 0; nb < T::NB; ++nb) multiply<bf16_t>(cb[nb].part[kTerms[t][1]], ca[mb].part[kTerms[t][0]], acc[mb][nb]);
            };
            auto go_on = [&](int kt) __attribute__((always_inline)) {
                landed(kt, min(nk - 1 - kt, NS - 2));
                on();
                if (next < k0 + nk) load_stage();
                read_cut();
            };
            read_cut();
            if constexpr (T::SUM_STAGES != 0) {
                f32x16_t sum[LIVE][T::NB];
                for (int kt = 1, from = 0;; from = kt - 1) {
                    const int to = min(nk, from + T::SUM_STAGES);
                    for (; kt < to; ++kt) {
                        multiply_cut();
                        go_on(kt);
                    }
                    if (ASK && kt == nk) ask();
                    multiply_cut();
                    const bool last = kt == nk;
                    if (last && from == 0) break;
#pragma unroll
                    for (int mb = 0; mb < LIVE; ++mb)
#pragma unroll
                        for (int nb = 0; nb < T::NB; ++nb)
#pragma unroll
                            for (int v = 0; v < 16; ++v) {
                                const float x = from ? sum[mb][nb][v] + acc[mb][nb][v] : acc[mb][nb][v];
                                sum[mb][nb][v] = x;
                                acc[mb][nb][v] = last ? x : 0.f;
                            }
                    if (last) break;
                    go_on(kt);
                    ++kt;
                }
            } else {
                for (int kt = 1; kt < nk; ++kt) {
                    multiply_cut();
                    go_on(kt);
                }
                if (ASK) ask();
                multiply_cut();
            }
#pragma unroll
            for (int mb = 0; mb < LIVE; ++mb)
#pragma unroll
                for (int nb = 0; nb < T::NB; ++nb) acc[mb][nb] *= 1.f / (kCutScale * kCutScale);
        } else {
            read(stage, 0, f0);
            first_steps(std::false_type{});
            int kt = 1;
            for (; kt <= nk - NS; ++kt) {
                landed(kt, NS - 2);
                on();
                begin_stage();
                step(stage, 0, f0, f1, std::true_type{}, 0);
                first_steps(std::true_type{});
                end_stage();
            }
            for (; kt < nk; ++kt) {
                landed(kt, min(nk - 1 - kt, NS - 2));
                on();
                step(stage, 0, f0, f1, std::false_type{}, 0);
                first_steps(std::false_type{});
            }
            if (ASK) ask();  // (no load is in flight any more: the wait for the answer holds nothing up)
#pragma unroll
            for (int mb = 0; mb < LIVE; ++mb)
#pragma unroll
                for (int nb = 0; nb < T::NB; ++nb) multiply<ET>(f1.b[nb], f1.a[mb], acc[mb][nb]);
        }
        if constexpr (T::KW > 1) {  // the sums of the wavefronts that shared the steps meet with the first one's
            static_assert(T::KW == 2 && 2 * T::WM * T::WN * T::MB * T::NB * 2048 <= T::ROOM, "two of them");
            __syncthreads();
            f32x4_t *x = (f32x4_t *)stages + (wave % (T::WM * T::WN)) * T::MB * T::NB * 256 + lane;
#pragma unroll
            for (int mb = 0; mb < T::MB; ++mb)
#pragma unroll
                for (int nb = 0; nb < T::NB; ++nb)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const f32x16_t &v = acc[mb][nb];
                        if (wk) x[((mb * T::NB + nb) * 4 + q) * 64] = f32x4_t{v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
                    }
            __syncthreads();
#pragma unroll
            for (int mb = 0; mb < T::MB; ++mb)
#pragma unroll
                for (int nb = 0; nb < T::NB; ++nb)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const f32x4_t v = x[((mb * T::NB + nb) * 4 + q) * 64];
#pragma unroll
                        for (int j = 0; j < 4; ++j) acc[mb][nb][4 * q + j] += v[j];
                    }
        }
        if (ASK) answer();
        __syncthreads();
    };

    // ---- out.  The matrix cores leave lane l of a block with row l & 31 and columns 8 q + 4 (l >> 5) + 0..3, q = 0..3: 16 bytes of fp32, but 8 of
    // bf16, where the halves of a wavefront swap what they have of two q, so that the lower one has 16 bytes of one and the upper one of the
    // other.  Then lanes of 16 to 31 and of 0 to 15 swap, so that an access reaches 64 bytes of each of 16 rows: piece 2 j + i of a lane is
    // row 16 i + (l & 15), columns (4 j + 2 (l >> 4 & 1) + (l >> 5)) * PIECE and on.
    constexpr int COL_BLOCKS = GATED ? T::NB / 2 : T::NB;
    constexpr int PIECES = 32 * SZ / 32;  // pieces of 16 bytes that a lane has of a block: 2 of bf16, 4 of fp32
    auto swap16 = [&](u32x4_t (&v)[PIECES]) __attribute__((always_inline)) {  // (its own inverse)
#pragma unroll
        for (int i = 0; i < PIECES; i += 2)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const auto x = __builtin_amdgcn_permlane16_swap(v[i][j], v[i + 1][j], false, false);
                v[i][j] = x[0], v[i + 1][j] = x[1];
            }
    };
    auto pieces_of = [&](auto value, u32x4_t (&v)[PIECES]) __attribute__((always_inline)) {  // value(register)
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            if constexpr (SZ == 2) {
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const auto x = __builtin_amdgcn_permlane32_swap(pack_bf16x2(value(8 * i + 2 * j), value(8 * i + 2 * j + 1)),
                                                                    pack_bf16x2(value(8 * i + 4 + 2 * j), value(8 * i + 4 + 2 * j + 1)), false, false);
                    v[i][j] = x[0], v[i][2 + j] = x[1];
                }
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) v[i][j] = __float_as_uint(value(4 * i + j));
            }
        }
        swap16(v);
    };
    auto values_of = [&](u32x4_t (&v)[PIECES], float (&x)[16]) __attribute__((always_inline)) {  // the other way
        swap16(v);
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            if constexpr (SZ == 2) {
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const auto y = __builtin_amdgcn_permlane32_swap(v[i][j], v[i][2 + j], false, false);
#pragma unroll
                    for (int h = 0; h < 2; ++h) x[8 * i + 4 * h + 2 * j] = __uint_as_float(y[h] << 16), x[8 * i + 4 * h + 2 * j + 1] = __uint_as_float(y[h] & 0xffff0000u);
                }
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) x[4 * i + j] = __uint_as_float(v[i][j]);
            }
        }
    };
    // Where a lane's pieces of block (mb, nb) of a tile are; f(number of the piece, row of the segment or matrix, column) for those there are.
    auto each_piece = [&](const Tile &w, int mb, int nb, int l, auto f) __attribute__((always_inline)) {
        const int m = w.row0 + (mb * T::WM + wm) * 32 + (l & 15), n = w.n0 + (wn * COL_BLOCKS + nb) * 32 + ((l >> 4 & 1) * 2 + (l >> 5)) * PIECE;
        const int rows = DW ? a.M : w.s.extent;
#pragma unroll
        for (int i = 0; i < PIECES; ++i)
            if (m + i % 2 * 16 < rows && n + i / 2 * 4 * PIECE < a.N) f(i, m + i % 2 * 16, n + i / 2 * 4 * PIECE);
    };
    auto there = [&](const Tile &w, int mb, int nb) __attribute__((always_inline)) {  // any of the block
        return w.n0 + (wn * COL_BLOCKS + nb) * 32 < a.N && w.row0 + (mb * T::WM + wm) * 32 < (DW ? a.M : w.s.extent);
    };
    // dh: g and u of the blocks, GU_AHEAD ahead of the one that takes them
    constexpr int BLOCKS = T::MB * COL_BLOCKS, GU_MOST = SZ == 4 ? 1 : T::OCC == 1 ? 6 : 3, GU_AHEAD = OP != kFfnDh ? 0 : BLOCKS < GU_MOST ? BLOCKS : GU_MOST;
    u32x4_t gv[GU_AHEAD + 1][PIECES], uv[GU_AHEAD + 1][PIECES];
    auto load_gu = [&](const Tile &w, int block) __attribute__((always_inline)) {
        const int mb = block / COL_BLOCKS, nb = block % COL_BLOCKS, at = block % (GU_AHEAD + (OP != kFfnDh));
        if (!there(w, mb, nb)) return;
        int l = lane;
        asm volatile("" : "+v"(l));
        each_piece(w, mb, nb, l, [&](int i, int m, int n) __attribute__((always_inline)) {
            const size_t from = (size_t)(w.s.begin + m) * a.ldg + n;
            gv[at][i] = *(const u32x4_t *)((const ET *)a.g + from), uv[at][i] = *(const u32x4_t *)((const ET *)a.u + from);
        });
    };
    auto write_tile = [&](const Tile &w) __attribute__((always_inline)) {
        if (T::KW > 1 && wk) return;
#pragma unroll
        for (int mb = 0; mb < T::MB; ++mb)
#pragma unroll
            for (int nb = 0; nb < COL_BLOCKS; ++nb) {
                constexpr int PER = T::MB * COL_BLOCKS / T::stages(T::MB) > 1 ? T::MB * COL_BLOCKS / T::stages(T::MB) : 1;
                if (DEAL && (mb * COL_BLOCKS + nb) % PER == 0 && next < until) load_stage();
                __builtin_amdgcn_sched_barrier(0);  // (results of one block at a time: registers)
                constexpr int GU = GU_AHEAD ? GU_AHEAD : 1;
                const int block = mb * COL_BLOCKS + nb;
                if (!there(w, mb, nb)) {
                    if (OP == kFfnDh && a.o0 && a.split == 1 && block + GU < BLOCKS) load_gu(w, block + GU);
                    continue;
                }
                // (or the places and sums of all blocks are fetched ahead into vector registers, and spilled)
                int l = lane;
                asm volatile("" : "+v"(l));
                asm volatile("" : "+a"(acc[mb][nb]));
                if (GATED) asm volatile("" : "+a"(acc[mb][nb + T::NB / 2]));
                const size_t first = DW ? 0 : (size_t)w.s.begin;
                if (a.split > 1) {  // the sums themselves: 4 columns of a row at a time
#pragma unroll
                    for (int h = 0; h < (GATED ? 2 : 1); ++h) {
                        const f32x16_t &v = acc[mb][nb + h * (GATED ? T::NB / 2 : 0)];
                        const int m = w.row0 + (mb * T::WM + wm) * 32 + (l & 31), n = w.n0 + (wn * COL_BLOCKS + nb) * 32 + (l >> 5) * 4;
                        const size_t row = DW ? ((size_t)w.part * (a.o1 ? 2 : 1) + w.matrix) * a.E * a.M + (size_t)w.s.e * a.M + m
                                              : ((size_t)w.part * (GATED ? 2 : 1) + h) * a.rows + first + m;
#pragma unroll
                        for (int q = 0; q < 4; ++q)
                            if (m < (DW ? a.M : w.s.used) && n + 8 * q < a.N)
                                *(f32x4_t *)(a.part + row * a.N + n + 8 * q) = f32x4_t{v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
                    }
                    continue;
                }
                auto put = [&](auto value, void *to, long long ld) __attribute__((always_inline)) {
                    u32x4_t v[PIECES];
                    pieces_of(value, v);
                    each_piece(w, mb, nb, l, [&](int i, int m, int n) __attribute__((always_inline)) {
                        if (!DW && m >= w.s.used) v[i] = u32x4_t{0, 0, 0, 0};  // (an unused row has the sums of a used one)
                        *(u32x4_t *)((ET *)to + (first + m) * ld + n) = v[i];
                    });
                };
                auto sum = [&](int i) __attribute__((always_inline)) { return acc[mb][nb][i]; };
                if constexpr (OP == kFfnUp) {
                    auto u = [&](int i) __attribute__((always_inline)) { return acc[mb][nb + T::NB / 2][i]; };
                    if (a.o0) put(sum, a.o0, a.ldo), put(u, a.o1, a.ldo);
                    if (a.o2) put([&](int i) __attribute__((always_inline)) { return sum(i) * sigmoid<ET>(sum(i)) * u(i); }, a.o2, a.N);
                } else if constexpr (OP == kFfnDh) {
                    if (a.o2) put(sum, a.o2, a.N);
                    if (!a.o0) continue;
                    const int at = block % GU;
                    float g[16], u[16];
                    values_of(gv[at], g);
                    values_of(uv[at], u);
                    if (block + GU < BLOCKS) load_gu(w, block + GU);
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float s = sigmoid<ET>(g[i]);
                        u[i] = u[i] * (s * (1.f + g[i] * (1.f - s)));
                        g[i] = g[i] * s;
                    }
                    put([&](int i) __attribute__((always_inline)) { return sum(i) * u[i]; }, a.o0, a.ldo);
                    put([&](int i) __attribute__((always_inline)) { return sum(i) * g[i]; }, a.o1, a.ldo);
                } else if constexpr (DW) {
                    put(sum, (ET *)(w.matrix ? a.o1 : a.o0) + (size_t)w.s.e * a.eo, a.ldo);
                } else {
                    put(sum, a.o0, a.N);
                }
            }
        __builtin_amdgcn_sched_barrier(0);
        load_first();
        if constexpr (OP == kFfnDh) {  // (what was fetched and not used is waited for here, not among the next tile's loads)
#pragma unroll
            for (int at = 0; at < GU_AHEAD; ++at)
#pragma unroll
                for (int i = 0; i < PIECES; ++i) asm volatile("" : : "v"(gv[at][i]), "v"(uv[at][i]));
        }
    };

    // The next tile's first stages are on their way while this one's results go out.
    Tile now = tile_at(tile);
    start(now);
    load_first();
    auto clear = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int mb = 0; mb < T::MB; ++mb)
#pragma unroll
            for (int nb = 0; nb < T::NB; ++nb)
#pragma unroll
                for (int v = 0; v < 16; ++v) acc[mb][nb][v] = 0.f;
    };
    while (true) {
        clear();
        if (nk) {
            auto run = [&](auto blocks) __attribute__((always_inline)) { products(blocks, std::integral_constant<bool, SZ == 4>{}); };
            if constexpr (SHORT) {
                if (live == T::MB)
                    run(std::integral_constant<int, T::MB>{});
                else if (live == T::MB / 4 * 3)
                    run(std::integral_constant<int, T::MB / 4 * 3>{});
                else if (live == T::MB / 2)
                    run(std::integral_constant<int, T::MB / 2>{});
                else
                    run(std::integral_constant<int, T::MB / 4>{});
            } else {
                run(std::integral_constant<int, T::MB>{});
            }
            if constexpr (SZ == 4) {  // again on the fp32 instructions where a sum is not finite: numbers or sums may have been scaled out of range
                bool bad = false;
#pragma unroll
                for (int mb = 0; mb < T::MB; ++mb)
#pragma unroll
                    for (int nb = 0; nb < T::NB; ++nb)
#pragma unroll
                        for (int v = 0; v < 16; ++v) bad |= !(fabsf(acc[mb][nb][v]) <= 3.402823466e38f);
                if (__syncthreads_or(bad)) {
                    clear();
                    start(now);
                    load_first();
                    products(std::integral_constant<int, T::MB>{}, std::false_type{});
                }
            }
        }
        else {
            ask();
            __syncthreads();  // (everybody has read the answer before)
            answer();
            __syncthreads();
        }
        if constexpr (OP == kFfnDh) {
            if (a.o0 && a.split == 1) {
#pragma unroll
                for (int i = 0; i < GU_AHEAD; ++i) load_gu(now, i);
            }
        }
        if (a.plan)
            tile = uniform(tables->next);
        else if ((tile += per_list) >= uniform(tables->edge[list + 1]))
            tile = -1;
        const Tile done = now;
        if (tile >= 0) now = tile_at(tile), start(now);
        write_tile(done);
        if (tile < 0) break;
    }
}

template <class T, FfnOp OP>
__global__ __launch_bounds__(kThreads, T::OCC) void k_ffn(FfnArgs a) {
    ffn<T, OP>(a, blockIdx.x, gridDim.x);
}
// A backward call's two products in one launch: workgroups of dw take the CUs that the rows' product leaves, at its end or, where it is small, from
// the start.  us, kernels one after the other / this: fp32 256 x 2 of 8 of 512 x 1024 dg, du and dW2 44 / 36, 1001 x 6 of 48 of
// 1040 x 368 dx, dW1 and dW3 232 / 217;
// bf16 4096 x 8 of 128 of 2048 x 768 458 / 405 and 698 / 672, 16384 x 2 of 8 of 4096 x 14336 13880 / 13600.
template <class T, FfnOp OP, class TDW>
__global__ __launch_bounds__(kThreads, T::OCC) void k_ffn_both(FfnArgs a, FfnArgs dw, u32 first) {
    static_assert(T::OCC == TDW::OCC && T::SMEM == TDW::SMEM, "room");
    if (blockIdx.x < first)
        ffn<T, OP>(a, blockIdx.x, first);
    else
        ffn<TDW, kFfnDw>(dw, blockIdx.x - first, gridDim.x - first);
}

// The outputs of a product whose reduction was cut: the parts' sums added in order, 8 columns a thread.  5.5 us (kernel), most of it the launch.
template <typename ET, FfnOp OP>
__global__ __launch_bounds__(kThreads) void k_ffn_join(FfnArgs a) {
    __shared__ u64 lds[8];
    constexpr bool DW = OP == kFfnDw;
    const int tid = threadIdx.x, cols = a.N / 8;
    int last = 0;  // ragged: the rows that are anybody's
    if (!DW && !a.capacity) {
        u64 all;
        scan_workgroup((u64)(tid < a.E ? min(max(a.counts[tid], 0), a.rows) : 0), lds, &all);
        last = (int)min(all, (u64)a.rows);
    }
    const size_t rows = DW ? (size_t)a.E * a.M : a.rows, mats = DW ? (a.o1 ? 2 : 1) : 1;
    const size_t part = rows * a.N * (OP == kFfnUp ? 2 : mats);
    for (size_t i = (size_t)blockIdx.x * kThreads + tid; i < rows * mats * cols; i += (size_t)gridDim.x * kThreads) {
        const size_t r = i / cols;
        const int n = (int)(i - r * cols) * 8;
        const size_t matrix = r / rows, row = r - matrix * rows;
        bool used = true;
        if (!DW) {
            const int e = a.capacity ? (int)(row / a.capacity) : 0;
            used = a.capacity ? (int)row - e * a.capacity < a.counts[e] : (int)row < last;
        }
        float v[8] = {}, w[8] = {};
        if (used) {
            const float *p = a.part + r * a.N + n;
            for (int s = 0; s < a.split; ++s, p += part) {
                const f32x4_t lo = *(const f32x4_t *)p, hi = *(const f32x4_t *)(p + 4);
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] += lo[j], v[4 + j] += hi[j];
                if (OP == kFfnUp) {
                    const float *q = p + rows * a.N;
                    const f32x4_t lo = *(const f32x4_t *)q, hi = *(const f32x4_t *)(q + 4);
#pragma unroll
                    for (int j = 0; j < 4; ++j) w[j] += lo[j], w[4 + j] += hi[j];
                }
            }
        }
        auto put = [&](void *to, size_t at, const float *x) {
#pragma unroll
            for (int j = 0; j < 8; j += Piece<ET>::N) *(u32x4_t *)((ET *)to + at + j) = Piece<ET>::pack(x + j);
        };
        auto get = [&](const void *from, size_t at, float *x) {
#pragma unroll
            for (int j = 0; j < 8; j += Piece<ET>::N) Piece<ET>::unpack(*(const u32x4_t *)((const ET *)from + at + j), x + j);
        };
        const size_t at = row * a.N + n;
        if (OP == kFfnUp) {
            if (a.o0) put(a.o0, row * a.ldo + n, v), put(a.o1, row * a.ldo + n, w);
            if (a.o2) {
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = v[j] * sigmoid<ET>(v[j]) * w[j];
                put(a.o2, at, v);
            }
        } else if (OP == kFfnDh) {
            if (a.o2) put(a.o2, at, v);
            if (a.o0) {
                float g[8], u[8];
                get(a.g, row * a.ldg + n, g);
                get(a.u, row * a.ldg + n, u);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float s = sigmoid<ET>(g[j]);
                    w[j] = used ? v[j] * (g[j] * s) : 0.f;
                    v[j] = used ? v[j] * (u[j] * (s * (1.f + g[j] * (1.f - s)))) : 0.f;
                }
                put(a.o0, row * a.ldo + n, v);
                put(a.o1, row * a.ldo + n, w);
            }
        } else if (DW) {
            const size_t e = row / a.M;
            put(matrix ? a.o1 : a.o0, e * a.eo + (row - e * a.M) * a.ldo + n, v);
        } else {
            put(a.o0, at, v);
        }
    }
}

}  // namespace moe
