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
#pragma once
#include <type_traits>

#include "gemm_bf16.hpp"
#include "pieces.hpp"
#include "swiglu8.hpp"

namespace moe {

typedef long long i64;

enum FfnOp { kFfnUp, kFfnDown, kFfnDh, kFfnDx, kFfnDw };

struct FfnArgs {
    int E, rows, capacity;
    const int32_t *counts;
    int M, N, K;     // N columns per matrix; K reduction steps per pair of operands; dw: M x N per matrix, reduction over the rows
    int mt, nt;      // column tiles of all matrices; dw: row tiles
    long long lda, ldb, ldo, ldg;  // elements from one row to the next: operands, outputs, g and u
    long long eb, eo;              // elements from one expert's matrix to the next: weights; dw: outputs
    const void *A0, *A1, *B0, *B1;
    const void *g, *u;  // dh: the activation's inputs
    void *o0, *o1, *o2;
};

constexpr int kDwStart = 96;  // rows of reduction that the start and end of a tile of dw cost as much as

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
    static __device__ __forceinline__ int instr(int wave, int i) { return (wave * PER_WAVE + i) % INSTR; }
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
// Where every expert's rows lie, as a workgroup finds out once.
struct FfnTables {
    u64 sum[16];
    int begin[kMaxExperts + 1], used[kMaxExperts];  // begin[E]: behind the last one's (ragged)
    int first[kMaxExperts + 1];  // first row block of an expert, of the rows of nobody behind the last (ragged); dw: rows before, and kDwStart for each expert
    int n_tiles;
};

// MB x NB blocks of 32 x 32 per wavefront, WM x WN wavefronts, stages of KB bytes of the reduction, NS of them.
template <typename ET_, int MB_, int NB_, int WM_, int WN_, int KB_, int NS_>
struct FfnTile {
    typedef ET_ ET;
    static constexpr int MB = MB_, NB = NB_, WM = WM_, WN = WN_, KB = KB_, NS = NS_, WAVES = WM * WN, THREADS = 64 * WAVES;
    static constexpr int BM = 32 * MB * WM, BN = 32 * NB * WN, STAGE = (BM + BN) * KB;
    // a block of a wavefront's sums on its way out, 32 rows x 32 columns of fp32
    static constexpr int OUT_ROW = 32 * 4 + 16, OUT = 32 * OUT_ROW;
    static constexpr int AT_OUT = NS * STAGE, AT_TABLES = AT_OUT + WAVES * OUT;
    static constexpr int SMEM = AT_TABLES + (int)sizeof(FfnTables);
    static_assert(SMEM <= 160 * 1024, "LDS");
};

template <int WAVES>
__device__ __forceinline__ u64 scan_workgroup(u64 v, u64 *lds, u64 *total) {  // inclusive
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
    for (int w = 0; w < WAVES; ++w) {
        if (w < wave) before += lds[w];
        all += lds[w];
    }
    *total = all;
    return v + before;
}

// The tables, by all threads.  Ragged: thread i has expert i.
template <class T, bool DW>
__device__ __forceinline__ void make_tables(const FfnArgs &a, FfnTables *t) {
    const int tid = threadIdx.x;
    const int n = tid < a.E ? max(a.counts[tid], 0) : 0;
    int begin, used, blocks;
    if (a.capacity) {
        begin = tid * a.capacity, used = min(n, a.capacity), blocks = (a.capacity + T::BM - 1) / T::BM;
    } else {
        u64 all;
        const u64 end = scan_workgroup<T::WAVES>((u64)min(n, a.rows), t->sum, &all);
        begin = (int)min(end - min(n, a.rows), (u64)a.rows), used = (int)min(end, (u64)a.rows) - begin, blocks = (used + T::BM - 1) / T::BM;
        if (tid == 0) t->begin[a.E] = (int)min(all, (u64)a.rows);
    }
    if (DW) blocks = used + kDwStart;
    if (tid >= a.E) blocks = 0;
    u64 all;
    const int to = (int)scan_workgroup<T::WAVES>((u64)blocks, t->sum + 8, &all);
    if (tid < a.E) t->begin[tid] = begin, t->used[tid] = used, t->first[tid] = to - blocks;
    if (tid == 0) t->first[a.E] = (int)all;
    __syncthreads();
}
// The last of the E + 1 ascending numbers that is `v` or less (the first one is).
__device__ __forceinline__ int last_up_to(const int *list, int n, int v) {
    int found = 0;
    for (int i = threadIdx.x & 63; i - (int)(threadIdx.x & 63) < n; i += 64) found += __popcll(__ballot(i < n && list[i] <= v));
    return uniform(found) - 1;
}

// Tiles in groups of kTileGroup rows of tiles, column by column inside a group.
constexpr int kTileGroup = 4;
__device__ __forceinline__ void tile_in_groups(int t, int rows, int cols, int *r, int *c) {
    const int group = t / (kTileGroup * cols), in = t - group * kTileGroup * cols, first = group * kTileGroup;
    const int n = min(kTileGroup, rows - first);
    *r = first + in % n, *c = in / n;
}

// Workgroups go round the eight XCDs; each XCD takes a stretch of the tiles, whose neighbours read the same operands, from its own L2: tiles
// [from, to), workgroup number `id` / 8 of the XCD every `step`-th.
struct TileRange {
    int next, to, step;
};
template <bool DW>
__device__ __forceinline__ TileRange tiles_of(const FfnArgs &a, const FfnTables *t, int row_blocks) {
    const int x = blockIdx.x % kTileQueues;
    int edge[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if (DW) {
            // stretches of about the same work: a tile is worth its expert's rows and kDwStart
            const u64 at = (u64)(x + i) * (u32)t->first[a.E];
            const int e = min(last_up_to(t->first, a.E + 1, (int)(at / kTileQueues)), a.E - 1), per = a.mt * a.nt;
            edge[i] = x + i == kTileQueues ? a.E * per : e * per + (int)((at - (u64)kTileQueues * t->first[e]) * per / (u64)(kTileQueues * (t->used[e] + kDwStart)));
        } else {
            edge[i] = (int)((i64)row_blocks * a.nt * (x + i) / kTileQueues);
        }
    }
    return TileRange{edge[0] + (int)(blockIdx.x / kTileQueues), edge[1], (int)(gridDim.x / kTileQueues)};
}

// The fragments of N blocks of an operand for step `kk` (32 bytes of the reduction) of a stage: lane l has index l & 31 of a block and the
// steps of its half, l >> 5: 8 of bf16, 4 of fp32.
template <class O, int N>
__device__ __forceinline__ void read_frags(const char *stage, int kk, const int (&at)[N], int lane, u32x4_t (&f)[N]) {
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
template <typename ET>
__device__ __forceinline__ void multiply(const u32x4_t &b, const u32x4_t &a, f32x16_t &acc) {
    if constexpr (sizeof(ET) == 2) {
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, b), __builtin_bit_cast(bf16x8_t, a), acc, 0, 0, 0);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(b[j]), __uint_as_float(a[j]), acc, 0, 0, 0);
    }
}

template <class T, FfnOp OP>
__global__ __launch_bounds__(T::THREADS) void k_ffn(FfnArgs a) {
    typedef typename T::ET ET;
    constexpr bool DW = OP == kFfnDw, AK = !DW, BK = OP == kFfnDh || OP == kFfnDx, GATED = OP == kFfnUp;
    typedef Operand<ET, T::BM, AK, T::KB, T::WAVES> OA;
    typedef Operand<ET, T::BN, BK, T::KB, T::WAVES> OB;
    constexpr int LPS = OA::PER_WAVE + OB::PER_WAVE, SZ = sizeof(ET), STEPS = OA::STEPS, PIECE = 16 / SZ;
    constexpr int COLS = GATED ? T::BN / 2 : T::BN;  // columns of a matrix per tile
    static_assert(T::THREADS >= kMaxExperts, "a thread per expert");
    static_assert(!GATED || T::NB % 2 == 0, "g and u of the same columns");
    extern __shared__ __align__(128) char smem[];
    char *stages = smem;
    const FfnTables *tables = (const FfnTables *)(smem + T::AT_TABLES);
    make_tables<T, DW>(a, (FfnTables *)tables);
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), wm = wave / T::WN, wn = wave % T::WN;
    const int used_blocks = tables->first[a.E];
    const int row_blocks = uniform(DW || a.capacity ? used_blocks : used_blocks + (a.rows - tables->begin[a.E] + T::BM - 1) / T::BM);
    TileRange range = tiles_of<DW>(a, tables, row_blocks);
    if (range.next >= range.to) return;

    const int half = a.K / STEPS;  // stages of a pair of operands
    const int per_matrix = (a.N + COLS - 1) / COLS;  // dw: column tiles of the second matrix lie behind those of the first
    struct Tile {
        Segment s;
        int row0, n0, matrix, nk;  // first row (of the segment's; dw: of the matrix) and column, stages
    };
    auto tile_at = [&](int t) __attribute__((always_inline)) {
        Tile w;
        int r, c;
        if (DW) {
            const int per = a.mt * a.nt;
            w.s.e = t / per, w.s.block = 0;
            tile_in_groups(t - w.s.e * per, a.mt, a.nt, &r, &c);
            w.s.begin = uniform(tables->begin[w.s.e]), w.s.used = w.s.extent = uniform(tables->used[w.s.e]);
            w.row0 = r * T::BM;
            w.nk = (w.s.used + STEPS - 1) / STEPS;
        } else {
            tile_in_groups(t, row_blocks, a.nt, &r, &c);
            const int e = last_up_to(tables->first, a.E + 1, r);
            w.s.e = e, w.s.block = r - uniform(tables->first[e]);
            w.s.begin = uniform(a.capacity ? e * a.capacity : tables->begin[e]);
            w.s.used = e < a.E ? uniform(tables->used[e]) : 0;
            w.s.extent = a.capacity ? a.capacity : e < a.E ? w.s.used : a.rows - w.s.begin;
            w.row0 = w.s.block * T::BM;
            w.nk = w.row0 >= w.s.used ? 0 : OP == kFfnDx ? 2 * half : half;
        }
        w.matrix = DW ? c / per_matrix : 0;
        w.n0 = (c - w.matrix * per_matrix) * COLS;
        return w;
    };

    // ---- loads.  A lane's places in the operands; they go on from stage to stage.
    const char *ap[OA::PER_WAVE], *bp[OB::PER_WAVE];
    const size_t lda = (size_t)a.lda * SZ, ldb = (size_t)a.ldb * SZ;
    const size_t a_step = AK ? T::KB : STEPS * lda, b_step = BK ? T::KB : STEPS * ldb;
    const u32 lds = lds_offset(stages);
    int next, nk, used;  // the stage to load; stages and rows of the tile that is loaded
    u32 to;              // where it goes
    // before a stage's loads: on to the second pair of operands; rows past the expert's last one are that one again
    auto begin_stage = [&]() __attribute__((always_inline)) {
        if (OP == kFfnDx && next == half) {
            const long long da = (const char *)a.A1 - (const char *)a.A0 - (long long)half * T::KB, db = (const char *)a.B1 - (const char *)a.B0 - (long long)half * T::KB;
#pragma unroll
            for (int i = 0; i < OA::PER_WAVE; ++i) ap[i] += da;
#pragma unroll
            for (int i = 0; i < OB::PER_WAVE; ++i) bp[i] += db;
        }
        if (OP == kFfnDw && next == nk - 1) {
            const int left = used - 1 - next * STEPS;
#pragma unroll
            for (int i = 0; i < OA::PER_WAVE; ++i) ap[i] -= (size_t)max(OA::row_of(OA::instr(wave, i), lane) - left, 0) * lda;
#pragma unroll
            for (int i = 0; i < OB::PER_WAVE; ++i) bp[i] -= (size_t)max(OB::row_of(OB::instr(wave, i), lane) - left, 0) * ldb;
        }
    };
    auto load_one = [&](int i) __attribute__((always_inline)) {
        if (i < OA::PER_WAVE) {
            load_to_lds(ap[i], to + OA::instr(wave, i) * 1024);
            ap[i] += a_step;
        } else {
            const int j = i - OA::PER_WAVE;
            load_to_lds(bp[j], to + OA::BYTES + OB::instr(wave, j) * 1024);
            bp[j] += b_step;
        }
    };
    auto end_stage = [&]() __attribute__((always_inline)) {
        ++next;
        to += T::STAGE;
        if (to == lds + T::NS * T::STAGE) to = lds;
    };
    auto load_stage = [&]() __attribute__((always_inline)) {
        begin_stage();
#pragma unroll
        for (int i = 0; i < LPS; ++i) load_one(i);
        end_stage();
    };
    // The first stages of a tile: nobody may be reading the stages any more.
    auto start = [&](const Tile &w) __attribute__((always_inline)) {
        nk = w.nk, used = w.s.used, next = 0, to = lds;
        if (!nk) return;
        const char *A = (const char *)a.A0, *B = (const char *)(DW && w.matrix ? a.B1 : a.B0);
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
                if (GATED && n >= COLS) from = (const char *)a.B1, n -= COLS;
                n += w.n0;
                const size_t first = DW ? (size_t)w.s.begin * ldb : (size_t)w.s.e * a.eb * SZ;
                bp[i] = from + first + (size_t)r * ldb + (size_t)(n < a.N ? n : 0) * SZ;
            }
        }
        const int ahead = min(nk, T::NS);
        for (int i = 0; i < ahead; ++i) load_stage();
    };

    // ---- products
    f32x16_t acc[T::MB][T::NB];
    int a_at[T::MB], b_at[T::NB];
#pragma unroll
    for (int mb = 0; mb < T::MB; ++mb) a_at[mb] = (wm * T::MB + mb) * 32;
#pragma unroll
    for (int nb = 0; nb < T::NB; ++nb)
        b_at[nb] = !GATED ? (wn * T::NB + nb) * 32 : nb < T::NB / 2 ? (wn * T::NB / 2 + nb) * 32 : COLS + (wn * T::NB / 2 + nb - T::NB / 2) * 32;

    // Fragments are read a step ahead of the products that take them; a stage's buffer is free when everybody has read its last
    // fragments, and the loads of the stage that goes there are dealt out over the steps that follow.
    constexpr int KK = T::KB / 32;  // steps per stage
    static_assert(KK % 2 == 0, "two sets of fragments in turn");
    constexpr int LPK = (LPS + KK - 1) / KK;
    constexpr int NREAD = T::MB * OA::READS + T::NB * OB::READS, NMUL = T::MB * T::NB, NMFMA = NMUL * (SZ == 2 ? 1 : 4);
    struct Frags {
        u32x4_t a[T::MB], b[T::NB];
    };
    Frags f0, f1;
    auto read = [&](const char *stage, int kk, Frags &f) __attribute__((always_inline)) {
        read_frags<OA>(stage, kk, a_at, lane, f.a);
        read_frags<OB>(stage + OA::BYTES, kk, b_at, lane, f.b);
    };
    // products of `cur`, with the reads of `nxt` and, if LOADS, share `part` of a stage's loads in between
    auto step = [&](const char *stage, int kk, Frags &nxt, const Frags &cur, auto loads, int part) __attribute__((always_inline)) {
        constexpr bool LOADS = decltype(loads)::value;
        read(stage, kk, nxt);
#pragma unroll
        for (int mb = 0; mb < T::MB; ++mb)
#pragma unroll
            for (int nb = 0; nb < T::NB; ++nb) {
                const int i = mb * T::NB + nb;
                if (LOADS) {
#pragma unroll
                    for (int j = 0; j < LPK; ++j)
                        if (j * NMUL / LPK == i && part * LPK + j < LPS) load_one(part * LPK + j);
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
        static_assert(T::NS <= 4, "waits");
        if (T::NS >= 4 && behind >= 3)
            wait_vmcnt<3 * LPS>();
        else if (T::NS >= 4 && behind == 2)
            wait_vmcnt<2 * LPS>();
        else if (T::NS >= 3 && behind == 2)
            wait_vmcnt<2 * LPS>();
        else if (behind == 1)
            wait_vmcnt<LPS>();
        else
            wait_vmcnt<0>();
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __syncthreads();
        if (OP == kFfnDw && kt == nk - 1 && used % STEPS) {
            // the steps past the expert's last row: zeros in both operands, whatever lies there
            char *stage = stages + kt % T::NS * T::STAGE;
            const int from = used % STEPS;
            for (int i = tid; i < (STEPS - from) * (T::BM * SZ / 16); i += T::THREADS) *(u32x4_t *)(stage + from * T::BM * SZ + i * 16) = u32x4_t{0, 0, 0, 0};
            for (int i = tid; i < (STEPS - from) * (T::BN * SZ / 16); i += T::THREADS)
                *(u32x4_t *)(stage + OA::BYTES + from * T::BN * SZ + i * 16) = u32x4_t{0, 0, 0, 0};
            __syncthreads();
        }
    };

    // ---- out.  128 bytes of 32 rows (64 columns of bf16, 32 of fp32; less where a wavefront has less) go through LDS of the wavefront's own: the
    // matrix cores leave lane l with row l & 31, columns 8 q + 4 (l >> 5) + 0..3 of a block; memory is reached in pieces of 16 bytes.
    constexpr int COL_BLOCKS = GATED ? T::NB / 2 : T::NB;
    constexpr int GROUP = SZ == 2 && COL_BLOCKS % 2 == 0 ? 2 : 1;  // blocks at a time
    constexpr int LANES = GROUP * 32 / PIECE, ROWS = 64 / LANES;  // lanes per row, rows at a time
    char *out = smem + T::AT_OUT + wave * T::OUT;
    typedef u32x4_t __attribute__((may_alias)) Piece16;
    typedef __attribute__((ext_vector_type(2))) u32 u32x2_t;
    typedef u32x2_t __attribute__((may_alias)) Piece8;
    auto write_tile = [&](const Tile &w) __attribute__((always_inline)) {
        const int rows = DW ? a.M : w.s.extent;
#pragma unroll
        for (int mb = 0; mb < T::MB; ++mb)
#pragma unroll
            for (int gb = 0; gb < COL_BLOCKS; gb += GROUP) {
                __builtin_amdgcn_sched_barrier(0);  // (results of one group at a time: registers)
                const int m0 = w.row0 + (wm * T::MB + mb) * 32, n0 = w.n0 + (wn * COL_BLOCKS + gb) * 32;
                if (n0 >= a.N || m0 >= rows) continue;
                const size_t first = DW ? 0 : (size_t)w.s.begin;
                // (or the places and sums of all groups are fetched ahead into vector registers, and spilled)
                int l = lane;
                asm volatile("" : "+v"(l));
#pragma unroll
                for (int b = 0; b < GROUP; ++b) {
                    asm volatile("" : "+a"(acc[mb][gb + b]));
                    if (GATED) asm volatile("" : "+a"(acc[mb][gb + b + T::NB / 2]));
                }
                const int out_r = l / LANES, out_c = l % LANES * PIECE;
                // f(row of the matrix, column, number of the piece) where there are such elements
                auto each_piece = [&](auto f) __attribute__((always_inline)) {
#pragma unroll
                    for (int i = 0; i < 32 / ROWS; ++i) {
                        const int m = m0 + i * ROWS + out_r, n = n0 + out_c;
                        if (n < a.N && m < rows) f(m, first + m, n, i);
                    }
                };
                auto put = [&](auto value, void *to, long long ld) __attribute__((always_inline)) {  // value(block, register)
                    asm volatile("" ::: "memory");
#pragma unroll
                    for (int b = 0; b < GROUP; ++b)
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            char *p = out + (l & 31) * T::OUT_ROW + (b * 32 + q * 8 + (l >> 5) * 4) * SZ;
                            const float v[4] = {value(b, 4 * q), value(b, 4 * q + 1), value(b, 4 * q + 2), value(b, 4 * q + 3)};
                            if constexpr (SZ == 2)
                                *(Piece8 *)p = u32x2_t{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
                            else
                                *(Piece16 *)p = Piece<float>::pack(v);
                        }
                    asm volatile("" ::: "memory");
                    each_piece([&](int m, size_t row, int n, int i) __attribute__((always_inline)) {
                        u32x4_t v = *(const Piece16 *)(out + (i * ROWS + out_r) * T::OUT_ROW + out_c * SZ);
                        if (!DW && m >= w.s.used) v = u32x4_t{0, 0, 0, 0};  // (an unused row has the sums of a used one)
                        *(Piece16 *)((ET *)to + row * ld + n) = v;
                    });
                };
                if constexpr (OP == kFfnUp) {
                    auto g = [&](int b, int i) __attribute__((always_inline)) { return acc[mb][gb + b][i]; };
                    auto u = [&](int b, int i) __attribute__((always_inline)) { return acc[mb][gb + b + T::NB / 2][i]; };
                    if (a.o0) put(g, a.o0, a.ldo), put(u, a.o1, a.ldo);
                    if (a.o2) put([&](int b, int i) __attribute__((always_inline)) { return g(b, i) * sigmoid<ET>(g(b, i)) * u(b, i); }, a.o2, a.N);
                } else if constexpr (OP == kFfnDh) {
                    auto dh = [&](int b, int i) __attribute__((always_inline)) { return acc[mb][gb + b][i]; };
                    if (a.o2) put(dh, a.o2, a.N);
                    if (!a.o0) continue;
                    u32x4_t gv[32 / ROWS] = {}, uv[32 / ROWS] = {};
                    each_piece([&](int, size_t row, int n, int i) __attribute__((always_inline)) {
                        gv[i] = *(const Piece16 *)((const ET *)a.g + row * a.ldg + n), uv[i] = *(const Piece16 *)((const ET *)a.u + row * a.ldg + n);
                    });
                    float s[GROUP * 16], u[GROUP * 16];
                    auto take = [&](const u32x4_t (&v)[32 / ROWS], float *x) __attribute__((always_inline)) {  // pieces to where the sums are
                        asm volatile("" ::: "memory");
#pragma unroll
                        for (int i = 0; i < 32 / ROWS; ++i) *(Piece16 *)(out + (i * ROWS + out_r) * T::OUT_ROW + out_c * SZ) = v[i];
                        asm volatile("" ::: "memory");
#pragma unroll
                        for (int b = 0; b < GROUP; ++b)
#pragma unroll
                            for (int q = 0; q < 4; ++q) {
                                const char *p = out + (l & 31) * T::OUT_ROW + (b * 32 + q * 8 + (l >> 5) * 4) * SZ;
                                if constexpr (SZ == 2) {
                                    const u32x2_t y = *(const Piece8 *)p;
#pragma unroll
                                    for (int j = 0; j < 4; ++j) x[b * 16 + 4 * q + j] = __uint_as_float(j & 1 ? y[j / 2] & 0xffff0000u : y[j / 2] << 16);
                                } else {
                                    Piece<float>::unpack(*(const Piece16 *)p, x + b * 16 + 4 * q);
                                }
                            }
                    };
                    take(gv, s);
                    take(uv, u);
#pragma unroll
                    for (int i = 0; i < GROUP * 16; ++i) {
                        const float g = s[i], sg = sigmoid<ET>(g);
                        s[i] = g * sg;
                        u[i] = u[i] * (sg * (1.f + g * (1.f - sg)));
                    }
                    put([&](int b, int i) __attribute__((always_inline)) { return dh(b, i) * u[b * 16 + i]; }, a.o0, a.ldo);
                    put([&](int b, int i) __attribute__((always_inline)) { return dh(b, i) * s[b * 16 + i]; }, a.o1, a.ldo);
                } else if constexpr (DW) {
                    put([&](int b, int i) __attribute__((always_inline)) { return acc[mb][gb + b][i]; }, (ET *)(w.matrix ? a.o1 : a.o0) + (size_t)w.s.e * a.eo, a.ldo);
                } else {
                    put([&](int b, int i) __attribute__((always_inline)) { return acc[mb][gb + b][i]; }, a.o0, a.N);
                }
            }
        __builtin_amdgcn_sched_barrier(0);
    };

    // The next tile's first stages are on their way while this one's results go out.
    Tile now = tile_at(range.next);
    start(now);
    while (true) {
#pragma unroll
        for (int mb = 0; mb < T::MB; ++mb)
#pragma unroll
            for (int nb = 0; nb < T::NB; ++nb)
#pragma unroll
                for (int v = 0; v < 16; ++v) acc[mb][nb][v] = 0.f;
        if (nk) {
            landed(0, min(nk, T::NS) - 1);
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
                stage += T::STAGE;
                if (stage == stages + T::NS * T::STAGE) stage = stages;
            };
            read(stage, 0, f0);
            first_steps(std::false_type{});
            int kt = 1;
            for (; kt <= nk - T::NS; ++kt) {  // (T::NS - 2 stages are in flight behind this one)
                landed(kt, T::NS - 2);
                on();
                begin_stage();
                step(stage, 0, f0, f1, std::true_type{}, 0);
                first_steps(std::true_type{});
                end_stage();
            }
            for (; kt < nk; ++kt) {
                landed(kt, min(nk - 1 - kt, T::NS - 2));
                on();
                step(stage, 0, f0, f1, std::false_type{}, 0);
                first_steps(std::false_type{});
            }
#pragma unroll
            for (int mb = 0; mb < T::MB; ++mb)
#pragma unroll
                for (int nb = 0; nb < T::NB; ++nb) multiply<ET>(f1.b[nb], f1.a[mb], acc[mb][nb]);
            __syncthreads();
        }
        range.next += range.step;
        const bool more = range.next < range.to;
        const Tile done = now;
        if (more) now = tile_at(range.next), start(now);
        write_tile(done);
        if (!more) break;
    }
}

}  // namespace moe
