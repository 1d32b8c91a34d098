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
#include "gemm_bf16.hpp"
#include "pieces.hpp"
#include "swiglu8.hpp"

namespace moe {

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

// One operand's stage: R indices x 64 bytes of the reduction (32 steps of bf16, 16 of fp32), R * 64 bytes of LDS.
//   KC:     [R][64 bytes]
//   not KC: [steps][R]
// A load instruction moves 64 x 16 bytes into consecutive LDS, so a lane's place there says which piece of 16 bytes it fetches: pieces are
// placed so that the reads below meet no bank twice.
template <typename ET, int R, bool KC, int WAVES>
struct Operand {
    static constexpr int SZ = sizeof(ET), STEPS = 64 / SZ, BYTES = R * 64;
    static constexpr int INSTR = BYTES / 1024, PER_WAVE = (INSTR + WAVES - 1) / WAVES;
    static constexpr int ROW = KC ? 64 : R * SZ;  // bytes of a row in LDS
    static constexpr int PIECES = ROW / 16, ROWS_PER_INSTR = 64 / PIECES;
    static_assert(KC || SZ * R >= 128, "rows the placement is made for");
    static __device__ __forceinline__ int place(int row, int c) {  // (its own inverse)
        if (KC) return c ^ ((row >> 2) & 3);
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

// MB x NB blocks of 32 x 32 per wavefront, WM x WN wavefronts, NS stages.
template <typename ET_, int MB_, int NB_, int WM_, int WN_, int NS_>
struct FfnTile {
    typedef ET_ ET;
    static constexpr int MB = MB_, NB = NB_, WM = WM_, WN = WN_, NS = NS_, WAVES = WM * WN, THREADS = 64 * WAVES;
    static constexpr int BM = 32 * MB * WM, BN = 32 * NB * WN, STAGE = (BM + BN) * 64;
    // a wavefront's sums on their way out: 32 rows x 64 columns of fp32, two of them (up: g and u)
    static constexpr int OUT_ROW = 64 * 4 + 16, OUT_HALF = 32 * OUT_ROW, OUT = 2 * OUT_HALF;
    static constexpr int HEAD = 256;  // bytes in front of the stages: which rows the workgroup has
    static constexpr int SMEM = HEAD + (NS * STAGE > WAVES * OUT ? NS * STAGE : WAVES * OUT);
    static_assert(NB == 2 || NB == 4, "columns of a wavefront");
};

// Rows that a workgroup has: [begin, begin + used) are expert e's, those up to begin + extent belong to nobody.
struct Segment {
    int e, begin, used, extent, block;
};
struct FfnHead {
    u64 sum[16];
    Segment seg;
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

// Tile number `id` of the launch -> which one of `n` this workgroup takes: workgroups go round the eight XCDs, and each XCD takes a stretch of
// the tiles, whose neighbours read the same operands, from its own L2.
__device__ __forceinline__ int tile_of_xcd(int id, int n) {
    const int each = (n + kTileQueues - 1) / kTileQueues, t = (id % kTileQueues) * each + id / kTileQueues;
    return id / kTileQueues < each && t < n ? t : -1;
}
// Tiles in groups of kTileGroup rows of tiles, column by column inside a group.
constexpr int kTileGroup = 4;
__device__ __forceinline__ void tile_in_groups(int t, int rows, int cols, int *r, int *c) {
    const int group = t / (kTileGroup * cols), in = t - group * kTileGroup * cols, first = group * kTileGroup;
    const int n = min(kTileGroup, rows - first);
    *r = first + in % n, *c = in / n;
}

// The workgroup's row block and column tile; false: none.  Every expert has ceil(rows / BM) row blocks of its own, and the rows of nobody
// (padded: behind an expert's; ragged: behind the last one's) are in row blocks too, whose results are zeros.
template <class T>
__device__ __forceinline__ bool find_rows(const FfnArgs &a, FfnHead *h, Segment *s, int *col) {
    const int tid = threadIdx.x;
    int r;
    if (a.capacity) {
        const int per = (a.capacity + T::BM - 1) / T::BM, t = tile_of_xcd(blockIdx.x, a.E * per * a.nt);
        if (t < 0) return false;
        tile_in_groups(t, a.E * per, a.nt, &r, col);
        s->e = r / per, s->block = r - s->e * per;
        s->begin = s->e * a.capacity, s->extent = a.capacity, s->used = min(max(a.counts[s->e], 0), a.capacity);
        return true;
    }
    // ragged: thread i has expert i
    u64 all, blocks;
    const u64 n = tid < a.E ? (u64)min(max(a.counts[tid], 0), a.rows) : 0;
    const u64 end = scan_workgroup<T::WAVES>(n, h->sum, &all);
    const int last = (int)min(all, (u64)a.rows), begin = (int)min(end - n, (u64)a.rows), used = (int)min(end, (u64)a.rows) - begin;
    const int mine = (used + T::BM - 1) / T::BM;
    const int to = (int)scan_workgroup<T::WAVES>((u64)mine, h->sum + 8, &blocks), rest = (a.rows - last + T::BM - 1) / T::BM;
    const int t = tile_of_xcd(blockIdx.x, ((int)blocks + rest) * a.nt);
    if (t < 0) return false;
    tile_in_groups(t, (int)blocks + rest, a.nt, &r, col);
    if (r >= to - mine && r < to) h->seg = Segment{tid, begin, used, used, r - (to - mine)};
    if (r >= (int)blocks && tid == 0) h->seg = Segment{0, last, 0, a.rows - last, r - (int)blocks};
    __syncthreads();
    *s = h->seg;
    return true;
}

// dw: the workgroup's expert and tile.
template <class T>
__device__ __forceinline__ bool find_matrix(const FfnArgs &a, FfnHead *h, Segment *s, int *row, int *col) {
    const int per = a.mt * a.nt, t = tile_of_xcd(blockIdx.x, a.E * per), tid = threadIdx.x;
    if (t < 0) return false;
    s->e = t / per, s->block = 0;
    tile_in_groups(t - s->e * per, a.mt, a.nt, row, col);
    if (a.capacity) {
        s->begin = s->e * a.capacity, s->extent = s->used = min(max(a.counts[s->e], 0), a.capacity);
        return true;
    }
    u64 before = 0;
    for (int i = tid; i < s->e; i += T::THREADS) before += (u64)max(a.counts[i], 0);
#pragma unroll
    for (int d = 32; d; d >>= 1) before += __shfl_xor(before, d);
    if ((tid & 63) == 0) h->sum[tid >> 6] = before;
    __syncthreads();
    before = 0;
#pragma unroll
    for (int w = 0; w < T::WAVES; ++w) before += h->sum[w];
    s->begin = (int)min(before, (u64)a.rows);
    s->extent = s->used = min(max(a.counts[s->e], 0), a.rows - s->begin);
    return true;
}

// The fragments of N blocks of an operand for step `kk` (32 bytes of the reduction) of a stage: lane l has index l & 31 of a block and the
// steps of its half, l >> 5: 8 of bf16, 4 of fp32.
template <class O, int N>
__device__ __forceinline__ void read_frags(const char *stage, int kk, const int (&at)[N], int lane, u32x4_t (&f)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if constexpr (O::PIECES == 4) {
            const int r = at[i] + (lane & 31);
            f[i] = *(const u32x4_t *)(stage + r * 64 + O::place(r, kk * 2 + (lane >> 5)) * 16);
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

template <typename ET>
__device__ __forceinline__ void store8(void *p, size_t i, const float *v) {
    typedef Piece<ET> P;
#pragma unroll
    for (int j = 0; j < 8; j += P::N) *(u32x4_t *)((ET *)p + i + j) = P::pack(v + j);
}
template <typename ET>
__device__ __forceinline__ void load8(const void *p, size_t i, float *v) {
    typedef Piece<ET> P;
#pragma unroll
    for (int j = 0; j < 8; j += P::N) P::unpack(*(const u32x4_t *)((const ET *)p + i + j), v + j);
}

template <class T, FfnOp OP>
__global__ __launch_bounds__(T::THREADS) void k_ffn(FfnArgs a) {
    typedef typename T::ET ET;
    constexpr bool AK = OP != kFfnDw, BK = OP == kFfnDh || OP == kFfnDx, GATED = OP == kFfnUp;
    typedef Operand<ET, T::BM, AK, T::WAVES> OA;
    typedef Operand<ET, T::BN, BK, T::WAVES> OB;
    constexpr int LPS = OA::PER_WAVE + OB::PER_WAVE, SZ = sizeof(ET), STEPS = OA::STEPS, PIECE = 16 / SZ;
    constexpr int COLS = GATED ? T::BN / 2 : T::BN;  // columns of a matrix per tile
    extern __shared__ __align__(128) char smem[];
    FfnHead *head = (FfnHead *)smem;
    static_assert(sizeof(FfnHead) <= T::HEAD, "head");
    char *stages = smem + T::HEAD;

    Segment s;
    int row0, col;
    if constexpr (OP == kFfnDw) {
        int row;
        if (!find_matrix<T>(a, head, &s, &row, &col)) return;
        row0 = row * T::BM;
    } else {
        if (!find_rows<T>(a, head, &s, &col)) return;
        row0 = s.block * T::BM;
    }
    // dw: column tiles of the second matrix behind those of the first
    const int per_matrix = (a.N + COLS - 1) / COLS;
    const int matrix = OP == kFfnDw ? col / per_matrix : 0;
    const int n0 = (col - matrix * per_matrix) * COLS;
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), wm = wave / T::WN, wn = wave % T::WN;

    f32x16_t acc[T::MB][T::NB];
#pragma unroll
    for (int mb = 0; mb < T::MB; ++mb)
#pragma unroll
        for (int nb = 0; nb < T::NB; ++nb)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[mb][nb][v] = 0.f;

    const int half = a.K / STEPS;  // stages of a pair of operands
    const int nk = OP == kFfnDw ? (s.used + STEPS - 1) / STEPS : row0 >= s.used ? 0 : OP == kFfnDx ? 2 * half : half;
    if (nk) {
        const char *ap[OA::PER_WAVE], *bp[OB::PER_WAVE];
        const size_t lda = (size_t)a.lda * SZ, ldb = (size_t)a.ldb * SZ;
        const char *A = (const char *)a.A0, *B = (const char *)(OP == kFfnDw && matrix ? a.B1 : a.B0);
#pragma unroll
        for (int i = 0; i < OA::PER_WAVE; ++i) {
            const int in = OA::instr(wave, i), r = OA::row_of(in, lane), c = OA::piece_of(in, lane);
            if constexpr (AK) {
                ap[i] = A + (size_t)(s.begin + min(row0 + r, s.used - 1)) * lda + c * 16;
            } else {
                const int m = row0 + c * PIECE;
                ap[i] = A + (size_t)(s.begin + r) * lda + (size_t)(m < a.M ? m : 0) * SZ;
            }
        }
#pragma unroll
        for (int i = 0; i < OB::PER_WAVE; ++i) {
            const int in = OB::instr(wave, i), r = OB::row_of(in, lane), c = OB::piece_of(in, lane);
            if constexpr (BK) {
                bp[i] = B + (size_t)s.e * a.eb * SZ + (size_t)min(n0 + r, a.N - 1) * ldb + c * 16;
            } else {
                int n = c * PIECE;
                const char *from = B;
                if (GATED && n >= COLS) from = (const char *)a.B1, n -= COLS;
                n += n0;
                const size_t first = OP == kFfnDw ? (size_t)s.begin * ldb : (size_t)s.e * a.eb * SZ;
                bp[i] = from + first + (size_t)r * ldb + (size_t)(n < a.N ? n : 0) * SZ;
            }
        }
        const size_t a_step = AK ? 64 : STEPS * lda, b_step = BK ? 64 : STEPS * ldb;
        const u32 lds = lds_offset(stages);
        int next = 0, next_buf = 0;  // the stage to load, and where
        auto load_stage = [&]() {
            const u32 to = lds + next_buf * T::STAGE;
            if (OP == kFfnDx && next == half) {  // on to the second pair
                const long long da = (const char *)a.A1 - (const char *)a.A0 - (long long)half * 64, db = (const char *)a.B1 - (const char *)a.B0 - (long long)half * 64;
#pragma unroll
                for (int i = 0; i < OA::PER_WAVE; ++i) ap[i] += da;
#pragma unroll
                for (int i = 0; i < OB::PER_WAVE; ++i) bp[i] += db;
            }
            const int left = OP == kFfnDw ? s.used - 1 - next * STEPS : STEPS;  // the last row there is
#pragma unroll
            for (int i = 0; i < OA::PER_WAVE; ++i) {
                const int in = OA::instr(wave, i);
                const char *p = ap[i];
                if (OP == kFfnDw) p -= (size_t)max(OA::row_of(in, lane) - left, 0) * lda;
                load_to_lds(p, to + in * 1024);
                ap[i] += a_step;
            }
#pragma unroll
            for (int i = 0; i < OB::PER_WAVE; ++i) {
                const int in = OB::instr(wave, i);
                const char *p = bp[i];
                if (OP == kFfnDw) p -= (size_t)max(OB::row_of(in, lane) - left, 0) * ldb;
                load_to_lds(p, to + OA::BYTES + in * 1024);
                bp[i] += b_step;
            }
            ++next;
            next_buf = next_buf + 1 == T::NS ? 0 : next_buf + 1;
        };
        int a_at[T::MB], b_at[T::NB];
#pragma unroll
        for (int mb = 0; mb < T::MB; ++mb) a_at[mb] = (wm * T::MB + mb) * 32;
#pragma unroll
        for (int nb = 0; nb < T::NB; ++nb)
            b_at[nb] = !GATED ? (wn * T::NB + nb) * 32 : nb < T::NB / 2 ? (wn * T::NB / 2 + nb) * 32 : COLS + (wn * T::NB / 2 + nb - T::NB / 2) * 32;

        for (int i = 0; i < T::NS - 1 && i < nk; ++i) load_stage();
        int buf = 0;
        for (int kt = 0; kt < nk; ++kt) {
            // stage kt has landed when no more loads are in flight than those of the stages behind it
            const int behind = min(nk - 1 - kt, T::NS - 2);
            if (T::NS >= 4 && behind >= 2)
                wait_vmcnt<2 * LPS>();
            else if (T::NS >= 3 && behind >= 1)
                wait_vmcnt<LPS>();
            else
                wait_vmcnt<0>();
            __syncthreads();  // ... and everybody has read the stage that the next load replaces
            if (next < nk) load_stage();
            char *stage = stages + buf * T::STAGE;
            if (OP == kFfnDw && kt == nk - 1 && s.used % STEPS) {
                // the steps past the expert's last row: zeros in both operands, whatever lies there
                const int from = s.used % STEPS;
                for (int i = tid; i < (STEPS - from) * (T::BM * SZ / 16); i += T::THREADS) *(u32x4_t *)(stage + from * T::BM * SZ + i * 16) = u32x4_t{0, 0, 0, 0};
                for (int i = tid; i < (STEPS - from) * (T::BN * SZ / 16); i += T::THREADS)
                    *(u32x4_t *)(stage + OA::BYTES + from * T::BN * SZ + i * 16) = u32x4_t{0, 0, 0, 0};
                __syncthreads();
            }
#pragma unroll
            for (int kk = 0; kk < 2; ++kk) {
                u32x4_t fa[T::MB], fb[T::NB];
                read_frags<OA>(stage, kk, a_at, lane, fa);
                read_frags<OB>(stage + OA::BYTES, kk, b_at, lane, fb);
#pragma unroll
                for (int mb = 0; mb < T::MB; ++mb)
#pragma unroll
                    for (int nb = 0; nb < T::NB; ++nb) multiply<ET>(fb[nb], fa[mb], acc[mb][nb]);
            }
            buf = buf + 1 == T::NS ? 0 : buf + 1;
        }
        __syncthreads();
    }

    // Out through LDS of the wavefront's own: 32 rows x 64 columns of sums at a time (up: 32 or 64 of g, and of u), written as the
    // matrix cores leave them and read as rows, 8 columns a lane.
    char *out = stages + wave * T::OUT;
    constexpr int BLOCKS = GATED ? T::NB / 2 : 2, CHUNKS = GATED ? 1 : T::NB / 2;  // blocks of columns at a time, and how often
    constexpr int LANES = BLOCKS * 4, ROWS = 64 / LANES;
#pragma unroll
    for (int mb = 0; mb < T::MB; ++mb)
#pragma unroll
        for (int ch = 0; ch < CHUNKS; ++ch) {
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
            for (int h = 0; h < (GATED ? 2 : 1); ++h)
#pragma unroll
                for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const f32x16_t &v = acc[mb][GATED ? h * (T::NB / 2) + b : ch * 2 + b];
                        *(f32x4_t *)(out + h * T::OUT_HALF + (lane & 31) * T::OUT_ROW + (b * 32 + q * 8 + (lane >> 5) * 4) * 4) =
                            f32x4_t{v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
                    }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            const int c = (lane % LANES) * 8;
            const int n = n0 + (GATED ? wn * T::NB / 2 * 32 : (wn * T::NB + ch * 2) * 32) + c;
#pragma unroll
            for (int r0 = 0; r0 < 32; r0 += ROWS) {
                const int r = r0 + lane / LANES, m = row0 + (wm * T::MB + mb) * 32 + r;
                if (n >= a.N || m >= (OP == kFfnDw ? a.M : s.extent)) continue;
                const bool used = OP == kFfnDw || m < s.used;
                float v[8], w[8];
                const float *p = (const float *)(out + r * T::OUT_ROW) + c;
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = used ? p[j] : 0.f;  // (an unused row has the sums of a used one)
                const size_t row = (size_t)(s.begin + m), at = row * a.N + n;
                if constexpr (OP == kFfnUp) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) w[j] = used ? p[T::OUT_HALF / 4 + j] : 0.f;
                    if (a.o0) {
                        store8<ET>(a.o0, row * a.ldo + n, v);
                        store8<ET>(a.o1, row * a.ldo + n, w);
                    }
                    if (a.o2) {
#pragma unroll
                        for (int j = 0; j < 8; ++j) v[j] = v[j] * sigmoid<ET>(v[j]) * w[j];
                        store8<ET>(a.o2, at, v);
                    }
                } else if constexpr (OP == kFfnDh) {
                    if (a.o2) store8<ET>(a.o2, at, v);
                    if (a.o0) {
                        float g[8], u[8];
                        load8<ET>(a.g, row * a.ldg + n, g);
                        load8<ET>(a.u, row * a.ldg + n, u);
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            const float sg = sigmoid<ET>(g[j]);
                            w[j] = used ? v[j] * (g[j] * sg) : 0.f;
                            v[j] = used ? v[j] * (u[j] * (sg * (1.f + g[j] * (1.f - sg)))) : 0.f;
                        }
                        store8<ET>(a.o0, row * a.ldo + n, v);
                        store8<ET>(a.o1, row * a.ldo + n, w);
                    }
                } else if constexpr (OP == kFfnDw) {
                    store8<ET>(matrix ? a.o1 : a.o0, (size_t)s.e * a.eo + (size_t)m * a.ldo + n, v);
                } else {
                    store8<ET>(a.o0, at, v);
                }
            }
        }
}

}  // namespace moe
