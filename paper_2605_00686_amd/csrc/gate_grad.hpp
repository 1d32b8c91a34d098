// The gradient of the gate: softmax over the chosen logits, x Wg.
//
// With dl[t,j] = w[t,j] (dw[t,j] - sum_i w[t,i] dw[t,i]), token t has k numbers that are not zero among E.
//
// dx = dl Wg^T is taken over those alone, on the vector ALU: a task keeps a chunk's columns of Wg in LDS, by expert (256 bytes of
// every column), and 16 lanes add up a token's k pieces.  Alone it is bound by memory (4096 x 8 of 128 of 2048 8.4 us, 2048 x 8 of 256 of 7168
// 14.4 us: 34 and 62 MB).
//
// dWg = x^T dl is a product of the matrix cores, with the zeros: one instruction takes 16 tokens x 32 columns x 32 experts.  Listing a
// block's slots by expert and adding up their rows on the vector ALU took 30 us where this takes 17 (the listing is a chain of five
// barriers, and the rows of an expert few).  fp32 numbers are cut into three bf16 numbers that add up to them exactly, and the products
// of the smaller ones are left out: a product is then off by less than 2^-24 of itself, a rounding of fp32, and towards neither side
// (see cut3).  A number of x that is not finite is left out of the dense product, where it would make a NaN of every expert's sum, and
// added for its token's experts alone; an infinite dl makes a NaN of its own expert's sums there, which are then taken again.
// What bounds it: a task's chain per 64 tokens of LDS writes, three barriers and 12 matrix instructions per wavefront, 0.8 us of
// which the matrix cores are busy 0.3, with one task per CU because every part of the tokens costs its sums (d E fp32) a trip to
// memory and back.
// Measured, MI355X, all three gradients, calls in a row (a call by itself, or traced, takes longer): 4096 x 8 of 128 of 2048 20 us,
// 2048 x 8 of 256 of 7168 34 us, 16384 x 2 of 8 of 4096 73 us, fp32 256 x 2 of 8 of 512 7.1 us, 9683 x 3 of 3 of 720 19.8 us, 2048 x 8 of 128
// of 2048 22.5 us; one token's kernel 5.5 us.  More than 128 experts: x is read by each of two groups of them, 65 MB where 33 must be.
#pragma once
#include <type_traits>

#include "pieces.hpp"

namespace moe {

constexpr int kGateGradThreads = 512, kGateGradWaves = kGateGradThreads / 64;
constexpr int kChunkBytes = 256;      // dx: of a row, and of a column of Wg
constexpr int kGateDwCols = 64;       // dWg: columns of a task ...
constexpr int kGateDwExperts = 128;   // ... and experts, at most
constexpr int kGateGradSlots = 1024;  // dx: slots of a block of tokens, at most

struct GateGradArgs {
    int T, d, E, k;
    int dx_chunks;             // dx: chunks of columns
    int block;                 // dx: tokens of a block, of 8, 16 or 32 slots each (the power of two that holds k): kGateGradSlots in all
    int dx_parts, dx_blocks;   // dx: the tokens are cut into so many parts (0: no dx wanted) of so many blocks
    int dw_chunks;             // dWg: chunks of columns (0: not wanted)
    int dw_groups, dw_experts; // ... groups of so many experts (a multiple of 4)
    int dw_parts, dw_tokens;   // dWg and dbias: the tokens are cut into so many parts (0: neither wanted) of so many (a multiple of a reduction block)
    const void *x, *Wg;
    const int32_t *idx;
    const float *w, *dw;
    void *dx;
    float *dWg, *dbias;
    float *parts;              // workspace: the parts' sums, dWg's [d][E] and dbias's [E], part_stride floats apart, if there is more than one part
    size_t part_stride;
    int32_t *status;
};

struct GateGradSlot {
    int at;  // bytes from the first expert's columns of Wg in LDS to those of the slot's, or to zeros
    float dl;
};

// Slots of tokens in registers: G lanes (the power of two from 8 on that holds k) take a token, kGateGradThreads / G tokens a pass.
__device__ __forceinline__ int gate_lanes_log2(int k) { return k <= 8 ? 3 : k <= 16 ? 4 : 5; }
// A sum over the 8, 16 or 32 lanes of a token, in every one of them.
__device__ __forceinline__ float gate_lanes_sum(float v, int log2) {
    auto add = [&](auto ctrl) { v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), decltype(ctrl)::value, 0xf, 0xf, true)); };
    add(std::integral_constant<int, 0xB1>());   // the neighbour,
    add(std::integral_constant<int, 0x4E>());   // the other pair of four,
    add(std::integral_constant<int, 0x141>());  // the other four of eight (mirrored; within four all have the same),
    if (log2 > 3) add(std::integral_constant<int, 0x140>());  // the other eight of sixteen
    if (log2 > 4) v += __shfl_xor(v, 16);
    return v;
}
// The gradient of the logit that one of those lanes has; all of them call it together.
__device__ __forceinline__ float gate_dl(float w, float dw, int log2) { return w * (dw - gate_lanes_sum(w * dw, log2)); }
__device__ __forceinline__ bool finite(float v) { return (__float_as_uint(v) & 0x7f800000u) != 0x7f800000u; }
template <int PER>
struct GateSlots {
    float w[PER], dw[PER];
    int e[PER];
    // tokens t0 .. t0 + n - 1
    __device__ __forceinline__ void load(const GateGradArgs &a, int log2, int t0, int n) {
        const int j = threadIdx.x & ((1 << log2) - 1);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int t = (threadIdx.x + i * kGateGradThreads) >> log2;
            const bool in = t < n && j < a.k;  // (else the first slot of all: no load is conditional)
            const u32 s = in ? (u32)(t0 + t) * (u32)a.k + j : 0u;  // (T k is at most 2^30)
            w[i] = a.w[s], dw[i] = a.dw[s], e[i] = a.idx[s];
            if (!in) w[i] = dw[i] = 0.f;
        }
    }
    // put(i, token, choice, expert or -1, dl) for those of the tokens' slots that this thread has, its i-th
    template <typename F>
    __device__ __forceinline__ void finish(const GateGradArgs &a, int log2, int n, F &&put) {
        const int j = threadIdx.x & ((1 << log2) - 1);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int t = (threadIdx.x + i * kGateGradThreads) >> log2;
            const float dl = gate_dl(w[i], dw[i], log2);
            if (t >= n || j >= a.k) continue;
            if ((u32)e[i] >= (u32)a.E) report(a.status, MOE_ERR_BAD_ROUTING), e[i] = -1;
            put(i, t, j, e[i], dl);
        }
    }
};

// LDS of a dx task; behind it the chunk's columns of Wg by expert, and one of zeros
struct alignas(16) GateDxLds {
    GateGradSlot slot[kGateGradSlots];
};

// dx[tokens of a part, columns of a chunk] = sum_j dl Wg[:, e_j]
template <typename ET>
__device__ __forceinline__ void gate_dx_task(const GateGradArgs &a, char *smem, int chunk, int part) {
    using P = Piece<ET>;
    constexpr int COLS = kChunkBytes / (int)sizeof(ET);
    GateDxLds *l = (GateDxLds *)smem;
    char *wt = smem + sizeof(GateDxLds);  // [E + 1][COLS]
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), col0 = chunk * COLS, log2 = gate_lanes_log2(a.k);
    GateSlots<kGateGradSlots / kGateGradThreads> slots;
    slots.load(a, log2, part * a.dx_blocks * a.block, min(a.block, a.T - part * a.dx_blocks * a.block));
    // the chunk's rows of Wg, by expert: a wavefront takes some experts of all rows, so that its lanes write side by side
    if constexpr (sizeof(ET) == 2) {
        const int i = min(col0 + 2 * lane, a.d - 2);
        const bf16_t *row = (const bf16_t *)a.Wg + (size_t)i * a.E;
        if (a.E % 8 == 0) {
            for (int e = wave * 8; e < a.E; e += kGateGradWaves * 8) {
                const u32x4_t p = *(const u32x4_t *)(row + e), q = *(const u32x4_t *)(row + a.E + e);
#pragma unroll
                for (int n = 0; n < 4; ++n) {
                    *(u32 *)(wt + (e + 2 * n) * kChunkBytes + lane * 4) = (p[n] & 0xffffu) | (q[n] << 16);
                    *(u32 *)(wt + (e + 2 * n + 1) * kChunkBytes + lane * 4) = (p[n] >> 16) | (q[n] & 0xffff0000u);
                }
            }
        } else {
            for (int e = wave; e < a.E; e += kGateGradWaves)
                *(u32 *)(wt + e * kChunkBytes + lane * 4) = (u32)row[e] | ((u32)row[a.E + e] << 16);
        }
    } else {
        const float *row = (const float *)a.Wg + (size_t)min(col0 + lane, a.d - 1) * a.E;
        for (int e = wave; e < a.E; e += kGateGradWaves) *(float *)(wt + e * kChunkBytes + lane * 4) = row[e];
    }
    if (wave == 0) *(u32 *)(wt + a.E * kChunkBytes + lane * 4) = 0u;
    const int group = threadIdx.x / 16, l16 = lane & 15, col = col0 + l16 * P::N;
    const char *my_wt = wt + l16 * 16;
    for (int b = 0; b < a.dx_blocks; ++b) {
        const int t0 = (part * a.dx_blocks + b) * a.block, n = min(a.block, a.T - t0);
        if (n <= 0) break;
        __syncthreads();
        if ((int)(threadIdx.x & ((1 << log2) - 1)) >= a.k) {
#pragma unroll
            for (int i = 0; i < kGateGradSlots / kGateGradThreads; ++i) l->slot[threadIdx.x + i * kGateGradThreads] = GateGradSlot{a.E * kChunkBytes, 0.f};
        }
        slots.finish(a, log2, n, [&](int, int t, int j, int e, float dl) {
            l->slot[(t << log2) + j] = e < 0 ? GateGradSlot{a.E * kChunkBytes, 0.f} : GateGradSlot{e * kChunkBytes, dl};
        });
        __syncthreads();
        slots.load(a, log2, t0 + a.block, b + 1 < a.dx_blocks ? min(a.block, a.T - t0 - a.block) : 0);
        for (int t = group; t < n; t += kGateGradThreads / 16) {
            float acc[P::N] = {};
            const GateGradSlot *mine = l->slot + (t << log2);
            for (int j = 0; j < a.k; j += 4) {  // (four rows at a time, the last ones made up with rows of zeros)
                u32x4_t s[2], v[4];
                s[0] = *(const u32x4_t *)(mine + j), s[1] = *(const u32x4_t *)(mine + j + 2);
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = *(const u32x4_t *)(my_wt + s[i / 2][i % 2 * 2]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float f[P::N];
                    P::unpack(v[i], f);
                    const float dl = __uint_as_float(s[i / 2][i % 2 * 2 + 1]);
#pragma unroll
                    for (int q = 0; q < P::N; ++q) acc[q] = fmaf(dl, f[q], acc[q]);
                }
            }
            if (col < a.d) store_past((u32x4_t *)((ET *)a.dx + (size_t)(t0 + t) * a.d + col), P::pack(acc));
        }
    }
}

// Two finite fp32 numbers as three bf16 numbers each that add up to them exactly, in the halves of b[0], b[1], b[2] (of a number that is
// not finite one is a NaN at least).  Each is the bf16 number nearest to what those before it leave: with 2^e <= |v| < 2^(e+1) the second is
// 2^(e-8) at most and the third, of the 7 bits that are left, 2^(e-17), so the two products of order 3 come to 2^-24 of the whole at
// most, of either sign.  (Cut off instead of rounded they came to 2^-21, always towards zero: 0.7 * 2^-24 of a sum on average, however
// many terms it has.)  Only the first may be rounded past bf16's largest: it stops there.  Bits below 2^-133, bf16's smallest number, are
// lost: a number from 2^-110 on has all of its own.
__device__ __forceinline__ void cut3(float lo, float hi, u32 *b) {
    constexpr float kLargest = 0x1.fep127f;
    b[0] = pack_bf16x2(__builtin_amdgcn_fmed3f(lo, -kLargest, kLargest), __builtin_amdgcn_fmed3f(hi, -kLargest, kLargest));
#pragma unroll
    for (int n = 1; n < 3; ++n) {
        lo -= __uint_as_float(b[n - 1] << 16), hi -= __uint_as_float(b[n - 1] & 0xffff0000u);
        b[n] = pack_bf16x2(lo, hi);
    }
}
// One such number cut off every 8 bits, in the lower halves: where no product is left out (x of bf16) that is exact too, and a shorter
// chain (rounded: 2048 x 8 of 256 of 7168 33.4 -> 34.1 us, 16384 x 2 of 8 of 4096 71.6 -> 73.4).
__device__ __forceinline__ void cut3_off(float v, u32 *b) {
    b[0] = __float_as_uint(v) >> 16;
    const float r = v - __uint_as_float(b[0] << 16);
    b[1] = __float_as_uint(r) >> 16;
    b[2] = __float_as_uint(r - __uint_as_float(b[1] << 16)) >> 16;
}

// What a dWg task meets that is not finite.
struct GateOdd {
    int x_first, x_last;    // first and last token whose x has such a number here
    int sum;                // whether a sum has become a NaN
    int dl_first, dl_last;  // then: first and last token with such a dl here,
    u32 again[kGateDwExperts / 32];  // and a bit for each of the experts with an infinite one
};

// Shape of a dWg task: KT tokens per reduction block; a wavefront has 32 of up to 32 WE experts and all columns, and the 8 / WE
// wavefronts that have the same multiply a share of the block each.  FEW: at most 8 choices.  (What a step reads from LDS bounds it:
// three pieces of dl per block of 32 experts, so every wavefront uses them on 64 columns.)
template <typename ET_, int WE_, int KT_, bool FEW_>
struct GateDwShape {
    using ET = ET_;
    static constexpr int WE = WE_, KT = KT_, SHARES = kGateGradWaves / WE, STEPS = KT / 16 / SHARES, COLS = kGateDwCols, CB = COLS / 32, EPAD = WE * 32;
    static_assert(STEPS * SHARES * 16 == KT && EPAD <= kGateDwExperts, "");
    static constexpr bool FEW = FEW_;
    static constexpr int XP = sizeof(ET) == 4 ? 3 : 1;  // bf16 numbers that make up one of x
    // Rows of LDS.  dl, [3][EPAD][KT] bf16: 16 bytes behind each row, so that 16 lanes' pieces of 16 bytes meet no bank twice; x,
    // [XP][KT][COLS] bf16: rows 16 banks apart modulo 64, for the transposing read of 4 rows x 64 bytes.
    static constexpr int DROW = KT * 2 + 16, XROW = COLS * 2 + 64;
    static constexpr int DPLANE = EPAD * DROW, XPLANE = KT * XROW;
    static constexpr int O_X = 3 * DPLANE, TROW = EPAD + 4, TURN = SHARES * COLS * TROW * 4;
    static constexpr int O_ODD = O_X + XP * XPLANE > TURN ? O_X + XP * XPLANE : TURN, LDS = O_ODD + (int)sizeof(GateOdd);
    static constexpr int SLOT_LANES = KT * (FEW ? 8 : 32), PER = SLOT_LANES < kGateGradThreads ? 1 : SLOT_LANES / kGateGradThreads;  // passes over a block's slots
    static constexpr int GROUP = FEW ? 2 : 1;          // blocks whose numbers are loaded together
    static constexpr int LANES = COLS / Piece<ET>::N;  // of a row of x, a piece each
    static constexpr int NX = KT * LANES / kGateGradThreads, XSTEP = kGateGradThreads / LANES;  // pieces per thread, tokens apart
    static_assert(NX * kGateGradThreads == KT * LANES, "whole pieces per thread");
};

// dWg[columns of a chunk, experts of a group] over the tokens of a part.  For a reduction block of tokens dl
// lies dense in LDS, by expert: its slots are written there, multiplied, and cleared again.
template <class C>
__device__ __forceinline__ void gate_dw_task(const GateGradArgs &a, char *smem, int chunk, int group, int part) {
    using ET = typename C::ET;
    using P = Piece<ET>;
    typedef __attribute__((ext_vector_type(16))) float f32x16_t;
    typedef __attribute__((ext_vector_type(8))) short s16x8_t;
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    const int col0 = chunk * C::COLS, log2 = C::FEW ? 3 : gate_lanes_log2(a.k);
    const int t_begin = part * a.dw_tokens, t_end = min(a.T, t_begin + a.dw_tokens);
    const int e_first = group * a.dw_experts, n_e = min(a.E - e_first, a.dw_experts);
    char *xs = smem + C::O_X;
    GateOdd *odd = (GateOdd *)(smem + C::O_ODD);
    // Loads run a group of blocks ahead, whole groups at a time: a block's tokens are few, and a CU may have one workgroup
    constexpr int GROUP = C::GROUP;
    u32x4_t rows[GROUP][C::NX];
    GateSlots<C::PER> slots[GROUP];
    const int x_tok = tid / C::LANES, x_lane = tid % C::LANES;
    const ET *x = (const ET *)a.x + min(col0 + x_lane * P::N, a.d - P::N);
    // (no load is conditional: the number of loads in flight is then known at every wait)
    auto load_x = [&](u32x4_t(&v)[C::NX], int t0) __attribute__((always_inline)) {
#pragma unroll
        for (int n = 0; n < C::NX; ++n) v[n] = *(const u32x4_t *)(x + (size_t)min(t0 + x_tok + n * C::XSTEP, t_end - 1) * a.d);
    };
    auto load_group = [&](int t0) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < GROUP; ++i) slots[i].load(a, log2, t0 + i * C::KT, min(C::KT, t_end - t0 - i * C::KT));
#pragma unroll
        for (int i = 0; i < GROUP; ++i) load_x(rows[i], t0 + i * C::KT);
    };
    load_group(t_begin);
    for (int i = tid * 16; i < C::O_X; i += kGateGradThreads * 16) *(u32x4_t *)(smem + i) = u32x4_t{0, 0, 0, 0};
    if (tid == 0) *odd = GateOdd{0x7fffffff, -1, 0, 0x7fffffff, -1, {}};
    const int share = wave / C::WE, e0 = wave % C::WE * 32;
    f32x16_t acc[C::CB];
#pragma unroll
    for (int j = 0; j < C::CB; ++j)
#pragma unroll
        for (int q = 0; q < 16; ++q) acc[j][q] = 0.f;
    // A block's numbers on their way from memory to LDS: this thread's piece of x as bf16 numbers, and its slots
    uint2 piece[C::NX][sizeof(ET) == 2 ? 2 : 3];
    int at[C::PER], old[C::PER];  // where its slots lie in dl, -1 = it has none; and those of the block before
    u32 cut[C::PER][3];
#pragma unroll
    for (int i = 0; i < C::PER; ++i) at[i] = old[i] = -1;
    bool bad_id = false;
    u32 odd_bits[C::NX];  // not 0: the piece has a number that is not finite
    // (no branch on a number in here: the compiler deals these instructions out among a multiplication's)
    auto prepare = [&](int t0, u32x4_t(&row)[C::NX], GateSlots<C::PER> &slot) __attribute__((always_inline)) {
#pragma unroll
        for (int m = 0; m < C::NX; ++m) {
            const u32x4_t v = row[m];
            odd_bits[m] = 0u;
            if constexpr (sizeof(ET) == 2) {
#pragma unroll
                for (int q = 0; q < 4; ++q) odd_bits[m] |= ((v[q] & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
                piece[m][0] = uint2{v[0], v[1]}, piece[m][1] = uint2{v[2], v[3]};
            } else {
                float f[4];
                u32 b[2][3];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    odd_bits[m] |= ((v[q] & 0x7f800000u) + 0x00800000u) & 0x80000000u;
                    f[q] = (v[q] & 0x7f800000u) != 0x7f800000u ? __uint_as_float(v[q]) : 0.f;
                }
                cut3(f[0], f[1], b[0]), cut3(f[2], f[3], b[1]);
#pragma unroll
                for (int n = 0; n < 3; ++n) piece[m][n] = uint2{b[0][n], b[1][n]};
            }
        }
        const int j = tid & ((1 << log2) - 1), n_tok = min(C::KT, t_end - t0);
#pragma unroll
        for (int i = 0; i < C::PER; ++i) {
            const int t = (tid + i * kGateGradThreads) >> log2, e = slot.e[i] - e_first;
            const float dl = gate_dl(slot.w[i], slot.dw[i], log2);
            const bool there = t < n_tok && j < a.k;
            bad_id |= there && (u32)slot.e[i] >= (u32)a.E;
            old[i] = at[i];
            at[i] = there && (u32)e < (u32)n_e ? e * C::DROW + t * 2 : -1;
            if constexpr (C::XP == 1)
                cut3_off(dl, cut[i]);
            else
                cut3(dl, 0.f, cut[i]);
        }
    };
    auto multiply = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int n = 0; n < C::STEPS; ++n) {
            const int kk = share * C::STEPS + n;
            bf16x8_t dl[3], xv[C::XP][C::CB];
#pragma unroll
            for (int c = 2; c >= 0; --c)
                dl[c] = __builtin_bit_cast(bf16x8_t, *(const u32x4_t *)(smem + c * C::DPLANE + (e0 + (lane & 31)) * C::DROW + (kk * 16 + 8 * (lane >> 5)) * 2));
#pragma unroll
            for (int c = 0; c < C::XP; ++c)
#pragma unroll
                for (int j = 0; j < C::CB; ++j) {
                    const char *p = xs + c * C::XPLANE + (kk * 16 + 8 * (lane >> 5) + ((lane & 15) >> 2)) * C::XROW + (j * 32 + 16 * ((lane >> 4) & 1) + 4 * (lane & 3)) * 2;
                    const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4_t __attribute__((address_space(3))) *)p);
                    const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4_t __attribute__((address_space(3))) *)(p + 4 * C::XROW));
                    xv[c][j] = __builtin_bit_cast(bf16x8_t, (s16x8_t)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
                }
            // the smallest products first; those of order 3 and 4 are left out (cut3)
#pragma unroll
            for (int order = 2; order >= 0; --order)
#pragma unroll
                for (int c = 0; c < C::XP && c <= order; ++c)
#pragma unroll
                    for (int j = 0; j < C::CB; ++j) acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(dl[order - c], xv[c][j], acc[j], 0, 0, 0);
        }
    };
    // The block at t0, whose numbers are prepared; `after` prepares the next one's, beside the products.
    auto block = [&](int t0, auto after) __attribute__((always_inline)) {
        __syncthreads();  // (the block before is done with the LDS)
#pragma unroll
        for (int i = 0; i < C::PER; ++i)
            if (old[i] >= 0) {
#pragma unroll
                for (int n = 0; n < 3; ++n) *(unsigned short *)(smem + n * C::DPLANE + old[i]) = 0;
            }
#pragma unroll
        for (int m = 0; m < C::NX; ++m) {
            char *to = xs + (x_tok + m * C::XSTEP) * C::XROW;
            if (odd_bits[m]) {
                if constexpr (sizeof(ET) == 2) {
                    u32 *v = (u32 *)piece[m];
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        if ((v[q] & 0x7f80u) == 0x7f80u) v[q] &= 0xffff0000u;
                        if ((v[q] & 0x7f800000u) == 0x7f800000u) v[q] &= 0xffffu;
                    }
                }
                const int t = min(t0 + x_tok + m * C::XSTEP, t_end - 1);
                atomicMin(&odd->x_first, t), atomicMax(&odd->x_last, t);
            }
            if constexpr (sizeof(ET) == 2)
                *(u32x4_t *)(to + x_lane * 16) = u32x4_t{piece[m][0].x, piece[m][0].y, piece[m][1].x, piece[m][1].y};
            else
#pragma unroll
                for (int n = 0; n < 3; ++n) *(uint2 *)(to + n * C::XPLANE + x_lane * 8) = piece[m][n];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < C::PER; ++i)
            if (at[i] >= 0) {
#pragma unroll
                for (int n = 0; n < 3; ++n) *(unsigned short *)(smem + n * C::DPLANE + at[i]) = (unsigned short)cut[i][n];
            }
        __syncthreads();
        if (e0 < n_e) {
            multiply();
            after();
        } else {
            after();
        }
    };
    __syncthreads();  // (`odd` is set)
    for (int t0 = t_begin; t0 < t_end; t0 += GROUP * C::KT) {
        u32x4_t x_now[GROUP][C::NX];
        GateSlots<C::PER> slots_now[GROUP];
#pragma unroll
        for (int i = 0; i < GROUP; ++i) {
            slots_now[i] = slots[i];
#pragma unroll
            for (int n = 0; n < C::NX; ++n) x_now[i][n] = rows[i][n];
        }
        load_group(t0 + GROUP * C::KT);
        prepare(t0, x_now[0], slots_now[0]);
#pragma unroll
        for (int i = 0; i < GROUP; ++i) {
            if (t0 + i * C::KT >= t_end) break;
            block(t0 + i * C::KT, [&]() __attribute__((always_inline)) {
                if (i + 1 < GROUP) prepare(t0 + (i + 1) * C::KT, x_now[(i + 1) % GROUP], slots_now[(i + 1) % GROUP]);
            });
        }
    }
    if (bad_id) report(a.status, MOE_ERR_BAD_ROUTING);
    float *out = a.dw_parts == 1 ? a.dWg : a.parts + part * a.part_stride;
    // A lane has column lane % 32 of a block, and experts 8 q + 4 (lane / 32) .. + 3.  Through LDS, so that memory sees the chunk's rows of
    // dWg, which lie one behind the other, in one piece.
    float *turn = (float *)smem;  // [SHARES][COLS][TROW]
    __syncthreads();
#pragma unroll
    for (int j = 0; j < C::CB; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const f32x16_t &v = acc[j];
            *(f32x4_t *)(turn + (share * C::COLS + j * 32 + (lane & 31)) * C::TROW + e0 + 8 * q + 4 * (lane >> 5)) = f32x4_t{v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
        }
    __syncthreads();
    // (of all experts a chunk's rows are one piece of memory)
    const int step = a.E % 4 == 0 ? 4 : 1, n_out = min(C::COLS, a.d - col0) * n_e;
    float *to = out + (size_t)col0 * a.E + e_first;
    int c = tid * step / n_e, e = tid * step - c * n_e;
    const int dc = kGateGradThreads * step / n_e, de = kGateGradThreads * step - dc * n_e;
    bool odd_sum = false;
    for (int i = tid * step; i < n_out; i += kGateGradThreads * step) {
        const float *from = turn + c * C::TROW + e;
        if (step == 4) {
            f32x4_t sum = *(const f32x4_t *)from;
#pragma unroll
            for (int h = 1; h < C::SHARES; ++h) sum += *(const f32x4_t *)(from + h * C::COLS * C::TROW);
            *(f32x4_t *)(to + (size_t)c * a.E + e) = sum;
#pragma unroll
            for (int q = 0; q < 4; ++q) odd_sum |= sum[q] != sum[q];
        } else {
            float sum = *from;
#pragma unroll
            for (int h = 1; h < C::SHARES; ++h) sum += from[h * C::COLS * C::TROW];
            to[(size_t)c * a.E + e] = sum;
            odd_sum |= sum != sum;
        }
        c += dc, e += de;
        if (e >= n_e) e -= n_e, ++c;
    }
    if (odd_sum) odd->sum = 1;
    sync_stores();
    if (odd->x_last < 0 && !odd->sum) return;
    if (odd->sum) {  // a NaN among the dl, or an infinite one?
        const int pass = kGateGradThreads >> log2;
        int t_first = 0x7fffffff, t_last = -1;
        for (int t0 = t_begin; t0 < t_end; t0 += pass) {
            GateSlots<1> slot;
            slot.load(a, log2, t0, min(pass, t_end - t0));
            const int t = t0 + (tid >> log2), e = slot.e[0] - e_first;
            const float dl = gate_dl(slot.w[0], slot.dw[0], log2);
            if (t >= t_end || (tid & ((1 << log2) - 1)) >= a.k || (u32)e >= (u32)n_e || finite(dl)) continue;
            t_first = min(t_first, t), t_last = t;
            if (dl == dl) atomicOr(&odd->again[e >> 5], 1u << (e & 31));
        }
        if (t_last >= 0) atomicMin(&odd->dl_first, t_first), atomicMax(&odd->dl_last, t_last);
        __syncthreads();
    }
    if (wave > 0) return;
    // A lane has a column, and a token's slots lie across the lanes as above.  The sums of an expert with an infinite dl have nothing
    // finite in them: they start over, from the products that are not finite.
    static_assert(C::COLS == 64 && kGateDwExperts == 128, "a column per lane, four words of experts");
    const int col = min(col0 + lane, a.d - 1), j = lane & ((1 << log2) - 1);
    const bool mine = col0 + lane < a.d, any = (odd->again[0] | odd->again[1] | odd->again[2] | odd->again[3]) != 0u;
    for (int e = 0; any && e < n_e; ++e)
        if (mine && (odd->again[e >> 5] >> (e & 31) & 1u)) out[(size_t)col * a.E + e_first + e] = 0.f;
    const int first = any ? min(odd->x_first, odd->dl_first) : odd->x_first, last = any ? max(odd->x_last, odd->dl_last) : odd->x_last;
    for (int t = first; t <= last; ++t) {
        const float v = Elem<ET>::load((const ET *)a.x, (size_t)t * a.d + col);
        if (!any && !__any(!finite(v))) continue;
        const u32 s = (u32)t * (u32)a.k + min(j, a.k - 1);
        const float dl = gate_dl(j < a.k ? a.w[s] : 0.f, j < a.k ? a.dw[s] : 0.f, log2);
        const int e_mine = a.idx[s] - e_first;
        for (int i = 0; i < a.k; ++i) {
            const int e = __shfl(e_mine, i);
            const float dl_e = __shfl(dl, i);
            if ((u32)e >= (u32)n_e) continue;
            const bool again = odd->again[e >> 5] >> (e & 31) & 1u;
            if (mine && (!finite(v) || (again && !finite(dl_e)))) out[(size_t)col * a.E + e_first + e] += v * dl_e;
        }
    }
}

// dbias over the tokens of a part: the lanes that take a token have sums of their own in LDS, since two tokens may choose the same expert.
__device__ __forceinline__ void gate_bias_task(const GateGradArgs &a, char *smem, int part) {
    const int log2 = gate_lanes_log2(a.k), groups = kGateGradThreads >> log2;
    const int tid = threadIdx.x, group = tid >> log2;
    float *sums = (float *)smem, *mine = sums + group * a.E;  // [groups][E]
    const int t_begin = part * a.dw_tokens, t_end = min(a.T, t_begin + a.dw_tokens);
    for (int i = tid; i < groups * a.E; i += kGateGradThreads) sums[i] = 0.f;
    __syncthreads();
    for (int t0 = t_begin; t0 < t_end; t0 += groups) {
        GateSlots<1> slots;
        slots.load(a, log2, t0, min(groups, t_end - t0));
        slots.finish(a, log2, min(groups, t_end - t0), [&](int, int, int, int e, float dl) {
            if (e >= 0) mine[e] += dl;
        });
    }
    __syncthreads();
    if (tid >= a.E) return;
    float sum = 0.f;
    for (int g = 0; g < groups; ++g) sum += sums[g * a.E + tid];
    (a.dw_parts == 1 ? a.dbias : a.parts + part * a.part_stride + (size_t)a.d * a.E)[tid] = sum;
}

template <class C>
__global__ __launch_bounds__(kGateGradThreads, 4) void k_gate_grad(GateGradArgs a) {
    extern __shared__ __align__(16) char smem[];
    // dWg's tasks, dbias's, then dx's
    const int n_c = a.dw_chunks * a.dw_groups, n_w = n_c * a.dw_parts, n_b = n_w + (a.dbias ? a.dw_parts : 0), task = blockIdx.x;
    if (task < n_w)
        gate_dw_task<C>(a, smem, task % n_c / a.dw_groups, task % a.dw_groups, task / n_c);
    else if (task < n_b)
        gate_bias_task(a, smem, task - n_w);
    else
        gate_dx_task<typename C::ET>(a, smem, (task - n_b) % a.dx_chunks, (task - n_b) / a.dx_chunks);
}

// The parts' sums added up: dWg's d E (a multiple of 4), then dbias's E.  A workgroup takes 64 pieces of 4, every wavefront a quarter
// of the parts of each (one lane after all parts in turn took 7 us for 49 of them, whatever their size).
static __global__ __launch_bounds__(kThreads) void k_gate_grad_join(GateGradArgs a) {
    __shared__ f32x4_t sums[4][64];
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const size_t n = (size_t)a.d * a.E / 4, i = blockIdx.x * (size_t)64 + lane, all = n + (a.E + 3) / 4;
    const bool wanted = i < n ? a.dWg != nullptr : i < all && a.dbias;
    f32x4_t sum = {0.f, 0.f, 0.f, 0.f};
    if (wanted) {
#pragma unroll 4
        for (int p = wave; p < a.dw_parts; p += 4) sum += *(const f32x4_t *)(a.parts + p * a.part_stride + i * 4);
    }
    sums[wave][lane] = sum;
    __syncthreads();
    if (wave > 0 || !wanted) return;
    sum = (sums[0][lane] + sums[1][lane]) + (sums[2][lane] + sums[3][lane]);
    if (i < n)
        *(f32x4_t *)(a.dWg + i * 4) = sum;
    else
        for (int q = 0; q < 4 && (i - n) * 4 + q < (size_t)a.E; ++q) a.dbias[(i - n) * 4 + q] = sum[q];
}

}  // namespace moe
