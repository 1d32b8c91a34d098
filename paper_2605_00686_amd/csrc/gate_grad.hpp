// The gradient of the gate: softmax over the chosen logits, x Wg.
//
// With dl[t,j] = w[t,j] (dw[t,j] - sum_i w[t,i] dw[t,i]), token t has k numbers that are not zero among E: both products,
// dx = dl Wg^T and dWg = x^T dl, are taken over those alone, so that what no token chose has no part in it (a dense product would turn a
// zero times an infinity into a NaN of every expert), on the vector ALU in fp32.  A task works on the columns of a chunk: 256
// bytes of a row, 16 lanes with 16 bytes each, four tokens' (or slots') rows per instruction of a wavefront.
#pragma once
#include "pieces.hpp"

namespace moe {

constexpr int kGateGradThreads = 1024, kGateGradWaves = kGateGradThreads / 64;
constexpr int kChunkBytes = 256;       // of a row of x, of dx, and of a column of Wg
constexpr int kGateGradSlots = 2048;   // slots of a block of tokens, at most
constexpr int kGateGradTokens = 256;   // tokens of a block, at most

struct GateGradArgs {
    int T, d, E, k;
    int block;         // tokens of a block: block * k <= kGateGradSlots
    int chunks, dw_chunks;     // of columns; those that dWg's tasks take (one if dbias alone is wanted)
    int dw_parts;      // the tokens of dWg's sums are cut into so many parts, whole blocks each (0: no dWg and no dbias wanted)
    int dx_parts;      // tokens per dx task, likewise (0: no dx wanted)
    int dw_blocks, dx_blocks;  // blocks of a part
    const void *x, *Wg;
    const int32_t *idx;
    const float *w, *dw;
    void *dx;
    float *dWg, *dbias;  // of one part (dw_parts == 1), else the parts' sums in the workspace, part_stride apart
    size_t part_stride;
    int32_t *status;
};

struct GateGradSlot {
    int row;  // dx: the slot's expert, -1 = none; dWg: its token in the block
    float dl;
};

// LDS of a task, in this order (the transposition of a task's end takes the same bytes again)
struct alignas(16) GateGradLds {
    GateGradSlot slot[kGateGradSlots];
    float prod[kGateGradSlots];
    u64 chosen[kMaxExperts][kGateGradTokens / 64];  // dWg: the block's tokens that chose an expert, one bit each
    int first[kMaxExperts + 1];                     // ... and the first of its slots
    int wave_sum[4];
    // behind it: a block's rows of x, or the chunk's columns of Wg by expert
};

// dl of the block's slots: calls `put(i, slot, expert or -1, dl)` for the slots that this thread has, its i-th.
template <typename F>
__device__ __forceinline__ void gate_block_slots(const GateGradArgs &a, GateGradLds *l, int t0, int n, F &&put) {
    constexpr int PER = kGateGradSlots / kGateGradThreads;
    float w[PER], dw[PER];
    int e[PER];
    const int slots = n * a.k;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int s = threadIdx.x + i * kGateGradThreads;
        if (s >= slots) continue;
        const size_t g = (size_t)t0 * a.k + s;
        w[i] = a.w[g], dw[i] = a.dw[g], e[i] = a.idx[g];
        l->prod[s] = w[i] * dw[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int s = threadIdx.x + i * kGateGradThreads;
        if (s >= slots) continue;
        const int from = s / a.k * a.k;
        float mean = 0.f;
        for (int j = 0; j < a.k; ++j) mean += l->prod[from + j];
        if ((u32)e[i] >= (u32)a.E) report(a.status, MOE_ERR_BAD_ROUTING), e[i] = -1;
        put(i, s, e[i], w[i] * (dw[i] - mean));
    }
}

// dx[tokens of a part, columns of a chunk] = sum_j dl Wg[:, e_j]
template <typename ET>
__device__ __forceinline__ void gate_dx_task(const GateGradArgs &a, char *smem, int chunk, int part) {
    using P = Piece<ET>;
    constexpr int COLS = kChunkBytes / (int)sizeof(ET);
    GateGradLds *l = (GateGradLds *)smem;
    char *wt = smem + sizeof(GateGradLds);  // [E][COLS]
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), col0 = chunk * COLS;
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
    const int group = threadIdx.x / 16, l16 = lane & 15, col = col0 + l16 * P::N;
    for (int b = 0; b < a.dx_blocks; ++b) {
        const int t0 = (part * a.dx_blocks + b) * a.block, n = min(a.block, a.T - t0);
        if (n <= 0) break;
        __syncthreads();
        gate_block_slots(a, l, t0, n, [&](int, int s, int e, float dl) { l->slot[s] = GateGradSlot{e, dl}; });
        __syncthreads();
        for (int t = group; t < n; t += kGateGradThreads / 16) {
            float acc[P::N] = {};
            for (int j = 0; j < a.k; ++j) {
                const GateGradSlot s = l->slot[t * a.k + j];
                if (s.row < 0) continue;
                float f[P::N];
                P::unpack(*(const u32x4_t *)(wt + s.row * kChunkBytes + l16 * 16), f);
#pragma unroll
                for (int i = 0; i < P::N; ++i) acc[i] = fmaf(s.dl, f[i], acc[i]);
            }
            if (col < a.d) *(u32x4_t *)((ET *)a.dx + (size_t)(t0 + t) * a.d + col) = P::pack(acc);
        }
    }
}

// A sum over the four groups of 16 lanes, dealt out: of N values per lane, a lane keeps N / 4.  Value i of group 0 .. 3 is then value
// i + N/2 * (upper 32 lanes) + N/4 * (upper 16 of 32).
template <int N>
__device__ __forceinline__ void sum_groups(float *v) {
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v[i]), __float_as_uint(v[i + N / 2]), false, false);
        v[i] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v[i]), __float_as_uint(v[i + N / 4]), false, false);
        v[i] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
}

// dWg[columns of a chunk, :] and dbias over the tokens of a part.  A block's slots are listed by expert (their places counted from bit
// masks, so the order of every sum is that of the tokens); a wavefront takes every 16th expert and keeps its sums in registers from
// block to block.  NE = experts per wavefront, at most.
template <typename ET, int NE>
__device__ __forceinline__ void gate_dw_task(const GateGradArgs &a, char *smem, int chunk, int part) {
    using P = Piece<ET>;
    constexpr int COLS = kChunkBytes / (int)sizeof(ET), KEEP = P::N / 4;
    GateGradLds *l = (GateGradLds *)smem;
    char *tile = smem + sizeof(GateGradLds);  // [tokens][COLS]
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), col0 = chunk * COLS;
    const int l16 = lane & 15, group = lane >> 4, words = (a.block + 63) / 64;
    float acc[NE][KEEP], bias = 0.f;  // (lane n keeps that of the wavefront's n-th expert)
#pragma unroll
    for (int n = 0; n < NE; ++n)
#pragma unroll
        for (int i = 0; i < KEEP; ++i) acc[n][i] = 0.f;
    for (int b = 0; b < a.dw_blocks; ++b) {
        const int t0 = (part * a.dw_blocks + b) * a.block, n_tok = min(a.block, a.T - t0);
        if (n_tok <= 0) break;
        u32x4_t rows[4];
        if (a.x) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int t = min(tid / 16 + i * (kGateGradThreads / 16), n_tok - 1), c = min(col0 + l16 * P::N, a.d - P::N);
                rows[i] = *(const u32x4_t *)((const ET *)a.x + (size_t)(t0 + t) * a.d + c);
            }
        }
        __syncthreads();  // (the block before is done with the LDS)
        for (int i = tid; i < a.E * words; i += kGateGradThreads) l->chosen[i / words][i % words] = 0ull;
        int es[2] = {-1, -1}, ts[2];
        float dls[2];
        gate_block_slots(a, l, t0, n_tok, [&](int i, int s, int e, float dl) {
            es[i] = e, ts[i] = s / a.k, dls[i] = dl;
            if (e >= 0) atomicOr(&l->chosen[e][ts[i] / 64], 1ull << (ts[i] & 63));
        });
        if (a.x) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (const int t = tid / 16 + i * (kGateGradThreads / 16); t < a.block) *(u32x4_t *)(tile + t * kChunkBytes + l16 * 16) = rows[i];
        }
        __syncthreads();
        int count = 0, sum = 0;
        if (tid < kMaxExperts) {
            if (tid < a.E)
                for (int i = 0; i < words; ++i) count += __popcll(l->chosen[tid][i]);
            sum = count;
#pragma unroll
            for (int m = 1; m < 64; m <<= 1) {
                const int v = __shfl_up(sum, m);
                if (lane >= m) sum += v;
            }
            if (lane == 63) l->wave_sum[wave] = sum;
        }
        __syncthreads();
        if (tid < kMaxExperts) {
            for (int i = 0; i < wave; ++i) sum += l->wave_sum[i];
            if (tid < a.E) l->first[tid + 1] = sum;
            if (tid == 0) l->first[0] = 0;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (es[i] >= 0) {
                const int t = ts[i];
                int at = l->first[es[i]] + __popcll(l->chosen[es[i]][t / 64] & ((1ull << (t & 63)) - 1ull));
                for (int m = 0; m < t / 64; ++m) at += __popcll(l->chosen[es[i]][m]);
                l->slot[at] = GateGradSlot{t, dls[i]};
            }
        __syncthreads();
#pragma unroll
        for (int n = 0; n < NE; ++n) {
            const int e = wave + n * kGateGradWaves;
            if (e >= a.E) break;
            const int from = uniform(l->first[e]), cnt = uniform(l->first[e + 1]) - from;
            float v[P::N] = {}, vb = 0.f;
            for (int i = group; i < cnt; i += 4) {
                const GateGradSlot s = l->slot[from + i];
                vb += s.dl;
                if (a.x) {
                    float f[P::N];
                    P::unpack(*(const u32x4_t *)(tile + s.row * kChunkBytes + l16 * 16), f);
#pragma unroll
                    for (int q = 0; q < P::N; ++q) v[q] = fmaf(s.dl, f[q], v[q]);
                }
            }
            sum_groups<P::N>(v);
#pragma unroll
            for (int i = 0; i < KEEP; ++i) acc[n][i] += v[i];
            vb += __shfl_xor(vb, 16);
            vb += __shfl_xor(vb, 32);
            if (lane == n) bias += vb;
            __builtin_amdgcn_sched_barrier(0);  // (or the loops' loads are drawn together, and registers spilled for them)
        }
    }
    float *out = a.dWg ? a.dWg + part * a.part_stride : nullptr, *out_bias = a.dbias ? a.dbias + part * a.part_stride : nullptr;
    if (const int e = wave + lane * kGateGradWaves; out_bias && chunk == 0 && e < a.E) out_bias[e] = bias;
    if (!a.x) return;
    // [COLS][E] in pieces of 32 columns through LDS, so that rows of dWg are stored whole
    float *turn = (float *)smem;
    const int my_col = l16 * P::N + (lane >> 5) * (P::N / 2) + (group & 1) * (P::N / 4), stride = a.E + 1;
    for (int c0 = 0; c0 < COLS && col0 + c0 < a.d; c0 += 32) {
        __syncthreads();
        if (my_col >= c0 && my_col < c0 + 32) {
#pragma unroll
            for (int n = 0; n < NE; ++n)
                if (const int e = wave + n * kGateGradWaves; e < a.E) {
#pragma unroll
                    for (int i = 0; i < KEEP; ++i) turn[(my_col - c0 + i) * stride + e] = acc[n][i];
                }
        }
        __syncthreads();
        const int n_out = min(32, a.d - col0 - c0) * a.E;
        for (int i = tid; i < n_out; i += kGateGradThreads) {
            const int c = i / a.E;
            out[(size_t)(col0 + c0) * a.E + i] = turn[c * stride + i - c * a.E];
        }
    }
}

template <typename ET, int NE>
__global__ __launch_bounds__(kGateGradThreads) void k_gate_grad(GateGradArgs a) {
    extern __shared__ __align__(16) char smem[];
    const int n_dw = a.dw_chunks * a.dw_parts;
    if ((int)blockIdx.x < n_dw)
        gate_dw_task<ET, NE>(a, smem, blockIdx.x % a.dw_chunks, blockIdx.x / a.dw_chunks);
    else
        gate_dx_task<ET>(a, smem, (blockIdx.x - n_dw) % a.chunks, (blockIdx.x - n_dw) / a.chunks);
}

// The parts' sums, added up part by part: n sums each, the first n_w of them dWg's.
static __global__ __launch_bounds__(kThreads) void k_gate_grad_join(const float *parts, size_t stride, int n_parts, size_t from, size_t n_w, size_t n, float *dWg, float *dbias) {
    for (size_t i = from + blockIdx.x * (size_t)kThreads + threadIdx.x; i < n; i += (size_t)gridDim.x * kThreads) {
        float sum = 0.f;
        for (int p = 0; p < n_parts; ++p) sum += parts[p * stride + i];
        if (i < n_w)
            dWg[i] = sum;
        else
            dbias[i - n_w] = sum;
    }
}

}  // namespace moe
