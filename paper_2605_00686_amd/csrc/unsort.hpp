// Rows sorted by expert back to their tokens, and the gradient of that.  Both move rows and do next to nothing else with them: bound
// by memory, (k + 1) T d elements (forward) and (2 k + 1) T d (backward, k T d of them written).  So a wavefront takes 1 KB of a
// token's row, with all its k rows (up to 8) in flight at once, and lives for one trip to memory: many short wavefronts keep more
// loads in flight than one per token, which also waits for its stores between pieces (4096 x 8 rows of 2048: 46 us, gradient 71).
// Measured, MI355X, bf16, inputs that change from call to call (where the runtime's copy moves 4.7 TB/s): 4096 x 8 rows of 2048 27.1 us =
// 5.6 TB/s, their gradient 55.5 us = 5.2; 16384 x 2 of 4096 with an addend 88.2 us = 6.1; fp32 1001 x 6 of 1040 padded to 256 per expert,
// gradient 16.0 us = 5.0; 16384 x 8 of 64 6.1 us and 7.8; one token's 8 rows of 2048 2.9 us, three trips to memory one behind the other.
#pragma once
#include "pieces.hpp"

namespace moe {

struct UnsortArgs {
    int T, d, k, rows, capacity;  // rows of the sorted order; capacity 0 = ragged
    int parts;                    // forward: groups of lanes per token
    int token_groups, batches;    // backward: workgroups that take tokens, `batches` the slots of one; those behind them clear unused rows
    const void *sorted, *addend, *dout;
    const int32_t *inv_perm, *counts;
    const float *w;  // NULL = ones
    void *out, *drows;
    float *dw;
    int32_t *status;
};

// KB slots of a token, from slot j0 on: their rows (a valid one where there is none, so that no load is conditional), which have one,
// and their weights.
template <int KB>
struct SlotRows {
    int row[KB];
    bool has[KB];
    float w[KB];
    __device__ __forceinline__ void load(const UnsortArgs &a, int t, int j0) {
#pragma unroll
        for (int j = 0; j < KB; ++j) {
            const int s = t * a.k + min(j0 + j, a.k - 1);
            row[j] = a.inv_perm[s];
            w[j] = a.w ? a.w[s] : 1.f;
        }
#pragma unroll
        for (int j = 0; j < KB; ++j) {
            has[j] = (u32)row[j] < (u32)a.rows && j0 + j < a.k;
            if (!has[j]) {
                if (row[j] != -1 && j0 + j < a.k) report(a.status, MOE_ERR_BAD_ROUTING);
                row[j] = 0;
            }
        }
    }
};

// out[t] = addend[t] + sum_j w[t,j] sorted[inv_perm[t*k+j]]: G lanes take U pieces each of a token's row, KB rows in flight.  G < 64:
// rows of at most G pieces, 64 / G tokens per wavefront.  STREAM: rows are read past the caches.
template <typename ET, int KB, int U, int G, bool STREAM>
__global__ __launch_bounds__(kThreads) void k_unsort(UnsortArgs a) {
    using P = Piece<ET>;
    static_assert(U == 1 || G == 64, "");
    const int lane = threadIdx.x & (G - 1), pieces = a.d / P::N;
    const u32 units = (u32)a.T * (u32)a.parts;
    for (u32 unit = blockIdx.x * (kThreads / G) + (G == 64 ? (u32)uniform(threadIdx.x / G) : threadIdx.x / G); unit < units; unit += gridDim.x * (kThreads / G)) {
        const int t = (int)(unit / (u32)a.parts), first = (int)(unit - (u32)t * (u32)a.parts) * (64 * U) + lane;
        float acc[U][P::N] = {};
        u32 c[U];
#pragma unroll
        for (int u = 0; u < U; ++u) c[u] = (u32)min(first + u * 64, pieces - 1);
        if (a.addend) {
#pragma unroll
            for (int u = 0; u < U; ++u) P::unpack(((const u32x4_t *)a.addend)[(size_t)t * pieces + c[u]], acc[u]);
        }
        for (int j0 = 0; j0 < a.k; j0 += KB) {
            SlotRows<KB> s;
            s.load(a, t, j0);
            u32x4_t v[KB][U];
#pragma unroll
            for (int j = 0; j < KB; ++j) {
                const u32x4_t *row = (const u32x4_t *)a.sorted + (size_t)s.row[j] * pieces;
#pragma unroll
                for (int u = 0; u < U; ++u) v[j][u] = STREAM ? load_past(row + c[u]) : row[c[u]];
            }
#pragma unroll
            for (int j = 0; j < KB; ++j)
                if (s.has[j]) {
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        float f[P::N];
                        P::unpack(v[j][u], f);
#pragma unroll
                        for (int i = 0; i < P::N; ++i) acc[u][i] = fmaf(s.w[j], f[i], acc[u][i]);
                    }
                }
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (first + u * 64 < pieces) store_past((u32x4_t *)a.out + (size_t)t * pieces + c[u], P::pack(acc[u]));
    }
}

constexpr int unsort_backward_threads(int lanes) { return lanes > kThreads ? lanes : kThreads; }

// drows[inv_perm[t*k+j]] = w[t,j] dout[t], dw[t,j] = <sorted[inv_perm[t*k+j]], dout[t]>: L lanes take a token (64 and fewer: of one
// wavefront; more: wavefronts of a workgroup), KB rows at a time.  Every piece is read before it is written, by the same lane: drows may
// be the rows.
template <typename ET, int KB, int L, bool STREAM>
__global__ __launch_bounds__(unsort_backward_threads(L)) void k_unsort_backward(UnsortArgs a) {
    using P = Piece<ET>;
    constexpr int NT = unsort_backward_threads(L), G = L < 64 ? L : 64, WT = L / G, TOKENS = NT / L;
    __shared__ float sums[NT / 64][KB];
    const int lane = threadIdx.x & (G - 1), wave = uniform(threadIdx.x >> 6), pieces = a.d / P::N;
    if ((int)blockIdx.x >= a.token_groups) {  // padded layout: the rows behind an expert's used ones become zero
        const int groups = gridDim.x - a.token_groups;
        for (int r = ((int)blockIdx.x - a.token_groups) * (NT / 64) + wave; r < a.rows; r += groups * (NT / 64)) {
            const int e = r / a.capacity;
            if (r - e * a.capacity < a.counts[e]) continue;
            for (int c = threadIdx.x & 63; c < pieces; c += 64) store_past((u32x4_t *)a.drows + (size_t)r * pieces + c, u32x4_t{0, 0, 0, 0});
        }
        return;
    }
    const int step = a.token_groups / a.batches * TOKENS;
    for (int t0 = (int)blockIdx.x / a.batches * TOKENS; t0 < a.T; t0 += step) {
        const int t = t0 + (L < 64 ? (int)threadIdx.x / L : wave / WT);
        for (int j0 = (int)blockIdx.x % a.batches * KB; j0 < a.k; j0 += a.batches * KB) {
            SlotRows<KB> s;
            s.load(a, min(t, a.T - 1), j0);
            float sum[KB] = {};
            if (t < a.T)
                for (int first = (wave % WT) * 64; first < pieces; first += WT * 64) {
                    const int c = min(first + lane, pieces - 1);
                    const bool mine = first + lane < pieces;
                    float g[P::N];
                    const u32x4_t gv = ((const u32x4_t *)a.dout)[(size_t)t * pieces + c];
                    u32x4_t v[KB];
                    if (a.dw) {
#pragma unroll
                        for (int j = 0; j < KB; ++j) {
                            const u32x4_t *at = (const u32x4_t *)a.sorted + (size_t)s.row[j] * pieces + c;
                            v[j] = STREAM ? load_past(at) : *at;
                        }
                    }
                    P::unpack(gv, g);
#pragma unroll
                    for (int j = 0; j < KB; ++j)
                        if (s.has[j]) {
                            if (a.dw && mine) {
                                float f[P::N];
                                P::unpack(v[j], f);
#pragma unroll
                                for (int i = 0; i < P::N; ++i) sum[j] = fmaf(g[i], f[i], sum[j]);
                            }
                            if (a.drows && mine) {
                                float f[P::N];
#pragma unroll
                                for (int i = 0; i < P::N; ++i) f[i] = g[i] * s.w[j];
                                store_past((u32x4_t *)a.drows + (size_t)s.row[j] * pieces + c, P::pack(f));
                            }
                        }
                }
            if (!a.dw) continue;
#pragma unroll
            for (int j = 0; j < KB; ++j)
#pragma unroll
                for (int m = G / 2; m > 0; m >>= 1) sum[j] += __shfl_xor(sum[j], m);
            const int n = min(KB, a.k - j0);
            float mine = 0.f;  // lane j's: the sum of slot j
#pragma unroll
            for (int j = 0; j < KB; ++j) mine = lane == j ? sum[j] : mine;
            if (WT > 1) {
                __syncthreads();
                if (lane < KB) sums[wave][lane] = mine;
                __syncthreads();
                mine = 0.f;
#pragma unroll
                for (int i = 0; i < WT; ++i) mine += sums[wave / WT * WT + i][lane % KB];
            }
            if (wave % WT == 0 && lane < n && t < a.T) a.dw[(size_t)t * a.k + j0 + lane] = mine;
        }
    }
}

}  // namespace moe
