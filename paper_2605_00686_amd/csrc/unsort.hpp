// Rows sorted by expert back to their tokens, and the gradient of that.
#pragma once
#include "pieces.hpp"

namespace moe {

struct UnsortArgs {
    int T, d, k, rows, capacity, E;  // rows of the sorted order; capacity 0 = ragged
    const void *sorted, *addend, *dout;
    const int32_t *inv_perm, *counts;
    const float *w;  // NULL = ones
    void *out, *drows;
    float *dw;
    int32_t *status;
};

// out[t] = addend[t] + sum_j w[t,j] sorted[inv_perm[t*k+j]]: a wavefront per token.
template <typename ET>
__global__ __launch_bounds__(kThreads) void k_unsort(UnsortArgs a) {
    using P = Piece<ET>;
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), pieces = a.d / P::N;
    for (int t = blockIdx.x * 4 + wave; t < a.T; t += gridDim.x * 4) {
        for (int c = lane; c < pieces; c += 64) {
            float acc[P::N], f[P::N];
#pragma unroll
            for (int i = 0; i < P::N; ++i) acc[i] = 0.f;
            if (a.addend) P::unpack(((const u32x4_t *)a.addend)[(size_t)t * pieces + c], acc);
            for (int j = 0; j < a.k; ++j) {
                const int r = row_of_slot(a.inv_perm[t * a.k + j], a.rows, a.status);
                if (r < 0) continue;
                const float w = a.w ? a.w[t * a.k + j] : 1.f;
                P::unpack(((const u32x4_t *)a.sorted)[(size_t)r * pieces + c], f);
#pragma unroll
                for (int i = 0; i < P::N; ++i) acc[i] = fmaf(w, f[i], acc[i]);
            }
            ((u32x4_t *)a.out)[(size_t)t * pieces + c] = P::pack(acc);
        }
    }
}

// drows[inv_perm[t*k+j]] = w[t,j] dout[t], dw[t,j] = <sorted[inv_perm[t*k+j]], dout[t]>: a wavefront per token.
template <typename ET>
__global__ __launch_bounds__(kThreads) void k_unsort_backward(UnsortArgs a) {
    using P = Piece<ET>;
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), pieces = a.d / P::N;
    for (int t = blockIdx.x * 4 + wave; t < a.T; t += gridDim.x * 4)
        for (int j = 0; j < a.k; ++j) {
            const int s = t * a.k + j, r = row_of_slot(a.inv_perm[s], a.rows, a.status);
            const float w = a.w ? a.w[s] : 1.f;
            float sum = 0.f;
            if (r >= 0)
                for (int c = lane; c < pieces; c += 64) {
                    float g[P::N], f[P::N];
                    P::unpack(((const u32x4_t *)a.dout)[(size_t)t * pieces + c], g);
                    if (a.dw) {
                        P::unpack(((const u32x4_t *)a.sorted)[(size_t)r * pieces + c], f);
#pragma unroll
                        for (int i = 0; i < P::N; ++i) sum = fmaf(g[i], f[i], sum);
                    }
                    if (a.drows) {
#pragma unroll
                        for (int i = 0; i < P::N; ++i) g[i] *= w;
                        ((u32x4_t *)a.drows)[(size_t)r * pieces + c] = P::pack(g);
                    }
                }
            if (!a.dw) continue;
#pragma unroll
            for (int m = 32; m > 0; m >>= 1) sum += __shfl_xor(sum, m);
            if (lane == 0) a.dw[s] = sum;
        }
}

// Padded layout: the rows behind an expert's used ones become zero.
static __global__ __launch_bounds__(kThreads) void k_zero_unused(const int32_t *counts, int rows, int capacity, size_t row_bytes, void *out) {
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), pieces = (int)(row_bytes / 16);
    for (int r = blockIdx.x * 4 + wave; r < rows; r += gridDim.x * 4) {
        const int e = r / capacity;
        if (r - e * capacity < counts[e]) continue;
        for (int c = lane; c < pieces; c += 64) ((u32x4_t *)out)[(size_t)r * pieces + c] = u32x4_t{0, 0, 0, 0};
    }
}

}  // namespace moe
