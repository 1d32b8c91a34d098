// The gradient of the gate: softmax over the chosen logits, x Wg.
#pragma once
#include "pieces.hpp"

namespace moe {

struct GateGradArgs {
    int T, d, E, k;
    const void *x, *Wg;
    const int32_t *idx;
    const float *w, *dw;
    void *dx;
    float *dWg, *dbias;
    int32_t *status;
};

// dl[t,j] = w[t,j] (dw[t,j] - sum_i w[t,i] dw[t,i])
__device__ __forceinline__ float gate_mean(const GateGradArgs &a, int t) {
    float m = 0.f;
    for (int j = 0; j < a.k; ++j) m = fmaf(a.w[(size_t)t * a.k + j], a.dw[(size_t)t * a.k + j], m);
    return m;
}

template <typename ET>
__global__ __launch_bounds__(kThreads) void k_gate_dx(GateGradArgs a) {
    using P = Piece<ET>;
    const int pieces = a.d / P::N;
    for (size_t q = blockIdx.x * (size_t)kThreads + threadIdx.x; q < (size_t)a.T * pieces; q += (size_t)gridDim.x * kThreads) {
        const int t = (int)(q / pieces), c = (int)(q - (size_t)t * pieces) * P::N;
        const float m = gate_mean(a, t);
        float acc[P::N] = {};
        for (int j = 0; j < a.k; ++j) {
            const size_t s = (size_t)t * a.k + j;
            const int e = a.idx[s];
            if ((u32)e >= (u32)a.E) {
                report(a.status, MOE_ERR_BAD_ROUTING);
                continue;
            }
            const float dl = a.w[s] * (a.dw[s] - m);
#pragma unroll
            for (int i = 0; i < P::N; ++i) acc[i] = fmaf(dl, Elem<ET>::load((const ET *)a.Wg, (size_t)(c + i) * a.E + e), acc[i]);
        }
        ((u32x4_t *)a.dx)[q] = P::pack(acc);
    }
}

// dWg[:, e] and dbias[e]: a workgroup per expert and 256 columns, over all tokens.
template <typename ET>
__global__ __launch_bounds__(kThreads) void k_gate_dw(GateGradArgs a) {
    __shared__ float dl[kThreads];
    const int e = blockIdx.x, col = blockIdx.y * kThreads + threadIdx.x;
    float acc = 0.f, bias = 0.f;
    for (int t0 = 0; t0 < a.T; t0 += kThreads) {
        const int t = t0 + threadIdx.x;
        float v = 0.f;
        if (t < a.T)
            for (int j = 0; j < a.k; ++j) {
                const size_t s = (size_t)t * a.k + j;
                if ((u32)a.idx[s] >= (u32)a.E) report(a.status, MOE_ERR_BAD_ROUTING);
                if (a.idx[s] == e) v = a.w[s] * (a.dw[s] - gate_mean(a, t));
            }
        __syncthreads();
        dl[threadIdx.x] = v;
        __syncthreads();
        for (int i = 0; i < kThreads; ++i)
            if (const float g = dl[i]; g != 0.f) {
                bias += g;
                if (col < a.d && a.x) acc = fmaf(g, Elem<ET>::load((const ET *)a.x, (size_t)(t0 + i) * a.d + col), acc);
            }
    }
    if (col < a.d && a.dWg) a.dWg[(size_t)col * a.E + e] = acc;
    if (col == 0 && a.dbias) a.dbias[e] = bias;
}

}  // namespace moe
