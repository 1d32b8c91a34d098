// The norm of many gradients together, and all of them scaled to a largest norm.
//
//   sum = sum over all tensors and numbers of g^2, in 64 bits;  norm = sqrt(sum);  out = min(1, max_norm / norm) g
//
// A square of an fp32 number is exact in 64 bits and inside its range, so nothing overflows or vanishes before the root.  Bound by memory: every
// number is read for the norm, and read and written for the scaling; the conversions and fused products in 64 bits are a third of what the
// vector ALU could do meanwhile.  Tensors are cut into chunks that the workgroups go through in turn, sums are added in a fixed order.
#pragma once
#include <type_traits>

#include "pieces.hpp"

namespace moe {

constexpr int kGradTensors = 96;     // per launch: their places are kernel arguments
constexpr int kGradPieces = 8;       // of 16 bytes per thread and chunk
constexpr int kGradGroups = 2048;    // workgroups, at most

struct GradArgs {
    int n, f32[(kGradTensors + 31) / 32];  // tensors; a bit each: fp32 (else bf16)
    const void *in[kGradTensors];
    void *out[kGradTensors];
    long long count[kGradTensors];
    u32 end[kGradTensors];  // chunks up to and including the tensor's
    double *parts;
    const double *sum;
    float max_norm;
};
static_assert(sizeof(GradArgs) <= 4096, "kernel arguments");

// Eight or four numbers of a tensor that starts anywhere.
struct __attribute__((packed)) Unaligned16 {
    u32x4_t v;
};

// f(piece of 16 bytes, its numbers there are) for the pieces of the thread in the workgroup's chunks
template <class Whole, class Rest>
__device__ __forceinline__ void for_each_chunk(const GradArgs &a, Whole whole, Rest rest) {
    constexpr u32 kChunk = kThreads * kGradPieces;  // pieces
    const u32 chunks = a.n ? a.end[a.n - 1] : 0;
    int t = 0;
    for (u32 c = blockIdx.x; c < chunks; c += gridDim.x) {
        while (c >= a.end[t]) ++t;
        const u32 in = c - (t ? a.end[t - 1] : 0);
        const bool f32 = a.f32[t >> 5] >> (t & 31) & 1;
        const int per = f32 ? 4 : 8;
        const long long first = (long long)in * kChunk * per, left = a.count[t] - first;
        if (left >= (long long)kChunk * per)
            whole(t, f32, first);
        else
            rest(t, f32, first, (int)left);
    }
}

template <bool F32>
__device__ __forceinline__ double square_sum(const u32x4_t &v, double s) {
    typedef Piece<typename std::conditional<F32, float, bf16_t>::type> P;
    float f[P::N];
    P::unpack(v, f);
#pragma unroll
    for (int i = 0; i < P::N; ++i) s = fma((double)f[i], (double)f[i], s);
    return s;
}
__device__ __forceinline__ float grad_at(const void *p, bool f32, long long i) { return f32 ? ((const float *)p)[i] : bf16_to_f32(((const bf16_t *)p)[i]); }

__device__ __forceinline__ double sum_workgroup(double v, double *lds) {
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) v += lds[w];
    return v;
}

__global__ __launch_bounds__(kThreads) void k_grad_squares(GradArgs a) {
    __shared__ double lds[kThreads / 64];
    double s = 0;
    for_each_chunk(
        a,
        [&](int t, bool f32, long long first) {
            const Unaligned16 *p = (const Unaligned16 *)((const char *)a.in[t] + first * (f32 ? 4 : 2)) + threadIdx.x;
            u32x4_t v[kGradPieces];
#pragma unroll
            for (int i = 0; i < kGradPieces; ++i) v[i] = p[i * kThreads].v;
#pragma unroll
            for (int i = 0; i < kGradPieces; ++i) s = f32 ? square_sum<true>(v[i], s) : square_sum<false>(v[i], s);
        },
        [&](int t, bool f32, long long first, int left) {
            for (int i = threadIdx.x; i < left; i += kThreads) {
                const double g = grad_at(a.in[t], f32, first + i);
                s = fma(g, g, s);
            }
        });
    s = sum_workgroup(s, lds);
    if (threadIdx.x == 0) a.parts[blockIdx.x] = s;
}

__global__ __launch_bounds__(kThreads) void k_grad_norm(const double *parts, int n, double *sum, float *norm) {
    __shared__ double lds[kThreads / 64];
    double s = 0;
    for (int i = threadIdx.x; i < n; i += kThreads) s += parts[i];
    s = sum_workgroup(s, lds);
    if (threadIdx.x) return;
    *sum = s;
    if (norm) *norm = (float)sqrt(s);
}

// (a norm that is no number, or none at all, scales nothing)
__device__ __forceinline__ double clip_factor(double sum, float max_norm) {
    const double norm = sqrt(sum);
    return norm > max_norm && norm < __builtin_inf() ? max_norm / norm : 1.0;
}
// fp32 in 64 bits and bf16 in 32: one rounding that counts
template <bool F32>
__device__ __forceinline__ u32x4_t scaled(const u32x4_t &v, double factor) {
    typedef Piece<typename std::conditional<F32, float, bf16_t>::type> P;
    float f[P::N];
    P::unpack(v, f);
#pragma unroll
    for (int i = 0; i < P::N; ++i) f[i] = F32 ? (float)(f[i] * factor) : f[i] * (float)factor;
    return P::pack(f);
}

__global__ __launch_bounds__(kThreads) void k_grad_clip(GradArgs a) {
    const double factor = clip_factor(*a.sum, a.max_norm);
    for_each_chunk(
        a,
        [&](int t, bool f32, long long first) {
            if (factor == 1.0 && a.in[t] == a.out[t]) return;
            const Unaligned16 *p = (const Unaligned16 *)((const char *)a.in[t] + first * (f32 ? 4 : 2)) + threadIdx.x;
            Unaligned16 *q = (Unaligned16 *)((char *)a.out[t] + first * (f32 ? 4 : 2)) + threadIdx.x;
            u32x4_t v[kGradPieces];
#pragma unroll
            for (int i = 0; i < kGradPieces; ++i) v[i] = p[i * kThreads].v;
#pragma unroll
            for (int i = 0; i < kGradPieces; ++i) q[i * kThreads].v = f32 ? scaled<true>(v[i], factor) : scaled<false>(v[i], factor);
        },
        [&](int t, bool f32, long long first, int left) {
            if (factor == 1.0 && a.in[t] == a.out[t]) return;
            for (int i = threadIdx.x; i < left; i += kThreads) {
                const float g = grad_at(a.in[t], f32, first + i);
                if (f32)
                    ((float *)a.out[t])[first + i] = (float)(g * factor);
                else
                    ((bf16_t *)a.out[t])[first + i] = (bf16_t)pack_bf16x2(g * (float)factor, 0.f);
            }
        });
}

}  // namespace moe
