// The norm of many gradients together, and all of them scaled to a largest norm.
//
//   sum = sum over all tensors and numbers of g^2, in 64 bits;  norm = sqrt(sum);  out = min(1, max_norm / norm) g
//
// A square of an fp32 number is exact in 64 bits and inside its range, so nothing overflows or vanishes before the root.  Bound by memory: every
// number is read for the norm, and read and written for the scaling; the conversions and fused products in 64 bits are a third of what the
// vector ALU could do meanwhile.  Tensors are cut into chunks that the workgroups go through in turn, sums are added in a fixed order.
// 1.2e9 bf16 numbers, calls in a row: norm 396 us (6.1 TB/s), scaling 908 (5.3 TB/s of reads and writes; from the first number on
// instead of from the last one back 923).  120 tensors of 8 to 32768 numbers: kernels of 5 + 2 + 6 us, launches and the latency of one chunk.
#pragma once
#include "pieces.hpp"

namespace moe {

constexpr int kGradTensors = 140;    // per launch: their places are kernel arguments
constexpr int kGradPieces = 8;       // of 16 bytes per thread and chunk
constexpr int kGradGroups = 4096;    // workgroups, at most

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

// 16 bytes of a tensor that starts anywhere.
struct __attribute__((packed)) Unaligned16 {
    u32x4_t v;
};

// f(tensor, whether it is fp32, its first number, how many) for the workgroup's chunks, from the last one on if BACK
template <bool BACK, class F>
__device__ __forceinline__ void for_each_chunk(const GradArgs &a, F f) {
    constexpr u32 kChunk = kThreads * kGradPieces;  // pieces
    const u32 chunks = a.end[a.n - 1];
    for (u32 i = blockIdx.x; i < chunks; i += gridDim.x) {
        const u32 c = BACK ? chunks - 1 - i : i;
        int t = 0, hi = a.n - 1;  // the first tensor that ends behind the chunk
        while (t < hi) {
            const int mid = (t + hi) / 2;
            if (c < a.end[mid])
                hi = mid;
            else
                t = mid + 1;
        }
        const u32 in = c - (t ? a.end[t - 1] : 0);
        const bool f32 = a.f32[t >> 5] >> (t & 31) & 1;
        const long long each = (long long)kChunk * (f32 ? 4 : 8), first = in * each;
        f(t, f32, first, (int)min(a.count[t] - first, each));
    }
}
// The thread's pieces of a chunk of `n` numbers: whole ones in v, zeros where there is none; returns how many numbers the one piece that the
// tensor ends inside has, if it is the thread's (its number in *part).
template <int PER>
__device__ __forceinline__ int load_pieces(const void *p, int n, u32x4_t (&v)[kGradPieces], int *part) {
    int rest = 0;
#pragma unroll
    for (int i = 0; i < kGradPieces; ++i) {
        const int k = (int)threadIdx.x + i * kThreads;
        v[i] = u32x4_t{0, 0, 0, 0};
        if ((k + 1) * PER <= n)
            v[i] = ((const Unaligned16 *)p)[k].v;
        else if (k * PER < n)
            rest = n - k * PER, *part = k;
    }
    return rest;
}

template <typename ET>
__device__ __forceinline__ double square_sum(const u32x4_t &v, double s) {
    float f[Piece<ET>::N];
    Piece<ET>::unpack(v, f);
#pragma unroll
    for (int i = 0; i < Piece<ET>::N; ++i) s = fma((double)f[i], (double)f[i], s);
    return s;
}

template <int THREADS>
__device__ __forceinline__ double sum_workgroup(double v, double *lds) {
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) v += lds[w];
    return v;
}

__global__ __launch_bounds__(kThreads) void k_grad_squares(GradArgs a) {
    __shared__ double lds[kThreads / 64];
    double s = 0;
    for_each_chunk<false>(a, [&](int t, bool f32, long long first, int n) {
        auto chunk = [&](auto zero) {
            typedef decltype(zero) ET;
            constexpr int PER = Piece<ET>::N;
            const ET *p = (const ET *)a.in[t] + first;
            u32x4_t v[kGradPieces];
            int part = 0;
            const int rest = load_pieces<PER>(p, n, v, &part);
#pragma unroll
            for (int i = 0; i < kGradPieces; ++i) s = square_sum<ET>(v[i], s);
            for (int i = 0; i < rest; ++i) {
                const double g = Elem<ET>::load(p, (size_t)part * PER + i);
                s = fma(g, g, s);
            }
        };
        if (f32)
            chunk(0.f);
        else
            chunk(bf16_t{0});
    });
    s = sum_workgroup<kThreads>(s, lds);
    if (threadIdx.x == 0) a.parts[blockIdx.x] = s;
}

constexpr int kGradNormThreads = 1024;
__global__ __launch_bounds__(kGradNormThreads) void k_grad_norm(const double *parts, int n, double *sum, float *norm) {
    __shared__ double lds[kGradNormThreads / 64];
    double s = 0;
    for (int i = threadIdx.x; i < n; i += kGradNormThreads) s += parts[i];
    s = sum_workgroup<kGradNormThreads>(s, lds);
    if (threadIdx.x) return;
    *sum = s;
    if (norm) *norm = (float)sqrt(s);
}

// (a norm that is no number, or none at all, scales nothing)
__device__ __forceinline__ double clip_factor(double sum, float max_norm) {
    const double norm = sqrt(sum);
    return norm > max_norm && norm < __builtin_inf() ? max_norm / norm : 1.0;
}
// One rounding that counts: products in 64 bits for fp32, in 32 for bf16, but for a factor below fp32's normal numbers (a norm past 2^100, say,
// clipped to 10^-8), of which fp32 has a few bits or none where the results are numbers like any other.
struct InFp32 {
    float factor;
    __device__ __forceinline__ float operator()(float g) const { return g * factor; }
};
struct InFp64 {
    double factor;
    __device__ __forceinline__ float operator()(float g) const { return (float)(g * factor); }
};

__global__ __launch_bounds__(kThreads) void k_grad_clip(GradArgs a) {
    const double factor = clip_factor(*a.sum, a.max_norm);
    // (backwards: the norm has left the last numbers in the caches)
    for_each_chunk<true>(a, [&](int t, bool f32, long long first, int n) {
        if (factor == 1.0 && a.in[t] == a.out[t]) return;
        auto chunk = [&](auto zero, auto scaled) {
            typedef decltype(zero) ET;
            constexpr int PER = Piece<ET>::N;
            const ET *p = (const ET *)a.in[t] + first;
            ET *q = (ET *)a.out[t] + first;
            u32x4_t v[kGradPieces];
            int part = 0;
            const int rest = load_pieces<PER>(p, n, v, &part);
            const bool aligned = ((uintptr_t)q & 15) == 0;
#pragma unroll
            for (int i = 0; i < kGradPieces; ++i) {
                const int k = (int)threadIdx.x + i * kThreads;
                if ((k + 1) * PER > n) continue;
                float f[PER];
                Piece<ET>::unpack(v[i], f);
#pragma unroll
                for (int j = 0; j < PER; ++j) f[j] = scaled(f[j]);
                const u32x4_t w = Piece<ET>::pack(f);
                if (aligned)
                    store_past((u32x4_t *)q + k, w);
                else
                    ((Unaligned16 *)q)[k].v = w;
            }
            for (int i = 0; i < rest; ++i) {
                const size_t at = (size_t)part * PER + i;
                const float g = scaled(Elem<ET>::load(p, at));
                if constexpr (sizeof(ET) == 4)
                    q[at] = g;
                else
                    q[at] = (bf16_t)pack_bf16x2(g, 0.f);
            }
        };
        if (f32)
            chunk(0.f, InFp64{factor});
        else if (factor >= 0x1p-126)
            chunk(bf16_t{0}, InFp32{(float)factor});
        else
            chunk(bf16_t{0}, InFp64{factor});
    });
}

}  // namespace moe
