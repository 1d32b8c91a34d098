// SwiGLU with its inputs kept in 8 bits, and its gradient from them.
//
// Blocks of 32 values of a row share a power of two: e4m3 has 4 bits of precision wherever its exponent reaches (2^-6 to 448), so
// a block's scale only has to bring its values there, and a power of two does that without a rounding of its own.
#pragma once
#include "pieces.hpp"

namespace moe {

struct SwigluArgs {
    int rows, f, capacity;  // capacity 0 = ragged, every row is used
    long long ld;           // elements from one row of g and u (or of their gradients) to the next
    const void *g, *u, *dh;
    const int32_t *counts;
    void *h, *dg, *du;
    uint8_t *codes, *scales;
};

constexpr int kScaleBlock = 32;  // values
constexpr int kLaneValues = 8;   // consecutive values of a row that a lane holds: four lanes per block

template <typename ET>
__device__ __forceinline__ void load8(const void *p, size_t i, float *v) {
    using P = Piece<ET>;
#pragma unroll
    for (int n = 0; n < 8 / P::N; ++n) P::unpack(*(const u32x4_t *)((const ET *)p + i + n * P::N), v + n * P::N);
}
template <typename ET>
__device__ __forceinline__ void store8(void *p, size_t i, const float *v) {
    using P = Piece<ET>;
#pragma unroll
    for (int n = 0; n < 8 / P::N; ++n) *(u32x4_t *)((ET *)p + i + n * P::N) = P::pack(v + n * P::N);
}

// Eight values as codes; `byte` is the block's scale.  The four lanes of a block call it together.
__device__ __forceinline__ uint2 encode8(const float *v, u32 &byte) {
    u32 most = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const u32 b = __float_as_uint(v[i]) & 0x7fffffffu;
        most = max(most, b < 0x7f800000u ? b : 0u);
    }
    most = max(most, quad_swap<0xB1>(most));
    most = max(most, quad_swap<0x4E>(most));
    // most = m 2^a with 1 <= m < 2 (448 = 1.75 * 2^8): 2^(a - 8), or twice that where m > 1.75
    byte = (u32)max((int)(most >> 23) - 8 + ((most & 0x7fffffu) > 0x600000u ? 1 : 0), 0);
    float s[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const bool finite = (__float_as_uint(v[i]) & 0x7fffffffu) < 0x7f800000u;
        s[i] = finite ? ldexpf(v[i], 127 - (int)byte) : __uint_as_float(0x7fc00000u);
    }
    uint2 c = {0u, 0u};
    c.x = (u32)__builtin_amdgcn_cvt_pk_fp8_f32(s[0], s[1], (int)c.x, false);
    c.x = (u32)__builtin_amdgcn_cvt_pk_fp8_f32(s[2], s[3], (int)c.x, true);
    c.y = (u32)__builtin_amdgcn_cvt_pk_fp8_f32(s[4], s[5], (int)c.y, false);
    c.y = (u32)__builtin_amdgcn_cvt_pk_fp8_f32(s[6], s[7], (int)c.y, true);
    return c;
}
__device__ __forceinline__ void decode8(uint2 c, u32 byte, float *v) {
    const f32x2_t p[4] = {__builtin_amdgcn_cvt_pk_f32_fp8((int)c.x, false), __builtin_amdgcn_cvt_pk_f32_fp8((int)c.x, true),
                          __builtin_amdgcn_cvt_pk_f32_fp8((int)c.y, false), __builtin_amdgcn_cvt_pk_f32_fp8((int)c.y, true)};
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = ldexpf(p[i >> 1][i & 1], (int)byte - 127);
}

// 1 / (1 + exp(-g)); the exponential and the reciprocal of the hardware are within 2 units of fp32's last place for the g that
// matter, far inside what the outputs are rounded to or compared at
__device__ __forceinline__ float sigmoid(float g) { return __builtin_amdgcn_rcpf(1.0f + __expf(-g)); }

__device__ __forceinline__ bool row_used(const SwigluArgs &a, int row) {
    if (a.capacity == 0) return true;
    const int e = row / a.capacity;
    return row - e * a.capacity < a.counts[e];
}

template <typename ET>
__global__ __launch_bounds__(kThreads) void k_swiglu(SwigluArgs a) {
    const int blocks = (a.f + kScaleBlock - 1) / kScaleBlock, per_row = blocks * 4;  // (lanes past the end of a row stay idle)
    const size_t total = (size_t)a.rows * per_row, all = (total + kThreads - 1) / kThreads * kThreads;
    for (size_t q = blockIdx.x * (size_t)kThreads + threadIdx.x; q < all; q += (size_t)gridDim.x * kThreads) {
        const int row = (int)min(q / per_row, (size_t)a.rows - 1), piece = (int)(q - (size_t)row * per_row), c = piece * kLaneValues;
        const bool mine = q < total && c < a.f;
        float g[8] = {}, u[8] = {}, h[8];
        if (mine && row_used(a, row)) {
            load8<ET>(a.g, (size_t)row * a.ld + c, g);
            load8<ET>(a.u, (size_t)row * a.ld + c, u);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) h[i] = g[i] * sigmoid(g[i]) * u[i];
        if (mine && a.h) store8<ET>(a.h, (size_t)row * a.f + c, h);
        if (!a.codes) continue;
        u32 sg, su;
        const uint2 cg = encode8(g, sg), cu = encode8(u, su);
        if (!mine) continue;
        *(uint2 *)(a.codes + (size_t)row * 2 * a.f + c) = cg;
        *(uint2 *)(a.codes + ((size_t)row * 2 + 1) * a.f + c) = cu;
        if ((piece & 3) == 0) {
            a.scales[(size_t)row * 2 * blocks + piece / 4] = (uint8_t)sg;
            a.scales[((size_t)row * 2 + 1) * blocks + piece / 4] = (uint8_t)su;
        }
    }
}

template <typename ET>
__global__ __launch_bounds__(kThreads) void k_swiglu_backward(SwigluArgs a) {
    const int blocks = (a.f + kScaleBlock - 1) / kScaleBlock, per_row = a.f / kLaneValues;
    const size_t total = (size_t)a.rows * per_row;
    for (size_t q = blockIdx.x * (size_t)kThreads + threadIdx.x; q < total; q += (size_t)gridDim.x * kThreads) {
        const int row = (int)(q / per_row), piece = (int)(q - (size_t)row * per_row), c = piece * kLaneValues;
        float g[8] = {}, u[8] = {}, dh[8] = {}, dg[8], du[8], h[8];
        if (row_used(a, row)) {
            load8<ET>(a.dh, (size_t)row * a.f + c, dh);
            decode8(*(const uint2 *)(a.codes + (size_t)row * 2 * a.f + c), a.scales[(size_t)row * 2 * blocks + piece / 4], g);
            decode8(*(const uint2 *)(a.codes + ((size_t)row * 2 + 1) * a.f + c), a.scales[((size_t)row * 2 + 1) * blocks + piece / 4], u);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float s = sigmoid(g[i]), silu = g[i] * s;
            h[i] = silu * u[i];
            du[i] = dh[i] * silu;
            dg[i] = dh[i] * u[i] * s * (1.f + g[i] * (1.f - s));
        }
        store8<ET>(a.dg, (size_t)row * a.ld + c, dg);
        store8<ET>(a.du, (size_t)row * a.ld + c, du);
        if (a.h) store8<ET>(a.h, (size_t)row * a.f + c, h);
    }
}

}  // namespace moe
