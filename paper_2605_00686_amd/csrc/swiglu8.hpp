// SwiGLU with its inputs kept in 8 bits, and its gradient from them.
//
// Blocks of 32 values of a row share a power of two: e4m3 has 4 bits of precision wherever its exponent reaches (2^-6 to 448), so
// a block's scale only has to bring its values there, and a power of two does that without a rounding of its own.  A value is
// then off by at most 2^-4 of itself (or 2^-10 of the scale), which is what halving bf16's bytes costs the gradient; sums are not
// concerned.  The largest of a block is found among the lanes that hold it, the conversions are the hardware's scaled ones.
//
// Bound by memory: 2 f elements read, f written and 2 f (1 + 1/32) bytes kept per row; backward f elements and the kept bytes read, 3 f
// elements written.  A lane holds 16 bytes of an input (wider pieces leave half lines per store: fp32 4096 x 1040, gradient, 16.4 us
// with 8 values per lane, 13.2 with 4), two pieces per thread.  Measured, MI355X, bf16, inputs that change from call to call (the
// runtime's copy moves 4.7 TB/s there): 32768 rows of 768 36.2 us = 5.6 TB/s, 8192 of 2048 21.5 us, gradient 25.5; 32768 of 14336 627 us = 6.0
// TB/s, gradient 808 us = 5.9.
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

// A piece of a row (16 bytes; 8 values of bf16, 4 of fp32) is a lane's: a block is 4 or 8 neighbouring lanes.
template <typename ET, bool STREAM>
__device__ __forceinline__ u32x4_t load_piece(const void *p, size_t i) {
    const u32x4_t *at = (const u32x4_t *)((const ET *)p + i);
    return STREAM ? load_past(at) : *at;
}
template <typename ET>
__device__ __forceinline__ void store_piece(void *p, size_t i, const float *v) {
    store_past((u32x4_t *)((ET *)p + i), Piece<ET>::pack(v));
}
// Codes of a piece: as many bytes as it has values
template <int N> struct CodesOf;
template <> struct CodesOf<8> { typedef u64 type; };
template <> struct CodesOf<4> { typedef u32 type; };

// N values as codes; `byte` is the block's scale.  The lanes of a block call it together.
template <int N>
__device__ __forceinline__ typename CodesOf<N>::type encode(const float *v, u32 &byte) {
    typedef __attribute__((ext_vector_type(2))) short s16x2_t;
    u32 most = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const u32 b = __float_as_uint(v[i]) & 0x7fffffffu;
        most = max(most, b < 0x7f800000u ? b : 0u);
    }
    most = max(most, lane_swap<0xB1>(most));  // the neighbour,
    most = max(most, lane_swap<0x4E>(most));  // the other pair of four,
    if (N == 4) most = max(most, lane_swap<0x141>(most));  // the other four of eight
    // most = m 2^a with 1 <= m < 2 (448 = 1.75 * 2^8): 2^(a - 8), or twice that where m > 1.75
    byte = (u32)max((int)(most >> 23) - 8 + ((most & 0x7fffffu) > 0x600000u ? 1 : 0), 0);
    // the conversion takes the exponent of its scale alone, of an fp32 number's bits; it makes a NaN of what is not finite
    const float scale = __uint_as_float(byte << 23);
    u32 c[2] = {0u, 0u};
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
        s16x2_t w = {0, 0};
        w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, v[4 * i], v[4 * i + 1], scale, false);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, v[4 * i + 2], v[4 * i + 3], scale, true);
        c[i] = __builtin_bit_cast(u32, w);
    }
    return (typename CodesOf<N>::type)(N == 8 ? ((u64)c[1] << 32) | c[0] : (u64)c[0]);
}
template <int N>
__device__ __forceinline__ void decode(typename CodesOf<N>::type codes, u32 byte, float *v) {
    const float scale = __uint_as_float(byte << 23);
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
        const u32 c = (u32)((u64)codes >> (32 * i));
        const f32x2_t lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c, scale, false), hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c, scale, true);
        v[4 * i] = lo[0], v[4 * i + 1] = lo[1], v[4 * i + 2] = hi[0], v[4 * i + 3] = hi[1];
    }
}

// 1 / (1 + exp(-g)); the hardware's exponential and reciprocal are within one unit of fp32's last place each.  The reciprocal of a number past
// 2^126 may be zero, as it was from g = -87.3 on, where silu is -88 * 2^-126: the sum is formed 2^24 times smaller, and leaves the
// range no sooner than the sigmoid does.
//
// fp32: within 3 units for every g.  exp(-g) = 2^(n + f) with |f| <= 1/2: f is taken with log2(e) in two parts, since the rounding of
// one product would come to |g| / 2 units.
//
// bf16: the exponent in one rounding, (|g| + 17) / 2 units: 2^-17 where the sigmoid ends, at |g| = 104, and far inside what h and the
// gradients are rounded to.  us, this / fp32's: 1001 x 6 of 1408 padded 17.6 / 20.7, 8192 x 2048 21.5 / 22.3.
template <typename ET>
__device__ __forceinline__ float sigmoid(float g) {
    constexpr float kLog2e = 1.44269502162933349609375f, kRest = 1.92596299e-8f;
    if constexpr (sizeof(ET) == 2) return __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(fmaf(g, -kLog2e, -24.f)) + 0x1p-24f) * 0x1p-24f;
    const float n = __builtin_rintf(__builtin_amdgcn_fmed3f(g * -kLog2e, -300.f, 300.f));
    const float f = fmaf(g, -kRest, fmaf(g, -kLog2e, -n));
    const float e = __builtin_amdgcn_ldexpf(__builtin_amdgcn_exp2f(f), (int)n - 24);
    return __builtin_amdgcn_rcpf(e + 0x1p-24f) * 0x1p-24f;
}

// A workgroup takes U * 256 pieces of the rows, a thread every 256th.  Rows are a whole number of blocks long here, so that the
// lanes of a block are neighbours; pieces past a row's end stay idle.
template <int N, int U>
struct Pieces {
    int row[U], c[U];  // c: first value
    bool in[U];        // whether there is such a piece, in a row that is used
    bool dead[U];      // ... in one that is not
    __device__ __forceinline__ void find(const SwigluArgs &a) {
        const int per_row = (a.f + kScaleBlock - 1) / kScaleBlock * (kScaleBlock / N);
        const u64 q = blockIdx.x * (u64)(U * kThreads);
        const u32 r0 = (u32)(q / (u32)per_row), x = (u32)(q - (u64)r0 * (u32)per_row) + threadIdx.x;
        int r = (int)(r0 + x / (u32)per_row), p = (int)(x % (u32)per_row);
        const int dr = kThreads / per_row, dp = kThreads - dr * per_row;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            row[u] = min(r, a.rows - 1), c[u] = min(p * N, a.f - N);
            const bool there = r < a.rows && p * N < a.f;
            bool used = true;
            if (a.capacity) {
                const int e = row[u] / a.capacity;
                used = row[u] - e * a.capacity < a.counts[e];
            }
            in[u] = there && used, dead[u] = there && !used;
            r += dr, p += dp;
            if (p >= per_row) p -= per_row, ++r;
        }
    }
};
constexpr int kSwigluPieces = 2;  // per thread

template <typename ET, bool STREAM>
__global__ __launch_bounds__(kThreads) void k_swiglu(SwigluArgs a) {
    constexpr int U = kSwigluPieces, N = Piece<ET>::N;
    typedef typename CodesOf<N>::type Codes;
    Pieces<N, U> at;
    at.find(a);
    u32x4_t gr[U], ur[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {  // (no load is conditional: the first row's where there is nothing to read)
        const size_t i = at.in[u] ? (size_t)at.row[u] * a.ld + at.c[u] : 0;
        gr[u] = load_piece<ET, STREAM>(a.g, i), ur[u] = load_piece<ET, STREAM>(a.u, i);
    }
    const int blocks = (a.f + kScaleBlock - 1) / kScaleBlock;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        float g[N], v[N], h[N];
        Piece<ET>::unpack(gr[u], g);
        Piece<ET>::unpack(ur[u], v);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            g[i] = at.in[u] ? g[i] : 0.f, v[i] = at.in[u] ? v[i] : 0.f;
            h[i] = g[i] * sigmoid<ET>(g[i]) * v[i];
        }
        const bool mine = at.in[u] || at.dead[u];
        const size_t row = at.row[u];
        const int c = at.c[u];
        if (mine && a.h) store_piece<ET>(a.h, row * a.f + c, h);
        if (!a.codes) continue;
        u32 sg, su;
        const Codes cg = encode<N>(g, sg), cu = encode<N>(v, su);
        if (!mine) continue;
        store_past((Codes *)(a.codes + row * 2 * a.f + c), cg);
        store_past((Codes *)(a.codes + (row * 2 + 1) * a.f + c), cu);
        if (c % kScaleBlock == 0) {
            a.scales[row * 2 * blocks + c / kScaleBlock] = (uint8_t)sg;
            a.scales[(row * 2 + 1) * blocks + c / kScaleBlock] = (uint8_t)su;
        }
    }
}

template <typename ET, bool STREAM>
__global__ __launch_bounds__(kThreads) void k_swiglu_backward(SwigluArgs a) {
    constexpr int U = kSwigluPieces, N = Piece<ET>::N;
    typedef typename CodesOf<N>::type Codes;
    Pieces<N, U> at;
    at.find(a);
    const int blocks = (a.f + kScaleBlock - 1) / kScaleBlock;
    u32x4_t dr[U];
    Codes cg[U], cu[U];
    u32 sg[U], su[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const size_t row = at.in[u] ? at.row[u] : 0;
        const int c = at.in[u] ? at.c[u] : 0;
        dr[u] = load_piece<ET, STREAM>(a.dh, row * a.f + c);
        const Codes *pg = (const Codes *)(a.codes + row * 2 * a.f + c), *pu = (const Codes *)(a.codes + (row * 2 + 1) * a.f + c);
        cg[u] = STREAM ? load_past(pg) : *pg, cu[u] = STREAM ? load_past(pu) : *pu;
        sg[u] = a.scales[row * 2 * blocks + c / kScaleBlock], su[u] = a.scales[(row * 2 + 1) * blocks + c / kScaleBlock];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (!at.in[u] && !at.dead[u]) continue;
        float g[N], v[N], dh[N], dg[N], du[N], h[N];
        Piece<ET>::unpack(dr[u], dh);
        decode<N>(cg[u], sg[u], g);
        decode<N>(cu[u], su[u], v);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (at.dead[u]) g[i] = v[i] = dh[i] = 0.f;
            const float s = sigmoid<ET>(g[i]), silu = g[i] * s;
            h[i] = silu * v[i];
            du[i] = dh[i] * silu;
            dg[i] = dh[i] * (v[i] * (s * (1.f + g[i] * (1.f - s))));  // (dh u may be past the range where a closed gate's gradient is not)
        }
        const size_t row = at.row[u];
        store_piece<ET>(a.dg, row * a.ld + at.c[u], dg);
        store_piece<ET>(a.du, row * a.ld + at.c[u], du);
        if (a.h) store_piece<ET>(a.h, row * a.f + at.c[u], h);
    }
}

}  // namespace moe
