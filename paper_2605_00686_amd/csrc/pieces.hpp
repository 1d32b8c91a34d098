// Rows in pieces of 16 bytes, as the training calls move them.  gfx950 only.
#pragma once
#include "common.hpp"

namespace moe {

template <typename ET> struct Piece;
template <> struct Piece<float> {
    static constexpr int N = 4;
    static __device__ __forceinline__ void unpack(const u32x4_t &v, float *f) {
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(v[i]);
    }
    static __device__ __forceinline__ u32x4_t pack(const float *f) {
        return u32x4_t{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
    }
};
template <> struct Piece<bf16_t> {
    static constexpr int N = 8;
    static __device__ __forceinline__ void unpack(const u32x4_t &v, float *f) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(v[i] << 16);
            f[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ u32x4_t pack(const float *f) {
        return u32x4_t{pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7])};
    }
};

// Stores of results go past the caches (whoever reads them next finds them in memory; what the caches hold instead is the rows that are
// read), and so do loads where a call reads more than they hold anyway.  us, loads and stores cached / stores past / both: 4096 x 8 rows
// of 2048 (134 MB) 33.0 / 30.9 / 27.2, their gradient 60.5 / 59.1 / 55.3; 8192 x 16 of 320 (84 MB) 18.2 / 17.3 / 19.5, 16384 x 4 of 256
// (34 MB) 9.5 / 9.5 / 11.4: from kStreamBytes on.
constexpr size_t kStreamBytes = (size_t)96 << 20;
template <typename T>
__device__ __forceinline__ void store_past(T *p, T v) {
    __builtin_nontemporal_store(v, p);
}
template <typename T>
__device__ __forceinline__ T load_past(const T *p) {
    return __builtin_nontemporal_load(p);
}

// A lane's value from another of its row of 16, without a trip through LDS: the lane whose number differs in bit 0 (0xB1) or bit 1
// (0x4E), or the mirrored one of 8 (0x141).
template <int CTRL>
__device__ __forceinline__ u32 lane_swap(u32 v) {
    return (u32)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
}

__device__ __forceinline__ void report(int32_t *status, int code) {
    if (status) *status = code;  // (whoever writes, writes the same)
}

}  // namespace moe
