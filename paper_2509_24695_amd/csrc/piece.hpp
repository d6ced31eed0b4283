// Sixteen bytes of a row as fp32 numbers and back.
#pragma once

#include "common.hpp"

namespace sv {

template <typename T> struct Piece;
template <> struct Piece<uint16_t> {
    typedef u32x4 V;
    static constexpr int kN = 8;
    static __device__ __forceinline__ void open(u32x4 v, float (&x)[8])
    {
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            x[2 * p] = bf16_lo(v[p]);
            x[2 * p + 1] = bf16_hi(v[p]);
        }
    }
    static __device__ __forceinline__ u32x4 close(const float (&x)[8])
    {
        return u32x4{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])};
    }
};
template <> struct Piece<float> {
    typedef u32x4 V;
    static constexpr int kN = 4;
    static __device__ __forceinline__ void open(u32x4 v, float (&x)[4])
    {
#pragma unroll
        for (int p = 0; p < 4; ++p) x[p] = __uint_as_float(v[p]);
    }
    static __device__ __forceinline__ u32x4 close(const float (&x)[4])
    {
        return u32x4{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
    }
};

// Four numbers of either type, for kernels that keep much beside each.
template <typename T> struct Quad;
template <> struct Quad<float> : Piece<float> {};
template <> struct Quad<uint16_t> {
    typedef u32x2 V;
    static constexpr int kN = 4;
    static __device__ __forceinline__ void open(u32x2 v, float (&x)[4])
    {
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            x[2 * p] = bf16_lo(v[p]);
            x[2 * p + 1] = bf16_hi(v[p]);
        }
    }
    static __device__ __forceinline__ u32x2 close(const float (&x)[4]) { return u32x2{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3])}; }
};

}  // namespace sv
