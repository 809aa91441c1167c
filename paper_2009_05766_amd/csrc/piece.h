// Rows of float or bfloat16 values in pieces of 16 bytes, for kernels that stream them.
#pragma once
#include "gemm.h"

namespace netmax {

// 16 bytes of a row, at any address of a value.
template <typename T> struct Piece;
template <> struct Piece<float> {
    static constexpr int VALUES = 4;
    typedef f32x4_any Memory;
    f32x4 v;
    __device__ __forceinline__ float get(int k) const { return v[k]; }
    __device__ __forceinline__ void set(const float (&x)[4]) { v = f32x4{x[0], x[1], x[2], x[3]}; }
};
template <> struct Piece<uint16_t> {
    static constexpr int VALUES = 8;
    typedef u32x4_any Memory;
    u32x4 v;
    __device__ __forceinline__ float get(int k) const { return __uint_as_float(k & 1 ? v[k >> 1] & 0xFFFF0000u : v[k >> 1] << 16); }
    __device__ __forceinline__ void set(const float (&x)[8])
    {
        v = u32x4{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])};
    }
};

// A piece of a row from p on, where `left` values of the row lie (1 or more); those behind the row are 0.
template <typename T> __device__ __forceinline__ Piece<T> load_piece(const T *p, int64_t left)
{
    constexpr int VALUES = Piece<T>::VALUES;
    Piece<T> x;
    if (left >= VALUES) {
        x.v = *reinterpret_cast<const typename Piece<T>::Memory *>(p);
    } else {
        float v[VALUES];
#pragma unroll
        for (int k = 0; k < VALUES; ++k) v[k] = k < left ? load_value(p + k) : 0.0f;
        x.set(v);
    }
    return x;
}
template <typename T> __device__ __forceinline__ void store_piece(T *p, int64_t left, const Piece<T> &x)
{
    constexpr int VALUES = Piece<T>::VALUES;
    if (left >= VALUES) {
        *reinterpret_cast<typename Piece<T>::Memory *>(p) = x.v;
    } else {
#pragma unroll
        for (int k = 0; k < VALUES; ++k)
            if (k < left) store_value(p + k, x.get(k));
    }
}

// Sums of a whole workgroup, in a fixed order; every thread gets them.  One barrier: the caller separates two sums through the same LDS by another.
template <int THREADS, int N, typename S> __device__ __forceinline__ void workgroup_sum(S (&v)[N], S (*room)[N])
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1)
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] += __shfl_xor(v[k], d);
    if constexpr (THREADS > 64) {
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int k = 0; k < N; ++k) room[threadIdx.x >> 6][k] = v[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = 0;
#pragma unroll
        for (int w = 0; w < THREADS / 64; ++w)
#pragma unroll
            for (int k = 0; k < N; ++k) v[k] += room[w][k];
    }
}

}  // namespace netmax
