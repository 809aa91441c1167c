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

// Moves values of a piece down by `by` places (1 .. VALUES - 1); zeros come in at the end.
__device__ __forceinline__ void shift_down(Piece<float> &x, int by)
{
    f32x4 v = x.v;
    if (by & 1) v = f32x4{v[1], v[2], v[3], 0.0f};
    if (by & 2) v = f32x4{v[2], v[3], 0.0f, 0.0f};
    x.v = v;
}
__device__ __forceinline__ void shift_down(Piece<uint16_t> &x, int by)
{
    u32x4 v = x.v;
    if (by & 1) v = u32x4{v[0] >> 16 | v[1] << 16, v[1] >> 16 | v[2] << 16, v[2] >> 16 | v[3] << 16, v[3] >> 16};
    if (by & 2) v = u32x4{v[1], v[2], v[3], 0u};
    if (by & 4) v = u32x4{v[2], v[3], 0u, 0u};
    x.v = v;
}

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
// The piece of a row of `cols` values from column col on (0 .. cols - 1).  One that ends behind the row is read as the row's last full piece and moved when it has come (settled), so that no
// value is read by itself and no read waits for another.  Rows shorter than a piece are read by their values.
template <typename T> __device__ __forceinline__ Piece<T> fetch_piece(const T *row, int64_t col, int64_t cols)
{
    constexpr int VALUES = Piece<T>::VALUES;
    if (cols < VALUES) return load_piece(row + col, cols - col);
    Piece<T> x;
    x.v = *reinterpret_cast<const typename Piece<T>::Memory *>(row + (col <= cols - VALUES ? col : cols - VALUES));
    return x;
}
template <typename T> __device__ __forceinline__ void settle_piece(Piece<T> &x, int64_t col, int64_t cols)
{
    constexpr int VALUES = Piece<T>::VALUES;
    if (cols >= VALUES && col > cols - VALUES) shift_down(x, (int)(col - (cols - VALUES)));
}
// A row's last values in as few writes as their number has bits.
__device__ __forceinline__ void store_some(float *p, Piece<float> x, int left)
{
    typedef float f32x2_any __attribute__((ext_vector_type(2), aligned(4)));
    if (left & 2) {
        *reinterpret_cast<f32x2_any *>(p) = f32x2_any{x.v[0], x.v[1]};
        p += 2;
        x.v[0] = x.v[2];
    }
    if (left & 1) *p = x.v[0];
}
__device__ __forceinline__ void store_some(uint16_t *p, Piece<uint16_t> x, int left)
{
    typedef uint32_t u32_any __attribute__((aligned(2)));
    if (left & 4) {
        *reinterpret_cast<u32x2_any *>(p) = u32x2{x.v[0], x.v[1]};
        p += 4;
        x.v[0] = x.v[2];
        x.v[1] = x.v[3];
    }
    if (left & 2) {
        *reinterpret_cast<u32_any *>(p) = x.v[0];
        p += 2;
        x.v[0] = x.v[1];
    }
    if (left & 1) *p = (uint16_t)x.v[0];
}
template <typename T> __device__ __forceinline__ void store_piece(T *p, int64_t left, const Piece<T> &x)
{
    if (left >= Piece<T>::VALUES) *reinterpret_cast<typename Piece<T>::Memory *>(p) = x.v;
    else store_some(p, x, (int)left);
}

// Sums over LANES neighbouring lanes (a power of two, 64 at most), each of which gets them: the lanes of a row of 16 exchange values on their way into the addition.
template <int CONTROL> __device__ __forceinline__ uint32_t moved(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CONTROL, 0xF, 0xF, true); }
template <int CONTROL> __device__ __forceinline__ float moved(float v) { return __uint_as_float(moved<CONTROL>(__float_as_uint(v))); }
template <int CONTROL> __device__ __forceinline__ double moved(double v)
{
    return __hiloint2double((int)moved<CONTROL>((uint32_t)__double2hiint(v)), (int)moved<CONTROL>((uint32_t)__double2loint(v)));
}
template <bool HALVES> __device__ __forceinline__ float both(float v)
{
    const uint32_t u = __float_as_uint(v);
    const auto w = HALVES ? __builtin_amdgcn_permlane32_swap(u, u, false, false) : __builtin_amdgcn_permlane16_swap(u, u, false, false);
    return __uint_as_float(w[0]) + __uint_as_float(w[1]);
}
template <bool HALVES> __device__ __forceinline__ double both(double v)
{
    const uint32_t lo = (uint32_t)__double2loint(v), hi = (uint32_t)__double2hiint(v);
    const auto l = HALVES ? __builtin_amdgcn_permlane32_swap(lo, lo, false, false) : __builtin_amdgcn_permlane16_swap(lo, lo, false, false);
    const auto h = HALVES ? __builtin_amdgcn_permlane32_swap(hi, hi, false, false) : __builtin_amdgcn_permlane16_swap(hi, hi, false, false);
    return __hiloint2double((int)h[0], (int)l[0]) + __hiloint2double((int)h[1], (int)l[1]);
}
template <int LANES, typename S> __device__ __forceinline__ S lanes_sum(S v)
{
    if constexpr (LANES >= 2) v += moved<0xB1>(v);                  // lanes 1 0 3 2
    if constexpr (LANES >= 4) v += moved<0x4E>(v);                  // lanes 2 3 0 1
    if constexpr (LANES >= 8) v += moved<0x141>(v);                 // eight in reverse
    if constexpr (LANES >= 16) v += moved<0x140>(v);                // sixteen in reverse
    if constexpr (LANES >= 32) v = both<false>(v);
    if constexpr (LANES >= 64) v = both<true>(v);
    return v;
}

// Sums over the LANES lanes that work on one row: part of a wave, or a workgroup of so many threads (whole waves), through `room`, with one barrier; before a `room` is used again there is
// another one (of another sum, or the caller's).
template <int LANES, int N, typename S> __device__ __forceinline__ void row_sum(S (&v)[N], S (*room)[N])
{
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = lanes_sum<(LANES < 64 ? LANES : 64)>(v[k]);
    if constexpr (LANES > 64) {
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int k = 0; k < N; ++k) room[threadIdx.x >> 6][k] = v[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < N; ++k) {
            constexpr int WAVES = LANES / 64, EVEN = WAVES <= 2 ? 2 : WAVES <= 4 ? 4 : WAVES <= 8 ? 8 : 16;      // the power of two from there on
            const int w = threadIdx.x & (EVEN - 1);
            const S part = room[w < WAVES ? w : 0][k];
            v[k] = lanes_sum<EVEN>(w < WAVES ? part : S(0));
        }
    }
}

}  // namespace netmax
