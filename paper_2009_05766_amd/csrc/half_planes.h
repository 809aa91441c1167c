// float values as two planes of halves: v = hi + lo, 22 bits and more where v is scaled into the halves' range.
#pragma once
#include "gemm16.h"

namespace netmax {

__device__ __forceinline__ uint32_t half_bits(_Float16 h) { return (uint32_t)__builtin_bit_cast(uint16_t, h); }

struct TwoHalves {
    _Float16 hi, lo;
    __device__ __forceinline__ explicit TwoHalves(float v)
    {
        hi = (_Float16)v;
        lo = (_Float16)(v - (float)hi);
    }
};
__device__ __forceinline__ float joined(uint16_t hi, uint16_t lo) { return (float)__builtin_bit_cast(_Float16, lo) + (float)__builtin_bit_cast(_Float16, hi); }

// Four neighbours of a row of planes, as they lie in memory; the planes' rows are padded to multiples of 8.  Read as global memory by name: where the compiler
// does not know (behind a choice), its requests are waited for with those to LDS.
struct RawPlanes { u32x2 hi, lo; };
__device__ __forceinline__ f32x4 joined(const RawPlanes &p)
{
    return f32x4{joined((uint16_t)p.hi[0], (uint16_t)p.lo[0]), joined((uint16_t)(p.hi[0] >> 16), (uint16_t)(p.lo[0] >> 16)), joined((uint16_t)p.hi[1], (uint16_t)p.lo[1]),
                 joined((uint16_t)(p.hi[1] >> 16), (uint16_t)(p.lo[1] >> 16))};
}
__device__ __forceinline__ u32x2 load_half_fours(const uint16_t *p) { return *(const __attribute__((address_space(1))) u32x2 *)p; }
__device__ __forceinline__ f32x4 load_planes(const uint16_t *hi, const uint16_t *lo)
{
    const uint2 h = *reinterpret_cast<const uint2 *>(hi), l = *reinterpret_cast<const uint2 *>(lo);
    return f32x4{joined((uint16_t)h.x, (uint16_t)l.x), joined((uint16_t)(h.x >> 16), (uint16_t)(l.x >> 16)), joined((uint16_t)h.y, (uint16_t)l.y),
                 joined((uint16_t)(h.y >> 16), (uint16_t)(l.y >> 16))};
}
__device__ __forceinline__ f32x4 load_plane(const uint16_t *hi)
{
    const uint2 h = *reinterpret_cast<const uint2 *>(hi);
    return f32x4{joined((uint16_t)h.x, 0), joined((uint16_t)(h.x >> 16), 0), joined((uint16_t)h.y, 0), joined((uint16_t)(h.y >> 16), 0)};
}
__device__ __forceinline__ void store_planes(uint16_t *hi, uint16_t *lo, f32x4 v)
{
    const TwoHalves a(v[0]), b(v[1]), c(v[2]), d(v[3]);
    *reinterpret_cast<uint2 *>(hi) = make_uint2(half_bits(a.hi) | half_bits(b.hi) << 16, half_bits(c.hi) | half_bits(d.hi) << 16);
    if (lo) *reinterpret_cast<uint2 *>(lo) = make_uint2(half_bits(a.lo) | half_bits(b.lo) << 16, half_bits(c.lo) | half_bits(d.lo) << 16);
}

// One launch for every block shape: `go` gets it.
template <bool SPLIT, class Blocks, class Go> static void with_small_shape(int64_t M, int64_t N, int64_t K, const Blocks &blocks, const Go &go)
{
    // the largest blocks that still give most compute units one; the fewer there are, the more waves and steps under way each has (1 x 2660 x 512, X^T X:
    // 17.3 us in one group of waves, 15.1 in two; short contractions lose by the join)
    const bool far = worth_blocks(128, M, N);
    if (blocks(128) >= 512 && far) go(Shape<128, 128, 2, 2, SPLIT ? 32 : 64, 2>());
    else if (blocks(128) >= 128 && far) go(Shape<128, 128, 2, 4, SPLIT ? 32 : 64, 4>());
    else if (blocks(64) > 256 || K < 512) go(Shape<64, 64, 2, 2, SPLIT ? 32 : 64, 4>());
    else go(Shape<64, 64, 2, 2, SPLIT ? 32 : 64, 4, 2>());
}

}  // namespace netmax
