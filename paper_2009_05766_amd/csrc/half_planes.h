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
    // the fewer blocks, the more waves and steps under way each has (1 x 2660 x 512, X^T X: 17.3 us in one group of waves, 15.1 in two; short contractions lose by the
    // join).  Whole updates of five steps with these on both sides of each line, bfloat16: steps of 60 x 256 x 256 (240 blocks of 128) in four waves and two stages 198 and
    // in eight and four 194, 68 (272) 216 and 230, squares of 24 x 512 x 512 (240) 312 and 264, 88 x 256 x 256 (264) 286 and 322; in blocks of 128 and of 64, steps of 8 x 512 x 512 (128)
    // 158 and 148, 36 x 256 x 256 (144) 145 and 152, squares of 13 x 512 x 784 (130) 276 and 238, 2048 x 2048 (136) 410 and 451; blocks of 64 in one group and
    // two, 3 x 576 x 576 (243) 142 and 137, 4 (324) 144 and 167; on two planes (float) the same lines
    const bool far = worth_blocks(128, M, N);
    if (blocks(128) > 256 && far) go(Shape<128, 128, 2, 2, SPLIT ? 32 : 64, 2>());
    else if (blocks(128) > 128 && far) go(Shape<128, 128, 2, 4, SPLIT ? 32 : 64, 4>());
    else if (blocks(64) > 256 || K < 512) go(Shape<64, 64, 2, 2, SPLIT ? 32 : 64, 4>());
    else go(Shape<64, 64, 2, 2, SPLIT ? 32 : 64, 4, 2>());
}

}  // namespace netmax
