// Matrix products C = A B of the operators for language models: operands, epilogues and launchers.
//
// A is [M][K] and B [K][N]; either may be stored with its contraction index K next to each other in memory ("k_near") or
// with M (of A), N (of B) next to each other.  ld: elements from one stored row to the next; step: from one matrix of the
// batch to the next.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "bf16.h"
#include "vec.h"

namespace netmax {

struct Operand { const void *p; int64_t ld, step; bool k_near; };

inline int64_t up_to(int64_t n, int64_t to) { return (n + to - 1) / to * to; }
// Whether blocks of `side` squared do not waste behind the edges of M x N results what they gain over blocks of half that side (batches of small matrices:
// 600 x 512 x 120 x 120 bfloat16 74 us in blocks of 256, 46 in blocks of 128; 300 x 200 x 512 x 64 43 and 21).
inline bool worth_blocks(int64_t side, int64_t M, int64_t N)
{
    return 4 * up_to(M, side) * up_to(N, side) <= 5 * up_to(M, side / 2) * up_to(N, side / 2);
}

// Shapes of blocks are chosen by how many workgroups each would have for the card's 256 compute units: larger blocks read less per product, smaller ones
// share the card better as long as they do not take another turn.  The figures beside each choice are times of the kernel (us) on both sides of its line.

typedef float f32x16 __attribute__((ext_vector_type(16)));

// LDS that lanes of one wave exchange values through: what is written before is read behind.
__device__ __forceinline__ void wave_order()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Workgroup `id` of two products in one launch, numbered as if the `first` ones of the first product came first; `swap`: the second product's start before them.
// The one with the longer chains of steps has to (float, 300 x 1024 x 40 x 100, dx and dw: 125 us, the other way round 172).
__device__ __forceinline__ uint32_t pair_place(uint32_t id, uint32_t first, uint32_t both, int swap)
{
    if (!swap || id >= both) return id;
    return id < both - first ? id + first : id - (both - first);
}

enum Act : int { ACT_NONE = 0, ACT_RELU = 1, ACT_GELU = 2, ACT_SILU = 3 };

// The normal distribution function and the bell exp(-z^2 / 2), which it needs anyway: for z < 0 it is the bell times 0.5 erfc(x) exp(x^2), x = -z / sqrt 2,
// and that factor is a polynomial without a constant term in t = 1 / (1 + 0.43 x).  The coefficients are a least-squares fit of the relative error, reweighted
// to its smallest maximum over 0 <= x <= 9.8 (where the bell leaves the type's range): 9.2e-8.  In float the result is within (8 + z^2) 2^-23 of itself: the tails, where
// 0.5 (1 + erf) cancels, keep their bits.  (The library's erff took as long as all other work of an epilogue.)
__device__ __forceinline__ float normal_distribution(float z, float &bell)
{
    const float t = __builtin_amdgcn_rcpf(fmaf(0.30405593f, fabsf(z), 1.0f));
    bell = __builtin_amdgcn_exp2f(-0.72134752f * z * z);
    float factor = fmaf(t, 0.0367018394f, -0.154570311f);
    factor = fmaf(t, factor, 0.190819323f);
    factor = fmaf(t, factor, -0.0419362932f);
    factor = fmaf(t, factor, 0.122944094f);
    factor = fmaf(t, factor, 0.102617107f);
    factor = fmaf(t, factor, 0.122165523f);
    factor = fmaf(t, factor, 0.121258728f);
    const float tail = t * factor * bell;
    return z < 0.0f ? tail : 1.0f - tail;
}
__device__ __forceinline__ float sigmoid_of(float z) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -1.44269504f)); }

// act(z); GELU with the normal distribution function (not its tanh form).
__device__ __forceinline__ float act_of(int act, float z)
{
    float bell;
    if (act == ACT_RELU) return z < 0.0f ? 0.0f : z;                // a NaN stays one
    if (act == ACT_GELU) return z * normal_distribution(z, bell);
    if (act == ACT_SILU) return z * sigmoid_of(z);
    return z;
}

// act'(z); ReLU's is 0 at 0.  Far out a factor that grows with z meets one that has vanished: such products are 0.
__device__ __forceinline__ float act_slope(int act, float z)
{
    if (act == ACT_RELU) return z > 0.0f ? 1.0f : z != z ? z : 0.0f;
    if (act == ACT_GELU) {
        float bell;
        const float below = normal_distribution(z, bell);
        return below + (bell == 0.0f ? 0.0f : z * (bell * 0.39894228f));
    }
    if (act == ACT_SILU) {
        const float s = sigmoid_of(z);
        return s == 0.0f ? 0.0f : s * (1.0f + z * (1.0f - s));
    }
    return 1.0f;
}

// ---- values in memory: float or bfloat16 (as its 16 bits) ------------------------------------------------------------

__device__ __forceinline__ float load_value(const float *p) { return *p; }
__device__ __forceinline__ float load_value(const uint16_t *p) { return bf16_bits_to_float(*p); }
__device__ __forceinline__ void store_value(float *p, float v) { *p = v; }
__device__ __forceinline__ void store_value(uint16_t *p, float v) { *p = (uint16_t)bf16_bits(v); }
// Four neighbours at any address of a value, in one request.
typedef f32x4 f32x4_any __attribute__((aligned(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef u32x2 u32x2_any __attribute__((aligned(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_any __attribute__((aligned(2)));
template <typename T> struct Raw;                                   // as they lie in memory
template <> struct Raw<float> { typedef f32x4 four; };
template <> struct Raw<uint16_t> { typedef u32x2 four; };
__device__ __forceinline__ f32x4 load_raw(const float *p) { return *reinterpret_cast<const f32x4_any *>(p); }
__device__ __forceinline__ u32x2 load_raw(const uint16_t *p) { return *reinterpret_cast<const u32x2_any *>(p); }
__device__ __forceinline__ f32x4 widened(f32x4 v) { return v; }
__device__ __forceinline__ f32x4 widened(u32x2 u)
{
    return f32x4{__uint_as_float(u[0] << 16), __uint_as_float(u[0] & 0xFFFF0000u), __uint_as_float(u[1] << 16), __uint_as_float(u[1] & 0xFFFF0000u)};
}
template <typename T> __device__ __forceinline__ f32x4 load_four(const T *p) { return widened(load_raw(p)); }
__device__ __forceinline__ void store_four(float *p, f32x4 v) { *reinterpret_cast<f32x4_any *>(p) = v; }
__device__ __forceinline__ void store_four(uint16_t *p, f32x4 v)
{
    *reinterpret_cast<u32x2_any *>(p) = u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
}
// Four values from column n of `cols`; those behind the last are 0.
template <typename T> __device__ __forceinline__ f32x4 load_up_to_four(const T *row, int64_t n, int64_t cols)
{
    if (n + 4 <= cols) return load_four(row + n);
    f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (n + e < cols) v[e] = load_value(row + n + e);
    return v;
}
__device__ __forceinline__ f32x4 load_raw_up_to_four(const float *row, int64_t n, int64_t cols) { return load_up_to_four(row, n, cols); }
__device__ __forceinline__ u32x2 load_raw_up_to_four(const uint16_t *row, int64_t n, int64_t cols)
{
    if (n + 4 <= cols) return load_raw(row + n);
    uint32_t v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = n + e < cols ? row[n + e] : 0u;
    return u32x2{v[0] | v[1] << 16, v[2] | v[3] << 16};
}
template <typename T> __device__ __forceinline__ void store_up_to_four(T *row, int64_t n, int64_t cols, f32x4 v)
{
    if (n + 4 <= cols) { store_four(row + n, v); return; }
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (n + e < cols) store_value(row + n + e, v[e]);
}

// ---- epilogues: told of four neighbouring columns n .. n + 3 of row m of matrix g of the batch -----------------------
//
// What an epilogue reads it can be asked for ahead: columns() is the same for all rows, see() belongs to one call of leave().  Reads and writes of a wave
// are waited for in their order, so that a read behind writes costs their whole way to memory: a kernel with many results per wave sees what comes next
// before it writes (8192 x 1024 x 8192 bfloat16 with GELU, residual and z: 245 us, each read where it is used 304).  FULL: all columns and rows asked for exist.

// y = act(acc + bias) + residual, z = acc + bias; bias, residual and z may be null.
template <typename T> struct LinearEpilogue {
    int64_t M, N;
    const T *bias, *residual; T *y, *z;
    int64_t ldr, ldy, ldz, sb, sr, sy, sz;
    int act;
    __device__ __forceinline__ int64_t rows_here() const { return M; }
    __device__ __forceinline__ int64_t cols_here() const { return N; }
    struct Columns { f32x4 bias; };
    struct Seen { typename Raw<T>::four residual; };
    template <bool FULL> __device__ __forceinline__ Columns columns(int64_t g, int64_t n) const
    {
        return Columns{bias && (FULL || n < N) ? load_up_to_four(bias + g * sb, n, N) : f32x4{0, 0, 0, 0}};
    }
    template <bool FULL> __device__ __forceinline__ Seen see(int64_t g, int64_t m, int64_t n) const
    {
        if (!residual || (!FULL && (m >= M || n >= N))) return Seen{};
        const T *row = residual + g * sr + m * ldr;
        return Seen{FULL ? load_raw(row + n) : load_raw_up_to_four(row, n, N)};
    }
    template <bool FULL> __device__ __forceinline__ void leave(int64_t g, int64_t m, int64_t n, f32x4 v, const Columns &c, const Seen &s) const
    {
        if (!FULL && (m >= M || n >= N)) return;
        if (bias) v += c.bias;
        if (z) store<FULL>(z + g * sz + m * ldz, n, v);
        if (act != ACT_NONE)
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = act_of(act, v[e]);
        if (residual) v += widened(s.residual);
        store<FULL>(y + g * sy + m * ldy, n, v);
    }
    template <bool FULL> __device__ __forceinline__ void store(T *row, int64_t n, f32x4 v) const
    {
        if (FULL) store_four(row + n, v); else store_up_to_four(row, n, N, v);
    }
    __device__ __forceinline__ void operator()(int64_t g, int64_t m, int64_t n, f32x4 v) const { leave<false>(g, m, n, v, columns<false>(g, n), see<false>(g, m, n)); }
};

}  // namespace netmax
