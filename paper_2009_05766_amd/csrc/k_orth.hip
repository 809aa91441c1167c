// An orthogonalised momentum update for a batch of matrices:
//     m' = mu m + g,   u = g + mu m' (Nesterov) or m',   X = u / max(||u||_F, eps),
//     `steps` times:   A = X X^T,   B = b A + c A A,   X <- a X + B X,        out = scale X.
// The polynomial a s + b s^3 + c s^5 drives the singular values of X towards 1 and leaves the singular vectors alone.  Matrices with
// more rows than columns are multiplied from the other side, A = X^T X and X <- a X + X B, which is the same polynomial on the smaller
// square.
//
// X, A and B are held as two planes of halves, scaled by powers of two: 2^11 X = hi + lo, 2^8 A, 2^8 B.  hi carries 11 bits and lo the next ones, down to
// the halves' smallest step, 2^-24: 2^-35 of X, whose entries are about one over the root of the longer side in the end and smaller by the root
// of the other side at the start, 2^-32 of A and B.  Halves reach to 65504: |X| <= 1 at the start, and singular values stay below 1.3 with the
// usual coefficients (a polynomial that lets X grow past 32, or A or B past 255, is not for this operator).
//   float        hi hi + hi lo + lo hi (SPLIT): as exact as float products, at three times the cost of one product of halves instead of sixteen times
//   bfloat16     products of hi planes (11 bits), the term a X from both planes.  B's diagonal, its large part near the end, is kept in float and
//                joins a X: the rounding of B then halves the result's error, to 0.6e-3 where the rounding of the result itself is 1.7e-3
// A and B are symmetric: their blocks on and below the diagonal are computed and written to both sides.
// 8 x 2048 x 4096 bfloat16, five steps: 3.77 ms, of it momentum and norm 0.30 (1.34 GB), A and B 1.66, X 1.81 (its planes, in and
// out, take as long as half of the products).  16 x 784 x 512 float: 0.42 ms, bound by the chain of seventeen launches of 14 to 32 us.
#include "half_planes.h"
#include "orth.h"

#include <type_traits>

namespace netmax {

constexpr int NORM_BLOCKS = 256;      // partial sums of squares of one matrix, at most: one for each thread that adds them up

constexpr float X_SCALE = 0x1p11f, SQUARE_SCALE = 0x1p8f;

// A symmetric result alpha acc + beta own as planes [batch][side][wide], zeros behind each row; lo may be null.  With `diagonal` its diagonal goes
// there and is 0 in the planes.  Squares of 64 x 64 on the diagonal lie whole inside computed blocks and are kept as they come; of all others those
// below it are, and their mirror images.
struct SquareEpilogue {
    int64_t side, wide; float alpha, beta;
    const uint16_t *own_hi, *own_lo; uint16_t *hi, *lo; float *diagonal;
    __device__ __forceinline__ void keep(int64_t g, int64_t m, int64_t n, f32x4 v) const
    {
        const int64_t at = (g * side + m) * wide + n;
        v *= alpha;
        if (own_hi) v += beta * (own_lo ? load_planes(own_hi + at, own_lo + at) : load_plane(own_hi + at));
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (n + e >= side) v[e] = 0.0f;
            if (diagonal && n + e == m) { diagonal[g * side + m] = v[e] * (1.0f / SQUARE_SCALE); v[e] = 0.0f; }
        }
        store_planes(hi + at, lo ? lo + at : nullptr, v);
    }
    __device__ __forceinline__ void operator()(int64_t g, int64_t m, int64_t n, f32x4 v) const
    {
        if (m < side && n < wide && m / 64 >= n / 64) keep(g, m, n, v);
    }
    __device__ __forceinline__ void mirror(int64_t g, int64_t m, int64_t n, f32x4 v) const
    {
        if (m < side && n < wide && n / 64 > m / 64) keep(g, m, n, v);
    }
};

// X <- acc + (a + diagonal) X as planes [batch][rows][wide]; the diagonal goes by rows or, `tall`, by columns.
struct StepEpilogue {
    int64_t rows, cols, wide; float a; bool tall;
    const uint16_t *own_hi, *own_lo; uint16_t *hi, *lo; const float *diagonal;
    __device__ __forceinline__ int64_t rows_here() const { return rows; }
    __device__ __forceinline__ int64_t cols_here() const { return cols; }
    struct Columns { f32x4 f; };
    struct Seen { RawPlanes x; float diagonal; };
    template <bool FULL> __device__ __forceinline__ Columns columns(int64_t g, int64_t n) const
    {
        Columns c{f32x4{a, a, a, a}};
        if (diagonal && tall)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (FULL || n + e < cols) c.f[e] += diagonal[g * cols + n + e];
        return c;
    }
    template <bool FULL> __device__ __forceinline__ Seen see(int64_t g, int64_t m, int64_t n) const
    {
        Seen s{};
        if (!FULL && (m >= rows || n >= wide)) return s;
        const int64_t at = (g * rows + m) * wide + n;
        s.x = RawPlanes{load_half_fours(own_hi + at), load_half_fours(own_lo + at)};
        if (diagonal && !tall) s.diagonal = diagonal[g * rows + m];
        return s;
    }
    template <bool FULL> __device__ __forceinline__ f32x4 value(int64_t n, f32x4 v, const Columns &c, const Seen &s) const
    {
        const f32x4 x = joined(s.x);
        v *= 1.0f / SQUARE_SCALE;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = FULL || n + e < cols ? fmaf(c.f[e] + s.diagonal, x[e], v[e]) : 0.0f;
        return v;
    }
    template <bool FULL> __device__ __forceinline__ void leave(int64_t g, int64_t m, int64_t n, f32x4 v, const Columns &c, const Seen &s) const
    {
        if (!FULL && (m >= rows || n >= wide)) return;
        const int64_t at = (g * rows + m) * wide + n;
        store_planes(hi + at, lo + at, value<FULL>(n, v, c, s));
    }
};

// The last step: scale X to the caller's memory.
template <typename T> struct LastEpilogue {
    StepEpilogue step; float scale; T *out; int64_t ldo, so;
    __device__ __forceinline__ int64_t rows_here() const { return step.rows; }
    __device__ __forceinline__ int64_t cols_here() const { return step.cols; }
    typedef StepEpilogue::Columns Columns;
    typedef StepEpilogue::Seen Seen;
    template <bool FULL> __device__ __forceinline__ Columns columns(int64_t g, int64_t n) const { return step.columns<FULL>(g, n); }
    template <bool FULL> __device__ __forceinline__ Seen see(int64_t g, int64_t m, int64_t n) const { return step.see<FULL>(g, m, n); }
    template <bool FULL> __device__ __forceinline__ void leave(int64_t g, int64_t m, int64_t n, f32x4 v, const Columns &c, const Seen &s) const
    {
        if (!FULL && (m >= step.rows || n >= step.cols)) return;
        v = scale * step.value<FULL>(n, v, c, s);
        T *row = out + g * so + m * ldo;
        if (FULL) store_four(row + n, v); else store_up_to_four(row, n, step.cols, v);
    }
};

// Four neighbours q of a matrix, in units of four of rows padded to `wide`: their row and column.
__device__ __forceinline__ void unit_place(int64_t q, uint32_t units, int64_t &r, int64_t &c)
{
    if (q <= 0xFFFFFFFF) { const uint32_t row = (uint32_t)q / units; r = row; c = ((uint32_t)q - row * units) * 4; }
    else { r = q / units; c = (q - r * units) * 4; }
}

// Two kernels with the same workgroups: a workgroup takes every NORM_BLOCKS-th run of 256 units, four of them in flight per thread.
constexpr int NORM_AHEAD = 4;

// m' and a part of the sum of squares of u (in double; the parts are added in order by whoever needs the norm).
template <typename T>
__global__ void __launch_bounds__(256) momentum_kernel(OrthArgs a, double *__restrict__ parts)
{
    __shared__ double part[256];
    const int64_t g = blockIdx.y;
    const uint32_t units = (uint32_t)((a.cols + 3) / 4);
    const int64_t count = a.rows * units, stride = (int64_t)gridDim.x * 256;
    const T *from = (const T *)a.g + g * a.sg;
    double sum = 0.0;
    for (int64_t q0 = (int64_t)blockIdx.x * 256 + threadIdx.x; q0 < count; q0 += NORM_AHEAD * stride) {
        f32x4 u[NORM_AHEAD], m[NORM_AHEAD];
        int64_t r[NORM_AHEAD], c[NORM_AHEAD];
#pragma unroll
        for (int k = 0; k < NORM_AHEAD; ++k) {
            const int64_t q = q0 + k * stride;
            if (q >= count) { u[k] = m[k] = f32x4{0, 0, 0, 0}; continue; }
            unit_place(q, units, r[k], c[k]);
            u[k] = load_up_to_four(from + r[k] * a.ldg, c[k], a.cols);
            if (a.m) m[k] = load_up_to_four(a.m + g * a.sm + r[k] * a.ldm, c[k], a.cols);
        }
#pragma unroll
        for (int k = 0; k < NORM_AHEAD; ++k) {
            if (q0 + k * stride >= count) continue;
            if (a.m) {
                m[k] = fma4(a.mu, m[k], u[k]);
                store_up_to_four(a.m_out + g * a.sm + r[k] * a.ldm, c[k], a.cols, m[k]);
                u[k] = a.nesterov ? fma4(a.mu, m[k], u[k]) : m[k];
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) sum += (double)u[k][e] * (double)u[k][e];
        }
    }
    part[threadIdx.x] = sum;
    __syncthreads();
    for (int d = 128; d > 0; d >>= 1) {
        if ((int)threadIdx.x < d) part[threadIdx.x] += part[threadIdx.x + d];
        __syncthreads();
    }
    if (threadIdx.x == 0) parts[g * gridDim.x + blockIdx.x] = part[0];
}

// The planes of s u / max(||u||, eps).
template <typename T>
__global__ void __launch_bounds__(256) normalise_kernel(OrthArgs a, const double *__restrict__ parts, float s, int64_t wide, uint16_t *__restrict__ hi,
                                                        uint16_t *__restrict__ lo)
{
    const int64_t g = blockIdx.y;
    const uint32_t units = (uint32_t)(wide / 4);
    const int64_t count = a.rows * units, stride = (int64_t)gridDim.x * 256;
    // every workgroup adds the parts in the same order
    __shared__ double total[4];
    double sum = threadIdx.x < gridDim.x ? parts[g * gridDim.x + threadIdx.x] : 0.0;
    for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
    if ((threadIdx.x & 63) == 0) total[threadIdx.x >> 6] = sum;
    __syncthreads();
    sum = (total[0] + total[1]) + (total[2] + total[3]);
    const double norm = sqrt(sum), factor = (double)s / (norm > (double)a.eps || norm != norm ? norm : (double)a.eps);
    const T *from = (const T *)a.g + g * a.sg;
    for (int64_t q0 = (int64_t)blockIdx.x * 256 + threadIdx.x; q0 < count; q0 += NORM_AHEAD * stride) {
        f32x4 u[NORM_AHEAD], m[NORM_AHEAD];
#pragma unroll
        for (int k = 0; k < NORM_AHEAD; ++k) {
            const int64_t q = q0 + k * stride;
            u[k] = m[k] = f32x4{0, 0, 0, 0};
            if (q >= count) continue;
            int64_t r, c;
            unit_place(q, units, r, c);
            if (!a.m || a.nesterov) u[k] = load_up_to_four(from + r * a.ldg, c, a.cols);
            if (a.m) m[k] = load_up_to_four(a.m_out + g * a.sm + r * a.ldm, c, a.cols);
        }
#pragma unroll
        for (int k = 0; k < NORM_AHEAD; ++k) {
            const int64_t q = q0 + k * stride;
            if (q >= count) continue;
            if (a.m) u[k] = a.nesterov ? fma4(a.mu, m[k], u[k]) : m[k];
#pragma unroll
            for (int e = 0; e < 4; ++e) u[k][e] = (float)((double)u[k][e] * factor);
            store_planes(hi + (g * count + q) * 4, lo + (g * count + q) * 4, u[k]);
        }
    }
}

// Workgroups for one matrix: enough for the card, and not more than have something to do.
static uint32_t norm_blocks(const OrthArgs &a)
{
    const int64_t work = (a.rows * ((a.cols + 3) / 4) + 256 * NORM_AHEAD - 1) / (256 * NORM_AHEAD), fill = (2048 + a.batch - 1) / a.batch;
    const int64_t n = work < fill ? work : fill;
    return (uint32_t)(n < 1 ? 1 : n > NORM_BLOCKS ? NORM_BLOCKS : n);
}

static int64_t side_of(const OrthArgs &a) { return a.rows < a.cols ? a.rows : a.cols; }
static int64_t up8(int64_t n) { return (n + 7) / 8 * 8; }
static int64_t up256(int64_t n) { return (n + 255) / 256 * 256; }
static int64_t x_bytes(const OrthArgs &a) { return up256(a.batch * a.rows * up8(a.cols) * 2); }               // one plane
static int64_t square_bytes(const OrthArgs &a) { return up256(a.batch * side_of(a) * up8(side_of(a)) * 2); }

int64_t orth_workspace(const OrthArgs &a)
{
    return 4 * x_bytes(a) + (a.bf16 ? 2 : 4) * square_bytes(a) + up256(a.batch * side_of(a) * 4) + up256(8 * a.batch * NORM_BLOCKS);
}

// Many blocks: 256 x 128, two workgroups on a compute unit, so that the results of one (planes in and out, as long as half of the products) leave under
// the products of the other.  8 x 2048 x 4096, step: 404 us, in blocks of 256 x 256 446 us (388 since the epilogue sees ahead).  Whole updates on two planes (float), steps in
// these blocks and in 128 x 128: 16 x 784 x 512 423 and 436 us, 4 x 2048 x 2048 2.69 and 2.71 ms, 20 x 784 x 512 545 and 515 us; their squares are better off in
// 128 x 128 (24 x 768 x 768 1.12 ms, 1.38 with the squares in 256 x 128; 43 x 512 x 520 0.85 and 1.10).
typedef Shape<256, 128, 4, 2, 32, 3> Paired;

template <bool SPLIT> static void launch_square(hipStream_t s, int64_t batch, int64_t side, int64_t K, const Planes16 &x, bool near, const SquareEpilogue &e)
{
    const auto go = [&](auto f) { launch_gemm16_triangle<half8, f.BM, f.BN, f.WM, f.WN, f.STEP, f.STAGES, f.GROUPS, SPLIT>(s, batch, side, K, x, near, e); };
    const auto blocks = [&](int64_t b) { const int64_t n = (side + b - 1) / b; return batch * n * (n + 1) / 2; };
    // in 256 x 128 blocks and in 128 x 128, us of a whole update: 3 x 2048 x 2048 (108 squares of 256) 868 and 892, 14 x 1024 x 1024 (140) 728 and 635, 6 x 2048 x 2048 (216) 1566 and 1622
    if constexpr (!SPLIT)
        if (blocks(256) >= 192 && worth_blocks(256, side, side)) { go(Paired()); return; }
    with_small_shape<SPLIT>(side, side, K, blocks, go);
}

template <bool SPLIT, class Epilogue>
static void launch_step(hipStream_t s, const OrthArgs &a, const Planes16 &x, const Planes16 &b, const Epilogue &e)
{
    const bool tall = a.rows > a.cols;
    const int64_t k = side_of(a);
    const Planes16 &l = tall ? x : b, &r = tall ? b : x;            // B is symmetric: its rows are its columns
    const auto go = [&](auto f) { launch_gemm16_step<half8, f.BM, f.BN, f.WM, f.WN, f.STEP, f.STAGES, f.GROUPS, SPLIT>(s, a.batch, a.rows, a.cols, k, l, r, tall, e); };
    const auto blocks = [&](int64_t n) { return a.batch * ((a.rows + n - 1) / n) * ((a.cols + n - 1) / n); };
    if constexpr (SPLIT) {
        if (blocks(256) >= 128 && worth_blocks(128, a.rows, a.cols) && worth_blocks(256, a.rows, a.cols)) { go(Paired()); return; }
    } else
        if (blocks(256) >= 192 && worth_blocks(256, a.rows, a.cols)) {
            if constexpr (std::is_same<Epilogue, StepEpilogue>::value) go(Paired());
            else go(Shape<256, 256, 2, 4, 64, 2>());
            return;
        }
    with_small_shape<SPLIT>(a.rows, a.cols, k, blocks, go);
}

template <typename T> static void orth_of(hipStream_t s, const OrthArgs &a, char *work)
{
    constexpr bool SPLIT = sizeof(T) == 4;
    const auto take = [&](int64_t n) { char *p = work; work += n; return (uint16_t *)p; };
    uint16_t *xh = take(x_bytes(a)), *xl = take(x_bytes(a)), *yh = take(x_bytes(a)), *yl = take(x_bytes(a));
    uint16_t *ah = take(square_bytes(a)), *bh = take(square_bytes(a)), *al = SPLIT ? take(square_bytes(a)) : nullptr, *bl = SPLIT ? take(square_bytes(a)) : nullptr;
    float *diagonal = (float *)take(up256(a.batch * side_of(a) * 4));
    double *parts = (double *)work;
    const int64_t side = side_of(a), wide = up8(a.cols), swide = up8(side);
    const bool tall = a.rows > a.cols;
    const dim3 grid(norm_blocks(a), (uint32_t)a.batch);
    momentum_kernel<T><<<grid, 256, 0, s>>>(a, parts);
    normalise_kernel<T><<<grid, 256, 0, s>>>(a, parts, X_SCALE, wide, xh, xl);
    const auto planes = [](const uint16_t *h, const uint16_t *l, int64_t ld, int64_t rows) { return Planes16{(const char *)h, (const char *)l, ld, rows * ld}; };
    for (int i = 0; i < a.steps; ++i) {
        launch_square<SPLIT>(s, a.batch, side, tall ? a.rows : a.cols, planes(xh, xl, wide, a.rows), !tall,
                             SquareEpilogue{side, swide, SQUARE_SCALE / (X_SCALE * X_SCALE), 0.0f, nullptr, nullptr, ah, al, nullptr});
        launch_square<SPLIT>(s, a.batch, side, side, planes(ah, al, swide, side), true,
                             SquareEpilogue{side, swide, a.c / SQUARE_SCALE, a.b, ah, al, bh, bl, SPLIT ? nullptr : diagonal});
        const StepEpilogue step{a.rows, a.cols, wide, a.a, tall, xh, xl, yh, yl, SPLIT ? nullptr : diagonal};
        const Planes16 x = planes(xh, xl, wide, a.rows), b = planes(bh, bl, swide, side);
        if (i + 1 < a.steps) launch_step<SPLIT>(s, a, x, b, step);
        else launch_step<SPLIT>(s, a, x, b, LastEpilogue<T>{step, a.scale / X_SCALE, (T *)a.out, a.ldo, a.so});
        uint16_t *t = xh; xh = yh; yh = t;
        t = xl; xl = yl; yl = t;
    }
}

void launch_orth(hipStream_t s, const OrthArgs &a, void *work)
{
    if (a.bf16) orth_of<uint16_t>(s, a, (char *)work); else orth_of<float>(s, a, (char *)work);
}

}  // namespace netmax
