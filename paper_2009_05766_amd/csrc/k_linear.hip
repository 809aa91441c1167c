// y = act(x w + b) + r for a batch of layers, and its gradients:
//     dz = dy act'(z),  dx = dz w^T,  dw = x^T dz,  db = sum over the rows of dz.
// bfloat16 is multiplied as it is (gemm16.h); operands whose rows that cannot take where they lie are laid out anew first.  float is multiplied in
// float (gemm_f32.h) or, in products large enough to pay for the planes, as planes of halves.
#include "gemm_f32.h"
#include "half_planes.h"
#include "linear.h"

namespace netmax {

static inline int64_t round_up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

// ---- operands of 16 bits laid out anew -------------------------------------------------------------------------------

// One matrix [batch][rows][cols] (rows ld, matrices step apart) that goes to [batch][rows][wide] with zeros behind each row; wide a multiple of 8.
struct Layout { int64_t batch, rows, cols, wide, ld, step; const uint16_t *in; uint16_t *out; };
constexpr int MOST_LAYOUTS = 3;
struct Layouts { int n; Layout of[MOST_LAYOUTS]; uint32_t end[MOST_LAYOUTS]; };     // end: workgroups up to and with each

// All matrices that a call lays out anew in one launch.
__global__ void __launch_bounds__(256) lay_out_kernel(Layouts l)
{
    int k = 0;
    while (k + 1 < l.n && blockIdx.x >= l.end[k]) ++k;
    const Layout m = k == 0 ? l.of[0] : k == 1 ? l.of[1] : l.of[2];
    const uint32_t before = k == 0 ? 0 : l.end[k - 1], here = l.end[k] - before;
    const int64_t units = m.wide / 8, all = m.batch * m.rows * units;
    for (int64_t q = (int64_t)(blockIdx.x - before) * 256 + threadIdx.x; q < all; q += (int64_t)here * 256) {
        // in 32 bits where they do: a division in 64 takes longer than the copy
        const int64_t row = all < (int64_t)1 << 32 ? (uint32_t)q / (uint32_t)units : q / units, g = m.batch == 1 ? 0 : row / m.rows, c = (q - row * units) * 8;
        const uint16_t *p = m.in + g * m.step + (row - g * m.rows) * m.ld + c;
        u32x4 u;
        if (c + 8 <= m.cols) {
            u = *reinterpret_cast<const u32x4_any *>(p);
        } else {
            uint32_t v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = c + e < m.cols ? p[e] : 0u;
            u = u32x4{v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16};
        }
        *reinterpret_cast<u32x4 *>(m.out + q * 8) = u;
    }
}

// A matrix [rows][cols] of a batch as an operand; `copy`: it has to be laid out anew.
struct Source {
    const void *p; int64_t ld, step, rows, cols; bool copy;
    Source(const void *p_, int64_t ld_, int64_t step_, int64_t rows_, int64_t cols_) : p(p_), ld(ld_), step(step_), rows(rows_), cols(cols_), copy(!fits16(p_, ld_, step_, cols_)) { }
    int64_t bytes(int64_t batch) const { return copy ? round_up((step || batch == 0 ? batch : 1) * rows * round_up(cols, 8) * 2, 256) : 0; }
    // The operand; where a copy is needed, in `work` (advanced), and noted in `l`.
    Planes16 take(int64_t batch, char *&work, Layouts &l) const
    {
        if (!copy || rows == 0) return Planes16{(const char *)p, nullptr, ld, step};
        const int64_t wide = round_up(cols, 8), own = step ? batch : 1, want = (own * rows * wide / 8 + 255) / 256;
        char *to = work;
        work += bytes(batch);
        l.of[l.n] = Layout{own, rows, cols, wide, ld, step, (const uint16_t *)p, (uint16_t *)to};
        l.end[l.n] = (l.n ? l.end[l.n - 1] : 0) + (uint32_t)(want < 4096 ? want : 4096);
        ++l.n;
        return Planes16{to, nullptr, wide, step ? rows * wide : 0};
    }
};
static void lay_out(hipStream_t s, const Layouts &l)
{
    if (l.n) lay_out_kernel<<<l.end[l.n - 1], 256, 0, s>>>(l);
}

// ---- products whose contraction is shared out ------------------------------------------------------------------------

// Partial results of one share of the contraction: [splits][batch][M][wide], float.
struct PartEpilogue {
    int64_t M, N, wide; float *p;
    __device__ __forceinline__ int64_t rows_here() const { return M; }
    __device__ __forceinline__ int64_t cols_here() const { return N; }
    struct Columns { };
    struct Seen { };
    template <bool FULL> __device__ __forceinline__ Columns columns(int64_t, int64_t) const { return Columns{}; }
    template <bool FULL> __device__ __forceinline__ Seen see(int64_t, int64_t, int64_t) const { return Seen{}; }
    template <bool FULL> __device__ __forceinline__ void leave(int64_t g, int64_t m, int64_t n, f32x4 v, const Columns &, const Seen &) const
    {
        if (FULL || (m < M && n < N)) store4(p + (g * M + m) * wide + n, v);
    }
};

// The partial results added up in order, then the epilogue.
template <class Epilogue>
__global__ void __launch_bounds__(256) join_parts_kernel(int64_t batch, int64_t M, int64_t wide, int splits, const float *__restrict__ parts, Epilogue epilogue)
{
    const int64_t quads = wide / 4, all = batch * M * quads;
    for (int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x; q < all; q += (int64_t)gridDim.x * 256) {
        f32x4 v = load4(parts + q * 4);
        for (int k = 1; k < splits; ++k) v += load4(parts + ((int64_t)k * all + q) * 4);
        const int64_t row = q / quads, g = row / M;
        epilogue(g, row - g * M, (q - row * quads) * 4, v);
    }
}

// Blocks and shares of a product: large blocks where they fill the card, smaller ones otherwise, and the contraction shared out where even those are few
// and long: a share is at least 16 steps (about 8 us, what the join costs; 1111 x 777 x 2049 in two shares of 64 x 64 blocks took 16 + 8 us, in one 17).
struct Plan16 { int block; int splits; };
static Plan16 plan16(int64_t batch, int64_t M, int64_t N, int64_t K)
{
    const auto blocks = [&](int64_t b) { return batch * ((M + b - 1) / b) * ((N + b - 1) / b); };
    const int64_t steps = (K + 63) / 64;
    if (blocks(256) >= 192 && worth_blocks(256, M, N)) return {256, 1};
    const int block = blocks(128) >= 96 && worth_blocks(128, M, N) ? 128 : 64;
    const int64_t here = blocks(block) > 0 ? blocks(block) : 1, want = 256 / here, most = steps / 16;
    const int64_t splits = want < most ? want : most;
    return {block, (int)(splits < 1 ? 1 : splits > 32 ? 32 : splits)};
}
// Few rows that lie along the contraction have a kernel of their own (few_rows_kernel).
constexpr int64_t FEW_ROWS = 64;
static int64_t part_bytes(int64_t batch, int64_t M, int64_t N, int64_t K, bool ak)
{
    if (M <= FEW_ROWS && ak) return 0;
    const Plan16 p = plan16(batch, M, N, K);
    return p.splits > 1 ? round_up(p.splits * batch * M * round_up(N, 4) * 4, 256) : 0;
}

template <class Epilogue>
static void launch_blocks16(hipStream_t s, int block, int64_t batch, int64_t M, int64_t N, int64_t K, const Planes16 &a, bool ak, const Planes16 &b, bool bk, int splits,
                            const Epilogue &e)
{
    const int64_t blocks = batch * ((M + block - 1) / block) * ((N + block - 1) / block) * splits;
    if (block == 256) launch_gemm16_blocks<bf16x8, 256, 256, 2, 4, 64, 2, 1, false>(s, batch, M, N, K, a, ak, b, bk, splits, e);
    else if (block == 128 && blocks >= 512) launch_gemm16_blocks<bf16x8, 128, 128, 2, 2, 64, 2, 1, false>(s, batch, M, N, K, a, ak, b, bk, splits, e);
    else if (block == 128) launch_gemm16_blocks<bf16x8, 128, 128, 2, 4, 64, 4, 1, false>(s, batch, M, N, K, a, ak, b, bk, splits, e);
    else if (blocks > 256 || K < 512 * splits) launch_gemm16_blocks<bf16x8, 64, 64, 2, 2, 64, 4, 1, false>(s, batch, M, N, K, a, ak, b, bk, splits, e);
    else launch_gemm16_blocks<bf16x8, 64, 64, 2, 2, 64, 4, 2, false>(s, batch, M, N, K, a, ak, b, bk, splits, e);
}

// `work`: part_bytes() of it.
template <class Epilogue>
static void launch_product16(hipStream_t s, int64_t batch, int64_t M, int64_t N, int64_t K, const Planes16 &a, bool ak, const Planes16 &b, bool bk, const Epilogue &e, char *work)
{
    if (M <= FEW_ROWS && ak) {
        launch_few_rows<bf16x8>(s, batch, M, N, K, a, b, bk, e);
        return;
    }
    const Plan16 p = plan16(batch, M, N, K);
    if (p.splits == 1) {
        launch_blocks16(s, p.block, batch, M, N, K, a, ak, b, bk, 1, e);
        return;
    }
    const int64_t wide = round_up(N, 4), quads = batch * M * wide / 4;
    launch_blocks16(s, p.block, batch, M, N, K, a, ak, b, bk, p.splits, PartEpilogue{M, N, wide, (float *)work});
    join_parts_kernel<<<(uint32_t)((quads + 255) / 256 < 2048 ? (quads + 255) / 256 : 2048), 256, 0, s>>>(batch, M, wide, p.splits, (const float *)work, e);
}

// ---- float operands as planes of halves ------------------------------------------------------------------------------
//
// Every row of results (column, for the right operand) has a power of two of its own that brings its largest operand value to 2^14 .. 2^15, so that an
// operand's error is 2^-39 of the largest value that meets it or 2^-22 of itself, whichever is more, and a row of small values is as exact as
// any other.  The three products of planes are then as exact as float ones and take a third of the matrix instructions' time of
// 16-bit products instead of sixteen times that.  Infinities and NaNs stay what they are, reach their own rows and columns only, and do
// not count for the power.

__device__ __forceinline__ float finite_size(float v) { const float a = fabsf(v); return a < INFINITY ? a : 0.0f; }
// The power for a largest value: 0 for a row of zeros.
__device__ __forceinline__ int power_for(float most) { return most > 0.0f ? 15 - (most < 0x1p-126f ? -125 : __builtin_amdgcn_frexp_expf(most)) : 0; }
__device__ __forceinline__ f32x4 scaled(f32x4 v, int power)
{
    return f32x4{ldexpf(v[0], power), ldexpf(v[1], power), ldexpf(v[2], power), ldexpf(v[3], power)};
}
// An infinity has no low plane (inf - inf).
__device__ __forceinline__ void store_split(uint16_t *hi, uint16_t *lo, f32x4 v)
{
    uint32_t h[4], l[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const TwoHalves t(v[e]);
        h[e] = half_bits(t.hi);
        l[e] = fabsf(v[e]) < INFINITY ? half_bits(t.lo) : 0u;
    }
    *reinterpret_cast<uint2 *>(hi) = make_uint2(h[0] | h[1] << 16, h[2] | h[3] << 16);
    *reinterpret_cast<uint2 *>(lo) = make_uint2(l[0] | l[1] << 16, l[2] | l[3] << 16);
}

// [batch][rows][cols] with a power for each row; planes [batch][rows][wide], zeros behind each row; a wave per row at a time.
__global__ void __launch_bounds__(256)
split_rows_kernel(int64_t all_rows, int64_t rows, int64_t cols, int64_t wide, const float *__restrict__ in, int64_t ld, int64_t step, uint16_t *__restrict__ hi,
                  uint16_t *__restrict__ lo, int *__restrict__ powers)
{
    const int lane = threadIdx.x & 63;
    for (int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); row < all_rows; row += (int64_t)gridDim.x * 4) {
        const int64_t g = row / rows;
        const float *p = in + g * step + (row - g * rows) * ld;
        float most = 0.0f;
#pragma unroll 4
        for (int64_t c = lane * 4; c < cols; c += 256) {
            const f32x4 v = load_up_to_four(p, c, cols);
            most = fmaxf(fmaxf(most, fmaxf(finite_size(v[0]), finite_size(v[1]))), fmaxf(finite_size(v[2]), finite_size(v[3])));
        }
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) most = fmaxf(most, __shfl_xor(most, d));
        const int power = power_for(most);
        if (lane == 0) powers[row] = -power;
#pragma unroll 4
        for (int64_t c = lane * 4; c < wide; c += 256) store_split(hi + row * wide + c, lo + row * wide + c, scaled(load_up_to_four(p, c, cols), power));
    }
}

// The largest values of the columns in runs of `run` rows: [batch][runs][cols].  A workgroup has 256 columns, a wave every fourth row.
__global__ void __launch_bounds__(256)
column_sizes_kernel(int64_t rows, int64_t cols, int64_t run, const float *__restrict__ in, int64_t ld, int64_t step, float *__restrict__ sizes)
{
    __shared__ __align__(16) float part[4][256];
    const int wave = threadIdx.x >> 6, at = (threadIdx.x & 63) * 4;
    const int64_t g = blockIdx.z, n = (int64_t)blockIdx.x * 256 + at, end = (int64_t)(blockIdx.y + 1) * run < rows ? (int64_t)(blockIdx.y + 1) * run : rows;
    f32x4 most = {0, 0, 0, 0};
    if (n < cols)
#pragma unroll 4
        for (int64_t r = (int64_t)blockIdx.y * run + wave; r < end; r += 4) {
            const f32x4 v = load_up_to_four(in + g * step + r * ld, n, cols);
#pragma unroll
            for (int e = 0; e < 4; ++e) most[e] = fmaxf(most[e], finite_size(v[e]));
        }
    store4(&part[wave][at], most);
    __syncthreads();
    const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (c < cols)
        sizes[(g * gridDim.y + blockIdx.y) * cols + c] = fmaxf(fmaxf(part[0][threadIdx.x], part[1][threadIdx.x]), fmaxf(part[2][threadIdx.x], part[3][threadIdx.x]));
}

// [batch][rows][cols] with a power for each column, from the sizes of its runs.
__global__ void __launch_bounds__(256)
split_columns_kernel(int64_t rows, int64_t cols, int64_t wide, int run, int runs, const float *__restrict__ in, int64_t ld, int64_t step, const float *__restrict__ sizes,
                     uint16_t *__restrict__ hi, uint16_t *__restrict__ lo, int *__restrict__ powers)
{
    const int wave = threadIdx.x >> 6;
    const int64_t g = blockIdx.z, n = (int64_t)blockIdx.x * 256 + (threadIdx.x & 63) * 4, r0 = (int64_t)blockIdx.y * run;
    if (n >= wide) return;
    f32x4 most = {0, 0, 0, 0};
#pragma unroll 4
    for (int k = 0; k < runs; ++k) {
        const f32x4 v = load_up_to_four(sizes + (g * runs + k) * cols, n, cols);
#pragma unroll
        for (int e = 0; e < 4; ++e) most[e] = fmaxf(most[e], v[e]);
    }
    int power[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        power[e] = power_for(most[e]);
        if (blockIdx.y == 0 && wave == 0 && n + e < cols) powers[g * cols + n + e] = -power[e];
    }
#pragma unroll 4
    for (int64_t r = r0 + wave; r < r0 + run && r < rows; r += 4) {
        const f32x4 v = load_up_to_four(in + g * step + r * ld, n, cols);
        const int64_t at = (g * rows + r) * wide + n;
        store_split(hi + at, lo + at, f32x4{ldexpf(v[0], power[0]), ldexpf(v[1], power[1]), ldexpf(v[2], power[2]), ldexpf(v[3], power[3])});
    }
}

// The powers taken back, then another epilogue.
template <class Inner> struct PowerEpilogue {
    Inner inner; const int *by_row, *by_column; int64_t M, N, sr, sc;
    __device__ __forceinline__ int64_t rows_here() const { return M; }
    __device__ __forceinline__ int64_t cols_here() const { return N; }
    struct Columns { int power[4]; typename Inner::Columns inner; };
    struct Seen { int power; typename Inner::Seen inner; };
    template <bool FULL> __device__ __forceinline__ Columns columns(int64_t g, int64_t n) const
    {
        Columns c{{0, 0, 0, 0}, inner.template columns<FULL>(g, n)};
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (FULL || n + e < N) c.power[e] = by_column[g * sc + n + e];
        return c;
    }
    template <bool FULL> __device__ __forceinline__ Seen see(int64_t g, int64_t m, int64_t n) const
    {
        return Seen{FULL || m < M ? by_row[g * sr + m] : 0, inner.template see<FULL>(g, m, n)};
    }
    template <bool FULL> __device__ __forceinline__ void leave(int64_t g, int64_t m, int64_t n, f32x4 v, const Columns &c, const Seen &s) const
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = ldexpf(v[e], s.power + c.power[e]);
        inner.template leave<FULL>(g, m, n, v, c.inner, s.inner);
    }
};

// Whether a float product is multiplied as planes: where the time that it saves (100 against 300 TFLOP/s) is several times what planes take (reading
// an operand two or three times and writing it once, and up to five launches).  4096 x 4096 x 4096: 1.37 ms in float, 0.52 ms as planes; 1200 x 1000 x 1100: 45
// and 57 us.
static bool as_planes(int64_t batch, int64_t M, int64_t N, int64_t K) { return M * N >= 256 * (M + N) && (double)batch * M * N * K >= 2.5e9; }

// A float matrix [rows][cols] of a batch as planes, with a power for each row (`near`: the contraction runs along the rows) or each column.
struct FloatSource {
    const void *p; int64_t ld, step, rows, cols; bool near;
    int64_t own(int64_t batch) const { return step ? batch : 1; }
    int64_t runs() const { return rows < 2048 ? (rows + 63) / 64 : 32; }
    int64_t plane_bytes(int64_t batch) const { return round_up(own(batch) * rows * round_up(cols, 8) * 2, 256); }
    int64_t power_bytes(int64_t batch) const { return round_up(own(batch) * (near ? rows : cols) * 4, 256); }
    int64_t size_bytes(int64_t batch) const { return near ? 0 : round_up(own(batch) * runs() * cols * 4, 256); }
    int64_t bytes(int64_t batch) const { return 2 * plane_bytes(batch) + power_bytes(batch) + size_bytes(batch); }
    Planes16 take(hipStream_t s, int64_t batch, char *work, const int *&powers, int64_t &between) const
    {
        const int64_t wide = round_up(cols, 8), all = own(batch) * rows;
        uint16_t *hi = (uint16_t *)work, *lo = (uint16_t *)(work + plane_bytes(batch));
        int *to = (int *)(work + 2 * plane_bytes(batch));
        float *sizes = (float *)(work + 2 * plane_bytes(batch) + power_bytes(batch));
        powers = to;
        between = step ? (near ? rows : cols) : 0;
        if (near) {
            split_rows_kernel<<<(uint32_t)(all < 1 << 20 ? (all + 3) / 4 : 1 << 18), 256, 0, s>>>(all, rows, cols, wide, (const float *)p, ld, step, hi, lo, to);
        } else {
            const int64_t run = round_up((rows + runs() - 1) / runs(), 4), each = rows < 4096 ? 16 : 64;     // rows of a workgroup: few leave compute units without work
            const uint32_t across = (uint32_t)((wide + 255) / 256), n = (uint32_t)((rows + run - 1) / run);
            column_sizes_kernel<<<dim3(across, n, (uint32_t)own(batch)), 256, 0, s>>>(rows, cols, run, (const float *)p, ld, step, sizes);
            split_columns_kernel<<<dim3(across, (uint32_t)((rows + each - 1) / each), (uint32_t)own(batch)), 256, 0, s>>>(rows, cols, wide, (int)each, (int)n, (const float *)p, ld, step, sizes,
                                                                                                              hi, lo, to);
        }
        return Planes16{(const char *)hi, (const char *)lo, wide, step ? rows * wide : 0};
    }
};

// C = A B of float operands; `work`: product32_bytes() of it.
static int64_t product32_bytes(int64_t batch, int64_t M, int64_t N, int64_t K, const FloatSource &a, const FloatSource &b)
{
    return as_planes(batch, M, N, K) ? a.bytes(batch) + b.bytes(batch) : 0;
}
template <class Epilogue>
static void launch_product32(hipStream_t s, int64_t batch, int64_t M, int64_t N, int64_t K, const FloatSource &a, const FloatSource &b, const Epilogue &e, char *work)
{
    if (!as_planes(batch, M, N, K)) {
        launch_gemm_f32<float>(s, batch, M, N, K, Operand{a.p, a.ld, a.step, a.near}, Operand{b.p, b.ld, b.step, b.near}, e);
        return;
    }
    PowerEpilogue<Epilogue> powers{e, nullptr, nullptr, M, N, 0, 0};
    const Planes16 pa = a.take(s, batch, work, powers.by_row, powers.sr), pb = b.take(s, batch, work + a.bytes(batch), powers.by_column, powers.sc);
    with_small_shape<true>(M, N, K, [&](int64_t n) { return batch * ((M + n - 1) / n) * ((N + n - 1) / n); }, [&](auto f) {
        launch_gemm16_blocks<half8, f.BM, f.BN, f.WM, f.WN, f.STEP, f.STAGES, f.GROUPS, true>(s, batch, M, N, K, pa, a.near, pb, b.near, 1, powers);
    });
}

// out [rows][cols] alone
template <typename T> static LinearEpilogue<T> plain_epilogue(int64_t rows, int64_t cols, void *out, int64_t ld, int64_t step)
{
    return LinearEpilogue<T>{rows, cols, nullptr, nullptr, (T *)out, nullptr, 0, ld, 0, 0, 0, step, 0, ACT_NONE};
}

// ---- db --------------------------------------------------------------------------------------------------------------

// Column sums of dz from those of runs of rows: 64 columns per workgroup; four waves take the runs in turn, then their sums are added in order.
template <typename T> struct BiasSum {
    int64_t batch, cols, parts; const float *sums; T *db; int64_t sdb;
    __host__ __device__ uint32_t across() const { return (uint32_t)((cols + 63) / 64); }
    uint32_t blocks() const { return db ? (uint32_t)batch * across() : 0; }
    __device__ __forceinline__ void operator()(uint32_t id, float *space) const
    {
        const int wave = threadIdx.x >> 6, at = threadIdx.x & 63;
        const int64_t g = id / across(), n = (int64_t)(id % across()) * 64 + at;
        if (wave < 4) {
            float sum = 0.0f;
            if (n < cols)
#pragma unroll 8
                for (int64_t k = wave; k < parts; k += 4) sum += sums[(g * parts + k) * cols + n];
            space[wave * 64 + at] = sum;
        }
        __syncthreads();
        if (wave == 0 && n < cols) store_value(db + g * sdb + n, (space[at] + space[64 + at]) + (space[128 + at] + space[192 + at]));
    }
};
template <typename T> __global__ void __launch_bounds__(256) bias_sum_kernel(BiasSum<T> b)
{
    __shared__ float space[256];
    b(blockIdx.x, space);
}

// ---- dx and dw in one launch -----------------------------------------------------------------------------------------

// Whether the workgroups of both products and of db, at most, are less than a launch can have.
static bool one_launch(const LinearGradArgs &a)
{
    const auto up = [](int64_t n) { return (n + 63) / 64; };
    return a.batch * (up(a.rows) * up(a.din) + up(a.din) * up(a.dout) + up(a.dout)) < 1 << 24;
}

// dx = d w^T, dw = x^T d and db where neither product would fill the card alone, or false.
static bool launch_pair16(hipStream_t s, const LinearGradArgs &a, const Planes16 &d, const Planes16 &w, const Planes16 &x, const BiasSum<uint16_t> &bias)
{
    if (!one_launch(a)) return false;
    if (a.rows <= FEW_ROWS && a.dout > 1024) return false;         // dx from few_rows_kernel: a long chain of steps otherwise
    const Plan16 px = plan16(a.batch, a.rows, a.din, a.dout), pw = plan16(a.batch, a.din, a.dout, a.rows);
    if (px.block == 256 || pw.block == 256 || px.splits > 1 || pw.splits > 1) return false;
    const auto blocks = [&](int64_t b, int64_t m, int64_t n) { return a.batch * ((m + b - 1) / b) * ((n + b - 1) / b); };
    const auto both = [&](int64_t b) { return blocks(b, a.rows, a.din) + blocks(b, a.din, a.dout); };
    const int swap = a.rows > a.dout;                               // the longer chains of steps start first
    const auto go = [&](auto f) {
        const auto product = [&](int64_t M, int64_t N, int64_t K, const Planes16 &l, const Planes16 &r, void *out, int64_t ld, int64_t step) {
            return Product16<LinearEpilogue<uint16_t>>{M, N, K, l, r, (uint32_t)((M + f.BM - 1) / f.BM), (uint32_t)((N + f.BM - 1) / f.BM), plain_epilogue<uint16_t>(M, N, out, ld, step)};
        };
        const uint32_t first = (uint32_t)blocks(f.BM, a.rows, a.din), all = (uint32_t)both(f.BM);
        gemm16_pair_kernel<bf16x8, f.BM, f.WM, f.WN, f.STEP, f.STAGES, f.GROUPS><<<all + bias.blocks(), f.WM * f.WN * 64 * f.GROUPS, 0, s>>>(
            product(a.rows, a.din, a.dout, d, w, a.dx, a.lddx, a.sdx), product(a.din, a.dout, a.rows, x, d, a.dw, a.lddw, a.sdw), first, all, swap, bias);
    };
    const bool far = worth_blocks(128, a.rows, a.din) && worth_blocks(128, a.din, a.dout);
    if (both(128) >= 512 && far) go(Shape<128, 128, 2, 2, 64, 2>());
    else if (both(128) >= 128 && far) go(Shape<128, 128, 2, 4, 64, 4>());
    else if (both(64) > 256 || (a.dout < 512 && a.rows < 512)) go(Shape<64, 64, 2, 2, 64, 4>());
    else go(Shape<64, 64, 2, 2, 64, 4, 2>());
    return true;
}

static bool launch_pair32(hipStream_t s, const LinearGradArgs &a, const void *d, int64_t ldd, int64_t sd, const BiasSum<float> &bias)
{
    if (!one_launch(a)) return false;
    const auto blocks = [&](int64_t b, int64_t m, int64_t n) { return a.batch * ((m + b - 1) / b) * ((n + b - 1) / b); };
    if (as_planes(a.batch, a.rows, a.din, a.dout) || as_planes(a.batch, a.din, a.dout, a.rows)) return false;
    if ((blocks(128, a.rows, a.din) >= 256 && a.dout >= 256 && worth_blocks(128, a.rows, a.din)) ||
        (blocks(128, a.din, a.dout) >= 256 && a.rows >= 256 && worth_blocks(128, a.din, a.dout))) return false;
    const auto product = [&](int64_t M, int64_t N, int64_t K, const void *l, int64_t ldl, int64_t sl, const void *r, int64_t ldr, int64_t sr, void *out, int64_t ld, int64_t step) {
        return ProductF32<LinearEpilogue<float>>{M, N, K, (const float *)l, (const float *)r, ldl, sl, ldr, sr, (uint32_t)((M + 63) / 64), (uint32_t)((N + 63) / 64),
                                                 plain_epilogue<float>(M, N, out, ld, step)};
    };
    const auto p = product(a.rows, a.din, a.dout, d, ldd, sd, a.w, a.ldw, a.sw, a.dx, a.lddx, a.sdx);
    const auto q = product(a.din, a.dout, a.rows, a.x, a.ldx, a.sx, d, ldd, sd, a.dw, a.lddw, a.sdw);
    const int swap = a.rows > a.dout;
    const uint32_t first = (uint32_t)blocks(64, a.rows, a.din), all = first + (uint32_t)blocks(64, a.din, a.dout);
    if (all >= 768) gemm_f32_pair_kernel<64, 32, 1><<<all + bias.blocks(), 256, 0, s>>>(p, q, first, all, swap, bias);
    else if (all >= 384) gemm_f32_pair_kernel<64, 32, 2><<<all + bias.blocks(), 512, 0, s>>>(p, q, first, all, swap, bias);
    else gemm_f32_pair_kernel<64, 32, 4><<<all + bias.blocks(), 1024, 0, s>>>(p, q, first, all, swap, bias);
    return true;
}

// ---- dz and db -------------------------------------------------------------------------------------------------------

// A workgroup takes `run` rows of SLOPE_COLS columns, a wave every fourth row, a lane 16 bytes: dz, and the column sums of dz (before its rounding) over
// these rows, in float, in a fixed order.  Bound by memory, dy and z in, dz out, and close behind by GELU's slope: 8192 x 8192 100 us (4.0 TB/s).
template <typename T> constexpr int SLOPE_COLS = 1024 / sizeof(T);

// 16 bytes from column n of `cols` as floats, 0 behind the last; and back.
template <typename T> __device__ __forceinline__ void load_16_bytes(const T *row, int64_t n, int64_t cols, float (&v)[16 / sizeof(T)])
{
    if constexpr (sizeof(T) == 4) {
        const f32x4 x = load_up_to_four(row, n, cols);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = x[e];
    } else if (n + 8 <= cols) {
        const u32x4 x = *reinterpret_cast<const u32x4_any *>(row + n);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(e & 1 ? x[e >> 1] & 0xFFFF0000u : x[e >> 1] << 16);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = n + e < cols ? load_value(row + n + e) : 0.0f;
    }
}
template <typename T> __device__ __forceinline__ void store_16_bytes(T *row, int64_t n, int64_t cols, const float (&v)[16 / sizeof(T)])
{
    if constexpr (sizeof(T) == 4) store_up_to_four(row, n, cols, f32x4{v[0], v[1], v[2], v[3]});
    else if (n + 8 <= cols)
        *reinterpret_cast<u32x4_any *>(row + n) = u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
    else
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (n + e < cols) store_value(row + n + e, v[e]);
}

template <typename T>
__global__ void __launch_bounds__(256)
slope_kernel(int64_t rows, int64_t cols, int run, const T *__restrict__ dy, int64_t lddy, int64_t sdy, const T *__restrict__ z, int64_t ldz, int64_t sz, int act,
             T *__restrict__ dz, int64_t wide, float *__restrict__ sums)
{
    // dz has rows of `wide` values, zeros behind the columns: what the product's contraction over them needs
    constexpr int VALUES = 16 / sizeof(T), COLS = SLOPE_COLS<T>;
    __shared__ __align__(16) float part[4][COLS];
    const int wave = threadIdx.x >> 6, at = (threadIdx.x & 63) * VALUES;
    const int64_t g = blockIdx.z, n = (int64_t)blockIdx.x * COLS + at, r0 = (int64_t)blockIdx.y * run + wave;
    const int64_t end = (int64_t)(blockIdx.y + 1) * run < rows ? (int64_t)(blockIdx.y + 1) * run : rows;
    dy += g * sdy;
    z += g * sz;
    float sum[VALUES] = {};
    if (n < wide)
#pragma unroll 4
        for (int64_t r = r0; r < end; r += 4) {
            float v[VALUES];
            load_16_bytes(dy + r * lddy, n, cols, v);
            if (act != ACT_NONE) {
                float pre[VALUES];
                load_16_bytes(z + r * ldz, n, cols, pre);
#pragma unroll
                for (int e = 0; e < VALUES; ++e) v[e] = n + e < cols ? v[e] * act_slope(act, pre[e]) : 0.0f;
            }
#pragma unroll
            for (int e = 0; e < VALUES; ++e) sum[e] += v[e];
            if (dz) store_16_bytes(dz + (g * rows + r) * wide, n, wide, v);
        }
    if (!sums) return;
#pragma unroll
    for (int e = 0; e < VALUES; ++e) part[wave][at + e] = sum[e];
    __syncthreads();
    for (int c = threadIdx.x; c < COLS && (int64_t)blockIdx.x * COLS + c < cols; c += 256)
        sums[((int64_t)g * gridDim.y + blockIdx.y) * cols + (int64_t)blockIdx.x * COLS + c] = (part[0][c] + part[1][c]) + (part[2][c] + part[3][c]);
}

// ---- launchers -------------------------------------------------------------------------------------------------------

template <typename T> static LinearEpilogue<T> forward_epilogue(const LinearArgs &a)
{
    return LinearEpilogue<T>{a.rows, a.dout, (const T *)a.bias, (const T *)a.residual, (T *)a.y, (T *)a.z, a.ldr, a.ldy, a.ldz, a.sb, a.sr, a.sy, a.sz, a.act};
}
static FloatSource float_source(const void *p, int64_t ld, int64_t step, int64_t rows, int64_t cols, bool near) { return FloatSource{p, ld, step, rows, cols, near}; }

int64_t linear_workspace(const LinearArgs &a)
{
    if (!a.bf16)
        return product32_bytes(a.batch, a.rows, a.dout, a.din, float_source(a.x, a.ldx, a.sx, a.rows, a.din, true), float_source(a.w, a.ldw, a.sw, a.din, a.dout, false));
    return Source(a.x, a.ldx, a.sx, a.rows, a.din).bytes(a.batch) + Source(a.w, a.ldw, a.sw, a.din, a.dout).bytes(a.batch) + part_bytes(a.batch, a.rows, a.dout, a.din, true);
}

void launch_linear(hipStream_t s, const LinearArgs &a, void *work)
{
    if (!a.bf16) {
        launch_product32(s, a.batch, a.rows, a.dout, a.din, float_source(a.x, a.ldx, a.sx, a.rows, a.din, true), float_source(a.w, a.ldw, a.sw, a.din, a.dout, false),
                         forward_epilogue<float>(a), (char *)work);
        return;
    }
    char *at = (char *)work;
    Layouts l{};
    const Planes16 x = Source(a.x, a.ldx, a.sx, a.rows, a.din).take(a.batch, at, l), w = Source(a.w, a.ldw, a.sw, a.din, a.dout).take(a.batch, at, l);
    lay_out(s, l);
    launch_product16(s, a.batch, a.rows, a.dout, a.din, x, true, w, false, forward_epilogue<uint16_t>(a), at);
}

static int64_t dz_wide(const LinearGradArgs &a) { return a.bf16 ? round_up(a.dout, 8) : a.dout; }
// Rows of a workgroup of slope_kernel: 64, or fewer where that leaves compute units without work (at 1111 x 2049, rows at odd places, 64: 35 us).
static int slope_run(const LinearGradArgs &a)
{
    const int64_t across = a.batch * ((dz_wide(a) + 255) / 256);
    int run = 64;
    while (run > 8 && across * ((a.rows + run - 1) / run) < 1024) run /= 2;
    return run;
}
static int64_t sum_parts(const LinearGradArgs &a) { return (a.rows + slope_run(a) - 1) / slope_run(a); }
static int64_t sum_bytes(const LinearGradArgs &a) { return round_up(a.batch * sum_parts(a) * a.dout * 4, 256); }

int64_t linear_grad_workspace(const LinearGradArgs &a)
{
    int64_t n = sum_bytes(a);
    if (a.act != ACT_NONE) n += round_up(a.batch * a.rows * dz_wide(a) * (a.bf16 ? 2 : 4), 256);
    else if (a.bf16) n += Source(a.dy, a.lddy, a.sdy, a.rows, a.dout).bytes(a.batch);
    if (!a.bf16) {
        // dz (or dy) lies in rows of dout either way; the two products use the same memory in turn
        const int64_t sd = a.batch > 1 ? 1 : 0;
        const int64_t dx = product32_bytes(a.batch, a.rows, a.din, a.dout, float_source(nullptr, 0, sd, a.rows, a.dout, true), float_source(a.w, a.ldw, a.sw, a.din, a.dout, true));
        const int64_t dw = product32_bytes(a.batch, a.din, a.dout, a.rows, float_source(a.x, a.ldx, a.sx, a.rows, a.din, false), float_source(nullptr, 0, sd, a.rows, a.dout, false));
        return n + (dx > dw ? dx : dw);
    }
    const int64_t dx = part_bytes(a.batch, a.rows, a.din, a.dout, true), dw = part_bytes(a.batch, a.din, a.dout, a.rows, false);
    return n + Source(a.x, a.ldx, a.sx, a.rows, a.din).bytes(a.batch) + Source(a.w, a.ldw, a.sw, a.din, a.dout).bytes(a.batch) + (dx > dw ? dx : dw);
}

template <typename T> static void launch_bias(hipStream_t s, const BiasSum<T> &b)
{
    if (b.blocks()) bias_sum_kernel<T><<<b.blocks(), 256, 0, s>>>(b);
}

// dz, and what is left to do for db.
template <typename T> static BiasSum<T> launch_slopes(hipStream_t s, const LinearGradArgs &a, T *dz, float *sums)
{
    if ((dz || a.db) && a.rows > 0)
        slope_kernel<T><<<dim3((uint32_t)((dz_wide(a) + SLOPE_COLS<T> - 1) / SLOPE_COLS<T>), (uint32_t)sum_parts(a), (uint32_t)a.batch), 256, 0, s>>>(
            a.rows, a.dout, slope_run(a), (const T *)a.dy, a.lddy, a.sdy, (const T *)a.z, a.ldz, a.sz, a.act, dz,
            dz_wide(a), a.db ? sums : nullptr);
    return BiasSum<T>{a.batch, a.dout, sum_parts(a), sums, (T *)a.db, a.sdb};
}

void launch_linear_grad(hipStream_t s, const LinearGradArgs &a, void *work)
{
    char *at = (char *)work;
    float *sums = (float *)at;
    at += sum_bytes(a);
    void *dz = nullptr;
    if (a.act != ACT_NONE) {
        dz = at;
        at += round_up(a.batch * a.rows * dz_wide(a) * (a.bf16 ? 2 : 4), 256);
    }
    if (!a.bf16) {
        const BiasSum<float> bias = launch_slopes<float>(s, a, (float *)dz, sums);
        const void *d = dz ? dz : a.dy;
        const int64_t ldd = dz ? a.dout : a.lddy, sd = dz ? (a.batch > 1 ? a.rows * a.dout : 0) : a.sdy;
        if (a.dx && a.dw && a.rows > 0 && launch_pair32(s, a, d, ldd, sd, bias)) return;
        launch_bias(s, bias);
        if (a.dx && a.rows > 0)
            launch_product32(s, a.batch, a.rows, a.din, a.dout, float_source(d, ldd, sd, a.rows, a.dout, true), float_source(a.w, a.ldw, a.sw, a.din, a.dout, true),
                             plain_epilogue<float>(a.rows, a.din, a.dx, a.lddx, a.sdx), at);
        if (a.dw)
            launch_product32(s, a.batch, a.din, a.dout, a.rows, float_source(a.x, a.ldx, a.sx, a.rows, a.din, false), float_source(d, ldd, sd, a.rows, a.dout, false),
                             plain_epilogue<float>(a.din, a.dout, a.dw, a.lddw, a.sdw), at);
        return;
    }
    const BiasSum<uint16_t> bias = launch_slopes<uint16_t>(s, a, (uint16_t *)dz, sums);
    Layouts l{};
    const Planes16 d = dz ? Planes16{(const char *)dz, nullptr, dz_wide(a), a.rows * dz_wide(a)} : Source(a.dy, a.lddy, a.sdy, a.rows, a.dout).take(a.batch, at, l);
    Planes16 w{}, x{};
    if (a.dx && a.rows > 0) w = Source(a.w, a.ldw, a.sw, a.din, a.dout).take(a.batch, at, l);
    if (a.dw) x = Source(a.x, a.ldx, a.sx, a.rows, a.din).take(a.batch, at, l);
    lay_out(s, l);
    if (a.dx && a.dw && a.rows > 0 && launch_pair16(s, a, d, w, x, bias)) return;
    launch_bias(s, bias);
    if (a.dx && a.rows > 0)
        launch_product16(s, a.batch, a.rows, a.din, a.dout, d, true, w, true, plain_epilogue<uint16_t>(a.rows, a.din, a.dx, a.lddx, a.sdx), at);
    if (a.dw)
        launch_product16(s, a.batch, a.din, a.dout, a.rows, x, false, d, false, plain_epilogue<uint16_t>(a.din, a.dout, a.dw, a.lddw, a.sdw), at);
}

}  // namespace netmax
