// y = act(x w + b) + r for a batch of layers, and its gradients:
//     dz = dy act'(z),  dx = dz w^T,  dw = x^T dz,  db = sum over the rows of dz.
// bfloat16 is multiplied as it is (gemm16.h); operands whose rows that cannot take where they lie are laid out anew first.  float is multiplied in
// float (gemm_f32.h) at every size: a row split into 16-bit planes with one power of two for all of it loses its small values beside a large one, and an
// infinity there meets low planes of either sign, so that a result would depend on the size of its layer.
#include "gemm16.h"
#include "gemm_f32.h"
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
//   256 or 128   2816 x 4096 x 2816 (121 large blocks) 89 and 83, 2816 x 4096 x 3328 (143) 86 and 108, 4096 cubed 118 and 143
//   128 or 64    1024 x 1024 x 2048 (128 blocks) 12.3 and 10.7, 1536 x 1024 x 1536 (144) 12.7 and 16.2; with shares 1152 x 4096 x 1152 (81) 24 and 27, 1280 x 8192 x 1280
//                (100) 41 and 55, but 896 x 4096 x 896 (49) 20 and 18
struct Plan16 { int block; int splits; };
static Plan16 plan16(int64_t batch, int64_t M, int64_t N, int64_t K)
{
    const auto blocks = [&](int64_t b) { return batch * ((M + b - 1) / b) * ((N + b - 1) / b); };
    const int64_t steps = (K + 63) / 64;
    if (blocks(256) > 128 && worth_blocks(256, M, N)) return {256, 1};
    const int block = (blocks(128) > 128 || (blocks(128) >= 80 && K >= 4096)) && worth_blocks(128, M, N) ? 128 : 64;
    const int64_t here = blocks(block) > 0 ? blocks(block) : 1, want = 256 / here, most = steps / 16;
    const int64_t splits = want < most ? want : most;
    return {block, (int)(splits < 1 ? 1 : splits > 32 ? 32 : splits)};
}
// Few rows that lie along the contraction have a kernel of their own (few_rows_kernel).  In a graph, 1 x 2048 x 8192: 6.8 us, in blocks with shares 10.2; 32 x 4096 x 4096: 13.9, in blocks 12.6 and a second launch; 64 x 2048 x 2048: 6.8
// and 9.5; long contractions of 64 rows, 64 x 4096 x 4096, are better off in blocks (17.6 and 13.4), which as a call are bound by the host at 14.
constexpr int64_t FEW_ROWS = 64;
static int64_t part_bytes(int64_t batch, int64_t M, int64_t N, int64_t K, bool ak)
{
    if (M <= FEW_ROWS && ak) return 0;
    const Plan16 p = plan16(batch, M, N, K);
    return p.splits > 1 ? round_up(p.splits * batch * M * round_up(N, 4) * 4, 256) : 0;
}

// Blocks of 128 in four waves and two stages, two of them on a compute unit, or in eight waves and four stages, alone there: 2048 cubed (256 blocks) 29.4 and 24.3, 2176 x 2048 x
// 2176 (289) 34.5 and 38.8.  Blocks of 64 in one group or two: 960 x 1024 x 960 (225 blocks) 8.5 and 7.8, 1088 x 1024 x 1088 (289) 10.4 and 13.9; 640 x 512 x 640 6.2 and 6.3, with
// 128 indices 4.5 and 4.9.
template <class Epilogue>
static void launch_blocks16(hipStream_t s, int block, int64_t batch, int64_t M, int64_t N, int64_t K, const Planes16 &a, bool ak, const Planes16 &b, bool bk, const Epilogue &e)
{
    const int64_t blocks = batch * ((M + block - 1) / block) * ((N + block - 1) / block);
    if (block == 256) launch_gemm16_blocks<bf16x8, 256, 256, 2, 4, 64, 2, 1>(s, batch, M, N, K, a, ak, b, bk, 1, e);
    else if (block == 128 && blocks > 256) launch_gemm16_blocks<bf16x8, 128, 128, 2, 2, 64, 2, 1>(s, batch, M, N, K, a, ak, b, bk, 1, e);
    else if (block == 128) launch_gemm16_blocks<bf16x8, 128, 128, 2, 4, 64, 4, 1>(s, batch, M, N, K, a, ak, b, bk, 1, e);
    else if (blocks > 256 || K < 512) launch_gemm16_blocks<bf16x8, 64, 64, 2, 2, 64, 4, 1>(s, batch, M, N, K, a, ak, b, bk, 1, e);
    else launch_gemm16_blocks<bf16x8, 64, 64, 2, 2, 64, 4, 2>(s, batch, M, N, K, a, ak, b, bk, 1, e);
}
// Shares of a contraction: at most 256 workgroups in all, each with 16 steps or more.
static void launch_parts16(hipStream_t s, const Plan16 &p, int64_t batch, int64_t M, int64_t N, int64_t K, const Planes16 &a, bool ak, const Planes16 &b, bool bk, const PartEpilogue &e)
{
    if (p.block == 128) launch_gemm16_blocks<bf16x8, 128, 128, 2, 4, 64, 4, 1>(s, batch, M, N, K, a, ak, b, bk, (uint32_t)p.splits, e);
    else launch_gemm16_blocks<bf16x8, 64, 64, 2, 2, 64, 4, 2>(s, batch, M, N, K, a, ak, b, bk, (uint32_t)p.splits, e);
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
        launch_blocks16(s, p.block, batch, M, N, K, a, ak, b, bk, e);
        return;
    }
    const int64_t wide = round_up(N, 4), quads = batch * M * wide / 4;
    launch_parts16(s, p, batch, M, N, K, a, ak, b, bk, PartEpilogue{M, N, wide, (float *)work});
    join_parts_kernel<<<(uint32_t)((quads + 255) / 256 < 2048 ? (quads + 255) / 256 : 2048), 256, 0, s>>>(batch, M, wide, p.splits, (const float *)work, e);
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
    if (px.splits > 1 || pw.splits > 1) return false;
    const auto blocks = [&](int64_t b, int64_t m, int64_t n) { return a.batch * ((m + b - 1) / b) * ((n + b - 1) / b); };
    // 3328 cubed (169 blocks of 256 in each) in one launch 164, in large blocks one after the other 170; 4096 cubed (256) so 248
    if ((px.block == 256 && blocks(256, a.rows, a.din) >= 192) || (pw.block == 256 && blocks(256, a.din, a.dout) >= 192)) return false;
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
    // as launch_blocks16, by the blocks of both: 1408 cubed (242) 22.4 and 17.9, 1536 cubed (288) 27.4 and 31.2; 128 or 64, 1024 cubed (128) 13.6 and 10.1, 1152 cubed
    // (162) 14.5 and 16.7; blocks of 64 in one group or two, 512 cubed (128) 5.9 and 6.3, 704 cubed (242) 6.9 and 7.4, 768 cubed (288) 8.4 and 12.3
    const bool far = worth_blocks(128, a.rows, a.din) && worth_blocks(128, a.din, a.dout);
    if (both(128) > 256 && far) go(Shape<128, 128, 2, 2, 64, 2>());
    else if (both(128) > 128 && far) go(Shape<128, 128, 2, 4, 64, 4>());
    else if (both(64) > 256 || (a.dout < 512 && a.rows < 512)) go(Shape<64, 64, 2, 2, 64, 4>());
    else go(Shape<64, 64, 2, 2, 64, 4, 2>());
    return true;
}

static bool launch_pair32(hipStream_t s, const LinearGradArgs &a, const void *d, int64_t ldd, int64_t sd, const BiasSum<float> &bias)
{
    if (!one_launch(a)) return false;
    const auto blocks = [&](int64_t b, int64_t m, int64_t n) { return a.batch * ((m + b - 1) / b) * ((n + b - 1) / b); };
    // one after the other where one of them is worth blocks of 128 (4096 cubed 2.24 ms, 2.55 in blocks of 64), or fills the card and the other has few and long chains, which then
    // have more waves each: 16384 x 256 x 256 223 us, in one launch 478; 2048 cubed 352 and 339, 8192 x 512 x 4096 766 and 683
    const auto large = [&](int64_t m, int64_t n, int64_t k, int64_t from) { return blocks(128, m, n) >= from && k >= 256 && worth_blocks(128, m, n); };
    const int64_t dx_from = blocks(64, a.din, a.dout) < 128 ? 256 : F32_LARGE, dw_from = blocks(64, a.rows, a.din) < 128 ? 256 : F32_LARGE;
    if (large(a.rows, a.din, a.dout, dx_from) || large(a.din, a.dout, a.rows, dw_from)) return false;
    const auto product = [&](int64_t M, int64_t N, int64_t K, const void *l, int64_t ldl, int64_t sl, const void *r, int64_t ldr, int64_t sr, void *out, int64_t ld, int64_t step) {
        return ProductF32<LinearEpilogue<float>>{M, N, K, (const float *)l, (const float *)r, ldl, sl, ldr, sr, (uint32_t)((M + 63) / 64), (uint32_t)((N + 63) / 64),
                                                 plain_epilogue<float>(M, N, out, ld, step)};
    };
    const auto p = product(a.rows, a.din, a.dout, d, ldd, sd, a.w, a.ldw, a.sw, a.dx, a.lddx, a.sdx);
    const auto q = product(a.din, a.dout, a.rows, a.x, a.ldx, a.sx, d, ldd, sd, a.dw, a.lddw, a.sdw);
    const int swap = a.rows > a.dout;
    const uint32_t first = (uint32_t)blocks(64, a.rows, a.din), all = first + (uint32_t)blocks(64, a.din, a.dout);
    // one group of waves or two: 960 cubed (450 blocks) 53 and 45 us, 1216 cubed (722) 86 and 85, 1280 cubed (800) 109 in both; two or four: 1400 x 640 x 640 (320) 46 and 39, 832
    // cubed (338) 39 and 48, 600 x 2048 x 64 (352) 20 and 18, 896 cubed (392) 42 and 48
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

int64_t linear_workspace(const LinearArgs &a)
{
    if (!a.bf16) return 0;
    return Source(a.x, a.ldx, a.sx, a.rows, a.din).bytes(a.batch) + Source(a.w, a.ldw, a.sw, a.din, a.dout).bytes(a.batch) + part_bytes(a.batch, a.rows, a.dout, a.din, true);
}

void launch_linear(hipStream_t s, const LinearArgs &a, void *work)
{
    if (!a.bf16) {
        launch_gemm_f32(s, a.batch, a.rows, a.dout, a.din, Operand{a.x, a.ldx, a.sx, true}, Operand{a.w, a.ldw, a.sw, false}, forward_epilogue<float>(a));
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
    if (!a.bf16) return n;
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
            launch_gemm_f32(s, a.batch, a.rows, a.din, a.dout, Operand{d, ldd, sd, true}, Operand{a.w, a.ldw, a.sw, true},
                                   plain_epilogue<float>(a.rows, a.din, a.dx, a.lddx, a.sdx));
        if (a.dw)
            launch_gemm_f32(s, a.batch, a.din, a.dout, a.rows, Operand{a.x, a.ldx, a.sx, false}, Operand{d, ldd, sd, false},
                                   plain_epilogue<float>(a.din, a.dout, a.dw, a.lddw, a.sdw));
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
