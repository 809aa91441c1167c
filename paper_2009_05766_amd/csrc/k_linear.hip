// y = act(x w + b) + r for a batch of layers, and its gradients:
//     dz = dy act'(z),  dx = dz w^T,  dw = x^T dz,  db = sum over the rows of dz.
// float is multiplied in float (gemm_f32.h), bfloat16 as it is (gemm16.h); bfloat16 operands whose rows the latter cannot take where they lie
// are laid out anew first.
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
    __device__ __forceinline__ void operator()(int64_t g, int64_t m, int64_t n, f32x4 v) const
    {
        if (m < M && n < N) store4(p + (g * M + m) * wide + n, v);
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
    if (blocks(256) >= 192) return {256, 1};
    const int block = blocks(128) >= 96 && M > 64 && N > 64 ? 128 : 64;
    const int64_t here = blocks(block) > 0 ? blocks(block) : 1, want = (block == 128 ? 256 : 512) / here, most = steps / 16;
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
    if (block == 256) launch_gemm16_blocks<bf16x8, 256, 256, 2, 4, 64, 2, false>(s, batch, M, N, K, a, ak, b, bk, splits, e);
    else if (block == 128 && blocks >= 512) launch_gemm16_blocks<bf16x8, 128, 128, 2, 2, 64, 2, false>(s, batch, M, N, K, a, ak, b, bk, splits, e);
    else if (block == 128) launch_gemm16_blocks<bf16x8, 128, 128, 2, 4, 64, 4, false>(s, batch, M, N, K, a, ak, b, bk, splits, e);
    else launch_gemm16_blocks<bf16x8, 64, 64, 2, 2, 64, 4, false>(s, batch, M, N, K, a, ak, b, bk, splits, e);
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

// ---- dz and db -------------------------------------------------------------------------------------------------------

// A workgroup takes `run` rows of 256 columns, a wave every fourth row, a lane four columns: dz, and the column sums of dz (before its rounding) over
// these rows, in float, in a fixed order.  Bound by memory: dy and z in, dz out.
constexpr int SLOPE_COLS = 256;

template <typename T>
__global__ void __launch_bounds__(256)
slope_kernel(int64_t rows, int64_t cols, int run, const T *__restrict__ dy, int64_t lddy, int64_t sdy, const T *__restrict__ z, int64_t ldz, int64_t sz, int act,
             T *__restrict__ dz, int64_t wide, float *__restrict__ sums)
{
    // dz has rows of `wide` values, zeros behind the columns: what the product's contraction over them needs
    __shared__ __align__(16) float part[4][SLOPE_COLS];
    const int wave = threadIdx.x >> 6, at = (threadIdx.x & 63) * 4;
    const int64_t g = blockIdx.z, n = (int64_t)blockIdx.x * SLOPE_COLS + at, r0 = (int64_t)blockIdx.y * run + wave;
    const int64_t end = (int64_t)(blockIdx.y + 1) * run < rows ? (int64_t)(blockIdx.y + 1) * run : rows;
    dy += g * sdy;
    z += g * sz;
    f32x4 sum = {0, 0, 0, 0};
    if (n < wide)
#pragma unroll 4
        for (int64_t r = r0; r < end; r += 4) {
            f32x4 v = load_up_to_four(dy + r * lddy, n, cols);
            if (act != ACT_NONE) {
                const f32x4 pre = load_up_to_four(z + r * ldz, n, cols);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = n + e < cols ? v[e] * act_slope(act, pre[e]) : 0.0f;
            }
            sum += v;
            if (dz) store_up_to_four(dz + (g * rows + r) * wide, n, wide, v);
        }
    if (!sums) return;
    store4(&part[wave][at], sum);
    __syncthreads();
    const int64_t col = (int64_t)blockIdx.x * SLOPE_COLS + threadIdx.x;
    if (col < cols)
        sums[((int64_t)g * gridDim.y + blockIdx.y) * cols + col] = (part[0][threadIdx.x] + part[1][threadIdx.x]) + (part[2][threadIdx.x] + part[3][threadIdx.x]);
}

// 64 columns per workgroup; four waves take the parts in turn, then their sums are added in order.
template <typename T>
__global__ void __launch_bounds__(256) bias_sum_kernel(int64_t cols, int64_t parts, const float *__restrict__ sums, T *__restrict__ db, int64_t sdb)
{
    __shared__ float part[4][64];
    const int wave = threadIdx.x >> 6, at = threadIdx.x & 63;
    const int64_t g = blockIdx.y, n = (int64_t)blockIdx.x * 64 + at;
    float sum = 0.0f;
    if (n < cols)
#pragma unroll 8
        for (int64_t k = wave; k < parts; k += 4) sum += sums[(g * parts + k) * cols + n];
    part[wave][at] = sum;
    __syncthreads();
    if (wave == 0 && n < cols) store_value(db + g * sdb + n, (part[0][at] + part[1][at]) + (part[2][at] + part[3][at]));
}

// ---- launchers -------------------------------------------------------------------------------------------------------

template <typename T> static LinearEpilogue<T> forward_epilogue(const LinearArgs &a)
{
    return LinearEpilogue<T>{a.rows, a.dout, (const T *)a.bias, (const T *)a.residual, (T *)a.y, (T *)a.z, a.ldr, a.ldy, a.ldz, a.sb, a.sr, a.sy, a.sz, a.act};
}
// out [rows][cols] alone
template <typename T> static LinearEpilogue<T> plain_epilogue(int64_t rows, int64_t cols, void *out, int64_t ld, int64_t step)
{
    return LinearEpilogue<T>{rows, cols, nullptr, nullptr, (T *)out, nullptr, 0, ld, 0, 0, 0, step, 0, ACT_NONE};
}

int64_t linear_workspace(const LinearArgs &a)
{
    if (!a.bf16) return 0;
    return Source(a.x, a.ldx, a.sx, a.rows, a.din).bytes(a.batch) + Source(a.w, a.ldw, a.sw, a.din, a.dout).bytes(a.batch) + part_bytes(a.batch, a.rows, a.dout, a.din, true);
}

void launch_linear(hipStream_t s, const LinearArgs &a, void *work)
{
    if (!a.bf16) {
        launch_gemm_f32<float>(s, a.batch, a.rows, a.dout, a.din, Operand{a.x, a.ldx, a.sx, true}, Operand{a.w, a.ldw, a.sw, false}, forward_epilogue<float>(a));
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
    const int64_t across = a.batch * ((dz_wide(a) + SLOPE_COLS - 1) / SLOPE_COLS);
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

template <typename T> static void launch_slopes(hipStream_t s, const LinearGradArgs &a, T *dz, float *sums)
{
    if ((dz || a.db) && a.rows > 0)
        slope_kernel<T><<<dim3((uint32_t)((dz_wide(a) + SLOPE_COLS - 1) / SLOPE_COLS), (uint32_t)sum_parts(a), (uint32_t)a.batch), 256, 0, s>>>(
            a.rows, a.dout, slope_run(a), (const T *)a.dy, a.lddy, a.sdy, (const T *)a.z, a.ldz, a.sz, a.act, dz,
            dz_wide(a), a.db ? sums : nullptr);
    if (a.db)
        bias_sum_kernel<T><<<dim3((uint32_t)((a.dout + 63) / 64), (uint32_t)a.batch), 256, 0, s>>>(a.dout, sum_parts(a), sums, (T *)a.db, a.sdb);
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
        launch_slopes<float>(s, a, (float *)dz, sums);
        const Operand d = dz ? Operand{dz, a.dout, a.rows * a.dout, true} : Operand{a.dy, a.lddy, a.sdy, true};
        if (a.dx && a.rows > 0)
            launch_gemm_f32<float>(s, a.batch, a.rows, a.din, a.dout, d, Operand{a.w, a.ldw, a.sw, true}, plain_epilogue<float>(a.rows, a.din, a.dx, a.lddx, a.sdx));
        if (a.dw)
            launch_gemm_f32<float>(s, a.batch, a.din, a.dout, a.rows, Operand{a.x, a.ldx, a.sx, false}, Operand{d.p, d.ld, d.step, false},
                                   plain_epilogue<float>(a.din, a.dout, a.dw, a.lddw, a.sdw));
        return;
    }
    launch_slopes<uint16_t>(s, a, (uint16_t *)dz, sums);
    Layouts l{};
    const Planes16 d = dz ? Planes16{(const char *)dz, nullptr, dz_wide(a), a.rows * dz_wide(a)} : Source(a.dy, a.lddy, a.sdy, a.rows, a.dout).take(a.batch, at, l);
    Planes16 w{}, x{};
    if (a.dx && a.rows > 0) w = Source(a.w, a.ldw, a.sw, a.din, a.dout).take(a.batch, at, l);
    if (a.dw) x = Source(a.x, a.ldx, a.sx, a.rows, a.din).take(a.batch, at, l);
    lay_out(s, l);
    if (a.dx && a.rows > 0)
        launch_product16(s, a.batch, a.rows, a.din, a.dout, d, true, w, true, plain_epilogue<uint16_t>(a.rows, a.din, a.dx, a.lddx, a.sdx), at);
    if (a.dw)
        launch_product16(s, a.batch, a.din, a.dout, a.rows, x, false, d, false, plain_epilogue<uint16_t>(a.din, a.dout, a.dw, a.lddw, a.sdw), at);
}

}  // namespace netmax
