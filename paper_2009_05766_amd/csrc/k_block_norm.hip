// The norms before and after a block with its gate and the residual stream, and their gradients.
//
//   N(v) = v r, r = 1 / sqrt(mean v^2 + eps)                               or, as a layer norm, with v - mean v in the place of v
//   u = N(f) g1 + b1,  h = a x + b act(q) u,  y = N(h) g2 + b2             f: the block's output, x: the residual stream, q: the gate
// Gradients from dy and dh (what reaches h by other ways), with fn = N(f), hn = N(h) and means over a row (those of the mean itself for a layer norm only):
//   e = dy g2,      D = dh + r2 (e - mean e - hn mean(e hn)),              dx = a D,  dq = b act'(q) u D
//   c = b act(q) D g1,                                                     df = r1 (c - mean c - fn mean(c fn))
//   dg2 = sum dy hn,  db2 = sum dy,  dg1 = sum b act(q) D fn,  db1 = sum b act(q) D over the rows; dq too, if q is the same for all rows
// h is computed anew from x and f, in float, so that nothing has to be kept and the gradients do not depend on h's rounding.
// Bound by memory: x, f and q are read, h and y written; the gradients read dy and dh as well and write dx, df and dq.
//
// Means and squares are summed in double (a float's square is exact there): rows of any size have their mean square, over the whole range of the type.  Where a lane holds few values of a
// row it sums their squares in float, as long as that is far from both ends of float's range.  A layer norm's mean is subtracted as two floats, so that rows far from 0 keep their bits.
#include "block_norm.h"
#include "piece.h"

#include <algorithm>
#include <type_traits>

namespace netmax {

constexpr int THREADS = 256;

// ---- a row -----------------------------------------------------------------------------------------------------------

__device__ __forceinline__ float unit_of(const Unit &n, float v) { return ((v - n.mean) - n.rest) * n.r; }

// act(q) and act'(q).  With w = exp(-|z|), 1 / (1 + exp(-z)) is d = 1 / (1 + w) or w d and its slope w d^2: nothing cancels far out.  tanh q is the same with z = 2 q: (1 - w) d, which cancels near 0,
// where its series takes over (below 1/4 its next term is less than 2^-26 of it), and 4 w d^2.
__device__ __forceinline__ void gate_of(int act, float q, float &value, float &slope)
{
    if (act == GATE_NONE) {
        value = q;
        slope = 1.0f;
        return;
    }
    const float w = __builtin_amdgcn_exp2f(fabsf(q) * (act == GATE_TANH ? -2.88539008f : -1.44269504f)), d = __builtin_amdgcn_rcpf(1.0f + w);
    slope = w * d * d;
    if (act == GATE_SIGMOID) {
        value = q < 0.0f ? w * d : d;
        return;
    }
    slope *= 4.0f;
    const float square = q * q;
    float series = fmaf(square, 62.0f / 2835.0f, -17.0f / 315.0f);
    series = fmaf(square, series, 2.0f / 15.0f);
    series = fmaf(square, series, -1.0f / 3.0f);
    value = fabsf(q) < 0.25f ? fmaf(q * square, series, q) : copysignf((1.0f - w) * d, q);
}

// scale times values or slopes of a piece of a gate.
template <typename T> __device__ __forceinline__ void gates_of(int act, float scale, const Piece<T> &q, float (&gate)[Piece<T>::VALUES])
{
    if (act == GATE_NONE) {
#pragma unroll
        for (int e = 0; e < Piece<T>::VALUES; ++e) gate[e] = scale * q.get(e);
    } else {
#pragma unroll
        for (int e = 0; e < Piece<T>::VALUES; ++e) {
            float value, slope;
            gate_of(act, q.get(e), value, slope);
            gate[e] = scale * value;
        }
    }
}
template <typename T> __device__ __forceinline__ void slopes_of(int act, float scale, const Piece<T> &q, float (&slopes)[Piece<T>::VALUES])
{
#pragma unroll
    for (int e = 0; e < Piece<T>::VALUES; ++e) {
        float value, slope;
        gate_of(act, q.get(e), value, slope);
        slopes[e] = scale * slope;
    }
}

// Where a row's operands lie.
template <typename T> struct RowAt {
    const T *x, *f, *q, *g1, *b1, *g2, *b2;
    __device__ __forceinline__ RowAt(const NormArgs &a, int64_t b, int64_t t)
        : x(at(a.x, b, t)), f(at(a.f, b, t)), q(at(a.gate, b, a.gate_rows ? t : 0)), g1(at(a.post_gain, b, 0)), b1(at(a.post_bias, b, 0)), g2(at(a.pre_gain, b, 0)), b2(at(a.pre_bias, b, 0)) { }
    static __device__ __forceinline__ T *at(const Span &s, int64_t b, int64_t t) { return s.p ? (T *)s.p + b * s.s + t * s.ld : nullptr; }
};

// Values of one piece of a row, with those of operands that are not there by what leaves them out.
template <typename T> struct Values {
    static constexpr int VALUES = Piece<T>::VALUES;
    float fn[VALUES], u[VALUES], q[VALUES], slope[VALUES], h[VALUES];
    __device__ __forceinline__ Values(const NormArgs &a, const RowAt<T> &row, int64_t col, const Unit &post)
    {
        const int64_t left = a.width - col;
        const Piece<T> x = load_piece(row.x + col, left);
#pragma unroll
        for (int e = 0; e < VALUES; ++e) { fn[e] = 0.0f; u[e] = 0.0f; q[e] = 1.0f; slope[e] = 0.0f; h[e] = a.x_scale * x.get(e); }
        if (!row.f) return;
        const Piece<T> f = load_piece(row.f + col, left);
#pragma unroll
        for (int e = 0; e < VALUES; ++e) fn[e] = u[e] = a.post ? unit_of(post, f.get(e)) : f.get(e);
        if (row.g1) {
            const Piece<T> g = load_piece(row.g1 + col, left);
#pragma unroll
            for (int e = 0; e < VALUES; ++e) u[e] *= g.get(e);
        }
        if (row.b1) {
            const Piece<T> g = load_piece(row.b1 + col, left);
#pragma unroll
            for (int e = 0; e < VALUES; ++e) u[e] += g.get(e);
        }
        if (row.q) {
            const Piece<T> g = load_piece(row.q + col, left);
#pragma unroll
            for (int e = 0; e < VALUES; ++e) gate_of(a.act, g.get(e), q[e], slope[e]);
        }
#pragma unroll
        for (int e = 0; e < VALUES; ++e) h[e] = fmaf(a.f_scale * q[e], u[e], h[e]);
    }
};

// ---- rows of any length, read anew for each of their sums ------------------------------------------------------------

template <int N, typename S> __device__ __forceinline__ void sum_over(S (&v)[N], S (*room)[N])
{
    __syncthreads();                               // the sums before have been read
    row_sum<THREADS>(v, room);
}

// value(col, v): the values at a column.
template <typename T, class Get> __device__ __forceinline__ Unit unit_over(const NormArgs &a, const Get &get, double (*room)[1])
{
    constexpr int VALUES = Piece<T>::VALUES;
    double mean = 0.0;
    if (a.layer) {
        double sum[1] = {0.0};
        for (int64_t col = (int64_t)threadIdx.x * VALUES; col < a.width; col += THREADS * VALUES) {
            float v[VALUES];
            get(col, v);
            for (int e = 0; e < VALUES && col + e < a.width; ++e) sum[0] += v[e];
        }
        sum_over(sum, room);
        mean = sum[0] * a.share;
    }
    double sum[1] = {0.0};
    for (int64_t col = (int64_t)threadIdx.x * VALUES; col < a.width; col += THREADS * VALUES) {
        float v[VALUES];
        get(col, v);
        for (int e = 0; e < VALUES && col + e < a.width; ++e) sum[0] = fma((double)v[e] - mean, (double)v[e] - mean, sum[0]);
    }
    sum_over(sum, room);
    Unit n;
    n.mean = (float)mean;
    n.rest = (float)(mean - (double)n.mean);
    n.r = (float)rsqrt(sum[0] * a.share + a.eps);
    return n;
}

template <typename T> __device__ __forceinline__ void units_of(const NormArgs &a, const RowAt<T> &row, Unit &post, Unit &pre, double (*room)[1])
{
    constexpr int VALUES = Piece<T>::VALUES;
    if (a.post && row.f)
        post = unit_over<T>(a, [&](int64_t col, float (&v)[VALUES]) {
            const Piece<T> f = load_piece(row.f + col, a.width - col);
            for (int e = 0; e < VALUES; ++e) v[e] = f.get(e);
        }, room);
    if (a.pre)
        pre = unit_over<T>(a, [&](int64_t col, float (&v)[VALUES]) {
            const Values<T> at(a, row, col, post);
            for (int e = 0; e < VALUES; ++e) v[e] = at.h[e];
        }, room);
}

template <typename T> __global__ void __launch_bounds__(THREADS) long_norm_kernel(NormArgs a)
{
    constexpr int VALUES = Piece<T>::VALUES;
    __shared__ double room[THREADS / 64][1];
    for (int64_t t = blockIdx.x; t < a.rows; t += gridDim.x) {
        const RowAt<T> row(a, blockIdx.y, t);
        Unit post{}, pre{};
        units_of(a, row, post, pre, room);
        T *h = RowAt<T>::at(a.h, blockIdx.y, t), *y = RowAt<T>::at(a.y, blockIdx.y, t);
        for (int64_t col = (int64_t)threadIdx.x * VALUES; col < a.width; col += THREADS * VALUES) {
            const int64_t left = a.width - col;
            const Values<T> at(a, row, col, post);
            Piece<T> out;
            float v[VALUES];
            if (a.pre) {
#pragma unroll
                for (int e = 0; e < VALUES; ++e) v[e] = unit_of(pre, at.h[e]);
                if (row.g2) {
                    const Piece<T> g = load_piece(row.g2 + col, left);
#pragma unroll
                    for (int e = 0; e < VALUES; ++e) v[e] *= g.get(e);
                }
                if (row.b2) {
                    const Piece<T> g = load_piece(row.b2 + col, left);
#pragma unroll
                    for (int e = 0; e < VALUES; ++e) v[e] += g.get(e);
                }
                out.set(v);
                if (y) store_piece(y + col, left, out);
            }
            if (h) {
                out.set(at.h);
                store_piece(h + col, left, out);
            }
        }
    }
}

template <typename T> __global__ void __launch_bounds__(THREADS) long_norm_grad_kernel(NormArgs a, Partials to)
{
    constexpr int VALUES = Piece<T>::VALUES;
    __shared__ double room[THREADS / 64][1];
    __shared__ float pair[THREADS / 64][2];
    const float share = (float)a.share;
    for (int64_t t = blockIdx.x; t < a.rows; t += gridDim.x) {
        const RowAt<T> row(a, blockIdx.y, t);
        Unit post{}, pre{};
        units_of(a, row, post, pre, room);
        const T *dy = RowAt<T>::at(a.dy, blockIdx.y, t), *dh = RowAt<T>::at(a.dh, blockIdx.y, t);
        float along[2] = {0.0f, 0.0f}, back[2] = {0.0f, 0.0f};
        // e and hn
        const auto before = [&](const Values<T> &at, int64_t col, float (&d)[VALUES], float (&e)[VALUES], float (&hn)[VALUES]) {
            const int64_t left = a.width - col;
            const Piece<T> v = load_piece(dy + col, left);
#pragma unroll
            for (int k = 0; k < VALUES; ++k) { d[k] = e[k] = v.get(k); hn[k] = unit_of(pre, at.h[k]); }
            if (!row.g2) return;
            const Piece<T> g = load_piece(row.g2 + col, left);
#pragma unroll
            for (int k = 0; k < VALUES; ++k) e[k] *= g.get(k);
        };
        if (a.pre) {
            for (int64_t col = (int64_t)threadIdx.x * VALUES; col < a.width; col += THREADS * VALUES) {
                const Values<T> at(a, row, col, post);
                float d[VALUES], e[VALUES], hn[VALUES];
                before(at, col, d, e, hn);
                for (int k = 0; k < VALUES && col + k < a.width; ++k) { along[0] += e[k]; along[1] = fmaf(e[k], hn[k], along[1]); }
            }
            sum_over(along, pair);
        }
        const float mean_e = a.layer ? along[0] * share : 0.0f, mean_eh = along[1] * share;
        if (to.rows && threadIdx.x == 0) to.rows[blockIdx.y * a.rows + t] = RowSums{post, pre, mean_e, mean_eh};
        // D
        const auto reaches = [&](const Values<T> &at, int64_t col, float (&D)[VALUES], float (&d)[VALUES], float (&hn)[VALUES]) {
#pragma unroll
            for (int k = 0; k < VALUES; ++k) D[k] = d[k] = hn[k] = 0.0f;
            if (dh) {
                const Piece<T> v = load_piece(dh + col, a.width - col);
#pragma unroll
                for (int k = 0; k < VALUES; ++k) D[k] = v.get(k);
            }
            if (!a.pre) return;
            float e[VALUES];
            before(at, col, d, e, hn);
#pragma unroll
            for (int k = 0; k < VALUES; ++k) D[k] = fmaf(pre.r, (e[k] - mean_e) - hn[k] * mean_eh, D[k]);
        };
        const auto gain_post = [&](int64_t col, float (&g)[VALUES]) {
#pragma unroll
            for (int k = 0; k < VALUES; ++k) g[k] = 1.0f;
            if (!row.g1) return;
            const Piece<T> v = load_piece(row.g1 + col, a.width - col);
#pragma unroll
            for (int k = 0; k < VALUES; ++k) g[k] = v.get(k);
        };
        if (row.f && a.post) {
            for (int64_t col = (int64_t)threadIdx.x * VALUES; col < a.width; col += THREADS * VALUES) {
                const Values<T> at(a, row, col, post);
                float D[VALUES], d[VALUES], hn[VALUES], g[VALUES];
                reaches(at, col, D, d, hn);
                gain_post(col, g);
                for (int k = 0; k < VALUES && col + k < a.width; ++k) {
                    const float c = a.f_scale * at.q[k] * D[k] * g[k];
                    back[0] += c;
                    back[1] = fmaf(c, at.fn[k], back[1]);
                }
            }
            sum_over(back, pair);
        }
        const float mean_c = a.layer ? back[0] * share : 0.0f, mean_cf = back[1] * share;
        T *dx = RowAt<T>::at(a.dx, blockIdx.y, t), *df = RowAt<T>::at(a.df, blockIdx.y, t), *dq = a.gate_rows ? RowAt<T>::at(a.dgate, blockIdx.y, t) : nullptr;
        for (int64_t col = (int64_t)threadIdx.x * VALUES; col < a.width; col += THREADS * VALUES) {
            const int64_t left = a.width - col;
            const Values<T> at(a, row, col, post);
            float D[VALUES], d[VALUES], hn[VALUES], g[VALUES], v[VALUES], slopes[VALUES];
            reaches(at, col, D, d, hn);
            Piece<T> out;
#pragma unroll
            for (int k = 0; k < VALUES; ++k) v[k] = a.x_scale * D[k];
            out.set(v);
            if (dx) store_piece(dx + col, left, out);
            gain_post(col, g);
#pragma unroll
            for (int k = 0; k < VALUES; ++k) {
                const float du = a.f_scale * at.q[k] * D[k];
                slopes[k] = a.f_scale * at.slope[k] * at.u[k] * D[k];
                v[k] = a.post ? post.r * ((du * g[k] - mean_c) - at.fn[k] * mean_cf) : du;
            }
            if (df) {
                out.set(v);
                store_piece(df + col, left, out);
            }
            if (dq) {
                out.set(slopes);
                store_piece(dq + col, left, out);
            }
        }
    }
}

// Column sums: 16 columns for a workgroup, whose 64 groups of lanes take turns at the partial sums.
constexpr int JOIN_COLUMNS = 16, JOIN_TURNS = 64;
template <typename T> __global__ void __launch_bounds__(JOIN_COLUMNS * JOIN_TURNS) join_sums_kernel(NormArgs a, Partials from)
{
    __shared__ double part[JOIN_TURNS][JOIN_COLUMNS];
    const int32_t turn = threadIdx.x / JOIN_COLUMNS;
    const int64_t col = (int64_t)blockIdx.x * JOIN_COLUMNS + threadIdx.x % JOIN_COLUMNS, row = from.sums * from.padded;
    const float *p = from.p + (blockIdx.z * from.workgroups * from.sums + blockIdx.y) * from.padded + col;
    double sum = 0.0;
    if (col < a.width)
#pragma unroll 8
        for (int64_t w = turn; w < from.workgroups; w += JOIN_TURNS) sum += p[w * row];
    part[turn][threadIdx.x % JOIN_COLUMNS] = sum;
    __syncthreads();
    if (threadIdx.x >= 4 * JOIN_COLUMNS) return;
    sum = 0.0;
#pragma unroll
    for (int k = 0; k < JOIN_TURNS / 4; ++k) sum += part[k * 4 + turn][threadIdx.x % JOIN_COLUMNS];
    sum += __shfl_xor(sum, JOIN_COLUMNS);
    sum += __shfl_xor(sum, 2 * JOIN_COLUMNS);
    if (turn == 0 && col < a.width) store_value(RowAt<T>::at(from.out[blockIdx.y], blockIdx.z, 0) + col, (float)sum);
}

// ---- rows that a group of lanes keeps in registers -------------------------------------------------------------------
//
// LANES lanes hold a row's operands, PIECES pieces each, between its sums: everything is read once.  Narrow rows share a workgroup.

constexpr int threads_of(int lanes) { return lanes <= 64 ? THREADS : lanes; }

// What of a row the lane's piece k holds: `left` values from its column on, none if that is not positive.  Rows are short here: 32 bits count their bytes.
//
// Rows are fetched without a branch around any load, whose result would have to be waited for where the branches meet: a lane whose piece ends behind the row reads the row's last full piece, and
// moves its values once they have come (settle); what is not there is fetched from another operand's row and cleared.
template <typename T, int LANES> struct Lane {
    static constexpr int VALUES = Piece<T>::VALUES;
    int32_t width; uint32_t first;
    __device__ __forceinline__ Lane(int64_t width_) : width((int32_t)width_), first(threadIdx.x % LANES * VALUES) { }
    __device__ __forceinline__ uint32_t col(int k) const { return first + k * LANES * VALUES; }
    __device__ __forceinline__ int32_t left(int k) const { return width - (int32_t)col(k); }
    __device__ __forceinline__ T *at(const T *row, uint32_t column) const { return (T *)((char *)row + (uint32_t)(column * sizeof(T))); }
    template <int PIECES> __device__ __forceinline__ void fetch(const T *row, Piece<T> (&to)[PIECES]) const
    {
#pragma unroll
        for (int k = 0; k < PIECES; ++k) to[k].v = *reinterpret_cast<const typename Piece<T>::Memory *>(at(row, left(k) >= VALUES ? col(k) : (uint32_t)(width - VALUES)));
    }
    template <int PIECES> __device__ __forceinline__ void settle(Piece<T> (&v)[PIECES], bool there = true) const
    {
#pragma unroll
        for (int k = 0; k < PIECES; ++k) {
            if (left(k) >= VALUES && there) continue;
            if (left(k) <= 0 || !there) v[k].v = decltype(v[k].v){};
            else shift_down(v[k], VALUES - left(k));
        }
    }
    template <int PIECES> __device__ __forceinline__ void load(const T *row, Piece<T> (&to)[PIECES]) const
    {
        fetch(row, to);
        settle(to);
    }
    // values that are not there are `other`; behind the row 0
    template <int PIECES> __device__ __forceinline__ void load_or(const T *row, Piece<T> (&to)[PIECES], float other) const
    {
        if (row) { load(row, to); return; }
#pragma unroll
        for (int k = 0; k < PIECES; ++k) {
            float v[VALUES];
#pragma unroll
            for (int e = 0; e < VALUES; ++e) v[e] = e < left(k) ? other : 0.0f;
            to[k].set(v);
        }
    }
    __device__ __forceinline__ void store(T *row, int k, const Piece<T> &v) const
    {
        if (row && left(k) > 0) store_piece(at(row, col(k)), left(k), v);
    }
    __device__ __forceinline__ void store(T *row, int k, const float (&v)[VALUES]) const
    {
        Piece<T> out;
        out.set(v);
        store(row, k, out);
    }
    // values behind the row become 0
    __device__ __forceinline__ void once(int k, float (&v)[VALUES]) const
    {
        if (left(k) < VALUES)
#pragma unroll
            for (int e = 0; e < VALUES; ++e) v[e] = e < left(k) ? v[e] : 0.0f;
    }
};

// 1 / sqrt(v), v > 0: the hardware's in float on a mantissa, one step of Newton's iteration, to 1.5 units in the last place; 0 for inf.
__device__ __forceinline__ float inverse_root(double v)
{
    const int twice = __builtin_amdgcn_frexp_exp(v) & ~1;
    const float m = (float)__builtin_amdgcn_ldexp(v, -twice), r = __builtin_amdgcn_rsqf(m);
    return __builtin_amdgcn_ldexpf(r > 0.0f ? fmaf(r * 0.5f, fmaf(-m * r, r, 1.0f), r) : r, -twice / 2);
}

// get(k, v): the values of the lane's piece k, of which lane.once() leaves those that count.
template <typename T, int LANES, int PIECES, bool LAYER, class Columns, class Get>
__device__ __forceinline__ Unit unit_held(const Columns &lane, const Get &get, double share, double eps, double (*room)[1], double (*second)[1])
{
    constexpr int VALUES = Piece<T>::VALUES;
    Unit n{};
    if constexpr (LAYER) {
        double sum[1] = {0.0};
#pragma unroll
        for (int k = 0; k < PIECES; ++k) {
            float v[VALUES];
            get(k, v);
            lane.once(k, v);
#pragma unroll
            for (int e = 0; e < VALUES; ++e) sum[0] += v[e];
        }
        row_sum<LANES>(sum, room);
        const double mean = sum[0] * share;
        n.mean = (float)mean;
        n.rest = (float)(mean - (double)n.mean);
    }
    const auto centred = [&](int k, float (&v)[VALUES]) {
        get(k, v);
        if constexpr (LAYER) {
#pragma unroll
            for (int e = 0; e < VALUES; ++e) v[e] = (v[e] - n.mean) - n.rest;
        }
        lane.once(k, v);
    };
    float square[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < PIECES; ++k) {
        float v[VALUES];
        centred(k, v);
#pragma unroll
        for (int e = 0; e < VALUES; ++e) square[e & 3] = fmaf(v[e], v[e], square[e & 3]);
    }
    const float all = (square[0] + square[1]) + (square[2] + square[3]);
    double sum[1] = {(double)all};
    if (!(all > 0x1p-90f && all < 0x1p120f)) {     // squares that left float's range, or may have
        sum[0] = 0.0;
#pragma unroll
        for (int k = 0; k < PIECES; ++k) {
            float v[VALUES];
            centred(k, v);
#pragma unroll
            for (int e = 0; e < VALUES; ++e) sum[0] = fma((double)v[e], (double)v[e], sum[0]);
        }
    }
    row_sum<LANES>(sum, second);
    n.r = inverse_root(sum[0] * share + eps);
    return n;
}
template <bool LAYER> __device__ __forceinline__ float unit_held_of(const Unit &n, float v) { return LAYER ? unit_of(n, v) : v * n.r; }

template <typename T, int LANES, int PIECES, bool LAYER>
__global__ void __launch_bounds__(threads_of(LANES)) norm_kernel(NormArgs a)
{
    constexpr int VALUES = Piece<T>::VALUES, GROUPS = threads_of(LANES) / LANES;
    __shared__ double room[4][LANES > 64 ? LANES / 64 : 1][1];
    const int64_t t = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * GROUPS + threadIdx.x / LANES;
    if (t >= a.rows) return;                       // whole groups; with barriers a whole workgroup
    const RowAt<T> row(a, blockIdx.z, t);
    const Lane<T, LANES> lane(a.width);
    const double share = a.share;
    Piece<T> x[PIECES], f[PIECES], q[PIECES], g1[PIECES], b1[PIECES], g2[PIECES], b2[PIECES];
    lane.fetch(row.x, x);
    if (row.f) lane.fetch(row.f, f);
    if (row.q) lane.fetch(row.q, q);
    if (row.g1) lane.fetch(row.g1, g1);
    if (row.b1) lane.fetch(row.b1, b1);
    if (row.g2) lane.fetch(row.g2, g2);
    if (row.b2) lane.fetch(row.b2, b2);
    lane.settle(x);
    lane.settle(f);
    float h[PIECES][VALUES];
#pragma unroll
    for (int k = 0; k < PIECES; ++k)
#pragma unroll
        for (int e = 0; e < VALUES; ++e) h[k][e] = a.x_scale * x[k].get(e);
    if (row.f) {
        Unit post{0.0f, 0.0f, 1.0f};
        if (a.post) post = unit_held<T, LANES, PIECES, LAYER>(lane, [&](int k, float (&v)[VALUES]) {
#pragma unroll
            for (int e = 0; e < VALUES; ++e) v[e] = f[k].get(e);
        }, share, a.eps, room[0], room[1]);
        lane.settle(q);
        lane.settle(g1);
        lane.settle(b1);
#pragma unroll
        for (int k = 0; k < PIECES; ++k) {
            float u[VALUES], gate[VALUES];
#pragma unroll
            for (int e = 0; e < VALUES; ++e) u[e] = unit_held_of<LAYER>(post, f[k].get(e));
            if (row.g1)
#pragma unroll
                for (int e = 0; e < VALUES; ++e) u[e] *= g1[k].get(e);
            if (row.b1)
#pragma unroll
                for (int e = 0; e < VALUES; ++e) u[e] += b1[k].get(e);
            if (row.q) gates_of<T>(a.act, a.f_scale, q[k], gate);
            else
#pragma unroll
                for (int e = 0; e < VALUES; ++e) gate[e] = a.f_scale;
#pragma unroll
            for (int e = 0; e < VALUES; ++e) h[k][e] = fmaf(gate[e], u[e], h[k][e]);
        }
    }
    T *to_h = RowAt<T>::at(a.h, blockIdx.z, t), *to_y = RowAt<T>::at(a.y, blockIdx.z, t);
    if (to_h)
#pragma unroll
        for (int k = 0; k < PIECES; ++k) lane.store(to_h, k, h[k]);
    if (!to_y) return;
    const Unit pre = unit_held<T, LANES, PIECES, LAYER>(lane, [&](int k, float (&v)[VALUES]) {
#pragma unroll
        for (int e = 0; e < VALUES; ++e) v[e] = h[k][e];
    }, share, a.eps, room[2], room[3]);
    lane.settle(g2);
    lane.settle(b2);
#pragma unroll
    for (int k = 0; k < PIECES; ++k) {
#pragma unroll
        for (int e = 0; e < VALUES; ++e) h[k][e] = unit_held_of<LAYER>(pre, h[k][e]);
        if (row.g2)
#pragma unroll
            for (int e = 0; e < VALUES; ++e) h[k][e] *= g2[k].get(e);
        if (row.b2)
#pragma unroll
            for (int e = 0; e < VALUES; ++e) h[k][e] += b2[k].get(e);
        lane.store(to_y, k, h[k]);
    }
}

// Gradients: workgroups go through the rows, the next of which is under way while one is worked on.  Reads and writes are waited for in their order, and behind a branch the compiler counts on the
// fewest of them, so that there is no branch around any: a lane whose piece ends behind the row works on the row's last full piece instead and leaves what its neighbour leaves there, too, in the same bits; it takes part in
// no sum twice.  Operands that are not there are read from x, results that nobody wants are written to a row of the workspace.  (With branches 16384 x 8192 bfloat16 took 354 us.)
template <typename T, int LANES, int PIECES> struct Window {
    static constexpr int VALUES = Piece<T>::VALUES;
    uint32_t column[PIECES]; int32_t twice[PIECES];                 // first column of a piece; its values that are a neighbour's
    __device__ __forceinline__ Window(int64_t width)
    {
#pragma unroll
        for (int k = 0; k < PIECES; ++k) {
            const int32_t col = (int32_t)(threadIdx.x % LANES + k * LANES) * VALUES, last = (int32_t)width - VALUES;
            column[k] = col < last ? col : last;
            twice[k] = col <= last ? 0 : col - last < VALUES ? col - last : VALUES;
        }
    }
    __device__ __forceinline__ T *at(const T *row, int k) const { return (T *)((char *)row + (uint32_t)(column[k] * sizeof(T))); }
    __device__ __forceinline__ void fetch(const T *row, Piece<T> (&to)[PIECES]) const
    {
#pragma unroll
        for (int k = 0; k < PIECES; ++k) to[k].v = *reinterpret_cast<const typename Piece<T>::Memory *>(at(row, k));
    }
    __device__ __forceinline__ void fetch_or(const T *row, Piece<T> (&to)[PIECES], float other) const
    {
        if (row) { fetch(row, to); return; }
        float v[VALUES];
#pragma unroll
        for (int e = 0; e < VALUES; ++e) v[e] = other;
#pragma unroll
        for (int k = 0; k < PIECES; ++k) to[k].set(v);
    }
    __device__ __forceinline__ void leave(T *row, const Piece<T> (&from)[PIECES]) const
    {
#pragma unroll
        for (int k = 0; k < PIECES; ++k) *reinterpret_cast<typename Piece<T>::Memory *>(at(row, k)) = from[k].v;
    }
    // for a sum: values that a neighbour counts become 0
    __device__ __forceinline__ void once(int k, float (&v)[VALUES]) const
    {
        if (twice[k] > 0)
#pragma unroll
            for (int e = 0; e < VALUES; ++e) v[e] = e < twice[k] ? 0.0f : v[e];
    }
};

// The compiler does not know any more what these hold: they have come by now, and what was unpacked from them is not kept, but unpacked anew.
template <typename T, int PIECES> __device__ __forceinline__ void let_go(Piece<T> (&p)[PIECES])
{
#pragma unroll
    for (int k = 0; k < PIECES; ++k) asm volatile("" : "+v"(p[k].v));
}

// What a kernel holds in registers: operands and sums over the rows of a norm alone, of a block without biases, or of any block; of a block whose gate has rows of its own, or of others.
enum Form : int { NORM_ALONE = 0, BLOCK_GAINS = 1, BLOCK_ALL = 2, GATED_GAINS = 3, GATED_ALL = 4 };

template <typename T, int LANES, int PIECES, bool LAYER, int FORM, bool HELD>
__global__ void __launch_bounds__(threads_of(LANES)) norm_grad_kernel(NormArgs a, Partials to)
{
    constexpr int VALUES = Piece<T>::VALUES, GROUPS = threads_of(LANES) / LANES, MEANS = LAYER ? 2 : 1;
    constexpr bool BLOCK = FORM != NORM_ALONE, BIASES = FORM != BLOCK_GAINS && FORM != GATED_GAINS, GATED = FORM == GATED_GAINS || FORM == GATED_ALL;
    constexpr bool AHEAD = LANES < 1024 ? PIECES == 1 || !GATED : PIECES == 1 ? !BLOCK || FORM == BLOCK_GAINS : PIECES == 2 && !BLOCK && (sizeof(T) == 4 || !HELD);      // as far as registers go
    __shared__ double room[4][LANES > 64 ? LANES / 64 : 1][1];
    __shared__ float pairs[2][LANES > 64 ? LANES / 64 : 1][MEANS];
    __shared__ float shared_sums[GROUPS > 1 ? GROUPS : 1][GROUPS > 1 ? LANES * PIECES * VALUES : 1];
    const Window<T, LANES, PIECES> lane(a.width);
    const float share = (float)a.share;
    const RowAt<T> vectors(a, blockIdx.y, 0);
    T *const unwanted = (T *)to.unwanted + to.unwanted_row(blockIdx.y, blockIdx.x, threadIdx.x / LANES, GROUPS);
    Piece<T> g1[PIECES], b1[PIECES], g2[PIECES];
    float gate[BLOCK ? PIECES : 1][VALUES];        // b act(q)
    lane.fetch_or(vectors.g2, g2, 1.0f);
    if constexpr (BLOCK) {
        Piece<T> q[PIECES];
        lane.fetch_or(vectors.g1, g1, 1.0f);
        if constexpr (BIASES) lane.fetch_or(vectors.b1, b1, 0.0f);
        lane.fetch_or(GATED ? nullptr : vectors.q, q, 1.0f);
#pragma unroll
        for (int k = 0; k < PIECES; ++k) gates_of<T>(GATED || !vectors.q ? GATE_NONE : a.act, a.f_scale, q[k], gate[k]);
    }
    float sums[SUMS][PIECES][VALUES] = {};
    struct Operands { Piece<T> x[PIECES], f[PIECES], q[PIECES], dy[PIECES], dh[PIECES]; };
    const auto fetch = [&](int64_t t, Operands &o) {
        const RowAt<T> row(a, blockIdx.y, t);
        const T *dy = RowAt<T>::at(a.dy, blockIdx.y, t), *dh = RowAt<T>::at(a.dh, blockIdx.y, t);
        lane.fetch(row.x, o.x);
        if constexpr (BLOCK) lane.fetch(row.f, o.f);
        if constexpr (GATED) lane.fetch(row.q, o.q);
        lane.fetch(a.dy.p ? dy : row.x, o.dy);
        lane.fetch(a.dh.p ? dh : row.x, o.dh);
    };
    const int64_t step = (int64_t)gridDim.x * GROUPS;
    int64_t t = (int64_t)blockIdx.x * GROUPS + threadIdx.x / LANES;
    Operands next;
    if constexpr (AHEAD) {
        fetch(t < a.rows ? t : a.rows - 1, next);
        let_go(next.x); let_go(next.dy); let_go(next.dh);           // come before the loop, as in its turns: what is waited for at its top holds for all of them
        if constexpr (BLOCK) let_go(next.f);
        if constexpr (GATED) let_go(next.q);
    }
    for (; t < a.rows; t += step) {
        Operands row = next;
        if (AHEAD) fetch(t + step < a.rows ? t + step : t, next);
        else fetch(t, row);
        // all of the row has come before the first barrier, behind which other waves may write over it
        let_go(row.x); let_go(row.dy); let_go(row.dh); let_go(g2);
        if constexpr (BLOCK) { let_go(row.f); let_go(g1); }
        if constexpr (BLOCK && BIASES) let_go(b1);
        if constexpr (GATED) let_go(row.q);
        if (LANES > 64 && !a.pre && !(BLOCK && a.post)) __syncthreads();
        Unit post{0.0f, 0.0f, 1.0f};
        if constexpr (BLOCK) {
            if (a.post) post = unit_held<T, LANES, PIECES, LAYER>(lane, [&](int k, float (&v)[VALUES]) {
#pragma unroll
                for (int e = 0; e < VALUES; ++e) v[e] = row.f[k].get(e);
            }, a.share, a.eps, room[0], room[1]);
            if constexpr (GATED)
#pragma unroll
                for (int k = 0; k < PIECES; ++k) gates_of<T>(a.act, a.f_scale, row.q[k], gate[k]);
        }
        // fn and u
        const auto branch = [&](int k, float (&fn)[VALUES], float (&u)[VALUES]) {
#pragma unroll
            for (int e = 0; e < VALUES; ++e) {
                fn[e] = unit_held_of<LAYER>(post, row.f[k].get(e));
                u[e] = BIASES ? fmaf(fn[e], g1[k].get(e), b1[k].get(e)) : fn[e] * g1[k].get(e);
            }
        };
        float d[PIECES][VALUES];                   // h, hn, then D
        Unit pre{};
        float mean_e = 0.0f, mean_eh = 0.0f;
        if (a.pre) {
#pragma unroll
            for (int k = 0; k < PIECES; ++k) {
#pragma unroll
                for (int e = 0; e < VALUES; ++e) d[k][e] = a.x_scale * row.x[k].get(e);
                if constexpr (BLOCK) {
                    float fn[VALUES], u[VALUES];
                    branch(k, fn, u);
#pragma unroll
                    for (int e = 0; e < VALUES; ++e) d[k][e] = fmaf(gate[k][e], u[e], d[k][e]);
                }
            }
            pre = unit_held<T, LANES, PIECES, LAYER>(lane, [&](int k, float (&v)[VALUES]) {
#pragma unroll
                for (int e = 0; e < VALUES; ++e) v[e] = d[k][e];
            }, a.share, a.eps, room[2], room[3]);
            float along[MEANS] = {};
#pragma unroll
            for (int k = 0; k < PIECES; ++k) {
                float w[VALUES];
#pragma unroll
                for (int e = 0; e < VALUES; ++e) {
                    const float v = row.dy[k].get(e);
                    w[e] = v * g2[k].get(e);
                    d[k][e] = unit_held_of<LAYER>(pre, d[k][e]);
                    if (HELD) sums[2][k][e] = fmaf(v, d[k][e], sums[2][k][e]);
                    if (HELD && BIASES) sums[3][k][e] += v;
                }
                lane.once(k, w);
#pragma unroll
                for (int e = 0; e < VALUES; ++e) {
                    along[0] = fmaf(w[e], d[k][e], along[0]);
                    if (LAYER) along[MEANS - 1] += w[e];
                }
            }
            row_sum<LANES>(along, pairs[0]);
            let_go(row.dy);
            let_go(g2);
            mean_eh = along[0] * share;
            if (LAYER) mean_e = along[MEANS - 1] * share;
#pragma unroll
            for (int k = 0; k < PIECES; ++k)
#pragma unroll
                for (int e = 0; e < VALUES; ++e) {
                    const float w = row.dy[k].get(e) * g2[k].get(e);
                    d[k][e] = pre.r * fmaf(-d[k][e], mean_eh, LAYER ? w - mean_e : w);
                }
            if (a.dh.p)
#pragma unroll
                for (int k = 0; k < PIECES; ++k)
#pragma unroll
                    for (int e = 0; e < VALUES; ++e) d[k][e] += row.dh[k].get(e);
        } else {
#pragma unroll
            for (int k = 0; k < PIECES; ++k)
#pragma unroll
                for (int e = 0; e < VALUES; ++e) d[k][e] = row.dh[k].get(e);
        }
        if (!HELD && to.rows && threadIdx.x % LANES == 0) {
            RowSums &left = to.rows[blockIdx.y * a.rows + t];
            left.post = post;
            left.pre = pre;
            left.mean_e = mean_e;
            left.mean_eh = mean_eh;
        }
        Piece<T> out[PIECES];
#pragma unroll
        for (int k = 0; k < PIECES; ++k) {
            float v[VALUES];
#pragma unroll
            for (int e = 0; e < VALUES; ++e) v[e] = a.x_scale * d[k][e];
            out[k].set(v);
        }
        lane.leave(a.dx.p ? RowAt<T>::at(a.dx, blockIdx.y, t) : unwanted, out);
        if constexpr (BLOCK) {
            float back[MEANS] = {};
            let_go(row.f);
            let_go(g1);
#pragma unroll
            for (int k = 0; k < PIECES; ++k) {
                float fn[VALUES], u[VALUES];
                branch(k, fn, u);
                if constexpr (GATED) {
                    float v[VALUES];
                    slopes_of<T>(a.act, a.f_scale, row.q[k], v);
#pragma unroll
                    for (int e = 0; e < VALUES; ++e) v[e] *= u[e] * d[k][e];
                    out[k].set(v);
                }
#pragma unroll
                for (int e = 0; e < VALUES; ++e) {
                    if (HELD && !GATED) sums[4][k][e] = fmaf(u[e], d[k][e], sums[4][k][e]);
                    const float du = gate[k][e] * d[k][e];
                    if (HELD && BIASES) sums[1][k][e] += du;
                    if (HELD) sums[0][k][e] = fmaf(du, fn[e], sums[0][k][e]);
                    d[k][e] = u[e] = du * g1[k].get(e);             // c
                }
                lane.once(k, u);
#pragma unroll
                for (int e = 0; e < VALUES; ++e) {
                    back[0] = fmaf(u[e], fn[e], back[0]);
                    if (LAYER) back[MEANS - 1] += u[e];
                }
            }
            if constexpr (GATED) lane.leave(a.dgate.p ? RowAt<T>::at(a.dgate, blockIdx.y, t) : unwanted, out);
            if (a.post) row_sum<LANES>(back, pairs[1]);
            const float mean_cf = a.post ? back[0] * share : 0.0f, mean_c = LAYER && a.post ? back[MEANS - 1] * share : 0.0f;
#pragma unroll
            for (int k = 0; k < PIECES; ++k) {
                float v[VALUES];
#pragma unroll
                for (int e = 0; e < VALUES; ++e) {
                    const float fn = unit_held_of<LAYER>(post, row.f[k].get(e));
                    v[e] = a.post ? post.r * fmaf(-fn, mean_cf, LAYER ? d[k][e] - mean_c : d[k][e]) : d[k][e];      // without a norm c itself, wherever f is infinite
                }
                out[k].set(v);
            }
            lane.leave(a.df.p ? RowAt<T>::at(a.df, blockIdx.y, t) : unwanted, out);
        }
    }
    if constexpr (!HELD) return;
    if constexpr (BLOCK && !GATED)                 // a gate that is the same for all rows has one slope, too
        if (to.place[4] >= 0) {
            Piece<T> q[PIECES];
            lane.fetch_or(vectors.q, q, 1.0f);
#pragma unroll
            for (int k = 0; k < PIECES; ++k) {
                float slope[VALUES];
                slopes_of<T>(a.act, a.f_scale, q[k], slope);
#pragma unroll
                for (int e = 0; e < VALUES; ++e) sums[4][k][e] *= slope[e];
            }
        }
    float *mine = to.p + (blockIdx.y * to.workgroups + blockIdx.x) * to.sums * to.padded;
#pragma unroll
    for (int s = 0; s < SUMS; ++s) {
        if ((!BLOCK && s != 2 && s != 3) || (!BIASES && (s == 1 || s == 3)) || (GATED && s == 4)) continue;
        if (to.place[s] < 0) continue;
        float *row = mine + to.place[s] * to.padded;
        if constexpr (GROUPS > 1) {                // rows of the same workgroup, in order
            __syncthreads();
#pragma unroll
            for (int k = 0; k < PIECES; ++k)
#pragma unroll
                for (int e = 0; e < VALUES; ++e)
                    if (e >= lane.twice[k]) shared_sums[threadIdx.x / LANES][lane.column[k] + e] = sums[s][k][e];
            __syncthreads();
            for (int c = threadIdx.x; c < a.width; c += THREADS) {
                float sum = 0.0f;
                for (int g = 0; g < GROUPS; ++g) sum += shared_sums[g][c];
                row[c] = sum;
            }
        } else {
#pragma unroll
            for (int k = 0; k < PIECES; ++k) {
                if (lane.twice[k] == 0) {
#pragma unroll
                    for (int e = 0; e < VALUES; e += 4)
                        *reinterpret_cast<f32x4 *>(row + lane.column[k] + e) = f32x4{sums[s][k][e], sums[s][k][e + 1], sums[s][k][e + 2], sums[s][k][e + 3]};
                } else {
#pragma unroll
                    for (int e = 0; e < VALUES; ++e)
                        if (e >= lane.twice[k]) row[lane.column[k] + e] = sums[s][k][e];
                }
            }
        }
    }
}

// ---- sums over the rows by themselves ----------------------------------------------------------------------------------
//
// Rows that are too long for their lanes to hold sums as well: with the means of every row known, a thread goes down the rows with one piece of them.  The operands are read a second
// time (3333 x 9000 bfloat16 725 us with sums that spilled out of the registers, 5000 x 6000 float 285).
template <typename T, int FORM> __global__ void __launch_bounds__(THREADS) norm_columns_kernel(NormArgs a, Partials to)
{
    constexpr int VALUES = Piece<T>::VALUES;
    constexpr bool BLOCK = FORM != NORM_ALONE, BIASES = FORM != BLOCK_GAINS && FORM != GATED_GAINS, GATED = FORM == GATED_GAINS || FORM == GATED_ALL;
    const int64_t col = ((int64_t)blockIdx.x * THREADS + threadIdx.x) * VALUES;
    if (col >= a.width) return;
    const RowAt<T> vectors(a, blockIdx.z, 0);
    const auto vector = [&](const T *p, float other, float (&v)[VALUES]) {
        Piece<T> x;
        if (p) {
            x = fetch_piece(p, col, a.width);
            settle_piece(x, col, a.width);
        }
#pragma unroll
        for (int e = 0; e < VALUES; ++e) v[e] = p ? x.get(e) : other;
    };
    float g1[VALUES], b1[VALUES], g2[VALUES], q[VALUES], gate[VALUES], slope[VALUES];
    vector(vectors.g2, 1.0f, g2);
    if constexpr (BLOCK) {
        vector(vectors.g1, 1.0f, g1);
        if constexpr (BIASES) vector(vectors.b1, 0.0f, b1);
        if constexpr (!GATED) {
            vector(vectors.q, 1.0f, q);
#pragma unroll
            for (int e = 0; e < VALUES; ++e) gate_of(vectors.q ? a.act : GATE_NONE, q[e], gate[e], slope[e]);
        }
    }
    float sums[SUMS][VALUES] = {};
    const auto fetch = [&](const Span &s, int64_t t) {
        Piece<T> x;
        x.v = decltype(x.v){};
        return s.p ? fetch_piece(RowAt<T>::at(s, blockIdx.z, t), col, a.width) : x;
    };
#pragma unroll 2
    for (int64_t t = blockIdx.y; t < a.rows; t += gridDim.y) {
        Piece<T> x = fetch(a.x, t), f, p, dy = fetch(a.dy, t), dh = fetch(a.dh, t);
        if constexpr (BLOCK) f = fetch(a.f, t);
        if constexpr (GATED) p = fetch(a.gate, t);
        const RowSums row = to.rows[blockIdx.z * a.rows + t];
        settle_piece(x, col, a.width);
        settle_piece(dy, col, a.width);
        settle_piece(dh, col, a.width);
        if constexpr (BLOCK) settle_piece(f, col, a.width);
        if constexpr (GATED) settle_piece(p, col, a.width);
#pragma unroll
        for (int e = 0; e < VALUES; ++e) {
            float fn = 0.0f, u = 0.0f, h = a.x_scale * x.get(e), value = 0.0f, D = dh.get(e);
            if constexpr (BLOCK) {
                fn = a.post ? unit_of(row.post, f.get(e)) : f.get(e);
                u = BIASES ? fmaf(fn, g1[e], b1[e]) : fn * g1[e];
                if constexpr (GATED) gate_of(a.act, p.get(e), value, slope[e]);
                else value = gate[e];
                value *= a.f_scale;
                h = fmaf(value, u, h);
            }
            if (a.pre) {
                const float hn = unit_of(row.pre, h), v = dy.get(e);
                D += row.pre.r * fmaf(-hn, row.mean_eh, v * g2[e] - row.mean_e);
                sums[2][e] = fmaf(v, hn, sums[2][e]);
                sums[3][e] += v;
            }
            if constexpr (BLOCK) {
                const float du = value * D;
                sums[0][e] = fmaf(du, fn, sums[0][e]);
                sums[1][e] += du;
                sums[4][e] = fmaf(u, D, sums[4][e]);
            }
        }
    }
    if constexpr (BLOCK && !GATED)
#pragma unroll
        for (int e = 0; e < VALUES; ++e) sums[4][e] *= a.f_scale * slope[e];
    float *mine = to.p + (blockIdx.z * to.workgroups + blockIdx.y) * to.sums * to.padded + col;
#pragma unroll
    for (int s = 0; s < SUMS; ++s)
        if (to.place[s] >= 0)
#pragma unroll
            for (int e = 0; e < VALUES; e += 4) *reinterpret_cast<f32x4 *>(mine + to.place[s] * to.padded + e) = f32x4{sums[s][e], sums[s][e + 1], sums[s][e + 2], sums[s][e + 3]};
}

// ---- launches --------------------------------------------------------------------------------------------------------

template <typename T> static int64_t pieces_of(int64_t width) { return (width + Piece<T>::VALUES - 1) / Piece<T>::VALUES; }

// Lanes and pieces for a row of n pieces; longer ones than any of them hold are streamed.  Two pieces for a lane while a wave's registers allow it: what a row's sums cost is shared by more
// values.  768 lanes: 6000 x 5000 float 103 us, with 1024 of them 150; 384 would be slower than 512 (6000 x 5000 bfloat16 60 us and 52).  Three and four pieces of float against rows read
// again: 2500 x 12000 113 us and 157, with a gate of rows and layer norms 168 and 280, a norm alone 55 and 72; 1831 x 16384 128 and 185, a norm alone 90 and 82.
// Rows of no more than a piece (4 float or 8 bfloat16 values) are too short to be read in whole pieces from their ends: they are streamed, by one thread of a workgroup, and slow where there are
// many (1000000 x 8 of a norm alone: bfloat16 1585 us and 3893 for the gradients, float, two pieces, 37 and 37; 1000 x 8 4.5 and 3.8 us, gradients 18 and 9.8).
template <int LANES_, int PIECES_> struct Held { static constexpr int LANES = LANES_, PIECES = PIECES_; };
template <typename T, class Go, class Long> static void with_row(const NormArgs &a, const Go &go, const Long &stream)
{
    const int64_t n = pieces_of<T>(a.width);
    if (n <= 1) stream();
    else if (n <= 8) go(Held<8, 1>());
    else if (n <= 16) go(Held<16, 1>());
    else if (n <= 32) go(Held<32, 1>());
    else if (n <= 64) go(Held<64, 1>());
    else if (n <= 128) go(Held<64, 2>());
    else if (n <= 256) go(Held<256, 1>());
    else if (n <= 512) go(Held<256, 2>());
    else if (n <= 1024) go(Held<512, 2>());
    else if (n <= 1536) go(Held<768, 2>());
    else if (n <= 2048) go(Held<1024, 2>());
    else if constexpr (sizeof(T) == 4) {
        if (n <= 3 * 1024) go(Held<1024, 3>());
        else if (a.f.p && n <= 4096) go(Held<1024, 4>());
        else stream();
    }
    else stream();
}

// Gradients hold sums over the rows as well: one piece for a lane as long as there are lanes, as few idle ones as whole waves allow (6000 x 5000 bfloat16 with a gate of rows: 181 us by 768
// lanes, 233 by 1024; 20000 x 1500: 152 by 192, 165 by 256).  Of longer rows the sums have a kernel of their own; float's still
// fit with two pieces (3662 x 8192 with a gate for all rows 161 us, by two kernels 259; with a gate of rows and biases 282 and 360).
// A norm alone has fewer sums, and two pieces for a lane pay where they keep the row in one wave (42857 x 700 bfloat16 49 us, one piece 74; 30000 x 1000 43 and 56) or in one kernel with
// few idle lanes (3333 x 9000 bfloat16 65 us, by two kernels 101; 6000 x 5000 float 93, by 1024 lanes 101); between the two, one piece is as fast or faster (7324 x 4096 bfloat16 51 and 53).
// Without the sums, lanes that fill a row: 3333 x 9000 float 283 us with three pieces (2 to 17 registers spilled) and 411 with four (27 to 131 spilled; layer norms, a gate of rows and biases 441
// and 661); bfloat16 172 us by 768 lanes (none spilled) and 197 by 1024 (286 and 391).  A norm alone has room for its sums here too (3333 x 9000 float 105 us, without them 137; 1831 x 16384
// bfloat16 69 and 80), but for float in four pieces (2142 x 14000 165 us, without them 134).  With sums, float rows in two pieces and biases spill 18 to 23 registers.
template <int LANES_, int PIECES_, bool SUMMED_> struct HeldGrad { static constexpr int LANES = LANES_, PIECES = PIECES_; static constexpr bool SUMMED = SUMMED_; };
template <typename T, class Go, class Long> static void with_row_grad(const NormArgs &a, const Go &go, const Long &stream)
{
    const int64_t n = pieces_of<T>(a.width);
    if (n <= 1) stream();
    else if (n <= 8) go(HeldGrad<8, 1, true>());
    else if (n <= 16) go(HeldGrad<16, 1, true>());
    else if (n <= 32) go(HeldGrad<32, 1, true>());
    else if (n <= 64) go(HeldGrad<64, 1, true>());
    else if (!a.f.p && n <= 128) go(HeldGrad<64, 2, true>());
    else if (n <= 128) go(HeldGrad<128, 1, true>());
    else if (n <= 192) go(HeldGrad<192, 1, true>());
    else if (n <= 256) go(HeldGrad<256, 1, true>());
    else if (n <= 384) go(HeldGrad<384, 1, true>());
    else if (n <= 512) go(HeldGrad<512, 1, true>());
    else if (n <= 768) go(HeldGrad<768, 1, true>());
    else if (n <= 1024) go(HeldGrad<1024, 1, true>());
    else if (!a.f.p && n <= 1536) go(HeldGrad<768, 2, true>());
    else if constexpr (sizeof(T) == 4) {
        if (n <= 2048) go(HeldGrad<1024, 2, true>());
        else if (!a.f.p && n <= 3 * 1024) go(HeldGrad<1024, 3, true>());
        else if (n <= 3 * 1024) go(HeldGrad<1024, 3, false>());
        else if (n <= 4096) go(HeldGrad<1024, 4, false>());
        else stream();
    } else if (n <= 1536) {
        go(HeldGrad<768, 2, false>());
    } else if (!a.f.p && n <= 2048) {
        go(HeldGrad<1024, 2, true>());
    } else if (n <= 2048) {
        go(HeldGrad<1024, 2, false>());
    }
    else stream();
}

template <typename T> static void block_norm_of(hipStream_t s, const NormArgs &a)
{
    with_row<T>(a, [&](auto held) {
        constexpr int LANES = decltype(held)::LANES, PIECES = decltype(held)::PIECES, GROUPS = threads_of(LANES) / LANES;
        // threads along a dimension of a launch have to be fewer than 2^32
        const int64_t n = (a.rows + GROUPS - 1) / GROUPS, across = n < (1 << 20) ? n : 1 << 20;
        const dim3 grid((uint32_t)across, (uint32_t)((n + across - 1) / across), (uint32_t)a.batch);
        if (a.layer) norm_kernel<T, LANES, PIECES, true><<<grid, threads_of(LANES), 0, s>>>(a);
        else norm_kernel<T, LANES, PIECES, false><<<grid, threads_of(LANES), 0, s>>>(a);
    }, [&]() {
        long_norm_kernel<T><<<dim3((uint32_t)(a.rows < (1 << 20) ? a.rows : 1 << 20), (uint32_t)a.batch), THREADS, 0, s>>>(a);
    });
}

void launch_block_norm(hipStream_t s, const NormArgs &a)
{
    if (a.batch == 0 || a.rows == 0) return;
    if (a.bf16) block_norm_of<uint16_t>(s, a);
    else block_norm_of<float>(s, a);
}

// Whether rows are written over rows that are read.
static bool in_place(const NormArgs &a)
{
    for (const Span *o : {&a.dx, &a.df, &a.dgate})
        for (const Span *i : {&a.dy, &a.dh, &a.x, &a.f, &a.gate})
            if (o->p && o->p == i->p) return true;
    return false;
}

struct GradPlan { Partials to; bool summed, twice; };               // sums held by the rows' kernel; that one run twice

template <typename T> static GradPlan grad_plan(const NormArgs &a, void *work)
{
    GradPlan plan{};
    Partials &to = plan.to;
    const Span *const outs[SUMS] = {&a.dpost_gain, &a.dpost_bias, &a.dpre_gain, &a.dpre_bias, &a.dgate};
    for (int s = 0; s < SUMS; ++s) {
        const bool there = outs[s]->p && !(s == 4 && a.gate_rows);
        to.place[s] = there ? to.sums : -1;
        if (there) to.out[to.sums++] = *outs[s];
    }
    to.padded = up_to(a.width, 8);
    int64_t rows = 1, threads = THREADS;           // rows of a workgroup at once
    with_row_grad<T>(a, [&](auto held) {
        threads = threads_of(decltype(held)::LANES);
        rows = threads / decltype(held)::LANES;
        plan.summed = decltype(held)::SUMMED;
    }, []() { });
    // as many as the card holds at once, if each has two turns
    const int64_t places = 256 * (1024 / threads), most = a.batch * 8 < places ? places / a.batch : 8, turns = (a.rows + rows - 1) / rows, all = (turns + 1) / 2;
    to.workgroups = to.row_workgroups = all < most ? all : most;
    if (!plan.summed) {                            // eight workgroups of the columns' kernel on every compute unit
        const int64_t slabs = (pieces_of<T>(a.width) + THREADS - 1) / THREADS, blocks = 2048 / (slabs * a.batch);
        to.workgroups = std::min(std::max<int64_t>(blocks, 1), a.rows);
    }
    // the rows' kernel leaves the means for the columns' kernel, which needs the operands as they were
    plan.twice = !plan.summed && to.sums > 0 && in_place(a);
    const bool all_wanted = !plan.twice && a.dx.p && (!a.f.p || a.df.p) && (!a.f.p || !a.gate_rows || !a.gate.p || a.dgate.p);
    char *at = (char *)work;
    const auto take = [&](int64_t n) { char *p = at; at += up_to(n, 256); return p; };
    to.p = (float *)take(4 * a.batch * to.workgroups * to.sums * to.padded);
    to.rows = (RowSums *)take(!plan.summed && to.sums > 0 ? (int64_t)sizeof(RowSums) * a.batch * a.rows : 0);
    to.unwanted = take(all_wanted ? 0 : (int64_t)sizeof(T) * a.batch * to.row_workgroups * rows * to.padded);
    if (plan.summed || to.sums == 0) to.rows = nullptr;
    to.bytes = at - (char *)work;
    return plan;
}

int64_t block_norm_grad_workspace(const NormArgs &a)
{
    if (a.batch == 0) return 0;
    return a.bf16 ? grad_plan<uint16_t>(a, nullptr).to.bytes : grad_plan<float>(a, nullptr).to.bytes;
}

// go(form): what kind of block it is.
template <class Go> static void with_form(const NormArgs &a, const Partials &to, const Go &go)
{
    const bool gated = a.gate_rows && a.gate.p, biases = a.post_bias.p || to.place[1] >= 0 || to.place[3] >= 0;
    if (!a.f.p) go(std::integral_constant<int, NORM_ALONE>());
    else if (gated && biases) go(std::integral_constant<int, GATED_ALL>());
    else if (gated) go(std::integral_constant<int, GATED_GAINS>());
    else if (biases) go(std::integral_constant<int, BLOCK_ALL>());
    else go(std::integral_constant<int, BLOCK_GAINS>());
}

template <typename T> static void launch_rows(hipStream_t s, const NormArgs &a, const GradPlan &plan)
{
    if (plan.to.row_workgroups == 0) return;
    const dim3 grid((uint32_t)plan.to.row_workgroups, (uint32_t)a.batch);
    with_row_grad<T>(a, [&](auto held) {
        constexpr int LANES = decltype(held)::LANES, PIECES = decltype(held)::PIECES;
        constexpr bool SUMMED = decltype(held)::SUMMED;
        with_form(a, plan.to, [&](auto form) {
            // what with_row_grad asks for of a norm alone, and of a block
            if constexpr (form() == NORM_ALONE ? LANES != 128 && (SUMMED || PIECES == 4) : PIECES == 1 || !SUMMED || (sizeof(T) == 4 && LANES == 1024 && PIECES == 2)) {
                if (a.layer) norm_grad_kernel<T, LANES, PIECES, true, form(), SUMMED><<<grid, threads_of(LANES), 0, s>>>(a, plan.to);
                else norm_grad_kernel<T, LANES, PIECES, false, form(), SUMMED><<<grid, threads_of(LANES), 0, s>>>(a, plan.to);
            }
        });
    }, [&]() {
        long_norm_grad_kernel<T><<<grid, THREADS, 0, s>>>(a, plan.to);
    });
}

template <typename T> static void block_norm_grad_of(hipStream_t s, const NormArgs &a, void *work)
{
    const GradPlan plan = grad_plan<T>(a, work);
    const Partials &to = plan.to;
    if (plan.twice) {
        NormArgs means = a;
        means.dx.p = means.df.p = nullptr;
        if (a.gate_rows) means.dgate.p = nullptr;
        launch_rows<T>(s, means, plan);
    } else {
        launch_rows<T>(s, a, plan);
    }
    if (!plan.summed && to.sums > 0 && a.rows > 0) {
        const dim3 grid((uint32_t)((pieces_of<T>(a.width) + THREADS - 1) / THREADS), (uint32_t)to.workgroups, (uint32_t)a.batch);
        with_form(a, to, [&](auto form) { norm_columns_kernel<T, form()><<<grid, THREADS, 0, s>>>(a, to); });
    }
    if (to.sums > 0) join_sums_kernel<T><<<dim3((uint32_t)((a.width + JOIN_COLUMNS - 1) / JOIN_COLUMNS), to.sums, (uint32_t)a.batch), JOIN_COLUMNS * JOIN_TURNS, 0, s>>>(a, to);
    if (plan.twice) launch_rows<T>(s, a, plan);
}

void launch_block_norm_grad(hipStream_t s, const NormArgs &a, void *work)
{
    if (a.batch == 0) return;
    if (a.bf16) block_norm_grad_of<uint16_t>(s, a, work);
    else block_norm_grad_of<float>(s, a, work);
}

}  // namespace netmax
