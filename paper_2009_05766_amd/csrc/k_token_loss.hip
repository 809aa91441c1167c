// The clipped policy loss with a KL term and the loss of paired log ratios, on the logits of sampled tokens.
//
// For a row z with label y:  log p = z_y - max z - log sum exp(z - max z),  d log p / d z_j = [j = y] - p_j,
// so that a loss whose derivative by log p is s has the gradient s ([j = y] - p_j).
//   policy      r = exp(log p - old);  l = w (-min(r A, clip(r, 1 - low, 1 + high) A) + kl (exp(ref - log p) - (ref - log p) - 1))
//   preference  R_q = sum over the sequence of w (log p - ref);  h = beta (R_chosen - R_rejected);
//               l = scale (-(1 - e) log sigma(h) - e log sigma(-h)),  dl / dh = scale (sigma(h) - (1 - e))
// Bound by memory: a row is read, and its gradient written.  A workgroup keeps a row in registers between the two, up to 65536 float or 131072 bfloat16
// logits (longer rows are read twice).  Sums of exponentials are held in float, log probabilities and their sums over a sequence in double.
//
// A thread takes its exponentials piece by piece as the row arrives, relative to the largest value that it has seen, and brings its sum down where a piece
// has a larger one: the exponential of a value that decides the row is then 1, and its log probability is not spoilt by the rounding of a large argument
// (2^-24 of it).  Pieces are counted from the row's first value, wherever that lies in memory, so that a row's results do not depend on its place.
//
// policy, 8192 x 131072 bfloat16 (a row in ten without weight): 795 us for 4.08 GB, the rate of a large copy (5.1 TB/s); read twice, without
// registers, 2.7 ms.  preference, 16384 x 50000 (a quarter without weight): rows 233 us, gradient 518 us for 1.23 and 2.87 GB: the slopes of a
// sequence's rows depend on all of them, so rows that count are read twice.
#include "gemm.h"
#include "token_loss.h"

#include <type_traits>

namespace netmax {

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LOWEST = -0x1.fffffep127f;         // less than any value but -inf, and differences to it are no NaN

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

template <typename T> struct Row {
    T *p; int64_t vocab;
    __device__ __forceinline__ Row(const T *row, int64_t vocab_) : p(const_cast<T *>(row)), vocab(vocab_) { }
    __device__ __forceinline__ int64_t pieces() const { return (vocab + Piece<T>::VALUES - 1) / Piece<T>::VALUES; }
    // values behind the row are -inf
    __device__ __forceinline__ Piece<T> load(int64_t c) const
    {
        constexpr int VALUES = Piece<T>::VALUES;
        const int64_t j = c * VALUES;
        Piece<T> x;
        if (j + VALUES <= vocab) {
            x.v = *reinterpret_cast<const typename Piece<T>::Memory *>(p + j);
        } else {
            float v[VALUES];
#pragma unroll
            for (int k = 0; k < VALUES; ++k) v[k] = j + k < vocab ? load_value(p + j + k) : -INFINITY;
            x.set(v);
        }
        return x;
    }
    __device__ __forceinline__ void store(int64_t c, const Piece<T> &x) const
    {
        constexpr int VALUES = Piece<T>::VALUES;
        const int64_t j = c * VALUES;
        if (j + VALUES <= vocab) {
            *reinterpret_cast<typename Piece<T>::Memory *>(p + j) = x.v;
        } else {
#pragma unroll
            for (int k = 0; k < VALUES; ++k)
                if (j + k < vocab) store_value(p + j + k, x.get(k));
        }
    }
};

// sum = the sum of exp(z - top) over some values; no value yet (or only -inf): {-inf, 0}.
struct Partial {
    float top, sum;
    __device__ __forceinline__ void join(float t, float u)
    {
        const float m = fmaxf(top, t);
        if (m == -INFINITY) { sum += u; return; }                   // nothing on either side, or a NaN
        sum = sum * __expf(top - m) + u * __expf(t - m);
        top = m;
    }
};

__device__ __forceinline__ float exp_from(float z, float top) { return __builtin_amdgcn_exp2f((z - top) * LOG2E); }
// The same where top may be -inf: values of -inf have 0 then, too.
__device__ __forceinline__ float exp_or_zero(float z, float top) { return z > -INFINITY ? exp_from(z, top) : z != z ? z : 0.0f; }

template <int THREADS> __device__ __forceinline__ Partial join_workgroup(Partial r)
{
    __shared__ float tops[THREADS / 64], sums[THREADS / 64];
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) r.join(__shfl_xor(r.top, d), __shfl_xor(r.sum, d));
    if ((threadIdx.x & 63) == 0) { tops[threadIdx.x >> 6] = r.top; sums[threadIdx.x >> 6] = r.sum; }
    __syncthreads();
    r.top = tops[threadIdx.x & (THREADS / 64 - 1)]; r.sum = sums[threadIdx.x & (THREADS / 64 - 1)];
#pragma unroll
    for (int d = THREADS / 128; d > 0; d >>= 1) r.join(__shfl_xor(r.top, d), __shfl_xor(r.sum, d));
    return r;
}

// The row's sum, with PIECES pieces per thread left in `held`.
template <typename T, int THREADS, int PIECES> __device__ __forceinline__ Partial held_sum(const Row<T> &z, Piece<T> (&held)[PIECES])
{
    constexpr int VALUES = Piece<T>::VALUES;
    const int64_t n = z.pieces();
#pragma unroll
    for (int k = 0; k < PIECES; ++k)
        if (k * THREADS + (int)threadIdx.x < n) held[k] = z.load(k * THREADS + (int)threadIdx.x);
    Partial r = {LOWEST, 0.0f};
#pragma unroll
    for (int k = 0; k < PIECES; ++k)
        if (k * THREADS + (int)threadIdx.x < n) {
            float top = r.top, part[VALUES];
#pragma unroll
            for (int e = 0; e < VALUES; ++e) top = fmaxf(top, held[k].get(e));
#pragma unroll
            for (int e = 0; e < VALUES; ++e) part[e] = exp_from(held[k].get(e), top);
#pragma unroll
            for (int d = VALUES / 2; d > 0; d >>= 1)
#pragma unroll
                for (int e = 0; e < d; ++e) part[e] += part[e + d];
            r.sum = fmaf(r.sum, exp_from(r.top, top), part[0]);
            r.top = top;
        }
    if (r.sum == 0.0f) r.top = -INFINITY;
    return join_workgroup<THREADS>(r);
}

// The same for a row of any length, which is not kept.
template <typename T, int THREADS> __device__ __forceinline__ Partial streamed_sum(const Row<T> &z)
{
    const int64_t n = z.pieces();
    Partial r = {-INFINITY, 0.0f};
    for (int64_t c = threadIdx.x; c < n; c += THREADS) {
        const Piece<T> x = z.load(c);
        float top = -INFINITY, sum = 0.0f;
#pragma unroll
        for (int e = 0; e < Piece<T>::VALUES; ++e) top = fmaxf(top, x.get(e));
#pragma unroll
        for (int e = 0; e < Piece<T>::VALUES; ++e) sum += exp_or_zero(x.get(e), top);
        r.join(top, sum);
    }
    return join_workgroup<THREADS>(r);
}

// What the gradient of a row needs to know: its exponentials are taken from `top`, `scale` is -slope over their sum.  top = -inf: a row of nothing
// but -inf, whose probabilities are 0.
struct Slope {
    float top, scale, slope; int64_t label;
    __device__ __forceinline__ Slope(float top_, float inverse, float slope_, int64_t label_)
        : top(top_ > -INFINITY || top_ != top_ ? top_ : 0.0f), scale(-slope_ * inverse), slope(slope_), label(label_) { }
};

// slope ([j = label] - p_j) for piece c.
template <typename T> __device__ __forceinline__ Piece<T> gradient_of(const Piece<T> &x, int64_t c, const Slope &s)
{
    constexpr int VALUES = Piece<T>::VALUES;
    float g[VALUES];
#pragma unroll
    for (int e = 0; e < VALUES; ++e) g[e] = s.scale * exp_from(x.get(e), s.top);
    if (s.label / VALUES == c)
#pragma unroll
        for (int e = 0; e < VALUES; ++e)
            if (c * VALUES + e == s.label) g[e] += s.slope;
    Piece<T> out;
    out.set(g);
    return out;
}

template <typename T, int THREADS> __device__ __forceinline__ void write_zeros(const Row<T> &to)
{
    const float zeros[Piece<T>::VALUES] = {};
    Piece<T> x;
    x.set(zeros);
    const int64_t n = to.pieces();
    for (int64_t c = threadIdx.x; c < n; c += THREADS) to.store(c, x);
}

template <typename T, int THREADS> __device__ __forceinline__ void streamed_gradient(const Row<T> &z, const Row<T> &to, const Slope &s)
{
    const int64_t n = z.pieces();
#pragma unroll 4
    for (int64_t c = threadIdx.x; c < n; c += THREADS) to.store(c, gradient_of<T>(z.load(c), c, s));
}

__device__ __forceinline__ bool row_counts(const TokenRows &rows, int64_t t, float &w, int &label)
{
    w = rows.weight ? rows.weight[t] : 1.0f;
    label = rows.labels[t];
    return w != 0.0f && label >= 0 && label < rows.vocab;
}

// The label's log probability: zy - top - log(sum).
__device__ __forceinline__ double label_logp(float zy, const Partial &r)
{
    if (r.top == -INFINITY) return r.sum != r.sum ? (double)r.sum : -INFINITY;      // no logit that is more than -inf
    return (double)zy - (double)r.top - log((double)r.sum);
}

// A workgroup per row (or pair): threads along a dimension of a launch have to be fewer than 2^32, so many rows take two.
static dim3 grid_of(int64_t rows)
{
    constexpr int64_t ACROSS = 1 << 21;
    return dim3((uint32_t)(rows < ACROSS ? rows : ACROSS), (uint32_t)((rows + ACROSS - 1) / ACROSS));
}
__device__ __forceinline__ int64_t workgroup() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }

// PIECES = 0: the row is read twice.
template <typename T, int THREADS, int PIECES>
__global__ void __launch_bounds__(THREADS) policy_loss_kernel(TokenRows rows, PolicyArgs a)
{
    const int64_t t = workgroup();
    if (t >= rows.tokens) return;
    const Row<T> z((const T *)rows.logits + t * rows.ld, rows.vocab), out((T *)a.grad + t * a.ldg, rows.vocab);
    float w;
    int label;
    if (!row_counts(rows, t, w, label)) {
        if (threadIdx.x == 0) { a.loss[t] = 0.0f; if (a.logp) a.logp[t] = 0.0f; }
        if (a.grad) write_zeros<T, THREADS>(out);
        return;
    }
    const float zy = load_value(z.p + label);
    Piece<T> held[PIECES > 0 ? PIECES : 1];
    Partial r;
    if constexpr (PIECES > 0) r = held_sum<T, THREADS, PIECES>(z, held);
    else r = streamed_sum<T, THREADS>(z);
    const double logp = label_logp(zy, r);
    const float adv = a.advantage[t], ratio = expf((float)(logp - (double)a.old_logp[t]));
    // a ratio past the type's range is inf, and no advantage is none of it
    const float kept = fminf(fmaxf(ratio, 1.0f - a.low), 1.0f + a.high), free = adv == 0.0f && ratio == INFINITY ? 0.0f : ratio * adv, clipped = kept * adv;
    float loss = free <= clipped ? -free : clipped < free ? -clipped : free + clipped, slope = free <= clipped ? -free : clipped < free ? 0.0f : free + clipped;
    if (a.ref_logp && a.kl != 0.0f) {
        const float d = (float)((double)a.ref_logp[t] - logp), more = expm1f(d);
        loss += a.kl * (more < INFINITY ? more - d : more);          // exp(d) past the type's range: inf, not inf - inf
        slope -= a.kl * more;
    }
    if (threadIdx.x == 0) { a.loss[t] = w * loss; if (a.logp) a.logp[t] = (float)logp; }
    if (!a.grad) return;
    slope *= w;
    if (slope == 0.0f && r.sum == r.sum) {
        write_zeros<T, THREADS>(out);
        return;
    }
    const Slope s(r.top, r.sum > 0.0f ? 1.0f / r.sum : r.sum, slope, label);
    if constexpr (PIECES > 0) {
#pragma unroll
        for (int k = 0; k < PIECES; ++k) {
            const int64_t c = k * THREADS + (int)threadIdx.x;
            if (c < z.pieces()) out.store(c, gradient_of<T>(held[k], c, s));
        }
    } else {
        streamed_gradient<T, THREADS>(z, out, s);
    }
}

template <typename T, int THREADS, int PIECES>
__global__ void __launch_bounds__(THREADS) preference_rows_kernel(TokenRows rows, PreferenceArgs a)
{
    const int64_t t = workgroup();
    if (t >= rows.tokens) return;
    const Row<T> z((const T *)rows.logits + t * rows.ld, rows.vocab);
    float w;
    int label;
    if (!row_counts(rows, t, w, label)) {
        if (threadIdx.x == 0) a.terms[t] = 0.0;
        return;
    }
    const float zy = load_value(z.p + label);
    Piece<T> held[PIECES > 0 ? PIECES : 1];
    Partial r;
    if constexpr (PIECES > 0) r = held_sum<T, THREADS, PIECES>(z, held);
    else r = streamed_sum<T, THREADS>(z);
    if (threadIdx.x == 0) {
        a.terms[t] = (double)w * (label_logp(zy, r) - (double)a.ref_logp[t]);
        a.stats[t] = make_float2(r.top, r.sum > 0.0f ? 1.0f / r.sum : r.sum);
    }
}

constexpr int PAIR_THREADS = 256;

// The rows of sequence q that lie inside the matrix.
__device__ __forceinline__ void sequence_rows(const int32_t *offsets, int64_t q, int64_t tokens, int64_t &first, int64_t &end)
{
    first = offsets[q] < 0 ? 0 : offsets[q];
    end = offsets[q + 1] > tokens ? tokens : offsets[q + 1];
}

// One workgroup per pair: the sums over both sequences in a fixed order, the pair's loss and the slopes of its rows.
__global__ void __launch_bounds__(PAIR_THREADS) preference_pairs_kernel(int64_t tokens, PreferenceArgs a)
{
    __shared__ double part[2][PAIR_THREADS];
    const int64_t p = workgroup();
    if (p >= a.pairs) return;
    for (int side = 0; side < 2; ++side) {
        int64_t first, end;
        sequence_rows(a.offsets, 2 * p + side, tokens, first, end);
        double sum = 0.0;
        for (int64_t t = first + threadIdx.x; t < end; t += PAIR_THREADS) sum += a.terms[t];
        part[side][threadIdx.x] = sum;
    }
    __syncthreads();
    for (int d = PAIR_THREADS / 2; d > 0; d >>= 1) {
        if ((int)threadIdx.x < d)
            for (int side = 0; side < 2; ++side) part[side][threadIdx.x] += part[side][threadIdx.x + d];
        __syncthreads();
    }
    if (threadIdx.x != 0) return;
    const double e = a.smoothing, h = (double)a.beta * (part[0][0] - part[1][0]), tail = log1p(exp(-fabs(h)));
    const double below = tail + (h < 0.0 ? -h : 0.0), above = tail + (h > 0.0 ? h : 0.0);       // -log sigma(h), -log sigma(-h)
    const double dh = h >= 0.0 ? e - exp(-h) / (1.0 + exp(-h)) : exp(h) / (1.0 + exp(h)) - (1.0 - e);
    // a sequence with a masked label has the ratio -inf and h may be infinite: a term without weight is left out, 0 inf would be no number
    a.loss[p] = (float)((double)a.scale * ((e < 1.0 ? (1.0 - e) * below : 0.0) + (e > 0.0 ? e * above : 0.0)));
    for (int side = 0; side < 2; ++side) {
        a.ratio[2 * p + side] = (float)part[side][0];
        a.slope[2 * p + side] = (float)((double)a.scale * (double)a.beta * (side ? -dh : dh));
    }
}

// Rows in the reverse order of preference_rows_kernel's, so that those it read last come first: they may still be in the last cache.
template <typename T, int THREADS>
__global__ void __launch_bounds__(THREADS) preference_gradient_kernel(TokenRows rows, PreferenceArgs a)
{
    const int64_t t = rows.tokens - 1 - workgroup();
    if (t < 0) return;
    const Row<T> z((const T *)rows.logits + t * rows.ld, rows.vocab), out((T *)a.grad + t * a.ldg, rows.vocab);
    float w;
    int label;
    int64_t lo = 0, hi = 2 * a.pairs;                               // the sequence is in lo .. hi - 1
    while (hi - lo > 1) {
        const int64_t mid = (lo + hi) / 2;
        if ((int64_t)a.offsets[mid] <= t) lo = mid; else hi = mid;
    }
    int64_t first, end;
    sequence_rows(a.offsets, lo, rows.tokens, first, end);
    if (t < first || t >= end || !row_counts(rows, t, w, label)) {
        write_zeros<T, THREADS>(out);
        return;
    }
    const float2 st = a.stats[t];
    streamed_gradient<T, THREADS>(z, out, Slope(st.x, st.y, w * a.slope[lo], label));
}

// Workgroups and pieces per thread by the length of a row: the fewest threads with few pieces each, so that several rows share a compute unit.
template <typename T, class Go> static void with_row(int64_t vocab, const Go &go)
{
    const int64_t n = (vocab + Piece<T>::VALUES - 1) / Piece<T>::VALUES;
    if (n <= 256 * 2) go(std::integral_constant<int, 256>(), std::integral_constant<int, 2>());
    else if (n <= 256 * 4) go(std::integral_constant<int, 256>(), std::integral_constant<int, 4>());
    else if (n <= 512 * 4) go(std::integral_constant<int, 512>(), std::integral_constant<int, 4>());
    else if (n <= 512 * 8) go(std::integral_constant<int, 512>(), std::integral_constant<int, 8>());
    else if (n <= 1024 * 8) go(std::integral_constant<int, 1024>(), std::integral_constant<int, 8>());
    else if (n <= 1024 * 16) go(std::integral_constant<int, 1024>(), std::integral_constant<int, 16>());
    else go(std::integral_constant<int, 1024>(), std::integral_constant<int, 0>());
}

template <typename T> static void policy_of(hipStream_t s, const TokenRows &rows, const PolicyArgs &a)
{
    with_row<T>(rows.vocab, [&](auto threads, auto pieces) {
        policy_loss_kernel<T, threads(), pieces()><<<grid_of(rows.tokens), threads(), 0, s>>>(rows, a);
    });
}

void launch_policy_loss(hipStream_t s, const TokenRows &rows, const PolicyArgs &a)
{
    if (rows.tokens == 0) return;
    if (rows.bf16) policy_of<uint16_t>(s, rows, a);
    else policy_of<float>(s, rows, a);
}

template <typename T> static void preference_of(hipStream_t s, const TokenRows &rows, const PreferenceArgs &a)
{
    with_row<T>(rows.vocab, [&](auto threads, auto pieces) {
        if (rows.tokens > 0) preference_rows_kernel<T, threads(), pieces()><<<grid_of(rows.tokens), threads(), 0, s>>>(rows, a);
        preference_pairs_kernel<<<grid_of(a.pairs), PAIR_THREADS, 0, s>>>(rows.tokens, a);
        if (rows.tokens > 0 && a.grad) preference_gradient_kernel<T, threads() < 512 ? 256 : 512><<<grid_of(rows.tokens), threads() < 512 ? 256 : 512, 0, s>>>(rows, a);
    });
}

void launch_preference_loss(hipStream_t s, const TokenRows &rows, const PreferenceArgs &a)
{
    if (rows.bf16) preference_of<uint16_t>(s, rows, a);
    else preference_of<float>(s, rows, a);
}

}  // namespace netmax
