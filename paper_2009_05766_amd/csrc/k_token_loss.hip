// The clipped policy loss with a KL term and the loss of paired log ratios, on the logits of sampled tokens.
//
// For a row z with label y:  log p = z_y - max z - log sum exp(z - max z),  d log p / d z_j = [j = y] - p_j,
// so that a loss whose derivative by log p is s has the gradient s ([j = y] - p_j).
//   policy      r = exp(log p - old);  l = w (-min(r A, clip(r, 1 - low, 1 + high) A) + kl (exp(ref - log p) - (ref - log p) - 1))
//   preference  R_q = sum over the sequence of w (log p - ref);  h = beta (R_chosen - R_rejected);
//               l = scale (-(1 - e) log sigma(h) - e log sigma(-h)),  dl / dh = scale (sigma(h) - (1 - e))
// Bound by memory: a row is read, and its gradient written.  Sums of exponentials are held in float, log probabilities and their sums
// over a sequence in double.
#include "gemm.h"
#include "token_loss.h"

namespace netmax {

constexpr int ROW_THREADS = 256;

// Maximum and sum of exp(z - maximum) of the values seen so far; no value yet (or only -inf): {-inf, 0}.
struct RunningSum {
    float top = -INFINITY, sum = 0.0f;
    __device__ __forceinline__ void add(float v)
    {
        if (v > top) { sum = sum * __expf(top - v) + 1.0f; top = v; }
        else if (v > -INFINITY) sum += __expf(v - top);
        else if (v != v) { sum = v; }                               // a NaN stays one
    }
    __device__ __forceinline__ void join(float t, float u)
    {
        const float m = fmaxf(top, t);
        if (m == -INFINITY) { sum += u; return; }                   // nothing on either side, or a NaN
        sum = sum * __expf(top - m) + u * __expf(t - m);
        top = m;
    }
};

__device__ __forceinline__ RunningSum join_workgroup(RunningSum r)
{
    __shared__ float tops[ROW_THREADS / 64], sums[ROW_THREADS / 64];
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) r.join(__shfl_xor(r.top, d), __shfl_xor(r.sum, d));
    if ((threadIdx.x & 63) == 0) { tops[threadIdx.x >> 6] = r.top; sums[threadIdx.x >> 6] = r.sum; }
    __syncthreads();
    r.top = tops[0]; r.sum = sums[0];
    for (int k = 1; k < ROW_THREADS / 64; ++k) r.join(tops[k], sums[k]);
    return r;
}

template <typename T> __device__ __forceinline__ RunningSum row_sum(const T *z, int64_t vocab)
{
    RunningSum r;
    for (int64_t j = threadIdx.x; j < vocab; j += ROW_THREADS) r.add(load_value(z + j));
    return join_workgroup(r);
}

// slope ([j = label] - p_j); z and out may be the same memory.
template <typename T> __device__ __forceinline__ void write_gradient(const T *z, T *out, int64_t vocab, float top, float inv, float slope, int label)
{
    for (int64_t j = threadIdx.x; j < vocab; j += ROW_THREADS) {
        const float v = load_value(z + j), p = v > -INFINITY ? __expf(v - top) * inv : v != v ? v : 0.0f;
        store_value(out + j, j == label ? slope - slope * p : -slope * p);
    }
}

template <typename T> __device__ __forceinline__ void write_zeros(T *out, int64_t vocab)
{
    for (int64_t j = threadIdx.x; j < vocab; j += ROW_THREADS) out[j] = T(0);
}

__device__ __forceinline__ bool row_counts(const TokenRows &rows, int64_t t, float &w, int &label)
{
    w = rows.weight ? rows.weight[t] : 1.0f;
    label = rows.labels[t];
    return w != 0.0f && label >= 0 && label < rows.vocab;
}

__device__ __forceinline__ double label_logp(float zy, const RunningSum &r)
{
    if (r.top == -INFINITY) return r.sum != r.sum ? (double)r.sum : -INFINITY;      // no logit that is more than -inf
    return (double)zy - (double)r.top - log((double)r.sum);
}

template <typename T> __global__ void __launch_bounds__(ROW_THREADS)
policy_loss_kernel(TokenRows rows, PolicyArgs a)
{
    const int64_t t = blockIdx.x;
    const T *z = (const T *)rows.logits + t * rows.ld;
    T *out = a.grad ? (T *)a.grad + t * a.ldg : nullptr;
    float w;
    int label;
    if (!row_counts(rows, t, w, label)) {
        if (threadIdx.x == 0) { a.loss[t] = 0.0f; if (a.logp) a.logp[t] = 0.0f; }
        if (out) write_zeros(out, rows.vocab);
        return;
    }
    const float zy = load_value(z + label);
    const RunningSum r = row_sum(z, rows.vocab);
    const double logp = label_logp(zy, r);
    const float adv = a.advantage[t], ratio = expf((float)(logp - (double)a.old_logp[t]));
    const float kept = fminf(fmaxf(ratio, 1.0f - a.low), 1.0f + a.high), free = ratio * adv, clipped = kept * adv;
    float loss = free <= clipped ? -free : clipped < free ? -clipped : free + clipped, slope = free <= clipped ? -free : clipped < free ? 0.0f : free + clipped;
    if (a.ref_logp && a.kl != 0.0f) {
        const float d = (float)((double)a.ref_logp[t] - logp), more = expm1f(d);
        loss += a.kl * (more < INFINITY ? more - d : more);          // exp(d) past the type's range: inf, not inf - inf
        slope -= a.kl * more;
    }
    if (threadIdx.x == 0) { a.loss[t] = w * loss; if (a.logp) a.logp[t] = (float)logp; }
    if (out) write_gradient(z, out, rows.vocab, r.top, 1.0f / r.sum, w * slope, label);
}

template <typename T> __global__ void __launch_bounds__(ROW_THREADS)
preference_rows_kernel(TokenRows rows, PreferenceArgs a)
{
    const int64_t t = blockIdx.x;
    const T *z = (const T *)rows.logits + t * rows.ld;
    float w;
    int label;
    if (!row_counts(rows, t, w, label)) {
        if (threadIdx.x == 0) a.terms[t] = 0.0;
        return;
    }
    const float zy = load_value(z + label);
    const RunningSum r = row_sum(z, rows.vocab);
    if (threadIdx.x == 0) {
        a.terms[t] = (double)w * (label_logp(zy, r) - (double)a.ref_logp[t]);
        a.stats[t] = make_float2(r.top, 1.0f / r.sum);
    }
}

// The rows of sequence q that lie inside the matrix.
__device__ __forceinline__ void sequence_rows(const int32_t *offsets, int64_t q, int64_t tokens, int64_t &first, int64_t &end)
{
    first = offsets[q] < 0 ? 0 : offsets[q];
    end = offsets[q + 1] > tokens ? tokens : offsets[q + 1];
}

// One workgroup per pair: the sums over both sequences in a fixed order, the pair's loss and the slopes of its rows.
__global__ void __launch_bounds__(ROW_THREADS) preference_pairs_kernel(int64_t tokens, PreferenceArgs a)
{
    __shared__ double part[2][ROW_THREADS];
    for (int side = 0; side < 2; ++side) {
        int64_t first, end;
        sequence_rows(a.offsets, 2 * (int64_t)blockIdx.x + side, tokens, first, end);
        double sum = 0.0;
        for (int64_t t = first + threadIdx.x; t < end; t += ROW_THREADS) sum += a.terms[t];
        part[side][threadIdx.x] = sum;
    }
    __syncthreads();
    for (int d = ROW_THREADS / 2; d > 0; d >>= 1) {
        if ((int)threadIdx.x < d)
            for (int side = 0; side < 2; ++side) part[side][threadIdx.x] += part[side][threadIdx.x + d];
        __syncthreads();
    }
    if (threadIdx.x != 0) return;
    const int64_t p = blockIdx.x;
    const double e = a.smoothing, h = (double)a.beta * (part[0][0] - part[1][0]), tail = log1p(exp(-fabs(h)));
    const double below = tail + (h < 0.0 ? -h : 0.0), above = tail + (h > 0.0 ? h : 0.0);       // -log sigma(h), -log sigma(-h)
    const double dh = h >= 0.0 ? e - exp(-h) / (1.0 + exp(-h)) : exp(h) / (1.0 + exp(h)) - (1.0 - e);
    a.loss[p] = (float)((double)a.scale * ((1.0 - e) * below + e * above));
    for (int side = 0; side < 2; ++side) {
        a.ratio[2 * p + side] = (float)part[side][0];
        a.slope[2 * p + side] = (float)((double)a.scale * (double)a.beta * (side ? -dh : dh));
    }
}

template <typename T> __global__ void __launch_bounds__(ROW_THREADS)
preference_gradient_kernel(TokenRows rows, PreferenceArgs a)
{
    const int64_t t = blockIdx.x;
    const T *z = (const T *)rows.logits + t * rows.ld;
    T *out = (T *)a.grad + t * a.ldg;
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
        write_zeros(out, rows.vocab);
        return;
    }
    const float2 st = a.stats[t];
    write_gradient(z, out, rows.vocab, st.x, st.y, w * a.slope[lo], label);
}

void launch_policy_loss(hipStream_t s, const TokenRows &rows, const PolicyArgs &a)
{
    if (rows.tokens == 0) return;
    const dim3 grid((uint32_t)rows.tokens);
    if (rows.bf16) policy_loss_kernel<uint16_t><<<grid, ROW_THREADS, 0, s>>>(rows, a);
    else policy_loss_kernel<float><<<grid, ROW_THREADS, 0, s>>>(rows, a);
}

void launch_preference_loss(hipStream_t s, const TokenRows &rows, const PreferenceArgs &a)
{
    const dim3 grid((uint32_t)rows.tokens);
    if (rows.tokens > 0) {
        if (rows.bf16) preference_rows_kernel<uint16_t><<<grid, ROW_THREADS, 0, s>>>(rows, a);
        else preference_rows_kernel<float><<<grid, ROW_THREADS, 0, s>>>(rows, a);
    }
    if (a.pairs > 0) preference_pairs_kernel<<<(uint32_t)a.pairs, ROW_THREADS, 0, s>>>(rows.tokens, a);
    if (rows.tokens > 0 && a.grad) {
        if (rows.bf16) preference_gradient_kernel<uint16_t><<<grid, ROW_THREADS, 0, s>>>(rows, a);
        else preference_gradient_kernel<float><<<grid, ROW_THREADS, 0, s>>>(rows, a);
    }
}

}  // namespace netmax
