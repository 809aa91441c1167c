// An orthogonalised momentum update for a batch of matrices:
//     m' = mu m + g,   u = g + mu m' (Nesterov) or m',   X = u / max(||u||_F, eps),
//     `steps` times:   A = X X^T,   B = b A + c A A,   X <- a X + B X,        out = scale X.
// The polynomial a s + b s^3 + c s^5 drives the singular values of X towards 1 and leaves the singular vectors alone.  Matrices with
// more rows than columns are multiplied from the other side, A = X^T X and X <- a X + X B, which is the same polynomial on the smaller
// square.
#include "gemm_f32.h"
#include "orth.h"

namespace netmax {

constexpr int NORM_BLOCKS = 64;       // partial sums of squares of one matrix

// m' and a part of the sum of squares of u (double; the parts are added in order by whoever needs the norm).
template <typename T>
__global__ void __launch_bounds__(256) momentum_kernel(OrthArgs a, double *__restrict__ parts)
{
    __shared__ double part[256];
    const int64_t g = blockIdx.y, count = a.rows * a.cols;
    double sum = 0.0;
    for (int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x; q < count; q += (int64_t)gridDim.x * 256) {
        const int64_t r = q / a.cols, c = q % a.cols;
        float u = load_value((const T *)a.g + g * a.sg + r * a.ldg + c);
        if (a.m) {
            const int64_t at = g * a.sm + r * a.ldm + c;
            const float m = fmaf(a.mu, a.m[at], u);
            a.m_out[at] = m;
            u = a.nesterov ? fmaf(a.mu, m, u) : m;
        }
        sum += (double)u * (double)u;
    }
    part[threadIdx.x] = sum;
    __syncthreads();
    for (int d = 128; d > 0; d >>= 1) {
        if ((int)threadIdx.x < d) part[threadIdx.x] += part[threadIdx.x + d];
        __syncthreads();
    }
    if (threadIdx.x == 0) parts[g * NORM_BLOCKS + blockIdx.x] = part[0];
}

template <typename T>
__global__ void __launch_bounds__(256) normalise_kernel(OrthArgs a, const double *__restrict__ parts, float *__restrict__ X)
{
    const int64_t g = blockIdx.y, count = a.rows * a.cols;
    double sum = 0.0;
    for (int k = 0; k < NORM_BLOCKS; ++k) sum += parts[g * NORM_BLOCKS + k];
    const double norm = sqrt(sum);
    const float inv = (float)(1.0 / (norm > (double)a.eps || norm != norm ? norm : (double)a.eps));
    for (int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x; q < count; q += (int64_t)gridDim.x * 256) {
        const int64_t r = q / a.cols, c = q % a.cols;
        float u = load_value((const T *)a.g + g * a.sg + r * a.ldg + c);
        if (a.m) {
            const float m = a.m_out[g * a.sm + r * a.ldm + c];
            u = a.nesterov ? fmaf(a.mu, m, u) : m;
        }
        X[g * count + q] = u * inv;
    }
}

template <typename T>
__global__ void __launch_bounds__(256) result_kernel(OrthArgs a, const float *__restrict__ X)
{
    const int64_t g = blockIdx.y, count = a.rows * a.cols;
    for (int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x; q < count; q += (int64_t)gridDim.x * 256)
        store_value((T *)a.out + g * a.so + q / a.cols * a.ldo + q % a.cols, a.scale * X[g * count + q]);
}

static int64_t side(const OrthArgs &a) { return a.rows < a.cols ? a.rows : a.cols; }
static int64_t x_floats(const OrthArgs &a) { return (a.batch * a.rows * a.cols + 63) / 64 * 64; }
static int64_t a_floats(const OrthArgs &a) { return (a.batch * side(a) * side(a) + 63) / 64 * 64; }

int64_t orth_workspace(const OrthArgs &a) { return 4 * (2 * x_floats(a) + 2 * a_floats(a)) + 8 * a.batch * NORM_BLOCKS; }

template <typename T> static void orth_of(hipStream_t s, const OrthArgs &a, float *work)
{
    float *X = work, *Y = X + x_floats(a), *A = Y + x_floats(a), *B = A + a_floats(a);
    double *parts = (double *)(B + a_floats(a));
    const int64_t k = side(a), xs = a.rows * a.cols;
    const dim3 grid(NORM_BLOCKS, (uint32_t)a.batch);
    momentum_kernel<T><<<grid, 256, 0, s>>>(a, parts);
    normalise_kernel<T><<<grid, 256, 0, s>>>(a, parts, X);
    const bool tall = a.rows > a.cols;
    for (int i = 0; i < a.steps; ++i) {
        launch_gemm_f32<float>(s, a.batch, k, k, tall ? a.rows : a.cols, Operand{X, a.cols, xs, !tall}, Operand{X, a.cols, xs, !tall},
                               SumEpilogue<float>{k, k, 1.0f, 0.0f, nullptr, A});
        launch_gemm_f32<float>(s, a.batch, k, k, k, Operand{A, k, k * k, true}, Operand{A, k, k * k, true}, SumEpilogue<float>{k, k, a.c, a.b, A, B});
        const Operand x{X, a.cols, xs, tall}, p{B, k, k * k, true};
        launch_gemm_f32<float>(s, a.batch, a.rows, a.cols, k, tall ? x : p, tall ? p : x, SumEpilogue<float>{a.rows, a.cols, 1.0f, a.a, X, Y});
        float *t = X; X = Y; Y = t;
    }
    result_kernel<T><<<grid, 256, 0, s>>>(a, X);
}

void launch_orth(hipStream_t s, const OrthArgs &a, void *work)
{
    if (a.bf16) orth_of<uint16_t>(s, a, (float *)work); else orth_of<float>(s, a, (float *)work);
}

}  // namespace netmax
