// y = act(x w + b) + r for a batch of layers, and its gradients:
//     dz = dy act'(z),  dx = dz w^T,  dw = x^T dz,  db = sum over the rows of dz.
#include "gemm_f32.h"
#include "linear.h"

namespace netmax {

static inline int64_t round_up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

// ---- dz and db -------------------------------------------------------------------------------------------------------

// A workgroup takes SLOPE_ROWS rows of 64 columns: dz, and the column sums of dz over these rows (float, rows in order).
constexpr int SLOPE_ROWS = 64;

template <typename T>
__global__ void __launch_bounds__(256)
slope_kernel(int64_t rows, int64_t cols, const T *__restrict__ dy, int64_t lddy, int64_t sdy, const T *__restrict__ z, int64_t ldz, int64_t sz, int act,
             T *__restrict__ dz, float *__restrict__ sums)
{
    __shared__ float part[4][64];
    const int64_t g = blockIdx.z, n = (int64_t)blockIdx.x * 64 + (threadIdx.x & 63), r0 = (int64_t)blockIdx.y * SLOPE_ROWS;
    float sum = 0.0f;
    if (n < cols)
        for (int64_t r = r0 + (threadIdx.x >> 6); r < r0 + SLOPE_ROWS && r < rows; r += 4) {
            float v = load_value(dy + g * sdy + r * lddy + n);
            if (act != ACT_NONE) v *= act_slope(act, load_value(z + g * sz + r * ldz + n));
            sum += v;
            if (dz) store_value(dz + (g * rows + r) * cols + n, v);
        }
    part[threadIdx.x >> 6][threadIdx.x & 63] = sum;
    __syncthreads();
    if (sums && threadIdx.x < 64 && n < cols)
        sums[((int64_t)g * gridDim.y + blockIdx.y) * cols + n] = (part[0][threadIdx.x] + part[1][threadIdx.x]) + (part[2][threadIdx.x] + part[3][threadIdx.x]);
}

template <typename T>
__global__ void __launch_bounds__(256) bias_sum_kernel(int64_t cols, int64_t parts, const float *__restrict__ sums, T *__restrict__ db, int64_t sdb)
{
    const int64_t g = blockIdx.y, n = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (n >= cols) return;
    float sum = 0.0f;
    for (int64_t k = 0; k < parts; ++k) sum += sums[(g * parts + k) * cols + n];
    store_value(db + g * sdb + n, sum);
}

// ---- launchers -------------------------------------------------------------------------------------------------------

int64_t linear_workspace(const LinearArgs &) { return 0; }

template <typename T> static void linear_of(hipStream_t s, const LinearArgs &a)
{
    const bool whole = whole_pieces(a.y, a.ldy, a.sy, sizeof(T)) && (!a.z || whole_pieces(a.z, a.ldz, a.sz, sizeof(T))) &&
                       (!a.residual || whole_pieces(a.residual, a.ldr, a.sr, sizeof(T))) && (!a.bias || whole_pieces(a.bias, 0, a.sb, sizeof(T)));
    const LinearEpilogue<T> e{a.rows, a.dout, (const T *)a.bias, (const T *)a.residual, (T *)a.y, (T *)a.z, a.ldr, a.ldy, a.ldz,
                              a.sb, a.sr, a.sy, a.sz, a.act, whole};
    launch_gemm_f32<T>(s, a.batch, a.rows, a.dout, a.din, Operand{a.x, a.ldx, a.sx, true}, Operand{a.w, a.ldw, a.sw, false}, e);
}

void launch_linear(hipStream_t s, const LinearArgs &a, void *)
{
    if (a.bf16) linear_of<uint16_t>(s, a); else linear_of<float>(s, a);
}

static int64_t dz_bytes(const LinearGradArgs &a)
{
    return a.act == ACT_NONE ? 0 : round_up(a.batch * a.rows * a.dout * (a.bf16 ? 2 : 4), 256);
}
static int64_t sum_parts(const LinearGradArgs &a) { return (a.rows + SLOPE_ROWS - 1) / SLOPE_ROWS; }
int64_t linear_grad_workspace(const LinearGradArgs &a) { return dz_bytes(a) + round_up(a.batch * sum_parts(a) * a.dout * 4, 256); }

template <typename T> static void linear_grad_of(hipStream_t s, const LinearGradArgs &a, char *work)
{
    T *dz = a.act == ACT_NONE ? nullptr : (T *)work;
    float *sums = a.db ? (float *)(work + dz_bytes(a)) : nullptr;
    if ((dz || sums) && a.rows > 0)
        slope_kernel<T><<<dim3((uint32_t)((a.dout + 63) / 64), (uint32_t)sum_parts(a), (uint32_t)a.batch), 256, 0, s>>>(
            a.rows, a.dout, (const T *)a.dy, a.lddy, a.sdy, (const T *)a.z, a.ldz, a.sz, a.act, dz, sums);
    if (a.db)
        bias_sum_kernel<T><<<dim3((uint32_t)((a.dout + 255) / 256), (uint32_t)a.batch), 256, 0, s>>>(a.dout, sum_parts(a), sums, (T *)a.db, a.sdb);
    const Operand d = dz ? Operand{dz, a.dout, a.rows * a.dout, true} : Operand{a.dy, a.lddy, a.sdy, true};
    if (a.dx && a.rows > 0) {
        const LinearEpilogue<T> e{a.rows, a.din, nullptr, nullptr, (T *)a.dx, nullptr, 0, a.lddx, 0, 0, 0, a.sdx, 0, ACT_NONE,
                                  whole_pieces(a.dx, a.lddx, a.sdx, sizeof(T))};
        launch_gemm_f32<T>(s, a.batch, a.rows, a.din, a.dout, d, Operand{a.w, a.ldw, a.sw, true}, e);
    }
    if (a.dw) {
        const LinearEpilogue<T> e{a.din, a.dout, nullptr, nullptr, (T *)a.dw, nullptr, 0, a.lddw, 0, 0, 0, a.sdw, 0, ACT_NONE,
                                  whole_pieces(a.dw, a.lddw, a.sdw, sizeof(T))};
        launch_gemm_f32<T>(s, a.batch, a.din, a.dout, a.rows, Operand{a.x, a.ldx, a.sx, false}, Operand{d.p, d.ld, d.step, false}, e);
    }
}

void launch_linear_grad(hipStream_t s, const LinearGradArgs &a, void *work)
{
    if (a.bf16) linear_grad_of<uint16_t>(s, a, (char *)work); else linear_grad_of<float>(s, a, (char *)work);
}

}  // namespace netmax
