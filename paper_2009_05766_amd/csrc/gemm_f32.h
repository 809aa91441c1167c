// C = A B for operands of any type, shape, stride and orientation, multiplied in float on v_mfma_f32_32x32x2_f32.
//
// A workgroup of four waves has a block of BM x BN results; a step of 16 contraction indices lies in LDS as [k][m] and [k][n], the
// instruction's own layout (lane l: row l % 32, index l / 32), while the next step is on its way in registers.  B goes in as the
// instruction's first operand, so that a lane ends with four neighbouring columns of a row.
#pragma once
#include "gemm.h"

namespace netmax {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int GEMM_STEP = 16;

// The values of one step that a thread brings: pieces of four neighbours in memory.
template <typename T, int ROWS, bool K_NEAR> struct StepPieces {
    static constexpr int PIECES = ROWS * GEMM_STEP / 4 / 256;
    static constexpr int PITCH = ROWS + 4;
    f32x4 v[PIECES];
    __device__ __forceinline__ void request(const T *p, int64_t ld, int64_t row0, int64_t rows, int64_t k0, int64_t K, bool whole)
    {
#pragma unroll
        for (int u = 0; u < PIECES; ++u) {
            const int q = u * 256 + (int)threadIdx.x;
            if (K_NEAR) {
                const int64_t r = row0 + q / (GEMM_STEP / 4), k = k0 + q % (GEMM_STEP / 4) * 4;
                v[u] = r < rows ? load_up_to_four(p + r * ld, k, K, whole) : f32x4{0, 0, 0, 0};
            } else {
                const int64_t k = k0 + q / (ROWS / 4), r = row0 + q % (ROWS / 4) * 4;
                v[u] = k < K ? load_up_to_four(p + k * ld, r, rows, whole) : f32x4{0, 0, 0, 0};
            }
        }
    }
    __device__ __forceinline__ void place(float *lds) const
    {
#pragma unroll
        for (int u = 0; u < PIECES; ++u) {
            const int q = u * 256 + (int)threadIdx.x;
            if (K_NEAR) {
                const int r = q / (GEMM_STEP / 4), k = q % (GEMM_STEP / 4) * 4;
#pragma unroll
                for (int e = 0; e < 4; ++e) lds[(k + e) * PITCH + r] = v[u][e];
            } else {
                const int k = q / (ROWS / 4), r = q % (ROWS / 4) * 4;
                *reinterpret_cast<f32x4 *>(lds + k * PITCH + r) = v[u];
            }
        }
    }
};

template <typename T, int BM, int BN, bool AK, bool BK, class Epilogue>
__global__ void __launch_bounds__(256)
gemm_f32_kernel(int64_t M, int64_t N, int64_t K, const T *__restrict__ A, int64_t lda, int64_t sa, bool wa, const T *__restrict__ B, int64_t ldb,
                int64_t sb, bool wb, uint32_t mblocks, uint32_t nblocks, Epilogue epilogue)
{
    typedef StepPieces<T, BM, AK> PiecesA;
    typedef StepPieces<T, BN, BK> PiecesB;
    constexpr int TM = BM / 64, TN = BN / 64;                       // 32 x 32 results of a wave; the waves lie 2 x 2
    __shared__ __align__(16) float la[2][GEMM_STEP * PiecesA::PITCH], lb[2][GEMM_STEP * PiecesB::PITCH];
    const uint32_t per = mblocks * nblocks, g = blockIdx.x / per, b = blockIdx.x % per;
    const int64_t m0 = (int64_t)(b / nblocks) * BM, n0 = (int64_t)(b % nblocks) * BN;
    A += (int64_t)g * sa;
    B += (int64_t)g * sb;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5, at = lane & 31;
    const int wm = (wave >> 1) * (BM / 2), wn = (wave & 1) * (BN / 2);
    PiecesA pa;
    PiecesB pb;
    f32x16 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
    const int64_t steps = (K + GEMM_STEP - 1) / GEMM_STEP;
    if (steps > 0) {
        pa.request(A, lda, m0, M, 0, K, wa);
        pb.request(B, ldb, n0, N, 0, K, wb);
    }
    for (int64_t s = 0; s < steps; ++s) {
        float *ca = la[s & 1], *cb = lb[s & 1];
        pa.place(ca);
        pb.place(cb);
        __syncthreads();
        if (s + 1 < steps) {
            pa.request(A, lda, m0, M, (s + 1) * GEMM_STEP, K, wa);
            pb.request(B, ldb, n0, N, (s + 1) * GEMM_STEP, K, wb);
        }
#pragma unroll
        for (int k = 0; k < GEMM_STEP; k += 2) {
            float a[TM], c[TN];
#pragma unroll
            for (int i = 0; i < TM; ++i) a[i] = ca[(k + half) * PiecesA::PITCH + wm + i * 32 + at];
#pragma unroll
            for (int j = 0; j < TN; ++j) c[j] = cb[(k + half) * PiecesB::PITCH + wn + j * 32 + at];
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(c[j], a[i], acc[i][j], 0, 0, 0);
        }
    }
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                epilogue(g, m0 + wm + i * 32 + at, n0 + wn + j * 32 + e * 8 + half * 4,
                         f32x4{acc[i][j][4 * e], acc[i][j][4 * e + 1], acc[i][j][4 * e + 2], acc[i][j][4 * e + 3]});
}

template <typename T, int BM, int BN, class Epilogue>
void launch_gemm_f32_blocks(hipStream_t s, int64_t batch, int64_t M, int64_t N, int64_t K, const Operand &a, const Operand &b, const Epilogue &epilogue)
{
    const uint32_t mb = (uint32_t)((M + BM - 1) / BM), nb = (uint32_t)((N + BN - 1) / BN);
    const dim3 grid((uint32_t)(batch * mb * nb));
    const T *pa = (const T *)a.p, *pb = (const T *)b.p;
    const bool wa = whole_pieces(a.p, a.ld, a.step, sizeof(T)), wb = whole_pieces(b.p, b.ld, b.step, sizeof(T));
    if (a.k_near && b.k_near)
        gemm_f32_kernel<T, BM, BN, true, true><<<grid, 256, 0, s>>>(M, N, K, pa, a.ld, a.step, wa, pb, b.ld, b.step, wb, mb, nb, epilogue);
    else if (a.k_near)
        gemm_f32_kernel<T, BM, BN, true, false><<<grid, 256, 0, s>>>(M, N, K, pa, a.ld, a.step, wa, pb, b.ld, b.step, wb, mb, nb, epilogue);
    else if (b.k_near)
        gemm_f32_kernel<T, BM, BN, false, true><<<grid, 256, 0, s>>>(M, N, K, pa, a.ld, a.step, wa, pb, b.ld, b.step, wb, mb, nb, epilogue);
    else
        gemm_f32_kernel<T, BM, BN, false, false><<<grid, 256, 0, s>>>(M, N, K, pa, a.ld, a.step, wa, pb, b.ld, b.step, wb, mb, nb, epilogue);
}

template <typename T, class Epilogue>
void launch_gemm_f32(hipStream_t s, int64_t batch, int64_t M, int64_t N, int64_t K, const Operand &a, const Operand &b, const Epilogue &epilogue)
{
    if (batch * ((M + 127) / 128) * ((N + 127) / 128) >= 256)
        launch_gemm_f32_blocks<T, 128, 128>(s, batch, M, N, K, a, b, epilogue);
    else
        launch_gemm_f32_blocks<T, 64, 64>(s, batch, M, N, K, a, b, epilogue);
}

}  // namespace netmax
