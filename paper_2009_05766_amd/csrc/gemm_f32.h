// C = A B for float operands of any shape and stride on v_mfma_f32_32x32x2_f32.
//
// Four waves have a block of BM x BN results; a step of STEP contraction indices lies in LDS as [k][m] and [k][n], the instruction's own layout (lane
// l: row l % 32, index l / 32), while the next step is on its way in registers.  Where blocks are few, GROUPS groups of four waves share a block's
// steps in turn and add up their results in LDS: few workgroups are bound by the chain of loads, barrier and products of a step, and four waves
// by the instruction's 64 cycles (16 x 64 x 784 x 512: 18.9 us in 64 x 32 blocks and four groups, 31.6 us in 64 x 64 blocks, one group and steps of 16).
// Large products run at 121 TFLOP/s of the 157 that the instruction gives (4096 cubed, 1.14 ms).  B goes in as the instruction's first operand, so that a
// lane ends with four neighbouring columns of a row.
#pragma once
#include "gemm.h"

namespace netmax {

// The values of one step that a thread brings: pieces of four neighbours in memory.
template <int ROWS, int STEP, bool K_NEAR> struct StepPieces {
    static constexpr int PIECES = ROWS * STEP / 4 / 256;
    static constexpr int PITCH = ROWS + 4;
    f32x4 v[PIECES];
    __device__ __forceinline__ void request(const float *p, int64_t ld, int64_t row0, int64_t rows, int64_t k0, int64_t K)
    {
#pragma unroll
        for (int u = 0; u < PIECES; ++u) {
            const int q = u * 256 + (int)(threadIdx.x & 255);
            if (K_NEAR) {
                const int64_t r = row0 + q / (STEP / 4), k = k0 + q % (STEP / 4) * 4;
                v[u] = r < rows ? load_up_to_four(p + r * ld, k, K) : f32x4{0, 0, 0, 0};
            } else {
                const int64_t k = k0 + q / (ROWS / 4), r = row0 + q % (ROWS / 4) * 4;
                v[u] = k < K ? load_up_to_four(p + k * ld, r, rows) : f32x4{0, 0, 0, 0};
            }
        }
    }
    __device__ __forceinline__ void place(float *lds) const
    {
#pragma unroll
        for (int u = 0; u < PIECES; ++u) {
            const int q = u * 256 + (int)(threadIdx.x & 255);
            if (K_NEAR) {
                const int r = q / (STEP / 4), k = q % (STEP / 4) * 4;
#pragma unroll
                for (int e = 0; e < 4; ++e) lds[(k + e) * PITCH + r] = v[u][e];
            } else {
                const int k = q / (ROWS / 4), r = q % (ROWS / 4) * 4;
                *reinterpret_cast<f32x4 *>(lds + k * PITCH + r) = v[u];
            }
        }
    }
};

template <int BM, int BN, int STEP, int GROUPS> constexpr int space_f32() { return GROUPS * 2 * STEP * (BM + BN + 8); }

// Workgroup `id`; `space`: space_f32() floats of LDS.
template <int BM, int BN, int STEP, int GROUPS, bool AK, bool BK, class Epilogue>
__device__ __forceinline__ void gemm_f32_block(int64_t M, int64_t N, int64_t K, const float *__restrict__ A, int64_t lda, int64_t sa, const float *__restrict__ B, int64_t ldb,
                                               int64_t sb, uint32_t mblocks, uint32_t nblocks, const Epilogue &epilogue, uint32_t id, float *space)
{
    typedef StepPieces<BM, STEP, AK> PiecesA;
    typedef StepPieces<BN, STEP, BK> PiecesB;
    // a wave has TM x TN squares of 32 x 32 results; SHARES waves of a group share a square and the indices of a step
    constexpr int TM = BM >= 128 ? 2 : 1, TN = BN >= 128 ? 2 : 1, ACROSS = BN / 32 / TN, TILES = BM / 32 / TM * ACROSS, SHARES = 4 / TILES, PARTS = GROUPS * SHARES;
    constexpr int STEP_FLOATS = STEP * (PiecesA::PITCH + PiecesB::PITCH);
    static_assert(TILES * 32 * 36 <= 2 * GROUPS * STEP_FLOATS, "results leave by way of the steps' space");
    static_assert((PARTS - 1) * BM * BN <= 2 * GROUPS * STEP_FLOATS, "partial results fit the steps' space");
    static_assert(GROUPS * 2 * STEP_FLOATS == space_f32<BM, BN, STEP, GROUPS>(), "the caller's space");
    float (*lds)[2][STEP_FLOATS] = reinterpret_cast<float (*)[2][STEP_FLOATS]>(space);
    const uint32_t per = mblocks * nblocks, g = id / per, b = id % per;
    const int64_t m0 = (int64_t)(b / nblocks) * BM, n0 = (int64_t)(b % nblocks) * BN;
    A += (int64_t)g * sa;
    B += (int64_t)g * sb;
    const int lane = threadIdx.x & 63, wave = (threadIdx.x >> 6) & 3, group = threadIdx.x >> 8, half = lane >> 5, at = lane & 31;
    const int tile = wave % TILES, share = wave / TILES, wm = tile / ACROSS * (TM * 32), wn = tile % ACROSS * (TN * 32);
    PiecesA pa;
    PiecesB pb;
    f32x16 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
    const int64_t steps = (K + STEP - 1) / STEP, turns = (steps + GROUPS - 1) / GROUPS;         // a group without a step has zeros
    pa.request(A, lda, m0, M, (int64_t)group * STEP, K);
    pb.request(B, ldb, n0, N, (int64_t)group * STEP, K);
    for (int64_t s = 0; s < turns; ++s) {
        float *ca = lds[group][s & 1], *cb = ca + STEP * PiecesA::PITCH;
        pa.place(ca);
        pb.place(cb);
        __syncthreads();
        if (s + 1 < turns) {
            pa.request(A, lda, m0, M, ((s + 1) * GROUPS + group) * STEP, K);
            pb.request(B, ldb, n0, N, ((s + 1) * GROUPS + group) * STEP, K);
        }
#pragma unroll
        for (int q = 0; q < STEP / SHARES; q += 2) {
            const int k = share * (STEP / SHARES) + q;
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
    if constexpr (PARTS > 1) {
        constexpr int STRIDE = TM * TN * 4 * TILES * 64;            // pieces of four of one part
        const int part = group * SHARES + share;
        f32x4 *mine = reinterpret_cast<f32x4 *>(space) + tile * 64 + lane;
        __syncthreads();
        if (part > 0)
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        mine[(part - 1) * STRIDE + ((i * TN + j) * 4 + e) * (TILES * 64)] =
                            f32x4{acc[i][j][4 * e], acc[i][j][4 * e + 1], acc[i][j][4 * e + 2], acc[i][j][4 * e + 3]};
        __syncthreads();
#pragma unroll
        for (int o = 0; o < PARTS - 1 && part == 0; ++o)
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const f32x4 v = mine[o * STRIDE + ((i * TN + j) * 4 + e) * (TILES * 64)];
#pragma unroll
                        for (int q = 0; q < 4; ++q) acc[i][j][4 * e + q] += v[q];
                    }
    }
    // results leave by way of LDS, so that neighbouring lanes have neighbouring columns of a row
    __syncthreads();
    if (group * SHARES + share > 0) return;
    float *stage = space + __builtin_amdgcn_readfirstlane(tile) * (32 * 36);
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                store4(stage + at * 36 + e * 8 + half * 4, f32x4{acc[i][j][4 * e], acc[i][j][4 * e + 1], acc[i][j][4 * e + 2], acc[i][j][4 * e + 3]});
            wave_order();
#pragma unroll
            for (int r = 0; r < 32; r += 8)
                epilogue(g, m0 + wm + i * 32 + r + lane / 8, n0 + wn + j * 32 + lane % 8 * 4, load4(stage + (r + lane / 8) * 36 + lane % 8 * 4));
            wave_order();
        }
}

template <int BM, int BN, int STEP, int GROUPS, bool AK, bool BK, class Epilogue>
__global__ void __launch_bounds__(256 * GROUPS)
gemm_f32_kernel(int64_t M, int64_t N, int64_t K, const float *__restrict__ A, int64_t lda, int64_t sa, const float *__restrict__ B, int64_t ldb,
                int64_t sb, uint32_t mblocks, uint32_t nblocks, Epilogue epilogue)
{
    __shared__ __align__(16) float space[space_f32<BM, BN, STEP, GROUPS>()];
    gemm_f32_block<BM, BN, STEP, GROUPS, AK, BK>(M, N, K, A, lda, sa, B, ldb, sb, mblocks, nblocks, epilogue, blockIdx.x, space);
}

// Two products in one launch, the first with both contraction indices near and the second with both row indices near (a layer's dx and dw).  Workgroups from
// `both` on do `extra`, which depends on neither.
template <class Epilogue> struct ProductF32 { int64_t M, N, K; const float *A, *B; int64_t lda, sa, ldb, sb; uint32_t mblocks, nblocks; Epilogue epilogue; };
template <int BM, int STEP, int GROUPS, class Epilogue, class Extra>
__global__ void __launch_bounds__(256 * GROUPS) gemm_f32_pair_kernel(ProductF32<Epilogue> p, ProductF32<Epilogue> q, uint32_t first, uint32_t both, int swap,
                                                                         Extra extra)
{
    __shared__ __align__(16) float space[space_f32<BM, BM, STEP, GROUPS>()];
    const uint32_t id = pair_place(blockIdx.x, first, both, swap);
    if (id < first)
        gemm_f32_block<BM, BM, STEP, GROUPS, true, true>(p.M, p.N, p.K, p.A, p.lda, p.sa, p.B, p.ldb, p.sb, p.mblocks, p.nblocks, p.epilogue, id, space);
    else if (id < both)
        gemm_f32_block<BM, BM, STEP, GROUPS, false, false>(q.M, q.N, q.K, q.A, q.lda, q.sa, q.B, q.ldb, q.sb, q.mblocks, q.nblocks, q.epilogue, id - first, space);
    else
        extra(id - both, space);
}

// An operator's products have one of three pairs of orientations: A's contraction index is near in the first two, and where it is not, neither is B's.
template <int BM, int BN, int STEP, int GROUPS, class Epilogue>
void launch_gemm_f32_blocks(hipStream_t s, int64_t batch, int64_t M, int64_t N, int64_t K, const Operand &a, const Operand &b, const Epilogue &epilogue)
{
    const uint32_t mb = (uint32_t)((M + BM - 1) / BM), nb = (uint32_t)((N + BN - 1) / BN);
    const dim3 grid((uint32_t)(batch * mb * nb));
    const float *pa = (const float *)a.p, *pb = (const float *)b.p;
    if (a.k_near && b.k_near)
        gemm_f32_kernel<BM, BN, STEP, GROUPS, true, true><<<grid, 256 * GROUPS, 0, s>>>(M, N, K, pa, a.ld, a.step, pb, b.ld, b.step, mb, nb, epilogue);
    else if (a.k_near)
        gemm_f32_kernel<BM, BN, STEP, GROUPS, true, false><<<grid, 256 * GROUPS, 0, s>>>(M, N, K, pa, a.ld, a.step, pb, b.ld, b.step, mb, nb, epilogue);
    else
        gemm_f32_kernel<BM, BN, STEP, GROUPS, false, false><<<grid, 256 * GROUPS, 0, s>>>(M, N, K, pa, a.ld, a.step, pb, b.ld, b.step, mb, nb, epilogue);
}

// Blocks of 128 x 128 where they are many and the contraction pays for their start: 2944 x 1024 x 2944 (529 blocks) 225 us and 192 in blocks of 64, 3328 (676) 226 and 232,
// 4096 cubed (1024) 1137 and 1301.
constexpr int64_t F32_LARGE = 640;

template <class Epilogue>
void launch_gemm_f32(hipStream_t s, int64_t batch, int64_t M, int64_t N, int64_t K, const Operand &a, const Operand &b, const Epilogue &epilogue)
{
    const auto blocks = [&](int64_t m, int64_t n) { return batch * ((M + m - 1) / m) * ((N + n - 1) / n); };
    // the fewer blocks, the more waves on each.  One group of waves or four: 1408 x 1024 x 1408 (484 blocks) 56 and 53, 1472 (529) 72 and 78; blocks of 64 x 64 or 64 x 32:
    // 704 x 1024 x 704 (121) 27 and 18, 768 (144) 27 and 34
    if (blocks(128, 128) >= F32_LARGE && K >= 256 && worth_blocks(128, M, N)) launch_gemm_f32_blocks<128, 128, 16, 1>(s, batch, M, N, K, a, b, epilogue);
    else if (blocks(64, 64) >= 512) launch_gemm_f32_blocks<64, 64, 32, 1>(s, batch, M, N, K, a, b, epilogue);
    else if (blocks(64, 64) > 128) launch_gemm_f32_blocks<64, 64, 32, 4>(s, batch, M, N, K, a, b, epilogue);
    else launch_gemm_f32_blocks<64, 32, 32, 4>(s, batch, M, N, K, a, b, epilogue);
}

}  // namespace netmax
