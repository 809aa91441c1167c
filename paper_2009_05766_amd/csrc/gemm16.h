// C = A B for operands of 16 bits (bfloat16 or half) on v_mfma_f32_32x32x16, accumulated in float.
//
// A workgroup has a block of BM x BN results.  Steps of STEP contraction indices of both operands go from memory straight into LDS (16 bytes per lane and
// request), STAGES of them under way or in use; one barrier per step.  Large products are bound by the card's power: 8192 x 4096 x 8192 with a plain epilogue runs at 1.25
// PFLOP/s in all three pairs of orientations, with the matrix instructions busy 63 % of 1.8 GHz (without its loads 2.0 GHz, on zeros 2.3 GHz); with GELU and z 515 us.  Blocks of 256 x 256 in eight
// waves read the least per product: 440 us, 256 x 128 510 us, 128 x 128 540 us.  Small ones are bound by the latency of steps: 16 products 512 x 512 x 784
// take 14.2 us with eight waves and four stages on a 128 x 128 block, 16.0 us with four waves and two.
// Each operand lies in LDS as it lies in memory:
//   contraction index near   [rows][STEP]: lanes read 16 bytes of a row; the 16-byte units of a row are permuted by (row / 2) % 8 (STEP 32: row / 4 % 4), so
//                            that sixteen rows at one index lie in different banks
//   row index near           [STEP][rows]: ds_read_b64_tr_b16 hands each lane four contraction indices of its row; groups of 64 bytes are permuted by
//                            k % 4 (rows of 128 bytes: k / 2 % 2, of 64 bytes: not at all), so that the four stored rows that one such read touches lie in different banks
// The permutations are applied to the memory addresses, since a request to LDS fills consecutive units.
// B goes in as the instruction's first operand, so that a lane ends with four neighbouring columns of a row.
//
// Memory: 16-byte aligned, ld and step multiples of 8, extents along memory rounded up to 8 readable; where the contraction index is near and K is
// no multiple of 8, zeros from K to the next multiple.  Rows past the end are read as the last ones (their results are not kept); contraction
// indices past the end as zeros.
#pragma once
#include "gemm.h"

#include <type_traits>

namespace netmax {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

// Where a unit of 16 bytes of row r lies in a row of STEP indices: sixteen rows at one index in different banks.
template <int STEP> __device__ __forceinline__ int near_unit(int r, int c) { return STEP == 32 ? c ^ ((r >> 2) & 3) : c ^ ((r >> 1) & 7); }

__device__ __forceinline__ f32x16 mfma16(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 mfma16(half8 a, half8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }

static __device__ const uint4 g16_zeros = {0, 0, 0, 0};

// 16 bytes of every lane to LDS, next to each other from `to` on.  Restrict: what is requested is never what is read before the next wait and barrier.
__device__ __forceinline__ void to_lds(const char *__restrict__ from, char *__restrict__ to)
{
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from, (__attribute__((address_space(3))) void *)to, 16, 0, 0);
}
__device__ __forceinline__ s16x4 read_turned(const char *__restrict__ p)
{
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)p);
}
template <typename V> __device__ __forceinline__ V read_unit(const char *__restrict__ p) { return *reinterpret_cast<const V *>(p); }

template <int ROWS> __device__ __forceinline__ int turned_group(int k) { return ROWS == 32 ? 0 : ROWS == 64 ? (k >> 1) & 1 : k & 3; }

// One operand's step: ROWS results' rows x STEP contraction indices, brought by THREADS threads.
template <int ROWS, bool K_NEAR, int STEP, int THREADS> struct Step16 {
    static constexpr int BYTES = ROWS * STEP * 2, PIECES = BYTES / 16 / THREADS, ROW_UNITS = ROWS / 8;
    uint32_t offset[PIECES];                                        // of this lane's piece from the step's first byte
    int first_k[PIECES];

    __device__ __forceinline__ void place(int thread, int64_t row0, int64_t rows, int64_t ld)
    {
        // rows past the end are the last ones, so an offset stays below ROWS (64) rows of ld; ld < 2^22
#pragma unroll
        for (int u = 0; u < PIECES; ++u) {
            const int q = u * THREADS + thread;
            if (K_NEAR) {
                const int r = q / (STEP / 8), c = near_unit<STEP>(r, q % (STEP / 8));
                const int64_t row = row0 + r < rows ? row0 + r : rows - 1;
                first_k[u] = c * 8;
                offset[u] = (uint32_t)((row - row0) * ld * 2 + c * 16);
            } else {
                const int k = q / ROW_UNITS, c = (q % ROW_UNITS) ^ (turned_group<ROWS>(k) << 2);
                const int64_t last = (rows + 7) / 8 - 1, unit = row0 / 8 + c < last ? row0 / 8 + c : last;
                first_k[u] = k;
                offset[u] = (uint32_t)((int64_t)k * ld * 2 + (unit - row0 / 8) * 16);
            }
        }
    }
    // Piece u of the step that starts at `from` (row row0, first index of the step) and has `left` indices (fewer than a step's: zeros behind them); a wave's units lie next to each other.
    __device__ __forceinline__ void request(int u, int wave, const char *from, char *lds, int left) const
    {
        to_lds(first_k[u] < left ? from + offset[u] : (const char *)&g16_zeros, lds + u * THREADS * 16 + wave * 1024);
    }
};

// Where a lane reads its part of 32 rows from `first` (a multiple of 32) on.
template <int ROWS, bool K_NEAR, int STEP> struct Fragment16 {
    int base[STEP / 16];                                                     // K_NEAR: one for each 16 indices of the step; else base[0]
    __device__ __forceinline__ void place(int first)
    {
        const int lane = threadIdx.x & 63, at = lane & 31, half = lane >> 5;
        if (K_NEAR) {
#pragma unroll
            for (int kk = 0; kk < STEP / 16; ++kk) base[kk] = (first + at) * (STEP * 2) + near_unit<STEP>(at, kk * 2 + half) * 16;
        } else {
            const int group = (lane >> 4) & 1, t = lane & 15;
            base[0] = (half * 8 + t / 4) * (ROWS * 2) + ((first / 32) ^ turned_group<ROWS>(t / 4)) * 64 + group * 32 + (t & 3) * 8;
        }
    }
    template <typename V> __device__ __forceinline__ V read(const char *lds, int kk) const
    {
        if (K_NEAR) return read_unit<V>(lds + base[kk]);
        const s16x4 lo = read_turned(lds + base[0] + kk * 16 * (ROWS * 2)), hi = read_turned(lds + base[0] + (kk * 16 + 4) * (ROWS * 2));
        return __builtin_bit_cast(V, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
};

// Renumbers workgroups so that those of one L2 (every eighth) are neighbours.
__device__ __forceinline__ uint32_t l2_neighbours(uint32_t id, uint32_t all)
{
    const uint32_t each = all / 8, more = all % 8, part = id % 8;
    return part * each + (part < more ? part : more) + id / 8;
}

// Numbers workgroups so that those of one L2 (every eighth) have neighbouring blocks, and blocks in columns of eight rows of blocks.
__device__ __forceinline__ void block_place(uint32_t id, uint32_t all, uint32_t mblocks, uint32_t nblocks, uint32_t &g, uint32_t &mb, uint32_t &nb)
{
    id = l2_neighbours(id, all);
    const uint32_t per = mblocks * nblocks;
    g = id / per;
    id -= g * per;
    const uint32_t band = id / (8 * nblocks), high = mblocks - band * 8 < 8 ? mblocks - band * 8 : 8, in = id - band * 8 * nblocks;
    nb = in / high;
    mb = band * 8 + in % high;
}

// The same for the lower triangle of a square in blocks RATIO times as high as wide: row mb of blocks has RATIO (mb + 1) of them.
template <int RATIO> __device__ __forceinline__ void triangle_place(uint32_t id, uint32_t all, uint32_t side, uint32_t &g, uint32_t &mb, uint32_t &nb)
{
    id = l2_neighbours(id, all);
    const uint32_t per = RATIO * side * (side + 1) / 2;
    g = id / per;
    id -= g * per;
    mb = (uint32_t)((sqrtf((8.0f / RATIO) * (float)id + 1.0f) - 1.0f) * 0.5f);
    while (RATIO * (mb + 1) * (mb + 2) / 2 <= id) ++mb;             // the root is rounded
    while (RATIO * mb * (mb + 1) / 2 > id) --mb;
    nb = id - RATIO * mb * (mb + 1) / 2;
}

// With SPLIT an operand is two planes, hi + lo: both planes of both operands come to LDS, and hi hi, hi lo and lo hi are added up; lo lo, below 2^-22 of
// the terms, is left out.
struct Planes16 { const char *hi, *lo; int64_t ld, step; };          // ld, step in elements

template <int BM, int BN, int STEP, int STAGES, int GROUPS, bool SPLIT> constexpr int space16() { return GROUPS * STAGES * (SPLIT ? 2 : 1) * (BM + BN) * STEP * 2; }

// GROUPS groups of waves take a block's steps in turn, each with its own space, and add up their results in LDS: for few blocks, which are bound by the chain
// of steps.
// Workgroup `id` of `count`; `space`: space16() bytes of LDS.
template <typename V, int BM, int BN, int WAVES_M, int WAVES_N, int STEP, int STAGES, int GROUPS, bool AK, bool BK, bool SPLIT, bool TRIANGLE, class Epilogue>
__device__ __forceinline__ void gemm16_block(int64_t M, int64_t N, int64_t K, const Planes16 &A, const Planes16 &B, uint32_t mblocks, uint32_t nblocks, uint32_t splits,
                                             const Epilogue &epilogue, uint32_t id, uint32_t count, char *space_)
{
    constexpr int THREADS = WAVES_M * WAVES_N * 64, TM = BM / WAVES_M / 32, TN = BN / WAVES_N / 32;
    typedef Step16<BM, AK, STEP, THREADS> StepA;
    typedef Step16<BN, BK, STEP, THREADS> StepB;
    constexpr int PLANES = SPLIT ? 2 : 1, STAGE = PLANES * (StepA::BYTES + StepB::BYTES), REQUESTS = PLANES * (StepA::PIECES + StepB::PIECES);
    const int group = GROUPS > 1 ? __builtin_amdgcn_readfirstlane((int)threadIdx.x / THREADS) : 0, thread = (int)threadIdx.x - group * THREADS;
    static_assert(GROUPS * STAGES * STAGE == space16<BM, BN, STEP, STAGES, GROUPS, SPLIT>(), "the caller's space");
    char (*lds)[STAGE] = reinterpret_cast<char (*)[STAGE]>(space_ + group * (STAGES * STAGE));
    uint32_t g, mb, nb;
    const uint32_t all = count / splits, split = id / all;
    if (TRIANGLE) {
        triangle_place<BM / BN>(id % all, all, mblocks, g, mb, nb);
        if ((int64_t)nb * BN >= N) return;                          // the last row's blocks may reach past the square
    } else block_place(id % all, all, mblocks, nblocks, g, mb, nb);
    const int64_t m0 = (int64_t)mb * BM, n0 = (int64_t)nb * BN;
    const int64_t kstepA = AK ? STEP * 2 : A.ld * (STEP * 2), kstepB = BK ? STEP * 2 : B.ld * (STEP * 2);
    const int64_t from_a = ((int64_t)g * A.step + (AK ? m0 * A.ld : m0)) * 2, from_b = ((int64_t)g * B.step + (BK ? n0 * B.ld : n0)) * 2;
    const int wave = thread >> 6, wm = wave / WAVES_N * (TM * 32), wn = wave % WAVES_N * (TN * 32);
    StepA sa;
    StepB sb;
    sa.place(thread, m0, M, A.ld);
    sb.place(thread, n0, N, B.ld);
    Fragment16<BM, AK, STEP> fa[TM];
    Fragment16<BN, BK, STEP> fb[TN];
#pragma unroll
    for (int i = 0; i < TM; ++i) fa[i].place(wm + i * 32);
#pragma unroll
    for (int j = 0; j < TN; ++j) fb[j].place(wn + j * 32);
    f32x16 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;

    const int64_t whole = (K + STEP - 1) / STEP;
    const int first = (int)(whole * split / splits), total = (int)(whole * (split + 1) / splits) - first;
    // A step on its way to LDS: its pieces are requested one by one.  Steps behind the last one are requested, too, as zeros that nobody reads, so that the
    // loop below has no branches.
    const int mine = __builtin_amdgcn_readfirstlane(wave);
    int64_t next_a, next_b;
    char *next_to;
    int next_left;
    const auto aim = [&](int s) {
        const int64_t k = first + (int64_t)s * GROUPS + group, left = K - k * STEP;
        next_a = from_a + k * kstepA;
        next_b = from_b + k * kstepB;
        next_to = lds[s % STAGES];
        next_left = s * GROUPS + group >= total ? 0 : left < STEP ? (int)left : STEP;
    };
    const auto request = [&](int u) {                               // pieces of A, of B, then those of the low planes
        const bool low = u >= StepA::PIECES + StepB::PIECES;
        char *to = next_to + (low ? StepA::BYTES + StepB::BYTES : 0);
        if (low) u -= StepA::PIECES + StepB::PIECES;
        if (u < StepA::PIECES) sa.request(u, mine, (low ? A.lo : A.hi) + next_a, to, next_left);
        else sb.request(u - StepA::PIECES, mine, (low ? B.lo : B.hi) + next_b, to + StepA::BYTES, next_left);
    };
    // While 16 indices are multiplied the next 16 come from LDS into registers.  Before the last 16 of step s are multiplied, step s + 1 has arrived and all
    // waves hold the rest of step s: the barrier and the first reads behind it are covered by those products, and step s + STAGES may fill the space of
    // step s.  Its requests are spread over the products that follow (a wave waits at each one while the others' are taken, and so would its
    // products behind them).  STAGES - 2 steps are under way at every wait.
    constexpr int PARTS = STEP / 16, HALF = (REQUESTS + 1) / 2;      // half of the requests go with the step's last products, the others with the next step's first
    V a[2][PLANES][TM], b[2][PLANES][TN];
    const auto read = [&](int set, const char *from, int kk) {
#pragma unroll
        for (int p = 0; p < PLANES; ++p) {
            const char *plane = from + p * (StepA::BYTES + StepB::BYTES);
#pragma unroll
            for (int i = 0; i < TM; ++i) a[set][p][i] = fa[i].template read<V>(plane, kk);
#pragma unroll
            for (int j = 0; j < TN; ++j) b[set][p][j] = fb[j].template read<V>(plane + StepA::BYTES, kk);
        }
    };
    const auto multiply = [&](int set, int first_piece, int end_piece) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                const int at = i * TN + j, before = at * HALF / (TM * TN), here = (at + 1) * HALF / (TM * TN);
                if constexpr (SPLIT) {
                    acc[i][j] = mfma16(b[set][0][j], a[set][1][i], acc[i][j]);
                    acc[i][j] = mfma16(b[set][1][j], a[set][0][i], acc[i][j]);
                }
                acc[i][j] = mfma16(b[set][0][j], a[set][0][i], acc[i][j]);
#pragma unroll
                for (int u = before; u < here; ++u)
                    if (first_piece + u < end_piece) request(first_piece + u);
            }
    };
    for (int s = 0; s < STAGES - 1; ++s) {
        aim(s);
#pragma unroll
        for (int u = 0; u < REQUESTS; ++u) request(u);
    }
    aim(STAGES - 1);
#pragma unroll
    for (int u = 0; u < HALF; ++u) request(u);
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((STAGES - 2) * REQUESTS + HALF) : "memory");
    read(0, lds[0], 0);
    const int turns = (total + GROUPS - 1) / GROUPS;                 // a group without a step has zeros
    for (int s = 0; s < turns; ++s) {
#pragma unroll
        for (int kk = 0; kk < PARTS - 1; ++kk) {
            read((kk + 1) & 1, lds[s % STAGES], kk + 1);
            if (kk == 0) multiply(0, HALF, REQUESTS);
            else multiply(kk & 1, 0, 0);
        }
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((STAGES - 2) * REQUESTS) : "memory");
        read(0, lds[(s + 1) % STAGES], 0);
        aim(s + STAGES);
        multiply(1, 0, HALF);
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    if constexpr (GROUPS > 1) {
        // behind the space that results leave by
        constexpr int OUT = WAVES_M * WAVES_N * 32 * (TN * 32 + 4), QUADS = TM * TN * 4;
        static_assert(OUT * 4 + (GROUPS - 1) * QUADS * THREADS * 16 <= GROUPS * STAGES * STAGE, "the groups' results fit the steps' space");
        f32x4 *sums = reinterpret_cast<f32x4 *>((float *)space_ + OUT) + thread;
        if (group > 0)
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        sums[((group - 1) * QUADS + (i * TN + j) * 4 + e) * THREADS] = f32x4{acc[i][j][4 * e], acc[i][j][4 * e + 1], acc[i][j][4 * e + 2], acc[i][j][4 * e + 3]};
        __syncthreads();
        if (group > 0) return;
#pragma unroll
        for (int o = 0; o < GROUPS - 1; ++o)
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const f32x4 v = sums[(o * QUADS + (i * TN + j) * 4 + e) * THREADS];
#pragma unroll
                        for (int q = 0; q < 4; ++q) acc[i][j][4 * e + q] += v[q];
                    }
    }
    // Results leave by way of LDS, 32 rows of a wave at a time, so that neighbouring lanes have neighbouring columns of a row: straight from the
    // instruction's layout a request would touch 32 rows, 16 bytes in each.
    constexpr int COLS = TN * 32, PITCH = COLS + 4, ROWS = 256 / COLS, CALLS = 32 / ROWS;
    const int lane = threadIdx.x & 63, at = lane & 31, half = lane >> 5, row = lane / (COLS / 4), col = lane % (COLS / 4) * 4;
    float *stage = (float *)space_ + __builtin_amdgcn_readfirstlane(wave) * (32 * PITCH);
    const int64_t where = !TRIANGLE && splits > 1 ? (int64_t)split * (all / (mblocks * nblocks)) + g : g, n = n0 + wn + col;
    const auto put = [&](int i) {
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                store4(stage + at * PITCH + j * 32 + e * 8 + half * 4, f32x4{acc[i][j][4 * e], acc[i][j][4 * e + 1], acc[i][j][4 * e + 2], acc[i][j][4 * e + 3]});
        wave_order();
    };
    if constexpr (TRIANGLE) {                                       // read where it is used: seen ahead, 1 x 2660 x 512 took 8 us more per product
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            put(i);
#pragma unroll
            for (int r = 0; r < 32; r += ROWS) epilogue(where, m0 + wm + i * 32 + r + row, n, load4(stage + (r + row) * PITCH + col));
#pragma unroll
            for (int c = 0; c < COLS; c += 8) {                     // the mirror image: rows are columns
                const int down = c + lane / 8, across = lane % 8 * 4;
                const float *p = stage + across * PITCH + down;
                epilogue.mirror(where, n0 + wn + down, m0 + wm + i * 32 + across, f32x4{p[0], p[PITCH], p[2 * PITCH], p[3 * PITCH]});
            }
            wave_order();
        }
    } else {
        const auto leave = [&](auto full) {
            constexpr bool FULL = decltype(full)::value;
            const typename Epilogue::Columns columns = epilogue.template columns<FULL>(where, n);
            typename Epilogue::Seen seen[CALLS];
#pragma unroll
            for (int r = 0; r < CALLS; ++r) seen[r] = epilogue.template see<FULL>(where, m0 + wm + r * ROWS + row, n);
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                put(i);
#pragma unroll
                for (int r = 0; r < CALLS; ++r) {
                    const int64_t m = m0 + wm + i * 32 + r * ROWS + row;
                    const typename Epilogue::Seen now = seen[r];
                    if (i + 1 < TM) seen[r] = epilogue.template see<FULL>(where, m + 32, n);
                    epilogue.template leave<FULL>(where, m, n, load4(stage + (r * ROWS + row) * PITCH + col), columns, now);
                }
                wave_order();
            }
        };
        if (m0 + wm + TM * 32 <= epilogue.rows_here() && n0 + wn + COLS <= epilogue.cols_here()) leave(std::true_type());
        else leave(std::false_type());
    }
}

template <typename V, int BM, int BN, int WAVES_M, int WAVES_N, int STEP, int STAGES, int GROUPS, bool AK, bool BK, bool SPLIT, bool TRIANGLE, class Epilogue>
__global__ void __launch_bounds__(WAVES_M * WAVES_N * 64 * GROUPS)
gemm16_kernel(int64_t M, int64_t N, int64_t K, Planes16 A, Planes16 B, uint32_t mblocks, uint32_t nblocks, uint32_t splits, Epilogue epilogue)
{
    __shared__ __align__(16) char space[space16<BM, BN, STEP, STAGES, GROUPS, SPLIT>()];
    gemm16_block<V, BM, BN, WAVES_M, WAVES_N, STEP, STAGES, GROUPS, AK, BK, SPLIT, TRIANGLE>(M, N, K, A, B, mblocks, nblocks, splits, epilogue, blockIdx.x, gridDim.x, space);
}

// Two products in one launch, the first with both contraction indices near and the second with both row indices near (a layer's dx and dw): where neither fills
// the card, its compute units and the latency of a launch are shared.  Workgroups from `both` on do `extra`, which depends on neither.
template <class Epilogue> struct Product16 { int64_t M, N, K; Planes16 A, B; uint32_t mblocks, nblocks; Epilogue epilogue; };
template <typename V, int BM, int WAVES_M, int WAVES_N, int STEP, int STAGES, int GROUPS, class Epilogue, class Extra>
__global__ void __launch_bounds__(WAVES_M * WAVES_N * 64 * GROUPS)
gemm16_pair_kernel(Product16<Epilogue> p, Product16<Epilogue> q, uint32_t first, uint32_t both, int swap, Extra extra)
{
    __shared__ __align__(16) char space[space16<BM, BM, STEP, STAGES, GROUPS, false>()];
    const uint32_t id = pair_place(blockIdx.x, first, both, swap);
    if (id < first)
        gemm16_block<V, BM, BM, WAVES_M, WAVES_N, STEP, STAGES, GROUPS, true, true, false, false>(p.M, p.N, p.K, p.A, p.B, p.mblocks, p.nblocks, 1, p.epilogue, id, first, space);
    else if (id < both)
        gemm16_block<V, BM, BM, WAVES_M, WAVES_N, STEP, STAGES, GROUPS, false, false, false, false>(q.M, q.N, q.K, q.A, q.B, q.mblocks, q.nblocks, 1, q.epilogue,
                                                                                                   id - first, both - first, space);
    else
        extra(id - both, reinterpret_cast<float *>(space));
}

// A block's shape as a value: what gemm16_kernel is instantiated with.
template <int BM_, int BN_, int WM_, int WN_, int STEP_, int STAGES_, int GROUPS_ = 1>
struct Shape { static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, STEP = STEP_, STAGES = STAGES_, GROUPS = GROUPS_; };

// C = A B for few rows, at most 32 TM: the weights are what has to be read.  A workgroup has 32 columns; its eight waves take steps of 32 indices in turn,
// each with its own space in LDS for a few steps under way and without a barrier.  The waves' sums are added in LDS in order.  Neighbouring
// workgroups share an L2, as they share the lines of 128 bytes that 64 bytes of a row of weights lie in.  Bound by what is under way per compute unit: one
// row, 2048 x 8192 7.5 us (4.5 TB/s), 32 rows, 4096 x 4096 14.8 us (2.3 TB/s: 128 workgroups, and A is as much again).
constexpr int FEW_WAVES = 8;

template <typename V, int TM, bool BK, class Epilogue>
__global__ void __launch_bounds__(FEW_WAVES * 64)
few_rows_kernel(int64_t M, int64_t N, int64_t K, Planes16 A, Planes16 B, Epilogue epilogue)
{
    constexpr int STEP = 32, STAGES = TM == 1 ? 4 : 3;
    typedef Step16<32 * TM, true, STEP, 64> StepA;
    typedef Step16<32, BK, STEP, 64> StepB;
    constexpr int STAGE = StepA::BYTES + StepB::BYTES, REQUESTS = StepA::PIECES + StepB::PIECES;
    constexpr int PITCH = 36, SUMS = FEW_WAVES * TM * 32 * PITCH * 4, SPACE = FEW_WAVES * STAGES * STAGE;
    __shared__ __align__(16) char lds[SPACE > SUMS ? SPACE : SUMS];
    const int64_t g = blockIdx.y, n0 = (int64_t)l2_neighbours(blockIdx.x, gridDim.x) * 32;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), at = lane & 31, half = lane >> 5;
    const char *from_a = A.hi + g * A.step * 2, *from_b = B.hi + (g * B.step + (BK ? n0 * B.ld : n0)) * 2;
    char *space = lds + wave * (STAGES * STAGE);
    const int64_t kstep = BK ? STEP * 2 : B.ld * (STEP * 2);
    StepA sa;
    StepB sb;
    sa.place(lane, 0, M, A.ld);
    sb.place(lane, n0, N, B.ld);
    Fragment16<32 * TM, true, STEP> fa[TM];
    Fragment16<32, BK, STEP> fb;
#pragma unroll
    for (int i = 0; i < TM; ++i) fa[i].place(i * 32);
    fb.place(0);
    f32x16 acc[TM];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[i][e] = 0.0f;
    const int steps = (int)((K + STEP - 1) / STEP), turns = steps > wave ? (steps - wave + FEW_WAVES - 1) / FEW_WAVES : 0;
    const auto bring = [&](int s) {                                 // steps behind the last one as zeros that nobody reads
        const int64_t k = wave + (int64_t)s * FEW_WAVES, all = K - k * STEP;
        const int left = s >= turns ? 0 : all < STEP ? (int)all : STEP;
        char *to = space + s % STAGES * STAGE;
#pragma unroll
        for (int u = 0; u < StepB::PIECES; ++u) sb.request(u, 0, from_b + k * kstep, to + StepA::BYTES, left);
#pragma unroll
        for (int u = 0; u < StepA::PIECES; ++u) sa.request(u, 0, from_a + k * (STEP * 2), to, left);
    };
    for (int s = 0; s < STAGES - 1; ++s) bring(s);
    for (int s = 0; s < turns; ++s) {
        bring(s + STAGES - 1);
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"((STAGES - 1) * REQUESTS) : "memory");
        const char *now = space + s % STAGES * STAGE;
#pragma unroll
        for (int kk = 0; kk < STEP / 16; ++kk) {
            const V v = fb.template read<V>(now + StepA::BYTES, kk);
#pragma unroll
            for (int i = 0; i < TM; ++i) acc[i] = mfma16(v, fa[i].template read<V>(now, kk), acc[i]);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");           // the step's space is free
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    float *sums = (float *)lds;
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            store4(sums + ((wave * TM + i) * 32 + at) * PITCH + e * 8 + half * 4, f32x4{acc[i][4 * e], acc[i][4 * e + 1], acc[i][4 * e + 2], acc[i][4 * e + 3]});
    __syncthreads();
    const int row = threadIdx.x / 8, col = threadIdx.x % 8 * 4;     // 64 rows of 8 pieces
    if (row >= TM * 32) return;
    f32x4 v = load4(sums + row * PITCH + col);
#pragma unroll
    for (int w = 1; w < FEW_WAVES; ++w) v += load4(sums + (w * TM * 32 + row) * PITCH + col);
    epilogue(g, row, n0 + col, v);
}

template <typename V, class Epilogue>
void launch_few_rows(hipStream_t s, int64_t batch, int64_t M, int64_t N, int64_t K, const Planes16 &a, const Planes16 &b, bool bk, const Epilogue &e)
{
    const dim3 grid((uint32_t)((N + 31) / 32), (uint32_t)batch);
    if (M <= 32) {
        if (bk) few_rows_kernel<V, 1, true><<<grid, FEW_WAVES * 64, 0, s>>>(M, N, K, a, b, e);
        else few_rows_kernel<V, 1, false><<<grid, FEW_WAVES * 64, 0, s>>>(M, N, K, a, b, e);
    } else {
        if (bk) few_rows_kernel<V, 2, true><<<grid, FEW_WAVES * 64, 0, s>>>(M, N, K, a, b, e);
        else few_rows_kernel<V, 2, false><<<grid, FEW_WAVES * 64, 0, s>>>(M, N, K, a, b, e);
    }
}

// Whether a matrix can be multiplied where it lies (see the top); `stored`: its extent along memory.
inline bool fits16(const void *p, int64_t ld, int64_t step, int64_t stored)
{
    return (uintptr_t)p % 16 == 0 && ld % 8 == 0 && step % 8 == 0 && stored % 8 == 0 && ld < (1 << 22);
}

// Three pairs of orientations: where A's contraction index is not near, neither is B's.
template <typename V, int BM, int BN, int WM, int WN, int STEP, int STAGES, int GROUPS, class Epilogue>
void launch_gemm16_blocks(hipStream_t s, int64_t batch, int64_t M, int64_t N, int64_t K, const Planes16 &a, bool ak, const Planes16 &b, bool bk, uint32_t splits,
                          const Epilogue &e)
{
    const uint32_t mb = (uint32_t)((M + BM - 1) / BM), nb = (uint32_t)((N + BN - 1) / BN);
    const dim3 grid((uint32_t)(batch * mb * nb * splits)), block(WM * WN * 64 * GROUPS);
    if (ak && bk) gemm16_kernel<V, BM, BN, WM, WN, STEP, STAGES, GROUPS, true, true, false, false><<<grid, block, 0, s>>>(M, N, K, a, b, mb, nb, splits, e);
    else if (ak) gemm16_kernel<V, BM, BN, WM, WN, STEP, STAGES, GROUPS, true, false, false, false><<<grid, block, 0, s>>>(M, N, K, a, b, mb, nb, splits, e);
    else gemm16_kernel<V, BM, BN, WM, WN, STEP, STAGES, GROUPS, false, false, false, false><<<grid, block, 0, s>>>(M, N, K, a, b, mb, nb, splits, e);
}

// The lower triangle of blocks of a symmetric product, A B with B = A transposed as stored: both operands have the same orientation.
template <typename V, int BM, int BN, int WM, int WN, int STEP, int STAGES, int GROUPS, bool SPLIT, class Epilogue>
void launch_gemm16_triangle(hipStream_t s, int64_t batch, int64_t M, int64_t K, const Planes16 &a, bool near, const Epilogue &e)
{
    const uint32_t side = (uint32_t)((M + BM - 1) / BM);
    const dim3 grid((uint32_t)(batch * (BM / BN) * side * (side + 1) / 2)), block(WM * WN * 64 * GROUPS);
    if (near) gemm16_kernel<V, BM, BN, WM, WN, STEP, STAGES, GROUPS, true, true, SPLIT, true><<<grid, block, 0, s>>>(M, M, K, a, a, side, side, 1, e);
    else gemm16_kernel<V, BM, BN, WM, WN, STEP, STAGES, GROUPS, false, false, SPLIT, true><<<grid, block, 0, s>>>(M, M, K, a, a, side, side, 1, e);
}

// C = A B with A's contraction index near and B's as `bk` says, in blocks of BM x BN.
template <typename V, int BM, int BN, int WM, int WN, int STEP, int STAGES, int GROUPS, bool SPLIT, class Epilogue>
void launch_gemm16_step(hipStream_t s, int64_t batch, int64_t M, int64_t N, int64_t K, const Planes16 &a, const Planes16 &b, bool bk, const Epilogue &e)
{
    const uint32_t mb = (uint32_t)((M + BM - 1) / BM), nb = (uint32_t)((N + BN - 1) / BN);
    const dim3 grid((uint32_t)(batch * mb * nb)), block(WM * WN * 64 * GROUPS);
    if (bk) gemm16_kernel<V, BM, BN, WM, WN, STEP, STAGES, GROUPS, true, true, SPLIT, false><<<grid, block, 0, s>>>(M, N, K, a, b, mb, nb, 1, e);
    else gemm16_kernel<V, BM, BN, WM, WN, STEP, STAGES, GROUPS, true, false, SPLIT, false><<<grid, block, 0, s>>>(M, N, K, a, b, mb, nb, 1, e);
}

}  // namespace netmax
