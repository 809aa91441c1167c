// Rows of an embedding table for given tokens, and the gradient of the table.
//
//   y[t] = scale table[id[t]]                        (zeros where id[t] lies outside of the vocabulary)
//   dtable[v] = scale (sum of dy[t] over the tokens t with id[t] = v, in float, in a fixed order)
// Bound by memory: a row read and one written per token; dy read and the whole table written.  No atomics on values: every row of the table is summed by one place in
// a fixed order, so that a gradient's bits do not change from run to run.
//
// Few tokens: a wave or a workgroup for each token looks through all of them and, if its token is the first of its kind, sums the rows of the others; one launch.
// Many tokens: they are sorted (stable, by two digits) and the sorted ones cut into chunks of equal length, so that a frequent token's rows are read by as many workgroups as rare ones'; tokens
// whose rows end in another chunk than they begin leave partial sums, which are joined in order by four groups of lanes: n equal tokens are chains of 32 and of n / 128 additions.
#include "embed.h"
#include "piece.h"

#include <type_traits>

namespace netmax {

constexpr int THREADS = 256;

// Workgroups are numbered along x and y together: threads along a dimension of a launch have to be fewer than 2^32.
static dim3 grid_of(int64_t n, int64_t batch)
{
    constexpr int64_t ACROSS = 1 << 21;
    return dim3((uint32_t)(n < ACROSS ? n : ACROSS), (uint32_t)((n + ACROSS - 1) / ACROSS), (uint32_t)batch);
}
__device__ __forceinline__ uint32_t workgroup() { return blockIdx.y * gridDim.x + blockIdx.x; }

template <typename T> static int64_t pieces_of(int64_t width) { return (width + Piece<T>::VALUES - 1) / Piece<T>::VALUES; }

// ---- lookup ----------------------------------------------------------------------------------------------------------

constexpr int DEEP = 4;                            // pieces that a lane has under way at once

// LANES lanes for LANES * DEEP pieces of a row.
template <typename T, int LANES>
__global__ void __launch_bounds__(THREADS) embed_kernel(EmbedArgs a, uint32_t slabs)
{
    constexpr int VALUES = Piece<T>::VALUES, ROWS = THREADS / LANES;
    const uint32_t id = workgroup();
    const int64_t t = (int64_t)(id / slabs) * ROWS + threadIdx.x / LANES;
    if (t >= a.tokens) return;
    const int32_t token = a.ids[blockIdx.z * a.s_ids + t];
    const bool known = token >= 0 && token < a.vocab;
    const T *from = (const T *)a.table + blockIdx.z * a.st + (known ? token : 0) * a.ldt;
    T *to = (T *)a.y + blockIdx.z * a.sy + t * a.ldy;
    const int64_t at = ((int64_t)(id % slabs) * LANES * DEEP + threadIdx.x % LANES) * VALUES;
    Piece<T> x[DEEP];
#pragma unroll
    for (int k = 0; k < DEEP; ++k) {
        const int64_t col = at + k * LANES * VALUES;
        if (known && col < a.width) x[k] = fetch_piece(from, col, a.width);
    }
#pragma unroll
    for (int k = 0; k < DEEP; ++k) {
        const int64_t col = at + k * LANES * VALUES;
        if (col >= a.width) continue;
        settle_piece(x[k], col, a.width);
        float v[VALUES];
#pragma unroll
        for (int e = 0; e < VALUES; ++e) v[e] = known ? a.scale * x[k].get(e) : 0.0f;
        x[k].set(v);
        store_piece(to + col, a.width - col, x[k]);
    }
}

template <typename T> static void embed_of(hipStream_t s, const EmbedArgs &a)
{
    const auto go = [&](auto lanes) {
        constexpr int LANES = lanes(), ROWS = THREADS / LANES;
        const int64_t slabs = (pieces_of<T>(a.width) + LANES * DEEP - 1) / (LANES * DEEP);
        embed_kernel<T, LANES><<<grid_of((a.tokens + ROWS - 1) / ROWS * slabs, a.batch), THREADS, 0, s>>>(a, (uint32_t)slabs);
    };
    const int64_t n = pieces_of<T>(a.width);
    if (n <= 8 * DEEP) go(std::integral_constant<int, 8>());
    else go(std::integral_constant<int, 64>());
}

void launch_embed(hipStream_t s, const EmbedArgs &a)
{
    if (a.batch == 0 || a.tokens == 0) return;
    if (a.bf16) embed_of<uint16_t>(s, a);
    else embed_of<float>(s, a);
}

// ---- gradient: rows of the table ---------------------------------------------------------------------------------------

// A row of the table, or what is added to it.
template <typename T> __device__ __forceinline__ void leave_row(const EmbedArgs &a, T *row, int64_t col, const float (&sum)[Piece<T>::VALUES])
{
    constexpr int VALUES = Piece<T>::VALUES;
    float v[VALUES];
#pragma unroll
    for (int e = 0; e < VALUES; ++e) v[e] = a.scale * sum[e];
    Piece<T> out;
    if (a.accumulate) {
        Piece<T> old = fetch_piece(row, col, a.width);
        settle_piece(old, col, a.width);
#pragma unroll
        for (int e = 0; e < VALUES; ++e) v[e] += old.get(e);
    }
    out.set(v);
    store_piece(row + col, a.width - col, out);
}

// Rows first .. first + count - 1 (64 at most) without a bit in `hit` become zeros.
template <typename T> __device__ __forceinline__ void zero_rows(const EmbedArgs &a, T *table, int64_t first, int count, uint64_t hit)
{
    constexpr int VALUES = Piece<T>::VALUES;
    const uint32_t each = (uint32_t)((a.width + VALUES - 1) / VALUES);
    Piece<T> none;
    none.v = decltype(none.v){};
    if (each >= THREADS) {
        for (int r = 0; r < count; ++r) {
            if (hit >> r & 1) continue;
            for (uint32_t c = threadIdx.x; c < each; c += THREADS) store_piece(table + (first + r) * a.ldt + (int64_t)c * VALUES, a.width - (int64_t)c * VALUES, none);
        }
    } else {
        for (uint32_t k = threadIdx.x; k < each * count; k += THREADS) {
            const uint32_t r = k / each, c = k - r * each;
            if (!(hit >> r & 1)) store_piece(table + (first + r) * a.ldt + (int64_t)c * VALUES, a.width - (int64_t)c * VALUES, none);
        }
    }
}

// ---- gradient for few tokens -------------------------------------------------------------------------------------------

constexpr int FEW = 2048;                          // tokens
constexpr uint32_t AHEAD = 16;                     // rows that a lane has under way at once

// Clears rows of the table that no token has.
template <typename T> __device__ __forceinline__ void clear_few(const EmbedArgs &a, const int32_t *ids, T *table, int64_t first, int count)
{
    __shared__ unsigned long long hits;
    if (threadIdx.x == 0) hits = 0;
    int32_t seen[FEW / THREADS];
#pragma unroll
    for (int i = 0; i < FEW / THREADS; ++i) seen[i] = i * THREADS + threadIdx.x < a.tokens ? ids[i * THREADS + threadIdx.x] : -1;
    __syncthreads();
    unsigned long long hit = 0;
#pragma unroll
    for (int i = 0; i < FEW / THREADS; ++i) {
        const int64_t r = (int64_t)seen[i] - first;
        if (r >= 0 && r < count) hit |= 1ull << r;
    }
    if (hit) atomicOr(&hits, hit);
    __syncthreads();
    zero_rows(a, table, first, a.vocab - first < count ? (int)(a.vocab - first) : count, hits);
}

// The sum over `all` rows of dy of a piece from column col on: those of turn share, share + SHARES, ...
template <typename T, int SHARES> __device__ __forceinline__ void sum_rows(const EmbedArgs &a, const T *dy, const uint16_t *rows, uint32_t all, uint32_t share, int64_t col, float (&sum)[Piece<T>::VALUES])
{
    constexpr int VALUES = Piece<T>::VALUES;
    for (uint32_t k0 = share; k0 < all; k0 += SHARES * AHEAD) {
        Piece<T> x[AHEAD];
#pragma unroll
        for (uint32_t k = 0; k < AHEAD; ++k)
            if (k0 + k * SHARES < all) x[k] = fetch_piece(dy + (int64_t)rows[k0 + k * SHARES] * a.ldy, col, a.width);
#pragma unroll
        for (uint32_t k = 0; k < AHEAD; ++k)
            if (k0 + k * SHARES < all) {
                settle_piece(x[k], col, a.width);
#pragma unroll
                for (int e = 0; e < VALUES; ++e) sum[e] += x[k].get(e);
            }
    }
}

// Narrow rows: a wave for each token, LANES lanes for a row, the others take turns with them.
template <typename T, int LANES>
__global__ void __launch_bounds__(THREADS) embed_grad_narrow_kernel(EmbedArgs a, GradTurns turns, int rows_to_clear)
{
    constexpr int VALUES = Piece<T>::VALUES, SHARES = 64 / LANES, ROUNDS = 8;
    __shared__ uint16_t places[THREADS / 64][FEW];
    const int32_t *ids = a.ids + blockIdx.z * a.s_ids;
    T *table = (T *)a.table + blockIdx.z * a.st;
    const uint32_t id = workgroup(), tokens = (uint32_t)a.tokens, lane = threadIdx.x & 63;
    if (id >= turns.sums) {
        if (turns.clears(id)) clear_few(a, ids, table, (int64_t)(id - turns.sums) * rows_to_clear, rows_to_clear);
        return;
    }
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), t = id * (THREADS / 64) + wave;
    if (t >= tokens) return;
    const int32_t token = ids[t];
    if (token < 0 || token >= a.vocab) return;
    uint16_t *rows = places[wave];
    uint32_t all = 0;
    for (uint32_t u0 = 0; u0 < tokens; u0 += 64 * ROUNDS) {
        int32_t seen[ROUNDS];
#pragma unroll
        for (int i = 0; i < ROUNDS; ++i) seen[i] = u0 + i * 64 + lane < tokens ? ids[u0 + i * 64 + lane] : -1;
#pragma unroll
        for (int i = 0; i < ROUNDS; ++i) {
            const uint32_t u = u0 + i * 64;
            const bool same = seen[i] == token;
            const uint64_t mask = __ballot(same);
            if (mask != 0 && u + (uint32_t)__builtin_ctzll(mask) < t) return;              // it has been before
            if (same) rows[all + __popcll(mask & (((uint64_t)1 << lane) - 1))] = (uint16_t)(u + lane);
            all += (uint32_t)__popcll(mask);
        }
    }
    wave_order();
    const int64_t col = (int64_t)(lane % LANES) * VALUES;
    float sum[VALUES] = {};
    if (col < a.width) sum_rows<T, SHARES>(a, (const T *)a.y + blockIdx.z * a.sy, rows, all, lane / LANES, col, sum);
#pragma unroll
    for (int d = LANES; d < 64; d <<= 1)
#pragma unroll
        for (int e = 0; e < VALUES; ++e) sum[e] += __shfl_xor(sum[e], d);
    if (lane < LANES && col < a.width) leave_row(a, table + token * a.ldt, col, sum);
}

// Others: a workgroup for each token and slab of LANES pieces, whose lanes take turns at the token's rows.
template <typename T, int LANES>
__global__ void __launch_bounds__(THREADS) embed_grad_few_kernel(EmbedArgs a, uint32_t slabs, GradTurns turns, int rows_to_clear)
{
    constexpr int VALUES = Piece<T>::VALUES, SHARES = THREADS / LANES;
    __shared__ uint64_t place[FEW / 64];
    __shared__ uint16_t rows[FEW];
    __shared__ uint32_t count;
    __shared__ float part[SHARES > 1 ? SHARES : 1][SHARES > 1 ? LANES * VALUES : 1];
    const int32_t *ids = a.ids + blockIdx.z * a.s_ids;
    T *table = (T *)a.table + blockIdx.z * a.st;
    const uint32_t id = workgroup(), tokens = (uint32_t)a.tokens;
    if (id >= turns.sums) {
        if (turns.clears(id)) clear_few(a, ids, table, (int64_t)(id - turns.sums) * rows_to_clear, rows_to_clear);
        return;
    }
    int32_t seen[FEW / THREADS];                   // a share of the ids, all under way at once
#pragma unroll
    for (int i = 0; i < FEW / THREADS; ++i) seen[i] = i * THREADS + threadIdx.x < tokens ? ids[i * THREADS + threadIdx.x] : -1;
    const uint32_t t = id / slabs;
    const int32_t token = ids[t];
    if (token < 0 || token >= a.vocab) return;
    // where the token stands: a bit for each place; nothing to do if it has been before
    bool before = false;
#pragma unroll
    for (int i = 0; i < FEW / THREADS; ++i) {
        const uint32_t u = i * THREADS + threadIdx.x;
        const bool same = seen[i] == token;
        const uint64_t mask = __ballot(same);
        if ((threadIdx.x & 63) == 0) place[u / 64] = mask;
        before |= same && u < t;
    }
    if (__syncthreads_or(before)) return;
    // its places in order: a lane of the first wave for each 64 of them
    if (threadIdx.x < 64) {
        uint64_t m = threadIdx.x < FEW / 64 ? place[threadIdx.x] : 0;
        uint32_t upto = (uint32_t)__popcll(m);
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t v = __shfl_up(upto, d);
            upto += (int)threadIdx.x >= d ? v : 0u;
        }
        if (threadIdx.x == 63) count = upto;
        for (uint32_t at = upto - (uint32_t)__popcll(m); m; m &= m - 1) rows[at++] = (uint16_t)(threadIdx.x * 64 + (uint32_t)__builtin_ctzll(m));
    }
    __syncthreads();
    const uint32_t share = threadIdx.x / LANES;
    const int64_t col = ((int64_t)(id % slabs) * LANES + threadIdx.x % LANES) * VALUES;
    float sum[VALUES] = {};
    if (col < a.width) sum_rows<T, SHARES>(a, (const T *)a.y + blockIdx.z * a.sy, rows, count, share, col, sum);
    if constexpr (SHARES > 1) {
#pragma unroll
        for (int e = 0; e < VALUES; ++e) part[share][threadIdx.x % LANES * VALUES + e] = sum[e];
        __syncthreads();
        if (share != 0) return;
        for (int k = 1; k < SHARES; ++k)
#pragma unroll
            for (int e = 0; e < VALUES; ++e) sum[e] += part[k][threadIdx.x % LANES * VALUES + e];
    }
    if (col < a.width) leave_row(a, table + token * a.ldt, col, sum);
}

// ---- gradient for many tokens: sorting ---------------------------------------------------------------------------------
//
// Tokens outside of the vocabulary count as token `vocab`, which comes last.  Two stable passes by the lower and the upper half of a token's bits (one where 11 bits
// hold them all).  A pass is cut into tiles: a tile's workgroup counts its digits, and its first places come from the counts of all tiles.

constexpr int MOST_TILES = 64, MOST_BINS = 2048, WAVES = THREADS / 64, STEPS = 4;          // STEPS times 64 tokens of a wave are read at once

struct Sorting {
    int64_t tokens, vocab, tile; int32_t tiles, bits, passes;                               // bits of a digit
    const int32_t *ids; int64_t s_ids;
    uint32_t *counts[2];                           // [batch][tiles][1 << bits] of each pass
    uint32_t *token[2], *place[2];                 // [batch][tokens]: after each pass
    __device__ __forceinline__ uint32_t key(int64_t b, int64_t t) const
    {
        const int32_t k = ids[b * s_ids + t];
        return k >= 0 && k < vocab ? (uint32_t)k : (uint32_t)vocab;
    }
};

// Counts of the first pass's digits; those of the second start at 0.
__global__ void __launch_bounds__(THREADS) embed_count_kernel(Sorting s)
{
    __shared__ uint32_t count[MOST_BINS];
    const int bins = 1 << s.bits;
    const int64_t b = blockIdx.y, first = blockIdx.x * s.tile, end = first + s.tile < s.tokens ? first + s.tile : s.tokens, at = (b * s.tiles + blockIdx.x) * bins;
    for (int k = threadIdx.x; k < bins; k += THREADS) count[k] = 0;
    __syncthreads();
    for (int64_t t = first + threadIdx.x; t < end; t += THREADS) atomicAdd(&count[s.key(b, t) & (bins - 1)], 1u);
    __syncthreads();
    for (int k = threadIdx.x; k < bins; k += THREADS) {
        s.counts[0][at + k] = count[k];
        if (s.passes == 2) s.counts[1][at + k] = 0;
    }
}

// One pass: every wave takes a part of the tile, so that a token's place is the sum of what lies before its tile, before its wave's part and before it there.
template <bool SECOND> __global__ void __launch_bounds__(THREADS) embed_sort_kernel(Sorting s)
{
    __shared__ uint32_t next[WAVES][MOST_BINS], sums[THREADS];
    const int bins = 1 << s.bits, shift = SECOND ? s.bits : 0, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t b = blockIdx.y, part = s.tile / WAVES, first = blockIdx.x * s.tile + wave * part;
    const int64_t end = first + part < s.tokens ? first + part : s.tokens, row = b * s.tokens;
    const auto key = [&](int64_t t) { return SECOND ? s.token[0][row + t] : s.key(b, t); };
    for (int k = threadIdx.x; k < bins; k += THREADS)
#pragma unroll
        for (int w = 0; w < WAVES; ++w) next[w][k] = 0;
    __syncthreads();
#pragma unroll 4
    for (int64_t t = first + lane; t < end; t += 64) atomicAdd(&next[wave][key(t) >> shift & (bins - 1)], 1u);
    __syncthreads();
    // THREADS neighbours at a time: all tokens of smaller digits, and those of the same digit in tiles before
    uint32_t smaller = 0;
    const uint32_t *counts = s.counts[SECOND] + b * s.tiles * bins;
    for (int k0 = 0; k0 < bins; k0 += THREADS) {
        const int k = k0 + threadIdx.x;
        uint32_t all = 0, before = 0;
        if (k < bins)
#pragma unroll 32
            for (int i = 0; i < s.tiles; ++i) {
                const uint32_t c = counts[(int64_t)i * bins + k];
                all += c;
                before += i < (int)blockIdx.x ? c : 0u;
            }
        uint32_t upto = all;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t v = __shfl_up(upto, d);
            upto += lane >= d ? v : 0u;
        }
        __syncthreads();                           // the sums of the turn before have been read
        if (lane == 63) sums[wave] = upto;
        __syncthreads();
        uint32_t at = smaller + upto - all + before;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            if (w < wave) at += sums[w];
            smaller += sums[w];
        }
        if (k < bins)
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const uint32_t c = next[w][k];
                next[w][k] = at;
                at += c;
            }
    }
    __syncthreads();
    for (int64_t t0 = first; t0 < end; t0 += 64 * STEPS) {
        uint32_t tokens[STEPS], places[STEPS];
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            const int64_t t = t0 + i * 64 + lane;
            tokens[i] = t < end ? key(t) : 0u;
            places[i] = SECOND ? (t < end ? s.place[0][row + t] : 0u) : (uint32_t)t;
        }
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            if (t0 + i * 64 >= end) break;
            const bool here = t0 + i * 64 + lane < end;
            const uint32_t token = tokens[i], digit = token >> shift & (bins - 1);
            uint64_t same = __ballot(here);
            for (int j = 0; j < s.bits; ++j) {
                const uint64_t ones = __ballot(digit >> j & 1);
                same &= digit >> j & 1 ? ones : ~ones;
            }
            const int rank = __popcll(same & (((uint64_t)1 << lane) - 1));
            const uint32_t equal = (uint32_t)__popcll(same);
            const uint32_t at = here ? next[wave][digit] + rank : 0u;
            if (here) {
                s.token[SECOND][row + at] = token;
                s.place[SECOND][row + at] = places[i];
            }
            if (!SECOND && s.passes == 2) {        // the second pass's counts: one addition for all of a wave that have a token and a tile in common
                const uint32_t tile = at / (uint32_t)s.tile, upper = token >> s.bits;
                for (int j = 0; j < s.bits; ++j) {
                    const uint64_t ones = __ballot(upper >> j & 1);
                    same &= upper >> j & 1 ? ones : ~ones;
                }
                if (here) {
                    const int first = __builtin_ctzll(same), last = 63 - __builtin_clzll(same);
                    const bool together = __shfl(tile, first) == __shfl(tile, last);
                    if (!together) atomicAdd(&s.counts[1][(b * s.tiles + tile) * bins + upper], 1u);
                    else if (lane == first) atomicAdd(&s.counts[1][(b * s.tiles + tile) * bins + upper], (uint32_t)__popcll(same));
                }
            }
            wave_order();
            if (here && rank == 0) next[wave][digit] += equal;
            wave_order();
        }
    }
}

// ---- gradient for many tokens: sums ------------------------------------------------------------------------------------

constexpr int CHUNK = 32, MANY_ROWS = 64;

struct Sorted {
    const uint32_t *token, *place; int64_t padded; // [batch][tokens]; values of a row of partial sums
    float *head, *tail;                            // [batch][chunks][padded]: of a token that began in a chunk before; of one that goes on behind
    int64_t chunks;
};

template <typename T, int LANES>
__global__ void __launch_bounds__(THREADS) embed_sum_kernel(EmbedArgs a, Sorted s, uint32_t slabs, GradTurns turns)
{
    constexpr int VALUES = Piece<T>::VALUES, GROUPS = THREADS / LANES, DEEP = 8;
    __shared__ uint32_t token[GROUPS][CHUNK + 2], place[GROUPS][CHUNK];
    const uint32_t id = workgroup();
    const int64_t tokens = a.tokens, row = blockIdx.z * tokens;
    T *table = (T *)a.table + blockIdx.z * a.st;
    if (id >= turns.sums) {
        if (!turns.clears(id)) return;
        const int64_t first = (int64_t)(id - turns.sums) * MANY_ROWS, v = first + (threadIdx.x & 63);
        int64_t lo = 0, hi = tokens;               // the first token that is not less than v
        while (lo < hi) {
            const int64_t mid = (lo + hi) >> 1;
            if (s.token[row + mid] < (uint64_t)v) lo = mid + 1; else hi = mid;
        }
        const uint64_t hit = __ballot(lo < tokens && s.token[row + lo] == (uint64_t)v);
        zero_rows(a, table, first, a.vocab - first < MANY_ROWS ? (int)(a.vocab - first) : MANY_ROWS, hit);
        return;
    }
    const int64_t c0 = (int64_t)(id / slabs) * GROUPS;
    for (int k = threadIdx.x; k < GROUPS * (CHUNK + 2); k += THREADS) {
        const int g = k / (CHUNK + 2), i = k - g * (CHUNK + 2);
        const int64_t at = (c0 + g) * CHUNK + i - 1;
        token[g][i] = at >= 0 && at < tokens ? s.token[row + at] : 0xFFFFFFFFu;
        if (i >= 1 && i <= CHUNK) place[g][i - 1] = at < tokens ? s.place[row + at] : 0u;
    }
    __syncthreads();
    const int g = threadIdx.x / LANES;
    const int64_t c = c0 + g, piece = (int64_t)(id % slabs) * LANES + threadIdx.x % LANES, col = piece * VALUES;
    if (c >= s.chunks || col >= a.width) return;
    const T *dy = (const T *)a.y + blockIdx.z * a.sy;
    const uint32_t vocab = (uint32_t)a.vocab;
    float sum[VALUES] = {};
    bool begun = token[g][0] != token[g][1];       // the token at hand began in this chunk
    for (int i0 = 0; i0 < CHUNK; i0 += DEEP) {
        Piece<T> x[DEEP];
#pragma unroll
        for (int k = 0; k < DEEP; ++k)
            if (token[g][1 + i0 + k] < vocab) x[k] = fetch_piece(dy + (int64_t)place[g][i0 + k] * a.ldy, col, a.width);
#pragma unroll
        for (int k = 0; k < DEEP; ++k) {
            const uint32_t here = token[g][1 + i0 + k], after = token[g][2 + i0 + k];
            if (here >= vocab) return;             // the last ones
            settle_piece(x[k], col, a.width);
#pragma unroll
            for (int e = 0; e < VALUES; ++e) sum[e] += x[k].get(e);
            const bool last = here != after;
            if (!last && !(k == DEEP - 1 && i0 + DEEP == CHUNK)) continue;
            if (last && begun) {
                leave_row(a, table + here * a.ldt, col, sum);
            } else {
                float *to = (begun ? s.tail : s.head) + ((int64_t)blockIdx.z * s.chunks + c) * s.padded + col;
#pragma unroll
                for (int e = 0; e < VALUES; e += 4) *reinterpret_cast<f32x4 *>(to + e) = f32x4{sum[e], sum[e + 1], sum[e + 2], sum[e + 3]};
            }
#pragma unroll
            for (int e = 0; e < VALUES; ++e) sum[e] = 0.0f;
            begun = true;
        }
    }
}

// Tokens that begin in a chunk and go on behind it: their tail and the heads of the chunks that follow.
constexpr int JOIN_LANES = 64, JOIN_SHARES = THREADS / JOIN_LANES;
template <typename T> __device__ __forceinline__ void join_token(const EmbedArgs &a, const Sorted &s, int64_t c, uint32_t slab, float (*part)[JOIN_LANES * Piece<T>::VALUES])
{
    constexpr int VALUES = Piece<T>::VALUES;
    const uint32_t *token = s.token + blockIdx.z * a.tokens;
    const uint32_t v = token[(c + 1) * CHUNK];
    int64_t more = 0;                              // chunks behind this one that begin with it: a lane looks at each
    for (uint64_t m = ~(uint64_t)0; m == ~(uint64_t)0; more += __popcll(m)) {
        const int64_t k = c + 1 + more + (threadIdx.x & 63);
        m = __ballot(k < s.chunks && token[k * CHUNK] == v);
    }
    const int64_t last = c + more, col = ((int64_t)slab * JOIN_LANES + threadIdx.x % JOIN_LANES) * VALUES;
    const int share = threadIdx.x / JOIN_LANES;
    const int64_t at = ((int64_t)blockIdx.z * s.chunks + c) * s.padded + col;
    float sum[VALUES] = {};
    if (col < a.width) {
        if (share == 0)
#pragma unroll
            for (int e = 0; e < VALUES; ++e) sum[e] = s.tail[at + e];
#pragma unroll 4
        for (int64_t k = 1 + share; k <= last - c; k += JOIN_SHARES)
#pragma unroll
            for (int e = 0; e < VALUES; ++e) sum[e] += s.head[at + k * s.padded + e];
    }
    __syncthreads();                               // the token before has been added up
#pragma unroll
    for (int e = 0; e < VALUES; ++e) part[share][threadIdx.x % JOIN_LANES * VALUES + e] = sum[e];
    __syncthreads();
    if (share != 0 || col >= a.width) return;
    for (int k = 1; k < JOIN_SHARES; ++k)
#pragma unroll
        for (int e = 0; e < VALUES; ++e) sum[e] += part[k][threadIdx.x * VALUES + e];
    leave_row(a, (T *)a.table + blockIdx.z * a.st + v * a.ldt, col, sum);
}

// A workgroup looks through JOIN_CHUNKS chunks, a lane for each.
constexpr int JOIN_CHUNKS = 2;
template <typename T> __global__ void __launch_bounds__(THREADS) embed_join_kernel(EmbedArgs a, Sorted s, uint32_t slabs)
{
    __shared__ float part[JOIN_SHARES][JOIN_LANES * Piece<T>::VALUES];
    const uint32_t id = workgroup();
    const int64_t first = (int64_t)(id / slabs) * JOIN_CHUNKS, c = first + (threadIdx.x & 63), behind = (c + 1) * CHUNK;
    const uint32_t *token = s.token + blockIdx.z * a.tokens;
    bool begins = false;
    if ((threadIdx.x & 63) < JOIN_CHUNKS && behind < a.tokens) {
        const uint32_t v = token[behind];
        begins = v < (uint64_t)a.vocab && token[behind - 1] == v && (c == 0 || token[c * CHUNK - 1] != v);
    }
    for (uint64_t m = __ballot(begins); m; m &= m - 1) join_token<T>(a, s, first + __builtin_ctzll(m), id % slabs, part);
}

// ---- launches --------------------------------------------------------------------------------------------------------

static int64_t part_of_workspace(int64_t bytes) { return up_to(bytes, 256); }

struct Plan {
    Sorting sorting; Sorted sorted; int64_t bytes;
    Plan(const EmbedArgs &a, void *work)
    {
        int bits = 1;
        while ((int64_t)1 << bits <= a.vocab) ++bits;                                       // vocab itself, too
        sorting.passes = (1 << bits) <= MOST_BINS ? 1 : 2;
        sorting.bits = sorting.passes == 1 ? bits : (bits + 1) / 2;
        sorting.tokens = a.tokens; sorting.vocab = a.vocab; sorting.ids = a.ids; sorting.s_ids = a.s_ids;
        sorting.tile = up_to((a.tokens + MOST_TILES - 1) / MOST_TILES, 4 * THREADS);        // whole waves in every part
        sorting.tiles = (int32_t)((a.tokens + sorting.tile - 1) / sorting.tile);
        sorted.padded = up_to(a.width, 8);
        sorted.chunks = (a.tokens + CHUNK - 1) / CHUNK;
        char *at = (char *)work;
        const auto take = [&](int64_t n) { char *p = at; at += part_of_workspace(n * 4); return p; };
        const int64_t all = a.batch * a.tokens, counts = a.batch * sorting.tiles << sorting.bits, partial = a.batch * sorted.chunks * sorted.padded;
        for (int p = 0; p < 2; ++p) {
            const bool used = p < sorting.passes;
            sorting.counts[p] = (uint32_t *)take(used ? counts : 0);
            sorting.token[p] = (uint32_t *)take(used ? all : 0);
            sorting.place[p] = (uint32_t *)take(used ? all : 0);
        }
        sorted.token = sorting.token[sorting.passes - 1];
        sorted.place = sorting.place[sorting.passes - 1];
        sorted.head = (float *)take(partial);
        sorted.tail = (float *)take(partial);
        bytes = at - (char *)work;
    }
};

int64_t embed_grad_workspace(const EmbedArgs &a)
{
    return a.tokens <= FEW || a.batch == 0 ? 0 : Plan(a, nullptr).bytes;
}

template <typename T, class Go> static void with_lanes(int64_t width, const Go &go)
{
    const int64_t n = pieces_of<T>(width);
    if (n <= 8) go(std::integral_constant<int, 8>());
    else if (n <= 16) go(std::integral_constant<int, 16>());
    else if (n <= 32) go(std::integral_constant<int, 32>());
    else if (n <= 64) go(std::integral_constant<int, 64>());
    else if (n <= 128) go(std::integral_constant<int, 128>());
    else go(std::integral_constant<int, 256>());
}

template <typename T> static void embed_grad_of(hipStream_t s, const EmbedArgs &a, void *work)
{
    with_lanes<T>(a.width, [&](auto lanes) {
        constexpr int LANES = lanes(), GROUPS = THREADS / LANES;
        const int64_t slabs = (pieces_of<T>(a.width) + LANES - 1) / LANES;
        if (a.tokens <= FEW) {
            // rows that a workgroup looks whether to clear: 64 while they are short
            const int rows_to_clear = a.width * (int64_t)sizeof(T) <= 1024 ? 64 : 16;
            const int64_t zeros = a.accumulate ? 0 : (a.vocab + rows_to_clear - 1) / rows_to_clear;
            if constexpr (LANES <= 64) {
                const int64_t sums = (a.tokens + THREADS / 64 - 1) / (THREADS / 64);
                if (sums + zeros > 0) embed_grad_narrow_kernel<T, LANES><<<grid_of(sums + zeros, a.batch), THREADS, 0, s>>>(a, GradTurns{(uint32_t)sums, (uint32_t)zeros}, rows_to_clear);
            } else {
                const int64_t sums = a.tokens * slabs;
                if (sums + zeros > 0) embed_grad_few_kernel<T, LANES><<<grid_of(sums + zeros, a.batch), THREADS, 0, s>>>(a, (uint32_t)slabs, GradTurns{(uint32_t)sums, (uint32_t)zeros}, rows_to_clear);
            }
            return;
        }
        const Plan plan(a, work);
        const dim3 tiles(plan.sorting.tiles, (uint32_t)a.batch);
        embed_count_kernel<<<tiles, THREADS, 0, s>>>(plan.sorting);
        embed_sort_kernel<false><<<tiles, THREADS, 0, s>>>(plan.sorting);
        if (plan.sorting.passes == 2) embed_sort_kernel<true><<<tiles, THREADS, 0, s>>>(plan.sorting);
        const int64_t sums = (plan.sorted.chunks + GROUPS - 1) / GROUPS * slabs, zeros = a.accumulate ? 0 : (a.vocab + MANY_ROWS - 1) / MANY_ROWS;
        embed_sum_kernel<T, LANES><<<grid_of(sums + zeros, a.batch), THREADS, 0, s>>>(a, plan.sorted, (uint32_t)slabs, GradTurns{(uint32_t)sums, (uint32_t)zeros});
        const int64_t join = (pieces_of<T>(a.width) + JOIN_LANES - 1) / JOIN_LANES;
        embed_join_kernel<T><<<grid_of((plan.sorted.chunks + JOIN_CHUNKS - 1) / JOIN_CHUNKS * join, a.batch), THREADS, 0, s>>>(a, plan.sorted, (uint32_t)join);
    });
}

void launch_embed_grad(hipStream_t s, const EmbedArgs &a, void *work)
{
    if (a.batch == 0) return;
    if (a.bf16) embed_grad_of<uint16_t>(s, a, work);
    else embed_grad_of<float>(s, a, work);
}

}  // namespace netmax
