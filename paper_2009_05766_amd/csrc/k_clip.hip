// The norm of all gradients of a model, or of every model of a batch, and the gradients scaled down to a largest norm.
//
//   norm = sqrt(sum over all tensors of g^2),  factor = norm <= max ? 1 : max / norm,  out = factor g
// A square of a float is exact in double and sums are held in double, so that the norm is right to its last bit over the whole range of the type; factor g is taken in
// double and rounded once.  Bound by memory: everything is read once before the first value can be scaled, and again to scale it.
//
// A launch holds the places of up to LAUNCH tensors in its arguments.  A tensor's rows are cut into pieces of 16 bytes from each row's start, its pieces into
// units that the workgroups take in turn.  A wave finds a unit's tensor by comparing it with all tensors' first units at once, one in each lane.
#include "clip.h"
#include "piece.h"

namespace netmax {

constexpr int THREADS = 256, DEEP = 4;             // pieces that a thread has under way at once
constexpr int UNIT = THREADS * DEEP;
constexpr int MOST_WORKGROUPS = 2048;              // of a launch for all models: eight on every compute unit, and as many sums for every workgroup of the second pass to add up

struct Item { const void *g; void *out; int64_t ldg, sg, ldo, so, rows, cols; uint32_t first, bf16; };
constexpr int LAUNCH = 54;                         // arguments of a launch stay below 4096 bytes, and a wave has a lane for each tensor
struct Items { Item at[LAUNCH]; int32_t n; uint32_t units; };
static_assert(sizeof(Items) + 64 <= 4096, "arguments of a launch");

__device__ __forceinline__ int64_t row_pieces(const Item &t) { return t.bf16 ? (t.cols + 7) >> 3 : (t.cols + 3) >> 2; }

// The tensor of unit u: the last one whose first unit is not behind it.
struct Finder {
    uint32_t first;
    __device__ __forceinline__ Finder(const Items &items) : first((int)(threadIdx.x & 63) < items.n ? items.at[threadIdx.x & 63].first : 0xFFFFFFFFu) { }
    __device__ __forceinline__ int tensor(uint32_t u) const { return __builtin_amdgcn_readfirstlane(__popcll(__ballot(first <= u)) - 1); }
};

// Piece p of a tensor: its row and the first column there.
template <int VALUES> __device__ __forceinline__ void place_of(const Item &t, int64_t p, int64_t &row, int64_t &col)
{
    const int64_t each = row_pieces(t);
    if (t.rows == 1) row = 0;
    else if (each * t.rows <= 0xFFFFFFFFll) row = (uint32_t)p / (uint32_t)each;
    else row = p / each;
    col = (p - row * each) * VALUES;
}

template <typename T> __device__ __forceinline__ double squares_of(const Item &t, uint32_t u, int64_t model)
{
    constexpr int VALUES = Piece<T>::VALUES;
    const T *g = (const T *)t.g + model * t.sg;
    const int64_t all = row_pieces(t) * t.rows, p0 = (int64_t)(u - t.first) * UNIT + threadIdx.x;
    Piece<T> x[DEEP];
    int64_t row[DEEP], col[DEEP];
#pragma unroll
    for (int k = 0; k < DEEP; ++k) {
        place_of<VALUES>(t, p0 + k * THREADS, row[k], col[k]);
        if (p0 + k * THREADS < all) x[k] = fetch_piece(g + row[k] * t.ldg, col[k], t.cols);
    }
    double sum = 0.0;
#pragma unroll
    for (int k = 0; k < DEEP; ++k)
        if (p0 + k * THREADS < all) {
            settle_piece(x[k], col[k], t.cols);
#pragma unroll
            for (int e = 0; e < VALUES; ++e) sum = fma((double)x[k].get(e), (double)x[k].get(e), sum);
        }
    return sum;
}

__global__ void __launch_bounds__(THREADS) squares_kernel(Items items, double *partials, int64_t row_of_partials)
{
    __shared__ double room[THREADS / 64][1];
    const Finder find(items);
    double sum[1] = {0.0};
    for (uint32_t u = blockIdx.x; u < items.units; u += gridDim.x) {
        const Item &t = items.at[find.tensor(u)];
        sum[0] += t.bf16 ? squares_of<uint16_t>(t, u, blockIdx.y) : squares_of<float>(t, u, blockIdx.y);
    }
    row_sum<THREADS>(sum, room);
    if (threadIdx.x == 0) partials[blockIdx.y * row_of_partials + blockIdx.x] = sum[0];
}

__device__ __forceinline__ double total_of(const double *partials, int64_t n)
{
    __shared__ double room[THREADS / 64][1];
    double sum[1] = {0.0};
#pragma unroll 8
    for (int64_t k = threadIdx.x; k < n; k += THREADS) sum[0] += partials[k];
    row_sum<THREADS>(sum, room);
    return sum[0];
}

// One workgroup per model: its partial sums as one, and its norm.
__global__ void __launch_bounds__(THREADS) total_kernel(const double *partials, int64_t n, int64_t row_of_partials, double *total, float *norm)
{
    const double sum = total_of(partials + blockIdx.x * row_of_partials, n);
    if (threadIdx.x != 0) return;
    if (total) total[blockIdx.x] = sum;
    if (norm) norm[blockIdx.x] = (float)sqrt(sum);
}

template <typename T> __device__ __forceinline__ void scale_unit(const Item &t, uint32_t u, int64_t model, double factor)
{
    constexpr int VALUES = Piece<T>::VALUES;
    if (factor == 1.0 && t.out == t.g) return;
    const T *g = (const T *)t.g + model * t.sg;
    T *out = (T *)t.out + model * t.so;
    const int64_t all = row_pieces(t) * t.rows, p0 = (int64_t)(u - t.first) * UNIT + threadIdx.x;
    Piece<T> x[DEEP];
    int64_t row[DEEP], col[DEEP];
#pragma unroll
    for (int k = 0; k < DEEP; ++k) {
        place_of<VALUES>(t, p0 + k * THREADS, row[k], col[k]);
        if (p0 + k * THREADS < all) x[k] = fetch_piece(g + row[k] * t.ldg, col[k], t.cols);
    }
#pragma unroll
    for (int k = 0; k < DEEP; ++k)
        if (p0 + k * THREADS < all) {
            settle_piece(x[k], col[k], t.cols);
            float v[VALUES];
#pragma unroll
            for (int e = 0; e < VALUES; ++e) v[e] = (float)((double)x[k].get(e) * factor);
            Piece<T> y;
            y.set(v);
            store_piece(out + row[k] * t.ldo + col[k], t.cols - col[k], y);
        }
}

// Every workgroup adds up the n sums of its model itself.  Units from the last to the first: what the norm read last may still be in the last cache.
__global__ void __launch_bounds__(THREADS) scale_kernel(Items items, const double *sums, int64_t n, int64_t row_of_sums, float max_norm, float *norm)
{
    const Finder find(items);
    const double size = sqrt(total_of(sums + blockIdx.y * row_of_sums, n)), factor = size <= (double)max_norm ? 1.0 : (double)max_norm / size;
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) norm[blockIdx.y] = (float)size;
    for (uint32_t k = blockIdx.x; k < items.units; k += gridDim.x) {
        const uint32_t u = items.units - 1 - k;
        const Item &t = items.at[find.tensor(u)];
        if (t.bf16) scale_unit<uint16_t>(t, u, blockIdx.y, factor);
        else scale_unit<float>(t, u, blockIdx.y, factor);
    }
}

static uint32_t workgroups_of(uint32_t units, int64_t batch)
{
    const int64_t most = batch * 16 < MOST_WORKGROUPS ? MOST_WORKGROUPS / batch : 16;
    return units < most ? units : (uint32_t)most;
}

// The launches of a call: go(items, workgroups for each model).
template <class Go> static void with_launches(const ClipArgs &a, const Go &go)
{
    Items items;
    items.n = 0; items.units = 0;
    for (int64_t k = 0; k < a.n; ++k) {
        const netmax_gradient &t = a.tensors[k];
        if (t.rows == 0 || t.cols == 0) continue;
        const bool bf16 = t.dtype == NETMAX_BF16, dense = t.rows > 1 && t.ldg == t.cols && (!a.scale || t.ldo == t.cols);
        const int64_t rows = dense ? 1 : t.rows, cols = dense ? t.rows * t.cols : t.cols, each = bf16 ? (cols + 7) / 8 : (cols + 3) / 4;
        items.at[items.n++] = Item{t.g, a.scale ? t.out : nullptr, t.ldg, t.sg, t.ldo, t.so, rows, cols, items.units, bf16};
        items.units += (uint32_t)((each * rows + UNIT - 1) / UNIT);
        if (items.n == LAUNCH) {
            go(items, workgroups_of(items.units, a.batch));
            items.n = 0; items.units = 0;
        }
    }
    if (items.n > 0) go(items, workgroups_of(items.units, a.batch));
}

static int64_t partials_of(const ClipArgs &a)
{
    int64_t all = 0;
    with_launches(a, [&](const Items &, uint32_t workgroups) { all += workgroups; });
    return all;
}

int64_t clip_workspace(int64_t batch, int64_t n, const netmax_gradient *tensors)
{
    const ClipArgs norm{batch, n, tensors, false, 0.0f, nullptr}, scale{batch, n, tensors, true, 0.0f, nullptr};
    const int64_t p = partials_of(norm), q = partials_of(scale);    // rows that are dense in g alone are cut in other units for the norm alone
    return 8 * batch * ((p > q ? p : q) + 1);
}

void launch_clip(hipStream_t s, const ClipArgs &a, void *work)
{
    const uint32_t batch = (uint32_t)a.batch;
    const int64_t n = partials_of(a);
    double *total = (double *)work, *partials = total + batch;
    int64_t at = 0, launches = 0;
    with_launches(a, [&](const Items &items, uint32_t workgroups) {
        squares_kernel<<<dim3(workgroups, batch), THREADS, 0, s>>>(items, partials + at, n);
        at += workgroups;
        ++launches;
    });
    if (!a.scale || n > MOST_WORKGROUPS || launches == 0) {
        total_kernel<<<batch, THREADS, 0, s>>>(partials, n, n, total, a.norm);
        if (!a.scale) return;
        with_launches(a, [&](const Items &items, uint32_t workgroups) {
            scale_kernel<<<dim3(workgroups, batch), THREADS, 0, s>>>(items, total, 1, 1, a.max_norm, nullptr);
        });
        return;
    }
    bool first = true;
    with_launches(a, [&](const Items &items, uint32_t workgroups) {
        scale_kernel<<<dim3(workgroups, batch), THREADS, 0, s>>>(items, partials, n, n, a.max_norm, first ? a.norm : nullptr);
        first = false;
    });
}

}  // namespace netmax
