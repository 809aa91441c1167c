// The norm of all gradients of a model, or of every model of a batch, and the gradients scaled down to a largest norm.
//
//   norm = sqrt(sum over all tensors of g^2),  factor = norm <= max ? 1 : max / norm,  out = factor g
// A square of a float is exact in double and sums are held in double, so that the norm is right to its last bit over the whole range of the type; factor g is taken in
// double and rounded once (bfloat16 by way of a float that keeps what the double was beside: 8 us of 1012 for 906 M values, 0.9 of 18 for 37 odd tensors).  Bound by memory: everything is read once
// before the first value can be scaled, and again to scale it.
//
// A launch holds the places of many tensors in its arguments.  A tensor's rows are cut into pieces of 16 bytes from each row's start, its pieces into
// units that the workgroups take in turn.  A wave finds a unit's tensor by comparing it with all tensors' first units at once, one or two in each lane.
//
// 96 tensors of a model of 24 layers, 906 M values in bfloat16: 1012 us for 5.4 GB read and written, the rate of a large copy; 37 tensors of odd sizes, 18 MB, 18 us.
#include "clip.h"
#include "piece.h"

#include <type_traits>

namespace netmax {

constexpr int THREADS = 256, DEEP = 4;             // pieces that a thread has under way at once
constexpr int UNIT = THREADS * DEEP;
constexpr int MOST_WORKGROUPS = 2048;              // of a launch for all models: eight on every compute unit, and as many sums for every workgroup of the second pass to add up

// Tensors of one row each whose models lie equally far apart take less room: more of them go into one launch (400 tensors of 16 x 16 in 4 pairs of launches instead of 8).
template <bool DENSE> struct Item;
template <> struct Item<true> {
    const void *g; void *out; int64_t cols; uint32_t first, bf16;
    __device__ __forceinline__ int64_t rows() const { return 1; }
    __device__ __forceinline__ int64_t ldg() const { return 0; }
    __device__ __forceinline__ int64_t ldo() const { return 0; }
};
template <> struct Item<false> {
    const void *g; void *out; int64_t cols; uint32_t first, bf16; int64_t rows_, ldg_, ldo_, sg, so;
    __device__ __forceinline__ int64_t rows() const { return rows_; }
    __device__ __forceinline__ int64_t ldg() const { return ldg_; }
    __device__ __forceinline__ int64_t ldo() const { return ldo_; }
};
template <bool DENSE> struct Items {
    static constexpr int MOST = DENSE ? 120 : 54;  // arguments of a launch stay below 4096 bytes, and a wave has two lanes' words for each tensor
    Item<DENSE> at[MOST]; int64_t sg, so; int32_t n; uint32_t units;
    __device__ __forceinline__ int64_t g_apart(const Item<DENSE> &t) const { if constexpr (DENSE) return sg; else return t.sg; }
    __device__ __forceinline__ int64_t out_apart(const Item<DENSE> &t) const { if constexpr (DENSE) return so; else return t.so; }
};
static_assert(sizeof(Items<true>) + 64 <= 4096 && sizeof(Items<false>) + 64 <= 4096, "arguments of a launch");

template <bool DENSE> __device__ __forceinline__ int64_t row_pieces(const Item<DENSE> &t) { return t.bf16 ? (t.cols + 7) >> 3 : (t.cols + 3) >> 2; }

// The tensor of unit u: the last one whose first unit is not behind it.
template <bool DENSE> struct Finder {
    uint32_t first, second;
    __device__ __forceinline__ Finder(const Items<DENSE> &items)
    {
        const int lane = threadIdx.x & 63;
        first = lane < items.n ? items.at[lane].first : 0xFFFFFFFFu;
        second = DENSE && lane + 64 < items.n ? items.at[lane + 64].first : 0xFFFFFFFFu;
    }
    __device__ __forceinline__ int tensor(uint32_t u) const
    {
        int before = __popcll(__ballot(first <= u));
        if (DENSE) before += __popcll(__ballot(second <= u));
        return __builtin_amdgcn_readfirstlane(before - 1);
    }
};

// Piece p of a tensor: its row and the first column there.
template <int VALUES, bool DENSE> __device__ __forceinline__ void place_of(const Item<DENSE> &t, int64_t p, int64_t &row, int64_t &col)
{
    const int64_t each = row_pieces(t);
    if (t.rows() == 1) row = 0;
    else if (each * t.rows() <= 0xFFFFFFFFll) row = (uint32_t)p / (uint32_t)each;
    else row = p / each;
    col = (p - row * each) * VALUES;
}

// A unit's pieces in the hands of THREADS threads, of which this is number `thread`.
template <typename T, bool DENSE> struct Held {
    static constexpr int VALUES = Piece<T>::VALUES;
    Piece<T> x[DEEP]; int64_t row[DEEP], col[DEEP], p0, all;
    __device__ __forceinline__ Held(const Items<DENSE> &items, const Item<DENSE> &t, uint32_t u, int64_t model, uint32_t thread)
    {
        const T *g = (const T *)t.g + model * items.g_apart(t);
        all = row_pieces(t) * t.rows();
        p0 = (int64_t)(u - t.first) * UNIT + thread;
#pragma unroll
        for (int k = 0; k < DEEP; ++k) {
            place_of<VALUES>(t, p0 + k * THREADS, row[k], col[k]);
            if (there(k)) x[k] = fetch_piece(g + row[k] * t.ldg(), col[k], t.cols);
        }
    }
    __device__ __forceinline__ bool there(int k) const { return p0 + k * THREADS < all; }
};

template <typename T, bool DENSE> __device__ __forceinline__ double squares_of(const Items<DENSE> &items, const Item<DENSE> &t, uint32_t u, int64_t model, uint32_t thread)
{
    Held<T, DENSE> held(items, t, u, model, thread);
    double sum = 0.0;
#pragma unroll
    for (int k = 0; k < DEEP; ++k)
        if (held.there(k)) {
            settle_piece(held.x[k], held.col[k], t.cols);
#pragma unroll
            for (int e = 0; e < Piece<T>::VALUES; ++e) sum = fma((double)held.x[k].get(e), (double)held.x[k].get(e), sum);
        }
    return sum;
}

// v for a value of type T, in float.  bfloat16 is rounded from that float, which therefore holds v cut to 10 bits behind the point, with a last bit of 1 where anything was cut: so it is the middle of
// two bfloat16 values only where v is, and float has it as it is (but below half of bfloat16's smallest value, where all is 0).
template <typename T> __device__ __forceinline__ float rounded_for(double v)
{
    if constexpr (sizeof(T) == 4) return (float)v;
    const uint32_t hi = (uint32_t)__double2hiint(v), cut = (hi & 0x3FFu) | (uint32_t)__double2loint(v);
    return (float)__hiloint2double((int)((hi & ~0x3FFu) | (cut != 0 ? 0x400u : 0u)), 0);
}

template <typename T, bool DENSE> __device__ __forceinline__ void scale_unit(const Items<DENSE> &items, const Item<DENSE> &t, uint32_t u, int64_t model, uint32_t thread, double factor)
{
    constexpr int VALUES = Piece<T>::VALUES;
    if (factor == 1.0 && t.out == t.g) return;
    T *out = (T *)t.out + model * items.out_apart(t);
    Held<T, DENSE> held(items, t, u, model, thread);
#pragma unroll
    for (int k = 0; k < DEEP; ++k)
        if (held.there(k)) {
            settle_piece(held.x[k], held.col[k], t.cols);
            float v[VALUES];
#pragma unroll
            for (int e = 0; e < VALUES; ++e) v[e] = rounded_for<T>((double)held.x[k].get(e) * factor);
            Piece<T> y;
            y.set(v);
            store_piece(out + held.row[k] * t.ldo() + held.col[k], t.cols - held.col[k], y);
        }
}

__device__ __forceinline__ double factor_of(double size, float max_norm) { return size <= (double)max_norm ? 1.0 : (double)max_norm / size; }

template <bool DENSE> __global__ void __launch_bounds__(THREADS) squares_kernel(Items<DENSE> items, double *partials, int64_t row_of_partials)
{
    __shared__ double room[THREADS / 64][1];
    const Finder<DENSE> find(items);
    double sum[1] = {0.0};
    for (uint32_t u = blockIdx.x; u < items.units; u += gridDim.x) {
        const Item<DENSE> &t = items.at[find.tensor(u)];
        sum[0] += t.bf16 ? squares_of<uint16_t>(items, t, u, blockIdx.y, threadIdx.x) : squares_of<float>(items, t, u, blockIdx.y, threadIdx.x);
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
    total[blockIdx.x] = sum;
    if (norm) norm[blockIdx.x] = (float)sqrt(sum);
}

// Every workgroup adds up the n sums of its model itself.  Units from the last to the first: what the norm read last may still be in the last cache.
template <bool DENSE> __global__ void __launch_bounds__(THREADS) scale_kernel(Items<DENSE> items, const double *sums, int64_t n, int64_t row_of_sums, float max_norm, float *norm)
{
    const Finder<DENSE> find(items);
    const double size = sqrt(total_of(sums + blockIdx.y * row_of_sums, n)), factor = factor_of(size, max_norm);
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) norm[blockIdx.y] = (float)size;
    for (uint32_t k = blockIdx.x; k < items.units; k += gridDim.x) {
        const uint32_t u = items.units - 1 - k;
        const Item<DENSE> &t = items.at[find.tensor(u)];
        if (t.bf16) scale_unit<uint16_t>(items, t, u, blockIdx.y, threadIdx.x, factor);
        else scale_unit<float>(items, t, u, blockIdx.y, threadIdx.x, factor);
    }
}

// Models of few units: norm and scaling by one workgroup, whose every THREADS threads take units in turn, in one launch (a gradient of 256 values 10.4 -> 6.7 us).
constexpr int SMALL_THREADS = 1024;
constexpr uint32_t SMALL_UNITS = 4;                // one for each THREADS threads (with 12, 90000 bfloat16 values in four padded tensors took 23 us, by two launches 11)
template <bool DENSE> __global__ void __launch_bounds__(SMALL_THREADS) clip_small_kernel(Items<DENSE> items, int scale, float max_norm, float *norm)
{
    __shared__ double room[SMALL_THREADS / 64][1];
    const Finder<DENSE> find(items);
    const uint32_t thread = threadIdx.x % THREADS, mine = __builtin_amdgcn_readfirstlane(threadIdx.x / THREADS);
    double sum[1] = {0.0};
    for (uint32_t u = mine; u < items.units; u += SMALL_THREADS / THREADS) {
        const Item<DENSE> &t = items.at[find.tensor(u)];
        sum[0] += t.bf16 ? squares_of<uint16_t>(items, t, u, blockIdx.x, thread) : squares_of<float>(items, t, u, blockIdx.x, thread);
    }
    row_sum<SMALL_THREADS>(sum, room);             // everything has been read before anything is written
    const double size = sqrt(sum[0]), factor = factor_of(size, max_norm);
    if (norm && threadIdx.x == 0) norm[blockIdx.x] = (float)size;
    if (!scale) return;
    for (uint32_t u = mine; u < items.units; u += SMALL_THREADS / THREADS) {
        const Item<DENSE> &t = items.at[find.tensor(u)];
        if (t.bf16) scale_unit<uint16_t>(items, t, u, blockIdx.x, thread, factor);
        else scale_unit<float>(items, t, u, blockIdx.x, thread, factor);
    }
}

static uint32_t workgroups_of(uint32_t units, int64_t batch)
{
    const int64_t most = batch * 16 < MOST_WORKGROUPS ? MOST_WORKGROUPS / batch : 16;
    return units < most ? units : (uint32_t)most;
}

static bool is_dense(const ClipArgs &a, const netmax_gradient &t) { return t.rows <= 1 || (t.ldg == t.cols && (!a.scale || t.ldo == t.cols)); }
static bool all_dense(const ClipArgs &a)
{
    const netmax_gradient *first = nullptr;
    for (int64_t k = 0; k < a.n; ++k) {
        const netmax_gradient &t = a.tensors[k];
        if (t.rows == 0 || t.cols == 0) continue;
        if (!first) first = &t;
        if (!is_dense(a, t) || (a.batch > 1 && (t.sg != first->sg || (a.scale && t.so != first->so)))) return false;
    }
    return true;
}

// The launches of a call: go(items, workgroups for each model, whether there are others).
template <bool DENSE, class Go> static void with_launches_of(const ClipArgs &a, const Go &go)
{
    Items<DENSE> items;
    items.n = 0; items.units = 0;
    bool others = false;
    for (int64_t k = 0; k < a.n; ++k) {
        const netmax_gradient &t = a.tensors[k];
        if (t.rows == 0 || t.cols == 0) continue;
        if (items.n == Items<DENSE>::MOST) {
            others = true;
            go(items, workgroups_of(items.units, a.batch), others);
            items.n = 0; items.units = 0;
        }
        const bool bf16 = t.dtype == NETMAX_BF16, dense = is_dense(a, t);
        const int64_t rows = dense ? 1 : t.rows, cols = dense ? t.rows * t.cols : t.cols, each = bf16 ? (cols + 7) / 8 : (cols + 3) / 4;
        Item<DENSE> &to = items.at[items.n++];
        to.g = t.g; to.out = a.scale ? t.out : nullptr; to.cols = cols; to.first = items.units; to.bf16 = bf16;
        if constexpr (DENSE) { items.sg = t.sg; items.so = t.so; }
        else { to.rows_ = rows; to.ldg_ = t.ldg; to.ldo_ = t.ldo; to.sg = t.sg; to.so = t.so; }
        items.units += (uint32_t)((each * rows + UNIT - 1) / UNIT);
    }
    if (items.n > 0) go(items, workgroups_of(items.units, a.batch), others);
}
template <class Go> static void with_launches(const ClipArgs &a, const Go &go)
{
    if (all_dense(a)) with_launches_of<true>(a, go);
    else with_launches_of<false>(a, go);
}

static int64_t partials_of(const ClipArgs &a)
{
    int64_t all = 0;
    with_launches(a, [&](const auto &, uint32_t workgroups, bool) { all += workgroups; });
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
    int64_t at = 0;
    bool done = false;
    with_launches(a, [&](const auto &items, uint32_t workgroups, bool others) {
        constexpr bool DENSE = std::is_same_v<std::decay_t<decltype(items)>, Items<true>>;
        if (!others && n == workgroups && items.units <= SMALL_UNITS) {
            clip_small_kernel<DENSE><<<batch, SMALL_THREADS, 0, s>>>(items, a.scale, a.max_norm, a.norm);
            done = true;
            return;
        }
        squares_kernel<DENSE><<<dim3(workgroups, batch), THREADS, 0, s>>>(items, partials + at, n);
        at += workgroups;
    });
    if (done) return;
    const bool few = n > 0 && n <= MOST_WORKGROUPS;
    if (!a.scale || !few) total_kernel<<<batch, THREADS, 0, s>>>(partials, n, n, total, a.norm);
    if (!a.scale) return;
    bool first = few;
    with_launches(a, [&](const auto &items, uint32_t workgroups, bool) {
        constexpr bool DENSE = std::is_same_v<std::decay_t<decltype(items)>, Items<true>>;
        if (few) scale_kernel<DENSE><<<dim3(workgroups, batch), THREADS, 0, s>>>(items, partials, n, n, a.max_norm, first ? a.norm : nullptr);
        else scale_kernel<DENSE><<<dim3(workgroups, batch), THREADS, 0, s>>>(items, total, 1, 1, a.max_norm, nullptr);
        first = false;
    });
}

}  // namespace netmax
