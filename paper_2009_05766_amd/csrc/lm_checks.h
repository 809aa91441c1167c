// What the C entry points of the operators for language models look at before they launch anything.
#pragma once
#include "errors.h"
#include "places.h"

#include <hip/hip_runtime.h>

#include <cstdio>

namespace netmax {

inline int launched(const char *what)
{
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return NETMAX_OK;
    char buf[200];
    snprintf(buf, sizeof buf, "%s: %s", what, hipGetErrorString(e));
    return netmax_fail(NETMAX_EDEVICE, buf);
}

inline bool dtype_known(int32_t d) { return d == NETMAX_F32 || d == NETMAX_BF16; }
inline int64_t size_of(int32_t dtype) { return dtype == NETMAX_BF16 ? 2 : 4; }
inline bool aligned(const void *p, int32_t dtype) { return (uintptr_t)p % size_of(dtype) == 0; }

// Sizes that keep every product of them, in bytes, far inside 64 bits.
constexpr int64_t MOST = (int64_t)1 << 40;
inline bool product_fits(int64_t a, int64_t b, int64_t c)
{
    return a >= 0 && b >= 0 && c >= 0 && (double)a * (double)b * (double)c <= (double)MOST && a <= MOST && b <= MOST && c <= MOST;
}
// Blocks of 64 x 64 results of a whole batch: one launch's workgroups of 256 threads, and a launch has fewer than 2^32 of them.
inline bool blocks_fit(int64_t batch, int64_t m, int64_t n) { return (double)batch * (double)((m + 63) / 64) * (double)((n + 63) / 64) < 16777216.0; }

inline bool strides_ok(int64_t batch, int64_t rows, int64_t cols, int64_t ld, int64_t step)
{
    return (rows <= 1 || ld >= cols) && ld >= 0 && ld <= MOST && step >= 0 && step <= MOST && (rows == 0 || product_fits(rows, ld, 1)) && product_fits(batch, step, 1);
}

// `written`: results of a batch need memory of their own each, if there are any.
inline int check_matrix(const char *name, const void *p, bool needed, int32_t dtype, int64_t batch, int64_t rows, int64_t cols, int64_t ld, int64_t step, bool written = false)
{
    char buf[160];
    if (!p) {
        if (!needed) return NETMAX_OK;
        snprintf(buf, sizeof buf, "%s is NULL", name);
        return netmax_fail(NETMAX_EINVAL, buf);
    }
    if (aligned(p, dtype) && strides_ok(batch, rows, cols, ld, step) &&
        !(written && batch > 1 && rows > 0 && cols > 0 && (step == 0 || batch_overlaps(Place(p, size_of(dtype), batch, rows, cols, ld, step))))) return NETMAX_OK;
    snprintf(buf, sizeof buf, "%s: misaligned, or rows closer together than they are long, or a negative stride, or results in the same place", name);
    return netmax_fail(NETMAX_EINVAL, buf);
}

#define TRY(call) do { const int rc_ = (call); if (rc_ != NETMAX_OK) return rc_; } while (0)

inline int check_work(const void *work, int64_t have, int64_t need)
{
    if (need == 0 || (work && have >= need && (uintptr_t)work % 256 == 0)) return NETMAX_OK;
    char buf[160];
    snprintf(buf, sizeof buf, "the workspace must be 256-byte aligned and hold %lld bytes (%lld given)", (long long)need, (long long)have);
    return netmax_fail(NETMAX_EINVAL, buf);
}

// ---- memory that a call writes: nothing that it still reads, and nothing twice ---------------------------------------

struct Named { const char *name; Place at; };

inline int check_apart(const Named &a, const Named &b)
{
    if (!share_memory(a.at, b.at)) return NETMAX_OK;
    char buf[160];
    snprintf(buf, sizeof buf, "%s and %s share memory", a.name, b.name);
    return netmax_fail(NETMAX_EINVAL, buf);
}
template <int N> int check_apart(const Named &a, const Named (&others)[N])
{
    for (const Named &o : others) TRY(check_apart(a, o));
    return NETMAX_OK;
}
// The workspace, if the call needs one, lies apart from everything else.
inline Named workspace_at(const void *work, int64_t bytes) { return Named{"the workspace", Place(bytes ? work : nullptr, 1, 1, 1, bytes, 0, 0)}; }

inline int64_t up(int64_t n) { return (n + 255) / 256 * 256; }      // parts of a workspace

}  // namespace netmax
