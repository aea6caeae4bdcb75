// heads.h -- host-side checks of the entry points that take tensors of heads
// (mx_heads; internal).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "mxnorm.h"
#include "status.h"

namespace mxk {

inline bool aligned(const void *p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

// One tensor of heads: an input (any strides, 0 among them) or an output,
// whose heads must not share elements.
inline mx_status check_heads(const mx_heads *h, const char *name, int64_t T, int64_t D, int64_t heads, bool out)
{
    if (!h)
        return fail(MX_EINVAL, "%s is NULL", name);
    if (h->heads != heads)
        return fail(MX_EINVAL, "%s has %lld heads, not %lld", name, (long long)h->heads, (long long)heads);
    if (T == 0 || heads == 0)
        return MX_OK;
    const int64_t t = T > 1 ? h->token_stride : 0, s = heads > 1 ? h->head_stride : 0;
    if (!h->data || !aligned(h->data, 16) || t % 8 != 0 || s % 8 != 0)
        return fail(MX_EINVAL, "%s must be non-NULL, 16-byte aligned, its strides multiples of 8", name);
    if (t < 0 || s < 0 || t > INT64_MAX / 4 / T || s > INT64_MAX / 4 / heads)
        return fail(MX_EINVAL, "%s: bad strides", name);
    if (out) {
        const bool by_token = (heads == 1 || s >= D) && (T == 1 || t >= s * (heads - 1) + D);
        const bool by_head = (T == 1 || t >= D) && (heads == 1 || s >= t * (T - 1) + D);
        if (!by_token && !by_head)
            return fail(MX_EINVAL, "%s: its heads overlap", name);
    }
    return MX_OK;
}

// A launch's threads are counted in 32 bits.
inline bool launchable(int64_t workgroups, int64_t threads) { return workgroups <= (int64_t)UINT32_MAX / threads; }

inline mx_status launched()
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? MX_OK : fail(MX_EHIP, "kernel launch failed: %s", hipGetErrorString(e));
}

} // namespace mxk
