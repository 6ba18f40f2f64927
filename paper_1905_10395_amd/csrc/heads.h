// Activations of attention, [B, T, H, D] with dense columns and any other strides: their checks on the host.
#pragma once

#include <stdint.h>

#include <algorithm>

#include "common.h"

namespace lsgd {

struct Heads {
    void* p;
    int64_t lb, lt, lh;      // elements between entries, tokens, heads
};
inline Heads heads(const lsgd_heads& a) { return Heads{a.data, a.batch_stride, a.token_stride, a.head_stride}; }

inline bool on(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// There or not, aligned to its elements, and if it is written, rows that do not overlap.
inline lsgd_status check_heads(const char* who, const char* name, const lsgd_heads& a, int64_t B, int64_t T, int64_t H, int64_t D, int es, bool wanted,
                               bool written)
{
    if (wanted && !a.data) return set_error(LSGD_ERR_INVALID_ARG, "%s: %s is required", who, name);
    if (!wanted && a.data) return set_error(LSGD_ERR_INVALID_ARG, "%s: %s has no meaning here and must be NULL", who, name);
    if (!a.data) return LSGD_OK;
    if (!on(a.data, es)) return set_error(LSGD_ERR_INVALID_ARG, "%s: %s is not aligned to its element", who, name);
    struct Dim {
        int64_t stride, n;
    } d[3] = {{a.batch_stride, B}, {a.token_stride, T}, {a.head_stride, H}};
    for (const Dim& q : d)
        if (q.n > 1 && (q.stride < 0 || q.stride > INT64_C(1) << 40))
            return set_error(LSGD_ERR_SHAPE, "%s: %s has a negative or too large stride", who, name);
    if (!written) return LSGD_OK;
    // from the smallest stride on, each dimension steps over all that lies within it
    std::sort(d, d + 3, [](const Dim& x, const Dim& y) { return x.stride < y.stride; });
    int64_t extent = D;
    for (const Dim& q : d) {
        if (q.n <= 1) continue;
        if (q.stride < extent) return set_error(LSGD_ERR_SHAPE, "%s: rows of %s overlap", who, name);
        extent += (q.n - 1) * q.stride;
    }
    return LSGD_OK;
}

// Every row begins on 16 bytes.
inline bool wide_heads(const lsgd_heads& a, int64_t B, int64_t T, int64_t H, int es)
{
    const int64_t per = 16 / es;
    return !a.data || (on(a.data, 16) && (B <= 1 || a.batch_stride % per == 0) && (T <= 1 || a.token_stride % per == 0) && (H <= 1 || a.head_stride % per == 0));
}

} // namespace lsgd
