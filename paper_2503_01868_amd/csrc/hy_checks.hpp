// Argument checks that the entry points share.  None of them makes a HIP call.
#pragma once
#include <stdint.h>

#include "hyena.h"

namespace hy {

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline bool overlaps2(const void* a, int64_t abytes, const void* b, int64_t bbytes) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x < y + (uintptr_t)bbytes && y < x + (uintptr_t)abytes;
}

inline bool overlaps(const void* a, const void* b, int64_t bytes) { return overlaps2(a, bytes, b, bytes); }

// A device buffer an entry point reads or writes.
struct Range {
    const void* p;
    int64_t bytes;
};

inline int64_t filter_bytes(int64_t D, int32_t group, int32_t lh) { return (D / group) * (int64_t)lh * (int64_t)sizeof(float); }

// Every written buffer must be disjoint from every other buffer of the call (activations, filter tables, filter
// gradient, workspace alike).  Empty ranges never overlap anything.
inline hy_status check_disjoint(const Range* rd, int n_rd, const Range* wr, int n_wr) {
    for (int o = 0; o < n_wr; ++o) {
        if (wr[o].bytes <= 0) continue;
        for (int i = 0; i < n_rd; ++i)
            if (rd[i].bytes > 0 && overlaps2(wr[o].p, wr[o].bytes, rd[i].p, rd[i].bytes)) return HY_ERR_ALIGN;
        for (int o2 = o + 1; o2 < n_wr; ++o2)
            if (wr[o2].bytes > 0 && overlaps2(wr[o].p, wr[o].bytes, wr[o2].p, wr[o2].bytes)) return HY_ERR_ALIGN;
    }
    return HY_OK;
}

// The workspace of a call must be present, aligned, large enough and disjoint from every other buffer.
inline hy_status check_workspace(const void* ws, int64_t ws_bytes, int64_t need, const Range* others, int n_others) {
    if (need <= 0) return HY_OK;
    if (!ws) return HY_ERR_NULL;
    if (!aligned16(ws)) return HY_ERR_ALIGN;
    if (ws_bytes < need) return HY_ERR_SHAPE;
    const Range w{ws, need};
    return check_disjoint(others, n_others, &w, 1);
}

inline bool empty(int64_t B, int64_t L, int64_t D) { return B == 0 || L == 0 || D == 0; }

}  // namespace hy
