// Argument checks of the entry points around the mixers.  None of them makes a HIP call.
#pragma once
#include "hy_checks.hpp"

namespace hy {

constexpr int64_t kMostElements = INT64_C(1) << 56;  // of one tensor, gaps between its rows included: no sum of bytes passes 63 bits

inline bool known(int32_t dtype) { return dtype == HY_F32 || dtype == HY_BF16; }

inline int64_t size_of(int32_t dtype) { return dtype == HY_F32 ? 4 : 2; }

// a * b * c <= kMostElements, for values that are not negative
inline bool fits(int64_t a, int64_t b, int64_t c) {
    return a == 0 || b == 0 || c == 0 || (a <= kMostElements / b && a * b <= kMostElements / c);
}

inline hy_status all_aligned(const Range* r, int n) {
    for (int i = 0; i < n; ++i)
        if (!aligned16(r[i].p)) return HY_ERR_ALIGN;
    return HY_OK;
}

// Begins where an element can.
inline bool on_element(const void* p, int64_t bytes) { return reinterpret_cast<uintptr_t>(p) % (uintptr_t)bytes == 0; }

}  // namespace hy
