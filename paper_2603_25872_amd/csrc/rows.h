// Tensors [slots][tokens][columns] of the operators around a block's Linears: checks shared by their entry points.
#pragma once
#include <algorithm>
#include <utility>

#include "common.h"

namespace drf {

// The tensor with a stride of zero where a dimension has one element, as used_strides() of common.h.
inline drf_rows used_rows(const drf_rows& t, int slots, int tokens)
{
    return { t.data, slots > 1 ? t.slot_stride : 0, tokens > 1 ? t.token_stride : 0 };
}

// Whether two rows of such a tensor lie on one another: some i slots and j tokens apart, |i slot_stride - j token_stride| below a row's columns.  (Either direction of a stride
// gives the same distances.)  Where the rows of one index lie between two of the other, as in every layout that is in use, that is one comparison; otherwise one pass over the
// index with fewer elements, 2^15 of them at most.
inline bool rows_overlap(const drf_rows& t, int slots, int tokens, int columns)
{
    typedef __int128 wide;
    auto size = [](int64_t v) { return v < 0 ? -(wide)v : (wide)v; };
    wide a = size(t.slot_stride), b = size(t.token_stride);
    if ((slots > 1 && a < columns) || (tokens > 1 && b < columns)) return true;
    if (slots < 2 || tokens < 2) return false;
    int n = slots, m = tokens;
    if (a > b) { std::swap(a, b); std::swap(n, m); }                // a the smaller stride, of n elements
    if (b - (n - 1) * a >= columns) return false;
    auto near = [&](wide i, wide j) {
        const wide d = j * b - i * a;
        return i < n && j < m && (d < 0 ? -d : d) < columns;
    };
    for (int k = 1; k < std::min(n, m); ++k) {
        if (m <= n) {
            const wide i = k * b / a;
            if (near(i, k) || near(i + 1, k)) return true;
        } else {
            const wide j = k * a / b;
            if (near(k, j) || near(k, j + 1)) return true;
        }
    }
    return false;
}

inline drf_status check_rows_sizes(int slots, int tokens)
{
    if (slots < 0 || tokens < 0) DRF_FAIL(DRF_EINVAL, "slots and tokens must be >= 0");
    if ((long long)slots * tokens > 1LL << 30 || tokens > 1 << 30) DRF_FAIL(DRF_ESHAPE, "more than 2^30 tokens");
    return DRF_OK;
}

inline bool known_dtype(drf_dtype t) { return t == DRF_F32 || t == DRF_BF16; }

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool rows_aligned(const drf_rows& t, int unit) { return aligned16(t.data) && t.slot_stride % unit == 0 && t.token_stride % unit == 0; }

}  // namespace drf
