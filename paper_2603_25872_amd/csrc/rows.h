// Tensors [slots][tokens][columns] of the operators around a block's Linears: checks shared by their entry points.
#pragma once
#include "common.h"

namespace drf {

// The tensor with a stride of zero where a dimension has one element, as used_strides() of common.h.
inline drf_rows used_rows(const drf_rows& t, int slots, int tokens)
{
    return { t.data, slots > 1 ? t.slot_stride : 0, tokens > 1 ? t.token_stride : 0 };
}

inline bool rows_overlap(const drf_rows& t, int slots, int tokens, int columns)
{
    return rows_overlap(drf_heads{ t.data, t.slot_stride, t.token_stride, 0 }, slots, tokens, 1, columns);
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
