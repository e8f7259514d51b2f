// Shared by the translation units of the 8-bit key/value cache.
#pragma once

#include "qtz_internal.cuh"

#define QTZ_KV_MIN_SCALE 7.888609052210118e-31f   // 2^-100: the scale of an all-zero block

// Strides in elements of [tokens][heads][head_dim], for rows that start on 16 bytes; an axis of one element has none to keep.
static inline bool qtz_kv_strides_ok(int64_t tokens, int64_t token_stride, int64_t heads, int64_t head_stride)
{
    return ((tokens > 1 ? token_stride : 0) | (heads > 1 ? head_stride : 0)) % 8 == 0;
}

// Geometry and pointers of a cache handed to an entry point.
qtz_status qtz_kv_check(const qtz_kv_cache* c);
