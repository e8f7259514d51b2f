// Shared by the translation units of the 8-bit key/value cache.
#pragma once

#include "qtz_internal.cuh"

#define QTZ_KV_MIN_SCALE 7.888609052210118e-31f   // 2^-100: the scale of an all-zero block

// Geometry and pointers of a cache handed to an entry point.
qtz_status qtz_kv_check(const qtz_kv_cache* c);
