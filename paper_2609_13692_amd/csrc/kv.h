// Device pieces shared by the kernels of the paged key/value cache.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "common.h"

namespace mptkv {

// MPT_OK, or fails with the reason the descriptor cannot be used.
int check_cache(const mpt_kv_cache *c);

inline bool aligned16(const void *p) { return ((uintptr_t)p & 15) == 0; }

inline __device__ void flag(const mpt_kv_cache &c, uint32_t bits) { atomicOr(c.status, bits); }

}  // namespace mptkv
