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

// Inclusive sum over the lanes of a wave, by row moves (a shuffle through LDS
// costs tens of times an addition, and the sums stand at the start of kernels
// of a few microseconds).
template <int CTRL, int ROWS>
inline __device__ int64_t moved(int64_t x) {
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xf, false);
    const int hi = __builtin_amdgcn_update_dpp(0, (int)(x >> 32), CTRL, ROWS, 0xf, false);
    return (int64_t)((uint64_t)(uint32_t)hi << 32 | lo);
}
inline __device__ int64_t wave_sums(int64_t x) {
    x += moved<0x111, 0xf>(x);                 // from 1, 2, 4, 8 lanes below, inside 16
    x += moved<0x112, 0xf>(x);
    x += moved<0x114, 0xf>(x);
    x += moved<0x118, 0xf>(x);
    x += moved<0x142, 0xa>(x);                 // the last lane of the 16 below, to the odd 16s
    x += moved<0x143, 0xc>(x);                 // the last lane of the lower 32
    return x;
}

// A value of one lane, or the same in all lanes, in scalar registers.
inline __device__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
inline __device__ int64_t uniform(int64_t x) {
    return (int64_t)((uint64_t)(uint32_t)uniform((int)(x >> 32)) << 32 | (uint32_t)uniform((int)x));
}
inline __device__ int64_t of_lane(int64_t x, int lane) {
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), lane) << 32 |
                     (uint32_t)__builtin_amdgcn_readlane((int)x, lane));
}

}  // namespace mptkv
