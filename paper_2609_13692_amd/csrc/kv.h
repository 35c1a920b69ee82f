// Device pieces shared by the kernels of the paged key/value cache.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "common.h"

namespace mptkv {

// MPT_OK, or fails with the reason the descriptor cannot be used.
int check_cache(const mpt_kv_cache *c);

// Caches in 4 bits: their 16-bit type, and the bytes E of their rows.
inline __host__ __device__ bool is_mx4(const mpt_kv_cache &c) { return c.dtype >= MPT_KV_BF16_MX4; }
inline __host__ __device__ int value_type(const mpt_kv_cache &c) { return is_mx4(c) ? c.dtype - MPT_KV_BF16_MX4 : c.dtype; }

struct Scales {
    char *k, *v;
    int64_t k_stride[4], v_stride[4];     // bytes
    int bytes;                            // of a row; 0: the cache has 16 bits
};
inline Scales scales_of(const mpt_kv_cache &c) {
    Scales e = {};
    if (!is_mx4(c)) return e;
    const mpt_kv_cache_mx4 &x = reinterpret_cast<const mpt_kv_cache_mx4 &>(c);   // c is its first member
    e.k = (char *)x.k_scale, e.v = (char *)x.v_scale, e.bytes = c.head_dim / 32;
    for (int i = 0; i < 4; ++i) e.k_stride[i] = x.k_scale_stride[i], e.v_stride[i] = x.v_scale_stride[i];
    return e;
}

inline bool aligned16(const void *p) { return ((uintptr_t)p & 15) == 0; }

inline __device__ void flag(const mpt_kv_cache &c, uint32_t bits) { atomicOr(c.status, bits); }

// rows.hip: the checks of layer and sizes that appends and reads share, and an
// append into a cache of 4 bits.
int check_append(const mpt_kv_cache *c, int layer, int n, int64_t n_tokens);
int append_mx4(const mpt_kv_cache *c, int layer, int n, const int32_t *seqs, const int32_t *q_off, int64_t n_tokens,
               const void *k, int64_t kt, int64_t kh, const void *v, int64_t vt, int64_t vh, hipStream_t s);

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

inline __device__ bool slot_ok(const mpt_kv_cache &c, int s) { return s >= 0 && s < c.max_seqs; }
inline __device__ bool page_ok(const mpt_kv_cache &c, int p) { return p >= 0 && p < c.n_pages; }

// Index of the last entry of off[0 .. n] that is <= x (off ascends), found by
// the 64 lanes of a wave together, 64 places a step.
inline __device__ int wave_find(const int32_t *off, int n, int x) {
    const int lane = threadIdx.x & 63;
    int lo = 0, len = n + 1;
    while (len > 1) {
        const int step = (len + 63) / 64, at = lo + lane * step;
        const uint64_t le = __ballot(lane * step < len && off[at] <= x);
        if (!le) return -1;
        const int k = 63 - __clzll(le);
        lo += k * step;
        len = min(step, len - k * step);
    }
    return off[lo] <= x ? lo : -1;
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
