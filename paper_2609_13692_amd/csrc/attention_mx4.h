// Shared by the attention kernels over caches in 4 bits: where the bytes E of a
// row lie, codes turned into operands, and values that are NaN.
#pragma once

#include "attention.h"

namespace mptkv {

// Strides of pages and slots are in bytes here, those of Attn too.
struct Attn4 : Attn {
    const char *ke, *ve;                              // the layer's bytes E
    int64_t ke_head, ve_head;
    uint32_t ke_page, ke_slot, ve_page, ve_slot;
};

// x at index i of so many bytes: one instruction.
inline __device__ const char *at(const char *x, uint32_t i, uint32_t bytes) { return x + (uint64_t)i * bytes; }

template <class V>
__device__ inline void to_lds(uint32_t at, V x) {
    *(__attribute__((address_space(3))) V *)(uintptr_t)at = x;
}

// The largest E that appends write; all above count as 255, which is NaN.
template <class T>
constexpr uint32_t kMaxScale = __is_same(T, __bf16) ? 127 + 125 : 127 + 13;

// What a byte E multiplies codes by, as the conversions take it: the exponent
// of a 32-bit number.
inline __device__ float unit_of(uint32_t scale) { return __builtin_bit_cast(float, scale << 23); }

// Eight codes as eight elements of the 16-bit type, exactly.
template <class T>
__device__ inline s16x8 from_codes(uint32_t codes, float unit) {
    typedef T t2 __attribute__((ext_vector_type(2)));
    u32x4 x;
    if constexpr (__is_same(T, __bf16)) {
        x[0] = __builtin_bit_cast(uint32_t, (t2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 0));
        x[1] = __builtin_bit_cast(uint32_t, (t2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 1));
        x[2] = __builtin_bit_cast(uint32_t, (t2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 2));
        x[3] = __builtin_bit_cast(uint32_t, (t2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 3));
    } else {
        x[0] = __builtin_bit_cast(uint32_t, (t2)__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, unit, 0));
        x[1] = __builtin_bit_cast(uint32_t, (t2)__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, unit, 1));
        x[2] = __builtin_bit_cast(uint32_t, (t2)__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, unit, 2));
        x[3] = __builtin_bit_cast(uint32_t, (t2)__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, unit, 3));
    }
    return __builtin_bit_cast(s16x8, x);
}

template <class T>
__device__ inline s16x8 nans() {
    constexpr short n = Type<T>::kExponent | 0x200 >> (__is_same(T, __bf16) ? 3 : 0);
    return s16x8{n, n, n, n, n, n, n, n};
}

// NaN in values (there are no infinities). Products take
// zeros in their place, for under the weight 0 of a row that does not see the
// token they would spread, and a tile that has met one ends here: the E of the
// values of tokens t0 .. t1 - 1 are looked through once more, and the sums of the
// rows that see such a block become NaN. Arguments as those of odd_values;
// scales: the head's bytes E of the values.
template <class T>
__device__ inline void nan_values(const Attn4 &a, const int32_t *table, int shift, const char *scales, int t0, int t1, int lo,
                                  int hi, float l, bool whole, int d0, int step, char *to, int inc, bool f32) {
    const int lane = threadIdx.x & 63, dim = 8 * a.units, blocks = dim / 32;
    uint32_t mine = 0;
#pragma unroll 1
    for (int base = t0; base < t1; base += 64) {
        const int t = base + lane, page = t < t1 ? table[t >> shift] : -1;
        uint32_t odd = 0;
        if ((unsigned)page < (unsigned)a.c.n_pages) {
            const uint8_t *e = (const uint8_t *)at(at(scales, page, a.ve_page), t & (a.c.page_size - 1), a.ve_slot);
            for (int b = 0; b < blocks; ++b) odd |= (uint32_t)(e[b] > kMaxScale<T>) << b;
        }
#pragma unroll 1
        for (uint64_t todo = __ballot(odd != 0); todo; todo &= todo - 1) {
            const int at = __ffsll((unsigned long long)todo) - 1;
            const uint32_t which = __builtin_amdgcn_readlane((int)odd, at);
            if (base + at >= lo && base + at < hi) mine |= which;
        }
    }
    if (!(l > 0 || (l == 0 && !whole))) return;
#pragma unroll 1
    for (int k = 0; d0 + k * step < dim; ++k) {
        if (!(mine >> (d0 + k * step) / 32 & 1)) continue;
        if (f32)
            *(f32x4 *)(to + k * inc) = f32x4{NAN, NAN, NAN, NAN};
        else
            *(s16x4 *)(to + k * inc) = __builtin_shufflevector(nans<T>(), nans<T>(), 0, 1, 2, 3);
    }
}

void launch_wide_mx4(const Attn4 &a, int waves, hipStream_t s);
void launch_narrow_mx4(const Attn4 &a, hipStream_t s);

}  // namespace mptkv
