// Rows on their way into the paged key/value cache and out of it: appends with
// the rotation of keys and queries to their positions, rows in 4 bits, and
// tokens read back.
//
// A wave takes a token, or a part of one where there are few: pieces of 8
// elements, 64 at a time, of its keys, its values and its queries. The angles of
// a token are formed once per wave, in 64 bits (an angle of position 10^6 in 32
// bits would be off by 0.06), and handed out through LDS.

#include "kv.h"

#include <cmath>
#include <type_traits>

namespace mptkv {

using mptlib::fail;

struct Append {
    mpt_kv_cache c;
    Scales e;
    int layer, n, n_tokens, heads, parts;            // parts: waves of a token
    const int32_t *seqs, *q_off, *position;
    const char *k, *v, *q;
    char *q_out;
    int64_t k_token, k_head, v_token, v_head, q_token, q_head, out_token, out_head;
    const float *freq;
    float factor;
    int pairs, dim, e_min, e_max;                    // rotated pairs of a row; head_dim
    uint32_t turn_mul, copy_mul;                     // of divisions by a row's units
};

struct Turn64 { double c, s; };
struct Turn32 { float c, s; };

template <class T>
__device__ inline void widen(uint4 x, float *y) {
    union { uint4 u; T t[8]; } v;
    v.u = x;
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = (float)v.t[i];
}
template <class T>
__device__ inline uint4 narrow(const float *y) {
    union { uint4 u; T t[8]; } v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v.t[i] = (T)y[i];
    return v.u;
}

// x / units by a product: mul = ceil(2^32 / units), x below 2^21, units up to 32.
__device__ inline int divided(int x, uint32_t mul) { return mul ? (int)__umulhi((uint32_t)x, mul) : x; }

// Units of a row that is rotated in 16 bits: with pairs apart a unit is the two
// pieces of eight pairs, so that who reads a pair writes it (rows may be rotated
// in place), and then come the pieces that stay as they are.
template <bool NEIGHBOURS>
__host__ __device__ inline int turn_units(int dim, int pairs) {
    return NEIGHBOURS ? dim / 8 : pairs / 8 + (dim - 2 * pairs) / 8;
}

// One unit of a row of queries or of 16-bit keys.
template <class T, bool NEIGHBOURS>
__device__ inline void turn_row(const Append &a, const char *in, char *out, int u, const Turn32 *turns) {
    if (NEIGHBOURS ? 4 * u < a.pairs : 8 * u < a.pairs) {
        float x[8], y[8];
        if (NEIGHBOURS) {
            widen<T>(*(const uint4 *)(in + 16 * u), x);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const Turn32 t = turns[4 * u + i];
                y[2 * i] = x[2 * i] * t.c - x[2 * i + 1] * t.s;
                y[2 * i + 1] = x[2 * i + 1] * t.c + x[2 * i] * t.s;
            }
            *(uint4 *)(out + 16 * u) = narrow<T>(y);
        } else {
            float z[8], w[8];
            widen<T>(*(const uint4 *)(in + 16 * u), x);
            widen<T>(*(const uint4 *)(in + 2 * a.pairs + 16 * u), z);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const Turn32 t = turns[8 * u + i];
                y[i] = x[i] * t.c - z[i] * t.s;
                w[i] = z[i] * t.c + x[i] * t.s;
            }
            *(uint4 *)(out + 16 * u) = narrow<T>(y);
            *(uint4 *)(out + 2 * a.pairs + 16 * u) = narrow<T>(w);
        }
    } else {
        const int at = NEIGHBOURS ? 16 * u : 4 * a.pairs + 16 * (u - a.pairs / 8);
        *(uint4 *)(out + at) = *(const uint4 *)(in + at);
    }
}

// y rounded to 24 bits so that a later rounding to fewer gives what y itself
// would: what is cut off leaves the last bit set.
__device__ inline float to_odd(double y) {
    const uint64_t b = __builtin_bit_cast(uint64_t, y);
    const uint32_t lo = (uint32_t)b, cut = (lo & 0x1fffffffu) + 0x1fffffffu;    // bit 29: something is cut off
    const uint32_t kept = (lo | (cut & 0x20000000u)) & 0xe0000000u;
    return (float)__builtin_bit_cast(double, (b & 0xffffffff00000000ull) | kept);
}

__device__ inline uint32_t umax(uint32_t x, uint32_t y) { return x > y ? x : y; }

// Eight elements of a row in 4 bits, with those of the three lanes beside it that
// have the rest of their 32: the codes, and the byte E that belongs to them.
__device__ inline uint32_t to_codes(const float *y, int e_min, int e_max, int &scale) {
    uint32_t top = 0;                                // by their bits: a NaN is above all numbers
#pragma unroll
    for (int i = 0; i < 8; ++i) top = umax(top, __builtin_bit_cast(uint32_t, y[i]) & 0x7fffffffu);
    top = umax(top, (uint32_t)__builtin_amdgcn_mov_dpp((int)top, 0xb1, 0xf, 0xf, true));    // lanes 1 0 3 2
    top = umax(top, (uint32_t)__builtin_amdgcn_mov_dpp((int)top, 0x4e, 0xf, 0xf, true));    // lanes 2 3 0 1
    // max <= 7 2^e: 7 = 1.75 2^2
    int e = (int)(top >> 23) - 127 - 2 + ((top & 0x7fffffu) > 0x600000u);
    e = min(max(e, e_min), e_max);
    const float unit = __builtin_bit_cast(float, (uint32_t)(e + 127) << 23);
    uint32_t codes = 0;
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, y[0], y[1], unit, 0);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, y[2], y[3], unit, 1);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, y[4], y[5], unit, 2);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, y[6], y[7], unit, 3);
    const bool odd = top >= 0x7f800000u;
    scale = odd ? 255 : e + 127;
    return odd ? 0 : codes;
}

// One piece of a row of keys in 64 bits, rotated, as the sums' 24 odd bits.
template <class T, bool NEIGHBOURS>
__device__ inline void turn_piece(const Append &a, const char *in, int u, const Turn64 *turns, float *y) {
    float x[8];
    widen<T>(*(const uint4 *)(in + 16 * u), x);
    if (4 * u >= a.pairs) {
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = x[i];
    } else if (NEIGHBOURS) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const Turn64 t = turns[4 * u + i];
            const double p = x[2 * i], r = x[2 * i + 1];
            y[2 * i] = to_odd(p * t.c - r * t.s);
            y[2 * i + 1] = to_odd(r * t.c + p * t.s);
        }
    } else {
        float z[8];
        const bool upper = 8 * u >= a.pairs;
        const int first = 8 * u - (upper ? a.pairs : 0);
        widen<T>(*(const uint4 *)(in + 16 * u + (upper ? -2 : 2) * a.pairs), z);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const Turn64 t = turns[first + i];
            y[i] = to_odd((double)x[i] * t.c + (double)z[i] * (upper ? t.s : -t.s));
        }
    }
}

template <class T, bool FOUR, bool NEIGHBOURS>
__global__ __launch_bounds__(256) void k_kv_append_rotated(Append a) {
    __shared__ Turn32 turns32[4][MPT_KV_MAX_DIM / 2];
    __shared__ Turn64 turns64[FOUR ? 4 : 1][FOUR ? MPT_KV_MAX_DIM / 2 : 1];
    const mpt_kv_cache &c = a.c;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int shift = 31 - __clz(c.page_size), units = turn_units<NEIGHBOURS>(a.dim, a.pairs);
    const int pieces = c.n_heads * (a.dim / 8);
    const int k_all = a.k ? FOUR ? pieces : c.n_heads * units : 0, q_all = a.q ? a.heads * units : 0;
    const int kc = (k_all + 63) / 64, vc = a.k ? (pieces + 63) / 64 : 0, qc = (q_all + 63) / 64;
    Turn32 *t32 = turns32[wave];
    Turn64 *t64 = turns64[FOUR ? wave : 0];
    const int64_t all = (int64_t)a.n_tokens * a.parts;
    for (int64_t at = blockIdx.x * 4 + wave; at < all; at += gridDim.x * 4) {
        const int token = uniform((int)(a.parts == 1 ? at : at / a.parts)), part = uniform((int)(at - (int64_t)token * a.parts));
        // where the token stands and goes
        int slot = -1, length = 0;
        int64_t pos = 0;
        const int i = a.n > 0 ? uniform(wave_find(a.q_off, a.n, token)) : -1;
        bool known = false, write = false;
        if (i >= 0 && i < a.n && slot_ok(c, a.seqs[i])) {
            slot = a.seqs[i], length = c.length[slot];
            pos = (int64_t)length - a.q_off[i + 1] + token;
            known = true;
            if (pos < 0 || pos >= length || (pos >> shift) >= c.max_pages) {
                if (a.k && lane == 0 && part == 0) flag(c, MPT_KV_BAD_LENGTH);
            } else {
                write = a.k != nullptr;
            }
        } else if (lane == 0 && part == 0 && (a.k || !a.position)) {
            flag(c, MPT_KV_BAD_SLOT);
        }
        int page = 0;
        if (write) {
            page = c.table[(int64_t)slot * c.max_pages + (pos >> shift)];
            if (!page_ok(c, page) || c.ref[page] != 1) {
                if (lane == 0 && part == 0) flag(c, page_ok(c, page) && c.ref[page] > 1 ? MPT_KV_SHARED : MPT_KV_BAD_PAGE);
                write = false;
            }
        }
        const int64_t in_page = pos & (c.page_size - 1);
        if (a.position) pos = a.position[token], known = true;
        if (a.pairs && known) {
            __builtin_amdgcn_wave_barrier();                 // the last token's are read
            for (int p = lane; p < a.pairs; p += 64) {
                double s, co;
                sincos((double)pos * (double)a.freq[p], &s, &co);
                co *= a.factor, s *= a.factor;
                if (FOUR) t64[p] = Turn64{co, s};
                t32[p] = Turn32{(float)co, (float)s};
            }
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        }
        for (int j = part; j < kc + vc + qc; j += a.parts) {
            if (j >= kc + vc) {
                const int x = (j - kc - vc) * 64 + lane, h = divided(x, a.turn_mul);
                if (known && x < q_all)
                    turn_row<T, NEIGHBOURS>(a, a.q + 2 * (token * a.q_token + h * a.q_head),
                                            a.q_out + 2 * (token * a.out_token + h * a.out_head), x - h * units, t32);
                continue;
            }
            if (!write) continue;
            if constexpr (FOUR) {
                const bool keys = j < kc;
                const int x = (keys ? j : j - kc) * 64 + lane, h = divided(x, a.copy_mul), u = x - h * (a.dim / 8);
                float y[8] = {};
                if (x < pieces) {
                    if (keys)
                        turn_piece<T, NEIGHBOURS>(a, a.k + 2 * (token * a.k_token + h * a.k_head), u, t64, y);
                    else
                        widen<T>(*(const uint4 *)(a.v + 2 * (token * a.v_token + h * a.v_head) + 16 * u), y);
                }
                int scale;
                const uint32_t codes = to_codes(y, a.e_min, a.e_max, scale);
                if (x < pieces) {
                    const int64_t *st = keys ? c.k_stride : c.v_stride, *es = keys ? a.e.k_stride : a.e.v_stride;
                    char *to = (char *)(keys ? c.k : c.v) + a.layer * st[0] + page * st[1] + in_page * st[2] + h * st[3];
                    char *e = (keys ? a.e.k : a.e.v) + a.layer * es[0] + page * es[1] + in_page * es[2] + h * es[3];
                    *(uint32_t *)(to + 4 * u) = codes;
                    if (u % 4 == 0) e[u / 4] = (char)scale;
                }
            } else if (j < kc) {
                const int x = j * 64 + lane, h = divided(x, a.turn_mul);
                if (x < k_all)
                    turn_row<T, NEIGHBOURS>(a, a.k + 2 * (token * a.k_token + h * a.k_head),
                                            (char *)c.k + 2 * (a.layer * c.k_stride[0] + page * c.k_stride[1] +
                                                               in_page * c.k_stride[2] + h * c.k_stride[3]),
                                            x - h * units, t32);
            } else {
                const int x = (j - kc) * 64 + lane, h = divided(x, a.copy_mul), u = x - h * (a.dim / 8);
                if (x < pieces)
                    *(uint4 *)((char *)c.v + 2 * (a.layer * c.v_stride[0] + page * c.v_stride[1] + in_page * c.v_stride[2] +
                                                  h * c.v_stride[3]) + 16 * u) =
                        *(const uint4 *)(a.v + 2 * (token * a.v_token + h * a.v_head) + 16 * u);
            }
        }
    }
}

struct Read {
    mpt_kv_cache c;
    Scales e;
    int layer, n, n_tokens, dim;
    const int32_t *seqs, *off, *first;
    char *k, *v;
    int64_t k_token, k_head, v_token, v_head;
    uint32_t copy_mul;
};

// Eight elements in 4 bits as those of the 16-bit type.
template <class T>
__device__ inline uint4 from_codes(uint32_t codes, uint32_t scale) {
    const float unit = __builtin_bit_cast(float, scale << 23);
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    typedef _Float16 h2 __attribute__((ext_vector_type(2)));
    auto two = [&](auto which) -> uint32_t {
        if constexpr (__is_same(T, __bf16))
            return __builtin_bit_cast(uint32_t, (b2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, which));
        else
            return __builtin_bit_cast(uint32_t, (h2)__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, unit, which));
    };
    const uint32_t nan = __is_same(T, __bf16) ? 0x7fc07fc0u : 0x7e007e00u;
    if (scale == 255) return uint4{nan, nan, nan, nan};
    return uint4{two(std::integral_constant<int, 0>()), two(std::integral_constant<int, 1>()),
                 two(std::integral_constant<int, 2>()), two(std::integral_constant<int, 3>())};
}

// One wave per token, a piece of 8 elements per lane.
template <class T, bool FOUR>
__global__ __launch_bounds__(256) void k_kv_read(Read a) {
    const mpt_kv_cache &c = a.c;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, shift = 31 - __clz(c.page_size);
    const int units = a.dim / 8, pieces = c.n_heads * units;
    for (int64_t at = blockIdx.x * 4 + wave; at < a.n_tokens; at += gridDim.x * 4) {
        const int token = uniform((int)at), i = uniform(wave_find(a.off, a.n, token));
        if (i < 0 || i >= a.n) {
            if (lane == 0) flag(c, MPT_KV_BAD_SLOT);
            continue;
        }
        int page = -1;
        int64_t pos = 0;
        uint32_t bad = 0;
        if (slot_ok(c, a.seqs[i])) {
            const int slot = a.seqs[i], length = c.length[slot];
            pos = a.first ? (int64_t)a.first[i] + token - a.off[i] : (int64_t)length - a.off[i + 1] + token;
            if (pos < 0 || pos >= length || (pos >> shift) >= c.max_pages) {
                bad = MPT_KV_BAD_LENGTH;
            } else {
                page = c.table[(int64_t)slot * c.max_pages + (pos >> shift)];
                if (!page_ok(c, page)) page = -1, bad = MPT_KV_BAD_PAGE;
            }
        } else {
            bad = MPT_KV_BAD_SLOT;
        }
        if (bad && lane == 0) flag(c, bad);
        const int64_t in_page = pos & (c.page_size - 1);
        for (int x = lane; x < pieces; x += 64) {
            const int h = divided(x, a.copy_mul), u = x - h * units;
            auto one = [&](const void *base, const int64_t *st, const char *e, const int64_t *es) -> uint4 {
                if (page < 0) return uint4{0, 0, 0, 0};
                const int64_t row = a.layer * st[0] + page * st[1] + in_page * st[2] + h * st[3];
                if constexpr (FOUR) {
                    const uint8_t scale = *(const uint8_t *)(e + a.layer * es[0] + page * es[1] + in_page * es[2] + h * es[3] + u / 4);
                    return from_codes<T>(*(const uint32_t *)((const char *)base + row + 4 * u), scale);
                }
                return *(const uint4 *)((const char *)base + 2 * row + 16 * u);
            };
            uint4 k, v;
            if (a.k) k = one(c.k, c.k_stride, a.e.k, a.e.k_stride);
            if (a.v) v = one(c.v, c.v_stride, a.e.v, a.e.v_stride);
            if (a.k) *(uint4 *)(a.k + 2 * (token * a.k_token + h * a.k_head) + 16 * u) = k;
            if (a.v) *(uint4 *)(a.v + 2 * (token * a.v_token + h * a.v_head) + 16 * u) = v;
        }
    }
}

// --- host side ------------------------------------------------------------

static uint32_t reciprocal(int units) { return units == 1 ? 0 : (uint32_t)((((uint64_t)1 << 32) + units - 1) / units); }

static void launch_append(Append &a, bool neighbours, hipStream_t s) {
    const mpt_kv_cache &c = a.c;
    a.dim = c.head_dim;
    a.copy_mul = reciprocal(a.dim / 8);
    a.turn_mul = reciprocal(neighbours ? turn_units<true>(a.dim, a.pairs) : turn_units<false>(a.dim, a.pairs));
    const bool bf16 = value_type(c) == MPT_KV_BF16;
    a.e_min = bf16 ? -125 : -23, a.e_max = bf16 ? 125 : 13;
    a.parts = 1;
    using Kernel = void (*)(Append);
    static constexpr Kernel kernels[2][2][2] = {
        {{k_kv_append_rotated<__bf16, false, false>, k_kv_append_rotated<__bf16, false, true>},
         {k_kv_append_rotated<__bf16, true, false>, k_kv_append_rotated<__bf16, true, true>}},
        {{k_kv_append_rotated<_Float16, false, false>, k_kv_append_rotated<_Float16, false, true>},
         {k_kv_append_rotated<_Float16, true, false>, k_kv_append_rotated<_Float16, true, true>}}};
    mptlib::LaunchScope scope("k_kv_append_rotated", (double)a.n_tokens, s);
    kernels[bf16 ? 0 : 1][is_mx4(c)][neighbours]<<<mptlib::grid_for((int64_t)a.n_tokens * a.parts, 4, 4096), 256, 0, s>>>(a);
}

int check_append(const mpt_kv_cache *c, int layer, int n, int64_t n_tokens) {
    if (layer < 0 || layer >= c->n_layers) return fail(MPT_E_INVALID, "layer = %d", layer);
    if (n < 0 || n_tokens < 0 || n_tokens > INT32_MAX)
        return fail(MPT_E_INVALID, "n = %d, n_tokens = %lld", n, (long long)n_tokens);
    return MPT_OK;
}

// An append into a cache of 4 bits, arguments checked.
int append_mx4(const mpt_kv_cache *c, int layer, int n, const int32_t *seqs, const int32_t *q_off, int64_t n_tokens,
               const void *k, int64_t kt, int64_t kh, const void *v, int64_t vt, int64_t vh, hipStream_t s) {
    Append a = {};
    a.c = *c, a.e = scales_of(*c), a.layer = layer, a.n = n, a.n_tokens = (int)n_tokens;
    a.seqs = seqs, a.q_off = q_off, a.k = (const char *)k, a.v = (const char *)v;
    a.k_token = kt, a.k_head = kh, a.v_token = vt, a.v_head = vh;
    launch_append(a, false, s);
    MPT_HIP_TRY(hipGetLastError());
    return MPT_OK;
}

}  // namespace mptkv

using namespace mptkv;

extern "C" int mpt_kv_append_rotated(const mpt_kv_cache *cache, int layer, int n, const int32_t *seqs, const int32_t *q_off,
                                     int64_t n_tokens, const void *k_new, int64_t k_token_stride, int64_t k_head_stride,
                                     const void *v_new, int64_t v_token_stride, int64_t v_head_stride,
                                     const mpt_kv_rotation *rotation, int n_q_heads, const void *q, int64_t q_token_stride,
                                     int64_t q_head_stride, void *q_out, int64_t out_token_stride, int64_t out_head_stride,
                                     void *stream) {
    mptlib::clear_error();
    return mptlib::guarded(__func__, [&]() -> int {
        if (int rc = check_cache(cache)) return rc;
        if (int rc = check_append(cache, layer, n, n_tokens)) return rc;
        const mpt_kv_rotation *r = rotation;
        if (!r) return fail(MPT_E_INVALID, "rotation is NULL");
        if (r->dim < 16 || r->dim % 16 || r->dim > cache->head_dim)
            return fail(MPT_E_INVALID, "rotation: dim = %d is no multiple of 16 up to %d", r->dim, cache->head_dim);
        if (!std::isfinite(r->factor)) return fail(MPT_E_INVALID, "rotation: factor = %g", r->factor);
        if ((k_new == nullptr) != (v_new == nullptr)) return fail(MPT_E_INVALID, "k_new without v_new, or v_new without k_new");
        if ((q == nullptr) != (q_out == nullptr)) return fail(MPT_E_INVALID, "q without q_out, or q_out without q");
        if (q && (n_q_heads < 1 || n_q_heads > 65535)) return fail(MPT_E_INVALID, "n_q_heads = %d", n_q_heads);
        if (n_tokens == 0 || (!k_new && !q) || (n == 0 && !(q && r->position))) return MPT_OK;
        if (!r->freq || (n > 0 && (!seqs || !q_off))) return fail(MPT_E_INVALID, "an array is NULL");
        for (const void *p : {k_new, v_new, q, (const void *)q_out})
            if (!aligned16(p)) return fail(MPT_E_INVALID, "k_new, v_new, q and q_out must be 16-byte aligned");
        if ((k_token_stride | k_head_stride | v_token_stride | v_head_stride | q_token_stride | q_head_stride | out_token_stride |
             out_head_stride) % 8)
            return fail(MPT_E_INVALID, "strides must be multiples of 8");
        if (q && q == q_out && (q_token_stride != out_token_stride || q_head_stride != out_head_stride))
            return fail(MPT_E_INVALID, "q_out is q with other strides");
        Append a = {};
        a.c = *cache, a.e = scales_of(*cache), a.layer = layer, a.n = n, a.n_tokens = (int)n_tokens, a.heads = n_q_heads;
        a.seqs = seqs, a.q_off = q_off, a.position = r->position, a.freq = r->freq, a.factor = r->factor, a.pairs = r->dim / 2;
        a.k = (const char *)k_new, a.v = (const char *)v_new, a.q = (const char *)q, a.q_out = (char *)q_out;
        if (n == 0) a.k = a.v = nullptr;                 // no entry has the tokens
        a.k_token = k_token_stride, a.k_head = k_head_stride, a.v_token = v_token_stride, a.v_head = v_head_stride;
        a.q_token = q_token_stride, a.q_head = q_head_stride, a.out_token = out_token_stride, a.out_head = out_head_stride;
        launch_append(a, r->interleaved != 0, (hipStream_t)stream);
        MPT_HIP_TRY(hipGetLastError());
        return MPT_OK;
    });
}

extern "C" int mpt_kv_read(const mpt_kv_cache *cache, int layer, int n, const int32_t *seqs, const int32_t *off,
                           const int32_t *first, int64_t n_tokens, void *k_out, int64_t k_token_stride, int64_t k_head_stride,
                           void *v_out, int64_t v_token_stride, int64_t v_head_stride, void *stream) {
    mptlib::clear_error();
    return mptlib::guarded(__func__, [&]() -> int {
        if (int rc = check_cache(cache)) return rc;
        if (int rc = check_append(cache, layer, n, n_tokens)) return rc;
        if (n == 0 || n_tokens == 0 || (!k_out && !v_out)) return MPT_OK;
        if (!seqs || !off) return fail(MPT_E_INVALID, "an array is NULL");
        if (!aligned16(k_out) || !aligned16(v_out)) return fail(MPT_E_INVALID, "k_out and v_out must be 16-byte aligned");
        if ((k_token_stride | k_head_stride | v_token_stride | v_head_stride) % 8)
            return fail(MPT_E_INVALID, "strides must be multiples of 8");
        Read a = {};
        a.c = *cache, a.e = scales_of(*cache), a.layer = layer, a.n = n, a.n_tokens = (int)n_tokens, a.dim = cache->head_dim;
        a.seqs = seqs, a.off = off, a.first = first, a.k = (char *)k_out, a.v = (char *)v_out;
        a.k_token = k_token_stride, a.k_head = k_head_stride, a.v_token = v_token_stride, a.v_head = v_head_stride;
        a.copy_mul = reciprocal(a.dim / 8);
        using Kernel = void (*)(Read);
        static constexpr Kernel kernels[2][2] = {{k_kv_read<__bf16, false>, k_kv_read<__bf16, true>},
                                                 {k_kv_read<_Float16, false>, k_kv_read<_Float16, true>}};
        hipStream_t s = (hipStream_t)stream;
        {
            mptlib::LaunchScope scope("k_kv_read", (double)n_tokens, s);
            kernels[value_type(*cache)][is_mx4(*cache)]<<<mptlib::grid_for(n_tokens, 4, 4096), 256, 0, s>>>(a);
        }
        MPT_HIP_TRY(hipGetLastError());
        return MPT_OK;
    });
}
