// Rows on their way into the paged key/value cache and out of it: appends with
// the rotation of keys and queries to their positions, rows in 4 bits, and
// tokens read back.
//
// A wave takes a run of tokens, whose places its lanes find together, or a part of
// one token where there are few. It forms their angles, in 64 bits (an angle of
// position 10^6 in 32 bits would be off by 0.06), of several tokens at a time where
// 64 lanes do, and hands them out through LDS;
// its keys, values and queries go 64 units of 8 or 16 elements at a time.
//
// What bounds them is memory, where there is something to move: 25 chunks of 60 to
// 600 tokens (32 heads and 8 key heads of 128), rotated into 16 bits with their
// queries, 43 to 47 us (203 MB, 4.3 to 4.7 TB/s; a large copy reaches 5.0), 25 of 60 to
// 1201 into 4 bits 76, 261 MB of codes read out as 983 MB 239 (5.2 TB/s). Few tokens
// are a launch. Angles formed once for the waves of a workgroup instead of once for a
// wave's token took 55 to 120 us of the first, workgroups for keys, values and queries
// apart as long. Of few heads it is a chain of reads a token: 64000 tokens of 4 query
// heads and 2 key heads of 64, 63 us (2.1 TB/s).

#include "kv.h"

#include <cmath>
#include <type_traits>

namespace mptkv {

using mptlib::fail;

struct Append {
    mpt_kv_cache c;
    Scales e;
    int layer, n, n_tokens, heads, run, parts_log;   // run: tokens of a wave; 2^parts_log waves share them
    const int32_t *seqs, *q_off, *position;
    const char *k, *v, *q;
    char *q_out;
    int64_t k_token, k_head, v_token, v_head, q_token, q_head, out_token, out_head;
    const float *freq;
    float factor;
    int pairs, dim, e_min, e_max;                    // rotated pairs of a row; head_dim
    int batch;                                       // tokens of a wave whose angles are there at a time
    uint32_t turn_mul, copy_mul, pair_mul;           // of divisions by a row's units, and by its pairs
};

// Where a token goes: lane l knows it of the l-th of the wave's tokens.
struct Place {
    int page, slot;          // page -1: nowhere
    int pos;                 // place in its sequence
    bool known;              // it has one
    uint32_t bad;            // MPT_KV_* bits
};

// Places of tokens x0 + lane, lane < count, cut into entries by off. first: where an
// entry's tokens begin (NULL: they are the sequence's newest).
__device__ inline Place locate(const mpt_kv_cache &c, int n, const int32_t *seqs, const int32_t *off, const int32_t *first, int x0,
                               int count) {
    const int lane = threadIdx.x & 63, shift = 31 - __clz(c.page_size);
    Place p = {-1, 0, 0, false, 0};
    int i = n > 0 ? wave_find(off, n, x0) : -1;
    if (lane >= count) return p;
    const int x = x0 + lane;
    if (n > 0 && i < n && x >= off[i + 1]) {             // a later entry's than x0's (-1: before the first)
        int lo = i + 1, hi = n;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (off[mid] <= x)
                lo = mid;
            else
                hi = mid - 1;
        }
        i = lo;
    }
    p.bad = MPT_KV_BAD_SLOT;
    if (i < 0 || i >= n || !slot_ok(c, seqs[i])) return p;
    const int s = seqs[i];
    const int length = c.length[s];
    // in 64 bits: a length may be any number (a place below -2^31 counts as that)
    const int64_t pos = first ? (int64_t)first[i] + (x - off[i]) : (int64_t)length - off[i + 1] + x;
    p.pos = (int)max((int64_t)INT32_MIN, min(pos, (int64_t)INT32_MAX));
    p.known = true;
    p.bad = MPT_KV_BAD_LENGTH;
    if (pos < 0 || pos >= length || (pos >> shift) >= c.max_pages) return p;
    p.bad = MPT_KV_BAD_PAGE;
    const int page = c.table[(int64_t)s * c.max_pages + (p.pos >> shift)];
    if (!page_ok(c, page)) return p;
    p.page = page, p.slot = p.pos & (c.page_size - 1), p.bad = 0;
    return p;
}

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

// The wave's number in its launch, and a launch of so many waves, four to a
// workgroup: a dimension of it holds less than 2^32 threads.
__device__ inline int64_t wave_number() {
    return ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 4 + uniform((int)threadIdx.x >> 6);
}
static dim3 grid_of(int64_t waves) {
    constexpr int64_t kAcross = 1 << 23;
    const int64_t blocks = (waves + 3) / 4;
    return dim3((unsigned)(blocks < kAcross ? blocks : kAcross), (unsigned)((blocks + kAcross - 1) / kAcross));
}

// x / units by a product: mul = ceil(2^32 / units), x units below 2^32 (and so the
// product's error below one part in units).
__device__ inline int divided(int x, uint32_t mul) { return mul ? (int)__umulhi((uint32_t)x, mul) : x; }

// Units of a row that is rotated in 16 bits: with pairs apart a unit is the two
// pieces of eight pairs, so that who reads a pair writes it (rows may be rotated
// in place), and then come the pieces that stay as they are.
template <bool NEIGHBOURS>
__host__ __device__ inline int turn_units(int dim, int pairs) {
    return NEIGHBOURS ? dim / 8 : pairs / 8 + (dim - 2 * pairs) / 8;
}

// Where a unit's one or two pieces lie in a row of 16 bits, in bytes, and whether it
// is rotated.
template <bool NEIGHBOURS>
__device__ inline void unit_at(int pairs, int u, int &first, int &second, bool &turns) {
    turns = NEIGHBOURS ? 4 * u < pairs : 8 * u < pairs;
    first = NEIGHBOURS || turns ? 16 * u : 4 * pairs + 16 * (u - pairs / 8);
    second = NEIGHBOURS || !turns ? first : 16 * u + 2 * pairs;
}

// One unit of a row of queries or of 16-bit keys.
template <class T, bool NEIGHBOURS>
__device__ inline void turn_unit(int pairs, uint4 a, uint4 b, char *out, int u, const Turn32 *table) {
    int first, second;
    bool turns;
    unit_at<NEIGHBOURS>(pairs, u, first, second, turns);
    if (!turns) {
        *(uint4 *)(out + first) = a;
        return;
    }
    float x[8], y[8];
    widen<T>(a, x);
    if (NEIGHBOURS) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const Turn32 t = table[4 * u + i];
            y[2 * i] = x[2 * i] * t.c - x[2 * i + 1] * t.s;
            y[2 * i + 1] = x[2 * i + 1] * t.c + x[2 * i] * t.s;
        }
    } else {
        float z[8], w[8];
        widen<T>(b, z);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const Turn32 t = table[8 * u + i];
            y[i] = x[i] * t.c - z[i] * t.s;
            w[i] = z[i] * t.c + x[i] * t.s;
        }
        *(uint4 *)(out + second) = narrow<T>(w);
    }
    *(uint4 *)(out + first) = narrow<T>(y);
}

// y rounded to 23 bits so that a later rounding to fewer gives what y itself
// would: what is cut off leaves the last bit set. Of 24 bits the last would be lost
// in numbers of 32 bits below 2^-126, which are 2^-149 apart: between 2^-127, the
// smallest border of codes (half of 2^-126), and 2^-126 those have 23.
__device__ inline float to_odd(double y) {
    const uint64_t b = __builtin_bit_cast(uint64_t, y);
    const uint32_t lo = (uint32_t)b, cut = (lo & 0x3fffffffu) + 0x3fffffffu;    // bit 30: something is cut off
    const uint32_t kept = (lo | (cut & 0x40000000u)) & 0xc0000000u;
    return (float)__builtin_bit_cast(double, (b & 0xffffffff00000000ull) | kept);
}

__device__ inline uint32_t umax(uint32_t x, uint32_t y) { return x > y ? x : y; }

// 32 elements in 4 bits: the codes, and the byte E that belongs to them.
__device__ inline uint4 to_codes(const float *y, int e_min, int e_max, int &scale) {
    uint32_t top = 0;                                // by their bits: a NaN is above all numbers
#pragma unroll
    for (int i = 0; i < 32; ++i) top = umax(top, __builtin_bit_cast(uint32_t, y[i]) & 0x7fffffffu);
    // max <= 7 2^e: 7 = 1.75 2^2
    int e = (int)(top >> 23) - 127 - 2 + ((top & 0x7fffffu) > 0x600000u);
    e = min(max(e, e_min), e_max);
    const float unit = __builtin_bit_cast(float, (uint32_t)(e + 127) << 23);
    const bool odd = top >= 0x7f800000u;
    scale = odd ? 255 : e + 127;
    uint32_t codes[4];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const float *z = y + 8 * w;
        codes[w] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, z[0], z[1], unit, 0);
        codes[w] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes[w], z[2], z[3], unit, 1);
        codes[w] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes[w], z[4], z[5], unit, 2);
        codes[w] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes[w], z[6], z[7], unit, 3);
        if (odd) codes[w] = 0;
    }
    return uint4{codes[0], codes[1], codes[2], codes[3]};
}

// How keys are rotated: not at all, pairs of neighbours, pairs half the rotated
// elements apart.
enum Keys { kWhole, kNeighbours, kApart };

// The 32 elements from 32 b on of a row of keys, rotated in 64 bits and cut so that
// they round as they are.
template <class T, int KEYS>
__device__ inline void turn_block(int pairs, const char *row, int b, const Turn64 *table, float *y) {
#pragma unroll
    for (int w = 0; w < 4; ++w) widen<T>(*(const uint4 *)(row + 64 * b + 16 * w), y + 8 * w);
    if (KEYS == kWhole || 16 * b >= pairs) return;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const int u = 4 * b + w;
        float *x = y + 8 * w;
        if (4 * u >= pairs) continue;
        if (KEYS == kNeighbours) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const Turn64 t = table[4 * u + i];
                const double p = x[2 * i], r = x[2 * i + 1];
                x[2 * i] = to_odd(p * t.c - r * t.s);
                x[2 * i + 1] = to_odd(r * t.c + p * t.s);
            }
        } else {
            const bool upper = 8 * u >= pairs;
            const int first = 8 * u - (upper ? pairs : 0);
            float z[8];
            widen<T>(*(const uint4 *)(row + 16 * u + (upper ? -2 : 2) * pairs), z);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const Turn64 t = table[first + i];
                x[i] = to_odd((double)x[i] * t.c + (double)z[i] * (upper ? t.s : -t.s));
            }
        }
    }
}

enum Role { kKeys, kValues, kQueries };              // rows that a chunk of 64 units belongs to

// How the rows of a role are cut into units, in 16 bits.
template <class T, bool NEIGHBOURS, int ROLE>
struct Units {
    const Append &a;
    int pairs, units, all, chunks;
    uint32_t mul;

    __device__ explicit Units(const Append &a, bool any) : a(a) {
        pairs = ROLE == kValues ? 0 : a.pairs;
        units = ROLE == kValues ? a.dim / 8 : turn_units<NEIGHBOURS>(a.dim, a.pairs);
        mul = ROLE == kValues ? a.copy_mul : a.turn_mul;
        all = any ? (ROLE == kQueries ? a.heads : a.c.n_heads) * units : 0;
        chunks = (all + 63) / 64;
    }

    // The pieces of unit y: lanes past the last read that one.
    __device__ void load(int64_t token, int y, uint4 &one, uint4 &two) const {
        y = min(y, all - 1);
        const int h = divided(y, mul), u = y - h * units;
        int first, second;
        bool turns;
        unit_at<NEIGHBOURS>(pairs, u, first, second, turns);
        const char *row = ROLE == kKeys     ? a.k + 2 * (token * a.k_token + h * a.k_head)
                          : ROLE == kValues ? a.v + 2 * (token * a.v_token + h * a.v_head)
                                            : a.q + 2 * (token * a.q_token + h * a.q_head);
        one = *(const uint4 *)(row + first);
        if (ROLE != kValues && !NEIGHBOURS) two = *(const uint4 *)(row + second);
    }

    __device__ void put(int64_t token, int page, int slot, int y, uint4 one, uint4 two, const Turn32 *table) const {
        const mpt_kv_cache &c = a.c;
        const int h = divided(y, mul), u = y - h * units;
        if (y >= all) return;
        if (ROLE == kQueries) {
            turn_unit<T, NEIGHBOURS>(pairs, one, two, a.q_out + 2 * (token * a.out_token + h * a.out_head), u, table);
            return;
        }
        const int64_t *st = ROLE == kKeys ? c.k_stride : c.v_stride;
        char *to = (char *)(ROLE == kKeys ? c.k : c.v) + 2 * (a.layer * st[0] + page * st[1] + slot * st[2] + h * st[3]);
        if (ROLE == kKeys)
            turn_unit<T, NEIGHBOURS>(pairs, one, two, to, u, table);
        else
            *(uint4 *)(to + 16 * u) = one;
    }
};

constexpr int kRun4 = 4;                             // tokens of a wave, at most, in a cache of 4 bits

// In a cache of 4 bits a lane takes 32 elements of a row, of any of the wave's
// tokens: no two lanes need to agree on an E, and 16 bytes of codes go out at a time.
template <class T, bool FOUR, int KEYS>
__global__ __launch_bounds__(256, 4) void k_kv_append_rotated(Append a) {
    constexpr bool NEIGHBOURS = KEYS == kNeighbours;
    extern __shared__ char tables[];                 // of each wave
    const mpt_kv_cache &c = a.c;
    const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6);
    const Units<T, NEIGHBOURS, kKeys> keys(a, !FOUR && a.k);
    const Units<T, NEIGHBOURS, kValues> values(a, !FOUR && a.k);
    const Units<T, NEIGHBOURS, kQueries> queries(a, a.q);
    Turn32 *t32 = (Turn32 *)(tables + (FOUR ? 4 * a.batch * a.pairs * sizeof(Turn64) : 0)) + wave * a.batch * a.pairs;
    Turn64 *t64 = (Turn64 *)tables + wave * a.batch * a.pairs;
    const int64_t at = wave_number(), group = at >> a.parts_log;
    const int parts = 1 << a.parts_log, part = (int)at & (parts - 1);
    if (group * a.run >= a.n_tokens) return;
    const int x0 = (int)(group * a.run), count = min(a.run, a.n_tokens - x0);
    Place place = locate(c, a.n, a.seqs, a.q_off, nullptr, x0, count);
    if (a.k) {
        if (place.page >= 0 && c.ref[place.page] != 1) {
            place.bad = c.ref[place.page] > 1 ? MPT_KV_SHARED : MPT_KV_BAD_PAGE;
            place.page = -1;
        }
    } else {
        place.bad = a.position || place.known ? 0 : place.bad;      // nothing is written
    }
    if (part == 0 && place.bad) flag(c, place.bad);
    if (a.position && lane < count) place.pos = a.position[x0 + lane], place.known = true;
    // angles of tokens x .. x + n - 1, a pair a lane
    auto turn = [&](int x, int n) {
        for (int y0 = 0; y0 < n * a.pairs; y0 += 64) {
            const int y = min(y0 + lane, n * a.pairs - 1), z = divided(y, a.pair_mul), p = y - z * a.pairs;
            const double pos = __shfl(place.pos, x + z);
            double s, co;
            sincos(pos * (double)a.freq[p], &s, &co);
            co *= a.factor, s *= a.factor;
            if (FOUR) t64[y] = Turn64{co, s};
            t32[y] = Turn32{(float)co, (float)s};
        }
    };
    auto handed_out = [&]() {
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    };
    // all roles' chunks in turn over the parts
    int before = 0;
    auto first_of = [&](int chunks) {
        const int x = (part - before) & (parts - 1);
        before += chunks;
        return x;
    };
    if constexpr (FOUR) {
        turn(0, count);
        handed_out();
        const int blocks = a.dim / 32, units = c.n_heads * blocks, all = a.k ? count * units : 0, chunks = (all + 63) / 64;
        auto put = [&](auto role, int y) {
            constexpr bool KEY = decltype(role)::value == kKeys;
            const int x = (y >= units) + (y >= 2 * units) + (y >= 3 * units), z = y - x * units, h = divided(z, a.copy_mul), b = z - h * blocks;
            const int page = __shfl(place.page, x);
            const int64_t slot = __shfl(place.slot, x), token = x0 + x;
            if (y >= all || page < 0) return;
            const int64_t *st = KEY ? c.k_stride : c.v_stride, *es = KEY ? a.e.k_stride : a.e.v_stride;
            float f[32];
            if (KEY)
                turn_block<T, KEYS>(a.pairs, a.k + 2 * (token * a.k_token + h * a.k_head), b, t64 + x * a.pairs, f);
            else
                turn_block<T, kWhole>(0, a.v + 2 * (token * a.v_token + h * a.v_head), b, nullptr, f);
            int scale;
            const uint4 codes = to_codes(f, a.e_min, a.e_max, scale);
            *(uint4 *)((char *)(KEY ? c.k : c.v) + (a.layer * st[0] + page * st[1] + slot * st[2] + h * st[3]) + 16 * b) = codes;
            *(uint8_t *)((KEY ? a.e.k : a.e.v) + (a.layer * es[0] + page * es[1] + slot * es[2] + h * es[3]) + b) = (uint8_t)scale;
        };
        for (int j = first_of(chunks); j < chunks; j += parts) put(std::integral_constant<int, kKeys>(), j * 64 + lane);
        for (int j = first_of(chunks); j < chunks; j += parts) put(std::integral_constant<int, kValues>(), j * 64 + lane);
        const int q0 = first_of(0);
        for (int x = 0; x < count; ++x) {
            if (!__builtin_amdgcn_readlane(place.known, x)) continue;
            for (int j = q0; j < queries.chunks; j += 2 * parts) {
                uint4 one[2], two[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) queries.load(x0 + x, (j + i * parts) * 64 + lane, one[i], two[i]);
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    queries.put(x0 + x, 0, 0, (j + i * parts) * 64 + lane, one[i], two[i], t32 + x * a.pairs);
            }
        }
    } else {
        const int k0 = first_of(keys.chunks), v0 = first_of(values.chunks), q0 = first_of(0);
        for (int x = 0, first = 0; x < count; ++x) {         // first: of those whose angles are there
            const int64_t token = x0 + x;
            const int page = __builtin_amdgcn_readlane(place.page, x), slot = __builtin_amdgcn_readlane(place.slot, x);
            const bool known = __builtin_amdgcn_readlane(place.known, x);
            uint4 k1, k2, q1[2], q2[2], none;
            auto load_queries = [&](int j) {
#pragma unroll
                for (int i = 0; i < 2; ++i) queries.load(token, (j + i * parts) * 64 + lane, q1[i], q2[i]);
            };
            if (k0 < keys.chunks) keys.load(token, k0 * 64 + lane, k1, k2);
            if (q0 < queries.chunks) load_queries(q0);
            if (x == 0 || x == first + a.batch) {
                first = x;
                __builtin_amdgcn_wave_barrier();             // the last tokens' are read
                turn(x, min(a.batch, count - x));
                handed_out();
            }
            const Turn32 *turns = t32 + (x - first) * a.pairs;
            if (page >= 0) {
                for (int j = k0; j < keys.chunks;) {
                    keys.put(token, page, slot, j * 64 + lane, k1, k2, turns);
                    if ((j += parts) < keys.chunks) keys.load(token, j * 64 + lane, k1, k2);
                }
                for (int j = v0; j < values.chunks; j += 2 * parts) {
                    uint4 v[2];
#pragma unroll
                    for (int i = 0; i < 2; ++i) values.load(token, (j + i * parts) * 64 + lane, v[i], none);
#pragma unroll
                    for (int i = 0; i < 2; ++i) values.put(token, page, slot, (j + i * parts) * 64 + lane, v[i], none, turns);
                }
            }
            if (known)
                for (int j = q0; j < queries.chunks;) {
#pragma unroll
                    for (int i = 0; i < 2; ++i) queries.put(token, 0, 0, (j + i * parts) * 64 + lane, q1[i], q2[i], turns);
                    if ((j += 2 * parts) < queries.chunks) load_queries(j);
                }
        }
    }
}

struct Read {
    mpt_kv_cache c;
    Scales e;
    int layer, n, n_tokens, dim, run;
    const int32_t *seqs, *off, *first;
    char *k, *v;
    int64_t k_token, k_head, v_token, v_head;
    uint32_t copy_mul, row_mul;                      // of divisions by a row's pieces, and by a token's
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
    if (scale > (__is_same(T, __bf16) ? 127 + 125 : 127 + 13)) return uint4{nan, nan, nan, nan};
    return uint4{two(std::integral_constant<int, 0>()), two(std::integral_constant<int, 1>()),
                 two(std::integral_constant<int, 2>()), two(std::integral_constant<int, 3>())};
}

// A wave per run of tokens, a piece of 8 elements per lane: of one token, or (MANY)
// where a token has few pieces of as many tokens as there are lanes for. One head of 64,
// 237 thousand tokens in 4 bits: 58 us with the other lanes idle.
template <class T, bool FOUR, bool MANY>
__global__ __launch_bounds__(256) void k_kv_read(Read a) {
    const mpt_kv_cache &c = a.c;
    const int lane = threadIdx.x & 63;
    const int units = a.dim / 8, pieces = c.n_heads * units;
    const int64_t group = wave_number();
    if (group * a.run >= a.n_tokens) return;
    const int x0 = (int)(group * a.run), count = min(a.run, a.n_tokens - x0);
    const Place place = locate(c, a.n, a.seqs, a.off, a.first, x0, count);
    if (place.bad) flag(c, place.bad);
    // tokens of no entry keep their rows: off[n] on, or before off[0]
    const int begin = a.off[0], end = a.off[a.n];
    constexpr int U = 4;
    typedef uint32_t u4 __attribute__((ext_vector_type(4)));
    struct Got { uint4 k, v; uint32_t kc, vc, ks, vs; };
    // Piece u of head h of the token in a place, which is nowhere where page is negative.
    auto load = [&](Got &g, int page, int64_t slot, int h, int u) {
        g.k = g.v = uint4{0, 0, 0, 0};
        g.kc = g.vc = g.ks = g.vs = 0;
        if (page < 0) return;
        const int64_t k_row = a.layer * c.k_stride[0] + page * c.k_stride[1] + slot * c.k_stride[2];
        const int64_t v_row = a.layer * c.v_stride[0] + page * c.v_stride[1] + slot * c.v_stride[2];
        const int64_t k_in = h * c.k_stride[3], v_in = h * c.v_stride[3];
        if constexpr (FOUR) {
            const int64_t *ek = a.e.k_stride, *ev = a.e.v_stride;
            if (a.k) g.kc = *(const uint32_t *)((const char *)c.k + k_row + (k_in + 4 * u));
            if (a.k) g.ks = *(const uint8_t *)(a.e.k + (a.layer * ek[0] + page * ek[1] + slot * ek[2]) + (h * ek[3] + u / 4));
            if (a.v) g.vc = *(const uint32_t *)((const char *)c.v + v_row + (v_in + 4 * u));
            if (a.v) g.vs = *(const uint8_t *)(a.e.v + (a.layer * ev[0] + page * ev[1] + slot * ev[2]) + (h * ev[3] + u / 4));
        } else {
            if (a.k) g.k = *(const uint4 *)((const char *)c.k + 2 * k_row + (2 * k_in + 16 * u));
            if (a.v) g.v = *(const uint4 *)((const char *)c.v + 2 * v_row + (2 * v_in + 16 * u));
        }
    };
    auto store = [&](Got &g, int64_t token, int h, int u) {
        if (token < begin || token >= end) return;
        if (FOUR) g.k = from_codes<T>(g.kc, g.ks), g.v = from_codes<T>(g.vc, g.vs);
        // past the caches: 983 MB and 261 MB of codes 241 us, 253 through them
        if (a.k) __builtin_nontemporal_store(__builtin_bit_cast(u4, g.k), (u4 *)(a.k + 2 * token * a.k_token + (2 * h * a.k_head + 16 * u)));
        if (a.v) __builtin_nontemporal_store(__builtin_bit_cast(u4, g.v), (u4 *)(a.v + 2 * token * a.v_token + (2 * h * a.v_head + 16 * u)));
    };
    if constexpr (MANY) {
        const int all = count * pieces;
        for (int y0 = 0; y0 < all; y0 += 64 * U) {
            Got g[U];
            int x[U], h[U], u[U];
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const int y = min(y0 + 64 * i + lane, all - 1);
                x[i] = divided(y, a.row_mul);
                const int z = y - x[i] * pieces;
                h[i] = divided(z, a.copy_mul), u[i] = z - h[i] * units;
                load(g[i], __shfl(place.page, x[i]), __shfl(place.slot, x[i]), h[i], u[i]);
            }
#pragma unroll
            for (int i = 0; i < U; ++i)
                if (y0 + 64 * i + lane < all) store(g[i], x0 + x[i], h[i], u[i]);
        }
    } else {
        for (int z0 = 0; z0 < pieces; z0 += 64) {
            // lanes past the last piece read that one: all stay to the end, for any may be
            // asked for a token's place
            const int z = min(z0 + lane, pieces - 1), h = divided(z, a.copy_mul), u = z - h * units;
            for (int x = 0; x < count; x += U) {
                Got g[U];
#pragma unroll
                for (int i = 0; i < U; ++i) {
                    const int from = min(x + i, count - 1);
                    load(g[i], __builtin_amdgcn_readlane(place.page, from), __builtin_amdgcn_readlane(place.slot, from), h, u);
                }
#pragma unroll
                for (int i = 0; i < U; ++i)
                    if (x + i < count && z0 + lane < pieces) store(g[i], x0 + x + i, h, u);
            }
        }
    }
}

// --- host side ------------------------------------------------------------

static uint32_t reciprocal(int units) { return units == 1 ? 0 : (uint32_t)((((uint64_t)1 << 32) + units - 1) / units); }

// Tokens of a wave of a launch over n_tokens, at most `most`: what makes `waves`.
static int run_of(int n_tokens, int waves, int most) {
    const int64_t run = ((int64_t)n_tokens + waves - 1) / waves;
    return run < 1 ? 1 : run < most ? (int)run : most;
}

static void launch_append(Append &a, bool neighbours, hipStream_t s) {
    const mpt_kv_cache &c = a.c;
    const bool mx4 = is_mx4(c), bf16 = value_type(c) == MPT_KV_BF16;
    a.dim = c.head_dim;
    a.turn_mul = reciprocal(neighbours ? turn_units<true>(a.dim, a.pairs) : turn_units<false>(a.dim, a.pairs));
    a.copy_mul = reciprocal(mx4 ? a.dim / 32 : a.dim / 8);
    a.e_min = bf16 ? -125 : -23, a.e_max = bf16 ? 125 : 13;
    const int lanes = c.n_heads * (a.dim / 32);          // of a token's keys, in 4 bits
    // Tokens of a wave: as many as leave enough waves. In 4 bits a lane has 32 elements of a
    // token's keys, and several tokens fill a wave where heads are few.
    // Waves share tokens where there are few: 8 key heads of 128 and 32 query heads, in
    // microseconds a launch with 1 / 2 / 4 waves, 256 tokens 8.0 / 6.9 / 6.0 (into 4 bits
    // 9.4 / 8.1 / 7.7), 1024 tokens 9.3 / 8.9 / 9.4 (10.5 / 9.9 / 10.6), 2048 13.5 / 12.9 /
    // 16.9 (14.9 / 14.6 / 19.7), 4096 20.3 / 23.3 / 28.1 (21.5 / 24.6 / 33.3).
    a.run = mx4 ? run_of(a.n_tokens, 4096, lanes >= 64 ? 1 : lanes >= 32 ? 2 : kRun4) : run_of(a.n_tokens, 16384, 16);
    a.parts_log = a.n_tokens <= 512 ? 2 : a.n_tokens <= 2048 ? 1 : 0;
    using Kernel = void (*)(Append);
    static constexpr Kernel wide[2][2] = {
        {k_kv_append_rotated<__bf16, false, kApart>, k_kv_append_rotated<__bf16, false, kNeighbours>},
        {k_kv_append_rotated<_Float16, false, kApart>, k_kv_append_rotated<_Float16, false, kNeighbours>}};
    static constexpr Kernel four[2][3] = {
        {k_kv_append_rotated<__bf16, true, kWhole>, k_kv_append_rotated<__bf16, true, kNeighbours>,
         k_kv_append_rotated<__bf16, true, kApart>},
        {k_kv_append_rotated<_Float16, true, kWhole>, k_kv_append_rotated<_Float16, true, kNeighbours>,
         k_kv_append_rotated<_Float16, true, kApart>}};
    const Kernel kernel = mx4 ? four[!bf16][a.pairs == 0 ? kWhole : neighbours ? kNeighbours : kApart] : wide[!bf16][neighbours];
    // 64000 tokens of 4 query heads and 2 key heads of 64, 32 elements rotated: 63 us with four
    // tokens' angles formed at a time, 72 with one's
    a.batch = mx4 ? a.run : a.pairs < 64 ? 64 / a.pairs : 1;
    a.pair_mul = reciprocal(a.pairs ? a.pairs : 1);
    const size_t lds = 4 * (size_t)a.pairs * a.batch * (mx4 ? sizeof(Turn32) + sizeof(Turn64) : sizeof(Turn32));
    const int64_t waves = ((int64_t)a.n_tokens + a.run - 1) / a.run << a.parts_log;
    mptlib::LaunchScope scope("k_kv_append_rotated", (double)a.n_tokens, s);
    kernel<<<grid_of(waves), 256, lds, s>>>(a);
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
        const int pieces = cache->n_heads * (a.dim / 8);
        const bool many = pieces <= 32;
        a.row_mul = reciprocal(pieces);
        a.run = run_of(a.n_tokens, 8192, !many ? 4 : pieces >= 4 ? 256 / pieces : 64);
        using Kernel = void (*)(Read);
        static constexpr Kernel kernels[2][2][2] = {
            {{k_kv_read<__bf16, false, false>, k_kv_read<__bf16, false, true>}, {k_kv_read<__bf16, true, false>, k_kv_read<__bf16, true, true>}},
            {{k_kv_read<_Float16, false, false>, k_kv_read<_Float16, false, true>}, {k_kv_read<_Float16, true, false>, k_kv_read<_Float16, true, true>}}};
        hipStream_t s = (hipStream_t)stream;
        {
            mptlib::LaunchScope scope("k_kv_read", (double)n_tokens, s);
            const int64_t waves = ((int64_t)a.n_tokens + a.run - 1) / a.run;
            kernels[value_type(*cache)][is_mx4(*cache)][many]<<<grid_of(waves), 256, 0, s>>>(a);
        }
        MPT_HIP_TRY(hipGetLastError());
        return MPT_OK;
    });
}
