// Shared by the two attention kernels: their arguments, how the work of a
// ragged batch is cut over workgroups, and the matrix instructions.
//
// Rows. The queries of an entry that read one key head are n tokens x G heads
// = n G rows (row r: token r / G, head r % G), cut into tiles of M rows. A
// tile reads the keys [lo, hi) that any of its rows sees, in steps of BN
// tokens: its units.
//
// Cut. All steps of all tiles, in the order entry, key head, tile, step, each
// tile's preceded by C units for what it costs besides its steps, are one line
// of U units. Worker w takes about [w U / W, (w + 1) U / W): the same
// amount of work each whatever the lengths, with at most two tiles of its own
// cut (its first and its last). Lengths are on the device, so every workgroup
// finds its part itself, from sums over the entries. A tile that one worker
// holds alone is finished by it; of the others each worker leaves the
// unnormalised sums in the workspace, and a second launch joins them in the
// order of the workers, so results do not depend on scheduling.
#pragma once

#include "kv.h"

namespace mptkv {

struct Attn {
    mpt_kv_cache c;
    int layer, n, n_tokens, heads, group, units;     // units: 16-byte pieces of a row
    const int32_t *seqs, *q_off, *kv_begin;
    const char *q;
    char *out;
    int64_t q_token, q_head, out_token, out_head;
    uint32_t div_mul, div_s1, div_s2;                 // of a division by group
    float *lse;
    int out_f32, causal, window, flip;
    float factor;                                     // |scale| log2(e), or |scale| / softcap
    float cap;                                        // softcap log2(e)
    uint32_t k_page, k_slot, v_page, v_slot;          // strides in 16-byte units
    int near;                                         // offsets of a head's rows have 32 bits, factors 24
    const char *k, *v;                                // of the layer
    int64_t k_head, v_head;                           // bytes
    int workers;
    struct Part *parts;                               // [workers]
    float *sums;                                      // [workers][2][tile rows * (padded dim + 2)]
};

// What a worker's first tile is, if it is the second worker of that tile:
// the join's work list.
struct Part {
    int count, entry, head, tile;                     // count: workers of the tile (0: nothing to join)
    int q0, n;                                        // the entry's first token and tokens
};

constexpr int kEntries = 256;                         // entries whose sizes are held at a time
static_assert(MPT_KV_MAX_ENTRIES == kEntries * kEntries, "Entries::chunk has a place for each 256");

struct Entries {
    int q0[kEntries], n[kEntries], len[kEntries], begin[kEntries], slot[kEntries];
    int64_t steps[kEntries];                          // units of one key head
    int64_t chunk[kEntries];                          // units of each 256 entries, all heads
    int64_t wave[4];
};

struct Range {
    int lo, hi, first, count;                         // visible tokens; first step and steps (at least 1)
};

// row / group, by a product with a fraction of 2^32 and two shifts.
__device__ inline int token_of(const Attn &a, int row) {
    const uint32_t t = __umulhi(a.div_mul, (uint32_t)row);
    return (int)((t + (((uint32_t)row - t) >> a.div_s1)) >> a.div_s2);
}

template <int M, int BN>
__device__ inline Range tile_range(const Attn &a, int n, int len, int begin, int tile) {
    const int rows = n * a.group, r0 = tile * M, r1 = min(r0 + M, rows) - 1;
    Range g;
    const int p0 = len - n + token_of(a, r0), p1 = len - n + token_of(a, r1);
    g.hi = max(0, a.causal ? min(len, p1 + 1) : len);
    g.lo = a.window ? max(begin, p0 + 1 - a.window) : begin;
    if (g.hi <= g.lo) g.lo = g.hi = 0;
    g.first = g.lo / BN;
    g.count = max(1, (g.hi + BN - 1) / BN - g.first);
    return g;
}

// Tokens [lo, hi) that all rows first .. last of an entry see.
__device__ inline void seen_by_all(const Attn &a, int n, int len, int begin, int first, int last, int &lo, int &hi) {
    const int p0 = len - n + token_of(a, first), p1 = len - n + token_of(a, last);
    hi = a.causal ? min(len, p0 + 1) : len;
    lo = a.window ? max(begin, p1 + 1 - a.window) : begin;
}

template <int M>
__device__ inline int tiles_of(const Attn &a, int n) {
    return (n * a.group + M - 1) / M;
}

// Sizes of entries base .. base + 255; returns their units (all heads).
template <int M, int BN, int C>
__device__ inline int64_t load_entries(const Attn &a, Entries &s, int base) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, i = base + tid;   // a thread each
    const bool mine = tid < kEntries;
    const mpt_kv_cache &c = a.c;
    int n = 0, len = 0, begin = 0, q0 = 0, slot = 0;
    if (mine && i < a.n) {
        q0 = a.q_off[i];
        const int q1 = a.q_off[i + 1];
        slot = a.seqs[i];
        const bool csr = q0 >= 0 && q0 <= q1 && q1 <= a.n_tokens;
        const bool ok = slot >= 0 && slot < c.max_seqs;
        if (csr) n = q1 - q0;
        if (ok) len = max(0, min(c.length[slot], c.max_pages * c.page_size));
        if (a.kv_begin) begin = max(0, a.kv_begin[i]);
        if (blockIdx.x == 0 && !(csr && ok)) flag(c, MPT_KV_BAD_SLOT);
        if (!ok) slot = 0;
    }
    const int tiles = tiles_of<M>(a, n);
    int64_t steps = 0;
    if (tiles <= 8)
        for (int t = 0; t < tiles; ++t) steps += C + tile_range<M, BN>(a, n, len, begin, t).count;
    // long entries: the lanes of a wave take the tiles
    for (uint64_t todo = __ballot(tiles > 8); todo; todo &= todo - 1) {
        const int src = __ffsll((unsigned long long)todo) - 1;
        const int n2 = __builtin_amdgcn_readlane(n, src), len2 = __builtin_amdgcn_readlane(len, src);
        const int begin2 = __builtin_amdgcn_readlane(begin, src);
        int64_t x = 0;
        for (int t = lane; t < tiles_of<M>(a, n2); t += 64) x += C + tile_range<M, BN>(a, n2, len2, begin2, t).count;
        x = of_lane(wave_sums(x), 63);
        if (lane == src) steps = x;
    }
    if (mine) s.q0[tid] = q0, s.n[tid] = n, s.len[tid] = len, s.begin[tid] = begin, s.slot[tid] = slot, s.steps[tid] = steps;
    const int64_t sum = of_lane(wave_sums(steps), 63);
    __syncthreads();
    if (mine && lane == 0) s.wave[wave] = sum;
    __syncthreads();
    return (s.wave[0] + s.wave[1] + s.wave[2] + s.wave[3]) * c.n_heads;
}

// A workgroup's walk over its units.
template <int M, int BN, int C>
struct Walk {
    int64_t total, at, end;           // units: all, this worker's next, its end
    int64_t before;                   // units before the current entry
    int worker, workers, base, e;     // entries base .. are loaded, e is the current one
    int head, tile;
    int64_t tile_at;                  // units before the current tile

    // Units before worker w's. In doubles, where a 64-bit division would be a
    // hundred instructions: every workgroup gets the same, it rises with w,
    // and it ends at the total.
    __device__ int64_t cut(int w) const {
        return w >= workers ? total : (int64_t)((double)total * (double)w / (double)workers);
    }
    // The worker that holds unit u.
    __device__ int owner(int64_t u) const {
        int w = min(workers - 1, (int)((double)u * (double)workers / (double)total));
        while (w + 1 < workers && cut(w + 1) <= u) ++w;
        while (w > 0 && cut(w) > u) --w;
        return w;
    }

    // False if this workgroup has no work. least: units that are worth a worker.
    __device__ bool begin(const Attn &a, Entries &s, int least) {
        const int tid = threadIdx.x;
        int64_t sum = 0;
        for (base = 0; base < a.n; base += kEntries) {
            const int64_t x = load_entries<M, BN, C>(a, s, base);
            if (tid == 0) s.chunk[base / kEntries] = x;
            sum += x;
        }
        total = uniform(sum);
        workers = a.workers;
        if (total < (int64_t)least * workers) workers = max(1, (int)total / least);
        // neighbours, which read the same keys, on one XCD (the grid is a
        // multiple of 8: every number below it is one workgroup's)
        const int per = (workers + 7) / 8, bid = blockIdx.x;
        worker = (bid >> 3) < per ? (bid & 7) * per + (bid >> 3) : bid;
        if (tid == 0) a.parts[worker].count = 0;
        if (total == 0 || worker >= workers) return false;
        at = uniform(cut(worker));
        end = uniform(cut(worker + 1));
        if (at == end) return false;
        __syncthreads();
        before = 0;
        int k = 0;
        while (before + uniform(s.chunk[k]) <= at) before += uniform(s.chunk[k++]);
        if (a.n > kEntries) {
            __syncthreads();
            load_entries<M, BN, C>(a, s, k * kEntries);
        }
        base = k * kEntries;
        // the entry, by the lanes of each wave: 64 at a time
        const int lane = tid & 63;
        e = 0;
        for (;;) {
            const int64_t x = s.steps[e + lane] * a.c.n_heads, y = wave_sums(x);
            const uint64_t past = __ballot(before + y > at);
            if (past) {
                const int k2 = __ffsll((unsigned long long)past) - 1;
                before += of_lane(y - x, k2);
                e += k2;
                break;
            }
            before += of_lane(y, 63);
            e += 64;
        }
        const int64_t in = at - before, steps = uniform(s.steps[e]);
        head = (int)((double)in / (double)steps);
        while (head > 0 && head * steps > in) --head;
        while ((head + 1) * steps <= in) ++head;
        head = uniform(head);
        find_tile(a, s, in - head * steps);
        return true;
    }

    // The tile that holds the given unit of a head of the current entry.
    __device__ void find_tile(const Attn &a, const Entries &s, int64_t unit) {
        const int lane = threadIdx.x & 63, tiles = tiles_of<M>(a, s.n[e]);
        int64_t sum = 0;
        for (tile = 0;; tile += 64) {
            const int64_t x = tile + lane < tiles ? C + tile_range<M, BN>(a, s.n[e], s.len[e], s.begin[e], tile + lane).count : 0;
            const int64_t y = wave_sums(x);
            const uint64_t past = __ballot(sum + y > unit);
            if (past) {
                const int k = __ffsll((unsigned long long)past) - 1;
                tile += k;
                tile_at = before + head * uniform(s.steps[e]) + sum + of_lane(y - x, k);
                return;
            }
            sum += of_lane(y, 63);
        }
    }

    // The worker's steps [first, last) of the current tile of `count`, and
    // past them in the line.
    __device__ void take(int count, int &first, int &last) {
        first = uniform((int)max((int64_t)0, at - tile_at - C));
        last = uniform((int)max((int64_t)0, min((int64_t)count, end - tile_at - C)));
        at = min(end, tile_at + C + count);
    }

    // Where this worker is the second of a tile of `count` steps: the tile's workers, else 0.
    __device__ int second_of(int count) const {
        const int w0 = owner(tile_at + C);
        return w0 + 1 == worker ? owner(tile_at + C + count - 1) - w0 + 1 : 0;
    }

    // To the next tile, after all units of the current one.
    __device__ void next(const Attn &a, Entries &s) {
        tile_at = at;
        if (++tile < tiles_of<M>(a, uniform(s.n[e]))) return;
        tile = 0;
        if (++head < a.c.n_heads) return;
        head = 0;
        before = at;
        do {
            if (++e == kEntries) {
                __syncthreads();
                base += kEntries;
                load_entries<M, BN, C>(a, s, base);
                e = 0;
            }
        } while (uniform(s.n[e]) == 0);
    }
};

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

template <class T> struct Type;
template <> struct Type<__bf16> {
    using x8 = bf16x8;
    static constexpr int kExponent = 0x7f80;
    __device__ static f32x16 mfma32(s16x8 x, s16x8 y, f32x16 z) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), z, 0, 0, 0);
    }
    __device__ static f32x4 mfma16(s16x8 x, s16x8 y, f32x4 z) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), z, 0, 0, 0);
    }
};
template <> struct Type<_Float16> {
    using x8 = f16x8;
    static constexpr int kExponent = 0x7c00;
    __device__ static f32x16 mfma32(s16x8 x, s16x8 y, f32x16 z) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, x), __builtin_bit_cast(f16x8, y), z, 0, 0, 0);
    }
    __device__ static f32x4 mfma16(s16x8 x, s16x8 y, f32x4 z) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, x), __builtin_bit_cast(f16x8, y), z, 0, 0, 0);
    }
};

// A row of zeros in memory: what is read in place of tokens outside a tile's
// range, of pages that do not exist and of dimensions past head_dim. Rows of
// zeros take part in every product without a trace; the stale contents of a
// page may be NaN, and 0 x NaN is none.
static __device__ const uint4 kZeros[MPT_KV_MAX_DIM / 8] = {};

// from, or zeros; a select that is not turned into branches around two loads.
__device__ inline const char *or_zeros(bool there, const char *from) {
    uint64_t p = (uint64_t)(there ? from : (const char *)kZeros);
    asm("" : "+v"(p));
    return (const char *)p;
}

// x, as a value that may differ from one pass of a loop to the next: addresses
// formed from it are formed anew instead of being kept in registers.
__device__ inline int renewed(int x) {
    asm volatile("" : "+v"(x));
    return x;
}

template <class V>
__device__ inline V load(const char *from) {
    return *(const __attribute__((address_space(1))) V *)(uint64_t)from;
}

// 16 bytes per lane from memory to LDS, lane i at lds + 16 i, without a stop
// in registers. The instruction is written out because the compiler takes any
// later LDS read for one of its result and would wait for the loads of the
// next tile there; who uses it waits (arrived) before the barrier that lets
// the tile be read. m0, which the address goes through, is named as written:
// the compiler, which keeps no value there, may else take two settings of its
// own for one where a statement stands between them. It warns that it would
// not restore a register of that kind: nothing needs it restored.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ inline void load_lds16(const char *from, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(uniform((int)lds)), "v"(from) : "memory", "m0");
}
// The same with 4 bytes per lane.
__device__ inline void load_lds4(const void *from, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(uniform((int)lds)), "v"(from) : "memory", "m0");
}
// The same at 32-bit offsets from one address.
__device__ inline void load_lds16(const void *base, uint32_t offset, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(uniform((int)lds)), "v"(offset), "s"(uniform((int64_t)base)) : "memory", "m0");
}
__device__ inline void load_lds4(const void *base, uint32_t offset, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(uniform((int)lds)), "v"(offset), "s"(uniform((int64_t)base)) : "memory", "m0");
}
#pragma clang diagnostic pop
// Waits until at most N of the wave's later loads are on their way: loads
// arrive in order, so all before those N have.
template <int N>
__device__ inline void arrived() {
    static_assert(N >= 0 && N < 64, "the counter has six bits");
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

__device__ inline uint32_t lds_address(const void *p) {
    return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void *)p;
}

// Bytes from a layer's and head's first row to that of a token: strides are
// counted in 16 bytes, so that 32-bit factors reach 64 GiB per page.
__device__ inline uint64_t row_at(uint32_t page, uint32_t slot, uint32_t page_stride, uint32_t slot_stride) {
    return ((uint64_t)page * page_stride + (uint64_t)slot * slot_stride) << 4;
}

template <class V>
__device__ inline V from_lds(uint32_t at) {
    return *(const __attribute__((address_space(3))) V *)(uintptr_t)at;
}

// Four elements of one column from four rows: the lanes of 16 exchange what
// they read, lane i of them getting column i.
__device__ inline s16x4 read_column4(uint32_t at) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(uintptr_t)at);
}
__device__ inline s16x4 read_column4(const char *lds) { return read_column4(lds_address(lds)); }

template <class T>
__device__ inline uint32_t pack(float x, float y) {
    typedef T t2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x, y}, t2));
}

// Positions in log2 units of a score x = q.k: x |scale| log2(e), or with a
// cap c log2(e) tanh(x |scale| / c). tanh z = 1 - 2 / (1 + e^2z); below 1/4,
// where that cancels, its series to z^9 (relative error 1e-8).
template <bool CAP>
__device__ inline float score(const Attn &a, float x) {
    if constexpr (!CAP) return x * a.factor;
    const float z = x * a.factor, y = z * z;
    const float e = __builtin_amdgcn_exp2f(2.885390081777927f * z);
    const float big = 1.0f - 2.0f * __builtin_amdgcn_rcpf(1.0f + e);
    const float small = z * (1.0f + y * (-0.333333333f + y * (0.133333333f + y * (-0.053968254f + y * 0.021869489f))));
    return a.cap * (fabsf(z) < 0.25f ? small : big);
}

template <class T>
__device__ inline bool finite16(short x) {
    return (x & Type<T>::kExponent) != Type<T>::kExponent;
}

// By value: __builtin_bit_cast of an element of a vector takes its first one.
template <class T>
__device__ inline float value16(short x) {
    return (float)__builtin_bit_cast(T, x);
}

// Whether any of 8 elements is an infinity or NaN.
template <class T>
__device__ inline uint32_t odd8(s16x8 x) {
    const uint4 u = __builtin_bit_cast(uint4, x);
    constexpr uint32_t kE = Type<T>::kExponent * 0x10001u, kOne = (0x8000u - Type<T>::kExponent) * 0x10001u;
    return (((u.x & kE) + kOne) | ((u.y & kE) + kOne) | ((u.z & kE) + kOne) | ((u.w & kE) + kOne)) & 0x80008000u;
}

// Not a zero if one of a lane's sums is an infinity or NaN.
__device__ inline float not_finite(f32x4 x) {
    return __builtin_fmaf(x[0], 0.0f, __builtin_fmaf(x[1], 0.0f, __builtin_fmaf(x[2], 0.0f, x[3] * 0.0f)));
}

// Infinities and NaN in values. A product cannot hold them: under the weight 0
// of a row that does not see the token, or sees it with a weight that the type
// rounds to 0, it is NaN. So where some rows do not see a step's tokens, the
// step's product takes zeros in their place; and a tile that has met one, or
// whose sums came out infinite or NaN, ends here: a wave looks through the
// values of tokens t0 .. t1 - 1 once more, and every sum that an infinity or NaN
// belongs to becomes the sum of those alone, which is what the definition
// gives. Two bits a dimension hold it (infinities of either sign, both: NaN),
// and the look ends where nothing can change any more. Chunks of 1024 tokens
// over 16k as a lone call, 1.3 ms: 2.8 with one infinity among the values, 11
// with one in every page, 1.3 with NaN everywhere, 149 with infinities
// everywhere.
//
// A lane's row sees lo .. hi - 1; its sums, groups of four dimensions from d0 on,
// `step` apart, lie at `to`, `inc` bytes apart, in 32 bits or T. l: the row's sum
// of weights (NaN: so are its sums). Without any weight a whole row is zeros;
// parts keep what they saw, and their join decides.
template <class T, int GROUPS>
__device__ inline void odd_values(const Attn &a, const int32_t *table, int shift, const char *values, int t0, int t1, int lo,
                                  int hi, float l, bool whole, int d0, int step, char *to, int inc, bool f32) {
    static_assert(GROUPS <= 16, "four bits a group");
    const int lane = threadIdx.x & 63, dim = 8 * a.units;
    if (whole && l == 0)
        for (int k = 0; d0 + k * step < dim; ++k) {
            if (f32)
                *(f32x4 *)(to + k * inc) = f32x4{0, 0, 0, 0};
            else
                *(s16x4 *)(to + k * inc) = s16x4{0, 0, 0, 0};
        }
    const bool mine = l > 0 || (l == 0 && !whole);
#pragma unroll 1
    for (; __any(d0 < dim); d0 += GROUPS * step, to += GROUPS * inc) {          // GROUPS at a time
        uint64_t up = 0, down = 0, all = 0;
        for (int k = 0; k < GROUPS && d0 + k * step < dim; ++k) all |= 15ull << 4 * k;
#pragma unroll 1
        for (int base = t0; base < t1 && !__all(!mine || (up & down) == all); base += 64) {
            const int t = base + lane, page = t < t1 ? table[t >> shift] : -1;
            const char *row = values + row_at(page, t & (a.c.page_size - 1), a.v_page, a.v_slot);
            uint32_t odd = 0;
            if ((unsigned)page < (unsigned)a.c.n_pages)
                for (int u = 0; u < a.units; ++u) odd |= odd8<T>(load<s16x8>(row + 16 * u));
#pragma unroll 1
            for (uint64_t todo = __ballot(odd != 0); todo; todo &= todo - 1) {
                const int at = __ffsll((unsigned long long)todo) - 1;
                const char *token = (const char *)of_lane((int64_t)row, at) + 2 * d0;
                if (!mine || base + at < lo || base + at >= hi || (up & down) == all) continue;
#pragma unroll 4
                for (int k = 0; k < GROUPS; ++k) {
                    if (d0 + k * step >= dim) break;
                    const s16x4 y = load<s16x4>(token + 2 * k * step);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float x = value16<T>(y[i]);
                        up |= (uint64_t)(!finite16<T>(y[i]) && !(x < 0)) << (4 * k + i);
                        down |= (uint64_t)(!finite16<T>(y[i]) && !(x > 0)) << (4 * k + i);
                    }
                }
            }
        }
#pragma unroll 1
        for (uint64_t set = up | down; set; set &= set - 1) {
            const int b = __ffsll((unsigned long long)set) - 1;
            const float x = !(down >> b & 1) ? INFINITY : up >> b & 1 ? NAN : -INFINITY;
            char *z = to + (b >> 2) * inc;
            if (f32)
                ((float *)z)[b & 3] = x;
            else
                ((T *)z)[b & 3] = (T)x;
        }
    }
}

// The same in a join: a part's infinity under a factor that is too small for 32
// bits has made the sum o NaN, and is what it should be. part(i): where part i's
// four sums lie.
template <class Place>
__device__ inline f32x4 odd_parts(f32x4 o, int count, Place part) {
    if (__builtin_expect(!__any(not_finite(o) != 0), 1)) return o;
    f32x4 sum = {0, 0, 0, 0};
    bool odd[4] = {};
#pragma unroll 1
    for (int i = 0; i < count; ++i) {
        const f32x4 x = *(const f32x4 *)part(i);
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (!(fabsf(x[k]) < INFINITY)) sum[k] += x[k], odd[k] = true;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) o[k] = odd[k] ? sum[k] : o[k];
    return o;
}

template <class T, bool F32>
__device__ inline void put4(char *out, int64_t at, f32x4 x) {
    if constexpr (F32) {
        *(f32x4 *)(out + 4 * at) = x;
    } else {
        typedef T t4 __attribute__((ext_vector_type(4)));
        *(t4 *)(out + 2 * at) = __builtin_convertvector(x, t4);
    }
}
template <class T>
__device__ inline void store4(const Attn &a, int64_t at, f32x4 x) {
    a.out_f32 ? put4<T, true>(a.out, at, x) : put4<T, false>(a.out, at, x);
}

inline int pad_dim(int dim) { return dim <= 64 ? 64 : dim <= 128 ? 128 : 256; }

// Launch of a kernel and of its join; the joins alone.
void launch_wide(const Attn &a, int waves, hipStream_t s);
void launch_narrow(const Attn &a, hipStream_t s);
void join_wide(const Attn &a, int waves, hipStream_t s);
void join_narrow(const Attn &a, hipStream_t s);

}  // namespace mptkv
