// Attention kernel over a cache in 4 bits for few rows per key head (decoding):
// tiles of 16 rows, the four waves of a workgroup 32 tokens each of a step of 128,
// as over 16 bits.
//
// Codes of keys go to LDS as they come: a lane reads back a quarter of a token's
// row, which is one E (heads of 128), as the operand of S' = K Q', whose dimensions
// may come in any order if the queries agree on it. Values become 16-bit rows on
// their way into LDS, where they are read by columns. What a load brings costs the
// same in the address units whether its lanes take one byte or 16, so the bytes E of
// a step's keys and values are one load of a row a lane, and its page ids another;
// lanes ask each other for them.
//
// What bounds it is memory, where a worker has one tile: 64 contexts of 4000 tokens,
// 32 heads on 8 of 128, 50 us (5.5 TB/s). Ragged contexts cost the starts and ends of
// the tiles that a worker's part of the line cuts: 64 of 700 to 9000 tokens 82 us (4.1
// TB/s) with a start counted as 3 steps, 84.5 as one, and 37 short ones of 64 19.9,
// 21.3. Nothing else moved it: steps loaded two ahead instead of one (86), three
// workgroups to a CU instead of two (79 to 88, with registers put into memory), cheaper
// instructions in forming addresses.

#include "attention_mx4.h"

#include <type_traits>

#define INLINE __attribute__((always_inline))

namespace mptkv {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

template <int DP>
struct Narrow4 {
    static constexpr int M = 16, BN = 128, KK = DP / 32, DT = DP / 16, ROW = 2 * DP, CH = DP / 8;
    static constexpr int C = 3;                                        // a tile's cost besides its steps, in steps
    static constexpr int CODES = DP / 2, CP = CODES / 16, L = CP / 2;  // bytes and pieces of a row of codes; loads of 1 KiB
    static constexpr int E = DP == 256 ? 2 : 1;                        // bytes E of a quarter of a row
    static constexpr int kKeys = 32 * CODES, kValues = 32 * ROW;       // of a wave

    static constexpr int EW = DP == 256 ? 2 : 1;                       // words of E a row

    // Where the 16-byte pieces of a token's row of codes lie: those that eight lanes
    // read at a time (a quarter of eight tokens each) on different banks.
    __device__ static int k_swizzle(int t) { return DP == 64 ? (t >> 2) & 1 : DP == 128 ? (t >> 1) & 3 : t & 7; }
    // And of a row of values: those that eight lanes write at a time (the same
    // quarter of eight pieces) and that 16 read (32 bytes of four tokens each).
    __host__ __device__ static constexpr int v_fold(int u) { return DP == 64 ? u : DP == 128 ? u ^ ((u >> 3) & 1) : u ^ ((u >> 3) & 3); }
    __device__ static int v_swizzle(int t) { return DP == 64 ? 2 * (t & 3) + ((t >> 1) & 1) : 2 * (t & 7); }
};

template <class T, int DP, bool CAP, bool PAD>
__global__ __launch_bounds__(256, DP == 256 ? 1 : DP == 128 ? 2 : 3) void k_kv_narrow_mx4(Attn4 a) {
    using N = Narrow4<DP>;
    constexpr int M = N::M, BN = N::BN, C = N::C, KK = N::KK, DT = N::DT, ROW = N::ROW, CP = N::CP, L = N::L, E = N::E, EW = N::EW;
    __shared__ Entries ent;
    __shared__ __attribute__((aligned(1024))) char tiles[4 * (N::kKeys + N::kValues)];
    __shared__ float stat[4][2][16];
    __shared__ __attribute__((aligned(4))) char met_odd[4];
    const mpt_kv_cache &c = a.c;
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), col = lane & 15, quad = lane >> 4;
    const int shift = 31 - __clz(c.page_size), pieces = a.units / 4;
    char *vw = tiles + wave * N::kValues, *kw = tiles + 4 * N::kValues + wave * N::kKeys;
    // Where a lane writes and reads: swizzles are the same 8 tokens on, so all other
    // places are these with bits turned over, and constants from there.
    const int put_t = lane / CP, put_p = lane & (CP - 1), own_row = lane >> 2;   // own_row: 4 quad + col / 4
    const uint32_t k_put = lds_address(kw) + put_t * N::CODES + ((put_p ^ N::k_swizzle(put_t)) << 4);
    const uint32_t v_put = lds_address(vw) + put_t * ROW + ((N::v_fold(4 * put_p) ^ N::v_swizzle(put_t)) << 4);
    const uint32_t k_get = lds_address(kw) + col * N::CODES +
                           (DP == 64 ? ((quad / 2 ^ N::k_swizzle(col)) << 4) + (quad & 1) * 8 : (E * quad ^ N::k_swizzle(col)) << 4);
    const uint32_t v_get = lds_address(vw) + own_row * ROW + (((lane & 3) / 2 ^ N::v_swizzle(own_row)) << 4) + (lane & 1) * 8;
    bool lost = false;                         // a page id outside the pool

    Walk<M, BN, C> walk;
    if (!walk.begin(a, ent, 1)) return;

    while (walk.at < walk.end) {
        const int e = uniform(walk.e), n = uniform(ent.n[e]), len = uniform(ent.len[e]), q0 = uniform(ent.q0[e]);
        const int begin = uniform(ent.begin[e]), head = uniform(walk.head), tile = uniform(walk.tile);
        const Range range = tile_range<M, BN>(a, n, len, begin, tile);
        int from, to;
        walk.take(range.count, from, to);
        const bool starts = from == 0, ends = to == range.count;
        if (from == to) {                      // only what comes before its steps: the next worker's tile
            break;
        }
        const int first = range.first + from, last = range.first + to;
        const int rows = n * a.group;
        const int32_t *table = c.table + (int64_t)uniform(ent.slot[e]) * c.max_pages;

        const int r = tile * M + col, rr = min(r, rows - 1), j = token_of(a, rr), hq = rr - j * a.group, p = len - n + j;
        const int see_hi = a.causal ? min(len, p + 1) : len;
        const int see_lo = a.window ? max(begin, p + 1 - a.window) : begin;
        const int64_t token = q0 + j, hh = (int64_t)head * a.group + hq;
        int all_lo, all_hi;
        seen_by_all(a, n, len, begin, tile * M, min(tile * M + M, rows) - 1, all_lo, all_hi);
        s16x8 qf[KK];                          // a quarter of the row a lane
        {
            const char *q = a.q + 2 * (token * a.q_token + hh * a.q_head);
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) {
                const int piece = KK * quad + kk;
                u32x4 x = mptkv::load<u32x4>(or_zeros(r < rows && piece < a.units, q + 16 * piece));
                if (a.flip) x ^= 0x80008000u;
                qf[kk] = __builtin_bit_cast(s16x8, x);
            }
        }
        f32x4 o[DT];
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[dt] = f32x4{0, 0, 0, 0};
        float m = -INFINITY, l = 0;
        bool met = false;                      // a NaN that was taken out of a product

        // Tokens of a step that the tile does not reach are read as others of it
        // (their scores are masked, and a weight of 0 times a finite value is 0),
        // and so are pieces past the row's end (their queries are 0). A page id
        // outside the pool becomes the last page, and is reported.
        // A step's tokens are 32 slots of a page, or pages are of the step: a lane's
        // places in them are the same for all steps but for what is uniform.
        constexpr int T16 = 64 / CP;                               // tokens of a load: 8, 16 or 32
        const int piece = min(put_p, pieces - 1);
        const uint32_t own_slot = put_t & (c.page_size - 1);
        const char *kx = at(a.k + head * a.k_head + 16 * piece, own_slot, a.k_slot), *vx = at(a.v + head * a.v_head + 16 * piece, own_slot, a.v_slot);
        // Bytes E: of the step's 32 tokens, keys' in the lower half of the wave, values' in
        // the upper, a row a lane.
        const uint32_t e_slot = (lane & 31) & (c.page_size - 1);
        const char *ex = lane < 32 ? at(a.ke + head * a.ke_head, e_slot, a.ke_slot) : at(a.ve + head * a.ve_head, e_slot, a.ve_slot);
        const uint32_t e_page = lane < 32 ? a.ke_page : a.ve_page, e_stride = lane < 32 ? a.ke_slot : a.ve_slot;
        // The next step is on its way while one is worked on, and the page ids of the one
        // after it: loads arrive in order, so ids have to be asked for before the codes
        // that are waited for when they are used. Lane l and l + 32 have the page of token
        // l of the wave's 32. Every load costs the address units the same whether its
        // lanes take one byte or 16.
        u32x4 kr[L], vr[L];
        uint32_t er[EW];
        uint8_t eb[PAD ? CP : 1];
        int ids;
        auto find_pages = [&](int step) INLINE {
            const int t = step * BN + wave * 32 + (lane & 31);
            return table[max(range.lo, min(range.hi - 1, t)) >> shift];
        };
        struct Pages { uint32_t of[L], e; };
        auto pages_of = [&](int ids) INLINE {
            const uint32_t page = min((uint32_t)ids, (uint32_t)c.n_pages - 1);
            lost |= page != (uint32_t)ids;
            Pages p;
#pragma unroll
            for (int i = 0; i < L; ++i) p.of[i] = __shfl((int)page, i * T16 + put_t);
            p.e = page;
            return p;
        };
        auto load = [&](const Pages &p, int step) INLINE {
            const uint32_t slot0 = (uint32_t)(step * BN + wave * 32) & (c.page_size - 1);
#pragma unroll
            for (int i = 0; i < L; ++i) {
                const uint64_t slot = slot0 + (i * T16 & (c.page_size - 1));
                kr[i] = mptkv::load<u32x4>(at(kx, p.of[i], a.k_page) + slot * a.k_slot);
                vr[i] = mptkv::load<u32x4>(at(vx, p.of[i], a.v_page) + slot * a.v_slot);
            }
            const char *e = at(at(ex, p.e, e_page), slot0, e_stride);
            if constexpr (PAD) {
#pragma unroll
                for (int x = 0; x < CP; ++x) eb[x] = mptkv::load<uint8_t>(e + min(x, pieces - 1));
            } else if constexpr (DP == 64) {
                er[0] = mptkv::load<uint16_t>(e);
            } else if constexpr (DP == 128) {
                er[0] = mptkv::load<uint32_t>(e);
            } else {
                const u32x2 x = mptkv::load<u32x2>(e);
                er[0] = x[0], er[1] = x[1];
            }
        };
        auto one_step = [&](int step) INLINE {
            const int t0 = step * BN + wave * 32;
            if constexpr (PAD) {
#pragma unroll
                for (int x = 0; x < EW; ++x) er[x] = 0;
#pragma unroll
                for (int x = 0; x < CP; ++x) er[x / 4] |= (uint32_t)eb[x] << 8 * (x % 4);
            }
            // E from the lanes that have them: of block b of the row that lane `from` holds
            auto scale_of = [&](int from, int b) INLINE -> uint32_t {
                uint32_t x = __shfl((int)er[0], from);
                if constexpr (EW == 2) {
                    const uint32_t y = __shfl((int)er[1], from);
                    x = b >= 4 ? y : x;
                }
                return __builtin_amdgcn_ubfe(x, 8 * (b & 3), 8);
            };
            uint32_t vs[L];
            bool k_odd = false, v_odd = false;
#pragma unroll
            for (int i = 0; i < L; ++i) vs[i] = scale_of(32 + i * T16 + put_t, piece), v_odd |= vs[i] > kMaxScale<T>;
            float ku[2][E];
#pragma unroll
            for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                for (int x = 0; x < E; ++x) {
                    const uint32_t y = scale_of(mt * 16 + col, DP == 64 ? quad / 2 : quad * E + x);
                    k_odd |= y > kMaxScale<T>;
                    ku[mt][x] = unit_of(y);
                }
            if (__builtin_expect(__any(v_odd), 0)) {               // NaN: zeros (nan_values)
                met = true;
#pragma unroll
                for (int i = 0; i < L; ++i)
                    if (vs[i] > kMaxScale<T>) vr[i] = u32x4{0, 0, 0, 0}, vs[i] = 0;
            }
#pragma unroll
            for (int i = 0; i < L; ++i) {
                to_lds(k_put + i * T16 * N::CODES, kr[i]);
                const float unit = unit_of(vs[i]);
#pragma unroll
                for (int w = 0; w < 4; ++w) to_lds((v_put ^ w << 4) + i * T16 * ROW, from_codes<T>(vr[i][w], unit));
            }
            // past the last step too, whose tokens are then others of the range: what is on
            // its way has to be the same on all ways here, or a step would wait for all of it
            const Pages p = pages_of(ids);
            ids = find_pages(step + 2);
            load(p, step + 1);
            if (t0 >= range.hi || t0 + 32 <= range.lo) return;     // nothing for this wave
            float s[8];
#pragma unroll
            for (int mt = 0; mt < 2; ++mt) {
                uint32_t codes[KK];
                if constexpr (DP == 64) {
                    const u32x2 x = from_lds<u32x2>(k_get + mt * 16 * N::CODES);
                    codes[0] = x[0], codes[1] = x[1];
                } else {
#pragma unroll
                    for (int x = 0; x < E; ++x) {
                        const u32x4 y = from_lds<u32x4>((k_get ^ x << 4) + mt * 16 * N::CODES);
#pragma unroll
                        for (int w = 0; w < 4; ++w) codes[4 * x + w] = y[w];
                    }
                }
                s16x8 kf[KK];
#pragma unroll
                for (int kk = 0; kk < KK; ++kk) kf[kk] = from_codes<T>(codes[kk], ku[mt][kk * E / KK]);
                if (__builtin_expect(__any(k_odd), 0)) {           // scores that are NaN
#pragma unroll
                    for (int kk = 0; kk < KK; ++kk)
                        if (ku[mt][kk * E / KK] > unit_of(kMaxScale<T>)) kf[kk] = nans<T>();
                }
                f32x4 x = {0, 0, 0, 0};
#pragma unroll
                for (int kk = 0; kk < KK; ++kk) x = Type<T>::mfma16(kf[kk], qf[kk], x);
#pragma unroll
                for (int i = 0; i < 4; ++i) s[mt * 4 + i] = x[i];
            }
            const bool masked = t0 < all_lo || t0 + 32 > all_hi;
            if constexpr (CAP) {
#pragma unroll
                for (int i = 0; i < 8; ++i) s[i] = score<true>(a, s[i]);
            }
            if (masked) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int t = t0 + 16 * (i / 4) + 4 * quad + i % 4;
                    s[i] = t >= see_lo && t < see_hi ? s[i] : -INFINITY;
                }
            }
            float top = -INFINITY;
#pragma unroll
            for (int i = 0; i < 8; ++i) top = fmaxf(top, s[i]);
            if constexpr (!CAP) top *= a.factor;
            if (__any(top > m + 8.0f)) {
                top = fmaxf(top, __shfl_xor(top, 16));
                top = fmaxf(top, __shfl_xor(top, 32));
                const float now = fmaxf(m, top), keep = now == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - now);
                m = now;
                l *= keep;
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) o[dt] *= keep;
            }
            const float base = m == -INFINITY ? 0.0f : m;
            // rounded to the 16-bit type for the product, as over 16 bits
            u32x4 packed;
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                const float x = __builtin_amdgcn_exp2f(CAP ? s[i] - base : __builtin_fmaf(s[i], a.factor, -base));
                const float y = __builtin_amdgcn_exp2f(CAP ? s[i + 1] - base : __builtin_fmaf(s[i + 1], a.factor, -base));
                l += x + y;
                packed[i / 2] = pack<T>(x, y);
            }
            const s16x8 pf = __builtin_bit_cast(s16x8, packed);
#pragma unroll
            for (int g = 0; g < DT; g += 4) {
                s16x8 vf[4];
#pragma unroll
                for (int dt = 0; dt < 4; ++dt) {
                    const uint32_t q = v_get ^ N::v_fold(2 * (g + dt)) << 4;
                    const s16x4 x = read_column4(q), y = read_column4(q + 16 * ROW);
                    vf[dt] = __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
                }
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int dt = 0; dt < 4; ++dt) o[g + dt] = Type<T>::mfma16(vf[dt], pf, o[g + dt]);
            }
        };
        if (range.hi > range.lo) {
            ids = find_pages(first);
            const Pages p = pages_of(ids);
            ids = find_pages(first + 1);
            load(p, first);
#pragma unroll 1
            for (int step = first; step < last; ++step) one_step(step);
        }

        // the waves' parts: each in its own LDS, DT vectors of 1 KiB
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        if (quad == 0) stat[wave][0][col] = m, stat[wave][1][col] = l;
        if (lane == 0) met_odd[wave] = met;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) *(f32x4 *)(vw + dt * 1024 + lane * 16) = o[dt];
        __syncthreads();
        float f[4], all_m = -INFINITY, all_l = 0;
#pragma unroll
        for (int w = 0; w < 4; ++w) all_m = fmaxf(all_m, stat[w][0][col]);
        const float base = all_m == -INFINITY ? 0.0f : all_m;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            f[w] = __builtin_amdgcn_exp2f(stat[w][0][col] - base);
            all_l += f[w] * stat[w][1][col];
        }
        const float scale = !(starts && ends) ? 1.0f : all_l == 0 ? 0.0f : 1.0f / all_l;
        float *sums = a.sums + ((int64_t)uniform(walk.worker) * 2 + (starts ? 1 : 0)) * (M * (DP + 2));
#pragma unroll
        for (int k = 0; k < DT / 4; ++k) {
            const int dt = k * 4 + wave;
            f32x4 x = {0, 0, 0, 0};
#pragma unroll
            for (int w = 0; w < 4; ++w) x += f[w] * *(const f32x4 *)(tiles + w * N::kValues + dt * 1024 + lane * 16);
            x *= scale;
            if (starts && ends) {
                const int d = dt * 16 + 4 * quad;
                if (r < rows && d < 8 * a.units) store4<T>(a, token * a.out_token + hh * a.out_head + d, x);
            } else {
                *(f32x4 *)(sums + (dt * 64 + lane) * 4) = x;
            }
        }
        if (starts && ends) {
            if (a.lse && wave == 0 && quad == 0 && r < rows)
                a.lse[token * a.heads + hh] = all_l == 0 ? -INFINITY : 0.693147180559945f * (all_m + __builtin_amdgcn_logf(all_l));
        } else {
            if (wave == 0 && quad == 0) sums[M * DP + col] = all_m, sums[M * DP + 16 + col] = all_l;
            if (!starts && tid == 0) {
                const int workers = walk.second_of(range.count);
                if (workers) a.parts[walk.worker] = Part{workers, e + walk.base, head, tile, q0, n};
            }
        }
        if (__builtin_expect(*(const uint32_t *)met_odd != 0, 0)) {
            const bool whole = starts && ends, f32 = !whole || a.out_f32;
            const int d = wave * 16 + 4 * quad, size = f32 ? 4 : 2;
            nan_values<T>(a, table, shift, a.ve + head * a.ve_head, max(range.lo, first * BN), min(range.hi, last * BN), see_lo, see_hi,
                          r < rows ? all_l : NAN, whole, d, 64,
                          whole ? a.out + size * (token * a.out_token + hh * a.out_head + d) : (char *)(sums + (wave * 64 + lane) * 4),
                          whole ? 64 * size : 4 * 64 * 16, f32);
        }
        __syncthreads();                      // the LDS is free again
        if (ends && walk.at < walk.end) walk.next(a, ent);
    }
    if (lost) flag(c, MPT_KV_BAD_PAGE);
}

template <class T, int DP>
static void launch(const Attn4 &a, hipStream_t s) {
    mptlib::LaunchScope scope("k_kv_narrow_mx4", (double)a.n_tokens * a.heads, s);
    const bool pad = 8 * a.units < DP;
    const auto kernel = a.cap != 0 ? (pad ? k_kv_narrow_mx4<T, DP, true, true> : k_kv_narrow_mx4<T, DP, true, false>)
                                   : (pad ? k_kv_narrow_mx4<T, DP, false, true> : k_kv_narrow_mx4<T, DP, false, false>);
    kernel<<<a.workers, 256, 0, s>>>(a);
}

template <class T>
static void launch_dim(const Attn4 &a, hipStream_t s) {
    const int dim = pad_dim(8 * a.units);
    dim == 64 ? launch<T, 64>(a, s) : dim == 128 ? launch<T, 128>(a, s) : launch<T, 256>(a, s);
}

void launch_narrow_mx4(const Attn4 &a, hipStream_t s) {
    value_type(a.c) == MPT_KV_BF16 ? launch_dim<__bf16>(a, s) : launch_dim<_Float16>(a, s);
    join_narrow(a, s);
}

}  // namespace mptkv
