// Attention kernel over a cache in 4 bits for few rows per key head (decoding):
// tiles of 16 rows, the four waves of a workgroup 32 tokens each of a step of 128,
// as over 16 bits.
//
// Codes go to LDS as they come, keys as codes: a lane reads back a quarter of a
// token's row, which is one E (heads of 128), as the operand of S' = K Q', whose
// dimensions may come in any order if the queries agree on it. Values become 16-bit
// rows on their way into LDS, where they are read by columns.

#include "attention_mx4.h"

namespace mptkv {

template <int DP>
struct Narrow4 {
    static constexpr int M = 16, BN = 128, KK = DP / 32, DT = DP / 16, ROW = 2 * DP, CH = DP / 8;
    static constexpr int C = 1;                                        // a tile's cost besides its steps, in steps
    static constexpr int CODES = DP / 2, CP = CODES / 16, L = CP / 2;  // bytes and pieces of a row of codes; loads of 1 KiB
    static constexpr int E = DP == 256 ? 2 : 1;                        // bytes E of a quarter of a row
    static constexpr int kKeys = 32 * CODES, kValues = 32 * ROW;       // of a wave

    // 16 tokens' pieces fall on different banks.
    __device__ static int k_swizzle(int t) { return DP == 64 ? (t >> 3) & 1 : DP == 128 ? (t >> 2) & 3 : (t >> 1) & 7; }
    // Eight tokens' 32 bytes fall on different banks, and so do the first (second,
    // ...) quarters of four tokens' pieces, which are written at a time.
    __device__ static int v_swizzle(int t) {
        return DP == 64 ? 2 * ((t >> 1) & 3) + ((t >> 2) & 1) : 2 * (t & 7) + ((t >> 1) & 1);
    }
};

template <class T, int DP, bool CAP, bool PAD>
__global__ __launch_bounds__(256, DP == 256 ? 1 : DP == 128 ? 3 : 4) void k_kv_narrow_mx4(Attn4 a) {
    using N = Narrow4<DP>;
    constexpr int M = N::M, BN = N::BN, C = N::C, KK = N::KK, DT = N::DT, ROW = N::ROW, CP = N::CP, L = N::L, E = N::E;
    __shared__ Entries ent;
    __shared__ __attribute__((aligned(1024))) char tiles[4 * (N::kKeys + N::kValues)];
    __shared__ float stat[4][2][16];
    __shared__ __attribute__((aligned(4))) char met_odd[4];
    const mpt_kv_cache &c = a.c;
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), col = lane & 15, quad = lane >> 4;
    const int shift = 31 - __clz(c.page_size), pieces = a.units / 4;
    char *vw = tiles + wave * N::kValues, *kw = tiles + 4 * N::kValues + wave * N::kKeys;

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

        // lane t < 32 knows the page of token t of the wave's part of a step,
        // looked at a step later
        auto find_page = [&](int step) {
            const int t = step * BN + wave * 32 + (lane & 31);
            return t >= range.lo && t < range.hi ? table[t >> shift] : -1;
        };
        const char *kh = a.k + head * a.k_head, *vh = a.v + head * a.v_head;
        const char *keh = a.ke + head * a.ke_head, *veh = a.ve + head * a.ve_head;
        u32x4 kr[L], vr[L];
        uint8_t ks[2][E], vs[L];
        auto load = [&](int step, int pages) __attribute__((always_inline)) {
            const int t0 = step * BN + wave * 32, ln = renewed(lane), piece = ln & (CP - 1);
            if ((unsigned)pages >= (unsigned)c.n_pages) {
                if (t0 + (ln & 31) >= range.lo && t0 + (ln & 31) < range.hi) flag(c, MPT_KV_BAD_PAGE);
                pages = -1;
            }
#pragma unroll
            for (int i = 0; i < L; ++i) {
                const int t = i * (64 / CP) + ln / CP, page = __shfl(pages, t);
                const uint32_t slot = (t0 + t) & (c.page_size - 1);
                const bool there = page >= 0 && (!PAD || piece < pieces);
                kr[i] = mptkv::load<u32x4>(or_zeros(there, kh + 16 * piece + row_at(page, slot, a.k_page, a.k_slot)));
                vr[i] = mptkv::load<u32x4>(or_zeros(there, vh + 16 * piece + row_at(page, slot, a.v_page, a.v_slot)));
                vs[i] = mptkv::load<uint8_t>(or_zeros(there, veh + piece + scale_at(page, slot, a.ve_page, a.ve_slot)));
            }
#pragma unroll
            for (int mt = 0; mt < 2; ++mt) {
                const int t = mt * 16 + (ln & 15), page = __shfl(pages, t);
                const uint32_t slot = (t0 + t) & (c.page_size - 1);
#pragma unroll
                for (int x = 0; x < E; ++x) {
                    const int block = DP == 64 ? (ln >> 4) / 2 : (ln >> 4) * E + x;
                    const bool there = page >= 0 && (!PAD || block < pieces);
                    ks[mt][x] = mptkv::load<uint8_t>(or_zeros(there, keh + block + scale_at(page, slot, a.ke_page, a.ke_slot)));
                }
            }
        };

        int pages = find_page(first);
        load(first, pages);
        pages = find_page(first + 1);
        for (int step = first; step < last; ++step) {
            const int t0 = step * BN + wave * 32, ln = renewed(lane);
            float ku[2][E];
            bool k_odd = false, v_odd = false;
#pragma unroll
            for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                for (int x = 0; x < E; ++x) ku[mt][x] = unit_of(ks[mt][x]), k_odd |= ks[mt][x] == 255;
#pragma unroll
            for (int i = 0; i < L; ++i) {
                const int t = i * (64 / CP) + ln / CP, piece = ln & (CP - 1);
                *(u32x4 *)(kw + t * N::CODES + ((piece ^ N::k_swizzle(t)) << 4)) = kr[i];
                const bool odd = vs[i] == 255;
                v_odd |= odd;
                const float unit = unit_of(vs[i]);
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const uint32_t codes = odd ? 0 : vr[i][w];
                    *(s16x8 *)(vw + t * ROW + (((4 * piece + w) ^ N::v_swizzle(t)) << 4)) = from_codes<T>(codes, odd ? 1.0f : unit);
                }
            }
            met |= __any(v_odd);
            if (step + 1 < last) {
                load(step + 1, pages);
                pages = find_page(step + 2);
            }
            if (t0 >= range.hi || t0 + 32 <= range.lo) continue;   // nothing for this wave
            float s[8];
            s16x8 kf[2][KK];
#pragma unroll
            for (int mt = 0; mt < 2; ++mt) {
                const int t = mt * 16 + (ln & 15);
                const char *row = kw + t * N::CODES;
                uint32_t codes[KK];
                if constexpr (DP == 64) {
                    const uint2 x = *(const uint2 *)(row + (((ln >> 5) ^ N::k_swizzle(t)) << 4) + ((ln >> 4) & 1) * 8);
                    codes[0] = x.x, codes[1] = x.y;
                } else {
#pragma unroll
                    for (int x = 0; x < E; ++x) {
                        const u32x4 y = *(const u32x4 *)(row + (((E * (ln >> 4) + x) ^ N::k_swizzle(t)) << 4));
#pragma unroll
                        for (int w = 0; w < 4; ++w) codes[4 * x + w] = y[w];
                    }
                }
#pragma unroll
                for (int kk = 0; kk < KK; ++kk) kf[mt][kk] = from_codes<T>(codes[kk], ku[mt][kk * E / KK]);
            }
            if (__builtin_expect(__any(k_odd), 0)) {               // scores that are NaN
#pragma unroll
                for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                    for (int kk = 0; kk < KK; ++kk)
                        if (ku[mt][kk * E / KK] == unit_of(255)) kf[mt][kk] = nans<T>();
            }
#pragma unroll
            for (int mt = 0; mt < 2; ++mt) {
                f32x4 x = {0, 0, 0, 0};
#pragma unroll
                for (int kk = 0; kk < KK; ++kk) x = Type<T>::mfma16(kf[mt][kk], qf[kk], x);
#pragma unroll
                for (int i = 0; i < 4; ++i) s[mt * 4 + i] = x[i];
            }
            const bool masked = t0 < all_lo || t0 + 32 > all_hi;
            float top = -INFINITY;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float x = score<CAP>(a, s[i]);
                if (masked) {
                    const int t = t0 + 16 * (i / 4) + 4 * quad + i % 4;
                    x = t >= see_lo && t < see_hi ? x : -INFINITY;
                }
                s[i] = x;
                top = fmaxf(top, x);
            }
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
            typename Type<T>::x8 w;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float x = __builtin_amdgcn_exp2f(s[i] - base);
                l += x;
                w[i] = (T)x;
            }
            const s16x8 pf = __builtin_bit_cast(s16x8, w);
            const int row = ln >> 2;                               // 4 quad + col / 4
            s16x8 vf[DT];
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                const char *q = vw + row * ROW + (((dt * 2 + (ln & 3) / 2) ^ N::v_swizzle(row)) << 4) + (ln & 1) * 8;
                const s16x4 x = read_column4(q), y = read_column4(q + 16 * ROW);
                vf[dt] = __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) o[dt] = Type<T>::mfma16(vf[dt], pf, o[dt]);
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
            nan_values<T>(a, table, shift, veh, max(range.lo, first * BN), min(range.hi, last * BN), see_lo, see_hi,
                          r < rows ? all_l : NAN, whole, d, 64,
                          whole ? a.out + size * (token * a.out_token + hh * a.out_head + d) : (char *)(sums + (wave * 64 + lane) * 4),
                          whole ? 64 * size : 4 * 64 * 16, f32);
        }
        __syncthreads();                      // the LDS is free again
        if (ends && walk.at < walk.end) walk.next(a, ent);
    }
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
