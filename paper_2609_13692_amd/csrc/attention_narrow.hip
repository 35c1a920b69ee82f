// Attention kernel for few rows per key head (decoding): tiles of 16 rows. The
// four waves of a workgroup take 32 tokens each of a step of 128 and are
// joined at the end of the tile.
//
// The work is one pass over keys and values: 2 x 2 D bytes a token against
// 16 x 4 D flops, a few hundredths of what the matrix cores could do, so a
// wave only has to keep loads in flight. Loads take whole rows (neighbouring
// lanes neighbouring bytes: read as the operand of a product needs them, 16
// rows at a time, keys cost the address units four times the lookups and held
// the kernel at 3.8 TB/s); the wave's own LDS then hands out keys as the operand of
// S' = K Q' (16x16x32) and values, transposed, as that of O' += V' P'. A step
// begins with its keys and values going to LDS and the next step's loads, which
// then have all of its products and weights to arrive. No barrier until the
// tile's end.
// 64 tokens over contexts of 700 to 9000, 32 heads on 8 of 128: 248 us, 5.1
// TB/s; one over 1800: 13 us with the join, two launches of dependent reads. The
// join is a launch of its own (4 to 6 us): by the last worker of a tile it took
// 6 us more, for the others' sums then come past the caches of two dies.

#include "attention.h"

namespace mptkv {

template <int DP>
struct Narrow {
    static constexpr int M = 16, BN = 128, KK = DP / 32, DT = DP / 16, ROW = 2 * DP, CH = DP / 8;
    static constexpr int C = 1;                                        // a tile's cost besides its steps, in steps
    static constexpr int kTile = 32 * ROW, L = kTile / 1024;           // a wave's keys of a step; loads of 1 KiB
    static constexpr int kShift = DP == 64 ? 3 : DP == 128 ? 4 : 5;    // log2 CH

    // Eight tokens' 32 bytes, and their 16 bytes, fall on different banks.
    __device__ static int swizzle(int token) { return DP == 64 ? 2 * ((token >> 1) & 3) : 2 * (token & 7); }
};

// Two workgroups to a CU, three with heads of 64, one with heads of 256, and
// registers for no fewer: 37 contexts with heads of 64 21 us, 25 with two.
template <class T, int DP, bool CAP, bool PAD>
__global__ __launch_bounds__(256, DP == 256 ? 1 : DP == 128 ? 2 : 3) void k_kv_narrow(Attn a) {
    using N = Narrow<DP>;
    constexpr int M = N::M, BN = N::BN, C = N::C, KK = N::KK, DT = N::DT, ROW = N::ROW, CH = N::CH, L = N::L;
    __shared__ Entries ent;
    __shared__ __attribute__((aligned(1024))) char tiles[4 * 2 * N::kTile];
    __shared__ float stat[4][2][16];
    __shared__ __attribute__((aligned(4))) char met_odd[4];
    const mpt_kv_cache &c = a.c;
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), col = lane & 15, quad = lane >> 4;
    const int shift = 31 - __clz(c.page_size);
    char *kw = tiles + wave * 2 * N::kTile, *vw = kw + N::kTile;      // the wave's keys and values

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
        s16x8 qf[KK];
        {
            const char *q = a.q + 2 * (token * a.q_token + hh * a.q_head);
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) {
                const int piece = 4 * kk + quad;
                u32x4 x = mptkv::load<u32x4>(or_zeros(r < rows && piece < a.units, q + 16 * piece));
                if (a.flip) x ^= 0x80008000u;
                qf[kk] = __builtin_bit_cast(s16x8, x);
            }
        }
        f32x4 o[DT];
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[dt] = f32x4{0, 0, 0, 0};
        float m = -INFINITY, l = 0;
        bool met = false;                      // an infinity or NaN that was taken out of a product

        // lane t < 32 knows the page of token t of the wave's part of a step.
        // It is looked at only when it is used, a step later: a wait for it
        // here would be one for all loads before it.
        auto find_page = [&](int step) {
            const int t = step * BN + wave * 32 + (lane & 31);
            return t >= range.lo && t < range.hi ? table[t >> shift] : -1;
        };
        const char *kh = a.k + head * a.k_head, *vh = a.v + head * a.v_head;
        u32x4 kr[L], vr[L];
        auto load = [&](int step, int pages) __attribute__((always_inline)) {
            const int t0 = step * BN + wave * 32, ln = renewed(lane), piece = ln & (CH - 1);
            if ((unsigned)pages >= (unsigned)c.n_pages) {
                if (t0 + (ln & 31) >= range.lo && t0 + (ln & 31) < range.hi) flag(c, MPT_KV_BAD_PAGE);
                pages = -1;
            }
            const char *kx = kh + 16 * piece, *vx = vh + 16 * piece;
#pragma unroll
            for (int i = 0; i < L; ++i) {
                const int t = i * (64 / CH) + (ln >> N::kShift), page = __shfl(pages, t);
                const uint32_t slot = (t0 + t) & (c.page_size - 1);
                const bool there = page >= 0 && (!PAD || piece < a.units);
                kr[i] = mptkv::load<u32x4>(or_zeros(there, kx + row_at(page, slot, a.k_page, a.k_slot)));
                vr[i] = mptkv::load<u32x4>(or_zeros(there, vx + row_at(page, slot, a.v_page, a.v_slot)));
            }
        };
        auto put = [&](const u32x4 (&x)[L], char *to) __attribute__((always_inline)) {
            const int ln = renewed(lane);
#pragma unroll
            for (int i = 0; i < L; ++i) {
                const int t = i * (64 / CH) + (ln >> N::kShift);
                *(u32x4 *)(to + t * ROW + (((ln & (CH - 1)) ^ N::swizzle(t)) << 4)) = x[i];
            }
        };

        int pages = find_page(first);
        load(first, pages);
        pages = find_page(first + 1);
        for (int step = first; step < last; ++step) {
            const int t0 = step * BN + wave * 32, ln = renewed(lane);
            put(kr, kw);
            put(vr, vw);
            if (step + 1 < last) {
                load(step + 1, pages);
                pages = find_page(step + 2);
            }
            if (t0 >= range.hi || t0 + 32 <= range.lo) continue;   // nothing for this wave
            float s[8];
            s16x8 kf[2][KK];
#pragma unroll
            for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                for (int kk = 0; kk < KK; ++kk) {
                    const int t = mt * 16 + (ln & 15);
                    kf[mt][kk] = *(const s16x8 *)(kw + t * ROW + (((4 * kk + (ln >> 4)) ^ N::swizzle(t)) << 4));
                }
            __builtin_amdgcn_sched_barrier(0);
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
            // rounded to the values' type for the product, as in the chunk kernel
            typename Type<T>::x8 w;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float x = __builtin_amdgcn_exp2f(s[i] - base);
                l += x;
                w[i] = (T)x;
            }
            const s16x8 pf = __builtin_bit_cast(s16x8, w);
            if (masked) {
                // zeros for infinities and NaN (odd_values)
                uint32_t odd = 0;
#pragma unroll 1
                for (int x = lane; x < 32 * CH; x += 64) odd |= odd8<T>(*(const s16x8 *)(vw + 16 * x));
                if (__any(odd != 0)) {
                    met = true;
#pragma unroll 1
                    for (int x = lane; x < 32 * CH * 8; x += 64)
                        if (!finite16<T>(((const short *)vw)[x])) ((short *)vw)[x] = 0;
                }
            }
            const int row = ln >> 2;                               // 4 quad + col / 4
            s16x8 vf[DT];
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                const char *q = vw + row * ROW + (((dt * 2 + (ln & 3) / 2) ^ N::swizzle(row)) << 4) + (ln & 1) * 8;
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
        float odd = 0;
#pragma unroll
        for (int k = 0; k < DT / 4; ++k) {
            const int dt = k * 4 + wave;
            f32x4 x = {0, 0, 0, 0};
#pragma unroll
            for (int w = 0; w < 4; ++w) x += f[w] * *(const f32x4 *)(tiles + (2 * w + 1) * N::kTile + dt * 1024 + lane * 16);
            odd += not_finite(x);
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
        if (__builtin_expect(__any(*(const uint32_t *)met_odd | (odd != 0)), 0)) {
            const bool whole = starts && ends, f32 = !whole || a.out_f32;
            const int d = wave * 16 + 4 * quad, size = f32 ? 4 : 2;
            odd_values<T, DT / 4>(a, table, shift, vh, max(range.lo, first * BN), min(range.hi, last * BN), see_lo, see_hi,
                          r < rows ? all_l : NAN, whole, d, 64,
                          whole ? a.out + size * (token * a.out_token + hh * a.out_head + d) : (char *)(sums + (wave * 64 + lane) * 4),
                          whole ? 64 * size : 4 * 64 * 16, f32);
        }
        __syncthreads();                      // the LDS is free again
        if (ends && walk.at < walk.end) walk.next(a, ent);
    }
}

// Joins the parts of a tile: workgroup (w, 16 dimensions). The waves share the
// parts, four at a time in flight (one after the other, their latencies would
// add up to more than the attention of a short context).
template <class T, int DP>
__global__ __launch_bounds__(256) void k_kv_join_narrow(Attn a) {
    constexpr int M = 16;
    __shared__ float stat[4][2][16];
    __shared__ f32x4 other[4][64];
    const int w = blockIdx.x, dt = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, quad = lane >> 4;
    const Part part = a.parts[w];
    if (part.count == 0) return;
    // part i: worker w - 1 + i; the first one's second slot, the others' first
    auto sums = [&](int i) { return a.sums + ((int64_t)(w - 1 + i) * 2 + (i == 0)) * (M * (DP + 2)); };
    float m = -INFINITY, l = 0;
    f32x4 o = {0, 0, 0, 0};
    for (int i = wave; i < part.count; i += 16) {
        float pm[4], pl[4];
        f32x4 po[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const bool there = i + 4 * k < part.count;
            const float *p = sums(there ? i + 4 * k : i);
            pm[k] = there ? p[M * DP + col] : -INFINITY;
            pl[k] = p[M * DP + 16 + col];
            po[k] = *(const f32x4 *)(p + (dt * 64 + lane) * 4);
        }
        float now = m;
#pragma unroll
        for (int k = 0; k < 4; ++k) now = fmaxf(now, pm[k]);
        const float base = now == -INFINITY ? 0.0f : now, keep = __builtin_amdgcn_exp2f(m - base);
        l *= keep;
        o *= keep;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float f = __builtin_amdgcn_exp2f(pm[k] - base);
            if (i + 4 * k < part.count) {
                l += f * pl[k];
                o += f * po[k];
            }
        }
        m = now;
    }
    if (quad == 0) stat[wave][0][col] = m, stat[wave][1][col] = l;
    other[wave][lane] = o;
    __syncthreads();
    if (wave) return;
    float top = -INFINITY;
#pragma unroll
    for (int k = 0; k < 4; ++k) top = fmaxf(top, stat[k][0][col]);
    const float base = top == -INFINITY ? 0.0f : top;
    l = 0;
    o = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float f = __builtin_amdgcn_exp2f(stat[k][0][col] - base);
        l += f * stat[k][1][col];
        o += f * other[k][lane];
    }
    o = odd_parts(o, part.count, [&](int i) { return sums(i) + (dt * 64 + lane) * 4; });
    const int rows = part.n * a.group, r = part.tile * M + col;
    if (r >= rows) return;
    const int j = token_of(a, r), d = dt * 16 + 4 * quad;
    const int64_t token = part.q0 + j, h = (int64_t)part.head * a.group + r - j * a.group;
    if (a.lse && dt == 0 && quad == 0)
        a.lse[token * a.heads + h] = l == 0 ? -INFINITY : 0.693147180559945f * (top + __builtin_amdgcn_logf(l));
    if (d < 8 * a.units) store4<T>(a, token * a.out_token + h * a.out_head + d, l == 0 ? f32x4{0, 0, 0, 0} : o * (1.0f / l));
}

template <class T, int DP>
static void launch_join(const Attn &a, hipStream_t s) {
    mptlib::LaunchScope scope("k_kv_join_narrow", a.workers, s);
    k_kv_join_narrow<T, DP><<<dim3(a.workers, (a.units + 1) / 2), 256, 0, s>>>(a);
}

template <class T, int DP>
static void launch(const Attn &a, hipStream_t s) {
    {
        mptlib::LaunchScope scope("k_kv_narrow", (double)a.n_tokens * a.heads, s);
        const bool pad = 8 * a.units < DP;
        const auto kernel = a.cap != 0 ? (pad ? k_kv_narrow<T, DP, true, true> : k_kv_narrow<T, DP, true, false>)
                                       : (pad ? k_kv_narrow<T, DP, false, true> : k_kv_narrow<T, DP, false, false>);
        kernel<<<a.workers, 256, 0, s>>>(a);
    }
    launch_join<T, DP>(a, s);
}

template <class T>
static void launch_dim(const Attn &a, hipStream_t s) {
    const int dim = pad_dim(8 * a.units);
    dim == 64 ? launch<T, 64>(a, s) : dim == 128 ? launch<T, 128>(a, s) : launch<T, 256>(a, s);
}

void join_narrow(const Attn &a, hipStream_t s) {
    const int dim = pad_dim(8 * a.units);
    if (value_type(a.c) == MPT_KV_BF16)
        dim == 64 ? launch_join<__bf16, 64>(a, s) : dim == 128 ? launch_join<__bf16, 128>(a, s) : launch_join<__bf16, 256>(a, s);
    else
        dim == 64 ? launch_join<_Float16, 64>(a, s) : dim == 128 ? launch_join<_Float16, 128>(a, s) : launch_join<_Float16, 256>(a, s);
}

void launch_narrow(const Attn &a, hipStream_t s) {
    if (a.c.dtype == MPT_KV_BF16)
        launch_dim<__bf16>(a, s);
    else
        launch_dim<_Float16>(a, s);
}

}  // namespace mptkv
