// Attention kernel over a cache in 4 bits for many rows per key head (chunks of
// new tokens): tiles of 128 or 256 rows, 32 to each of the four or eight waves,
// with the products of the kernel over 16 bits (scores transposed, weights as the
// second operand of O' += V' P' as they lie).
//
// A workgroup turns each tile of 64 tokens into 16 bits once, for all of its rows:
// a thread takes one piece of 32 elements of keys or of values (heads of 128, eight
// waves), loaded a tile ahead, and writes them to LDS where its products read them.
// Two tiles of keys and two of values are there at a time.

#include "attention_mx4.h"

#include <type_traits>

namespace mptkv {

#define INLINE __attribute__((always_inline))

template <int DP, int WAVES>
struct Wide4 {
    static constexpr int kThreads = 64 * WAVES, BN = 64, KK = DP / 16, DT = DP / 32, ROW = 2 * DP;
    static constexpr int kTile = BN * ROW, CP = DP / 32, kPieces = BN * CP;   // bytes in 16 bits; pieces of a row, of a tile
    static constexpr int L = (2 * kPieces + kThreads - 1) / kThreads;          // pieces of keys and values per thread
    static constexpr int C = 8;                                                // a tile's cost besides its steps, in steps
    static constexpr int kAhead = DP == 256 ? 3 : 2;                           // operands read from LDS ahead of their products

    // Where the 16-byte pieces of a token's row lie: keys so that eight tokens'
    // pieces, values so that four tokens' 64 bytes, fall on all banks, and so do
    // the first (second, ...) quarters of 16 threads' elements, which are written at
    // a time; equal for tokens 8 apart (values) and 32 (keys).
    __device__ static int k_swizzle(int t) { return DP == 64 ? (t >> 1) & 7 : DP == 128 ? t & 15 : t & 7; }
    __device__ static int v_swizzle(int t) { return DP == 64 ? 5 * ((t >> 1) & 1) + 2 * ((t >> 2) & 1) : 5 * (t & 3); }
};

template <class T, int DP, int WAVES, bool CAP>
__global__ __launch_bounds__(64 * WAVES, DP == 256 ? 1 : 2) void k_kv_wide_mx4(Attn4 a) {
    using W = Wide4<DP, WAVES>;
    constexpr int M = 32 * WAVES, THREADS = W::kThreads, BN = W::BN, KK = W::KK, DT = W::DT, ROW = W::ROW, L = W::L, TILE = W::kTile;
    constexpr int C = W::C, AHEAD = W::kAhead, CP = W::CP;
    __shared__ Entries ent;
    __shared__ __attribute__((aligned(1024))) char keys[2 * TILE], values[2 * TILE];
    const mpt_kv_cache &c = a.c;
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), col = lane & 31, half = lane >> 5;
    const int shift = 31 - __clz(c.page_size), pieces = a.units / 4;
    // Where a lane reads its operands: rows of 32 tokens of keys, 8 of values.
    const uint32_t k_at = lds_address(keys) + col * ROW + 16 * (half ^ W::k_swizzle(col));
    const int v_of = 4 * half + (lane & 15) / 4;
    const uint32_t v_at = lds_address(values) + v_of * ROW + (lane & 1) * 8 + 16 * ((((lane >> 4) & 1) * 2 + (lane & 3) / 2) ^ W::v_swizzle(v_of));
    bool lost = false;                         // a page id outside the pool
    // A thread's pieces, and where their elements go: the first quarter of each.
    auto is_key = [&](int i) INLINE { return i * THREADS + wave * 64 < W::kPieces; };
    auto has_piece = [&](int i) INLINE { return i * THREADS + wave * 64 < 2 * W::kPieces; };
    auto piece_of = [&](int i) INLINE { return (i * THREADS + renewed(tid)) & (CP - 1); };
    auto token_of_piece = [&](int i) INLINE { return (int)((uint32_t)((i * THREADS + renewed(tid)) & (W::kPieces - 1)) / CP); };
    uint32_t put_at[L];
#pragma unroll
    for (int i = 0; i < L; ++i) {
        const int t = token_of_piece(i), swizzle = is_key(i) ? W::k_swizzle(t) : W::v_swizzle(t);
        put_at[i] = lds_address(is_key(i) ? keys : values) + t * ROW + ((4 * piece_of(i) ^ swizzle) << 4);
    }

    Walk<M, BN, C> walk;
    if (!walk.begin(a, ent, 4)) return;

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
        const int rows = n * a.group, row_base = tile * M + wave * 32;
        const int32_t *table = c.table + (int64_t)uniform(ent.slot[e]) * c.max_pages;
        const bool active = row_base < rows;

        // Turn j, between the barriers in tiles j - 1 and j, makes the keys of tile
        // j + 1 and the values of tile j: of each thread L pieces, keys first, a wave's
        // all of one kind. Their codes are loaded a turn before, their pages' ids one
        // before that.
        // Tokens that the tile does not reach are read as others of it (their scores are
        // masked, and a weight of 0 times a finite value is 0), and so are pieces past the
        // row's end (their queries are 0). A page id outside the pool becomes the last
        // page, and is reported.
        // A tile's tokens are 64 slots of a page, or pages are of the tile: a thread's
        // places in them are the same for all tiles but for what is uniform.
        const char *from_codes_of[L], *from_scales_of[L];
#pragma unroll
        for (int i = 0; i < L; ++i) {
            const bool key = is_key(i);
            const int piece = min(piece_of(i), pieces - 1);
            const uint32_t slot = token_of_piece(i) & (c.page_size - 1);
            from_codes_of[i] = at((key ? a.k + head * a.k_head : a.v + head * a.v_head) + 16 * piece, slot, key ? a.k_slot : a.v_slot);
            from_scales_of[i] = at((key ? a.ke + head * a.ke_head : a.ve + head * a.ve_head) + piece, slot, key ? a.ke_slot : a.ve_slot);
        }
        u32x4 codes[L];
        uint8_t scale[L];
        int ids[L];
        bool met = false;                      // a NaN among the values
        auto fetch_ids = [&](int j) INLINE {
#pragma unroll
            for (int i = 0; i < L; ++i) {
                const int t = (j + is_key(i)) * BN + token_of_piece(i);
                ids[i] = table[max(0, max(range.lo, min(range.hi - 1, t))) >> shift];
            }
        };
        auto fetch = [&](int j) INLINE {
#pragma unroll
            for (int i = 0; i < L; ++i) {
                if (!has_piece(i)) break;
                const bool key = is_key(i);
                const uint32_t id = min((uint32_t)ids[i], (uint32_t)c.n_pages - 1);
                lost |= id != (uint32_t)ids[i] && range.hi > 0;
                const uint64_t slot = (uint32_t)((j + key) * BN) & (c.page_size - 1);
                codes[i] = mptkv::load<u32x4>(at(from_codes_of[i], id, key ? a.k_page : a.v_page) + slot * (key ? a.k_slot : a.v_slot));
                scale[i] = mptkv::load<uint8_t>(at(from_scales_of[i], id, key ? a.ke_page : a.ve_page) + slot * (key ? a.ke_slot : a.ve_slot));
            }
        };
        // odd: whether the values' tile, j, is of odd number from `first` on (the keys' is the other kind)
        auto make = [&](int odd) INLINE {
#pragma unroll
            for (int i = 0; i < L; ++i) {
                if (!has_piece(i)) break;
                const bool key = is_key(i);
                const uint32_t to = put_at[i] + (odd ^ key ? TILE : 0);
                const float unit = unit_of(scale[i]);
                s16x8 x[4];
#pragma unroll
                for (int w = 0; w < 4; ++w) x[w] = from_codes<T>(codes[i][w], unit);
                if (__builtin_expect(__any(scale[i] > kMaxScale<T>), 0)) {
                    if (scale[i] > kMaxScale<T>) {
                        const s16x8 y = key ? nans<T>() : s16x8{0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
                        for (int w = 0; w < 4; ++w) x[w] = y;
                        met |= !key;
                    }
                }
#pragma unroll
                for (int w = 0; w < 4; ++w) to_lds(to ^ w << 4, x[w]);
            }
        };
        fetch_ids(first - 1);
        // queries of the wave's rows as operands, and what each may see
        s16x8 qf[KK];
        const int r0 = row_base + col, rr = min(r0, rows - 1), j0 = token_of(a, rr), p0 = len - n + j0;
        const int see_hi = a.causal ? min(len, p0 + 1) : len, see_lo = a.window ? max(begin, p0 + 1 - a.window) : begin;
        const char *q = a.q + 2 * ((int64_t)(q0 + j0) * a.q_token + ((int64_t)head * a.group + rr - j0 * a.group) * a.q_head);
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
            const int piece = 2 * kk + half;
            u32x4 x = mptkv::load<u32x4>(or_zeros(r0 < rows && piece < a.units, q + 16 * piece));
            if (a.flip) x ^= 0x80008000u;
            qf[kk] = __builtin_bit_cast(s16x8, x);
            // wide heads: in the registers that only products read, where they stay
            if constexpr (DP == 256) asm volatile("" : "+a"(qf[kk]));
        }
        // tokens that all rows of the wave, and of the tile, see
        int wave_lo, wave_hi, tile_lo, tile_hi;
        seen_by_all(a, n, len, begin, min(row_base, rows - 1), min(row_base + 31, rows - 1), wave_lo, wave_hi);
        seen_by_all(a, n, len, begin, tile * M, min(tile * M + M, rows) - 1, tile_lo, tile_hi);

        f32x16 o[DT], s0, s1;
        s16x8 pf[2];
        float m = -INFINITY, l = 0;
        pf[0] = pf[1] = s16x8{0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[dt][r] = 0;

        // The products of a step, in groups that the compiler keeps in order:
        // an operand from LDS (read some groups ahead), its product, and beside
        // it a share of the step's other work.
        // S' = K Q' of 32 tokens (base: where the lane's first operand lies; kb, vb: bytes
        // from there, constants)
        auto multiply = [&](uint32_t base, int kb, f32x16 &s, auto beside) INLINE {
            s16x8 kf[AHEAD + 1];
            auto read = [&](int kk) INLINE { kf[kk % (AHEAD + 1)] = from_lds<s16x8>((base ^ 32 * kk) + kb); };
#pragma unroll
            for (int kk = 0; kk < AHEAD; ++kk) read(kk);
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) {
                if (kk + AHEAD < KK) read(kk + AHEAD);
                s = Type<T>::mfma32(kf[kk % (AHEAD + 1)], qf[kk], kk ? s : f32x16{0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0});
                beside(kk);
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        // O' += V' P' of 32 tokens
        auto add = [&](uint32_t base, int vb, auto beside) INLINE {
            s16x8 vf[AHEAD + 1];
            auto read = [&](int i) INLINE {
                const uint32_t x = (base ^ 64 * (i % DT)) + vb + (i / DT) * 16 * ROW;
                const s16x4 y = read_column4(x), z = read_column4(x + 8 * ROW);
                vf[i % (AHEAD + 1)] = __builtin_shufflevector(y, z, 0, 1, 2, 3, 4, 5, 6, 7);
            };
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) read(i);
#pragma unroll
            for (int i = 0; i < 2 * DT; ++i) {
                if (i + AHEAD < 2 * DT) read(i + AHEAD);
                o[i % DT] = Type<T>::mfma32(vf[i % (AHEAD + 1)], pf[i / DT], o[i % DT]);
                beside(i);
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        auto nothing = [](int) INLINE {};
        // One step of 32 tokens from t0 with scores x: products with the values
        // of the step before beside this step's maximum, scores of the next
        // step beside this step's weights.
        auto step32 = [&](auto all_seen, f32x16 &x, f32x16 &next, int t0, uint32_t k_base, int k_next, uint32_t v_base, int v_before) INLINE {
            if constexpr (CAP) {
#pragma unroll
                for (int r = 0; r < 16; ++r) x[r] = score<true>(a, x[r]);
            }
            if (!all_seen && (t0 < wave_lo || t0 + 32 > wave_hi)) {
                const int before = t0 + 4 * renewed(half), lo = see_lo - before, hi = see_hi - before;
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int t = 8 * (r / 4) + r % 4;
                    if (!(t >= lo && t < hi)) x[r] = -INFINITY;
                }
            }
            __builtin_amdgcn_s_setprio(1);
            float top = -INFINITY;
            add(v_base, v_before, [&](int i) INLINE {
                constexpr int N = 8 / DT;
#pragma unroll
                for (int y = i * N; y < i * N + N; ++y) top = fmaxf(top, x[y]);
            });
            if constexpr (!CAP) top *= a.factor;
            if (__any(top > m + 8.0f)) {
                const float now = fmaxf(m, fmaxf(top, __shfl_xor(top, 32)));
                const float keep = now == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - now);
                if (!__all(m == -INFINITY)) {                         // else the sums are zeros
                    l *= keep;
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                        for (int r = 0; r < 16; ++r) o[dt][r] *= keep;
                }
                m = now;
            }
            const float base = m == -INFINITY ? 0.0f : m;
            // Weights are rounded to the 16-bit type, so that both operands of the
            // product are of one, as over 16 bits.
            float even = 0;
            u32x4 packed[2];
            multiply(k_base, k_next, next, [&](int i) INLINE {
                constexpr int N = 16 / KK;
#pragma unroll
                for (int r = i * N; r < i * N + N; ++r) {
                    const float w = __builtin_amdgcn_exp2f(CAP ? x[r] - base : __builtin_fmaf(x[r], a.factor, -base));
                    l += w;
                    if (r % 2)
                        packed[r / 8][r % 8 / 2] = pack<T>(even, w);
                    else
                        even = w;
                }
            });
            pf[0] = __builtin_bit_cast(s16x8, packed[0]), pf[1] = __builtin_bit_cast(s16x8, packed[1]);
            __builtin_amdgcn_s_setprio(0);
        };

        __syncthreads();                       // the previous rows' products have read their buffers
        fetch(first - 1);
        fetch_ids(first);
        make(1);                               // keys of the first tile, some values as those before it
        fetch(first);
        fetch_ids(first + 1);
        make(0);
        fetch(first + 1);
        fetch_ids(first + 2);
        __syncthreads();
        if (active) multiply(k_at, 0, s0, nothing);
        for (int step = first; step < last;) {
            if constexpr (DP < 256) {
                // Two tiles whose tokens every row of the tile sees, in places that are
                // constants.
                const int t0 = step * BN;
                if (((step - first) & 1) == 0 && step + 2 <= last && t0 >= tile_lo && t0 + 2 * BN <= tile_hi) {
                    auto turn = [&](auto r_) INLINE {
                        constexpr int R = decltype(r_)::value, O = 1 - R;
                        if (active) step32(std::true_type(), s0, s1, 0, k_at, R * TILE + 32 * ROW, v_at, O * TILE + 32 * ROW);
                        __syncthreads();
                        make(O);
                        fetch(step + R + 2);
                        fetch_ids(step + R + 3);
                        if (active) step32(std::true_type(), s1, s0, 0, k_at, O * TILE, v_at, R * TILE);
                    };
                    turn(std::integral_constant<int, 0>());
                    turn(std::integral_constant<int, 1>());
                    step += 2;
                    continue;
                }
            }
            const int odd = (step - first) & 1, now = odd * TILE, other = TILE - now;
            // its two halves by one piece of code: a call with few steps waits for its
            // instructions more than for anything else
#pragma unroll 1
            for (int h = 0; h < 2; ++h) {
                if (active) {
                    step32(std::false_type(), s0, s1, step * BN + 32 * h, k_at + (h ? other : now + 32 * ROW), 0,
                           v_at + (h ? now : other + 32 * ROW), 0);
                    s0 = s1;
                }
                if (h) break;
                __syncthreads();
                make(!odd);
                fetch(step + 2);
                fetch_ids(step + 3);
            }
            ++step;
        }
        if (active) add(v_at + ((last - 1 - first) & 1) * TILE + 32 * ROW, 0, nothing);

        float *sums = a.sums + ((int64_t)uniform(walk.worker) * 2 + (from == 0)) * (M * (DP + 2)) + wave * 32 * DP;
        const float sum = l + __shfl_xor(l, 32);
        if (starts && ends) {
            const int r = row_base + renewed(col);
            if (r < rows) {
                const float scale = sum == 0 ? 0.0f : 1.0f / sum;
                const int j = token_of(a, r);
                const int64_t token = q0 + j, hq = (int64_t)head * a.group + r - j * a.group;
                if (a.lse && half == 0)
                    a.lse[token * a.heads + hq] = sum == 0 ? -INFINITY : 0.693147180559945f * (m + __builtin_amdgcn_logf(sum));
                const int64_t to = token * a.out_token + hq * a.out_head + 4 * half;
                auto store = [&](auto f32) INLINE {
                    char *row = a.out + (f32 ? 4 : 2) * to;
#pragma unroll
                    for (int x = 0; x < DT * 4; ++x) {
                        if (x >= a.units) break;
                        const f32x16 &y = o[x / 4];
                        const int i = x % 4 * 4;
                        put4<T, f32>(row, 8 * x, f32x4{y[i], y[i + 1], y[i + 2], y[i + 3]} * scale);
                    }
                };
                a.out_f32 ? store(std::true_type()) : store(std::false_type());
            }
        } else {
            // unnormalised sums, in the order of the registers
            if (active) {
#pragma unroll
                for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                    for (int r = 0; r < 16; r += 4)
                        *(f32x4 *)(sums + ((dt * 4 + r / 4) * 64 + lane) * 4) = f32x4{o[dt][r], o[dt][r + 1], o[dt][r + 2], o[dt][r + 3]};
                (sums - wave * 32 * DP + M * DP + wave * 64)[lane] = half ? sum : m;
            }
            if (!starts && tid == 0) {
                const int workers = walk.second_of(range.count);
                if (workers) a.parts[walk.worker] = Part{workers, e + walk.base, head, tile, q0, n};
            }
        }
        if (__builtin_expect(__syncthreads_or(met), 0)) {
            const bool whole = starts && ends, f32 = !whole || a.out_f32;
            const int size = f32 ? 4 : 2;
            if (active)
                nan_values<T>(a, table, shift, a.ve + head * a.ve_head, max(range.lo, first * BN), min(range.hi, last * BN), see_lo, see_hi,
                              r0 < rows ? sum : NAN, whole, 4 * half, 8,
                              whole ? a.out + size * ((int64_t)(q0 + j0) * a.out_token + ((int64_t)head * a.group + rr - j0 * a.group) * a.out_head + 4 * half)
                                    : (char *)(sums + lane * 4),
                              whole ? 8 * size : 64 * 16, f32);
        }
        if (ends && walk.at < walk.end) walk.next(a, ent);
    }
    if (lost) flag(c, MPT_KV_BAD_PAGE);
}

template <class T, int DP, int WAVES>
static void launch(const Attn4 &a, hipStream_t s) {
    mptlib::LaunchScope scope("k_kv_wide_mx4", (double)a.n_tokens * a.heads, s);
    if (a.cap != 0)
        k_kv_wide_mx4<T, DP, WAVES, true><<<a.workers, 64 * WAVES, 0, s>>>(a);
    else
        k_kv_wide_mx4<T, DP, WAVES, false><<<a.workers, 64 * WAVES, 0, s>>>(a);
}

template <class T>
static void launch_dim(const Attn4 &a, int waves, hipStream_t s) {
    const int dim = pad_dim(8 * a.units);
    if (dim == 64)
        waves == 8 ? launch<T, 64, 8>(a, s) : launch<T, 64, 4>(a, s);
    else if (dim == 128)
        waves == 8 ? launch<T, 128, 8>(a, s) : launch<T, 128, 4>(a, s);
    else
        launch<T, 256, 4>(a, s);
}

void launch_wide_mx4(const Attn4 &a, int waves, hipStream_t s) {
    value_type(a.c) == MPT_KV_BF16 ? launch_dim<__bf16>(a, waves, s) : launch_dim<_Float16>(a, waves, s);
    join_wide(a, waves, s);
}

}  // namespace mptkv
