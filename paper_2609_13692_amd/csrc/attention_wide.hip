// Attention kernel for many rows per key head (chunks of new tokens): tiles of
// 128 or 256 rows, 32 to each of the four or eight waves.
//
// Scores are formed transposed, S' = K Q', with 32x32x16 products: lane l then
// holds query l % 32 and 16 of 32 tokens, so the running maximum and sum of a
// query are values of its own two lanes, and the weights, rounded, are the
// second operand of O' += V' P' as they lie (the tokens of a product may come
// in any order if both operands agree on it). Keys and values go from memory
// to LDS directly, one to three tiles of 64 tokens ahead of the products;
// values are read back by the transposing LDS loads.
//
// The maximum that weights are taken against is moved only when a score
// exceeds it by 2^8: products with weights up to 256 are as exact, and the
// sums are rescaled a few times per row instead of at every step.
//
// What bounds it is the instructions that the vector units issue beside the
// products: 16 exponentials and 56 others for 32 tokens of a wave with heads
// of 128, against 16 products, with two waves to a SIMD. So tiles that nothing
// is masked in run in groups, where places in LDS are constants, page ids are
// clamped instead of selected by, and offsets into the pool have 32 bits; one
// more instruction per operand read cost 3%. Chunks of 1024 tokens over 16k,
// 32 heads on 8 of 128: 1140 us without such groups, 1053 with them.
//
// What bounds calls with few steps is the fetching of instructions, each of
// which a workgroup meets for the first time. So outside the groups one piece
// of code serves both halves of a tile, and one the loads of all tiles: the
// kernels went from 70 to 47 KB (heads of 256) and from 52 to 40 (128), nine
// chunks over up to 4099 tokens with a window from 101 to 92 us, 25 ragged
// chunks over up to 8400 from 816 to 775 (797 TFLOP/s), the chunks above to
// 1031 (1021 TFLOP/s; a library product of 8192^3 reaches 1210 on this card).
// Infinities among the values at the tile's end instead of at its steps: 46 and
// 43 KB with fewer registers put into memory; 91.9 to 86.5, 781 to 756 and 1039 to
// 1021 us, both sides on one card.

#include "attention.h"

#include <type_traits>

namespace mptkv {

// Lambdas whose bodies the compiler would rather call, with every register
// that they touch put into memory.
#define INLINE __attribute__((always_inline))

template <int DP, int WAVES>
struct Wide {
    static constexpr int kThreads = 64 * WAVES, BN = 64, KK = DP / 16, DT = DP / 32, ROW = 2 * DP, CH = DP / 8;
    static constexpr int kTile = BN * ROW, kLoads = kTile / (16 * kThreads);   // 16-byte loads per thread, of keys or values
    static constexpr int kStride = kThreads / CH;                       // tokens between a thread's loads
    // Tiles of keys (and of values) in LDS: two where two workgroups share a
    // CU or rows are long, else four. Page ids are fetched for twice as many.
    static constexpr int C = 8;                                        // a tile's cost besides its steps, in steps
    static constexpr int S = WAVES == 8 ? 4 : 2, IDS = 2 * S;
    // Operands read from LDS ahead of their products (heads of 128: one 1118
    // us, two 1053, three, with more registers than there are, 1163); with one
    // wave to a SIMD nothing else covers the latency.
    static constexpr int kAhead = DP == 256 ? 3 : 2;

    // Where the 16-byte pieces of a token's row lie: keys so that eight
    // tokens' pieces, values so that four tokens' 64 bytes, fall on all banks;
    // equal for tokens kStride apart, so that a thread loads one piece of its
    // tokens.
    __device__ static int k_swizzle(int token) { return DP == 64 ? (token >> 1) & 7 : DP == 128 ? token & 15 : token & 7; }
    __device__ static int v_swizzle(int token) { return DP == 64 ? 4 * ((token >> 1) & 1) : 4 * (token & 3); }
};

template <class T, int DP, int WAVES, bool CAP>
__global__ __launch_bounds__(64 * WAVES, DP == 256 ? 1 : 2) void k_kv_wide(Attn a) {
    using W = Wide<DP, WAVES>;
    constexpr int M = 32 * WAVES, THREADS = W::kThreads, BN = W::BN, KK = W::KK, DT = W::DT, ROW = W::ROW, CH = W::CH, L = W::kLoads, TILE = W::kTile;
    constexpr int C = W::C, S = W::S, IDS = W::IDS, AHEAD = W::kAhead;
    __shared__ Entries ent;
    __shared__ __attribute__((aligned(1024))) char keys[S * TILE], values[S * TILE];
    __shared__ __attribute__((aligned(256))) int ids[WAVES * IDS * BN];       // each wave its own
    const mpt_kv_cache &c = a.c;
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), col = lane & 31, half = lane >> 5;
    const int shift = 31 - __clz(c.page_size);
    const uint32_t k_lds = uniform((int)(lds_address(keys) + wave * 1024)), v_lds = uniform((int)(lds_address(values) + wave * 1024));
    const uint32_t id_lds = uniform((int)(lds_address(ids) + wave * IDS * BN * 4));
    // The thread's tokens of a tile are kStride apart from `own` on: its pieces
    // of their rows, and with them the first one's place in a page whose slots
    // are counted from the tile's first (a tile is a part of a page, or pages
    // are of the tile), for pools whose offsets have 32 bits.
    const int own = tid / CH, kp = (tid % CH) ^ W::k_swizzle(own), vp = (tid % CH) ^ W::v_swizzle(own);
    const uint32_t k_near = (uint32_t)(own & (c.page_size - 1)) * a.k_slot + kp, v_near = (uint32_t)(own & (c.page_size - 1)) * a.v_slot + vp;
    const bool near = a.near && a.units == CH;
    // Where a lane reads its operands: rows of 32 tokens of keys, 8 of values.
    // Rows are as long as the swizzle reaches, so a piece's place is the
    // first's with some bits turned over.
    const uint32_t k_at = lds_address(keys) + col * ROW + 16 * (half ^ W::k_swizzle(col));
    const int v_of = 4 * half + (lane & 15) / 4;
    const uint32_t v_at = lds_address(values) + v_of * ROW + (lane & 1) * 8 + 16 * ((((lane >> 4) & 1) * 2 + (lane & 3) / 2) ^ W::v_swizzle(v_of));
    bool lost = false;                         // a page id outside the pool

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

        // The pages of a tile's tokens (of some token of the range for those
        // outside it, whose loads take zeros), on their way before the queries.
        const char *kh = a.k + head * a.k_head, *vh = a.v + head * a.v_head;
        auto fetch_ids = [&](int step) INLINE {
            const int t = max(0, max(range.lo, min(range.hi - 1, step * BN + lane)));
            load_lds4(table + (t >> shift), id_lds + ((step - first) & (IDS - 1)) * BN * 4);
        };
#pragma unroll
        for (int i = 0; i < S; ++i) fetch_ids(first + i);
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

        // The keys or values of a tile. What places them is formed here, not
        // kept: the main loop takes every register.
        auto load = [&](int step, const char *rows0, auto swizzle, uint32_t page_stride, uint32_t slot_stride, uint32_t lds) INLINE {
            const int at = renewed(tid), token = at / CH, piece = (at % CH) ^ swizzle(token);
            const bool in = piece < a.units;
            const char *tile0 = rows0 + 16 * piece + ((uint64_t)((uint32_t)(step * BN) & (c.page_size - 1)) * slot_stride << 4);
            const int *page = ids + (wave * IDS + ((step - first) & (IDS - 1))) * BN + token;
#pragma unroll
            for (int i = 0; i < L; ++i) {
                const int id = page[i * W::kStride];
                const bool there = (unsigned)id < (unsigned)c.n_pages;
                const bool see = (unsigned)(step * BN + i * W::kStride + token - range.lo) < (unsigned)(range.hi - range.lo);
                lost |= see && !there;
                const uint32_t slot = (uint32_t)(i * W::kStride + token) & (c.page_size - 1);
                load_lds16(or_zeros(see && there && in, tile0 + row_at(id, slot, page_stride, slot_stride)),
                           lds + ((step - first) & (S - 1)) * TILE + i * 16 * THREADS);
            }
        };
        auto load_keys = [&](int step) INLINE { load(step, kh, [](int t) INLINE { return W::k_swizzle(t); }, a.k_page, a.k_slot, k_lds); };
        auto load_values = [&](int step) INLINE { load(step, vh, [](int t) INLINE { return W::v_swizzle(t); }, a.v_page, a.v_slot, v_lds); };
        // The same for whole tiles (CH pieces a row) of pools whose offsets have 32 bits. A page
        // id outside the pool becomes the last page, and is reported.
        auto fetch_ids_near = [&](int step) INLINE {
            const int t = min(range.hi - 1, step * BN + renewed(lane));
            load_lds4(table, (uint32_t)(t >> shift) * 4, id_lds + ((step - first) & (IDS - 1)) * BN * 4);
        };
        auto load_near = [&](int step, const char *rows0, uint32_t slot, uint32_t page_stride, uint32_t slot_stride, uint32_t lds) INLINE {
            const int *page = ids + (wave * IDS + ((step - first) & (IDS - 1))) * BN + own;
#pragma unroll
            for (int i = 0; i < L; ++i) {
                const uint32_t id = page[i * W::kStride], there = min(id, (uint32_t)c.n_pages - 1);
                lost |= id != there;
                // own is less than kStride: the other tokens' bits of a slot are the same for all lanes
                const char *from = rows0 + ((uint64_t)((uint32_t)(step * BN + i * W::kStride) & (c.page_size - 1)) * slot_stride << 4);
                load_lds16(from, (__umul24(there, page_stride) + slot) << 4, lds + i * 16 * THREADS);
            }
        };
        // The products of a step, in groups that the compiler keeps in order:
        // an operand from LDS (read some groups ahead), its product, and beside
        // it a share of the step's other work.
        // S' = K Q' of 32 tokens (base: where the lane's first
        // operand lies; kb, vb: bytes from there, constants)
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
            // between the two waves of a SIMD, the one with products to issue
            // goes before the one that forms addresses: 2% of the kernel
            __builtin_amdgcn_s_setprio(1);
            float top = -INFINITY;
            add(v_base, v_before, [&](int i) INLINE {
                constexpr int E = 8 / DT;
#pragma unroll
                for (int y = i * E; y < i * E + E; ++y) top = fmaxf(top, x[y]);
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
            // Weights are rounded to the values' type, so that both operands of
            // the product are of one: with 32-bit weights it would take three
            // products of split weights or go without the matrix units. Against
            // 64 bits the outputs are off by 0.0023 in bfloat16 (0.0017 of it
            // their own rounding) and 0.00028 in float16 (0.00021). The sum
            // takes them as they are, for the logarithm.
            float even = 0;
            u32x4 packed[2];
            multiply(k_base, k_next, next, [&](int i) INLINE {
                constexpr int E = 16 / KK;
#pragma unroll
                for (int r = i * E; r < i * E + E; ++r) {
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
        float *sums = a.sums + ((int64_t)uniform(walk.worker) * 2 + (from == 0)) * (M * (DP + 2)) + wave * 32 * DP;
        // Zeros for infinities and NaN in the values of 32 tokens (odd_values).
        bool met = false;
        auto take_odd = [&](char *vb) INLINE {
            uint32_t odd = 0;
#pragma unroll 1
            for (int x = tid; x < 32 * CH; x += THREADS) odd |= odd8<T>(*(const s16x8 *)(vb + 16 * x));
            if (!__syncthreads_or(odd != 0)) return;
            met = true;
#pragma unroll 1
            for (int x = tid; x < 32 * CH * 8; x += THREADS) {
                short *y = (short *)vb + x;
                if (!finite16<T>(*y)) *y = 0;
            }
            __syncthreads();
        };
        auto partly_seen = [&](int t0) INLINE { return t0 < tile_lo || t0 + 32 > tile_hi; };

        // Tile i's keys are needed from the second half of tile i - 1 on, its
        // values until the first half of tile i + 1: one barrier a tile, in
        // its middle. Turn i, after that of tile i, fetches the page ids of
        // tile i + 2 S - 1, the values of i + S - 1 and the keys of i + S: PER
        // loads a wave. Turns first - S .. first - 1 come before the loop.
        constexpr int PER = 2 * L + 1;
        __syncthreads();                       // the previous rows' products have read their buffers
#pragma unroll
        for (int i = 0; i < L; ++i)            // the values "before" the first tile
            *(uint4 *)(values + (S - 1) * TILE + (i * THREADS + tid) * 16) = uint4{0, 0, 0, 0};
        arrived<0>();
#pragma unroll 1
        for (int i = 0; i < S; ++i) {
            if (i) {
                fetch_ids(first + S - 1 + i);
                if (first + i - 1 < last) load_values(first + i - 1);
            }
            if (first + i < last) load_keys(first + i);
        }
        if (first + S - 1 < last)
            arrived<(S - 1) * PER>();
        else
            arrived<0>();
        __syncthreads();
        if (active) multiply(k_at, 0, s0, nothing);
        for (int step = first; step < last;) {
            if constexpr (DP < 256) {
                // S tiles whose tokens every row of the tile sees, with S more
                // to load: places in LDS are constants, nothing is masked, and
                // offsets into the pool have 32 bits. (Heads of 256 run out of
                // registers here: 109 us against 98 for nine chunks with a
                // window.)
                const int t0 = step * BN;
                if (near && ((step - first) & (S - 1)) == 0 && (step == first ? t0 : t0 - 32) >= tile_lo &&
                    t0 + S * BN <= tile_hi && step + 2 * S <= last && t0 + 2 * S * BN <= range.hi) {
                    auto turn = [&](auto r_) INLINE {
                        constexpr int R = decltype(r_)::value, N = (R + 1) % S, B = (R + S - 1) % S;
                        if (active) step32(std::true_type(), s0, s1, 0, k_at, R * TILE + 32 * ROW, v_at, B * TILE + 32 * ROW);
                        arrived<(S - 2) * PER>();
                        __syncthreads();
                        fetch_ids_near(step + R + 2 * S - 1);
                        load_near(step + R + S - 1, vh, v_near, a.v_page, a.v_slot, v_lds + B * TILE);
                        load_near(step + R + S, kh, k_near, a.k_page, a.k_slot, k_lds + R * TILE);
                        if (active) step32(std::true_type(), s1, s0, 0, k_at, N * TILE, v_at, R * TILE);
                    };
                    turn(std::integral_constant<int, 0>());
                    turn(std::integral_constant<int, 1>());
                    if constexpr (S == 4) {
                        turn(std::integral_constant<int, 2>());
                        turn(std::integral_constant<int, 3>());
                    }
                    step += S;
                    continue;
                }
            }
            // any other tile, its two halves by one piece of code: a call with
            // few steps waits for its instructions more than for anything else
            const int at = (step - first) & (S - 1), now = at * TILE, next = ((at + 1) & (S - 1)) * TILE, before = ((at - 1) & (S - 1)) * TILE;
#pragma unroll 1
            for (int h = 0; h < 2; ++h) {
                const int t = step * BN + 32 * h, v_before = h ? now : before + 32 * ROW;
                if (t > first * BN && partly_seen(t - 32)) take_odd(values + v_before);
                if (active) {
                    step32(std::false_type(), s0, s1, t, k_at + (h ? next : now + 32 * ROW), 0, v_at + v_before, 0);
                    s0 = s1;
                }
                if (h) break;
                // all up to turn step + 1 - S; where turns had no tile left to
                // load their count is short of PER, and everything is waited for
                if (step + S - 1 < last)
                    arrived<(S - 2) * PER>();
                else
                    arrived<0>();
                __syncthreads();
                if (step + S - 1 < last) {
                    fetch_ids(step + 2 * S - 1);
                    load_values(step + S - 1);
                    if (step + S < last) load_keys(step + S);
                }
            }
            ++step;
        }
        {
            const int v_last = ((last - 1 - first) & (S - 1)) * TILE + 32 * ROW, t0 = last * BN - 32;
            if (partly_seen(t0)) take_odd(values + v_last);
            if (active) add(v_at + v_last, 0, nothing);
        }

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
        float odd = 0;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int r = 0; r < 16; r += 4) odd += not_finite(f32x4{o[dt][r], o[dt][r + 1], o[dt][r + 2], o[dt][r + 3]});
        if (__builtin_expect(active && __any(met | (odd != 0)), 0)) {
            const bool whole = starts && ends, f32 = !whole || a.out_f32;
            const int size = f32 ? 4 : 2;
            odd_values<T, DP == 64 ? 8 : 16>(a, table, shift, vh, max(range.lo, first * BN), min(range.hi, last * BN), see_lo, see_hi,
                          r0 < rows ? sum : NAN, whole, 4 * half, 8,
                          whole ? a.out + size * ((int64_t)(q0 + j0) * a.out_token + ((int64_t)head * a.group + rr - j0 * a.group) * a.out_head + 4 * half)
                                : (char *)(sums + lane * 4),
                          whole ? 8 * size : 64 * 16, f32);
        }
        if (ends && walk.at < walk.end) walk.next(a, ent);
    }
    if (lost) flag(c, MPT_KV_BAD_PAGE);
}

// Joins the parts of a tile: workgroup (w, block of 32 rows); the waves share
// the dimensions.
template <class T, int DP, int WAVES>
__global__ __launch_bounds__(256) void k_kv_join_wide(Attn a) {
    constexpr int M = 32 * WAVES, DT = DP / 32;
    const int w = blockIdx.x, block = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5;
    const Part part = a.parts[w];
    if (part.count == 0) return;
    const int rows = part.n * a.group, r = part.tile * M + block * 32 + (lane & 31);
    if (part.tile * M + block * 32 >= rows) return;
    // part i: worker w - 1 + i; the first one's second slot, the others' first
    auto sums = [&](int i) { return a.sums + ((int64_t)(w - 1 + i) * 2 + (i == 0)) * (M * (DP + 2)); };
    float m = -INFINITY, l = 0;
    f32x4 o[(DT + 3) / 4][4] = {};
    for (int i = 0; i < part.count; i += 2) {
        float pm[2], pl[2];
        f32x4 po[2][(DT + 3) / 4][4];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const bool there = i + u < part.count;
            const float *p = sums(there ? i + u : i), *st = p + M * DP + block * 64 + (lane & 31);
            pm[u] = there ? st[0] : -INFINITY;
            pl[u] = st[32];
#pragma unroll
            for (int k = 0; k < (DT + 3) / 4; ++k)
                if (wave + 4 * k < DT)
#pragma unroll
                    for (int x = 0; x < 4; ++x)
                        po[u][k][x] = *(const f32x4 *)(p + block * 32 * DP + (((wave + 4 * k) * 4 + x) * 64 + lane) * 4);
        }
        const float now = fmaxf(m, fmaxf(pm[0], pm[1])), base = now == -INFINITY ? 0.0f : now;
        const float keep = __builtin_amdgcn_exp2f(m - base);
        l *= keep;
#pragma unroll
        for (int k = 0; k < (DT + 3) / 4; ++k)
#pragma unroll
            for (int x = 0; x < 4; ++x) o[k][x] *= keep;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            if (i + u >= part.count) break;
            const float f = __builtin_amdgcn_exp2f(pm[u] - base);
            l += f * pl[u];
#pragma unroll
            for (int k = 0; k < (DT + 3) / 4; ++k)
                if (wave + 4 * k < DT)
#pragma unroll
                    for (int x = 0; x < 4; ++x) o[k][x] += f * po[u][k][x];
        }
        m = now;
    }
#pragma unroll
    for (int k = 0; k < (DT + 3) / 4; ++k)
        if (wave + 4 * k < DT)
#pragma unroll
            for (int x = 0; x < 4; ++x)
                o[k][x] = odd_parts(o[k][x], part.count,
                                    [&](int i) { return sums(i) + block * 32 * DP + (((wave + 4 * k) * 4 + x) * 64 + lane) * 4; });
    if (r >= rows) return;
    const int j = token_of(a, r);
    const int64_t token = part.q0 + j, h = (int64_t)part.head * a.group + r - j * a.group;
    const float scale = 1.0f / l;
    if (a.lse && wave == 0 && half == 0)
        a.lse[token * a.heads + h] = l == 0 ? -INFINITY : 0.693147180559945f * (m + __builtin_amdgcn_logf(l));
#pragma unroll
    for (int k = 0; k < (DT + 3) / 4; ++k)
        if (wave + 4 * k < DT)
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int d = (wave + 4 * k) * 32 + 8 * x + 4 * half;
                if (d < 8 * a.units) store4<T>(a, token * a.out_token + h * a.out_head + d, l == 0 ? f32x4{0, 0, 0, 0} : o[k][x] * scale);
            }
}

template <class T, int DP, int WAVES>
static void launch(const Attn &a, hipStream_t s) {
    {
        mptlib::LaunchScope scope("k_kv_wide", (double)a.n_tokens * a.heads, s);
        if (a.cap != 0)
            k_kv_wide<T, DP, WAVES, true><<<a.workers, 64 * WAVES, 0, s>>>(a);
        else
            k_kv_wide<T, DP, WAVES, false><<<a.workers, 64 * WAVES, 0, s>>>(a);
    }
    mptlib::LaunchScope scope("k_kv_join_wide", a.workers, s);
    k_kv_join_wide<T, DP, WAVES><<<dim3(a.workers, WAVES), 256, 0, s>>>(a);
}

template <class T>
static void launch_dim(const Attn &a, int waves, hipStream_t s) {
    const int dim = pad_dim(8 * a.units);
    if (dim == 64)
        waves == 8 ? launch<T, 64, 8>(a, s) : launch<T, 64, 4>(a, s);
    else if (dim == 128)
        waves == 8 ? launch<T, 128, 8>(a, s) : launch<T, 128, 4>(a, s);
    else
        launch<T, 256, 4>(a, s);
}

void launch_wide(const Attn &a, int waves, hipStream_t s) {
    if (a.c.dtype == MPT_KV_BF16)
        launch_dim<__bf16>(a, waves, s);
    else
        launch_dim<_Float16>(a, waves, s);
}

}  // namespace mptkv
