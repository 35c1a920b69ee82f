// Attention kernel over a cache in 4 bits for many rows per key head (chunks of
// new tokens): tiles of 128 or 256 rows, 32 to each of the four or eight waves,
// with the products of the kernel over 16 bits (scores transposed, weights as the
// second operand of O' += V' P' as they lie). Heads of 256 have eight waves of 16
// rows, with products of 16 by 16: four of 32 fill the registers, and one wave a SIMD
// leaves a vector instruction's place empty in two (128 rows of 128 entries over 4000
// tokens 880 us, eight waves 684).
//
// A workgroup turns each tile of 64 tokens into 16 bits once, for all of its rows:
// a thread takes one piece of 32 elements of keys or of values (heads of 128, eight
// waves), loaded a tile ahead, and writes them to LDS where its products read them.
// Two tiles of keys and two of values are there at a time.
//
// What bounds it: the matrix units and what their clock is under load (chunks of
// 1024 tokens over 16k, 32 heads on 8 of 128: 0.95 to 1.06 ms, 1.0 to 1.1 PFLOP/s,
// where a library product of 8192^3 reaches 1.24), then vector instructions: scores
// and weights as over 16 bits, and 16 conversions and 4 stores a piece. Where a
// workgroup has few steps, it is what surrounds them. The numbers that a tile starts
// from do not fit the scalar registers beside the loop's: eight waves and heads of 128
// keep 108 of them and 6 vector registers elsewhere (of 256, 167 and 16), and a
// start takes 106 lane moves and 5 reads of memory for them (162 and 8), a step none
// (2 moves).
// And a tile that is cut goes through memory: 9 chunks of heads of 256 with a window
// are 140 tiles over 256 workgroups, of which 127 are cut into 313 parts of 132 KB, 41
// MB written and read again beside the 27 MB of the case itself (59 us in all).

#include "attention_mx4.h"

#include <type_traits>

namespace mptkv {

#define INLINE __attribute__((always_inline))

template <int DP, int WAVES>
struct Wide4 {
    static constexpr bool kSmall = DP == 256;                                  // products of 16 rows
    static constexpr int kThreads = 64 * WAVES, BN = 64, ROW = 2 * DP, R = kSmall ? 16 : 32, M = R * WAVES;
    static constexpr int KK = DP * R / 512, DT = DP / R;                       // operands of a row, and of an output row
    static constexpr int S = R / 2;                                            // scores a lane of 32 tokens
    typedef float Scores __attribute__((ext_vector_type(S)));
    typedef float Sums __attribute__((ext_vector_type(R == 16 ? 4 : 16)));
    static constexpr int kTile = BN * ROW, CP = DP / 32, kPieces = BN * CP;   // bytes in 16 bits; pieces of a row, of a tile
    static constexpr int L = (2 * kPieces + kThreads - 1) / kThreads;          // pieces of keys and values per thread
    static constexpr int C = DP == 256 ? 4 : 8;                                                // a tile's cost besides its steps, in steps
    static constexpr int kAhead = DP == 256 ? 3 : 2;                           // operands read from LDS ahead of their products

    // Where the 16-byte pieces of a token's row lie: keys so that eight tokens'
    // pieces (wide heads: 16 tokens'), values so that four tokens' 64 bytes (32), fall
    // on all banks, and so do the first (second, ...) quarters of the elements that 16
    // threads (eight) write at a time; equal for tokens 8 apart (values) and 32 (keys; 16).
    __host__ __device__ static constexpr int fold(int u) { return kSmall ? u ^ ((u >> 3) & 3) : u; }
    __device__ static int k_swizzle(int t) { return DP == 64 ? (t >> 1) & 7 : t & 15; }
    __device__ static int v_swizzle(int t) { return DP == 64 ? 5 * ((t >> 1) & 1) + 2 * ((t >> 2) & 1) : DP == 128 ? 5 * (t & 3) : 2 * (t & 7); }
};

template <class T, int DP, int WAVES, bool CAP>
__global__ __launch_bounds__(64 * WAVES, 2) void k_kv_wide_mx4(Attn4 a) {
    using W = Wide4<DP, WAVES>;
    constexpr int M = W::M, THREADS = W::kThreads, BN = W::BN, KK = W::KK, DT = W::DT, ROW = W::ROW, L = W::L, TILE = W::kTile, R = W::R;
    constexpr int C = W::C, AHEAD = W::kAhead, CP = W::CP, S = W::S;
    constexpr bool SMALL = W::kSmall;
    __shared__ Entries ent;
    __shared__ __attribute__((aligned(1024))) char keys[2 * TILE], values[2 * TILE];
    const mpt_kv_cache &c = a.c;
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), col = lane & (R - 1), part = lane / R;   // part: half, or quarter, of the wave
    const int shift = 31 - __clz(c.page_size), pieces = a.units / 4;
    // Where a lane reads its operands: rows of 32 tokens of keys (16), 8 of values (16).
    const uint32_t k_at = lds_address(keys) + col * ROW + 16 * (part ^ W::k_swizzle(col));
    const int v_of = (SMALL ? 4 * part : 4 * (lane >> 5)) + (lane & 15) / 4, v_piece = (SMALL ? 0 : ((lane >> 4) & 1) * 2) + (lane & 3) / 2;
    const uint32_t v_at = lds_address(values) + v_of * ROW + (lane & 1) * 8 + 16 * (v_piece ^ W::v_swizzle(v_of));
    int lost = 0;                              // a page id outside the pool
    // A thread's pieces, and where their elements go: the first quarter of each.
    auto is_key = [&](int i) INLINE { return i * THREADS + wave * 64 < W::kPieces; };
    // (waves without a piece load another's: what is on its way is the same on all ways,
    // or the compiler would wait for it as soon as it is asked for)
    auto has_piece = [&](int i) INLINE { return L * THREADS == 2 * W::kPieces || i * THREADS + wave * 64 < 2 * W::kPieces; };
    auto piece_of = [&](int i) INLINE { return (i * THREADS + renewed(tid)) & (CP - 1); };
    auto token_of_piece = [&](int i) INLINE { return (int)((uint32_t)((i * THREADS + renewed(tid)) & (W::kPieces - 1)) / CP); };
    uint32_t put_at[L];
#pragma unroll
    for (int i = 0; i < L; ++i) {
        const int t = token_of_piece(i), swizzle = is_key(i) ? W::k_swizzle(t) : W::v_swizzle(t);
        put_at[i] = lds_address(is_key(i) ? keys : values) + t * ROW + ((W::fold(4 * piece_of(i)) ^ swizzle) << 4);
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
        const int rows = n * a.group, row_base = tile * M + wave * R;
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
                const bool key = is_key(i);
                const uint32_t id = min((uint32_t)ids[i], (uint32_t)c.n_pages - 1);
                lost |= id != (uint32_t)ids[i] && range.hi > 0;
                // at this place: the old id and the one that is loaded next then have one register
                asm volatile("" : "+v"(lost));
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
            const int piece = 64 / R * kk + part;
            u32x4 x = mptkv::load<u32x4>(or_zeros(r0 < rows && piece < a.units, q + 16 * piece));
            if (a.flip) x ^= 0x80008000u;
            qf[kk] = __builtin_bit_cast(s16x8, x);
        }
        // tokens that all rows of the wave, and of the tile, see
        int wave_lo, wave_hi, tile_lo, tile_hi;
        seen_by_all(a, n, len, begin, min(row_base, rows - 1), min(row_base + R - 1, rows - 1), wave_lo, wave_hi);
        seen_by_all(a, n, len, begin, tile * M, min(tile * M + M, rows) - 1, tile_lo, tile_hi);

        typename W::Sums o[DT];
        typename W::Scores s0, s1;
        s16x8 pf[S / 8];
        float m = -INFINITY, l = 0;
#pragma unroll
        for (int x = 0; x < S / 8; ++x) pf[x] = s16x8{0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[dt] = 0;

        // The products of a step, in groups that the compiler keeps in order:
        // an operand from LDS (read some groups ahead), its product, and beside
        // it a share of the step's other work.
        // S' = K Q' of 32 tokens (base: where the lane's first operand lies; kb, vb: bytes
        // from there, constants)
        constexpr int KG = SMALL ? 2 * KK : KK, VG = SMALL ? DT : 2 * DT;       // products of 32 tokens
        auto multiply = [&](uint32_t base, int kb, typename W::Scores &s, auto beside) INLINE {
            s16x8 kf[AHEAD + 1];
            auto read = [&](int i) INLINE {
                const int kk = i % KK;
                kf[i % (AHEAD + 1)] = from_lds<s16x8>((base ^ 16 * W::fold(64 / R * kk)) + i / KK * 16 * ROW + kb);
            };
            f32x4 two[2];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) read(i);
#pragma unroll
            for (int i = 0; i < KG; ++i) {
                if (i + AHEAD < KG) read(i + AHEAD);
                const s16x8 x = kf[i % (AHEAD + 1)];
                if constexpr (SMALL)
                    two[i / KK] = Type<T>::mfma16(x, qf[i % KK], i % KK ? two[i / KK] : f32x4{0, 0, 0, 0});
                else
                    s = Type<T>::mfma32(x, qf[i], i ? s : f32x16{0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0});
                beside(i);
                __builtin_amdgcn_sched_barrier(0);
            }
            if constexpr (SMALL) s = __builtin_shufflevector(two[0], two[1], 0, 1, 2, 3, 4, 5, 6, 7);
        };
        // O' += V' P' of 32 tokens
        auto add = [&](uint32_t base, int vb, auto beside) INLINE {
            s16x8 vf[AHEAD + 1];
            auto read = [&](int i) INLINE {
                const uint32_t x = (base ^ 16 * W::fold(R / 8 * (i % DT))) + vb + (i / DT) * 16 * ROW;
                const s16x4 y = read_column4(x), z = read_column4(x + (SMALL ? 16 : 8) * ROW);
                vf[i % (AHEAD + 1)] = __builtin_shufflevector(y, z, 0, 1, 2, 3, 4, 5, 6, 7);
            };
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) read(i);
#pragma unroll
            for (int i = 0; i < VG; ++i) {
                if (i + AHEAD < VG) read(i + AHEAD);
                const s16x8 x = vf[i % (AHEAD + 1)];
                if constexpr (SMALL)
                    o[i] = Type<T>::mfma16(x, pf[0], o[i]);
                else
                    o[i % DT] = Type<T>::mfma32(x, pf[i / DT], o[i % DT]);
                beside(i);
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        auto nothing = [](int) INLINE {};
        // the largest of what a row's lanes have
        auto over_row = [&](float x, auto f) INLINE {
            x = f(x, __shfl_xor(x, 32));
            return SMALL ? f(x, __shfl_xor(x, 16)) : x;
        };
        const auto larger = [](float x, float y) INLINE { return fmaxf(x, y); };
        const auto sum_of = [](float x, float y) INLINE { return x + y; };
        // One step of 32 tokens from t0 with scores x: products with the values
        // of the step before beside this step's maximum, scores of the next
        // step beside this step's weights.
        auto step32 = [&](auto all_seen, typename W::Scores &x, typename W::Scores &next, int t0, uint32_t k_base, int k_next, uint32_t v_base, int v_before) INLINE {
            if constexpr (CAP) {
#pragma unroll
                for (int r = 0; r < S; ++r) x[r] = score<true>(a, x[r]);
            }
            if (!all_seen && (t0 < wave_lo || t0 + 32 > wave_hi)) {
                const int before = t0 + 4 * renewed(part), lo = see_lo - before, hi = see_hi - before;
#pragma unroll
                for (int r = 0; r < S; ++r) {
                    const int t = (SMALL ? 16 : 8) * (r / 4) + r % 4;
                    if (!(t >= lo && t < hi)) x[r] = -INFINITY;
                }
            }
            __builtin_amdgcn_s_setprio(1);
            float top = -INFINITY;
            add(v_base, v_before, [&](int i) INLINE {
#pragma unroll
                for (int y = i * S / VG; y < (i + 1) * S / VG; ++y) top = fmaxf(top, x[y]);
            });
            if constexpr (!CAP) top *= a.factor;
            if (__any(top > m + 8.0f)) {
                const float now = fmaxf(m, over_row(top, larger));
                const float keep = now == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - now);
                if (!__all(m == -INFINITY)) {                         // else the sums are zeros
                    l *= keep;
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt) o[dt] *= keep;
                }
                m = now;
            }
            const float base = m == -INFINITY ? 0.0f : m;
            // Weights are rounded to the 16-bit type, so that both operands of the
            // product are of one, as over 16 bits.
            float even = 0;
            u32x4 packed[S / 8];
            multiply(k_base, k_next, next, [&](int i) INLINE {
#pragma unroll
                for (int r = i * S / KG; r < (i + 1) * S / KG; ++r) {
                    const float w = __builtin_amdgcn_exp2f(CAP ? x[r] - base : __builtin_fmaf(x[r], a.factor, -base));
                    l += w;
                    if (r % 2)
                        packed[r / 8][r % 8 / 2] = pack<T>(even, w);
                    else
                        even = w;
                }
            });
#pragma unroll
            for (int y = 0; y < S / 8; ++y) pf[y] = __builtin_bit_cast(s16x8, packed[y]);
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
            if (active) step32(std::false_type(), s0, s1, step * BN, k_at + now + 32 * ROW, 0, v_at + other + 32 * ROW, 0);
            __syncthreads();
            make(!odd);
            fetch(step + 2);
            fetch_ids(step + 3);
            if (active) step32(std::false_type(), s1, s0, step * BN + 32, k_at + other, 0, v_at + now, 0);
            ++step;
        }
        if (active) add(v_at + ((last - 1 - first) & 1) * TILE + 32 * ROW, 0, nothing);

        // sums of 32 rows, as the join reads them: rows in products of 32, dimensions 4 at a time
        float *sums = a.sums + ((int64_t)uniform(walk.worker) * 2 + (from == 0)) * (M * (DP + 2)) + wave * R / 32 * 32 * DP;
        const int at_lane = SMALL ? (part / 2) * 64 + (part & 1) * 32 + (wave & 1) * 16 + col : lane;
        const float sum = over_row(l, sum_of);
        if (starts && ends) {
            const int r = row_base + renewed(col);
            if (r < rows) {
                const float scale = sum == 0 ? 0.0f : 1.0f / sum;
                const int j = token_of(a, r);
                const int64_t token = q0 + j, hq = (int64_t)head * a.group + r - j * a.group;
                if (a.lse && part == 0)
                    a.lse[token * a.heads + hq] = sum == 0 ? -INFINITY : 0.693147180559945f * (m + __builtin_amdgcn_logf(sum));
                const int64_t to = token * a.out_token + hq * a.out_head + 4 * part;
                auto store = [&](auto f32) INLINE {
                    char *row = a.out + (f32 ? 4 : 2) * to;
                    if constexpr (SMALL) {
#pragma unroll
                        for (int x = 0; x < DT; ++x) {
                            if (2 * x >= a.units) break;
                            put4<T, f32>(row, 16 * x, o[x] * scale);
                        }
                    } else {
#pragma unroll
                        for (int x = 0; x < DT * 4; ++x) {
                            if (x >= a.units) break;
                            const f32x16 &y = o[x / 4];
                            const int i = x % 4 * 4;
                            put4<T, f32>(row, 8 * x, f32x4{y[i], y[i + 1], y[i + 2], y[i + 3]} * scale);
                        }
                    }
                };
                a.out_f32 ? store(std::true_type()) : store(std::false_type());
            }
        } else {
            // unnormalised sums, also those of rows behind the last beside others
            if (row_base / 32 * 32 < rows) {
                if constexpr (SMALL) {
#pragma unroll
                    for (int x = 0; x < DT; ++x) *(f32x4 *)(sums + (2 * x * 64 + at_lane) * 4) = o[x];
                } else {
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                        for (int r = 0; r < 16; r += 4)
                            *(f32x4 *)(sums + ((dt * 4 + r / 4) * 64 + lane) * 4) = f32x4{o[dt][r], o[dt][r + 1], o[dt][r + 2], o[dt][r + 3]};
                }
                float *stats = sums - wave * R / 32 * 32 * DP + M * DP + wave * R / 32 * 64;
                if (part < 2) stats[SMALL ? part * 32 + (wave & 1) * 16 + col : lane] = part ? sum : m;
            }
            if (!starts && tid == 0) {
                const int workers = walk.second_of(range.count);
                if (workers) a.parts[walk.worker] = Part{workers, e + walk.base, head, tile, q0, n};
            }
        }
        if (__builtin_expect(__syncthreads_or(met), 0)) {
            const bool whole = starts && ends, f32 = !whole || a.out_f32;
            const int size = f32 ? 4 : 2;
            constexpr int STEP = SMALL ? 16 : 8;             // dimensions from one of a lane's four to the next
            if (active)
                nan_values<T>(a, table, shift, a.ve + head * a.ve_head, max(range.lo, first * BN), min(range.hi, last * BN), see_lo, see_hi,
                              r0 < rows ? sum : NAN, whole, 4 * part, STEP,
                              whole ? a.out + size * ((int64_t)(q0 + j0) * a.out_token + ((int64_t)head * a.group + rr - j0 * a.group) * a.out_head + 4 * part)
                                    : (char *)(sums + at_lane * 4),
                              whole ? STEP * size : STEP * 128, f32);
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
        launch<T, 256, 8>(a, s);
}

void launch_wide_mx4(const Attn4 &a, int waves, hipStream_t s) {
    value_type(a.c) == MPT_KV_BF16 ? launch_dim<__bf16>(a, waves, s) : launch_dim<_Float16>(a, waves, s);
    join_wide(a, waves, s);
}

}  // namespace mptkv
