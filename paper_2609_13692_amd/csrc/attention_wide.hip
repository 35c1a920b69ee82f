// Attention kernel for many rows per key head (chunks of new tokens): tiles of
// 128 NB rows, each of the four waves holding NB blocks of 32.
//
// Scores are formed transposed, S' = K Q', with 32x32x16 products: lane l then
// holds query l % 32 and 16 of 32 tokens, so the running maximum and sum of a
// query are values of its own two lanes, and the weights, rounded, are the
// second operand of O' += V' P' as they lie (the tokens of a product may come
// in any order if both operands agree on it). Keys and values go from memory
// to LDS directly, one tile of 64 tokens (32 at 256 dimensions) ahead of the
// products; values are read back by the transposing LDS loads.
//
// The maximum that weights are taken against is moved only when a score
// exceeds it by 2^8: products with weights up to 256 are as exact, and the
// sums are rescaled a few times per row instead of at every step.

#include "attention.h"

namespace mptkv {

template <int DP>
struct Wide {
    static constexpr int BN = 64, KK = DP / 16, DT = DP / 32, ROW = 2 * DP, CH = DP / 8;
    static constexpr int kTile = BN * ROW, kLoads = kTile / 4096;     // 16-byte loads per thread, of keys or values
    static constexpr int kStride = 256 / CH;                          // tokens between a thread's loads

    // Where the 16-byte pieces of a token's row lie: keys so that eight
    // tokens' pieces, values so that four tokens' 64 bytes, fall on all banks;
    // equal for tokens kStride apart, so that a thread loads one piece of its
    // tokens.
    __device__ static int k_swizzle(int token) { return DP == 64 ? (token >> 1) & 7 : DP == 128 ? token & 15 : token & 7; }
    __device__ static int v_swizzle(int token) { return DP == 64 ? 4 * ((token >> 1) & 1) : 4 * (token & 3); }
};

template <class T, int DP, int NB, bool CAP>
__global__ __launch_bounds__(256, NB == 2 || DP == 256 ? 1 : 2) void k_kv_wide(Attn a) {
    using W = Wide<DP>;
    constexpr int M = 128 * NB, BN = W::BN, KK = W::KK, DT = W::DT, ROW = W::ROW, CH = W::CH, L = W::kLoads, TILE = W::kTile;
    __shared__ Entries ent;
    __shared__ __attribute__((aligned(1024))) char keys[2 * TILE], values[2 * TILE];
    const mpt_kv_cache &c = a.c;
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), col = lane & 31, half = lane >> 5;
    const int shift = 31 - __clz(c.page_size);
    const uint32_t k_lds = __builtin_amdgcn_readfirstlane(lds_address(keys) + wave * 1024);
    const uint32_t v_lds = __builtin_amdgcn_readfirstlane(lds_address(values) + wave * 1024);
    // the thread's tokens of a tile, its pieces of their rows
    const int own = tid / CH, kp = (tid % CH) ^ W::k_swizzle(own), vp = (tid % CH) ^ W::v_swizzle(own);
    const bool k_in = kp < a.units, v_in = vp < a.units;
    // where a lane reads its operands: rows of 32 tokens of keys, 8 of values
    const int k_row = col * ROW, k_flip = half ^ W::k_swizzle(col);
    const int v_of = 4 * half + (lane & 15) / 4;
    const int v_row = v_of * ROW + (lane & 1) * 8, v_flip = (((lane >> 4) & 1) * 2 + (lane & 3) / 2) ^ W::v_swizzle(v_of);

    Walk<M, BN> walk;
    if (!walk.begin(a, ent, 4)) return;

    while (walk.at < walk.end) {
        const int e = uniform(walk.e), n = uniform(ent.n[e]), len = uniform(ent.len[e]), q0 = uniform(ent.q0[e]);
        const int begin = uniform(ent.begin[e]), head = uniform(walk.head), tile = uniform(walk.tile);
        const Range range = tile_range<M, BN>(a, n, len, begin, tile);
        const int from = uniform((int)(walk.at - walk.tile_at)), first = range.first + from;
        const int last = uniform(range.first + (int)min((int64_t)range.count, from + (walk.end - walk.at)));
        const int rows = n * a.group, row_base = tile * M + wave * 32 * NB;
        const int32_t *table = c.table + (int64_t)uniform(ent.slot[e]) * c.max_pages;
        const bool active = row_base < rows;

        // queries of the wave's blocks as operands, and what each may see
        s16x8 qf[NB][KK];
        int see_lo[NB], see_hi[NB], wave_lo = 0, wave_hi = 1 << 30;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            const int r = row_base + nb * 32 + col, rr = min(r, rows - 1), j = rr / a.group;
            const int p = len - n + j;
            see_hi[nb] = a.causal ? min(len, p + 1) : len;
            see_lo[nb] = a.window ? max(begin, p + 1 - a.window) : begin;
            const char *q = a.q + 2 * ((int64_t)(q0 + j) * a.q_token + ((int64_t)head * a.group + rr - j * a.group) * a.q_head);
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) {
                const int piece = 2 * kk + half;
                u32x4 x = mptkv::load<u32x4>(or_zeros(r < rows && piece < a.units, q + 16 * piece));
                if (a.flip) x ^= 0x80008000u;
                qf[nb][kk] = __builtin_bit_cast(s16x8, x);
            }
            int lo = see_lo[nb], hi = see_hi[nb];
            for (int d = 1; d < 32; d <<= 1) lo = max(lo, __shfl_xor(lo, d)), hi = min(hi, __shfl_xor(hi, d));
            wave_lo = max(wave_lo, lo), wave_hi = min(wave_hi, hi);
        }
        wave_lo = __builtin_amdgcn_readfirstlane(wave_lo), wave_hi = __builtin_amdgcn_readfirstlane(wave_hi);
        // tokens that all rows of the tile see
        const int pa = len - n + tile * M / a.group, pb = len - n + (min(tile * M + M, rows) - 1) / a.group;
        const int tile_hi = a.causal ? min(len, pa + 1) : len, tile_lo = a.window ? max(begin, pb + 1 - a.window) : begin;

        f32x16 o[NB][DT], s[NB];
        s16x8 pf[NB][2];
        float m[NB], l[NB];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            m[nb] = -INFINITY, l[nb] = 0;
            pf[nb][0] = pf[nb][1] = s16x8{0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[nb][dt][r] = 0;
        }

        // pages of the thread's tokens of a tile, and the tile's loads
        const char *kh = a.k + head * a.k_head + 16 * kp, *vh = a.v + head * a.v_head + 16 * vp;
        auto find_pages = [&](int step, int (&page)[L]) {
#pragma unroll
            for (int i = 0; i < L; ++i) {
                const int t = step * BN + i * W::kStride + own;
                page[i] = t >= range.lo && t < range.hi ? table[t >> shift] : -1;
            }
        };
        auto load = [&](int step, const int (&page)[L], const char *rows0, bool in, uint32_t page_stride, uint32_t slot_stride, uint32_t lds) {
#pragma unroll
            for (int i = 0; i < L; ++i) {
                const int t = step * BN + i * W::kStride + own;
                const bool there = (unsigned)page[i] < (unsigned)c.n_pages;
                if (!there && t >= range.lo && t < range.hi) flag(c, MPT_KV_BAD_PAGE);
                load_lds16(or_zeros(there && in, rows0 + row_at(page[i], t & (c.page_size - 1), page_stride, slot_stride)), lds + i * 4096);
            }
        };
        // S' = K Q' of 32 tokens
        auto multiply = [&](const char *kb) {
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[nb][r] = 0;
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) {
                const s16x8 kf = *(const s16x8 *)(kb + k_row + (((2 * kk) ^ k_flip) << 4));
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) s[nb] = Type<T>::mfma32(kf, qf[nb][kk], s[nb]);
            }
        };
        // O' += V' P' of 32 tokens
        auto add = [&](const char *vb) {
#pragma unroll
            for (int g = 0; g < 2; ++g)
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) {
                    const char *p = vb + g * 16 * ROW + v_row + (((dt * 4) ^ v_flip) << 4);
                    const s16x4 x = read_column4(p), y = read_column4(p + 8 * ROW);
                    const s16x8 vf = __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) o[nb][dt] = Type<T>::mfma32(vf, pf[nb][g], o[nb][dt]);
                }
        };
        // One step of 32 tokens from t0: products with the values of the step
        // before beside this step's maximum, scores of the next step beside
        // this step's weights.
        auto step32 = [&](int t0, const char *k_next, const char *v_before) {
            f32x16 x[NB];
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                x[nb] = s[nb];
                if constexpr (CAP) {
#pragma unroll
                    for (int r = 0; r < 16; ++r) x[nb][r] = score<true>(a, x[nb][r]);
                }
            }
            if (t0 < wave_lo || t0 + 32 > wave_hi) {
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const int t = t0 + 4 * half + 8 * (r / 4) + r % 4;
                        if (!(t >= see_lo[nb] && t < see_hi[nb])) x[nb][r] = -INFINITY;
                    }
            }
            add(v_before);
            float top[NB];
            bool up = false;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                top[nb] = x[nb][0];
#pragma unroll
                for (int r = 1; r < 16; ++r) top[nb] = fmaxf(top[nb], x[nb][r]);
                if constexpr (!CAP) top[nb] = fmaxf(top[nb] * a.factor, -INFINITY);
                up |= top[nb] > m[nb] + 8.0f;
            }
            if (__any(up)) {
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    const float now = fmaxf(m[nb], fmaxf(top[nb], __shfl_xor(top[nb], 32)));
                    const float keep = now == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m[nb] - now);
                    m[nb] = now;
                    l[nb] *= keep;
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                        for (int r = 0; r < 16; ++r) o[nb][dt][r] *= keep;
                }
            }
            multiply(k_next);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                const float base = m[nb] == -INFINITY ? 0.0f : m[nb];
                typename Type<T>::x8 p;
                float sum[4] = {0, 0, 0, 0};
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const float w = __builtin_amdgcn_exp2f(CAP ? x[nb][r] - base : __builtin_fmaf(x[nb][r], a.factor, -base));
                    sum[r % 4] += w;
                    p[r % 8] = (T)w;
                    if (r % 8 == 7) pf[nb][r / 8] = __builtin_bit_cast(s16x8, p);
                }
                l[nb] += (sum[0] + sum[1]) + (sum[2] + sum[3]);
            }
        };
        // Infinities and NaN in values of 32 tokens: a weight of zero does not
        // cancel them in a row that does not see them. Rows that do see them
        // get them added here, in memory, which costs the products no
        // registers; then they are zeros for the product.
        float *sums = a.sums + ((int64_t)uniform(walk.worker) * 2 + (from == 0)) * (M * (DP + 2)) + wave * NB * 32 * DP;
        auto put_sums = [&]() {
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                    for (int r = 0; r < 16; r += 4)
                        *(f32x4 *)(sums + (((nb * DT + dt) * 4 + r / 4) * 64 + lane) * 4) =
                            f32x4{o[nb][dt][r], o[nb][dt][r + 1], o[nb][dt][r + 2], o[nb][dt][r + 3]};
        };
        auto odd_values = [&](int t0, char *vb) {
            uint32_t odd = 0;
#pragma unroll 1
            for (int x = tid; x < 32 * CH; x += 256) odd |= odd8<T>(*(const s16x8 *)(vb + 16 * x));
            if (!__syncthreads_or(odd != 0)) return;
            put_sums();
#pragma unroll 1
            for (int token = 0; token < 32; ++token)
#pragma unroll 1
                for (int x = 0; x < NB * DT * 4; ++x) {
                    const int nb = x / (DT * 4), d = (x % (DT * 4)) * 8 + 4 * half, t = t0 + token;
                    const s16x4 y = *(const s16x4 *)(vb + token * ROW + (((d / 8) ^ W::v_swizzle(token)) << 4) + (d % 8) * 2);
                    const bool seen = t >= (nb ? see_lo[NB - 1] : see_lo[0]) && t < (nb ? see_hi[NB - 1] : see_hi[0]);
                    float *p = sums + (x * 64 + lane) * 4;
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (seen && !finite16<T>(y[i])) p[i] += value16<T>(y[i]);
                }
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                    for (int r = 0; r < 16; r += 4) {
                        const f32x4 y = *(const f32x4 *)(sums + (((nb * DT + dt) * 4 + r / 4) * 64 + lane) * 4);
                        o[nb][dt][r] = y[0], o[nb][dt][r + 1] = y[1], o[nb][dt][r + 2] = y[2], o[nb][dt][r + 3] = y[3];
                    }
            __syncthreads();
#pragma unroll 1
            for (int x = tid; x < 32 * CH * 8; x += 256) {
                short *p = (short *)vb + x;
                if (!finite16<T>(*p)) *p = 0;
            }
            __syncthreads();
        };
        auto partly_seen = [&](int t0) { return t0 < tile_lo || t0 + 32 > tile_hi; };

        // Tile i's keys are needed from the second half of tile i - 1 on, its
        // values until the first half of tile i + 1: one barrier a tile, in
        // its middle, and loads half a tile to a tile and a half ahead.
        __syncthreads();                       // the previous rows' products have read their buffers
        int page[L], ahead[L];
        find_pages(first, page);
        find_pages(first + 1, ahead);
        load(first, page, kh, k_in, a.k_page, a.k_slot, k_lds);
#pragma unroll
        for (int i = 0; i < L; ++i) *(uint4 *)(values + TILE + (i * 256 + tid) * 16) = uint4{0, 0, 0, 0};   // "before"
        arrived();
        __syncthreads();
        load(first, page, vh, v_in, a.v_page, a.v_slot, v_lds);
        load(first + 1, ahead, kh, k_in, a.k_page, a.k_slot, k_lds + TILE);
#pragma unroll
        for (int i = 0; i < L; ++i) page[i] = ahead[i];
        find_pages(first + 2, ahead);
        if (active) multiply(keys);
        for (int step = first; step < last; ++step) {
            const int b = (step - first) & 1, t0 = step * BN;
            char *k_now = keys + b * TILE, *k_next = keys + (b ^ 1) * TILE, *v_now = values + b * TILE, *v_before = values + (b ^ 1) * TILE;
            if (step > first && partly_seen(t0 - 32)) odd_values(t0 - 32, v_before + 32 * ROW);
            if (active) step32(t0, k_now + 32 * ROW, v_before + 32 * ROW);
            arrived();
            __syncthreads();
            if (step + 1 < last) {
                load(step + 1, page, vh, v_in, a.v_page, a.v_slot, v_lds + (b ^ 1) * TILE);
                load(step + 2, ahead, kh, k_in, a.k_page, a.k_slot, k_lds + b * TILE);
#pragma unroll
                for (int i = 0; i < L; ++i) page[i] = ahead[i];
                find_pages(step + 3, ahead);
            }
            if (partly_seen(t0)) odd_values(t0, v_now);
            if (active) step32(t0 + 32, k_next, v_now);
        }
        {
            char *v_last = values + ((last - 1 - first) & 1) * TILE + 32 * ROW;
            const int t0 = last * BN - 32;
            if (partly_seen(t0)) odd_values(t0, v_last);
            if (active) add(v_last);
        }

        const bool starts = from == 0, ends = last == range.first + range.count;
        walk.at += last - first;
        if (starts && ends) {
            if (active) {
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    const float sum = l[nb] + __shfl_xor(l[nb], 32), scale = sum == 0 ? 0.0f : 1.0f / sum;
                    const int r = row_base + nb * 32 + col, j = r / a.group;
                    if (r >= rows) continue;
                    const int64_t token = q0 + j, hq = (int64_t)head * a.group + r - j * a.group;
                    const int64_t to = token * a.out_token + hq * a.out_head;
                    if (a.lse && half == 0)
                        a.lse[token * a.heads + hq] = sum == 0 ? -INFINITY : 0.693147180559945f * (m[nb] + __builtin_amdgcn_logf(sum));
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                        for (int x = 0; x < 16; x += 4) {
                            const int d = dt * 32 + 2 * x + 4 * half;
                            if (d < 8 * a.units)
                                store4<T>(a, to + d, f32x4{o[nb][dt][x] * scale, o[nb][dt][x + 1] * scale,
                                                           o[nb][dt][x + 2] * scale, o[nb][dt][x + 3] * scale});
                        }
                }
            }
        } else {
            // unnormalised sums, in the order of the registers
            if (active) {
                put_sums();
                float *st = sums - wave * NB * 32 * DP + M * DP + wave * NB * 64;
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    const float sum = l[nb] + __shfl_xor(l[nb], 32);
                    st[nb * 64 + lane] = half ? sum : m[nb];
                }
            }
            if (!starts && tid == 0) {
                const int64_t t0 = walk.tile_at;
                const int w0 = Walk<M, BN>::owner(t0, walk.total, walk.workers);
                const int w1 = Walk<M, BN>::owner(t0 + range.count - 1, walk.total, walk.workers);
                if (w0 + 1 == walk.worker) a.parts[walk.worker] = Part{w1 - w0 + 1, e + walk.base, head, tile, q0, n};
            }
        }
        if (ends && walk.at < walk.end) walk.next(a, ent);
    }
}

// Joins the parts of a tile: workgroup (w, block of 32 rows); the waves share
// the dimensions.
template <class T, int DP, int NB>
__global__ __launch_bounds__(256) void k_kv_join_wide(Attn a) {
    constexpr int M = 128 * NB, DT = DP / 32;
    const int w = blockIdx.x, block = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5;
    const Part part = a.parts[w];
    if (part.count == 0) return;
    const int rows = part.n * a.group, r = part.tile * M + block * 32 + (lane & 31);
    if (part.tile * M + block * 32 >= rows) return;
    // part i: worker w - 1 + i; the first one's second slot, the others' first
    auto sums = [&](int i) { return a.sums + ((int64_t)(w - 1 + i) * 2 + (i == 0)) * (M * (DP + 2)); };
    float m = -INFINITY;
    for (int i = 0; i < part.count; ++i) m = fmaxf(m, sums(i)[M * DP + block * 64 + (lane & 31)]);
    const float base = m == -INFINITY ? 0.0f : m;
    float l = 0;
    f32x4 o[(DT + 3) / 4][4] = {};
    for (int i = 0; i < part.count; ++i) {
        const float *p = sums(i), *st = p + M * DP + block * 64 + (lane & 31);
        const float f = __builtin_amdgcn_exp2f(st[0] - base);
        l += st[32] * f;
#pragma unroll
        for (int k = 0; k < (DT + 3) / 4; ++k)
            if (wave + 4 * k < DT)
#pragma unroll
                for (int x = 0; x < 4; ++x)
                    o[k][x] += f * *(const f32x4 *)(p + block * 32 * DP + (((wave + 4 * k) * 4 + x) * 64 + lane) * 4);
    }
    if (r >= rows) return;
    const int j = r / a.group;
    const int64_t token = part.q0 + j, h = (int64_t)part.head * a.group + r - j * a.group;
    const float scale = l == 0 ? 0.0f : 1.0f / l;
    if (a.lse && wave == 0 && half == 0)
        a.lse[token * a.heads + h] = l == 0 ? -INFINITY : 0.693147180559945f * (m + __builtin_amdgcn_logf(l));
#pragma unroll
    for (int k = 0; k < (DT + 3) / 4; ++k)
        if (wave + 4 * k < DT)
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int d = (wave + 4 * k) * 32 + 8 * x + 4 * half;
                if (d < 8 * a.units) store4<T>(a, token * a.out_token + h * a.out_head + d, o[k][x] * scale);
            }
}

template <class T, int DP, int NB>
static void launch(const Attn &a, hipStream_t s) {
    {
        mptlib::LaunchScope scope("k_kv_wide", (double)a.n_tokens * a.heads, s);
        if (a.cap != 0)
            k_kv_wide<T, DP, NB, true><<<a.workers, 256, 0, s>>>(a);
        else
            k_kv_wide<T, DP, NB, false><<<a.workers, 256, 0, s>>>(a);
    }
    mptlib::LaunchScope scope("k_kv_join_wide", a.workers, s);
    k_kv_join_wide<T, DP, NB><<<dim3(a.workers, 4 * NB), 256, 0, s>>>(a);
}

template <class T>
static void launch(const Attn &a, int blocks32, hipStream_t s) {
    const int dim = pad_dim(8 * a.units);
    if (dim == 64)
        blocks32 == 1 ? launch<T, 64, 1>(a, s) : launch<T, 64, 2>(a, s);
    else if (dim == 128)
        blocks32 == 1 ? launch<T, 128, 1>(a, s) : launch<T, 128, 2>(a, s);
    else
        launch<T, 256, 1>(a, s);
}

void launch_wide(const Attn &a, int blocks32, hipStream_t s) {
    if (a.c.dtype == MPT_KV_BF16)
        launch<__bf16>(a, blocks32, s);
    else
        launch<_Float16>(a, blocks32, s);
}

}  // namespace mptkv
