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

template <class T, int DP, int NB, bool CAP>
struct Wide {
    static constexpr int M = 128 * NB, BN = DP == 256 ? 32 : 64;
    static constexpr int MT = BN / 32, KK = DP / 16, DT = DP / 32, ROW = 2 * DP, CH = DP / 8;
    static constexpr int kTile = BN * ROW, kLoads = kTile / 4096;     // 16-byte loads per thread and tile

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
    using W = Wide<T, DP, NB, CAP>;
    constexpr int M = W::M, BN = W::BN, MT = W::MT, KK = W::KK, DT = W::DT, ROW = W::ROW, CH = W::CH, L = W::kLoads;
    __shared__ Entries ent;
    __shared__ __attribute__((aligned(1024))) char k0[W::kTile], v0[W::kTile], k1[W::kTile], v1[W::kTile];
    const mpt_kv_cache &c = a.c;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 31, half = lane >> 5;
    const int shift = 31 - __clz(c.page_size);

    Walk<M, BN> walk;
    if (!walk.begin(a, ent, 4)) return;

    while (walk.at < walk.end) {
        const int e = walk.e, n = ent.n[e], len = ent.len[e], q0 = ent.q0[e], slot = ent.slot[e];
        const Range range = tile_range<M, BN>(a, n, len, ent.begin[e], walk.tile);
        const int64_t from = walk.at - walk.tile_at;
        const int first = range.first + (int)from;
        const int last = range.first + (int)min((int64_t)range.count, from + (walk.end - walk.at));
        const int head = walk.head, rows = n * a.group, row_base = walk.tile * M + wave * 32 * NB;
        const int32_t *table = c.table + (int64_t)slot * c.max_pages;
        const bool active = row_base < rows;

        // queries of the wave's blocks: operand pieces, and what each may see
        s16x8 qf[NB][KK];
        int see_lo[NB], see_hi[NB], wave_lo = 0, wave_hi = 1 << 30;
        int64_t out_at[NB];
        int64_t lse_at[NB];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            const int r = row_base + nb * 32 + col, rr = min(r, rows - 1), j = rr / a.group, hq = rr - j * a.group;
            const int p = len - n + j;
            see_hi[nb] = a.causal ? min(len, p + 1) : len;
            see_lo[nb] = a.window ? max(ent.begin[e], p + 1 - a.window) : ent.begin[e];
            const int64_t token = q0 + j, h = (int64_t)head * a.group + hq;
            out_at[nb] = r < rows ? token * a.out_token + h * a.out_head : -1;
            lse_at[nb] = token * a.heads + h;
            const char *q = a.q + 2 * (token * a.q_token + h * a.q_head);
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) {
                const int piece = 2 * kk + half;
                uint4 x = *(const uint4 *)(r < rows && piece < a.units ? q + 16 * piece : (const char *)kZeros);
                if (a.flip) x.x ^= 0x80008000u, x.y ^= 0x80008000u, x.z ^= 0x80008000u, x.w ^= 0x80008000u;
                qf[nb][kk] = __builtin_bit_cast(s16x8, x);
            }
            int lo = see_lo[nb], hi = see_hi[nb];
            for (int d = 1; d < 32; d <<= 1) lo = max(lo, __shfl_xor(lo, d)), hi = min(hi, __shfl_xor(hi, d));
            wave_lo = max(wave_lo, lo), wave_hi = min(wave_hi, hi);
        }
        // tokens that all rows of the tile see
        int tile_lo, tile_hi;
        {
            const int ra = walk.tile * M, rb = min(ra + M, rows) - 1;
            const int pa = len - n + ra / a.group, pb = len - n + rb / a.group;
            tile_hi = a.causal ? min(len, pa + 1) : len;
            tile_lo = a.window ? max(ent.begin[e], pb + 1 - a.window) : ent.begin[e];
        }
        f32x16 o[NB][DT];
        float m[NB], l[NB];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            m[nb] = -INFINITY, l[nb] = 0;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[nb][dt][r] = 0;
        }

        // the thread's tokens of a step, its piece of their rows, their pages
        const int own = tid / CH;
        const int kp = (tid % CH) ^ W::k_swizzle(own), vp = (tid % CH) ^ W::v_swizzle(own);
        const char *kh = a.k + head * a.k_head + 16 * kp, *vh = a.v + head * a.v_head + 16 * vp;
        const bool k_in = kp < a.units, v_in = vp < a.units;
        int page[L];
        auto find_pages = [&](int step) {
#pragma unroll
            for (int i = 0; i < L; ++i) {
                const int t = step * BN + i * W::kStride + own;
                page[i] = t >= range.lo && t < range.hi ? table[t >> shift] : -1;
            }
        };
        auto load = [&](int step, char *kb, char *vb) {
#pragma unroll
            for (int i = 0; i < L; ++i) {
                const int t = step * BN + i * W::kStride + own;
                const bool there = (unsigned)page[i] < (unsigned)c.n_pages;
                if (!there && t >= range.lo && t < range.hi) flag(c, MPT_KV_BAD_PAGE);
                const uint32_t slot = t & (c.page_size - 1);
                load_lds16(there && k_in ? kh + row_at(page[i], slot, a.k_page, a.k_slot) : (const char *)kZeros, kb + (i * 4 + wave) * 1024);
                load_lds16(there && v_in ? vh + row_at(page[i], slot, a.v_page, a.v_slot) : (const char *)kZeros, vb + (i * 4 + wave) * 1024);
            }
        };
        // scores and weights of a step
        s16x8 pf[NB][MT * 2];
        auto weigh = [&](int step, const char *kb) {
            const int t0 = step * BN;
            f32x16 s[MT][NB];
            const int k_row = col * ROW, k_flip = half ^ W::k_swizzle(col);
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[mt][nb][r] = 0;
#pragma unroll
                for (int kk = 0; kk < KK; ++kk) {
                    const s16x8 kf = *(const s16x8 *)(kb + mt * 32 * ROW + k_row + (((2 * kk) ^ k_flip) << 4));
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) s[mt][nb] = Type<T>::mfma32(kf, qf[nb][kk], s[mt][nb]);
                }
            }
            // tokens that some row of the wave does not see
            const bool masked = t0 < wave_lo || t0 + BN > wave_hi;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[mt][nb][r] = score<CAP>(a, s[mt][nb][r]);
                if (masked) {
                    const int t1 = t0 + 4 * half;
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                        for (int r = 0; r < 16; ++r) {
                            const int t = t1 + mt * 32 + 8 * (r / 4) + r % 4;
                            if (!(t >= see_lo[nb] && t < see_hi[nb])) s[mt][nb][r] = -INFINITY;
                        }
                }
                float top = -INFINITY;
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int r = 0; r < 16; ++r) top = fmaxf(top, s[mt][nb][r]);
                if (__any(top > m[nb] + 8.0f)) {
                    top = fmaxf(top, __shfl_xor(top, 32));
                    const float now = fmaxf(m[nb], top), keep = now == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m[nb] - now);
                    m[nb] = now;
                    l[nb] *= keep;
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                        for (int r = 0; r < 16; ++r) o[nb][dt][r] *= keep;
                }
                const float base = m[nb] == -INFINITY ? 0.0f : m[nb];
                typename Type<T>::x8 p;
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const float x = __builtin_amdgcn_exp2f(s[mt][nb][r] - base);
                        l[nb] += x;
                        p[r % 8] = (T)x;
                        if (r % 8 == 7) pf[nb][mt * 2 + r / 8] = __builtin_bit_cast(s16x8, p);
                    }
            }
        };
        // O' += V' P'
        auto add = [&](const char *vb) {
            const int row = 4 * half + (lane & 15) / 4;
            const int v_row = row * ROW + (lane & 1) * 8, v_piece = ((lane >> 4) & 1) * 2 + (lane & 3) / 2;
#pragma unroll
            for (int g = 0; g < MT * 2; ++g)
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) {
                    const char *p = vb + g * 16 * ROW + v_row + (((dt * 4 + v_piece) ^ W::v_swizzle(row)) << 4);
                    const s16x4 x = read_column4(p), y = read_column4(p + 8 * ROW);
                    const s16x8 vf = __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) o[nb][dt] = Type<T>::mfma32(vf, pf[nb][g], o[nb][dt]);
                }
        };
        // Infinities and NaN in values: a weight of zero does not cancel them
        // in a row that does not see them. Rows that do see them get them
        // added here; then they are zeros for the product.
        auto odd_values = [&](int step, char *vb) {
            uint32_t odd = 0;
#pragma unroll 1
            for (int x = tid; x < BN * CH; x += 256) odd |= odd8<T>(*(const s16x8 *)(vb + 16 * x));
            if (!__syncthreads_or(odd != 0)) return;
#pragma unroll 1
            for (int token = 0; token < BN; ++token)
#pragma unroll
                for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                    for (int r = 0; r < 16; r += 4) {
                        const int d = dt * 32 + 2 * r + 4 * half;
                        const s16x4 x = *(const s16x4 *)(vb + token * ROW + (((d / 8) ^ W::v_swizzle(token)) << 4) + (d % 8) * 2);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float y = finite16<T>(x[i]) ? 0.0f : value16<T>(x[i]);
#pragma unroll
                            for (int nb = 0; nb < NB; ++nb)
                                if (step * BN + token >= see_lo[nb] && step * BN + token < see_hi[nb]) o[nb][dt][r + i] += y;
                        }
                    }
            __syncthreads();
#pragma unroll 1
            for (int x = tid; x < BN * CH * 8; x += 256) {
                short *p = (short *)vb + x;
                if (!finite16<T>(*p)) *p = 0;
            }
            __syncthreads();
        };
        auto compute = [&](int step, const char *kb, char *vb) {
            if (active) weigh(step, kb);
            if (step * BN < tile_lo || step * BN + BN > tile_hi) odd_values(step, vb);
            if (active) add(vb);
        };

        __syncthreads();                       // the previous tile's last products have read their buffers
        find_pages(first);
        load(first, k0, v0);
        find_pages(first + 1);
        for (int step = first; step < last; step += 2) {
            __syncthreads();
            if (step + 1 < last) {
                load(step + 1, k1, v1);
                find_pages(step + 2);
            }
            compute(step, k0, v0);
            if (step + 1 >= last) break;
            __syncthreads();
            if (step + 2 < last) {
                load(step + 2, k0, v0);
                find_pages(step + 3);
            }
            compute(step + 1, k1, v1);
        }

        const bool starts = from == 0, ends = last == range.first + range.count;
        walk.at += last - first;
        if (starts && ends) {
            if (active) {
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    const float sum = l[nb] + __shfl_xor(l[nb], 32), scale = sum == 0 ? 0.0f : 1.0f / sum;
                    if (out_at[nb] < 0) continue;
                    if (a.lse && half == 0)
                        a.lse[lse_at[nb]] = sum == 0 ? -INFINITY : 0.693147180559945f * (m[nb] + __builtin_amdgcn_logf(sum));
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                        for (int r = 0; r < 16; r += 4) {
                            const int d = dt * 32 + 2 * r + 4 * half;
                            if (d < 8 * a.units)
                                store4<T>(a, out_at[nb] + d, f32x4{o[nb][dt][r] * scale, o[nb][dt][r + 1] * scale,
                                                                   o[nb][dt][r + 2] * scale, o[nb][dt][r + 3] * scale});
                        }
                }
            }
        } else {
            // unnormalised sums, in the order of the registers
            float *sums = a.sums + ((int64_t)walk.worker * 2 + (starts ? 1 : 0)) * (M * (DP + 2));
            if (active) {
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    const int block = wave * NB + nb;
                    float *p = sums + block * 32 * DP;
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                        for (int r = 0; r < 16; r += 4)
                            *(f32x4 *)(p + ((dt * 4 + r / 4) * 64 + lane) * 4) =
                                f32x4{o[nb][dt][r], o[nb][dt][r + 1], o[nb][dt][r + 2], o[nb][dt][r + 3]};
                    const float sum = l[nb] + __shfl_xor(l[nb], 32);
                    float *st = sums + M * DP + block * 64;
                    st[lane] = half ? sum : m[nb];
                }
            }
            if (!starts && tid == 0) {
                const int64_t t0 = walk.tile_at;
                const int w0 = Walk<M, BN>::owner(t0, walk.total, walk.workers);
                const int w1 = Walk<M, BN>::owner(t0 + range.count - 1, walk.total, walk.workers);
                if (w0 + 1 == walk.worker) a.parts[walk.worker] = Part{w1 - w0 + 1, e + walk.base, head, walk.tile, q0, n};
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
