// Attention kernel for few rows per key head (decoding): tiles of 16 rows. The
// four waves of a workgroup take 32 tokens each of a step of 128 and are
// joined at the end of the tile.
//
// The work is one pass over keys and values: 2 x 2 D bytes a token against
// 16 x 4 D flops, a few hundredths of what the matrix cores could do, so a
// wave only has to keep loads in flight. Keys go from memory to registers as
// the operand of S' = K Q' (16x16x32), one step ahead; values go to the
// wave's own LDS, one step ahead, and come back transposed as the operand of
// O' += V' P'. No barrier until the tile's end.

#include "attention.h"

namespace mptkv {

template <int DP>
struct Narrow {
    static constexpr int M = 16, BN = 128, KK = DP / 32, DT = DP / 16, ROW = 2 * DP, CH = DP / 8;
    static constexpr int kTile = 32 * ROW, L = kTile / 1024;           // a wave's values of a step; loads of 1 KiB

    // Eight tokens' 32 bytes fall on all banks.
    __device__ static int swizzle(int token) { return DP == 64 ? 2 * ((token >> 1) & 3) : 2 * (token & 7); }
};

template <class T, int DP, bool CAP>
__global__ __launch_bounds__(256, DP == 256 ? 1 : 2) void k_kv_narrow(Attn a) {
    using N = Narrow<DP>;
    constexpr int M = N::M, BN = N::BN, KK = N::KK, DT = N::DT, ROW = N::ROW, CH = N::CH, L = N::L;
    __shared__ Entries ent;
    __shared__ __attribute__((aligned(1024))) char v0[4 * N::kTile], v1[4 * N::kTile];
    __shared__ float stat[4][2][16];
    const mpt_kv_cache &c = a.c;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 15, quad = lane >> 4;
    const int shift = 31 - __clz(c.page_size);
    char *vw0 = v0 + wave * N::kTile, *vw1 = v1 + wave * N::kTile;

    Walk<M, BN> walk;
    if (!walk.begin(a, ent, 1)) return;

    while (walk.at < walk.end) {
        const int e = walk.e, n = ent.n[e], len = ent.len[e], q0 = ent.q0[e], slot = ent.slot[e];
        const Range range = tile_range<M, BN>(a, n, len, ent.begin[e], walk.tile);
        const int64_t from = walk.at - walk.tile_at;
        const int first = range.first + (int)from;
        const int last = range.first + (int)min((int64_t)range.count, from + (walk.end - walk.at));
        const int head = walk.head, rows = n * a.group;
        const int32_t *table = c.table + (int64_t)slot * c.max_pages;

        const int r = walk.tile * M + col, rr = min(r, rows - 1), j = rr / a.group, hq = rr - j * a.group, p = len - n + j;
        const int see_hi = a.causal ? min(len, p + 1) : len;
        const int see_lo = a.window ? max(ent.begin[e], p + 1 - a.window) : ent.begin[e];
        const int64_t token = q0 + j, hh = (int64_t)head * a.group + hq;
        int all_lo = see_lo, all_hi = see_hi;
        for (int d = 1; d < 16; d <<= 1) all_lo = max(all_lo, __shfl_xor(all_lo, d)), all_hi = min(all_hi, __shfl_xor(all_hi, d));
        s16x8 qf[KK];
        {
            const char *q = a.q + 2 * (token * a.q_token + hh * a.q_head);
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) {
                const int piece = 4 * kk + quad;
                uint4 x = *(const uint4 *)(r < rows && piece < a.units ? q + 16 * piece : (const char *)kZeros);
                if (a.flip) x.x ^= 0x80008000u, x.y ^= 0x80008000u, x.z ^= 0x80008000u, x.w ^= 0x80008000u;
                qf[kk] = __builtin_bit_cast(s16x8, x);
            }
        }
        f32x4 o[DT];
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[dt] = f32x4{0, 0, 0, 0};
        float m = -INFINITY, l = 0;

        // lane t < 32 knows the page of token t of the wave's part of a step
        auto find_page = [&](int step) {
            const int t = step * BN + wave * 32 + (lane & 31);
            int page = -1;
            if (t >= range.lo && t < range.hi) {
                page = table[t >> shift];
                if ((unsigned)page >= (unsigned)c.n_pages) {
                    flag(c, MPT_KV_BAD_PAGE);
                    page = -1;
                }
            }
            return page;
        };
        const char *kh = a.k + head * a.k_head + 16 * quad, *vh = a.v + head * a.v_head;
        auto load_v = [&](int step, int pages, char *vb) {
#pragma unroll
            for (int i = 0; i < L; ++i) {
                const int tok = i * (64 / CH) + lane / CH, piece = (lane % CH) ^ N::swizzle(tok);
                const int page = __shfl(pages, tok), t = step * BN + wave * 32 + tok;
                const char *vf = vh + row_at(page, t & (c.page_size - 1), a.v_page, a.v_slot) + 16 * piece;
                load_lds16(page >= 0 && piece < a.units ? vf : (const char *)kZeros, vb + i * 1024);
            }
        };
        struct Keys { s16x8 f[2][KK]; };
        auto load_k = [&](int step, int pages, Keys &k) {
#pragma unroll
            for (int mt = 0; mt < 2; ++mt) {
                const int page = __shfl(pages, mt * 16 + col), t = step * BN + wave * 32 + mt * 16 + col;
                const char *kf = page >= 0 ? kh + row_at(page, t & (c.page_size - 1), a.k_page, a.k_slot) : (const char *)kZeros;
#pragma unroll
                for (int kk = 0; kk < KK; ++kk)
                    k.f[mt][kk] = *(const s16x8 *)(page >= 0 && 4 * kk + quad < a.units ? kf + 64 * kk : (const char *)kZeros);
            }
        };
        auto compute = [&](int step, const Keys &k, const char *vb) {
            const int t0 = step * BN + wave * 32;
            if (t0 >= range.hi) return;
            float s[8];
#pragma unroll
            for (int mt = 0; mt < 2; ++mt) {
                f32x4 x = {0, 0, 0, 0};
#pragma unroll
                for (int kk = 0; kk < KK; ++kk) x = Type<T>::mfma16(k.f[mt][kk], qf[kk], x);
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
            typename Type<T>::x8 w;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float x = __builtin_amdgcn_exp2f(s[i] - base);
                l += x;
                w[i] = (T)x;
            }
            const s16x8 pf = __builtin_bit_cast(s16x8, w);
            auto read_v = [&](int dt) {
                const int row = 4 * quad + col / 4, piece = dt * 2 + (lane & 3) / 2;
                const char *q = vb + row * ROW + ((piece ^ N::swizzle(row)) << 4) + (lane & 1) * 8;
                const s16x4 x = read_column4(q), y = read_column4(q + 16 * ROW);
                return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
            };
            s16x8 vf[DT];
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) vf[dt] = read_v(dt);
            if (masked) {
                // a weight of zero does not cancel an infinity or NaN in a
                // value that the row does not see
                uint32_t odd = 0;
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) odd |= odd8<T>(vf[dt]);
                if (__any(odd != 0)) {
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                        for (int i = 0; i < 8; ++i) vf[dt][i] = finite16<T>(vf[dt][i]) ? vf[dt][i] : (short)0;
#pragma unroll 1
                    for (int tok = 0; tok < 32; ++tok) {
                        const bool seen = t0 + tok >= see_lo && t0 + tok < see_hi;
#pragma unroll
                        for (int dt = 0; dt < DT; ++dt) {
                            const int d = dt * 16 + 4 * quad;
                            const s16x4 x = *(const s16x4 *)(vb + tok * ROW + (((d / 8) ^ N::swizzle(tok)) << 4) + (d % 8) * 2);
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                if (seen && !finite16<T>(x[i])) o[dt][i] += value16<T>(x[i]);
                        }
                    }
                }
            }
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) o[dt] = Type<T>::mfma16(vf[dt], pf, o[dt]);
        };

        Keys ka, kb;
        int pages = find_page(first);
        load_v(first, pages, vw0);
        load_k(first, pages, ka);
        pages = find_page(first + 1);
        for (int step = first; step < last; step += 2) {
            if (step + 1 < last) {
                load_v(step + 1, pages, vw1);
                load_k(step + 1, pages, kb);
                pages = find_page(step + 2);
            }
            compute(step, ka, vw0);
            if (step + 1 >= last) break;
            if (step + 2 < last) {
                load_v(step + 2, pages, vw0);
                load_k(step + 2, pages, ka);
                pages = find_page(step + 3);
            }
            compute(step + 1, kb, vw1);
        }

        // the waves' parts: sums in the waves' halves of the two buffers
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        __syncthreads();
        if (quad == 0) stat[wave][0][col] = m, stat[wave][1][col] = l;
        // DT vectors of 1 KiB a wave: half of them in each buffer
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) *(f32x4 *)((dt % 2 ? v1 : v0) + ((dt / 2) * 4 + wave) * 1024 + lane * 16) = o[dt];
        __syncthreads();
        float f[4], all_m = -INFINITY, all_l = 0;
        for (int w = 0; w < 4; ++w) all_m = fmaxf(all_m, stat[w][0][col]);
        const float base = all_m == -INFINITY ? 0.0f : all_m;
        for (int w = 0; w < 4; ++w) {
            f[w] = __builtin_amdgcn_exp2f(stat[w][0][col] - base);
            all_l += f[w] * stat[w][1][col];
        }
        const bool starts = from == 0, ends = last == range.first + range.count;
        walk.at += last - first;
        const float scale = !(starts && ends) ? 1.0f : all_l == 0 ? 0.0f : 1.0f / all_l;
        float *sums = a.sums + ((int64_t)walk.worker * 2 + (starts ? 1 : 0)) * (M * (DP + 2));
#pragma unroll
        for (int k = 0; k < DT / 4; ++k) {
            const int dt = k * 4 + wave;
            f32x4 x = {0, 0, 0, 0};
#pragma unroll
            for (int w = 0; w < 4; ++w) x += f[w] * *(const f32x4 *)((dt % 2 ? v1 : v0) + ((dt / 2) * 4 + w) * 1024 + lane * 16);
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
                const int w0 = Walk<M, BN>::owner(walk.tile_at, walk.total, walk.workers);
                const int w1 = Walk<M, BN>::owner(walk.tile_at + range.count - 1, walk.total, walk.workers);
                if (w0 + 1 == walk.worker) a.parts[walk.worker] = Part{w1 - w0 + 1, e + walk.base, head, walk.tile, q0, n};
            }
        }
        __syncthreads();                      // the buffers are free again
        if (ends && walk.at < walk.end) walk.next(a, ent);
    }
}

// Joins the parts of a tile, as k_kv_join_wide: workgroup w, the waves share
// the dimensions.
template <class T, int DP>
__global__ __launch_bounds__(256) void k_kv_join_narrow(Attn a) {
    constexpr int M = 16, DT = DP / 16, K = DT / 4;
    const int w = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, quad = lane >> 4;
    const Part part = a.parts[w];
    if (part.count == 0) return;
    auto sums = [&](int i) { return a.sums + ((int64_t)(w - 1 + i) * 2 + (i == 0)) * (M * (DP + 2)); };
    float m = -INFINITY;
    for (int i = 0; i < part.count; ++i) m = fmaxf(m, sums(i)[M * DP + col]);
    const float base = m == -INFINITY ? 0.0f : m;
    float l = 0;
    f32x4 o[K] = {};
    for (int i = 0; i < part.count; ++i) {
        const float *p = sums(i);
        const float f = __builtin_amdgcn_exp2f(p[M * DP + col] - base);
        l += p[M * DP + 16 + col] * f;
#pragma unroll
        for (int k = 0; k < K; ++k) o[k] += f * *(const f32x4 *)(p + ((k * 4 + wave) * 64 + lane) * 4);
    }
    const int rows = part.n * a.group, r = part.tile * M + col;
    if (r >= rows) return;
    const int j = r / a.group;
    const int64_t token = part.q0 + j, h = (int64_t)part.head * a.group + r - j * a.group;
    const float scale = l == 0 ? 0.0f : 1.0f / l;
    if (a.lse && wave == 0 && quad == 0)
        a.lse[token * a.heads + h] = l == 0 ? -INFINITY : 0.693147180559945f * (m + __builtin_amdgcn_logf(l));
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int d = (k * 4 + wave) * 16 + 4 * quad;
        if (d < 8 * a.units) store4<T>(a, token * a.out_token + h * a.out_head + d, o[k] * scale);
    }
}

template <class T, int DP>
static void launch(const Attn &a, hipStream_t s) {
    {
        mptlib::LaunchScope scope("k_kv_narrow", (double)a.n_tokens * a.heads, s);
        if (a.cap != 0)
            k_kv_narrow<T, DP, true><<<a.workers, 256, 0, s>>>(a);
        else
            k_kv_narrow<T, DP, false><<<a.workers, 256, 0, s>>>(a);
    }
    mptlib::LaunchScope scope("k_kv_join_narrow", a.workers, s);
    k_kv_join_narrow<T, DP><<<a.workers, 256, 0, s>>>(a);
}

template <class T>
static void launch_dim(const Attn &a, hipStream_t s) {
    const int dim = pad_dim(8 * a.units);
    dim == 64 ? launch<T, 64>(a, s) : dim == 128 ? launch<T, 128>(a, s) : launch<T, 256>(a, s);
}

void launch_narrow(const Attn &a, hipStream_t s) {
    if (a.c.dtype == MPT_KV_BF16)
        launch_dim<__bf16>(a, s);
    else
        launch_dim<_Float16>(a, s);
}

}  // namespace mptkv
