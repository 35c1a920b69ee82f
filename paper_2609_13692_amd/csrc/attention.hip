// Attention of new tokens over the paged key/value cache.

#include "kv.h"

#include <cmath>

namespace mptkv {

struct Attn {
    mpt_kv_cache c;
    int layer, n, n_tokens, heads, group;
    const int32_t *seqs, *q_off, *kv_begin;
    const char *q;
    char *out;
    int64_t q_token, q_head, out_token, out_head;
    float *lse;
    int out_f32, causal, window;
    float softcap, scale;
};

template <class T>
__global__ __launch_bounds__(256) void k_kv_attention(Attn a) {
    __shared__ float qs[MPT_KV_MAX_DIM], ps[4][64], part[4][MPT_KV_MAX_DIM], stat[4][2];
    const mpt_kv_cache &c = a.c;
    const int i = blockIdx.z, h = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, dim = c.head_dim;
    const int q0 = max(0, a.q_off[i]), q1 = min(a.n_tokens, a.q_off[i + 1]), s = a.seqs[i];
    const bool slot = s >= 0 && s < c.max_seqs;
    const int length = slot ? max(0, min(c.length[s], c.max_pages * c.page_size)) : 0;
    const int shift = 31 - __clz(c.page_size);
    for (int token = q0 + blockIdx.x; token < q1; token += gridDim.x) {
        const int pos = length - (q1 - token);
        int hi = a.causal ? min(length, pos + 1) : length;
        int lo = a.kv_begin ? max(0, a.kv_begin[i]) : 0;
        if (a.window > 0) lo = max(lo, pos + 1 - a.window);
        __syncthreads();
        for (int d = threadIdx.x; d < dim; d += 256)
            qs[d] = (float)((const T *)a.q)[token * a.q_token + h * a.q_head + d];
        __syncthreads();
        float m = -INFINITY, l = 0, o[4] = {};
        for (int base = lo + wave * 64; base < hi; base += 256) {
            const int t = base + lane;
            float x = -INFINITY;
            if (t < hi) {
                const int page = c.table[(int64_t)s * c.max_pages + (t >> shift)];
                x = 0;
                if (page >= 0 && page < c.n_pages) {
                    const T *k = (const T *)c.k + a.layer * c.k_stride[0] + page * c.k_stride[1] +
                                 (t & (c.page_size - 1)) * c.k_stride[2] + (h / a.group) * c.k_stride[3];
                    for (int d = 0; d < dim; ++d) x += qs[d] * (float)k[d];
                } else {
                    flag(c, MPT_KV_BAD_PAGE);
                }
                x *= a.scale;
                if (a.softcap > 0) x = a.softcap * tanhf(x / a.softcap);
            }
            float top = x;
            for (int w = 1; w < 64; w <<= 1) top = fmaxf(top, __shfl_xor(top, w));
            const float now = fmaxf(m, top), use = now == -INFINITY ? 0 : now;
            const float keep = expf(m - use), p = expf(x - use);
            float sum = p;
            for (int w = 1; w < 64; w <<= 1) sum += __shfl_xor(sum, w);
            l = l * keep + sum;
            m = now;
            ps[wave][lane] = p;
            for (int r = 0; r < 4; ++r) o[r] *= keep;
            for (int j = 0; j < 64 && base + j < hi; ++j) {
                const int page = c.table[(int64_t)s * c.max_pages + ((base + j) >> shift)];
                if (page < 0 || page >= c.n_pages) continue;
                const T *v = (const T *)c.v + a.layer * c.v_stride[0] + page * c.v_stride[1] +
                             ((base + j) & (c.page_size - 1)) * c.v_stride[2] + (h / a.group) * c.v_stride[3];
                for (int r = 0; r < 4; ++r)
                    if (r * 64 + lane < dim) o[r] += ps[wave][j] * (float)v[r * 64 + lane];
            }
        }
        for (int r = 0; r < 4; ++r) part[wave][r * 64 + lane] = o[r];
        if (lane == 0) stat[wave][0] = m, stat[wave][1] = l;
        __syncthreads();
        float top = -INFINITY, sum = 0;
        for (int w = 0; w < 4; ++w) top = fmaxf(top, stat[w][0]);
        const float use = top == -INFINITY ? 0 : top;
        for (int w = 0; w < 4; ++w) sum += stat[w][1] * expf(stat[w][0] - use);
        const float inv = sum == 0 ? 0 : 1 / sum;
        for (int d = threadIdx.x; d < dim; d += 256) {
            float x = 0;
            for (int w = 0; w < 4; ++w) x += part[w][d] * expf(stat[w][0] - use);
            x *= inv;
            const int64_t at = token * a.out_token + h * a.out_head + d;
            if (a.out_f32)
                ((float *)a.out)[at] = x;
            else
                ((T *)a.out)[at] = (T)x;
        }
        if (a.lse && threadIdx.x == 0)
            a.lse[(int64_t)token * a.heads + h] = sum == 0 ? -INFINITY : use + logf(sum);
    }
    if (!slot && threadIdx.x == 0) flag(c, MPT_KV_BAD_SLOT);
}

using mptlib::fail;

static size_t attention_bytes(const mpt_kv_cache &, int, int64_t, int) { return 256; }

}  // namespace mptkv

using namespace mptkv;

extern "C" size_t mpt_kv_attention_workspace_bytes(const mpt_kv_cache *cache, int n, int64_t n_tokens, int n_q_heads) {
    mptlib::clear_error();
    if (check_cache(cache) != MPT_OK || n < 0 || n_tokens < 0 || n_tokens > INT32_MAX || n_q_heads < 1 ||
        n_q_heads > 65535 || n_q_heads % cache->n_heads)
        return 0;
    return attention_bytes(*cache, n, n_tokens, n_q_heads);
}

extern "C" int mpt_kv_attention(const mpt_kv_cache *cache, int layer, int n, const int32_t *seqs, const int32_t *q_off,
                                int64_t n_tokens, int n_q_heads, const void *q, int64_t q_token_stride,
                                int64_t q_head_stride, void *out, int64_t out_token_stride, int64_t out_head_stride,
                                int out_dtype, float *lse, const int32_t *kv_begin, int causal, int window,
                                float softcap, float scale, void *workspace, size_t workspace_bytes, void *stream) {
    mptlib::clear_error();
    return mptlib::guarded(__func__, [&]() -> int {
        if (int rc = check_cache(cache)) return rc;
        if (layer < 0 || layer >= cache->n_layers) return fail(MPT_E_INVALID, "layer = %d", layer);
        if (n < 0 || n > (1 << 20) || n_tokens < 0 || n_tokens > INT32_MAX)
            return fail(MPT_E_INVALID, "n = %d, n_tokens = %lld", n, (long long)n_tokens);
        if (n_q_heads < 1 || n_q_heads > 65535 || n_q_heads % cache->n_heads)
            return fail(MPT_E_INVALID, "n_q_heads = %d is no multiple of the cache's %d", n_q_heads, cache->n_heads);
        if (out_dtype != cache->dtype && out_dtype != MPT_KV_F32)
            return fail(MPT_E_INVALID, "out_dtype = %d is neither the cache's type nor MPT_KV_F32", out_dtype);
        if (window < 0 || !(softcap >= 0) || !std::isfinite(softcap) || !std::isfinite(scale))
            return fail(MPT_E_INVALID, "window = %d, softcap = %g, scale = %g", window, softcap, scale);
        if (n == 0 || n_tokens == 0) return MPT_OK;
        if (!seqs || !q_off || !q || !out) return fail(MPT_E_INVALID, "an array is NULL");
        if (!aligned16(q) || !aligned16(out)) return fail(MPT_E_INVALID, "q and out must be 16-byte aligned");
        if ((q_token_stride | q_head_stride | out_token_stride | out_head_stride) % 8)
            return fail(MPT_E_INVALID, "strides must be multiples of 8");
        const size_t need = attention_bytes(*cache, n, n_tokens, n_q_heads);
        if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < need)
            return fail(MPT_E_WORKSPACE, "workspace %p of %zu bytes: needs %zu, 256-byte aligned", workspace,
                        workspace_bytes, need);
        hipStream_t s = (hipStream_t)stream;
        Attn a = {*cache, layer, n, (int)n_tokens, n_q_heads, n_q_heads / cache->n_heads, seqs, q_off, kv_begin,
                  (const char *)q, (char *)out, q_token_stride, q_head_stride, out_token_stride, out_head_stride, lse,
                  out_dtype == MPT_KV_F32, causal != 0, window, softcap, scale};
        {
            mptlib::LaunchScope scope("k_kv_attention", (double)n_tokens * n_q_heads, s);
            const dim3 grid((unsigned)(n_tokens < 1024 ? n_tokens : 1024), n_q_heads, n);
            if (n > 65535) return fail(MPT_E_INVALID, "n = %d", n);
            if (cache->dtype == MPT_KV_BF16)
                k_kv_attention<__bf16><<<grid, 256, 0, s>>>(a);
            else
                k_kv_attention<_Float16><<<grid, 256, 0, s>>>(a);
        }
        MPT_HIP_TRY(hipGetLastError());
        return MPT_OK;
    });
}
