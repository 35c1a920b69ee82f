// Attention of new tokens over the paged key/value cache: checks, the choice
// of a kernel and its workspace.

#include "attention.h"

#include <cmath>

namespace mptkv {

using mptlib::fail;

// Which kernel, and how many workers: what the card holds at once.
struct Choice {
    int waves;               // of a workgroup of the wide kernel, 32 rows each; 0: the narrow kernel
    int workers, rows;       // workgroups, rows of a tile
};

// By the rows that an entry has for a key head on average, and for heads of 128
// by whether a tile can have a CU for itself. The call knows neither the lengths
// nor how the tokens are spread over the entries (both are on the device), so
// decodes beside one long chunk go by the mean of the two, and the rule stands
// between the figures for short contexts and for long ones.
// Microseconds, narrow / 4 waves / 8 waves, 4 query heads on each of 8 key
// heads (other groups go by the rows alone):
//   dim 128, 32 entries over 4000 tokens: 16 rows 115/130/122; 32 rows
//   123/131/122; 48 rows 297/138/122; 128 rows 444/149/124; 160 rows
//   555/159/145; 256 rows 890/219/170. 32 over 300: 48 rows 32/28/26; 128 rows
//   48/33/31. 8 over 4000: 48 rows 73/50/45; 128 rows 76/67/52; over 300 20/23/23
//   dim 128, 128 entries over 300: 16 rows 36/43/66; 32 rows 60/44/66; 48 rows
//   86/47/69; 128 rows 205/65/92; 256 rows 436/118/130. 128 over 4000: 48 rows
//   1049/401/398; 128 rows 2733/416/447
//   dim 64, 32 entries over 4000: 16 rows 53/62/67; 20 rows 94/61/65; 128 rows
//   327/73/75; 256 rows 633/111/105. 128 over 4000: 128 rows 1445/250/292; 160
//   rows 1817/425/349
//   dim 256, 32 entries over 2000: 16 rows 105/121; 20 rows 195/119
// The limit of 32 rows for heads of 128 was drawn when 4 waves took 164 us where
// they now take 131 and 52 where they take 44: at 17 to 32 rows narrow tiles no
// longer gain.
static Choice choose(const mpt_kv_cache &c, int n, int64_t n_tokens, int n_q_heads) {
    const int64_t rows = (n_tokens + (n > 0 ? n : 1) - 1) / (n > 0 ? n : 1) * (n_q_heads / c.n_heads);
    const int dim = pad_dim(c.head_dim);
    const bool own_cu = dim == 128 && (int64_t)n * c.n_heads <= 256;
    if (rows <= (dim == 128 ? 32 : 16)) return {0, dim == 256 ? 256 : dim == 128 ? 512 : 768, 16};
    if ((rows <= 128 && !own_cu) || dim == 256) return {4, dim == 256 ? 256 : 512, 128};
    return {8, 256, 256};
}

static size_t attention_bytes(const mpt_kv_cache &c, int n, int64_t n_tokens, int n_q_heads) {
    const Choice ch = choose(c, n, n_tokens, n_q_heads);
    return mptlib::align256(sizeof(Part) * ch.workers) +
           mptlib::align256(sizeof(float) * 2 * ch.workers * ch.rows * (size_t)(pad_dim(c.head_dim) + 2));
}

}  // namespace mptkv

using namespace mptkv;

extern "C" size_t mpt_kv_attention_workspace_bytes(const mpt_kv_cache *cache, int n, int64_t n_tokens, int n_q_heads) {
    mptlib::clear_error();
    if (check_cache(cache) != MPT_OK || n < 0 || n > MPT_KV_MAX_ENTRIES || n_tokens < 0 || n_tokens > (1 << 30) || n_q_heads < 1 ||
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
        if (n < 0 || n > MPT_KV_MAX_ENTRIES || n_tokens < 0 || n_tokens > (1 << 30))
            return fail(MPT_E_INVALID, "n = %d, n_tokens = %lld", n, (long long)n_tokens);
        if (n_q_heads < 1 || n_q_heads > 65535 || n_q_heads % cache->n_heads)
            return fail(MPT_E_INVALID, "n_q_heads = %d is no multiple of the cache's %d", n_q_heads, cache->n_heads);
        if (out_dtype != cache->dtype && out_dtype != MPT_KV_F32)
            return fail(MPT_E_INVALID, "out_dtype = %d is neither the cache's type nor MPT_KV_F32", out_dtype);
        if (n_tokens * (n_q_heads / cache->n_heads) > (1 << 30))
            return fail(MPT_E_INVALID, "%lld tokens with %d query heads a key head", (long long)n_tokens,
                        n_q_heads / cache->n_heads);
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
        const Choice ch = choose(*cache, n, n_tokens, n_q_heads);
        Attn a = {};
        a.c = *cache;
        a.layer = layer, a.n = n, a.n_tokens = (int)n_tokens, a.heads = n_q_heads, a.group = n_q_heads / cache->n_heads;
        a.units = cache->head_dim / 8;
        int bits = 0;                                       // ceil(log2 group)
        while ((1 << bits) < a.group) ++bits;
        a.div_mul = (uint32_t)(((uint64_t)((1 << bits) - a.group) << 32) / a.group + 1);
        a.div_s1 = bits < 1 ? bits : 1, a.div_s2 = bits > 1 ? bits - 1 : 0;
        a.seqs = seqs, a.q_off = q_off, a.kv_begin = kv_begin;
        a.q = (const char *)q, a.out = (char *)out, a.lse = lse;
        a.q_token = q_token_stride, a.q_head = q_head_stride, a.out_token = out_token_stride, a.out_head = out_head_stride;
        a.out_f32 = out_dtype == MPT_KV_F32, a.causal = causal != 0, a.flip = scale < 0;
        a.window = window < (1 << 30) ? window : 0;         // no sequence is longer
        const float log2e = 1.44269504088896341f;
        // not 0, which times the minus infinity of a hidden token would be NaN
        a.factor = std::fmax(softcap > 0 ? std::fabs(scale) / softcap : std::fabs(scale) * log2e, 1e-37f);
        if (!std::isfinite(a.factor) || !std::isfinite(softcap * log2e))
            return fail(MPT_E_INVALID, "scale = %g, softcap = %g", scale, softcap);
        a.cap = softcap * log2e;
        for (int i = 1; i < 3; ++i)
            if (cache->k_stride[i] / 8 * (i == 2 ? cache->page_size : 1) > UINT32_MAX ||
                cache->v_stride[i] / 8 * (i == 2 ? cache->page_size : 1) > UINT32_MAX)
                return fail(MPT_E_INVALID, "cache: a page, or the stride of pages, of 64 GiB or more");
        a.k_page = (uint32_t)(cache->k_stride[1] / 8), a.k_slot = (uint32_t)(cache->k_stride[2] / 8);
        a.v_page = (uint32_t)(cache->v_stride[1] / 8), a.v_slot = (uint32_t)(cache->v_stride[2] / 8);
        const auto near = [&](uint64_t page, uint64_t slot) {
            return cache->n_pages <= 1 << 24 && page < 1 << 24 &&
                   (cache->n_pages - 1) * page + (cache->page_size - 1) * slot + a.units <= 1 << 28;
        };
        a.near = near(a.k_page, a.k_slot) && near(a.v_page, a.v_slot);
        a.k = (const char *)cache->k + 2 * layer * cache->k_stride[0];
        a.v = (const char *)cache->v + 2 * layer * cache->v_stride[0];
        a.k_head = 2 * cache->k_stride[3], a.v_head = 2 * cache->v_stride[3];
        a.workers = ch.workers;
        a.parts = (Part *)workspace;
        a.sums = (float *)((char *)workspace + mptlib::align256(sizeof(Part) * ch.workers));
        if (ch.waves)
            launch_wide(a, ch.waves, s);
        else
            launch_narrow(a, s);
        MPT_HIP_TRY(hipGetLastError());
        return MPT_OK;
    });
}
