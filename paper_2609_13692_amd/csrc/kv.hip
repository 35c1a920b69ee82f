// The paged key/value cache: pages of tables (forks, growth, frees,
// compaction), copies of their contents, appends, and the join of attention
// over parts of a context.
//
// A page call is two launches: one workgroup checks the lists and the pages
// that they refer to, sums up what they need and picks the pages (k_kv_plan,
// k_kv_plan_free, k_kv_plan_moves), and a wide launch applies it, or returns at
// once if the plan found an error. The pages of long lists are checked by a
// launch of their own before it.
// Free pages are the set bits of one word per 64 pages, so a pool of 2^20
// pages is picked from by reading 128 KiB.

#include "kv.h"

#include <cfloat>
#include <type_traits>

namespace mptkv {

constexpr int kSlotBits = 1 << 16;            // slots whose marks are bits in LDS

// A plan is one workgroup: small for short lists on small pools (a launch of a
// few microseconds either way: forks and growth of 9 entries on 1000 pages 8.3
// and 5.6 us with 1024 threads, 6.8 and 4.2 with 256), 16 waves where there is
// more to read.
inline int plan_threads(int n, int n_pages) { return n <= 512 && n_pages <= (1 << 16) ? 256 : 1024; }

// The first 256 bytes of the workspace: what a plan tells its second launch
// and, where it asks, the host.
struct Head {
    uint32_t err;
    int32_t moves;      // pages that move (compaction, copies)
    int64_t value;      // free pages afterwards, live pages, or pages copied
};

struct Plan {
    Head *head;
    int32_t *a, *b;              // [n_pages]: fresh pages; or pages that move, and where to
    int32_t *start, *from, *mark;  // [max_seqs]: first fresh page of an entry, page whose tokens it copies; marks
};

static size_t plan_bytes(const mpt_kv_cache &c) {
    return 256 + 2 * mptlib::align256(4 * (size_t)c.n_pages) + 3 * mptlib::align256(4 * (size_t)c.max_seqs);
}

static Plan plan_at(const mpt_kv_cache &c, void *ws) {
    char *p = (char *)ws;
    const size_t pages = mptlib::align256(4 * (size_t)c.n_pages), seqs = mptlib::align256(4 * (size_t)c.max_seqs);
    Plan q;
    q.head = (Head *)p;
    q.a = (int32_t *)(p + 256);
    q.b = (int32_t *)(p + 256 + pages);
    q.start = (int32_t *)(p + 256 + 2 * pages);
    q.from = (int32_t *)(p + 256 + 2 * pages + seqs);
    q.mark = (int32_t *)(p + 256 + 2 * pages + 2 * seqs);
    return q;
}

// Exclusive sum over the workgroup's threads; *total is the whole sum.
template <int THREADS>
__device__ inline int64_t block_scan(int64_t v, int64_t *total, int64_t *lds) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t x = wave_sums(v);
    if (lane == 63) lds[wave] = x;
    __syncthreads();
    int64_t before = 0, all = 0;
    for (int w = 0; w < THREADS / 64; ++w) {
        const int64_t t = lds[w];
        if (w < wave) before += t;
        all += t;
    }
    __syncthreads();
    *total = all;
    return before + x - v;
}

__device__ inline int pages_of(const mpt_kv_cache &c, int tokens) {
    return (int)(((int64_t)tokens + c.page_size - 1) >> (31 - __clz(c.page_size)));
}

// A page of the pool that a table can refer to: one with references.
__device__ inline bool page_held(const mpt_kv_cache &c, int p) { return page_ok(c, p) && c.ref[p] > 0; }

// Listed indexes outside [0, bound) and those that two entries list: by bits
// in LDS where they fit, else by marks in memory (an index gets its entry's
// number there; the barriers order the stores, all in L2).
template <int THREADS>
__device__ inline uint32_t check_list(int n, const int32_t *list, int bound, int32_t *mark, uint32_t *bits, uint32_t bad) {
    uint32_t err = 0;
    const bool in_lds = bound <= kSlotBits;
    if (in_lds) {
        for (int i = threadIdx.x; i < (bound + 31) / 32; i += THREADS) bits[i] = 0;
    } else {
        for (int i = threadIdx.x; i < n; i += THREADS) {
            const int s = list[i];
            if (s >= 0 && s < bound) atomicExch(&mark[s], -1);
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += THREADS) {
        const int s = list[i];
        if (s < 0 || s >= bound)
            err |= bad;
        else if (in_lds ? atomicOr(&bits[s >> 5], 1u << (s & 31)) >> (s & 31) & 1 : atomicExch(&mark[s], i) != -1)
            err |= MPT_KV_DUPLICATE;
    }
    return err;
}

// Whether one of the pages first .. last - 1 of slot s cannot be referred to, a
// lane each, four on their way at a time.
__device__ inline bool bad_pages(const mpt_kv_cache &c, int s, int first, int last, int lane, int step) {
    const int32_t *row = c.table + (int64_t)s * c.max_pages;
    bool bad = false;
    for (int j = first + lane; j < last; j += 4 * step) {
        int page[4], ref[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) page[u] = row[j + u * step < last ? j + u * step : j];
#pragma unroll
        for (int u = 0; u < 4; ++u) ref[u] = c.ref[page_ok(c, page[u]) ? page[u] : 0];
#pragma unroll
        for (int u = 0; u < 4; ++u) bad |= !page_ok(c, page[u]) || ref[u] < 1;
    }
    return bad;
}

// Pages that a fork shares: keep / page_size of slot s, none if the two are refused.
__device__ inline int shared_pages(const mpt_kv_cache &c, int s, int keep) {
    if (!slot_ok(c, s) || keep < 0 || keep > c.length[s]) return 0;
    return min(keep / c.page_size, c.max_pages);
}

// Pages of slot s that a cut to k tokens drops end there (0: the two are refused).
__device__ inline int dropped_end(const mpt_kv_cache &c, int s, int k) {
    const int now = slot_ok(c, s) ? c.length[s] : 0;
    return k < 0 || k > now || now > (int64_t)c.max_pages * c.page_size ? 0 : pages_of(c, now);
}

// Lists and tables whose pages one workgroup checks beside its plan (0.4 us for
// 9 entries of 45 pages, whose chains of reads overlap); past it a launch before
// the plan does, a workgroup per entry (4.5 us for 48 of up to 560).
constexpr int64_t kSmallTables = 8192;

// The pages that forks of list[i] share, or that cuts of it drop.
template <bool DROP>
__global__ __launch_bounds__(256) void k_kv_check(mpt_kv_cache c, const int32_t *list, const int32_t *keep, Plan p) {
    const int i = blockIdx.x, s = list[i], k = keep ? keep[i] : 0;
    const int first = DROP ? pages_of(c, k) : 0, last = DROP ? dropped_end(c, s, k) : shared_pages(c, s, k);
    const int any = __syncthreads_or(bad_pages(c, s, first, last, threadIdx.x, 256));
    if (threadIdx.x == 0) p.from[i] = any;
}

// Plan of forks (src != null) and growth: checks, pages needed and the
// lowest-numbered free pages in ascending order, which leave free_bits here.
// Each thread owns a run of words, so ranks are one sum over the workgroup.
template <int THREADS>
__global__ __launch_bounds__(THREADS) void k_kv_plan(mpt_kv_cache c, int n, const int32_t *src, const int32_t *dst,
                                                     const int32_t *keep, const int32_t *new_len, bool checked, Plan p) {
    __shared__ int64_t lds[THREADS / 64];
    __shared__ uint32_t slots[kSlotBits / 32];
    __shared__ uint32_t err_all;
    const int tid = threadIdx.x;
    // the free pages first: their words are on their way beside the lists
    const int words = (c.n_pages + 63) / 64, per = (words + THREADS - 1) / THREADS;
    const int w0 = tid * per < words ? tid * per : words, w1 = w0 + per < words ? w0 + per : words;
    int64_t mine = 0;
    for (int w = w0; w < w1; ++w) mine += __popcll(c.free_bits[w]);
    if (tid == 0) err_all = 0;
    __syncthreads();
    uint32_t err = check_list<THREADS>(n, dst, c.max_seqs, p.mark, slots, MPT_KV_BAD_SLOT);
    // sixteen lanes an entry: the chains of reads of as many at a time
    if (src && !checked)
        for (int i = tid >> 4; i < n; i += THREADS / 16)
            if (bad_pages(c, src[i], 0, shared_pages(c, src[i], keep[i]), tid & 15, 16)) err |= MPT_KV_BAD_PAGE;
    const int64_t most = (int64_t)c.max_pages * c.page_size;
    int64_t need_all = 0;
    for (int base = 0; base < n; base += THREADS) {
        const int i = base + tid;
        int64_t need = 0;
        if (i < n) {
            const int d = dst[i], now = slot_ok(c, d) ? c.length[d] : 0, want = new_len[i];
            int from = -1, k;
            if (src) {
                const int s = src[i];
                k = keep[i];
                if (checked && p.from[i]) err |= MPT_KV_BAD_PAGE;
                if (s < -1 || s >= c.max_seqs)
                    err |= MPT_KV_BAD_SLOT;
                else if (k < 0 || k > (s < 0 ? 0 : c.length[s]) || want < k || want > most)
                    err |= MPT_KV_BAD_LENGTH;
                else {
                    const int full = k / c.page_size;
                    if (k % c.page_size) {
                        from = c.table[(int64_t)s * c.max_pages + full];
                        if (!page_held(c, from)) err |= MPT_KV_BAD_PAGE;
                    }
                    need = pages_of(c, want) - full;
                }
                if (now != 0) err |= MPT_KV_NOT_EMPTY;
            } else if (now < 0 || want < now || want > most) {
                err |= MPT_KV_BAD_LENGTH;
            } else {
                need = pages_of(c, want) - pages_of(c, now);
                // a last page with room that others refer to is copied first
                if (want > now && now % c.page_size && slot_ok(c, d)) {
                    const int page = c.table[(int64_t)d * c.max_pages + now / c.page_size];
                    if (!page_held(c, page)) {
                        err |= MPT_KV_BAD_PAGE;
                    } else if (c.ref[page] > 1) {
                        from = page;
                        ++need;
                    }
                }
            }
            p.from[i] = from;
        }
        int64_t sum;
        const int64_t at = need_all + block_scan<THREADS>(need, &sum, lds);
        need_all += sum;
        if (i < n) {
            p.start[i] = (int32_t)(at < c.n_pages ? at : c.n_pages);
            // the marks have been looked at: the tokens that the slot has now
            if (slot_ok(c, dst[i])) p.mark[dst[i]] = src ? keep[i] : c.length[dst[i]];
        }
    }
    int64_t free_all, at = block_scan<THREADS>(mine, &free_all, lds);
    if (need_all > free_all) err |= MPT_KV_NO_PAGES;
    if (err) atomicOr(&err_all, err);
    __syncthreads();
    err = err_all;
    if (tid == 0) {
        p.head->err = err;
        p.head->value = err ? free_all : free_all - need_all;
        if (err) flag(c, err);
    }
    if (err) return;
    for (int w = w0; w < w1 && at < need_all; ++w) {
        uint64_t bits = c.free_bits[w];
        while (bits && at < need_all) {
            p.a[at++] = w * 64 + __ffsll((unsigned long long)bits) - 1;
            bits &= bits - 1;
        }
        c.free_bits[w] = bits;
    }
}

// One tensor's rows of the first `tokens` slots, page a to page b of a layer:
// 16 bytes per lane and step, in the order in which the rows lie in memory.
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ inline void copy_rows(char *base, const int64_t *stride, int64_t layer, int a, int b, int tokens,
                                 int page_size, int heads, int units) {
    const int64_t from = layer * stride[0] + (int64_t)a * stride[1], to = layer * stride[0] + (int64_t)b * stride[1];
    const bool slots_inside = stride[2] < stride[3];
    // rows without gaps between them: as one run
    const int64_t row_size = units * 8, other = (slots_inside ? page_size : heads) * row_size;
    if ((slots_inside ? stride[2] == row_size && stride[3] == other && tokens == page_size
                      : stride[3] == row_size && stride[2] == other)) {
        const char *a0 = base + 2 * from;
        char *b0 = base + 2 * to;
        const int total = tokens * heads * units;
        // eight loads on their way at a time, of short runs too (one after the
        // other, the tokens of a partial page took seven round trips)
        for (int x = threadIdx.x; x < total; x += 8 * blockDim.x) {
            u32x4 v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u)
                if (x + u * (int)blockDim.x < total) v[u] = __builtin_nontemporal_load((const u32x4 *)a0 + x + u * blockDim.x);
#pragma unroll
            for (int u = 0; u < 8; ++u)
                if (x + u * (int)blockDim.x < total) __builtin_nontemporal_store(v[u], (u32x4 *)b0 + x + u * blockDim.x);
        }
        return;
    }
    const int inner = slots_inside ? tokens : heads, total = tokens * heads * units;
    const int64_t s_in = slots_inside ? stride[2] : stride[3], s_out = slots_inside ? stride[3] : stride[2];
    int x = threadIdx.x;
    for (; x + 3 * (int)blockDim.x < total; x += 4 * blockDim.x) {
        uint4 v[4];
        int64_t off[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int y = x + u * blockDim.x, row = y / units, o = row / inner;
            off[u] = o * s_out + (row - o * inner) * s_in + (y - row * units) * 8;
            v[u] = *(const uint4 *)(base + 2 * (from + off[u]));
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) *(uint4 *)(base + 2 * (to + off[u])) = v[u];
    }
    for (; x < total; x += blockDim.x) {
        const int row = x / units, o = row / inner;
        const int64_t off = o * s_out + (row - o * inner) * s_in + (x - row * units) * 8;
        *(uint4 *)(base + 2 * (to + off)) = *(const uint4 *)(base + 2 * (from + off));
    }
}

// The bytes E of the same rows, in words W that divide a row. Rows without gaps
// go as one run, of 16 bytes where its ends are aligned to that.
template <class W>
__device__ inline void copy_words(char *base, int64_t from, int64_t to, int64_t s_slot, int64_t s_head, int tokens, int heads,
                                  int words) {
    const int total = tokens * heads * words;
    for (int x = threadIdx.x; x < total; x += blockDim.x) {
        const int row = x / words, head = row / tokens;
        const int64_t off = head * s_head + (row - head * tokens) * s_slot + (x - row * words) * (int)sizeof(W);
        *(W *)(base + to + off) = *(const W *)(base + from + off);
    }
}
__device__ inline void copy_scales(char *base, const int64_t *stride, int64_t layer, int a, int b, int tokens, int page_size,
                                   int heads, int bytes) {
    const int64_t from = layer * stride[0] + (int64_t)a * stride[1], to = layer * stride[0] + (int64_t)b * stride[1];
    const int64_t run = (int64_t)tokens * heads * bytes;
    if (((stride[2] == bytes && stride[3] == (int64_t)page_size * bytes && tokens == page_size) ||
         (stride[3] == bytes && stride[2] == (int64_t)heads * bytes)) &&
        (((uintptr_t)base | (uint64_t)from | (uint64_t)to | (uint64_t)run) & 15) == 0) {
        for (int64_t x = 16 * (int)threadIdx.x; x < run; x += 16 * (int)blockDim.x)
            *(uint4 *)(base + to + x) = *(const uint4 *)(base + from + x);
        return;
    }
    if (bytes % 8 == 0)
        copy_words<uint64_t>(base, from, to, stride[2], stride[3], tokens, heads, bytes / 8);
    else if (bytes % 4 == 0)
        copy_words<uint32_t>(base, from, to, stride[2], stride[3], tokens, heads, bytes / 4);
    else if (bytes % 2 == 0)
        copy_words<uint16_t>(base, from, to, stride[2], stride[3], tokens, heads, bytes / 2);
    else
        copy_words<uint8_t>(base, from, to, stride[2], stride[3], tokens, heads, bytes);
}

// A reference less. A page that counts fewer than the tables have, which no
// look at one entry shows, stays at none.
__device__ inline void drop(const mpt_kv_cache &c, int page) {
    const int old = atomicSub(&c.ref[page], 1);
    if (old == 1) atomicOr((unsigned long long *)&c.free_bits[page >> 6], 1ull << (page & 63));
    if (old <= 0) {
        atomicAdd(&c.ref[page], 1);
        flag(c, MPT_KV_BAD_PAGE);
    }
}

// The bytes E of a cache in 4 bits; others launch without (with them, and a look at
// whether there are any, half of a cache replaced took 1617 us instead of 1613, 9
// requests forked, grown and freed 29.2 instead of 28.6).
struct NoScales {};
template <bool FOUR>
using ScalesOf = std::conditional_t<FOUR, Scales, NoScales>;

// Forks and growth as planned: workgroup (i, 0) writes entry i's row of the
// table and the references, workgroups (i, y) copy the keys or the values of
// a partial page's tokens in a layer.
template <bool FOUR>
__global__ __launch_bounds__(256) void k_kv_apply(mpt_kv_cache c, ScalesOf<FOUR> e, const int32_t *src, const int32_t *dst,
                                                  const int32_t *new_len, Plan p) {
    if (p.head->err) return;
    const int i = blockIdx.x, tid = threadIdx.x, d = dst[i], first = p.start[i], from = p.from[i];
    const int now = p.mark[d];                            // tokens that d has without its fresh pages
    const int full = now / c.page_size, part = now - full * c.page_size;
    if (from >= 0) {
        const int to = p.a[first], units = c.head_dim / 8;
        for (int y = blockIdx.y; y < 2 * c.n_layers; y += gridDim.y) {
            if (y & 1)
                copy_rows((char *)c.v, c.v_stride, y >> 1, from, to, part, c.page_size, c.n_heads, units);
            else
                copy_rows((char *)c.k, c.k_stride, y >> 1, from, to, part, c.page_size, c.n_heads, units);
            if constexpr (FOUR)
                copy_scales(y & 1 ? e.v : e.k, y & 1 ? e.v_stride : e.k_stride, y >> 1, from, to, part, c.page_size, c.n_heads,
                            e.bytes);
        }
    }
    if (blockIdx.y) return;
    int32_t *row = c.table + (int64_t)d * c.max_pages;
    const int total = pages_of(c, new_len[i]);
    const int have = src || from >= 0 ? full : pages_of(c, now);
    if (src && full) {
        const int32_t *other = c.table + (int64_t)src[i] * c.max_pages;
        for (int j = tid; j < full; j += blockDim.x) {
            const int page = other[j];
            row[j] = page;
            atomicAdd(&c.ref[page], 1);
        }
    }
    for (int j = have + tid; j < total; j += blockDim.x) {
        const int page = p.a[first + j - have];
        row[j] = page;
        c.ref[page] = 1;
    }
    if (tid == 0) {
        if (!src && from >= 0) drop(c, from);
        c.length[d] = new_len[i];
    }
}

template <int THREADS>
__device__ inline uint32_t check_free(const mpt_kv_cache &c, int n, const int32_t *seqs, const int32_t *keep, bool checked,
                                      const Plan &p) {
    __shared__ uint32_t err_all, slots[kSlotBits / 32];
    if (threadIdx.x == 0) err_all = 0;
    uint32_t err = check_list<THREADS>(n, seqs, c.max_seqs, p.mark, slots, MPT_KV_BAD_SLOT);
    const int64_t most = (int64_t)c.max_pages * c.page_size;
    for (int i = threadIdx.x; i < n; i += THREADS) {
        const int s = seqs[i], now = slot_ok(c, s) ? c.length[s] : 0, k = keep ? keep[i] : 0;
        if (k < 0 || k > now || now > most) err |= MPT_KV_BAD_LENGTH;
        if (checked && p.from[i]) err |= MPT_KV_BAD_PAGE;
    }
    if (!checked)
        for (int i = threadIdx.x >> 4; i < n; i += THREADS / 16) {
            const int s = seqs[i], k = keep ? keep[i] : 0;
            if (bad_pages(c, s, pages_of(c, k), dropped_end(c, s, k), threadIdx.x & 15, 16)) err |= MPT_KV_BAD_PAGE;
        }
    if (err) atomicOr(&err_all, err);
    __syncthreads();
    if (threadIdx.x == 0) {
        p.head->err = err_all;
        if (err_all) flag(c, err_all);
    }
    return err_all;
}

// Pages of slot s past its first k tokens, a lane each.
__device__ inline void drop_pages(const mpt_kv_cache &c, int s, int k, int now, int first, int step) {
    const int32_t *row = c.table + (int64_t)s * c.max_pages;
    for (int j = pages_of(c, k) + first; j < pages_of(c, now); j += step) drop(c, row[j]);
}

__global__ __launch_bounds__(1024) void k_kv_plan_free(mpt_kv_cache c, int n, const int32_t *seqs, const int32_t *keep, Plan p) {
    check_free<1024>(c, n, seqs, keep, true, p);
}

__global__ __launch_bounds__(256) void k_kv_free(mpt_kv_cache c, const int32_t *seqs, const int32_t *keep, Plan p) {
    if (p.head->err) return;
    const int s = seqs[blockIdx.x], k = keep ? keep[blockIdx.x] : 0, now = c.length[s];
    drop_pages(c, s, k, now, threadIdx.x, 256);
    __syncthreads();
    if (threadIdx.x == 0) c.length[s] = k;
}

// Checks and drops of short lists with short tables in one launch: a wave per
// sequence.
__global__ __launch_bounds__(1024) void k_kv_free_small(mpt_kv_cache c, int n, const int32_t *seqs, const int32_t *keep, Plan p) {
    if (check_free<1024>(c, n, seqs, keep, false, p)) return;
    const int lane = threadIdx.x & 63;
    for (int i = threadIdx.x >> 6; i < n; i += 16) {
        const int s = seqs[i], k = keep ? keep[i] : 0, now = c.length[s];
        drop_pages(c, s, k, now, lane, 64);
        if (lane == 0) c.length[s] = k;
    }
}

// Number of free pages, for calls whose caller asks.
__global__ __launch_bounds__(1024) void k_kv_count(mpt_kv_cache c, Plan p) {
    __shared__ int64_t lds[16];
    int64_t mine = 0, all;
    for (int w = threadIdx.x; w < (c.n_pages + 63) / 64; w += 1024) mine += __popcll(c.free_bits[w]);
    block_scan<1024>(mine, &all, lds);
    if (threadIdx.x == 0) p.head->value = all;
}

// The pages of all tables, a wave per slot.
__global__ __launch_bounds__(256) void k_kv_check_tables(mpt_kv_cache c, Plan p) {
    const int lane = threadIdx.x & 63;
    for (int64_t s = blockIdx.x * 4 + (threadIdx.x >> 6); s < c.max_seqs; s += gridDim.x * 4) {
        const int any = __any(bad_pages(c, (int)s, 0, min(pages_of(c, c.length[s]), c.max_pages), lane, 64));
        if (lane == 0) p.from[s] = any;
    }
}

// Plan of a compaction: the j-th used page from n_live on goes to the j-th
// free page below. a[j] and b[j] are the two; the words are rewritten here.
__global__ __launch_bounds__(1024) void k_kv_plan_moves(mpt_kv_cache c, Plan p) {
    __shared__ int64_t lds[16];
    bool bad = false;
    for (int64_t s = threadIdx.x; s < c.max_seqs; s += 1024) bad |= p.from[s] != 0;
    if (__syncthreads_or(bad)) {
        if (threadIdx.x == 0) {
            p.head->err = MPT_KV_BAD_PAGE;
            flag(c, MPT_KV_BAD_PAGE);
        }
        return;
    }
    const int tid = threadIdx.x, words = (c.n_pages + 63) / 64, per = (words + 1024 - 1) / 1024;
    const int w0 = tid * per < words ? tid * per : words, w1 = w0 + per < words ? w0 + per : words;
    int64_t mine = 0, free_all;
    for (int w = w0; w < w1; ++w) mine += __popcll(c.free_bits[w]);
    block_scan<1024>(mine, &free_all, lds);
    const int live = c.n_pages - (int)free_all;
    // bits of word w whose pages lie below x
    auto below = [](int w, int x) -> uint64_t {
        const int d = x - w * 64;
        return d <= 0 ? 0 : d >= 64 ? ~0ull : (1ull << d) - 1;
    };
    int64_t holes = 0, movers = 0, all;
    for (int w = w0; w < w1; ++w) {
        const uint64_t f = c.free_bits[w], lo = below(w, live), in = below(w, c.n_pages);
        holes += __popcll(f & lo);
        movers += __popcll(~f & ~lo & in);
    }
    int64_t h = block_scan<1024>(holes, &all, lds), m = block_scan<1024>(movers, &all, lds);
    for (int w = w0; w < w1; ++w) {
        const uint64_t f = c.free_bits[w], lo = below(w, live), in = below(w, c.n_pages);
        for (uint64_t x = ~f & ~lo & in; x; x &= x - 1) p.a[m++] = w * 64 + __ffsll((unsigned long long)x) - 1;
        for (uint64_t x = f & lo; x; x &= x - 1) p.b[h++] = w * 64 + __ffsll((unsigned long long)x) - 1;
        c.free_bits[w] = ~lo & in;
    }
    if (tid == 0) {
        p.head->err = 0;
        p.head->moves = (int)all;
        p.head->value = live;
    }
}

// Moves contents (every layer), references and the tables' entries. Bound by
// memory: 3.9 GB each way in 1.51 ms, 5.2 TB/s together (2048 workgroups, keys
// and values of a page apart, eight loads of 16 bytes a thread in flight) at
// pages of 16 slots of 8 heads of 128; at pages of one slot a workgroup has half
// a load a thread, which was not measured. Used
// pages that move are found from their number by a search in a, which
// ascends; no table entry below n_live changes.
template <bool FOUR>
__global__ __launch_bounds__(256) void k_kv_move(mpt_kv_cache c, ScalesOf<FOUR> e, Plan p, int tables) {
    const int moves = p.head->moves, units = c.head_dim / 8;
    if (p.head->err || moves == 0) return;
    for (int64_t x = blockIdx.x; x < 2ll * moves * c.n_layers; x += gridDim.x) {
        const int j = (int)(x / (2 * c.n_layers)), rest = (int)(x - (int64_t)j * 2 * c.n_layers);
        const int a = p.a[j], b = p.b[j];
        if (rest & 1)
            copy_rows((char *)c.v, c.v_stride, rest >> 1, a, b, c.page_size, c.page_size, c.n_heads, units);
        else
            copy_rows((char *)c.k, c.k_stride, rest >> 1, a, b, c.page_size, c.page_size, c.n_heads, units);
        if constexpr (FOUR)
            copy_scales(rest & 1 ? e.v : e.k, rest & 1 ? e.v_stride : e.k_stride, rest >> 1, a, b, c.page_size, c.page_size,
                        c.n_heads, e.bytes);
        if (tables && rest == 0 && threadIdx.x == 0) {
            c.ref[b] = c.ref[a];
            c.ref[a] = 0;
        }
    }
    if (!tables) return;
    const int live = (int)p.head->value;
    // in 64 bits: the next number past max_seqs, which may be 2^31 - 1
    for (int64_t s = blockIdx.x; s < c.max_seqs; s += gridDim.x) {
        int32_t *row = c.table + s * c.max_pages;
        const int pages = min(pages_of(c, c.length[s]), c.max_pages);
        for (int j = threadIdx.x; j < pages; j += 256) {
            const int page = row[j];
            if (page < live) continue;
            int lo = 0, hi = moves;
            while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                if (p.a[mid] < page)
                    lo = mid + 1;
                else
                    hi = mid;
            }
            if (lo < moves && p.a[lo] == page)
                row[j] = p.b[lo];
            else
                flag(c, MPT_KV_BAD_PAGE);
        }
    }
}

// Checks of a list of copies: marks of the destinations (each once, and none
// of them a source) in b, then the two lists in a and b.
__global__ __launch_bounds__(1024) void k_kv_plan_copy(mpt_kv_cache c, int n, const int32_t *src,
                                                               const int32_t *dst, Plan p) {
    __shared__ uint32_t err_all;
    if (threadIdx.x == 0) err_all = 0;
    uint32_t err = 0;
    for (int i = threadIdx.x; i < n; i += 1024)
        if (page_ok(c, src[i])) atomicExch(&p.b[src[i]], -1);
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += 1024)
        if (page_ok(c, dst[i])) atomicExch(&p.b[dst[i]], -1);
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += 1024) {
        if (!page_ok(c, dst[i]))
            err |= MPT_KV_BAD_PAGE;
        else if (atomicExch(&p.b[dst[i]], i) != -1)
            err |= MPT_KV_DUPLICATE;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += 1024) {
        if (!page_ok(c, src[i]))
            err |= MPT_KV_BAD_PAGE;
        else if (atomicAdd(&p.b[src[i]], 0) != -1)
            err |= MPT_KV_DUPLICATE;
    }
    if (err) atomicOr(&err_all, err);
    __syncthreads();
    err = err_all;
    for (int i = threadIdx.x; i < n; i += 1024) p.a[i] = src[i];
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += 1024) p.b[i] = dst[i];
    if (threadIdx.x == 0) {
        p.head->err = err;
        p.head->moves = n;
        p.head->value = err ? 0 : n;
        if (err) flag(c, err);
    }
}

__global__ __launch_bounds__(256) void k_kv_reset(mpt_kv_cache c) {
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x, step = (int64_t)gridDim.x * 256;
    for (int64_t i = at; i < c.n_pages; i += step) c.ref[i] = 0;
    for (int64_t i = at; i < c.max_seqs; i += step) c.length[i] = 0;
    for (int64_t i = at; i < (c.n_pages + 63) / 64; i += step)
        c.free_bits[i] = i < c.n_pages / 64 ? ~0ull : (1ull << (c.n_pages & 63)) - 1;
    if (at == 0) *c.status = 0;
}

__global__ void k_kv_clear_status(mpt_kv_cache c, uint32_t bits) { atomicAnd(c.status, ~bits); }

// One wave per token: the row of keys and the row of values, 16 bytes per lane.
// Bound by memory: 15763 tokens of 8 heads of 128 in 21 us (6 TB/s read and
// written); 64 tokens in 4, a launch.
__global__ __launch_bounds__(256) void k_kv_append(mpt_kv_cache c, int layer, int n, const int32_t *seqs,
                                                   const int32_t *q_off, int n_tokens, const char *k_new, int64_t kt,
                                                   int64_t kh, const char *v_new, int64_t vt, int64_t vh) {
    const int lane = threadIdx.x & 63, units = c.head_dim / 8, total = c.n_heads * units;
    const int shift = 31 - __clz(c.page_size);
    // in 64 bits: the next number past n_tokens, which may be 2^31 - 1
    for (int64_t token = blockIdx.x * 4 + (threadIdx.x >> 6); token < n_tokens; token += gridDim.x * 4) {
        const int i = wave_find(q_off, n, (int)token);
        if (i < 0 || i >= n || !slot_ok(c, seqs[i])) {
            if (lane == 0) flag(c, MPT_KV_BAD_SLOT);
            continue;
        }
        const int s = seqs[i], length = c.length[s];
        const int64_t pos = (int64_t)length - q_off[i + 1] + token;
        if (pos < 0 || pos >= length || (pos >> shift) >= c.max_pages) {
            if (lane == 0) flag(c, MPT_KV_BAD_LENGTH);
            continue;
        }
        const int page = c.table[(int64_t)s * c.max_pages + (pos >> shift)];
        if (!page_ok(c, page) || c.ref[page] != 1) {
            if (lane == 0) flag(c, page_ok(c, page) && c.ref[page] > 1 ? MPT_KV_SHARED : MPT_KV_BAD_PAGE);
            continue;
        }
        const int64_t slot = pos & (c.page_size - 1);
        char *ko = (char *)c.k + 2 * (layer * c.k_stride[0] + page * c.k_stride[1] + slot * c.k_stride[2]);
        char *vo = (char *)c.v + 2 * (layer * c.v_stride[0] + page * c.v_stride[1] + slot * c.v_stride[2]);
        const char *ki = k_new + 2 * (token * kt), *vi = v_new + 2 * (token * vt);
        for (int x = lane; x < total; x += 64) {
            const int h = x / units, u = (x - h * units) * 8;
            const uint4 a = *(const uint4 *)(ki + 2 * (h * kh + u)), b = *(const uint4 *)(vi + 2 * (h * vh + u));
            *(uint4 *)(ko + 2 * (h * c.k_stride[3] + u)) = a;
            *(uint4 *)(vo + 2 * (h * c.v_stride[3] + u)) = b;
        }
    }
}

struct Parts {
    const void *o[MPT_KV_MAX_PARTS];
    const float *lse[MPT_KV_MAX_PARTS];
};

template <int T>
__device__ inline void load8(const void *p, int64_t at, float *x) {
    if constexpr (T == MPT_KV_F32) {
        const float4 a = ((const float4 *)p)[at / 4], b = ((const float4 *)p)[at / 4 + 1];
        x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
    } else {
        union { uint4 u; __bf16 b[8]; _Float16 h[8]; } v;
        v.u = ((const uint4 *)p)[at / 8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = T == MPT_KV_BF16 ? (float)v.b[i] : (float)v.h[i];
    }
}

template <int T>
__device__ inline void store8(void *p, int64_t at, const float *x) {
    if constexpr (T == MPT_KV_F32) {
        ((float4 *)p)[at / 4] = make_float4(x[0], x[1], x[2], x[3]);
        ((float4 *)p)[at / 4 + 1] = make_float4(x[4], x[5], x[6], x[7]);
    } else {
        union { uint4 u; __bf16 b[8]; _Float16 h[8]; } v;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (T == MPT_KV_BF16)
                v.b[i] = (__bf16)x[i];
            else
                v.h[i] = (_Float16)x[i];
        }
        ((uint4 *)p)[at / 8] = v.u;
    }
}

// Eight elements of a row per thread, whole rows per workgroup. Every thread
// of a row forms the weights itself: n_parts exponentials against 8 n_parts
// products. Bound by memory: four parts of 8191 x 32 rows of 128 in 108 us, 5.6
// TB/s.
template <int TI, int TO>
__global__ __launch_bounds__(256) void k_kv_merge(int n_parts, int64_t rows, int dim, Parts p, void *out, float *lse) {
    const int units = dim / 8, per = 256 / units, r = threadIdx.x / units, u = threadIdx.x - r * units;
    const int64_t row = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * per + r, at = row * dim + u * 8;
    const bool there = r < per && row < rows;
    float top = -INFINITY, sum = 0, acc[8] = {}, total = 0;
    if (there) {
        for (int i = 0; i < n_parts; ++i) top = fmaxf(top, p.lse[i][row]);
        for (int i = 0; i < n_parts; ++i) {
            const float l = p.lse[i][row];
            if (l == -INFINITY) continue;
            float v[8];
            load8<TI>(p.o[i], at, v);
            const float w = expf(l - top);      // NaN where l is, or where the largest is +inf
            sum += w;
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[j] += w == 0 && fabsf(v[j]) == INFINITY ? v[j] : w * v[j];   // no NaN
        }
        const float scale = sum == 0 ? 0.0f : 1.0f / sum;
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] *= scale;
        total = sum == 0 ? -INFINITY : top + logf(sum);
    }
    __syncthreads();                             // lse may be one of the parts'
    if (!there) return;
    store8<TO>(out, at, acc);
    if (lse && u == 0) lse[row] = total;
}

// --- host side ------------------------------------------------------------

using mptlib::fail;

int check_cache(const mpt_kv_cache *c) {
    if (!c) return fail(MPT_E_INVALID, "cache is NULL");
    if (c->dtype < MPT_KV_BF16 || c->dtype > MPT_KV_F16_MX4 || c->dtype == MPT_KV_F32)
        return fail(MPT_E_INVALID, "cache: dtype = %d", c->dtype);
    if (c->n_layers < 1 || c->n_pages < 1 || c->n_pages > MPT_KV_MAX_PAGES)
        return fail(MPT_E_INVALID, "cache: n_layers = %d, n_pages = %d", c->n_layers, c->n_pages);
    if (c->page_size < 1 || c->page_size > MPT_KV_MAX_PAGE_SIZE || (c->page_size & (c->page_size - 1)))
        return fail(MPT_E_INVALID, "cache: page_size = %d is no power of two up to %d", c->page_size,
                    MPT_KV_MAX_PAGE_SIZE);
    if (c->n_heads < 1 || c->n_heads > 65535) return fail(MPT_E_INVALID, "cache: n_heads = %d", c->n_heads);
    if (c->head_dim < 8 || c->head_dim > MPT_KV_MAX_DIM || c->head_dim % 8)
        return fail(MPT_E_INVALID, "cache: head_dim = %d is no multiple of 8 up to %d", c->head_dim, MPT_KV_MAX_DIM);
    if (c->max_seqs < 1 || c->max_pages < 1 || (int64_t)c->max_pages * c->page_size > (1 << 30))
        return fail(MPT_E_INVALID, "cache: max_seqs = %d, max_pages = %d", c->max_seqs, c->max_pages);
    if (!c->k || !c->v || !c->table || !c->length || !c->ref || !c->free_bits || !c->status)
        return fail(MPT_E_INVALID, "cache: an array is NULL");
    if (!aligned16(c->k) || !aligned16(c->v)) return fail(MPT_E_INVALID, "cache: k and v must be 16-byte aligned");
    for (int i = 0; i < 4; ++i)
        if (c->k_stride[i] < 0 || c->v_stride[i] < 0 || c->k_stride[i] % 8 || c->v_stride[i] % 8)
            return fail(MPT_E_INVALID, "cache: strides must be multiples of 8, not negative");
    if (!is_mx4(*c)) return MPT_OK;
    if (c->head_dim % 32) return fail(MPT_E_INVALID, "cache: head_dim = %d in 4 bits is no multiple of 32", c->head_dim);
    const Scales e = scales_of(*c);
    if (!e.k || !e.v) return fail(MPT_E_INVALID, "cache: an array is NULL");
    const int word = e.bytes & -e.bytes;              // the largest power of two that divides a row
    if (((uintptr_t)e.k | (uintptr_t)e.v) & (word - 1))
        return fail(MPT_E_INVALID, "cache: k_scale and v_scale must be aligned to %d bytes", word);
    for (int i = 0; i < 4; ++i) {
        if (c->k_stride[i] % 16 || c->v_stride[i] % 16)
            return fail(MPT_E_INVALID, "cache: strides of codes must be multiples of 16 bytes");
        if (e.k_stride[i] < 0 || e.v_stride[i] < 0 || e.k_stride[i] % word || e.v_stride[i] % word)
            return fail(MPT_E_INVALID, "cache: strides of scales must be multiples of %d, not negative", word);
    }
    return MPT_OK;
}

// A cache in 4 bits as the page calls' launches take it: elements of two bytes. A
// row of head_dim / 2 bytes is one of head_dim / 4 of them.
static mpt_kv_cache in_two_bytes(const mpt_kv_cache &c) {
    mpt_kv_cache x = c;
    x.head_dim /= 4;
    for (int i = 0; i < 4; ++i) x.k_stride[i] /= 2, x.v_stride[i] /= 2;
    return x;
}

static void launch_move(const mpt_kv_cache &c, const Plan &p, int tables, hipStream_t s) {
    if (is_mx4(c))
        k_kv_move<true><<<2048, 256, 0, s>>>(in_two_bytes(c), scales_of(c), p, tables);
    else
        k_kv_move<false><<<2048, 256, 0, s>>>(c, {}, p, tables);
}

// Entries that a list of sequences can have: distinct slots, a workgroup each of
// a launch of less than 2^32 threads (a plan must not take pages that the
// launch after it cannot hand out).
static int list_limit(const mpt_kv_cache *c) { return !c ? 0 : c->max_seqs < MPT_KV_MAX_LIST ? c->max_seqs : MPT_KV_MAX_LIST; }
static_assert(MPT_KV_MAX_LIST * 256ull < 1ull << 32, "k_kv_apply and k_kv_free take 256 threads an entry");

static int check_plan(const mpt_kv_cache *c, int n, int most, void *ws, size_t bytes) {
    if (int rc = check_cache(c)) return rc;
    if (n < 0 || n > most) return fail(MPT_E_INVALID, "n = %d outside [0, %d]", n, most);
    const size_t need = plan_bytes(*c);
    if (!ws || ((uintptr_t)ws & 255) || bytes < need)
        return fail(MPT_E_WORKSPACE, "workspace %p of %zu bytes: needs %zu, 256-byte aligned", ws, bytes, need);
    return MPT_OK;
}

// The plan's verdict, for callers that ask for it.
static int report(const Plan &p, int64_t *value, const char *what, hipStream_t s) {
    MPT_HIP_TRY(hipGetLastError());
    if (!value) return MPT_OK;
    Head h;
    MPT_HIP_TRY(mptlib::read_back(&h, p.head, sizeof h, s));
    if (h.err & (MPT_KV_BAD_SLOT | MPT_KV_BAD_LENGTH | MPT_KV_BAD_PAGE))
        return fail(MPT_E_RANGE, "%s: a %s out of range", what,
                    h.err & MPT_KV_BAD_SLOT ? "slot" : h.err & MPT_KV_BAD_LENGTH ? "length" : "page");
    if (h.err & MPT_KV_DUPLICATE) return fail(MPT_E_DUP, "%s: listed twice", what);
    if (h.err & MPT_KV_NOT_EMPTY) return fail(MPT_E_STATE, "%s: a destination holds tokens", what);
    if (h.err & MPT_KV_NO_PAGES) return fail(MPT_E_PAGES, "%s: %lld free pages are too few", what, (long long)h.value);
    *value = h.value;
    return MPT_OK;
}

static int grow(const mpt_kv_cache *c, int n, const int32_t *src, const int32_t *dst, const int32_t *keep,
                const int32_t *new_len, int64_t *free_pages, void *ws, size_t bytes, hipStream_t s, const char *what) {
    if (int rc = check_plan(c, n, list_limit(c), ws, bytes)) return rc;
    const Plan p = plan_at(*c, ws);
    const bool checked = src && (int64_t)n * c->max_pages > kSmallTables;
    if (checked) {
        mptlib::LaunchScope scope("k_kv_check", n, s);
        k_kv_check<false><<<n, 256, 0, s>>>(*c, src, keep, p);
    }
    {
        mptlib::LaunchScope scope("k_kv_plan", n, s);
        if (plan_threads(n, c->n_pages) == 256)
            k_kv_plan<256><<<1, 256, 0, s>>>(*c, n, src, dst, keep, new_len, checked, p);
        else
            k_kv_plan<1024><<<1, 1024, 0, s>>>(*c, n, src, dst, keep, new_len, checked, p);
    }
    if (n) {
        mptlib::LaunchScope scope("k_kv_apply", n, s);
        const dim3 grid(n, c->n_layers < 32 ? 2 * c->n_layers : 64);
        if (is_mx4(*c))
            k_kv_apply<true><<<grid, 256, 0, s>>>(in_two_bytes(*c), scales_of(*c), src, dst, new_len, p);
        else
            k_kv_apply<false><<<grid, 256, 0, s>>>(*c, {}, src, dst, new_len, p);
    }
    if (free_pages && !src) {                  // copies of shared pages may have left some without references
        mptlib::LaunchScope scope("k_kv_count", c->n_pages, s);
        k_kv_count<<<1, 1024, 0, s>>>(*c, p);
    }
    return report(p, free_pages, what, s);
}

}  // namespace mptkv

using namespace mptkv;

extern "C" size_t mpt_kv_workspace_bytes(const mpt_kv_cache *cache) {
    mptlib::clear_error();
    return check_cache(cache) == MPT_OK ? plan_bytes(*cache) : 0;
}

extern "C" int mpt_kv_reset(const mpt_kv_cache *cache, void *stream) {
    mptlib::clear_error();
    return mptlib::guarded(__func__, [&]() -> int {
        if (int rc = check_cache(cache)) return rc;
        hipStream_t s = (hipStream_t)stream;
        {
            mptlib::LaunchScope scope("k_kv_reset", cache->n_pages, s);
            k_kv_reset<<<mptlib::grid_for(cache->n_pages, 256, 2048), 256, 0, s>>>(*cache);
        }
        MPT_HIP_TRY(hipGetLastError());
        return MPT_OK;
    });
}

extern "C" int mpt_kv_status(const mpt_kv_cache *cache, uint32_t *bits, void *stream) {
    mptlib::clear_error();
    return mptlib::guarded(__func__, [&]() -> int {
        if (int rc = check_cache(cache)) return rc;
        if (!bits) return fail(MPT_E_INVALID, "bits is NULL");
        hipStream_t s = (hipStream_t)stream;
        MPT_HIP_TRY(mptlib::read_back(bits, cache->status, sizeof *bits, s));
        if (*bits) {
            k_kv_clear_status<<<1, 1, 0, s>>>(*cache, *bits);
            MPT_HIP_TRY(hipGetLastError());
        }
        return MPT_OK;
    });
}

extern "C" int mpt_kv_fork(const mpt_kv_cache *cache, int n, const int32_t *src, const int32_t *dst,
                           const int32_t *keep, const int32_t *new_len, int64_t *free_pages, void *workspace,
                           size_t workspace_bytes, void *stream) {
    mptlib::clear_error();
    return mptlib::guarded(__func__, [&]() -> int {
        if (n > 0 && (!src || !dst || !keep || !new_len)) return fail(MPT_E_INVALID, "a list is NULL");
        return grow(cache, n, src, dst, keep, new_len, free_pages, workspace, workspace_bytes, (hipStream_t)stream,
                    "mpt_kv_fork");
    });
}

extern "C" int mpt_kv_extend(const mpt_kv_cache *cache, int n, const int32_t *seqs, const int32_t *new_len,
                             int64_t *free_pages, void *workspace, size_t workspace_bytes, void *stream) {
    mptlib::clear_error();
    return mptlib::guarded(__func__, [&]() -> int {
        if (n > 0 && (!seqs || !new_len)) return fail(MPT_E_INVALID, "a list is NULL");
        return grow(cache, n, nullptr, seqs, nullptr, new_len, free_pages, workspace, workspace_bytes,
                    (hipStream_t)stream, "mpt_kv_extend");
    });
}

extern "C" int mpt_kv_free(const mpt_kv_cache *cache, int n, const int32_t *seqs, const int32_t *keep,
                           int64_t *free_pages, void *workspace, size_t workspace_bytes, void *stream) {
    mptlib::clear_error();
    return mptlib::guarded(__func__, [&]() -> int {
        if (n > 0 && !seqs) return fail(MPT_E_INVALID, "seqs is NULL");
        if (int rc = check_plan(cache, n, list_limit(cache), workspace, workspace_bytes)) return rc;
        hipStream_t s = (hipStream_t)stream;
        const Plan p = plan_at(*cache, workspace);
        if ((int64_t)n * cache->max_pages <= kSmallTables) {
            mptlib::LaunchScope scope("k_kv_free_small", n, s);
            k_kv_free_small<<<1, 1024, 0, s>>>(*cache, n, seqs, keep, p);
        } else {
            {
                mptlib::LaunchScope scope("k_kv_check", n, s);
                k_kv_check<true><<<n, 256, 0, s>>>(*cache, seqs, keep, p);
            }
            {
                mptlib::LaunchScope scope("k_kv_plan_free", n, s);
                k_kv_plan_free<<<1, 1024, 0, s>>>(*cache, n, seqs, keep, p);
            }
            mptlib::LaunchScope scope("k_kv_free", n, s);
            k_kv_free<<<n, 256, 0, s>>>(*cache, seqs, keep, p);
        }
        if (free_pages) {
            mptlib::LaunchScope scope("k_kv_count", cache->n_pages, s);
            k_kv_count<<<1, 1024, 0, s>>>(*cache, p);
        }
        return report(p, free_pages, "mpt_kv_free", s);
    });
}

extern "C" int mpt_kv_compact(const mpt_kv_cache *cache, int64_t *live_pages, void *workspace, size_t workspace_bytes,
                              void *stream) {
    mptlib::clear_error();
    return mptlib::guarded(__func__, [&]() -> int {
        if (int rc = check_plan(cache, 0, 0, workspace, workspace_bytes)) return rc;
        hipStream_t s = (hipStream_t)stream;
        const Plan p = plan_at(*cache, workspace);
        {
            mptlib::LaunchScope scope("k_kv_check_tables", cache->max_seqs, s);
            k_kv_check_tables<<<mptlib::grid_for(cache->max_seqs, 4, 2048), 256, 0, s>>>(*cache, p);
        }
        {
            mptlib::LaunchScope scope("k_kv_plan_moves", cache->n_pages, s);
            k_kv_plan_moves<<<1, 1024, 0, s>>>(*cache, p);
        }
        {
            mptlib::LaunchScope scope("k_kv_move", cache->n_pages, s);
            launch_move(*cache, p, 1, s);
        }
        return report(p, live_pages, "mpt_kv_compact", s);
    });
}

extern "C" int mpt_kv_copy(const mpt_kv_cache *cache, int n, const int32_t *src, const int32_t *dst, int64_t *checked,
                           void *workspace, size_t workspace_bytes, void *stream) {
    mptlib::clear_error();
    return mptlib::guarded(__func__, [&]() -> int {
        if (n > 0 && (!src || !dst)) return fail(MPT_E_INVALID, "a list is NULL");
        if (int rc = check_plan(cache, n, cache ? cache->n_pages : 0, workspace, workspace_bytes)) return rc;
        hipStream_t s = (hipStream_t)stream;
        const Plan p = plan_at(*cache, workspace);
        {
            mptlib::LaunchScope scope("k_kv_plan_copy", n, s);
            k_kv_plan_copy<<<1, 1024, 0, s>>>(*cache, n, src, dst, p);
        }
        if (n) {
            mptlib::LaunchScope scope("k_kv_move", n, s);
            launch_move(*cache, p, 0, s);
        }
        return report(p, checked, "mpt_kv_copy", s);
    });
}

extern "C" int mpt_kv_append(const mpt_kv_cache *cache, int layer, int n, const int32_t *seqs, const int32_t *q_off,
                             int64_t n_tokens, const void *k_new, int64_t k_token_stride, int64_t k_head_stride,
                             const void *v_new, int64_t v_token_stride, int64_t v_head_stride, void *stream) {
    mptlib::clear_error();
    return mptlib::guarded(__func__, [&]() -> int {
        if (int rc = check_cache(cache)) return rc;
        if (int rc = check_append(cache, layer, n, n_tokens)) return rc;
        if (n == 0 || n_tokens == 0) return MPT_OK;
        if (!seqs || !q_off || !k_new || !v_new) return fail(MPT_E_INVALID, "an array is NULL");
        if (!aligned16(k_new) || !aligned16(v_new)) return fail(MPT_E_INVALID, "k_new and v_new must be 16-byte aligned");
        if ((k_token_stride | k_head_stride | v_token_stride | v_head_stride) % 8)
            return fail(MPT_E_INVALID, "strides must be multiples of 8");
        hipStream_t s = (hipStream_t)stream;
        if (is_mx4(*cache))
            return append_mx4(cache, layer, n, seqs, q_off, n_tokens, k_new, k_token_stride, k_head_stride, v_new,
                              v_token_stride, v_head_stride, s);
        {
            mptlib::LaunchScope scope("k_kv_append", (double)n_tokens, s);
            k_kv_append<<<mptlib::grid_for(n_tokens, 4, 4096), 256, 0, s>>>(
                *cache, layer, n, seqs, q_off, (int)n_tokens, (const char *)k_new, k_token_stride, k_head_stride,
                (const char *)v_new, v_token_stride, v_head_stride);
        }
        MPT_HIP_TRY(hipGetLastError());
        return MPT_OK;
    });
}

extern "C" int mpt_kv_merge(int n_parts, int64_t rows, int dim, const void *const *parts,
                            const float *const *part_lse, int part_dtype, void *out, int out_dtype, float *lse,
                            void *stream) {
    mptlib::clear_error();
    return mptlib::guarded(__func__, [&]() -> int {
        if (n_parts < 1 || n_parts > MPT_KV_MAX_PARTS) return fail(MPT_E_INVALID, "n_parts = %d", n_parts);
        if (dim < 8 || dim > MPT_KV_MAX_DIM || dim % 8) return fail(MPT_E_INVALID, "dim = %d", dim);
        if (rows < 0 || rows > (int64_t)INT32_MAX * 8) return fail(MPT_E_INVALID, "rows = %lld", (long long)rows);
        if (part_dtype < 0 || part_dtype > 2 || out_dtype < 0 || out_dtype > 2)
            return fail(MPT_E_INVALID, "part_dtype = %d, out_dtype = %d", part_dtype, out_dtype);
        if (rows == 0) return MPT_OK;
        if (!parts || !part_lse || !out) return fail(MPT_E_INVALID, "an array is NULL");
        Parts p = {};
        for (int i = 0; i < n_parts; ++i) {
            if (!parts[i] || !part_lse[i]) return fail(MPT_E_INVALID, "part %d is NULL", i);
            if (!aligned16(parts[i])) return fail(MPT_E_INVALID, "part %d is not 16-byte aligned", i);
            if (parts[i] == out && part_dtype != out_dtype)
                return fail(MPT_E_INVALID, "out is part %d but of another type", i);
            p.o[i] = parts[i];
            p.lse[i] = part_lse[i];
        }
        if (!aligned16(out)) return fail(MPT_E_INVALID, "out is not 16-byte aligned");
        using Kernel = void (*)(int, int64_t, int, Parts, void *, float *);
        static constexpr Kernel kernels[3][3] = {
            {k_kv_merge<0, 0>, k_kv_merge<0, 1>, k_kv_merge<0, 2>},
            {k_kv_merge<1, 0>, k_kv_merge<1, 1>, k_kv_merge<1, 2>},
            {k_kv_merge<2, 0>, k_kv_merge<2, 1>, k_kv_merge<2, 2>}};
        hipStream_t s = (hipStream_t)stream;
        const int per = 256 / (dim / 8);
        // a dimension of a launch holds less than 2^32 threads, and more are
        // not refused: they are cut off
        constexpr int64_t kAcross = 1 << 23;
        const int64_t blocks = (rows + per - 1) / per;
        const dim3 grid((unsigned)(blocks < kAcross ? blocks : kAcross), (unsigned)((blocks + kAcross - 1) / kAcross));
        {
            mptlib::LaunchScope scope("k_kv_merge", (double)rows, s);
            kernels[part_dtype][out_dtype]<<<grid, 256, 0, s>>>(n_parts, rows, dim, p, out, lse);
        }
        MPT_HIP_TRY(hipGetLastError());
        return MPT_OK;
    });
}
