/*
 * mpt.h -- C ABI of libmpt.so, an exact solver for the Minimum Prefix Trie
 * with Free Permutations (MPT) problem on AMD Instinct MI355X (gfx950).
 *
 * Problem (Section 2 of "Prefix Sharing Is a Sorting Problem"): a universe
 * of n_chunks chunks with weights w(x) > 0 and m requests R_i (sets of chunk
 * ids). Choose one permutation pi_i of every R_i so that the trie of the m
 * resulting sequences has the smallest total weight of non-root nodes
 * (Eq. 1). By the structure theorem (Theorem 1, Eqs. 2-3) the optimum is
 *     OPT_free = sum_i w(R_i) - max_H sum_{v internal in H} w(I(v)),
 * a maximum over binary hierarchies H on the requests, with
 * I(B) = intersection of R_i over i in B. The solver computes it with the
 * O(3^m) subset DP of Section 3.1, in cost form:
 *     C({i}) = w(R_i),
 *     C(S)   = min over A (+) B = S, A holding the lowest request of S,
 *              both non-empty, of C(A) + C(B)  -  W(S),     W(S) = w(I(S)),
 * and reads the orders off the optimal hierarchy top-down (proof of
 * Theorem 1, "<=" half).
 *
 * Conventions shared by every entry point
 *  - Subsets of requests are m-bit masks: bit i set = request i is in the set.
 *  - Every array argument is DEVICE memory (HBM) owned by the caller; the
 *    library allocates no device memory and keeps no pointer after a call
 *    returns. It allocates 512 KiB of pinned host memory once per process,
 *    in the first call that reads a result back (mpt_solve_exact_noalloc
 *    never does), for those results; threads share it safely.
 *  - `stream` is a hipStream_t (NULL = the null stream). All device work of a
 *    call is enqueued on it. Calls that return a host value synchronise it.
 *  - `workspace` is caller-owned device scratch of at least
 *    mpt_workspace_bytes(m, nnz) bytes, 256-byte aligned. Calls that share
 *    one workspace must not run concurrently.
 *  - Return value: MPT_OK (0) or a negative mpt_status. On error no output is
 *    guaranteed to be written; mpt_last_error() describes the failure for
 *    the calling thread. No C++ exception crosses this interface.
 *  - Integer ranges: 1 <= m <= MPT_MAX_M; 0 <= n_chunks <= MPT_MAX_CHUNKS;
 *    0 <= nnz <= 2^31 - 1 (request slots, the same for every call below);
 *    1 <= w(x) <= MPT_MAX_CHUNK_WEIGHT; sum_i w(R_i) < 2^61. These keep
 *    every W, C and pair sum inside int64.
 */
#ifndef MPT_H
#define MPT_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define MPT_MAX_M 30
#define MPT_MAX_CHUNKS (1LL << 30)
#define MPT_MAX_CHUNK_WEIGHT (1LL << 32)
/* C[0] after mpt_solve_exact: the empty set never takes part in a split. */
#define MPT_COST_SENTINEL (1LL << 62)

enum mpt_status {
    MPT_OK = 0,
    MPT_E_INVALID = -1,   /* bad size, null pointer, or req_off not a CSR offset array */
    MPT_E_RANGE = -2,     /* a chunk id outside [0, n_chunks) */
    MPT_E_DUP = -3,       /* a chunk repeated inside one request */
    MPT_E_WEIGHT = -4,    /* a weight <= 0 or > MPT_MAX_CHUNK_WEIGHT */
    MPT_E_OVERFLOW = -5,  /* sum_i w(R_i) >= 2^61 */
    MPT_E_WORKSPACE = -6, /* workspace missing, misaligned or too small */
    MPT_E_STATE = -7,     /* context call out of order (e.g. a solve before a build) */
    MPT_E_DEVICE = -8,    /* HIP runtime error (detail in mpt_last_error) */
    MPT_E_INTERNAL = -9,  /* internal error (e.g. a host allocation failed) */
    MPT_E_PAGES = -10     /* a page call asks for more pages than are free */
};

/* Bytes of device workspace that every entry point below needs for an
 * instance with m requests and nnz = req_off[m] request slots. */
size_t mpt_workspace_bytes(int m, int64_t nnz);

/*
 * Phase 1 -- intersection weights W(B) = w(I(B)) for all 2^m subsets B
 * (W(B) is the weight of the chunks shared by every request of B; Section 3,
 * proof of Theorem 1; I(empty) = U, so W(0) is the total weight of all
 * chunks). Also returns the demand sets S_x = { i : x in R_i } (Section 3).
 *
 *   chunk_w    [n_chunks]  int64 weights w(x)
 *   req_off    [m+1]       int64 CSR offsets, req_off[0] = 0, non-decreasing,
 *                          req_off[m] = nnz; request i is
 *                          req_chunks[req_off[i] .. req_off[i+1])
 *   req_chunks [nnz]       int32 chunk ids, distinct inside each request;
 *                          requests may be empty or equal to each other
 *   sig        [n_chunks]  out: uint32 S_x masks
 *   W          [2^m]       out: int64 table, 16-byte aligned
 * Validates the device inputs (MPT_E_INVALID / RANGE / DUP / WEIGHT /
 * OVERFLOW) and synchronises `stream` to report the result. With n_chunks = 0
 * the chunk ids are not looked at: W is 0 everywhere.
 */
int mpt_build_weights(int m, int64_t n_chunks, int64_t nnz,
                      const int64_t *chunk_w, const int64_t *req_off,
                      const int32_t *req_chunks, uint32_t *sig, int64_t *W,
                      void *workspace, size_t workspace_bytes, void *stream);

/*
 * Phase 2 -- the exact DP of Section 3.1 over all 2^m subsets, layer by
 * layer in |S|.
 *   W      [2^m]  int64 table from mpt_build_weights
 *   C      [2^m]  out: C(S) = OPT_free of the sub-instance {R_i : i in S};
 *                 C[0] = MPT_COST_SENTINEL
 *   split  [2^m]  out: for |S| >= 2 the optimal part A that holds the lowest
 *                 request of S; among optimal parts the numerically smallest;
 *                 0 for |S| <= 1. split encodes the optimal hierarchy: the
 *                 children of S are split[S] and S ^ split[S].
 *   opt_cost      HOST out, nullable: C(full set) = OPT_free (Theorem 1).
 *                 When non-null the call synchronises `stream`.
 * W, C and split need only the alignment of their element types.
 * For m >= 13 the call also synchronises `stream` once before its kernels,
 * to read sum_i W({i}) back: that total picks the key representation of the
 * packed kernels (32-bit keys for the cross and self pairs while it is below
 * 2^20 - 1, else exact doubles, uint64, or the plain kernels). Every
 * representation gives the same C and split.
 */
int mpt_solve_exact(int m, const int64_t *W, int64_t *C, uint32_t *split,
                    int64_t *opt_cost, void *workspace, size_t workspace_bytes,
                    void *stream);

/*
 * Phase 3 -- the layout read off the hierarchy (proof of Theorem 1): at node
 * B of the hierarchy each request below B emits I(B) \ I(parent(B)) in
 * ascending chunk id, with I(parent(root)) = empty. Chunk x of R_i is thus
 * emitted at the first node on request i's root-to-leaf path that is a
 * subset of S_x.
 *   req_off, req_chunks  the instance (as for mpt_build_weights)
 *   sig, split           outputs of the two calls above
 *   order_chunks [nnz]   out: pi_i at order_chunks[req_off[i] .. req_off[i+1])
 * Fails with MPT_E_INVALID (offsets, or a split table that does not encode
 * a hierarchy below the full set) or MPT_E_RANGE (a chunk id) before
 * anything is written; synchronises `stream` once to report those checks.
 */
int mpt_extract_orders(int m, int64_t n_chunks, int64_t nnz,
                       const int64_t *req_off, const int32_t *req_chunks,
                       const uint32_t *sig, const uint32_t *split,
                       int32_t *order_chunks, void *workspace,
                       size_t workspace_bytes, void *stream);

/*
 * mpt_solve_exact without a workspace, for callers that cannot allocate
 * device memory (code under HIP graph capture, serving loops, harnesses that
 * forbid hipMalloc). Same arguments, outputs and errors as mpt_solve_exact;
 * the scratch is a device array of MPT_NOALLOC_SCRATCH_BYTES inside the
 * library (one per device, kept until the process ends), enough for
 * m <= MPT_NOALLOC_MAX_M; larger m fails with MPT_E_INVALID. The call itself
 * allocates nothing. All calls on one device share that array: calls that
 * overlap on one device (other threads or streams) race and must be
 * serialised by the caller; consecutive calls on one stream are safe.
 */
#define MPT_NOALLOC_MAX_M 20
#define MPT_NOALLOC_SCRATCH_BYTES (37u << 20)
int mpt_solve_exact_noalloc(int m, const int64_t *W, int64_t *C, uint32_t *split, int64_t *opt_cost,
                            void *stream);

/*
 * ---- The context layer: the three phases of one instance on one device ----
 *
 * A context holds a device, a stream, a caller-owned workspace and the state
 * of one instance: created -> built (mpt_ctx_build_weights) -> solved
 * (mpt_ctx_solve_exact) -> extracted (mpt_ctx_extract_orders). Each phase
 * needs the one before it (else MPT_E_STATE); a new build starts over. A
 * failed build leaves the context created (no instance); a failed solve or
 * extraction leaves it where it was before that phase. Inputs are borrowed
 * for the duration of the build and copied into the workspace, which also
 * holds W, C, split, the demand sets and the orders; mpt_copy_table reads
 * them out. Compared with the stateless calls above, the solve needs no
 * read-back of sum_i w(R_i) (the build keeps it) and the extraction no
 * validation of a split table the library made, so the solve and the
 * extraction synchronise the stream only when they return host data.
 * A context serves one thread at a time; contexts are independent.
 */
typedef struct mpt_ctx mpt_ctx;

#define MPT_TABLE_W 0       /* int64 [2^m]      after a build */
#define MPT_TABLE_SIG 1     /* uint32 [n_chunks] after a build */
#define MPT_TABLE_C 2       /* int64 [2^m]      after a solve (C[0] = MPT_COST_SENTINEL) */
#define MPT_TABLE_SPLIT 3   /* uint32 [2^m]     after a solve */
#define MPT_TABLE_ORDERS 4  /* int32 [nnz]      after an extraction (CSR with req_off) */

/* Options (mpt_set_option). MPT_OPT_CHUNK_PAIRS: 0 (default) lets the
 * library plan how the cross pairs of each DP level are split over
 * workgroups; k >= 1 runs every level in chunks of at most k pairs (a level
 * whose pairs fit one chunk finishes its rows in the same kernel). Results
 * do not depend on it (it exists to test exactly that); it changes the
 * workspace size. */
#define MPT_OPT_CHUNK_PAIRS 1

/* MPT_OPT_WEIGHT_ROUTE: how a build computes W (Section 3.1's superset
 * sums). 0 (default) picks by size; MPT_ROUTE_LIST makes each 2^12-subset
 * tile scan the list of (S_x, w(x)) and write its part of W once (cost grows
 * with tiles x list length); MPT_ROUTE_DENSE scatters the list into W and
 * runs the superset zeta in place over the whole table (cost grows with
 * 2^m). The tables are the same on either route. */
#define MPT_OPT_WEIGHT_ROUTE 2
#define MPT_ROUTE_AUTO 0
#define MPT_ROUTE_LIST 1
#define MPT_ROUTE_DENSE 2

/* New context on HIP device hip_device, enqueueing on hip_stream (a
 * hipStream_t created on that device; NULL = its null stream). *out = NULL
 * on failure. Every context call makes hip_device current for its duration
 * and restores the caller's device. */
int mpt_create(mpt_ctx **out, int hip_device, void *hip_stream);

/* Frees the context (host memory only: the workspace is the caller's).
 * NULL-safe. Waits for nothing: the caller must not destroy a context whose
 * work is still in flight on its stream and then reuse the workspace. */
void mpt_destroy(mpt_ctx *ctx);

/* Sets an option (see MPT_OPT_*); MPT_E_INVALID for an unknown option or
 * value. Resets the context to created. */
int mpt_set_option(mpt_ctx *ctx, int option, int64_t value);

/* Device bytes the context needs for an instance of m requests, n_chunks
 * chunks and nnz request slots, with the context's options (ctx NULL:
 * default options). 0 for sizes out of range. */
size_t mpt_ctx_workspace_bytes(const mpt_ctx *ctx, int m, int64_t n_chunks, int64_t nnz);

/* Hands the context a caller-owned device workspace (256-byte aligned, on
 * the context's device, alive until the next mpt_set_workspace or
 * mpt_destroy). Its size is checked at each build. Resets the context to
 * created. dev_ptr NULL detaches it. */
int mpt_set_workspace(mpt_ctx *ctx, void *dev_ptr, size_t bytes);

/*
 * Phase 1 (as mpt_build_weights): copies the instance into the workspace,
 * validates it and builds W and the demand sets. chunk_w [n_chunks],
 * req_off [m+1] and req_chunks [nnz] may be host or device memory (copied
 * with hipMemcpyDefault). Synchronises the stream to report validation
 * errors. MPT_E_WORKSPACE if the workspace is missing or smaller than
 * mpt_ctx_workspace_bytes(ctx, m, n_chunks, nnz).
 */
int mpt_ctx_build_weights(mpt_ctx *ctx, int m, int64_t n_chunks, int64_t nnz, const int64_t *chunk_w,
                          const int64_t *req_off, const int32_t *req_chunks);

/*
 * Phase 2 (as mpt_solve_exact), after a build (else MPT_E_STATE).
 *   opt_cost    HOST out, nullable: OPT_free = C(full set) (Theorem 1)
 *   savings     HOST out, nullable: sum_i w(R_i) - OPT_free, the weight the
 *               optimal trie saves over no sharing (Eq. 3)
 *   split_host  HOST out, nullable: uint32 [2^m] split table
 * Synchronises the stream only if one of them is non-NULL.
 */
int mpt_ctx_solve_exact(mpt_ctx *ctx, int64_t *opt_cost, int64_t *savings, uint32_t *split_host);

/*
 * OPT_free and the savings of the last solve (HOST outs, nullable), after a
 * solve (else MPT_E_STATE): reads C(full set) back, synchronising the stream.
 * With this call a solve that returns no host data, the extraction and the
 * read-back run as one stream of work with a single synchronisation.
 */
int mpt_ctx_optimum(const mpt_ctx *ctx, int64_t *opt_cost, int64_t *savings);

/*
 * Phase 3 (as mpt_extract_orders), after a solve (else MPT_E_STATE).
 *   order_chunks_host  HOST out, nullable: int32 [nnz], pi_i at
 *                      [req_off[i], req_off[i+1])
 * Synchronises the stream only if order_chunks_host is non-NULL.
 */
int mpt_ctx_extract_orders(mpt_ctx *ctx, int32_t *order_chunks_host);

/*
 * Copies table `which` (MPT_TABLE_*) to host_dst, which holds `bytes` bytes
 * (at least the table's size, else MPT_E_INVALID); MPT_E_STATE if the phase
 * that writes the table has not run since the last build. Synchronises.
 */
int mpt_copy_table(const mpt_ctx *ctx, int which, void *host_dst, size_t bytes);

/* Device address and size of table `which` inside the workspace (valid
 * until the next build or workspace change), under the same state rules. */
int mpt_table_device(const mpt_ctx *ctx, int which, const void **dev_ptr, size_t *bytes);

/*
 * ---- Sections 6.2-6.3: heuristic and bound for large request counts ----
 *
 * These calls take any m in [1, MPT_GREEDY_MAX_M]; requests are identified
 * by index. Same conventions as above; they share one workspace of
 * mpt_greedy_workspace_bytes(m, n_chunks, nnz) bytes: 8 m^2 + max(8 min(m,
 * 2048)^2, 16 nnz) + 20 nnz + 8 n_chunks + 112 m, and less than 8 KiB of
 * padding. Instances are validated as for
 * mpt_build_weights.
 */
#define MPT_GREEDY_MAX_M 16384

/* Bytes of device workspace for the calls below (0 for sizes out of range). */
size_t mpt_greedy_workspace_bytes(int m, int64_t n_chunks, int64_t nnz);

/*
 * Pair weights P[i*m + j] = w(R_i ∩ R_j) for all requests i, j (so
 * P[i*m + i] = w(R_i)): the edge weights of the spanning-tree bound and the
 * values of the greedy's first merge (Sections 6.2-6.3).
 *   P [m*m]         out: int64, row-major, device
 *   request_total   HOST out, nullable: sum_i w(R_i)
 * Cost: one write of P plus sum_x |S_x|^2 additions, in on-chip memory,
 * one per pair of requests sharing a chunk -- meant for sparse demand
 * (small |S_x|).
 * Synchronises `stream` once to report validation errors (twice when a
 * request has more than 512 chunks).
 */
int mpt_pair_weights(int m, int64_t n_chunks, int64_t nnz, const int64_t *chunk_w,
                     const int64_t *req_off, const int32_t *req_chunks, int64_t *P,
                     int64_t *request_total, void *workspace, size_t workspace_bytes,
                     void *stream);

/*
 * Agglomerative common-prefix hierarchy H_g (Section 6.2; Theorem 6 shows
 * SAV(H_g) >= SAV* / 2). Every request starts as a cluster with signature
 * R_i; m-1 times, the two clusters whose signatures share the most weight
 * merge, and the merged signature is their intersection. A cluster is named
 * by its smallest request; among pairs of equal value the lexicographically
 * smallest pair of names (a, b), a < b, merges and keeps the name a.
 *   merge_a, merge_b [m-1]  out: int32 names of step t's pair, a < b
 *   gain [m-1]              out: int64 w(I(A) ∩ I(B)) of step t
 *                           (non-increasing, Theorem 6 part i)
 *   node_parent [2m-1]      out: int32 parent of each node (-1 at the root);
 *                           leaf i is node i, step t creates node m + t
 *   order_chunks [nnz]      out, nullable: the layout read off H_g (proof of
 *                           Theorem 1): top-down, node v emits
 *                           I(v) \ I(parent(v)) in ascending chunk id;
 *                           pi_i at order_chunks[req_off[i] ..)
 *   savings                 HOST out, nullable: SAV(H_g) = sum of the gains;
 *                           the layout costs at most sum_i w(R_i) - SAV(H_g)
 * The merges are found in parallel rounds (every mutually best pair of
 * clusters at once) and put in the sequence above afterwards; the outputs
 * are those of the one-merge-at-a-time procedure. Synchronises `stream`
 * once per eight rounds and before returning.
 */
int mpt_greedy_hierarchy(int m, int64_t n_chunks, int64_t nnz, const int64_t *chunk_w,
                         const int64_t *req_off, const int32_t *req_chunks,
                         int32_t *merge_a, int32_t *merge_b, int64_t *gain,
                         int32_t *node_parent, int32_t *order_chunks, int64_t *savings,
                         void *workspace, size_t workspace_bytes, void *stream);

/*
 * Spanning-tree lower bound (Section 6.3): every hierarchy's savings are at
 * most the weight of a maximum spanning tree of the complete graph on the
 * requests with edge weights P[i][j] (from mpt_pair_weights), so
 *     OPT_free >= sum_i P[i][i] - MST.
 *   P            [m*m] int64 pair weights, device
 *   mst_weight   HOST out: weight of a maximum spanning tree
 * Boruvka rounds over the whole device (ceil(log2 m) of them); uses
 * 256 + 32 m bytes of the workspace (rounded up per array); synchronises
 * `stream`.
 */
int mpt_spanning_tree_bound(int m, const int64_t *P, int64_t *mst_weight,
                            void *workspace, size_t workspace_bytes, void *stream);

/*
 * ---- Sections 7-8: layouts, serving schedules and the radix cache ----
 *
 * A layout is a CSR of chunk sequences: seq_off[m+1] (int64, device) and
 * seqs[nnz] (int32 chunk ids, device), e.g. the order_chunks output of
 * mpt_extract_orders or mpt_greedy_hierarchy with the request offsets.
 * Chunk ids must lie in [0, n_chunks); weights as above. The calls share one
 * workspace of mpt_layout_workspace_bytes(m, n_chunks, nnz, n_configs) bytes
 * (n_configs = 0 for the first two calls): 12 nnz + 8 n_chunks + 20 m, 8 per
 * leaf of a tree of at least m and 1024 leaves (a power of two), per
 * configuration 16 nnz + 12 m, and the largest of 16 max(nnz, n_chunks), 72 m
 * past 4096 requests and, per configuration, 16 max(m, nnz) and 8 nnz + 24 (nnz
 * rounded up to 1024); and less than 16 KiB of padding.
 */
#define MPT_LAYOUT_MAX_M (1 << 24)
#define MPT_CACHE_MAX_CONFIGS 256
#define MPT_ORDER_ID 0          /* chunk id ascending */
#define MPT_ORDER_POPULARITY 1  /* number of requests holding the chunk descending, id ascending */

size_t mpt_layout_workspace_bytes(int m, int64_t n_chunks, int64_t nnz, int n_configs);

/*
 * Global-order layout (Section 3.1's global orders; the id and popularity
 * baselines of Section 7): every request's chunks sorted by one order of the
 * chunks.
 *   req_off, req_chunks  the instance (as for mpt_build_weights)
 *   order_kind           MPT_ORDER_ID or MPT_ORDER_POPULARITY
 *   seqs [nnz]           out: the layout, CSR with req_off
 * Synchronises `stream` once to report validation errors.
 */
int mpt_global_order_layout(int m, int64_t n_chunks, int64_t nnz, const int64_t *req_off,
                            const int32_t *req_chunks, int order_kind, int32_t *seqs,
                            void *workspace, size_t workspace_bytes, void *stream);

/*
 * Trie cost of a layout (Eq. 1: the total weight of the non-root nodes of
 * the trie of the m sequences), and the DFS serving order of that trie
 * (Theorem 7): requests sorted lexicographically by their sequences, a
 * proper prefix first, equal sequences by request index.
 *   dfs_order [m]   out, nullable: request ids in DFS order
 *   trie_cost       HOST out
 * Synchronises `stream`.
 */
int mpt_layout_cost(int m, int64_t n_chunks, int64_t nnz, const int64_t *chunk_w,
                    const int64_t *seq_off, const int32_t *seqs, int32_t *dfs_order,
                    int64_t *trie_cost, void *workspace, size_t workspace_bytes, void *stream);

/*
 * Radix cache (Section 8): serving a request touches every node of its
 * root-to-leaf path in the layout's trie; the nodes not cached are computed
 * (their weight is billed) and inserted; then, while the cached weight
 * exceeds the capacity, the least-recently-used cached leaf is evicted
 * (cached nodes always include their ancestors). The cache starts empty.
 * Configuration c serves the requests in arrival order 0 .. m-1 cut into
 * windows of windows[c] requests, each window in DFS order (Section 8.1;
 * windows[c] <= 0 or >= m: the whole stream in DFS order, 1: arrival
 * order), with capacity capacities[c] (weight units; Theorem 7: in DFS
 * order max_i w(R_i) already bills exactly the trie cost).
 *   n_configs              1 .. MPT_CACHE_MAX_CONFIGS
 *   windows, capacities    HOST arrays [n_configs]
 *   costs                  HOST out [n_configs]: the billed weight
 *   trie_cost              HOST out, nullable: the unbounded-cache bill
 * Such a cache always holds the longest prefix of its recency stack that
 * fits (the stack property of LRU), so an access hits iff the distinct
 * weight accessed since its node's previous access, plus its own, fits.
 * Configurations with equal windows share one schedule and one pass that
 * prices all their capacities. Synchronises `stream`.
 */
int mpt_cache_simulate(int m, int64_t n_chunks, int64_t nnz, const int64_t *chunk_w,
                       const int64_t *seq_off, const int32_t *seqs, int n_configs,
                       const int64_t *windows, const int64_t *capacities, int64_t *costs,
                       int64_t *trie_cost, void *workspace, size_t workspace_bytes, void *stream);

/*
 * ---- Section 7.1: the quality-preserving pinned variant ----
 *
 * The first t chunks of every request in its input (relevance) order are
 * pinned at the end of its sequence, most relevant last; the rest (the free
 * part) is permuted. The construction: the distinct free sets are laid out
 * by the exact DP (mpt_build_weights, mpt_solve_exact, mpt_extract_orders)
 * or the greedy (mpt_greedy_hierarchy), every request takes its set's free
 * sequence, then its pinned suffix. Requests with equal free sets thereby
 * share one free sequence, and their suffixes can share trie nodes.
 */
/* 20 nnz + 36 m bytes (past 4096 requests at least 4 nnz + 108 m), and less
 * than 8 KiB of padding. */
size_t mpt_pinned_workspace_bytes(int m, int64_t nnz);

/*
 * Split into free sets and pinned suffixes.
 *   t                 pinned chunks per request (0: nothing pinned)
 *   dmap [m]          out: index of each request's free set among the
 *                     distinct sets, numbered in order of their first request
 *   free_off [m+1]    out: CSR offsets of the distinct free sets (the first
 *                     n_distinct + 1 entries are written)
 *   free_chunks [nnz] out: the distinct free sets, each in ascending chunk id
 *   n_distinct        HOST out: number of distinct free sets (>= 1)
 * Synchronises `stream`.
 */
int mpt_pinned_split(int m, int64_t n_chunks, int64_t nnz, const int64_t *req_off,
                     const int32_t *req_chunks, int t, int32_t *dmap, int64_t *free_off,
                     int32_t *free_chunks, int *n_distinct, void *workspace,
                     size_t workspace_bytes, void *stream);

/*
 * The layout: seqs[req_off[i] ..) = free sequence of set dmap[i] (from
 * free_layout, CSR with free_off, e.g. the orders of the exact or greedy
 * call on the distinct sets) followed by request i's pinned suffix.
 * Uses the first 256 bytes of the workspace; synchronises `stream`.
 */
int mpt_pinned_assemble(int m, int64_t nnz, const int64_t *req_off, const int32_t *req_chunks,
                        int t, const int32_t *dmap, int n_distinct, const int64_t *free_off,
                        const int32_t *free_layout, int32_t *seqs, void *workspace,
                        size_t workspace_bytes, void *stream);

/*
 * ---- Serving a layout: a paged key/value cache ----
 *
 * The prompts of a layout share prefixes (the nodes of its trie). These calls
 * hold the keys and values of those prefixes in pages that several sequences
 * refer to, so that a request forked off a cached prefix computes only the
 * tokens that the trie cost bills for it.
 *
 * Token t of the sequence in slot s lies in page table[s * max_pages + t /
 * page_size], at slot t % page_size of that page. ref[p] counts the
 * references to page p from the sequences' tables; bit p % 64 of
 * free_bits[p / 64] is set iff ref[p] = 0 (bits past n_pages are 0). A page
 * taken by a call is the lowest-numbered free one, so tables do not depend on
 * how the device schedules work. Table entries past a sequence's last page
 * mean nothing and are not touched.
 *
 * The caller owns every array and fills in the descriptor; mpt_kv_reset
 * empties the tables. A row (layer, page, slot, head) holds head_dim
 * consecutive elements. Strides are in elements and multiples of 8, bases
 * are 16-byte aligned, head_dim is a multiple of 8; the other orders of the
 * dimensions are free (heads inside or outside the slots, layers or keys and
 * values interleaved). Rows must not overlap.
 *
 * Errors in device data: a call that finds one ORs MPT_KV_* bits into *status,
 * where they stay until mpt_kv_status reads them. The page calls (forks to
 * copies below) then change nothing in tables and pages, appends write the
 * tokens that are in order. The page calls take a nullable HOST output; with
 * it they synchronise `stream` and return the error of this call
 * (MPT_E_RANGE, MPT_E_DUP, MPT_E_STATE or MPT_E_PAGES). Without it, and in
 * mpt_kv_append, mpt_kv_attention and mpt_kv_merge, nothing synchronises, and
 * the calls can be captured into a graph. Page ids outside [0, n_pages) and
 * slots outside [0, max_seqs) are never followed. The page calls look at every
 * page that they share, copy from, drop or (compaction) move, not at those
 * that stay as they are. Counts in ref that are lower than the tables' show
 * only when a page would lose a reference that it does not count: it then keeps
 * none, MPT_KV_BAD_PAGE is set and the call goes through.
 * Calls on one cache must be ordered by the caller (one stream, or events).
 */
#define MPT_KV_BF16 0
#define MPT_KV_F16 1
#define MPT_KV_F32 2              /* outputs and merged parts only */
#define MPT_KV_MAX_DIM 256
#define MPT_KV_MAX_PAGE_SIZE 1024
#define MPT_KV_MAX_PAGES (1 << 26)
#define MPT_KV_MAX_PARTS 16
#define MPT_KV_MAX_LIST ((1 << 24) - 1)   /* entries of a list of sequences in a page call */

#define MPT_KV_BAD_SLOT 1u        /* a slot outside [0, max_seqs), or offsets that are no CSR */
#define MPT_KV_BAD_LENGTH 2u      /* a length outside its range */
#define MPT_KV_BAD_PAGE 4u        /* a page id outside [0, n_pages) or without references */
#define MPT_KV_DUPLICATE 8u       /* a slot or page listed twice */
#define MPT_KV_NOT_EMPTY 16u      /* a fork into a slot that holds tokens */
#define MPT_KV_NO_PAGES 32u       /* more pages asked for than are free */
#define MPT_KV_SHARED 64u         /* an append into a page of several sequences */

typedef struct mpt_kv_cache {
    void *k, *v;                  /* device: keys and values */
    int64_t k_stride[4];          /* elements from one layer, page, slot, head to the next */
    int64_t v_stride[4];
    int32_t *table;               /* device [max_seqs * max_pages]: page ids */
    int32_t *length;              /* device [max_seqs]: tokens per sequence (0: an empty slot) */
    int32_t *ref;                 /* device [n_pages] */
    uint64_t *free_bits;          /* device [(n_pages + 63) / 64] */
    uint32_t *status;             /* device: MPT_KV_* bits */
    int dtype;                    /* MPT_KV_BF16 or MPT_KV_F16 */
    int n_layers, n_pages;
    int page_size;                /* a power of two, 1 .. MPT_KV_MAX_PAGE_SIZE */
    int n_heads, head_dim;        /* key/value heads; a multiple of 8, 8 .. MPT_KV_MAX_DIM */
    int max_seqs, max_pages;      /* max_pages * page_size <= 2^30 */
} mpt_kv_cache;

/* Empties the cache: every page free, every length 0, status 0. Does not
 * synchronise. */
int mpt_kv_reset(const mpt_kv_cache *cache, void *stream);

/* *bits (HOST) = the cache's status bits, which are then cleared.
 * Synchronises `stream`. */
int mpt_kv_status(const mpt_kv_cache *cache, uint32_t *bits, void *stream);

/* Bytes of device workspace (256-byte aligned) for the page calls: 8 n_pages
 * + 12 max_seqs and less than 4 KiB (0 for a descriptor that is not valid). */
size_t mpt_kv_workspace_bytes(const mpt_kv_cache *cache);

/*
 * Forks: for each i < n the empty slot dst[i] becomes a sequence of
 * new_len[i] tokens whose first keep[i] are those of src[i]. The
 * keep / page_size full pages are shared; then come fresh pages, taken in the
 * order of the list, and the keep % page_size tokens of a last partial page
 * are copied into the first of them (all layers). src[i] = -1 with keep[i] = 0
 * shares nothing. Sources are read as they were before the call.
 *   src, dst, keep, new_len [n]  device; dst distinct and empty; 0 <= keep[i]
 *                                <= length[src[i]], keep[i] <= new_len[i]
 *   free_pages                   HOST out, nullable: free pages afterwards
 * n <= MPT_KV_MAX_LIST, here and in the two calls below. All or nothing.
 */
int mpt_kv_fork(const mpt_kv_cache *cache, int n, const int32_t *src, const int32_t *dst,
                const int32_t *keep, const int32_t *new_len, int64_t *free_pages,
                void *workspace, size_t workspace_bytes, void *stream);

/*
 * Grows sequences to new_len[i] >= length[seqs[i]] tokens with fresh pages,
 * as mpt_kv_fork takes them. A partial last page that other sequences refer
 * to (left by mpt_kv_free with a keep) is first replaced by a copy.
 *   seqs, new_len [n]  device; seqs distinct
 */
int mpt_kv_extend(const mpt_kv_cache *cache, int n, const int32_t *seqs, const int32_t *new_len,
                  int64_t *free_pages, void *workspace, size_t workspace_bytes, void *stream);

/*
 * Cuts sequences to keep[i] <= length[seqs[i]] tokens (keep NULL: to none).
 * Pages past the last kept token lose a reference and are free without any.
 *   seqs, keep [n]  device; seqs distinct; empty ones are allowed
 */
int mpt_kv_free(const mpt_kv_cache *cache, int n, const int32_t *seqs, const int32_t *keep,
                int64_t *free_pages, void *workspace, size_t workspace_bytes, void *stream);

/*
 * Moves pages so that the n_live pages in use are 0 .. n_live - 1: the used
 * pages from n_live on, in ascending order, go to the free ones below, in
 * ascending order. Tables, references and contents (all layers) move along.
 *   live_pages  HOST out, nullable: n_live
 */
int mpt_kv_compact(const mpt_kv_cache *cache, int64_t *live_pages,
                   void *workspace, size_t workspace_bytes, void *stream);

/*
 * Copies the contents of page src[i] to page dst[i] (all layers), i < n.
 * No page may be in both lists or twice in dst. Tables stay as they are.
 *   checked  HOST out, nullable: pages copied (n, or 0 after an error)
 */
int mpt_kv_copy(const mpt_kv_cache *cache, int n, const int32_t *src, const int32_t *dst,
                int64_t *checked, void *workspace, size_t workspace_bytes, void *stream);

/*
 * Writes new keys and values of one layer: entry i < n has the tokens
 * q_off[i] .. q_off[i+1] - 1 of k_new and v_new, the newest of the sequence in
 * slot seqs[i] (which mpt_kv_fork or mpt_kv_extend has made long enough):
 * they go to positions length - (q_off[i+1] - q_off[i]) .. length - 1.
 *   seqs [n]             device; distinct
 *   q_off [n+1]          device; q_off[0] = 0, non-decreasing, q_off[n] = n_tokens
 *   k_new, v_new         device, the cache's type, [n_tokens, n_heads,
 *                        head_dim]; strides in elements, multiples of 8;
 *                        16-byte aligned
 * Tokens before position 0, in bad slots or pages, or in pages that other
 * sequences refer to are not written (and set status bits).
 */
int mpt_kv_append(const mpt_kv_cache *cache, int layer, int n, const int32_t *seqs,
                  const int32_t *q_off, int64_t n_tokens, const void *k_new,
                  int64_t k_token_stride, int64_t k_head_stride, const void *v_new,
                  int64_t v_token_stride, int64_t v_head_stride, void *stream);

/* Bytes of device workspace (256-byte aligned) for mpt_kv_attention of n
 * entries and n_tokens tokens with n_q_heads query heads: at most 68 MiB, the
 * partial sums of two tiles per workgroup (0 for sizes out of range: n <=
 * MPT_KV_MAX_ENTRIES, n_tokens <= 2^30, and as many rows n_tokens * n_q_heads /
 * n_heads). */
#define MPT_KV_MAX_ENTRIES 65536
size_t mpt_kv_attention_workspace_bytes(const mpt_kv_cache *cache, int n, int64_t n_tokens,
                                        int n_q_heads);

/*
 * Attention of new tokens over the cache, one layer. Entry i < n has the
 * queries q_off[i] .. q_off[i+1] - 1, the newest n_i tokens of the sequence
 * in slot seqs[i] of length L: query j stands at position p = L - n_i + j.
 * Query head h reads key head h / (n_q_heads / n_heads). Token t is visible
 * iff kv_begin[i] <= t < L, t <= p if causal, and t > p - window if
 * window > 0. With s_t = scale q.k_t, or softcap tanh(scale q.k_t / softcap)
 * if softcap > 0, over the visible t:
 *     lse = log sum exp(s_t),   out = sum exp(s_t - lse) v_t.
 * Rows that see no token (or only scores of minus infinity) get out = 0 and
 * lse = minus infinity. What lies in tokens that a row does not see, NaN and
 * infinities included, has no effect on it. An infinite value that a row does
 * see makes its output infinite however small its weight (NaN beside a NaN or the
 * other infinity). The sums are formed with weights of up to 2^8, in 32 bits:
 * they overflow where weights times values pass 2^128. Bad slots count as empty,
 * tokens on bad pages as zeros or as some tokens of the pool, and tokens of no
 * entry get no output. Decoding is a chunk of one token;
 * a prefix that several sequences share is one slot with all of their queries
 * and causal = 0, joined with their own parts (kv_begin) by mpt_kv_merge.
 *   seqs [n]       device; a slot may be listed several times
 *   q_off [n+1]    device; q_off[0] = 0, non-decreasing, q_off[n] = n_tokens
 *   q, out         device [n_tokens, n_q_heads, head_dim]; strides in
 *                  elements, multiples of 8; 16-byte aligned. q has the
 *                  cache's type, out that type or MPT_KV_F32 (out_dtype)
 *   lse            device out, nullable: float [n_tokens * n_q_heads],
 *                  natural logarithms
 *   kv_begin [n]   device, nullable (0): first visible token
 * Scores, statistics and sums are held in 32 bits; the weights exp(s_t - max)
 * are rounded to the cache's type for the product with the values.
 */
int mpt_kv_attention(const mpt_kv_cache *cache, int layer, int n, const int32_t *seqs,
                     const int32_t *q_off, int64_t n_tokens, int n_q_heads, const void *q,
                     int64_t q_token_stride, int64_t q_head_stride, void *out,
                     int64_t out_token_stride, int64_t out_head_stride, int out_dtype, float *lse,
                     const int32_t *kv_begin, int causal, int window, float softcap, float scale,
                     void *workspace, size_t workspace_bytes, void *stream);

/*
 * Joins attention over disjoint parts of a context: for each row r < rows
 *     lse = log sum_p exp(lse_p),   out = sum_p exp(lse_p - lse) out_p,
 * which is attention over all parts together. An infinity in a part stays one
 * however small the part's weight. Parts whose lse is minus infinity are not
 * read; without any other, out = 0 and lse = minus infinity.
 *   n_parts         1 .. MPT_KV_MAX_PARTS
 *   parts, part_lse HOST arrays [n_parts] of device pointers: [rows, dim]
 *                   (contiguous, 16-byte aligned, MPT_KV_* part_dtype) and
 *                   float [rows]
 *   dim             a multiple of 8, 8 .. MPT_KV_MAX_DIM
 *   out [rows, dim] device, contiguous, 16-byte aligned, out_dtype; may be
 *                   one of the parts if the types are equal
 *   lse [rows]      device out, nullable; may be one of part_lse
 */
int mpt_kv_merge(int n_parts, int64_t rows, int dim, const void *const *parts,
                 const float *const *part_lse, int part_dtype, void *out, int out_dtype, float *lse,
                 void *stream);

/* Static text for a status code. */
const char *mpt_status_string(int status);

/* Detail of the calling thread's last failed call ("" if none). */
const char *mpt_last_error(void);

/*
 * Diagnostics: per-kernel device time with HIP events recorded on the
 * caller's stream around every launch. mpt_profile_begin() clears and
 * enables recording (process-wide); mpt_profile_begin_prefix(p) does the
 * same for the launches whose label starts with p only (the events add a few
 * microseconds between launches, so a timing run records only the kernels it
 * needs); mpt_profile_end() waits for the events,
 * fills up to max_entries rows, disables recording and returns the number of
 * distinct kernels seen (or a negative status).
 *   work: the algorithmic units the launches processed -- evaluated
 *         bipartitions for the DP kernels, bytes written for the W kernel.
 */
typedef struct mpt_profile_row {
    char kernel[48];
    int64_t launches;
    double total_ms;
    double work;
} mpt_profile_row;

int mpt_profile_begin(void);
int mpt_profile_begin_prefix(const char *prefix);
int mpt_profile_end(mpt_profile_row *rows, int max_entries);

#ifdef __cplusplus
}
#endif

#endif /* MPT_H */
