/*
 * peek.h - batched longest-prefix match of a waiting queue against a KV
 * prefix-cache radix tree, plus the queue-side signals derived from it,
 * on one AMD Instinct MI355X (gfx950).
 *
 * The problem (PEEK, Sec. 3.1 and Alg. 1): for every waiting request r,
 * find the LPM hit length H[r] of its prompt against the engine's radix
 * cache, where a partially matched edge still counts (Alg. 1: h = d + delta
 * with delta the matched tokens of an edge). Engines cache whole blocks of B
 * tokens, so the reported hit is h = B * floor(m / B) with m the raw match.
 * The same queue yields its prefix-sharing clusters (Sec. 3.1: the deepest
 * pending-tree node with pending_count >= 2 on a request's path, its count
 * being the cluster size) and the per-cache-node pending demand read by the
 * eviction score (Eq. 2).
 *
 * What the hit is for follows at the end of this header: the K and V of
 * cached tokens in 8-bit pages, attention that reads them, and the eviction
 * of a sequence's blocks by the attention weight they get.
 *
 * Conventions for every call:
 *  - Plain C ABI; no exceptions cross it; nothing aborts the process.
 *  - Errors return a negative peek_status; peek_last_error() then describes
 *    the failure for the calling thread. Outputs are not written on error.
 *  - "d_" pointers are device memory on the current HIP device, owned by the
 *    caller, and must stay valid until `stream` has executed the call. Host
 *    pointers are read before the call returns and may be freed afterwards.
 *  - `stream` is a hipStream_t (NULL = the default stream). GPU work is
 *    enqueued on it; calls do not synchronize it unless stated.
 *  - Token ids are opaque int32 values compared for equality; child order
 *    uses signed comparison.
 *  - A prompt set is packed: request r's prompt is
 *    d_tokens[d_offsets[r] : d_offsets[r+1]], offsets int64, non-decreasing.
 *    Offsets and tokens live on the device, so they are preconditions the
 *    library does not re-check. Each prompt must be shorter than 2^31 tokens.
 *  - Debugging aid: with the environment variable PEEK_VALIDATE set (to
 *    anything but 0), peek_lpm_batch, peek_queue_signals, peek_clpm_signals,
 *    peek_offline_order and peek_block_lpm_batch first check their device
 *    inputs on the device (offsets non-decreasing from >= 0, prompt lengths
 *    < 2^31, last nodes inside the cache, match lengths inside their
 *    prompts) and return INVALID_ARGUMENT before any other work if one
 *    fails; so do peek_kv_append, peek_prefill_attention,
 *    peek_decode_attention and peek_kv_evict (offsets, lengths, page ids,
 *    scales).
 *    The check adds a small allocation, a launch and a stream
 *    synchronization per call, so it is not for use under graph capture.
 */
#ifndef PEEK_H
#define PEEK_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define PEEK_ABI_VERSION 1

typedef enum peek_status {
  PEEK_OK = 0,
  PEEK_ERR_INVALID_ARGUMENT = -1,    /* null pointer, negative size, bad parameter */
  PEEK_ERR_INVALID_TREE = -2,        /* tree description is not a radix tree */
  PEEK_ERR_OUT_OF_MEMORY = -3,       /* host or device allocation failed */
  PEEK_ERR_DEVICE = -4,              /* a HIP call failed; message names it */
  PEEK_ERR_WORKSPACE_TOO_SMALL = -5, /* see peek_queue_signals_workspace */
  PEEK_ERR_UNSUPPORTED_DEVICE = -6   /* current device is not gfx950 */
} peek_status;

/* Opaque handle: a cache tree flattened into device memory. Immutable after
 * build, so concurrent calls on different streams may share it. */
typedef struct peek_cache peek_cache;

int32_t peek_abi_version(void);

/* Description of the most recent failure on the calling thread (never NULL;
 * empty after success). Valid until the thread's next peek_ call. */
const char* peek_last_error(void);

/* ------------------------------------------------------------------------
 * Cache tree description (host).
 *
 * A tree of num_nodes nodes: node i has parent parent[i] (-1 for exactly one
 * root) and the edge label edge_tokens[edge_offsets[i] : edge_offsets[i+1]].
 * The root's edge is empty; every other edge is non-empty; siblings have
 * distinct first tokens (SGLang's RadixCache keys children by the first edge
 * token, App. A implementation details); every node is reachable from the
 * root. Unary nodes are allowed and kept.
 *
 * Canonical node ids: depth-first preorder from the root (id 0), children
 * visited by ascending first token. Every device output that names a node
 * (last_node, demand) uses canonical ids, so results do not depend on how
 * the caller numbered its nodes.
 * ---------------------------------------------------------------------- */

/* Validates a description and writes canon_id[i] = canonical id of input
 * node i (host only; no GPU needed). PEEK_ERR_INVALID_TREE if invalid. */
peek_status peek_tree_canonical_ids(int32_t num_nodes, const int32_t* parent,
                                    const int64_t* edge_offsets, const int32_t* edge_tokens,
                                    int32_t* canon_id);

/* Builds the compressed radix tree of raw cached sequences (host only).
 * Sequence s is tokens[offsets[s] : offsets[s+1]]. Nodes are the root,
 * every branch point and every sequence end; the output description is in
 * canonical order (node i has canonical id i). The three output arrays are
 * allocated by the library; release each with peek_free_host. */
peek_status peek_tree_from_sequences(const int32_t* tokens, const int64_t* offsets, int64_t num_seqs,
                                     int32_t* num_nodes_out, int32_t** parent_out,
                                     int64_t** edge_offsets_out, int32_t** edge_tokens_out);
void peek_free_host(void* p);

/* ------------------------------------------------------------------------
 * peek_cache_build: validate a host description, renumber it canonically,
 * and upload it as CSR arrays to the current device (the engine's prefix
 * cache, Sec. 2, flattened for the device). Host arrays are copied; the call
 * waits for the upload to finish before returning. On success *out owns all
 * device memory of the cache. canon_id (host, nullable) receives
 * canon_id[i] = canonical id of input node i, so demand[] can be mapped back
 * to the caller's nodes. Errors: INVALID_ARGUMENT, INVALID_TREE,
 * OUT_OF_MEMORY, DEVICE, UNSUPPORTED_DEVICE; *out is left untouched.
 * ---------------------------------------------------------------------- */
peek_status peek_cache_build(int32_t num_nodes, const int32_t* parent, const int64_t* edge_offsets,
                             const int32_t* edge_tokens, void* stream, peek_cache** out,
                             int32_t* canon_id);

/* Any output pointer may be NULL. max_depth is the longest root-to-node
 * path in tokens; device_bytes the device memory the handle owns. */
peek_status peek_cache_stats(const peek_cache* cache, int64_t* num_nodes, int64_t* num_edge_tokens,
                             int32_t* max_fanout, int64_t* max_depth, int64_t* device_bytes);

/* Host copies of the canonical node table (each output nullable, length
 * num_nodes): parent id, depth at the end of the edge, edge length,
 * preorder end of the subtree (subtree(c) = [c, subtree_end[c])). */
peek_status peek_cache_export(const peek_cache* cache, int32_t* parent, int32_t* depth,
                              int32_t* edge_len, int32_t* subtree_end);

/* Frees the handle and its device memory (NULL is a no-op). The caller must
 * ensure no enqueued work still uses it. */
peek_status peek_cache_free(peek_cache* cache);

/* ------------------------------------------------------------------------
 * peek_lpm_batch: LPM hit of every waiting request (Alg. 1 ENSURE clause:
 * H[r] for every waiting request r; MatchInRadix counts partial edges).
 *
 * For request r with prompt p:
 *   match_len[r] = m = max over cached paths P(c) of LCP(p, P(c))
 *   h[r]         = block_size * floor(m / block_size)
 *   last_node[r] = canonical id of the deepest node c the walk enters, i.e.
 *                  with LCP(p, P(c)) > depth(parent(c)); 0 if none.
 * d_h is required; d_last_node and d_match_len may be NULL. All outputs are
 * int32[n]. n = 0 is a no-op. Asynchronous on `stream`; no workspace.
 * Errors: INVALID_ARGUMENT (n < 0, block_size < 1, null cache/pointers,
 * cache built on another device), DEVICE.
 * ---------------------------------------------------------------------- */
peek_status peek_lpm_batch(const peek_cache* cache, int32_t n, const int32_t* d_tokens,
                           const int64_t* d_offsets, int32_t block_size, int32_t* d_h,
                           int32_t* d_last_node, int32_t* d_match_len, void* stream);

/* ------------------------------------------------------------------------
 * peek_queue_signals: prefix-sharing clusters of the waiting queue and the
 * pending demand of every cache node (Sec. 3.1, App. A.3, Eq. 2).
 *
 * Demand (when d_demand != NULL; needs the cache and d_last_node):
 *   d_demand[c] = number of requests whose walk enters cache node c
 *               = #{r : last_node[r] in subtree(c)}; int32[num_nodes],
 *                 canonical ids; d_demand[0] = n.
 * Clusters (when d_cluster_id and d_cluster_size != NULL; need d_tokens and
 * d_offsets):
 *   share_r = max over r' != r of LCP(p_r, p_r')   (0 when n = 1)
 *   if share_r >= threshold:
 *     cluster_size[r] = #{r' : LCP(p_r, p_r') >= share_r}   (pending_count)
 *     cluster_id[r]   = min{r' : share_r' = share_r and LCP(p_r, p_r') >= share_r}
 *   else cluster_id[r] = -1, cluster_size[r] = 1 (in no cluster).
 * Request indices are positions in the submitted batch (arrival order).
 *
 * d_last_node and d_match_len, when given, must be the outputs of
 * peek_lpm_batch for the same prompts and cache. The cluster pass then
 * starts from the prefixes the walk already proved shared and does not read
 * them again; with either pointer NULL (or no cache) it starts from scratch.
 * The results are the same either way.
 *
 * Scratch comes from d_workspace (device, 256-byte aligned, at least
 * peek_queue_signals_workspace(n, num_nodes) bytes, num_nodes = 0 without a
 * cache); the library allocates nothing here. Asynchronous on `stream`: the
 * call only enqueues kernels and returns without waiting for the device
 * (however many refinement rounds the queue needs, they run on the device),
 * so the workspace and every output must stay untouched until `stream` has
 * run the work. Calls on different streams need distinct workspaces.
 * threshold >= 1. Errors: INVALID_ARGUMENT, WORKSPACE_TOO_SMALL, DEVICE.
 * Up to 512 requests, workgroups wait for others of the same kernel. Such a
 * wait always ends; were it to last seconds all the same, the kernel gives it
 * up and fills cluster_id and cluster_size (and peek_clpm_signals' outputs)
 * with -1, which no finished call leaves in cluster_size.
 * ---------------------------------------------------------------------- */
size_t peek_queue_signals_workspace(int32_t n, int64_t num_nodes);

peek_status peek_queue_signals(const peek_cache* cache, int32_t n, const int32_t* d_tokens,
                               const int64_t* d_offsets, const int32_t* d_last_node,
                               const int32_t* d_match_len, int32_t threshold,
                               int32_t* d_cluster_id, int32_t* d_cluster_size, int32_t* d_demand,
                               void* d_workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------
 * peek_queue_signals_noalloc: peek_queue_signals without a workspace, for
 * callers that cannot allocate device memory (code under HIP graph capture,
 * tight serving loops, harnesses that forbid hipMalloc). Same arguments,
 * outputs and errors as peek_queue_signals minus the workspace pair. The
 * call allocates nothing (no hipMalloc, hipFree or allocating library
 * routine) and is asynchronous on `stream`.
 * Its scratch is a static device array of PEEK_NOALLOC_SCRATCH_BYTES per
 * GPU, reserved when the library is loaded onto that GPU and held until the
 * process ends. A call that needs more (peek_queue_signals_workspace(n,
 * num_nodes) > PEEK_NOALLOC_SCRATCH_BYTES, e.g. 64K requests against a cache
 * of more than about 3.6M nodes) fails with WORKSPACE_TOO_SMALL before any
 * launch.
 * Every call on one GPU shares that GPU's array: calls whose work may
 * overlap on the device (different streams, host threads racing) race on it
 * and must not be issued; calls ordered on one stream are safe. The array
 * keeps the last call's contents; each call clears what it needs.
 * PEEK_VALIDATE has no effect here (its checks allocate).
 * ---------------------------------------------------------------------- */
#define PEEK_NOALLOC_SCRATCH_BYTES (32u << 20)

peek_status peek_queue_signals_noalloc(const peek_cache* cache, int32_t n, const int32_t* d_tokens,
                                       const int64_t* d_offsets, const int32_t* d_last_node,
                                       const int32_t* d_match_len, int32_t threshold, int32_t* d_cluster_id,
                                       int32_t* d_cluster_size, int32_t* d_demand, void* stream);

/* ------------------------------------------------------------------------
 * peek_clpm_signals: everything peek_queue_signals computes plus the rest
 * of cLPM's per-request signal vector (Sec. 3.2 signals (2)-(3); Alg. 2,
 * which reads them as section, score and cluster info):
 *   d_score[r]   = sum over the nodes v on r's path in the pending tree of
 *                  pending_count(v) * |edge(v)|  (int64; equals the sum over
 *                  every request q, q = r included, of LCP(p_r, p_q))
 *   d_section[r] = 0 (warm) if d_h[r] > tau; otherwise, scanning requests in
 *                  arrival order, 1 (cold pioneer) for the first cold request
 *                  whose prompt[:theta] (whole prompt when shorter) is new
 *                  among cold requests, 2 (cold sibling) for later ones (int32)
 *   *d_has_sharing = 1 if two requests share their first token, else 0
 *                  (the pending tree's check over its root's children)
 * d_h is the LPM hit per request (peek_lpm_batch's d_h, or any int32 hit
 * vector); it is needed when d_section is given. d_score, d_section and
 * d_has_sharing are each optional (NULL: not written); d_cluster_id and
 * d_cluster_size are required. theta >= 0 (the paper uses 32); tau is any
 * int32 (the paper leaves it unset). Same workspace, asynchrony and errors
 * as peek_queue_signals.
 * ---------------------------------------------------------------------- */
peek_status peek_clpm_signals(const peek_cache* cache, int32_t n, const int32_t* d_tokens,
                              const int64_t* d_offsets, const int32_t* d_h, const int32_t* d_last_node,
                              const int32_t* d_match_len, int32_t threshold, int32_t tau, int32_t theta,
                              int32_t* d_cluster_id, int32_t* d_cluster_size, int32_t* d_demand,
                              int64_t* d_score, int32_t* d_section, int32_t* d_has_sharing,
                              void* d_workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------
 * peek_evict_rank: eviction ranking of the cached nodes (Eq. 2).
 *   d_score[c] = max over c and its ancestors a of demand[a] * depth(a)
 *                (int64[num_nodes], canonical ids; depth = tokens from the
 *                root to the end of a's edge; a cache node's pending count is
 *                its demand). The lowest score evicts first.
 *   d_order    = the num_nodes - 1 non-root nodes in the order a leaf-only
 *                eviction loop frees them: always the available leaf with the
 *                smallest (score, id), a node becoming available once its
 *                last child is freed (int32[num_nodes - 1]).
 * d_demand is peek_queue_signals' demand (int32[num_nodes], device). Either
 * output may be NULL, not both. Scratch comes only from d_workspace (device,
 * 256-byte aligned, at least peek_evict_rank_workspace(num_nodes) bytes).
 * Asynchronous on `stream`. As with the signals of few requests, a wait
 * between workgroups that lasts seconds is given up: d_order is then -1
 * throughout (d_score needs no wait).
 * Errors: INVALID_ARGUMENT, WORKSPACE_TOO_SMALL, DEVICE.
 * ---------------------------------------------------------------------- */
size_t peek_evict_rank_workspace(int64_t num_nodes);

peek_status peek_evict_rank(const peek_cache* cache, const int32_t* d_demand, int64_t* d_score,
                            int32_t* d_order, void* d_workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------
 * Hashed-block prefix cache: the engine variant whose cache is a flat table
 * of block hashes rather than a radix tree (Sec. 3.1 on vLLM, where one
 * longest-cache-hit probe per request gives H[r]).
 *
 * Every full block of block_size tokens on a cached root-to-node path is
 * stored as the chained hash of the path up to and including that block:
 *   mix64(z)   = SplitMix64 output mix (z ^= z>>30; z *= 0xbf58476d1ce4e5b9;
 *                z ^= z>>27; z *= 0x94d049bb133111eb; z ^= z>>31)
 *   key(j)     = mix64(j + 0x6A09E667F3BCC909); a_j = low, b_j = high 32 bits
 *   n_a        = sum over token pairs (2i, 2i+1) of the block of
 *                ((u_2i + a_2i) mod 2^32) * ((u_2i+1 + a_2i+1) mod 2^32) mod 2^64
 *                (an NH pass, as in UMAC; u = tokens as uint32); n_b with b
 *   digest_i   = mix64(n_a ^ rotl64(n_b, 32) ^ 0x9E3779B97F4A7C15 * (i + 1)),
 *                i = the block's index along the path (0-based)
 *   k_0 = 0x243F6A8885A308D3,   k_{i+1} = k_i + digest_i   (mod 2^64)
 * This hash is the library's own definition; equal hashes are taken as equal
 * blocks, so with no collision the hit equals B * floor(m / B) of
 * peek_lpm_batch on the same tree.
 * ---------------------------------------------------------------------- */
typedef struct peek_block_table peek_block_table;

/* Builds the table of every path's chained full-block hashes from a tree
 * description (same rules and errors as peek_cache_build; node numbering is
 * irrelevant here) and uploads it to the current device. block_size is a
 * power of two in [4, 256]. Open addressing with linear probing, at most
 * half full. Host arrays are read before return; the call waits for the
 * upload. *out owns the device memory; release with peek_block_table_free.
 * Errors: INVALID_ARGUMENT, INVALID_TREE, OUT_OF_MEMORY, DEVICE,
 * UNSUPPORTED_DEVICE; *out is set to NULL. */
peek_status peek_block_table_build(int32_t num_nodes, const int32_t* parent, const int64_t* edge_offsets,
                                   const int32_t* edge_tokens, int32_t block_size, void* stream,
                                   peek_block_table** out);

/* Any output pointer may be NULL: distinct stored hashes, slots, block size. */
peek_status peek_block_table_stats(const peek_block_table* table, int64_t* num_blocks, int64_t* num_slots,
                                   int32_t* block_size);

/* Frees the table (NULL is a no-op); no enqueued work may still use it. */
peek_status peek_block_table_free(peek_block_table* table);

/* Hit of every request against the table: d_h[r] = block_size * (number of
 * leading full blocks of prompt r whose chained hash is stored), int32[n].
 * One probe walk per request stops at the first missing block. n = 0 is a
 * no-op. Asynchronous on `stream`; no workspace.
 * Errors: INVALID_ARGUMENT (n < 0, null pointers, table built on another
 * device), DEVICE. */
peek_status peek_block_lpm_batch(const peek_block_table* table, int32_t n, const int32_t* d_tokens,
                                 const int64_t* d_offsets, int32_t* d_h, void* stream);

/* ------------------------------------------------------------------------
 * peek_offline_order: PEEK-offline Phase 1 (appendix on PEEK-offline,
 * Phase 1).
 *
 * Over the token trie of the prompts' first depth_limit tokens (the paper
 * uses D = 128), a depth-first traversal emits at every node the requests
 * whose truncated prompt ends there, in arrival order, then visits the
 * node's children by descending subtree request count; children with equal
 * counts go by their earliest request (the paper leaves this tie open).
 *   d_perm[k] = the request emitted k-th (int32[n], device).
 * Requests that share a truncated prefix are therefore contiguous in d_perm.
 * No cache is involved (the paper's regime is a cold cache). depth_limit >= 0
 * (0: arrival order); n < 2^30. Scratch comes only from d_workspace (device, 256-byte
 * aligned, at least peek_offline_order_workspace(n) bytes). Asynchronous on
 * `stream`, as peek_queue_signals.
 * Errors: INVALID_ARGUMENT, WORKSPACE_TOO_SMALL, DEVICE.
 * ---------------------------------------------------------------------- */
size_t peek_offline_order_workspace(int32_t n);

peek_status peek_offline_order(int32_t n, const int32_t* d_tokens, const int64_t* d_offsets, int32_t depth_limit,
                               int32_t* d_perm, void* d_workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------
 * The cache's contents: keys and values of 8 bits in pages, the attention
 * that reads them, and what attention says may go.
 *
 * peek_lpm_batch says how many leading tokens of a prompt are cached (h).
 * These calls are what the hit is for: the K and V of those tokens in pages
 * of block_size tokens, attention of the prompt's other tokens over them,
 * attention of the tokens generated after it, and the eviction of a
 * sequence's blocks that attention hardly reads.
 *
 * Pool: pages[num_pages][2][kv_heads][block_size][head_dim] of 8-bit codes
 * (K at 0, V at 1), scales[num_pages][2][kv_heads] float32. A value is its
 * code times its scale. Scales of keys are finite, those of values 0 (which
 * counts as 2^-60) or 2^-60 to 2^60; peek_kv_append leaves 2^-60 to 2^60 and
 * asks for 0 to 2^60 of a block that it adds to (PEEK_VALIDATE reports others). Formats: PEEK_TYPE_F8E4M3 (OCP e4m3) and
 * PEEK_TYPE_I8. block_size is a power of two in [4, 256], as of a block
 * table; head_dim is 64 or 128; kv_heads is in [1, 1024].
 *
 * Block table: int32[n][max_blocks], rows table_stride entries apart;
 * sequence r's token t lies in page table[r][t / block_size], at slot
 * t % block_size. Sequences may share pages (a prefix found by the match);
 * a page that a call writes must be named by one sequence only.
 *
 * Rows of heads (q, k, v, out): element (token t, head j, i) lies at
 * t * token_stride + j * head_stride + i, in elements of type
 * PEEK_TYPE_BF16 or PEEK_TYPE_F16, so slices of a fused projection need no
 * copy. Base pointers are 16-byte aligned, strides multiples of 8 that are
 * not negative; no two rows of out share an element. Query heads are a
 * multiple of the kv heads, at most 65536; query head j reads kv head
 * j / (q_heads / kv_heads).
 *
 * Sums, maxima and weights are held in 32 bits; weights are rounded to the
 * query's type where they meet the values, the output once at the end.
 *
 * Tokens of other sequences, slots past a sequence's end and pages it does
 * not name may hold anything, NaN included: they do not reach its outputs.
 * A page id outside the pool is a broken precondition (PEEK_VALIDATE reports
 * it); memory outside the pool is not touched: peek_kv_append leaves such a
 * block out, attention reads page 0 in its place. Lengths beyond the table
 * (max_blocks * block_size tokens) and negative ones are cut to it.
 * PEEK_VALIDATE checks offsets, lengths, page ids and scales of these calls.
 * ---------------------------------------------------------------------- */
typedef enum peek_type {
  PEEK_TYPE_BF16 = 0,
  PEEK_TYPE_F16 = 1,
  PEEK_TYPE_F8E4M3 = 2,
  PEEK_TYPE_I8 = 3
} peek_type;

/* A pool of pages: device memory of the caller's, described by value (read
 * before a call returns). */
typedef struct peek_kv_pool {
  void* d_pages;      /* 16-byte aligned */
  float* d_scales;
  int64_t num_pages;  /* < 2^31 */
  int32_t kv_heads;
  int32_t block_size;
  int32_t head_dim;
  int32_t type;       /* PEEK_TYPE_F8E4M3 or PEEK_TYPE_I8 */
} peek_kv_pool;

/* ------------------------------------------------------------------------
 * peek_kv_append: quantises the K and V of new tokens into the pool.
 *
 * Sequence r has d_context[r] tokens in the cache; its new ones are rows
 * d_offsets[r] .. d_offsets[r+1] of k and v (num_tokens rows in all) and
 * get the positions after them. d_context is not changed. For every block
 * that gets new tokens, for K and for V and for every head:
 *   a  = the largest finite magnitude among the block's new values
 *   s' = F8E4M3: the smallest power of two with a <= 448 * s'
 *        I8:     a * (1 / 127), both in 32 bits
 *        (both kept within 2^-60 .. 2^60)
 *   s  = s' if the block's first token is new, else max(s', old scale)
 *   code = x / s (in 32 bits) to the nearest the format holds, ties to even,
 *        larger magnitudes (infinities) to the largest; NaN stays NaN in
 *        F8E4M3 and becomes 0 in I8
 * If s is larger than the old scale, the block's older tokens (slots before
 * the first new one) are rounded again to it. Asynchronous on `stream`; no
 * workspace. n = 0 or num_tokens = 0 is a no-op.
 * Errors: INVALID_ARGUMENT, DEVICE.
 * ---------------------------------------------------------------------- */
peek_status peek_kv_append(const peek_kv_pool* pool, int32_t n, int64_t num_tokens, int32_t type, const void* d_k,
                           int64_t k_token_stride, int64_t k_head_stride, const void* d_v, int64_t v_token_stride,
                           int64_t v_head_stride, const int64_t* d_offsets, const int32_t* d_context,
                           const int32_t* d_block_table, int32_t max_blocks, int64_t table_stride, void* stream);

/* ------------------------------------------------------------------------
 * peek_prefill_attention: attention of packed prompts, causal, each after
 * its cached prefix.
 *
 * Sequence r's rows of q, k and v are d_offsets[r] .. d_offsets[r+1] of
 * num_tokens; before them stand d_prefix[r] cached tokens (d_prefix, pool
 * and table may be NULL together: nothing is cached). For its i-th row and
 * every query head, with key and value j running over the prefix and then
 * over its own rows 0 .. i:
 *   x_j = scale * q . k_j
 *   out = sum_j exp(x_j) v_j / sum_j exp(x_j),   lse = log sum_j exp(x_j)
 * d_lse (nullable) is float32[num_tokens][q_heads]. Rows in no sequence are
 * left as they are. A prompt's later tokens do not reach its earlier rows,
 * whatever they hold.
 * Scratch comes only from d_workspace (device, 256-byte aligned, at least
 * peek_prefill_attention_workspace bytes for these sizes; max_context =
 * max_blocks * block_size, 0 without a cache). Asynchronous on `stream`.
 * The token strides of k and v are below 2^23.
 * Errors: INVALID_ARGUMENT, WORKSPACE_TOO_SMALL, DEVICE.
 * ---------------------------------------------------------------------- */
size_t peek_prefill_attention_workspace(int32_t n, int64_t num_tokens, int32_t q_heads, int32_t kv_heads,
                                        int32_t head_dim, int64_t max_context);

peek_status peek_prefill_attention(const peek_kv_pool* pool, int32_t n, int64_t num_tokens, int32_t type,
                                   int32_t q_heads, int32_t kv_heads, int32_t head_dim, const void* d_q,
                                   int64_t q_token_stride, int64_t q_head_stride, const void* d_k,
                                   int64_t k_token_stride, int64_t k_head_stride, const void* d_v,
                                   int64_t v_token_stride, int64_t v_head_stride, const int64_t* d_offsets,
                                   const int32_t* d_prefix, const int32_t* d_block_table, int32_t max_blocks,
                                   int64_t table_stride, float scale, void* d_out, int64_t out_token_stride,
                                   int64_t out_head_stride, float* d_lse, void* d_workspace, size_t workspace_bytes,
                                   void* stream);

/* ------------------------------------------------------------------------
 * peek_decode_attention: attention of one token per sequence over its
 * cached tokens, the d_context[r] first of its pages (the token's own K and V
 * appended before the call where it attends to itself). Row r of q and out
 * is sequence r's; d_lse (nullable) is float32[n][q_heads]. A sequence of no
 * tokens has out = 0 and lse = -infinity.
 *
 * d_mass (nullable) float32[n][kv_heads][max_blocks] receives the weight
 * that falls on every block, summed over the kv head's query heads, on top
 * of d_mass_in (same shape; NULL: zeros; may be d_mass itself):
 *   mass[r][h][b] = mass_in[r][h][b] + sum over those heads and the tokens
 *                   of block b of exp(x - lse)
 * Blocks past the sequence's end keep mass_in. Sums run in a fixed order:
 * equal inputs give equal bits.
 * Scratch comes only from d_workspace (device, 256-byte aligned, at least
 * peek_decode_attention_workspace bytes; with_mass = whether d_mass is
 * given). Asynchronous on `stream`. n = 0 is a no-op.
 * Errors: INVALID_ARGUMENT, WORKSPACE_TOO_SMALL, DEVICE.
 * ---------------------------------------------------------------------- */
size_t peek_decode_attention_workspace(const peek_kv_pool* pool, int32_t n, int32_t q_heads, int32_t max_blocks,
                                       int32_t with_mass);

peek_status peek_decode_attention(const peek_kv_pool* pool, int32_t n, int32_t type, int32_t q_heads, const void* d_q,
                                  int64_t q_token_stride, int64_t q_head_stride, const int32_t* d_context,
                                  const int32_t* d_block_table, int32_t max_blocks, int64_t table_stride, float scale,
                                  void* d_out, int64_t out_token_stride, int64_t out_head_stride, float* d_lse,
                                  const float* d_mass_in, float* d_mass, void* d_workspace, size_t workspace_bytes,
                                  void* stream);

/* ------------------------------------------------------------------------
 * peek_kv_evict: drops the blocks of least accumulated attention weight from
 * sequences that hold more than they may keep.
 *
 * Sequence r of d_context[r] tokens has nb = ceil(context / block_size)
 * blocks and may keep d_keep[r]. A block's score is the sum of its masses
 * over the kv heads (32 bits, heads in ascending order, NaN above all).
 * Candidates are the blocks b with sink <= b < nb - recent (recent >= 1, so
 * the last, perhaps unfinished block stays). The nb - keep candidates of
 * lowest score go (all of them, if there are fewer), equal scores by
 * position. Entries that stay move up in order, those past nb (pages held
 * for tokens to come) included:
 *   d_table_out int32[n][max_blocks], the rest of a row -1
 *   d_mass_out  float32[n][kv_heads][max_blocks], the rest 0
 *   d_freed     int32[n][max_blocks]: the evicted entries by position, then -1
 *               (d_num_freed counts them: an entry may itself be -1)
 *   d_num_freed int32[n],  d_context_out[r] = context - block_size * freed
 * (the context as it was cut to the table, where it was).
 * A page that several sequences name is listed for each that lets go of it,
 * and stays in the tables of the others: the caller counts a shared page's
 * users before it takes one as free.
 * Keys carry their positions already, so attention over what stays needs
 * nothing else. Input and output arrays must not overlap, but d_context_out
 * may be d_context. Scratch comes only from d_workspace (device, 256-byte
 * aligned, at least peek_kv_evict_workspace bytes). Asynchronous on
 * `stream`. n = 0 is a no-op.
 * Errors: INVALID_ARGUMENT, WORKSPACE_TOO_SMALL, DEVICE.
 * ---------------------------------------------------------------------- */
size_t peek_kv_evict_workspace(int32_t n, int32_t kv_heads, int32_t max_blocks);

peek_status peek_kv_evict(int32_t n, int32_t kv_heads, int32_t block_size, const int32_t* d_context,
                          const int32_t* d_block_table, int32_t max_blocks, int64_t table_stride, const float* d_mass,
                          const int32_t* d_keep, int32_t sink, int32_t recent, int32_t* d_context_out,
                          int32_t* d_table_out, float* d_mass_out, int32_t* d_freed, int32_t* d_num_freed,
                          void* d_workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* PEEK_H */
