/*
 * packinfer.h -- C ABI of the MI355X (gfx950) packed-attention library.
 *
 * The calls follow the problem statement of the PackInfer paper (Alg. 1,
 * inputs and outputs; Sec. 3.1 packed computation; Sec. 3.2 packed I/O):
 *
 *   pk_pack_plan            lengths, prefix families, budget C -> groups S_g,
 *                           offset tables O_g                    (Alg. 1)
 *   pk_kv_reorganize        paged KV -> group-contiguous buffers B_g
 *                           (Alg. 1 Part 2, Sec. 3.2 consolidation)
 *   pk_packed_prefill_attn  causal attention over the packed query-key
 *                           regions of each group                (Sec. 3.1)
 *   pk_packed_decode_attn   one query per request over B_g, shared prefix
 *                           read once per group, split-KV + LSE merge
 *                           (Sec. 3.2; Sec. 1 lossless merge)
 *   pk_padded_*             per-request padded execution, the in-run
 *                           comparison the paper argues against (Sec. 2.2)
 *
 * Conventions
 *   - "host" / "device" is stated for every pointer.  Device buffers are
 *     caller-owned; the library never allocates or frees device memory.
 *   - Kernels are enqueued on the caller's hipStream_t (passed as void*,
 *     NULL = default stream) and the call returns without synchronising.
 *     Small integer tables are copied host->device on that stream when a
 *     plan is first used with a workspace (see pk_plan_bind); a host that is
 *     64 such copies ahead of the GPU waits for one of the same stream.
 *   - All tensors are in CALLER REQUEST ORDER; the permutation into groups
 *     is internal.  Every tensor pointer (q, k, v, out, pages, kv_buf, new
 *     rows) must be 16-byte aligned (PK_EINVAL otherwise).
 *   - A plan carries its device tables and the workspace it is bound to:
 *     calls on ONE plan must not run concurrently from several host threads,
 *     and launches that share a workspace must be ordered on the stream(s)
 *     by the caller: decode keeps partial results there, a packed prefill that
 *     works on pieces of key-tile lists does (pk_plan_stat 13), and a first
 *     call may copy tables there.  Different plans
 *     may be used from different threads.  A workspace has ONE owner at a
 *     time, the plan that bound it last: a compute call of another plan on
 *     the same workspace uploads that plan's tables again (the library keeps
 *     track of the last binder per workspace address).  The caller must not
 *     write to, free or reuse the memory of a workspace while a plan that is
 *     bound to it is still in use; after doing so, call pk_plan_bind, which
 *     always uploads.
 *   - Return value: PK_OK (0) or a negative PK_E* code; the message is
 *     available from pk_last_error() (thread-local).  Arguments are checked
 *     before anything is launched.  Nothing throws or aborts: every entry
 *     point catches host exceptions (PK_ENOMEM when host memory runs out).
 *   - dtype: PK_BF16 (MFMA path) or PK_F32 (plain-FMA debug path).  The calls
 *     of the second half of this file (norm, rotation, paged cache, drafted
 *     tokens, branching and judging) need no plan; their lengths and tables are device arrays, which
 *     the kernels bound by the sizes given on the host.
 *     out_dtype: PK_BF16 or PK_F32 for the attention outputs.
 */
#ifndef PACKINFER_H
#define PACKINFER_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum { PK_OK = 0, PK_EINVAL = -1, PK_ENOMEM = -2, PK_EUNSUPPORTED = -3, PK_EHIP = -4 };
enum { PK_BF16 = 0, PK_F32 = 1, PK_F8 = 2 };   /* PK_F8: of a pk_cache only */

/* Layout constants of the group-contiguous buffer. */
#define PK_GROUP_ALIGN 32      /* group bases are multiples of this many tokens */
#define PK_KV_BLOCK    32      /* tokens per tile of the bf16 buffer layout     */

typedef struct pk_plan pk_plan; /* opaque; host memory owned by the library */

/* ------------------------------------------------------------------------
 * pk_pack_plan -- Alg. 1 Part 1 (greedy length-balanced grouping under the
 * feasibility test of Eq. 2, token term) and the bookkeeping of Part 2
 * (prefix-first layout, offset tables O_g).  Deterministic, integer only.
 *
 *   kv_lens     host [n]  L_i: KV tokens request i attends to (incl. the
 *                         current token); > 0
 *   q_lens      host [n]  query rows of request i; NULL = kv_lens (plain
 *                         prefill); 1 = decode; < kv_len = chunked prefill.
 *                         Queries are the last q_len positions.
 *   prefix_ids  host [n]  family id (>= 0) or -1; NULL = no families
 *   prefix_lens host [n]  shared-prefix length, equal inside a family,
 *                         0 <= prefix_len <= kv_len; NULL iff prefix_ids NULL
 *   n                     number of requests (0 is allowed: empty plan)
 *   token_budget          C > 0, unique KV tokens per group (Sec. 3.2)
 *   headroom              delta >= 0 tokens reserved after every suffix
 *   out                   receives the plan; free with pk_plan_destroy
 *
 * Grouping rules: a family is one atomic item of length L_P + sum(L_Q); a
 * family longer than C is cut in member order into the fewest consecutive
 * sub-families that fit; items are sorted by (length desc, lowest member
 * index), the least-loaded group (lowest index on ties) takes the item if it
 * stays within C, otherwise a new group is opened; an item longer than C is
 * alone in its group; empty groups are dropped.
 * Errors: PK_EINVAL for any violated precondition.
 */
int pk_pack_plan(const int32_t* kv_lens, const int32_t* q_lens,
                 const int32_t* prefix_ids, const int32_t* prefix_lens,
                 int32_t n, int64_t token_budget, int32_t headroom, pk_plan** out);

/* pk_pack_plan_tree -- the same planner for NESTED shared prefixes (Sec. 3.2
 * "Prefix-Aware Grouping and Reuse": TriePartition yields shared prefixes at
 * every level of the prefix tree; Eq. 5 counts each shared segment once).
 * The prefixes are given as a forest of segments:
 *   node_parent host [n_nodes]  parent of node k, in [-1, k) (-1: a root)
 *   node_len    host [n_nodes]  tokens of the segment, > 0; a node stands for
 *                               the tokens [depth(parent), depth(parent)+len)
 *                               of every request below it
 *   req_node    host [n]        deepest node above request i, or -1; the
 *                               request's own suffix is what follows
 *                               depth(req_node[i]) (it may be empty)
 *   kv_lens, q_lens, token_budget, headroom, out: as for pk_pack_plan.
 * Every node needs at least one request below it.  The caller guarantees
 * that requests below a node hold identical K/V on that segment.
 * Grouping: a whole tree is one atomic item of length sum(node_len) +
 * sum(suffixes) and is never cut (a tree above C is alone in its group);
 * otherwise as pk_pack_plan.  Layout inside a group, per tree in pre-order:
 * the node's segment, the suffixes (+ headroom) of the requests attached
 * directly to it in ascending order, then its children in ascending order.
 * pk_trie_tree produces this input from token ids.  A forest of roots only
 * gives the layout of pk_pack_plan with uncut families.
 * Errors: PK_EINVAL for any violated precondition.
 */
int pk_pack_plan_tree(const int32_t* kv_lens, const int32_t* q_lens, int32_t n,
                      const int32_t* node_parent, const int32_t* node_len, int32_t n_nodes,
                      const int32_t* req_node, int64_t token_budget, int32_t headroom,
                      pk_plan** out);

void pk_plan_destroy(pk_plan* plan);

/* Read-only accessors (host). */
int32_t pk_plan_num_requests(const pk_plan* plan);
int32_t pk_plan_num_groups(const pk_plan* plan);
/* Tokens of the whole buffer (all groups, each base rounded up to
 * PK_GROUP_ALIGN; the total is a multiple of PK_KV_BLOCK). */
int64_t pk_plan_buf_tokens(const pk_plan* plan);
/* Unique KV tokens summed over groups: the I/O volume M of Eq. 5 without
 * headroom. */
int64_t pk_plan_unique_tokens(const pk_plan* plan);

/* Canonical serialisation, int32 words:
 *   magic 0x504B504C, version 1, n, G, C lo, C hi, headroom, PK_GROUP_ALIGN,
 *   buf_tokens lo, hi, then per group:
 *   load lo, hi, buf_tokens lo, hi, buf_base lo, hi, n_members, then per
 *   member (layout order): request, prefix_off, L_P, suffix_off, L_Q
 *   (offsets in tokens relative to the group base) -- the tuple O_g[i] of
 *   Alg. 1.
 * A plan of pk_pack_plan_tree has version 2 and per group, after buf_base:
 *   n_nodes, n_members, then per node (layout order): caller's node number,
 *   offset, tokens, parent (index among the group's nodes or -1), then per
 *   member (layout order): request, node (index among the group's nodes or
 *   -1), suffix_off, suffix tokens.
 * pk_plan_serialized_words returns the word count; pk_plan_serialize copies
 * them to host `out` (capacity `cap` words) and returns the count or
 * PK_EINVAL if cap is too small. */
int64_t pk_plan_serialized_words(const pk_plan* plan);
int64_t pk_plan_serialize(const pk_plan* plan, int32_t* out, int64_t cap);

/* ------------------------------------------------------------------------
 * Sizes of the caller-allocated device buffers.
 *
 * pk_kv_buf_bytes: bytes of the group-contiguous KV buffer.
 *   PK_BF16 layout: [Hkv][buf_tokens / 32] tiles; one tile holds 32 tokens of
 *   one KV head: first the K part (32*d bf16), then the V part (32*d bf16).
 *     K part: two sub-tiles u (tokens 16u..16u+15), each d/32 steps s of
 *       64 chunks l of 8 bf16: chunk (u,s,l)[j] = K[16u + l%16][32s + 8(l/16) + j]
 *     V part: d/16 column blocks t of 64 chunks l of 8 bf16:
 *       chunk (t,l)[j] = V[kappa(l/16, j)][16t + l%16],
 *       kappa(g, j) = 4g + j for j < 4, 16 + 4g + (j-4) otherwise.
 *   (This is the operand order of the 16x16x32 bf16 MFMA, so the decode
 *   kernel streams tiles with fully coalesced 16-byte loads.)  Token slots
 *   that hold no valid token (headroom, alignment) are written as zeros.
 *   PK_F32 layout: K as [Hkv][buf_tokens][d] floats, then V likewise.
 *
 * pk_workspace_bytes: bytes of the workspace that carries the plan's device
 *   tables and the partial results (of split-KV decode, of pieces of key-tile
 *   lists in prefill) for the given head shape.
 */
size_t pk_kv_buf_bytes(const pk_plan* plan, int Hkv, int d, int dtype);
size_t pk_workspace_bytes(const pk_plan* plan, int Hq, int Hkv, int d, int dtype);

/* Builds the device tables of the plan for this head shape and copies them
 * into `workspace` (device, >= pk_workspace_bytes, 256-byte aligned) on
 * `stream`.  Optional: the compute calls bind on first use of a
 * (workspace, shape) pair; rebinding to another workspace is allowed.  The
 * caller must not modify the workspace while the plan is in use.
 * Two tables are built and copied later, by the first call that needs them,
 * on its stream: those of pk_padded_prefill_attn, and for a plan whose q_lens
 * are all 1 those of its packed prefill (pk_packed_prefill_attn, the prefill
 * half of a mixed step).
 * Under stream capture a copy of tables becomes a node of the graph, and the
 * host memory that it reads stays with the graph.  It counts for the later
 * calls of the same capture only: calls outside of it, or in another capture,
 * copy again.  A captured call whose tables are already in place (the same
 * call was made on the workspace before, eagerly) is kernel launches alone. */
int pk_plan_bind(pk_plan* plan, int Hq, int Hkv, int d, int dtype,
                 void* workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------
 * pk_kv_reorganize -- Alg. 1 Part 2 / Sec. 3.2 "Contiguous Memory
 * Consolidation": gathers the valid tokens of every request from the paged
 * pool into the group buffers, each shared prefix once (taken through the
 * block table of the family's lowest-index member in the group).
 *
 *   k_pages, v_pages  device [num_blocks][page_size][Hkv][d], dtype
 *   block_table       device [n][max_blocks_per_req] int32, logical page b
 *                     of request i -> physical block; entries beyond the
 *                     request's length are ignored
 *   num_blocks        physical blocks in the pool (for bounds validation of
 *                     nothing but the caller's own sizes; block ids are
 *                     clamped into [0, num_blocks))
 *   kv_buf            device, pk_kv_buf_bytes; written
 * Errors: PK_EINVAL (null pointer, page_size <= 0, max_blocks too small for
 * the longest request), PK_EUNSUPPORTED (bf16 path needs d in {64, 128}).
 */
int pk_kv_reorganize(pk_plan* plan, const void* k_pages, const void* v_pages,
                     const int32_t* block_table, int32_t max_blocks_per_req,
                     int32_t page_size, int64_t num_blocks, int Hkv, int d, int dtype,
                     void* kv_buf, void* workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------
 * pk_packed_prefill_attn -- Sec. 3.1: attention computed directly over the
 * union of valid query-key regions of each group: query tiles are cut from
 * the group's packed token stream (a tile may span requests), only key tiles
 * holding at least one unmasked pair are visited, block-diagonal causal mask,
 * online softmax.  out[t,h,:] = softmax_j(scale * q[t,h].k[j,g(h)]) v[j,g(h)]
 * over the keys j <= ctx + t of the same request, g(h) = h / (Hq/Hkv).
 *
 *   q    device [sum q_lens][Hq][d]    k, v  device [sum kv_lens][Hkv][d]
 *   out  device [sum q_lens][Hq][d], out_dtype
 *   scale  finite and positive (here and in every attention call below)
 * Errors: PK_EINVAL; PK_EUNSUPPORTED (bf16 path: d in {64,128}, Hq % Hkv == 0).
 */
int pk_packed_prefill_attn(pk_plan* plan, const void* q, const void* k, const void* v,
                           void* out, float scale, int Hq, int Hkv, int d,
                           int dtype, int out_dtype,
                           void* workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------
 * pk_packed_decode_attn -- Sec. 3.2: every request has ONE query row (the
 * plan must have been made with q_lens == 1).  KV is read from the group
 * buffer written by pk_kv_reorganize; a shared prefix segment is streamed
 * once for all members of its (sub-)family in the group; segments are cut
 * into fixed-size splits whose partial results are merged by log-sum-exp
 * (the lossless merge of Sec. 1).
 *
 *   q    device [n][Hq][d]       kv_buf  device, as written by reorganize
 *   out  device [n][Hq][d], out_dtype
 * Errors: PK_EINVAL; PK_EUNSUPPORTED (bf16 path: d in {64,128}, Hq/Hkv <= 32,
 * any ratio; a work item carries 32 / (Hq/Hkv) requests of a shared prefix).
 */
int pk_packed_decode_attn(pk_plan* plan, const void* q, const void* kv_buf,
                          void* out, float scale, int Hq, int Hkv, int d,
                          int dtype, int out_dtype,
                          void* workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------
 * pk_packed_mixed_step -- Sec. 3 (overview): the prefill and the decode
 * requests of one continuous-batching step go through the same packed
 * execution.  One call for both halves of such a step: the packed prefill
 * tiles of `prefill_plan` and the packed decode work items of `decode_plan`
 * run in ONE launch in which workgroups of the two kinds alternate, so that
 * the HBM-bound decode work runs beside the matrix-bound prefill work on the
 * same compute units; the LSE merge of the decode partials follows as a
 * second launch.  Results are those of pk_packed_prefill_attn and
 * pk_packed_decode_attn (same arithmetic per tile and per work item; where the
 * prefill call cuts long key-tile lists into pieces, pk_plan_stat 13, and the
 * decode half outlasts the whole lists, they stay whole here, and the prefill
 * results are that call's but for rounding).
 *   prefill half: prefill_plan, q, k, v, out, prefill_workspace (as for
 *                 pk_packed_prefill_attn)
 *   decode half:  decode_plan (q_lens == 1), decode_q, kv_buf (written by
 *                 pk_kv_reorganize), decode_out, decode_workspace (as for
 *                 pk_packed_decode_attn); the workspaces must differ
 *   scale, Hq, Hkv, d, dtype, out_dtype: common to both halves (one layer)
 * A plan with n = 0 makes the call equal to the other half's own call.
 * Errors: as for the two calls; PK_EUNSUPPORTED unless dtype is PK_BF16 and
 * d is 64 or 128. */
int pk_packed_mixed_step(pk_plan* prefill_plan, const void* q, const void* k, const void* v, void* out,
                         void* prefill_workspace, size_t prefill_workspace_bytes,
                         pk_plan* decode_plan, const void* decode_q, const void* kv_buf, void* decode_out,
                         void* decode_workspace, size_t decode_workspace_bytes,
                         float scale, int Hq, int Hkv, int d, int dtype, int out_dtype, void* stream);

/* pk_packed_decode_attn_static -- pk_packed_decode_attn for callers that
 * cannot allocate device memory: code under HIP graph capture, tight serving
 * loops, harnesses that forbid hipMalloc.  It takes no workspace: the plan's
 * device tables and the split-KV partial results live in a fixed array of
 * PK_STATIC_SCRATCH_BYTES that is part of the library's code object (every
 * GPU the library runs on holds its own copy until the process ends).  The
 * call allocates and frees nothing, on the device or through the runtime.
 *   - The first call of a plan on a device (and the first after another plan
 *     used the scratch) uploads the plan's tables with one host-to-device copy
 *     on `stream`; further calls of that plan only launch kernels.
 *   - A plan whose tables (those of its packed prefill count) and partial
 *     results have more than PK_STATIC_SCRATCH_BYTES, with a wave for every
 *     work item and one split, is rejected with PK_EUNSUPPORTED and a message
 *     that states both sizes (use pk_packed_decode_attn with a workspace).
 *   - All calls on one GPU share the one array, which keeps the contents of
 *     the last call: calls that overlap in time on one GPU (different
 *     streams, different threads) race and must be ordered by the caller.
 *     Nothing in it has to be prepared: every partial slot is written before
 *     the merge reads it, and the counts of finished work items, which have
 *     to be zero when a launch begins, are zeroed by the upload of a plan's
 *     tables and left at zero by every launch.
 * Other arguments, results and errors as pk_packed_decode_attn; the outputs
 * are bit-identical to that call's. */
#define PK_STATIC_SCRATCH_BYTES (16u << 20)
int pk_packed_decode_attn_static(pk_plan* plan, const void* q, const void* kv_buf,
                                 void* out, float scale, int Hq, int Hkv, int d,
                                 int dtype, int out_dtype, void* stream);

/* ------------------------------------------------------------------------
 * pk_trie_partition -- TriePartition of Alg. 1 Part 2 from token ids (Sec.
 * 3.2: the requests of a batch form a prefix tree whose common prefixes are
 * stored once).  Produces the prefix_ids / prefix_lens that pk_pack_plan
 * takes: every request is assigned to at most one shared prefix, a prefix
 * has at least min_prefix tokens and at least two requests, and among all
 * such assignments the one with the largest saving sum d_k * (m_k - 1) is
 * returned (d_k tokens shared by m_k requests: the reduction of Eq. 5); on a
 * tie between a prefix and the prefixes nested below it the outer one wins.
 * Families are numbered by their lowest request index.  Host only.
 *
 *   token_ids     host, the n token sequences one after the other
 *   kv_lens       host [n], length of each sequence (> 0)
 *   prefix_ids    host [n] out: family or -1     prefix_lens  host [n] out
 *   saved_tokens  optional out: the saving
 * Errors: PK_EINVAL (NULL, n < 0, min_prefix < 1, kv_len <= 0).
 */
int pk_trie_partition(const int32_t* token_ids, const int32_t* kv_lens, int32_t n,
                      int32_t min_prefix, int32_t* prefix_ids, int32_t* prefix_lens,
                      int64_t* saved_tokens);

/* pk_trie_tree -- the whole prefix tree of a batch as the forest of shared
 * segments pk_pack_plan_tree takes (Sec. 3.2; Eq. 5 at every level: a segment
 * of len tokens above m requests saves len * (m - 1) tokens).  A node is made
 * for every branching point of the tree (or end of a request) below which at
 * least two requests lie and whose depth is at least min_prefix; runs without
 * branching are one segment.  Host only.
 *   token_ids, kv_lens, n, min_prefix: as for pk_trie_partition
 *   node_parent, node_len host [n] out: the first *n_nodes entries are set
 *                         (there are at most n - 1 nodes)
 *   n_nodes     host out
 *   req_node    host [n] out: deepest node above request i or -1
 *   saved_tokens host out (may be NULL)
 * Nodes are numbered by (lowest request below, depth), so parents precede
 * children and the output does not depend on the sort inside.
 * Errors: PK_EINVAL for any violated precondition.
 */
int pk_trie_tree(const int32_t* token_ids, const int32_t* kv_lens, int32_t n,
                 int32_t min_prefix, int32_t* node_parent, int32_t* node_len,
                 int32_t* n_nodes, int32_t* req_node, int64_t* saved_tokens);

/* ------------------------------------------------------------------------
 * Decoding over several steps with one plan (Sec. 3.2: every suffix is
 * allocated L_Q + delta tokens, "which reserves space for future token
 * generation"; Sec. 3.1 "Adaptive Grouping", Eq. 4: when to regroup).
 *
 * Step s = 0, 1, ... of a decode loop:
 *   1. pk_kv_append(step = s) writes the K/V rows of the token that every
 *      request has just produced into the headroom behind its suffix in
 *      kv_buf (buffer token suffix_off + L_Q + s; layout as documented at
 *      pk_kv_buf_bytes).  k_new, v_new: device [n][Hkv][d], dtype, request
 *      order.  Needs 0 <= s < headroom, else PK_EINVAL (no slot left: make a
 *      new plan from the grown lengths and reorganize).
 *   2. pk_packed_decode_attn_grown(grown = s + 1) is pk_packed_decode_attn
 *      with every request's suffix extended by the `grown` appended tokens
 *      (request i then has kv_len_i + grown keys).  grown in [0, headroom].
 * Both use the plan's tables as they are; nothing is re-planned or copied.
 * Calls of one step are ordered by the stream.
 *
 * pk_regroup_due evaluates the trigger of Eq. 4 after `steps` decode steps
 * since the plan was made: with L_g(steps) = L(S_g) + steps * |S_g| (every
 * member adds one unique token per step, prefixes do not grow) and
 * DeltaL = max_g L_g - min_g L_g, it sets PK_REGROUP_DRIFT in *flags when
 * steps * DeltaL >= C / 2, and PK_REGROUP_HEADROOM when steps >= headroom
 * (the next append has no slot).  *drift (optional) receives DeltaL.
 * PK_REGROUP_DRIFT_WITHIN_BUDGET is the same rule over the groups whose
 * initial load is at most C: a group that Alg. 1 opened for one item longer
 * than C cannot be balanced by regrouping and makes the plain rule fire at
 * the first step.  Host only, no device work.
 * Errors: PK_EINVAL (NULL, steps < 0).
 */
#define PK_REGROUP_DRIFT               1
#define PK_REGROUP_HEADROOM            2
#define PK_REGROUP_DRIFT_WITHIN_BUDGET 4
int pk_kv_append(pk_plan* plan, const void* k_new, const void* v_new, void* kv_buf,
                 int32_t step, int Hkv, int d, int dtype,
                 void* workspace, size_t workspace_bytes, void* stream);
int pk_packed_decode_attn_grown(pk_plan* plan, const void* q, const void* kv_buf,
                                void* out, float scale, int32_t grown, int Hq, int Hkv, int d,
                                int dtype, int out_dtype,
                                void* workspace, size_t workspace_bytes, void* stream);
int pk_regroup_due(const pk_plan* plan, int32_t steps, int32_t* flags, int64_t* drift);

/* ------------------------------------------------------------------------
 * In-run comparison: per-request padded execution (Sec. 2.2: request-aligned
 * tile grids, padding to the tile size, no cross-request packing).  Same
 * mathematics and tensor conventions as the packed calls.
 *   prefill: grid (request, query tile, head) sized by the longest request;
 *            every request's last tile is padded; natural request order.
 *   decode:  reads the PAGED pool through the block table, uniform number
 *            of splits sized by the longest request, shared prefixes re-read
 *            by every member.  bf16 only, d in {64,128}, Hq/Hkv <= 16
 *            (PK_EUNSUPPORTED otherwise).
 */
int pk_padded_prefill_attn(pk_plan* plan, const void* q, const void* k, const void* v,
                           void* out, float scale, int Hq, int Hkv, int d,
                           int dtype, int out_dtype,
                           void* workspace, size_t workspace_bytes, void* stream);
int pk_padded_decode_attn(pk_plan* plan, const void* q,
                          const void* k_pages, const void* v_pages,
                          const int32_t* block_table, int32_t max_blocks_per_req,
                          int32_t page_size, int64_t num_blocks,
                          void* out, float scale, int Hq, int Hkv, int d,
                          int dtype, int out_dtype,
                          void* workspace, size_t workspace_bytes, void* stream);

/* Counts for the benchmark's work accounting (host).  1..13 refer to the
 * tables of the head shape the plan was last sized or bound for (0 before).
 *   what = 0: unmasked (query,key) pairs per head summed over requests
 *   what = 1: (query,key) pairs issued to the MFMA units by the packed
 *             prefill schedule, per head
 *   what = 2: same for the padded prefill schedule
 *   what = 3: decode work items; 4: split-KV partial slots;
 *   what = 5: tokens per decode split chosen by the schedule builder (shared
 *             segments may have another unless PK_TUNE_DECODE_SPLIT says one)
 *   what = 6: query tiles of the packed prefill schedule, counted in tiles of
 *             128 rows whatever tiles the launch has (12); 7: of the padded
 *   what = 8: 1 if the packed bf16 prefill (also the prefill half of a mixed
 *             step) takes the kernels for launches of little work, 0 if the
 *             software-pipelined ones; 9: same for the padded schedule
 *   what = 10: waves that share a (decode work item, KV head) pair: 4 (a
 *             workgroup, which merges in the same launch), 1, or 0 (no items)
 *   what = 11: waves of a workgroup of the packed bf16 prefill: 8 or 4 (the
 *             prefill half of a mixed step always has 4; 0: no bf16 tables)
 *   what = 12: query rows of its tiles: 128, or 64 or 32 (a request's alone)
 *             which the workgroup's waves take for several heads
 *   what = 13: pieces that the packed prefill works on where it cuts long
 *             key-tile lists (few workgroups), 0 where it does not
 */
int64_t pk_plan_stat(const pk_plan* plan, int what);

/* Offline profiling of schedule parameters (Sec. 3.1: capacity and tile
 * shapes are found by profiling a range of settings).  Overrides a choice of
 * the schedule builder for this plan; the next pk_workspace_bytes /
 * pk_plan_bind builds the tables again.  Results never depend on it.
 *   PK_TUNE_DECODE_SPLIT     tokens per split-KV work item (rounded up to
 *                            PK_KV_BLOCK); 0 = the builder's own choice.
 *                            The kernel stays the one that 0 gives (a wave
 *                            or a workgroup for an item)
 *   PK_TUNE_PREFILL_PIPELINE how the bf16 prefill kernels (packed and padded)
 *                            bring K/V tiles into LDS: 0 = copied straight
 *                            from memory into LDS, three K and two V stages
 *                            (default); 1 = staged through registers, two
 *                            stages with padded rows.  Same query tiles and
 *                            key tiles of 64, same arithmetic.
 *                            (pk_packed_mixed_step always runs pipeline 0.)
 * Errors: PK_EINVAL (NULL plan, unknown knob, value out of range). */
#define PK_TUNE_DECODE_SPLIT 0
#define PK_TUNE_PREFILL_PIPELINE 1
int pk_plan_tune(pk_plan* plan, int knob, int64_t value);

/* ========================================================================
 * One step of a (speculative) decode loop on a paged cache: the projections
 * of the new tokens are normed and rotated, quantised into the cache as they
 * are written, attended to, and the drafted tokens that were accepted stay.
 *
 *   pk_qk_norm_rope    norm and rotation of queries and keys
 *   pk_kv_cache_write  rows of K and V into the cache
 *   pk_qkv_cache_write the two in one launch
 *   pk_kv_cache_read   the cache back as rows, as pk_packed_prefill_attn takes
 *                      the context of a chunk
 *   pk_tree_attn       drafted tokens of every request over its cache; with one
 *                      token a request a plain decode step
 *   pk_kv_cache_keep   accepted tokens move up behind the context
 *
 * Nothing here allocates, and nothing depends on host copies of lengths: a
 * step can be captured in a graph and replayed while the lengths grow.
 * ======================================================================== */

/* Rows [token][head][d] in device memory; strides in elements, the d columns of
 * a row contiguous.  dtype PK_BF16 or PK_F32.  data and both strides are whole
 * multiples of 16 bytes (PK_EINVAL otherwise); strides are not negative, lead
 * over no more than 2^59 elements, and those of outputs keep rows apart.  An output may be its own input (same data and
 * strides), and otherwise does not overlap any input. */
typedef struct pk_rows {
    void* data;
    int64_t token_stride, head_stride;
    int32_t dtype;
} pk_rows;

/* Rotary positions.  Pair p of a row is rotated by the angle whose cosine and
 * sine stand in row positions[axis(p)][token] of the table:
 *   (a, b) -> (a cos - b sin, b cos + a sin)
 *   table      device float [max_pos][2][rot_dim / 2]: cosines, then sines
 *   positions  device int32, axis x at positions + x * axis_stride, [tokens]
 *              each; clamped into [0, max_pos)
 *   rot_dim    a multiple of 16, at most d; columns from rot_dim on stay
 *   pair_axis  host [rot_dim / 2]: axis of every pair (several axes: time,
 *              height and width of images and video); NULL: axis 0
 *   interleaved  0: pair p is columns (p, p + rot_dim / 2); 1: (2p, 2p + 1) */
typedef struct pk_rope {
    const float* table;
    const int32_t* positions;
    int64_t axis_stride;
    const uint8_t* pair_axis;
    int32_t max_pos, rot_dim, n_axes, interleaved;
} pk_rope;

/* Paged cache of keys and values.
 *   k       device [num_blocks][Hkv][page_size][d]
 *   v       device [num_blocks][Hkv][page_size / 4][d][4]: four tokens
 *           interleaved, so that the four keys that a lane of an MFMA takes of a
 *           column lie side by side
 *   scales  device [num_blocks][Hkv][2][page_size] (of K, of V); PK_F8 only
 * page_size is a multiple of 16, d 64 or 128 (PK_EUNSUPPORTED otherwise).
 * dtype PK_BF16: k and v are bf16 and scales is not read.  dtype PK_F8: k and v
 * are E4M3 codes (4 exponent bits, 3 fraction bits, no infinities), scales are
 * exponent bytes: b stands for 2^(b - 127), 1 <= b <= 254.  A row's byte is the
 * smallest whose scale s keeps its largest finite magnitude within 448 s, and
 * the code of x is x / s rounded to nearest even: dividing is exact, and what a
 * code stands for, code * s, is a bf16 number (but for the ends of the range: below
 * 2^-126 bf16 has multiples of 2^-133, and 2^128, to which magnitudes from 1.9375
 * * 2^127 on are rounded, is read as infinite).  A row of zeros has b = 1.  NaN and
 * infinities become NaN.
 * Slot number s of the cache is token s % page_size of block s / page_size. */
typedef struct pk_cache {
    void* k;
    void* v;
    void* scales;
    int64_t num_blocks;
    int32_t page_size, Hkv, d, dtype;
} pk_cache;

/* pk_qk_norm_rope -- for every row x of q and k:  y = x * rsqrt(mean(x^2) + eps)
 * * weight, then the rotation; one pass, in fp32, rounded once to the type of
 * the output (any of the two, for any type of the input).
 *   q [tokens][Hq][d], k [tokens][Hkv][d], both of one dtype; q_out, k_out too
 *   q_weight, k_weight  device [d] in the dtype of q and k; NULL: no norm of q
 *                       (of k)
 *   rope                NULL: no rotation
 * d is a multiple of 8 and at most 256 (PK_EUNSUPPORTED otherwise).
 * Errors: PK_EINVAL; PK_EUNSUPPORTED. */
int pk_qk_norm_rope(const pk_rows* q, const pk_rows* k, const pk_rows* q_out, const pk_rows* k_out,
                    const void* q_weight, const void* k_weight, float eps, const pk_rope* rope,
                    int64_t tokens, int Hq, int Hkv, int d, void* stream);

/* pk_kv_cache_write -- rows of K and V [tokens][Hkv][d] (one dtype) into the
 * slots of the cache.
 *   slots  device int64 [tokens]; a token whose slot is outside of the cache
 *          (-1: padding) is not written.  Two tokens must not have one slot.
 * Errors: PK_EINVAL; PK_EUNSUPPORTED (page size, d). */
int pk_kv_cache_write(const pk_cache* cache, const pk_rows* k, const pk_rows* v, const int64_t* slots,
                      int64_t tokens, void* stream);

/* pk_qkv_cache_write -- pk_qk_norm_rope and pk_kv_cache_write in one launch: q
 * goes to q_out, k is normed and rotated in fp64 and rounded once, to what the
 * cache holds, v is written.  q, k and v of one dtype. */
int pk_qkv_cache_write(const pk_cache* cache, const pk_rows* q, const pk_rows* k, const pk_rows* v,
                       const int64_t* slots, const pk_rows* q_out,
                       const void* q_weight, const void* k_weight, float eps, const pk_rope* rope,
                       int64_t tokens, int Hq, void* stream);

/* pk_kv_cache_read -- tokens 0 .. kv_lens[i] - 1 of every request as rows
 * row_start[i] + 0, 1, ... of k_out and v_out ([rows][Hkv][d], one dtype).
 *   block_table  device int32 [n][max_blocks]: physical block of a request's
 *                logical pages, clamped into [0, num_blocks)
 *   kv_lens, row_start  device int32 [n]; lengths are clamped into
 *                [0, max_blocks * page_size]; tokens whose row would be `rows` or
 *                more are not written, nor is a request with a negative row_start.
 *                The requests' rows must not overlap.
 * Errors: PK_EINVAL; PK_EUNSUPPORTED. */
int pk_kv_cache_read(const pk_cache* cache, const int32_t* block_table, int32_t max_blocks,
                     const int32_t* kv_lens, const int32_t* row_start, int32_t n,
                     const pk_rows* k_out, const pk_rows* v_out, int64_t rows, void* stream);

/* pk_tree_attn -- attention of the last T_i = q_start[i + 1] - q_start[i] tokens
 * of every request (the drafted ones, whose rows are in the cache already) over
 * its kv_lens[i] tokens.  All see the kv_lens[i] - T_i tokens of the context;
 * among the drafted ones token t sees those whose bit is set in its mask word.
 * A row that sees nothing is zero.  What a row does not see cannot reach it, be
 * it infinite or NaN.
 *   q         device [total_q][Hq][d] bf16, 16-byte aligned
 *   q_start   device int32 [n + 1], not decreasing, within [0, total_q]
 *   max_q     the most drafted tokens of a request (at least the largest T_i;
 *             PK_EUNSUPPORTED above 64); tokens beyond it are not computed
 *   tree_mask device uint64 [total_q]: bit j for drafted token j of the same
 *             request; NULL: token t sees tokens 0 .. t
 *   block_table, kv_lens: as for pk_kv_cache_read (tokens of a length that the
 *             table has no pages for are not there, drafted ones first)
 *   out       device [total_q][Hq][d], out_dtype, 16-byte aligned
 *   workspace device, 256-byte aligned, at least pk_tree_attn_workspace_bytes.
 *             ZERO-FILLED BEFORE ITS FIRST USE; every call leaves it ready for the
 *             next.  One workspace serves all calls with the same Hkv for which it is
 *             large enough (PK_EINVAL otherwise), whatever it was made for; the
 *             caller orders them.
 * The partial results of a request are put together in a fixed order: results
 * repeat bit for bit.  Probabilities are rounded to bf16 for the matrix pipe,
 * whatever out_dtype is: a result is off by up to 2^-8 of sum p |v|, on the whole
 * by 1e-3 of its norm; PK_F32 output leaves out its own rounding alone.  Scores
 * and sums have 32 bits: where the largest score is s, sums of exp(score - s) v, in
 * parts times up to 2^8, have to stay below 2^128.
 * Errors: PK_EINVAL; PK_EUNSUPPORTED (page size, d, max_q). */
#define PK_MAX_DRAFTS 64
size_t pk_tree_attn_workspace_bytes(int32_t n, int32_t max_q, int Hq, int Hkv, int d);
int pk_tree_attn(const pk_cache* cache, const void* q, const int32_t* q_start, int64_t total_q, int32_t max_q,
                 const uint64_t* tree_mask, const int32_t* block_table, int32_t max_blocks,
                 const int32_t* kv_lens, int32_t n, void* out, float scale, int Hq, int out_dtype,
                 void* workspace, size_t workspace_bytes, void* stream);

/* pk_kv_cache_keep -- after the drafted tokens have been judged: drafted tokens
 * keep[i][0] < keep[i][1] < ... < keep[i][keep_count[i] - 1] of request i (the
 * accepted branch) become tokens 0, 1, ... behind its context, bit for bit, and
 * new_lens[i] = kv_lens[i] - T_i + keep_count[i].
 *   keep        device int32 [n][max_keep], rising in every row; numbers outside
 *               of [0, T_i) are passed over
 *   keep_count  device int32 [n]; clamped into [0, min(max_keep, T_i)]
 *   new_lens    device int32 [n], not kv_lens itself nor in another of the arrays
 * Other arguments as for pk_tree_attn.  Errors: PK_EINVAL; PK_EUNSUPPORTED. */
int pk_kv_cache_keep(const pk_cache* cache, const int32_t* block_table, int32_t max_blocks,
                     const int32_t* kv_lens, const int32_t* q_start, int32_t n,
                     const int32_t* keep, int32_t max_keep, const int32_t* keep_count,
                     int32_t* new_lens, void* stream);

/* ========================================================================
 * Branching and judging around that step: requests that come from one another
 * share pages, pages are handed out, copied and moved on the device, and the
 * drafted tokens that stay are found from the target's logits.
 *
 *   pk_kv_pages_select   a new batch out of rows of the old one: forked,
 *                        reordered and finished requests
 *   pk_kv_pages_reserve  pages for the next tokens of every request; a shared
 *                        page that would be written is replaced by a copy
 *   pk_kv_pages_compact  the pages in use get the lowest numbers
 *   pk_kv_cache_copy     pages of one layer's cache
 *   pk_shared_tree_attn  pk_tree_attn that reads shared pages once
 *   pk_draft_verify      which drafted tokens stay, and the token behind them
 *
 * Nothing here allocates or reads lengths on the host: a step of all of them
 * can be captured in a graph.
 *
 * The pages of a batch.  One batch serves all layers; what has to be copied is
 * therefore a list, which pk_kv_cache_copy takes for each layer's cache.
 *   block_table  device int32 [n][max_blocks]: the blocks of a request's pages
 *   lens         device int32 [n]: its tokens
 *   pages        device int32 [n]: entries of its row that it holds (at least
 *                those of its tokens; more where room was reserved, or where it
 *                was cut to fewer tokens)
 *   refs         device int32 [num_blocks]: how many requests hold a block;
 *                0: it is free.  A caller may count itself in for blocks that are
 *                to outlive the requests (a prefix that is kept).
 * Lengths and pages are clamped into what a row has room for; entries outside
 * of [0, num_blocks) are carried along and counted nowhere.
 * ======================================================================== */

/* pk_kv_pages_select -- request i of the new batch is request from[i] of the old
 * one (several times the same: forks; from[i] outside of [0, n): an empty
 * request) with the pages of its tokens; room that was reserved beyond them is
 * given up.  refs changes by what the new batch holds less what the old one
 * held, so a request that is not taken over is freed.
 *   from, new_lens, new_pages  device int32 [n_new]; new_table [n_new][max_blocks],
 *             whose entries behind a request's pages are left as they are
 * No output overlaps an input or another output.  Errors: PK_EINVAL. */
int pk_kv_pages_select(const int32_t* block_table, const int32_t* lens, const int32_t* pages, int32_t n, int32_t max_blocks,
                       const int32_t* from, int32_t n_new, int32_t* new_table, int32_t* new_lens, int32_t* new_pages,
                       int32_t* refs, int64_t num_blocks, int32_t page_size, void* stream);

/* pk_kv_pages_reserve -- every request gets pages for lens[i] + grow[i] tokens (no
 * more than max_blocks of them), in the order of requests the free blocks of
 * the lowest numbers.  Where its next token goes to a page that holds tokens of
 * its own and that others hold too, the page is replaced by a free block and
 * noted for copying: copy_src[i] -> copy_dst[i] (-1: nothing to copy), its block
 * before its other new ones.  If all holders of such a page grow in this call,
 * the one of the highest number keeps it.  Where tokens would go to a page
 * behind its own ones that others hold too (it was cut to fewer tokens behind a
 * fork), it gives that page and all behind it up and gets free blocks instead;
 * what nobody holds any more is free from the next call on.
 *   served    device int32 [n]: 1, or 0 where blocks run out: from the first request on for
 *             which they do, none that needs one (or keeps a page that others
 *             would have had to leave) gets any, and it is left as it was
 *   grow      device int32 [n], at least 0 (less counts as 0)
 *   workspace device, 256-byte aligned, at least pk_kv_pages_workspace_bytes.
 *             ZERO-FILLED BEFORE ITS FIRST USE; every call leaves it ready for the
 *             next.  One workspace serves both calls and all pools for which it
 *             is large enough; the caller orders them.
 * A row must not name a block twice.  Errors: PK_EINVAL. */
size_t pk_kv_pages_workspace_bytes(int64_t num_blocks);
int pk_kv_pages_reserve(int32_t* block_table, const int32_t* lens, int32_t* pages, int32_t n, int32_t max_blocks,
                        const int32_t* grow, int32_t* refs, int64_t num_blocks, int32_t page_size,
                        int32_t* served, int32_t* copy_src, int32_t* copy_dst,
                        void* workspace, size_t workspace_bytes, void* stream);

/* pk_kv_pages_compact -- with U blocks in use, those of the numbers U and up move to
 * the free ones below U: the k-th of them to the k-th, both by rising number, for
 * k < max_moves (the rest by further calls).  copy_src[k] -> copy_dst[k] are
 * the moves, -1 behind the last one; no block is in both lists.
 *   new_table  block_table with the new numbers (entries behind a request's pages are not
 *              written); may be block_table itself
 *   new_refs   [num_blocks]; not refs itself
 *   copy_src, copy_dst  device int32 [max_moves]
 * workspace as for pk_kv_pages_reserve.  Errors: PK_EINVAL. */
int pk_kv_pages_compact(const int32_t* block_table, const int32_t* pages, int32_t n, int32_t max_blocks,
                        const int32_t* refs, int64_t num_blocks, int32_t* new_table, int32_t* new_refs,
                        int32_t* copy_src, int32_t* copy_dst, int32_t max_moves,
                        void* workspace, size_t workspace_bytes, void* stream);

/* pk_kv_cache_copy -- block copy_src[i] of `from` to block copy_dst[i] of `to`, keys,
 * values and scales, for i < count; pairs with a number that the cache does not
 * have (-1) are passed over.  `to` may be `from`, or another cache of its dtype, page
 * size and head shape (of another size, to move requests there) that does not
 * overlap it.  No block is written twice, or read and written, in one call.
 * Errors: PK_EINVAL; PK_EUNSUPPORTED. */
int pk_kv_cache_copy(const pk_cache* from, const pk_cache* to, const int32_t* copy_src, const int32_t* copy_dst,
                     int32_t count, void* stream);

/* pk_shared_tree_attn -- pk_tree_attn for a batch in which neighbouring requests have
 * their leading pages in common (as pk_kv_pages_select leaves forks): those keys are read
 * once for all of them.
 *   family_start  device int32 [families + 1], not decreasing: family g is
 *             requests family_start[g] .. family_start[g + 1] - 1; requests in
 *             none share nothing
 *   families  0 .. n; 0: every request is taken alone, in one or two launches instead of
 *             three, which is faster where the requests have less than 256 MB of keys and
 *             values or so (lengths are on the device: without this only the
 *             table's width tells)
 * How many pages a family shares is found from its rows of block_table: what all of
 * its requests with drafted tokens have in common (one that has less in common with the
 * others belongs into a family of its own).  The result is that of
 * pk_tree_attn whatever the families are, but for the order of the sums.  It
 * repeats bit for bit.
 *   workspace as for pk_tree_attn, of at least
 *             pk_shared_tree_attn_workspace_bytes; not to be shared with
 *             pk_tree_attn
 * Other arguments and errors as for pk_tree_attn. */
size_t pk_shared_tree_attn_workspace_bytes(int32_t n, int32_t max_q, int64_t total_q, int Hq, int Hkv, int d);
int pk_shared_tree_attn(const pk_cache* cache, const void* q, const int32_t* q_start, int64_t total_q, int32_t max_q,
                        const uint64_t* tree_mask, const int32_t* block_table, int32_t max_blocks,
                        const int32_t* kv_lens, int32_t n, const int32_t* family_start, int32_t families,
                        void* out, float scale, int Hq, int out_dtype,
                        void* workspace, size_t workspace_bytes, void* stream);

/* pk_draft_verify -- speculative sampling: which of the drafted tokens of every
 * request stay, so that they and the token behind them are distributed as if the target
 * had drawn them one by one.  Requests, their tokens and tree_mask are those of
 * pk_tree_attn; token 0 of a request is the one that the last step drew (it
 * stays), the parent of a token t > 0 is the highest token below t in its mask
 * word (a token without one cannot stay).
 *   target    device [total_q][vocab] (dtype PK_BF16 or PK_F32, rows target_stride elements
 *             apart): row t of a request are the logits of the token behind its
 *             token t; -inf: cannot be drawn; NaN counts as -inf, inf as the
 *             largest fp32 number.  Logarithms of probabilities are logits too.
 *   draft     logits of the same form from which the children of token t were
 *             drawn, independently of one another, at the request's temperature; NULL: the
 *             drafted tokens were not drawn (they were looked up, or are the
 *             likeliest)
 *   tokens    device int32 [total_q]; one outside of [0, vocab) does not stay
 *   temperature  device float [n]; NULL: 1.  0 and less (and NaN): the first of the
 *             largest logits has probability 1, and draft is not read
 *   accept_u, sample_u  device float [total_q], [n]: independent uniform random
 *             numbers from [0, 1), one for each drafted token, one for the
 *             token behind
 * P and Q are softmax(target / temperature) and softmax(draft / temperature) of
 * the last token that stays so far.  Its children are looked at by rising number.  With
 * c = 0 and Z = 1 at first, child x stays if P(x) > (c + u Z) Q(x); otherwise
 * c := c + Z, Z := sum of max(P - c Q, 0).  Without draft x stays if P(x) > u Z;
 * otherwise Z := Z - P(x), P(x) := 0.  The token behind the last one that stays
 * is the first x with cumulative weight over sample_u times the whole, of the
 * weights max(P - c Q, 0) (P where all of them are zero).
 * Probabilities and sums have 64 bits.
 *   keep      device int32 [n][max_keep]: the tokens that stay, rising (as
 *             pk_kv_cache_keep takes them), -1 behind the last one.  Of a branch of more than
 *             max_keep tokens the first max_keep stay (max_keep >= 1)
 *   keep_count, next_token  device int32 [n]: how many (0 and -1 for a request without
 *             tokens); the token behind, -1 where no logit of its row is a number
 *             above -inf
 *   workspace device, 256-byte aligned, at least pk_draft_verify_workspace_bytes.
 *             ZERO-FILLED BEFORE ITS FIRST USE; every call leaves it ready for the
 *             next.  The size does not fall with n, total_q or vocab: one
 *             workspace serves all calls of up to the sizes that it was made
 *             for; the caller orders them.
 * No output overlaps an input, the workspace or another output (what lies between
 * two rows of logits is none of them).
 * With one token a request it draws from its logits.  Errors: PK_EINVAL;
 * PK_EUNSUPPORTED (max_q). */
size_t pk_draft_verify_workspace_bytes(int32_t n, int64_t total_q, int32_t vocab);
int pk_draft_verify(const void* target, int64_t target_stride, const void* draft, int64_t draft_stride, int dtype,
                    int32_t vocab, const int32_t* tokens, const int32_t* q_start, int64_t total_q, int32_t max_q,
                    const uint64_t* tree_mask, int32_t n, const float* temperature,
                    const float* accept_u, const float* sample_u,
                    int32_t* keep, int32_t max_keep, int32_t* keep_count, int32_t* next_token,
                    void* workspace, size_t workspace_bytes, void* stream);

/* Message of the last error on this thread ("" if none). */
const char* pk_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* PACKINFER_H */
