/*
 * rest.h - C ABI of the GPU hot path of one REST decoding step
 * (Retrieval-Based Speculative Decoding, arXiv 2311.08252).
 *
 * Set-up:       rest_suffix_array_build (_full, _in_groups, _append), rest_datastore_create
 *               (Sec. 3.2, datastore construction)
 * Draft side:   rest_draft                                 (Sec. 3.2, Algorithms 1 and 2)
 *               rest_retrieve, rest_gather_rows, rest_draft_from_runs: the same in pieces, for a
 *               datastore spread over several GPUs
 * Verify side:  rest_tree_attention, rest_accept           (Sec. 3.2, draft verification / acceptance)
 *               rest_paged_attention: the same attention over a cache cut into pages
 *               rest_paged_attention_scaled: over pages of 8-bit codes with scales
 *               rest_accept_sampled: acceptance against the verifier's probabilities
 *               rest_rotary: queries or keys rotated by the position ids of a draft
 * Between steps: rest_kv_commit                            (the accepted path joins the prefix)
 *               rest_paged_kv_write, rest_paged_kv_commit, rest_pages_fork, rest_pages_copy,
 *               rest_pages_reserve, rest_pages_release: the cache in pages
 *               rest_paged_kv_append: a step's rows rotated and written in one call
 *               rest_paged_kv_append_scaled, rest_paged_kv_commit_scaled, rest_pages_copy_scaled:
 *               the same cache in 8-bit codes with scales
 * Health:       rest_device_error_flags
 * (measurement and planning aids live in rest_aids.h)
 *
 * Conventions
 *   - Every pointer named d_* is a DEVICE pointer owned by the caller.  The library borrows
 *     it for the duration of the call (the datastore handle: for its lifetime), never frees
 *     it and never allocates device memory.  Scratch space is passed in by the caller; its
 *     size comes from the matching *_workspace_bytes query.
 *   - `stream` is a cudaStream_t passed as void*.  Calls enqueue work on it and return
 *     without synchronising (rest_datastore_create with REST_DS_VALIDATE is the exception).
 *   - Host-checkable problems return a non-zero rest_status before anything is launched.
 *     Data-dependent problems are reported per context in d_status and give an empty tree.
 *     Nothing aborts, traps or throws.
 *   - All integer outputs are fully determined by the inputs (no dependence on scheduling).
 */
#ifndef REST_H_
#define REST_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef int32_t rest_status;
enum {
  REST_OK = 0,
  REST_INVALID_ARG = 1,         /* null pointer, negative size, inconsistent shapes          */
  REST_UNSUPPORTED = 2,         /* outside the limits listed at rest_draft / rest_tree_attention */
  REST_WORKSPACE_TOO_SMALL = 3,
  REST_CUDA_ERROR = 4,          /* a CUDA runtime call failed; see rest_last_cuda_error()    */
  REST_BAD_DATASTORE = 5        /* validation found an unsorted / non-permutation suffix array
                                   or a token outside [0, vocab)                              */
};

/* Per-context codes written to d_status by rest_draft. */
enum {
  REST_CTX_OK = 0,
  REST_CTX_BAD_TOKEN = 1,       /* one of the last n_max context tokens is outside [0, vocab) */
  REST_CTX_BAD_DATASTORE = 2,   /* suffix-array entry out of range, or gathered continuations
                                   not in lexicographic order                                 */
  REST_CTX_INTERNAL = 3,
  /* written by rest_pages_fork and rest_pages_reserve */
  REST_CTX_NO_PAGES = 4,        /* too few free pages for this context and those before it:
                                   nothing was done                                           */
  REST_CTX_BAD_PAGES = 5        /* index out of range, child in use or named twice, length that
                                   the table cannot hold: nothing was done                      */
};

enum { REST_SAMPLE_STRIDED = 0, REST_SAMPLE_FIRST_K = 1 };
/* How rest_draft searches the suffix array (rest_draft_params.search_path); the results are the
 * same either way.  SINGLE: every suffix length at once, a warp per length, 32 probes per round
 * inside the range that the datastore's n-gram index gives for the query's first tokens (fewest
 * dependent reads, the fastest single context); 512 or 1024 threads per context.  BATCHED: 256
 * threads per context, six or seven searches instead of fifteen (the lengths that match are
 * n_min ... n* without a gap) and eight probes per round once the probes leave L2: more
 * dependent rounds, fewer random DRAM reads, more contexts in flight (most of all with the
 * scratch that rest_draft_workspace_bytes asks for, see d_ws).  AUTO picks BATCHED when the call
 * has at least 5 contexts per SM and that scratch, or at least 16 contexts per SM without it. */
enum { REST_SEARCH_AUTO = 0, REST_SEARCH_SINGLE = 1, REST_SEARCH_BATCHED = 2 };
enum { REST_DS_VALIDATE = 1u, REST_DS_INDEX = 2u };

/* Element types of caches, queries and logits. */
enum { REST_BF16 = 0, REST_FP16 = 1, REST_FP32 = 2 };

/* Limits of this implementation. */
enum {
  REST_MAX_SUFFIX = 16,   /* n_max */
  REST_MAX_M = 16,        /* continuation length */
  REST_MAX_N = 256,       /* draft tokens per tree */
  REST_MAX_K = 32768,     /* candidates per context */
  REST_HEAD_DIM = 128,
  REST_MAX_PAGES = 1 << 20,           /* pages of a pool handed out by rest_pages_fork / _reserve */
  REST_MAX_FORKS = 1024,              /* forks per rest_pages_fork call */
  REST_MAX_PAGED_CONTEXTS = 8192,     /* contexts per rest_pages_reserve call */
  REST_MAX_VOCAB_SAMPLED = 1 << 18    /* logits per row of rest_accept_sampled */
};

typedef struct rest_datastore rest_datastore;   /* opaque host object holding device pointers */

/* Draft hyper-parameters (Sec. 4.1 "Hyperparameters": n_max = 16, m = 10, c = 64).
 *   n_max, n_min  longest / shortest context suffix tried by Algorithm 1 (1 <= n_min <= n_max <= 16)
 *   K             cap on the number of continuation candidates used per context (1..32768)
 *   m             continuation length (1..16)
 *   N             maximum number of draft tokens, the paper's c (1..256)
 *   sample_mode   which K of cnt > K matches are used: REST_SAMPLE_STRIDED takes suffix-array
 *                 slot lo + floor(j*cnt/K), REST_SAMPLE_FIRST_K takes lo + j, j = 0..K-1
 *   search_path   REST_SEARCH_AUTO / SINGLE / BATCHED: a performance switch, never a result */
typedef struct {
  int32_t n_max, n_min, K, m, N, sample_mode, search_path;
} rest_draft_params;

/*
 * Datastore (Sec. 3.2 "Datastore construction" and "Retrieving from the datastore": a token
 * stream whose every position is a (context, continuation) pair, indexed by a suffix array).
 *
 *   d_tokens   int32[n_tokens], values in [0, vocab), vocab < 2^31
 *   d_sa       int32[n_tokens] (sa_bytes = 4, n_tokens < 2^31) or int64[n_tokens] (sa_bytes = 8):
 *              start positions of all suffixes in lexicographic order of their tokens (compared
 *              as unsigned integers, a suffix that is a proper prefix of another sorts first).
 *              Only the order on the first n_max + m tokens matters to rest_draft.
 *   flags      REST_DS_VALIDATE: check on the device that d_sa is a permutation ordered on the
 *              first 32 tokens and that tokens are in range; synchronises `stream`; returns
 *              REST_BAD_DATASTORE on failure.
 *              REST_DS_INDEX: build a bucket index into d_aux (asynchronously on `stream`): for
 *              every token the suffix-array range of the suffixes that start with it, and a hash
 *              table with the ranges of the frequent sequences of two, three and four tokens
 *              (up to 512 MiB).  rest_draft then starts each search inside such a range instead
 *              of over the whole array, and a frequent suffix of up to four tokens needs no
 *              search at all: fewer dependent reads, identical results.  Needs vocab <= 2^22
 *              (ignored beyond).
 *   d_aux      device scratch of rest_datastore_aux_bytes() bytes, 256-byte aligned, needed with
 *              either flag (NULL otherwise).  With REST_DS_INDEX the handle keeps using it: it
 *              must stay allocated and untouched until rest_datastore_destroy.
 *   out        receives a host handle; free it with rest_datastore_destroy (device arrays stay
 *              the caller's).
 */
size_t rest_datastore_aux_bytes(uint64_t n_tokens, int32_t sa_bytes, uint32_t vocab);
rest_status rest_datastore_create(const int32_t* d_tokens, uint64_t n_tokens, const void* d_sa,
                                  int32_t sa_bytes, uint32_t vocab, uint32_t flags, void* d_aux,
                                  size_t aux_bytes, void* stream, rest_datastore** out);
void rest_datastore_destroy(rest_datastore* ds);

/*
 * rest_datastore_create_shard - a datastore whose suffix array lists only n_sa <= n_tokens of
 * the positions, e.g. one shard of a token stream that is spread over several GPUs (Sec. 5,
 * "Effect of the datastore size": the datastore may outgrow one device).  A shard holds the
 * tokens of its own position range followed by the first tokens of the next shard (at least
 * n_max + m of them), and its suffix array orders the positions of its own range only, so that
 * every occurrence in the whole stream is found by exactly one shard and its continuation is
 * complete.  Everything else as rest_datastore_create; d_sa has n_sa entries, all distinct
 * positions in [0, n_tokens), ordered like a suffix array.
 */
rest_status rest_datastore_create_shard(const int32_t* d_tokens, uint64_t n_tokens, const void* d_sa,
                                        uint64_t n_sa, int32_t sa_bytes, uint32_t vocab, uint32_t flags,
                                        void* d_aux, size_t aux_bytes, void* stream, rest_datastore** out);

/*
 * rest_draft - Algorithm 1 (longest-suffix exact-match retrieval), Algorithm 2 (Trie weights,
 * the c heaviest nodes) and the breadth-first pseudo sequence with its tree-attention mask
 * (Sec. 3.2 "Draft verification"), for B independent contexts.
 *
 * Per context b:
 *   1. n runs from min(n_max, ctx_len[b]) down to n_min; q = last n context tokens; [lo, hi) is
 *      the suffix-array range of suffixes starting with q; the first non-empty range wins.
 *      No match (or ctx_len < n_min): empty tree, match_n = 0.  That is not an error.
 *   2. Candidates: the min(hi-lo, K) sampled slots (see sample_mode); candidate j is the up to m
 *      tokens that follow the match, cut at the end of the token stream.
 *   3. Trie node = distinct non-empty prefix of a candidate; weight = number of candidates
 *      having that prefix.  Kept: the N largest by (weight desc, depth asc, token path asc).
 *   4. Output order: by depth, then token path (breadth first, siblings ascending by token).
 *
 *   d_ctx        int32, context b starts at d_ctx + b*ctx_stride and holds ctx_len[b] tokens
 *   d_tokens     int32[B,N]  draft tokens;           unused slots -1
 *   d_parents    int32[B,N]  index of the parent node, -1 for children of the root; unused -1
 *   d_depth      int32[B,N]  1-based depth;          unused 0
 *   d_pos_ids    int32[B,N]  ctx_len + depth - 1;    unused ctx_len
 *   d_mask       uint32[B,N,ceil(N/32)]  bit (j & 31) of word (j >> 5) of row i is set iff node
 *                j is node i or an ancestor of i; unused rows hold their own bit only
 *   d_n_nodes    int32[B]
 *   d_match_n    int32[B]    matched suffix length (0 = none)
 *   d_match_range int64[B,2] lo, hi of the matched suffix-array range
 *   d_node_count int32[B,N]  weight of each kept node (may be NULL)
 *   d_status     int32[B]    REST_CTX_* code
 *   d_ws         optional scratch of rest_draft_workspace_bytes() bytes, 16-byte aligned (the
 *                query answers for the current device and may be 0).  Never needed for the
 *                results, only for speed; with NULL or fewer bytes every path runs as one launch
 *                of one block per context.  What it buys:
 *                - single-context path, 2 to 1024 contexts (48 to 1024 when K < 8192; never when
 *                  K <= 512): a context with a long candidate list lets idle blocks (those of
 *                  finished or lighter contexts, and blocks started on SMs that have no context)
 *                  read part of its rows; the scratch holds the contexts' counters and
 *                  node-start bitmaps (about 6 m K / 32 bytes per context).  The call zeroes the
 *                  counters itself.
 *                - batched path: three launches (search; build of the contexts with few
 *                  candidates on small blocks; build of the others on large blocks); the scratch
 *                  holds the two context lists (8 bytes per context).
 *                The scratch must not be shared by calls that may run at the same time.
 */
size_t rest_draft_workspace_bytes(const rest_draft_params* params, int32_t B);
rest_status rest_draft(const rest_datastore* ds, const rest_draft_params* params,
                       const int32_t* d_ctx, int64_t ctx_stride, const int32_t* d_ctx_len,
                       int32_t B, int32_t* d_tokens, int32_t* d_parents, int32_t* d_depth,
                       int32_t* d_pos_ids, uint32_t* d_mask, int32_t* d_n_nodes,
                       int32_t* d_match_n, int64_t* d_match_range, int32_t* d_node_count,
                       int32_t* d_status, void* d_ws, size_t ws_bytes, void* stream);

/*
 * The draft in pieces, for a datastore spread over several GPUs (Algorithms 1 and 2 over the
 * union of the shards; Sec. 5 "Effect of the datastore size").  Per decoding step:
 *   1. every GPU:  rest_retrieve on its shard -> its longest matching suffix length and range;
 *   2. exchange:   the winning length n* is the maximum over the shards (a shorter suffix of a
 *                  match is a match, so a shard either matches n* or contributes nothing);
 *                  shards that match n* report their hit counts cnt_i; with cnt = sum cnt_i,
 *                  shard i contributes all its rows when cnt <= K, else
 *                  floor(K C_i / cnt) - floor(K C_(i-1) / cnt) rows (C_i = cnt_1 + ... + cnt_i),
 *                  spread over its range like rest_draft spreads K over one range.  With one
 *                  shard this is exactly rest_draft's rule;
 *   3. every GPU:  rest_gather_rows -> its rows, in lexicographic order (one sorted run);
 *   4. exchange:   the runs of all shards travel to the GPU that builds the tree;
 *   5. builder:    rest_draft_from_runs merges the runs and runs Algorithm 2 and the tree
 *                  emission unchanged.
 * The exchanges are ordinary collectives on small tensors and belong to the caller (the Python
 * package does them with torch.distributed).
 *
 * rest_retrieve       Algorithm 1 alone: d_match_n[b], d_match_range[b] = {lo, hi}, d_status[b];
 *                     arguments as in rest_draft (K, m, N, sample_mode of `params` are not used).
 * rest_gather_rows    candidate j < take[b] of context b: the suffix-array slot
 *                     lo + floor(j cnt / take[b]) (lo + j with REST_SAMPLE_FIRST_K or when
 *                     take[b] = cnt), its up to m tokens after the match into d_rows[b][j][0..m)
 *                     (zero padded) and their number into d_row_len[b][j]; rows j >= take[b] get
 *                     length 0.  d_match_n / d_match_range as written by rest_retrieve (a shard
 *                     that lost sets take[b] = 0).  Kr = row capacity per context (<= 32768).
 *                     d_status[b] is OR-ed with REST_CTX_BAD_DATASTORE on an entry out of range.
 * rest_draft_from_runs  d_rows int32[B][R][Kr][m], d_row_len int32[B][R][Kr], d_run_rows
 *                     int32[B][R] (rows of run r in use; each run in lexicographic order, a row
 *                     that is a prefix of another first; R * Kr <= 32768).  Outputs as rest_draft
 *                     (d_node_count may be NULL); runs out of order give status
 *                     REST_CTX_BAD_DATASTORE and an empty tree.  d_ws: scratch of
 *                     rest_draft_from_runs_workspace_bytes(B, R, Kr) bytes.
 */
rest_status rest_retrieve(const rest_datastore* ds, const rest_draft_params* params,
                          const int32_t* d_ctx, int64_t ctx_stride, const int32_t* d_ctx_len,
                          int32_t B, int32_t* d_match_n, int64_t* d_match_range, int32_t* d_status,
                          void* stream);
rest_status rest_gather_rows(const rest_datastore* ds, const rest_draft_params* params,
                             const int32_t* d_match_n, const int64_t* d_match_range,
                             const int32_t* d_take, int32_t B, int32_t Kr, int32_t* d_rows,
                             int32_t* d_row_len, int32_t* d_status, void* stream);
size_t rest_draft_from_runs_workspace_bytes(int32_t B, int32_t R, int32_t Kr);
rest_status rest_draft_from_runs(const rest_draft_params* params, const int32_t* d_rows,
                                 const int32_t* d_row_len, const int32_t* d_run_rows, int32_t R,
                                 int32_t Kr, const int32_t* d_ctx_len, int32_t B, int32_t* d_tokens,
                                 int32_t* d_parents, int32_t* d_depth, int32_t* d_pos_ids,
                                 uint32_t* d_mask, int32_t* d_n_nodes, int32_t* d_node_count,
                                 int32_t* d_status, void* d_ws, size_t ws_bytes, void* stream);

/*
 * rest_tree_attention - attention of the N draft positions of each context over the prefix
 * KV cache and over their own ancestors (Sec. 3.2 "Draft verification": the pseudo sequence
 * is run with an attention mask under which every token sees exactly its dependencies).
 *
 *   For context b, head h, node i:  keys = {0..L-1} U {L+j : bit j of mask row i}, L = kv_len[b];
 *   out = softmax(scale * q.k) v  with natural exponent, fp32 accumulation, bf16 output.
 *
 *   d_q       bf16, element (b,i,h,d) at b*strides[0] + i*strides[1] + h*strides[2] + d
 *   d_k, d_v  bf16, element (b,hk,l,d) at b*strides[3] + hk*strides[4] + l*strides[5] + d;
 *             rows L..L+N-1 hold the K/V of the draft nodes; hk = h / (H / H_kv)
 *   d_out     bf16, element (b,i,h,d) at b*strides[6] + i*strides[7] + h*strides[8] + d
 *   strides   host array of 9 element strides; rows of D elements are contiguous and every
 *             stride is a multiple of 8 elements (16-byte rows); base pointers 16-byte aligned
 *   d_kv_len  int32[B], 0 <= L and L + N <= rows available
 *   max_kv    upper bound on L + N over the batch (sizes the split of the key range)
 *   d_mask    uint32[B,N,ceil(N/32)] as written by rest_draft
 *   d_lse     optional float[B,H,N]: log of the softmax denominator (natural log, of scaled
 *             scores); with N > 64 the denominator sums the bf16-rounded probabilities that the
 *             output is built from, so it carries bf16 precision (a few 1e-3 absolute)
 *   d_ws      scratch of rest_tree_attention_workspace_bytes() bytes
 *   scale     softmax scale, finite and > 0 (else REST_INVALID_ARG)
 *   Limits: D = 128; 1 <= N <= 256 (any tree rest_draft can write); H % H_kv == 0.
 */
size_t rest_tree_attention_workspace_bytes(int32_t B, int32_t H, int32_t N, int32_t D,
                                           int32_t max_kv);
rest_status rest_tree_attention(const void* d_q, const void* d_k, const void* d_v,
                                const int64_t* strides, const int32_t* d_kv_len,
                                const uint32_t* d_mask, int32_t B, int32_t H, int32_t H_kv,
                                int32_t N, int32_t D, int32_t max_kv, float scale, void* d_out,
                                float* d_lse, void* d_ws, size_t ws_bytes, void* stream);

/*
 * rest_tree_attention_static_scratch - rest_tree_attention for callers that cannot allocate.
 *
 * (The paper has no counterpart; this is a packaging variant of the call above.)
 *
 * Some users of this library cannot obtain the workspace that rest_tree_attention asks for:
 * a serving process that handed every free byte of device memory to its own KV-cache pool at
 * start-up, or a decode loop whose rules forbid allocation calls because cudaMalloc/cudaFree
 * may stall the whole device.  For them the split-KV partials live in a fixed array of
 * REST_STATIC_SCRATCH_BYTES (768 KiB) inside the library image.  Every GPU that loads the
 * library holds that array until the process exits, whether or not this call is used.
 *
 *   - Arguments, layouts, results and limits are those of rest_tree_attention, without
 *     d_ws / ws_bytes.  The call itself performs no device or host allocation.
 *   - Returns REST_WORKSPACE_TOO_SMALL, launching nothing, when
 *     rest_tree_attention_workspace_bytes(B, H, N, D, max_kv) exceeds REST_STATIC_SCRATCH_BYTES.
 *     Scratch is only needed when one (context, head) pair is cut into more than 8 key ranges,
 *     i.e. for very few pairs with long caches, and then holds one partial of N x 130 floats per
 *     cluster of 8 ranges; no more clusters are used than the GPU can run at once (about 30).
 *     B*H = 2, N = 64, max_kv = 4160 needs 0.51 MiB and fits; B*H = 1, N = 64, max_kv = 16448
 *     needs about 1 MiB and is refused.
 *   - The first call on each device looks up the array's device address (one runtime query,
 *     with that device current).  Make that first call outside any stream capture.
 *   - All calls on a device share the one array, and it keeps whatever the previous call left.
 *     That is harmless here: each call writes every partial it later reads, so nothing has to
 *     start at zero.  But two calls whose kernels may overlap on the GPU (different streams)
 *     race on the array: serialise them.
 */
enum { REST_STATIC_SCRATCH_BYTES = 768 * 1024 };
rest_status rest_tree_attention_static_scratch(
    const void* d_q, const void* d_k, const void* d_v, const int64_t* strides,
    const int32_t* d_kv_len, const uint32_t* d_mask, int32_t B, int32_t H, int32_t H_kv, int32_t N,
    int32_t D, int32_t max_kv, float scale, void* d_out, float* d_lse, void* stream);

/*
 * rest_accept - draft acceptance (Sec. 3.2 "Draft acceptance": draft tokens are accepted from
 * the start while they coincide with the tokens sampled from the verifier; everything after
 * the first mismatch is rejected).
 *
 *   d_verifier_tokens int32[B,N+1]: slot 0 = verifier's token after the prefix, slot i+1 = its
 *                     token after draft node i (greedy argmax or a sampled token).
 *   Walk from the root: if the current node has a child whose token equals the verifier's token
 *   at the current node, accept it and continue from that child; stop otherwise or after
 *   max_depth accepted nodes.
 *   d_accept_len   int32[B]
 *   d_accept_nodes int32[B,max_depth]    accepted node indices, unused -1
 *   d_out_tokens   int32[B,max_depth+1]  accepted tokens followed by the verifier's token at the
 *                  stopping node (what plain decoding would emit next); unused -1
 */
rest_status rest_accept(const int32_t* d_tokens, const int32_t* d_parents,
                        const int32_t* d_n_nodes, const int32_t* d_verifier_tokens, int32_t B,
                        int32_t N, int32_t max_depth, int32_t* d_accept_len,
                        int32_t* d_accept_nodes, int32_t* d_out_tokens, void* stream);

/*
 * rest_kv_commit - make the accepted draft path part of the prefix KV cache.
 *
 * The paper does not describe the cache; any implementation of its loop (Sec. 3.2: draft,
 * verify, accept, repeat with the longer context) has to do this between two steps.  For
 * context b with L = kv_len[b] and len = accept_len[b]: K/V row L + accept_nodes[b][i] of every
 * kv head is copied to row L + i, i = 0..len-1, in place (accept_nodes[b][i] >= i always holds
 * for trees written by rest_draft, and the kernel reads all source rows before it writes).
 *
 *   d_k, d_v        bf16, element (b,hk,l,d) at b*kv_strides[0] + hk*kv_strides[1] + l*kv_strides[2] + d,
 *                   same layout rules as rest_tree_attention (D = 128, 16-byte aligned rows)
 *   d_accept_nodes  int32[B,max_depth], d_accept_len int32[B]: as written by rest_accept
 *   N               number of tree slots (node indices are clamped to [0, N))
 *   d_new_kv_len    optional int32[B]: receives L + len (may alias d_kv_len)
 *   Limits: max_depth <= 16.  The token the verifier produced at the stop (out_tokens[len]) has
 *   no K/V yet: it is the next step's first input token.
 */
rest_status rest_kv_commit(void* d_k, void* d_v, const int64_t* kv_strides, const int32_t* d_kv_len,
                           const int32_t* d_accept_nodes, const int32_t* d_accept_len, int32_t B,
                           int32_t H_kv, int32_t N, int32_t D, int32_t max_depth,
                           int32_t* d_new_kv_len, void* stream);

/*
 * A KV cache in pages.  The paper does not describe the cache; a server that keeps many contexts
 * of unforeseen lengths cuts it into pages.  Row l of context b is row l % page of page
 * d_table[b * table_stride + l / page]; an entry outside [0, P) means that there is none.
 *
 *   d_k_pages, d_v_pages  16-bit elements, element (p,hk,r,d) at p*page_strides[0] +
 *                   hk*page_strides[1] + r*page_strides[2] + d; strides are host values, multiples
 *                   of 8 elements; base pointers 16-byte aligned; D = 64 or 128
 *   P, page         pages in the pool, rows per page: 16, 32, 64, 128 or 256
 *   d_table         int32, row b at d_table + b*table_stride, table_cols entries
 *   d_refs          int32[P]: how many contexts hold each page.  A page is free iff its count is
 *                   0; free pages are handed out lowest number first, to contexts in order
 *   d_n_pages       int32[B]: table entries of each context in use
 * Tables are shared by all layers of a model; the row and page copies are made per layer.
 * Rows from kv_len on are written wherever the table says: after rest_pages_fork those pages are the
 * context's own, and they stay so as long as its length does not shrink into a shared page.
 *
 * rest_paged_kv_write   rows i < n_nodes[b] (i < N with d_n_nodes NULL) of d_k_new, d_v_new
 *                   (element (b,i,hk,d) at b*new_strides[0] + i*new_strides[1] + hk*new_strides[2]
 *                   + d) become rows kv_len[b] + i.  A row whose page does not exist is left out.
 * rest_paged_kv_commit  rest_kv_commit over pages: row kv_len[b] + accept_nodes[b][i] is copied to
 *                   row kv_len[b] + i, i < accept_len[b]; d_new_kv_len (may be NULL, may be
 *                   d_kv_len) receives kv_len + accept_len.  max_depth <= 16.
 * rest_pages_fork   child context children[f] becomes a copy of parents[f], f < F <= 1024: whole
 *                   pages of the parent's kv_len rows are shared (their counts rise), a partly
 *                   filled last page gets a page of its own, named in d_copy_src[f] / d_copy_dst[f]
 *                   (-1: nothing to copy) for rest_pages_copy.  The child must hold no pages
 *                   (n_pages = 0); n_pages, kv_len and its table row are written.  d_status[f]:
 *                   REST_CTX_*.  A child named twice is forked for its first mention only.  All
 *                   parents count as they were before the call.
 * rest_pages_copy   page d_dst[i] of K and V becomes a copy of page d_src[i]; pairs with an index
 *                   outside [0, P) are left out.  No page may be a target twice, or a target and
 *                   a source.
 * rest_pages_reserve  context b gets pages until its table holds need_len[b] rows, all of them or
 *                   none (d_status[b]).  Pages are counted out in the contexts' order, those of a
 *                   refused context too: once the pool is too small for one context, it and every
 *                   later one that needs a page get REST_CTX_NO_PAGES, whatever is free.  Ask again
 *                   without it (need_len[b] = 0) to serve the others.
 * rest_pages_release  context b keeps the pages of its first keep_len[b] rows; with window > 0 also
 *                   the pages whose rows all lie behind the window of every later token (rows
 *                   >= sinks and <= keep_len - window) go.  Their table entries become -1.
 *                   keep_len[b] < 0: the context stays as it is.
 */
rest_status rest_paged_kv_write(void* d_k_pages, void* d_v_pages, const int64_t* page_strides, int32_t P,
                                int32_t page, const int32_t* d_table, int64_t table_stride,
                                int32_t table_cols, const int32_t* d_kv_len, const void* d_k_new,
                                const void* d_v_new, const int64_t* new_strides,
                                const int32_t* d_n_nodes, int32_t B, int32_t H_kv, int32_t N, int32_t D,
                                void* stream);
rest_status rest_paged_kv_commit(void* d_k_pages, void* d_v_pages, const int64_t* page_strides, int32_t P,
                                 int32_t page, const int32_t* d_table, int64_t table_stride,
                                 int32_t table_cols, const int32_t* d_kv_len,
                                 const int32_t* d_accept_nodes, const int32_t* d_accept_len, int32_t B,
                                 int32_t H_kv, int32_t N, int32_t D, int32_t max_depth,
                                 int32_t* d_new_kv_len, void* stream);
rest_status rest_pages_fork(int32_t* d_refs, int32_t P, int32_t* d_table, int64_t table_stride,
                            int32_t table_cols, int32_t* d_n_pages, int32_t* d_kv_len, int32_t B,
                            int32_t page, const int32_t* d_parents, const int32_t* d_children, int32_t F,
                            int32_t* d_copy_src, int32_t* d_copy_dst, int32_t* d_status, void* stream);
rest_status rest_pages_copy(void* d_k_pages, void* d_v_pages, const int64_t* page_strides, int32_t P,
                            int32_t page, int32_t H_kv, int32_t D, const int32_t* d_src,
                            const int32_t* d_dst, int32_t n, void* stream);
rest_status rest_pages_reserve(int32_t* d_refs, int32_t P, int32_t* d_table, int64_t table_stride,
                               int32_t table_cols, int32_t* d_n_pages, const int32_t* d_need_len,
                               int32_t B, int32_t page, int32_t* d_status, void* stream);
rest_status rest_pages_release(int32_t* d_refs, int32_t P, int32_t* d_table, int64_t table_stride,
                               int32_t table_cols, int32_t* d_n_pages, const int32_t* d_keep_len,
                               int32_t B, int32_t page, int32_t window, int32_t sinks, void* stream);

/*
 * rest_rotary - rotary positions: each pair of elements of a row turns by an angle that grows with the
 * row's position (the paper takes the verifier as given; the positions are rest_draft's pos_ids).
 *
 *   For context b, node i, head h and pair f < pairs, with p = d_pos[b,i] and t = p * d_inv_freq[f]:
 *   (y1, y2) = amplitude * (x1 cos t - x2 sin t, x2 cos t + x1 sin t).  interleaved = 0: the pair is
 *   elements f and pairs + f; 1: elements 2f and 2f + 1.  Elements from 2 * pairs on are copied.
 *   t is a product in 64 bits, and whole quarter turns are taken off it there; sine and cosine of the
 *   rest and y are computed in 32 bits (for |t| < 2^40 below 2^-22 amplitude (|x1| + |x2|) off), rounded once.
 *   With -d_inv_freq it is the inverse rotation (and, amplitude kept, the gradient of x).
 *
 *   d_x, d_out      element (b,i,h,d) at b*strides[0] + i*strides[1] + h*strides[2] + d, dtype REST_BF16,
 *                   REST_FP16 or REST_FP32; strides host values, multiples of 16 bytes; base pointers
 *                   16-byte aligned.  d_out is d_x with the same strides (in place), or overlaps no input
 *   d_pos           int32[B,N], any sign; d_inv_freq float[pairs] (both may be NULL with pairs = 0: a copy)
 *   d_n_nodes       optional int32[B]: rows i >= n_nodes[b] of d_out stay as they were
 *   Limits: D a multiple of 16, at most 512; 2 * pairs <= D; amplitude finite; H <= 65536; N <= 2^30.
 */
rest_status rest_rotary(const void* d_x, const int64_t* x_strides, int32_t dtype, const int32_t* d_pos,
                        const float* d_inv_freq, int32_t pairs, int32_t interleaved, float amplitude,
                        const int32_t* d_n_nodes, int32_t B, int32_t H, int32_t N, int32_t D, void* d_out,
                        const int64_t* out_strides, void* stream);

/*
 * rest_paged_kv_append - rest_paged_kv_write with the rotation of rest_rotary on the way: rows i < n_nodes[b]
 * of d_k_new, rotated, and of d_v_new, as they are, become rows kv_len[b] + i; with H > 0 the queries d_q
 * are rotated into d_q_out (all three in one launch).  pairs = 0: nothing is rotated.
 *   d_k_pages ... d_n_nodes  as in rest_paged_kv_write (16-bit pages of `dtype`, REST_BF16 or REST_FP16, which
 *                   d_k_new, d_v_new, d_q and d_q_out share)
 *   d_pos ... amplitude      as in rest_rotary
 *   d_q, d_q_out    element (b,i,h,d) as in rest_rotary, h < H (H = 0: none, both NULL)
 *   A row whose page does not exist is left out; its query is rotated all the same.  Limits: H and H_kv <= 65536,
 *   N <= 2^30.
 */
rest_status rest_paged_kv_append(void* d_k_pages, void* d_v_pages, const int64_t* page_strides, int32_t P,
                                 int32_t page, const int32_t* d_table, int64_t table_stride, int32_t table_cols,
                                 const int32_t* d_kv_len, const void* d_k_new, const void* d_v_new,
                                 const int64_t* new_strides, const int32_t* d_n_nodes, int32_t dtype,
                                 const int32_t* d_pos, const float* d_inv_freq, int32_t pairs, int32_t interleaved,
                                 float amplitude, const void* d_q, const int64_t* q_strides, void* d_q_out,
                                 const int64_t* out_strides, int32_t H, int32_t B, int32_t H_kv, int32_t N,
                                 int32_t D, void* stream);

/*
 * The cache in 8 bits: pages of e4m3 codes (1 byte an element; strides in elements, multiples of 16), and for
 * each page, head and block of 16 rows a scale, float[P][H_kv][page / 16], for K and for V.  Row r of a
 * page stands for scale[r / 16] * code.  Scales are positive; outside [2^-60, 2^60] they count as the nearer
 * limit (NaN as 2^-60).  Tables, counts, forks and lengths are those of 16-bit pages.
 *
 * rest_paged_kv_append_scaled  as rest_paged_kv_append (queries of many rows in a second launch); K (rotated in 64
 *                   bits, then rounded to 32) and V are rounded to codes.  A block that gets new rows gets the
 *                   smallest power of two s for which no finite new value exceeds 448 s; where it has older rows
 *                   (below kv_len) s is not less than its scale was, and if it grows, those rows' codes are rounded
 *                   to the new scale (exact down to 2^-9 s).  A scale that a row has raised stays when the row is
 *                   refused: older rows of its block are then off by up to 2^-4 of an element and 2^-9 s, however
 *                   often it grew.  Under an older scale that is no power of two codes may be one step off.
 *                   Rows behind the new ones lose what they held.  Values that are not finite become NaN;
 *                   beyond 448 * 2^60 they saturate.
 * rest_paged_kv_commit_scaled  as rest_paged_kv_commit: the accepted rows are put to the front as if the
 *                   values that they stand for had been appended there, by the same rule.  A row whose source or
 *                   target page does not exist is not moved and has no part in a scale; what its place held
 *                   is lost where the block's scale changes.
 * rest_pages_copy_scaled  as rest_pages_copy, with the pages' scales.
 */
rest_status rest_paged_kv_append_scaled(void* d_k_pages, void* d_v_pages, const int64_t* page_strides,
                                        float* d_k_scales, float* d_v_scales, int32_t P, int32_t page,
                                        const int32_t* d_table, int64_t table_stride, int32_t table_cols,
                                        const int32_t* d_kv_len, const void* d_k_new, const void* d_v_new,
                                        const int64_t* new_strides, const int32_t* d_n_nodes, int32_t dtype,
                                        const int32_t* d_pos, const float* d_inv_freq, int32_t pairs,
                                        int32_t interleaved, float amplitude, const void* d_q,
                                        const int64_t* q_strides, void* d_q_out, const int64_t* out_strides,
                                        int32_t H, int32_t B, int32_t H_kv, int32_t N, int32_t D, void* stream);
rest_status rest_paged_kv_commit_scaled(void* d_k_pages, void* d_v_pages, const int64_t* page_strides,
                                        float* d_k_scales, float* d_v_scales, int32_t P, int32_t page,
                                        const int32_t* d_table, int64_t table_stride, int32_t table_cols,
                                        const int32_t* d_kv_len, const int32_t* d_accept_nodes,
                                        const int32_t* d_accept_len, int32_t B, int32_t H_kv, int32_t N, int32_t D,
                                        int32_t max_depth, int32_t* d_new_kv_len, void* stream);
rest_status rest_pages_copy_scaled(void* d_k_pages, void* d_v_pages, const int64_t* page_strides, float* d_k_scales,
                                   float* d_v_scales, int32_t P, int32_t page, int32_t H_kv, int32_t D,
                                   const int32_t* d_src, const int32_t* d_dst, int32_t n, void* stream);

/*
 * rest_paged_attention - attention of N new positions of each context over its KV cache in pages
 * (the layout described above) and over one another.  The paper's tree attention (Sec. 3.2 "Draft
 * verification"), for a cache in pages, other head sizes and types, and models with a sliding
 * window; with N = 1 an ordinary decoding step.
 *
 *   For context b, node i, head h (KV head h / (H / H_kv)), L = kv_len[b], n = n_nodes[b]:
 *   keys: prefix rows l < L, and rows L + j of the nodes j < n that bit j of mask row i names.
 *   Node i stands at position L + depth - 1, depth = bits below N set in its mask row (itself and
 *   its ancestors; bits of nodes that do not exist count too), or 1 where none is.  window > 0: of these, a key at position p is seen by a node at position x only if
 *   p < sinks or p > x - window (prefix row l stands at position l).
 *   out = softmax(scale * q.k) v in fp32, rounded once; a node that sees nothing gets 0 and an lse
 *   of -infinity.  Keys that a node does not see never touch its result, whatever they hold
 *   (infinities and NaN included).  An infinity or NaN in v of a key that it does see decides that
 *   column of out however small the key's probability is; NaN among its scores makes the row NaN.
 *
 *   d_q, d_out      element (b,i,h,d) at b*strides[0] + i*strides[1] + h*strides[2] + d (d_out: 6..8)
 *                   (d_out overlaps no input)
 *   d_k_pages, d_v_pages  page p, KV head, row, d: strides[3..5]; strides are multiples of 8
 *                   elements, base pointers 16-byte aligned; dtype REST_BF16 or REST_FP16 for all four
 *   d_table         a page index outside [0, P) reads as rows of zeros: rows in sight need pages
 *   d_n_nodes       optional int32[B]: nodes n_nodes[b] .. N-1 do not exist; their rows of d_out and
 *                   d_lse stay as they were
 *   d_mask          uint32[B,N,ceil(N/32)] as written by rest_draft, or NULL: node i sees nodes 0..i
 *                   and stands at position L + i (a run of tokens)
 *   d_lse           optional float[B,H,N]: log of the softmax denominator (natural log)
 *   d_ws            scratch of rest_paged_attention_workspace_bytes() bytes, 16-byte aligned (the
 *                   query answers for the current device).  Calls that may run at the same time,
 *                   captured graphs among them, need scratch of their own.
 *   Limits: D = 64 or 128; 1 <= N <= 256; H % H_kv == 0, H / H_kv <= 1024, H <= 65536.
 */
size_t rest_paged_attention_workspace_bytes(int32_t B, int32_t H, int32_t H_kv, int32_t N, int32_t D);
rest_status rest_paged_attention(const void* d_q, const void* d_k_pages, const void* d_v_pages,
                                 const int64_t* strides, int32_t dtype, int32_t P, int32_t page,
                                 const int32_t* d_table, int64_t table_stride, int32_t table_cols,
                                 const int32_t* d_kv_len, const int32_t* d_n_nodes,
                                 const uint32_t* d_mask, int32_t B, int32_t H, int32_t H_kv, int32_t N,
                                 int32_t D, int32_t window, int32_t sinks, float scale, void* d_out,
                                 float* d_lse, void* d_ws, size_t ws_bytes, void* stream);

/*
 * rest_paged_attention_scaled - rest_paged_attention over pages of codes with scales (see the cache in 8 bits, above).
 *   The same formula with the values that the codes stand for: scores, maxima, sums and the output
 *   in fp32; probabilities rounded to fp16 for their product with V (half a step, 2^-11 of each; below 2^-31 of
 *   the row's largest p * scale of v they vanish there, and below 2^-130 of it in the sum).  With more than 16 rows a KV head (N * H / H_kv) queries are held as sums of
 *   e4m3 terms, off by at most 2^-11 of an element in fp16 or 2^-8 in bf16 where it is far below its row's largest,
 *   and never by more than 2^-19 of that or 2^-70.  bf16 queries beyond 2^60 saturate or make their row NaN there, and
 *   scale times a scale of K counts as within [2^-89, 2^66].
 *   d_q, d_out      dtype REST_BF16 or REST_FP16; strides as there, those of the pages (3..5) multiples of 16
 *   d_k_scales, d_v_scales  float[P][H_kv][page / 16], aligned to min(page, 64) / 4 bytes
 *   d_ws            scratch of rest_paged_attention_workspace_bytes() bytes
 *   Everything else as in rest_paged_attention (codes have no infinities; NaN codes are NaN there).
 *   Which is quicker goes by the rows of a KV head, N * H / H_kv: up to 16 this call, which takes 0.5 to 0.75 times as
 *   long on long caches; from 17 on rest_paged_attention, and what codes save is memory (this call 1.0 to 1.3 times as long).
 */
rest_status rest_paged_attention_scaled(const void* d_q, const void* d_k_pages, const void* d_v_pages,
                                        const int64_t* strides, const float* d_k_scales, const float* d_v_scales,
                                        int32_t dtype, int32_t P, int32_t page, const int32_t* d_table,
                                        int64_t table_stride, int32_t table_cols, const int32_t* d_kv_len,
                                        const int32_t* d_n_nodes, const uint32_t* d_mask, int32_t B, int32_t H,
                                        int32_t H_kv, int32_t N, int32_t D, int32_t window, int32_t sinks, float scale,
                                        void* d_out, float* d_lse, void* d_ws, size_t ws_bytes, void* stream);

/*
 * rest_accept_sampled - draft acceptance against the verifier's probabilities (Sec. 4.1 "Sampling
 * strategies": temperature and nucleus sampling), from random numbers that the caller supplies.
 * The tokens that come out are distributed exactly as plain sampling would distribute them.
 *
 *   Row s of context b (slot 0: after the prefix, slot i+1: after draft node i, as in
 *   rest_accept) has weights w_v = exp((logit_v - largest) / temperature[b]), cut to the nucleus:
 *   in the order (logit descending, token ascending) the shortest run whose weights sum to at least
 *   top_p[b] of the whole.  Walk from the root.  At a node, r = sum of the weights; its children
 *   are tried in index order: child c is accepted when uniforms[b][c+1] * r < w(token of c), else
 *   its token leaves the row (w = 0) and r drops by its weight.  When no child is accepted (or
 *   max_depth nodes are), the last token is drawn from what the row still holds: the first v with
 *   w_0 + ... + w_v > uniforms[b][0] * r.  (Drafts from retrieval are given, not drawn, so the
 *   proposal is certain and this is speculative sampling's rejection rule for it.)
 *
 *   d_logits        element (b,s,v) at b*ctx_stride + s*row_stride + v, dtype REST_BF16, REST_FP16
 *                   or REST_FP32; NaN counts as -infinity (never drawn)
 *   d_tokens, d_parents int32[B,N], d_n_nodes int32[B]: the tree, as written by rest_draft
 *   d_uniforms      float[B,N+1], in [0, 1)
 *   d_temperature, d_top_p  float[B]; temperature 0: the largest logit, lowest token first (then
 *                   the call equals rest_accept on the rows' argmax), above 1e30: 1e30; top_p >= 1:
 *                   no cut
 *   outputs         as rest_accept; a row without a finite logit gives -1 for the last token
 *   Weights are whole numbers of 2^-44 of the row's largest, rounded to 24 bits (each is off by at most
 *   2^-24 of itself; sums are exact in any order: results never depend on scheduling).  A token below
 *   2^-45 of the largest counts as impossible.  The nucleus goes by the logits where weights are a
 *   rounding apart.
 *   d_ws            optional scratch of rest_accept_sampled_workspace_bytes() bytes, 8-byte aligned
 *                   (the query answers for the current device and may be 0), not shared by calls
 *                   that may run at the same time.  Only for speed: with it the rows of few
 *                   contexts are all worked on at once, without it each context walks row by row.
 *   Limits: V <= 2^18, max_depth <= 16, N <= 256.
 */
size_t rest_accept_sampled_workspace_bytes(int32_t B, int32_t N);
rest_status rest_accept_sampled(const void* d_logits, int32_t dtype, int64_t ctx_stride,
                                int64_t row_stride, int32_t V, const int32_t* d_tokens,
                                const int32_t* d_parents, const int32_t* d_n_nodes,
                                const float* d_uniforms, const float* d_temperature,
                                const float* d_top_p, int32_t B, int32_t N, int32_t max_depth,
                                int32_t* d_accept_len, int32_t* d_accept_nodes, int32_t* d_out_tokens,
                                void* d_ws, size_t ws_bytes, void* stream);

/*
 * rest_suffix_array_build - the datastore's suffix array, built on the device (Sec. 3.2
 * "Datastore construction"; "Retrieving from the datastore" matches through a suffix array).
 * Set-up work: call it once, then rest_datastore_create on the result.
 *
 *   Order: suffixes compare on their first 32 tokens (unsigned, a suffix that ends early is
 *   smaller); suffixes equal on those are ordered by position.  rest_draft reads at most
 *   n_max + m <= 32 tokens of a suffix, so its results are those of the full order.
 *
 *   d_tokens  int32[n_tokens] device, values in [0, 2^31 - 1)
 *   sa_bytes  4 or 8: d_sa is int32[n_tokens] (n_tokens < 2^31) or int64[n_tokens] (device, written)
 *   d_ws      device scratch, 256-byte aligned.  Two methods, picked by what fits:
 *             - up to 2^31 - 1 tokens and at least rest_suffix_array_workspace_bytes(n_tokens)
 *               (about 32 bytes per token + 64 MiB): prefix doubling, five sorts of the whole
 *               stream, asynchronous on `stream`;
 *             - otherwise (longer streams, or a smaller workspace): positions are put into
 *               buckets by first token and groups of whole buckets are sorted one after the
 *               other on their packed 32-token keys.  Scratch: 32 bytes per position of the
 *               largest group + 0.2 GiB; rest_suffix_array_workspace_bytes answers for groups of
 *               2^30 positions, rest_suffix_array_min_workspace_bytes for groups just large
 *               enough for the most frequent first token.  This method reads the bucket
 *               histogram back (it synchronises `stream`) and returns REST_UNSUPPORTED when one
 *               first token starts more suffixes than the workspace can sort at once.
 *   Limits: n_tokens <= 2^40.
 */
size_t rest_suffix_array_workspace_bytes(uint64_t n_tokens);
size_t rest_suffix_array_min_workspace_bytes(uint64_t n_tokens, uint64_t largest_bucket);
rest_status rest_suffix_array_build(const int32_t* d_tokens, uint64_t n_tokens, int32_t sa_bytes,
                                    void* d_sa, void* d_ws, size_t ws_bytes, void* stream);
/* The true suffix array (whole suffixes compared, no ties left): prefix doubling carried on
 * past 32 tokens until every suffix is distinct, one flag read back per extra round (the call
 * synchronises `stream`).  Streams of up to 2^31 - 1 tokens; workspace as for the first method.
 * rest_draft gives the same results on either array; this one is for callers who want the
 * array itself. */
rest_status rest_suffix_array_build_full(const int32_t* d_tokens, uint64_t n_tokens, int32_t sa_bytes,
                                         void* d_sa, void* d_ws, size_t ws_bytes, void* stream);
/*
 * rest_suffix_array_append - the suffix array after n_new tokens were appended to a stream of
 * n_old tokens (Sec. 3.2 "Datastore construction": a datastore that grows).  Only the suffixes
 * of the last 31 old positions and of the new tokens can change place under the 32-token
 * order; they are sorted by themselves and merged into the old array in one pass.
 *   d_tokens   int32[n_old + n_new]: the whole stream, old tokens first
 *   d_sa_old   the array of the first n_old tokens as rest_suffix_array_build wrote it (NULL when n_old = 0)
 *   d_sa_new   receives n_old + n_new entries of sa_bytes bytes; must not be d_sa_old
 *   d_ws       rest_suffix_array_append_workspace_bytes(n_new) bytes (about 44 bytes per new
 *              token + 64 MiB), 256-byte aligned.  Asynchronous on `stream`.
 */
size_t rest_suffix_array_append_workspace_bytes(uint64_t n_new);
rest_status rest_suffix_array_append(const int32_t* d_tokens, uint64_t n_old, uint64_t n_new,
                                     const void* d_sa_old, int32_t sa_bytes, void* d_sa_new,
                                     void* d_ws, size_t ws_bytes, void* stream);
/* The second method whatever the size: groups of at most max_group positions (0: as many as the
 * workspace allows; at least the count of the most frequent first token). */
rest_status rest_suffix_array_build_in_groups(const int32_t* d_tokens, uint64_t n_tokens,
                                              int32_t sa_bytes, void* d_sa, uint64_t max_group,
                                              void* d_ws, size_t ws_bytes, void* stream);

/*
 * Device-side trouble that no per-call status can carry.  Every wait inside the kernels is
 * bounded; a kernel that gives up sets a bit here instead of spinning, and its output is then
 * undefined.  Reads and clears the flags of the current device (synchronises the device).
 *   bit 0: rest_tree_attention or rest_paged_attention (_scaled) gave up waiting for its tensor-core work
 *   bit 1: one of them found its shared-memory window misaligned and did nothing
 */
rest_status rest_device_error_flags(uint32_t* h_flags);

const char* rest_status_string(rest_status s);
/* Text of the last CUDA runtime error seen by this library on the calling thread. */
const char* rest_last_cuda_error(void);

#ifdef __cplusplus
}
#endif
#endif /* REST_H_ */
