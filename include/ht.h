/*
 * ht.h -- C ABI of the B200 tree-verify library for Hidden Transfer decoding
 * (arXiv 2404.12022).  One decoding round verifies a flattened draft tree and the
 * pseudo positions produced by the hidden-transfer projection in a single forward; this
 * library holds the data-parallel operations of that forward that are specific to the
 * method (projection, tree attention, verification, compaction) and the steps around them
 * (rotary embedding + cache append, draft tree, a paged cache).  Everything else of the
 * transformer layer (norms, Q/K/V/O and MLP GEMMs, lm-head) is the caller's.
 *
 * Conventions for every entry point
 *   - Pointers are DEVICE pointers unless a comment says "host".  The caller owns every
 *     buffer, workspace included; the library allocates no device memory.  What it keeps
 *     between calls is per-device set-up only (kernel attributes, SM count, how many of a
 *     kernel's blocks the device holds, the address of the built-in scratch array of
 *     ht_tree_attention_static); a cudaDeviceReset makes that stale.
 *   - Work is enqueued on the caller's stream (`stream` is a cudaStream_t passed as
 *     void*; NULL = the default stream) and the call returns without synchronising.
 *   - The return value is a host-checkable status (HT_OK or HT_ERR_*).  When it is not
 *     HT_OK nothing was launched and ht_last_error_string() describes why.
 *   - Errors only the device can see (an illegal parent array, a cache length that does
 *     not fit, a malformed accepted path) are written to `status` -- one int32 per
 *     sequence, HT_STATUS_* -- and that sequence's work is skipped.  Device code never
 *     traps or asserts.  Every call that takes `status` writes all B entries.
 *   - Tensors are dense row-major with the last index fastest; every base pointer must
 *     be 16-byte aligned.
 *
 * Shapes: B sequences; N query rows per sequence = T draft-tree nodes followed by P
 * pseudo positions; Hq query heads sharing Hkv KV heads (Hq % Hkv == 0); head size D;
 * `cap` rows of cache capacity per (sequence, KV head); vocabulary V; hidden size d;
 * k transfer steps.
 */
#ifndef HT_H_
#define HT_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { HT_F32 = 0, HT_F16 = 1, HT_BF16 = 2 } ht_dtype;

enum {
    HT_OK = 0,
    HT_ERR_INVALID_ARG = 1, /* null / misaligned pointer, non-positive or inconsistent size */
    HT_ERR_UNSUPPORTED = 2, /* a legal request this build has no kernel for */
    HT_ERR_BAD_TREE = 3,    /* reserved for host-side tree checks */
    HT_ERR_WORKSPACE = 4,   /* workspace smaller than ht_tree_attention_workspace() */
    HT_ERR_CUDA = 5,        /* the CUDA runtime reported an error at launch */
    HT_ERR_TIMEOUT = 6      /* a bounded device-side wait ran out (reported via status) */
};

enum {
    HT_STATUS_OK = 0,
    HT_STATUS_BAD_TREE = 1,      /* some parent[r] is outside [-1, r) */
    HT_STATUS_BAD_LEN = 2,       /* kv_len[b] < 0 or kv_len[b] + N > cap */
    HT_STATUS_BAD_PATH = 3,      /* accepted path not increasing / out of range */
    HT_STATUS_PATH_TOO_LONG = 4, /* the accepted path has more than max_path nodes */
    HT_STATUS_BAD_PAGE = 5,      /* paged cache: a block-table entry the sequence needs is outside the pool */
    HT_STATUS_TIMEOUT = 6,
    HT_STATUS_BAD_PARAM = 7      /* sampling: a parameter or a uniform number of the sequence is out of range */
};

/* ht_attn_desc.flags */
#define HT_ATTN_FORCE_SIMT 1u /* use the fp32-ALU kernel even where a tensor-core kernel applies */
/* The caller vouches that the first 64 KiB of the workspace are as a cudaMemset to zero, or any earlier attention
 * call on this workspace that reported no HT_STATUS_TIMEOUT (whatever its cache, its scores and the kernel it took), left
 * them: the call then leaves out the small kernel that clears the arrival counters kept there (every call
 * leaves the counters it used at zero).  Worth about a microsecond per call in a chain of calls; with the flag
 * set on a workspace that is not in that state, results of sequences whose work was split are undefined
 * (nothing faults, nothing waits). */
#define HT_ATTN_WORKSPACE_CLEAN 2u
/* The caller vouches that kv_len, parent, the cache rows below kv_len[b] of every sequence (and, for a paged
 * cache, the block-table entries of those rows) were final before the two kernels ahead of this call in `stream`
 * began.  (In a decoding step they are: the lengths change at the compaction, the rows below them are earlier
 * steps', and the tree is drafted before the first layer.)  The tensor-core kernels then make their plan and
 * fetch their first context tiles while the kernel ahead is still finishing, and wait for it only before they
 * read q or rows at or beyond kv_len[b] and before they write anything: about 3 us per call in a chain of calls.
 * A broken promise gives wrong results for the call, never a fault or a wait.  The fp32-ALU kernel ignores the
 * flag. */
#define HT_ATTN_CONTEXT_FINAL 4u
/* Test hook, never to be set in production: the tensor-core kernels' device-side waits give up after about a
 * microsecond instead of a second, so that their give-up path can be exercised: the call returns, the sequences'
 * status words read HT_STATUS_TIMEOUT and `out` is meaningless.  Nothing faults and nothing is left in flight:
 * a thread block that has given up still waits, with the full limit, for its own copies and tensor-core
 * operations before it frees what they write to. */
#define HT_ATTN_TEST_SHORT_WAITS 0x80000000u

typedef struct {
    int32_t B, N, Hq, Hkv, D, cap;
    int32_t dtype;        /* ht_dtype of q, caches and out */
    float scale;          /* softmax scale; <= 0 selects 1/sqrt(D) */
    int64_t kv_stride_b;  /* elements between sequences in each cache; 0 = Hkv*cap*D */
    int64_t kv_stride_h;  /* elements between KV heads; 0 = cap*D.  Rows are D apart. */
    int32_t num_splits;   /* KV splits per (sequence, head); 0 = library chooses */
    uint32_t flags;
} ht_attn_desc;

typedef struct {
    int32_t layers, B, Hkv, cap, D;
    int32_t dtype;        /* ht_dtype (only its width matters) */
    int32_t N;            /* tree rows behind each context: accepted indices lie in [0, N) */
    int64_t stride_layer; /* elements; 0 = B*Hkv*cap*D */
    int64_t stride_b;     /* elements; 0 = Hkv*cap*D */
    int64_t stride_h;     /* elements; 0 = cap*D */
} ht_cache_desc;

/* Knobs read once per process from the environment, for cross-checks and bug reports (results never need them):
 *   HT_LOG=1                        every entry point prints its arguments and the kernel it chose to stderr
 *   HT_FORCE_PATH=simt|mma|tcgen05  attention on the fp32-ALU kernel (simt); ht_transfer of 16-bit inputs on the
 *                                   warp-level kernel (mma) or, where the shape allows, on the tcgen05 kernel
 *   HT_SPLITS=n                     attention with n KV splits where the descriptor leaves the choice
 *                                   (num_splits == 0): the split-KV ALU kernel, as an explicit num_splits selects it
 * ht_tree_attention_workspace() and ht_tree_attention_launches() answer for the kernel the knobs select. */

/* Library version (major*10000 + minor*100 + patch). */
int ht_version(void);

/* Host string describing the most recent non-HT_OK return on the calling thread. */
const char *ht_last_error_string(void);

/*
 * Hidden-transfer projection -- Section "Hidden Transfer" and the displayed equation of
 * Section "Training stage":  h~ = W^i_{t_i} . h  with W^i in R^{d x d}, 1 <= i <= k, a
 * plain linear map (no bias, no activation).
 *   h_src [B, d]      hidden state of the source token of each sequence
 *   W     [k, d, d]   W[i][r][c]: output feature r, input feature c (W acts on a column)
 *   out   [B, k, d]   out[b][i][r] = sum_c W[i][r][c] * h_src[b][c]
 * fp32 accumulation, result rounded once to `dtype`.  d must be a multiple of 4 (fp32)
 * or 8 (fp16 / bf16).  B*k*d == 0 is a no-op.
 * B is the number of source rows, whatever they are: one per sequence (pseudo states
 * hanging off one node), or one per tree node of every sequence (the reading in which
 * every token gets its pseudo states), B x T rows, for which the 16-bit types run as a
 * matrix product on the tensor cores in one pass over W.  That kernel's waits are bounded
 * (about a second); should one run out, the outputs of the affected tile are NaN -- the call
 * has no status argument, so a NaN tile is the only signal (NaN inputs give NaN too).
 * All pointers are device pointers, 16-byte aligned; nothing is retained after the call.
 */
int ht_transfer(const void *h_src, const void *W, void *out, int B, int k, int d, int dtype,
                void *stream);

/*
 * Tree attention -- Section "Tree attention": the draft tree is flattened into a
 * sequence and "a token only attends to its ancestors" (and the context); pseudo
 * positions follow Section "Training stage" (a pseudo state sees the context, earlier
 * pseudo states and itself) and are given as ordinary rows of `parent`.
 *   q        [B, N, Hq, D]
 *   k_cache, v_cache  [B, Hkv, cap, D] (strides in desc); sequence b holds kv_len[b]
 *            context rows; the K/V of query row r must already sit at row kv_len[b] + r
 *   kv_len   [B] int32
 *   parent   [B, N] int32, parent[b][r] in [-1, r); -1 attaches r to the context
 *   out      [B, N, Hq, D]:  out[b,r,h] = softmax(scale * q[b,r,h] . K^T) V over cache rows
 *            [0, kv_len[b]) of KV head h / (Hq/Hkv) and rows kv_len[b] + c for c = r and
 *            every ancestor c of r.  fp32 (fp16 / bf16 inputs: tensor-core products with
 *            fp32 accumulation) softmax and accumulation, rounded once to `dtype`.
 *   workspace, workspace_bytes  scratch of at least ht_tree_attention_workspace(desc)
 *            bytes, 16-byte aligned; contents need no initialisation (but see
 *            HT_ATTN_WORKSPACE_CLEAN) and, beyond the first 64 KiB, are undefined afterwards.
 *            Calls that run concurrently need distinct workspaces.
 *   status   [B] int32 out: HT_STATUS_BAD_TREE / HT_STATUS_BAD_LEN sequences are skipped
 *            (their rows of `out` are left untouched).
 * Cache rows at or beyond kv_len[b] + N are never used for a result, whatever they hold.
 * Supported: D in {64, 128}; N <= 1024.  B == 0 or N == 0 is a no-op.
 * Stream behaviour (fp16 / bf16, D = 128): the call's kernels are launched with programmatic
 * stream serialization, i.e. their thread blocks may be set up while the kernel before them in
 * `stream` is still finishing; they read inputs, workspace and outputs only after that kernel
 * has completed, so the results are those of plain stream order.
 */
size_t ht_tree_attention_workspace(const ht_attn_desc *desc /* host */);
/* Number of this library's kernels that one ht_tree_attention call with this descriptor enqueues (1 or 2:
 * a kernel that zeroes arrival counters -- left out under HT_ATTN_WORKSPACE_CLEAN -- or one that merges split
 * partials, may accompany the attention kernel); 0 for a descriptor the call would reject or that has nothing
 * to do. */
int ht_tree_attention_launches(const ht_attn_desc *desc /* host */);
int ht_tree_attention(const ht_attn_desc *desc /* host */, const void *q, const void *k_cache,
                      const void *v_cache, const int32_t *kv_len, const int32_t *parent, void *out,
                      void *workspace, size_t workspace_bytes, int32_t *status, void *stream);

/*
 * Tree attention over a paged cache: the same operation as ht_tree_attention (Section "Tree
 * attention"), with the K / V rows of a sequence scattered over fixed-size pages of a shared pool,
 * the layout serving systems keep their caches in.
 *   pages->page_size   rows per page: a power of two >= 16
 *   pages->max_pages   block-table entries per sequence; the capacity of a sequence is
 *                      max_pages * page_size rows (desc->cap and desc's cache strides are ignored)
 *   pages->n_pages     pages in the pool
 *   pages->page_stride, head_stride   elements between pages / between the KV heads of a page;
 *                      0 = Hkv * page_size * D / page_size * D.  Rows are D apart.
 *   k_pages, v_pages   [n_pages, Hkv, page_size, D]
 *   block_table        [B, max_pages] int32: cache row r of sequence b is row r % page_size of page
 *                      block_table[b][r / page_size].  As in ht_tree_attention the K / V of query
 *                      row r must already sit at cache row kv_len[b] + r.  Entries of pages wholly
 *                      past row kv_len[b] + N are not consulted for a result and may hold anything.
 *   status             as in ht_tree_attention, plus HT_STATUS_BAD_PAGE for a sequence one of whose
 *                      needed entries lies outside [0, n_pages): page 0 is read in its place (no
 *                      access outside the pool) and the sequence's rows of `out` are meaningless.
 * q, kv_len, parent, out, workspace (ht_tree_attention_workspace(desc) bytes) as in
 * ht_tree_attention.  Supported: fp16 / bf16, D = 128, Hq / Hkv a power of two, N <= 1024,
 * B <= 256 (the tensor-core kernels); anything else returns HT_ERR_UNSUPPORTED.
 */
typedef struct {
    int32_t page_size, max_pages, n_pages;
    int64_t page_stride, head_stride;
} ht_paged_desc;
int ht_tree_attention_paged(const ht_attn_desc *desc /* host */, const ht_paged_desc *pages /* host */,
                            const void *q, const void *k_pages, const void *v_pages,
                            const int32_t *block_table, const int32_t *kv_len, const int32_t *parent,
                            void *out, void *workspace, size_t workspace_bytes, int32_t *status,
                            void *stream);

/*
 * Tree attention with shaped scores: ht_tree_attention / ht_tree_attention_paged (Section "Tree attention") for models
 * that cap their attention scores or give them a bias by distance in place of a rotary embedding.  With
 * s = scale * q[b,r,h] . k the raw score of a visible key, the softmax is over
 *     cap > 0       s := cap * tanh(s / cap)                (cap 0: none)
 *     slopes given  s := s - slopes[h] * (pos[b,r] - position of the key)
 * where the position of context row j is j and that of tree row c is pos[b,c].
 *   cap      finite, >= 0; neither cap nor cap / scale above 1e18, and with a cap no scale above 1e4 (squares of what lies
 *            in between are held in 32 bits)
 *            A score is held in 32 bits, its bias included; distances are exact up to 2^24.  Keys that weigh less than 2^-40 of
 *            a row's largest may be left out.  As in the two entry points, a 16-bit call's weights are rounded to its type for
 *            the product with V, but as a pair of two such values where a row may see few keys: in tiles with tree rows and,
 *            with slopes, in those of the last 128 context rows.
 *   slopes   [Hq] float or NULL; any sign, 0 for a head without a bias
 *   pos      [B, N] int32 position ids of the query rows (ht_draft_tree's `pos`, followed by the pseudo rows'); needed with
 *            slopes.  HT_ATTN_CONTEXT_FINAL says nothing about slopes and pos: the kernel ahead may write them.
 * All other arguments, the workspace, flags, statuses and supported shapes are those of the two entry points; a NULL
 * descriptor or one that asks for nothing is the plain call.
 */
typedef struct {
    float cap;
    const float *slopes;  /* device */
    const int32_t *pos;   /* device */
} ht_score_desc;
int ht_tree_attention_scored(const ht_attn_desc *desc /* host */, const ht_score_desc *score /* host */, const void *q,
                             const void *k_cache, const void *v_cache, const int32_t *kv_len, const int32_t *parent,
                             void *out, void *workspace, size_t workspace_bytes, int32_t *status, void *stream);
int ht_tree_attention_scored_paged(const ht_attn_desc *desc /* host */, const ht_paged_desc *pages /* host */,
                                   const ht_score_desc *score /* host */, const void *q, const void *k_pages,
                                   const void *v_pages, const int32_t *block_table, const int32_t *kv_len,
                                   const int32_t *parent, void *out, void *workspace, size_t workspace_bytes,
                                   int32_t *status, void *stream);

/*
 * The two row-moving steps on a paged cache (same pools, block table and descriptor as
 * ht_tree_attention_paged; one block table serves all layers):
 *   ht_rope_kv_append_paged  as ht_rope_kv_append, the rows of sequence b landing at logical cache rows
 *       kv_len[b] + r through the block table.  A row whose page entry lies outside the pool is
 *       not stored (its q row is still rotated) and marks the sequence HT_STATUS_BAD_PAGE.
 *   ht_kv_compact_paged      as ht_kv_compact on pools [layers, n_pages, Hkv, page_size, D];
 *       desc->cap, stride_b and stride_h are ignored (the capacity is max_pages * page_size, the strides
 *       are those of `pages`), desc->stride_layer is the distance between the layers' pools in
 *       elements (0 = n_pages * page_stride).  Rows move between pages as the table says; a
 *       needed entry outside the pool leaves the sequence unchanged with HT_STATUS_BAD_PAGE.
 */
int ht_rope_kv_append_paged(const ht_attn_desc *desc /* host */, const ht_paged_desc *pages /* host */,
                            const void *q_in, const void *k_in, const void *v_in, const int32_t *pos,
                            const int32_t *kv_len, const int32_t *block_table, float rope_base,
                            void *q_out, void *k_pages, void *v_pages, int32_t *status, void *stream);
int ht_kv_compact_paged(void *k_pages, void *v_pages, const ht_cache_desc *desc /* host */,
                        const ht_paged_desc *pages /* host */, const int32_t *block_table,
                        const int32_t *kv_len, const int32_t *accept_len, const int32_t *accept_path,
                        int max_path, int32_t *new_kv_len, int32_t *status, void *stream);

/*
 * Greedy verification -- Fig. 2 caption ("find the last accepted token position"),
 * Section "Inference stage", Section "Setup" (greedy sampling; output identical to
 * auto-regressive decoding).
 *   logits    [B, N, V] of `dtype`
 *   tokens    [B, T] int32 draft token of each tree node (T <= N)
 *   parent    [B, N] int32 (rows < T are consulted)
 *   root_pred [B] int32 or NULL: the token greedy decoding emits after the context (the
 *             argmax carried over from the previous round).  Top-level nodes (parent -1)
 *             are checked against it; with NULL they are taken as known-correct.
 *   pred      [B, N] int32 out, required: argmax_v logits[b,r,v]; the lowest index wins
 *             ties, NaN never wins, a row of NaNs gives 0
 *   accept_len  [B] out: number of nodes on the longest root path all of whose nodes c
 *             satisfy tokens[c] == pred[parent[c]] (top level: == root_pred); ties between
 *             paths of equal length go to the smallest terminal node index
 *   accept_path [B, max_path] out: that path, root first, padded with -1
 *   next_token  [B] out: pred at the path's last node; root_pred[b] (or -1 without
 *             root_pred) when nothing is accepted
 *   status    [B] out: HT_STATUS_BAD_TREE, HT_STATUS_PATH_TOO_LONG (accept_len 0, next -1)
 * max_path <= 255.
 * accept_len is also where the kernel counts, in the bits above the low eight, the rows of a sequence that are
 * done; the sequence's last thread block replaces the count by the length.  ON ENTRY every accept_len[b] must
 * therefore hold a value in [0, 255]: zero before the first call (the caller clears it once), afterwards what
 * the previous call left there will do.  Anything else (uninitialised memory, a buffer last used by a call that
 * did not finish) makes the count come out wrong and the sequence's outputs are not written.
 * One kernel, launched with programmatic stream serialization and waiting, at its first instruction, for the
 * work ahead of it in the stream: ordering is that of an ordinary launch.
 */
int ht_verify_greedy(const void *logits, int dtype, const int32_t *tokens, const int32_t *parent,
                     const int32_t *root_pred, int B, int N, int T, int V, int max_path,
                     int32_t *pred, int32_t *accept_len, int32_t *accept_path,
                     int32_t *next_token, int32_t *status, void *stream);

/*
 * Greedy verification and KV compaction in one launch -- Fig. 2 caption and Section "Inference stage" (find the
 * last accepted position, then go on from it): ht_verify_greedy followed by ht_kv_compact, with the same
 * arguments, results and restrictions as the two calls (max_path <= 64; new_kv_len must not overlap kv_len or
 * accept_len; accept_len[b] in [0, 255] on entry), and the same results bit for bit.
 *   rows     logits rows per sequence whose argmax is taken, T <= rows <= N; 0 selects T, the rows
 *            acceptance can consult.  pred[b][r] is written for r < rows only.
 *   status, compact_status   [B] out: the status words of the verification and of the compaction.
 *   desc     its B and N must equal B and N.
 * The thread blocks first take the argmax of the rows; the block that completes a sequence searches its
 * tree; then all blocks share out the compaction's (layer, sequence, head group) items, each waiting (bounded:
 * about a second, then HT_STATUS_TIMEOUT in compact_status and the sequence's cache left as it is) until the
 * sequence's accepted length has been stored.  The grid never exceeds what the GPU holds at once.
 */
int ht_verify_greedy_compact(const void *logits, int dtype, const int32_t *tokens, const int32_t *parent,
                             const int32_t *root_pred, int B, int N, int T, int V, int max_path, int rows,
                             int32_t *pred, int32_t *accept_len, int32_t *accept_path, int32_t *next_token,
                             int32_t *status, void *k_cache, void *v_cache, const ht_cache_desc *desc /* host */,
                             const int32_t *kv_len, int32_t *new_kv_len, int32_t *compact_status, void *stream);

/*
 * KV compaction -- implied by verifying under a KV cache (Fig. 1 caption; Section
 * "Inference stage"): after acceptance only the accepted path's K/V may follow the
 * context.  For every layer, sequence b, KV head and j < accept_len[b], cache row
 * kv_len[b] + j receives what row kv_len[b] + accept_path[b][j] held before the call (K and
 * V alike); new_kv_len[b] = kv_len[b] + accept_len[b].  In place and safe when source and
 * destination rows overlap.  Rows below kv_len[b] are untouched; rows at or beyond
 * new_kv_len[b] are unspecified afterwards.
 *   k_cache, v_cache  [layers, B, Hkv, cap, D] (strides in desc)
 *   accept_path [B, max_path], strictly increasing, accept_path[b][j] in [j, N)
 *   status [B] out: HT_STATUS_BAD_LEN / HT_STATUS_BAD_PATH sequences are left unchanged and
 *            new_kv_len[b] = kv_len[b].
 * max_path <= 64.  D * element size must be a multiple of 16 bytes.
 * new_kv_len must not overlap kv_len or accept_len (HT_ERR_INVALID_ARG): the sequence's thread blocks
 * read both throughout the kernel, so an update in place would be seen by some of them and not by
 * others.  Keep two length arrays and swap them between rounds.
 * The kernel is launched with programmatic stream serialization and waits, at its first instruction, for
 * the work ahead of it in the stream: ordering is that of an ordinary launch.
 */
int ht_kv_compact(void *k_cache, void *v_cache, const ht_cache_desc *desc /* host */,
                  const int32_t *kv_len, const int32_t *accept_len, const int32_t *accept_path,
                  int max_path, int32_t *new_kv_len, int32_t *status, void *stream);

/*
 * Draft tree for the next round -- Section "Inference stage" (the candidate sequences are made
 * "into a tree structure by merging their common ancestors" and the tree is flattened) and Section
 * "Tree attention" ("a pre-defined tree structure and parser"; tokens keep their positional indices).
 * The candidates are the most likely tokens of the pseudo positions' distributions (Section "Hidden
 * Transfer": the lm-head decodes the pseudo hidden states).  The pre-defined structure is a template
 * shared by all sequences: node n at level i takes the tmpl_rank[n]-th most likely token (0 = the
 * most likely) of pseudo position i, so merging common ancestors costs nothing at run time.
 *   logits      [B, rows, V] of `dtype`; pseudo position i (1..P) of sequence b is row first_row + i - 1
 *   tmpl_parent [T] int32, tmpl_parent[n] in [-1, n)
 *   tmpl_rank   [T] int32, in [0, K) for nodes of level >= 1
 *   root_token  [B] int32 or NULL.  Given: nodes with parent -1 are the known next token (level 0,
 *               e.g. next_token of ht_verify_greedy) and their children are level 1.  NULL: nodes
 *               with parent -1 are level 1 themselves (a forest of first drafts).
 *   base_pos    [B] int32: position id of the top-level nodes (e.g. new_kv_len of ht_kv_compact)
 *   topk        [B, P, K] out: the K most likely tokens per pseudo position -- larger value first,
 *               lower index first among equal values, NaN below everything
 *   tokens      [B, T] out: draft token of every template node
 *   pos         [B, T] out: base_pos[b] + depth of the node (top-level nodes: depth 0)
 *   status      [B] out: HT_STATUS_BAD_TREE when the template is malformed (a parent that is not an
 *               earlier node, a level beyond P, a rank outside [0, K)); tokens and pos are then -1.
 * 1 <= K <= 16, K <= V, T >= 1.  B == 0 is a no-op.  The parent array of the next round's
 * ht_tree_attention is tmpl_parent followed by the pseudo rows.
 */
int ht_draft_tree(const void *logits, int dtype, int B, int rows, int V, int first_row, int P, int K,
                  const int32_t *tmpl_parent, const int32_t *tmpl_rank, int T, const int32_t *root_token,
                  const int32_t *base_pos, int32_t *topk, int32_t *tokens, int32_t *pos, int32_t *status,
                  void *stream);

/*
 * Rotary position embedding at the tree's position ids, and placement of the rows' K / V behind
 * the context -- the step ahead of ht_tree_attention.  Section "Tree attention": the flattened tree
 * preserves "the original positional indices of each token"; Section "Training stage": a pseudo state
 * of step i has position id j + i; Section "Setup": LLaMA-2 / Vicuna models, i.e. the rotary embedding
 * in the half-split pairing (feature i with feature i + D/2, angle pos * rope_base^(-2i/D)).
 *   desc     B, N, Hq, Hkv, D, cap, dtype and the cache strides are used (scale, num_splits, flags are not)
 *   q_in     [B, N, Hq, D], k_in, v_in [B, N, Hkv, D]: the rows' projections before the rotation
 *   pos      [B, N] int32 position ids (e.g. ht_draft_tree's `pos`, followed by the pseudo rows')
 *   kv_len   [B] int32
 *   q_out    [B, N, Hq, D]: q_in rotated (may alias q_in)
 *   k_cache, v_cache [B, Hkv, cap, D]: row kv_len[b] + r receives k_in[b, r] rotated / v_in[b, r] as is
 *   status   [B] out: HT_STATUS_BAD_LEN sequences are skipped (nothing of theirs is written)
 * Angles are formed in fp64, products in fp32, one rounding to `dtype`.  D in {64, 128}.
 */
int ht_rope_kv_append(const ht_attn_desc *desc /* host */, const void *q_in, const void *k_in, const void *v_in,
                      const int32_t *pos, const int32_t *kv_len, float rope_base, void *q_out, void *k_cache,
                      void *v_cache, int32_t *status, void *stream);

/*
 * Norm of each head, rotary embedding and placement of the rows' K / V behind the context, in one pass: the step ahead
 * of ht_tree_attention for models that normalise their query and key heads, rotate a part of each head only, pair
 * neighbouring features, or scale the rotation for contexts longer than the trained one.  (Section "Tree attention":
 * the flattened tree keeps the tokens' positional indices; the paper's own models take ht_rope_kv_append.)
 * For each query and key head x of D features (the norm where `norm` asks for it):
 *     y = x * rsqrt(mean(x^2) + eps) * (weight + weight_offset)
 * then the first rot_dim features of y are rotated in pairs (a, b) by pos * f_i:  a' = a cos - b sin, b' = b cos + a sin,
 * with cosine and sine times `magnitude`.
 *   rot_dim       0..D, even; half-split pairing: a multiple of 16 (8 for fp32)
 *   interleaved   0: pair i = features (i, i + rot_dim/2); else features (2i, 2i + 1)
 *   scaling       HT_ROPE_PLAIN     f_i = rope_base^(-2i/rot_dim)
 *                 HT_ROPE_LINEAR    f_i / factor
 *                 HT_ROPE_BY_PARTS  turns = orig_len * f_i / (2 pi), keep = clamp((turns - low) / (high - low), 0, 1):
 *                                   f_i * (keep + (1 - keep) / factor)
 *   magnitude     0 selects 1
 *   q_stride, k_stride, v_stride   elements between consecutive rows of q_in / k_in / v_in (row r of sequence b is row
 *                 b*N + r); 0 = Hq*D / Hkv*D.  The heads of a row are D apart: a fused projection's output is passed by
 *                 three pointers into it and one stride.
 */
#define HT_HEAD_NORM_Q 1
#define HT_HEAD_NORM_K 2
enum { HT_ROPE_PLAIN = 0, HT_ROPE_LINEAR = 1, HT_ROPE_BY_PARTS = 2 };
typedef struct {
    int32_t norm;                  /* HT_HEAD_NORM_Q | HT_HEAD_NORM_K */
    int32_t rot_dim, interleaved, scaling;
    float eps, weight_offset, rope_base, factor, low, high, orig_len, magnitude;
    int64_t q_stride, k_stride, v_stride;
} ht_head_desc;

/*
 *   desc     B, N, Hq, Hkv, D, cap, dtype and the cache strides are used (scale, num_splits, flags are not)
 *   q_in [B, N, Hq, D], k_in, v_in [B, N, Hkv, D] (rows strided, see above), q_weight, k_weight [D] of `dtype` or NULL
 *            (ones, without weight_offset)
 *   pos [B, N] int32, kv_len [B] int32
 *   q_out    [B, N, Hq, D] dense; may be q_in itself where q_in is dense, and must not overlap the inputs otherwise
 *   k_cache, v_cache [B, Hkv, cap, D]: row kv_len[b] + r receives the key row / v_in[b, r] as is
 *   status   [B] out: HT_STATUS_BAD_LEN sequences are skipped (nothing of theirs is written)
 * The paged form takes pools, block table and descriptor as ht_rope_kv_append_paged does; a row whose page entry lies
 * outside the pool is not stored (its q row is still written) and marks the sequence HT_STATUS_BAD_PAGE.
 * Angles are formed in 64 bits, the norm, products and sums in fp32, one rounding to `dtype`.  D in {64, 128}.
 */
int ht_norm_rope_kv_append(const ht_attn_desc *desc /* host */, const ht_head_desc *head /* host */, const void *q_in,
                           const void *k_in, const void *v_in, const void *q_weight, const void *k_weight,
                           const int32_t *pos, const int32_t *kv_len, void *q_out, void *k_cache, void *v_cache,
                           int32_t *status, void *stream);
int ht_norm_rope_kv_append_paged(const ht_attn_desc *desc /* host */, const ht_head_desc *head /* host */,
                                 const ht_paged_desc *pages /* host */, const void *q_in, const void *k_in,
                                 const void *v_in, const void *q_weight, const void *k_weight, const int32_t *pos,
                                 const int32_t *kv_len, const int32_t *block_table, void *q_out, void *k_pages,
                                 void *v_pages, int32_t *status, void *stream);

/*
 * Tokens drawn from filtered distributions with given uniform numbers.  (The paper verifies greedily; with sampled tokens
 * in the argmax's place the emitted text is distributed as, and for the same uniform numbers equal to, what sampling one
 * token at a time gives.)  For a row of logits x with largest value m:
 *     w_i = exp((x_i - m) / temperature), 0 where that is below 2^-1000; larger x comes first in the order, the lower
 *     index among equals.  Kept are the first top_k of the order; of those, the ones before which less than
 *     top_p * (weight of the first top_k) has come; of those, the ones with w_i >= min_p.  The token is the first kept
 *     one, in index order, at which the running kept weight exceeds uniform * (kept weight); the last one with a
 *     weight where none does (uniform = 1).
 *   logits       [B, N, V] of `dtype`; NaN counts as -inf.  A row without anything above -inf gives its first -inf, a row
 *                of NaNs 0; where +inf occurs, those tokens share the weight.
 *   uniform      [B, N] float, in [0, 1]
 *   temperature  [B] float or NULL (1); 0: the argmax, lowest index among equals
 *   top_k        [B] int32 or NULL; <= 0 or >= V: off
 *   top_p        [B] float or NULL; >= 1: off; <= 0: the first of the order
 *   min_p        [B] float or NULL; <= 0: off
 *   token        [B, N] int32 out
 *   status       [B] out: HT_STATUS_BAD_PARAM where the temperature is negative, infinite or NaN, top_p or min_p NaN, min_p
 *                above 1 or a uniform number outside [0, 1]; the sequence's tokens are then -1.
 * Weights and their sums are held in 64 bits (in rows of up to 2^20, weights below 2^-31 of the largest are added up in
 * 32, which is off by less than 1e-8 of the whole).
 * N is the rows per sequence (1 for plain decoding); V <= 2^30.
 */
int ht_sample(const void *logits, int dtype, int B, int N, int V, const float *uniform, const float *temperature,
              const int32_t *top_k, const float *top_p, const float *min_p, int32_t *token, int32_t *status,
              void *stream);

/*
 * Sampled verification -- ht_verify_greedy with each tree row's token drawn as ht_sample draws it instead of its argmax:
 * a node is accepted where its draft token is the token drawn at its parent (top level: root_pred, the token drawn last).
 *   logits [B, N, V], uniform [B, N]: the T tree rows are used, 1 <= T <= N
 *   pred [B, N] out: the drawn tokens; -1 for the rows behind the tree
 *   tokens, parent, root_pred, accept_len (also on entry: [0, 255]), accept_path, next_token: as in ht_verify_greedy
 *   status [B] out: as ht_verify_greedy, and HT_STATUS_BAD_PARAM as ht_sample, which looks at the uniform numbers of the T
 *            tree rows (pred -1, accept_len 0, accept_path and next_token -1)
 */
int ht_verify_sampled(const void *logits, int dtype, const float *uniform, const float *temperature,
                      const int32_t *top_k, const float *top_p, const float *min_p, const int32_t *tokens,
                      const int32_t *parent, const int32_t *root_pred, int B, int N, int T, int V, int max_path,
                      int32_t *pred, int32_t *accept_len, int32_t *accept_path, int32_t *next_token, int32_t *status,
                      void *stream);

/*
 * An 8-bit cache: half the bytes of a 16-bit one.  (The paper has nothing to say on what the cache holds; the operations are
 * those of the sections named at their 16-bit forms.)  A row of a KV head is D codes in e4m3 (sign, four bits of exponent,
 * three of mantissa, largest 448) and one byte that scales them, and stands for code * 2^(byte - 127).  The codes are laid out
 * as any cache ([B, Hkv, cap, D], or pools of pages [n_pages, Hkv, page_size, D]); the bytes alike without the last index:
 *   k, v          [B, Hkv, cap] or [n_pages, Hkv, page_size], 16-byte aligned (kv_compact: with the layers in front)
 *   stride_layer, stride_b, stride_h   bytes between layers, sequences (paged: pages) and heads, multiples of 16; 0 = dense
 * A contiguous cache's cap is a multiple of 16.  In the cache descriptors `dtype` stays that of q and the inputs; the codes'
 * strides are in codes, multiples of 16.
 * A row is written with the smallest power of two for which no code exceeds 448, each code the nearest (ties to even); a power
 * of two divides exactly, so a row has one right set of codes, and K's norm and rotation are done in 64 bits to meet it.  A row
 * with an infinity or a NaN is marked by a byte of 255 and reads as a NaN throughout: attention gives NaN to the query rows
 * that see it and leaves the others alone.  The codes 0x7F and 0xFF, e4m3's own NaN, are never
 * written and must not stand in rows that hold keys.
 */
typedef struct {
    void *k, *v;          /* device */
    int64_t stride_layer, stride_b, stride_h;
} ht_q8_scales;

/*
 * ht_norm_rope_kv_append (_paged) with the new rows stored in an 8-bit cache (norm = 0 and rot_dim = 0: K as it is).  All other
 * arguments, checks and statuses are those of the two entry points.
 */
int ht_norm_rope_kv_append_q8(const ht_attn_desc *desc /* host */, const ht_head_desc *head /* host */,
                              const ht_q8_scales *scales /* host */, const void *q_in, const void *k_in, const void *v_in,
                              const void *q_weight, const void *k_weight, const int32_t *pos, const int32_t *kv_len, void *q_out,
                              void *k_cache, void *v_cache, int32_t *status, void *stream);
int ht_norm_rope_kv_append_q8_paged(const ht_attn_desc *desc /* host */, const ht_head_desc *head /* host */,
                                    const ht_paged_desc *pages /* host */, const ht_q8_scales *scales /* host */, const void *q_in,
                                    const void *k_in, const void *v_in, const void *q_weight, const void *k_weight,
                                    const int32_t *pos, const int32_t *kv_len, const int32_t *block_table, void *q_out,
                                    void *k_pages, void *v_pages, int32_t *status, void *stream);

/*
 * Tree attention over an 8-bit cache, whole or through a window (Section "Tree attention").  The softmax is that of
 * ht_tree_attention over the values the cache stands for, with q, the weights and the result in `dtype`; of the keys that
 * ht_tree_attention shows a row, a window leaves those at most window - 1 positions ahead of it, and those at positions below
 * `sinks`.  Context row j is at position j, a tree row at kv_len plus the number of its ancestors in the tree.
 *   window  NULL or window 0: none.  window >= 1 (a row sees itself at least), sinks >= 0
 *   scale, num_splits, flags, statuses, workspace: as ht_tree_attention, with ht_tree_attention_q8_workspace(desc) bytes (paged:
 *           of a desc whose cap is max_pages * page_size).
 *           HT_ATTN_CONTEXT_FINAL has no effect.  Workspaces may be shared with ht_tree_attention's calls.
 * Supported: what ht_tree_attention supports (fp16 / bf16 with D = 128 and Hq / Hkv a power of two on the tensor cores, B <= 256;
 * the rest on the fp32 ALUs), paged as well as contiguous.  On the tensor cores q goes as a sum of e4m3 parts relative to a
 * power of two of its row (bf16: two, fp16: three; exact where a value is not 2^9, fp16: 2^6, times smaller than the row's largest,
 * otherwise off by 2^-17 of that at most), K's codes as they are, their powers of two in fp32; V in fp16 relative to the largest
 * scale among the 128 rows of its tile that some query row of the sequence sees (not each of them need: rows of other branches
 * count), exactly where a row's is not 2^22 times smaller; the weights rounded to fp16 (as a pair of two such values in tiles with
 * tree rows and, with a window, in those of the last 128 context rows).
 * Rows that no row sees (ahead of every row's window and behind the first tokens) may hold anything; paged: so may the entries of
 * pages of such rows alone.
 */
typedef struct {
    int32_t window, sinks;
} ht_window_desc;
size_t ht_tree_attention_q8_workspace(const ht_attn_desc *desc /* host */);
int ht_tree_attention_q8(const ht_attn_desc *desc /* host */, const ht_window_desc *window /* host */,
                         const ht_q8_scales *scales /* host */, const void *q, const void *k_cache, const void *v_cache,
                         const int32_t *kv_len, const int32_t *parent, void *out, void *workspace, size_t workspace_bytes,
                         int32_t *status, void *stream);
int ht_tree_attention_q8_paged(const ht_attn_desc *desc /* host */, const ht_paged_desc *pages /* host */,
                               const ht_window_desc *window /* host */, const ht_q8_scales *scales /* host */, const void *q,
                               const void *k_pages, const void *v_pages, const int32_t *block_table, const int32_t *kv_len,
                               const int32_t *parent, void *out, void *workspace, size_t workspace_bytes, int32_t *status,
                               void *stream);

/*
 * ht_kv_compact (_paged) of an 8-bit cache: codes and bytes of the accepted rows move together.  desc->dtype is not used, D is
 * a multiple of 16; everything else as in the two entry points.
 */
int ht_kv_compact_q8(void *k_cache, void *v_cache, const ht_q8_scales *scales /* host */, const ht_cache_desc *desc /* host */,
                     const int32_t *kv_len, const int32_t *accept_len, const int32_t *accept_path, int max_path,
                     int32_t *new_kv_len, int32_t *status, void *stream);
int ht_kv_compact_q8_paged(void *k_pages, void *v_pages, const ht_q8_scales *scales /* host */, const ht_cache_desc *desc /* host */,
                           const ht_paged_desc *pages /* host */, const int32_t *block_table, const int32_t *kv_len,
                           const int32_t *accept_len, const int32_t *accept_path, int max_path, int32_t *new_kv_len,
                           int32_t *status, void *stream);

/*
 * Logits shaped before tokens are drawn from them (ht_sample, ht_verify_sampled, ht_verify_greedy): penalties for what the text
 * holds already, biases, masks.  In a draft tree each row has a text of its own: the sequence's, followed by the draft tokens
 * of its path, so that verification by sampling or by argmax goes on being what drawing one token at a time gives.  For token v
 * of row r, with n the times v was generated (counts[b][v] >> 1, and the nodes below T among r and its ancestors that carry v):
 *     x = logits[b][r][v]
 *     n > 0 or the prompt holds v (counts[b][v] & 1):  x = x > 0 ? x / repetition[b] : x * repetition[b]
 *     x = x - frequency[b] * n - presence[b] * (n > 0) + (sum of v's biases);  not allowed: -inf
 * in fp32, rounded once to `dtype`.
 *   logits, out  [B, N, V] of `dtype`; out may be logits itself and must not overlap it otherwise
 *   counts       [B, V] int32 (ht_count_tokens) or NULL (a text without tokens)
 *   tokens       [B, T] int32 draft tokens, parent [B, N] int32: T <= N <= 1024; T = 0 with NULL tokens and parent: plain decoding
 *   repetition, frequency, presence   [B] float or NULL (1, 0, 0); repetition positive, all finite
 *   bias_id, bias [B, n_bias] int32 / float, n_bias <= 1024: entries of one token add up, in the order of the list; ids outside
 *                [0, V) are passed over
 *   allowed      [B, N, ceil(V / 32)] uint32 or NULL: token v of row r is allowed where bit v % 32 of word v / 32 is set
 *   status       [B] out: HT_STATUS_BAD_TREE, HT_STATUS_BAD_PARAM; the sequence's rows of out are left as they were
 */
int ht_shape_logits(const void *logits, int dtype, int B, int N, int V, const int32_t *counts, const int32_t *tokens,
                    const int32_t *parent, int T, const float *repetition, const float *frequency, const float *presence,
                    const int32_t *bias_id, const float *bias, int n_bias, const uint32_t *allowed, void *out, int32_t *status,
                    void *stream);

/*
 * The counts that the penalties go by: counts[b][v] = 2 * (times v was generated) + (1 where the prompt holds v).
 *   tokens   [B, n_tokens] int32
 *   index    [B, n] int32 or NULL.  NULL: the tokens taken are the first length[b]; given: those at index[b][0 .. length[b]) --
 *            with accept_path and accept_len of a verification, the accepted draft tokens
 *   length   [B] int32 or NULL (all n; without index n is n_tokens)
 *   prompt   0: the tokens were generated; else they are a prompt's
 *   reset    0: they are added to what counts holds; else counts begins anew with them
 *   status   [B] out: HT_STATUS_BAD_PARAM where a length lies outside [0, n] (the sequence's counts are left as they were) or a
 *            token or an index is out of range (it is passed over)
 */
int ht_count_tokens(const int32_t *tokens, const int32_t *index, const int32_t *length, int B, int n_tokens, int n, int V,
                    int prompt, int reset, int32_t *counts, int32_t *status, void *stream);

/*
 * Tree attention without a caller-provided workspace.  (The paper has no counterpart: this
 * entry point exists for integration, not for the method.)
 *
 * Same operation, arguments and results as ht_tree_attention, computed by the split-KV
 * fp32-ALU kernel, for callers that cannot give the library scratch memory because they
 * cannot allocate any: code running where cudaMalloc must not be called, plugin
 * interfaces that pass only inputs and outputs, processes whose device memory is fully
 * committed.  The split partials live in a fixed array of HT_STATIC_SCRATCH_BYTES inside
 * the library image; every GPU context that loads the library holds that array until it
 * exits, used or not.  The call allocates and frees nothing.
 *   - A problem whose partials exceed the array is refused with HT_ERR_WORKSPACE and a
 *     message giving both sizes; desc->num_splits = 1 never needs scratch.
 *   - The first call on each device looks up the array's device address (with the caller's
 *     current device, which must be the one the pointers and the stream belong to; a q on
 *     another device is refused with HT_ERR_INVALID_ARG).  Make that first call outside any
 *     stream capture.  The address is kept for the life of the process: after
 *     cudaDeviceReset the library's per-device state is stale and the process must reload it.
 *   - All calls share the array and it keeps the previous call's contents.  Nothing in it
 *     needs clearing, but calls that overlap on the GPU (two streams, two host threads)
 *     race on it: serialise them.
 */
#define HT_STATIC_SCRATCH_BYTES (16u << 20)
int ht_tree_attention_static(const ht_attn_desc *desc /* host */, const void *q, const void *k_cache,
                             const void *v_cache, const int32_t *kv_len, const int32_t *parent,
                             void *out, int32_t *status, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* HT_H_ */
