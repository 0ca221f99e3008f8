/*
 * tsv.h -- C ABI of the tree-speculation verify path over online-compressed attention
 *          (CSA "C4" sparse cache + HCA "C128" dense cache + sliding window), B200 / sm_100a.
 *
 * Three calls make one verify cycle of one attention layer stack:
 *
 *     for every layer:  branch_state_build(...)  ->  tree_verify_attn(...)
 *     then once:        accept_and_refresh(all layers)
 *
 * tree_verify_layer(...) is the first two in one call.
 *
 * Conventions
 *   - Every `void*` / typed pointer inside the structs is a DEVICE pointer unless the
 *     comment says HOST.  The structs themselves and `tsv_shape` live in HOST memory and
 *     are read during the call only.
 *   - The caller owns every buffer.  The library allocates nothing and never synchronises: all
 *     work is enqueued on `stream` and the call returns.  Between calls it keeps nothing of the
 *     caller's data; what it does keep per process is set-up it does once (kernel attributes,
 *     the number of CTA pairs a device holds, the driver entry point for tensor maps), the
 *     launch counter behind tsv_kernel_launches(), the number that tsv_set_wait_tries() gave,
 *     and for tree_verify_attn_static the address of its built-in array.
 *   - Stream order: the calls of a layer run in the order given above on one stream.  The kernels are
 *     launched as programmatic dependents; those of branch_state_build and accept_and_refresh wait for
 *     all earlier work before they do anything (tree_verify_layer begins with branch_state_build's).  Some kernels of
 *     tree_verify_attn start earlier: the part
 *     of them that reads only the call's inputs (tsv_nodes, the committed tsv_cache) may run before the kernel before them
 *     has finished, and that part already writes the call's workspace, topk_idx and status; they wait for
 *     it before they read anything the library's own kernels write.  For the caller this matters in one
 *     case only: a kernel of the caller's that is enqueued directly before tree_verify_attn and itself
 *     signals its dependents early (griddepcontrol.launch_dependents /
 *     cudaTriggerProgrammaticLaunchCompletion) must, before it signals, have written whatever it writes
 *     of that call's inputs and have read whatever it reads of that call's workspace, topk_idx and
 *     status.  Kernels that do not use that feature are complete before any of the library's kernels
 *     starts, as always.
 *   - "storage dtype" = tsv_shape.dtype (fp32 or bf16): all vectors and cache rows.  All
 *     partial-block accumulators, gates and weights are fp32.
 *   - Row-major, innermost dimension contiguous, no padding.  Vector pointers must be
 *     16-byte aligned and d, di multiples of 8.
 *   - Cache buffers (csa_kv, csa_ik, hca_kv, win_kv) must hold finite numbers in EVERY allocated
 *     row, also in rows not committed yet (allocate them zero-filled): the tensor-core kernels
 *     fetch whole 32-row boxes and multiply the unused rows by an exact zero weight.
 *   - Node n of sequence b sits at depth delta_n (root = node 0 = depth 0) and at position
 *     p_n = L[b] + delta_n.  n_csa = L / m_csa and n_hca = L / m_hca committed entries.
 *   - Return value: 0 or a negative TSV_ERR_* for problems the host can see BEFORE any
 *     launch (nothing is enqueued then: argument checks, and on the tensor-core path the tensor maps
 *     and the attributes of its kernels, all precede the first launch).  Only TSV_ERR_CUDA out of a
 *     kernel launch itself, or out of a later kernel's attributes, can leave earlier kernels of the same call
 *     enqueued; skip accept_and_refresh for that cycle then.  Problems only the device can see (bad parent
 *     array, node count, capacity, length) are reported per sequence in `status[b]`
 *     (bit-or of TSV_ST_*): that sequence's outputs are zero-filled and
 *     accept_and_refresh commits nothing for it (L unchanged).  `status` is or-ed into, never
 *     cleared: zero it at the start of a cycle
 *     (or let tree_verify_layer of the first layer do it).  No kernel traps or waits without a bound.
 */
#ifndef TSV_H_
#define TSV_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define TSV_MAX_D 32          /* tree nodes per sequence the ABI can express (32-bit ancestor masks) */

enum { TSV_FP32 = 0, TSV_BF16 = 1 };

enum {
  TSV_OK = 0,
  TSV_ERR_NULL = -1,          /* a required pointer is NULL                                */
  TSV_ERR_ALIGN = -2,         /* a vector pointer is not 16-byte aligned                   */
  TSV_ERR_SHAPE = -3,         /* unsupported shape (see tsv_shape)                         */
  TSV_ERR_WORKSPACE = -4,     /* workspace NULL/too small/misaligned                       */
  TSV_ERR_CUDA = -5,          /* a CUDA runtime call failed (launch configuration etc.)    */
  TSV_ERR_LIMIT = -6          /* size beyond a built-in maximum of this entry point        */
};

enum {                         /* per-sequence status bits, device-written */
  TSV_ST_NODES = 1,           /* n_nodes[b] outside 1..D                                   */
  TSV_ST_PARENT = 2,          /* parent[0] != -1 or parent[n] outside [0, n)               */
  TSV_ST_LENGTH = 4,          /* L[b] < 0 or L[b] + D > max_L                              */
  TSV_ST_CSA_CAP = 8,         /* csa_cap[b] < (L + D) / m_csa                              */
  TSV_ST_HCA_CAP = 16,        /* hca_cap[b] < (L + D) / m_hca                              */
  TSV_ST_INTERNAL = 32,       /* a bounded wait inside a kernel gave up                    */
  TSV_ST_PAGE = 64,           /* a page-table entry, slot or reference count that the call needs is not valid */
  TSV_ST_POOL = 128           /* the pool has too few free pages                           */
};

enum {                         /* tsv_shape.flags */
  TSV_FLAG_FORCE_SIMT = 1,    /* tree_verify_attn: use the CUDA-core kernels even where the
                                  tensor-core kernels apply                                 */
  TSV_FLAG_HCA_DEFERRED = 2   /* C128-deferred refresh schedule (Section "Performance Optimization": C4 is refreshed
                                  timely, C128 writes are delayed and combined once the accepted path is known).
                                  For a sequence in which no HCA block can close inside the tree
                                  ((L % m_hca) + D < m_hca), branch_state_build builds no HCA branch states: the
                                  scratch fields hca_mx, hca_s, hca_acc_kv and new_hca_kv of that sequence are left
                                  untouched (hca_done is written, all 0), and accept_and_refresh folds the accepted
                                  path's (g_hca, c_hca) into the persistent open HCA block itself, in path order, with
                                  the arithmetic of branch_state_build -- the committed state is bit-identical to the
                                  timely schedule's.  Sequences in which a block may close inside the tree take the
                                  timely path.  Give the same flag to all three calls of a cycle.               */
};

/* Problem shape; HOST memory.
 * Supported: 1 <= D <= 32, window >= D, d and di multiples of 8 (d <= 1024, di <= 512),
 * H <= 256, HI <= 16, m_csa >= 1, m_hca >= 1, topk >= 1.  */
typedef struct tsv_shape {
  int32_t dtype;              /* TSV_FP32 | TSV_BF16                                        */
  int32_t B;                  /* sequences                                                  */
  int32_t D;                  /* node slots per sequence (verification budget, root incl.)  */
  int32_t H;                  /* query heads; one shared KV head (key == value)             */
  int32_t d;                  /* KV dim                                                     */
  int32_t m_csa, topk;        /* CSA block length; entries selected per node                */
  int32_t HI, di;             /* indexer heads x dim                                        */
  int32_t m_hca;              /* HCA block length                                           */
  int32_t window;             /* uncompressed window: query at p sees positions p-w+1 .. p  */
  float sm_scale;             /* softmax scale; <= 0 means 1/sqrt(d)                        */
  int64_t max_L;              /* bound on L[b] + D for every sequence; sizes grids/workspace */
  int32_t flags;              /* TSV_FLAG_*                                                 */
  int32_t reserved;
} tsv_shape;

/* Persistent state of ONE layer for all B sequences -- the committed prefix.
 * Read-only for branch_state_build / tree_verify_attn; written by accept_and_refresh only. */
typedef struct tsv_cache {
  int32_t *L;                 /* [B] committed tokens                                       */
  void *csa_kv;               /* CSA entries, rows of d;  sequence b owns rows               */
  void *csa_ik;               /*   csa_row0[b] .. csa_row0[b] + csa_cap[b]; same rows of di */
  const int64_t *csa_row0;    /* [B]                                                        */
  const int32_t *csa_cap;     /* [B] rows reserved                                          */
  void *hca_kv;               /* HCA entries, rows of d                                     */
  const int64_t *hca_row0;    /* [B]                                                        */
  const int32_t *hca_cap;     /* [B]                                                        */
  void *win_kv;               /* [B][window][d] ring of uncompressed KV, slot = pos % window */
  float *csa_mx, *csa_s;      /* [B] open CSA block: running max gate, sum of weights       */
  float *csa_acc_kv;          /* [B][d]  weighted sum of compression vectors                */
  float *csa_acc_ik;          /* [B][di] weighted sum of indexer-key vectors                */
  float *hca_mx, *hca_s;      /* [B] open HCA block                                         */
  float *hca_acc_kv;          /* [B][d]                                                     */
  int64_t csa_rows;           /* HOST value: rows allocated in csa_kv / csa_ik (all slabs); the tensor-core attention
                               * path builds its tensor maps from it: with 0 ("unknown") every shape runs on the
                               * CUDA-core path                                               */
  int64_t hca_rows;           /* HOST value: rows allocated in hca_kv (0: a layer without HCA entries) */
  /* Paged pool (Section "Temporary Branch States and Compressed-State Handling": a page-based pool seen as one logical
   * layer and several physical layers that share page-level pointers).  With page_table non-NULL the CSA and HCA entries
   * of a sequence do not sit in one slab each: logical page lp holds the entries of tokens [lp, lp + 1) * page_tokens, and
   * ONE table gives its physical page for every physical layer: entry e of the CSA cache (kv and indexer key) is row
   *     page_table[b][e / epp] * epp + e % epp,   epp = page_tokens / m_csa,
   * entry h of the HCA cache is row  page_table[b][h / hpp] * hpp + h % hpp,  hpp = page_tokens / m_hca.
   * The third physical layer is the token-level KV: win_kv is then not a ring but a pool of tok_rows rows, the KV of the
   * token at position p in row  page_table[b][p / page_tokens] * page_tokens + p % page_tokens  (only the last `window`
   * positions of a sequence are ever read; the refresh writes position L + i of every accepted node).
   * csa_row0 / hca_row0 are ignored then (may be NULL); csa_cap / hca_cap still give the entries the sequence's assigned
   * pages can hold, and the pages must cover positions up to L + D - 1.  page_tokens must be a multiple of m_csa and of
   * m_hca.  The tensor-core path fetches rows by 32-row TMA boxes where a page holds whole boxes of the layer (CSA: epp a
   * multiple of 32, e.g. 128-token pages with m_csa = 4: one box per page; window: page_tokens a multiple of 32); otherwise,
   * and for HCA rows beyond the first 32 entries unless hpp is a multiple of 32, it gathers the rows four at a time by
   * index. */
  const int32_t *page_table;  /* [B][max_pages] device, or NULL: flat slabs and window ring   */
  int32_t page_tokens;        /* HOST value                                                 */
  int32_t max_pages;          /* HOST value: columns of page_table                          */
  int64_t tok_rows;           /* HOST value: rows allocated in win_kv when it is a token pool */
} tsv_cache;

/* Per-cycle inputs of ONE layer for all tree nodes; read-only. */
typedef struct tsv_nodes {
  const void *q;              /* [B][D][H][d]   queries                                     */
  const void *kv;             /* [B][D][d]      the node's own uncompressed KV              */
  const void *c_csa;          /* [B][D][d]      CSA compression vector                      */
  const void *ikc;            /* [B][D][di]     CSA indexer-key compression vector          */
  const float *g_csa;         /* [B][D]         CSA gate logit                              */
  const void *c_hca;          /* [B][D][d]      HCA compression vector                      */
  const float *g_hca;         /* [B][D]         HCA gate logit                              */
  const void *iq;             /* [B][D][HI][di] indexer queries                             */
  const float *iw;            /* [B][D][HI]     indexer head weights                        */
  const int32_t *parent;      /* [B][D] parent[0] = -1, 0 <= parent[n] < n                  */
  const int32_t *n_nodes;     /* [B] 1..D; slots >= n_nodes[b] are padding                  */
} tsv_nodes;

/* Scratch pad of ONE layer: branch-private temporary state, written by branch_state_build,
 * read by tree_verify_attn and accept_and_refresh, dead afterwards. */
typedef struct tsv_scratch {
  float *csa_mx, *csa_s;      /* [B][D]  state of the open CSA block after node n           */
  float *csa_acc_kv;          /* [B][D][d]                                                  */
  float *csa_acc_ik;          /* [B][D][di]                                                 */
  float *hca_mx, *hca_s;      /* [B][D]                                                     */
  float *hca_acc_kv;          /* [B][D][d]                                                  */
  void *new_csa_kv;           /* [B][D][d]  entry closed at node n (valid where csa_done)   */
  void *new_csa_ik;           /* [B][D][di]                                                 */
  void *new_hca_kv;           /* [B][D][d]  (valid where hca_done)                          */
  uint8_t *csa_done;          /* [B][D] 1 iff (p_n + 1) % m_csa == 0                         */
  uint8_t *hca_done;          /* [B][D]                                                     */
} tsv_scratch;

/* Library version (major * 1000 + minor). */
int tsv_version(void);

/* Kernels this library has launched in this process so far (monotonic counter; reporting only). */
uint64_t tsv_kernel_launches(void);

/* How often the waits inside the token-level and page kernels (second half of this file) try before they give up, in launches
 * from now on; negative: their usual numbers, which stand unless this is called.  For tests of what a caller does then
 * (TSV_ST_INTERNAL).  Always TSV_OK. */
int tsv_set_wait_tries(int64_t tries);

/* Text for a TSV_ERR_* code; static storage. */
const char *tsv_error_string(int code);

/* Bytes of `workspace` tree_verify_attn needs for this shape (uses max_L).  0 on bad shape. */
size_t tsv_workspace_bytes(const tsv_shape *shape);

/*
 * branch_state_build -- temporary state isolation (Sections "Three-Stage Speculative Forward":
 * chains sharing a prefix reuse its state but compress independently after branching;
 * "Temporary Branch States and Compressed-State Handling": chain-private compressed tokens and
 * compression-intermediate buffers live in a scratch pad).
 *
 * For every node, in parent-before-child order: take the open-block state of the parent (the
 * root takes the persistent one), fold the node's (gate, compression vectors) into it by the
 * online softmax-pooling update  mx' = max(mx, g); s' = s e^{mx-mx'} + e^{g-mx'};
 * acc' = acc e^{mx-mx'} + e^{g-mx'} c  (an open block with p_n % m == 0 tokens is empty and its
 * stored numbers are ignored).  A node with (p_n + 1) % m == 0 closes the block: the entry
 * acc'/s' is rounded to the storage dtype into new_*[b][n], done[b][n] = 1 and the node's
 * state becomes empty (zeros).  Done for the CSA cache (kv entry + indexer key, same weights)
 * and the HCA cache.  Padding nodes get zero state and done = 0.  `cache` is not written.
 */
int branch_state_build(const tsv_shape *shape, const tsv_cache *cache, const tsv_nodes *nodes,
                       const tsv_scratch *scratch, int32_t *status /* [B] device */, void *stream);

/*
 * tree_verify_attn -- branch-aware causal verification (Section "Branch-Aware Causal Verification
 * and Isolation": a candidate attends to the accepted context and to the ancestors on its own
 * branch, never to other branches, whatever the physical order of the nodes).
 *
 * For node n and head h:  out = sum_j softmax_j(sm_scale q.K_j) K_j  with ONE softmax over
 *   (a) the top-k CSA entries by indexer score  sum_hi iw relu(iq . ik_e)  among the n_csa
 *       committed entries plus the entries closed inside the tree at strict ancestors of n
 *       (k_eff = min(topk, #candidates); ties to the lower block index),
 *   (b) all n_hca committed HCA entries plus those closed at strict ancestors,
 *   (c) the committed window positions max(0, p_n - w + 1) .. L-1,
 *   (d) the KV of n itself and of its ancestors.
 * out       [B][D][H][d] storage dtype; zero for padding nodes and flagged sequences.
 * topk_idx  [B][D][topk] int32 or NULL: ascending logical block indices of (a), -1 padded;
 *           index >= n_csa names the entry closed at the ancestor whose position lies in it.
 * workspace device, 256-byte aligned, >= tsv_workspace_bytes(shape); contents are scratch.
 * Needs `scratch` as written by branch_state_build of the same layer and cycle.
 */
int tree_verify_attn(const tsv_shape *shape, const tsv_cache *cache, const tsv_nodes *nodes,
                     const tsv_scratch *scratch, void *out, int32_t *topk_idx,
                     void *workspace, size_t workspace_bytes, int32_t *status, void *stream);

/*
 * tree_verify_layer -- branch_state_build and then tree_verify_attn of one layer in one call: the call of a model's layer.
 * Arguments, results and status handling are theirs; and what the two calls cannot know of each other is used: on the
 * tensor-core path the state build leaves the entries closed inside the tree in `workspace` as the attention reads them too.
 * first     non-zero for the first layer of a cycle: `status` is written (0 for a usable sequence) instead of or-ed into, so
 *           that the caller need not zero it.
 */
int tree_verify_layer(const tsv_shape *shape, const tsv_cache *cache, const tsv_nodes *nodes,
                      const tsv_scratch *scratch, void *out, int32_t *topk_idx,
                      void *workspace, size_t workspace_bytes, int32_t first, int32_t *status, void *stream);

/*
 * accept_and_refresh -- accepted-path state refresh (Sections "Compressed-State Consistency and
 * Accepted-Path Refresh" and "Temporary Branch States and Compressed-State Handling": select a
 * specific path, keep its token-level KV, its completed CSA/HCA entries and its
 * compression-intermediate buffers, drop every rejected branch).
 *
 * Walk: cur = 0, path = [0]; repeat: c = lowest-index child of cur with
 * draft_tok[c] == target_tok[cur]; stop if none; append c.  Then, for every layer and
 * i < accept_len with n = path[i]: win_kv[(L+i) % window] = kv[n]; entries closed at n are
 * appended at rows (L+i)/m_csa and (L+i)/m_hca; the persistent open-block states become the
 * scratch states of the last accepted node; L += accept_len.
 * caches / nodes / scratch: HOST arrays of n_layers HOST pointers to the per-layer structs
 * (parent and n_nodes are read from nodes[0]).  Tokens are [B][D] int32.
 * accept_len [B], accept_path [B][D] (-1 padded), bonus_tok [B] (= target at the last accepted
 * node): device outputs.  A sequence with status[b] != 0 (on entry or found here, over ALL
 * layers) commits nothing in any layer and reports accept_len 0.
 */
int accept_and_refresh(const tsv_shape *shape, int32_t n_layers, const tsv_cache *const *caches,
                       const tsv_nodes *const *nodes, const tsv_scratch *const *scratch,
                       const int32_t *draft_tok, const int32_t *target_tok, int32_t *accept_len,
                       int32_t *accept_path, int32_t *bonus_tok, int32_t *status, void *stream);

/*
 * tree_verify_attn_static -- tree_verify_attn without a caller-provided workspace.
 * (No counterpart in the paper: this is a convenience of this library.)
 *
 * For callers that cannot allocate device memory at the point of the call -- an engine that
 * gives out all device memory from its own pool at start-up, a plug-in that must leave its
 * host's allocator alone, a request loop where an allocation would stall the device.  The
 * workspace lives in a device array of TSV_STATIC_WORKSPACE_BYTES built into the library
 * (each GPU that loads the library holds that much until the process exits).  The call runs
 * no cudaMalloc / cudaFree and no allocating library routine; inputs and outputs are still the
 * caller's.  Arguments, results and status handling are those of tree_verify_attn.
 *   - Shapes whose tsv_workspace_bytes() exceeds TSV_STATIC_WORKSPACE_BYTES are refused with
 *     TSV_ERR_LIMIT and nothing is enqueued.
 *   - The first call on each device looks up the array's device address (with that device
 *     current); that look-up makes the runtime load the library's device code on the device,
 *     which is when the array's bytes are reserved there.  Make that first call at start-up:
 *     before the rest of the device memory is handed out, and before starting any stream capture.
 *     If it fails (TSV_ERR_CUDA), nothing was enqueued and no error is left pending.
 *   - All calls on a device share the one array, which keeps whatever the last call left in
 *     it.  Nothing in it has to start at zero -- every region is written before it is read
 *     within a call -- but two calls that overlap on the GPU (different streams, no
 *     dependency between them) race on it: order them.
 */
#define TSV_STATIC_WORKSPACE_BYTES (16u << 20)
int tree_verify_attn_static(const tsv_shape *shape, const tsv_cache *cache, const tsv_nodes *nodes,
                            const tsv_scratch *scratch, void *out, int32_t *topk_idx,
                            int32_t *status, void *stream);

/* ======================================================================================================================
 * Token-level layers: the operators of a layer that attends to tokens, not to compressed entries -- the sliding-window
 * layers that draft (Section "Three-Stage Speculative Forward": draft extend, draft decode) and every layer's window.
 *
 *     qk_norm_rope(new tokens)  ->  window_sink_attn(new tokens over the token cache)  ->  token_commit
 *
 * Conventions of the calls above hold: device pointers, host structs, no allocation, no synchronisation, 16-byte aligned
 * vectors, negative codes before any launch, `status[b]` or-ed into for what only the device can see.  Two calls on
 * different streams may overlap if they share no buffer that one of them writes (the workspace is one).
 *
 * New tokens are PACKED: those of sequence b are rows row0[b] .. row0[b] + n[b] - 1 of every [rows][...] array, in order
 * of their positions (a chain: token i is at position L[b] + i) or, with `parent`, as the nodes of a draft tree (node i is
 * at L[b] + its depth; parent before child).  n[b] may be 0; the ranges of two sequences must not overlap.  Rows of no
 * sequence are not written and have no influence; with rows = 0 the arrays may be NULL.  What the device finds wrong
 * with a sequence:
 *   TSV_ST_NODES     n[b] outside 0..max_n, or rows outside 0..rows: it counts as a sequence without rows, so what it names
 *                    as its output rows is left as it was
 *   TSV_ST_LENGTH    L[b] < 0 or L[b] + n[b] > max_L: zeros in its output rows (without rows only token_commit flags it)
 *   TSV_ST_PARENT    a bad parent array, or a tree of more than TSV_MAX_D nodes: zeros in its output rows.  token_commit
 *                    does not look at parents: `path` says what it takes, and status[b] of the calls before stops it
 *   TSV_ST_INTERNAL  a wait gave up (window_sink_attn sets it for all sequences of the call): output rows hold anything
 * A sequence with one of them commits nothing (TSV_ST_INTERNAL of a commit: L stays, cache rows behind it may be written).
 * Sums are fp32: a score q.k that is beyond its range counts as infinite, a weight below 2^-125 of the row's largest as zero.
 * ====================================================================================================================== */

/* HOST memory.  Supported: B <= 2^20, H a multiple of Hk, H <= 256, d a multiple of 8, 8 <= d <= 512, window >= 1, n_sink >= 0. */
typedef struct tsv_tok_shape {
  int32_t dtype;              /* TSV_FP32 | TSV_BF16                                        */
  int32_t B;                  /* sequences                                                  */
  int32_t H, Hk, d;           /* query heads, key/value heads (query head h reads h / (H / Hk)), head dim */
  int32_t window;             /* a query at position p sees p - window + 1 .. p ...         */
  int32_t n_sink;             /* ... and the first positions 0 .. n_sink - 1 (up to p)      */
  int32_t max_n;              /* bound on n[b], at most 2^22                                */
  int64_t max_L;              /* bound on L[b] + n[b], at most 2^30                          */
  float sm_scale;             /* softmax scale; <= 0 means 1/sqrt(d)                        */
  int32_t reserved;
} tsv_tok_shape;

/* Token-level keys and values of ONE layer.  Rows of Hk * d elements, one per token; the row of position pos of sequence b is
 *   ring (page_table NULL):  b * (n_sink + window) + (pos < n_sink ? pos : n_sink + (pos - n_sink) % window)
 *   pages:                   page_table[b][pos / page_tokens] * page_tokens + pos % page_tokens
 * With n_sink = 0 and the layer's window these are win_kv of tsv_cache, ring or token pool (v = NULL), for window_sink_attn
 * only: token_commit would move L without the layer's compressed entries and open blocks, which accept_and_refresh moves
 * with it.  Pages that hold no visible position may be missing (-1): a window layer can give back what lies between its
 * sinks and its window.  Rows that are not visible may
 * hold anything, also infinities and NaN. */
typedef struct tsv_tok_cache {
  int32_t *L;                 /* [B] committed tokens                                       */
  void *k;
  void *v;                    /* NULL: the keys are the values                              */
  int64_t rows;               /* HOST value: rows allocated in k (and v)                    */
  const int32_t *page_table;  /* [B][max_pages] or NULL: ring                               */
  int32_t page_tokens, max_pages;
} tsv_tok_cache;

typedef struct tsv_tok_batch {
  const int64_t *row0;        /* [B]                                                        */
  const int32_t *n;           /* [B]                                                        */
  const int32_t *parent;      /* [rows] node of the same sequence, -1 for node 0; or NULL: chains */
  int64_t rows;               /* HOST value: rows of the packed arrays                      */
} tsv_tok_batch;

/* Vectors of the new tokens: token row r starts at element r * ld, its heads follow each other.  ld >= heads * d, a multiple
 * of 8 (bf16) or 4 (fp32) elements: so q, k and v may be column ranges of one fused projection. */
typedef struct tsv_tok_rows {
  const void *q, *k, *v;
  int64_t q_ld, k_ld, v_ld;
} tsv_tok_rows;

/*
 * qk_norm_rope -- for every head of q and k of every new token, x / sqrt(mean(x^2) + eps) * w (wq, wk: [d] fp32, NULL: 1),
 * and then dims first .. first + rot - 1 turned by angle_i = position * inv_freq[i], i < rot / 2 (fp32 frequencies; the
 * product and its reduction in 64 bits), (a, b) -> (a cos - b sin, a sin + b cos) over the pairs
 *   pairs = 0:  a = x[first + i],     b = x[first + rot / 2 + i]
 *   pairs = 1:  a = x[first + 2 i],   b = x[first + 2 i + 1].
 * rot is 0 or a multiple of 16, first a multiple of 8, first + rot <= d.  in->q or in->k may be NULL (that part is left
 * out; not both).  q_out, k_out: rows of ldq, ldk elements; each may be its input (same address and stride), and shares no
 * other element with the inputs or the other output (TSV_ERR_SHAPE; rows of one stride may lie between each other's).
 * L [B] is read only.  in->v is not used.
 */
int qk_norm_rope(const tsv_tok_shape *shape, const int32_t *L, const tsv_tok_batch *batch, const tsv_tok_rows *in,
                 const float *wq, const float *wk, float eps, const float *inv_freq, int32_t rot, int32_t first, int32_t pairs,
                 void *q_out, int64_t ldq, void *k_out, int64_t ldk, int32_t *status, void *stream);

/* Bytes of `workspace` window_sink_attn needs for this shape and number of packed rows.  0 on bad shape; never 0 else. */
size_t tsv_tok_workspace_bytes(const tsv_tok_shape *shape, int64_t rows);

/*
 * window_sink_attn -- out [rows][H][d] (storage dtype, packed like the queries, no padding):
 *   out = sum_j softmax_j(sm_scale q.k_j) v_j  over the positions j <= p with j > p - window or j < n_sink,
 * where the committed positions j < L[b] come from the cache and the others from the rows `in` of the call (in->v NULL iff
 * cache->v is: the keys are the values).  In a tree a node sees, of the new tokens, itself and its ancestors, under the same
 * window.  The cache is not written.  What a query may not see has no influence on its result, also if it is not finite.
 * A page that a query needs and that is not one of the pool's (-1, beyond `rows`, or a position beyond max_pages) is left
 * out, and the sequence flagged TSV_ST_PAGE.  `out` must not overlap the rows of `in` (TSV_ERR_SHAPE): a result that is not
 * finite has them read once more.
 */
int window_sink_attn(const tsv_tok_shape *shape, const tsv_tok_cache *cache, const tsv_tok_batch *batch, const tsv_tok_rows *in,
                     void *out, void *workspace, size_t workspace_bytes, int32_t *status, void *stream);

/*
 * token_commit -- rows of new tokens become committed: count[b] of them (NULL: n[b]), the i-th being node path[b][i] (path:
 * [B][path_ld] int32, e.g. accept_path of accept_and_refresh; NULL: node i), into the cache rows of positions L[b] + i; then
 * L[b] += count.  A sequence with status[b] != 0, on entry or found here (count outside 0..n[b] or beyond path_ld, a node
 * outside 0..n[b] - 1: TSV_ST_NODES; a missing page: TSV_ST_PAGE), commits nothing.
 */
int token_commit(const tsv_tok_shape *shape, const tsv_tok_cache *cache, const tsv_tok_batch *batch, const tsv_tok_rows *in,
                 const int32_t *path, int32_t path_ld, const int32_t *count, int32_t *status, void *stream);

/* ======================================================================================================================
 * Pages of a paged pool: who holds them, and their contents.
 * The pool has n_pages pages; `ref[p]` counts the sequences whose table row names page p (0: free).  A PLANE is an array with
 * a fixed number of bytes per page (csa_kv, csa_ik, hca_kv, win_kv of every layer; k, v of a token cache): all planes are
 * addressed by the same table.  A ROW array has a fixed number of bytes per sequence slot (L, capacities, the open-block
 * states of every layer; a ring).  Fresh pages are always the free ones with the lowest numbers, in ascending order.
 * The lists of a call (n entries, at most TSV_MAX_PAGE_LIST) are device arrays; `status[i]` belongs to entry i.
 * Calls on one pool must be ordered (one stream).
 * ====================================================================================================================== */
#define TSV_MAX_PAGE_LIST 1024

typedef struct tsv_page_array {
  void *base;                 /* 16-byte aligned (planes), 4-byte aligned (rows)            */
  int64_t bytes;              /* of a page (multiple of 16) or of a slot (multiple of 4)    */
} tsv_page_array;

typedef struct tsv_page_pool {
  int32_t *page_table;        /* [slots][max_pages]; -1: no page                            */
  int32_t *ref;               /* [n_pages]                                                  */
  int32_t slots, max_pages, n_pages, page_tokens;
  const tsv_page_array *planes;   /* HOST array, n_planes entries                           */
  const tsv_page_array *rows;     /* HOST array, n_rows entries                             */
  int32_t n_planes, n_rows;
} tsv_page_pool;

/* Bytes of `workspace` that pages_assign, pages_fork and pages_compact need for this pool.  0 on a bad pool. */
size_t tsv_pages_workspace_bytes(const tsv_page_pool *pool);

/* pages_assign -- logical pages first[i] .. last[i] - 1 of slot[i] that have no page get fresh ones: entries in order, logical
 * pages ascending.  An entry for which too few pages are left gets none (TSV_ST_POOL; later entries still may). A slot may
 * occur once. */
int pages_assign(const tsv_page_pool *pool, int32_t n, const int32_t *slot, const int32_t *first, const int32_t *last, void *workspace,
                 size_t workspace_bytes, int32_t *status, void *stream);

/* pages_free -- slot[i] gives up its logical pages first[i] .. last[i] - 1 (those that it has); their contents stay until
 * another sequence gets them.  A slot may occur more than once. */
int pages_free(const tsv_page_pool *pool, int32_t n, const int32_t *slot, const int32_t *first, const int32_t *last, int32_t *status,
               void *stream);

/* pages_fork -- slot dst[i], which holds no pages, becomes a copy of slot src[i] with L[src[i]] committed tokens: its table row
 * names the same pages where those are full (logical pages below L / page_tokens), and fresh ones elsewhere, the contents of
 * the partly filled page copied in every plane; row dst[i] of every row array becomes row src[i].  All entries see the pool as
 * it was before the call; a slot may be src of many, dst of one, and not both (TSV_ST_PAGE).  Where too few pages are left
 * the entry changes nothing (TSV_ST_POOL; later entries still may).  L [slots] may be one of the row arrays. */
int pages_fork(const tsv_page_pool *pool, int32_t n, const int32_t *src, const int32_t *dst, const int32_t *L, void *workspace,
               size_t workspace_bytes, int32_t *status, void *stream);

/* pages_compact -- the used pages move to the numbers 0 .. n_used - 1: the page with the i-th lowest number >= n_used to the
 * i-th lowest free number, in every plane, the table and the counts with it.  n_used: device, 1 value, written (-1: a bounded wait
 * inside a kernel gave up, and contents are lost). */
int pages_compact(const tsv_page_pool *pool, int32_t *n_used, void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* TSV_H_ */
