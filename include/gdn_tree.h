/*
 * gdn_tree.h -- C ABI of libgdntree: rollback-free verification of a draft
 * token tree through one Gated DeltaNet (GDN) layer on AMD Instinct MI355X
 * (gfx950).
 *
 * Method: "Trees from Marginals", Sec. 3.4.  Every tree node's output is the
 * gated delta rule (Eq. 7) applied along that node's own root-to-node path,
 * starting from the cached per-sequence state S0, followed by the readout of
 * Eq. 8.  Verification only reads the cached state and conv state; the
 * state changes in one place per decode step, the commit, which runs Eq. 7
 * over the accepted node's path once that node has been chosen (Sec. 3.4.2).
 * The tree metadata (depths, a topological order, proper-ancestor bitmasks)
 * is computed once per decode step from the parent pointers and can be
 * shared by every GDN layer of the step (Sec. 3.4.2).
 *
 * Which entry point takes which tree size: gdn_tree_prepare, gdn_tree_commit,
 * gdn_tree_verify, gdn_tree_verify_noalloc, gdn_tree_verify_chunked and
 * gdn_tree_step all accept 1 <= T <= GDN_MAX_T = 512.  Up to 128 slots verify
 * and step run entirely on chip (step as one fused launch); above 128 they
 * go through a feature workspace (see gdn_tree_verify), and the step shifts
 * the conv state, writes the features and then commits each head's state
 * rows inside the verification launch (heads of dk dv < 512: the commit
 * kernels, then the verification).
 *
 * Conventions shared by all entry points
 * --------------------------------------
 *  * All tensor pointers are DEVICE pointers, contiguous row-major, owned by
 *    the caller.  Work is enqueued on the caller's stream and is ordered with
 *    it; nothing synchronises the host except a workspace allocation (see
 *    Workspaces below).  Pointers must be 16-byte aligned.
 *  * Workspaces.  gdn_tree_verify and gdn_tree_step above 128 slots,
 *    gdn_tree_verify_chunked, gdn_tree_attend and gdn_chain above
 *    GDN_CHAIN_STEP_T tokens pass intermediate results through a device buffer that the library allocates on the first call that
 *    needs it and keeps per (device, stream).  A call that needs more gets a
 *    larger buffer (hipMalloc) in its place; one that was handed out is not
 *    released before the process ends, so that a captured graph may go on
 *    using it.  Each is at least twice the one before if memory allows, so
 *    that all buffers of a stream together stay below four times its largest
 *    need.  A call under stream capture that would need a larger buffer
 *    returns GDN_EUNSUPPORTED: run the same sizes once uncaptured on that
 *    stream first.  Several host threads may make calls on one stream:
 *    the kernels of each such call are enqueued together.
 *    hipStreamPerThread has a buffer for every thread that uses it.
 *    A captured graph works in the buffer of the stream it was captured on,
 *    whichever stream replays it: it must not run at the same time as other
 *    such calls of that stream, or as another graph captured there.  Graphs
 *    that are to run side by side are captured on streams of their own.
 *  * Recurrence orientation: the stored state of (sequence b, value head h) is
 *    S[b][h] in R^{dv x dk} (dk contiguous), the transpose of the paper's
 *    S in R^{dk x dv}; one step is S <- alpha S (I - beta k k^T) + beta v k^T
 *    and the readout is o = scale * S q (Eq. 7-8).
 *  * Short convolution (width 4, depthwise, no bias) and activation: the raw
 *    inputs of node t are the C = 2 Hk dk + Hv dv channels
 *    x_t = [q_t (Hk heads) | k_t (Hk heads) | v_t (Hv heads)].  For a node i
 *    at depth d with path p_0 = root, ..., p_d = i:
 *        y_i[c] = SiLU( sum_{w=0..3} conv_w[c][w] * x_{p_{d-3+w}}[c] ),
 *    where a tap above the root (d-3+w < 0) reads conv_state[b][d+w][c]
 *    (slot 2 = most recent committed token, slot 0 = oldest).  q and k are
 *    then L2-normalised per head: x / sqrt(sum x^2 + 1e-6).  v is not.
 *  * GQA: value head h reads key head floor(h * Hk / Hv); Hv % Hk == 0.
 *  * alpha (decay) and beta (write strength) are per value head, in (0, 1].
 *  * Trees: parent[b][i] = -1 for the root, -2 for an absent (padding) slot,
 *    else the parent's slot index.  Node numbering is arbitrary.
 *
 * Errors: every entry point returns gdn_status.  Problems visible on the
 * host (null pointers, unsupported sizes) return an error before any work is
 * enqueued; gdn_last_error() then describes it.  Problems that only the
 * device can see (an invalid tree, an invalid accepted node) are reported per
 * sequence in the status arrays below and the affected sequence is skipped.
 */
#ifndef GDN_TREE_H
#define GDN_TREE_H

#include <stddef.h>
#include <stdint.h>

#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  GDN_OK = 0,
  GDN_EINVAL = -1,       /* null pointer, negative or inconsistent size */
  GDN_EUNSUPPORTED = -2, /* valid but unsupported shape (head dims, T)   */
  GDN_EHIP = -3          /* a HIP launch or attribute call failed        */
} gdn_status;

typedef enum { GDN_F32 = 0, GDN_BF16 = 1 } gdn_dtype;

/* Per-sequence status codes written by prepare (tree) and commit. */
enum {
  GDN_TREE_OK = 0,
  GDN_TREE_NO_ROOT = 1,      /* real nodes but none with parent -1              */
  GDN_TREE_MULTI_ROOT = 2,   /* more than one node with parent -1              */
  GDN_TREE_BAD_PARENT = 3,   /* parent outside {-2,-1,0..T-1}, self, or padding */
  GDN_TREE_CYCLE = 4,        /* a real node whose parent chain misses the root */
  GDN_TREE_BAD_ACCEPTED = 5, /* commit only: accepted outside [-1,T) or padding */
  GDN_KV_BAD_LEN = 6,  /* paged cache: ctx_len or n_new out of range, or no room in the page table */
  GDN_KV_BAD_PAGE = 7, /* paged cache: a needed page-table entry outside [0, n_pages) */
  GDN_KV_BAD_POS = 8,  /* paged cache: a position without a row in the rotation table */
  GDN_CHAIN_BAD_LEN = 9 /* chain: a length outside [0, T], rows outside the tensors or of another sequence */
};

/* Problem sizes.  B sequences, T node slots per tree (padded tree size),
 * Hk key heads, Hv value heads, head dims dk and dv.
 * in_dtype is the element type of q, k, v, alpha and beta (GDN_F32 or
 * GDN_BF16); the state, conv weights, conv state and outputs are fp32.
 * scale multiplies the readout; 0 selects 1/sqrt(dk) (Eq. 8).
 * Supported: dk, dv in {16, 32, 64, 128}; 1 <= T <= GDN_MAX_T; B >= 0. */
typedef struct {
  int32_t B, T, Hk, Hv, dk, dv;
  int32_t in_dtype;
  float scale;
} gdn_dims;

#define GDN_MAX_T 512

/* Size in bytes of the tree-metadata blob for B trees of T slots (host only,
 * no device work).  Layout, W = ceil(T/64); each array starts at the next
 * 16-byte aligned offset after the previous one, in this order:
 *   uint64 anc   [B][T][W]  bit (j mod 64) of word j/64 of anc[b][i] is set
 *                           iff slot j is a proper ancestor of slot i
 *                           (Sec. 3.4.2 bitmask, node-index space)
 *   int32  depth [B][T]     edges to the root; -1 for padding
 *   int32  order [B][T]     canonical topological order: real nodes sorted
 *                           by (depth, index), then padding by index
 *   int32  pos   [B][T]     inverse permutation of order
 *   int32  parent[B][T]     copy of the input parent array
 *   int32  status[B]        GDN_TREE_* code of each tree
 *   int32  nvalid[B]        number of real (non-padding) nodes
 *   int32  pdep  [B][T]     depth of the node at canonical position p
 *                           (depth[order[p]]), -1 for padding
 *   int32  ppos  [B][T]     canonical position of the parent of the node at
 *                           position p (pos[parent[order[p]]]), -1 for the
 *                           root and padding
 * The blob is padded to a multiple of 256 bytes.  A tree with a non-zero
 * status gets depth/pdep/ppos -1, identity order/pos, empty ancestor sets and
 * nvalid 0.  Returns 0 for B <= 0 or T <= 0. */
size_t gdn_tree_meta_bytes(int32_t B, int32_t T);

/* Tree preprocessing (Sec. 3.4.1 topological order and ancestor relation,
 * Sec. 3.4.2 metadata computed once per decode step).
 *   parent      int32 [B][T]   device, read-only
 *   meta        device buffer of gdn_tree_meta_bytes(B, T) bytes, written
 *   tree_status int32 [B]      device, written (may be NULL)
 * Reads only dims->B and dims->T.  One workgroup per tree. */
int gdn_tree_prepare(const gdn_dims* dims, const int32_t* parent, void* meta,
                     int32_t* tree_status, hipStream_t stream);

/* Read-only tree verification (Sec. 3.4: Eq. 7-8 per node along its path).
 * Up to 128 slots everything stays on chip and nothing is allocated; above
 * 128 the post-conv features go through a device workspace of
 * B T (2 C + 4 Hv) bytes (fp16 features, fp32 scales of the value rows;
 * C = 2 Hk dk + Hv dv, the first part rounded up to 256 bytes) and 6 T bytes
 * per tree (its depth-first order, T rounded up to 16) that the library
 * keeps (see Workspaces above).
 *   meta        written by gdn_tree_prepare for the same B, T
 *   q, k        in_dtype [B][T][Hk][dk]   raw (pre-conv) queries / keys
 *   v           in_dtype [B][T][Hv][dv]   raw values
 *   alpha, beta in_dtype [B][T][Hv]
 *   conv_w      fp32 [C][4]               C = 2 Hk dk + Hv dv
 *   conv_state  fp32 [B][3][C]            read-only
 *   S0          fp32 [B][Hv][dv][dk]      read-only cached state
 *   out         fp32 [B][T][Hv][dv]       written: o_i = scale * S_i q_i
 * Rows of padding slots and every row of a sequence whose tree status is
 * non-zero are written as zeros.  conv_state and S0 are never written. */
int gdn_tree_verify(const gdn_dims* dims, const void* meta, const void* q, const void* k,
                    const void* v, const void* alpha, const void* beta, const float* conv_w,
                    const float* conv_state, const float* S0, float* out, hipStream_t stream);

/* gdn_tree_verify for callers that cannot allocate device memory (code
 * under HIP graph capture, serving loops that forbid hipMalloc).  Same
 * arguments, layouts, outputs and errors as gdn_tree_verify, whose kernels
 * it runs; it calls no allocating routine.  Trees of more than 128 slots
 * need the feature workspace of gdn_tree_verify, B T (2 C + 4 Hv) bytes:
 * here it is a static device array of GDN_NOALLOC_SCRATCH_BYTES that the
 * library holds on every device it runs on until the process ends (with 4.5
 * MB for the orders of the trees), and larger problems return
 * GDN_EUNSUPPORTED before any device work.  All
 * calls on one device share that array: calls that overlap in time on one
 * device (different streams, or host threads) race and must be serialized
 * by the caller. */
#define GDN_NOALLOC_SCRATCH_BYTES (64u << 20)
int gdn_tree_verify_noalloc(const gdn_dims* dims, const void* meta, const void* q, const void* k,
                            const void* v, const void* alpha, const void* beta,
                            const float* conv_w, const float* conv_state, const float* S0,
                            float* out, hipStream_t stream);

/* The same verification in the paper's chunked form (Sec. 3.4.1-3.4.2,
 * Eq. 9-13): per (sequence, value head) the interaction matrices X (strict
 * ancestors: decayed key-key products scaled by beta) and Y (ancestors and
 * self: decayed query-key products) are built from Gram products, (I + X) U =
 * beta (V - a K S0^T) is solved by forward substitution over sub-blocks of 32
 * positions (each diagonal block inverted by repeated squaring), and O =
 * scale (a Q S0^T + Y U); the Gram, solve and readout products on bf16
 * MFMA as hi/lo three-product splits (about 16 significant bits), the
 * diagonal-block inverses on fp32 MFMA, features in fp32.  Arguments,
 * layouts, outputs and errors are those of gdn_tree_verify (any supported
 * dk, dv and T).  Needs a workspace of about B (T (C + Hv dv) + 1024 n (2 Hv +
 * (n - 1) Hk)) 4 bytes, n = ceil(T / 32), which the library keeps (see
 * Workspaces above; the pairs of blocks without an ancestor
 * have room in it, too).  Its cost grows with the pairs of 32-slot blocks of
 * which one holds an ancestor of a node of the other; gdn_tree_verify's up to
 * 128 slots with the sum of the path lengths, above with the number of 16-node
 * path chunks of its 16-node tiles. */
int gdn_tree_verify_chunked(const gdn_dims* dims, const void* meta, const void* q, const void* k,
                            const void* v, const void* alpha, const void* beta,
                            const float* conv_w, const float* conv_state, const float* S0,
                            float* out, hipStream_t stream);

/* Commit of the accepted node (Sec. 3.4.2): Eq. 7 is run over the path
 * root..accepted, starting from S, and the result replaces S.
 *   accepted      int32 [B]  accepted slot per sequence, -1 = commit nothing
 *   q, k, v, alpha, beta, conv_w: as for verify (same step's tensors)
 *   conv_state    fp32 [B][3][C]   in/out: replaced by the last 3 raw inputs
 *                 of (old slots 0..2 followed by the path's raw inputs)
 *   S             fp32 [B][Hv][dv][dk]  in/out: state after the path
 *   commit_status int32 [B] (may be NULL): the tree status if non-zero, else
 *                 GDN_TREE_BAD_ACCEPTED for an accepted slot outside [-1, T)
 *                 or naming padding, else 0.
 * Sequences with accepted == -1 or a non-zero commit status are untouched.
 * Enqueues two kernels (state replay, then conv-state shift). */
int gdn_tree_commit(const gdn_dims* dims, const void* meta, const int32_t* accepted,
                    const void* q, const void* k, const void* v, const void* alpha,
                    const void* beta, const float* conv_w, float* conv_state, float* S,
                    int32_t* commit_status, hipStream_t stream);

/* Fused decode step: the commit of the previous step's accepted node
 * (Sec. 3.4.2) followed by the verification of the current tree (Sec. 3.4,
 * Eq. 7-8) against the state it produces, in one launch up to 128 slots
 * (above: conv-state shift, features, then one launch that commits and
 * verifies each head).  Results equal gdn_tree_commit(previous step)
 * followed by gdn_tree_verify(current step) with the committed S and conv
 * state; the committed state is formed in registers and verified against
 * without being read back.
 *   prev_meta      meta of the previous step's tree (same B, T)
 *   prev_accepted  int32 [B]: accepted slot of the previous tree, -1 = none
 *   prev_q, prev_k, prev_v, prev_alpha, prev_beta: the previous step's raw
 *                  inputs (shapes and in_dtype as for verify)
 *   commit_status  int32 [B] (may be NULL): as for gdn_tree_commit
 *   meta, q, k, v, alpha, beta: the current step's tree and raw inputs
 *   conv_w         fp32 [C][4] (one layer: shared by both steps)
 *   conv_state     fp32 [B][3][C]  read-only: conv state before the commit
 *   conv_state_out fp32 [B][3][C]  written: conv state after the commit; must
 *                  not overlap conv_state (checked, GDN_EINVAL)
 *   S              fp32 [B][Hv][dv][dk]  in/out: the state before the commit
 *                  on entry, after it on return
 *   out            fp32 [B][T][Hv][dv]  written: outputs of the current tree
 * A sequence with nothing to commit (prev_accepted -1 or a non-zero commit
 * status) keeps S and gets conv_state_out = conv_state; a sequence whose
 * current tree is invalid still commits and gets zero outputs.  Each
 * (sequence, value head, dv slice) of S is read and written by one
 * workgroup only, so the in-place update is race-free; S must not alias
 * any other argument. */
int gdn_tree_step(const gdn_dims* dims, const void* prev_meta, const int32_t* prev_accepted,
                  const void* prev_q, const void* prev_k, const void* prev_v,
                  const void* prev_alpha, const void* prev_beta, int32_t* commit_status,
                  const void* meta, const void* q, const void* k, const void* v,
                  const void* alpha, const void* beta, const float* conv_w,
                  const float* conv_state, float* conv_state_out, float* S, float* out,
                  hipStream_t stream);

/* ------------------------------------------------------------------------
 * Softmax-attention layers of the same decode step
 *
 * A model with GDN layers has softmax-attention layers between them.  The
 * four calls below take the same trees (the metadata of gdn_tree_prepare)
 * through such a layer and through the sampling that ends the step:
 * gdn_kv_append, gdn_tree_attend, gdn_tree_sample, gdn_tree_accept; then
 * gdn_tree_commit / gdn_tree_step for the GDN layers and gdn_kv_commit for
 * the attention layers take the accepted slot.
 *
 * Paged cache.  A sequence's token at position p (0 = the first token of the
 * prompt) lies in page page_table[b][p / page] at place p % page.  Both
 * caches hold 16-byte packs of x = 16 / element size values:
 *   keys    [n_pages][Hkv][d / x][page][x]   packs along the head dim
 *   values  [n_pages][Hkv][page / x][d][x]   packs along the tokens
 * which are the operands of the matrix instructions as they stand: the keys
 * of a tile are rows of 16 bytes, the values columns of 16 bytes.
 *
 * Cached tokens fill positions 0 .. ctx_len[b] - 1.  Slot i of the current
 * tree is kept at position ctx_len[b] + i until the commit, and has the
 * rotation of position ctx_len[b] + depth(i).
 *
 * meta is the tree metadata, or NULL for a chain: slot i's parent is i - 1,
 * slots 0 .. n_new[b] - 1 are real (n_new NULL: all T).  T = 1 without
 * metadata is plain decoding, a chain of up to GDN_MAX_T tokens a chunk of a
 * prompt.  n_new is refused together with meta (padding slots carry it).
 *
 * A sequence whose tree status is non-zero, or whose ctx_len is negative or
 * leaves no room for its slots (ctx_len + T, or + n_new, above max_pages *
 * page), is skipped: outputs zero, caches untouched.
 * Page-table entries outside [0, n_pages) are never followed. */
typedef struct {
  int32_t B, T;      /* sequences, slots per tree (<= GDN_MAX_T)                 */
  int32_t Hq, Hkv;   /* query heads, key / value heads; Hq % Hkv == 0, query
                      * head h reads key / value head floor(h Hkv / Hq);
                      * T Hq / Hkv <= GDN_MAX_KV_ROWS                            */
  int32_t d;         /* head dim: 32, 64, 128 or 256                             */
  int32_t page;      /* tokens per page: 16, 32, 64, 128 or 256                  */
  int32_t n_pages;   /* pages of each cache                                      */
  int32_t max_pages; /* entries in a sequence's row of the page table            */
  int32_t dtype;     /* GDN_F32 or GDN_BF16: q, k, v, caches and outputs         */
  int32_t rot;       /* leading dims of a head that are rotated: even, 0 .. d    */
  int32_t n_pos;     /* rows of the rotation table                               */
  float scale;       /* of the scores; 0 selects 1 / sqrt(d)                     */
} gdn_attn_dims;

#define GDN_MAX_KV_ROWS (1 << 20) /* query rows of a key / value head */

/* Rotates the step's queries and keys and appends keys and values.
 *   q [B][T][Hq][d], k, v [B][T][Hkv][d]   dtype, the layer's new rows
 *   rope        fp32 [n_pos][rot / 2][2]   cos and sin of every position; the
 *               pair (x[e], x[e + rot / 2]) of a head becomes
 *               (x[e] cos - x[e + rot / 2] sin, x[e + rot / 2] cos + x[e] sin).
 *               May be NULL for rot 0.
 *   ctx_len     int32 [B]; page_table int32 [B][max_pages]
 *   k_cache, v_cache   written at the positions of the real slots
 *   q_out       dtype [B][T][Hq][d]  rotated queries, zero for padding slots;
 *               may be q itself (any other overlap, with k and v too, is
 *               not allowed)
 *   kv_status   int32 [B] (may be NULL): the tree status if non-zero, else
 *               GDN_KV_BAD_LEN, GDN_KV_BAD_POS, GDN_KV_BAD_PAGE (pages of the
 *               real slots) or 0; non-zero sequences are skipped.
 * Two sequences must not share a page that either of them writes. */
int gdn_kv_append(const gdn_attn_dims* dims, const void* meta, const int32_t* n_new, const void* q,
                  const void* k, const void* v, const float* rope, const int32_t* ctx_len,
                  const int32_t* page_table, void* k_cache, void* v_cache, void* q_out,
                  int32_t* kv_status, hipStream_t stream);

/* Attention of every slot over the cached tokens, its ancestors and itself:
 *   o_i = sum_j p_ij v_j,  p_ij = softmax_j(scale q_i . k_j)
 *   q    dtype [B][T][Hq][d]   rotated queries (gdn_kv_append's q_out)
 *   out  dtype [B][T][Hq][d]   written; zero for padding slots.  Must not
 *        overlap q.
 * Reads the rows that gdn_kv_append wrote.  Softmax statistics and sums are
 * fp32; with bf16 the weights p enter the second product rounded to bf16.
 * Keys of a page whose entry is outside [0, n_pages) are left out.  A row of
 * a slot that is not visible to a query does not reach it, whatever it holds
 * (infinities and NaN included), nor do cache rows past the last slot.
 * Work is split over the cached length, at one token too; the parts are
 * joined through a workspace that the library keeps (see Workspaces above),
 * 2 S Hkv T (Hq / Hkv) (d + 2) 4 bytes for S splits: about 2 MB for one token
 * and 68 MB for 16 trees of 128 slots, 32 + 8 heads of 128. */
int gdn_tree_attend(const gdn_attn_dims* dims, const void* meta, const int32_t* n_new, const void* q,
                    const void* k_cache, const void* v_cache, const int32_t* page_table,
                    const int32_t* ctx_len, void* out, hipStream_t stream);

/* Moves the rows of the accepted path root..accepted to positions
 * ctx_len[b] .. ctx_len[b] + depth(accepted), in place.
 *   accepted   int32 [B]   accepted slot, -1 = nothing
 *   new_len    int32 [B]   written: ctx_len + depth(accepted) + 1, or ctx_len
 *              of a sequence that commits nothing; must not overlap ctx_len
 *              or accepted
 *   kv_status  int32 [B] (may be NULL): the tree status if non-zero, else
 *              GDN_TREE_BAD_ACCEPTED, GDN_KV_BAD_LEN, GDN_KV_BAD_PAGE (pages
 *              of the path's rows, before and after) or 0; non-zero sequences
 *              are left as they are.
 * Without metadata (a chain) every row is in place already and only new_len
 * is written; the page table then needs room up to the accepted slot. */
int gdn_kv_commit(const gdn_attn_dims* dims, const void* meta, const int32_t* accepted,
                  const int32_t* page_table, const int32_t* ctx_len, void* k_cache, void* v_cache,
                  int32_t* new_len, int32_t* kv_status, hipStream_t stream);

/* Problem sizes of gdn_tree_sample.  ld: elements from one row of logits to
 * the next, 0 selects V.  1 <= V <= GDN_MAX_V. */
typedef struct {
  int32_t B, T, V;
  int32_t dtype; /* GDN_F32 or GDN_BF16: logits */
  int64_t ld;
} gdn_sample_dims;

#define GDN_MAX_V (1 << 20)

/* Samples one token per slot from its logits with a given random number.
 *   meta        tree metadata or NULL (all slots real); a padding slot and a
 *               sequence with a non-zero tree status get token -1, and their
 *               logits are not read
 *   logits      dtype [B][T][ld]
 *   temperature fp32 [B]  NULL = 1; 0 (or less, or NaN): the largest logit,
 *               the lowest index of equal ones
 *   top_k       int32 [B] NULL or <= 0: all; else the k largest logits
 *   top_p       fp32 [B]  NULL or >= 1: all; else, in falling order, a token
 *               stays while the mass before it is below top_p times the mass
 *               that top_k left; the first one always stays
 *   min_p       fp32 [B]  NULL or <= 0: all; else a token stays if its
 *               probability is at least min_p (at most 1) times the largest
 *   u           fp32 [B][T] in [0, 1)
 *   token       int32 [B][T] written: the first index, in vocabulary order,
 *               at which the running mass of the tokens that stay exceeds u
 *               times their whole mass; -1 if no logit is above -inf
 * Equal logits count in order of their index; NaN counts as -inf; +inf
 * logits share the whole mass.
 * The mass of a token is round(2^31 * 2^((z - z_max) log2(e) / temperature)),
 * a whole number, so that no sum depends on its order and equal inputs give
 * equal tokens however the work is split. */
int gdn_tree_sample(const gdn_sample_dims* dims, const void* meta, const void* logits,
                    const float* temperature, const int32_t* top_k, const float* top_p,
                    const float* min_p, const float* u, int32_t* token, hipStream_t stream);

/* Acceptance along the sampled tokens (Eq. 1-2, on a tree): from
 * the root, the child whose draft token is the one sampled at the current
 * node becomes the current node (the lowest slot of equal siblings); where
 * there is none the walk ends.  Every emitted token is then a sample of the
 * model given the tokens before it.  Reads only dims->B and dims->T.
 *   meta       tree metadata, or NULL for a chain of T slots
 *   draft      int32 [B][T]  token of every slot (the root's is not read as a
 *              draft: it is the last emitted token)
 *   token      int32 [B][T]  gdn_tree_sample's
 *   accepted   int32 [B]     written: last node of the walk, for
 *              gdn_tree_commit, gdn_tree_step and gdn_kv_commit; -1 for an
 *              empty tree or one with a non-zero status
 *   n_emitted  int32 [B]     written: depth(accepted) + 1
 *   emitted    int32 [B][T]  written: the tokens below the root, then the one
 *              sampled at the accepted node (-1 if it has none; n_emitted
 *              counts it all the same), then -1; must not overlap draft or
 *              token
 * A negative token matches no draft. */
int gdn_tree_accept(const gdn_dims* dims, const void* meta, const int32_t* draft,
                    const int32_t* token, int32_t* accepted, int32_t* n_emitted, int32_t* emitted,
                    hipStream_t stream);

/* ------------------------------------------------------------------------
 * Layers without draft trees: sequences of any length through the gated
 * delta rule, and the norms around a block
 *
 * gdn_chain takes whole sequences (prompts, single tokens) through one GDN
 * layer: outputs of every token, the state and the conv state behind the last
 * one, in one call.  gdn_gate_norm norms and gates its outputs head by head,
 * gdn_add_norm adds a block's result to the residual stream and norms that
 * for the next block. */

/* Rows of a call: sequence b has tokens in rows
 *   padded (start NULL)  b T .. b T + n_new[b] - 1   (n_new NULL: T of them)
 *   packed               start[b] .. start[b + 1] - 1
 * of q, k, v, alpha, beta and out, whose other rows are neither read nor
 * written. */
typedef struct {
  int32_t B, T;      /* sequences, the most tokens of one (<= GDN_MAX_CHAIN_T)   */
  int32_t Hk, Hv;    /* key and value heads, Hv % Hk == 0                        */
  int32_t dk, dv;    /* 16, 32, 64 or 128                                        */
  int32_t in_dtype;  /* q, k, v, alpha, beta: GDN_F32 or GDN_BF16                */
  int32_t out_dtype; /* out: GDN_F32 or GDN_BF16                                 */
  int64_t rows;      /* packed: rows of the tensors; not read otherwise (B T)    */
  float scale;       /* of the readout; 0 selects 1 / sqrt(dk)                   */
} gdn_chain_dims;

#define GDN_MAX_CHAIN_T (1 << 24)

/* The gated delta rule over sequences (Eq. 7-8 along a chain of any length),
 * with the short convolution, activation and norms of gdn_tree_verify.
 *   start      int32 [B + 1] or NULL (padded), see above; not with n_new
 *   n_new      int32 [B] or NULL
 *   q, k, v, alpha, beta   in_dtype [rows][Hk][dk], [rows][Hk][dk],
 *              [rows][Hv][dv], [rows][Hv], [rows][Hv]
 *   conv_w     fp32 [C][4], C = 2 Hk dk + Hv dv
 *   conv_state fp32 [B][3][C]   read-only: raw inputs before the first token
 *   conv_state_out  fp32 [B][3][C]  written: those before the next token; must
 *              not overlap conv_state
 *   S          fp32 [B][Hv][dv][dk]  in/out
 *   out        out_dtype [rows][Hv][dv]  written: o_t = scale S_t q_t; must not
 *              overlap an input
 *   status     int32 [B] (may be NULL): GDN_CHAIN_BAD_LEN for a sequence whose
 *              length is negative or above T, whose rows are outside [0, rows),
 *              or (where start goes backwards) among those of a sequence before
 *              it that has neither of these; 0 otherwise
 * A sequence without tokens, or with a non-zero status, keeps S and gets
 * conv_state_out = conv_state.  No tensor may overlap S, conv_state_out or
 * status.  A decay below the smallest normal float counts as that in the
 * chunked form.  Inputs have to be finite: an infinity or NaN may reach every
 * token of its chunk, those before it too.
 * Short sequences (T <= GDN_CHAIN_STEP_T) go token by token with the state in
 * registers, in fp32, and need no workspace.  Longer ones go in chunks of 64
 * tokens: operands are pairs of fp16 values (22 bits), products three on them
 * with fp32 sums, as near as fp32 products on ordinary inputs.  Beside that an
 * output, and the state, may be off by about 2^-34 of the largest value (or row of
 * the state) of its head in this chunk or the one before, also where the decays
 * have forgotten that since, which the token by token form does not have.  They go
 * through a workspace that the library keeps (see Workspaces above, also for how
 * much more than a call's need it may hold).  A call needs at most
 * GDN_CHAIN_WORKSPACE bytes, or what one chunk of one sequence does: a chunk takes
 * 768 Hk dk + 25600 Hv bytes (dk of 16 as 32). */
#define GDN_CHAIN_STEP_T 20
#define GDN_CHAIN_WORKSPACE (1u << 28)
int gdn_chain(const gdn_chain_dims* dims, const int32_t* start, const int32_t* n_new, const void* q,
              const void* k, const void* v, const void* alpha, const void* beta,
              const float* conv_w, const float* conv_state, float* conv_state_out, float* S,
              void* out, int32_t* status, hipStream_t stream);

typedef enum { GDN_SILU = 0, GDN_SIGMOID = 1 } gdn_act;

/* Problem sizes of gdn_gate_norm: N rows of H heads of d channels.  ldx, ldg:
 * elements from one row of x (of gate) to the next, 0 selects H d. */
typedef struct {
  int64_t N;
  int32_t H, d; /* 1 <= d <= GDN_MAX_NORM_D, H d <= GDN_MAX_ROW       */
  int32_t x_dtype, gate_dtype, out_dtype;
  int32_t act; /* GDN_SILU or GDN_SIGMOID                              */
  int64_t ldx, ldg;
  float eps; /* positive and not subnormal                             */
} gdn_gate_norm_dims;

#define GDN_MAX_NORM_D 16384
#define GDN_MAX_ROW (1 << 24)

/* Norm of every head, times a gate:
 *   out[n][h] = x[n][h] / sqrt(mean(x[n][h]^2) + eps) * weight * act(gate[n][h])
 *   x       x_dtype [N][ldx]
 *   gate    gate_dtype [N][ldg], or NULL: no gate
 *   weight  fp32 [d], or NULL: 1
 *   out     out_dtype [N][H d]  written; may be x itself where types and rows
 *           are the same (any other overlap is not allowed)
 * These pointers need the alignment of their elements only.
 * In 32 bits: the squares of a head have to sum to less than 2^128. */
int gdn_gate_norm(const gdn_gate_norm_dims* dims, const void* x, const void* gate,
                  const float* weight, void* out, hipStream_t stream);

/* Problem sizes of gdn_add_norm: N contiguous rows of D channels. */
typedef struct {
  int64_t N;
  int32_t D; /* 1 <= D <= GDN_MAX_NORM_D                               */
  int32_t x_dtype, res_dtype, out_dtype;
  int32_t post; /* non-zero: x is normed before it is added            */
  float eps;    /* positive and not subnormal                          */
} gdn_add_norm_dims;

/* The residual stream from one block to the next:
 *   y = x, or with post  x / sqrt(mean(x^2) + eps) * post_weight
 *   r = residual + scale * y             (written to res_out)
 *   out = r / sqrt(mean(r^2) + eps) * weight     (of r before it is rounded)
 *   x            x_dtype [N][D]
 *   residual     res_dtype [N][D], or NULL: 0
 *   weight, post_weight, scale   fp32 [D], or NULL: 1
 *   res_out      res_dtype [N][D], or NULL; may be residual itself
 *   out          out_dtype [N][D], or NULL (one of the two is needed); may be
 *                x itself where their types are the same
 * Any other overlap of an output is not allowed.  Alignment and range as for
 * gdn_gate_norm. */
int gdn_add_norm(const gdn_add_norm_dims* dims, const void* x, const void* residual,
                 const float* weight, const float* post_weight, const float* scale, void* res_out,
                 void* out, hipStream_t stream);

/* Message describing the last non-OK return on the calling thread. */
const char* gdn_last_error(void);

/* Library version string. */
const char* gdn_version(void);

#ifdef __cplusplus
}
#endif

#endif /* GDN_TREE_H */
