/*
 * libtrjacobi — the verify step of TR-Jacobi decoding on one MI355X (gfx950).
 *
 * Paper: "Make Some Noise", section "TR-Jacobi Decoding" (paragraph "Tree-based
 * Jacobi Decoding") and appendix "Templates for Token Tree".  The draft tokens of a
 * decoding round are held in a token tree; one decoder forward scores every node,
 * each node attending to the committed prefix and to its own ancestors (the sparse
 * tree-attention mask); the greedy prediction (Eq. 1) at every node is compared with
 * the draft tokens of its children and the path with the longest run of matches is
 * kept.  The paper leaves the decoder architecture, the positions of tree nodes, the
 * KV cache and the exact acceptance formula open; the readings used here are stated
 * next to each entry point.
 *
 * General rules
 *  - C linkage, plain pointers and sizes.  Every function returns a trj_status.
 *    Nothing throws, nothing aborts.
 *  - Pointers are DEVICE pointers unless the name starts with h_ (host).  The caller
 *    owns every buffer; the library allocates and frees nothing.  Process-wide state: the
 *    last HIP error code, the fixed scratch array of tree_attention_static_scratch and
 *    its per-device address, and what the development header trjacobi_dev.h adds (launch
 *    knobs, an event timer).  Entry points may be called from several threads as long as
 *    their buffers do not overlap.
 *  - Every call only enqueues work on `stream` (a hipStream_t passed as void*; NULL
 *    is the default stream) and returns; no host synchronisation happens inside.
 *  - Errors the host can see (null pointers, shapes, dtype, sizes) are returned
 *    before anything is enqueued and leave all outputs untouched.  Malformed trees
 *    are only visible on the device: they set status_dev[s] = 1 for that sequence
 *    (see accept_path).
 *
 * Tree encoding (per sequence): nodes are numbered so that parent[i] < i, node 0 is
 * the root with parent[0] = -1.  The root is the last committed token; its K/V is not
 * in the cache yet and it is always kept, so a step emits accept_len + 1 tokens.  At
 * most TRJ_N_MAX nodes per sequence.  Parent indices are local to the sequence.
 *
 * Packed batches: B sequences, T tree rows in total.  node_off[B+1] gives each
 * sequence's row range, kv_off[B] its first slot in the KV pool (a multiple of
 * TRJ_KV_BLOCK), prefix_len[B] its committed length.  Sequence s owns pool slots
 * [kv_off[s], kv_off[s] + prefix_len[s] + N_s); tree node i lives at slot
 * kv_off[s] + prefix_len[s] + i.
 *
 * Data layouts (element offsets; elements are 2 bytes for TRJ_BF16, 4 for TRJ_F32)
 *  - KV pool, one layer: K and V each hold one plane per K/V head (n_kv_heads, which is
 *    n_heads unless the model uses grouped-query attention) of s_pool * head_dim
 *    elements (s_pool a multiple of TRJ_KV_BLOCK, head_dim a multiple of 32); K is
 *    stored already rotated.  Inside a plane the slots are tiled in blocks of 32 so
 *    that a wavefront's 16-byte-per-lane load is one contiguous 1 KiB read that is
 *    already an MFMA operand:
 *      K(slot, c): ((slot/32 * head_dim/16 + c/16) * 64 + (c%16)/8 * 32 + slot%32) * 8 + c%8
 *      V(slot, c): (((slot/32 * head_dim/32 + c/32) * 2 + (slot%32)/16) * 64
 *                   + ((slot%16)/4 % 2) * 32 + c%32) * 8 + (slot%16)/8 * 4 + slot%4
 *    trj_kv_pack / trj_kv_unpack convert from / to plain [head][slot][head_dim].
 *    All layers: layer l starts kv_layer_stride elements after layer l-1.
 *  - Weight matrices W[n_out][n_in] (y = x W^T, no biases) are tiled 32 rows x 16
 *    columns by trj_pack_weight:
 *      W(r, k): ((r/32 * n_in/16 + k/16) * 64 + (k%16)/8 * 32 + r%32) * 8 + k%8
 *    where r is the packed row.  TRJ_PACK_PLAIN: r = n.  TRJ_PACK_GATE_UP (rows
 *    [Wg; Wu]): tile t holds gate rows 16t..16t+15 then up rows 16t..16t+15.
 *    TRJ_PACK_QKV (rows [Wq; Wk; Wv], head-major): inside every q and k head the tile
 *    j (0..head_dim/32-1) holds dims 16j..16j+15 then head_dim/2+16j.. (the rotary
 *    partners); v rows keep their order.
 *  - q and the attention output: plain [T][n_heads][head_dim].  Logits: [T][vocab]
 *    fp32.  Norm gains: fp32 [d_model].
 */
#ifndef TRJACOBI_H
#define TRJACOBI_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define TRJ_N_MAX 128
#define TRJ_KV_BLOCK 32

typedef enum {
  TRJ_OK = 0,
  TRJ_ERR_NULLPTR = -1,
  TRJ_ERR_BAD_SHAPE = -2,
  TRJ_ERR_BAD_DTYPE = -3,
  TRJ_ERR_TREE_TOO_LARGE = -4,
  TRJ_ERR_WORKSPACE_TOO_SMALL = -5,
  TRJ_ERR_HIP = -6
} trj_status;

typedef enum { TRJ_F32 = 0, TRJ_BF16 = 1 } trj_dtype;
typedef enum { TRJ_PACK_PLAIN = 0, TRJ_PACK_QKV = 1, TRJ_PACK_GATE_UP = 2 } trj_pack_kind;

typedef struct {
  int32_t n_layers, d_model, n_heads, head_dim, d_ffn, vocab;
  float rms_eps;    /* RMSNorm: x * g / sqrt(mean(x^2) + rms_eps) */
  float rope_theta; /* rotary base; pair (j, j+head_dim/2), angle pos*theta^(-2j/head_dim) */
  int32_t dtype;    /* trj_dtype of weights, KV pool and q; accumulation is fp32 */
  int32_t n_kv_heads; /* grouped-query attention: K/V heads, a divisor of n_heads; query head h
                       * reads K/V head h / (n_heads / n_kv_heads).  0 means n_heads. */
} trj_model_desc;

typedef struct {
  const float* g_attn;   /* [d_model] */
  const void* wqkv;      /* [(n_heads + 2*n_kv_heads)*head_dim][d_model], rows Wq;Wk;Wv, TRJ_PACK_QKV */
  const void* wo;        /* [d_model][n_heads*head_dim],   TRJ_PACK_PLAIN */
  const float* g_ffn;    /* [d_model] */
  const void* w_gate_up; /* [2*d_ffn][d_model],            TRJ_PACK_GATE_UP */
  const void* w_down;    /* [d_model][d_ffn],              TRJ_PACK_PLAIN */
} trj_layer_weights;

typedef struct {
  const void* embed;     /* [vocab][d_model], plain row-major, model dtype */
  const float* g_final;  /* [d_model] */
  const void* w_lm;      /* [vocab][d_model], TRJ_PACK_PLAIN */
  const trj_layer_weights* h_layers; /* HOST array of n_layers entries (device pointers inside) */
} trj_weights;

const char* trj_version(void);
/* hipError_t of the last failing HIP call seen by this library (0 if none). */
int32_t trj_last_hip_error(void);

/* Bytes of device scratch tr_verify_step / tree_attention need for a call with T = t_max
 * tree rows, B = b_max sequences and max_seq_slots = l_max.  The size is not monotonic in
 * these numbers: query every shape that will be used and take the largest.  A call whose
 * workspace is too small returns TRJ_ERR_WORKSPACE_TOO_SMALL and does nothing. */
int32_t trj_workspace_bytes(const trj_model_desc* desc, int32_t t_max, int32_t b_max,
                            int32_t l_max, size_t* h_bytes);

/* Layout helpers (see the layout section above).  src and dst must not overlap. */
int32_t trj_pack_weight(void* dst, const void* src_rowmajor, int32_t n_out, int32_t n_in,
                        int32_t dtype, int32_t kind, int32_t n_heads, int32_t head_dim,
                        void* stream);
/* plain [n_heads][n_slots][head_dim] <-> the tiled pool planes of one layer, slots
 * slot0 .. slot0+n_slots-1 of the pool.  n_heads here counts planes, i.e. K/V heads. */
int32_t trj_kv_pack(void* k_pool, void* v_pool, const void* k_plain, const void* v_plain,
                    int32_t n_heads, int32_t head_dim, int32_t s_pool, int32_t slot0,
                    int32_t n_slots, int32_t dtype, void* stream);
int32_t trj_kv_unpack(void* k_plain, void* v_plain, const void* k_pool, const void* v_pool,
                      int32_t n_heads, int32_t head_dim, int32_t s_pool, int32_t slot0,
                      int32_t n_slots, int32_t dtype, void* stream);

/* Tree bookkeeping: depth[i] = depth[parent[i]] + 1 (root 0) and the ancestor-or-self
 * bit rows of the sparse tree mask (appendix "Templates for Token Tree"): bit j%64 of
 * anc[i][j/64] is set when node j is on the path root..i.  A sequence whose tree is
 * malformed (parent[0] != -1, parent[i] outside [0, i), more than TRJ_N_MAX rows) gets
 * status_dev[s] = 1 and zeroed rows.  Outputs: depth[T], anc[T][2] (uint64),
 * status_dev[B]. */
int32_t trj_tree_mask(const int32_t* parent, const int32_t* node_off, int32_t B, int32_t T,
                      int32_t* depth, uint64_t* anc, int32_t* status_dev, void* stream);

/* Tree-masked attention for one layer (section "TR-Jacobi Decoding": every path runs
 * an ordinary Jacobi step through tree attention).  For row i of sequence s and each
 * head: softmax over {prefix slots 0..prefix_len[s]-1} U {tree slots of i's ancestors
 * and i itself} of scale * q.k, times V.  The tree's own K/V must already be in the
 * pool at slots kv_off[s] + prefix_len[s] + i.  q, out: [T][n_heads][head_dim] in
 * `dtype`.  k_layer, v_layer hold n_kv_heads planes (0: n_heads); with fewer K/V heads
 * than query heads, query head h reads plane h / (n_heads / n_kv_heads) (grouped-query
 * attention).  max_seq_slots: host upper bound of prefix_len[s] + N_s (sizes the
 * launch).  workspace: device scratch of at least trj_workspace_bytes(...) bytes. */
int32_t tree_attention(const void* q, const void* k_layer, const void* v_layer,
                       const int32_t* parent, const int32_t* node_off, const int32_t* kv_off,
                       const int32_t* prefix_len, int32_t B, int32_t T, int32_t n_heads,
                       int32_t n_kv_heads, int32_t head_dim, int32_t s_pool,
                       int32_t max_seq_slots, int32_t dtype, float scale, void* workspace,
                       size_t ws_bytes, void* out, void* stream);

/* Bytes of device scratch that let tree_attention choose its launch at these sizes, whatever
 * the number of K/V heads: where some number of them would have query heads worked on together,
 * room for the partial sums of that too.  A call is accepted with less as long as its query
 * heads fit one by one, which is then how they are worked on; what trj_workspace_bytes reports
 * for a model with these heads is always enough for that. */
int32_t tree_attention_workspace_bytes(int32_t B, int32_t T, int32_t n_heads, int32_t head_dim,
                                       int32_t max_seq_slots, int32_t dtype, size_t* h_bytes);

/* tree_attention for callers that cannot allocate device memory or pass a workspace
 * (code under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc):
 * the same kernels and results, with the scratch in a fixed array of
 * TRJ_STATIC_SCRATCH_BYTES inside the library (every GPU the library runs on holds one
 * copy until the process ends).  A call that needs more than that even
 * with its query heads one by one returns TRJ_ERR_WORKSPACE_TOO_SMALL and does nothing (the need is
 * the partial sums of sequences whose keys are split over several workgroups: with 32 heads of
 * 128, at any length and tree size, up to 17 MiB for one and two sequences, 19 for three and four, 21,
 * 25 and 29 for five, six and seven; from eight on below 0.5, and up to 17 where heads that share
 * K/V are worked on together; more only when a development knob asks for more splits).  No
 * hipMalloc, hipFree or other allocating call is made.  All calls on one GPU share that
 * GPU's array: calls that overlap in time on one GPU (two streams, two threads) race;
 * calls on one stream are ordered and safe.  Nothing in the array needs clearing between
 * calls: every call rewrites what it reads. */
#define TRJ_STATIC_SCRATCH_BYTES (32u << 20)
int32_t tree_attention_static_scratch(const void* q, const void* k_layer, const void* v_layer,
                                      const int32_t* parent, const int32_t* node_off,
                                      const int32_t* kv_off, const int32_t* prefix_len, int32_t B,
                                      int32_t T, int32_t n_heads, int32_t n_kv_heads,
                                      int32_t head_dim, int32_t s_pool, int32_t max_seq_slots,
                                      int32_t dtype, float scale, void* out, void* stream);

/* Greedy argmax (Eq. 1) and the longest accepted path (section "TR-Jacobi Decoding").
 * If logits != NULL: argmax_out[i] = lowest index of the row maximum of logits[i][0..V)
 * (NaN never wins).  If logits == NULL, argmax_out must already hold the predictions.
 * ok[root] = 1, ok[i] = ok[parent[i]] && tok[i] == argmax_out[parent[i]]; best = the
 * deepest ok node, lowest index among equals.  Outputs per sequence: accept_len =
 * depth[best] (accepted drafts), best_node, path[s][TRJ_N_MAX] = node indices root..best
 * then -1, bonus_tok = argmax_out[best].  Malformed tree: status_dev[s] = 1,
 * accept_len[s] = -1, best_node = -1, path all -1, bonus_tok = -1. */
int32_t accept_path(const float* logits, const int32_t* tok, const int32_t* parent,
                    const int32_t* node_off, int32_t B, int32_t T, int32_t V,
                    int32_t* argmax_out, int32_t* accept_len, int32_t* best_node,
                    int32_t* path, int32_t* bonus_tok, int32_t* status_dev, void* stream);

/* In-place compaction of the accepted path (the paper has no cache; this keeps the
 * accepted rows contiguous after the prefix): for every layer and head and
 * j = 0..accept_len[s], slot kv_off+prefix_len+j <- slot kv_off+prefix_len+path[s][j]
 * for K and V; new_len[s] = prefix_len[s] + accept_len[s] + 1.  Sequences with
 * accept_len[s] < 0 are skipped (new_len = prefix_len).  Slots beyond new_len are
 * unspecified afterwards.  n_heads counts the planes of a layer, i.e. K/V heads. */
int32_t kv_compact(void* k_pool, void* v_pool, size_t kv_layer_stride, const int32_t* path,
                   const int32_t* accept_len, const int32_t* kv_off, const int32_t* prefix_len,
                   int32_t B, int32_t n_layers, int32_t n_heads, int32_t head_dim,
                   int32_t s_pool, int32_t dtype, int32_t* new_len, void* stream);

/* The whole verify step: embedding of tok, n_layers x {RMSNorm, QKV, rotary at
 * position prefix_len + depth, tree K/V written to the pool, tree attention, output
 * projection + residual, RMSNorm, SwiGLU FFN + residual}, final RMSNorm, LM head,
 * greedy argmax, longest accepted path, compaction.  logits ([T][vocab] fp32) may be
 * NULL when only the predictions are wanted: in bf16 mode the argmax is then taken in
 * the LM head's epilogue and no logits are ever written to memory (same predictions,
 * bit for bit, as with a logits buffer); in fp32 mode they are kept in the workspace.
 * All other outputs as in accept_path / kv_compact. */
int32_t tr_verify_step(const trj_model_desc* desc, const trj_weights* weights, void* k_pool,
                       void* v_pool, size_t kv_layer_stride, int32_t s_pool,
                       const int32_t* tok, const int32_t* parent, const int32_t* node_off,
                       const int32_t* kv_off, const int32_t* prefix_len, int32_t B, int32_t T,
                       int32_t max_seq_slots, void* workspace, size_t ws_bytes, float* logits,
                       int32_t* argmax_out, int32_t* accept_len, int32_t* best_node,
                       int32_t* path, int32_t* bonus_tok, int32_t* new_len,
                       int32_t* status_dev, void* stream);

/* ---- Static tree template (appendix "Templates for Token Tree": one fixed sparse tree is
 * used for every verification step).  What depends on the tree alone is computed once
 * into a caller-owned device buffer: validity, depth and ancestor bit rows of every node,
 * and the rotary table cos/sin(p * theta^(-2j/head_dim)) for positions p = 0..max_pos-1.
 * tr_verify_step_template is tr_verify_step with that buffer: per step only the parts
 * that depend on the prefix lengths are recomputed (slot range checks, slot and position
 * of every row, the attention work list), in one launch, and results are identical.
 *  - tr_template_bytes: size of the buffer for B sequences, T rows, max_pos positions.
 *  - tr_template_prepare: fills it from parent[T] / node_off[B+1] (same meaning as in
 *    tr_verify_step).  A malformed tree is recorded in the buffer and marks its sequence
 *    (status_dev[s] = 1) in every step that uses it.
 *  - tr_verify_step_template: B, T, max_pos, the model's head_dim and node_off[] must be
 *    those the buffer was prepared with, and parent[] must hold the same tree (it is
 *    still read by the acceptance rule); a buffer prepared for other sizes or row
 *    ranges marks every affected sequence malformed instead of being used.  Every
 *    sequence needs prefix_len[s] + N_s <= max_pos, else it is marked as well.  The
 *    buffer is only read; several steps (and streams) may share it. */
int32_t tr_template_bytes(const trj_model_desc* desc, int32_t B, int32_t T, int32_t max_pos,
                          size_t* h_bytes);
int32_t tr_template_prepare(const trj_model_desc* desc, const int32_t* parent,
                            const int32_t* node_off, int32_t B, int32_t T, int32_t max_pos,
                            void* tmpl, size_t tmpl_bytes, void* stream);
int32_t tr_verify_step_template(const trj_model_desc* desc, const trj_weights* weights,
                                void* k_pool, void* v_pool, size_t kv_layer_stride, int32_t s_pool,
                                const int32_t* tok, const int32_t* parent, const int32_t* node_off,
                                const int32_t* kv_off, const int32_t* prefix_len, int32_t B,
                                int32_t T, int32_t max_seq_slots, const void* tmpl,
                                size_t tmpl_bytes, int32_t max_pos, void* workspace,
                                size_t ws_bytes, float* logits, int32_t* argmax_out,
                                int32_t* accept_len, int32_t* best_node, int32_t* path,
                                int32_t* bonus_tok, int32_t* new_len, int32_t* status_dev,
                                void* stream);

/* ---- TR-Jacobi decoding loop (section "TR-Jacobi Decoding") -------------------------
 * Generation starts from a tree whose nodes are ahead noise (Eq. 4), every round
 * verifies the tree with tr_verify_step's forward, commits the longest accepted path
 * plus the greedy token after it, and refills the tree from the predictions made below
 * the accepted node; one chain below the root carries tokens retrieved by prompt lookup
 * (paragraph "Retrieval-Augmented Jacobi Decoding").  The committed tokens equal plain
 * greedy decoding whatever the drafts are.
 *
 * Refill rule (the paper only says "the path's subsequent predictions"): the new tree
 * is laid over the old one with its root on the accepted node; a new node that is the
 * k-th child (index order) of its parent lies on the k-th child of the old node under
 * its parent, if there is one, and takes the prediction made there as its token; a new
 * node that lies on nothing takes ahead noise: ctx[r mod ctx_len] with r the
 * (step * TRJ_N_MAX + node + 1)-th SplitMix64 output for `seed` and ctx all committed
 * tokens.  The last retrieval_len nodes of the template must be a chain below the root;
 * prompt lookup tries suffix lengths max_ngram..1 of ctx, takes the most recent earlier
 * occurrence and copies up to retrieval_len following tokens over that chain.
 *
 * The four helpers below are pure host functions (no GPU is touched). */
typedef struct {
  int32_t n_nodes;         /* N, root included, 1..TRJ_N_MAX */
  const int32_t* h_parent; /* HOST [N]: parent[0] = -1, 0 <= parent[i] < i */
  int32_t retrieval_len;   /* R in 0..N-1 */
  int32_t max_ngram;       /* >= 1 */
  int32_t max_new_tokens;  /* >= 1 */
  int32_t eos_token;       /* generation stops after this token (kept); -1: never */
  uint64_t seed;
} trj_decode_config;

/* k-th output (k >= 1) of SplitMix64 started at state `seed`. */
uint64_t trj_splitmix64(uint64_t seed, uint64_t k);
int32_t trj_ahead_noise(const int32_t* h_ctx, int32_t ctx_len, uint64_t seed, int32_t step,
                        int32_t node, int32_t* h_token);
/* h_out[0..*h_found) = the retrieved tokens, *h_found <= r. */
int32_t trj_prompt_lookup(const int32_t* h_ctx, int32_t ctx_len, int32_t max_ngram, int32_t r,
                          int32_t* h_out, int32_t* h_found);
/* Tokens of the tree verified in round `step`; ctx's last token is the root.
 * h_argmax == NULL: first tree (all noise + lookup); else the previous round's
 * predictions [N] and accepted node `best`. */
int32_t trj_fill_tree(const int32_t* h_parent, int32_t n_nodes, int32_t retrieval_len,
                      const int32_t* h_ctx, int32_t ctx_len, int32_t max_ngram, uint64_t seed,
                      int32_t step, const int32_t* h_argmax, int32_t best, int32_t* h_tok);

/* Device scratch tr_jacobi_generate needs for these sizes and this pool capacity. */
int32_t tr_jacobi_generate_workspace_bytes(const trj_model_desc* desc, int32_t n_nodes,
                                           int32_t prompt_len, int32_t max_new_tokens,
                                           int32_t s_pool, size_t* h_bytes);

/* Greedy generation for ONE sequence whose K/V live at slot 0.. of the pool (kv offset
 * 0; s_pool slots per head, a multiple of TRJ_KV_BLOCK, at least prompt_len +
 * max_new_tokens + N).  The prompt's K/V are computed first by chain-shaped trees of
 * TRJ_N_MAX tokens (an ordinary causal forward), up to eight of them packed into one step
 * as "sequences" that share the K/V region; the pool's previous contents are ignored.  h_prompt: HOST [prompt_len], prompt_len >= 1, ids in [0, vocab).  Outputs
 * (HOST): h_tokens[max_new_tokens], *h_n_tokens, h_accept_hist[max_new_tokens] (accepted
 * drafts per round, may be NULL), *h_n_steps (rounds).  Synchronous: returns after the
 * stream has drained.  Errors as above; nothing is written to the host outputs'
 * token area on an argument error. */
int32_t tr_jacobi_generate(const trj_model_desc* desc, const trj_weights* weights, void* k_pool,
                           void* v_pool, size_t kv_layer_stride, int32_t s_pool,
                           const int32_t* h_prompt, int32_t prompt_len,
                           const trj_decode_config* cfg, void* workspace, size_t ws_bytes,
                           int32_t* h_tokens, int32_t* h_n_tokens, int32_t* h_accept_hist,
                           int32_t* h_n_steps, void* stream);

/* ---- Serving from a paged 8-bit cache ------------------------------------------------
 * A cache of half the size for batches whose lengths only the device knows: pages of
 * TRJ_KV_BLOCK slots that any sequence may own, found through a table; K and V in 8 bits
 * (e4m3: sign, 4 bits of exponent, 3 of mantissa, largest value 448) with one scale for
 * the K and one for the V of a page and head.  kv_block_tables hands the pages out,
 * tree_attention_q8 reads them, kv_append_q8 writes what has been committed; the rows of
 * the tree under verification stay in 16 bits with the caller until they are accepted, so
 * rejected drafts never touch the cache and nothing is compacted.  tree_logits turns raw
 * logits into those that sampling rules ask for, at every node.
 *
 * One layer of the cache: K and V codes [n_kv_heads][n_blocks][32 * head_dim] bytes, scales
 * [n_kv_heads][n_blocks] fp32; value = code * scale.  A scale is a power of two (of another
 * number the fraction is ignored), so that products with it are exact.  Inside a page, row
 * r (slot % 32) and column c lie at byte
 *   K: ((c/32 * 2 + c%32/16) * 32 + r) * 16 + c%16
 *   V: ((c/32 * 2 + r/4%2) * 32 + c%32) * 16 + r/16 * 8 + r/8%2 * 4 + r%4
 * block_table[B][max_blocks]: position p of sequence s is slot p % 32 of page
 * block_table[s][p / 32].  Entries behind a sequence's length are not read.  Positions are int32 to the end of their
 * page: where max_blocks is more than 2^26 - 1, a sequence can still hold no more than these.
 *
 * Rows (q_rows, k_rows, v_rows): [T][heads][head_dim] in `dtype` with *_stride elements from
 * row to row (a part of a wider row, as a common projection of q, k and v leaves it),
 * k already rotated; addresses are multiples of 16 bytes, strides of 8 elements up to 2^24, else
 * TRJ_ERR_BAD_SHAPE.  dtype is TRJ_BF16 (the 32-bit mode keeps its 32-bit pool:
 * TRJ_ERR_BAD_DTYPE), head_dim 64 or 128.  At most TRJ_SERVE_MAX_SEQS sequences per call.
 *
 * node_off need not cover all T rows, and a sequence may have no rows; rows that no sequence
 * owns are left as they were in every output.  No row belongs to two sequences: what is written for
 * rows that overlap, and for the sequences behind them, is undefined.  What the device finds wrong with a
 * sequence sets status_dev[s] = 1 (else 0) and is stated at each call. */
#define TRJ_SERVE_MAX_SEQS 4096

/* Pages follow lengths.  Sequence s is to hold want = ceil((prefix_len[s] + N_s) / 32) pages,
 * N_s = node_off[s+1] - node_off[s]; it holds held[s] now.
 *  - More than it wants: its last pages go back, in order, on top of the stack free_list[0 ..
 *    free_count) (sequences in index order).
 *  - Fewer: then pages are taken from the top, sequence by sequence, and written to the table
 *    behind those it holds.  Where the pages do not last for sequence s and all before it,
 *    it gets none: status_dev[s] = 1, it keeps what it holds, and so does every sequence behind it
 *    that wants more.
 * The table entries that a sequence with status 1 wanted behind those it holds become -1: pages that
 * it gave back from there may be another's by now, and kv_append_q8 refuses rows that would go there.
 * held_out[B], free_count_out[1]: the new counts; row_slot[T]: the slot of every row (page
 * number * 32 + position % 32), -1 for rows of sequences with status 1.
 * Also status 1, with what it holds unchanged: negative or descending sizes, more than max_blocks pages wanted
 * or held, rows outside [0, T).  A free_count outside [0, n_blocks] counts as 0.
 * free_list has n_blocks entries, the number of pages there are; what would be stacked beyond them
 * (pages held twice) is dropped.  Page numbers are copied, not judged.  Nothing that a call reads is
 * overwritten, so that it may be repeated: the counts come in pairs of buffers that must not
 * overlap (TRJ_ERR_BAD_SHAPE where they are the same), table entries below held and the stack
 * below free_count stay.  T = 0: row_slot may be NULL. */
int32_t kv_block_tables(int32_t* block_table, int32_t max_blocks, const int32_t* held,
                        const int32_t* prefix_len, const int32_t* node_off, int32_t B, int32_t T,
                        int32_t* free_list, int32_t n_blocks, const int32_t* free_count,
                        int32_t* held_out, int32_t* free_count_out, int32_t* row_slot,
                        int32_t* status_dev, void* stream);

/* Quantises rows into the cache, all layers in one call.  path == NULL: all N_s rows of a
 * sequence, of any number, go to positions prefix_len[s] + j.  Else the accepted path of
 * accept_path: row path[s][j] (path has TRJ_N_MAX columns) for j = 0..accept_len[s].
 * The scale of a page is the smallest power of two (from 2^-100 on) with which its largest
 * value fits; a page that holds earlier rows keeps at least theirs, and where it has to grow
 * the earlier codes are rounded to it (exact down to the type's subnormal values).  Codes
 * round to nearest, ties to even.  A value that is not finite is stored as NaN and has no part
 * in the scale.  Slots of a page behind the last row keep their bytes.
 * new_len[s] = prefix_len[s] + rows stored, in a buffer that must not overlap prefix_len
 * (TRJ_ERR_BAD_SHAPE).  Repeating a call changes nothing.
 * Pools: n_layers of the layout above, one behind the other; rows of layer l start
 * l * row_layer_stride elements behind layer 0's (a multiple of 8).
 * Nothing is stored, new_len = prefix_len and status 1: accept_len[s] < 0 or >= N_s, a path
 * entry outside [0, N_s), N_s > TRJ_N_MAX with a path, rows outside [0, T), a negative size, more than
 * max_blocks pages, a page number outside [0, n_blocks).  Rows go to the pages that the table names: they have to
 * be among those that kv_block_tables was last asked to hold, since entries behind these may be pages that the
 * sequence gave back.  Two sequences (or two entries of one) must not name the same page where rows are
 * stored: the result is undefined. */
int32_t kv_append_q8(void* k_pool, void* v_pool, float* k_scale, float* v_scale, const void* k_rows,
                     const void* v_rows, int32_t row_stride, size_t row_layer_stride,
                     const int32_t* path, const int32_t* accept_len, const int32_t* node_off,
                     const int32_t* block_table, int32_t max_blocks, const int32_t* prefix_len,
                     int32_t B, int32_t T, int32_t n_layers, int32_t n_kv_heads, int32_t head_dim,
                     int32_t n_blocks, int32_t dtype, int32_t* new_len, int32_t* status_dev,
                     void* stream);

/* Bytes of device scratch for tree_attention_q8 with these sizes. */
int32_t tree_attention_q8_workspace_bytes(int32_t B, int32_t T, int32_t n_heads, int32_t n_kv_heads,
                                          int32_t head_dim, int32_t max_prefix, size_t* h_bytes);

/* tree_attention for one layer of the paged cache: row i of sequence s sees the
 * prefix_len[s] positions of the cache and the rows of its own ancestors and itself in k_rows,
 * v_rows (which the cache need not hold).  A sequence of one row is plain decoding, a chain of rows a
 * causal pass: a prompt goes in chains of at most TRJ_N_MAX rows, each appended before the next, or whole through chunk_attention_q8.  out: [T][n_heads][head_dim].  A key that a row does not see has no part in it
 * whatever it holds, infinities and NaN included; a row that sees a value that is not finite
 * gets what the sums give.  max_prefix: host upper bound of prefix_len[s].  scale: positive, and a
 * finite fp32 number when multiplied by log2(e), else TRJ_ERR_BAD_SHAPE.
 * Rows of zeros and status 1: malformed tree (as trj_tree_mask), more than TRJ_N_MAX rows,
 * prefix_len[s] outside [0, max_prefix] or beyond max_blocks pages; nothing and status 1: rows outside [0, T).
 * NaN in all rows and status 1: a page number outside [0, n_blocks).
 * Calls that overlap in time need workspaces of their own; nothing in one needs clearing. */
int32_t tree_attention_q8(const void* q_rows, int32_t q_stride, const void* k_pool, const void* v_pool,
                          const float* k_scale, const float* v_scale, const void* k_rows,
                          const void* v_rows, int32_t row_stride, const int32_t* parent,
                          const int32_t* node_off, const int32_t* block_table, int32_t max_blocks,
                          const int32_t* prefix_len, int32_t B, int32_t T, int32_t n_heads,
                          int32_t n_kv_heads, int32_t head_dim, int32_t n_blocks, int32_t max_prefix,
                          int32_t dtype, float scale, void* workspace, size_t ws_bytes, void* out,
                          int32_t* status_dev, void* stream);

/* Bytes of device scratch for tree_logits with these sizes. */
int32_t tree_logits_workspace_bytes(int32_t B, int32_t T, int32_t V, size_t* h_bytes);

/* Logits of every tree node after penalties, biases and a mask, and the greedy prediction from
 * them: what accept_path (with logits NULL) then takes, so that a verified tree equals
 * token-by-token decoding under the same rules.  The text before the prediction at node i is the
 * committed tokens ctx[ctx_off[s] .. ctx_off[s+1]) (the root's token is the last of them, as in
 * trj_fill_tree) and the drafts tok on the path from the root, exclusive, to i.  For token v with count n
 * among the generated ones (ctx from ctx_off[s] + gen_start[s] on, and the drafts):
 *   x = logit;  if v occurs anywhere in the text: x = x > 0 ? x / repetition : x * repetition
 *   x = x - frequency * n;  x = x - (n > 0 ? presence : 0);  x = x + bias(v)
 *   x = -infinity unless the row's mask allows v
 * each step rounded to fp32.  penalties[B][3] = repetition, frequency, presence.  Biases of
 * sequence s: entries bias_off[s] .. bias_off[s+1] of bias_tok, bias_val; of a token named more than
 * once the last entry counts.  allowed: bit v%32 of allowed[t][v/32], rows of ceil(V/32) words.  Token
 * ids outside [0, V) are passed over in ctx, tok and bias_tok.
 * Parts may be left out: ctx NULL (with ctx_off, gen_start): the drafts are the only text; penalties
 * NULL: none, ctx and tok are not looked at; bias_off NULL; allowed NULL.  n_ctx, n_bias: how many tokens
 * ctx, and entries bias_tok and bias_val, hold, at most 2^30 (TRJ_ERR_BAD_SHAPE).
 * logits_out: [T][V], may be logits itself, NULL if only predictions are wanted; argmax_out[T], may
 * be NULL (not both): the lowest index of the largest value among the allowed tokens, NaN below all
 * numbers (of nothing but NaN the first), -1 if the mask allows none, which no draft
 * matches.  Malformed trees and offsets (descending, or outside their array): status 1, the sequence's
 * rows are left as they were. */
int32_t tree_logits(const float* logits, const int32_t* tok, const int32_t* parent,
                    const int32_t* node_off, int32_t B, int32_t T, int32_t V, const int32_t* ctx,
                    int32_t n_ctx, const int32_t* ctx_off, const int32_t* gen_start,
                    const float* penalties, const int32_t* bias_tok, const float* bias_val,
                    int32_t n_bias, const int32_t* bias_off,
                    const uint32_t* allowed, float* logits_out, int32_t* argmax_out, void* workspace,
                    size_t ws_bytes, int32_t* status_dev, void* stream);

/* ---- Prompts and sampled tokens on the paged 8-bit cache -------------------------------
 * What a serving program needs between its own projections besides the calls above: rotary_rows
 * turns the rows of a projection to their positions, chunk_attention_q8 takes prompts of any length
 * beside sequences that decode, tree_sample chooses tokens under sampling rules where accept_path
 * would else be given greedy predictions.  The rules of the section above hold here too: rows that no
 * sequence owns are left as they were, no row belongs to two sequences, at most TRJ_SERVE_MAX_SEQS of
 * them, status_dev[s] = 1 (else 0) for what the device finds wrong with sequence s. */
typedef enum {
  TRJ_ROTARY_HALVES = 0, /* pair j: columns j and j + rot_dim/2 */
  TRJ_ROTARY_PAIRS = 1   /* pair j: columns 2j and 2j + 1 */
} trj_rotary_layout;
typedef enum {
  TRJ_ROTARY_PLAIN = 0, /* f_j = theta^(-2j/rot_dim) */
  TRJ_ROTARY_LINEAR = 1, /* f_j / factor: positions of a text that is factor times as long as the trained one */
  TRJ_ROTARY_TURNS = 2,  /* by the turns that pair j makes in the trained length, t = trained * f_j / (2 pi): f_j / factor
                          * up to low of them, f_j from high on, between them f_j / factor * (1 - g) + f_j * g with
                          * g = (t - low) / (high - low) */
  TRJ_ROTARY_RAMP = 3    /* by the pair's number: f_j up to the pair that makes high turns, f_j / factor from the one that makes
                          * low turns on, between them in even steps: a = max(0, floor(pair(high))), b = min(rot_dim - 1,
                          * ceil(pair(low))), pair(t) = rot_dim * ln(trained / (2 pi t)) / (2 ln theta), r = (j - a) / (b - a)
                          * (b = a: b = a + 0.001) kept to 0 .. 1: f_j * (1 - r) + f_j / factor * r; rotated rows times
                          * 0.1 ln(factor) + 1 */
} trj_rotary_scaling;

/* Frequencies for rotary_rows, on the host (no GPU is touched): h_freqs[rot_dim / 2], *h_magnitude.  factor >= 1, 0 < low < high
 * and trained > 0 where the rule reads them; theta > 1. */
int32_t trj_rotary_freqs(int32_t rot_dim, float theta, int32_t scaling, float factor, float low, float high,
                         int32_t trained, double* h_freqs, float* h_magnitude);

/* Rotary positions: (x1, x2) of pair j becomes magnitude * (x1 cos a - x2 sin a, x1 sin a + x2 cos a), a = position * freqs[j],
 * for j < rot_dim / 2 in every head of q_rows [T][n_heads][head_dim] and k_rows [T][n_kv_heads][head_dim]; columns from
 * rot_dim on are copied.  The angle is worked out in 64 bits, products in 32, each result rounded once.
 * Position: prefix_len[s] + depth of the node in its tree, or with parent NULL prefix_len[s] + j for row j of a sequence of
 * any number of rows.  freqs: DEVICE [rot_dim / 2] doubles.  head_dim a multiple of 8 up to 1024, rot_dim even and from 2 to
 * head_dim, rows of TRJ_BF16 or TRJ_F32, addresses multiples of 16 bytes, strides of 8 elements.  Results may take the place of
 * their inputs (same address and stride, else TRJ_ERR_BAD_SHAPE); other overlaps are undefined.
 * Nothing and status 1: malformed tree (as trj_tree_mask), rows outside [0, T), a negative
 * prefix_len, prefix_len[s] + N_s beyond 2^31.  At most 2^20 rows in all. */
int32_t rotary_rows(const void* q_rows, int32_t q_stride, const void* k_rows, int32_t k_stride, const int32_t* parent,
                    const int32_t* node_off, const int32_t* prefix_len, int32_t B, int32_t T, int32_t n_heads,
                    int32_t n_kv_heads, int32_t head_dim, int32_t rot_dim, int32_t layout, const double* freqs,
                    float magnitude, int32_t dtype, void* q_out, int32_t q_out_stride, void* k_out, int32_t k_out_stride,
                    int32_t* status_dev, void* stream);

/* Bytes of device scratch for chunk_attention_q8 with these sizes. */
int32_t chunk_attention_q8_workspace_bytes(int32_t B, int32_t T, int32_t n_heads, int32_t n_kv_heads,
                                           int32_t head_dim, int32_t max_prefix, size_t* h_bytes);

/* Causal attention of new rows over one layer of the paged cache: row i of sequence s sees the prefix_len[s]
 * positions of the cache and the rows 0 .. i of its own in k_rows, v_rows (which the cache need not hold).  A sequence has any
 * number of rows: chunks of prompts and sequences that decode one row go in one call.  (Batches of tens of sequences that all
 * decode one row are up to a fifth faster in tree_attention_q8.)  Arguments and what is said of
 * values that are not finite as in tree_attention_q8.  At most 2^20 rows in all, T * n_heads at most 2^30, max_prefix + T at
 * most 2^31 - 64 (TRJ_ERR_BAD_SHAPE).
 * Rows of zeros and status 1: prefix_len[s] outside [0, max_prefix] or beyond max_blocks pages; nothing and status 1: rows
 * outside [0, T).  NaN in all rows and status 1: a page number outside [0, n_blocks).
 * Calls that overlap in time need workspaces of their own; nothing in one needs clearing. */
int32_t chunk_attention_q8(const void* q_rows, int32_t q_stride, const void* k_pool, const void* v_pool,
                           const float* k_scale, const float* v_scale, const void* k_rows, const void* v_rows,
                           int32_t row_stride, const int32_t* node_off, const int32_t* block_table, int32_t max_blocks,
                           const int32_t* prefix_len, int32_t B, int32_t T, int32_t n_heads, int32_t n_kv_heads,
                           int32_t head_dim, int32_t n_blocks, int32_t max_prefix, int32_t dtype, float scale,
                           void* workspace, size_t ws_bytes, void* out, int32_t* status_dev, void* stream);

/* Bytes of device scratch for tree_sample with these sizes. */
int32_t tree_sample_workspace_bytes(int32_t B, int32_t T, int32_t V, size_t* h_bytes);

/* A token for every row of logits [T][V] (fp32; any number of rows per sequence), for accept_path to compare drafts with (its
 * argmax_out, with logits NULL).  rules[B][4] = temperature, top-k, top-p, min-p of a sequence; uniform[T]: a random number of
 * [0, 1) per row (kept to 0 .. 1 - 2^-24, NaN: 0).  Where nodes of one position are given that position's number, what is
 * accepted equals token-by-token sampling with the same numbers.
 * Tokens are taken in order: larger logits first, of equal ones the lowest index first.  A token's weight is
 * exp((x - largest x) / temperature), held as a whole number of 2^-38, rounded to nearest; sums of weights are exact.
 *   top-k k >= 1 (of a number with a fraction the whole part): the first k tokens; less: all.
 *   top-p p < 1: of these the fewest first ones whose weights' sum is at least ceil(p * sum of these); p <= 0: the first one.
 *   min-p m > 0: of these those of weight ceil(m * 2^38) or more; m > 1: as 1.
 *   target = floor(uniform * sum of the kept); the token is the first one with which the running sum exceeds target.
 * Products in 64-bit floating point.  temperature 0: the first token, whatever the other rules.
 * -infinity and NaN are no tokens: a row of nothing else gets token -1, probability 0.  An infinity is a largest x, others
 * then weigh nothing.  prob_out[T] (may be NULL): the token's share of the sum of the kept.
 * V at most 2^24.  Left as they were, and status 1: rows outside [0, T), a temperature that is negative or not finite, a rule
 * that is NaN. */
int32_t tree_sample(const float* logits, const int32_t* node_off, int32_t B, int32_t T, int32_t V, const float* rules,
                    const float* uniform, int32_t* token_out, float* prob_out, void* workspace, size_t ws_bytes,
                    int32_t* status_dev, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* TRJACOBI_H */
