// C-ABI entry points for serving from the paged 8-bit cache: argument checks and launches.
#include <cstdint>

#include "kernels.h"
#include "q8.h"

using namespace trj;

#define TRJ_TRY(expr)              \
  do {                             \
    int rc_ = (expr);              \
    if (rc_ != TRJ_OK) return rc_; \
  } while (0)

static int check_serve_batch(int B, int T, int max_blocks, int n_blocks) {
  if (B < 1 || B > TRJ_SERVE_MAX_SEQS || T < 0 || max_blocks < 1 || n_blocks < 1 || n_blocks > Q8_MAX_PAGES ||
      (int64_t)B * max_blocks > INT32_MAX)
    return TRJ_ERR_BAD_SHAPE;
  return TRJ_OK;
}
// elements from row to row: 32 rows' offsets stay in 32 bits
static bool bad_stride(int stride, int64_t least) { return stride < least || (stride & 7) || stride > 1 << 24; }
static bool on16(const void* p) { return ((uintptr_t)p & 15) == 0; }

extern "C" {

int32_t kv_block_tables(int32_t* block_table, int32_t max_blocks, const int32_t* held, const int32_t* prefix_len,
                        const int32_t* node_off, int32_t B, int32_t T, int32_t* free_list, int32_t n_blocks,
                        const int32_t* free_count, int32_t* held_out, int32_t* free_count_out, int32_t* row_slot,
                        int32_t* status_dev, void* stream) {
  if (!block_table || !held || !prefix_len || !node_off || !free_list || !free_count || !held_out || !free_count_out ||
      (T > 0 && !row_slot) || !status_dev)
    return TRJ_ERR_NULLPTR;
  TRJ_TRY(check_serve_batch(B, T, max_blocks, n_blocks));
  if (held_out < held + B && held < held_out + B) return TRJ_ERR_BAD_SHAPE;
  if (free_count_out == free_count) return TRJ_ERR_BAD_SHAPE;
  return launch_block_tables(block_table, max_blocks, held, prefix_len, node_off, B, T, free_list, n_blocks, free_count,
                             held_out, free_count_out, row_slot, status_dev, (hipStream_t)stream);
}

int32_t kv_append_q8(void* k_pool, void* v_pool, float* k_scale, float* v_scale, const void* k_rows, const void* v_rows,
                     int32_t row_stride, size_t row_layer_stride, const int32_t* path, const int32_t* accept_len,
                     const int32_t* node_off, const int32_t* block_table, int32_t max_blocks, const int32_t* prefix_len,
                     int32_t B, int32_t T, int32_t n_layers, int32_t n_kv_heads, int32_t head_dim, int32_t n_blocks,
                     int32_t dtype, int32_t* new_len, int32_t* status_dev, void* stream) {
  if (!k_pool || !v_pool || !k_scale || !v_scale || !k_rows || !v_rows || !node_off || !block_table || !prefix_len ||
      !new_len || !status_dev || (path && !accept_len))
    return TRJ_ERR_NULLPTR;
  if (dtype != TRJ_BF16) return TRJ_ERR_BAD_DTYPE;
  TRJ_TRY(check_serve_batch(B, T, max_blocks, n_blocks));
  if (T < 1 || n_layers < 1 || n_layers > 32767 || n_kv_heads < 1 || n_kv_heads > 65535 ||
      (head_dim != 64 && head_dim != 128) || bad_stride(row_stride, n_kv_heads * (int64_t)head_dim) ||
      (row_layer_stride & 7) || !on16(k_pool) || !on16(v_pool) || !on16(k_rows) || !on16(v_rows))
    return TRJ_ERR_BAD_SHAPE;
  if (new_len < prefix_len + B && prefix_len < new_len + B) return TRJ_ERR_BAD_SHAPE;
  return launch_kv_append_q8(k_pool, v_pool, k_scale, v_scale, k_rows, v_rows, row_stride, row_layer_stride, path,
                             accept_len, node_off, block_table, max_blocks, prefix_len, B, T, n_layers, n_kv_heads, head_dim,
                             n_blocks, new_len, status_dev, (hipStream_t)stream);
}

static int check_attention(int B, int T, int n_heads, int n_kv_heads, int head_dim, int max_prefix) {
  if (B < 1 || B > TRJ_SERVE_MAX_SEQS || T < 1 || n_heads < 1 || n_kv_heads < 1 || n_heads % n_kv_heads != 0 ||
      n_heads > 65535 || (head_dim != 64 && head_dim != 128) || max_prefix < 0)
    return TRJ_ERR_BAD_SHAPE;
  if ((int64_t)T > (int64_t)B * TRJ_N_MAX) return TRJ_ERR_TREE_TOO_LARGE;
  return TRJ_OK;
}

int32_t tree_attention_q8_workspace_bytes(int32_t B, int32_t T, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                                          int32_t max_prefix, size_t* h_bytes) {
  if (!h_bytes) return TRJ_ERR_NULLPTR;
  TRJ_TRY(check_attention(B, T, n_heads, n_kv_heads, head_dim, max_prefix));
  *h_bytes = align_up(attn_q8_ws_floats(B, T, n_heads / n_kv_heads, n_kv_heads, head_dim, max_prefix) * 4 + 16, 256);
  return TRJ_OK;
}

int32_t tree_attention_q8(const void* q_rows, int32_t q_stride, const void* k_pool, const void* v_pool,
                          const float* k_scale, const float* v_scale, const void* k_rows, const void* v_rows,
                          int32_t row_stride, const int32_t* parent, const int32_t* node_off, const int32_t* block_table,
                          int32_t max_blocks, const int32_t* prefix_len, int32_t B, int32_t T, int32_t n_heads,
                          int32_t n_kv_heads, int32_t head_dim, int32_t n_blocks, int32_t max_prefix, int32_t dtype,
                          float scale, void* workspace, size_t ws_bytes, void* out, int32_t* status_dev, void* stream) {
  if (!q_rows || !k_pool || !v_pool || !k_scale || !v_scale || !k_rows || !v_rows || !parent || !node_off || !block_table ||
      !prefix_len || !workspace || !out || !status_dev)
    return TRJ_ERR_NULLPTR;
  if (dtype != TRJ_BF16) return TRJ_ERR_BAD_DTYPE;
  TRJ_TRY(check_attention(B, T, n_heads, n_kv_heads, head_dim, max_prefix));
  TRJ_TRY(check_serve_batch(B, T, max_blocks, n_blocks));
  // scores are worked out to base 2
  if (!(scale > 0.f) || !(scale * LOG2E < INFINITY) || bad_stride(q_stride, n_heads * (int64_t)head_dim) ||
      bad_stride(row_stride, n_kv_heads * (int64_t)head_dim) || !on16(q_rows) || !on16(k_pool) || !on16(v_pool) ||
      !on16(k_rows) || !on16(v_rows) || !on16(out))
    return TRJ_ERR_BAD_SHAPE;
  // the scratch starts at the workspace's first multiple of 16
  const size_t skip = (16 - ((uintptr_t)workspace & 15)) & 15;
  if (ws_bytes < skip ||
      ws_bytes - skip < attn_q8_ws_floats(B, T, n_heads / n_kv_heads, n_kv_heads, head_dim, max_prefix) * 4)
    return TRJ_ERR_WORKSPACE_TOO_SMALL;
  return launch_tree_attn_q8((const uint16_t*)q_rows, q_stride, k_pool, v_pool, k_scale, v_scale, (const uint16_t*)k_rows,
                             (const uint16_t*)v_rows, row_stride, parent, node_off, block_table, max_blocks, prefix_len, B, T,
                             n_heads, n_kv_heads, head_dim, n_blocks, max_prefix, scale,
                             reinterpret_cast<float*>((char*)workspace + skip), (uint16_t*)out, status_dev,
                             (hipStream_t)stream);
}

static int check_logits(int B, int T, int V) {
  if (B < 1 || B > TRJ_SERVE_MAX_SEQS || T < 1 || V < 1 || V > (1 << 24)) return TRJ_ERR_BAD_SHAPE;
  if ((int64_t)T > (int64_t)B * TRJ_N_MAX) return TRJ_ERR_TREE_TOO_LARGE;
  return TRJ_OK;
}
int32_t tree_logits_workspace_bytes(int32_t B, int32_t T, int32_t V, size_t* h_bytes) {
  if (!h_bytes) return TRJ_ERR_NULLPTR;
  TRJ_TRY(check_logits(B, T, V));
  *h_bytes = align_up(tree_logits_ws_bytes(T, V) + 16, 256);
  return TRJ_OK;
}

int32_t tree_logits(const float* logits, const int32_t* tok, const int32_t* parent, const int32_t* node_off, int32_t B,
                    int32_t T, int32_t V, const int32_t* ctx, int32_t n_ctx, const int32_t* ctx_off, const int32_t* gen_start,
                    const float* penalties, const int32_t* bias_tok, const float* bias_val, int32_t n_bias, const int32_t* bias_off,
                    const uint32_t* allowed, float* logits_out, int32_t* argmax_out, void* workspace, size_t ws_bytes,
                    int32_t* status_dev, void* stream) {
  if (!logits || !parent || !node_off || (penalties && !tok) || (ctx && (!ctx_off || !gen_start)) ||
      (bias_off && (!bias_tok || !bias_val)) || (!logits_out && !argmax_out) || !workspace || !status_dev)
    return TRJ_ERR_NULLPTR;
  TRJ_TRY(check_logits(B, T, V));
  if ((ctx && (n_ctx < 0 || n_ctx > 1 << 30)) || (bias_off && (n_bias < 0 || n_bias > 1 << 30))) return TRJ_ERR_BAD_SHAPE;
  const size_t skip = (16 - ((uintptr_t)workspace & 15)) & 15;
  if (ws_bytes < skip || ws_bytes - skip < tree_logits_ws_bytes(T, V)) return TRJ_ERR_WORKSPACE_TOO_SMALL;
  return launch_tree_logits(logits, tok, parent, node_off, B, T, V, ctx, n_ctx, ctx_off, gen_start, penalties, bias_tok, bias_val,
                            n_bias, bias_off, allowed, logits_out, argmax_out, reinterpret_cast<uint64_t*>((char*)workspace + skip),
                            status_dev, (hipStream_t)stream);
}

}  // extern "C"
