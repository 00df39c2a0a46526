// Logits of tree nodes after penalties, biases and masks, with the greedy prediction.
//
// One pass over [T][V] fp32.  A workgroup owns SLICE tokens of the vocabulary, four per thread, for some
// rows of one sequence.  What all rows of the sequence share (how often a token occurs in the committed text,
// its bias) it works out once: it scans the text, counts the tokens of its slice in LDS (integers, so the
// order of the atomics does not matter), and every thread keeps the counts of its four tokens in
// registers.  Per row remain the drafts above the node, of which few fall into a slice.
// Every step is rounded by itself (no fused multiply-add), so that a prediction does not depend on
// how the compiler joins them.
// Bytes: 4 V read and, where they are kept, 4 V written per row.  Rows come in batches of four, asked for together,
// the first while the text is scanned.  69 rows over 128256 tokens, 72 MB, take 24 us = 3.0 TB/s; 16 x 64 rows over 32000
// tokens without output, 135 MB, 56 us = 2.4 TB/s, 45 of it without any rule.  Some 150 vector instructions per row and
// wavefront, by the counters, are 32 us of that; a quarter fewer of them gained nothing (60 us: rows under drafts apart), nor did one more
// batch on its way (59; with more registers than four workgroups per compute unit have, 80), nor a wavefront per row
// and 1024 tokens (66).
#include <algorithm>

#include "kernels.h"
#include "q8.h"
#include "tree_anc.h"

namespace trj {

constexpr int LG_THREADS = 256, LG_SLICE = 4 * LG_THREADS, LG_BATCH = 4, LG_WGS = 1024;
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef int i32x4_any __attribute__((ext_vector_type(4), aligned(4)));  // rows of odd length start anywhere

struct LogitsBatch {  // four tokens of each of some rows, with the words of their masks
  float x[LG_BATCH][4];
  uint32_t words[LG_BATCH];
};
struct LogitsArgs {
  const float* x;
  const int32_t *tok, *parent, *node_off;
  int B, T, V;
  const int32_t *ctx, *ctx_off, *gen_start;
  int n_ctx, n_bias;
  const float* pen;
  const int32_t* bias_tok;
  const float* bias_val;
  const int32_t* bias_off;
  const uint32_t* allowed;
  float* out;
  int32_t* argmax;
  uint64_t* cand;  // [T][slices] if there are several
  int32_t* status;
  int rows;  // per workgroup
};

// larger value first, then lower index; 0: no token.  NaN is below all numbers, the zeros are equal
__device__ inline uint64_t pick_key(float x, int i) {
  const uint32_t u = __float_as_uint(x + 0.f);
  const uint32_t ord = x != x ? 0u : (u >> 31 ? ~u : u | 0x80000000u);
  return (uint64_t)ord << 32 | (uint32_t)~i;
}
__device__ inline uint64_t wave_max_key(uint64_t k) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    const uint64_t u = (uint64_t)(uint32_t)__shfl_xor((int)(k >> 32), o) << 32 | (uint32_t)__shfl_xor((int)k, o);
    k = u > k ? u : k;
  }
  return k;
}
// The largest of all lanes for four values at once, NaN passed over while there is a number.  The four take turns,
// which covers the two instructions that have to lie between a register's write and its move between lanes.
__device__ inline void wave_max4(float (&x)[4]) {
#define TRJ_STEP(MOVE)                                                                                    \
  "v_max_f32_dpp %0, %0, %0 " MOVE "\n v_max_f32_dpp %1, %1, %1 " MOVE "\n v_max_f32_dpp %2, %2, %2 " MOVE \
  "\n v_max_f32_dpp %3, %3, %3 " MOVE "\n "
  asm("s_nop 1\n " TRJ_STEP("row_shr:1 row_mask:0xf bank_mask:0xf") TRJ_STEP("row_shr:2 row_mask:0xf bank_mask:0xf")
          TRJ_STEP("row_shr:4 row_mask:0xf bank_mask:0xf") TRJ_STEP("row_shr:8 row_mask:0xf bank_mask:0xf")
              TRJ_STEP("row_bcast:15 row_mask:0xa bank_mask:0xf") TRJ_STEP("row_bcast:31 row_mask:0xc bank_mask:0xf")
      : "+v"(x[0]), "+v"(x[1]), "+v"(x[2]), "+v"(x[3]));
#undef TRJ_STEP
#pragma unroll
  for (int u = 0; u < 4; ++u) x[u] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x[u]), 63));
}
// The best of 256 tokens from `first` on, lane l's those from first + 4 l; tokens that are not allowed are -infinity.
// top: the largest of all.
__device__ inline uint64_t wave_pick(const float (&x)[4], uint32_t may, int first, float top) {
  if (top > -INFINITY) {  // the first token that has it
    uint32_t at = ~0u;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint64_t have = __ballot(x[e] == top);
      if (have) at = min(at, 4u * __builtin_ctzll(have) + e);
    }
    return pick_key(top, first + (int)at);
  }
  uint64_t k = 0;  // nothing but -infinity, NaN and what is not allowed
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint64_t u = (may >> e) & 1 ? pick_key(x[e], first + 4 * (int)(threadIdx.x & 63) + e) : 0;
    k = u > k ? u : k;
  }
  return wave_max_key(k);
}
// a where m's bits are set, b where not; all of them or none are
__device__ inline float choose(uint32_t m, float a, float b) {
  return __uint_as_float((m & __float_as_uint(a)) | (~m & __float_as_uint(b)));
}
__device__ inline uint64_t uniform(uint64_t x) {
  return (uint64_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)x);
}
__device__ inline int picked(uint64_t key) { return key == 0 ? -1 : (int)~(uint32_t)key; }

// rows of sequence s, -1: malformed offsets.  All of them are asked for at once.
__device__ inline int logits_rows(const LogitsArgs& a, int s) {
  const int r0 = a.node_off[s], r1 = a.node_off[s + 1];
  int c0 = 0, c1 = 0, b0 = 0, b1 = 0;
  if (a.ctx && a.pen) c0 = a.ctx_off[s], c1 = a.ctx_off[s + 1];
  if (a.bias_off) b0 = a.bias_off[s], b1 = a.bias_off[s + 1];
  const bool bad = (r0 < 0) | (r1 < r0) | (r1 > a.T) | (r1 - r0 > TRJ_N_MAX) | (c0 < 0) | (c1 < c0) | (c1 > a.n_ctx) | (b0 < 0) | (b1 < b0) |
                   (b1 > a.n_bias);
  return bad ? -1 : r1 - r0;
}

__global__ __launch_bounds__(LG_THREADS, 4) void tree_logits_kernel(LogitsArgs a) {
  __shared__ int seen_n[LG_SLICE], made_n[LG_SLICE], bias_at[LG_SLICE];
  __shared__ __align__(16) uint32_t above[TRJ_N_MAX][4];  // drafts of this slice on the path to a node
  __shared__ uint64_t under[2];             // nodes below such drafts
  __shared__ int draft[TRJ_N_MAX];          // a draft's place in the slice
  __shared__ uint64_t best[TRJ_N_MAX][LG_THREADS / 64];
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  const int v0 = blockIdx.x * LG_SLICE, mine = v0 + 4 * tid;
  const int words = (a.V + 31) >> 5;
  const uint32_t there = mine >= a.V ? 0u : mine + 4 <= a.V ? 15u : (1u << (a.V - mine)) - 1u;  // tokens of the vocabulary

  if (blockIdx.x == 0 && blockIdx.y == 0) {  // sequences without rows
    for (int s = tid; s < a.B; s += LG_THREADS) {
      const int n = logits_rows(a, s);
      if (n <= 0) a.status[s] = n < 0;
    }
  }
  for (int y = blockIdx.y;; y += gridDim.y) {
    int s, nth;
    if (!find_seq(y, a.B, [&](int q) { return max(0, (logits_rows(a, q) + a.rows - 1) / a.rows); }, s, nth)) return;
    const int r0 = a.node_off[s], n = a.node_off[s + 1] - r0, parts = (n + a.rows - 1) / a.rows,
              per = (n + parts - 1) / parts, i0 = min(n, nth * per), i1 = min(n, i0 + per);  // even parts
    auto load = [&](LogitsBatch& b, int ib) {
#pragma unroll
      for (int u = 0; u < LG_BATCH; ++u) {  // (the last row again behind the end)
        const size_t t = r0 + min(ib + u, i1 - 1);
        const float* src = a.x + t * a.V + mine;
        if (mine + 4 <= a.V) {
          const f32x4_any v = *reinterpret_cast<const f32x4_any*>(src);
#pragma unroll
          for (int e = 0; e < 4; ++e) b.x[u][e] = v[e];
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) b.x[u][e] = mine + e < a.V ? src[e] : 0.f;
        }
        b.words[u] = ~0u;
        if (a.allowed && mine < a.V) b.words[u] = a.allowed[t * words + (mine >> 5)];
      }
    };
    LogitsBatch next;
    load(next, i0);  // while the text is scanned
    const TreeParents par = load_parents(a.parent, r0, n);
    const bool ok = tree_valid(par, n);
    if (blockIdx.x == 0 && nth == 0 && tid == 0) a.status[s] = !ok;
    if (!ok) continue;  // uniform over the workgroup

    int made[4] = {0, 0, 0, 0};
    uint32_t seen[4] = {0, 0, 0, 0};  // all bits or none
    float bias[4] = {0.f, 0.f, 0.f, 0.f}, rep = 1.f, freq = 0.f, pres = 0.f;
    uint64_t below[2] = {0, 0};
    if (a.pen || a.bias_off) {
      for (int k = tid; k < LG_SLICE; k += LG_THREADS) seen_n[k] = made_n[k] = bias_at[k] = 0;
      __syncthreads();
      if (a.pen) {
        rep = a.pen[3 * s], freq = a.pen[3 * s + 1], pres = a.pen[3 * s + 2];
        if (a.ctx) {
          const int c0 = a.ctx_off[s], c1 = a.ctx_off[s + 1], g0 = a.gen_start[s];
          for (int k0 = c0 + 4 * tid; k0 < c1; k0 += 16 * LG_THREADS) {  // 16 tokens of a thread together
            i32x4_any t[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
              const int k = k0 + u * 4 * LG_THREADS;
              if (k + 4 <= c1) t[u] = *reinterpret_cast<const i32x4_any*>(a.ctx + k);
              else
#pragma unroll
                for (int e = 0; e < 4; ++e) t[u][e] = k + e < c1 ? a.ctx[k + e] : -1;
            }
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const int v = t[u][e] - v0;
                if (t[u][e] < 0 || (unsigned)v >= (unsigned)LG_SLICE) continue;
                atomicAdd(&seen_n[v], 1);
                if (k0 + u * 4 * LG_THREADS + e - c0 >= g0) atomicAdd(&made_n[v], 1);
              }
          }
        }
        if (wv == 0) {  // the drafts of this slice, and where they lie above a node
          uint32_t in[4];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int i = lane + 64 * h;
            const int t = i > 0 && i < n ? a.tok[r0 + i] : -1, v = t - v0;
            const bool here = t >= 0 && t < a.V && (unsigned)v < (unsigned)LG_SLICE;
            draft[i] = v;
            const uint64_t b = __ballot(here);
            in[2 * h] = (uint32_t)b;
            in[2 * h + 1] = (uint32_t)(b >> 32);
          }
          const TreeBits bits = tree_bits(par, n);
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int k = 0; k < 4; ++k) above[lane + 64 * h][k] = (uint32_t)bits.w[k][h] & in[k];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            uint32_t any = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) any |= (uint32_t)bits.w[k][h] & in[k];
            const uint64_t b = __ballot(any != 0);
            if (lane == 0) under[h] = b;
          }
        }
      }
      if (a.bias_off) {
        const int c0 = a.bias_off[s], c1 = a.bias_off[s + 1];
        for (int k = c0 + tid; k < c1; k += LG_THREADS) {
          const int v = a.bias_tok[k] - v0;
          if (a.bias_tok[k] >= 0 && (unsigned)v < (unsigned)LG_SLICE) atomicMax(&bias_at[v], k - c0 + 1);
        }
      }
      __syncthreads();
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        seen[e] = seen_n[4 * tid + e] ? ~0u : 0u;
        made[e] = made_n[4 * tid + e];
        const int at = bias_at[4 * tid + e];
        if (at > 0) bias[e] = a.bias_val[a.bias_off[s] + at - 1];
      }
      if (a.pen) below[0] = uniform(under[0]), below[1] = uniform(under[1]);
    }
    // x / rep from the rounded reciprocal, corrected twice with the exact remainder: the second correction rounds
    // as the division does, as long as nothing leaves the range of normal numbers
    const float one_rep = 1.f / rep;
    const bool plain_rep = rep >= 0x1p-30f && rep <= 0x1p30f;
    float freqs[4], press[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      freqs[e] = freq * (float)made[e];
      press[e] = made[e] ? pres : 0.f;
    }
    for (int ib = i0; ib < i1; ib += LG_BATCH) {
#pragma clang fp contract(off)
      float x[LG_BATCH][4];
      uint32_t may[LG_BATCH];
#pragma unroll
      for (int u = 0; u < LG_BATCH; ++u) {
        const int i = ib + u;
        may[u] = (next.words[u] >> (mine & 31)) & there;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[u][e] = next.x[u][e];
        if (a.pen && i < i1) {
          uint32_t had[4];
          float f[4], p[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) had[e] = seen[e], f[e] = freqs[e], p[e] = press[e];
          if ((below[i >> 6] >> (i & 63)) & 1) {  // uniform, and rare
            int more[4] = {0, 0, 0, 0};
#pragma unroll
            for (int k = 0; k < 4; ++k)
              for (uint32_t m = __builtin_amdgcn_readfirstlane(above[i][k]); m; m &= m - 1) {
                const int v = draft[32 * k + __builtin_ctz(m)];
#pragma unroll
                for (int e = 0; e < 4; ++e) more[e] += v == 4 * tid + e;
              }
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (more[e]) {
                had[e] = ~0u;
                f[e] = freq * (float)(made_n[4 * tid + e] + more[e]);
                p[e] = pres;
              }
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float y = x[u][e];
            float q = y * one_rep;
            q = __builtin_fmaf(__builtin_fmaf(-q, rep, y), one_rep, q);
            q = __builtin_fmaf(__builtin_fmaf(-q, rep, y), one_rep, q);
            if (y > 0.f && !(plain_rep && y >= 0x1p-60f && y <= 0x1p60f)) q = y / rep;  // rare
            x[u][e] = choose(had[e], y > 0.f ? q : y * rep, y) - f[e];
            x[u][e] = x[u][e] - p[e];
          }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (a.bias_off) x[u][e] = x[u][e] + bias[e];
          x[u][e] = choose((uint32_t)((int)(may[u] << (31 - e)) >> 31), x[u][e], -INFINITY);
        }
      }
      if (ib + LG_BATCH < i1) load(next, ib + LG_BATCH);
      if (a.out)
#pragma unroll
        for (int u = 0; u < LG_BATCH; ++u) {
          if (ib + u >= i1) break;
          float* dst = a.out + (size_t)(r0 + ib + u) * a.V + mine;
          if (mine + 4 <= a.V) {
            *reinterpret_cast<f32x4_any*>(dst) = f32x4_any{x[u][0], x[u][1], x[u][2], x[u][3]};
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (mine + e < a.V) dst[e] = x[u][e];
          }
        }
      if (a.argmax) {
        float top[LG_BATCH];
#pragma unroll
        for (int u = 0; u < LG_BATCH; ++u) top[u] = fmaxf(fmaxf(x[u][0], x[u][1]), fmaxf(x[u][2], x[u][3]));
        wave_max4(top);
#pragma unroll
        for (int u = 0; u < LG_BATCH; ++u) {
          if (ib + u >= i1) break;
          const uint64_t k = wave_pick(x[u], may[u], v0 + 256 * wv, top[u]);
          if (lane == 0) best[ib + u - i0][wv] = k;
        }
      }
    }
    __syncthreads();
    if (a.argmax)
      for (int i = tid; i < i1 - i0; i += LG_THREADS) {
        uint64_t k = best[i][0];
#pragma unroll
        for (int w = 1; w < LG_THREADS / 64; ++w) k = best[i][w] > k ? best[i][w] : k;
        const size_t t = r0 + i0 + i;
        if (gridDim.x == 1) a.argmax[t] = picked(k);
        else a.cand[t * gridDim.x + blockIdx.x] = k;
      }
    __syncthreads();
  }
}

// The best of a row's candidates, a wavefront per row.
__global__ __launch_bounds__(256) void logits_pick_kernel(LogitsArgs a, int slices) {
  const int lane = threadIdx.x & 63, w = blockIdx.x * 4 + (threadIdx.x >> 6);
  int s, i;
  if (!find_seq(w, a.B, [&](int q) { return max(0, logits_rows(a, q)); }, s, i)) return;
  const int r0 = a.node_off[s];
  if (a.status[s]) return;  // (as the launch before has found)
  uint64_t k = 0;
  for (int c = lane; c < slices; c += 64) {
    const uint64_t u = a.cand[(size_t)(r0 + i) * slices + c];
    k = u > k ? u : k;
  }
  k = wave_max_key(k);
  if (lane == 0) a.argmax[r0 + i] = picked(k);
}

static int logits_slices(int V) { return (V + LG_SLICE - 1) / LG_SLICE; }
size_t tree_logits_ws_bytes(int T, int V) {
  const int n = logits_slices(V);
  return n > 1 ? (size_t)T * n * sizeof(uint64_t) : 0;
}

int launch_tree_logits(const float* x, const int32_t* tok, const int32_t* parent, const int32_t* node_off, int B, int T, int V,
                       const int32_t* ctx, int n_ctx, const int32_t* ctx_off, const int32_t* gen_start, const float* pen,
                       const int32_t* bias_tok, const float* bias_val, int n_bias, const int32_t* bias_off, const uint32_t* allowed,
                       float* out, int32_t* argmax, uint64_t* cand, int32_t* status, hipStream_t st) {
  const int slices = logits_slices(V);
  // rows per workgroup, at most: the chip holds four workgroups per compute unit, and none is to wait for another to end
  // (rounded down instead, 69 nodes over 128256 tokens took 29 us instead of 24; half as many workgroups 80 us instead
  // of 56 for 16 x 64 nodes over 32000 tokens, twice as many 62)
  const int rows = (int)std::min(((long)slices * T + LG_WGS - 1) / LG_WGS, (long)TRJ_N_MAX);
  const LogitsArgs a{x, tok, parent, node_off, B, T, V, ctx, ctx_off, gen_start, n_ctx, n_bias, pen, bias_tok, bias_val, bias_off, allowed,
                     out, argmax, cand, status, rows};
  const dim3 grid(slices, std::min((long)T / rows + B, 65535l));
  tree_logits_kernel<<<grid, LG_THREADS, 0, st>>>(a);
  int rc = check_launch();
  if (rc != TRJ_OK || !argmax || slices == 1) return rc;
  logits_pick_kernel<<<(T + 3) / 4, 256, 0, st>>>(a, slices);
  return check_launch();
}

}  // namespace trj
