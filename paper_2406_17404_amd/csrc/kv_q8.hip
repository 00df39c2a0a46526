// Pages that follow lengths, and the append that quantises rows into the paged 8-bit cache.
#include <algorithm>

#include "kernels.h"
#include "q8.h"

namespace trj {

// ------------------------------------------------------------------ block tables and row slots
// Integer work on a few KiB, bound by one launch and its chain of dependent loads.  Every
// workgroup scans all sequences by itself (20 bytes each, from L2) rather than wait for a first
// launch to do it, then the workgroups share out table entries, released pages and rows.
// Nothing that one of them reads is written by another: pages taken by this call that this
// call released are read from the table row they leave, not from the stack.
// 16 sequences take 4.0 us, 1024 take 10.1 (four sequences of a thread asked for together, their first rows in
// LDS: 4.6 and 9.5).
constexpr int TABLES_THREADS = 256;
struct SeqPages {  // of one sequence
  int held, want, bad;
};
// of a sequence that need not be well-formed: the table entries that its positions reach
__device__ inline int pages_wanted(const int32_t* prefix_len, const int32_t* node_off, int max_blocks, int s) {
  const long rows = node_off[s + 1] - (long)node_off[s], L = prefix_len[s];
  return rows < 0 || L < 0 ? 0 : (int)min((L + rows + TRJ_KV_BLOCK - 1) / TRJ_KV_BLOCK, (long)max_blocks);
}
__device__ inline SeqPages seq_pages(const int32_t* held, const int32_t* prefix_len, const int32_t* node_off, int T,
                                     int max_blocks, int s) {
  const int h = held[s], L = prefix_len[s], r0 = node_off[s], r1 = node_off[s + 1];
  const long want = ((long)L + (r1 - (long)r0) + TRJ_KV_BLOCK - 1) / TRJ_KV_BLOCK;
  const bool bad = h < 0 || h > max_blocks || L < 0 || r0 < 0 || r1 < r0 || r1 > T ||
                   want > q8_pages_at_most(max_blocks);
  return bad ? SeqPages{h, h, 1} : SeqPages{h, (int)want, 0};
}

__global__ __launch_bounds__(TABLES_THREADS) void block_tables_kernel(
    int32_t* block_table, int max_blocks, const int32_t* held, const int32_t* prefix_len, const int32_t* node_off,
    int B, int T, int32_t* free_list, int n_blocks, const int32_t* free_count, int32_t* held_out,
    int32_t* free_count_out, int32_t* row_slot, int32_t* status) {
  // per sequence: pages needed and released by those before it; two further words close the lists
  extern __shared__ int smem[];
  int* need_at = smem;
  int* give_at = smem + B + 1;
  __shared__ int part[2][TABLES_THREADS / 64];
  __shared__ int mono, any_bad;
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  if (tid == 0) mono = 1, any_bad = 0;
  int base_need = 0, base_give = 0;
  for (int s0 = 0; s0 < B; s0 += TABLES_THREADS) {
    const int s = s0 + tid;
    SeqPages p{0, 0, 0};
    if (s < B) p = seq_pages(held, prefix_len, node_off, T, max_blocks, s);
    const int need = max(p.want - p.held, 0), give = max(p.held - p.want, 0);
    const int a = wave_scan(need), b = wave_scan(give);
    __syncthreads();
    if (lane == 63) part[0][wv] = a, part[1][wv] = b;
    if (s < B && node_off[s + 1] < node_off[s]) mono = 0;
    if (p.bad) any_bad = 1;
    __syncthreads();
    int before_need = base_need, before_give = base_give;
#pragma unroll
    for (int w = 0; w < TABLES_THREADS / 64; ++w) {
      if (w < wv) before_need += part[0][w], before_give += part[1][w];
      base_need += part[0][w];
      base_give += part[1][w];
    }
    if (s < B) {
      need_at[s] = before_need + a - need;
      give_at[s] = before_give + b - give;
    }
  }
  if (tid == 0) need_at[B] = base_need, give_at[B] = base_give;
  __syncthreads();

  int have0 = free_count[0];
  if (have0 < 0 || have0 > n_blocks) have0 = 0;
  const int have = (int)min((long)have0 + base_give, (long)n_blocks);
  // the sequence whose list entry is x: last s with at[s] <= x among those with entries
  auto owner = [&](const int* at, int x) {
    int lo = 0, hi = B;  // at[lo] <= x < at[hi]
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (at[mid] <= x) lo = mid;
      else hi = mid;
    }
    return lo;
  };
  auto stacked = [&](int i) {  // the page at place i of the stack once the released ones lie on it
    if (i < have0) return free_list[i];
    const int s = owner(give_at, i - have0);
    const SeqPages p = seq_pages(held, prefix_len, node_off, T, max_blocks, s);
    return block_table[(size_t)s * max_blocks + p.want + (i - have0 - give_at[s])];
  };
  auto served = [&](int s, const SeqPages& p) { return !p.bad && (p.want <= p.held || need_at[s + 1] <= have); };
  const int first = blockIdx.x * TABLES_THREADS + tid, step = gridDim.x * TABLES_THREADS;
  const int needed = base_need, given = have - have0;
  // pages taken: entry x of the list belongs to its sequence if all of that sequence's entries are there; else no page
  // is where it wanted one, not the one that the sequence gave back from there earlier and another may own
  for (unsigned x = first; x < (unsigned)needed; x += step) {
    const int s = owner(need_at, (int)x);
    block_table[(size_t)s * max_blocks + held[s] + (x - need_at[s])] = need_at[s + 1] <= have ? stacked(have - 1 - (int)x) : -1;
  }
  for (int x = first; x < given; x += step) free_list[have0 + x] = stacked(have0 + x);
  for (int t = first; t < T; t += step) {
    int s = -1;
    if (mono) {  // last s with node_off[s] <= t
      int lo = -1, hi = B;
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (node_off[mid] <= t) lo = mid;
        else hi = mid;
      }
      s = lo;
    } else {  // some range is malformed: the last sequence that has the row and is not
      for (int k = 0; k < B; ++k)
        if (node_off[k] <= t && t < node_off[k + 1] && served(k, seq_pages(held, prefix_len, node_off, T, max_blocks, k))) s = k;
    }
    int slot = -1;
    if (s >= 0 && t < node_off[s + 1]) {
      const SeqPages p = seq_pages(held, prefix_len, node_off, T, max_blocks, s);
      if (served(s, p)) {
        const int pos = prefix_len[s] + t - node_off[s], j = pos / TRJ_KV_BLOCK;
        const int page = j < p.held ? block_table[(size_t)s * max_blocks + j] : stacked(have - 1 - (need_at[s] + j - p.held));
        slot = (int)((unsigned)page * TRJ_KV_BLOCK + pos % TRJ_KV_BLOCK);
      }
    }
    row_slot[t] = slot;
  }
  for (int s = first; s < B; s += step) {
    const SeqPages p = seq_pages(held, prefix_len, node_off, T, max_blocks, s);
    held_out[s] = served(s, p) ? p.want : p.held;
    status[s] = !served(s, p);
  }
  if (any_bad)  // nor are there pages for what is malformed: rare, so all threads look for it together
    for (int s = 0; s < B; ++s) {
      const SeqPages p = seq_pages(held, prefix_len, node_off, T, max_blocks, s);
      if (!p.bad || p.held < 0) continue;
      const unsigned end = pages_wanted(prefix_len, node_off, max_blocks, s);
      for (unsigned j = (unsigned)p.held + first; j < end; j += step) block_table[(size_t)s * max_blocks + j] = -1;
    }
  if (first == 0) {
    int taken = needed;  // the sequences up to the first without room
    if (needed > have) {
      const int s = owner(need_at, have);
      taken = need_at[s];
    }
    free_count_out[0] = have - taken;
  }
}

int launch_block_tables(int32_t* block_table, int max_blocks, const int32_t* held, const int32_t* prefix_len,
                        const int32_t* node_off, int B, int T, int32_t* free_list, int n_blocks,
                        const int32_t* free_count, int32_t* held_out, int32_t* free_count_out, int32_t* row_slot,
                        int32_t* status, hipStream_t st) {
  const long most = (long)B * min(max_blocks, 8) + T;
  const int wgs = (int)min(256l, (most + TABLES_THREADS - 1) / TABLES_THREADS);
  block_tables_kernel<<<max(wgs, 1), TABLES_THREADS, (2 * (size_t)B + 2) * sizeof(int), st>>>(
      block_table, max_blocks, held, prefix_len, node_off, B, T, free_list, n_blocks, free_count, held_out,
      free_count_out, row_slot, status);
  return check_launch();
}

// ------------------------------------------------------------------ append
// A wavefront quantises one page of one head, K or V: 32 x DH values, a lane 4 rows x 8 columns at a time.
//   top = max |x| over the page's new rows;  2^k with top <= 448 * 2^k;  code = e4m3(x * 2^-k)
// With a power of two the products are exact, so a page whose scale grows is requantised by
// multiplying its codes with the (power of two) ratio.  K's bytes are stored as they are; V's, four rows
// to a word, go through LDS, where they meet those of rows that stay.
// Bound by memory for prompts (2 bytes read, 1 written per value), by a chain of latencies for a few rows
// (lengths, page number, rows, codes), so a workgroup finds its page once for several heads and
// layers, and no wavefront waits for another.
// 4096 rows of 32 heads of 128, 101 MB, take 27 us = 3.7 TB/s; the paths of 16 sequences with 6 rows each in 32 layers of 8
// heads 23 us, of which the 53 MB that they move (V pages read and written whole) would need 11; one row 5.8.
// The vector unit's work counts too: with every magnitude and every code checked by itself, and both halves of a page
// worked on whether rows go there or not, the paths took 42 us and the prompt 32.  (A plane asked for while the one
// before it is worked on costs a third of the wavefronts their registers: 29 to 33 us for the paths, 31 for the prompt.)
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
struct AppendArgs {
  uint8_t* pool[2];
  float* scale[2];
  const uint16_t* rows[2];
  int row_stride;
  size_t row_layer_stride;
  const int32_t *path, *accept_len, *node_off, *block_table, *prefix_len;
  int max_blocks, B, T, n_kv_heads, n_blocks;
  int32_t *new_len, *status;
};
// rows to store of sequence s; -1: the sequence is refused
__device__ inline int append_rows(const AppendArgs& a, int s) {
  const int L = a.prefix_len[s], r0 = a.node_off[s], r1 = a.node_off[s + 1];
  int acc = 0;
  if (a.path) acc = a.accept_len[s];
  bool bad = (L < 0) | (r0 < 0) | (r1 < r0) | (r1 > a.T);
  const int n = bad ? 0 : r1 - r0;
  if (a.path) bad |= (n > TRJ_N_MAX) | (acc < 0) | (acc >= n);
  const int m = a.path && !bad ? acc + 1 : n;
  return bad || (long)L + m > (long)q8_pages_at_most(a.max_blocks) * TRJ_KV_BLOCK ? -1 : m;
}
__device__ inline int pages_touched(int L, int m) {
  return m <= 0 ? 0 : (L + m - 1) / TRJ_KV_BLOCK - L / TRJ_KV_BLOCK + 1;
}
// whether the pages that m rows go to exist and the path's entries are nodes (one wavefront, uniform)
__device__ inline bool append_valid(const AppendArgs& a, int s, int L, int m) {
  const int lane = threadIdx.x & 63;
  bool bad = false;
  const int p0 = L / TRJ_KV_BLOCK, p1 = p0 + pages_touched(L, m);
  const int32_t* const table = a.block_table + (size_t)s * a.max_blocks;
  if (p1 - p0 <= 64) {
    if (p0 + lane < p1) bad = (unsigned)table[p0 + lane] >= (unsigned)a.n_blocks;
  } else {  // long prompts: eight entries of a lane are asked for together
    for (int p = p0; p < p1; p += 512) {
      int pages[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) pages[u] = table[min(p + 64 * u + lane, p1 - 1)];
#pragma unroll
      for (int u = 0; u < 8; ++u) bad |= (unsigned)pages[u] >= (unsigned)a.n_blocks;
    }
  }
  if (a.path) {
    const int n = a.node_off[s + 1] - a.node_off[s];
    for (int j = lane; j < m; j += 64) bad = bad || (unsigned)a.path[(size_t)s * TRJ_N_MAX + j] >= (unsigned)n;
  }
  return __ballot(bad) == 0;
}

// the lowest n bytes of a word, all of them from 4 on
__device__ inline uint32_t bytes_below(int n) { return n <= 0 ? 0u : n >= 4 ? ~0u : (1u << (8 * n)) - 1u; }
// place of 16-byte group g of a V page in LDS: the columns that a wavefront writes at once would meet a quarter of
// the banks
__device__ inline int v_group_place(int g) { return g ^ ((g >> 3) & 3) ^ (((g >> 6) & 1) << 2); }

template <int DH>
__global__ __launch_bounds__(256, 4) void kv_append_kernel(AppendArgs a, int planes) {
  constexpr int C8 = DH / 8, PASSES = 8 * C8 / 64, GROUPS = 2 * DH / 64;  // 16-byte groups of a page per lane
  __shared__ __align__(16) uint8_t tiles[4][32 * DH];
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  uint8_t* const tile = tiles[wv];
  for (int x = blockIdx.x;; x += gridDim.x) {
    int s, nth;
    if (!find_seq(x, a.B, [&](int q) { return pages_touched(a.prefix_len[q], append_rows(a, q)); }, s, nth)) break;
    const int L = a.prefix_len[s], m = append_rows(a, s), r0 = a.node_off[s];
    const int pg = L / TRJ_KV_BLOCK + nth, page = a.block_table[(size_t)s * a.max_blocks + pg];
    const int old_rows = max(0, min(32, L - pg * 32)), end = min(32, L + m - pg * 32);  // new: [old_rows, end)
    int row[PASSES][4];  // of the input, -1: none
#pragma unroll
    for (int p = 0; p < PASSES; ++p)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = (p * 64 + lane) / C8 * 4 + i, j = pg * 32 + r - L;
        row[p][i] = r >= old_rows && r < end ? (a.path ? a.path[(size_t)s * TRJ_N_MAX + j] : j) : -1;
      }
    if (!append_valid(a, s, L, m)) continue;
    for (int pl = blockIdx.y * 4 + wv; pl < planes; pl += gridDim.y * 4) {
      int ln = lane;
      asm("" : "+v"(ln));  // offsets are worked out again for every plane, not held in registers
      const int c0 = ln % C8 * 8;
      const int which = pl & 1, head = (pl >> 1) % a.n_kv_heads, layer = (pl >> 1) / a.n_kv_heads;
      const size_t plane = ((size_t)layer * a.n_kv_heads + head) * a.n_blocks + page;
      float* const scale = a.scale[which] + plane;
      uint8_t* const pool = a.pool[which] + plane * 32 * DH;
      const uint16_t* const src = a.rows[which] + layer * a.row_layer_stride + (size_t)head * DH + c0;
      u32x4 raw[PASSES][4];
#pragma unroll
      for (int p = 0; p < PASSES; ++p)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          raw[p][i] = u32x4{0, 0, 0, 0};
          if (row[p][i] >= 0) raw[p][i] = *reinterpret_cast<const u32x4*>(src + (size_t)(r0 + row[p][i]) * a.row_stride);
        }
      const bool keeps = which == 1 && (old_rows > 0 || end < 32);  // V words hold rows that stay
      u32x4 had[GROUPS];
      if (keeps)
#pragma unroll
        for (int k = 0; k < GROUPS; ++k) had[k] = reinterpret_cast<const u32x4*>(pool)[k * 64 + ln];
      int e_old = Q8_MIN_EXP;
      if (old_rows > 0) e_old = q8_exp_of(*scale);
      // the largest magnitude, two rows' halves at a time; only a page with numbers that are not finite looks at
      // them one by one
      u16x2 pair = {0, 0};
#pragma unroll
      for (int p = 0; p < PASSES; ++p)
#pragma unroll
        for (int i = 0; i < 16; ++i) pair = __builtin_elementwise_max(pair, __builtin_bit_cast(u16x2, raw[p][i >> 2][i & 3] & 0x7fff7fffu));
      uint32_t top = wave_max((uint32_t)max(pair[0], pair[1]) << 16);
      const bool odd_ones = top >= 0x7f800000u;  // uniform
      if (odd_ones) {
        top = 0;
#pragma unroll
        for (int p = 0; p < PASSES; ++p)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const uint32_t w = raw[p][i >> 2][i & 3], lo = (w << 16) & 0x7fffffffu, hi = w & 0x7fff0000u;
            top = max(top, max(lo < 0x7f800000u ? lo : 0u, hi < 0x7f800000u ? hi : 0u));
          }
        top = wave_max(top);
      }
      const int e = max(q8_exp(top), e_old);
      const float inv = q8_pow2(-e), ratio = q8_pow2(max(e_old - e, -126));
      const bool grew = old_rows > 0 && e > e_old;
      if (lane == 0) *scale = q8_pow2(e);
      auto lower = [&](uint32_t codes) {  // earlier codes to the new scale
        const f32x2 p = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false), q = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true);
        return q8_codes(p[0] * ratio, p[1] * ratio) | q8_codes(q[0] * ratio, q[1] * ratio) << 16;
      };
#pragma unroll
      for (int p = 0; p < PASSES; ++p) {
        if (old_rows >= (p + 1) * 4 * 64 / C8 || end <= p * 4 * 64 / C8) {  // no new rows here (uniform)
          if (which == 0 && grew && old_rows > p * 4 * 64 / C8)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              u32x2* const dst = reinterpret_cast<u32x2*>(pool + q8_k_off((p * 64 + ln) / C8 * 4 + i, c0));
              const u32x2 o = *dst;
              *dst = u32x2{lower(o[0]), lower(o[1])};
            }
          continue;
        }
        const int q = (p * 64 + ln) / C8;  // rows 4q ..
        uint32_t code[4][2];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint32_t u = raw[p][i][2 * h], v = raw[p][i][2 * h + 1];
            int c = __builtin_amdgcn_cvt_pk_fp8_f32(__uint_as_float(u << 16) * inv, __uint_as_float(u & 0xffff0000u) * inv, 0, false);
            code[i][h] = __builtin_amdgcn_cvt_pk_fp8_f32(__uint_as_float(v << 16) * inv, __uint_as_float(v & 0xffff0000u) * inv, c, true);
          }
        if (odd_ones)
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const uint32_t u = raw[p][i][2 * h], v = raw[p][i][2 * h + 1];
              code[i][h] = q8_codes(__uint_as_float(u << 16) * inv, __uint_as_float(u & 0xffff0000u) * inv) |
                           q8_codes(__uint_as_float(v << 16) * inv, __uint_as_float(v & 0xffff0000u) * inv) << 16;
            }
        if (which == 0) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            u32x2* const dst = reinterpret_cast<u32x2*>(pool + q8_k_off(4 * q + i, c0));
            if (row[p][i] >= 0) *dst = u32x2{code[i][0], code[i][1]};
            else if (grew && 4 * q + i < old_rows) {
              const u32x2 o = *dst;
              *dst = u32x2{lower(o[0]), lower(o[1])};
            }
          }
        } else {
#pragma unroll
          for (int c = 0; c < 8; ++c) {
            const uint32_t sel = 0x0c0c0400u + 0x0101u * (c & 3);  // byte c % 4 of each of two words
            const uint32_t ab = __builtin_amdgcn_perm(code[1][c >> 2], code[0][c >> 2], sel);
            const uint32_t cd = __builtin_amdgcn_perm(code[3][c >> 2], code[2][c >> 2], sel);
            const int g = q8_v_off(4 * q, c0 + c) >> 4;
            *reinterpret_cast<uint32_t*>(tile + v_group_place(g) * 16 + (q >> 1) * 4) = ab | cd << 16;
          }
        }
      }
      if (which == 1) {
        uint32_t is_new[4], is_old[4];  // bytes of a group's words: rows 8d + 4 ((ln / 32) % 2) ..
#pragma unroll
        for (int d = 0; d < 4; ++d) {
          const int r = 8 * d + 4 * ((ln >> 5) & 1);
          const uint32_t below_old = bytes_below(old_rows - r), below_end = bytes_below(end - r);
          is_old[d] = below_old;
          is_new[d] = below_end & ~below_old;
        }
        if (grew)
#pragma unroll
          for (int k = 0; k < GROUPS; ++k)
#pragma unroll
            for (int d = 0; d < 4; ++d) had[k][d] = (lower(had[k][d]) & is_old[d]) | (had[k][d] & ~is_old[d]);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // this wavefront's words, which it reads itself
#pragma unroll
        for (int k = 0; k < GROUPS; ++k) {
          const int g = k * 64 + ln;
          u32x4 put = *reinterpret_cast<const u32x4*>(tile + v_group_place(g) * 16);
          if (keeps)
#pragma unroll
            for (int d = 0; d < 4; ++d) put[d] = (put[d] & is_new[d]) | (had[k][d] & ~is_new[d]);
          reinterpret_cast<u32x4*>(pool)[g] = put;
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // read before the next page's are written
      }
    }
  }
  if (blockIdx.y == 0) {  // the verdicts
    for (int s = blockIdx.x * 4 + wv; s < a.B; s += gridDim.x * 4) {
      const int m = append_rows(a, s);
      const bool ok = m >= 0 && append_valid(a, s, a.prefix_len[s], m);
      if (lane == 0) {
        a.new_len[s] = a.prefix_len[s] + (ok ? m : 0);
        a.status[s] = !ok;
      }
    }
  }
}

int launch_kv_append_q8(void* k_pool, void* v_pool, float* k_scale, float* v_scale, const void* k_rows, const void* v_rows,
                        int row_stride, size_t row_layer_stride, const int32_t* path, const int32_t* accept_len,
                        const int32_t* node_off, const int32_t* block_table, int max_blocks, const int32_t* prefix_len,
                        int B, int T, int n_layers, int n_kv_heads, int head_dim, int n_blocks, int32_t* new_len,
                        int32_t* status, hipStream_t st) {
  const AppendArgs a{{(uint8_t*)k_pool, (uint8_t*)v_pool}, {k_scale, v_scale}, {(const uint16_t*)k_rows, (const uint16_t*)v_rows},
                     row_stride, row_layer_stride, path, accept_len, node_off, block_table, prefix_len, max_blocks, B, T,
                     n_kv_heads, n_blocks, new_len, status};
  // all rows: a sequence touches at most two pages more than its rows fill; a path mostly one or two
  const int pages = path ? 2 * B : T / TRJ_KV_BLOCK + 2 * B, planes = 2 * n_layers * n_kv_heads;
  // several planes per wavefront where there are more than the 4096 wavefronts that the chip holds at a time: what
  // finds the page is then done once for them (16 accepted paths, 32 layers, 8 heads: one plane 32 us, two 26, three or
  // four 23, five to eight 25 to 27)
  const int each = (int)std::min(std::max((long)pages * planes / 4096, 1l), 8l);
  const dim3 grid(std::min(pages, 1 << 20), std::min((planes + 4 * each - 1) / (4 * each), 65535));
  if (head_dim == 128) kv_append_kernel<128><<<grid, 256, 0, st>>>(a, planes);
  else kv_append_kernel<64><<<grid, 256, 0, st>>>(a, planes);
  return check_launch();
}

}  // namespace trj
