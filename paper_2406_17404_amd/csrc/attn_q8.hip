// Tree attention over the paged 8-bit cache, fp32 softmax and accumulation.
//
//   out_i = sum_j w_ij v_j / sum_j w_ij,  w_ij = 2^(s_ij - max_j s_ij),  s_ij = scale * log2(e) * q_i . k_j
// over the cached positions j < prefix and the rows j of the tree on the path of i.
//
// The work is streaming the sequence's codes once.  All query heads of a K/V head are worked on
// together: query p of a sequence is (node p / G, head p % G of the group).  A workgroup owns a
// contiguous range of 32-key blocks of one (sequence, K/V head) and NT tiles of 32 queries; each of its
// KS wavefronts is a key stream, which walks every KS-th block for all of them:
//   S^T[keys, queries] = K[keys, dh] * Q^T          (v_mfma_f32_32x32x16_bf16)
//   O^T[dh, queries]  += V^T[dh, keys] * P^T[keys, queries]
// A page is laid out so that 16 contiguous bytes per lane are two such A operands; codes times their
// power-of-two scale are bf16 numbers, exactly, in one instruction per two (v_cvt_scalef32_pk_bf16_fp8),
// so what is rounded to 16 bits is what the 16-bit attention rounds: the weights w (by at most
// 2^-8 of each) and the result.
// Cached blocks come first in a range, then the blocks of the tree's own rows, which are bf16
// in the order the projection left them; only these and the last cached page need a mask.
//
// Bound by memory for long prefixes: 64 rows over 32768 slots, 32 heads of 128, read 271 MB in 65 us = 4.2 TB/s (a
// large copy moves 4.5 to 4.7, a bare read 6.0), with the matrix units at work for a fifth of that time and the vector
// units for a third; 16 sequences of 4096 at most 362 MB in 99 to 107 us, with 43 GFLOP of products.  For few rows by the
// way of a workgroup from the lengths over the table and the scales to its first codes and, over the merge of its
// streams, to the result: one row over 500 slots takes 11 us, of which the cached blocks themselves take 2.4, and 69
// rows of 32 heads on 8 over 3001 slots 21, of which their products need 2.6 at the rate of a large one.
//
// How the keys are split is decided on the device, where the lengths are: every workgroup scans the
// sequences (64 per round), works out the same plan and finds its own part of it.
#include <algorithm>
#include <type_traits>

#include "attn_q8.h"
#include "kernels.h"
#include "q8.h"
#include "tree_anc.h"

namespace trj {

struct Q8Args {
  const uint16_t *q, *k_rows, *v_rows;
  const uint8_t *k_pool, *v_pool;
  const float *k_scale, *v_scale;
  const int32_t *parent, *node_off, *block_table, *prefix_len;
  int q_stride, row_stride, max_blocks, B, T, n_kv_heads, group, n_blocks, max_prefix;
  int max_parts;   // images that the workspace holds
  float scale_log2e;
  float *po, *pm, *pl;  // un-normalised partials: [part][tile] images of the accumulators, maxima and sums of 32 queries
  uint16_t* out;
  int32_t* status;
};

// What a sequence has to do, one per lane (MANY: of the 64 from s0 on).
struct Q8Seq {
  int r0, nodes, L, blocks;  // L < 0: refused, its rows read as zeros (one block of work); blocks 0: nothing to do
  __device__ inline int cached() const { return (L + 31) >> 5; }
};
__device__ inline Q8Seq q8_seq(const Q8Args& a, int s) {
  Q8Seq q{0, 0, 0, 0};
  if (s >= a.B) return q;
  const int r0 = a.node_off[s], r1 = a.node_off[s + 1], L = a.prefix_len[s];
  q.r0 = r0;
  q.L = L;
  q.nodes = r0 < 0 || r1 < r0 || r1 > a.T ? -1 : r1 - r0;
  if (q.nodes <= 0) return q;
  const bool fits = L >= 0 && L <= a.max_prefix && L <= q8_pages_at_most(a.max_blocks) * 32 && q.nodes <= TRJ_N_MAX;
  if (!fits) q.L = -1;
  q.blocks = fits ? q.cached() + (q.nodes + 31) / 32 : 1;
  return q;
}
__device__ inline int q8_groups(const Q8Args& a, const Q8Seq& q, int tile_queries) {  // query groups
  return q.blocks == 0 ? 0 : q.L < 0 ? 1 : (q.nodes * a.group + tile_queries - 1) / tile_queries;
}

// The plan, the same on every wavefront of every workgroup: a split has `chunk` blocks at most, of one
// sequence evenly many.  32 sizes are weighed at once, one per lane: the longest sequence in 1 .. 32 splits.
//   cost = rounds of workgroups * (START + blocks of one) + MERGE if anything is split
// in times that a compute unit takes for a block of its own (0.33 us): a workgroup's way to its first block and
// from its last to the result takes 8 us, the merge launch 5.
// Sequences come longest first, so that what starts last is short.  Beyond 64 sequences neither is done:
// index order, and chunks of an even share.
constexpr float START = 24.f, MERGE = 16.f, RESIDENT = 256.f;  // one workgroup per compute unit at a time
constexpr int MAX_PARTS = 512;  // partials that a call may leave to the merge
// Blocks that a split has at least where it is not weighed: beyond 64 sequences, and with so many workgroups that only
// what would outlast them is split.  Sequences of no more are never split, so a call without longer ones has neither
// partials nor a merge.
constexpr int LEAST_SPLIT = 16;
struct Q8Work {  // of an item
  Q8Seq seq;
  int s, nth, splits, part0;  // nth item of sequence s; its first partial
};
template <bool MANY, int QUERIES>
struct Q8Plan {
  const Q8Args& a;
  Q8Seq mine;   // sequence `id` (sorted)
  int id, chunk;

  __device__ inline explicit Q8Plan(const Q8Args& args) : a(args) {
    const int lane = threadIdx.x & 63;
    float work = 0.f;
    for (int s0 = 0; s0 < (MANY ? a.B : 1); s0 += 64) {
      mine = q8_seq(a, s0 + lane);
      if (!MANY && a.B == 1) break;
      work += wave_sum((float)q8_groups(a, mine, QUERIES) * (float)mine.blocks);
    }
    work *= a.n_kv_heads;
    id = lane;
    if (MANY) {  // (a split sequence has at most twice its share of parts)
      chunk = (int)fminf(fmaxf(ceilf(work * (1.0001f * 2 / MAX_PARTS)), (float)LEAST_SPLIT), 1e9f);
      return;
    }
    int longest = 0;
    if (a.B == 1) {
      longest = lane_value(mine.blocks, 0);
    } else {  // longest first
      int rank = 0;
      for (int t0 = 0; t0 < a.B; t0 += 8)  // (lanes behind the last sequence have no blocks)
#pragma unroll
        for (int t = t0; t < t0 + 8; ++t) {
          const int b = lane_value(mine.blocks, t);
          rank += b > mine.blocks || (b == mine.blocks && t < lane);
        }
      rank = lane < a.B ? rank : lane;
      auto to = [&](int v) { return __builtin_amdgcn_ds_permute(rank << 2, v); };
      mine = Q8Seq{to(mine.r0), to(mine.nodes), to(mine.L), to(mine.blocks)};
      id = to(lane);
      longest = lane_value(mine.blocks, 0);
    }
    if (a.max_parts == 0 || longest <= 1) {
      chunk = max(longest, 1);
      return;
    }
    const int groups = q8_groups(a, mine, QUERIES) * a.n_kv_heads;
    const float items = wave_sum((float)groups);
    if (items >= RESIDENT) {  // enough workgroups: only what would outlast them all is split
      const float share = work * (1.0001f * 2 / MAX_PARTS);
      chunk = longest > 2.f * share + START ? (int)ceilf(fmaxf(share, (float)LEAST_SPLIT)) : longest;
      return;
    }
    const int c = (longest + (lane & 31)) / ((lane & 31) + 1);
    const float each = __builtin_amdgcn_rcpf((float)c);
    float n = 0.f, parts = 0.f;
    if (a.B == 1) work = (float)lane_value(groups, 0) * (float)longest;
    for (int t = 0; t < a.B; ++t) {
      const int b = lane_value(mine.blocks, t), g = lane_value(groups, t);
      const float k = floorf(((float)(b + c) - 0.5f) * each);  // ceil(b / c)
      n += g * k;
      parts += k > 1.f ? g * k : 0.f;
    }
    const float rounds = ceilf(n * (1.f / RESIDENT));
    const float whole = START + c, even = START + work * __builtin_amdgcn_rcpf(n);
    float cost = (rounds > 1.f ? fmaxf(whole, rounds * even) : whole) + (parts > 0.f ? MERGE : 0.f);
    if (parts > a.max_parts) cost = INFINITY;  // no room for its partials
    const uint32_t best = wave_min((uint32_t)fminf(cost * 8.f, 60e6f) << 6 | lane);  // (of equals the fewest splits)
    chunk = lane_value(c, best & 63);
    // Up to 2^16 blocks ceil(b / c) is exact as above: off by at most 33 * 1.5 * 2^-23 where the next whole number is
    // 2^-17 away.  Beyond, whole numbers decide whether the partials have room.
    if (longest > 1 << 16) {
      const int k = splits(mine);
      if (wave_sum(k > 1 ? (float)groups * (float)k : 0.f) > a.max_parts) chunk = longest;
    }
  }
  __device__ inline int splits(const Q8Seq& q) const { return (q.blocks + chunk - 1) / chunk; }
  // item x of all, of which every (sequence, query group, K/V head) counts its splits, or, TILES > 0, once per
  // tile where there are several splits
  template <int TILES>
  __device__ inline bool find(int x, Q8Work& w) {
    const int lane = threadIdx.x & 63;
    if (!MANY && a.B == 1) {
      w.seq = Q8Seq{lane_value(mine.r0, 0), lane_value(mine.nodes, 0), lane_value(mine.L, 0), lane_value(mine.blocks, 0)};
      w.s = w.part0 = 0;
      w.nth = x;
      w.splits = splits(w.seq);
      const int g = q8_groups(a, w.seq, QUERIES) * a.n_kv_heads;
      return x < (TILES == 0 ? g * w.splits : w.splits > 1 ? g * TILES : 0);
    }
    int base = 0, parts = 0;
    for (int s0 = 0; s0 < (MANY ? a.B : 1); s0 += 64) {
      if (MANY) mine = q8_seq(a, s0 + lane), id = s0 + lane;
      const int k = splits(mine), g = q8_groups(a, mine, QUERIES) * a.n_kv_heads;
      const int n = TILES == 0 ? g * k : k > 1 ? g * TILES : 0;
      const int upto = base + wave_scan(n), pupto = parts + wave_scan(k > 1 ? g * k : 0);
      const uint64_t here = __ballot(x < upto);
      if (here) {
        const int l = __builtin_ctzll(here);
        w.seq = Q8Seq{lane_value(mine.r0, l), lane_value(mine.nodes, l), lane_value(mine.L, l), lane_value(mine.blocks, l)};
        w.s = lane_value(id, l);
        w.nth = x - (lane_value(upto, l) - lane_value(n, l));
        w.splits = lane_value(k, l);
        w.part0 = lane_value(pupto, l) - (w.splits > 1 ? lane_value(g, l) * w.splits : 0);
        return true;
      }
      base = lane_value(upto, 63);
      parts = lane_value(pupto, 63);
    }
    return false;
  }
};

// An infinity or NaN among the tree's V rows: times the weight 0 of a row that does not see it it
// would be NaN.  Such values are left out of the products; what they make of the rows that do see
// them does not depend on the weights, which are positive: it is added to the results here, rarely, by
// a walk up the tree.  Queries q0 .. q1 - 1 of a K/V head, columns c0 .. c0 + width - 1 of their results, which
// have been stored (all threads of the workgroup come).
__device__ inline void q8_add_odd_values(const Q8Args& a, int r0, int head, int dh, int q0, int q1, int c0, int width) {
  __builtin_amdgcn_s_waitcnt(0);  // the stores are in the L2
  __syncthreads();
#pragma unroll 1
  for (int u = threadIdx.x; u < (q1 - q0) * (width >> 1); u += blockDim.x) {
    const int q = q0 + u / (width >> 1), c = c0 + u % (width >> 1) * 2, node = q / a.group;
    const uint16_t* v = a.v_rows + (size_t)head * dh + c;
    float sum[2] = {0.f, 0.f};
    bool odd = false;
#pragma unroll 1
    for (int j = node; j >= 0; j = a.parent[r0 + j]) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const uint16_t x = v[(size_t)(r0 + j) * a.row_stride + e];
        if ((x & 0x7f80) == 0x7f80) sum[e] += bf2f(x), odd = true;
      }
    }
    if (!odd) continue;
    uint32_t* const at = reinterpret_cast<uint32_t*>(a.out + ((size_t)(r0 + node) * a.n_kv_heads * a.group + head * a.group + q % a.group) * dh + c);
    const uint32_t was = __hip_atomic_load(at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);  // from there
    *at = pack2bf(bf2f((uint16_t)was) + sum[0], bf2f((uint16_t)(was >> 16)) + sum[1]);
  }
}

// A stream's ring in LDS is its wavefront's own: loads go there without registers (1 KiB each, in
// order), nobody else reads it and nobody waits.  Slot of 32 keys: K pieces, then V pieces.
// No branch that the compiler sees: it would copy the accumulators around it.
// All loads have landed but the newest N0 .. N5 for sel 0 .. 5.
template <int N0, int N1, int N2, int N3, int N4, int N5>
__device__ __forceinline__ void wait_loads(int sel_) {
  const int sel = __builtin_amdgcn_readfirstlane(sel_);
  asm volatile(
      "s_cmp_gt_u32 %0, 4\n\ts_cbranch_scc1 5f\n\t"
      "s_cmp_eq_u32 %0, 0\n\ts_cbranch_scc1 0f\n\t"
      "s_cmp_eq_u32 %0, 1\n\ts_cbranch_scc1 1f\n\t"
      "s_cmp_eq_u32 %0, 2\n\ts_cbranch_scc1 2f\n\t"
      "s_cmp_eq_u32 %0, 3\n\ts_cbranch_scc1 3f\n\t"
      "s_waitcnt vmcnt(%5)\n\ts_branch 6f\n"
      "0:\n\ts_waitcnt vmcnt(%1)\n\ts_branch 6f\n"
      "1:\n\ts_waitcnt vmcnt(%2)\n\ts_branch 6f\n"
      "2:\n\ts_waitcnt vmcnt(%3)\n\ts_branch 6f\n"
      "3:\n\ts_waitcnt vmcnt(%4)\n\ts_branch 6f\n"
      "5:\n\ts_waitcnt vmcnt(%6)\n"
      "6:" ::"s"(sel), "n"(N0), "n"(N1), "n"(N2), "n"(N3), "n"(N4), "n"(N5) : "memory", "scc");
}
// How many K and V are on the way behind the one that is waited for, with r blocks behind the current one and
// rings of d.  They are asked for in the order K 0, V 0, K 1, V 1, ..
constexpr int at_most(int a, int b) { return a < b ? a : b; }
constexpr int behind_k0(int r, int d) { return 1 + 2 * at_most(r, d - 1); }  // K of the current block, V up to d - 1 blocks ahead
constexpr int behind_v(int r, int d) { return 2 * at_most(r, d - 1) + (r >= d); }  // V of it, K up to d blocks ahead
constexpr int behind_k1(int r, int d) { return r < 1 ? 15 : 1 + 2 * at_most(r - 1, d - 1); }  // K of the next, V up to d ahead
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
// P pieces of 1 KiB from base (uniform) to LDS at `lds` (uniform) if `yes`
template <int P>
__device__ __forceinline__ void request(const void* base, uint32_t lane16, uint32_t lds, int if_yes) {
  static_assert(P == 2 || P == 4, "");
  const int yes = __builtin_amdgcn_readfirstlane(if_yes);
  // what was read from these slots is in registers
  // (no instruction offsets: these loads add them to the LDS address as well)
  if constexpr (P == 4)
    asm volatile(
        "s_waitcnt lgkmcnt(0)\n\ts_cmp_eq_u32 %3, 0\n\ts_cbranch_scc1 1f\n\t"
        "s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1\n\t"
        "s_add_u32 m0, %2, 0x400\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %4, %1\n\t"
        "s_add_u32 m0, %2, 0x800\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %5, %1\n\t"
        "s_add_u32 m0, %2, 0xc00\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %6, %1\n"
        "1:" ::"v"(lane16), "s"(base), "s"(lds), "s"(yes), "v"(lane16 + 1024), "v"(lane16 + 2 * 1024), "v"(lane16 + 3 * 1024)
        : "memory", "m0", "scc");
  else
    asm volatile(
        "s_waitcnt lgkmcnt(0)\n\ts_cmp_eq_u32 %3, 0\n\ts_cbranch_scc1 1f\n\t"
        "s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1\n\t"
        "s_add_u32 m0, %2, 0x400\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %4, %1\n"
        "1:" ::"v"(lane16), "s"(base), "s"(lds), "s"(yes), "v"(lane16 + 1024) : "memory", "m0", "scc");
}
#pragma clang diagnostic pop

// rings and, with one tile, a block of the tree's rows; in the same place what the streams hand over at the end
template <int DH, int NT, int KS, int D>
constexpr size_t q8_lds() {
  const size_t ring = (size_t)KS * D * 64 * DH + (NT == 1 ? 2 * 64 * DH : 0), merge = (size_t)(DH / 32) * (KS - 1) * 4096;
  return ring > merge ? ring : merge;
}

// KS key streams of one wavefront each, which takes NT tiles of 32 queries
template <int DH, int NT, int KS, int D, bool MANY>
__global__ __launch_bounds__(KS * 64, KS / 4) void tree_attn_q8_kernel(Q8Args a) {
  constexpr int MTV = DH / 32, OW = MTV * 16 * 64, P = MTV, SLOT = 64 * DH, QUERIES = 32 * NT;
  constexpr int TILE = 64 * DH, CH = DH / 8;
  constexpr bool TREE_LDS = NT == 1;
  static_assert(D >= 2 && KS >= TRJ_N_MAX / 32 && NT <= 2, "a stream's ring takes a block of the tree's rows");
  extern __shared__ __align__(16) uint8_t smem[];  // rings, then parts handed over
  __shared__ float sm_m[KS][NT][32], sm_l[KS][NT][32];
  Q8Plan<MANY, QUERIES> plan(a);
  if (blockIdx.x == 0) {  // sequences without work
    if (!MANY && threadIdx.x < a.B && plan.mine.blocks == 0) a.status[plan.id] = plan.mine.nodes < 0;
    if (MANY)
      for (int s = threadIdx.x; s < a.B; s += KS * 64) {
        const Q8Seq q = q8_seq(a, s);
        if (q.blocks == 0) a.status[s] = q.nodes < 0;
      }
  }
  {
    Q8Work w;
    if (!plan.template find<0>(blockIdx.x, w)) return;
    const int tid = threadIdx.x;
    const int lane = tid & 63, n32 = lane & 31, hh = lane >> 5, ks = __builtin_amdgcn_readfirstlane(tid >> 6);
    const Q8Seq seq = w.seq;
    const int splits = w.splits, n = seq.nodes, nq = n * a.group;
    const int head = w.nth % a.n_kv_heads, sp = w.nth / a.n_kv_heads % splits, qg = w.nth / a.n_kv_heads / splits;
    const int row_len = a.n_kv_heads * a.group * DH;  // of out
    const bool first = sp == 0 && qg == 0;
    const TreeParents par = load_parents(a.parent, seq.r0, seq.L < 0 ? 0 : n);
    if (seq.L < 0 || !tree_valid(par, n)) {  // the same in every wavefront
      if (first) {  // rows of zeros, this K/V head's part
        const size_t width = (size_t)a.group * DH / 4;
        const u32x2 z = {0, 0};
        for (size_t i = tid; i < n * width; i += KS * 64)
          *reinterpret_cast<u32x2*>(a.out + (size_t)(seq.r0 + i / width) * row_len + head * a.group * DH + i % width * 4) = z;
        if (head == 0 && tid == 0) a.status[w.s] = 1;
      }
      return;
    }
    const int32_t* table = a.block_table + (size_t)w.s * a.max_blocks;
    const int cached = seq.cached();
    const int per = (seq.blocks + splits - 1) / splits, b0 = sp * per, b1 = min(seq.blocks, b0 + per);

    // ---- cached blocks b0 + ks, b0 + ks + KS, ..: page, K and V scale of block i in lane i % 64
    const int cend = min(b1, cached);
    const int mine = b0 + ks < cend ? (cend - b0 - ks + KS - 1) / KS : 0;
    const size_t plane = (size_t)head * a.n_blocks;
    int ids = 0;
    float ksc = 1.f, vsc = 1.f;
    auto look_up = [&](int i0) {
      const int i = i0 + lane;
      ids = i < mine ? table[b0 + ks + i * KS] : 0;
    };
    // Then no load that the compiler knows of is on the way: it would wait for it later, and with it for the
    // rings, which it does not know.
    auto look_up_scales = [&]() {
      const bool ok = (unsigned)ids < (unsigned)a.n_blocks;
      ids = ok ? ids : 0;
      ksc = ok ? a.k_scale[plane + ids] : NAN;  // a page that is not there makes its rows NaN
      vsc = a.v_scale[plane + ids];
      __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0)
    };
    look_up(0);
    // the verdict on the sequence's pages, by its first workgroup: most of them are asked for here, judged at the end
    const bool judge = first && head == 0;
    int32_t seen_page = judge && tid < cached ? table[tid] : 0;
    // queries: tile t, column n32; step 2j + i of the product: columns 32j + 16hh + 8i ..
    // (worked out where they are used: they would take registers over the whole walk)
    struct Query {
      int node, head;
      bool live;
    };
    auto query = [&](int t) {
      int l = threadIdx.x & 31;
      asm volatile("" : "+v"(l));
      const int qi = (qg * NT + t) * 32 + l, qc = min(qi, nq - 1);
      return Query{qc / a.group, head * a.group + qc % a.group, qi < nq};
    };
    bf16x8 qreg[NT][2 * MTV];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const Query u = query(t);
      const uint16_t* qp = a.q + (size_t)(seq.r0 + u.node) * a.q_stride + (size_t)u.head * DH + hh * 16;
#pragma unroll
      for (int j = 0; j < 2 * MTV; ++j) qreg[t][j] = *reinterpret_cast<const bf16x8*>(qp + 32 * (j >> 1) + 8 * (j & 1));
    }
    // The tree's own rows of this range go to LDS as they are, each block to the stream that takes it: the first to a
    // place of its own, if there is one (TREE_LDS), others into that stream's ring, which is then filled later.
    // 16-byte piece c of row r lies at c ^ r of its row, so that neither writing rows nor reading columns meets
    // a bank twice.
    const int t0 = max(b0, cached), tree = max(0, b1 - t0);  // blocks
    const int tb = (ks - (t0 - b0) % KS + KS) % KS;          // this stream's of them
    constexpr int UNITS = TRJ_N_MAX / 32 * 32 * CH / (KS * 64);
    constexpr int EARLY = D - 2;  // blocks that fit in front of it
    auto tree_at = [&](int b) {
      return TREE_LDS && b == 0 ? smem + (size_t)KS * D * SLOT : smem + ((size_t)((t0 - b0 + b) % KS) * D + EARLY) * SLOT;
    };
    bool odd = false;
    if (tree > 0) {
      u32x4 raw[UNITS][2];
#pragma unroll
      for (int i = 0; i < UNITS; ++i) {
        const int u = tid + i * KS * 64, rr = u / CH, c = u % CH;  // of all blocks' rows
        if (rr >= tree * 32) break;
        const size_t at = (size_t)(seq.r0 + min((t0 - cached) * 32 + rr, n - 1)) * a.row_stride + (size_t)head * DH + 8 * c;
        raw[i][0] = *reinterpret_cast<const u32x4*>(a.k_rows + at);
        raw[i][1] = *reinterpret_cast<const u32x4*>(a.v_rows + at);
      }
#pragma unroll
      for (int i = 0; i < UNITS; ++i) {
        const int u = tid + i * KS * 64, rr = u / CH, c = u % CH;
        if (rr >= tree * 32) break;
        uint8_t* const dst = tree_at(rr >> 5) + (rr & 31) * 2 * DH + (c ^ (rr & (CH - 1))) * 16;
        u32x4 v = raw[i][1];
        bool mine_odd = false;
#pragma unroll
        for (int e = 0; e < 4; ++e) mine_odd = mine_odd || (v[e] & 0x7f80u) == 0x7f80u || (v[e] & 0x7f800000u) == 0x7f800000u;
        if (mine_odd) {  // left out of the products, see q8_add_odd_values
          odd = true;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if ((v[e] & 0x7f80u) == 0x7f80u) v[e] &= 0xffff0000u;
            if ((v[e] & 0x7f800000u) == 0x7f800000u) v[e] &= 0xffffu;
          }
        }
        *reinterpret_cast<u32x4*>(dst) = raw[i][0];
        *reinterpret_cast<u32x4*>(dst + TILE) = v;
      }
    }
    look_up_scales();
    f32x16 o[NT][MTV];
    Softmax sm[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int mt = 0; mt < MTV; ++mt)
#pragma unroll
        for (int v = 0; v < 16; ++v) o[t][mt][v] = 0.f;

    // With two tiles of heads of 128 queries and sums fill the accumulation registers, from where the products read
    // and write them; said at the loop's ends, or the compiler moves all of them there and back.
    auto keep = [&](auto& x) {
      if constexpr (NT * MTV > 4) asm volatile("" : "+a"(x));
    };
    auto keep_all = [&]() {
#pragma unroll
      for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int j = 0; j < 2 * MTV; ++j) keep(qreg[t][j]);
#pragma unroll
        for (int mt = 0; mt < MTV; ++mt) keep(o[t][mt]);
      }
    };
    const uint32_t ring = __builtin_amdgcn_readfirstlane((uint32_t)(size_t)(__attribute__((address_space(3))) uint8_t*)smem + ks * D * SLOT);
    const u32x4* const ring_r = reinterpret_cast<const u32x4*>(smem + (size_t)ks * D * SLOT) + lane;
    auto ask = [&](const uint8_t* pool, int i, int part, int yes) {  // block i of this stream, K (0) or V (1)
      const size_t page = (uint32_t)__builtin_amdgcn_readlane(ids, i & 63);
      request<P>(pool + (plane + page) * 32 * DH, lane * 16, ring + (i % D) * SLOT + part * (SLOT / 2), yes);
    };
    u32x4 kraw[P];  // codes of the next K
    auto read_k = [&](int i) {
#pragma unroll
      for (int j = 0; j < P; ++j) kraw[j] = ring_r[(i % D) * (SLOT / 16) + j * 64];
    };
    f32x16 sacc[NT];  // products of the queries with a block's keys
    auto scores = [&](int t, const bf16x8 (&kop)[2 * MTV], f32x16& to) {
#pragma unroll
      for (int v = 0; v < 16; ++v) to[v] = 0.f;
#pragma unroll
      for (int j = 0; j < 2 * MTV; ++j) to = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kop[j], qreg[t][j], to, 0, 0, 0);
    };
    auto values = [&](int t, const bf16x8 (&vop)[2 * MTV], const u32x4 (&pk)[2]) {
#pragma unroll
      for (int mt = 0; mt < MTV; ++mt)
#pragma unroll
        for (int kg = 0; kg < 2; ++kg)
          o[t][mt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vop[2 * mt + kg], __builtin_bit_cast(bf16x8, pk[kg]), o[t][mt], 0, 0, 0);
    };
    auto operands = [&](bf16x8 (&op)[2 * MTV], const u32x4 (&raw)[P], float scale) {
#pragma unroll
      for (int j = 0; j < 2 * MTV; ++j) op[j] = operand(raw[j >> 1][2 * (j & 1)], raw[j >> 1][2 * (j & 1) + 1], scale);
    };
    auto scale_of = [&](float of, int i) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(of), i & 63)); };
    // (a page that is not there makes every weight NaN)
    auto factor = [&](int i) { const float k = scale_of(ksc, i); return k == k ? a.scale_log2e : NAN; };
    auto fill = [&](int c0, int c1, auto from_c, auto to_c) {
#pragma unroll
      for (int i = decltype(from_c)::value; i < decltype(to_c)::value; ++i) {
        ask(a.k_pool, c0 + i, 0, c0 + i < c1);
        ask(a.v_pool, c0 + i, 1, c0 + i < c1);
      }
    };
    // ---- the tree's own rows first, while the cached blocks come
    using std::integral_constant;
    const int first_end = min(mine, 64);
    fill(0, first_end, integral_constant<int, 0>{}, integral_constant<int, EARLY>{});
    const bool own_place = TREE_LDS && tb == 0;
    if (tb >= tree || own_place) fill(0, first_end, integral_constant<int, EARLY>{}, integral_constant<int, D>{});
    bool any_odd = false;
    if (tree > 0) any_odd = __syncthreads_or(odd);
    if (tb < tree) {
      {
        const TreeBits bits = tree_bits(par, n);
        const int key0 = (t0 + tb - cached) * 32;
        uint32_t sees[NT];
        int word[2];  // of the nodes' paths, this block's
#pragma unroll
        for (int h = 0; h < 2; ++h)
          word[h] = key0 == 0 ? bits.w[0][h] : key0 == 32 ? bits.w[1][h] : key0 == 64 ? bits.w[2][h] : bits.w[3][h];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const Query u = query(t);
          const int lo = from_node(word, u.node);
          sees[t] = u.live ? (uint32_t)lo : 0u;
        }
        const uint8_t* const rows = tree_at(tb);
        auto key_piece = [&](int j) {  // row n32, columns 32 (j / 2) + 16 hh + 8 (j % 2) ..
          const int c = (j >> 1) * 4 + hh * 2 + (j & 1);
          return *reinterpret_cast<const u32x4*>(rows + n32 * 2 * DH + (c ^ (n32 & (CH - 1))) * 16);
        };
        auto value_pair = [&](int mt, int kg, int e) {  // rows 16 kg + 8 (e / 2) + 4 hh + 2 (e % 2) and the next, column 32 mt + n32
          u16x2 x;
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int key = 16 * kg + 8 * (e >> 1) + 4 * hh + 2 * (e & 1) + i, c = 4 * mt + (n32 >> 3);
            x[i] = *reinterpret_cast<const uint16_t*>(rows + TILE + key * 2 * DH + (c ^ (key & (CH - 1))) * 16 + (n32 & 7) * 2);
          }
          return __builtin_bit_cast(uint32_t, x);
        };
        f32x16 sacc[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int v = 0; v < 16; ++v) sacc[t][v] = 0.f;
#pragma unroll
        for (int j = 0; j < 2 * MTV; ++j) {
          const bf16x8 kop = __builtin_bit_cast(bf16x8, key_piece(j));
#pragma unroll
          for (int t = 0; t < NT; ++t) sacc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kop, qreg[t][j], sacc[t], 0, 0, 0);
        }
        u32x4 pk[NT][2];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
          for (int v = 0; v < 16; ++v)
            if (!((sees[t] >> (8 * (v >> 2) + 4 * hh + (v & 3))) & 1)) sacc[t][v] = -INFINITY;
          q8_rescale<MTV>(o[t], sm[t].lift(Softmax::largest(sacc[t], a.scale_log2e)));
          sm[t].weigh(sacc[t], a.scale_log2e, pk[t]);
        }
#pragma unroll
        for (int mt = 0; mt < MTV; ++mt)
#pragma unroll
          for (int kg = 0; kg < 2; ++kg) {
            const bf16x8 vop = __builtin_bit_cast(bf16x8, u32x4{value_pair(mt, kg, 0), value_pair(mt, kg, 1), value_pair(mt, kg, 2), value_pair(mt, kg, 3)});
#pragma unroll
            for (int t = 0; t < NT; ++t)
              o[t][mt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vop, __builtin_bit_cast(bf16x8, pk[t][kg]), o[t][mt], 0, 0, 0);
          }
      }
      if (!own_place) fill(0, first_end, integral_constant<int, EARLY>{}, integral_constant<int, D>{});
    }

    // ---- the cached blocks
    for (int c0 = 0; c0 < mine; c0 += 64) {
      const int c1 = min(mine, c0 + 64);
      if (c0 > 0) {
        look_up(c0);
        look_up_scales();
        fill(c0, c1, integral_constant<int, 0>{}, integral_constant<int, D>{});
      }
      const int rest = seq.L - (b0 + ks + (c1 - 1) * KS) * 32;  // keys of the last block, if fewer than 32
#define Q8_WAIT(behind, r) \
  wait_loads<P * behind(0, D), P * behind(1, D), P * behind(2, D), P * behind(3, D), P * behind(4, D), P * behind(5, D)>(r)
      // K of a block is in registers when its turn begins.  With two tiles the softmax of one runs while the matrix
      // units work on the other.  The loop has one way out, in front of a reference that has to be lifted: a
      // condition around the accumulators inside it would have them copied every time.
      bf16x8 kop[2 * MTV], vop[2 * MTV];
      u32x4 pk[NT][2];
      float top[NT], f;
      auto begin = [&](int i) {  // products and their maxima, from K in registers
        f = factor(i);
        operands(kop, kraw, scale_of(ksc, i));
#pragma unroll
        for (int t = 0; t < NT; ++t) scores(t, kop, sacc[t]);
#pragma unroll
        for (int t = 0; t < NT; ++t) top[t] = Softmax::largest(sacc[t], f);
      };
      Q8_WAIT(behind_k0, c1 - 1 - c0);
      read_k(c0);
      keep_all();
      begin(c0);
      int i = c0;
      for (;;) {
        bool last;
        for (;;) {
          last = i == c1 - 1;
          bool low = last || sm[0].too_low(top[0]);
          if constexpr (NT == 2) low = low || sm[1].too_low(top[1]);
          if (__ballot(low)) break;
          ask(a.k_pool, i + D, 0, i + D < c1);
          sm[0].weigh(sacc[0], f, pk[0]);
          Q8_WAIT(behind_v, c1 - 1 - i);
          u32x4 vraw[P];
#pragma unroll
          for (int j = 0; j < P; ++j) vraw[j] = ring_r[(i % D) * (SLOT / 16) + (P + j) * 64];
          operands(vop, vraw, scale_of(vsc, i));
          ask(a.v_pool, i + D, 1, i + D < c1);
          if constexpr (NT == 2) {
            values(0, vop, pk[0]);
            sm[1].weigh(sacc[1], f, pk[1]);
          }
          Q8_WAIT(behind_k1, c1 - 1 - i);
          ++i;
          read_k(i);
          values(NT - 1, vop, pk[NT - 1]);
          begin(i);
        }
        keep_all();
        if (last) {
#pragma unroll
          for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int v = 0; v < 16; ++v)
              if (8 * (v >> 2) + 4 * hh + (v & 3) >= rest) sacc[t][v] = -INFINITY;
            top[t] = Softmax::largest(sacc[t], f);
          }
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) q8_rescale<MTV>(o[t], sm[t].lift(top[t]));
        keep_all();
        if (last) break;
      }
      wait_loads<0, 0, 0, 0, 0, 0>(0);
      u32x4 vraw[P];
#pragma unroll
      for (int j = 0; j < P; ++j) vraw[j] = ring_r[(i % D) * (SLOT / 16) + (P + j) * 64];
      // slots past the end may hold anything: their weights are 0, their values have to be numbers
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        const int keep = min(max(rest - 8 * d - 4 * hh, 0), 4);
        const uint32_t mask = keep == 4 ? 0xffffffffu : (1u << (8 * keep)) - 1u;
#pragma unroll
        for (int j = 0; j < P; ++j) vraw[j][d] &= mask;
      }
      operands(vop, vraw, scale_of(vsc, i));
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        sm[t].weigh(sacc[t], f, pk[t]);
        values(t, vop, pk[t]);
      }
    }
    // ---- merge the key streams of every query tile in a fixed order: stream k adds up registers R k .. of the tile
    constexpr int R = MTV * 16 / KS;
    static_assert(R % 4 == 0, "");
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const float l = sm[t].l + __shfl_xor(sm[t].l, 32);
      if (hh == 0) {
        sm_m[ks][t][n32] = sm[t].m;
        sm_l[ks][t][n32] = l;
      }
    }
    __syncthreads();  // the rings are free, too
    f32x4* const red = reinterpret_cast<f32x4*>(smem);
#pragma unroll
    for (int t = 0; t < NT; ++t) {  // tile by tile: all at once do not fit LDS
      if (t > 0) __syncthreads();
      float mg = NO_REFERENCE, lg = 0.f;
#pragma unroll
      for (int k = 0; k < KS; ++k) mg = fmaxf(mg, sm_m[k][t][n32]);
#pragma unroll
      for (int k = 0; k < KS; ++k) lg += sm_l[k][t][n32] * __builtin_amdgcn_exp2f(sm_m[k][t][n32] - mg);
      const float f = __builtin_amdgcn_exp2f(sm[t].m - mg);
      f32x4 sum[R / 4];
#pragma unroll
      for (int k = 0; k < KS; ++k) {  // to stream k
#pragma unroll
        for (int q = 0; q < R / 4; ++q) {
          const int reg = k * R + 4 * q;
          const f32x4 x = {o[t][reg >> 4][reg & 15] * f, o[t][reg >> 4][(reg & 15) + 1] * f, o[t][reg >> 4][(reg & 15) + 2] * f,
                           o[t][reg >> 4][(reg & 15) + 3] * f};
          if (ks == k) sum[q] = x;
          else red[((k * (KS - 1) + (ks < k ? ks : ks - 1)) * (R / 4) + q) * 64 + lane] = x;
        }
      }
      __syncthreads();
      if ((qg * NT + t) * 32 >= nq) continue;
      const int part = w.part0 + w.nth;
      if (splits > 1 && part >= a.max_parts) continue;  // more work than T rows can be: ranges that overlap
      const size_t tile = (size_t)part * NT + t;
      if (splits > 1 && ks == 0 && hh == 0) {
        a.pm[tile * 32 + n32] = mg;
        a.pl[tile * 32 + n32] = any_odd ? -lg : lg;  // (a sum of weights is not negative)
      }
#pragma unroll
      for (int k = 0; k < KS - 1; ++k)
#pragma unroll
        for (int q = 0; q < R / 4; ++q) sum[q] += red[((ks * (KS - 1) + k) * (R / 4) + q) * 64 + lane];
      const int reg0 = ks * R;  // 32-column part reg0 / 16, columns 8 (v / 4) + 4 hh + v % 4 of it
      if (splits == 1) {
        const float inv = 1.0f / lg;
        const Query u = query(t);
        if (u.live) {
          uint16_t* dst = a.out + (size_t)(seq.r0 + u.node) * row_len + (size_t)u.head * DH + 4 * hh + (reg0 >> 4) * 32 + (reg0 & 15) * 2;
#pragma unroll
          for (int q = 0; q < R / 4; ++q) {
            const u32x2 v = {pack2bf(sum[q][0] * inv, sum[q][1] * inv), pack2bf(sum[q][2] * inv, sum[q][3] * inv)};
            *reinterpret_cast<u32x2*>(dst + 8 * q) = v;
          }
        }
      } else {
#pragma unroll
        for (int q = 0; q < R / 4; ++q) *reinterpret_cast<f32x4*>(a.po + tile * OW + ((reg0 >> 2) + q) * 256 + lane * 4) = sum[q];
      }
    }
    if (judge) {
      bool bad = (unsigned)seen_page >= (unsigned)a.n_blocks;
      for (int j = tid + KS * 64; j < cached; j += KS * 64) bad = bad || (unsigned)table[j] >= (unsigned)a.n_blocks;
      bad = __syncthreads_or(bad);
      if (tid == 0) a.status[w.s] = bad;
    }
    if (any_odd && splits == 1) q8_add_odd_values(a, seq.r0, head, DH, qg * QUERIES, min(nq, (qg + 1) * QUERIES), 0, DH);
  }
}

// Merges the partials of a (sequence, query tile, K/V head) in split order, one 32-column part of the
// rows per workgroup.  Thread (lane, g, h) adds the accumulator registers 4g .. 4g+3 that lane held, over
// every fourth split from h on, with a running maximum; the four sums are joined through LDS.  All loads of a
// batch are asked for together (clamped, never predicated): one after the other 32 splits took 35 us.
template <int DH, int NT, bool MANY>
__global__ __launch_bounds__(1024) void attn_q8_combine_kernel(Q8Args a) {
  constexpr int MTV = DH / 32, PART = 16 * 64, BATCH = 4;
  __shared__ float sm_m[4][32], sm_l[4][32];
  __shared__ f32x4 sm_o[3][256];
  const int tid = threadIdx.x, lane = tid & 63, n32 = lane & 31, hh = lane >> 5, g = (tid >> 6) & 3, h = tid >> 8;
  Q8Plan<MANY, 32 * NT> plan(a);
  for (int x = blockIdx.x / MTV;; x += gridDim.x / MTV) {  // tiles
    const int mt = blockIdx.x % MTV;
    Q8Work w;
    if (!plan.template find<NT>(x, w)) return;
    const Q8Seq seq = w.seq;
    const int splits = w.splits, nt = w.nth % NT, head = w.nth / NT % a.n_kv_heads, qg = w.nth / NT / a.n_kv_heads;
    const int nq = seq.nodes * a.group, qi = (qg * NT + nt) * 32 + n32;
    if ((qg * NT + nt) * 32 >= nq) continue;
    if (w.part0 + (qg + 1) * splits * a.n_kv_heads > a.max_parts) continue;  // see there
    const TreeParents par = load_parents(a.parent, seq.r0, seq.nodes);
    float m = NO_REFERENCE, l = 0.f;
    bool odd = false;
    f32x4 o = {0, 0, 0, 0};
    for (int s0 = h; s0 < splits; s0 += 4 * BATCH) {
      float pm[BATCH], pl[BATCH];
      f32x4 po[BATCH];
#pragma unroll
      for (int k = 0; k < BATCH; ++k) {
        const int sp = min(s0 + 4 * k, splits - 1);
        const size_t p = (size_t)(w.part0 + (qg * splits + sp) * a.n_kv_heads + head) * NT + nt;
        pm[k] = a.pm[p * 32 + n32];
        pl[k] = a.pl[p * 32 + n32];
        po[k] = *reinterpret_cast<const f32x4*>(a.po + p * MTV * PART + (mt * 4 + g) * 256 + lane * 4);
      }
      float top = m;
#pragma unroll
      for (int k = 0; k < BATCH; ++k) top = fmaxf(top, pm[k]);
      const float alpha = __builtin_amdgcn_exp2f(m - top);
      m = top;
      l *= alpha;
      o *= alpha;
#pragma unroll
      for (int k = 0; k < BATCH; ++k) {
        if (s0 + 4 * k >= splits) break;
        const float f = __builtin_amdgcn_exp2f(pm[k] - m);
        odd = odd || (__float_as_uint(pl[k]) >> 31) != 0;
        l += f * fabsf(pl[k]);
        o += f * po[k];
      }
    }
    if (h > 0) sm_o[h - 1][tid & 255] = o;
    if (g == 0 && hh == 0) sm_m[h][n32] = m, sm_l[h][n32] = l;
    const bool valid = tree_valid(par, seq.nodes);  // else its rows are zeros already
    const bool any_odd = __syncthreads_or(odd);
    if (h == 0 && valid && qi < nq) {
      float top = m;
#pragma unroll
      for (int k = 1; k < 4; ++k) top = fmaxf(top, sm_m[k][n32]);
      const float alpha = __builtin_amdgcn_exp2f(m - top);
      l *= alpha;
      o *= alpha;
#pragma unroll
      for (int k = 1; k < 4; ++k) {
        const float f = __builtin_amdgcn_exp2f(sm_m[k][n32] - top);
        l += f * sm_l[k][n32];
        o += f * sm_o[k - 1][tid];
      }
      const float inv = 1.0f / l;
      const int node = qi / a.group, qhead = head * a.group + qi % a.group;
      uint16_t* dst = a.out + ((size_t)(seq.r0 + node) * a.n_kv_heads * a.group + qhead) * DH + 32 * mt + 4 * hh + 8 * g;
      const u32x2 v = {pack2bf(o[0] * inv, o[1] * inv), pack2bf(o[2] * inv, o[3] * inv)};
      *reinterpret_cast<u32x2*>(dst) = v;
    }
    if (any_odd && valid) {
      const int q0 = (qg * NT + nt) * 32;
      q8_add_odd_values(a, seq.r0, head, DH, q0, min(nq, q0 + 32), mt * 32, 32);
    }
    __syncthreads();  // LDS is free again
  }
}

// ------------------------------------------------------------------ launch
// Two tiles of queries per workgroup where a sequence has more than 32 (as the average of the batch has it):
// the codes are then converted once for both, on four streams; one tile on eight.  That pays for heads of 128 where the chip is
// full, which this rule does not look at (us per call with two tiles and with one):
//   16 sequences of 64 rows, up to 4096 slots   32 on 32 heads 103 117, 32 on 8 88 99, 16 on 16 heads of 64 43 34
//   64 and 128 sequences of 16 rows, up to 2048 32 on 8 heads 79 99, 134 153
//   one of 64 rows, 32 on 32 heads              over 500 24 17, 3001 27 22, 32768 72 to 76 69
//   one of 69 rows, 32 on 8 heads               over 500 25 18, 3001 29 24, 8000 37 30, 32768 75 75
// (Four streams and two workgroups per compute unit gain nothing for one tile: 64 sequences of one row on 8 K/V heads, up to
// 1000 slots 48.3 against 47.0 us.)
struct Q8Launch {
  int ntw, max_parts, grid, tiles;
};
static Q8Launch q8_launch(int B, int T, int group, int n_kv_heads, int max_prefix) {
  Q8Launch p;
  const long queries = ((long)T + B - 1) / B * group;  // of a sequence, if all are alike
  p.ntw = queries > 32 ? 2 : 1;
  const long items = ((long)T * group / (32 * p.ntw) + B) * n_kv_heads;  // unsplit
  const long most = ((long)max_prefix + 31) / 32 + TRJ_N_MAX / 32;       // blocks of a sequence
  p.max_parts = most <= LEAST_SPLIT ? 0 : MAX_PARTS;
  p.grid = (int)std::min(items + p.max_parts, 1l << 30);
  p.tiles = (int)std::min(items * p.ntw, 64l);
  return p;
}
size_t attn_q8_ws_floats(int B, int T, int group, int n_kv_heads, int head_dim, int max_prefix) {
  const Q8Launch p = q8_launch(B, T, group, n_kv_heads, max_prefix);
  return (size_t)p.max_parts * p.ntw * (32 * head_dim + 64);
}

template <int DH, int NT, int KS, int D, bool MANY>
static int q8_run(const Q8Args& a, const Q8Launch& p, hipStream_t st) {
  constexpr size_t lds = q8_lds<DH, NT, KS, D>();
  static DeviceOnce once;
  allow_lds(once, tree_attn_q8_kernel<DH, NT, KS, D, MANY>, lds);
  {
    ProfScope ps_(KC_ATTN, st);
    tree_attn_q8_kernel<DH, NT, KS, D, MANY><<<p.grid, KS * 64, lds, st>>>(a);
  }
  int rc = check_launch();
  if (rc != TRJ_OK || p.max_parts == 0) return rc;
  ProfScope ps_(KC_ATTN_COMBINE, st);
  attn_q8_combine_kernel<DH, NT, MANY><<<p.tiles * (DH / 32), 1024, 0, st>>>(a);
  return check_launch();
}
template <int DH, bool MANY>
static int q8_run_tiles(const Q8Args& a, const Q8Launch& p, hipStream_t st) {
  return p.ntw == 1 ? q8_run<DH, 1, 8, 2, MANY>(a, p, st) : q8_run<DH, 2, 4, 4, MANY>(a, p, st);
}

int launch_tree_attn_q8(const uint16_t* q, int q_stride, const void* k_pool, const void* v_pool, const float* k_scale,
                        const float* v_scale, const uint16_t* k_rows, const uint16_t* v_rows, int row_stride,
                        const int32_t* parent, const int32_t* node_off, const int32_t* block_table, int max_blocks,
                        const int32_t* prefix_len, int B, int T, int n_heads, int n_kv_heads, int head_dim, int n_blocks,
                        int max_prefix, float scale, float* ws, uint16_t* out, int32_t* status, hipStream_t st) {
  const int group = n_heads / n_kv_heads;
  const Q8Launch p = q8_launch(B, T, group, n_kv_heads, max_prefix);
  const size_t tiles = (size_t)p.max_parts * p.ntw;
  float* const pm = ws + tiles * 32 * head_dim;
  const Q8Args a{q, k_rows, v_rows, (const uint8_t*)k_pool, (const uint8_t*)v_pool, k_scale, v_scale, parent, node_off,
                 block_table, prefix_len, q_stride, row_stride, max_blocks, B, T, n_kv_heads, group, n_blocks, max_prefix,
                 p.max_parts, scale * LOG2E, ws, pm, pm + tiles * 32, out, status};
  if (B > 64) return head_dim == 128 ? q8_run_tiles<128, true>(a, p, st) : q8_run_tiles<64, true>(a, p, st);
  return head_dim == 128 ? q8_run_tiles<128, false>(a, p, st) : q8_run_tiles<64, false>(a, p, st);
}

}  // namespace trj
