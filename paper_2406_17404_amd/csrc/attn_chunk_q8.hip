// Causal attention of chunks of new rows over the paged 8-bit cache, fp32 softmax and accumulation.
//
//   out_i = sum_j w_ij v_j / sum_j w_ij,  w_ij = 2^(s_ij - max_j s_ij),  s_ij = scale * log2(e) * q_i . k_j
// over the cached positions j < prefix and the sequence's own rows j <= i.
//
// All query heads of a K/V head are worked on together: query p of a sequence is (row p / G, head p % G of the group).
// A workgroup owns QUERIES of them, 32 per wavefront, and a contiguous range of blocks of 64 keys, which its
// wavefronts bring to LDS together, as operands of
//   S^T[keys, queries] = K[keys, dh] * Q^T          (v_mfma_f32_32x32x16_bf16)
//   O^T[dh, queries]  += V^T[dh, keys] * P^T[keys, queries]
// Cached blocks (two pages) are converted on the way, codes times their power-of-two scale being bf16 numbers
// exactly; the sequence's own rows are bf16 already and V is transposed.
//
// The softmax's weights are rounded to bf16 for the second product, whose operands are 16 bits wide; their sum is not.  Beside the
// result's own rounding, 1.7e-3 of it as a whole, that makes 2.1e-3 to 2.3e-3, as in tree_attention_q8.
//
// Bound by vector instructions and products for long chunks: 2048 rows after 16384 positions, 32 heads of 128, are 584 GFLOP in 605
// to 700 us, 0.83 to 0.96 PFLOP/s where a large library product reaches 1.19 to 1.33.  A tile of 32 keys x 32 queries takes
// 1220 cycles of a SIMD, of which its 16 products are 512 (42 %) and its 149 vector instructions by count some 750, 16 exponentials
// at a quarter of the rate among them; the two wavefronts of a SIMD hardly overlap these.  Some 30 of the 149 are no part of the
// method: moves where the steps' states meet, selects of scales, scalars read back from lanes.  LDS is active in 38 % of the cycles;
// with the exponentials left out (675 us whole) 25 us are saved, reading operands 56, the conversion 75, conversion and loads
// 128.  Less per product would take more queries per wavefront, and two query tiles' accumulators, weights and queries do not fit its
// 256 registers.
// A whole prompt of 4096 rows, 32 heads on 8, takes 165 to 190 us (0.72 to 0.84): 65 blocks for each compute unit, which are 150 us at
// 2.3 us a block, and the start and end of two items; masked products are 1.5 % of those worked out.
// For short ones by the way to the first block and from the last: 12 us for an item of one block (plan 0.5, queries 0.8,
// first codes 1.2, their conversion and barrier 1.4, two masked tiles 2.9, end 2.1; code that is not in the instruction cache yet
// is in each), and by the merge's launch, 4 to 17 us with its traffic.
#include <algorithm>
#include <type_traits>

#include "attn_q8.h"
#include "kernels.h"

namespace trj {

struct ChunkArgs {
  const uint16_t *q, *k_rows, *v_rows;
  const uint8_t *k_pool, *v_pool;
  const float *k_scale, *v_scale;
  const int32_t *node_off, *block_table, *prefix_len;
  int q_stride, row_stride, max_blocks, B, T, n_kv_heads, group, n_blocks, max_prefix;
  int max_parts;
  float scale_log2e;
  float *po, *pm, *pl;  // un-normalised partials: [part][wavefront] images of the accumulators, maxima and sums of 32 queries
  int32_t* merges;      // how many tiles there are to merge, then from word 8 on 8 words for each (ChunkMerge)
  uint16_t* out;
  int32_t* status;
};
constexpr int CH_WAVES = 8, CH_THREADS = 64 * CH_WAVES, CH_QUERIES = 32 * CH_WAVES, CH_KEYS = 64;
constexpr int CH_MAX_PARTS = 512, CH_MAX_MERGES = CH_MAX_PARTS / 2;  // partials that a call may leave to the merge
// Calls in which no sequence can have more blocks have neither partials nor a merge; beyond 64 sequences a split's least span.
constexpr int CH_LEAST = 4;

// Queries of a sequence that are taken 32 at a time, with a wavefront per page (chunk_few): a block takes such a workgroup 0.4 to
// 0.9 us, one of the other form 1.5 with few wavefronts at work.  40 sequences of 8 rows over 2000 positions, 64 heads on 8: 78 us so,
// 130 else; of 128 queries, 64 sequences of 30 rows over 4000, 32 on 8, 342 and 285.
constexpr int CH_FEW = 64;

struct ChunkSeq {
  int r0, n, L, tiles;  // n < 0: refused, with nothing written; L < 0: refused, rows of zeros
  int few;              // 1: tiles of 32 queries, a wavefront per page (chunk_few), else of CH_QUERIES
  __device__ inline int cached() const { return (L + CH_KEYS - 1) / CH_KEYS; }
  __device__ inline int blocks() const { return n <= 0 ? 0 : L < 0 ? 1 : cached() + (n + CH_KEYS - 1) / CH_KEYS; }
  // blocks, of few queries four to a unit
  __device__ inline int units() const { return few ? (blocks() + 3) >> 2 : blocks(); }
  // units of all tiles, about: own rows are seen up to a tile's
  __device__ inline float work() const {
    return few || L < 0 ? (float)(tiles * units())
                        : (float)tiles * ((float)cached() + 0.5f * (float)((n + CH_KEYS - 1) / CH_KEYS + 1));
  }
};
__device__ inline ChunkSeq chunk_seq(const ChunkArgs& a, int s) {
  ChunkSeq q{0, 0, 0, 0, 0};
  if (s >= a.B) return q;
  const int r0 = a.node_off[s], r1 = a.node_off[s + 1], L = a.prefix_len[s];
  q.r0 = r0;
  q.n = r0 < 0 || r1 < r0 || r1 > a.T ? -1 : r1 - r0;
  q.L = L >= 0 && L <= a.max_prefix && L <= (int64_t)q8_pages_at_most(a.max_blocks) * 32 ? L : -1;
  q.few = q.n > 0 && q.n * a.group <= CH_FEW && q.L >= 0;
  q.tiles = q.n <= 0 ? 0 : q.few ? (q.n * a.group + 31) >> 5 : (q.n * a.group + CH_QUERIES - 1) / CH_QUERIES;
  return q;
}

struct ChunkWork {
  ChunkSeq seq;
  int s, nth, splits, part0, merge0;  // first partial and first merge of the sequence
};
struct ChunkMerge {
  int r0, q0, q1, head, splits, part, step, pad;  // queries of the sequence; partial of split k: part + k * step
};
// The plan, the same on every wavefront of every workgroup: a split has `span` units at most, of one sequence evenly many.
// Up to 64 sequences (not MANY) 64 spans are weighed, one per lane, the longest sequence in 1 .. 32 splits, then 36 .. 160
// (few heads and a long cache: 64 rows over 131072 positions, 8 heads on one, 147 us with 32 splits at most, 80 so; 62 since they
// come in tiles of 32):
//   cost = rounds of workgroups * (START + units of one), and if anything is split MERGE, PART for each of the parts and
//          EACH for each split of the longest
// A unit is what a compute unit takes for a block of 256 queries, 2.3 us, or for four of few queries (0.6 to 0.9 us each).
// Sequences come longest first, so that what starts last is short and rounds fill up: the middle between whole rounds of
// average items and no idle unit is taken.  Beyond 64 sequences neither is done: index order, and spans of an even share.
constexpr int SHORT = 96;  // blocks
constexpr float FEW_TILES = 32.f;
constexpr float START = 4.5f, MERGE = 2.5f, PART = 0.03f, EACH = 0.1f, RESIDENT = 256.f;  // one workgroup per compute unit at a time
template <bool MANY>
struct ChunkPlan {
  const ChunkArgs& a;
  ChunkSeq mine;  // sequence `id` (sorted)
  int id, span;
  __device__ inline explicit ChunkPlan(const ChunkArgs& args) : a(args) {
    const int lane = threadIdx.x & 63;
    float work = 0.f;
    for (int s0 = 0; s0 < (MANY ? a.B : 1); s0 += 64) {
      mine = chunk_seq(a, s0 + lane);
      if (!MANY) {
        // Where all tiles of 32 queries fit one round, short sequences come in such tiles, and longer ones of four tiles, or of any
        // number if they are few in all: 40 rows after 500 positions, 32 heads on 8, took 20 us in the other form and take 13, 100 after
        // 3500 38 and 29, 128 after 8000, the border, 45 and 48; 16 after 130000 119 and 66; 64 after 30000, 8 heads on one, 47 and 31.
        const int tiles = mine.n <= 0 ? 0 : (mine.n * a.group + 31) >> 5;
        const float all = wave_sum((float)tiles) * (float)a.n_kv_heads;
        if (all <= RESIDENT && mine.n > 0 && mine.L >= 0 && (mine.blocks() <= SHORT || tiles <= 4 || all <= FEW_TILES))
          mine.few = 1, mine.tiles = tiles;
      }
      if (!MANY && a.B == 1) break;
      work += wave_sum(MANY ? (float)mine.tiles * (float)mine.units() : mine.work());
    }
    work *= a.n_kv_heads;
    id = lane;
    if (MANY) {  // (a sequence that is split has fewer than twice blocks / span splits: CH_MAX_PARTS in all at most)
      span = a.max_parts == 0 ? 1 << 30 : (int)fminf(fmaxf(ceilf(work * (1.0001f * 2 / CH_MAX_PARTS)), (float)CH_LEAST), 1e9f);
      return;
    }
    if (a.B > 1) {  // longest first
      const int blocks = mine.units();
      int rank = 0;
      for (int t0 = 0; t0 < a.B; t0 += 8)  // (lanes behind the last sequence have no blocks)
#pragma unroll
        for (int t = t0; t < t0 + 8; ++t) {
          const int b = lane_value(blocks, t);
          rank += b > blocks || (b == blocks && t < lane);
        }
      rank = lane < a.B ? rank : lane;
      auto to = [&](int v) { return __builtin_amdgcn_ds_permute(rank << 2, v); };
      mine = ChunkSeq{to(mine.r0), to(mine.n), to(mine.L), to(mine.tiles), to(mine.few)};
      id = to(lane);
    }
    const int blocks = mine.units(), longest = max(lane_value(blocks, 0), 1), groups = mine.tiles * a.n_kv_heads;
    span = longest;
    if (a.max_parts == 0 || longest == 1) return;
    const int most = lane < 32 ? lane + 1 : 32 + 4 * (lane - 31), c = (longest + most - 1) / most;
    const float each = __builtin_amdgcn_rcpf((float)c);
    float n = 0.f, parts = 0.f;
    if (a.B == 1) work = wave_sum(mine.work()) * a.n_kv_heads;  // (lanes behind the first have none)
    for (int t = 0; t < a.B; ++t) {
      const int b = lane_value(blocks, t), g = lane_value(groups, t);
      const float k = floorf(((float)(b + c) - 0.5f) * each);  // ceil(b / c)
      n += (float)g * k;
      parts += k > 1.f ? (float)g * k : 0.f;
    }
    const float rounds = ceilf(n * (1.f / RESIDENT));
    const float whole = START + (float)c, even = START + work * __builtin_amdgcn_rcpf(n);
    float cost = (rounds > 1.f ? fmaxf(whole, 0.5f * even * (rounds + n * (1.f / RESIDENT))) : whole) + (parts > 0.f ? MERGE + PART * parts + EACH * (float)most : 0.f);
    if (parts > (float)a.max_parts) cost = INFINITY;  // no room for its partials
    const uint32_t best = wave_min((uint32_t)fminf(cost * 8.f, 60e6f) << 6 | lane);  // (of equals the fewest splits)
    span = lane_value(c, best & 63);
    // the reciprocal's division may be off for lengths beyond 2^16 blocks: whole numbers decide whether the partials have room
    if (longest > 1 << 16) {
      const int k = splits(mine);
      if (wave_sum(k > 1 ? (float)groups * (float)k : 0.f) > (float)a.max_parts) span = longest;
    }
  }
  __device__ inline int splits(const ChunkSeq& q) const { return (q.units() + span - 1) / span; }
  // item x of all, of which a (sequence, tile, K/V head) counts its splits
  __device__ inline bool find(int x, ChunkWork& w) {
    const int lane = threadIdx.x & 63;
    if (!MANY && a.B == 1) {
      w.seq = ChunkSeq{lane_value(mine.r0, 0), lane_value(mine.n, 0), lane_value(mine.L, 0), lane_value(mine.tiles, 0), lane_value(mine.few, 0)};
      w.s = w.part0 = w.merge0 = 0;
      w.nth = x;
      w.splits = splits(w.seq);
      return x < w.seq.tiles * a.n_kv_heads * w.splits;
    }
    int base = 0, parts = 0, merges = 0;
    for (int s0 = 0; s0 < (MANY ? a.B : 1); s0 += 64) {
      if (MANY) mine = chunk_seq(a, s0 + lane), id = s0 + lane;
      const int k = splits(mine), g = mine.tiles * a.n_kv_heads;
      const int upto = base + wave_scan(g * k), pupto = parts + wave_scan(k > 1 ? g * k : 0), mupto = merges + wave_scan(k > 1 ? g : 0);
      const uint64_t here = __ballot(x < upto);
      if (here) {
        const int l = __builtin_ctzll(here);
        w.seq = ChunkSeq{lane_value(mine.r0, l), lane_value(mine.n, l), lane_value(mine.L, l), lane_value(mine.tiles, l), lane_value(mine.few, l)};
        w.s = lane_value(id, l);
        w.splits = lane_value(k, l);
        const int gl = lane_value(g, l);
        w.nth = x - (lane_value(upto, l) - gl * w.splits);
        if ((unsigned)w.nth >= (unsigned)(gl * w.splits)) return false;  // (sums beyond 2^31: ranges that overlap)
        w.part0 = lane_value(pupto, l) - (w.splits > 1 ? gl * w.splits : 0);
        w.merge0 = lane_value(mupto, l) - (w.splits > 1 ? gl : 0);
        return true;
      }
      base = lane_value(upto, 63);
      parts = lane_value(pupto, 63);
      merges = lane_value(mupto, 63);
    }
    return false;
  }
  // tiles that are split
  __device__ inline int merges() {
    int sum = 0;
    for (int s0 = 0; s0 < (MANY ? a.B : 1); s0 += 64) {
      const ChunkSeq q = MANY ? chunk_seq(a, s0 + (threadIdx.x & 63)) : mine;
      sum += lane_value(wave_scan(splits(q) > 1 ? q.tiles * a.n_kv_heads : 0), 63);
    }
    return sum;
  }
};

// Infinities and NaN among V rows that some query of the tile does not see are left out of the products (times
// the weight 0 they would be NaN) and added here, rarely, to the stored results of those who do see them: rows
// from..row of the sequence.
__device__ inline void chunk_add_odd_values(const ChunkArgs& a, int r0, int head, int dh, int q0, int q1, int from) {
  __builtin_amdgcn_s_waitcnt(0);  // the stores are in the L2
  __syncthreads();
#pragma unroll 1
  for (int u = threadIdx.x; u < (q1 - q0) * (dh >> 1); u += blockDim.x) {
    const int q = q0 + u / (dh >> 1), c = u % (dh >> 1) * 2, row = q / a.group;
    const uint16_t* v = a.v_rows + (size_t)head * dh + c;
    float sum[2] = {0.f, 0.f};
    bool odd = false;
#pragma unroll 1
    for (int j = from; j <= row; ++j) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const uint16_t x = v[(size_t)(r0 + j) * a.row_stride + e];
        if ((x & 0x7f80) == 0x7f80) sum[e] += bf2f(x), odd = true;
      }
    }
    if (!odd) continue;
    uint32_t* const at = reinterpret_cast<uint32_t*>(a.out + ((size_t)(r0 + row) * a.n_kv_heads * a.group + head * a.group + q % a.group) * dh + c);
    const uint32_t was = __hip_atomic_load(at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    *at = pack2bf(bf2f((uint16_t)was) + sum[0], bf2f((uint16_t)(was >> 16)) + sum[1]);
  }
}
// first key of the sequence's own blocks with a key that row `row` does not see
__device__ inline int first_partly_seen(int row) { return (row + 1) / CH_KEYS * CH_KEYS; }

// LDS.  A block's operands lie one after the other, 64 lanes' 16 bytes each, with gaps with which neither reading operands
// nor writing them from codes or rows meets a bank more often than it has to; lane + constant, so that one register
// addresses all of a block's.  K has two places for blocks, V three.  Behind them is what comes from memory, codes or
// rows as they are: two blocks' worth, of each wavefront its own, which nobody else reads.
template <int DH>
struct ChunkLds {
  static constexpr int STEPS = DH / 16;
  static constexpr int K_HALF = 512 + 16, K_STEP = 2 * K_HALF, K_TILE = STEPS * K_STEP, K_BLOCK = 2 * K_TILE;
  static constexpr int V_HALF = 512 + 64, V_STEP = 2 * V_HALF, V_TILE = STEPS * V_STEP, V_BLOCK = 2 * V_TILE;
  static constexpr int UNITS = DH / 64;  // KiB of a wavefront and block: so many of codes, twice of K rows and of V rows
  static constexpr int V0 = 2 * K_BLOCK, RAW0 = V0 + 3 * V_BLOCK, RAW = 2 * UNITS * 1024, BYTES = RAW0 + 2 * CH_WAVES * RAW;
  // K: step 2j + i holds columns 32 j + 16 hh + 8 i .. of row r
  __device__ static inline int k_at(int kt, int step, int hh, int r) { return kt * K_TILE + step * K_STEP + hh * K_HALF + r * 16; }
  // V^T: columns 32 mt .., keys 16 kg + 8 b + 4 hh ..
  __device__ static inline int v_at(int kt, int mt, int kg, int hh, int c32) {
    return kt * V_TILE + (2 * mt + kg) * V_STEP + hh * V_HALF + c32 * 16 + (c32 >> 3) * 16;
  }
};

// A tile of 32 queries: every wavefront has them all and pages of its own, each CH_WAVES-th of the range, first of the
// sequence's own rows, then of the cache, whose codes come to slots of its own in LDS and go from there to the matrix units.
// The wavefronts' sums are joined at the end.  In the other form seven wavefronts would only bring blocks for one: 64 sequences of
// a row over 2000 positions, 32 heads on 8, took 142 us so and take 80 here, one row over 131072, 64 heads on 8, 112 and 56
// (268 MB, 4.8 TB/s).
template <int DH>
struct FewLds {
  static constexpr int P = DH / 32, SLOTS = 256 / DH, SLOT = 2 * P * 1024;  // P KiB of codes of a page, K or V
  static constexpr int IMAGE = DH / 32 * 16 * 64;                           // accumulators of a wavefront
  static constexpr int BYTES = std::max(CH_WAVES * SLOTS * SLOT, CH_WAVES * (IMAGE + 2 * 32) * 4);
};
template <int DH>
__device__ __forceinline__ bool chunk_few(const ChunkArgs& a, const ChunkWork& w, int head, int sp, int part, int q0, int q1, uint8_t* smem) {
  using Lds = FewLds<DH>;
  constexpr int MT = DH / 32, STEPS = DH / 16, OW = Lds::IMAGE, P = Lds::P, SLOTS = Lds::SLOTS, SLOT = Lds::SLOT;
  const int tid = threadIdx.x, lane = tid & 63, n32 = lane & 31, hh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const ChunkSeq& seq = w.seq;
  const int qi = min(q0 + n32, q1 - 1), my_row = qi / a.group;
  const int pages = (seq.L + 31) >> 5, all = pages + (q1 - 1) / a.group / 32 + 1;  // the cache's, then own rows, 32 to a page
  const int p0 = (int)((int64_t)all * sp / w.splits), p1 = (int)((int64_t)all * (sp + 1) / w.splits), pend = min(p1, pages);
  const int mine = __builtin_amdgcn_readfirstlane(p0 + wave < pend ? (pend - p0 - wave + CH_WAVES - 1) / CH_WAVES : 0);
  const int32_t* const table = a.block_table + (size_t)w.s * a.max_blocks;
  const size_t plane = (size_t)head * a.n_blocks;
  const float f = a.scale_log2e;
  int ids = 0;  // of this wavefront's pages i, one per lane i % 64, and their scales
  float ksc = 1.f, vsc = 1.f;
  auto look_up = [&](int i0) {
    const bool there = i0 + lane < mine;
    const int id = there ? table[p0 + wave + (i0 + lane) * CH_WAVES] : 0;
    const bool ok = (unsigned)id < (unsigned)a.n_blocks;
    ids = ok ? id : 0;
    const float of_k = a.k_scale[plane + ids];
    ksc = ok ? of_k : NAN;  // a page that is not there makes its rows NaN
    vsc = a.v_scale[plane + ids];
  };
  bf16x8 qreg[STEPS];
  const uint16_t* qp = a.q + (size_t)(seq.r0 + my_row) * a.q_stride + (size_t)(head * a.group + qi % a.group) * DH + hh * 16;
#pragma unroll
  for (int j = 0; j < STEPS; ++j) qreg[j] = *reinterpret_cast<const bf16x8*>(qp + 32 * (j >> 1) + 8 * (j & 1));
  f32x16 o[MT];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt)
#pragma unroll
    for (int v = 0; v < 16; ++v) o[mt][v] = 0.f;
  float m = NO_REFERENCE, l = 0.f;
  u32x4 pk[2];
  // weights of 32 keys from their scores; a higher reference by each query for itself
  auto weigh = [&](const f32x16& s) {
#pragma clang fp contract(off)
    const float top = Softmax::largest(s, f), ref = top > m + SLACK ? top : m, alpha = __builtin_amdgcn_exp2f(m - ref);
    m = ref;
    float p[16], sum = 0.f;
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      const float x = s[v] * f;  // rounded by itself, as the reference was
      p[v] = __builtin_amdgcn_exp2f(x - m);
      sum += p[v];
    }
    l = l * alpha + sum;
#pragma unroll
    for (int kg = 0; kg < 2; ++kg)
#pragma unroll
      for (int e = 0; e < 4; ++e) pk[kg][e] = pack2bf(p[8 * kg + 2 * e], p[8 * kg + 2 * e + 1]);
    if (__ballot(alpha != 1.f)) q8_rescale<MT>(o, alpha);
  };
  look_up(0);
  int odd = 0;
  const int own0 = max(p0, pages), partly = first_partly_seen(q0 / a.group);
#pragma unroll 1
  for (int p = own0 + ((wave - (own0 - p0)) & (CH_WAVES - 1)); p < p1; p += CH_WAVES) {  // own rows
    const int j0 = (p - pages) * 32;
    const size_t row = (size_t)a.row_stride, first = (size_t)seq.r0 * row + (size_t)head * DH;
    bf16x8 k[STEPS];
    const uint16_t* const kp = a.k_rows + first + min(j0 + n32, seq.n - 1) * row + hh * 16;
#pragma unroll
    for (int j = 0; j < STEPS; ++j) k[j] = *reinterpret_cast<const bf16x8*>(kp + 32 * (j >> 1) + 8 * (j & 1));
    uint32_t v[MT][2][4];
#pragma unroll
    for (int kg = 0; kg < 2; ++kg)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint16_t* const vp = a.v_rows + first + min(j0 + 16 * kg + 8 * (e >> 2) + 4 * hh + (e & 3), seq.n - 1) * row + n32;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          uint32_t x = vp[32 * mt];
          const bool is_odd = j0 >= partly && (x & 0x7f80u) == 0x7f80u;
          odd |= (int)is_odd;
          x = is_odd ? 0u : x;
          v[mt][kg][e >> 1] = e & 1 ? v[mt][kg][e >> 1] | x << 16 : x;
        }
      }
    f32x16 s;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
    for (int j = 0; j < STEPS; ++j) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k[j], qreg[j], s, 0, 0, 0);
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (j0 + 8 * (i >> 2) + (i & 3) + 4 * hh > my_row) s[i] = -INFINITY;
    weigh(s);
#pragma unroll
    for (int kg = 0; kg < 2; ++kg)
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
        o[mt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, u32x4{v[mt][kg][0], v[mt][kg][1], v[mt][kg][2], v[mt][kg][3]}),
                                                        __builtin_bit_cast(bf16x8, pk[kg]), o[mt], 0, 0, 0);
  }
  const uint32_t slot0 = __builtin_amdgcn_readfirstlane((uint32_t)(size_t)(__attribute__((address_space(3))) uint8_t*)smem + wave * SLOTS * SLOT);
  const uint8_t* const slot_r = smem + wave * SLOTS * SLOT + lane * 16;
  auto ask = [&](int i, bool v) {
    const size_t page = (plane + (uint32_t)__builtin_amdgcn_readlane(ids, i & 63)) * (32 * DH);
    const uint32_t to = slot0 + i % SLOTS * SLOT + (v ? P * 1024 : 0);
#pragma unroll
    for (int j = 0; j < P; ++j) load_to_lds<false>((v ? a.v_pool : a.k_pool) + page + j * 1024, lane * 16, to + j * 1024);
  };
  // all but the newest n asked for have come
  auto arrived = [&](int n) {
    if (n >= 2 * SLOTS - 1) __builtin_amdgcn_s_waitcnt(P * (2 * SLOTS - 1) < 16 ? 0x0f70 + P * (2 * SLOTS - 1) : 0);
    else if (n >= 2) __builtin_amdgcn_s_waitcnt(0x0f70 + 2 * P);
    else if (n == 1) __builtin_amdgcn_s_waitcnt(0x0f70 + P);
    else __builtin_amdgcn_s_waitcnt(0x0f70);
    asm volatile("" ::: "memory");
  };
  float k_scales[SLOTS], v_scales[SLOTS];  // of the pages on their way
  auto scales_of = [&](int i, int to) {
    k_scales[to] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(ksc), i & 63));
    v_scales[to] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(vsc), i & 63));
  };
#pragma unroll
  for (int i = 0; i < SLOTS; ++i) {
    scales_of(i, i);
    if (i < mine) ask(i, false), ask(i, true);
  }
#pragma unroll 1
  for (int i = 0; i < mine; ++i) {
    const float k_of = k_scales[0], v_of = v_scales[0];
#pragma unroll
    for (int k = 0; k + 1 < SLOTS; ++k) k_scales[k] = k_scales[k + 1], v_scales[k] = v_scales[k + 1];
    const uint8_t* const at = slot_r + i % SLOTS * SLOT;
    const int behind = min(mine - 1 - i, SLOTS - 1), rest = seq.L - (p0 + wave + i * CH_WAVES) * 32;
    arrived(2 * behind + 1);
    u32x4 x[P];
#pragma unroll
    for (int j = 0; j < P; ++j) x[j] = *reinterpret_cast<const u32x4*>(at + j * 1024);
    f32x16 s;
#pragma unroll
    for (int v = 0; v < 16; ++v) s[v] = 0.f;
#pragma unroll
    for (int j = 0; j < P; ++j) {
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(operand(x[j][0], x[j][1], k_of), qreg[2 * j], s, 0, 0, 0);
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(operand(x[j][2], x[j][3], k_of), qreg[2 * j + 1], s, 0, 0, 0);
    }
    if ((__float_as_uint(k_of) & 0x7fffffffu) > 0x7f800000u)
#pragma unroll
      for (int v = 0; v < 16; ++v) s[v] = NAN;
    if (rest < 32)
#pragma unroll
      for (int v = 0; v < 16; ++v)
        if (8 * (v >> 2) + (v & 3) + 4 * hh >= rest) s[v] = -INFINITY;
    weigh(s);
    arrived(2 * behind);
#pragma unroll
    for (int j = 0; j < P; ++j) x[j] = *reinterpret_cast<const u32x4*>(at + P * 1024 + j * 1024);
    if (rest < 32)  // slots past the end may hold anything: their weights are 0, their values have to be numbers
#pragma unroll
      for (int j = 0; j < P; ++j)
#pragma unroll
        for (int d = 0; d < 4; ++d) {
          const int keep = min(max(rest - 8 * d - 4 * hh, 0), 4);
          x[j][d] &= keep == 4 ? 0xffffffffu : (1u << (8 * keep)) - 1u;
        }
#pragma unroll
    for (int kg = 0; kg < 2; ++kg)
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
        o[mt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(operand(x[mt][2 * kg], x[mt][2 * kg + 1], v_of), __builtin_bit_cast(bf16x8, pk[kg]), o[mt], 0, 0, 0);
    if (i + SLOTS < mine) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // what came has been read
      if (((i + SLOTS) & 63) == 0) look_up(i + SLOTS);
      scales_of(i + SLOTS, SLOTS - 1);
      ask(i + SLOTS, false);
      ask(i + SLOTS, true);
    }
  }
  // ---- the wavefronts' sums joined
  l += __shfl_xor(l, 32);
  const bool any_odd = __syncthreads_or(odd);
  float* const sum_o = reinterpret_cast<float*>(smem);
  float* const sum_m = sum_o + CH_WAVES * OW;
  float* const sum_l = sum_m + CH_WAVES * 32;
#pragma unroll
  for (int mt = 0; mt < MT; ++mt)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *reinterpret_cast<f32x4*>(sum_o + wave * OW + (mt * 4 + g) * 256 + lane * 4) = f32x4{o[mt][4 * g], o[mt][4 * g + 1], o[mt][4 * g + 2], o[mt][4 * g + 3]};
  if (hh == 0) sum_m[wave * 32 + n32] = m, sum_l[wave * 32 + n32] = l;
  __syncthreads();
  float top = NO_REFERENCE, share[CH_WAVES], sum = 0.f;
#pragma unroll
  for (int k = 0; k < CH_WAVES; ++k) top = fmaxf(top, sum_m[k * 32 + n32]);
#pragma unroll
  for (int k = 0; k < CH_WAVES; ++k) share[k] = __builtin_amdgcn_exp2f(sum_m[k * 32 + n32] - top), sum += share[k] * sum_l[k * 32 + n32];
  const size_t image = (size_t)part * CH_WAVES;
  const bool split = w.splits > 1;
  if (split && tid < 32 && part < a.max_parts) a.pm[image * 32 + n32] = top, a.pl[image * 32 + n32] = any_odd ? -sum : sum;
  const float inv = split ? 1.f : 1.0f / sum;
#pragma unroll
  for (int c = 0; c < MT * 4 / CH_WAVES; ++c) {
    const int u = c * CH_WAVES + wave;  // mt * 4 + g
    f32x4 r = {0, 0, 0, 0};
#pragma unroll
    for (int k = 0; k < CH_WAVES; ++k) r += *reinterpret_cast<const f32x4*>(sum_o + k * OW + u * 256 + lane * 4) * share[k];
    r *= inv;
    if (q0 + n32 >= q1) continue;
    if (!split)
      *reinterpret_cast<u32x2*>(a.out + ((size_t)(seq.r0 + my_row) * a.n_kv_heads * a.group + head * a.group + qi % a.group) * DH + 32 * (u >> 2) + 8 * (u & 3) + 4 * hh) =
          u32x2{pack2bf(r[0], r[1]), pack2bf(r[2], r[3])};
    else if (part < a.max_parts)
      *reinterpret_cast<f32x4*>(a.po + image * OW + u * 256 + lane * 4) = r;
  }
  return any_odd;
}

template <int DH, bool MANY>
__global__ __launch_bounds__(CH_THREADS, 2) void chunk_attn_q8_kernel(ChunkArgs a) {
  using Lds = ChunkLds<DH>;
  constexpr int MT = DH / 32, STEPS = DH / 16, OW = MT * 16 * 64;
  extern __shared__ __align__(16) uint8_t smem[];
  const int tid = threadIdx.x, lane = tid & 63, n32 = lane & 31, hh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  if (blockIdx.x == 0)  // sequences without work
    for (int s = tid; s < a.B; s += CH_THREADS) {
      const ChunkSeq q = chunk_seq(a, s);
      if (q.n <= 0) a.status[s] = q.n < 0;
    }
  ChunkPlan<MANY> plan(a);
  if (blockIdx.x == 0 && a.max_parts > 0) {
    const int n = plan.merges();
    if (tid == 0) a.merges[0] = min(n, CH_MAX_MERGES);
  }
  ChunkWork w;
  if (!plan.find(blockIdx.x, w)) return;
  const ChunkSeq seq = w.seq;
  const int nq = seq.n * a.group, splits = w.splits;
  const int head = w.nth % a.n_kv_heads, sp = w.nth / a.n_kv_heads % splits, tile = seq.tiles - 1 - w.nth / a.n_kv_heads / splits;
  const int row_len = a.n_kv_heads * a.group * DH;
  const int q0 = tile * (seq.few ? 32 : CH_QUERIES), q1 = min(nq, q0 + (seq.few ? 32 : CH_QUERIES));
  const bool judge = head == 0 && sp == 0 && tile == 0;
  if (seq.L < 0) {
    const int width = DH / 4;
    for (int i = tid; i < (q1 - q0) * width; i += CH_THREADS) {
      const int q = q0 + i / width;
      *reinterpret_cast<u32x2*>(a.out + (size_t)(seq.r0 + q / a.group) * row_len + (head * a.group + q % a.group) * DH + i % width * 4) = u32x2{0, 0};
    }
    if (judge && tid == 0) a.status[w.s] = 1;
    return;
  }
  const int32_t* table = a.block_table + (size_t)w.s * a.max_blocks;
  const int part = w.part0 + w.nth;
  if (splits > 1) {
    const int tiles_done = w.nth / a.n_kv_heads / splits, merge = w.merge0 + tiles_done * a.n_kv_heads + head;
    if (sp == 0 && tid == 0 && merge < CH_MAX_MERGES) {
      const bool room = w.part0 + (tiles_done + 1) * splits * a.n_kv_heads <= a.max_parts;  // (else ranges that overlap)
      reinterpret_cast<ChunkMerge*>(a.merges + 8)[merge] = ChunkMerge{seq.r0, q0, q1, head, room ? splits : 0, part, a.n_kv_heads, 0};
    }
  }
  auto verdict = [&]() {
    bool bad = false;
    for (int j = tid, pages = (seq.L + 31) >> 5; j < pages; j += CH_THREADS) bad = bad || (unsigned)table[j] >= (unsigned)a.n_blocks;
    bad = __syncthreads_or(bad);
    if (tid == 0) a.status[w.s] = bad;
  };
  if (seq.few) {
    const bool any_odd = chunk_few<DH>(a, w, head, sp, part, q0, q1, smem);
    if (any_odd && splits == 1) chunk_add_odd_values(a, seq.r0, head, DH, q0, q1, first_partly_seen(q0 / a.group));
    if (judge) verdict();
    return;
  }
  const int row_first = q0 / a.group, row_last = (q1 - 1) / a.group;
  const int cached = seq.cached(), blocks = cached + row_last / CH_KEYS + 1;  // of this tile
  const int b0 = __builtin_amdgcn_readfirstlane((int)((int64_t)blocks * sp / splits));
  const int b1 = __builtin_amdgcn_readfirstlane((int)((int64_t)blocks * (sp + 1) / splits));
  const size_t plane = (size_t)head * a.n_blocks;

  // queries: column n32; step 2j + i of the product: columns 32 j + 16 hh + 8 i ..
  const int qw = q0 + wave * 32, qi = min(qw + n32, nq - 1), my_row = qi / a.group;
  const bool live_wave = qw < nq;
  bf16x8 qreg[STEPS];
  {
    const uint16_t* qp = a.q + (size_t)(seq.r0 + my_row) * a.q_stride + (size_t)(head * a.group + qi % a.group) * DH + hh * 16;
#pragma unroll
    for (int j = 0; j < STEPS; ++j) qreg[j] = *reinterpret_cast<const bf16x8*>(qp + 32 * (j >> 1) + 8 * (j & 1));
  }
  int odd = 0;

  // ---- bringing blocks to LDS: asked for two blocks ahead, without registers, then turned into operands.
  // No branch in here that lanes take differently: the walk's accumulators would be copied around it.
  constexpr int UNITS = Lds::UNITS, PIECES = 4 * DH;  // 16 codes each, of K or V
  const uint32_t raw0 = __builtin_amdgcn_readfirstlane((uint32_t)(size_t)(__attribute__((address_space(3))) uint8_t*)smem + Lds::RAW0 + wave * Lds::RAW);
  uint8_t* const raw_r = smem + Lds::RAW0 + wave * Lds::RAW;
  constexpr int RAW_SLOT = CH_WAVES * Lds::RAW;
  // codes: this wavefront's units are of K or V, of one page of the block; this lane's place there and in LDS
  const int page_of = wave % (PIECES / 64) / (DH / 32), piece = tid % (2 * DH);
  auto is_v = [&](int i) { return (wave + i * CH_WAVES) / (PIECES / 64) != 0; };
  const int c16 = piece >> 5, unit_h = c16 & 1, unit_at = piece & 31;  // K: columns 16 c16 .. of row unit_at; V: column unit_at of 32 (c16 / 2)
  const int k_unit = Lds::k_at(page_of, c16 & ~1, unit_h, unit_at), v_unit = Lds::v_at(page_of, c16 >> 1, 0, unit_h, unit_at);
  // rows: each wavefront has eight of the block, this lane 16 bytes of K (of the same lane of V)
  constexpr int PER_ROW = DH / 8, ROWS_AT_ONCE = 64 / PER_ROW;
  const int my_p = lane % PER_ROW, my_r = lane / PER_ROW;
  int ids = 0, ids_from = -(1 << 30);  // pages ids_from .. + 63 of the sequence, one per lane, and their scales
  float ksc = 1.f, vsc = 1.f;
  float scale0[UNITS] = {}, scale1[UNITS] = {};  // of the codes on their way into slots 0 and 1
  auto ask = [&](int b) {  // into slot b % 2
    const uint32_t to = raw0 + (b & 1) * RAW_SLOT;
    if (b < cached) {
      if (b * 2 >= ids_from + 64 || ids_from < 0) {
        ids_from = b * 2;
        const int p = ids_from + lane, pages = (seq.L + 31) >> 5;
        const int id = table[min(p, pages - 1)];
        const bool there = p < pages, ok = (unsigned)id < (unsigned)a.n_blocks;
        ids = ok ? id : 0;
        const float of_k = a.k_scale[plane + ids], of_v = a.v_scale[plane + ids];
        ksc = !there ? 1.f : ok ? of_k : NAN;  // a page that is not there makes its rows NaN
        vsc = there ? of_v : 1.f;
      }
      const int at = 2 * b + page_of - ids_from;
      const size_t page = (plane + (uint32_t)__builtin_amdgcn_readlane(ids, at)) * (32 * DH);
#pragma unroll
      for (int i = 0; i < UNITS; ++i) load_to_lds<false>((is_v(i) ? a.v_pool : a.k_pool) + page, piece * 16, to + i * 1024);
#pragma unroll
      for (int i = 0; i < UNITS; ++i) {
        const float scale = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(is_v(i) ? vsc : ksc), at));
        scale0[i] = b & 1 ? scale0[i] : scale;
        scale1[i] = b & 1 ? scale : scale1[i];
      }
    } else {
      const int key0 = (b - cached) * CH_KEYS + wave * 8;
      const size_t first = (size_t)(seq.r0 + min(key0, seq.n - 1)) * a.row_stride + (size_t)head * DH;
      const int rows = max(seq.n - 1 - key0, 0);  // (those behind the last are the last)
#pragma unroll
      for (int i = 0; i < UNITS; ++i) {
        const uint32_t at = (uint32_t)min(i * ROWS_AT_ONCE + my_r, rows) * (uint32_t)(a.row_stride * 2) + my_p * 16;
        load_to_lds<false>(a.k_rows + first, at, to + i * 1024);
        load_to_lds<false>(a.v_rows + first, at, to + (UNITS + i) * 1024);
      }
    }
  };
  // block b has come; the operands of block b to its places
  auto arrived = [&](int b) {
    if (b + 1 >= b1) __builtin_amdgcn_s_waitcnt(0x0f70);           // vmcnt(0)
    else if (b + 1 < cached) __builtin_amdgcn_s_waitcnt(0x0f70 + UNITS);  // all but the next block's
    else __builtin_amdgcn_s_waitcnt(0x0f70 + 2 * UNITS);
    asm volatile("" ::: "memory");
  };
  auto convert = [&](int b, uint8_t* kbuf, uint8_t* vbuf) {
    const uint8_t* const raw = raw_r + (b & 1) * RAW_SLOT;
    if (b < cached) {
#pragma unroll
      for (int i = 0; i < UNITS; ++i) {
        u32x4 x = *reinterpret_cast<const u32x4*>(raw + i * 1024 + lane * 16);
        const float scale = b & 1 ? scale1[i] : scale0[i];
        const int rest = seq.L - (2 * b + page_of) * 32;
        if (is_v(i) && rest < 32) {  // slots past the end may hold anything: their weights are 0, their values have to be numbers
#pragma unroll
          for (int d = 0; d < 4; ++d) {
            const int keep = min(max(rest - 8 * d - 4 * unit_h, 0), 4);
            x[d] &= keep == 4 ? 0xffffffffu : (1u << (8 * keep)) - 1u;
          }
        }
        bf16x8 lo = operand(x[0], x[1], scale), hi = operand(x[2], x[3], scale);
        if (!is_v(i) && (__float_as_uint(scale) & 0x7fffffffu) > 0x7f800000u) {
          const u32x4 none = {0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u};
          lo = hi = __builtin_bit_cast(bf16x8, none);
        }
        uint8_t* const to = is_v(i) ? vbuf + v_unit : kbuf + k_unit;
        *reinterpret_cast<bf16x8*>(to) = lo;
        *reinterpret_cast<bf16x8*>(to + (is_v(i) ? Lds::V_STEP : Lds::K_STEP)) = hi;
      }
    } else {
      const int key0 = (b - cached) * CH_KEYS;
#pragma unroll
      for (int i = 0; i < UNITS; ++i) {
        const int row = wave * 8 + i * ROWS_AT_ONCE + my_r;
        *reinterpret_cast<u32x4*>(kbuf + Lds::k_at(row >> 5, (my_p >> 2) * 2 + (my_p & 1), (my_p >> 1) & 1, row & 31)) =
            *reinterpret_cast<const u32x4*>(raw + i * 1024 + lane * 16);
      }
      // four rows, four columns (for heads of 64 the upper lanes do what the lower ones do)
      const int quad = wave * 2 + (lane / (DH / 4) & 1), cq = lane % (DH / 4);
      uint32_t v[4][2];
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        const u32x2 x = *reinterpret_cast<const u32x2*>(raw + UNITS * 1024 + ((quad & 1) * 4 + d) * (2 * DH) + cq * 8);
        v[d][0] = x[0], v[d][1] = x[1];
      }
      if (key0 >= first_partly_seen(row_first)) {
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const bool lo = (v[d][e] & 0x7f80u) == 0x7f80u, hi = (v[d][e] & 0x7f800000u) == 0x7f800000u;
            v[d][e] &= (lo ? 0xffff0000u : ~0u) & (hi ? 0xffffu : ~0u);
            odd |= (int)lo | (int)hi;
          }
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int c = 4 * cq + e;
        const uint32_t x0 = v[0][e >> 1], x1 = v[1][e >> 1], x2 = v[2][e >> 1], x3 = v[3][e >> 1];
        const u32x2 col = e & 1 ? u32x2{(x0 >> 16) | (x1 & 0xffff0000u), (x2 >> 16) | (x3 & 0xffff0000u)}
                                : u32x2{(x0 & 0xffffu) | (x1 << 16), (x2 & 0xffffu) | (x3 << 16)};
        *reinterpret_cast<u32x2*>(vbuf + Lds::v_at(quad >> 3, c >> 5, (quad >> 2) & 1, quad & 1, c & 31) + ((quad >> 1) & 1) * 8) = col;
      }
    }
  };

  // ---- the walk, tile after tile of 32 keys, two in a block.  With a tile's scores in registers, a step has the last tile's
  // weights times its values beside this one's exponentials, then the products with the next tile's keys.
  f32x16 o[MT], s;
  u32x4 pk[2] = {};  // weights of the last tile
  float m = NO_REFERENCE, l = 0.f, top = 0.f;
  const float f = a.scale_log2e;
#pragma unroll
  for (int mt = 0; mt < MT; ++mt)
#pragma unroll
    for (int v = 0; v < 16; ++v) o[mt][v] = 0.f;
  const int k_lane = Lds::k_at(0, 0, hh, n32), v_lane = Lds::V0 + Lds::v_at(0, 0, 0, hh, n32);
  auto scores = [&](const uint8_t* at) {
    f32x16 to;
#pragma unroll
    for (int v = 0; v < 16; ++v) to[v] = 0.f;
#pragma unroll
    for (int j = 0; j < STEPS; ++j)
      to = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8*>(at + j * Lds::K_STEP), qreg[j], to, 0, 0, 0);
    s = to;
  };
  auto values = [&](const uint8_t* at) {
#pragma unroll
    for (int kg = 0; kg < 2; ++kg)
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
        o[mt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8*>(at + (2 * mt + kg) * Lds::V_STEP),
                                                        __builtin_bit_cast(bf16x8, pk[kg]), o[mt], 0, 0, 0);
  };
  auto pack = [&](const float (&p)[16]) {
#pragma unroll
    for (int kg = 0; kg < 2; ++kg)
#pragma unroll
      for (int e = 0; e < 4; ++e) pk[kg][e] = pack2bf(p[8 * kg + 2 * e], p[8 * kg + 2 * e + 1]);
  };
  const int tiles = 2 * (b1 - b0);
  // Block b + 1 takes the K place of block b - 1 and the V place of block b - 2.  Both were last read in the first step of
  // block b - 1, before that block's barrier.
  int b = b0, place = 0;  // the current block, and its V place
  auto k_block = [&](int ahead) { return smem + ((b - b0 + ahead) & 1) * Lds::K_BLOCK; };
  auto v_block = [&](int ahead) {
    const int i = place + ahead;
    return smem + (i - (3 & ~((i - 3) >> 31))) * Lds::V_BLOCK;
  };
  auto arrive = [&](int t) {  // in front of tile t
    if (t & 1) {
      __syncthreads();
    } else if (b + 1 < b1) {
      arrived(b + 1);
      convert(b + 1, k_block(1), v_block(1) + Lds::V0);
      if (b + 3 < b1) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // what came has been read
        ask(b + 3);
      }
    }
  };
  auto leave = [&](int t) {
    b += t & 1;
    const int next = place + (t & 1);
    place = next & ((next - 3) >> 31);
  };
  auto next_keys = [&](int t) { return k_block(t & 1) + (1 - (t & 1)) * Lds::K_TILE + k_lane; };
  auto last_values = [&](int t) { return v_block(2 - 2 * (t & 1)) + (1 - (t & 1)) * Lds::V_TILE + v_lane; };
  if (tiles > 0) {
    ask(b0);
    if (b0 + 1 < b1) ask(b0 + 1);
    arrived(b0);
    convert(b0, k_block(0), v_block(0) + Lds::V0);
    if (b0 + 2 < b1) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      ask(b0 + 2);
    }
    __syncthreads();
  }
  if (!live_wave) {
    for (int t = 0; t < tiles; ++t) {
      arrive(t);
      leave(t);
    }
  } else if (tiles > 0) {
    // tiles before `plain_end` of the cache and of the own rows are seen whole by all queries
    const int cached_end = 2 * (min(b1, cached) - b0) - (seq.L < cached * CH_KEYS && b1 >= cached ? 2 : 0);
    const int own_begin = max(2 * (cached - b0), 0), own_end = own_begin + 2 * ((row_first + 1) / CH_KEYS) - 2 * max(b0 - cached, 0);
    bool far = false;
    auto plain_until = [&](int t) {  // the first tile from t on that is not
      const int end = t < cached_end ? cached_end : t >= own_begin && t < own_end ? own_end : t;
      return far ? t : min(end, tiles - 1);
    };
    scores(k_block(0) + k_lane);
    top = Softmax::largest(s, f);
    int t = 0, until = 0;
    arrive(t);
    auto stop = [&]() {
      return (__ballot(top > m + SLACK) | (uint64_t)(int64_t)(__builtin_amdgcn_readfirstlane(until - 1 - t) >> 31)) != 0;
    };
    for (;;) {
      // The loop has one way out, at its end, in front of a tile that is masked or lifts a reference: a condition around the
      // accumulators, or a way out before they change, would have them copied every time.
      if (!stop()) do {
        float p[16], sum = 0.f;
#pragma unroll
        for (int v = 0; v < 16; ++v) p[v] = fmaf(s[v], f, -m);
        const uint8_t *const k_from = next_keys(t), *const v_from = last_values(t);
        // in this order: operands asked for a product before they are needed (2 to 4 took 1 to 4 % longer), exponentials beside the products
        constexpr int AHEAD = 1, EXPS = 16 / STEPS;
        bf16x8 kop[STEPS], vop[STEPS];
        auto ask = [&](int j) {
          kop[j] = *reinterpret_cast<const bf16x8*>(k_from + j * Lds::K_STEP);
          vop[j] = *reinterpret_cast<const bf16x8*>(v_from + (2 * (j % MT) + j / MT) * Lds::V_STEP);
        };
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) ask(j);
#pragma unroll
        for (int v = 0; v < 16; ++v) s[v] = 0.f;
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int j = 0; j < STEPS; ++j) {
          if (j + AHEAD < STEPS) ask(j + AHEAD);
          s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kop[j], qreg[j], s, 0, 0, 0);
#pragma unroll
          for (int e = 0; e < EXPS / 2; ++e) p[EXPS * j + e] = __builtin_amdgcn_exp2f(p[EXPS * j + e]);
          __builtin_amdgcn_sched_barrier(0);
          o[j % MT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vop[j], __builtin_bit_cast(bf16x8, pk[j / MT]), o[j % MT], 0, 0, 0);
#pragma unroll
          for (int e = EXPS / 2; e < EXPS; ++e) p[EXPS * j + e] = __builtin_amdgcn_exp2f(p[EXPS * j + e]);
#pragma unroll
          for (int e = 0; e < EXPS; ++e) sum += p[EXPS * j + e];
          // (else they would be worked out where they are used, a step later)
#pragma unroll
          for (int e = 0; e < EXPS; ++e) asm volatile("" : "+v"(p[EXPS * j + e]));
          asm volatile("" : "+v"(sum));
          __builtin_amdgcn_sched_barrier(0);
        }
        l += sum;
        pack(p);
        asm volatile("" : "+v"(pk[0]), "+v"(pk[1]), "+v"(l));
        top = Softmax::largest(s, f);
        leave(t);
        ++t;
        arrive(t);
      } while (!stop());
      {
        const bool own = b >= cached;
        const int limit = (own ? my_row + 1 : seq.L) - (own ? b - cached : b) * CH_KEYS - 32 * (t & 1) - 4 * hh;
#pragma unroll
        for (int v = 0; v < 16; ++v)
          if (8 * (v >> 2) + (v & 3) >= limit) s[v] = -INFINITY;
      }
      top = Softmax::largest(s, f);
      // Each query's reference by itself, and its weights by one formula whatever the step: its result does not depend, in any bit,
      // on those beside it, which decide which step a tile goes through.
      const float ref = top > m + SLACK ? top : m, alpha = __builtin_amdgcn_exp2f(m - ref);
      m = ref;
      const bool is_far = fabsf(m) > 1048576.f && m != NO_REFERENCE;
      far = __ballot(is_far) != 0;
      float p[16], sum = 0.f;
      {
#pragma clang fp contract(off)
        // Fused as above, what the reference's own product was rounded by stays in the exponent: the same for all keys, so that it
        // goes out with the sum, while it is small.  Far from zero it would overflow, and product and difference are rounded one by one.
#pragma unroll
        for (int v = 0; v < 16; ++v) p[v] = fmaf(s[v], f, -m);
        if (far)
#pragma unroll
          for (int v = 0; v < 16; ++v) {
            const float x = s[v] * f;
            p[v] = is_far ? x - m : p[v];
          }
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          p[v] = __builtin_amdgcn_exp2f(p[v]);
          sum += p[v];
        }
      }
      if (t > 0) values(last_values(t));
      l = l * alpha + sum;
      pack(p);
      if (__ballot(alpha != 1.f)) q8_rescale<MT>(o, alpha);
      if (t == tiles - 1) break;
      scores(next_keys(t));
      top = Softmax::largest(s, f);
      leave(t);
      until = __builtin_amdgcn_readfirstlane(plain_until(++t));
      arrive(t);
    }
    values(v_block(0) + Lds::V_TILE + v_lane);
  }
  const bool any_odd = __syncthreads_or(odd);

  l += __shfl_xor(l, 32);
  if (splits == 1) {
    if (qw + n32 < nq) {
      const float inv = 1.0f / l;
      uint16_t* dst = a.out + (size_t)(seq.r0 + my_row) * row_len + (size_t)(head * a.group + qi % a.group) * DH + 4 * hh;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const u32x2 v = {pack2bf(o[mt][4 * g] * inv, o[mt][4 * g + 1] * inv), pack2bf(o[mt][4 * g + 2] * inv, o[mt][4 * g + 3] * inv)};
          *reinterpret_cast<u32x2*>(dst + 32 * mt + 8 * g) = v;
        }
    }
    if (any_odd) chunk_add_odd_values(a, seq.r0, head, DH, q0, q1, first_partly_seen(row_first));
  } else {
    if (live_wave && part < a.max_parts) {  // (else more work than T rows can be: ranges that overlap)
      const size_t image = (size_t)part * CH_WAVES + wave;
      if (hh == 0) {
        a.pm[image * 32 + n32] = m;
        a.pl[image * 32 + n32] = any_odd ? -l : l;  // (a sum of weights is not negative)
      }
      if (qw + n32 < nq) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int g = 0; g < 4; ++g)
            *reinterpret_cast<f32x4*>(a.po + image * OW + (mt * 4 + g) * 256 + lane * 4) =
                f32x4{o[mt][4 * g], o[mt][4 * g + 1], o[mt][4 * g + 2], o[mt][4 * g + 3]};
      }
    }
  }
  if (judge) verdict();
}

// Merges the partials of 32 queries of a (sequence, tile, K/V head) in split order, 32 columns per wavefront, every second
// split from h on, four at a time with all their loads together; the two sums are joined through LDS.
template <int DH>
__global__ __launch_bounds__(128 * (DH / 32)) void chunk_merge_kernel(ChunkArgs a) {
  constexpr int MT = DH / 32, OW = MT * 16 * 64, BATCH = 4, H = 2;
  __shared__ float sm_m[32], sm_l[32];
  __shared__ f32x4 sm_o[4][64 * MT];
  const int tid = threadIdx.x, lane = tid & 63, n32 = lane & 31, hh = lane >> 5, mt = (tid >> 6) % MT, h = tid / (64 * MT);
  const int all = a.merges[0] * CH_WAVES;
  for (int u = blockIdx.x; u < all; u += gridDim.x) {
    const int x = u / CH_WAVES, wave = u % CH_WAVES;
    const ChunkMerge w = reinterpret_cast<const ChunkMerge*>(a.merges + 8)[x];
    const int qw = w.q0 + wave * 32, qi = qw + n32;
    if (qw >= w.q1 || w.splits == 0) continue;
    float m = NO_REFERENCE, l = 0.f;
    bool odd = false;
    f32x4 o[4] = {};
    for (int s0 = h; s0 < w.splits; s0 += H * BATCH) {
      float pm[BATCH], pl[BATCH];
      f32x4 po[BATCH][4];
#pragma unroll
      for (int k = 0; k < BATCH; ++k) {
        const size_t image = (size_t)(w.part + min(s0 + H * k, w.splits - 1) * w.step) * CH_WAVES + wave;
        pm[k] = a.pm[image * 32 + n32];
        pl[k] = a.pl[image * 32 + n32];
#pragma unroll
        for (int g = 0; g < 4; ++g)
          po[k][g] = qi < w.q1 ? *reinterpret_cast<const f32x4*>(a.po + image * OW + (mt * 4 + g) * 256 + lane * 4) : f32x4{0, 0, 0, 0};
      }
      float top = m;
#pragma unroll
      for (int k = 0; k < BATCH; ++k) top = fmaxf(top, pm[k]);
      const float keep = __builtin_amdgcn_exp2f(m - top);
      m = top;
      l *= keep;
#pragma unroll
      for (int g = 0; g < 4; ++g) o[g] *= keep;
#pragma unroll
      for (int k = 0; k < BATCH; ++k) {
        if (s0 + H * k >= w.splits) break;
        const float f = __builtin_amdgcn_exp2f(pm[k] - m);
        odd = odd || (__float_as_uint(pl[k]) >> 31) != 0;
        l += f * fabsf(pl[k]);
#pragma unroll
        for (int g = 0; g < 4; ++g) o[g] += po[k][g] * f;
      }
    }
    if (h > 0) {
#pragma unroll
      for (int g = 0; g < 4; ++g) sm_o[g][mt * 64 + lane] = o[g];
      if (mt == 0 && hh == 0) sm_m[n32] = m, sm_l[n32] = l;
    }
    const bool any_odd = __syncthreads_or(odd);
    if (h == 0 && qi < w.q1) {
      const float top = fmaxf(m, sm_m[n32]), keep = __builtin_amdgcn_exp2f(m - top), f = __builtin_amdgcn_exp2f(sm_m[n32] - top);
      const float inv = 1.0f / (l * keep + sm_l[n32] * f);
      uint16_t* dst = a.out + ((size_t)(w.r0 + qi / a.group) * a.n_kv_heads * a.group + w.head * a.group + qi % a.group) * DH + 32 * mt + 4 * hh;
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4 r = (o[g] * keep + sm_o[g][mt * 64 + lane] * f) * inv;
        *reinterpret_cast<u32x2*>(dst + 8 * g) = u32x2{pack2bf(r[0], r[1]), pack2bf(r[2], r[3])};
      }
    }
    if (any_odd) chunk_add_odd_values(a, w.r0, w.head, DH, qw, min(w.q1, qw + 32), first_partly_seen(w.q0 / a.group));
    __syncthreads();  // LDS is free again
  }
}

// ------------------------------------------------------------------ launch
static int chunk_max_parts(int T, int max_prefix) {
  const long most = ((long)max_prefix + CH_KEYS - 1) / CH_KEYS + ((long)T + CH_KEYS - 1) / CH_KEYS;  // blocks of a sequence
  return most <= CH_LEAST ? 0 : CH_MAX_PARTS;
}
size_t attn_chunk_ws_floats(int B, int T, int group, int n_kv_heads, int head_dim, int max_prefix) {
  const size_t parts = (size_t)chunk_max_parts(T, max_prefix);
  return parts == 0 ? 0 : parts * CH_WAVES * (32 * head_dim + 64) + 8 * (CH_MAX_MERGES + 1);
}

template <int DH, bool MANY>
static int chunk_run(const ChunkArgs& a, hipStream_t st) {
  constexpr size_t lds = std::max(ChunkLds<DH>::BYTES, FewLds<DH>::BYTES);
  static DeviceOnce once;
  allow_lds(once, chunk_attn_q8_kernel<DH, MANY>, lds);
  const long queries = (long)a.T * a.group, most = (queries / 32 + a.B) * a.n_kv_heads;
  const long tiles = std::min(most, (queries / CH_QUERIES + CH_FEW / 32 * a.B) * a.n_kv_heads);
  const long items = MANY ? tiles : std::min(most, tiles + (long)RESIDENT);  // with those of short sequences
  const int grid = (int)std::min(items + a.max_parts, 1l << 30);
  chunk_attn_q8_kernel<DH, MANY><<<grid, CH_THREADS, lds, st>>>(a);
  int rc = check_launch();
  if (rc != TRJ_OK || a.max_parts == 0) return rc;
  chunk_merge_kernel<DH><<<CH_WAVES * (int)std::min(items, 64l), 128 * (DH / 32), 0, st>>>(a);
  return check_launch();
}

int launch_attn_chunk_q8(const uint16_t* q, int q_stride, const void* k_pool, const void* v_pool, const float* k_scale,
                         const float* v_scale, const uint16_t* k_rows, const uint16_t* v_rows, int row_stride,
                         const int32_t* node_off, const int32_t* block_table, int max_blocks, const int32_t* prefix_len,
                         int B, int T, int n_heads, int n_kv_heads, int head_dim, int n_blocks, int max_prefix, float scale,
                         float* ws, uint16_t* out, int32_t* status, hipStream_t st) {
  const int group = n_heads / n_kv_heads, parts = chunk_max_parts(T, max_prefix);
  const size_t images = (size_t)parts * CH_WAVES;
  float* const pm = ws + images * 32 * head_dim;
  const ChunkArgs a{q, k_rows, v_rows, (const uint8_t*)k_pool, (const uint8_t*)v_pool, k_scale, v_scale, node_off, block_table,
                    prefix_len, q_stride, row_stride, max_blocks, B, T, n_kv_heads, group, n_blocks, max_prefix, parts,
                    scale * LOG2E, ws, pm, pm + images * 32, (int32_t*)(pm + images * 64), out, status};
  if (B > 64) return head_dim == 128 ? chunk_run<128, true>(a, st) : chunk_run<64, true>(a, st);
  return head_dim == 128 ? chunk_run<128, false>(a, st) : chunk_run<64, false>(a, st);
}

}  // namespace trj
