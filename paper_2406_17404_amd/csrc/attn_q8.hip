// Tree attention over the paged 8-bit cache, fp32 softmax and accumulation.
//
//   out_i = sum_j w_ij v_j / sum_j w_ij,  w_ij = 2^(s_ij - max_j s_ij),  s_ij = scale * log2(e) * q_i . k_j
// over the cached positions j < prefix and the rows j of the tree on the path of i.
//
// The work is streaming the sequence's codes once.  All query heads of a K/V head are worked on
// together: query p of a sequence is (node p / G, head p % G of the group).  A workgroup owns a
// contiguous range of 32-key blocks of one (sequence, K/V head) and NTW tiles of 32 queries;
// wavefront (key stream, tile) walks every KS-th block for one tile:
//   S^T[keys, queries] = K[keys, dh] * Q^T          (v_mfma_f32_32x32x16_bf16)
//   O^T[dh, queries]  += V^T[dh, keys] * P^T[keys, queries]
// A page is laid out so that 16 contiguous bytes per lane are two such A operands; codes times their
// power-of-two scale are bf16 numbers, exactly, in one instruction per two (v_cvt_scalef32_pk_bf16_fp8),
// so what is rounded to 16 bits is what the 16-bit attention rounds: the weights w (relative
// error 2^-9 each, independent) and the result.
// Cached blocks come first in a range, then the blocks of the tree's own rows, which are bf16
// in the order the projection left them; only these and the last cached page need a mask.
//
// How the keys are split is decided on the device, where the lengths are: every workgroup scans the
// sequences (64 per round), works out the same plan and finds its own part of it.
#include <algorithm>

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
  int target;  // workgroups aimed at
  int min_blocks;  // of a split, at least
  int max_parts;   // images that the workspace holds
  float scale_log2e;
  float *po, *pm, *pl;  // un-normalised partials: [part][tile] images of the accumulators, maxima and sums of 32 queries
  uint16_t* out;
  int32_t* status;
};

// what a sequence has to do; nodes < 0: nothing but the verdict
struct Q8Seq {
  int r0, nodes, L, cached, blocks;
};
__device__ inline Q8Seq q8_seq(const Q8Args& a, int s) {
  const int r0 = a.node_off[s], r1 = a.node_off[s + 1], L = a.prefix_len[s];
  Q8Seq q{r0, r1 - r0, L, 0, 0};
  if (r0 < 0 || r1 < r0 || r1 > a.T) q.nodes = -1;
  const bool fits = L >= 0 && L <= a.max_prefix && (L + 31) / 32 <= a.max_blocks && q.nodes <= TRJ_N_MAX;
  if (q.nodes > 0 && fits) {
    q.cached = (L + 31) / 32;
    q.blocks = q.cached + (q.nodes + 31) / 32;
  } else if (q.nodes > 0) {
    q.L = -1;  // rows of zeros: one block of work
    q.blocks = 1;
  }
  return q;
}
// The plan: a split has `chunk` blocks at most, of one sequence evenly many.
struct Q8Plan {
  int chunk;
};
template <int NTW>
__device__ inline int q8_groups(const Q8Args& a, const Q8Seq& q) {  // query groups
  const int n = min(q.nodes, q.L < 0 ? 1 : TRJ_N_MAX);
  return n <= 0 ? 0 : (n * a.group + 32 * NTW - 1) / (32 * NTW);
}
template <int NTW>
__device__ inline Q8Plan q8_plan(const Q8Args& a) {
  long work = 0;
  for (int s0 = 0; s0 < a.B; s0 += 64) {
    const int s = s0 + (int)(threadIdx.x & 63);
    long w = 0;
    if (s < a.B) {
      const Q8Seq q = q8_seq(a, s);
      w = (long)q8_groups<NTW>(a, q) * a.n_kv_heads * q.blocks;
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) w += __shfl_xor(w, o);
    work += w;
  }
  const long c = (work + a.target - 1) / a.target;
  return Q8Plan{(int)max(c, (long)a.min_blocks)};
}
__device__ inline int q8_splits(const Q8Plan& p, const Q8Seq& q) { return (q.blocks + p.chunk - 1) / p.chunk; }

__device__ inline uint32_t bf16_pair(uint32_t codes, float scale, bool hi) {
  return hi ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, true))
            : __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, false));
}
__device__ inline bf16x8 operand(uint32_t a, uint32_t b, float scale) {  // 8 codes
  const u32x4 v = {bf16_pair(a, scale, false), bf16_pair(a, scale, true), bf16_pair(b, scale, false), bf16_pair(b, scale, true)};
  return __builtin_bit_cast(bf16x8, v);
}

// Running softmax of one tile of 32 queries, a query per lane and its partner lane + 32: scores of 32
// keys in, -infinity where not visible; bf16 weights out (the B operand of the second product).
struct Softmax {
  float m = -INFINITY, l = 0.f;
  __device__ inline float take(const float (&s)[16], u32x4 (&pk)[2]) {  // the factor of the sums so far
    float mx = s[0];
#pragma unroll
    for (int v = 1; v < 16; ++v) mx = fmaxf(mx, s[v]);
    mx = fmaxf(mx, __shfl_xor(mx, 32));
    const float top = fmaxf(m, mx);
    const float ref = top == -INFINITY ? 0.f : top;  // nothing visible yet: weights 2^-inf = 0
    const float alpha = __builtin_amdgcn_exp2f(m - ref);
    float p[16], sum = 0.f;
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      p[v] = __builtin_amdgcn_exp2f(s[v] - ref);
      sum += p[v];
    }
    l = l * alpha + sum;
    m = top;
#pragma unroll
    for (int kg = 0; kg < 2; ++kg)
#pragma unroll
      for (int e = 0; e < 4; ++e) pk[kg][e] = pack2bf(p[8 * kg + 2 * e], p[8 * kg + 2 * e + 1]);
    return alpha;
  }
};

template <int MTV>
__device__ inline void q8_rescale(f32x16 (&o)[MTV], float alpha) {
  if (__builtin_amdgcn_ballot_w64(alpha != 1.0f) == 0) return;
#pragma unroll
  for (int mt = 0; mt < MTV; ++mt)
#pragma unroll
    for (int v = 0; v < 16; ++v) o[mt][v] *= alpha;
}

// An infinity or NaN among the tree's V rows: times the weight 0 of a row that does not see it it
// would be NaN.  Such values are taken out of the operand and added to the rows that do see
// them.  key: of the block's 32; value: V(key, c) as bits.
template <int MTV, class F, class G>
__device__ __forceinline__ void q8_add_odd_values(f32x16 (&o)[MTV], const u32x4 (&pk)[2], int keys, F visible, G value) {
  const int lane = threadIdx.x & 63, hh = lane >> 5;
#pragma unroll 1
  for (int key = 0; key < keys; ++key) {
    const int v = (key >> 3) * 4 + (key & 3);  // the register that holds its weight, on half (key >> 2) & 1
    uint32_t word = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i == v >> 1) word = pk[i >> 2][i & 3];
    word = (uint32_t)__shfl((int)word, (lane & 31) + 32 * ((key >> 2) & 1));
    const float w = bf2f((uint16_t)(v & 1 ? word >> 16 : word));
    if (!visible(key)) continue;
#pragma unroll
    for (int mt = 0; mt < MTV; ++mt)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const uint16_t x = value(key, 32 * mt + 8 * (r >> 2) + 4 * hh + (r & 3));
        if ((x & 0x7f80) == 0x7f80) o[mt][r] += w * bf2f(x);
      }
  }
}

template <int DH, int NTW, int KS>
__global__ __launch_bounds__(KS* NTW * 64, 2) void tree_attn_q8_kernel(Q8Args a) {
  constexpr int MTV = DH / 32, OW = MTV * 16 * 64;
  extern __shared__ __align__(16) uint8_t smem[];  // parts handed over
  __shared__ float sm_m[KS * NTW][32], sm_l[KS * NTW][32];
  const int tid = threadIdx.x, lane = tid & 63, n32 = lane & 31, hh = lane >> 5;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int nt = wv % NTW, ks = wv / NTW;
  const Q8Plan plan = q8_plan<NTW>(a);
  if (blockIdx.x == 0)  // sequences without work
    for (int s = tid; s < a.B; s += KS * NTW * 64) {
      const Q8Seq q = q8_seq(a, s);
      if (q8_groups<NTW>(a, q) == 0) a.status[s] = q.nodes < 0;
    }
  auto item = [&](int x) -> bool {  // false: behind the last one
  // item -> (sequence, query group, split, K/V head), K/V head fastest: the groups that read the same
  // blocks are a multiple of the heads apart, which is mostly one die (XCD)
  int s, nth;
  if (!find_seq(x, a.B, [&](int y) {
        const Q8Seq q = q8_seq(a, y);
        return q8_groups<NTW>(a, q) * a.n_kv_heads * q8_splits(plan, q);
      }, s, nth)) return false;
  const Q8Seq seq = q8_seq(a, s);
  const int splits = q8_splits(plan, seq);
  const int head = nth % a.n_kv_heads, sp = nth / a.n_kv_heads % splits, qg = nth / a.n_kv_heads / splits;
  const int nq = seq.nodes * a.group, n = seq.nodes;
  const int row_len = a.n_kv_heads * a.group * DH;  // of out
  auto zero_rows = [&](int i0, int i1) {  // nodes i0.. of the sequence, this K/V head's part
    const size_t w = (size_t)a.group * DH / 4;
    const u32x2 z = {0, 0};
    for (size_t i = tid; i < (i1 - i0) * w; i += KS * NTW * 64)
      *reinterpret_cast<u32x2*>(a.out + (size_t)(seq.r0 + i0 + i / w) * row_len + head * a.group * DH + i % w * 4) = z;
  };
  const bool first = sp == 0 && qg == 0;
  if (seq.L < 0) {
    zero_rows(0, n);
    if (first && head == 0 && tid == 0) a.status[s] = 1;
    return true;
  }
  const TreeParents par = load_parents(a.parent, seq.r0, n);
  if (!tree_valid(par, n)) {  // the same in every wavefront
    if (first) zero_rows(0, n);
    if (first && head == 0 && tid == 0) a.status[s] = 1;
    return true;
  }
  const int32_t* table = a.block_table + (size_t)s * a.max_blocks;
  if (first && head == 0) {  // the verdict on the sequence's pages
    bool bad = false;
    for (int j = tid; j < seq.cached; j += KS * NTW * 64) bad = bad || (unsigned)table[j] >= (unsigned)a.n_blocks;
    bad = __syncthreads_or(bad);
    if (tid == 0) a.status[s] = bad;
  }
  const int per = (seq.blocks + splits - 1) / splits;
  const int b0 = sp * per, b1 = min(seq.blocks, b0 + per);

  // this lane's query
  const int qi = (qg * NTW + nt) * 32 + n32, qc = min(qi, nq - 1);
  const int node = qc / a.group, qhead = head * a.group + qc % a.group;
  const bool live = (qg * NTW + nt) * 32 < nq;
  bf16x8 qreg[2 * MTV];  // step 2j + i: columns 32j + 16hh + 8i ..
  {
    const uint16_t* qp = a.q + (size_t)(seq.r0 + node) * a.q_stride + (size_t)qhead * DH + hh * 16;
#pragma unroll
    for (int j = 0; j < MTV; ++j) {
      qreg[2 * j] = *reinterpret_cast<const bf16x8*>(qp + 32 * j);
      qreg[2 * j + 1] = *reinterpret_cast<const bf16x8*>(qp + 32 * j + 8);
    }
  }
  f32x16 o[MTV];
#pragma unroll
  for (int mt = 0; mt < MTV; ++mt)
#pragma unroll
    for (int v = 0; v < 16; ++v) o[mt][v] = 0.f;
  Softmax sm;

  // ---- cached blocks b0 + ks, b0 + ks + KS, ..
  const int cend = min(b1, seq.cached);
  const int mine = live && b0 + ks < cend ? (cend - b0 - ks + KS - 1) / KS : 0;
  const size_t plane = (size_t)head * a.n_blocks;
  int ids = 0;           // page, K and V scale of block i of this stream, i % 64 == lane
  float ksc = 0.f, vsc = 0.f;
  auto look_up = [&](int i0) {
    const int i = i0 + lane;
    if (i < mine) {
      ids = table[b0 + ks + i * KS];
      const bool ok = (unsigned)ids < (unsigned)a.n_blocks;
      ids = ok ? ids : 0;
      ksc = a.k_scale[plane + ids] ;
      vsc = a.v_scale[plane + ids];
      if (!ok) ksc = NAN;
    }
  };
  u32x4 kreg[MTV], vreg[MTV];
  auto load = [&](u32x4 (&r)[MTV], const uint8_t* pool, int i) {
    const size_t page = (uint32_t)__builtin_amdgcn_readlane(ids, i & 63);
    const u32x4* p = reinterpret_cast<const u32x4*>(pool + (plane + page) * 32 * DH) + lane;
#pragma unroll
    for (int j = 0; j < MTV; ++j) r[j] = p[j * 64];
  };
  if (mine > 0) {
    look_up(0);
    load(kreg, a.k_pool, 0);
    load(vreg, a.v_pool, 0);
  }
  for (int i = 0; i < mine; ++i) {
    const float kscale = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(ksc), i & 63));
    const float vscale = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(vsc), i & 63));
    if (((i + 1) & 63) == 0) look_up(i + 1);
    const int key0 = (b0 + ks + i * KS) * 32, rest = seq.L - key0;
    f32x16 sacc;
#pragma unroll
    for (int v = 0; v < 16; ++v) sacc[v] = 0.f;
#pragma unroll
    for (int j = 0; j < MTV; ++j) {
      sacc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(operand(kreg[j][0], kreg[j][1], kscale), qreg[2 * j], sacc, 0, 0, 0);
      sacc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(operand(kreg[j][2], kreg[j][3], kscale), qreg[2 * j + 1], sacc, 0, 0, 0);
    }
    if (i + 1 < mine) load(kreg, a.k_pool, i + 1);
    float sc[16];
    const float f = kscale == kscale ? a.scale_log2e : NAN;  // a page that is not there
#pragma unroll
    for (int v = 0; v < 16; ++v) sc[v] = sacc[v] * f;
    if (rest < 32) {
#pragma unroll
      for (int v = 0; v < 16; ++v)
        if (8 * (v >> 2) + 4 * hh + (v & 3) >= rest) sc[v] = -INFINITY;
      // slots past the end may hold anything: their weights are 0, their values have to be numbers
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        const int keep = min(max(rest - 8 * d - 4 * hh, 0), 4);
        const uint32_t mask = keep == 4 ? 0xffffffffu : (1u << (8 * keep)) - 1u;
#pragma unroll
        for (int mt = 0; mt < MTV; ++mt) vreg[mt][d] &= mask;
      }
    }
    u32x4 pk[2];
    q8_rescale<MTV>(o, sm.take(sc, pk));
#pragma unroll
    for (int mt = 0; mt < MTV; ++mt) {
      o[mt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(operand(vreg[mt][0], vreg[mt][1], vscale), __builtin_bit_cast(bf16x8, pk[0]), o[mt], 0, 0, 0);
      o[mt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(operand(vreg[mt][2], vreg[mt][3], vscale), __builtin_bit_cast(bf16x8, pk[1]), o[mt], 0, 0, 0);
    }
    if (i + 1 < mine) load(vreg, a.v_pool, i + 1);
  }

  // ---- the tree's own rows
  int tb = max(b0, seq.cached);
  tb += (ks - (tb - b0) % KS + KS) % KS;  // this stream's first
  if (live && tb < b1) {
    const TreeBits bits = tree_bits(par, n);
    uint32_t anc[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t w = (uint32_t)from_node(bits.w[k], node);
      anc[k] = qi < nq ? w : 0u;
    }
    for (; tb < b1; tb += KS) {
      const int key0 = (tb - seq.cached) * 32;  // node
      const uint32_t sees = key0 == 0 ? anc[0] : key0 == 32 ? anc[1] : key0 == 64 ? anc[2] : anc[3];
      const size_t at = (size_t)head * DH;
      f32x16 sacc;
#pragma unroll
      for (int v = 0; v < 16; ++v) sacc[v] = 0.f;
      {
        const uint16_t* kp = a.k_rows + (size_t)(seq.r0 + min(key0 + n32, n - 1)) * a.row_stride + at + hh * 16;
#pragma unroll
        for (int j = 0; j < MTV; ++j) {
          sacc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8*>(kp + 32 * j), qreg[2 * j], sacc, 0, 0, 0);
          sacc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8*>(kp + 32 * j + 8), qreg[2 * j + 1], sacc, 0, 0, 0);
        }
      }
      float sc[16];
#pragma unroll
      for (int v = 0; v < 16; ++v)
        sc[v] = (sees >> (8 * (v >> 2) + 4 * hh + (v & 3))) & 1 ? sacc[v] * a.scale_log2e : -INFINITY;
      u32x4 pk[2];
      q8_rescale<MTV>(o, sm.take(sc, pk));
      auto value = [&](int key, int c) -> uint16_t {
        return key0 + key < n ? a.v_rows[(size_t)(seq.r0 + key0 + key) * a.row_stride + at + c] : (uint16_t)0;
      };
      bool odd = false;
#pragma unroll
      for (int mt = 0; mt < MTV; ++mt)
#pragma unroll
        for (int kg = 0; kg < 2; ++kg) {
          u32x4 v;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int key = 16 * kg + 8 * (e >> 1) + 4 * hh + 2 * (e & 1);
            uint32_t lo = value(key, 32 * mt + n32), hi = value(key + 1, 32 * mt + n32);
            if ((lo & 0x7f80u) == 0x7f80u) odd = true, lo = 0;
            if ((hi & 0x7f80u) == 0x7f80u) odd = true, hi = 0;
            v[e] = lo | hi << 16;
          }
          o[mt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v), __builtin_bit_cast(bf16x8, pk[kg]), o[mt], 0, 0, 0);
        }
      if (__ballot(odd))
        q8_add_odd_values<MTV>(o, pk, min(32, n - key0), [&](int key) { return ((sees >> key) & 1) != 0; }, value);
    }
  }

  // ---- merge the key streams of every query tile in a fixed order: stream mt % KS owns part mt
  const float lt = sm.l + __shfl_xor(sm.l, 32);
  if (hh == 0) {
    sm_m[wv][n32] = sm.m;
    sm_l[wv][n32] = lt;
  }
  __syncthreads();
  float* red = reinterpret_cast<float*>(smem);
  float mg = -INFINITY;
#pragma unroll
  for (int k = 0; k < KS; ++k) mg = fmaxf(mg, sm_m[nt + NTW * k][n32]);
  const float ref = mg == -INFINITY ? 0.f : mg;
  float lg = 0.f;
#pragma unroll
  for (int k = 0; k < KS; ++k) lg += sm_l[nt + NTW * k][n32] * __builtin_amdgcn_exp2f(sm_m[nt + NTW * k][n32] - ref);
  const float mine_f = __builtin_amdgcn_exp2f(sm.m - ref);
#pragma unroll
  for (int mt = 0; mt < MTV; ++mt)
#pragma unroll
    for (int v = 0; v < 16; ++v) o[mt][v] *= mine_f;
  constexpr int PART = 16 * 64;
#pragma unroll
  for (int mt = 0; mt < MTV; ++mt) {
    const int owner = mt % KS;
    if (ks != owner) {
      float* dst = red + (((nt * MTV + mt) * (KS - 1)) + (ks < owner ? ks : ks - 1)) * PART + lane;
#pragma unroll
      for (int v = 0; v < 16; ++v) dst[v * 64] = o[mt][v];
    }
  }
  __syncthreads();
  if (!live) return true;
  size_t part = 0;
  if (splits > 1) {  // place among the partials: those of the split sequences before, then this one's in item order
    int before = 0;
    for (int s0 = 0; s0 < s; s0 += 64) {
      int c = 0;
      if (s0 + lane < s) {
        const Q8Seq q = q8_seq(a, s0 + lane);
        const int k = q8_splits(plan, q);
        c = k > 1 ? q8_groups<NTW>(a, q) * a.n_kv_heads * k : 0;
      }
      before += __shfl(wave_scan(c), 63);
    }
    part = (size_t)(before + nth) * NTW + nt;
    if (before + nth >= a.max_parts) return true;  // more work than T rows can be: ranges that overlap
    if (ks == 0 && hh == 0) {
      a.pm[part * 32 + n32] = mg;
      a.pl[part * 32 + n32] = lg;
    }
  }
  const float inv = 1.0f / lg;
#pragma unroll
  for (int mt = 0; mt < MTV; ++mt) {
    if (ks != mt % KS) continue;
    const float* src = red + ((nt * MTV + mt) * (KS - 1)) * PART + lane;
#pragma unroll
    for (int k = 0; k < KS - 1; ++k)
#pragma unroll
      for (int v = 0; v < 16; ++v) o[mt][v] += src[(k * 16 + v) * 64];
    if (splits == 1) {
      if (qi < nq) {
        uint16_t* dst = a.out + (size_t)(seq.r0 + node) * row_len + (size_t)qhead * DH + 32 * mt + 4 * hh;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const u32x2 v = {pack2bf(o[mt][4 * g] * inv, o[mt][4 * g + 1] * inv), pack2bf(o[mt][4 * g + 2] * inv, o[mt][4 * g + 3] * inv)};
          *reinterpret_cast<u32x2*>(dst + 8 * g) = v;
        }
      }
    } else {
      float* img = a.po + part * OW + mt * PART + lane;
#pragma unroll
      for (int v = 0; v < 16; ++v) img[v * 64] = o[mt][v];
    }
  }
  return true;
  };
  for (int x = blockIdx.x; item(x); x += gridDim.x) __syncthreads();  // LDS is free again
}

// Merges the partials of a (sequence, query tile, K/V head) in split order, one 32-column part of the
// rows per workgroup: thread (lane, g) owns the accumulator registers 4g .. 4g+3 that lane held.
template <int DH, int NTW>
__global__ __launch_bounds__(256) void attn_q8_combine_kernel(Q8Args a) {
  constexpr int MTV = DH / 32, PART = 16 * 64;
  const int tid = threadIdx.x, lane = tid & 63, n32 = lane & 31, hh = lane >> 5, g = tid >> 6;
  const Q8Plan plan = q8_plan<NTW>(a);
  auto count = [&](int x) {
    const Q8Seq q = q8_seq(a, x);
    const int k = q8_splits(plan, q);
    return k > 1 ? q8_groups<NTW>(a, q) * a.n_kv_heads * k : 0;
  };
  for (int x = blockIdx.x / MTV;; x += gridDim.x / MTV) {  // tiles, in the order of the partials
    const int mt = blockIdx.x % MTV;
    int s, nth, base = 0;
    if (!find_seq(x, a.B, [&](int y) {
          const Q8Seq q = q8_seq(a, y);
          return q8_splits(plan, q) > 1 ? q8_groups<NTW>(a, q) * a.n_kv_heads * NTW : 0;
        }, s, nth)) return;
    for (int s0 = 0; s0 < s; s0 += 64) base += __shfl(wave_scan(s0 + lane < s ? count(s0 + lane) : 0), 63);
    const Q8Seq seq = q8_seq(a, s);
    const int splits = q8_splits(plan, seq);
    const int nt = nth % NTW, head = nth / NTW % a.n_kv_heads, qg = nth / NTW / a.n_kv_heads;
    const int nq = seq.nodes * a.group, qi = (qg * NTW + nt) * 32 + n32;
    if ((qg * NTW + nt) * 32 >= nq) continue;
    if (!tree_valid(load_parents(a.parent, seq.r0, seq.nodes), seq.nodes)) continue;  // zeros are there already
    if (base + (qg + 1) * splits * a.n_kv_heads > a.max_parts) continue;  // see there
    auto at = [&](int sp) { return (size_t)(base + (qg * splits + sp) * a.n_kv_heads + head) * NTW + nt; };
    float m = -INFINITY;
    for (int sp = 0; sp < splits; ++sp) m = fmaxf(m, a.pm[at(sp) * 32 + n32]);
    const float ref = m == -INFINITY ? 0.f : m;
    float l = 0.f;
    f32x4 o = {0, 0, 0, 0};
    for (int sp = 0; sp < splits; ++sp) {
      const size_t p = at(sp);
      const float w = __builtin_amdgcn_exp2f(a.pm[p * 32 + n32] - ref);
      l += w * a.pl[p * 32 + n32];
      const float* img = a.po + p * MTV * PART + mt * PART + 4 * g * 64 + lane;
#pragma unroll
      for (int v = 0; v < 4; ++v) o[v] += w * img[v * 64];
    }
    const float inv = 1.0f / l;
    if (qi < nq) {
      const int node = qi / a.group, qhead = head * a.group + qi % a.group;
      uint16_t* dst = a.out + ((size_t)(seq.r0 + node) * a.n_kv_heads * a.group + qhead) * DH + 32 * mt + 4 * hh + 8 * g;
      const u32x2 v = {pack2bf(o[0] * inv, o[1] * inv), pack2bf(o[2] * inv, o[3] * inv)};
      *reinterpret_cast<u32x2*>(dst) = v;
    }
  }
}

// ------------------------------------------------------------------ launch
struct Q8Launch {
  int ntw, target, min_blocks, max_parts, grid, tiles;
};
static Q8Launch q8_launch(int B, int T, int group, int n_kv_heads, int max_prefix) {
  Q8Launch p;
  const int queries = (T + B - 1) / B * group;  // of a sequence, if all are alike
  p.ntw = queries > 32 ? 2 : 1;
  p.target = p.ntw == 1 ? 512 : 256;
  p.min_blocks = 16;
  const long items = ((long)T * group / (32 * p.ntw) + B) * n_kv_heads;  // unsplit
  const long most = ((long)max_prefix + 31) / 32 + TRJ_N_MAX / 32;       // blocks of a sequence
  // splits: a split sequence has more than `chunk` blocks, so at most twice as many splits as whole chunks
  const long parts = most <= p.min_blocks ? 0 : std::min(2l * p.target, items * ((most + p.min_blocks - 1) / p.min_blocks));
  p.max_parts = (int)parts;
  p.grid = (int)std::min(items + (parts ? p.target : 0), 1l << 20);
  p.tiles = (int)std::min(parts * p.ntw, 256l);
  return p;
}
size_t attn_q8_ws_floats(int B, int T, int group, int n_kv_heads, int head_dim, int max_prefix) {
  const Q8Launch p = q8_launch(B, T, group, n_kv_heads, max_prefix);
  return (size_t)p.max_parts * p.ntw * (32 * head_dim + 64);
}

template <int DH, int NTW>
static int q8_run(const Q8Args& a, const Q8Launch& p, hipStream_t st) {
  constexpr int KS = 4;
  constexpr size_t lds = (size_t)NTW * (DH / 32) * (KS - 1) * 16 * 64 * 4;
  static DeviceOnce once;
  allow_lds(once, tree_attn_q8_kernel<DH, NTW, KS>, lds);
  {
    ProfScope ps_(KC_ATTN, st);
    tree_attn_q8_kernel<DH, NTW, KS><<<p.grid, KS * NTW * 64, lds, st>>>(a);
  }
  int rc = check_launch();
  if (rc != TRJ_OK || p.max_parts == 0) return rc;
  ProfScope ps_(KC_ATTN_COMBINE, st);
  attn_q8_combine_kernel<DH, NTW><<<p.tiles * (DH / 32), 256, 0, st>>>(a);
  return check_launch();
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
                 p.target, p.min_blocks, p.max_parts, scale * 1.4426950408889634f, ws, pm, pm + tiles * 32, out, status};
  if (head_dim == 128) return p.ntw == 1 ? q8_run<128, 1>(a, p, st) : q8_run<128, 2>(a, p, st);
  return p.ntw == 1 ? q8_run<64, 1>(a, p, st) : q8_run<64, 2>(a, p, st);
}

}  // namespace trj
