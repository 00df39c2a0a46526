// Rotary positions of query and key rows.
//
//   (x1, x2) -> m (x1 cos a - x2 sin a, x1 sin a + x2 cos a),  a = position * f_j,  pair j of every head
//
// Angle, reduction and the two polynomials are worked out in 64 bits, once per row and pair for all heads, and
// rounded to 32 bits; products are 32-bit, each result is rounded once.
//
// Bound by memory for many rows: 4096 rows of 64 heads of 128 in bf16, 134 MB, take 29 us = 4.6 TB/s (a large copy moves 4.9).
// For few by one chain of latencies, from the lengths over the tree to the position, its angles in 64 bits and the rows: 4.0 us
// for a row, 4.3 for a tree of 69, in calls of 8.6 and 9.1.
#include <algorithm>
#include <cmath>

#include "kernels.h"
#include "q8.h"
#include "tree_anc.h"

namespace trj {

struct RotaryArgs {
  const void *q, *k;
  void *q_out, *k_out;
  const int32_t *parent, *node_off, *prefix_len;
  const double* freqs;
  int q_stride, k_stride, qo_stride, ko_stride, B, T, n_heads, n_kv_heads, head_dim, half;
  float magnitude;
  int32_t* status;
};
constexpr int ROT_THREADS = 256, ROT_MAX_HALF = 512;

// cos and sin of an angle >= 0: quarter turns off in two parts, then Taylor's polynomials on [-pi/4, pi/4], whose
// first missing terms are below 7e-12 (x^13 / 13!) and 4e-13 (x^14 / 14!) there
__device__ inline float2 cos_sin(double a, float magnitude) {
  constexpr double PIO2_HI = 1.5707963267948966, PIO2_LO = 6.123233995736766e-17;
  const double n = rint(a * (1.0 / PIO2_HI));
  const double x = fma(-n, PIO2_LO, fma(-n, PIO2_HI, a)), z = x * x;
  double s = -1.0 / 39916800;
  s = fma(s, z, 1.0 / 362880);
  s = fma(s, z, -1.0 / 5040);
  s = fma(s, z, 1.0 / 120);
  s = fma(s, z, -1.0 / 6);
  s = fma(s * z, x, x);
  double c = 1.0 / 479001600;
  c = fma(c, z, -1.0 / 3628800);
  c = fma(c, z, 1.0 / 40320);
  c = fma(c, z, -1.0 / 720);
  c = fma(c, z, 1.0 / 24);
  c = fma(c, z, -0.5);
  c = fma(c, z, 1.0);
  const int quarter = (int)((long long)n & 3);
  const double cr = quarter & 1 ? s : c, sr = quarter & 1 ? c : s;
  return float2{(float)((quarter == 1 || quarter == 2 ? -cr : cr) * magnitude), (float)((quarter >= 2 ? -sr : sr) * magnitude)};
}

struct RotaryRow {
  int s, r0, n, L;  // sequence, its first row, rows, prefix; n < 0: none, or refused
};
// The sequence of row t and its verdict but for the tree; the same on all lanes of a wavefront.
__device__ inline RotaryRow rotary_row(const RotaryArgs& a, int t) {
  const int lane = threadIdx.x & 63;
  for (int s0 = 0; s0 < a.B; s0 += 64) {
    const int s = min(s0 + lane, a.B - 1), r0 = a.node_off[s], r1 = a.node_off[s + 1], L = a.prefix_len[s];
    const bool owns = s0 + lane < a.B && r0 >= 0 && r0 <= t && t < r1 && r1 <= a.T;
    const uint64_t here = __ballot(owns);
    if (!here) continue;
    const int l = __builtin_ctzll(here);
    RotaryRow r{s0 + l, __builtin_amdgcn_readlane(r0, l), 0, __builtin_amdgcn_readlane(L, l)};
    r.n = __builtin_amdgcn_readlane(r1, l) - r.r0;
    if (r.L < 0 || r.L > INT32_MAX - (r.n - 1) || (a.parent && r.n > TRJ_N_MAX)) r.L = -1;
    return r;
  }
  return RotaryRow{-1, 0, -1, -1};
}

template <class E>
__device__ inline float to_float(E x) {
  if constexpr (sizeof(E) == 2) return bf2f(x);
  else return x;
}
template <class E>
__device__ inline E from_float(float x) {
  if constexpr (sizeof(E) == 2) return f2bf(x);
  else return x;
}
template <class E>
struct Vec16 {
  E v[16 / sizeof(E)];
};
__device__ inline float2 turned(float x1, float x2, float2 cs) {
  return float2{x1 * cs.x - x2 * cs.y, x1 * cs.y + x2 * cs.x};
}

// A workgroup per row.  Four rows per workgroup, a wavefront looking for the sequence of each, took 18.5 us instead of 16.4 for
// 4096 rows of 40 heads of 128, 66.9 instead of 62.4 for 16384, and more for fewer (of 9 heads 10 % less for 16384).
// WIDE: 16 bytes at a time, where pairs (or halves of them) come in such pieces.
template <class E, bool PAIRS, bool WIDE>
__global__ __launch_bounds__(ROT_THREADS) void rotary_kernel(RotaryArgs a) {
  constexpr int N = 16 / sizeof(E);
  __shared__ float2 cs[ROT_MAX_HALF];
  __shared__ int position;
  const int tid = threadIdx.x, t = blockIdx.x;
  if (blockIdx.x == 0)  // sequences without rows of their own
    for (int s = tid; s < a.B; s += ROT_THREADS) {
      const int r0 = a.node_off[s], r1 = a.node_off[s + 1];
      const bool bad = r0 < 0 || r1 < r0 || r1 > a.T;
      if (bad || r0 == r1) a.status[s] = bad;
    }
  if (tid < 64) {
    const RotaryRow row = rotary_row(a, t);
    int at = -1;
    if (row.n > 0) {
      if (row.L >= 0) {
        const int node = t - row.r0;
        if (a.parent) {
          const TreeParents p = load_parents(a.parent, row.r0, row.n);
          if (tree_valid(p, row.n)) {
            const TreeBits b = tree_bits(p, row.n);
            int depth[2];
#pragma unroll
            for (int h = 0; h < 2; ++h)
              depth[h] = __popc(b.w[0][h]) + __popc(b.w[1][h]) + __popc(b.w[2][h]) + __popc(b.w[3][h]) - 1;
            at = row.L + from_node(depth, node);
          }
        } else {
          at = row.L + node;
        }
      }
      if (t == row.r0 && tid == 0) a.status[row.s] = at < 0;
    }
    if (tid == 0) position = at;
  }
  __syncthreads();
  const int at = position;
  if (at < 0) return;
  for (int j = tid; j < a.half; j += ROT_THREADS) cs[j] = cos_sin((double)at * a.freqs[j], a.magnitude);
  __syncthreads();
  const int heads = a.n_heads + a.n_kv_heads, rot = 2 * a.half;
  // units of a head: what is turned, then what is copied
  const int turns = WIDE ? (PAIRS ? rot / N : a.half / N) : a.half;
  const int units = turns + (a.head_dim - rot) / (WIDE ? N : 1);
  for (int i = tid; i < heads * units; i += ROT_THREADS) {
    const int h = i / units, u = i % units;
    const bool is_q = h < a.n_heads;
    const int hk = is_q ? h : h - a.n_heads;
    const E* src = (const E*)(is_q ? a.q : a.k) + (size_t)t * (is_q ? a.q_stride : a.k_stride) + (size_t)hk * a.head_dim;
    E* dst = (E*)(is_q ? a.q_out : a.k_out) + (size_t)t * (is_q ? a.qo_stride : a.ko_stride) + (size_t)hk * a.head_dim;
    if constexpr (WIDE) {
      if (u >= turns) {
        const int c = rot + (u - turns) * N;
        *reinterpret_cast<u32x4*>(dst + c) = *reinterpret_cast<const u32x4*>(src + c);
      } else if constexpr (PAIRS) {
        Vec16<E> x = *reinterpret_cast<const Vec16<E>*>(src + u * N);
#pragma unroll
        for (int e = 0; e < N / 2; ++e) {
          const float2 y = turned(to_float(x.v[2 * e]), to_float(x.v[2 * e + 1]), cs[u * (N / 2) + e]);
          x.v[2 * e] = from_float<E>(y.x), x.v[2 * e + 1] = from_float<E>(y.y);
        }
        *reinterpret_cast<Vec16<E>*>(dst + u * N) = x;
      } else {
        Vec16<E> x1 = *reinterpret_cast<const Vec16<E>*>(src + u * N), x2 = *reinterpret_cast<const Vec16<E>*>(src + a.half + u * N);
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const float2 y = turned(to_float(x1.v[e]), to_float(x2.v[e]), cs[u * N + e]);
          x1.v[e] = from_float<E>(y.x), x2.v[e] = from_float<E>(y.y);
        }
        *reinterpret_cast<Vec16<E>*>(dst + u * N) = x1;
        *reinterpret_cast<Vec16<E>*>(dst + a.half + u * N) = x2;
      }
    } else {
      if (u >= turns) {
        const int c = rot + u - turns;
        dst[c] = src[c];
      } else {
        const int c1 = PAIRS ? 2 * u : u, c2 = PAIRS ? 2 * u + 1 : u + a.half;
        const float2 y = turned(to_float(src[c1]), to_float(src[c2]), cs[u]);
        dst[c1] = from_float<E>(y.x), dst[c2] = from_float<E>(y.y);
      }
    }
  }
}

template <class E, bool PAIRS, bool WIDE>
static int rotary_run(const RotaryArgs& a, hipStream_t st) {
  rotary_kernel<E, PAIRS, WIDE><<<a.T, ROT_THREADS, 0, st>>>(a);
  return check_launch();
}
template <class E>
static int rotary_layout(const RotaryArgs& a, int layout, hipStream_t st) {
  constexpr int N = 16 / sizeof(E);
  if (layout == TRJ_ROTARY_PAIRS)
    return 2 * a.half % N == 0 ? rotary_run<E, true, true>(a, st) : rotary_run<E, true, false>(a, st);
  return a.half % N == 0 ? rotary_run<E, false, true>(a, st) : rotary_run<E, false, false>(a, st);
}

int launch_rotary_rows(const void* q, int q_stride, const void* k, int k_stride, const int32_t* parent,
                       const int32_t* node_off, const int32_t* prefix_len, int B, int T, int n_heads, int n_kv_heads,
                       int head_dim, int rot_dim, int layout, const double* freqs, float magnitude, int dtype, void* q_out,
                       int q_out_stride, void* k_out, int k_out_stride, int32_t* status, hipStream_t st) {
  const RotaryArgs a{q, k, q_out, k_out, parent, node_off, prefix_len, freqs, q_stride, k_stride, q_out_stride, k_out_stride,
                     B, T, n_heads, n_kv_heads, head_dim, rot_dim / 2, magnitude, status};
  return dtype == TRJ_BF16 ? rotary_layout<uint16_t>(a, layout, st) : rotary_layout<float>(a, layout, st);
}

}  // namespace trj
