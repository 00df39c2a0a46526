// Ancestor bits of a token tree on one wavefront, from the parents alone.
#pragma once
#include "common.h"

namespace trj {

// Parents of nodes lane and lane + 64 of a tree of n nodes (anything from node n on).
struct TreeParents {
  int p[2];
};
__device__ inline TreeParents load_parents(const int32_t* parent, int r0, int n) {
  const int lane = threadIdx.x & 63;
  return TreeParents{{lane < n ? parent[r0 + lane] : -1, lane + 64 < n ? parent[r0 + lane + 64] : -1}};
}
// parent[0] = -1 and every other parent an earlier node; the same answer on all lanes
__device__ inline bool tree_valid(const TreeParents& t, int n) {
  bool bad = false;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int i = (threadIdx.x & 63) + 64 * h;
    bad = bad || (i < n && (i == 0 ? t.p[h] != -1 : (t.p[h] < 0 || t.p[h] >= i)));
  }
  return __ballot(bad) == 0;
}
// The nodes on the path root .. i, i itself included, of this lane's nodes i = lane (w[0..3]: word k
// holds nodes 32k ..) and lane + 64: pointer doubling, at most 7 rounds.
struct TreeBits {
  int w[4][2];
};
__device__ inline TreeBits tree_bits(const TreeParents& t, int n) {
  const int lane = threadIdx.x & 63;
  TreeBits b;
  int jump[2];  // nearest ancestor whose bits are not in the row yet, 255: none
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int i = lane + 64 * h;
    jump[h] = i < n && t.p[h] >= 0 ? t.p[h] & 127 : 255;
#pragma unroll
    for (int k = 0; k < 4; ++k) b.w[k][h] = i >> 5 == k ? (int)(1u << (i & 31)) : 0;
  }
  while (__ballot(jump[0] != 255 || jump[1] != 255)) {
    int u[5][2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      u[4][h] = from_node(jump, jump[h] & 127);
#pragma unroll
      for (int k = 0; k < 4; ++k) u[k][h] = from_node(b.w[k], jump[h] & 127);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (jump[h] == 255) continue;
#pragma unroll
      for (int k = 0; k < 4; ++k) b.w[k][h] |= u[k][h];
      jump[h] = u[4][h];
    }
  }
  return b;
}

}  // namespace trj
