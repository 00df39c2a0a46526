// A token per row of logits under temperature, top-k, top-p and min-p, from a given random number.
//
//   w_v = round(2^38 exp((x_v - max x) / t)), tokens in the order of falling x, of equal ones rising index
//   top-k, top-p and min-p each keep a first part of that order; target = floor(u * sum of the kept w);
//   the token is the first one with which the running sum exceeds target
//
// Weights are whole numbers, so that sums do not depend on their order and every comparison with a border is exact.
// As all three rules keep first parts, only the sum of what each keeps matters: of the smallest the target is a share.  No
// row is sorted: a histogram over max x - x finds the bin in which a count or a running sum crosses a border, and the
// tokens of that bin alone are put in order.
#include <algorithm>

#include "kernels.h"
#include "q8.h"

namespace trj {

constexpr int SMP_THREADS = 1024, SMP_BINS = 2048, SMP_LIST = 2048;
constexpr double SMP_UNIT = 274877906944.0;      // 2^38
constexpr float SMP_RANGE = 27.1f;               // exp(-27.1) * 2^38 rounds to 0
typedef float f32x4_row __attribute__((ext_vector_type(4), aligned(4)));  // rows of odd length start anywhere

struct SampleArgs {
  const float* x;
  const int32_t* node_off;
  int B, T, V;
  const float *rules, *uniform;
  int32_t* token;
  float* prob;
  int32_t* status;
};

__device__ inline bool is_token(float x) { return x > -INFINITY; }  // neither -infinity nor NaN
// Place in the order, larger first: the logit's bits, ascending, then the index from behind.  Never 0 for a token.
__device__ inline uint64_t place_key(float x, int i) {
  const uint32_t u = __float_as_uint(x + 0.f);  // the zeros are equal
  return (uint64_t)(u >> 31 ? ~u : u | 0x80000000u) << 24 | (uint32_t)(0xffffff - i);
}
__device__ inline float key_logit(uint64_t k) {
  const uint32_t u = (uint32_t)(k >> 24);
  return __uint_as_float(u >> 31 ? u & 0x7fffffffu : ~u);
}
__device__ inline int key_index(uint64_t k) { return 0xffffff - (int)(k & 0xffffff); }

struct SampleRow {
  float top, per_bin;  // largest logit; bins per logit
  double inv;          // 1 / temperature
  __device__ inline SampleRow(float m, float t) : top(m), per_bin(SMP_BINS / (SMP_RANGE * t)), inv(1.0 / (double)t) {}
  __device__ inline uint64_t weight(float x) const {
    if (x == top) return (uint64_t)SMP_UNIT;
    const double y = ((double)x - (double)top) * inv;
    return y > -(double)SMP_RANGE ? (uint64_t)rint(exp(y) * SMP_UNIT) : 0;
  }
  __device__ inline int bin(float x) const { return x == top ? 0 : (int)fminf((top - x) * per_bin, (float)(SMP_BINS - 1)); }
};

// sums over the workgroup
__device__ inline uint64_t lane_up64(uint64_t v, int d) {
  return (uint64_t)(uint32_t)__shfl_up((int)(v >> 32), d) << 32 | (uint32_t)__shfl_up((int)v, d);
}
__device__ inline uint64_t wave_scan64(uint64_t v) {  // inclusive
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint64_t u = lane_up64(v, d);
    if (lane >= d) v += u;
  }
  return v;
}
template <class F>
__device__ inline uint64_t wave_all64(uint64_t v, F join) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v = join(v, (uint64_t)(uint32_t)__shfl_xor((int)(v >> 32), d) << 32 | (uint32_t)__shfl_xor((int)v, d));
  return v;
}
template <class F>
__device__ inline uint64_t block_all64(uint64_t v, uint64_t (&part)[SMP_THREADS / 64], F join) {
  v = wave_all64(v, join);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  v = part[0];
#pragma unroll
  for (int w = 1; w < SMP_THREADS / 64; ++w) v = join(v, part[w]);
  return v;
}

// Tokens per bin and the sum of their weights; after scan() those of all bins before, [SMP_BINS]: all.
struct Histogram {
  uint64_t w[SMP_BINS + 1];
  uint32_t n[SMP_BINS + 1];
  __device__ inline void clear() {
    for (int i = threadIdx.x; i <= SMP_BINS; i += SMP_THREADS) w[i] = 0, n[i] = 0;
  }
  __device__ inline void add(int b, uint64_t weight) {
    atomicAdd((unsigned long long*)&w[b], (unsigned long long)weight);
    atomicAdd(&n[b], 1u);
  }
  __device__ inline void scan(uint64_t (&part_w)[SMP_THREADS / 64], uint64_t (&part_n)[SMP_THREADS / 64]) {
    constexpr int PER = SMP_BINS / SMP_THREADS;
    const int tid = threadIdx.x, wave = tid >> 6;
    __syncthreads();
    uint64_t mw = 0, mn = 0, cw[PER], cn[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      cw[i] = w[tid * PER + i], cn[i] = n[tid * PER + i];
      mw += cw[i], mn += cn[i];
    }
    uint64_t sw = wave_scan64(mw), sn = wave_scan64(mn);
    if ((tid & 63) == 63) part_w[wave] = sw, part_n[wave] = sn;
    __syncthreads();
    for (int k = 0; k < wave; ++k) sw += part_w[k], sn += part_n[k];
    if (tid == SMP_THREADS - 1) w[SMP_BINS] = sw, n[SMP_BINS] = (uint32_t)sn;
    sw -= mw, sn -= mn;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      w[tid * PER + i] = sw, n[tid * PER + i] = (uint32_t)sn;
      sw += cw[i], sn += cn[i];
    }
    __syncthreads();
  }
  // the bin with which the running count (or sum) exceeds `target`
  __device__ inline int crossing(bool by_count, uint64_t target) const {
    int lo = 0, hi = SMP_BINS;  // before(lo) <= target < before(hi)
    while (hi - lo > 1) {
      const int m = (lo + hi) >> 1;
      if ((by_count ? (uint64_t)n[m] : w[m]) <= target) lo = m;
      else hi = m;
    }
    return lo;
  }
};

__global__ __launch_bounds__(SMP_THREADS) void sample_kernel(SampleArgs a) {
  __shared__ Histogram first;
  __shared__ union {  // never both at once
    Histogram hist;
    struct { uint64_t key[SMP_LIST], w[SMP_LIST]; } list;
  } second;
  Histogram& zoom = second.hist;
  uint64_t *const list_key = second.list.key, *const list_w = second.list.w;
  __shared__ uint64_t part_w[SMP_THREADS / 64], part_n[SMP_THREADS / 64];
  __shared__ uint64_t found_key, found_w, found_upto;
  __shared__ int list_n;
  const int tid = threadIdx.x, lane = tid & 63, t = blockIdx.x;
  if (t == 0)  // sequences without rows of their own
    for (int s = tid; s < a.B; s += SMP_THREADS) {
      const int r0 = a.node_off[s], r1 = a.node_off[s + 1];
      const bool bad = r0 < 0 || r1 < r0 || r1 > a.T;
      if (bad || r0 == r1) a.status[s] = bad;
    }
  int s = -1, r0 = 0;
  for (int s0 = 0; s0 < a.B && s < 0; s0 += 64) {
    const int q = min(s0 + lane, a.B - 1), b = a.node_off[q], e = a.node_off[q + 1];
    const uint64_t here = __ballot(s0 + lane < a.B && b >= 0 && b <= t && t < e && e <= a.T);
    if (here) {
      const int l = __builtin_ctzll(here);
      s = s0 + l;
      r0 = __builtin_amdgcn_readlane(b, l);
    }
  }
  if (s < 0) return;
  const float temperature = a.rules[4 * s], top_k = a.rules[4 * s + 1], top_p = a.rules[4 * s + 2], min_p = a.rules[4 * s + 3];
  const bool bad = !(temperature >= 0.f && temperature < INFINITY) || top_k != top_k || top_p != top_p || min_p != min_p;
  if (t == r0 && tid == 0) a.status[s] = bad;
  if (bad) return;

  const float* const x = a.x + (size_t)t * a.V;
  auto each = [&](auto f) {
    for (int i = tid * 4; i < a.V; i += SMP_THREADS * 4) {
      if (i + 4 <= a.V) {
        const f32x4_row v = *reinterpret_cast<const f32x4_row*>(x + i);
#pragma unroll
        for (int e = 0; e < 4; ++e) f(v[e], i + e);
      } else {
        for (int e = i; e < a.V; ++e) f(x[e], e);
      }
    }
  };
  auto larger = [](uint64_t p, uint64_t q) { return p > q ? p : q; };
  auto smaller = [](uint64_t p, uint64_t q) { return p < q ? p : q; };
  auto plus = [](uint64_t p, uint64_t q) { return p + q; };

  uint64_t best = 0;
  each([&](float v, int i) {
    if (is_token(v)) best = larger(best, place_key(v, i));
  });
  best = block_all64(best, part_w, larger);
  if (best == 0 || temperature == 0.f) {
    if (tid == 0) {
      a.token[t] = best == 0 ? -1 : key_index(best);
      if (a.prob) a.prob[t] = best == 0 ? 0.f : 1.f;
    }
    return;
  }
  const SampleRow row(key_logit(best), temperature);
  const uint64_t least = min_p > 0.f ? (uint64_t)ceil((double)fminf(min_p, 1.f) * SMP_UNIT) : 0;
  first.clear();
  __syncthreads();
  uint64_t over = 0;  // weights of `least` or more
  each([&](float v, int i) {
    if (!is_token(v)) return;
    const uint64_t w = row.weight(v);
    if (w == 0) return;
    first.add(row.bin(v), w);
    if (w >= least) over += w;
  });
  first.scan(part_w, part_n);
  over = block_all64(over, part_n, plus);

  uint64_t kept = first.w[SMP_BINS];
#pragma unroll 1
  for (int step = 0; step < 3; ++step) {  // top-k, top-p, the token
    bool by_count = false;
    uint64_t target;  // the first token with which the running count or sum exceeds it is wanted
    if (step == 0) {
      if (!(top_k >= 1.f) || top_k >= (float)first.n[SMP_BINS]) continue;
      by_count = true;
      target = (uint64_t)top_k - 1;
    } else if (step == 1) {
      if (!(top_p < 1.f)) continue;
      const double need = ceil((double)top_p * (double)kept);
      target = need > 1.0 ? (uint64_t)need - 1 : 0;
    } else {
      kept = smaller(kept, over);
      const double u = fmin(fmax((double)a.uniform[t], 0.0), 1.0 - 1.0 / (1 << 24));
      target = smaller((uint64_t)floor(u * (double)kept), kept - 1);
    }
    const int b = first.crossing(by_count, target);
    uint64_t before_w = first.w[b], lo = 0, hi = ~0ull;
    uint32_t before_n = first.n[b], n = first.n[b + 1] - before_n;
    if (n > SMP_LIST) {  // many alike: closer, over the whole order
      uint64_t kmin = ~0ull, kmax = 0;
      each([&](float v, int i) {
        if (is_token(v) && row.bin(v) == b && row.weight(v) > 0) kmin = smaller(kmin, place_key(v, i)), kmax = larger(kmax, place_key(v, i));
      });
      lo = block_all64(kmin, part_w, smaller);
      hi = block_all64(kmax, part_w, larger);
      while (n > SMP_LIST) {
        const int bits = 64 - __clzll((long long)(hi - lo)), shift = max(0, bits - 11);  // (hi - lo) >> shift < SMP_BINS
        zoom.clear();
        __syncthreads();
        each([&](float v, int i) {
          if (!is_token(v) || row.bin(v) != b) return;
          const uint64_t k = place_key(v, i), w = row.weight(v);
          if (k >= lo && k <= hi && w > 0) zoom.add((int)((hi - k) >> shift), w);
        });
        zoom.scan(part_w, part_n);
        const int z = zoom.crossing(by_count, target - (by_count ? before_n : before_w));
        before_w += zoom.w[z];
        before_n += zoom.n[z];
        n = zoom.n[z + 1] - zoom.n[z];
        const uint64_t top = hi - ((uint64_t)z << shift);
        const uint64_t width = (1ull << shift) - 1;
        lo = top - lo > width ? top - width : lo;
        hi = top;
        __syncthreads();
      }
    }
    if (tid == 0) list_n = 0;
    __syncthreads();
    each([&](float v, int i) {
      if (!is_token(v) || row.bin(v) != b) return;
      const uint64_t k = place_key(v, i), w = row.weight(v);
      if (w == 0 || k < lo || k > hi) return;
      const int at = atomicAdd(&list_n, 1);
      if (at < SMP_LIST) list_key[at] = k, list_w[at] = w;
    });
    __syncthreads();
    for (int e = tid; e < (int)n; e += SMP_THREADS) {
      const uint64_t k = list_key[e], w = list_w[e];
      uint64_t sum = before_w, rank = before_n;
      for (int j = 0; j < (int)n; ++j)
        if (list_key[j] > k) sum += list_w[j], ++rank;
      if (by_count ? rank == target : (sum <= target && target < sum + w)) found_key = k, found_w = w, found_upto = sum + w;
    }
    __syncthreads();
    if (step < 2) kept = found_upto;
  }
  if (tid == 0) {
    a.token[t] = key_index(found_key);
    if (a.prob) a.prob[t] = (float)((double)found_w / (double)kept);
  }
}

size_t tree_sample_ws_bytes(int, int) { return 16; }
int launch_tree_sample(const float* x, const int32_t* node_off, int B, int T, int V, const float* rules,
                       const float* uniform, int32_t* token, float* prob, void*, int32_t* status, hipStream_t st) {
  const SampleArgs a{x, node_off, B, T, V, rules, uniform, token, prob, status};
  sample_kernel<<<T, SMP_THREADS, 0, st>>>(a);
  return check_launch();
}

}  // namespace trj
