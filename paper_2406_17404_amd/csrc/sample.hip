// A token per row of logits under temperature, top-k, top-p and min-p, from a given random number.
//
//   w_v = round(2^38 exp((x_v - max x) / t)), tokens in the order of falling x, of equal ones rising index
//   top-k, top-p and min-p each keep a first part of that order; target = floor(u * sum of the kept w);
//   the token is the first one with which the running sum exceeds target
//
// Weights are whole numbers, so that sums do not depend on their order and every comparison with a border is exact.
// As all three rules keep first parts, only the sum of what each keeps matters: of the smallest the target is a share.  No
// row is sorted.  Two ways:
//   the short list  where top-k (or min-p without top-p) leaves few tokens: of the threads' largest logits the k-th is
//                   a bound that k tokens reach and few more (of more than half the threads' number the k-th of all, by
//                   counting); those are collected, put in order and weighed
//   the histogram   of the weights over max x - x, which finds the bin in which a running sum (or count) crosses a
//                   border; the tokens of that bin alone are put in order
// A top-k of more than SMP_SHORT, and rows with thousands of tokens in a bin that a border crosses, take a third way, which
// reads the row from memory for every step: 61 us for one row of 32000 and top-k 2000, 190 for 1024 rows.
//
// Rows of up to 32768 logits come to the registers of one workgroup.  Short lists and greedy rows are made from there, with one
// read: 1024 x 32000 take 34 us with top-k 50 (131 MB, 3.9 TB/s; a large copy moves 4.9).  The histogram reads the row twice more, for
// the weights and for the tokens of the bins that count: 75 us without any rule, where 33 million weights are worked out in 64 bits and
// added up in LDS, 58 to 69 under mixed rules with half of the logits masked.  One row takes 10 to 13 us with a short list and 20
// without: a chain of barriers.
// Longer rows are cut, for few rows to fill the chip: 69 x 128256 take 24 to 29 us, 13.7 for the chunks (2.6 TB/s), 3.8 for a launch
// that finds nothing to weigh and 10.1 for the lists of seven chunks put together; 59 without rules.
#include <algorithm>

#include "kernels.h"
#include "q8.h"

namespace trj {

constexpr int SMP_ABREAST = 2;
constexpr int SMP_THREADS = 512, SMP_WAVES = SMP_THREADS / 64, SMP_BINS = 2048, SMP_LIST = 2048, SMP_SHORT = SMP_LIST * 3 / 4;
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
__device__ inline uint32_t place_bits(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);  // the zeros are equal
  return u >> 31 ? ~u : u | 0x80000000u;
}
__device__ inline float bits_logit(uint32_t u) { return __uint_as_float(u >> 31 ? u & 0x7fffffffu : ~u); }
__device__ inline uint64_t place_key(float x, int i) { return (uint64_t)place_bits(x) << 24 | (uint32_t)(0xffffff - i); }
__device__ inline float key_logit(uint64_t k) { return bits_logit((uint32_t)(k >> 24)); }
__device__ inline int key_index(uint64_t k) { return 0xffffff - (int)(k & 0xffffff); }

struct SampleRules {
  float t, top_k, top_p;
  uint64_t least;  // of a weight, by min-p
  bool bad;
  __device__ inline SampleRules(const float* r) : t(r[0]), top_k(r[1]), top_p(r[2]) {
    const float m = r[3];
    bad = !(t >= 0.f && t < INFINITY) || top_k != top_k || top_p != top_p || m != m;
    least = m > 0.f ? (uint64_t)ceil((double)fminf(m, 1.f) * SMP_UNIT) : 0;
  }
  __device__ inline bool short_by_k() const { return top_k >= 1.f && top_k <= SMP_SHORT; }
  __device__ inline bool short_by_min() const { return least > 0 && !(top_p < 1.f) && !(top_k >= 1.f); }
};

// What a row's weights and bins are worked out from.  Weights: 2^y, y <= 0, is Taylor's polynomial of e^(f ln 2) on
// |f| <= 1/2 times a power of two; the first missing term is below 6.3e-15, 2^-9 of a unit.  (A table of 2^(j / 128) with
// a polynomial of five terms took as long.)  Without branches: what lies far below (-infinity, NaN) is taken for 2^-40, a quarter of a unit, and rounds to 0.  Whole numbers come from adding 1.5 * 2^52, which
// leaves them in a sum's low bits: rounding and conversion are instructions at a fraction of the rate.
struct LogitRange {
  float lo, hi;
  __device__ inline int has(float x) const { return (int)(x >= lo) & (int)(x <= hi); }
};
struct SampleScale {
  float half_top, per_bin;  // half the largest logit; bins per half a logit
  double top, inv;          // log2(e) / temperature
  bool infinite;            // then the infinities count as 0 and all others as -infinity
  __device__ inline SampleScale(float m, float t)
      : half_top(m == INFINITY ? 0.f : 0.5f * m), per_bin(fminf((2 * SMP_BINS / SMP_RANGE) / t, 1e30f)),
        top(m == INFINITY ? 0.0 : (double)m), inv(1.4426950408889634 / (double)t), infinite(m == INFINITY) {}
  __device__ inline float seen(float x) const { return !infinite ? x : x == INFINITY ? 0.f : -INFINITY; }
  __device__ inline uint64_t weight(float x) const {
    constexpr double L = 0.6931471805599453, WHOLE = 6755399441055744.0;
    constexpr double L2 = L * L, L4 = L2 * L2, L6 = L4 * L2, L8 = L4 * L4, L10 = L8 * L2;
    const double y = fmax(((double)x - top) * inv, -40.0), n = y + WHOLE, f = y - (n - WHOLE);
    const int k = (int)__double_as_longlong(n);
    double p = fma(L10 * L / 39916800, f, L10 / 3628800);
    p = fma(p, f, L8 * L / 362880);
    p = fma(p, f, L8 / 40320);
    p = fma(p, f, L6 * L / 5040);
    p = fma(p, f, L6 / 720);
    p = fma(p, f, L4 * L / 120);
    p = fma(p, f, L4 / 24);
    p = fma(p, f, L2 * L / 6);
    p = fma(p, f, L2 / 2);
    p = fma(p, f, L);
    p = fma(p, f, 1.0);
    const uint64_t r = (uint64_t)__double_as_longlong(p);
    // times 2^(k + 38), in the exponent
    const uint64_t scaled = (uint64_t)((uint32_t)(r >> 32) + ((uint32_t)(k + 38) << 20)) << 32 | (uint32_t)r;
    const double whole = __longlong_as_double((long long)scaled) + WHOLE;
    return (uint64_t)__double_as_longlong(whole) & 0x7ffffffffffffull;
  }
  // logits that bins b0 .. b1 can hold (a token's bin is off by less than 2^-20 of its place)
  __device__ inline LogitRange range(int b0, int b1, float t) const {
    if (infinite) return LogitRange{INFINITY, INFINITY};
    if (t > 1e30f) return LogitRange{-INFINITY, INFINITY};
    const float off = fabsf(half_top) * 1e-6f + 1e-37f;  // (half a subnormal number is rounded)
    return LogitRange{2.f * (half_top - (float)(b1 + 1) / per_bin * 1.00001f - off), 2.f * (half_top - (float)b0 / per_bin * 0.99999f + off)};
  }
  // Falling with x.  The last bin's tokens weigh nothing: exp(-27.1 * 2047 / 2048) * 2^38 = 0.47.
  __device__ inline int bin(float x) const { return (int)fminf(fmaf(-0.5f, x, half_top) * per_bin, (float)(SMP_BINS - 1)); }
};

// ---- sums over the workgroup
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
struct Parts {
  uint64_t w[SMP_WAVES];
  uint32_t least[SMP_WAVES], most[SMP_WAVES];
  float f[SMP_WAVES];
};
template <class F>
__device__ inline uint64_t block_all64(uint64_t v, Parts& part, F join) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v = join(v, (uint64_t)(uint32_t)__shfl_xor((int)(v >> 32), d) << 32 | (uint32_t)__shfl_xor((int)v, d));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) part.w[threadIdx.x >> 6] = v;
  __syncthreads();
  v = part.w[0];
#pragma unroll
  for (int w = 1; w < SMP_WAVES; ++w) v = join(v, part.w[w]);
  return v;
}
__device__ inline float block_max(float v, Parts& part) {  // of numbers
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) part.f[threadIdx.x >> 6] = v;
  __syncthreads();
  v = part.f[0];
#pragma unroll
  for (int w = 1; w < SMP_WAVES; ++w) v = fmaxf(v, part.f[w]);
  return v;
}
// exclusive sum over the threads, and the whole
__device__ inline uint64_t block_before64(uint64_t v, uint64_t (&part)[SMP_WAVES], uint64_t& all) {
  const uint64_t upto = wave_scan64(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 63) part[threadIdx.x >> 6] = upto;
  __syncthreads();
  uint64_t before = upto - v;
  all = 0;
#pragma unroll
  for (int k = 0; k < SMP_WAVES; ++k) {
    if (k < (int)(threadIdx.x >> 6)) before += part[k];
    all += part[k];
  }
  return before;
}
struct Larger { __device__ uint64_t operator()(uint64_t p, uint64_t q) const { return p > q ? p : q; } };
struct Smaller { __device__ uint64_t operator()(uint64_t p, uint64_t q) const { return p < q ? p : q; } };
struct Plus { __device__ uint64_t operator()(uint64_t p, uint64_t q) const { return p + q; } };

// Tokens per bin and the sum of their weights; after sum_bins() those of all bins before, [SMP_BINS]: all.
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
};

struct ListLds {  // of what makes a list
  Parts part;
  uint32_t count[SMP_THREADS];
  int list_n, bound_bin;
  __device__ inline void start_list() {
    __syncthreads();
    if (threadIdx.x == 0) list_n = 0;
    __syncthreads();
  }
};
struct ChunkLds : ListLds {
  uint32_t counts[SMP_BINS + 1];
};
struct WeighLds {  // of what adds up weights
  uint64_t before[SMP_BINS + 1];
  Parts part;
};
struct SampleLds : ListLds {
  uint64_t before[SMP_BINS + 1];  // weights per bin; after sum_bins() of all bins before, [SMP_BINS]: all
  union {                         // never two at once
    struct {
      uint64_t key[SMP_LIST], sorted[SMP_LIST];
      uint32_t bin[SMP_BINS + 1];
    } few;
    Histogram zoom;
    struct { uint64_t key[SMP_LIST], w[SMP_LIST]; } list;
    uint32_t counts[SMP_BINS + 1];  // (leaves few.bin as it is)
  };
  uint64_t found_upto, found_key, found_w;
  int found_bin[2];
};
template <class T>
__device__ inline int crossing(const T (&before)[SMP_BINS + 1], uint64_t target) {  // before[lo] <= target < before[lo + 1]
  int lo = 0, hi = SMP_BINS;
  while (hi - lo > 1) {
    const int m = (lo + hi) >> 1;
    if (before[m] <= target) lo = m;
    else hi = m;
  }
  return lo;
}
// the same of l.before for two targets, by all threads at once
struct BinPair {
  int first, second;
};
__device__ inline BinPair crossings(SampleLds& l, uint64_t target0, uint64_t target1) {
  constexpr int PER = SMP_BINS / SMP_THREADS;
  __syncthreads();
  uint64_t lower = l.before[threadIdx.x * PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const uint64_t upper = l.before[threadIdx.x * PER + i + 1];
    if (lower <= target0 && target0 < upper) l.found_bin[0] = threadIdx.x * PER + i;
    if (lower <= target1 && target1 < upper) l.found_bin[1] = threadIdx.x * PER + i;
    lower = upper;
  }
  __syncthreads();
  return BinPair{l.found_bin[0], l.found_bin[1]};
}
// counts or weights per bin to those of all bins before; the sum of all
template <class T>
__device__ inline uint64_t sum_bins(T (&x)[SMP_BINS + 1], Parts& part) {
  constexpr int PER = SMP_BINS / SMP_THREADS;
  const int tid = threadIdx.x;
  __syncthreads();
  T c[PER];
  uint64_t sum = 0, all;
#pragma unroll
  for (int i = 0; i < PER; ++i) c[i] = x[tid * PER + i], sum += c[i];
  uint64_t before = block_before64(sum, part.w, all);
  if (tid == 0) x[SMP_BINS] = (T)all;
#pragma unroll
  for (int i = 0; i < PER; ++i) x[tid * PER + i] = (T)before, before += c[i];
  __syncthreads();
  return all;
}

// the first position at which the running sum has to be at least this much, by top-p, less one
__device__ inline uint64_t top_p_target(float p, uint64_t sum) {
  const double need = ceil((double)p * (double)sum);
  return need > 1.0 ? (uint64_t)need - 1 : 0;
}
__device__ inline uint64_t uniform_target(float u, uint64_t kept) {
  const double v = fmin(fmax((double)u, 0.0), 1.0 - 1.0 / (1 << 24));  // NaN: 0
  const uint64_t target = (uint64_t)floor(v * (double)kept);
  return target < kept ? target : kept - 1;
}
__device__ inline void give(const SampleArgs& a, int t, uint64_t key, uint64_t w, uint64_t kept) {
  a.token[t] = key_index(key);
  if (a.prob) a.prob[t] = (float)((double)w / (double)kept);
}

// few.key[0 .. n) in order: by bins over the keys' range, then within each bin, which is few but for tokens that are much alike
__device__ inline void order_list(SampleLds& l, int n) {
  constexpr int PER = SMP_LIST / SMP_THREADS;
  const int tid = threadIdx.x;
  auto& f = l.few;
  for (int i = tid; i <= SMP_BINS; i += SMP_THREADS) f.bin[i] = 0;
  uint64_t key[PER];
  int b[PER], at[PER];
  uint32_t lo = ~0u, hi = 0;  // of the logits' bits
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int e = tid + j * SMP_THREADS;
    key[j] = e < n ? f.key[e] : 0;
    if (e < n) lo = min(lo, (uint32_t)(key[j] >> 24)), hi = max(hi, (uint32_t)(key[j] >> 24));
  }
  lo = wave_min(lo), hi = wave_max(hi);
  if ((tid & 63) == 0) l.part.least[tid >> 6] = lo, l.part.most[tid >> 6] = hi;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < SMP_WAVES; ++w) lo = min(lo, l.part.least[w]), hi = max(hi, l.part.most[w]);
  const uint64_t most = (uint64_t)hi << 24 | 0xffffff, range = most - ((uint64_t)lo << 24);
  const int shift = max(0, 53 - __clzll((long long)range));  // range >> shift < SMP_BINS
#pragma unroll
  for (int j = 0; j < PER; ++j)
    if (tid + j * SMP_THREADS < n) b[j] = (int)((most - key[j]) >> shift), at[j] = (int)atomicAdd(&f.bin[b[j]], 1u);
  sum_bins(f.bin, l.part);
#pragma unroll
  for (int j = 0; j < PER; ++j)
    if (tid + j * SMP_THREADS < n) f.sorted[f.bin[b[j]] + at[j]] = key[j];
  __syncthreads();
#pragma unroll
  for (int j = 0; j < PER; ++j)
    if (tid + j * SMP_THREADS < n) {
      int place = (int)f.bin[b[j]];
      const int end = (int)f.bin[b[j] + 1];
      int ahead = 0;
      for (int i = place; i < end; ++i) ahead += f.sorted[i] > key[j];
      f.key[place + ahead] = key[j];
    }
  __syncthreads();
}
// The first n of the ordered list: every thread's keys, weights and running sums.
struct Weighed {
  static constexpr int PER = SMP_LIST / SMP_THREADS;
  uint64_t key[PER], w[PER], upto[PER], all;
  __device__ inline Weighed(const SampleScale& sc, SampleLds& l, int n) {
    uint64_t sum = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int e = (int)threadIdx.x * PER + i;
      key[i] = e < n ? l.few.key[e] : 0;
      w[i] = e < n ? sc.weight(sc.seen(key_logit(key[i]))) : 0;
      upto[i] = sum += w[i];
    }
    const uint64_t before = block_before64(sum, l.part.w, all);
#pragma unroll
    for (int i = 0; i < PER; ++i) upto[i] += before;
  }
  // the token with which the running sum exceeds a target is in one thread's hands
  __device__ inline bool crosses(int i, uint64_t target) const { return upto[i] - w[i] <= target && target < upto[i]; }
};

// The n tokens of few.key, unsorted, among which the first n_keep (n or fewer) are all that top-k keeps.
__device__ inline void finish_list(const SampleArgs& a, int t, float u, const SampleRules& r, const SampleScale& sc, SampleLds& l, int n, int n_keep) {
  order_list(l, n);
  const Weighed x(sc, l, n_keep);
  uint64_t kept = x.all;
  if (r.top_p < 1.f) {
    const uint64_t target = top_p_target(r.top_p, kept);
#pragma unroll
    for (int i = 0; i < Weighed::PER; ++i)
      if (x.crosses(i, target)) l.found_upto = x.upto[i];
    __syncthreads();
    kept = l.found_upto;
  }
  if (r.least > 0) {
    uint64_t over = 0;
#pragma unroll
    for (int i = 0; i < Weighed::PER; ++i) over += x.w[i] >= r.least ? x.w[i] : 0;
    over = block_all64(over, l.part, Plus());
    kept = over < kept ? over : kept;
  }
  const uint64_t target = uniform_target(u, kept);
#pragma unroll
  for (int i = 0; i < Weighed::PER; ++i)
    if (x.crosses(i, target)) give(a, t, x.key[i], x.w[i], kept);
}

// From the weights per bin (before, summed), with one `scan` over all tokens of the row (others may be among them); over:
// the sum of the weights that min-p allows.  False, with nothing given, where a count decides or the list is too short.
template <class Scan>
__device__ inline bool finish_bins(const SampleArgs& a, int t, float u, const SampleRules& r, const SampleScale& sc,
                                   SampleLds& l, uint64_t over, Scan scan) {
  if (r.top_k >= 1.f && r.top_k < (float)a.V) return false;
  // top-p crosses its border in bin bp, which leaves from `least` to `most`; the token is then in bins b0 .. b1
  uint64_t least = l.before[SMP_BINS], most = least;
  uint64_t p_target = 0;
  int bp = SMP_BINS;
  if (r.top_p < 1.f) {
    p_target = top_p_target(r.top_p, most);
    bp = crossings(l, p_target, p_target).first;
    least = l.before[bp] + 1, most = l.before[bp + 1];
  }
  const BinPair b01 = crossings(l, uniform_target(u, least < over ? least : over), uniform_target(u, most < over ? most : over));
  const int b0 = b01.first, b1 = b01.second;
  l.start_list();
  const LogitRange in_t = sc.range(b0, b1, r.t);
  auto take = [&](float v, int i) {
    const int b = sc.bin(sc.seen(v));
    if (!(b == bp || (b >= b0 && b <= b1))) return;  // (what is no token is in the last bin, in which nothing crosses)
    const int at = atomicAdd(&l.list_n, 1);
    if (at < SMP_LIST) l.few.key[at] = place_key(v, i);
  };
  auto any = [](const LogitRange& q, const float(&v)[4]) { return q.has(v[0]) | q.has(v[1]) | q.has(v[2]) | q.has(v[3]); };
  if (bp == SMP_BINS || bp <= b1) {
    scan([&](const float(&v)[4]) { return any(in_t, v) != 0; }, take);
  } else {
    const LogitRange in_p = sc.range(bp, bp, r.t);
    scan([&](const float(&v)[4]) { return (any(in_t, v) | any(in_p, v)) != 0; }, take);
  }
  __syncthreads();
  const int n = l.list_n;
  if (n > SMP_LIST) return false;
  order_list(l, n);
  const Weighed x(sc, l, n);
  // the list's running sums lack the bins before b0, and from bp on, where that is apart, those behind b1
  const uint64_t front = l.before[b0], back = bp > b1 ? l.before[min(bp, SMP_BINS)] - (l.before[b1 + 1] - front) : front;
  uint64_t kept = most;
  if (r.top_p < 1.f) {
#pragma unroll
    for (int i = 0; i < Weighed::PER; ++i)
      if (x.crosses(i, p_target - back)) l.found_upto = x.upto[i] + back;
    __syncthreads();
    kept = l.found_upto;
  }
  kept = over < kept ? over : kept;
  const uint64_t target = uniform_target(u, kept) - front;
#pragma unroll
  for (int i = 0; i < Weighed::PER; ++i)
    if (x.crosses(i, target)) give(a, t, x.key[i], x.w[i], kept);
  return true;
}

// The same for every row, with `each` over its tokens.
template <class Each>
__device__ inline void finish_histogram(const SampleArgs& a, int t, const SampleRules& r, const SampleScale& sc, SampleLds& l,
                                        uint64_t over, Each each) {
  const int tid = threadIdx.x;
  SampleLds& h = l;
  uint64_t kept = h.before[SMP_BINS];
#pragma unroll 1
  for (int step = 0; step < 3; ++step) {  // top-k, top-p, the token
    const bool by_count = step == 0;
    uint64_t target, before_n = 0;  // the first token with which the running count or sum exceeds it is wanted
    int b;
    if (step == 0) {
      if (!(r.top_k >= 1.f) || r.top_k >= (float)a.V) continue;
      target = (uint64_t)r.top_k - 1;
      for (int i = tid; i <= SMP_BINS; i += SMP_THREADS) h.counts[i] = 0;
      __syncthreads();
      each([&](float v, int) { atomicAdd(&h.counts[sc.bin(v)], 1u); });
      sum_bins(h.counts, l.part);
      if (target >= h.counts[SMP_BINS - 1]) continue;  // among those that weigh nothing, or beyond all
      b = crossing(h.counts, target);
      before_n = h.counts[b];
      __syncthreads();
    } else {
      if (step == 1) {
        if (!(r.top_p < 1.f)) continue;
        target = top_p_target(r.top_p, kept);
      } else {
        kept = over < kept ? over : kept;
        target = uniform_target(a.uniform[t], kept);
      }
      b = crossing(h.before, target);
    }
    uint64_t before_w = h.before[b], lo = 0, hi = ~0ull;
    // the tokens lo .. hi of bin b; their number, and as many as there is room for in the list
    auto list = [&]() {
      __syncthreads();
      if (tid == 0) l.list_n = 0;
      __syncthreads();
      each([&](float v, int i) {
        if (sc.bin(v) != b) return;
        const uint64_t k = place_key(v, i);
        if (k < lo || k > hi) return;
        const int at = atomicAdd(&l.list_n, 1);
        if (at < SMP_LIST) h.list.key[at] = k, h.list.w[at] = sc.weight(v);
      });
      __syncthreads();
      return l.list_n;
    };
    int n = list();
    if (n > SMP_LIST) {  // many alike: closer, over the whole order
      uint64_t kmin = ~0ull, kmax = 0;
      each([&](float v, int i) {
        if (sc.bin(v) == b) kmin = Smaller()(kmin, place_key(v, i)), kmax = Larger()(kmax, place_key(v, i));
      });
      lo = block_all64(kmin, l.part, Smaller());
      hi = block_all64(kmax, l.part, Larger());
      do {
        const int bits = 64 - __clzll((long long)(hi - lo)), shift = max(0, bits - 11);  // (hi - lo) >> shift < SMP_BINS
        __syncthreads();
        h.zoom.clear();
        __syncthreads();
        each([&](float v, int i) {
          if (sc.bin(v) != b) return;
          const uint64_t k = place_key(v, i);
          if (k >= lo && k <= hi) h.zoom.add((int)((hi - k) >> shift), sc.weight(v));
        });
        sum_bins(h.zoom.w, l.part);
        sum_bins(h.zoom.n, l.part);
        const int z = by_count ? crossing(h.zoom.n, target - before_n) : crossing(h.zoom.w, target - before_w);
        before_w += h.zoom.w[z];
        before_n += h.zoom.n[z];
        n = h.zoom.n[z + 1] - h.zoom.n[z];
        const uint64_t top = hi - ((uint64_t)z << shift);
        const uint64_t width = (1ull << shift) - 1;
        lo = top - lo > width ? top - width : lo;
        hi = top;
      } while (n > SMP_LIST);
      list();
    }
    for (int e = tid; e < n; e += SMP_THREADS) {
      const uint64_t k = h.list.key[e], w = h.list.w[e];
      uint64_t sum = before_w, rank = before_n;
#pragma unroll 4
      for (int j = 0; j < n; ++j)
        if (h.list.key[j] > k) sum += h.list.w[j], ++rank;
      if (by_count ? rank == target : (sum <= target && target < sum + w)) l.found_key = k, l.found_w = w, l.found_upto = sum + w;
    }
    __syncthreads();
    if (step < 2) kept = l.found_upto;
  }
  if (tid == 0) give(a, t, l.found_key, l.found_w, kept);
}

// The sequence of row t, -1: none; the same on all lanes.  Its first row's workgroup answers for its rules.
__device__ inline int sample_sequence(const SampleArgs& a, int t, bool& first_row) {
  const int lane = threadIdx.x & 63;
  for (int s0 = 0; s0 < a.B; s0 += 64) {
    const int q = min(s0 + lane, a.B - 1), b = a.node_off[q], e = a.node_off[q + 1];
    const uint64_t here = __ballot(s0 + lane < a.B && b >= 0 && b <= t && t < e && e <= a.T);
    if (here) {
      const int l = __builtin_ctzll(here);
      first_row = __builtin_amdgcn_readlane(b, l) == t;
      return s0 + l;
    }
  }
  return -1;
}
__device__ inline void empty_sequences(const SampleArgs& a) {
  for (int s = threadIdx.x; s < a.B; s += SMP_THREADS) {
    const int r0 = a.node_off[s], r1 = a.node_off[s + 1];
    const bool bad = r0 < 0 || r1 < r0 || r1 > a.T;
    if (bad || r0 == r1) a.status[s] = bad;
  }
}

// Every token of a row, read from memory.
struct Streamed {
  const float* x;
  int V;
  SampleScale sc;
  template <class F>
  __device__ inline void operator()(F f) const {
#pragma unroll 1
    for (int i = (int)threadIdx.x * 4; i < V; i += SMP_THREADS * 4) {
      float v[4];
      if (i + 4 <= V) {
        const f32x4_row q = *reinterpret_cast<const f32x4_row*>(x + i);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = q[e];
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = i + e < V ? x[i + e] : -INFINITY;
      }
#pragma unroll 1
      for (int e = 0; e < 4; ++e) {
        const float u = sc.seen(e == 0 ? v[0] : e == 1 ? v[1] : e == 2 ? v[2] : v[3]);
        if (is_token(u)) f(u, i + e);
      }
    }
  }
};
// 4 * NV logits per thread of x[0 .. n), 2048 apart in groups of four, -infinity where there are none.
template <int NV>
struct Held {
  float v[NV][4];
  __device__ inline void load(const float* x, int n) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int at = (i * SMP_THREADS + threadIdx.x) * 4;
      if (at + 4 <= n) {
        const f32x4_row q = *reinterpret_cast<const f32x4_row*>(x + at);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[i][e] = q[e];
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[i][e] = at + e < n ? x[at + e] : -INFINITY;
      }
    }
  }
  __device__ inline float top() const {
    float m = -INFINITY;  // (NaN is passed over)
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) m = fmaxf(m, v[i][e]);
    return m;
  }
  template <class F>
  __device__ inline void each(F f) const {
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) f(v[i][e], (i * SMP_THREADS + (int)threadIdx.x) * 4 + e);
  }
  // of the groups of four of which `some`(v0, v1, v2, v3) holds: a branch per group, not per logit
  template <class S, class F>
  __device__ inline void each_of(S some, F f) const {
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (some(v[i])) {
#pragma unroll
        for (int e = 0; e < 4; ++e) f(v[i][e], (i * SMP_THREADS + (int)threadIdx.x) * 4 + e);
      }
  }
  __device__ inline void only_infinities() {
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) v[i][e] = v[i][e] == INFINITY ? 0.f : -INFINITY;
  }
  // weights per bin; LEAST: the sum of this thread's of `least` or more
  template <bool LEAST, class Lds>
  __device__ inline uint64_t add_weights(const SampleScale& sc, uint64_t least, Lds& l) const {
    uint64_t over = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int g = 0; g < 4; g += SMP_ABREAST) {
        uint64_t w[SMP_ABREAST];
        int b[SMP_ABREAST];
#pragma unroll
        for (int e = 0; e < SMP_ABREAST; ++e) {
          w[e] = sc.weight(v[i][g + e]), b[e] = sc.bin(v[i][g + e]);
        }
#pragma unroll
        for (int e = 0; e < SMP_ABREAST; ++e) {
          atomicAdd((unsigned long long*)&l.before[b[e]], (unsigned long long)w[e]);
          if (LEAST) over += w[e] >= least ? w[e] : 0;
        }
        __builtin_amdgcn_sched_barrier(0);  // group after group, for registers
      }
    return over;
  }
};
// All logits of a part of a row, piece after piece from memory, the next one on its way.
template <int NV>
struct Pieces {
  const float* x;
  int from, to;
  template <class F>
  __device__ inline void held(F f) const {
    constexpr int STEP = 4 * NV * SMP_THREADS;
    Held<NV> ahead;
    ahead.load(x + from, to - from);
#pragma unroll 1
    for (int i = from; i < to; i += STEP) {
      Held<NV> h = ahead;
      if (i + STEP < to) ahead.load(x + i + STEP, to - i - STEP);
      f(h, i);
    }
  }
  template <class S, class F>
  __device__ inline void operator()(S some, F f) const {
    held([&](Held<NV>& h, int i0) { h.each_of(some, [&](float v, int i) { f(v, i0 + i); }); });
  }
};
// Weights of a part of a row per bin (l.before, cleared here), and the sum of those of `least` or more if that is not 0.
template <class Lds>
__device__ inline uint64_t weigh_part(const Pieces<2>& part, const SampleScale& sc, uint64_t least, Lds& l) {
  uint64_t over = 0;
  __syncthreads();
  for (int i = threadIdx.x; i <= SMP_BINS; i += SMP_THREADS) l.before[i] = 0;
  __syncthreads();
  part.held([&](Held<2>& h, int) {
    if (sc.infinite) h.only_infinities();
    if (least > 0) over += h.template add_weights<true>(sc, least, l);
    else h.template add_weights<false>(sc, 0, l);
  });
  __syncthreads();
  return over;
}
// A logit that at least k tokens of the workgroup reach, and few more: the lower end of the bin, of as many as threads over
// the range that weighs anything, in which the k-th of the threads' largest ones lies.  Where fewer threads hold tokens that
// weigh anything, one that all of those reach: behind them top-k has nothing to choose.
__device__ inline float reached_by(int k, float mine, const SampleScale& sc, ListLds& l) {
  constexpr float WIDE = (float)SMP_BINS / SMP_THREADS;
  const int tid = threadIdx.x;
  __syncthreads();
  l.count[tid] = 0;
  if (tid == 0) l.bound_bin = SMP_THREADS - 1;
  __syncthreads();
  const int b = sc.bin(sc.seen(mine));
  if (b < SMP_BINS - 1) atomicAdd(&l.count[b / (SMP_BINS / SMP_THREADS)], 1u);
  __syncthreads();
  const int c = (int)l.count[tid];
  int upto = wave_scan(c);
  if ((tid & 63) == 63) l.part.least[tid >> 6] = upto;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < SMP_WAVES - 1; ++w) upto += w < (tid >> 6) ? (int)l.part.least[w] : 0;
  if (upto >= k && upto - c < k) l.bound_bin = tid;
  __syncthreads();
  // (a token's bin is off by less than 2^-20 of its place)
  const float below = 2.f * ((float)(l.bound_bin + 1) * WIDE) / sc.per_bin * 1.00001f;
  return sc.infinite ? INFINITY : fmaxf(2.f * sc.half_top - below - fabsf(sc.half_top) * 1e-6f, -3.4028235e38f);
}
// The same for a k beyond half the threads, of all tokens that `each` goes over: the lower end of the bin in which the k-th lies.
template <class Lds, class Each>
__device__ inline float reached_by_count(int k, const SampleScale& sc, Lds& l, Each each) {
  __syncthreads();
  for (int i = threadIdx.x; i <= SMP_BINS; i += SMP_THREADS) l.counts[i] = 0;
  __syncthreads();
  each([&](float v) {
    const int b = sc.bin(sc.seen(v));
    if (b < SMP_BINS - 1) atomicAdd(&l.counts[b], 1u);
  });
  const int all = (int)sum_bins(l.counts, l.part);
  const int b = all < k ? SMP_BINS - 1 : crossing(l.counts, k - 1);
  const float below = 2.f * (float)(b + 1) / sc.per_bin * 1.00001f;  // (as above)
  return sc.infinite ? INFINITY : fmaxf(2.f * sc.half_top - below - fabsf(sc.half_top) * 1e-6f, -3.4028235e38f);
}
// Tokens from `bound` on to out[0 .. cap), in any order; their number
template <int NV>
__device__ inline int collect(const Held<NV>& x, float bound, int first_index, uint64_t* out, int cap, ListLds& l) {
  l.start_list();
  x.each_of([&](const float(&v)[4]) { return fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])) >= bound; }, [&](float v, int i) {
    if (!(v >= bound)) return;
    const int at = atomicAdd(&l.list_n, 1);
    const uint64_t k = place_key(v, first_index + i);
    if (at < cap) out[at] = k;
  });
  __syncthreads();
  return l.list_n;
}
// Row t without tokens, or greedy
__device__ inline void give_first(const SampleArgs& a, int t, uint64_t best) {
  a.token[t] = best == 0 ? -1 : key_index(best);
  if (a.prob) a.prob[t] = best == 0 ? 0.f : 1.f;
}

__device__ inline float min_p_bound(const SampleRules& r, float top) {
  // A weight is rounded to nearest: `least` from least - 0.5 of a unit on.  A token below the bound is less than that by a
  // thousandth, far more than the errors of weights (2^-40 of them) and of the bound (2^-24 of its two terms).
  return (float)((double)top + log(((double)r.least - 0.5) * 0.999 / SMP_UNIT) * r.t - fabs((double)top) * 1e-6);
}

// Everything from the row in memory, for the few rows that need it.
__device__ inline void finish_slowly(const SampleArgs& a, int t, const SampleRules& r, const SampleScale& sc, SampleLds& l) {
  const int tid = threadIdx.x;
  const Streamed each{a.x + (size_t)t * a.V, a.V, sc};
  __syncthreads();
  for (int i = tid; i <= SMP_BINS; i += SMP_THREADS) l.before[i] = 0;
  __syncthreads();
  uint64_t over = 0;
  each([&](float v, int) {
    const uint64_t w = sc.weight(v);
    atomicAdd((unsigned long long*)&l.before[sc.bin(v)], (unsigned long long)w);
    over += w >= r.least ? w : 0;
  });
  sum_bins(l.before, l.part);
  over = block_all64(over, l.part, Plus());
  finish_histogram(a, t, r, sc, l, over, each);
}

// One workgroup per row, the row in registers.
template <int NV>
__global__ __launch_bounds__(SMP_THREADS, 4) void sample_row_kernel(SampleArgs a) {
  __shared__ SampleLds l;
  const int tid = threadIdx.x, t = blockIdx.x;
  if (t == 0) empty_sequences(a);
  Held<NV> row;
  const float* const x = a.x + (size_t)t * a.V;
  row.load(x, a.V);
  bool first_row = false;
  const int s = sample_sequence(a, t, first_row);
  if (s < 0) return;
  const SampleRules r(a.rules + 4 * s);
  const float u = a.uniform[t];
  if (first_row && tid == 0) a.status[s] = r.bad;
  if (r.bad) return;
  const float mine = row.top(), top = block_max(mine, l.part);
  if (!is_token(top) || r.t == 0.f) {
    uint64_t best = 0;
    row.each([&](float v, int i) {
      if (v == top && is_token(v)) best = Larger()(best, place_key(v, i));
    });
    best = block_all64(best, l.part, Larger());
    if (tid == 0) give_first(a, t, best);
    return;
  }
  const SampleScale sc(top, r.t);
  // ---- the short list
  if (r.short_by_k() || r.short_by_min()) {
    const int k = r.short_by_k() ? (int)r.top_k : 0;
    const float bound = k == 0                 ? min_p_bound(r, top)
                        : k <= SMP_THREADS / 2 ? reached_by(k, mine, sc, l)
                                               : reached_by_count(k, sc, l, [&](auto f) { row.each([&](float v, int) { f(v); }); });
    if (bound > -INFINITY) {
      const int n = collect(row, bound, 0, l.few.key, SMP_LIST, l);
      if (n <= SMP_LIST) {
        finish_list(a, t, u, r, sc, l, n, k > 0 ? min(n, k) : n);
        return;
      }
    }
  }
  // ---- the histogram
  uint64_t over = weigh_part(Pieces<2>{x, 0, a.V}, sc, r.least, l);
  sum_bins(l.before, l.part);
  over = r.least > 0 ? block_all64(over, l.part, Plus()) : l.before[SMP_BINS];
  if (!finish_bins(a, t, u, r, sc, l, over, Pieces<4>{x, 0, a.V})) finish_slowly(a, t, r, sc, l);
}

// ---- rows cut into chunks: what every chunk finds out by itself, then the weights of the rows that need them all, then the rows
struct ChunkedRows {
  int row0, rows, chunks, size;  // of the launch; per row; logits, a multiple of 4
  float* top;                    // [rows][chunks]
  int32_t* n;                    // tokens listed, -1: not all that top-k or min-p could keep
  uint64_t *over, *data;         // weights that min-p allows; the list, or the weights per bin, [SMP_BINS]
  __device__ inline size_t at(int t, int c) const { return (size_t)(t - row0) * chunks + c; }
};
constexpr int SMP_CHUNK_LIST = SMP_BINS;  // as many as a chunk has room for

template <int NV>
__global__ __launch_bounds__(SMP_THREADS) void sample_chunk_kernel(SampleArgs a, ChunkedRows ch) {
  __shared__ ChunkLds l;
  const int tid = threadIdx.x, t = ch.row0 + blockIdx.x / ch.chunks, c = blockIdx.x % ch.chunks, first = c * ch.size;
  if (blockIdx.x == 0 && ch.row0 == 0) empty_sequences(a);
  Held<NV> row;
  row.load(a.x + (size_t)t * a.V + first, min(ch.size, a.V - first));
  const size_t at = ch.at(t, c);
  bool first_row = false;
  const int s = sample_sequence(a, t, first_row);
  const SampleRules r(a.rules + 4 * max(s, 0));
  if (s >= 0 && first_row && c == 0 && tid == 0) a.status[s] = r.bad;
  if (s < 0 || r.bad) {
    if (tid == 0) ch.n[at] = 0;  // nothing to weigh
    return;
  }
  const float mine = row.top(), top = block_max(mine, l.part);
  int n = -1;
  if (!is_token(top) || r.t == 0.f) {
    n = 0;
  } else if (r.short_by_k() || r.short_by_min()) {
    const int k = r.short_by_k() ? (int)r.top_k : 0;
    const SampleScale sc(top, r.t);
    const float bound = k == 0                 ? min_p_bound(r, top)
                        : k <= SMP_THREADS / 2 ? reached_by(k, mine, sc, l)
                                               : reached_by_count(k, sc, l, [&](auto f) { row.each([&](float v, int) { f(v); }); });
    if (bound > -INFINITY) n = collect(row, bound, first, ch.data + at * SMP_BINS, SMP_CHUNK_LIST, l);
    if (n > SMP_CHUNK_LIST) n = -1;
  }
  if (tid == 0) ch.top[at] = top, ch.n[at] = n;
}
// largest logit of a row, and whether its chunks list all that top-k or min-p could keep (or have no need to)
struct ChunkedTop {
  float top;
  bool listed;
};
__device__ inline ChunkedTop chunked_top(const ChunkedRows& ch, int t) {
  float top = -INFINITY;
  bool listed = true;
  for (int c = threadIdx.x & 63; c < ch.chunks; c += 64) {
    const size_t at = ch.at(t, c);
    top = fmaxf(top, ch.top[at]);
    listed = listed && ch.n[at] >= 0;
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
  return ChunkedTop{top, __ballot(!listed) == 0};
}
__global__ __launch_bounds__(SMP_THREADS) void sample_weigh_kernel(SampleArgs a, ChunkedRows ch) {
  __shared__ WeighLds l;
  const int tid = threadIdx.x, t = ch.row0 + blockIdx.x / ch.chunks, c = blockIdx.x % ch.chunks, first = c * ch.size;
  const ChunkedTop x = chunked_top(ch, t);
  if (x.listed) return;
  bool first_row = false;
  const SampleRules r(a.rules + 4 * sample_sequence(a, t, first_row));
  const SampleScale sc(x.top, r.t);
  uint64_t over = weigh_part(Pieces<2>{a.x + (size_t)t * a.V, first, min(first + ch.size, a.V)}, sc, r.least, l);
  if (r.least > 0) over = block_all64(over, l.part, Plus());
  const size_t at = ch.at(t, c);
  for (int i = tid; i < SMP_BINS; i += SMP_THREADS) ch.data[at * SMP_BINS + i] = l.before[i];
  if (tid == 0) ch.over[at] = over;
}
__global__ __launch_bounds__(SMP_THREADS) void sample_finish_kernel(SampleArgs a, ChunkedRows ch) {
  __shared__ SampleLds l;
  const int tid = threadIdx.x, t = ch.row0 + blockIdx.x;
  bool first_row = false;
  const int s = sample_sequence(a, t, first_row);
  if (s < 0) return;
  const SampleRules r(a.rules + 4 * s);
  const float u = a.uniform[t];
  if (r.bad) return;
  const ChunkedTop x = chunked_top(ch, t);
  const float* const row = a.x + (size_t)t * a.V;
  if (!is_token(x.top) || r.t == 0.f) {
    uint64_t best = 0;
    if (is_token(x.top)) {
      int c = 0;
      while (ch.top[ch.at(t, c)] != x.top) ++c;  // (one of them is the largest)
      Pieces<8>{row, c * ch.size, min(a.V, (c + 1) * ch.size)}([&](const float(&v)[4]) { return fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])) == x.top; }, [&](float v, int i) {
        if (v == x.top) best = Larger()(best, place_key(v, i));
      });
    }
    best = block_all64(best, l.part, Larger());
    if (tid == 0) give_first(a, t, best);
    return;
  }
  const SampleScale sc(x.top, r.t);
  if (x.listed) {
    const int k = r.short_by_k() ? (int)r.top_k : 0;
    // entry e of all: chunk c's from upto[c] on
    uint32_t* const upto = l.few.bin;
    for (int c = tid; c <= SMP_BINS; c += SMP_THREADS) upto[c] = c < ch.chunks ? ch.n[ch.at(t, c)] : 0;
    const int all = (int)sum_bins(l.few.bin, l.part);
    auto entries = [&](auto f) {
#pragma unroll 4
      for (int e = tid; e < all; e += SMP_THREADS) {
        const int c = crossing(l.few.bin, e);
        f(ch.data[ch.at(t, c) * SMP_BINS + (e - upto[c])]);
      }
    };
    float bound = k > 0 ? -INFINITY : min_p_bound(r, x.top);
    if (k > SMP_THREADS / 2 && all > SMP_LIST) {  // (the counts lie before upto)
      bound = reached_by_count(k, sc, l, [&](auto f) { entries([&](uint64_t key) { f(key_logit(key)); }); });
    } else if (k > 0 && all > SMP_LIST) {
      uint64_t best = 0;
      entries([&](uint64_t key) { best = Larger()(best, key); });
      bound = reached_by(k, best == 0 ? -INFINITY : key_logit(best), sc, l);
    }
    l.start_list();
    entries([&](uint64_t key) {
      if (!(key_logit(key) >= bound)) return;
      const int at = atomicAdd(&l.list_n, 1);
      if (at < SMP_LIST) l.few.key[at] = key;
    });
    __syncthreads();
    const int n = l.list_n;
    if (n <= SMP_LIST) {
      finish_list(a, t, u, r, sc, l, n, k > 0 ? min(n, k) : n);
      return;
    }
  }
  // ---- the histogram of the chunks, or, where the lists were too long after all, from the row itself
  if (!x.listed) {
    for (int i = tid; i <= SMP_BINS; i += SMP_THREADS) {
      uint64_t w = 0;
      if (i < SMP_BINS)
#pragma unroll 8
        for (int c = 0; c < ch.chunks; ++c) w += ch.data[ch.at(t, c) * SMP_BINS + i];
      l.before[i] = w;
    }
    __syncthreads();
    uint64_t over = 0;
    if (r.least > 0)
      for (int c = tid; c < ch.chunks; c += SMP_THREADS) over += ch.over[ch.at(t, c)];
    sum_bins(l.before, l.part);
    over = r.least > 0 ? block_all64(over, l.part, Plus()) : l.before[SMP_BINS];
    if (finish_bins(a, t, u, r, sc, l, over, Pieces<8>{row, 0, a.V})) return;
  }
  finish_slowly(a, t, r, sc, l);
}

// ------------------------------------------------------------------ launch
constexpr int SMP_ROW = 64 * SMP_THREADS, SMP_CHUNK = 64 * SMP_THREADS;  // logits that a workgroup holds
struct SampleLaunch {
  int chunks, size, rows;  // per row; logits; rows of a launch
};
static SampleLaunch sample_launch(int T, int V) {
  SampleLaunch p{0, 0, T};
  if (V <= SMP_ROW) return p;
  const int least = (V + SMP_CHUNK - 1) / SMP_CHUNK, most = (V + 16 * SMP_THREADS - 1) / (16 * SMP_THREADS);
  // Two workgroups per compute unit at a time, but no fewer than 16 logits per thread: of one row of 128256, top-k 200, chunks of
  // 8 per thread took 46 us, of 16 34 (their lists are put together by one workgroup); of 69 rows no difference.
  p.chunks = std::min(std::max(least, 512 / T), most);
  p.size = ((V + p.chunks - 1) / p.chunks + 3) / 4 * 4;
  p.chunks = (V + p.size - 1) / p.size;
  p.rows = std::max(1, std::min(T, 4096 / p.chunks));
  return p;
}
size_t tree_sample_ws_bytes(int T, int V) {
  const SampleLaunch p = sample_launch(T, V);
  return (size_t)p.rows * p.chunks * (8 * SMP_BINS + 16) + 16;
}
template <int NV>
static int sample_chunked(const SampleArgs& a, const ChunkedRows& ch, hipStream_t st) {
  sample_chunk_kernel<NV><<<ch.rows * ch.chunks, SMP_THREADS, 0, st>>>(a, ch);
  sample_weigh_kernel<<<ch.rows * ch.chunks, SMP_THREADS, 0, st>>>(a, ch);
  sample_finish_kernel<<<ch.rows, SMP_THREADS, 0, st>>>(a, ch);
  return check_launch();
}
int launch_tree_sample(const float* x, const int32_t* node_off, int B, int T, int V, const float* rules,
                       const float* uniform, int32_t* token, float* prob, void* ws, int32_t* status, hipStream_t st) {
  const SampleArgs a{x, node_off, B, T, V, rules, uniform, token, prob, status};
  const SampleLaunch p = sample_launch(T, V);
  if (p.chunks == 0) {
    if (V <= 8 * SMP_THREADS) sample_row_kernel<2><<<T, SMP_THREADS, 0, st>>>(a);
    else if (V <= 32 * SMP_THREADS) sample_row_kernel<8><<<T, SMP_THREADS, 0, st>>>(a);
    else sample_row_kernel<16><<<T, SMP_THREADS, 0, st>>>(a);
    return check_launch();
  }
  const size_t all = (size_t)p.rows * p.chunks;
  uint64_t* const data = (uint64_t*)ws;
  for (int row0 = 0; row0 < T; row0 += p.rows) {
    const ChunkedRows ch{row0, std::min(p.rows, T - row0), p.chunks, p.size, (float*)(data + all * (SMP_BINS + 1)),
                         (int32_t*)(data + all * (SMP_BINS + 1)) + all, data + all * SMP_BINS, data};
    const int rc = p.size <= 32 * SMP_THREADS ? sample_chunked<8>(a, ch, st) : sample_chunked<16>(a, ch, st);
    if (rc != TRJ_OK) return rc;
  }
  return TRJ_OK;
}

}  // namespace trj
