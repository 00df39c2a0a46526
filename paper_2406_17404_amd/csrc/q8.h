// The paged 8-bit cache: where a page keeps its codes, what a scale is, and how a workgroup
// finds its sequence from device-side lengths.  Layout and rules: include/trjacobi.h.
#pragma once
#include "common.h"

namespace trj {

constexpr int Q8_MIN_EXP = -100;  // of a scale
constexpr float LOG2E = 1.4426950408889634f;
// Positions and slots are int32, and so are those up to the end of their page: a table may be wider than this, a
// sequence may not be longer.
constexpr int Q8_MAX_PAGES = INT32_MAX / TRJ_KV_BLOCK;
__host__ __device__ inline int q8_pages_at_most(int max_blocks) { return max_blocks < Q8_MAX_PAGES ? max_blocks : Q8_MAX_PAGES; }

__host__ __device__ inline int q8_k_off(int r, int c) { return ((c >> 4) * 32 + r) * 16 + (c & 15); }
__host__ __device__ inline int q8_v_off(int r, int c) {
  return (((c >> 5) * 2 + ((r >> 2) & 1)) * 32 + (c & 31)) * 16 + (r >> 4) * 8 + ((r >> 3) & 1) * 4 + (r & 3);
}
__host__ __device__ inline float q8_pow2(int e) {  // e in -126..127
  union { uint32_t u; float f; } c;
  c.u = (uint32_t)(e + 127) << 23;
  return c.f;
}
// Exponent of the smallest power of two with which a largest magnitude (the bits of a finite fp32 >= 0)
// fits: 448 = 1.75 * 2^8, so 1.m * 2^e needs 2^(e - 8) up to 1.75 * 2^e and twice that beyond.
__host__ __device__ inline int q8_exp(uint32_t top) {
  const int e = (int)(top >> 23) - 127 - ((top & 0x7fffffu) <= 0x600000u ? 8 : 7);
  return top == 0 || e < Q8_MIN_EXP ? Q8_MIN_EXP : e;
}
// exponent of a stored scale, whose fraction does not count; kept to where the powers of two are numbers
__device__ inline int q8_exp_of(float scale) {
  const int e = (int)((__float_as_uint(scale) >> 23) & 255) - 127;
  return e < -126 ? -126 : e > 126 ? 126 : e;
}
// Two numbers to two codes (bits 0..15), round to nearest even; what is not finite to the NaN 0x7f (the
// instruction would take infinities to the largest number and choose the NaN's sign itself).
__device__ inline uint32_t q8_codes(float a, float b) {
  const uint32_t c = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (fabsf(a) < INFINITY ? c & 0xffu : 0x7fu) | (fabsf(b) < INFINITY ? c & 0xff00u : 0x7f00u);
}

// Sums over the lanes by data-parallel moves inside the vector unit: rows of 16 lanes, then the rows' last lanes
// into the rows behind them.  (Through __shfl, which goes by way of LDS, a scan took 0.4 us.)
template <int MOVE, int ROWS>
__device__ inline int moved(int none, int x) {
  return __builtin_amdgcn_update_dpp(none, x, MOVE, ROWS, 0xf, false);
}
#define TRJ_WAVE_STEPS(STEP) \
  STEP(0x111, 0xf) STEP(0x112, 0xf) STEP(0x114, 0xf) STEP(0x118, 0xf) STEP(0x142, 0xa) STEP(0x143, 0xc)
__device__ inline int wave_scan(int x) {  // inclusive sum
#define TRJ_STEP(MOVE, ROWS) x += moved<MOVE, ROWS>(0, x);
  TRJ_WAVE_STEPS(TRJ_STEP)
#undef TRJ_STEP
  return x;
}
__device__ inline float wave_sum(float x) {  // the same for all lanes
#define TRJ_STEP(MOVE, ROWS) x += __int_as_float(moved<MOVE, ROWS>(0, __float_as_int(x)));
  TRJ_WAVE_STEPS(TRJ_STEP)
#undef TRJ_STEP
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
}
__device__ inline uint32_t wave_min(uint32_t x) {
#define TRJ_STEP(MOVE, ROWS) x = min(x, (uint32_t)moved<MOVE, ROWS>(-1, (int)x));
  TRJ_WAVE_STEPS(TRJ_STEP)
#undef TRJ_STEP
  return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}
__device__ inline uint32_t wave_max(uint32_t x) {
#define TRJ_STEP(MOVE, ROWS) x = max(x, (uint32_t)moved<MOVE, ROWS>(0, (int)x));
  TRJ_WAVE_STEPS(TRJ_STEP)
#undef TRJ_STEP
  return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}
// The sequence that owns item x when sequence s has count(s) items, and which of its items it is; false
// behind the last item.  Every wavefront by itself, 128 sequences a round, uniform answers.
template <class F>
__device__ inline bool find_seq(int x, int B, F count, int& s, int& nth) {
  const int lane = threadIdx.x & 63;
  int base = 0;
  for (int s0 = 0; s0 < B; s0 += 128) {
    int c[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {  // both asked for together
      const int q = s0 + 64 * u + lane, n = count(min(q, B - 1));
      c[u] = q < B ? n : 0;
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int upto = base + wave_scan(c[u]);
      const uint64_t here = __ballot(x < upto);
      if (here) {
        const int l = __builtin_ctzll(here);
        s = s0 + 64 * u + l;
        nth = x - (__builtin_amdgcn_readlane(upto, l) - __builtin_amdgcn_readlane(c[u], l));
        return true;
      }
      base = __builtin_amdgcn_readlane(upto, 63);
    }
  }
  return false;
}

}  // namespace trj
