// The paged 8-bit cache: where a page keeps its codes, what a scale is, and how a workgroup
// finds its sequence from device-side lengths.  Layout and rules: include/trjacobi.h.
#pragma once
#include "common.h"

namespace trj {

constexpr int Q8_MIN_EXP = -100;  // of a scale

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

__device__ inline int wave_scan(int x) {  // inclusive sum over the lanes
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(x, o);
    if (lane >= o) x += y;
  }
  return x;
}
// The sequence that owns item x when sequence s has count(s) items, and which of its items it is; false
// behind the last item.  Every wavefront by itself, 64 sequences a round, uniform answers.
template <class F>
__device__ inline bool find_seq(int x, int B, F count, int& s, int& nth) {
  const int lane = threadIdx.x & 63;
  int base = 0;
  for (int s0 = 0; s0 < B; s0 += 64) {
    const int c = s0 + lane < B ? count(s0 + lane) : 0;
    const int upto = base + wave_scan(c);
    const uint64_t here = __ballot(x < upto);
    if (here) {
      const int l = __builtin_ctzll(here);
      s = s0 + l;
      nth = x - (__shfl(upto, l) - __shfl(c, l));
      s = __builtin_amdgcn_readfirstlane(s);
      nth = __builtin_amdgcn_readfirstlane(nth);
      return true;
    }
    base = __shfl(upto, 63);
  }
  return false;
}

}  // namespace trj
