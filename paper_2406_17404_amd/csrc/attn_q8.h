// What the attentions over the paged 8-bit cache share: operands from codes and the running softmax.
#pragma once
#include "q8.h"

namespace trj {

template <class T>
__device__ inline T lane_value(T v, int lane) { return (T)__builtin_amdgcn_readlane((int)v, lane); }

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
__device__ inline uint32_t bf16_pair(uint32_t codes, float scale, bool hi) {
  return hi ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, true))
            : __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, false));
}
__device__ inline bf16x8 operand(uint32_t a, uint32_t b, float scale) {  // 8 codes
  const u32x4 v = {bf16_pair(a, scale, false), bf16_pair(a, scale, true), bf16_pair(b, scale, false), bf16_pair(b, scale, true)};
  return __builtin_bit_cast(bf16x8, v);
}

// Running softmax of one tile of 32 queries, a query per lane and its partner lane + 32: products with
// 32 keys in (times f: log2 scores), -infinity where not visible; bf16 weights out (the B operand of the
// second product).  Weights are relative to a reference: the largest score when it was last lifted, which
// happens once a score exceeds it by more than SLACK.  Weights of up to 2^SLACK cost no
// precision (they are floating-point numbers), and with the running maximum itself some query of a tile
// would move it, and have the sums rescaled, in nearly every block.
constexpr float SLACK = 16.f, NO_REFERENCE = -3.4028235e38f;
struct Softmax {
  float m = NO_REFERENCE, l = 0.f;
  __device__ __forceinline__ static float largest(const f32x16& s, float f) {
    float mx = s[0];
#pragma unroll
    for (int v = 1; v < 16; ++v) mx = fmaxf(mx, s[v]);
    const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
    return fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1])) * f;
  }
  __device__ __forceinline__ bool too_low(float top) const { return top > m + SLACK; }
  __device__ __forceinline__ float lift(float top) {  // the factor of the sums so far
    const float ref = fmaxf(m, top), alpha = __builtin_amdgcn_exp2f(m - ref);
    l *= alpha;
    m = ref;
    return alpha;
  }
  __device__ __forceinline__ void weigh(const f32x16& s, float f, u32x4 (&pk)[2]) {
#pragma clang fp contract(off)
    float p[16], sum = 0.f;
    // product and difference rounded one by one: fused, the rounding of the reference's own product would
    // stay in the exponent, 1 and more for scores beyond 2^24
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      const float x = s[v] * f;
      p[v] = __builtin_amdgcn_exp2f(x - m);
      sum += p[v];
    }
    l += sum;
#pragma unroll
    for (int kg = 0; kg < 2; ++kg)
#pragma unroll
      for (int e = 0; e < 4; ++e) pk[kg][e] = pack2bf(p[8 * kg + 2 * e], p[8 * kg + 2 * e + 1]);
  }
};

template <int MTV>
__device__ inline void q8_rescale(f32x16 (&o)[MTV], float alpha) {
#pragma unroll
  for (int mt = 0; mt < MTV; ++mt) {
#pragma unroll
    for (int v = 0; v < 16; ++v) o[mt][v] *= alpha;
    __builtin_amdgcn_sched_barrier(0);  // part after part, for registers
  }
}

}  // namespace trj
