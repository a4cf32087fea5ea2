// The 4-bit form of a K or V row (vatp_cache_q4 in vatp.h describes it): device helpers of the kernels that write and read it.
#pragma once
#include "vatp_internal.cuh"

namespace vatp {

constexpr int Q4_GROUP = 32;              // channels that share a scale and a low end
constexpr float Q4_LEAST = 7.888609052210118e-31f;     // 2^-100: a smaller scale counts as none

// scale, low end and reciprocal of a group whose values span [mn, mx].  The low end is rounded down and the scale up, so that no
// value lies outside [lo, lo + 15 sc] and the nearest code is off by half a step at most.
// A group with a value that is not finite, or with a range beyond that of fp32, stands for NaN: both parameters are, whatever the codes.
struct Q4Group {
  float sc, lo, inv;
};
// (of a NaN and a number: NaN)
__device__ __forceinline__ float min_nan(float a, float b) {
  float x;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(x) : "f"(a), "f"(b));
  return x;
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float x;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(x) : "f"(a), "f"(b));
  return x;
}
__device__ __forceinline__ Q4Group q4_group(float mn, float mx) {
  Q4Group g;
  g.lo = __bfloat162float(__float2bfloat16_rd(mn));
  g.sc = __bfloat162float(__float2bfloat16_ru(__fdiv_rn(__fsub_rn(mx, g.lo), 15.f)));
  if (g.sc < Q4_LEAST) g.sc = 0.f;
  if (!(g.sc < INFINITY)) g.sc = g.lo = __uint_as_float(0x7fff0000u);
  g.inv = g.sc > 0.f ? __frcp_rn(g.sc) : 0.f;
  return g;
}
// rint((x - lo) / sc) of four values, 0 .. 15 each (the scale is rounded up: 15 is not exceeded), each operation rounded by itself; the
// four nibbles in the low half of the result, the first lowest.  Adding 1.5 * 2^23 rounds to the nearest integer, which then
// stands in the low bits.
__device__ __forceinline__ uint32_t q4_codes(const Q4Group& g, float x0, float x1, float x2, float x3) {
  constexpr float M = 12582912.f;
  const uint32_t c0 = __float_as_uint(__fadd_rn(__fmul_rn(__fsub_rn(x0, g.lo), g.inv), M)), c1 = __float_as_uint(__fadd_rn(__fmul_rn(__fsub_rn(x1, g.lo), g.inv), M));
  const uint32_t c2 = __float_as_uint(__fadd_rn(__fmul_rn(__fsub_rn(x2, g.lo), g.inv), M)), c3 = __float_as_uint(__fadd_rn(__fmul_rn(__fsub_rn(x3, g.lo), g.inv), M));
  return (c0 + 16u * c1) + 256u * (c2 + 16u * c3);       // (above the low half: whatever the float's upper bits add up to)
}
// a group's parameters as stored: the scale in the low half, the low end in the high half (both are bf16 values)
__device__ __forceinline__ uint32_t q4_params(const Q4Group& g) {
  return (__float_as_uint(g.sc) >> 16) | (__float_as_uint(g.lo) & 0xffff0000u);
}
__device__ __forceinline__ float q4_scale(uint32_t params) { return __uint_as_float(params << 16); }
__device__ __forceinline__ float q4_low(uint32_t params) { return __uint_as_float(params & 0xffff0000u); }

// byte of a row of HD channels that holds channel 32 g + 4 j (low nibble) and the one after it; the next two are in the next byte
template <int HD> __host__ __device__ constexpr int q4_byte(int g, int j) { return j * (HD / 16) + 2 * g; }

// One row by one warp: lane l < HD / 4 has channels 4 l .. 4 l + 3 (group l / 8, j = l mod 8) in x.  Returns the two code bytes
// and sets `params` of the lane's group; lanes from HD / 4 on take part in the exchange only.
__device__ __forceinline__ uint32_t q4_row(const float (&x)[4], uint32_t& params) {
  float mn = min_nan(min_nan(x[0], x[1]), min_nan(x[2], x[3])), mx = max_nan(max_nan(x[0], x[1]), max_nan(x[2], x[3]));
#pragma unroll
  for (int o = 1; o < 8; o <<= 1) {
    mn = min_nan(mn, __shfl_xor_sync(0xffffffffu, mn, o));
    mx = max_nan(mx, __shfl_xor_sync(0xffffffffu, mx, o));
  }
  const Q4Group g = q4_group(mn, mx);
  params = q4_params(g);
  return q4_codes(g, x[0], x[1], x[2], x[3]) & 0xffffu;
}

}  // namespace vatp
