// The cache in 4 bits: its layout, its quantiser, its values.
//
// A row of D elements is NG = D / 32 groups. A group's (step, mid) are two bf16 (step in the low half of a 32-bit word):
//   mid = bf16((lo + hi) / 2),  step = bf16((hi - lo) / 15),  lo and hi the group's extremes
//   code(x) = clamp(floor((x - mid) / step) + 8, 0, 15),  8 where step = 0;   value = mid + (code - 7.5) step
// The code of element 32 G + 4 i + e (i < 8, e < 4) is nibble e of the row's 16-bit word i * NG + G: the products of decode attention
// take their operands in this order, every load a whole word of it.
#pragma once

#include "common.cuh"

namespace madakv {
namespace {

template <int D>
struct QuantRow {
  static constexpr int NG = D / 32;
  static constexpr int LANES = D / 4;      // lanes that share a row: lane i * NG + G holds elements 32 G + 4 i .. + 3
  static constexpr int CODE_BYTES = D / 2;
  static constexpr int PAR_BYTES = NG * 4;
};

__device__ __forceinline__ float min_nan(float a, float b) {
  float r;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// (step, mid) of a group with these extremes. In 64 bits, because the two are functions of the exact sum and difference; one that
// is not finite makes both NaN, and with them all values of the group.
__device__ __forceinline__ uint32_t group_par(float lo, float hi) {
  const float mid = (float)(((double)lo + (double)hi) * 0.5), step = (float)(((double)hi - (double)lo) * (1.0 / 15.0));
  const __nv_bfloat162 r = __floats2bfloat162_rn(step, mid);
  const uint32_t w = *reinterpret_cast<const uint32_t*>(&r);
  return isfinite(bf16_lo(w)) && isfinite(bf16_hi(w)) ? w : 0x7fc07fc0u;
}

// floor((x - mid) / step) + 8 to the last bit. The quotient in 64 bits is never below a whole number that the true one reaches, but may have been
// rounded up to one, and so may the difference. The multiple of step that it claims is exact (a few bits times eight), and so is d + rest = x - mid:
// neither d nor the multiple lies within `rest`, half a last bit of d, of the other one without being equal to it.
__device__ __forceinline__ uint32_t code_of(float x, float step, float mid) {
  if (!(step > 0.f)) return 8u;
  const double d = __dsub_rn(x, mid), y = __dsub_rn(d, x), rest = __dadd_rn(__dsub_rn(x, __dsub_rn(d, y)), __dsub_rn(-(double)mid, y));
  double t = floor(d / (double)step);
  const double border = t * (double)step;
  if (d < border || (d == border && rest < 0.0)) t -= 1.0;
  return (uint32_t)fmin(fmax(t + 8.0, 0.0), 15.0);
}

// The codes of a lane's four elements and its group's (step, mid); all lanes of the row take part.
template <int D>
__device__ __forceinline__ void quantise4(const float (&x)[4], uint32_t& codes, uint32_t& par) {
  float lo = min_nan(min_nan(x[0], x[1]), min_nan(x[2], x[3])), hi = max_nan(max_nan(x[0], x[1]), max_nan(x[2], x[3]));
#pragma unroll
  for (int off = QuantRow<D>::NG; off < QuantRow<D>::LANES; off *= 2) {
    lo = min_nan(lo, __shfl_xor_sync(0xffffffffu, lo, off));
    hi = max_nan(hi, __shfl_xor_sync(0xffffffffu, hi, off));
  }
  par = group_par(lo, hi);
  const float step = bf16_lo(par), mid = bf16_hi(par);
  codes = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) codes |= code_of(x[e], step, mid) << (4 * e);
}

__device__ __forceinline__ void load4(const float* p, float (&x)[4]) {
  const float4 v = *reinterpret_cast<const float4*>(p);
  x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
}
__device__ __forceinline__ void load4(const __nv_bfloat16* p, float (&x)[4]) {
  const uint2 v = *reinterpret_cast<const uint2*>(p);
  x[0] = bf16_lo(v.x); x[1] = bf16_hi(v.x); x[2] = bf16_lo(v.y); x[3] = bf16_hi(v.y);
}

}  // namespace
}  // namespace madakv
