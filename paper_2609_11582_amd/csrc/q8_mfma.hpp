// Operands and constants of the 8-bit cache's attention kernels.
#pragma once

#include "q8.hpp"
#include "wave_ops.hpp"

namespace okvq {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx16 __attribute__((ext_vector_type(16)));

constexpr float kNoScore = -1e30f;   // a reference before any token; finite, so that differences with -inf are -inf
constexpr float kLazy = 8.0f;        // references move when passed by 2^8
constexpr float kWeightExp = 7.0f;   // weights are at most 2^(kLazy + kWeightExp)

__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  const half2v v = {(_Float16)lo, (_Float16)hi};
  return __builtin_bit_cast(uint32_t, v);
}

__device__ __forceinline__ uint32_t or4(uint4 v) { return v.x | v.y | v.z | v.w; }

// Two of a dword's codes as fp16, exactly. int8: byte code ^ 0x80 under the exponent of 1024 is 1024 + 128 + code.
template <int kFmt, bool kHigh>
__device__ __forceinline__ uint32_t widen2(uint32_t w) {
  if constexpr (kFmt == OKVQ_Q8_INT8) {
    const uint32_t u = __builtin_amdgcn_perm(0x64646464u, w, kHigh ? 0x04030402u : 0x04010400u);
    return __builtin_bit_cast(uint32_t, __builtin_bit_cast(half2v, u) - half2v{(_Float16)1152.0f, (_Float16)1152.0f});
  } else {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, kHigh));
  }
}
// eight codes, in order
template <int kFmt>
__device__ __forceinline__ half8 widen8(uint32_t a, uint32_t b) {
  if constexpr (kFmt == OKVQ_Q8_INT8) {
    a ^= 0x80808080u;
    b ^= 0x80808080u;
  }
  return __builtin_bit_cast(half8, make_uint4(widen2<kFmt, false>(a), widen2<kFmt, true>(a), widen2<kFmt, false>(b),
                                              widen2<kFmt, true>(b)));
}

// The factor 2^(M - m - kWeightExp) / l of a row's sums of products, 0 for a row without weight. The power of two may lie far
// below fp32's normal numbers (value scales down to 2^-126, l up to 2^27 tokens), where the exponential gives zero:
// its whole part is added to the product's exponent at the end.
struct RowFactor {
  float f;
  int e;
  __device__ __forceinline__ RowFactor(float M, float m, float l) {
    const float x = fmaxf(M - m - kWeightExp, -1000.0f), whole = rintf(x);
    f = l > 0.0f ? __builtin_amdgcn_exp2f(x - whole) / l : 0.0f;
    e = (int)whole;
  }
  __device__ __forceinline__ float operator()(float v) const { return ldexpf(v * f, e); }
};

// A lane's query channels as fp16 operands; returns the factor that belongs to the scores. fp16 rows enter as they
// are. bfloat16 rows are scaled by a power of two that puts the row's largest magnitude into [2^14, 2^15): their
// 8 bits fit fp16, and what lies 2^-29 or more below the largest is lost at most. row_max: the maximum over the lanes
// that share the row.
template <bool kBf16, int kN, typename RowMax>
__device__ __forceinline__ float query_operands(const uint4 (&raw)[kN], half8 (&op)[kN], RowMax&& row_max) {
  if constexpr (!kBf16) {
#pragma unroll
    for (int i = 0; i < kN; ++i) op[i] = __builtin_bit_cast(half8, raw[i]);
    return 1.0f;
  } else {
    float top = 0.0f;
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
#pragma unroll
      for (int d = 0; d < 4; ++d) top = fmaxf(top, fmaxf(fabsf(row_lo<true>(w[d])), fabsf(row_hi<true>(w[d]))));
    }
    top = row_max(top);
    // exponent of the largest: its biased field, at least that of the smallest normal number
    const int e = max((int)(__builtin_bit_cast(uint32_t, top) >> 23), 1) - 127;
    const float up = ldexpf(1.0f, min(14 - e, 127)), down = ldexpf(1.0f, max(e - 14, -127));
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
      uint32_t y[4];
#pragma unroll
      for (int d = 0; d < 4; ++d) y[d] = pack_f16(row_lo<true>(w[d]) * up, row_hi<true>(w[d]) * up);
      op[i] = __builtin_bit_cast(half8, make_uint4(y[0], y[1], y[2], y[3]));
    }
    return down;
  }
}

}  // namespace okvq
