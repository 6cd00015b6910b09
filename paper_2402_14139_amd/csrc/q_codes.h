// Codes of 8 and 4 bits with an exponent shared by 32 elements.
#pragma once
#include "pw_math.h"

namespace nf {
namespace {

constexpr int GROUP = 32;  // elements that share an exponent

// Largest code: its mantissa (1 <= m < 2) and exponent.
template <int F>
struct Format;
template <>
struct Format<NF_Q_INT8> {
  static constexpr float top = 127.f / 64.f;
  static constexpr int k = 6, bits = 8;
};
template <>
struct Format<NF_Q_E4M3> {
  static constexpr float top = 1.75f;
  static constexpr int k = 8, bits = 8;
};
template <>
struct Format<NF_Q_E2M1> {
  static constexpr float top = 1.5f;
  static constexpr int k = 2, bits = 4;
};

// 8 elements to codes: 8 bytes, or 4 of e2m1.  The elements lie within the codes' range after the division by 2^E, an exact
// step down to the codes' own precision.  The conversions round to nearest, ties to even.
template <int F>
__device__ inline void encode8(const float v[8], int E, uint32_t out[2]) {
  float s[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) s[e] = ldexpf(v[e], -E);
  if constexpr (F == NF_Q_INT8) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint32_t w = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) w |= ((uint32_t)(int)rintf(s[4 * h + e]) & 0xFFu) << (8 * e);
      out[h] = w;
    }
  } else if constexpr (F == NF_Q_E4M3) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      int w = __builtin_amdgcn_cvt_pk_fp8_f32(s[4 * h], s[4 * h + 1], 0, false);
      out[h] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(s[4 * h + 2], s[4 * h + 3], w, true);
    }
  } else {
    uint32_t w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, s[0], s[1], 1.f, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, s[2], s[3], 1.f, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, s[4], s[5], 1.f, 2);
    out[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, s[6], s[7], 1.f, 3);
    out[1] = 0;
  }
}

template <int F>
__device__ inline void decode8(const uint32_t in[2], float v[8]) {
  if constexpr (F == NF_Q_INT8) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (float)(int)(int8_t)(in[e >> 2] >> (8 * (e & 3)));
  } else {
    using floatx2 = __attribute__((ext_vector_type(2))) float;
    floatx2 p[4];
    if constexpr (F == NF_Q_E4M3) {
      p[0] = __builtin_amdgcn_cvt_pk_f32_fp8((int)in[0], false), p[1] = __builtin_amdgcn_cvt_pk_f32_fp8((int)in[0], true);
      p[2] = __builtin_amdgcn_cvt_pk_f32_fp8((int)in[1], false), p[3] = __builtin_amdgcn_cvt_pk_f32_fp8((int)in[1], true);
    } else {
      p[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(in[0], 1.f, 0), p[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(in[0], 1.f, 1);
      p[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(in[0], 1.f, 2), p[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(in[0], 1.f, 3);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = p[e >> 1][e & 1];
  }
}

// E + 127, or 255 where a group holds no number.  frexp's exponent is one above that of a mantissa 1 <= m < 2.
template <int F>
__device__ inline int exponent_byte(float amax) {
  if (!(amax < INFINITY)) return 255;
  if (amax == 0.f) return 0;
  int e;
  const float m = 2.f * frexpf(amax, &e);
  e = e - 1 - Format<F>::k + (m > Format<F>::top ? 1 : 0);
  return max(e, -127) + 127;
}

}  // namespace
}  // namespace nf
