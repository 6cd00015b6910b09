// What the kernels of the pointwise layers share: the three element types, vectors of 8 elements at any
// alignment, activations with their slopes, and dropout's random numbers.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "nf_internal.h"

namespace nf {

using floatx4 = __attribute__((ext_vector_type(4))) float;
using uintx4 = __attribute__((ext_vector_type(4))) uint32_t;

// 8 neighbouring elements as fp32.  A row may start at any element: the copies below carry no alignment, and the
// memory system takes 16-byte accesses at element boundaries.
template <typename T>
__device__ inline void load8(const T *p, float v[8]) {
  T t[8];
  __builtin_memcpy(t, p, sizeof(t));
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = (float)t[e];
}
template <typename T>
__device__ inline void store8(T *p, const float v[8]) {
  T t[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) t[e] = (T)v[e];  // to nearest, ties to even
  __builtin_memcpy(p, t, sizeof(t));
}
// the first n of them (n may exceed 8); the others read as 0 and are not written
template <typename T>
__device__ inline void load8(const T *p, float v[8], int n) {
  if (n >= 8) return load8(p, v);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = e < n ? (float)p[e] : 0.f;
}
template <typename T>
__device__ inline void store8(T *p, const float v[8], int n) {
  if (n >= 8) return store8(p, v);
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (e < n) p[e] = (T)v[e];
}

// e^v and 1/v: as accurate as fp32 for fp32 results; two instructions (relative error about 1e-6) where the result is
// rounded to 16 bits, whose half step is 2^-12 or more
template <typename T>
__device__ inline float exp_of(float v) {
  if constexpr (sizeof(T) == 4) return expf(v);
  return __expf(v);
}
template <typename T>
__device__ inline float recip(float v) {
  if constexpr (sizeof(T) == 4) return 1.f / v;
  return __builtin_amdgcn_rcpf(v);
}

// The normal distribution's tail Q(|z|) = erfc(|z| / sqrt 2) / 2 and e^(-z^2 / 2).  erfc(x) = t e^(-x^2) P(t) with
// t = 1 / (1 + 0.45 x); P is a minimax fit of degree 9 of erfc(x) e^(x^2) / t over 0 <= x <= 12 (relative error 1.6e-8,
// 1.2e-7 with its fp32 evaluation; beyond 12 e^(-x^2) is 0 in fp32).
template <typename T>
__device__ inline float normal_tail(float z, float &bell) {
  const float x = fabsf(z) * 0.70710678118654752f;
  const float t = recip<T>(fmaf(0.45f, x, 1.f));
  float P = -0.03643337f;
  P = fmaf(P, t, 0.16440561f);
  P = fmaf(P, t, -0.24082965f);
  P = fmaf(P, t, 0.06623675f);
  P = fmaf(P, t, 0.03736064f);
  P = fmaf(P, t, 0.09022658f);
  P = fmaf(P, t, 0.184595f);
  P = fmaf(P, t, 0.22649258f);
  P = fmaf(P, t, 0.25406855f);
  P = fmaf(P, t, 0.25387729f);
  bell = exp_of<T>(-0.5f * z * z);
  return 0.5f * t * bell * P;
}

// The activation of N values, and its slope at them (times what s holds).  The activation is the same for a whole launch: one
// branch to a vector, not to an element.
template <typename T, int N>
__device__ inline void act_of(int act, float (&v)[N]) {
  if (act == NF_ACT_RELU) {
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = v[e] < 0.f ? 0.f : v[e];  // a NaN stays one
  } else if (act == NF_ACT_SILU) {
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] *= recip<T>(1.f + exp_of<T>(-v[e]));
  } else if (act == NF_ACT_GELU) {
#pragma unroll
    for (int e = 0; e < N; ++e) {
      float bell;
      const float q = normal_tail<T>(v[e], bell);
      v[e] *= v[e] > 0.f ? 1.f - q : q;
    }
  }
}

template <typename T, int N>
__device__ inline void times_slope(int act, const float (&z)[N], float (&s)[N]) {
  if (act == NF_ACT_RELU) {
#pragma unroll
    for (int e = 0; e < N; ++e) s[e] = z[e] > 0.f ? s[e] : 0.f;
  } else if (act == NF_ACT_SILU) {
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const float q = recip<T>(1.f + exp_of<T>(-z[e]));
      s[e] *= q * (1.f + z[e] * (1.f - q));
    }
  } else if (act == NF_ACT_GELU) {
#pragma unroll
    for (int e = 0; e < N; ++e) {
      float bell;
      const float q = normal_tail<T>(z[e], bell);
      s[e] *= (z[e] > 0.f ? 1.f - q : q) + z[e] * bell * 0.39894228040143268f;
    }
  }
}

// Dropout as the kernels take it: T = 0 means none.
struct DropArgs {
  uint32_t T;
  float scale;
  uint32_t k0, k1, s0, s1;
};
DropArgs drop_args(const nf_dropout_desc *d);  // d may be null; checked already

// Philox4x32-10 at counter (group, step): the half words of the 8 elements of a group, two to a word.  A round is two
// 32x32 -> 64 products (quarter rate) and two three-way xors, about 440 cycles of a wave per 512 elements: a chip that streams
// bf16 rows at 5 TB/s spends a third of its vector cycles here.
__device__ inline void philox8(const DropArgs &d, unsigned long long group, uint32_t w[4]) {
  uint32_t a = (uint32_t)group, b = (uint32_t)(group >> 32), c = d.s0, e = d.s1, k0 = d.k0, k1 = d.k1;
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const unsigned long long p = (unsigned long long)a * 0xD2511F53u, q = (unsigned long long)c * 0xCD9E8D57u;
    a = (uint32_t)(q >> 32) ^ b ^ k0, b = (uint32_t)q;
    c = (uint32_t)(p >> 32) ^ e ^ k1, e = (uint32_t)p;
    k0 += 0x9E3779B9u, k1 += 0xBB67AE85u;
  }
  w[0] = a, w[1] = b, w[2] = c, w[3] = e;
}

// D of 8 elements of one group, in place.  A dropped element is 0 whatever it was.
__device__ inline void drop8(const DropArgs &d, unsigned long long group, float v[8]) {
  if (!d.T) return;
  uint32_t w[4];
  philox8(d, group, w);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t u = (e & 1) ? w[e >> 1] >> 16 : w[e >> 1] & 0xFFFFu;
    v[e] = u >= d.T ? v[e] * d.scale : 0.f;
  }
}

// ---- launches (sizes and pointers checked already) ----
hipError_t launch_dropout(const DropArgs &d, int dtype, long long rows, long long cols, const void *x, const void *r,
                          void *y, hipStream_t st);

struct QcacheRows {
  uint8_t *codes, *scales;
  int32_t *labels;
  long long capacity, n, first;
  long long code_bytes, scale_bytes;
};
void qcache_row_bytes(int format, long long n, long long *code_bytes, long long *scale_bytes);
hipError_t launch_qcache_write(int format, int dtype, const QcacheRows &q, int B, const void *x, const int32_t *labels,
                               hipStream_t st);
hipError_t launch_qcache_read(int format, int dtype, const QcacheRows &q, const long long *idx, int B, void *x,
                              int32_t *labels, hipStream_t st);

struct GnShape {
  int dtype, B, HW, C, G, act;
  float eps;
};
size_t gn_workspace_bytes(const GnShape &s);
hipError_t launch_gn_fwd(const GnShape &s, const void *x, const float *gamma, const float *beta, void *y, float *mean,
                         float *rstd, void *ws, hipStream_t st);
hipError_t launch_gn_bwd(const GnShape &s, const void *dy, const void *x, const float *gamma, const float *beta,
                         const float *mean, const float *rstd, void *dx, float *dgamma, float *dbeta, void *ws,
                         hipStream_t st);

struct LinearCall {
  int dtype, act;
  long long M;
  int K, N;
};
size_t linear_workspace_bytes(const LinearCall &c);
hipError_t launch_linear_fwd(const LinearCall &c, const void *x, const void *W, const float *b, const void *r,
                             const DropArgs &drop, void *y, void *z, void *ws, hipStream_t st);
hipError_t launch_linear_epilogue(const LinearCall &c, const void *dy, const void *z, const DropArgs &drop, void *dz,
                                  float *db, void *ws, hipStream_t st);
hipError_t launch_linear_bwd(const LinearCall &c, const void *dz, const void *x, const void *W, void *dx, float *dW,
                             void *ws, hipStream_t st);

}  // namespace nf
