// What the kernels of the pointwise layers share: the three element types, vectors of 8 elements at any
// alignment, activations with their slopes, and dropout's random numbers.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "nf_internal.h"

namespace nf {

using floatx4 = __attribute__((ext_vector_type(4))) float;
using uintx4 = __attribute__((ext_vector_type(4))) uint32_t;

// 8 neighbouring elements as fp32.  A row may start at any element: the copies below carry no alignment, and the memory
// system takes 16-byte accesses at element boundaries.
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
  uintx4 w[sizeof(T) / 2];
  __builtin_memcpy(w, t, sizeof(t));
  // whole: the compiler would share the first elements' store with the branch that writes fewer, and split this one
#pragma unroll
  for (int i = 0; i < (int)(sizeof(T) / 2); ++i) asm volatile("" : "+v"(w[i]));
  __builtin_memcpy(p, w, sizeof(w));
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

// 8 elements as they lie in memory: half the registers of their fp32 forms for a 16-bit type.  unpack8 hides them from the
// compiler, which would convert them as soon as they arrive.
template <typename T>
struct Raw8 {
  uintx4 w[sizeof(T) / 2];
};
template <typename T>
__device__ inline Raw8<T> raw8(const T *p, int n) {
  Raw8<T> r;
  if (n >= 8) {
    __builtin_memcpy(&r, p, sizeof(r));
    asm volatile("");  // a branch of its own: its reads stay whole
  } else {
    T t[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) t[e] = e < n ? p[e] : (T)0.f;
    __builtin_memcpy(&r, t, sizeof(r));
  }
  return r;
}
template <typename T>
__device__ inline void unpack8(Raw8<T> r, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < (int)(sizeof(T) / 2); ++i) asm volatile("" : "+v"(r.w[i]));
  T t[8];
  __builtin_memcpy(t, &r, sizeof(r));
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = (float)t[e];
}

// e^v and 1/v: as accurate as fp32 for fp32 results; two instructions and one (e^v off by up to (|v| + 1) 2^-23 of itself, 1/v by 2^-23) where
// the result is rounded to 16 bits, whose half step is 2^-11 or more
template <typename T>
__device__ inline float exp_of(float v) {
  if constexpr (sizeof(T) == 4) return expf(v);
  return __builtin_amdgcn_exp2f(v * 1.4426950408889634f);
}
template <typename T>
__device__ inline float recip(float v) {
  if constexpr (sizeof(T) == 4) return 1.f / v;
  return __builtin_amdgcn_rcpf(v);
}

// The normal distribution's tail Q(|z|) = erfc(|z| / sqrt 2) / 2 in its factors: Q = t bell P(t), bell = e^(-z^2 / 2), t = 1 / (1 + c |z|),
// P a minimax fit of Q / (t bell), which is returned.  fp32: c = 0.45 / sqrt 2, degree 9, |z| up to 17 (relative error 1.6e-8, 1.2e-7 with its
// evaluation; beyond 17 the bell is 0 in fp32).  Results of 16 bits: c = 0.3, degree 5, |z| up to 9 (2.1e-6; beyond, Q is below
// 1e-19).  Slopes take the first form (FINE), since their sums are fp32 results.
template <typename T, bool FINE>
__device__ inline float normal_tail(float z, float &bell, float &t) {
  if constexpr (sizeof(T) == 4 || FINE) {
    t = recip<T>(fmaf(0.31819805153394639f, fabsf(z), 1.f));
    float P = -0.018216685f;
    P = fmaf(P, t, 0.082202805f);
    P = fmaf(P, t, -0.120414825f);
    P = fmaf(P, t, 0.033118375f);
    P = fmaf(P, t, 0.01868032f);
    P = fmaf(P, t, 0.04511329f);
    P = fmaf(P, t, 0.0922975f);
    P = fmaf(P, t, 0.11324629f);
    P = fmaf(P, t, 0.127034275f);
    P = fmaf(P, t, 0.126938645f);
    bell = sizeof(T) == 4 ? expf(-0.5f * z * z) : __builtin_amdgcn_exp2f(z * z * -0.72134752044448170f);
    return P;
  } else {
    t = __builtin_amdgcn_rcpf(fmaf(0.3f, fabsf(z), 1.f));
    float P = -0.08183746907f;
    P = fmaf(P, t, 0.23058672288f);
    P = fmaf(P, t, -0.03403829558f);
    P = fmaf(P, t, 0.15375138749f);
    P = fmaf(P, t, 0.11121039917f);
    P = fmaf(P, t, 0.12032773274f);
    bell = __builtin_amdgcn_exp2f(z * z * -0.72134752044448170f);
    return P;
  }
}

// v f where 0 times anything is 0: an activation's vanishing factor (q, the bell) holds against an infinite v or e^-v, so that
// infinities give the limits (activations inf and 0, slopes 1 and 0) and not 0 * inf.  A NaN is one in both factors and stays.
__device__ float mul_legacy(float, float) __asm("llvm.amdgcn.fmul.legacy");
__device__ inline float fading(float v, float f) { return mul_legacy(v, f); }

// The activation of N values, and its slope at them (times what s holds).  The activation is the same for a whole launch: one
// branch to a vector, not to an element.
template <typename T, int N>
__device__ inline void act_of(int act, float (&v)[N]) {
  if (act == NF_ACT_RELU) {
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = v[e] < 0.f ? 0.f : v[e];  // a NaN stays one
  } else if (act == NF_ACT_SILU) {
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = fading(v[e], recip<T>(1.f + exp_of<T>(-v[e])));
  } else if (act == NF_ACT_GELU) {
#pragma unroll
    for (int e = 0; e < N; ++e) {  // v Phi(v) = max(v, 0) - |v| Q(|v|); a NaN stays one through Q
      float bell, t;
      const float P = normal_tail<T, false>(v[e], bell, t);
      const float up = __builtin_bit_cast(float, max(__builtin_bit_cast(int, v[e]), 0));  // max(v, 0) in one instruction
      v[e] = fmaf(-fading(fabsf(v[e]), bell) * t, P, up);
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
    for (int e = 0; e < N; ++e) {  // q + z q (1 - q), q = 1 / (1 + a), a = e^-z; 1 - q is a q, which keeps its digits where q is next to 1
      const float a = exp_of<T>(-z[e]), q = recip<T>(1.f + a);
      s[e] *= fmaf(fading(z[e], fading(a, q)), q, q);
    }
  } else if (act == NF_ACT_GELU) {
#pragma unroll
    for (int e = 0; e < N; ++e) {
      float bell, t;
      const float P = normal_tail<T, true>(z[e], bell, t), Q = t * bell * P;
      s[e] *= fmaf(fading(z[e], bell), 0.39894228040143268f, z[e] > 0.f ? 1.f - Q : Q);
    }
  }
}

// Dropout as the kernels take it: T = 0 (and scale 1) means none.
struct DropArgs {
  uint32_t T;
  float scale;
  uint32_t k0, k1, s0, s1;
};
DropArgs drop_args(const nf_dropout_desc *d);  // d may be null; checked already

// Philox4x32-10 at counter (group, step): the half words of the 8 elements of a group, two to a word.  A round is two
// 32x32 -> 64 products (quarter rate) and two three-way xors, 10 cycles of the vector ALU an element's wave-instruction in all: a
// chip that streams bf16 rows at 5 TB/s spends a third of its vector cycles here.
__device__ inline void philox8(const DropArgs &d, unsigned long long group, uint32_t w[4]) {
  uint32_t a = (uint32_t)group, b = (uint32_t)(group >> 32), c = d.s0, e = d.s1, k0 = d.k0, k1 = d.k1;
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const unsigned long long p = (unsigned long long)a * 0xD2511F53u, q = (unsigned long long)c * 0xCD9E8D57u;
    a = __builtin_amdgcn_bitop3_b32((uint32_t)(q >> 32), b, k0, 0x96), b = (uint32_t)q;  // 0x96: the xor of three
    c = __builtin_amdgcn_bitop3_b32((uint32_t)(p >> 32), e, k1, 0x96), e = (uint32_t)p;
    k0 += 0x9E3779B9u, k1 += 0xBB67AE85u;
  }
  w[0] = a, w[1] = b, w[2] = c, w[3] = e;
}

// Zeros for the dropped of 8 elements of one group, in place, whatever they were; the others are left for `scale`.
__device__ inline void drop8(const DropArgs &d, unsigned long long group, float (&v)[8]) {
  if (!d.T) return;
  uint32_t w[4];
  philox8(d, group, w);
  const uint32_t high = d.T << 16;  // u >= T for the half words as they lie: high ones compare whole
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = ((e & 1) ? w[e >> 1] : w[e >> 1] << 16) >= high ? v[e] : 0.f;
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
size_t gn_fwd_workspace_bytes(const GnShape &s);
hipError_t launch_gn_fwd(const GnShape &s, const void *x, const float *gamma, const float *beta, void *y, float *mean,
                         float *rstd, void *ws, hipStream_t st);
hipError_t launch_gn_bwd(const GnShape &s, const void *dy, const void *x, const float *gamma, const float *beta,
                         const float *mean, const float *rstd, void *dx, float *dgamma, float *dbeta, void *ws,
                         hipStream_t st);

struct LnShape {
  int dtype;
  long long M;
  int C;
  float eps;
};
size_t ln_workspace_bytes(const LnShape &s);
hipError_t launch_ln_fwd(const LnShape &s, const void *x, const float *gamma, const float *beta, void *y, float *mean, float *rstd, hipStream_t st);
hipError_t launch_ln_bwd(const LnShape &s, const void *dy, const void *x, const float *gamma, const float *mean, const float *rstd, const void *dr, void *dx,
                         float *dgamma, float *dbeta, void *ws, hipStream_t st);

struct LinearCall {
  int dtype, act;
  long long M;
  int K, N;
};
size_t linear_workspace_bytes(const LinearCall &c);
size_t linear_fwd_workspace_bytes(const LinearCall &c);
hipError_t launch_linear_fwd(const LinearCall &c, const void *x, const void *W, const float *b, const void *r,
                             const DropArgs &drop, void *y, void *z, void *ws, hipStream_t st);
hipError_t launch_linear_epilogue(const LinearCall &c, const void *dy, const void *z, const DropArgs &drop, void *dz,
                                  float *db, void *ws, hipStream_t st);
hipError_t launch_linear_bwd(const LinearCall &c, const void *dz, const void *x, const void *W, void *dx, float *dW,
                             void *ws, hipStream_t st);

struct MxRows {
  uint8_t *codes, *scales;
  long long cb, sb;  // row strides
};
struct MxCall {
  int dtype, act;
  long long M;
  int N;
  long long K;
};
bool mx_quantise_fits(long long rows, long long cols, bool by_columns);
hipError_t launch_mx_quantise(int dtype, long long rows, long long cols, const void *x, void *codes, void *scales, void *codes_t, void *scales_t, hipStream_t st);
size_t mx_product_workspace_bytes(const MxCall &c);
size_t mx_linear_workspace_bytes(const MxCall &c);
hipError_t launch_mx_product(const MxCall &c, const void *a, const void *as, const void *b, const void *bs, const float *bias, const void *r, const DropArgs &drop,
                             void *y, void *z, void *ws, hipStream_t st);
hipError_t launch_mx_linear(const MxCall &c, const void *x, const void *W, const void *Ws, const float *bias, const void *r, const DropArgs &drop, void *y, void *z,
                            void *ws, hipStream_t st);

}  // namespace nf
