// Group norm over channels-last activations with an activation behind it, forward and backward.
//
// A workgroup takes one image's slab of W neighbouring channels (whole groups, VEC of them to a vector): a thread keeps
// one vector of channels and walks the pixels, so that sums per channel stay in registers until the slab is done.  The
// slab is read again for the next pass (mean, squares about the mean, result): its second and third reading come from the
// caches.
#include "pw_math.h"

namespace nf {
namespace {

// The 16 bytes of VEC neighbouring elements.  Where rows are not whole vectors (WHOLE false), they start at any element and
// the slab's last vector has n of them; the others read as 0 and are not written.
template <typename T>
struct Vec {
  static constexpr int N = 16 / sizeof(T);
  T v[N];
};
template <typename T, bool WHOLE>
__device__ inline Vec<T> load_vec(const T *p, int n) {
  Vec<T> t;
  if (WHOLE)
    __builtin_memcpy(&t, __builtin_assume_aligned(p, 16), 16);
  else if (n >= Vec<T>::N)
    __builtin_memcpy(&t, p, 16);
  else
#pragma unroll
    for (int e = 0; e < Vec<T>::N; ++e) t.v[e] = e < n ? p[e] : (T)0.f;
  return t;
}
template <typename T, bool WHOLE>
__device__ inline void store_vec(T *p, const Vec<T> &t, int n) {
  if (WHOLE)
    __builtin_memcpy(__builtin_assume_aligned(p, 16), &t, 16);
  else if (n >= Vec<T>::N)
    __builtin_memcpy(p, &t, 16);
  else
#pragma unroll
    for (int e = 0; e < Vec<T>::N; ++e)
      if (e < n) p[e] = t.v[e];
}

struct GnArgs {
  int HW, C, G, Cg, W, Wp;  // W: channels of a slab, Wp: in whole vectors
  int cv, px;               // vectors across a slab, pixels that the workgroup takes at once
  int act;
  float eps;
};

// Sums over the slab's pixels of every channel, from the threads' own sums: csum[Wp].  buf holds NT * VEC floats.
template <int VEC, int NT>
__device__ inline void channel_sums(const GnArgs &a, const float s[VEC], float *buf, float *csum) {
  const int t = threadIdx.x;
  __syncthreads();  // buf and csum may still be read
  if (t < a.cv * a.px) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) buf[t * VEC + e] = s[e];  // [pixel][channel]
  }
  __syncthreads();
  const int P = a.Wp < NT ? min(a.px, NT / a.Wp) : 1;
  if (P > 1) {  // threads share a channel's sum
    const int p = t / a.Wp, c = t - p * a.Wp;
    float sum = 0.f;
    if (p < P)
      for (int q = p; q < a.px; q += P) sum += buf[q * a.Wp + c];
    __syncthreads();
    if (p < P) buf[p * a.Wp + c] = sum;
    __syncthreads();
  }
  const int rows = P > 1 ? P : a.px;
  for (int c = t; c < a.Wp; c += NT) {
    float sum = 0.f;
    for (int q = 0; q < rows; ++q) sum += buf[q * a.Wp + c];
    csum[c] = sum;
  }
  __syncthreads();
}

// sum over each group of the slab of csum[c] (times w[c], where given), for gsum[W / Cg]
template <int NT>
__device__ inline void group_sums(const GnArgs &a, const float *csum, const float *w, float *gsum) {
  const int lane = threadIdx.x & 63;
  for (int g = threadIdx.x >> 6; g < a.W / a.Cg; g += NT / 64) {
    float sum = 0.f;
    for (int c = lane; c < a.Cg; c += 64) sum += w ? csum[g * a.Cg + c] * w[g * a.Cg + c] : csum[g * a.Cg + c];
#pragma unroll
    for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
    if (lane == 0) gsum[g] = sum;
  }
  __syncthreads();
}

// HBM-bound: 2 * sizeof(T) bytes an element.
template <typename T, bool WHOLE, int NT>
__global__ __launch_bounds__(NT) void gn_fwd_kernel(GnArgs a, const T *__restrict__ x, const float *__restrict__ gamma,
                                                    const float *__restrict__ beta, T *__restrict__ y,
                                                    float *__restrict__ mean, float *__restrict__ rstd) {
  constexpr int VEC = Vec<T>::N;
  extern __shared__ float lds[];
  float *buf = lds, *csum = buf + NT * VEC, *gsum = csum + a.Wp;  // gsum [2][groups]: means, reciprocal deviations
  const int t = threadIdx.x, b = blockIdx.y, c0 = blockIdx.x * a.W, groups = a.W / a.Cg;
  const int pr = t / a.cv, cl = (t - pr * a.cv) * VEC;
  const bool live = pr < a.px;
  const int n = a.W - cl;  // the slab's channels from here on
  const T *const src = x + ((long long)b * a.HW + pr) * a.C + c0 + cl;
  T *const dst = y + ((long long)b * a.HW + pr) * a.C + c0 + cl;
  const long long step = (long long)a.px * a.C;
  const int mine = live ? (a.HW - pr + a.px - 1) / a.px : 0;
  const float inv = 1.f / ((float)a.Cg * (float)a.HW);
  float s[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) s[e] = 0.f;
  for (int i = 0; i < mine; ++i) {
    const Vec<T> v = load_vec<T, WHOLE>(src + i * step, n);
#pragma unroll
    for (int e = 0; e < VEC; ++e) s[e] += (float)v.v[e];
  }
  channel_sums<VEC, NT>(a, s, buf, csum);
  group_sums<NT>(a, csum, nullptr, gsum);
  float mu[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) mu[e] = live && e < n ? gsum[(cl + e) / a.Cg] * inv : 0.f, s[e] = 0.f;
  for (int i = 0; i < mine; ++i) {
    const Vec<T> v = load_vec<T, WHOLE>(src + i * step, n);
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const float d = (float)v.v[e] - mu[e];
      s[e] = fmaf(d, d, s[e]);
    }
  }
  channel_sums<VEC, NT>(a, s, buf, csum);
  group_sums<NT>(a, csum, nullptr, gsum + groups);
  for (int g = t; g < groups; g += NT) {
    const long long o = (long long)b * a.G + c0 / a.Cg + g;
    const float r = 1.f / sqrtf(gsum[groups + g] * inv + a.eps);
    mean[o] = gsum[g] * inv, rstd[o] = r;
    gsum[groups + g] = r;
  }
  __syncthreads();
  if (!live) return;
  float k[VEC], be[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
    k[e] = be[e] = 0.f;
    if (e < n) k[e] = gsum[groups + (cl + e) / a.Cg] * gamma[c0 + cl + e], be[e] = beta[c0 + cl + e];
  }
  for (int i = 0; i < mine; ++i) {
    Vec<T> v = load_vec<T, WHOLE>(src + i * step, n);
#pragma unroll
    for (int e = 0; e < VEC; ++e) v.v[e] = (T)act_of<T>(a.act, fmaf((float)v.v[e] - mu[e], k[e], be[e]));
    store_vec<T, WHOLE>(dst + i * step, v, n);
  }
}

// dy * act'(z) of one element.  The sign of a rectified z next to 0 decides whether dy counts: there z is formed again in 64
// bits from the same fp32 numbers.
template <typename T>
__device__ inline float gated(int act, float dy, float x, float mu, float rs, float xh, float ga, float be) {
  const float z = fmaf(xh, ga, be);
  if (act == NF_ACT_RELU) {
    bool on = z > 0.f;
    if (fabsf(z) <= 1e-5f * (fabsf(xh * ga) + fabsf(be)))  // fp32's z is off by a few 2^-24 of its terms, and x - mean exact or better
      on = ((double)x - (double)mu) * (double)rs * (double)ga + (double)be > 0.0;
    return on ? dy : 0.f;
  }
  return dy * act_slope<T>(act, z);
}

// HBM-bound: 3 * sizeof(T) bytes an element.  part [image][2][C]: sums over the image's pixels of g xh and g.
template <typename T, bool WHOLE, int NT>
__global__ __launch_bounds__(NT) void gn_bwd_kernel(GnArgs a, const T *__restrict__ dy, const T *__restrict__ x,
                                                    const float *__restrict__ gamma, const float *__restrict__ beta,
                                                    const float *__restrict__ mean, const float *__restrict__ rstd,
                                                    T *__restrict__ dx, float *__restrict__ part) {
  constexpr int VEC = Vec<T>::N;
  extern __shared__ float lds[];
  float *buf = lds, *csum = buf + NT * VEC, *csumx = csum + a.Wp, *gsum = csumx + a.Wp;  // gsum [2][groups]
  const int t = threadIdx.x, b = blockIdx.y, c0 = blockIdx.x * a.W, groups = a.W / a.Cg;
  const int pr = t / a.cv, cl = (t - pr * a.cv) * VEC;
  const bool live = pr < a.px;
  const int n = a.W - cl;  // the slab's channels from here on
  const long long at = ((long long)b * a.HW + pr) * a.C + c0 + cl;
  const long long step = (long long)a.px * a.C;
  const int mine = live ? (a.HW - pr + a.px - 1) / a.px : 0;
  const float inv = 1.f / ((float)a.Cg * (float)a.HW);
  float mu[VEC], rs[VEC], ga[VEC], be[VEC], s[VEC], sx[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
    s[e] = sx[e] = 0.f;
    mu[e] = rs[e] = ga[e] = be[e] = 0.f;
    if (live && e < n) {
      const long long o = (long long)b * a.G + (c0 + cl + e) / a.Cg;
      mu[e] = mean[o], rs[e] = rstd[o], ga[e] = gamma[c0 + cl + e], be[e] = beta[c0 + cl + e];
    }
  }
  for (int i = 0; i < mine; ++i) {
    const Vec<T> v = load_vec<T, WHOLE>(x + at + i * step, n), d = load_vec<T, WHOLE>(dy + at + i * step, n);
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const float xh = ((float)v.v[e] - mu[e]) * rs[e];
      const float g = gated<T>(a.act, (float)d.v[e], (float)v.v[e], mu[e], rs[e], xh, ga[e], be[e]);
      s[e] += g, sx[e] = fmaf(g, xh, sx[e]);
    }
  }
  channel_sums<VEC, NT>(a, s, buf, csum);
  channel_sums<VEC, NT>(a, sx, buf, csumx);
  group_sums<NT>(a, csum, gamma + c0, gsum);
  group_sums<NT>(a, csumx, gamma + c0, gsum + groups);
  for (int c = t; c < a.W; c += NT) {
    part[((long long)b * 2 + 0) * a.C + c0 + c] = csumx[c];
    part[((long long)b * 2 + 1) * a.C + c0 + c] = csum[c];
  }
  if (!live) return;
  float m1[VEC], m2[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
    const int g = min(cl + e, a.W - 1) / a.Cg;
    m1[e] = gsum[g] * inv, m2[e] = gsum[groups + g] * inv;
  }
  for (int i = 0; i < mine; ++i) {
    Vec<T> v = load_vec<T, WHOLE>(x + at + i * step, n);
    const Vec<T> d = load_vec<T, WHOLE>(dy + at + i * step, n);
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const float xh = ((float)v.v[e] - mu[e]) * rs[e];
      const float g = gated<T>(a.act, (float)d.v[e], (float)v.v[e], mu[e], rs[e], xh, ga[e], be[e]);
      v.v[e] = (T)(rs[e] * (fmaf(g, ga[e], -m1[e]) - xh * m2[e]));
    }
    store_vec<T, WHOLE>(dx + at + i * step, v, n);
  }
}

// dgamma[c] and dbeta[c]: sums over the images, 16 rows of threads to 16 columns, in a fixed order
constexpr int RT = 256;
__global__ __launch_bounds__(RT) void gn_params_kernel(const float *__restrict__ part, int B, int C,
                                                       float *__restrict__ dgamma, float *__restrict__ dbeta) {
  __shared__ float s[16][17];
  const int c = blockIdx.x * 16 + (threadIdx.x & 15), r = threadIdx.x >> 4;  // columns of [2][C]
  float sum = 0.f;
  if (c < 2 * C)
    for (int b = r; b < B; b += 16) sum += part[(long long)b * 2 * C + c];
  s[r][threadIdx.x & 15] = sum;
  __syncthreads();
  if (r == 0 && c < 2 * C) {
#pragma unroll
    for (int q = 1; q < 16; ++q) sum += s[q][threadIdx.x];
    if (c < C)
      dgamma[c] = sum;
    else
      dbeta[c - C] = sum;
  }
}

int gcd(int a, int b) {
  while (b) {
    const int t = a % b;
    a = b, b = t;
  }
  return a;
}

constexpr int NT = 1024;

// Channels of a slab: whole groups and, where rows are whole vectors, whole vectors; 64 bytes of a pixel or more where there are
// that many.  A slab is at most 2048 channels (16 KB of sums): wider units of groups and vectors give way to single groups.
GnArgs gn_args(const GnShape &s, bool *whole) {
  const int size = s.dtype == NF_F32 ? 4 : 2, vec = 16 / size;
  GnArgs a;
  a.HW = s.HW, a.C = s.C, a.G = s.G, a.Cg = s.C / s.G, a.act = s.act, a.eps = s.eps;
  const int unit = a.Cg / gcd(a.Cg, vec) * vec;
  *whole = s.C % vec == 0 && unit <= 2048;
  a.W = *whole ? unit : a.Cg;
  while (a.W < 64 / size && s.C % (2 * a.W) == 0) a.W *= 2;
  a.cv = (a.W + vec - 1) / vec, a.Wp = a.cv * vec, a.px = NT / a.cv;
  return a;
}

template <typename T>
hipError_t fwd_as(const GnShape &s, const void *x, const float *gamma, const float *beta, void *y, float *mean,
                  float *rstd, hipStream_t st) {
  bool whole;
  const GnArgs a = gn_args(s, &whole);
  const size_t lds = 4 * ((size_t)NT * Vec<T>::N + a.Wp + 2 * (a.W / a.Cg));
  const dim3 grid(s.C / a.W, s.B);
  if (whole)
    hipLaunchKernelGGL((gn_fwd_kernel<T, true, NT>), grid, dim3(NT), lds, st, a, (const T *)x, gamma, beta, (T *)y, mean, rstd);
  else
    hipLaunchKernelGGL((gn_fwd_kernel<T, false, NT>), grid, dim3(NT), lds, st, a, (const T *)x, gamma, beta, (T *)y, mean, rstd);
  return hipGetLastError();
}
template <typename T>
hipError_t bwd_as(const GnShape &s, const void *dy, const void *x, const float *gamma, const float *beta,
                  const float *mean, const float *rstd, void *dx, float *part, hipStream_t st) {
  bool whole;
  const GnArgs a = gn_args(s, &whole);
  const size_t lds = 4 * ((size_t)NT * Vec<T>::N + 2 * a.Wp + 2 * (a.W / a.Cg));
  const dim3 grid(s.C / a.W, s.B);
  if (whole)
    hipLaunchKernelGGL((gn_bwd_kernel<T, true, NT>), grid, dim3(NT), lds, st, a, (const T *)dy, (const T *)x, gamma, beta, mean, rstd, (T *)dx, part);
  else
    hipLaunchKernelGGL((gn_bwd_kernel<T, false, NT>), grid, dim3(NT), lds, st, a, (const T *)dy, (const T *)x, gamma, beta, mean, rstd, (T *)dx, part);
  return hipGetLastError();
}

}  // namespace

size_t gn_workspace_bytes(const GnShape &s) { return (size_t)s.B * 2 * s.C * 4; }

hipError_t launch_gn_fwd(const GnShape &s, const void *x, const float *gamma, const float *beta, void *y, float *mean,
                         float *rstd, void *ws, hipStream_t st) {
  if (s.dtype == NF_BF16) return fwd_as<__bf16>(s, x, gamma, beta, y, mean, rstd, st);
  if (s.dtype == NF_F16) return fwd_as<_Float16>(s, x, gamma, beta, y, mean, rstd, st);
  return fwd_as<float>(s, x, gamma, beta, y, mean, rstd, st);
}

hipError_t launch_gn_bwd(const GnShape &s, const void *dy, const void *x, const float *gamma, const float *beta,
                         const float *mean, const float *rstd, void *dx, float *dgamma, float *dbeta, void *ws,
                         hipStream_t st) {
  float *part = (float *)ws;
  const hipError_t e = s.dtype == NF_BF16  ? bwd_as<__bf16>(s, dy, x, gamma, beta, mean, rstd, dx, part, st)
                       : s.dtype == NF_F16 ? bwd_as<_Float16>(s, dy, x, gamma, beta, mean, rstd, dx, part, st)
                                           : bwd_as<float>(s, dy, x, gamma, beta, mean, rstd, dx, part, st);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(gn_params_kernel, dim3((2 * s.C + 15) / 16), dim3(RT), 0, st, part, s.B, s.C, dgamma, dbeta);
  return hipGetLastError();
}

}  // namespace nf
