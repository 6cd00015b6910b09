// Group norm with an activation, backward.  gn.h holds the slabs and their sums.
#include "gn.h"

namespace nf {
namespace {

// (x - mu) rs gamma + beta, k = rs gamma rounded, in two fp32 numbers: the roundings of sums and products are carried along.
// Its sign, which decides whether a rectified element's dy counts, is right down to 2^-44 of the terms.
__device__ inline float careful_z(float x, float mu, float rs, float gamma, float k, float beta) {
#pragma clang fp contract(off)
  const float d = x - mu, back = d - x, dl = (x - (d - back)) - (mu + back);
  const float t = d * k, kl = fmaf(rs, gamma, -k);
  const float tl = fmaf(d, k, -t) + fmaf(d, kl, dl * k);
  const float sum = t + beta, from = sum - t;
  return sum + (((t - (sum - from)) + (beta - from)) + tl);
}

// HBM-bound: 3 * sizeof(T) bytes an element.  part [image * chunks + chunk][2][C]: sums over pixels of g xh and g.
template <typename T, bool WHOLE, bool ONE, int MODE, int R, int NTMAX>
__global__ __launch_bounds__(NTMAX) void gn_bwd_kernel(GnArgs a, const T *__restrict__ dy, const T *__restrict__ x,
                                                       const float *__restrict__ gamma, const float *__restrict__ beta,
                                                       const float *__restrict__ mean, const float *__restrict__ rstd,
                                                       T *__restrict__ dx, float *__restrict__ part) {
  constexpr int VEC = Vec<T>::N, PV = ONE ? 1 : VEC;  // mean and deviation: one for the vector, or one per channel
  extern __shared__ float lds[];
  const int pitch = 2 * a.W + 1;
  float *const buf = lds, *const csum = buf + (MODE == APPLY ? 0 : a.px * pitch), *const gsum = csum + 2 * a.W;
  const int t = threadIdx.x;
  const int slabs = a.div_slabs.d;
  const int id = xcd_run(blockIdx.x, gridDim.x), bc = a.div_slabs.div(id), slab = id - bc * slabs;
  const int b = MODE == FUSED ? bc : (int)a.div_chunks.div(bc), chunk = MODE == FUSED ? 0 : bc - b * a.chunks;
  const int c0 = slab * a.W, p0 = chunk * a.per, p1 = min(a.HW, p0 + a.per);
  const int pr = a.div_cv.div(t), cl = (t - pr * a.cv) * VEC, n = a.W - cl;
  const bool live = pr < a.px;
  // offsets within the slab fit 32 bits (gn_plan)
  const long long first = ((long long)b * a.HW + p0) * a.C + c0;
  const char *const xs = (const char *)(x + first), *const ds = (const char *)(dy + first);
  char *const dst = (char *)(dx + first);
  const uint32_t off = (uint32_t)((pr * a.C + cl) * (int)sizeof(T)), step = (uint32_t)(a.px * a.C * (int)sizeof(T));
  const int mine = live ? (int)a.div_px.div(p1 - p0 - pr + a.px - 1) : 0;
  uintx4 v[R], d[R];
#pragma unroll
  for (int i = 0; i < R; ++i)
    if (i < mine) v[i] = load_vec<T, WHOLE>((const T *)(xs + (off + i * step)), n), d[i] = load_vec<T, WHOLE>((const T *)(ds + (off + i * step)), n);
  auto group_of = [&](int e) { return ONE ? (int)a.div_cg.div(cl) : (int)a.div_cg.div(WHOLE ? cl + e : min(cl + e, a.W - 1)); };
  const long long first_group = (long long)b * a.G + slab * a.groups;
  float mu[PV], k[VEC], be[VEC];  // k = rs gamma
#pragma unroll
  for (int e = 0; e < PV; ++e) mu[e] = live ? mean[first_group + group_of(e)] : 0.f;
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
    k[e] = be[e] = 0.f;
    if (live && (WHOLE || e < n)) k[e] = rstd[first_group + group_of(e)] * gamma[c0 + cl + e], be[e] = beta[c0 + cl + e];
  }
  // of 4 elements of the vector at pixel i: xc = x - mu and g = dy act'(z), z = xc k + beta
  auto grad = [&](int i, int h, float (&xc)[4], float (&g)[4]) {
    float z[4];
    unpack4<T>(v[i], h, xc), unpack4<T>(d[i], h, g);
    if (a.act == NF_ACT_RELU) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int q = 4 * h + e;
        const float ga = WHOLE || q < n ? gamma[c0 + cl + q] : 0.f, rs = live ? rstd[first_group + group_of(q)] : 0.f;
        z[e] = careful_z(xc[e], mu[ONE ? 0 : q], rs, ga, k[q], be[q]);
        xc[e] -= mu[ONE ? 0 : q];
      }
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) xc[e] -= mu[ONE ? 0 : 4 * h + e], z[e] = fmaf(xc[e], k[4 * h + e], be[4 * h + e]);
    }
    times_slope<T>(a.act, z, g);
  };
  if (MODE != APPLY) {
#pragma unroll
    for (int h = 0; h < VEC / 4; ++h) {
      float s[4] = {0.f, 0.f, 0.f, 0.f}, sx[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < R; ++i)
        if (i < mine) {
          float xc[4], g[4];
          grad(i, h, xc, g);
#pragma unroll
          for (int e = 0; e < 4; ++e) s[e] += g[e], sx[e] = fmaf(g[e], xc[e], sx[e]);
        }
      if (live) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int q = 4 * h + e;
          if (WHOLE || q < n) buf[pr * pitch + cl + q] = sx[e] * rstd[first_group + group_of(q)], buf[pr * pitch + a.W + cl + q] = s[e];
        }
      }
    }
    __syncthreads();
    column_sums(buf, a.px, 2 * a.W, pitch, 1, a.share_2w, csum);
    __syncthreads();
    for (int c = t; c < 2 * a.W; c += blockDim.x) part[((long long)bc * 2 + (c >= a.W)) * a.C + c0 + (c >= a.W ? c - a.W : c)] = csum[c];
    if (MODE == STATS) return;
  } else {
    // the image's sums: the chunks' in order
    for (int c = t; c < 2 * a.W; c += blockDim.x) {
      const float *q = part + ((long long)b * a.chunks * 2 + (c >= a.W)) * a.C + c0 + (c >= a.W ? c - a.W : c);
      float s = 0.f;
      for (int k = 0; k < a.chunks; ++k) s += q[2ll * k * a.C];
      csum[c] = s;
    }
    __syncthreads();
  }
  // averages over the group of g gamma xh and g gamma
  {
    const int lane = t & 63;
    for (int q = t >> 6; q < 2 * a.groups; q += blockDim.x >> 6) {
      const int g = q >= a.groups ? q - a.groups : q;
      float s = 0.f;
      for (int c = g * a.Cg + lane; c < (g + 1) * a.Cg; c += 64) s = fmaf(csum[(q >= a.groups ? a.W : 0) + c], gamma[c0 + c], s);
      s = lanes_sum(s, 6);
      if (lane == 0) gsum[q] = s * a.inv;
    }
  }
  __syncthreads();
  float m1[PV], m2[PV];  // rs avg(g gamma), rs^2 avg(g gamma xh)
#pragma unroll
  for (int e = 0; e < PV; ++e) {
    m1[e] = m2[e] = 0.f;
    if (live) {
      const float rs = rstd[first_group + group_of(e)];
      m1[e] = rs * gsum[a.groups + group_of(e)], m2[e] = rs * rs * gsum[group_of(e)];
    }
  }
#pragma unroll
  for (int h = 0; h < VEC / 4; ++h) {
#pragma unroll
    for (int i = 0; i < R; ++i)
      if (i < mine) {
        float xc[4], g[4];
        grad(i, h, xc, g);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int q = 4 * h + e;
          g[e] = fmaf(g[e], k[q], -m1[ONE ? 0 : q]) - xc[e] * m2[ONE ? 0 : q];
        }
        pack4<T>(d[i], h, g);  // dy's place holds dx now
        if (h == VEC / 4 - 1) store_vec<T, WHOLE>((T *)(dst + (off + i * step)), d[i], n);
      }
  }
}

// dgamma[c] and dbeta[c]: sums over the rows of part [rows][2][C], 16 columns by 64 lanes each, in a fixed order
constexpr int RT = 1024;
__global__ __launch_bounds__(RT) void gn_params_kernel(const float *__restrict__ part, int rows, int C,
                                                       float *__restrict__ dgamma, float *__restrict__ dbeta) {
  __shared__ float s[64][17];
  const int x = threadIdx.x & 15, y = threadIdx.x >> 4, c = blockIdx.x * 16 + x;  // columns of [2][C]
  float sum = 0.f;
  if (c < 2 * C) {
#pragma unroll 4
    for (int r = y; r < rows; r += 64) sum += part[(long long)r * 2 * C + c];
  }
  s[y][x] = sum;
  __syncthreads();
  const int col = threadIdx.x >> 6, lane = threadIdx.x & 63, o = blockIdx.x * 16 + col;
  sum = s[lane][col];
#pragma unroll
  for (int k = 32; k; k >>= 1) sum += __shfl_xor(sum, k);
  if (lane == 0 && o < 2 * C) {
    if (o < C)
      dgamma[o] = sum;
    else
      dbeta[o - C] = sum;
  }
}

template <typename T, bool WHOLE, bool ONE>
hipError_t bwd_as(const GnShape &s, const GnPlan &p, const void *dy, const void *x, const float *gamma, const float *beta,
                  const float *mean, const float *rstd, void *dx, float *part, hipStream_t st) {
  constexpr int R = ONE ? 8 : 4;
  const GnArgs &a = p.a;
  const size_t lds = 4 * ((size_t)a.px * (2 * a.W + 1) + 2 * a.W + 2 * a.groups);
  const dim3 grid((unsigned)(p.slabs * s.B * a.chunks)), nt(p.nt);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, nt, lds, st, a, (const T *)dy, (const T *)x, gamma, beta, mean, rstd, (T *)dx, part); };
  if (p.split) {
    go(gn_bwd_kernel<T, WHOLE, ONE, STATS, R, 1024>);
    go(gn_bwd_kernel<T, WHOLE, ONE, APPLY, R, 1024>);
  } else if (p.tiny) {
    go(gn_bwd_kernel<T, WHOLE, ONE, FUSED, 1, TINY>);
  } else if (p.small) {
    go(gn_bwd_kernel<T, WHOLE, ONE, FUSED, 4, 256>);
  } else {
    go(gn_bwd_kernel<T, WHOLE, ONE, FUSED, R, 1024>);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_gn_bwd(const GnShape &s, const void *dy, const void *x, const float *gamma, const float *beta,
                         const float *mean, const float *rstd, void *dx, float *dgamma, float *dbeta, void *ws,
                         hipStream_t st) {
  const GnPlan p = gn_plan(s, true);
  const hipError_t e = by_type(s, p, [&](auto t, auto whole, auto one) {
    return bwd_as<decltype(t), decltype(whole)::value, decltype(one)::value>(s, p, dy, x, gamma, beta, mean, rstd, dx, (float *)ws, st);
  });
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(gn_params_kernel, dim3((2 * s.C + 15) / 16), dim3(RT), 0, st, (const float *)ws, s.B * p.a.chunks, s.C, dgamma, dbeta);
  return hipGetLastError();
}

}  // namespace nf
