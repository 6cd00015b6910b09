// Group norm with an activation, forward.  gn.h holds the slabs and their sums.
#include "gn.h"

namespace nf {
namespace {

// HBM-bound: 2 * sizeof(T) bytes an element (APPLY after STATS: half as much again, which the memory-side cache serves up to
// its 256 MB).  part [image][chunk][group][2]: a chunk's mean and its squares about that.
template <typename T, bool WHOLE, bool ONE, int MODE, int R, int NTMAX>
__global__ __launch_bounds__(NTMAX) void gn_fwd_kernel(GnArgs a, const T *__restrict__ x, const float *__restrict__ gamma,
                                                       const float *__restrict__ beta, T *__restrict__ y,
                                                       float *__restrict__ mean, float *__restrict__ rstd,
                                                       float *__restrict__ part) {
  constexpr int VEC = Vec<T>::N;
  extern __shared__ float lds[];
  // the channels' means, rstd gamma and beta; the groups' sums; the matrix and the channels' sums
  float *const pm = lds, *const pk = pm + a.Wp, *const pb = pk + a.Wp, *const gm = pb + a.Wp, *const gr = gm + a.groups;
  float *const buf = gr + a.groups, *const csum = buf + a.px * (a.W | 1);
  const int t = threadIdx.x;
  const int slabs = a.div_slabs.d;
  const int id = xcd_run(blockIdx.y * gridDim.x + blockIdx.x, gridDim.x * gridDim.y), bc = a.div_slabs.div(id), slab = id - bc * slabs;
  const int b = MODE == FUSED ? bc : (int)a.div_chunks.div(bc), chunk = MODE == FUSED ? 0 : bc - b * a.chunks;
  const int c0 = slab * a.W, W = min(a.W, a.C - c0), groups = W == a.W ? a.groups : (int)a.div_cg.div(W);  // of this slab
  const int p0 = chunk * a.per, p1 = min(a.HW, p0 + a.per);
  const int pr = a.div_cv.div(t), cl = (t - pr * a.cv) * VEC, n = W - cl;  // n: the slab's channels from here on
  const bool live = pr < a.px && n > 0;
  // offsets within the slab fit 32 bits (gn_plan)
  const long long first = ((long long)b * a.HW + p0) * a.C + c0;
  const char *const xs = (const char *)(x + first);
  char *const dst = (char *)(y + first);
  const uint32_t off = (uint32_t)((pr * a.C + cl) * (int)sizeof(T)), step = (uint32_t)(a.px * a.C * (int)sizeof(T));
  const int mine = live ? (int)a.div_px.div(p1 - p0 - pr + a.px - 1) : 0;  // at most R
  uintx4 v[R];
#pragma unroll
  for (int i = 0; i < R; ++i)
    if (i < mine) v[i] = load_vec<T, WHOLE>((const T *)(xs + (off + i * step)), n);
  if (MODE != STATS) {
    for (int c = t; c < a.Wp; c += blockDim.x) pk[c] = c < W ? gamma[c0 + c] : 0.f, pb[c] = c < W ? beta[c0 + c] : 0.f;
  }
  float mu[VEC], s[VEC];
  if (MODE != APPLY) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) s[e] = 0.f;
#pragma unroll
    for (int i = 0; i < R; ++i)
      if (i < mine) {
        float f[VEC];
        unpack<T>(v[i], f);
#pragma unroll
        for (int e = 0; e < VEC; ++e) s[e] += f[e];
      }
    group_sums<VEC, ONE>(a, W, groups, pr, cl, s, buf, csum, gm);
    const float inv = MODE == FUSED ? a.inv : 1.f / ((float)(p1 - p0) * (float)a.Cg);
    for (int c = t; c < a.Wp; c += blockDim.x) pm[c] = c < W ? gm[a.div_cg.div(c)] * inv : 0.f;
    __syncthreads();
    read_channels(pm + (live ? cl : 0), mu);
#pragma unroll
    for (int e = 0; e < VEC; ++e) s[e] = 0.f;
#pragma unroll
    for (int i = 0; i < R; ++i)
      if (i < mine) {
        float f[VEC];
        unpack<T>(v[i], f);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const float d = f[e] - mu[e];
          s[e] = fmaf(d, d, s[e]);
        }
      }
    group_sums<VEC, ONE>(a, W, groups, pr, cl, s, buf, csum, gr);
    for (int g = t; g < groups; g += blockDim.x) {
      const long long o = (long long)bc * a.G + slab * a.groups + g;
      if (MODE == STATS) {
        part[2 * o] = gm[g] * inv, part[2 * o + 1] = gr[g];
      } else {
        mean[o] = gm[g] * inv;
        rstd[o] = 1.f / sqrtf(gr[g] * inv + a.eps);
      }
    }
    if (MODE == STATS) return;
    for (int c = t; c < W; c += blockDim.x) pk[c] *= 1.f / sqrtf(gr[a.div_cg.div(c)] * a.inv + a.eps);
  } else {
    // chunks' means and squares to the image's: the squares about the image's mean are those about the chunks' plus
    // count * (chunk's mean - image's mean)^2
    const int lane = t & 63;
    for (int g = t >> 6; g < groups; g += blockDim.x >> 6) {
      const float *q = part + 2 * ((long long)b * a.chunks * a.G + slab * a.groups + g);
      float sum = 0.f, sq = 0.f;
      for (int k = lane; k < a.chunks; k += 64) sum += q[2ll * k * a.G] * (float)(min(a.HW, (k + 1) * a.per) - k * a.per);
      sum = lanes_sum(sum, 6);
      const float m = sum / (float)a.HW;
      for (int k = lane; k < a.chunks; k += 64) {
        const float d = q[2ll * k * a.G] - m;
        sq += q[2ll * k * a.G + 1] + d * d * ((float)(min(a.HW, (k + 1) * a.per) - k * a.per) * (float)a.Cg);
      }
      sq = lanes_sum(sq, 6);
      if (lane == 0) {
        const float r = 1.f / sqrtf(sq * a.inv + a.eps);
        gm[g] = m, gr[g] = r;
        if (chunk == 0) mean[(long long)b * a.G + slab * a.groups + g] = m, rstd[(long long)b * a.G + slab * a.groups + g] = r;
      }
    }
    __syncthreads();
    for (int c = t; c < W; c += blockDim.x) pm[c] = gm[a.div_cg.div(c)], pk[c] *= gr[a.div_cg.div(c)];
  }
  __syncthreads();
  if (!live) return;
  float ga[VEC], be[VEC];
  if (MODE == APPLY) read_channels(pm + cl, mu);
  read_channels(pk + cl, ga), read_channels(pb + cl, be);
#pragma unroll
  for (int i = 0; i < R; ++i)
    if (i < mine) {
      float f[VEC];
      unpack<T>(v[i], f);
#pragma unroll
      for (int e = 0; e < VEC; ++e) f[e] = fmaf(f[e] - mu[e], ga[e], be[e]);
      act_of<T>(a.act, f);
      Vec<T> t;
#pragma unroll
      for (int e = 0; e < VEC; ++e) t.v[e] = (T)f[e];
      store_vec<T, WHOLE>((T *)(dst + (off + i * step)), __builtin_bit_cast(uintx4, t), n);
    }
}

constexpr SlabNames FWD_NAMES = {{"groupnorm_fwd_tiny", "groupnorm_fwd_tiny_mixed", "groupnorm_fwd_tiny_odd"},
                                 {"groupnorm_fwd_small", "groupnorm_fwd_small_mixed", "groupnorm_fwd_small_odd"},
                                 {"groupnorm_fwd_slab", "groupnorm_fwd_slab_mixed", "groupnorm_fwd_slab_odd"},
                                 {"groupnorm_fwd_stats", "groupnorm_fwd_stats_mixed", "groupnorm_fwd_stats_odd"},
                                 {"groupnorm_fwd_apply", "groupnorm_fwd_apply_mixed", "groupnorm_fwd_apply_odd"}};

template <typename T, bool WHOLE, bool ONE>
hipError_t fwd_as(const GnShape &s, const GnPlan &p, const void *x, const float *gamma, const float *beta, void *y,
                  float *mean, float *rstd, float *part, hipStream_t st) {
  const GnArgs &a = p.a;
  const size_t lds = 4 * (size_t)(3 * a.Wp + 2 * a.groups + matrix_floats(a, Vec<T>::N, ONE));
  const dim3 grid(p.slabs * a.chunks, s.B), nt(p.nt);  // a grid's axis ends at 2^32 threads
  auto go = [&](int which, double passes, auto kernel) {
    return recorded(st, FWD_NAMES[which][ONE ? 0 : WHOLE ? 1 : 2], 0.0, gn_bytes<T>(s, passes),
                    [&] { hipLaunchKernelGGL(kernel, grid, nt, lds, st, a, (const T *)x, gamma, beta, (T *)y, mean, rstd, part); });
  };
  if (p.split) {
    const hipError_t e = go(SLAB_STATS, 1.0, gn_fwd_kernel<T, WHOLE, ONE, STATS, 8, 1024>);
    return e != hipSuccess ? e : go(SLAB_APPLY, 2.0, gn_fwd_kernel<T, WHOLE, ONE, APPLY, 8, 1024>);
  }
  if (p.tiny) return go(TINY_SLAB, 2.0, gn_fwd_kernel<T, WHOLE, ONE, FUSED, 1, TINY>);
  if (p.small) return go(SMALL_SLAB, 2.0, gn_fwd_kernel<T, WHOLE, ONE, FUSED, 4, 256>);
  return go(SLAB, 2.0, gn_fwd_kernel<T, WHOLE, ONE, FUSED, 16, 1024>);
}

// ---- small groups ----
template <typename T, int NT, int R>
__global__ __launch_bounds__(NT < 256 ? 256 : NT) void gn_fwd_few_kernel(GnFew a, const T *__restrict__ x, const float *__restrict__ gamma,
                                                                         const float *__restrict__ beta, T *__restrict__ y,
                                                                         float *__restrict__ mean, float *__restrict__ rstd) {
  const int t = NT == 64 ? threadIdx.x & 63 : threadIdx.x;
  const int unit = NT == 64 ? blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : blockIdx.x;
  if (unit >= a.units) return;
  const int b = a.div_g.div(unit), grp = unit - b * a.G;
  const int p = a.div_cg.div(t), c = t - p * a.Cg, ch = grp * a.Cg + c;
  const int mine = p < a.px ? (int)a.div_px.div(a.HW - p + a.px - 1) : 0;
  const long long at = ((long long)b * a.HW + p) * a.C + ch, step = (long long)a.px * a.C;
  float v[R], s = 0.f;
#pragma unroll
  for (int i = 0; i < R; ++i)
    if (i < mine) v[i] = (float)x[at + i * step];
  float ga = 0.f, be = 0.f;
  if (mine) ga = gamma[ch], be = beta[ch];
#pragma unroll
  for (int i = 0; i < R; ++i)
    if (i < mine) s += v[i];
  const float mu = few_sum<NT>(s, 0) * a.inv;
  s = 0.f;
#pragma unroll
  for (int i = 0; i < R; ++i)
    if (i < mine) v[i] -= mu, s = fmaf(v[i], v[i], s);
  const float rs = 1.f / sqrtf(few_sum<NT>(s, 1) * a.inv + a.eps);
  if (t == 0) mean[unit] = mu, rstd[unit] = rs;
  ga *= rs;
#pragma unroll
  for (int i = 0; i < R; ++i)
    if (i < mine) {
      float z[1] = {fmaf(v[i], ga, be)};
      act_of<T>(a.act, z);
      y[at + i * step] = (T)z[0];
    }
}

template <typename T>
hipError_t fwd_few_as(const GnFew &a, const void *x, const float *gamma, const float *beta, void *y, float *mean, float *rstd,
                      hipStream_t st) {
  static const char *const names[4] = {"groupnorm_fwd_few_64", "groupnorm_fwd_few_256", "groupnorm_fwd_few_1024", "groupnorm_fwd_few_1024_deep"};
  return gn_few_variant(a, names, 2.0 * sizeof(T) * a.units * a.HW * a.Cg, st, [&](auto nt, auto r, dim3 grid, dim3 block) {
    hipLaunchKernelGGL((gn_fwd_few_kernel<T, decltype(nt)::value, decltype(r)::value>), grid, block, 0, st, a, (const T *)x, gamma, beta, (T *)y, mean, rstd);
  });
}

}  // namespace

size_t gn_fwd_workspace_bytes(const GnShape &s) {
  const GnPlan p = gn_plan(s, false);
  return p.split ? (size_t)s.B * p.a.chunks * 2 * s.G * 4 : 0;
}

size_t gn_workspace_bytes(const GnShape &s) {
  const GnPlan b = gn_plan(s, true);
  return std::max((size_t)s.B * (1 + (b.split ? b.a.chunks : 0)) * 2 * s.C * 4, gn_fwd_workspace_bytes(s));
}

hipError_t launch_gn_fwd(const GnShape &s, const void *x, const float *gamma, const float *beta, void *y, float *mean,
                         float *rstd, void *ws, hipStream_t st) {
  const GnPlan p = gn_plan(s, false);
  GnFew few;
  if (gn_few(s, false, p, &few)) {
    if (s.dtype == NF_BF16) return fwd_few_as<__bf16>(few, x, gamma, beta, y, mean, rstd, st);
    if (s.dtype == NF_F16) return fwd_few_as<_Float16>(few, x, gamma, beta, y, mean, rstd, st);
    return fwd_few_as<float>(few, x, gamma, beta, y, mean, rstd, st);
  }
  return by_type(s, p, [&](auto t, auto whole, auto one) {
    return fwd_as<decltype(t), decltype(whole)::value, decltype(one)::value>(s, p, x, gamma, beta, y, mean, rstd, (float *)ws, st);
  });
}

}  // namespace nf
