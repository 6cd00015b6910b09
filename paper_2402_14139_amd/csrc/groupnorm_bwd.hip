// Group norm with an activation, backward.  gn.h holds the slabs and their sums.
#include "gn.h"

namespace nf {
namespace {

// HBM-bound: 3 * sizeof(T) bytes an element.  sum_gx and sum_g, rows of 2 C floats: sums over pixels of g xh and g, of
// every (image, chunk); APPLY reads those of the images.  64x1024x512 bf16 in 32 groups with SiLU 75 us, 2.7 TB/s: one workgroup of 1024 threads
// to a CU and two rounds of them, which load, compute (36 vector instructions an element: each pass evaluates the slope) and store in
// step, so that the times of memory and of the vector ALU add up.  33x675x72 fp16 in 12 groups 11.9 us: 99 slabs (24 channels: no
// whole vectors in fewer) leave 157 of 256 CUs idle.
template <typename T, bool WHOLE, bool ONE, int MODE, int R, int NTMAX>
__global__ __launch_bounds__(NTMAX) void gn_bwd_kernel(GnArgs a, const T *__restrict__ dy, const T *__restrict__ x,
                                                       const float *__restrict__ gamma, const float *__restrict__ beta,
                                                       const float *__restrict__ mean, const float *__restrict__ rstd,
                                                       T *__restrict__ dx, float *sum_gx, float *sum_g) {
  constexpr int VEC = Vec<T>::N, PV = ONE ? 1 : VEC;  // mean and deviation: one for the vector, or one per channel
  extern __shared__ float lds[];
  const int pitch = 2 * a.W + 1;
  // the channels' means, rstd gamma and beta, then averages in two of their places; rstd and gamma; sums of channels and groups; the matrix
  float *const pm = lds, *const pk = pm + a.Wp, *const pb = pk + a.Wp, *const prs = pb + a.Wp, *const pg = prs + a.Wp;
  float *const csum = pg + a.Wp, *const gsum = csum + 2 * a.W, *const buf = gsum + 2 * a.groups;
  const int t = threadIdx.x;
  const int slabs = a.div_slabs.d;
  const int id = xcd_run(blockIdx.y * gridDim.x + blockIdx.x, gridDim.x * gridDim.y), bc = a.div_slabs.div(id), slab = id - bc * slabs;
  const int b = MODE == FUSED ? bc : (int)a.div_chunks.div(bc), chunk = MODE == FUSED ? 0 : bc - b * a.chunks;
  const int c0 = slab * a.W, W = min(a.W, a.C - c0), groups = W == a.W ? a.groups : (int)a.div_cg.div(W);  // of this slab
  const int p0 = chunk * a.per, p1 = min(a.HW, p0 + a.per);
  const int pr = a.div_cv.div(t), cl = (t - pr * a.cv) * VEC, n = W - cl;
  const bool live = pr < a.px && n > 0;
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
  const long long first_group = (long long)b * a.G + slab * a.groups;
  for (int c = t; c < a.Wp; c += blockDim.x) {
    float m = 0.f, r = 0.f, g = 0.f, bt = 0.f;
    if (c < W) {
      const int q = a.div_cg.div(c);
      m = mean[first_group + q], r = rstd[first_group + q], g = gamma[c0 + c], bt = beta[c0 + c];
    }
    pm[c] = m, pk[c] = r * g, pb[c] = bt, prs[c] = r, pg[c] = g;
  }
  __syncthreads();
  float mu[PV], k[VEC], be[VEC];  // k = rs gamma
  const int at = live ? cl : 0;
  if constexpr (ONE)
    mu[0] = pm[at];
  else
    read_channels(pm + at, mu);
  read_channels(pk + at, k), read_channels(pb + at, be);
  // of 4 elements of the vector at pixel i: xc = x - mu and g = dy act'(z), z = xc k + beta
  auto grad = [&](int i, int h, float (&xc)[4], float (&g)[4]) {
    float z[4];
    unpack4<T>(v[i], h, xc), unpack4<T>(d[i], h, g);
#pragma unroll
    for (int e = 0; e < 4; ++e) xc[e] -= mu[ONE ? 0 : 4 * h + e], z[e] = fmaf(xc[e], k[4 * h + e], be[4 * h + e]);
    if (a.act == NF_ACT_RELU) {
      bool near = false;  // fp32's z is off by a few 2^-24 of beta there
#pragma unroll
      for (int e = 0; e < 4; ++e) near |= fabsf(z[e]) <= 1e-5f * fabsf(be[4 * h + e]);
      if (near) {
        float x[4];
        unpack4<T>(v[i], h, x);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int q = 4 * h + e;
          if (WHOLE || q < n) z[e] = careful_z(x[e], mu[ONE ? 0 : q], prs[cl + q], pg[cl + q], k[q], be[q]);
        }
      }
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
          if (WHOLE || q < n) buf[pr * pitch + cl + q] = sx[e], buf[pr * pitch + a.W + cl + q] = s[e];
        }
      }
    }
    __syncthreads();
    column_sums(buf, a.px, 2 * a.W, pitch, 1, a.share_2w, csum);
    __syncthreads();
    for (int c = t; c < 2 * a.W; c += blockDim.x) {
      const int second = c >= a.W, ch = second ? c - a.W : c;
      if (ch >= W) continue;
      const float v = second ? csum[c] : csum[c] * prs[ch];
      csum[c] = v;
      (second ? sum_g : sum_gx)[(long long)bc * 2 * a.C + c0 + ch] = v;
    }
    if (MODE == STATS) return;
    __syncthreads();
  } else {
    for (int c = t; c < 2 * a.W; c += blockDim.x) {
      const int second = c >= a.W, ch = second ? c - a.W : c;
      if (ch < W) csum[c] = (second ? sum_g : sum_gx)[(long long)b * 2 * a.C + c0 + ch];
    }
    __syncthreads();
  }
  // averages over the group of g gamma xh and g gamma
  {
    const int lane = t & 63;
    for (int q = t >> 6; q < 2 * groups; q += blockDim.x >> 6) {
      const int second = q >= groups, g = second ? q - groups : q;
      float s = 0.f;
      for (int c = g * a.Cg + lane; c < (g + 1) * a.Cg; c += 64) s = fmaf(csum[(second ? a.W : 0) + c], pg[c], s);
      s = lanes_sum(s, 6);
      if (lane == 0) gsum[second * a.groups + g] = s * a.inv;
    }
  }
  __syncthreads();
  for (int c = t; c < W; c += blockDim.x) {  // rs avg(g gamma), rs^2 avg(g gamma xh)
    const int q = a.div_cg.div(c);
    const float r = prs[c];
    pm[c] = r * gsum[a.groups + q], pk[c] = r * r * gsum[q];
  }
  __syncthreads();
  float m1[PV], m2[PV];
  if constexpr (ONE)
    m1[0] = pm[at], m2[0] = pk[at];
  else
    read_channels(pm + at, m1), read_channels(pk + at, m2);
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

// Sums over `rows` rows of part [blockIdx.y][rows][2][C], by 16 columns to 64 lanes each, in a fixed order: chunks to images' sums,
// images to dgamma and dbeta.  A launch's latency: 3.8 us for 33 images of 72 channels, 5.2 for 64 of 512.
constexpr int RT = 1024;
__global__ __launch_bounds__(RT) void gn_rows_kernel(const float *__restrict__ part, int rows, int C, float *__restrict__ out0,
                                                     float *__restrict__ out1, long long out_stride) {
  __shared__ float s[64][17];
  const int x = threadIdx.x & 15, y = threadIdx.x >> 4, c = blockIdx.x * 16 + x;  // columns of [2][C]
  const float *const p = part + (long long)blockIdx.y * rows * 2 * C;
  float sum = 0.f;
  if (c < 2 * C) {
#pragma unroll 4
    for (int r = y; r < rows; r += 64) sum += p[(long long)r * 2 * C + c];
  }
  s[y][x] = sum;
  __syncthreads();
  const int col = threadIdx.x >> 6, lane = threadIdx.x & 63, o = blockIdx.x * 16 + col;
  sum = lanes_sum(s[lane][col], 6);
  if (lane == 0 && o < 2 * C) {
    if (o < C)
      out0[blockIdx.y * out_stride + o] = sum;
    else
      out1[blockIdx.y * out_stride + o - C] = sum;
  }
}
hipError_t sum_rows(const char *name, const float *part, int images, int rows, int C, float *out0, float *out1, hipStream_t st) {
  return recorded(st, name, 0.0, 8.0 * C * images * (rows + 1.0), [&] {
    hipLaunchKernelGGL(gn_rows_kernel, dim3((2 * C + 15) / 16, images), dim3(RT), 0, st, part, rows, C, out0, out1, 2ll * C);
  });
}

constexpr SlabNames BWD_NAMES = {{"groupnorm_bwd_tiny", "groupnorm_bwd_tiny_mixed", "groupnorm_bwd_tiny_odd"},
                                 {"groupnorm_bwd_small", "groupnorm_bwd_small_mixed", "groupnorm_bwd_small_odd"},
                                 {"groupnorm_bwd_slab", "groupnorm_bwd_slab_mixed", "groupnorm_bwd_slab_odd"},
                                 {"groupnorm_bwd_stats", "groupnorm_bwd_stats_mixed", "groupnorm_bwd_stats_odd"},
                                 {"groupnorm_bwd_apply", "groupnorm_bwd_apply_mixed", "groupnorm_bwd_apply_odd"}};

template <typename T, bool WHOLE, bool ONE>
hipError_t bwd_as(const GnShape &s, const GnPlan &p, const void *dy, const void *x, const float *gamma, const float *beta,
                  const float *mean, const float *rstd, void *dx, float *part, float *sum_gx, float *sum_g, hipStream_t st) {
  constexpr int R = ONE ? 8 : 4;
  const GnArgs &a = p.a;
  const size_t lds = 4 * ((size_t)a.px * (2 * a.W + 1) + 5 * a.Wp + 2 * a.W + 2 * a.groups);
  const dim3 grid(p.slabs * a.chunks, s.B), nt(p.nt);  // a grid's axis ends at 2^32 threads
  auto go = [&](int which, double passes, auto kernel, float *gx, float *g) {
    return recorded(st, BWD_NAMES[which][ONE ? 0 : WHOLE ? 1 : 2], 0.0, gn_bytes<T>(s, passes), [&] {
      hipLaunchKernelGGL(kernel, grid, nt, lds, st, a, (const T *)dy, (const T *)x, gamma, beta, mean, rstd, (T *)dx, gx, g);
    });
  };
  if (p.split) {
    hipError_t e = go(SLAB_STATS, 2.0, gn_bwd_kernel<T, WHOLE, ONE, STATS, R, 1024>, part, part + s.C);
    if (e == hipSuccess) e = sum_rows("groupnorm_bwd_chunk_sums", part, s.B, a.chunks, s.C, sum_gx, sum_g, st);
    return e != hipSuccess ? e : go(SLAB_APPLY, 3.0, gn_bwd_kernel<T, WHOLE, ONE, APPLY, R, 1024>, sum_gx, sum_g);
  }
  if (p.tiny) return go(TINY_SLAB, 3.0, gn_bwd_kernel<T, WHOLE, ONE, FUSED, 1, TINY>, sum_gx, sum_g);
  if (p.small) return go(SMALL_SLAB, 3.0, gn_bwd_kernel<T, WHOLE, ONE, FUSED, 4, 256>, sum_gx, sum_g);
  return go(SLAB, 3.0, gn_bwd_kernel<T, WHOLE, ONE, FUSED, R, 1024>, sum_gx, sum_g);
}

// ---- small groups ----
template <typename T, int NT, int R>
__global__ __launch_bounds__(NT < 256 ? 256 : NT) void gn_bwd_few_kernel(GnFew a, const T *__restrict__ dy, const T *__restrict__ x,
                                                                         const float *__restrict__ gamma, const float *__restrict__ beta,
                                                                         const float *__restrict__ mean, const float *__restrict__ rstd,
                                                                         T *__restrict__ dx, float *__restrict__ sum_gx,
                                                                         float *__restrict__ sum_g) {
  __shared__ float lds[2][NT < 256 ? 256 : NT];
  const int t = NT == 64 ? threadIdx.x & 63 : threadIdx.x;
  const int unit = NT == 64 ? blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : blockIdx.x;
  if (unit >= a.units) return;
  const int b = a.div_g.div(unit), grp = unit - b * a.G;
  const int p = a.div_cg.div(t), c = t - p * a.Cg, ch = grp * a.Cg + c;
  const int mine = p < a.px ? (int)a.div_px.div(a.HW - p + a.px - 1) : 0;
  const long long at = ((long long)b * a.HW + p) * a.C + ch, step = (long long)a.px * a.C;
  float xv[R], g[R];
#pragma unroll
  for (int i = 0; i < R; ++i)
    if (i < mine) xv[i] = (float)x[at + i * step], g[i] = (float)dy[at + i * step];
  float ga = 0.f, be = 0.f;
  if (mine) ga = gamma[ch], be = beta[ch];
  const float mu = mean[unit], rs = rstd[unit], k = rs * ga;
  float s = 0.f, sx = 0.f;
#pragma unroll
  for (int i = 0; i < R; ++i)
    if (i < mine) {
      const float x0 = xv[i];
      xv[i] -= mu;
      float z[1] = {fmaf(xv[i], k, be)}, v[1] = {g[i]};
      if (a.act == NF_ACT_RELU && fabsf(z[0]) <= 1e-5f * fabsf(be)) z[0] = careful_z(x0, mu, rs, ga, k, be);
      times_slope<T>(a.act, z, v);
      g[i] = v[0];
      s += g[i], sx = fmaf(g[i], xv[i], sx);
    }
  sx *= rs;
  const float m1 = rs * few_sum<NT>(s * ga, 0) * a.inv, m2 = rs * rs * few_sum<NT>(sx * ga, 1) * a.inv;
#pragma unroll
  for (int i = 0; i < R; ++i)
    if (i < mine) dx[at + i * step] = (T)(fmaf(g[i], k, -m1) - xv[i] * m2);
  // the channels' sums: [pixel][channel] in LDS, which only this wave uses where it is the whole group
  const int base = NT == 64 ? threadIdx.x & ~63 : 0;
  lds[0][base + t] = sx, lds[1][base + t] = s;
  if constexpr (NT > 64) __syncthreads();
  const int first = t & ((1 << a.share) - 1);
  for (int q = t >> a.share; q < a.Cg; q += NT >> a.share) {
    float gx = 0.f, g0 = 0.f;
    for (int r = first; r < a.px; r += 1 << a.share) gx += lds[0][base + r * a.Cg + q], g0 += lds[1][base + r * a.Cg + q];
    gx = lanes_sum(gx, a.share), g0 = lanes_sum(g0, a.share);
    const long long o = (long long)b * 2 * a.C + grp * a.Cg + q;
    if (first == 0) sum_gx[o] = gx, sum_g[o] = g0;
  }
}

template <typename T>
hipError_t bwd_few_as(const GnFew &a, const void *dy, const void *x, const float *gamma, const float *beta, const float *mean,
                      const float *rstd, void *dx, float *sum_gx, float *sum_g, hipStream_t st) {
  static const char *const names[4] = {"groupnorm_bwd_few_64", "groupnorm_bwd_few_256", "groupnorm_bwd_few_1024", "groupnorm_bwd_few_1024_deep"};
  return gn_few_variant(a, names, 3.0 * sizeof(T) * a.units * a.HW * a.Cg, st, [&](auto nt, auto r, dim3 grid, dim3 block) {
    hipLaunchKernelGGL((gn_bwd_few_kernel<T, decltype(nt)::value, decltype(r)::value>), grid, block, 0, st, a, (const T *)dy, (const T *)x, gamma, beta, mean, rstd, (T *)dx, sum_gx, sum_g);
  });
}

}  // namespace

hipError_t launch_gn_bwd(const GnShape &s, const void *dy, const void *x, const float *gamma, const float *beta,
                         const float *mean, const float *rstd, void *dx, float *dgamma, float *dbeta, void *ws,
                         hipStream_t st) {
  const GnPlan p = gn_plan(s, true);
  GnFew few;
  const bool is_few = gn_few(s, true, p, &few);
  // the images' sums [B][2][C], of which one image's are the result; the chunks' lie behind
  float *const sums = (float *)ws, *const part = sums + (size_t)s.B * 2 * s.C;
  float *const sum_gx = s.B == 1 ? dgamma : sums, *const sum_g = s.B == 1 ? dbeta : sums + s.C;
  hipError_t e;
  if (is_few) {
    e = s.dtype == NF_BF16  ? bwd_few_as<__bf16>(few, dy, x, gamma, beta, mean, rstd, dx, sum_gx, sum_g, st)
        : s.dtype == NF_F16 ? bwd_few_as<_Float16>(few, dy, x, gamma, beta, mean, rstd, dx, sum_gx, sum_g, st)
                            : bwd_few_as<float>(few, dy, x, gamma, beta, mean, rstd, dx, sum_gx, sum_g, st);
  } else {
    e = by_type(s, p, [&](auto t, auto whole, auto one) {
      return bwd_as<decltype(t), decltype(whole)::value, decltype(one)::value>(s, p, dy, x, gamma, beta, mean, rstd, dx, part, sum_gx, sum_g, st);
    });
  }
  if (e != hipSuccess || s.B == 1) return e;
  return sum_rows("groupnorm_bwd_sums", sums, 1, s.B, s.C, dgamma, dbeta, st);
}

}  // namespace nf
