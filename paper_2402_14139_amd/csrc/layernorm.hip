// Layer norm over rows, forward and backward.
//   y = (x - mean) rstd gamma + beta, rstd = (var + eps)^-1/2
//   with xh = (x - mean) rstd, g = dy gamma:  dx = rstd (g - avg(g) - xh avg(g xh)) + dr,  dgamma = sum dy xh,  dbeta = sum dy
// Memory-bound: 2 tensors forward, 3 or 4 backward.  A row stays in the registers of TPR threads, U pieces of 8 elements to a thread, so
// that it is read once; its mean and its squares about the mean come from the registers.  Up to 2048 channels a row belongs to lanes of
// one wave, which add without LDS and without barriers; up to 16384 to a workgroup.  Longer rows are read again from the caches.
// The parameters' gradients are running sums of a thread's columns over the rows that its workgroup takes; the workgroups' sums are added in
// order by a second launch.
#include <algorithm>
#include <type_traits>

#include "nf_enqueue.h"
#include "pw_math.h"

namespace nf {
namespace {

constexpr int STREAM = 1024;  // threads for rows that do not fit registers

template <int CTRL>
__device__ inline float row_partner(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true));
}
// A sum over N neighbouring lanes, the same bits on all of them: partners add the same two numbers.
template <int N>
__device__ inline float lanes_sum(float v) {
  if constexpr (N >= 2) v += row_partner<0xB1>(v);    // the other of two
  if constexpr (N >= 4) v += row_partner<0x4E>(v);    // the other two of four
  if constexpr (N >= 8) v += row_partner<0x141>(v);   // the other four of eight, mirrored
  if constexpr (N >= 16) v += row_partner<0x140>(v);  // the other eight of sixteen
  if constexpr (N >= 32) {
    const auto t = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
    const uint32_t a = t[0], b = t[1];
    v = __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b);
  }
  if constexpr (N >= 64) {
    const auto t = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
    const uint32_t a = t[0], b = t[1];
    v = __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b);
  }
  return v;
}

// Sums of K values over a row's TPR threads.  Beyond a wave they go through LDS; calls alternate between two buffers, so that one barrier
// a call is enough.
template <int TPR, int K>
__device__ inline void row_sums(float (&v)[K], float *lds, int &turn) {
#pragma unroll
  for (int k = 0; k < K; ++k) v[k] = lanes_sum<(TPR < 64 ? TPR : 64)>(v[k]);
  if constexpr (TPR > 64) {
    constexpr int W = TPR / 64;
    float *const at = lds + (turn & 1) * W * K;
    ++turn;
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int k = 0; k < K; ++k) at[(threadIdx.x >> 6) * K + k] = v[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
      v[k] = at[k];
#pragma unroll
      for (int w = 1; w < W; ++w) v[k] += at[w * K + k];
    }
  }
}

struct LnArgs {
  long long M;
  int C, ld;  // ld: C in whole pieces
  float inv, eps;
};

template <int TPR>
constexpr int threads_of() {
  return TPR > 256 ? TPR : 256;
}

// Inputs from HBM: 65536x512 bf16 28 us a call (26 traced), 4.8 TB/s; 16384x2048 fp32 63, 4.3; one row of 2048 takes the launch's 2.5 and 2 more for its two sums.
template <typename T, int TPR, int U, bool WHOLE>
__global__ __launch_bounds__(threads_of<TPR>()) void ln_fwd_kernel(LnArgs a, const T *x, const float *__restrict__ gamma,
                                                                   const float *__restrict__ beta, T *y, float *mean, float *rstd) {
  constexpr int BT = threads_of<TPR>(), SLOTS = BT / TPR;
  __shared__ float lds[2 * (BT / 64)];
  const int slot = threadIdx.x / TPR, j = threadIdx.x % TPR;
  int turn = 0, n[U];
  float ga[U][8], be[U][8];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int at = (j + u * TPR) * 8;
    n[u] = min(max(a.C - at, 0), 8);
#pragma unroll
    for (int e = 0; e < 8; ++e) ga[u][e] = 1.f, be[u][e] = 0.f;
    if (n[u] > 0 && gamma) load8(gamma + at, ga[u], n[u]);
    if (n[u] > 0 && beta) load8(beta + at, be[u], n[u]);
  }
  const long long step = (long long)gridDim.x * SLOTS;
  Raw8<T> next[U] = {};
  auto fetch = [&](long long row) {
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (row < a.M && n[u] > 0) next[u] = raw8(x + row * a.C + (j + u * TPR) * 8, n[u]);
  };
  fetch((long long)blockIdx.x * SLOTS + slot);
  for (long long base = (long long)blockIdx.x * SLOTS; base < a.M; base += step) {
    const long long row = base + slot;
    float v[U][8], s[1] = {0.f};
#pragma unroll
    for (int u = 0; u < U; ++u) {
      unpack8(next[u], v[u]);
#pragma unroll
      for (int e = 0; e < 8; ++e) s[0] += v[u][e];
    }
    fetch(row + step);
    row_sums<TPR>(s, lds, turn);
    const float mu = s[0] * a.inv;
    s[0] = 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (n[u] > 0) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          v[u][e] -= mu;
          if (WHOLE || e < n[u]) s[0] = fmaf(v[u][e], v[u][e], s[0]);
        }
      }
    row_sums<TPR>(s, lds, turn);
    const float rs = 1.f / sqrtf(fmaf(s[0], a.inv, a.eps));
    if (row < a.M) {
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (n[u] > 0) {
#pragma unroll
          for (int e = 0; e < 8; ++e) v[u][e] = fmaf(v[u][e] * rs, ga[u][e], be[u][e]);
          store8(y + row * a.C + (j + u * TPR) * 8, v[u], n[u]);
        }
      if (mean && j == 0) mean[row] = mu, rstd[row] = rs;
    }
  }
}

// Inputs from HBM: 16384x2048 bf16 with dr 64 us a call, 4.2 TB/s (traced 61, and 4.7 for the workgroups' sums); 22275x100 fp32 12.2 (traced 10, and 3.6).
// part [workgroups][2][ld] (or the gradients themselves where there is one workgroup); null where no parameter's gradient is wanted
template <typename T, int TPR, int U, bool WHOLE>
__global__ __launch_bounds__(threads_of<TPR>()) void ln_bwd_kernel(LnArgs a, const T *dy, const T *__restrict__ x, const float *__restrict__ gamma,
                                                                   const float *__restrict__ mean, const float *__restrict__ rstd, const T *dr, T *dx,
                                                                   float *part, float *dgamma, float *dbeta) {
  constexpr int BT = threads_of<TPR>(), SLOTS = BT / TPR, W = BT / 64, ACROSS = TPR * U * 8;
  __shared__ float lds[TPR > 64 ? 4 * W : W * (TPR < 64 ? TPR * U * 8 : ACROSS)];
  const int slot = threadIdx.x / TPR, j = threadIdx.x % TPR;
  int turn = 0, n[U];
  float ga[U][8], dg[U][8], db[U][8];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int at = (j + u * TPR) * 8;
    n[u] = min(max(a.C - at, 0), 8);
#pragma unroll
    for (int e = 0; e < 8; ++e) ga[u][e] = 1.f, dg[u][e] = db[u][e] = 0.f;
    if (n[u] > 0 && gamma) load8(gamma + at, ga[u], n[u]);
  }
  const long long step = (long long)gridDim.x * SLOTS;
  for (long long base = (long long)blockIdx.x * SLOTS; base < a.M; base += step) {
    const long long row = base + slot;
    const bool live = row < a.M;
    Raw8<T> rx[U] = {}, rd[U] = {}, rr[U] = {};
    float mu = 0.f, rs = 0.f;
    if (live) {
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (n[u] > 0) {
          const long long at = row * a.C + (j + u * TPR) * 8;
          rx[u] = raw8(x + at, n[u]), rd[u] = raw8(dy + at, n[u]);
          if (dr) rr[u] = raw8(dr + at, n[u]);
        }
      mu = mean[row], rs = rstd[row];
    }
    float s[2] = {0.f, 0.f}, xh[U][8], g[U][8];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      unpack8(rx[u], xh[u]), unpack8(rd[u], g[u]);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        xh[u][e] = (WHOLE ? n[u] > 0 : e < n[u]) ? (xh[u][e] - mu) * rs : 0.f;
        db[u][e] += g[u][e];
        dg[u][e] = fmaf(g[u][e], xh[u][e], dg[u][e]);
        g[u][e] *= ga[u][e];
        s[0] += g[u][e];
        s[1] = fmaf(g[u][e], xh[u][e], s[1]);
      }
    }
    if (dx) {
      row_sums<TPR>(s, lds, turn);
      const float m0 = s[0] * a.inv, m1 = s[1] * a.inv;
      if (live) {
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (n[u] > 0) {
            float r[8];
            unpack8(rr[u], r);
#pragma unroll
            for (int e = 0; e < 8; ++e) r[e] = fmaf(rs, g[u][e] - m0 - xh[u][e] * m1, r[e]);
            store8(dx + row * a.C + (j + u * TPR) * 8, r, n[u]);
          }
      }
    }
  }
  if (!part) return;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    float *const out = gridDim.x == 1 ? (which ? dbeta : dgamma) : part + ((long long)blockIdx.x * 2 + which) * a.ld;
    if constexpr (TPR > 64) {
      if (!out) continue;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float t[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) t[e] = which ? db[u][e] : dg[u][e];
        if (n[u] > 0) store8(out + (j + u * TPR) * 8, t, n[u]);
      }
    } else {  // over the wave's rows, then over the waves
      __syncthreads();
      const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float t = which ? db[u][e] : dg[u][e];
#pragma unroll
          for (int k = TPR; k < 64; k *= 2) t += __shfl_xor(t, k);
          if (lane < TPR) lds[wave * ACROSS + (lane + u * TPR) * 8 + e] = t;
        }
      __syncthreads();
      for (int c = threadIdx.x; c < min(ACROSS, a.C); c += BT) {
        float t = lds[c];
#pragma unroll
        for (int w = 1; w < W; ++w) t += lds[w * ACROSS + c];
        if (out) out[c] = t;
      }
    }
  }
}

// Rows longer than the registers of a workgroup hold: read once for the mean, again for the squares and again for the result; the row
// stays in the caches.  2000x20000 bf16 93 us, 1.7 TB/s of what has to move; its gradients 171 (x and dy three times), 1.4.
__device__ inline float all_sum(float v, float *lds) {
  v = lanes_sum<64>(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  v = lds[0];
#pragma unroll
  for (int w = 1; w < STREAM / 64; ++w) v += lds[w];
  return v;
}
template <typename T>
__global__ __launch_bounds__(STREAM) void ln_fwd_long_kernel(LnArgs a, const T *x, const float *__restrict__ gamma, const float *__restrict__ beta,
                                                             T *y, float *mean, float *rstd) {
  __shared__ float lds[STREAM / 64];
  for (long long row = blockIdx.x; row < a.M; row += gridDim.x) {
    const T *const p = x + row * a.C;
    float s = 0.f, v[8];
    for (int c = threadIdx.x * 8; c < a.C; c += STREAM * 8) {
      load8(p + c, v, a.C - c);
#pragma unroll
      for (int e = 0; e < 8; ++e) s += v[e];
    }
    const float mu = all_sum(s, lds) * a.inv;
    s = 0.f;
    for (int c = threadIdx.x * 8; c < a.C; c += STREAM * 8) {
      load8(p + c, v, a.C - c);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < a.C - c) s = fmaf(v[e] - mu, v[e] - mu, s);
    }
    const float rs = 1.f / sqrtf(fmaf(all_sum(s, lds), a.inv, a.eps));
    for (int c = threadIdx.x * 8; c < a.C; c += STREAM * 8) {
      float ga[8], be[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) ga[e] = 1.f, be[e] = 0.f;
      load8(p + c, v, a.C - c);
      if (gamma) load8(gamma + c, ga, a.C - c);
      if (beta) load8(beta + c, be, a.C - c);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = fmaf((v[e] - mu) * rs, ga[e], be[e]);
      store8(y + row * a.C + c, v, a.C - c);
    }
    if (mean && threadIdx.x == 0) mean[row] = mu, rstd[row] = rs;
  }
}
template <typename T>
__global__ __launch_bounds__(STREAM) void ln_bwd_long_kernel(LnArgs a, const T *dy, const T *__restrict__ x, const float *__restrict__ gamma,
                                                             const float *__restrict__ mean, const float *__restrict__ rstd, const T *dr, T *dx) {
  __shared__ float lds[STREAM / 64];
  for (long long row = blockIdx.x; row < a.M; row += gridDim.x) {
    const float mu = mean[row], rs = rstd[row];
    float s0 = 0.f, s1 = 0.f;
    auto piece = [&](int c, float (&g)[8], float (&xh)[8]) {
      float ga[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) ga[e] = 1.f;
      load8(dy + row * a.C + c, g, a.C - c);
      load8(x + row * a.C + c, xh, a.C - c);
      if (gamma) load8(gamma + c, ga, a.C - c);
#pragma unroll
      for (int e = 0; e < 8; ++e) g[e] *= ga[e], xh[e] = e < a.C - c ? (xh[e] - mu) * rs : 0.f;
    };
    for (int c = threadIdx.x * 8; c < a.C; c += STREAM * 8) {
      float g[8], xh[8];
      piece(c, g, xh);
#pragma unroll
      for (int e = 0; e < 8; ++e) s0 += g[e], s1 = fmaf(g[e], xh[e], s1);
    }
    const float m0 = all_sum(s0, lds) * a.inv, m1 = all_sum(s1, lds) * a.inv;
    for (int c = threadIdx.x * 8; c < a.C; c += STREAM * 8) {
      float g[8], xh[8], r[8];
      piece(c, g, xh);
#pragma unroll
      for (int e = 0; e < 8; ++e) r[e] = 0.f;
      if (dr) load8(dr + row * a.C + c, r, a.C - c);
#pragma unroll
      for (int e = 0; e < 8; ++e) r[e] = fmaf(rs, g[e] - m0 - xh[e] * m1, r[e]);
      store8(dx + row * a.C + c, r, a.C - c);
    }
  }
}
// the parameters' gradients of long rows: a thread has 8 columns and walks the rows of its part
template <typename T>
__global__ __launch_bounds__(256) void ln_columns_kernel(LnArgs a, long long per, const T *__restrict__ dy, const T *__restrict__ x,
                                                         const float *__restrict__ mean, const float *__restrict__ rstd, float *part, float *dgamma, float *dbeta) {
  const int c = (blockIdx.x * 256 + threadIdx.x) * 8, n = a.C - c;
  if (n <= 0) return;
  float dg[8], db[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) dg[e] = db[e] = 0.f;
  const long long r1 = min(a.M, (blockIdx.y + 1) * per);
  for (long long row = blockIdx.y * per; row < r1; ++row) {
    float g[8], xh[8];
    load8(dy + row * a.C + c, g, n);
    load8(x + row * a.C + c, xh, n);
    const float mu = mean[row], rs = rstd[row];
#pragma unroll
    for (int e = 0; e < 8; ++e) db[e] += g[e], dg[e] = fmaf(g[e], (xh[e] - mu) * rs, dg[e]);
  }
  float *const og = gridDim.y == 1 ? dgamma : part + (long long)blockIdx.y * 2 * a.ld, *const ob = gridDim.y == 1 ? dbeta : part + ((long long)blockIdx.y * 2 + 1) * a.ld;
  if (og) store8(og + c, dg, n);
  if (ob) store8(ob + c, db, n);
}

// The workgroups' sums: 16 columns to a workgroup of 64 x 16 threads, in a fixed order.
constexpr int CT = 1024;
__global__ __launch_bounds__(CT) void ln_sums_kernel(const float *__restrict__ part, int rows, int ld, int C, float *dgamma, float *dbeta) {
  __shared__ float s[64][17];
  const int x = threadIdx.x & 15, y = threadIdx.x >> 4, c = blockIdx.x * 16 + x;
  float sum = 0.f;
  if (c < 2 * ld) {
#pragma unroll 8
    for (int r = y; r < rows; r += 64) sum += part[2ll * r * ld + c];
  }
  s[y][x] = sum;
  __syncthreads();
  const int col = threadIdx.x >> 6, lane = threadIdx.x & 63;
  sum = lanes_sum<64>(s[lane][col]);
  const int at = blockIdx.x * 16 + col;
  if (lane != 0 || at >= 2 * ld) return;
  float *const out = at < ld ? dgamma : dbeta;
  const int k = at < ld ? at : at - ld;
  if (out && k < C) out[k] = sum;
}

// ---- plans ----
struct LnPlan {
  int tpr, u;      // u = 0: long rows
  unsigned blocks;  // of the row kernels
  long long per, parts;  // long rows: rows of a part, and parts; else parts = blocks
};
LnPlan ln_plan(long long M, int C, bool bwd) {
  LnPlan p = {};
  const int pieces = (C + 7) / 8;
  p.u = 1;
  if (pieces <= 64) {
    for (p.tpr = 2; p.tpr < pieces; p.tpr *= 2) {
    }
  } else if (pieces <= 256) {
    p.tpr = 64, p.u = pieces <= 128 ? 2 : 4;
  } else if (pieces <= 2048) {
    p.tpr = pieces <= 512 ? 256 : 512, p.u = pieces <= 1024 ? 2 : 4;  // 1024 threads would leave each other 128 registers
  } else {
    p.u = 0;
    p.blocks = (unsigned)std::min<long long>(M, 512);
    p.parts = std::max<long long>(1, std::min<long long>(256, M / 16));
    p.per = (M + p.parts - 1) / p.parts, p.parts = (M + p.per - 1) / p.per;
    return p;
  }
  const int slots = std::max(256, p.tpr) / p.tpr;
  // The gradients' workgroups leave a sum for every column each.  Rows of a workgroup each, 4 to one: 1000x8192 bf16 23 us (two rows each: 30), 4096x8192 47 in 256
  // and 53 in 512, 4096x4096 35 and 30; rows of waves: 65536x512 bf16 38 in 1024, 50 in 512, 46 in 2048, 22275x100 fp32 11.8, 11.8, 15.3.
  const long long most = !bwd ? 2048 : p.tpr <= 64 ? 1024 / p.u : std::min<long long>(pieces <= 512 ? 512 : 256, std::max<long long>(64, M / 4));
  p.blocks = (unsigned)std::min<long long>((M + slots - 1) / slots, most);
  p.parts = p.blocks;
  return p;
}

template <typename T, typename F>
void by_shape(const LnPlan &p, bool whole, F go) {
  auto as = [&](auto tpr, auto u) { whole ? go(tpr, u, std::true_type()) : go(tpr, u, std::false_type()); };
  using std::integral_constant;
  using I1 = integral_constant<int, 1>;
  using I2 = integral_constant<int, 2>;
  switch (p.tpr) {
    case 2: return as(integral_constant<int, 2>(), I1());
    case 4: return as(integral_constant<int, 4>(), I1());
    case 8: return as(integral_constant<int, 8>(), I1());
    case 16: return as(integral_constant<int, 16>(), I1());
    case 32: return as(integral_constant<int, 32>(), I1());
    case 64:
      if (p.u == 1) return as(integral_constant<int, 64>(), I1());
      if (p.u == 2) return as(integral_constant<int, 64>(), I2());
      return as(integral_constant<int, 64>(), integral_constant<int, 4>());
    case 256: return as(integral_constant<int, 256>(), I2());
    default:
      if (p.u == 2) return as(integral_constant<int, 512>(), I2());
      return as(integral_constant<int, 512>(), integral_constant<int, 4>());
  }
}

template <typename T>
hipError_t fwd_as(const LnShape &s, const T *x, const float *gamma, const float *beta, T *y, float *mean, float *rstd, hipStream_t st) {
  const LnPlan p = ln_plan(s.M, s.C, false);
  const LnArgs a = {s.M, s.C, (s.C + 7) / 8 * 8, 1.f / s.C, s.eps};
  return recorded(st, p.u ? "layernorm_fwd" : "layernorm_fwd_long", 0.0, 2.0 * sizeof(T) * s.M * s.C, [&] {
    if (!p.u) {
      hipLaunchKernelGGL(ln_fwd_long_kernel<T>, dim3(p.blocks), dim3(STREAM), 0, st, a, x, gamma, beta, y, mean, rstd);
      return;
    }
    by_shape<T>(p, s.C % 8 == 0, [&](auto tpr, auto u, auto whole) {
      constexpr int R = decltype(tpr)::value;
      hipLaunchKernelGGL((ln_fwd_kernel<T, R, decltype(u)::value, decltype(whole)::value>), dim3(p.blocks), dim3(threads_of<R>()), 0, st, a, x, gamma, beta, y, mean, rstd);
    });
  });
}

template <typename T>
hipError_t bwd_as(const LnShape &s, const T *dy, const T *x, const float *gamma, const float *mean, const float *rstd, const T *dr, T *dx, float *dgamma,
                  float *dbeta, float *ws, hipStream_t st) {
  const LnPlan p = ln_plan(s.M, s.C, true);
  const LnArgs a = {s.M, s.C, (s.C + 7) / 8 * 8, 1.f / s.C, s.eps};
  const bool sums = dgamma || dbeta;
  float *const part = !sums ? nullptr : p.parts == 1 ? (dgamma ? dgamma : dbeta) : ws;  // one part: only whether it is null counts
  const double bytes = (2.0 + (dr != nullptr) + (dx != nullptr)) * sizeof(T) * s.M * s.C;
  hipError_t e = hipSuccess;
  if (p.u) {
    e = recorded(st, "layernorm_bwd", 0.0, bytes, [&] {
      by_shape<T>(p, s.C % 8 == 0, [&](auto tpr, auto u, auto whole) {
        constexpr int R = decltype(tpr)::value;
        hipLaunchKernelGGL((ln_bwd_kernel<T, R, decltype(u)::value, decltype(whole)::value>), dim3(p.blocks), dim3(threads_of<R>()), 0, st, a, dy, x, gamma, mean,
                           rstd, dr, dx, part, dgamma, dbeta);
      });
    });
  } else {
    if (sums)  // first: dx may be dy
      e = recorded(st, "layernorm_columns", 0.0, 2.0 * sizeof(T) * s.M * s.C, [&] {
        hipLaunchKernelGGL(ln_columns_kernel<T>, dim3((a.ld / 8 + 255) / 256, (unsigned)p.parts), dim3(256), 0, st, a, p.per, dy, x, mean, rstd, part, dgamma, dbeta);
      });
    if (e == hipSuccess && dx)
      e = recorded(st, "layernorm_bwd_long", 0.0, bytes, [&] {
        hipLaunchKernelGGL(ln_bwd_long_kernel<T>, dim3(p.blocks), dim3(STREAM), 0, st, a, dy, x, gamma, mean, rstd, dr, dx);
      });
  }
  if (e != hipSuccess || !sums || p.parts == 1) return e;
  return recorded(st, "layernorm_sums", 0.0, 8.0 * p.parts * s.C, [&] {
    hipLaunchKernelGGL(ln_sums_kernel, dim3((2 * a.ld + 15) / 16), dim3(CT), 0, st, part, (int)p.parts, a.ld, s.C, dgamma, dbeta);
  });
}

}  // namespace

size_t ln_workspace_bytes(const LnShape &s) {
  const LnPlan p = ln_plan(s.M, s.C, true);
  return p.parts == 1 ? 0 : (size_t)p.parts * 2 * ((s.C + 7) / 8 * 8) * 4;
}

hipError_t launch_ln_fwd(const LnShape &s, const void *x, const float *gamma, const float *beta, void *y, float *mean, float *rstd, hipStream_t st) {
  if (s.dtype == NF_BF16) return fwd_as(s, (const __bf16 *)x, gamma, beta, (__bf16 *)y, mean, rstd, st);
  if (s.dtype == NF_F16) return fwd_as(s, (const _Float16 *)x, gamma, beta, (_Float16 *)y, mean, rstd, st);
  return fwd_as(s, (const float *)x, gamma, beta, (float *)y, mean, rstd, st);
}

hipError_t launch_ln_bwd(const LnShape &s, const void *dy, const void *x, const float *gamma, const float *mean, const float *rstd, const void *dr, void *dx,
                         float *dgamma, float *dbeta, void *ws, hipStream_t st) {
  auto as = [&](auto t) {
    using T = decltype(t);
    return bwd_as<T>(s, (const T *)dy, (const T *)x, gamma, mean, rstd, (const T *)dr, (T *)dx, dgamma, dbeta, (float *)ws, st);
  };
  if (s.dtype == NF_BF16) return as((__bf16)0.f);
  if (s.dtype == NF_F16) return as((_Float16)0.f);
  return as(0.f);
}

}  // namespace nf
