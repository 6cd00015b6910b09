// Group norm over channels-last activations with an activation behind it, forward and backward.
//
// A workgroup takes a slab: W neighbouring channels of one image (whole groups), W chosen for 32 bytes of a pixel or more.  A
// thread keeps one vector of 16 bytes of channels and up to R of the slab's pixels in registers, so that memory is read once:
// the mean, the squares about the mean and the result come from the registers (two launches' worth of traffic less than
// reading again, and no cancellation between a sum of squares and a square).  Sums over the slab go through LDS as a matrix
// [pixels that the workgroup takes at once][columns], each column added by up to 64 lanes and a shuffle tree: the order is fixed.
// A slab that does not fit the registers of one workgroup (a group of more than 256 KB of an image; 128 or 64 KB backward) is
// cut into chunks of pixels and two launches: sums of every chunk, then results, whose workgroups add the chunks' sums first.
#pragma once
#include <algorithm>
#include <type_traits>

#include "nf_enqueue.h"
#include "pw_math.h"

namespace nf {
namespace {

// A vector: the 16 bytes of N neighbouring elements, held as they lie in memory.  Where rows are not whole vectors (WHOLE
// false), they start at any element and the slab's last vector has n of them; the others read as 0 and are not written.
template <typename T>
struct Vec {
  static constexpr int N = 16 / sizeof(T);
  T v[N];
};
template <typename T, bool WHOLE>
__device__ inline uintx4 load_vec(const T *p, int n) {
  uintx4 u;
  if (WHOLE) {
    u = *reinterpret_cast<const uintx4 *>(p);
  } else if (n >= Vec<T>::N) {
    __builtin_memcpy(&u, p, 16);
    asm volatile("");  // a branch of its own: its read stays whole
  } else {
    Vec<T> t;
#pragma unroll
    for (int e = 0; e < Vec<T>::N; ++e) t.v[e] = e < n ? p[e] : (T)0.f;
    u = __builtin_bit_cast(uintx4, t);
  }
  return u;
}
// To fp32.  Behind the asm the bits are numbers that the compiler has not seen: it would keep the fp32 forms from one
// pass over the registers to the next, twice the registers and more.
template <typename T>
__device__ inline void unpack(uintx4 &u, float (&f)[16 / sizeof(T)]) {
  asm volatile("" : "+v"(u));
  const Vec<T> t = __builtin_bit_cast(Vec<T>, u);
#pragma unroll
  for (int e = 0; e < Vec<T>::N; ++e) f[e] = (float)t.v[e];
}
// the same of 4 elements from element 4 h on, and back: half of the registers at a time for a 16-bit vector
template <typename T>
struct Four {
  T v[4];
};
template <typename T>
__device__ inline void unpack4(const uintx4 &u, int h, float (&f)[4]) {
  if constexpr (sizeof(T) == 4) {
    uintx4 w = u;
    unpack<T>(w, f);
  } else {
    uint32_t w0 = u[2 * h], w1 = u[2 * h + 1];
    asm volatile("" : "+v"(w0), "+v"(w1));
    const Four<T> t = __builtin_bit_cast(Four<T>, make_uint2(w0, w1));
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = (float)t.v[e];
  }
}
template <typename T>
__device__ inline void pack4(uintx4 &u, int h, const float (&f)[4]) {
  Four<T> t;
#pragma unroll
  for (int e = 0; e < 4; ++e) t.v[e] = (T)f[e];
  if constexpr (sizeof(T) == 4) {
    u = __builtin_bit_cast(uintx4, t);
  } else {
    const uint2 w = __builtin_bit_cast(uint2, t);
    u[2 * h] = w.x, u[2 * h + 1] = w.y;
  }
}
template <typename T, bool WHOLE>
__device__ inline void store_vec(T *p, const uintx4 &u, int n) {
  if (WHOLE) {
    *reinterpret_cast<uintx4 *>(p) = u;
  } else if (n >= Vec<T>::N) {
    uintx4 w = u;
    asm volatile("" : "+v"(w));  // likewise
    __builtin_memcpy(p, &w, 16);
  } else {
    const Vec<T> t = __builtin_bit_cast(Vec<T>, u);
#pragma unroll
    for (int e = 0; e < Vec<T>::N; ++e)
      if (e < n) p[e] = t.v[e];
  }
}
template <typename T, bool WHOLE>
__device__ inline void store_vec(T *p, const float (&f)[16 / sizeof(T)], int n) {
  Vec<T> t;
#pragma unroll
  for (int e = 0; e < Vec<T>::N; ++e) t.v[e] = (T)f[e];
  if (WHOLE)
    *reinterpret_cast<uintx4 *>(p) = __builtin_bit_cast(uintx4, t);
  else if (n >= Vec<T>::N)
    __builtin_memcpy(p, &t, 16);
  else
#pragma unroll
    for (int e = 0; e < Vec<T>::N; ++e)
      if (e < n) p[e] = t.v[e];
}

enum { FUSED, STATS, APPLY };  // one launch; or a chunk's sums, and the results

struct GnArgs {
  int HW, C, G, Cg, W;  // W: channels of a slab; the last of an image may have fewer
  int groups;           // of a slab
  int cv, px;           // vectors across a slab, pixels that the workgroup takes at once
  int Wp;               // W in whole vectors: the length of the channels' parameters in LDS
  int chunks, per;      // chunks of an image, pixels of a chunk
  int act;
  float eps, inv;  // inv = 1 / (Cg HW)
  int share_w, share_2w, share_g;  // log2 of the lanes that share a column of W, 2 W and `groups` columns (column_sums)
  FastDiv div_cv, div_cg, div_slabs, div_chunks, div_px;
};

// workgroups go round the 8 XCDs: neighbouring slabs, which share memory lines, go to one XCD one after the other
__device__ inline int xcd_run(int id, int n) {
  const int x = id & 7, q = n >> 3, r = n & 7;
  return x * q + min(x, r) + (id >> 3);
}

// A sum over 2^share neighbouring lanes, on all of them.  Up to 16 lanes the partners lie in a row of 16, which the vector
// ALU's operand paths reach.
template <int CTRL>
__device__ inline float row_partner(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true));
}
__device__ inline float lanes_sum(float v, int share) {
  if (share >= 1) v += row_partner<0xB1>(v);   // the other of two
  if (share >= 2) v += row_partner<0x4E>(v);   // the other two of four
  if (share >= 3) v += row_partner<0x141>(v);  // the other half of eight, mirrored: its four lanes hold one sum
  if (share >= 4) v += row_partner<0x140>(v);  // the other half of sixteen
  if (share >= 5) v += __shfl_xor(v, 16);
  if (share >= 6) v += __shfl_xor(v, 32);
  return v;
}

// out[c] = sum over rows of buf[row * pitch + c * step]; all threads take part.  2^share lanes share a column.
__device__ inline void column_sums(const float *buf, int rows, int cols, int pitch, int step, int share, float *out) {
  const int k = threadIdx.x & ((1 << share) - 1), across = blockDim.x >> share;
  for (int c = threadIdx.x >> share; c < cols; c += across) {
    float s = 0.f;
    for (int r = k; r < rows; r += 1 << share) s += buf[r * pitch + c * step];
    s = lanes_sum(s, share);
    if (k == 0) out[c] = s;
  }
}

// a thread's channels' parameters
template <int N>
__device__ inline void read_channels(const float *lds, float (&f)[N]) {
#pragma unroll
  for (int e = 0; e < N; e += 4) {
    const floatx4 q = *reinterpret_cast<const floatx4 *>(lds + e);
#pragma unroll
    for (int k = 0; k < 4; ++k) f[e + k] = q[k];
  }
}

// Sums of the slab's groups from the threads' sums of their channels.  ONE: a vector lies in one group.
// gsum[groups] is ready behind the last barrier; buf [px][cv or W, odd pitch], csum[W].
// W, groups: this slab's.
template <int VEC, bool ONE>
__device__ inline void group_sums(const GnArgs &a, int W, int groups, int pr, int cl, const float s[VEC], float *buf, float *csum, float *gsum) {
  __syncthreads();  // the buffers may still be read
  if constexpr (ONE) {
    const int vg = a.Cg / VEC, c = cl / VEC, g = a.div_cg.div(cl);  // vectors of a group; rows are (pixel, vector of the group)
    float t = 0.f;
#pragma unroll
    for (int e = 0; e < VEC; ++e) t += s[e];
    if (pr < a.px && cl < W) buf[(pr * vg + c - g * vg) * (a.groups | 1) + g] = t;
    __syncthreads();
    column_sums(buf, a.px * vg, groups, a.groups | 1, 1, a.share_g, gsum);
  } else {
    if (pr < a.px) {
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        if (cl + e < W) buf[pr * (a.W | 1) + cl + e] = s[e];
    }
    __syncthreads();
    column_sums(buf, a.px, W, a.W | 1, 1, a.share_w, csum);
    __syncthreads();
    column_sums(csum, a.Cg, groups, 1, a.Cg, a.share_g, gsum);
  }
  __syncthreads();
}

// floats of the matrix and the channels' sums
inline int matrix_floats(const GnArgs &a, int vec, bool one) { return one ? a.px * (a.Cg / vec) * (a.groups | 1) : a.px * (a.W | 1) + a.W; }

int gcd(int a, int b) {
  while (b) {
    const int t = a % b;
    a = b, b = t;
  }
  return a;
}

constexpr int TINY = 512;  // vectors of a slab that get a thread each

struct GnPlan {
  GnArgs a;
  bool whole, one, split, tiny, small;
  int nt, slabs;
};

// The slab: whole groups (and whole vectors, where rows are; a unit of both wider than 2048 channels gives way to single groups),
// at most 128 bytes of a pixel, 64 or 32 where 128 leave fewer than 512 workgroups.  Threads: enough for 4 pixels each on slabs
// of up to 64 KB, else 8, up to what the registers hold.
GnPlan gn_plan(const GnShape &s, bool backward) {
  const int size = s.dtype == NF_F32 ? 4 : 2, vec = 16 / size;
  GnPlan p;
  GnArgs &a = p.a;
  a.HW = s.HW, a.C = s.C, a.G = s.G, a.Cg = s.C / s.G, a.act = s.act, a.eps = s.eps;
  a.inv = (float)(1.0 / ((double)a.Cg * a.HW));
  int unit = a.Cg / gcd(a.Cg, vec) * vec;
  p.whole = s.C % vec == 0 && unit <= 2048;
  if (!p.whole) unit = a.Cg;
  p.one = p.whole && a.Cg % vec == 0;
  const int most = backward ? (p.one ? 8 : 4) : 16;  // pixels that a thread's registers hold
  auto across = [&](int W) { return (W + vec - 1) / vec; };
  auto fits = [&](int W) {  // the registers of 1024 threads, and 31 bits of offset
    return (long long)(1024 / across(W)) * most >= s.HW && (long long)s.HW * s.C * size < (1ll << 31);
  };
  const int units = s.C / unit;
  auto slabs = [&](int m) { return (units + m - 1) / m; };
  int m = 1;
  for (int k = 2; k <= units && k * unit * size <= 128; ++k)
    if (fits(k * unit) && slabs(k) < slabs(m)) m = k;
  while (m > 1 && (long long)s.B * slabs(m) < 512 && (m + 1) / 2 * unit * size >= 32) m = (m + 1) / 2;
  a.W = m * unit, a.groups = a.W / a.Cg, a.cv = across(a.W), a.Wp = a.cv * vec;
  p.split = !fits(a.W);
  int pixels = s.HW;
  a.chunks = 1;
  if (p.split) {
    // pixels of a chunk: what 1024 threads hold, fewer where that leaves fewer than 512 workgroups; 30 bits of offset
    const int at_once = 1024 / a.cv;
    int deep = std::min(most, 8);
    while (deep > 1 && (long long)s.B * slabs(m) * ((s.HW + at_once * deep - 1) / (at_once * deep)) < 512) --deep;
    a.per = (int)std::min<long long>(at_once * deep, std::max<long long>(1, (1ll << 30) / ((long long)s.C * size)));
    a.chunks = (s.HW + a.per - 1) / a.per;
    a.per = (s.HW + a.chunks - 1) / a.chunks;
    a.chunks = (s.HW + a.per - 1) / a.per;
    pixels = a.per;
  } else {
    a.per = s.HW;
  }
  const long long vectors = (long long)pixels * a.cv;
  const int aim = std::min(most, vectors <= TINY ? 1 : vectors <= 4096 ? 4 : 8);
  p.nt = 1024;
  for (int nt = 64; nt < 1024; nt += 64)
    if (nt >= a.cv && (long long)(nt / a.cv) * aim >= pixels) {
      p.nt = nt;
      break;
    }
  a.px = p.nt / a.cv;
  p.tiny = !p.split && p.nt <= TINY && a.px >= s.HW;
  p.small = !p.split && p.nt <= 256 && (long long)a.px * 4 >= s.HW;
  p.slabs = slabs(m);
  auto share = [&](int cols) {  // all threads have a column, as far as 64 lanes to each go
    int k = 6;
    while (k > 0 && (cols << k) > p.nt) --k;
    return k;
  };
  a.share_w = share(a.W), a.share_2w = share(2 * a.W), a.share_g = share(a.groups);
  a.div_cv = FastDiv(a.cv), a.div_cg = FastDiv(a.Cg), a.div_slabs = FastDiv(p.slabs), a.div_chunks = FastDiv(a.chunks), a.div_px = FastDiv(a.px);
  return p;
}

// names of the slab kernels: a group to a vector, several, rows of any alignment
enum { TINY_SLAB, SMALL_SLAB, SLAB, SLAB_STATS, SLAB_APPLY };
using SlabNames = const char *const[5][3];
template <typename T>
double gn_bytes(const GnShape &s, double passes) {  // passes: tensors read and written
  return passes * sizeof(T) * s.B * s.HW * s.C;
}

template <typename T, typename F>
hipError_t by_rows(const GnPlan &p, F run) {
  if (p.one) return run((T)0.f, std::true_type(), std::true_type());
  if (p.whole) return run((T)0.f, std::true_type(), std::false_type());
  return run((T)0.f, std::false_type(), std::false_type());
}
template <typename F>
hipError_t by_type(const GnShape &s, const GnPlan &p, F run) {
  if (s.dtype == NF_BF16) return by_rows<__bf16>(p, run);
  if (s.dtype == NF_F16) return by_rows<_Float16>(p, run);
  return by_rows<float>(p, run);
}

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

// ---- small groups ----
// A wave (four of them to a workgroup) or a workgroup of 256 or 1024 threads to a group, an element to a thread: threads go over the
// group's channels first, then over `px` pixels, and up to FEW_R times further.  What a short launch waits for is mostly its
// instructions' first fetch (a launch that does next to nothing takes 1.6 us, the slab kernels 5 to 7), and this is a fifth of
// their code: 3x3x17 fp32 4.9 -> 2.0 us, 13x23x16 7.1 -> 3.1.
constexpr int FEW_R = 16;
struct GnFew {
  int HW, C, G, Cg, px, units, act;
  int threads;  // of a group: 64, 256 or 1024
  int share;    // log2 of the threads that add up a channel's sums
  float eps, inv;
  FastDiv div_cg, div_g, div_px;
};
// What a call takes this way and in slabs, in us with the launch, by least squares over 48000 calls (24000 shapes of 2^16 to 2^21
// elements; one standard deviation is 9 to 17 %): turns of a thread; thousands of waves times turns, more of them beyond 8 and with several waves
// to a group; the same by how short a pixel's run is.  Slabs: turns, which SiLU and GELU lengthen; thousands of waves times turns; turns of the sums over
// groups (backward).  By them the choice is on average 2 % behind the faster of the two and 4 % faster than one limit of 1.5 * 2^20 elements:
//   256x128 in 32 groups fp32, 48 images     forward 13.8 and in slabs 6.7    gradients 22.7 and 10.7
//   100x48 in 4 bf16, 109 and 218 images     4.9 and 5.9, 7.3 and 6.4         7.9 and 8.4, 12.9 and 9.1
//   16x512 in 32 fp32, 192 images            5.6 and 6.5                      9.4 and 11.2
//   905x64 in 8 bf16 with GELU, 7 images, 28 slabs                            10.7 and 14.9
inline double few_time(const GnFew &a, int pixel_bytes, bool backward) {
  constexpr double T[2][5] = {{5.3, 0.11, 0.04, 0.026, 0.044}, {8.5, 0.09, 0.035, 0.12, 0.068}};
  const double *t = T[backward];
  const int turns = (a.HW + a.px - 1) / a.px;
  const double work = (double)a.units * (a.threads / 64) * turns * 1e-3;
  return t[0] + t[1] * turns + (a.threads > 64 ? t[2] * work + t[3] * std::max(0.0, work - 8) : 0.0) + t[4] * work * std::min(16.0 / pixel_bytes, 4.0);
}
inline double slab_time(const GnPlan &p, int images, bool backward) {
  constexpr double T[2][3][5] = {{{5.8, 0.23, 0.25, 0.14, 0}, {5.5, 0.49, 0.41, 0.24, 0}, {5.4, 0.9, 0.32, 0.25, 0}},
                                 {{8.7, 0.15, 0.5, 0.39, 0.165}, {8, 0.4, 0.55, 0.46, 0.19}, {8.1, 0.8, 0.5, 0.55, 0.19}}};
  const double *t = T[backward][p.one ? 0 : p.whole ? 1 : 2];
  const GnArgs &a = p.a;
  const int turns = p.split ? 4 : (a.HW + a.px - 1) / a.px, waves = p.nt / 64;
  const double groups = (double)images * p.slabs * (p.split ? (double)a.HW / (4.0 * a.px) : 1.0);
  return t[0] + (t[1] + (a.act >= NF_ACT_SILU ? t[2] : 0.0)) * turns + t[3] * groups * waves * turns * 1e-3 + t[4] * ((2 * a.groups + waves - 1) / waves);
}
// Whether a shape goes this way: groups of up to 16 elements a thread, up to 1.5 * 2^20 in all (beyond, slabs were faster or within 10 %); always up
// to 2^16, where a call is its launch and first fetches
inline bool gn_few(const GnShape &s, bool backward, const GnPlan &slabs, GnFew *a) {
  a->HW = s.HW, a->C = s.C, a->G = s.G, a->Cg = s.C / s.G, a->act = s.act, a->eps = s.eps;
  const long long elements = (long long)s.B * s.HW * s.C;
  if (elements > 3 << 19) return false;
  a->threads = 0;
  // few elements a thread, or the most threads
  for (int nt : {64, 256, 1024})
    if (a->Cg <= nt && s.HW <= (nt == 1024 ? FEW_R : 4) * (nt / a->Cg)) {
      a->threads = nt;
      break;
    }
  if (!a->threads) return false;
  a->px = a->threads / a->Cg;
  a->share = 6;
  while (a->share > 0 && (a->Cg << a->share) > a->threads) --a->share;
  a->units = s.B * s.G;
  a->inv = (float)(1.0 / ((double)a->Cg * s.HW));
  a->div_cg = FastDiv(a->Cg), a->div_g = FastDiv(s.G), a->div_px = FastDiv(a->px);
  return elements <= 1 << 16 || few_time(*a, a->Cg * (s.dtype == NF_F32 ? 4 : 2), backward) <= slab_time(slabs, s.B, backward);
}
// run(threads of a group, elements of a thread, workgroups, their threads), recorded under one of the names
template <typename F>
hipError_t gn_few_variant(const GnFew &a, const char *const (&names)[4], double bytes, hipStream_t st, F run) {
  const int k = a.threads == 64 ? 0 : a.threads == 256 ? 1 : a.HW <= 4 * a.px ? 2 : 3;
  return recorded(st, names[k], 0.0, bytes, [&] {
    if (k == 0)
      run(std::integral_constant<int, 64>(), std::integral_constant<int, 4>(), dim3((a.units + 3) / 4), dim3(256));
    else if (k == 1)
      run(std::integral_constant<int, 256>(), std::integral_constant<int, 4>(), dim3(a.units), dim3(256));
    else if (k == 2)
      run(std::integral_constant<int, 1024>(), std::integral_constant<int, 4>(), dim3(a.units), dim3(1024));
    else
      run(std::integral_constant<int, 1024>(), std::integral_constant<int, FEW_R>(), dim3(a.units), dim3(1024));
  });
}
// the sum over a group's threads, on all of them; `slot` differs from one call of a kernel to the next
template <int NT>
__device__ inline float few_sum(float v, int slot) {
  v = lanes_sum(v, 6);
  if constexpr (NT > 64) {
    __shared__ float parts[2][NT / 64];
    if ((threadIdx.x & 63) == 0) parts[slot][threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) v += parts[slot][w];
  }
  return v;
}

}  // namespace
}  // namespace nf
