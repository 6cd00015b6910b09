// Matrices made orthogonal by Newton-Schulz steps, and weights updated with them.
//   X0 = G / (|G| + eps);  X' = a X + (b A + c A^2) X,  A = X X^T over the shorter side
// The steps amplify errors (by a^steps where singular values are small: 485 for 5 steps of a = 3.4445), so products keep fp32's digits: every
// matrix is held as two fp16 pieces, h + l = v 2^s to 22 bits, and a product is h h + h l + l h on the fp16 matrix instructions, summed in fp32.  That is
// three products at 1.4 PFLOP/s where the fp32 instructions reach 150 TFLOP/s.  s is chosen from a bound of the singular values after each step
// (orth_scales), so that the largest element fits fp16 and what falls below its smallest is 2^-39 of that.
//   layout   [row][32 columns' h, their l]: a row's step of 32 columns is 128 bytes; sides are padded with zeros to whole tiles
//   a step   A = X X^T and P = b A + c A^2, both symmetric: the tiles on and above the diagonal, each written twice; X' = a X + P X
//   a long side lies along the columns: a tall G is held transposed and written back so
// All matrices of a call share the launches.
#include <algorithm>
#include <cmath>

#include "linear.h"
#include "nf_enqueue.h"
#include "orth.h"

namespace nf {
namespace {

using halfx4 = __attribute__((ext_vector_type(4))) _Float16;
using f16x8 = __attribute__((ext_vector_type(8))) _Float16;
using shortx4 = __attribute__((ext_vector_type(4))) short;

constexpr int MOST = NF_ORTH_MATRICES;

struct Item {
  long long x[2], A, P, part, squares;  // bytes from the workspace's start
  int rows, cols, n, m, np, mp;         // n <= m, padded; rows > cols: held transposed
  int splits, per;                      // of A's sums: parts, and their steps of 32 terms
  int square_parts, chunk;              // of |G|^2
};
struct Args {
  char *ws;
  int count, cur;
  int first[MOST + 1];  // first workgroup of each matrix
  Item it[MOST];
  float a, b, c, eps;
  float up_x, down_x, up_a, down_a, up_p, down_p, up_next;  // 2^s and 2^-s of X, A, P and X'
};
struct Tensors {
  const void *g[MOST];
  float *v[MOST];
  void *y[MOST];
  float momentum, keep, lr;  // y = keep y - lr sqrt(max(1, rows / cols)) X
  int nesterov;
};

// the matrix that a workgroup works on: the last whose first workgroup is not behind it
__device__ inline int item_of(const Args &a, int id) {
  const int lane = threadIdx.x & 63;
  const bool at = lane < a.count && a.first[lane < MOST ? lane : MOST] <= id;
  return __popcll(__ballot(at)) - 1;
}

// element (r, c) of a matrix in pieces: its h, and its l 64 bytes further
__device__ inline char *piece(char *p, long long ld, long long r, int c) { return p + r * ld + (c >> 5) * 128 + (c & 31) * 2; }
template <typename V>
__device__ inline void split(float v, V &h, V &l) {
  h = (_Float16)v;
  l = (_Float16)(v - (float)h);
}
__device__ inline void load4(const char *p, float (&v)[4]) {
  const halfx4 h = *reinterpret_cast<const halfx4 *>(p), l = *reinterpret_cast<const halfx4 *>(p + 64);
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = (float)h[e] + (float)l[e];
}
__device__ inline void store4(char *p, const float (&v)[4]) {
  halfx4 h, l;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    _Float16 x, y;
    split(v[e], x, y);
    h[e] = x, l[e] = y;
  }
  *reinterpret_cast<halfx4 *>(p) = h, *reinterpret_cast<halfx4 *>(p + 64) = l;
}
__device__ inline void store1(char *p, float v) {
  _Float16 h, l;
  split(v, h, l);
  *reinterpret_cast<_Float16 *>(p) = h, *reinterpret_cast<_Float16 *>(p + 64) = l;
}

// ---- |G|^2, and the momentum ----
constexpr int NT = 256;
// A sum over the workgroup, on its first thread; sums of squares are held in 64 bits, which no fp32 number's square leaves.
__device__ inline double all_sum(double v, double *lds) {
#pragma unroll
  for (int k = 32; k; k >>= 1) v += __shfl_xor(v, k);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  return lds[0] + lds[1] + lds[2] + lds[3];
}
// What is made orthogonal: G, or the momentum's direction (v holds the new momentum already).
template <typename T, bool MUON>
__device__ inline float direction(const Tensors &t, const T *g, const float *v, long long at) {
  if constexpr (!MUON) return (float)g[at];
  const float gv = (float)g[at];
  if (!v) return gv;
  return t.nesterov ? fmaf(t.momentum, v[at], gv) : v[at];
}
template <typename T, bool MUON>
__global__ __launch_bounds__(NT) void orth_squares_kernel(Args a, Tensors t) {
  __shared__ double lds[4];
  const int k = item_of(a, blockIdx.x);
  const Item &it = a.it[k];
  const int part = blockIdx.x - a.first[k];
  const T *const g = (const T *)t.g[k];
  float *const v = MUON ? t.v[k] : nullptr;
  const long long all = (long long)it.rows * it.cols, from = (long long)part * it.chunk, to = min(all, from + it.chunk);
  double s = 0;
  for (long long i = from + threadIdx.x * 8; i < to; i += NT * 8) {
    const int n = (int)min(to - i, 8ll);
    float x[8];
    load8(g + i, x, n);
    if constexpr (MUON) {
      if (v) {
        float m[8];
        load8(v + i, m, n);
#pragma unroll
        for (int e = 0; e < 8; ++e) m[e] = fmaf(t.momentum, m[e], x[e]), x[e] = t.nesterov ? fmaf(t.momentum, m[e], x[e]) : m[e];
        store8(v + i, m, n);
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) s += e < n ? (double)x[e] * x[e] : 0.0;
  }
  s = all_sum(s, lds);
  if (threadIdx.x == 0) reinterpret_cast<double *>(a.ws + it.squares)[part] = s;
}

// X0 in pieces, a tile of 64 x 64 to a workgroup
template <typename T, bool MUON>
__global__ __launch_bounds__(NT) void orth_start_kernel(Args a, Tensors t) {
  __shared__ double lds[4];
  __shared__ float tile[64][65];
  const int k = item_of(a, blockIdx.x);
  const Item &it = a.it[k];
  const int id = blockIdx.x - a.first[k], across = it.mp / 64, tr = id / across, r0 = tr * 64, c0 = (id - tr * across) * 64;
  double s = 0;
  const double *const squares = reinterpret_cast<const double *>(a.ws + it.squares);
  for (int i = threadIdx.x; i < it.square_parts; i += NT) s += squares[i];
  const float norm = (float)sqrt(all_sum(s, lds)) + a.eps;
  const T *const g = (const T *)t.g[k];
  const float *const v = MUON ? t.v[k] : nullptr;
  const int x = threadIdx.x & 63, y = threadIdx.x >> 6;
  const bool tall = it.rows > it.cols;
  for (int i = y; i < 64; i += 4) {  // along G's rows
    const int row = (tall ? c0 : r0) + i, col = (tall ? r0 : c0) + x;
    const float w = row < it.rows && col < it.cols ? direction<T, MUON>(t, g, v, (long long)row * it.cols + col) / norm * a.up_x : 0.f;
    (tall ? tile[x][i] : tile[i][x]) = w;
  }
  __syncthreads();
  char *const X = a.ws + it.x[0];
  for (int i = threadIdx.x; i < 1024; i += NT) {
    const int r = i >> 4, c = (i & 15) * 4;
    const float w[4] = {tile[r][c], tile[r][c + 1], tile[r][c + 2], tile[r][c + 3]};
    store4(piece(X, 4ll * it.mp, r0 + r, c0 + c), w);
  }
}

// ---- products ----
enum { GRAM, POLY, APPLY, LAST };

template <int BLOCK>
struct Tile {
  static constexpr int BYTES = BLOCK * 128, STAGE = 2 * BYTES, PIECES = BLOCK / 32;
  static constexpr int ROWB = BLOCK * 4, CPR = ROWB / 16;  // of an operand whose terms lie apart: a term's row
};
// chunks of 16 bytes of a row, and units of 32 bytes of a term's row, are exchanged so that what is read together lies in different banks
__device__ inline int chunk_swizzle(int row) { return (row >> 1) & 7; }
__device__ inline int unit_swizzle(int term) { return (term & 3) | ((term >> 3) & 1) << 2; }

// rows rb .. rb+15 of an operand, piece pl: lane l has 8 terms 8 (l / 16) .. of row l % 16
template <int BLOCK, bool APART>
__device__ inline f16x8 fragment(const char *lds, int rb, int pl, int lane) {
  const int i = lane & 15, q = lane >> 4;
  if constexpr (!APART) {
    const int row = rb + i;
    return *reinterpret_cast<const f16x8 *>(lds + row * 128 + (((pl * 4 + q) ^ chunk_swizzle(row)) << 4));
  } else {
    uintx4 f;
    const int unit = (rb >> 5) * 4 + pl * 2 + ((rb >> 4) & 1);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int term = q * 8 + h * 4 + (i >> 2);
      const char *p = lds + term * Tile<BLOCK>::ROWB + ((unit ^ unit_swizzle(term)) << 5) + (i & 3) * 8;
      const uint2 t = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) shortx4 *)p));
      f[2 * h] = t.x, f[2 * h + 1] = t.y;
    }
    return __builtin_bit_cast(f16x8, f);
  }
}

// Finished sums, 4 neighbours of a row, to where they go.
template <int KIND, typename OUT, bool MUON>
__device__ inline void finish4(const Args &a, const Tensors &t, const Item &it, int k, int r, int c, bool mirror, float (&v)[4]) {
  if constexpr (KIND == GRAM) {
    const float s = a.down_x * a.down_x * a.up_a;
    char *const A = a.ws + it.A;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] *= s;
    store4(piece(A, 4ll * it.np, r, c), v);
    if (mirror) {
#pragma unroll
      for (int e = 0; e < 4; ++e) store1(piece(A, 4ll * it.np, c + e, r), v[e]);
    }
  } else if constexpr (KIND == POLY) {
    float A[4];
    load4(piece(a.ws + it.A, 4ll * it.np, r, c), A);
    const float sa = a.b * a.down_a * a.up_p, ss = a.c * a.down_a * a.down_a * a.up_p;
    char *const P = a.ws + it.P;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = fmaf(A[e], sa, v[e] * ss);
    store4(piece(P, 4ll * it.np, r, c), v);
    if (mirror) {
#pragma unroll
      for (int e = 0; e < 4; ++e) store1(piece(P, 4ll * it.np, c + e, r), v[e]);
    }
  } else {
    float X[4];
    load4(piece(a.ws + it.x[a.cur], 4ll * it.mp, r, c), X);
    const float up = KIND == LAST ? 1.f : a.up_next, sx = a.a * a.down_x * up, ss = a.down_p * a.down_x * up;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = fmaf(X[e], sx, v[e] * ss);
    if constexpr (KIND == APPLY) {
      store4(piece(a.ws + it.x[a.cur ^ 1], 4ll * it.mp, r, c), v);
    } else {
      const bool tall = it.rows > it.cols;
      const float shape = tall ? sqrtf((float)it.rows / (float)it.cols) : 1.f;
      if (r >= it.n) return;
      OUT *const y = (OUT *)t.y[k];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (c + e >= it.m) continue;
        const long long at = tall ? (long long)(c + e) * it.cols + r : (long long)r * it.cols + c + e;
        if constexpr (MUON)
          y[at] = fmaf(-t.lr * shape, v[e], t.keep * (float)y[at]);
        else
          y[at] = (OUT)v[e];
      }
    }
  }
}

// The tile t of those on and above the diagonal, column by column.
__device__ inline void triangle(int t, int &tr, int &tc) {
  tc = (int)((sqrtf(8.f * t + 1.f) - 1.f) * 0.5f);
  while ((tc + 1) * (tc + 2) / 2 <= t) ++tc;
  while (tc * (tc + 1) / 2 > t) --tc;
  tr = t - tc * (tc + 1) / 2;
}

// BLOCK x BLOCK results by four waves of BLOCK/2 x BLOCK/2; a step is 32 terms.  STAGES of them are in flight: one barrier a step, behind which its
// stage is whole and the one before it free.  Steps beyond the last are copies of nothing, so that the waits count the same.
template <int BLOCK, int STAGES, int KIND, typename OUT, bool MUON>
__global__ __launch_bounds__(LT) void orth_product_kernel(Args a, Tensors t) {
  using S = Tile<BLOCK>;
  constexpr bool APART = KIND >= APPLY;
  constexpr int MT = BLOCK / 32, PIECES = S::PIECES;
  __shared__ __align__(1024) char lds[STAGES * S::STAGE];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i16 = lane & 15, q = lane >> 4;
  const int k = __builtin_amdgcn_readfirstlane(item_of(a, blockIdx.x));
  const Item &it = a.it[k];
  int id = blockIdx.x - a.first[k], split = 0, tr, tc;
  if constexpr (KIND <= POLY) {
    const int T = it.np / BLOCK, tiles = T * (T + 1) / 2;
    if (KIND == GRAM) split = id / tiles, id -= split * tiles;
    triangle(id, tr, tc);
  } else {
    const int down = it.np / BLOCK;
    tc = id / down, tr = id - tc * down;
  }
  const long long ld_a = 4ll * (KIND == GRAM ? it.mp : it.np), ld_b = 4ll * (KIND == POLY ? it.np : it.mp);
  const char *const A = a.ws + (KIND == GRAM ? it.x[a.cur] : KIND == POLY ? it.A : it.P) + (long long)tr * BLOCK * ld_a;
  const char *const B = a.ws + (KIND == POLY ? it.A : it.x[a.cur]) + (APART ? (long long)tc * BLOCK * 4 : (long long)tc * BLOCK * ld_b);
  const int all = (KIND == GRAM ? it.mp : it.np) / 32, s0 = KIND == GRAM ? split * it.per : 0, steps = KIND == GRAM ? min(it.per, all - s0) : all;
  uint32_t av[PIECES], bv[PIECES];
#pragma unroll
  for (int p = 0; p < PIECES; ++p) {
    const int at = (p * 4 + wave) * 64 + lane, row = at >> 3;
    av[p] = (uint32_t)(row * ld_a) + (((at & 7) ^ chunk_swizzle(row)) << 4);
    if (APART) {
      const int term = at / S::CPR, c = at % S::CPR;
      bv[p] = (uint32_t)(term * ld_b) + ((c ^ (unit_swizzle(term) << 1)) << 4);
    } else {
      bv[p] = (uint32_t)(row * ld_b) + (((at & 7) ^ chunk_swizzle(row)) << 4);
    }
  }
  const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds;
  auto fetch = [&](int s, int stage) {
    const uintx4 ba = buffer_of(A + (s0 + s) * 128ll), bb = buffer_of(B + (APART ? (long long)s * 32 * ld_b : (s0 + s) * 128ll));
    const uint32_t to = base + stage * S::STAGE + wave * 1024;
    const bool live = s < steps;
#pragma unroll
    for (int p = 0; p < PIECES; ++p) copy16(ba, live ? av[p] : OUTSIDE, to + p * 4096);
#pragma unroll
    for (int p = 0; p < PIECES; ++p) copy16(bb, live ? bv[p] : OUTSIDE, to + S::BYTES + p * 4096);
  };
  const int wm = (wave >> 1) * (BLOCK / 2), wn = (wave & 1) * (BLOCK / 2);
  floatx4 acc[MT][MT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < MT; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int s = 0; s < STAGES - 1; ++s) fetch(s, s);
  int stage = 0;
  for (int s = 0; s < steps; ++s) {
    wait_copies<(STAGES - 2) * 2 * PIECES>();
    wait_lds();
    barrier();
    fetch(s + STAGES - 1, stage == 0 ? STAGES - 1 : stage - 1);
    const char *const la = lds + stage * S::STAGE, *const lb = la + S::BYTES;
    f16x8 fa[MT][2], fb[MT][2];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int pl = 0; pl < 2; ++pl) fa[i][pl] = fragment<BLOCK, false>(la, wm + 16 * i, pl, lane), fb[i][pl] = fragment<BLOCK, APART>(lb, wn + 16 * i, pl, lane);
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < MT; ++j) {
        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(fb[j][0], fa[i][1], acc[i][j], 0, 0, 0);
        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(fb[j][1], fa[i][0], acc[i][j], 0, 0, 0);
        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(fb[j][0], fa[i][0], acc[i][j], 0, 0, 0);
      }
    stage = stage + 1 == STAGES ? 0 : stage + 1;
  }
  wait_copies<0>();
  // a lane has 4 neighbouring columns of a row
  float *const part = KIND == GRAM && it.splits > 1 ? reinterpret_cast<float *>(a.ws + it.part) + (long long)(blockIdx.x - a.first[k]) * BLOCK * BLOCK : nullptr;
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < MT; ++j) {
      const int r = wm + 16 * i + i16, c = wn + 16 * j + 4 * q;
      if (KIND == GRAM && part) {
        *reinterpret_cast<floatx4 *>(part + r * BLOCK + c) = acc[i][j];
      } else {
        float v[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
        finish4<KIND, OUT, MUON>(a, t, it, k, tr * BLOCK + r, tc * BLOCK + c, tr != tc, v);
      }
    }
}

// the parts of A's sums, in order; 4 neighbours of a row to a thread
template <int BLOCK>
__global__ __launch_bounds__(LT) void orth_parts_kernel(Args a) {
  constexpr int WGS = BLOCK * BLOCK / 4 / LT;  // workgroups of a tile
  const int k = __builtin_amdgcn_readfirstlane(item_of(a, blockIdx.x));
  const Item &it = a.it[k];
  const int id = blockIdx.x - a.first[k], tile = id / WGS, i = (id - tile * WGS) * LT + threadIdx.x, r = i / (BLOCK / 4), c = i % (BLOCK / 4) * 4;
  const int T = it.np / BLOCK, tiles = T * (T + 1) / 2;
  int tr, tc;
  triangle(tile, tr, tc);
  const float *const part = reinterpret_cast<const float *>(a.ws + it.part) + (long long)tile * BLOCK * BLOCK + r * BLOCK + c;
  floatx4 s = *reinterpret_cast<const floatx4 *>(part);
#pragma unroll 4
  for (int z = 1; z < it.splits; ++z) s += *reinterpret_cast<const floatx4 *>(part + (long long)z * tiles * BLOCK * BLOCK);
  float v[4] = {s[0], s[1], s[2], s[3]};
  const Tensors none = {};
  finish4<GRAM, float, false>(a, none, it, k, tr * BLOCK + r, tc * BLOCK + c, tr != tc, v);
}

// ---- plans ----
struct Plan {
  Args a;
  int block;
  bool parts;
  size_t bytes;
};

inline long long triangle_tiles(const Item &it, int block) {
  const long long T = it.np / block;
  return T * (T + 1) / 2;
}

Plan plan_of(const nf_orth_desc &d, int count, const int32_t *rows, const int32_t *cols) {
  Plan p = {};
  Args &a = p.a;
  a.count = count, a.eps = d.eps;
  long long tiles = 0;
  for (int k = 0; k < count; ++k) {
    const long long n = std::min(rows[k], cols[k]), T = (n + 127) / 128;
    tiles += T * (T + 1) / 2;
  }
  p.block = tiles >= 128 ? 128 : 64;
  const int B = p.block;
  long long work = 0;
  for (int k = 0; k < count; ++k) {
    Item &it = a.it[k];
    it.rows = rows[k], it.cols = cols[k], it.n = std::min(rows[k], cols[k]), it.m = std::max(rows[k], cols[k]);
    it.np = (it.n + B - 1) / B * B, it.mp = (it.m + B - 1) / B * B;
    const long long all = (long long)it.rows * it.cols;
    it.chunk = 8192;
    while ((all + it.chunk - 1) / it.chunk > 1024) it.chunk *= 2;
    it.square_parts = (int)((all + it.chunk - 1) / it.chunk);
    work += triangle_tiles(it, B) * (it.mp / 32);
  }
  // parts of A's sums: towards 512 workgroups of the same length, 16 steps each at least
  const int each = (int)std::max<long long>(16, (work + 511) / 512);
  size_t at = 0;
  auto take = [&](size_t n) {
    const size_t was = at;
    at = (at + n + 255) / 256 * 256;
    return (long long)was;
  };
  for (int k = 0; k < count; ++k) {
    Item &it = a.it[k];
    const int steps = it.mp / 32;
    it.splits = std::max(1, (steps + each / 2) / each);
    it.per = (steps + it.splits - 1) / it.splits, it.splits = (steps + it.per - 1) / it.per;
    it.x[0] = take(4ull * it.np * it.mp), it.x[1] = take(4ull * it.np * it.mp);
    it.A = take(4ull * it.np * it.np), it.P = take(4ull * it.np * it.np);
    it.squares = take(8ull * it.square_parts);
    it.part = it.splits > 1 ? take(4ull * it.splits * triangle_tiles(it, B) * B * B) : 0;
    p.parts |= it.splits > 1;
  }
  p.bytes = at;
  return p;
}

// fills the first workgroups; returns their number
template <typename F>
unsigned lay(Args &a, F workgroups) {
  long long at = 0;
  for (int k = 0; k < a.count; ++k) a.first[k] = (int)at, at += workgroups(a.it[k]);
  a.first[a.count] = (int)at;
  return (unsigned)at;
}

template <int KIND, typename OUT, bool MUON>
hipError_t product(Plan &p, const Tensors &t, const char *name128, const char *name64, hipStream_t st) {
  const int B = p.block;
  double flops = 0;
  const unsigned grid = lay(p.a, [&](const Item &it) -> long long {
    const double side = KIND == POLY ? it.n : it.m;
    flops += (KIND <= POLY ? 1.0 : 2.0) * it.n * it.n * side;
    if (KIND == GRAM) return triangle_tiles(it, B) * it.splits;
    if (KIND == POLY) return triangle_tiles(it, B);
    return (long long)(it.np / B) * (it.mp / B);
  });
  return recorded(st, B == 128 ? name128 : name64, flops, 0.0, [&] {
    if (B == 128)
      hipLaunchKernelGGL((orth_product_kernel<128, 2, KIND, OUT, MUON>), dim3(grid), dim3(LT), 0, st, p.a, t);
    else
      hipLaunchKernelGGL((orth_product_kernel<64, 4, KIND, OUT, MUON>), dim3(grid), dim3(LT), 0, st, p.a, t);
  });
}

// The exponents s of X, A, P and X' at every step, from a bound u of the singular values: |x| <= u, elements of A are at most u^2, of P = b A + c A^2
// the largest |b y + c y^2| over y <= u^2, and the next u is the largest |f(x)| over x <= u.  Extremes lie at the ends or where the slope is 0.
struct Scales {
  int x, a, p;
};
bool orth_scales(const nf_orth_desc &d, Scales *s, int *last) {
  double u = 1;
  auto exponent = [](double bound) { return 15 - (int)std::ceil(std::log2(std::max(bound * 1.01, 1e-12))); };
  for (int k = 0; k <= d.steps; ++k) {
    if (!(u < 1e9)) return false;
    if (k == d.steps) {
      *last = exponent(u);
      return true;
    }
    const double a = d.a[k], b = d.b[k], c = d.c[k], y1 = u * u;
    if (!std::isfinite(a) || !std::isfinite(b) || !std::isfinite(c)) return false;
    double p = 0, f = 0;
    auto see = [&](double y) {
      if (!(y >= 0 && y <= y1)) return;
      p = std::max(p, std::fabs(b * y + c * y * y));
      f = std::max(f, std::fabs(std::sqrt(y) * (a + b * y + c * y * y)));
    };
    see(y1);
    if (c != 0) see(-b / (2 * c));
    if (c != 0) {
      const double disc = 9 * b * b - 20 * a * c;
      if (disc >= 0) see((-3 * b + std::sqrt(disc)) / (10 * c)), see((-3 * b - std::sqrt(disc)) / (10 * c));
    } else if (b != 0) {
      see(-a / (3 * b));
    }
    if (!(p < 1e9) || !(f < 1e9)) return false;
    s[k] = Scales{exponent(u), exponent(u * u), exponent(p)};
    u = std::max(f, 1e-9);
  }
  return true;
}

template <typename T, bool MUON>
hipError_t run(const nf_orth_desc &d, Plan &p, const Tensors &t, hipStream_t st) {
  Scales s[NF_ORTH_STEPS];
  int last;
  if (!orth_scales(d, s, &last)) return hipErrorInvalidValue;
  Args &a = p.a;
  auto two = [](int e) { return (float)std::ldexp(1.0, e); };
  double elements = 0;
  for (int k = 0; k < a.count; ++k) elements += (double)a.it[k].rows * a.it[k].cols;
  a.up_x = two(s[0].x);
  unsigned grid = lay(a, [](const Item &it) { return (long long)it.square_parts; });
  hipError_t e = recorded(st, "orth_squares", 0.0, sizeof(T) * (MUON ? 3.0 : 1.0) * elements,
                          [&] { hipLaunchKernelGGL((orth_squares_kernel<T, MUON>), dim3(grid), dim3(NT), 0, st, a, t); });
  if (e != hipSuccess) return e;
  grid = lay(a, [](const Item &it) { return (long long)(it.np / 64) * (it.mp / 64); });
  e = recorded(st, "orth_start", 0.0, (sizeof(T) * (MUON ? 2.0 : 1.0) + 4.0) * elements,
               [&] { hipLaunchKernelGGL((orth_start_kernel<T, MUON>), dim3(grid), dim3(NT), 0, st, a, t); });
  for (int k = 0; k < d.steps && e == hipSuccess; ++k) {
    const bool end = k + 1 == d.steps;
    a.cur = k & 1, a.a = d.a[k], a.b = d.b[k], a.c = d.c[k];
    a.up_x = two(s[k].x), a.down_x = two(-s[k].x), a.up_a = two(s[k].a), a.down_a = two(-s[k].a), a.up_p = two(s[k].p), a.down_p = two(-s[k].p);
    a.up_next = two(end ? last : s[k + 1].x);
    e = product<GRAM, float, false>(p, t, "orth_gram_128x128", "orth_gram_64x64", st);
    if (e == hipSuccess && p.parts) {
      const int B = p.block;
      grid = lay(a, [&](const Item &it) { return it.splits > 1 ? triangle_tiles(it, B) * (B * B / 4 / LT) : 0ll; });
      e = recorded(st, "orth_parts", 0.0, 0.0, [&] {
        if (B == 128)
          hipLaunchKernelGGL(orth_parts_kernel<128>, dim3(grid), dim3(LT), 0, st, a);
        else
          hipLaunchKernelGGL(orth_parts_kernel<64>, dim3(grid), dim3(LT), 0, st, a);
      });
    }
    if (e == hipSuccess) e = product<POLY, float, false>(p, t, "orth_poly_128x128", "orth_poly_64x64", st);
    if (e != hipSuccess) break;
    e = end ? product<LAST, T, MUON>(p, t, "orth_last_128x128", "orth_last_64x64", st) : product<APPLY, float, false>(p, t, "orth_apply_128x128", "orth_apply_64x64", st);
  }
  return e;
}

}  // namespace

bool orth_bounded(const nf_orth_desc &d) {
  Scales s[NF_ORTH_STEPS];
  int last;
  return orth_scales(d, s, &last);
}

size_t orth_workspace_bytes(const nf_orth_desc &d, int count, const int32_t *rows, const int32_t *cols) { return plan_of(d, count, rows, cols).bytes; }

hipError_t launch_orth(const nf_orth_desc &d, int dtype, int count, const void *const *g, void *const *y, const int32_t *rows, const int32_t *cols, void *ws,
                       hipStream_t st) {
  Plan p = plan_of(d, count, rows, cols);
  p.a.ws = (char *)ws;
  Tensors t = {};
  for (int k = 0; k < count; ++k) t.g[k] = g[k], t.y[k] = y[k];
  if (dtype == NF_BF16) return run<__bf16, false>(d, p, t, st);
  if (dtype == NF_F16) return run<_Float16, false>(d, p, t, st);
  return run<float, false>(d, p, t, st);
}

hipError_t launch_muon(const nf_muon_desc &d, int count, float *const *w, const float *const *g, float *const *v, const int32_t *rows, const int32_t *cols, void *ws,
                       hipStream_t st) {
  Plan p = plan_of(d.orth, count, rows, cols);
  p.a.ws = (char *)ws;
  Tensors t = {};
  for (int k = 0; k < count; ++k) t.g[k] = g[k], t.y[k] = w[k], t.v[k] = v && d.momentum != 0 ? v[k] : nullptr;
  t.momentum = d.momentum, t.lr = d.lr, t.keep = (float)(1.0 - (double)d.lr * d.weight_decay), t.nesterov = d.nesterov;
  return run<float, true>(d.orth, p, t, st);
}

}  // namespace nf
