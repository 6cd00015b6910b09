// Matrices made orthogonal by Newton-Schulz steps, and weights updated with them.
//   X0 = G / (|G| + eps);  X' = a X + (b A + c A^2) X,  A = X X^T over the shorter side
// The steps amplify errors (by a^steps where singular values are small: 485 for 5 steps of a = 3.4445), so products keep fp32's digits: every
// matrix is held as two fp16 pieces, h + l = v 2^s to 22 bits, and a product is h h + h l + l h on the fp16 matrix instructions, summed in fp32.  That is
// three products at 1.4 PFLOP/s where the fp32 instructions reach 150 TFLOP/s.  s is chosen from a bound of the singular values after each step
// (orth_scales), so that the largest element fits fp16 and what falls below its smallest is 2^-39 of that.
//   layout   [row][32 columns' h, their l]: a row's step of 32 columns is 128 bytes; sides are padded with zeros to 32
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

using f16x8 = __attribute__((ext_vector_type(8))) _Float16;
using shortx4 = __attribute__((ext_vector_type(4))) short;

constexpr int MOST = NF_ORTH_MATRICES;

struct Item {
  unsigned x[2], A, P, part, squares;  // where they begin in the workspace, in units of 256 bytes
  int rows, cols, n, m, np, mp;        // n <= m, padded; rows > cols: held transposed
  int splits, per;                     // of A's sums: parts, and their steps of 32 terms
  int square_parts, chunk;             // of |G|^2
};
struct Tensors {
  const void *g[MOST];
  float *v[MOST];
  void *y[MOST];
  float momentum, keep, lr;  // y = keep y - lr sqrt(max(1, rows / cols)) X
  int nesterov;
};
// What all launches of a call read.  The first one gets it as an argument and leaves it at the workspace's start: an argument is read from the host's
// memory, and a workgroup goes there once for the place of its matrix and again for the matrix (17 launches for 64x576: 104 us, 84 from the workspace).
enum { SQUARES, START, A_TILES, A_PARTS, P_TILES, X_TILES, LAUNCHES };
struct Table {
  int first[LAUNCHES][MOST + 1];  // first workgroup of each matrix; of X' = a X + P X, an XCD's first
  Item it[MOST];
  Tensors t;
};
constexpr unsigned TABLE = (sizeof(Table) + 255) / 256;  // units of the workspace
struct Args {
  char *ws;
  int count, cur;
  float a, b, c, eps;
  float up_x, down_x, up_a, down_a, up_p, down_p, up_next;  // 2^s and 2^-s of X, A, P and X'
  __host__ __device__ char *at(unsigned unit) const { return ws + 256ull * unit; }
};

// the matrix that a workgroup works on: the last whose first workgroup is not behind it
__device__ inline int item_of(const int *first, int count, int id) {
  const int lane = threadIdx.x & 63;
  const bool at = lane < count && first[lane < MOST ? lane : MOST] <= id;
  return __builtin_amdgcn_readfirstlane(__popcll(__ballot(at)) - 1);
}

// element (r, c) of a matrix in pieces: its h, and its l 64 bytes further
__device__ inline char *piece(char *p, long long ld, long long r, int c) { return p + r * ld + (c >> 5) * 128 + (c & 31) * 2; }
template <typename V>
__device__ inline void split(float v, V &h, V &l) {
  h = (_Float16)v;
  l = (_Float16)(v - (float)h);
}
// 8 neighbours of a row
__device__ inline void get8(const char *p, float (&v)[8]) {
  const f16x8 h = *reinterpret_cast<const f16x8 *>(p), l = *reinterpret_cast<const f16x8 *>(p + 64);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = (float)h[e] + (float)l[e];
}
__device__ inline void put8(char *p, const float (&v)[8]) {
  f16x8 h, l;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    _Float16 x, y;
    split(v[e], x, y);
    h[e] = x, l[e] = y;
  }
  *reinterpret_cast<f16x8 *>(p) = h, *reinterpret_cast<f16x8 *>(p + 64) = l;
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
__global__ __launch_bounds__(NT) void orth_squares_kernel(Args a, Table table) {
  __shared__ double lds[4];
  if (blockIdx.x == 0)
    for (int i = threadIdx.x; i < (int)(sizeof(Table) / 4); i += NT) reinterpret_cast<int *>(a.ws)[i] = reinterpret_cast<const int *>(&table)[i];
  const int k = item_of(table.first[SQUARES], a.count, blockIdx.x);
  const Item &it = table.it[k];
  const Tensors &t = table.t;
  const int part = blockIdx.x - table.first[SQUARES][k];
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
  if (threadIdx.x == 0) reinterpret_cast<double *>(a.at(it.squares))[part] = s;
}

// X0 in pieces, a tile of 64 x 64 to a workgroup
template <typename T, bool MUON>
__global__ __launch_bounds__(NT) void orth_start_kernel(Args a, const Table *__restrict__ table) {
  __shared__ double lds[4];
  __shared__ float tile[64][65];
  const int k = item_of(table->first[START], a.count, blockIdx.x);
  const Item it = table->it[k];
  const Tensors &t = table->t;
  const int id = blockIdx.x - table->first[START][k], across = (it.mp + 63) / 64, tr = id / across, r0 = tr * 64, c0 = (id - tr * across) * 64;
  const T *const g = (const T *)t.g[k];
  const float *const v = MUON ? t.v[k] : nullptr;
  const bool tall = it.rows > it.cols;
  const int x = (threadIdx.x & 7) * 8, y = threadIdx.x >> 3;  // along G's rows
  float u[2][8];  // on their way before the sum's barrier
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int row = (tall ? c0 : r0) + y + 32 * i, col = (tall ? r0 : c0) + x, n = row < it.rows ? it.cols - col : 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) u[i][e] = 0.f;
    if (n <= 0) continue;
    const long long at = (long long)row * it.cols + col;
    load8(g + at, u[i], n);
    if constexpr (MUON) {
      if (!v) continue;
      float m[8];
      load8(v + at, m, n);  // the new momentum
#pragma unroll
      for (int e = 0; e < 8; ++e) u[i][e] = t.nesterov ? fmaf(t.momentum, m[e], u[i][e]) : m[e];
    }
  }
  double s = 0;
  const double *const squares = reinterpret_cast<const double *>(a.at(it.squares));
  for (int i = threadIdx.x; i < it.square_parts; i += NT) s += squares[i];
  const double inv = 1.0 / (sqrt(all_sum(s, lds)) + a.eps);  // in 64 bits: |G| may leave fp32 where no element does
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) (tall ? tile[x + e][y + 32 * i] : tile[y + 32 * i][x + e]) = (float)(u[i][e] * inv) * a.up_x;
  __syncthreads();
  char *const X = a.at(it.x[0]);
  for (int i = threadIdx.x; i < 512; i += NT) {
    const int r = i >> 3, c = (i & 7) * 8;
    if (r0 + r >= it.np || c0 + c >= it.mp) continue;
    float w[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = tile[r][c + e];
    put8(piece(X, 4ll * it.mp, r0 + r, c0 + c), w);
  }
}

// ---- products ----
enum { GRAM, POLY, APPLY, LAST };

template <int BLOCK>
struct Tile {
  static constexpr int DOWN = BLOCK == 96 ? 3 : 2, ACROSS = BLOCK == 128 ? 4 : 2;  // waves of 64 x 32, 32 x 48 (12 of 16 x 48 1.5 us slower at 2048x2048) and 32 x 32
  static constexpr int STAGES = 4;
  static constexpr int WAVES = DOWN * ACROSS, THREADS = 64 * WAVES, MT = BLOCK / 16 / DOWN, NT = BLOCK / 16 / ACROSS;
  static constexpr int BYTES = BLOCK * 128, STAGE = 2 * BYTES, PIECES = BYTES / 1024 / WAVES;
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

// Finished sums, 8 neighbours of a row.  A and P are written here; what is written across as well, or as the caller's matrix, stays in v.
template <int KIND>
__device__ inline void finish8(const Args &a, const Item &it, int r, int c, float (&v)[8]) {
  if constexpr (KIND == GRAM) {
    const float s = a.down_x * a.down_x * a.up_a;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= s;
    put8(piece(a.at(it.A), 4ll * it.np, r, c), v);
  } else if constexpr (KIND == POLY) {
    float A[8];
    get8(piece(a.at(it.A), 4ll * it.np, r, c), A);
    const float sa = a.b * a.down_a * a.up_p, ss = a.c * a.down_a * a.down_a * a.up_p;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = fmaf(A[e], sa, v[e] * ss);
    put8(piece(a.at(it.P), 4ll * it.np, r, c), v);
  } else {
    float X[8];
    get8(piece(a.at(a.cur ? it.x[1] : it.x[0]), 4ll * it.mp, r, c), X);
    const float up = KIND == LAST ? 1.f : a.up_next, sx = a.a * a.down_x * up, ss = a.down_p * a.down_x * up;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = fmaf(X[e], sx, v[e] * ss);
    if constexpr (KIND == APPLY) put8(piece(a.at(a.cur ? it.x[0] : it.x[1]), 4ll * it.mp, r, c), v);
  }
}
// 8 neighbours of a row of the caller's matrix, n of which lie inside
template <typename OUT, bool MUON>
__device__ inline void give8(const Tensors &t, const Item &it, int k, int row, int col, int n, float (&v)[8]) {
  OUT *const y = (OUT *)t.y[k] + (long long)row * it.cols + col;
  if constexpr (MUON) {
    const float rate = t.lr * (it.rows > it.cols ? sqrtf((float)it.rows / (float)it.cols) : 1.f);
    float w[8];
    load8(y, w, n);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = fmaf(-rate, v[e], t.keep * w[e]);
  }
  store8(y, v, n);
}

// A tile of sums in LDS (rows of LDW words) to memory.  Symmetric results of a tile off the diagonal are written across, too.
template <int BLOCK, int THREADS, int KIND, typename OUT, bool MUON>
__device__ inline void tile_out(const Args &a, const Tensors &t, const Item &it, int k, int tr, int tc, float *W) {
  constexpr int LDW = BLOCK + 4, ITEMS = BLOCK * BLOCK / 8;
  const int rows = it.np - tr * BLOCK, cols = (KIND <= POLY ? it.np : it.mp) - tc * BLOCK;  // inside, whole 32s
  const bool tall = it.rows > it.cols, across = KIND <= POLY ? tr != tc : KIND == LAST && tall;
  __syncthreads();
  for (int i = threadIdx.x; i < ITEMS; i += THREADS) {
    const int r = i / (BLOCK / 8), c = i % (BLOCK / 8) * 8;
    if (r >= rows || c >= cols) continue;
    float v[8];
    floatx4 *const at = reinterpret_cast<floatx4 *>(W + r * LDW + c);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = at[0][e], v[e + 4] = at[1][e];
    finish8<KIND>(a, it, tr * BLOCK + r, tc * BLOCK + c, v);
    if (across) {
      at[0] = floatx4{v[0], v[1], v[2], v[3]}, at[1] = floatx4{v[4], v[5], v[6], v[7]};
    } else if constexpr (KIND == LAST) {
      const int row = tr * BLOCK + r, col = tc * BLOCK + c;
      if (row < it.n && col < it.m) give8<OUT, MUON>(t, it, k, row, col, it.m - col, v);
    }
  }
  if (!across) return;
  __syncthreads();
  for (int i = threadIdx.x; i < ITEMS; i += THREADS) {  // 8 neighbours of a column
    const int c = i / (BLOCK / 8), r = i % (BLOCK / 8) * 8;
    if (r >= rows || c >= cols) continue;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = W[(r + e) * LDW + c];
    const int row = tc * BLOCK + c, col = tr * BLOCK + r;
    if constexpr (KIND <= POLY)
      put8(piece(a.at(KIND == GRAM ? it.A : it.P), 4ll * it.np, row, col), v);
    else if (row < it.m && col < it.n)
      give8<OUT, MUON>(t, it, k, row, col, it.n - col, v);
  }
}

// The tile t of those on and above the diagonal, column by column.
__device__ inline void triangle(int t, int &tr, int &tc) {
  tc = (int)((sqrtf(8.f * t + 1.f) - 1.f) * 0.5f);
  while ((tc + 1) * (tc + 2) / 2 <= t) ++tc;
  while (tc * (tc + 1) / 2 > t) --tc;
  tr = t - tc * (tc + 1) / 2;
}

// BLOCK x BLOCK results; a step is 32 terms.  While a step's products run, the next one's fragments are read and the
// copies of the STAGES-th next are on their way: one barrier a step, behind which the next stage is whole and this one free.  Steps go in pairs
// (two sets of fragments); those beyond the last are copies of nothing, so that the waits count the same.
// 2048x2048: X' in 256 tiles of 128 48 us, 1070 TFLOP/s of fp16 products (the matrix instructions by themselves 38, copies and reads by themselves 32: they
// overlap but for a third); A and A^2 in 253 tiles of 96 35 each.  17 matrices of 64x27 to 512x4608: X' 45, which reads and writes 132 MB besides.
template <int BLOCK, int KIND, typename OUT, bool MUON>
__global__ __launch_bounds__(Tile<BLOCK>::THREADS) void orth_product_kernel(Args a, const Table *__restrict__ table) {
  using S = Tile<BLOCK>;
  constexpr bool APART = KIND >= APPLY;
  constexpr int MT = S::MT, NT = S::NT, STAGES = S::STAGES, WAVES = S::WAVES, PIECES = S::PIECES;
  constexpr int OUT_BYTES = BLOCK * (BLOCK + 4) * 4, RING = STAGES * S::STAGE;
  __shared__ __align__(1024) char lds[RING > OUT_BYTES ? RING : OUT_BYTES];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i16 = lane & 15, q = lane >> 4;
  // A's and P's tiles: an XCD has few matrices, whose operands its L2 holds (17 matrices of 64x27 to 512x4608: A 26 us, 32 by eighths); X's: an eighth of each, so
  // that all XCDs have as much to do (46, 49)
  constexpr int LAUNCH = KIND == GRAM ? A_TILES : KIND == POLY ? P_TILES : X_TILES;
  const int block = APART ? blockIdx.x >> 3 : xcd_run(blockIdx.x, gridDim.x), k = item_of(table->first[LAUNCH], a.count, block), first = table->first[LAUNCH][k];
  const Item it = table->it[k];
  const Tensors &t = table->t;
  const int place = block - first + (APART ? (blockIdx.x & 7) * (table->first[LAUNCH][k + 1] - first) : 0);
  int id = place, split = 0, tr, tc;
  if constexpr (KIND <= POLY) {
    const int T = (it.np + BLOCK - 1) / BLOCK, tiles = T * (T + 1) / 2;
    if (KIND == GRAM) split = id / tiles, id -= split * tiles;
    triangle(id, tr, tc);
  } else {
    // four rows of tiles at a time, column by column: workgroups of an XCD share few rows and columns
    const int down = (it.np + BLOCK - 1) / BLOCK, across = (it.mp + BLOCK - 1) / BLOCK;
    if (id >= down * across) return;
    const int band = id / (4 * across), deep = min(4, down - 4 * band);
    id -= band * 4 * across, tc = id / deep, tr = 4 * band + id - tc * deep;
  }
  const long long ld_a = 4ll * (KIND == GRAM ? it.mp : it.np), ld_b = 4ll * (KIND == POLY ? it.np : it.mp);
  const char *const A = a.at(KIND == GRAM ? (a.cur ? it.x[1] : it.x[0]) : KIND == POLY ? it.A : it.P) + (long long)tr * BLOCK * ld_a;
  const char *const B = a.at(KIND == POLY ? it.A : (a.cur ? it.x[1] : it.x[0])) + (APART ? (long long)tc * BLOCK * 4 : (long long)tc * BLOCK * ld_b);
  const int all = (KIND == GRAM ? it.mp : it.np) / 32, s0 = KIND == GRAM ? split * it.per : 0, steps = KIND == GRAM ? min(it.per, all - s0) : all;
  const int rows = it.np - tr * BLOCK, cols = (KIND <= POLY ? it.np : it.mp) - tc * BLOCK;  // inside
  uint32_t av[PIECES], bv[PIECES];
#pragma unroll
  for (int p = 0; p < PIECES; ++p) {
    const int at = (p * WAVES + wave) * 64 + lane, row = at >> 3;
    av[p] = row < rows ? (uint32_t)(row * ld_a) + (((at & 7) ^ chunk_swizzle(row)) << 4) : OUTSIDE;
    if (APART) {
      const int term = at / S::CPR, c = (at % S::CPR) ^ (unit_swizzle(term) << 1);
      bv[p] = c * 4 < cols ? (uint32_t)(term * ld_b) + (c << 4) : OUTSIDE;
    } else {
      bv[p] = row < cols ? (uint32_t)(row * ld_b) + (((at & 7) ^ chunk_swizzle(row)) << 4) : OUTSIDE;
    }
  }
  const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds + wave * 1024;
  auto fetch = [&](int s, int stage, int from, int until) {
    const uintx4 ba = buffer_of(A + (s0 + s) * 128ll), bb = buffer_of(B + (APART ? (long long)s * 32 * ld_b : (s0 + s) * 128ll));
    const uint32_t to = base + stage * S::STAGE, none = s < steps ? 0u : OUTSIDE;  // an offset with OUTSIDE's bits lies outside, whatever the others
#pragma unroll
    for (int p = 0; p < 2 * PIECES; ++p)
      if (p >= from && p < until)
        p < PIECES ? copy16(ba, av[p % PIECES] | none, to + p * (1024 * WAVES)) : copy16(bb, bv[p % PIECES] | none, to + S::BYTES + (p - PIECES) * (1024 * WAVES));
  };
  const int wm = wave / S::ACROSS * (16 * MT), wn = wave % S::ACROSS * (16 * NT);
  floatx4 acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
  struct Set {
    f16x8 a[MT][2], b[NT][2];
  };
  auto read = [&](Set &f, int stage) {
    const char *const la = lds + stage * S::STAGE, *const lb = la + S::BYTES;
#pragma unroll
    for (int pl = 0; pl < 2; ++pl)
#pragma unroll
      for (int i = 0; i < MT; ++i) f.a[i][pl] = fragment<BLOCK, false>(la, wm + 16 * i, pl, lane);
#pragma unroll
    for (int pl = 0; pl < 2; ++pl)
#pragma unroll
      for (int j = 0; j < NT; ++j) f.b[j][pl] = fragment<BLOCK, APART>(lb, wn + 16 * j, pl, lane);
  };
  int stage = 0;
  auto step = [&](int s, Set &now, Set &next) {
    wait_copies<(STAGES - 2) * 2 * PIECES>();
    wait_lds();
    barrier();
    const int free = stage;
    stage = stage + 1 == STAGES ? 0 : stage + 1;
    read(next, stage);
    constexpr int EACH = (2 * PIECES + MT - 1) / MT;  // copies between a row of fragments and the next
#pragma unroll
    for (int i = 0; i < MT; ++i) {
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(now.b[j][0], now.a[i][1], acc[i][j], 0, 0, 0);
        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(now.b[j][1], now.a[i][0], acc[i][j], 0, 0, 0);
        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(now.b[j][0], now.a[i][0], acc[i][j], 0, 0, 0);
      }
      fetch(s + STAGES, free, i * EACH, (i + 1) * EACH);
    }
  };
#pragma unroll
  for (int s = 0; s < STAGES; ++s) fetch(s, s, 0, 2 * PIECES);
  wait_copies<(STAGES - 1) * 2 * PIECES>();
  barrier();
  Set even, odd;
  read(even, 0);
  for (int s = 0; s < steps; s += 2) {
    step(s, even, odd);
    step(s + 1, odd, even);
  }
  wait_copies<0>();
  wait_lds();
  // a lane has 4 neighbouring columns of a row
  if (KIND == GRAM && it.splits > 1) {
    float *const part = reinterpret_cast<float *>(a.at(it.part)) + (long long)place * BLOCK * BLOCK;
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j) *reinterpret_cast<floatx4 *>(part + (wm + 16 * i + i16) * BLOCK + wn + 16 * j + 4 * q) = acc[i][j];
    return;
  }
  barrier();
  float *const W = reinterpret_cast<float *>(lds);
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) *reinterpret_cast<floatx4 *>(W + (wm + 16 * i + i16) * (BLOCK + 4) + wn + 16 * j + 4 * q) = acc[i][j];
  tile_out<BLOCK, S::THREADS, KIND, OUT, MUON>(a, t, it, k, tr, tc, W);
}

// the parts of A's sums, in order, a tile to a workgroup
__global__ __launch_bounds__(LT) void orth_parts_kernel(Args a, const Table *__restrict__ table) {
  constexpr int BLOCK = 64;
  __shared__ __align__(16) float W[BLOCK * (BLOCK + 4)];
  const int k = item_of(table->first[A_PARTS], a.count, blockIdx.x);
  const Item it = table->it[k];
  const int tile = blockIdx.x - table->first[A_PARTS][k], T = (it.np + BLOCK - 1) / BLOCK, tiles = T * (T + 1) / 2;
  int tr, tc;
  triangle(tile, tr, tc);
  const float *const part = reinterpret_cast<const float *>(a.at(it.part)) + (long long)tile * BLOCK * BLOCK;
  constexpr int EACH = BLOCK * BLOCK / 4 / LT;
  floatx4 s[EACH] = {};
#pragma unroll 4
  for (int z = 0; z < it.splits; ++z)
#pragma unroll
    for (int e = 0; e < EACH; ++e) s[e] += reinterpret_cast<const floatx4 *>(part + (long long)z * tiles * BLOCK * BLOCK)[threadIdx.x + e * LT];
#pragma unroll
  for (int e = 0; e < EACH; ++e) {
    const int i = threadIdx.x + e * LT;
    *reinterpret_cast<floatx4 *>(W + i / (BLOCK / 4) * (BLOCK + 4) + i % (BLOCK / 4) * 4) = s[e];
  }
  tile_out<BLOCK, LT, GRAM, float, false>(a, table->t, it, k, tr, tc, W);
}

// ---- small matrices ----
// A matrix to a workgroup, all steps in LDS: nothing but barriers between the products of 16 x 16 results, which are shared out among the waves.  16x27 12 us,
// in the launches above 70 (17 of 4 us each); 64x200 42, of which each step's barriers and short chains of products take most.  Rows are 16 bytes longer than their elements: the 16 that a fragment takes lie in different banks.
struct Small {
  float a[NF_ORTH_STEPS], b[NF_ORTH_STEPS], c[NF_ORTH_STEPS];
  float up_x[NF_ORTH_STEPS + 1], up_a[NF_ORTH_STEPS], up_p[NF_ORTH_STEPS];  // 2^s, as Args has them
  int steps;
};
constexpr int FEW_LDS = 32 << 10, MANY_LDS = (160 << 10) - 256;
__host__ __device__ inline int small_row(int columns) { return columns * 4 + 16; }
inline int small_bytes(const Item &it) { return it.np * (small_row(it.mp) + 2 * small_row(it.np)); }

template <typename T, bool MUON, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void orth_small_kernel(float eps, Table table, Small m) {
  constexpr int THREADS = 64 * WAVES;
  __shared__ __align__(16) char lds[WAVES == 4 ? FEW_LDS : MANY_LDS];
  __shared__ double sums[WAVES];
  const int k = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i16 = lane & 15, q = lane >> 4;
  const Item &it = table.it[k];
  const Tensors &t = table.t;
  const int ldx = small_row(it.mp), lda = small_row(it.np), down = it.np / 16;
  char *const X = lds, *const A = X + it.np * ldx, *const P = A + it.np * lda;
  const T *const g = (const T *)t.g[k];
  float *const v = MUON ? t.v[k] : nullptr;
  const bool tall = it.rows > it.cols;
  const int all = it.rows * it.cols;
  double s = 0;
  for (int i = tid; i < all; i += THREADS) {
    float x = (float)g[i];
    if (MUON && v) {
      const float n = fmaf(t.momentum, v[i], x);
      v[i] = n;
      x = t.nesterov ? fmaf(t.momentum, n, x) : n;
    }
    s += (double)x * x;
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) s += __shfl_xor(s, o);
  if (lane == 0) sums[wave] = s;
  for (int i = tid; i < it.np * ldx / 16; i += THREADS) reinterpret_cast<uintx4 *>(X)[i] = uintx4{0, 0, 0, 0};
  __syncthreads();
  s = 0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) s += sums[w];
  const double inv = 1.0 / (sqrt(s) + eps);
  for (int i = tid; i < all; i += THREADS) {  // the elements that this thread has read and written above
    const int row = i / it.cols, col = i - row * it.cols, r = tall ? col : row, c = tall ? row : col;
    _Float16 h, l;
    split((float)(direction<T, MUON>(t, g, v, i) * inv) * m.up_x[0], h, l);
    char *const p = piece(X, ldx, r, c);
    *reinterpret_cast<_Float16 *>(p) = h, *reinterpret_cast<_Float16 *>(p + 64) = l;
  }
  __syncthreads();
  auto rows16 = [&](const char *p, int ld, int rb, int kk, int pl) { return *reinterpret_cast<const f16x8 *>(p + (rb + i16) * ld + kk * 128 + pl * 64 + q * 16); };
  auto terms16 = [&](const char *p, int ld, int cb, int kk, int pl) {  // columns cb .. of an operand whose rows are terms
    uintx4 f;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const char *at = p + (kk * 32 + q * 8 + h * 4 + (i16 >> 2)) * ld + (cb >> 5) * 128 + pl * 64 + (cb & 31) * 2 + (i16 & 3) * 8;
      const uint2 w = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) shortx4 *)at));
      f[2 * h] = w.x, f[2 * h + 1] = w.y;
    }
    return __builtin_bit_cast(f16x8, f);
  };
  // The pieces' four products: next to no time here, and what l l leaves out shows where sums are short (8x8: 1.35 times the error of fp32 steps, 1.15
  // with it).
  auto four = [&](const f16x8 &ah, const f16x8 &al, const f16x8 &bh, const f16x8 &bl, floatx4 acc) {
    acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(bl, al, acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(bh, al, acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(bl, ah, acc, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(bh, ah, acc, 0, 0, 0);
  };
  auto get4 = [&](const char *p, float (&x)[4]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = (float)reinterpret_cast<const _Float16 *>(p)[e] + (float)reinterpret_cast<const _Float16 *>(p + 64)[e];
  };
  auto put4 = [&](char *p, const float (&x)[4]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      _Float16 h, l;
      split(x[e], h, l);
      reinterpret_cast<_Float16 *>(p)[e] = h, reinterpret_cast<_Float16 *>(p + 64)[e] = l;
    }
  };
  for (int step = 0; step < m.steps; ++step) {
    const bool last = step + 1 == m.steps;
    const float up_x = m.up_x[step], up_a = m.up_a[step], up_p = m.up_p[step], up_next = last ? 1.f : m.up_x[step + 1];
    for (int z = wave; z < down * down; z += WAVES) {  // A = X X^T
      const int rb = z / down * 16, cb = z % down * 16;
      // four sums: they wait less for each other, and lose less: the matrix instructions cut what does not fit (8x1000: 43 us and 2.3 times the error of fp32
      // steps in one)
      floatx4 part[4] = {};
      for (int kk = 0; kk < it.mp / 32; kk += 4) {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const int k32 = kk + c;
          if (k32 < it.mp / 32)
            part[c] = four(rows16(X, ldx, rb, k32, 0), rows16(X, ldx, rb, k32, 1), rows16(X, ldx, cb, k32, 0), rows16(X, ldx, cb, k32, 1), part[c]);
        }
      }
      const floatx4 acc = (part[0] + part[1]) + (part[2] + part[3]);
      const float scale = up_a / (up_x * up_x), w[4] = {acc[0] * scale, acc[1] * scale, acc[2] * scale, acc[3] * scale};
      put4(piece(A, lda, rb + i16, cb + 4 * q), w);
    }
    __syncthreads();
    for (int z = wave; z < down * down; z += WAVES) {  // P = b A + c A^2
      const int rb = z / down * 16, cb = z % down * 16;
      floatx4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 2
      for (int kk = 0; kk < it.np / 32; ++kk)
        acc = four(rows16(A, lda, rb, kk, 0), rows16(A, lda, rb, kk, 1), rows16(A, lda, cb, kk, 0), rows16(A, lda, cb, kk, 1), acc);
      float w[4];
      get4(piece(A, lda, rb + i16, cb + 4 * q), w);
      const float sa = m.b[step] / up_a * up_p, ss = m.c[step] / up_a / up_a * up_p;  // b and c first: up_p / up_a^2 may leave fp32's range
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = fmaf(w[e], sa, acc[e] * ss);
      put4(piece(P, lda, rb + i16, cb + 4 * q), w);
    }
    __syncthreads();
    const float sx = m.a[step] * (up_next / up_x), ss = up_next / up_p / up_x;
    for (int cb = wave * 16; cb < it.mp; cb += WAVES * 16) {  // X' = a X + P X, in place: 16 columns need no others
      f16x8 bh[2], bl[2];
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
        if (kk * 32 < it.np) bh[kk] = terms16(X, ldx, cb, kk, 0), bl[kk] = terms16(X, ldx, cb, kk, 1);
      float w[4][4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (i * 16 >= it.np) break;
        floatx4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kk = 0; kk < 2; ++kk)
          if (kk * 32 < it.np) acc = four(rows16(P, lda, i * 16, kk, 0), rows16(P, lda, i * 16, kk, 1), bh[kk], bl[kk], acc);
        get4(piece(X, ldx, i * 16 + i16, cb + 4 * q), w[i]);
#pragma unroll
        for (int e = 0; e < 4; ++e) w[i][e] = fmaf(w[i][e], sx, acc[e] * ss);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (i * 16 >= it.np) break;
        const int r = i * 16 + i16, c = cb + 4 * q;
        if (!last) {
          put4(piece(X, ldx, r, c), w[i]);
        } else if (r < it.n) {
          T *const y = (T *)t.y[k];
          const float rate = t.lr * (tall ? sqrtf((float)it.rows / (float)it.cols) : 1.f);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if (c + e >= it.m) continue;
            const int at = tall ? (c + e) * it.cols + r : r * it.cols + c + e;
            y[at] = MUON ? (T)fmaf(-rate, w[i][e], t.keep * (float)y[at]) : (T)w[i][e];
          }
        }
      }
    }
    __syncthreads();
  }
}

// ---- plans ----
struct Plan {
  Args a;
  Table table;
  unsigned grid[LAUNCHES];
  int sym, app;  // tiles of the symmetric products, and of the others
  int small;     // waves to a matrix where all fit a workgroup each, or 0
  bool parts;
  size_t bytes;
};

inline long long tiles_of(int side, int block) { return (side + block - 1) / block; }
inline long long triangle_tiles(const Item &it, int block) {
  const long long T = tiles_of(it.np, block);
  return T * (T + 1) / 2;
}

// Tiles of the symmetric products, by rounds over the workgroups that run together (two of 64 to a CU, one of 96 or 128) and a step's time, and whether A's
// sums are cut into parts, towards 512 workgroups of tiles of 64, 16 steps each at least, and added in a launch of their own.  2048x2048: 253 tiles of
// 96 35 us, 528 of 64 44, 136 of 128 46.  17 matrices of 64x27 to 512x4608, whose tiles differ in length: 64 and parts 34, 96 42, 128 60.  1000x1000,
// 136 tiles of 64, one to a CU: 14, and with parts 19.
struct Symmetric {
  int side;
  bool parts;
};
Symmetric symmetric_tile(const Item *it, int count) {
  constexpr int sides[3] = {64, 96, 128}, slots[3] = {512, 256, 256};
  constexpr double time[3] = {0.60, 0.56, 0.72}, alone = 0.33;  // us a step; of a tile of 64 on a CU of its own
  double best = 1e300;
  Symmetric s = {64, false};
  auto see = [&](double t, int side, bool parts) {
    if (t < best) best = t, s = Symmetric{side, parts};
  };
  for (int i = 0; i < 3; ++i) {
    double tiles = 0, work = 0, longest = 0;
    for (int k = 0; k < count; ++k) {
      const double t = (double)triangle_tiles(it[k], sides[i]), steps = it[k].mp / 32;
      tiles += t, work += t * steps, longest = std::max(longest, steps);
    }
    const double rounds = count == 1 ? std::ceil(tiles / slots[i]) : std::max(1.0, tiles / slots[i]);
    see(i == 0 && tiles <= 256 ? alone * longest : tiles <= slots[i] ? time[i] * longest : time[i] * rounds * work / tiles, sides[i], false);
    if (i == 0) see(time[0] * std::max(16.0, work / 512) + 8, 64, true);
  }
  return s;
}

Plan plan_of(const nf_orth_desc &d, int count, const int32_t *rows, const int32_t *cols) {
  Plan p = {};
  Args &a = p.a;
  a.count = count, a.eps = d.eps;
  for (int k = 0; k < count; ++k) {
    Item &it = p.table.it[k];
    it.rows = rows[k], it.cols = cols[k], it.n = std::min(rows[k], cols[k]), it.m = std::max(rows[k], cols[k]);
    it.np = (it.n + 31) / 32 * 32, it.mp = (it.m + 31) / 32 * 32;
    const long long all = (long long)it.rows * it.cols;
    it.chunk = 8192;
    while ((all + it.chunk - 1) / it.chunk > 1024) it.chunk *= 2;
    it.square_parts = (int)((all + it.chunk - 1) / it.chunk);
  }
  long long large = 0;
  for (int k = 0; k < count; ++k) large += tiles_of(p.table.it[k].np, 128) * tiles_of(p.table.it[k].mp, 128);
  const Symmetric sym = symmetric_tile(p.table.it, count);
  p.sym = sym.side;
  p.app = large >= 192 ? 128 : 64;  // the same 17 matrices, 683 tiles of 128: 45 us, of 64 51; 2048x2048, 256 tiles: 48 and 62
  int most = 0, tiles = 0;
  for (int k = 0; k < count; ++k) most = std::max(most, p.table.it[k].np <= 64 ? small_bytes(p.table.it[k]) : MANY_LDS + 1), tiles = std::max(tiles, p.table.it[k].np / 16 * (p.table.it[k].mp / 16));
  p.small = most <= FEW_LDS && tiles <= 16 ? 4 : most <= MANY_LDS ? 16 : 0;
  const int B = p.sym;
  long long work = 0;
  for (int k = 0; k < count; ++k) work += triangle_tiles(p.table.it[k], B) * (p.table.it[k].mp / 32);
  const int each = (int)std::max<long long>(16, sym.parts ? (work + 511) / 512 : 1ll << 20);
  size_t at = 256ull * TABLE;
  auto take = [&](size_t n) {
    const size_t was = at;
    at = (at + n + 255) / 256 * 256;
    return (unsigned)(was / 256);
  };
  for (int k = 0; k < count; ++k) {
    Item &it = p.table.it[k];
    const int steps = it.mp / 32;
    it.splits = std::max(1, (steps + each / 2) / each);
    it.per = (steps + it.splits - 1) / it.splits, it.splits = (steps + it.per - 1) / it.per;
    it.x[0] = take(4ull * it.np * it.mp), it.x[1] = take(4ull * it.np * it.mp);
    it.A = take(4ull * it.np * it.np), it.P = take(4ull * it.np * it.np);
    it.squares = take(8ull * it.square_parts);
    it.part = it.splits > 1 ? take(4ull * it.splits * triangle_tiles(it, B) * B * B) : 0u;
    p.parts |= it.splits > 1;
  }
  p.bytes = at;
  return p;
}

// Fills the first workgroups of a launch, or those of each share of its matrices.
template <typename F>
void lay(Plan &p, int launch, F workgroups, int shares = 1) {
  long long at = 0;
  int *const first = p.table.first[launch];
  for (int k = 0; k < p.a.count; ++k) first[k] = (int)at, at += (workgroups(p.table.it[k]) + shares - 1) / shares;
  first[p.a.count] = (int)at;
  p.grid[launch] = (unsigned)(at * shares);
}

template <int KIND, typename OUT, bool MUON>
hipError_t product(const Plan &p, const char *const (&names)[3], hipStream_t st) {
  const int B = KIND <= POLY ? p.sym : p.app;
  const unsigned grid = p.grid[KIND == GRAM ? A_TILES : KIND == POLY ? P_TILES : X_TILES];
  double flops = 0;
  for (int k = 0; k < p.a.count; ++k) {
    const Item &it = p.table.it[k];
    flops += (KIND <= POLY ? 1.0 : 2.0) * it.n * it.n * (KIND == POLY ? it.n : it.m);
  }
  return recorded(st, names[B == 64 ? 0 : B == 96 ? 1 : 2], flops, 0.0, [&] {
    auto go = [&](auto kernel, int threads) { hipLaunchKernelGGL(kernel, dim3(grid), dim3(threads), 0, st, p.a, (const Table *)p.a.ws); };
    if (B == 64) return go(orth_product_kernel<64, KIND, OUT, MUON>, Tile<64>::THREADS);
    if constexpr (KIND <= POLY) {
      if (B == 96) return go(orth_product_kernel<96, KIND, OUT, MUON>, Tile<96>::THREADS);
    }
    go(orth_product_kernel<128, KIND, OUT, MUON>, Tile<128>::THREADS);
  });
}

// The exponents s of X, A, P and X' at every step, from a bound u of the singular values: |x| <= u, elements of A are at most u^2, of P = b A + c A^2
// the largest |b y + c y^2| over y <= u^2, and the next u is the largest |f(x)| over x <= u.  Extremes lie at the ends or where the slope is 0.
// Bounds from 1e-6 to 1e9 (or 0) keep all scales, and what the kernels form of them, in fp32's range.
struct Scales {
  int x, a, p;
};
bool orth_scales(const nf_orth_desc &d, Scales *s, int *last) {
  double u = 1;
  auto exponent = [](double bound) { return 15 - (int)std::ceil(std::log2(bound * 1.01)); };
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
    if (!(p < 1e9) || !(f < 1e9) || (f > 0 && f < 1e-6)) return false;
    // beside a X, P's digits count from 2^-10 of f / u on; where f is 0, all results are
    s[k] = Scales{exponent(u), exponent(u * u), exponent(f > 0 ? std::max(p, f / u / 1024) : 1.0)};
    u = f > 0 ? f : 1.0;
  }
  return true;
}

template <typename T, bool MUON>
hipError_t run(const nf_orth_desc &d, Plan &p, hipStream_t st) {
  Scales s[NF_ORTH_STEPS];
  int last;
  if (!orth_scales(d, s, &last)) return hipErrorInvalidValue;
  Args &a = p.a;
  auto two = [](int e) { return (float)std::ldexp(1.0, e); };
  double elements = 0;
  for (int k = 0; k < a.count; ++k) elements += (double)p.table.it[k].rows * p.table.it[k].cols;
  if (p.small) {
    Small m = {};
    m.steps = d.steps;
    double flops = 0;
    for (int k = 0; k < d.steps; ++k) {
      m.a[k] = d.a[k], m.b[k] = d.b[k], m.c[k] = d.c[k];
      m.up_x[k] = two(s[k].x), m.up_a[k] = two(s[k].a), m.up_p[k] = two(s[k].p);
    }
    for (int k = 0; k < a.count; ++k) flops += d.steps * (2.0 * p.table.it[k].n * p.table.it[k].n * (2.0 * p.table.it[k].m + p.table.it[k].n));
    return recorded(st, p.small == 4 ? "orth_small_4_waves" : "orth_small_16_waves", flops, sizeof(T) * (MUON ? 5.0 : 2.0) * elements, [&] {
      if (p.small == 4)
        hipLaunchKernelGGL((orth_small_kernel<T, MUON, 4>), dim3(a.count), dim3(256), 0, st, a.eps, p.table, m);
      else
        hipLaunchKernelGGL((orth_small_kernel<T, MUON, 16>), dim3(a.count), dim3(1024), 0, st, a.eps, p.table, m);
    });
  }
  a.up_x = two(s[0].x);
  lay(p, SQUARES, [](const Item &it) { return (long long)it.square_parts; });
  lay(p, START, [](const Item &it) { return tiles_of(it.np, 64) * tiles_of(it.mp, 64); });
  lay(p, A_TILES, [&](const Item &it) { return triangle_tiles(it, p.sym) * it.splits; });
  lay(p, A_PARTS, [&](const Item &it) { return it.splits > 1 ? triangle_tiles(it, 64) : 0ll; });
  lay(p, P_TILES, [&](const Item &it) { return triangle_tiles(it, p.sym); });
  lay(p, X_TILES, [&](const Item &it) { return tiles_of(it.np, p.app) * tiles_of(it.mp, p.app); }, 8);
  hipError_t e = recorded(st, "orth_squares", 0.0, sizeof(T) * (MUON ? 3.0 : 1.0) * elements,
                          [&] { hipLaunchKernelGGL((orth_squares_kernel<T, MUON>), dim3(p.grid[SQUARES]), dim3(NT), 0, st, a, p.table); });
  if (e != hipSuccess) return e;
  const Table *const table = (const Table *)a.ws;
  e = recorded(st, "orth_start", 0.0, (sizeof(T) * (MUON ? 2.0 : 1.0) + 4.0) * elements,
               [&] { hipLaunchKernelGGL((orth_start_kernel<T, MUON>), dim3(p.grid[START]), dim3(NT), 0, st, a, table); });
  for (int k = 0; k < d.steps && e == hipSuccess; ++k) {
    const bool end = k + 1 == d.steps;
    a.cur = k & 1, a.a = d.a[k], a.b = d.b[k], a.c = d.c[k];
    a.up_x = two(s[k].x), a.down_x = two(-s[k].x), a.up_a = two(s[k].a), a.down_a = two(-s[k].a), a.up_p = two(s[k].p), a.down_p = two(-s[k].p);
    a.up_next = two(end ? last : s[k + 1].x);
    e = product<GRAM, float, false>(p, {"orth_gram_64x64", "orth_gram_96x96", "orth_gram_128x128"}, st);
    if (e == hipSuccess && p.parts)
      e = recorded(st, "orth_parts", 0.0, 0.0, [&] { hipLaunchKernelGGL(orth_parts_kernel, dim3(p.grid[A_PARTS]), dim3(LT), 0, st, a, table); });
    if (e == hipSuccess) e = product<POLY, float, false>(p, {"orth_poly_64x64", "orth_poly_96x96", "orth_poly_128x128"}, st);
    if (e != hipSuccess) break;
    e = end ? product<LAST, T, MUON>(p, {"orth_last_64x64", "", "orth_last_128x128"}, st) : product<APPLY, float, false>(p, {"orth_apply_64x64", "", "orth_apply_128x128"}, st);
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
  Tensors &t = p.table.t;
  for (int k = 0; k < count; ++k) t.g[k] = g[k], t.y[k] = y[k];
  if (dtype == NF_BF16) return run<__bf16, false>(d, p, st);
  if (dtype == NF_F16) return run<_Float16, false>(d, p, st);
  return run<float, false>(d, p, st);
}

hipError_t launch_muon(const nf_muon_desc &d, int count, float *const *w, const float *const *g, float *const *v, const int32_t *rows, const int32_t *cols, void *ws,
                       hipStream_t st) {
  Plan p = plan_of(d.orth, count, rows, cols);
  p.a.ws = (char *)ws;
  Tensors &t = p.table.t;
  for (int k = 0; k < count; ++k) t.g[k] = g[k], t.y[k] = w[k], t.v[k] = v && d.momentum != 0 ? v[k] : nullptr;
  t.momentum = d.momentum, t.lr = d.lr, t.keep = (float)(1.0 - (double)d.lr * d.weight_decay), t.nesterov = d.nesterov;
  return run<float, true>(d.orth, p, st);
}

}  // namespace nf
