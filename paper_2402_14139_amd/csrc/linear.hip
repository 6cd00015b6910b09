// Products of the linear layers, y = r + D(act(x W^T + b)), dx = dz W, dW = dz^T x, and the epilogue's gradient.
//
// One tile kernel serves the three products.  It forms results[r][c] = sum over l of A(r, l) B(c, l) in tiles of BM x BN by four
// waves of BM/2 x BN/2 on 16x16 MFMAs.  A step is 128 bytes of the sum's axis: 64 terms of 16 bits or 32 of fp32.  An operand
// lies in memory with its terms together (x and W of the forward) or apart (a row of W, dz or x per term); the latter is
// staged as it lies and turned by the transposing LDS read (16 bits) or read word by word (fp32).
//   fragment    lane l holds row l % 16; with q = l / 16, the 8 terms 32 kk + 8 q + 0..7 of 16 bits (one 16x16x32 MFMA), or the
//               4 terms 16 kk + 4 q + 0..3 of fp32, one to each of four 16x16x4 MFMAs: the MFMAs' own term order does not
//               matter as long as A's and B's agree
//   LDS         terms together: rows of 128 bytes, 16-byte chunk c of row r at c ^ ((r >> 1) & 7), so that the 16 rows of a
//               fragment lie in 16 different bank groups; terms apart: see turned_swizzle
//   copies      memory to LDS without registers (buffer loads with LDS as their target, zeros for what lies outside) where rows
//               are whole 16 bytes, else through registers
//   order       the MFMA takes B's fragment first, so that a lane ends with 4 neighbouring columns of one row
#include <algorithm>

#include "pw_math.h"

namespace nf {
namespace {

constexpr int LT = 256;

using shortx4 = __attribute__((ext_vector_type(4))) short;
using bf16x8 = __attribute__((ext_vector_type(8))) __bf16;
using f16x8 = __attribute__((ext_vector_type(8))) _Float16;

enum { EPI_FWD, EPI_STORE, EPI_F32 };

struct Epilogue {
  const float *bias;
  const void *res;
  void *z, *out;
  DropArgs drop;
  int act;
};

struct GemmArgs {
  const char *a, *b;
  long long lda, ldb;  // bytes from a stored row to the next
  long long R, L;      // rows of the result, terms of a sum
  int C, tiles_c, tiles, splits;
  long long per;  // terms of a split, whole steps
  float *part;    // sums of the splits [splits][R][part_ld], or null
  long long part_ld;
  Epilogue e;
};

// 8 neighbouring results of a row through the forward's epilogue
template <typename T>
__device__ inline void finish_fwd(const Epilogue &e, long long row, int col, int C, const float bias[8], float (&v)[8]) {
  const int n = C - col;
  const long long at = row * C + col;
  float s[8];
  if (e.res) load8((const T *)e.res + at, s, n);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] += bias[i];
  if (e.z) store8((T *)e.z + at, v, n);
  act_of<T>(e.act, v);
  drop8(e.drop, (unsigned long long)row * (unsigned)((C + 7) >> 3) + (unsigned)(col >> 3), v);
  if (e.res) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += s[i];
  }
  store8((T *)e.out + at, v, n);
}

// Where the terms lie apart an LDS row is one term's BR elements, and a fragment's read takes 32 bytes (16 bits) or 64 bytes
// (fp32) from each of several rows.  The row's units of that size are exchanged by this number so that rows read together
// lie in different banks: the transposing read takes rows 8 q + 0..3 of two q at a time, the word read rows 4 q of all four.
template <typename T, int BR>
__device__ inline int turned_swizzle(int row) {
  if constexpr (sizeof(T) == 4) return (row >> 2) & 3;
  if constexpr (BR >= 128) return (row & 3) | ((row >> 3) & 1) << 2;
  return ((row >> 1) & 1) | ((row >> 3) & 1) << 1;  // two rows to 256 bytes: their parity separates them already
}

// One operand's part of a tile: BR rows of results (or columns), one step of terms.
template <typename T, int BR, bool APART>
struct Staged {
  static constexpr int EPC = 16 / sizeof(T), STEP = 128 / sizeof(T);
  static constexpr int ROWB = APART ? BR * (int)sizeof(T) : 128, CPR = ROWB / 16;
  static constexpr int BYTES = BR * 128, PIECES = BYTES / 1024 / 4;  // pieces of 1024 bytes per wave

  // row and 16-byte chunk (in memory) that this lane brings for piece q
  static __device__ inline void place(int q, int wave, int lane, int &row, int &chunk) {
    const int at = ((q * 4 + wave) * 64 + lane);
    row = at / CPR;
    const int c = at % CPR;
    if constexpr (APART)
      chunk = c ^ (turned_swizzle<T, BR>(row) << (sizeof(T) == 4 ? 2 : 1));
    else
      chunk = c ^ ((row >> 1) & 7);
  }

  // fragment of rows rb .. rb+15, half kk of the step
  static __device__ inline uintx4 fragment(const char *lds, int rb, int kk, int lane) {
    const int i = lane & 15, q = lane >> 4;
    if constexpr (!APART) {
      const int row = rb + i;
      return *reinterpret_cast<const uintx4 *>(lds + row * 128 + (((kk * 4 + q) ^ ((row >> 1) & 7)) << 4));
    } else if constexpr (sizeof(T) == 2) {
      uintx4 f;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int row = kk * 32 + q * 8 + h * 4 + (i >> 2);
        const char *p = lds + row * ROWB + (((rb >> 4) ^ turned_swizzle<T, BR>(row)) << 5) + (i & 3) * 8;
        const uint2 t = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                                      (__attribute__((address_space(3))) shortx4 *)p));
        f[2 * h] = t.x, f[2 * h + 1] = t.y;
      }
      return f;
    } else {
      uintx4 f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int row = kk * 16 + q * 4 + j;
        f[j] = *reinterpret_cast<const uint32_t *>(lds + row * ROWB + (((rb >> 4) ^ turned_swizzle<T, BR>(row)) << 6) + i * 4);
      }
      return f;
    }
  }
};

template <typename T>
__device__ inline floatx4 mfma(const uintx4 &a, const uintx4 &b, floatx4 c) {
  if constexpr (sizeof(T) == 4) {
    const floatx4 x = __builtin_bit_cast(floatx4, a), y = __builtin_bit_cast(floatx4, b);
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[j], y[j], c, 0, 0, 0);
    return c;
  } else if constexpr (__is_same(T, __bf16)) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  } else {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
}

constexpr uint32_t OUTSIDE = 0xF0000000u;  // beyond every buffer's end: reads as zeros

__device__ inline uintx4 buffer_of(const char *p) {
  const unsigned long long u = (unsigned long long)p;
  uintx4 r;
  r[0] = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)u);
  r[1] = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(u >> 32)) & 0xFFFFu;
  r[2] = 0x7FFFFFFFu, r[3] = 0x00020000u;
  return r;
}
// 16 bytes per lane from memory to LDS at `to` + 16 * lane.  Nothing lands in a register, so nothing but the wait on vmcnt and the
// barrier behind it orders the LDS reads that follow.  Nothing else in these kernels uses m0.
__device__ inline void copy16(const uintx4 &buf, uint32_t voff, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(voff), "s"(buf) : "memory");
}
template <int N>
__device__ inline void wait_copies() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
__device__ inline void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// workgroups go round the 8 XCDs: each XCD gets a run of neighbouring tiles, which share operands in its L2
__device__ inline int xcd_run(int id, int n) {
  const int x = id & 7, q = n >> 3, r = n & 7;
  return x * q + min(x, r) + (id >> 3);
}

template <typename T, int BM, int BN, bool AT, bool BT, int EPI, bool COPY>
__global__ __launch_bounds__(LT) void gemm_kernel(GemmArgs g) {
  using A = Staged<T, BM, AT>;
  using B = Staged<T, BN, BT>;
  constexpr int STEP = A::STEP, MT = BM / 32, NT = BN / 32, STAGE = A::BYTES + B::BYTES;
  __shared__ __align__(1024) char lds[2 * STAGE];  // holds the tile's fp32 results, BM * BN * 4, at the end
  static_assert(BM * BN * 4 <= 2 * STAGE, "");
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int id = xcd_run(blockIdx.x, g.tiles * g.splits);
  const int split = id / g.tiles, tile = id - split * g.tiles, tr = tile / g.tiles_c;
  const long long r0 = (long long)tr * BM;
  const int c0 = (tile - tr * g.tiles_c) * BN;
  const long long l0 = split * g.per, l1 = min(g.L, l0 + g.per);
  const int steps = (int)((l1 - l0 + STEP - 1) / STEP);
  const int rest = (int)(l1 - l0 - (long long)(steps - 1) * STEP);  // terms of the last step
  // what this lane brings, as offsets from the step's first byte, and the same for the last step
  uint32_t av[A::PIECES], avl[A::PIECES], bv[B::PIECES], bvl[B::PIECES];
  const long long rows_left = g.R - r0;
  const int cols_left = g.C - c0;
#pragma unroll
  for (int q = 0; q < A::PIECES; ++q) {
    int row, chunk;
    A::place(q, wave, lane, row, chunk);
    av[q] = (uint32_t)(row * g.lda + chunk * 16);
    if (AT ? (long long)chunk * A::EPC >= rows_left : row >= rows_left) av[q] = OUTSIDE;
    avl[q] = (AT ? row : chunk * A::EPC) >= rest ? OUTSIDE : av[q];
  }
#pragma unroll
  for (int q = 0; q < B::PIECES; ++q) {
    int row, chunk;
    B::place(q, wave, lane, row, chunk);
    bv[q] = (uint32_t)(row * g.ldb + chunk * 16);
    if (BT ? chunk * B::EPC >= cols_left : row >= cols_left) bv[q] = OUTSIDE;
    bvl[q] = (BT ? row : chunk * B::EPC) >= rest ? OUTSIDE : bv[q];
  }
  const char *pa = g.a + (AT ? l0 * g.lda + r0 * (long long)sizeof(T) : r0 * g.lda + l0 * (long long)sizeof(T));
  const char *pb = g.b + (BT ? l0 * g.ldb + c0 * (long long)sizeof(T) : c0 * g.ldb + l0 * (long long)sizeof(T));
  const long long sa = AT ? STEP * g.lda : 128, sb = BT ? STEP * g.ldb : 128;
  const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds;

  uintx4 hold[A::PIECES + B::PIECES];  // !COPY only
  // elements of a chunk that lie inside: the chunk's own terms or neighbours may end in its middle
  auto edge16 = [&](const char *p, uint32_t off, int inside) -> uintx4 {
    uintx4 v = {0, 0, 0, 0};
    if (off == OUTSIDE) return v;
    if (inside >= A::EPC) {
      __builtin_memcpy(&v, p + off, 16);
    } else {
      T t[A::EPC];
#pragma unroll
      for (int e = 0; e < A::EPC; ++e) t[e] = (T)0.f;
#pragma unroll
      for (int e = 0; e < A::EPC; ++e)
        if (e < inside) t[e] = reinterpret_cast<const T *>(p + off)[e];
      __builtin_memcpy(&v, t, 16);
    }
    return v;
  };
  auto fetch = [&](int s, int stage) {
    const bool last = s + 1 == steps;
    const char *qa = pa + s * sa, *qb = pb + s * sb;
    if constexpr (COPY) {
      const uintx4 ba = buffer_of(qa), bb = buffer_of(qb);
      const uint32_t to = base + stage * STAGE + wave * 1024;
#pragma unroll
      for (int q = 0; q < A::PIECES; ++q) copy16(ba, last ? avl[q] : av[q], to + q * 4096);
#pragma unroll
      for (int q = 0; q < B::PIECES; ++q) copy16(bb, last ? bvl[q] : bv[q], to + A::BYTES + q * 4096);
    } else {
      const int terms = last ? rest : STEP;
#pragma unroll
      for (int q = 0; q < A::PIECES; ++q) {
        int row, chunk;
        A::place(q, wave, lane, row, chunk);
        hold[q] = edge16(qa, last ? avl[q] : av[q], (AT ? (int)min(rows_left, 1ll << 30) : terms) - chunk * A::EPC);
      }
#pragma unroll
      for (int q = 0; q < B::PIECES; ++q) {
        int row, chunk;
        B::place(q, wave, lane, row, chunk);
        hold[A::PIECES + q] = edge16(qb, last ? bvl[q] : bv[q], (BT ? cols_left : terms) - chunk * B::EPC);
      }
    }
  };
  auto put = [&](int stage) {
    char *to = lds + stage * STAGE + wave * 1024 + lane * 16;
#pragma unroll
    for (int q = 0; q < A::PIECES; ++q) *reinterpret_cast<uintx4 *>(to + q * 4096) = hold[q];
#pragma unroll
    for (int q = 0; q < B::PIECES; ++q) *reinterpret_cast<uintx4 *>(to + A::BYTES + q * 4096) = hold[A::PIECES + q];
  };

  const int wm = (wave >> 1) * (BM / 2), wn = (wave & 1) * (BN / 2);
  floatx4 acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};

  fetch(0, 0);
  if constexpr (!COPY) put(0);
  for (int s = 0; s < steps; ++s) {
    const int cur = s & 1;
    if (s + 1 < steps) {
      fetch(s + 1, cur ^ 1);
      if constexpr (COPY) wait_copies<A::PIECES + B::PIECES>();
    } else {
      if constexpr (COPY) wait_copies<0>();
    }
    wait_lds();
    __builtin_amdgcn_s_barrier();
    const char *la = lds + cur * STAGE, *lb = la + A::BYTES;
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      uintx4 fa[MT], fb[NT];
#pragma unroll
      for (int i = 0; i < MT; ++i) fa[i] = A::fragment(la, wm + i * 16, kk, lane);
#pragma unroll
      for (int j = 0; j < NT; ++j) fb[j] = B::fragment(lb, wn + j * 16, kk, lane);
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = mfma<T>(fb[j], fa[i], acc[i][j]);
    }
    if constexpr (!COPY)
      if (s + 1 < steps) put(cur ^ 1);  // read last a step ago, behind the barrier above
    wait_lds();
    __builtin_amdgcn_s_barrier();
  }

  // the tile's results through LDS: row-wise 8 neighbours per thread, 16-byte stores and one Philox call each
  float *const res = reinterpret_cast<float *>(lds);
  constexpr int CH = BN / 4;  // 16-byte chunks of a row; chunk c of row r lies at c ^ (r & 15)
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const int r = wm + i * 16 + (lane & 15), c = (wn + j * 16) / 4 + (lane >> 4);
      reinterpret_cast<floatx4 *>(res)[r * CH + (c ^ (r & 15))] = acc[i][j];
    }
  __syncthreads();
  const int c8 = tid % (BN / 8), col = c0 + c8 * 8;
  if (col >= g.C) return;
  float bias[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) bias[e] = 0.f;
  if (EPI == EPI_FWD && g.e.bias) load8(g.e.bias + col, bias, g.C - col);
#pragma unroll 2
  for (int r = tid / (BN / 8); r < BM; r += LT / (BN / 8)) {
    if (r0 + r >= g.R) break;
    float v[8];
    const floatx4 lo = reinterpret_cast<const floatx4 *>(res)[r * CH + ((2 * c8) ^ (r & 15))];
    const floatx4 hi = reinterpret_cast<const floatx4 *>(res)[r * CH + ((2 * c8 + 1) ^ (r & 15))];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = lo[e], v[e + 4] = hi[e];
    if (EPI == EPI_F32 || g.part)
      store8(g.part + (split * g.R + r0 + r) * g.part_ld + col, v, (int)min(g.part_ld - col, 8ll));
    else if (EPI == EPI_FWD)
      finish_fwd<T>(g.e, r0 + r, col, g.C, bias, v);
    else
      store8((T *)g.e.out + (r0 + r) * g.C + col, v, g.C - col);
  }
}

// Sums of the splits in order, and what follows them.  OUT is the results' type; FWD: the forward's epilogue.
template <typename T, typename OUT, bool FWD>
__global__ __launch_bounds__(LT) void gemm_finish_kernel(const float *__restrict__ part, int splits, long long R, int C,
                                                         Epilogue e) {
  const int groups = (C + 7) / 8;
  const long long i = (long long)blockIdx.x * LT + threadIdx.x, ld = 8ll * groups;
  if (i >= R * groups) return;
  const long long row = i / groups;
  const int col = (int)(i - row * groups) * 8;
  float v[8];
  load8(part + row * ld + col, v);
  for (int z = 1; z < splits; ++z) {
    float t[8];
    load8(part + (z * R + row) * ld + col, t);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] += t[k];
  }
  if constexpr (FWD) {
    float bias[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) bias[k] = 0.f;
    if (e.bias) load8(e.bias + col, bias, C - col);
    finish_fwd<T>(e, row, col, C, bias, v);
  } else {
    store8((OUT *)e.out + row * C + col, v, C - col);
  }
}

// ---- the epilogue's gradient ----
// dz = act'(z) D(dy); a thread keeps 8 columns and walks the rows of its workgroup's part, so that the columns' sums stay in
// registers.  part [row parts][groups * 8].  HBM-bound: 3 * sizeof(T) bytes an element.
template <typename T>
__global__ __launch_bounds__(LT) void linear_epilogue_kernel(long long M, int N, long long per, int tx, const T *dy, const T *z,
                                                             Epilogue e, float *part) {
  __shared__ float sums[LT * 8];
  const int groups = (N + 7) / 8, ty = LT / tx;  // tx threads across, ty down
  const int x = threadIdx.x % tx, y = threadIdx.x / tx, g8 = blockIdx.x * tx + x, col = g8 * 8, n = N - col;
  float s[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) s[k] = 0.f;
  const long long m0 = blockIdx.y * per, m1 = min(M, m0 + per);
  if (g8 < groups && y < ty) {
    for (long long m = m0 + y; m < m1; m += ty) {
      float v[8], zv[8];
      load8(dy + m * N + col, v, n);
      if (e.act != NF_ACT_NONE) load8(z + m * N + col, zv, n);
      drop8(e.drop, (unsigned long long)m * (unsigned)groups + (unsigned)g8, v);
      if (e.act != NF_ACT_NONE) times_slope<T>(e.act, zv, v);
#pragma unroll
      for (int k = 0; k < 8; ++k) s[k] += v[k];
      store8((T *)e.out + m * N + col, v, n);
    }
  }
  if (!part) return;
#pragma unroll
  for (int k = 0; k < 8; ++k) sums[threadIdx.x * 8 + k] = s[k];
  __syncthreads();
  const int across = tx * 8;
  for (int c = threadIdx.x; c < across; c += LT) {
    float t = 0.f;
    for (int q = 0; q < ty; ++q) t += sums[q * across + c];
    const int cc = blockIdx.x * across + c;
    if (cc < groups * 8) part[(long long)blockIdx.y * groups * 8 + cc] = t;
  }
}

// out[c] = sum over rows of part[row][c], 16 rows of threads to 16 columns, in a fixed order
__global__ __launch_bounds__(LT) void column_sums_kernel(const float *__restrict__ part, int rows, long long ld, int C,
                                                         float *__restrict__ out) {
  __shared__ float s[16][17];
  const int x = threadIdx.x & 15, y = threadIdx.x >> 4, c = blockIdx.x * 16 + x;
  float sum = 0.f;
  if (c < C)
    for (int r = y; r < rows; r += 16) sum += part[r * ld + c];
  s[y][x] = sum;
  __syncthreads();
  if (y == 0 && c < C) {
#pragma unroll
    for (int q = 1; q < 16; ++q) sum += s[q][x];
    out[c] = sum;
  }
}

// ---- plans ----
struct Plan {
  int tile, splits;
  long long per;
  size_t bytes;  // of the splits' sums
};

Plan plan_of(long long R, int C, long long L, int size, bool to_f32) {
  const int step = 128 / size;
  const long long steps = (L + step - 1) / step;
  auto tiles = [&](int b) { return ((R + b - 1) / b) * ((C + b - 1) / b); };
  Plan p;
  p.tile = tiles(128) * steps >= 2048 || tiles(128) >= 192 ? 128 : 64;
  const long long t = tiles(p.tile);
  long long s = std::min<long long>(512 / t, steps / 4);
  if (s < 1) s = 1;
  const long long each = (steps + s - 1) / s;
  p.splits = (int)((steps + each - 1) / each);
  p.per = each * step;
  p.bytes = p.splits > 1 ? (size_t)p.splits * R * ((C + 7) / 8 * 8) * 4 : 0;
  return p;
}

template <typename T, bool AT, bool BT, int EPI>
hipError_t run_gemm(const Plan &p, GemmArgs g, bool copy, hipStream_t st) {
  const int b = p.tile;
  g.tiles_c = (g.C + b - 1) / b;
  g.tiles = (int)((g.R + b - 1) / b) * g.tiles_c;
  g.splits = p.splits, g.per = p.per;
  const dim3 grid((unsigned)(g.tiles * g.splits));
  if (b == 128) {
    if (copy)
      hipLaunchKernelGGL((gemm_kernel<T, 128, 128, AT, BT, EPI, true>), grid, dim3(LT), 0, st, g);
    else
      hipLaunchKernelGGL((gemm_kernel<T, 128, 128, AT, BT, EPI, false>), grid, dim3(LT), 0, st, g);
  } else {
    if (copy)
      hipLaunchKernelGGL((gemm_kernel<T, 64, 64, AT, BT, EPI, true>), grid, dim3(LT), 0, st, g);
    else
      hipLaunchKernelGGL((gemm_kernel<T, 64, 64, AT, BT, EPI, false>), grid, dim3(LT), 0, st, g);
  }
  return hipGetLastError();
}

template <typename T, typename OUT, bool FWD>
hipError_t run_finish(const Plan &p, const GemmArgs &g, hipStream_t st) {
  const long long items = g.R * ((g.C + 7) / 8);
  hipLaunchKernelGGL((gemm_finish_kernel<T, OUT, FWD>), dim3((unsigned)((items + LT - 1) / LT)), dim3(LT), 0, st, g.part, p.splits, g.R, g.C, g.e);
  return hipGetLastError();
}

template <typename T>
hipError_t fwd_as(const LinearCall &c, const void *x, const void *W, const float *b, const void *r, const DropArgs &drop,
                  void *y, void *z, void *ws, hipStream_t st) {
  const Plan p = plan_of(c.M, c.N, c.K, sizeof(T), false);
  GemmArgs g = {};
  g.a = (const char *)x, g.b = (const char *)W, g.lda = g.ldb = (long long)c.K * sizeof(T);
  g.R = c.M, g.C = c.N, g.L = c.K;
  g.e = Epilogue{b, r, z, y, drop, c.act};
  if (p.splits > 1) g.part = (float *)ws, g.part_ld = (c.N + 7) / 8 * 8;
  const hipError_t e = run_gemm<T, false, false, EPI_FWD>(p, g, g.lda % 16 == 0, st);
  if (e != hipSuccess || p.splits == 1) return e;
  return run_finish<T, T, true>(p, g, st);
}

template <typename T>
hipError_t bwd_as(const LinearCall &c, const void *dz, const void *x, const void *W, void *dx, float *dW, void *ws,
                  hipStream_t st) {
  const long long ldn = (long long)c.N * sizeof(T), ldk = (long long)c.K * sizeof(T);
  const bool copy = ldn % 16 == 0 && ldk % 16 == 0;
  if (dx) {
    const Plan p = plan_of(c.M, c.K, c.N, sizeof(T), false);
    GemmArgs g = {};
    g.a = (const char *)dz, g.b = (const char *)W, g.lda = ldn, g.ldb = ldk;
    g.R = c.M, g.C = c.K, g.L = c.N;
    g.e.out = dx;
    if (p.splits > 1) g.part = (float *)ws, g.part_ld = (c.K + 7) / 8 * 8;
    hipError_t e = run_gemm<T, false, true, EPI_STORE>(p, g, copy, st);
    if (e == hipSuccess && p.splits > 1) e = run_finish<T, T, false>(p, g, st);
    if (e != hipSuccess) return e;
  }
  if (dW) {
    const Plan p = plan_of(c.N, c.K, c.M, sizeof(T), true);
    GemmArgs g = {};
    g.a = (const char *)dz, g.b = (const char *)x, g.lda = ldn, g.ldb = ldk;
    g.R = c.N, g.C = c.K, g.L = c.M;
    g.e.out = dW;
    g.part = p.splits > 1 ? (float *)ws : dW, g.part_ld = p.splits > 1 ? (c.K + 7) / 8 * 8 : c.K;
    hipError_t e = run_gemm<T, true, true, EPI_F32>(p, g, copy, st);
    if (e == hipSuccess && p.splits > 1) e = run_finish<T, float, false>(p, g, st);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// the epilogue gradient's row parts: about 1024 workgroups, 8 rows or more to a thread
struct EpiPlan {
  int tx, nx, ny;
  long long per;
};
EpiPlan epi_plan(long long M, int N) {
  EpiPlan p;
  const int groups = (N + 7) / 8;
  p.tx = std::min(groups, LT);
  p.nx = (groups + p.tx - 1) / p.tx;
  const int ty = LT / p.tx;
  long long ny = std::max<long long>(1, std::min<long long>(1024 / p.nx, M / (8ll * ty)));
  p.per = (M + ny - 1) / ny;
  p.ny = (int)((M + p.per - 1) / p.per);
  return p;
}

}  // namespace

size_t linear_workspace_bytes(const LinearCall &c) {
  const int size = c.dtype == NF_F32 ? 4 : 2;
  const EpiPlan e = epi_plan(c.M, c.N);
  const size_t all[] = {plan_of(c.M, c.N, c.K, size, false).bytes, plan_of(c.M, c.K, c.N, size, false).bytes,
                        plan_of(c.N, c.K, c.M, size, true).bytes, (size_t)e.ny * ((c.N + 7) / 8) * 32};
  return *std::max_element(all, all + 4);
}

hipError_t launch_linear_fwd(const LinearCall &c, const void *x, const void *W, const float *b, const void *r,
                             const DropArgs &drop, void *y, void *z, void *ws, hipStream_t st) {
  if (c.dtype == NF_BF16) return fwd_as<__bf16>(c, x, W, b, r, drop, y, z, ws, st);
  if (c.dtype == NF_F16) return fwd_as<_Float16>(c, x, W, b, r, drop, y, z, ws, st);
  return fwd_as<float>(c, x, W, b, r, drop, y, z, ws, st);
}

hipError_t launch_linear_bwd(const LinearCall &c, const void *dz, const void *x, const void *W, void *dx, float *dW,
                             void *ws, hipStream_t st) {
  if (c.dtype == NF_BF16) return bwd_as<__bf16>(c, dz, x, W, dx, dW, ws, st);
  if (c.dtype == NF_F16) return bwd_as<_Float16>(c, dz, x, W, dx, dW, ws, st);
  return bwd_as<float>(c, dz, x, W, dx, dW, ws, st);
}

hipError_t launch_linear_epilogue(const LinearCall &c, const void *dy, const void *z, const DropArgs &drop, void *dz,
                                  float *db, void *ws, hipStream_t st) {
  const EpiPlan p = epi_plan(c.M, c.N);
  Epilogue e = {};
  e.out = dz, e.drop = drop, e.act = c.act;
  float *part = db ? (float *)ws : nullptr;
  const dim3 grid(p.nx, p.ny);
  if (c.dtype == NF_BF16)
    hipLaunchKernelGGL((linear_epilogue_kernel<__bf16>), grid, dim3(LT), 0, st, c.M, c.N, p.per, p.tx, (const __bf16 *)dy, (const __bf16 *)z, e, part);
  else if (c.dtype == NF_F16)
    hipLaunchKernelGGL((linear_epilogue_kernel<_Float16>), grid, dim3(LT), 0, st, c.M, c.N, p.per, p.tx, (const _Float16 *)dy, (const _Float16 *)z, e, part);
  else
    hipLaunchKernelGGL((linear_epilogue_kernel<float>), grid, dim3(LT), 0, st, c.M, c.N, p.per, p.tx, (const float *)dy, (const float *)z, e, part);
  hipError_t err = hipGetLastError();
  if (err != hipSuccess || !db) return err;
  const int ld = (c.N + 7) / 8 * 8;
  hipLaunchKernelGGL(column_sums_kernel, dim3((c.N + 15) / 16), dim3(LT), 0, st, part, p.ny, (long long)ld, c.N, db);
  return hipGetLastError();
}

}  // namespace nf
