// Products of the linear layers, y = r + D(act(x W^T + b)), dx = dz W, dW = dz^T x, and the epilogue's gradient.
//
// One tile kernel serves the three products.  It forms results[r][c] = sum over l of A(r, l) B(c, l) in tiles of BM x BN by four
// waves of BM/2 x BN/2 on 16x16 MFMAs.  A step is 128 bytes of the sum's axis: 64 terms of 16 bits or 32 of fp32.  An operand
// lies in memory with its terms together (x and W of the forward) or apart (a row of W, dz or x per term); the latter is
// staged as it lies and turned by the transposing LDS read (16 bits) or read word by word (fp32).
//   fragment    lane l holds row l % 16; with q = l / 16, the 8 terms 32 kk + 8 q + 0..7 of 16 bits (one 16x16x32 MFMA), or the
//               4 terms 16 kk + 4 q + 0..3 of fp32, one to each of four 16x16x4 MFMAs: the MFMAs' own term order does not
//               matter as long as A's and B's agree
//   LDS         rows of a step's bytes, or of a term's elements, whose chunks are exchanged so that those read together lie in
//               different banks (Staged::swizzle, turned_swizzle)
//   copies      memory to LDS without registers (buffer loads with LDS as their target, zeros for what lies outside) where rows
//               are whole 16 bytes, else through registers
//   order       the MFMA takes B's fragment first, so that a lane ends with 4 neighbouring columns of one row (write_sums)
#include <algorithm>
#include <type_traits>

#include "linear.h"
#include "nf_enqueue.h"

namespace nf {
namespace {

using shortx4 = __attribute__((ext_vector_type(4))) short;
using bf16x8 = __attribute__((ext_vector_type(8))) __bf16;
using f16x8 = __attribute__((ext_vector_type(8))) _Float16;

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
template <typename T, int BR, bool APART, int SB>
struct Staged {
  static constexpr int EPC = 16 / sizeof(T), STEP = SB / sizeof(T);
  static constexpr int ROWB = APART ? BR * (int)sizeof(T) : SB, CPR = ROWB / 16;
  static constexpr int BYTES = BR * SB, PIECES = BYTES / 1024 / 4;  // pieces of 1024 bytes per wave

  // Terms together: the LDS serves 16 lanes of a 16-byte read at a time, lanes 0-3, 12-15, 20-23 and 24-27 together, and so on: rows
  // 0-3 and 12-15 of one quarter, 4-11 of the next.  Their chunks lie in different banks with chunk c of a row of 128 bytes at
  // c ^ (row / 2 % 8); of 64 bytes, at c ^ (0, 2, 3, 1 by row / 4 % 4).
  static __device__ inline int swizzle(int row) {
    return SB == 128 ? (row >> 1) & 7 : ((row >> 2 ^ row >> 3) & 1) << 1 | (row >> 3 & 1);
  }

  // row and 16-byte chunk (in memory) that this lane brings for piece q
  static __device__ inline void place(int q, int wave, int lane, int &row, int &chunk) {
    const int at = ((q * 4 + wave) * 64 + lane);
    row = at / CPR;
    const int c = at % CPR;
    if constexpr (APART)
      chunk = c ^ (turned_swizzle<T, BR>(row) << (sizeof(T) == 4 ? 2 : 1));
    else
      chunk = c ^ swizzle(row);
  }

  // fragment of rows rb .. rb+15, half kk of the step
  static __device__ inline uintx4 fragment(const char *lds, int rb, int kk, int lane) {
    const int i = lane & 15, q = lane >> 4;
    if constexpr (!APART) {
      const int row = rb + i;
      return *reinterpret_cast<const uintx4 *>(lds + row * SB + (((kk * 4 + q) ^ swizzle(row)) << 4));
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

// bytes of LDS of a tile: two stages
template <int BM, int BN, int SB>
constexpr int tile_lds() {
  return 2 * (BM + BN) * SB;
}

template <typename T, int BM, int BN, int SB, bool AT, bool BT, int EPI, bool COPY>
__device__ inline void gemm_tile(const GemmArgs &g, int id, char *lds) {
  using A = Staged<T, BM, AT, SB>;
  using B = Staged<T, BN, BT, SB>;
  constexpr int STEP = A::STEP, MT = BM / 32, NT = BN / 32, STAGE = A::BYTES + B::BYTES;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
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
  const long long sa = AT ? STEP * g.lda : SB, sb = BT ? STEP * g.ldb : SB;
  const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds;

  // !COPY: through registers.  A chunk may begin at any element and end, as its row or the results do, in its middle: 16 bytes are read
  // all the same, from the neighbours behind it or, at the operand's last element, from those before it, without a branch
  // that would wait for them; they are shifted and cut when they go to LDS.
  uintx4 hold[A::PIECES + B::PIECES];
  int held[A::PIECES + B::PIECES];  // elements of it that lie inside, and from bit 8 on those read before it
  auto read16 = [&](int q, const char *p, const char *end, uint32_t off, int inside) {  // operands of 16 bytes or more (gemm_short)
    const int most = (int)min(end - p - 16, 0x7FFFFFF0ll), at = min((int)min(off, 0x7FFFFFFFu), most);
    held[q] = off == OUTSIDE ? 0 : max(min(inside, A::EPC), 0) | ((int)off - at) / (int)sizeof(T) << 8;
    __builtin_memcpy(&hold[q], p + at, 16);
  };
  auto cut = [&](int q) {
    asm volatile("" : "+v"(hold[q])::"memory");
    uintx4 v = hold[q];
    for (int d = held[q] >> 8; d > 0; --d) {
      if constexpr (sizeof(T) == 4)
        v[0] = v[1], v[1] = v[2], v[2] = v[3];
      else
        v[0] = v[0] >> 16 | v[1] << 16, v[1] = v[1] >> 16 | v[2] << 16, v[2] = v[2] >> 16 | v[3] << 16, v[3] >>= 16;
    }
    const int n = held[q] & 255;
    if (n < A::EPC) {
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        if constexpr (sizeof(T) == 4)
          v[w] = n > w ? v[w] : 0u;
        else
          v[w] = n > 2 * w + 1 ? v[w] : n == 2 * w + 1 ? v[w] & 0xFFFFu : 0u;
      }
    }
    return v;
  };
  const char *const end_a = g.a + (AT ? g.L : g.R) * g.lda, *const end_b = g.b + (BT ? g.L : (long long)g.C) * g.ldb;
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
        read16(q, qa, end_a, last ? avl[q] : av[q], (AT ? (int)min(rows_left, 1ll << 30) : terms) - chunk * A::EPC);
      }
#pragma unroll
      for (int q = 0; q < B::PIECES; ++q) {
        int row, chunk;
        B::place(q, wave, lane, row, chunk);
        read16(A::PIECES + q, qb, end_b, last ? bvl[q] : bv[q], (BT ? cols_left : terms) - chunk * B::EPC);
      }
    }
  };
  auto put = [&](int stage) {
    char *to = lds + stage * STAGE + wave * 1024 + lane * 16;
#pragma unroll
    for (int q = 0; q < A::PIECES; ++q) *reinterpret_cast<uintx4 *>(to + q * 4096) = cut(q);
#pragma unroll
    for (int q = 0; q < B::PIECES; ++q) *reinterpret_cast<uintx4 *>(to + A::BYTES + q * 4096) = cut(A::PIECES + q);
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
    barrier();
    const char *la = lds + cur * STAGE, *lb = la + A::BYTES;
#pragma unroll
    for (int kk = 0; kk < SB / 64; ++kk) {
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
    if constexpr (!COPY) {
      __builtin_amdgcn_sched_barrier(0);  // the reads are waited for here, not before the step's products
      if (s + 1 < steps) put(cur ^ 1);    // read last a step ago, behind the barrier above
    }
    wait_lds();
    barrier();
  }

  if (EPI == EPI_FWD && !g.part)
    write_fwd<T, false, MT * NT * 4096 <= 2 * STAGE ? MT : MT / 2>(g, r0 + wm, c0 + wn, lane, acc, reinterpret_cast<floatx4 *>(lds) + wave * (2 * STAGE / 64));
  else
    write_sums<T, EPI, false>(g, split, r0 + wm, c0 + wn, lane, acc);
}

// Two workgroups of 128x128 or five of 64x64 to a CU, whose waits overlap.  8192x1024x1024 bf16 24 us (717 TFLOP/s), fp32 133 (129);
// dW of 16384x2048x2048 bf16 140 (980); 22275x72x100 fp32 with its epilogue 12 us: a sum of 288 bytes is three steps, the last of 8 terms, that each
// wait for memory and two barriers, and the second tile of columns holds 36 of 64.
template <typename T, int BLOCK, int SB, bool AT, bool BT, int EPI, bool COPY>
__global__ __launch_bounds__(LT) void gemm_kernel(GemmArgs g) {
  __shared__ __align__(1024) char lds[tile_lds<BLOCK, BLOCK, SB>()];
  gemm_tile<T, BLOCK, BLOCK, SB, AT, BT, EPI, COPY>(g, xcd_run(blockIdx.x, gridDim.x), lds);
}

// ---- 256 x 256 tiles, 16 bits ----
// Eight waves of 128 x 64, two to a SIMD: one's MFMAs run while the other issues its copies (32 of the pipe's cycles each, measured)
// and address arithmetic.  A step is 32 terms; four stages of 32 KB.  While a step's MFMAs run, the next step's fragments are read
// and the copies of the third next are issued, between the MFMAs: one barrier a step, behind which a stage is whole and the one before
// it free.  128 accumulators and two sets of fragments take the 256 registers that two waves leave each other.
constexpr int WIDE = 256, WT = 512;

template <typename T, bool APART>
struct StagedWide {
  static constexpr int ROWB = APART ? WIDE * 2 : 64, CPR = ROWB / 16, BYTES = WIDE * 64, PIECES = BYTES / 8192;
  static __device__ inline void place(int q, int wave, int lane, int &row, int &chunk) {
    const int at = (q * 8 + wave) * 64 + lane;
    row = at / CPR;
    const int c = at % CPR;
    chunk = APART ? c ^ (turned_swizzle<T, WIDE>(row) << 1) : c ^ swizzle(row);
  }
  static __device__ inline int swizzle(int row) { return Staged<T, WIDE, false, 64>::swizzle(row); }
  // this lane's part of a fragment's address; fragment t of the wave's at rows w + 16 t
  static __device__ inline uint32_t lane_address(int w, int lane) {
    const int i = lane & 15, q = lane >> 4;
    if (!APART) return (uint32_t)((w + i) * 64 + ((q ^ swizzle(i)) << 4));
    const int row = q * 8 + (i >> 2);
    return (uint32_t)(row * ROWB + (((w >> 4) ^ turned_swizzle<T, WIDE>(row)) << 5) + (i & 3) * 8);
  }
  static __device__ inline uintx4 fragment(const char *lds, uint32_t at, int t) {
    if constexpr (!APART) {
      return *reinterpret_cast<const uintx4 *>(lds + at + t * 1024);
    } else {
      uintx4 f;
#pragma unroll
      for (int h = 0; h < 2; ++h) {  // the swizzle is the same for both halves: rows 4 apart
        const uint2 v = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                                      (__attribute__((address_space(3))) shortx4 *)(lds + (at ^ (t << 5)) + h * 4 * ROWB)));
        f[2 * h] = v.x, f[2 * h + 1] = v.y;
      }
      return f;
    }
  }
};

// c += the MFMA of a and b, in place in the accumulator registers: left to itself the compiler gives sums new registers, and
// with most of them taken moves them about.  What it does not see: a result may be read 18 cycles after its MFMA at the earliest, by another
// instruction than an MFMA that adds to it (settle_sums).
template <typename T>
__device__ inline void mfma_in_place(floatx4 &c, const uintx4 &a, const uintx4 &b) {
  if constexpr (__is_same(T, __bf16))
    asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
  else
    asm volatile("v_mfma_f32_16x16x32_f16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
}
template <int N>
__device__ inline void settle_sums(floatx4 (&c)[8][N]) {
#pragma unroll
  for (int i = 0; i < 8 * N; ++i) asm volatile("" : "+a"(c[i / N][i % N]));
  asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
#pragma unroll
  for (int i = 0; i < 8 * N; ++i) asm volatile("" : "+a"(c[i / N][i % N]));
}

// One workgroup to a CU: dx of 16384x2048x2048 bf16 112 us called by itself (1230 TFLOP/s), 127-131 between dW's kernels (1050-1080), bound by the
// matrix pipe and one barrier a step; 65536x512x512 forward 54 us, with GELU, dropout, residual and z 85 (bound by the epilogue behind the main loop).
template <typename T, bool AT, bool BT, int EPI>
__global__ __launch_bounds__(WT, 2) void gemm_wide_kernel(GemmArgs g) {
  using A = StagedWide<T, AT>;
  using B = StagedWide<T, BT>;
  constexpr int STEP = 32, STAGE = A::BYTES + B::BYTES, STAGES = 4;
  __shared__ __align__(1024) char lds[STAGES * STAGE];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int id = xcd_run(blockIdx.x, gridDim.x);
  const int split = id / g.tiles, tile = id - split * g.tiles, tr = tile / g.tiles_c;
  const long long r0 = (long long)tr * WIDE;
  const int c0 = (tile - tr * g.tiles_c) * WIDE;
  const long long l0 = split * g.per, l1 = min(g.L, l0 + g.per);
  const int steps = (int)((l1 - l0 + STEP - 1) / STEP), rest = (int)(l1 - l0 - (long long)(steps - 1) * STEP);
  uint32_t av[A::PIECES], bv[B::PIECES];
  uint32_t last = 0;  // bits of the pieces that lie inside the last step, too
#pragma unroll
  for (int q = 0; q < A::PIECES; ++q) {
    int row, chunk;
    A::place(q, wave, lane, row, chunk);
    av[q] = (uint32_t)(row * g.lda + chunk * 16);
    if (AT ? (long long)chunk * 8 >= g.R - r0 : row >= g.R - r0) av[q] = OUTSIDE;
    last |= (uint32_t)((AT ? row : chunk * 8) < rest) << q;
  }
#pragma unroll
  for (int q = 0; q < B::PIECES; ++q) {
    int row, chunk;
    B::place(q, wave, lane, row, chunk);
    bv[q] = (uint32_t)(row * g.ldb + chunk * 16);
    if (BT ? chunk * 8 >= g.C - c0 : row >= g.C - c0) bv[q] = OUTSIDE;
    last |= (uint32_t)((BT ? row : chunk * 8) < rest) << (A::PIECES + q);
  }
  const char *pa = g.a + (AT ? l0 * g.lda + r0 * 2 : r0 * g.lda + l0 * 2);
  const char *pb = g.b + (BT ? l0 * g.ldb + (long long)c0 * 2 : c0 * g.ldb + l0 * 2);
  const long long sa = AT ? STEP * g.lda : 64, sb = BT ? STEP * g.ldb : 64;
  const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds + wave * 1024;
  // piece q of step s, which lies `stage` stages into LDS; beyond the last step zeros, so that the counts of copies stay
  auto copy_piece = [&](int s, int stage, int q, const uintx4 &ba, const uintx4 &bb) {
    uint32_t off = q < A::PIECES ? av[q % A::PIECES] : bv[q % B::PIECES];
    if (s >= steps - 1) off = s == steps - 1 && (last >> q & 1) ? off : OUTSIDE;
    copy16(q < A::PIECES ? ba : bb, off, base + stage * STAGE + (q < A::PIECES ? q * 8192 : A::BYTES + (q - A::PIECES) * 8192));
  };
  constexpr int PIECES = A::PIECES + B::PIECES;
  const int wm = (wave >> 2) * 128, wn = (wave & 3) * 64;
  const uint32_t at_a = A::lane_address(wm, lane), at_b = B::lane_address(wn, lane) + A::BYTES;
  floatx4 acc[8][4];
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};

#pragma unroll
  for (int s = 0; s < STAGES - 1; ++s) {
    const uintx4 ba = buffer_of(pa), bb = buffer_of(pb);
#pragma unroll
    for (int q = 0; q < PIECES; ++q) copy_piece(s, s, q, ba, bb);
    pa += sa, pb += sb;
  }
  wait_copies<(STAGES - 2) * PIECES>();
  barrier();
  settle_sums(acc);  // the zeros, too, are there before the first MFMA reads them
  uintx4 fa[2][8], fb[2][4];
#pragma unroll
  for (int t = 0; t < 8; ++t) fa[0][t] = A::fragment(lds, at_a, t);
#pragma unroll
  for (int t = 0; t < 4; ++t) fb[0][t] = B::fragment(lds, at_b, t);
  // step s, the u-th of a turn, after which stages and sets of fragments are as before
  auto step = [&](auto turn, int s) {
    constexpr int u = decltype(turn)::value, cur = u & 1;
    wait_copies<(STAGES - 3) * PIECES>();  // of step s + 1: this wave's
    barrier();                             // everyone's; and step s - 1's fragments have been read
    const uintx4 ba = buffer_of(pa), bb = buffer_of(pb);
    pa += sa, pb += sb;
    const char *const next = lds + (u + 1) % STAGES * STAGE;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (i % 2 == 0) copy_piece(s + STAGES - 1, (u + STAGES - 1) % STAGES, i / 2, ba, bb);
      fa[cur ^ 1][i] = A::fragment(next, at_a, i);
      if (i % 2 == 1) fb[cur ^ 1][i / 2] = B::fragment(next, at_b, i / 2);
#pragma unroll
      for (int j = 0; j < 4; ++j) mfma_in_place<T>(acc[i][j], fb[cur][j], fa[cur][i]);
    }
    return s + 1 < steps;
  };
  for (int s = 0;; s += STAGES) {
    if (!step(std::integral_constant<int, 0>(), s)) break;
    if (!step(std::integral_constant<int, 1>(), s + 1)) break;
    if (!step(std::integral_constant<int, 2>(), s + 2)) break;
    if (!step(std::integral_constant<int, 3>(), s + 3)) break;
  }
  wait_copies<0>();
  settle_sums(acc);
  barrier();  // every wave has read its last fragments
  if (EPI == EPI_FWD && !g.part)
    write_fwd<T, true, 4>(g, r0 + wm, c0 + wn, lane, acc, reinterpret_cast<floatx4 *>(lds) + wave * 1024);
  else
    write_sums<T, EPI, true>(g, split, r0 + wm, c0 + wn, lane, acc);
}

// Both gradients in one launch: the first workgroups take dx's tiles, the others dW's.  Neither waits for the other, so the tail
// of one is filled by the other, and small layers pay one launch.
template <typename T, int BX, int BW, bool COPY>
__global__ __launch_bounds__(LT) void gemm_gradients_kernel(GemmArgs x, GemmArgs w) {
  constexpr int BIG = BX > BW ? BX : BW;
  __shared__ __align__(1024) char lds[tile_lds<BIG, BIG, 128>()];
  const int nx = x.tiles * x.splits, nx8 = (nx + 7) & ~7;  // dW starts at a multiple of the XCDs' number
  if ((int)blockIdx.x < nx8) {
    const int id = xcd_run(blockIdx.x, nx);
    if ((int)blockIdx.x < nx) gemm_tile<T, BX, BX, 128, false, true, EPI_STORE, COPY>(x, id, lds);
  } else {
    gemm_tile<T, BW, BW, 128, true, true, EPI_F32, COPY>(w, xcd_run(blockIdx.x - nx8, w.tiles * w.splits), lds);
  }
}

// The forward of few rows: 16 columns and up to 64 rows to a workgroup, whose waves share the sum's axis.  Weights and rows go
// from memory into the fragments, without LDS: nothing is used twice, and a wave's loads are in flight together.  A lane's 16 bytes
// need not follow the MFMA's term order (any order that x and W share will do): the four lanes of a row take 128 neighbouring bytes.
// Up to 8 rows (HALVES): the MFMA's 16 x 16 results hold 8 columns of W's first half of terms by x's, and 8 of the second by the
// second, so that twice as many workgroups share W.  Latency-bound; reads of W bound it from some MB on.
// Weights of a few elements (fwd_plan) come here with any number of rows: a grid's second axis ends at 65535, so 2^FEW_DOWN
// workgroups lie along it and the rest along the third.
constexpr int FEW_DOWN = 15;
template <typename T, int MT, int NW, bool HALVES, bool ALIGNED>
__global__ __launch_bounds__(64 * NW) void linear_few_rows_kernel(GemmArgs g) {
  constexpr int EPC = 16 / sizeof(T), ROWS = HALVES ? 8 : 16 * MT, COLS = HALVES ? 8 : 16;
  __shared__ floatx4 lds[NW * MT * 64];  // [wave][row of 16][4 chunks of 4 columns], chunk c at c ^ (row & 3)
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 15, q = lane >> 4;
  const int c0 = blockIdx.x * COLS;
  const long long r0 = (long long)(blockIdx.z << FEW_DOWN | blockIdx.y) * ROWS;
  if (r0 >= g.R) return;
  const int K = (int)g.L, all = (K * (int)sizeof(T) + 127) / 128, steps = HALVES ? (all + 1) / 2 : all;
  const int own = HALVES ? i & 7 : i, first = HALVES && i >= 8 ? steps * 8 : 0;  // first chunk
  const char *const w = g.b + min(c0 + own, g.C - 1) * g.ldb;  // rows beyond the last read it again; their results are not used
  const char *x[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) x[m] = g.a + min(r0 + 16 * m + own, g.R - 1) * g.lda;
  floatx4 acc[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) acc[m] = floatx4{0.f, 0.f, 0.f, 0.f};
  auto load = [&](const char *row, int term) -> uintx4 {
    uintx4 v;
    const int inside = K - term;
    if (ALIGNED) {  // whole chunks lie inside or outside: no branch, what lies outside is the last chunk, replaced by zeros
      v = *reinterpret_cast<const uintx4 *>(row + (long long)min(term, K - EPC) * (int)sizeof(T));
      const uint32_t keep = inside > 0 ? ~0u : 0u;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] &= keep;
    } else if (inside >= EPC) {
      __builtin_memcpy(&v, row + (long long)term * (int)sizeof(T), 16);
    } else {
      T t[EPC];
#pragma unroll
      for (int e = 0; e < EPC; ++e) t[e] = e < inside ? reinterpret_cast<const T *>(row)[term + e] : (T)0.f;
      __builtin_memcpy(&v, t, 16);
    }
    return v;
  };
  constexpr int U = MT == 4 ? 1 : 2;  // steps whose loads are in flight together
  for (int s0 = wave; s0 < steps; s0 += NW * U) {
    uintx4 fw[U][2], fx[U][MT][2];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (u == 0 || s0 + u * NW < steps) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int term = (first + (s0 + u * NW) * 8 + 2 * q + j) * EPC;
          fw[u][j] = load(w, term);
#pragma unroll
          for (int m = 0; m < MT; ++m) fx[u][m][j] = load(x[m], term);
        }
      }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (u == 0 || s0 + u * NW < steps) {
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int m = 0; m < MT; ++m) acc[m] = mfma<T>(fw[u][j], fx[u][m][j], acc[m]);
      }
  }
#pragma unroll
  for (int m = 0; m < MT; ++m) lds[(wave * MT * 16 + 16 * m + i) * 4 + (q ^ (i & 3))] = acc[m];
  __syncthreads();
  float *const sums = reinterpret_cast<float *>(lds);
  for (int t = threadIdx.x; t < MT * 256; t += 64 * NW) {
    float v = sums[t];
#pragma unroll
    for (int k = 1; k < NW; ++k) v += sums[k * MT * 256 + t];
    sums[t] = v;  // no other thread reads or writes these places before the barrier
  }
  __syncthreads();
  constexpr int GROUPS = COLS / 8;
  for (int t = threadIdx.x; t < ROWS * GROUPS; t += 64 * NW) {
    const int r = t / GROUPS, h = t % GROUPS, col = c0 + h * 8;
    if (r0 + r >= g.R || col >= g.C) continue;
    float v[8];
    const floatx4 lo = lds[r * 4 + ((2 * h) ^ (r & 3))], hi = lds[r * 4 + ((2 * h + 1) ^ (r & 3))];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = lo[e], v[e + 4] = hi[e];
    if (HALVES) {  // row r + 8, columns 8 ... 15
      const floatx4 lo2 = lds[(r + 8) * 4 + (2 ^ (r & 3))], hi2 = lds[(r + 8) * 4 + (3 ^ (r & 3))];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += lo2[e], v[e + 4] += hi2[e];
    }
    finish_fwd<T>(g.e, r0 + r, col, g.C, v);
  }
}

// Gradients with an operand of less than 16 bytes: sums of at most 7 terms, a thread each, bound by the launch or the results' writes.
// Strides in elements.
template <typename T, typename OUT>
__global__ __launch_bounds__(LT) void gemm_short_kernel(const T *__restrict__ a, long long ra, long long la, const T *__restrict__ b,
                                                        long long cb, long long lb, OUT *__restrict__ out, long long R, int C, int L) {
  const long long i = (long long)blockIdx.x * LT + threadIdx.x;
  if (i >= R * C) return;
  const long long r = i / C;
  const int c = (int)(i - r * C);
  float s = 0.f;
  for (int l = 0; l < L; ++l) s = fmaf((float)a[r * ra + l * la], (float)b[c * cb + l * lb], s);
  out[i] = (OUT)s;
}

// of both gradients: the first nx workgroups finish dx, the others dW
template <typename T>
__global__ __launch_bounds__(LT) void gradients_finish_kernel(FinishArgs x, FinishArgs w, unsigned nx) {
  __shared__ float lds[LT * 9];
  if (blockIdx.x < nx)
    gemm_finish<T, T, false>(x, blockIdx.x, lds);
  else
    gemm_finish<T, float, false>(w, blockIdx.x - nx, lds);
}

// ---- the epilogue's gradient ----
// dz = act'(z) D(dy); a thread keeps 8 columns and walks the rows of its workgroup's part, so that the columns' sums stay in
// registers.  part [row parts][ld], or db itself where there is one row part.  HBM-bound: 3 * sizeof(T) bytes an element; the random
// numbers, the slope and conversions are 39 vector instructions an element.  65536x512 bf16 with both 47 us, 4.3 TB/s, and 4.7 for the parts' sums.
template <typename T>
__global__ __launch_bounds__(LT) void linear_epilogue_kernel(long long M, int N, long long per, int tx, const T *__restrict__ dy, const T *__restrict__ z,
                                                             Epilogue e, float *part, int ld) {
  __shared__ float sums[LT * 8];
  const int groups = (N + 7) / 8, ty = LT / tx;  // tx threads across, ty down
  const int x = threadIdx.x % tx, y = threadIdx.x / tx, g8 = blockIdx.x * tx + x, col = g8 * 8, n = N - col;
  float s[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) s[k] = 0.f;
  const long long m0 = blockIdx.y * per, m1 = min(M, m0 + per);
  T *const out = (T *)e.out;
  if (g8 < groups && y < ty) {
    constexpr int U = 4;  // rows whose reads are in flight together
    for (long long m = m0 + y; m < m1; m += U * ty) {
      Raw8<T> d[U], zr[U];
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (m + u * ty < m1) {
          d[u] = raw8(dy + (m + u * ty) * N + col, n);
          if (e.act != NF_ACT_NONE) zr[u] = raw8(z + (m + u * ty) * N + col, n);
        }
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (m + u * ty < m1) {
          const long long row = m + u * ty;
          float v[8];
          unpack8(d[u], v);
          drop8(e.drop, (unsigned long long)row * (unsigned)groups + (unsigned)g8, v);
          if (e.act != NF_ACT_NONE) {
            float zv[8];
            unpack8(zr[u], zv);
            times_slope<T>(e.act, zv, v);
          }
#pragma unroll
          for (int k = 0; k < 8; ++k) v[k] *= e.drop.scale, s[k] += v[k];
          store8(out + row * N + col, v, n);
        }
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
    if (cc < ld) part[(long long)blockIdx.y * ld + cc] = t;
  }
}

// out[c] = sum over rows of part[row][c]: 16 columns to a workgroup of 64 x 16 threads, in a fixed order
constexpr int CT = 1024;
__global__ __launch_bounds__(CT) void column_sums_kernel(const float *__restrict__ part, int rows, long long ld, int C,
                                                         float *__restrict__ out) {
  __shared__ float s[64][17];
  const int x = threadIdx.x & 15, y = threadIdx.x >> 4, c = blockIdx.x * 16 + x;
  float sum = 0.f;
  if (c < C) {
#pragma unroll 8
    for (int r = y; r < rows; r += 64) sum += part[r * ld + c];
  }
  s[y][x] = sum;
  __syncthreads();
  const int col = threadIdx.x >> 6, lane = threadIdx.x & 63;
  sum = s[lane][col];
#pragma unroll
  for (int k = 32; k; k >>= 1) sum += __shfl_xor(sum, k);
  if (lane == 0 && blockIdx.x * 16 + col < C) out[blockIdx.x * 16 + col] = sum;
}

// ---- plans ----
struct Plan {
  int tile, splits;
  long long per;
  size_t bytes;  // of the splits' sums
};

// What a product in tiles of 128 or 64 takes, its sum in `splits` parts, in us: the first copies and the results, then steps of 128
// bytes.  With c workgroups on the busiest CU a step takes c times the CU's own time for it, or a single step's latency; parts are
// written and read again (6.3 TB/s) in a launch of their own.  The figures are a fit to 900 runs of products from 300x300x4000
// to 128x128x65536.  By them the choice is on average 1 % behind the fastest tiles and parts measured, at most 15 %; splitting until 512
// workgroups run, whatever the parts weigh, was 30 % (16 bits) and 16 % behind (4096x1024x1024 bf16 26.6 us in 512 workgroups, 16.2 in 1024
// of tiles of 64 without parts).
struct TileTimes {
  double first, latency, rate;
};
double product_time(long long tiles, long long steps, int splits, double results, bool large, int size, bool whole) {
  constexpr TileTimes T16[2][2] = {{{5.5, 0.93, 0.39}, {8, 1.63, 1.0}}, {{5, 0.26, 0.19}, {8, 0.5, 0.4}}};
  constexpr TileTimes T32[2][2] = {{{7.5, 1.17, 0.74}, {10, 2.9, 2.45}}, {{6, 0.63, 0.52}, {9, 2.0, 1.9}}};
  const TileTimes &t = size == 2 ? T16[whole][large] : T32[whole][large];
  const double each = (double)((steps + splits - 1) / splits), c = (double)((tiles * splits + 255) / 256);
  return t.first + each * std::max(t.latency, t.rate * c) + (splits > 1 ? 2.5 + splits * results * 8 / 6.3e6 : 0.0);
}

// Tiles of 256 (16 bits, whole 16-byte rows) where their rounds over the 256 CUs take less time than those of two 128s to a CU:
// 1.55 us a step of 128 bytes and 13 more a round against 0.95 and 7.5; not where the sum must be split, whose parts are four times as
// large, nor where a tile's columns or rows are a quarter empty (33770x512x136 forward 28 us, in tiles of 128 and 64 17).  And only in
// rounds that are nearly whole, since smaller tiles share out what is left (us in tiles of 256, and of 128 and 64):
//   forward, whose epilogue a round waits for: 7/8 of the last round and 4 steps.  65536x1024x256 51 and 58, 65536x192x256 26 and 25, 65536x64x512 41
//     and 35; 20000x256x512, 158 tiles, 25 and 18; 40000x1024x1000, 628 tiles, 128 and 116
//   gradients: 3/4 of it, or 8 steps.  dx 65536x256x1024 39 and 50, 65536x256x32 11 and 12; 20000x512x1024, 158 tiles, 28 and 30, 20000x512x192 13
//     and 12; dW 3000x4000 of 1024 rows, 192 tiles, 36 and 39, of 128 19 and 18
// (8192x1024x1024, 128 tiles, 39 and 25: their times decide.)  Else the quickest of tiles of 128 or 64 and of 1 to 512 parts.
Plan plan_of(long long R, int C, long long L, int size, bool whole, bool fwd) {
  const int step = 128 / size;
  const long long steps = (L + step - 1) / step;
  auto tiles = [&](int b) { return ((R + b - 1) / b) * ((C + b - 1) / b); };
  Plan p;
  p.tile = 128, p.splits = 1;
  const long long large = tiles(WIDE), rounds = (large + 255) / 256;
  const bool wide = size == 2 && whole && large >= 128 && 4 * R * C >= 3 * large * WIDE * WIDE &&
                    (fwd ? steps >= 4 && 8 * large >= 7 * 256 * rounds : steps >= 8 || 4 * large >= 3 * 256 * rounds) &&
                    (double)rounds * (1.55 * steps + 13) < (double)((tiles(128) + 511) / 512) * (0.95 * steps + 7.5);
  if (wide) {
    p.tile = WIDE;
  } else {
    double best = 1e300;
    for (const int b : {128, 64}) {
      const long long t = tiles(b);
      for (int s = 1; s <= steps && (s == 1 || (s <= 512 && t * s <= 2048)); s += s < 4 ? 1 : (s & (s - 1)) ? s / 3 : s / 2) {
        const double time = product_time(t, steps, s, (double)R * C, b == 128, size, whole);
        if (time < best) best = time, p.tile = b, p.splits = s;
      }
    }
  }
  const long long each = (steps + p.splits - 1) / p.splits;
  p.splits = (int)((steps + each - 1) / each);
  p.per = each * step;
  p.bytes = p.splits > 1 ? (size_t)p.splits * R * ((C + 7) / 8 * 8) * 4 : 0;
  return p;
}

// The forward: tiles, or few rows.  Few rows where there are up to 32 (1x2048x2048 bf16 4.4 us, tiles 7.1; 16 rows 6.7 and 8.2), and
// for small products (256x512x256 5.7 and 7.3); from sums of 2 KB and more than 32 rows on, tiles that share x and W through LDS
// (64x2048x2048 12.4 and 9.9).  And weights of less than the 16 bytes that the tile kernel reads at a time.
constexpr int FEW_ROWS = 0;
Plan fwd_plan(long long M, int N, int K, int size) {
  Plan p = plan_of(M, N, K, size, K * size % 16 == 0, true);
  const long long t64 = ((M + 63) / 64) * ((N + 63) / 64);
  if (M <= 32 || (t64 <= 64 && (long long)K * size <= 2048) || (long long)N * K * size < 16) p.tile = FEW_ROWS, p.splits = 1, p.bytes = 0;
  return p;
}

// fills the tiles of a plan; returns the number of workgroups
int lay(const Plan &p, GemmArgs &g) {
  g.tiles_c = (g.C + p.tile - 1) / p.tile;
  g.tiles = (int)((g.R + p.tile - 1) / p.tile) * g.tiles_c;
  g.splits = p.splits, g.per = p.per;
  return g.tiles * g.splits;
}

template <typename T, bool AT, bool BT, int EPI, typename F>
void go_wide(F go) {
  if constexpr (sizeof(T) == 2) go(gemm_wide_kernel<T, AT, BT, EPI>);
}

// bytes of a product's operands and results
template <typename T>
double product_bytes(const GemmArgs &g, double result_size) {
  return sizeof(T) * ((double)g.R * g.L + (double)g.C * g.L) + result_size * g.R * g.C;
}
inline double product_flops(const GemmArgs &g) { return 2.0 * g.R * g.C * g.L; }

template <typename T, int MT, int NW, bool HALVES>
hipError_t few_rows_as(const GemmArgs &g, const char *const (&names)[2], hipStream_t st) {
  constexpr int ROWS = HALVES ? 8 : 16 * MT, COLS = HALVES ? 8 : 16;
  const unsigned down = (unsigned)((g.R + ROWS - 1) / ROWS);
  const dim3 grid((g.C + COLS - 1) / COLS, std::min(down, 1u << FEW_DOWN), (down + (1u << FEW_DOWN) - 1) >> FEW_DOWN);
  const bool aligned = g.lda % 16 == 0;
  return recorded(st, names[!aligned], product_flops(g), product_bytes<T>(g, sizeof(T) * (1.0 + (g.e.res != nullptr) + (g.e.z != nullptr))), [&] {
    if (aligned)
      hipLaunchKernelGGL((linear_few_rows_kernel<T, MT, NW, HALVES, true>), grid, dim3(64 * NW), 0, st, g);
    else
      hipLaunchKernelGGL((linear_few_rows_kernel<T, MT, NW, HALVES, false>), grid, dim3(64 * NW), 0, st, g);
  });
}
template <typename T>
hipError_t run_few_rows(const GemmArgs &g, hipStream_t st) {
  static const char *const names[4][2][2] = {
      {{"linear_fwd_8_rows", "linear_fwd_8_rows_odd"}, {"linear_fwd_8_rows_long", "linear_fwd_8_rows_long_odd"}},
      {{"linear_fwd_16_rows", "linear_fwd_16_rows_odd"}, {"linear_fwd_16_rows_long", "linear_fwd_16_rows_long_odd"}},
      {{"linear_fwd_32_rows", "linear_fwd_32_rows_odd"}, {"linear_fwd_32_rows_long", "linear_fwd_32_rows_long_odd"}},
      {{"linear_fwd_64_rows", "linear_fwd_64_rows_odd"}, {"linear_fwd_64_rows_long", "linear_fwd_64_rows_long_odd"}}};
  const bool many = g.L * (int)sizeof(T) > 8 * 128;  // waves without a step would only wait
  if (g.R <= 8) return many ? few_rows_as<T, 1, 16, true>(g, names[0][1], st) : few_rows_as<T, 1, 4, true>(g, names[0][0], st);
  if (g.R <= 16) return many ? few_rows_as<T, 1, 16, false>(g, names[1][1], st) : few_rows_as<T, 1, 4, false>(g, names[1][0], st);
  if (g.R <= 32) return many ? few_rows_as<T, 2, 16, false>(g, names[2][1], st) : few_rows_as<T, 2, 4, false>(g, names[2][0], st);
  return many ? few_rows_as<T, 4, 16, false>(g, names[3][1], st) : few_rows_as<T, 4, 4, false>(g, names[3][0], st);
}

// names of the tile kernels of a product: tiles of 256, of 128 and of 64, those for rows of any alignment behind
using TileNames = const char *const[5];
inline const char *tile_name(const TileNames &n, int tile, bool copy) { return n[tile == WIDE ? 0 : (tile == 128 ? 1 : 2) + (copy ? 0 : 2)]; }
constexpr TileNames FWD_NAMES = {"linear_fwd_256x256", "linear_fwd_128x128", "linear_fwd_64x64", "linear_fwd_128x128_odd", "linear_fwd_64x64_odd"};
constexpr TileNames DX_NAMES = {"linear_dx_256x256", "linear_dx_128x128", "linear_dx_64x64", "linear_dx_128x128_odd", "linear_dx_64x64_odd"};
constexpr TileNames DW_NAMES = {"linear_dw_256x256", "linear_dw_128x128", "linear_dw_64x64", "linear_dw_128x128_odd", "linear_dw_64x64_odd"};

template <typename T>
hipError_t fwd_as(const LinearCall &c, const void *x, const void *W, const float *b, const void *r, const DropArgs &drop,
                  void *y, void *z, void *ws, hipStream_t st) {
  const Plan p = fwd_plan(c.M, c.N, c.K, sizeof(T));
  GemmArgs g = {};
  g.a = (const char *)x, g.b = (const char *)W, g.lda = g.ldb = (long long)c.K * sizeof(T);
  g.R = c.M, g.C = c.N, g.L = c.K;
  g.e = Epilogue{b, r, z, y, drop, c.act};
  if (p.tile == FEW_ROWS) return run_few_rows<T>(g, st);
  if (p.splits > 1) g.part = (float *)ws, g.part_ld = (c.N + 7) / 8 * 8;
  const dim3 grid(lay(p, g));
  const bool copy = g.lda % 16 == 0;
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(LT), 0, st, g); };
  auto wide = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(WT), 0, st, g); };
  const double ends = sizeof(T) * (1.0 + (r != nullptr) + (z != nullptr));
  const hipError_t e = recorded(st, tile_name(FWD_NAMES, p.tile, copy), product_flops(g), product_bytes<T>(g, p.splits > 1 ? 4.0 * p.splits : ends), [&] {
    if (p.tile == WIDE)
      go_wide<T, false, false, EPI_FWD>(wide);
    else if (p.tile == 128)
      copy ? go(gemm_kernel<T, 128, 128, false, false, EPI_FWD, true>) : go(gemm_kernel<T, 128, 128, false, false, EPI_FWD, false>);
    else
      copy ? go(gemm_kernel<T, 64, 128, false, false, EPI_FWD, true>) : go(gemm_kernel<T, 64, 128, false, false, EPI_FWD, false>);
  });
  if (e != hipSuccess || p.splits == 1) return e;
  const FinishArgs f = finish_args(p.splits, g);
  return recorded(st, "linear_fwd_finish", 0.0, (4.0 * p.splits + ends) * g.R * g.C,
                  [&] { hipLaunchKernelGGL(fwd_finish_kernel<T>, dim3(finish_blocks(f)), dim3(LT), 0, st, f); });
}

// whether an operand of a product, of a or b elements, is shorter than the 16 bytes that the tile kernel reads at a time
inline bool gemm_short(long long a, long long b, int size) { return std::min(a, b) * size < 16; }

// The workspace holds dx's splits, then dW's.  Products in the same kind of tiles share a launch, and so does what adds up their
// splits; a measurement that wants them one by one gets them so.
template <typename T>
hipError_t bwd_as(const LinearCall &c, const void *dz, const void *x, const void *W, void *dx, float *dW, void *ws,
                  hipStream_t st) {
  const long long ldn = (long long)c.N * sizeof(T), ldk = (long long)c.K * sizeof(T);
  const bool copy = ldn % 16 == 0 && ldk % 16 == 0, apart = g_prof.on && g_prof.apart;
  auto blocks = [](long long n) { return dim3((unsigned)((n + LT - 1) / LT)); };
  GemmArgs gx = {}, gw = {};
  gx.a = (const char *)dz, gx.b = (const char *)W, gx.lda = ldn, gx.ldb = ldk;
  gx.R = c.M, gx.C = c.K, gx.L = c.N, gx.e.out = dx;
  gw.a = (const char *)dz, gw.b = (const char *)x, gw.lda = ldn, gw.ldb = ldk;
  gw.R = c.N, gw.C = c.K, gw.L = c.M, gw.e.out = dW;
  hipError_t e = hipSuccess;
  if (dx && gemm_short(c.M * c.N, (long long)c.N * c.K, sizeof(T))) {
    e = recorded(st, "linear_dx_short", product_flops(gx), product_bytes<T>(gx, sizeof(T)), [&] {
      hipLaunchKernelGGL((gemm_short_kernel<T, T>), blocks(c.M * c.K), dim3(LT), 0, st, (const T *)dz, (long long)c.N, 1ll, (const T *)W, 1ll,
                         (long long)c.K, (T *)dx, c.M, c.K, c.N);
    });
    dx = nullptr;
  }
  if (e == hipSuccess && dW && gemm_short(c.M * c.N, c.M * c.K, sizeof(T))) {
    e = recorded(st, "linear_dw_short", product_flops(gw), product_bytes<T>(gw, 4.0), [&] {
      hipLaunchKernelGGL((gemm_short_kernel<T, float>), blocks((long long)c.N * c.K), dim3(LT), 0, st, (const T *)dz, 1ll, (long long)c.N,
                         (const T *)x, 1ll, (long long)c.K, dW, (long long)c.N, c.K, (int)c.M);
    });
    dW = nullptr;
  }
  if (e != hipSuccess || (!dx && !dW)) return e;
  const Plan px = plan_of(c.M, c.K, c.N, sizeof(T), copy, false), pw = plan_of(c.N, c.K, c.M, sizeof(T), copy, false);
  if (px.splits > 1) gx.part = (float *)ws, gx.part_ld = (c.K + 7) / 8 * 8;
  gw.part = pw.splits > 1 ? (float *)((char *)ws + px.bytes) : dW, gw.part_ld = pw.splits > 1 ? (c.K + 7) / 8 * 8 : c.K;
  const int nx = lay(px, gx), nw = lay(pw, gw);
  const double bytes_x = product_bytes<T>(gx, px.splits > 1 ? 4.0 * px.splits : sizeof(T)), bytes_w = product_bytes<T>(gw, 4.0 * pw.splits);
  if (dx && dW && px.tile != WIDE && pw.tile != WIDE && !apart) {
    static const char *const names[2][2][2] = {{{"linear_gradients_64_64", "linear_gradients_64_64_odd"}, {"linear_gradients_64_128", "linear_gradients_64_128_odd"}},
                                               {{"linear_gradients_128_64", "linear_gradients_128_64_odd"}, {"linear_gradients_128_128", "linear_gradients_128_128_odd"}}};
    const dim3 grid((unsigned)((nx + 7) / 8 * 8 + nw));
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(LT), 0, st, gx, gw); };
    auto sized = [&](auto cp) {
      constexpr bool C = decltype(cp)::value;
      if (px.tile == 128)
        pw.tile == 128 ? go(gemm_gradients_kernel<T, 128, 128, C>) : go(gemm_gradients_kernel<T, 128, 64, C>);
      else
        pw.tile == 128 ? go(gemm_gradients_kernel<T, 64, 128, C>) : go(gemm_gradients_kernel<T, 64, 64, C>);
    };
    e = recorded(st, names[px.tile == 128][pw.tile == 128][!copy], product_flops(gx) + product_flops(gw), bytes_x + bytes_w,
                 [&] { copy ? sized(std::true_type()) : sized(std::false_type()); });
  } else {
    if (dx) {
      auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(nx), dim3(LT), 0, st, gx); };
      auto wide = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(nx), dim3(WT), 0, st, gx); };
      e = recorded(st, tile_name(DX_NAMES, px.tile, copy), product_flops(gx), bytes_x, [&] {
        if (px.tile == WIDE)
          go_wide<T, false, true, EPI_STORE>(wide);
        else if (px.tile == 128)
          copy ? go(gemm_kernel<T, 128, 128, false, true, EPI_STORE, true>) : go(gemm_kernel<T, 128, 128, false, true, EPI_STORE, false>);
        else
          copy ? go(gemm_kernel<T, 64, 128, false, true, EPI_STORE, true>) : go(gemm_kernel<T, 64, 128, false, true, EPI_STORE, false>);
      });
    }
    if (e == hipSuccess && dW) {
      auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(nw), dim3(LT), 0, st, gw); };
      auto wide = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(nw), dim3(WT), 0, st, gw); };
      e = recorded(st, tile_name(DW_NAMES, pw.tile, copy), product_flops(gw), bytes_w, [&] {
        if (pw.tile == WIDE)
          go_wide<T, true, true, EPI_F32>(wide);
        else if (pw.tile == 128)
          copy ? go(gemm_kernel<T, 128, 128, true, true, EPI_F32, true>) : go(gemm_kernel<T, 128, 128, true, true, EPI_F32, false>);
        else
          copy ? go(gemm_kernel<T, 64, 128, true, true, EPI_F32, true>) : go(gemm_kernel<T, 64, 128, true, true, EPI_F32, false>);
      });
    }
  }
  if (e != hipSuccess) return e;
  FinishArgs fx = finish_args(px.splits, gx), fw = finish_args(pw.splits, gw);
  if (!dx) fx.R = 0;
  if (!dW) fw.R = 0;
  auto finish = [&](const char *name, unsigned bx, unsigned bw) {
    return recorded(st, name, 0.0, (4.0 * px.splits + sizeof(T)) * (bx ? (double)gx.R * gx.C : 0.0) + 4.0 * (pw.splits + 1) * (bw ? (double)gw.R * gw.C : 0.0),
                    [&] { hipLaunchKernelGGL(gradients_finish_kernel<T>, dim3(bx + bw), dim3(LT), 0, st, fx, fw, bx); });
  };
  const unsigned bx = finish_blocks(fx), bw = finish_blocks(fw);
  if (bx && bw && !apart) return finish("linear_gradients_finish", bx, bw);
  if (bx) e = finish("linear_dx_finish", bx, 0);
  if (e == hipSuccess && bw) e = finish("linear_dw_finish", 0, bw);
  return e;
}

// the epilogue gradient's row parts: up to 1024 workgroups, 4 rows or more to a thread
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
  long long ny = std::max<long long>(1, std::min<long long>(1024 / p.nx, M / (4ll * ty)));
  p.per = (M + ny - 1) / ny;
  p.ny = (int)((M + p.per - 1) / p.per);
  return p;
}

}  // namespace

size_t linear_fwd_workspace_bytes(const LinearCall &c) { return fwd_plan(c.M, c.N, c.K, c.dtype == NF_F32 ? 4 : 2).bytes; }

size_t linear_workspace_bytes(const LinearCall &c) {
  const int size = c.dtype == NF_F32 ? 4 : 2;
  const EpiPlan e = epi_plan(c.M, c.N);
  const size_t fwd = linear_fwd_workspace_bytes(c);
  const bool whole = c.N * size % 16 == 0 && c.K * size % 16 == 0;
  const size_t bwd = plan_of(c.M, c.K, c.N, size, whole, false).bytes + plan_of(c.N, c.K, c.M, size, whole, false).bytes;
  return std::max(std::max(fwd, bwd), (size_t)e.ny * ((c.N + 7) / 8) * 32);
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
  const Epilogue e = {nullptr, nullptr, nullptr, dz, drop, c.act};
  // one row part's sums are db
  const int ld = p.ny == 1 ? c.N : (c.N + 7) / 8 * 8;
  float *part = !db ? nullptr : p.ny == 1 ? db : (float *)ws;
  const dim3 grid(p.nx, p.ny);
  const double size = c.dtype == NF_F32 ? 4.0 : 2.0;
  const hipError_t err = recorded(st, "linear_bwd_epilogue", 0.0, size * (c.act != NF_ACT_NONE ? 3.0 : 2.0) * c.M * c.N, [&] {
    auto go = [&](auto t) {
      using T = decltype(t);
      hipLaunchKernelGGL((linear_epilogue_kernel<T>), grid, dim3(LT), 0, st, c.M, c.N, p.per, p.tx, (const T *)dy, (const T *)z, e, part, ld);
    };
    if (c.dtype == NF_BF16)
      go((__bf16)0.f);
    else if (c.dtype == NF_F16)
      go((_Float16)0.f);
    else
      go(0.f);
  });
  if (err != hipSuccess || !db || p.ny == 1) return err;
  return recorded(st, "linear_bias_sums", 0.0, 4.0 * (p.ny + 1) * c.N, [&] {
    hipLaunchKernelGGL(column_sums_kernel, dim3((c.N + 15) / 16), dim3(CT), 0, st, part, p.ny, (long long)ld, c.N, db);
  });
}

}  // namespace nf
