// What the kernels of products share: their arguments, the copies from memory to LDS, and a tile's way from the accumulators through the
// forward's epilogue (bias, activation, dropout, residual) to memory, whole or as parts of sums that a second launch adds.
#pragma once
#include <hip/hip_runtime.h>

#include "pw_math.h"

namespace nf {
namespace {

constexpr int LT = 256;

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

// 8 neighbouring results of a row through the forward's epilogue; s holds the residual as it lies.  What a launch does not ask for is branched over:
// left to itself the compiler carries out both sides and chooses, 4 instructions an element, where GELU and all else take 27.
template <typename T>
__device__ inline void finish_fwd(const Epilogue &e, long long row, int col, int C, const float (&bias)[8], const Raw8<T> &s, float (&v)[8]) {
  const int n = C - col;
  const long long at = row * C + col;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] += bias[i];
  if (e.z) store8((T *)e.z + at, v, n);
  act_of<T>(e.act, v);
  drop8(e.drop, (unsigned long long)row * (unsigned)((C + 7) >> 3) + (unsigned)(col >> 3), v);
  if (e.res) {
    asm volatile("");
    float r[8];
    unpack8(s, r);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = fmaf(v[i], e.drop.scale, r[i]);
  } else if (e.drop.T) {  // else the scale is 1
    asm volatile("");
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] *= e.drop.scale;
  }
  store8((T *)e.out + at, v, n);
}
template <typename T>
__device__ inline void finish_fwd(const Epilogue &e, long long row, int col, int C, float (&v)[8]) {
  float bias[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) bias[i] = 0.f;
  Raw8<T> s = {};
  if (e.res) s = raw8((const T *)e.res + row * C + col, C - col);
  if (e.bias) load8(e.bias + col, bias, C - col);
  finish_fwd<T>(e, row, col, C, bias, s, v);
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

__device__ inline void barrier() {  // no LDS access moves across it
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// workgroups go round the 8 XCDs: each XCD gets a run of neighbouring tiles, which share operands in its L2
__device__ inline int xcd_run(int id, int n) {
  const int x = id & 7, q = n >> 3, r = n & 7;
  return x * q + min(x, r) + (id >> 3);
}

// A wave's sums, MT x NT fragments from row r0 and column c0 on, to where they go.  KEPT: sums stay in the accumulator registers until
// their turn (mfma_in_place).
// Gradients and parts of sums go straight from the registers.  A lane holds 4 neighbouring columns of a row; it gives those of every
// second fragment to the lane 16 further and takes its for the others, and then has 8.
template <typename T, int EPI, bool KEPT, int MT, int NT>
__device__ inline void write_sums(const GemmArgs &g, int split, long long r0, int c0, int lane, floatx4 (&acc)[MT][NT]) {
  const int i16 = lane & 15, q = lane >> 4, col0 = c0 + 16 * (q & 1) + 8 * (q >> 1);
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int p = 0; p < NT / 2; ++p) {  // a row's fragments one after the other: its memory lines are whole soon
      if constexpr (KEPT) asm volatile("" : "+a"(acc[i][2 * p]), "+a"(acc[i][2 * p + 1]));
      float v[8];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const auto t = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, (float)acc[i][2 * p][e]),
                                                        __builtin_bit_cast(uint32_t, (float)acc[i][2 * p + 1][e]), false, false);
        const uint32_t own = t[0], got = t[1];
        v[e] = __builtin_bit_cast(float, own), v[e + 4] = __builtin_bit_cast(float, got);
      }
      const long long row = r0 + 16 * i + i16;
      const int col = col0 + 32 * p, n = g.C - col;
      if (row >= g.R || n <= 0) continue;
      if (EPI == EPI_F32 || g.part)
        store8(g.part + (split * g.R + row) * g.part_ld + col, v, (int)min(g.part_ld - col, 8ll));
      else
        store8((T *)g.e.out + row * g.C + col, v, n);
    }
}

// The forward's go through LDS that only this wave uses, all rows or half of them at a time (HALF fragments): its epilogue is a loop, not a copy of its code to every
// fragment (80 KB of instructions, more than their cache holds), and a lane has 8 neighbours of a row: 16-byte accesses of 16 bits,
// whole lines, and one Philox call.  lds: 16 rows x NT fragments x 1 KB per 16 rows; chunk c of row r at c ^ (r & 15).
template <typename T, bool KEPT, int HALF, int MT, int NT>
__device__ inline void write_fwd(const GemmArgs &g, long long r0, int c0, int lane, floatx4 (&acc)[MT][NT], floatx4 *lds) {
  constexpr int CH = 4 * NT, ACROSS = 2 * NT, DOWN = 64 / ACROSS, TURNS = 16 * HALF / DOWN;
  const int c8 = lane % ACROSS, rr = lane / ACROSS, col = c0 + 8 * c8, n = g.C - col;
  float bias[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) bias[e] = 0.f;
  if (g.e.bias && n > 0) load8(g.e.bias + col, bias, n);
  auto fetch = [&](long long row) {
    Raw8<T> w = {};
    if (g.e.res && row < g.R && n > 0) w = raw8((const T *)g.e.res + row * g.C + col, n);
    return w;
  };
  constexpr int AHEAD = TURNS < 4 ? TURNS : 4;  // turns whose residuals are in flight while as many are finished
  Raw8<T> next[AHEAD];
  constexpr bool ALWAYS = sizeof(T) == 4;  // a branch over both costs fp32 results of a tile of 256 registers that they do not have
  if (ALWAYS || g.e.res) {
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) next[u] = fetch(r0 + rr + u * DOWN);
  }
#pragma unroll 1
  for (int h = 0; h < MT / HALF; ++h) {
    auto put = [&](int from) {
#pragma unroll
      for (int i = 0; i < HALF; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          if constexpr (KEPT) asm volatile("" : "+a"(acc[from + i][j]));
          const int r = 16 * i + (lane & 15), c = 4 * j + (lane >> 4);
          lds[r * CH + (c ^ (r & (CH - 1) & 15))] = acc[from + i][j];
        }
    };
    if (h == 0) {
      put(0);
      asm volatile("; the first rows" ::: "memory");  // else both halves' writes become one, with a choice of every sum
    } else {
      put(MT - HALF);
      asm volatile("; the others" ::: "memory");
    }
#pragma unroll 1
    for (int k0 = 0; k0 < TURNS; k0 += AHEAD) {
      Raw8<T> now[AHEAD];
      const long long first = r0 + rr + (h * TURNS + k0) * DOWN;  // turns run on through both halves
      if (ALWAYS || g.e.res) {
        if (!ALWAYS) asm volatile("");
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) now[u] = next[u];
        if (h * TURNS + k0 + AHEAD < MT / HALF * TURNS) {
#pragma unroll
          for (int u = 0; u < AHEAD; ++u) next[u] = fetch(first + (AHEAD + u) * DOWN);
        }
      }
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const int r = (k0 + u) * DOWN + rr;
        const floatx4 lo = lds[r * CH + ((2 * c8) ^ (r & (CH - 1) & 15))], hi = lds[r * CH + ((2 * c8 + 1) ^ (r & (CH - 1) & 15))];
        const long long row = first + u * DOWN;
        if (row >= g.R || n <= 0) continue;
        float v[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = lo[e], v[e + 4] = hi[e];
        finish_fwd<T>(g.e, row, col, g.C, bias, now[u], v);
      }
    }
  }
}

// Sums of the splits in order, and what follows them.  OUT is the results' type; FWD: the forward's epilogue.  A thread takes 8
// columns of a row; where there are few of those, `lanes` groups of a workgroup's threads share the splits of one.
struct FinishArgs {
  const float *part;
  int splits, C, lanes;  // lanes: 1, 4 or 16
  long long R;
  Epilogue e;
};
template <typename T, typename OUT, bool FWD>
__device__ inline void gemm_finish(const FinishArgs &f, long long block, float *lds) {
  const int items = f.lanes == 1 ? LT : f.lanes == 4 ? LT / 4 : LT / 16;
  const int groups = (f.C + 7) / 8, k = threadIdx.x & (items - 1), zl = f.lanes == 1 ? 0 : threadIdx.x / (f.lanes == 4 ? LT / 4 : LT / 16);
  const long long i = block * items + k, ld = 8ll * groups;
  const bool live = i < f.R * groups;
  const long long row = live ? i / groups : 0;
  const int col = live ? (int)(i - row * groups) * 8 : 0;
  float v[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = 0.f;
#pragma unroll 4
  for (int z = zl; z < f.splits; z += f.lanes) {
    float t[8];
    load8(f.part + (z * f.R + row) * ld + col, t);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += t[e];
  }
  if (f.lanes > 1) {
    float *const at = lds + threadIdx.x * 9;  // 9: neighbours in other banks
#pragma unroll
    for (int e = 0; e < 8; ++e) at[e] = v[e];
    __syncthreads();
    if (zl > 0) return;
    for (int q = 1; q < f.lanes; ++q) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += at[q * items * 9 + e];
    }
  }
  if (!live) return;
  if constexpr (FWD) {
    finish_fwd<T>(f.e, row, col, f.C, v);
  } else {
    store8((OUT *)f.e.out + row * f.C + col, v, f.C - col);
  }
}
template <typename T>
__global__ __launch_bounds__(LT) void fwd_finish_kernel(FinishArgs f) {
  __shared__ float lds[LT * 9];
  gemm_finish<T, T, true>(f, blockIdx.x, lds);
}
inline FinishArgs finish_args(int splits, const GemmArgs &g) {
  FinishArgs f = {g.part, splits, g.C, 1, g.R, g.e};
  // groups of threads that share an item's splits: towards 65536 threads, at least 2 splits each
  const long long items = g.R * ((g.C + 7) / 8);
  if (items < 65536 && splits >= 8) f.lanes = items >= 16384 || splits < 32 ? 4 : 16;
  if (splits == 1) f.R = 0;
  return f;
}
inline unsigned finish_blocks(const FinishArgs &f) { return (unsigned)((f.R * ((f.C + 7) / 8) * f.lanes + LT - 1) / LT); }

}  // namespace
}  // namespace nf
