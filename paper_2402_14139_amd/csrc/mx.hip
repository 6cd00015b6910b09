// Matrices in 4 bits an element with an exponent to every 32 (rows as those of the e2m1 cache): quantisation by rows and by columns, and
// products of two such matrices, y = r + D(act(a b^T + bias)), on the scaled matrix instructions.
#include <algorithm>
#include <type_traits>

#include "linear.h"
#include "nf_enqueue.h"
#include "q_codes.h"

namespace nf {
namespace {

constexpr int QT = 256;

// ---- quantisation ----
// The largest magnitude of a group is found on the elements' bits, whose order is that of the magnitudes (an infinity and a NaN behind all numbers): two
// 16-bit elements to an instruction.  The conversion divides by 2^E, rounds to nearest, ties to even, and takes elements as they lie; of its scale
// it reads the exponent bits, which are the group's exponent byte.
template <typename T>
__device__ inline uint32_t most(uint32_t m, const Raw8<T> &r) {
#pragma unroll
  for (int i = 0; i < (int)(sizeof(T) / 2) * 4; ++i) {
    const uint32_t w = r.w[i / 4][i % 4];
    if constexpr (sizeof(T) == 4) {
      m = max(m, w & 0x7FFFFFFFu);
    } else {
      using ushort2v = __attribute__((ext_vector_type(2))) unsigned short;
      m = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(ushort2v, m), __builtin_bit_cast(ushort2v, w & 0x7FFF7FFFu)));
    }
  }
  return m;
}
// E + 127 of a group from most()'s bits, or 255 where the group holds no number: with the magnitude m 2^e, 1 <= m < 2, E = e - 2, or e - 1 where m > 1.5
template <typename T>
__device__ inline int group_exponent(uint32_t m) {
  uint32_t bits = m;
  if constexpr (sizeof(T) == 2) {
    const uint32_t h = max(m & 0xFFFFu, m >> 16);
    bits = __is_same(T, __bf16) ? h << 16 : __builtin_bit_cast(uint32_t, (float)__builtin_bit_cast(_Float16, (unsigned short)h));
  }
  if (bits >= 0x7F800000u) return 255;
  return max((int)(bits >> 23) - 2 + ((bits & 0x7FFFFFu) > 0x400000u), 0);
}
template <typename T>
__device__ inline uint32_t codes8(const Raw8<T> &r, int eb) {
  const float scale = __builtin_bit_cast(float, (uint32_t)eb << 23);
  uint32_t w = 0;
  if constexpr (sizeof(T) == 4) {
    const floatx4 a = __builtin_bit_cast(floatx4, r.w[0]), b = __builtin_bit_cast(floatx4, r.w[1]);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, a[0], a[1], scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, a[2], a[3], scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, b[0], b[1], scale, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, b[2], b[3], scale, 3);
  } else {
    using V = __attribute__((ext_vector_type(2))) T;
    const uint32_t p0 = r.w[0][0], p1 = r.w[0][1], p2 = r.w[0][2], p3 = r.w[0][3];  // a bit_cast of a vector's element would take its first
    auto two = [](uint32_t p) { return __builtin_bit_cast(V, p); };
    if constexpr (__is_same(T, __bf16)) {
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, two(p0), scale, 0);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, two(p1), scale, 1);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, two(p2), scale, 2);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, two(p3), scale, 3);
    } else {
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(w, two(p0), scale, 0);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(w, two(p1), scale, 1);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(w, two(p2), scale, 2);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(w, two(p3), scale, 3);
    }
  }
  return w;
}
// a group of 32 elements that a thread holds
template <typename T>
__device__ inline int group32(const Raw8<T> (&r)[4], uintx4 &codes) {
  uint32_t m = 0;
#pragma unroll
  for (int h = 0; h < 4; ++h) m = most(m, r[h]);
  const int eb = group_exponent<T>(m);
#pragma unroll
  for (int h = 0; h < 4; ++h) codes[h] = eb < 255 ? codes8(r[h], eb) : 0u;
  return eb;
}

struct QuantArgs {
  long long rows, cols, tiles_c, groups;         // groups of a row
  uint8_t *codes, *scales, *codes_t, *scales_t;  // one pair may be null
  long long cb, sb, cbt, sbt;                    // row strides
};

// By rows: a group to a thread, whose reads are in flight together.  Memory-bound: sizeof(T) + 1/2 + 1/32 bytes an element.  16384x2048 bf16 19 us from HBM
// (4.4 TB/s), 14.5 from the last-level cache; by columns 21.6 and 15, both ways 32.5 and 21.8, whose codes are lines of 32 and 64 bytes.
template <typename T>
__global__ __launch_bounds__(QT) void mx_rows_kernel(QuantArgs a, const T *__restrict__ x) {
  const long long first = (long long)blockIdx.x * QT, row0 = first / a.groups;
  const unsigned at = (unsigned)(first - row0 * a.groups) + threadIdx.x, groups = (unsigned)a.groups;  // at most 2^31 groups to a row
  const long long row = row0 + at / groups;
  const unsigned group = at % groups;
  if (row >= a.rows) return;
  const long long col = (long long)group * GROUP;
  const int n = (int)min(a.cols - col, (long long)GROUP);
  Raw8<T> r[4] = {};
#pragma unroll
  for (int h = 0; h < 4; ++h)
    if (n > 8 * h) r[h] = raw8(x + row * a.cols + col + 8 * h, n - 8 * h);
  uintx4 codes;
  const int eb = group32(r, codes);
  *reinterpret_cast<uintx4 *>(a.codes + row * a.cb + col / 2) = codes;
  a.scales[row * a.sb + group] = (uint8_t)eb;
}

// By columns, or both: a tile of 128 rows x 64 columns to a workgroup.  A thread reads pieces of 8 elements of a row, of which 4 neighbours share an
// exponent and write their codes; for the columns the tile goes through LDS as it lies, and a thread takes 32 rows of a column, four neighbours
// the 128 (64 bytes of codes; a column to 64 lanes, 16 bytes here and there, took 21.8 us for 65536x512 bf16 instead of 16.2).
constexpr int TR = 128, TC = 64;
template <typename T, bool BY_ROWS>
__global__ __launch_bounds__(QT) void mx_columns_kernel(QuantArgs a, const T *__restrict__ x) {
  constexpr int LD = TC + 4 / sizeof(T), BAND = 32 * LD + 16;  // 32 rows; the four that a wave reads from lie in different banks
  __shared__ T lds[TR / 32 * BAND];
  const long long tr = blockIdx.x / a.tiles_c, r0 = tr * TR, c0 = (blockIdx.x - tr * a.tiles_c) * TC;
  const int j = threadIdx.x & 7, down = threadIdx.x >> 3;
  const long long col = c0 + 8 * j;
  const int n = (int)min(max(a.cols - col, 0ll), 8ll);
  Raw8<T> raw[TR / 32] = {};
#pragma unroll
  for (int k = 0; k < TR / 32; ++k) {
    const long long row = r0 + k * 32 + down;
    if (row < a.rows && n > 0) raw[k] = raw8(x + row * a.cols + col, n);
  }
#pragma unroll
  for (int k = 0; k < TR / 32; ++k) {
    __builtin_memcpy(&lds[k * BAND + down * LD + 8 * j], &raw[k], sizeof(raw[k]));
    if constexpr (BY_ROWS) {
      const long long row = r0 + k * 32 + down;
      uint32_t m = most(0u, raw[k]);
      if constexpr (sizeof(T) == 2) m = max(m & 0xFFFFu, m >> 16);
      m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xB1, 0xF, 0xF, true));  // the other of two, the other two of four
      m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x4E, 0xF, 0xF, true));
      const int eb = group_exponent<T>(m);
      if (row < a.rows && (col & ~31ll) < a.cols) {  // whole groups: zeros behind the last element
        *reinterpret_cast<uint32_t *>(a.codes + row * a.cb + col / 2) = eb < 255 ? codes8(raw[k], eb) : 0u;
        if ((j & 3) == 0) a.scales[row * a.sb + col / GROUP] = (uint8_t)eb;
      }
    }
  }
  __syncthreads();
  const int c = threadIdx.x >> 2, k = threadIdx.x & 3;
  const long long first = r0 + k * 32;
  if (c0 + c >= a.cols || first >= a.rows) return;
  Raw8<T> r[4];
#pragma unroll
  for (int h = 0; h < 4; ++h) {
    T t[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) t[e] = lds[k * BAND + (8 * h + e) * LD + c];
    __builtin_memcpy(&r[h], t, sizeof(t));
  }
  uintx4 codes;
  const int eb = group32(r, codes);
  *reinterpret_cast<uintx4 *>(a.codes_t + (c0 + c) * a.cbt + first / 2) = codes;
  a.scales_t[(c0 + c) * a.sbt + first / GROUP] = (uint8_t)eb;
}

// ---- products ----
// results[r][c] = sum over groups g of 2^(Ea + Eb) sum over a group's elements of a b.  One 16x16x128 instruction takes 16 rows of each operand by 4
// groups: lane l holds group l / 16 of row l % 16, 16 bytes, and its exponent byte.  A group that held no number has the exponent byte 255,
// which the instruction reads as NaN.
using intx8 = __attribute__((ext_vector_type(8))) int;

__device__ inline floatx4 mx_mfma(const uintx4 &a, uint32_t sa, const uintx4 &b, uint32_t sb, floatx4 c) {
  const intx8 x = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0}, y = {(int)b[0], (int)b[1], (int)b[2], (int)b[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, c, 4, 4, 0, (int)sa, 0, (int)sb);  // 4: e2m1; exponents in the low byte
}

// The same in place: left to itself the compiler gives sums new registers where paths meet, and beside 128 of them it has none left.  What it does not see: an
// operand that a vector instruction wrote is read two cycles later at the earliest (these come from LDS), a result 18
// cycles after its instruction by another one than an MFMA that adds to it (settle_results).
__device__ inline void mx_mfma_in_place(floatx4 &c, const uintx4 &a, uint32_t sa, const uintx4 &b, uint32_t sb) {
  asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel_hi:[0,0,0] cbsz:4 blgp:4" : "+v"(c) : "v"(a), "v"(b), "v"(sa), "v"(sb));
}
template <int M, int N>
__device__ inline void settle_results(floatx4 (&c)[M][N]) {
#pragma unroll
  for (int i = 0; i < M * N; ++i) asm volatile("" : "+v"(c[i / N][i % N]));
  asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
#pragma unroll
  for (int i = 0; i < M * N; ++i) asm volatile("" : "+v"(c[i / N][i % N]));
}

struct MxArgs {
  GemmArgs g;  // strides of codes; L = groups, per = groups of a split
  const uint8_t *sa, *sb;
  long long lsa, lsb;
  int K;
};

// the codes of a row's last group, of which n elements count
__device__ inline uintx4 first_codes(uintx4 v, int n) {
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const int k = n - 8 * w;
    v[w] &= k >= 8 ? ~0u : k <= 0 ? 0u : (1u << 4 * k) - 1;
  }
  return v;
}

// 4 bytes per lane from memory to LDS at `to` + 4 * lane
__device__ inline void copy4(const uintx4 &buf, uint32_t voff, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(to), "v"(voff), "s"(buf) : "memory");
}

// A wave's parts of sums; their rows are whole pieces of 8.
template <int MT, int NT>
__device__ inline void write_parts(const GemmArgs &g, int split, long long r0, int c0, int lane, floatx4 (&acc)[MT][NT]) {
  const int i16 = lane & 15, q = lane >> 4;
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const long long row = r0 + 16 * i + i16;
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const int col = c0 + 16 * j + 4 * q;
      if (row < g.R && col < g.part_ld) *reinterpret_cast<floatx4 *>(g.part + (split * g.R + row) * g.part_ld + col) = acc[i][j];
    }
  }
}

// The steps of a tile of 256: a wave's 128 x 64 results leave registers for the fragments of B and four of A.  A row of fragments of A is read two rows
// ahead of its products, B's half a step ahead; the barrier that makes the next step's stage whole stands two rows before the end of a step,
// when all of its own have been read.
template <typename S, typename F>
struct WideSteps {
  static constexpr int MT = S::MT, NT = S::NT;
  const char *lds;
  int oa, ob, ea, eb, at[2];  // this lane's place in a stage: codes of A and B without the chunk, exponents, and the chunks of both halves
  F next;  // behind the barrier that ends step s
  uintx4 fa[4], fb[2][NT];
  uint32_t xa[4], xb[2][NT];
  __device__ inline void read_a(int to, int s, int kk, int i) {
    const char *const from = lds + (s & 1) * S::STAGE;
    fa[to] = *reinterpret_cast<const uintx4 *>(from + oa + i * 2048 + at[kk]);
    xa[to] = *reinterpret_cast<const uint8_t *>(from + ea + i * 16 * 8 + kk * 4);
  }
  __device__ inline void read_b(int s, int kk, int j) {
    const char *const from = lds + (s & 1) * S::STAGE;
    fb[kk][j] = *reinterpret_cast<const uintx4 *>(from + ob + j * 2048 + at[kk]);
    xb[kk][j] = *reinterpret_cast<const uint8_t *>(from + eb + j * 16 * 8 + kk * 4);
  }
  __device__ inline void begin() {  // the first stage is whole
#pragma unroll
    for (int j = 0; j < NT; ++j) read_b(0, 0, j);
    read_a(0, 0, 0, 0), read_a(1, 0, 0, 1);
  }
  template <bool LAST, int KK>
  __device__ inline void half(floatx4 (&acc)[MT][NT], int s) {
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      constexpr int first = KK * MT;
      if (KK == 1 && i == MT - 2 && !LAST) {
        wait_copies<0>();
        wait_lds();
        barrier();
        next(s);
      }
      const int ahead = first + i + 2, to = ahead % 4;
      if (ahead < 2 * MT)
        read_a(to, s, ahead / MT, ahead % MT);
      else if (!LAST)
        read_a(to, s + 1, 0, ahead - 2 * MT);
      if (KK == 0 && i >= MT - NT) read_b(s, 1, i - (MT - NT));
      if (KK == 1 && i >= MT - 2 && !LAST) {
#pragma unroll
        for (int j = 0; j < NT / 2; ++j) read_b(s + 1, 0, (i - (MT - 2)) * (NT / 2) + j);
      }
#pragma unroll
      for (int j = 0; j < NT; ++j) mx_mfma_in_place(acc[i][j], fb[KK][j], xb[KK][j], fa[(first + i) % 4], xa[(first + i) % 4]);
    }
  }
};

// A tile of BLOCK x BLOCK by 2 x ACROSS waves; a step is 8 groups of the sum: 128 bytes of codes and 8 of exponents to a row, copied while the step before
// it is carried out.  A row's chunks of 16 bytes (groups) are exchanged in LDS so that the 16 rows of a fragment's read lie in different banks.
// Sums of at most 16 groups take steps of 4 in three stages of 17 KB: three workgroups to a CU, which hide each other's first copies and epilogues.
// 8192x8192x8192 bf16 276 us, 4 PFLOP/s: copies from L2, reads of LDS and matrix instructions take 1.0, 0.8 and 0.9 us of a step's 2.3 in a tile of 256 and
// overlap in part.  65536x512x2048 106 us, with GELU 125: 3.9 us a tile of 128, of which the results' 32 KB need 1.2 at a fill's 6.9 TB/s;
// its vector instructions, 25 an element with GELU, two of them an exponential and a reciprocal, 3.4.
template <int BLOCK, int ACROSS, int STEP>
struct MxTile {
  static constexpr int WAVES = 2 * ACROSS, THREADS = 64 * WAVES, MT = BLOCK / 32, NT = BLOCK / 16 / ACROSS;
  static constexpr int ROW = STEP * 16, CODES = BLOCK * ROW, SCALES = BLOCK * STEP, STAGE = 2 * (CODES + SCALES), PIECES = CODES / 1024 / WAVES;
  static constexpr int LOADERS = THREADS < SCALES / 2 ? THREADS : SCALES / 2, WORDS = SCALES / 2 / LOADERS;  // of exponents: threads (others bring the same again), and 4 bytes of a row each
  static constexpr int STAGES = STEP == 4 ? 3 : 2, SUMS = STEP == 4 ? MT / 2 : BLOCK == 256 ? MT / 2 : MT;
  static constexpr int PER_SIMD = STEP == 4 ? WAVES * 3 / 4 : BLOCK == 64 || (BLOCK == 128 && ACROSS == 4) ? 4 : 2;  // waves to a SIMD
};
template <int STEP>
__device__ inline int mx_swizzle(int row) { return (row >> 1) & (STEP - 1); }

template <typename T, int BLOCK, int ACROSS, int STEP, bool PARTS>
__global__ __launch_bounds__((MxTile<BLOCK, ACROSS, STEP>::THREADS), (MxTile<BLOCK, ACROSS, STEP>::PER_SIMD)) void mx_gemm_kernel(MxArgs m) {
  using S = MxTile<BLOCK, ACROSS, STEP>;
  constexpr int MT = S::MT, NT = S::NT, PIECES = S::PIECES, WAVES = S::WAVES, STAGES = S::STAGES;
  __shared__ __align__(1024) char lds[STAGES * S::STAGE];
  const GemmArgs &g = m.g;
  const int id = xcd_run(blockIdx.x, gridDim.x);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i16 = lane & 15, q = lane >> 4;
  const int split = PARTS ? id / g.tiles : 0, tile = id - split * g.tiles, tr = tile / g.tiles_c;
  const long long r0 = (long long)tr * BLOCK, l0 = split * g.per, l1 = min(g.L, l0 + g.per);
  const int c0 = (tile - tr * g.tiles_c) * BLOCK;
  const int steps = (int)((l1 - l0 + STEP - 1) / STEP);
  const int rows_left = (int)min(g.R - r0, (long long)BLOCK), cols_left = g.C - c0;
  // what this lane brings: chunks of codes, and words of exponents: half of the waves those of A, the others those of B
  uint32_t av[PIECES], bv[PIECES], sv[S::WORDS];
  const int chunk = (lane & (STEP - 1)) ^ mx_swizzle<STEP>((wave * 64 + lane) / STEP);  // the same for all pieces: they are whole eights of rows apart
#pragma unroll
  for (int p = 0; p < PIECES; ++p) {
    const int row = ((p * WAVES + wave) * 64 + lane) / STEP;
    av[p] = row < rows_left ? row * (uint32_t)g.lda + chunk * 16 : OUTSIDE;
    bv[p] = row < cols_left ? row * (uint32_t)g.ldb + chunk * 16 : OUTSIDE;
  }
  constexpr int LOADERS = S::LOADERS;
  const bool of_b = (wave & (LOADERS / 64 - 1)) >= LOADERS / 128;
#pragma unroll
  for (int w = 0; w < S::WORDS; ++w) {
    const int at = (tid & (LOADERS / 2 - 1)) + w * (LOADERS / 2), row = at / (STEP / 4);
    sv[w] = row < (of_b ? cols_left : rows_left) ? row * (uint32_t)(of_b ? m.lsb : m.lsa) + at % (STEP / 4) * 4 : OUTSIDE;
  }
  const char *const pa = g.a + r0 * g.lda + l0 * 16, *const pb = g.b + c0 * g.ldb + l0 * 16;
  const char *const ps = of_b ? (const char *)m.sb + c0 * m.lsb + l0 : (const char *)m.sa + r0 * m.lsa + l0;
  const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds;
  auto fetch = [&](int s) {
    const uint32_t none = chunk < (int)(l1 - l0) - s * STEP ? 0u : OUTSIDE;  // groups behind the last; an offset with OUTSIDE's bits lies outside
    const uintx4 ba = buffer_of(pa + s * (long long)S::ROW), bb = buffer_of(pb + s * (long long)S::ROW), bs = buffer_of(ps + s * STEP);
    const uint32_t to = base + s % STAGES * S::STAGE;
#pragma unroll
    for (int p = 0; p < PIECES; ++p) copy16(ba, av[p] | none, to + (p * WAVES + wave) * 1024);
#pragma unroll
    for (int p = 0; p < PIECES; ++p) copy16(bb, bv[p] | none, to + S::CODES + (p * WAVES + wave) * 1024);
#pragma unroll
    for (int w = 0; w < S::WORDS; ++w)
      copy4(bs, sv[w], to + 2 * S::CODES + (of_b ? S::SCALES : 0) + (w * (LOADERS / 128) + (wave & (LOADERS / 128 - 1))) * 256);
  };
  const int wm = wave / ACROSS * (16 * MT), wn = wave % ACROSS * (16 * NT);
  floatx4 acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
  const int swz = mx_swizzle<STEP>(i16);  // rows of a wave's fragments are multiples of 16 apart
  auto step = [&](int s) {
    const char *const from = lds + s % STAGES * S::STAGE, *const la = from + (wm + i16) * S::ROW, *const lb = from + S::CODES + (wn + i16) * S::ROW;
    const char *const ea = from + 2 * S::CODES + (wm + i16) * STEP + q, *const eb = from + 2 * S::CODES + S::SCALES + (wn + i16) * STEP + q;
#pragma unroll
    for (int kk = 0; kk < STEP / 4; ++kk) {
      uintx4 fa[MT], fb[NT];
      uint32_t xa[MT], xb[NT];
      const int at = ((kk * 4 + q) ^ swz) << 4;
#pragma unroll
      for (int j = 0; j < NT; ++j) fb[j] = *reinterpret_cast<const uintx4 *>(lb + j * 16 * S::ROW + at), xb[j] = *reinterpret_cast<const uint8_t *>(eb + j * 16 * STEP + kk * 4);
#pragma unroll
      for (int i = 0; i < MT; ++i) fa[i] = *reinterpret_cast<const uintx4 *>(la + i * 16 * S::ROW + at), xa[i] = *reinterpret_cast<const uint8_t *>(ea + i * 16 * STEP + kk * 4);
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) mx_mfma_in_place(acc[i][j], fb[j], xb[j], fa[i], xa[i]);
    }
  };
  // What lies behind a row's last element may be anything: zeros take its place in the last step's stage, where that is not a step's end, too.
  const bool ragged = l1 == g.L && m.K % (STEP * GROUP) != 0;
  auto end_rows = [&] {
    char *const stage = lds + (steps - 1) % STAGES * S::STAGE;
    const int inside = (int)(l1 - l0) - (steps - 1) * STEP, n = m.K % GROUP;  // groups of the step, elements of its last one (0: all)
    using Exponents = std::conditional_t<STEP == 8, unsigned long long, uint32_t>;
    const Exponents keep = inside >= STEP ? ~(Exponents)0 : ((Exponents)1 << 8 * inside) - 1;
    for (int r = tid; r < 2 * BLOCK; r += S::THREADS) *reinterpret_cast<Exponents *>(stage + 2 * S::CODES + r * STEP) &= keep;
    if (n) {
      for (int r = tid; r < BLOCK; r += S::THREADS) {
        uintx4 *const p = reinterpret_cast<uintx4 *>(stage + r * S::ROW + (((inside - 1) ^ mx_swizzle<STEP>(r)) << 4));
        *p = first_codes(*p, n);
      }
    }
    wait_lds();
    barrier();
  };
  fetch(0);
  if (steps > 1) fetch(1);
  auto first = [&] {
    if (steps > 1)
      wait_copies<2 * PIECES + S::WORDS>();
    else
      wait_copies<0>();
    barrier();
  };
  auto next = [&](int s) {  // step s + 1 is whole, s read by all
    if (s + 2 < steps)
      fetch(s + 2);
    else if (ragged)
      end_rows();
  };
  if constexpr (STEP == 4) {
    for (int s = 0; s + 1 < steps; ++s) {
      wait_copies<2 * PIECES + S::WORDS>();  // all but the next step's
      wait_lds();
      barrier();
      if (s + 2 < steps) fetch(s + 2);
      step(s);
    }
    wait_copies<0>();
    wait_lds();
    barrier();
    if (ragged) end_rows();
    step(steps - 1);
  } else if constexpr (BLOCK == 256) {
    first();
    WideSteps<S, decltype(next)> w = {lds, (wm + i16) * 128, S::CODES + (wn + i16) * 128, 2 * S::CODES + (wm + i16) * STEP + q, 2 * S::CODES + S::SCALES + (wn + i16) * STEP + q,
                                      {(q ^ swz) << 4, ((4 + q) ^ swz) << 4}, next};
    if (ragged && steps == 1) end_rows();
    w.begin();
    for (int s = 0; s + 1 < steps; ++s) {
      w.template half<false, 0>(acc, s);
      w.template half<false, 1>(acc, s);
    }
    w.template half<true, 0>(acc, steps - 1);
    w.template half<true, 1>(acc, steps - 1);
  } else {
    first();
    for (int s = 0; s + 1 < steps; ++s) {
      step(s);
      wait_copies<0>();
      wait_lds();
      barrier();  // the next step's stage is whole, this one's read
      if (s + 2 < steps) fetch(s + 2);
    }
    if (ragged) end_rows();
    step(steps - 1);
  }
  settle_results(acc);
  if constexpr (PARTS) {
    write_parts(g, split, r0 + wm, c0 + wn, lane, acc);
  } else {
    wait_lds();
    barrier();
    write_fwd<T, false, S::SUMS>(g, r0 + wm, c0 + wn, lane, acc, reinterpret_cast<floatx4 *>(lds) + wave * S::SUMS * NT * 64);
  }
}

// Few rows: 16 columns and up to 32 rows to a workgroup, whose waves share the sum's axis; fragments come from memory without LDS.  x is quantised on the
// way where it is not held in 4 bits yet (RAW): a lane's fragment is a group, whose 32 elements it reads and codes by itself.  Up to 8 rows
// (HALVES) the instruction's 16 x 16 results hold 8 columns of W's first half of groups by x's, and 8 of the second by the second, so
// that twice as many workgroups share W.  1 row, 2048x2048 bf16 4.1 us: the launch's 2.5, and the time of one chain of reads.
template <typename T, int MT, int NW, bool HALVES, bool RAW>
__global__ __launch_bounds__(64 * NW) void mx_few_rows_kernel(MxArgs m) {
  constexpr int ROWS = HALVES ? 8 : 16 * MT, COLS = HALVES ? 8 : 16;
  __shared__ floatx4 lds[NW * MT * 64];  // [wave][row of 16][4 chunks of 4 columns], chunk c at c ^ (row & 3)
  const GemmArgs &g = m.g;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 15, q = lane >> 4;
  const int c0 = blockIdx.x * COLS, groups = (int)g.L;
  const int all = (groups + 3) / 4, steps = HALVES ? (all + 1) / 2 : all;
  const int own = HALVES ? i & 7 : i, first = HALVES && i >= 8 ? steps * 4 : 0;
  const long long wr = min(c0 + own, g.C - 1);  // rows beyond the last read it again; their results are not used
  const char *const w = g.b + wr * g.ldb;
  const uint8_t *const ws = m.sb + wr * m.lsb;
  floatx4 acc[MT];
#pragma unroll
  for (int k = 0; k < MT; ++k) acc[k] = floatx4{0.f, 0.f, 0.f, 0.f};
  for (int s = wave; s < steps; s += NW) {
    const int group = first + s * 4 + q, n = min(max(m.K - group * GROUP, 0), GROUP);
    uintx4 fw = {0, 0, 0, 0}, fx[MT];
    uint32_t ew = 0, ex[MT];
    if (n > 0) fw = *reinterpret_cast<const uintx4 *>(w + group * 16ll), ew = ws[group];
#pragma unroll
    for (int k = 0; k < MT; ++k) {
      const long long row = min((long long)16 * k + own, g.R - 1);
      fx[k] = uintx4{0, 0, 0, 0}, ex[k] = 0;
      if (n <= 0) continue;
      if constexpr (RAW) {
        const T *const p = (const T *)(g.a + row * g.lda) + (long long)group * GROUP;
        Raw8<T> r[4];
#pragma unroll
        for (int h = 0; h < 4; ++h) r[h] = raw8(p + 8 * h, n - 8 * h);
        ex[k] = group32(r, fx[k]);
      } else {
        fx[k] = first_codes(*reinterpret_cast<const uintx4 *>(g.a + row * g.lda + group * 16ll), n);
        ex[k] = m.sa[row * m.lsa + group];
      }
    }
#pragma unroll
    for (int k = 0; k < MT; ++k) acc[k] = mx_mfma(fw, ew, fx[k], ex[k], acc[k]);
  }
#pragma unroll
  for (int k = 0; k < MT; ++k) lds[(wave * MT * 16 + 16 * k + i) * 4 + (q ^ (i & 3))] = acc[k];
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
    if (r >= g.R || col >= g.C) continue;
    float v[8];
    const floatx4 lo = lds[r * 4 + ((2 * h) ^ (r & 3))], hi = lds[r * 4 + ((2 * h + 1) ^ (r & 3))];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = lo[e], v[e + 4] = hi[e];
    if (HALVES) {  // row r + 8, columns 8 ... 15
      const floatx4 lo2 = lds[(r + 8) * 4 + (2 ^ (r & 3))], hi2 = lds[(r + 8) * 4 + (3 ^ (r & 3))];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += lo2[e], v[e + 4] += hi2[e];
    }
    finish_fwd<T>(g.e, r, col, g.C, v);
  }
}

// ---- plans ----
constexpr int FEW = 32;  // rows
constexpr int STEP = 8;  // groups
struct MxPlan {
  int tile, splits;
  long long per;  // groups of a split
  size_t bytes;   // of the splits' sums
};
// Tiles of 256 or 128 by rounds over the workgroups that run together (one to a CU and two, three where sums are short) and a round's time: steps, then
// what ends a tile, with no other workgroup's steps beside it in a CU that holds one (us, in tiles of 256 and of 128: 8192x8192x8192 bf16 276 and 389,
// 16384x2048x2048 48 and 57, 16384x1500x2048 with GELU 60 and 55, 65536x512x2048 131 and 106, with GELU 167 and 125, fp32 results
// 147 and 215).  Few tiles of 128 become tiles of 64 or parts of sums: towards 512 workgroups, four steps each at least.
MxPlan mx_plan(int dtype, int act, long long M, int N, long long K) {
  MxPlan p = {0, 1, 0, 0};
  if (M <= FEW) return p;
  const long long steps = ((K + GROUP - 1) / GROUP + STEP - 1) / STEP;
  auto tiles = [&](int b) { return ((M + b - 1) / b) * ((N + b - 1) / b); };
  const bool wide = dtype == NF_F32, exps = act != NF_ACT_NONE && act != NF_ACT_RELU;
  const double large = (double)((tiles(256) + 255) / 256) * (2.3 * steps + (wide ? 14 : 12) + (exps ? 4.5 : 0));
  const double medium = std::max(1.0, tiles(128) / 512.0) * (1.5 * steps + (wide ? 8 : 4) + (exps ? 1.4 : 0));
  p.tile = tiles(128) < 256 ? 64 : tiles(128) >= 512 && large < medium ? 256 : 128;
  const long long t = tiles(p.tile);
  const long long splits = std::max<long long>(1, std::min<long long>(512 / t, steps / 4));
  const long long each = (steps + splits - 1) / splits;
  p.splits = p.tile == 256 ? 1 : (int)((steps + each - 1) / each), p.per = p.splits == 1 ? steps * STEP : each * STEP;
  p.bytes = p.splits > 1 ? (size_t)p.splits * M * ((N + 7) / 8 * 8) * 4 : 0;
  return p;
}
inline size_t whole256(size_t n) { return (n + 255) / 256 * 256; }

template <typename T>
hipError_t product_as(const MxCall &c, const void *raw, const MxRows &a, const MxRows &b, const Epilogue &e, void *ws, hipStream_t st) {
  const MxPlan p = mx_plan(c.dtype, c.act, c.M, c.N, c.K);
  MxArgs m = {};
  GemmArgs &g = m.g;
  g.a = raw ? (const char *)raw : (const char *)a.codes, g.b = (const char *)b.codes, g.lda = raw ? (long long)c.K * sizeof(T) : a.cb, g.ldb = b.cb;
  m.sa = a.scales, m.sb = b.scales, m.lsa = a.sb, m.lsb = b.sb, m.K = (int)c.K;
  g.R = c.M, g.C = c.N, g.L = (c.K + GROUP - 1) / GROUP, g.e = e;
  const double flops = 2.0 * c.M * c.N * c.K, ends = sizeof(T) * (1.0 + (e.res != nullptr) + (e.z != nullptr)) * c.M * c.N;
  const double bytes = (raw ? sizeof(T) : 0.53) * c.M * c.K + 0.53 * c.N * c.K;
  if (!p.tile) {
    auto go = [&](auto kernel, int threads, int cols) { hipLaunchKernelGGL(kernel, dim3((c.N + cols - 1) / cols), dim3(threads), 0, st, m); };
    return recorded(st, raw ? "mx_linear_few_rows" : "mx_product_few_rows", flops, bytes + ends, [&] {
      if (c.M <= 8)
        raw ? go(mx_few_rows_kernel<T, 1, 8, true, true>, 512, 8) : go(mx_few_rows_kernel<T, 1, 8, true, false>, 512, 8);
      else if (c.M <= 16)
        raw ? go(mx_few_rows_kernel<T, 1, 8, false, true>, 512, 16) : go(mx_few_rows_kernel<T, 1, 8, false, false>, 512, 16);
      else
        raw ? go(mx_few_rows_kernel<T, 2, 8, false, true>, 512, 16) : go(mx_few_rows_kernel<T, 2, 8, false, false>, 512, 16);
    });
  }
  g.tiles_c = (c.N + p.tile - 1) / p.tile, g.tiles = (int)((c.M + p.tile - 1) / p.tile) * g.tiles_c;
  g.splits = p.splits, g.per = p.per;
  if (p.splits > 1) g.part = (float *)ws, g.part_ld = (c.N + 7) / 8 * 8;
  const hipError_t err = recorded(st, p.tile == 256 ? "mx_product_256x256" : p.tile == 128 ? "mx_product_128x128" : "mx_product_64x64", flops, bytes + (p.splits > 1 ? 4.0 * p.splits * c.M * c.N : ends), [&] {
    const dim3 grid((unsigned)(g.tiles * g.splits));
    auto go = [&](auto tile, auto across, auto step) {
      constexpr int B = decltype(tile)::value, A = decltype(across)::value, G = decltype(step)::value;
      if constexpr (G == 8 && B != 256) {  // tiles of 256 and sums of at most 16 groups have no parts
        if (g.part) {
          hipLaunchKernelGGL((mx_gemm_kernel<T, B, A, 8, true>), grid, dim3((MxTile<B, A, 8>::THREADS)), 0, st, m);
          return;
        }
      }
      hipLaunchKernelGGL((mx_gemm_kernel<T, B, A, G, false>), grid, dim3((MxTile<B, A, G>::THREADS)), 0, st, m);
    };
    using std::integral_constant;
    using I2 = integral_constant<int, 2>;
    using I4 = integral_constant<int, 4>;
    using I8 = integral_constant<int, 8>;
    if (p.tile == 256)
      go(integral_constant<int, 256>(), I4(), I8());
    else if (p.tile == 64)
      go(integral_constant<int, 64>(), I2(), I8());
    else if (sizeof(T) == 2 && g.L <= 2 * STEP)  // fp32 results' epilogue wants more registers than three workgroups leave
      go(integral_constant<int, 128>(), I2(), integral_constant<int, sizeof(T) == 2 ? 4 : 8>());
    else if (g.L >= 8 * STEP)
      go(integral_constant<int, 128>(), I2(), I8());
    else
      go(integral_constant<int, 128>(), I4(), I8());
  });
  if (err != hipSuccess || p.splits == 1) return err;
  const FinishArgs f = finish_args(p.splits, g);
  return recorded(st, "mx_product_finish", 0.0, 4.0 * p.splits * c.M * c.N + ends,
                  [&] { hipLaunchKernelGGL(fwd_finish_kernel<T>, dim3(finish_blocks(f)), dim3(LT), 0, st, f); });
}

template <typename T>
hipError_t quantise_as(const QuantArgs &a, const T *x, hipStream_t st) {
  const double n = (double)a.rows * a.cols;
  return recorded(st, a.codes_t ? a.codes ? "mx_quantise_both" : "mx_quantise_columns" : "mx_quantise_rows", 0.0, n * (sizeof(T) + (a.codes ? 0.53 : 0.0) + (a.codes_t ? 0.53 : 0.0)), [&] {
    const dim3 tiles((unsigned)(a.tiles_c * ((a.rows + TR - 1) / TR)));
    if (!a.codes_t)
      hipLaunchKernelGGL(mx_rows_kernel<T>, dim3((unsigned)((a.rows * a.groups + QT - 1) / QT)), dim3(QT), 0, st, a, x);
    else if (a.codes)
      hipLaunchKernelGGL((mx_columns_kernel<T, true>), tiles, dim3(QT), 0, st, a, x);
    else
      hipLaunchKernelGGL((mx_columns_kernel<T, false>), tiles, dim3(QT), 0, st, a, x);
  });
}

MxRows rows_at(void *codes, void *scales, long long n) {
  MxRows r = {(uint8_t *)codes, (uint8_t *)scales, 0, 0};
  qcache_row_bytes(NF_Q_E2M1, n, &r.cb, &r.sb);
  return r;
}

}  // namespace

bool mx_quantise_fits(long long rows, long long cols, bool by_columns) {
  const double blocks = by_columns ? (double)((rows + TR - 1) / TR) * (double)((cols + TC - 1) / TC) : (double)rows * (double)((cols + GROUP - 1) / GROUP) / QT;
  return blocks < (1 << 24) - 1;  // a launch has less than 2^32 threads
}

size_t mx_product_workspace_bytes(const MxCall &c) { return mx_plan(c.dtype, c.act, c.M, c.N, c.K).bytes; }
size_t mx_linear_workspace_bytes(const MxCall &c) {
  const MxPlan p = mx_plan(c.dtype, c.act, c.M, c.N, c.K);
  if (!p.tile) return 0;
  const MxRows r = rows_at(nullptr, nullptr, c.K);
  return whole256(p.bytes) + whole256((size_t)c.M * r.cb) + (size_t)c.M * r.sb;
}

hipError_t launch_mx_quantise(int dtype, long long rows, long long cols, const void *x, void *codes, void *scales, void *codes_t, void *scales_t, hipStream_t st) {
  const MxRows r = rows_at(codes, scales, cols), t = rows_at(codes_t, scales_t, rows);
  const QuantArgs a = {rows, cols, (cols + TC - 1) / TC, (cols + GROUP - 1) / GROUP, r.codes, r.scales, t.codes, t.scales, r.cb, r.sb, t.cb, t.sb};
  if (dtype == NF_BF16) return quantise_as(a, (const __bf16 *)x, st);
  if (dtype == NF_F16) return quantise_as(a, (const _Float16 *)x, st);
  return quantise_as(a, (const float *)x, st);
}

hipError_t launch_mx_product(const MxCall &c, const void *a, const void *as, const void *b, const void *bs, const float *bias, const void *r, const DropArgs &drop,
                             void *y, void *z, void *ws, hipStream_t st) {
  const Epilogue e = {bias, r, z, y, drop, c.act};
  const MxRows ra = rows_at((void *)a, (void *)as, c.K), rb = rows_at((void *)b, (void *)bs, c.K);
  if (c.dtype == NF_BF16) return product_as<__bf16>(c, nullptr, ra, rb, e, ws, st);
  if (c.dtype == NF_F16) return product_as<_Float16>(c, nullptr, ra, rb, e, ws, st);
  return product_as<float>(c, nullptr, ra, rb, e, ws, st);
}

// The workspace holds the splits' sums, then x's codes and exponents.
hipError_t launch_mx_linear(const MxCall &c, const void *x, const void *W, const void *Ws, const float *bias, const void *r, const DropArgs &drop, void *y, void *z,
                            void *ws, hipStream_t st) {
  const MxPlan p = mx_plan(c.dtype, c.act, c.M, c.N, c.K);
  if (p.tile) {
    const MxRows sizes = rows_at(nullptr, nullptr, c.K);
    char *const codes = (char *)ws + whole256(p.bytes), *const scales = codes + whole256((size_t)c.M * sizes.cb);
    const hipError_t e = launch_mx_quantise(c.dtype, c.M, c.K, x, codes, scales, nullptr, nullptr, st);
    return e != hipSuccess ? e : launch_mx_product(c, codes, scales, W, Ws, bias, r, drop, y, z, ws, st);
  }
  const Epilogue e = {bias, r, z, y, drop, c.act};
  const MxRows none = {}, rb = rows_at((void *)W, (void *)Ws, c.K);
  if (c.dtype == NF_BF16) return product_as<__bf16>(c, x, none, rb, e, ws, st);
  if (c.dtype == NF_F16) return product_as<_Float16>(c, x, none, rb, e, ws, st);
  return product_as<float>(c, x, none, rb, e, ws, st);
}

}  // namespace nf
