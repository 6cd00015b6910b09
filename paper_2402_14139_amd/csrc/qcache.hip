// The activation cache in 8 or 4 bits an element: rows quantised as they are written, gathered and read back.
#include <type_traits>

#include "pw_math.h"

namespace nf {
namespace {

constexpr int QT = 256;
constexpr int GROUP = 32;  // elements that share an exponent

// Largest code: its mantissa (1 <= m < 2) and exponent.
template <int F>
struct Format;
template <>
struct Format<NF_Q_INT8> {
  static constexpr float top = 127.f / 64.f;
  static constexpr int k = 6, bits = 8;
};
template <>
struct Format<NF_Q_E4M3> {
  static constexpr float top = 1.75f;
  static constexpr int k = 8, bits = 8;
};
template <>
struct Format<NF_Q_E2M1> {
  static constexpr float top = 1.5f;
  static constexpr int k = 2, bits = 4;
};

// 8 elements to codes: 8 bytes, or 4 of e2m1.  The elements lie within the codes' range after the division by 2^E, an exact
// step down to the codes' own precision.  The conversions round to nearest, ties to even.
template <int F>
__device__ inline void encode8(const float v[8], int E, uint32_t out[2]) {
  float s[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) s[e] = ldexpf(v[e], -E);
  if constexpr (F == NF_Q_INT8) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint32_t w = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) w |= ((uint32_t)(int)rintf(s[4 * h + e]) & 0xFFu) << (8 * e);
      out[h] = w;
    }
  } else if constexpr (F == NF_Q_E4M3) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      int w = __builtin_amdgcn_cvt_pk_fp8_f32(s[4 * h], s[4 * h + 1], 0, false);
      out[h] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(s[4 * h + 2], s[4 * h + 3], w, true);
    }
  } else {
    uint32_t w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, s[0], s[1], 1.f, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, s[2], s[3], 1.f, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, s[4], s[5], 1.f, 2);
    out[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, s[6], s[7], 1.f, 3);
    out[1] = 0;
  }
}

template <int F>
__device__ inline void decode8(const uint32_t in[2], float v[8]) {
  if constexpr (F == NF_Q_INT8) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (float)(int)(int8_t)(in[e >> 2] >> (8 * (e & 3)));
  } else {
    using floatx2 = __attribute__((ext_vector_type(2))) float;
    floatx2 p[4];
    if constexpr (F == NF_Q_E4M3) {
      p[0] = __builtin_amdgcn_cvt_pk_f32_fp8((int)in[0], false), p[1] = __builtin_amdgcn_cvt_pk_f32_fp8((int)in[0], true);
      p[2] = __builtin_amdgcn_cvt_pk_f32_fp8((int)in[1], false), p[3] = __builtin_amdgcn_cvt_pk_f32_fp8((int)in[1], true);
    } else {
      p[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(in[0], 1.f, 0), p[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(in[0], 1.f, 1);
      p[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(in[0], 1.f, 2), p[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(in[0], 1.f, 3);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = p[e >> 1][e & 1];
  }
}

// E + 127, or 255 where a group holds no number.  frexp's exponent is one above that of a mantissa 1 <= m < 2.
template <int F>
__device__ inline int exponent_byte(float amax) {
  if (!(amax < INFINITY)) return 255;
  if (amax == 0.f) return 0;
  int e;
  const float m = 2.f * frexpf(amax, &e);
  e = e - 1 - Format<F>::k + (m > Format<F>::top ? 1 : 0);
  return max(e, -127) + 127;
}

struct Rows {
  uint8_t *codes, *scales;
  int32_t *labels;
  long long capacity, n, first, code_bytes, scale_bytes;
  int per_row;  // pieces of 8 elements, whole groups: a multiple of 4
  int rows_per;  // rows a workgroup takes at once
};

// A thread takes U pieces of 8 elements, whose reads are in flight together; the 4 neighbours of a group find its largest
// magnitude together.  HBM-bound: sizeof(T) + 1 + 1/32 bytes an element (e2m1: half a byte less).  512 fp32 rows of 16384 to int8 9.5 us,
// 4.4 TB/s with the launch.
template <typename T, int F, int U>
__global__ __launch_bounds__(QT) void qcache_write_kernel(Rows q, int B, const T *__restrict__ x,
                                                          const int32_t *__restrict__ labels) {
  const int per = q.rows_per > 1 ? q.per_row : QT;  // threads of a row
  const int r = threadIdx.x / per, j0 = threadIdx.x - r * per + (q.rows_per == 1 ? blockIdx.x * QT * U : 0);
  const long long row = (long long)blockIdx.y * q.rows_per + r;
  const bool live = r < q.rows_per && row < B;  // threads beyond take part in the exchanges
  if (live && labels && j0 == 0) q.labels[q.first + row] = labels[row];
  const long long at = q.first + row;
  Raw8<T> raw[U] = {};
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int j = j0 + u * QT;
    if (live && 8ll * j < q.n) raw[u] = raw8(x + row * q.n + 8ll * j, (int)min(q.n - 8ll * j, 8ll));
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int j = j0 + u * QT;
    float v[8];
    unpack8(raw[u], v);
    float top = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) top = fabsf(v[e]) <= INFINITY ? fmaxf(top, fabsf(v[e])) : INFINITY;  // a NaN counts as infinite
    top = fmaxf(top, __shfl_xor(top, 1));
    top = fmaxf(top, __shfl_xor(top, 2));
    if (!live || 8ll * j >= q.n) continue;
    const int eb = exponent_byte<F>(top);
    uint32_t w[2] = {0, 0};
    if (eb < 255) encode8<F>(v, eb - 127, w);
    if ((threadIdx.x & 3) == 0) q.scales[at * q.scale_bytes + (j >> 2)] = (uint8_t)eb;
    if constexpr (Format<F>::bits == 8)
      *reinterpret_cast<uint2 *>(q.codes + at * q.code_bytes + 8ll * j) = make_uint2(w[0], w[1]);
    else
      *reinterpret_cast<uint32_t *>(q.codes + at * q.code_bytes + 4ll * j) = w[0];
  }
}

// The same bytes the other way: those rows 10.8 us; 512 rows of 65536 from e2m1 to bf16 17.4 us, 4.9 TB/s.
template <typename T, int F, int U>
__global__ __launch_bounds__(QT) void qcache_read_kernel(Rows q, const long long *__restrict__ idx, int B,
                                                         T *__restrict__ x, int32_t *__restrict__ labels) {
  const int per = q.rows_per > 1 ? q.per_row : QT;
  const int r = threadIdx.x / per, j0 = threadIdx.x - r * per + (q.rows_per == 1 ? blockIdx.x * QT * U : 0);
  const long long row = (long long)blockIdx.y * q.rows_per + r;
  if (r >= q.rows_per || row >= B) return;
  long long src = idx ? idx[row] : q.first + row;
  if (idx) src = src < 0 ? 0 : (src >= q.capacity ? q.capacity - 1 : src);
  if (labels && j0 == 0) labels[row] = q.labels[src];
  const uint8_t *const codes = q.codes + src * q.code_bytes, *const scales = q.scales + src * q.scale_bytes;
  uint32_t w[U][2];
  int eb[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int j = j0 + u * QT;
    if (8ll * j >= q.n) continue;
    w[u][1] = 0;
    if constexpr (Format<F>::bits == 8) {
      const uint2 t = *reinterpret_cast<const uint2 *>(codes + 8ll * j);
      w[u][0] = t.x, w[u][1] = t.y;
    } else {
      w[u][0] = *reinterpret_cast<const uint32_t *>(codes + 4ll * j);
    }
    eb[u] = scales[j >> 2];
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int j = j0 + u * QT;
    if (8ll * j >= q.n) continue;
    float v[8];
    decode8<F>(w[u], v);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = eb[u] == 255 ? NAN : ldexpf(v[e], eb[u] - 127);
    store8(x + row * q.n + 8ll * j, v, (int)min(q.n - 8ll * j, 8ll));
  }
}

Rows rows_of(const QcacheRows &q) {
  Rows r = {q.codes, q.scales, q.labels, q.capacity, q.n, q.first, q.code_bytes, q.scale_bytes, 0, 1};
  r.per_row = (int)((q.n + GROUP - 1) / GROUP * (GROUP / 8));
  if (r.per_row <= QT / 2) r.rows_per = QT / r.per_row;  // short rows share a workgroup
  return r;
}
// pieces to a thread: several where a row has work for several workgroups all the same
constexpr int MANY = 4;
inline bool many(const Rows &r) { return r.per_row >= 2 * QT * MANY; }
dim3 grid_of(const Rows &r, int B) {
  const int block = QT * (many(r) ? MANY : 1);
  return dim3(r.rows_per > 1 ? 1 : (r.per_row + block - 1) / block, (B + r.rows_per - 1) / r.rows_per);
}

template <typename T, int F>
hipError_t write_as(const QcacheRows &q, int B, const void *x, const int32_t *labels, hipStream_t st) {
  const Rows r = rows_of(q);
  if (many(r))
    hipLaunchKernelGGL((qcache_write_kernel<T, F, MANY>), grid_of(r, B), dim3(QT), 0, st, r, B, (const T *)x, labels);
  else
    hipLaunchKernelGGL((qcache_write_kernel<T, F, 1>), grid_of(r, B), dim3(QT), 0, st, r, B, (const T *)x, labels);
  return hipGetLastError();
}
template <typename T, int F>
hipError_t read_as(const QcacheRows &q, const long long *idx, int B, void *x, int32_t *labels, hipStream_t st) {
  const Rows r = rows_of(q);
  if (many(r))
    hipLaunchKernelGGL((qcache_read_kernel<T, F, MANY>), grid_of(r, B), dim3(QT), 0, st, r, idx, B, (T *)x, labels);
  else
    hipLaunchKernelGGL((qcache_read_kernel<T, F, 1>), grid_of(r, B), dim3(QT), 0, st, r, idx, B, (T *)x, labels);
  return hipGetLastError();
}

// run(type, format)
template <typename T, typename R>
hipError_t by_format(int format, R run) {
  if (format == NF_Q_INT8) return run((T)0.f, std::integral_constant<int, NF_Q_INT8>());
  if (format == NF_Q_E4M3) return run((T)0.f, std::integral_constant<int, NF_Q_E4M3>());
  return run((T)0.f, std::integral_constant<int, NF_Q_E2M1>());
}
template <typename R>
hipError_t by_type(int format, int dtype, R run) {
  if (dtype == NF_BF16) return by_format<__bf16>(format, run);
  if (dtype == NF_F16) return by_format<_Float16>(format, run);
  return by_format<float>(format, run);
}

}  // namespace

void qcache_row_bytes(int format, long long n, long long *code_bytes, long long *scale_bytes) {
  const long long code = format == NF_Q_E2M1 ? (n + 1) / 2 : n;
  *code_bytes = (code + 15) / 16 * 16;
  *scale_bytes = ((n + GROUP - 1) / GROUP + 15) / 16 * 16;
}

hipError_t launch_qcache_write(int format, int dtype, const QcacheRows &q, int B, const void *x, const int32_t *labels,
                               hipStream_t st) {
  return by_type(format, dtype, [&](auto t, auto f) { return write_as<decltype(t), decltype(f)::value>(q, B, x, labels, st); });
}
hipError_t launch_qcache_read(int format, int dtype, const QcacheRows &q, const long long *idx, int B, void *x,
                              int32_t *labels, hipStream_t st) {
  return by_type(format, dtype, [&](auto t, auto f) { return read_as<decltype(t), decltype(f)::value>(q, idx, B, x, labels, st); });
}

}  // namespace nf
