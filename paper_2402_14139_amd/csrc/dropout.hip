// Dropout over row-major matrices, forward with a residual and backward.
#include "pw_math.h"

namespace nf {
namespace {

constexpr int DT = 256;

// y = r + D(x), 8 elements of a row per thread: one Philox call each.  HBM-bound: sizeof(T) * 3 (with r) or 2 bytes an
// element.
template <typename T, bool WHOLE>
__global__ __launch_bounds__(DT) void dropout_kernel(DropArgs d, long long total, long long cols, long long groups,
                                                     const T *x, const T *r, T *y) {
  const long long i = (long long)blockIdx.x * DT + threadIdx.x;
  if (i >= total) return;
  long long at = i * 8;
  int n = 8;
  if constexpr (!WHOLE) {  // rows that end inside a group
    const long long row = i / groups, g = i - row * groups;
    at = row * cols + g * 8, n = (int)min(8ll, cols - g * 8);
  }
  float v[8], s[8];
  load8(x + at, v, n);
  if (r) load8(r + at, s, n);
  drop8(d, (unsigned long long)i, v);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = r ? fmaf(v[e], d.scale, s[e]) : v[e] * d.scale;
  store8(y + at, v, n);
}

template <typename T>
hipError_t launch(const DropArgs &d, long long rows, long long cols, const void *x, const void *r, void *y,
                  hipStream_t st) {
  const long long groups = (cols + 7) / 8, total = rows * groups;
  const unsigned nb = (unsigned)((total + DT - 1) / DT);
  if (cols % 8 == 0)
    hipLaunchKernelGGL((dropout_kernel<T, true>), dim3(nb), dim3(DT), 0, st, d, total, cols, groups, (const T *)x, (const T *)r, (T *)y);
  else
    hipLaunchKernelGGL((dropout_kernel<T, false>), dim3(nb), dim3(DT), 0, st, d, total, cols, groups, (const T *)x, (const T *)r, (T *)y);
  return hipGetLastError();
}

}  // namespace

DropArgs drop_args(const nf_dropout_desc *d) {
  DropArgs a = {0, 1.f, 0, 0, 0, 0};
  if (!d) return a;
  a.T = (uint32_t)__builtin_rint(65536.0 * d->p);
  a.scale = (float)(65536.0 / (65536.0 - a.T));
  a.k0 = (uint32_t)d->seed, a.k1 = (uint32_t)(d->seed >> 32);
  a.s0 = (uint32_t)d->step, a.s1 = (uint32_t)(d->step >> 32);
  return a;
}

hipError_t launch_dropout(const DropArgs &d, int dtype, long long rows, long long cols, const void *x, const void *r,
                          void *y, hipStream_t st) {
  if (dtype == NF_BF16) return launch<__bf16>(d, rows, cols, x, r, y, st);
  if (dtype == NF_F16) return launch<_Float16>(d, rows, cols, x, r, y, st);
  return launch<float>(d, rows, cols, x, r, y, st);
}

}  // namespace nf
