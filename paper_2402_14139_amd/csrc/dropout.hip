// Dropout over row-major matrices, forward with a residual and backward.
#include <algorithm>

#include "pw_math.h"

namespace nf {
namespace {

constexpr int DT = 256;

// y = r + D(x), 8 elements of a row to a Philox call; a thread takes U of them, whose reads are in flight together.  HBM-bound:
// sizeof(T) * 3 (with r) or 2 bytes an element.  y may be x or r.  65536x512 bf16 36.7 us, 5.5 TB/s without r; 22275x100 fp32, which the
// launch and one round of reads bound, 5.8 us.
template <typename T, bool WHOLE, int U>
__global__ __launch_bounds__(DT) void dropout_kernel(DropArgs d, long long total, long long cols, long long groups, FastDiv div_groups,
                                                     const T *x, const T *r, T *y) {
  for (long long i0 = (long long)blockIdx.x * DT * U + threadIdx.x; i0 < total; i0 += (long long)gridDim.x * DT * U) {
    Raw8<T> xv[U], rv[U];
    long long at[U];
    int n[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long long i = i0 + u * DT;
      at[u] = i * 8, n[u] = i < total ? 8 : 0;
      if constexpr (!WHOLE) {  // rows that end inside a group
        const long long row = total <= 0x7FFFFFFFll ? (long long)div_groups.div((uint32_t)i) : i / groups, g = i - row * groups;
        at[u] = row * cols + g * 8;
        if (n[u]) n[u] = (int)min(8ll, cols - g * 8);
      }
      if (n[u]) {
        xv[u] = raw8(x + at[u], n[u]);
        if (r) rv[u] = raw8(r + at[u], n[u]);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (!n[u]) continue;
      float v[8];
      unpack8(xv[u], v);
      drop8(d, (unsigned long long)(i0 + u * DT), v);
      if (r) {
        float s[8];
        unpack8(rv[u], s);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = fmaf(v[e], d.scale, s[e]);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= d.scale;
      }
      store8(y + at[u], v, n[u]);
    }
  }
}

template <typename T, int U>
hipError_t launch(const DropArgs &d, long long rows, long long cols, const void *x, const void *r, void *y,
                  hipStream_t st) {
  const long long groups = (cols + 7) / 8, total = rows * groups;
  const unsigned nb = (unsigned)std::min<long long>((total + DT * U - 1) / (DT * U), 1 << 22);
  const FastDiv div((uint32_t)groups);
  if (cols % 8 == 0)
    hipLaunchKernelGGL((dropout_kernel<T, true, U>), dim3(nb), dim3(DT), 0, st, d, total, cols, groups, div, (const T *)x, (const T *)r, (T *)y);
  else
    hipLaunchKernelGGL((dropout_kernel<T, false, U>), dim3(nb), dim3(DT), 0, st, d, total, cols, groups, div, (const T *)x, (const T *)r, (T *)y);
  return hipGetLastError();
}
// several groups to a thread where there are enough for 4 workgroups to a CU all the same
template <typename T>
hipError_t launch_as(const DropArgs &d, long long rows, long long cols, const void *x, const void *r, void *y, hipStream_t st) {
  return rows * ((cols + 7) / 8) >= 1024 * DT * 2 ? launch<T, 2>(d, rows, cols, x, r, y, st) : launch<T, 1>(d, rows, cols, x, r, y, st);
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
  if (dtype == NF_BF16) return launch_as<__bf16>(d, rows, cols, x, r, y, st);
  if (dtype == NF_F16) return launch_as<_Float16>(d, rows, cols, x, r, y, st);
  return launch_as<float>(d, rows, cols, x, r, y, st);
}

}  // namespace nf
