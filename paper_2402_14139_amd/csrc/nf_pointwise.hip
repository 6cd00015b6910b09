// Entry points of the pointwise layers' operators and of the quantised cache (include/nf.h): argument checks, then the
// launches.  Nothing is enqueued before every check has passed.
#include <algorithm>
#include <cmath>

#include "nf_enqueue.h"
#include "pw_math.h"

namespace nf {
namespace {

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
template <typename... P>
bool all_aligned16(P... p) {
  return (aligned16(p) && ...);
}
inline bool dtype_ok(int32_t t) { return t == NF_F32 || t == NF_BF16 || t == NF_F16; }
inline bool act_ok(int32_t a) { return a >= NF_ACT_NONE && a <= NF_ACT_GELU; }
inline double size_of(int32_t t) { return t == NF_F32 ? 4.0 : 2.0; }

int32_t check_drop(const nf_dropout_desc *d) {
  if (!(d->p >= 0.0) || !(std::rint(65536.0 * d->p) < 65536.0)) return NF_ERR_BAD_DESC;
  return NF_OK;
}

int32_t check_dropout(const nf_dropout_desc *d, int32_t dtype, int64_t rows, int64_t cols, const void *x, const void *y) {
  if (!d || !x || !y) return NF_ERR_NULL;
  if (!dtype_ok(dtype) || rows <= 0 || cols <= 0) return NF_ERR_BAD_DESC;
  if (cols >= (1ll << 31) - 8 || rows > (1ll << 62) / cols) return NF_ERR_UNSUPPORTED;
  return check_drop(d);
}

int32_t check_linear(const nf_linear_desc *d, int64_t M, LinearCall *c) {
  if (!d) return NF_ERR_NULL;
  if (!dtype_ok(d->dtype) || !act_ok(d->act) || d->K <= 0 || d->N <= 0 || M <= 0) return NF_ERR_BAD_DESC;
  if (d->K > (1 << 20) || d->N > (1 << 20) || M >= (1ll << 31) - 512) return NF_ERR_UNSUPPORTED;
  // grids count tiles of 64 x 64 at the least in 31 bits
  const int64_t big = std::max<int64_t>(M, std::max(d->K, d->N)), mid = std::max(d->K, d->N);
  if (((big + 63) / 64) * ((mid + 63) / 64) >= (1ll << 31) / 256) return NF_ERR_UNSUPPORTED;
  *c = LinearCall{d->dtype, d->act, M, d->K, d->N};
  return NF_OK;
}

int32_t check_ws(const void *ws, size_t have, size_t need) {
  if (need == 0) return NF_OK;
  if (!ws || (reinterpret_cast<uintptr_t>(ws) & 255u) || have < need) return NF_ERR_WORKSPACE;
  return NF_OK;
}

int32_t check_groupnorm(const nf_groupnorm_desc *d, int32_t B, GnShape *s) {
  if (!d) return NF_ERR_NULL;
  if (!dtype_ok(d->dtype) || !act_ok(d->act) || d->C <= 0 || d->G <= 0 || d->HW <= 0 || B <= 0 || d->C % d->G || !(d->eps >= 0.f))
    return NF_ERR_BAD_DESC;
  if (B > 65535 || d->C > (1 << 16) || d->C / d->G > 2048 || d->HW >= (1 << 24)) return NF_ERR_UNSUPPORTED;
  *s = GnShape{d->dtype, B, d->HW, d->C, d->G, d->act, d->eps};
  return NF_OK;
}

int32_t check_layernorm(const nf_layernorm_desc *d, int64_t M, LnShape *s) {
  if (!d) return NF_ERR_NULL;
  if (!dtype_ok(d->dtype) || d->C <= 0 || M <= 0 || !(d->eps >= 0.f)) return NF_ERR_BAD_DESC;
  if (d->C > (1 << 16) || M >= (1ll << 40)) return NF_ERR_UNSUPPORTED;
  *s = LnShape{d->dtype, M, d->C, d->eps};
  return NF_OK;
}

int32_t check_qcache(int32_t format, int32_t dtype, const void *codes, const void *scales, const void *clab,
                     int64_t capacity, int64_t n, int64_t first, int32_t B, const void *buf, const void *lab, bool by_index,
                     QcacheRows *q) {
  if (!codes || !scales || !buf) return NF_ERR_NULL;
  if ((clab == nullptr) != (lab == nullptr)) return NF_ERR_NULL;
  if (format < NF_Q_INT8 || format > NF_Q_E2M1 || !dtype_ok(dtype) || capacity <= 0 || n <= 0 || B <= 0 || B > 65535)
    return NF_ERR_BAD_DESC;
  if (n > (1ll << 33)) return NF_ERR_UNSUPPORTED;
  if (!all_aligned16(codes, scales, buf)) return NF_ERR_BAD_DESC;
  if (!by_index && (first < 0 || first > capacity - B)) return NF_ERR_CACHE_RANGE;
  q->codes = (uint8_t *)codes, q->scales = (uint8_t *)scales, q->labels = (int32_t *)clab;
  q->capacity = capacity, q->n = n, q->first = by_index ? 0 : first;
  qcache_row_bytes(format, n, &q->code_bytes, &q->scale_bytes);
  return NF_OK;
}

int32_t check_mx(const nf_linear_desc *d, int64_t M, MxCall *c) {
  if (!d) return NF_ERR_NULL;
  if (!dtype_ok(d->dtype) || !act_ok(d->act) || d->K <= 0 || d->N <= 0 || M <= 0) return NF_ERR_BAD_DESC;
  if (d->K > (1 << 24) || d->N > (1 << 20) || M >= (1ll << 31) - 512) return NF_ERR_UNSUPPORTED;
  if (((M + 63) / 64) * ((d->N + 63) / 64) >= (1ll << 31) / 256) return NF_ERR_UNSUPPORTED;
  *c = MxCall{d->dtype, d->act, M, d->N, d->K};
  return NF_OK;
}

}  // namespace
}  // namespace nf

using namespace nf;

extern "C" {

int32_t nf_dropout_fwd(const nf_dropout_desc *drop, int32_t dtype, int64_t rows, int64_t cols, const void *x,
                       const void *r, void *y, void *stream) {
  const int32_t rc = check_dropout(drop, dtype, rows, cols, x, y);
  if (rc) return rc;
  if (!all_aligned16(x, r, y)) return NF_ERR_BAD_DESC;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  NF_RUN(st, "dropout_fwd", 0.0, size_of(dtype) * (r ? 3.0 : 2.0) * rows * cols,
         launch_dropout(drop_args(drop), dtype, rows, cols, x, r, y, st));
  return NF_OK;
}

int32_t nf_dropout_bwd(const nf_dropout_desc *drop, int32_t dtype, int64_t rows, int64_t cols, const void *dy,
                       void *dx, void *stream) {
  const int32_t rc = check_dropout(drop, dtype, rows, cols, dy, dx);
  if (rc) return rc;
  if (!all_aligned16(dy, dx)) return NF_ERR_BAD_DESC;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  NF_RUN(st, "dropout_bwd", 0.0, size_of(dtype) * 2.0 * rows * cols,
         launch_dropout(drop_args(drop), dtype, rows, cols, dy, nullptr, dx, st));
  return NF_OK;
}

int32_t nf_linear_workspace_bytes(const nf_linear_desc *d, int64_t M, size_t *out) {
  LinearCall c;
  const int32_t rc = check_linear(d, M, &c);
  if (rc) return rc;
  if (!out) return NF_ERR_NULL;
  *out = linear_workspace_bytes(c);
  return NF_OK;
}

int32_t nf_linear_fwd_workspace_bytes(const nf_linear_desc *d, int64_t M, size_t *out) {
  LinearCall c;
  const int32_t rc = check_linear(d, M, &c);
  if (rc) return rc;
  if (!out) return NF_ERR_NULL;
  *out = linear_fwd_workspace_bytes(c);
  return NF_OK;
}

int32_t nf_linear_fwd(const nf_linear_desc *d, int64_t M, const void *x, const void *W, const float *b, const void *r,
                      const nf_dropout_desc *drop, void *y, void *z, void *ws, size_t ws_bytes, void *stream) {
  LinearCall c;
  int32_t rc = check_linear(d, M, &c);
  if (rc) return rc;
  if (!x || !W || !y) return NF_ERR_NULL;
  if (drop && (rc = check_drop(drop))) return rc;
  if (!all_aligned16(x, W, b, r, y, z)) return NF_ERR_BAD_DESC;
  if ((rc = check_ws(ws, ws_bytes, linear_fwd_workspace_bytes(c)))) return rc;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  NF_HIP(launch_linear_fwd(c, x, W, b, r, drop_args(drop), y, z, ws, st));
  return NF_OK;
}

int32_t nf_linear_bwd_epilogue(const nf_linear_desc *d, int64_t M, const void *dy, const void *z,
                               const nf_dropout_desc *drop, void *dz, float *db, void *ws, size_t ws_bytes,
                               void *stream) {
  LinearCall c;
  int32_t rc = check_linear(d, M, &c);
  if (rc) return rc;
  if (!dy || !dz || (c.act != NF_ACT_NONE && !z)) return NF_ERR_NULL;
  if (drop && (rc = check_drop(drop))) return rc;
  if (!all_aligned16(dy, z, dz, db)) return NF_ERR_BAD_DESC;
  if ((rc = check_ws(ws, ws_bytes, linear_workspace_bytes(c)))) return rc;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  NF_HIP(launch_linear_epilogue(c, dy, z, drop_args(drop), dz, db, ws, st));
  return NF_OK;
}

int32_t nf_linear_bwd(const nf_linear_desc *d, int64_t M, const void *dz, const void *x, const void *W, void *dx,
                      float *dW, void *ws, size_t ws_bytes, void *stream) {
  LinearCall c;
  int32_t rc = check_linear(d, M, &c);
  if (rc) return rc;
  if (!dz || (!dx && !dW) || (dx && !W) || (dW && !x)) return NF_ERR_NULL;
  if (!all_aligned16(dz, x, W, dx, dW)) return NF_ERR_BAD_DESC;
  if ((rc = check_ws(ws, ws_bytes, linear_workspace_bytes(c)))) return rc;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  NF_HIP(launch_linear_bwd(c, dz, x, W, dx, dW, ws, st));
  return NF_OK;
}

int32_t nf_groupnorm_workspace_bytes(const nf_groupnorm_desc *d, int32_t B, size_t *out) {
  GnShape s;
  const int32_t rc = check_groupnorm(d, B, &s);
  if (rc) return rc;
  if (!out) return NF_ERR_NULL;
  *out = gn_workspace_bytes(s);
  return NF_OK;
}

int32_t nf_groupnorm_fwd_workspace_bytes(const nf_groupnorm_desc *d, int32_t B, size_t *out) {
  GnShape s;
  const int32_t rc = check_groupnorm(d, B, &s);
  if (rc) return rc;
  if (!out) return NF_ERR_NULL;
  *out = gn_fwd_workspace_bytes(s);
  return NF_OK;
}

int32_t nf_groupnorm_fwd(const nf_groupnorm_desc *d, int32_t B, const void *x, const float *gamma, const float *beta,
                         void *y, float *mean, float *rstd, void *ws, size_t ws_bytes, void *stream) {
  GnShape s;
  int32_t rc = check_groupnorm(d, B, &s);
  if (rc) return rc;
  if (!x || !gamma || !beta || !y || !mean || !rstd) return NF_ERR_NULL;
  if (!all_aligned16(x, gamma, beta, y, mean, rstd)) return NF_ERR_BAD_DESC;
  if ((rc = check_ws(ws, ws_bytes, gn_fwd_workspace_bytes(s)))) return rc;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  NF_HIP(launch_gn_fwd(s, x, gamma, beta, y, mean, rstd, ws, st));
  return NF_OK;
}

int32_t nf_groupnorm_bwd(const nf_groupnorm_desc *d, int32_t B, const void *dy, const void *x, const float *gamma,
                         const float *beta, const float *mean, const float *rstd, void *dx, float *dgamma,
                         float *dbeta, void *ws, size_t ws_bytes, void *stream) {
  GnShape s;
  int32_t rc = check_groupnorm(d, B, &s);
  if (rc) return rc;
  if (!dy || !x || !gamma || !beta || !mean || !rstd || !dx || !dgamma || !dbeta) return NF_ERR_NULL;
  if (!all_aligned16(dy, x, gamma, beta, mean, rstd, dx, dgamma, dbeta)) return NF_ERR_BAD_DESC;
  if ((rc = check_ws(ws, ws_bytes, gn_workspace_bytes(s)))) return rc;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  NF_HIP(launch_gn_bwd(s, dy, x, gamma, beta, mean, rstd, dx, dgamma, dbeta, ws, st));
  return NF_OK;
}

int32_t nf_layernorm_workspace_bytes(const nf_layernorm_desc *d, int64_t M, size_t *out) {
  LnShape s;
  const int32_t rc = check_layernorm(d, M, &s);
  if (rc) return rc;
  if (!out) return NF_ERR_NULL;
  *out = ln_workspace_bytes(s);
  return NF_OK;
}

int32_t nf_layernorm_fwd(const nf_layernorm_desc *d, int64_t M, const void *x, const float *gamma, const float *beta,
                         void *y, float *mean, float *rstd, void *stream) {
  LnShape s;
  const int32_t rc = check_layernorm(d, M, &s);
  if (rc) return rc;
  if (!x || !y || (mean == nullptr) != (rstd == nullptr)) return NF_ERR_NULL;
  if (!all_aligned16(x, gamma, beta, y, mean, rstd)) return NF_ERR_BAD_DESC;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  NF_HIP(launch_ln_fwd(s, x, gamma, beta, y, mean, rstd, st));
  return NF_OK;
}

int32_t nf_layernorm_bwd(const nf_layernorm_desc *d, int64_t M, const void *dy, const void *x, const float *gamma,
                         const float *mean, const float *rstd, const void *dr, void *dx, float *dgamma, float *dbeta,
                         void *ws, size_t ws_bytes, void *stream) {
  LnShape s;
  int32_t rc = check_layernorm(d, M, &s);
  if (rc) return rc;
  if (!dy || !x || !mean || !rstd || (!dx && !dgamma && !dbeta)) return NF_ERR_NULL;
  if (!all_aligned16(dy, x, gamma, mean, rstd, dr, dx, dgamma, dbeta)) return NF_ERR_BAD_DESC;
  if ((dgamma || dbeta) && (rc = check_ws(ws, ws_bytes, ln_workspace_bytes(s)))) return rc;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  NF_HIP(launch_ln_bwd(s, dy, x, gamma, mean, rstd, dr, dx, dgamma, dbeta, ws, st));
  return NF_OK;
}

int32_t nf_qcache_row_bytes(int32_t format, int64_t n, size_t *code_bytes, size_t *scale_bytes) {
  if (!code_bytes || !scale_bytes) return NF_ERR_NULL;
  if (format < NF_Q_INT8 || format > NF_Q_E2M1 || n <= 0) return NF_ERR_BAD_DESC;
  if (n > (1ll << 33)) return NF_ERR_UNSUPPORTED;
  long long c, s;
  qcache_row_bytes(format, n, &c, &s);
  *code_bytes = (size_t)c, *scale_bytes = (size_t)s;
  return NF_OK;
}

int32_t nf_qcache_write(int32_t format, int32_t dtype, uint8_t *codes, uint8_t *scales, int32_t *cache_labels,
                        int64_t capacity, int64_t n, int64_t first, int32_t B, const void *x, const int32_t *labels,
                        void *stream) {
  QcacheRows q;
  const int32_t rc = check_qcache(format, dtype, codes, scales, cache_labels, capacity, n, first, B, x, labels, false, &q);
  if (rc) return rc;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  NF_RUN(st, "qcache_write", 0.0, (double)B * (size_of(dtype) * n + n * (format == NF_Q_E2M1 ? 0.5 : 1.0) + n / 32.0),
         launch_qcache_write(format, dtype, q, B, x, labels, st));
  return NF_OK;
}

int32_t nf_qcache_read(int32_t format, int32_t dtype, const uint8_t *codes, const uint8_t *scales,
                       const int32_t *cache_labels, int64_t capacity, int64_t n, int64_t first, const int64_t *idx,
                       int32_t B, void *x_out, int32_t *labels_out, void *stream) {
  QcacheRows q;
  const int32_t rc = check_qcache(format, dtype, codes, scales, cache_labels, capacity, n, first, B, x_out, labels_out, idx != nullptr, &q);
  if (rc) return rc;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  NF_RUN(st, "qcache_read", 0.0, (double)B * (size_of(dtype) * n + n * (format == NF_Q_E2M1 ? 0.5 : 1.0) + n / 32.0),
         launch_qcache_read(format, dtype, q, reinterpret_cast<const long long *>(idx), B, x_out, labels_out, st));
  return NF_OK;
}

int32_t nf_mx_quantise(int32_t dtype, int64_t rows, int64_t cols, const void *x, uint8_t *codes, uint8_t *scales,
                       uint8_t *codes_t, uint8_t *scales_t, void *stream) {
  if (!x || (codes == nullptr) != (scales == nullptr) || (codes_t == nullptr) != (scales_t == nullptr) || (!codes && !codes_t)) return NF_ERR_NULL;
  if (!dtype_ok(dtype) || rows <= 0 || cols <= 0) return NF_ERR_BAD_DESC;
  if (rows > (1ll << 44) / cols || (codes && !codes_t && !mx_quantise_fits(rows, cols, false)) || (codes_t && !mx_quantise_fits(rows, cols, true))) return NF_ERR_UNSUPPORTED;
  if (!all_aligned16(x, codes, scales, codes_t, scales_t)) return NF_ERR_BAD_DESC;
  NF_HIP(launch_mx_quantise(dtype, rows, cols, x, codes, scales, codes_t, scales_t, static_cast<hipStream_t>(stream)));
  return NF_OK;
}

int32_t nf_mx_product_workspace_bytes(const nf_linear_desc *d, int64_t M, size_t *out) {
  MxCall c;
  const int32_t rc = check_mx(d, M, &c);
  if (rc) return rc;
  if (!out) return NF_ERR_NULL;
  *out = mx_product_workspace_bytes(c);
  return NF_OK;
}

int32_t nf_mx_product(const nf_linear_desc *d, int64_t M, const uint8_t *a, const uint8_t *a_scales, const uint8_t *b,
                      const uint8_t *b_scales, const float *bias, const void *r, void *y, void *ws, size_t ws_bytes,
                      void *stream) {
  MxCall c;
  int32_t rc = check_mx(d, M, &c);
  if (rc) return rc;
  if (!a || !a_scales || !b || !b_scales || !y) return NF_ERR_NULL;
  if (!all_aligned16(a, a_scales, b, b_scales, bias, r, y)) return NF_ERR_BAD_DESC;
  if ((rc = check_ws(ws, ws_bytes, mx_product_workspace_bytes(c)))) return rc;
  NF_HIP(launch_mx_product(c, a, a_scales, b, b_scales, bias, r, drop_args(nullptr), y, nullptr, ws, static_cast<hipStream_t>(stream)));
  return NF_OK;
}

int32_t nf_mx_linear_workspace_bytes(const nf_linear_desc *d, int64_t M, size_t *out) {
  MxCall c;
  const int32_t rc = check_mx(d, M, &c);
  if (rc) return rc;
  if (!out) return NF_ERR_NULL;
  *out = mx_linear_workspace_bytes(c);
  return NF_OK;
}

int32_t nf_mx_linear_fwd(const nf_linear_desc *d, int64_t M, const void *x, const uint8_t *W, const uint8_t *W_scales,
                         const float *b, const void *r, const nf_dropout_desc *drop, void *y, void *z, void *ws,
                         size_t ws_bytes, void *stream) {
  MxCall c;
  int32_t rc = check_mx(d, M, &c);
  if (rc) return rc;
  if (!x || !W || !W_scales || !y) return NF_ERR_NULL;
  if (drop && (rc = check_drop(drop))) return rc;
  if (!mx_quantise_fits(M, d->K, false)) return NF_ERR_UNSUPPORTED;
  if (!all_aligned16(x, W, W_scales, b, r, y, z)) return NF_ERR_BAD_DESC;
  if ((rc = check_ws(ws, ws_bytes, mx_linear_workspace_bytes(c)))) return rc;
  NF_HIP(launch_mx_linear(c, x, W, W_scales, b, r, drop_args(drop), y, z, ws, static_cast<hipStream_t>(stream)));
  return NF_OK;
}

}  // extern "C"
