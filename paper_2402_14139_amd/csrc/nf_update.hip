// Entry points of the orthogonal updates (include/nf.h): argument checks, then the launches.  Nothing is enqueued before every check has passed.
#include "nf_enqueue.h"
#include "orth.h"

namespace nf {
namespace {

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

int32_t check_orth(const nf_orth_desc *d, int32_t n, const int32_t *rows, const int32_t *cols) {
  if (!d || !rows || !cols) return NF_ERR_NULL;
  if (n <= 0 || n > NF_ORTH_MATRICES || d->steps <= 0 || d->steps > NF_ORTH_STEPS || !(d->eps >= 0.f)) return NF_ERR_BAD_DESC;
  for (int i = 0; i < n; ++i) {
    if (rows[i] <= 0 || cols[i] <= 0) return NF_ERR_BAD_DESC;
    if (rows[i] > (1 << 20) || cols[i] > (1 << 20) || (rows[i] > (1 << 14) && cols[i] > (1 << 14))) return NF_ERR_UNSUPPORTED;
  }
  if (!orth_bounded(*d)) return NF_ERR_UNSUPPORTED;
  return NF_OK;
}

// pointers of n matrices: given, aligned, and (where they are written) each its own
int32_t check_pointers(int32_t n, const void *const *p, bool written) {
  if (!p) return NF_ERR_NULL;
  for (int i = 0; i < n; ++i) {
    if (!p[i]) return NF_ERR_NULL;
    if (!aligned16(p[i])) return NF_ERR_BAD_DESC;
    for (int k = 0; written && k < i; ++k)
      if (p[k] == p[i]) return NF_ERR_BAD_DESC;
  }
  return NF_OK;
}

int32_t check_ws(const void *ws, size_t have, size_t need) {
  if (!ws || (reinterpret_cast<uintptr_t>(ws) & 255u) || have < need) return NF_ERR_WORKSPACE;
  return NF_OK;
}

}  // namespace
}  // namespace nf

using namespace nf;

extern "C" {

int32_t nf_orthogonalise_workspace_bytes(const nf_orth_desc *d, int32_t n_matrices, const int32_t *rows,
                                         const int32_t *cols, size_t *out) {
  const int32_t rc = check_orth(d, n_matrices, rows, cols);
  if (rc) return rc;
  if (!out) return NF_ERR_NULL;
  *out = orth_workspace_bytes(*d, n_matrices, rows, cols);
  return NF_OK;
}

int32_t nf_orthogonalise(const nf_orth_desc *d, int32_t dtype, int32_t n_matrices, const void *const *g, void *const *y,
                         const int32_t *rows, const int32_t *cols, void *ws, size_t ws_bytes, void *stream) {
  int32_t rc = check_orth(d, n_matrices, rows, cols);
  if (rc) return rc;
  if (dtype != NF_F32 && dtype != NF_BF16 && dtype != NF_F16) return NF_ERR_BAD_DESC;
  if ((rc = check_pointers(n_matrices, g, false)) || (rc = check_pointers(n_matrices, y, true))) return rc;
  for (int i = 0; i < n_matrices; ++i)  // a matrix may be done before another one is read
    for (int k = 0; k < n_matrices; ++k)
      if (i != k && y[i] == g[k]) return NF_ERR_BAD_DESC;
  if ((rc = check_ws(ws, ws_bytes, orth_workspace_bytes(*d, n_matrices, rows, cols)))) return rc;
  NF_HIP(launch_orth(*d, dtype, n_matrices, g, y, rows, cols, ws, static_cast<hipStream_t>(stream)));
  return NF_OK;
}

int32_t nf_muon_update(const nf_muon_desc *d, int32_t n_matrices, float *const *w, const float *const *g,
                       float *const *v, const int32_t *rows, const int32_t *cols, void *ws, size_t ws_bytes,
                       void *stream) {
  if (!d) return NF_ERR_NULL;
  int32_t rc = check_orth(&d->orth, n_matrices, rows, cols);
  if (rc) return rc;
  auto plain = [](auto p) { return reinterpret_cast<const void *const *>(p); };
  if ((rc = check_pointers(n_matrices, plain(w), true)) || (rc = check_pointers(n_matrices, plain(g), false))) return rc;
  if (d->momentum == 0.f) v = nullptr;
  if (v && (rc = check_pointers(n_matrices, plain(v), true))) return rc;
  for (int i = 0; i < n_matrices; ++i)  // what is written is nothing else's
    for (int k = 0; k < n_matrices; ++k)
      if (w[i] == g[k] || (v && (v[i] == g[k] || v[i] == w[k]))) return NF_ERR_BAD_DESC;
  if ((rc = check_ws(ws, ws_bytes, orth_workspace_bytes(d->orth, n_matrices, rows, cols)))) return rc;
  NF_HIP(launch_muon(*d, n_matrices, w, g, v, rows, cols, ws, static_cast<hipStream_t>(stream)));
  return NF_OK;
}

}  // extern "C"
