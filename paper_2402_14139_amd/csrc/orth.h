// Launches of the orthogonal updates (sizes and pointers checked already).
#pragma once
#include "nf_internal.h"

namespace nf {

// whether every step's results are bounded where singular values begin at most at 1
bool orth_bounded(const nf_orth_desc &d);
size_t orth_workspace_bytes(const nf_orth_desc &d, int count, const int32_t *rows, const int32_t *cols);
hipError_t launch_orth(const nf_orth_desc &d, int dtype, int count, const void *const *g, void *const *y, const int32_t *rows, const int32_t *cols, void *ws,
                       hipStream_t st);
hipError_t launch_muon(const nf_muon_desc &d, int count, float *const *w, const float *const *g, float *const *v, const int32_t *rows, const int32_t *cols, void *ws,
                       hipStream_t st);

}  // namespace nf
