// Launchers of the orthogonalised updates (ortho.hip).
#pragma once

#include "dfp_internal.h"

namespace dfp {

size_t ortho_workspace_bytes(const dfp_ortho_desc& d);
// out = orthogonalised x (type d.type).
dfp_status launch_orthogonalize(const dfp_ortho_desc& d, const void* x, void* out, void* ws, hipStream_t st);
// v and w updated in place (see dfp.h); alpha = lr scale, keep = 1 - lr wd.
dfp_status launch_muon(const dfp_ortho_desc& d, float alpha, float keep, float mu, bool nesterov, float* w, float* v,
                       const void* dw, void* ws, hipStream_t st);

}  // namespace dfp
