// C ABI of the INT8 linear layers and the orthogonalised updates: host-side
// validation and dispatch, every argument check before the first HIP call.
#include <algorithm>
#include <cmath>

#include "dfp_internal.h"
#include "dfp_types.h"
#include "linear_i8.h"
#include "ortho.h"

namespace dfp {
namespace {

// Elements of a tensor or operand, and sides of a product: beyond what the card holds,
// and few enough that no launch reaches 2^32 threads (a third of it at worst).
constexpr int64_t kMaxElems = (int64_t)1 << 36;
constexpr int64_t kMaxSide = ((int64_t)1 << 31) - 256, kMaxProductSide = 1 << 26;

bool aligned(const void* p, uintptr_t a) { return ((uintptr_t)p % a) == 0; }
bool type_ok(int32_t t) { return t >= DFP_F32 && t <= DFP_F16; }
bool i8_rounding_ok(int32_t r) { return r == DFP_ROUND_NEAREST || r == DFP_ROUND_STOCHASTIC; }

dfp_status linear_checks(const dfp_linear_desc* d) {
  if (!d) return DFP_ERR_NULL;
  if (!type_ok(d->type) || !i8_rounding_ok(d->rounding)) return DFP_ERR_PARAM;
  if (d->m < 1 || d->n < 1 || d->k < 1 || std::max({d->m, d->n, d->k}) > kMaxProductSide) return DFP_ERR_SHAPE;
  const int64_t m = i8_ld(d->m), n = i8_ld(d->n), k = i8_ld(d->k);
  if (m * n > kMaxElems || m * k > kMaxElems || n * k > kMaxElems) return DFP_ERR_SHAPE;
  return DFP_OK;
}

// One workspace serves every call of a descriptor: an INT8 operand, its scales,
// what the column maxima of the backward-weights call need, and the sums of a
// sliced product.
struct LinearWs {
  int64_t op, scale, cols, slices, bytes;
};
LinearWs linear_ws(const dfp_linear_desc& d) {
  LinearWs w;
  int64_t at = 0;
  auto take = [&](int64_t bytes) {
    const int64_t o = at;
    at += (bytes + 255) / 256 * 256;
    return o;
  };
  w.op = take(std::max({d.m * i8_ld(d.k), d.m * i8_ld(d.n), d.n * i8_ld(d.m)}));
  w.scale = take((int64_t)std::max(d.m, d.n) * 4);
  w.cols = take(plan_cols_i8(d.m, d.n).bytes);
  w.slices = take(std::max({plan_gemm_i8(d.m, d.n, d.k).bytes, plan_gemm_i8(d.m, d.k, d.n).bytes,
                            plan_gemm_i8(d.n, d.k, d.m).bytes}));
  w.bytes = at;
  return w;
}

dfp_status ws_checks(const void* ws, size_t have, size_t need) {
  if (!ws || have < need) return DFP_ERR_WORKSPACE;
  if (!aligned(ws, 256)) return DFP_ERR_ALIGN;
  return DFP_OK;
}

dfp_status ortho_checks(const dfp_ortho_desc* d) {
  if (!d) return DFP_ERR_NULL;
  if (!type_ok(d->type) || d->steps < 1 || d->steps > DFP_ORTHO_MAX_STEPS) return DFP_ERR_PARAM;
  if (!(d->eps > 0.f) || !std::isfinite(d->eps)) return DFP_ERR_PARAM;
  for (int s = 0; s < d->steps; ++s)
    for (int i = 0; i < 3; ++i)
      if (!(std::fabs(d->coef[s][i]) <= 64.f)) return DFP_ERR_PARAM;
  if (d->batch < 1 || d->rows < 1 || d->cols < 1 || d->batch > 65535 || d->rows > 65536 || d->cols > 65536)
    return DFP_ERR_SHAPE;
  if (i8_ld(d->rows) * i8_ld(d->cols) > kMaxElems / d->batch) return DFP_ERR_SHAPE;
  return DFP_OK;
}

}  // namespace
}  // namespace dfp

using namespace dfp;

extern "C" {

int64_t dfp_i8_ld(int64_t cols) { return cols < 1 || cols > kMaxSide ? 0 : i8_ld(cols); }

dfp_status dfp_quantize_i8(int64_t rows, int64_t cols, int32_t type, int32_t rounding, uint64_t seed, int32_t role,
                           const void* src, int8_t* q, float* scale, int8_t* qt, void* stream) {
  if (!src || !q || !scale) return DFP_ERR_NULL;
  if (!type_ok(type) || !i8_rounding_ok(rounding) || role < DFP_ROLE_X || role > DFP_ROLE_DX) return DFP_ERR_PARAM;
  if (rows < 1 || cols < 1 || rows > kMaxSide || cols > kMaxSide) return DFP_ERR_SHAPE;
  if (i8_ld(rows) * i8_ld(cols) > kMaxElems) return DFP_ERR_SHAPE;
  if (!aligned(src, 16) || !aligned(q, 16) || !aligned(qt, 16) || !aligned(scale, 4)) return DFP_ERR_ALIGN;
  hipStream_t st = (hipStream_t)stream;
  dfp_status rc = launch_rows_i8(type, rounding, seed, (uint32_t)role, src, rows, cols, nullptr, q, scale, st);
  if (rc == DFP_OK && qt) rc = launch_transpose_i8(q, rows, cols, qt, st);
  return rc;
}

size_t dfp_linear_i8_workspace_bytes(const dfp_linear_desc* d) {
  return linear_checks(d) == DFP_OK ? (size_t)linear_ws(*d).bytes : 0;
}

dfp_status dfp_gemm_i8(const dfp_linear_desc* d, const int8_t* a, const float* sa, const int8_t* b, const float* sb,
                       const float* bias, void* out, void* workspace, size_t ws_bytes, void* stream) {
  if (!d || !a || !sa || !b || !sb || !out) return DFP_ERR_NULL;
  dfp_status rc = linear_checks(d);
  if (rc != DFP_OK) return rc;
  if (d->k > DFP_I8_MAX_SUM) return DFP_ERR_SHAPE;
  if (!aligned(a, 16) || !aligned(b, 16) || !aligned(out, 16) || !aligned(sa, 4) || !aligned(sb, 4) ||
      !aligned(bias, 4))
    return DFP_ERR_ALIGN;
  const LinearWs w = linear_ws(*d);
  if ((rc = ws_checks(workspace, ws_bytes, w.bytes)) != DFP_OK) return rc;
  return launch_gemm_i8(d->m, d->n, d->k, a, sa, b, sb, bias, d->type, out, (uint8_t*)workspace + w.slices,
                        (hipStream_t)stream);
}

dfp_status dfp_linear_i8_fwd(const dfp_linear_desc* d, const void* x, const int8_t* wq, const float* sw,
                             const float* bias, void* y, int8_t* xq, float* sx, int8_t* xqt, void* workspace,
                             size_t ws_bytes, void* stream) {
  if (!d || !x || !wq || !sw || !y) return DFP_ERR_NULL;
  dfp_status rc = linear_checks(d);
  if (rc != DFP_OK) return rc;
  if (d->k > DFP_I8_MAX_SUM) return DFP_ERR_SHAPE;
  if (!aligned(x, 16) || !aligned(wq, 16) || !aligned(y, 16) || !aligned(xq, 16) || !aligned(xqt, 16) ||
      !aligned(sw, 4) || !aligned(bias, 4) || !aligned(sx, 4))
    return DFP_ERR_ALIGN;
  const LinearWs w = linear_ws(*d);
  if ((rc = ws_checks(workspace, ws_bytes, w.bytes)) != DFP_OK) return rc;
  hipStream_t st = (hipStream_t)stream;
  if (!xq && !sx && !xqt && fits_token_i8(d->m, d->k))
    return launch_token_i8(d->m, d->n, d->k, d->type, d->rounding, d->seed, x, wq, sw, bias, y, st);
  int8_t* q = xq ? xq : (int8_t*)workspace + w.op;
  float* s = sx ? sx : (float*)((uint8_t*)workspace + w.scale);
  rc = launch_rows_i8(d->type, d->rounding, d->seed, DFP_ROLE_X, x, d->m, d->k, nullptr, q, s, st);
  if (rc == DFP_OK) rc = launch_gemm_i8(d->m, d->n, d->k, q, s, wq, sw, bias, d->type, y, (uint8_t*)workspace + w.slices, st);
  if (rc == DFP_OK && xqt) rc = launch_transpose_i8(q, d->m, d->k, xqt, st);
  return rc;
}

dfp_status dfp_linear_i8_bwd_data(const dfp_linear_desc* d, const void* dy, const int8_t* wqt, const float* sw,
                                  void* dx, void* workspace, size_t ws_bytes, void* stream) {
  if (!d || !dy || !wqt || !sw || !dx) return DFP_ERR_NULL;
  dfp_status rc = linear_checks(d);
  if (rc != DFP_OK) return rc;
  if (d->n > DFP_I8_MAX_SUM) return DFP_ERR_SHAPE;
  if (!aligned(dy, 16) || !aligned(wqt, 16) || !aligned(dx, 16) || !aligned(sw, 4)) return DFP_ERR_ALIGN;
  const LinearWs w = linear_ws(*d);
  if ((rc = ws_checks(workspace, ws_bytes, w.bytes)) != DFP_OK) return rc;
  hipStream_t st = (hipStream_t)stream;
  int8_t* q = (int8_t*)workspace + w.op;
  float* s = (float*)((uint8_t*)workspace + w.scale);
  rc = launch_rows_i8(d->type, d->rounding, d->seed, DFP_ROLE_DY, dy, d->m, d->n, sw, q, s, st);
  if (rc == DFP_OK) rc = launch_gemm_i8(d->m, d->k, d->n, q, s, wqt, nullptr, nullptr, d->type, dx,
                                         (uint8_t*)workspace + w.slices, st);
  return rc;
}

dfp_status dfp_linear_i8_bwd_weights(const dfp_linear_desc* d, const void* dy, const int8_t* xqt, const float* sx,
                                     float* dw, float* db, void* workspace, size_t ws_bytes, void* stream) {
  if (!d || !dy || !xqt || !sx || !dw) return DFP_ERR_NULL;
  dfp_status rc = linear_checks(d);
  if (rc != DFP_OK) return rc;
  if (d->m > DFP_I8_MAX_SUM) return DFP_ERR_SHAPE;
  if (!aligned(dy, 16) || !aligned(xqt, 16) || !aligned(dw, 16) || !aligned(sx, 4) || !aligned(db, 4))
    return DFP_ERR_ALIGN;
  const LinearWs w = linear_ws(*d);
  if ((rc = ws_checks(workspace, ws_bytes, w.bytes)) != DFP_OK) return rc;
  hipStream_t st = (hipStream_t)stream;
  int8_t* q = (int8_t*)workspace + w.op;
  float* s = (float*)((uint8_t*)workspace + w.scale);
  rc = launch_cols_i8_t(d->type, d->rounding, d->seed, DFP_ROLE_DY, dy, d->m, d->n, sx, q, s, db,
                        (uint8_t*)workspace + w.cols, st);
  if (rc == DFP_OK) rc = launch_gemm_i8(d->n, d->k, d->m, q, s, xqt, nullptr, nullptr, DFP_F32, dw,
                                         (uint8_t*)workspace + w.slices, st);
  return rc;
}

size_t dfp_ortho_workspace_bytes(const dfp_ortho_desc* d) {
  return ortho_checks(d) == DFP_OK ? ortho_workspace_bytes(*d) : 0;
}

dfp_status dfp_orthogonalize(const dfp_ortho_desc* d, const void* x, void* out, void* workspace, size_t ws_bytes,
                             void* stream) {
  if (!d || !x || !out) return DFP_ERR_NULL;
  dfp_status rc = ortho_checks(d);
  if (rc != DFP_OK) return rc;
  if (!aligned(x, 16) || !aligned(out, 16)) return DFP_ERR_ALIGN;
  if ((rc = ws_checks(workspace, ws_bytes, ortho_workspace_bytes(*d))) != DFP_OK) return rc;
  return launch_orthogonalize(*d, x, out, workspace, (hipStream_t)stream);
}

dfp_status dfp_muon_quantize(const dfp_ortho_desc* d, float lr, float mu, float wd, float scale, int32_t nesterov,
                             float* w, float* v, const void* dw, int8_t* wq, float* sw, int8_t* wqt, void* workspace,
                             size_t ws_bytes, void* stream) {
  if (!d || !w || !v || !dw) return DFP_ERR_NULL;
  if (!wq != !sw || (wqt && !wq)) return DFP_ERR_NULL;
  dfp_status rc = ortho_checks(d);
  if (rc != DFP_OK) return rc;
  if (nesterov != 0 && nesterov != 1) return DFP_ERR_PARAM;
  if (wqt && d->batch != 1) return DFP_ERR_PARAM;
  if (!aligned(w, 16) || !aligned(v, 16) || !aligned(dw, 16) || !aligned(wq, 16) || !aligned(wqt, 16) ||
      !aligned(sw, 4))
    return DFP_ERR_ALIGN;
  if ((rc = ws_checks(workspace, ws_bytes, ortho_workspace_bytes(*d))) != DFP_OK) return rc;
  hipStream_t st = (hipStream_t)stream;
  rc = launch_muon(*d, (float)((double)lr * scale), (float)(1. - (double)lr * wd), mu, nesterov != 0, w, v, dw,
                   workspace, st);
  const int64_t rows = (int64_t)d->batch * d->rows;
  if (rc == DFP_OK && wq)
    rc = launch_rows_i8(DFP_F32, DFP_ROUND_NEAREST, 0, DFP_ROLE_W, w, rows, d->cols, nullptr, wq, sw, st);
  if (rc == DFP_OK && wqt) rc = launch_transpose_i8(wq, rows, d->cols, wqt, st);
  return rc;
}

}  // extern "C"
