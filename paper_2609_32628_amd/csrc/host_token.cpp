// Host side of the token operators: argument validation, workspace sizes and
// the stream-ordered entry points. Validation never touches the GPU.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "../../include/da2.h"
#include "host_util.hpp"
#include "token.hpp"

namespace {

using da2::check_device;
using da2::hip_status;
using da2::OutView;
using da2::View;

bool dtype_ok(int32_t t) { return t == DA2_BF16 || t == DA2_FP32 || t == DA2_FP16; }

// Extents of a [B, H, N, C] tensor.
struct Ext {
  int64_t B, H, N, C;
};

int32_t check_ext(const Ext& e) {
  if (e.B < 1 || e.H < 1 || e.N < 1 || e.C < 1) return DA2_ERR_INVALID_ARG;
  if (e.B > 65535 || e.H * e.N > (1ll << 31) - 1) return DA2_ERR_INVALID_ARG;
  return DA2_OK;
}

// A descriptor against the extents; an output's rows must not overlap: in the
// order of their strides, each dimension's rows end before its next begins.
int32_t check_view(const da2_tensor* t, const Ext& e, int32_t dtype, bool out) {
  if (!t || !dtype_ok(t->dtype) || t->dtype != dtype) return DA2_ERR_INVALID_ARG;
  std::pair<int64_t, int64_t> d[3] = {{t->stride_b, e.B}, {t->stride_h, e.H}, {t->stride_n, e.N}};
  for (auto& s : d) {
    if (s.second == 1) s.first = 0;
    if (s.first < 0 || s.first > (1ll << 40)) return DA2_ERR_INVALID_ARG;
  }
  if (!out) return DA2_OK;
  std::sort(d, d + 3);
  int64_t span = e.C;
  for (const auto& s : d) {
    if (s.second == 1) continue;
    if (s.first < span) return DA2_ERR_INVALID_ARG;
    span += s.first * (s.second - 1);
  }
  return DA2_OK;
}

bool same_strides(const da2_tensor* a, const da2_tensor* b, const Ext& e) {
  return (e.B == 1 || a->stride_b == b->stride_b) && (e.H == 1 || a->stride_h == b->stride_h) &&
         (e.N == 1 || a->stride_n == b->stride_n);
}

// Kernels read no stride of an extent of 1 but multiply it by zero.
View view(const void* p, const da2_tensor* t) { return View{p, t->stride_b, t->stride_h, t->stride_n}; }
OutView out_view(void* p, const da2_tensor* t) { return OutView{p, t->stride_b, t->stride_h, t->stride_n}; }

// ---- row norms ---------------------------------------------------------------------
int32_t check_norm(const da2_rows* r, const da2_norm_desc* n, Ext* e) {
  if (!r || !n) return DA2_ERR_INVALID_ARG;
  *e = Ext{r->B, r->H, r->N, r->C};
  int32_t st = check_ext(*e);
  if (st) return st;
  if (e->C > (1 << 24) || e->B * e->H * e->N > (1ll << 31) - 1) return DA2_ERR_INVALID_ARG;
  if (n->kind != DA2_NORM_LAYER && n->kind != DA2_NORM_RMS) return DA2_ERR_INVALID_ARG;
  if (!dtype_ok(n->wdtype) || (n->plus_one != 0 && n->plus_one != 1)) return DA2_ERR_INVALID_ARG;
  if (n->stride_b != 0 && (n->stride_b < e->C || n->stride_b > (1ll << 40))) return DA2_ERR_INVALID_ARG;
  if (!(n->eps >= 0.0) || !std::isfinite(n->eps)) return DA2_ERR_INVALID_ARG;
  return DA2_OK;
}

int64_t norm_ws(const Ext& e, int32_t dtype, bool adaptive) {
  const int64_t groups = adaptive ? e.B : 1, rows = e.B * e.H * e.N / groups;
  return 8 * e.C * groups * da2::norm_parts(rows, groups, (int)e.C, dtype);
}

da2::NormArgs norm_args(const Ext& e, const da2_norm_desc* n, int32_t dtype) {
  da2::NormArgs a{};
  a.B = (int)e.B;
  a.H = (int)e.H;
  a.N = (int)e.N;
  a.C = (int)e.C;
  a.dtype = dtype;
  a.wdtype = n->wdtype;
  a.kind = n->kind;
  a.plus = (float)n->plus_one;
  a.w_sb = n->stride_b;
  a.eps = n->eps;
  return a;
}

}  // namespace

extern "C" {

int32_t da2_norm(const void* X, const da2_tensor* x, const da2_rows* r, const da2_norm_desc* n, const void* w,
                 const void* b, void* Y, const da2_tensor* y, float* stats, void* stream) {
  Ext e;
  int32_t st = check_norm(r, n, &e);
  if (st) return st;
  if (!x || (st = check_view(x, e, x->dtype, false)) || (st = check_view(y, e, x->dtype, true)))
    return DA2_ERR_INVALID_ARG;
  if (!X || !Y || (X == Y && !same_strides(x, y, e))) return DA2_ERR_INVALID_ARG;
  if ((st = check_device())) return st;
  da2::NormArgs a = norm_args(e, n, x->dtype);
  a.x = view(X, x);
  a.y = out_view(Y, y);
  a.w = w;
  a.b = b;
  a.stats = stats;
  return hip_status(da2::launch_norm(a, static_cast<hipStream_t>(stream)));
}

int32_t da2_norm_ws_bytes(const da2_rows* r, int32_t dtype, int32_t adaptive, int64_t* bytes) {
  const da2_norm_desc n{DA2_NORM_LAYER, DA2_FP32, 0, 0, 0, 0.0};
  Ext e;
  int32_t st = check_norm(r, &n, &e);
  if (st) return st;
  if (!bytes || !dtype_ok(dtype) || (adaptive != 0 && adaptive != 1)) return DA2_ERR_INVALID_ARG;
  *bytes = norm_ws(e, dtype, adaptive);
  return DA2_OK;
}

int32_t da2_norm_bwd(const void* dY, const da2_tensor* dy, const void* X, const da2_tensor* x, const da2_rows* r,
                     const da2_norm_desc* n, const void* w, const float* stats, void* dX, const da2_tensor* dx,
                     void* dw, void* db, void* ws, int64_t ws_bytes, void* stream) {
  Ext e;
  int32_t st = check_norm(r, n, &e);
  if (st) return st;
  if (!x || (st = check_view(x, e, x->dtype, false)) || (st = check_view(dy, e, x->dtype, false)))
    return DA2_ERR_INVALID_ARG;
  if (dX && ((st = check_view(dx, e, x->dtype, true)) || (dX == X && !same_strides(dx, x, e)) ||
             (dX == dY && !same_strides(dx, dy, e))))
    return DA2_ERR_INVALID_ARG;
  if (!X || !dY || !stats || (!dX && !dw && !db)) return DA2_ERR_INVALID_ARG;
  if (dw || db) {
    if (!ws) return DA2_ERR_INVALID_ARG;
    if (ws_bytes < norm_ws(e, x->dtype, n->stride_b != 0)) return DA2_ERR_WORKSPACE;
  }
  if ((st = check_device())) return st;
  da2::NormArgs a = norm_args(e, n, x->dtype);
  a.x = view(X, x);
  a.dy = view(dY, dy);
  if (dX) a.dx = out_view(dX, dx);
  a.w = w;
  a.rstats = stats;
  a.dw = dw;
  a.db = db;
  a.ws = static_cast<float*>(ws);
  return hip_status(da2::launch_norm_bwd(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
