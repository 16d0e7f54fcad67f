// Host side of the token operators: argument validation, workspace sizes and
// the stream-ordered entry points. Validation never touches the GPU.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "../../include/da2.h"
#include "host_rows.hpp"

namespace {

using namespace da2;

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

// ---- differential attention --------------------------------------------------------------
struct DiffExt {
  Ext q, k;
};

int32_t check_diff(const da2_diff_problem* p, DiffExt* e) {
  if (!p) return DA2_ERR_INVALID_ARG;
  *e = DiffExt{Ext{p->B, p->Hq, p->N, p->d}, Ext{p->B, p->Hk, p->M, p->d}};
  int32_t st = check_ext(e->q);
  if (st || (st = check_ext(e->k))) return st;
  if (p->Hq % p->Hk || (p->causal != 0 && p->causal != 1)) return DA2_ERR_INVALID_ARG;
  if (!(p->scale >= 0x1p-64 && p->scale <= 0x1p64)) return DA2_ERR_INVALID_ARG;
  if (p->d != 64 && p->d != 128) return DA2_ERR_UNSUPPORTED;
  // Positions in 32 bits. The launch grids end at 2^32 threads: row tiles of 256 threads; key tiles and the query heads'
  // dlambda beside them, the latter with 512 threads where key tiles are few.
  const int64_t rows = (int64_t)p->N * (p->Hq / p->Hk);
  if (p->N > (1 << 30) || p->M > (1 << 30) || rows > (1ll << 31) - 1) return DA2_ERR_INVALID_ARG;
  const int64_t heads = (int64_t)p->B * p->Hk, most = (1 << 24) - 8;
  if (heads * ((rows + 31) / 32) > most || heads * (((int64_t)p->M + 127) / 128) + 2ll * p->Hq + 1024 > most)
    return DA2_ERR_INVALID_ARG;
  return DA2_OK;
}

// A tensor of the attention: 16-byte vectors; 128 rows of an input, as a tile has, within 32 bits of byte offset.
int32_t check_attn(const void* p, const da2_tensor* t, const Ext& e, int32_t dtype, bool out) {
  if (!p || !aligned16(p)) return DA2_ERR_INVALID_ARG;
  const int32_t st = check_view(t, e, dtype, out);
  if (st) return st;
  if (dtype == DA2_FP32) return DA2_ERR_UNSUPPORTED;
  if ((e.B > 1 && t->stride_b % 8) || (e.H > 1 && t->stride_h % 8) || (e.N > 1 && t->stride_n % 8))
    return DA2_ERR_INVALID_ARG;
  return !out && e.N > 1 && t->stride_n > (1 << 24) ? DA2_ERR_INVALID_ARG : DA2_OK;
}

da2::DiffArgs diff_args(const da2_diff_problem* p, int32_t dtype) {
  da2::DiffArgs a{};
  a.B = p->B;
  a.Hq = p->Hq;
  a.Hk = p->Hk;
  a.N = p->N;
  a.M = p->M;
  a.d = p->d;
  a.causal = p->causal;
  a.dtype = dtype;
  a.scale = (float)p->scale;
  return a;
}

int64_t diff_ws(const da2_diff_problem* p, bool train) {
  const int64_t f = da2::diff_fwd_ws_bytes(p->B, p->Hq, p->Hk, p->N, p->M, p->d);
  return train ? std::max(f, da2::diff_bwd_ws_bytes(p->B, p->Hq, p->Hk, p->N, p->M, p->d)) : f;
}

// A stride of an extent of 1 is never multiplied by more than zero, but the copies of tiles form row * stride in 32 bits.
View attn_view(const void* p, const da2_tensor* t, const Ext& e) {
  return View{p, t->stride_b, t->stride_h, e.N > 1 ? t->stride_n : 0};
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
  if (!X || !dY || !stats || (!dX && !dw && !db) || (dw && dw == db)) return DA2_ERR_INVALID_ARG;
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

int32_t da2_rope_plan(const da2_rope_desc* r, const da2_rope_freq* f, double* turns, double* scale) {
  if (rope_rot(r) < 0 || !f || !turns || !scale) return DA2_ERR_INVALID_ARG;
  if (f->scaling < DA2_ROPE_PLAIN || f->scaling > DA2_ROPE_YARN) return DA2_ERR_INVALID_ARG;
  if (!(f->base > 1.0) || !(f->factor >= 1.0) || !std::isfinite(f->base) || !std::isfinite(f->factor))
    return DA2_ERR_INVALID_ARG;
  if (f->scaling == DA2_ROPE_PLAIN && f->factor != 1.0) return DA2_ERR_INVALID_ARG;
  const bool yarn = f->scaling == DA2_ROPE_YARN;
  if (yarn && (f->orig_len < 1 || !(f->beta_slow > 0.0) || !(f->beta_fast >= f->beta_slow) ||
               !std::isfinite(f->beta_fast)))
    return DA2_ERR_INVALID_ARG;
  constexpr double kTwoPi = 6.283185307179586476925286766559;
  int64_t p = 0;
  for (int ax = 0; ax < r->axes; ++ax) {
    const double D = r->rot_axis[ax];
    const double base =
        f->scaling == DA2_ROPE_NTK && D > 2 ? f->base * std::pow(f->factor, D / (D - 2)) : f->base;
    // the pair that turns n times over orig_len positions: base^(-2i/D) orig_len / (2 pi) = n
    const auto pair_of = [&](double n) { return D * std::log(f->orig_len / (n * kTwoPi)) / (2 * std::log(f->base)); };
    double lo = 0, hi = 0;
    if (yarn) {
      lo = std::max(std::floor(pair_of(f->beta_fast)), 0.0);
      hi = std::min(std::ceil(pair_of(f->beta_slow)), D - 1);
    }
    for (int i = 0; i < r->rot_axis[ax] / 2; ++i) {
      double w = std::pow(base, -2.0 * i / D);
      if (f->scaling == DA2_ROPE_LINEAR) w /= f->factor;
      if (yarn) {
        const double ramp = std::min(std::max((i - lo) / std::max(hi - lo, 0.001), 0.0), 1.0);
        w = w / f->factor * ramp + w * (1.0 - ramp);
      }
      turns[p++] = w / kTwoPi;
    }
  }
  *scale = yarn ? 0.1 * std::log(f->factor) + 1.0 : 1.0;
  return DA2_OK;
}

int32_t da2_rope(const da2_rope_desc* r, const double* turns, double scale, const int32_t* pos, int64_t pos_stride_b,
                 const da2_rope_rows* s, const void* Q, const da2_tensor* q, void* Qo, const da2_tensor* qo,
                 const void* K, const da2_tensor* k, void* Ko, const da2_tensor* ko, void* stream) {
  const int64_t rot = rope_rot(r);
  if (rot < 0 || !s || !turns || !std::isfinite(scale)) return DA2_ERR_INVALID_ARG;
  if (s->d < 1 || s->d > 65536 || s->d % r->block || s->Hk < 0 || (s->inverse != 0 && s->inverse != 1))
    return DA2_ERR_INVALID_ARG;
  const Ext eq{s->B, s->Hq, s->N, s->d}, ek{s->B, s->Hk, s->N, s->d};
  int32_t st = check_ext(eq);
  if (st || (s->Hk && (st = check_ext(ek)))) return st;
  if ((int64_t)s->Hq + s->Hk > 65535) return DA2_ERR_INVALID_ARG;
  // one thread per unit of a token: the grid ends at 2^32 threads
  if ((int64_t)s->B * s->N * r->block > (1ll << 32) - 256) return DA2_ERR_INVALID_ARG;
  if (pos) {
    if (s->grid_h || s->grid_w || (pos_stride_b != 0 && pos_stride_b < (int64_t)s->N * r->axes))
      return DA2_ERR_INVALID_ARG;
    if (pos_stride_b > (1ll << 40)) return DA2_ERR_INVALID_ARG;
  } else if (r->axes > 1 && (s->grid_w < 1 || (r->axes > 2 && s->grid_h < 1))) {
    return DA2_ERR_INVALID_ARG;
  }
  if (!q || check_view(q, eq, q->dtype, false) || check_view(qo, eq, q->dtype, true)) return DA2_ERR_INVALID_ARG;
  if (!Q || !Qo || (Q == Qo && !same_strides(q, qo, eq))) return DA2_ERR_INVALID_ARG;
  if (s->Hk) {
    if (check_view(k, ek, q->dtype, false) || check_view(ko, ek, q->dtype, true)) return DA2_ERR_INVALID_ARG;
    if (!K || !Ko || (K == Ko && !same_strides(k, ko, ek))) return DA2_ERR_INVALID_ARG;
    if (Ko == Qo || Ko == Q || K == Qo) return DA2_ERR_INVALID_ARG;
  }
  if ((st = check_device())) return st;
  da2::RopeArgs a{};
  a.q = view(Q, q);
  a.qo = out_view(Qo, qo);
  a.q_in_place = Q == Qo;
  if (s->Hk) {
    a.k = view(K, k);
    a.ko = out_view(Ko, ko);
    a.k_in_place = K == Ko;
  }
  a.turns = turns;
  a.pos = pos;
  a.pos_sb = pos_stride_b;
  a.B = s->B;
  a.Hq = s->Hq;
  a.Hk = s->Hk;
  a.N = s->N;
  a.d = s->d;
  a.block = r->block;
  a.rot = (int)rot;
  a.axes = r->axes;
  a.pair0 = r->rot_axis[0] / 2;
  a.pair1 = a.pair0 + r->rot_axis[1] / 2;
  a.grid_h = s->grid_h;
  a.grid_w = s->grid_w;
  a.layout = r->layout;
  a.dtype = q->dtype;
  a.scale = (float)scale;
  a.sign = s->inverse ? -1.0f : 1.0f;
  return hip_status(da2::launch_rope(a, static_cast<hipStream_t>(stream)));
}

int32_t da2_diff_ws_bytes(const da2_diff_problem* p, int32_t train, int64_t* bytes) {
  DiffExt e;
  const int32_t st = check_diff(p, &e);
  if (st) return st;
  if (!bytes || (train != 0 && train != 1)) return DA2_ERR_INVALID_ARG;
  *bytes = diff_ws(p, train != 0);
  return DA2_OK;
}

int32_t da2_diff_attn(const da2_diff_problem* p, const void* Q, const da2_tensor* q, const void* K,
                      const da2_tensor* k, const void* V, const da2_tensor* v, const float* lambda,
                      const int32_t* kv_lens, const int32_t* q_start, void* O, const da2_tensor* o, float* lse,
                      void* ws, int64_t ws_bytes, void* stream) {
  DiffExt e;
  int32_t st = check_diff(p, &e);
  if (st) return st;
  if (!q) return DA2_ERR_INVALID_ARG;
  const int32_t t = q->dtype;
  if ((st = check_attn(Q, q, e.q, t, false)) || (st = check_attn(K, k, e.k, t, false)) ||
      (st = check_attn(V, v, e.k, t, false)) || (st = check_attn(O, o, e.q, t, true)))
    return st;
  if (!lambda || O == Q || O == K || O == V) return DA2_ERR_INVALID_ARG;
  const int64_t need = diff_ws(p, false);
  if (need && (!ws || !aligned16(ws))) return DA2_ERR_INVALID_ARG;
  if (ws_bytes < need) return DA2_ERR_WORKSPACE;
  if ((st = check_device())) return st;
  da2::DiffArgs a = diff_args(p, t);
  a.q = attn_view(Q, q, e.q);
  a.k = attn_view(K, k, e.k);
  a.v = attn_view(V, v, e.k);
  a.o = out_view(O, o);
  a.lam = lambda;
  a.kv_lens = kv_lens;
  a.q_start = q_start;
  a.lse = lse;
  a.ws = static_cast<float*>(ws);
  return hip_status(da2::launch_diff_fwd(a, static_cast<hipStream_t>(stream)));
}

int32_t da2_diff_attn_bwd(const da2_diff_problem* p, const void* Q, const da2_tensor* q, const void* K,
                          const da2_tensor* k, const void* V, const da2_tensor* v, const float* lambda,
                          const int32_t* kv_lens, const int32_t* q_start, const float* lse, const void* dO,
                          const da2_tensor* d_o, void* dQ, const da2_tensor* dq, void* dK, const da2_tensor* dk,
                          void* dV, const da2_tensor* dv, float* dlambda, void* ws, int64_t ws_bytes, void* stream) {
  DiffExt e;
  int32_t st = check_diff(p, &e);
  if (st) return st;
  if (!q) return DA2_ERR_INVALID_ARG;
  const int32_t t = q->dtype;
  if ((st = check_attn(Q, q, e.q, t, false)) || (st = check_attn(K, k, e.k, t, false)) ||
      (st = check_attn(V, v, e.k, t, false)) || (st = check_attn(dO, d_o, e.q, t, false)) ||
      (st = check_attn(dQ, dq, e.q, t, true)) || (st = check_attn(dK, dk, e.k, t, true)) ||
      (st = check_attn(dV, dv, e.k, t, true)))
    return st;
  if (!lambda || !lse || !dlambda || !ws || !aligned16(ws)) return DA2_ERR_INVALID_ARG;
  const void* in[] = {Q, K, V, dO, dQ, dK, dV};
  for (int i = 4; i < 7; ++i)
    for (int j = 0; j < i; ++j)
      if (in[i] == in[j]) return DA2_ERR_INVALID_ARG;
  if (ws_bytes < diff_ws(p, true)) return DA2_ERR_WORKSPACE;
  if ((st = check_device())) return st;
  da2::DiffArgs a = diff_args(p, t);
  a.q = attn_view(Q, q, e.q);
  a.k = attn_view(K, k, e.k);
  a.v = attn_view(V, v, e.k);
  a.dout = attn_view(dO, d_o, e.q);
  a.dq = out_view(dQ, dq);
  a.dk = out_view(dK, dk);
  a.dv = out_view(dV, dv);
  a.lam = lambda;
  a.kv_lens = kv_lens;
  a.q_start = q_start;
  a.rlse = lse;
  a.dlam = dlambda;
  a.ws = static_cast<float*>(ws);
  return hip_status(da2::launch_diff_bwd(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
