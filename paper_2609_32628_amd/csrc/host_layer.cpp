// Host side of the projections, the gated block and the norm and rotation of Q and K:
// argument validation, workspace layouts and the stream-ordered entry points.
// Validation never touches the GPU.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "../../include/da2.h"
#include "host_rows.hpp"
#include "layer.hpp"

namespace {

using namespace da2;

// ---- norm and rotation of Q and K ------------------------------------------------------
int32_t check_qk_rows(const da2_rope_rows* s) {
  if (!s || s->Hk < 0 || s->inverse) return DA2_ERR_INVALID_ARG;
  const Ext eq{s->B, s->Hq, s->N, s->d}, ek{s->B, s->Hk, s->N, s->d};
  int32_t st = check_ext(eq);
  if (st || (s->Hk && (st = check_ext(ek)))) return st;
  // a row's threads are a wave at most, and the grid ends at 2^32 threads
  if ((int64_t)s->Hq + s->Hk > 65535 || (int64_t)s->B * s->N > (1 << 26) - 4) return DA2_ERR_INVALID_ARG;
  return s->d > kQkMaxD ? DA2_ERR_UNSUPPORTED : DA2_OK;
}

int32_t check_qk(const da2_rope_desc* r, const double* turns, double scale, const int32_t* pos, int64_t pos_stride_b,
                 const da2_rope_rows* s, const da2_norm_desc* n) {
  const int64_t rot = rope_rot(r);
  if (rot < 0 || !turns || !std::isfinite(scale)) return DA2_ERR_INVALID_ARG;
  const int32_t st = check_qk_rows(s);
  if (st) return st;
  if (s->d % r->block) return DA2_ERR_INVALID_ARG;
  if (pos) {
    if (s->grid_h || s->grid_w || (pos_stride_b != 0 && pos_stride_b < (int64_t)s->N * r->axes) || pos_stride_b > (1ll << 40))
      return DA2_ERR_INVALID_ARG;
  } else if (r->axes > 1 && (s->grid_w < 1 || (r->axes > 2 && s->grid_h < 1))) {
    return DA2_ERR_INVALID_ARG;
  }
  if (!n || (n->kind != DA2_NORM_LAYER && n->kind != DA2_NORM_RMS) || !dtype_ok(n->wdtype) || n->stride_b != 0 ||
      (n->plus_one != 0 && n->plus_one != 1) || !(n->eps >= 0.0) || !std::isfinite(n->eps))
    return DA2_ERR_INVALID_ARG;
  return DA2_OK;
}

QkArgs qk_args(const da2_rope_desc* r, const double* turns, double scale, const int32_t* pos, int64_t pos_stride_b,
               const da2_rope_rows* s, const da2_norm_desc* n, int32_t dtype) {
  QkArgs a{};
  a.r.turns = turns;
  a.r.pos = pos;
  a.r.pos_sb = pos_stride_b;
  a.r.B = s->B;
  a.r.Hq = s->Hq;
  a.r.Hk = s->Hk;
  a.r.N = s->N;
  a.r.d = s->d;
  a.r.block = r->block;
  a.r.rot = (int)rope_rot(r);
  a.r.axes = r->axes;
  a.r.pair0 = r->rot_axis[0] / 2;
  a.r.pair1 = a.r.pair0 + r->rot_axis[1] / 2;
  a.r.grid_h = s->grid_h;
  a.r.grid_w = s->grid_w;
  a.r.layout = r->layout;
  a.r.dtype = dtype;
  a.r.scale = (float)scale;
  a.r.sign = 1.0f;
  a.kind = n->kind;
  a.wdtype = n->wdtype;
  a.plus = (float)n->plus_one;
  a.eps = n->eps;
  return a;
}

// An output against an input that may be the same memory.
bool meets(const void* out, const da2_tensor* o, const void* in, const da2_tensor* i, const Ext& e) {
  return out == in && !same_strides(o, i, e);
}

// ---- projections -----------------------------------------------------------------------
struct Proj {
  Ext x, y;
  int64_t M, K, F, R;  // tokens, input features, output features, rows of W
  int parts;
  int64_t F8, F64, Np, ldt;
  int dtype;
};

bool same(const void* a, const void* b) { return a == b; }
int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

int32_t check_proj(const da2_proj* p, int parts, Proj* e) {
  if (!p) return DA2_ERR_INVALID_ARG;
  e->x = Ext{p->B, p->Hx, p->N, p->Cx};
  e->y = Ext{p->B, p->Hy, p->N, p->Cy};
  int32_t st = check_ext(e->x);
  if (st || (st = check_ext(e->y))) return st;
  e->M = (int64_t)p->B * p->N;
  e->K = (int64_t)p->Hx * p->Cx;
  e->F = (int64_t)p->Hy * p->Cy;
  e->parts = parts;
  e->R = e->F * parts;
  if (e->K > (1 << 20) || e->F > (1 << 20) || e->M > (1ll << 31) - 1) return DA2_ERR_INVALID_ARG;
  if (p->act < DA2_ACT_NONE || p->act > DA2_ACT_SIGMOID || !dtype_ok(p->dtype)) return DA2_ERR_INVALID_ARG;
  if ((p->Hx > 1 && p->Cx % 64) || (p->Hy > 1 && p->Cy % 8)) return DA2_ERR_INVALID_ARG;
  if (p->dtype == DA2_FP32) return DA2_ERR_UNSUPPORTED;
  const int64_t tiles = (e->M + 127) / 128, wide = std::max(e->R, e->K);
  if (tiles * ((wide + 127) / 128) > (1 << 24) - 8) return DA2_ERR_INVALID_ARG;
  e->F8 = up(e->F, 8);
  e->F64 = up(e->F, 64);
  e->Np = up(p->N, 8);
  e->ldt = up(p->B * e->Np, 64);
  e->dtype = p->dtype;
  return DA2_OK;
}

// Rows of a projection's tensor: 16-byte vectors; 256 rows of an input, as a tile has, within 2^31 bytes.
int32_t check_side(const void* p, const da2_tensor* t, const Ext& e, int32_t dtype, bool out) {
  if (!p || !aligned16(p)) return DA2_ERR_INVALID_ARG;
  const int32_t st = check_view(t, e, dtype, out);
  if (st) return st;
  if ((e.B > 1 && t->stride_b % 8) || (e.H > 1 && t->stride_h % 8) || (e.N > 1 && t->stride_n % 8)) return DA2_ERR_INVALID_ARG;
  return !out && e.N > 1 && t->stride_n > (1 << 22) ? DA2_ERR_INVALID_ARG : DA2_OK;
}
int32_t check_weights(const void* W, int64_t stride, const Proj& e) {
  if (!W || !aligned16(W) || stride < e.K || stride % 8 || stride > (1 << 22)) return DA2_ERR_INVALID_ARG;
  return e.parts > 1 && (e.F + 256) * stride >= (1ll << 31) - (1 << 16) ? DA2_ERR_INVALID_ARG : DA2_OK;
}
bool gate_ok(const void* gate, int64_t stride, const Proj& e) {
  return !gate || stride == 0 || (stride >= e.F && stride <= (1ll << 40));
}

Side rows_side(const void* p, const da2_tensor* t, const Ext& e) {
  return Side{p, e.B > 1 ? t->stride_b : 0, e.H > 1 ? t->stride_h : 0, e.N > 1 ? t->stride_n : 0, (int)e.N, (int)e.C, (int)e.B};
}

Finish plain_finish(OutView y, int64_t H, int64_t C, int64_t N) {
  Finish f{};
  f.y = y;
  f.Hy = (int)H;
  f.Cy = (int)C;
  f.N = (int)N;
  f.F = (int)(H * C);
  return f;
}

// The workspace of the backward pass, in the order of the fields.
struct BwdSpace {
  int64_t dz, dzt, wt, xt, pbias, pgate, scale, product, bytes;
};
BwdSpace bwd_space(const Proj& e, int64_t B, int64_t N) {
  BwdSpace s{};
  int64_t at = 0;
  const auto take = [&](int64_t n) {
    const int64_t here = at;
    at += up(n, 256);
    return here;
  };
  const int64_t blocks = B * dz_blocks(B, N, e.F);
  const int64_t both = e.M <= kFewTokens ? 2 : 1;  // dZ, and what its rounding left over
  s.dz = take(2 * both * e.M * e.parts * e.F64);
  s.dzt = take(2 * both * e.parts * e.F64 * e.ldt);
  s.wt = take(2 * e.K * e.parts * e.F64);
  s.xt = take(2 * e.K * e.ldt);
  s.pbias = take(4 * blocks * e.R);
  s.pgate = take(e.parts == 1 ? 4 * blocks * e.F : 0);
  s.scale = take(e.dtype == DA2_FP16 ? 4 * (1 + dz_tops(e.M, e.F)) : 0);
  int64_t product = 0;
  for (int64_t n = 1; n <= both; ++n)
    product = std::max({product, product_ws_bytes(e.M, N, e.K, e.parts * e.F64, 1, n == 2), product_ws_bytes(e.R, e.F, e.K, e.ldt, 1, n == 2)});
  s.product = take(product);
  s.bytes = at;
  return s;
}

int64_t proj_ws(const Proj& e, int64_t B, int64_t N, bool train) {
  const int64_t f = product_ws_bytes(e.M, N, e.F, e.K, e.parts, false);
  return train ? std::max(f, bwd_space(e, B, N).bytes) : f;
}

int32_t ws_bytes_of(const da2_proj* p, int parts, int32_t train, int64_t* bytes) {
  Proj e;
  const int32_t st = check_proj(p, parts, &e);
  if (st) return st;
  if (!bytes || (train != 0 && train != 1)) return DA2_ERR_INVALID_ARG;
  *bytes = proj_ws(e, p->B, p->N, train != 0);
  return DA2_OK;
}

int32_t forward(const da2_proj* p, int parts, const void* X, const da2_tensor* x, const void* W, int64_t w_stride,
                const void* bias, const void* gate, int64_t gate_stride_b, const void* R, const da2_tensor* r, void* Y,
                const da2_tensor* y, float* Z, void* ws, int64_t ws_bytes, void* stream) {
  Proj e;
  int32_t st = check_proj(p, parts, &e);
  if (st) return st;
  if ((st = check_side(X, x, e.x, p->dtype, false)) || (st = check_weights(W, w_stride, e)) ||
      (st = check_side(Y, y, e.y, p->dtype, true)) || (R && (st = check_side(R, r, e.y, p->dtype, false))))
    return st;
  if (!gate_ok(gate, gate_stride_b, e) || Y == X || Y == W || (Z && (!aligned16(Z) || same(Z, X) || same(Z, W) || same(Z, Y) || same(Z, R))))
    return DA2_ERR_INVALID_ARG;
  if (R && meets(Y, y, R, r, e.y)) return DA2_ERR_INVALID_ARG;
  const int64_t need = proj_ws(e, p->B, p->N, false);
  if (need && (!ws || !aligned16(ws))) return DA2_ERR_INVALID_ARG;
  if (ws_bytes < need) return DA2_ERR_WORKSPACE;
  if ((st = check_device())) return st;
  ProductArgs a{};
  a.t = rows_side(X, x, e.x);
  a.w = Side{W, e.F * w_stride, 0, w_stride, (int)e.F, (int)e.K, parts};
  a.f = plain_finish(out_view(Y, y), p->Hy, p->Cy, p->N);
  a.f.bias = bias;
  a.f.gate = gate;
  a.f.gate_sb = gate_stride_b;
  if (R) a.f.r = view(R, r);
  a.f.z = Z;
  a.f.z_ld = e.F8;
  a.f.act = p->act;
  a.ws = static_cast<float*>(ws);
  a.M = e.M;
  a.K = (int)e.K;
  a.parts = parts;
  a.dtype = p->dtype;
  return hip_status(launch_product(a, static_cast<hipStream_t>(stream)));
}

int32_t backward(const da2_proj* p, int parts, const void* dY, const da2_tensor* dy, const void* X, const da2_tensor* x,
                 const void* W, int64_t w_stride, const void* gate, int64_t gate_stride_b, const float* Z, void* dX,
                 const da2_tensor* dx, void* dW, int64_t dw_stride, void* dbias, void* dgate, void* ws, int64_t ws_bytes,
                 void* stream_) {
  Proj e;
  int32_t st = check_proj(p, parts, &e);
  if (st) return st;
  if ((st = check_side(dY, dy, e.y, p->dtype, false)) || (st = check_side(X, x, e.x, p->dtype, false)) ||
      (st = check_weights(W, w_stride, e)) || (dX && (st = check_side(dX, dx, e.x, p->dtype, true))) ||
      (dW && (st = check_weights(dW, dw_stride, e))))
    return st;
  if (!gate_ok(gate, gate_stride_b, e) || (dgate && !gate) || (!dX && !dW && !dbias && !dgate)) return DA2_ERR_INVALID_ARG;
  const bool plain = parts == 1 && p->act == DA2_ACT_NONE;  // act' is 1
  if ((!plain || dgate) && (!Z || !aligned16(Z))) return DA2_ERR_INVALID_ARG;
  const void* t[] = {dY, X, W, Z, gate, dX, dW, dbias, dgate};
  for (int i = 5; i < 9; ++i)
    for (int j = 0; j < i; ++j)
      if (t[i] && t[i] == t[j]) return DA2_ERR_INVALID_ARG;
  if (dW && e.ldt > (1 << 22)) return DA2_ERR_INVALID_ARG;
  if (!ws || !aligned16(ws)) return DA2_ERR_INVALID_ARG;
  if (ws_bytes < proj_ws(e, p->B, p->N, true)) return DA2_ERR_WORKSPACE;
  if ((st = check_device())) return st;

  const hipStream_t stream = static_cast<hipStream_t>(stream_);
  char* at = static_cast<char*>(ws);
  const BwdSpace s = bwd_space(e, p->B, p->N);
  const int64_t wide = parts * e.F64;
  // dZ is dY where nothing is between them and dY's blocks of features are whole steps of a product
  const bool direct = plain && !gate && (p->Hy == 1 || p->Cy % 64 == 0);
  DzArgs z{};
  z.dy = view(dY, dy);
  z.B = p->B;
  z.N = p->N;
  z.Hy = p->Hy;
  z.Cy = p->Cy;
  z.F = (int)e.F;
  z.parts = parts;
  z.z = plain && !dgate ? nullptr : Z;
  z.z_ld = e.F8;
  z.gate = gate;
  z.gate_sb = gate_stride_b;
  z.act = p->act;
  z.dtype = p->dtype;
  if (dX && !direct) z.dz = at + s.dz;
  if (dW) z.dzt = at + s.dzt;
  z.F64 = e.F64;
  z.Np = e.Np;
  z.ldt = e.ldt;
  // Over many tokens and features the rounding of dZ averages out to as much as the gradients' own; over a few it need not.
  z.lo = !direct && e.M <= kFewTokens;
  if (p->dtype == DA2_FP16 && !(plain && !gate) && (dX || dW)) {
    z.back = reinterpret_cast<float*>(at + s.scale);
    z.n_tops = dz_tops(e.M, e.F);
  }
  if (dbias) z.pbias = reinterpret_cast<float*>(at + s.pbias);
  if (dgate) z.pgate = reinterpret_cast<float*>(at + s.pgate);
  z.dbias = dbias;
  z.dgate = dgate;
  z.dgate_sb = gate_stride_b;
  hipError_t err = hipSuccess;
  // A copy is made just before the product that reads it (both in front: 3 to 5% slower); with the largest gradients to be found, the
  // first has to be in front.
  const auto copy_w = [&](const DzArgs* top) {
    return launch_transpose(TransposeArgs{Side{W, e.F * w_stride, 0, w_stride, (int)e.F, (int)e.K, parts}, parts, (int)e.K, at + s.wt, e.F64, wide}, top, stream);
  };
  const auto copy_x = [&](const DzArgs* top) {
    return launch_transpose(TransposeArgs{rows_side(X, x, e.x), p->B, (int)e.K, at + s.xt, e.Np, e.ldt}, top, stream);
  };
  if (z.back) err = dX ? copy_w(&z) : copy_x(&z);
  if (err == hipSuccess && (z.dz || z.dzt || dbias || dgate)) err = launch_dz(z, stream);
  ProductArgs a{};
  a.ws = reinterpret_cast<float*>(at + s.product);
  a.parts = 1;
  a.dtype = p->dtype;
  if (err == hipSuccess && dX) {
    if (!z.back) err = copy_w(nullptr);
    a.t = direct ? rows_side(dY, dy, e.y) : Side{z.dz, 0, wide, wide << z.lo, (int)e.M, (int)wide, 1};
    a.lo = z.lo;
    a.K = direct ? (int)e.F : (int)wide;
    a.w = Side{at + s.wt, 0, 0, wide, (int)e.K, a.K, 1};
    a.f = plain_finish(out_view(dX, dx), p->Hx, p->Cx, p->N);
    a.f.back = z.back;
    a.M = e.M;
    if (err == hipSuccess) err = launch_product(a, stream);
  }
  if (err == hipSuccess && dW) {
    if (!z.back || dX) err = copy_x(nullptr);
    const int64_t ld = e.ldt << z.lo;
    a.t = Side{at + s.dzt, e.F64 * ld, e.ldt, ld, (int)e.F, (int)e.ldt, parts};
    a.lo = z.lo;
    a.w = Side{at + s.xt, 0, 0, e.ldt, (int)e.K, (int)e.ldt, 1};
    a.K = (int)e.ldt;
    a.f = plain_finish(OutView{dW, e.F * dw_stride, 0, dw_stride}, 1, e.K, e.F);
    a.f.back = z.back;
    a.M = e.R;
    if (err == hipSuccess) err = launch_product(a, stream);
  }
  return hip_status(err);
}

}  // namespace

extern "C" {

int32_t da2_qk_norm_rope(const da2_rope_desc* r, const double* turns, double scale, const int32_t* pos,
                         int64_t pos_stride_b, const da2_rope_rows* s, const da2_norm_desc* n, const void* w_q,
                         const void* w_k, const void* Q, const da2_tensor* q, void* Qo, const da2_tensor* qo,
                         const void* K, const da2_tensor* k, void* Ko, const da2_tensor* ko, void* stream) {
  int32_t st = check_qk(r, turns, scale, pos, pos_stride_b, s, n);
  if (st) return st;
  const Ext eq{s->B, s->Hq, s->N, s->d}, ek{s->B, s->Hk, s->N, s->d};
  if (!q || check_view(q, eq, q->dtype, false) || check_view(qo, eq, q->dtype, true)) return DA2_ERR_INVALID_ARG;
  if (!Q || !Qo || meets(Qo, qo, Q, q, eq)) return DA2_ERR_INVALID_ARG;
  if (s->Hk) {
    if (check_view(k, ek, q->dtype, false) || check_view(ko, ek, q->dtype, true)) return DA2_ERR_INVALID_ARG;
    if (!K || !Ko || meets(Ko, ko, K, k, ek)) return DA2_ERR_INVALID_ARG;
    if (Ko == Qo || Ko == Q || K == Qo) return DA2_ERR_INVALID_ARG;
  }
  if ((st = check_device())) return st;
  QkArgs a = qk_args(r, turns, scale, pos, pos_stride_b, s, n, q->dtype);
  a.r.q = view(Q, q);
  a.r.qo = out_view(Qo, qo);
  if (s->Hk) {
    a.r.k = view(K, k);
    a.r.ko = out_view(Ko, ko);
  }
  a.wq = w_q;
  a.wk = w_k;
  return hip_status(launch_qk(a, static_cast<hipStream_t>(stream)));
}

int32_t da2_qk_norm_rope_ws_bytes(const da2_rope_rows* s, int64_t* bytes) {
  const int32_t st = check_qk_rows(s);
  if (st) return st;
  if (!bytes) return DA2_ERR_INVALID_ARG;
  *bytes = qk_ws_bytes(s->B, s->Hq, s->Hk, s->N, s->d);
  return DA2_OK;
}

int32_t da2_qk_norm_rope_bwd(const da2_rope_desc* r, const double* turns, double scale, const int32_t* pos,
                             int64_t pos_stride_b, const da2_rope_rows* s, const da2_norm_desc* n, const void* w_q,
                             const void* w_k, const void* dQo, const da2_tensor* dqo, const void* Q,
                             const da2_tensor* q, void* dQ, const da2_tensor* dq, const void* dKo,
                             const da2_tensor* dko, const void* K, const da2_tensor* k, void* dK,
                             const da2_tensor* dk, void* dw_q, void* dw_k, void* ws, int64_t ws_bytes,
                             void* stream) {
  int32_t st = check_qk(r, turns, scale, pos, pos_stride_b, s, n);
  if (st) return st;
  const Ext eq{s->B, s->Hq, s->N, s->d}, ek{s->B, s->Hk, s->N, s->d};
  if (!q || check_view(q, eq, q->dtype, false) || check_view(dqo, eq, q->dtype, false) || check_view(dq, eq, q->dtype, true))
    return DA2_ERR_INVALID_ARG;
  if (!Q || !dQo || !dQ || meets(dQ, dq, Q, q, eq) || meets(dQ, dq, dQo, dqo, eq)) return DA2_ERR_INVALID_ARG;
  if (s->Hk) {
    if (check_view(k, ek, q->dtype, false) || check_view(dko, ek, q->dtype, false) || check_view(dk, ek, q->dtype, true))
      return DA2_ERR_INVALID_ARG;
    if (!K || !dKo || !dK || meets(dK, dk, K, k, ek) || meets(dK, dk, dKo, dko, ek)) return DA2_ERR_INVALID_ARG;
    if (dK == dQ || dK == Q || dK == dQo || dQ == K || dQ == dKo) return DA2_ERR_INVALID_ARG;
  }
  if ((dw_q && dw_q == dw_k) || (dw_k && !s->Hk)) return DA2_ERR_INVALID_ARG;
  if (dw_q || dw_k) {
    if (!ws || !aligned16(ws)) return DA2_ERR_INVALID_ARG;
    if (ws_bytes < qk_ws_bytes(s->B, s->Hq, s->Hk, s->N, s->d)) return DA2_ERR_WORKSPACE;
  }
  if ((st = check_device())) return st;
  QkArgs a = qk_args(r, turns, scale, pos, pos_stride_b, s, n, q->dtype);
  a.r.sign = -1.0f;
  a.r.q = view(dQo, dqo);
  a.r.qo = out_view(dQ, dq);
  a.xq = view(Q, q);
  if (s->Hk) {
    a.r.k = view(dKo, dko);
    a.r.ko = out_view(dK, dk);
    a.xk = view(K, k);
  }
  a.wq = w_q;
  a.wk = w_k;
  a.dwq = dw_q;
  a.dwk = dw_k;
  a.ws = static_cast<float*>(ws);
  return hip_status(launch_qk_bwd(a, static_cast<hipStream_t>(stream)));
}

int32_t da2_linear_ws_bytes(const da2_proj* p, int32_t train, int64_t* bytes) { return ws_bytes_of(p, 1, train, bytes); }

int32_t da2_linear(const da2_proj* p, const void* X, const da2_tensor* x, const void* W, int64_t w_stride,
                   const void* bias, const void* gate, int64_t gate_stride_b, const void* R, const da2_tensor* r,
                   void* Y, const da2_tensor* y, float* Z, void* ws, int64_t ws_bytes, void* stream) {
  return forward(p, 1, X, x, W, w_stride, bias, gate, gate_stride_b, R, r, Y, y, Z, ws, ws_bytes, stream);
}

int32_t da2_linear_bwd(const da2_proj* p, const void* dY, const da2_tensor* dy, const void* X, const da2_tensor* x,
                       const void* W, int64_t w_stride, const void* gate, int64_t gate_stride_b, const float* Z,
                       void* dX, const da2_tensor* dx, void* dW, int64_t dw_stride, void* dbias, void* dgate,
                       void* ws, int64_t ws_bytes, void* stream) {
  return backward(p, 1, dY, dy, X, x, W, w_stride, gate, gate_stride_b, Z, dX, dx, dW, dw_stride, dbias, dgate, ws, ws_bytes,
                  stream);
}

int32_t da2_glu_ws_bytes(const da2_proj* p, int32_t train, int64_t* bytes) { return ws_bytes_of(p, 2, train, bytes); }

int32_t da2_glu(const da2_proj* p, const void* X, const da2_tensor* x, const void* W, int64_t w_stride,
                const void* bias, void* Y, const da2_tensor* y, float* Z, void* ws, int64_t ws_bytes, void* stream) {
  return forward(p, 2, X, x, W, w_stride, bias, nullptr, 0, nullptr, nullptr, Y, y, Z, ws, ws_bytes, stream);
}

int32_t da2_glu_bwd(const da2_proj* p, const void* dY, const da2_tensor* dy, const void* X, const da2_tensor* x,
                    const void* W, int64_t w_stride, const float* Z, void* dX, const da2_tensor* dx, void* dW,
                    int64_t dw_stride, void* dbias, void* ws, int64_t ws_bytes, void* stream) {
  return backward(p, 2, dY, dy, X, x, W, w_stride, nullptr, 0, Z, dX, dx, dW, dw_stride, dbias, nullptr, ws, ws_bytes, stream);
}

}  // extern "C"
