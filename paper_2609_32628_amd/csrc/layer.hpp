// Kernel arguments and launchers of the projections, the gated feed-forward block and
// the norm and rotation of Q and K in one pass. Internal to libda2.
#pragma once

#include "plan.hpp"
#include "token.hpp"

namespace da2 {

// Rows of a product's operand: row r is token r % N of sample r / N (or row r % N of
// part r / N of a weight matrix); its k-th element lies in block ("head") k / C.
// Strides in elements; sh is not used when C covers the whole row.
struct Side {
  const void* p;
  int64_t sb, sh, sn;
  int N, C, B;  // B: samples (or parts)
};

// What is done with the sums z of a row of features before they are stored.
struct Finish {
  const void* bias;  // [parts F], or null
  const void* gate;  // [F] of each sample, gate_sb elements apart, or null
  int64_t gate_sb;
  View r;            // residual rows, or p null
  OutView y;
  int Hy, Cy;        // features are Hy blocks of Cy
  float* z;          // the sums, [rows][parts][z_ld], or null
  int64_t z_ld;
  const float* back; // factor of the sums before anything else (fp16), or null: 1
  int act;           // da2_act
  int N;             // tokens of a sample
  int F;             // features (of each part)
};

// Products of the rows of t (tokens) with the rows of w (weights) over K elements. lo: t's elements are the sums of two
// blocks of K, t.sh apart (values, and what their rounding left over); K is whole steps.
struct ProductArgs {
  Side t, w;
  Finish f;
  float* ws;    // partial sums of a split product
  int64_t M;    // rows of t
  int K, parts; // parts: 2 for a gated block (w's rows are part 0, then part 1), else 1
  int dtype;
  bool lo;
};
// Workspace of a product of M rows, which may be taken N at a time.
int64_t product_ws_bytes(int64_t M, int64_t N, int64_t F, int64_t K, int parts, bool lo);
hipError_t launch_product(const ProductArgs& a, hipStream_t stream);

// Gradients of the sums: dz of a row from dY, the saved sums z, activation and gate.
struct DzArgs {
  View dy;
  int B, N, Hy, Cy, F, parts;
  const float* z;     // [B N][parts][z_ld], or null: no activation
  int64_t z_ld;
  const void* gate;
  int64_t gate_sb;
  int act, dtype;
  void* dz;           // [B N][1 + lo][parts][F64], or null
  void* dzt;          // [parts][F64][1 + lo][ldt], column b Np + n; or null
  int64_t F64, Np, ldt;
  int lo;             // 1: behind the rounded values what rounding left over
  float *pbias, *pgate;  // partial sums [B][blocks][parts][F] and [B][blocks][F], or null
  void *dbias, *dgate;
  int64_t dgate_sb;   // 0: one gate for all samples
  float* back;        // fp16: what undoes the scale of dz, then the n_tops values it comes from; null: dz is not scaled
  int n_tops;
};
// Whether dz of T is stored times a power of two.
template <typename T>
constexpr bool kScaledDz = __is_same(T, fp16_t);
int dz_tops(int64_t M, int64_t F);
int dz_blocks(int64_t B, int64_t N, int64_t F);
hipError_t launch_dz(const DzArgs& a, hipStream_t stream);

// Sums over the parts of float32 p[groups][parts][cols]: columns below split to out0 (out_sb elements between the
// groups), the others to out1; of type dtype.
hipError_t launch_column_sum(const float* p, int64_t parts, int64_t cols, int64_t groups, int dtype, void* out0, void* out1,
                             int64_t split, int64_t out_sb, hipStream_t stream);

// out[k][b Np + n] = element k of row (b, n), zeros for n from N on and up to column ld of the last sample.
struct TransposeArgs {  // of 16-bit elements
  Side s;
  int B, K;
  void* out;
  int64_t Np, ld;
};
// With top, the same launch finds the largest gradients of the sums, which launch_dz needs (fp16).
hipError_t launch_transpose(const TransposeArgs& a, const DzArgs* top, hipStream_t stream);

// Norm of the heads of Q and K, then rotary positions.
struct QkArgs {
  RopeArgs r;         // forward: q, k in and qo, ko out; backward: gradients of the results in, of the inputs out
  View xq, xk;        // backward: the inputs
  const void *wq, *wk;
  void *dwq, *dwk;
  float* ws;
  int kind, wdtype;
  float plus;
  double eps;
};
constexpr int kQkMaxD = 512;  // channels of a head: a row's threads are a wave at most
int64_t qk_ws_bytes(int B, int Hq, int Hk, int N, int d);
hipError_t launch_qk(const QkArgs& a, hipStream_t stream);
hipError_t launch_qk_bwd(const QkArgs& a, hipStream_t stream);

}  // namespace da2
