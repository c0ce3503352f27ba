// What the translation units of the residual stream's norms share.
#pragma once
#include "cct_internal.h"
#include "number_types.h"

namespace cct {

struct ResidualNorm {
  int M, D, type, before, after, gate_rows;
  float eps, scale;
  const void *r, *b, *gate, *w_after, *c_after, *w_before, *c_before;
  void *s, *h;
  long long ldr, ldb, ldgate, lds, ldh;
};
int launch_residual_norm(const ResidualNorm& p, hipStream_t st);

// Sums over rows: of dh, dh * n (before), of dp, dp * n (after), and the gate's.
enum { kDcBefore, kDwBefore, kDcAfter, kDwAfter, kDgate, kNormSums };
struct ResidualNormBack {
  int M, D, type, before, after, gate_rows;
  float eps, scale;
  const void *s, *b, *gate, *w_after, *c_after, *w_before, *ds, *dh;
  void *dr, *db;
  long long lds, ldb, ldgate, ldds, lddh, lddr, lddb;
  void* out[kNormSums];  // the sums' results: vectors, the gate's a matrix
  long long lddgate;
};
// How the rows are cut: `count` runs of `rows`, so that a run's rows are whole gate rows' (`whole`), or `per_gate` runs belong to
// each gate row.  In the workspace: what the rows' gradients are made of, and a row of partial sums per run and kind.
struct ResidualNormPlan {
  bool whole;
  int rows, count, per_gate;
  long long part_off, part_bytes /* of a kind */, total;
};
ResidualNormPlan residual_norm_plan(const cct_residual_norm_desc_t& d);
int launch_residual_norm_back(const ResidualNormBack& p, const ResidualNormPlan& plan, char* ws, hipStream_t st);

}  // namespace cct
