// The feed-forward operators' entry points (cct_linear_*, cct_gated_*): checks of arguments, workspace layouts, and which
// kernels a call runs.
#include <algorithm>

#include "activation.h"
#include "feed_forward.h"

namespace cct {
namespace {

long long up(long long v, long long to) { return (v + to - 1) / to * to; }

// Parts of a workspace, one behind the other.
struct Layout {
  long long total = 0;
  long long take(long long bytes) {
    const long long at = total;
    total += up(bytes, 256);
    return at;
  }
};

typedef FfOperand Matrix;
// A tensor of rows x cols of a type: there, aligned to a value, rows that do not overlap.
bool matrix_ok(const Matrix& m, long long rows, long long cols, int type) {
  if (!m.p || ((uintptr_t)m.p & (type_bytes(type) - 1)) || m.ld < 0) return false;
  return rows <= 1 || m.ld >= cols;
}
bool vector_ok(const void* p, int type) { return !((uintptr_t)p & (type_bytes(type) - 1)); }

// Sizes up to which no product of two of them, a stride and a value's bytes passes 63 bits and a size and a tile 31, and each
// matrix is no larger than 2^38 bytes, which no card holds: the kernels' launches count on that.
int dims_ok(int32_t M, int32_t N, int32_t K, int32_t type, int32_t activation) {
  if (M < 0 || N < 1 || K < 1 || !type_known(type) || !activation_known(activation)) return CCT_EINVAL;
  if (std::max(M, std::max(N, K)) > 0x7fffff00) return CCT_EUNSUPPORTED;
  const long long most = (1LL << 38) / type_bytes(type);
  return std::max((long long)M * N, std::max((long long)M * K, (long long)N * K)) <= most ? CCT_OK : CCT_EUNSUPPORTED;
}
int workspace_ok(const void* workspace, size_t have, long long need) {
  if (!workspace || ((uintptr_t)workspace & 255)) return CCT_EINVAL;
  return have >= (size_t)need ? CCT_OK : CCT_EWORKSPACE;
}

// Room for a copy of a matrix whose rows begin at multiples of 16 bytes (16-bit types only: see ff_in_place).
long long copy_bytes(long long rows, long long cols, int type) {
  return type == CCT_TYPE_F32 ? 0 : rows * up(cols, 8) * type_bytes(type);
}
// Room for a product's packed operand (fp32) and its partial sums.
struct Room {
  long long pack, part;
};
Room room(const FfProduct& p) {
  if (p.M == 0) return {0, 0};
  if (p.type != CCT_TYPE_F32) return {0, ff_tile_plan(p).part_bytes};
  const FfF32Plan plan = ff_f32_plan(p);
  return {plan.pack_bytes, plan.part_bytes};
}
Room larger(const Room& a, const Room& b) { return {std::max(a.pack, b.pack), std::max(a.part, b.part)}; }

// out (rows x cols) = sum over segments of A_s B_s^T, rounded, nothing else
FfProduct plain_product(int type, int rows, int cols, int k, bool a_across, bool b_across, void* out, long long ldo) {
  FfProduct p = {};
  p.M = rows;
  p.N = cols;
  p.K = k;
  p.type = type;
  p.a_across = a_across;
  p.b_across = b_across;
  p.segments = 1;
  p.epilogue = kFfLinear;
  p.activation = CCT_ACT_NONE;
  p.out = out;
  p.ldo = ldo;
  return p;
}
// Whether a forward product runs on ff_rows.hip wherever its operands lie (see few_rows): they are not copied then.
bool always_rows(int M, int N, int type) {
  return ff_rows_fits(N, type) && M <= (type == CCT_TYPE_F32 ? kFfRowsF32 : kFfRows);
}
// Room for a forward product, whichever kernel takes it.
Room forward_room(int type, int M, int N, int K, FfEpilogue epilogue) {
  if (always_rows(M, N, type)) return {0, ff_rows_part_bytes(M, N, K, type, epilogue)};
  FfProduct p = plain_product(type, M, N, K, false, false, nullptr, 0);
  p.epilogue = epilogue;
  const Room r = room(p);
  return {r.pack, std::max(r.part, ff_rows_part_bytes(M, N, K, type, epilogue))};
}

// The products of a backward pass, with their results' places and nothing else yet; their number.
int linear_gradients(const cct_linear_desc_t& d, void* dx, long long lddx, void* dw, long long lddw, FfProduct* p) {
  int count = 0;
  if (d.M > 0) p[count++] = plain_product(d.type, d.M, d.K, d.N, false, true, dx, lddx);
  p[count++] = plain_product(d.type, d.N, d.K, d.M, true, true, dw, lddw);
  return count;
}
int gated_gradients(const cct_gated_desc_t& d, void* dx, long long lddx, void* dwg, long long lddwg, void* dwu, long long lddwu,
                    FfProduct* p) {
  int count = 0;
  if (d.M > 0) {
    p[count] = plain_product(d.type, d.M, d.K, d.F, false, true, dx, lddx);
    p[count++].segments = 2;
  }
  p[count++] = plain_product(d.type, d.F, d.K, d.M, true, true, dwg, lddwg);
  p[count++] = plain_product(d.type, d.F, d.K, d.M, true, true, dwu, lddwu);
  return count;
}
// Room for them in one launch, or one after the other.
Room backward_room(const FfProduct* p, int count) {
  Room r = {0, p[0].type == CCT_TYPE_F32 ? 0 : ff_together_plan(p, count).part_bytes};
  for (int i = 0; i < count; ++i) r = larger(r, room(p[i]));
  return r;
}

struct LinearLayout {
  long long x, w, dz, sums, pack, part, ld, total;
};
LinearLayout linear_layout(const cct_linear_desc_t& d, bool backward) {
  Layout l;
  LinearLayout b;
  const bool copies = backward || !always_rows(d.M, d.N, d.type);
  b.x = l.take(copies ? copy_bytes(d.M, d.K, d.type) : 0);
  b.w = l.take(copies ? copy_bytes(d.N, d.K, d.type) : 0);
  b.ld = up(d.N, 8);
  b.dz = l.take(backward ? (long long)d.M * b.ld * type_bytes(d.type) : 0);
  b.sums = l.take(backward ? (long long)ff_sum_rows(d.M, d.N) * d.N * 4 : 0);
  FfProduct p[2];
  const Room r = backward ? backward_room(p, linear_gradients(d, nullptr, 0, nullptr, 0, p)) : forward_room(d.type, d.M, d.N, d.K, kFfLinear);
  b.pack = l.take(r.pack);
  b.part = l.take(r.part);
  b.total = std::max(l.total, 256LL);
  return b;
}
struct GatedLayout {
  long long x, wg, wu, dg, du, pack, part, ld, total;
};
GatedLayout gated_layout(const cct_gated_desc_t& d, bool backward) {
  Layout l;
  GatedLayout b;
  const bool copies = backward || !always_rows(d.M, d.F, d.type);
  b.x = l.take(copies ? copy_bytes(d.M, d.K, d.type) : 0);
  b.wg = l.take(copies ? copy_bytes(d.F, d.K, d.type) : 0);
  b.wu = l.take(copies ? copy_bytes(d.F, d.K, d.type) : 0);
  b.ld = up(d.F, 8);
  b.dg = l.take(backward ? (long long)d.M * b.ld * type_bytes(d.type) : 0);
  b.du = l.take(backward ? (long long)d.M * b.ld * type_bytes(d.type) : 0);
  FfProduct p[3];
  const Room r = backward ? backward_room(p, gated_gradients(d, nullptr, 0, nullptr, 0, nullptr, 0, p))
                          : forward_room(d.type, d.M, d.F, d.K, kFfGated);
  b.pack = l.take(r.pack);
  b.part = l.take(r.part);
  b.total = std::max(l.total, 256LL);
  return b;
}

// Whether a forward product runs on ff_rows.hip.  4096 -> 4096, other weights in every call, us there and in tiles, bf16: 2 rows
// 9.0 and 11.5, 16 rows 11.5 and 12.0, 32 rows 15.2 and 12.2, 64 rows 22.9 and 12.9; but tiles may need a copy of the weight
// first (three times its bytes): 64 rows 26 and 31.  Rows that begin between multiples of four bytes: 16 rows 25.5 and 29, 32
// rows 39.5 and 30.5, so that more than 16 are copied.  fp32: 16 rows 20.3 and 32.7, 32 rows 29.4 and 33.9 (16384 outputs
// 102 and 97).
bool few_rows(int M, int N, int type, bool in_place, bool words) {
  return always_rows(M, N, type) || (type != CCT_TYPE_F32 && ff_rows_fits(N, type) && M <= kFfRowsMost && words && !in_place);
}

void add_copy(const Matrix& m, long long rows, long long cols, int type, void* to, Matrix* use, FfDzJobs* jobs) {
  *use = {to, up(cols, 8)};
  jobs->job[jobs->count++] = {(int)rows, (int)cols, type, CCT_ACT_NONE, m.p, nullptr, m.ld, 0, to, use->ld, nullptr, nullptr};
}
// The matrix itself, or where its copy at `to` will be, added to the jobs, if the products do not take it in place.
void operand(const Matrix& m, long long rows, long long cols, int type, void* to, Matrix* use, FfDzJobs* jobs) {
  *use = {m.p, rows <= 1 ? up(cols, 8) : m.ld};
  if (type != CCT_TYPE_F32 && rows > 0 && !ff_in_place(use->p, use->ld, cols)) add_copy(m, rows, cols, type, to, use, jobs);
}
// Two weights that one product takes must have the same strides.
void weight_pair(const Matrix& g, const Matrix& u, long long rows, long long cols, int type, char* to_g, char* to_u, Matrix* use_g,
                 Matrix* use_u, FfDzJobs* jobs) {
  operand(g, rows, cols, type, to_g, use_g, jobs);
  operand(u, rows, cols, type, to_u, use_u, jobs);
  if (type == CCT_TYPE_F32 || use_g->ld == use_u->ld) return;
  if (use_g->p != to_g) add_copy(g, rows, cols, type, to_g, use_g, jobs);
  if (use_u->p != to_u) add_copy(u, rows, cols, type, to_u, use_u, jobs);
}

}  // namespace
}  // namespace cct

using namespace cct;

extern "C" {

int cct_linear_workspace_bytes(const cct_linear_desc_t* desc, int32_t backward, size_t* bytes) {
  if (!desc || !bytes) return CCT_EINVAL;
  const cct_linear_desc_t& d = *desc;
  const int rc = dims_ok(d.M, d.N, d.K, d.type, d.activation);
  if (rc != CCT_OK) return rc;
  *bytes = (size_t)linear_layout(d, backward != 0).total;
  return CCT_OK;
}

int cct_gated_workspace_bytes(const cct_gated_desc_t* desc, int32_t backward, size_t* bytes) {
  if (!desc || !bytes) return CCT_EINVAL;
  const cct_gated_desc_t& d = *desc;
  const int rc = dims_ok(d.M, d.F, d.K, d.type, d.activation);
  if (rc != CCT_OK) return rc;
  *bytes = (size_t)gated_layout(d, backward != 0).total;
  return CCT_OK;
}

int cct_linear_forward(const cct_linear_desc_t* desc, const void* x, int64_t ldx, const void* w, int64_t ldw,
                       const void* bias, const void* residual, int64_t ldr, void* y, int64_t ldy, void* z, int64_t ldz,
                       void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (!desc) return CCT_EINVAL;
  const cct_linear_desc_t& d = *desc;
  int rc = dims_ok(d.M, d.N, d.K, d.type, d.activation);
  if (rc != CCT_OK) return rc;
  if (d.M == 0) return CCT_OK;
  if (!matrix_ok({x, ldx}, d.M, d.K, d.type) || !matrix_ok({w, ldw}, d.N, d.K, d.type) ||
      !matrix_ok({y, ldy}, d.M, d.N, d.type) || !vector_ok(bias, d.type) ||
      (residual && !matrix_ok({residual, ldr}, d.M, d.N, d.type)) || (z && !matrix_ok({z, ldz}, d.M, d.N, d.type)))
    return CCT_EINVAL;
  const LinearLayout b = linear_layout(d, false);
  rc = workspace_ok(workspace, workspace_bytes, b.total);
  if (rc != CCT_OK) return rc;
  hipStream_t st = (hipStream_t)hip_stream;
  char* ws = (char*)workspace;
  const bool few = few_rows(d.M, d.N, d.type, ff_in_place(w, d.N <= 1 ? up(d.K, 8) : ldw, d.K),
                            ff_words({x, ldx}) && ff_words({w, ldw}));
  Matrix mx = {x, ldx}, mw = {w, ldw};
  if (!few) {
    FfDzJobs jobs = {};
    operand({x, ldx}, d.M, d.K, d.type, ws + b.x, &mx, &jobs);
    operand({w, ldw}, d.N, d.K, d.type, ws + b.w, &mw, &jobs);
    FfBiasSum none;
    rc = launch_ff_dz(jobs, &none, st);
    if (rc != CCT_OK) return rc;
  }
  FfProduct p = plain_product(d.type, d.M, d.N, d.K, false, false, y, ldy);
  p.A[0] = mx;
  p.B[0] = mw;
  p.activation = d.activation;
  p.bias = bias;
  p.residual = residual;
  p.ldr = ldr;
  p.z = z;
  p.ldz = ldz;
  return few ? launch_ff_rows(p, (float*)(ws + b.part), st) : launch_ff_product(p, ws + b.pack, (float*)(ws + b.part), st);
}

int cct_linear_backward(const cct_linear_desc_t* desc, const void* x, int64_t ldx, const void* w, int64_t ldw,
                        const void* z, int64_t ldz, const void* dy, int64_t lddy, void* dx, int64_t lddx, void* dw,
                        int64_t lddw, void* dbias, void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (!desc) return CCT_EINVAL;
  const cct_linear_desc_t& d = *desc;
  int rc = dims_ok(d.M, d.N, d.K, d.type, d.activation);
  if (rc != CCT_OK) return rc;
  const bool act = d.activation != CCT_ACT_NONE;
  // an empty batch's tensors have no address; gradients of weights are written all the same
  if (d.M > 0 && ((dw && !matrix_ok({x, ldx}, d.M, d.K, d.type)) || (act && !matrix_ok({z, ldz}, d.M, d.N, d.type)) ||
                  !matrix_ok({dy, lddy}, d.M, d.N, d.type) || (dx && !matrix_ok({w, ldw}, d.N, d.K, d.type)) ||
                  (dx && !matrix_ok({dx, lddx}, d.M, d.K, d.type))))
    return CCT_EINVAL;
  if ((dw && !matrix_ok({dw, lddw}, d.N, d.K, d.type)) || !vector_ok(dbias, d.type)) return CCT_EINVAL;
  const LinearLayout b = linear_layout(d, true);
  rc = workspace_ok(workspace, workspace_bytes, b.total);
  if (rc != CCT_OK) return rc;
  hipStream_t st = (hipStream_t)hip_stream;
  char* ws = (char*)workspace;
  // dy itself is dz without an activation, where the products take it in place
  const bool copy = (dx || dw) && (act || (d.type != CCT_TYPE_F32 && !ff_in_place(dy, d.M <= 1 ? b.ld : lddy, d.N)));
  FfDzJobs jobs = {};
  if (copy || dbias)
    jobs.job[jobs.count++] = {d.M, d.N, d.type, d.activation, dy, act ? z : nullptr, lddy, ldz, copy ? ws + b.dz : nullptr, b.ld,
                              dbias, (float*)(ws + b.sums)};
  Matrix mx = {}, mw = {};
  if (dx && d.M > 0) operand({w, ldw}, d.N, d.K, d.type, ws + b.w, &mw, &jobs);
  if (dw) operand({x, ldx}, d.M, d.K, d.type, ws + b.x, &mx, &jobs);
  FfBiasSum sum;
  rc = launch_ff_dz(jobs, &sum, st);
  if (rc != CCT_OK) return rc;
  const Matrix dz = {copy ? ws + b.dz : dy, copy || d.M <= 1 ? b.ld : lddy};
  FfProduct p[2];
  const int count = linear_gradients(d, dx, lddx, dw, lddw, p);
  for (int i = 0; i < count; ++i) {
    p[i].A[0] = dz;
    p[i].B[0] = i == count - 1 ? mx : mw;
  }
  return launch_ff_products(p, count, sum, ws + b.pack, (float*)(ws + b.part), st);
}

int cct_gated_forward(const cct_gated_desc_t* desc, const void* x, int64_t ldx, const void* wg, int64_t ldwg,
                      const void* wu, int64_t ldwu, void* h, int64_t ldh, void* g, int64_t ldg, void* u, int64_t ldu,
                      void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (!desc) return CCT_EINVAL;
  const cct_gated_desc_t& d = *desc;
  int rc = dims_ok(d.M, d.F, d.K, d.type, d.activation);
  if (rc != CCT_OK) return rc;
  if (d.M == 0) return CCT_OK;
  if (!matrix_ok({x, ldx}, d.M, d.K, d.type) || !matrix_ok({wg, ldwg}, d.F, d.K, d.type) ||
      !matrix_ok({wu, ldwu}, d.F, d.K, d.type) || !matrix_ok({h, ldh}, d.M, d.F, d.type) || (!g != !u) ||
      (g && (!matrix_ok({g, ldg}, d.M, d.F, d.type) || !matrix_ok({u, ldu}, d.M, d.F, d.type))))
    return CCT_EINVAL;
  const GatedLayout b = gated_layout(d, false);
  rc = workspace_ok(workspace, workspace_bytes, b.total);
  if (rc != CCT_OK) return rc;
  hipStream_t st = (hipStream_t)hip_stream;
  char* ws = (char*)workspace;
  const bool in_place = ff_in_place(wg, d.F <= 1 ? up(d.K, 8) : ldwg, d.K) && ff_in_place(wu, d.F <= 1 ? up(d.K, 8) : ldwu, d.K) &&
                        ldwg == ldwu;
  const bool few = few_rows(d.M, d.F, d.type, in_place, ff_words({x, ldx}) && ff_words({wg, ldwg}) && ff_words({wu, ldwu}));
  Matrix mx = {x, ldx}, mg = {wg, ldwg}, mu = {wu, ldwu};
  if (!few) {
    FfDzJobs jobs = {};
    operand({x, ldx}, d.M, d.K, d.type, ws + b.x, &mx, &jobs);
    weight_pair({wg, ldwg}, {wu, ldwu}, d.F, d.K, d.type, ws + b.wg, ws + b.wu, &mg, &mu, &jobs);
    FfBiasSum none;
    rc = launch_ff_dz(jobs, &none, st);
    if (rc != CCT_OK) return rc;
  }
  FfProduct p = plain_product(d.type, d.M, d.F, d.K, false, false, h, ldh);
  p.epilogue = kFfGated;
  p.activation = d.activation;
  p.A[0] = mx;
  p.B[0] = mg;
  p.B[1] = mu;
  p.z = g;
  p.ldz = ldg;
  p.z2 = u;
  p.ldz2 = ldu;
  return few ? launch_ff_rows(p, (float*)(ws + b.part), st) : launch_ff_product(p, ws + b.pack, (float*)(ws + b.part), st);
}

int cct_gated_backward(const cct_gated_desc_t* desc, const void* x, int64_t ldx, const void* wg, int64_t ldwg,
                       const void* wu, int64_t ldwu, const void* g, int64_t ldg, const void* u, int64_t ldu,
                       const void* dh, int64_t lddh, void* dx, int64_t lddx, void* dwg, int64_t lddwg, void* dwu,
                       int64_t lddwu, void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (!desc) return CCT_EINVAL;
  const cct_gated_desc_t& d = *desc;
  int rc = dims_ok(d.M, d.F, d.K, d.type, d.activation);
  if (rc != CCT_OK) return rc;
  if (!dwg != !dwu) return CCT_EINVAL;
  if (d.M > 0 && ((dwg && !matrix_ok({x, ldx}, d.M, d.K, d.type)) || !matrix_ok({g, ldg}, d.M, d.F, d.type) ||
                  !matrix_ok({u, ldu}, d.M, d.F, d.type) || !matrix_ok({dh, lddh}, d.M, d.F, d.type) ||
                  (dx && (!matrix_ok({wg, ldwg}, d.F, d.K, d.type) || !matrix_ok({wu, ldwu}, d.F, d.K, d.type) ||
                          !matrix_ok({dx, lddx}, d.M, d.K, d.type)))))
    return CCT_EINVAL;
  if (dwg && (!matrix_ok({dwg, lddwg}, d.F, d.K, d.type) || !matrix_ok({dwu, lddwu}, d.F, d.K, d.type))) return CCT_EINVAL;
  const GatedLayout b = gated_layout(d, true);
  rc = workspace_ok(workspace, workspace_bytes, b.total);
  if (rc != CCT_OK) return rc;
  if (!dx && !dwg) return CCT_OK;
  hipStream_t st = (hipStream_t)hip_stream;
  char* ws = (char*)workspace;
  const Matrix dg = {ws + b.dg, b.ld}, du = {ws + b.du, b.ld};
  FfDzJobs jobs = {};
  Matrix mx = {}, mg = {}, mu = {};
  if (dx && d.M > 0) weight_pair({wg, ldwg}, {wu, ldwu}, d.F, d.K, d.type, ws + b.wg, ws + b.wu, &mg, &mu, &jobs);
  if (dwg) operand({x, ldx}, d.M, d.K, d.type, ws + b.x, &mx, &jobs);
  rc = launch_ff_gated_dz({d.M, d.F, d.type, d.activation, dh, g, u, lddh, ldg, ldu, ws + b.dg, ws + b.du, b.ld}, jobs, st);
  if (rc != CCT_OK) return rc;
  FfProduct p[3];
  const int count = gated_gradients(d, dx, lddx, dwg, lddwg, dwu, lddwu, p);
  if (d.M > 0) {
    p[0].A[0] = dg;
    p[0].A[1] = du;
    p[0].B[0] = mg;
    p[0].B[1] = mu;
  }
  for (int i = count - 2; i < count; ++i) {
    p[i].A[0] = i == count - 2 ? dg : du;
    p[i].B[0] = mx;
  }
  return launch_ff_products(p, count, {}, ws + b.pack, (float*)(ws + b.part), st);
}

}  // extern "C"
