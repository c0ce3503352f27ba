// The microscaled 4-bit operators' entry points (cct_mx_*): checks of arguments, workspaces, and which kernels a product runs on.
#include "mx.h"

#include <algorithm>

#include "activation.h"
#include "number_types.h"

namespace cct {
namespace {

bool rows_ok(const void* p, long long ld, long long rows, long long cols, int align) {
  return p && !((uintptr_t)p & (align - 1)) && ld >= 0 && (rows <= 1 || ld >= cols);
}
bool matrix_ok(const void* p, long long ld, long long rows, long long cols, int type) { return rows_ok(p, ld, rows, cols, type_bytes(type)); }
bool mx_ok(const void* codes, long long ldc, const void* scales, long long lds, int rows, int cols) {
  return rows_ok(codes, ldc, rows, mx_code_bytes(cols), 16) && ldc % 16 == 0 && rows_ok(scales, lds, rows, mx_scale_bytes(cols), 4) &&
         lds % 4 == 0;
}
// As the 16- and 32-bit products' sizes; codes are smaller.
int sizes_ok(int rows, int cols, int type) {
  if (rows < 0 || cols < 1 || !type_known(type)) return CCT_EINVAL;
  return std::max(rows, cols) <= 0x7fffff00 && (long long)rows * cols <= (1LL << 38) / type_bytes(type) ? CCT_OK : CCT_EUNSUPPORTED;
}
int product_ok(const cct_linear_desc_t& d) {
  if (d.N < 1 || !activation_known(d.activation)) return CCT_EINVAL;
  const int a = sizes_ok(d.M, d.K, d.type), b = sizes_ok(d.N, d.K, d.type), c = sizes_ok(d.M, d.N, d.type);
  return a != CCT_OK ? a : b != CCT_OK ? b : c;
}

struct MxLayout {
  long long codes, scales, part, total;
};
MxLayout layout_of(const cct_linear_desc_t& d, bool quantize) {
  MxLayout b = {};
  auto take = [&](long long bytes) {
    const long long at = b.total;
    b.total += (bytes + 255) / 256 * 256;
    return at;
  };
  b.codes = take(quantize ? d.M * mx_code_bytes(d.K) : 0);
  b.scales = take(quantize ? d.M * mx_scale_bytes(d.K) : 0);
  b.part = take(d.M > 0 ? mx_plan(d.M, d.N, d.K).part_bytes : 0);
  b.total = std::max(b.total, 256LL);
  return b;
}

}  // namespace

namespace {

constexpr int kCus = 256;
// A tile: its workgroups on a CU, and us a stage takes where the CUs are full of them, and one alone, measured on products of 64 to 8192
// rows.  Stages of small tiles are mostly waiting, so that they do best where no CU has many (256 x 4096 x 4096: in tiles of 128 18 us, of
// 64 x 128 12, of 64 10, and 9.5 with four stages; 48 x 16384 x 4096: 17.6, 14.0, 12.2 and 9.6; 8192 x 8192 x 8192: 348, 436, 524 and 576).
struct MxTileCost {
  int tile;
  bool deep;
  int bm, bn, threads, per_cu;
  double full, alone, around;  // what stands around a contraction, in stages
};
constexpr MxTileCost kMxTiles[] = {{kTile256, false, 256, 256, 512, 1, 2.2, 1.9, 2},
                                   {kTile128, false, 128, 128, 256, 2, 1.35, 0.95, 2},
                                   {kTile64x128, false, 64, 128, 256, 3, 1.25, 0.6, 2},
                                   {kTile64, false, 64, 64, 256, 4, 1.02, 0.5, 2},
                                   {kTile64, true, 64, 64, 256, 2, 0.56, 0.36, 4}};
constexpr double kLaunchMicros = 3.0, kJoinMicros = 3.0, kJoinBytesPerMicro = 3.0e6;

// Few columns of long rows leave most CUs idle: splits of 32 steps (a turn of a workgroup's waves) or more.
MxPlan rows_plan(int M, int N, int K) {
  const int steps = pieces(mx_blocks(K), 4);
  MxPlan plan = {kNoTile, 1, steps, false, 0};
  const long long groups = (long long)pieces(N, 16) * pieces(M, M <= 16 ? 16 : M <= 32 ? 32 : 64);
  if (groups <= 64 && steps >= 128) {
    const int splits = (int)std::min(128 / groups, steps / 32LL);
    plan.steps = pieces(steps, splits);
    plan.splits = pieces(steps, plan.steps);
  }
  return plan;
}
// us of it: the weight from memory, or both operands of every workgroup of 16 columns from L2 (48 x 16384 x 4096: 27, in tiles of
// 64 x 128 14), or what a turn takes at least, or a workgroup itself (6148 x 2954 x 16: 18 000 of them 181, in tiles 26).
double rows_micros(int M, int N, int K, const MxPlan& plan) {
  const double row = K * 17.0 / 32, wide = pieces(N, 16), high = pieces(M, 64);
  const double bytes = wide * (16 * high + M) * row;
  const int blocks = M <= 16 ? 1 : M <= 32 ? 2 : 4;
  const double turns = (M <= 16 ? 1.0 : M <= 32 ? 2.0 : 3.2) * pieces(plan.steps, 32);
  const double each = 0.002 * (1 + blocks) * wide * pieces(M, 16 * blocks);
  const double us = std::max(std::max(2.0 + (double)N * row / 5.0e6, 3.0 + each), 4.5 + std::max(bytes / 7.5e6, turns));
  return us + (plan.splits > 1 ? kJoinMicros : 0.0);
}

}  // namespace

MxPlan mx_plan(int M, int N, int K) {
  MxPlan best = rows_plan(M, N, K);
  double least = rows_micros(M, N, K, best);
  const int stages = pieces(mx_blocks(K), 8);
  for (const MxTileCost& c : kMxTiles) {
    const long long tiles = (long long)pieces(M, c.bm) * pieces(N, c.bn);
    for (int splits = 1; splits <= (c.tile == kTile256 ? 1 : 16) && splits <= std::max(1, stages / 4); ++splits) {
      const int each = pieces(stages, splits), have = pieces(stages, each);
      const long long groups = tiles * have, slots = (long long)kCus * c.per_cu, rest = groups % slots;
      if (groups * c.threads > kMostThreads) continue;
      const double last = rest == 0 ? 0.0 : rest <= kCus ? c.alone : c.full;
      double us = ((double)(groups / slots) * c.full + last) * (each + c.around) + kLaunchMicros;
      if (mx_quantizes(M, N, K)) us += kLaunchMicros;  // of x's codes, if it has none yet: the choice is the same for both
      if (have > 1) us += kJoinMicros + 8.0 * have * M * N / kJoinBytesPerMicro;
      if (us < least) {
        least = us;
        best = {c.tile, have, each, c.deep, 0};
      }
    }
  }
  if (best.splits > 1) best.part_bytes = 4LL * best.splits * M * ((N + 3) / 4 * 4);
  return best;
}

}  // namespace cct

using namespace cct;

extern "C" {

int cct_mx_quantize(int32_t rows, int32_t cols, int32_t type, const void* x, int64_t ldx, void* codes, int64_t ld_codes,
                    void* scales, int64_t ld_scales, void* hip_stream) {
  const int rc = sizes_ok(rows, cols, type);
  if (rc != CCT_OK || rows == 0) return rc;
  if (!matrix_ok(x, ldx, rows, cols, type) || !mx_ok(codes, ld_codes, scales, ld_scales, rows, cols)) return CCT_EINVAL;
  return launch_mx_quantize(rows, cols, type, x, ldx, (unsigned char*)codes, ld_codes, (unsigned char*)scales, ld_scales,
                            (hipStream_t)hip_stream);
}

int cct_mx_dequantize(int32_t rows, int32_t cols, int32_t type, const void* codes, int64_t ld_codes, const void* scales,
                      int64_t ld_scales, void* x, int64_t ldx, void* hip_stream) {
  const int rc = sizes_ok(rows, cols, type);
  if (rc != CCT_OK || rows == 0) return rc;
  if (!matrix_ok(x, ldx, rows, cols, type) || !mx_ok(codes, ld_codes, scales, ld_scales, rows, cols)) return CCT_EINVAL;
  return launch_mx_dequantize(rows, cols, type, {(const unsigned char*)codes, ld_codes, (const unsigned char*)scales, ld_scales}, x,
                              ldx, (hipStream_t)hip_stream);
}

int cct_mx_linear_workspace_bytes(const cct_linear_desc_t* desc, int32_t quantize, size_t* bytes) {
  if (!desc || !bytes) return CCT_EINVAL;
  const int rc = product_ok(*desc);
  if (rc != CCT_OK) return rc;
  *bytes = (size_t)layout_of(*desc, quantize != 0).total;
  return CCT_OK;
}

int cct_mx_linear_forward(const cct_linear_desc_t* desc, const void* x, int64_t ldx, const void* x_scales, int64_t ldxs,
                          const void* w, int64_t ldw, const void* w_scales, int64_t ldws, const void* bias,
                          const void* residual, int64_t ldr, void* y, int64_t ldy, void* z, int64_t ldz, void* workspace,
                          size_t workspace_bytes, void* hip_stream) {
  if (!desc) return CCT_EINVAL;
  const cct_linear_desc_t& d = *desc;
  int rc = product_ok(d);
  if (rc != CCT_OK) return rc;
  if (d.M == 0) return CCT_OK;
  const bool quantize = !x_scales;
  if (quantize ? !matrix_ok(x, ldx, d.M, d.K, d.type) : !mx_ok(x, ldx, x_scales, ldxs, d.M, d.K)) return CCT_EINVAL;
  if (!mx_ok(w, ldw, w_scales, ldws, d.N, d.K) || !matrix_ok(y, ldy, d.M, d.N, d.type) || ((uintptr_t)bias & (type_bytes(d.type) - 1)) ||
      (residual && !matrix_ok(residual, ldr, d.M, d.N, d.type)) || (z && !matrix_ok(z, ldz, d.M, d.N, d.type)))
    return CCT_EINVAL;
  const MxLayout b = layout_of(d, quantize);
  if (!workspace || ((uintptr_t)workspace & 255)) return CCT_EINVAL;
  if (workspace_bytes < (size_t)b.total) return CCT_EWORKSPACE;
  hipStream_t st = (hipStream_t)hip_stream;
  unsigned char* ws = (unsigned char*)workspace;
  MxPlan plan = mx_plan(d.M, d.N, d.K);
  MxProduct a = {};
  a.blocks = mx_blocks(d.K);
  a.w = {(const unsigned char*)w, ldw, (const unsigned char*)w_scales, ldws};
  a.x = {(const unsigned char*)x, ldx, (const unsigned char*)x_scales, ldxs};
  a.quantize = quantize && plan.tile == kNoTile && mx_quantizes(d.M, d.N, d.K);
  if (quantize && !a.quantize) {
    a.x = {ws + b.codes, mx_code_bytes(d.K), ws + b.scales, mx_scale_bytes(d.K)};
    rc = launch_mx_quantize(d.M, d.K, d.type, x, ldx, ws + b.codes, a.x.ldc, ws + b.scales, a.x.lds, st);
    if (rc != CCT_OK) return rc;
  }
  // a tile's offsets have 32 bits, of 256 rows
  constexpr long long kMost = 1 << 23;
  if (plan.tile != kNoTile && std::max(std::max(a.x.ldc, a.w.ldc), std::max(a.x.lds, a.w.lds)) >= kMost) plan = {kNoTile, 1, 0, false, 0};
  FfProduct& p = a.p;
  p.M = d.M;
  p.N = d.N;
  p.K = d.K;
  p.type = d.type;
  p.activation = d.activation;
  p.segments = 1;
  p.epilogue = kFfLinear;
  p.bias = bias;
  p.residual = residual;
  p.ldr = ldr;
  p.out = y;
  p.ldo = ldy;
  p.z = z;
  p.ldz = ldz;
  return plan.tile == kNoTile ? launch_mx_rows(a, plan, (float*)(ws + b.part), st) : launch_mx_tile(a, plan, (float*)(ws + b.part), st);
}

}  // extern "C"
