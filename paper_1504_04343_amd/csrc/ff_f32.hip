// The fp32 products of the feed-forward operators, on the bf16 matrix cores as sums of three terms (gemm_split.hip), which is
// as exact as fp32 instructions and faster.
//
// The rows' operand (x of a forward product, dz or its transpose in a backward one) is packed or split in place, the other
// one is read in place, along or across the contraction.  The contraction may be cut into splits, and two contractions
// (dx of a gated block) may be summed; then, and where an activation, a residual or z follow, the sums go through the
// workspace and ff_join_kernel finishes them: 8 to 12 bytes per result against 2 K operations (4096 x 4096 x 4096: 27 of
// 690 us).
//
// Strides that gemm_split cannot address (2^22 values and more) and empty contractions run on ff_general_kernel.
#include <algorithm>
#include <cstring>

#include "ff_tile.h"

namespace cct {
namespace {

constexpr int kIntMax = 2147483647;
constexpr long long kMostPack = 1LL << 30;  // bytes; more rows run one part after the other
constexpr int kLeastSplit = 256;            // steps of the contraction

GemmTN split_problem(int M, int N, int K, int splits) {
  GemmTN t;
  std::memset(&t, 0, sizeof(t));
  t.M = M;
  t.Mpad = gemm_split_mpad(M);
  t.Ncols = N;
  t.Kdim = K;
  t.Kpad = gemm_split_kpad(K);
  t.G = splits;
  t.bmap = t.cmap = ColMap{kIntMax, 0};
  return t;
}

bool fits(const FfF32Plan& plan, int N, long long ldb, bool along) {
  GemmTN t = split_problem(plan.rows, N, plan.len, plan.splits);
  t.b_ks = ldb;
  return gemm_split_fits(t, along);
}

}  // namespace

FfF32Plan ff_f32_plan(const FfProduct& p) {
  const int M = p.M, N = p.N, K = p.K, planes = p.epilogue == kFfGated ? 2 : p.segments;
  const bool along = !p.b_across;
  FfF32Plan best = {1, K, M, 0, 0, {1, 0, 0}};
  const long long ld = (N + 3) / 4 * 4;
  if (M > 0 && K > 0) {
    double least = 1e30;
    const long long kpad = gemm_split_kpad(K);
    best.rows = (int)std::min<long long>(M, std::max(64LL, kMostPack / (6 * kpad) / 64 * 64));
    // in tiles of 32 x 128 at the least, one launch
    while (best.rows > 32 && (best.rows + 31LL) / 32 * ((N + 127LL) / 128) * 256 > kMostThreads)
      best.rows = std::max(32, best.rows / 2 / 64 * 64);
    for (int sp = 1; sp <= 32 && (sp == 1 || K >= sp * kLeastSplit); sp += sp < 8 ? 1 : 4) {
      const int len = sp == 1 ? K : gemm_split_kpad((K + sp - 1) / sp), n = pieces(K, len);
      const double t = gemm_split_seconds(along, true, best.rows, len, N, n) + (n > 1 ? 8.0 * n * best.rows * N / 5.5e12 + 2.5e-6 : 0.0);
      if (t >= least) continue;
      least = t;
      best.splits = n;
      best.len = len;
    }
    best.pack_bytes = 6LL * best.splits * gemm_split_mpad(best.rows) * gemm_split_kpad(best.len);
  }
  // a gradient of one contraction that is not cut is stored as it is; behind a forward product anything may follow
  best.part_bytes = p.b_across && planes * best.splits == 1 ? 0 : 4LL * best.splits * planes * M * ld;
  // rows so long that the split product does not address them wherever they lie
  if (M > 0 && K > 0 && !fits(best, N, along ? K : N, along)) {
    best.general = ff_general_plan(p);
    best.pack_bytes = 0;
    best.part_bytes = best.general.part_bytes;
  }
  return best;
}

int launch_ff_f32(const FfProduct& p, char* pack, float* ws, hipStream_t st) {
  const bool gated = p.epilogue == kFfGated, along = !p.b_across;
  const int products = gated ? 2 : p.segments;
  const FfF32Plan plan = ff_f32_plan(p);
  const bool join = plan.splits > 1 || products > 1 || p.residual || p.z || p.activation != CCT_ACT_NONE;
  const long long ld = join ? (p.N + 3) / 4 * 4 : p.ldo;
  for (int q = 0; q < products; ++q)
    if (p.K < 1 || !fits(plan, p.N, p.B[q].ld, along)) return launch_ff_general(p, plan.general, ws, st);
  for (long long m0 = 0; m0 < p.M; m0 += plan.rows) {
    GemmTN t = split_problem((int)std::min<long long>(plan.rows, p.M - m0), p.N, plan.len, plan.splits);
    for (int q = 0; q < products; ++q) {
      const FfOperand &A = p.A[gated ? 0 : q], &B = p.B[q];
      t.B = B.p;
      t.b_ks = B.ld;
      t.b_gs = plan.len * ff_step(B, !along);
      t.b_len = along ? (p.N - 1) * B.ld + p.K : (p.K - 1) * B.ld + p.N;
      if (q == 0 || !gated) {  // a gated block's products have the same rows
        const long long row = ff_row(A, p.a_across), step = ff_step(A, p.a_across);
        const int rc = gemm_split_operand(&t, along, (const float*)A.p + m0 * row, pack, p.K, row, step, plan.len * step, 1, st);
        if (rc != CCT_OK) return rc;
      }
      t.c_ms = ld;
      if (join) {
        t.C = ws + ((gated ? q : (long long)q * plan.splits) * p.M + m0) * ld;
        t.c_gs = (gated ? 2LL : 1LL) * p.M * ld;
      } else {
        t.C = (float*)p.out + m0 * ld;
        t.bias = (const float*)p.bias;
        t.bias_gs = -1;
      }
      const int rc = launch_gemm_split(t, p.K, along, st);
      if (rc != CCT_OK) return rc;
    }
  }
  if (!join) return CCT_OK;
  const FfPart part = {ws, (int)ld, plan.splits * (gated ? 1 : products), 0};
  const double mn = (double)p.M * p.N;
  ProfScope ps("ff_join_kernel", mn * plan.splits * products,
               4.0 * mn * (plan.splits * products + 1 + (p.residual != nullptr) + (p.z != nullptr) + (p.z2 != nullptr)), st);
  if (gated)
    launch_join<CCT_TYPE_F32, kFfGated>(p, part, st);
  else
    launch_join<CCT_TYPE_F32, kFfLinear>(p, part, st);
  CCT_CHECK_LAUNCH();
  return CCT_OK;
}

}  // namespace cct
