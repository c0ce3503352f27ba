// How the matrix products of the feed-forward operators are cut into tiles and splits (16-bit types: ff_tile.h; fp32:
// ff_f32.hip).
#include <algorithm>

#include "ff_bias_sum.h"

namespace cct {
namespace {

// Microseconds of a stage (64 steps of the contraction) with one workgroup on a CU and with as many as fit, forward and with
// operands across the contraction (whose LDS reads are twice as many), measured on products of 512 to 8192 rows.
struct TileCost {
  int bm, bn, per_cu, threads;
  double alone[2], full[2];
};
constexpr TileCost kTileCosts[] = {{256, 256, 1, 512, {1.58, 1.65}, {1.58, 1.70}},
                                   {192, 256, 1, 512, {1.24, 1.30}, {1.24, 1.34}},
                                   {128, 128, 2, 256, {0.65, 0.93}, {1.10, 1.08}},
                                   {64, 128, 2, 256, {0.39, 0.75}, {0.72, 0.83}},
                                   {64, 64, 2, 256, {0.29, 0.50}, {0.54, 0.60}}};
constexpr double kJoinMicros = 4.0, kJoinBytesPerMicro = 7.5e6;  // a launch and its gap; partial sums, written and read
constexpr int kCus = 256, kLeastStages = 4;                       // of a split
// What stands around a contraction, in stages: two tell tiles of short contractions of backward products apart (linear 4000 x
// 200 x 9000 91 -> 82 us, 77 x 14144 x 9696 226 -> 211; one and three 82 and 227, 82 and 211), forward ones gain nothing.
constexpr int kAround = 2;
constexpr double kLaunchMicros = 3.0, kBytesPerMicro = 5.0e6;  // operands, from memory

// Whether a tile's loads reach the operands.  A lane's offset from its tile's first row, or from its stage's first step, is 32
// bits, and what lies 2^31 bytes behind that is taken for what lies behind the operand.  Matrices in place always are reached
// (ff_in_place); rows of a copy, and of dz, are as far apart as they are long, so that 128 rows of 2^24 steps are not.
bool reaches(const FfProduct& p, const TileCost& c) {
  constexpr long long most = 1LL << 30;  // 16-bit values
  auto operand = [&](bool across, int rows, int tile) {
    const long long ld = ((across ? rows : p.K) + 7LL) / 8 * 8;
    if (!across) return (std::min(rows, tile) - 1) * ld + kFfStage <= most;
    // steps past the contraction's end may lie anywhere beyond it, if they do not come round to its beginning
    return (std::min(p.K, kFfStage) - 1) * ld + tile <= most && (kFfStage - 1) * ld + tile < 2 * most;
  };
  return operand(p.a_across, p.M, c.bm) && operand(p.b_across, p.N, p.epilogue == kFfGated ? c.bn / 2 : c.bn);
}

// The tile and the number of splits of the contraction with the least estimate: rounds of workgroups over the card times the
// stages of one, and what joining the splits costs.  Few large tiles leave CUs idle, small ones read LDS more often per
// product.  1024 x 4096 x 9216 (forward, bf16): 181 us in tiles of 256 (64 of them), 96 in 128, 82 in 128 and two splits.
// For M x N of the product's results.
FfTilePlan whole_plan(const FfProduct& p, int M, int N) {
  const bool along = !p.b_across;
  const int segments = p.epilogue == kFfGated ? 1 : p.segments;
  const long long cols = p.epilogue == kFfGated ? 2LL * N : N;
  const int stages = std::max(pieces(p.K, kFfStage), 1) * segments;
  const double bytes = 2.0 * (M + (double)cols) * p.K * segments;
  FfTilePlan best = {kNoTile, 1, stages, 0, 1e30, 0, 0};
  for (int tile = kTile256; tile <= kTile64; ++tile) {
    const TileCost& c = kTileCosts[tile];
    if (!reaches(p, c)) continue;
    const long long tiles = pieces(M, c.bm) * ((cols + c.bn - 1) / c.bn);
    if (tiles * c.threads > kMostThreads) continue;  // more than 2^30 rows of few columns in tiles of 64
    for (int splits = 1; splits <= 32; splits *= 2) {
      if (splits > 1 && (tile <= kTile192 || stages < splits * kLeastStages || tiles * splits > 4 * kCus)) break;
      const int each = (stages + splits - 1) / splits;
      const long long groups = tiles * splits, slots = (long long)kCus * c.per_cu, rest = groups % slots;
      double us = (double)(groups / slots) * c.full[!along] + (rest == 0 ? 0.0 : (rest <= kCus ? c.alone : c.full)[!along]);
      // (fewer workgroups than a third of the CUs' places do not keep memory busy)
      us = std::max(us * (each + (along ? 0 : kAround)), bytes / kBytesPerMicro * std::max(1.0, 170.0 / groups)) + kLaunchMicros;
      if (splits > 1) us += kJoinMicros + 8.0 * splits * M * cols / kJoinBytesPerMicro;
      if (us < best.micros) best = {tile, (stages + each - 1) / each, each, 0, us, 0, 0};
    }
  }
  if (best.tile == kNoTile) best.part_bytes = ff_general_plan(p).part_bytes;
  else if (best.splits > 1) best.part_bytes = 4LL * best.splits * M * (cols + 8);
  return best;
}

}  // namespace

// The same, or whole rounds of tiles of 256 and what is left of the columns or rows in a launch of its own: 17 x 16 tiles are
// two rounds, of which the second one is 16 workgroups (4160 columns of 4096 rows and steps: 187 us in tiles of
// 128, 133 so).
FfTilePlan ff_tile_plan(const FfProduct& p) {
  const int M = p.M, N = p.N;
  FfTilePlan best = whole_plan(p, M, N);
  const int wide = p.epilogue == kFfGated ? 128 : 256;
  const long long tm = pieces(M, 256), tn = pieces(N, wide), rounds = tm * tn / kCus;
  if (rounds < 1 || !reaches(p, kTileCosts[kTile256]) || tm * tn * kTileCosts[kTile256].threads > kMostThreads) return best;
  const int stages = std::max(pieces(p.K, kFfStage), 1) * (p.epilogue == kFfGated ? 1 : p.segments);
  const double full = rounds * stages * kTileCosts[kTile256].full[p.b_across] + kLaunchMicros;
  auto consider = [&](long long rows, long long cols) {  // what the full rounds take
    if ((rows < M) == (cols < N)) return;
    const FfTilePlan rest = rows < M ? whole_plan(p, M - (int)rows, N) : whole_plan(p, M, N - (int)cols);
    if (full + rest.micros >= best.micros) return;
    best = {kTile256, 1, stages, rest.part_bytes, full + rest.micros, rows < M ? (int)rows : 0, cols < N ? (int)cols : 0};
  };
  if (tm <= rounds * kCus) consider(M, rounds * kCus / tm * wide);
  if (tn <= rounds * kCus) consider(rounds * kCus / tn * 256, N);
  return best;
}

namespace {

// The results from row m and column n on, rows x cols of them.
FfProduct part_of(FfProduct p, int m, int n, int rows, int cols) {
  auto at = [&](const void* q, long long ld) { return q ? (void*)((char*)q + (m * ld + n) * 2) : nullptr; };
  for (int s = 0; s < 2; ++s) {
    if (p.A[s].p) p.A[s].p = (const char*)p.A[s].p + m * ff_row(p.A[s], p.a_across) * 2;
    if (p.B[s].p) p.B[s].p = (const char*)p.B[s].p + n * ff_row(p.B[s], p.b_across) * 2;
  }
  p.M = rows;
  p.N = cols;
  p.bias = p.bias ? (const char*)p.bias + n * 2LL : nullptr;
  p.residual = at(p.residual, p.ldr);
  p.out = at(p.out, p.ldo);
  p.z = at(p.z, p.ldz);
  p.z2 = at(p.z2, p.ldz2);
  return p;
}

const char* const kTileNames[] = {"256x256", "192x256", "128x128", "64x128", "64x64"};

int launch_tiles(const FfProduct& p, const FfTilePlan& plan, float* ws, hipStream_t st) {
  const double mn = (double)p.M * p.N, ops = p.epilogue == kFfGated ? 2 : p.segments;
  const double bytes = 2.0 * ((double)(p.epilogue == kFfGated ? 1 : p.segments) * p.M * p.K + ops * p.N * p.K +
                              mn * (1 + (p.residual != nullptr) + (p.z != nullptr) + (p.z2 != nullptr)));
  ProfScope ps(2.0 * mn * p.K * ops, bytes, st, "ff_tile_kernel<%s, %d splits>", kTileNames[plan.tile], plan.splits);
  return p.type == CCT_TYPE_BF16 ? launch_ff_tile_bf16(p, plan, ws, st) : launch_ff_tile_f16(p, plan, ws, st);
}

}  // namespace

int launch_ff_product(const FfProduct& p, char* pack, float* ws, hipStream_t st) {
  if (p.type == CCT_TYPE_F32) return launch_ff_f32(p, pack, ws, st);
  const FfTilePlan plan = ff_tile_plan(p);
  if (plan.tile == kNoTile) return launch_ff_general(p, ff_general_plan(p), ws, st);
  if (!plan.cut_rows && !plan.cut_cols) return launch_tiles(p, plan, ws, st);
  const int m = plan.cut_rows, n = plan.cut_cols;  // one of them is 0
  const int rc = launch_tiles(part_of(p, 0, 0, m ? m : p.M, n ? n : p.N), plan, ws, st);
  if (rc != CCT_OK) return rc;
  const FfProduct rest = part_of(p, m, n, p.M - m, p.N - n);
  return launch_tiles(rest, whole_plan(p, rest.M, rest.N), ws, st);
}

namespace {
int stages_of(const FfProduct& p) { return std::max(pieces(p.K, kFfStage), 1) * p.segments; }
double operand_bytes(const FfProduct& p) { return 2.0 * p.segments * p.K * ((double)p.M + p.N); }
}  // namespace

// The tile, and the stages that a workgroup has at most, with the least estimate: the workgroups' stages (three more for what
// stands around the contraction) over the places on the card and a quarter of a short one's behind that, or the longest one's,
// and what joining costs.  4096 rows, gated 256 -> 1024,
// backward: 43 us so, 59 without splits.
FfTogetherPlan ff_together_plan(const FfProduct* p, int count) {
  FfTogetherPlan best = {};
  best.tile = -1;
  if (count < 2) return best;
  for (int i = 0; i < count; ++i) best.micros += ff_tile_plan(p[i]).micros;
  for (int tile = kTile128; tile <= kTile64; ++tile) {
    const TileCost& c = kTileCosts[tile];
    if (!std::all_of(p, p + count, [&](const FfProduct& q) { return reaches(q, c); })) continue;
    for (int most = kLeastStages; most <= 512; most *= 2) {
      FfTogetherPlan plan = {};
      double groups = 0, work = 0, bytes = 0, joined = 0, joining = 0;  // `joining`: threads
      int longest = 0, shortest = 0x7fffffff;
      for (int i = 0; i < count; ++i) {
        const int all = stages_of(p[i]);
        const int splits = std::min(32, std::max(1, (all + most - 1) / most)), each = (all + splits - 1) / splits;
        plan.splits[i] = (all + each - 1) / each;
        plan.stages[i] = each;
        plan.at[i] = plan.part_bytes;
        if (plan.splits[i] > 1) {
          const double values = (double)p[i].M * ((p[i].N + 3) / 4 * 4) * plan.splits[i];
          plan.part_bytes += ((long long)values * 4 + 255) / 256 * 256;
          joined += 8.0 * values;
          joining += values / plan.splits[i] / 4 + 256;
        }
        const double tiles = (double)pieces(p[i].M, c.bm) * pieces(p[i].N, c.bn) * plan.splits[i];
        groups += tiles;
        work += tiles * (each + 3);
        longest = std::max(longest, each);
        shortest = std::min(shortest, each);
        bytes += operand_bytes(p[i]);
      }
      if ((groups + kBiasMost) * c.threads > kMostThreads || joining > kMostThreads) continue;
      const double slots = (double)kCus * c.per_cu;
      const double us = groups <= kCus ? longest * c.alone[1] : std::max<double>(longest, work / slots + 0.25 * shortest) * c.full[1];
      plan.tile = tile;
      plan.micros = std::max(us, bytes / kBytesPerMicro * std::max(1.0, 170.0 / groups)) + kLaunchMicros;
      if (joined > 0) plan.micros += kJoinMicros + joined / kJoinBytesPerMicro;
      if (plan.micros < best.micros) best = plan;
      if (joined == 0) break;  // more stages split nothing either
    }
  }
  return best;
}

int launch_ff_products(const FfProduct* p, int count, const FfBiasSum& sum, char* pack, float* ws, hipStream_t st) {
  FfTogetherPlan plan = {};
  plan.tile = -1;
  if (p[0].type != CCT_TYPE_F32) plan = ff_together_plan(p, count);
  int order[kFfTogether], n = 0;
  for (int i = 0; i < count; ++i)
    if (p[i].out) order[n++] = i;
  const bool apart = plan.tile < 0 || n == 0 || sum.N > kBiasMost * kBiasColumns;  // the sum of columns, the same bits
  int rc = apart ? launch_ff_bias_sum(sum, st) : CCT_OK;
  if (rc != CCT_OK) return rc;
  const FfBiasSum beside = apart ? FfBiasSum{} : sum;
  if (plan.tile < 0 || n == 0) {
    for (int i = 0; i < n && rc == CCT_OK; ++i) rc = launch_ff_product(p[order[i]], pack, ws, st);
    return rc;
  }
  // the longest first
  std::stable_sort(order, order + n, [&](int a, int b) { return plan.stages[a] > plan.stages[b]; });
  FfProduct wanted[kFfTogether];
  FfTogetherPlan theirs = plan;
  double flops = 0, bytes = 0;
  for (int i = 0; i < n; ++i) {
    const FfProduct& q = wanted[i] = p[order[i]];
    theirs.splits[i] = plan.splits[order[i]];
    theirs.stages[i] = plan.stages[order[i]];
    theirs.at[i] = plan.at[order[i]];
    flops += 2.0 * q.M * q.N * q.K * q.segments;
    bytes += operand_bytes(q) + 2.0 * q.M * q.N;
  }
  ProfScope ps(flops, bytes, st, "ff_tile_kernel_together<%s, %d products, %d splits>", kTileNames[plan.tile], n,
               *std::max_element(theirs.splits, theirs.splits + n));
  return p[0].type == CCT_TYPE_BF16 ? launch_ff_together_bf16(wanted, n, beside, theirs, (char*)ws, st)
                                    : launch_ff_together_f16(wanted, n, beside, theirs, (char*)ws, st);
}

}  // namespace cct
