// What the translation units of the feed-forward operators share.
#pragma once
#include "cct_internal.h"
#include "number_types.h"

namespace cct {

// How many pieces of `of` make n >= 0.  Unsigned: sizes go up to 2^31 - 256, and pieces are as large.
__host__ __device__ inline int pieces(int n, int of) { return (int)(((unsigned)n + (unsigned)of - 1u) / (unsigned)of); }

// One matrix product of a feed-forward operator: sum over segments s and k of A_s(m, k) B_s(n, k), M x N results, and what
// becomes of them.
struct FfOperand {
  const void* p;
  long long ld;  // elements between rows in memory
};
// An operand's element (row, k) lies at p + row * ff_row + k * ff_step elements: along the contraction or across it.
inline long long ff_row(const FfOperand& o, bool across) { return across ? 1 : o.ld; }
inline long long ff_step(const FfOperand& o, bool across) { return across ? o.ld : 1; }
enum FfEpilogue {
  kFfLinear,  // z = sum + bias (kept if z is there), out = act(z) + residual
  kFfGated    // two products of the same A: g and u (kept if z and z2 are there), out = act(g) * u
};
// What a kernel needs first stands first: a launch's arguments come from memory, and every 64 bytes of them that it waits for
// take about 0.5 us (one row of 4096 x 4096, 8 us: 0.6 more with a fifth such line).
struct FfProduct {
  int M, N, K;
  int activation;
  FfOperand B[2], A[2];  // kFfGated: B[0] and B[1] are the two products'
  const void* bias;
  const void* residual;
  long long ldr;
  void* out;
  long long ldo;
  void *z, *z2;
  long long ldz, ldz2;
  int type;
  int segments;  // 1 or 2: contractions that are summed
  int epilogue;
  bool a_across, b_across;  // in both segments, whose strides are the same
};
// `pack` (fp32) and `ws`: room for an operand's terms and for partial sums, as the plans below say.
int launch_ff_product(const FfProduct& p, char* pack, float* ws, hipStream_t st);
// How a 16-bit product is cut (ff_tile.h): its tile, splits of the contraction of so many stages, the bytes of their partial
// sums (launch_ff_product's `ws`) and an estimate; rows or columns behind which the rest is a launch with a plan of its own.
enum { kTile256, kTile192 /* 192 x 256 */, kTile128, kTile64x128, kTile64, kNoTile /* ff_general_kernel */ };
constexpr int kFfStage = 64;
struct FfTilePlan {
  int tile, splits, stages;
  long long part_bytes;
  double micros;
  int cut_rows, cut_cols;
};
// From the product's sizes and how its operands lie; pointers and strides are not looked at.
FfTilePlan ff_tile_plan(const FfProduct& p);
int launch_ff_tile_bf16(const FfProduct& p, const FfTilePlan& plan, float* ws, hipStream_t st);
int launch_ff_tile_f16(const FfProduct& p, const FfTilePlan& plan, float* ws, hipStream_t st);
// Products that neither those nor the fp32 ones take (ff_general.hip), in splits of so many steps of 16.
struct FfGeneralPlan {
  int splits, steps;
  long long part_bytes;
};
FfGeneralPlan ff_general_plan(const FfProduct& p);
int launch_ff_general(const FfProduct& p, const FfGeneralPlan& plan, float* ws, hipStream_t st);
// fp32 (ff_f32.hip): splits of `len` steps, rows that are packed at a time, and the bytes for them and for the sums; how the
// general kernel runs where it has to.
struct FfF32Plan {
  int splits, len, rows;
  long long pack_bytes, part_bytes;
  FfGeneralPlan general;
};
FfF32Plan ff_f32_plan(const FfProduct& p);
int launch_ff_f32(const FfProduct& p, char* pack, float* ws, hipStream_t st);
// A forward product (operands along the contraction, at any address) of few rows: up to kFfRowsMost run, up to kFfRows (fp32:
// kFfRowsF32) are faster so.
constexpr int kFfRows = 16, kFfRowsF32 = 32, kFfRowsMost = 64;
bool ff_rows_fits(int N, int type);  // whether a launch takes so many columns
// `ws`: ff_rows_part_bytes.
long long ff_rows_part_bytes(int M, int N, int K, int type, int epilogue);
int launch_ff_rows(const FfProduct& p, float* ws, hipStream_t st);
// Whether the 16-bit product takes a matrix of `cols` consecutive values and rows `ld` apart in place: 16-byte loads, 256 rows
// within 32-bit offsets (a copy's rows are as long as they are: ff_tile_plan chooses a tile that reaches them).  Rows that are
// no multiple of 8 values must be followed by zeros up to one, as copies are.
inline bool ff_in_place(const void* p, long long ld, long long cols) {
  return !((uintptr_t)p & 15) && ld % 8 == 0 && cols % 8 == 0 && ld < (1LL << 21);
}
// Whether the rows of a matrix of 16-bit values begin at multiples of four bytes.
inline bool ff_words(const FfOperand& m) { return !((uintptr_t)m.p & 3) && m.ld % 2 == 0; }

// dz = dy * act'(z) into rows of ld values (a multiple of 8; zeros behind the N values of a row), and the column sums of the
// unrounded dz; any of the two may be missing.  z NULL: dz = dy.  `part`: ff_sum_rows(M, N) * N floats.
struct FfDz {
  int M, N, type, activation;
  const void *dy, *z;
  long long lddy, ldz;
  void* dz;
  long long ld;
  void* dbias;
  float* part;
};
int ff_sum_rows(int M, int N);
// Up to three of them, independent of each other, in one launch (all of one type): dz next to copies of x and w.
struct FfDzJobs {
  FfDz job[3];
  int count;
};
// What is left of a sum of columns, if dbias is there: rows of partial sums.
struct FfBiasSum {
  const float* part;
  void* dbias;
  int rows, N, type;
};
// Only the first job may have a dbias, which *left finishes: launch_ff_bias_sum or launch_ff_products.
int launch_ff_dz(const FfDzJobs& p, FfBiasSum* left, hipStream_t st);
int launch_ff_bias_sum(const FfBiasSum& p, hipStream_t st);
// dg = dh * u * act'(g), du = dh * act(g), both with rows of ld values as dz above.
struct FfGatedDz {
  int M, F, type, activation;
  const void *dh, *g, *u;
  long long lddh, ldg, ldu;
  void *dg, *du;
  long long ld;
};
// With copies (no dbias) in the same launch.
int launch_ff_gated_dz(const FfGatedDz& p, const FfDzJobs& copies, hipStream_t st);
// Up to kFfTogether products whose B lies across the contraction, nothing added, none of which needs another's results, and
// a sum of columns: one launch for all, or one after the other.  Those without `out` are not wanted; they are there because
// the choice is made for all, so that a result's last bits do not depend on what else is asked for.
constexpr int kFfTogether = 3;
int launch_ff_products(const FfProduct* p, int count, const FfBiasSum& sum, char* pack, float* ws, hipStream_t st);
// That choice (16-bit types), which follows from sizes alone: tile < 0 if one after the other; splits, stages of one, and where
// in `ws` each product's partial sums lie.
struct FfTogetherPlan {
  int tile, splits[kFfTogether], stages[kFfTogether];
  long long at[kFfTogether], part_bytes;
  double micros;
};
FfTogetherPlan ff_together_plan(const FfProduct* p, int count);
int launch_ff_together_bf16(const FfProduct* p, int count, const FfBiasSum& sum, const FfTogetherPlan& plan, char* ws, hipStream_t st);
int launch_ff_together_f16(const FfProduct* p, int count, const FfBiasSum& sum, const FfTogetherPlan& plan, char* ws, hipStream_t st);

}  // namespace cct
