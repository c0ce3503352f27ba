// What the translation units of the microscaled 4-bit operators share.
#pragma once
#include "feed_forward.h"

namespace cct {

constexpr int kMxBlock = 32;  // values that share a scale: 16 bytes of codes
inline int mx_blocks(int cols) { return pieces(cols, kMxBlock); }
inline long long mx_code_bytes(int cols) { return 16LL * mx_blocks(cols); }
inline long long mx_scale_bytes(int cols) { return (mx_blocks(cols) + 3LL) / 4 * 4; }

struct MxMatrix {
  const unsigned char* codes;
  long long ldc;  // bytes between rows
  const unsigned char* scales;
  long long lds;
};
int launch_mx_quantize(int rows, int cols, int type, const void* x, long long ldx, unsigned char* codes, long long ldc,
                       unsigned char* scales, long long lds, hipStream_t st);
int launch_mx_dequantize(int rows, int cols, int type, const MxMatrix& m, void* x, long long ldx, hipStream_t st);

// `p` has the sizes and what becomes of the sums; its operands are not looked at.
struct MxProduct {
  FfProduct p;
  MxMatrix x, w;
  int blocks;     // of a row
  bool quantize;  // x are values yet, in rows of x.ldc (up to kMxQuantizeRows rows on mx_rows.hip)
};
constexpr int kMxQuantizeRows = 4;
// How it runs: kNoTile: mx_rows.hip; splits of the contraction, of so many steps of 128 values (rows) or stages of 256 (tiles);
// deep: tiles of 64 x 64 that hold four stages, not two.
struct MxPlan {
  int tile, splits, steps;
  bool deep;
  long long part_bytes;
};
MxPlan mx_plan(int M, int N, int K);
int launch_mx_rows(const MxProduct& p, const MxPlan& plan, float* part, hipStream_t st);
int launch_mx_tile(const MxProduct& p, const MxPlan& plan, float* part, hipStream_t st);

}  // namespace cct
