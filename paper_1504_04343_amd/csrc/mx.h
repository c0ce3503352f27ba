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
  bool quantize;  // x are values yet, in rows of x.ldc (mx_rows.hip, where mx_quantizes says so)
};
// Whether the workgroups that multiply quantise x as well, each all of it: a launch (3.5 us) less, as long as every CU has one of them
// (16 columns) and rows are not too long (one row, weights from memory, and with a launch for x: 4096 x 4096 7.4 and 10.7 us, 4096 x
// 8192 10.6 and 10.7, 2048 x 16384 17.8 and 12.3, 5120 x 5120 14.4 and 10.9, 8192 x 4096 11.5 and 10.7, 14144 x 8960 42 and 19).
inline bool mx_quantizes(int M, int N, int K) { return M <= 4 && N <= 4096 && K <= 8192; }
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
