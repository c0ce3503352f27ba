// The elementwise half of the feed-forward operators' backward passes:
//   linear  dz = dy act'(z), and dbias = column sums of dz;
//   gated   dg = dh u act'(g), du = dh act(g).
// Each input is read once and each output written once; the rounding of dz, dg and du to 16 bits is the matrix cores', which
// take no more of an operand (bf16 at most 2^-8 of a value, fp16 2^-11, as the operands themselves were rounded by; a gradient
// then has sqrt(2) times the error that its own rounding makes; in fp16 what passes 65504 is an infinity).
//
// A workgroup takes 256 columns x 64 rows (more from 2^35 values on), or 8 where that leaves CUs idle (1531 x 1000: 5.3 us,
// 9.9 before), a thread 8 neighbouring columns of every eighth row: its column sums stay in registers, meet in LDS in a fixed
// order and leave as one row of partial sums per workgroup, which ff_bias_sum.h adds in order.  Rows of any alignment; the
// outputs' rows are padded with zeros to a multiple of 8 values, which the products rely on.
#include <algorithm>

#include "activation.h"
#include "ff_bias_sum.h"

namespace cct {
namespace {

constexpr int NT = 256, kCols = 256;

template <class F>
void with_type(int type, F f) {
  if (type == CCT_TYPE_F32)
    f(std::integral_constant<int, CCT_TYPE_F32>());
  else if (type == CCT_TYPE_BF16)
    f(std::integral_constant<int, CCT_TYPE_BF16>());
  else
    f(std::integral_constant<int, CCT_TYPE_F16>());
}

// 8 values from column c on of a row of n, those past its end zero
template <int TYPE>
__device__ __forceinline__ void load_columns(float (&v)[8], const void* p, long long row, int c, int n) {
  if (c + 8 <= n) {
    const f32x8 all = load8<TYPE>(p, row + c);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = all[e];
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = c + e < n ? load1<TYPE>(p, row + c + e) : 0.f;
  }
}
// into a row that has room for whole eights
template <int TYPE>
__device__ __forceinline__ void store_columns(void* p, long long at, const float (&v)[8]) {
  f32x8 all;
#pragma unroll
  for (int e = 0; e < 8; ++e) all[e] = v[e];
  store8<TYPE>(p, at, all);
}

struct DzArgs {
  FfDz job[3];
  int first[3], rows[3];  // workgroup that a job begins at, rows of a workgroup
};
template <int TYPE>
__device__ __forceinline__ void do_dz(const DzArgs& a, int block) {
  const int which = (block >= a.first[1]) + (block >= a.first[2]), rows = a.rows[which];
  const FfDz& p = a.job[which];
  const int group = block - a.first[which], wide = pieces(p.N, kCols), down = group / wide;
  const int c0 = (group - down * wide) * kCols;
  const int c = c0 + (threadIdx.x & 31) * 8, lane_row = threadIdx.x >> 5;
  const int r0 = down * rows, r1 = rows < p.M - r0 ? r0 + rows : p.M;
  float sum[8] = {};
  if (c < p.N)
    for (int r = r0 + lane_row; r < r1; r += NT / 32) {
      float v[8];
      load_columns<TYPE>(v, p.dy, r * p.lddy, c, p.N);
      if (p.z) {
        float z[8];
        load_columns<TYPE>(z, p.z, r * p.ldz, c, p.N);
        activate_back<false>(p.activation, z, v, v);
      }
      if (p.dz) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (c + e >= p.N) v[e] = 0.f;
        store_columns<TYPE>(p.dz, r * p.ld + c, v);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[e] += v[e];
    }
  if (!p.dbias) return;
  __shared__ float sums[NT / 32][kCols];
#pragma unroll
  for (int e = 0; e < 8; ++e) sums[lane_row][(threadIdx.x & 31) * 8 + e] = sum[e];
  __syncthreads();
  const int col = c0 + threadIdx.x;
  if (col >= p.N) return;
  float s = 0.f;
#pragma unroll
  for (int k = 0; k < NT / 32; ++k) s += sums[k][threadIdx.x];
  if (p.M <= rows)
    store1<TYPE>(p.dbias, col, s);
  else
    p.part[(long long)down * p.N + col] = s;
}
template <int TYPE>
__global__ __launch_bounds__(NT) void ff_dz_kernel(DzArgs a) {
  do_dz<TYPE>(a, blockIdx.x);
}

constexpr int kSumThreads = kBiasColumns * kBiasRuns;
template <int TYPE>
__global__ __launch_bounds__(kSumThreads) void ff_bias_sum_kernel(FfBiasSum p, int first) {
  __shared__ float sums[kBiasRuns][kBiasColumns + 1];
  sum_bias<TYPE, kSumThreads>(p, first + blockIdx.x, sums);
}

template <int TYPE>
__global__ __launch_bounds__(NT) void ff_gated_dz_kernel(FfGatedDz p, int rows, int groups, DzArgs copies) {
  if ((int)blockIdx.x >= groups) return do_dz<TYPE>(copies, blockIdx.x - groups);
  const int wide = pieces(p.F, kCols), down = blockIdx.x / wide;
  const int c = (blockIdx.x - down * wide) * kCols + (threadIdx.x & 31) * 8;
  const int r0 = down * rows, r1 = rows < p.M - r0 ? r0 + rows : p.M;
  if (c >= p.F) return;
  for (int r = r0 + (threadIdx.x >> 5); r < r1; r += NT / 32) {
    float dh[8], g[8], u[8];
    load_columns<TYPE>(dh, p.dh, r * p.lddh, c, p.F);
    load_columns<TYPE>(g, p.g, r * p.ldg, c, p.F);
    load_columns<TYPE>(u, p.u, r * p.ldu, c, p.F);
#pragma unroll
    for (int e = 0; e < 8; ++e) u[e] *= dh[e];
    activate_back<true>(p.activation, g, u, dh);
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (c + e >= p.F) u[e] = dh[e] = 0.f;
    store_columns<TYPE>(p.dg, r * p.ld + c, u);
    store_columns<TYPE>(p.du, r * p.ld + c, dh);
  }
}

}  // namespace

namespace {
// Up to four matrices share a launch: of each at most 2^21 workgroups, or one for every 256 columns (2^23), which together
// are less than 2^24.
int rows_of_group(int M, int N) {
  const long long wide = pieces(N, kCols);
  if (pieces(M, 64) * wide < 1024) return 8;
  int rows = 64;
  while (rows < M && pieces(M, rows) * wide > 1 << 21) rows *= 2;
  return rows;
}
// Column sums of up to 32 rows need no second launch if a workgroup takes them all (4 rows per thread).
int rows_of_group(const FfDz& p) { return p.dbias && p.M <= 32 ? 32 : rows_of_group(p.M, p.N); }

// What a launch's workgroups need to know of the jobs, and how many they are.
int place(const FfDzJobs& p, DzArgs* a, double* ops, double* bytes) {
  int groups = 0;
  for (int i = 0; i < 3; ++i) {
    a->first[i] = i < p.count ? groups : 0x7fffffff;
    if (i >= p.count) continue;
    const FfDz& q = a->job[i] = p.job[i];
    a->rows[i] = rows_of_group(q);
    groups += pieces(q.M, a->rows[i]) * pieces(q.N, kCols);
    *ops += 2.0 * q.M * q.N;
    *bytes += (double)type_bytes(q.type) * q.M * q.N * (1 + (q.z != nullptr) + (q.dz != nullptr));
  }
  return groups;
}
}  // namespace
int ff_sum_rows(int M, int N) { return pieces(M, rows_of_group(M, N)); }

int launch_ff_dz(const FfDzJobs& p, FfBiasSum* left, hipStream_t st) {
  *left = {};
  if (p.count == 0) return CCT_OK;
  DzArgs a = {};
  double ops = 0.0, bytes = 0.0;
  const int groups = place(p, &a, &ops, &bytes);
  const FfDz& q = p.job[0];
  if (q.dbias && (q.M == 0 || q.M > a.rows[0])) *left = {q.part, q.dbias, ff_sum_rows(q.M, q.N), q.N, q.type};
  if (groups == 0) return CCT_OK;
  const char* const names[] = {"ff_dz_kernel<f32>", "ff_dz_kernel<bf16>", "ff_dz_kernel<f16>"};
  with_type(q.type, [&](auto type) {
    ProfScope ps(names[q.type], ops, bytes, st);
    hipLaunchKernelGGL(HIP_KERNEL_NAME(ff_dz_kernel<decltype(type)::value>), dim3(groups), dim3(NT), 0, st, a);
  });
  CCT_CHECK_LAUNCH();
  return CCT_OK;
}

int launch_ff_bias_sum(const FfBiasSum& p, hipStream_t st) {
  if (!p.dbias) return CCT_OK;
  with_type(p.type, [&](auto type) {
    ProfScope ps("ff_bias_sum_kernel", (double)p.rows * p.N, 4.0 * p.rows * p.N, st);
    const int groups = pieces(p.N, kBiasColumns), most = (int)(kMostThreads / kSumThreads);
    for (int first = 0; first < groups; first += most)
      hipLaunchKernelGGL(HIP_KERNEL_NAME(ff_bias_sum_kernel<decltype(type)::value>), dim3(std::min(most, groups - first)),
                         dim3(kSumThreads), 0, st, p, first);
  });
  CCT_CHECK_LAUNCH();
  return CCT_OK;
}

int launch_ff_gated_dz(const FfGatedDz& p, const FfDzJobs& copies, hipStream_t st) {
  if (p.M == 0) return CCT_OK;  // and nothing to copy: x has no rows, and dx, which takes the weights, has none
  DzArgs a = {};
  const double n = (double)p.M * p.F, e = type_bytes(p.type);
  double ops = 6.0 * n, bytes = 5.0 * e * n;
  const int groups = pieces(p.F, kCols) * ff_sum_rows(p.M, p.F), more = place(copies, &a, &ops, &bytes);
  with_type(p.type, [&](auto type) {
    ProfScope ps("ff_gated_dz_kernel", ops, bytes, st);
    hipLaunchKernelGGL(HIP_KERNEL_NAME(ff_gated_dz_kernel<decltype(type)::value>), dim3(groups + more), dim3(NT), 0, st, p,
                       rows_of_group(p.M, p.F), groups, a);
  });
  CCT_CHECK_LAUNCH();
  return CCT_OK;
}

}  // namespace cct
