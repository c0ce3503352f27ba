// Norms before and after a block with its gate on the residual stream (cct_residual_norm_*): forward
//   p = N_after(b),  s = r + scale gate p,  h = N_before(s),
// and backward, with n the normalised rows, dn = dh w and <.> a row's mean,
//   ds += rstd (dn - n <dn n> [- <dn>]),  dr = ds,  dp = scale gate ds,  and db from dp as ds from dh.
#include <algorithm>

#include "feed_forward.h"
#include "residual_norm.h"

namespace cct {
namespace {

template <class F>
void with_type(int type, F f) {
  if (type == CCT_TYPE_F32)
    f(std::integral_constant<int, CCT_TYPE_F32>());
  else if (type == CCT_TYPE_BF16)
    f(std::integral_constant<int, CCT_TYPE_BF16>());
  else
    f(std::integral_constant<int, CCT_TYPE_F16>());
}

// The sum over a wave's lanes, in all of them.
__device__ __forceinline__ float wave_sum(float v) {
  auto other = [](float x, auto how) {
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), decltype(how)::value, 0xf, 0xf, true));
  };
  v += other(v, std::integral_constant<int, 0xb1>());   // neighbours
  v += other(v, std::integral_constant<int, 0x4e>());   // pairs of them
  v += other(v, std::integral_constant<int, 0x141>());  // fours of a half row, mirrored
  v += other(v, std::integral_constant<int, 0x140>());  // eights of a row, mirrored
  v += __shfl_xor(v, 16, 64);
  return v + __shfl_xor(v, 32, 64);
}

constexpr int kMostWaves = 16;
// Sums over a workgroup's waves, in all threads.  Two places in LDS in turn: a wave that is a sum ahead does not write over what
// others still read.
struct RowSums {
  float (*lds)[kMostWaves][4];
  int waves, turn;
  template <int N>
  __device__ __forceinline__ void operator()(float (&v)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = wave_sum(v[i]);
    if (waves == 1) return;
    turn ^= 1;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) lds[turn][threadIdx.x >> 6][i] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = lds[turn][0][i];
    for (int w = 1; w < waves; ++w)
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] += lds[turn][w][i];
  }
};

__device__ __forceinline__ float sum8(const f32x8& v) { return ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7])); }
__device__ __forceinline__ f32x8 first_of(f32x8 v, int n) {
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = e < n ? v[e] : 0.f;
  return v;
}
// Values of a vector that may not be there.
template <int TYPE>
__device__ __forceinline__ f32x8 vector_or(const void* p, int c, int n, float none) {
  if (p) return load_first<TYPE>(p, c, n);
  f32x8 v;
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = none;
  return v;
}
__device__ __forceinline__ float rstd_of(float squares, const int D, float eps) { return 1.f / sqrtf(squares / (float)D + eps); }

// Rows of any length: each sum is a pass over the row, which a cache holds.
template <int TYPE>
__global__ __launch_bounds__(1024) void residual_norm_long_kernel(ResidualNorm p) {
  __shared__ float lds[2][kMostWaves][4];
  RowSums sums = {lds, (int)blockDim.x >> 6, 0};
  const int D = p.D, step = blockDim.x * 8, c0 = threadIdx.x * 8;
  for (long long row = blockIdx.x; row < p.M; row += gridDim.x) {
    const long long gate = p.gate ? row / p.gate_rows * p.ldgate : 0;
    float mean_b = 0.f, rstd_b = 1.f, mean_s = 0.f, rstd_s = 1.f;
    auto over = [&](auto f) {
      float v[1] = {0.f};
      for (long long c = c0; c < D; c += step) v[0] += sum8(first_of(f((int)c, (int)(D - c)), (int)(D - c)));
      sums(v);
      return v[0];
    };
    auto old = [&](int c, int n) { return load_first<TYPE>(p.b, row * p.ldb + c, n); };
    if (p.after == CCT_NORM_LAYER && p.b) mean_b = over(old) / (float)D;
    if (p.after != CCT_NORM_NONE && p.b)
      rstd_b = rstd_of(over([&](int c, int n) {
                         const f32x8 v = old(c, n) - mean_b;
                         return v * v;
                       }), D, p.eps);
    auto stream = [&](int c, int n) {
      f32x8 s = load_first<TYPE>(p.r, row * p.ldr + c, n);
      if (p.b) {
        f32x8 v = old(c, n);
        if (p.after != CCT_NORM_NONE) {
          v = (v - mean_b) * rstd_b * vector_or<TYPE>(p.w_after, c, n, 1.f);
          if (p.c_after) v += load_first<TYPE>(p.c_after, c, n);
        }
        if (p.gate) v *= load_first<TYPE>(p.gate, gate + c, n);
        s += v * p.scale;
      }
      return s;
    };
    if (p.h) {
      if (p.before == CCT_NORM_LAYER) mean_s = over(stream) / (float)D;
      rstd_s = rstd_of(over([&](int c, int n) {
                         const f32x8 v = stream(c, n) - mean_s;
                         return v * v;
                       }), D, p.eps);
    }
    for (long long at = c0; at < D; at += step) {
      const int c = (int)at, n = D - c;
      const f32x8 s = stream(c, n);
      if (p.s) store_first<TYPE>(p.s, row * p.lds + c, s, n);
      if (p.h) {
        f32x8 h = (s - mean_s) * rstd_s * vector_or<TYPE>(p.w_before, c, n, 1.f);
        if (p.c_before) h += load_first<TYPE>(p.c_before, c, n);
        store_first<TYPE>(p.h, row * p.ldh + c, h, n);
      }
    }
  }
}

// What a row's gradients are made of, with n_s = (s - mean_s) rstd_s: ds += rstd_s (dn - n_s slope_s - level_s), db alike.
struct RowStats {
  float mean_s, rstd_s, slope_s, level_s, mean_b, rstd_b, slope_b, level_b;
};

// The rows of a run.
struct NormRun {
  long long first, end;
};
__device__ __forceinline__ NormRun norm_run(const ResidualNormBack& p, const ResidualNormPlan& plan, int i) {
  if (plan.whole) return {(long long)i * plan.rows, min((long long)p.M, (long long)(i + 1) * plan.rows)};
  const int g = i / plan.per_gate;
  const long long first = (long long)g * p.gate_rows, end = min((long long)p.M, first + p.gate_rows);
  const long long at = first + (long long)(i - g * plan.per_gate) * plan.rows;
  return {at, min(end, at + plan.rows)};
}

// The stream's gradient at 8 columns; dh and n_s there, if there is a dh.
template <int TYPE>
__device__ __forceinline__ f32x8 stream_gradient(const ResidualNormBack& p, const RowStats& q, long long row, int c, int n, f32x8* dh,
                                                 f32x8* n_s) {
  f32x8 ds = {};
  if (p.ds) ds = load_first<TYPE>(p.ds, row * p.ldds + c, n);
  if (!p.dh) return ds;
  *dh = load_first<TYPE>(p.dh, row * p.lddh + c, n);
  *n_s = (load_first<TYPE>(p.s, row * p.lds + c, n) - q.mean_s) * q.rstd_s;
  return ds + (*dh * vector_or<TYPE>(p.w_before, c, n, 1.f) - *n_s * q.slope_s - q.level_s) * q.rstd_s;
}

template <int TYPE>
__global__ __launch_bounds__(1024) void residual_norm_stats_kernel(ResidualNormBack p, RowStats* __restrict__ stats) {
  __shared__ float lds[2][kMostWaves][4];
  RowSums sums = {lds, (int)blockDim.x >> 6, 0};
  const int D = p.D, step = blockDim.x * 8, c0 = threadIdx.x * 8;
  const bool block = p.b && p.after != CCT_NORM_NONE;
  for (long long row = blockIdx.x; row < p.M; row += gridDim.x) {
    RowStats q = {0.f, 1.f, 0.f, 0.f, 0.f, 1.f, 0.f, 0.f};
    auto over = [&](auto f) {
      float v[2] = {0.f, 0.f};
      for (long long c = c0; c < D; c += step) {
        f32x8 a = {}, b = {};
        const int n = (int)(D - c);
        f((int)c, n, a, b);
        v[0] += sum8(first_of(a, n));
        v[1] += sum8(first_of(b, n));
      }
      sums(v);
      return make_float2(v[0], v[1]);
    };
    auto at_s = [&](int c, int n) { return load_first<TYPE>(p.s, row * p.lds + c, n); };
    auto at_b = [&](int c, int n) { return load_first<TYPE>(p.b, row * p.ldb + c, n); };
    auto dn = [&](int c, int n) { return load_first<TYPE>(p.dh, row * p.lddh + c, n) * vector_or<TYPE>(p.w_before, c, n, 1.f); };
    if (p.dh) {
      if (p.before == CCT_NORM_LAYER) {
        const float2 t = over([&](int c, int n, f32x8& a, f32x8& b) {
          a = at_s(c, n);
          b = dn(c, n);
        });
        q.mean_s = t.x / (float)D;
        q.level_s = t.y / (float)D;
      }
      const float2 t = over([&](int c, int n, f32x8& a, f32x8& b) {
        const f32x8 v = at_s(c, n) - q.mean_s;
        a = v * v;
        b = v * dn(c, n);
      });
      q.rstd_s = rstd_of(t.x, D, p.eps);
      q.slope_s = t.y * q.rstd_s / (float)D;
    }
    if (block) {
      if (p.after == CCT_NORM_LAYER) q.mean_b = over([&](int c, int n, f32x8& a, f32x8&) { a = at_b(c, n); }).x / (float)D;
      q.rstd_b = rstd_of(over([&](int c, int n, f32x8& a, f32x8&) {
                           const f32x8 v = at_b(c, n) - q.mean_b;
                           a = v * v;
                         }).x, D, p.eps);
      const long long gate = p.gate ? row / p.gate_rows * p.ldgate : 0;
      const float2 t = over([&](int c, int n, f32x8& a, f32x8& b) {
        f32x8 dh, n_s;
        b = stream_gradient<TYPE>(p, q, row, c, n, &dh, &n_s) * p.scale;
        if (p.gate) b *= load_first<TYPE>(p.gate, gate + c, n);
        b *= vector_or<TYPE>(p.w_after, c, n, 1.f);
        a = b * ((at_b(c, n) - q.mean_b) * q.rstd_b);
      });
      q.slope_b = t.x / (float)D;
      q.level_b = p.after == CCT_NORM_LAYER ? t.y / (float)D : 0.f;
    }
    if (threadIdx.x == 0) stats[row] = q;
  }
}

// What a run of rows adds up, 8 columns of a thread.
struct ColumnSums {
  f32x8 v[kNormSums];
};

// 2048 columns of a run of rows: dr, db and the run's sums.
constexpr int kColumnThreads = 256;
template <int TYPE>
__global__ __launch_bounds__(kColumnThreads) void residual_norm_columns_kernel(ResidualNormBack p, ResidualNormPlan plan,
                                                                              const RowStats* __restrict__ stats,
                                                                              float* __restrict__ part) {
  const long long c8 = ((long long)blockIdx.y * kColumnThreads + threadIdx.x) * 8;
  if (c8 >= p.D) return;
  const int c = (int)c8, n = p.D - c;
  const NormRun run = norm_run(p, plan, blockIdx.x);
  ColumnSums sums = {};
  const f32x8 w_after = vector_or<TYPE>(p.w_after, c, n, 1.f);
  const bool block = p.b && p.after != CCT_NORM_NONE;
  for (long long row = run.first; row < run.end; ++row) {
    const RowStats q = stats[row];
    f32x8 dh = {}, n_s = {}, gate;
    const f32x8 ds = stream_gradient<TYPE>(p, q, row, c, n, &dh, &n_s);
    sums.v[kDcBefore] += dh;
    sums.v[kDwBefore] += dh * n_s;
    if (p.dr) store_first<TYPE>(p.dr, row * p.lddr + c, ds, n);
    f32x8 dp = ds * p.scale, n_b = {};
    if (block) n_b = (load_first<TYPE>(p.b, row * p.ldb + c, n) - q.mean_b) * q.rstd_b;
    if (p.gate) {
      gate = load_first<TYPE>(p.gate, row / p.gate_rows * p.ldgate + c, n);
      if (p.out[kDgate]) {
        f32x8 normed = block ? n_b * w_after : load_first<TYPE>(p.b, row * p.ldb + c, n);
        if (p.c_after) normed += load_first<TYPE>(p.c_after, c, n);
        sums.v[kDgate] += dp * normed;
        if (plan.whole && (row + 1 == run.end || (row + 1) % p.gate_rows == 0)) {
          store_first<TYPE>(p.out[kDgate], row / p.gate_rows * p.lddgate + c, sums.v[kDgate], n);
          sums.v[kDgate] = f32x8{};
        }
      }
      dp *= gate;
    }
    if (block) {
      sums.v[kDcAfter] += dp;
      sums.v[kDwAfter] += dp * n_b;
      dp = (dp * w_after - n_b * q.slope_b - q.level_b) * q.rstd_b;
    }
    if (p.db) store_first<TYPE>(p.db, row * p.lddb + c, dp, n);
  }
#pragma unroll
  for (int k = 0; k < kNormSums; ++k)
    if (p.out[k] && !(k == kDgate && plan.whole))
      store_first<CCT_TYPE_F32>((char*)part + k * plan.part_bytes, (long long)blockIdx.x * p.D + c, sums.v[k], n);
}

// The runs' sums, added in order: 32 columns of one result, 32 threads a column.  blockIdx.y: four vectors, then the gate's rows.
template <int TYPE>
__global__ __launch_bounds__(1024) void residual_norm_join_kernel(ResidualNormBack p, ResidualNormPlan plan, const float* __restrict__ part) {
  __shared__ float lds[32][33];
  const int k = min((int)blockIdx.y, (int)kDgate), group = (int)blockIdx.y - k;
  if (!p.out[k]) return;
  const int rows = k == kDgate ? plan.per_gate : plan.count, x = threadIdx.x & 31, y = threadIdx.x >> 5;
  const int c = blockIdx.x * 32 + x;
  const float* from = (const float*)((const char*)part + k * plan.part_bytes) + (long long)group * rows * p.D + c;
  float v = 0.f;
  if (c < p.D)
#pragma unroll 8
    for (int r = y; r < rows; r += 32) v += from[(long long)r * p.D];
  lds[y][x] = v;
  __syncthreads();
#pragma unroll
  for (int half = 16; half > 0; half >>= 1) {
    if (y < half) lds[y][x] += lds[y + half][x];
    __syncthreads();
  }
  if (y == 0 && c < p.D) store1<TYPE>(p.out[k], k == kDgate ? group * p.lddgate + c : c, lds[0][x]);
}

int row_threads(int D) { return std::min(kMostWaves, pieces(D, 512)) * 64; }
double forward_bytes(const ResidualNorm& p) {
  return (double)type_bytes(p.type) * p.M * p.D * (1 + (p.b != nullptr) + (p.s != nullptr) + (p.h != nullptr));
}

}  // namespace

ResidualNormPlan residual_norm_plan(const cct_residual_norm_desc_t& d) {
  ResidualNormPlan p = {};
  const int most = 512;
  const int wanted = std::max(4, pieces(d.M, most)), shared = std::min(d.gate_rows, std::max(d.M, 1));
  p.whole = shared <= wanted;
  if (p.whole) {
    p.rows = pieces(wanted, shared) * shared;
    p.per_gate = 0;
    p.count = pieces(d.M, p.rows);
  } else {
    p.per_gate = pieces(shared, wanted);
    p.rows = pieces(shared, p.per_gate);
    p.count = pieces(d.M, shared) * p.per_gate;
  }
  auto up = [](long long v) { return (v + 255) / 256 * 256; };
  p.part_off = up((long long)d.M * sizeof(RowStats));
  p.part_bytes = up((long long)p.count * d.D * 4);
  p.total = std::max(256LL, p.part_off + kNormSums * p.part_bytes);
  return p;
}

int launch_residual_norm(const ResidualNorm& p, hipStream_t st) {
  ProfScope ps("residual_norm_long_kernel", 0.0, forward_bytes(p), st);
  const int threads = row_threads(p.D);
  with_type(p.type, [&](auto type) {
    hipLaunchKernelGGL(HIP_KERNEL_NAME(residual_norm_long_kernel<decltype(type)::value>), dim3(std::min(p.M, 1 << 20)), dim3(threads),
                       0, st, p);
  });
  CCT_CHECK_LAUNCH();
  return CCT_OK;
}

int launch_residual_norm_back(const ResidualNormBack& p, const ResidualNormPlan& plan, char* ws, hipStream_t st) {
  RowStats* stats = (RowStats*)ws;
  float* part = (float*)(ws + plan.part_off);
  const double all = (double)type_bytes(p.type) * p.M * p.D;
  if (p.M > 0) {
    {
      ProfScope ps("residual_norm_stats_kernel", 0.0, all * ((p.ds != nullptr) + 2 * (p.dh != nullptr) + (p.b != nullptr)), st);
      with_type(p.type, [&](auto type) {
        hipLaunchKernelGGL(HIP_KERNEL_NAME(residual_norm_stats_kernel<decltype(type)::value>), dim3(std::min(p.M, 1 << 20)),
                           dim3(row_threads(p.D)), 0, st, p, stats);
      });
      CCT_CHECK_LAUNCH();
    }
    ProfScope ps("residual_norm_columns_kernel", 0.0,
                 all * ((p.ds != nullptr) + 2 * (p.dh != nullptr) + (p.b != nullptr) + (p.dr != nullptr) + (p.db != nullptr)), st);
    with_type(p.type, [&](auto type) {
      hipLaunchKernelGGL(HIP_KERNEL_NAME(residual_norm_columns_kernel<decltype(type)::value>),
                         dim3(plan.count, pieces(p.D, kColumnThreads * 8)), dim3(kColumnThreads), 0, st, p, plan, stats, part);
    });
    CCT_CHECK_LAUNCH();
  }
  const bool vectors = p.out[kDcBefore] || p.out[kDwBefore] || p.out[kDcAfter] || p.out[kDwAfter];
  const bool gate = p.out[kDgate] && !plan.whole && p.M > 0;
  if (vectors || gate) {
    ProfScope ps("residual_norm_join_kernel", 0.0, 0.0, st);
    with_type(p.type, [&](auto type) {
      hipLaunchKernelGGL(HIP_KERNEL_NAME(residual_norm_join_kernel<decltype(type)::value>),
                         dim3(pieces(p.D, 32), kDgate + (gate ? plan.count / plan.per_gate : 0)), dim3(1024), 0, st, p, plan, part);
    });
    CCT_CHECK_LAUNCH();
  }
  return CCT_OK;
}

}  // namespace cct

using namespace cct;

namespace {

bool matrix_ok(const void* p, long long ld, long long rows, long long cols, int type) {
  return p && !((uintptr_t)p & (type_bytes(type) - 1)) && ld >= 0 && (rows <= 1 || ld >= cols);
}
bool maybe_ok(const void* p, long long ld, long long rows, long long cols, int type) { return !p || matrix_ok(p, ld, rows, cols, type); }
bool vector_ok(const void* p, int type) { return !((uintptr_t)p & (type_bytes(type) - 1)); }
bool norm_known(int kind) { return kind >= CCT_NORM_NONE && kind <= CCT_NORM_LAYER; }

// As the products' sizes, so that counts and offsets stay within their types.
int dims_ok(const cct_residual_norm_desc_t& d) {
  if (d.M < 0 || d.D < 1 || d.gate_rows < 1 || !type_known(d.type) || !norm_known(d.before) || !norm_known(d.after) ||
      !(d.eps >= 0.f && d.eps <= 3.4e38f) || !(d.scale >= -3.4e38f && d.scale <= 3.4e38f))
    return CCT_EINVAL;
  if (std::max(d.M, d.D) > 0x7fffff00) return CCT_EUNSUPPORTED;
  return (long long)std::max(d.M, 1) * d.D * type_bytes(d.type) <= 1LL << 38 ? CCT_OK : CCT_EUNSUPPORTED;
}
int gate_count(const cct_residual_norm_desc_t& d) { return pieces(d.M, d.gate_rows); }

}  // namespace

extern "C" {

int cct_residual_norm_forward(const cct_residual_norm_desc_t* desc, const void* r, int64_t ldr, const void* b, int64_t ldb,
                              const void* gate, int64_t ldgate, const void* w_after, const void* c_after,
                              const void* w_before, const void* c_before, void* s, int64_t lds, void* h, int64_t ldh,
                              void* hip_stream) {
  if (!desc) return CCT_EINVAL;
  const cct_residual_norm_desc_t& d = *desc;
  const int rc = dims_ok(d);
  if (rc != CCT_OK) return rc;
  if ((d.after == CCT_NORM_NONE && (w_after || c_after)) || (d.before == CCT_NORM_NONE && (w_before || c_before || h))) return CCT_EINVAL;
  if (d.M == 0) return CCT_OK;  // its tensors have no address
  if (!b && (gate || w_after || c_after)) return CCT_EINVAL;
  if (!matrix_ok(r, ldr, d.M, d.D, d.type) || !maybe_ok(b, ldb, d.M, d.D, d.type) ||
      !maybe_ok(gate, ldgate, gate_count(d), d.D, d.type) || !maybe_ok(s, lds, d.M, d.D, d.type) ||
      !maybe_ok(h, ldh, d.M, d.D, d.type) || !vector_ok(w_after, d.type) || !vector_ok(c_after, d.type) ||
      !vector_ok(w_before, d.type) || !vector_ok(c_before, d.type))
    return CCT_EINVAL;
  if (!s && !h) return CCT_OK;
  return launch_residual_norm({d.M, d.D, d.type, d.before, d.after, d.gate_rows, d.eps, d.scale, r, b, gate, w_after, c_after,
                               w_before, c_before, s, h, ldr, ldb, ldgate, lds, ldh},
                              (hipStream_t)hip_stream);
}

int cct_residual_norm_workspace_bytes(const cct_residual_norm_desc_t* desc, size_t* bytes) {
  if (!desc || !bytes) return CCT_EINVAL;
  const int rc = dims_ok(*desc);
  if (rc != CCT_OK) return rc;
  *bytes = (size_t)residual_norm_plan(*desc).total;
  return CCT_OK;
}

int cct_residual_norm_backward(const cct_residual_norm_desc_t* desc, const void* s, int64_t lds, const void* b, int64_t ldb,
                               const void* gate, int64_t ldgate, const void* w_after, const void* c_after,
                               const void* w_before, const void* ds, int64_t ldds, const void* dh, int64_t lddh, void* dr,
                               int64_t lddr, void* db, int64_t lddb, void* dgate, int64_t lddgate, void* dw_after,
                               void* dc_after, void* dw_before, void* dc_before, void* workspace, size_t workspace_bytes,
                               void* hip_stream) {
  if (!desc) return CCT_EINVAL;
  const cct_residual_norm_desc_t& d = *desc;
  const int rc = dims_ok(d);
  if (rc != CCT_OK) return rc;
  const bool normed = d.after != CCT_NORM_NONE;
  if ((!normed && (w_after || c_after || dw_after || dc_after)) ||
      (d.before == CCT_NORM_NONE && (w_before || dh || dw_before || dc_before)) || (dgate && !gate))
    return CCT_EINVAL;
  const void* vectors[] = {w_after, c_after, w_before, dw_after, dc_after, dw_before, dc_before};
  for (const void* v : vectors)
    if (!vector_ok(v, d.type)) return CCT_EINVAL;
  if (d.M > 0) {
    const bool needs_b = dgate || (normed && (db || dw_after || dc_after));
    if ((!ds && !dh) || (dh && !s) || (needs_b && !b)) return CCT_EINVAL;
    const struct {
      const void* p;
      int64_t ld;
    } matrices[] = {{s, lds}, {b, ldb}, {ds, ldds}, {dh, lddh}, {dr, lddr}, {db, lddb}};
    for (const auto& m : matrices)
      if (!maybe_ok(m.p, m.ld, d.M, d.D, d.type)) return CCT_EINVAL;
    if (!maybe_ok(gate, ldgate, gate_count(d), d.D, d.type) || !maybe_ok(dgate, lddgate, gate_count(d), d.D, d.type))
      return CCT_EINVAL;
  }
  const ResidualNormPlan plan = residual_norm_plan(d);
  if (!workspace || ((uintptr_t)workspace & 255)) return CCT_EINVAL;
  if (workspace_bytes < (size_t)plan.total) return CCT_EWORKSPACE;
  const bool block = db || dgate || dw_after || dc_after;  // else b is not looked at
  return launch_residual_norm_back({d.M, d.D, d.type, d.before, d.after, d.gate_rows, d.eps, d.scale, s, block ? b : nullptr,
                                    block ? gate : nullptr, w_after, c_after, w_before, ds, dh, dr, db, lds, ldb, ldgate, ldds, lddh,
                                    lddr, lddb, {dc_before, dw_before, dc_after, dw_after, dgate}, lddgate},
                                   plan, (char*)workspace, (hipStream_t)hip_stream);
}

}  // extern "C"
