// Norms before and after a block with its gate on the residual stream (cct_residual_norm_*): forward
//   p = N_after(b),  s = r + scale gate p,  h = N_before(s),
// and backward, with n the normalised rows, dn = dh w and <.> a row's mean,
//   ds += rstd (dn - n <dn n> [- <dn>]),  dr = ds,  dp = scale gate ds,  and db from dp as ds from dh.
#include <algorithm>

#include "feed_forward.h"
#include "residual_norm.h"
#include "wave_ops.h"

namespace cct {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

template <class F>
void with_type(int type, F f) {
  if (type == CCT_TYPE_F32)
    f(std::integral_constant<int, CCT_TYPE_F32>());
  else if (type == CCT_TYPE_BF16)
    f(std::integral_constant<int, CCT_TYPE_BF16>());
  else
    f(std::integral_constant<int, CCT_TYPE_F16>());
}

template <class F>
void with_bool(bool b, F f) {
  if (b)
    f(std::true_type());
  else
    f(std::false_type());
}

constexpr int kMostWaves = 16, kRegisterColumns = kMostWaves * 512;
constexpr int kNormTeams = 4;  // rows of up to 512 columns that a workgroup takes at a time
// Sums over a workgroup's waves, in all threads.  Two places in LDS in turn: a wave that is a sum ahead does not write over what
// others still read.  Each lane reads one wave's sum: one after the other they were a trip to LDS each.
struct RowSums {
  float (*lds)[4][kMostWaves];
  int waves, turn;
  int first = 0;  // of the workgroup's waves
  template <int N>
  __device__ __forceinline__ void operator()(float (&v)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = wave_sum(v[i]);
    if (waves == 1) return;
    turn ^= 1;
    const int lane = threadIdx.x & 15;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) lds[turn][i][threadIdx.x >> 6] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = lane < waves ? lds[turn][i][first + lane] : 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = row_sum(v[i]);
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
  if (p) return load_row<TYPE>(p, 0, c, n);
  f32x8 v;
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = none;
  return v;
}
__device__ __forceinline__ float rstd_of(float squares, const int D, float eps) { return 1.f / sqrtf(squares / (float)D + eps); }

// Rows of any length: each sum is a pass over the row, which a cache holds (bf16, 4096 x 12296, two norms: 125 us, 3.2 TB/s of what
// has to be moved).
template <int TYPE>
__global__ __launch_bounds__(1024) void residual_norm_long_kernel(ResidualNorm p) {
  __shared__ float lds[2][4][kMostWaves];
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
    auto old = [&](int c, int n) { return load_row<TYPE>(p.b, row * p.ldb, c, n); };
    if (p.after == CCT_NORM_LAYER && p.b) mean_b = over(old) / (float)D;
    if (p.after != CCT_NORM_NONE && p.b)
      rstd_b = rstd_of(over([&](int c, int n) {
                         const f32x8 v = old(c, n) - mean_b;
                         return v * v;
                       }), D, p.eps);
    auto stream = [&](int c, int n) {
      f32x8 s = load_row<TYPE>(p.r, row * p.ldr, c, n);
      if (p.b) {
        f32x8 v = old(c, n);
        if (p.after != CCT_NORM_NONE) {
          v = (v - mean_b) * rstd_b * vector_or<TYPE>(p.w_after, c, n, 1.f);
          if (p.c_after) v += load_row<TYPE>(p.c_after, 0, c, n);
        }
        if (p.gate) v *= load_row<TYPE>(p.gate, gate, c, n);
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
        if (p.c_before) h += load_row<TYPE>(p.c_before, 0, c, n);
        store_first<TYPE>(p.h, row * p.ldh + c, h, n);
      }
    }
  }
}

// load_row_raw, settle_row and store_first where a row is whole eights (EIGHTS): less code and fewer registers.
template <int TYPE, bool EIGHTS>
__device__ __forceinline__ typename Number<TYPE>::V8 row_raw(const void* p, long long row, int c, int n) {
  if constexpr (!EIGHTS) return load_row_raw<TYPE>(p, row, c, n);
  typename Number<TYPE>::V8 v = {};
  if (n > 0) v = *(const typename Number<TYPE>::U8*)((const typename Number<TYPE>::T*)p + row + c);
  return v;
}
template <int TYPE, bool EIGHTS>
__device__ __forceinline__ f32x8 settled(const typename Number<TYPE>::V8& v, int c, int n) {
  if constexpr (EIGHTS) return __builtin_convertvector(v, f32x8);
  return __builtin_convertvector(settle_row<TYPE>(v, c, n), f32x8);
}
template <int TYPE, bool EIGHTS>
__device__ __forceinline__ void store_row(void* p, long long i, const f32x8& v, int n) {
  if constexpr (!EIGHTS) return store_first<TYPE>(p, i, v, n);
  if (n > 0) store8<TYPE>(p, i, v);
}

// A vector that may not be there.
template <int TYPE, bool EIGHTS>
__device__ __forceinline__ typename Number<TYPE>::V8 row_vector(const void* p, int c, int n, float none) {
  typename Number<TYPE>::V8 v;
  if (p) {
    v = row_raw<TYPE, EIGHTS>(p, 0, c, n);
    return EIGHTS ? v : settle_row<TYPE>(v, c, n);
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = (typename Number<TYPE>::T)none;
  return v;
}

// A row in registers, 8 columns a thread: a workgroup takes one at a time, or a wave where 512 columns are all.  What it waits for
// is memory, and between loads and stores the meetings of its waves (two norms: one each, layer norms two), so that other
// workgroups, or, where a row takes half a CU or more (AHEAD), the next row's loads have to fill them.  bf16, one norm after the
// addition, 8192 x 4096: 48 us, 5.6 TB/s (fp32 95, 5.7); 8192 x 8192: 102 us, with weights loaded behind the next row 130, without the next row
// on its way 156.
template <int TYPE, bool EIGHTS, bool AHEAD>
__global__ __launch_bounds__(1024) void residual_norm_kernel(ResidualNorm p, bool wave_rows) {
  typedef typename Number<TYPE>::V8 V8;
  __shared__ float lds[2][4][kMostWaves];
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), waves = blockDim.x >> 6;
  RowSums total = {lds, wave_rows ? 1 : waves, 0};
  const int c = (wave_rows ? threadIdx.x & 63 : threadIdx.x) * 8, n = p.D - c;
  const long long first = wave_rows ? (long long)blockIdx.x * waves + wave : blockIdx.x;
  const long long stride = wave_rows ? (long long)gridDim.x * waves : gridDim.x;
  // v becomes v - mean, zeros behind the row; the factor
  auto center = [&](int kind, f32x8& v) {
    float t[1];
    if (kind == CCT_NORM_LAYER) {
      t[0] = sum8(v);
      total(t);
      v = first_of(v - t[0] / (float)p.D, n);
    }
    t[0] = sum8(v * v);
    total(t);
    return rstd_of(t[0], p.D, p.eps);
  };
  V8 r, b, gate;
  auto load = [&](long long row) {
    r = row_raw<TYPE, EIGHTS>(p.r, row * p.ldr, c, n);
    if (p.b) b = row_raw<TYPE, EIGHTS>(p.b, row * p.ldb, c, n);
    if (p.gate) gate = row_raw<TYPE, EIGHTS>(p.gate, (long long)((unsigned)row / (unsigned)p.gate_rows) * p.ldgate, c, n);
  };
  auto wide = [](const V8& v) { return __builtin_convertvector(v, f32x8); };
  if (first < p.M) load(first);
  // what all rows take, so that in the loop nothing is loaded behind the next row: what comes last is waited for with all before it
  V8 w_after, c_after, w_before, c_before;
  if (p.b && p.after != CCT_NORM_NONE) {
    w_after = row_vector<TYPE, EIGHTS>(p.w_after, c, n, 1.f);
    c_after = row_vector<TYPE, EIGHTS>(p.c_after, c, n, 0.f);
  }
  if (p.h) {
    w_before = row_vector<TYPE, EIGHTS>(p.w_before, c, n, 1.f);
    c_before = row_vector<TYPE, EIGHTS>(p.c_before, c, n, 0.f);
  }
  for (long long row = first; row < p.M; row += stride) {
    if (!AHEAD && row != first) load(row);
    f32x8 s = settled<TYPE, EIGHTS>(r, c, n), v, g;
    if (p.b) v = settled<TYPE, EIGHTS>(b, c, n);
    if (p.gate) g = settled<TYPE, EIGHTS>(gate, c, n);
    if (AHEAD && row + stride < p.M) load(row + stride);
    if (p.b) {
      if (p.after != CCT_NORM_NONE) {
        const float rstd = center(p.after, v);
        v = v * rstd * wide(w_after) + wide(c_after);
      }
      if (p.gate) v *= g;
      s += v * p.scale;
    }
    if (p.s) store_row<TYPE, EIGHTS>(p.s, row * p.lds + c, s, n);
    if (p.h) {
      const float rstd = center(p.before, s);
      store_row<TYPE, EIGHTS>(p.h, row * p.ldh + c, s * rstd * wide(w_before) + wide(c_before), n);
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
  if (p.ds) ds = load_row<TYPE>(p.ds, row * p.ldds, c, n);
  if (!p.dh) return ds;
  *dh = load_row<TYPE>(p.dh, row * p.lddh, c, n);
  *n_s = (load_row<TYPE>(p.s, row * p.lds, c, n) - q.mean_s) * q.rstd_s;
  return ds + (*dh * vector_or<TYPE>(p.w_before, c, n, 1.f) - *n_s * q.slope_s - q.level_s) * q.rstd_s;
}

template <int TYPE>
__global__ __launch_bounds__(1024) void residual_norm_stats_kernel(ResidualNormBack p, RowStats* __restrict__ stats) {
  __shared__ float lds[2][4][kMostWaves];
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
    auto at_s = [&](int c, int n) { return load_row<TYPE>(p.s, row * p.lds, c, n); };
    auto at_b = [&](int c, int n) { return load_row<TYPE>(p.b, row * p.ldb, c, n); };
    auto dn = [&](int c, int n) { return load_row<TYPE>(p.dh, row * p.lddh, c, n) * vector_or<TYPE>(p.w_before, c, n, 1.f); };
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
        if (p.gate) b *= load_row<TYPE>(p.gate, gate, c, n);
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
  const long long c8 = ((long long)blockIdx.x * kColumnThreads + threadIdx.x) * 8;
  if (c8 >= p.D) return;
  const int c = (int)c8, n = p.D - c;
  const NormRun run = norm_run(p, plan, blockIdx.y);
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
    if (block) n_b = (load_row<TYPE>(p.b, row * p.ldb, c, n) - q.mean_b) * q.rstd_b;
    if (p.gate) {
      gate = load_row<TYPE>(p.gate, row / p.gate_rows * p.ldgate, c, n);
      if (p.out[kDgate]) {
        f32x8 normed = block ? n_b * w_after : load_row<TYPE>(p.b, row * p.ldb, c, n);
        if (p.c_after) normed += load_row<TYPE>(p.c_after, 0, c, n);
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
      store_first<CCT_TYPE_F32>((char*)part + k * plan.part_bytes, (long long)blockIdx.y * p.D + c, sums.v[k], n);
}

// Where the norms' sums are: LDS, where a workgroup may be of up to sixteen waves: four on a SIMD leave a thread 128 registers, too few
// for the sums and a row, so that the next row is not on its way either.  The sums take 128 KiB, one workgroup a CU, which is what
// the plan counts on.  Up to 512 threads have 256 registers.
template <int THREADS>
constexpr bool norm_sums_in_lds = THREADS == 1024;

// The same of rows of up to 8192 columns in one pass: a thread has 8 columns, a workgroup a run of rows, one at a time, or as many as
// it has teams of waves for a row each (in spans: of a gate row's rows, so that its sum is one team's): four of one wave where 512
// columns are all, two of five or six.  The next row is on its way while one is worked on; its sums over columns stay with the thread.
// Between a row's loads and stores its waves meet two or three times, which is what the time went into (8192 x 4096, bf16, two norms
// and a gate: 84 to 93 us by card in calls that follow one another, 103 to 108 in a kernel trace, where each launch stands alone; 79 at
// a copy's rate; 15 more with sums over waves that read LDS one after the other); the runs' sums and their joining take 6 to 10 us
// more.  Two teams, since a CU starts no second workgroup of five waves: 8192 x 2560 89 -> 67 us, 1531 x 2049 fp16 with layer norms 39
// -> 34 (two such workgroups a CU in the plan were 49 for 41 then).
template <int TYPE, int THREADS, bool EIGHTS>
__global__ __launch_bounds__(THREADS) __attribute__((amdgpu_waves_per_eu(THREADS / 256 < 2 ? 2 : THREADS / 256)))
void residual_norm_back_kernel(ResidualNormBack p, ResidualNormPlan plan, float* __restrict__ part) {
  typedef typename Number<TYPE>::V8 V8;
  constexpr bool IN_LDS = norm_sums_in_lds<THREADS>, AHEAD = !IN_LDS;
  __shared__ float lds[2][4][kMostWaves];
  __shared__ __attribute__((aligned(16))) float meet[THREADS == 512 ? (kNormTeams - 1) * 512 : THREADS == 768 ? 6 * 512 : 1];
  extern __shared__ f32x4 norm_sums[];
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), waves = (p.D + 511) >> 9;  // of a team
  const int teams = AHEAD ? (int)(blockDim.x >> 6) / waves : 1, team = AHEAD ? wave / waves : 0, thread = threadIdx.x - team * waves * 64;
  RowSums total = {lds, waves, 0, team * waves};
  const int c = thread * 8, n = p.D - c;
  const float D = (float)p.D;
  const bool block = p.b && p.after != CCT_NORM_NONE;
  const NormRun run = norm_run(p, plan, blockIdx.x);
  const int span = plan.whole ? p.gate_rows : 1;
  const long long begin = (long long)team * span, skip = (long long)(teams - 1) * span;
  const V8 raw_before = row_vector<TYPE, EIGHTS>(p.w_before, c, n, 1.f), raw_after = row_vector<TYPE, EIGHTS>(p.w_after, c, n, 1.f),
           raw_c = row_vector<TYPE, EIGHTS>(p.c_after, c, n, 0.f);
  ColumnSums sums = {};
  auto own = [&](int k, int half) { return norm_sums + (k * 2 + half) * THREADS + threadIdx.x; };
  if constexpr (IN_LDS)
#pragma unroll
    for (int k = 0; k < kDgate; ++k) *own(k, 0) = *own(k, 1) = f32x4{};
  auto add = [&](auto which, const f32x8& v) {
    constexpr int K = decltype(which)::value;
    if constexpr (!IN_LDS || K == kDgate) {
      sums.v[K] += v;
    } else if (p.out[K]) {
      *own(K, 0) += __builtin_shufflevector(v, v, 0, 1, 2, 3);
      *own(K, 1) += __builtin_shufflevector(v, v, 4, 5, 6, 7);
    }
  };

  struct Row {
    V8 s, b, ds, dh, gate;
  };
  auto load = [&](Row& to, long long row, long long before) {
    if (p.ds) to.ds = row_raw<TYPE, EIGHTS>(p.ds, row * p.ldds, c, n);
    if (p.dh) {
      to.s = row_raw<TYPE, EIGHTS>(p.s, row * p.lds, c, n);
      to.dh = row_raw<TYPE, EIGHTS>(p.dh, row * p.lddh, c, n);
    }
    if (p.b) to.b = row_raw<TYPE, EIGHTS>(p.b, row * p.ldb, c, n);
    if (p.gate) {
      const unsigned g = (unsigned)row / (unsigned)p.gate_rows;
      if (before < 0 || g != (unsigned)before / (unsigned)p.gate_rows) to.gate = row_raw<TYPE, EIGHTS>(p.gate, (long long)g * p.ldgate, c, n);
    }
  };
  long long row = run.first + begin;
  int left = span;
  Row at = {};
  if (AHEAD && row < run.end) load(at, row, -1);
  while (row - begin < run.end) {  // all teams as often as the first one, for their meetings
    const bool live = row < run.end, turn = left == 1;
    const long long next = row + 1 + (turn ? skip : 0);
    left = turn ? span : left - 1;
    Row ahead;
    if constexpr (AHEAD) {
      ahead = at;
      if (next < run.end) load(ahead, next, row);
    } else {
      load(at, row, -1);
    }

    f32x8 ds = {}, dh = {}, n_s = {}, n_b = {}, dn = {};
    if (p.ds) ds = settled<TYPE, EIGHTS>(at.ds, c, n);
    if (p.dh) {
      dh = settled<TYPE, EIGHTS>(at.dh, c, n);
      n_s = settled<TYPE, EIGHTS>(at.s, c, n);
      dn = dh * __builtin_convertvector(raw_before, f32x8);
    }
    if (p.b) n_b = settled<TYPE, EIGHTS>(at.b, c, n);
    float level_s = 0.f;
    const bool layer_s = p.dh && p.before == CCT_NORM_LAYER, layer_b = block && p.after == CCT_NORM_LAYER;
    if (layer_s || layer_b) {
      float t[3] = {sum8(n_s), sum8(dn), sum8(n_b)};
      total(t);
      if (layer_s) {
        n_s = first_of(n_s - t[0] / D, n);
        level_s = t[1] / D;
      }
      if (layer_b) n_b = first_of(n_b - t[2] / D, n);
    }
    float t[3] = {sum8(n_s * n_s), sum8(n_s * dn), sum8(n_b * n_b)};
    if (p.dh || block) total(t);
    if (p.dh) {
      const float rstd = rstd_of(t[0], p.D, p.eps);
      n_s *= rstd;
      ds += (dn - n_s * (t[1] * rstd / D) - level_s) * rstd;
      // the level is subtracted behind the row's end too, where nothing may come from: without a gate and w_after db's mean would hold it
      if (layer_s) ds = first_of(ds, n);
    }
    if (live) {
      if (p.dr) store_row<TYPE, EIGHTS>(p.dr, row * p.lddr + c, ds, n);
      add(std::integral_constant<int, kDcBefore>(), dh);
      add(std::integral_constant<int, kDwBefore>(), dh * n_s);
    }
    f32x8 dp = ds * p.scale;
    const float rstd_b = block ? rstd_of(t[2], p.D, p.eps) : 1.f;
    if (block) n_b *= rstd_b;
    const f32x8 w_after = __builtin_convertvector(raw_after, f32x8);
    if (p.gate) {
      if (p.out[kDgate] && live) {
        sums.v[kDgate] += dp * (n_b * w_after + __builtin_convertvector(raw_c, f32x8));
        if (plan.whole && (turn || row + 1 == run.end)) {
          store_row<TYPE, EIGHTS>(p.out[kDgate], (long long)((unsigned)row / (unsigned)p.gate_rows) * p.lddgate + c, sums.v[kDgate], n);
          sums.v[kDgate] = f32x8{};
        }
      }
      dp *= settled<TYPE, EIGHTS>(at.gate, c, n);
    }
    if (block) {
      if (live) {
        add(std::integral_constant<int, kDcAfter>(), dp);
        add(std::integral_constant<int, kDwAfter>(), dp * n_b);
      }
      if (p.db) {
        dp *= w_after;
        float u[2] = {sum8(dp * n_b), sum8(dp)};
        total(u);
        dp = (dp - n_b * (u[0] / D) - (layer_b ? u[1] / D : 0.f)) * rstd_b;
      }
    }
    if (p.db && live) store_row<TYPE, EIGHTS>(p.db, row * p.lddb + c, dp, n);
    if constexpr (AHEAD) at = ahead;
    row = next;
  }

#pragma unroll
  for (int k = 0; k < kNormSums; ++k) {
    if (!p.out[k] || (k == kDgate && plan.whole)) continue;
    if constexpr (IN_LDS)
      if (k != kDgate) sums.v[k] = __builtin_shufflevector(*own(k, 0), *own(k, 1), 0, 1, 2, 3, 4, 5, 6, 7);
    if (AHEAD && teams > 1) {
      if (team > 0) *(f32x8*)&meet[((team - 1) * waves * 64 + thread) * 8] = sums.v[k];
      __syncthreads();
      if (team == 0)
        for (int t = 1; t < teams; ++t) sums.v[k] += *(const f32x8*)&meet[((t - 1) * waves * 64 + thread) * 8];
      __syncthreads();
      if (team > 0) continue;
    }
    if (plan.count == 1)  // nothing to join
      store_first<TYPE>(p.out[k], c, sums.v[k], n);
    else
      store_first<CCT_TYPE_F32>((char*)part + k * plan.part_bytes, (long long)blockIdx.x * p.D + c, sums.v[k], n);
  }
}

// The runs' sums, added in order: 32 columns of one result, 8 threads a column.  blockIdx.y: four vectors, then the gate's rows.
// Bound by the trip to memory (256 runs of 4096 columns, five results, 21 MB: 5 us).
constexpr int kJoinRows = 8;
template <int TYPE>
__global__ __launch_bounds__(kJoinRows * 32) void residual_norm_join_kernel(ResidualNormBack p, ResidualNormPlan plan,
                                                                            const float* __restrict__ part) {
  __shared__ float lds[kJoinRows][33];
  const int k = min((int)blockIdx.y, (int)kDgate), group = (int)blockIdx.y - k;
  if (!p.out[k]) return;
  const int rows = k == kDgate ? plan.per_gate : plan.count, x = threadIdx.x & 31, y = threadIdx.x >> 5;
  for (long long c = blockIdx.x * 32LL + x; c - x < p.D; c += gridDim.x * 32LL) {
    const float* from = (const float*)((const char*)part + k * plan.part_bytes) + (long long)group * rows * p.D + c;
    float v[4] = {};  // four chains: one waits for itself
    if (c < p.D) {
      int r = y;
#pragma unroll 2
      for (; r + 3 * kJoinRows < rows; r += 4 * kJoinRows)
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] += from[(long long)(r + q * kJoinRows) * p.D];
      for (; r < rows; r += kJoinRows) v[0] += from[(long long)r * p.D];
    }
    lds[y][x] = (v[0] + v[1]) + (v[2] + v[3]);
    __syncthreads();
#pragma unroll
    for (int half = kJoinRows / 2; half > 0; half >>= 1) {
      if (y < half) lds[y][x] += lds[y + half][x];
      __syncthreads();
    }
    if (y == 0 && c < p.D) store1<TYPE>(p.out[k], k == kDgate ? group * p.lddgate + c : c, lds[0][x]);
    __syncthreads();
  }
}

constexpr int kRowsAhead = 512;  // workgroups, two a CU, of rows that leave no room for more
int norm_teams(int D, int type) {
  const int waves = pieces(D, 512);
  return waves == 1 ? kNormTeams : type != CCT_TYPE_F32 && (waves == 5 || waves == 6) ? 2 : 1;
}
int row_threads(int D) { return std::min(kMostWaves, pieces(D, 512)) * 64; }
double forward_bytes(const ResidualNorm& p) {
  return (double)type_bytes(p.type) * p.M * p.D * (1 + (p.b != nullptr) + (p.s != nullptr) + (p.h != nullptr));
}

}  // namespace

ResidualNormPlan residual_norm_plan(const cct_residual_norm_desc_t& d) {
  ResidualNormPlan p = {};
  // as many runs as the chip takes at a time: a CU has places for 12 waves of residual_norm_back_kernel (fp32: 8), three for each
  // of its SIMDs; of workgroups of more than four waves one
  const int waves = d.D <= 512 ? kNormTeams : pieces(d.D, 512), places = d.type == CCT_TYPE_F32 ? 8 : 12;
  const int most = 256 * (waves <= 4 ? std::min(3, places / waves) : 1);
  // (four rows a run at least, so that the runs' sums are little beside the rows, unless that leaves CUs idle: 4 x 6464 fp32 27 -> 16 us;
  // two rows are a run, which has nothing to join: 12.7 us, 15.5 as two)
  const int fewest = std::min(4, std::max(norm_teams(d.D, d.type), d.M <= 2 ? 2 : pieces(d.M, 256)));
  const int wanted = std::max(fewest, pieces(d.M, most)), shared = std::min(d.gate_rows, std::max(d.M, 1));
  p.whole = shared <= wanted;
  if (p.whole) {
    p.rows = pieces(wanted, shared) * shared;
    p.per_gate = 0;
    p.count = pieces(d.M, p.rows);
  } else {
    p.per_gate = std::max(1, std::min(pieces(shared, wanted), most / pieces(d.M, shared)));
    p.rows = pieces(shared, p.per_gate);
    p.count = pieces(d.M, shared) * p.per_gate;
  }
  auto up = [](long long v) { return (v + 255) / 256 * 256; };
  p.part_off = d.D <= kRegisterColumns ? 0 : up((long long)d.M * sizeof(RowStats));
  p.part_bytes = up((long long)p.count * d.D * 4);
  p.total = std::max(256LL, p.part_off + kNormSums * p.part_bytes);
  return p;
}

int launch_residual_norm(const ResidualNorm& p, hipStream_t st) {
  const int threads = row_threads(p.D);
  if (p.D <= kRegisterColumns) {
    ProfScope ps("residual_norm_kernel", 0.0, forward_bytes(p), st);
    const bool wave_rows = p.D <= 512;
    const int groups = std::min(wave_rows ? pieces(p.M, kNormTeams) : p.M, 1 << 20);
    with_type(p.type, [&](auto type) {
      constexpr int TYPE = decltype(type)::value;
      with_bool(p.D % 8 == 0, [&](auto eights) {
        constexpr bool EIGHTS = decltype(eights)::value;
        if (p.D <= kRegisterColumns / 2)
          hipLaunchKernelGGL(HIP_KERNEL_NAME(residual_norm_kernel<TYPE, EIGHTS, false>), dim3(groups),
                             dim3(wave_rows ? kNormTeams * 64 : threads), 0, st, p, wave_rows);
        else
          hipLaunchKernelGGL(HIP_KERNEL_NAME(residual_norm_kernel<TYPE, EIGHTS, true>), dim3(std::min(groups, kRowsAhead)),
                             dim3(threads), 0, st, p, false);
      });
    });
    CCT_CHECK_LAUNCH();
    return CCT_OK;
  }
  ProfScope ps("residual_norm_long_kernel", 0.0, forward_bytes(p), st);
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
  if (p.M > 0 && p.D <= kRegisterColumns) {
    ProfScope ps("residual_norm_back_kernel", 0.0,
                 all * ((p.ds != nullptr) + 2 * (p.dh != nullptr) + (p.b != nullptr) + (p.dr != nullptr) + (p.db != nullptr)), st);
    int rc = CCT_OK;
    with_type(p.type, [&](auto type) {
      constexpr int TYPE = decltype(type)::value;
      const int teams = norm_teams(p.D, TYPE), threads = teams * pieces(p.D, 512) * 64;
      with_bool(p.D % 8 == 0, [&](auto eights) {
        constexpr bool EIGHTS = decltype(eights)::value;
        auto run = [&](auto most) {
          constexpr int THREADS = decltype(most)::value;
          const int lds = norm_sums_in_lds<THREADS> ? kDgate * THREADS * 32 : 0;
          if (lds) rc = ensure_dynamic_lds<residual_norm_back_kernel<TYPE, THREADS, EIGHTS>>(lds);
          if (rc == CCT_OK)
            hipLaunchKernelGGL(HIP_KERNEL_NAME(residual_norm_back_kernel<TYPE, THREADS, EIGHTS>), dim3(plan.count), dim3(threads), lds,
                               st, p, plan, part);
        };
        if (threads <= 512) return run(std::integral_constant<int, 512>());
        if constexpr (TYPE != CCT_TYPE_F32)
          if (teams == 2) return run(std::integral_constant<int, 768>());
        run(std::integral_constant<int, 1024>());
      });
    });
    if (rc != CCT_OK) return rc;
    CCT_CHECK_LAUNCH();
    if (plan.count == 1) return CCT_OK;
  } else if (p.M > 0) {
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
                         dim3(pieces(p.D, kColumnThreads * 8), plan.count), dim3(kColumnThreads), 0, st, p, plan, stats, part);
    });
    CCT_CHECK_LAUNCH();
  }
  const bool vectors = p.out[kDcBefore] || p.out[kDwBefore] || p.out[kDcAfter] || p.out[kDwAfter];
  const bool gate = p.out[kDgate] && !plan.whole && p.M > 0;
  if (vectors || gate) {
    ProfScope ps("residual_norm_join_kernel", 0.0, 0.0, st);
    with_type(p.type, [&](auto type) {
      hipLaunchKernelGGL(HIP_KERNEL_NAME(residual_norm_join_kernel<decltype(type)::value>),
                         dim3(std::min(pieces(p.D, 32), 1 << 20), kDgate + (gate ? plan.count / plan.per_gate : 0)),
                         dim3(kJoinRows * 32), 0, st, p, plan, part);
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
