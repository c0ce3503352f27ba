// Forward products of few rows (serving: one token, or a batch of sequences with one each): the weights are read once and
// nothing else matters.
//
// A workgroup takes 16 rows of the weight (gated: of both) and all rows of x, its waves (eight; fp32 with up to 16 rows
// sixteen) one step of the contraction after the other: 64 bytes of each weight row, which go from memory straight into the
// registers that the matrix cores take (32 values of 16 bits per instruction, 4 of fp32 in an order of their own that x
// follows).  No LDS and no meeting in the loop; eight steps' loads are in flight per wave, and x comes from L2 the same way.  The waves' sums meet in LDS in a fixed
// order.  fp32 runs on v_mfma_f32_16x16x4_f32, which memory outlasts.
//
// One row, bf16, other weights in every call, which come from memory: 4096 x 4096 8.9 us (3.8 TB/s; 6.8 at the rate of a large
// copy), 16384 x 4096 26.5 (5.1 TB/s), gated 2 x 8192 x 4096 28.8 (4.7); the same weights again and again, which the 256 MiB
// behind the L2s hold: 7.0 to 7.7, 22.6, 23.0 to 26.9.  fp32: 17.3, 54.3, 56.0.  What was tried (weights partly held):
// two batches of four steps in turn 9.0, 29.1 and 29.8 for 7.9, 25.6 and 27.0: the compiler waits for all of a batch before it
// loads the next one into the same registers, so that they are only smaller; sixteen waves 8.0, 26.8 and 26.8.  fp32, eight and
// sixteen waves: 18.7 and 16.6, 56.7 and 52.0, 62.5 and 56.5 (4096 x 16384).
//
// Few columns of long rows leave most CUs idle: the contraction is then cut into splits, whose sums ff_join_kernel adds (64
// outputs of 16384 inputs, bf16: 19.3 us on four CUs, 9.8 in eight splits).
//
// Any alignment: gfx950 loads 16 bytes at any address, at multiples of four as fast as at multiples of sixteen while memory is
// the bound.  16-bit rows that begin between them (up to 16 rows of x; with more the caller has such weights copied) are loaded
// from the words below and shifted: 4096 x 4096, bf16, rows 4097 apart, 1 / 16 rows of x: 16.1 / 20.2 us (other weights in
// every call 20.9 / 25.0), loaded as they lie 16.0 / 26.7, with a copy first 23 / 29.  A last step that is not whole is loaded value by value.
#include <algorithm>

#include "activation.h"
#include "feed_forward.h"
#include "ff_tile.h"

namespace cct {
namespace {

template <int TYPE>
struct Step {  // 16-bit types
  typedef s16x8 V;
  static constexpr int CH = 8, K = 32;  // values per lane, per step
  static __device__ __forceinline__ V load(const void* p, long long at) {
    typedef s16x8 U __attribute__((aligned(2)));
    return *(const U*)((const short*)p + at);
  }
  // Eight values at any even address, from the four words that hold the first seven and the eighth by itself.  The first word's
  // lower half may lie in front of the value, in the same four bytes and so in the same page.
  static __device__ __forceinline__ V load_odd(const void* p, long long at) {
    typedef int i32x4 __attribute__((ext_vector_type(4)));
    typedef i32x4 U __attribute__((aligned(4)));
    const unsigned long long a = (unsigned long long)((const short*)p + at);
    const i32x4 d = *(const U*)(a & ~3ull);
    const int last = ((const unsigned short*)p)[at + 7], by = a & 2 ? 16 : 0;
    const i32x4 v = {(int)__builtin_amdgcn_alignbit(d[1], d[0], by), (int)__builtin_amdgcn_alignbit(d[2], d[1], by),
                     (int)__builtin_amdgcn_alignbit(d[3], d[2], by), by ? (int)__builtin_amdgcn_alignbit(last, d[3], 16) : d[3]};
    return __builtin_bit_cast(V, v);
  }
  static __device__ __forceinline__ V part(const void* p, long long at, int n) {
    V v = {};
#pragma unroll
    for (int e = 0; e < CH; ++e)
      if (e < n) v[e] = ((const short*)p)[at + e];
    return v;
  }
  static __device__ __forceinline__ f32x4 mfma(V w, V x, f32x4 c) { return tile_mfma<TYPE>(w, x, c); }
};
template <>
struct Step<CCT_TYPE_F32> {
  typedef f32x4 V;
  static constexpr int CH = 4, K = 16;
  static __device__ __forceinline__ V load(const void* p, long long at) {
    typedef f32x4 U __attribute__((aligned(4)));
    return *(const U*)((const float*)p + at);
  }
  static __device__ __forceinline__ V part(const void* p, long long at, int n) {
    V v = {};
#pragma unroll
    for (int e = 0; e < CH; ++e)
      if (e < n) v[e] = ((const float*)p)[at + e];
    return v;
  }
  static __device__ __forceinline__ f32x4 mfma(V w, V x, f32x4 c) {
#pragma unroll
    for (int e = 0; e < CH; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(w[e], x[e], c, 0, 0, 0);
    return c;
  }
};

// RM: blocks of 16 rows of x
template <int TYPE, int RM>
constexpr int kWaves = TYPE == CCT_TYPE_F32 && RM == 1 ? 16 : 8;

// SPLIT: the contraction is cut (a form of its own: what tells it how is a cache line of arguments more, 0.6 of 8 us)
template <int TYPE, int RM, int EPI, bool SPLIT, bool ODD>
__global__ __launch_bounds__((kWaves<TYPE, RM> * 64)) void ff_rows_kernel(FfProduct p, FfPart part) {
  typedef Step<TYPE> S;
  typedef typename S::V V;
  constexpr int NB = EPI == kFfGated ? 2 : 1, BATCH = RM == 4 ? 4 : 8;
  constexpr int NW = kWaves<TYPE, RM>;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int split = SPLIT ? blockIdx.y : 0, n0 = blockIdx.x * 16, lo = lane & 15, kq = (lane >> 4) * S::CH;
  long long w_at = (long long)min(n0 + lo, p.N - 1) * p.B[0].ld, u_at = (long long)min(n0 + lo, p.N - 1) * p.B[NB - 1].ld, x_at[RM];
#pragma unroll
  for (int i = 0; i < RM; ++i) x_at[i] = (long long)min(i * 16 + lo, p.M - 1) * p.A[0].ld;

  f32x4 acc[NB][RM];
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int i = 0; i < RM; ++i) acc[b][i] = f32x4{0.f, 0.f, 0.f, 0.f};

  const int all = p.K / S::K, first = SPLIT ? split * part.stages : 0, whole = SPLIT ? min(all, first + part.stages) : all;  // steps
  V w[BATCH][NB], x[BATCH][RM];
  auto fetch = [](const void* from, long long at) {
    if constexpr (ODD)
      return S::load_odd(from, at);
    else
      return S::load(from, at);
  };
  // steps past the last one load it again and multiply zeros
  auto load = [&](int s0) {
#pragma unroll
    for (int q = 0; q < BATCH; ++q) {
      const long long k = (long long)min(s0 + q * NW, whole - 1) * S::K + kq;
      w[q][0] = fetch(p.B[0].p, w_at + k);
      if constexpr (NB == 2) w[q][1] = fetch(p.B[1].p, u_at + k);
#pragma unroll
      for (int i = 0; i < RM; ++i) x[q][i] = fetch(p.A[0].p, x_at[i] + k);
    }
  };
  auto multiply = [&](int s0) {
    __builtin_amdgcn_sched_barrier(0);  // the loads in front of it are not moved behind
#pragma unroll
    for (int q = 0; q < BATCH; ++q) {
      const bool live = s0 + q * NW < whole;
#pragma unroll
      for (int i = 0; i < RM; ++i) {
        const V xv = live ? x[q][i] : V{};
#pragma unroll
        for (int b = 0; b < NB; ++b) acc[b][i] = S::mfma(live ? w[q][b] : V{}, xv, acc[b][i]);
      }
    }
  };
  for (int s = first + wave; s < whole; s += BATCH * NW) {
    load(s);
    multiply(s);
  }
  if (p.K % S::K && (!SPLIT || split == part.splits - 1) && all % NW == wave) {
    const int k = all * S::K + kq, n = max(0, min(S::CH, p.K - k));
    V wv[NB];
    wv[0] = S::part(p.B[0].p, w_at + k, n);
    if constexpr (NB == 2) wv[1] = S::part(p.B[1].p, u_at + k, n);
#pragma unroll
    for (int i = 0; i < RM; ++i) {
      const V xv = S::part(p.A[0].p, x_at[i] + k, n);
#pragma unroll
      for (int b = 0; b < NB; ++b) acc[b][i] = S::mfma(wv[b], xv, acc[b][i]);
    }
  }

  __shared__ f32x4 sums[NW][NB * RM][64];
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int i = 0; i < RM; ++i) sums[wave][b * RM + i][lane] = acc[b][i];
  __syncthreads();
  for (int i = wave; i < RM; i += NW) {
    f32x4 s[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      s[b] = sums[0][b * RM + i][lane];
#pragma unroll
      for (int q = 1; q < NW; ++q) s[b] += sums[q][b * RM + i][lane];
    }
    const int m = i * 16 + lo, n = n0 + (lane >> 4) * 4;
    if (m >= p.M || n >= p.N) continue;
    if constexpr (SPLIT) {
#pragma unroll
      for (int b = 0; b < NB; ++b) *(f32x4*)(part.p + (((long long)split * NB + b) * p.M + m) * part.ld + n) = s[b];
      continue;
    }
    float v[4], u[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[e] = s[0][e];
      u[e] = s[NB - 1][e];
    }
    finish<TYPE, EPI>(p, m, n, v, u);
  }
}

int rows_splits(int N, int K, int type) {
  const int groups = pieces(N, 16), least = type == CCT_TYPE_F32 ? 1024 : 2048;  // steps of a split
  return groups > 64 || K < 4 * least ? 1 : std::min(128 / groups, K / least);
}

template <int TYPE, int EPI>
void launch(const FfProduct& p, float* ws, hipStream_t st) {
  const int groups = pieces(p.N, 16), steps = std::max(p.K / Step<TYPE>::K, 1);
  FfPart part = {ws, (p.N + 3) / 4 * 4, rows_splits(p.N, p.K, TYPE), 0};
  part.stages = (steps + part.splits - 1) / part.splits;
  part.splits = (steps + part.stages - 1) / part.stages;
  auto run = [&](auto rm, auto odd) {
    constexpr int RM = decltype(rm)::value;
    constexpr bool ODD = decltype(odd)::value;
    const dim3 grid(groups, part.splits), block(kWaves<TYPE, RM> * 64);
    if (part.splits > 1)
      hipLaunchKernelGGL(HIP_KERNEL_NAME(ff_rows_kernel<TYPE, RM, EPI, true, ODD>), grid, block, 0, st, p, part);
    else
      hipLaunchKernelGGL(HIP_KERNEL_NAME(ff_rows_kernel<TYPE, RM, EPI, false, ODD>), grid, block, 0, st, p, part);
  };
  constexpr bool F32 = TYPE == CCT_TYPE_F32;
  const bool words = F32 || (ff_words(p.A[0]) && ff_words(p.B[0]) && (EPI != kFfGated || ff_words(p.B[1])));
  if (p.M <= 16 && words)
    run(std::integral_constant<int, 1>(), std::false_type());
  else if (p.M <= 16)
    run(std::integral_constant<int, 1>(), std::integral_constant<bool, !F32>());
  else if (p.M <= 32 || F32)
    run(std::integral_constant<int, 2>(), std::false_type());
  else
    run(std::integral_constant<int, F32 ? 2 : 4>(), std::false_type());
  if (part.splits > 1)
    launch_join<TYPE, EPI>(p, part, st);
}
template <int TYPE>
void launch(const FfProduct& p, float* ws, hipStream_t st) {
  if (p.epilogue == kFfGated)
    launch<TYPE, kFfGated>(p, ws, st);
  else
    launch<TYPE, kFfLinear>(p, ws, st);
}

}  // namespace

bool ff_rows_fits(int N, int type) { return (long long)pieces(N, 16) * (type == CCT_TYPE_F32 ? 1024 : 512) <= kMostThreads; }

long long ff_rows_part_bytes(int M, int N, int K, int type, int epilogue) {
  const int splits = M <= kFfRowsMost ? rows_splits(N, K, type) : 1;
  return splits == 1 ? 0 : 4LL * splits * (epilogue == kFfGated ? 2 : 1) * M * ((N + 3) / 4 * 4);
}

int launch_ff_rows(const FfProduct& p, float* ws, hipStream_t st) {
  const double e = type_bytes(p.type), mn = (double)p.M * p.N, ops = p.epilogue == kFfGated ? 2 : 1;
  const double bytes = e * ((double)p.M * p.K + ops * p.N * p.K +
                            mn * (1 + (p.residual != nullptr) + (p.z != nullptr) + (p.z2 != nullptr)));
  ProfScope ps("ff_rows_kernel", 2.0 * mn * p.K * ops, bytes, st);
  if (p.type == CCT_TYPE_F32)
    launch<CCT_TYPE_F32>(p, ws, st);
  else if (p.type == CCT_TYPE_BF16)
    launch<CCT_TYPE_BF16>(p, ws, st);
  else
    launch<CCT_TYPE_F16>(p, ws, st);
  CCT_CHECK_LAUNCH();
  return CCT_OK;
}

}  // namespace cct
