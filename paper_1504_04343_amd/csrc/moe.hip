// A layer of experts for a few tokens (cct_moe_forward), which is bound by reading the weights of the experts that some token
// chooses, each once.  Launches:
//   moe_logits_kernel  a workgroup an expert and up to 8 tokens: the router's sums in 64 bits, so that which expert is chosen does
//                      not hang on their order (products of 16-bit values are exact);
//   moe_route_kernel   one workgroup: a wave a token, its chosen experts by rounds of a largest key, their weights; then the experts
//                      that are used, and for each the rows of h of its tokens (a single token: every wave of the next kernel
//                      chooses for itself, which takes less than a launch);
//   moe_gated_kernel   16 columns of both gate and up of one used expert and its tokens: weight * act(g) * u, in fp32;
//   moe_down_kernel    16 columns of one used expert's results and its tokens, or of all experts' for a single token (where that
//                      keeps the chip busy);
//   moe_join_kernel    (unless a workgroup had all experts') a token's results added in the order of its choice, and the residual.
// The two products are those of few rows (ff_rows.hip): weights go from memory into the registers of the matrix cores, waves take
// steps in turn, their sums meet in LDS in a fixed order.  A token's results do not depend on the other tokens.
//
// us of each kernel (within 2 %), bf16 (the last fp16):                          logits route gated down join   weights
//   1 token, 2 of 16 experts, 4096 -> 8192                                             5     -    53   31    -    403 MB
//   16 tokens, 4 of 64 experts, 2048 -> 2048                                           7     7   131   76    5   1038 MB
//   37 tokens, 3 of 24 experts, 1000 -> 1531, rows at odd distances                    7    10    35   34    5    219 MB
// The products read at 4.6 to 5.4 TB/s (fp32 too: 16 tokens, 4 of 64, 2048 -> 1024, 213 us in all) where there are weights enough to
// fill the chip; what is in front of and behind them are launches.
// Of the last line's workgroups, two or three rounds of which fill the chip, each waits for its tokens' numbers, weights and sums in turn.
#include <algorithm>

#include "activation.h"
#include "ff_step.h"
#include "ff_tile.h"
#include "split_bf16.h"
#include "wave_ops.h"

namespace cct {
namespace {

constexpr int kMostTokens = 64, kMostExperts = 512, kMostChosen = 16, kMostPairs = kMostTokens * kMostChosen;

struct MoeMatrix {
  const void* p;
  long long ld, e;  // values between rows, between experts
};
struct Moe {
  int T, E, k, D, F, Fp, slots, activation, normalize;
  const void *x, *router;
  long long ldx, ldrouter;
  MoeMatrix wg, wu, wd;
  // in the workspace
  float* logits;    // T x E
  short* chosen;    // T x k
  float* weight;    // of each of these
  int* slot;        // for each used expert its number and its tokens'; -1 behind them
  short* rows;      // kMostTokens for each: its tokens' rows (token * k + place among its chosen ones), the last again
  float* h;         // T k rows of Fp values
  short* terms;     // a single token's, 16-bit types: three rows for each of them
  float* part;      // T k rows of Dp results
  int Dp;
  int32_t* chosen_out;
  float* weights_out;
};

constexpr int kLogitTokens = 8;
template <int TYPE>
__global__ __launch_bounds__(256) void moe_logits_kernel(Moe a) {
  const int e = blockIdx.x, t0 = blockIdx.y * kLogitTokens, tokens = min(kLogitTokens, a.T - t0);
  double sum[kLogitTokens] = {};
  for (int c = threadIdx.x * 8; c < a.D; c += 256 * 8) {
    const f32x8 w = load_row<TYPE>(a.router, e * a.ldrouter, c, a.D - c);
#pragma unroll
    for (int t = 0; t < kLogitTokens; ++t)
      if (t < tokens) {
        const f32x8 x = load_row<TYPE>(a.x, (t0 + t) * a.ldx, c, a.D - c);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[t] = fma((double)w[i], (double)x[i], sum[t]);
      }
  }
  // eight sums over 64 lanes: halves of the lanes keep halves of the sums, then one is left in each lane
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int half = kLogitTokens / 2, off = 32; half > 0; half /= 2, off /= 2)
#pragma unroll
    for (int t = 0; t < half; ++t) {
      const bool upper = lane & off;
      const double give = upper ? sum[t] : sum[t + half], keep = upper ? sum[t + half] : sum[t];
      sum[t] = keep + __shfl_xor(give, off, 64);
    }
#pragma unroll
  for (int off = 32 / kLogitTokens; off > 0; off >>= 1) sum[0] += __shfl_xor(sum[0], off, 64);
  __shared__ double sums[4][kLogitTokens];
  if (lane % (64 / kLogitTokens) == 0) sums[threadIdx.x >> 6][lane / (64 / kLogitTokens)] = sum[0];
  __syncthreads();
  const int t = threadIdx.x;
  if (t < tokens) a.logits[(long long)(t0 + t) * a.E + e] = (float)((sums[0][t] + sums[1][t]) + (sums[2][t] + sums[3][t]));
}

// The chosen experts of a token, one wave: lane j < k has the j-th, largest logit first, equal ones by the lower expert, NaN last,
// and its weight.
constexpr int kOwn = kMostExperts / 64;
__device__ __forceinline__ void select_experts(const Moe& a, int t, int lane, int* which, float* weight) {
  // logits as whole numbers of the same order; 1: NaN, 0: not there or chosen already
  unsigned key[kOwn];
  float logit[kOwn];
#pragma unroll
  for (int i = 0; i < kOwn; ++i) {
    const int e = i * 64 + lane;
    logit[i] = e < a.E ? a.logits[(long long)t * a.E + e] : 0.f;
  }
#pragma unroll
  for (int i = 0; i < kOwn; ++i) {
    const float v = logit[i] == 0.f ? 0.f : logit[i];  // -0 is 0
    const unsigned b = __builtin_bit_cast(unsigned, v);
    key[i] = i * 64 + lane >= a.E ? 0u : v != v ? 1u : b >> 31 ? ~b : b | 0x80000000u;
  }
  float most = 0.f, mine = 0.f;
  *which = 0;
  for (int j = 0; j < a.k; ++j) {
    unsigned best = key[0], first = 0xffffffffu;
#pragma unroll
    for (int i = 1; i < kOwn; ++i)
      if (i * 64 < a.E) best = max(best, key[i]);
    best = wave_max(best);
#pragma unroll
    for (int i = kOwn - 1; i >= 0; --i)
      if (i * 64 < a.E) first = key[i] == best ? (unsigned)(i * 64 + lane) : first;
    first = wave_min(first);
#pragma unroll
    for (int i = 0; i < kOwn; ++i)
      if (i * 64 < a.E && (unsigned)(i * 64 + lane) == first) key[i] = 0;
    const float value = best == 1u ? NAN : __builtin_bit_cast(float, best >> 31 ? best ^ 0x80000000u : ~best);
    if (j == 0) most = value;
    if (lane == j) {
      mine = value;
      *which = (int)first;
    }
  }
  const float own = expf(mine - most);
  float sum = 0.f;
  if (a.normalize) {
    sum = lane < a.k ? own : 0.f;
  } else {
#pragma unroll
    for (int i = 0; i < kOwn; ++i) sum += i * 64 + lane < a.E ? expf(logit[i] - most) : 0.f;
  }
  *weight = own / wave_sum(sum);
}
__device__ __forceinline__ void write_selected(const Moe& a, int t, int lane, int which, float weight) {
  if (lane >= a.k) return;
  const int i = t * a.k + lane;
  a.chosen[i] = (short)which;
  a.weight[i] = weight;
  if (a.chosen_out) a.chosen_out[i] = which;
  if (a.weights_out) a.weights_out[i] = weight;
}
constexpr int kRouteThreads = 1024;
__global__ __launch_bounds__(kRouteThreads) void moe_route_kernel(Moe a) {
  __shared__ short chosen[kMostPairs];
  __shared__ unsigned long long tokens_of[kMostExperts];
  __shared__ int used[kMostExperts], total;
  __shared__ short row_of[kRouteThreads / 64][kMostTokens];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int e = threadIdx.x; e < a.E; e += kRouteThreads) tokens_of[e] = 0;
  __syncthreads();
  for (int t = wave; t < a.T; t += kRouteThreads / 64) {
    int which;
    float weight;
    select_experts(a, t, lane, &which, &weight);
    write_selected(a, t, lane, which, weight);
    if (lane < a.k) {
      chosen[t * a.k + lane] = (short)which;
      atomicOr(&tokens_of[which], 1ull << t);
    }
  }
  __syncthreads();
  if (wave == 0) {
    int n = 0;
    for (int e0 = 0; e0 < a.E; e0 += 64) {
      const bool in = e0 + lane < a.E && tokens_of[min(e0 + lane, a.E - 1)] != 0;
      const unsigned long long who = __ballot(in);
      if (in) used[n + __popcll(who & ((1ull << lane) - 1))] = e0 + lane;
      n += __popcll(who);
    }
    if (lane == 0) total = n;
  }
  __syncthreads();
  for (int s = wave; s < a.slots; s += kRouteThreads / 64) {
    const int e = s < total ? used[s] : -1;
    const unsigned long long tokens = e < 0 ? 0 : tokens_of[e];
    const int n = __popcll(tokens);
    if (lane == 0) {
      a.slot[2 * s] = e;
      a.slot[2 * s + 1] = n;
    }
    if (tokens >> lane & 1) {
      int j = 0;
      while (j < a.k - 1 && chosen[lane * a.k + j] != e) ++j;
      row_of[wave][__popcll(tokens & ((1ull << lane) - 1))] = (short)(lane * a.k + j);
    }
    __builtin_amdgcn_wave_barrier();
    if (n > 0) a.rows[s * kMostTokens + lane] = row_of[wave][min(lane, n - 1)];
    __builtin_amdgcn_wave_barrier();
  }
}

// h is fp32 in the second product too.  Beside 16-bit weights it is three bf16 numbers, each the eight leading bits of what is left, which
// together are the 24 bits of fp32 over its whole range (of numbers below 2^-110 the last bits are lost); an fp16 weight is two.  Two
// 16-bit terms of h were 16 bits in bf16, and in fp16 ended at 2^-24: 8 bits of a value of 1e-5, an infinity beyond 65504.  Values are
// split behind their load: terms in memory are half as much again for every workgroup to read (64 tokens, one expert, 4096 -> 8192:
// 184 us, split in registers 150).  Not a single token's, which are few: they lie beside h, and a term is a column of the product (2 of 16
// experts, 4096 -> 8192: 91.4 and 89.4 us, fp16 93.1 and 90.3).
template <int TYPE>
constexpr int kWeightTerms = TYPE == CCT_TYPE_F16 ? 2 : 1;
__device__ __forceinline__ float leading(float v) { return __uint_as_float(__float_as_uint(v) & 0xffff0000u); }
// The eight leading bits of values as bf16; v keeps the rest.
template <int N>
__device__ __forceinline__ void take_leading(float (&v)[N], unsigned (&to)[N / 2]) {
#pragma unroll
  for (int e = 0; e < N / 2; ++e) {
    to[e] = __builtin_amdgcn_perm(__float_as_uint(v[2 * e + 1]), __float_as_uint(v[2 * e]), 0x07060302u);
    v[2 * e] -= leading(v[2 * e]);
    v[2 * e + 1] -= leading(v[2 * e + 1]);
  }
}
__device__ __forceinline__ s16x8 next_term(float (&v)[8]) {
  unsigned to[4];
  take_leading(v, to);
  return __builtin_bit_cast(s16x8, u32x4{to[0], to[1], to[2], to[3]});
}
template <int TYPE>
__device__ __forceinline__ void weight_terms(s16x8 w, s16x8 (&to)[kWeightTerms<TYPE>]) {
  if constexpr (TYPE == CCT_TYPE_F16) {
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (float)__builtin_bit_cast(f16x8, w)[e];
    to[0] = next_term(v);
    to[1] = next_term(v);
  } else {
    to[0] = w;
  }
}

// What a lane has of h in a step, beside its weights; TERMS: it is one of its terms.
template <int TYPE, bool TERMS>
struct HStep {
  typedef float V __attribute__((ext_vector_type(Step<TYPE>::CH)));
};
template <int TYPE>
struct HStep<TYPE, true> {
  typedef s16x8 V;
};
template <int TYPE, bool TERMS, int RM>
__device__ __forceinline__ void multiply_h(typename Step<TYPE>::V w, const typename HStep<TYPE, TERMS>::V (&h)[RM], int tokens, f32x4 (&acc)[RM]) {
  if constexpr (TYPE == CCT_TYPE_F32) {
#pragma unroll
    for (int i = 0; i < RM; ++i)
      if (i == 0 || i * 16 < tokens) acc[i] = Step<TYPE>::mfma(w, h[i], acc[i]);
  } else {
    s16x8 wt[kWeightTerms<TYPE>];
    weight_terms<TYPE>(w, wt);
    auto add = [&](s16x8 term, f32x4& to) {
#pragma unroll
      for (int q = 0; q < kWeightTerms<TYPE>; ++q) to = tile_mfma<CCT_TYPE_BF16>(wt[q], term, to);
    };
#pragma unroll
    for (int i = 0; i < RM; ++i) {
      if (i > 0 && i * 16 >= tokens) continue;
      if constexpr (TERMS) {
        add(h[i], acc[i]);
      } else {
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = h[i][e];
#pragma unroll
        for (int t = 0; t < 3; ++t) add(next_term(v), acc[i]);
      }
    }
  }
}

// A step's operand from column k on of a row of n values, zeros behind its end: as it comes (of the last columns those that end with
// the row), and brought into place, which waits for it.
template <int TYPE>
__device__ __forceinline__ typename Step<TYPE>::V tail_raw(const void* p, long long row, int k, int n) {
  typedef Step<TYPE> S;
  if (n >= S::CH) return S::load(p, row + min(k, n - S::CH));
  return S::part(p, row, k == 0 ? n : 0);
}
template <int TYPE>
__device__ __forceinline__ typename Step<TYPE>::V tail_settled(typename Step<TYPE>::V v, int k, int n) {
  typedef Step<TYPE> S;
  const int left = n - k;
  if (left >= S::CH || n < S::CH) return v;
  if (left <= 0) return typename S::V{};
  if constexpr (TYPE == CCT_TYPE_F32) {
    const int by = S::CH - left;
    if (by & 1) v = f32x4{v[1], v[2], v[3], 0.f};
    if (by & 2) v = f32x4{v[2], v[3], 0.f, 0.f};
    return v;
  } else {
    return move_down(v, S::CH - left);
  }
}

// RM: blocks of 16 tokens that are multiplied at once; ONE: a single token, whose experts are not chosen yet; NW: waves
template <int TYPE, int RM, bool ONE, int NW>
__global__ __launch_bounds__(NW * 64) void moe_gated_kernel(Moe a) {
  typedef Step<TYPE> S;
  typedef typename S::V V;
  constexpr int BATCH = ONE ? 8 : 4;
  extern __shared__ __attribute__((aligned(16))) unsigned char moe_smem[];
  f32x4(*sums)[2 * RM][64] = (f32x4(*)[2 * RM][64])moe_smem;  // [NW]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int slot = blockIdx.y, lo = lane & 15;
  int e, all = 1, row[RM];  // the expert, its tokens, their rows of h
  float weight[RM];
  if constexpr (ONE) {
    int which;
    float of;
    select_experts(a, 0, lane, &which, &of);
    if (blockIdx.x == 0 && slot == 0 && wave == 0) {
      write_selected(a, 0, lane, which, of);
      if (lane < a.k) {
        a.slot[2 * lane] = which;
        a.slot[2 * lane + 1] = 1;
      }
      for (int j = 0; j < a.k; ++j) a.rows[j * kMostTokens + lane] = (short)j;
    }
    e = __builtin_amdgcn_readlane(which, slot);
    row[0] = slot;
    weight[0] = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, of), slot));
  } else {
    e = a.slot[2 * slot];
    all = a.slot[2 * slot + 1];
#pragma unroll
    for (int i = 0; i < RM; ++i) row[i] = a.rows[slot * kMostTokens + i * 16 + lo];
    if (e < 0) return;
  }
  const int f0 = blockIdx.x * 16, kq = (lane >> 4) * S::CH;
  const long long f = min(f0 + lo, a.F - 1), g_at = e * a.wg.e + f * a.wg.ld, u_at = e * a.wu.e + f * a.wu.ld;
  for (int m0 = 0; m0 < all; m0 += RM * 16) {
    const int n = all - m0;
    if constexpr (!ONE) {
      if (m0 > 0) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < RM; ++i) row[i] = a.rows[slot * kMostTokens + m0 + i * 16 + lo];
      }
#pragma unroll
      for (int i = 0; i < RM; ++i) weight[i] = a.weight[row[i]];
    }
    long long x_at[RM];
#pragma unroll
    for (int i = 0; i < RM; ++i) x_at[i] = ONE ? 0 : row[i] / a.k * a.ldx;
    f32x4 acc[2][RM];
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < RM; ++i) acc[b][i] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int whole = a.D / S::K, steps = (a.D + S::K - 1) / S::K;  // the last one may end within
    V w[BATCH][2], x[BATCH][RM];
    for (int s0 = wave; s0 < steps; s0 += BATCH * NW) {
#pragma unroll
      for (int q = 0; q < BATCH; ++q) {
        const int step = s0 + q * NW, k = step * S::K + kq;
        if (step >= steps) break;
        auto operand = [&](const void* p, long long at) { return step < whole ? S::load(p, at + k) : tail_raw<TYPE>(p, at, k, a.D); };
        w[q][0] = operand(a.wg.p, g_at);
        w[q][1] = operand(a.wu.p, u_at);
#pragma unroll
        for (int i = 0; i < RM; ++i)
          if (i == 0 || i * 16 < n) x[q][i] = i * 16 + lo < n ? operand(a.x, x_at[i]) : V{};  // lanes without a token ask for nothing
      }
      __builtin_amdgcn_sched_barrier(0);  // the loads in front of it are not moved behind
#pragma unroll
      for (int q = 0; q < BATCH; ++q) {
        const int step = s0 + q * NW, k = step * S::K + kq;
        if (step >= steps) break;
        if (step >= whole) {
#pragma unroll
          for (int b = 0; b < 2; ++b) w[q][b] = tail_settled<TYPE>(w[q][b], k, a.D);
#pragma unroll
          for (int i = 0; i < RM; ++i) x[q][i] = tail_settled<TYPE>(x[q][i], k, a.D);
        }
#pragma unroll
        for (int i = 0; i < RM; ++i)
          if (i == 0 || i * 16 < n)
#pragma unroll
            for (int b = 0; b < 2; ++b) acc[b][i] = S::mfma(w[q][b], x[q][i], acc[b][i]);
      }
    }
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < RM; ++i) sums[wave][b * RM + i][lane] = acc[b][i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < RM; ++i) {
      const int at = f0 + (lane >> 4) * 4;
      if (wave != i % NW || i * 16 + lo >= n) continue;
      float g[4], u[4];
      f32x4 s[2];
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        s[b] = sums[0][b * RM + i][lane];
#pragma unroll
        for (int q = 1; q < NW; ++q) s[b] += sums[q][b * RM + i][lane];
      }
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        g[c] = s[0][c];
        u[c] = s[1][c];
      }
      activate<true>(a.activation, g, u);
#pragma unroll
      for (int c = 0; c < 4; ++c) g[c] = at + c < a.F ? g[c] * weight[i] : 0.f;  // zeros up to whole steps
      *(f32x4*)(a.h + (long long)row[i] * a.Fp + at) = f32x4{g[0], g[1], g[2], g[3]};
      if constexpr (ONE && TYPE != CCT_TYPE_F32)
#pragma unroll
        for (int t = 0; t < 3; ++t) {
          unsigned term[2];
          take_leading(g, term);
          typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
          *(u32x2*)(a.terms + ((long long)row[i] * 3 + t) * a.Fp + at) = u32x2{term[0], term[1]};
        }
    }
  }
}

// The down product.  ONE: a single token, whose chosen experts' features are one contraction; else an expert and its tokens, whose
// results go to `part`.  A sum that is not finite may be one by the terms alone (0 times an infinite weight): it is formed again, of
// the values, in fp32.  One block of tokens has three steps on their way and five waves a SIMD: 16 tokens, 4 of 64 experts, 2048 ->
// 2048, 221 us, four steps and four waves 228 to 231.
template <int TYPE, int RM, bool ONE, int NW>
__global__ __launch_bounds__(NW * 64) __attribute__((amdgpu_waves_per_eu(ONE ? 4 : RM == 1 ? 5 : 2)))
void moe_down_kernel(Moe a, FfProduct p) {
  typedef Step<TYPE> S;
  typedef typename S::V V;
  constexpr bool TERMS = ONE && TYPE != CCT_TYPE_F32;  // of h are there: lanes 0 to 2 of 16 have one each
  typedef typename HStep<TYPE, TERMS>::V H;
  constexpr int BATCH = ONE ? 8 : RM == 4 ? 2 : RM == 1 ? 3 : 4;
  static_assert(!ONE || RM == 1, "one token");
  extern __shared__ __attribute__((aligned(16))) unsigned char moe_smem[];
  f32x4(*sums)[RM][64] = (f32x4(*)[RM][64])moe_smem;  // [NW]
  __shared__ short chosen[ONE ? kMostChosen : 1];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lo = lane & 15;
  int e = 0, all = 1, row[RM] = {};
  if constexpr (ONE) {
    if ((int)threadIdx.x < a.k) chosen[threadIdx.x] = a.chosen[threadIdx.x];
    __syncthreads();
  } else {
    e = a.slot[2 * blockIdx.y];
    all = a.slot[2 * blockIdx.y + 1];
#pragma unroll
    for (int i = 0; i < RM; ++i) row[i] = a.rows[blockIdx.y * kMostTokens + i * 16 + lo];
    if (e < 0) return;
  }
  const int count = ONE ? a.k : 1;  // experts
  const int n0 = blockIdx.x * 16, kq = (lane >> 4) * S::CH;
  const long long w_row = min(n0 + lo, a.D - 1) * a.wd.ld;
  for (int m0 = 0; m0 < all; m0 += RM * 16) {
    const int n = all - m0;
    if (m0 > 0) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < RM; ++i) row[i] = a.rows[blockIdx.y * kMostTokens + m0 + i * 16 + lo];
    }
    long long h_at[RM];
#pragma unroll
    for (int i = 0; i < RM; ++i) h_at[i] = row[i] * (long long)a.Fp;
    f32x4 acc[RM];
#pragma unroll
    for (int i = 0; i < RM; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int whole = a.F / S::K, steps = (a.F + S::K - 1) / S::K, total = count * steps;  // an expert's last step may end within
    V w[BATCH];
    H h[BATCH][RM];
    for (int s0 = wave; s0 < total; s0 += BATCH * NW) {
#pragma unroll
      for (int q = 0; q < BATCH; ++q) {
        const int at = s0 + q * NW, slot = ONE ? at / steps : 0, step = at - slot * steps, k = step * S::K + kq;
        if (at >= total) break;
        const long long row_of_w = (ONE ? (int)chosen[slot] : e) * a.wd.e + w_row;
        w[q] = step < whole ? S::load(a.wd.p, row_of_w + k) : tail_raw<TYPE>(a.wd.p, row_of_w, k, a.F);
#pragma unroll
        for (int i = 0; i < RM; ++i) {  // lanes without a token ask for nothing
          if (i > 0 && i * 16 >= n) continue;
          if constexpr (TERMS)
            h[q][i] = lo < 3 ? *(const H*)(a.terms + (slot * 3LL + lo) * a.Fp + k) : H{};
          else
            h[q][i] = i * 16 + lo < n ? *(const H*)(a.h + h_at[i] + (ONE ? slot * (long long)a.Fp : 0) + k) : H{};
        }
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int q = 0; q < BATCH; ++q) {
        const int at = s0 + q * NW, step = ONE ? at % steps : at;
        if (at >= total) break;
        if (step >= whole) w[q] = tail_settled<TYPE>(w[q], step * S::K + kq, a.F);
        multiply_h<TYPE, TERMS, RM>(w[q], h[q], n, acc);
      }
    }
#pragma unroll
    for (int i = 0; i < RM; ++i) sums[wave][i][lane] = acc[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < RM; ++i) {
      const int m = i * 16 + lo, c = n0 + (lane >> 4) * 4;
      if (wave != i % NW) continue;
      const bool live = m < n && c < a.D;
      f32x4 s = sums[0][i][lane];
#pragma unroll
      for (int q = 1; q < NW; ++q) s += sums[q][i][lane];
      if constexpr (TERMS)
#pragma unroll
        for (int r = 0; r < 4; ++r) s[r] += __shfl_down(s[r], 1, 64) + __shfl_down(s[r], 2, 64);
      if constexpr (TYPE != CCT_TYPE_F32) {
#pragma unroll 1
        for (int r = 0; r < 4; ++r) {
          const float v = r == 0 ? s[0] : r == 1 ? s[1] : r == 2 ? s[2] : s[3];
          const bool again = live && c + r < a.D && !finite(v);
          if (!__any(again)) continue;
          struct Result {
            long long w, h;
          };
          const float exact = fp32_sum(
              again, count * a.F,
              [&](int of) {
                return Result{(n0 + (of >> 4) * 4 + r) * a.wd.ld, __shfl(row[i], of & 15, 64) * (long long)a.Fp};
              },
              [&](const Result& to, int k, float* x, float* y) {
                const int slot = ONE ? k / a.F : 0, f = k - slot * a.F;
                *x = load1<TYPE>(a.wd.p, (ONE ? (int)chosen[slot] : e) * a.wd.e + to.w + f);
                *y = a.h[to.h + slot * (long long)a.Fp + f];
                return true;
              });
#pragma unroll
          for (int q = 0; q < 4; ++q) s[q] = again && q == r ? exact : s[q];
        }
      }
      if (!live) continue;
      if constexpr (ONE) {
        float v[4] = {s[0], s[1], s[2], s[3]}, u[4] = {};
        finish<TYPE, kFfLinear>(p, m, c, v, u);
      } else {
        *(f32x4*)(a.part + row[i] * (long long)a.Dp + c) = s;
      }
    }
  }
}

// A thread takes 4 columns of a token.
template <int TYPE>
__global__ __launch_bounds__(256) void moe_join_kernel(Moe a, FfProduct p) {
  const int t = blockIdx.y, c = ((int)blockIdx.x * 256 + (int)threadIdx.x) * 4;
  if (c >= a.D) return;
  const float* from = a.part + (long long)t * a.k * a.Dp + c;
  f32x4 s = *(const f32x4*)from;
#pragma unroll 4
  for (int j = 1; j < a.k; ++j) s += *(const f32x4*)(from + (long long)j * a.Dp);
  float v[4] = {s[0], s[1], s[2], s[3]}, u[4] = {};
  finish<TYPE, kFfLinear>(p, t, c, v, u);
}

template <auto KERNEL, class... ARGS>
int launch_with_lds(dim3 grid, int threads, int lds, hipStream_t st, ARGS... args) {
  const int rc = ensure_dynamic_lds<KERNEL>(lds);
  if (rc != CCT_OK) return rc;
  hipLaunchKernelGGL(KERNEL, grid, dim3(threads), lds, st, args...);
  CCT_CHECK_LAUNCH();
  return CCT_OK;
}

// Waves that a contraction of so many steps feeds (16 tokens, 8 of 64 experts, 1024 -> 512, bf16: 61 us, with eight always 67; 39, 8 of 99,
// 2648 -> 141: 103 and 131; from 32 steps on eight are the fastest: 2 of 16, 4096 -> 8192: 89 us, with four 109).
template <class F>
void with_waves(int steps, F f) {
  if (steps <= 8)
    f(std::integral_constant<int, 2>());
  else if (steps <= 24)
    f(std::integral_constant<int, 4>());
  else
    f(std::integral_constant<int, 8>());
}

template <int TYPE, int RM>
int launch(const Moe& a, const FfProduct& p, hipStream_t st) {
  const double size = type_bytes(TYPE), pairs = (double)a.T * a.k;
  {
    ProfScope ps("moe_logits_kernel", 2.0 * a.T * a.E * a.D, size * a.D * ((double)a.E + a.T), st);
    hipLaunchKernelGGL(HIP_KERNEL_NAME(moe_logits_kernel<TYPE>), dim3(a.E, pieces(a.T, kLogitTokens)), dim3(256), 0, st, a);
    CCT_CHECK_LAUNCH();
  }
  if (a.T > 1) {
    ProfScope ps("moe_route_kernel", 0.0, 4.0 * a.T * a.E, st);
    hipLaunchKernelGGL(moe_route_kernel, dim3(1), dim3(kRouteThreads), 0, st, a);
    CCT_CHECK_LAUNCH();
  }
  int rc;
  {
    ProfScope ps("moe_gated_kernel", 4.0 * pairs * a.D * a.F, 2.0 * size * a.slots * (double)a.D * a.F, st);
    const dim3 grid(a.Fp / 16, a.slots);
    with_waves(pieces(a.D, Step<TYPE>::K), [&](auto waves) {
      constexpr int NW = decltype(waves)::value, lds = NW * 2 * 1024;
      rc = a.T == 1 ? launch_with_lds<moe_gated_kernel<TYPE, 1, true, NW>>(grid, NW * 64, lds, st, a)
                    : launch_with_lds<moe_gated_kernel<TYPE, RM, false, NW>>(grid, NW * 64, lds * RM, st, a);
    });
    if (rc != CCT_OK) return rc;
  }
  const int tiles = pieces(a.D, 16);
  {
    ProfScope ps("moe_down_kernel", 2.0 * pairs * a.D * a.F, size * a.slots * (double)a.D * a.F, st);
    const int steps = pieces(a.F, Step<TYPE>::K);
    // a single token's experts one after the other, unless that leaves half of the CUs idle for longer than a join takes (a step of a
    // workgroup 0.045 us; 8 of 32 experts, 1024 -> 4096 and back: 64 us, 95 one after the other)
    if (a.T == 1 && (tiles > 128 || (a.k - 1) * steps < 128))
      return launch_with_lds<moe_down_kernel<TYPE, 1, true, 16>>(dim3(tiles), 1024, 16 * 1024, st, a, p);
    with_waves(steps, [&](auto waves) {
      constexpr int NW = decltype(waves)::value;
      rc = launch_with_lds<moe_down_kernel<TYPE, RM, false, NW>>(dim3(tiles, a.slots), NW * 64, NW * RM * 1024, st, a, p);
    });
    if (rc != CCT_OK) return rc;
  }
  ProfScope ps("moe_join_kernel", 0.0, 4.0 * pairs * a.D + size * a.T * (double)a.D, st);
  hipLaunchKernelGGL(HIP_KERNEL_NAME(moe_join_kernel<TYPE>), dim3(pieces(a.Dp / 4, 256), a.T), dim3(256), 0, st, a, p);
  CCT_CHECK_LAUNCH();
  return CCT_OK;
}
template <int TYPE>
int launch(const Moe& a, const FfProduct& p, hipStream_t st) {
  // blocks of 16 tokens that a workgroup takes at once: more of an expert's come in further passes over its weights, from a cache, so
  // that there is room for twice the tokens that an expert has on average (37 tokens, 3 of 24 experts, gated: in one block 35 us, in
  // four, which leave half the loads in flight, 46)
  const int most = std::min(a.T, pieces(2 * a.T * a.k, a.E));
  return most <= 16 ? launch<TYPE, 1>(a, p, st) : most <= 32 ? launch<TYPE, 2>(a, p, st) : launch<TYPE, 4>(a, p, st);
}

int dims_ok(const cct_moe_desc_t& d) {
  if (d.tokens < 0 || d.experts < 1 || d.chosen < 1 || d.chosen > d.experts || d.D < 1 || d.F < 1 || !type_known(d.type) ||
      !activation_known(d.activation))
    return CCT_EINVAL;
  if (d.tokens > kMostTokens || d.experts > kMostExperts || d.chosen > kMostChosen) return CCT_EUNSUPPORTED;
  // a launch's threads, 32-bit places in a matrix's contraction
  if (std::max(d.D, d.F) > (1 << 24)) return CCT_EUNSUPPORTED;
  return (long long)d.D * d.F <= (1LL << 38) / type_bytes(d.type) ? CCT_OK : CCT_EUNSUPPORTED;
}

// The workspace's parts, from `ws`; their bytes.
long long lay_out(const cct_moe_desc_t& d, char* ws, Moe* a) {
  long long total = 0;
  auto take = [&](long long bytes) {
    char* at = ws + total;
    total += (bytes + 255) / 256 * 256;
    return (void*)at;
  };
  a->T = d.tokens;
  a->E = d.experts;
  a->k = d.chosen;
  a->D = d.D;
  a->F = d.F;
  a->Fp = (d.F + 31) / 32 * 32;
  a->slots = std::min(d.experts, d.tokens * d.chosen);
  a->activation = d.activation;
  a->normalize = d.normalize;
  a->logits = (float*)take(4LL * a->T * a->E);
  a->chosen = (short*)take(2LL * a->T * a->k);
  a->weight = (float*)take(4LL * a->T * a->k);
  a->slot = (int*)take(8LL * a->slots);
  a->rows = (short*)take(2LL * kMostTokens * a->slots);
  a->h = (float*)take(4LL * a->T * a->k * a->Fp);
  a->terms = (short*)take(a->T == 1 && d.type != CCT_TYPE_F32 ? 6LL * a->k * a->Fp : 0);
  a->Dp = (d.D + 3) / 4 * 4;
  a->part = (float*)take(4LL * a->T * a->k * a->Dp);
  return std::max(total, 256LL);
}

bool matrix_ok(const void* p, long long ld, long long rows, long long cols, int type) {
  return p && !((uintptr_t)p & (type_bytes(type) - 1)) && ld >= 0 && (rows <= 1 || ld >= cols);
}
bool experts_ok(const MoeMatrix& m, int experts, long long rows, long long cols, int type) {
  if (!matrix_ok(m.p, m.ld, rows, cols, type) || m.e < 0) return false;
  if (experts == 1) return true;
  // distances up to what no card holds, so that no product of them passes 63 bits
  if (m.ld > 1LL << 38 || m.e > 1LL << 40) return false;
  return m.e >= (rows - 1) * (rows > 1 ? m.ld : 0) + cols;
}

}  // namespace
}  // namespace cct

using namespace cct;

extern "C" {

int cct_moe_workspace_bytes(const cct_moe_desc_t* desc, size_t* bytes) {
  if (!desc || !bytes) return CCT_EINVAL;
  const int rc = dims_ok(*desc);
  if (rc != CCT_OK) return rc;
  Moe a = {};
  *bytes = (size_t)lay_out(*desc, nullptr, &a);
  return CCT_OK;
}

int cct_moe_forward(const cct_moe_desc_t* desc, const void* x, int64_t ldx, const void* router, int64_t ldrouter, const void* wg,
                    int64_t ldwg, int64_t wg_e, const void* wu, int64_t ldwu, int64_t wu_e, const void* wd, int64_t ldwd,
                    int64_t wd_e, const void* residual, int64_t ldr, void* y, int64_t ldy, int32_t* chosen_out,
                    float* weights_out, void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (!desc) return CCT_EINVAL;
  const cct_moe_desc_t& d = *desc;
  const int rc = dims_ok(d);
  if (rc != CCT_OK) return rc;
  if (d.tokens == 0) return CCT_OK;
  Moe a = {};
  a.wg = {wg, ldwg, wg_e};
  a.wu = {wu, ldwu, wu_e};
  a.wd = {wd, ldwd, wd_e};
  if (!matrix_ok(x, ldx, d.tokens, d.D, d.type) || !matrix_ok(router, ldrouter, d.experts, d.D, d.type) ||
      !experts_ok(a.wg, d.experts, d.F, d.D, d.type) || !experts_ok(a.wu, d.experts, d.F, d.D, d.type) ||
      !experts_ok(a.wd, d.experts, d.D, d.F, d.type) || (residual && !matrix_ok(residual, ldr, d.tokens, d.D, d.type)) ||
      !matrix_ok(y, ldy, d.tokens, d.D, d.type) || ((uintptr_t)chosen_out & 3) || ((uintptr_t)weights_out & 3))
    return CCT_EINVAL;
  if (!workspace || ((uintptr_t)workspace & 255)) return CCT_EINVAL;
  if (workspace_bytes < (size_t)lay_out(d, (char*)workspace, &a)) return CCT_EWORKSPACE;
  a.x = x;
  a.ldx = ldx;
  a.router = router;
  a.ldrouter = ldrouter;
  a.chosen_out = chosen_out;
  a.weights_out = weights_out;
  FfProduct p = {};
  p.M = d.tokens;
  p.N = d.D;
  p.K = d.F;
  p.type = d.type;
  p.activation = CCT_ACT_NONE;
  p.segments = 1;
  p.epilogue = kFfLinear;
  p.residual = residual;
  p.ldr = ldr;
  p.out = y;
  p.ldo = ldy;
  hipStream_t st = (hipStream_t)hip_stream;
  if (d.type == CCT_TYPE_F32) return launch<CCT_TYPE_F32>(a, p, st);
  return d.type == CCT_TYPE_BF16 ? launch<CCT_TYPE_BF16>(a, p, st) : launch<CCT_TYPE_F16>(a, p, st);
}

}  // extern "C"
