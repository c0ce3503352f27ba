// A layer of experts for a few tokens (cct_moe_forward), which is bound by reading the weights of the experts that some token
// chooses, each once.  Four launches:
//   moe_logits_kernel  a workgroup an expert and up to 8 tokens: the router's sums in 64 bits, so that which expert is chosen does
//                      not hang on their order (products of 16-bit values are exact);
//   moe_route_kernel   one workgroup: a wave a token, its chosen experts by rounds of a largest key, their weights; the list of
//                      experts that are used, and for each the rows of h of its tokens;
//   moe_gated_kernel   16 columns of both gate and up of one used expert and all its tokens: weight * act(g) * u, kept as two 16-bit
//                      terms (16 bits of a value in bf16, 22 in fp16; fp32 as it is), which the next product multiplies both;
//   moe_down_kernel    16 columns of y and all tokens, the contraction over all used experts' features.
// The two products are those of few rows (ff_rows.hip): weights go from memory into the registers of the matrix cores, waves take
// steps in turn, their sums meet in LDS in a fixed order.  A token that an expert is not for keeps its sum: zeros in its place
// would turn an infinite weight into NaN.
#include <algorithm>

#include "activation.h"
#include "ff_step.h"
#include "ff_tile.h"

namespace cct {
namespace {

constexpr int kMostTokens = 64, kMostExperts = 512, kMostChosen = 16;

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
  int* used;        // number of used experts, then their numbers
  short* rows;      // for each used expert and token its row of h, or -1
  float* weight;    // of each row of h
  void *h, *h_low;  // T k rows of Fp values: the terms; fp32: h alone
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
  __shared__ double sums[4][kLogitTokens];
#pragma unroll
  for (int t = 0; t < kLogitTokens; ++t) {
    if (t >= tokens) break;
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) sum[t] += __shfl_xor(sum[t], off, 64);
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6][t] = sum[t];
  }
  __syncthreads();
  const int t = threadIdx.x;
  if (t < tokens) a.logits[(long long)(t0 + t) * a.E + e] = (float)((sums[0][t] + sums[1][t]) + (sums[2][t] + sums[3][t]));
}

// Keys that order logits as numbers, the largest first, equal ones by the lower expert, NaN behind all others.
__device__ __forceinline__ unsigned long long logit_key(float v, int e) {
  v = v == 0.f ? 0.f : v;  // -0 is 0
  const unsigned b = __builtin_bit_cast(unsigned, v), up = v != v ? 0u : b >> 31 ? ~b : b | 0x80000000u;
  return (unsigned long long)up << 32 | (0xffffffffu - (unsigned)e);
}
constexpr int kRouteThreads = 1024, kOwn = kMostExperts / 64;
__global__ __launch_bounds__(kRouteThreads) void moe_route_kernel(Moe a) {
  __shared__ short chosen[kMostTokens][kMostChosen];
  __shared__ unsigned long long tokens_of[kMostExperts];
  __shared__ int used[kMostExperts], count;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int e = threadIdx.x; e < a.E; e += kRouteThreads) tokens_of[e] = 0;
  __syncthreads();
  for (int t = wave; t < a.T; t += kRouteThreads / 64) {
    unsigned long long key[kOwn];  // 0: not there, or chosen
    float logit[kOwn];
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
      const int e = i * 64 + lane;
      logit[i] = e < a.E ? a.logits[(long long)t * a.E + e] : -INFINITY;
      key[i] = e < a.E ? logit_key(logit[i], e) : 0;
    }
    float most = 0.f, mine = 0.f;  // the largest logit; lane j: of the j-th chosen expert
    int which = 0;
    for (int j = 0; j < a.k; ++j) {
      unsigned long long best = key[0];
      float value = logit[0];
#pragma unroll
      for (int i = 1; i < kOwn; ++i)
        if (key[i] > best) {
          best = key[i];
          value = logit[i];
        }
#pragma unroll
      for (int off = 32; off > 0; off >>= 1) {
        const unsigned long long other = __shfl_xor(best, off, 64);
        const float theirs = __shfl_xor(value, off, 64);
        if (other > best) {
          best = other;
          value = theirs;
        }
      }
      const int e = (int)(0xffffffffu - (unsigned)best);
#pragma unroll
      for (int i = 0; i < kOwn; ++i)
        if (key[i] == best) key[i] = 0;
      if (j == 0) most = value;
      if (lane == j) {
        mine = value;
        which = e;
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
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off, 64);
    if (lane < a.k) {
      const float w = own / sum;
      chosen[t][lane] = (short)which;
      a.weight[t * a.k + lane] = w;
      if (a.chosen_out) a.chosen_out[t * a.k + lane] = which;
      if (a.weights_out) a.weights_out[t * a.k + lane] = w;
      atomicOr(&tokens_of[which], 1ull << t);
    }
  }
  __syncthreads();
  if (wave == 0) {
    int n = 0;
    for (int e0 = 0; e0 < a.E; e0 += 64) {
      const bool in = e0 + lane < a.E && tokens_of[min(e0 + lane, a.E - 1)] != 0;
      const unsigned long long who = __ballot(in);
      if (in) {
        const int at = n + __popcll(who & ((1ull << lane) - 1));
        used[at] = e0 + lane;
        a.used[1 + at] = e0 + lane;
      }
      n += __popcll(who);
    }
    if (lane == 0) a.used[0] = count = n;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < count * a.T; i += kRouteThreads) {
    const int s = i / a.T, t = i - s * a.T, e = used[s];
    int row = -1;
    if (tokens_of[e] >> t & 1)
      for (int j = 0; j < a.k; ++j)
        if (chosen[t][j] == e) row = t * a.k + j;
    a.rows[i] = (short)row;
  }
}

// Four neighbouring values of a row of h.
template <int TYPE>
__device__ __forceinline__ void store_terms(const Moe& a, long long at, const float (&v)[4]) {
  if constexpr (TYPE == CCT_TYPE_F32) {
    *(f32x4*)((float*)a.h + at) = f32x4{v[0], v[1], v[2], v[3]};
  } else {
    typedef typename Number<TYPE>::T T;
    typedef T T4 __attribute__((ext_vector_type(4)));
    T4 high, low;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      high[e] = (T)v[e];
      const float rest = v[e] - (float)high[e];
      low[e] = (T)(fabsf((float)high[e]) < INFINITY ? rest : 0.f);  // an infinity is one term
    }
    *(T4*)((T*)a.h + at) = high;
    *(T4*)((T*)a.h_low + at) = low;
  }
}

constexpr int kGatedWaves = 8;
// RM: blocks of 16 tokens that an expert may have
template <int TYPE, int RM>
__global__ __launch_bounds__(kGatedWaves * 64) void moe_gated_kernel(Moe a) {
  typedef Step<TYPE> S;
  typedef typename S::V V;
  constexpr int NW = kGatedWaves, BATCH = RM == 4 ? 4 : 8;
  __shared__ short token[kMostTokens], place[kMostTokens];
  __shared__ int tokens;
  __shared__ f32x4 sums[NW][2 * RM][64];
  const int slot = blockIdx.y, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int e = a.used[1 + slot];
  if (slot >= a.used[0]) return;
  if (wave == 0) {
    const int row = lane < a.T ? a.rows[slot * a.T + lane] : -1;
    const unsigned long long who = __ballot(row >= 0);
    if (row >= 0) {
      const int at = __popcll(who & ((1ull << lane) - 1));
      token[at] = (short)lane;
      place[at] = (short)row;
    }
    if (lane == 0) tokens = __popcll(who);
  }
  __syncthreads();
  const int n = tokens, f0 = blockIdx.x * 16, lo = lane & 15, kq = (lane >> 4) * S::CH;
  const long long f = min(f0 + lo, a.F - 1), g_at = e * a.wg.e + f * a.wg.ld, u_at = e * a.wu.e + f * a.wu.ld;
  long long x_at[RM];
#pragma unroll
  for (int i = 0; i < RM; ++i) x_at[i] = token[min(i * 16 + lo, n - 1)] * a.ldx;
  f32x4 acc[2][RM];
#pragma unroll
  for (int b = 0; b < 2; ++b)
#pragma unroll
    for (int i = 0; i < RM; ++i) acc[b][i] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int whole = a.D / S::K;
  V w[BATCH][2], x[BATCH][RM];
  for (int s0 = wave; s0 < whole; s0 += BATCH * NW) {
    // steps past the last one load it again and multiply zeros
#pragma unroll
    for (int q = 0; q < BATCH; ++q) {
      const long long k = (long long)min(s0 + q * NW, whole - 1) * S::K + kq;
      w[q][0] = S::load(a.wg.p, g_at + k);
      w[q][1] = S::load(a.wu.p, u_at + k);
#pragma unroll
      for (int i = 0; i < RM; ++i)
        if (i == 0 || i * 16 < n) x[q][i] = S::load(a.x, x_at[i] + k);
    }
    __builtin_amdgcn_sched_barrier(0);  // the loads in front of it are not moved behind
#pragma unroll
    for (int q = 0; q < BATCH; ++q) {
      const bool live = s0 + q * NW < whole;
#pragma unroll
      for (int i = 0; i < RM; ++i)
        if (i == 0 || i * 16 < n) {
          const V xv = live ? x[q][i] : V{};
#pragma unroll
          for (int b = 0; b < 2; ++b) acc[b][i] = S::mfma(live ? w[q][b] : V{}, xv, acc[b][i]);
        }
    }
  }
  if (a.D % S::K && whole % NW == wave) {
    const int k = whole * S::K + kq, left = max(0, min(S::CH, a.D - k));
    const V wv[2] = {S::part(a.wg.p, g_at + k, left), S::part(a.wu.p, u_at + k, left)};
#pragma unroll
    for (int i = 0; i < RM; ++i)
      if (i == 0 || i * 16 < n) {
        const V xv = S::part(a.x, x_at[i] + k, left);
#pragma unroll
        for (int b = 0; b < 2; ++b) acc[b][i] = S::mfma(wv[b], xv, acc[b][i]);
      }
  }
#pragma unroll
  for (int b = 0; b < 2; ++b)
#pragma unroll
    for (int i = 0; i < RM; ++i) sums[wave][b * RM + i][lane] = acc[b][i];
  __syncthreads();
  for (int i = wave; i < RM; i += NW) {
    const int m = i * 16 + lo, at = f0 + (lane >> 4) * 4;
    if (m >= n) continue;
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
    const int row = place[m];
    const float weight = a.weight[row];
#pragma unroll
    for (int c = 0; c < 4; ++c) g[c] = at + c < a.F ? g[c] * weight : 0.f;  // zeros up to whole steps
    store_terms<TYPE>(a, (long long)row * a.Fp + at, g);
  }
}

constexpr int kDownWaves = 16;
template <int TYPE, int RM>
__global__ __launch_bounds__(kDownWaves * 64) void moe_down_kernel(Moe a, FfProduct p) {
  typedef Step<TYPE> S;
  typedef typename S::V V;
  constexpr int NW = kDownWaves, TERMS = TYPE == CCT_TYPE_F32 ? 1 : 2, BATCH = RM == 4 ? 2 : RM == 2 ? 4 : 8;
  extern __shared__ __attribute__((aligned(16))) unsigned char moe_smem[];
  f32x4(*sums)[RM][64] = (f32x4(*)[RM][64])moe_smem;        // [NW]
  int* experts = (int*)(moe_smem + NW * RM * 1024);          // [slots]
  short* rows = (short*)(experts + a.slots);                 // [slots][T]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int count = a.used[0];
  for (int i = threadIdx.x; i < a.slots; i += NW * 64) experts[i] = a.used[1 + i];
  for (int i = threadIdx.x; i < a.slots * a.T; i += NW * 64) rows[i] = a.rows[i];
  __syncthreads();
  const int n0 = blockIdx.x * 16, lo = lane & 15, kq = (lane >> 4) * S::CH;
  const long long w_row = min(n0 + lo, a.D - 1) * a.wd.ld;
  f32x4 acc[RM];
#pragma unroll
  for (int i = 0; i < RM; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int whole = a.F / S::K, total = count * whole;
  V w[BATCH], h[BATCH][RM][TERMS];
  short row[BATCH][RM];
  auto fetch = [&](int q, int slot, long long k) {
#pragma unroll
    for (int i = 0; i < RM; ++i) {
      const int t = i * 16 + lo;
      row[q][i] = t < a.T ? rows[slot * a.T + t] : (short)-1;
      const long long at = max((int)row[q][i], 0) * (long long)a.Fp + k;
      h[q][i][0] = S::load(a.h, at);
      if constexpr (TERMS == 2) h[q][i][1] = S::load(a.h_low, at);
    }
  };
  auto multiply = [&](int q, const V& wv, bool live) {
#pragma unroll
    for (int i = 0; i < RM; ++i) {
      f32x4 s = acc[i];
#pragma unroll
      for (int t = 0; t < TERMS; ++t) s = S::mfma(wv, h[q][i][t], s);
      if (live && row[q][i] >= 0) acc[i] = s;  // else the token's sum stays as it is
    }
  };
  for (int s0 = wave; s0 < total; s0 += BATCH * NW) {
#pragma unroll
    for (int q = 0; q < BATCH; ++q) {
      const int step = min(s0 + q * NW, total - 1), slot = step / whole;
      const long long k = (long long)(step - slot * whole) * S::K + kq;
      w[q] = S::load(a.wd.p, experts[slot] * a.wd.e + w_row + k);
      fetch(q, slot, k);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int q = 0; q < BATCH; ++q) multiply(q, w[q], s0 + q * NW < total);
  }
  if (a.F % S::K)
    for (int slot = wave; slot < count; slot += NW) {
      const int k = whole * S::K + kq;
      w[0] = S::part(a.wd.p, experts[slot] * a.wd.e + w_row + k, max(0, min(S::CH, a.F - k)));
      fetch(0, slot, k);
      multiply(0, w[0], true);
    }
#pragma unroll
  for (int i = 0; i < RM; ++i) sums[wave][i][lane] = acc[i];
  __syncthreads();
  for (int i = wave; i < RM; i += NW) {
    f32x4 s = sums[0][i][lane];
#pragma unroll
    for (int q = 1; q < NW; ++q) s += sums[q][i][lane];
    const int m = i * 16 + lo, n = n0 + (lane >> 4) * 4;
    if (m >= a.T || n >= a.D) continue;
    float v[4] = {s[0], s[1], s[2], s[3]}, u[4] = {};
    finish<TYPE, kFfLinear>(p, m, n, v, u);
  }
}

template <int TYPE, int RM>
int launch(const Moe& a, const FfProduct& p, hipStream_t st) {
  const double size = type_bytes(TYPE), pairs = (double)a.T * a.k;
  {
    ProfScope ps("moe_logits_kernel", 2.0 * a.T * a.E * a.D, size * a.D * ((double)a.E + a.T), st);
    hipLaunchKernelGGL(HIP_KERNEL_NAME(moe_logits_kernel<TYPE>), dim3(a.E, pieces(a.T, kLogitTokens)), dim3(256), 0, st, a);
    CCT_CHECK_LAUNCH();
  }
  {
    ProfScope ps("moe_route_kernel", 0.0, 4.0 * a.T * a.E, st);
    hipLaunchKernelGGL(moe_route_kernel, dim3(1), dim3(kRouteThreads), 0, st, a);
    CCT_CHECK_LAUNCH();
  }
  {
    ProfScope ps("moe_gated_kernel", 4.0 * pairs * a.D * a.F, 2.0 * size * a.slots * (double)a.D * a.F, st);
    hipLaunchKernelGGL(HIP_KERNEL_NAME(moe_gated_kernel<TYPE, RM>), dim3(a.Fp / 16, a.slots), dim3(kGatedWaves * 64), 0, st, a);
    CCT_CHECK_LAUNCH();
  }
  constexpr auto down = moe_down_kernel<TYPE, RM>;
  const int most = kDownWaves * RM * 1024 + kMostExperts * (4 + 2 * RM * 16);
  const int rc = ensure_dynamic_lds<down>(most);
  if (rc != CCT_OK) return rc;
  ProfScope ps("moe_down_kernel", 2.0 * pairs * a.D * a.F, size * a.slots * (double)a.D * a.F, st);
  hipLaunchKernelGGL(down, dim3(pieces(a.D, 16)), dim3(kDownWaves * 64), kDownWaves * RM * 1024 + a.slots * (4 + 2 * a.T), st, a, p);
  CCT_CHECK_LAUNCH();
  return CCT_OK;
}
template <int TYPE>
int launch(const Moe& a, const FfProduct& p, hipStream_t st) {
  return a.T <= 16 ? launch<TYPE, 1>(a, p, st) : a.T <= 32 ? launch<TYPE, 2>(a, p, st) : launch<TYPE, 4>(a, p, st);
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
  a->used = (int*)take(4LL * (1 + a->slots));
  a->rows = (short*)take(2LL * a->slots * a->T);
  a->weight = (float*)take(4LL * a->T * a->k);
  a->h = take((long long)type_bytes(d.type) * a->T * a->k * a->Fp);
  a->h_low = take(d.type == CCT_TYPE_F32 ? 0 : 2LL * a->T * a->k * a->Fp);
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
