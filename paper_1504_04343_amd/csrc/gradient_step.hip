// From gradients to new weights over lists of tensors: the 2-norm of all gradients, the gradients scaled down to a largest
// norm, and the step with momentum and weight decay (Caffe's rules, as the other layers').
//
//   norm    n = sqrt(sum g^2), s = max_norm / n where n > max_norm, else 1
//   scale   out = s g
//   update  v = momentum v + rate (s g + decay w),  w = w - v,  copy = w rounded
//
// All of it is memory: the norm reads every gradient once, scaling reads and writes each, the update reads gradient, weight
// and moment and writes the latter two.  A model's list holds hundreds of tensors, most of them small, so that a launch
// takes as many as its arguments hold (4 KiB; nothing is uploaded or kept); a workgroup takes some thousand values of one of
// them.  Scaling and updating walk the lists from the end: what the norm read last is what the 256 MiB cache behind the
// eight L2s still holds, and what is written, and the weights and moments, which nobody reads again soon, go past it
// (nontemporal).  CaffeNet's 61 million fp32 gradients, us: norm 45 (5.4 TB/s), norm and scaling 117 (139 without, 141 from the
// beginning too), norm and update 218 (266, 274): 5.6 TB/s of gradients read once, weights and moments.
//
// The squares are summed in 64 bits: with 2^-53 per addition no order matters to the fp32 result, 3e38 squared does not
// overflow, and the kernel waits for memory all the same (4 conversions and fused multiply-adds per 16 bytes).  Every
// workgroup leaves one sum; one workgroup adds them in a fixed order, so that the norm is bit-reproducible.
#include <algorithm>
#include <cmath>

#include "cct_internal.h"
#include "number_types.h"

namespace cct {
namespace {

constexpr int NT = 256;

// What a launch is told: tensors with P pointers each, at which workgroup each begins, of which one takes RUN values, and how
// many values its last one takes.  Small, so that few launches do: what a tensor is follows from 6 bytes besides its pointers
// (400 tensors: two launches for the norm, three for scaling, four for the update; with 64-bit counts 3, 4 and 6, each of
// which costs 3 to 4 us before it streams).
template <int P, int COUNT, int RUN>
struct ListArgs {
  static constexpr int kCount = COUNT, kRun = RUN;
  static_assert(RUN <= 8192, "13 bits; 12 where there is a second type");
  void* p[P][COUNT];
  int first[COUNT + 1];
  unsigned short tail[COUNT];  // values of the last workgroup - 1, above three bits (RUN up to 4096: four) that hold p[0]'s
                               // type and, from bit 2 on, the copy's
  int count;
};
typedef ListArgs<1, 270, 8192> NormArgs;
typedef ListArgs<2, 172, 8192> ScaleArgs;
typedef ListArgs<4, 100, 4096> UpdateArgs;
static_assert(sizeof(NormArgs) < 3900 && sizeof(ScaleArgs) < 3900 && sizeof(UpdateArgs) < 3900, "a launch's arguments");

// which tensor workgroup b of the launch belongs to
template <class Args>
__device__ __forceinline__ int tensor_of(const Args& a, int b) {
  int lo = 0, hi = a.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.first[mid] <= b)
      lo = mid;
    else
      hi = mid - 1;
  }
  return lo;
}

// A workgroup's part of the list: tensor, its types, the first value and the number of them.
struct Run {
  int tensor, type, other, n;
  long long at;
};
template <class Args>
__device__ __forceinline__ Run run_of(const Args& a, int b) {
  Run r;
  r.tensor = tensor_of(a, b);
  const int k = b - a.first[r.tensor], tail = a.tail[r.tensor];
  r.type = tail & 3;
  r.other = tail >> 2 & 3;
  r.at = (long long)k * Args::kRun;
  r.n = b + 1 == a.first[r.tensor + 1] ? (Args::kRun > 4096 ? tail >> 3 : tail >> 4) + 1 : Args::kRun;
  return r;
}

template <class F>
__device__ __forceinline__ void with_type(int type, F f) {
  if (type == CCT_TYPE_F32)
    f(std::integral_constant<int, CCT_TYPE_F32>());
  else if (type == CCT_TYPE_BF16)
    f(std::integral_constant<int, CCT_TYPE_BF16>());
  else
    f(std::integral_constant<int, CCT_TYPE_F16>());
}

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
  return v;
}

// W values at any address that is a multiple of one of them
template <int TYPE, int W>
struct Some {
  typedef typename Number<TYPE>::T T;
  typedef T V __attribute__((ext_vector_type(W)));
  typedef V U __attribute__((aligned(sizeof(T))));
  typedef float F __attribute__((ext_vector_type(W)));
  static __device__ __forceinline__ V load(const T* p) { return *(const U*)p; }
  static __device__ __forceinline__ V load_once(const T* p) { return __builtin_nontemporal_load((const U*)p); }
  static __device__ __forceinline__ F wide(V v) { return __builtin_convertvector(v, F); }
  static __device__ __forceinline__ void store(T* p, F v) { __builtin_nontemporal_store(__builtin_convertvector(v, V), (U*)p); }
};
template <int TYPE>
constexpr int kLane = 16 / (int)sizeof(typename Number<TYPE>::T);  // values of a 16-byte load

// every(k, q): W values from k on, the q-th such piece of the thread's batch, B of which are visited by `first` before any of
// them is visited by `then`; one(k): the values behind the last whole piece.
template <int W, int B, class First, class Then, class One>
__device__ __forceinline__ void walk(int n, First first, Then then, One one) {
  int k = threadIdx.x * W;
  for (; k + ((B - 1) * NT + 1) * W <= n; k += B * NT * W) {
#pragma unroll
    for (int q = 0; q < B; ++q) first(k + q * NT * W, q);
#pragma unroll
    for (int q = 0; q < B; ++q) then(k + q * NT * W, q);
  }
  for (; k < n; k += NT * W)
    if (k + W <= n) {
      first(k, 0);
      then(k, 0);
    } else {
      for (int e = k; e < n; ++e) one(e);
    }
}

__global__ __launch_bounds__(NT) void grad_norm_kernel(NormArgs a, double* __restrict__ part) {
  const Run r = run_of(a, blockIdx.x);
  double part_sum[4] = {};  // four chains: one waits for itself
  with_type(r.type, [&](auto type) {
    constexpr int TYPE = decltype(type)::value, W = kLane<TYPE>, B = 4;
    typedef Some<TYPE, W> S;
    const typename S::T* g = (const typename S::T*)a.p[0][r.tensor] + r.at;
    auto add = [&](float v, int e) { part_sum[e & 3] = fma((double)v, (double)v, part_sum[e & 3]); };
    typename S::V v[B];
    walk<W, B>(
        r.n, [&](int k, int q) { v[q] = S::load(g + k); },
        [&](int, int q) {
          const typename S::F f = S::wide(v[q]);
#pragma unroll
          for (int e = 0; e < W; ++e) add(f[e], e);
        },
        [&](int e) { add((float)g[e], 0); });
  });
  double sum = (part_sum[0] + part_sum[1]) + (part_sum[2] + part_sum[3]);
  __shared__ double sums[NT / 64];
  sum = wave_sum(sum);
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0) part[blockIdx.x] = (sums[0] + sums[1]) + (sums[2] + sums[3]);
}

constexpr int kFinalThreads = 1024;
__global__ __launch_bounds__(kFinalThreads) void grad_norm_final_kernel(const double* __restrict__ part, int n,
                                                                        float max_norm, float* __restrict__ clip) {
  double sum = 0.0;
  for (int k = threadIdx.x; k < n; k += kFinalThreads) sum += part[k];
  __shared__ double sums[kFinalThreads / 64];
  sum = wave_sum(sum);
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x != 0) return;
  for (int w = 1; w < kFinalThreads / 64; ++w) sum += sums[w];
  const double norm = sqrt(sum);
  clip[0] = (float)norm;
  clip[1] = norm != norm ? (float)norm : norm > (double)max_norm ? (float)((double)max_norm / norm) : 1.f;
}

__global__ __launch_bounds__(NT) void grad_scale_kernel(ScaleArgs a, const float* __restrict__ clip) {
  const Run r = run_of(a, (int)(gridDim.x - 1 - blockIdx.x));
  const float s = clip[1];
  if (a.p[0][r.tensor] == a.p[1][r.tensor] && s == 1.f) return;
  with_type(r.type, [&](auto type) {
    constexpr int TYPE = decltype(type)::value, W = kLane<TYPE>, B = 4;
    typedef Some<TYPE, W> S;
    const typename S::T* g = (const typename S::T*)a.p[0][r.tensor] + r.at;
    typename S::T* out = (typename S::T*)a.p[1][r.tensor] + r.at;
    typename S::V v[B];
    walk<W, B>(
        r.n, [&](int k, int q) { v[q] = S::load(g + k); }, [&](int k, int q) { S::store(out + k, S::wide(v[q]) * s); },
        [&](int e) { out[e] = (typename S::T)((float)g[e] * s); });
  });
}

struct StepRule {
  float rate, momentum, decay;
};

template <int TYPE, int COPY>  // COPY: the copy's type, -1 for none
__device__ __forceinline__ void update_run(const void* gp, float* w, float* v, void* cp, int n, float s, StepRule r) {
  constexpr int W = 4, B = 4;
  typedef Some<TYPE, W> G;
  typedef Some<CCT_TYPE_F32, W> S;
  typedef Some<COPY < 0 ? CCT_TYPE_F32 : COPY, W> C;
  const typename G::T* g = (const typename G::T*)gp;
  typename C::T* copy = (typename C::T*)cp;
  typename G::V gv[B];
  typename S::V wv[B], mv[B];
  walk<W, B>(
      n,
      [&](int k, int q) {
        gv[q] = G::load(g + k);
        wv[q] = S::load_once(w + k);
        mv[q] = S::load_once(v + k);
      },
      [&](int k, int q) {
        const typename S::F m = r.momentum * mv[q] + r.rate * (s * G::wide(gv[q]) + r.decay * wv[q]), t = wv[q] - m;
        S::store(v + k, m);
        S::store(w + k, t);
        if constexpr (COPY >= 0) C::store(copy + k, t);
      },
      [&](int e) {
        v[e] = r.momentum * v[e] + r.rate * (s * (float)g[e] + r.decay * w[e]);
        w[e] -= v[e];
        if constexpr (COPY >= 0) copy[e] = (typename C::T)w[e];
      });
}

__global__ __launch_bounds__(NT) void sgd_update_kernel(UpdateArgs a, const float* __restrict__ clip, StepRule rule) {
  const Run r = run_of(a, (int)(gridDim.x - 1 - blockIdx.x));
  const float s = clip ? clip[1] : 1.f;
  const int i = r.tensor;
  with_type(r.type, [&](auto type) {
    constexpr int TYPE = decltype(type)::value;
    const void* g = (const typename Number<TYPE>::T*)a.p[0][i] + r.at;
    float *w = (float*)a.p[1][i] + r.at, *v = (float*)a.p[2][i] + r.at;
    if (!a.p[3][i])
      update_run<TYPE, -1>(g, w, v, nullptr, r.n, s, rule);
    else
      with_type(r.other, [&](auto other) {
        constexpr int COPY = decltype(other)::value;
        update_run<TYPE, COPY>(g, w, v, (typename Number<COPY>::T*)a.p[3][i] + r.at, r.n, s, rule);
      });
  });
}

long long runs(long long n, int run) { return (n + run - 1) / run; }

constexpr long long kMostRuns = kMostThreads / NT;  // of a launch

// CCT_OK, and how many workgroups the list takes at `run` values each; a tensor's must fit one launch (2^37 values, 2^36 for
// the update: no card holds more).  Every pointer of a tensor with values must be there and aligned to one.
int check_list(const cct_tensor_t* list, int count, int run, long long* blocks) {
  if (count < 0 || (count > 0 && !list)) return CCT_EINVAL;
  *blocks = 0;
  for (int i = 0; i < count; ++i) {
    const cct_tensor_t& t = list[i];
    if (t.n < 0 || !type_known(t.type) || (t.n > 0 && !t.data) || ((uintptr_t)t.data & (type_bytes(t.type) - 1)))
      return CCT_EINVAL;
    if (t.n > kMostRuns * run) return CCT_EUNSUPPORTED;
    *blocks += runs(t.n, run);
  }
  return *blocks < 0x7fffffffLL ? CCT_OK : CCT_EUNSUPPORTED;
}
int check_same(const cct_tensor_t* a, const cct_tensor_t* b, int count, int run) {
  long long blocks;
  const int rc = check_list(b, count, run, &blocks);
  if (rc != CCT_OK) return rc;
  for (int i = 0; i < count; ++i)
    if (a[i].n != b[i].n) return CCT_EINVAL;
  return CCT_OK;
}

// Tensors [from, to) of the lists as one launch's arguments, as many as it takes; returns the first tensor left out.
// `forward`: from `from` up, else from `to` down.  *values, *bytes: of the gradients (and copies).
template <class Args, int P>
int fill(Args* a, const cct_tensor_t* const (&lists)[P], int from, int to, bool forward, double* values, double* bytes) {
  *values = *bytes = 0.0;
  int lo = forward ? from : to, hi = lo, held = 0;
  long long blocks_held = 0;
  auto take = [&](int i) {
    blocks_held += runs(lists[0][i].n, Args::kRun);
    return lists[0][i].n == 0 || (++held <= Args::kCount && blocks_held <= kMostRuns);
  };
  if (forward)
    while (hi < to && take(hi)) ++hi;
  else
    while (lo > from && take(lo - 1)) --lo;
  a->count = 0;
  a->first[0] = 0;
  for (int i = lo; i < hi; ++i) {
    if (lists[0][i].n == 0) continue;
    const int c = a->count++;
    for (int q = 0; q < P; ++q) a->p[q][c] = lists[q] ? lists[q][i].data : nullptr;
    const int blocks = (int)runs(lists[0][i].n, Args::kRun), last = (int)(lists[0][i].n - (blocks - 1LL) * Args::kRun) - 1;
    const int copy = P == 4 && lists[P - 1] ? lists[P - 1][i].type : 0;
    a->tail[c] = (unsigned short)(last << (Args::kRun > 4096 ? 3 : 4) | copy << 2 | lists[0][i].type);
    a->first[c + 1] = a->first[c] + blocks;
    *values += (double)lists[0][i].n;
    *bytes += (double)lists[0][i].n * (type_bytes(lists[0][i].type) + (P == 4 && lists[P - 1] ? type_bytes(copy) : 0));
  }
  return forward ? hi : lo;
}

}  // namespace
}  // namespace cct

using namespace cct;

extern "C" {

int cct_grad_norm_workspace_bytes(const cct_tensor_t* grads, int32_t count, size_t* bytes) {
  long long blocks;
  if (!bytes) return CCT_EINVAL;
  const int rc = check_list(grads, count, NormArgs::kRun, &blocks);
  if (rc != CCT_OK) return rc;
  *bytes = (size_t)std::max(1LL, blocks) * sizeof(double);
  return CCT_OK;
}

int cct_grad_norm(const cct_tensor_t* grads, int32_t count, float max_norm, float* clip, void* workspace,
                  size_t workspace_bytes, void* hip_stream) {
  long long blocks;
  const int rc = check_list(grads, count, NormArgs::kRun, &blocks);
  if (rc != CCT_OK) return rc;
  if (!clip || ((uintptr_t)clip & 3) || !(max_norm > 0.f)) return CCT_EINVAL;
  if (!workspace || ((uintptr_t)workspace & 255)) return CCT_EINVAL;
  if (workspace_bytes < (size_t)std::max(1LL, blocks) * sizeof(double)) return CCT_EWORKSPACE;
  hipStream_t st = (hipStream_t)hip_stream;
  double* part = (double*)workspace;
  const cct_tensor_t* const lists[1] = {grads};
  for (int at = 0; at < count;) {
    NormArgs a;
    double n, by;
    at = fill(&a, lists, at, count, true, &n, &by);
    if (a.count == 0) continue;
    ProfScope ps("grad_norm_kernel", 2.0 * n, by, st);
    hipLaunchKernelGGL(grad_norm_kernel, dim3(a.first[a.count]), dim3(NT), 0, st, a, part);
    CCT_CHECK_LAUNCH();
    part += a.first[a.count];
  }
  ProfScope ps("grad_norm_final_kernel", (double)blocks, 8.0 * (double)blocks, st);
  hipLaunchKernelGGL(grad_norm_final_kernel, dim3(1), dim3(kFinalThreads), 0, st, (const double*)workspace, (int)blocks,
                     max_norm, clip);
  CCT_CHECK_LAUNCH();
  return CCT_OK;
}

int cct_grad_scale(const cct_tensor_t* grads, int32_t count, const float* clip, const cct_tensor_t* out,
                   void* hip_stream) {
  long long blocks;
  int rc = check_list(grads, count, ScaleArgs::kRun, &blocks);
  if (rc == CCT_OK) rc = check_same(grads, out, count, ScaleArgs::kRun);
  if (rc != CCT_OK) return rc;
  if (!clip || ((uintptr_t)clip & 3)) return CCT_EINVAL;
  for (int i = 0; i < count; ++i)
    if (grads[i].type != out[i].type) return CCT_EINVAL;
  hipStream_t st = (hipStream_t)hip_stream;
  const cct_tensor_t* const lists[2] = {grads, out};
  for (int to = count; to > 0;) {
    ScaleArgs a;
    double n, by;
    to = fill(&a, lists, 0, to, false, &n, &by);
    if (a.count == 0) continue;
    ProfScope ps("grad_scale_kernel", n, 2.0 * by, st);
    hipLaunchKernelGGL(grad_scale_kernel, dim3(a.first[a.count]), dim3(NT), 0, st, a, clip);
    CCT_CHECK_LAUNCH();
  }
  return CCT_OK;
}

int cct_sgd_update(const cct_tensor_t* grads, int32_t count, const float* clip, const cct_tensor_t* weights,
                   const cct_tensor_t* moments, const cct_tensor_t* copies, float rate, float momentum, float decay,
                   void* hip_stream) {
  long long blocks;
  int rc = check_list(grads, count, UpdateArgs::kRun, &blocks);
  if (rc == CCT_OK) rc = check_same(grads, weights, count, UpdateArgs::kRun);
  if (rc == CCT_OK) rc = check_same(grads, moments, count, UpdateArgs::kRun);
  if (rc == CCT_OK && copies) rc = check_same(grads, copies, count, UpdateArgs::kRun);
  if (rc != CCT_OK) return rc;
  if ((uintptr_t)clip & 3) return CCT_EINVAL;
  if (!std::isfinite(rate) || !std::isfinite(momentum) || !std::isfinite(decay)) return CCT_EINVAL;
  for (int i = 0; i < count; ++i)
    if (weights[i].type != CCT_TYPE_F32 || moments[i].type != CCT_TYPE_F32) return CCT_EINVAL;
  hipStream_t st = (hipStream_t)hip_stream;
  const cct_tensor_t* const lists[4] = {grads, weights, moments, copies};
  const StepRule r = {rate, momentum, decay};
  for (int to = count; to > 0;) {
    UpdateArgs a;
    double n, by;
    to = fill(&a, lists, 0, to, false, &n, &by);
    if (a.count == 0) continue;
    ProfScope ps("sgd_update_kernel", 7.0 * n, by + 16.0 * n, st);
    hipLaunchKernelGGL(sgd_update_kernel, dim3(a.first[a.count]), dim3(NT), 0, st, a, clip, r);
    CCT_CHECK_LAUNCH();
  }
  return CCT_OK;
}

}  // extern "C"
