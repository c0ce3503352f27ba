// Products of microscaled 4-bit matrices of few rows (serving), which are bound by reading the weight, and of any that the tiles
// do not take.
//
// A workgroup takes 16 rows of the weight and 16, 32 or 64 of x, its waves in turn four steps of 128 values of the contraction:
// codes go from memory into the registers that v_mfma_scale_f32_16x16x128_f8f6f4 takes, a lane a block of 32 of one row, with
// its scale; 256 bytes of each row and 16 scales a wave and turn.  The waves' sums meet in LDS in a
// fixed order; few columns of long rows are cut into splits, which ff_join_kernel adds.
//
// One row of 4096 values to 4096 (8.9 MB): 6.9 us, of which launching and one trip to memory are most; with x quantised by a launch
// of its own 9.9.  The next turn's codes on their way while one is multiplied leave fewer waves on a CU: 1 x 16384 x 4096 12.9
// us instead of 9.5.
//
// Blocks behind the row's end: their codes are zeros and their scales one, whatever lies there.
#include <algorithm>

#include "ff_tile.h"
#include "mx.h"
#include "mx_steps.h"

namespace cct {
namespace {

constexpr int NW = 8, kBatch = 4;

// QUANTIZE: x are values (x.codes, x.ldc of them), which every workgroup rounds for itself.
template <int TYPE, int RM, bool SPLIT, bool QUANTIZE>
__global__ __launch_bounds__(NW * 64) void mx_rows_kernel(MxProduct a, FfPart part) {
  const FfProduct& p = a.p;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lo = lane & 15, q = lane >> 4;
  const int steps = pieces(a.blocks, 4), tiles = pieces(p.N, 16), tall = pieces(p.M, RM * 16);
  const int split = SPLIT ? blockIdx.z : 0;
  const bool eights = p.K % 8 == 0;
  const int first = SPLIT ? split * part.stages : 0, end = SPLIT ? min(steps, first + part.stages) : steps;
  __shared__ f32x4 sums[NW][RM][64];
  for (int mb = blockIdx.y; mb < tall; mb += gridDim.y)
    for (int tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
      const int n0 = tile * 16, m0 = mb * RM * 16;
      const long long wr = min((long long)n0 + lo, p.N - 1LL);
      const unsigned char *wc = a.w.codes + wr * a.w.ldc, *ws = a.w.scales + wr * a.w.lds;
      const unsigned char *xc[RM], *xs[RM];
#pragma unroll
      for (int i = 0; i < RM; ++i) {
        const long long r = min((long long)m0 + i * 16 + lo, p.M - 1LL);
        xc[i] = a.x.codes + (QUANTIZE ? 0 : r * a.x.ldc);
        xs[i] = a.x.scales + r * a.x.lds;
      }
      f32x4 acc[RM];
#pragma unroll
      for (int i = 0; i < RM; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
      struct Turn {
        i32x4 w[kBatch], ws, x[RM][kBatch], xs[RM];
        typename Number<TYPE>::V8 v[QUANTIZE ? kBatch : 1][4];
      };
      auto load = [&](Turn& t, int s0) {
        t.ws = mx_scales4(ws, s0, a.blocks);
        if constexpr (!QUANTIZE)
#pragma unroll
          for (int i = 0; i < RM; ++i) t.xs[i] = mx_scales4(xs[i], s0, a.blocks);
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
          const int block = min((s0 + j) * 4 + q, a.blocks - 1);
          t.w[j] = *(const i32x4*)(wc + 16LL * block);
          if constexpr (QUANTIZE) {
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              const int col = block * kMxBlock + c * 8;
              const long long row = min((long long)m0 + lo, p.M - 1LL) * a.x.ldc;
              if (eights)  // less between the loads and their use
                t.v[j][c] = col < p.K ? *(const typename Number<TYPE>::U8*)((const typename Number<TYPE>::T*)a.x.codes + row + col)
                                      : typename Number<TYPE>::V8{};
              else
                t.v[j][c] = load_row_raw<TYPE>(a.x.codes, row, col, p.K - col);
            }
          } else {
#pragma unroll
            for (int i = 0; i < RM; ++i) t.x[i][j] = *(const i32x4*)(xc[i] + 16LL * block);
          }
        }
      };
      auto multiply = [&](Turn& t, int s0) {
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
          i32x4 own = {};
          int own_scale = 127;
          if constexpr (QUANTIZE) {
            if (!eights)
#pragma unroll
              for (int c = 0; c < 4; ++c) {
                const int col = min((s0 + j) * 4 + q, a.blocks - 1) * kMxBlock + c * 8;
                t.v[j][c] = settle_row<TYPE>(t.v[j][c], col, p.K - col);
              }
            own = mx_quantize_block<TYPE>(t.v[j], &own_scale);
          }
          const bool live = s0 + j < end && (s0 + j) * 4 + q < a.blocks;
          const i32x4 w = live ? t.w[j] : i32x4{0, 0, 0, 0};
          const int sw = live ? (int)((unsigned)t.ws[j] >> (8 * q)) : 127;
#pragma unroll
          for (int i = 0; i < RM; ++i) {
            const i32x4 x = QUANTIZE ? own : t.x[i][j];
            const int sx = QUANTIZE ? own_scale : (int)((unsigned)t.xs[i][j] >> (8 * q));
            acc[i] = mx_mfma<0, 0>(w, live ? x : i32x4{0, 0, 0, 0}, acc[i], sw, live ? sx : 127);
          }
        }
      };
      for (int s = first + wave * kBatch; s < end; s += NW * kBatch) {
        Turn t;
        load(t, s);
        __builtin_amdgcn_sched_barrier(0);
        multiply(t, s);
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < RM; ++i) sums[wave][i][lane] = acc[i];
      __syncthreads();
      for (int i = wave; i < RM; i += NW) {
        f32x4 t = sums[0][i][lane];
#pragma unroll
        for (int w = 1; w < NW; ++w) t += sums[w][i][lane];
        const int m = m0 + i * 16 + lo, n = n0 + q * 4;
        if (m >= p.M || n >= p.N) continue;
        if constexpr (SPLIT) {
          *(f32x4*)(part.p + ((long long)split * p.M + m) * part.ld + n) = t;
          continue;
        }
        float v[4] = {t[0], t[1], t[2], t[3]}, u[4] = {};
        finish<TYPE, kFfLinear, true>(p, m, n, v, u);
      }
    }
}

template <int TYPE>
void launch(const MxProduct& a, const MxPlan& plan, float* ws, hipStream_t st) {
  const FfPart part = {ws, (a.p.N + 3) / 4 * 4, plan.splits, plan.steps};
  auto run = [&](auto rm, auto quantize) {
    constexpr int RM = decltype(rm)::value;
    constexpr bool QUANTIZE = decltype(quantize)::value;
    const dim3 grid(std::min(pieces(a.p.N, 16), 1 << 16), std::min(pieces(a.p.M, RM * 16), 64), plan.splits);
    if (plan.splits > 1)
      hipLaunchKernelGGL(HIP_KERNEL_NAME(mx_rows_kernel<TYPE, RM, true, QUANTIZE>), grid, dim3(NW * 64), 0, st, a, part);
    else
      hipLaunchKernelGGL(HIP_KERNEL_NAME(mx_rows_kernel<TYPE, RM, false, QUANTIZE>), grid, dim3(NW * 64), 0, st, a, part);
  };
  if (a.p.M <= 16 && a.quantize)
    run(std::integral_constant<int, 1>(), std::true_type());
  else if (a.p.M <= 16)
    run(std::integral_constant<int, 1>(), std::false_type());
  else if (a.p.M <= 32)
    run(std::integral_constant<int, 2>(), std::false_type());
  else
    run(std::integral_constant<int, 4>(), std::false_type());
  if (plan.splits > 1) launch_join<TYPE, kFfLinear>(a.p, part, st);
}

}  // namespace

int launch_mx_rows(const MxProduct& a, const MxPlan& plan, float* part, hipStream_t st) {
  const double mn = (double)a.p.M * a.p.N, k = (double)a.p.K;
  ProfScope ps("mx_rows_kernel", 2.0 * mn * k,
               (a.p.M + (double)a.p.N) * k * 17 / 32 + type_bytes(a.p.type) * mn * (1 + (a.p.residual != nullptr) + (a.p.z != nullptr)), st);
  if (a.p.type == CCT_TYPE_F32)
    launch<CCT_TYPE_F32>(a, plan, part, st);
  else if (a.p.type == CCT_TYPE_BF16)
    launch<CCT_TYPE_BF16>(a, plan, part, st);
  else
    launch<CCT_TYPE_F16>(a, plan, part, st);
  CCT_CHECK_LAUNCH();
  return CCT_OK;
}

}  // namespace cct
