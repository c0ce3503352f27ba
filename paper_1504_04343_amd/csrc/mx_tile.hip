// The product of microscaled 4-bit matrices on the matrix cores, as tiles of one workgroup (v_mfma_scale_f32_16x16x128_f8f6f4).
//
// The structure is that of the 16-bit tiles (ff_tile.h): a stage is 128 bytes of every row, here 256 values, which loads of 16
// bytes a lane write into a ring in LDS; a piece of 16 bytes is a block of 32 values, so that what a lane reads for an
// instruction is one block of one row, as the instruction takes it.  The scales of two stages are 16 bytes a row, which come in one
// load a lane, every second stage; a lane reads a stage's words (four blocks a step) of its rows and keeps its own blocks' bytes,
// two rows' and two steps' to a register.
//
// 8192 x 8192 x 8192: 276 to 300 us by card, 3.7 to 4.0 PFLOP/s, in calls that follow one another on the same codes; with bias and GELU
// 318 to 330, and about 355 in a kernel trace, where each launch stands alone.  The instructions alone, in a loop on registers, reach 9.3 PFLOP/s
// on zeros and 6.2 to 7.0 on random codes (the card's clock falls); what keeps a tile of 256 x 256 from that is LDS, which a stage
// asks for 24 KiB x 8 waves of operands and gives 64 KiB of new ones, as long as its matrix instructions take.  Without loads 245 of
// then 311 us, without LDS reads 274, without scales 289, without waves meeting 288.  Slower: scales in loads of 4 bytes (298), a ring
// of four stages of 128 values (308), four waves of 128 x 128, which read a third less but are alone on their SIMDs (356).
#include <algorithm>

#include "ff_tile.h"
#include "mx.h"
#include "mx_steps.h"

namespace cct {
namespace {

constexpr int kStageBlocks = 8;  // of a row and stage: two steps of 128 values

// The instruction with the scales in bytes `ba` and `bb` (known when loops are unrolled; it takes them as part of its code).
template <int BA>
__device__ __forceinline__ f32x4 mx_mfma_b(i32x4 a, i32x4 b, f32x4 c, int sa, int bb, int sb) {
  switch (bb) {
    case 0: return mx_mfma<BA, 0>(a, b, c, sa, sb);
    case 1: return mx_mfma<BA, 1>(a, b, c, sa, sb);
    case 2: return mx_mfma<BA, 2>(a, b, c, sa, sb);
    default: return mx_mfma<BA, 3>(a, b, c, sa, sb);
  }
}
__device__ __forceinline__ f32x4 mx_mfma_at(i32x4 a, i32x4 b, f32x4 c, int ba, int sa, int bb, int sb) {
  switch (ba) {
    case 0: return mx_mfma_b<0>(a, b, c, sa, bb, sb);
    case 1: return mx_mfma_b<1>(a, b, c, sa, bb, sb);
    case 2: return mx_mfma_b<2>(a, b, c, sa, bb, sb);
    default: return mx_mfma_b<3>(a, b, c, sa, bb, sb);
  }
}

// The scales of a wave's RBLK blocks of 16 rows, of one stage: rows 16 bytes apart in LDS.  Byte (i & 1) * 2 + h of s[i / 2]: block i,
// step h.
template <int RBLK>
__device__ __forceinline__ void read_scales(const unsigned char* rows, int lane, int (&s)[RBLK / 2]) {
  typedef int i32x2 __attribute__((ext_vector_type(2)));
  const unsigned q = lane >> 4, pick = (q + 4) << 8 | q;
  i32x2 w[RBLK];
#pragma unroll
  for (int i = 0; i < RBLK; ++i) w[i] = *(const i32x2*)(rows + (i * 16 + (lane & 15)) * 16);
#pragma unroll
  for (int i = 0; i < RBLK; i += 2) {
    const unsigned a = __builtin_amdgcn_perm(w[i][1], w[i][0], pick), b = __builtin_amdgcn_perm(w[i + 1][1], w[i + 1][0], pick);
    s[i / 2] = (int)__builtin_amdgcn_perm(b, a, 0x05040100u);
  }
}
// One in place of what lies there for blocks behind the end, of which `left` are there and this lane's is the q-th.
template <int N>
__device__ __forceinline__ void end_scales(int q, int left, int (&s)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    unsigned v = (unsigned)s[i];
    v = q < left ? v : (v & 0xff00ff00u) | 0x007f007fu;
    s[i] = (int)(q + 4 < left ? v : (v & 0x00ff00ffu) | 0x7f007f00u);
  }
}

template <int TYPE, int BM, int BN, int WM, int WN, int RING, bool SPLIT>
__global__ __launch_bounds__(WM* WN * 64) __attribute__((amdgpu_waves_per_eu(2))) void mx_tile_kernel(MxProduct a, int tiles_m, int tiles_n,
                                                                                                      FfPart part) {
  constexpr int NW = WM * WN, RB = BM / WM / 16, CB = BN / WN / 16;
  typedef TileOperand<BM, NW, false> OpA;
  typedef TileOperand<BN, NW, false> OpB;
  constexpr int STAGE = OpA::BYTES + OpB::BYTES, SCALES = (BM + BN) * 16, UNITS = (BM + BN) / 64;  // loads of scales: one of a wave
  static_assert(UNITS <= NW && BM % 64 == 0, "one load");
  static_assert((RING & (RING - 1)) == 0, "places of a ring");  // of as many pairs of stages the scales, those in use and those ahead

  extern __shared__ __attribute__((aligned(1024))) unsigned char tile_smem[];

  const FfProduct& p = a.p;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int wm = wave / WN, wn = wave % WN;
  const int tiles = tiles_m * tiles_n, split = SPLIT ? (int)blockIdx.x / tiles : 0;
  int tm, tn;
  tile_of(blockIdx.x - split * tiles, tiles, tiles_m, tiles_n, &tm, &tn);
  const int m0 = tm * BM, n0 = tn * BN, left_m = p.M - m0, left_n = p.N - n0;
  const int all = pieces(a.blocks, kStageBlocks), first = SPLIT ? split * part.stages : 0;
  const int stages = SPLIT ? min(part.stages, all - first) : all;

  // codes as the 16-bit tiles' values: 8 to a block
  OpA opa;
  OpB opb;
  const long long lda = a.x.ldc / 2, ldb = a.w.ldc / 2;
  opa.template init<1>(wave, lane, left_m, lda);
  opb.template init<1>(wave, lane, left_n, ldb);
  auto ca = OpA::begin((const char*)a.x.codes + m0 * a.x.ldc, nullptr, lda, left_m, first * 64, a.blocks * 8);
  auto cb = OpB::begin((const char*)a.w.codes + n0 * a.w.ldc, nullptr, ldb, left_n, first * 64, a.blocks * 8);
  // this wave's load of scales: 64 rows of one of the two (waves that have none load the last again)
  const int unit = min(wave, UNITS - 1);
  const bool of_a = unit < BM / 64;
  const MxMatrix& sm = of_a ? a.x : a.w;
  const int sc_rows = min(of_a ? left_m : left_n, of_a ? BM : BN), sc_row = (of_a ? unit : unit - BM / 64) * 64 + lane;
  const unsigned sc_at = (unsigned)(min(sc_row, sc_rows - 1) * (int)sm.lds);
  const unsigned char* sc_from = sm.scales + (of_a ? m0 : n0) * sm.lds + first * kStageBlocks;
  long long sc_bytes = (sc_rows - 1) * sm.lds + ((a.blocks + 3) & ~3) - first * kStageBlocks;  // to the last row's end
  int loaded = 0;
  auto load = [&]() {
    unsigned char* st = tile_smem + (loaded & (RING - 1)) * STAGE;
    const int left = loaded < stages ? (a.blocks - (first + loaded) * kStageBlocks) * 8 : 0;
    opa.template load<1>(st, wave, ca, left);
    opb.template load<1>(st + OpA::BYTES, wave, cb, left);
    if ((loaded & 1) == 0) {
      const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(sc_from), 0,
                                                                         left > 0 ? (int)min(sc_bytes, 0x7fffffffLL) : 0, 0x00020000);
      unsigned char* to = tile_smem + RING * STAGE + (loaded >> 1 & (RING - 1)) * SCALES + unit * 1024;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_ptr)to, 16, (int)sc_at, 0, 0, 0);
      sc_from += 2 * kStageBlocks;
      sc_bytes -= 2 * kStageBlocks;
    }
    ++loaded;
    OpA::next(ca, lda);
    OpB::next(cb, ldb);
  };

  f32x4 acc[CB][RB];
#pragma unroll
  for (int j = 0; j < CB; ++j)
#pragma unroll
    for (int i = 0; i < RB; ++i) acc[j][i] = f32x4{0.f, 0.f, 0.f, 0.f};
  constexpr int L = OpA::UNITS + OpB::UNITS;
  s16x8 fa[2][RB], fb[2][CB];
  int sa[RB / 2], sb[CB / 2];
  auto read = [&](int set, int h, int t) {
    const unsigned char* st = tile_smem + (t & (RING - 1)) * STAGE;
#pragma unroll
    for (int j = 0; j < CB; ++j) fb[set][j] = OpB::read(st + OpA::BYTES, lane, wn * (BN / WN) + j * 16, h);
#pragma unroll
    for (int i = 0; i < RB; ++i) fa[set][i] = OpA::read(st, lane, wm * (BM / WM) + i * 16, h);
  };
  auto scales = [&](int t, int (&to_a)[RB / 2], int (&to_b)[CB / 2]) {
    const unsigned char* sc = tile_smem + RING * STAGE + (t >> 1 & (RING - 1)) * SCALES + (t & 1) * 8;
    read_scales<RB>(sc + wm * (BM / WM) * 16, lane, to_a);
    read_scales<CB>(sc + (BM + wn * (BN / WN)) * 16, lane, to_b);
  };
  auto multiply = [&](int h, bool loads) {
#pragma unroll
    for (int i = 0; i < RB; ++i)
#pragma unroll
      for (int j = 0; j < CB; ++j)
        acc[j][i] = mx_mfma_at(__builtin_bit_cast(i32x4, fb[h][j]), __builtin_bit_cast(i32x4, fa[h][i]), acc[j][i], (j & 1) * 2 + h, sb[j >> 1],
                               (i & 1) * 2 + h, sa[i >> 1]);
    // one by one between the matrix instructions, as in ff_tile.h
    const int reads = (RB + CB) * (loads ? 2 : 1), each = RB * CB > reads ? RB * CB / reads : 1;
#pragma unroll
    for (int q = 0; q < reads; ++q) {
      if (each == 2) __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
      if (each != 2) __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      if (loads && q < L) __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  // the stage that is read has landed, this wave's LDS reads too, and everybody's
#define CCT_MEET(behind)                                                        \
  __builtin_amdgcn_s_waitcnt(0x0070 | ((behind) & 15) | ((behind) >> 4) << 14); \
  asm volatile("" ::: "memory");                                                \
  __builtin_amdgcn_s_barrier();                                                 \
  asm volatile("" ::: "memory")
  static_assert((RING - 1) * L < 64, "vmcnt has six bits");
  for (int q = 0; q < RING; ++q) load();
  CCT_MEET((RING - 1) * L);  // (loads of scales are some more: this waits for a little more than it must)
  read(0, 0, 0);
  scales(0, sa, sb);
  for (int t = 0; t < stages; ++t) {
    const int left = a.blocks - (first + t) * kStageBlocks;
    if (left < kStageBlocks) {
      end_scales(lane >> 4, left, sa);
      end_scales(lane >> 4, left, sb);
    }
    read(1, 1, t);
    multiply(0, false);
    CCT_MEET((RING - 2) * L);
    load();
    int na[RB / 2], nb[CB / 2];
    scales(t + 1, na, nb);
    read(0, 0, t + 1);
    multiply(1, true);
#pragma unroll
    for (int i = 0; i < RB / 2; ++i) sa[i] = na[i];
#pragma unroll
    for (int j = 0; j < CB / 2; ++j) sb[j] = nb[j];
  }
#undef CCT_MEET
  __builtin_amdgcn_s_waitcnt(0x0f70);  // the empty loads write LDS too
  finish_tile<TYPE, BM, BN, WM, WN, kFfLinear, true>(p, part, SPLIT, split, m0, n0, acc);
}

template <int TYPE, int BM, int BN, int WM, int WN, int RING, bool SPLIT>
int launch_one(const MxProduct& a, const FfPart& part, hipStream_t st) {
  constexpr int ring = RING * (BM + BN) * (128 + 16), out = TileEpilogue<BM, BN, WM, WN>::BYTES, lds = ring > out ? ring : out;
  constexpr auto kernel = mx_tile_kernel<TYPE, BM, BN, WM, WN, RING, SPLIT>;
  const int rc = ensure_dynamic_lds<kernel>(lds);
  if (rc != CCT_OK) return rc;
  const int tiles_m = pieces(a.p.M, BM), tiles_n = pieces(a.p.N, BN);
  hipLaunchKernelGGL(kernel, dim3(tiles_m * tiles_n * part.splits), dim3(WM * WN * 64), lds, st, a, tiles_m, tiles_n, part);
  CCT_CHECK_LAUNCH();
  return CCT_OK;
}

template <int TYPE, bool SPLIT>
int launch_planned(const MxProduct& a, const MxPlan& plan, const FfPart& part, hipStream_t st) {
  switch (plan.tile) {
    case kTile128: return launch_one<TYPE, 128, 128, 2, 2, 2, SPLIT>(a, part, st);
    case kTile64x128: return launch_one<TYPE, 64, 128, 2, 2, 2, SPLIT>(a, part, st);
    default: return plan.deep ? launch_one<TYPE, 64, 64, 2, 2, 4, SPLIT>(a, part, st) : launch_one<TYPE, 64, 64, 2, 2, 2, SPLIT>(a, part, st);
  }
}
template <int TYPE>
int launch(const MxProduct& a, const MxPlan& plan, float* ws, hipStream_t st) {
  const FfPart part = {ws, (a.p.N + 3) / 4 * 4, plan.splits, plan.steps};
  if (plan.tile == kTile256) return launch_one<TYPE, 256, 256, 2, 4, 2, false>(a, part, st);
  if (plan.splits == 1) return launch_planned<TYPE, false>(a, plan, part, st);
  const int rc = launch_planned<TYPE, true>(a, plan, part, st);
  if (rc != CCT_OK) return rc;
  launch_join<TYPE, kFfLinear>(a.p, part, st);
  CCT_CHECK_LAUNCH();
  return CCT_OK;
}

}  // namespace

int launch_mx_tile(const MxProduct& a, const MxPlan& plan, float* part, hipStream_t st) {
  const double mn = (double)a.p.M * a.p.N, k = (double)a.p.K;
  ProfScope ps(2.0 * mn * k,
               (a.p.M + (double)a.p.N) * k * 17 / 32 + type_bytes(a.p.type) * mn * (1 + (a.p.residual != nullptr) + (a.p.z != nullptr)), st,
               "mx_tile_kernel<%s, %d splits, %d stages>",
               plan.tile == kTile256 ? "256x256" : plan.tile == kTile128 ? "128x128" : plan.tile == kTile64x128 ? "64x128" : "64x64",
               plan.splits, plan.deep ? 4 : 2);
  if (a.p.type == CCT_TYPE_F32) return launch<CCT_TYPE_F32>(a, plan, part, st);
  return a.p.type == CCT_TYPE_BF16 ? launch<CCT_TYPE_BF16>(a, plan, part, st) : launch<CCT_TYPE_F16>(a, plan, part, st);
}

}  // namespace cct
