// The matrix product of 16-bit operands on the matrix cores, as tiles of one workgroup (v_mfma_f32_16x16x32, fp32 sums).
//
// An operand is taken from memory as it lies, with its values consecutive along the contraction (x and a weight in a forward
// product) or across it (a weight in dx, both in dw).  A stage is 64 steps of the contraction: 128 bytes of every row, or 64
// rows of the tile's width.  Loads of 16 bytes a lane write LDS directly, without registers, into a ring of stages of which
// one is multiplied while the others are on their way; the workgroup meets once per stage.
//
// LDS, where an operand's 16-byte pieces are permuted so that reads do not conflict (a load cannot place its lanes, but each
// lane chooses what it loads):
//   along the contraction: rows of 8 pieces, piece c of row r at c ^ (r & 7).  A matrix instruction's operand is one piece
//     per lane, 16 rows x 4 pieces.
//   across it: rows of the tile's width, in windows of 16 values; window v of row k at v ^ (k & 3 | (k >> 1) & 4)
//     (64 and 192 wide, whose windows come in fours: v ^ (k & 3)).  The operand is read with the transposing 8-byte LDS load: 16 lanes
//     fetch 4 rows x 16 values and each gets 4 rows of one column; two of them make a lane's 8 steps.
//
// What bounds the tiles of 256 (8192 x 8192 x 4096 forward: 405 to 425 us by card, 1290 to 1360 TFLOP/s): LDS reads and matrix
// instructions without the loads take 326 us, loads and LDS reads without the matrix instructions 263.  Half of what they
// take more together is the clock that the card holds (zeros as operands: 4096 x 4096 x 4096 in 89 us, 102 with normals).
// Latency it is not: 64 steps at a time with a third stage for one operand, lines asked for two stages ahead and 32 steps at
// a time in rings of 3 to 5 (428, 440, 450 us) gain nothing; nor LDS (four waves of 128 x 128, which read a third less, hide
// nothing behind each other: 561).
//
// The weights' side is the instruction's first operand: a lane then holds 4 neighbouring columns of one row of the result.
#pragma once
#include "activation.h"
#include "ff_bias_sum.h"
#include "gemm_common.h"

namespace cct {
namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) void* lds_ptr;
typedef __attribute__((address_space(3))) s16x4* lds_s16x4;

constexpr int SK = kFfStage;  // steps of the contraction per stage

template <int TYPE>
__device__ __forceinline__ f32x4 tile_mfma(s16x8 a, s16x8 b, f32x4 c) {
  if constexpr (TYPE == CCT_TYPE_BF16)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// One operand of a tile: ROWS rows of it, moved by NW waves.  ACROSS: consecutive across the contraction.
template <int ROWS, int NW, bool ACROSS>
struct TileOperand {
  static constexpr int BYTES = ROWS * SK * 2;
  static constexpr int UNITS = BYTES / 1024 / NW;  // loads of 1 KiB per wave and stage
  static_assert(UNITS * NW * 1024 == BYTES, "whole loads");
  static constexpr int PIECES = ACROSS ? ROWS / 8 : SK / 8;  // of a row in LDS
  unsigned voff[UNITS];                    // a lane's bytes from the tile's first row (and the stage's first step)
  int piece;                               // along: which of a row's pieces a lane loads

  static __device__ __forceinline__ int swizzle(int k) { return (k & 3) | (ROWS % 128 ? 0 : (k >> 1) & 4); }

  // rows (along) or columns (across, in whole eights) past `left` load the last again: their results are not stored.
  // PARTS == 2: the second half of the rows is another matrix's (each with `left`).
  template <int PARTS>
  __device__ __forceinline__ void init(int wave, int lane, int left, long long ld) {
    piece = (lane & 7) ^ (lane >> 3);
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
      const int unit = wave * UNITS + u;
      if constexpr (ACROSS) {
        const int at = unit * 64 + lane, k = at / PIECES, c = at % PIECES;
        const int src = (((c >> 1) ^ swizzle(k)) << 1) | (c & 1);
        voff[u] = (unsigned)(k * (int)ld + min(src * 8, ((left + 7) & ~7) - 8)) * 2u;
      } else {
        int r = unit * (64 / PIECES) + lane / PIECES;
        if (PARTS == 2 && r >= ROWS / 2) r -= ROWS / 2;
        voff[u] = (unsigned)(min(r, left - 1) * (int)ld + piece * 8) * 2u;
      }
    }
  }
  // Where the next stage lies: the address of the tile's first row (or, across, the stage's first step), and the bytes from
  // there to the operand's end, past which loads answer zero.  Rows have room for whole eights, zeros behind a contraction's
  // end.  PARTS == 2: `second` is where the other matrix's rows begin.
  struct Cursor {
    const char *first, *second;
    long long bytes;
  };
  static __device__ __forceinline__ Cursor begin(const char* first, const char* second, long long ld, int left, int k0, int K) {
    Cursor c;
    const long long skip = (long long)k0 * (ACROSS ? ld * 2 : 2);
    c.first = first + skip;
    c.second = second + skip;
    c.bytes = (ACROSS ? (long long)(K - 1) * ld + ((left + 7) & ~7) : (long long)(min(left, ROWS) - 1) * ld + ((K + 7) & ~7)) * 2 - skip;
    return c;
  }
  static __device__ __forceinline__ void next(Cursor& c, long long ld) {
    const long long step = SK * (ACROSS ? ld * 2 : 2);
    c.first += step;
    c.second += step;
    c.bytes -= step;
  }
  // kl: steps that are left; 0: nothing is loaded, LDS receives zeros
  template <int PARTS>
  __device__ __forceinline__ void load(unsigned char* lds, int wave, const Cursor& c, int kl) const {
    const int range = kl <= 0 ? 0 : c.bytes >> 31 ? 0x7fffffff : (int)c.bytes;
    const __amdgpu_buffer_rsrc_t r0 = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(c.first), 0, range, 0x00020000);
    const __amdgpu_buffer_rsrc_t r1 =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(PARTS == 2 ? c.second : c.first), 0, range, 0x00020000);
    // along: pieces past the contraction's end ask beyond the range (across: their rows lie beyond it)
    const bool live = ACROSS || piece * 8 < kl;
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
      const bool two = PARTS == 2 && (wave * UNITS + u) * (64 / PIECES) >= ROWS / 2;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(two ? r1 : r0, (lds_ptr)(lds + (wave * UNITS + u) * 1024), 16,
                                               (int)(live ? voff[u] : 0x80000000u), 0, 0, 0);
    }
  }
  // the 8 steps h * 32 + lane / 16 * 8 .. of row r0 + lane % 16 (r0 a multiple of 16)
  static __device__ __forceinline__ s16x8 read(const unsigned char* lds, int lane, int r0, int h) {
    if constexpr (ACROSS) {
      const int k = h * 32 + (lane >> 4) * 8 + ((lane >> 2) & 3);
      s16x4 v[2];
#pragma unroll
      for (int q = 0; q < 2; ++q)
        v[q] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (lds_s16x4)(lds + (k + 4 * q) * (ROWS * 2) + (((r0 >> 4) ^ swizzle(k + 4 * q)) << 5) + (lane & 3) * 8));
      return __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
      const int r = r0 + (lane & 15), c = h * 4 + (lane >> 4);
      return *(const s16x8*)(lds + r * (SK * 2) + ((c ^ (r & 7)) << 4));
    }
  }
};

// W neighbouring values of one row at any address, those past `left` not there
template <int TYPE, int W>
__device__ __forceinline__ void load_some(float (&v)[W], const void* p, long long at, int left) {
  typedef typename Number<TYPE>::T T;
  typedef T VW __attribute__((ext_vector_type(W)));
  typedef VW UW __attribute__((aligned(sizeof(T))));
  const T* from = (const T*)p + at;
  if (left >= W) {
    const VW all = *(const UW*)from;
#pragma unroll
    for (int e = 0; e < W; ++e) v[e] = (float)all[e];
  } else {
#pragma unroll
    for (int e = 0; e < W; ++e) v[e] = e < left ? (float)from[e] : 0.f;
  }
}
template <int TYPE, int W>
__device__ __forceinline__ void store_some(void* p, long long at, const float (&v)[W], int left) {
  typedef typename Number<TYPE>::T T;
  typedef T VW __attribute__((ext_vector_type(W)));
  typedef VW UW __attribute__((aligned(sizeof(T))));
  T* to = (T*)p + at;
  if (left >= W) {
    VW all;
#pragma unroll
    for (int e = 0; e < W; ++e) all[e] = (T)v[e];
    *(UW*)to = all;
  } else {
#pragma unroll
    for (int e = 0; e < W; ++e)
      if (e < left) to[e] = (T)v[e];
  }
}

// What becomes of W neighbouring sums of row m from column n on (kFfGated: of both products').  `early`: the residual's values
// if they are there already.
template <int TYPE, int EPI, int W>
__device__ __forceinline__ void finish(const FfProduct& p, int m, int n, float (&v)[W], float (&u)[W],
                                       const float (*early)[W] = nullptr) {
  const int left = p.N - n;
  if constexpr (EPI == kFfGated) {
    if (p.z) {
      store_some<TYPE>(p.z, m * p.ldz + n, v, left);
      store_some<TYPE>(p.z2, m * p.ldz2 + n, u, left);
    }
    activate<true>(p.activation, v, u);
  } else {
    float r[W] = {};
    if (early) {
#pragma unroll
      for (int e = 0; e < W; ++e) r[e] = (*early)[e];
    } else if (p.residual) {
      load_some<TYPE>(r, p.residual, m * p.ldr + n, left);
    }
    if (p.bias) {
      float b[W];
      load_some<TYPE>(b, p.bias, n, left);
#pragma unroll
      for (int e = 0; e < W; ++e) v[e] += b[e];
    }
    if (p.z) store_some<TYPE>(p.z, m * p.ldz + n, v, left);
    activate<false>(p.activation, v, u);
    if (p.residual)
#pragma unroll
      for (int e = 0; e < W; ++e) v[e] += r[e];
  }
  store_some<TYPE>(p.out, m * p.ldo + n, v, left);
}

// Which tile a workgroup computes: every XCD (they take workgroups in turn) gets a contiguous run of tiles, which walks over
// strips of 8 tiles of rows, so that what runs at a time shares both operands in its L2.
__device__ __forceinline__ void tile_of(int idx, int total, int tiles_m, int tiles_n, int* tm, int* tn) {
  const int per = total >> 3, rem = total & 7, xcd = idx & 7;
  idx = xcd * per + min(xcd, rem) + (idx >> 3);
  const int strip = idx / (8 * tiles_n), inner = idx - strip * 8 * tiles_n, rows = min(8, tiles_m - strip * 8);
  *tn = inner / rows;
  *tm = strip * 8 + inner - *tn * rows;
}

// The sums of one split of the contraction, for ff_join_kernel: M rows of `ld` floats, the second product's behind the first's.
struct FfPart {
  float* p;
  int ld;
  int splits, stages;  // of one split
};

// A wave's results on their way out: EROWS rows of PITCH floats in LDS.
template <int BM, int BN, int WM, int WN>
struct TileEpilogue {
  static constexpr int EROWS = BM / WM % 64 == 0 ? 64 : BM / WM % 48 == 0 ? 48 : 32, PITCH = BN / WN + 4;
  static_assert(BM / WM % EROWS == 0, "whole passes");
  static constexpr int BYTES = WM * WN * EROWS * PITCH * 4;
};

// BM x BN results (kFfGated: BM x BN / 2 of each product) with WM x WN waves; RING stages in LDS; SPLIT: the sums go to `part`,
// always or if it says so.
enum { kWhole, kSplit, kEither };
template <int TYPE, int BM, int BN, int WM, int WN, int RING, bool AX, bool BX, int EPI, int SPLIT>
__device__ __forceinline__ void compute_tile(const FfProduct& p, int tiles_m, int tiles_n, const FfPart& part, int index) {
  constexpr int NW = WM * WN, RB = BM / WM / 16, CB = BN / WN / 16;
  constexpr int PARTS = EPI == kFfGated ? 2 : 1;
  typedef TileOperand<BM, NW, AX> OpA;
  typedef TileOperand<BN, NW, BX> OpB;
  constexpr int STAGE = OpA::BYTES + OpB::BYTES;
  extern __shared__ __attribute__((aligned(1024))) unsigned char tile_smem[];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int wm = wave / WN, wn = wave % WN;
  // splits of a tile lie far apart: what runs at a time shares stages of the contraction
  const int tiles = tiles_m * tiles_n, split = SPLIT ? index / tiles : 0;
  int tm, tn;
  tile_of(index - split * tiles, tiles, tiles_m, tiles_n, &tm, &tn);
  const int m0 = tm * BM, n0 = tn * (BN / PARTS);
  const int left_m = p.M - m0, left_n = p.N - n0;

  const int per = max(pieces(p.K, SK), 1), all = per * (EPI == kFfGated ? 1 : p.segments);
  const int first = SPLIT ? split * part.stages : 0, stages = SPLIT ? min(part.stages, all - first) : all;
  OpA a;
  OpB b;
  const long long lda = p.A[0].ld, ldb = p.B[0].ld;
  a.template init<1>(wave, lane, left_m, lda);
  b.template init<PARTS>(wave, lane, left_n, ldb);
  const long long a_at = (AX ? m0 : m0 * lda) * 2, b_at = (BX ? n0 : n0 * ldb) * 2;
  // the stage that is loaded next; past the last one nothing is, but as many loads are in flight as ever
  unsigned k_next = first % per * SK;  // goes a ring past K, up to 2^31
  int to_load = stages;
  auto cursor_a = [&](int s, int k0) { return OpA::begin((const char*)p.A[s].p + a_at, nullptr, lda, left_m, k0, p.K); };
  auto cursor_b = [&](int s, int k0) {
    return OpB::begin((const char*)p.B[s].p + b_at, (const char*)p.B[1].p + b_at, ldb, left_n, k0, p.K);
  };
  auto ca = cursor_a(first / per, k_next);
  auto cb = cursor_b(first / per, k_next);
  auto load = [&](int slot) {
    unsigned char* st = tile_smem + slot * STAGE;
    const int kl = to_load > 0 ? (int)(p.K - k_next) : 0;
    a.template load<1>(st, wave, ca, kl);
    b.template load<PARTS>(st + OpA::BYTES, wave, cb, kl);
    --to_load;
    k_next += SK;
    OpA::next(ca, lda);
    OpB::next(cb, ldb);
    if (EPI != kFfGated && k_next >= (unsigned)p.K && to_load > 0) {  // the second contraction
      k_next = 0;
      ca = cursor_a(1, 0);
      cb = cursor_b(1, 0);
    }
  };
  // the weights' rows of block j: half of a wave's are of the second product
  auto row_b = [&](int j) {
    if constexpr (PARTS == 2) return (j >= CB / 2 ? BN / 2 : 0) + wn * (BN / 2 / WN) + (j % (CB / 2)) * 16;
    return wn * (BN / WN) + j * 16;
  };
  f32x4 acc[CB][RB];
#pragma unroll
  for (int j = 0; j < CB; ++j)
#pragma unroll
    for (int i = 0; i < RB; ++i) acc[j][i] = f32x4{0.f, 0.f, 0.f, 0.f};

  // Half a stage's operands are read from LDS behind the matrix instructions of the half before.  The workgroup meets between
  // the halves: then the stage's second half is in registers, so that the next loads take its place, and the next stage has
  // landed, whose first half is read.
  constexpr int L = OpA::UNITS + OpB::UNITS;  // loads of a wave and stage
  s16x8 fa[2][RB], fb[2][CB];
  auto read = [&](int set, int h, int slot) {
    const unsigned char *sa = tile_smem + slot * STAGE, *sb = sa + OpA::BYTES;
#pragma unroll
    for (int j = 0; j < CB; ++j) fb[set][j] = OpB::read(sb, lane, row_b(j), h);
#pragma unroll
    for (int i = 0; i < RB; ++i) fa[set][i] = OpA::read(sa, lane, wm * (BM / WM) + i * 16, h);
  };
  auto multiply = [&](int h, bool loads) {
#pragma unroll
    for (int i = 0; i < RB; ++i)
#pragma unroll
      for (int j = 0; j < CB; ++j) acc[j][i] = tile_mfma<TYPE>(fb[h][j], fa[h][i], acc[j][i]);
    // a wave issues in order, and what eight waves read and load takes LDS and the address unit as long as the matrix
    // instructions take: one by one between them, not in front of them (8192 x 8192 x 4096 forward 433 -> 411 us for the
    // reads, 405 for the loads too)
    constexpr int READS = (AX ? 2 : 1) * RB + (BX ? 2 : 1) * CB, EACH = RB * CB > READS ? RB * CB / READS : 1;
#pragma unroll
    for (int q = 0; q < READS; ++q) {
      __builtin_amdgcn_sched_group_barrier(0x008, EACH, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      if (loads && q < L) __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  // all but the last `behind` loads of this wave have landed, its LDS reads too, and everybody's (a meeting and nothing else:
  // __syncthreads() would wait for all loads)
  static_assert((RING - 1) * L < 64, "vmcnt has six bits");
#define CCT_MEET(behind)                                                               \
  __builtin_amdgcn_s_waitcnt(0x0070 | ((behind) & 15) | ((behind) >> 4) << 14);        \
  asm volatile("" ::: "memory");                                                       \
  __builtin_amdgcn_s_barrier();                                                        \
  asm volatile("" ::: "memory")
  for (int q = 0; q < RING; ++q) load(q);
  CCT_MEET((RING - 1) * L);
  int slot = 0;
  read(0, 0, 0);
  for (int t = 0; t < stages; ++t) {
    read(1, 1, slot);
    multiply(0, false);
    // the stage's second half is multiplied, the next one's first half read
    CCT_MEET((RING - 2) * L);
    load(slot);
    slot = slot + 1 == RING ? 0 : slot + 1;
    read(0, 0, slot);
    multiply(1, true);
  }
#undef CCT_MEET
  __builtin_amdgcn_s_waitcnt(0x0f70);  // the empty loads write LDS too

  constexpr int OUT = CB / PARTS;  // blocks of columns of the result
  if (SPLIT == kSplit || (SPLIT == kEither && part.splits > 1)) {
#pragma unroll
    for (int i = 0; i < RB; ++i) {
      const int m = m0 + wm * (BM / WM) + i * 16 + (lane & 15);
#pragma unroll
      for (int j = 0; j < OUT; ++j) {
        const int n = n0 + row_b(j) + (lane >> 4) * 4;
        if (m >= p.M || n >= p.N) continue;
        float* to = part.p + ((long long)split * PARTS * p.M + m) * part.ld + n;
        *(f32x4*)to = acc[j][i];
        if constexpr (PARTS == 2) *(f32x4*)(to + (long long)p.M * part.ld) = acc[j + OUT][i];
      }
    }
    return;
  }
  // Through LDS, EROWS rows of a wave at a time: a lane then has 8 neighbouring columns, stores are whole rows of the wave's
  // columns, and the code stands once and not for every block.  The residual's rows are asked for in front of that, all at
  // once: one by one they were a trip to memory each (4096 x 4096 x 4096 with a residual 119 us, 104 without).
  typedef TileEpilogue<BM, BN, WM, WN> Ep;
  typedef typename Number<TYPE>::V8 V8;
  constexpr int COLS = OUT * 16, PER = COLS / 8, STEPS = Ep::EROWS * PER / 64, DOWN = 64 / PER;  // lanes of a row; rows of a step
  static_assert(STEPS * 64 == Ep::EROWS * PER, "whole steps");
  __syncthreads();
  float* mine = (float*)tile_smem + wave * (Ep::EROWS * Ep::PITCH);
  const int row = lane / PER, c = lane % PER * 8, n = n0 + wn * COLS + c;
  const bool ahead = EPI == kFfLinear && p.residual && n + 8 <= p.N;
#pragma unroll
  for (int half = 0; half < BM / WM / Ep::EROWS; ++half) {
    constexpr int IB = Ep::EROWS / 16;
    const int m1 = m0 + wm * (BM / WM) + half * Ep::EROWS + row;
    V8 res[STEPS] = {};
    if (ahead)
#pragma unroll
      for (int s = 0; s < STEPS; ++s)
        if (m1 + s * DOWN < p.M)
          res[s] = *(const typename Number<TYPE>::U8*)((const typename Number<TYPE>::T*)p.residual + (m1 + s * DOWN) * p.ldr + n);
#pragma unroll
    for (int i = 0; i < IB; ++i)
#pragma unroll
      for (int j = 0; j < CB; ++j)
        *(f32x4*)(mine + (i * 16 + (lane & 15)) * Ep::PITCH + j * 16 + (lane >> 4) * 4) = acc[j][half * IB + i];
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
#pragma unroll 1
    for (int s = 0; s < STEPS; ++s) {
      const int m = m1 + s * DOWN;
      if (m >= p.M || n >= p.N) continue;
      float v[8], u[8], r[8];
      V8 rs = res[0];  // a step's, chosen by comparing: an index would put them into memory
#pragma unroll
      for (int q = 1; q < STEPS; ++q) rs = s == q ? res[q] : rs;
      const float* from = mine + (row + s * DOWN) * Ep::PITCH + c;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        v[e] = from[e];
        u[e] = PARTS == 2 ? from[COLS + e] : 0.f;
        r[e] = (float)rs[e];
      }
      if (ahead)
        finish<TYPE, EPI>(p, m, n, v, u, &r);
      else
        finish<TYPE, EPI>(p, m, n, v, u);
    }
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
  }
}

template <int TYPE, int BM, int BN, int WM, int WN, int RING, bool AX, bool BX, int EPI, int SPLIT>
__global__ __launch_bounds__(WM* WN * 64) __attribute__((amdgpu_waves_per_eu(2))) void ff_tile_kernel(FfProduct p, int tiles_m, int tiles_n, FfPart part) {
  compute_tile<TYPE, BM, BN, WM, WN, RING, AX, BX, EPI, SPLIT>(p, tiles_m, tiles_n, part, blockIdx.x);
}

// The products of a backward pass, which do not wait for one another, in one launch: the first workgroups finish a sum of
// columns, those from first[i] on are p[i]'s.  Alone each leaves CUs idle at its end, or all along; a launch more is 5 us where
// the host is the bound.  bf16, backward, one after the other and so: linear 1024 x 1024 x 1024 25.2 -> 18.1 us, 2048 x 2048 x
// 2048 68 -> 53; gated 512 x 512 x 512 27.6 -> 17.1, 2048 x 2048 x 2048 123 -> 93; fp16 linear 1531 x 1000 x 2049 61.7 -> 44.2.
// Contractions in splits, which one ff_join_kernel_together adds: gated 60 x 1301 x 64 27.7 -> 19.5, 1024 x 4096 x 1024 87 -> 70.
struct FfTogether {
  int count, first[kFfTogether], tiles_m[kFfTogether], tiles_n[kFfTogether];
  FfPart part[kFfTogether];
  FfProduct p[kFfTogether];
  FfBiasSum sum;
};
template <int TYPE, int BM, int BN, int WM, int WN, int RING>
__global__ __launch_bounds__(WM* WN * 64) __attribute__((amdgpu_waves_per_eu(2))) void ff_tile_kernel_together(FfTogether a) {
  if ((int)blockIdx.x < a.first[0]) {
    __shared__ float sums[WM * WN * 64 / kBiasColumns][kBiasColumns + 1];
    return sum_bias<TYPE, WM * WN * 64>(a.sum, blockIdx.x, sums);
  }
  int i = 0;
#pragma unroll
  for (int q = 1; q < kFfTogether; ++q) i += q < a.count && (int)blockIdx.x >= a.first[q];
  const int index = blockIdx.x - a.first[i];
  if (a.p[i].a_across)
    compute_tile<TYPE, BM, BN, WM, WN, RING, true, true, kFfLinear, kEither>(a.p[i], a.tiles_m[i], a.tiles_n[i], a.part[i], index);
  else
    compute_tile<TYPE, BM, BN, WM, WN, RING, false, true, kFfLinear, kEither>(a.p[i], a.tiles_m[i], a.tiles_n[i], a.part[i], index);
}

// The splits' sums added in order, and finished.  A thread takes 4 columns of a row.
template <int TYPE, int EPI>
__device__ __forceinline__ void join(const FfProduct& p, const FfPart& part, int block) {
  constexpr int PARTS = EPI == kFfGated ? 2 : 1;
  const int wide = part.ld / 4;
  const long long at = (long long)block * 256 + threadIdx.x;
  const int m = (int)(at / wide), n = (int)(at - (long long)m * wide) * 4;
  if (m >= p.M) return;
  f32x4 sum[PARTS];
#pragma unroll
  for (int q = 0; q < PARTS; ++q) sum[q] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < part.splits; ++s)
#pragma unroll
    for (int q = 0; q < PARTS; ++q)
      sum[q] += *(const f32x4*)(part.p + (((long long)s * PARTS + q) * p.M + m) * part.ld + n);
  float v[4], u[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    v[e] = sum[0][e];
    u[e] = sum[PARTS - 1][e];
  }
  finish<TYPE, EPI>(p, m, n, v, u);
}
template <int TYPE, int EPI>
__global__ __launch_bounds__(256) void ff_join_kernel(FfProduct p, FfPart part, int first) {
  join<TYPE, EPI>(p, part, first + blockIdx.x);
}
template <int TYPE, int EPI>
void launch_join(const FfProduct& p, const FfPart& part, hipStream_t st) {
  const long long groups = ((long long)p.M * part.ld / 4 + 255) / 256, most = kMostThreads / 256;
  for (long long first = 0; first < groups; first += most)
    hipLaunchKernelGGL(HIP_KERNEL_NAME(ff_join_kernel<TYPE, EPI>), dim3((unsigned)(groups - first < most ? groups - first : most)),
                       dim3(256), 0, st, p, part, (int)first);
}
// Those of several products: workgroups from first[i] on are p[i]'s.
template <int TYPE>
__global__ __launch_bounds__(256) void ff_join_kernel_together(FfTogether a) {
  int i = 0;
#pragma unroll
  for (int q = 1; q < kFfTogether; ++q) i += q < a.count && (int)blockIdx.x >= a.first[q];
  join<TYPE, kFfLinear>(a.p[i], a.part[i], blockIdx.x - a.first[i]);
}

}  // namespace
}  // namespace cct
