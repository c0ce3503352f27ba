// The matrix product of 16-bit operands on the matrix cores, as tiles of one workgroup (v_mfma_f32_16x16x32, fp32 sums).
//
// An operand is taken from memory as it lies, with its values consecutive along the contraction (x and a weight in a forward
// product) or across it (a weight in dx, both in dw).  A stage is 64 steps of the contraction: 128 bytes of every row, or 64
// rows of the tile's width.  Loads of 16 bytes a lane write LDS directly, without registers, one stage ahead of the one that
// is multiplied; two stages alternate and the workgroup meets once per stage.
//
// LDS, where an operand's 16-byte pieces are permuted so that reads do not conflict (a load cannot place its lanes, but each
// lane chooses what it loads):
//   along the contraction: rows of 8 pieces, piece c of row r at c ^ (r & 7).  A matrix instruction's operand is one piece
//     per lane, 16 rows x 4 pieces.
//   across it: 64 rows of the tile's width, in windows of 16 values; window v of row k at v ^ (k & 3 | (k >> 1) & 4).  The
//     operand is read with the transposing 8-byte LDS load: 16 lanes fetch 4 rows x 16 values and each gets 4 rows of one
//     column; two of them make a lane's 8 steps.
//
// The weights' side is the instruction's first operand: a lane then holds 4 neighbouring columns of one row of the result,
// stored as 8 bytes.
#pragma once
#include "activation.h"
#include "feed_forward.h"
#include "gemm_common.h"

namespace cct {
namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) void* lds_ptr;
typedef __attribute__((address_space(3))) s16x4* lds_s16x4;

constexpr int kStageK = 64;

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
  static constexpr int BYTES = ROWS * kStageK * 2;
  static constexpr int UNITS = BYTES / 1024 / NW;  // loads of 1 KiB per wave and stage
  static_assert(UNITS * NW * 1024 == BYTES, "whole loads");
  static constexpr int PIECES = ROWS / 8;  // per row, across
  unsigned voff[UNITS];                    // a lane's bytes from the tile's first row (and the stage's first step)
  int piece;                               // along: which of a row's 8 pieces a lane loads

  static __device__ __forceinline__ int swizzle(int k) { return (k & 3) | ((k >> 1) & 4); }

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
        int r = unit * 8 + (lane >> 3);
        if (PARTS == 2 && r >= ROWS / 2) r -= ROWS / 2;
        voff[u] = (unsigned)(min(r, left - 1) * (int)ld + piece * 8) * 2u;
      }
    }
  }
  // steps [k0, k0 + 64) of a contraction of K; `first` and, for the second half of the rows, `second`: the tile's first row
  template <int PARTS>
  __device__ __forceinline__ void load(unsigned char* lds, int wave, const char* first, const char* second, long long ld, int left,
                                       int k0, int K) const {
    const int kl = min(K - k0, kStageK);
    const long long skip = ACROSS ? (long long)k0 * ld * 2 : (long long)k0 * 2;
    // rows have room for whole eights, zeros behind a contraction's end
    const long long bytes = ACROSS ? ((long long)(kl - 1) * ld + ((left + 7) & ~7)) * 2
                                   : ((long long)(min(left, ROWS) - 1) * ld + ((K - k0 + 7) & ~7)) * 2;
    const int range = (int)min(bytes, 0x7fffffffLL);
    const __amdgpu_buffer_rsrc_t r0 = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(first + skip), 0, range, 0x00020000);
    const __amdgpu_buffer_rsrc_t r1 =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>((PARTS == 2 ? second : first) + skip), 0, range, 0x00020000);
    // along: pieces past the contraction's end ask beyond the range, which answers zero (across: their rows lie beyond it)
    const bool live = ACROSS || piece * 8 < kl;
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
      const bool two = PARTS == 2 && (wave * UNITS + u) * 8 >= ROWS / 2;
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
      return *(const s16x8*)(lds + r * 128 + ((c ^ (r & 7)) << 4));
    }
  }
};

// 4 neighbouring values of one row at any address, those past `left` not there
template <int TYPE>
__device__ __forceinline__ void load4(float (&v)[4], const void* p, long long at, int left) {
  typedef typename Number<TYPE>::T T;
  typedef T V4 __attribute__((ext_vector_type(4)));
  typedef V4 U4 __attribute__((aligned(sizeof(T))));
  const T* from = (const T*)p + at;
  if (left >= 4) {
    const V4 all = *(const U4*)from;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = (float)all[e];
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = e < left ? (float)from[e] : 0.f;
  }
}
template <int TYPE>
__device__ __forceinline__ void store4(void* p, long long at, const float (&v)[4], int left) {
  typedef typename Number<TYPE>::T T;
  typedef T V4 __attribute__((ext_vector_type(4)));
  typedef V4 U4 __attribute__((aligned(sizeof(T))));
  T* to = (T*)p + at;
  if (left >= 4) {
    V4 all;
#pragma unroll
    for (int e = 0; e < 4; ++e) all[e] = (T)v[e];
    *(U4*)to = all;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < left) to[e] = (T)v[e];
  }
}

// What becomes of 4 neighbouring sums of row m from column n on (kFfGated: of both products'); `bias`: theirs.
template <int TYPE, int EPI>
__device__ __forceinline__ void finish4(const FfProduct& p, int m, int n, float (&v)[4], float (&u)[4], const float (&bias)[4]) {
  const int left = p.N - n;
  if constexpr (EPI == kFfGated) {
    if (p.z) {
      store4<TYPE>(p.z, m * p.ldz + n, v, left);
      store4<TYPE>(p.z2, m * p.ldz2 + n, u, left);
    }
    activate(p.activation, v);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] *= u[e];
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] += bias[e];
    if (p.z) store4<TYPE>(p.z, m * p.ldz + n, v, left);
    activate(p.activation, v);
    if (p.residual) {
      float r[4];
      load4<TYPE>(r, p.residual, m * p.ldr + n, left);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += r[e];
    }
  }
  store4<TYPE>(p.out, m * p.ldo + n, v, left);
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

// BM x BN results (kFfGated: BM x BN / 2 of each product) with WM x WN waves.
template <int TYPE, int BM, int BN, int WM, int WN, bool AX, bool BX, int EPI>
__global__ __launch_bounds__(WM* WN * 64) void ff_tile_kernel(FfProduct p, int tiles_m, int tiles_n) {
  constexpr int NW = WM * WN, RB = BM / WM / 16, CB = BN / WN / 16;
  constexpr int PARTS = EPI == kFfGated ? 2 : 1;
  typedef TileOperand<BM, NW, AX> OpA;
  typedef TileOperand<BN, NW, BX> OpB;
  constexpr int STAGE = OpA::BYTES + OpB::BYTES;
  extern __shared__ __attribute__((aligned(1024))) unsigned char tile_smem[];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int wm = wave / WN, wn = wave % WN;
  int tm, tn;
  tile_of(blockIdx.x, tiles_m * tiles_n, tiles_m, tiles_n, &tm, &tn);
  const int m0 = tm * BM, n0 = tn * (BN / PARTS);
  const int left_m = p.M - m0, left_n = p.N - n0;

  const int per = (p.K + kStageK - 1) / kStageK, stages = per * (EPI == kFfGated ? 1 : p.segments);
  OpA a;
  OpB b;
  const long long lda = AX ? p.A[0].ks : p.A[0].rs, ldb = BX ? p.B[0].ks : p.B[0].rs;
  a.template init<1>(wave, lane, left_m, lda);
  b.template init<PARTS>(wave, lane, left_n, ldb);
  const long long a_at = (AX ? m0 : m0 * lda) * 2, b_at = (BX ? n0 : n0 * ldb) * 2;
  auto load = [&](int t) {
    unsigned char* st = tile_smem + (t & 1) * STAGE;
    const int s = t >= per ? 1 : 0, k0 = (t - s * per) * kStageK;
    a.template load<1>(st, wave, (const char*)p.A[s].p + a_at, nullptr, lda, left_m, k0, p.K);
    b.template load<PARTS>(st + OpA::BYTES, wave, (const char*)p.B[s].p + b_at, (const char*)p.B[1].p + b_at, ldb, left_n, k0, p.K);
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

  if (stages > 0) load(0);
  for (int t = 0; t < stages; ++t) {
    // this stage's loads have landed and nobody reads the other buffer any more
    __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0)
    __syncthreads();
    if (t + 1 < stages) load(t + 1);
    const unsigned char *sa = tile_smem + (t & 1) * STAGE, *sb = sa + OpA::BYTES;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      s16x8 fa[RB], fb[CB];
#pragma unroll
      for (int j = 0; j < CB; ++j) fb[j] = OpB::read(sb, lane, row_b(j), h);
#pragma unroll
      for (int i = 0; i < RB; ++i) fa[i] = OpA::read(sa, lane, wm * (BM / WM) + i * 16, h);
#pragma unroll
      for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int j = 0; j < CB; ++j) acc[j][i] = tile_mfma<TYPE>(fb[j], fa[i], acc[j][i]);
    }
  }

  constexpr int OUT = CB / PARTS;  // blocks of columns of the result
  float bias[OUT][4] = {};
  if (EPI == kFfLinear && p.bias)
#pragma unroll
    for (int j = 0; j < OUT; ++j) load4<TYPE>(bias[j], p.bias, n0 + row_b(j) + (lane >> 4) * 4, p.N - (n0 + row_b(j) + (lane >> 4) * 4));
#pragma unroll
  for (int i = 0; i < RB; ++i) {
    const int m = m0 + wm * (BM / WM) + i * 16 + (lane & 15);
    if (m >= p.M) continue;
#pragma unroll
    for (int j = 0; j < OUT; ++j) {
      const int n = n0 + row_b(j) + (lane >> 4) * 4;
      if (n >= p.N) continue;
      float v[4], u[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[e] = acc[j][i][e];
        u[e] = acc[PARTS == 2 ? j + OUT : j][i][e];
      }
      finish4<TYPE, EPI>(p, m, n, v, u, bias[j]);
    }
  }
}

}  // namespace
}  // namespace cct
