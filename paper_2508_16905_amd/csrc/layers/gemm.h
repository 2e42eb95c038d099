// The matrix products of the layer operators: C[i][j] = sum_k A(i, k) B(j, k) with an epilogue, on the matrix cores.
//
// An operand lies with its k contiguous (KC: element (i, k) at p[i ld + k]) or with its rows contiguous (KS: at p[k ld + i]):
//   y = x W^T    A = x (KC),   B = W (KC)
//   dx = dz W    A = dz (KC),  B = W (KS)
//   dW = dz^T x  A = dz (KS),  B = x (KS)
// A tile of an operand goes to LDS as it lies in memory; a KS tile is turned on its way to the registers (ds_read_b64_tr_b16).
//
// FP32 operands are split into three bf16 parts, x = h + 2^-8 m + 2^-16 l with |m| <= |x| / 2 and |l| <= |x| / 4 (exact: 3 x 8 bits;
// the parts are kept scaled up, so that those of subnormal numbers do not fall below bf16's own), and of the nine partial
// products the six largest are summed, those of one scale in one accumulator; what is dropped is at most 2^-26 of a product.
// Six bf16 products have 2.6 times the rate of the fp32 matrix instructions (2.5 PFLOP/s / 6 = 417 and 157 TFLOP/s).
#pragma once
#include "layer_util.h"

namespace triaccel {
namespace layers {

enum Layout : int { KC = 0, KS = 1 };
enum Epi : int { kEpiLinear = 0, kEpiGated = 1, kEpiStore = 2 };

struct GemmArgs {
  const void *a, *b, *b2;   // b2: B of the second segment of k, or with kEpiGated the second matrix
  int64_t lda, ldb;
  int32_t m, n;             // rows and columns of the result (kEpiGated: n columns from each of b and b2)
  int32_t seg, nseg;        // k = nseg segments of `seg`
  int32_t seg_step;         // where segment 1 of A (KC) begins
  int32_t tiles_m, tiles_n, splits, tiles_per_split;
  float* partial;           // splits > 1: [splits][m][n or 2 n] sums
  // epilogue
  void *c, *c2;             // kEpiStore: rows >= csplit of the result are rows of c2, rows crows .. csplit - 1 go nowhere
  int64_t ldc;
  int32_t crows, csplit, c_fp32;
  void *pre, *pre2;
  int64_t ldpre;
  const void *bias, *bias2;
  const void* residual;
  int64_t ldr;
  int32_t bias_dtype, act;
  Drop drop;
};

__device__ const uint32_t kZeroPage[4] = {0, 0, 0, 0};

// ---- epilogue of eight columns of one row ------------------------------------------------------------------------
struct ColumnState {
  float bias[8], bias2[8];
  DropKey key;
};
template <int EPI>
__device__ __forceinline__ void epi_columns(const GemmArgs& g, int64_t col, ColumnState& s) {
  if constexpr (EPI != kEpiStore) {
#pragma unroll
    for (int i = 0; i < 8; ++i) s.bias[i] = s.bias2[i] = 0.0f;
    if (g.bias && col < g.n) {
      load8_of(g.bias_dtype, g.bias, col, g.n - col, s.bias);
      if constexpr (EPI == kEpiGated) load8_of(g.bias_dtype, g.bias2, col, g.n - col, s.bias2);
    }
  }
  if constexpr (EPI == kEpiLinear) {
    if (g.drop.limit) s.key = drop_key(g.drop);
  }
}
template <int DT, int EPI>
__device__ __forceinline__ void epi_row(const GemmArgs& g, const ColumnState& s, int64_t row, int64_t col, float (&v)[8], float (&u)[8]) {
  const int64_t left = g.n - col;
  constexpr bool kExact = DT == kFP32;
  if constexpr (EPI == kEpiStore) {
    const bool second = row >= g.csplit;
    if (!second && row >= g.crows) return;
    void* c = second ? g.c2 : g.c;
    const int64_t at = (second ? row - g.csplit : row) * g.ldc + col;
    if (g.c_fp32) store8<kFP32>(c, at, left, v);
    else store8<DT>(c, at, left, v);
  } else if constexpr (EPI == kEpiGated) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[i] += s.bias[i];
      u[i] += s.bias2[i];
    }
    if (g.pre) {
      store8<DT>(g.pre, row * g.ldpre + col, left, v);
      store8<DT>(g.pre2, row * g.ldpre + col, left, u);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = act_value<kExact>(g.act, v[i]) * u[i];
    store8<DT>(g.c, row * g.ldc + col, left, v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += s.bias[i];
    if (g.pre) store8<DT>(g.pre, row * g.ldpre + col, left, v);
    if (g.act != kNone) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = act_value<kExact>(g.act, v[i]);
    }
    scale_drop8(g.drop, s.key, (uint64_t)row * (uint32_t)g.n + (uint64_t)col, v);
    if (g.residual) {
      float r[8];
      load8<DT>(g.residual, row * g.ldr + col, left, r);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] += r[i];
    }
    store8<DT>(g.c, row * g.ldc + col, left, v);
  }
}

// ---- tiles in LDS ------------------------------------------------------------------------------------------------
// In units of eight elements (16 bytes) of one plane.  KC: row after row of BK, the units of a row exchanged by its number, so
// that eight rows' reads of one k fall on all banks.  KS: k after k of R rows, pairs of units exchanged by k: an instruction
// that turns reads 32 bytes of each of sixteen k.
template <int L, int R, int BK>
__device__ __forceinline__ int tile_unit(int row_or_k, int unit) {
  if constexpr (L == KC) {
    constexpr int kUnits = BK / 8;
    const int x = kUnits >= 8 ? (row_or_k & 7) : ((row_or_k >> 1) & (kUnits - 1));
    return row_or_k * kUnits + (unit ^ x);
  } else {
    constexpr int kUnits = R / 8;
    const int f = (row_or_k & 3) | ((row_or_k >> 1) & 4);
    const int x = (f & (kUnits / 2 - 1)) << 1;
    return row_or_k * kUnits + (unit ^ x);
  }
}
// The fragment of sixteen rows at `row0` and 32 k at `k0` (a lane's row: lane % 16, its eight k: 8 (lane / 16) ...).
template <int L, int R, int BK>
__device__ __forceinline__ s16x8 fragment(const short* tile, int row0, int k0, int lane) {
  if constexpr (L == KC) {
    const int row = row0 + (lane & 15);
    return *(const s16x8*)(tile + 8 * tile_unit<L, R, BK>(row, (k0 >> 3) + (lane >> 4)));
  } else {
    typedef __attribute__((address_space(3))) s16x4 Lds4;
    const int k = k0 + 8 * (lane >> 4) + ((lane & 15) >> 2);
    const int unit = (row0 >> 3) + ((lane >> 1) & 1), half = (lane & 1) * 4;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds4*)(tile + 8 * tile_unit<L, R, BK>(k, unit) + half));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds4*)(tile + 8 * tile_unit<L, R, BK>(k + 4, unit) + half));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  }
}

template <int DT>
__device__ __forceinline__ f32x4 mfma(s16x8 a, s16x8 b, f32x4 c) {
  if constexpr (DT == kFP16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Rounded to bf16; cut off instead where rounding would make an infinity of a number.
__device__ __forceinline__ uint32_t part_bits(float x) {
  const uint32_t b = f32_to_bf16_bits(x);
  return (b & 0x7fffu) == 0x7f80u ? f2u(x) >> 16 : b;
}
// fp32 -> three bf16 parts.  A rest is below 2^120 and its multiple below 2^128; what is not finite has no rest.
__device__ __forceinline__ void split3(const Elem8<kFP32>& v, s16x8 (&out)[3]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t h = part_bits(v[i]);
    const float r = __builtin_isfinite(v[i]) ? (v[i] - bf16_bits_to_f32(h)) * 256.0f : 0.0f;
    const uint32_t m = part_bits(r);
    out[0][i] = (short)h;
    out[1][i] = (short)m;
    out[2][i] = (short)part_bits((r - bf16_bits_to_f32(m)) * 256.0f);
  }
}

template <int DT, int LA, int LB, int BM, int BN, int WR, int WC, int EPI, bool DIRECT>
struct Gemm {
  static constexpr int kPlanes = DT == kFP32 ? 3 : 1;
  static constexpr int BK = DT == kFP32 ? 32 : 64;
  static constexpr int NT = WR * WC * 64;
  static constexpr int FM = BM / WR / 16, FN = BN / WC / 16;
  static constexpr int kAUnits = BM * BK / 8, kBUnits = BN * BK / 8;
  static constexpr int TA = kAUnits / NT, TB = kBUnits / NT;
  static constexpr int kTile = kPlanes * (BM + BN) * BK;  // elements of one buffer
  static constexpr int kSlabCols = FN * 16, kSlabLd = kSlabCols + 4;
  static constexpr int kRound = FM < 4 ? FM : 4;          // fragments of rows that its slab holds at a time
  static constexpr int kSlab = 16 * kRound * kSlabLd;     // floats of a wavefront
  static constexpr int kTileBytes = 2 * kTile * 2, kSlabBytes = WR * WC * kSlab * 4;
  static constexpr int kLdsBytes = kTileBytes > kSlabBytes ? kTileBytes : kSlabBytes;
  // columns of the result that a tile has
  static constexpr int kCols = EPI == kEpiGated ? BN / 2 : BN;
  static_assert(TA >= 1 && TB >= 1 && kAUnits % NT == 0 && kBUnits % NT == 0, "whole units per thread");
  static_assert(EPI != kEpiGated || FN % 2 == 0, "half of a wavefront's columns from each matrix");
  typedef Elem<DT> E;
  typedef f32x4 Acc[kPlanes][FM][FN];  // [q]: what counts 2^-8q

  // Row of B (0 .. BN - 1) -> its matrix and row there.  With two matrices each wavefront has as many rows of the one as of
  // the other, for the same columns of the result, so that the epilogue has both in one lane.
  static __device__ __forceinline__ int b_row(int j, bool& second) {
    if constexpr (EPI == kEpiGated) {
      constexpr int kHalf = FN * 8, kFull = FN * 16;
      second = (j % kFull) >= kHalf;
      return j / kFull * kHalf + j % kHalf;
    } else {
      second = false;
      return j;
    }
  }

  // One tile of k: where it begins.
  struct At {
    int seg, k0, left;  // `left`: k in its segment from k0 on
  };
  static __device__ __forceinline__ At at(const GemmArgs& g, int kt) {
    const int per = g.seg > 0 ? (g.seg + BK - 1) / BK : 1;
    const int s = kt >= per ? 1 : 0;
    const int k0 = (kt - s * per) * BK;
    return At{s, k0, g.seg - k0};
  }

  // --- straight to LDS: aligned operands (see direct_ok) ---
  template <int L, int R, int T, bool IS_B>
  static __device__ __forceinline__ void issue(const GemmArgs& g, const At& w, int r0, int rows, short* tile, int tid) {
    const int64_t ld = IS_B ? g.ldb : g.lda;
    const bool full = w.left >= BK;
    const E* p0 = (const E*)(IS_B ? (w.seg ? g.b2 : g.b) : g.a);
    const E* p1 = (const E*)g.b2;
    const int64_t koff = (IS_B ? 0 : (int64_t)w.seg * g.seg_step) + w.k0;
    const int64_t skip = L == KC ? (int64_t)r0 * ld + koff : koff * ld + r0;
#pragma unroll
    for (int t = 0; t < T; ++t) {
      const int slot = t * NT + tid;
      const char* src;
      if constexpr (L == KC) {
        const int row = slot / (BK / 8), unit = (tile_unit<KC, R, BK>(row, slot % (BK / 8))) % (BK / 8);
        bool second = false;
        int r = IS_B ? b_row(row, second) : row;
        r = r0 + r < rows ? r : rows - 1 - r0;
        src = (const char*)((second ? p1 : p0) + skip) + (uint32_t)(r * (int)ld + unit * 8) * 2u;
        if (!full && unit * 8 >= w.left) src = (const char*)kZeroPage;
      } else {
        const int k = slot / (R / 8), unit = (tile_unit<KS, R, BK>(k, slot % (R / 8))) % (R / 8);
        int c = unit * 8;
        c = r0 + c < rows ? c : ((rows + 7) & ~7) - 8 - r0;  // the row's stride has room for whole units
        src = (const char*)(p0 + skip) + (uint32_t)(k * (int)ld + c) * 2u;
        if (!full && k >= w.left) src = (const char*)kZeroPage;
      }
      // lane i's 16 bytes go to the wavefront's place plus 16 i: slot `slot`
      __builtin_amdgcn_global_load_lds((const TA_GLOBAL char*)src,
                                       (__attribute__((address_space(3))) char*)tile + (t * NT + (tid & ~63)) * 16, 16, 0, 0);
    }
  }

  // --- through registers: any alignment, any strides, any sizes ---
  template <int L, int R, int T, bool IS_B>
  static __device__ __forceinline__ void fetch(const GemmArgs& g, const At& w, int r0, int rows, Elem8<DT> (&out)[T], int tid) {
    const int64_t ld = IS_B ? g.ldb : g.lda;
    const E* p = (const E*)(IS_B ? (w.seg ? g.b2 : g.b) : g.a);
    const int64_t koff = (IS_B ? 0 : (int64_t)w.seg * g.seg_step) + w.k0;
#pragma unroll
    for (int t = 0; t < T; ++t) {
      const int slot = t * NT + tid;
      if constexpr (L == KC) {
        const int row = slot / (BK / 8), unit = slot % (BK / 8);
        bool second = false;
        const int r = r0 + (IS_B ? b_row(row, second) : row);
        const E* q = second ? (const E*)g.b2 : p;
        out[t] = load_raw8<DT>(q + (int64_t)r * ld + koff + unit * 8, r < rows ? w.left - unit * 8 : 0);
      } else {
        const int k = slot / (R / 8), c = r0 + slot % (R / 8) * 8;
        out[t] = load_raw8<DT>(p + (koff + k) * ld + c, k < w.left ? rows - c : 0);
      }
    }
  }
  template <int L, int R, int T>
  static __device__ __forceinline__ void place(const Elem8<DT> (&in)[T], short* tile, int tid) {
#pragma unroll
    for (int t = 0; t < T; ++t) {
      const int slot = t * NT + tid;
      const int u = L == KC ? tile_unit<KC, R, BK>(slot / (BK / 8), slot % (BK / 8)) : tile_unit<KS, R, BK>(slot / (R / 8), slot % (R / 8));
      if constexpr (DT == kFP32) {
        s16x8 part[3];
        split3(in[t], part);
#pragma unroll
        for (int q = 0; q < 3; ++q) *(s16x8*)(tile + q * R * BK + 8 * u) = part[q];
      } else {
        *(s16x8*)(tile + 8 * u) = __builtin_bit_cast(s16x8, in[t]);
      }
    }
  }

  static __device__ __forceinline__ void multiply(const short* tile, Acc& acc, int wm, int wn, int lane) {
    const short* ta = tile;
    const short* tb = tile + kPlanes * BM * BK;
#pragma unroll
    for (int k0 = 0; k0 < BK; k0 += 32) {
      s16x8 b[FN][kPlanes];
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int q = 0; q < kPlanes; ++q) b[j][q] = fragment<LB, BN, BK>(tb + q * BN * BK, wn * FN * 16 + j * 16, k0, lane);
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        s16x8 a[kPlanes];
#pragma unroll
        for (int q = 0; q < kPlanes; ++q) a[q] = fragment<LA, BM, BK>(ta + q * BM * BK, wm * FM * 16 + i * 16, k0, lane);
        // B first: a lane then has four neighbouring columns of one row of the result
#pragma unroll
        for (int j = 0; j < FN; ++j) {
          if constexpr (kPlanes == 3) {
            acc[2][i][j] = mfma<kBF16>(b[j][2], a[0], acc[2][i][j]);
            acc[1][i][j] = mfma<kBF16>(b[j][1], a[0], acc[1][i][j]);
            acc[0][i][j] = mfma<kBF16>(b[j][0], a[0], acc[0][i][j]);
            acc[2][i][j] = mfma<kBF16>(b[j][0], a[2], acc[2][i][j]);
            acc[1][i][j] = mfma<kBF16>(b[j][0], a[1], acc[1][i][j]);
            acc[2][i][j] = mfma<kBF16>(b[j][1], a[1], acc[2][i][j]);
          } else {
            acc[0][i][j] = mfma<DT>(b[j][0], a[0], acc[0][i][j]);
          }
        }
      }
    }
  }

  // Up to 64 rows at a time through the wavefront's own slab of LDS: a lane's four columns become eight of one row, so that
  // bias, dropout's generator, residual and stores work on 16 bytes.
  static __device__ __forceinline__ void finish(const GemmArgs& g, const f32x4 (&acc)[FM][FN], float* slab, int row0, int col0, int lane, int split) {
    constexpr int kOut = EPI == kEpiGated ? kSlabCols / 2 : kSlabCols, kLanes = kOut / 8, kRows = 64 / kLanes < 16 ? 64 / kLanes : 16;
    const int col = col0 + lane % kLanes * 8, sub = lane / kLanes;
    const bool mine = col < g.n && sub < kRows;
    const bool partial = g.splits > 1;
    ColumnState state;
    if (!partial) epi_columns<EPI>(g, col, state);
    static_assert(FM % kRound == 0, "whole rounds");
#pragma unroll
    for (int h = 0; h < FM; h += kRound) {
#pragma unroll
      for (int i = 0; i < kRound; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) *(f32x4*)(slab + (i * 16 + (lane & 15)) * kSlabLd + j * 16 + (lane >> 4) * 4) = acc[h + i][j];
      __builtin_amdgcn_wave_barrier();
#pragma unroll 1
      for (int r = sub; r < 16 * kRound; r += kRows) {
        const int row = row0 + h * 16 + r;
        if (mine && row < g.m) {
          const float* q = slab + r * kSlabLd + lane % kLanes * 8;
          float v[8], u[8];
          *(f32x4*)v = *(const f32x4*)q;
          *(f32x4*)(v + 4) = *(const f32x4*)(q + 4);
          if constexpr (EPI == kEpiGated) {
            *(f32x4*)u = *(const f32x4*)(q + kOut);
            *(f32x4*)(u + 4) = *(const f32x4*)(q + kOut + 4);
          }
          if (partial) {
            const int64_t width = EPI == kEpiGated ? 2 * (int64_t)g.n : g.n;
            const int64_t base = ((int64_t)split * g.m + row) * width + col;
            store8<kFP32>(g.partial, base, g.n - col, v);
            if constexpr (EPI == kEpiGated) store8<kFP32>(g.partial, base + g.n, g.n - col, u);
          } else {
            epi_row<DT, EPI>(g, state, row, col, v, u);
          }
        }
      }
      __builtin_amdgcn_wave_barrier();
    }
  }

  // Workgroups go to the eight XCDs in turn.  Each XCD gets a run of neighbouring tiles, four tile rows at a time, so that what
  // its workgroups read at one time is shared in its L2.
  static __device__ __forceinline__ void place_of(const GemmArgs& g, int& tm, int& tn, int& split) {
    const int total = g.tiles_m * g.tiles_n * g.splits, id = blockIdx.x;
    const int xcd = id & 7, per = total >> 3, more = total & 7;
    const int lin = xcd * per + (xcd < more ? xcd : more) + (id >> 3);
    const int tiles = g.tiles_m * g.tiles_n;
    split = lin / tiles;
    const int t = lin - split * tiles;
    constexpr int kGroup = 4;
    const int band = t / (kGroup * g.tiles_n), in = t - band * kGroup * g.tiles_n;
    const int high = g.tiles_m - band * kGroup < kGroup ? g.tiles_m - band * kGroup : kGroup;
    tm = band * kGroup + in % high;
    tn = in / high;
  }

  static __device__ __forceinline__ void run(const GemmArgs& g, short* lds) {
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave / WC, wn = wave % WC;
    int tm, tn, split;
    place_of(g, tm, tn, split);
    const int r0 = tm * BM, c0 = tn * kCols;
    const int all = g.seg > 0 ? (g.seg + BK - 1) / BK * g.nseg : 0;
    const int first = split * g.tiles_per_split, last = first + g.tiles_per_split < all ? first + g.tiles_per_split : all;
    Acc acc;
#pragma unroll
    for (int q = 0; q < kPlanes; ++q)
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[q][i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    if constexpr (DIRECT) {
      auto load = [&](int kt, short* to) {
        const At w = at(g, kt);
        issue<LA, BM, TA, false>(g, w, r0, g.m, to, tid);
        issue<LB, BN, TB, true>(g, w, c0, g.n, to + BM * BK, tid);
      };
      if (first < last) load(first, lds);
      for (int kt = first; kt < last; ++kt) {
        __builtin_amdgcn_s_waitcnt(0);
        __syncthreads();  // this tile has arrived for all wavefronts, and nobody reads the other buffer any more
        if (kt + 1 < last) load(kt + 1, lds + ((kt - first + 1) & 1) * kTile);
        multiply(lds + ((kt - first) & 1) * kTile, acc, wm, wn, lane);
      }
    } else {
      Elem8<DT> ra[TA], rb[TB];
      auto load = [&](int kt) {
        const At w = at(g, kt);
        fetch<LA, BM, TA, false>(g, w, r0, g.m, ra, tid);
        fetch<LB, BN, TB, true>(g, w, c0, g.n, rb, tid);
      };
      auto put = [&](short* to) {
        place<LA, BM, TA>(ra, to, tid);
        place<LB, BN, TB>(rb, to + kPlanes * BM * BK, tid);
      };
      if (first < last) {
        load(first);
        put(lds);
      }
      for (int kt = first; kt < last; ++kt) {
        __syncthreads();
        if (kt + 1 < last) load(kt + 1);
        multiply(lds + ((kt - first) & 1) * kTile, acc, wm, wn, lane);
        if (kt + 1 < last) put(lds + ((kt - first + 1) & 1) * kTile);
      }
    }
    __syncthreads();
    if constexpr (kPlanes == 3) {
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[0][i][j][e] = fmaf(fmaf(acc[2][i][j][e], 0.00390625f, acc[1][i][j][e]), 0.00390625f, acc[0][i][j][e]);
    }
    finish(g, acc[0], (float*)lds + wave * kSlab, r0 + wm * FM * 16, c0 + wn * (EPI == kEpiGated ? FN * 8 : FN * 16), lane, split);
  }
};

template <typename G>
__global__ __launch_bounds__(G::NT) void k_gemm(GemmArgs g) {
  __shared__ __attribute__((aligned(16))) short lds[G::kLdsBytes / 2];
  G::run(g, lds);
}

// The sums of a product whose k was split: eight columns of a row per thread, the splits in order, then the epilogue.
template <int DT, int EPI>
__global__ __launch_bounds__(256) void k_join(GemmArgs g) {
  const int64_t groups = (g.n + 7) / 8, id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t row = id / groups, col = (id - row * groups) * 8;
  if (row >= g.m) return;
  const int64_t width = EPI == kEpiGated ? 2 * (int64_t)g.n : g.n, left = g.n - col;
  float v[8] = {}, u[8] = {};
  for (int s = 0; s < g.splits; ++s) {
    const int64_t base = ((int64_t)s * g.m + row) * width + col;
    float t[8];
    load8<kFP32>(g.partial, base, left, t);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += t[i];
    if constexpr (EPI == kEpiGated) {
      load8<kFP32>(g.partial, base + g.n, left, t);
#pragma unroll
      for (int i = 0; i < 8; ++i) u[i] += t[i];
    }
  }
  ColumnState state;
  epi_columns<EPI>(g, col, state);
  epi_row<DT, EPI>(g, state, row, col, v, u);
}

}  // namespace layers
}  // namespace triaccel
