// How a product is cut into workgroups: host side, from sizes and the alignment of its operands alone.
#pragma once
#include <stdint.h>

namespace triaccel {
namespace layers {

// S: 64 x 64, staged.  M: 128 x 128, L: 256 x 256, both in the wide form.
// Short: as S, where an operand's rows are shorter than eight.  Thin: forward products of at most 16 rows (thin.h).
enum Tile : int { kTileS = 0, kTileM = 1, kTileL = 2, kTileShort = 3, kTileThin = 4 };

struct GemmPlan {
  int tile, groups;         // groups: of wavefronts that share the k of a tile (S)
  int32_t tiles_m, tiles_n, whole, splits, per_split;
  uint64_t partial_bytes;
  double us;                // what the model below expects
};

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// The model, in microseconds: a workgroup computes a tile at a rate of its own, the card holds `slots` of them, and what is
// left over after whole rounds of `slots` tiles is shared out over k where that is shorter (the sums then go through memory
// and a second launch).
inline GemmPlan plan_tile(int tile, bool fp32, bool gated, int64_t m, int64_t n, int64_t seg, int64_t nseg) {
  const int64_t half = gated ? 2 : 1, bk = fp32 ? 32 : 64;
  const int64_t edge = tile == kTileL ? 256 : tile == kTileM ? 128 : 64;
  GemmPlan p{};
  p.tile = tile;
  p.tiles_m = (int32_t)ceil_div(m, edge);
  p.tiles_n = (int32_t)ceil_div(n * half, edge);
  const int64_t k_tiles = seg > 0 ? ceil_div(seg, bk) * nseg : 1, all = (int64_t)p.tiles_m * p.tiles_n;
  const bool small = tile == kTileS || tile == kTileShort;
  p.groups = tile == kTileS && k_tiles >= 4 && all <= 512 ? (fp32 ? 2 : 4) : 1;
  // microseconds of a tile of k, and of what a workgroup has besides
  const double per_k = tile == kTileL ? 1.75 : tile == kTileM ? (fp32 ? 1.85 : all > 256 ? 1.45 : 1.0) : (fp32 ? 2.7 : 1.2) / p.groups, fixed = 5.0;
  const int64_t slots = tile == kTileL ? 256 : tile == kTileM ? (fp32 ? 256 : 512) : p.groups > 1 ? 256 : 1024;
  const int64_t rounds = all / slots, rest = all % slots;
  const int64_t least = small ? 4 * p.groups : 8;  // tiles of k that a share has at least
  p.whole = (int32_t)all;
  p.splits = 1;
  p.per_split = (int32_t)k_tiles;
  p.us = (double)(rounds + (rest ? 1 : 0)) * (per_k * (double)k_tiles + fixed);
  if (rest) {
    int64_t s = slots / rest;
    if (s > k_tiles / least) s = k_tiles / least;
    if (s > 32) s = 32;
    if (s > 1) {
      const int64_t per = ceil_div(k_tiles, s);
      const uint64_t bytes = (uint64_t)rest * (uint64_t)ceil_div(k_tiles, per) * (uint64_t)(edge * edge) * 4u;
      const double us = (double)rounds * (per_k * (double)k_tiles + fixed) + per_k * (double)per + fixed + 7.0 + (double)bytes * 2.0 / 4.0e6;
      if (us < p.us) {
        p.us = us;
        p.whole = (int32_t)(all - rest);
        p.per_split = (int32_t)per;
        p.splits = (int32_t)ceil_div(k_tiles, per);
        p.partial_bytes = bytes;
      }
    }
  }
  return p;
}

// m x n results (gated: n columns of two products), k = nseg segments of seg.  `pack_us`: what it takes to lay the operands out
// for the wide form.
// `shortest`: the shortest row of an operand.
inline GemmPlan plan_gemm(bool fp32, bool gated, double pack_us, int64_t shortest, int64_t m, int64_t n, int64_t seg, int64_t nseg) {
  if (shortest < 8) return plan_tile(kTileShort, fp32, gated, m, n, seg, nseg);
  GemmPlan best = plan_tile(kTileS, fp32, gated, m, n, seg, nseg);
  for (int tile = kTileM; tile <= (fp32 ? kTileM : kTileL); ++tile) {
    const int64_t edge = tile == kTileL ? 256 : 128;
    // the wide form shifts its last tiles inwards: the result is no smaller than one of them, nor k than a unit
    if (m < edge || n * (gated ? 2 : 1) < edge || seg < 8) continue;
    const GemmPlan p = plan_tile(tile, fp32, gated, m, n, seg, nseg);
    if (p.us + pack_us < best.us + (best.tile == kTileS ? 0.0 : pack_us)) best = p;
  }
  return best;
}

}  // namespace layers
}  // namespace triaccel
