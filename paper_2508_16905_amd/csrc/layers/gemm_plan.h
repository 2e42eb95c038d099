// How a product is cut into workgroups: host side, from sizes alone.
#pragma once
#include <stdint.h>

namespace triaccel {
namespace layers {

enum Tile : int { kTileS = 0, kTileM = 1, kTileL = 2 };

struct GemmPlan {
  int tile;
  int32_t tiles_m, tiles_n, splits, tiles_per_split;
  uint64_t partial_bytes;
};

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// m x n results (gated: n columns of two products), k = nseg segments of seg.  `direct`: operands that can go straight to LDS.
inline GemmPlan plan_gemm(bool fp32, bool gated, bool direct, int64_t m, int64_t n, int64_t seg, int64_t nseg) {
  GemmPlan p{};
  const int64_t half = gated ? 2 : 1;
  const auto tiles = [&](int64_t edge) { return ceil_div(m, edge) * ceil_div(n * half, edge); };
  p.tile = !fp32 && direct && tiles(256) >= 160 ? kTileL : tiles(128) >= 128 ? kTileM : kTileS;
  const int64_t edge = p.tile == kTileL ? 256 : p.tile == kTileM ? 128 : 64;
  p.tiles_m = (int32_t)ceil_div(m, edge);
  p.tiles_n = (int32_t)ceil_div(n * half, edge);
  const int64_t k_tiles = seg > 0 ? ceil_div(seg, fp32 ? 32 : 64) * nseg : 1, all = (int64_t)p.tiles_m * p.tiles_n;
  int64_t splits = 1;
  if (all < 256 && k_tiles >= 8) {
    splits = 512 / all;
    if (splits > k_tiles / 4) splits = k_tiles / 4;
    if (splits > 32) splits = 32;
    if (splits < 1) splits = 1;
  }
  p.tiles_per_split = (int32_t)ceil_div(k_tiles, splits);
  p.splits = (int32_t)ceil_div(k_tiles, p.tiles_per_split);
  p.partial_bytes = p.splits > 1 ? (uint64_t)p.splits * (uint64_t)m * (uint64_t)(n * half) * 4u : 0;
  return p;
}

}  // namespace layers
}  // namespace triaccel
