// The instances of the product kernels for one element type, and the choice among them.
#pragma once
#include "gemm.h"
#include "gemm_plan.h"
#include "layers.h"

namespace triaccel {
namespace layers {

template <int DT, int LA, int LB, int EPI>
hipError_t launch_product(const GemmPlan& p, bool direct, GemmArgs g, hipStream_t stream) {
  g.tiles_m = p.tiles_m;
  g.tiles_n = p.tiles_n;
  g.splits = p.splits;
  g.tiles_per_split = p.tiles_per_split;
  const dim3 grid((uint32_t)(p.tiles_m * p.tiles_n * p.splits));
  if constexpr (DT == kFP32) {
    if (p.tile == kTileM) {
      typedef Gemm<DT, LA, LB, 128, 128, 2, 2, EPI, false> M;
      k_gemm<M><<<grid, M::NT, 0, stream>>>(g);
    } else {
      typedef Gemm<DT, LA, LB, 64, 64, 2, 2, EPI, false> S;
      k_gemm<S><<<grid, S::NT, 0, stream>>>(g);
    }
  } else {
    if (p.tile == kTileL) {
      typedef Gemm<DT, LA, LB, 256, 256, 2, 4, EPI, true> L;
      k_gemm<L><<<grid, L::NT, 0, stream>>>(g);
    } else if (p.tile == kTileM && direct) {
      typedef Gemm<DT, LA, LB, 128, 128, 2, 2, EPI, true> M;
      k_gemm<M><<<grid, M::NT, 0, stream>>>(g);
    } else if (p.tile == kTileM) {
      typedef Gemm<DT, LA, LB, 128, 128, 2, 2, EPI, false> M;
      k_gemm<M><<<grid, M::NT, 0, stream>>>(g);
    } else {
      typedef Gemm<DT, LA, LB, 64, 64, 2, 2, EPI, false> S;
      k_gemm<S><<<grid, S::NT, 0, stream>>>(g);
    }
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.splits == 1) return e;
  const int64_t threads = (int64_t)g.m * ((g.n + 7) / 8);
  k_join<DT, EPI><<<dim3((uint32_t)ceil_div(threads, 256)), 256, 0, stream>>>(g);
  return hipGetLastError();
}

template <int DT>
hipError_t launch_any(Product kind, const GemmPlan& p, bool direct, const GemmArgs& g, hipStream_t stream) {
  switch (kind) {
    case kForward: return launch_product<DT, KC, KC, kEpiLinear>(p, direct, g, stream);
    case kGatedForward: return launch_product<DT, KC, KC, kEpiGated>(p, direct, g, stream);
    case kInputGrad: return launch_product<DT, KC, KS, kEpiStore>(p, direct, g, stream);
    default: return launch_product<DT, KS, KS, kEpiStore>(p, direct, g, stream);
  }
}

}  // namespace layers
}  // namespace triaccel
