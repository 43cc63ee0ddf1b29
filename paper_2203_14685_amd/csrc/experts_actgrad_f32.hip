// The product with the activation's gradient behind it, f32.
#include "experts_tiles_f32.hpp"

namespace hetumoe {

hipError_t expert_actgrad_f32(const ExpertArgs& x, const ExpertGemmArgs& a, hipStream_t st) {
  return by_tile(x, a.M, a.N, a.K, [&](auto tile) {
    using TL = decltype(tile);
    return x.gated ? launch_tile_f32<TL, kRows, kRows, kEpiActGrad, true>(x, a, st)
                   : launch_tile_f32<TL, kRows, kRows, kEpiActGrad, false>(x, a, st);
  });
}

int expert_parts_f32(const ExpertArgs& x) {
  int parts = 0;
  (void)by_tile(x, x.C, x.h, x.d, [&](auto tile) {
    using TL = decltype(tile);
    parts = (x.C + TL::bm - 1) / TL::bm * TL::wm;
    return hipSuccess;
  });
  return parts;
}

}  // namespace hetumoe
