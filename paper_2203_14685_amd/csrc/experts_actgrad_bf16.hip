// The product with the activation's gradient behind it, bf16.
#include "experts_tiles_bf16.hpp"

namespace hetumoe {

hipError_t expert_actgrad_bf16(const ExpertArgs& x, const ExpertGemmArgs& a, hipStream_t st) {
  return by_tile(x, a.M, a.N, [&](auto tile) {
    using TL = decltype(tile);
    return x.gated ? launch_tile_bf16<TL, kRows, kRows, kEpiActGrad, true>(x, a, st)
                   : launch_tile_bf16<TL, kRows, kRows, kEpiActGrad, false>(x, a, st);
  });
}

int expert_parts_bf16(const ExpertArgs& x) {
  int parts = 0;
  (void)by_tile(x, x.C, x.h, [&](auto tile) {
    using TL = decltype(tile);
    parts = (x.C + TL::bm - 1) / TL::bm * TL::wm;
    return hipSuccess;
  });
  return parts;
}

}  // namespace hetumoe
