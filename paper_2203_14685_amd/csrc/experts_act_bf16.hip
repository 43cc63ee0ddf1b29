// The product with the activation behind it, bf16.
#include "experts_tiles_bf16.hpp"

namespace hetumoe {

hipError_t expert_act_bf16(const ExpertArgs& x, const ExpertGemmArgs& a, hipStream_t st) {
  return by_tile(x, a.M, x.gated ? 2 * a.N : a.N, [&](auto tile) {
    using TL = decltype(tile);
    return x.gated ? launch_tile_bf16<TL, kRows, kCols, kEpiAct, true>(x, a, st)
                   : launch_tile_bf16<TL, kRows, kCols, kEpiAct, false>(x, a, st);
  });
}

}  // namespace hetumoe
