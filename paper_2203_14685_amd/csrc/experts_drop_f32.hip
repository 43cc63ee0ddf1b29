// The products of the activation and of its gradient with dropout of hidden, f32.
#include "experts_tiles_f32.hpp"

namespace hetumoe {

hipError_t expert_act_drop_f32(const ExpertArgs& x, const ExpertGemmArgs& a, hipStream_t st) {
  return by_tile(x, a.M, x.gated ? 2 * a.N : a.N, a.K, [&](auto tile) {
    using TL = decltype(tile);
    return x.gated ? launch_tile_f32<TL, kRows, kCols, kEpiActDrop, true>(x, a, st)
                   : launch_tile_f32<TL, kRows, kCols, kEpiActDrop, false>(x, a, st);
  });
}

hipError_t expert_actgrad_drop_f32(const ExpertArgs& x, const ExpertGemmArgs& a, hipStream_t st) {
  return by_tile(x, a.M, a.N, a.K, [&](auto tile) {
    using TL = decltype(tile);
    return x.gated ? launch_tile_f32<TL, kRows, kRows, kEpiActGradDrop, true>(x, a, st)
                   : launch_tile_f32<TL, kRows, kRows, kEpiActGradDrop, false>(x, a, st);
  });
}

}  // namespace hetumoe
