// The products that are stored as they are (plus a bias), f32.
#include "experts_tiles_f32.hpp"

namespace hetumoe {

hipError_t expert_store_f32(const ExpertArgs& x, const ExpertGemmArgs& a, int ka, int kb, hipStream_t st) {
  return by_tile(x, a.M, a.N, a.k_is_rows ? a.C : a.K, [&](auto tile) {
    using TL = decltype(tile);
    if (ka == kCols) return launch_tile_f32<TL, kCols, kCols, kEpiStore, false>(x, a, st);
    if (kb == kCols) return launch_tile_f32<TL, kRows, kCols, kEpiStore, false>(x, a, st);
    return launch_tile_f32<TL, kRows, kRows, kEpiStore, false>(x, a, st);
  });
}

}  // namespace hetumoe
