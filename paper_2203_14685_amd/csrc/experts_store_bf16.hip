// The products that are stored as they are (plus a bias), bf16.
#include "experts_tiles_bf16.hpp"

namespace hetumoe {

hipError_t expert_store_bf16(const ExpertArgs& x, const ExpertGemmArgs& a, int ka, int kb, hipStream_t st) {
  return by_tile(x, a.M, a.N, [&](auto tile) {
    using TL = decltype(tile);
    if (ka == kCols) return launch_tile_bf16<TL, kCols, kCols, kEpiStore, false>(x, a, st);
    if (kb == kCols) return launch_tile_bf16<TL, kRows, kCols, kEpiStore, false>(x, a, st);
    return launch_tile_bf16<TL, kRows, kRows, kEpiStore, false>(x, a, st);
  });
}

}  // namespace hetumoe
