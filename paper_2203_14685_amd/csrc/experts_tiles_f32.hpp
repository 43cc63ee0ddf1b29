// Tile choice of the batched f32 products.
#pragma once

#include "experts_f32.hpp"
#include "experts_launch.hpp"

namespace hetumoe {

// KG: groups of waves along K; PER: blocks that a CU holds.
template <int BM, int BN, int WM, int WN, int KG, int PER>
struct Tile {
  static constexpr int bm = BM, bn = BN, wm = WM, wn = WN, kg = KG, per_cu = PER;
};

template <class Fn>
static hipError_t by_tile(const ExpertArgs& x, int M, int N, Fn fn) {
  // tiles of 128 x 128 once they fill the CUs, else 64 x 64
  const int64_t big = static_cast<int64_t>(x.E) * ((M + 127) / 128) * ((N + 127) / 128);
  if (M > 64 && big >= 256) return fn(Tile<128, 128, 2, 2, 1, 2>());
  return fn(Tile<64, 64, 4, 1, 4, 1>());
}

template <class TL, int KA, int KB, int EPI, bool GATED>
static hipError_t launch_tile_f32(const ExpertArgs& x, ExpertGemmArgs a, hipStream_t st) {
  expert_set_tiles(a, x.E, TL::bm, EPI == kEpiAct && GATED ? TL::bn / 2 : TL::bn);
  experts_gemm_f32_kernel<TL::bm, TL::bn, TL::wm, TL::wn, TL::kg, KA, KB, EPI, GATED>
      <<<dim3(expert_blocks(a.tiles, TL::per_cu * device_cu_count())), dim3(TL::wm * TL::wn * TL::kg * kWave), 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace hetumoe
