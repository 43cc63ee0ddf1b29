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
static hipError_t by_tile(const ExpertArgs& x, int M, int N, int K, Fn fn) {
  // Tiles of 128 x 128 for sums over 256 and more where two such blocks per CU find one and the
  // smaller tiles' rounds of 256, at 10/11 of the rate, do not take less (K = 1024, 8 x 1024 x
  // 1024: 153 us, tiles of 64 172; 8 x 512 x 1024, 512 tiles: 83 and 85; 8 x 128 x 4096, 256 tiles:
  // 107 and 96; dw of 16 x 64 x 1024 x 2048, whose sums are over 64: 99 and 69).
  //
  // For sums over 512 and more groups of waves share a tile of 64 x 64: two where two such
  // blocks per CU find a tile, four where one does, and where even that is not so, tiles of 32 x 32
  // by eight: what a CU has on its way from memory is what such products wait for (8 x 256 x 1024,
  // K = 1024, 512 tiles: four groups 50 us, two 45; 4 x 202 x 1792, K = 3264, 448 tiles: 132 and
  // 178; 8 x 128 x 256, K = 1024: one group 27 us, four 26, 32 x 32 by eight 12; 8 x 128 x 1024,
  // K = 256: one group 13.6 us, four 17.4).
  //
  // For at most 32 rows, whose weights are what there is to read, tiles of 32 x 64 by two groups
  // (forward of 82 x 1 x 3424 x 1216 752 us in tiles of 64, 517; of 64 x 32 x 1024 x 1024 158 and
  // 122; of 20 x 11 x 128 x 4952, whose second product has 40 tiles of 64, 50 us with 32 x 32 there,
  // 73 without).
  auto tiles = [&](int t) { return static_cast<int64_t>(x.E) * ((M + t - 1) / t) * ((N + t - 1) / t); };
  auto rounds = [&](int t) { return (tiles(t) + 255) / 256; };
  if (K >= 256 && tiles(128) >= 512 && 40 * rounds(128) <= 11 * rounds(64)) return fn(Tile<128, 128, 2, 2, 1, 2>());
  if (M <= 32 && tiles(64) >= 256) return fn(Tile<32, 64, 2, 2, 2, 2>());
  if (K < 512) return fn(Tile<64, 64, 4, 1, 1, 4>());
  if (tiles(64) >= 512) return fn(Tile<64, 64, 4, 1, 2, 2>());
  if (tiles(64) >= 256) return fn(Tile<64, 64, 4, 1, 4, 1>());
  return fn(Tile<32, 32, 2, 1, 8, 1>());
}

template <class TL, int KA, int KB, int EPI, bool GATED>
static hipError_t launch_tile_f32(const ExpertArgs& x, ExpertGemmArgs a, hipStream_t st) {
  expert_set_tiles(a, x.E, TL::bm, EPI == kEpiAct && GATED ? TL::bn / 2 : TL::bn);
  experts_gemm_f32_kernel<TL::bm, TL::bn, TL::wm, TL::wn, TL::kg, KA, KB, EPI, GATED>
      <<<dim3(expert_blocks(a.tiles, TL::per_cu * device_cu_count())), dim3(TL::wm * TL::wn * TL::kg * kWave), 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace hetumoe
