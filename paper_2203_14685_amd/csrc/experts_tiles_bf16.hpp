// Tile choice of the batched bf16 products.
#pragma once

#include "experts_bf16.hpp"
#include "experts_launch.hpp"

namespace hetumoe {

// PER: blocks that a CU holds.
template <int BM, int BN, int WM, int WN, int PER>
struct Tile {
  static constexpr int bm = BM, bn = BN, wm = WM, wn = WN, per_cu = PER;
};

// Rounds of tiles up to which the last one is worth a launch of its own.
constexpr int kMaxRounds = 16;

using SMALL = Tile<64, 64, 2, 1, 2>;
template <class Fn>
static hipError_t by_tile(const ExpertArgs& x, int M, int N, int K, Fn fn) {
  (void)K;
  // tiles of 256 x 256 once they fill the CUs, 64 x 256 where an expert has few
  // rows, else 128 x 128
  if (M <= 64) return fn(SMALL());
  const int64_t big = static_cast<int64_t>(x.E) * ((M + 255) / 256) * ((N + 255) / 256);
  if (big >= 256) return fn(Tile<256, 256, 2, 4, 1>());
  const int64_t mid = static_cast<int64_t>(x.E) * ((M + 127) / 128) * ((N + 127) / 128);
  if (mid < 256) return fn(SMALL());
  return fn(Tile<128, 128, 2, 2, 2>());
}

template <class TL, int KA, int KB, int EPI, bool GATED>
static hipError_t launch_tile_bf16(const ExpertArgs& x, ExpertGemmArgs a, hipStream_t st) {
  expert_set_tiles(a, x.E, TL::bm, EPI == kEpiAct && GATED ? TL::bn / 2 : TL::bn);
  const int resident = TL::per_cu * device_cu_count();
  constexpr bool kQuarters = TL::bm == 256 && EPI != kEpiActGrad;  // that one's column sums go by tile
  if (kQuarters && a.tiles <= kMaxRounds * resident) {
    // without counts that cut M the tiles are known here
    const int last = a.tiles % resident;
    if ((a.counts && !a.k_is_rows) || (last > 0 && 2 * last <= resident)) a.round = resident;
  }
  experts_gemm_bf16_kernel<TL::bm, TL::bn, TL::wm, TL::wn, KA, KB, EPI, GATED>
      <<<dim3(expert_blocks(a.tiles, resident)), dim3(TL::wm * TL::wn * kWave), 0, st>>>(a);
  if constexpr (kQuarters) {
    if (a.round) {
      using Q = Tile<TL::bm / 2, TL::bn / 2, 2, 2, 2>;
      a.quarters = 1;
      experts_gemm_bf16_kernel<Q::bm, Q::bn, Q::wm, Q::wn, KA, KB, EPI, GATED>
          <<<dim3(expert_blocks(2 * resident, Q::per_cu * device_cu_count())), dim3(Q::wm * Q::wn * kWave), 0, st>>>(a);
    }
  }
  return hipGetLastError();
}

}  // namespace hetumoe
