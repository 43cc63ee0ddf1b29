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

// Rounds of tiles up to which the last one is worth a launch of its own, which costs 4 to 5 us
// where it finds nothing to do (dxe of 16 x 1280 x 1024 x 4096 gated, 1024 rows in use: 407 us in
// whole tiles, 237 + 71 with the second round in quarters).  Few blocks have only their own
// loads to wait for: eight waves and four stages, one block per CU (these 32 quarter tiles of K =
// 8192 71 us, by four waves with two stages, two blocks per CU, 108; 320 of them 148 and 130).
constexpr int kMaxRounds = 16;

// Tiles of 256 x 256 once they fill the CUs (dw of 64 x 512 x 2048 x 8192: 1.12 ms, 128 x 128
// 1.47; 8 x 1024 x 1024 x 1024, where they do not: forward 52 us, 128 x 128 47) and an expert's slots
// are more than half of one's rows (the rows in use are known on the device alone: 154 of 313
// take 256 x 256 too; forward of 64 x 128 x 1024 x 4096 289 us, 128 x 128 264), of 128 x
// 128 once those fill the CUs, and else, or where an expert has few rows, of 64 x 64, whose four stages
// keep memory busy from few blocks (forward of 8 x 128 x 1024 x 4096 44 us, 128 x 128 61; of
// 32 x 128 x 1024 x 1024, where 128 x 128 fill the CUs, 45 and 35; dpre of 36 x 2 x 64, K =
// 2760: 21 us, two stages of 64 x 256 35).
template <class Fn>
static hipError_t by_tile(const ExpertArgs& x, int M, int N, Fn fn) {
  auto tiles = [&](int t) { return static_cast<int64_t>(x.E) * ((M + t - 1) / t) * ((N + t - 1) / t); };
  if (M > 128 && tiles(256) >= 256) return fn(Tile<256, 256, 2, 4, 1>());
  if (M > 64 && tiles(128) >= 256) return fn(Tile<128, 128, 2, 2, 2>());
  return fn(Tile<64, 64, 2, 1, 2>());
}

template <class TL, int KA, int KB, int EPI, bool GATED>
static hipError_t launch_tile_bf16(const ExpertArgs& x, ExpertGemmArgs a, hipStream_t st) {
  expert_set_tiles(a, x.E, TL::bm, expert_acts(EPI) && GATED ? TL::bn / 2 : TL::bn);
  const int resident = TL::per_cu * device_cu_count();
  constexpr bool kQuarters = TL::bm == 256 && !expert_act_grads(EPI);  // that one's column sums go by tile
  if (kQuarters && a.tiles <= kMaxRounds * resident) {
    // without counts that cut M the tiles are known here
    const int last = a.tiles % resident;
    if ((a.counts && !a.k_is_rows) || (last > 0 && 2 * last <= resident)) a.round = resident;
  }
  experts_gemm_bf16_kernel<TL::bm, TL::bn, TL::wm, TL::wn, KA, KB, EPI, GATED>
      <<<dim3(expert_blocks(a.tiles, resident)), dim3(TL::wm * TL::wn * kWave), 0, st>>>(a);
  if constexpr (kQuarters) {
    if (a.round) {
      using Q = Tile<TL::bm / 2, TL::bn / 2, 4, 2, 1>;
      a.quarters = 1;
      experts_gemm_bf16_kernel<Q::bm, Q::bn, Q::wm, Q::wn, KA, KB, EPI, GATED>
          <<<dim3(expert_blocks(2 * resident, Q::per_cu * device_cu_count())), dim3(Q::wm * Q::wn * kWave), 0, st>>>(a);
    }
  }
  return hipGetLastError();
}

}  // namespace hetumoe
