// The expert networks in 8-bit integers: rows and hidden rows are quantized by launches of their own
// (a row's scale is known when all of it is), the products are the bf16 ones' loop on
// v_mfma_i32_16x16x64_i8.  A fragment's 16 bytes are 16 integers for 8 bf16, in the same places along K
// in both operands, so tiles, LDS and loads are those of bf16 rows half as long; both
// operands' rows run along K.
//
// The loop takes the time of as many bytes in bf16 (tiles of 256 x 256, per 1024 bytes of K: 13.3 us for 7
// that the matrix units need, bf16 12.3): what it moves through LDS, which for these tiles is as
// long as the products and for 128 x 128 half as long again.  A tile's ends, 8 to 13 us (scales, conversions, 128 KB
// of stores, which the next tile's loads wait behind), weigh twice as much.  64 x 2560 x 2048 x 2048,
// gated, 1666 rows in use on average: 1.9 and 1.7 POP/s; a library product of 8192^3 2.09.
#include "experts_tiles_bf16.hpp"

namespace hetumoe {

namespace {

// Tiles of 256 x 256 where the slots fill them (rows in use vary below them) and there are two
// rounds of them; the others as for bf16.  (us of the whole call, 256 and 128: 64 x 2560 x 2048 x 2048
// gated 1775 and 2105, 16 x 1280 x 1024 x 4096 243 and 262, 64 x 256 x 2048 x 2048 gated 298 and 327; 60 x 313
// x 1408 x 1008 gated 180 and 160, 32 x 640 x 1024 x 2048 gated 229 and 219, 8 x 2048 x 1024 x 1024, one round, 97
// and 89.  128 x 256: slower everywhere, 64 x 64 where 128 x 128 fill the CUs: 32 x 128 x 1024 x 1024 50 and 40.)
template <class Fn>
hipError_t by_tile_int8(const ExpertArgs& x, int M, int N, Fn fn) {
  auto tiles = [&](int t) { return static_cast<int64_t>(x.E) * ((M + t - 1) / t) * ((N + t - 1) / t); };
  const int rows256 = (M + 255) / 256 * 256;
  if (10 * rows256 <= 11 * M && tiles(256) >= 512) return fn(Tile<256, 256, 2, 4, 1>());
  if (M > 64 && tiles(128) >= 256) return fn(Tile<128, 128, 2, 2, 2>());
  return fn(Tile<64, 64, 2, 1, 2>());
}

template <int EPI>
hipError_t product(const ExpertArgs& x, const ExpertGemmArgs& a, hipStream_t st) {
  constexpr bool kAct = expert_acts(EPI);
  return by_tile_int8(x, a.M, kAct && x.gated ? 2 * a.N : a.N, [&](auto tile) {
    using TL = decltype(tile);
    if constexpr (kAct) {
      if (x.gated) return launch_tile_bf16<TL, kRows, kRows, EPI, true>(x, a, st);
    }
    return launch_tile_bf16<TL, kRows, kRows, EPI, false>(x, a, st);
  });
}

}  // namespace

hipError_t launch_experts_int8(const ExpertInt8Args& x, hipStream_t st) {
  ExpertArgs shape{};
  shape.E = x.E; shape.C = x.C; shape.d = x.d; shape.h = x.h; shape.act = x.act; shape.gated = x.gated;
  shape.dtype = x.dtype; shape.counts = x.counts;
  const int h1 = x.gated ? 2 * x.h : x.h;
  const int64_t rows = static_cast<int64_t>(x.E) * x.C;
  QuantArgs q{};
  q.rows = rows; q.n = x.d; q.C = x.C; q.dtype = x.dtype; q.counts = x.counts;
  q.x = x.xe; q.q = x.q; q.scale = x.scale;
  hipError_t err = launch_quantize(q, st);
  if (err != hipSuccess) return err;
  // K, and elements from one row to the next, in units of two integers
  ExpertGemmArgs a = expert_base_args(shape);
  a.M = x.C; a.N = x.h; a.K = x.d / 2;
  a.A = x.q; a.lda = x.d / 2; a.sA = static_cast<int64_t>(x.C) * (x.d / 2);
  a.B = x.q1; a.ldb = x.d / 2; a.sB = static_cast<int64_t>(h1) * (x.d / 2);
  a.sa = x.scale; a.sb = x.s1; a.bias = x.b1;
  a.out = x.hidden; a.ldo = x.h; a.sO = static_cast<int64_t>(x.C) * x.h;
  err = x.dtype == 1 ? product<kEpiInt8Act>(shape, a, st) : product<kEpiInt8ActF32>(shape, a, st);
  if (err != hipSuccess) return err;
  // ye's rows behind the counts are cleared here, where their waves have nothing to quantize (as tiles behind
  // all others in the product: 64 x 2560 x 2048 x 2048 gated 1670 -> 1651 us, 60 x 313 x 1408 x 1008 139 -> 134)
  q.n = x.h; q.x = x.hidden;
  q.clear = x.ye; q.clear_bytes = x.d * (x.dtype == 1 ? 2 : 4);
  if ((err = launch_quantize(q, st)) != hipSuccess) return err;
  a = expert_base_args(shape);
  a.M = x.C; a.N = x.d; a.K = x.h / 2;
  a.A = x.q; a.lda = x.h / 2; a.sA = static_cast<int64_t>(x.C) * (x.h / 2);
  a.B = x.q2; a.ldb = x.h / 2; a.sB = static_cast<int64_t>(x.d) * (x.h / 2);
  a.sa = x.scale; a.sb = x.s2; a.bias = x.b2;
  a.out = x.ye; a.ldo = x.d; a.sO = static_cast<int64_t>(x.C) * x.d;
  return x.dtype == 1 ? product<kEpiInt8>(shape, a, st) : product<kEpiInt8F32>(shape, a, st);
}

}  // namespace hetumoe
