// Batched bf16 products of the expert networks on v_mfma_f32_16x16x32_bf16.
//
// A block forms BM x BN of one expert's product, WM x WN waves, 64 columns each.
// Per stage of 64 K elements both operands go straight from memory to LDS as
// they lie there (16 bytes per lane, no registers), two stages in turn (four for small tiles
// and where a block has a CU to itself).  Operands
// whose rows run along K are read as 16-byte fragments, the others through LDS
// transpose reads.  16-byte pieces are placed by an exclusive-or with bits of
// their row, so that the 16 lanes of a fragment read touch different banks; since
// a load to LDS fills it in lane order, the lane fetches the piece that belongs
// where it writes.
//
// While one half of a stage (32 K) is multiplied the fragments of the next half are
// read between them, so the reads' latency and the barrier lie behind products; the
// stage after next is requested as soon as every wave has read the last half of the
// stage in its place.  Where both operands are read through transposes, four stages of
// 32 K take turns instead: the loads run further ahead, which the short sums over an
// expert's rows need (dw of 64 x 512 x 2048 x 8192 1.31 -> 1.20 ms).  Towards the end of a
// tile the loads are the next tile's, behind the products and the stores of this one.
//
// The product is formed transposed (columns n are the rows of the matrix unit), so a lane
// holds 4 neighbouring columns of one row; a swap with the neighbouring 16 lanes over a
// pair of tiles makes that 8, one 16-byte store.
//
// Rows past the expert's count and pieces past K are zeros from outside the buffer
// resource; nothing behind the count is read.
//
// Large products: 64 experts of 2560 rows in use x 2048 x 2048, the gated first product 2.40
// ms and the second 1.14, 1.15 and 1.20 PFLOP/s, the matrix units busy 56 and 60 % of the time at
// 1.94 and 1.90 GHz.  The clock falls as the units get busier, so power takes part of what a
// better fed loop would gain (a library product of 8192^3: 70 % at 1.90 GHz, 1.36 PFLOP/s; of zeros
// 71 % at 2.42), but a seventh to a fifth is this loop's own: its reads, barriers and epilogues.  Rows
// 16 KB apart feed it worse (one expert of 8192^3: 1.02 ms, 44 % at 2.33 GHz).  Blocks of four
// waves with half of the LDS reads were slower (gated, uneven rows: 1.86 and 0.91 -> 1.95 and
// 0.95 ms).  The weight gradients are bound by what their transpose reads, loads and stores take
// (64 x 460 rows x 2048 x 8192: 1.12 ms, without the stores 0.80, without the loads 0.75; the units
// busy 32 % at 2.3 GHz).
#pragma once

#include "experts.hpp"

namespace hetumoe {

constexpr int kEBK = kExpertBk<bf16_t>;

// Fragments: of step ks (32 K elements) lane (g, m) gets K 8 g .. 8 g + 7 of row (or
// column) x0 + 16 i + m, i = 0 .. MT - 1, x0 a multiple of 16 MT.
template <int KIND, bool RIGHT, int W, int MT>
struct ExpertFrag {
  unsigned at;  // byte of (i = 0, ks = 0)
  __device__ __forceinline__ void init(int x0, int g, int m) {
    if constexpr (KIND == kRows) {
      at = (x0 + m) * 128 + ((g ^ expert_swz<bf16_t, KIND, RIGHT, W>(m)) * 16);
    } else {
      const int row = 8 * g + m / 4;
      at = row * W * 2 + (((x0 / 8 + m % 4 / 2) ^ expert_swz<bf16_t, KIND, RIGHT, W>(row)) * 16) + m % 2 * 8;
    }
  }
  // kRows: tiles are 16 rows apart, the steps' pieces differ in bit 2 of their place.
  // kCols: a tile is 32 bytes, bits that are free of carries; rows 4 and 32 on keep their order.
  __device__ __forceinline__ u32x4 read(const bf16_t* lds, unsigned from, int ks, int i) const {
    const char* p = reinterpret_cast<const char*>(lds);
    if constexpr (KIND == kRows) {
      return *reinterpret_cast<const u32x4*>(p + (from ^ (ks * 64)) + i * 2048);
    } else {
      const char* q = p + (from ^ (i * 32)) + ks * 64 * W;
      const uint2 lo = expert_tr16(reinterpret_cast<const bf16_t*>(q));
      const uint2 hi = expert_tr16(reinterpret_cast<const bf16_t*>(q + 8 * W));
      return u32x4{lo.x, lo.y, hi.x, hi.y};
    }
  }
};

template <int BM, int BN, int WM, int WN, int KA, int KB, int EPI, bool GATED>
__global__ __launch_bounds__(WM* WN * 64) void experts_gemm_bf16_kernel(ExpertGemmArgs a) {
  constexpr int WAVES = WM * WN;
  constexpr int MT = BM / WM / 16, NT = BN / WN / 16, NP = NT / 2;
  static_assert(NT == 4, "64 columns per wave");
  // columns of the output per block and wave: with GATED in the forward product half of
  // them are the gate's, half the other factor's, 32 and 32 of each wave's 64
  constexpr bool kSplit = EPI == kEpiAct && GATED;
  constexpr int BNO = kSplit ? BN / 2 : BN;
  constexpr bool kDeep = BM * BN <= 64 * 128 || WM == 4;        // four stages: few blocks
  constexpr bool kRing = !kDeep && KA == kCols && KB == kCols;  // four stages of half the length
  constexpr int BK = kRing ? kEBK / 2 : kEBK;
  constexpr int kTurn = kDeep ? 4 * kEBK : 2 * kEBK;  // K elements in which all stages had their turn
  __shared__ __align__(1024) bf16_t A0[BM * BK], A1[BM * BK], B0[BN * BK], B1[BN * BK];
  __shared__ __align__(1024) bf16_t A2[kDeep || kRing ? BM * BK : 8], A3[kDeep || kRing ? BM * BK : 8];
  __shared__ __align__(1024) bf16_t B2[kDeep || kRing ? BN * BK : 8], B3[kDeep || kRing ? BN * BK : 8];
  __shared__ int tile_before[kMaxExperts], tile_rows[kMaxExperts];
  __shared__ int4 tile_list[kTileList];

  const int lane = lane_id(), g = lane / 16, m = lane % 16;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int wm = wave / WN, wn = wave % WN;
  const int xcd = blockIdx.x % 8, step = gridDim.x / 8;
  int slot = blockIdx.x / 8;  // of the list's first tile
  ExpertTiles<BM> tiles;
  tiles.init(a, tile_before, tile_rows);
  if (a.quarters && tiles.end == 0) return;
  auto list_tiles = [&]() {
    for (int i = threadIdx.x; i < kTileList; i += WAVES * kWave) tile_list[i] = tiles.slot_tile(a, xcd, slot + i * step);
    __syncthreads();
  };
  list_tiles();

  ExpertOperand<bf16_t, KA, false, BM, WAVES, BK> oa;
  ExpertOperand<bf16_t, KB, true, BN, WAVES, BK> ob;
  int left = 0;  // K elements of the loads' tile from the next stage on
  // Points the loads at tile t (none: zeros).
  auto aim = [&](bool any, const ExpertTile& t) {
    const int n = any ? __builtin_amdgcn_readfirstlane(tile_rows[t.e]) : 0;
    const int m0 = t.bm * BM, n0 = t.bn * BNO;
    // a quarter tile may lie behind the rows in use: zeros are all it writes
    const int K = a.k_is_rows ? n : any && m0 < n ? a.K : 0;
    oa.init(reinterpret_cast<const bf16_t*>(a.A) + t.e * a.sA, a.lda, m0, a.k_is_rows ? BM : min(BM, n - m0), wave,
            [&](int piece) { return m0 + piece * 8 < a.M ? m0 + piece * 8 : -1; });
    ob.init(reinterpret_cast<const bf16_t*>(a.B) + t.e * a.sB, a.ldb, n0, min(BN, a.N - n0), wave, [&](int piece) {
      if constexpr (kSplit) {
        // pieces 0..3 of each wave's 8 are the gate's
        const int c = n0 + (piece / 8) * 32 + (piece % 4) * 8;
        return c < a.N ? c + (piece % 8 < 4 ? 0 : a.N) : -1;
      } else {
        return n0 + piece * 8 < a.N ? n0 + piece * 8 : -1;
      }
    });
    left = __builtin_amdgcn_readfirstlane(K);
  };
  ExpertFrag<KA, false, BM, MT> ra;
  ExpertFrag<KB, true, BN, NT> rb;
  ra.init(wm * MT * 16, g, m);
  rb.init(wn * NT * 16, g, m);
  constexpr int kLoads = ExpertOperand<bf16_t, KA, false, BM, WAVES, BK>::N + ExpertOperand<bf16_t, KB, true, BN, WAVES, BK>::N;
  // Stores that every tile's epilogue ends with at least, all issued whatever is masked.
  constexpr int kStores = EPI == kEpiStore ? MT * NP : EPI == kEpiAct ? MT * (kSplit ? 1 : NP) : MT * NP * (GATED ? 2 : 1);
  // and with pre written too
  constexpr int kStoresPre = EPI == kEpiAct ? kStores + MT * NP : kStores;
  f32x4 acc[MT][NT];
  u32x4 fa[MT], fb[NT], fn[NT];
  auto load = [&](bf16_t* As, bf16_t* Bs) __attribute__((always_inline)) {
    oa.load(As, wave, left);
    ob.load(Bs, wave, left);
    left -= BK;
  };
  // Stores of the tile before may still be on their way where the loads waited for were
  // issued ahead of them (the counter counts in order): `fresh`.
  bool fresh = false;
  auto barrier = [&](auto ahead) __attribute__((always_inline)) {
    constexpr int N = decltype(ahead)::v;  // loads that may be on their way
    if (!fresh) expert_stage_barrier<N>();
    else if (kStoresPre > kStores && a.pre) expert_stage_barrier<N + kStoresPre>();
    else expert_stage_barrier<N + kStores>();
  };
  // Products of 32 K, their fragments in fa and cur, in MT groups of NT; between them
  //   SYNC  behind the first groups, the barrier after which the next fragments' stage is in
  //         LDS and the place (As, Bs) free, and the loads of the stage that goes there;
  //   READ  the fragments of the next 32 K, step ks of (An, Bn), the left ones into the
  //         registers of those already used (a tile's last fragments make room for its epilogue).
  // All in their places so that products follow products: the barrier finds the reads
  // before it returned.  The products are written out to tie each sum to its registers
  // and to keep that order: left to the compiler, sums and fragments moved between
  // registers and scratch memory.  The empty slots cover a move into an operand right before.
  auto half = [&](auto read, auto sync, u32x4 (&cur)[NT], u32x4 (&next)[NT], bf16_t* As, bf16_t* Bs, const bf16_t* An,
                  const bf16_t* Bn, int ks) __attribute__((always_inline)) {
    constexpr bool READ = decltype(read)::v != 0, SYNC = decltype(sync)::v >= 0;
    constexpr int kFirst = SYNC ? (MT >= 8 ? 1 : 0) : 0;  // group behind which the rest begins
    constexpr int kParts = MT - kFirst > 1 ? MT - kFirst - 1 : 1;
    const unsigned at_a = expert_opaque(ra.at), at_b = expert_opaque(rb.at);
    typename decltype(oa)::Stage la;
    typename decltype(ob)::Stage lb;
#pragma unroll
    for (int i = 0; i < MT; ++i) {
#pragma unroll
      for (int j = 0; j < NT; ++j)
        asm volatile("s_nop 1\n\tv_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+v"(acc[i][j]) : "v"(cur[j]), "v"(fa[i]));
      if constexpr (SYNC) {
        if (i == kFirst) {
          barrier(sync);
          la = oa.next(left);
          lb = ob.next(left);
          left -= BK;
        }
      }
      if (i < kFirst) continue;
      const int part = i - kFirst;
      if constexpr (READ) {
#pragma unroll
        for (int j = 0; j < NT; ++j)
          if (j * kParts / NT == part) next[j] = rb.read(Bn, at_b, ks, j);
#pragma unroll
        for (int q = 0; q <= i; ++q)
          if (q == i || part == 0) fa[q] = ra.read(An, at_a, ks, q);
      }
      if constexpr (SYNC) {
#pragma unroll
        for (int q = 0; q < kLoads; ++q)
          if (q * kParts / kLoads == part) {
            if (q < decltype(oa)::N) la.issue(As, wave, q);
            else lb.issue(Bs, wave, q - decltype(oa)::N);
          }
      }
    }
  };
  // The stage in (As, Bs), its first half in fa and fb; the next one in (An, Bn).
  auto stage = [&](auto read_last, bf16_t* As, bf16_t* Bs, const bf16_t* An, const bf16_t* Bn) __attribute__((always_inline)) {
    half(ExpertInt<1>(), ExpertInt<-1>(), fb, fn, nullptr, nullptr, As, Bs, 1);
    half(read_last, ExpertInt<kDeep ? 2 * kLoads : 0>(), fn, fb, As, Bs, An, Bn, 0);
    if (!kDeep) fresh = false;
  };
  // One of four stages, in fa and cur.
  auto quarter = [&](auto read, u32x4 (&cur)[NT], u32x4 (&next)[NT], bf16_t* As, bf16_t* Bs, const bf16_t* An,
                     const bf16_t* Bn) __attribute__((always_inline)) {
    half(read, ExpertInt<2 * kLoads>(), cur, next, As, Bs, An, Bn, 0);
  };
  // All stages' turn.
  auto turn = [&](auto read_last) __attribute__((always_inline)) {
    if constexpr (kRing) {
      quarter(ExpertInt<1>(), fb, fn, A0, B0, A1, B1);
      quarter(ExpertInt<1>(), fn, fb, A1, B1, A2, B2);
      quarter(ExpertInt<1>(), fb, fn, A2, B2, A3, B3);
      fresh = false;
      quarter(read_last, fn, fb, A3, B3, A0, B0);
    } else if constexpr (kDeep) {
      stage(ExpertInt<1>(), A0, B0, A1, B1);
      stage(ExpertInt<1>(), A1, B1, A2, B2);
      stage(ExpertInt<1>(), A2, B2, A3, B3);
      fresh = false;
      stage(read_last, A3, B3, A0, B0);
    } else {
      stage(ExpertInt<1>(), A0, B0, A1, B1);
      stage(read_last, A1, B1, A0, B0);
    }
  };

  ExpertTile at{0, 0, 0}, next{0, 0, 0};
  int index = 0;  // in the list
  bool work = expert_listed(tile_list, 0, at);
  if (work) {
    aim(true, at);
    load(A0, B0);
    load(A1, B1);
    if constexpr (kDeep || kRing) {
      load(A2, B2);
      load(A3, B3);
      expert_stage_barrier<3 * kLoads>();
    } else {
      expert_stage_barrier<kLoads>();
    }
  }
  // the tiles without work that this block clears
  int idle = blockIdx.x;
  if (!work && !tiles.clear(a, idle, at)) return;
  for (;;) {
  bool more = false;
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  if (work) {
    // the first stages of the next tile are on their way before this one's results are
    // stored; behind the last tile: zeros, so that the count of loads stays the same
    const int n = __builtin_amdgcn_readfirstlane(tile_rows[at.e]);
    const int K = a.k_is_rows ? n : at.bm * BM < n ? a.K : 0;
    if (++index == kTileList) {
      __syncthreads();
      slot += kTileList * step;
      index = 0;
      list_tiles();
    }
    more = expert_listed(tile_list, index, next);
    const unsigned at_a = expert_opaque(ra.at), at_b = expert_opaque(rb.at);
#pragma unroll
    for (int j = 0; j < NT; ++j) fb[j] = rb.read(B0, at_b, 0, j);
#pragma unroll
    for (int i = 0; i < MT; ++i) fa[i] = ra.read(A0, at_a, 0, i);
    for (int k = kTurn; k < K; k += kTurn) turn(ExpertInt<1>());
    aim(more, next);
    turn(ExpertInt<0>());
    // the last sums leave the matrix unit before they are read
    asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
  }
  const int e = at.e, bm = at.bm;
  const int m0 = bm * BM, n0 = at.bn * BNO;
  const int rows = a.k_is_rows ? a.M : work ? __builtin_amdgcn_readfirstlane(tile_rows[e]) : 0;

  // lane (g, m): row m of tile i, columns 4 g .. 4 g + 3 of each tile.  Odd groups of 16
  // lanes swap their first tile of a pair for the second one of the group before:
  // 8 neighbouring columns each, from 16 (g % 2) + 8 (g / 2).
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(acc[i][2 * p][q]),
                                                        __float_as_uint(acc[i][2 * p + 1][q]), false, false);
        acc[i][2 * p][q] = __uint_as_float(r[0]);
        acc[i][2 * p + 1][q] = __uint_as_float(r[1]);
      }
  const int ln = expert_opaque(lane), lm = ln % 16, lg = ln / 16;
  const int lrow = wm * MT * 16 + lm;  // of the tile; 16 i on
  const int col0 = n0 + (kSplit ? wn * 32 : wn * 64) + 16 * (lg % 2) + 8 * (lg / 2);
  auto value = [&](int i, int p, int q) { return acc[i][2 * p + q / 4][q % 4]; };
  // byte of (lrow, column c) in rows of ld, or past everything
  auto place = [&](int ld, int c, bool in) { return static_cast<unsigned>(in ? (lrow * ld + c) * 2 : kExpertOob); };
  auto put = [&](__amdgpu_buffer_rsrc_t r, unsigned off, const float (&v)[8]) {
    __builtin_amdgcn_raw_buffer_store_b128(Chunk<bf16_t>::pack(v), r, static_cast<int>(off), 0, 0);
  };
  const int valid = min(BM, a.M - m0);  // rows of the output
  if constexpr (EPI == kEpiStore) {
    const __amdgpu_buffer_rsrc_t out =
        expert_rows<bf16_t>(reinterpret_cast<const bf16_t*>(a.out) + e * a.sO, m0, a.ldo, valid);
    float bias[NP][8];
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
      for (int q = 0; q < 8; ++q)
        bias[p][q] = a.bias && col0 + 32 * p < a.N ? a.bias[static_cast<int64_t>(e) * a.N + col0 + 32 * p + q] : 0.f;
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const bool used = m0 + lrow + 16 * i < rows;
#pragma unroll
      for (int p = 0; p < NP; ++p) {
        float v[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] = used ? value(i, p, q) + bias[p][q] : 0.f;
        put(out, place(a.ldo, col0 + 32 * p, col0 + 32 * p < a.N) + i * 32 * a.ldo, v);
      }
    }
  } else if constexpr (EPI == kEpiAct) {
    const int N1 = GATED ? 2 * a.N : a.N;
    constexpr int NPO = kSplit ? 1 : NP;
    const __amdgpu_buffer_rsrc_t hid =
        expert_rows<bf16_t>(reinterpret_cast<const bf16_t*>(a.out) + e * a.sO, m0, a.ldo, valid);
    const __amdgpu_buffer_rsrc_t pre =
        expert_rows<bf16_t>(a.pre, static_cast<int64_t>(e) * a.C + m0, N1, a.pre ? valid : 0);
    float bias[NP][8];
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      const int c = kSplit ? col0 : col0 + 32 * p;
#pragma unroll
      for (int q = 0; q < 8; ++q)
        bias[p][q] = a.bias && c < a.N ? a.bias[static_cast<int64_t>(e) * N1 + c + q + (kSplit && p ? a.N : 0)] : 0.f;
    }
    expert_by_act(a.act, [&](auto which) {
      constexpr int ACT = decltype(which)::v;
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        const bool used = m0 + lrow + 16 * i < rows;
#pragma unroll
        for (int p = 0; p < NPO; ++p) {
          const int c = col0 + 32 * p;
          float v[8], u[8], f[8];
#pragma unroll
          for (int q = 0; q < 8; ++q) {
            v[q] = used ? value(i, p, q) + bias[p][q] : 0.f;
            f[q] = expert_act<ACT>(v[q]);
            if constexpr (kSplit) {
              u[q] = used ? value(i, 1, q) + bias[1][q] : 0.f;
              f[q] *= u[q];
            }
          }
          if (a.pre) {
            const unsigned at_pre = place(N1, c, c < a.N) + i * 32 * N1;
            put(pre, at_pre, v);
            if constexpr (kSplit) put(pre, at_pre + 2 * a.N, u);
          }
          put(hid, place(a.ldo, c, c < a.N) + i * 32 * a.ldo, f);
        }
      }
    });
  } else {
    // dpre, and its sums over the wave's rows before the rounding: [E, tm * WM, N1]
    const int N1 = GATED ? 2 * a.N : a.N;
    float* part = a.colsum ? a.colsum + (static_cast<int64_t>(e) * a.tm * WM + bm * WM + wm) * N1 : nullptr;
    const __amdgpu_buffer_rsrc_t out = expert_rows<bf16_t>(a.out, static_cast<int64_t>(e) * a.C + m0, N1, valid);
    // rows behind the count read as zeros; their products are chosen away below: zero rows
    // times an infinite weight are NaN, which would reach the sums
    const __amdgpu_buffer_rsrc_t pre =
        expert_rows<bf16_t>(a.pre, static_cast<int64_t>(e) * a.C + m0, N1, min(BM, rows - m0));
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      const int c = col0 + 32 * p;
      const unsigned off0 = place(N1, c, c < a.N);
      constexpr int kRowsAhead = GATED && MT > 1 ? MT / 2 : MT;  // rows requested together
      float s0[8], s1[8];
#pragma unroll
      for (int q = 0; q < 8; ++q) s0[q] = s1[q] = 0.f;
#pragma unroll
      for (int i0 = 0; i0 < MT; i0 += kRowsAhead) {
        u32x4 pv[kRowsAhead], pu[kRowsAhead];
#pragma unroll
        for (int i = 0; i < kRowsAhead; ++i) {
          const int off = static_cast<int>(off0 + (i0 + i) * 32 * N1);
          pv[i] = __builtin_amdgcn_raw_buffer_load_b128(pre, off, 0, 0);
          if constexpr (GATED) pu[i] = __builtin_amdgcn_raw_buffer_load_b128(pre, static_cast<int>(off + 2u * a.N), 0, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < kRowsAhead; ++i) {
          const bool used = m0 + lrow + 16 * (i0 + i) < rows;
          float v[8], u[8];
          Chunk<bf16_t>::unpack(pv[i], v);
          if constexpr (GATED) Chunk<bf16_t>::unpack(pu[i], u);
          // chosen per row: branches around all rows would hold all their loads at once
          expert_by_act(a.act, [&](auto which) {
            constexpr int ACT = decltype(which)::v;
#pragma unroll
            for (int q = 0; q < 8; ++q) {
              float f, df;
              expert_act_grad<ACT>(v[q], f, df);
              const float dh = used ? value(i0 + i, p, q) : 0.f;
              v[q] = GATED ? dh * u[q] * df : dh * df;
              if constexpr (GATED) u[q] = dh * f;
            }
          });
#pragma unroll
          for (int q = 0; q < 8; ++q) {
            s0[q] += v[q];
            if constexpr (GATED) s1[q] += u[q];
          }
          put(out, off0 + (i0 + i) * 32 * N1, v);
          if constexpr (GATED) put(out, off0 + (i0 + i) * 32 * N1 + 2 * a.N, u);
        }
      }
      if (part) {
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          s0[q] = group_reduce<16>(s0[q], OpAdd());
          if constexpr (GATED) s1[q] = group_reduce<16>(s1[q], OpAdd());
        }
        if (lm == 0 && c < a.N) {
#pragma unroll
          for (int q = 0; q < 8; ++q) {
            part[c + q] = s0[q];
            if constexpr (GATED) part[a.N + c + q] = s1[q];
          }
        }
      }
    }
  }
  if (more) {
    at = next;
    fresh = true;
    continue;
  }
  if (work) expert_stage_barrier();  // nothing is on its way to LDS when the block ends
  else idle += gridDim.x;
  work = false;
  if (!tiles.clear(a, idle, at)) return;
  }
}

}  // namespace hetumoe
