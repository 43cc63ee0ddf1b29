// Batched fp32 products of the expert networks on v_mfma_f32_16x16x4_f32: the
// scheme of experts_bf16.hpp with 32 K elements per stage.
//
// The order of K inside a product is free, so lane group g of a step of 16 takes
// K 4 g .. 4 g + 3, one 16-byte read where rows run along K, and its i-th product
// K 4 g + i; an operand whose rows run the other way is read NT (2 or 4) columns at a
// time.  Which of its 16 NT columns a row of the matrix unit takes is free too: they are
// chosen so that lane group g ends with columns 16 r + 4 g + 0..3, r = 0 .. NT - 1, and each
// store covers 64 bytes of a row (8 x 128 x 1024, K = 256 17.1 -> 15.4 us, its dw 10.6 -> 9.5).
// Each 256 K are summed on their own and then added to the running sum.
//
// Small products leave most CUs idle, and a wave's sums over K are what they take: there
// KG groups of waves take every KG-th stage each, and their sums are added pairwise.
//
// Large products are bound by the matrix units: 8 x 2048 x 2048 x 2048 1.00 to 1.09 ms per
// product (126 to 137 TFLOP/s), the units busy 82 to 87 % of the time.
#pragma once

#include "experts.hpp"

namespace hetumoe {

constexpr int kFBK = kExpertBk<float>;
constexpr int kFSum = 8;  // stages summed on their own (a multiple of 2)

// Left operand, step ks of 16: lane (g, m) gets K 4 g + 0..3 of row (column) x0 + m.  `off`:
// of the group's part of the array.  (The array itself is passed, and added to once: only
// so does the compiler see that loads on their way to the other stage's arrays are none of
// this read's business, and does not wait for them.)
template <int KIND, int W>
__device__ __forceinline__ f32x4 expert_left_f32(const float* lds, int off, int x0, int ks, int g, int m) {
  if constexpr (KIND == kRows) {
    const int row = x0 + m;
    const int piece = (4 * ks + g) ^ expert_swz<float, KIND, false, W>(row);
    return *reinterpret_cast<const f32x4*>(lds + (off + row * kFBK + piece * 4));
  } else {
    const float* p = lds + (off + (16 * ks + 4 * g) * W + x0 + m);
    return f32x4{p[0], p[W], p[2 * W], p[3 * W]};
  }
}

// The first of the NT columns that row m of the matrix unit takes.
template <int NT>
__device__ __forceinline__ int expert_column_f32(int m) {
  if constexpr (NT == 4) return m % 4 * 16 + m / 4 * 4;
  else return m % 4 / 2 * 16 + m / 4 * 4 + m % 2 * 2;
}

// Right operand: fb[j][i] is K 4 g + i of row (column) x0 + expert_column_f32(m) + j.
template <int KIND, int W, int NT>
__device__ __forceinline__ void expert_right_f32(const float* lds, int off, int x0, int ks, int g, int m, f32x4 (&fb)[NT]) {
  typedef float fv __attribute__((ext_vector_type(NT)));
  if constexpr (KIND == kRows) {
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const int row = x0 + expert_column_f32<NT>(m) + j;
      const int piece = (4 * ks + g) ^ expert_swz<float, KIND, true, W>(row);
      fb[j] = *reinterpret_cast<const f32x4*>(lds + (off + row * kFBK + piece * 4));
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const fv v = *reinterpret_cast<const fv*>(lds + (off + (16 * ks + 4 * g + i) * W + x0 + expert_column_f32<NT>(m)));
#pragma unroll
      for (int j = 0; j < NT; ++j) fb[j][i] = v[j];
    }
  }
}

template <int BM, int BN, int WM, int WN, int KG, int KA, int KB, int EPI, bool GATED>
__global__ __launch_bounds__(WM* WN* KG * 64, BM == 128 ? 2 : 4) void experts_gemm_f32_kernel(ExpertGemmArgs a) {
  constexpr int WAVES = WM * WN;
  constexpr int MT = BM / WM / 16, NT = BN / WN / 16;
  static_assert(NT == 4 || NT == 2, "64 or 32 columns per wave");
  constexpr bool kSplit = EPI == kEpiAct && GATED;  // half of a wave's columns are the gate's
  constexpr int BNO = kSplit ? BN / 2 : BN;
  __shared__ __align__(1024) float A0[KG * BM * kFBK], B0[KG * BN * kFBK], A1[KG * BM * kFBK], B1[KG * BN * kFBK];
  __shared__ int tile_before[kMaxExperts], tile_rows[kMaxExperts];

  const int lane = lane_id(), g = lane / 16, m = lane % 16;
  const int kg = KG > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / (WAVES * kWave)) : 0;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave) - kg * WAVES;
  const int wm = wave / WN, wn = wave % WN;
  const int xcd = blockIdx.x % 8, step = gridDim.x / 8;
  int slot = blockIdx.x / 8, idle = blockIdx.x;
  ExpertTiles<BM> tiles;
  tiles.init(a, tile_before, tile_rows);
  for (;;) {
  // the tiles with work, then those that are only cleared
  ExpertTile at{0, 0, 0};
  const int4 found = tiles.slot_tile(a, xcd, slot);
  const bool work = __builtin_amdgcn_readfirstlane(found.x) >= 0;
  if (work) {
    at = {__builtin_amdgcn_readfirstlane(found.x), __builtin_amdgcn_readfirstlane(found.y),
          __builtin_amdgcn_readfirstlane(found.z)};
    slot += step;
  } else {
    if (!tiles.clear(a, idle, at)) return;
    idle += gridDim.x;
  }
  const int e = at.e, bm = at.bm, bn = at.bn;
  const int cnt = __builtin_amdgcn_readfirstlane(tile_rows[e]);
  const int K = a.k_is_rows ? cnt : a.K;
  const int rows = a.k_is_rows ? a.M : cnt;
  const int m0 = bm * BM, n0 = bn * BNO;
  const int mvalid = max(0, min(BM, rows - m0));

  f32x4 acc[MT][NT], sum[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = sum[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

  if (mvalid > 0 && K > 0) {
    ExpertOperand<float, KA, false, BM, WAVES> oa;
    ExpertOperand<float, KB, true, BN, WAVES> ob;
    oa.init(reinterpret_cast<const float*>(a.A) + e * a.sA, a.lda, m0, mvalid, wave,
            [&](int piece) { return m0 + piece * 4 < a.M ? m0 + piece * 4 : -1; });
    ob.init(reinterpret_cast<const float*>(a.B) + e * a.sB, a.ldb, n0, min(BN, a.N - n0), wave, [&](int piece) {
      if constexpr (kSplit) {
        // the first half of a wave's 4 NT pieces is the gate's
        const int c = n0 + piece / (4 * NT) * 8 * NT + piece % (2 * NT) * 4;
        return c < a.N ? c + (piece % (4 * NT) >= 2 * NT ? a.N : 0) : -1;
      } else {
        return n0 + piece * 4 < a.N ? n0 + piece * 4 : -1;
      }
    });
    auto multiply = [&](const float* As, const float* Bs) __attribute__((always_inline)) {
#pragma unroll
      for (int ks = 0; ks < kFBK / 16; ++ks) {
        f32x4 fb[NT], fa[MT];
        expert_right_f32<KB, BN, NT>(Bs, kg * BN * kFBK, wn * 16 * NT, ks, g, m, fb);
#pragma unroll
        for (int i = 0; i < MT; ++i) fa[i] = expert_left_f32<KA, BM>(As, kg * BM * kFBK, (wm * MT + i) * 16, ks, g, m);
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
          for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j)
              acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(fb[j][q], fa[i][q], acc[i][j], 0, 0, 0);
      }
    };
    auto flush = [&]() {
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          sum[i][j] += acc[i][j];
          acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    };
    expert_stage_barrier();  // the tile before is read
    oa.skip(kg);
    ob.skip(kg);
    const int stages = (K + KG * kFBK - 1) / (KG * kFBK);  // per group
    int left = K - kg * kFBK;
    auto load = [&](float* As, float* Bs) __attribute__((always_inline)) {
      oa.load(As, kg * oa.N * WAVES + wave, left);
      ob.load(Bs, kg * ob.N * WAVES + wave, left);
      oa.skip(KG - 1);
      ob.skip(KG - 1);
      left -= KG * kFBK;
      __builtin_amdgcn_sched_barrier(0);  // ahead of the products, not just before the next barrier
    };
    load(A0, B0);
    int s = 0;
    for (; s + 1 < stages; s += 2) {
      expert_stage_barrier();
      load(A1, B1);
      multiply(A0, B0);
      expert_stage_barrier();
      if (s + 2 < stages) load(A0, B0);
      multiply(A1, B1);
      if ((s + 2) % kFSum == 0) flush();
    }
    if (s < stages) {
      expert_stage_barrier();
      multiply(A0, B0);
    }
    flush();
    if constexpr (KG > 1) {
      // the upper half of the groups hands its sums to the lower one, until one is left
      float* part = A0;
      static_assert(KG / 2 * WAVES * kWave * MT * NT * 4 <= KG * BM * kFBK, "room for half of the sums");
      const int at = wave * kWave + lane;
      auto place = [&](int q, int i, int j) {
        return reinterpret_cast<f32x4*>(part + ((q * MT * NT + i * NT + j) * WAVES * kWave + at) * 4);
      };
#pragma unroll
      for (int h = KG / 2; h >= 1; h /= 2) {
        expert_stage_barrier();
        if (kg >= h && kg < 2 * h) {
#pragma unroll
          for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j) *place(kg - h, i, j) = sum[i][j];
        }
        expert_stage_barrier();
        if (kg < h) {
#pragma unroll
          for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j) sum[i][j] += *place(kg, i, j);
        }
      }
    }
  }

  if (kg > 0) continue;
  // lane (g, m): row m of tile i, columns 16 r + 4 g + 0..3, r = 0 .. NT - 1
  const int row0 = m0 + wm * MT * 16 + m;
  const int col0 = n0 + (kSplit ? 8 * NT : 16 * NT) * wn + 4 * g;
  auto value = [&](int i, int r, int q) { return sum[i][(4 * r + q) % NT][(4 * r + q) / NT]; };
  auto put = [](float* p, const float (&v)[4]) { *reinterpret_cast<f32x4*>(p) = f32x4{v[0], v[1], v[2], v[3]}; };
  if constexpr (EPI == kEpiStore) {
#pragma unroll
    for (int r = 0; r < NT; ++r) {
      const int c = col0 + 16 * r;
      if (c >= a.N) continue;
      float bias[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) bias[q] = a.bias ? a.bias[static_cast<int64_t>(e) * a.N + c + q] : 0.f;
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        const int row = row0 + 16 * i;
        if (row >= a.M) continue;
        float v[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = row < rows ? value(i, r, q) + bias[q] : 0.f;
        put(reinterpret_cast<float*>(a.out) + e * a.sO + static_cast<int64_t>(row) * a.ldo + c, v);
      }
    }
  } else if constexpr (EPI == kEpiAct) {
    const int N1 = GATED ? 2 * a.N : a.N;
    constexpr int R = kSplit ? NT / 2 : NT;
    expert_by_act(a.act, [&](auto which) {
      constexpr int ACT = decltype(which)::v;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const int c = col0 + 16 * r;
        if (c >= a.N) continue;
        float b0[4], b1[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          b0[q] = a.bias ? a.bias[static_cast<int64_t>(e) * N1 + c + q] : 0.f;
          b1[q] = kSplit && a.bias ? a.bias[static_cast<int64_t>(e) * N1 + a.N + c + q] : 0.f;
        }
#pragma unroll
        for (int i = 0; i < MT; ++i) {
          const int row = row0 + 16 * i;
          if (row >= a.M) continue;
          float v[4], u[4], f[4];
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            v[q] = row < rows ? value(i, r, q) + b0[q] : 0.f;
            f[q] = expert_act<ACT>(v[q]);
            if constexpr (kSplit) {
              u[q] = row < rows ? value(i, r + NT / 2, q) + b1[q] : 0.f;
              f[q] *= u[q];
            }
          }
          if (a.pre) {
            float* pre = reinterpret_cast<float*>(a.pre) + (static_cast<int64_t>(e) * a.C + row) * N1 + c;
            put(pre, v);
            if constexpr (kSplit) put(pre + a.N, u);
          }
          put(reinterpret_cast<float*>(a.out) + e * a.sO + static_cast<int64_t>(row) * a.ldo + c, f);
        }
      }
    });
  } else {
    const int N1 = GATED ? 2 * a.N : a.N;
    float* part = a.colsum ? a.colsum + (static_cast<int64_t>(e) * a.tm * WM + bm * WM + wm) * N1 : nullptr;
    expert_by_act(a.act, [&](auto which) {
      constexpr int ACT = decltype(which)::v;
#pragma unroll
      for (int r = 0; r < NT; ++r) {
        const int c = col0 + 16 * r;
        float s0[4] = {0.f, 0.f, 0.f, 0.f}, s1[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < MT; ++i) {
          const int row = row0 + 16 * i;
          if (row >= a.M || c >= a.N) continue;
          const int64_t at = (static_cast<int64_t>(e) * a.C + row) * N1 + c;
          float v[4] = {0.f, 0.f, 0.f, 0.f}, u[4] = {0.f, 0.f, 0.f, 0.f};
          if (row < rows) {
            const float* src = reinterpret_cast<const float*>(a.pre) + at;
            Chunk<float>::unpack(*reinterpret_cast<const u32x4*>(src), v);
            if constexpr (GATED) Chunk<float>::unpack(*reinterpret_cast<const u32x4*>(src + a.N), u);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              float f, df;
              expert_act_grad<ACT>(v[q], f, df);
              const float dh = value(i, r, q);
              v[q] = GATED ? dh * u[q] * df : dh * df;
              u[q] = dh * f;
              s0[q] += v[q];
              if constexpr (GATED) s1[q] += u[q];
            }
          }
          put(reinterpret_cast<float*>(a.out) + at, v);
          if constexpr (GATED) put(reinterpret_cast<float*>(a.out) + at + a.N, u);
        }
        if (part) {
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            s0[q] = group_reduce<16>(s0[q], OpAdd());
            if constexpr (GATED) s1[q] = group_reduce<16>(s1[q], OpAdd());
          }
          if (m == 0 && c < a.N) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              part[c + q] = s0[q];
              if constexpr (GATED) part[a.N + c + q] = s1[q];
            }
          }
        }
      }
    });
  }
  }
}

}  // namespace hetumoe
