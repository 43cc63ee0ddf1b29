// The whole layer for a few tokens: expert networks on the rows that chose them,
// without slots or dispatch, and the weighted sum of the choices.
//
// With few rows per expert the weights are what there is to read, so a block streams
// a strip of one expert's matrix past all rows that chose it: its waves take
// steps of 32 rows of the matrix in turn (each lane one piece of 8 of them, whole
// 256- or 128-byte stretches per row), turn them into matrix-core operands in
// registers, and add their sums in LDS at the end.  The second matrix's K is also
// split over blocks where that is needed to occupy the chip; the last kernel adds
// those parts in order.  No atomics: results repeat bit for bit.  Bound by the weights' bytes:
// 64 experts of 2048 x 2048, gated, 32 tokens of two choices: 115 and 59 us, 5.8 TB/s; one
// token, two experts of 2048 x 8192: 15 us each, 4.5 TB/s, with other experts each pass, whose
// weights no cache holds (14 to 15 with the same ones, 134 MB that the Infinity Cache may hold).
#include <algorithm>

#include "experts.hpp"
#include "select.hpp"

namespace hetumoe {

namespace {

constexpr int kStep = 32;  // K per wave step

template <int CB> struct Piece;
template <> struct Piece<16> { typedef u32x4 T; };
template <> struct Piece<8> { typedef unsigned T __attribute__((ext_vector_type(2))); };

// Non-temporal: a step's weights are read once (64 experts of 2048 x 2048, gated, 32 tokens:
// first product 139 -> 126 us, second 65 -> 59).
template <int CB>
__device__ __forceinline__ typename Piece<CB>::T load_piece(__amdgpu_buffer_rsrc_t r, int off) {
  if constexpr (CB == 16) return __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, 2);
  else return __builtin_amdgcn_raw_buffer_load_b64(r, off, 0, 2);
}

// in[i]: row i of 8, NC bf16 columns; out[j]: the 8 rows of column j.
__device__ __forceinline__ void columns_of(const u32x4 (&in)[8], u32x4 (&out)[8]) { transpose8x8_b16(in, out); }
__device__ __forceinline__ void columns_of(const Piece<8>::T (&in)[8], u32x4 (&out)[4]) {
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const uint32_t a = in[2 * q][j / 2], b = in[2 * q + 1][j / 2];
      out[j][q] = (j & 1) ? ((a >> 16) | (b & 0xffff0000u)) : ((a & 0xffffu) | (b << 16));
    }
}

// Sums of MT tiles of 16 rows of A times a strip of 16 NC columns of a matrix with K rows:
// lane (g, m) holds rows 4 g + r of each tile, columns NC m + j.  A wave takes steps of
// kStep rows of the matrix, from `step` on, `stride` apart.  TERMS 2: A is the sum of two
// matrices, `plane` bytes apart.
template <class T, int CB, int MT, int TERMS>
struct StripSums {
  static constexpr int ELT = static_cast<int>(sizeof(T));
  static constexpr int NC = CB / ELT;
  static constexpr int AP = 8 * ELT / 16;  // 16-byte pieces of A per row and lane
  typedef typename Piece<CB>::T piece_t;
  struct Regs {
    piece_t w[8];
    u32x4 x[MT][TERMS * AP];
  };
  f32x4 acc[MT][NC];

  // wcol: byte of the lane's columns in a row of `pitch` bytes, or kExpertOob; arow: byte of
  // the lane's row of A per tile, or -1.
  __device__ __forceinline__ void run(__amdgpu_buffer_rsrc_t w, unsigned wcol, int pitch, __amdgpu_buffer_rsrc_t x,
                                      const int (&arow)[MT], int plane, int K, int step, int stride) {
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NC; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int steps = (K + kStep - 1) / kStep;
    const int g = lane_id() / 16;
    // rows past K lie past the matrix's resource: zeros
    auto load = [&](Regs& r, int st) __attribute__((always_inline)) {
      const int k = st * kStep + 8 * g;
      const unsigned o = st < steps ? wcol + static_cast<unsigned>(k) * static_cast<unsigned>(pitch)
                                    : static_cast<unsigned>(kExpertOob);
#pragma unroll
      for (int i = 0; i < 8; ++i) r.w[i] = load_piece<CB>(w, static_cast<int>(o + static_cast<unsigned>(i * pitch)));
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int q = 0; q < TERMS * AP; ++q) {
          const int kq = k + q % AP * (16 / ELT);
          r.x[i][q] = __builtin_amdgcn_raw_buffer_load_b128(
              x, arow[i] >= 0 && kq < K ? arow[i] + q / AP * plane + kq * ELT : kExpertOob, 0, 0);
        }
    };
    auto multiply = [&](const Regs& r) __attribute__((always_inline)) {
      if constexpr (ELT == 2) {
        u32x4 col[NC];
        columns_of(r.w, col);
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int q = 0; q < TERMS; ++q)
#pragma unroll
            for (int j = 0; j < NC; ++j)
              acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, r.x[i][q]),
                                                                  __builtin_bit_cast(bf16x8, col[j]), acc[i][j], 0, 0, 0);
      } else {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int q = 0; q < 8; ++q)
#pragma unroll
            for (int j = 0; j < NC; ++j)
              acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(r.x[i][q / 4][q % 4]),
                                                               __uint_as_float(r.w[q][j]), acc[i][j], 0, 0, 0);
      }
    };
    // the next step's loads are on their way while this one is multiplied
    Regs ra, rb;
    load(ra, step);
    for (; step + stride < steps; step += 2 * stride) {
      load(rb, step + stride);
      multiply(ra);
      load(ra, step + 2 * stride);
      multiply(rb);
    }
    if (step < steps) multiply(ra);
  }

  // Tile i to this wave's 16 rows of 16 NC columns in LDS.
  __device__ __forceinline__ void put(float* red, int i) const {
    const int g = lane_id() / 16, m = lane_id() % 16;
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int j = 0; j < NC; ++j) red[(4 * g + r) * 16 * NC + NC * m + j] = acc[i][j][r];
  }
};

// One expert's strip: the rows of A that `list` names times NB columns of its matrix.
// FIRST: A = x (row list / k), out = hidden; else A = hidden (row list), out = partial sums.
// Rows past those that fit the registers take further passes, dealt to `shares` blocks.
template <class T, int CB, int MAXT, int WAVES, bool FIRST, bool GATED>
__global__ __launch_bounds__(WAVES* kWave) void layer_strip_kernel(LayerArgs a, int shares) {
  constexpr int ELT = static_cast<int>(sizeof(T));
  constexpr int NC = CB / ELT, NB = 16 * NC;   // columns per lane and strip
  constexpr bool kSplit = FIRST && GATED;      // half of the strip's lanes take the gate's columns
  constexpr int NBO = kSplit ? NB / 2 : NB;
  constexpr int THREADS = WAVES * kWave;
  __shared__ __align__(16) float red[WAVES * 16 * NB];
  __shared__ int lists[kLayerMaxChoices];
  __shared__ int wave_n[WAVES];

  const int tid = threadIdx.x, lane = lane_id(), m = lane % 16;
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int choices = a.S * a.k;
  int e = blockIdx.y;
  int n = 0;
  const int* list;  // the choices of e, in order
  if (choices <= kWave) {
    // each wave for itself, without a barrier
    const int mine = lane < choices ? a.ids[lane] : -1;
    if (a.by_choice) {
      e = __builtin_amdgcn_readlane(mine, blockIdx.y);
      if (e < 0 || e >= a.E) return;
    }
    const uint64_t mask = __ballot(mine == e);
    // the first choice of an expert takes all of its rows
    if (a.by_choice && (mask & ((uint64_t(1) << blockIdx.y) - 1)) != 0) return;
    n = __popcll(mask);
    if (mine == e) lists[wave * kWave + popc_below(mask)] = lane;
    list = lists + wave * kWave;
    __builtin_amdgcn_wave_barrier();
  } else {
    if (a.by_choice) {
      const int c = blockIdx.y;
      e = a.ids[c];
      if (e < 0 || e >= a.E) return;
      bool earlier = false;
      for (int i = lane; i < c; i += kWave) earlier |= a.ids[i] == e;
      if (__ballot(earlier)) return;
    }
    for (int base = 0; base < choices; base += THREADS) {
      const int c = base + tid;
      const bool mine = c < choices && a.ids[c] == e;
      const uint64_t mask = __ballot(mine);
      if (lane == 0) wave_n[wave] = __popcll(mask);
      __syncthreads();
      int at = n;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) {
        const int wn = wave_n[w];
        at += w < wave ? wn : 0;
        n += wn;
      }
      if (mine) lists[at + popc_below(mask)] = c;
      __syncthreads();
    }
    list = lists;
  }
  const int share = blockIdx.z % shares, z = blockIdx.z / shares, zs = gridDim.z / shares;
  if (n <= 16 * MAXT * share) return;

  const int K = FIRST ? a.d : a.h;
  const int N = FIRST ? a.h : a.d;             // columns of the output
  const int N1 = kSplit ? 2 * N : N;           // of the matrix
  const int n0 = blockIdx.x * NBO;
  const int oc = n0 + NC * (kSplit ? m % 8 : m);
  const unsigned wcol = oc < N ? (oc + (kSplit && m >= 8 ? N : 0)) * ELT : kExpertOob;
  const __amdgpu_buffer_rsrc_t wsrc =
      expert_rsrc(reinterpret_cast<const T*>(FIRST ? a.w1 : a.w2) + static_cast<int64_t>(e) * K * N1, K * N1 * ELT);
  // bf16: hidden as the sum of two, so that it keeps 16 bits on its way to the second product,
  // which reads the weights all the same (one: y off by 1.4 times its own rounding)
  constexpr int TERMS = ELT == 2 && !FIRST ? 2 : 1;
  const int plane = choices * a.h * ELT;
  const __amdgpu_buffer_rsrc_t asrc = expert_rsrc(FIRST ? a.x : a.hidden, FIRST ? a.S * K * ELT : TERMS * plane);

  // MT tiles of 16 rows of the list, from r0 on
  auto run = [&](auto tiles, int r0) {
    constexpr int MT = decltype(tiles)::v;
    int arow[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int li = r0 + 16 * i + m;
      arow[i] = li < n ? (FIRST ? list[li] / a.k : list[li]) * K * ELT : -1;
    }
    StripSums<T, CB, MT, TERMS> sums;
    sums.run(wsrc, wcol, N1 * ELT, asrc, arow, plane, K, z * WAVES + wave, zs * WAVES);

    // added over the waves, 16 rows at a time
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      sums.put(red + wave * 16 * NB, i);
      __syncthreads();
      for (int o = tid; o < 16 * NBO; o += THREADS) {
        const int row = o / NBO, c = o % NBO;
        const int li = r0 + 16 * i + row;
        if (li >= n || n0 + c >= N) continue;
        float v = 0.f, u = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
          v += red[(w * 16 + row) * NB + c];
          if constexpr (kSplit) u += red[(w * 16 + row) * NB + NBO + c];
        }
        if constexpr (FIRST) {
          if (a.b1) {
            v += a.b1[static_cast<int64_t>(e) * N1 + n0 + c];
            if constexpr (kSplit) u += a.b1[static_cast<int64_t>(e) * N1 + N + n0 + c];
          }
          float f = 0.f;
          expert_by_act(a.act, [&](auto which) { f = expert_act<decltype(which)::v>(v); });
          if constexpr (kSplit) f *= u;
          T* out = reinterpret_cast<T*>(a.hidden) + static_cast<int64_t>(list[li]) * N + n0 + c;
          if constexpr (ELT == 2) {
            // Both of f's sign and neither zero unless f is, so that times an infinite weight they
            // add up to an infinity: the first is cut, not rounded, and a second one below the
            // normal numbers becomes the least of them.  The 8 bits of the second follow the
            // 8 of the first: off by 2^-16 of f at most (by 2^-126 where that is more).
            uint32_t hi = __float_as_uint(f) >> 16, lo;
            if ((hi & 0x7f80u) == 0x7f80u) {
              hi = lo = f32_to_bf16_bits(f);  // an infinity or a NaN
            } else {
              lo = f32_to_bf16_bits(f - __uint_as_float(hi << 16));
              if ((lo & 0x7f80u) == 0) lo = f == 0.f ? 0u : (hi & 0x8000u) | 0x0080u;
            }
            out->bits = static_cast<uint16_t>(hi);
            out[static_cast<int64_t>(choices) * a.h].bits = static_cast<uint16_t>(lo);
          }
          else *out = f;
        } else {
          a.part[(static_cast<int64_t>(z) * choices + list[li]) * N + n0 + c] = v;
        }
      }
      __syncthreads();
    }
  };
  // no more row tiles than the list has: matrix units idle beside them cost nothing, but
  // in fp32 the products of 48 rows take longer than the weights that they share
  for (int r0 = 16 * MAXT * share; r0 < n; r0 += 16 * MAXT * shares) {
    const int left = n - r0;
    if (MAXT == 1 || left <= 16) run(ExpertInt<1>(), r0);
    else if (MAXT == 2 || left <= 32) run(ExpertInt<(MAXT > 1 ? 2 : 1)>(), r0);
    else run(ExpertInt<(MAXT > 2 ? 3 : 1)>(), r0);
  }
}

// The gate, in two launches: logits of 16 tokens x a strip of experts over one range of K per
// block, every wave's loads in flight at once ([z, S, E] partial sums); then, a wave per
// token, the ranges' sum, noise and temperature, selection and weights.  (All in one launch
// a single CU reads the whole matrix: 10.2 us for one token, 2048 x 64.)
template <class T, int CB>
__global__ __launch_bounds__(kLayerGateWaves* kWave) void layer_logits_kernel(LayerGateArgs a) {
  constexpr int ELT = static_cast<int>(sizeof(T));
  constexpr int NB = 16 * CB / ELT;
  __shared__ __align__(16) float red[kLayerGateWaves * 16 * NB];
  const int tid = threadIdx.x, m = lane_id() % 16;
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int tok0 = blockIdx.y * 16, E = a.E, n0 = blockIdx.z * NB;
  const __amdgpu_buffer_rsrc_t w = expert_rsrc(a.wg, a.d * E * ELT), x = expert_rsrc(a.x, a.S * a.d * ELT);
  const int arow[1] = {tok0 + m < a.S ? (tok0 + m) * a.d * ELT : -1};
  const int col = n0 + CB / ELT * m;
  StripSums<T, CB, 1, 1> sums;
  sums.run(w, col < E ? col * ELT : kExpertOob, E * ELT, x, arow, 0, a.d, blockIdx.x * kLayerGateWaves + wave,
           gridDim.x * kLayerGateWaves);
  sums.put(red + wave * 16 * NB, 0);
  __syncthreads();
  for (int o = tid; o < 16 * NB; o += kLayerGateWaves * kWave) {
    const int row = o / NB, e = n0 + o % NB;
    if (e >= E || tok0 + row >= a.S) continue;
    float v = 0.f;
#pragma unroll
    for (int q = 0; q < kLayerGateWaves; ++q) v += red[(q * 16 + row) * NB + o % NB];
    a.part[(static_cast<int64_t>(blockIdx.x) * a.S + tok0 + row) * E + e] = v;
  }
}

__global__ __launch_bounds__(kBlock) void layer_select_kernel(LayerGateArgs a) {
  extern __shared__ float lds[];  // a row of logits per wave, then the selection's counts (not used here)
  const int wave = threadIdx.x / kWave, lane = lane_id(), E = a.E;
  const int s = blockIdx.x * kWavesPerBlock + wave;
  const bool valid = s < a.S;
  float* row = lds + wave * E;
  int* counted = reinterpret_cast<int*>(lds + kWavesPerBlock * E);
  const int64_t at = static_cast<int64_t>(valid ? s : 0) * E, plane = static_cast<int64_t>(a.S) * E;
  for (int e = lane; e < E; e += kWave) {
    float p[kLayerGateSplits];
#pragma unroll
    for (int z = 0; z < kLayerGateSplits; ++z) p[z] = z < a.z ? a.part[z * plane + at + e] : 0.f;
    float v = 0.f;
#pragma unroll
    for (int z = 0; z < kLayerGateSplits; ++z) v += p[z];
    if (a.bias) v += a.bias[e];
    if (a.temperature > 0.f) {
      if (a.noise) v += a.noise[at + e];
      v = v / a.temperature;
    }
    row[e] = v;
  }
  __syncthreads();
  int32_t* ids = a.ids + static_cast<int64_t>(s) * a.k;
  float* wt = a.weights + static_cast<int64_t>(s) * a.k;
  auto select = [&](auto kmax, auto mode) {
    select_row<kWave, decltype(kmax)::v, decltype(mode)::v>(row, E, a.k, a.groups, a.normalize, lane, valid, ids, wt, counted);
  };
  if (a.kind == 1) select(ExpertInt<1>(), ExpertInt<1>());
  else if (a.kind == 3) a.k <= 2 ? select(ExpertInt<2>(), ExpertInt<3>()) : select(ExpertInt<8>(), ExpertInt<3>());
  else if (a.k <= 2) select(ExpertInt<2>(), ExpertInt<0>());
  else select(ExpertInt<8>(), ExpertInt<0>());
}

// y[s, c] = sum over r of weights[s, r] (b2[ids[s, r], c] + sum over z of part[z, s k + r, c]).
template <class T>
__global__ __launch_bounds__(kBlock) void layer_combine_kernel(LayerArgs a) {
  const int s = blockIdx.y;
  const int c = (blockIdx.x * kBlock + threadIdx.x) * 4;
  if (c >= a.d) return;
  const int64_t choices = static_cast<int64_t>(a.S) * a.k;
  f32x4 y = {0.f, 0.f, 0.f, 0.f};
  for (int r = 0; r < a.k; ++r) {
    const int64_t ch = static_cast<int64_t>(s) * a.k + r;
    const int e = a.ids[ch];
    if (e < 0 || e >= a.E) continue;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    for (int z0 = 0; z0 < a.z2; z0 += 4) {
      f32x4 p[4];
#pragma unroll
      for (int z = 0; z < 4; ++z)
        p[z] = *reinterpret_cast<const f32x4*>(a.part + (min(z0 + z, a.z2 - 1) * choices + ch) * a.d + c);
#pragma unroll
      for (int z = 0; z < 4; ++z)
        if (z0 + z < a.z2) v += p[z];
    }
    if (a.b2) {
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] += a.b2[static_cast<int64_t>(e) * a.d + c + q];
    }
    const float w = a.weights[ch];
#pragma unroll
    for (int q = 0; q < 4; ++q) y[q] += w * v[q];
  }
  T* out = reinterpret_cast<T*>(a.y) + static_cast<int64_t>(s) * a.d + c;
  if constexpr (sizeof(T) == 2) {
    *reinterpret_cast<uint2*>(out) = uint2{pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3])};
  } else {
    *reinterpret_cast<f32x4*>(out) = y;
  }
}

template <class T, int CB, int MT, int WAVES, bool FIRST>
hipError_t strip(const LayerArgs& a, int z, hipStream_t st) {
  constexpr int NB = 16 * CB / static_cast<int>(sizeof(T));
  const int slots = a.by_choice ? a.S * a.k : a.E;
  const int N = FIRST ? a.h : a.d;
  const int nbo = FIRST && a.gated ? NB / 2 : NB;
  const int64_t blocks = static_cast<int64_t>((N + nbo - 1) / nbo) * slots * z;
  // passes side by side where the blocks are fewer than two per CU (bf16, 256 tokens of one
  // choice, 2 experts of 1024 x 4096: the layer 80 -> 47 us; 8 experts of 1024 x 2048, two
  // choices: 64 -> 51), one after the other on the same weights where they are more
  const int passes = (a.S + 16 * MT - 1) / (16 * MT);
  const int shares = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(passes, 512 / blocks)));
  const dim3 grid((N + nbo - 1) / nbo, slots, z * shares);
  if (FIRST && a.gated) layer_strip_kernel<T, CB, MT, WAVES, FIRST, true><<<grid, WAVES * kWave, 0, st>>>(a, shares);
  else layer_strip_kernel<T, CB, MT, WAVES, FIRST, false><<<grid, WAVES * kWave, 0, st>>>(a, shares);
  return hipGetLastError();
}

// Strips of 256 bytes by four waves; of 128 bytes by sixteen where the wide ones are
// too few to occupy the chip and few rows leave the registers for it.
bool narrow(const LayerArgs& a, bool first) {
  const int elt = a.dtype == 1 ? 2 : 4;
  const int64_t cols = first ? (a.gated ? 2 * static_cast<int64_t>(a.h) : a.h) : a.d;
  const int64_t slots = a.by_choice ? a.S * a.k : a.E;
  return a.S <= 16 && slots * ((cols * elt + 255) / 256) < 512;
}

template <class T, bool FIRST>
hipError_t strips(const LayerArgs& a, hipStream_t st) {
  const int z = FIRST ? 1 : a.z2;
  if (narrow(a, FIRST)) return strip<T, 8, 1, 16, FIRST>(a, z, st);
  // row tiles in registers for about twice the mean rows of an expert, so that few need a
  // second pass over their weights: fewer tiles leave room for more waves
  const int64_t rows = std::min<int64_t>(a.S, 2 * ((static_cast<int64_t>(a.S) * a.k + a.E - 1) / a.E));
  if (rows <= 16) return strip<T, 16, 1, 4, FIRST>(a, z, st);
  if (rows <= 32) return strip<T, 16, 2, 4, FIRST>(a, z, st);
  // (16 experts of 1024 x 4096 in fp32, 100 tokens of four choices: 48 rows by four waves 75
  // and 69 us, 32 rows, where some experts take two passes, 87 and 92).  In bf16 eight
  // waves: four would leave a SIMD one.
  return strip<T, 16, 3, sizeof(T) == 2 ? 8 : 4, FIRST>(a, z, st);
}

template <class T>
hipError_t run_layer(const LayerArgs& a, hipStream_t st) {
  hipError_t err = strips<T, true>(a, st);
  if (err != hipSuccess) return err;
  if ((err = strips<T, false>(a, st)) != hipSuccess) return err;
  layer_combine_kernel<T><<<dim3((a.d + 4 * kBlock - 1) / (4 * kBlock), a.S), kBlock, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace

// Blocks along the second matrix's K: enough that two per CU run, with at least four steps
// for each wave (two where eight waves share a strip).
int layer_splits(const LayerArgs& a) {
  const int elt = a.dtype == 1 ? 2 : 4;
  const bool nar = narrow(a, false);
  const int64_t slots = a.by_choice ? a.S * a.k : a.E;
  const int64_t blocks = slots * ((static_cast<int64_t>(a.d) * elt + (nar ? 127 : 255)) / (nar ? 128 : 256));
  const int64_t most = a.h / (kStep * 4 * (nar ? 16 : 4));
  return static_cast<int>(std::max<int64_t>(1, std::min<int64_t>({8, most, 512 / std::max<int64_t>(1, blocks)})));
}

// Whether the gate runs in the two launches above: W in whole pieces at 32-bit offsets.
bool layer_gate_fits(const LayerGateArgs& a) {
  const int64_t elt = a.dtype == 1 ? 2 : 4;
  return a.E * elt % 16 == 0 && reinterpret_cast<uintptr_t>(a.wg) % 16 == 0 && a.d * a.E * elt < (int64_t(1) << 30);
}

// Ranges of K: one step per wave where that takes no more than kLayerGateSplits.
int layer_gate_splits(int d) {
  const int z = (d + kStep * kLayerGateWaves - 1) / (kStep * kLayerGateWaves);
  return z < kLayerGateSplits ? z : kLayerGateSplits;
}

hipError_t launch_layer_gate(const LayerGateArgs& a, hipStream_t st) {
  const int elt = a.dtype == 1 ? 2 : 4, nb = a.E * elt <= 128 ? 128 / elt : 256 / elt;
  const dim3 grid(a.z, (a.S + 15) / 16, (a.E + nb - 1) / nb);
  constexpr int kThreads = kLayerGateWaves * kWave;
  if (a.dtype == 1) {
    if (nb == 64) layer_logits_kernel<bf16_t, 8><<<grid, kThreads, 0, st>>>(a);
    else layer_logits_kernel<bf16_t, 16><<<grid, kThreads, 0, st>>>(a);
  } else {
    if (nb == 32) layer_logits_kernel<float, 8><<<grid, kThreads, 0, st>>>(a);
    else layer_logits_kernel<float, 16><<<grid, kThreads, 0, st>>>(a);
  }
  hipError_t err = hipGetLastError();
  if (err != hipSuccess) return err;
  const size_t lds = static_cast<size_t>(kWavesPerBlock + a.k) * a.E * 4;
  layer_select_kernel<<<(a.S + kWavesPerBlock - 1) / kWavesPerBlock, kBlock, lds, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_layer(const LayerArgs& a, hipStream_t st) {
  return a.dtype == 1 ? run_layer<bf16_t>(a, st) : run_layer<float>(a, st);
}

}  // namespace hetumoe
