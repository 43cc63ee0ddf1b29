// The whole layer for a few tokens: expert networks on the rows that chose them,
// without slots or dispatch, and the weighted sum of the choices.
//
// With few rows per expert the weights are what there is to read, so a block streams
// a strip of one expert's matrix past all rows that chose it: its waves take
// steps of 32 rows of the matrix in turn (each lane one piece of 8 of them, whole
// 256- or 128-byte stretches per row), turn them into matrix-core operands in
// registers, and add their sums in LDS at the end.  The second matrix's K is also
// split over blocks where that is needed to occupy the chip; the last kernel adds
// those parts in order.  No atomics: results repeat bit for bit.
#include <algorithm>

#include "experts.hpp"

namespace hetumoe {

namespace {

constexpr int kStep = 32;  // K per wave step

template <int CB> struct Piece;
template <> struct Piece<16> { typedef u32x4 T; };
template <> struct Piece<8> { typedef unsigned T __attribute__((ext_vector_type(2))); };

template <int CB>
__device__ __forceinline__ typename Piece<CB>::T load_piece(__amdgpu_buffer_rsrc_t r, int off) {
  if constexpr (CB == 16) return __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, 0);
  else return __builtin_amdgcn_raw_buffer_load_b64(r, off, 0, 0);
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

// One expert's strip: the rows of A that `list` names times NB columns of its matrix.
// FIRST: A = x (row list / k), out = hidden; else A = hidden (row list), out = partial sums.
template <class T, int CB, int MAXT, int WAVES, bool FIRST, bool GATED>
__global__ __launch_bounds__(WAVES* kWave) void layer_strip_kernel(LayerArgs a) {
  constexpr int ELT = static_cast<int>(sizeof(T));
  constexpr int NC = CB / ELT, NB = 16 * NC;   // columns per lane and strip
  constexpr bool kSplit = FIRST && GATED;      // half of the strip's lanes take the gate's columns
  constexpr int NBO = kSplit ? NB / 2 : NB;
  constexpr int AP = 8 * ELT / 16;             // 16-byte pieces of A per row and lane
  constexpr int THREADS = WAVES * kWave;
  __shared__ __align__(16) float red[WAVES * 16 * NB];
  __shared__ int list[kLayerMaxChoices];
  __shared__ int wave_n[WAVES];

  const int tid = threadIdx.x, lane = lane_id(), g = lane / 16, m = lane % 16;
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int choices = a.S * a.k;
  int e = blockIdx.y;
  if (a.by_choice) {
    // the first choice of an expert takes all of its rows (at most E choices here)
    const int c = blockIdx.y;
    e = a.ids[c];
    if (e < 0 || e >= a.E) return;
    bool earlier = false;
    for (int i = lane; i < c; i += kWave) earlier |= a.ids[i] == e;
    if (__ballot(earlier)) return;
  }
  // the choices of e, in order
  int n = 0;
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
    if (mine) list[at + popc_below(mask)] = c;
    __syncthreads();
  }
  if (n == 0) return;

  const int K = FIRST ? a.d : a.h;
  const int N = FIRST ? a.h : a.d;             // columns of the output
  const int N1 = kSplit ? 2 * N : N;           // of the matrix
  const int n0 = blockIdx.x * NBO;
  const int oc = n0 + NC * (kSplit ? m % 8 : m);
  const int wcol = oc < N ? oc + (kSplit && m >= 8 ? N : 0) : -1;
  const __amdgpu_buffer_rsrc_t wsrc =
      expert_rsrc(reinterpret_cast<const T*>(FIRST ? a.w1 : a.w2) + static_cast<int64_t>(e) * K * N1, K * N1 * ELT);
  const __amdgpu_buffer_rsrc_t asrc = expert_rsrc(FIRST ? a.x : a.hidden, (FIRST ? a.S : choices) * K * ELT);
  const int steps = (K + kStep - 1) / kStep;
  const int stride = gridDim.z * WAVES;

  // MT tiles of 16 rows of the list, from r0 on
  auto run = [&](auto tiles, int r0) {
    constexpr int MT = decltype(tiles)::v;
    int arow[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int li = r0 + 16 * i + m;
      arow[i] = li < n ? (FIRST ? list[li] / a.k : list[li]) * K * ELT : -1;
    }
    f32x4 acc[MT][NC];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NC; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

    typedef typename Piece<CB>::T piece_t;
    struct Regs {
      piece_t w[8];
      u32x4 x[MT][AP];
    };
    auto load = [&](Regs& r, int step) {
      const int k = step * kStep + 8 * g;
#pragma unroll
      for (int i = 0; i < 8; ++i)
        r.w[i] = load_piece<CB>(wsrc, wcol >= 0 && k + i < K ? ((k + i) * N1 + wcol) * ELT : kExpertOob);
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int q = 0; q < AP; ++q)
          r.x[i][q] = __builtin_amdgcn_raw_buffer_load_b128(
              asrc, arow[i] >= 0 && k + q * (16 / ELT) < K ? arow[i] + (k + q * (16 / ELT)) * ELT : kExpertOob, 0, 0);
    };
    auto multiply = [&](const Regs& r) {
      if constexpr (ELT == 2) {
        u32x4 col[NC];
        columns_of(r.w, col);
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int j = 0; j < NC; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, r.x[i][0]),
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
    // the next step's loads are on their way while this one is multiplied; a step past
    // the last one loads zeros from outside the resources
    Regs ra, rb;
    int step = blockIdx.z * WAVES + wave;
    load(ra, step);
    for (; step + stride < steps; step += 2 * stride) {
      load(rb, step + stride);
      multiply(ra);
      load(ra, step + 2 * stride);
      multiply(rb);
    }
    if (step < steps) multiply(ra);

    // sums of the waves, 16 rows at a time: lane (g, m) holds rows 4 g + r, columns NC m + j
#pragma unroll
    for (int i = 0; i < MT; ++i) {
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int j = 0; j < NC; ++j) red[(wave * 16 + 4 * g + r) * NB + NC * m + j] = acc[i][j][r];
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
          // rounded to the element type like the hidden rows of the experts call: the
          // second product's operand
          if constexpr (ELT == 2) out->bits = static_cast<uint16_t>(f32_to_bf16_bits(f));
          else *out = f;
        } else {
          a.part[(static_cast<int64_t>(blockIdx.z) * choices + list[li]) * N + n0 + c] = v;
        }
      }
      __syncthreads();
    }
  };
  // no more row tiles than the list has: matrix units idle beside them cost nothing, but
  // in fp32 the products of 64 rows take longer than the weights that they share
  for (int r0 = 0; r0 < n; r0 += 16 * MAXT) {
    const int left = n - r0;
    if (MAXT == 1 || left <= 16) run(ExpertInt<1>(), r0);
    else if (MAXT == 2 || left <= 32) run(ExpertInt<(MAXT > 1 ? 2 : 1)>(), r0);
    else if (MAXT == 3 || left <= 48) run(ExpertInt<(MAXT > 2 ? 3 : 1)>(), r0);
    else run(ExpertInt<(MAXT > 3 ? 4 : 1)>(), r0);
  }
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
    for (int z = 0; z < a.z2; ++z) v += *reinterpret_cast<const f32x4*>(a.part + (z * choices + ch) * a.d + c);
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
  if (FIRST && a.gated) {
    layer_strip_kernel<T, CB, MT, WAVES, FIRST, true>
        <<<dim3((N + NB / 2 - 1) / (NB / 2), slots, z), WAVES * kWave, 0, st>>>(a);
  } else {
    layer_strip_kernel<T, CB, MT, WAVES, FIRST, false><<<dim3((N + NB - 1) / NB, slots, z), WAVES * kWave, 0, st>>>(a);
  }
  return hipGetLastError();
}

// Strips of 256 bytes by eight waves; of 128 bytes by sixteen where the wide ones are
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
  if (a.S <= 16) return strip<T, 16, 1, 8, FIRST>(a, z, st);
  if (a.S <= 32) return strip<T, 16, 2, 8, FIRST>(a, z, st);
  // 48 rows are what the registers hold in bf16
  return strip<T, 16, sizeof(T) == 2 ? 3 : 4, 8, FIRST>(a, z, st);
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

// Blocks along the second matrix's K: enough that two per CU run, with at least
// four steps for each wave.
int layer_splits(const LayerArgs& a) {
  const int elt = a.dtype == 1 ? 2 : 4;
  const bool nar = narrow(a, false);
  const int64_t slots = a.by_choice ? a.S * a.k : a.E;
  const int64_t blocks = slots * ((static_cast<int64_t>(a.d) * elt + (nar ? 127 : 255)) / (nar ? 128 : 256));
  const int64_t most = a.h / (kStep * 4 * (nar ? 16 : 8));
  return static_cast<int>(std::max<int64_t>(1, std::min<int64_t>({8, most, 512 / std::max<int64_t>(1, blocks)})));
}

hipError_t launch_layer(const LayerArgs& a, hipStream_t st) {
  return a.dtype == 1 ? run_layer<bf16_t>(a, st) : run_layer<float>(a, st);
}

}  // namespace hetumoe
