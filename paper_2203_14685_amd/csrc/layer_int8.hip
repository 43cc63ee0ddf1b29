// The layer for a few tokens with weights in 8-bit integers.
//
// As layer.hip: the weights' bytes are what there is to read, a block streams a strip of one
// expert's matrix past all rows that chose it.  The matrix's rows are the product's columns and run
// along K, so 16 bytes of one are a lane's part of a matrix-core operand: 16 rows of the
// matrix are one operand, 16 tokens the other.  A block's waves take ranges of K and add their
// sums, which are exact, in LDS; K of the second product is also split over blocks.
// Tokens and hidden rows are quantized by launches of their own: a row's scale needs all of it.
#include <algorithm>

#include "experts.hpp"
#include "layer_choices.hpp"

namespace hetumoe {

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int kInt8Waves = 4;
constexpr int kInt8Tiles = 4;                  // of 16 rows of the matrix per block
constexpr int kInt8Strip = 16 * kInt8Tiles;
constexpr int kInt8Step = 256;                 // K of one stage: bytes of a row that are read together
constexpr int kInt8Stage = 16 * kInt8Step;     // bytes of a stage: 16 rows, four loads to LDS
constexpr int kInt8Ring = 4;                   // stages of a wave

// A wave's stages come straight to its own part of LDS, 16 rows x 256 bytes each, so that memory is
// read in whole stretches (40 experts of 4096 rows of 2048 bytes: 6.9 TB/s non-temporal; with
// 64 bytes of each of 16 rows at a time, as the operands would take them, 4.8): per 256 of K the token
// tiles first, then the strip's tiles.  Four stages take turns; no wave waits for another.
//
// Piece c (16 bytes) of row r lies at place c ^ r, which leaves the operand reads without bank
// conflicts; a load fills LDS in lane order, so the lane fetches the piece that belongs there.

// The four operands of a stage (64 of K each): waits until no more than the three stages behind it
// are on their way; when it returns the stage's place is free.
__device__ __forceinline__ void int8_operands(unsigned at, i32x4 (&f)[4]) {
  static_assert(kInt8Ring == 4, "12 loads of the three stages behind this one");
  asm volatile(
      "s_waitcnt vmcnt(12)\n\t"
      "ds_read_b128 %0, %4\n\tds_read_b128 %1, %5\n\tds_read_b128 %2, %6\n\tds_read_b128 %3, %7\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(f[0]), "=&v"(f[1]), "=&v"(f[2]), "=&v"(f[3])
      : "v"(at), "v"(at ^ 64), "v"(at ^ 128), "v"(at ^ 192)
      : "memory");
}

// Sums of the strip with MT tiles of 16 tokens over steps lo .. hi - 1 of K.
template <int MT>
struct Int8Sums {
  static constexpr int kStages = MT + kInt8Tiles;  // per step
  i32x4 acc[MT][kInt8Tiles];

  // w0, w1: the matrix from the strip's first row on, for the first and the other half of its
  // tiles; xrow[i][q]: byte of the row of tile i that the lane fetches in load q, or kExpertOob.
  __device__ __forceinline__ void run(__amdgpu_buffer_rsrc_t w0, __amdgpu_buffer_rsrc_t w1, int pitch,
                                      __amdgpu_buffer_rsrc_t x, const int (&xrow)[MT][4], int K, int lo, int hi,
                                      char* ring) {
    const int lane = lane_id(), g = lane / 16, m = lane % 16;
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < kInt8Tiles; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
    // load q of a stage: rows 4 q + g
    int wrow[4], piece[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      piece[q] = (m ^ (4 * q + g)) * 16;
      wrow[q] = (4 * q + g) * pitch + piece[q];
    }
    // stage s of step st, to place p; behind the last step: zeros, so that the count of loads stays
    auto load = [&](int s, int st, int p) __attribute__((always_inline)) {
      char* dst = ring + p * kInt8Stage;
      const int k = st * kInt8Step, j = s - MT;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const bool in = st < hi && k + piece[q] < K;
        if (s < MT) {
          const int off = in && xrow[s < MT ? s : 0][q] != kExpertOob ? xrow[s < MT ? s : 0][q] + k + piece[q] : kExpertOob;
          __builtin_amdgcn_raw_ptr_buffer_load_lds(x, (lds_void*)(dst + q * 1024), 16, off, 0, 0, 0);
        } else {
          // non-temporal: a strip is read once
          const int off = in ? j % (kInt8Tiles / 2) * 16 * pitch + wrow[q] + k : kExpertOob;
          if (j < kInt8Tiles / 2) __builtin_amdgcn_raw_ptr_buffer_load_lds(w0, (lds_void*)(dst + q * 1024), 16, off, 0, 0, 2);
          else __builtin_amdgcn_raw_ptr_buffer_load_lds(w1, (lds_void*)(dst + q * 1024), 16, off, 0, 0, 2);
        }
      }
    };
    const unsigned at = static_cast<unsigned>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char*)(ring))) +
                        m * kInt8Step + (g ^ m) * 16;
#pragma unroll
    for (int s = 0; s < kInt8Ring; ++s) load(s % kStages, lo + s / kStages, s);
    i32x4 xf[MT][4];
    int n = 0;  // stages taken: the next one lies at place n % 4
    for (int st = lo; st < hi; ++st) {
#pragma unroll
      for (int s = 0; s < kStages; ++s) {
        const int p = n++ % kInt8Ring;
        if (s < MT) {
          int8_operands(at + p * kInt8Stage, xf[s < MT ? s : 0]);
        } else {
          i32x4 wf[4];
          int8_operands(at + p * kInt8Stage, wf);
#pragma unroll
          for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int i = 0; i < MT; ++i)
              acc[i][s < MT ? 0 : s - MT] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wf[u], xf[i][u], acc[i][s < MT ? 0 : s - MT], 0, 0, 0);
        }
        load((s + kInt8Ring) % kStages, st + (s + kInt8Ring) / kStages, p);
      }
    }
    __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0): nothing is on its way to the ring
    asm volatile("" ::: "memory");
  }

  // Tile i to LDS: token m, the strip's rows next to each other.
  __device__ __forceinline__ void put(int* red, int i) const {
    const int g = lane_id() / 16, m = lane_id() % 16;
#pragma unroll
    for (int j = 0; j < kInt8Tiles; ++j)
      *reinterpret_cast<i32x4*>(red + m * (kInt8Strip + 4) + 16 * j + 4 * g) = acc[i][j];
  }
};

// One strip of an expert's matrix past its rows, MT tiles of them at a time, passes dealt to
// `shares` blocks.  FIRST: hidden (T), else partial integer sums.
template <class T, int MT, bool FIRST, bool GATED>
__global__ __launch_bounds__(kInt8Waves* kWave, 2) void layer_int8_kernel(LayerInt8Args b, int shares) {
  constexpr bool kSplit = FIRST && GATED;  // half of the strip's rows are the gate's
  constexpr int NBO = kSplit ? kInt8Strip / 2 : kInt8Strip;
  constexpr int kPitch = kInt8Strip + 4, kThreads = kInt8Waves * kWave;
  // the waves' rings; then, in the same places, a tile of sums of each
  __shared__ __align__(1024) char ring[kInt8Waves][kInt8Ring * kInt8Stage];
  static_assert(16 * kPitch * 4 <= kInt8Ring * kInt8Stage, "room for a tile");
  __shared__ int lists[kLayerMaxChoices];
  __shared__ int wave_n[kInt8Waves];
  const LayerArgs& a = b.a;
  const int tid = threadIdx.x, g = lane_id() / 16;
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  int e, n;
  const int* list;
  if (!layer_choices<kInt8Waves>(a, lists, wave_n, e, n, list)) return;
  e = __builtin_amdgcn_readfirstlane(e);
  const int share = blockIdx.z % shares, z = blockIdx.z / shares, zs = gridDim.z / shares;
  if (n <= 16 * MT * share) return;

  const int K = FIRST ? a.d : a.h, N = FIRST ? a.h : a.d, N1 = kSplit ? 2 * N : N;
  const int n0 = blockIdx.x * NBO;
  const int8_t* w = reinterpret_cast<const int8_t*>(FIRST ? a.w1 : a.w2) + (static_cast<int64_t>(e) * N1 + n0) * K;
  // rows of the matrix behind N: zeros
  const int half = kSplit ? NBO : NBO / 2;
  const int64_t apart = static_cast<int64_t>(kSplit ? N : half) * K;
  const int v0 = min(half, N - n0), v1 = kSplit ? v0 : max(0, min(half, N - n0 - half));
  const __amdgpu_buffer_rsrc_t w0 = expert_rsrc(w, __builtin_amdgcn_readfirstlane(v0 * K));
  const __amdgpu_buffer_rsrc_t w1 = expert_rsrc(w + apart, __builtin_amdgcn_readfirstlane(v1 * K));
  const __amdgpu_buffer_rsrc_t x = expert_rsrc(FIRST ? b.qx : b.qh, (FIRST ? a.S : a.S * a.k) * K);
  const int steps = (K + kInt8Step - 1) / kInt8Step, parts = zs * kInt8Waves;
  const int per = (steps + parts - 1) / parts, lo = (z * kInt8Waves + wave) * per;

  for (int r0 = 16 * MT * share; r0 < n; r0 += 16 * MT * shares) {
    int xrow[MT][4];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int li = r0 + 16 * i + 4 * q + g;
        xrow[i][q] = li < n ? (FIRST ? list[li] / a.k : list[li]) * K : kExpertOob;
      }
    Int8Sums<MT> sums;
    sums.run(w0, w1, K, x, xrow, K, lo, min(steps, lo + per), ring[wave]);
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      if (r0 + 16 * i >= n) break;
      sums.put(reinterpret_cast<int*>(ring[wave]), i);
      __syncthreads();
      for (int o = tid; o < 16 * NBO; o += kThreads) {
        const int row = o / NBO, c = o % NBO, li = r0 + 16 * i + row;
        if (li >= n || n0 + c >= N) continue;
        int v = 0, u = 0;
#pragma unroll
        for (int q = 0; q < kInt8Waves; ++q) {
          const int* red = reinterpret_cast<const int*>(ring[q]) + row * kPitch + c;
          v += red[0];
          if constexpr (kSplit) u += red[NBO];
        }
        const int choice = list[li];
        if constexpr (FIRST) {
          const float sx = b.sx[choice / a.k];
          const int64_t at = static_cast<int64_t>(e) * N1 + n0 + c;
          const float p = static_cast<float>(v) * sx * b.s1[at] + (a.b1 ? a.b1[at] : 0.f);
          float f = 0.f;
          expert_by_act(a.act, [&](auto which) { f = expert_act<decltype(which)::v>(p); });
          if constexpr (kSplit) f *= static_cast<float>(u) * sx * b.s1[at + N] + (a.b1 ? a.b1[at + N] : 0.f);
          T* out = reinterpret_cast<T*>(a.hidden) + static_cast<int64_t>(choice) * N + n0 + c;
          if constexpr (sizeof(T) == 2) out->bits = static_cast<uint16_t>(f32_to_bf16_bits(f));
          else *out = f;
        } else {
          reinterpret_cast<int*>(a.part)[(static_cast<int64_t>(z) * a.S * a.k + choice) * N + n0 + c] = v;
        }
      }
      __syncthreads();
    }
  }
}

// y[s, c] = sum over r of weights[s, r] (sum over z of part[z, s k + r, c] sh[s k + r] s2[e, c] + b2[e, c]).
template <class T>
__global__ __launch_bounds__(kBlock) void layer_int8_combine_kernel(LayerInt8Args b) {
  const LayerArgs& a = b.a;
  const int s = blockIdx.y, c = (blockIdx.x * kBlock + threadIdx.x) * 4;
  if (c >= a.d) return;
  const int64_t choices = static_cast<int64_t>(a.S) * a.k;
  const int* part = reinterpret_cast<const int*>(a.part);
  f32x4 y = {0.f, 0.f, 0.f, 0.f};
  for (int r = 0; r < a.k; ++r) {
    const int64_t ch = static_cast<int64_t>(s) * a.k + r;
    const int e = a.ids[ch];
    if (e < 0 || e >= a.E) continue;
    i32x4 v = {0, 0, 0, 0};
    for (int z = 0; z < a.z2; ++z) v += *reinterpret_cast<const i32x4*>(part + (z * choices + ch) * a.d + c);
    const float w = a.weights[ch], sh = b.sh[ch];
    const int64_t at = static_cast<int64_t>(e) * a.d + c;
#pragma unroll
    for (int q = 0; q < 4; ++q) y[q] += w * (static_cast<float>(v[q]) * sh * b.s2[at + q] + (a.b2 ? a.b2[at + q] : 0.f));
  }
  T* out = reinterpret_cast<T*>(a.y) + static_cast<int64_t>(s) * a.d + c;
  if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(out) = uint2{pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3])};
  else *reinterpret_cast<f32x4*>(out) = y;
}

int slots(const LayerArgs& a) { return a.by_choice ? a.S * a.k : a.E; }

template <class T, int MT, bool FIRST>
hipError_t strip(const LayerInt8Args& b, int z, hipStream_t st) {
  const LayerArgs& a = b.a;
  const int N = FIRST ? a.h : a.d, nbo = FIRST && a.gated ? kInt8Strip / 2 : kInt8Strip;
  const int64_t strips = (N + nbo - 1) / nbo, blocks = strips * slots(a) * z;
  const int passes = (a.S + 16 * MT - 1) / (16 * MT);
  const int shares = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(passes, 512 / blocks)));
  const dim3 grid(static_cast<unsigned>(strips), slots(a), z * shares);
  constexpr int kThreads = kInt8Waves * kWave;
  if (FIRST && a.gated) layer_int8_kernel<T, MT, FIRST, true><<<grid, kThreads, 0, st>>>(b, shares);
  else layer_int8_kernel<T, MT, FIRST, false><<<grid, kThreads, 0, st>>>(b, shares);
  return hipGetLastError();
}

template <class T, bool FIRST>
hipError_t strips(const LayerInt8Args& b, hipStream_t st) {
  const LayerArgs& a = b.a;
  const int z = FIRST ? 1 : a.z2;
  // token tiles in registers for about twice the mean rows of an expert
  const int64_t rows = std::min<int64_t>(a.S, 2 * ((static_cast<int64_t>(a.S) * a.k + a.E - 1) / a.E));
  if (rows <= 16) return strip<T, 1, FIRST>(b, z, st);
  if (rows <= 32) return strip<T, 2, FIRST>(b, z, st);
  return strip<T, 4, FIRST>(b, z, st);
}

template <class T>
hipError_t run_layer(const LayerInt8Args& b, hipStream_t st) {
  const LayerArgs& a = b.a;
  QuantArgs q{};
  q.rows = a.S; q.n = a.d; q.dtype = a.dtype; q.x = a.x; q.q = b.qx; q.scale = b.sx;
  hipError_t err = launch_quantize(q, st);
  if (err != hipSuccess) return err;
  if ((err = strips<T, true>(b, st)) != hipSuccess) return err;
  q.rows = static_cast<int64_t>(a.S) * a.k; q.n = a.h; q.x = a.hidden; q.q = b.qh; q.scale = b.sh;
  if ((err = launch_quantize(q, st)) != hipSuccess) return err;
  if ((err = strips<T, false>(b, st)) != hipSuccess) return err;
  layer_int8_combine_kernel<T><<<dim3((a.d + 4 * kBlock - 1) / (4 * kBlock), a.S), kBlock, 0, st>>>(b);
  return hipGetLastError();
}

}  // namespace

// Blocks along the second matrix's K: enough that two per CU run, a step for each wave at least.
int layer_int8_splits(const LayerArgs& a) {
  const int64_t blocks = static_cast<int64_t>(slots(a)) * ((a.d + kInt8Strip - 1) / kInt8Strip);
  const int64_t most = a.h / (kInt8Step * kInt8Waves);
  return static_cast<int>(std::max<int64_t>(1, std::min<int64_t>({8, most, 512 / std::max<int64_t>(1, blocks)})));
}

hipError_t launch_layer_int8(const LayerInt8Args& b, hipStream_t st) {
  return b.a.dtype == 1 ? run_layer<bf16_t>(b, st) : run_layer<float>(b, st);
}

}  // namespace hetumoe
