// The layer for a few tokens with weights in 8-bit integers.
//
// As layer.hip: the weights' bytes are what there is to read, a block streams a strip of one
// expert's matrix past all rows that chose it.  The matrix's rows are the product's columns and run
// along K, so 16 bytes of one are a lane's part of a matrix-core operand: 16 rows of the
// matrix are one operand, 16 tokens the other.  A block's waves take ranges of K and add their
// sums, which are exact, in LDS; K of the second product is also split over blocks.
// Tokens and hidden rows are quantized by launches of their own, since a row's scale needs all of it, or,
// few rows, by every block that reads them.
#include <algorithm>

#include "experts.hpp"
#include "int8.hpp"
#include "layer_choices.hpp"
#include "layer_int8_rows.hpp"

namespace hetumoe {

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int kInt8Tiles = 4;                  // of 16 rows of the matrix per block
constexpr int kInt8Strip = 16 * kInt8Tiles;
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

// The same of tokens in LDS, whose places the block has filled.
__device__ __forceinline__ void int8_tokens(unsigned at, i32x4 (&f)[4]) {
  asm volatile(
      "ds_read_b128 %0, %4\n\tds_read_b128 %1, %5\n\tds_read_b128 %2, %6\n\tds_read_b128 %3, %7\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(f[0]), "=&v"(f[1]), "=&v"(f[2]), "=&v"(f[3])
      : "v"(at), "v"(at + 64), "v"(at + 128), "v"(at + 192)
      : "memory");
}

__device__ __forceinline__ unsigned lds_address(const void* p) {
  return static_cast<unsigned>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const char*)(p)));
}

// Sums of the strip with MT tiles of 16 tokens over steps lo .. hi - 1 of K.  HELD: the tokens lie in
// LDS already, else they come with the matrix.
template <int MT, bool HELD>
struct Int8Sums {
  static constexpr int kTokens = HELD ? 0 : MT;       // stages of tokens
  static constexpr int kStages = kTokens + kInt8Tiles;  // per step
  i32x4 acc[MT][kInt8Tiles];
  __amdgpu_buffer_rsrc_t w0, w1;  // the matrix from the strip's first row on: of the first and the other half of its tiles
  __amdgpu_buffer_rsrc_t x;
  int pitch, K, lo, hi;
  int xrow[MT][4];                // byte of the row of tile i that the lane fetches in load q, or kExpertOob
  char* ring;

  // Stage s of step st, to place p; behind the last step: zeros, so that the count of loads stays.  Load
  // q of a stage: rows 4 q + g.
  __device__ __forceinline__ void load(int s, int st, int p) const {
    const int lane = lane_id(), g = lane / 16, m = lane % 16;
    char* dst = ring + p * kInt8Stage;
    const int k = st * kInt8Step, j = s - kTokens;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int piece = (m ^ (4 * q + g)) * 16;
      const bool in = st < hi && k + piece < K;
      if (s < kTokens) {
        const int row = xrow[s < MT ? s : 0][q];
        __builtin_amdgcn_raw_ptr_buffer_load_lds(x, (lds_void*)(dst + q * 1024), 16,
                                                 in && row != kExpertOob ? row + k + piece : kExpertOob, 0, 0, 0);
      } else {
        // non-temporal: a strip is read once
        const int off = in ? (j % (kInt8Tiles / 2) * 16 + 4 * q + g) * pitch + piece + k : kExpertOob;
        if (j < kInt8Tiles / 2) __builtin_amdgcn_raw_ptr_buffer_load_lds(w0, (lds_void*)(dst + q * 1024), 16, off, 0, 0, 2);
        else __builtin_amdgcn_raw_ptr_buffer_load_lds(w1, (lds_void*)(dst + q * 1024), 16, off, 0, 0, 2);
      }
    }
  }

  // The first stages.
  __device__ __forceinline__ void begin() {
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < kInt8Tiles; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
#pragma unroll
    for (int s = 0; s < kInt8Ring; ++s) load(s % kStages, lo + s / kStages, s);
  }

  // HELD: token row m lies at `tokens`, the steps from `first` on, for m < n.
  __device__ __forceinline__ void finish(unsigned tokens, int first, int n) {
    const int lane = lane_id(), g = lane / 16, m = lane % 16;
    const unsigned at = lds_address(ring) + m * kInt8Step + (g ^ m) * 16;
    i32x4 xf[MT][4];
    int taken = 0;  // stages: the next one lies at place taken % 4
    for (int st = lo; st < hi; ++st) {
      if constexpr (HELD) {
        int8_tokens(tokens + (st - first) * kInt8Step + g * 16, xf[0]);
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
          for (int q = 0; q < 4; ++q) xf[0][u][q] = m < n ? xf[0][u][q] : 0;
      }
#pragma unroll
      for (int s = 0; s < kStages; ++s) {
        const int p = taken++ % kInt8Ring;
        if (s < kTokens) {
          int8_operands(at + p * kInt8Stage, xf[s < MT ? s : 0]);
        } else {
          i32x4 wf[4];
          int8_operands(at + p * kInt8Stage, wf);
#pragma unroll
          for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int i = 0; i < MT; ++i)
              acc[i][s < kTokens ? 0 : s - kTokens] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wf[u], xf[i][u], acc[i][s < kTokens ? 0 : s - kTokens], 0, 0, 0);
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

// Row `row` of K elements of T quantized by the block: its bytes p0 .. p0 + bytes - 1 (zeros behind K) to
// `to`; returns the scale.  `most`: LDS of a value per wave, not in use by other rows.  between() runs while
// the row is on its way.
template <class T, class Fn>
__device__ __forceinline__ float int8_hold(const T* row, int K, int p0, int bytes, char* to, int* most, Fn between) {
  constexpr int N = 16 / Chunk<T>::kElems, kThreads = kInt8Waves * kWave, kPieces = kInt8HeldK / 16 / kThreads;
  const __amdgpu_buffer_rsrc_t r = expert_rsrc(row, K * static_cast<int>(sizeof(T)));
  u32x4 v[kPieces][N];
#pragma unroll
  for (int i = 0; i < kPieces; ++i)
#pragma unroll
    for (int q = 0; q < N; ++q)  // zeros behind the row
      v[i][q] = __builtin_amdgcn_raw_buffer_load_b128(
          r, (i * kThreads + static_cast<int>(threadIdx.x)) * 16 * static_cast<int>(sizeof(T)) + 16 * q, 0, 0);
  __builtin_amdgcn_sched_barrier(0);
  between();
  __builtin_amdgcn_sched_barrier(0);
  MostOf<T> running;
#pragma unroll
  for (int i = 0; i < kPieces; ++i)
#pragma unroll
    for (int q = 0; q < N; ++q) running.take(v[i][q]);
  int a = group_reduce<kWave>(running.bits(), OpMaxI());
  if (lane_id() == 0) most[threadIdx.x / kWave] = a;
  expert_stage_barrier<63>();  // the stages on their way need not arrive
#pragma unroll
  for (int w = 0; w < kInt8Waves; ++w) a = max(a, most[w]);
  const Quantizer quant(a);
#pragma unroll
  for (int i = 0; i < kPieces; ++i) {
    const int k = (i * kThreads + static_cast<int>(threadIdx.x)) * 16 - p0;
    if (k >= 0 && k < bytes) *reinterpret_cast<u32x4*>(to + k) = quantize_piece<T>(quant, v[i]);
  }
  return quant.scale;
}

// One strip of an expert's matrix past its rows, MT tiles of them at a time, passes dealt to
// `shares` blocks.  FIRST: hidden (T), else partial integer sums.  HELD: the block quantizes its few rows
// itself (x or hidden in T) while its first stages are on their way, else they were before.
template <class T, int MT, bool FIRST, bool GATED, bool HELD>
__global__ __launch_bounds__(kInt8Waves* kWave, 2) void layer_int8_kernel(LayerInt8Args b, int shares) {
  constexpr bool kSplit = FIRST && GATED;  // half of the strip's rows are the gate's
  constexpr int NBO = kSplit ? kInt8Strip / 2 : kInt8Strip;
  constexpr int kPitch = kInt8Strip + 4, kThreads = kInt8Waves * kWave;
  // the waves' rings; then, in the same places, a tile of sums of each
  __shared__ __align__(1024) char ring[kInt8Waves][kInt8Ring * kInt8Stage];
  static_assert(16 * kPitch * 4 <= kInt8Ring * kInt8Stage, "room for a tile");
  __shared__ __align__(16) char tokens[HELD ? kInt8HeldBytes : 16];
  __shared__ float token_scale[kInt8HeldRows];
  __shared__ int most[kInt8HeldRows][kInt8Waves];
  __shared__ int lists[HELD ? kInt8Waves * kWave : kLayerMaxChoices];  // HELD: a list per wave
  __shared__ int wave_n[kInt8Waves];
  const LayerArgs& a = b.a;
  const int tid = threadIdx.x, g = lane_id() / 16;
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  int e, n;
  const int* list;
  if (!layer_choices<kInt8Waves>(a, lists, wave_n, e, n, list)) return;
  e = __builtin_amdgcn_readfirstlane(e);
  n = __builtin_amdgcn_readfirstlane(n);
  const int share = blockIdx.z % shares, z = blockIdx.z / shares, zs = gridDim.z / shares;
  const int K = FIRST ? a.d : a.h;
  const int per = layer_int8_steps(K, zs), first = z * kInt8Waves * per;
  const int bytes = layer_int8_row_bytes(K, zs);               // HELD: of a row, from step `first` on
  const int pass = HELD ? layer_int8_held_rows(bytes) : 16 * MT;  // rows at a time
  if (n <= pass * share) return;

  const int N = FIRST ? a.h : a.d, N1 = kSplit ? 2 * N : N;
  const int n0 = blockIdx.x * NBO;
  const int8_t* w = reinterpret_cast<const int8_t*>(FIRST ? a.w1 : a.w2) + (static_cast<int64_t>(e) * N1 + n0) * K;
  // rows of the matrix behind N: zeros
  const int half = kSplit ? NBO : NBO / 2;
  const int64_t apart = static_cast<int64_t>(kSplit ? N : half) * K;
  const int v0 = min(half, N - n0), v1 = kSplit ? v0 : max(0, min(half, N - n0 - half));
  const int steps = (K + kInt8Step - 1) / kInt8Step;
  Int8Sums<MT, HELD> sums;
  sums.w0 = expert_rsrc(w, __builtin_amdgcn_readfirstlane(v0 * K));
  sums.w1 = expert_rsrc(w + apart, __builtin_amdgcn_readfirstlane(v1 * K));
  sums.x = expert_rsrc(FIRST ? b.qx : b.qh, (FIRST ? a.S : a.S * a.k) * K);
  sums.pitch = sums.K = K;
  sums.lo = first + wave * per;
  sums.hi = min(steps, sums.lo + per);
  sums.ring = ring[wave];

  for (int r0 = pass * share; r0 < n; r0 += pass * shares) {
    const int end = min(n, r0 + pass);
    if constexpr (HELD) {
      const int held = end - r0;
      for (int r = 0; r < held; ++r) {
        const int64_t row = __builtin_amdgcn_readfirstlane(FIRST ? list[r0 + r] / a.k : list[r0 + r]);
        const float scale = int8_hold(reinterpret_cast<const T*>(FIRST ? a.x : a.hidden) + row * K, K, first * kInt8Step, bytes,
                                      tokens + r * bytes, most[r], [&]() { if (r == 0) sums.begin(); });
        if (tid == 0) token_scale[r] = scale;
        if (!FIRST && tid == 0 && blockIdx.x == 0 && z == 0) b.sh[row] = scale;
      }
      expert_stage_barrier<63>();
      const int m = min(static_cast<int>(lane_id() % 16), held - 1);
      sums.finish(lds_address(tokens) + m * bytes, first, held);
    } else {
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int li = r0 + 16 * i + 4 * q + g;
          sums.xrow[i][q] = li < n ? (FIRST ? list[li] / a.k : list[li]) * K : kExpertOob;
        }
      sums.begin();
      sums.finish(0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      if (r0 + 16 * i >= n) break;
      sums.put(reinterpret_cast<int*>(ring[wave]), i);
      __syncthreads();
      for (int o = tid; o < (HELD ? kInt8HeldRows : 16) * NBO; o += kThreads) {
        const int row = o / NBO, c = o % NBO, li = r0 + 16 * i + row;
        if (li >= end || n0 + c >= N) continue;
        int v = 0, u = 0;
#pragma unroll
        for (int q = 0; q < kInt8Waves; ++q) {
          const int* red = reinterpret_cast<const int*>(ring[q]) + row * kPitch + c;
          v += red[0];
          if constexpr (kSplit) u += red[NBO];
        }
        const int choice = list[li];
        if constexpr (FIRST) {
          const float sx = HELD ? token_scale[row] : b.sx[choice / a.k];
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
// Two choices and four parts of each are requested together: with one block per 256 columns it is
// their latency that counts (one token, two choices, four parts: 7.0 -> 4.5 us).
template <class T>
__global__ __launch_bounds__(kWave) void layer_int8_combine_kernel(LayerInt8Args b) {
  const LayerArgs& a = b.a;
  const int s = blockIdx.y, c = (blockIdx.x * kWave + threadIdx.x) * 4;
  if (c >= a.d) return;
  const int64_t choices = static_cast<int64_t>(a.S) * a.k;
  const int* part = reinterpret_cast<const int*>(a.part);
  f32x4 y = {0.f, 0.f, 0.f, 0.f};
  for (int r0 = 0; r0 < a.k; r0 += 2) {
    int e[2];
    float w[2], sh[2];
    i32x4 v[2];
    f32x4 s2[2], b2[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int64_t ch = static_cast<int64_t>(s) * a.k + min(r0 + i, a.k - 1);
      e[i] = r0 + i < a.k ? a.ids[ch] : -1;
      w[i] = a.weights[ch];
      sh[i] = b.sh[ch];
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int64_t ch = static_cast<int64_t>(s) * a.k + min(r0 + i, a.k - 1);
      const bool in = e[i] >= 0 && e[i] < a.E;
      const int64_t at = static_cast<int64_t>(in ? e[i] : 0) * a.d + c;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        s2[i][q] = b.s2[at + q];
        b2[i][q] = a.b2 ? a.b2[at + q] : 0.f;
      }
      v[i] = i32x4{0, 0, 0, 0};
      if (!in) continue;
      for (int z0 = 0; z0 < a.z2; z0 += 4) {
        i32x4 p[4];
#pragma unroll
        for (int z = 0; z < 4; ++z) p[z] = *reinterpret_cast<const i32x4*>(part + (min(z0 + z, a.z2 - 1) * choices + ch) * a.d + c);
#pragma unroll
        for (int z = 0; z < 4; ++z)
          if (z0 + z < a.z2) v[i] += p[z];
      }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if (e[i] < 0 || e[i] >= a.E) continue;  // padding adds nothing, whatever lies there
#pragma unroll
      for (int q = 0; q < 4; ++q) y[q] += w[i] * (static_cast<float>(v[i][q]) * sh[i] * s2[i][q] + b2[i][q]);
    }
  }
  T* out = reinterpret_cast<T*>(a.y) + static_cast<int64_t>(s) * a.d + c;
  if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(out) = uint2{pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3])};
  else *reinterpret_cast<f32x4*>(out) = y;
}

int slots(const LayerArgs& a) { return a.by_choice ? a.S * a.k : a.E; }

// Whether the strips' blocks quantize their rows themselves, which saves two launches: a few tokens, or no
// more choices than experts (32 tokens, two of 64 experts of 2048 x 2048, gated: 106 -> 100 us; two of
// 32 of 1024 x 2048, twice as many rows per expert: 56 -> 62).
bool held(const LayerArgs& a, bool first, int z) {
  static_assert(kWave == 64, "a wave lists all choices");
  return layer_int8_held(a.S, a.k, a.by_choice != 0, first ? a.d : a.h, z);
}

template <class T, int MT, bool FIRST, bool HELD>
hipError_t strip(const LayerInt8Args& b, int z, hipStream_t st) {
  const LayerArgs& a = b.a;
  const int N = FIRST ? a.h : a.d, nbo = FIRST && a.gated ? kInt8Strip / 2 : kInt8Strip;
  const int64_t strips = (N + nbo - 1) / nbo, blocks = strips * slots(a) * z;
  const int pass = HELD ? layer_int8_held_rows(layer_int8_row_bytes(FIRST ? a.d : a.h, z)) : 16 * MT;
  const int passes = (a.S + pass - 1) / pass;
  const int shares = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(passes, 512 / blocks)));
  const dim3 grid(static_cast<unsigned>(strips), slots(a), z * shares);
  constexpr int kThreads = kInt8Waves * kWave;
  if (FIRST && a.gated) layer_int8_kernel<T, MT, FIRST, true, HELD><<<grid, kThreads, 0, st>>>(b, shares);
  else layer_int8_kernel<T, MT, FIRST, false, HELD><<<grid, kThreads, 0, st>>>(b, shares);
  return hipGetLastError();
}

// Tokens (x) or hidden rows quantized, and the strips.
template <class T, bool FIRST>
hipError_t strips(const LayerInt8Args& b, hipStream_t st) {
  const LayerArgs& a = b.a;
  const int z = FIRST ? 1 : a.z2;
  if (held(a, FIRST, z)) return strip<T, 1, FIRST, true>(b, z, st);
  QuantArgs q{};
  q.dtype = a.dtype;
  if (FIRST) {
    q.rows = a.S; q.n = a.d; q.x = a.x; q.q = b.qx; q.scale = b.sx;
  } else {
    q.rows = static_cast<int64_t>(a.S) * a.k; q.n = a.h; q.x = a.hidden; q.q = b.qh; q.scale = b.sh;
  }
  const hipError_t err = launch_quantize(q, st);
  if (err != hipSuccess) return err;
  // token tiles in registers for about twice the mean rows of an expert
  const int64_t rows = std::min<int64_t>(a.S, 2 * ((static_cast<int64_t>(a.S) * a.k + a.E - 1) / a.E));
  if (rows <= 16) return strip<T, 1, FIRST, false>(b, z, st);
  if (rows <= 32) return strip<T, 2, FIRST, false>(b, z, st);
  return strip<T, 4, FIRST, false>(b, z, st);
}

template <class T>
hipError_t run_layer(const LayerInt8Args& b, hipStream_t st) {
  const LayerArgs& a = b.a;
  hipError_t err = strips<T, true>(b, st);
  if (err != hipSuccess) return err;
  if ((err = strips<T, false>(b, st)) != hipSuccess) return err;
  layer_int8_combine_kernel<T><<<dim3((a.d + 4 * kWave - 1) / (4 * kWave), a.S), kWave, 0, st>>>(b);
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
