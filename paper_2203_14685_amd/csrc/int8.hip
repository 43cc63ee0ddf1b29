// Rows and weights as 8-bit integers with a scale each.
//
// Rows: bound by memory, one read and half (bf16) or a quarter (fp32) of it written; a row's
// threads hold it in registers between its maximum and its quantization (218 million bf16
// in use in rows of 2048: 121 to 128 us, 5.1 to 5.4 TB/s; with a test per element for quotients on a border 137).
// Weights: once, when they are loaded: a pass for the columns' maxima, one that quantizes and transposes.
#include <algorithm>

#include "int8.hpp"
#include "kernels.hpp"

namespace hetumoe {

namespace {

constexpr int kPiece = 16;  // elements that a thread takes at a time: 16 bytes of integers

// TPR threads per row; the first HELD pieces of each stay in registers, those of longer rows
// are read again.
template <class T, int TPR, int HELD>
__global__ __launch_bounds__(kBlock) void quantize_rows_kernel(QuantArgs a) {
  __shared__ int wave_most[kWavesPerBlock];
  constexpr int PE = Chunk<T>::kElems, N = kPiece / PE;
  const int64_t row = long_block() * (kBlock / TPR) + threadIdx.x / TPR;
  const int lane = threadIdx.x % TPR;
  bool in = row < a.rows;
  if (in && a.counts) {
    const int e = static_cast<int>(row / a.C);
    in = row - static_cast<int64_t>(e) * a.C < a.counts[e];
  }
  const T* x = static_cast<const T*>(a.x) + (in ? row : 0) * a.n;
  const int pieces = in ? a.n / kPiece : 0;
  u32x4 held[HELD][N];
  MostOf<T> running;
#pragma unroll
  for (int i = 0; i < HELD; ++i) {
    const int p = lane + i * TPR;
#pragma unroll
    for (int q = 0; q < N; ++q)
      held[i][q] = p < pieces ? reinterpret_cast<const u32x4*>(x + p * kPiece)[q] : u32x4{0, 0, 0, 0};
  }
#pragma unroll
  for (int i = 0; i < HELD; ++i)
#pragma unroll
    for (int q = 0; q < N; ++q) running.take(held[i][q]);
  for (int p = lane + HELD * TPR; p < pieces; p += TPR)
#pragma unroll
    for (int q = 0; q < N; ++q) running.take(reinterpret_cast<const u32x4*>(x + p * kPiece)[q]);
  int most = group_reduce<(TPR < kWave ? TPR : kWave)>(running.bits(), OpMaxI());
  if constexpr (TPR > kWave) {
    static_assert(TPR == kBlock, "a row per block");
    if (lane_id() == 0) wave_most[threadIdx.x / kWave] = most;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWavesPerBlock; ++w) most = max(most, wave_most[w]);
  }
  if (!in) {
    if (a.clear && row < a.rows) {
      u32x4* p = reinterpret_cast<u32x4*>(static_cast<char*>(a.clear) + row * a.clear_bytes);
      for (int i = lane; i < a.clear_bytes / 16; i += TPR) p[i] = u32x4{0, 0, 0, 0};
    }
    return;
  }
  const Quantizer quant(most);
  int8_t* out = a.q + row * a.n;
  auto put = [&](const u32x4 (&v)[N], int p) __attribute__((always_inline)) {
    *reinterpret_cast<u32x4*>(out + p * kPiece) = quantize_piece<T>(quant, v);
  };
#pragma unroll
  for (int i = 0; i < HELD; ++i) {
    const int p = lane + i * TPR;
    if (p < pieces) put(held[i], p);
  }
  for (int p = lane + HELD * TPR; p < pieces; p += TPR) {
    u32x4 v[N];
#pragma unroll
    for (int q = 0; q < N; ++q) v[q] = reinterpret_cast<const u32x4*>(x + p * kPiece)[q];
    put(v, p);
  }
  if (lane == 0) a.scale[row] = quant.scale;
}

template <class T>
hipError_t run_rows(const QuantArgs& a, hipStream_t st) {
  auto grid = [&](int tpr) { return long_grid((a.rows + kBlock / tpr - 1) / (kBlock / tpr)); };
  const int pieces = a.n / kPiece;
  if (pieces <= 16) quantize_rows_kernel<T, 16, 1><<<grid(16), kBlock, 0, st>>>(a);
  else if (pieces <= 64) quantize_rows_kernel<T, 64, 1><<<grid(64), kBlock, 0, st>>>(a);
  else if (pieces <= 128) quantize_rows_kernel<T, 64, 2><<<grid(64), kBlock, 0, st>>>(a);
  else if (pieces <= 256) quantize_rows_kernel<T, 256, 1><<<grid(256), kBlock, 0, st>>>(a);
  else quantize_rows_kernel<T, 256, 4><<<grid(256), kBlock, 0, st>>>(a);
  return hipGetLastError();
}

// ---------------------------------------------------------------- weights
__global__ __launch_bounds__(kBlock) void quantize_clear_kernel(int* most, int64_t n) {
  const int64_t i = long_block() * kBlock + threadIdx.x;
  if (i < n) most[i] = 0;
}

// Largest |w| of 16 pieces of columns over kMostRows rows; maxima are the same in any order.
constexpr int kMostRows = 256;
template <class T>
__global__ __launch_bounds__(kBlock) void quantize_most_kernel(const T* w, int* most, int K, int N) {
  constexpr int PE = Chunk<T>::kElems;
  __shared__ int lds[16][16 * PE + 1];
  const int l = threadIdx.x % 16, r = threadIdx.x / 16, e = blockIdx.z;
  const int strips = (N + 16 * PE - 1) / (16 * PE);
  const int strip = blockIdx.x % strips, k0 = static_cast<int>(blockIdx.x / strips) * kMostRows;
  const int c = (strip * 16 + l) * PE;
  int m[PE];
#pragma unroll
  for (int j = 0; j < PE; ++j) m[j] = 0;
  if (c < N) {
    for (int k = k0 + r; k < min(K, k0 + kMostRows); k += 16) {
      float f[PE];
      Chunk<T>::unpack(*reinterpret_cast<const u32x4*>(w + (static_cast<int64_t>(e) * K + k) * N + c), f);
#pragma unroll
      for (int j = 0; j < PE; ++j) m[j] = max(m[j], abs_bits(f[j]));
    }
  }
#pragma unroll
  for (int j = 0; j < PE; ++j) lds[r][l * PE + j] = m[j];
  __syncthreads();
  for (int i = threadIdx.x; i < 16 * PE; i += kBlock) {
    const int col = strip * 16 * PE + i;
    if (col >= N) continue;
    int v = 0;
#pragma unroll
    for (int q = 0; q < 16; ++q) v = max(v, lds[q][i]);
    atomicMax(most + static_cast<int64_t>(e) * N + col, v);
  }
}

// A tile of 64 rows x 64 columns, through LDS.
template <class T>
__global__ __launch_bounds__(kBlock) void quantize_turn_kernel(const T* w, const int* most, int8_t* q, int K, int N) {
  constexpr int PE = Chunk<T>::kElems, kTile = 64;
  __shared__ __align__(16) int8_t lds[kTile][kTile + 16];  // [column][row]
  const int e = blockIdx.z, tn = (N + kTile - 1) / kTile;
  const int n0 = static_cast<int>(blockIdx.x % tn) * kTile, k0 = static_cast<int>(blockIdx.x / tn) * kTile;
  constexpr int P = kTile / PE;  // pieces of a row
  const int piece = threadIdx.x % P, c = n0 + piece * PE;
  if (c < N) {
    for (int r = threadIdx.x / P; r < kTile && k0 + r < K; r += kBlock / P) {
      float f[PE];
      Chunk<T>::unpack(*reinterpret_cast<const u32x4*>(w + (static_cast<int64_t>(e) * K + k0 + r) * N + c), f);
#pragma unroll
      for (int j = 0; j < PE; ++j)
        lds[piece * PE + j][r] = static_cast<int8_t>(Quantizer(most[static_cast<int64_t>(e) * N + c + j])(f[j]));
    }
  }
  __syncthreads();
  const int col = threadIdx.x / 4, k = threadIdx.x % 4 * 16;
  if (n0 + col < N && k0 + k < K)
    *reinterpret_cast<u32x4*>(q + (static_cast<int64_t>(e) * N + n0 + col) * K + k0 + k) =
        *reinterpret_cast<const u32x4*>(&lds[col][k]);
}

// The maxima become scales.
__global__ __launch_bounds__(kBlock) void quantize_scale_kernel(float* scale, int64_t n) {
  const int64_t i = long_block() * kBlock + threadIdx.x;
  if (i < n) scale[i] = Quantizer(abs_bits(scale[i])).scale;
}

template <class T>
hipError_t run_weights(int E, int K, int N, const T* w, int8_t* q, float* scale, hipStream_t st) {
  const int64_t n = static_cast<int64_t>(E) * N;
  int* most = reinterpret_cast<int*>(scale);  // as integers until the end
  const dim3 all = long_grid((n + kBlock - 1) / kBlock);
  quantize_clear_kernel<<<all, kBlock, 0, st>>>(most, n);
  const int strip = 16 * Chunk<T>::kElems;
  const unsigned strips = static_cast<unsigned>((N + strip - 1) / strip), ranges = static_cast<unsigned>((K + kMostRows - 1) / kMostRows);
  quantize_most_kernel<T><<<dim3(strips * ranges, 1, E), kBlock, 0, st>>>(w, most, K, N);
  const unsigned tn = static_cast<unsigned>((N + 63) / 64), tk = static_cast<unsigned>((K + 63) / 64);
  quantize_turn_kernel<T><<<dim3(tn * tk, 1, E), kBlock, 0, st>>>(w, most, q, K, N);
  quantize_scale_kernel<<<all, kBlock, 0, st>>>(scale, n);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_quantize(const QuantArgs& a, hipStream_t st) {
  return a.dtype == 1 ? run_rows<bf16_t>(a, st) : run_rows<float>(a, st);
}

hipError_t launch_quantize_weights(int E, int K, int N, int dtype, const void* w, int8_t* q, float* scale, hipStream_t st) {
  return dtype == 1 ? run_weights(E, K, N, static_cast<const bf16_t*>(w), q, scale, st)
                    : run_weights(E, K, N, static_cast<const float*>(w), q, scale, st);
}

}  // namespace hetumoe
