// Expert networks: the launches of a forward and a backward pass, and the bias
// gradients (column sums).
#include "experts_launch.hpp"

namespace hetumoe {

namespace {

constexpr int kSumRows = 256;  // rows of dye summed per block

// Sums of kSumRows rows of dye: 16 lanes of one 16-byte piece each along the row, 16 row
// groups; [E, ranges, d].  Blocks along a row first, then the ranges, in one grid dimension (the
// second holds 65536).
template <class T>
__global__ __launch_bounds__(kBlock) void experts_colsum_kernel(const T* dye, const int32_t* counts, float* part, int C,
                                                                int d) {
  constexpr int PE = Chunk<T>::kElems;
  __shared__ float lds[16][16 * PE + 1];
  const int e = blockIdx.z, l = threadIdx.x % 16, r = threadIdx.x / 16;
  const int strips = (d + 16 * PE - 1) / (16 * PE), range = blockIdx.x / strips, strip = blockIdx.x - range * strips;
  const int c = (strip * 16 + l) * PE;
  const int cnt = expert_count(counts, e, C);
  const int lo = range * kSumRows, hi = min(cnt, lo + kSumRows);
  float s[PE];
#pragma unroll
  for (int q = 0; q < PE; ++q) s[q] = 0.f;
  if (c < d) {
    const T* p = dye + (static_cast<int64_t>(e) * C) * d + c;
    for (int row = lo + r; row < hi; row += 16 * 8) {
      u32x4 v[8];
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (row + 16 * u < hi) v[u] = *reinterpret_cast<const u32x4*>(p + static_cast<int64_t>(row + 16 * u) * d);
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        if (row + 16 * u >= hi) continue;
        float f[PE];
        Chunk<T>::unpack(v[u], f);
#pragma unroll
        for (int q = 0; q < PE; ++q) s[q] += f[q];
      }
    }
  }
#pragma unroll
  for (int q = 0; q < PE; ++q) lds[r][l * PE + q] = s[q];
  __syncthreads();
  for (int i = threadIdx.x; i < 16 * PE; i += kBlock) {
    const int col = strip * 16 * PE + i;
    if (col >= d) continue;
    float t = 0.f;
#pragma unroll
    for (int q = 0; q < 16; ++q) t += lds[q][i];
    part[(static_cast<int64_t>(e) * (gridDim.x / strips) + range) * d + col] = t;
  }
}

// out[e, n] = sum over p of part[e, p, n], p in order; two such sums in one launch.
struct PartSum {
  const float* part;
  float* out;
  int parts, n;
};
__global__ __launch_bounds__(kBlock) void experts_partsum_kernel(PartSum a, PartSum b, int E) {
  int64_t i = static_cast<int64_t>(blockIdx.x) * kBlock + threadIdx.x;
  const int64_t na = static_cast<int64_t>(E) * a.n;
  if (i >= na) {
    i -= na;
    a = b;
    if (i >= static_cast<int64_t>(E) * a.n) return;
  }
  const int64_t e = i / a.n, n = i - e * a.n;
  const float* p = a.part + e * a.parts * a.n + n;
  float s = 0.f;
#pragma unroll 8
  for (int q = 0; q < a.parts; ++q) s += p[static_cast<int64_t>(q) * a.n];
  a.out[i] = s;
}

hipError_t store(const ExpertArgs& x, const ExpertGemmArgs& a, int ka, int kb, hipStream_t st) {
  return x.dtype == 1 ? expert_store_bf16(x, a, ka, kb, st) : expert_store_f32(x, a, ka, kb, st);
}

}  // namespace

int expert_parts(const ExpertArgs& x) { return x.dtype == 1 ? expert_parts_bf16(x) : expert_parts_f32(x); }
int expert_row_parts(const ExpertArgs& x) { return (x.C + kSumRows - 1) / kSumRows; }

// The second product reads hidden as it is stored, rounded once to the element type, and so do dw2
// (which is then the gradient of the very ye that was computed) and every later pass over it.  In
// bf16 ye is off by 0.0023 of its size for the 0.0017 of its own rounding.  Kept as the sum
// of two bf16 (the layer for few tokens does so, behind whose weights the products hide) the second
// product has twice the terms: 64 x 2560 x 2048 x 2048 1.18 -> 2.12 ms, beside the first one's 2.48.
// fp32 rows and weights lose nothing.
hipError_t launch_experts(const ExpertArgs& x, hipStream_t st) {
  const int h1 = x.gated ? 2 * x.h : x.h;
  const int64_t dh1 = static_cast<int64_t>(x.d) * h1, hd = static_cast<int64_t>(x.h) * x.d;
  ExpertGemmArgs a = expert_base_args(x);
  a.M = x.C; a.N = x.h; a.K = x.d;
  a.A = x.xe; a.lda = x.d; a.sA = static_cast<int64_t>(x.C) * x.d;
  a.B = x.w1; a.ldb = h1; a.sB = dh1;
  a.bias = x.b1;
  a.out = x.hidden; a.ldo = x.h; a.sO = static_cast<int64_t>(x.C) * x.h;
  a.pre = x.pre;
  hipError_t err = x.dtype == 1 ? expert_act_bf16(x, a, st) : expert_act_f32(x, a, st);
  if (err != hipSuccess) return err;
  a = expert_base_args(x);
  a.M = x.C; a.N = x.d; a.K = x.h;
  a.A = x.hidden; a.lda = x.h; a.sA = static_cast<int64_t>(x.C) * x.h;
  a.B = x.w2; a.ldb = x.d; a.sB = hd;
  a.bias = x.b2;
  a.out = x.ye; a.ldo = x.d; a.sO = static_cast<int64_t>(x.C) * x.d;
  return store(x, a, kRows, kCols, st);
}

// dxe and dw1 read dpre rounded once to the element type, for the same reason (in bf16 off by 0.0024
// for 0.0017).  As the sum of two bf16: 64 x 512 x 2048 x 8192 dxe 0.92 -> 1.95 ms, dw1 1.23 -> 2.04, of
// 4.7 for all.  db1 adds the unrounded values.
hipError_t launch_experts_bwd(const ExpertArgs& x, hipStream_t st) {
  const int h1 = x.gated ? 2 * x.h : x.h;
  const int64_t dh1 = static_cast<int64_t>(x.d) * h1, hd = static_cast<int64_t>(x.h) * x.d;
  const int64_t rows_d = static_cast<int64_t>(x.C) * x.d, rows_h = static_cast<int64_t>(x.C) * x.h;
  const int64_t rows_h1 = static_cast<int64_t>(x.C) * h1;
  hipError_t err = hipSuccess;
  ExpertGemmArgs a;
  const bool rows = x.C > 0;
  if (rows && (x.dxe || x.dw1 || x.db1)) {
    a = expert_base_args(x);
    a.M = x.C; a.N = x.h; a.K = x.d;
    a.A = x.dye; a.lda = x.d; a.sA = rows_d;
    a.B = x.w2; a.ldb = x.d; a.sB = hd;
    a.pre = x.pre;
    a.out = x.dpre; a.ldo = h1; a.sO = rows_h1;
    a.colsum = x.db1 ? x.colsum : nullptr;
    err = x.dtype == 1 ? expert_actgrad_bf16(x, a, st) : expert_actgrad_f32(x, a, st);
    if (err != hipSuccess) return err;
  }
  if (rows && x.dxe) {
    a = expert_base_args(x);
    a.M = x.C; a.N = x.d; a.K = h1;
    a.A = x.dpre; a.lda = h1; a.sA = rows_h1;
    a.B = x.w1; a.ldb = h1; a.sB = dh1;
    a.out = x.dxe; a.ldo = x.d; a.sO = rows_d;
    if ((err = store(x, a, kRows, kRows, st)) != hipSuccess) return err;
  }
  if (x.dw1) {
    a = expert_base_args(x);
    a.M = x.d; a.N = h1; a.k_is_rows = 1;
    a.A = x.xe; a.lda = x.d; a.sA = rows_d;
    a.B = x.dpre; a.ldb = h1; a.sB = rows_h1;
    a.out = x.dw1; a.ldo = h1; a.sO = dh1;
    if ((err = store(x, a, kCols, kCols, st)) != hipSuccess) return err;
  }
  if (x.dw2) {
    a = expert_base_args(x);
    a.M = x.h; a.N = x.d; a.k_is_rows = 1;
    a.A = x.hidden; a.lda = x.h; a.sA = rows_h;
    a.B = x.dye; a.ldb = x.d; a.sB = rows_d;
    a.out = x.dw2; a.ldo = x.d; a.sO = hd;
    if ((err = store(x, a, kCols, kCols, st)) != hipSuccess) return err;
  }
  if (x.db1 || x.db2) {
    PartSum s1{x.colsum, x.db1, expert_parts(x), x.db1 ? h1 : 0}, s2{x.rowsum, x.db2, expert_row_parts(x), x.db2 ? x.d : 0};
    if (x.db2 && rows) {
      const int pe = x.dtype == 1 ? 8 : 4;
      const dim3 grid((x.d + 16 * pe - 1) / (16 * pe) * s2.parts, 1, x.E);
      if (x.dtype == 1)
        experts_colsum_kernel<bf16_t><<<grid, kBlock, 0, st>>>(static_cast<const bf16_t*>(x.dye), x.counts, x.rowsum, x.C, x.d);
      else
        experts_colsum_kernel<float><<<grid, kBlock, 0, st>>>(static_cast<const float*>(x.dye), x.counts, x.rowsum, x.C, x.d);
      if ((err = hipGetLastError()) != hipSuccess) return err;
    }
    const int64_t n = static_cast<int64_t>(x.E) * (s1.n + s2.n);
    experts_partsum_kernel<<<dim3(static_cast<unsigned>((n + kBlock - 1) / kBlock)), kBlock, 0, st>>>(s1, s2, x.E);
    err = hipGetLastError();
  }
  return err;
}

}  // namespace hetumoe
