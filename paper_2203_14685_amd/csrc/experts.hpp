// Expert networks (step 4 of Algorithm 1): argument blocks, activations and the
// pieces that the tiled products of both element types share.
//
//   pre = xe w1 + b1,  hidden = act(pre)  or, gated, act(pre[:, :h]) * pre[:, h:],
//   ye = hidden w2 + b2
// and its gradients are six batched products D[m, n] = sum_k A(m, k) B(n, k), one
// matrix pair per expert, whose operands lie in memory in one of two ways:
//   kRows   row m holds its K elements next to each other (xe, hidden, dye, dpre as
//           left operands; both weights in the products with a transposed weight)
//   kCols   row k holds the elements of all m (both weights in the forward products;
//           both operands of the weight gradients, where K is the expert's rows)
#pragma once

#include "common.hpp"
#include "kernels.hpp"
#include "philox.hpp"

namespace hetumoe {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __attribute__((address_space(3))) void lds_void;

constexpr int kRows = 0, kCols = 1;
constexpr int kExpertOob = 0x7ffffff0;  // offset past every buffer resource: loads return zeros

// What becomes of the product.
constexpr int kEpiStore = 0;    // + bias, rounded once
constexpr int kEpiAct = 1;      // + bias: pre (optional); hidden
constexpr int kEpiActGrad = 2;  // dhidden: times the activation's gradient -> dpre; column sums of it
constexpr int kEpiActDrop = 3, kEpiActGradDrop = 4;  // kEpiAct and kEpiActGrad with dropout of hidden
// Products of 8-bit integers (bf16 units of two), times row and column scales, + bias: rounded
// once to bf16 or stored in fp32; with the activation (never `pre`).
constexpr int kEpiInt8 = 5, kEpiInt8Act = 6, kEpiInt8F32 = 7, kEpiInt8ActF32 = 8;
constexpr bool expert_int8(int epi) { return epi >= kEpiInt8; }
constexpr bool expert_int8_f32(int epi) { return epi >= kEpiInt8F32; }
constexpr bool expert_acts(int epi) {
  return epi == kEpiAct || epi == kEpiActDrop || epi == kEpiInt8Act || epi == kEpiInt8ActF32;
}
constexpr bool expert_act_grads(int epi) { return epi == kEpiActGrad || epi == kEpiActGradDrop; }
constexpr bool expert_drops(int epi) { return epi == kEpiActDrop || epi == kEpiActGradDrop; }

// gfx950's LDS transpose read (ds_read_b64_tr_b16): within each group of 16
// lanes, lane i receives element i % 4 of the four-element pieces addressed by
// lanes i / 4 + 4 j, j = 0..3.
__device__ __forceinline__ uint2 expert_tr16(const bf16_t* p) {
  return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p)));
}

// Loads straight into LDS: lane l's 16 bytes at `off` go to dst + 16 l; offsets
// past the resource bring zeros.
__device__ __forceinline__ void expert_dma(__amdgpu_buffer_rsrc_t r, void* dst, int off) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void*)(dst), 16, off, 0, 0, 0);
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t expert_rsrc(const void* p, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, bytes, 0x00020000);
}

// At most VM of this wave's loads to LDS are still on their way and every LDS read has
// returned; after the barrier that holds for the whole block.
template <int VM = 0>
__device__ __forceinline__ void expert_stage_barrier() {
  __builtin_amdgcn_s_waitcnt(0x0070 | (VM & 15) | ((VM >> 4) << 14));  // vmcnt(VM) lgkmcnt(0)
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// ---------------------------------------------------------------- operands
// Bytes of a row that runs along K in one stage, a cache line (with 64 bytes and twice the
// stages the L2's requests bound the products: dxe of 64 x 512 x 2048 x 8192 841 -> 958 us),
// and its K elements.
constexpr int kExpertRow = 128;
template <class T> constexpr int kExpertBk = kExpertRow / static_cast<int>(sizeof(T));
// Elements of a 16-byte piece.
template <class T> constexpr int kExpertPe = 16 / static_cast<int>(sizeof(T));

// Which 16-byte piece of its row lies at place `c` of LDS row `row`: piece c ^ swz.
//   kRows: 8 pieces per 128-byte row; two rows fill the 64 banks.  A fragment read takes rows
//          r .. r + 15 or, of the right operand in fp32, 4 i + t (with W = 32: 2 i + t), i = 0..15,
//          in some order.
//   kCols: bf16: a transpose read takes k rows 8 g + 4 h + 0..3, g = 0..3, of each 32
//          contiguous bytes; fp32 reads run along a row and need no other order.
template <class T, int KIND, bool RIGHT, int W>
__device__ __forceinline__ int expert_swz(int row) {
  if constexpr (KIND == kRows) return (RIGHT && sizeof(T) == 4 && W > 32 ? row >> 2 : row >> 1) & 7;
  else if constexpr (sizeof(T) == 4) return 0;
  else if constexpr (W >= 128) return ((row & 3) << 1) | (row & 8);
  else return (((row >> 1) & 1) << 1) | ((row & 8) >> 1);
}

// Keeps what is computed from v inside the loop: a sum or exclusive-or per use instead
// of a register held for each.
template <class V>
__device__ __forceinline__ V expert_opaque(V v) {
  asm volatile("" : "+v"(v));
  return v;
}

// One operand's loads: W rows (kRows) or columns (kCols) of the tile.
template <class T, int KIND, bool RIGHT, int W, int WAVES, int BK = kExpertBk<T>>
struct ExpertOperand {
  static constexpr int kBk = BK, kPe = kExpertPe<T>, kElt = static_cast<int>(sizeof(T));
  static constexpr int kBytes = W * BK * kElt;
  static_assert(KIND == kCols || BK == kExpertBk<T>, "whole cache lines along K");
  static constexpr int N = kBytes / 1024 / WAVES;  // loads per wave and stage
  static_assert(N * WAVES * 1024 == kBytes, "whole loads");
  static constexpr int P = KIND == kRows ? kExpertRow / 16 : W / kPe;  // pieces per LDS row
  static constexpr int R = 64 / P;                       // rows per load
  // a lane's rows are R * WAVES apart, which must not change the order of their pieces
  static_assert((KIND == kCols && kElt == 4) ||
                    R * WAVES % (KIND == kRows && RIGHT && kElt == 4 && W > 32 ? 32 : 16) == 0,
                "one order of the pieces per lane");
  const char* base;   // (first row or column, k = 0), moved on by the stages
  int rows;           // kRows: bytes behind base that may be read
  int pitch;          // bytes per row of the matrix
  unsigned off;       // of the lane's first piece in a stage
  int kc;             // kRows: the lane's K element in a stage

  // map(piece) gives the column of the tile's piece, or -1 behind the matrix.
  template <class Map>
  __device__ __forceinline__ void init(const T* p, int ld, int first, int valid, int wave, Map map) {
    const int lane = expert_opaque(lane_id());
    const int row0 = wave * R + lane / P;
    pitch = ld * kElt;
    kc = rows = 0;
    if constexpr (KIND == kRows) {
      base = reinterpret_cast<const char*>(p + static_cast<int64_t>(first) * ld);
      rows = max(0, valid) * pitch;
      const int piece = (lane % P) ^ expert_swz<T, KIND, RIGHT, W>(row0);
      kc = piece * kPe;
      off = static_cast<unsigned>(row0 * ld * kElt + piece * 16);
    } else {
      base = reinterpret_cast<const char*>(p);
      const int col = map((lane % P) ^ expert_swz<T, KIND, RIGHT, W>(row0));
      off = col >= 0 ? static_cast<unsigned>((row0 * ld + col) * kElt) : static_cast<unsigned>(kExpertOob);
    }
  }
  // Passes over n stages.
  __device__ __forceinline__ void skip(int n) {
    base += static_cast<int64_t>(n) * (KIND == kRows ? kExpertRow : kBk * pitch);
    if constexpr (KIND == kRows) rows -= n * kExpertRow;
  }
  // The loads of the stage `base` points at; `left` K elements remain (none: zeros).  An
  // offset past the resource stays past it (below 2^32) with the rows' strides added.
  struct Stage {
    __amdgpu_buffer_rsrc_t r;
    unsigned o, stride;
    __device__ __forceinline__ void issue(T* lds, int wave, int i) const {
      expert_dma(r, reinterpret_cast<char*>(lds) + (i * WAVES + wave) * 1024, static_cast<int>(o + i * stride));
    }
  };
  __device__ __forceinline__ Stage next(int left) {
    Stage s;
    s.r = expert_rsrc(base,
                      __builtin_amdgcn_readfirstlane(KIND == kRows ? max(rows, 0) : max(0, min(left, kBk)) * pitch));
    s.stride = static_cast<unsigned>(R * WAVES) * static_cast<unsigned>(pitch);
    s.o = expert_opaque(off);
    if constexpr (KIND == kRows) s.o = kc < left ? s.o : static_cast<unsigned>(kExpertOob);
    base += KIND == kRows ? kExpertRow : kBk * pitch;
    if constexpr (KIND == kRows) rows -= kExpertRow;
    return s;
  }
  __device__ __forceinline__ void load(T* lds, int wave, int left) {
    const Stage s = next(left);
#pragma unroll
    for (int i = 0; i < N; ++i) s.issue(lds, wave, i);
  }
};

// The right operand of a gated forward product whose weights' rows run along K: of each 64 rows
// of the tile 32 are the gate's, 32 the other factor's, `apart` rows behind them.
template <class T, int W, int WAVES>
struct ExpertSplitOperand {
  static constexpr int kElt = static_cast<int>(sizeof(T));
  static constexpr int N = W * kExpertRow / 1024 / WAVES, P = kExpertRow / 16, R = 64 / P;
  static_assert(N * WAVES * 1024 == W * kExpertRow && R * WAVES >= 16, "whole loads, one order of the pieces");
  const char *gate, *other;
  int rows, pitch, kc;
  unsigned off;  // of the lane's first piece in 32 rows

  __device__ __forceinline__ void init(const T* p, int ld, int first, int valid, int apart, int wave) {
    const int lane = expert_opaque(lane_id());
    pitch = ld * kElt;
    gate = reinterpret_cast<const char*>(p + static_cast<int64_t>(first) * ld);
    other = gate + static_cast<int64_t>(apart) * pitch;
    rows = max(0, valid) * pitch;
    const int piece = (lane % P) ^ expert_swz<T, kRows, true, W>(wave * R + lane / P);
    kc = piece * kExpertPe<T>;
    off = static_cast<unsigned>(lane / P * pitch + piece * 16);
  }
  struct Stage {
    __amdgpu_buffer_rsrc_t g, u;
    unsigned o;
    int pitch;
    __device__ __forceinline__ void issue(T* lds, int wave, int i) const {
      const int row = (i * WAVES + wave) * R;  // of the tile, the same for all lanes
      const unsigned at = o + static_cast<unsigned>((row / 64 * 32 + row % 32) * pitch);
      char* dst = reinterpret_cast<char*>(lds) + (i * WAVES + wave) * 1024;
      if (row / 32 % 2 == 0) expert_dma(g, dst, static_cast<int>(at));
      else expert_dma(u, dst, static_cast<int>(at));
    }
  };
  __device__ __forceinline__ Stage next(int left) {
    Stage s;
    const int bytes = __builtin_amdgcn_readfirstlane(max(rows, 0));
    s.g = expert_rsrc(gate, bytes);
    s.u = expert_rsrc(other, bytes);
    s.o = expert_opaque(off);
    s.o = kc < left ? s.o : static_cast<unsigned>(kExpertOob);
    s.pitch = pitch;
    gate += kExpertRow;
    other += kExpertRow;
    rows -= kExpertRow;
    return s;
  }
  __device__ __forceinline__ void load(T* lds, int wave, int left) {
    const Stage s = next(left);
#pragma unroll
    for (int i = 0; i < N; ++i) s.issue(lds, wave, i);
  }
};

// ---------------------------------------------------------------- activations
// sigmoid by the hardware exponential and reciprocal.  The exponential's argument is rounded
// after its factor log2(e), so its relative error grows as |x| 2^-24 (some units of the last
// place at |x| = 10, where 1 + it has long lost them for x > 0 and the result is below 5e-5 for
// x < 0); the reciprocal is within one unit.
__device__ __forceinline__ float expert_sigmoid(float x) { return __builtin_amdgcn_rcpf(1.f + __expf(-x)); }

constexpr float kGeluA = 0.7978845608028654f;  // sqrt(2 / pi)
constexpr float kGeluB = 0.044715f;

// 0.5 (1 + tanh u) = sigmoid(2 u)
template <int ACT>
__device__ __forceinline__ float expert_act(float a) {
  if constexpr (ACT == 0) return a < 0.f ? 0.f : a;  // a NaN stays one
  else if constexpr (ACT == 2) return a * expert_sigmoid(a);
  else return a * expert_sigmoid(2.f * kGeluA * (a + kGeluB * a * a * a));
}

// The activation and its derivative.
template <int ACT>
__device__ __forceinline__ void expert_act_grad(float a, float& f, float& df) {
  if constexpr (ACT == 0) {
    f = a < 0.f ? 0.f : a;
    df = a > 0.f ? 1.f : 0.f;
  } else if constexpr (ACT == 2) {
    const float p = expert_sigmoid(a);
    f = a * p;
    df = p + f * (1.f - p);
  } else {
    const float p = expert_sigmoid(2.f * kGeluA * (a + kGeluB * a * a * a));
    f = a * p;
    // p is exactly 0 or 1 long before 1e18; past 1.8e19 the square would be infinite, 0 times it NaN
    const float c = fminf(fabsf(a), 1e18f);
    df = p + f * (1.f - p) * (2.f * kGeluA) * (1.f + 3.f * kGeluB * c * c);
  }
}

// fn(ExpertInt<ACT>()) for a run-time activation.
template <int V> struct ExpertInt { static constexpr int v = V; };
template <class Fn>
__device__ __forceinline__ void expert_by_act(int act, Fn fn) {
  if (act == 0) fn(ExpertInt<0>());
  else if (act == 2) fn(ExpertInt<2>());
  else fn(ExpertInt<1>());
}

// Rows in use of expert e.
__device__ __forceinline__ int expert_count(const int32_t* counts, int e, int C) {
  return counts ? max(0, min(counts[e], C)) : C;
}

// ---------------------------------------------------------------- tiles
// A block takes one tile after another, those of its XCD (blocks go round the 8 XCDs in
// turn).  Groups of neighbouring tiles (an expert's m tiles first: they share its
// weights, and a few n tiles its rows) go to one XCD, whose L2 then serves them, the
// groups round the XCDs in order, so that experts of any load spread evenly (64 experts of
// uneven load, one contiguous piece of the tiles per XCD: CUs busy 62 % of the time).
// Tiles without rows in use, which are only cleared, come behind all others.
//
// Only the device knows the counts, and so how many tiles there are.  Where the last round
// of tiles would leave half the CUs idle or more, a launch may leave it out (a.round); a
// second one (a.quarters) then forms its tiles as four each.
constexpr int kTileGroup = 32;
constexpr int kMaxExperts = 1024;

struct ExpertTile {
  int e, bm, bn;
};

constexpr int kTileList = 256;  // a block's next tiles, found together by its threads

template <int BM>
struct ExpertTiles {
  int nv;    // tiles with work
  int end;   // listed ones
  int from;  // quarters: the first tile's number
  int used;  // slots per XCD that serve them
  int g;     // tiles per group
  int* before;  // LDS [E]: m tiles with work up to and with each expert (where counts cut M)
  int* rows;    // LDS [E]: rows in use

  // The whole block calls this; one barrier.
  __device__ __forceinline__ void init(const ExpertGemmArgs& a, int* before_, int* rows_) {
    before = before_;
    rows = rows_;
    const int lane = lane_id();
    const int rows_per = a.quarters ? 2 * BM : BM;
    int total = 0;
    if (threadIdx.x < kWave) {
      for (int e0 = 0; e0 < a.E; e0 += kWave) {
        const int e = e0 + lane;
        const int n = e < a.E ? expert_count(a.counts, e, a.C) : 0;
        int sum = a.k_is_rows ? (e < a.E ? a.tm : 0) : (n + rows_per - 1) / rows_per;
#pragma unroll
        for (int s = 1; s < kWave; s <<= 1) {
          const int up = __shfl_up(sum, s);
          sum += lane >= s ? up : 0;
        }
        if (e < a.E) {
          before[e] = total + sum;
          rows[e] = n;
        }
        total += __builtin_amdgcn_readlane(sum, kWave - 1);
      }
    }
    __syncthreads();
    nv = __builtin_amdgcn_readfirstlane(before[a.E - 1]) * a.tn;
    end = nv;
    from = 0;
    if (a.round) {
      const int last = nv % a.round, left_out = 2 * last <= a.round ? last : 0;
      from = nv - left_out;
      end = a.quarters ? 4 * left_out : from;
    }
    g = end >= 8 * kTileGroup ? kTileGroup : end >= 8 ? (end + 7) / 8 : 1;
    used = ((end + g - 1) / g + 7) / 8 * g;
  }

  // The tile of slot j of XCD x; e = -1 behind the last one (and then for all later slots).
  __device__ __forceinline__ int4 slot_tile(const ExpertGemmArgs& a, int x, int j) const {
    const int q = j / g;
    int v = (q * 8 + x) * g + (j - q * g);
    if (j >= used || v >= end) return int4{-1, 0, 0, 0};
    const int quarter = v % 4;
    if (a.quarters) v = from + v / 4;
    int lo = 0, hi = a.E - 1;  // the first expert whose tiles end behind v
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if (before[mid] * a.tn > v) hi = mid;
      else lo = mid + 1;
    }
    const int first = lo > 0 ? before[lo - 1] : 0;
    const int mt = before[lo] - first;
    const int r = v - first * a.tn;
    if (a.quarters) return int4{lo, 2 * (r % mt) + quarter % 2, 2 * (r / mt) + quarter / 2, 0};
    return int4{lo, r % mt, r / mt, 0};
  }

  // Tile `want` of those without work.
  __device__ __forceinline__ bool clear(const ExpertGemmArgs& a, int want, ExpertTile& t) const {
    if (a.quarters || want >= a.tiles - nv) return false;
    const int lane = lane_id();
    for (int e0 = 0; e0 < a.E; e0 += kWave) {
      const int i = min(e0 + lane, a.E - 1);
      // such tiles along M up to and with expert i
      const int upto = (i + 1) * a.tm - before[i];
      const uint64_t past = __ballot(e0 + lane < a.E && upto * a.tn > want);
      if (past) {
        const int e = e0 + __builtin_ctzll(past);
        const int last = __builtin_amdgcn_readfirstlane(before[e]);
        const int first = e > 0 ? __builtin_amdgcn_readfirstlane(before[e - 1]) : 0;
        const int mt = a.tm - (last - first);
        const int r = want - (e * a.tm - first) * a.tn;
        const int bn = r / mt;
        t.e = __builtin_amdgcn_readfirstlane(e);
        t.bn = __builtin_amdgcn_readfirstlane(bn);
        t.bm = __builtin_amdgcn_readfirstlane(r - bn * mt + a.tm - mt);
        return true;
      }
    }
    return false;
  }
};

__device__ __forceinline__ bool expert_listed(const int4* list, int i, ExpertTile& t) {
  const int4 q = list[i];
  t.e = __builtin_amdgcn_readfirstlane(q.x);
  t.bm = __builtin_amdgcn_readfirstlane(q.y);
  t.bn = __builtin_amdgcn_readfirstlane(q.z);
  return t.e >= 0;
}

// The rows of a tile in a row-major matrix of `ld` columns, for 16-byte accesses at
// 32-bit offsets: those past `valid` rows, or at kExpertOob, read zeros and write nothing.
template <class T>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t expert_rows(const void* p, int64_t row0, int ld, int valid) {
  return expert_rsrc(reinterpret_cast<const T*>(p) + row0 * ld,
                     __builtin_amdgcn_readfirstlane(max(0, valid) * ld * static_cast<int>(sizeof(T))));
}

// Blocks: at most `resident`, a multiple of 8.
inline unsigned expert_blocks(int tiles, int resident) {
  const int need = (tiles + 7) / 8 * 8;
  return static_cast<unsigned>(need < resident ? need : (resident + 7) / 8 * 8);
}

}  // namespace hetumoe
