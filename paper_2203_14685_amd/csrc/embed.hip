// The embedding rows that a layer starts from, and their table's gradient.
//
// Forward: a gather of rows, bound by the rows written.  Backward: the tokens are sorted by id
// (stable, so that every sum runs over its tokens in their order), then the rows' gradients are
// added in runs of equal ids: the sorted tokens are cut into chunks of equal length, one group of lanes
// per chunk and strip of columns, so the first sums take as long however the ids are spread.  A run
// inside one chunk is written at once; the parts of a run that crosses chunks go to the workspace and
// are added by a last launch, one block per run and strip, whose time does grow with the longest run's parts
// (262144 rows of 64 bf16, chunks of 8: 476 us with a run of 101073, 159 with even ids; 65536 rows of
// 512: 118 with one id on half of them, 71; of 4096 with a tenth on one: 8 of 205).  The table is cleared
// beside the sorting, whose few blocks wait for one another most of the time; rows in use are written
// again later, which is less than to find the others.
#include <algorithm>

#include "common.hpp"
#include "kernels.hpp"

namespace hetumoe {

namespace {

// ---------------------------------------------------------------- forward
// A block's threads as groups of `tpr` (a power of two) along a row, R rows per group at a time.
// NT: non-temporal stores.
template <class T, int R, bool NT>
__global__ __launch_bounds__(kBlock) void embed_kernel(const int32_t* ids, const T* table, T* y, int T_, int V, int d,
                                                       float scale, int tpr) {
  constexpr int PE = Chunk<T>::kElems;
  const int group = threadIdx.x / tpr, lane = threadIdx.x % tpr;
  const int64_t row0 = (long_block() * (kBlock / tpr) + group) * R;
  if (row0 >= T_) return;
  int id[R];
#pragma unroll
  for (int r = 0; r < R; ++r) id[r] = row0 + r < T_ ? ids[row0 + r] : -1;
  for (int c = lane * PE; c < d; c += tpr * PE) {
    u32x4 v[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const bool in = id[r] >= 0 && id[r] < V;
      v[r] = in ? *reinterpret_cast<const u32x4*>(table + static_cast<int64_t>(id[r]) * d + c) : u32x4{0, 0, 0, 0};
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (row0 + r >= T_) continue;
      const bool in = id[r] >= 0 && id[r] < V;
      float f[PE];
      Chunk<T>::unpack(v[r], f);
#pragma unroll
      for (int q = 0; q < PE; ++q) f[q] = in ? f[q] * scale : 0.f;  // zeros of padding whatever the scale's sign
      u32x4* to = reinterpret_cast<u32x4*>(y + (row0 + r) * d + c);
      if constexpr (NT) __builtin_nontemporal_store(Chunk<T>::pack(f), to);
      else *to = Chunk<T>::pack(f);
    }
  }
}

template <class T>
hipError_t run_embed(const EmbedArgs& a, hipStream_t st) {
  const int pieces = a.d / Chunk<T>::kElems;
  int tpr = 1;
  while (tpr < pieces && tpr < kBlock) tpr *= 2;
  const int groups = kBlock / tpr;
  const T* table = static_cast<const T*>(a.table);
  T* y = static_cast<T*>(a.y);
  const auto blocks = [&](int r) {
    return long_grid((a.T + static_cast<int64_t>(groups) * r - 1) / (static_cast<int64_t>(groups) * r));
  };
  // Rows that no cache holds until they are read (the Infinity Cache has 256 MB) are stored
  // non-temporally, two per group at once (65536 rows of 4096 bf16: 122 us; one 163, four 127; with
  // ordinary stores, four, 158).
  if (static_cast<int64_t>(a.T) * a.d * sizeof(T) > (int64_t(256) << 20))
    embed_kernel<T, 2, true><<<blocks(2), kBlock, 0, st>>>(a.ids, table, y, a.T, a.V, a.d, a.scale, tpr);
  else
    embed_kernel<T, 1, false><<<blocks(1), kBlock, 0, st>>>(a.ids, table, y, a.T, a.V, a.d, a.scale, tpr);
  return hipGetLastError();
}

// ---------------------------------------------------------------- sorting the tokens
// Keys: the id, V for padding (behind all others).
__device__ __forceinline__ int embed_key(const int32_t* ids, int64_t t, int V) {
  const int id = ids[t];
  return id >= 0 && id < V ? id : V;
}

// Clears a share of the table's gradient: block `block` of those of a launch.
constexpr int kClearPieces = 8;  // of 16 bytes per thread
template <int THREADS>
__device__ __forceinline__ void embed_clear(const EmbedClear& c, int64_t block) {
  u32x4* p = static_cast<u32x4*>(c.to);
  const int64_t first = c.first + block * (THREADS * kClearPieces) + threadIdx.x;
#pragma unroll
  for (int i = 0; i < kClearPieces; ++i)
    if (first + i * THREADS < c.end) p[first + i * THREADS] = u32x4{0, 0, 0, 0};
}
template <int THREADS>
int64_t clear_blocks(const EmbedClear& c) {
  return (c.end - c.first + THREADS * kClearPieces - 1) / (THREADS * kClearPieces);
}

// Few tokens: token t's place is the number of keys below its own, and of equal ones before
// it.  A block places 64 tokens, its waves count in a share of all keys each, 64 at a time: those lie before
// the block's tokens, behind them or are theirs.  T^2 comparisons, two
// instructions each (the whole gradient of 8192 tokens of 256 bf16, on top of one that is there: 23 us, with
// the passes below 31; twice as many would take four times as long here, 35 us there).
constexpr int kRankWaves = 16;
constexpr int kRankKeys = 4096;  // in LDS at a time
__global__ __launch_bounds__(kRankWaves* kWave) void embed_rank_kernel(EmbedArgs a, EmbedClear clear) {
  constexpr int kThreads = kRankWaves * kWave;
  __shared__ __align__(16) unsigned keys[kRankKeys];
  __shared__ int part[kRankWaves][kWave];
  const int64_t block = long_block(), ranks = (a.T + kWave - 1) / kWave;
  if (block >= ranks) {
    embed_clear<kThreads>(clear, block - ranks);
    return;
  }
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int t0 = static_cast<int>(block) * kWave, t = t0 + lane;
  const unsigned mine = t < a.T ? embed_key(a.ids, t, a.V) : 0;
  int below = 0;
  for (int base = 0; base < a.T; base += kRankKeys) {
    __syncthreads();
    // behind the last token: above all keys
#pragma unroll
    for (int i = 0; i < kRankKeys / kThreads; ++i) {
      const int u = base + i * kThreads + static_cast<int>(threadIdx.x);
      keys[u - base] = u < a.T ? static_cast<unsigned>(embed_key(a.ids, u, a.V)) : 0xffffffffu;
    }
    __syncthreads();
    for (int from = wave * kWave; from < min(kRankKeys, a.T - base); from += kThreads) {
      const int u0 = base + from;
      if (u0 == t0) {
        for (int i = 0; i < kWave; ++i) below += keys[from + i] < mine || (keys[from + i] == mine && i < lane) ? 1 : 0;
      } else {
        const unsigned limit = mine + (u0 < t0 ? 1u : 0u);  // keys are below 2^31
#pragma unroll
        for (int i = 0; i < kWave; i += 4) {
          const u32x4 k = *reinterpret_cast<const u32x4*>(keys + from + i);
#pragma unroll
          for (int q = 0; q < 4; ++q) below += k[q] < limit ? 1 : 0;
        }
      }
    }
  }
  part[wave][lane] = below;
  __syncthreads();
  if (wave == 0 && t < a.T) {
    int at = 0;
#pragma unroll
    for (int w = 0; w < kRankWaves; ++w) at += part[w][lane];
    a.keys[at] = static_cast<int>(mine);
    a.order[at] = t;
  }
  if (block == 0 && threadIdx.x == 0) *a.crossing = 0;
}

// More tokens: passes over digits of the key, lowest first, each stable.  A tile of keys
// belongs to one block, its waves hold consecutive parts of it.
constexpr int kDigits = kEmbedDigits;
static_assert(kDigits == kBlock, "a thread per digit");
constexpr int kSortItems = 4;                       // keys per thread
constexpr int kSortTile = kBlock * kSortItems;

__device__ __forceinline__ int sort_key(const EmbedSortPass& s, int64_t i) {
  return s.first ? embed_key(s.ids, i, s.V) : s.keys_in[i];
}

__global__ __launch_bounds__(kBlock) void sort_count_kernel(EmbedSortPass s, EmbedClear clear) {
  const int64_t block = long_block();
  if (block >= s.tiles) {
    embed_clear<kBlock>(clear, block - s.tiles);
    return;
  }
  __shared__ int count[kDigits];
  count[threadIdx.x] = 0;
  __syncthreads();
#pragma unroll
  for (int q = 0; q < kSortItems; ++q) {
    const int64_t i = block * kSortTile + q * kBlock + threadIdx.x;
    if (i < s.T) atomicAdd(&count[(sort_key(s, i) >> s.shift) & (kDigits - 1)], 1);
  }
  __syncthreads();
  s.counts[static_cast<int64_t>(threadIdx.x) * s.tiles + block] = count[threadIdx.x];
  if (block == 0 && threadIdx.x == 0) *s.crossing = 0;
}

// Block `digit`: its counts of the tiles become the sums of those before; their total.
__global__ __launch_bounds__(kBlock) void sort_scan_kernel(EmbedSortPass s, EmbedClear clear) {
  __shared__ int wave_sum[kWavesPerBlock];
  const int64_t block = long_block();
  if (block >= kDigits) {
    embed_clear<kBlock>(clear, block - kDigits);
    return;
  }
  int32_t* c = s.counts + block * s.tiles;
  const int lane = lane_id(), wave = threadIdx.x / kWave;
  int carry = 0;
  for (int base = 0; base < s.tiles; base += kBlock) {
    const int i = base + threadIdx.x;
    const int v = i < s.tiles ? c[i] : 0;
    int sum = v;
#pragma unroll
    for (int k = 1; k < kWave; k <<= 1) {
      const int up = __shfl_up(sum, k);
      sum += lane >= k ? up : 0;
    }
    if (lane == kWave - 1) wave_sum[wave] = sum;
    __syncthreads();
    int before = carry;
#pragma unroll
    for (int w = 0; w < kWavesPerBlock; ++w) {
      before += w < wave ? wave_sum[w] : 0;
      carry += wave_sum[w];
    }
    if (i < s.tiles) c[i] = before + sum - v;
    __syncthreads();
  }
  if (threadIdx.x == 0) s.totals[block] = carry;
}

__global__ __launch_bounds__(kBlock) void sort_place_kernel(EmbedSortPass s, EmbedClear clear) {
  const int64_t block = long_block();
  if (block >= s.tiles) {
    embed_clear<kBlock>(clear, block - s.tiles);
    return;
  }
  __shared__ int at[kWavesPerBlock][kDigits];  // keys of a wave's part by digit, then their first place
  __shared__ int wave_sum[kWavesPerBlock];
  const int lane = lane_id(), wave = threadIdx.x / kWave, tid = threadIdx.x;
#pragma unroll
  for (int w = 0; w < kWavesPerBlock; ++w) at[w][tid] = 0;
  __syncthreads();
  const int64_t base = block * kSortTile + wave * (kWave * kSortItems);
  int key[kSortItems], token[kSortItems], rank[kSortItems];
#pragma unroll
  for (int q = 0; q < kSortItems; ++q) {
    const int64_t i = base + q * kWave + lane;
    key[q] = i < s.T ? sort_key(s, i) : 0;
    token[q] = i < s.T && !s.first ? s.order_in[i] : static_cast<int>(i);
  }
#pragma unroll
  for (int q = 0; q < kSortItems; ++q) {
    const bool in = base + q * kWave + lane < s.T;
    const int digit = (key[q] >> s.shift) & (kDigits - 1);
    uint64_t same = __ballot(in);
#pragma unroll
    for (int b = 0; b < 8; ++b) {
      const uint64_t set = __ballot(digit >> b & 1);
      same &= (digit >> b & 1) ? set : ~set;
    }
    const int before = at[wave][digit];
    rank[q] = before + popc_below(same);
    __builtin_amdgcn_wave_barrier();
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (in && popc_below(same) == 0) at[wave][digit] = before + __popcll(same);
    __builtin_amdgcn_wave_barrier();
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  }
  // keys of smaller digits, by a sum over the digits' totals
  const int total = s.totals[tid];
  int sum = total;
#pragma unroll
  for (int k = 1; k < kWave; k <<= 1) {
    const int up = __shfl_up(sum, k);
    sum += lane >= k ? up : 0;
  }
  if (lane == kWave - 1) wave_sum[wave] = sum;
  __syncthreads();
  int first = sum - total;
#pragma unroll
  for (int w = 0; w < kWavesPerBlock; ++w) first += w < wave ? wave_sum[w] : 0;
  first += s.counts[static_cast<int64_t>(tid) * s.tiles + block];
#pragma unroll
  for (int w = 0; w < kWavesPerBlock; ++w) {
    const int n = at[w][tid];
    at[w][tid] = first;
    first += n;
  }
  __syncthreads();
#pragma unroll
  for (int q = 0; q < kSortItems; ++q) {
    if (base + q * kWave + lane >= s.T) continue;
    const int to = at[wave][(key[q] >> s.shift) & (kDigits - 1)] + rank[q];
    s.keys_out[to] = key[q];
    s.order_out[to] = token[q];
  }
}

// ---------------------------------------------------------------- sums of runs
// Writes scale * sum (+ what is there) to a piece of the table's gradient.
template <class T>
__device__ __forceinline__ void embed_write(const EmbedArgs& a, int key, int c, const float* sum) {
  constexpr int PE = Chunk<T>::kElems;
  u32x4* p = reinterpret_cast<u32x4*>(static_cast<T*>(a.dtable) + static_cast<int64_t>(key) * a.d + c);
  float f[PE];
  if (a.accumulate) {
    Chunk<T>::unpack(*p, f);
#pragma unroll
    for (int q = 0; q < PE; ++q) f[q] += a.scale * sum[q];
  } else {
#pragma unroll
    for (int q = 0; q < PE; ++q) f[q] = a.scale * sum[q];
  }
  *p = Chunk<T>::pack(f);
}

// Which part of a run that crosses chunks a partial sum is: kHead goes on from the chunk
// before, kTail starts in its chunk and goes on in the next.
constexpr int kHead = 0, kTail = 1;
template <class T>
__device__ __forceinline__ float* embed_part(const EmbedArgs& a, int64_t chunk, int which, int c) {
  return a.part + (chunk * 2 + which) * a.d + c;
}

// L lanes per chunk and strip of L pieces; chunks of a.chunk sorted tokens.
template <class T, int L>
__device__ __forceinline__ void embed_chunk(const EmbedArgs& a, int64_t unit) {
  constexpr int PE = Chunk<T>::kElems, U = L < 16 ? 8 : 16;  // rows in flight
  const int strips = (a.d + L * PE - 1) / (L * PE);
  const int64_t chunk = unit / strips;
  const int strip = static_cast<int>(unit - chunk * strips);
  const int64_t lo = chunk * a.chunk, hi = min(static_cast<int64_t>(a.T), lo + a.chunk);
  if (lo >= a.T) return;
  const int c = (strip * L + lane_id() % L) * PE;
  const bool in = c < a.d;
  const T* dy = static_cast<const T*>(a.dy) + (in ? c : 0);
  const int last_key = a.keys[hi - 1];
  const bool from_left = lo > 0 && a.keys[lo - 1] == a.keys[lo];
  const bool to_right = hi < a.T && a.keys[hi] == last_key;
  float sum[PE];
#pragma unroll
  for (int q = 0; q < PE; ++q) sum[q] = 0.f;
  int cur = a.keys[lo];
  bool head = from_left;
  auto flush = [&](bool right) {
    if (!in || cur >= a.V) return;
    if (head || right) {
      float* p = embed_part<T>(a, chunk, head ? kHead : kTail, c);
#pragma unroll
      for (int q = 0; q < PE; q += 4) *reinterpret_cast<u32x4*>(p + q) = Chunk<float>::pack(sum + q);
    } else {
      embed_write<T>(a, cur, c, sum);
    }
  };
  const int lane = lane_id();
  for (int64_t base = lo; base < hi; base += L) {
    // a key and a token per lane, then from lane to lane: loads of single ones would wait for each
    // other (1024 rows of 256 fp32: 7.9 -> 4.4 us).  Rows are read once, non-temporally (65536 rows of
    // 4096 bf16: 169 -> 125).
    const int64_t mine = min(base + lane % L, hi - 1);
    const int keys = a.keys[mine], tokens = a.order[mine];
    auto of = [&](int held, int i) {
      if constexpr (L == kWave) return __builtin_amdgcn_readlane(held, i);
      else return __shfl(held, i, L);
    };
    const int count = static_cast<int>(min(static_cast<int64_t>(L), hi - base));
    for (int i = 0; i < count; i += U) {
      u32x4 v[U];
      // past the chunk's end the last row again, not added; sums of padding rows go nowhere
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(dy + static_cast<int64_t>(of(tokens, i + u)) * a.d));
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int key = of(keys, i + u);
        if (i + u >= count) continue;
        if (key != cur) {
          flush(false);
          cur = key;
          head = false;
#pragma unroll
          for (int q = 0; q < PE; ++q) sum[q] = 0.f;
        }
        float f[PE];
        Chunk<T>::unpack(v[u], f);
#pragma unroll
        for (int q = 0; q < PE; ++q) sum[q] += f[q];
      }
    }
  }
  flush(to_right);
  // one entry for each run that starts here and crosses into the next chunk
  if (to_right && !head && cur < a.V && strip == 0 && lane_id() % L == 0) {
    a.crossers[atomicAdd(a.crossing, 1)] = static_cast<int32_t>(chunk);
  }
}

template <class T, int L>
__global__ __launch_bounds__(kBlock) void embed_sums_kernel(EmbedArgs a) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  embed_chunk<T, L>(a, L == kWave ? long_block() * kWavesPerBlock + wave : long_block() * (kBlock / L) + threadIdx.x / L);
}

// The runs that cross chunks: the parts are added by the block's waves, every kJoinWaves-th
// each, then over the waves, in an order that the ids and sizes decide.
constexpr int kJoinWaves = 8;
template <class T>
__global__ __launch_bounds__(kJoinWaves* kWave) void embed_join_kernel(EmbedArgs a) {
  constexpr int PE = Chunk<T>::kElems;
  __shared__ float red[kJoinWaves][kWave * PE + 4];
  const int lane = lane_id(), wave = threadIdx.x / kWave;
  const int strips = (a.d + kWave * PE - 1) / (kWave * PE);
  const int64_t items = static_cast<int64_t>(*a.crossing) * strips;
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const int64_t chunk = a.crossers[item / strips];
    const int c = (static_cast<int>(item % strips) * kWave + lane) * PE;
    const int key = a.keys[(chunk + 1) * a.chunk];  // that of the run, which goes on there
    // one part per chunk that begins inside the run, and the first
    int64_t parts = 1;
    for (;;) {
      const int64_t begin = (chunk + parts + lane) * a.chunk;
      const uint64_t outside = __ballot(begin >= a.T || a.keys[min(begin, static_cast<int64_t>(a.T) - 1)] != key);
      parts += outside ? __builtin_ctzll(outside) : kWave;
      if (outside) break;
    }
    float sum[PE];
#pragma unroll
    for (int q = 0; q < PE; ++q) sum[q] = 0.f;
    if (c < a.d) {
      constexpr int U = 4;
      for (int64_t p = wave; p < parts; p += kJoinWaves * U) {
        u32x4 v[U][PE / 4];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int64_t at = min(p + u * kJoinWaves, parts - 1);
          const float* src = embed_part<T>(a, chunk + at, at == 0 ? kTail : kHead, c);
#pragma unroll
          for (int q = 0; q < PE / 4; ++q) v[u][q] = reinterpret_cast<const u32x4*>(src)[q];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (p + u * kJoinWaves >= parts) continue;
#pragma unroll
          for (int q = 0; q < PE; ++q) sum[q] += __uint_as_float(v[u][q / 4][q % 4]);
        }
      }
    }
    __syncthreads();  // the sums of the item before are read
#pragma unroll
    for (int q = 0; q < PE; ++q) red[wave][lane * PE + q] = sum[q];
    __syncthreads();
    if (wave == 0 && c < a.d) {
#pragma unroll
      for (int q = 0; q < PE; ++q) {
        sum[q] = 0.f;
#pragma unroll
        for (int w = 0; w < kJoinWaves; ++w) sum[q] += red[w][lane * PE + q];
      }
      embed_write<T>(a, key, c, sum);
    }
  }
}

// Passes over the digits of keys up to V.
int sort_passes(int V) {
  int bits = 1;
  while (bits < 31 && (V >> bits) != 0) ++bits;
  return (bits + 7) / 8;
}

// Lanes per chunk: those that a row's pieces fill.
int chunk_lanes(const EmbedArgs& a) {
  const int pieces = a.d / (a.dtype == 1 ? 8 : 4);
  return pieces <= 8 ? 8 : pieces <= 16 ? 16 : pieces <= 32 ? 32 : 64;
}

template <class T, int L>
hipError_t run_sums(const EmbedArgs& a, hipStream_t st) {
  const int64_t strips = (a.d + L * Chunk<T>::kElems - 1) / (L * Chunk<T>::kElems);
  const int64_t units = static_cast<int64_t>(embed_chunks(a)) * strips;
  embed_sums_kernel<T, L><<<long_grid((units + kBlock / L - 1) / (kBlock / L)), kBlock, 0, st>>>(a);
  return hipGetLastError();
}

template <class T>
hipError_t run_bwd(const EmbedArgs& a, hipStream_t st) {
  if (a.T == 0) return hipSuccess;
  hipError_t err = hipSuccess;
  switch (chunk_lanes(a)) {
    case 8: err = run_sums<T, 8>(a, st); break;
    case 16: err = run_sums<T, 16>(a, st); break;
    case 32: err = run_sums<T, 32>(a, st); break;
    default: err = run_sums<T, 64>(a, st); break;
  }
  if (err != hipSuccess || embed_chunks(a) < 2) return err;
  const int64_t strips = (a.d + kWave * Chunk<T>::kElems - 1) / (kWave * Chunk<T>::kElems);
  const int64_t most = std::min<int64_t>(embed_chunks(a) * strips, 2048);
  embed_join_kernel<T><<<dim3(static_cast<unsigned>(most)), kJoinWaves * kWave, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace

// Sorted tokens per chunk: so that about 4096 waves' worth of chunks and strips run, 8 at least.  (65536
// tokens of 8 KB by Zipf's law: 16384 waves leave 19 us of parts to join, 4096 leave 8.)
int embed_chunk_length(int T, int d, int dtype) {
  if (T <= 32) return 32;  // no parts to join
  const int64_t row = static_cast<int64_t>(d) * (dtype == 1 ? 2 : 4);
  const int64_t want = T * std::max<int64_t>(row, 128) / 1024 / 4096;
  int n = 8;
  while (n < 1024 && n < want) n *= 2;
  return n;
}

int embed_chunks(const EmbedArgs& a) { return (a.T + a.chunk - 1) / a.chunk; }
int embed_sort_tiles(int T) { return (T + kSortTile - 1) / kSortTile; }
hipError_t launch_embed(const EmbedArgs& a, hipStream_t st) {
  return a.dtype == 1 ? run_embed<bf16_t>(a, st) : run_embed<float>(a, st);
}

// a.keys and a.order: where the sorted tokens are to be; spare_keys and spare_order: as much again.
hipError_t launch_embed_bwd(const EmbedArgs& a, int32_t* spare_keys, int32_t* spare_order, int32_t* counts,
                            int32_t* totals, hipStream_t st) {
  hipError_t err = hipSuccess;
  EmbedClear clear{a.dtable, 0, 0};
  const int64_t pieces = a.accumulate ? 0 : static_cast<int64_t>(a.V) * a.d * (a.dtype == 1 ? 2 : 4) / 16;
  if (a.T <= kEmbedRankMax) {
    clear.end = pieces;
    constexpr int kThreads = kRankWaves * kWave;
    const int64_t blocks = (a.T + kWave - 1) / kWave + clear_blocks<kThreads>(clear);
    if (blocks > 0) embed_rank_kernel<<<long_grid(blocks), kThreads, 0, st>>>(a, clear);
    err = hipGetLastError();
  } else {
    EmbedSortPass s{};
    s.ids = a.ids; s.T = a.T; s.V = a.V; s.tiles = embed_sort_tiles(a.T);
    s.counts = counts; s.totals = totals; s.crossing = a.crossing;
    const int passes = sort_passes(a.V);
    int launch = 0;
    // the next launch's share of the table
    auto share = [&](int64_t blocks) {
      clear.first = clear.end;
      clear.end = pieces * ++launch / (3 * passes);
      return long_grid(blocks + clear_blocks<kBlock>(clear));
    };
    for (int p = 0; p < passes && err == hipSuccess; ++p) {
      const bool to_end = (passes - 1 - p) % 2 == 0;  // the last pass ends in a.keys
      s.first = p == 0;
      s.shift = 8 * p;
      s.keys_in = to_end ? spare_keys : a.keys;
      s.order_in = to_end ? spare_order : a.order;
      s.keys_out = to_end ? a.keys : spare_keys;
      s.order_out = to_end ? a.order : spare_order;
      dim3 grid = share(s.tiles);
      sort_count_kernel<<<grid, kBlock, 0, st>>>(s, clear);
      grid = share(kDigits);
      sort_scan_kernel<<<grid, kBlock, 0, st>>>(s, clear);
      grid = share(s.tiles);
      sort_place_kernel<<<grid, kBlock, 0, st>>>(s, clear);
      err = hipGetLastError();
    }
  }
  if (err != hipSuccess) return err;
  return a.dtype == 1 ? run_bwd<bf16_t>(a, st) : run_bwd<float>(a, st);
}

}  // namespace hetumoe
