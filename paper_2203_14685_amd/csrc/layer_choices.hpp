// The layer for few tokens: which choices a block serves.
#pragma once

#include "common.hpp"
#include "kernels.hpp"

namespace hetumoe {

// The expert e of this block (blockIdx.y: an expert, or with a.by_choice a choice, the first one of an
// expert taking all of its rows) and the n choices that name it, in order, in `lists`
// (kLayerMaxChoices, LDS; wave_n: WAVES).  False: nothing to do.
template <int WAVES>
__device__ __forceinline__ bool layer_choices(const LayerArgs& a, int* lists, int* wave_n, int& e, int& n,
                                              const int*& list) {
  const int tid = threadIdx.x, lane = lane_id();
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int choices = a.S * a.k;
  e = blockIdx.y;
  n = 0;
  if (choices <= kWave) {
    // each wave for itself, without a barrier
    const int mine = lane < choices ? a.ids[lane] : -1;
    if (a.by_choice) {
      e = __builtin_amdgcn_readlane(mine, blockIdx.y);
      if (e < 0 || e >= a.E) return false;
    }
    const uint64_t mask = __ballot(mine == e);
    // the first choice of an expert takes all of its rows
    if (a.by_choice && (mask & ((uint64_t(1) << blockIdx.y) - 1)) != 0) return false;
    n = __popcll(mask);
    if (mine == e) lists[wave * kWave + popc_below(mask)] = lane;
    list = lists + wave * kWave;
    __builtin_amdgcn_wave_barrier();
  } else {
    if (a.by_choice) {
      const int c = blockIdx.y;
      e = a.ids[c];
      if (e < 0 || e >= a.E) return false;
      bool earlier = false;
      for (int i = lane; i < c; i += kWave) earlier |= a.ids[i] == e;
      if (__ballot(earlier)) return false;
    }
    for (int base = 0; base < choices; base += WAVES * kWave) {
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
  return true;
}

}  // namespace hetumoe
