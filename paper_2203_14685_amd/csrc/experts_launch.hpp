// Which products a pass launches, in which tiles (shared by the two element types).
#pragma once

#include "experts.hpp"

namespace hetumoe {

// What every product of the pass shares; tm, tn and tiles are left to the tile choice.
inline ExpertGemmArgs expert_base_args(const ExpertArgs& x) {
  ExpertGemmArgs a{};
  a.E = x.E;
  a.C = x.C;
  a.counts = x.counts;
  a.act = x.act;
  return a;
}

inline void expert_set_tiles(ExpertGemmArgs& a, int E, int BM, int BNO) {
  a.tm = (a.M + BM - 1) / BM;
  a.tn = (a.N + BNO - 1) / BNO;
  a.tiles = E * a.tm * a.tn;
}

// a.N: columns of hidden
hipError_t expert_act_bf16(const ExpertArgs& x, const ExpertGemmArgs& a, hipStream_t st);
hipError_t expert_act_f32(const ExpertArgs& x, const ExpertGemmArgs& a, hipStream_t st);
hipError_t expert_actgrad_bf16(const ExpertArgs& x, const ExpertGemmArgs& a, hipStream_t st);
hipError_t expert_actgrad_f32(const ExpertArgs& x, const ExpertGemmArgs& a, hipStream_t st);
// epilogue kEpiStore: kinds of the operands as (ka, kb) = (rows, cols), (rows, rows), (cols, cols)
hipError_t expert_store_bf16(const ExpertArgs& x, const ExpertGemmArgs& a, int ka, int kb, hipStream_t st);
hipError_t expert_store_f32(const ExpertArgs& x, const ExpertGemmArgs& a, int ka, int kb, hipStream_t st);
// Row ranges per expert whose column sums kEpiActGrad writes.
int expert_parts_bf16(const ExpertArgs& x);
int expert_parts_f32(const ExpertArgs& x);

}  // namespace hetumoe
