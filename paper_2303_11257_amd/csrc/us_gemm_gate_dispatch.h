// Host-side choice of tile for the gated block's two products with epilogues of their own, one operand type per translation unit.
#pragma once

#include "us_gemm_dispatch.h"

namespace us {

// EPI: of the forward product (NN) or of dH (NT).
template <bool FP8, bool NT, int EPI>
hipError_t launch_gate(const GemmProblem& p, hipStream_t st) {
  constexpr int FA = FP8 && NT ? 1 : 0;                // dH: G is E5M2
  if (!offsets_fit(p)) return hipErrorInvalidValue;
  const SmallTileChoice c = small_tile_choice(p);
  if (c == SmallTileChoice::T32x32 || c == SmallTileChoice::T32x64 || (c == SmallTileChoice::None && p.M <= 32)) return launch_small<CfgT32x64, FP8, FA, 0, true, NT, EPI, false>(p, st);
  if (c == SmallTileChoice::T64x64) return launch_small<CfgT64x64, FP8, FA, 0, true, NT, EPI, false>(p, st);
  if (use_big_tile(p.M, p.N, 1)) return launch_one<true, CfgD256, FP8, FA, 0, true, NT, EPI, false>(p, 1, p.K, st);
  return launch_one<true, CfgD128, FP8, FA, 0, true, NT, EPI, false>(p, 1, p.K, st);
}

}  // namespace us
