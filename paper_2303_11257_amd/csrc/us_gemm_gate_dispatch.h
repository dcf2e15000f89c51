// Host-side choice of tile for the gated block's two products with epilogues of their own, one operand type per translation unit.
#pragma once

#include "us_gemm_dispatch.h"

namespace us {

//   G256: D256 with its waves 4 x 2, 64 x 128 accumulators each, for the forward product: a wave's rows of Z and H leave in pieces twice as long.  Pieces of
//         32 or 64 bytes (8-bit blocks and codes) are less than the memory's lines: us, forward call, D256 -> G256: FP8 16384 x 4096 x 11008 with 8-bit blocks
//         1946 -> 1693, 8192 x 1024 x 4096 128.7 -> 115.6, with FP16 Z 120.5 -> 111.0; FP16 4096 x 2048 x 5632 with 8-bit blocks 254 -> 249, but with FP16 Z
//         4096 x 768 x 2048 48.6 -> 50.2, 2048 x 4096 x 8192 347 -> 344
using CfgG256 = GemmCfg<256, 256, 4, 2, 128, 2, 1>;

// EPI: of the forward product (NN) or of dH (NT).
template <bool FP8, bool NT, int EPI>
hipError_t launch_gate(const GemmProblem& p, hipStream_t st) {
  constexpr int FA = FP8 && NT ? 1 : 0;                // dH: G is E5M2
  if (!offsets_fit(p)) return hipErrorInvalidValue;
  const SmallTileChoice c = small_tile_choice(p);
  if (c == SmallTileChoice::T32x32 || c == SmallTileChoice::T32x64 || (c == SmallTileChoice::None && p.M <= 32)) return launch_small<CfgT32x64, FP8, FA, 0, true, NT, EPI, false>(p, st);
  if (c == SmallTileChoice::T64x64) return launch_small<CfgT64x64, FP8, FA, 0, true, NT, EPI, false>(p, st);
  using Big = typename std::conditional<!NT && (FP8 || EPI == EPI_GATE8), CfgG256, CfgD256>::type;
  if (use_big_tile(p.M, p.N, 1)) return launch_one<true, Big, FP8, FA, 0, true, NT, EPI, false>(p, 1, p.K, st);
  return launch_one<true, CfgD128, FP8, FA, 0, true, NT, EPI, false>(p, 1, p.K, st);
}

}  // namespace us
