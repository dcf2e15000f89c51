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
  // dH with Z in FP16 and a short reduction: two workgroups per CU, one of which reads its Z and stores its dZ under the other's products, where large
  // tiles all read at once.  us, dZ alone, D256 -> D128: FP8 8192 x K x 4096, K = 512 72.1 -> 52.8, 1024 82.1 -> 64.8, 2048 100 -> 89, 2560 115 -> 108,
  // 4096 x 4096 x 4096 71.5 -> 74.4; FP16 K = 512 96 -> 75, 1024 111 -> 109, 2048 161 -> 162; with 8-bit blocks, half of the bytes, FP8 K = 512 54.5 -> 56.1,
  // 1024 64.6 -> 68.9, FP16 1024 98 -> 108: not taken
  const bool two_per_cu = EPI == EPI_GATE_GRAD && p.K * (FP8 ? 1 : 2) <= 2560;
  if (use_big_tile(p.M, p.N, 1) && !two_per_cu) return launch_one<true, Big, FP8, FA, 0, true, NT, EPI, false>(p, 1, p.K, st);
  return launch_one<true, CfgD128, FP8, FA, 0, true, NT, EPI, false>(p, 1, p.K, st);
}

}  // namespace us
