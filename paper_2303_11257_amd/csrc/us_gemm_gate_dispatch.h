// Host-side choice of tile for the gated block's two products with epilogues of their own, one operand type per translation unit.
#pragma once

#include "us_gemm_dispatch.h"

namespace us {

//   G256: D256 with its waves 4 x 2, 64 x 128 accumulators each, for the forward product: a wave's rows of Z and H leave in pieces twice as long.  Pieces of
//         32 or 64 bytes (8-bit blocks and codes) are less than the memory's lines: us, forward call, D256 -> G256: FP8 16384 x 4096 x 11008 with 8-bit blocks
//         1946 -> 1693, 8192 x 1024 x 4096 128.7 -> 115.6, with FP16 Z 120.5 -> 111.0; FP16 4096 x 2048 x 5632 with 8-bit blocks 254 -> 249, but with FP16 Z
//         4096 x 768 x 2048 48.6 -> 50.2, 2048 x 4096 x 8192 347 -> 344
using CfgG256 = GemmCfg<256, 256, 4, 2, 128, 2, 1>;

// FP8 products of at most so many tokens go to the matrix core as FP16.  H and dZ are rounded to codes an eighth and a quarter wide: where the FP8 adder moves a
// code of dZ across a border, a column of dWgu = T^-1/2 X^T dZ moves by step * X * T^-1/2, which few tokens do not average out.  The limit is where that is a
// quarter of the RMS for a step of 2 (codes from 8 to 16; larger ones are a few per tensor) and an X of 4: 8 T^-1/2 = 1/4 at 1024 tokens.  Largest deviation of an
// element of dWgu from 64 bits, of the RMS, silu and gelu, d = 512 to 2048, FP8 adder / as FP16: 256 tokens 0.47 / 0.13, 512 0.36 / 0.09, 1024 0.25 / 0.10, 1216 0.22 / 0.11,
// 1536 0.19 / 0.10, 2048 0.17 / 0.08, 4096 0.14 / 0.06; 2-norm 2.0e-3 to 2.6e-3 / 4e-4 to 7e-4 throughout.
// It costs, us, FP8 -> FP16: forward and backward 14 x 1072 x 2848
// 45.9 -> 46.1, 409 x 1920 x 7680 158 -> 171, 1024 x 4096 x 11008 621 -> 685; forward 16 x 2048 x 5632 23.5 -> 23.3, 512 x 4096 x 11008 88 -> 131.
// (The forward call without Z takes it too: what is kept does not change the answer.)
constexpr long kAsF16Rows = 1024;

// EPI: of the forward product (NN) or of dH (NT).
template <bool FP8, bool NT, int EPI, bool AS_F16 = false>
hipError_t launch_gate(const GemmProblem& p, hipStream_t st) {
  constexpr int FB = AS_F16 ? kAsF16 : 0, FA = FB + (FP8 && NT ? 1 : 0);      // dH: G is E5M2
  if (!offsets_fit(p)) return hipErrorInvalidValue;
  if constexpr (FP8 && !AS_F16) {
    if (p.M <= kAsF16Rows) return launch_gate<FP8, NT, EPI, true>(p, st);
  }
  const SmallTileChoice c = small_tile_choice(p);
  if (c == SmallTileChoice::T32x32 || c == SmallTileChoice::T32x64 || (c == SmallTileChoice::None && p.M <= 32)) return launch_small<CfgT32x64, FP8, FA, FB, true, NT, EPI, false>(p, st);
  if (c == SmallTileChoice::T64x64) return launch_small<CfgT64x64, FP8, FA, FB, true, NT, EPI, false>(p, st);
  if constexpr (!AS_F16) {                             // (fragments of larger tiles do not fit the registers as FP16)
    using Big = typename std::conditional<!NT && (FP8 || EPI == EPI_GATE8), CfgG256, CfgD256>::type;
    // dH with Z in FP16 and a short reduction: two workgroups per CU, one of which reads its Z and stores its dZ under the other's products, where large
    // tiles all read at once.  us, dZ alone, D256 -> D128: FP8 8192 x K x 4096, K = 512 72.1 -> 52.8, 1024 82.1 -> 64.8, 2048 100 -> 89, 2560 115 -> 108,
    // 4096 x 4096 x 4096 71.5 -> 74.4; FP16 K = 512 96 -> 75, 1024 111 -> 109, 2048 161 -> 162; with 8-bit blocks, half of the bytes, FP8 K = 512 54.5 -> 56.1,
    // 1024 64.6 -> 68.9, FP16 1024 98 -> 108: not taken
    const bool two_per_cu = EPI == EPI_GATE_GRAD && p.K * (FP8 ? 1 : 2) <= 2560;
    // one round of large tiles instead of two of small ones, as for the layers' products: us, forward call, D128 -> large, FP16 1999 x 1552 x 2064 78.1 -> 63.1,
    // FP8 50.0 -> 40.6, 2300 x 2048 x 2048 49.1 -> 41.8
    if (use_big_single(p, false) && !two_per_cu) return launch_one<true, Big, FP8, FA, FB, true, NT, EPI, false>(p, 1, p.K, st);
    // Tiles that give every CU at most one, and a reduction of 2048 bytes or more: two wave groups.  us, forward call / dZ, D128 -> W128: FP16 512 x 4096 x 4096
    // 74.2 / 44.5 -> 64.6 / 31.0, 1024 x 1024 x 1376 24.4 / 12.2 -> 22.1 / 12.0, FP8 (its own adder) 1024 x 2048 x 2048 29.3 / 13.0 -> 27.7 / 13.1; shorter: FP8 1024 x 1024 x 1376
    // 17.0 / 11.3 -> 17.5 / 11.3, FP16 1024 x 512 x 1376 15.9 / 9.3 -> 16.5 / 9.7
    if (ceil_div(p.M, 128) * ceil_div(p.N, 128) <= cu_count() && p.K * (FP8 ? 1 : 2) >= 2048)
      return launch_one<true, CfgW128, FP8, FA, FB, true, NT, EPI, false>(p, 1, p.K, st);
  }
  return launch_one<true, CfgD128, FP8, FA, FB, true, NT, EPI, false>(p, 1, p.K, st);
}

// The three products behind dZ in one launch, the one with the longest tiles first: dX = dZ Wgu^T (NT), dWgu = X^T dZ and dWd = H^T G (TN), plain results.  Their
// tiles fill each other's last rounds, and for small blocks two launches fall away, which is most of their time.
template <class Cfg, bool FP8, bool SMALL>
struct GradTile {
  static constexpr int FG = FP8 ? 1 : 0;
  template <bool NT>
  __device__ static __forceinline__ void run(const GemmArgs& g, int bid, uint8_t* lds) {
    constexpr int FA = NT ? FG : 0, FB = NT ? 0 : FG;
    if constexpr (SMALL) gemm_small_tile<Cfg, FP8, FA, FB, NT, NT, EPI_STORE, false>(g, bid, lds);
    else gemm_direct_tile<Cfg, FP8, FA, FB, NT, NT, EPI_STORE, false>(g, bid, 0, lds);
  }
};
template <class Cfg, bool FP8, bool SMALL, int MINB>
__global__ void __launch_bounds__(Cfg::THREADS, MINB) gemm_three_kernel(int n_first, int n_second, bool dx_first, GemmArgs dx, GemmArgs dwgu, GemmArgs dwd) {
  extern __shared__ __attribute__((aligned(256))) uint8_t lds[];
  using T = GradTile<Cfg, FP8, SMALL>;
  const int bid = (int)blockIdx.x;
  // dx, dwgu, dwd or dwgu, dwd, dx
  const int at = bid < n_first ? 0 : bid < n_second ? 1 : 2, b = bid - (at == 0 ? 0 : at == 1 ? n_first : n_second);
  if (at == (dx_first ? 0 : 2)) T::template run<true>(dx, b, lds);
  else if (at == (dx_first ? 1 : 0)) T::template run<false>(dwgu, b, lds);
  else T::template run<false>(dwd, b, lds);
}

template <class Cfg, bool FP8, bool SMALL>
hipError_t launch_three(const GemmProblem& dx, const GemmProblem& dwgu, const GemmProblem& dwd, hipStream_t st) {
  int LDS, waves_k;
  void (*kern)(int, int, bool, GemmArgs, GemmArgs, GemmArgs);
  if constexpr (SMALL) {
    constexpr int A = SmallTile<Cfg, FP8, true, true>::LDS_BYTES, B = SmallTile<Cfg, FP8, false, false>::LDS_BYTES;
    LDS = A > B ? A : B;
    waves_k = Cfg::WAVES;
    kern = gemm_three_kernel<Cfg, FP8, true, 1>;
  } else {
    constexpr int A = DirectTile<Cfg, FP8, true, true, false>::LDS_BYTES, B = DirectTile<Cfg, FP8, false, false, false>::LDS_BYTES;
    LDS = A > B ? A : B;
    waves_k = Cfg::WAVES_K;
    kern = gemm_three_kernel<Cfg, FP8, false, Cfg::MINB>;
  }
  note_gemm_launch("three", Cfg::BM, Cfg::BN, waves_k, Cfg::NST, FP8, true, true, EPI_STORE, false, 1);
  for (int i = 0; i < 2; ++i) note_gemm_launch("three", Cfg::BM, Cfg::BN, waves_k, Cfg::NST, FP8, false, false, EPI_STORE, false, 1);
  static FuncConfig cfg;
  if (hipError_t e = cfg.ensure((const void*)kern, LDS); e != hipSuccess) return e;
  auto tiles = [](const GemmProblem& p) { return (int)(ceil_div(p.M, Cfg::BM) * ceil_div(p.N, Cfg::BN)); };
  const int tx = tiles(dx), tg = tiles(dwgu), td = tiles(dwd);
  const bool dx_first = dx.K > dwgu.K;
  kern<<<(unsigned)(tx + tg + td), Cfg::THREADS, LDS, st>>>(dx_first ? tx : tg, dx_first ? tx + tg : tg + td, dx_first, make_args(dx, dx.K, Cfg::BM, Cfg::BN),
                                                         make_args(dwgu, dwgu.K, Cfg::BM, Cfg::BN), make_args(dwd, dwd.K, Cfg::BM, Cfg::BN));
  return hipGetLastError();
}

template <bool FP8>
hipError_t launch_three_grads(const GemmProblem& dx, const GemmProblem& dwgu, const GemmProblem& dwd, hipStream_t st) {
  const SmallTileChoice a = small_tile_choice(dx), b = small_tile_choice(dwgu), c = small_tile_choice(dwd);
  const SmallTileChoice m = a > b ? (a > c ? a : c) : (b > c ? b : c);
  if (a != SmallTileChoice::None && b != SmallTileChoice::None && c != SmallTileChoice::None) {
    if (m == SmallTileChoice::T32x32) return launch_three<CfgT32x32, FP8, true>(dx, dwgu, dwd, st);
    if (m == SmallTileChoice::T32x64) return launch_three<CfgT32x64, FP8, true>(dx, dwgu, dwd, st);
    return launch_three<CfgT64x64, FP8, true>(dx, dwgu, dwd, st);
  }
  return launch_three<CfgD128, FP8, false>(dx, dwgu, dwd, st);
}

}  // namespace us
