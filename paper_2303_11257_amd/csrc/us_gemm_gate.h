// Epilogues of the gated feed-forward block on the GEMM kernels' tiles.
//
// EPI_GATE / EPI_GATE8 (forward, X [M,d] times Wgu [d,2f]): a tile's columns are f columns of the gate's half and the same columns of the other
// half, interleaved so that a wave's left half of columns holds the gate's values Zg and its right half, in the same lanes and
// registers, the factors Zu that belong to them.  H = a f(Zg) Zu is therefore made in registers from the FP32 sums, before any rounding, and both
// products, the gate and the product are one launch.  Z leaves in FP16 (EPI_GATE; not at all where the caller keeps nothing), or as 8-bit
// blocks of 32 (EPI_GATE8) whose largest magnitude a row's lanes find among themselves.
// EPI_GATE_GRAD / EPI_GATE8_GRAD (backward, G [M,d] times Wd^T): the tile is dH; the epilogue takes it through FP32 strips to lanes of eight
// consecutive columns, reads Zg and Zu there and stores dZ = [b f'(Zg) Zu dH | c f(Zg) dH]; from 8-bit blocks also H again, which was not kept.
// What bounds them: on long reductions the matrix core (FP8 16384 x 4096 x 11008: forward product 2.95 TFLOP in 1167 us = 2.53 PFLOP/s, 8192 cubed reaches
// 2.74), on short ones the results' way to memory, which a tile's last workgroup waits for (FP8 8192 x 1024 x 4096: 64 us for 0.137 TFLOP and 168 MB, 50 and
// 33 us on their own), next to some 20 vector instructions per value.
#pragma once

#include "us_gate.h"
#include "us_gemm_common.h"

namespace us {

constexpr bool is_gate(int epi) { return epi == EPI_GATE || epi == EPI_GATE8; }
constexpr bool is_gate_grad(int epi) { return epi == EPI_GATE_GRAD || epi == EPI_GATE8_GRAD; }

// LDS strip of a wave: 32 rows of Z (both halves) and H, or of dH in FP32.
template <class Cfg, bool FP8, int EPI>
struct GateStrip {
  static constexpr int HW = Cfg::WN / 2;                                        // columns of either half
  static constexpr int ZB = HW * (EPI == EPI_GATE8 ? 1 : 2), HB = HW * (FP8 ? 1 : 2);
  static constexpr int ROW = is_gate(EPI) ? 2 * ZB + HB : Cfg::WN * 4;
  static constexpr int PITCH = ROW + 16;
  static constexpr int BYTES = 32 * PITCH * Cfg::WAVES;
};

// The four words of a buffer resource, in scalar registers whatever the compiler made their values with.
__device__ __forceinline__ v4i uniform_words(const void* base, uint32_t bytes) {
  const v4i w = buffer_words(base, bytes);
  return v4i{__builtin_amdgcn_readfirstlane(w.x), __builtin_amdgcn_readfirstlane(w.y), __builtin_amdgcn_readfirstlane(w.z), w.w};
}

// 32 rows of SB bytes from the strip (rows EP bytes apart) to `to`, rows `pitch` bytes apart, of which `left` rows and `cols` bytes exist
template <int SB, int EP>
__device__ __forceinline__ void store_section(const uint8_t* strip, void* to, uint32_t pitch, int left, int cols, int lane) {
  constexpr int CPR = SB / 16;
  static_assert(SB % 16 == 0 && 32 * CPR % 64 == 0, "");
  const v4i r = uniform_words(to, (uint32_t)left * pitch);
#pragma unroll
  for (int t = 0; t < 32 * CPR / 64; ++t) {
    const int c = lane + 64 * t, row = c / CPR, at = c % CPR * 16;
    const v4i v = *US_LDS_PTR(const v4i, strip + row * EP + at);
    wt_buffer_store(r, at < cols ? (uint32_t)row * pitch + (uint32_t)at : kOutOfRange, 0, v);
  }
}

// FP8 codes of four values that are known to be numbers within the type's range.
template <int FMT>
__device__ __forceinline__ int codes_in_range(const float* v) {
  if constexpr (FMT == US_E4M3) return __builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], 0, false), true);
  else return __builtin_amdgcn_cvt_pk_bf8_f32(v[2], v[3], __builtin_amdgcn_cvt_pk_bf8_f32(v[0], v[1], 0, false), true);
}
// The larger of m and the magnitudes of N values, NaN if one is (one instruction per two values).
template <int N>
__device__ __forceinline__ float most(float m, const float* v) {
#pragma unroll
  for (int k = 0; k < N; k += 2) m = __builtin_elementwise_maximum(__builtin_elementwise_maximum(m, __builtin_fabsf(v[k])), __builtin_fabsf(v[k + 1]));
  return m;
}

// Largest magnitude of a row's 32 values: a lane has `own`, the others are in the lanes 16 and 32 (16 x 16 results) or 32 (32 x 32) apart.
template <bool M16>
__device__ __forceinline__ float row_max_across(float own, bool ignore_nan) {
  auto f = [&](float a, float b) { return ignore_nan ? __builtin_fmaxf(a, b) : __builtin_elementwise_maximum(a, b); };
  float v = own;
  if constexpr (M16) {
    const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false);
    const unsigned a = r[0], b = r[1];
    v = f(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b));
  }
  const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false);
  const unsigned a = r[0], b = r[1];
  return f(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b));
}

// Codes of a row's share of a block, NQ quads of a lane, and the block's scale.  half_block: its last 16 columns, the second half of a lane's quads, do not
// exist; their sums are zero, but NaN in a row of X with an infinity, which must not mark the block.
template <bool M16, int NQ>
__device__ __forceinline__ uint32_t keep_quads(const v4f (&z)[NQ], int (&code)[NQ], bool half_block) {
  float m = 0.0f;
#pragma unroll
  for (int q = 0; q < NQ; ++q)
#pragma unroll
    for (int e = 0; e < 4; ++e) m = __builtin_elementwise_maximum(m, __builtin_fabsf(z[q][e]));
  m = row_max_across<M16>(m, false);
  // NaN or beyond the largest step: rare, so the wave looks for one first
  if (__builtin_amdgcn_ballot_w64(!(m < kKeepClip)) != 0) {
    m = 0.0f;
#pragma unroll
    for (int q = 0; q < NQ; ++q)
#pragma unroll
      for (int e = 0; e < 4; ++e) m = __builtin_fmaxf(m, __builtin_fabsf(z[q][e]));
    m = row_max_across<M16>(m, true);
    const uint32_t s = keep_scale(m);
    bool nan = false;
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      code[q] = keep_codes_any(z[q][0], z[q][1], z[q][2], z[q][3], keep_inverse(s));
#pragma unroll
      for (int e = 0; e < 4; ++e) nan |= z[q][e] != z[q][e] && !(half_block && q >= NQ / 2);
    }
    return s + (row_max_across<M16>(nan ? 1.0f : 0.0f, true) != 0.0f ? kKeepNan : 0);
  }
  const uint32_t s = keep_scale(m);
  const float inv = keep_inverse(s);
#pragma unroll
  for (int q = 0; q < NQ; ++q) code[q] = keep_codes(z[q][0], z[q][1], z[q][2], z[q][3], inv);
  return s;
}

// Forward.  tn: the tile's column; a wave finishes its 32-row blocks I0 .. I1-1.
template <class Cfg, bool FP8, int EPI, int I0, int I1, class Acc>
__device__ __forceinline__ void gate_epilogue(const GemmArgs& g, const Acc& acc, uint8_t* lds, long m0, long tn) {
  using S = GateStrip<Cfg, FP8, EPI>;
  constexpr int EP = S::PITCH, HW = S::HW, HJ = Cfg::FN / 2;                   // HJ: 32-column blocks of either half
  constexpr bool M16 = Acc::COLS == 2, KEEP8 = EPI == EPI_GATE8;
  constexpr int NQ = M16 ? 2 : 4;                                               // quads of a lane in a row
  static_assert(Cfg::FN % 2 == 0, "");
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int wmn = wave % Cfg::WAVES_MN;
  const long f = g.N / 2;
  const long m = m0 + (wmn % Cfg::WAVES_M) * Cfg::WM + I0 * 32;
  const long n = tn * (Cfg::BN / 2) + (wmn / Cfg::WAVES_M) * HW;                // first column in either half
  const int cols = __builtin_amdgcn_readfirstlane(f - n > HW ? HW : f - n < 0 ? 0 : (int)(f - n));
  const int blocks = (int)((f + 31) / 32);
  uint8_t* strip = lds + wave * (32 * EP);
  with_gate(g.act, [&](auto gate) {
    constexpr int GATE = decltype(gate)::value;
#pragma unroll
    for (int i = 0; i < I1 - I0; ++i) {
      const int left = __builtin_amdgcn_readfirstlane(g.M - m - i * 32 > 32 ? 32 : g.M - m - i * 32 < 0 ? 0 : (int)(g.M - m - i * 32));
#pragma unroll
      for (int j = 0; j < HJ; ++j) {
#pragma unroll
        for (int h = 0; h < 4 / NQ; ++h) {                                      // groups of quads of one row
          v4f zg[NQ], zu[NQ];
          float y[NQ][4];
          const int row = Acc::row(h * NQ, lane);
          uint8_t* const p = strip + row * EP;
#pragma unroll
          for (int q = 0; q < NQ; ++q) {
            zg[q] = acc.quad(I0 + i, j, h * NQ + q) * g.scale;
            zu[q] = acc.quad(I0 + i, HJ + j, h * NQ + q) * g.scale;
#pragma unroll
            for (int e = 0; e < 4; ++e) y[q][e] = gate_terms<GATE>(zg[q][e]).f * (zu[q][e] * g.epi_scale);
          }
          if constexpr (FP8) {
            // a NaN or a value to clip is rare, so the wave looks for one first
            int c[NQ];
            if (__builtin_expect(__builtin_amdgcn_ballot_w64(!(most<NQ * 4>(0.0f, &y[0][0]) <= 448.0f)) != 0, 0)) {
#pragma unroll
              for (int q = 0; q < NQ; ++q) c[q] = (int)cvt4_fp8<US_E4M3>(y[q][0], y[q][1], y[q][2], y[q][3]);
            } else {
#pragma unroll
              for (int q = 0; q < NQ; ++q) c[q] = codes_in_range<US_E4M3>(y[q]);
            }
#pragma unroll
            for (int q = 0; q < NQ; ++q) *US_LDS_PTR(int, p + 2 * S::ZB + j * 32 + Acc::col(h * NQ + q, lane)) = c[q];
          }
#pragma unroll
          for (int q = 0; q < NQ; ++q) {
            const int col = j * 32 + Acc::col(h * NQ + q, lane);
            if constexpr (!FP8) {
              const v4h o = {to_half(y[q][0]), to_half(y[q][1]), to_half(y[q][2]), to_half(y[q][3])};
              *US_LDS_PTR(v4h, p + 2 * S::ZB + col * 2) = o;
            }
            if constexpr (!KEEP8) {
              const v4h a = {to_half(zg[q][0]), to_half(zg[q][1]), to_half(zg[q][2]), to_half(zg[q][3])};
              const v4h b = {to_half(zu[q][0]), to_half(zu[q][1]), to_half(zu[q][2]), to_half(zu[q][3])};
              *US_LDS_PTR(v4h, p + col * 2) = a;
              *US_LDS_PTR(v4h, p + S::ZB + col * 2) = b;
            }
          }
          if constexpr (KEEP8) {
            int cg[NQ], cu[NQ];
            const bool half_block = cols - j * 32 == 16;
            const uint32_t sg = keep_quads<M16>(zg, cg, half_block), su = keep_quads<M16>(zu, cu, half_block);
#pragma unroll
            for (int q = 0; q < NQ; ++q) {
              const int col = j * 32 + Acc::col(h * NQ + q, lane);
              *US_LDS_PTR(int, p + col) = cg[q];
              *US_LDS_PTR(int, p + S::ZB + col) = cu[q];
            }
            if (lane < (M16 ? 16 : 32) && row < left && j * 32 < cols) {
              uint8_t* s = g.keep_scale + (m + i * 32 + row) * (2l * blocks) + (n >> 5) + j;
              s[0] = (uint8_t)sg;
              s[blocks] = (uint8_t)su;
            }
          }
        }
      }
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      const long r0 = m + i * 32;
      if (g.C) {
        constexpr int ES = KEEP8 ? 1 : 2;
        uint8_t* z = (uint8_t*)g.C + (r0 * g.ldc + n) * ES;
        store_section<S::ZB, EP>(strip, z, (uint32_t)g.ldc * ES, left, cols * ES, lane);
        store_section<S::ZB, EP>(strip + S::ZB, z + f * ES, (uint32_t)g.ldc * ES, left, cols * ES, lane);
      }
      constexpr int HS = FP8 ? 1 : 2;
      store_section<S::HB, EP>(strip + 2 * S::ZB, (uint8_t*)g.gate_h + (r0 * f + n) * HS, (uint32_t)f * HS, left, cols * HS, lane);
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
  });
}

// Zg and Zu (times `factor`) of eight consecutive columns as they were kept.
template <bool KEEP8>
struct KeptPair;
template <>
struct KeptPair<false> {
  v8h zg, zu;
  __device__ __forceinline__ void get(float factor, float (&a)[8], float (&b)[8]) const {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      a[k] = (float)zg[k];
      b[k] = __builtin_fmaf((float)zu[k], factor, -0.0f);       // one mixed instruction
    }
  }
};
template <>
struct KeptPair<true> {
  v2i zg, zu;
  uint32_t sg, su;
  __device__ __forceinline__ void get(float factor, float (&a)[8], float (&b)[8]) const {
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(sg > kKeepMost || su > kKeepMost) != 0, 0)) {      // a block with a NaN
      keep_values(zg, keep_step(sg > kKeepMost ? sg - kKeepNan : sg), a);
      keep_values(zu, keep_step(su > kKeepMost ? su - kKeepNan : su) * factor, b);
      if (sg > kKeepMost) keep_put_nan(zg, a);
      if (su > kKeepMost) keep_put_nan(zu, b);
      return;
    }
    keep_values(zg, keep_step(sg), a);
    keep_values(zu, keep_step(su) * factor, b);
  }
};

// dZ (and H) of eight consecutive columns.  dh comes with dZ's second factor (beta_up) in it, and the first one's ratio to it goes into Zu, so that the
// three results take five products: [f' (k Zu) dh | f dh] and H = f (k Zu) (alpha / k), k = beta_gate / beta_up.
struct GateFactors {
  float up, k, h;      // beta_up, beta_gate / beta_up, alpha / k
  __device__ __forceinline__ explicit GateFactors(const GemmArgs& g) : up(g.skip_scale), k(g.epi_scale / g.skip_scale), h(g.gate_alpha * g.skip_scale / g.epi_scale) {}
};
template <int GATE, bool FP8, bool KEEP8>
__device__ __forceinline__ void gate_gradients(const GateFactors& c, const float (&dh)[8], const KeptPair<KEEP8>& z, v8h (&half)[3], v2i (&code)[3]) {
  constexpr int N = KEEP8 ? 3 : 2;
  float zg[8], zu[8], r[3][8];
  z.get(c.k, zg, zu);
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const GateTerms t = gate_terms<GATE>(zg[k]);
    r[0][k] = t.slope * (zu[k] * dh[k]);
    r[1][k] = t.f * dh[k];
    r[2][k] = t.f * zu[k] * c.h;
  }
  if constexpr (FP8) {
    // a NaN or a value to clip is rare, so the wave looks for one first
    const float m = most<8>(most<8>(0.0f, r[0]), r[1]), mh = KEEP8 ? most<8>(0.0f, r[2]) : 0.0f;
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(!(m <= 57344.0f && mh <= 448.0f)) != 0, 0)) {
#pragma unroll
      for (int w = 0; w < 2; ++w)
        code[w] = v2i{(int)cvt4_fp8<US_E5M2>(r[w][0], r[w][1], r[w][2], r[w][3]), (int)cvt4_fp8<US_E5M2>(r[w][4], r[w][5], r[w][6], r[w][7])};
      if constexpr (KEEP8) code[2] = v2i{(int)cvt4_fp8<US_E4M3>(r[2][0], r[2][1], r[2][2], r[2][3]), (int)cvt4_fp8<US_E4M3>(r[2][4], r[2][5], r[2][6], r[2][7])};
    } else {
#pragma unroll
      for (int w = 0; w < 2; ++w) code[w] = v2i{codes_in_range<US_E5M2>(r[w]), codes_in_range<US_E5M2>(r[w] + 4)};
      if constexpr (KEEP8) code[2] = v2i{codes_in_range<US_E4M3>(r[2]), codes_in_range<US_E4M3>(r[2] + 4)};
    }
  } else {
#pragma unroll
    for (int w = 0; w < N; ++w)
#pragma unroll
      for (int k = 0; k < 8; ++k) half[w][k] = to_half(r[w][k]);
  }
}

// Backward.  g.ldc: row pitch of Z and dZ (2f).
template <class Cfg, bool FP8, int EPI, int I0, int I1, class Acc>
__device__ __forceinline__ void gate_grad_epilogue(const GemmArgs& g, const Acc& acc, uint8_t* lds, long m0, long n0) {
  using S = GateStrip<Cfg, FP8, EPI>;
  constexpr bool KEEP8 = EPI == EPI_GATE8_GRAD;
  constexpr int EP = S::PITCH, CPR = Cfg::WN / 8, PER_LANE = 32 * CPR / 64, NI = I1 - I0;
  static_assert(64 % CPR == 0, "a lane keeps to its columns");
  constexpr int RPP = 64 / CPR;                                                 // rows from one chunk of a lane to its next
  constexpr int ZES = KEEP8 ? 1 : 2, OES = FP8 ? 1 : 2;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int wmn = wave % Cfg::WAVES_MN;
  const long f = g.N;
  const long m = m0 + (wmn % Cfg::WAVES_M) * Cfg::WM + I0 * 32;
  const long n = n0 + (wmn / Cfg::WAVES_M) * Cfg::WN;
  const int lrow = lane / CPR, lcol = lane % CPR * 8;
  const bool in = n + lcol < f;
  const uint32_t blocks = (uint32_t)((f + 31) / 32), pitch = (uint32_t)g.ldc;
  uint8_t* strip = lds + wave * (32 * EP);
  const uint32_t zoff = in ? ((uint32_t)lrow * pitch + (uint32_t)lcol) * ZES : kOutOfRange;
  const uint32_t soff = in ? (uint32_t)lrow * (2 * blocks) + (uint32_t)(lcol >> 5) : kOutOfRange;
  const uint32_t doff = in ? ((uint32_t)lrow * pitch + (uint32_t)lcol) * OES : kOutOfRange;
  const uint32_t hoff = in ? ((uint32_t)lrow * (uint32_t)f + (uint32_t)lcol) * OES : kOutOfRange;
  auto rows_left = [&](int i) {
    return (uint32_t)__builtin_amdgcn_readfirstlane(g.M - m - i * 32 > 32 ? 32 : g.M - m - i * 32 < 0 ? 0 : (int)(g.M - m - i * 32));
  };
  // Z of a strip is requested when the strip before it has been computed, ahead of that strip's stores: loads and stores share one in-order
  // counter, so that a load behind stores could only be waited for together with them, each a round trip to memory.  The stores are
  // the compiler's own, so that it counts them: it leaves them pending when it waits for the loads in front of them.  (Against two strips fetched
  // together and their stores waited for in the middle, FP16 8192 x 2048 x 4096 dZ 170 -> 161 us, FP8 x 1024 85.5 -> 82.1.)
  KeptPair<KEEP8> kept[PER_LANE];
  auto fetch = [&](int i) {
    const long r0 = m + i * 32;
    const uint32_t left = rows_left(i);
    const uint8_t* z = (const uint8_t*)g.Zpre + (r0 * g.ldc + n) * ZES;
    const auto rg = __builtin_amdgcn_make_buffer_rsrc((void*)z, 0, (int)(left * pitch * ZES), 0x00027000);
    const auto ru = __builtin_amdgcn_make_buffer_rsrc((void*)(z + f * ZES), 0, (int)(left * pitch * ZES), 0x00027000);
#pragma unroll
    for (int u = 0; u < PER_LANE; ++u) {
      const int below = (int)((uint32_t)(u * RPP) * pitch * ZES);
      if constexpr (KEEP8) {
        kept[u].zg = __builtin_bit_cast(v2i, __builtin_amdgcn_raw_buffer_load_b64(rg, (int)zoff, below, 0));
        kept[u].zu = __builtin_bit_cast(v2i, __builtin_amdgcn_raw_buffer_load_b64(ru, (int)zoff, below, 0));
      } else {
        kept[u].zg = __builtin_bit_cast(v8h, __builtin_amdgcn_raw_buffer_load_b128(rg, (int)zoff, below, 0));
        kept[u].zu = __builtin_bit_cast(v8h, __builtin_amdgcn_raw_buffer_load_b128(ru, (int)zoff, below, 0));
      }
    }
    if constexpr (KEEP8) {
      const uint8_t* s = g.keep_scale + r0 * (2l * blocks) + (n >> 5);
      const auto sg = __builtin_amdgcn_make_buffer_rsrc((void*)s, 0, (int)(left * 2 * blocks), 0x00027000);
      const auto su = __builtin_amdgcn_make_buffer_rsrc((void*)(s + blocks), 0, (int)(left * 2 * blocks), 0x00027000);
#pragma unroll
      for (int u = 0; u < PER_LANE; ++u) {
        const int below = (int)((uint32_t)(u * RPP) * 2 * blocks);
        kept[u].sg = (uint8_t)__builtin_amdgcn_raw_buffer_load_b8(sg, (int)soff, below, 0);
        kept[u].su = (uint8_t)__builtin_amdgcn_raw_buffer_load_b8(su, (int)soff, below, 0);
      }
    }
  };
  fetch(0);
  const GateFactors factors(g);
  const float scale = g.scale * factors.up;
  with_gate(g.act, [&](auto gate) {
    constexpr int GATE = decltype(gate)::value;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
#pragma unroll
      for (int j = 0; j < Cfg::FN; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) *US_LDS_PTR(v4f, strip + Acc::row(q, lane) * EP + (j * 32 + Acc::col(q, lane)) * 4) = acc.quad(I0 + i, j, q) * scale;
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      const long r0 = m + i * 32;
      const uint32_t left = rows_left(i);
      uint8_t* dz = (FP8 ? g.aux8 : (uint8_t*)g.C) + (r0 * g.ldc + n) * OES;
      const auto to_g = __builtin_amdgcn_make_buffer_rsrc((void*)dz, 0, (int)(left * pitch * OES), 0x00027000);
      const auto to_u = __builtin_amdgcn_make_buffer_rsrc((void*)(dz + f * OES), 0, (int)(left * pitch * OES), 0x00027000);
      [[maybe_unused]] const auto to_h = __builtin_amdgcn_make_buffer_rsrc((void*)((uint8_t*)g.gate_h + (r0 * f + n) * OES), 0, (int)(left * (uint32_t)f * OES), 0x00027000);
      v8h half[PER_LANE][3];
      v2i code[PER_LANE][3];
#pragma unroll
      for (int u = 0; u < PER_LANE; ++u) {
        const uint8_t* p = strip + (u * RPP + lrow) * EP + lcol * 4;
        const v4f lo = *US_LDS_PTR(const v4f, p), hi = *US_LDS_PTR(const v4f, p + 16);
        const float dh[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        gate_gradients<GATE, FP8, KEEP8>(factors, dh, kept[u], half[u], code[u]);
      }
      __builtin_amdgcn_sched_barrier(0);
      if (i + 1 < NI) fetch(i + 1);
      __builtin_amdgcn_sched_barrier(0);
      // (the rows of a chunk go into the lane's offset, which an absent column leaves beyond every resource: no scalar offset, see wt_buffer_store)
      constexpr int kWriteThrough = 1 | 16;                                     // sc0 sc1
#pragma unroll
      for (int u = 0; u < PER_LANE; ++u) {
        const int d = (int)(in ? doff + (uint32_t)(u * RPP) * pitch * OES : kOutOfRange);
        [[maybe_unused]] const int hd = (int)(in ? hoff + (uint32_t)(u * RPP) * (uint32_t)f * OES : kOutOfRange);
        typedef unsigned v2u __attribute__((ext_vector_type(2)));
        typedef unsigned v4u __attribute__((ext_vector_type(4)));
        if constexpr (FP8) {
          __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(v2u, code[u][0]), to_g, d, 0, kWriteThrough);
          __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(v2u, code[u][1]), to_u, d, 0, kWriteThrough);
          if constexpr (KEEP8) __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(v2u, code[u][2]), to_h, hd, 0, kWriteThrough);
        } else {
          __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(v4u, half[u][0]), to_g, d, 0, kWriteThrough);
          __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(v4u, half[u][1]), to_u, d, 0, kWriteThrough);
          if constexpr (KEEP8) __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(v4u, half[u][2]), to_h, hd, 0, kWriteThrough);
        }
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
  });
}

// What a thread of the few-tiles kernel does with eight consecutive columns: forward, columns n .. n+7 of both halves; the four threads of a
// block of 32 columns are neighbours and here together, those beyond the matrix with zeros (in: the columns exist).
template <int EPI, bool FP8, int GATE>
__device__ __forceinline__ void gate_point(const GemmArgs& g, long m, long n, bool in, const float (&zg)[8], const float (&zu)[8]) {
  const long f = g.N / 2;
  if constexpr (EPI == EPI_GATE8) {
    const int blocks = (int)((f + 31) / 32);
    auto keep = [&](const float (&z)[8], long half) {
      float big = 0.0f;
      bool rare = false;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        big = __builtin_fmaxf(big, __builtin_fabsf(z[k]));
        rare |= in && z[k] != z[k];          // (columns beyond the matrix: NaN in a row of X with an infinity)
      }
      big = __builtin_fmaxf(big, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, big), 0xB1, 0xf, 0xf, true)));
      big = __builtin_fmaxf(big, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, big), 0x4E, 0xf, 0xf, true)));
      uint32_t s = keep_scale(big);
      const float inv = keep_inverse(s);
      if (__builtin_amdgcn_ballot_w64(rare) >> (threadIdx.x & 60) & 15) s += kKeepNan;      // in any of the block's four lanes
      v2i c;
      if (rare || big >= kKeepClip) c = v2i{keep_codes_any(z[0], z[1], z[2], z[3], inv), keep_codes_any(z[4], z[5], z[6], z[7], inv)};
      else c = v2i{keep_codes(z[0], z[1], z[2], z[3], inv), keep_codes(z[4], z[5], z[6], z[7], inv)};
      if (in) wt_store(reinterpret_cast<v2i*>((uint8_t*)g.C + m * g.ldc + half * f + n), c);
      if (in && (n & 31) == 0) g.keep_scale[m * 2 * blocks + half * blocks + (n >> 5)] = (uint8_t)s;
    };
    keep(zg, 0);
    keep(zu, 1);
  } else if (in && g.C) {
    v8h a, b;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      a[k] = to_half(zg[k]);
      b[k] = to_half(zu[k]);
    }
    wt_store(reinterpret_cast<v8h*>((_Float16*)g.C + m * g.ldc + n), a);
    wt_store(reinterpret_cast<v8h*>((_Float16*)g.C + m * g.ldc + f + n), b);
  }
  if (!in) return;
  float y[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) y[k] = gate_terms<GATE>(zg[k]).f * (zu[k] * g.epi_scale);
  if constexpr (FP8) {
    const v2i c = {(int)cvt4_fp8<US_E4M3>(y[0], y[1], y[2], y[3]), (int)cvt4_fp8<US_E4M3>(y[4], y[5], y[6], y[7])};
    wt_store(reinterpret_cast<v2i*>((uint8_t*)g.gate_h + m * f + n), c);
  } else {
    v8h o;
#pragma unroll
    for (int k = 0; k < 8; ++k) o[k] = to_half(y[k]);
    wt_store(reinterpret_cast<v8h*>((_Float16*)g.gate_h + m * f + n), o);
  }
}

template <int EPI, bool FP8, int GATE>
__device__ __forceinline__ void gate_grad_point(const GemmArgs& g, long m, long n, const float (&dh)[8]) {
  constexpr bool KEEP8 = EPI == EPI_GATE8_GRAD;
  const long f = g.N;
  KeptPair<KEEP8> z;
  if constexpr (KEEP8) {
    const long blocks = (f + 31) / 32;
    z.zg = *reinterpret_cast<const v2i*>((const uint8_t*)g.Zpre + m * g.ldc + n);
    z.zu = *reinterpret_cast<const v2i*>((const uint8_t*)g.Zpre + m * g.ldc + f + n);
    z.sg = g.keep_scale[m * 2 * blocks + (n >> 5)];
    z.su = g.keep_scale[m * 2 * blocks + blocks + (n >> 5)];
  } else {
    z.zg = *reinterpret_cast<const v8h*>(g.Zpre + m * g.ldc + n);
    z.zu = *reinterpret_cast<const v8h*>(g.Zpre + m * g.ldc + f + n);
  }
  const GateFactors factors(g);
  float up[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) up[k] = dh[k] * factors.up;
  v8h half[3];
  v2i code[3];
  gate_gradients<GATE, FP8, KEEP8>(factors, up, z, half, code);
  if constexpr (FP8) {
    wt_store(reinterpret_cast<v2i*>(g.aux8 + m * g.ldc + n), code[0]);
    wt_store(reinterpret_cast<v2i*>(g.aux8 + m * g.ldc + f + n), code[1]);
    if constexpr (KEEP8) wt_store(reinterpret_cast<v2i*>((uint8_t*)g.gate_h + m * f + n), code[2]);
  } else {
    wt_store(reinterpret_cast<v8h*>((_Float16*)g.C + m * g.ldc + n), half[0]);
    wt_store(reinterpret_cast<v8h*>((_Float16*)g.C + m * g.ldc + f + n), half[1]);
    if constexpr (KEEP8) wt_store(reinterpret_cast<v8h*>((_Float16*)g.gate_h + m * f + n), half[2]);
  }
}

}  // namespace us
