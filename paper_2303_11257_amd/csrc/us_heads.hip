// From the fused projection to attention's heads: norm of every query and key head, position rotation, head layout, and the way back.
//   forward   x^ = x rstd, rstd = (mean x^2 + eps)^-1/2 over a head's dh values;  y = R(w x^);  V is copied; K's and V's heads are
//             repeated for the query heads that share them
//   backward  g = R^-1(dy) (K, V: the sharing heads' gradients added in FP32, times repeats^-1/2);  dw = beta sum g x^;
//             dx = rstd (g w - x^ mean(g w x^))
// Bound: HBM; every value is read and written once: 16384 tokens of 32 query and 2 x 8 shared heads of 128, forward 604 MB in 129 us = 4.7 TB/s (a large copy: 5.1),
// backward 805 MB in 177 us = 4.6, bound by two waves per SIMD (in heads above 64 the weights' sums and the angles stay in registers; held to three or
// four, the compiler spills: 208 and 323 us).  Heads of 64, 80 and 96 have fewer bytes per angle: forward 4.4, 2.7 and 3.0 TB/s,
// backward 4.2 (three waves), 2.6 and 3.0.  A lane holds 16 values of a head as two chunks of 8 that are each other's partners in the
// rotation (or hold whole pairs), dh / 16 neighbouring lanes a head, so the norm's sum stays inside 16 lanes and no value changes lanes.
// A power of two of such lane groups takes a token at a time: the angles depend on the token and the lane only and are made once for all of
// its heads.
// Angles: a frequency is held as a 64-bit fraction of a turn per position, position * frequency modulo 1 is then integer arithmetic
// that drops whole turns exactly, for any 32-bit position and frequencies of many turns; v_sin / v_cos take the rest, in turns.
#include <type_traits>

#include "us_device.h"
#include "us_launch.h"
#include "us_rows.h"

namespace us {

namespace {

constexpr int kThreads = 256;

// What both directions need of a call.
struct HeadsArgs {
  const _Float16* x;       // [tokens, ld]: query heads, key heads, value heads
  const _Float16 *wq, *wk; // [dh] or NULL
  const int* pos;          // [tokens] or NULL
  const double* freq;      // [rot / 2]
  long ld, tokens;
  int s, h, kv, rep, dh, rot;
  float eps;
};

template <int G>
__device__ __forceinline__ float head_sum(float v) {
  if constexpr (G >= 2) v += lane_dpp<0xB1>(v);
  if constexpr (G >= 4) v += lane_dpp<0x4E>(v);
  if constexpr (G >= 8) v += lane_dpp<0x141>(v);
  if constexpr (G >= 16) v += lane_dpp<0x140>(v);
  return v;
}

// radians -> turns as a 64-bit fraction of one, whole turns dropped.  1 / 2 pi is the sum of two doubles; the product's rounding and the second part are
// kept in `rest`.  Everything in units of 2^-32 turns; adding 1.5 * 2^52 rounds to a whole number, which is then the low bits of the sum.  For frequencies up to
// 2^40 the fraction is right to its last bit, and so an angle at any position to 2^-31 of a turn before its FP32 rounding (2^-26).
__device__ __forceinline__ uint64_t turn_fraction(double w) {
  constexpr double kHi = 0x1.45f306dc9c883p+29, kLo = -0x1.6b01ec5417056p-25, kMagic = 0x1.8p52;
  double t = w * kHi;
  const double rest = __builtin_fma(w, kLo, __builtin_fma(w, kHi, -t));
  t = __builtin_fma(__builtin_rint(t * 0x1p-32), -0x1p32, t);      // at most half a turn
  const double whole = (t + rest) + kMagic, low = __builtin_fma((t - (whole - kMagic)) + rest, 0x1p32, kMagic);
  return (__builtin_bit_cast(uint64_t, whole) << 32) + (__builtin_bit_cast(uint64_t, low) - __builtin_bit_cast(uint64_t, kMagic));
}
// The lane's eight frequencies as 64-bit fractions of a turn, and their angles at a position.
struct LaneAngles {
  uint32_t hi[8], lo[8];
  float c[8], s[8];
  __device__ __forceinline__ void init(const double* freq, int first, bool rotated) {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      hi[k] = lo[k] = 0;
      c[k] = 1.0f;
      s[k] = 0.0f;
      if (rotated) {
        const uint64_t f = turn_fraction(freq[first + k]);
        hi[k] = (uint32_t)(f >> 32);
        lo[k] = (uint32_t)f;
      }
    }
  }
  __device__ __forceinline__ void at(int pos, bool rotated) {
    if (!rotated) return;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      uint32_t f = (uint32_t)pos * hi[k] + __umulhi((uint32_t)pos, lo[k]);
      if (pos < 0) f -= lo[k];
      const float turns = (float)(int)f * 0x1p-32f;
      c[k] = __builtin_amdgcn_cosf(turns);
      s[k] = __builtin_amdgcn_sinf(turns);
    }
  }
};

// The pairs of a lane's 16 values turned by its angles (BACK: the other way).
template <bool HALVES, bool BACK>
__device__ __forceinline__ void turn(float (&v)[16], const LaneAngles& g, bool rotated) {
  if (!rotated) return;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int i = HALVES ? k : 2 * k, j = HALVES ? k + 8 : 2 * k + 1;
    const float a = v[i], b = v[j], s = BACK ? -g.s[k] : g.s[k];
    v[i] = __builtin_fmaf(a, g.c[k], -(b * s));
    v[j] = __builtin_fmaf(b, g.c[k], a * s);
  }
}

struct Lane {
  int a, b;                // columns of the two chunks
  int first;               // first of the eight frequencies
  bool on, rotated;
  template <bool HALVES>
  __device__ __forceinline__ static Lane of(int j, int dh, int rot) {
    Lane l;
    l.on = j * 16 < dh;
    l.rotated = j * 16 < rot;
    l.first = 8 * j;
    const bool split = HALVES && l.rotated;
    l.a = split ? 8 * j : 16 * j;
    l.b = split ? rot / 2 + 8 * j : 16 * j + 8;
    return l;
  }
};

// A lane's values as they lie in memory.
struct Raw {
  v8h a, b;
  __device__ __forceinline__ void load(const _Float16* p, const Lane& l) {
    a = b = v8h{0, 0, 0, 0, 0, 0, 0, 0};
    if (l.on) {
      a = *reinterpret_cast<const v8h*>(p + l.a);
      b = *reinterpret_cast<const v8h*>(p + l.b);
    }
  }
  __device__ __forceinline__ void get(float (&v)[16]) const {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      v[k] = (float)a[k];
      v[k + 8] = (float)b[k];
    }
  }
  __device__ __forceinline__ void add_to(float (&v)[16]) const {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      v[k] += (float)a[k];
      v[k + 8] += (float)b[k];
    }
  }
};
__device__ __forceinline__ void load16(float (&v)[16], const _Float16* p, const Lane& l) {
  Raw r;
  r.load(p, l);
  r.get(v);
}
__device__ __forceinline__ void store16(_Float16* p, const float (&v)[16], const Lane& l) {
  v8h a, b;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    a[k] = to_half(v[k]);
    b[k] = to_half(v[k + 8]);
  }
  if (l.on) {
    wt_store(reinterpret_cast<v8h*>(p + l.a), a);
    wt_store(reinterpret_cast<v8h*>(p + l.b), b);
  }
}
__device__ __forceinline__ void weights16(float (&w)[16], const _Float16* p, const Lane& l) {
  if (p) {
    load16(w, p, l);
  } else {
#pragma unroll
    for (int k = 0; k < 16; ++k) w[k] = 1.0f;
  }
}

// 2^lg lane groups share a token.
template <int G, bool HALVES>
__global__ void __launch_bounds__(kThreads) heads_fwd_kernel(HeadsArgs a, int lg, _Float16* __restrict__ Q, _Float16* __restrict__ K, _Float16* __restrict__ V) {
  const Lane lane = Lane::of<HALVES>((int)threadIdx.x % G, a.dh, a.rot);
  const int slice = (int)threadIdx.x / G, groups = 1 << lg, group = slice & (groups - 1), tokens = kThreads / G >> lg;
  const float per = 1.0f / (float)a.dh;
  LaneAngles ang;
  ang.init(a.freq, lane.first, lane.rotated);
  for (long t = (long)blockIdx.x * tokens + (slice >> lg); t < a.tokens; t += (long)gridDim.x * tokens) {
    const long b = t / a.s, i = t - b * a.s;
    const _Float16* row = a.x + t * a.ld;
    // a head's values are requested while the head before it, or the token's angles, are computed
    Raw x, next;
    if (group < a.h + 2 * a.kv) x.load(row + (long)group * a.dh, lane);
    ang.at(a.pos ? a.pos[t] : (int)i, lane.rotated);
    for (int slot = group; slot < a.h + 2 * a.kv; slot += groups, x = next) {
      if (slot + groups < a.h + 2 * a.kv) next.load(row + (long)(slot + groups) * a.dh, lane);
      float v[16];
      x.get(v);
      const bool is_v = slot >= a.h + a.kv, is_q = slot < a.h;
      if (!is_v) {
        float ss = 0.0f;
#pragma unroll
        for (int k = 0; k < 16; ++k) ss = __builtin_fmaf(v[k], v[k], ss);
        const float rstd = 1.0f / __builtin_sqrtf(__builtin_fmaf(head_sum<G>(ss), per, a.eps));
        float w[16];
        weights16(w, is_q ? a.wq : a.wk, lane);
#pragma unroll
        for (int k = 0; k < 16; ++k) v[k] = v[k] * rstd * w[k];
        turn<HALVES, false>(v, ang, lane.rotated);
      }
      const int rep = is_q ? 1 : a.rep;
      _Float16* out = is_q ? Q : is_v ? V : K;
      const int head = is_q ? slot : (is_v ? slot - a.h - a.kv : slot - a.h) * a.rep;
      for (int r = 0; r < rep; ++r) store16(out + ((b * a.h + head + r) * a.s + i) * a.dh, v, lane);
    }
  }
}

// Partial weights' gradients: one FP32 row [2][dh] (wq, wk) per workgroup in `partial`, added by the next kernel in order.
// 2^lg lane groups share a token.
template <int G, bool HALVES>
__global__ void __launch_bounds__(kThreads) heads_bwd_kernel(HeadsArgs a, int lg, const _Float16* __restrict__ dQ, const _Float16* __restrict__ dK,
                                                             const _Float16* __restrict__ dV, _Float16* __restrict__ dx, long ld_dx,
                                                             float rep_scale, float* __restrict__ partial) {
  // The weights' sums over a lane group's heads and tokens, added up in program order.  Heads of up to 64 keep them in LDS, which leaves registers for a third
  // wave per SIMD; wider heads keep them in registers, as their rounds wait for memory and not for each other (registers -> LDS, us: 16384 tokens of
  // 2 + 2 x 1 heads of 32 20.4 -> 14.5, 65536 of 12 + 2 x 12 of 64 275 -> 262, 16384 of 32 + 2 x 8 of 128 185 -> 189, 16384 of 16 + 2 x 2 of 256 170 -> 177).
  constexpr bool kInLds = G <= 4;
  __shared__ __attribute__((aligned(16))) float sums[kInLds ? 2 : 1][kThreads / G][16 * G];
  const Lane lane = Lane::of<HALVES>((int)threadIdx.x % G, a.dh, a.rot);
  const int slice = (int)threadIdx.x / G, groups = 1 << lg, group = slice & (groups - 1), tokens = kThreads / G >> lg;
  const float per = 1.0f / (float)a.dh;
  LaneAngles ang;
  ang.init(a.freq, lane.first, lane.rotated);
  float sq[16], sk[16];
  if constexpr (kInLds) {
    for (int c = (int)threadIdx.x; c < 2 * kThreads * 16; c += kThreads) (&sums[0][0][0])[c] = 0.0f;
    __syncthreads();
  } else {
#pragma unroll
    for (int k = 0; k < 16; ++k) sq[k] = sk[k] = 0.0f;
  }
  for (long t = (long)blockIdx.x * tokens + (slice >> lg); t < a.tokens; t += (long)gridDim.x * tokens) {
    const long b = t / a.s, i = t - b * a.s;
    ang.at(a.pos ? a.pos[t] : (int)i, lane.rotated);
    const _Float16* row = a.x + t * a.ld;
    _Float16* drow = dx + t * ld_dx;
    const long head_step = (long)a.s * a.dh;
    for (int slot = group; slot < a.h + 2 * a.kv; slot += groups) {
      const bool is_v = slot >= a.h + a.kv, is_q = slot < a.h;
      const int rep = is_q ? 1 : a.rep;
      const _Float16* dy = is_q ? dQ : is_v ? dV : dK;
      const int head = is_q ? slot : (is_v ? slot - a.h - a.kv : slot - a.h) * a.rep;
      dy += ((b * a.h + head) * a.s + i) * a.dh;
      // everything that is read first, the sharing heads' gradients four at a time: one chain of memory latencies per round
      Raw x, y[4];
      if (!is_v) x.load(row + (long)slot * a.dh, lane);
      float g[16];
#pragma unroll
      for (int k = 0; k < 16; ++k) g[k] = 0.0f;
      for (int r = 0; r < rep; r += 4) {
#pragma unroll
        for (int q = 0; q < 4; ++q)
          if (r + q < rep) y[q].load(dy + (r + q) * head_step, lane);
#pragma unroll
        for (int q = 0; q < 4; ++q)
          if (r + q < rep) y[q].add_to(g);
      }
      if (rep > 1) {
#pragma unroll
        for (int k = 0; k < 16; ++k) g[k] *= rep_scale;
      }
      if (!is_v) {
        float v[16], w[16];
        x.get(v);
        weights16(w, is_q ? a.wq : a.wk, lane);
        turn<HALVES, true>(g, ang, lane.rotated);
        float ss = 0.0f;
#pragma unroll
        for (int k = 0; k < 16; ++k) ss = __builtin_fmaf(v[k], v[k], ss);
        const float rstd = 1.0f / __builtin_sqrtf(__builtin_fmaf(head_sum<G>(ss), per, a.eps));
        float dot = 0.0f;
        if constexpr (kInLds) {
          float* const mine = sums[is_q ? 0 : 1][slice];
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            v4f* const at = reinterpret_cast<v4f*>(mine + (q < 2 ? lane.a : lane.b - 8) + 4 * q);
            v4f s = {0.0f, 0.0f, 0.0f, 0.0f};
            if (lane.on) s = *at;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int k = 4 * q + e;
              v[k] *= rstd;
              s[e] += g[k] * v[k];
              g[k] *= w[k];
              dot = __builtin_fmaf(g[k], v[k], dot);
            }
            if (lane.on) *at = s;
          }
        } else {
#pragma unroll
          for (int k = 0; k < 16; ++k) {
            v[k] *= rstd;
            const float gv = g[k] * v[k];
            sq[k] += is_q ? gv : 0.0f;
            sk[k] += is_q ? 0.0f : gv;
            g[k] *= w[k];
            dot = __builtin_fmaf(g[k], v[k], dot);
          }
        }
        dot = head_sum<G>(dot) * per;
#pragma unroll
        for (int k = 0; k < 16; ++k) g[k] = rstd * __builtin_fmaf(-v[k], dot, g[k]);
      }
      store16(drow + (long)slot * a.dh, g, lane);
    }
  }
  // the workgroup's sums, group after group
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    __syncthreads();
    if constexpr (!kInLds) {
      if (lane.on) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          sums[0][slice][lane.a + k] = which ? sk[k] : sq[k];
          sums[0][slice][lane.b + k] = which ? sk[k + 8] : sq[k + 8];
        }
      }
      __syncthreads();
    }
    for (int c = (int)threadIdx.x; c < a.dh; c += kThreads) {
      float s = 0.0f;
      for (int q = 0; q < kThreads / G; ++q) s += sums[kInLds ? which : 0][q][c];
      partial[((long)blockIdx.x * 2 + which) * a.dh + c] = s;
    }
  }
}

// dw[c] = fp16(beta * sum of the workgroups' rows): 16 columns a workgroup, each of 16 threads adds every sixteenth row of one
__global__ void __launch_bounds__(kThreads) heads_dw_kernel(const float* __restrict__ partial, _Float16* dwq, _Float16* dwk, int rows, int dh,
                                                            float beta_q, float beta_k) {
  __shared__ float sums[16][16];
  const int c = (int)threadIdx.x % 16, part = (int)threadIdx.x / 16, col = (int)blockIdx.x * 16 + c;      // of 2 * dh, whole workgroups
  float s = 0.0f;
  int r = part;
  for (; r + 7 * 16 < rows; r += 8 * 16) {             // eight reads in flight
    float v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = partial[(long)(r + k * 16) * 2 * dh + col];
#pragma unroll
    for (int k = 0; k < 8; ++k) s += v[k];
  }
  for (; r < rows; r += 16) s += partial[(long)r * 2 * dh + col];
  sums[part][c] = s;
  __syncthreads();
  if (part == 0) {
    s = 0.0f;
    for (int q = 0; q < 16; ++q) s += sums[q][c];
    const bool is_q = col < dh;
    _Float16* out = is_q ? dwq : dwk;
    if (out) out[is_q ? col : col - dh] = to_half((is_q ? beta_q : beta_k) * s);
  }
}

// Workgroups of the backward kernel: one per wave that its registers leave a SIMD, so that all run at once and each makes its frequencies and its row of sums once
// (us, four per CU -> this: 65536 tokens of 12 + 2 x 12 heads of 64 264 -> 216, 16384 of 1 + 2 x 1 of 64 17.0 -> 13.3, 16384 of 32 + 2 x 8 of 128
// 185 -> 178), or one per token.
constexpr long kMostCus = 256;     // of a gfx950 device; partitions have fewer
long bwd_groups(long tokens, long dh, long cus) {
  const long most = (dh <= 64 ? 3 : 2) * (cus < kMostCus ? cus : kMostCus);
  return tokens < most ? tokens : most;
}
// Lane groups (2^lg) on a token: as many as it has heads, up to `most`.
int log_groups(long slots, int most) {
  int lg = 0;
  while ((1l << lg) < slots && (2 << lg) <= most) ++lg;
  return lg;
}
// ... of the backward kernel: up to a wave's where there are tokens for every wave (a token's query, key and value heads then come round after round, and no
// wave waits for another's share: 16384 tokens of 32 + 2 x 8 heads of 128 292 -> 185 us), else up to a workgroup's.
int bwd_most(long tokens, int G) { return (tokens >= 16 * (long)device_info().cus ? 64 : kThreads) / G; }

// f(integral_constant<int, G>, bool_constant<HALVES>), G: the power of two of lanes that holds dh / 16
template <class F>
hipError_t with_shape(long dh, int pairs, F f) {
  auto go = [&](auto g) {
    if (pairs == US_ROPE_HALVES) f(g, std::true_type{});
    else f(g, std::false_type{});
  };
  if (dh <= 16) go(std::integral_constant<int, 1>{});
  else if (dh <= 32) go(std::integral_constant<int, 2>{});
  else if (dh <= 64) go(std::integral_constant<int, 4>{});
  else if (dh <= 128) go(std::integral_constant<int, 8>{});
  else go(std::integral_constant<int, 16>{});
  return hipGetLastError();
}

HeadsArgs heads_args(const HeadsCall& c) {
  return HeadsArgs{(const _Float16*)c.QKV, (const _Float16*)c.wq, (const _Float16*)c.wk, c.pos, c.freq, c.ld, c.batch * c.s, (int)c.s,
                   (int)c.heads, (int)c.kv_heads, (int)(c.heads / c.kv_heads), (int)c.dh, (int)c.rot, c.eps};
}

}  // namespace

// (the most rows any device's grid makes: the size does not depend on which device asks)
size_t heads_workspace_bytes(long tokens, long dh) { return (size_t)bwd_groups(tokens, dh, kMostCus) * 2 * (size_t)dh * sizeof(float); }

constexpr long kFwdPerCu = 16;     // workgroups per CU: three rounds of what its registers allow even out better than one
// From so many tokens per CU on a wave has one of its own and makes its angles once, as in the backward kernel.  us, four waves on a token -> one: 65536 tokens of
// 12 + 2 x 12 heads of 64 186 -> 134, 12000 of 9 + 2 x 9 of 80 34.8 -> 27.8, 16384 of 32 + 2 x 8 of 128 130 even; 8192 of 64 + 2 x 8 of 128 118 -> 129
constexpr long kFwdWaveTokens = 40;
hipError_t launch_heads_fwd(const HeadsCall& c, void* Q, void* K, void* V, hipStream_t st) {
  const long tokens = c.batch * c.s;
  return with_shape(c.dh, c.pairs, [&](auto g, auto halves) {
    constexpr int G = decltype(g)::value;
    const int lg = log_groups(c.heads + 2 * c.kv_heads, tokens >= kFwdWaveTokens * (long)device_info().cus ? 64 / G : kThreads / G);
    // (a workgroup's frequencies cost as much as a token of a few heads: workgroups for the CUs, not for the tokens)
    const long per = kThreads / G >> lg, need = (tokens + per - 1) / per, most = kFwdPerCu * (long)device_info().cus;
    heads_fwd_kernel<G, decltype(halves)::value><<<(unsigned)(need < most ? need : most), kThreads, 0, st>>>(heads_args(c), lg, (_Float16*)Q, (_Float16*)K, (_Float16*)V);
  });
}

hipError_t launch_heads_bwd(const HeadsCall& c, const void* dQ, const void* dK, const void* dV, void* dQKV, long ld_dx, void* dwq, void* dwk,
                            float beta_wq, float beta_wk, void* workspace, hipStream_t st) {
  const long rows = bwd_groups(c.batch * c.s, c.dh, device_info().cus);
  float* partial = (float*)workspace;
  const float rep_scale = (float)(1.0 / __builtin_sqrt((double)(c.heads / c.kv_heads)));
  const hipError_t e = with_shape(c.dh, c.pairs, [&](auto g, auto halves) {
    constexpr int G = decltype(g)::value;
    heads_bwd_kernel<G, decltype(halves)::value><<<(unsigned)rows, kThreads, 0, st>>>(
        heads_args(c), log_groups(c.heads + 2 * c.kv_heads, bwd_most(c.batch * c.s, G)), (const _Float16*)dQ, (const _Float16*)dK, (const _Float16*)dV, (_Float16*)dQKV, ld_dx,
        rep_scale, partial);
  });
  if (e != hipSuccess || (!dwq && !dwk)) return e;
  heads_dw_kernel<<<(unsigned)(2 * c.dh / 16), kThreads, 0, st>>>(partial, (_Float16*)dwq, (_Float16*)dwk, (int)rows, (int)c.dh, beta_wq, beta_wk);
  return hipGetLastError();
}

}  // namespace us
