// Products of a few rows (the tokens of one generation step) with a weight matrix, for the gated block's two projections: as streams of the
// weights (one to eight rows), and on the few-tiles kernel with the reduction in slices (up to 64).
//
// Streams.  Y = X W with X [T,K], T <= 8 (FP8: 4), W [K,N] row-major.  What bounds it: every weight is read once from HBM and used T times, so nothing but the rate of
// that stream counts.  Weights go from memory to registers in 16-byte loads and into FP32 multiply-adds there: no LDS, no matrix
// instructions, whose operands would have to be transposed on the way.  (FP16: v_fma_mix takes the halves as they are; FP8: two values per
// conversion.  Per 16 bytes of weights of a lane 8 T, FP8 8 + 16 T instructions.)
// A workgroup takes 256 bytes of columns and a slice of the rows; its 4 waves take 16 rows at a time, 4 for each of a wave's
// four groups of 16 lanes, two such batches in flight.  Slices are as many as give every CU four workgroups for one and two rows, three for three and
// four, two for more; their FP32 sums are added in order by a second kernel, which also makes the gate (nothing else knows a whole sum).
// One FP8 token, 4096 x 11008: first projection 18.8 us = 4.8 TB/s, second 11.2 us = 4.0, the two sums 4.6 and 3.8, which is little more than a launch; a
// large copy reaches 5.1 TB/s.
// (The second projection's workgroups making H from the slices themselves, each for its rows while their first weights are on the way, save
// that kernel and cost as much: one FP8 token, 4096 x 11008, 39.4 us with it, 40.0 without.)
#include <type_traits>

#include "us_gemm_gate_dispatch.h"

namespace us {

namespace {

constexpr int kWaves = 4, kThreads = 64 * kWaves, kU = 4, kBatch = kWaves * 4 * kU;      // kBatch: rows of a workgroup's step

struct RowsArgs {
  const uint8_t* X;        // [T][K]
  const uint8_t* W;        // [K][N]
  float* partial;          // [slices][T][N]
  long K, N;
  int T, rows;             // rows of a slice, a multiple of kBatch
};

// acc[c] += w[c] * x[t] over the lane's columns
template <bool FP8, int TT>
__device__ __forceinline__ void add_row(float (&acc)[TT][FP8 ? 16 : 8], v4i w, const float (&x)[TT]) {
  constexpr int CW = FP8 ? 16 : 8;
  float v[CW];
  if constexpr (FP8) {
    typedef float v2f __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const v2f lo = __builtin_amdgcn_cvt_pk_f32_fp8(w[q], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w[q], true);
      v[4 * q] = lo.x; v[4 * q + 1] = lo.y; v[4 * q + 2] = hi.x; v[4 * q + 3] = hi.y;
    }
  } else {
    const v8h h = __builtin_bit_cast(v8h, w);
#pragma unroll
    for (int c = 0; c < 8; ++c) v[c] = (float)h[c];
  }
#pragma unroll
  for (int t = 0; t < TT; ++t)
#pragma unroll
    for (int c = 0; c < CW; ++c) acc[t][c] = __builtin_fmaf(v[c], x[t], acc[t][c]);
}

// The sum of a value over the lanes l, l ^ 16, l ^ 32, l ^ 48, in the vector ALU (as group_reduce of us_rows.h does).
__device__ __forceinline__ float add_groups(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false);
  const unsigned a = r[0], b = r[1];     // (a bit cast of r[1] itself reads element 0 with this compiler)
  v = __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b);
  const auto s = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false);
  const unsigned c = s[0], d = s[1];
  return __builtin_bit_cast(float, c) + __builtin_bit_cast(float, d);
}

template <bool FP8, int TT>
__global__ void __launch_bounds__(kThreads) rows_kernel(RowsArgs a) {
  constexpr int ES = FP8 ? 1 : 2, CW = 16 / ES, STRIP = 16 * CW;               // columns of a lane, of the workgroup
  extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
  float* const xs = reinterpret_cast<float*>(lds);                              // [TT][rows], zeros beyond the matrix
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int grp = lane >> 4, l16 = lane & 15;
  const long k0 = (long)blockIdx.y * a.rows, n0 = (long)blockIdx.x * STRIP;
  const int left = (int)(a.K - k0 < a.rows ? a.K - k0 : a.rows);
  const uint32_t pitch = (uint32_t)a.N * ES;
  // rows beyond the slice or the matrix and columns beyond the matrix read zeros by the resource's range check
  const auto rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)(a.W + (k0 * a.N + n0) * ES), 0, (int)((uint32_t)left * pitch), 0x00027000);
  const uint32_t off = n0 + l16 * CW < a.N ? (uint32_t)((wave * 4 + grp) * kU) * pitch + (uint32_t)l16 * 16u : kOutOfRange;
  auto fetch = [&](v4i (&w)[kU], int step) {
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      // (a row beyond the slice: its offset is beyond the resource, whatever the column)
      const int below = (int)((uint32_t)(step * kBatch + u) * pitch);
      w[u] = __builtin_bit_cast(v4i, __builtin_amdgcn_raw_buffer_load_b128(rsrc, (int)off, below, 0));
    }
  };
  const int steps = (left + kBatch - 1) / kBatch;
  v4i w[2][kU];
  fetch(w[0], 0);
  if (steps > 1) fetch(w[1], 1);
  // the slice's part of X, as floats
  for (int i = tid; i < TT * (a.rows / 8); i += kThreads) {
    const int t = i / (a.rows / 8), k = i % (a.rows / 8) * 8;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = 0.0f;
    if (t < a.T && k < left) {                                                  // K is a multiple of 16
      if constexpr (FP8) {
        const v2i c = *reinterpret_cast<const v2i*>(a.X + t * a.K + k0 + k);
        typedef float v2f __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          const v2f lo = __builtin_amdgcn_cvt_pk_f32_fp8(c[q], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(c[q], true);
          v[4 * q] = lo.x; v[4 * q + 1] = lo.y; v[4 * q + 2] = hi.x; v[4 * q + 3] = hi.y;
        }
      } else {
        const v8h h = *reinterpret_cast<const v8h*>((const _Float16*)a.X + t * a.K + k0 + k);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = (float)h[e];
      }
    }
    v4f* const to = reinterpret_cast<v4f*>(xs + t * a.rows + k);
    to[0] = v4f{v[0], v[1], v[2], v[3]};
    to[1] = v4f{v[4], v[5], v[6], v[7]};
  }
  __syncthreads();
  float acc[TT][CW];
#pragma unroll
  for (int t = 0; t < TT; ++t)
#pragma unroll
    for (int c = 0; c < CW; ++c) acc[t][c] = 0.0f;
  auto use = [&](v4i (&v)[kU], int step) {
    const int k = step * kBatch + (wave * 4 + grp) * kU;
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      float x[TT];
#pragma unroll
      for (int t = 0; t < TT; ++t) x[t] = xs[t * a.rows + k + u];
      add_row<FP8, TT>(acc, v[u], x);
    }
  };
  for (int s = 0; s < steps; s += 2) {
    use(w[0], s);
    if (s + 2 < steps) fetch(w[0], s + 2);
    if (s + 1 < steps) {
      use(w[1], s + 1);
      if (s + 3 < steps) fetch(w[1], s + 3);
    }
  }
  // the four lane groups of a wave, then the waves in order
#pragma unroll
  for (int t = 0; t < TT; ++t)
#pragma unroll
    for (int c = 0; c < CW; ++c) acc[t][c] = add_groups(acc[t][c]);
  __syncthreads();
  float* const red = reinterpret_cast<float*>(lds);                             // [waves][TT][STRIP]
  if (grp == 0) {
#pragma unroll
    for (int t = 0; t < TT; ++t)
#pragma unroll
      for (int c = 0; c < CW; c += 4)
        *reinterpret_cast<v4f*>(red + (wave * TT + t) * STRIP + l16 * CW + c) = v4f{acc[t][c], acc[t][c + 1], acc[t][c + 2], acc[t][c + 3]};
  }
  __syncthreads();
  for (int i = tid; i < TT * STRIP / 4; i += kThreads) {
    const int t = i / (STRIP / 4), c = i % (STRIP / 4) * 4;
    v4f s = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int q = 0; q < kWaves; ++q) s += *reinterpret_cast<const v4f*>(red + (q * TT + t) * STRIP + c);
    if (t < a.T && n0 + c < a.N) *reinterpret_cast<v4f*>(a.partial + ((long)blockIdx.y * a.T + t) * a.N + n0 + c) = s;
  }
}

// Whole sums of eight consecutive columns: a wave has 64 columns, eight lanes 8 apart share eight of them and take every eighth slice
// each (a chain of one eighth of the slices' memory latencies); then their sums are added crosswise.  All eight lanes receive them.
__device__ __forceinline__ void add_slices(const float* p, long step, int slices, float scale, bool in, float (&v)[8]) {
  v4f lo = {0.0f, 0.0f, 0.0f, 0.0f}, hi = lo;
  const int part = (int)(threadIdx.x & 63) >> 3;
  if (in) {
#pragma unroll 4
    for (int s = part; s < slices; s += 8) {
      lo += *reinterpret_cast<const v4f*>(p + s * step);
      hi += *reinterpret_cast<const v4f*>(p + s * step + 4);
    }
  }
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    float x = k < 4 ? lo[k & 3] : hi[k & 3];
#pragma unroll
    for (int off = 8; off < 64; off <<= 1) x += __shfl_xor(x, off, 64);
    v[k] = x * scale;
  }
}

// Y = fp16(scale * sum)
__global__ void __launch_bounds__(64) rows_store_kernel(const float* partial, _Float16* Y, int T, long N, int slices, float scale) {
  const long n = (long)blockIdx.x * 64 + threadIdx.x % 8 * 8;
  const int t = (int)blockIdx.y;
  float v[8];
  add_slices(partial + t * N + n, T * N, slices, scale, n < N, v);
  v8h y;
#pragma unroll
  for (int k = 0; k < 8; ++k) y[k] = to_half(v[k]);
  if (threadIdx.x < 8 && n < N) wt_store(reinterpret_cast<v8h*>(Y + t * N + n), y);
}

// The gate on whole sums; a block of 32 columns is four neighbouring lanes, and all of a wave's eight groups of lanes make the same values.
template <int EPI, bool FP8>
__global__ void __launch_bounds__(64) rows_gate_kernel(const float* partial, GemmArgs g, int slices) {
  const long f = g.N / 2, n = (long)blockIdx.x * 64 + threadIdx.x % 8 * 8;
  const int t = (int)blockIdx.y;
  const bool in = n < f;
  float zg[8], zu[8];
  add_slices(partial + t * g.N + n, g.M * g.N, slices, g.scale, in, zg);
  add_slices(partial + t * g.N + f + n, g.M * g.N, slices, g.scale, in, zu);
  with_gate(g.act, [&](auto gate) { gate_point<EPI, FP8, decltype(gate)::value>(g, t, n, in && threadIdx.x < 8, zg, zu); });
}

// Rows of a slice: whole steps, and as few as give every CU the workgroups that its registers hold.
long slice_rows(long T, long K, long N, bool fp8) {
  const long strips = ceil_div(N, fp8 ? 256 : 128), steps = ceil_div(K, kBatch), want = ceil_div((T <= 2 ? 4 : T <= 4 ? 3 : 2) * cu_count(), strips);
  const long per = ceil_div(steps, want < steps ? want : steps);
  return (per < kMostSteps ? per : kMostSteps) * kBatch;
}

}  // namespace

// Whether the gated block of T tokens, d and f, takes these kernels.  us, both projections, tiles of the matrix core (us_gemm_small.h) -> these; the more
// weights there are, the more rows pay (a row adds its share of the slices' sums, which go through memory, and multiply-adds):
//   FP8   4096 x 11008 (135 MB)  T = 1 75.8 -> 37.4, 2 76.2 -> 41.4, 4 76.6 -> 48.6, 6 77.6 -> 88.6 (the sums of 8 rows do not fit twice into a CU's registers)
//         2048 x 5632 (35 MB)    T = 1 22.4 -> 20.4, 2 22.5 -> 23.5, 4 22.7 -> 30.0;  1024 x 2736 (8 MB)  T = 1 15.0 -> 15.1
//   FP16  4096 x 11008 (271 MB)  T = 1 94.1 -> 61.2, 4 96.8 -> 64.2, 8 99.6 -> 71.2, 12 101.8 -> 158.7
//         2048 x 5632 (69 MB)    T = 1 38.3 -> 23.1, 4 38.3 -> 27.4, 8 39.2 -> 34.7;  1024 x 2736 (17 MB)  T = 1 16.1 -> 15.9, 2 16.3 -> 17.5
bool gemm_rows_take(long T, long d, long f, bool fp8) {
  const long es = fp8 ? 1 : 2, bytes = 3 * d * f * es, most = bytes < (24l << 20) ? 0 : fp8 ? (bytes < (64l << 20) ? 1 : 4) : kRowsMost;
  // (a slice's rows are addressed with 32-bit offsets)
  return T >= 1 && T <= most && 2 * f * es < (1l << 31) / (kMostSteps * kBatch) && d * es < (1l << 31) / (kMostSteps * kBatch);
}
// Slices of a product of at most kSliceRows rows on the few-tiles kernel: the number that leaves the least of the last round empty (`tile`: columns of a
// tile, of which `per_cu` fit on a CU), each with at least 1024 bytes of the reduction; 1 where they would not save a quarter, where the weights are
// below 4 MB (the second kernel costs what they save), and for more than 32 rows unless there are four (unsliced, such a product
// takes a taller tile and reads its weights once).  us, forward call without Z, unsliced -> this rule (slices of up, down):
//   FP16 2048 x 5632 T = 9 38.5 -> 28.7 (1, 8), 32 44.9 -> 32.6, 64 44.5 -> 38.9 (1, 4); 4096 x 11008 T = 13 102 -> 80 (5, 4), 32 116 -> 90; 1536 x 4096 T = 13 22.5 -> 20.2;
//   FP8 4096 x 11008 T = 9 77 -> 66 (1, 4), 2048 x 5632 T = 13 22.5 -> 20.1 (1, 5); not taken: FP16 512 x 1376 11.0 -> 11.9 (1, 2), FP8 4096 x 11008 T = 64 76 -> 81 (1, 2)
long slice_length(long K, int slices) { return ceil_div(ceil_div(K, slices), 64) * 64; }
int gemm_small_slices(long T, long K, long N, bool fp8, int tile, int per_cu) {
  if (T < 1 || T > kSliceRows || K * N * (fp8 ? 1 : 2) < (4l << 20)) return 1;
  const long tiles = ceil_div(T, 32) * ceil_div(N, tile), slots = per_cu * cu_count(), most = K * (fp8 ? 1 : 2) / 1024;
  int best = 1;
  double least = (double)ceil_div(tiles, slots) * 0.75;
  for (int s = 2; s <= 16 && s <= most; ++s) {
    const double t = (double)ceil_div(tiles * s, slots) / s;
    if (t < least * 0.97) {
      best = s;
      least = t;
    }
  }
  return best == 1 || (T > 32 && best < 4) ? 1 : (int)ceil_div(K, slice_length(K, best));
}
int gemm_up_slices(long T, long d, long f, bool fp8) { return gemm_small_slices(T, d, 2 * f, fp8, 64, 1); }
int gemm_down_slices(long T, long d, long f, bool fp8) { return gemm_small_slices(T, f, d, fp8, 32, 2); }

size_t gemm_rows_workspace_bytes(long T, long d, long f, bool fp8) {
  if (!gemm_rows_take(T, d, f, fp8)) {
    const long u = gemm_up_slices(T, d, f, fp8), v = gemm_down_slices(T, d, f, fp8), a = u > 1 ? u * 2 * f : 0, b = v > 1 ? v * d : 0;
    return T < 1 ? 0 : (size_t)T * (size_t)(a > b ? a : b) * sizeof(float);
  }
  const long up = ceil_div(d, slice_rows(T, d, 2 * f, fp8)) * 2 * f, down = ceil_div(f, slice_rows(T, f, d, fp8)) * d;
  return (size_t)T * (size_t)(up > down ? up : down) * sizeof(float);
}

namespace {

template <bool FP8, int TT>
hipError_t launch_tt(const GemmProblem& p, float* partial, hipStream_t st, int* slices) {
  const long rows = slice_rows(p.M, p.K, p.N, FP8), strips = ceil_div(p.N, FP8 ? 256 : 128);
  *slices = (int)ceil_div(p.K, rows);
  const int strip = FP8 ? 256 : 128;
  const long xs = TT * rows * 4, red = (long)kWaves * TT * strip * 4;
  constexpr int LDS = TT * kMostSteps * kBatch * 4 > kWaves * TT * (FP8 ? 256 : 128) * 4 ? TT * kMostSteps * kBatch * 4 : kWaves * TT * (FP8 ? 256 : 128) * 4;
  static FuncConfig cfg;
  if (hipError_t e = cfg.ensure((const void*)rows_kernel<FP8, TT>, LDS); e != hipSuccess) return e;
  note_gemm_launch("stream", (int)p.M, strip, kWaves, 2, FP8, true, false, EPI_PARTIAL, true, *slices);
  const RowsArgs a{(const uint8_t*)p.A, (const uint8_t*)p.B, partial, p.K, p.N, (int)p.M, (int)rows};
  rows_kernel<FP8, TT><<<dim3((unsigned)strips, (unsigned)*slices), kThreads, (size_t)(xs > red ? xs : red), st>>>(a);
  return hipGetLastError();
}

template <bool FP8>
hipError_t launch_rows(const GemmProblem& p, float* partial, hipStream_t st, int* slices) {
  if (p.M <= 1) return launch_tt<FP8, 1>(p, partial, st, slices);
  if (p.M <= 2) return launch_tt<FP8, 2>(p, partial, st, slices);
  if (p.M <= 4) return launch_tt<FP8, 4>(p, partial, st, slices);
  if constexpr (!FP8) {
    if (p.M <= 8) return launch_tt<FP8, 8>(p, partial, st, slices);
  }
  return hipErrorInvalidValue;
}

// The first projection's or the second one's sums in slices, and what makes Z and H or Y of them.
template <bool FP8>
hipError_t launch_gate_of_sums(const GemmProblem& up, bool keep8, const float* partial, int slices, hipStream_t st) {
  const dim3 grid((unsigned)ceil_div(up.N / 2, 64), (unsigned)up.M);
  const GemmArgs g = make_args(up, up.K, 64, 64);
  if (keep8) rows_gate_kernel<EPI_GATE8, FP8><<<grid, 64, 0, st>>>(partial, g, slices);
  else rows_gate_kernel<EPI_GATE, FP8><<<grid, 64, 0, st>>>(partial, g, slices);
  return hipGetLastError();
}
hipError_t launch_store_of_sums(const GemmProblem& down, const float* partial, int slices, hipStream_t st) {
  rows_store_kernel<<<dim3((unsigned)ceil_div(down.N, 64), (unsigned)down.M), 64, 0, st>>>(partial, (_Float16*)down.C, (int)down.M, down.N, slices, down.scale);
  return hipGetLastError();
}

// Both projections as streams.
template <bool FP8>
hipError_t launch_rows_ffn(const GemmProblem& up, const GemmProblem& down, bool keep8, float* partial, hipStream_t st) {
  int slices = 0;
  if (hipError_t e = launch_rows<FP8>(up, partial, st, &slices); e != hipSuccess) return e;
  if (hipError_t e = launch_gate_of_sums<FP8>(up, keep8, partial, slices, st); e != hipSuccess) return e;
  if (hipError_t e = launch_rows<FP8>(down, partial, st, &slices); e != hipSuccess) return e;
  return launch_store_of_sums(down, partial, slices, st);
}

// A product on the few-tiles kernel with its reduction in slices, FP32 sums.  F: formats (the gate's sums as FP16, as in launch_gate).
template <class Cfg, bool FP8, int F>
hipError_t launch_small_slices(const GemmProblem& p, int slices, float* partial, hipStream_t st) {
  constexpr int LDS = SmallTile<Cfg, FP8, true, false>::LDS_BYTES;
  auto kern = gemm_small_kernel<Cfg, FP8, F, F, true, false, EPI_PARTIAL, true>;
  note_gemm_launch("direct", Cfg::BM, Cfg::BN, Cfg::WAVES, Cfg::NST, FP8, true, false, EPI_PARTIAL, true, slices, 0, (F & kAsF16) != 0);
  static FuncConfig cfg;
  if (hipError_t e = cfg.ensure((const void*)kern, LDS); e != hipSuccess) return e;
  GemmArgs g = make_args(p, slice_length(p.K, slices), Cfg::BM, Cfg::BN);
  g.partial = partial;
  kern<<<dim3((unsigned)(ceil_div(p.M, Cfg::BM) * ceil_div(p.N, Cfg::BN)), (unsigned)slices), Cfg::THREADS, LDS, st>>>(g);
  return hipGetLastError();
}

}  // namespace

hipError_t gemm_rows_ffn(const GemmProblem& up, const GemmProblem& down, bool keep8, void* partial, hipStream_t st) {
  return up.a_dt == US_F16 ? launch_rows_ffn<false>(up, down, keep8, (float*)partial, st) : launch_rows_ffn<true>(up, down, keep8, (float*)partial, st);
}

hipError_t gemm_small_gate(const GemmProblem& up, int slices, bool keep8, void* partial, hipStream_t st) {
  const bool fp8 = up.a_dt != US_F16;
  const hipError_t e = fp8 ? launch_small_slices<CfgT32x64, true, kAsF16>(up, slices, (float*)partial, st) : launch_small_slices<CfgT32x64, false, 0>(up, slices, (float*)partial, st);
  if (e != hipSuccess) return e;
  return fp8 ? launch_gate_of_sums<true>(up, keep8, (const float*)partial, slices, st) : launch_gate_of_sums<false>(up, keep8, (const float*)partial, slices, st);
}
hipError_t gemm_small_store(const GemmProblem& down, int slices, void* partial, hipStream_t st) {
  const hipError_t e = down.a_dt != US_F16 ? launch_small_slices<CfgT32x32, true, 0>(down, slices, (float*)partial, st)
                                           : launch_small_slices<CfgT32x32, false, 0>(down, slices, (float*)partial, st);
  return e != hipSuccess ? e : launch_store_of_sums(down, (const float*)partial, slices, st);
}

}  // namespace us
