// Attention of a few query rows per key head (one new token's heads that share it) over many keys: over the pages of a cache, or over the rows of
// another sequence.
//   p = softmax(c q k), c = dh^-1/2;  O = a sum p v;  weights += sum of p over the rows
// Bound: HBM, keys and values are read once (four sequences of 131072, 8 key heads of 128 codes: 188 us, 5.7 TB/s; 48 of up to 4096 in FP16 85 us, 4.9).  A workgroup takes 16 rows of a key head and a part of its positions, its four waves every fourth tile of
// 32 positions; running statistics per wave, joined through LDS, and over the parts by a second kernel.
// The matrix core gets 16 keys as its first operand, so that a lane holds one row and four keys of each sixteen; rounded to FP16 these are the second
// operand of the product with the values, whose first operand is read transposed from LDS in the same order.  E4M3 codes become FP16 on their way
// (exactly); a head's columns are taken in any order that keys and queries share.
#include "us_flash.h"

namespace us {

namespace {

constexpr int kThreads = 256, kWaves = 4, kStep = 32;      // positions of a wave's tile

struct Pages {
  const uint8_t *k, *v;
  const int* table;
  float* weights;           // or NULL
  float* scores;            // [batch * heads][score_ld], base 2, if weights are wanted
  long score_ld, table_ld, pages;
  int shift;                // log2 of the positions of a page
  FastDiv by_groups, by_tiles, by_kv, by_rep;
  uint32_t groups;          // workgroups of a part
};

__device__ __forceinline__ v4f mfma16(v8h a, v8h b, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

// eight E4M3 codes
__device__ __forceinline__ v8h codes8(int a, int b) {
  const v2h p = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.0f, false), q = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.0f, true);
  const v2h r = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.0f, false), s = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.0f, true);
  return v8h{p[0], p[1], q[0], q[1], r[0], r[1], s[0], s[1]};
}

// maximum / sum over the four lanes that hold a row
template <class F>
__device__ __forceinline__ float row_reduce(float v, F f) {
  const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false);
  const unsigned a = r[0], b = r[1];     // (a bit cast of r[1] itself reads element 0 with this compiler)
  return halves(f(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b)), f);
}

// A tile of values in LDS: rows of P bytes, 16-byte chunk c at c ^ swz(row).  The 32 lanes that a transposing read serves together touch 32 bytes in each of eight
// neighbouring rows (FP16), or 16 bytes in each of those and of the eight rows that lie 16 further on (codes): every bank once.
template <int NB, bool FP8>
struct ValueTile {
  static constexpr int P = FP8 ? (NB <= 2 ? 64 : NB <= 4 ? 128 : 256) : RowTile<NB>::P;
  static constexpr int LOADS = P / 64;      // of 16 rows by a wave
  __device__ __forceinline__ static int swz(int row) {
    if (FP8) {
      if (P == 64) return ((row >> 2) & 1) | ((row >> 4) & 1) << 1;
      if (P == 128) return ((row >> 1) & 3) | ((row >> 4) & 1) << 2;
      return (row & 7) | ((row >> 4) & 1) << 3;
    }
    if (P % 128) return ((row >> 2) & 1) << 1;
    if (P % 256) return ((row >> 1) & 3) << 1;
    return (row & 7) << 1;
  }
};

// A wave's keys of 32 positions, and whether their two sixteens are there.
template <int UNITS>
struct KeyTile {
  v4i k[2][UNITS];
  bool there0, there1;
};

// s_waitcnt vmcnt(N), and nothing that reads memory moves across it
template <int N>
__device__ __forceinline__ void wait_newest() {
  static_assert(N >= 0 && N < 64, "");
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

template <int NB, bool FP8, bool PAGED>
__global__ void __launch_bounds__(kThreads, NB <= 4 ? 2 : 1) few_rows_kernel(AttendArgs a, Pages pg) {
  using T = ValueTile<NB, FP8>;
  constexpr int ES = FP8 ? 1 : 2, UNITS = FP8 ? (NB + 1) / 2 : NB;      // 16-byte chunks of a key per lane
  constexpr int VL = T::LOADS, REQUEST = 2 * (VL + UNITS);              // loads of a tile
  extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
  const int lane = threadIdx.x & 63, l16 = lane & 15, l4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int nrows = a.sq * a.rep;
  // (the parts come last: workgroups go to the XCDs in turn, and one that got the same part of every sequence would have all the short ones' idle parts, or none:
  // 48 sequences of up to 4096 positions in eight parts of their own 112 us, this way 92)
  const uint32_t split = pg.by_groups.of(blockIdx.x);
  const uint32_t i0 = blockIdx.x - split * pg.groups, group = pg.by_tiles.of(i0);
  const int rb = (int)(i0 - group * a.tiles);
  // (the longest sequences first: 93 us -> 85 there; not over another sequence's keys, us in order and ranked: 32 x 16 heads of 64, one query, 1500 keys each 42.7 and 44.5, 47 to 1500
  // 23.0 and 23.3; 48 x 32 by 8 of 128, 85 to 4096 88.2 and 89.6; 32 x 32 by 8 of 128, 47 to 1500 30.5 and 28.8; 16 x 12 of 64, 32 to 512 11.2 and 12.0)
  const int slot = (int)pg.by_kv.of(group), kvh = (int)(group - (uint32_t)slot * a.kv), b = PAGED ? a.by_keys(slot) : slot;
  const int n = a.keys_of(b);
  const int begin = (int)split * a.per_split, end = begin + a.per_split < n ? begin + a.per_split : n;
  const int r0 = rb * 16 + l16, token = (int)pg.by_rep.of((uint32_t)r0), head = kvh * a.rep + (r0 - token * a.rep);
  const bool on = r0 < nrows;
  uint8_t* const tiles = lds + wave * 2 * kStep * T::P;

  const long row_bytes = PAGED ? (long)a.dh * ES : a.k.row;
  // where the 16 positions at `pos` start, in rows: -1 beyond the end, or on a page that there is not
  auto block_of = [&](int pos) -> long {
    if (pos >= end) return -1;
    if constexpr (PAGED) {
      const int page = pg.table[(long)b * pg.table_ld + (pos >> pg.shift)];
      if (page < 0 || page >= pg.pages) return -1;
      return (((long)page * a.kv + kvh) << pg.shift) + (pos & ((1 << pg.shift) - 1));
    } else {
      return pos;
    }
  };
  const uint8_t* kbase = PAGED ? pg.k : (const uint8_t*)(a.k.p + b * a.k.batch + kvh * a.k.head);
  const uint8_t* vbase = PAGED ? pg.v : (const uint8_t*)(a.v.p + b * a.v.batch + kvh * a.v.head);
  // a lane's chunks of a block of 16 positions: of its key, and of the values on their way to LDS; beyond the head's columns nothing (zeros)
  constexpr int kNowhere = 0x7ffffff0;
  int koff[UNITS], voff[FP8 ? 2 : 1][VL];
#pragma unroll
  for (int t = 0; t < UNITS; ++t) {
    const int byte = (4 * t + l4) * 16;
    koff[t] = byte < a.dh * ES ? l16 * (int)row_bytes + byte : kNowhere;
  }
#pragma unroll
  for (int i = 0; i < (FP8 ? 2 : 1); ++i)
#pragma unroll
    for (int j = 0; j < VL; ++j) {
      const int o = (j * 64 + lane) * 16, row = o / T::P, byte = (o % T::P) ^ (T::swz(row + 16 * i) << 4);
      voff[i][j] = byte < a.dh * ES ? row * (int)row_bytes + byte : kNowhere;
    }

  // A tile on its way, requested while its predecessor is computed: the values first, so that they have landed when the keys are there.
  using Tile = KeyTile<UNITS>;
  auto request = [&](Tile& x, uint8_t* vt, int pos, long at0, long at1) {
    x.there0 = at0 >= 0;
    x.there1 = at1 >= 0;
    auto bytes = [&](int from, long at) -> int {
      const int rows = end - from < 16 ? end - from : 16;
      return at < 0 || rows <= 0 ? 0 : (rows - 1) * (int)row_bytes + a.dh * ES;
    };
    const int bytes0 = bytes(pos, at0), bytes1 = bytes(pos + 16, at1);
    const long o0 = at0 < 0 ? 0 : at0 * row_bytes, o1 = at1 < 0 ? 0 : at1 * row_bytes;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const v4i res = buffer_words(vbase + (i ? o1 : o0), (uint32_t)(i ? bytes1 : bytes0));
#pragma unroll
      for (int j = 0; j < VL; ++j) load_to_lds(res, vt + i * 16 * T::P + j * 1024, (uint32_t)voff[FP8 ? i : 0][j]);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const __amdgpu_buffer_rsrc_t res = __builtin_amdgcn_make_buffer_rsrc((void*)(kbase + (i ? o1 : o0)), 0, i ? bytes1 : bytes0, 0x00027000);
#pragma unroll
      for (int t = 0; t < UNITS; ++t) x.k[i][t] = __builtin_bit_cast(v4i, __builtin_amdgcn_raw_buffer_load_b128(res, koff[t], 0, 0));
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  constexpr int kRound = kWaves * kStep;
  Tile tile[2];
  int pos = begin + wave * kStep;
  if (pos < end) request(tile[0], tiles, pos, block_of(pos), block_of(pos + 16));
  long n0 = block_of(pos + kRound), n1 = block_of(pos + kRound + 16);

  // the rows' fragments: the columns that a lane's chunk of a key holds
  v8h qf[FP8 ? 2 * UNITS : UNITS];
  {
    const _Float16* q = (const _Float16*)((const uint8_t*)(a.q.p + b * a.q.batch + head * a.q.head) + (long)token * a.q.row);
#pragma unroll
    for (int t = 0; t < (FP8 ? 2 * UNITS : UNITS); ++t) {
      const int col = FP8 ? 64 * (t / 2) + 16 * l4 + 8 * (t % 2) : 32 * t + 8 * l4;
      qf[t] = v8h{0, 0, 0, 0, 0, 0, 0, 0};
      if (on && col < a.dh) qf[t] = *reinterpret_cast<const v8h*>(q + col);
    }
  }
  v4f acc[2 * NB];
#pragma unroll
  for (int j = 0; j < 2 * NB; ++j) acc[j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
  float m = -__builtin_inff(), sum = 0.0f;
  auto compute = [&](const Tile& x, const uint8_t* vt, int pos, bool newer) {
    // scores of 2 x 16 positions: a lane holds its row's 4 l4 .. + 3 of either
    v4f s[2];
    float top = -__builtin_inff();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      s[i] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int t = 0; t < UNITS; ++t) {
        if constexpr (FP8) {
          s[i] = mfma16(codes8(x.k[i][t][0], x.k[i][t][1]), qf[2 * t], s[i]);
          s[i] = mfma16(codes8(x.k[i][t][2], x.k[i][t][3]), qf[2 * t + 1], s[i]);
        } else {
          s[i] = mfma16(__builtin_bit_cast(v8h, x.k[i][t]), qf[t], s[i]);
        }
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s[i][e] *= a.c2;
        if (!(i ? x.there1 : x.there0) || pos + 16 * i + 4 * l4 + e >= end) s[i][e] = -__builtin_inff();
        top = __builtin_fmaxf(top, s[i][e]);
      }
      if (PAGED && pg.scores && on && pos + 16 * i < end)
        *reinterpret_cast<v4f*>(pg.scores + ((long)b * a.heads + head) * pg.score_ld + pos + 16 * i + 4 * l4) = s[i];
    }
    top = __builtin_fmaxf(m, row_reduce(top, [](float x, float y) { return __builtin_fmaxf(x, y); }));
    // (positions that are all on pages that there are not: nothing is there yet)
    const float use = top == -__builtin_inff() ? 0.0f : top;
    if (__builtin_amdgcn_ballot_w64(top > m)) {
      const float f = __builtin_amdgcn_exp2f(m - use);
      sum *= f;
#pragma unroll
      for (int j = 0; j < 2 * NB; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[j][e] *= f;
    }
    m = top;
    v8h p;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float y = __builtin_amdgcn_exp2f(s[i][e] - use);
        sum += y;
        p[4 * i + e] = (_Float16)y;
      }
    // the values have landed: what may still be on its way is the next tile
    if (newer) wait_newest<REQUEST>();
    else wait_newest<0>();
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int j = 0; j < 2 * NB; ++j) {
      // lane: column 16 j + l16, positions 4 l4 .. + 3 of either sixteen
      if constexpr (FP8) {
        const int row = (l16 >> 3) * 16 + 4 * l4 + ((l16 >> 1) & 3);
        const v2i c = __builtin_amdgcn_ds_read_tr8_b64_v2i32(US_LDS_AT(v2i, vt + row * T::P + ((j ^ T::swz(row)) << 4) + (l16 & 1) * 8));
        acc[j] = mfma16(codes8(c[0], c[1]), p, acc[j]);
      } else {
        const int row = 4 * l4 + (l16 >> 2), chunk = 2 * j + ((l16 & 3) >> 1);
        const uint8_t* at = vt + row * T::P + ((chunk ^ T::swz(row)) << 4) + (l16 & 1) * 8;      // (16 rows on: the same swizzle)
        const v4s y = __builtin_amdgcn_ds_read_tr16_b64_v4i16(US_LDS_AT(v4s, at));
        const v4s z = __builtin_amdgcn_ds_read_tr16_b64_v4i16(US_LDS_AT(v4s, at + 16 * T::P));
        struct { v4s y, z; } both = {y, z};
        acc[j] = mfma16(__builtin_bit_cast(v8h, both), p, acc[j]);
      }
    }
    // (the next request to this half of LDS comes after these reads have been used)
    __builtin_amdgcn_s_waitcnt(0xC07F);
    __builtin_amdgcn_sched_barrier(0);
  };
  for (; pos < end; pos += 2 * kRound) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int at = pos + h * kRound;
      if (at >= end) break;
      const bool newer = at + kRound < end;
      if (newer) request(tile[h ^ 1], tiles + (h ^ 1) * kStep * T::P, at + kRound, n0, n1);
      n0 = block_of(at + 2 * kRound);
      n1 = block_of(at + 2 * kRound + 16);
      compute(tile[h], tiles + h * kStep * T::P, at, newer);
    }
  }
  sum = row_reduce(sum, [](float x, float y) { return x + y; });

  // the waves' sums, in their order
  __shared__ float wm[kWaves][16], ws[kWaves][16];
  __syncthreads();
  if (l4 == 0) {
    wm[wave][l16] = m;
    ws[wave][l16] = sum;
  }
  float* mine = reinterpret_cast<float*>(lds) + (wave * 16 + l16) * 32 * NB;
#pragma unroll
  for (int j = 0; j < 2 * NB; ++j) *reinterpret_cast<v4f*>(mine + 16 * j + 4 * l4) = acc[j];
  __syncthreads();
  const float alpha = a.factor(n);
  const bool parts = a.splits > 1;
  for (int i = (int)threadIdx.x; i < 16 * 8 * NB; i += kThreads) {
    const int r = i / (8 * NB), col = i % (8 * NB) * 4, row = rb * 16 + r;
    if (row >= nrows) continue;
    float top = wm[0][r], total = 0.0f;
#pragma unroll
    for (int w = 1; w < kWaves; ++w) top = __builtin_fmaxf(top, wm[w][r]);
    v4f o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      if (ws[w][r] == 0.0f) continue;
      const float f = __builtin_amdgcn_exp2f(wm[w][r] - top);
      total = __builtin_fmaf(f, ws[w][r], total);
      const v4f x = *reinterpret_cast<const v4f*>(reinterpret_cast<const float*>(lds) + (w * 16 + r) * 32 * NB + col);
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = __builtin_fmaf(f, x[e], o[e]);
    }
    const int t = row / a.rep, hd = kvh * a.rep + (row - t * a.rep);
    const long at = ((long)b * a.heads + hd) * a.sq + t;
    if (col == 0 && a.stats) a.stats[split * (a.part_stride / a.dh) + at] = make_float2(top, total);
    if (col == 0 && !parts && a.lse) a.lse[at] = total > 0.0f || total != total ? (top + __builtin_amdgcn_logf(total)) * kLn2F : -__builtin_inff();
    if (col >= a.dh) continue;
    if (parts) {
      wt_store(reinterpret_cast<v4f*>(a.part + split * a.part_stride + at * a.dh + col), o);
    } else {
      const float f = total == 0.0f ? 0.0f : alpha / total;
      const v4h h = {to_half(o[0] * f), to_half(o[1] * f), to_half(o[2] * f), to_half(o[3] * f)};
      wt_store(reinterpret_cast<v4h*>(a.out + b * a.out_batch + hd * a.out_head + (long)t * a.out_row + col), h);
    }
  }
  if constexpr (PAGED) {
    // all scores of the key head's rows are this workgroup's: their weights, without another launch
    if (pg.scores && !a.stats) {
      __shared__ float ms[16], inv[16];
      if (threadIdx.x < 16) {
        const int r = (int)threadIdx.x;
        float top = wm[0][r], total = 0.0f;
#pragma unroll
        for (int w = 1; w < kWaves; ++w) top = __builtin_fmaxf(top, wm[w][r]);
#pragma unroll
        for (int w = 0; w < kWaves; ++w)
          if (ws[w][r] != 0.0f) total = __builtin_fmaf(__builtin_amdgcn_exp2f(wm[w][r] - top), ws[w][r], total);
        ms[r] = top;
        inv[r] = 1.0f / total;
      }
      __threadfence_block();
      __syncthreads();
      for (int at = (int)threadIdx.x; at < end; at += kThreads) {
        const int page = pg.table[(long)b * pg.table_ld + (at >> pg.shift)];
        if (page < 0 || page >= pg.pages) continue;
        float* const to = pg.weights + (((long)page * a.kv + kvh) << pg.shift) + (at & ((1 << pg.shift) - 1));
        const float* s = pg.scores + ((long)b * a.heads + kvh * a.rep) * pg.score_ld + at;
        // (the rows first and in finish_kernel's order: one rounding at the size of what has been added up so far, and the same bits whichever of the two adds)
        float w = 0.0f;
        for (int r = 0; r < nrows; ++r) w = __builtin_fmaf(__builtin_amdgcn_exp2f(s[r * pg.score_ld] - ms[r]), inv[r], w);
        *to += w;
      }
    }
  }
}

// What is left when all parts are there.  The first `joins` workgroups join a row each: O = a sum_s 2^(m_s - m) O_s / sum_s 2^(m_s - m) l_s (parts without
// positions have l_s = 0 and are not read); the others add the weights of 256 positions of a key head: sum over its rows of 2^(score - m) / l.
// (13 x 16 heads of 2500 positions, weights: 5.5 us, most of it the launch and one read after another.)
constexpr int kMostParts = 1024;
__global__ void __launch_bounds__(kThreads) finish_kernel(AttendArgs a, Pages pg, long joins, int segments) {
  const int tid = (int)threadIdx.x;
  const long stride = a.part_stride / a.dh;
  __shared__ float fs[kMostParts];
  __shared__ __attribute__((aligned(16))) float red[kThreads * 4];
  if ((long)blockIdx.x < joins) {
    const long row = blockIdx.x, bh = row / a.sq;
    const int q = (int)(row - bh * a.sq), b = (int)(bh / a.heads), head = (int)(bh - (long)b * a.heads);
    float m = -__builtin_inff(), sum = 0.0f;
    float2 st[kMostParts / kThreads];
#pragma unroll
    for (int i = 0; i < kMostParts / kThreads; ++i) {
      st[i] = make_float2(-__builtin_inff(), 0.0f);
      if (tid + i * kThreads < a.splits) st[i] = a.stats[(tid + i * kThreads) * stride + row];
      m = __builtin_fmaxf(m, st[i].x);
    }
    red[tid] = wave_max(m);
    __syncthreads();
    m = __builtin_fmaxf(__builtin_fmaxf(red[0], red[64]), __builtin_fmaxf(red[128], red[192]));
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kMostParts / kThreads; ++i) {
      const float f = st[i].y == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(st[i].x - m);      // (a NaN sum is not zero)
      if (tid + i * kThreads < a.splits) fs[tid + i * kThreads] = f;
      if (st[i].y != 0.0f) sum = __builtin_fmaf(f, st[i].y, sum);
    }
    sum = wave_sum(sum);
    red[tid] = sum;
    __syncthreads();
    sum = (red[0] + red[64]) + (red[128] + red[192]);
    __syncthreads();
    // a thread takes four columns of every G-th part
    const int cols = a.dh / 4, G = kThreads / cols, g = tid / cols, col = (tid - g * cols) * 4;
    v4f o = {0.0f, 0.0f, 0.0f, 0.0f};
    if (g < G)
      for (int s = g; s < a.splits; s += G) {
        const float f = fs[s];
        if (f == 0.0f) continue;
        const v4f x = *reinterpret_cast<const v4f*>(a.part + s * a.part_stride + row * a.dh + col);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = __builtin_fmaf(f, x[e], o[e]);
      }
    *reinterpret_cast<v4f*>(red + 4 * tid) = o;
    __syncthreads();
    const bool any = sum != 0.0f;      // (NaN: some)
    if (g == 0) {
      for (int k = 1; k < G; ++k) {
        const v4f x = *reinterpret_cast<const v4f*>(red + 4 * (tid + k * cols));
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] += x[e];
      }
      const float f = any ? a.factor(a.keys_of(b)) / sum : 0.0f;
      const v4h h = {to_half(o[0] * f), to_half(o[1] * f), to_half(o[2] * f), to_half(o[3] * f)};
      wt_store(reinterpret_cast<v4h*>(a.out + b * a.out_batch + head * a.out_head + (long)q * a.out_row + col), h);
    }
    if (a.lse && tid == 0) a.lse[row] = any ? (m + __builtin_amdgcn_logf(sum)) * kLn2F : -__builtin_inff();
    return;
  }
  const long block = blockIdx.x - joins, group = block / segments;
  const int seg = (int)(block - group * segments), b = (int)(group / a.kv), kvh = (int)(group % a.kv);
  const int n = a.keys_of(b), pos = seg * kThreads + tid;
  if (seg * kThreads >= n) return;
  // (everything that can be read at once is: the page, the first rows' scores, the parts' statistics)
  int page = -1;
  if (pos < n) page = pg.table[(long)b * pg.table_ld + (pos >> pg.shift)];
  const float* scores = pg.scores + ((long)b * a.heads + kvh * a.rep) * pg.score_ld + pos;
  float early[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) early[i] = pos < n && i < a.rep ? scores[i * pg.score_ld] : 0.0f;
  float *ms = red, *inv = red + 64, w = 0.0f;
  for (int r0 = 0; r0 < a.rep; r0 += 64) {
    __syncthreads();
    const int r = r0 + tid;
    if (tid < 64 && r < a.rep) {
      const float2* st = a.stats + (long)b * a.heads + kvh * a.rep + r;
      float m = -__builtin_inff(), sum = 0.0f;
      // running, eight parts' statistics in flight
      for (int s = 0; s < a.splits; s += 8) {
        float2 x[8];
        float top = m;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          x[k] = s + k < a.splits ? st[(s + k) * stride] : make_float2(-__builtin_inff(), 0.0f);
          top = __builtin_fmaxf(top, x[k].x);
        }
        sum = sum == 0.0f ? 0.0f : sum * __builtin_amdgcn_exp2f(m - top);
        m = top;
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (x[k].y != 0.0f) sum = __builtin_fmaf(__builtin_amdgcn_exp2f(x[k].x - m), x[k].y, sum);
      }
      ms[tid] = m;
      inv[tid] = 1.0f / sum;
    }
    __syncthreads();
    if (pos < n) {
      const int most = a.rep - r0 < 64 ? a.rep - r0 : 64;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (r0 == 0 && i < most) w = __builtin_fmaf(__builtin_amdgcn_exp2f(early[i] - ms[i]), inv[i], w);
#pragma unroll 4
      for (int i = r0 == 0 ? 4 : 0; i < most; ++i) w = __builtin_fmaf(__builtin_amdgcn_exp2f(scores[(r0 + i) * pg.score_ld] - ms[i]), inv[i], w);
    }
  }
  if (page < 0 || page >= pg.pages) return;
  pg.weights[(((long)page * a.kv + kvh) << pg.shift) + (pos & ((1 << pg.shift) - 1))] += w;
}

template <bool FP8, bool PAGED, class F>
hipError_t with_kernel(long dh, F f) {
  auto go = [&](auto nb) {
    constexpr int NB = decltype(nb)::value;
    static FuncConfig config;
    constexpr int lds = kWaves * 2 * kStep * ValueTile<NB, FP8>::P;
    static_assert(lds >= kWaves * 16 * 32 * NB * 4, "the waves' sums fit");
    if (const hipError_t e = config.ensure((const void*)few_rows_kernel<NB, FP8, PAGED>, lds); e != hipSuccess) return e;
    return f(few_rows_kernel<NB, FP8, PAGED>, lds);
  };
  if (dh <= 32) return go(std::integral_constant<int, 1>{});
  if (dh <= 64) return go(std::integral_constant<int, 2>{});
  if (dh <= 96) return go(std::integral_constant<int, 3>{});
  if (dh <= 128) return go(std::integral_constant<int, 4>{});
  if (dh <= 192) return go(std::integral_constant<int, 6>{});
  return go(std::integral_constant<int, 8>{});
}

long ceil_div(long a, long b) { return (a + b - 1) / b; }
size_t up256(size_t n) { return (n + 255) / 256 * 256; }

// Parts of the positions: workgroups for the device, and no part below one round of the four waves.  Three per CU, which is how many of a cache of codes run at
// once (us with 2, 3, 4, 6, 8, 12 per CU: four sequences of 131072 codes 196, 190, 223, 191, 198, 196; 48 of up to 4096 in FP16, where two run, 104, 92, 92, 91, 90, 93).
constexpr long kPerCu = 3;
struct Parts {
  int splits, per;
};
Parts parts_of(long groups, long most) {
  const long want = kPerCu * device_info().cus, rounds = ceil_div(most, kWaves * kStep);
  long splits = groups >= want || groups < 1 ? 1 : want / groups;
  if (splits > rounds) splits = rounds;
  if (splits > kMostParts) splits = kMostParts;
  if (splits < 1) splits = 1;
  const long per = ceil_div(rounds, splits) * kWaves * kStep;
  return {(int)(most > 0 ? ceil_div(most, per) : 1), (int)per};
}

void divisors(const AttendArgs& a, Pages& pg) {
  pg.groups = (uint32_t)((long)a.batch * a.kv * a.tiles);
  pg.by_groups = FastDiv::by(pg.groups);
  pg.by_tiles = FastDiv::by((uint32_t)a.tiles);
  pg.by_kv = FastDiv::by((uint32_t)a.kv);
  pg.by_rep = FastDiv::by((uint32_t)a.rep);
}
// weighted: positions that get weights
hipError_t finish(const AttendArgs& a, const Pages& pg, long weighted, hipStream_t st) {
  const long joins = a.splits > 1 ? (long)a.batch * a.heads * a.sq : 0, segments = ceil_div(weighted, kThreads), blocks = joins + (long)a.batch * a.kv * segments;
  if (blocks > 0) finish_kernel<<<(unsigned)blocks, kThreads, 0, st>>>(a, pg, joins, (int)segments);
  return hipGetLastError();
}

constexpr long kOwnWeights = 1024;      // four positions a thread
struct Room {
  size_t stats, part, scores;      // bytes
  Parts p;
};
Room room(long batch, long heads, long kv, long rows_per_kv, long sq, long dh, long most, bool weights) {
  Room r{};
  r.p = parts_of(batch * kv * ceil_div(rows_per_kv, 16), most);
  const size_t rows = (size_t)batch * heads * sq;
  // (one part of all of a key head's rows and not many positions: its workgroup adds the weights itself)
  if (r.p.splits > 1 || (weights && (rows_per_kv > 16 || most > kOwnWeights))) r.stats = up256(r.p.splits * rows * 8);
  if (r.p.splits > 1) r.part = up256(r.p.splits * rows * dh * 4);
  if (weights) r.scores = rows * ((most + 31) / 32 * 32) * 4;
  return r;
}

}  // namespace

size_t paged_workspace_bytes(long batch, long heads, long kv, long dh, long most, bool weights) {
  const Room r = room(batch, heads, kv, heads / kv, 1, dh, most, weights);
  return r.stats + r.part + r.scores;
}

hipError_t launch_paged(const PagedCall& c, void* workspace, hipStream_t st) {
  const long rep = c.heads / c.kv_heads;
  const Room r = room(c.batch, c.heads, c.kv_heads, rep, 1, c.dh, c.max_len, c.weights != nullptr);
  AttendArgs a{};
  a.q = Side{(const _Float16*)c.Q, c.ldq, c.dh, 0};
  a.klen = c.len;
  a.out = (_Float16*)c.O;
  a.out_batch = c.ldo;
  a.out_head = c.dh;
  uint8_t* ws = (uint8_t*)workspace;
  a.stats = r.stats ? (float2*)ws : nullptr;
  a.part = (float*)(ws + r.stats);
  a.part_stride = c.batch * c.heads * c.dh;
  a.batch = (int)c.batch;
  a.heads = (int)c.heads;
  a.kv = (int)c.kv_heads;
  a.rep = (int)rep;
  a.sq = 1;
  const long held = c.cache.table_ld << c.cache.shift;
  a.sk = (int)(c.max_len < held ? c.max_len : held);
  a.dh = (int)c.dh;
  a.tiles = (int)ceil_div(rep, 16);
  a.splits = r.p.splits;
  a.per_split = r.p.per;
  a.c2 = (float)(1.0 / sqrt((double)c.dh) * 1.44269504088896340736);
  a.alpha = c.alpha;
  Pages pg{(const uint8_t*)c.cache.k, (const uint8_t*)c.cache.v, c.cache.table, (float*)c.weights, c.weights ? (float*)(ws + r.stats + r.part) : nullptr,
           (c.max_len + 31) / 32 * 32, c.cache.table_ld, c.cache.pages, c.cache.shift};
  const long blocks = c.batch * c.kv_heads * a.tiles * a.splits;
  divisors(a, pg);
  auto go = [&](auto kernel, int lds) {
    kernel<<<(unsigned)blocks, kThreads, lds, st>>>(a, pg);
    return hipGetLastError();
  };
  const hipError_t e = c.cache.fp8 ? with_kernel<true, true>(c.dh, go) : with_kernel<false, true>(c.dh, go);
  if (e != hipSuccess) return e;
  return finish(a, pg, c.weights && a.stats ? c.max_len : 0, st);
}

// Up to one tile of rows.  us of this kernel, and of the forward kernel of many queries (us_cross.hip): 32 x 16 heads of 64 over 1500 keys, 1 / 16 rows 37.6 / 38.2, 48.4 / 42.8;
// 2 x 32 by 8 of 128 over 8192, 16 rows 21.4, 20.7; one of 8 heads of 64 over 20000, 8 rows 13.1, 13.1; 16 x 16 of 64 over 512, 1 / 16 rows 14.3 / 18.1, 11.5 / 11.3; 4 x 8 of 256
// over 1500, 1 / 16 rows 23.0 / 28.3, 21.9 / 22.1.  Two tiles, 32 rows: 58 and 43, 30.0 and 21.0, 14.0 and 13.8, 14.0 and 11.5, 42 and 23.
bool few_rows_take(long heads, long kv_heads, long sq) { return sq * (heads / kv_heads) <= 16; }
size_t few_rows_workspace_bytes(long batch, long heads, long kv, long sq, long sk, long dh) {
  const Room r = room(batch, heads, kv, heads / kv * sq, sq, dh, sk, false);
  return r.stats + r.part;
}
// `a` as the forward kernel of us_cross.hip takes it
hipError_t launch_few_rows(AttendArgs a, void* workspace, hipStream_t st) {
  Room r = room(a.batch, a.heads, a.kv, (long)a.rep * a.sq, a.sq, a.dh, a.sk, false);
  if (!workspace) r = Room{0, 0, 0, {1, (int)(ceil_div(a.sk, kWaves * kStep) * kWaves * kStep)}};
  a.stats = r.stats ? (float2*)workspace : nullptr;
  a.part = (float*)((uint8_t*)workspace + r.stats);
  a.part_stride = (long)a.batch * a.heads * a.sq * a.dh;
  a.tiles = 1;
  a.splits = r.p.splits;
  a.per_split = r.p.per;
  const long blocks = (long)a.batch * a.kv * a.splits;
  Pages pg{};
  divisors(a, pg);
  const hipError_t e = with_kernel<false, false>(a.dh, [&](auto kernel, int lds) {
    kernel<<<(unsigned)blocks, kThreads, lds, st>>>(a, pg);
    return hipGetLastError();
  });
  return e != hipSuccess || a.splits == 1 ? e : finish(a, Pages{}, 0, st);
}

}  // namespace us
