// Attention of a few query rows per key head (one new token's heads that share it) over many keys: over the pages of a cache, or over the rows of
// another sequence.
//   p = softmax(c q k), c = dh^-1/2;  O = a sum p v;  weights += sum of p over the rows
// Bound: HBM, keys and values are read once.  A workgroup takes 16 rows of a key head and a part of its positions, its four waves every fourth tile of
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

template <int NB, bool FP8, bool PAGED>
__global__ void __launch_bounds__(kThreads, NB <= 4 ? 2 : 1) few_rows_kernel(AttendArgs a, Pages pg) {
  using T = RowTile<NB>;
  constexpr int ES = FP8 ? 1 : 2, UNITS = FP8 ? (NB + 1) / 2 : NB;      // 16-byte chunks of a key per lane
  constexpr int CPR = FP8 ? 2 * NB : 4 * NB, VL = kStep * CPR / 64;     // ... of a row of values, and a lane's share of a tile
  extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
  const int lane = threadIdx.x & 63, l16 = lane & 15, l4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int nrows = a.sq * a.rep;
  const int split = (int)(blockIdx.x % a.splits), rb = (int)(blockIdx.x / a.splits % a.tiles);
  const long group = blockIdx.x / a.splits / a.tiles;
  const int b = (int)(group / a.kv), kvh = (int)(group % a.kv);
  const int n = a.keys_of(b);
  const int begin = split * a.per_split, end = begin + a.per_split < n ? begin + a.per_split : n;
  const int r0 = rb * 16 + l16, token = r0 / a.rep, head = kvh * a.rep + (r0 - token * a.rep);
  const bool on = r0 < nrows;
  uint8_t* vt = lds + wave * kStep * T::P;

  // the rows' fragments; the columns that a lane's chunk of a key holds
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
  const v4i zero4 = {0, 0, 0, 0};
  const long row_bytes = PAGED ? (long)a.dh * ES : a.k.row;
  // the base of the 16 positions at `pos`, or NULL: beyond the end, or on a page that there is not
  auto block_of = [&](int pos, const uint8_t* base) -> const uint8_t* {
    if (pos >= end) return nullptr;
    if constexpr (PAGED) {
      const int page = pg.table[(long)b * pg.table_ld + (pos >> pg.shift)];
      if (page < 0 || page >= pg.pages) return nullptr;
      return base + ((((long)page * a.kv + kvh) << pg.shift) + (pos & ((1 << pg.shift) - 1))) * row_bytes;
    } else {
      return base + (long)pos * row_bytes;
    }
  };
  const uint8_t* kbase = PAGED ? pg.k : (const uint8_t*)(a.k.p + b * a.k.batch + kvh * a.k.head);
  const uint8_t* vbase = PAGED ? pg.v : (const uint8_t*)(a.v.p + b * a.v.batch + kvh * a.v.head);

  v4f acc[2 * NB];
#pragma unroll
  for (int j = 0; j < 2 * NB; ++j) acc[j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
  float m = -__builtin_inff(), sum = 0.0f;
  for (int pos = begin + wave * kStep; pos < end; pos += kWaves * kStep) {
    const uint8_t *k0 = block_of(pos, kbase), *k1 = block_of(pos + 16, kbase), *v0 = block_of(pos, vbase), *v1 = block_of(pos + 16, vbase);
    v4i kr[2][UNITS], vr[VL];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint8_t* at = i ? k1 : k0;
      const bool live = at && pos + 16 * i + l16 < end;
#pragma unroll
      for (int t = 0; t < UNITS; ++t) {
        const int byte = (4 * t + l4) * 16;
        kr[i][t] = zero4;
        if (live && byte < a.dh * ES) kr[i][t] = *reinterpret_cast<const v4i*>(at + l16 * row_bytes + byte);
      }
    }
#pragma unroll
    for (int j = 0; j < VL; ++j) {
      const int x = j * 64 + lane, row = x / CPR, byte = (x - row * CPR) * 16;
      const uint8_t* at = row < 16 ? v0 : v1;
      vr[j] = zero4;
      if (at && pos + row < end && byte < a.dh * ES) vr[j] = *reinterpret_cast<const v4i*>(at + (row & 15) * row_bytes + byte);
    }
    // scores of 2 x 16 positions: a lane holds its row's 4 l4 .. + 3 of either
    v4f s[2];
    float top = -__builtin_inff();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      s[i] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int t = 0; t < UNITS; ++t) {
        if constexpr (FP8) {
          s[i] = mfma16(codes8(kr[i][t][0], kr[i][t][1]), qf[2 * t], s[i]);
          s[i] = mfma16(codes8(kr[i][t][2], kr[i][t][3]), qf[2 * t + 1], s[i]);
        } else {
          s[i] = mfma16(__builtin_bit_cast(v8h, kr[i][t]), qf[t], s[i]);
        }
      }
      const bool there = i ? k1 != nullptr : k0 != nullptr;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s[i][e] *= a.c2;
        if (!there || pos + 16 * i + 4 * l4 + e >= end) s[i][e] = -__builtin_inff();
        top = __builtin_fmaxf(top, s[i][e]);
      }
      if (PAGED && pg.scores && on && pos + 16 * i < end)
        *reinterpret_cast<v4f*>(pg.scores + ((long)b * a.heads + head) * pg.score_ld + pos + 16 * i + 4 * l4) = s[i];
    }
    top = __builtin_fmaxf(m, row_reduce(top, [](float x, float y) { return __builtin_fmaxf(x, y); }));
    // (positions that are all on pages that there are not: nothing is there yet)
    const float use = top == -__builtin_inff() ? 0.0f : top;
    const float f = __builtin_amdgcn_exp2f(m - use);
    m = top;
    sum *= f;
#pragma unroll
    for (int j = 0; j < 2 * NB; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[j][e] *= f;
    v8h p;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x = __builtin_amdgcn_exp2f(s[i][e] - use);
        sum += x;
        p[4 * i + e] = (_Float16)x;
      }
    // the values through LDS, which only this wave uses
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int j = 0; j < VL; ++j) {
      const int x = j * 64 + lane, row = x / CPR, chunk = x - row * CPR;
      uint8_t* to = vt + row * T::P;
      if constexpr (FP8) {
        *US_LDS_AT(v8h, to + (((2 * chunk) ^ T::swz(row)) << 4)) = codes8(vr[j][0], vr[j][1]);
        *US_LDS_AT(v8h, to + (((2 * chunk + 1) ^ T::swz(row)) << 4)) = codes8(vr[j][2], vr[j][3]);
      } else {
        *US_LDS_AT(v4i, to + ((chunk ^ T::swz(row)) << 4)) = vr[j];
      }
    }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int j = 0; j < 2 * NB; ++j) {
      // lane: column 16 j + l16, positions 4 l4 .. + 3 of either sixteen
      const int row = 4 * l4 + (l16 >> 2), chunk = 2 * j + ((l16 & 3) >> 1);
      const v4s x = __builtin_amdgcn_ds_read_tr16_b64_v4i16(US_LDS_AT(v4s, vt + row * T::P + ((chunk ^ T::swz(row)) << 4) + (l16 & 1) * 8));
      const v4s y = __builtin_amdgcn_ds_read_tr16_b64_v4i16(US_LDS_AT(v4s, vt + (row + 16) * T::P + ((chunk ^ T::swz(row + 16)) << 4) + (l16 & 1) * 8));
      struct { v4s x, y; } both = {x, y};
      acc[j] = mfma16(__builtin_bit_cast(v8h, both), p, acc[j]);
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
  const float alpha = a.alpha > 0.0f ? a.alpha : __builtin_sqrtf((float)n);
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
    if (col == 0 && (parts || a.stats)) a.stats[split * (a.part_stride / a.dh) + at] = make_float2(top, total);
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
}

// weights of 256 positions of a key head: += sum over its rows of 2^(s - m) / l, m and l joined from the parts
__global__ void __launch_bounds__(kThreads) weights_kernel(AttendArgs a, Pages pg, int segments) {
  __shared__ float ms[64], inv[64];
  const int seg = (int)(blockIdx.x % segments);
  const long group = blockIdx.x / segments;
  const int b = (int)(group / a.kv), kvh = (int)(group % a.kv);
  const int n = a.keys_of(b), pos = seg * kThreads + (int)threadIdx.x;
  if (seg * kThreads >= n) return;
  const long stride = a.part_stride / a.dh;
  float w = 0.0f;
  for (int r0 = 0; r0 < a.rep; r0 += 64) {
    __syncthreads();
    const int r = r0 + (int)threadIdx.x;
    if (threadIdx.x < 64 && r < a.rep) {
      const long row = (long)b * a.heads + kvh * a.rep + r;
      float m = -__builtin_inff(), sum = 0.0f;
      for (int s = 0; s < a.splits; ++s) m = __builtin_fmaxf(m, a.stats[s * stride + row].x);
      for (int s = 0; s < a.splits; ++s) {
        const float2 st = a.stats[s * stride + row];
        if (st.y != 0.0f) sum = __builtin_fmaf(__builtin_amdgcn_exp2f(st.x - m), st.y, sum);
      }
      ms[threadIdx.x] = m;
      inv[threadIdx.x] = 1.0f / sum;
    }
    __syncthreads();
    if (pos < n) {
      const float* s = pg.scores + ((long)b * a.heads + kvh * a.rep + r0) * pg.score_ld + pos;
      const int most = a.rep - r0 < 64 ? a.rep - r0 : 64;
      for (int i = 0; i < most; ++i) w = __builtin_fmaf(__builtin_amdgcn_exp2f(s[i * pg.score_ld] - ms[i]), inv[i], w);
    }
  }
  if (pos >= n) return;
  const int page = pg.table[(long)b * pg.table_ld + (pos >> pg.shift)];
  if (page < 0 || page >= pg.pages) return;
  pg.weights[(((long)page * a.kv + kvh) << pg.shift) + (pos & ((1 << pg.shift) - 1))] += w;
}

template <bool FP8, bool PAGED, class F>
hipError_t with_kernel(long dh, F f) {
  auto go = [&](auto nb) {
    constexpr int NB = decltype(nb)::value;
    static FuncConfig config;
    constexpr int lds = kWaves * kStep * RowTile<NB>::P;
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

// Parts of the positions: workgroups for the device, and no part below one round of the four waves.
struct Parts {
  int splits, per;
};
Parts parts_of(long groups, long most) {
  const long want = 4l * device_info().cus, rounds = ceil_div(most, kWaves * kStep);
  long splits = groups >= want || groups < 1 ? 1 : want / groups;
  if (splits > rounds) splits = rounds;
  if (splits < 1) splits = 1;
  const long per = ceil_div(rounds, splits) * kWaves * kStep;
  return {(int)(most > 0 ? ceil_div(most, per) : 1), (int)per};
}

struct Room {
  size_t stats, part, scores;      // bytes
  Parts p;
};
Room room(long batch, long heads, long kv, long rows_per_kv, long sq, long dh, long most, bool weights) {
  Room r{};
  r.p = parts_of(batch * kv * ceil_div(rows_per_kv, 16), most);
  const size_t rows = (size_t)batch * heads * sq;
  if (r.p.splits > 1 || weights) r.stats = up256(r.p.splits * rows * 8);
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
  auto go = [&](auto kernel, int lds) {
    kernel<<<(unsigned)blocks, kThreads, lds, st>>>(a, pg);
    return hipGetLastError();
  };
  hipError_t e = c.cache.fp8 ? with_kernel<true, true>(c.dh, go) : with_kernel<false, true>(c.dh, go);
  if (e != hipSuccess) return e;
  if (a.splits > 1)
    if (e = launch_join(a, st); e != hipSuccess) return e;
  if (c.weights && c.max_len > 0) {
    const long segments = ceil_div(c.max_len, kThreads);
    weights_kernel<<<(unsigned)(c.batch * c.kv_heads * segments), kThreads, 0, st>>>(a, pg, (int)segments);
    e = hipGetLastError();
  }
  return e;
}

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
  const hipError_t e = with_kernel<false, false>(a.dh, [&](auto kernel, int lds) {
    kernel<<<(unsigned)blocks, kThreads, lds, st>>>(a, Pages{});
    return hipGetLastError();
  });
  return e != hipSuccess || a.splits == 1 ? e : launch_join(a, st);
}

}  // namespace us
