// Attention of sq queries over the first n keys of another sequence, forward and backward, without storing the scores.
//   forward   p = softmax(c q k), c = dh^-1/2;  O = a sum p v;  L = ln sum exp(c q k)
//   backward  P = a p = exp(c q k - L + ln a),  D = dO O / a = sum p (dO v),  dS = P (dO v - D)
//             dQ = c dS K,  dK = b c dS^T Q,  dV = b P^T dO
// The matrix core gets keys (forward, dQ) or queries (dK, dV) as its first operand, so that a lane holds one query (one key) and sixteen of the
// other side: the softmax statistics are scalars of a lane, and its sixteen results are, rounded to FP16, the second operand of the next
// product as they lie; the first operand is the tile in LDS, read transposed in the same order.
#include "us_flash.h"

namespace us {

namespace {

constexpr int kThreads = 256, kWaves = 4;
constexpr int kRows = 32 * kWaves;      // queries of a forward or dQ workgroup, keys of a dK / dV workgroup

// A lane's fragments of its row (second operand): columns 16 t + 8 half ..
template <int NB>
__device__ __forceinline__ void load_fragments(v8h (&f)[2 * NB], const _Float16* row, bool on, int dh, int half) {
#pragma unroll
  for (int t = 0; t < 2 * NB; ++t) {
    const int col = 16 * t + 8 * half;
    f[t] = v8h{0, 0, 0, 0, 0, 0, 0, 0};
    if (on && col < dh) f[t] = *reinterpret_cast<const v8h*>(row + col);
  }
}

// ---- forward -----------------------------------------------------------------------------------------------------------
template <int NB>
struct FwdCfg {
  static constexpr int BK = NB <= 4 ? 64 : 32;
  static constexpr int TILE = BK * RowTile<NB>::P, LDS = 4 * TILE;
};

template <int NB>
__global__ void __launch_bounds__(kThreads, NB <= 4 ? 2 : 1) cross_fwd_kernel(AttendArgs a) {
  using C = FwdCfg<NB>;
  using T = RowTile<NB>;
  constexpr int BK = C::BK, KB = BK / 32;
  extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
  const int lane = threadIdx.x & 63, l32 = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  long group, item;
  group_item(blockIdx.x, (long)a.batch * a.kv, (long)a.rep * a.tiles * a.splits, a.xcds, group, item);
  const int b = (int)(group / a.kv), kvh = (int)(group % a.kv);
  const int tile = (int)(item % a.tiles), split = (int)(item / a.tiles % a.splits), head = kvh * a.rep + (int)(item / a.tiles / a.splits);
  const int n = a.keys_of(b);
  const int begin = split * a.per_split, end = begin + a.per_split < n ? begin + a.per_split : n;
  const int q = tile * kRows + wave * 32 + l32;
  const bool on = q < a.sq;
  const _Float16* K = a.k.p + b * a.k.batch + kvh * a.k.head;
  const _Float16* V = a.v.p + b * a.v.batch + kvh * a.v.head;

  TileLoads<NB, BK, kThreads> loads;
  loads.init(a.k.row, a.dh);
  auto request = [&](int key, int buffer) {
    uint8_t* to = lds + buffer * 2 * C::TILE;
    loads.request((const uint8_t*)K + (long)key * a.k.row, n - key, a.k.row, a.dh, to, wave);
    loads.request((const uint8_t*)V + (long)key * a.v.row, n - key, a.v.row, a.dh, to + C::TILE, wave);
  };
  if (begin < end) request(begin, 0);
  v8h qf[2 * NB];
  load_fragments<NB>(qf, (const _Float16*)((const uint8_t*)(a.q.p + b * a.q.batch + head * a.q.head) + (long)q * a.q.row), on, a.dh, half);

  v16f acc[NB];
#pragma unroll
  for (int j = 0; j < NB; ++j) acc[j] = zero16();
  float m = -__builtin_inff(), sum = 0.0f;      // largest raw score, this lane's part of the sum
  for (int key = begin, i = 0; key < end; key += BK, ++i) {
    wait_all();
    __builtin_amdgcn_s_barrier();               // tile i has landed for everyone, tile i - 1 is used up
    if (key + BK < end) request(key + BK, (i + 1) & 1);
    const uint8_t *kt = lds + (i & 1) * 2 * C::TILE, *vt = kt + C::TILE;
    v16f s[KB];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      s[kb] = zero16();
#pragma unroll
      for (int t = 0; t < 2 * NB; ++t) s[kb] = mfma32(T::row_fragment(kt, kb, t, l32, half), qf[t], s[kb]);
    }
    if (key + BK > end) {
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (key + kb * 32 + 8 * (r / 4) + 4 * half + r % 4 >= end) s[kb][r] = -__builtin_inff();
    }
    float top = s[0][0];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) top = __builtin_fmaxf(top, s[kb][r]);
    top = __builtin_fmaxf(m, halves_max(top));
    const float f = __builtin_amdgcn_exp2f((m - top) * a.c2), neg = -top * a.c2;
    const bool moved = top > m;
    m = top;
    if (__builtin_amdgcn_ballot_w64(moved)) {
      sum *= f;
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[j][r] *= f;
    }
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[kb][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kb][r], a.c2, neg));
        sum += s[kb][r];
      }
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const v8h p = round8(s[kb], t);
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[j] = mfma32(T::column_fragment(vt, 2 * kb + t, j, lane), p, acc[j]);
      }
  }
  sum = halves_sum(sum);
  const long row = ((long)b * a.heads + head) * a.sq + q;
  if (a.splits > 1) {
    float* out = a.part + split * a.part_stride + row * a.dh;
    if (begin < end) {
#pragma unroll
      for (int j = 0; j < NB; ++j) store_block_f32(out, 32 * j, a.dh, on, half, acc[j], 1.0f);
    }
    if (on && half == 0) a.stats[split * (a.part_stride / a.dh) + row] = make_float2(m * a.c2, sum);
    return;
  }
  const float alpha = a.alpha > 0.0f ? a.alpha : __builtin_sqrtf((float)n);
  const float f = n > 0 ? alpha / sum : 0.0f;
  _Float16* out = a.out + b * a.out_batch + head * a.out_head + (long)q * a.out_row;
#pragma unroll
  for (int j = 0; j < NB; ++j) store_block(out, 32 * j, a.dh, on, half, acc[j], f);
  if (a.lse && on && half == 0) a.lse[row] = n > 0 ? __builtin_fmaf(__builtin_amdgcn_logf(sum), kLn2F, m * a.c2 * kLn2F) : -__builtin_inff();
}

// The parts of split rows: O = a sum_s 2^(m_s - m) O_s / sum_s 2^(m_s - m) l_s; parts without keys have l_s = 0 and no O_s.  A wave per row.
__global__ void __launch_bounds__(kThreads) join_kernel(AttendArgs a, long rows) {
  const int lane = threadIdx.x & 63;
  const long row = (long)blockIdx.x * kWaves + (threadIdx.x >> 6);
  if (row >= rows) return;
  const long bh = row / a.sq;
  const int q = (int)(row - bh * a.sq), b = (int)(bh / a.heads), head = (int)(bh - (long)b * a.heads);
  const long stat_stride = a.part_stride / a.dh;
  float m = -__builtin_inff();
  for (int s = 0; s < a.splits; ++s) m = __builtin_fmaxf(m, a.stats[s * stat_stride + row].x);
  float sum = 0.0f, acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int s = 0; s < a.splits; ++s) {
    const float2 st = a.stats[s * stat_stride + row];
    if (st.y == 0.0f) continue;
    const float f = __builtin_amdgcn_exp2f(st.x - m);
    sum = __builtin_fmaf(f, st.y, sum);
    if (4 * lane < a.dh) {
      const v4f x = *reinterpret_cast<const v4f*>(a.part + s * a.part_stride + row * a.dh + 4 * lane);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] = __builtin_fmaf(f, x[e], acc[e]);
    }
  }
  const int n = a.keys_of(b);
  const bool any = sum != 0.0f;      // (NaN: some)
  const float f = any ? (a.alpha > 0.0f ? a.alpha : __builtin_sqrtf((float)n)) / sum : 0.0f;
  if (4 * lane < a.dh) {
    const v4h o = {to_half(acc[0] * f), to_half(acc[1] * f), to_half(acc[2] * f), to_half(acc[3] * f)};
    wt_store(reinterpret_cast<v4h*>(a.out + b * a.out_batch + head * a.out_head + (long)q * a.out_row + 4 * lane), o);
  }
  if (a.lse && lane == 0) a.lse[row] = any ? (m + __builtin_amdgcn_logf(sum)) * kLn2F : -__builtin_inff();
}

// ---- backward: what the rows need -----------------------------------------------------------------------------------------
// {log2(e) L - log2(a), D} of every query row, {inf, 0} of the rows that fill the last tile: their P is zero.  16 lanes a row.
__global__ void __launch_bounds__(kThreads) cross_rows_kernel(AttendArgs a, const float* lse, float2* rows, long total) {
  const int part = threadIdx.x & 15;
  const long i = (long)blockIdx.x * (kThreads / 16) + (threadIdx.x >> 4);
  if (i >= total) return;
  const long bh = i / a.sqp;
  const int q = (int)(i - bh * a.sqp), b = (int)(bh / a.heads), head = (int)(bh - (long)b * a.heads);
  float dot = 0.0f;
  const int n = a.keys_of(b);
  const bool on = q < a.sq && n > 0;
  if (on) {
    const _Float16* o = (const _Float16*)((const uint8_t*)(a.o.p + b * a.o.batch + head * a.o.head) + (long)q * a.o.row);
    const _Float16* g = (const _Float16*)((const uint8_t*)(a.g.p + b * a.g.batch + head * a.g.head) + (long)q * a.g.row);
    for (int c = part * 8; c < a.dh; c += 128) {
      const v8h x = *reinterpret_cast<const v8h*>(o + c), y = *reinterpret_cast<const v8h*>(g + c);
#pragma unroll
      for (int e = 0; e < 8; ++e) dot = __builtin_fmaf((float)x[e], (float)y[e], dot);
    }
  }
  dot = group_sum<16>(dot);
  if (part == 0) {
    const float alpha = a.alpha > 0.0f ? a.alpha : __builtin_sqrtf((float)n);
    rows[i] = on ? make_float2(__builtin_fmaf(lse[bh * a.sq + q], kLog2eF, -__builtin_amdgcn_logf(alpha)), dot / alpha) : make_float2(__builtin_inff(), 0.0f);
  }
}

// ---- backward: dK and dV ------------------------------------------------------------------------------------------------------
// Heads above 128 columns are accumulated in two halves by two workgroups, whose products with all columns are made twice: 512 registers hold no more.
template <int NB>
struct DkvCfg {
  static constexpr int HALVES = NB > 4 ? 2 : 1, ACC = NB / HALVES;
};
template <int NB>
__global__ void __launch_bounds__(kThreads, 1) cross_dkv_kernel(AttendArgs a) {
  using T = RowTile<NB>;
  constexpr int BQ = 32, TILE = BQ * T::P, HALVES = DkvCfg<NB>::HALVES, ACC = DkvCfg<NB>::ACC;
  extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
  const int lane = threadIdx.x & 63, l32 = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  long group, item;
  group_item(blockIdx.x, (long)a.batch * a.kv, (long)HALVES * a.tiles * a.splits, a.xcds, group, item);
  const int b = (int)(group / a.kv), kvh = (int)(group % a.kv), first = (int)(item % HALVES) * ACC;
  const int tile = (int)(item / HALVES % a.tiles), split = (int)(item / HALVES / a.tiles);
  const int n = a.keys_of(b);
  const int key = tile * kRows + wave * 32 + l32;
  const bool on = key < a.sk, live = key < n;
  // the tiles of the sharing heads' queries, one head after the other; a split takes per_split of them
  const int qtiles = (a.sq + BQ - 1) / BQ, total = a.rep * qtiles;
  const int begin = split * a.per_split;
  int end = begin + a.per_split < total ? begin + a.per_split : total;
  if (tile * kRows >= n) end = begin;

  TileLoads<NB, BQ, kThreads> lq, lg;
  lq.init(a.q.row, a.dh);
  lg.init(a.g.row, a.dh);
  auto request = [&](int i, int buffer) {
    const int head = kvh * a.rep + i / qtiles, q0 = i % qtiles * BQ;
    uint8_t* to = lds + buffer * 2 * TILE;
    lq.request((const uint8_t*)(a.q.p + b * a.q.batch + head * a.q.head) + (long)q0 * a.q.row, a.sq - q0, a.q.row, a.dh, to, wave);
    lg.request((const uint8_t*)(a.g.p + b * a.g.batch + head * a.g.head) + (long)q0 * a.g.row, a.sq - q0, a.g.row, a.dh, to + TILE, wave);
  };
  if (begin < end) request(begin, 0);
  v8h kf[2 * NB], vf[2 * NB];
  load_fragments<NB>(kf, (const _Float16*)((const uint8_t*)(a.k.p + b * a.k.batch + kvh * a.k.head) + (long)key * a.k.row), live, a.dh, half);
  load_fragments<NB>(vf, (const _Float16*)((const uint8_t*)(a.v.p + b * a.v.batch + kvh * a.v.head) + (long)key * a.v.row), live, a.dh, half);
  v16f dk[ACC], dv[ACC];
#pragma unroll
  for (int j = 0; j < ACC; ++j) dk[j] = dv[j] = zero16();

  for (int i = begin; i < end; ++i) {
    wait_all();
    __builtin_amdgcn_s_barrier();
    if (i + 1 < end) request(i + 1, (i + 1 - begin) & 1);
    const uint8_t *qt = lds + ((i - begin) & 1) * 2 * TILE, *gt = qt + TILE;
    const int head = kvh * a.rep + i / qtiles, q0 = i % qtiles * BQ;
    const float2* rows = a.rows + ((long)b * a.heads + head) * a.sqp + q0 + 4 * half;
    v16f s = zero16(), dp = zero16();
#pragma unroll
    for (int t = 0; t < 2 * NB; ++t) s = mfma32(T::row_fragment(qt, 0, t, l32, half), kf[t], s);
#pragma unroll
    for (int t = 0; t < 2 * NB; ++t) dp = mfma32(T::row_fragment(gt, 0, t, l32, half), vf[t], dp);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float2 ld = rows[8 * (r / 4) + r % 4];
      s[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], a.c2, -ld.x));
      dp[r] = s[r] * (dp[r] - ld.y);
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const v8h p = round8(s, t), ds = round8(dp, t);
#pragma unroll
      for (int j = 0; j < ACC; ++j) {
        dv[j] = mfma32(T::column_fragment(gt, t, first + j, lane), p, dv[j]);
        dk[j] = mfma32(T::column_fragment(qt, t, first + j, lane), ds, dk[j]);
      }
    }
  }
  const float c = a.c2 * kLn2F;
#pragma unroll
  for (int j = 0; j < ACC; ++j) {
    if (!live) dk[j] = dv[j] = zero16();
    if (n == 1) dk[j] = zero16();       // the softmax of one key has no gradient
  }
  if (a.splits > 1) {
    float* out = a.part + split * a.part_stride + (((long)b * a.kv + kvh) * a.sk + key) * 2 * a.dh;
#pragma unroll
    for (int j = 0; j < ACC; ++j) {
      store_block_f32(out, 32 * (first + j), a.dh, on, half, dk[j], c);
      store_block_f32(out + a.dh, 32 * (first + j), a.dh, on, half, dv[j], 1.0f);
    }
    return;
  }
  const long at = b * a.k.batch + kvh * a.k.head;
  _Float16 *pk = (_Float16*)((uint8_t*)(a.dk + at) + (long)key * a.k.row), *pv = (_Float16*)((uint8_t*)(a.dv + at) + (long)key * a.k.row);
#pragma unroll
  for (int j = 0; j < ACC; ++j) {
    store_block(pk, 32 * (first + j), a.dh, on, half, dk[j], c * a.beta);
    store_block(pv, 32 * (first + j), a.dh, on, half, dv[j], a.beta);
  }
}

// ---- backward: dQ ---------------------------------------------------------------------------------------------------------
template <int NB>
__global__ void __launch_bounds__(kThreads, NB <= 4 ? 2 : 1) cross_dq_kernel(AttendArgs a) {
  using T = RowTile<NB>;
  constexpr int BK = 32, TILE = BK * T::P;
  extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
  const int lane = threadIdx.x & 63, l32 = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  long group, item;
  group_item(blockIdx.x, (long)a.batch * a.kv, (long)a.rep * a.tiles * a.splits, a.xcds, group, item);
  const int b = (int)(group / a.kv), kvh = (int)(group % a.kv);
  const int tile = (int)(item % a.tiles), split = (int)(item / a.tiles % a.splits), head = kvh * a.rep + (int)(item / a.tiles / a.splits);
  const int n = a.keys_of(b);
  const int begin = split * a.per_split, end = begin + a.per_split < n ? begin + a.per_split : n;
  const int q = tile * kRows + wave * 32 + l32;
  const bool on = q < a.sq;
  const _Float16* K = a.k.p + b * a.k.batch + kvh * a.k.head;
  const _Float16* V = a.v.p + b * a.v.batch + kvh * a.v.head;
  TileLoads<NB, BK, kThreads> loads;
  loads.init(a.k.row, a.dh);
  auto request = [&](int key, int buffer) {
    uint8_t* to = lds + buffer * 2 * TILE;
    loads.request((const uint8_t*)K + (long)key * a.k.row, n - key, a.k.row, a.dh, to, wave);
    loads.request((const uint8_t*)V + (long)key * a.v.row, n - key, a.v.row, a.dh, to + TILE, wave);
  };
  if (begin < end) request(begin, 0);
  v8h qf[2 * NB], gf[2 * NB];
  load_fragments<NB>(qf, (const _Float16*)((const uint8_t*)(a.q.p + b * a.q.batch + head * a.q.head) + (long)q * a.q.row), on, a.dh, half);
  load_fragments<NB>(gf, (const _Float16*)((const uint8_t*)(a.g.p + b * a.g.batch + head * a.g.head) + (long)q * a.g.row), on, a.dh, half);
  const long row = ((long)b * a.heads + head);
  float2 ld = make_float2(__builtin_inff(), 0.0f);
  if (on) ld = a.rows[row * a.sqp + q];
  v16f acc[NB];
#pragma unroll
  for (int j = 0; j < NB; ++j) acc[j] = zero16();
  for (int key = begin, i = 0; key < end; key += BK, ++i) {
    wait_all();
    __builtin_amdgcn_s_barrier();
    if (key + BK < end) request(key + BK, (i + 1) & 1);
    const uint8_t *kt = lds + (i & 1) * 2 * TILE, *vt = kt + TILE;
    v16f s = zero16(), dp = zero16();
#pragma unroll
    for (int t = 0; t < 2 * NB; ++t) s = mfma32(T::row_fragment(kt, 0, t, l32, half), qf[t], s);
#pragma unroll
    for (int t = 0; t < 2 * NB; ++t) dp = mfma32(T::row_fragment(vt, 0, t, l32, half), gf[t], dp);
    if (key + BK > end) {
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (key + 8 * (r / 4) + 4 * half + r % 4 >= end) s[r] = -__builtin_inff();
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) dp[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], a.c2, -ld.x)) * (dp[r] - ld.y);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const v8h ds = round8(dp, t);
#pragma unroll
      for (int j = 0; j < NB; ++j) acc[j] = mfma32(T::column_fragment(kt, t, j, lane), ds, acc[j]);
    }
  }
  const float c = a.c2 * kLn2F;
  if (n == 1) {
#pragma unroll
    for (int j = 0; j < NB; ++j) acc[j] = zero16();
  }
  if (a.splits > 1) {
    float* out = a.part + split * a.part_stride + (row * a.sq + q) * a.dh;
#pragma unroll
    for (int j = 0; j < NB; ++j) store_block_f32(out, 32 * j, a.dh, on, half, acc[j], c);
    return;
  }
  _Float16* out = a.out + b * a.out_batch + head * a.out_head + (long)q * a.out_row;
#pragma unroll
  for (int j = 0; j < NB; ++j) store_block(out, 32 * j, a.dh, on, half, acc[j], c * a.beta);
}

// Sums of split gradients, part after part: `rows` rows of dh columns `row_stride` elements apart in a part; row = (batch * heads + head) * s + t.
__global__ void __launch_bounds__(kThreads) cross_sum_kernel(const float* part, long part_stride, long row_stride, int splits, long rows, int heads, int s, int dh,
                                                             _Float16* out, long out_batch, long out_head, long out_row, float beta) {
  const int per = dh / 4;
  const long i = (long)blockIdx.x * kThreads + threadIdx.x;
  const long row = i / per;
  if (row >= rows) return;
  const int col = (int)(i - row * per) * 4;
  const float* p = part + row * row_stride + col;
  v4f sum = *reinterpret_cast<const v4f*>(p);
  for (int k = 1; k < splits; ++k) {
    const v4f x = *reinterpret_cast<const v4f*>(p + k * part_stride);
#pragma unroll
    for (int e = 0; e < 4; ++e) sum[e] += x[e];
  }
  const long bh = row / s, t = row - bh * s, b = bh / heads, head = bh - b * heads;
  const v4h o = {to_half(sum[0] * beta), to_half(sum[1] * beta), to_half(sum[2] * beta), to_half(sum[3] * beta)};
  wt_store(reinterpret_cast<v4h*>(out + b * out_batch + head * out_head + t * out_row + col), o);
}

// f(integral_constant<int, NB>): blocks of 32 columns that hold a head
template <class F>
hipError_t with_blocks(long dh, F f) {
  if (dh <= 32) return f(std::integral_constant<int, 1>{});
  if (dh <= 64) return f(std::integral_constant<int, 2>{});
  if (dh <= 96) return f(std::integral_constant<int, 3>{});
  if (dh <= 128) return f(std::integral_constant<int, 4>{});
  if (dh <= 192) return f(std::integral_constant<int, 6>{});
  return f(std::integral_constant<int, 8>{});
}

Side side(const void* p, const us_heads_layout& l) { return Side{(const _Float16*)p, l.batch, l.head, (int)(2 * l.row)}; }

AttendArgs cross_args(const CrossCall& c) {
  AttendArgs a{};
  a.q = side(c.Q, c.lq);
  a.k = side(c.K, c.lkv);
  a.v = side(c.V, c.lkv);
  a.o = side(c.O, c.lo);
  a.g = side(c.dO, c.lo);
  a.klen = c.klen;
  a.batch = (int)c.batch;
  a.heads = (int)c.heads;
  a.kv = (int)c.kv_heads;
  a.rep = (int)(c.heads / c.kv_heads);
  a.sq = (int)c.sq;
  a.sqp = (int)((c.sq + 31) / 32 * 32);
  a.sk = (int)c.sk;
  a.dh = (int)c.dh;
  a.xcds = device_info().xcds;
  a.c2 = (float)(1.0 / sqrt((double)c.dh) * 1.44269504088896340736);
  a.alpha = c.alpha;
  return a;
}

long ceil_div(long a, long b) { return (a + b - 1) / b; }

// How a reduction of `steps` tiles is cut so that `items` workgroups become enough for the device.
struct Cut {
  int splits;
  long per;       // steps of a part
};
Cut cut(long items, long steps, long least) {
  const long want = 2l * device_info().cus;
  long splits = items >= want || items < 1 ? 1 : want / items;
  if (splits > steps / least) splits = steps / least;
  if (splits < 1) splits = 1;
  const long per = steps > 0 ? ceil_div(steps, splits) : 1;
  return {steps > 0 ? (int)ceil_div(steps, per) : 1, per};
}
Cut fwd_cut(const CrossCall& c) { return cut(c.batch * c.heads * ceil_div(c.sq, kRows), ceil_div(c.sk, 64), 4); }
Cut dq_cut(const CrossCall& c) { return cut(c.batch * c.heads * ceil_div(c.sq, kRows), ceil_div(c.sk, 32), 8); }
Cut dkv_cut(const CrossCall& c) { return cut(c.batch * c.kv_heads * ceil_div(c.sk, kRows), c.heads / c.kv_heads * ceil_div(c.sq, 32), 8); }

size_t up256(size_t n) { return (n + 255) / 256 * 256; }
size_t rows_bytes(const CrossCall& c) { return up256((size_t)c.batch * c.heads * ((c.sq + 31) / 32 * 32) * 8); }

template <class K>
hipError_t launch(K kernel, FuncConfig& config, long blocks, int lds, const AttendArgs& a, hipStream_t st) {
  if (const hipError_t e = config.ensure((const void*)kernel, lds); e != hipSuccess) return e;
  kernel<<<(unsigned)blocks, kThreads, lds, st>>>(a);
  return hipGetLastError();
}

}  // namespace

size_t cross_fwd_workspace_bytes(const CrossCall& c) {
  if (few_rows_take(c.heads, c.kv_heads, c.sq)) return few_rows_workspace_bytes(c.batch, c.heads, c.kv_heads, c.sq, c.sk, c.dh);
  const Cut s = fwd_cut(c);
  const size_t rows = (size_t)c.batch * c.heads * c.sq;
  return s.splits == 1 ? 0 : up256(s.splits * rows * 8) + s.splits * rows * c.dh * 4;
}
size_t cross_bwd_workspace_bytes(const CrossCall& c) {
  const Cut q = dq_cut(c), k = dkv_cut(c);
  const size_t nq = q.splits == 1 ? 0 : (size_t)q.splits * c.batch * c.heads * c.sq * c.dh * 4;
  const size_t nk = k.splits == 1 ? 0 : (size_t)k.splits * c.batch * c.kv_heads * c.sk * c.dh * 8;
  return rows_bytes(c) + (nq > nk ? nq : nk);
}

hipError_t launch_join(const AttendArgs& a, hipStream_t st) {
  const long rows = (long)a.batch * a.heads * a.sq;
  join_kernel<<<(unsigned)ceil_div(rows, kWaves), kThreads, 0, st>>>(a, rows);
  return hipGetLastError();
}

hipError_t launch_cross_fwd(const CrossCall& c, void* workspace, hipStream_t st) {
  AttendArgs a = cross_args(c);
  a.out = (_Float16*)c.O;
  a.out_batch = c.lo.batch;
  a.out_head = c.lo.head;
  a.out_row = c.lo.row;
  a.lse = c.lse;
  if (few_rows_take(c.heads, c.kv_heads, c.sq)) return launch_few_rows(a, workspace, st);
  a.tiles = (int)ceil_div(c.sq, kRows);
  Cut s = fwd_cut(c);
  if (!workspace) s = {1, ceil_div(c.sk, 64)};
  a.splits = s.splits;
  a.per_split = (int)(s.per * 64);
  const long rows = c.batch * c.heads * c.sq;
  a.stats = (float2*)workspace;
  a.part = (float*)((uint8_t*)workspace + up256((size_t)s.splits * rows * 8));
  a.part_stride = rows * c.dh;
  const hipError_t e = with_blocks(c.dh, [&](auto nb) {
    constexpr int NB = decltype(nb)::value;
    static FuncConfig config;
    return launch(cross_fwd_kernel<NB>, config, c.batch * c.heads * a.tiles * a.splits, FwdCfg<NB>::LDS, a, st);
  });
  if (e != hipSuccess || a.splits == 1) return e;
  return launch_join(a, st);
}

hipError_t launch_cross_bwd(const CrossCall& c, void* dQ, void* dK, void* dV, float beta_q, float beta_kv, void* workspace, hipStream_t st) {
  AttendArgs a = cross_args(c);
  float2* row_values = (float2*)workspace;
  a.rows = row_values;
  a.part = (float*)((uint8_t*)workspace + rows_bytes(c));
  const long total = c.batch * c.heads * a.sqp;
  hipError_t e = hipSuccess;
  if (total > 0) {
    cross_rows_kernel<<<(unsigned)ceil_div(total, kThreads / 16), kThreads, 0, st>>>(a, c.lse, row_values, total);
    if (e = hipGetLastError(); e != hipSuccess) return e;
  }

  AttendArgs k = a;
  k.dk = (_Float16*)dK;
  k.dv = (_Float16*)dV;
  k.beta = beta_kv;
  k.tiles = (int)ceil_div(c.sk, kRows);
  const Cut ks = dkv_cut(c);
  k.splits = ks.splits;
  k.per_split = (int)ks.per;
  k.part_stride = c.batch * c.kv_heads * c.sk * c.dh * 2;
  if (c.sk > 0) e = with_blocks(c.dh, [&](auto nb) {
    constexpr int NB = decltype(nb)::value;
    static FuncConfig config;
    return launch(cross_dkv_kernel<NB>, config, DkvCfg<NB>::HALVES * c.batch * c.kv_heads * k.tiles * k.splits, 4 * 32 * RowTile<NB>::P, k, st);
  });
  if (e != hipSuccess) return e;
  if (k.splits > 1) {
    const long rows = c.batch * c.kv_heads * c.sk;
    for (int i = 0; i < 2; ++i)
      cross_sum_kernel<<<(unsigned)ceil_div(rows * (c.dh / 4), kThreads), kThreads, 0, st>>>(k.part + i * c.dh, k.part_stride, 2 * c.dh, k.splits, rows, (int)c.kv_heads,
                                                                                            (int)c.sk, (int)c.dh, i ? k.dv : k.dk, c.lkv.batch, c.lkv.head, c.lkv.row, beta_kv);
    if (e = hipGetLastError(); e != hipSuccess) return e;
  }

  if (c.sq == 0) return e;
  a.out = (_Float16*)dQ;
  a.out_batch = c.lq.batch;
  a.out_head = c.lq.head;
  a.out_row = c.lq.row;
  a.beta = beta_q;
  a.tiles = (int)ceil_div(c.sq, kRows);
  const Cut qs = dq_cut(c);
  a.splits = qs.splits;
  a.per_split = (int)(qs.per * 32);
  a.part_stride = c.batch * c.heads * c.sq * c.dh;
  e = with_blocks(c.dh, [&](auto nb) {
    constexpr int NB = decltype(nb)::value;
    static FuncConfig config;
    return launch(cross_dq_kernel<NB>, config, c.batch * c.heads * a.tiles * a.splits, 4 * 32 * RowTile<NB>::P, a, st);
  });
  if (e != hipSuccess || a.splits == 1) return e;
  const long rows = c.batch * c.heads * c.sq;
  cross_sum_kernel<<<(unsigned)ceil_div(rows * (c.dh / 4), kThreads), kThreads, 0, st>>>(a.part, a.part_stride, c.dh, a.splits, rows, (int)c.heads, (int)c.sq, (int)c.dh, a.out,
                                                                                        a.out_batch, a.out_head, a.out_row, beta_q);
  return hipGetLastError();
}

}  // namespace us
