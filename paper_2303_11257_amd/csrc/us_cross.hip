// Attention of sq queries over the first n keys of another sequence, forward and backward, without storing the scores.
//   forward   p = softmax(c q k), c = dh^-1/2;  O = a sum p v;  L = ln sum exp(c q k)
//   backward  P = f p = exp(c q k - L + ln f),  D = dO O / a = sum p (dO v),  dS = P (dO v - D)
//             dQ = a / f c dS K,  dK = a / f b c dS^T Q,  dV = a / f b P^T dO        (f: AttendArgs::inner_factor)
// The matrix core gets keys (forward, dQ) or queries (dK, dV) as its first operand, so that a lane holds one query (one key) and sixteen of the
// other side: the softmax statistics are scalars of a lane, and its sixteen results are, rounded to FP16, the second operand of the next
// product as they lie; the first operand is the tile in LDS, read transposed in the same order.
// Two products and an exponential per score forward, three for dQ, four for dK and dV.  2 x 32 by 8 heads of 128, 4096 over 8192: forward 1065 to 1145 us by card (1.0 PFLOP/s) and
// dQ 1475 to 1600 (1.1), bound by power (1.7 GHz, matrix core busy 58 and 64 % of a CU's busy cycles, vector ALU 47 and 39); dK and dV 2230 to 2390 (0.96), bound by latency (49 and
// 29 %; 1.9 to 2.2 GHz by card): a wave's gradients fill half of the registers.  16 x 16 heads of 64, 512 over 64 to 1024: 31, 46 and 67: matrix core busy 36, 40 and 38 %, vector ALU
// (which the products' issue is part of) 70, 60 and 37 %, one after the other for the most part, and CUs busy for 63 to 70 % of the time, for the items' lengths differ.
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

// Row r of a key head: query q of its h-th head.
struct RowAt {
  int h, q, head;
  __device__ __forceinline__ RowAt(const AttendArgs& a, int kvh, int r) {
    h = (int)a.by_sq.of((uint32_t)r);
    q = r - h * a.sq;
    head = kvh * a.rep + h;
  }
  __device__ __forceinline__ long of_all(const AttendArgs& a, int b) const { return ((long)b * a.heads + head) * a.sq + q; }
};
// The lane, and its row of a wave's 32 from row0 on, worked out anew: no register holds it through the loop over the keys (the forward kernel of 64 columns, 512 x 1024: 130
// registers a lane and three waves a SIMD 38 us, 126 and four 34).
__device__ __forceinline__ int lane_again() {
  int t = threadIdx.x;
  asm volatile("" : "+v"(t));
  return t & 63;
}
__device__ __forceinline__ int row_again(int row0) { return row0 + (lane_again() & 31); }
// The number of keys, likewise for what is worked out from it.
__device__ __forceinline__ int keys_again(int n) {
  asm volatile("" : "+s"(n));
  return n;
}
// Where the rows of a key head's O or dQ start, and those of dK or dV.  (No reference to the kernel's arguments: those are then no longer scalars.)
struct RowsOfHeads {
  FastDiv by_sq;
  _Float16* base;
  long head, row;
  int sq, rows;
  __device__ __forceinline__ RowsOfHeads(const AttendArgs& a, int b, int kvh, int nrows)
      : by_sq(a.by_sq), base(a.out + b * a.out_batch + kvh * a.rep * a.out_head), head(a.out_head), row(a.out_row), sq(a.sq), rows(nrows) {}
  __device__ __forceinline__ _Float16* operator()(int r) const {
    if (r >= rows) return nullptr;
    const int h = (int)by_sq.of((uint32_t)r);
    return base + h * head + (r - h * sq) * row;
  }
};
struct RowsOf {
  uint8_t* base;
  int row_bytes, rows;
  __device__ __forceinline__ _Float16* operator()(int r) const { return r < rows ? (_Float16*)(base + (long)r * row_bytes) : nullptr; }
};

// ---- forward -----------------------------------------------------------------------------------------------------------
template <int NB>
struct FwdCfg {
  // (two blocks of 32 keys at a time, so that a product need not wait for the one before it; above 128 columns as well: 64 heads of 192, 1024 x 1024, 103 -> 97 us, ragged
  // batches of 256 columns 172 -> 160 and 264 -> 234)
  static constexpr int BK = 64, STAGES = 2;
  static constexpr int TILE = BK * RowTile<NB>::P, LDS = STAGES * 2 * TILE;
};

// Fragments of rows that are on their way from LDS to the matrix core.
template <int NB>
constexpr int kAhead = NB == 1 ? 2 : 4;

// step(integral_constant<int, buffer>, key) for every tile, the buffers in turn
template <int STAGES, class F>
__device__ __forceinline__ void for_stages(int begin, int end, int tile, F step) {
  for (int key = begin; key < end; key += STAGES * tile) {
    step(std::integral_constant<int, 0>{}, key);
    if (key + tile < end) step(std::integral_constant<int, 1>{}, key + tile);
    if constexpr (STAGES > 2) {
      if (key + 2 * tile < end) step(std::integral_constant<int, 2>{}, key + 2 * tile);
      if (key + 3 * tile < end) step(std::integral_constant<int, 3>{}, key + 3 * tile);
    }
  }
  if constexpr (STAGES > 2) tile_landed();      // zeros that were still on their way
}

// A row's maximum follows its scores only when they outgrow it by 2^kSlack: probabilities are then up to 2^kSlack in between, which FP16 and FP32 hold as exactly,
// and the sums are hardly ever multiplied again.
constexpr float kSlack = 8.0f;

template <int NB>
__global__ void __launch_bounds__(kThreads, NB <= 4 ? 2 : 1) cross_fwd_kernel(AttendArgs a) {
  using C = FwdCfg<NB>;
  constexpr int BK = C::BK, KB = BK / 32;
  extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
  const int lane = threadIdx.x & 63, l32 = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Items::Item it = a.items.at(blockIdx.x);
  if (it.b < 0) return;
  const int b = a.by_keys(it.b), kvh = it.kvh, split = it.y, row0 = it.x * kRows + wave * 32;
  const int n = a.keys_of(b);
  const int begin = split * a.per_split, end = begin + a.per_split < n ? begin + a.per_split : n;
  // the queries of the heads that share a key head are the rows of its tiles, one head after the other
  const int nrows = a.rep * a.sq;
  const bool on = row0 + l32 < nrows;
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
  {
    const RowAt mine(a, kvh, row0 + l32);
    load_fragments<NB>(qf, (const _Float16*)((const uint8_t*)(a.q.p + b * a.q.batch + mine.head * a.q.head) + (long)mine.q * a.q.row), on, a.dh, half);
  }
  TileReads<NB> at;
  at.init(lane);

  v16f acc[NB];
#pragma unroll
  for (int j = 0; j < NB; ++j) acc[j] = zero16();
  float m = -__builtin_inff(), sum = 0.0f;      // largest raw score, this lane's part of the sum
  const float slack = kSlack / a.c2;
  constexpr int N = KB * 2 * NB, AHEAD = kAhead<NB>;
  // raw scores of a tile of keys; each fragment is read while its predecessors are multiplied
  auto scores = [&](const uint8_t* kt, v16f (&x)[KB]) {
    // (the blocks of 32 keys in turn: a product that adds to the one just before it has to wait for it)
    v8h kf[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) kf[i] = at.rows(kt, i % KB, i / KB);
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) x[kb] = zero16();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      x[i % KB] = mfma32(kf[i % AHEAD], qf[i / KB], x[i % KB]);
      if (i + AHEAD < N) kf[i % AHEAD] = at.rows(kt, (i + AHEAD) % KB, (i + AHEAD) / KB);
    }
  };
  // ... made part of the running statistics
  auto follow = [&](v16f (&x)[KB], int key) {
    if (key + BK > end) {
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (key + kb * 32 + 8 * (r / 4) + 4 * half + r % 4 >= end) x[kb][r] = -__builtin_inff();
    }
    float top = x[0][0];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) top = __builtin_fmaxf(top, x[kb][r]);
    top = halves_max(top);
    const bool moved = top > m + slack;
    if (__builtin_amdgcn_ballot_w64(moved)) {
      const float f = moved ? __builtin_amdgcn_exp2f((m - top) * a.c2) : 1.0f;
      if (moved) m = top;
      sum *= f;
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[j][r] *= f;
    }
  };
  auto step = [&](auto buffer, int key) {
    constexpr int B = decltype(buffer)::value;
    tile_landed();                              // this tile has landed for everyone, the one before it is used up
    if (key + BK < end) request(key + BK, B ^ 1);
    const uint8_t *kt = lds + B * 2 * C::TILE, *vt = kt + C::TILE;
    v16f s[KB];
    v8h vf[NB], p[2 * KB];
    __builtin_amdgcn_sched_barrier(0);
    scores(kt, s);
#pragma unroll
    for (int j = 0; j < NB; ++j) vf[j] = at.columns(vt, 0, j);
    next_lds_reads<AHEAD>();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      next_mfma<1>();
      next_lds_reads<1>();
    }
    if constexpr (2 * NB > AHEAD) next_lds_reads<2 * NB - AHEAD>();
    __builtin_amdgcn_sched_barrier(0);
    follow(s, key);
    const float neg = -m * a.c2;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[kb][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kb][r], a.c2, neg));
        sum += s[kb][r];
      }
      p[2 * kb] = round8(s[kb], 0);
      p[2 * kb + 1] = round8(s[kb], 1);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int t = 0; t < 2 * KB; ++t)
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        acc[j] = mfma32(vf[j], p[t], acc[j]);
        if (t + 1 < 2 * KB) vf[j] = at.columns(vt, t + 1, j);
      }
#pragma unroll
    for (int t = 0; t < (2 * KB - 1) * NB; ++t) {
      next_mfma<1>();
      next_lds_reads<2>();
    }
    next_mfma<NB>();
    __builtin_amdgcn_sched_barrier(0);
  };
  for_stages<C::STAGES>(begin, end, BK, step);
  sum = halves_sum(sum);
  const long row = RowAt(a, kvh, row_again(row0)).of_all(a, b);
  if (a.splits > 1) {
    float* out = a.part + split * a.part_stride + row * a.dh;
    if (begin < end) {
#pragma unroll
      for (int j = 0; j < NB; ++j) store_block_f32(out, 32 * j, a.dh, on, half, acc[j], 1.0f);
    }
    if (on && half == 0) a.stats[split * (a.part_stride / a.dh) + row] = make_float2(m * a.c2, sum);
    return;
  }
  const float f = n > 0 ? a.factor(n) / sum : 0.0f;
  store_rows<NB>(lds, acc, f, row0, RowsOfHeads(a, b, kvh, nrows), a.dh, 0, lane, wave);
  if (a.lse && on && half == 0) a.lse[row] = n > 0 ? __builtin_fmaf(__builtin_amdgcn_logf(sum), kLn2F, m * a.c2 * kLn2F) : -__builtin_inff();
}

// The parts of split rows: O = a sum_s 2^(m_s - m) O_s / sum_s 2^(m_s - m) l_s; parts without keys have l_s = 0 and no O_s.  A wave per row: its lanes read the
// statistics together, and `1 << log_lanes` of them (16 bytes each) a part's row, so that parts are read side by side.  (260 rows of two parts 4 us, the launch;
// 5152 of eleven 7, one part after the other 15.)
__global__ void __launch_bounds__(kThreads) join_kernel(AttendArgs a, long rows, int log_lanes) {
  const int lane = threadIdx.x & 63;
  const long row = (long)blockIdx.x * kWaves + (threadIdx.x >> 6);
  if (row >= rows) return;
  const long bh = row / a.sq;
  const int q = (int)(row - bh * a.sq), b = (int)(bh / a.heads), head = (int)(bh - (long)b * a.heads);
  const long stat_stride = a.part_stride / a.dh;
  const int group = lane >> log_lanes, groups = 64 >> log_lanes, col = (lane & ((1 << log_lanes) - 1)) * 4;
  float m = -__builtin_inff(), sum = 0.0f, acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int s0 = 0; s0 < a.splits; s0 += 64) {
    const float2 mine = s0 + lane < a.splits ? a.stats[(s0 + lane) * stat_stride + row] : make_float2(-__builtin_inff(), 0.0f);
    const float most = __builtin_fmaxf(m, wave_max(mine.x));
    // (no key yet: both are -inf)
    const float old = most == m ? 1.0f : __builtin_amdgcn_exp2f(m - most), f = mine.y == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(mine.x - most);
    sum = __builtin_fmaf(old, sum, wave_sum(mine.y == 0.0f ? 0.0f : f * mine.y));
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] *= old;
    m = most;
    const int here = a.splits - s0 < 64 ? a.splits - s0 : 64;
    for (int i = 0; i < here; i += 4 * groups) {
      v4f x[4];
      float fs[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int s = i + u * groups + group;
        fs[u] = __shfl(f, s & 63);
        if (s >= here) fs[u] = 0.0f;
        x[u] = fs[u] != 0.0f && col < a.dh ? *reinterpret_cast<const v4f*>(a.part + (s0 + s) * a.part_stride + row * a.dh + col) : v4f{};
      }
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] = __builtin_fmaf(fs[u], x[u][e], acc[e]);
    }
  }
  for (int step = 1 << log_lanes; step < 64; step <<= 1)
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] += __shfl_xor(acc[e], step);
  const int n = a.keys_of(b);
  const bool any = sum != 0.0f;      // (NaN: some)
  const float f = any ? a.factor(n) / sum : 0.0f;
  if (group == 0 && col < a.dh) {
    const v4h o = {to_half(acc[0] * f), to_half(acc[1] * f), to_half(acc[2] * f), to_half(acc[3] * f)};
    wt_store(reinterpret_cast<v4h*>(a.out + b * a.out_batch + head * a.out_head + (long)q * a.out_row + col), o);
  }
  if (a.lse && lane == 0) a.lse[row] = any ? (m + __builtin_amdgcn_logf(sum)) * kLn2F : -__builtin_inff();
}

// ---- backward: dQ ---------------------------------------------------------------------------------------------------------
// Comes first and leaves what dK and dV need of every query row, log2(e) L - log2(f) and D.
// D from the rounded O is off by 2^-12 |O| / a of dO, which next to dO v of n keys is 2^-12 (sum p^2)^1/2: of few keys as much as dS's own rounding, and of narrow heads more.
// Up to kFewKeys keys D is therefore the sum of p dO v itself, from products made twice.  The aim: a 2-norm error of dQ of at most 3.2e-4, a tenth above that of its two roundings
// to FP16 (2.93e-4), with queries of 1.5 and unit normal keys.  There, in 1e-4, of 100 / 256 / 1024 / 2000 keys: from O 16 columns 3.54 / 3.54 / 3.51 / 3.52, 32: 3.29 / 3.28 / 3.23 / 3.22,
// 64: 3.21 / 3.14 / 3.09 / 3.09, 96: 3.15 / 3.10 / 3.05 / 3.03, 128: 3.13 / 3.07 / 3.04 / 3.00; from the products 3.10 to 3.24, 3.02 to 3.07, 2.98 to 3.02, 2.96 to 2.98, 2.95 to 2.97.  (Queries of 3, whose
// rows are peaked: about 5.1, 4.5, 4.1, 4.0 and 4.0 from O, 3.2 to 3.4 and 3.0 to 3.2 from the products.)  So: all keys that one workgroup has up to 32 columns, 256 up to 64 (48: 3.20 there),
// 128 above.  Keys in parts, where workgroups are few, take O.  dQ of 16 x 16 heads, 512 queries, us from O and from the products: 32 columns, 64 to 1024 keys 33 and 46; 16 columns,
// 2000 keys 85 and 150; 64 columns, 256 keys 28.5 and 34; 128 columns, 128 keys 43 and 43.
template <int NB>
constexpr int kFewKeys = NB == 1 ? 1 << 30 : NB == 2 ? 256 : 128;
// Heads of up to 64 columns: 124 registers a lane, so four waves a SIMD.  Of up to 96: three, with fewer fragments read ahead (us: 4 x 32 heads by 8 of 96, 2048 x 2048 370 ->
// 339, 59 x 6 by 3, 470 x 547 70 -> 65; where a SIMD has one wave it loses half a microsecond of 10).
// Where a tile is one block of keys (dh > 128) three of them are on their way at a time (us: 32 heads of 256, ragged batch of 5, 869 x 528: 166 -> 156; 130 x 1030:
// 36 -> 33; the forward pass gains nothing by it: 112 -> 117, 26 -> 26).  Requests then go on behind the last tile, for zeros: every wave has as many loads on its way.
template <int NB>
struct DqCfg {
  static constexpr int BK = NB <= 4 ? 64 : 32, STAGES = NB <= 4 ? 2 : 4, TILE = BK * RowTile<NB>::P, LDS = STAGES * 2 * TILE;
};
template <int NB>
__global__ void __launch_bounds__(kThreads, NB <= 2 ? 4 : NB == 3 ? 3 : NB <= 4 ? 2 : 1) cross_dq_kernel(AttendArgs a) {
  using C = DqCfg<NB>;
  constexpr int BK = C::BK, KB = BK / 32, TILE = C::TILE;
  extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
  const int lane = threadIdx.x & 63, l32 = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Items::Item it = a.items.at(blockIdx.x);
  if (it.b < 0) return;
  const int b = a.by_keys(it.b), kvh = it.kvh, split = it.y, row0 = it.x * kRows + wave * 32;
  const int n = a.keys_of(b);
  const int begin = split * a.per_split, end = begin + a.per_split < n ? begin + a.per_split : n;
  // the queries of the heads that share a key head are the rows of its tiles, one head after the other
  const int nrows = a.rep * a.sq;
  const bool on = row0 + l32 < nrows;
  const _Float16* K = a.k.p + b * a.k.batch + kvh * a.k.head;
  const _Float16* V = a.v.p + b * a.v.batch + kvh * a.v.head;
  TileLoads<NB, BK, kThreads> loads;
  loads.init(a.k.row, a.dh);
  auto request = [&](int key, int buffer) {
    uint8_t* to = lds + buffer * 2 * TILE;
    loads.request((const uint8_t*)K + (long)key * a.k.row, n - key, a.k.row, a.dh, to, wave);
    loads.request((const uint8_t*)V + (long)key * a.v.row, n - key, a.v.row, a.dh, to + TILE, wave);
  };
  auto first_requests = [&] {
#pragma unroll
    for (int i = 0; i < C::STAGES - 1; ++i)
      if (begin + i * BK < end || (C::STAGES > 2 && begin < end)) request(begin + i * BK, i);
  };
  first_requests();
  v8h qf[2 * NB], gf[2 * NB];
  {
    const RowAt mine(a, kvh, row0 + l32);
    load_fragments<NB>(qf, (const _Float16*)((const uint8_t*)(a.q.p + b * a.q.batch + mine.head * a.q.head) + (long)mine.q * a.q.row), on, a.dh, half);
    load_fragments<NB>(gf, (const _Float16*)((const uint8_t*)(a.g.p + b * a.g.batch + mine.head * a.g.head) + (long)mine.q * a.g.row), on, a.dh, half);
  }
  TileReads<NB> at;
  at.init(lane);
  constexpr int AHEAD = NB == 3 ? 3 : kAhead<NB>, CA = NB == 3 ? 1 : NB <= 4 ? NB : 4;
  // raw scores and dO v of 32 keys, in turn: a product that adds to the one just before it has to wait for it
  auto products = [&](const uint8_t* kt, int kb, v16f& s, v16f& dp) {
    auto fragment = [&](int i) { return at.rows(i % 2 ? kt + TILE : kt, kb, i / 2); };
    v8h rf[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) rf[i] = fragment(i);
    s = dp = zero16();
#pragma unroll
    for (int i = 0; i < 4 * NB; ++i) {
      if (i % 2) dp = mfma32(rf[i % AHEAD], gf[i / 2], dp);
      else s = mfma32(rf[i % AHEAD], qf[i / 2], s);
      if (i + AHEAD < 4 * NB) rf[i % AHEAD] = fragment(i + AHEAD);
    }
  };
  auto mask = [&](v16f& s, int key) {
    if (key + 32 > end) {
      const int first = key + 4 * (lane_again() >> 5);
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (first + 8 * (r / 4) + r % 4 >= end) s[r] = -__builtin_inff();
    }
  };
  float2 ld = make_float2(__builtin_inff(), 0.0f);
  if (on && n > 0) ld.x = __builtin_fmaf(a.lse[RowAt(a, kvh, row_again(row0)).of_all(a, b)], kLog2eF, -__builtin_amdgcn_logf(a.inner_factor(n)));
  if (n > kFewKeys<NB> || (begin < end && end - begin < n)) {
    float dot = 0.0f;
    const RowAt mine(a, kvh, row_again(row0));
    const _Float16* o = (const _Float16*)((const uint8_t*)(a.o.p + b * a.o.batch + mine.head * a.o.head) + (long)mine.q * a.o.row);
#pragma unroll
    for (int t = 0; t < 2 * NB; ++t) {
      const int col = 16 * t + 8 * half;
      if (on && col < a.dh) {
        const v8h x = *reinterpret_cast<const v8h*>(o + col);
#pragma unroll
        for (int e = 0; e < 8; ++e) dot = __builtin_fmaf((float)x[e], (float)gf[t][e], dot);
      }
    }
    if (on) ld.y = halves_sum(dot) / a.factor(n);
  } else if (begin < end) {
    float ps = 0.0f, pd = 0.0f;
    for (int key = begin, buffer = 0; key < end; key += BK, buffer = (buffer + 1) % C::STAGES) {
      tile_landed<(C::STAGES - 2) * 2 * decltype(loads)::LD>();
      if (C::STAGES > 2 || key + BK < end) request(key + (C::STAGES - 1) * BK, (buffer + C::STAGES - 1) % C::STAGES);
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        v16f s, dp;
        products(lds + buffer * 2 * TILE, kb, s, dp);
        mask(s, key + 32 * kb);
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], a.c2, -ld.x));
          ps += p;
          pd = __builtin_fmaf(p, dp[r], pd);
        }
      }
    }
    ps = halves_sum(ps);
    pd = halves_sum(pd);
    if (on) ld.y = pd / ps;
    tile_landed();
    first_requests();
  }
  if (split == 0 && on && lane_again() < 32) {
    // (infinite L, of rows without keys: large, as zeros times infinity are no zeros)
    const float l = ld.x / a.c2;
    a.rows[RowAt(a, kvh, row_again(row0)).of_all(a, b)] = row_stat(l > 1e38f ? 1e38f : l, ld.y);
  }
  v16f acc[NB];
#pragma unroll
  for (int j = 0; j < NB; ++j) acc[j] = zero16();
  auto step = [&](auto buffer, int key) {
    constexpr int B = decltype(buffer)::value, S = C::STAGES;
    tile_landed<(S - 2) * 2 * decltype(loads)::LD>();
    if (S > 2 || key + BK < end) request(key + (S - 1) * BK, (B + S - 1) % S);
    const uint8_t* kt = lds + B * 2 * TILE;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      v8h cf[CA];
      v16f s, dp;
      __builtin_amdgcn_sched_barrier(0);
      products(kt, kb, s, dp);
#pragma unroll
      for (int j = 0; j < CA; ++j) cf[j] = at.columns(kt, 2 * kb, j);
      next_lds_reads<AHEAD>();
#pragma unroll
      for (int t = 0; t < 4 * NB; ++t) {
        next_mfma<1>();
        next_lds_reads<1>();
      }
      if constexpr (2 * CA > AHEAD) next_lds_reads<2 * CA - AHEAD>();
      __builtin_amdgcn_sched_barrier(0);
      mask(s, key + 32 * kb);
#pragma unroll
      for (int r = 0; r < 16; ++r) dp[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], a.c2, -ld.x)) * (dp[r] - ld.y);
      const v8h ds[2] = {round8(dp, 0), round8(dp, 1)};
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < 2 * NB; ++i) {
        acc[i % NB] = mfma32(cf[i % CA], ds[i / NB], acc[i % NB]);
        if (i + CA < 2 * NB) cf[i % CA] = at.columns(kt, 2 * kb + (i + CA) / NB, (i + CA) % NB);
      }
#pragma unroll
      for (int t = 0; t < 2 * NB - CA; ++t) {
        next_mfma<1>();
        next_lds_reads<2>();
      }
      next_mfma<CA>();
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  for_stages<C::STAGES>(begin, end, BK, step);
  const float c = a.c2 * kLn2F * a.outer_factor(keys_again(n));
  if (n == 1) {
#pragma unroll
    for (int j = 0; j < NB; ++j) acc[j] = zero16();
  }
  if (a.splits > 1) {
    float* out = a.part + split * a.part_stride + RowAt(a, kvh, row_again(row0)).of_all(a, b) * a.dh;
#pragma unroll
    for (int j = 0; j < NB; ++j) store_block_f32(out, 32 * j, a.dh, on, lane_again() >> 5, acc[j], c);
    return;
  }
  store_rows<NB>(lds, acc, c * a.beta, row0, RowsOfHeads(a, b, kvh, nrows), a.dh, 0, lane_again(), wave);
}

// ---- backward: dK and dV ------------------------------------------------------------------------------------------------------
// A wave takes 32 keys, whose fragments and gradients stay in registers, and all queries of the heads that share them, tile by tile through LDS.
// Heads above 128 columns are accumulated in two halves by two workgroups, whose products with all columns are made twice: 512 registers hold no more.
// Up to 96 columns two waves a SIMD (us, 16 x 16 heads of 96, 512 queries over up to 1024 keys: one wave with four fragments read ahead 128, two with two 82; of the rows across
// heads only one fragment more fits the registers).
template <int NB>
struct DkvCfg {
  static constexpr int HALVES = NB > 4 ? 2 : 1, ACC = NB / HALVES;
  static constexpr int BQ = NB <= 4 ? 64 : 32, TILE = BQ * RowTile<NB>::P, STATS = 1024, STAGE = 2 * TILE + STATS, LDS = 3 * STAGE;
};
// Scores and dO v of 32 queries and a wave's keys.
struct DkvBlock {
  v16f s, dp;
};
template <int NB, bool ACROSS>
__global__ void __launch_bounds__(kThreads, NB <= 3 ? 2 : 1) cross_dkv_kernel(AttendArgs a) {
  using C = DkvCfg<NB>;
  // Column fragments are read further ahead where registers are left (us: 2 x 32 by 8 heads of 128, 4096 over 8192, 2690 -> 2480; 64 heads of 192 and of 256, 1024 x 1024,
  // 219 -> 202 and 277 -> 250; 16 x 16 heads of 32 41 -> 39.4; eight row fragments instead of four 2600 at the first)
  constexpr bool FAR = NB != 3;
  constexpr int BQ = C::BQ, QB = BQ / 32, TILE = C::TILE, ACC = C::ACC, AHEAD = NB == 3 ? (ACROSS ? 1 : 2) : kAhead<NB>;
  extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
  const int lane = threadIdx.x & 63, l32 = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Items::Item it = a.items.at(blockIdx.x);
  if (it.b < 0) return;
  const int b = it.b, kvh = it.kvh, tile = it.y, split = it.z, first = it.x * ACC;
  const int n = a.keys_of(b);
  const int row0 = tile * kRows + wave * 32;      // of the wave's keys
  // the tiles of the sharing heads' queries, one head after the other, each with tiles of its own or all in the same ones (across); a split takes per_split of them
  const int nrows = a.rep * a.sq, qtiles = ACROSS ? (nrows + BQ - 1) / BQ : (a.sq + BQ - 1) / BQ, total = ACROSS ? qtiles : a.rep * qtiles;
  const int begin = split * a.per_split;
  int end = begin + a.per_split < total ? begin + a.per_split : total;
  if (tile * kRows >= n) end = begin;
  const long at_head = b * a.k.batch + kvh * a.k.head;
  const RowsOf dk_rows{(uint8_t*)(a.dk + at_head), a.k.row, a.sk}, dv_rows{(uint8_t*)(a.dv + at_head), a.k.row, a.sk};
  if (begin >= end && a.splits == 1) {      // zeros, without the detour through LDS (the same: 73 -> 70 us)
#pragma unroll
    for (int i = 0; i < 2 * ACC; ++i) {
      const int c = i * 64 + lane, row = c / (4 * ACC), col = 32 * first + 8 * (c - row * (4 * ACC)), r = row0 + row;
      if (r < a.sk && col < a.dh) {
        wt_store(reinterpret_cast<v4i*>(dk_rows(r) + col), v4i{});
        wt_store(reinterpret_cast<v4i*>(dv_rows(r) + col), v4i{});
      }
    }
    return;
  }

  TileLoads<NB, BQ, kThreads> lq, lg;
  lq.init(a.q.row, a.dh);
  lg.init(a.g.row, a.dh);
  int rhead = begin / (qtiles > 0 ? qtiles : 1), rtile = begin - rhead * qtiles;      // of the next request
  auto request = [&](int buffer) {
    const int head = kvh * a.rep + rhead, q0 = rtile * BQ;
    uint8_t* to = lds + buffer * C::STAGE;
    const _Float16 *Q = a.q.p + b * a.q.batch + head * a.q.head, *G = a.g.p + b * a.g.batch + head * a.g.head;
    if constexpr (ACROSS) {
      auto across = [&](const _Float16* p, const Side& x, uint8_t* lds_tile) {
        TileLoads<NB, BQ, kThreads>::request_across(p, q0, nrows, a.by_sq, a.sq, (int)(2 * x.head), x.row, (int)((a.rep - 1) * 2 * x.head) + (a.sq - 1) * x.row + 2 * a.dh, a.dh,
                                                    lds_tile, wave);
      };
      across(Q, a.q, to);
      across(G, a.g, to + TILE);
    } else {
      lq.request((const uint8_t*)Q + (long)q0 * a.q.row, a.sq - q0, a.q.row, a.dh, to, wave);
      lg.request((const uint8_t*)G + (long)q0 * a.g.row, a.sq - q0, a.g.row, a.dh, to + TILE, wave);
    }
    const int left = (ACROSS ? nrows : a.sq) - q0;      // (zeros behind them, as Q and dO are there: P is then 1, and all that it meets 0)
    if (wave == 0) load_to_lds(buffer_words(a.rows + ((long)b * a.heads + head) * a.sq + q0, (left < BQ ? left : BQ) * 16), to + 2 * TILE, threadIdx.x * 16);
    if (++rtile == qtiles) { rtile = 0; ++rhead; }
  };
  if (begin < end) request(0);
  v8h kf[2 * NB], vf[2 * NB];
  {
    const int key = row0 + l32;
    load_fragments<NB>(kf, (const _Float16*)((const uint8_t*)(a.k.p + b * a.k.batch + kvh * a.k.head) + (long)key * a.k.row), key < n, a.dh, half);
    load_fragments<NB>(vf, (const _Float16*)((const uint8_t*)(a.v.p + b * a.v.batch + kvh * a.v.head) + (long)key * a.v.row), key < n, a.dh, half);
  }
  TileReads<NB, ACC> at;
  at.init(lane, first);
  v16f dk[ACC], dv[ACC];
#pragma unroll
  for (int j = 0; j < ACC; ++j) dk[j] = dv[j] = zero16();

  const v4i ones_s = row_ones(false, half), ones_dp = row_ones(true, half);
  auto products = [&](const uint8_t* qt, int qb, DkvBlock& x) {
    // (scores and dO v in turn: a product that adds to the one just before it has to wait for it)
    auto fragment = [&](int i) { return at.rows(i % 2 ? qt + TILE : qt, qb, i / 2); };
    const v4i stat = *US_LDS_AT(const v4i, qt + 2 * TILE + (qb * 32 + l32) * 16);
    v8h rf[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) rf[i] = fragment(i);
    x.s = x.dp = zero16();
#pragma unroll
    for (int i = 0; i < 4 * NB; ++i) {
      if (i % 2) x.dp = mfma32(rf[i % AHEAD], vf[i / 2], x.dp);
      else x.s = mfma32(rf[i % AHEAD], kf[i / 2], x.s);
      if (i + AHEAD < 4 * NB) rf[i % AHEAD] = fragment(i + AHEAD);
    }
    x.s = mfma32_bf16(stat, ones_s, x.s);
    x.dp = mfma32_bf16(stat, ones_dp, x.dp);
  };
  // Block qb of the tile at qt becomes part of the gradients; meanwhile block nqb of the tile at nt is made, so that matrix core and vector ALU both have work.
  auto block = [&](DkvBlock& cur, const uint8_t* qt, int qb, DkvBlock& next, const uint8_t* nt, int nqb) {
    const uint8_t* gt = qt + TILE;
    v8h p[2], ds[2], gc[FAR ? 2 : 1][ACC], qc[FAR ? 2 : 1][ACC];
    __builtin_amdgcn_sched_barrier(0);
    products(nt, nqb, next);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      cur.s[r] = __builtin_amdgcn_exp2f(cur.s[r] * a.c2);
      cur.dp[r] *= cur.s[r];
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      p[t] = round8(cur.s, t);
      ds[t] = round8(cur.dp, t);
    }
#pragma unroll
    for (int j = 0; j < ACC; ++j) gc[0][j] = at.columns(gt, 2 * qb, j);
    if constexpr (FAR) {
#pragma unroll
      for (int j = 0; j < ACC; ++j) qc[0][j] = at.columns(qt, 2 * qb, j);
    }
    next_lds_reads<1 + AHEAD>();
#pragma unroll
    for (int i = 0; i < 4 * NB; ++i) {
      next_mfma<1>();
      next_lds_reads<FAR ? 2 : 1>();
      next_exp<(16 + 4 * NB - 1) / (4 * NB)>();
      next_valu<(48 + 4 * NB - 1) / (4 * NB)>();
    }
    next_mfma<2>();
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int here = FAR ? t : 0;
#pragma unroll
      for (int j = 0; j < ACC; ++j) {
        dv[j] = mfma32(gc[here][j], p[t], dv[j]);
        if (!FAR) qc[0][j] = at.columns(qt, 2 * qb + t, j);
        else if (t == 0) gc[FAR][j] = at.columns(gt, 2 * qb + 1, j);
      }
#pragma unroll
      for (int j = 0; j < ACC; ++j) {
        dk[j] = mfma32(qc[here][j], ds[t], dk[j]);
        if (t == 0) {
          if (FAR) qc[FAR][j] = at.columns(qt, 2 * qb + 1, j);
          else gc[0][j] = at.columns(gt, 2 * qb + 1, j);
        }
      }
    }
#pragma unroll
    for (int t = 0; t < (FAR ? 2 : 3) * ACC; ++t) {
      next_mfma<1>();
      next_lds_reads<2>();
    }
    next_mfma<(FAR ? 2 : 1) * ACC>();
    __builtin_amdgcn_sched_barrier(0);
  };
  // A tile's last block is needed while the next tile's first one is made, and the tile behind that is on its way: three buffers.  Behind the last tile a block is
  // made of what the next buffer happens to hold, and not used: a branch around it would have the accumulators moved about at its end.
  DkvBlock x, y;
  if (begin < end) {
    tile_landed();
    if (begin + 1 < end) request(1);
    products(lds, 0, x);
    for (int i = begin, buffer = 0; i < end; ++i) {
      const int after = buffer == 2 ? 0 : buffer + 1;
      const uint8_t *qt = lds + buffer * C::STAGE, *nt = lds + after * C::STAGE;
      if constexpr (QB > 1) block(x, qt, 0, y, qt, 1);
      tile_landed();                            // the next tile has landed for everyone, the one before this is used up
      if (i + 2 < end) request(after == 2 ? 0 : after + 1);
      if constexpr (QB > 1) {
        block(y, qt, 1, x, nt, 0);
      } else {
        block(x, qt, 0, y, nt, 0);
        x = y;
      }
      buffer = after;
    }
  }
  const float f = a.outer_factor(keys_again(n)), c = a.c2 * kLn2F * f;
  const int key = NB == 3 ? row_again(row0) : row0 + l32;      // (three blocks have not one register to spare)
#pragma unroll
  for (int j = 0; j < ACC; ++j) {
    if (key >= n) dk[j] = dv[j] = zero16();
    if (n == 1) dk[j] = zero16();       // the softmax of one key has no gradient
  }
  if (a.splits > 1) {
    float* out = a.part + split * a.part_stride + (((long)b * a.kv + kvh) * a.sk + key) * 2 * a.dh;
    const bool on = key < a.sk;
    const int half_again = lane_again() >> 5;
#pragma unroll
    for (int j = 0; j < ACC; ++j) {
      store_block_f32(out, 32 * (first + j), a.dh, on, half_again, dk[j], c);
      store_block_f32(out + a.dh, 32 * (first + j), a.dh, on, half_again, dv[j], f);
    }
    return;
  }
  store_rows<ACC>(lds, dk, c * a.beta, row0, dk_rows, a.dh, 32 * first, lane_again(), wave);
  store_rows<ACC>(lds, dv, a.beta * f, row0, dv_rows, a.dh, 32 * first, lane_again(), wave);
}

// Sums of split gradients, part after part: `rows` rows of dh columns `row_stride` elements apart in a part; row = (batch * heads + head) * s + t.
// blockIdx.y = 1: the second gradient, dh columns further on.
__global__ void __launch_bounds__(kThreads) cross_sum_kernel(const float* part, long part_stride, long row_stride, int splits, long rows, int heads, int s, int dh,
                                                             _Float16* first, _Float16* second, long out_batch, long out_head, long out_row, float beta) {
  const int per = dh / 4;
  const long i = (long)blockIdx.x * kThreads + threadIdx.x;
  const long row = i / per;
  if (row >= rows) return;
  const int col = (int)(i - row * per) * 4;
  const float* p = part + row * row_stride + col + blockIdx.y * dh;
  v4f sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
  for (int k = 0; k < splits; ++k) {
    const v4f x = *reinterpret_cast<const v4f*>(p + k * part_stride);
#pragma unroll
    for (int e = 0; e < 4; ++e) sum[e] += x[e];
  }
  const long bh = row / s, t = row - bh * s, b = bh / heads, head = bh - b * heads;
  const v4h o = {to_half(sum[0] * beta), to_half(sum[1] * beta), to_half(sum[2] * beta), to_half(sum[3] * beta)};
  wt_store(reinterpret_cast<v4h*>((blockIdx.y ? second : first) + b * out_batch + head * out_head + t * out_row + col), o);
}

// f(integral_constant<int, NB>): blocks of 32 columns that hold a head
template <class F>
auto with_blocks(long dh, F f) {
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
  a.by_sq = FastDiv::by((uint32_t)(c.sq > 0 ? c.sq : 1));
  a.sk = (int)c.sk;
  a.dh = (int)c.dh;
  a.c2 = (float)(1.0 / sqrt((double)c.dh) * 1.44269504088896340736);
  a.alpha = c.alpha;
  return a;
}

long ceil_div(long a, long b) { return (a + b - 1) / b; }

// How a reduction of `steps` tiles is cut into parts of at least `least`: the fewest steps one after the other, where a CU holds `per_cu` of the workgroups at once, each
// starts and ends in the time of `fixed` steps, and parts are added in that of four; none where that saves less than an eighth.  Only the most parts that fit one to four
// rounds are looked at.  (us, against parts for two workgroups per CU whatever runs at once: 12 heads of 128, 829 x 912, both directions 102 -> 88; 12 by 6, 370 x 2505 120 -> 97;
// 56 by 14 heads of 96, 75 x 519 58 -> 55.  The forward pass with parts for 2, 3, 4 and 6 workgroups per CU, where two run: 16 heads of 128, 512 x 4096 32, 38, 62, 65; 42 over
// ragged 9000 keys 52, 62, 72, 70; of 64 columns, where four run, 64 over ragged 8192 keys 58, 57, 60, 63.)
struct Cut {
  int splits;
  long per;       // steps of a part
};
Cut cut(long items, long steps, long least, long per_cu, long fixed) {
  if (items < 1 || steps < 1) return {1, steps > 0 ? steps : 1};
  const long slots = per_cu * device_info().cus;
  Cut best{1, steps};
  long least_cost = ceil_div(items, slots) * (steps + fixed) * 7 / 8;
  for (long rounds = 1; rounds <= 4; ++rounds) {
    long splits = rounds * slots / items;
    if (splits > steps / least) splits = steps / least;
    if (splits < 2) continue;
    const long per = ceil_div(steps, splits), parts = ceil_div(steps, per), cost = ceil_div(items * parts, slots) * (per + fixed) + 4;
    if (cost < least_cost) {
      least_cost = cost;
      best = {(int)parts, per};
    }
  }
  return best;
}
long row_tiles(const CrossCall& c) { return ceil_div(c.heads / c.kv_heads * c.sq, kRows); }
// (two waves on a SIMD are as fast as three or four)
Cut fwd_cut(const CrossCall& c) { return cut(c.batch * c.kv_heads * row_tiles(c), ceil_div(c.sk, 64), 4, c.dh <= 128 ? 2 : 1, 3); }
Cut dq_cut(const CrossCall& c) { return fwd_cut(c); }
// How dK's and dV's workgroups take the queries: tiles of each head, or of all heads that share a key head, where that makes fewer tiles and 31 bits hold the
// heads' distances (us: batch 4, 24 heads by 8 key heads of 80, 2 queries over 12283 keys 72 -> 28; 8 by 4 of 96, 644 queries, 22 tiles or 21: 59 or 62).
struct QueryTiles {
  bool across;
  long tiles;      // of a key head
};
QueryTiles query_tiles(const CrossCall& c, int bq, bool near) {
  const long rep = c.heads / c.kv_heads, own = rep * ceil_div(c.sq, bq), all = ceil_div(rep * c.sq, bq);
  return 8 * all <= 7 * own && near ? QueryTiles{true, all} : QueryTiles{false, own};
}
bool heads_near(const CrossCall& c) {
  const long most = c.lq.head > c.lo.head ? c.lq.head : c.lo.head, row = c.lq.row > c.lo.row ? c.lq.row : c.lo.row;
  return most < (1l << 30) && 2 * ((c.heads / c.kv_heads - 1) * most + c.sq * row) < (1l << 30);
}
// (As many parts whatever the layouts, which the workspace's size is not asked with.)
Cut dkv_cut(const CrossCall& c) {
  return with_blocks(c.dh, [&](auto nb) {
    using C = DkvCfg<decltype(nb)::value>;
    Cut s = cut(C::HALVES * c.batch * c.kv_heads * ceil_div(c.sk, kRows), query_tiles(c, C::BQ, true).tiles, 256 / C::BQ, c.dh <= 96 ? 2 : 1, 384 / C::BQ);
    const long tiles = query_tiles(c, C::BQ, heads_near(c)).tiles;
    if (tiles > 0) s.per = ceil_div(tiles, s.splits), s.splits = (int)ceil_div(tiles, s.per);
    return s;
  });
}

size_t up256(size_t n) { return (n + 255) / 256 * 256; }
// What dQ's kernel leaves of every query row for dK and dV, one row after the other; the parts behind it start on whole 4 KB.
size_t rows_bytes(const CrossCall& c) { return ((size_t)c.batch * c.heads * c.sq * 16 + 4095) / 4096 * 4096; }

template <class K>
hipError_t launch(K kernel, FuncConfig& config, int lds, const AttendArgs& a, hipStream_t st) {
  if (const hipError_t e = config.ensure((const void*)kernel, lds); e != hipSuccess) return e;
  kernel<<<a.items.blocks, kThreads, lds, st>>>(a);
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
  CrossCall near = c;
  near.lq = near.lo = us_heads_layout{};
  const Cut q = dq_cut(c), k = dkv_cut(near);
  const size_t nq = q.splits == 1 ? 0 : (size_t)q.splits * c.batch * c.heads * c.sq * c.dh * 4;
  const size_t nk = k.splits == 1 ? 0 : (size_t)k.splits * c.batch * c.kv_heads * c.sk * c.dh * 8;
  return rows_bytes(c) + (nq > nk ? nq : nk);
}

hipError_t launch_join(const AttendArgs& a, hipStream_t st) {
  const long rows = (long)a.batch * a.heads * a.sq;
  int log_lanes = 1;
  while ((4 << log_lanes) < a.dh) ++log_lanes;
  join_kernel<<<(unsigned)ceil_div(rows, kWaves), kThreads, 0, st>>>(a, rows, log_lanes);
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
    a.items = Items::of(c.batch * c.kv_heads, c.kv_heads, row_tiles(c), a.splits, 1, device_info().xcds);
    return launch(cross_fwd_kernel<NB>, config, FwdCfg<NB>::LDS, a, st);
  });
  if (e != hipSuccess || a.splits == 1) return e;
  return launch_join(a, st);
}

hipError_t launch_cross_bwd(const CrossCall& c, void* dQ, void* dK, void* dV, float beta_q, float beta_kv, void* workspace, hipStream_t st) {
  const int xcds = device_info().xcds;
  AttendArgs a = cross_args(c);
  a.rows = (v4i*)workspace;
  a.part = (float*)((uint8_t*)workspace + rows_bytes(c));
  a.lse = c.lse;
  const QueryTiles qt = with_blocks(c.dh, [&](auto nb) { return query_tiles(c, DkvCfg<decltype(nb)::value>::BQ, heads_near(c)); });
  if (c.sq > 0) {
    AttendArgs q = a;
    q.out = (_Float16*)dQ;
    q.out_batch = c.lq.batch;
    q.out_head = c.lq.head;
    q.out_row = c.lq.row;
    q.beta = beta_q;
    const Cut s = dq_cut(c);
    q.splits = s.splits;
    q.per_split = (int)(s.per * 64);
    q.part_stride = c.batch * c.heads * c.sq * c.dh;
    q.items = Items::of(c.batch * c.kv_heads, c.kv_heads, row_tiles(c), q.splits, 1, xcds);
    hipError_t e = with_blocks(c.dh, [&](auto nb) {
      constexpr int NB = decltype(nb)::value;
      static FuncConfig config;
      return launch(cross_dq_kernel<NB>, config, DqCfg<NB>::LDS, q, st);
    });
    if (e != hipSuccess) return e;
    if (q.splits > 1) {
      const long rows = c.batch * c.heads * c.sq;
      cross_sum_kernel<<<(unsigned)ceil_div(rows * (c.dh / 4), kThreads), kThreads, 0, st>>>(q.part, q.part_stride, c.dh, q.splits, rows, (int)c.heads, (int)c.sq, (int)c.dh, q.out, nullptr,
                                                                                            q.out_batch, q.out_head, q.out_row, beta_q);
      if (e = hipGetLastError(); e != hipSuccess) return e;
    }
  }
  if (c.sk == 0) return hipSuccess;
  a.dk = (_Float16*)dK;
  a.dv = (_Float16*)dV;
  a.beta = beta_kv;
  const Cut s = dkv_cut(c);
  a.splits = s.splits;
  a.per_split = (int)s.per;
  a.part_stride = c.batch * c.kv_heads * c.sk * c.dh * 2;
  hipError_t e = with_blocks(c.dh, [&](auto nb) {
    constexpr int NB = decltype(nb)::value;
    using C = DkvCfg<NB>;
    static FuncConfig config;
    a.items = Items::of(c.batch * c.kv_heads, c.kv_heads, C::HALVES, ceil_div(c.sk, kRows), a.splits, xcds);
    static FuncConfig across;
    return qt.across ? launch(cross_dkv_kernel<NB, true>, across, C::LDS, a, st) : launch(cross_dkv_kernel<NB, false>, config, C::LDS, a, st);
  });
  if (e != hipSuccess || a.splits == 1) return e;
  const long rows = c.batch * c.kv_heads * c.sk;
  cross_sum_kernel<<<dim3((unsigned)ceil_div(rows * (c.dh / 4), kThreads), 2), kThreads, 0, st>>>(a.part, a.part_stride, 2 * c.dh, a.splits, rows, (int)c.kv_heads, (int)c.sk,
                                                                                                 (int)c.dh, a.dk, a.dv, c.lkv.batch, c.lkv.head, c.lkv.row, beta_kv);
  return hipGetLastError();
}

}  // namespace us
