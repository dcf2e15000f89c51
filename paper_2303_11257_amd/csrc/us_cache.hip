// A paged key-value cache: new rows into it, and eviction of the positions that attention hardly looked at.
// Position i of sequence b lies in slot i % page of page table[b][i / page]; pools are [pages][kv_heads][page][dh], the weights [pages][kv_heads][page].
// Both are bound by HBM: rows are read and written once (16 sequences of up to 4096 new tokens, 8 heads of 128, to E4M3: 43.6 us, 4.9 TB/s).
#include <type_traits>

#include "us_device.h"
#include "us_launch.h"

namespace us {

namespace {

constexpr int kThreads = 256;

struct Pool {
  uint8_t *k, *v;
  const int* table;
  long table_ld, pages;
  int shift, batch, kv, dh;
  // row of a position's slot among the pools' rows, or -1: a page that there is not
  __device__ __forceinline__ long row_of(const int* tab, long ld, int b, int head, int pos) const {
    if (pos < 0 || (pos >> shift) >= ld) return -1;
    const int page = tab[(long)b * ld + (pos >> shift)];
    if (page < 0 || page >= pages) return -1;
    return ((((long)page * kv + head) << shift)) + (pos & ((1 << shift) - 1));
  }
};

struct New {
  const _Float16 *k, *v;
  long batch, head, row;
};

// A thread takes 16 bytes of a stored row; blockIdx.y = 2 b + (keys or values).
template <bool FP8>
__global__ void __launch_bounds__(kThreads) cache_store_kernel(Pool p, New x, const int* len, const int* count, int s, FastDiv by_token, FastDiv by_chunks, int chunks, uint32_t total) {
  constexpr int PER = FP8 ? 16 : 8;
  const uint32_t i = blockIdx.x * (uint32_t)kThreads + threadIdx.x;
  const int b = (int)(blockIdx.y >> 1), which = (int)(blockIdx.y & 1);
  const int c0 = count ? count[b] : s, c = c0 < s ? c0 : s;
  const int t = (int)by_token.of(i);
  if (i >= total || t >= c) return;
  const uint32_t j = i - (uint32_t)t * (uint32_t)(p.kv * chunks);
  const int head = (int)by_chunks.of(j), chunk = (int)(j - (uint32_t)head * (uint32_t)chunks);
  const long row = p.row_of(p.table, p.table_ld, b, head, (int)((long)len[b] - c + t > 0x7fffffffl ? -1 : (long)len[b] - c + t));
  if (row < 0) return;
  const _Float16* from = (which ? x.v : x.k) + b * x.batch + head * x.head + t * x.row + chunk * PER;
  uint8_t* to = (which ? p.v : p.k) + (row * p.dh + chunk * PER) * (FP8 ? 1 : 2);
  const v8h a = *reinterpret_cast<const v8h*>(from);
  if constexpr (FP8) {
    const v8h d = *reinterpret_cast<const v8h*>(from + 8);
    const v2i lo = cvt8_fp8_from_half<US_E4M3>(a), hi = cvt8_fp8_from_half<US_E4M3>(d);
    wt_store(reinterpret_cast<v4i*>(to), v4i{lo[0], lo[1], hi[0], hi[1]});
  } else {
    wt_store(reinterpret_cast<v8h*>(to), a);
  }
}

// ---- eviction: which positions ---------------------------------------------------------------------------------------------
// A number's place in the order of weights: NaN above everything, -0 as 0, a page that there is not below everything.
__device__ __forceinline__ uint32_t order_of(float w) {
  if (w != w) return 0xffffffffu;
  const uint32_t u = __builtin_bit_cast(uint32_t, w + 0.0f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

constexpr int kSelect = 1024, kSelectWaves = kSelect / 64;

// Bound by latency: four rounds, each a pass over LDS bins and two barriers (16 x 8 heads of up to 8192 positions 17.8 us for 4 MB).
// A workgroup per sequence and key head: the k-th largest weight by four rounds of 256 bins, then the positions above it, and of those equal to it the
// first ones, in their order.  A wave has a run of neighbouring positions, so that its part of the order needs one exchange of counts with the others;
// up to PER of them per lane stay in registers (PER = 0: longer sequences read the weights again each round, page by page: 4 x 8 heads of 131072 positions 378 us for 17 MB).
template <int PER>
__global__ void __launch_bounds__(kSelect) cache_select_kernel(Pool p, const float* weights, const int* len, int* kept, int max_len, int keep, int recent) {
  __shared__ uint32_t bins[2][256];
  __shared__ uint32_t found[2];      // the order's bits so far, how many are still wanted
  __shared__ uint32_t above[kSelectWaves], equal[kSelectWaves];
  const int b = (int)(blockIdx.x / p.kv), head = (int)(blockIdx.x % p.kv), tid = (int)threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int n = len[b];
  n = n < 0 ? 0 : n > max_len ? max_len : n;
  int* out = kept + (long)blockIdx.x * keep;
  if (n <= keep) {
    for (int i = tid; i < keep; i += kSelect) out[i] = i < n ? i : -1;
    return;
  }
  const int rest = n - recent, want = keep - recent;      // want of the first rest positions; want < rest
  for (int i = tid; i < recent; i += kSelect) out[want + i] = rest + i;
  if (want == 0) return;
  const int steps = (rest + kSelect - 1) / kSelect, first = wave * steps * 64 + lane;      // of this lane: first + 64 j, j < steps
  uint32_t mine[PER ? PER : 1];
  auto load = [&](int i) -> uint32_t {
    const long row = i < rest ? p.row_of(p.table, p.table_ld, b, head, i) : -1;
    return row < 0 ? 0u : order_of(weights[row]);
  };
  if constexpr (PER > 0) {
    long row[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) row[j] = j < steps && first + 64 * j < rest ? p.row_of(p.table, p.table_ld, b, head, first + 64 * j) : -1;
    float w[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) w[j] = row[j] >= 0 ? weights[row[j]] : 0.0f;
#pragma unroll
    for (int j = 0; j < PER; ++j) mine[j] = row[j] >= 0 ? order_of(w[j]) : 0u;
  }
  // f(order, position, whether it is one) of every position of the lane, in steps that the wave takes together
  auto each = [&](auto f) {
    if constexpr (PER > 0) {
#pragma unroll
      for (int j = 0; j < PER; ++j)
        if (j < steps) f(mine[j], first + 64 * j, first + 64 * j < rest);
    } else {
      for (int j = 0; j < steps; ++j) f(load(first + 64 * j), first + 64 * j, first + 64 * j < rest);
    }
  };
  if (tid < 256) bins[0][tid] = 0;
  __syncthreads();
  uint32_t prefix = 0, left = (uint32_t)want;
#pragma unroll
  for (int round = 0; round < 4; ++round) {
    const int shift = 24 - 8 * round;
    uint32_t* bin = bins[round & 1];
    each([&](uint32_t o, int, bool on) {
      on = on && (round == 0 || ((o ^ prefix) >> (shift + 8)) == 0);
      // weights crowd in a few bins: the lanes that agree with the first one are counted together, and the rest one by one
      const uint32_t d = (o >> shift) & 255;
      const uint64_t any = __builtin_amdgcn_ballot_w64(on);
      if (any == 0) return;
      const uint32_t d0 = __builtin_amdgcn_readlane(d, __builtin_ctzll(any));
      const uint64_t same = __builtin_amdgcn_ballot_w64(on && d == d0);
      if (lane == 0) atomicAdd(&bin[d0], (uint32_t)__builtin_popcountll(same));
      if (on && d != d0) atomicAdd(&bin[d], 1u);
    });
    __syncthreads();
    if (tid < 256) bins[(round & 1) ^ 1][tid] = 0;
    if (wave == 0) {
      // lane l: the bins 252 - 4 l .. 255 - 4 l, summed from the top
      uint32_t c[4], sum = 0;
#pragma unroll
      for (int q = 0; q < 4; ++q) sum += c[q] = bin[255 - 4 * lane - q];
      uint32_t upto = sum;
#pragma unroll
      for (int off = 1; off < 64; off <<= 1) {
        const uint32_t x = __shfl_up(upto, off, 64);
        if (lane >= off) upto += x;
      }
      uint32_t seen = upto - sum;
      if (seen < left && upto >= left) {      // one lane
        int q = 0;
#pragma unroll
        for (int k = 0; k < 3; ++k)
          if (q == k && seen + c[k] < left) { seen += c[k]; q = k + 1; }
        found[0] = prefix | ((uint32_t)(255 - 4 * lane - q) << shift);
        found[1] = left - seen;
      }
    }
    __syncthreads();
    prefix = found[0];
    left = found[1];
  }
  // `left` of the positions whose order is `prefix`, and all above it
  uint32_t gt = 0, eq = 0;
  each([&](uint32_t o, int, bool on) {
    gt += (uint32_t)__builtin_popcountll(__builtin_amdgcn_ballot_w64(on && o > prefix));
    eq += (uint32_t)__builtin_popcountll(__builtin_amdgcn_ballot_w64(on && o == prefix));
  });
  if (lane == 0) {
    above[wave] = gt;
    equal[wave] = eq;
  }
  __syncthreads();
  uint32_t g = 0, e = 0;
  for (int w = 0; w < wave; ++w) {
    g += above[w];
    e += equal[w];
  }
  const uint64_t before = ((uint64_t)1 << lane) - 1;
  each([&](uint32_t o, int i, bool on) {
    const uint64_t mg = __builtin_amdgcn_ballot_w64(on && o > prefix), me = __builtin_amdgcn_ballot_w64(on && o == prefix);
    const uint32_t ge = g + (uint32_t)__builtin_popcountll(mg & before), ee = e + (uint32_t)__builtin_popcountll(me & before);
    if (on && (o > prefix || (o == prefix && ee < left))) out[ge + (ee < left ? ee : left)] = i;
    g += (uint32_t)__builtin_popcountll(mg);
    e += (uint32_t)__builtin_popcountll(me);
  });
}

// ---- eviction: the rows ------------------------------------------------------------------------------------------------------
// Kept row i goes to position i.  In place a destination never lies behind its source, and sources are in order: a workgroup that takes the rows of a key
// head in rounds, reading a whole round before it writes it, overwrites nothing that is still to be read.  A round has kUnroll rows per thread group, their
// reads in flight together; in place the next round's are looked up meanwhile (us: 11 x 8 heads of 96, up to 6756 -> 2594 in FP16 72 -> 64, 64 x 8 of 128, 2000 kept
// 193 -> 176), and there are no more threads than pieces (29 x 23 heads, 19 kept: 12 -> 5.5).  Elsewhere a workgroup has one round (16 x 8 heads of 128 codes, 4096
// kept of up to 8192: 64; the loop around it leaves the order of its reads as it is: without it 73).
constexpr int kUnroll = 4;
template <bool IN_PLACE>
__global__ void __launch_bounds__(kSelect) cache_move_kernel(Pool p, float* weights, const int* table_to, long table_to_ld, const int* len, int* new_len, const int* kept,
                                                             int max_len, int keep, int row_bytes, int per_part) {
  const int which = (int)(blockIdx.x % 3), head = (int)(blockIdx.x / 3 % p.kv), b = (int)(blockIdx.x / 3 / p.kv), tid = (int)threadIdx.x;
  // (the lengths are written here, where no other workgroup reads them: new_len may be len)
  if (new_len && which == 2 && head == 0 && blockIdx.y == 0 && tid == 0) {
    int n = len[b];
    n = n < 0 ? 0 : n > max_len ? max_len : n;
    new_len[b] = n < keep ? n : keep;
  }
  const int* from = kept + ((long)b * p.kv + head) * keep;
  const int chunks = which < 2 ? row_bytes / 16 : 1, rows = (int)blockDim.x / chunks;
  const int r = tid / chunks, chunk = tid % chunks;
  const int first = (int)blockIdx.y * per_part, last = keep < first + per_part ? keep : first + per_part;
  uint8_t* const base = which ? p.v : p.k;
  constexpr int U = kUnroll;
  long src[U], dst[U];
  // where the rows of a round come from and go to, -1: nowhere.  A round's are looked up while the rows of the one before it are on their way.
  auto look = [&](int i0) {
    int pos[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * rows + r;
      pos[u] = r < rows && i < last ? from[i] : -1;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * rows + r;
      src[u] = pos[u] < 0 || (IN_PLACE && pos[u] == i) ? -1 : p.row_of(p.table, p.table_ld, b, head, pos[u]);
      dst[u] = src[u] < 0 ? -1 : p.row_of(table_to, table_to_ld, b, head, i);
    }
  };
  v4i x[U];
  float w[U];
  auto load = [&] {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      x[u] = v4i{0, 0, 0, 0};
      w[u] = 0.0f;
      if (dst[u] >= 0) {
        if (which < 2) x[u] = *reinterpret_cast<const v4i*>(base + src[u] * row_bytes + chunk * 16);
        else w[u] = weights[src[u]];
      }
    }
  };
  auto store = [&](const long (&to)[U]) {
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (to[u] >= 0) {
        if (which < 2) *reinterpret_cast<v4i*>(base + to[u] * row_bytes + chunk * 16) = x[u];
        else weights[to[u]] = w[u];
      }
  };
  if constexpr (IN_PLACE) look(first);
  for (int i0 = first; i0 < last; i0 += U * rows) {
    if constexpr (IN_PLACE) {
      load();
      long to[U];
#pragma unroll
      for (int u = 0; u < U; ++u) to[u] = dst[u];
      if (i0 + U * rows < last) look(i0 + U * rows);
#pragma unroll
      for (int u = 0; u < U; ++u) asm volatile("" : "+v"(x[u]), "+v"(w[u]));      // (used here: the loads have landed, not only left, when the others go on)
      __syncthreads();
      store(to);
      __syncthreads();
    } else {
      look(i0);
      load();
      store(dst);
    }
  }
}
__global__ void __launch_bounds__(kThreads) cache_len_kernel(int* new_len, int batch) {
  const int b = (int)blockIdx.x * kThreads + (int)threadIdx.x;
  if (b < batch) new_len[b] = 0;
}

Pool pool_of(const CacheCall& c) {
  return Pool{(uint8_t*)c.k, (uint8_t*)c.v, c.table, c.table_ld, c.pages, c.shift, (int)c.batch, (int)c.kv_heads, (int)c.dh};
}

}  // namespace

hipError_t launch_cache_store(const CacheCall& c, const void* K, const void* V, const us_heads_layout& l, const int* len, const int* count, long s, hipStream_t st) {
  const int chunks = (int)(c.dh / (c.fp8 ? 16 : 8));
  const uint32_t total = (uint32_t)(s * c.kv_heads * chunks);
  const New x{(const _Float16*)K, (const _Float16*)V, l.batch, l.head, l.row};
  const FastDiv by_token = FastDiv::by((uint32_t)(c.kv_heads * chunks)), by_chunks = FastDiv::by((uint32_t)chunks);
  // (blockIdx.y has 16 bits)
  for (long b0 = 0; b0 < c.batch; b0 += 32767) {
    CacheCall part = c;
    part.batch = c.batch - b0 < 32767 ? c.batch - b0 : 32767;
    part.table = c.table + b0 * c.table_ld;
    New y = x;
    y.k += b0 * x.batch;
    y.v += b0 * x.batch;
    const dim3 grid((total + kThreads - 1) / kThreads, (unsigned)(2 * part.batch));
    const int *len_b = len + b0, *count_b = count ? count + b0 : nullptr;
    if (c.fp8) cache_store_kernel<true><<<grid, kThreads, 0, st>>>(pool_of(part), y, len_b, count_b, (int)s, by_token, by_chunks, chunks, total);
    else cache_store_kernel<false><<<grid, kThreads, 0, st>>>(pool_of(part), y, len_b, count_b, (int)s, by_token, by_chunks, chunks, total);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_cache_evict(const CacheCall& c, float* weights, const int* table_to, long table_to_ld, const int* len, int* new_len, int* kept, long max_len, long keep,
                              long recent, hipStream_t st) {
  const Pool p = pool_of(c);
  const bool in_place = table_to == c.table;
  const unsigned groups = (unsigned)(c.batch * c.kv_heads);
  if (keep == 0) {
    if (new_len) cache_len_kernel<<<(unsigned)((c.batch + kThreads - 1) / kThreads), kThreads, 0, st>>>(new_len, (int)c.batch);
    return hipGetLastError();
  }
  auto select = [&](auto per) {
    cache_select_kernel<decltype(per)::value><<<groups, kSelect, 0, st>>>(p, weights, len, kept, (int)max_len, (int)keep, (int)recent);
    return hipGetLastError();
  };
  const long per = (max_len - recent + kSelect - 1) / kSelect;
  const hipError_t e = per <= 1 ? select(std::integral_constant<int, 1>{}) : per <= 4 ? select(std::integral_constant<int, 4>{})
                     : per <= 16 ? select(std::integral_constant<int, 16>{}) : select(std::integral_constant<int, 0>{});
  if (e != hipSuccess) return e;
  const int row_bytes = (int)(c.dh * (c.fp8 ? 1 : 2));
  if (in_place) {
    // no more threads than there are pieces for
    const long pieces = (keep * (row_bytes / 16) + kUnroll - 1) / kUnroll;
    const unsigned threads = pieces >= kSelect ? kSelect : (unsigned)((pieces + 63) / 64 * 64);
    cache_move_kernel<true><<<3 * groups, threads, 0, st>>>(p, weights, table_to, table_to_ld, len, new_len, kept, (int)max_len, (int)keep, row_bytes, (int)keep);
  } else {
    // a round of a workgroup's rows each
    const int per_part = kUnroll * (kThreads / (row_bytes / 16));
    cache_move_kernel<false><<<dim3(3 * groups, (unsigned)((keep + per_part - 1) / per_part)), kThreads, 0, st>>>(p, weights, table_to, table_to_ld, len, new_len, kept,
                                                                                                              (int)max_len, (int)keep, row_bytes, per_part);
  }
  return hipGetLastError();
}

}  // namespace us
