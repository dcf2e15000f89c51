// A paged key-value cache: new rows into it, and eviction of the positions that attention hardly looked at.
// Position i of sequence b lies in slot i % page of page table[b][i / page]; pools are [pages][kv_heads][page][dh], the weights [pages][kv_heads][page].
// Both are bound by HBM: rows are read and written once.
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

// A thread takes 16 bytes of a stored row.
template <bool FP8>
__global__ void __launch_bounds__(kThreads) cache_store_kernel(Pool p, New x, const int* len, const int* count, long s, int chunks, long total) {
  constexpr int PER = FP8 ? 16 : 8;
  for (long i = (long)blockIdx.x * kThreads + threadIdx.x; i < total; i += (long)gridDim.x * kThreads) {
    const int chunk = (int)(i % chunks);
    long r = i / chunks;
    const int head = (int)(r % p.kv);
    r /= p.kv;
    const long t = r % s;
    r /= s;
    const int b = (int)(r >> 1), which = (int)(r & 1);
    const long c = count ? count[b] : s;
    if (t >= c) continue;
    const long pos = (long)len[b] - (c < s ? c : s) + t;
    if (pos < 0 || pos > 0x7fffffffl) continue;
    const long row = p.row_of(p.table, p.table_ld, b, head, (int)pos);
    if (row < 0) continue;
    const _Float16* from = (which ? x.v : x.k) + b * x.batch + head * x.head + t * x.row + chunk * PER;
    uint8_t* to = (which ? p.v : p.k) + (row * p.dh + chunk * PER) * (FP8 ? 1 : 2);
    const v8h a = *reinterpret_cast<const v8h*>(from);
    if constexpr (FP8) {
      const v8h c8 = *reinterpret_cast<const v8h*>(from + 8);
      const v2i lo = cvt8_fp8_from_half<US_E4M3>(a), hi = cvt8_fp8_from_half<US_E4M3>(c8);
      wt_store(reinterpret_cast<v4i*>(to), v4i{lo[0], lo[1], hi[0], hi[1]});
    } else {
      wt_store(reinterpret_cast<v8h*>(to), a);
    }
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

// A workgroup per sequence and key head: the k-th largest weight by four rounds of 256 bins, then the positions above it, and of those equal to it the
// first ones, in their order.
__global__ void __launch_bounds__(kSelect) cache_select_kernel(Pool p, const float* weights, const int* len, int* kept, int max_len, int keep, int recent) {
  __shared__ uint32_t bins[256];
  __shared__ uint32_t found[3];      // the order's bits so far, how many are still wanted
  __shared__ uint32_t above[kSelectWaves], equal[kSelectWaves];
  const int b = (int)(blockIdx.x / p.kv), head = (int)(blockIdx.x % p.kv), tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6;
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
  auto order_at = [&](int pos) -> uint32_t {
    const long row = p.row_of(p.table, p.table_ld, b, head, pos);
    return row < 0 ? 0u : order_of(weights[row]);
  };
  uint32_t prefix = 0, left = (uint32_t)want;
  for (int shift = 24; shift >= 0; shift -= 8) {
    if (tid < 256) bins[tid] = 0;
    __syncthreads();
    for (int i = tid; i < rest; i += kSelect) {
      const uint32_t o = order_at(i);
      if (shift == 24 || (o >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&bins[(o >> shift) & 255], 1u);
    }
    __syncthreads();
    if (tid == 0) {
      uint32_t seen = 0;
      int d = 255;
      for (; d > 0 && seen + bins[d] < left; --d) seen += bins[d];
      found[0] = prefix | ((uint32_t)d << shift);
      found[1] = left - seen;
    }
    __syncthreads();
    prefix = found[0];
    left = found[1];
  }
  // `left` of the positions whose order is `prefix`, and all above it
  int base = 0, same = 0;
  for (int i0 = 0; i0 < rest; i0 += kSelect) {
    const int i = i0 + tid;
    const uint32_t o = i < rest ? order_at(i) : 0u;
    const bool gt = i < rest && o > prefix, eq = i < rest && o == prefix;
    const uint64_t mgt = __builtin_amdgcn_ballot_w64(gt), meq = __builtin_amdgcn_ballot_w64(eq);
    if (lane == 0) {
      above[wave] = (uint32_t)__builtin_popcountll(mgt);
      equal[wave] = (uint32_t)__builtin_popcountll(meq);
    }
    __syncthreads();
    int g = 0, e = 0, gall = 0, eall = 0;
    for (int w = 0; w < kSelectWaves; ++w) {
      if (w < wave) { g += above[w]; e += equal[w]; }
      gall += above[w];
      eall += equal[w];
    }
    const uint64_t before = ((uint64_t)1 << lane) - 1;
    g += __builtin_popcountll(mgt & before);
    e += same + __builtin_popcountll(meq & before);
    const int taken = e < (int)left ? e : (int)left;      // equal ones in front that are kept
    if (gt || (eq && e < (int)left)) out[base + g + taken] = i;
    base += gall;
    same += eall;
    __syncthreads();
  }
}

// ---- eviction: the rows ------------------------------------------------------------------------------------------------------
// Kept row i goes to position i.  In place a destination never lies behind its source, and sources are in order: a workgroup that takes the rows of a key
// head in rounds, reading a whole round before it writes it, overwrites nothing that is still to be read.  Each round's rows are spread over its threads.
__global__ void __launch_bounds__(kSelect) cache_move_kernel(Pool p, float* weights, const int* table_to, long table_to_ld, const int* len, const int* kept,
                                                             int max_len, int keep, int row_bytes, int parts, bool in_place) {
  const int which = (int)(blockIdx.x % 3), head = (int)(blockIdx.x / 3 % p.kv), b = (int)(blockIdx.x / 3 / p.kv), tid = (int)threadIdx.x;
  const int part = (int)blockIdx.y;
  int n = len[b];
  n = n < 0 ? 0 : n > max_len ? max_len : n;
  const int all = n < keep ? n : keep;
  if (in_place && n <= keep) return;
  const int* from = kept + ((long)b * p.kv + head) * keep;
  const int chunks = which < 2 ? row_bytes / 16 : 1, rows = kSelect / chunks;      // rows of a round
  const int r = tid / chunks, chunk = tid % chunks;
  const int first = (int)((long)all * part / parts), last = (int)((long)all * (part + 1) / parts);
  for (int i0 = first; i0 < last; i0 += rows) {
    const int i = i0 + r;
    long src = -1, dst = -1;
    v4i x = {0, 0, 0, 0};
    float w = 0.0f;
    if (r < rows && i < last) {
      src = p.row_of(p.table, p.table_ld, b, head, from[i]);
      dst = p.row_of(table_to, table_to_ld, b, head, i);
      if (src >= 0) {
        if (which < 2) x = *reinterpret_cast<const v4i*>((which ? p.v : p.k) + src * row_bytes + chunk * 16);
        else w = weights[src];
      }
    }
    if (in_place) {
      asm volatile("" : "+v"(x), "+v"(w));      // (used here: the loads have landed, not only left, when the others go on)
      __syncthreads();
    }
    if (src >= 0 && dst >= 0 && src != dst) {
      if (which < 2) *reinterpret_cast<v4i*>((which ? p.v : p.k) + dst * row_bytes + chunk * 16) = x;
      else weights[dst] = w;
    }
    if (in_place) __syncthreads();
  }
}
__global__ void __launch_bounds__(kThreads) cache_len_kernel(const int* len, int* new_len, int batch, int max_len, int keep) {
  const int b = (int)blockIdx.x * kThreads + (int)threadIdx.x;
  if (b < batch) {
    int n = len[b];
    n = n < 0 ? 0 : n > max_len ? max_len : n;
    new_len[b] = n < keep ? n : keep;
  }
}

Pool pool_of(const CacheCall& c) {
  return Pool{(uint8_t*)c.k, (uint8_t*)c.v, c.table, c.table_ld, c.pages, c.shift, (int)c.batch, (int)c.kv_heads, (int)c.dh};
}

}  // namespace

hipError_t launch_cache_store(const CacheCall& c, const void* K, const void* V, const us_heads_layout& l, const int* len, const int* count, long s, hipStream_t st) {
  const int chunks = (int)(c.dh / (c.fp8 ? 16 : 8));
  const long total = 2 * c.batch * s * c.kv_heads * chunks, need = (total + kThreads - 1) / kThreads, most = 32l * device_info().cus;
  const New x{(const _Float16*)K, (const _Float16*)V, l.batch, l.head, l.row};
  const unsigned blocks = (unsigned)(need < most ? need : most);
  if (c.fp8) cache_store_kernel<true><<<blocks, kThreads, 0, st>>>(pool_of(c), x, len, count, s, chunks, total);
  else cache_store_kernel<false><<<blocks, kThreads, 0, st>>>(pool_of(c), x, len, count, s, chunks, total);
  return hipGetLastError();
}

hipError_t launch_cache_evict(const CacheCall& c, float* weights, const int* table_to, long table_to_ld, const int* len, int* new_len, int* kept, long max_len, long keep,
                              long recent, hipStream_t st) {
  const Pool p = pool_of(c);
  const bool in_place = table_to == c.table;
  const long groups = c.batch * c.kv_heads;
  if (keep > 0) {
    cache_select_kernel<<<(unsigned)groups, kSelect, 0, st>>>(p, weights, len, kept, (int)max_len, (int)keep, (int)recent);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    const int parts = in_place ? 1 : (int)(keep > 256 ? (keep + 255) / 256 : 1);
    cache_move_kernel<<<dim3((unsigned)(3 * groups), (unsigned)parts), kSelect, 0, st>>>(p, weights, table_to, table_to_ld, len, kept, (int)max_len, (int)keep,
                                                                                       (int)(c.dh * (c.fp8 ? 1 : 2)), parts, in_place);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  if (new_len) cache_len_kernel<<<(unsigned)((c.batch + kThreads - 1) / kThreads), kThreads, 0, st>>>(len, new_len, (int)c.batch, (int)max_len, (int)keep);
  return hipGetLastError();
}

}  // namespace us
