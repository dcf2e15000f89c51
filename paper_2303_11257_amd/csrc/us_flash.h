// Pieces shared by the kernels that attend over keys tile by tile with running softmax statistics (us_cross.hip, us_paged.hip).
#pragma once

#include "us_device.h"
#include "us_launch.h"
#include "us_rows.h"

namespace us {

constexpr float kLog2eF = 1.44269504088896340736f, kLn2F = 0.69314718055994530942f;
#define US_LDS_AT(T, p) ((__attribute__((address_space(3))) T*)(p))

// f of this lane's value and of that of the lane 32 away
template <class F>
__device__ __forceinline__ float halves(float v, F f) {
  const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false);
  const unsigned a = r[0], b = r[1];     // (a bit cast of r[1] itself reads element 0 with this compiler)
  return f(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b));
}
__device__ __forceinline__ float halves_max(float v) {
  return halves(v, [](float a, float b) { return __builtin_fmaxf(a, b); });
}
__device__ __forceinline__ float halves_sum(float v) {
  return halves(v, [](float a, float b) { return a + b; });
}

// ---- tiles of rows in LDS ---------------------------------------------------------------------------------------------
// A row of up to 32 NB halves takes P bytes; its 16-byte chunk c lies at c ^ swz(row).  The bits are chosen for both ways of reading: sixteen lanes that read the same
// chunk of rows r .. r + 15, and a transposing read whose 32 lanes touch 64 bytes in each of four rows; both meet every bank once.  Where P is no multiple of the
// banks' 256 bytes the rows themselves start on other banks: 192 moves each by three quarters, 384 by a half, as 64 and 128 do by one quarter and a half.
template <int NB>
struct RowTile {
  static constexpr int P = 64 * NB;
  static_assert(NB <= 4 || NB == 6 || NB == 8, "");
  __device__ __forceinline__ static int swz(int row) {
    if (P % 128) return (row >> 2) & 3;
    if (P % 256) return (((row >> 1) & 1) << 2) | ((row >> 2) & 3);
    return ((row & 3) << 2) | ((row >> 2) & 3);
  }
};

// Where a lane reads its parts of a tile, in bytes from the tile's start.
// (COLS: blocks of columns that it takes transposed, from block `first` on)
template <int NB, int COLS = NB>
struct TileReads {
  using T = RowTile<NB>;
  uint32_t row[2 * NB], col[2][COLS];
  __device__ __forceinline__ void init(int lane, int first = 0) {
    const int l32 = lane & 31, half = lane >> 5, l16 = lane & 15;
#pragma unroll
    for (int t = 0; t < 2 * NB; ++t) row[t] = (uint32_t)(l32 * T::P + (((2 * t + half) ^ T::swz(l32)) << 4));
    // (a bit of the swizzle changes from a row to the row 8 further on)
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int j = 0; j < COLS; ++j) {
        const int r = 4 * half + (l16 >> 2) + 8 * e, chunk = (first + j) * 4 + ((lane >> 4) & 1) * 2 + ((l16 & 3) >> 1);
        col[e][j] = (uint32_t)(r * T::P + ((chunk ^ T::swz(r)) << 4) + (l16 & 1) * 8);
      }
  }
  // rows as the first operand of the 32 x 32 x 16 instruction: lane l has row 32 rb + l % 32, columns 16 t + 8 (l / 32) ..
  __device__ __forceinline__ v8h rows(const uint8_t* tile, int rb, int t) const { return *US_LDS_AT(const v8h, tile + row[t] + rb * 32 * T::P); }
  // ... and transposed: lane l has column 32 j + l % 32 and the rows 16 t + 4 (l / 32) + (0 .. 3, 8 .. 11), which are the rows that the
  // results of a 32 x 32 instruction leave in a lane
  __device__ __forceinline__ v8h columns(const uint8_t* tile, int t, int j) const {
    const v4s a = __builtin_amdgcn_ds_read_tr16_b64_v4i16(US_LDS_AT(v4s, tile + col[0][j] + t * 16 * T::P));
    const v4s b = __builtin_amdgcn_ds_read_tr16_b64_v4i16(US_LDS_AT(v4s, tile + col[1][j] + t * 16 * T::P));
    struct { v4s a, b; } both = {a, b};
    return __builtin_bit_cast(v8h, both);
  }
};

// 16 bytes per lane straight to LDS, lane after lane from `lds` on; zeros where the offset lies beyond the resource (its four words: buffer_words).  In assembly,
// because the compiler makes transposing reads of LDS wait for every such load that it knows of, the next tile's too: the kernels wait for what they need themselves
// (tile_landed, wait_newest).  The compiler's own waits count fewer loads than there are, and so wait longer, never shorter.  (s_nop: five wait states between a
// vector instruction that writes a scalar register and this load's reading it, one between m0 and the load.  m0 is an operand, so that the compiler knows what it holds.)
__device__ __forceinline__ void load_to_lds(v4i from, uint8_t* lds, uint32_t off) {
  asm volatile("s_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"{m0}"((uint32_t)(uintptr_t)US_LDS_AT(uint8_t, lds)), "v"(off), "s"(from) : "memory");
}
// All loads of the workgroup to LDS but each wave's newest N have landed, all its reads of LDS are done; nothing that reads or writes memory moves across.
template <int N = 0>
__device__ __forceinline__ void tile_landed() {
  static_assert(N >= 0 && N < 64, "");
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// The loads of a tile of ROWS rows by THREADS threads, straight to LDS; rows from `rows` on and columns from dh on are zeros.
template <int NB, int ROWS, int THREADS>
struct TileLoads {
  using T = RowTile<NB>;
  static constexpr int BYTES = ROWS * T::P, LD = (BYTES / 16 + THREADS - 1) / THREADS;
  uint32_t off[LD];
  __device__ __forceinline__ void init(int row_bytes, int dh) {
#pragma unroll
    for (int j = 0; j < LD; ++j) {
      const int o = (j * THREADS + (int)threadIdx.x) * 16, row = o / T::P, chunk = ((o % T::P) >> 4) ^ T::swz(row);
      off[j] = chunk * 8 < dh ? (uint32_t)(row * row_bytes + chunk * 16) : 0x7ffffff0u;
    }
  }
  // the tile's rows are rows r0 .. of several heads one after the other (by_s divides by a head's s rows), `head_bytes` apart, `rows` in all; the whole lies
  // within 31 bits of `base`
  __device__ __forceinline__ static void request_across(const void* base, int r0, int rows, FastDiv by_s, int s, int head_bytes, int row_bytes, int bytes, int dh,
                                                        uint8_t* lds, int wave) {
    const v4i res = buffer_words(base, (uint32_t)bytes);
#pragma unroll
    for (int j = 0; j < LD; ++j)
      if (BYTES / 16 % THREADS == 0 || j * THREADS + wave * 64 < BYTES / 16) {
        const int o = (j * THREADS + (int)threadIdx.x) * 16, row = o / T::P, chunk = ((o % T::P) >> 4) ^ T::swz(row), r = r0 + row;
        const int h = (int)by_s.of((uint32_t)r);
        const uint32_t at = (uint32_t)(h * head_bytes + (r - h * s) * row_bytes + chunk * 16);
        load_to_lds(res, lds + (j * THREADS + wave * 64) * 16, r < rows && chunk * 8 < dh ? at : 0x7ffffff0u);
      }
  }
  __device__ __forceinline__ void request(const void* base, long rows, int row_bytes, int dh, uint8_t* lds, int wave) const {
    const int r = rows > ROWS ? ROWS : rows < 0 ? 0 : (int)rows;
    const v4i res = buffer_words(base, r > 0 ? (uint32_t)((r - 1) * row_bytes + dh * 2) : 0u);
#pragma unroll
    for (int j = 0; j < LD; ++j)
      if (BYTES / 16 % THREADS == 0 || j * THREADS + wave * 64 < BYTES / 16)
        load_to_lds(res, lds + (j * THREADS + wave * 64) * 16, off[j]);
  }
};

__device__ __forceinline__ v16f zero16() {
  v16f z;
#pragma unroll
  for (int r = 0; r < 16; ++r) z[r] = 0.0f;
  return z;
}
__device__ __forceinline__ v16f mfma32(v8h a, v8h b, v16f c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }

// What dK and dV need of a query row, L / c2 and D (below, us_cross.hip), as an operand of one more product: -x as the sum of three BF16 values, exactly, each
// of 8 bits.  In slots 0 .. 2 and 3 .. 5 of the sixteen that the product adds up, against ones there and zeros elsewhere (row_ones).
__device__ __forceinline__ v4i row_stat(float x, float y) {
  auto part = [](float& v) {      // takes its highest 8 bits off
    const uint32_t top = __builtin_bit_cast(uint32_t, v) & 0xffff0000u;
    v -= __builtin_bit_cast(float, top);
    return top;
  };
  x = -x;
  y = -y;
  const uint32_t x0 = part(x), x1 = part(x), x2 = part(x), y0 = part(y), y1 = part(y), y2 = part(y);
  return v4i{(int)(x0 >> 16 | x1), (int)(x2 >> 16 | y0), (int)(y1 >> 16 | y2), 0};
}
__device__ __forceinline__ v4i row_ones(bool second, int half) {
  return half ? v4i{0, 0, 0, 0} : second ? v4i{0, 0x3f800000, 0x3f803f80, 0} : v4i{0x3f803f80, 0x00003f80, 0, 0};
}
__device__ __forceinline__ v16f mfma32_bf16(v4i a, v4i b, v16f c) {
  typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
}

// eight of a lane's sixteen results, rounded: the operand of the next product (t: which eight)
__device__ __forceinline__ v8h round8(const v16f& x, int t) {
  v8h h;
#pragma unroll
  for (int i = 0; i < 8; ++i) h[i] = (_Float16)x[8 * t + i];
  return h;
}

// Eight of a lane's sixteen results of a 32 x 32 block, rounded: the block's column l % 32 is a row of memory, a lane has the columns 8 q + 4 (l / 32) .. + 3 of
// that row; the two halves of the wave exchange quads, so that each lane gets the columns 16 k + 8 (l / 32) .. + 7.
__device__ __forceinline__ v4i eight_columns(const v16f& x, int k, float f) {
  v4i o;
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const v2h a = {to_half(x[8 * k + 2 * e] * f), to_half(x[8 * k + 2 * e + 1] * f)};
    const v2h b = {to_half(x[8 * k + 4 + 2 * e] * f), to_half(x[8 * k + 5 + 2 * e] * f)};
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, a), __builtin_bit_cast(unsigned, b), false, false);
    const unsigned p = r[0], q = r[1];
    o[e] = (int)p;
    o[2 + e] = (int)q;
  }
  return o;
}
// A wave's 32 rows of COLS blocks of 32 columns (from column `col0` on) to memory, through LDS: whole rows at a time.  From the registers a store would write 32 bytes
// of each row, and memory takes such pieces at a fraction of its rate (16 x 16 heads of 64, 512 queries over up to 1024 keys: dK and dV 92 -> 73 us, O 41 -> 34).  Every wave of the workgroup calls it; columns from dh on stay as they are.
// row_of(r): where row r (of 32 from row0 on) starts, or NULL
template <int COLS, class R>
__device__ __forceinline__ void store_rows(uint8_t* lds, const v16f (&x)[COLS], float f, int row0, R row_of, int dh, int col0, int lane, int wave) {
  constexpr int G = COLS <= 4 ? COLS : COLS / 2, PITCH = 64 * G + 16;      // blocks at a time
  uint8_t* mine = lds + wave * 32 * PITCH;
#pragma unroll
  for (int g = 0; g < COLS; g += G) {
    __syncthreads();                 // the tiles, or the blocks before these, are used up
#pragma unroll
    for (int j = 0; j < G; ++j)
#pragma unroll
      for (int k = 0; k < 2; ++k) *US_LDS_AT(v4i, mine + (lane & 31) * PITCH + (4 * j + 2 * k + (lane >> 5)) * 16) = eight_columns(x[g + j], k, f);
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < 2 * G; ++i) {
      const int c = i * 64 + lane, row = c / (4 * G), chunk = c - row * (4 * G), col = col0 + 32 * g + 8 * chunk;
      const v4i o = *US_LDS_AT(const v4i, mine + row * PITCH + chunk * 16);
      _Float16* const to = row_of(row0 + row);
      if (to && col < dh) wt_store(reinterpret_cast<v4i*>(to + col), o);
    }
  }
}
// Such a block in FP32, 16 bytes a lane.
__device__ __forceinline__ void store_block_f32(float* row, int col0, int dh, bool on, int half, const v16f& x, float f) {
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int col = col0 + 8 * q + 4 * half;
    if (on && col < dh) wt_store(reinterpret_cast<v4f*>(row + col), v4f{x[4 * q] * f, x[4 * q + 1] * f, x[4 * q + 2] * f, x[4 * q + 3] * f});
  }
}

// What a workgroup does: item `x` of `nx`, `y` of `ny`, `z` of `nz` of a group that reads the same keys, all of them on one XCD where the groups can be dealt out
// evenly.  The host prepares the divisions.
struct Items {
  FastDiv by_xcds, by_per, by_x, by_y, by_kv;
  uint32_t xcds, per, nx, ny, kv, groups, blocks;
  static Items of(long groups, long kv, long nx, long ny, long nz, int xcds) {
    Items i;
    // Not where a group is one workgroup, which has nothing to share (54 x 53 heads of 128, 3 x 184, dQ: 60 us in order, 69 by XCD).  A few idle workgroups even the
    // groups out (124 heads of 2943 x 2909 x 128, dK and dV: 1560 us in order, 1460 with 128 groups).
    const long even = (groups + xcds - 1) / xcds * xcds;
    i.xcds = even * 10 <= groups * 11 && nx * ny * nz > 1 ? (uint32_t)xcds : 1u;
    i.groups = (uint32_t)groups;
    i.blocks = (uint32_t)((i.xcds > 1 ? even : groups) * nx * ny * nz);
    i.per = (uint32_t)(nx * ny * nz);
    i.nx = (uint32_t)nx;
    i.ny = (uint32_t)ny;
    i.kv = (uint32_t)kv;
    i.by_xcds = FastDiv::by(i.xcds);
    i.by_per = FastDiv::by(i.per);
    i.by_x = FastDiv::by(i.nx);
    i.by_y = FastDiv::by(i.ny);
    i.by_kv = FastDiv::by(i.kv);
    return i;
  }
  struct Item {
    int b, kvh, x, y, z;      // b < 0: nothing to do
  };
  __device__ __forceinline__ Item at(uint32_t block) const {
    const uint32_t i = by_xcds.of(block), xcd = block - i * xcds, q = by_per.of(i), group = q * xcds + xcd;
    uint32_t r = i - q * per;
    Item it;
    it.b = (int)by_kv.of(group);
    it.kvh = (int)(group - (uint32_t)it.b * kv);
    if (group >= groups) it.b = -1;
    const uint32_t rx = by_x.of(r), ry = by_y.of(rx);
    it.x = (int)(r - rx * nx);
    it.y = (int)(rx - ry * ny);
    it.z = (int)ry;
    return it;
  }
};

// Scheduling: n instructions of a kind next
template <int N> __device__ __forceinline__ void next_mfma() { __builtin_amdgcn_sched_group_barrier(0x008, N, 0); }
template <int N> __device__ __forceinline__ void next_valu() { __builtin_amdgcn_sched_group_barrier(0x002, N, 0); }
template <int N> __device__ __forceinline__ void next_exp() { __builtin_amdgcn_sched_group_barrier(0x400, N, 0); }
template <int N> __device__ __forceinline__ void next_lds_reads() { __builtin_amdgcn_sched_group_barrier(0x100, N, 0); }

// What the kernels need of a call.
struct Side {               // a tensor of heads, strides in elements
  const _Float16* p;
  long batch, head;
  int row;                  // bytes
};
struct AttendArgs {
  Side q, k, v, o, g;       // g: dO
  const int* klen;
  _Float16 *out, *dk, *dv;  // O or dQ (out_batch ..), dK and dV (laid out as k)
  long out_batch, out_head, out_row;
  float* lse;               // forward: L, or NULL
  v4i* rows;                // backward: RowStat of every query row, [batch * heads][sq]
  float* part;              // parts of split sums
  float2* stats;            // forward: {largest score (base 2), sum} of a part's rows
  long part_stride;         // elements between parts
  Items items;
  FastDiv by_sq;
  int batch, heads, kv, rep, sq, sk, dh, splits, per_split, tiles;      // tiles: of 16 rows (us_paged.hip)
  float c2, alpha, beta;    // c2 = dh^-1/2 log2(e);  alpha <= 0: n^1/2;  beta: factor of the gradient's store
  // The item with the slot-th most keys, of up to 64, which the lanes rank against one another: the longest first, so that the CUs' shares come out even (us: 16 items
  // of 16 heads of 64, 512 queries, 64 to 1024 keys: forward 35 -> 31, dQ 50 -> 44.  dK and dV, whose workgroups have equal work or none, do without: 70 or 75).
  __device__ __forceinline__ int by_keys(int slot) const {
    if (!klen || batch > 64) return slot;
    const int lane = threadIdx.x & 63, mine = lane < batch ? keys_of(lane) : 0;
    int rank = 0;
    for (int j = 0; j < batch; ++j) {
      const int other = __builtin_amdgcn_readlane(mine, j);
      rank += other > mine || (other == mine && j < lane) ? 1 : 0;
    }
    return __builtin_ctzll(__builtin_amdgcn_ballot_w64(lane < batch && rank == slot));
  }
  __device__ __forceinline__ int keys_of(int b) const {
    const int n = klen ? klen[b] : sk;
    return n < 0 ? 0 : n > sk ? sk : n;
  }
  // The factor a of a row over n keys; the factor f with which the backward pass rounds f p and f dS to FP16; and a / f, which its stores take.  f is a itself down to a mean
  // of a p of 2^-11, from which on it stays there, or at the default's n^1/2 if that is less (from 2^22 keys on).  Smaller ones leave FP16's normal numbers: 2-norm error of
  // dV, unit normal inputs, a = 1: 131072 keys 1.3e-3, 2^20 1.1e-2.  At 2^-11 the subnormal ones add at most 2^-25 / 3^1/2 each, 3.5e-5, to two roundings' 2.9e-4.
  __device__ __forceinline__ float factor(int n) const { return alpha > 0.0f ? alpha : __builtin_sqrtf((float)n); }
  __device__ __forceinline__ float inner_factor(int n) const {
    return __builtin_fmaxf(factor(n), __builtin_fminf(__builtin_sqrtf((float)n), (float)n * 0x1p-11f));
  }
  __device__ __forceinline__ float outer_factor(int n) const { return n > 0 ? factor(n) / inner_factor(n) : 1.0f; }
};
// The forward pass where a key head has few rows (us_paged.hip).
bool few_rows_take(long heads, long kv_heads, long sq);
size_t few_rows_workspace_bytes(long batch, long heads, long kv, long sq, long sk, long dh);
hipError_t launch_few_rows(AttendArgs a, void* workspace, hipStream_t st);

}  // namespace us
