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
// A row of up to 32 NB halves takes `pitch` bytes, a power of two; its 16-byte chunk c lies at c ^ swz(row).  The bits are chosen for both
// ways of reading: sixteen lanes that read the same chunk of rows r .. r + 15, and a transposing read whose 32 lanes touch 64 bytes in each of
// four rows; both meet every bank once.
template <int NB>
struct RowTile {
  static constexpr int P = NB == 1 ? 64 : NB == 2 ? 128 : NB <= 4 ? 256 : 512;
  static constexpr int CHUNKS = P / 16;
  __device__ __forceinline__ static int swz(int row) {
    if (P == 64) return (row >> 2) & 3;
    if (P == 128) return (((row >> 1) & 1) << 2) | ((row >> 2) & 3);
    return ((row & 3) << 2) | ((row >> 2) & 3);
  }
  // rows as the first operand of the 32 x 32 x 16 instruction: lane l has row l % 32 (+ 32 rb), columns 16 t + 8 (l / 32) ..
  __device__ __forceinline__ static v8h row_fragment(const uint8_t* tile, int rb, int t, int l32, int half) {
    const int row = rb * 32 + l32;
    return *US_LDS_AT(const v8h, tile + row * P + (((2 * t + half) ^ swz(row)) << 4));
  }
  // ... and transposed: lane l has column 32 nb + l % 32 and the rows 16 t + 4 (l / 32) + (0 .. 3, 8 .. 11), which are the rows that the
  // results of a 32 x 32 instruction leave in a lane
  __device__ __forceinline__ static v8h column_fragment(const uint8_t* tile, int t, int nb, int lane) {
    const int l16 = lane & 15, row = 16 * t + 4 * (lane >> 5) + (l16 >> 2);
    const int chunk = nb * 4 + ((lane >> 4) & 1) * 2 + ((l16 & 3) >> 1);
    // (the rows 8 further on: swz() changes by a bit that the four rows share)
    const uint8_t* at = tile + row * P + ((chunk ^ swz(row)) << 4) + (l16 & 1) * 8;
    const uint8_t* at8 = tile + (row + 8) * P + ((chunk ^ swz(row + 8)) << 4) + (l16 & 1) * 8;
    const v4s a = __builtin_amdgcn_ds_read_tr16_b64_v4i16(US_LDS_AT(v4s, at));
    const v4s b = __builtin_amdgcn_ds_read_tr16_b64_v4i16(US_LDS_AT(v4s, at8));
    struct { v4s a, b; } both = {a, b};
    return __builtin_bit_cast(v8h, both);
  }
};

// 16 bytes per lane straight to LDS, lane after lane from `lds` on; zeros where the offset lies beyond the resource.  (A function of its own: from inside a lambda
// that a kernel template calls, the compiler's host pass leaves out the kernel's stub.)
__device__ __forceinline__ void load_to_lds(__amdgpu_buffer_rsrc_t from, uint8_t* lds, int off) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(from, US_LDS_AT(void, lds), 16, off, 0, 0, 0);
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
  __device__ __forceinline__ void request(const void* base, long rows, int row_bytes, int dh, uint8_t* lds, int wave) const {
    const int r = rows > ROWS ? ROWS : rows < 0 ? 0 : (int)rows;
    const __amdgpu_buffer_rsrc_t res = __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, r > 0 ? (r - 1) * row_bytes + dh * 2 : 0, 0x00027000);
#pragma unroll
    for (int j = 0; j < LD; ++j)
      if (BYTES / 16 % THREADS == 0 || j * THREADS + wave * 64 < BYTES / 16)
        load_to_lds(res, lds + (j * THREADS + wave * 64) * 16, (int)off[j]);
  }
};

// all of the wave's loads have landed and its LDS reads are done
__device__ __forceinline__ void wait_all() { __builtin_amdgcn_s_waitcnt(0x0070); }

__device__ __forceinline__ v16f zero16() {
  v16f z;
#pragma unroll
  for (int r = 0; r < 16; ++r) z[r] = 0.0f;
  return z;
}
__device__ __forceinline__ v16f mfma32(v8h a, v8h b, v16f c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }

// eight of a lane's sixteen results, rounded: the operand of the next product (t: which eight)
__device__ __forceinline__ v8h round8(const v16f& x, int t) {
  v8h h;
#pragma unroll
  for (int i = 0; i < 8; ++i) h[i] = (_Float16)x[8 * t + i];
  return h;
}

// A lane's 32 x 32 block of results, column l % 32 of the block being a row of memory: rows 8 q + 4 (l / 32) .. + 3 are four of that row's columns;
// the two halves of the wave exchange quads, so that each lane stores 16 bytes: columns 16 k + 8 (l / 32) .. + 7, k = 0, 1.
__device__ __forceinline__ void store_block(_Float16* row, int col0, int dh, bool on, int half, const v16f& x, float f) {
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    v2i lo, hi;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const v2h a = {to_half(x[8 * k + 2 * e] * f), to_half(x[8 * k + 2 * e + 1] * f)};
      const v2h b = {to_half(x[8 * k + 4 + 2 * e] * f), to_half(x[8 * k + 5 + 2 * e] * f)};
      const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, a), __builtin_bit_cast(unsigned, b), false, false);
      const unsigned p = r[0], q = r[1];
      lo[e] = (int)p;
      hi[e] = (int)q;
    }
    const int col = col0 + 16 * k + 8 * half;
    if (on && col < dh) wt_store(reinterpret_cast<v4i*>(row + col), v4i{lo[0], lo[1], hi[0], hi[1]});
  }
}
// ... and in FP32
__device__ __forceinline__ void store_block_f32(float* row, int col0, int dh, bool on, int half, const v16f& x, float f) {
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int col = col0 + 8 * q + 4 * half;
    if (on && col < dh) wt_store(reinterpret_cast<v4f*>(row + col), v4f{x[4 * q] * f, x[4 * q + 1] * f, x[4 * q + 2] * f, x[4 * q + 3] * f});
  }
}

// Work item of a workgroup whose groups (of `per` items that read the same keys) go to one XCD each, where there are enough of them.
__device__ __forceinline__ void group_item(long block, long groups, long per, int xcds, long& group, long& item) {
  if (xcds > 1 && groups % xcds == 0) {
    const long xcd = block % xcds, i = block / xcds;
    group = i / per * xcds + xcd;
    item = i % per;
  } else {
    group = block / per;
    item = block % per;
  }
}

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
  const float2* rows;       // backward: {log2(e) L - log2(a), D} of [batch * heads][sqp]
  float* part;              // parts of split sums
  float2* stats;            // forward: {largest score (base 2), sum} of a part's rows
  long part_stride;         // elements between parts
  int batch, heads, kv, rep, sq, sqp, sk, dh, tiles, splits, per_split, xcds;
  float c2, alpha, beta;    // c2 = dh^-1/2 log2(e);  alpha <= 0: n^1/2;  beta: factor of the gradient's store
  __device__ __forceinline__ int keys_of(int b) const {
    const int n = klen ? klen[b] : sk;
    return n < 0 ? 0 : n > sk ? sk : n;
  }
};
hipError_t launch_join(const AttendArgs& a, hipStream_t st);      // us_cross.hip
// The forward pass where a key head has few rows (us_paged.hip).
bool few_rows_take(long heads, long kv_heads, long sq);
size_t few_rows_workspace_bytes(long batch, long heads, long kv, long sq, long sk, long dh);
hipError_t launch_few_rows(AttendArgs a, void* workspace, hipStream_t st);

}  // namespace us
