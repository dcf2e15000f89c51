// 8-bit checkpoints of FP16 activations: rows in blocks of 32 values that share a power of two (us_gate.h says how a block is held).
// Bound: HBM, 2 + 1 + 1/32 bytes a value in either direction; 16384 x 8192 of rows 12288 apart: store 76 us = 5.3 TB/s, load 72 us = 5.6 (a large copy: 5.1);
// short rows, 1048576 x 16: 13.8 and 12.5 us, 3.7 and 4.1 TB/s.  A call of a few rows is its launch, 2.7 us on the device.  A thread holds 8 consecutive values, four neighbouring lanes a block, so the
// block's largest magnitude takes two exchanges inside a quad of lanes.
#include <type_traits>

#include "us_gate.h"
#include "us_launch.h"
#include "us_rows.h"

namespace us {

namespace {

constexpr int kThreads = 256;

// largest of the four lanes of a quad; a NaN does not count
__device__ __forceinline__ float quad_max(float v) {
  v = __builtin_fmaxf(v, lane_dpp<0xB1>(v));
  return __builtin_fmaxf(v, lane_dpp<0x4E>(v));
}

// 2^lx threads of a workgroup next to each other take chunks (8 values) of a row, the others more rows, so that short rows leave at most half of them
// idle; lanes beyond a row hold zeros, so a last block of 16 values is a block of 32.
__global__ void __launch_bounds__(kThreads) keep8_store_kernel(const _Float16* __restrict__ X, long ld, int8_t* __restrict__ codes,
                                                               uint8_t* __restrict__ scales, long rows, int n, int blocks, int lx) {
  const int chunk = (int)((blockIdx.x << lx) + (threadIdx.x & ((1u << lx) - 1))), col = chunk * 8, per = kThreads >> lx;
  for (long r = (long)blockIdx.y * per + (threadIdx.x >> lx); r < rows; r += (long)gridDim.y * per) {
    v8h x = {0, 0, 0, 0, 0, 0, 0, 0};
    if (col < n) x = *reinterpret_cast<const v8h*>(X + r * ld + col);
    float m = 0.0f;
    bool rare = false;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      m = __builtin_fmaxf(m, __builtin_fabsf((float)x[k]));
      rare |= x[k] != x[k];
    }
    m = quad_max(m);
    uint32_t s = keep_scale(m);
    const float inv = keep_inverse(s);
    // a NaN in any of the block's four lanes
    const uint64_t nans = __builtin_amdgcn_ballot_w64(rare) >> (threadIdx.x & 60) & 15;
    if (nans) s += kKeepNan;
    v2i c;
    if (rare || m >= kKeepClip) {
      c.x = keep_codes_any((float)x[0], (float)x[1], (float)x[2], (float)x[3], inv);
      c.y = keep_codes_any((float)x[4], (float)x[5], (float)x[6], (float)x[7], inv);
    } else {
      c.x = keep_codes((float)x[0], (float)x[1], (float)x[2], (float)x[3], inv);
      c.y = keep_codes((float)x[4], (float)x[5], (float)x[6], (float)x[7], inv);
    }
    if (col < n) {
      *reinterpret_cast<v2i*>(codes + r * n + col) = c;
      if ((chunk & 3) == 0) scales[r * blocks + (chunk >> 2)] = (uint8_t)s;
    }
  }
}

__global__ void __launch_bounds__(kThreads) keep8_load_kernel(const int8_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                                                              _Float16* __restrict__ X, long ld, long rows, int n, int blocks, int lx) {
  const int chunk = (int)((blockIdx.x << lx) + (threadIdx.x & ((1u << lx) - 1))), col = chunk * 8, per = kThreads >> lx;
  if (col >= n) return;
  for (long r = (long)blockIdx.y * per + (threadIdx.x >> lx); r < rows; r += (long)gridDim.y * per) {
    const v2i c = *reinterpret_cast<const v2i*>(codes + r * n + col);
    const uint32_t s = scales[r * blocks + (chunk >> 2)];
    float v[8];
    keep_values(c, keep_step(s > kKeepMost ? s - kKeepNan : s), v);
    if (s > kKeepMost) keep_put_nan(c, v);
    v8h x;
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = (_Float16)v[k];
    *reinterpret_cast<v8h*>(X + r * ld + col) = x;
  }
}

// Threads on a row: the power of two that holds its whole blocks, four (one block) at least.
int log_threads(long n) {
  int lx = 2;
  while ((8l << lx) < n && (1 << lx) < kThreads) ++lx;
  return lx;
}
dim3 grid_of(long rows, long n, int lx) {
  const long x = (n / 8 + (1l << lx) - 1) >> lx, per = kThreads >> lx, y = (rows + per - 1) / per;
  return dim3((unsigned)x, (unsigned)(y < 65535 ? y : 65535));
}

}  // namespace

hipError_t launch_keep8_store(const void* X, long ld, void* codes, void* scales, long rows, long n, hipStream_t st) {
  const int lx = log_threads(n);
  keep8_store_kernel<<<grid_of(rows, n, lx), kThreads, 0, st>>>((const _Float16*)X, ld, (int8_t*)codes, (uint8_t*)scales, rows, (int)n, (int)((n + 31) / 32), lx);
  return hipGetLastError();
}
hipError_t launch_keep8_load(const void* codes, const void* scales, void* X, long ld, long rows, long n, hipStream_t st) {
  const int lx = log_threads(n);
  keep8_load_kernel<<<grid_of(rows, n, lx), kThreads, 0, st>>>((const int8_t*)codes, (const uint8_t*)scales, (_Float16*)X, ld, rows, (int)n, (int)((n + 31) / 32), lx);
  return hipGetLastError();
}

}  // namespace us
