// Routing of a GEMM problem to its kernel family, and the split-K policy of the grad_W reduction.
#include <stdio.h>

#include "us_gemm_dispatch.h"

namespace us {

namespace {
// The current device as the entry point that is running found it, and what it launched.
constexpr int kNoCall = -1, kNotAsked = -2;
thread_local int g_call_device = kNoCall;
struct LaunchNote {
  const char* kind;
  int bm, bn, waves_k, nst, epi, splits, waves;
  bool fp8, a_kc, b_kc, wide, as_f16;
};
constexpr int kMaxNotes = 12;
thread_local LaunchNote g_notes[kMaxNotes];
thread_local int g_note_count = 0;
thread_local char g_record[1024];
}  // namespace

CallScope::CallScope() : outer(g_call_device) {
  g_note_count = 0;
  g_call_device = kNotAsked;
}
CallScope::~CallScope() { g_call_device = outer; }

hipError_t current_device(int* dev) {
  *dev = g_call_device;
  if (g_call_device >= 0) return hipSuccess;
  const hipError_t e = hipGetDevice(dev);
  if (e == hipSuccess && g_call_device == kNotAsked) g_call_device = *dev;
  return e;
}

const DeviceInfo& device_info() {
  static const DeviceInfo fallback{256, 8};
  static DeviceInfo info[kMaxDevices];
  static std::once_flag once[kMaxDevices];
  int dev = 0;
  if (current_device(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) return fallback;
  std::call_once(once[dev], [dev] {
    int cus = 0, xcds = 0;
    if (hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || cus < 1) cus = fallback.cus;
    if (hipDeviceGetAttribute(&xcds, hipDeviceAttributeNumberOfXccs, dev) != hipSuccess || xcds < 1) xcds = fallback.xcds;
    info[dev] = DeviceInfo{cus, xcds};
  });
  return info[dev];
}

void note_gemm_launch(const char* kind, int bm, int bn, int waves_k, int nst, bool fp8, bool a_kc, bool b_kc, int epi, bool wide,
                      int splits, int waves, bool as_f16) {
  if (g_note_count < kMaxNotes) g_notes[g_note_count++] = LaunchNote{kind, bm, bn, waves_k, nst, epi, splits, waves, fp8, a_kc, b_kc, wide, as_f16};
}

const char* last_launch_record() {
  static const char* const epi_name[] = {"store", "act", "act_grad", "partial", "gelu_tab", "gelu_grad_tab", "gelu_tab16", "residual",
                                         "softmax", "softmax_grad", "gate", "gate8", "gate_grad", "gate8_grad"};
  int len = 0;
  g_record[0] = 0;
  for (int i = 0; i < g_note_count; ++i) {
    const LaunchNote& n = g_notes[i];
    const int room = (int)sizeof(g_record) - len;
    char waves[16] = "";
    if (n.waves > 0) snprintf(waves, sizeof(waves), ":w%d", n.waves);
    const int w = snprintf(g_record + len, (size_t)room, "%s%s:%dx%d:wk%d:st%d:%s:%s:%s%s:s%d%s%s", i ? " + " : "", n.kind, n.bm, n.bn, n.waves_k,
                           n.nst, n.fp8 ? "fp8" : "f16", n.a_kc ? (n.b_kc ? "NT" : "NN") : (n.b_kc ? "TT" : "TN"),
                           (n.epi >= 0 && n.epi < 14) ? epi_name[n.epi] : "?", n.wide ? ":f32" : "", n.splits, waves, n.as_f16 ? ":as16" : "");
    if (w < 0 || w >= room) break;
    len += w;
  }
  return g_record;
}

// out[m][n] = round( scale * sum_s partial[s][m][n] ), slices added in order (deterministic).
__global__ void __launch_bounds__(256) splitk_reduce_kernel(const float* __restrict__ partial, void* out, long total,
                                                            int splits, float scale, int out_is_f32) {
  const long i4 = ((long)blockIdx.x * 256 + threadIdx.x) * 4;
  if (i4 >= total) return;
  v4f s = *reinterpret_cast<const v4f*>(partial + i4);
  for (int k = 1; k < splits; ++k) s += *reinterpret_cast<const v4f*>(partial + (size_t)k * total + i4);
  s *= scale;
  if (out_is_f32) {
    wt_store(reinterpret_cast<v4f*>((float*)out + i4), s);
  } else {
    v4h o = {to_half(s.x), to_half(s.y), to_half(s.z), to_half(s.w)};
    wt_store(reinterpret_cast<v4h*>((_Float16*)out + i4), o);
  }
}

hipError_t launch_splitk_reduce(const float* partial, void* out, long total, int splits, float scale, bool out_is_f32,
                                hipStream_t st) {
  splitk_reduce_kernel<<<(unsigned)((total / 4 + 255) / 256), 256, 0, st>>>(partial, out, total, splits, scale,
                                                                          out_is_f32 ? 1 : 0);
  return hipGetLastError();
}

// grad_W has a small output (fan_in x fan_out) and a long reduction (tokens).  When its large tiles
// cannot occupy the chip the small tile is used (two workgroups per CU: twice the CU count in slots), and if even those
// are too few the token range is cut into slices of whole 128-token stages, at least 512 tokens each.
long gemm_k_per_split(long K, int splits) {
  const long unit = 128;
  return ((K + splits - 1) / splits + unit - 1) / unit * unit;
}

int gemm_splits(long M, long N, long K) {
  if (use_big_tile(M, N, 1) || K < 1024 || use_wave_split_tile(M, N, K)) return 1;
  const long tiles = ceil_div(M, 128) * ceil_div(N, 128);
  long s = 2 * cu_count() / tiles;
  const long max_by_k = K / 512;
  if (s > max_by_k) s = max_by_k;
  if (s > 8) s = 8;
  if (s < 1) s = 1;
  const long kps = gemm_k_per_split(K, (int)s);
  return (int)((K + kps - 1) / kps);
}

size_t gemm_workspace_bytes(long M, long N, long K) {
  const int s = gemm_splits(M, N, K);
  return s <= 1 ? 0 : (size_t)s * (size_t)M * (size_t)N * sizeof(float);
}

hipError_t gemm_gate_fwd_f16(const GemmProblem& p, bool keep8, hipStream_t st);
hipError_t gemm_gate_fwd_fp8(const GemmProblem& p, bool keep8, hipStream_t st);
hipError_t gemm_gate_grad_f16(const GemmProblem& p, bool keep8, hipStream_t st);
hipError_t gemm_gate_grad_fp8(const GemmProblem& p, bool keep8, hipStream_t st);
hipError_t gemm_gate_three_f16(const GemmProblem& dx, const GemmProblem& dwgu, const GemmProblem& dwd, hipStream_t st);
hipError_t gemm_gate_three_fp8(const GemmProblem& dx, const GemmProblem& dwgu, const GemmProblem& dwd, hipStream_t st);

// All three products of the gated block behind dZ in one launch: where all are few tiles (two launches fall away: FP16 64 x 256 x 688 backward call 14.4 -> 11.6 us),
// or on 128 x 128 tiles, two workgroups per CU, where the longest tile takes half to two and a half times a workgroup's share of the work and none of
// them makes large tiles for all CUs.  Backward call, two or three launches with K slices -> one: FP16 4096 x 768 x 2048 112.8 -> 87.6, FP8 3000 x 768 x 2048
// 65.4 -> 41.8, 1024 x 2048 x 5632 106 -> 95; over 32 drawn blocks that the rule takes the geometric mean is 0.85, none slower.
//  Outside: longest / share = 0.4 FP8 8192 x 1024 x 4096 233.9 -> 233.4, FP16 6189 x 1360 x 2720 352 -> 359; 3.2 FP16 1024 x 1024 x 2048 54.9 -> 58.2, FP8 1024 x 1024 x 2736 50.5 -> 55.4, 9 FP8 16000 x 256 x 688 81 -> 124.
bool gemm_gate_three_ok(const GemmProblem& dx, const GemmProblem& dwgu, const GemmProblem& dwd) {
  if (!offsets_fit(dx) || !offsets_fit(dwgu) || !offsets_fit(dwd)) return false;
  if (small_tile_choice(dx) != SmallTileChoice::None && small_tile_choice(dwgu) != SmallTileChoice::None && small_tile_choice(dwd) != SmallTileChoice::None) return true;
  if (use_big_tile(dx.M, dx.N, 1) || use_big_tile(dwgu.M, dwgu.N, 1) || use_big_tile(dwd.M, dwd.N, 1)) return false;
  auto tiles = [](const GemmProblem& p) { return ceil_div(p.M, 128) * ceil_div(p.N, 128); };
  const long work = tiles(dx) * dx.K + (tiles(dwgu) + tiles(dwd)) * dwd.K, longest = dx.K > dwd.K ? dx.K : dwd.K;
  return 4 * cu_count() * longest >= work && 4 * cu_count() * longest <= 5 * work;
}
hipError_t gemm_gate_three(const GemmProblem& dx, const GemmProblem& dwgu, const GemmProblem& dwd, hipStream_t st) {
  return dx.a_dt == US_F16 ? gemm_gate_three_f16(dx, dwgu, dwd, st) : gemm_gate_three_fp8(dx, dwgu, dwd, st);
}
bool gemm_gate_offsets_fit(const GemmProblem& p) { return offsets_fit(p); }
hipError_t gemm_gate_fwd(const GemmProblem& p, bool keep8, hipStream_t st) {
  return p.a_dt == US_F16 ? gemm_gate_fwd_f16(p, keep8, st) : gemm_gate_fwd_fp8(p, keep8, st);
}
hipError_t gemm_gate_grad(const GemmProblem& p, bool keep8, hipStream_t st) {
  return p.a_dt == US_F16 ? gemm_gate_grad_f16(p, keep8, st) : gemm_gate_grad_fp8(p, keep8, st);
}

hipError_t launch_gemm(const GemmProblem& p, hipStream_t st) {
  const bool fp8 = (p.a_dt != US_F16);
  if (p.a_kc && !p.b_kc) return fp8 ? gemm_nn_fp8(p, st) : gemm_nn_f16(p, st);
  if (p.a_kc && p.b_kc) return fp8 ? gemm_nt_fp8(p, st) : gemm_nt_f16(p, st);
  if (!p.a_kc && !p.b_kc) return fp8 ? gemm_tn_fp8(p, st) : gemm_tn_f16(p, st);
  return hipErrorInvalidValue;
}

}  // namespace us
