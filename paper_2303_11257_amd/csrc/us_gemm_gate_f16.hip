// GEMM family: the gated block's forward product with both halves of Wgu, and dH with the gate's gradient.
#include "us_gemm_gate_dispatch.h"

namespace us {

hipError_t gemm_gate_fwd_f16(const GemmProblem& p, bool keep8, hipStream_t st) {
  return keep8 ? launch_gate<false, false, EPI_GATE8>(p, st) : launch_gate<false, false, EPI_GATE>(p, st);
}
hipError_t gemm_gate_grad_f16(const GemmProblem& p, bool keep8, hipStream_t st) {
  return keep8 ? launch_gate<false, true, EPI_GATE8_GRAD>(p, st) : launch_gate<false, true, EPI_GATE_GRAD>(p, st);
}
hipError_t gemm_gate_three_f16(const GemmProblem& dx, const GemmProblem& dwgu, const GemmProblem& dwd, hipStream_t st) {
  return launch_three_grads<false>(dx, dwgu, dwd, st);
}

}  // namespace us
