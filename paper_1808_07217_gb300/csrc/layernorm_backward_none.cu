#include "layernorm_backward.cuh"

namespace lsgd {
cudaError_t launch_ln_backward_none(const LnArgs& a, int G, bool xb, bool yb, int vmax, cudaStream_t st) {
  return ln_backward_any<LSGD_ACT_NONE>(a, G, xb, yb, vmax, st);
}
int take_ln_backward_late_none() { return take_rows_late(); }
}  // namespace lsgd
