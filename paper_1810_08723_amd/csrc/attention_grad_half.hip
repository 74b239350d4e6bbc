// Gradient of attention over whole sequences: kernels for half.
#include "attention_backward.hpp"

namespace ocn {
int run_attention_grad_half(AttentionArgs &a, const AttentionSizes &s, const AttentionGrad &p, bool vec, void *workspace, void *stream) {
  return run_grad_type<f16>(a, s, p, vec, workspace, (hipStream_t)stream);
}
}  // namespace ocn
