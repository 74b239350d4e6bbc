// Attention over whole sequences: kernels for half.
#include "attention_forward.hpp"

namespace ocn {
int run_attention_half(AttentionArgs &a, const AttentionPlan &p, bool vec, void *stream) { return run_type<f16>(a, p, vec, (hipStream_t)stream); }
}  // namespace ocn
