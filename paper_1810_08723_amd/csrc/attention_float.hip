// Attention over whole sequences: kernels for float.
#include "attention_forward.hpp"

namespace ocn {
int run_attention_float(AttentionArgs &a, const AttentionPlan &p, bool vec, void *stream) { return run_type<float>(a, p, vec, (hipStream_t)stream); }
}  // namespace ocn
