// Attention over whole sequences: kernels for bfloat16.
#include "attention_forward.hpp"

namespace ocn {
int run_attention_bfloat16(AttentionArgs &a, const AttentionPlan &p, bool vec, void *stream) { return run_type<bf16>(a, p, vec, (hipStream_t)stream); }
}  // namespace ocn
