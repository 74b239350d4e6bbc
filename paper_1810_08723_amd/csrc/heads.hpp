// Host side of the operators over heads (rotary positions, norms, the 4-bit cache, attention): argument checks and the
// leading dimensions of their tensors, merged.  Plain C++ with no HIP dependency.
//
// They take one type more than the planner's fifteen, OCN_BFLOAT16, so their checks are here and not in the planner.
#pragma once

#include <stdint.h>

#include "../../include/ocn.h"
#include "planner.hpp"

namespace ocn {

constexpr int kMaxLead = OCN_MAX_DIMS - 2;   // dimensions before heads and channels

// An operand of a call as its checks see it (t null: none).
struct HeadOperand {
  const ocn_tensor *t;
  bool output;
  int in_place = -1, in_place_b = -1;   // places among the operands of the inputs that an output may be the identical view of (one descriptor may be at several)
};

// The tokens: leading dimensions, merged where every operand's strides allow it, fastest last; with strides for each operand.
struct Lead {
  int32_t n;                          // dimensions left, at least 1
  uint32_t tokens;
  FastDiv div[kMaxLead];
};

int head_type_size(int32_t dtype);    // bytes of OCN_HALF, OCN_BFLOAT16, OCN_FLOAT and what index tensors hold; 0 for others

// One tensor by itself: pointer, rank, sizes, byte order, alignment; `types` is a bit set of the codes below.
enum { kHeadTypes = 1, kIndexTypes = 2, kDoubleType = 4, kByteType = 8, kFloatType = 16 };
int check_operand(const ocn_tensor *t, int types);
// One device; outputs that address no byte twice; nothing shared but what may be in place.
int check_operands(const HeadOperand *o, int n);
bool share_bytes(const ocn_tensor *a, const ocn_tensor *b);
bool identical_views(const ocn_tensor *a, const ocn_tensor *b);

// The merged leading dimensions of `x` (its last `inner` dimensions are not among them) and the strides along them of the n
// tensors of `with`, each broadcast against x's leading dimensions; inner_of[i]: how many trailing dimensions of with[i] are not leading ones.
int merge_lead(const ocn_tensor *x, int inner, const ocn_tensor *const *with, const int *inner_of, int n, Lead *lead,
               int64_t (*strides)[kMaxLead]);

// The cache of `heads` heads of `channels` channels; *page: the tokens of its pages.
constexpr int64_t kMaxPage = 1 << 20;
inline bool cache_channels(int64_t d) { return d == 64 || d == 128 || d == 256; }
int check_cache(const ocn_tensor *cache, int64_t channels, int64_t heads, int64_t *page);

int check_rotation(const ocn_rotation *r, int64_t channels, int32_t device);

}  // namespace ocn
