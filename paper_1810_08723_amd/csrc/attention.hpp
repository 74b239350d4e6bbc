// Host side of attention over whole sequences: arguments, checks, and how queries or keys go to workgroups.  Plain C++ with no HIP dependency.
#pragma once

#include <stdint.h>

#include "heads.hpp"

namespace ocn {

// A tensor of heads: strides in bytes
struct HeadView {
  char *base;
  int64_t batch, token, head, channel;
};

// Starts of packed sequences; p null: `sequences` of `all` tokens each
struct Starts {
  const char *p;
  int64_t stride, all;
  int32_t wide, sequences;
};

struct AttentionArgs {
  HeadView q, k, v, out, log_sum;
  HeadView gout, gq, gk, gv;               // of the gradient
  Starts q_starts, k_starts;
  int32_t channels, kv, per_kv;            // per_kv: query heads to a head of keys and values
  int32_t causal, window;                  // window 0: none
  int32_t negative, nothing;               // the scale is below zero; is zero
  float scale, plain_scale, true_scale;    // of scores: to powers of two and to those of e, as magnitudes; as it is
  // blocks of a sequence: of `tokens` queries (keys, where a block has keys), and of `heads` query heads of a group
  int32_t heads, head_blocks, tokens, splits;
  int32_t rows;                            // of a block
  int32_t rows_of_tile;                    // gradients of keys: queries that a tile of rows has
  uint32_t slots, per_sequence;            // of all sequences; of one, where they are not packed
  FastDiv heads_div, head_blocks_div, across_div, tokens_div, splits_div, sequences_div;
  uint32_t *order;                         // [slots], those with most to do first; null: as they come
  float *parts, *part_sums;                // forward: [units][splits][rows][channels], [..][2]: largest score and sum
};

struct AttentionSizes {
  bool packed;
  int64_t sequences, queries, keys;        // tokens in all
  int64_t kv, per_kv;
};

// q, k and q_starts by themselves; what the checks of a whole call begin with
int check_attention_sizes(const ocn_tensor *q, const ocn_tensor *k, const ocn_tensor *q_starts);
AttentionSizes sizes_of(const ocn_tensor *q, const ocn_tensor *k, const ocn_tensor *q_starts);
// inputs, starts, scale and window of a call, checked, into `a`
int fill_attention(AttentionArgs &a, const ocn_tensor *q, const ocn_tensor *k, const ocn_tensor *v, const ocn_tensor *q_starts, const ocn_tensor *k_starts,
                   double scale, int64_t window, uint32_t flags);
int check_like(const ocn_tensor *t, const ocn_tensor *q);          // the type and sizes of q
int check_sums(const ocn_tensor *log_sum, const ocn_tensor *q);    // or NULL
HeadView view_of(const ocn_tensor *t, bool channels = true);
bool whole_rows(const ocn_tensor *t);                              // rows of whole, aligned 16 bytes

// Blocks of `rows` rows (a query with a head of its group each): units in all, a unit being a block of a head of keys and values
int64_t units_of(const AttentionSizes &s, int64_t rows);
// ... of `keys` keys
int64_t key_units_of(const AttentionSizes &s, int64_t keys);
// Sets what find_work goes by; false where there are too many
bool set_blocks(AttentionArgs &a, const AttentionSizes &s, int64_t rows, int64_t splits);
bool set_key_blocks(AttentionArgs &a, const AttentionSizes &s, int64_t keys, int64_t splits);

// channels that kernels are made for
inline int padded_channels(int64_t d) { return d <= 64 ? 64 : d <= 80 ? 80 : d <= 96 ? 96 : d <= 128 ? 128 : d <= 192 ? 192 : 256; }

// ... and those of a result, whole tiles
inline int64_t result_channels(int32_t dtype, int64_t d) { return dtype == OCN_FLOAT ? padded_channels(d) : (padded_channels(d) + 31) / 32 * 32; }

// What the shapes alone decide of a call: whether rows are few (the wavefronts of a workgroup then share them and take keys in turn), rows of a block, the parts that a
// sequence's keys go to, units.
constexpr int kFewWaves = 4;
constexpr int kLeastTiles = 2 * kFewWaves;        // tiles of keys of a part, at least
constexpr int kLeastRowTiles = 3;                 // ... where rows are many, and tiles larger
struct AttentionPlan { bool few; int waves, rows, splits; int64_t units; };      // waves: of a workgroup
int run_attention_half(AttentionArgs &a, const AttentionPlan &p, bool vec, void *stream);
int run_attention_bfloat16(AttentionArgs &a, const AttentionPlan &p, bool vec, void *stream);
int run_attention_float(AttentionArgs &a, const AttentionPlan &p, bool vec, void *stream);

// From so many workgroups on, which are more than there are CUs, packed sequences' blocks of keys are put in order, by a launch of 5 us (32 query heads, 8 of keys, 128 channels,
// bfloat16, all gradients: 1.89 for 2.27 ms of 4 sequences of 4096 tokens, 2.89 for 3.40 of 16 of 100 to 4096 in any order).  Blocks of queries, which are smaller and of which
// neighbours that share keys are better kept together, take as long either way (forward: 0.90 and 0.90 ms of those 16).  One workgroup puts them in order, two blocks to a lane at
// most: more are so many that the last ones matter little (400 sequences of 10 to 1000 tokens, 8 heads, 1189 blocks of each: 2.09 for 2.19 ms; 2000 of 10 to 100, 2860 blocks: 0.65 for 0.61).
constexpr int64_t kOrderUnits = kNumCUs + 1;
constexpr int kOrderLanes = 1024;
inline bool ordered(const AttentionSizes &s, int64_t units, int64_t slots) { return s.packed && units >= kOrderUnits && slots <= 2 * kOrderLanes; }
int64_t slots_of_key_units(const AttentionSizes &s, int64_t keys);

// The gradient: rows (query heads of all tokens), and which gradients are wanted
constexpr int kGradWaves = 4;
struct AttentionGrad { int64_t rows; bool keys, queries; };
// ... wavefronts and parts of a block of keys
size_t grad_head_bytes(const AttentionSizes &s, int side, int waves);       // of the workspace before what parts leave
struct KeyPlan { int waves, splits; int64_t units; };
KeyPlan key_plan_of(const AttentionSizes &s, int32_t dtype, int64_t channels);
constexpr int kLeastKeyTiles = 4;        // tiles of rows of a part, at least
int run_attention_grad_half(AttentionArgs &a, const AttentionSizes &s, const AttentionGrad &p, bool vec, void *workspace, void *stream);
int run_attention_grad_bfloat16(AttentionArgs &a, const AttentionSizes &s, const AttentionGrad &p, bool vec, void *workspace, void *stream);
int run_attention_grad_float(AttentionArgs &a, const AttentionSizes &s, const AttentionGrad &p, bool vec, void *workspace, void *stream);

// CALL(type, padded channels, whole rows)
#define OCN_BY_ROWS(T, D, vec, CALL) \
  do {                               \
    if (vec) CALL(T, D, true);       \
    else CALL(T, D, false);          \
  } while (0)
#define OCN_BY_PADDED(T, d, vec, CALL)             \
  do {                                             \
    switch (padded_channels(d)) {                  \
      case 64: OCN_BY_ROWS(T, 64, vec, CALL);      \
      case 80: OCN_BY_ROWS(T, 80, vec, CALL);      \
      case 96: OCN_BY_ROWS(T, 96, vec, CALL);      \
      case 128: OCN_BY_ROWS(T, 128, vec, CALL);    \
      case 192: OCN_BY_ROWS(T, 192, vec, CALL);    \
      default: OCN_BY_ROWS(T, 256, vec, CALL);     \
    }                                              \
  } while (0)

}  // namespace ocn
