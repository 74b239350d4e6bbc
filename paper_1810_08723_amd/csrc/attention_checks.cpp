// Attention over whole sequences and its gradient: arguments, how work is cut into blocks, and the entry points.
#include <algorithm>
#include <cmath>
#include <cstring>

#include "attention.hpp"

namespace ocn {

constexpr int64_t kMostRows = (int64_t)1 << 31;       // query heads of all tokens, and whatever else is counted in 32 bits: fewer than so many
constexpr int64_t kMostTokens = (int64_t)1 << 30;     // of all sequences: sums of two positions and a window stay below 2^31

static int check_rows(const ocn_tensor *t, bool packed) {
  const int rc = check_operand(t, kHeadTypes);
  if (rc != OCN_OK) return rc;
  if (t->ndim != (packed ? 3 : 4)) return OCN_ERR_NDIM;
  const int64_t *s = t->size + (packed ? 0 : 1);
  if (s[2] > OCN_MAX_ATTENTION_CHANNELS || s[1] >= ((int64_t)1 << 24) || s[0] > kMostTokens) return OCN_ERR_SHAPE;
  if (!packed && (t->size[0] >= kMostRows || (t->size[0] && s[0] > kMostTokens / t->size[0]))) return OCN_ERR_SHAPE;
  return OCN_OK;
}

int check_attention_sizes(const ocn_tensor *q, const ocn_tensor *k, const ocn_tensor *q_starts) {
  const bool packed = q_starts != nullptr;
  int rc;
  if ((rc = check_rows(q, packed)) != OCN_OK || (rc = check_rows(k, packed)) != OCN_OK) return rc;
  if (packed) {
    if ((rc = check_operand(q_starts, kIndexTypes)) != OCN_OK) return rc;
    if (q_starts->ndim != 1) return OCN_ERR_NDIM;
    if (q_starts->size[0] < 1 || q_starts->size[0] >= kMostRows) return OCN_ERR_SHAPE;
  }
  if (q->dtype != k->dtype) return OCN_ERR_DTYPE;
  const int at = packed ? 0 : 1;
  if (!packed && q->size[0] != k->size[0]) return OCN_ERR_SHAPE;
  if (q->size[at + 2] != k->size[at + 2]) return OCN_ERR_SHAPE;
  const int64_t heads = q->size[at + 1], kv = k->size[at + 1];
  if (kv == 0 ? heads != 0 : heads % kv != 0) return OCN_ERR_SHAPE;
  // (rows of a head of keys and values, and of all heads)
  const int64_t tokens = packed ? q->size[0] : q->size[0] * q->size[1];
  if (tokens && heads >= kMostRows / tokens) return OCN_ERR_SHAPE;
  return OCN_OK;
}

AttentionSizes sizes_of(const ocn_tensor *q, const ocn_tensor *k, const ocn_tensor *q_starts) {
  AttentionSizes s;
  s.packed = q_starts != nullptr;
  const int at = s.packed ? 0 : 1;
  s.sequences = s.packed ? q_starts->size[0] - 1 : q->size[0];
  s.queries = s.packed ? q->size[0] : q->size[0] * q->size[1];
  s.keys = s.packed ? k->size[0] : k->size[0] * k->size[1];
  s.kv = k->size[at + 1];
  s.per_kv = s.kv ? q->size[at + 1] / s.kv : 0;
  return s;
}

static bool same_sizes(const ocn_tensor *a, const ocn_tensor *b) {
  if (a->ndim != b->ndim) return false;
  for (int d = 0; d < a->ndim; ++d)
    if (a->size[d] != b->size[d]) return false;
  return true;
}

int check_like(const ocn_tensor *t, const ocn_tensor *q) {
  const int rc = check_operand(t, kHeadTypes);
  if (rc != OCN_OK) return rc;
  if (t->dtype != q->dtype) return OCN_ERR_DTYPE;
  return same_sizes(t, q) ? OCN_OK : OCN_ERR_SHAPE;
}

int check_sums(const ocn_tensor *log_sum, const ocn_tensor *q) {
  if (!log_sum) return OCN_OK;
  const int rc = check_operand(log_sum, kFloatType);
  if (rc != OCN_OK) return rc;
  if (log_sum->ndim != q->ndim - 1) return OCN_ERR_NDIM;
  for (int d = 0; d < log_sum->ndim; ++d)
    if (log_sum->size[d] != q->size[d]) return OCN_ERR_SHAPE;
  return OCN_OK;
}

HeadView view_of(const ocn_tensor *t, bool channels) {
  HeadView v;
  const int token = t->ndim - (channels ? 3 : 2);      // 1 where there is a dimension of sequences
  v.base = (char *)t->base + t->offset;
  v.batch = token ? t->stride[0] : 0;
  v.token = t->stride[token];
  v.head = t->stride[token + 1];
  v.channel = channels ? t->stride[token + 2] : 0;
  return v;
}

bool whole_rows(const ocn_tensor *t) {
  const int64_t size = head_type_size(t->dtype);
  if (t->size[t->ndim - 1] * size % 16 != 0 || (t->size[t->ndim - 1] > 1 && t->stride[t->ndim - 1] != size) || ((intptr_t)t->base + t->offset) % 16 != 0) return false;
  for (int d = 0; d + 1 < t->ndim; ++d)
    if (t->size[d] > 1 && t->stride[d] % 16 != 0) return false;
  return true;
}

static Starts starts_of(const ocn_tensor *starts, const ocn_tensor *x) {
  Starts s;
  s.p = starts ? (const char *)starts->base + starts->offset : nullptr;
  s.stride = starts ? starts->stride[0] : 0;
  s.all = starts ? x->size[0] : x->size[1];
  s.wide = starts && starts->dtype == OCN_INT64;
  s.sequences = (int32_t)(starts ? starts->size[0] - 1 : x->size[0]);
  return s;
}

int fill_attention(AttentionArgs &a, const ocn_tensor *q, const ocn_tensor *k, const ocn_tensor *v, const ocn_tensor *q_starts, const ocn_tensor *k_starts,
                   double scale, int64_t window, uint32_t flags) {
  if (!q || !k || !v || (!q_starts) != (!k_starts)) return OCN_ERR_NULLPTR;
  if (flags & ~OCN_CAUSAL) return OCN_ERR_OP;
  int rc = check_attention_sizes(q, k, q_starts);
  if (rc != OCN_OK || (rc = check_like(v, k)) != OCN_OK) return rc;
  if (k_starts) {
    if ((rc = check_operand(k_starts, kIndexTypes)) != OCN_OK) return rc;
    if (k_starts->ndim != 1) return OCN_ERR_NDIM;
    if (k_starts->size[0] != q_starts->size[0]) return OCN_ERR_SHAPE;
  }
  const bool causal = (flags & OCN_CAUSAL) != 0;
  if (window < 0 || (window > 0 && !causal)) return OCN_ERR_SHAPE;
  const double powers = std::fabs(scale) * 1.4426950408889634074;
  if (!(powers <= 3.4028234663852886e38)) return OCN_ERR_DOMAIN;
  const AttentionSizes s = sizes_of(q, k, q_starts);
  a.q = view_of(q), a.k = view_of(k), a.v = view_of(v);
  a.q_starts = starts_of(q_starts, q);
  a.k_starts = starts_of(k_starts, k);
  a.channels = (int32_t)q->size[q->ndim - 1];
  a.kv = (int32_t)s.kv;
  a.per_kv = (int32_t)s.per_kv;
  a.causal = causal;
  a.window = window >= a.k_starts.all ? 0 : (int32_t)window;      // (one of all keys is none)
  // (With a scale of zero, as single precision has it, queries are taken as zeros: places that are not seen have scores of minus infinity, which times zero would be NaN.)
  a.nothing = (float)powers == 0.0f || (float)std::fabs(scale) == 0.0f;
  a.negative = scale < 0.0;
  a.scale = a.nothing ? 1.0f : (float)powers;
  a.plain_scale = a.nothing ? 1.0f : (float)std::fabs(scale);
  a.true_scale = (float)scale;
  return OCN_OK;
}

// heads of a block of so many rows, and queries
static int64_t heads_of_block(const AttentionSizes &s, int64_t rows) { return std::max<int64_t>(1, std::min(s.per_kv, rows)); }

static int64_t slots_of(const AttentionSizes &s, int64_t all, int64_t tokens) {
  if (s.sequences == 0 || all == 0) return 0;
  return s.packed ? all / tokens + s.sequences : s.sequences * ((all / s.sequences + tokens - 1) / tokens);
}

static int64_t slots_of_units(const AttentionSizes &s, int64_t rows) { return slots_of(s, s.queries, rows / heads_of_block(s, rows)); }
int64_t slots_of_key_units(const AttentionSizes &s, int64_t keys) { return slots_of(s, s.keys, keys); }
int64_t units_of(const AttentionSizes &s, int64_t rows) {
  const int64_t heads = heads_of_block(s, rows);
  return slots_of_units(s, rows) * s.kv * ((s.per_kv + heads - 1) / heads);
}
int64_t key_units_of(const AttentionSizes &s, int64_t keys) { return slots_of_key_units(s, keys) * s.kv; }

static bool set_all(AttentionArgs &a, const AttentionSizes &s, int64_t all, int64_t heads, int64_t head_blocks, int64_t tokens, int64_t splits) {
  const int64_t slots = slots_of(s, all, tokens);
  if (slots >= kMostRows || s.kv * head_blocks >= kMostRows || slots * (s.kv * head_blocks) >= kMostRows / splits) return false;
  a.heads = (int32_t)heads;
  a.head_blocks = (int32_t)head_blocks;
  a.tokens = (int32_t)tokens;
  a.splits = (int32_t)splits;
  a.slots = (uint32_t)slots;
  a.per_sequence = (uint32_t)(s.packed || !s.sequences ? 1 : slots / s.sequences);
  a.heads_div = make_fastdiv((uint32_t)heads);
  a.head_blocks_div = make_fastdiv((uint32_t)head_blocks);
  a.across_div = make_fastdiv((uint32_t)std::max<int64_t>(1, s.kv * head_blocks));
  a.tokens_div = make_fastdiv((uint32_t)tokens);
  a.splits_div = make_fastdiv((uint32_t)splits);
  a.sequences_div = make_fastdiv((uint32_t)std::max<int64_t>(1, s.sequences));
  return true;
}

size_t grad_head_bytes(const AttentionSizes &s, int side, int waves) {
  const size_t n = (size_t)(s.queries * s.kv * s.per_kv + 1) * 4 * sizeof(float) +
                   (size_t)slots_of_key_units(s, side * waves) * sizeof(uint32_t);
  return (n + 255) / 256 * 256;
}

bool set_blocks(AttentionArgs &a, const AttentionSizes &s, int64_t rows, int64_t splits) {
  const int64_t heads = heads_of_block(s, rows);
  return set_all(a, s, s.queries, heads, std::max<int64_t>(1, (s.per_kv + heads - 1) / heads), rows / heads, splits);
}
bool set_key_blocks(AttentionArgs &a, const AttentionSizes &s, int64_t keys, int64_t splits) {
  return set_all(a, s, s.keys, std::max<int64_t>(1, s.per_kv), 1, keys, splits);
}

// Rows of few blocks of keys in parts (one sequence of 2048 tokens, 16 heads, 2 of keys, 128 channels, forward and gradient: 214 for 938 us)
constexpr int64_t kSplitKeyWorkgroups = 512;
// Sequences of so many keys on average have blocks of four wavefronts, so that few are left without keys (64 of 100 tokens, 8 heads, forward and gradient: 91 for 101 us)
constexpr int64_t kShortKeys = 128;

KeyPlan key_plan_of(const AttentionSizes &s, int32_t dtype, int64_t channels) {
  const int side = dtype == OCN_FLOAT ? 16 : 32, d = padded_channels(channels);
  KeyPlan p;
  p.waves = dtype != OCN_FLOAT && d > 64 && d <= 128 && s.keys > kShortKeys * s.sequences ? 8 : 4;
  p.units = key_units_of(s, side * p.waves);
  p.splits = 1;
  if (p.units > 0 && s.sequences > 0) {
    // (of the average sequence; the longest may be as long as all)
    const int64_t tiles = s.queries * s.per_kv / (s.sequences * side);
    p.splits = (int)std::max<int64_t>(1, std::min({(int64_t)kWave, kSplitKeyWorkgroups / p.units, tiles / kLeastKeyTiles}));
  }
  return p;
}

// Eight wavefronts, which share keys and values that four would read twice, where that leaves enough workgroups (32 query heads of 128 channels and 8 of keys, bfloat16: 377 for 393 us of
// 8 sequences of 2048 tokens, but 73 for 70 of one), and where sequences are not so short that wavefronts are left without rows (64 of 100 tokens, forward and gradient: 91 for 82 us).
constexpr int64_t kWideUnits = 512, kWideRows = 512;      // (the second: rows of a sequence, on average)
// Parts of many rows' keys, where there are few workgroups (one sequence of 2048 tokens, 4 heads: 32 for 52 us; 100 queries over 8000 keys, 8 heads: 31 for 177).  Two parts save less than
// it takes to join them (3 sequences of 1000 tokens, 8 heads: 43 for 33 us).
constexpr int64_t kSplitRowWorkgroups = 512, kLeastRowSplits = 3;
constexpr int64_t kRowKeys = 64;                 // keys of a tile of theirs (of floats half as many)
// Parts of few rows' keys: workgroups enough for all CUs (a token over 30000 keys, 32 heads, 8 of keys: 37 for 320 us), and more where sequences are so long that parts still have
// kLongTiles tiles on average, as they may be of different lengths (48 of 1 to 8192: 161 for 185 us; 16 of 4000 keys, in 14 parts instead of 3: 57 for 53).
constexpr int64_t kSplitWorkgroups = 512, kMostSplitWorkgroups = 2048, kLongTiles = 32;

static AttentionPlan plan_of(const ocn_tensor *q, const ocn_tensor *k, const ocn_tensor *q_starts) {
  AttentionPlan p;
  const int side = q->dtype == OCN_FLOAT ? 16 : 32;
  const AttentionSizes s = sizes_of(q, k, q_starts);
  p.few = s.sequences == 0 || s.queries * s.per_kv <= side * s.sequences;
  const int d = padded_channels(q->size[q->ndim - 1]);
  const bool many = s.queries * s.per_kv > kWideRows * s.sequences && units_of(s, 8 * side) >= kWideUnits;
  p.waves = p.few ? kFewWaves : q->dtype != OCN_FLOAT && d > 64 && d <= 128 && many ? 8 : 4;
  p.rows = p.few ? side : side * p.waves;
  p.units = units_of(s, p.rows);
  p.splits = 1;
  // (the longest sequence may be as long as all keys, and is not known here)
  const int64_t most = (int64_t)kWave, tiles = (s.keys + side - 1) / side;
  if (p.few && p.units > 0) {
    const int64_t longer = std::min(kMostSplitWorkgroups / p.units, tiles / (s.sequences * kLongTiles));
    p.splits = (int)std::max<int64_t>(1, std::min({most, std::max(kSplitWorkgroups / p.units, longer), tiles / kLeastTiles}));
  }
  if (!p.few && p.units > 0) p.splits = (int)std::min({most, kSplitRowWorkgroups / p.units, tiles * side / (kRowKeys * kLeastRowTiles)});
  if (!p.few && p.splits < kLeastRowSplits) p.splits = 1;
  return p;
}

// of the workspace: what parts of long sequences come to
static size_t part_bytes(const AttentionPlan &p, int32_t dtype, int64_t channels) {
  if (p.splits <= 1) return 0;
  const int64_t d = result_channels(dtype, channels), rows = p.units * p.splits * p.rows;
  return (size_t)(rows * d + rows * 2) * sizeof(float);
}


}  // namespace ocn

using namespace ocn;

extern "C" {

size_t ocn_attention_workspace_bytes(const ocn_tensor *q, const ocn_tensor *k, const ocn_tensor *q_starts) {
  if (check_attention_sizes(q, k, q_starts) != OCN_OK) return 0;
  const AttentionPlan p = plan_of(q, k, q_starts);
  return part_bytes(p, q->dtype, q->size[q->ndim - 1]);
}

int ocn_attention(const ocn_tensor *q, const ocn_tensor *k, const ocn_tensor *v, const ocn_tensor *q_starts, const ocn_tensor *k_starts, double scale,
                  int64_t window, uint32_t flags, const ocn_tensor *out, const ocn_tensor *log_sum, void *workspace, size_t workspace_bytes, void *stream) {
  AttentionArgs a;
  std::memset(&a, 0, sizeof a);
  int rc = fill_attention(a, q, k, v, q_starts, k_starts, scale, window, flags);
  if (rc != OCN_OK) return rc;
  if ((rc = check_like(out, q)) != OCN_OK || (rc = check_sums(log_sum, q)) != OCN_OK) return rc;
  const HeadOperand ops[7] = {{q, false}, {k, false}, {v, false}, {q_starts, false}, {k_starts, false}, {out, true}, {log_sum, true}};
  if ((rc = check_operands(ops, 7)) != OCN_OK) return rc;
  const AttentionPlan p = plan_of(q, k, q_starts);
  const size_t need = part_bytes(p, q->dtype, a.channels);
  if (need) {
    if (!workspace || workspace_bytes < need) return OCN_ERR_WORKSPACE;
    if ((uintptr_t)workspace % 256 != 0) return OCN_ERR_ALIGN;
  }
  if (p.units == 0) return OCN_OK;
  if (!set_blocks(a, sizes_of(q, k, q_starts), p.rows, p.splits)) return OCN_ERR_SHAPE;
  a.out = view_of(out);
  if (log_sum) a.log_sum = view_of(log_sum, false);
  a.rows = p.rows;
  if (p.splits > 1) {
    a.parts = (float *)workspace;
    a.part_sums = a.parts + p.units * p.splits * p.rows * result_channels(q->dtype, a.channels);
  }
  const bool vec = whole_rows(q) && whole_rows(k) && whole_rows(v) && whole_rows(out);
  switch (q->dtype) {
    case OCN_HALF: return run_attention_half(a, p, vec, stream);
    case OCN_BFLOAT16: return run_attention_bfloat16(a, p, vec, stream);
    default: return run_attention_float(a, p, vec, stream);
  }
}

// four numbers of each row, and of a row that is none; the order of blocks of keys; what parts of blocks of keys come to
static size_t grad_bytes(const AttentionSizes &s, int32_t dtype, int64_t channels) {
  const int side = dtype == OCN_FLOAT ? 16 : 32;
  const KeyPlan k = key_plan_of(s, dtype, channels);
  return grad_head_bytes(s, side, k.waves) + (k.splits > 1 ? (size_t)(k.units * k.splits * side * k.waves) * 2 * result_channels(dtype, channels) * sizeof(float) : 0);
}

size_t ocn_attention_grad_workspace_bytes(const ocn_tensor *q, const ocn_tensor *k, const ocn_tensor *q_starts) {
  if (check_attention_sizes(q, k, q_starts) != OCN_OK) return 0;
  const AttentionSizes s = sizes_of(q, k, q_starts);
  return grad_bytes(s, q->dtype, q->size[q->ndim - 1]);
}

int ocn_attention_grad(const ocn_tensor *gout, const ocn_tensor *q, const ocn_tensor *k, const ocn_tensor *v, const ocn_tensor *out, const ocn_tensor *log_sum,
                       const ocn_tensor *q_starts, const ocn_tensor *k_starts, double scale, int64_t window, uint32_t flags, const ocn_tensor *q_gin,
                       const ocn_tensor *k_gin, const ocn_tensor *v_gin, void *workspace, size_t workspace_bytes, void *stream) {
  AttentionArgs a;
  std::memset(&a, 0, sizeof a);
  if (!log_sum || (!k_gin) != (!v_gin)) return OCN_ERR_NULLPTR;
  int rc = fill_attention(a, q, k, v, q_starts, k_starts, scale, window, flags);
  if (rc != OCN_OK) return rc;
  if ((rc = check_like(gout, q)) != OCN_OK || (rc = check_like(out, q)) != OCN_OK || (rc = check_sums(log_sum, q)) != OCN_OK) return rc;
  if ((q_gin && (rc = check_like(q_gin, q)) != OCN_OK) || (k_gin && (rc = check_like(k_gin, k)) != OCN_OK) || (v_gin && (rc = check_like(v_gin, v)) != OCN_OK)) return rc;
  const HeadOperand ops[11] = {{gout, false}, {q, false}, {k, false}, {v, false}, {out, false}, {log_sum, false}, {q_starts, false}, {k_starts, false},
                               {q_gin, true}, {k_gin, true}, {v_gin, true}};
  if ((rc = check_operands(ops, 11)) != OCN_OK) return rc;
  const AttentionSizes s = sizes_of(q, k, q_starts);
  AttentionGrad p;
  p.rows = s.queries * s.kv * s.per_kv;
  p.keys = k_gin != nullptr && s.keys > 0;
  p.queries = q_gin != nullptr && p.rows > 0;
  if (!workspace || workspace_bytes < grad_bytes(s, q->dtype, a.channels)) return OCN_ERR_WORKSPACE;
  if ((uintptr_t)workspace % 256 != 0) return OCN_ERR_ALIGN;
  if (!p.keys && !p.queries) return OCN_OK;
  bool vec = whole_rows(q) && whole_rows(k) && whole_rows(v) && whole_rows(out) && whole_rows(gout);
  a.gout = view_of(gout), a.out = view_of(out), a.log_sum = view_of(log_sum, false);
  if (q_gin) a.gq = view_of(q_gin), vec = vec && whole_rows(q_gin);
  if (k_gin) a.gk = view_of(k_gin), a.gv = view_of(v_gin), vec = vec && whole_rows(k_gin) && whole_rows(v_gin);
  switch (q->dtype) {
    case OCN_HALF: return run_attention_grad_half(a, s, p, vec, workspace, stream);
    case OCN_BFLOAT16: return run_attention_grad_bfloat16(a, s, p, vec, workspace, stream);
    default: return run_attention_grad_float(a, s, p, vec, workspace, stream);
  }
}

}  // extern "C"
