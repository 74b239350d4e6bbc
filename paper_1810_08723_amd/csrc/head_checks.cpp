// Argument checks of the operators over heads, and the frequencies of a rotation.
#include "heads.hpp"

#include <algorithm>
#include <cmath>
#include <cstdlib>

namespace ocn {

int head_type_size(int32_t dtype) {
  switch (dtype) {
    case OCN_HALF: case OCN_BFLOAT16: return 2;
    case OCN_FLOAT: case OCN_INT32: return 4;
    case OCN_INT64: case OCN_DOUBLE: return 8;
    case OCN_UINT8: return 1;
    default: return 0;
  }
}

int check_operand(const ocn_tensor *t, int types) {
  if (!t) return OCN_ERR_NULLPTR;
  const int d = t->dtype;
  const bool ok = ((types & kHeadTypes) && (d == OCN_HALF || d == OCN_BFLOAT16 || d == OCN_FLOAT)) ||
                  ((types & kIndexTypes) && (d == OCN_INT32 || d == OCN_INT64)) || ((types & kDoubleType) && d == OCN_DOUBLE) ||
                  ((types & kByteType) && d == OCN_UINT8) || ((types & kFloatType) && d == OCN_FLOAT);
  if (!ok) return OCN_ERR_DTYPE;
  if (t->ndim < 0 || t->ndim > kMaxDims) return OCN_ERR_NDIM;
  bool empty = false;
  for (int i = 0; i < t->ndim; ++i) {
    if (t->size[i] < 0) return OCN_ERR_SHAPE;
    empty |= t->size[i] == 0;
  }
  if (t->byteswapped && d != OCN_UINT8) return OCN_ERR_BYTEORDER;
  if (!empty && !t->base) return OCN_ERR_NULLPTR;
  const int64_t size = head_type_size(d);
  if (((intptr_t)t->base + t->offset) % size != 0) return OCN_ERR_ALIGN;
  for (int i = 0; i < t->ndim; ++i)
    if (t->size[i] > 1 && t->stride[i] % size != 0) return OCN_ERR_ALIGN;
  return OCN_OK;
}

// sets of dimensions, a bit each
constexpr uint32_t kAllDims = ~0u;

// [lo, hi) of the bytes that dimensions `dims` span, relative to the element at their start
static void span_of(const ocn_tensor *t, uint32_t dims, int64_t *lo, int64_t *hi) {
  int64_t l = 0, h = 0;
  for (int d = 0; d < t->ndim; ++d) {
    if (t->size[d] <= 1 || !(dims >> d & 1)) continue;
    const int64_t s = (t->size[d] - 1) * t->stride[d];
    if (s < 0) l += s; else h += s;
  }
  *lo = l;
  *hi = h + head_type_size(t->dtype);
}

static bool empty_tensor(const ocn_tensor *t) {
  for (int d = 0; d < t->ndim; ++d)
    if (t->size[d] == 0) return true;
  return false;
}

// whether dimensions `dims` of t, taken by stride, each step over everything that lies below them: `extent` bytes at first
static bool steps_over(const ocn_tensor *t, uint32_t dims, int64_t extent) {
  int64_t st[kMaxDims], sz[kMaxDims];
  int m = 0;
  for (int d = 0; d < t->ndim; ++d)
    if (t->size[d] > 1 && (dims >> d & 1)) { st[m] = std::llabs(t->stride[d]); sz[m++] = t->size[d]; }
  for (int i = 1; i < m; ++i)
    for (int j = i; j > 0 && st[j] < st[j - 1]; --j) { std::swap(st[j], st[j - 1]); std::swap(sz[j], sz[j - 1]); }
  for (int i = 0; i < m; ++i) {
    if (st[i] < extent) return false;
    extent += (sz[i] - 1) * st[i];
  }
  return true;
}

bool identical_views(const ocn_tensor *a, const ocn_tensor *b) {
  if ((intptr_t)a->base + a->offset != (intptr_t)b->base + b->offset || a->dtype != b->dtype || a->ndim != b->ndim) return false;
  for (int d = 0; d < a->ndim; ++d)
    if (a->size[d] != b->size[d] || (a->size[d] > 1 && a->stride[d] != b->stride[d])) return false;
  return true;
}

bool share_bytes(const ocn_tensor *a, const ocn_tensor *b) {
  if (empty_tensor(a) || empty_tensor(b)) return false;
  const int64_t pa = (intptr_t)a->base + a->offset, pb = (intptr_t)b->base + b->offset;
  int64_t la, ha, lb, hb;
  span_of(a, kAllDims, &la, &ha);
  span_of(b, kAllDims, &lb, &hb);
  if (pa + ha <= pb + lb || pb + hb <= pa + la) return false;
  // Heads side by side in one buffer, whatever the order of its dimensions.  Where some dimensions, those of the longest strides, take both views through the
  // same steps, each over all that either view has below them, what lies below them need only not meet.
  if (a->ndim != b->ndim) return true;
  uint32_t outer = 0;
  for (;;) {
    int next = -1;
    for (int d = 0; d < a->ndim; ++d)
      if (!(outer >> d & 1) && a->size[d] > 1 && a->size[d] == b->size[d] && a->stride[d] == b->stride[d] &&
          (next < 0 || std::llabs(a->stride[d]) > std::llabs(a->stride[next])))
        next = d;
    if (next < 0) return true;
    outer |= 1u << next;
    span_of(a, ~outer, &la, &ha);
    span_of(b, ~outer, &lb, &hb);
    const bool apart = pa + ha <= pb + lb || pb + hb <= pa + la;
    if (apart && steps_over(a, outer, std::max(pa + ha, pb + hb) - std::min(pa + la, pb + lb))) return false;
  }
}

int check_operands(const HeadOperand *o, int n) {
  for (int i = 0; i < n; ++i) {
    if (!o[i].t) continue;
    for (int j = 0; j < i; ++j)
      if (o[j].t && o[j].t->device != o[i].t->device) return OCN_ERR_DEVICE;
  }
  for (int i = 0; i < n; ++i)
    if (o[i].t && o[i].output && !empty_tensor(o[i].t) && !steps_over(o[i].t, kAllDims, head_type_size(o[i].t->dtype)))
      return OCN_ERR_OVERLAP_OUT;
  for (int i = 0; i < n; ++i)
    for (int j = 0; o[i].t && o[i].output && j < n; ++j) {
      const ocn_tensor *in = o[j].t;
      if (j == i || !in || (o[j].output && j > i)) continue;
      if (!o[j].output && (j == o[i].in_place || j == o[i].in_place_b) && identical_views(in, o[i].t)) continue;
      if (share_bytes(in, o[i].t)) return OCN_ERR_ALIAS;
    }
  return OCN_OK;
}

int merge_lead(const ocn_tensor *x, int inner, const ocn_tensor *const *with, const int *inner_of, int n, Lead *lead,
               int64_t (*strides)[kMaxLead]) {
  const int dims = x->ndim - inner;
  int64_t size[kMaxDims], st[8][kMaxDims], tokens = 1;
  if (dims < 0 || dims > kMaxLead || n > 8) return OCN_ERR_NDIM;
  for (int i = 0; i < n; ++i)
    if (with[i] && with[i]->ndim - inner_of[i] > dims) return OCN_ERR_SHAPE;
  int m = 0;
  for (int d = 0; d < dims; ++d) {
    if (x->size[d] != 0 && tokens > ((int64_t)1 << 31) / x->size[d]) return OCN_ERR_SHAPE;
    tokens *= x->size[d];
    for (int i = 0; i < n; ++i) {
      const int own = with[i] ? with[i]->ndim - inner_of[i] : 0, at = d - (dims - own);
      if (with[i] && at >= 0 && with[i]->size[at] != x->size[d] && with[i]->size[at] != 1) return OCN_ERR_SHAPE;
      st[i][m] = !with[i] || at < 0 || with[i]->size[at] == 1 ? 0 : with[i]->stride[at];
    }
    if (x->size[d] == 1) continue;
    size[m] = x->size[d];
    bool joins = m > 0;
    for (int i = 0; i < n && joins; ++i) joins = st[i][m - 1] == st[i][m] * size[m];
    if (joins) {
      size[m - 1] *= size[m];
      for (int i = 0; i < n; ++i) st[i][m - 1] = st[i][m];
    } else {
      ++m;
    }
  }
  if (tokens >= ((int64_t)1 << 31)) return OCN_ERR_SHAPE;
  if (m == 0) {
    size[0] = 1;
    for (int i = 0; i < n; ++i) st[i][0] = 0;
    m = 1;
  }
  lead->n = m;
  lead->tokens = (uint32_t)tokens;
  for (int d = 0; d < kMaxLead; ++d) {
    lead->div[d] = make_fastdiv(d < m && size[d] > 0 ? (uint32_t)size[d] : 1);
    for (int i = 0; i < n; ++i) strides[i][d] = d < m ? st[i][d] : 0;
  }
  return OCN_OK;
}

int check_cache(const ocn_tensor *cache, int64_t channels, int64_t heads, int64_t *page) {
  const int rc = check_operand(cache, kByteType);
  if (rc != OCN_OK) return rc;
  if (cache->ndim != 3) return OCN_ERR_NDIM;
  if (!cache_channels(channels) || cache->size[1] != heads) return OCN_ERR_SHAPE;
  *page = cache->size[2] * 8 / (9 * channels);
  if (*page < 16 || *page % 16 != 0 || *page > kMaxPage || *page * channels * 9 / 8 != cache->size[2]) return OCN_ERR_SHAPE;
  if (cache->size[0] > ((int64_t)1 << 31)) return OCN_ERR_SHAPE;
  if (cache->stride[2] != 1 || ((intptr_t)cache->base + cache->offset) % 16 != 0) return OCN_ERR_ALIGN;
  for (int d = 0; d < 2; ++d)
    if (cache->size[d] > 1 && cache->stride[d] % 16 != 0) return OCN_ERR_ALIGN;
  return OCN_OK;
}

int check_rotation(const ocn_rotation *r, int64_t channels, int32_t device) {
  if (!r) return OCN_OK;
  int rc = check_operand(r->positions, kIndexTypes);
  if (rc == OCN_OK) rc = check_operand(r->frequencies, kDoubleType);
  if (rc != OCN_OK) return rc;
  if (r->layout != OCN_ROTARY_HALF && r->layout != OCN_ROTARY_INTERLEAVED) return OCN_ERR_OP;
  if (r->rotary_dim < 2 || r->rotary_dim % 2 != 0 || r->rotary_dim > channels) return OCN_ERR_SHAPE;
  const int own = r->frequencies->ndim;
  if ((own != 1 && own != 2) || r->frequencies->size[own - 1] != r->rotary_dim / 2) return OCN_ERR_SHAPE;
  if (own == 2) {      // a row for each axis, and positions on each
    const int64_t axes = r->frequencies->size[0];
    if (axes < 1 || axes > OCN_MAX_AXES || r->positions->ndim < 1 || r->positions->size[0] != axes) return OCN_ERR_SHAPE;
  }
  if (r->positions->device != device || r->frequencies->device != device) return OCN_ERR_DEVICE;
  return OCN_OK;
}

}  // namespace ocn

extern "C" int ocn_rotary_frequencies(int32_t rotary_dim, double base, int stretch, double factor, double original, double low, double high,
                                      double *frequencies, double *magnitude) {
  if (!frequencies || !magnitude) return OCN_ERR_NULLPTR;
  if (stretch < OCN_STRETCH_NONE || stretch > OCN_STRETCH_INDEX) return OCN_ERR_OP;
  if (rotary_dim < 2 || rotary_dim % 2 != 0 || !(base > 1.0) || !std::isfinite(base)) return OCN_ERR_SHAPE;
  if (stretch != OCN_STRETCH_NONE && (!(factor > 0.0) || !std::isfinite(factor))) return OCN_ERR_SHAPE;
  const bool mixed = stretch == OCN_STRETCH_TURNS || stretch == OCN_STRETCH_INDEX;
  if (mixed && (!(original > 0.0) || !std::isfinite(original) || !(low > 0.0) || !(high > low) || !std::isfinite(high))) return OCN_ERR_SHAPE;
  if (stretch == OCN_STRETCH_BASE) {
    if (rotary_dim < 4) return OCN_ERR_SHAPE;
    base *= std::pow(factor, rotary_dim / (rotary_dim - 2.0));
  }
  const double two_pi = 6.283185307179586476925286766559;
  // The index, as a real number, at which a frequency makes so many turns within the original length; rounded outwards (and apart, should
  // their logarithms be one number).  Either may lie the frequencies that there are: then the mixture begins or ends there.
  const auto index_of = [&](double turns) { return rotary_dim * (std::log(original) - std::log(turns) - std::log(two_pi)) / (2.0 * std::log(base)); };
  const double first = mixed ? std::floor(index_of(high)) : 0.0, last = mixed ? std::max(first + 1.0, std::ceil(index_of(low))) : 1.0;
  for (int i = 0; i < rotary_dim / 2; ++i) {
    const double f = std::pow(base, -2.0 * i / rotary_dim);
    double keep = 1.0;    // the share of the frequency as it is, the rest divided by factor
    if (stretch == OCN_STRETCH_LINEAR) keep = 0.0;
    if (stretch == OCN_STRETCH_TURNS) keep = std::min(1.0, std::max(0.0, (original * f / two_pi - low) / (high - low)));
    if (stretch == OCN_STRETCH_INDEX) keep = 1.0 - std::min(1.0, std::max(0.0, (i - first) / (last - first)));
    frequencies[i] = keep == 1.0 ? f : f / factor * (1.0 - keep) + f * keep;
  }
  *magnitude = stretch == OCN_STRETCH_INDEX && factor > 1.0 ? 0.1 * std::log(factor) + 1.0 : 1.0;
  return OCN_OK;
}

extern "C" int ocn_rotary_axes(int32_t axes, const int32_t *pairs, int order, const double *frequencies, double *table) {
  if (!pairs || !frequencies || !table) return OCN_ERR_NULLPTR;
  if (order != OCN_AXES_IN_ROW && order != OCN_AXES_IN_TURN) return OCN_ERR_OP;
  if (axes < 1 || axes > OCN_MAX_AXES) return OCN_ERR_SHAPE;
  int64_t all = 0, left[OCN_MAX_AXES];
  for (int a = 0; a < axes; ++a) {
    if (pairs[a] < 0) return OCN_ERR_SHAPE;
    all += left[a] = pairs[a];
  }
  if (all < 1 || all > OCN_MAX_CHANNELS / 2) return OCN_ERR_SHAPE;
  int at = 0;      // the axis whose turn it is
  for (int64_t i = 0; i < all; ++i) {
    while (left[at] == 0) at = (at + 1) % axes;
    for (int a = 0; a < axes; ++a) table[a * all + i] = a == at ? frequencies[i] : 0.0;
    --left[at];
    if (order == OCN_AXES_IN_TURN) at = (at + 1) % axes;
  }
  return OCN_OK;
}
