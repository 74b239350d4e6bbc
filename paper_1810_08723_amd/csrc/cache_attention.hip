// Attention over the paged cache of 4-bit values.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <type_traits>

#include "dev_types.hpp"
#include "head_types.hpp"
#include "heads.hpp"

namespace ocn {
namespace {

struct AttentionArgs {
  const char *q, *cache, *table, *seen;
  char *out, *log_sum;
  int64_t qb, qt, qh, qe, ob, ot, oh, oe;      // strides of q and out: batch, query, head, channel
  int64_t lb, lt, lh;                          // of log_sum
  int64_t tb, tc, sb, st;                      // of table (batch, column) and visible (batch, query)
  int64_t page_stride, head_stride;
  int64_t pages, window;
  int32_t queries, per_kv;                     // query heads to a head of the cache
  int32_t page, type, table_wide, seen_wide;
  int32_t capacity;                            // tokens that a row of the table has pages for
  int32_t least;                               // tiles of a split, at least
  int32_t whole_q, whole_out;                  // rows are aligned and without gaps
  uint32_t first_item;                         // of this launch
  uint32_t splits;
  FastDiv page_div, per_kv_div, units_div, blocks_div, kv_div;
  float *parts, *part_sums;                    // [items][rows of a unit][channels], [..][2]: maximum and sum
  float scale;                                 // of the scores, times log2(e)
};

constexpr int64_t kLeastTiles = 8;             // of a split: two for each wavefront
constexpr int64_t kAloneTiles = 20;            // up to so many a second launch costs more than splits gain (17 tiles: 10.2 us, 11.4 in splits)
constexpr int64_t kMaxSplits = kWave;          // a lane each when they are joined
constexpr int64_t kAtOnce = 512;               // workgroups that keep all CUs at work, two to each: so many units are not split where memory bounds them
                                               // (512 of 4000 tokens: 62 us, and in three splits)
constexpr int64_t kWorkgroups = 1536;          // fewer units are, into so many: sequences of different lengths even out (256 units of 1 to 8190 tokens: 50 us, 58 in 768;
constexpr int64_t kWorkgroupsWide = 768;       // of 256 channels, which two wavefronts of a SIMD take: 128 units of 100 to 8000 tokens 57.5 us, 58.5 in 1536)
constexpr int64_t kManyWorkgroups = 2048;      // where a workgroup's wavefronts have rows of their own
constexpr int64_t kManyLeast = 16;             // tiles of a table that a split has room for, at least, where units leave CUs without work (352 units of 256 tiles: 711 us in one
                                               // split, 589 in two, 464 in five); of a sequence shorter than its table it has kLeastTiles (32 units of 22 tiles: 30 us in three, 46 in two)
constexpr int64_t kManyLeastFull = 64;         // of either, where they do not (512 units of 47 tiles in a table of 256: 163 us in one split, 173 in four; of 256 tiles 723 and 648)
constexpr uint32_t kJoinRows = 1024;           // from so many on a wavefront joins a row, a workgroup below

// ---------------------------------------------------------------------------------------
// The kernel.  Query heads of one head of the cache, of one or more queries, are the rows of its tiles: 16 a tile.  For 32 tokens at a
// time a wavefront forms scores^T = K Q^T and out^T += V^T P^T with 16x16x32 products in half precision, sums in single:
//
//   scores^T   lane (n = lane % 16, g = lane / 16): row n, tokens 16 a + 4 g + r.  K is the left operand: its lane has token n of
//              a half tile and, of each step's 32 channels, eight; a code's eight channels are a word, and which 32 channels make a step is free as
//              long as Q has the same, so that a lane's words lie together in memory (16 bytes of a row of 128 channels).
//   out^T      row n, channels D/16 (4 g + r) + i of tile i.  The order of the 32 tokens inside a step is free as well: the
//              scores' own order is taken, and no weight crosses lanes between the two products.
//
// A code becomes a half in one conversion for two; times its group's scale it is exact (two bits of the code, nine of the
// scale), so that K and V lose nothing.  V's pairs are two tokens of a channel: nibbles of two rows are put side by side (one shift and one bit
// select for eight codes) before they are converted.  Q is exact where its type has no more than 11 bits: a row is scaled by a power of two so that its
// largest channel is near 2^13; for float tensors it has two parts.  A weight is the sum of two halves, and a second product adds what the first
// leaves (to half alone, 2^-11, bfloat16 results differed from those of single precision in one channel of twenty by a step; 62 us less of 495 for the prompt below).
//
// The maximum of a row that its weights are relative to is raised, and sums rescaled, only where a weight is 2^4 above it; weights are times 2^11, so
// that they stay below 2^15.  The difference of scores is formed before it is scaled: the other way round one subtraction is saved (486 for 493 us of the prompt below), but a score times the scale is
// off by half a step of itself, and from 2^23 on weights were infinite.  The sum of the weights is one more product, with ones.
//
// Two halves hold a weight to 2^-22 of itself, or, where the second is among the smallest that a half holds, to 2^-36 of the largest. Left at that, a channel that is
// zero in the tokens with large weights would lose what the others give it.  A tile with weights below Floor::kLeast
// takes them out and multiplies them apart, times a power of two, in as many steps as they need: down to 2^-122 of the largest no weight is further off than 2^-11 of
// itself (2^-21 for float results).  Below, the factors that sums are rescaled by, 2^4 less at most, leave the range of single precision and are zero.
// ---------------------------------------------------------------------------------------

constexpr float kWeightBits = 11.0f, kRaise = 4.0f;
constexpr int kWeightParts = 2;           // halves that a weight is the sum of
template <class T> constexpr int kQueryParts = sizeof(T) == 4 ? 2 : 1;    // ... and a channel of a query
template <class T> struct Floor {     // (float results keep 2^-21 of a small weight, the others 2^-11)
  static constexpr int kBits = kQueryParts<T> == 1 ? -14 : -4;       // log2 of the smallest weight that is taken as it is
  static constexpr int kStep = 14 - kBits;                    // what smaller ones are multiplied by, and again: below 2^14 then
  static constexpr float kLeast = kQueryParts<T> == 1 ? 0x1p-14f : 0x1p-4f, kUp = kQueryParts<T> == 1 ? 0x1p28f : 0x1p18f, kDown = 1.0f / kUp;
};
constexpr int kTile = 32;            // tokens
constexpr int kAhead = 1;             // tiles on their way (two: 103 for 65 us of two contexts of 100 k and 131 k tokens, for want of registers)

template <int D> struct Shape {
  static constexpr int kWords = D / 32;                   // of a token's codes in a lane; steps of the scores; groups
  static constexpr int kRun = kWords < 4 ? kWords : 4;    // words that lie together
  static constexpr int kChunks = kWords / kRun;
  static constexpr int kTiles = D / 16;                   // of out^T
};

// what a lane holds of a tile's codes and scales, as they come from memory
template <int D> struct Raw {
  uint32_t k[2][Shape<D>::kWords], v[2][Shape<D>::kWords];
  uint32_t k_scale[2][Shape<D>::kChunks];   // (a half in a word of its own: an array of halves would go to memory)
  uint32_t v_scale[2][2];
};

// A half tile's entry in the table, as loaded, and its page: the address of its tokens' codes and scales.  The same in all lanes.
struct Entry {
  uint32_t lo, hi;
  int at;
  bool in;
};
typedef const __attribute__((address_space(1))) char *Global;
struct Place {
  Global codes, scales;
  bool fine;
};

template <int N> __device__ __forceinline__ void load_words(uint32_t *to, Global from) {
  if constexpr (N % 4 == 0) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const u32x4 w = *(const __attribute__((address_space(1))) u32x4 *)(from + 4 * i);
      to[i] = w.x, to[i + 1] = w.y, to[i + 2] = w.z, to[i + 3] = w.w;
    }
  } else {
    const u32x2 w = *(const __attribute__((address_space(1))) u32x2 *)from;
    to[0] = w.x, to[1] = w.y;
  }
}

// the entry of 16 tokens from j on (a multiple of 16); past the sequence's end some other entry, which is not used
__device__ __forceinline__ Entry entry_of(const AttentionArgs &a, const char *row, int j, int end) {
  typedef const __attribute__((address_space(4))) uint32_t *Word;
  Entry e;
  e.in = j < end;
  const uint32_t k = e.in ? (uint32_t)j : 0, column = fast_quotient(k, a.page_div);
  e.at = (int)(k - column * (uint32_t)a.page);
  const char *entry = row + column * a.tc;
  e.lo = *(Word)(uintptr_t)entry;
  e.hi = *(Word)(uintptr_t)(entry + (a.table_wide ? 4 : 0));
  return e;
}
// tokens past the end and in pages outside the cache are read from page 0 and not seen
template <int D> __device__ __forceinline__ Place place_of(const AttentionArgs &a, int64_t head, const Entry &e) {
  const int64_t page = a.table_wide ? (int64_t)((uint64_t)e.hi << 32 | e.lo) : (int64_t)(int32_t)e.lo;
  Place p;
  p.fine = e.in && page >= 0 && page < a.pages;
  const int at = p.fine ? e.at : 0;
  // (said to be the same in all lanes, so that loads take it as a scalar with a lane's 32-bit offset)
  const uint64_t block = (uint64_t)a.cache + (p.fine ? page : 0) * a.page_stride + head;
  const uint64_t same = (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)block) |
                        (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(block >> 32)) << 32;
  p.codes = (Global)same + at * (D / 2);
  p.scales = (Global)same + at * 2;
  return p;
}

struct LaneOffsets { uint32_t k, v, k_scale, k_scale_step, v_scale; };

template <int D> __device__ __forceinline__ LaneOffsets lane_offsets(const AttentionArgs &a, int n, int g) {
  typedef Shape<D> S;
  LaneOffsets o;
  o.k = n * (D / 2) + g * (4 * S::kRun);
  o.v = a.page * (D / 2) + (g * 16 + n) * (D / 8);
  o.k_scale = a.page * D + 2 * ((S::kRun * g / 4) * a.page + n);
  o.k_scale_step = 2 * S::kRun * a.page;
  o.v_scale = a.page * D + 2 * ((S::kWords + S::kWords * n / 16) * a.page + 4 * g);
  return o;
}

template <int D> __device__ __forceinline__ void load_half(Raw<D> &r, int x, const Place &p, const LaneOffsets &o) {
  typedef Shape<D> S;
#pragma unroll
  for (int h = 0; h < S::kChunks; ++h) {
    load_words<S::kRun>(&r.k[x][h * S::kRun], p.codes + (o.k + h * 16 * S::kRun));
    r.k_scale[x][h] = *(const __attribute__((address_space(1))) uint16_t *)(p.scales + (o.k_scale + h * o.k_scale_step));
  }
  load_words<S::kWords>(r.v[x], p.codes + o.v);
  load_words<2>(r.v_scale[x], p.scales + o.v_scale);
}

template <int BYTE> __device__ __forceinline__ f16x2 two_codes(uint32_t w) { return __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 2.0f, BYTE); }

union Frag {
  f16x8 v;
  f16x2 p[4];
  uint32_t u[4];
};

// Weights 2 i and 2 i + 1 of eight as sums of two halves each.  (What the first leaves is one instruction a weight, which reads it as a half: the factor
// is hidden, or the compiler converts it back and subtracts.)
typedef float f32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void in_parts(Frag *p, int i, float w0, float w1) {
  p[0].p[i] = __builtin_convertvector((f32x2{w0, w1}), f16x2);
  asm("" : "+v"(p[0].u[i]));      // (or each is converted by itself once more)
  const f16x2 h = p[0].p[i];
  float minus = -1.0f;
  asm("" : "+s"(minus));
  p[1].p[i] = __builtin_convertvector((f32x2{__builtin_fmaf((float)h.x, minus, w0), __builtin_fmaf((float)h.y, minus, w1)}), f16x2);
}

// bits of a where the mask has ones, of b elsewhere
__device__ __forceinline__ uint32_t select_bits(uint32_t mask, uint32_t a, uint32_t b) { return (a & mask) | (b & ~mask); }

// The codes of a lane's tokens 2 i and 2 i + 1 side by side: byte k of even[q] (odd[q]) has both tokens' codes of channel 2 k (2 k + 1) of word q
template <int D> struct Twins { uint32_t even[D / 128 ? D / 128 : 1], odd[D / 128 ? D / 128 : 1]; };
template <int D> __device__ __forceinline__ Twins<D> twins_of(const uint32_t *v, int i) {
  constexpr uint32_t low = 0x0f0f0f0fu;
  Twins<D> w;
  if constexpr (D == 64) {
    w.even[0] = select_bits(low, v[i], v[i] >> 12);
    w.odd[0] = select_bits(low, v[i] >> 4, v[i] >> 16);
  } else {
#pragma unroll
    for (int q = 0; q < D / 128; ++q) {
      const uint32_t a = v[2 * i * (D / 128) + q], b = v[(2 * i + 1) * (D / 128) + q];
      w.even[q] = select_bits(low, a, b << 4);
      w.odd[q] = select_bits(low, a >> 4, b);
    }
  }
  return w;
}
// channel t of a lane's, of both tokens
template <int D> __device__ __forceinline__ f16x2 twin_codes(const Twins<D> &w, int t) {
  const uint32_t x = t % 2 ? w.odd[t / 8] : w.even[t / 8];
  switch (t % 8 / 2) {       // (t is known when this is compiled)
    case 0: return two_codes<0>(x);
    case 1: return two_codes<1>(x);
    case 2: return two_codes<2>(x);
    default: return two_codes<3>(x);
  }
}

// (the compiler's own maximum first quiets NaNs that it cannot rule out: two instructions more)
__device__ __forceinline__ float larger(float a, float b) {
  float c;
  asm("v_max_f32 %0, %1, %2" : "=v"(c) : "v"(a), "v"(b));
  return c;
}
// The largest and smallest of a lane's eight scores; NaNs are passed over.  (No assembly here: the compiler keeps a reader of a product's result
// waiting, assembly it does not.)
__device__ __forceinline__ float largest(const f32x4 *s) {
  float m = s[0][0];
#pragma unroll
  for (int i = 1; i < 8; ++i) m = fmaxf(m, s[i / 4][i % 4]);
  return m;
}
__device__ __forceinline__ float smallest(const f32x4 *s) {
  float m = s[0][0];
#pragma unroll
  for (int i = 1; i < 8; ++i) m = fminf(m, s[i / 4][i % 4]);
  return m;
}
// the largest of the four lanes that hold a row
__device__ __forceinline__ float row_max(float x) {
  const auto a = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
  const uint32_t a0 = a[0], a1 = a[1];
  x = larger(__builtin_bit_cast(float, a0), __builtin_bit_cast(float, a1));
  const auto b = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
  const uint32_t b0 = b[0], b1 = b[1];
  return larger(__builtin_bit_cast(float, b0), __builtin_bit_cast(float, b1));
}

// the largest of sixteen lanes, which the four lanes of a row repeat: of all rows
__device__ __forceinline__ int rows_max(int x) {
  x = max(x, __builtin_amdgcn_update_dpp(x, x, 0x128, 0xf, 0xf, false));    // (rotations by 8, 4, 2 and 1 lanes)
  x = max(x, __builtin_amdgcn_update_dpp(x, x, 0x124, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(x, x, 0x122, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(x, x, 0x121, 0xf, 0xf, false));
  return __builtin_amdgcn_readfirstlane(x);
}

__device__ __forceinline__ f32x4 product(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

// Sums of one wavefront's rows: row n of lane (n, g)
template <int D, int RT> struct Sums {
  f32x4 out[RT][Shape<D>::kTiles];   // out^T
  f32x4 total[RT];                   // of the weights (all four the same)
  f32x4 bad[RT];                     // how many tokens with a NaN as V's scale a row sees, in tiles that are not seen whole
  float best[RT];                    // a weight is 2^((score - best) * scale + kWeightBits); minus infinity before the first
};

template <int D, int RT, class T> struct Rows {
  f16x8 q[RT][kQueryParts<T>][Shape<D>::kWords];
  float scale[RT];                   // of a score
  int lo[RT], hi[RT];                // tokens that a row sees
};

// Scales of V that are NaN (or none that appending writes: places that were never written) count as zero in a tile that some row does not see whole,
// because weights of zero would not make a NaN go away; `bad` marks their tokens.
__device__ __forceinline__ Frag fix_scales(uint32_t (*v_scale)[2]) {
  Frag bad;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t two = v_scale[i / 2][i % 2];
    f16x2 sc = __builtin_bit_cast(f16x2, two), no = {0, 0};
#pragma unroll
    for (int e = 0; e < 2; ++e)
      if (!(sc[e] <= (f16)5456.0f && sc[e] >= (f16)-5456.0f)) { sc[e] = (f16)0.0f; no[e] = (f16)1.0f; }
    v_scale[i / 2][i % 2] = __builtin_bit_cast(uint32_t, sc);
    bad.p[i] = no;
  }
  return bad;
}

// Where a tile's operands come from: a wavefront's own registers ...
template <int D> struct FromRegisters {
  typedef Shape<D> S;
  Raw<D> &raw;
  Twins<D> twins[4];
  f16x2 scale[4];
  __device__ __forceinline__ f16x8 k(int x, int w) const {
    const uint32_t codes = raw.k[x][w], both = raw.k_scale[x][w / S::kRun];
    const f16x2 one = __builtin_bit_cast(f16x2, both), s = {one.x, one.x};
    Frag f;
    f.p[0] = two_codes<0>(codes) * s, f.p[1] = two_codes<1>(codes) * s;
    f.p[2] = two_codes<2>(codes) * s, f.p[3] = two_codes<3>(codes) * s;
    return f.v;
  }
  __device__ __forceinline__ f16x8 bad() { return fix_scales(raw.v_scale).v; }
  __device__ __forceinline__ void early() const {}
  __device__ __forceinline__ void start_v() {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      twins[i] = twins_of<D>(raw.v[i / 2], i % 2);
      const uint32_t two = raw.v_scale[i / 2][i % 2];
      scale[i] = __builtin_bit_cast(f16x2, two);
    }
  }
  __device__ __forceinline__ f16x8 v(int t) const {
    Frag f;
#pragma unroll
    for (int i = 0; i < 4; ++i) f.p[i] = twin_codes<D>(twins[i], t) * scale[i];
    return f.v;
  }
};

// ... or LDS, where a workgroup's wavefronts have put them: K [half tile][word], V [channel of a lane], the tokens with bad scales; 16 bytes of each lane
template <int D, int EARLY> struct FromLds {
  typedef Shape<D> S;
  const f16x8 *at;         // of this lane
  __device__ __forceinline__ f16x8 k(int x, int w) const { return at[(x * S::kWords + w) * kWave]; }
  f16x8 first[EARLY];     // V's, read before the weights are formed (the compiler moves no read over their branches): one before 693 us, six 646 (the prompt below, in one split)
  __device__ __forceinline__ f16x8 v(int t) const { return t < EARLY ? first[t] : at[(2 * S::kWords + t) * kWave]; }
  __device__ __forceinline__ f16x8 bad() const { return at[(2 * S::kWords + S::kTiles) * kWave]; }
  __device__ __forceinline__ void start_v() const {}
  __device__ __forceinline__ void early() {
#pragma unroll
    for (int t = 0; t < EARLY; ++t) first[t] = at[(2 * S::kWords + t) * kWave];
  }
};

// whole: every row sees every token of the tile
template <int D, int RT, class T, class Source>
__device__ __forceinline__ void one_tile(Sums<D, RT> &s, const Rows<D, RT, T> &rows, Source &source, int g, int j0, bool whole, bool fine0, bool fine1) {
  typedef Shape<D> S;
  typedef Floor<T> F;
  const f16x8 ones = {1, 1, 1, 1, 1, 1, 1, 1};
  f32x4 score[RT][2];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt)
#pragma unroll
    for (int x = 0; x < 2; ++x) score[rt][x] = f32x4{0, 0, 0, 0};
#pragma unroll
  for (int w = 0; w < S::kWords; ++w)
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const f16x8 k = source.k(x, w);
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int part = 0; part < kQueryParts<T>; ++part) score[rt][x] = product(k, rows.q[rt][part][w], score[rt][x]);
    }
  source.early();
  float least[RT];       // (unseen places may make it too small, and the tile takes longer)
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    least[rt] = smallest(score[rt]);
    asm volatile("" : "+v"(least[rt]));      // (here: put off to where it is used, it would keep a second copy of the scores)
  }
  uint32_t sees[RT];     // which of its eight tokens a lane's row sees
  if (!whole) {
    const f16x8 bad = source.bad();     // rows that see such tokens are marked by one more product
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      Frag seen;
      sees[rt] = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int j = j0 + 16 * (i / 4) + 4 * g + i % 4;
        const bool in = j >= rows.lo[rt] && j < rows.hi[rt] && (i < 4 ? fine0 : fine1);
        seen.v[i] = in ? (f16)1.0f : (f16)0.0f;
        sees[rt] |= in ? 1u << i : 0u;
        if (!in) score[rt][i / 4][i % 4] = -__builtin_inff();
      }
      s.bad[rt] = product(bad, seen.v, s.bad[rt]);
    }
  }
  Frag p[RT][kWeightParts];
  float weight[RT][8];
  bool apart = false;    // whether some weights are below the floor
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const float most = largest(score[rt]);
    if (__builtin_amdgcn_ballot_w64((most - s.best[rt]) * rows.scale[rt] > kRaise)) {
      // (the four lanes of a row meet here alone: most tiles do not come here)
      const float before = s.best[rt], now = fmaxf(before, row_max(most));
      const float keep = now == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f((before - now) * rows.scale[rt]);
      s.best[rt] = now;
#pragma unroll
      for (int i = 0; i < S::kTiles; ++i) s.out[rt][i] *= keep;
      s.total[rt] *= keep;
    }
    // (the difference first: a score times the scale, less its largest, is off by as much as the score's steps, and past 2^23 that is more than a half's range)
    const float best = s.best[rt];
#pragma unroll
    for (int i = 0; i < 8; ++i) weight[rt][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(score[rt][i / 4][i % 4] - best, rows.scale[rt], kWeightBits));
    if (!whole) {
#pragma unroll
      for (int i = 0; i < 8; ++i) weight[rt][i] = sees[rt] >> i & 1 ? weight[rt][i] : 0.0f;
    }
    if (__builtin_amdgcn_ballot_w64(__builtin_fmaf(least[rt] - best, rows.scale[rt], kWeightBits) < F::kBits)) apart = true;
  }
  source.start_v();
  if (apart) {
    float small[RT][8], down = F::kDown;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        small[rt][i] = weight[rt][i] < F::kLeast ? weight[rt][i] : 0.0f;
        weight[rt][i] = weight[rt][i] < F::kLeast ? 0.0f : weight[rt][i];
      }
#pragma nounroll
    for (int step = 0; step < (126 + F::kStep - 1) / F::kStep; ++step, down *= F::kDown) {
      bool left = false, any = false;
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        float two[2];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float x = small[rt][i] * F::kUp, w = x < F::kLeast ? 0.0f : x;
          small[rt][i] = x < F::kLeast ? x : 0.0f;
          any |= w > 0.0f;
          left |= small[rt][i] > 0.0f;
          two[i % 2] = w;
          if constexpr (kQueryParts<T> == 2) {      // (a weight at a time: pairs take four registers more than there are)
            p[rt][0].v[i] = (f16)w;
            p[rt][1].v[i] = (f16)(w - (float)p[rt][0].v[i]);
          } else if (i % 2) {
            in_parts(p[rt], i / 2, two[0], two[1]);
          }
        }
      }
      if (__builtin_amdgcn_ballot_w64(any)) {
#pragma unroll
        for (int t = 0; t < S::kTiles; ++t) {
          const f16x8 f = source.v(t);
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) {
            f32x4 add = {0, 0, 0, 0};
#pragma unroll
            for (int part = 0; part < kWeightParts; ++part) add = product(f, p[rt][part].v, add);
            s.out[rt][t] += add * down;
            if (t == 0) {
              add = f32x4{0, 0, 0, 0};
#pragma unroll
              for (int part = 0; part < kWeightParts; ++part) add = product(ones, p[rt][part].v, add);
              s.total[rt] += add * down;
            }
          }
        }
      }
      if (!__builtin_amdgcn_ballot_w64(left)) break;
    }
  }
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
    for (int i = 0; i < 4; ++i) in_parts(p[rt], i, weight[rt][2 * i], weight[rt][2 * i + 1]);
#pragma unroll
    for (int part = 0; part < kWeightParts; ++part) s.total[rt] = product(ones, p[rt][part].v, s.total[rt]);
  }
#pragma unroll
  for (int t = 0; t < S::kTiles; ++t) {
    const f16x8 f = source.v(t);
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
      for (int part = 0; part < kWeightParts; ++part) s.out[rt][t] = product(f, p[rt][part].v, s.out[rt][t]);
  }
}

// N channels of a row to memory
template <class T, int N> __device__ __forceinline__ void store_row(const AttentionArgs &a, char *row, int channel, const float *v) {
  if (a.whole_out) {
    typedef T Four __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int i = 0; i < N; i += 4) *(Four *)(row + (channel + i) * (int)sizeof(T)) = Four{(T)v[i], (T)v[i + 1], (T)v[i + 2], (T)v[i + 3]};
  } else {
    int64_t step = a.oe;
    asm volatile("" : "+s"(step)::"memory");
#pragma unroll
    for (int i = 0; i < N; ++i) *(T *)(row + (channel + i) * step) = (T)v[i];
  }
}

__device__ __forceinline__ float log_of(float top, float total) { return total == 0.0f ? -__builtin_inff() : 0.69314718f * (top - kWeightBits + __builtin_log2f(total)); }

// eight channels of a query, as they are in memory
template <class T> __device__ __forceinline__ void load_channels(uint32_t *to, const char *row, int channel, bool any, const AttentionArgs &a) {
  constexpr int N = 2 * (int)sizeof(T);
#pragma unroll
  for (int i = 0; i < N; ++i) to[i] = 0;
  if (!any) return;
  if (a.whole_q) {
#pragma unroll
    for (int i = 0; i < N; i += 4) load_words<4>(to + i, (Global)(uint64_t)(row + channel * (int)sizeof(T) + 4 * i));
  } else {
    int64_t step = a.qe;
    asm volatile("" : "+s"(step)::"memory");   // (here and now: hoisted out of all loops, the addresses took more registers than the tiles)
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if constexpr (sizeof(T) == 4) to[i] = *(const uint32_t *)(row + (channel + i) * step);
      else to[i] = *(const uint16_t *)(row + (channel + 2 * i) * step) | (uint32_t)*(const uint16_t *)(row + (channel + 2 * i + 1) * step) << 16;
    }
  }
}
template <class T> __device__ __forceinline__ void channels_of(float *x, const uint32_t *from) {
#pragma unroll
  for (int i = 0; i < 2 * (int)sizeof(T); ++i) {
    if constexpr (sizeof(T) == 4) {
      x[i] = __builtin_bit_cast(float, from[i]);
    } else if constexpr (std::is_same_v<T, bf16>) {
      x[2 * i] = __builtin_bit_cast(float, from[i] << 16);
      x[2 * i + 1] = __builtin_bit_cast(float, from[i] & 0xffff0000u);
    } else {
      const f16x2 h = __builtin_bit_cast(f16x2, from[i]);
      x[2 * i] = (float)h.x, x[2 * i + 1] = (float)h.y;
    }
  }
}

// what an item's rows see: the tokens of a row, and the ends of all of them
struct Reach { int hi_most, hi_least, lo_least, lo_most; };

template <int D, int RT, class T>
__device__ __forceinline__ Reach reach_of(const AttentionArgs &a, Rows<D, RT, T> &rows, int b, int first_row, int all_rows, int n) {
  Reach r = {0, 0x7fffffff, 0x7fffffff, 0};
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int row = first_row + rt * 16 + n;
    rows.lo[rt] = 0;
    rows.hi[rt] = 0x7fffffff;
    if (row < all_rows) {
      const int64_t seen = load_index(a.seen + b * a.sb + fast_quotient((uint32_t)row, a.per_kv_div) * a.st, a.seen_wide);
      rows.hi[rt] = (int)max((int64_t)0, min(seen, (int64_t)a.capacity));
      rows.lo[rt] = a.window > 0 ? (int)max((int64_t)0, rows.hi[rt] - a.window) : 0;
      r.hi_most = max(r.hi_most, rows.hi[rt]);
      r.hi_least = min(r.hi_least, rows.hi[rt]);
      r.lo_most = max(r.lo_most, rows.lo[rt]);
      if (rows.hi[rt] > 0) r.lo_least = min(r.lo_least, rows.lo[rt]);
    }
  }
  r.hi_most = rows_max(r.hi_most);
  r.hi_least = -rows_max(-r.hi_least);
  r.lo_most = rows_max(r.lo_most);
  r.lo_least = -rows_max(-r.lo_least);
  return r;
}

// a split's tiles [from, stop): all of [lo_least, hi_most) in equal parts, none of fewer than a.least tiles
struct Part { int64_t from; int stop, end; };
__device__ __forceinline__ Part part_of(const AttentionArgs &a, const Reach &r, uint32_t split) {
  const int begin = r.hi_most > 0 ? r.lo_least / kTile : 0;
  Part p;
  p.end = (int)(((int64_t)r.hi_most + kTile - 1) / kTile);
  const int each = max(a.least, (int)((p.end - begin + a.splits - 1) / a.splits));
  p.from = begin + (int64_t)split * each;
  p.stop = (int)min((int64_t)p.end, p.from + each);
  return p;
}

// queries as operands, and sums at their start
template <int D, int RT, class T>
__device__ __forceinline__ void start_rows(const AttentionArgs &a, Rows<D, RT, T> &rows, Sums<D, RT> &sums, int b, int kv, int first_row, int all_rows, int n, int g) {
  typedef Shape<D> S;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int row = first_row + rt * 16 + n, t = row < all_rows ? (int)fast_quotient((uint32_t)row, a.per_kv_div) : 0;
    uint32_t q[S::kWords][2 * sizeof(T)];       // as they are in memory: two 16-bit channels, or a float, in a word
    float most = 0.0f;
    const char *from_row = a.q + b * a.qb + t * a.qt + (int64_t)(kv * a.per_kv + row - t * a.per_kv) * a.qh;
#pragma unroll
    for (int w = 0; w < S::kWords; ++w) {
      const int channel = 8 * (w / S::kRun * 4 * S::kRun + S::kRun * g + w % S::kRun);
      load_channels<T>(q[w], from_row, channel, row < all_rows, a);
      float x[8];
      channels_of<T>(x, q[w]);
#pragma unroll
      for (int i = 0; i < 8; ++i) most = fmaxf(most, __builtin_fabsf(x[i]));
    }
    most = row_max(most);
    const int up = most > 0.0f ? 13 - (int)((__builtin_bit_cast(uint32_t, most) >> 23) & 255) + 127 : 0;
    // (not zero, so that minus infinity stays what it is; a negative scale turns the queries)
    rows.scale[rt] = fmaxf(__builtin_amdgcn_ldexpf(__builtin_fabsf(a.scale), -up), 0x1p-126f);
    const float sign = a.scale < 0.0f ? -1.0f : 1.0f;
#pragma unroll
    for (int w = 0; w < S::kWords; ++w) {
      float x[8];
      channels_of<T>(x, q[w]);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[i] = __builtin_amdgcn_ldexpf(x[i], up) * sign;
        rows.q[rt][0][w][i] = (f16)x[i];
        if constexpr (kQueryParts<T> == 2) rows.q[rt][1][w][i] = (f16)(x[i] - (float)rows.q[rt][0][w][i]);
      }
    }
#pragma unroll
    for (int i = 0; i < S::kTiles; ++i) sums.out[rt][i] = f32x4{0, 0, 0, 0};
    sums.total[rt] = sums.bad[rt] = f32x4{0, 0, 0, 0};
    sums.best[rt] = -__builtin_inff();
  }
}

template <int D, int RT> __device__ __forceinline__ void mark_bad(Sums<D, RT> &sums) {
#pragma unroll
  for (int rt = 0; rt < RT; ++rt)
#pragma unroll
    for (int i = 0; i < Shape<D>::kTiles; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (sums.bad[rt][r] > 0.0f) sums.out[rt][i][r] = __builtin_nanf("");
}

// a workgroup's place: items are blocks of rows fastest, then heads of the cache, sequences, and splits.  (Workgroups go to the XCDs in turn, and where
// sequences are of different lengths the later splits are empty: with splits fastest some XCDs had most of the work.)
struct Work { uint32_t item, split, block; int b, kv; };
__device__ __forceinline__ Work work_of(const AttentionArgs &a, uint32_t item) {
  Work w;
  w.item = item;
  w.split = fast_quotient(item, a.units_div);
  const uint32_t unit = item - w.split * a.units_div.d, bh = fast_quotient(unit, a.blocks_div);
  w.block = unit - bh * a.blocks_div.d;
  w.b = (int)fast_quotient(bh, a.kv_div);
  w.kv = (int)bh - w.b * (int)a.kv_div.d;
  return w;
}

// Wavefronts of a SIMD: what registers allow (of 256 channels five spill, which whole tiles do not touch; one wavefront instead takes 65.9 us for 57.5 of 128 units of 100 to 8000 tokens).
// Three for 128 channels: 49.7 us for 54.7 of 256 units of 1 to 8190 tokens.
template <int D, int RT, class T> constexpr int kWavesOfSimd = kQueryParts<T> == 1 && D == 128 && RT == 1 ? 3 : D * RT <= (kQueryParts<T> == 1 ? 256 : 128) ? 2 : 1;

// Few rows: a workgroup's four wavefronts have the same rows and every fourth tile each, and join their sums in LDS.  Memory bounds this; what a
// wavefront needs of a tile goes from memory to its registers, 4-bit codes, and becomes halves there.  64 sequences of 4000 tokens, 8 heads of 128 channels, 4 query
// heads each (295 MB): 62.6 us, 4.7 TB/s, where a large copy has 5.2.
template <int D, int RT, class T>
__global__ __launch_bounds__(kBlock, (kWavesOfSimd<D, RT, T>)) void attention_kernel(const AttentionArgs a) {
  typedef Shape<D> S;
  constexpr int W = kBlock / kWave, kPart = S::kTiles < 8 ? S::kTiles : 8;
  constexpr int kRows = 16 * RT;             // of a unit
  __shared__ float part[W][16][16][kPart];
  __shared__ float tops[W][RT][16], totals[W][RT][16];
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), n = lane % 16, g = lane / 16;
  const LaneOffsets lanes = lane_offsets<D>(a, n, g);
  warm_arguments<AttentionArgs>();
  const Work work = work_of(a, a.first_item + blockIdx.x);
  const int b = work.b, kv = work.kv, first_row = (int)work.block * kRows, all_rows = a.queries * a.per_kv;
  Rows<D, RT, T> rows;
  const Reach reach = reach_of<D, RT, T>(a, rows, b, first_row, all_rows, n);
  const Part range = part_of(a, reach, work.split);
  if (a.splits > 1 && range.from >= range.end) {      // nothing left for this split
    if (threadIdx.x < kRows) *(float2 *)(a.part_sums + ((int64_t)work.item * kRows + threadIdx.x) * 2) = float2{-__builtin_inff(), 0.0f};
    return;
  }
  Sums<D, RT> sums;
  start_rows<D, RT, T>(a, rows, sums, b, kv, first_row, all_rows, n, g);
  const char *table = a.table + b * a.tb;
  const int64_t head = kv * a.head_stride, start = range.from + wave;
  const int stop = range.stop;
  if (start < stop) {
    // kAhead tiles are on their way while one is worked on, and the entries of one more: loads are issued whether or not there are tiles left,
    // so that every wait is for a known number of them (past the end they go to the sequence's first entry's page, or page 0).
    Raw<D> raw[kAhead + 1];
    uint32_t fine = 0;            // two bits for each buffer: whether its half tiles' pages are
    Entry e0, e1;
    const auto entries = [&](int64_t tile) {
      const int j = tile < stop ? (int)tile * kTile : reach.hi_most;       // (16 more stay below 2^31: a table has pages for 64 tokens fewer)
      e0 = entry_of(a, table, j, reach.hi_most);
      e1 = entry_of(a, table, j + 16, reach.hi_most);
    };
    const auto load = [&](Raw<D> &to, int buffer) {
      const Place p0 = place_of<D>(a, head, e0), p1 = place_of<D>(a, head, e1);
      fine = (fine & ~(3u << 2 * buffer)) | (p0.fine ? 1u : 0u) << 2 * buffer | (p1.fine ? 2u : 0u) << 2 * buffer;
      load_half<D>(to, 0, p0, lanes);
      load_half<D>(to, 1, p1, lanes);
    };
    entries(start);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      load(raw[i], i);
      entries(start + (i + 1) * W);
    }
    for (int64_t t = start; t < stop;) {
#pragma unroll
      for (int i = 0; i <= kAhead; ++i) {
        load(raw[(i + kAhead) % (kAhead + 1)], (i + kAhead) % (kAhead + 1));
        entries(t + (kAhead + 1) * W);
        const int j0 = (int)t * kTile;
        const uint32_t mine = fine >> 2 * i & 3;
        FromRegisters<D> source = {raw[i]};
        one_tile<D, RT, T>(sums, rows, source, g, j0, mine == 3 && j0 >= reach.lo_most && j0 + kTile <= reach.hi_least, (mine & 1) != 0,
                                          (mine & 2) != 0);
        t += W;
        if (t >= stop) break;
      }
    }
  }
  mark_bad<D, RT>(sums);
  const bool whole = a.splits == 1;
  // the wavefronts' sums, relative to the largest of their maxima
  if (g == 0) {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      tops[wave][rt][n] = sums.best[rt] * rows.scale[rt];
      totals[wave][rt][n] = sums.total[rt][0];
    }
  }
  __syncthreads();
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    float top = -__builtin_inff();
#pragma unroll
    for (int w = 0; w < W; ++w) top = fmaxf(top, tops[w][rt][n]);
    const float keep = top == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f(sums.best[rt] * rows.scale[rt] - top);
#pragma unroll
    for (int at = 0; at < S::kTiles; at += kPart) {
      if (rt + at > 0) __syncthreads();
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int i = 0; i < kPart; ++i) part[wave][n][4 * g + r][i] = sums.out[rt][at + i][r] * keep;
      __syncthreads();
      // a thread has D/16 (eight at a time) channels of a row now
      const int rn = threadIdx.x / 16, rj = threadIdx.x % 16, row = first_row + rt * 16 + rn;
      float v[kPart], most = -__builtin_inff(), total = 0.0f;
#pragma unroll
      for (int i = 0; i < kPart; ++i) v[i] = 0.0f;
#pragma unroll
      for (int w = 0; w < W; ++w) most = fmaxf(most, tops[w][rt][rn]);
#pragma unroll
      for (int w = 0; w < W; ++w) {
        total += most == -__builtin_inff() ? totals[w][rt][rn] : totals[w][rt][rn] * __builtin_amdgcn_exp2f(tops[w][rt][rn] - most);
#pragma unroll
        for (int i = 0; i < kPart; ++i) v[i] += part[w][rn][rj][i];
      }
      if (row >= all_rows) continue;
      const int channel = rj * S::kTiles + at;
      if (whole) {
        const int t = (int)fast_quotient((uint32_t)row, a.per_kv_div), h = kv * a.per_kv + row - t * a.per_kv;
        const float over = total == 0.0f ? 0.0f : 1.0f / total;
#pragma unroll
        for (int i = 0; i < kPart; ++i) v[i] = total == 0.0f ? 0.0f : v[i] * over;
        store_row<T, kPart>(a, a.out + b * a.ob + t * a.ot + h * a.oh, channel, v);
        if (a.log_sum && rj == 0 && at == 0) *(float *)(a.log_sum + b * a.lb + t * a.lt + h * a.lh) = log_of(most, total);
      } else {
        const int64_t at_row = (int64_t)work.item * kRows + rt * 16 + rn;
        float *to = a.parts + at_row * D + channel;
#pragma unroll
        for (int i = 0; i < kPart; i += 4) *(f32x4 *)(to + i) = f32x4{v[i], v[i + 1], v[i + 2], v[i + 3]};
        if (rj == 0 && at == 0) *(float2 *)(a.part_sums + at_row * 2) = float2{most, total};
      }
    }
  }
}

// Many rows: each of a workgroup's wavefronts has rows of its own, and all go over the same tiles.  Products bound this, and what is done to the codes before
// them: each wavefront makes a quarter of a tile's operands, for all four, in LDS; two tiles have room there, so that one is made while the other is used.  1024 queries of 32 heads over 3333 and 8192 tokens:
// 493 us, 358 TFLOP/s of the 1390 that a large product reaches: a wavefront has nothing else to do between its two products, and registers allow two to a SIMD.
template <int D, int RT, class T>
__global__ __launch_bounds__(kBlock, 2) void attention_many_kernel(const AttentionArgs a) {
  typedef Shape<D> S;
  constexpr int kEarly = kQueryParts<T> == 2 ? 1 : D == 128 ? 6 : 4;          // what the registers have room for
  constexpr int W = kBlock / kWave, kRows = 16 * RT * W, kFrags = 2 * S::kWords + S::kTiles + 1;
  constexpr int kMyK = 2 * S::kWords / W, kMyV = S::kTiles / W;        // operands that a wavefront makes
  __shared__ f16x8 operands[2][kFrags * kWave];
  __shared__ Reach reaches[W];
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), n = lane % 16, g = lane / 16;
  const LaneOffsets lanes = lane_offsets<D>(a, n, g);
  warm_arguments<AttentionArgs>();
  const Work work = work_of(a, a.first_item + blockIdx.x);
  const int b = work.b, kv = work.kv, first_row = (int)work.block * kRows + wave * 16 * RT, all_rows = a.queries * a.per_kv;
  Rows<D, RT, T> rows;
  Reach reach = reach_of<D, RT, T>(a, rows, b, first_row, all_rows, n);
  if (lane == 0) reaches[wave] = reach;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < W; ++w) {
    reach.hi_most = max(reach.hi_most, reaches[w].hi_most);
    reach.hi_least = min(reach.hi_least, reaches[w].hi_least);
    reach.lo_least = min(reach.lo_least, reaches[w].lo_least);
    reach.lo_most = max(reach.lo_most, reaches[w].lo_most);
  }
  reach.hi_most = __builtin_amdgcn_readfirstlane(reach.hi_most);
  reach.hi_least = __builtin_amdgcn_readfirstlane(reach.hi_least);
  reach.lo_least = __builtin_amdgcn_readfirstlane(reach.lo_least);
  reach.lo_most = __builtin_amdgcn_readfirstlane(reach.lo_most);
  const Part range = part_of(a, reach, work.split);
  if (a.splits > 1 && range.from >= range.end) {      // nothing left for this split
    for (int i = threadIdx.x; i < kRows; i += kBlock) *(float2 *)(a.part_sums + ((int64_t)work.item * kRows + i) * 2) = float2{-__builtin_inff(), 0.0f};
    return;
  }
  Sums<D, RT> sums;
  start_rows<D, RT, T>(a, rows, sums, b, kv, first_row, all_rows, n, g);
  const char *table = a.table + b * a.tb;
  const int64_t head = kv * a.head_stride;
  const int start = (int)range.from, stop = range.stop;
  if (start < stop) {
    // A wavefront's share: words wave, wave + 4 ... of K's (D = 64: one word of one half tile), channels of V likewise
    struct Share {
      uint32_t k[kMyK], k_scale[kMyK], v[2][S::kWords], v_scale[2][2];
      bool fine[2];
    } share;
    Entry e0, e1;
    const auto entries = [&](int tile) {
      const int j = tile < stop ? tile * kTile : reach.hi_most;
      e0 = entry_of(a, table, j, reach.hi_most);
      e1 = entry_of(a, table, j + 16, reach.hi_most);
    };
    const auto load = [&]() {
      const Place p0 = place_of<D>(a, head, e0), p1 = place_of<D>(a, head, e1);
      share.fine[0] = p0.fine;
      share.fine[1] = p1.fine;
#pragma unroll
      for (int i = 0; i < kMyK; ++i) {
        const int f = i * W + wave, w = S::kWords == 2 ? f % 2 : f % S::kWords;     // operand f: half tile f / words, word f % words
        const Place &p = f < S::kWords ? p0 : p1;
        share.k[i] = *(const __attribute__((address_space(1))) uint32_t *)(p.codes + (lanes.k + w / S::kRun * 16 * S::kRun + w % S::kRun * 4));
        share.k_scale[i] = *(const __attribute__((address_space(1))) uint16_t *)(p.scales + (lanes.k_scale + w / S::kRun * lanes.k_scale_step));
      }
      load_words<S::kWords>(share.v[0], p0.codes + lanes.v);
      load_words<S::kWords>(share.v[1], p1.codes + lanes.v);
      load_words<2>(share.v_scale[0], p0.scales + lanes.v_scale);
      load_words<2>(share.v_scale[1], p1.scales + lanes.v_scale);
    };
    const auto whole_tile = [&](int tile) {
      return share.fine[0] && share.fine[1] && tile * kTile >= reach.lo_most && tile * kTile + kTile <= reach.hi_least;
    };
    const auto make = [&](f16x8 *to, bool whole) {
#pragma unroll
      for (int i = 0; i < kMyK; ++i) {
        const uint32_t codes = share.k[i], both = share.k_scale[i];
        const f16x2 one = __builtin_bit_cast(f16x2, both), s = {one.x, one.x};
        Frag f;
        f.p[0] = two_codes<0>(codes) * s, f.p[1] = two_codes<1>(codes) * s;
        f.p[2] = two_codes<2>(codes) * s, f.p[3] = two_codes<3>(codes) * s;
        to[(i * W + wave) * kWave + lane] = f.v;
      }
      if (!whole) {
        const Frag bad = fix_scales(share.v_scale);
        if (wave == 0) to[(2 * S::kWords + S::kTiles) * kWave + lane] = bad.v;
      }
      // channels of V: two of a byte of the codes for each wavefront (one where there are four)
      Twins<D> twins[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) twins[i] = twins_of<D>(share.v[i / 2], i % 2);
#pragma unroll
      for (int c = 0; c < kMyV; ++c) {
        const int t = S::kTiles == 4 ? wave : c / 2 * 8 + 2 * wave + c % 2;
        Frag f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t two = share.v_scale[i / 2][i % 2];
          uint32_t word;
          if constexpr (S::kTiles == 4) word = select_bits(wave & 1 ? ~0u : 0u, twins[i].odd[0], twins[i].even[0]) >> 8 * (wave >> 1);      // (a choice between the two would put them into memory)
          else word = (c % 2 ? twins[i].odd[c / 2] : twins[i].even[c / 2]) >> 8 * wave;
          f.p[i] = two_codes<0>(word) * __builtin_bit_cast(f16x2, two);
        }
        to[(2 * S::kWords + t) * kWave + lane] = f.v;
      }
    };
    entries(start);
    load();
    entries(start + 1);
    bool fine0 = share.fine[0], fine1 = share.fine[1], whole = whole_tile(start);
    make(operands[0], whole);
    load();
    entries(start + 2);
    __syncthreads();
    for (int t = start; t < stop; ++t) {
      const int now = (t - start) & 1;
      const bool next_fine0 = share.fine[0], next_fine1 = share.fine[1], next_whole = whole_tile(t + 1);
      if (t + 1 < stop) make(operands[1 - now], next_whole);
      load();
      entries(t + 3);
      FromLds<D, kEarly> source = {&operands[now][lane]};
      one_tile<D, RT, T>(sums, rows, source, g, t * kTile, whole, fine0, fine1);
      fine0 = next_fine0, fine1 = next_fine1, whole = next_whole;
      __syncthreads();
    }
  }
  mark_bad<D, RT>(sums);
  const bool alone = a.splits == 1;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int row = first_row + rt * 16 + n;
    if (row >= all_rows) continue;
    const float total = sums.total[rt][0], over = total == 0.0f ? 0.0f : 1.0f / total;
    const int t = (int)fast_quotient((uint32_t)row, a.per_kv_div), h = kv * a.per_kv + row - t * a.per_kv;
    const int64_t at_row = (int64_t)work.item * kRows + wave * 16 * RT + rt * 16 + n;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int channel = (4 * g + r) * S::kTiles;
      float v[S::kTiles];
#pragma unroll
      for (int i = 0; i < S::kTiles; ++i) v[i] = !alone ? sums.out[rt][i][r] : total == 0.0f ? 0.0f : sums.out[rt][i][r] * over;
      if (alone) {
        store_row<T, S::kTiles>(a, a.out + b * a.ob + t * a.ot + h * a.oh, channel, v);
      } else {
#pragma unroll
        for (int i = 0; i < S::kTiles; i += 4) *(f32x4 *)(a.parts + at_row * D + channel + i) = f32x4{v[i], v[i + 1], v[i + 2], v[i + 3]};
      }
    }
    if (g == 0) {
      if (alone && a.log_sum) *(float *)(a.log_sum + b * a.lb + t * a.lt + h * a.lh) = log_of(sums.best[rt] * rows.scale[rt], total);
      if (!alone) *(float2 *)(a.part_sums + at_row * 2) = float2{sums.best[rt] * rows.scale[rt], total};
    }
  }
}

// The parts of a row joined.  Lanes first have the parts' sums; then WAVES wavefronts add up every WAVES-th part, four of them on their way at a time, and
// meet in LDS: all four of a workgroup where rows are few, one to a row where there are kJoinRows of them (65536 rows in four parts: 92 us less than with four).
// Parts that saw nothing have a sum of zero and are not read.
template <int D, int WAVES> __global__ __launch_bounds__(kBlock) void attention_join_kernel(const AttentionArgs a, uint32_t rows, int unit_rows) {
  constexpr int C = D / kWave, U = 4, R = kBlock / kWave / WAVES;     // R: rows of a workgroup
  __shared__ float part[WAVES > 1 ? WAVES : 1][WAVES > 1 ? D : 1];
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave) % WAVES;
  const int all_rows = a.queries * a.per_kv, splits = (int)a.splits;
  const int64_t units = a.units_div.d;
  for (uint32_t r0 = blockIdx.x; r0 < (rows + R - 1) / R; r0 += gridDim.x) {
    const uint32_t r = r0 * R + (R > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / kWave) : 0);
    if (r >= rows) break;            // (R > 1: of one wavefront, and no barrier follows)
    // rows: query heads fastest, then queries, heads of the cache, sequences
    const int bh = (int)(r / (uint32_t)all_rows), row = (int)(r % (uint32_t)all_rows), b = bh / (int)a.kv_div.d, kv = bh % (int)a.kv_div.d;
    const int64_t unit = (int64_t)bh * a.blocks_div.d + row / unit_rows, place = row % unit_rows;
    float2 ml = {-__builtin_inff(), 0.0f};
    if (lane < splits) ml = *(const float2 *)(a.part_sums + ((lane * units + unit) * unit_rows + place) * 2);
    float top = ml.x;
    for (int m = 1; m < kWave; m <<= 1) top = fmaxf(top, __shfl_xor(top, m));
    const float w = ml.y == 0.0f ? 0.0f : top == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f(ml.x - top);
    float total = ml.y == 0.0f ? 0.0f : ml.y * w;
    for (int m = 1; m < kWave; m <<= 1) total += __shfl_xor(total, m);
    const uint64_t any = __builtin_amdgcn_ballot_w64(ml.y != 0.0f);
    float v[C];
#pragma unroll
    for (int i = 0; i < C; ++i) v[i] = 0.0f;
    for (int s0 = wave; s0 < splits; s0 += WAVES * U) {
      float x[U][C];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int s = s0 + u * WAVES;
#pragma unroll
        for (int i = 0; i < C; ++i) x[u][i] = 0.0f;
        if (s < splits && any >> s & 1) {
          const float *from = a.parts + ((s * units + unit) * unit_rows + place) * D + lane * C;
#pragma unroll
          for (int i = 0; i < C; ++i) x[u][i] = from[i];
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float ws = __shfl(w, (s0 + u * WAVES) & 63);
#pragma unroll
        for (int i = 0; i < C; ++i) v[i] += ws * x[u][i];
      }
    }
    const int t = row / a.per_kv, h = kv * a.per_kv + row % a.per_kv;
    char *to = a.out + b * a.ob + t * a.ot + h * a.oh;
    if constexpr (WAVES == 1) {
#pragma unroll
      for (int i = 0; i < C; ++i) store_from_float(to + (lane * C + i) * a.oe, a.type, total == 0.0f ? 0.0f : v[i] / total);
      if (a.log_sum && lane == 0) *(float *)(a.log_sum + b * a.lb + t * a.lt + h * a.lh) = log_of(top, total);
    } else {
#pragma unroll
      for (int i = 0; i < C; ++i) part[wave][lane * C + i] = v[i];
      __syncthreads();
      for (int c = threadIdx.x; c < D; c += kBlock) {
        float x = 0.0f;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) x += part[i][c];
        store_from_float(to + c * a.oe, a.type, total == 0.0f ? 0.0f : x / total);
      }
      if (a.log_sum && threadIdx.x == 0) *(float *)(a.log_sum + b * a.lb + t * a.lt + h * a.lh) = log_of(top, total);
      __syncthreads();
    }
  }
}

// ---------------------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------------------

// How a call's rows and tokens go to workgroups; a function of the shapes alone.
struct Launch {
  int row_tiles;        // of a wavefront
  bool share;           // whether a workgroup's wavefronts have the same rows
  int64_t unit_rows, blocks, units, splits, items;
  int64_t least;        // tiles of a split, at least: of a sequence shorter than its table too
};

Launch launch_of(int64_t batch, int64_t queries, int64_t heads, int64_t kv, int64_t channels, int64_t capacity) {
  Launch l;
  const int64_t rows = queries * (heads / kv);
  l.row_tiles = rows <= 16 || channels == 256 ? 1 : 2;
  l.share = rows <= 64;
  l.unit_rows = 16 * l.row_tiles * (l.share ? 1 : kBlock / kWave);
  l.blocks = (rows + l.unit_rows - 1) / l.unit_rows;
  l.units = batch * kv * l.blocks;
  const int64_t tiles = (capacity + kTile - 1) / kTile, most = tiles <= kAloneTiles ? 1 : tiles / kLeastTiles;
  const int64_t wanted = l.units >= kAtOnce ? 1 : (channels == 256 ? kWorkgroupsWide : kWorkgroups) / std::max<int64_t>(l.units, 1);
  l.splits = std::max<int64_t>(1, std::min<int64_t>({most, kMaxSplits, wanted}));
  l.least = kLeastTiles;
  if (!l.share) {
    const bool full = l.units >= kAtOnce;
    if (full) l.least = kManyLeastFull;
    l.splits = std::max<int64_t>(1, std::min<int64_t>({most, tiles / (full ? kManyLeastFull : kManyLeast), kMaxSplits, kManyWorkgroups / std::max<int64_t>(l.units, 1)}));
  }
  l.items = l.units * l.splits;
  return l;
}

int done(hipError_t e) {
  if (e == hipSuccess) return OCN_OK;
  record_hip_error((int)e);
  return OCN_ERR_LAUNCH;
}

int check_shapes(const ocn_tensor *q, const ocn_tensor *cache, const ocn_tensor *table, int64_t *page) {
  int rc;
  if ((rc = check_operand(q, kHeadTypes)) != OCN_OK) return rc;
  if (q->ndim != 4) return OCN_ERR_NDIM;
  if ((rc = check_operand(cache, kByteType)) != OCN_OK) return rc;
  if (cache->ndim != 3) return OCN_ERR_NDIM;
  const int64_t kv = cache->size[1];
  if ((rc = check_cache(cache, q->size[3], kv, page)) != OCN_OK) return rc;
  if ((rc = check_operand(table, kIndexTypes)) != OCN_OK) return rc;
  if (table->ndim != 2) return OCN_ERR_NDIM;
  if (table->size[0] != q->size[0]) return OCN_ERR_SHAPE;
  if (q->size[2] > 0 && (kv == 0 || q->size[2] % kv != 0)) return OCN_ERR_SHAPE;
  const int64_t most = (int64_t)1 << 31;
  if (table->size[1] > (most - 64) / *page) return OCN_ERR_SHAPE;        // (tokens of a sequence)
  int64_t units = 1;
  for (int d = 0; d < 3; ++d) {
    if (q->size[d] != 0 && units > (most >> 6) / q->size[d]) return OCN_ERR_SHAPE;
    units *= q->size[d];
  }
  return OCN_OK;
}

bool whole_rows(const ocn_tensor *t) {
  if (t->stride[3] != head_type_size(t->dtype) || ((intptr_t)t->base + t->offset) % 16 != 0) return false;
  for (int d = 0; d < 3; ++d)
    if (t->size[d] > 1 && t->stride[d] % 16 != 0) return false;
  return true;
}

template <int D> void launch_attention(const AttentionArgs &a, const Launch &l, uint32_t grid, hipStream_t stream) {
#define OCN_ATTENTION(KERNEL, RT)                                                                                              \
  do {                                                                                                                         \
    if (a.type == OCN_BFLOAT16) hipLaunchKernelGGL((KERNEL<D, RT, bf16>), dim3(grid), dim3(kBlock), 0, stream, a);              \
    else if (a.type == OCN_HALF) hipLaunchKernelGGL((KERNEL<D, RT, f16>), dim3(grid), dim3(kBlock), 0, stream, a);             \
    else hipLaunchKernelGGL((KERNEL<D, RT, float>), dim3(grid), dim3(kBlock), 0, stream, a);                                     \
  } while (0)
  constexpr int kMany = D == 256 ? 1 : 2;      // row tiles whose sums and queries fit a wavefront's registers, two wavefronts to a SIMD
  if (!l.share) OCN_ATTENTION(attention_many_kernel, kMany);
  else if (l.row_tiles == 1) OCN_ATTENTION(attention_kernel, 1);
  else if constexpr (D < 256) OCN_ATTENTION(attention_kernel, 2);
#undef OCN_ATTENTION
}

template <int D> int run_attention(AttentionArgs &a, const Launch &l, uint32_t rows, hipStream_t stream) {
  // (no loop over items in the kernel: what a loop's first instructions share would be kept in registers that the tiles need)
  for (int64_t at = 0; at < l.items; at += max_launch_blocks()) {
    a.first_item = (uint32_t)at;
    launch_attention<D>(a, l, (uint32_t)std::min(l.items - at, max_launch_blocks()), stream);
    const int rc = done(hipGetLastError());
    if (rc != OCN_OK) return rc;
  }
  if (l.splits == 1) return OCN_OK;
  constexpr int kWaves = kBlock / kWave;
  if (rows >= kJoinRows) {
    const uint32_t joins = (uint32_t)std::min<int64_t>((rows + kWaves - 1) / kWaves, max_launch_blocks());
    hipLaunchKernelGGL((attention_join_kernel<D, 1>), dim3(joins), dim3(kBlock), 0, stream, a, rows, (int)l.unit_rows);
  } else {
    const uint32_t joins = (uint32_t)std::min<int64_t>(rows, max_launch_blocks());
    hipLaunchKernelGGL((attention_join_kernel<D, kWaves>), dim3(joins), dim3(kBlock), 0, stream, a, rows, (int)l.unit_rows);
  }
  return done(hipGetLastError());
}

}  // namespace
}  // namespace ocn

using namespace ocn;

extern "C" {

size_t ocn_cache_attention_workspace_bytes(const ocn_tensor *q, const ocn_tensor *cache, const ocn_tensor *table) {
  int64_t page;
  if (check_shapes(q, cache, table, &page) != OCN_OK || q->size[0] * q->size[1] * q->size[2] == 0) return 0;
  const Launch l = launch_of(q->size[0], q->size[1], q->size[2], cache->size[1], q->size[3], table->size[1] * page);
  return l.splits == 1 ? 0 : (size_t)l.items * l.unit_rows * (q->size[3] + 2) * sizeof(float);
}

int ocn_cache_attention(const ocn_tensor *q, const ocn_tensor *cache, const ocn_tensor *table, const ocn_tensor *visible,
                        double scale, int64_t window, const ocn_tensor *out, const ocn_tensor *log_sum, void *workspace,
                        size_t workspace_bytes, void *stream) {
  int64_t page;
  int rc = check_shapes(q, cache, table, &page);
  if (rc != OCN_OK) return rc;
  if ((rc = check_operand(visible, kIndexTypes)) != OCN_OK) return rc;
  if ((rc = check_operand(out, kHeadTypes)) != OCN_OK) return rc;
  if (log_sum && (rc = check_operand(log_sum, kFloatType)) != OCN_OK) return rc;
  if (visible->ndim != 2 || out->ndim != 4 || (log_sum && log_sum->ndim != 3)) return OCN_ERR_NDIM;
  if (out->dtype != q->dtype) return OCN_ERR_DTYPE;
  for (int d = 0; d < 4; ++d)
    if (out->size[d] != q->size[d]) return OCN_ERR_SHAPE;
  for (int d = 0; d < 3; ++d)
    if (log_sum && log_sum->size[d] != q->size[d]) return OCN_ERR_SHAPE;
  for (int d = 0; d < 2; ++d)
    if (visible->size[d] != q->size[d] && visible->size[d] != 1) return OCN_ERR_SHAPE;
  const float scale2 = (float)(scale * 1.4426950408889634074);      // (of exponents of two)
  if (!std::isfinite(scale2) || window < 0) return OCN_ERR_DOMAIN;
  const HeadOperand ops[6] = {{q, false}, {cache, false}, {table, false}, {visible, false}, {out, true, 0}, {log_sum, true}};
  if ((rc = check_operands(ops, 6)) != OCN_OK) return rc;
  AttentionArgs a;
  std::memset(&a, 0, sizeof a);
  a.q = (const char *)q->base + q->offset;
  a.out = (char *)out->base + out->offset;
  a.cache = (const char *)cache->base + cache->offset;
  a.table = (const char *)table->base + table->offset;
  a.seen = (const char *)visible->base + visible->offset;
  a.qb = q->stride[0], a.qt = q->stride[1], a.qh = q->stride[2], a.qe = q->stride[3];
  a.ob = out->stride[0], a.ot = out->stride[1], a.oh = out->stride[2], a.oe = out->stride[3];
  if (log_sum) {
    a.log_sum = (char *)log_sum->base + log_sum->offset;
    a.lb = log_sum->stride[0], a.lt = log_sum->stride[1], a.lh = log_sum->stride[2];
  }
  a.tb = table->stride[0], a.tc = table->stride[1];
  a.sb = visible->size[0] == 1 ? 0 : visible->stride[0];
  a.st = visible->size[1] == 1 ? 0 : visible->stride[1];
  a.page_stride = cache->stride[0];
  a.head_stride = cache->stride[1];
  a.pages = cache->size[0];
  a.window = window;
  const int64_t rows = q->size[0] * q->size[1] * q->size[2], d = q->size[3], kv = cache->size[1];
  if (rows == 0) return OCN_OK;
  const int64_t capacity = table->size[1] * page;
  const Launch l = launch_of(q->size[0], q->size[1], q->size[2], kv, d, capacity);
  if (l.items >= (int64_t)1 << 31) return OCN_ERR_SHAPE;
  if (l.splits > 1) {
    const size_t parts = (size_t)l.items * l.unit_rows * d;
    if (!workspace || workspace_bytes < (parts + (size_t)l.items * l.unit_rows * 2) * sizeof(float)) return OCN_ERR_WORKSPACE;
    if ((uintptr_t)workspace % 256 != 0) return OCN_ERR_ALIGN;
    a.parts = (float *)workspace;
    a.part_sums = a.parts + parts;
  }
  a.queries = (int32_t)q->size[1];
  a.per_kv = (int32_t)(q->size[2] / kv);
  a.capacity = a.pages > 0 ? (int32_t)capacity : 0;
  a.least = (int32_t)l.least;
  a.whole_q = whole_rows(q);
  a.whole_out = whole_rows(out);
  a.page = (int32_t)page;
  a.page_div = make_fastdiv((uint32_t)page);
  a.per_kv_div = make_fastdiv((uint32_t)a.per_kv);
  a.splits = (uint32_t)l.splits;
  a.units_div = make_fastdiv((uint32_t)l.units);
  a.blocks_div = make_fastdiv((uint32_t)l.blocks);
  a.kv_div = make_fastdiv((uint32_t)kv);
  a.type = q->dtype;
  a.table_wide = table->dtype == OCN_INT64;
  a.seen_wide = visible->dtype == OCN_INT64;
  a.scale = scale2;
  const hipStream_t s = (hipStream_t)stream;
  if (d == 64) return run_attention<64>(a, l, (uint32_t)rows, s);
  if (d == 128) return run_attention<128>(a, l, (uint32_t)rows, s);
  return run_attention<256>(a, l, (uint32_t)rows, s);
}

}  // extern "C"
