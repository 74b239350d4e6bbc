// Kernels of attention over whole sequences, for one type.
#pragma once

#include <algorithm>

#include "attention.hpp"
#include "attention_tiles.hpp"

namespace ocn {
namespace {

// ---------------------------------------------------------------------------------------
// One pass over the keys.  A wavefront has the rows of one tile; for some keys at a time it forms scores^T = K Q^T and out^T += V^T P^T, so that a lane holds scores
// and results of one row: the row's largest score, the sum of its weights and what results are scaled by need no other lane than the one or three that share the row.
//
// Weights are relative to a reference, the row's largest score when it was last set.  It is set by the first keys, and again, with results rescaled, only
// where a lane's weights come to more than kMost: no maximum is looked for otherwise.  A weight is 2^(s scale - reference scale), one multiply-add and one exponential: the
// reference's rounding is the same for all weights of a row.  Where scores are so large (kFine) that it could make weights too large, and for float,
// the difference is formed before it is scaled.
// ---------------------------------------------------------------------------------------

// log2 of the weight of a score that is the reference.  A half holds 2^-14 ... 2^16 without loss: weights are put near its upper end, 32 of a lane below kMost.
template <class T> constexpr float kTop = std::is_same<T, f16>::value ? 9.0f : 0.0f;
template <class T> constexpr float kMost = std::is_same<T, f16>::value ? 46341.0f : 512.0f;
constexpr float kFine = 1024.0f;

// What a wavefront has of its rows
template <class T, int D> struct Rows {
  frag_t<T> q[D / 16];
  acc_t<T> out[kTilesOf<Tile<T>, D>];
  float best, total;           // the score that weights are relative to (minus infinity: none yet), the sum of a lane's own weights
  int lo, hi;                  // keys that the row sees
  bool exact;                  // differences of scores are formed before they are scaled
};

template <class T> __device__ __forceinline__ acc_t<T> zero_acc() {
  acc_t<T> a;
#pragma unroll
  for (int i = 0; i < Tile<T>::kOwn; ++i) a[i] = 0.0f;
  return a;
}

// ---- values that are no numbers -------------------------------------------------------------------
//
// Weights of zero would make NaNs of infinities and NaNs in the products, so that they would reach rows that do not see them.  In tiles that some row does not see whole they are looked for; where there
// are any, it is found which keys have one in a channel, lanes note which of their row's results they reach, in two bits of a result that are kept in LDS (infinity, minus infinity; both: NaN), and the
// tile's values become zeros.  Results take from the bits what they are in the end.  (4096 tokens, 8 heads, all values NaN, call included: 135 us, with numbers 128; with rows by themselves, key by key, 75 ms.)

// Whether there are any among KEYS keys' values in LDS
template <class T, int D, int KEYS> __device__ __forceinline__ bool odd_values(const char *v, int lane) {
  constexpr uint32_t exponent = std::is_same<T, float>::value ? 0x7f800000u : std::is_same<T, f16>::value ? 0x7c007c00u : 0x7f807f80u;
  constexpr uint32_t one = std::is_same<T, float>::value ? 0x00800000u : std::is_same<T, f16>::value ? 0x04000400u : 0x00800080u;
  uint32_t odd = 0;
  asm volatile("" : "+v"(lane));      // (what hangs on it is not kept in registers from tile to tile)
  static_assert(KEYS * Held<T, D>::kPieces % kWave == 0, "all lanes have as many pieces");
#pragma unroll 4
  for (int n = 0; n < KEYS * Held<T, D>::kPieces / kWave; ++n) {
    const int i = n * kWave + lane;
    const u32x4 x = *(const u32x4 *)(v + Held<T, D>::at(i / Held<T, D>::kPieces, i % Held<T, D>::kPieces));
#pragma unroll
    for (int e = 0; e < 4; ++e) odd |= (x[e] & exponent) + one;      // (into the sign's place where all bits of an exponent are set)
  }
  return __any((odd & (sizeof(T) == 2 ? 0x80008000u : 0x80000000u)) != 0);
}

__device__ __forceinline__ bool is_odd(float x) { return !(__builtin_fabsf(x) < __builtin_inff()); }
// the bits of a lane's results: a word for each tile of channels
template <class T, int D, int WAVES> struct Bits { uint32_t words[kTilesOf<Tile<T>, D>][WAVES * kWave]; };

// ... and which of a tile's keys have one in a channel: infinities and NaNs, infinities below zero and NaNs
template <class T, int D, int KEYS> struct OddKeys { uint32_t of[kWidth<T, D>][2][(KEYS + 31) / 32]; };

// From KEYS keys' values in LDS, by LANES lanes
template <class T, int D, int KEYS, int LANES> __device__ __forceinline__ void find_odd_keys(OddKeys<T, D, KEYS> &keys, const char *v, int lane) {
  constexpr int EACH = KEYS < 32 ? KEYS : 32;
  asm volatile("" : "+v"(lane));      // (what hangs on it is not kept in registers from tile to tile)
#pragma nounroll
  for (int c = lane; c < D; c += LANES)
#pragma nounroll
    for (int w = 0; w < KEYS / EACH; ++w) {
      uint32_t up = 0, down = 0;
#pragma unroll 4
      for (int i = 0; i < EACH; ++i) {
        const float x = (float)*(const T *)(v + Held<T, D>::at(w * EACH + i, c * (int)sizeof(T) / 16) + c * (int)sizeof(T) % 16);
        const uint32_t one = is_odd(x) ? 1u << i : 0u;
        up |= x < 0.0f ? 0u : one, down |= x > 0.0f ? 0u : one;
      }
      keys.of[c][0][w] = up, keys.of[c][1][w] = down;
    }
}
// What of them reaches a lane's results, which see the keys lo ... hi - 1: into its bits, which are none so far where `any` is not set
template <class T, int D, int KEYS, int WAVES> __device__ __forceinline__ void note_odd_keys(Bits<T, D, WAVES> &bits, bool *any, const OddKeys<T, D, KEYS> &keys, int lo, int hi, int lane) {
  constexpr int WORDS = (KEYS + 31) / 32;
  int thread = threadIdx.x;
  asm volatile("" : "+v"(lane), "+v"(thread));
  uint32_t sees[WORDS];
#pragma unroll
  for (int w = 0; w < WORDS; ++w) {
    const auto below = [&](int n) { return n <= w * 32 ? 0u : n >= w * 32 + 32 ? ~0u : (1u << (n - w * 32)) - 1u; };      // keys before n
    sees[w] = below(hi) & ~below(lo);
  }
#pragma nounroll
  for (int ct = 0; ct < kTilesOf<Tile<T>, D>; ++ct) {
    uint32_t own = *any ? bits.words[ct][thread] : 0u;
#pragma unroll 2
    for (int i = 0; i < Tile<T>::kOwn; ++i) {
      const int c = ct * Tile<T>::kSide + own_index<T>(i) + 4 * (lane / Tile<T>::kSide);
      uint32_t up = 0, down = 0;
#pragma unroll
      for (int w = 0; w < WORDS; ++w) up |= keys.of[c][0][w] & sees[w], down |= keys.of[c][1][w] & sees[w];
      own |= ((up ? 1u : 0u) | (down ? 2u : 0u)) << 2 * i;
    }
    bits.words[ct][thread] = own;
  }
  *any = true;
}
// zeros in their places, by LANES lanes
template <class T, int D, int KEYS, int LANES> __device__ __forceinline__ void clear_odd_values(char *v, int lane) {
  asm volatile("" : "+v"(lane));
#pragma nounroll
  for (int i = lane; i < KEYS * Held<T, D>::kPieces; i += LANES) {
    union { u32x4 v; T t[16 / sizeof(T)]; } x;
    u32x4 *const at = (u32x4 *)(v + Held<T, D>::at(i / Held<T, D>::kPieces, i % Held<T, D>::kPieces));
    x.v = *at;
#pragma unroll
    for (int e = 0; e < 16 / (int)sizeof(T); ++e)
      if (is_odd((float)x.t[e])) x.t[e] = (T)0.0f;
    *at = x.v;
  }
}
// a lane's results in the end
template <class T, int D, int WAVES> __device__ __forceinline__ void take_odd_values(const Bits<T, D, WAVES> &bits, acc_t<T> *out) {
#pragma unroll
  for (int ct = 0; ct < kTilesOf<Tile<T>, D>; ++ct) {
    const uint32_t own = bits.words[ct][threadIdx.x];
#pragma unroll
    for (int i = 0; i < Tile<T>::kOwn; ++i) {
      const uint32_t two = own >> 2 * i & 3u;
      out[ct][i] += two == 3u ? __builtin_nanf("") : two == 2u ? -__builtin_inff() : two == 1u ? __builtin_inff() : 0.0f;
    }
    in_order();
  }
}

// operands that are read ahead of their products (one, as the compiler has it: 1833 us of the prompts below instead of 1763)
template <class T, int D> constexpr int kScoresAhead = 4;
template <class T, int D> constexpr int kValuesAhead = 5;

// the weights of scores, in their place, relative to the row's reference: their sum over a lane's own
template <class T, int TILES> __device__ __forceinline__ float weigh(const acc_t<T> *s, acc_t<T> *p, float best, float scale, bool exact) {
  float sum = 0.0f;
  if (exact) {
#pragma unroll
    for (int t = 0; t < TILES; ++t)
#pragma unroll
      for (int i = 0; i < Tile<T>::kOwn; ++i) p[t][i] = __builtin_fmaf(s[t][i] - best, scale, kTop<T>);
  } else {
    const float less = __builtin_fmaf(-best, scale, kTop<T>);
#pragma unroll
    for (int t = 0; t < TILES; ++t)
#pragma unroll
      for (int i = 0; i < Tile<T>::kOwn; ++i) p[t][i] = __builtin_fmaf(s[t][i], scale, less);
  }
#pragma unroll
  for (int t = 0; t < TILES; ++t)
#pragma unroll
    for (int i = 0; i < Tile<T>::kOwn; ++i) {
      p[t][i] = __builtin_amdgcn_exp2f(p[t][i]);
      sum += p[t][i];
    }
  return sum;
}

// KEYS keys of a tile in LDS, from key `first` of the sequence on.  MASKED: some row does not see all of them.
template <class T, int D, int KEYS, bool MASKED> __device__ __forceinline__ void attend(Rows<T, D> &r, const char *k, const char *v, int first, float scale, int lane) {
  constexpr int SIDE = Tile<T>::kSide, TILES = KEYS / SIDE, OWN = Tile<T>::kOwn, STEPS = Tile<T>::kSteps;
  const int h = lane / SIDE;
  const LanePlaces places = lane_places<T, D>(lane);
  acc_t<T> s[TILES], p[TILES];
#pragma unroll
  for (int t = 0; t < TILES; ++t) s[t] = zero_acc<T>();
  pipelined<TILES * D / 16, kScoresAhead<T, D>, frag_t<T>>([&](int i) { return rows_fragment<T, D>(k, i % TILES * SIDE, i / TILES, places); },
                                                           [&](int i, frag_t<T> x) { s[i % TILES] = product(x, r.q[i / TILES], s[i % TILES]); });
  if constexpr (MASKED) {
    const int lo = r.lo - first - 4 * h, hi = r.hi - first - 4 * h;
#pragma unroll
    for (int t = 0; t < TILES; ++t)
#pragma unroll
      for (int i = 0; i < OWN; ++i)
        if (t * SIDE + own_index<T>(i) < lo || t * SIDE + own_index<T>(i) >= hi) s[t][i] = -__builtin_inff();
  }
  float sum = weigh<T, TILES>(s, p, r.best, scale, r.exact);
  // The first scores, or some far above the reference (no score at all, and NaNs, are not)
  if (__any(!(sum <= kMost<T>))) {
    float top = s[0][0];
#pragma unroll
    for (int t = 0; t < TILES; ++t)
#pragma unroll
      for (int i = 0; i < OWN; ++i) top = fmaxf(top, s[t][i]);
    top = column_max<T>(top);
    const bool before = r.best > -__builtin_inff(), now = before || top > -__builtin_inff();
    const float best = before ? fmaxf(r.best, top) : now ? top : 0.0f, keep = before ? __builtin_amdgcn_exp2f((r.best - best) * scale) : 0.0f;
    r.exact = r.exact || __any(!(__builtin_fabsf(best * scale) < kFine));
    r.best = now ? best : -__builtin_inff();
    r.total *= keep;
#pragma unroll
    for (int ct = 0; ct < kTilesOf<Tile<T>, D>; ++ct)
#pragma unroll
      for (int i = 0; i < OWN; ++i) r.out[ct][i] *= keep;
    sum = weigh<T, TILES>(s, p, best, scale, r.exact);
  }
  r.total += sum;
  frag_t<T> f[TILES * STEPS];
#pragma unroll
  for (int x = 0; x < TILES * STEPS; ++x) f[x] = as_fragment<T>(p[x / STEPS], x % STEPS);
  constexpr int OUTS = kTilesOf<Tile<T>, D>;
  pipelined<TILES * STEPS * OUTS, kValuesAhead<T, D>, frag_t<T>>([&](int i) { return columns_fragment<T, D>(v, 16 * (i / OUTS), i % OUTS, places); },
                                                                 [&](int i, frag_t<T> x) { r.out[i % OUTS] = product(x, f[i / OUTS], r.out[i % OUTS]); });
}

// Keys [first, first + KEYS) of a sequence on their way into LDS, by `LANES` lanes; those past the end are zero.
template <class T, int D, bool VEC, int KEYS, int LANES> struct Carried {
  static constexpr int kAll = KEYS * Held<T, D>::kPieces, kEach = (kAll + LANES - 1) / LANES;
  u32x4 k[kEach], v[kEach];
  __device__ __forceinline__ void load(const AttentionArgs &a, const char *pk, const char *pv, int first, int count, int lane) {
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int at = i * LANES + lane, row = at / Held<T, D>::kPieces, e = at % Held<T, D>::kPieces * (16 / (int)sizeof(T)), j = first + row;
      const bool in = (kAll % LANES == 0 || at < kAll) && j < count;
      k[i] = load_piece<T, VEC>(pk + (int64_t)(in ? j : 0) * a.k.token, a.k.channel, e, in ? a.channels : 0);
      v[i] = load_piece<T, VEC>(pv + (int64_t)(in ? j : 0) * a.v.token, a.v.channel, e, in ? a.channels : 0);
    }
  }
  __device__ __forceinline__ void store(char *hk, char *hv, int lane) const {
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int at = i * LANES + lane;
      if (kAll % LANES != 0 && at >= kAll) continue;
      const int place = Held<T, D>::at(at / Held<T, D>::kPieces, at % Held<T, D>::kPieces);
      *(u32x4 *)(hk + place) = k[i];
      *(u32x4 *)(hv + place) = v[i];
    }
  }
};

// the row that lane n of a tile has, and its queries: Q, and the keys that it sees
template <class T, int D, bool VEC> __device__ __forceinline__ void start_rows(Rows<T, D> &r, const AttentionArgs &a, const Work &w, int row, int lane, const char *q) {
  constexpr int SIDE = Tile<T>::kSide;
  const int h = lane / SIDE;
  const RowPlace p = row_place(a, w, row);
  Limits l = limits_of(a, w, p.query);
  r.lo = l.lo, r.hi = l.hi;
  r.best = -__builtin_inff();
  r.total = 0.0f;
  r.exact = std::is_same<T, float>::value;
#pragma unroll
  for (int ct = 0; ct < kTilesOf<Tile<T>, D>; ++ct) r.out[ct] = zero_acc<T>();
  const char *at = q + (int64_t)p.query * a.q.token + (int64_t)p.head * a.q.head;
#pragma unroll
  for (int c = 0; c < D / 16; ++c) {
    union { u32x4 v; frag_t<T> f; uint32_t u[4]; } x;
    x.v = load_piece<T, VEC>(at, a.q.channel, 16 * c + Tile<T>::kFrag * h, p.in && !a.nothing ? a.channels : 0);
#pragma unroll
    for (int i = 0; i < 4; ++i) x.u[i] ^= a.negative ? (sizeof(T) == 2 ? 0x80008000u : 0x80000000u) : 0u;
    r.q[c] = x.f;
  }
}

// log of the sum of exponentials of a row, in natural logarithms
template <class T> __device__ __forceinline__ float log_sum_of(const AttentionArgs &a, float best, float total) {
  return total > 0.0f || total != total ? __builtin_fmaf(best > -__builtin_inff() ? best : 0.0f, a.plain_scale, (__builtin_amdgcn_logf(total) - kTop<T>) * 0.69314718055994530942f) : -__builtin_inff();
}

// where a row lies in a tensor of query heads
__device__ __forceinline__ int64_t row_offset(const HeadView &x, const AttentionArgs &a, const Work &w, const RowPlace &p) {
  return w.sequence * x.batch + (w.q.first + p.query) * x.token + ((int64_t)w.kv * a.per_kv + p.head) * x.head;
}

// a row's results, lanes having channels 64 apart
template <class T, int D> __device__ __forceinline__ void finish_row(const AttentionArgs &a, const Work &w, const RowPlace &p, const float *x, float best, float total, int lane) {
  const float over = total > 0.0f || total != total ? 1.0f / total : 0.0f;
  char *const out = a.out.base + row_offset(a.out, a, w, p);
#pragma unroll
  for (int c = 0; c < (D + kWave - 1) / kWave; ++c)
    if (c * kWave + lane < a.channels) *(T *)(out + (c * kWave + lane) * a.out.channel) = (T)(x[c] * over);
  if (a.log_sum.base && lane == 0) *(float *)(a.log_sum.base + row_offset(a.log_sum, a, w, p)) = log_sum_of<T>(a, best, total);
}

// a row's place among the parts
__device__ __forceinline__ int64_t part_row(const AttentionArgs &a, const Work &w, int row) { return ((int64_t)w.unit * a.splits + w.split) * a.rows + row; }

// The part of a block's keys, in tiles of so many, that a workgroup has
struct Split { int first, end, parts; bool alone, mine; };
__device__ __forceinline__ Split split_of(const AttentionArgs &a, const Limits &all, int keys, int least, int split) {
  const int lo = all.lo / keys, hi = (all.hi + keys - 1) / keys;
  const Part p = part_of(hi > lo ? hi - lo : 0, a.splits, least, split);
  Split s = {(lo + p.first) * keys, (lo + p.end) * keys, p.parts, p.alone, p.mine};
  if (s.end > all.hi) s.end = all.hi;
  return s;
}

// Many rows: the wavefronts of a workgroup have a tile of rows each and share the keys, which go through LDS once for all of them, the next ones on their way.
// Products bound it, and exponentials, which take about as many cycles (of 128 channels; of 64 more), at the clock that power allows: 16 prompts of 101 to 6000 tokens, 32 heads, 8 of
// keys, 128 channels in bfloat16 1690 to 1774 us on different cards (970 to 930 TFLOP/s; a large product 1263), one of 30011 tokens, 16 heads, 4 of keys, 64 channels in half precision 2040 to 2161 (905 to 855).  Two wavefronts to a SIMD, whose results
// and queries fill their registers, take each other's waits (3873 us of those prompts with one, and rows through registers).
template <class T, int D, bool VEC, int WAVES, int KEYS> __global__ __launch_bounds__(WAVES *kWave) __attribute__((amdgpu_waves_per_eu(sizeof(T) == 2 && (D <= 128 || VEC && D <= 192) ? 2 : 1))) void attention_rows_kernel(const AttentionArgs a, uint32_t first_block) {
  warm_arguments<AttentionArgs>();
  constexpr int SIDE = Tile<T>::kSide, PITCH = Held<T, D>::kPitch;
  __shared__ __align__(16) char lds[2 * 2 * KEYS * PITCH];        // [2][keys, values][KEYS][PITCH]
  __shared__ Bits<T, D, WAVES> bits;
  __shared__ OddKeys<T, D, KEYS> odd_keys;
  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  Work w;
  if (!find_work(a, first_block + blockIdx.x, &w)) return;
  const Limits block = limits_of_block(a, w), whole = limits_of_all(a, w);
  const Split split = split_of(a, block, KEYS, kLeastRowTiles, w.split);
  if (!split.mine) return;
  const struct { int lo, hi; } all = {split.first, split.end};
  const char *pk = a.k.base + w.sequence * a.k.batch + w.k.first * a.k.token + (int64_t)w.kv * a.k.head, *pv = a.v.base + w.sequence * a.v.batch + w.k.first * a.v.token + (int64_t)w.kv * a.v.head;
  Carrier<T, D, KEYS, WAVES, VEC> ck, cv;
  const auto load = [&](int at, int turn) {
    char *const k = lds + turn * 2 * KEYS * PITCH;
    const int last = w.k.count - 1 - at;        // (rows past the end are the last one again)
    ck.load(k, [&](int i) { return pk + (int64_t)(at + (i < last ? i : last)) * a.k.token; }, a.k.channel, a.channels);
    cv.load(k + KEYS * PITCH, [&](int i) { return pv + (int64_t)(at + (i < last ? i : last)) * a.v.token; }, a.v.channel, a.channels);
  };
  const auto store = [&](int turn) {
    ck.store(lds + turn * 2 * KEYS * PITCH);
    cv.store(lds + (turn * 2 + 1) * KEYS * PITCH);
  };
  int at = all.lo, turn = 0;
  if (VEC && a.channels < D) {
    clear_lds<WAVES * kWave>(lds, sizeof lds);
    __syncthreads();
  }
  if (at < all.hi) load(at, 0);
  Rows<T, D> r;
  const int row = wave * SIDE + (lane & (SIDE - 1));
  start_rows<T, D, VEC>(r, a, w, row, lane, a.q.base + w.sequence * a.q.batch + w.q.first * a.q.token + (int64_t)w.kv * a.per_kv * a.q.head);
  const int hi_first = __builtin_amdgcn_readfirstlane(r.hi), hi_last = __builtin_amdgcn_readlane(r.hi, SIDE - 1), lo_first = __builtin_amdgcn_readfirstlane(r.lo),
            lo_last = __builtin_amdgcn_readlane(r.lo, SIDE - 1);
  bool odd = false;
  if (at < all.hi) store(0);
  // Tiles that all rows of the workgroup see whole have a loop of their own: what masks need takes none of its registers.
  const auto step = [&](auto masked, auto turn) {
    arrived();
    __syncthreads();
    char *const k = lds + turn * 2 * KEYS * PITCH, *const v = k + KEYS * PITCH;
    const bool more = at + KEYS < all.hi;
    if (more) load(at + KEYS, turn ^ 1);
    if constexpr (masked) {
      if (__builtin_expect(odd_values<T, D, KEYS>(v, lane), 0)) {      // (all wavefronts find the same)
        find_odd_keys<T, D, KEYS, WAVES * kWave>(odd_keys, v, threadIdx.x);
        __syncthreads();
        clear_odd_values<T, D, KEYS, WAVES * kWave>(v, threadIdx.x);
        note_odd_keys<T, D, KEYS, WAVES>(bits, &odd, odd_keys, r.lo - at, r.hi - at, lane);
        __syncthreads();
      }
    }
    if (!masked || (at < hi_last && at + KEYS > lo_first)) attend<T, D, KEYS, masked>(r, k, v, at, a.scale, lane);
    if (more) store(turn ^ 1);
    at += KEYS;
  };
  while (at < all.hi) {
    if (turn == 0 && at >= whole.lo)      // two at a time, so that where they lie is known
      while (at + 2 * KEYS <= whole.hi && at + 2 * KEYS <= all.hi) {
        step(std::false_type(), std::integral_constant<int, 0>());
        step(std::false_type(), std::integral_constant<int, 1>());
      }
    if (at < all.hi) {
      step(std::true_type(), turn);
      turn ^= 1;
    }
  }
  arrived();
  if (odd) take_odd_values<T, D, WAVES>(bits, r.out);
  const float total = column_sum<T>(r.total), over = total > 0.0f || total != total ? 1.0f / total : 0.0f;
  const RowPlace p = row_place(a, w, row);
  if (!p.in) return;
  if (!split.alone) {
    const int64_t part = part_row(a, w, row);
#pragma unroll
    for (int ct = 0; ct < kTilesOf<Tile<T>, D>; ++ct)
#pragma unroll
      for (int i = 0; i < Tile<T>::kOwn; i += 4)
        *(f32x4 *)(a.parts + part * kWidth<T, D> + ct * SIDE + own_index<T>(i) + 4 * (lane / SIDE)) = f32x4{r.out[ct][i], r.out[ct][i + 1], r.out[ct][i + 2], r.out[ct][i + 3]};
    if (lane < SIDE) a.part_sums[2 * part] = r.best, a.part_sums[2 * part + 1] = total;
    return;
  }
  char *const out = a.out.base + row_offset(a.out, a, w, p);
#pragma unroll
  for (int ct = 0; ct < kTilesOf<Tile<T>, D>; ++ct)
#pragma unroll
    for (int i = 0; i < Tile<T>::kOwn; i += 4) {
      float v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = r.out[ct][i + e] * over;
      store_four<T, VEC>(out, a.out.channel, ct * SIDE + own_index<T>(i) + 4 * (lane / SIDE), a.channels, v);
    }
  if (a.log_sum.base && lane < SIDE)
    *(float *)(a.log_sum.base + row_offset(a.log_sum, a, w, p)) = log_sum_of<T>(a, r.best, total);
}

// Few rows (single tokens): the wavefronts of a workgroup have the same tile of rows and take every fourth tile of keys, through a part of LDS of their own; a long sequence is
// split over workgroups as well.  What they found is joined here, and that of several workgroups by a second launch.  Memory bounds it: the next token of 48 sequences of 1 to 8192, 8 heads of keys of
// 128 halves (806 MB), 161 us, 5.0 TB/s, as a large copy.

template <class T, int D, bool VEC>
__global__ __launch_bounds__(kFewWaves *kWave) __attribute__((amdgpu_waves_per_eu(kWavesAtOnce<T, D>))) void attention_few_kernel(const AttentionArgs a, uint32_t first_block) {
  warm_arguments<AttentionArgs>();
  constexpr int SIDE = Tile<T>::kSide, PITCH = Held<T, D>::kPitch, PART = 2 * SIDE * PITCH;
  static_assert(SIDE * kWidth<T, D> * 4 <= PART, "a wavefront's results take the place of its keys and values");
  __shared__ __align__(16) char lds[kFewWaves * PART];        // [wavefronts][keys, values][SIDE][PITCH]
  __shared__ float bests[kFewWaves][SIDE], totals[kFewWaves][SIDE];
  __shared__ Bits<T, D, kFewWaves> bits;
  __shared__ OddKeys<T, D, SIDE> odd_keys[kFewWaves];
  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), n = lane & (SIDE - 1);
  Work w;
  if (!find_work(a, first_block + blockIdx.x, &w)) return;
  const Limits all = limits_of_block(a, w);
  const Split split = split_of(a, all, SIDE, kLeastTiles, w.split);
  if (!split.mine) return;
  Rows<T, D> r;
  start_rows<T, D, VEC>(r, a, w, n, lane, a.q.base + w.sequence * a.q.batch + w.q.first * a.q.token + (int64_t)w.kv * a.per_kv * a.q.head);
  const char *pk = a.k.base + w.sequence * a.k.batch + w.k.first * a.k.token + (int64_t)w.kv * a.k.head, *pv = a.v.base + w.sequence * a.v.batch + w.k.first * a.v.token + (int64_t)w.kv * a.v.head;
  const int hi_first = __builtin_amdgcn_readfirstlane(r.hi), lo_last = __builtin_amdgcn_readlane(r.lo, SIDE - 1);
  char *const k = lds + wave * PART, *const v = k + SIDE * PITCH;
  Carried<T, D, VEC, SIDE, kWave> next;
  int at = split.first + wave * SIDE;
  bool odd = false;
  if (at < split.end) next.load(a, pk, pv, at, w.k.count, lane);
  const auto step = [&](auto masked) {
    next.store(k, v, lane);
    if (at + kFewWaves * SIDE < split.end) next.load(a, pk, pv, at + kFewWaves * SIDE, w.k.count, lane);
    __builtin_amdgcn_wave_barrier();
    if constexpr (masked) {
      if (__builtin_expect(odd_values<T, D, SIDE>(v, lane), 0)) {
        find_odd_keys<T, D, SIDE, kWave>(odd_keys[wave], v, lane);
        __builtin_amdgcn_wave_barrier();
        clear_odd_values<T, D, SIDE, kWave>(v, lane);
        note_odd_keys<T, D, SIDE, kFewWaves>(bits, &odd, odd_keys[wave], r.lo - at, r.hi - at, lane);
        __builtin_amdgcn_wave_barrier();
      }
    }
    attend<T, D, SIDE, masked>(r, k, v, at, a.scale, lane);
    __builtin_amdgcn_wave_barrier();
    at += kFewWaves * SIDE;
  };
  while (at < split.end) {
    while (at >= lo_last && at + SIDE <= hi_first && at < split.end) step(std::false_type());
    if (at < split.end) step(std::true_type());
  }
  if (odd) take_odd_values<T, D, kFewWaves>(bits, r.out);
  const float total = column_sum<T>(r.total);
  if (lane < SIDE) bests[wave][n] = r.best, totals[wave][n] = total;
  __syncthreads();
  float best = bests[0][n];
#pragma unroll
  for (int i = 1; i < kFewWaves; ++i) best = fmaxf(best, bests[i][n]);
  const float keep = r.best > -__builtin_inff() ? __builtin_amdgcn_exp2f((r.best - best) * a.scale) : 0.0f;
  float *const own = (float *)k;       // [SIDE][kWidth]
#pragma unroll
  for (int ct = 0; ct < kTilesOf<Tile<T>, D>; ++ct)
#pragma unroll
    for (int i = 0; i < Tile<T>::kOwn; ++i) own[n * kWidth<T, D> + ct * SIDE + own_index<T>(i) + 4 * (lane / SIDE)] = r.out[ct][i] * keep;
  __syncthreads();
  for (int i = threadIdx.x; i < SIDE * (kWidth<T, D> / 4); i += kFewWaves * kWave) {
    const int row = i / (kWidth<T, D> / 4), e = i % (kWidth<T, D> / 4) * 4;
    const RowPlace p = row_place(a, w, row);
    if (!p.in) continue;
    float top = bests[0][row], sum = 0.0f, x[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int u = 1; u < kFewWaves; ++u) top = fmaxf(top, bests[u][row]);
#pragma unroll
    for (int u = 0; u < kFewWaves; ++u) {
      const float b = bests[u][row];
      sum += totals[u][row] * (b > -__builtin_inff() ? __builtin_amdgcn_exp2f((b - top) * a.scale) : 1.0f);
      const f32x4 y = *(const f32x4 *)(lds + u * PART + (row * kWidth<T, D> + e) * 4);
#pragma unroll
      for (int c = 0; c < 4; ++c) x[c] += y[c];
    }
    if (split.alone) {
      const float over = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
#pragma unroll
      for (int c = 0; c < 4; ++c) x[c] *= over;
      store_four<T, VEC>(a.out.base + row_offset(a.out, a, w, p), a.out.channel, e, a.channels, x);
      if (a.log_sum.base && e == 0) *(float *)(a.log_sum.base + row_offset(a.log_sum, a, w, p)) = log_sum_of<T>(a, top, sum);
    } else {
      const int64_t part = part_row(a, w, row);
      *(f32x4 *)(a.parts + part * kWidth<T, D> + e) = f32x4{x[0], x[1], x[2], x[3]};
      if (e == 0) a.part_sums[2 * part] = top, a.part_sums[2 * part + 1] = sum;
    }
  }
}

// What several workgroups found of a row, joined: a wavefront to a row.  Latency bounds it (32 rows of 59 parts: 8 us).
template <class T, int D> __global__ __launch_bounds__(kBlock) void attention_join_kernel(const AttentionArgs a, uint32_t first, int keys, int least) {
  constexpr int EACH = (D + kWave - 1) / kWave;
  const int lane = threadIdx.x & (kWave - 1);
  Work w;
  const uint32_t chunks = (uint32_t)a.rows / kJoinRows, unit = (first + blockIdx.x) / chunks, chunk = first + blockIdx.x - unit * chunks;
  if (!find_work(a, unit * (uint32_t)a.splits, &w)) return;
  const Limits all = limits_of_block(a, w);
  const int parts = split_of(a, all, keys, least, 0).parts;
  if (parts == 1) return;
  for (int row = (int)chunk * kJoinRows + threadIdx.x / kWave; row < (int)(chunk + 1) * kJoinRows; row += kBlock / kWave) {
    const RowPlace p = row_place(a, w, row);
    if (!p.in) continue;
    const int64_t part = (int64_t)w.unit * a.splits * a.rows + row;
    const bool there = lane < parts;
    const float own = there ? a.part_sums[2 * (part + (int64_t)lane * a.rows)] : -__builtin_inff();
    float top = own;
#pragma unroll
    for (int o = 32; o > 0; o /= 2) top = fmaxf(top, __shfl_xor(top, o));
    const float keep = !there ? 0.0f : own > -__builtin_inff() ? __builtin_amdgcn_exp2f((own - top) * a.scale) : 1.0f;
    float sum = there ? a.part_sums[2 * (part + (int64_t)lane * a.rows) + 1] * keep : 0.0f;
#pragma unroll
    for (int o = 32; o > 0; o /= 2) sum += __shfl_xor(sum, o);
    float x[EACH];
#pragma unroll
    for (int c = 0; c < EACH; ++c) x[c] = 0.0f;
    for (int s = 0; s < parts; s += kJoinAtOnce) {
      float y[kJoinAtOnce][EACH];
#pragma unroll
      for (int u = 0; u < kJoinAtOnce; ++u) {
        const float *const from = a.parts + (part + (int64_t)(s + u < parts ? s + u : parts - 1) * a.rows) * kWidth<T, D>;
#pragma unroll
        for (int c = 0; c < EACH; ++c) y[u][c] = from[c * kWave + lane < D ? c * kWave + lane : 0];
      }
#pragma unroll
      for (int u = 0; u < kJoinAtOnce; ++u) {
        const float f = __shfl(keep, (s + u) & (kWave - 1));
#pragma unroll
        for (int c = 0; c < EACH; ++c) x[c] = s + u < parts ? __builtin_fmaf(y[u][c], f, x[c]) : x[c];
      }
    }
    finish_row<T, D>(a, w, p, x, top, sum, lane);
  }
}

// ---------------------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------------------

int done(hipError_t e) {
  if (e == hipSuccess) return OCN_OK;
  record_hip_error((int)e);
  return OCN_ERR_LAUNCH;
}

// Keys of a tile of many rows: half as many where a wavefront's results take half of its registers or more, which 64 scores to a row would drive to memory (half precision, 4 sequences of 4096 tokens, 16 heads of 192 channels: 511 for 714 us; 256 channels, which stay at one wavefront to a SIMD: 860 for 810 us, and 68 for 110 where rows begin anywhere).
template <class T, int D> constexpr int kRowKeys = sizeof(T) == 2 && D <= 128 ? 64 : 32;

template <class T, int D> constexpr bool kWide = sizeof(T) == 2 && (D > 64 && D <= 128);

template <class T, int D, bool VEC> int run(AttentionArgs &a, const AttentionPlan &p, hipStream_t stream) {
  const int64_t blocks = p.units * p.splits;
  int rc;
  const int64_t most = max_launch_blocks();
  for (int64_t at = 0; at < blocks; at += most) {
    const uint32_t grid = (uint32_t)std::min(blocks - at, most), first = (uint32_t)at;
    if (p.few) hipLaunchKernelGGL((attention_few_kernel<T, D, VEC>), dim3(grid), dim3(kFewWaves * kWave), 0, stream, a, first);
    else if (kWide<T, D> && p.waves == 8) hipLaunchKernelGGL((attention_rows_kernel<T, D, VEC, kWide<T, D> ? 8 : 4, kRowKeys<T, D>>), dim3(grid), dim3(8 * kWave), 0, stream, a, first);
    else hipLaunchKernelGGL((attention_rows_kernel<T, D, VEC, 4, kRowKeys<T, D>>), dim3(grid), dim3(4 * kWave), 0, stream, a, first);
    if ((rc = done(hipGetLastError())) != OCN_OK) return rc;
  }
  if (p.splits == 1) return OCN_OK;
  const int64_t joins = p.units * (p.rows / kJoinRows);
  for (int64_t at = 0; at < joins; at += most) {
    const uint32_t grid = (uint32_t)std::min(joins - at, most), first = (uint32_t)at;
    hipLaunchKernelGGL((attention_join_kernel<T, D>), dim3(grid), dim3(kBlock), 0, stream, a, first, p.few ? (int)Tile<T>::kSide : kRowKeys<T, D>, p.few ? kLeastTiles : kLeastRowTiles);
    if ((rc = done(hipGetLastError())) != OCN_OK) return rc;
  }
  return OCN_OK;
}

template <class T> int run_type(AttentionArgs &a, const AttentionPlan &p, bool vec, hipStream_t stream) {
#define OCN_RUN(T, D, VEC) return run<T, D, VEC>(a, p, stream)
  OCN_BY_PADDED(T, a.channels, vec, OCN_RUN);
#undef OCN_RUN
}

}  // namespace
}  // namespace ocn
