// Kernels of the gradient of attention over whole sequences, for one type.
//
// With weights p_ij = exp(scale q_i k_j - log_sum_i), made again from the queries and keys, and s_ij = p_ij (gout_i v_j - gout_i out_i):
//
//     gradient of v_j = sum_i p_ij gout_i,    of k_j = scale sum_i s_ij q_i,    of q_i = scale sum_j s_ij k_j.
//
// Two passes: one in which a workgroup has keys and goes over the rows (of all query heads that read them, so that their sums need no other workgroup), and one in which it has rows and goes over
// keys.  Scores and weights are made in both, seven products where five would do: the five of one pass leave the gradient of q in pieces of
// every block of keys, which would have to be added up in memory, in an order that changes from run to run or with more traffic than two products cost.
// Products bound both, at half of the matrix cores' cycles and the clock that power allows: 4 sequences of 4096 tokens, 32 heads, 8 of keys, 128 channels in bfloat16 1.88 ms, 1.09 of them over keys
// (with all seven products 1.03 PFLOP/s).
#pragma once

#include <algorithm>

#include "attention.hpp"
#include "attention_tiles.hpp"

namespace ocn {
namespace {

// log2 of what weights are multiplied by: a half holds 2^-14 ... 2^16 without loss, and weights are at most 1
template <class T> constexpr float kWeightTop = std::is_same<T, f16>::value ? 12.0f : 0.0f;

// A half's range is short for the s of all keys or rows: those of a lane's column are multiplied by a power of two of its own, chosen by the first of them and
// lowered, with what has been summed, where one would pass 2^15.  (Its logarithm is added to that of the weights where these are for nothing but s.)  It is up
// to 2^kMostShift, so that no product passes single precision's range (|s| < 2^41, weights up to 2^12): where all s are below 2^-60, they are short of bits that only a scale past 2^30 would show.
constexpr int kMostShift = 60;
template <class T> struct Range {
  static constexpr bool kNeeded = std::is_same<T, f16>::value;
  float factor = 1.0f, limit = 0.0f;
  __device__ __forceinline__ int exponent() const { return kNeeded ? __builtin_amdgcn_frexp_expf(factor) - 1 : 0; }
  // the largest s of a column, times its factor so far: what s and sums so far are to be multiplied by
  __device__ __forceinline__ float shift(float largest) {
    if (!(largest > limit)) return 1.0f;
    const int before = exponent(), e = before + 12 - __builtin_amdgcn_frexp_expf(largest);
    const float f = __builtin_ldexpf(1.0f, (e > kMostShift ? kMostShift : e < -kMostShift ? -kMostShift : e) - before);
    factor *= f, limit = 32768.0f;
    return f;
  }
  __device__ __forceinline__ float back() const { return kNeeded ? 1.0f / factor : 1.0f; }
};

// A weight from its exponent: a row's sum (2^kWeightTop) at most, and what that is off by.  (NaNs stay what they are, and where a query does not see the key it is set to zero behind this.)
__device__ __forceinline__ float weight(float x) { return __builtin_amdgcn_exp2f(x); }

// what to multiply a column's s and sums with, where some do not fit: s is times the factor
template <class T> __device__ __forceinline__ void in_range(acc_t<T> &s, Range<T> &range, acc_t<T> *out, int outs) {
  if constexpr (Range<T>::kNeeded) {
    float largest = 0.0f;
#pragma unroll
    for (int i = 0; i < Tile<T>::kOwn; ++i) largest = fmaxf(largest, __builtin_fabsf(s[i]));
    if (__any(largest > range.limit)) {
      const float f = range.shift(column_max<T>(largest));
#pragma unroll
      for (int ct = 0; ct < outs; ++ct)
#pragma unroll
        for (int i = 0; i < Tile<T>::kOwn; ++i) out[ct][i] *= f;
#pragma unroll
      for (int i = 0; i < Tile<T>::kOwn; ++i) s[i] *= f;
    }
  }
}

// (of results of TILE's products, in type T)
template <class T, int D, bool VEC, class TILE = Tile<T>> __device__ __forceinline__ void store_columns(const typename TILE::Acc *acc, char *row, int64_t step, int h, int d, float factor) {
#pragma unroll
  for (int ct = 0; ct < kTilesOf<TILE, D>; ++ct)
#pragma unroll
    for (int i = 0; i < TILE::kOwn; i += 4) {
      float v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = acc[ct][i + e] * factor;
      store_four<T, VEC>(row, step, ct * TILE::kSide + own_index<T>(i) + 4 * h, d, v);
    }
}

// a row's fragments in registers
template <class T, int D, bool VEC> __device__ __forceinline__ void load_fragments(frag_t<T> *f, const char *row, int64_t step, int d, int h, bool negative) {
#pragma unroll
  for (int c = 0; c < D / 16; ++c) {
    union { u32x4 v; frag_t<T> f; uint32_t u[4]; } x;
    x.v = load_piece<T, VEC>(row, step, 16 * c + Tile<T>::kFrag * h, d);
#pragma unroll
    for (int i = 0; i < 4; ++i) x.u[i] ^= negative ? (sizeof(T) == 2 ? 0x80008000u : 0x80000000u) : 0u;
    f[c] = x.f;
  }
}

template <class T> __device__ __forceinline__ acc_t<T> no_sum() {
  acc_t<T> a;
#pragma unroll
  for (int i = 0; i < Tile<T>::kOwn; ++i) a[i] = 0.0f;
  return a;
}

// ---- scores far from zero ------------------------------------------------------------------------
//
// A weight is 2^(score scale - log2 of the row's sum), and log_sum as it is given, rounded at its own size, is off by as much as a score of that size.  The four half steps of single precision that the exponent
// is off by change a weight by less than 3 10^-5 of itself up to kFar.  Past that a row has a reference, its largest score, as forward has one, and the sum of its weights relative to it: the
// pass over rows finds both, from its own scores, before anything else.  A weight is 2^((score - reference) scale - log2 of that sum), with the difference formed first.  Both passes make the same
// bits of a score: products of the same channels in the same order.  (4 sequences of 4096 tokens, 32 heads, 8 of keys, 128 channels in bfloat16: 2.64 ms instead of 1.91 where all rows are far; with a
// reference for every row 0.6 % more where none is.)
constexpr float kFar = 128.0f;

// What the passes need of a row, in the workspace, and of a row that is none, which has weights of zero: the exponent's part, minus gout * out, the reference (0: not far).  The order of blocks of
// keys is behind them.
constexpr int kRowPairs = 2;

// The largest score of the rows of a wavefront and the sum of their weights relative to it; `lo` and `hi`: what a row sees, `from` and `to`: what any of the rows do.  Keys come straight from memory.
template <class T, int D, bool VEC>
__device__ __forceinline__ void far_sums(const AttentionArgs &a, const frag_t<T> *q, const char *keys, int count, int lo, int hi, int from, int to, int lane, float *largest, float *sum) {
  constexpr int SIDE = Tile<T>::kSide, OWN = Tile<T>::kOwn;
  const int n = lane & (SIDE - 1), h = lane / SIDE;
  float best = -__builtin_inff(), total = 0.0f;
#pragma nounroll
  for (int first = from / SIDE * SIDE; first < to; first += SIDE) {
    frag_t<T> k[D / 16];
    load_fragments<T, D, VEC>(k, keys + (int64_t)(first + n < count ? first + n : count - 1) * a.k.token, a.k.channel, a.channels, h, false);
    acc_t<T> p = no_sum<T>();
    pipelined<D / 16, 0, frag_t<T>>([&](int c) { return k[c]; }, [&](int c, frag_t<T> x) { p = product(x, q[c], p); });
    float top = best;
#pragma unroll
    for (int i = 0; i < OWN; ++i) {
      const int j = first + 4 * h + own_index<T>(i);
      if (j < lo || j >= hi) p[i] = -__builtin_inff();
      top = fmaxf(top, p[i]);
    }
    top = column_max<T>(top);
    const float base = top > -__builtin_inff() ? top : 0.0f;
    total *= __builtin_amdgcn_exp2f((best - base) * a.scale);
#pragma unroll
    for (int i = 0; i < OWN; ++i) total += __builtin_amdgcn_exp2f((p[i] - base) * a.scale);
    best = top;
  }
  *largest = best, *sum = column_sum<T>(total);
}

// Queries that see some key of a block (query i sees the keys before i - ahead + 1), from a multiple of a tile's on, and the tiles that they make
struct KeyRows { int lo, hi, end, ahead, across, tiles; };
__device__ __forceinline__ KeyRows key_rows(const AttentionArgs &a, const Work &w, int block, int keys) {
  KeyRows r;
  r.end = block + keys < w.k.count ? block + keys : w.k.count;
  r.ahead = w.q.count - w.k.count;
  r.lo = 0, r.hi = w.q.count;
  if (a.causal) {
    r.lo = block + r.ahead > 0 ? (block + r.ahead) / a.rows_of_tile * a.rows_of_tile : 0;
    if (a.window && (int64_t)r.end - 1 + a.window + r.ahead < r.hi) r.hi = r.end - 1 + a.window + r.ahead;
  }
  r.across = (a.per_kv + a.heads - 1) / a.heads;         // tiles that a query's heads take
  r.tiles = r.hi > r.lo ? (r.hi - 1 - r.lo) / a.rows_of_tile * r.across + r.across : 0;
  return r;
}

// Gradients of keys and values: a wavefront has a tile's side of keys, in registers, with the sums for them (values, where registers are short, lie in LDS); rows go through
// LDS, the next ones on their way: some whole queries with the query heads of the group, or some of those.  (Up to 96 channels there are registers for values: nine sequences of 77 to 2903
// tokens, 16 heads of 80 halves, 961 us for 989 with them in LDS.)
template <int D> constexpr bool kValuesHeld = D > 96;

// operands of a step of both products
template <class T> struct Operands { frag_t<T> x, y, z; };

template <class T, int D, bool VEC, int WAVES>
__global__ __launch_bounds__(WAVES *kWave) __attribute__((amdgpu_waves_per_eu(kWavesAtOnce<T, D>))) void attention_keys_kernel(const AttentionArgs a, uint32_t first_block, const f32x2 *stats, const f32x2 *no_row) {
  warm_arguments<AttentionArgs>();
  constexpr int SIDE = Tile<T>::kSide, PITCH = Held<T, D>::kPitch, OWN = Tile<T>::kOwn, BLOCK = WAVES * SIDE;
  constexpr bool HELD = kValuesHeld<D>;
  __shared__ __align__(16) char held[2 * 2 * SIDE * PITCH];      // [2][q, gout][SIDE][PITCH]
  __shared__ __align__(16) char values[HELD ? BLOCK * PITCH : 16];
  __shared__ __align__(16) float of_row[2][4][kWave / 2];          // [2][exponent's part, minus gout out, reference, nothing]
  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), n = lane & (SIDE - 1), h = lane / SIDE;
  Work w;
  if (!find_work_of<true>(a, first_block + blockIdx.x, &w)) return;
  const int block = (int)(w.block * (uint32_t)BLOCK), key = block + wave * SIDE + n;
  const KeyRows rows = key_rows(a, w, block, BLOCK);
  const int end = rows.end, ahead = rows.ahead, lo = rows.lo, hi = rows.hi, across = rows.across;
  const Part part_here = part_of(rows.tiles, a.splits, kLeastKeyTiles, w.split);
  if (!part_here.mine) return;
  const bool mine = key < w.k.count;
  const int64_t token = w.k.first + (mine ? key : 0);
  if (VEC && a.channels < D) {
    clear_lds<WAVES * kWave>(held, sizeof held);
    if (HELD) clear_lds<WAVES * kWave>(values, sizeof values);
    __syncthreads();
  }
  const int64_t head = (int64_t)w.kv * a.per_kv, heads = (int64_t)a.kv * a.per_kv;
  const char *const pq = a.q.base + w.sequence * a.q.batch + w.q.first * a.q.token + head * a.q.head;
  const char *const pg = a.gout.base + w.sequence * a.gout.batch + w.q.first * a.gout.token + head * a.gout.head;
  const f32x2 *const ps = stats + kRowPairs * ((w.sequence * (a.q_starts.p ? 0 : a.q_starts.all) + w.q.first) * heads + head);
  Carrier<T, D, SIDE, WAVES, VEC> cq, cg;
  const auto load = [&](int at, int part, int turn) __attribute__((always_inline)) {
    char *const q = held + turn * 2 * SIDE * PITCH;
    const int last = hi - 1 - at, past = a.per_kv - 1 - part * a.heads;
    const auto row = [&](const HeadView &x, const char *p, int i) {       // (rows that are none are some other one)
      asm("" : "+v"(i));         // (nor is this)
      int t = (int)fast_quotient((uint32_t)i, a.heads_div), g = i - t * a.heads;
      t = t < last ? t : last, g = g < past ? g : past;
      return p + (int64_t)(at + t) * x.token + (int64_t)(part * a.heads + g) * x.head;
    };
    cq.load(q, [&](int i) { return row(a.q, pq, i); }, a.q.channel, a.channels);
    cg.load(q + SIDE * PITCH, [&](int i) { return row(a.gout, pg, i); }, a.gout.channel, a.channels);
    if (wave == 0) {      // what the rows have in stats: a word of each lane
      int i = lane & 31;
      asm("" : "+v"(i));
      const int t = (int)fast_quotient((uint32_t)i, a.heads_div), g = i - t * a.heads;
      const f32x2 *from = i < SIDE && t < a.rows_of_tile && t <= last && g <= past ? ps + kRowPairs * ((int64_t)(at + t) * heads + part * a.heads + g) : no_row;
      const uint32_t to = __builtin_amdgcn_readfirstlane(lds_address((const char *)of_row[turn]));
      load_word_to_lds(to, (const char *)from + (lane >> 5) * 4);
      load_word_to_lds(to + kWave * 4, (const char *)(from + 1) + (lane >> 5) * 4);
    }
  };
  const auto store = [&](int turn) {
    cq.store(held + turn * 2 * SIDE * PITCH);
    cg.store(held + (turn * 2 + 1) * SIDE * PITCH);
  };
  // From the last rows to the first: workgroups with other keys of a sequence, which start at other rows, then read the same ones at about the same time.
  int left = part_here.end - part_here.first, turn = 0;
  int at = lo + (part_here.end - 1) / across * a.rows_of_tile, part = (part_here.end - 1) % across;
  if constexpr (HELD) {
    Carrier<T, D, BLOCK, WAVES, VEC> cv;
    const char *const pv = a.v.base + w.sequence * a.v.batch + w.k.first * a.v.token + (int64_t)w.kv * a.v.head;
    cv.load(values, [&](int i) { return pv + (int64_t)(block + i < end ? block + i : end - 1) * a.v.token; }, a.v.channel, a.channels);
    cv.store(values);
  }
  if (left > 0) load(at, part, 0);
  frag_t<T> k[D / 16], v[HELD ? 1 : D / 16];
  load_fragments<T, D, VEC>(k, a.k.base + w.sequence * a.k.batch + token * a.k.token + w.kv * a.k.head, a.k.channel, mine && !a.nothing ? a.channels : 0, h, a.negative);
  if constexpr (!HELD)
    load_fragments<T, D, VEC>(v, a.v.base + w.sequence * a.v.batch + token * a.v.token + w.kv * a.v.head, a.v.channel, mine ? a.channels : 0, h, false);
  acc_t<T> gk[kTilesOf<Tile<T>, D>], gv[kTilesOf<Tile<T>, D>];
#pragma unroll
  for (int ct = 0; ct < kTilesOf<Tile<T>, D>; ++ct) gk[ct] = gv[ct] = no_sum<T>();
  Range<T> range;
  if (left > 0) store(0);
  const int from = block + wave * SIDE;
  const LanePlaces at_start = lane_places<T, D>(lane);
  const auto step = [&](auto masked, auto turn) __attribute__((always_inline)) {
    arrived();
    __syncthreads();
    const char *const q = held + turn * 2 * SIDE * PITCH, *const g = q + SIDE * PITCH;
    const int first_end = a.causal ? at - ahead + 1 : 0x7fffff00, last_end = first_end + a.rows_of_tile - 1;
    int next = at, next_part = part - 1;
    if (next_part < 0) next -= a.rows_of_tile, next_part = across - 1;
    if (left > 1) load(next, next_part, turn ^ 1);
    if (!masked || (from < last_end && (!a.window || from + SIDE > first_end - a.window))) {
      int here = h;
      LanePlaces places = at_start;
      asm("" : "+v"(here), "+v"(places.row), "+v"(places.column));      // (what hangs on them is not kept in registers from tile to tile)
      acc_t<T> p = no_sum<T>(), s;
#pragma unroll
      for (int i = 0; i < OWN; i += 4) {
        const f32x4 less = *(const f32x4 *)&of_row[turn][1][own_index<T>(i) + 4 * h];
#pragma unroll
        for (int e = 0; e < 4; ++e) s[i + e] = less[e];
      }
      const bool far = __any(of_row[turn][2][lane & 31] != 0.0f);
      pipelined<D / 16, 1, Operands<T>>(
          [&](int c) {
            Operands<T> o;
            o.x = rows_fragment<T, D>(q, 0, c, places);
            o.y = rows_fragment<T, D>(g, 0, c, places);
            if constexpr (HELD) o.z = rows_fragment<T, D>(values, wave * SIDE, c, places);
            return o;
          },
          [&](int c, const Operands<T> &o) {
            p = product(o.x, k[c], p);
            if constexpr (HELD) s = product(o.y, o.z, s);
            else s = product(o.y, v[c], s);
          });
      if (__builtin_expect(far, 0))
#pragma unroll
        for (int i = 0; i < OWN; ++i) p[i] -= of_row[turn][2][own_index<T>(i) + 4 * here];
#pragma unroll
      for (int i = 0; i < OWN; ++i) {
        p[i] = weight(__builtin_fmaf(p[i], a.scale, of_row[turn][0][own_index<T>(i) + 4 * h]));
        if constexpr (masked) {
          const int e = first_end + (int)fast_quotient((uint32_t)(own_index<T>(i) + 4 * here), a.heads_div);
          if (key >= e || (a.window && key < e - a.window)) p[i] = 0.0f;
        }
        s[i] *= p[i] * range.factor;
      }
      in_range<T>(s, range, gk, kTilesOf<Tile<T>, D>);
      frag_t<T> weights[Tile<T>::kSteps], slopes[Tile<T>::kSteps];
#pragma unroll
      for (int x = 0; x < Tile<T>::kSteps; ++x) weights[x] = as_fragment<T>(p, x), slopes[x] = as_fragment<T>(s, x);
      constexpr int TILES = kTilesOf<Tile<T>, D>, EACH = TILES * Tile<T>::kSteps;
      pipelined<2 * EACH, 2, frag_t<T>>([&](int i) { return columns_fragment<T, D>(i < EACH ? g : q, 16 * (i % EACH / TILES), i % TILES, places); },
                                        [&](int i, frag_t<T> x) {
                                          const int ct = i % TILES;
                                          if (i < EACH) gv[ct] = product(x, weights[i / TILES], gv[ct]);
                                          else gk[ct] = product(x, slopes[(i - EACH) / TILES], gk[ct]);
                                        });
    }
    if (left > 1) store(turn ^ 1);
    at = next, part = next_part, --left;
  };
  // Rows that see all of the workgroup's keys have a loop of their own
  const int first_whole = a.causal ? end - 1 + ahead : lo, past_whole = a.window ? block + a.window + ahead : 0x7fffffff;      // (rows past the last have no weights)
  const auto is_whole = [&] { return left > 0 && at >= first_whole && at <= past_whole - a.rows_of_tile; };
  while (left > 0) {
    if (turn == 0)      // two at a time, so that where they lie is known
      while (left > 1 && is_whole()) {
        step(std::false_type(), std::integral_constant<int, 0>());
        if (!is_whole()) {
          turn = 1;
          break;
        }
        step(std::false_type(), std::integral_constant<int, 1>());
      }
    if (left > 0) {
      step(std::true_type(), turn);
      turn ^= 1;
    }
  }
  arrived();      // (the values, where no query sees a key of the block and no step has waited for them: LDS may be another workgroup's once this one has ended)
  if (!mine) return;
  const float weight = kWeightTop<T> > 0.0f ? 0x1p-12f : 1.0f;
  if (!part_here.alone) {
    float *const to = a.parts + (((int64_t)w.unit * a.splits + w.split) * BLOCK + wave * SIDE + n) * (2 * kWidth<T, D>);
    store_columns<float, D, true, Tile<T>>(gk, (char *)to, 4, h, kWidth<T, D>, weight * range.back());
    store_columns<float, D, true, Tile<T>>(gv, (char *)(to + kWidth<T, D>), 4, h, kWidth<T, D>, weight);
    return;
  }
  store_columns<T, D, VEC>(gk, a.gk.base + w.sequence * a.gk.batch + token * a.gk.token + w.kv * a.gk.head, a.gk.channel, h, a.channels, a.true_scale * weight * range.back());
  store_columns<T, D, VEC>(gv, a.gv.base + w.sequence * a.gv.batch + token * a.gv.token + w.kv * a.gv.head, a.gv.channel, h, a.channels, weight);
}

// What parts of a block of keys came to, in their order: a wavefront to a key, lanes having channels.
template <class T, int D> __global__ __launch_bounds__(kBlock) void attention_keys_join_kernel(const AttentionArgs a, uint32_t first, int keys) {
  const int lane = threadIdx.x & (kWave - 1);
  Work w;
  const uint32_t chunks = (uint32_t)keys / kJoinRows, unit = (first + blockIdx.x) / chunks, chunk = first + blockIdx.x - unit * chunks;
  if (!find_work_of<true>(a, unit * (uint32_t)a.splits, &w)) return;
  const int block = (int)(w.block * (uint32_t)keys);
  const KeyRows rows = key_rows(a, w, block, keys);
  const int parts = part_of(rows.tiles, a.splits, kLeastKeyTiles, 0).parts;
  if (parts == 1) return;
  constexpr int EACH = (D + kWave - 1) / kWave, AT_ONCE = kJoinAtOnce / 2;
  for (int n = (int)chunk * kJoinRows + threadIdx.x / kWave; n < (int)(chunk + 1) * kJoinRows && block + n < rows.end; n += kBlock / kWave) {
    float gk[EACH], gv[EACH];
#pragma unroll
    for (int c = 0; c < EACH; ++c) gk[c] = gv[c] = 0.0f;
    for (int s = 0; s < parts; s += AT_ONCE) {
      float of_k[AT_ONCE][EACH], of_v[AT_ONCE][EACH];
#pragma unroll
      for (int u = 0; u < AT_ONCE; ++u) {
        const float *const from = a.parts + (((int64_t)w.unit * a.splits + (s + u < parts ? s + u : parts - 1)) * keys + n) * (2 * kWidth<T, D>);
#pragma unroll
        for (int c = 0; c < EACH; ++c) {
          const int e = c * kWave + lane < D ? c * kWave + lane : 0;
          of_k[u][c] = from[e], of_v[u][c] = from[kWidth<T, D> + e];
        }
      }
#pragma unroll
      for (int u = 0; u < AT_ONCE; ++u) {
#pragma unroll
        for (int c = 0; c < EACH; ++c) {
          gk[c] = s + u < parts ? gk[c] + of_k[u][c] : gk[c];
          gv[c] = s + u < parts ? gv[c] + of_v[u][c] : gv[c];
        }
      }
    }
    const int64_t token = w.k.first + block + n;
#pragma unroll
    for (int c = 0; c < EACH; ++c) {
      const int e = c * kWave + lane;
      if (e >= a.channels) continue;
      *(T *)(a.gk.base + w.sequence * a.gk.batch + token * a.gk.token + w.kv * a.gk.head + e * a.gk.channel) = (T)(gk[c] * a.true_scale);
      *(T *)(a.gv.base + w.sequence * a.gv.batch + token * a.gv.token + w.kv * a.gv.head + e * a.gv.channel) = (T)gv[c];
    }
  }
}

// Gradients of queries: a wavefront has a tile's side of rows, in registers, with the sums for them; keys and values go through LDS.
//
// gout * out, from the rounded out, is off by as much as out is.  Against the differences gout v - gout out that is little where a row sees many keys, but where it sees few it is as large as
// the rounding of the results.  Rows of workgroups that see kFewKeys keys at most sum p (gout v) instead, in a pass over the keys of its own, and leave it in stats for the pass over keys.
// (64 sequences of 100 tokens, 8 heads of 128 channels, forward and gradient: 82 us for 73 without, 250 tokens: 198 for 175.)
constexpr int kFewKeys = 256;

template <class T, int D, bool VEC, int WAVES, int KEYS>
__global__ __launch_bounds__(WAVES *kWave) __attribute__((amdgpu_waves_per_eu(kWavesAtOnce<T, D>))) void attention_queries_kernel(const AttentionArgs a, uint32_t first_block, f32x2 *stats, f32x2 *no_row) {
  warm_arguments<AttentionArgs>();
  constexpr int SIDE = Tile<T>::kSide, PITCH = Held<T, D>::kPitch, OWN = Tile<T>::kOwn;
  __shared__ __align__(16) char held[2 * 2 * KEYS * PITCH];      // [2][keys, values][KEYS][PITCH]
  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), n = lane & (SIDE - 1), h = lane / SIDE;
  if (first_block + blockIdx.x == 0 && threadIdx.x == 0) no_row[0] = f32x2{-__builtin_inff(), 0.0f}, no_row[1] = f32x2{0.0f, 0.0f};
  Work w;
  if (!find_work(a, first_block + blockIdx.x, &w)) return;
  const Limits all = limits_of_block(a, w), whole = limits_of_all(a, w);
  const bool few = all.hi - all.lo <= kFewKeys;
  const RowPlace place = row_place(a, w, wave * SIDE + n);
  const Limits own = limits_of(a, w, place.query);
  const int64_t token = w.q.first + place.query, head = (int64_t)w.kv * a.per_kv + place.head;
  const char *pk = a.k.base + w.sequence * a.k.batch + w.k.first * a.k.token + (int64_t)w.kv * a.k.head, *pv = a.v.base + w.sequence * a.v.batch + w.k.first * a.v.token + (int64_t)w.kv * a.v.head;
  if (VEC && a.channels < D) {
    clear_lds<WAVES * kWave>(held, sizeof held);
    __syncthreads();
  }
  Carrier<T, D, KEYS, WAVES, VEC> ck, cv;
  const auto load = [&](int at, int turn) {
    char *const k = held + turn * 2 * KEYS * PITCH;
    const int last = w.k.count - 1 - at;        // (rows past the end are the last one again)
    ck.load(k, [&](int i) { return pk + (int64_t)(at + (i < last ? i : last)) * a.k.token; }, a.k.channel, a.channels);
    cv.load(k + KEYS * PITCH, [&](int i) { return pv + (int64_t)(at + (i < last ? i : last)) * a.v.token; }, a.v.channel, a.channels);
  };
  const auto store = [&](int turn) {
    ck.store(held + turn * 2 * KEYS * PITCH);
    cv.store(held + (turn * 2 + 1) * KEYS * PITCH);
  };
  int at = all.lo / KEYS * KEYS, turn = 0;
  if (at < all.hi) load(at, 0);
  frag_t<T> q[D / 16], g[D / 16];
  load_fragments<T, D, VEC>(q, a.q.base + w.sequence * a.q.batch + token * a.q.token + head * a.q.head, a.q.channel, place.in && !a.nothing ? a.channels : 0, h, a.negative);
  load_fragments<T, D, VEC>(g, a.gout.base + w.sequence * a.gout.batch + token * a.gout.token + head * a.gout.head, a.gout.channel, place.in ? a.channels : 0, h, false);
  // What the passes need of a row: minus its log_sum in powers of two (plus kWeightTop), and minus gout * out.  (A row that sees nothing has weights of zero.)
  const int64_t stat_at = kRowPairs * ((w.sequence * (a.q_starts.p ? 0 : a.q_starts.all) + token) * ((int64_t)a.kv * a.per_kv) + head);
  const int hi_last = __builtin_amdgcn_readlane(own.hi, SIDE - 1), lo_first = __builtin_amdgcn_readfirstlane(own.lo);
  f32x2 stat;
  float reference = 0.0f;
  {
    frag_t<T> o[D / 16];
    load_fragments<T, D, VEC>(o, a.out.base + w.sequence * a.out.batch + token * a.out.token + head * a.out.head, a.out.channel, a.channels, h, false);
    const float log_sum = *(const float *)(a.log_sum.base + w.sequence * a.log_sum.batch + token * a.log_sum.token + head * a.log_sum.head);
    float sum = 0.0f;
#pragma unroll
    for (int c = 0; c < D / 16; ++c)
#pragma unroll
      for (int i = 0; i < Tile<T>::kFrag; ++i) sum = __builtin_fmaf((float)g[c][i], (float)o[c][i], sum);
    const float powers = log_sum * 1.44269504088896340736f;
    stat = f32x2{log_sum > -__builtin_inff() || log_sum != log_sum ? kWeightTop<T> - powers : -__builtin_inff(), -column_sum<T>(sum)};
    // (minus infinity, too, where a score past single precision's range may be what it stands for)
    const bool past = __builtin_fabsf(powers) > kFar && own.hi > own.lo;
    if (__any(past)) {
      float largest, total;
      far_sums<T, D, VEC>(a, q, pk, w.k.count, own.lo, own.hi, lo_first, hi_last, lane, &largest, &total);
      if (past && largest > -__builtin_inff()) stat.x = kWeightTop<T> - __builtin_amdgcn_logf(total), reference = largest;
    }
  }
  const bool far = __any(reference != 0.0f);
  const auto leave = [&] {
    if (!place.in || lane >= SIDE) return;
    stats[stat_at] = stat, stats[stat_at + 1] = f32x2{reference, 0.0f};
  };
  if (!few) leave();
  arrived();      // (the sums above have waited for loads behind these; LDS may be another workgroup's once this one has ended)
  if (!few && !a.gq.base) return;
  if (at < all.hi) store(0);
  const LanePlaces places = lane_places<T, D>(lane);
  Range<T> range;
  // the weights of a tile (times the range's factor), and gout v, which is added to s
  const auto weights = [&](const char *k, const char *v, int first, acc_t<T> &p, acc_t<T> &s, auto masked) {
    p = no_sum<T>();
    pipelined<D / 16, 2, Operands<T>>(
        [&](int c) {
          Operands<T> o;
          o.x = rows_fragment<T, D>(k, 0, c, places);
          o.y = rows_fragment<T, D>(v, 0, c, places);
          return o;
        },
        [&](int c, const Operands<T> &o) {
          p = product(o.x, q[c], p);
          s = product(o.y, g[c], s);
        });
    if (D > 128 || far)
#pragma unroll
      for (int i = 0; i < OWN; ++i) p[i] -= reference;
    const int lo = own.lo - first - 4 * h, hi = own.hi - first - 4 * h;
    const float less = stat.x + (float)range.exponent();
#pragma unroll
    for (int i = 0; i < OWN; ++i) {
      p[i] = weight(__builtin_fmaf(p[i], a.scale, less));
      if (masked && (own_index<T>(i) < lo || own_index<T>(i) >= hi)) p[i] = 0.0f;
    }
  };
  if (few) {
    float sum = 0.0f;
    for (; at < all.hi; at += KEYS, turn ^= 1) {
      arrived();
      __syncthreads();
      const char *const k = held + turn * 2 * KEYS * PITCH, *const v = k + KEYS * PITCH;
      const bool more = at + KEYS < all.hi;
      if (more) load(at + KEYS, turn ^ 1);
#pragma nounroll
      for (int t = 0; t < KEYS; t += SIDE) {
        if (at + t >= hi_last || at + t + SIDE <= lo_first) continue;
        acc_t<T> p, s = no_sum<T>();
        weights(k + t * PITCH, v + t * PITCH, at + t, p, s, std::true_type());
#pragma unroll
        for (int i = 0; i < OWN; ++i) sum = __builtin_fmaf(p[i], p[i] == 0.0f ? 0.0f : s[i], sum);
      }
      if (more) store(turn ^ 1);
    }
    stat.y = -column_sum<T>(sum) * (kWeightTop<T> > 0.0f ? 0x1p-12f : 1.0f);
    leave();
    arrived();
    __syncthreads();
    at = a.gq.base ? all.lo / KEYS * KEYS : all.hi, turn = 0;      // (no tile where nothing is left to do)
    if (at + KEYS < all.hi) {      // (a single tile is there already)
      load(at, 0);
      store(0);
    }
  }
  acc_t<T> gq[kTilesOf<Tile<T>, D>];
#pragma unroll
  for (int ct = 0; ct < kTilesOf<Tile<T>, D>; ++ct) gq[ct] = no_sum<T>();
  acc_t<T> start;      // of s
#pragma unroll
  for (int i = 0; i < OWN; ++i) start[i] = stat.y;
  const auto step = [&](auto masked, auto turn) __attribute__((always_inline)) {
    arrived();
    __syncthreads();
    const char *const keys = held + turn * 2 * KEYS * PITCH, *const values = keys + KEYS * PITCH;
    const bool more = at + KEYS < all.hi;
    if (more) load(at + KEYS, turn ^ 1);
#pragma unroll
    for (int t = 0; t < KEYS; t += SIDE) {
      const char *const k = keys + t * PITCH, *const v = values + t * PITCH;
      if (masked && (at + t >= hi_last || at + t + SIDE <= lo_first)) continue;
      acc_t<T> p, s = start;
      weights(k, v, at + t, p, s, masked);
#pragma unroll
      for (int i = 0; i < OWN; ++i) s[i] *= p[i];
      in_range<T>(s, range, gq, kTilesOf<Tile<T>, D>);
      frag_t<T> slopes[Tile<T>::kSteps];
#pragma unroll
      for (int x = 0; x < Tile<T>::kSteps; ++x) slopes[x] = as_fragment<T>(s, x);
      constexpr int TILES = kTilesOf<Tile<T>, D>;
      pipelined<TILES * Tile<T>::kSteps, 3, frag_t<T>>([&](int i) { return columns_fragment<T, D>(k, 16 * (i / TILES), i % TILES, places); },
                                                       [&](int i, frag_t<T> x) { gq[i % TILES] = product(x, slopes[i / TILES], gq[i % TILES]); });
    }
    if (more) store(turn ^ 1);
    at += KEYS;
  };
  while (at < all.hi) {
    if (turn == 0 && at >= whole.lo)      // two at a time, so that where they lie is known
      while (at + 2 * KEYS <= whole.hi) {
        step(std::false_type(), std::integral_constant<int, 0>());
        step(std::false_type(), std::integral_constant<int, 1>());
      }
    if (at < all.hi) {
      step(std::true_type(), turn);
      turn ^= 1;
    }
  }
  arrived();
  if (!place.in || !a.gq.base) return;
  const float weight = kWeightTop<T> > 0.0f ? 0x1p-12f : 1.0f;
  store_columns<T, D, VEC>(gq, a.gq.base + w.sequence * a.gq.batch + token * a.gq.token + head * a.gq.head, a.gq.channel, h, a.channels, a.true_scale * weight * range.back());
}

// ---------------------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------------------

template <class T, int D> constexpr bool kWideKeys = sizeof(T) == 2 && (D > 64 && D <= 128);
// keys of a tile of rows' gradients: half as many where they are on their way in registers (4 sequences of 2000 tokens, 16 heads of 100 channels: 704 us for 1014, of 228: 2534 for 3317)
template <class T, bool VEC> constexpr int kGradKeys = sizeof(T) == 2 && VEC ? 64 : 32;

int done(hipError_t e) {
  if (e == hipSuccess) return OCN_OK;
  record_hip_error((int)e);
  return OCN_ERR_LAUNCH;
}

template <class Launch> int in_launches(int64_t blocks, Launch launch) {
  for (int64_t at = 0; at < blocks; at += max_launch_blocks()) {
    launch((uint32_t)std::min<int64_t>(blocks - at, max_launch_blocks()), (uint32_t)at);
    const int rc = done(hipGetLastError());
    if (rc != OCN_OK) return rc;
  }
  return OCN_OK;
}

template <class T, int D, bool VEC> int run_grad(AttentionArgs &a, const AttentionSizes &sizes, const AttentionGrad &p, f32x2 *stats, hipStream_t stream) {
  constexpr int side = Tile<T>::kSide;
  int rc = OCN_OK;
  const uint32_t rows = (uint32_t)p.rows;
  const KeyPlan plan = key_plan_of(sizes, sizeof(T) == 4 ? OCN_FLOAT : OCN_HALF, D);
  AttentionArgs of_keys = a;
  if (!set_blocks(a, sizes, side * kGradWaves, 1) || !set_key_blocks(of_keys, sizes, side * plan.waves, plan.splits)) return OCN_ERR_SHAPE;
  const int64_t units = units_of(sizes, side * kGradWaves), key_units = p.keys ? plan.units : 0;
  if (ordered(sizes, key_units * plan.splits, slots_of_key_units(sizes, side * plan.waves))) {
    of_keys.order = (uint32_t *)(stats + kRowPairs * ((int64_t)rows + 1));
    hipLaunchKernelGGL(attention_order_kernel, dim3(1), dim3(kOrderLanes), 0, stream, of_keys);
    if ((rc = done(hipGetLastError())) != OCN_OK) return rc;
  }
  rc = in_launches(units, [&](uint32_t grid, uint32_t first) {
    hipLaunchKernelGGL((attention_queries_kernel<T, D, VEC, kGradWaves, kGradKeys<T, VEC>>), dim3(grid), dim3(kGradWaves * kWave), 0, stream, a, first, stats, stats + kRowPairs * (int64_t)rows);
  });
  if (rc != OCN_OK) return rc;
  // (rows of a tile: whole queries with the heads of the group, or some of those)
  of_keys.heads = std::max(1, std::min(a.per_kv, side));
  of_keys.heads_div = make_fastdiv((uint32_t)of_keys.heads);
  of_keys.rows_of_tile = side / of_keys.heads;
  of_keys.parts = (float *)((char *)stats + grad_head_bytes(sizes, side, plan.waves));
  rc = in_launches(key_units * plan.splits, [&](uint32_t grid, uint32_t first) {
    constexpr int wide = kWideKeys<T, D> ? 8 : 4;
    if (plan.waves == wide) hipLaunchKernelGGL((attention_keys_kernel<T, D, VEC, wide>), dim3(grid), dim3(wide * kWave), 0, stream, of_keys, first, stats, stats + kRowPairs * (int64_t)rows);
    else hipLaunchKernelGGL((attention_keys_kernel<T, D, VEC, 4>), dim3(grid), dim3(4 * kWave), 0, stream, of_keys, first, stats, stats + kRowPairs * (int64_t)rows);
  });
  if (rc != OCN_OK || plan.splits == 1) return rc;
  rc = in_launches(key_units * (side * plan.waves / kJoinRows), [&](uint32_t grid, uint32_t first) {
    hipLaunchKernelGGL((attention_keys_join_kernel<T, D>), dim3(grid), dim3(kBlock), 0, stream, of_keys, first, side * plan.waves);
  });
  return rc;
}

template <class T> int run_grad_type(AttentionArgs &a, const AttentionSizes &sizes, const AttentionGrad &p, bool vec, void *workspace, hipStream_t stream) {
#define OCN_RUN(T, D, VEC) return run_grad<T, D, VEC>(a, sizes, p, (f32x2 *)workspace, stream)
  OCN_BY_PADDED(T, a.channels, vec, OCN_RUN);
#undef OCN_RUN
}

}  // namespace
}  // namespace ocn
