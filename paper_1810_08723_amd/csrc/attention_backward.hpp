// Kernels of the gradient of attention over whole sequences, for one type.
//
// With weights p_ij = exp(scale q_i k_j - log_sum_i), made again from the queries and keys, and s_ij = p_ij (gout_i v_j - gout_i out_i):
//
//     gradient of v_j = sum_i p_ij gout_i,    of k_j = scale sum_i s_ij q_i,    of q_i = scale sum_j s_ij k_j.
//
// Two passes: one in which a workgroup has keys and goes over the rows (of all query heads that read them, so that their sums need no other workgroup), and one in which it has rows and goes over
// keys.  Scores and weights are made in both, seven products where five would do: the five of one pass leave the gradient of q in pieces of
// every block of keys, which would have to be added up in memory, in an order that changes from run to run or with more traffic than two products cost.
#pragma once

#include <algorithm>

#include "attention.hpp"
#include "attention_tiles.hpp"

namespace ocn {
namespace {

// log2 of what weights are multiplied by: a half holds 2^-14 ... 2^16 without loss, and weights are at most 1
template <class T> constexpr float kWeightTop = std::is_same<T, f16>::value ? 12.0f : 0.0f;

// What the passes need of a row: minus its log_sum in powers of two (plus kWeightTop), and gout * out.  The same for all keys: one launch of its own, which reads gout and out once.
template <class T, bool VEC> __global__ __launch_bounds__(kBlock) void attention_along_kernel(const AttentionArgs a, uint32_t rows, FastDiv heads, FastDiv queries, f32x2 *stats) {
  constexpr int LANES = 16, EACH = 16 / (int)sizeof(T);        // of a row; channels of a piece
  const int lane = threadIdx.x % LANES;
  for (uint32_t r = blockIdx.x * (kBlock / LANES) + threadIdx.x / LANES; r < rows; r += gridDim.x * (kBlock / LANES)) {
    const uint32_t t = fast_quotient(r, heads), h = r - t * heads.d, b = fast_quotient(t, queries);
    const int64_t token = t - b * queries.d;
    const char *g = a.gout.base + b * a.gout.batch + token * a.gout.token + h * a.gout.head, *o = a.out.base + b * a.out.batch + token * a.out.token + h * a.out.head;
    float s = 0.0f;
    for (int e = lane * EACH; e < a.channels; e += LANES * EACH) {
      union { u32x4 v; T t[EACH]; } x, y;
      x.v = load_piece<T, VEC>(g, a.gout.channel, e, a.channels);
      y.v = load_piece<T, VEC>(o, a.out.channel, e, a.channels);
#pragma unroll
      for (int i = 0; i < EACH; ++i) s = __builtin_fmaf((float)x.t[i], (float)y.t[i], s);
    }
    s = sum_over_row(s, LANES);
    if (lane == 0) {
      const float log_sum = *(const float *)(a.log_sum.base + b * a.log_sum.batch + token * a.log_sum.token + h * a.log_sum.head);
      // (a row that sees nothing has weights of zero)
      stats[r] = f32x2{log_sum > -__builtin_inff() || log_sum != log_sum ? kWeightTop<T> - log_sum * 1.44269504088896340736f : -__builtin_inff(), s};
    }
  }
}

// A half's range is short for the s of all keys or rows: those of a lane's column are multiplied by a power of two of its own, chosen by the first of them and
// lowered, with what has been summed, where one would pass 2^15.
template <class T> struct Range {
  static constexpr bool kNeeded = std::is_same<T, f16>::value;
  float factor = kNeeded ? 0.0f : 1.0f;
  // what sums so far are to be multiplied by
  __device__ __forceinline__ bool lower(float largest, float *keep) {
    if constexpr (!kNeeded) return false;
    const bool mine = largest * factor > 32768.0f || (factor == 0.0f && largest > 0.0f);
    if (!__any(mine)) return false;
    *keep = 1.0f;
    if (mine) {
      int e = 12 - __builtin_amdgcn_frexp_expf(largest);
      e = e > 120 ? 120 : e < -120 ? -120 : e;
      const float f = __builtin_ldexpf(1.0f, e);
      if (factor > 0.0f) *keep = f / factor;
      factor = f;
    }
    return true;
  }
  __device__ __forceinline__ float back() const { return !kNeeded ? 1.0f : factor > 0.0f ? 1.0f / factor : 0.0f; }
};

// p (times 2^kWeightTop) and s of a tile, out of scores and gout v.  `best` and `along`: of the elements' rows
template <class T, class Row> __device__ __forceinline__ void weights_of(acc_t<T> &p, acc_t<T> &s, float scale, const Row &row) {
#pragma unroll
  for (int i = 0; i < Tile<T>::kOwn; ++i) {
    const f32x2 r = row(i);
    // (above the row's sum by rounding alone, but of scores of any size)
    p[i] = __builtin_amdgcn_exp2f(fminf(__builtin_fmaf(p[i], scale, r.x), kWeightTop<T>));
    s[i] = p[i] * (s[i] - r.y);
  }
}

// s as fragments: times the column's factor
template <class T, int TILES, class Out> __device__ __forceinline__ void in_range(acc_t<T> *s, Range<T> &range, Out *out, int outs) {
  if constexpr (Range<T>::kNeeded) {
    float largest = 0.0f, keep;
#pragma unroll
    for (int t = 0; t < TILES; ++t)
#pragma unroll
      for (int i = 0; i < Tile<T>::kOwn; ++i) largest = fmaxf(largest, __builtin_fabsf(s[t][i]));
    if (range.lower(column_max<T>(largest), &keep)) {
#pragma unroll
      for (int ct = 0; ct < outs; ++ct)
#pragma unroll
        for (int i = 0; i < Tile<T>::kOwn; ++i) out[ct][i] *= keep;
    }
#pragma unroll
    for (int t = 0; t < TILES; ++t)
#pragma unroll
      for (int i = 0; i < Tile<T>::kOwn; ++i) s[t][i] *= range.factor;
  }
}

// four neighbouring channels of a row, rounded
template <class T, bool VEC> __device__ __forceinline__ void store_run(char *row, int64_t step, int e, int d, const float *v) {
  if constexpr (VEC) {
    typedef T V __attribute__((ext_vector_type(4)));
    V o;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = (T)v[i];
    if (e < d) *(V *)(row + e * (int)sizeof(T)) = o;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (e + i < d) *(T *)(row + (e + i) * step) = (T)v[i];
  }
}

template <class T, int D, bool VEC> __device__ __forceinline__ void store_columns(const acc_t<T> *acc, char *row, int64_t step, int h, int d, float factor) {
#pragma unroll
  for (int ct = 0; ct < D / Tile<T>::kSide; ++ct)
#pragma unroll
    for (int i = 0; i < Tile<T>::kOwn; i += 4) {
      float v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = acc[ct][i + e] * factor;
      store_run<T, VEC>(row, step, ct * Tile<T>::kSide + own_index<T>(i) + 4 * h, d, v);
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

// Two tensors' rows on their way into LDS
template <class T, int D, int ROWS, int LANES> struct Pair {
  static constexpr int kAll = ROWS * Held<T, D>::kPieces, kEach = (kAll + LANES - 1) / LANES;
  u32x4 x[kEach], y[kEach];
  // place(row, &x's row, &y's row): false where there is none
  template <bool VEC, class Place> __device__ __forceinline__ void load(const Place &place, int64_t x_step, int64_t y_step, int d, int lane) {
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int at = i * LANES + lane, row = at / Held<T, D>::kPieces, e = at % Held<T, D>::kPieces * (16 / (int)sizeof(T));
      const char *px, *py;
      const bool in = place(row, &px, &py) && (kAll % LANES == 0 || at < kAll);
      x[i] = load_piece<T, VEC>(px, x_step, e, in ? d : 0);
      y[i] = load_piece<T, VEC>(py, y_step, e, in ? d : 0);
    }
  }
  __device__ __forceinline__ void store(char *hx, char *hy, int lane) const {
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int at = i * LANES + lane;
      if (kAll % LANES != 0 && at >= kAll) continue;
      const int to = Held<T, D>::at(at / Held<T, D>::kPieces, at % Held<T, D>::kPieces);
      *(u32x4 *)(hx + to) = x[i];
      *(u32x4 *)(hy + to) = y[i];
    }
  }
};

// Gradients of keys and values: a wavefront has a tile's side of keys, in registers, with the sums for them; rows go through LDS, the next ones on their way.
template <class T, int D, bool VEC, int WAVES> __global__ __launch_bounds__(WAVES *kWave) void attention_keys_kernel(const AttentionArgs a, uint32_t first_block, const f32x2 *stats) {
  warm_arguments<AttentionArgs>();
  constexpr int SIDE = Tile<T>::kSide, PITCH = Held<T, D>::kPitch, OWN = Tile<T>::kOwn;
  __shared__ __align__(16) char held[2 * 2 * SIDE * PITCH];      // [2][q, gout][SIDE][PITCH]
  __shared__ __align__(16) f32x2 of_row[2][SIDE];
  __shared__ __align__(16) int ends[2][SIDE];                    // keys before which a row sees
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, n = lane & (SIDE - 1), h = lane / SIDE;
  Work w;
  if (!find_work_of<true>(a, first_block + blockIdx.x, &w)) return;
  const int block = (int)(w.block * (uint32_t)(WAVES * SIDE)), key = block + wave * SIDE + n;
  const bool mine = key < w.k.count;
  const int64_t token = w.k.first + (mine ? key : 0);
  frag_t<T> k[D / 16], v[D / 16];
  load_fragments<T, D, VEC>(k, a.k.base + w.sequence * a.k.batch + token * a.k.token + w.kv * a.k.head, a.k.channel, mine && !a.nothing ? a.channels : 0, h, a.negative);
  load_fragments<T, D, VEC>(v, a.v.base + w.sequence * a.v.batch + token * a.v.token + w.kv * a.v.head, a.v.channel, mine ? a.channels : 0, h, false);
  acc_t<T> gk[D / SIDE], gv[D / SIDE];
#pragma unroll
  for (int ct = 0; ct < D / SIDE; ++ct) gk[ct] = gv[ct] = no_sum<T>();
  Range<T> range;
  // queries that see some key of the workgroup's
  const int last = block + WAVES * SIDE < w.k.count ? block + WAVES * SIDE - 1 : w.k.count - 1, ahead = w.q.count - w.k.count;
  int lo = 0, hi = w.q.count;
  if (a.causal) {
    lo = block + ahead > 0 ? block + ahead : 0;
    if (a.window && (int64_t)last + a.window + ahead < hi) hi = last + a.window + ahead;
  }
  const uint32_t begin = (uint32_t)lo * (uint32_t)a.per_kv, end = hi > lo ? (uint32_t)hi * (uint32_t)a.per_kv : begin;
  const int64_t head = (int64_t)w.kv * a.per_kv;
  const char *const pq = a.q.base + w.sequence * a.q.batch + w.q.first * a.q.token + head * a.q.head;
  const char *const pg = a.gout.base + w.sequence * a.gout.batch + w.q.first * a.gout.token + head * a.gout.head;
  const f32x2 *const ps = stats + (w.sequence * (a.q_starts.p ? 0 : a.q_starts.all) + w.q.first) * ((int64_t)a.kv * a.per_kv) + head;
  Pair<T, D, SIDE, WAVES * kWave> next;
  f32x2 next_stat;
  int next_end;
  const auto load = [&](uint32_t at) {
    next.template load<VEC>(
        [&](int row, const char **x, const char **y) {
          const uint32_t r = at + row < end ? at + row : end - 1, query = fast_quotient(r, a.heads_div), g = r - query * a.heads_div.d;
          *x = pq + (int64_t)query * a.q.token + (int64_t)g * a.q.head;
          *y = pg + (int64_t)query * a.gout.token + (int64_t)g * a.gout.head;
          return at + row < end;
        },
        a.q.channel, a.gout.channel, a.channels, threadIdx.x);
    if (threadIdx.x < SIDE) {
      const uint32_t r = at + threadIdx.x < end ? at + threadIdx.x : end - 1, query = fast_quotient(r, a.heads_div), g = r - query * a.heads_div.d;
      next_stat = at + threadIdx.x < end ? ps[(int64_t)query * ((int64_t)a.kv * a.per_kv) + g] : f32x2{-__builtin_inff(), 0.0f};
      next_end = a.causal ? (int)query - ahead + 1 : w.k.count;
    }
  };
  const auto store = [&](int turn) {
    next.store(held + turn * 2 * SIDE * PITCH, held + (turn * 2 + 1) * SIDE * PITCH, threadIdx.x);
    if (threadIdx.x < SIDE) of_row[turn][threadIdx.x] = next_stat, ends[turn][threadIdx.x] = next_end;
  };
  int turn = 0;
  if (begin < end) {
    load(begin);
    store(0);
    __syncthreads();
  }
  for (uint32_t at = begin; at < end; at += SIDE, turn ^= 1) {
    const bool more = end - at > SIDE;
    if (more) load(at + SIDE);
    const char *const q = held + turn * 2 * SIDE * PITCH, *const g = q + SIDE * PITCH;
    // the keys that the first and the last of these rows see up to
    const int first_end = ends[turn][0], last_end = ends[turn][SIDE - 1], from = block + wave * SIDE;
    const bool some = from < last_end && (!a.window || from + SIDE > first_end - a.window);
    if (some) {
      acc_t<T> p = no_sum<T>(), s[1] = {no_sum<T>()};
#pragma unroll
      for (int c = 0; c < D / 16; ++c) p = product(rows_fragment<T, D>(q, 0, c, n, h), k[c], p);
#pragma unroll
      for (int c = 0; c < D / 16; ++c) s[0] = product(rows_fragment<T, D>(g, 0, c, n, h), v[c], s[0]);
      weights_of<T>(p, s[0], a.scale, [&](int i) { return of_row[turn][own_index<T>(i) + 4 * h]; });
      if (from + SIDE > first_end || (a.window && from < last_end - a.window)) {
#pragma unroll
        for (int i = 0; i < OWN; ++i) {
          const int e = ends[turn][own_index<T>(i) + 4 * h];
          if (key >= e || (a.window && key < e - a.window)) p[i] = s[0][i] = 0.0f;
        }
      }
#pragma unroll
      for (int x = 0; x < Tile<T>::kSteps; ++x) {
        const frag_t<T> f = as_fragment<T>(p, x);
#pragma unroll
        for (int ct = 0; ct < D / SIDE; ++ct) gv[ct] = product(columns_fragment<T, D>(g, 16 * x, ct, lane), f, gv[ct]);
      }
      in_range<T, 1>(s, range, gk, D / SIDE);
#pragma unroll
      for (int x = 0; x < Tile<T>::kSteps; ++x) {
        const frag_t<T> f = as_fragment<T>(s[0], x);
#pragma unroll
        for (int ct = 0; ct < D / SIDE; ++ct) gk[ct] = product(columns_fragment<T, D>(q, 16 * x, ct, lane), f, gk[ct]);
      }
    }
    if (more) store(turn ^ 1);
    __syncthreads();
  }
  if (!mine) return;
  const float weight = kWeightTop<T> > 0.0f ? 0x1p-12f : 1.0f;
  store_columns<T, D, VEC>(gk, a.gk.base + w.sequence * a.gk.batch + token * a.gk.token + w.kv * a.gk.head, a.gk.channel, h, a.channels, a.true_scale * weight * range.back());
  store_columns<T, D, VEC>(gv, a.gv.base + w.sequence * a.gv.batch + token * a.gv.token + w.kv * a.gv.head, a.gv.channel, h, a.channels, weight);
}

// Gradients of queries: a wavefront has a tile's side of rows, in registers, with the sums for them; keys and values go through LDS.
template <class T, int D, bool VEC, int WAVES> __global__ __launch_bounds__(WAVES *kWave) void attention_queries_kernel(const AttentionArgs a, uint32_t first_block, const f32x2 *stats) {
  warm_arguments<AttentionArgs>();
  constexpr int SIDE = Tile<T>::kSide, PITCH = Held<T, D>::kPitch, OWN = Tile<T>::kOwn;
  __shared__ __align__(16) char held[2 * 2 * SIDE * PITCH];      // [2][keys, values][SIDE][PITCH]
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, n = lane & (SIDE - 1), h = lane / SIDE;
  Work w;
  if (!find_work(a, first_block + blockIdx.x, &w)) return;
  const RowPlace place = row_place(a, w, wave * SIDE + n);
  const Limits own = limits_of(a, w, place.query), all = limits_of_block(a, w);
  const int64_t token = w.q.first + place.query, head = (int64_t)w.kv * a.per_kv + place.head;
  frag_t<T> q[D / 16], g[D / 16];
  load_fragments<T, D, VEC>(q, a.q.base + w.sequence * a.q.batch + token * a.q.token + head * a.q.head, a.q.channel, place.in && !a.nothing ? a.channels : 0, h, a.negative);
  load_fragments<T, D, VEC>(g, a.gout.base + w.sequence * a.gout.batch + token * a.gout.token + head * a.gout.head, a.gout.channel, place.in ? a.channels : 0, h, false);
  const f32x2 stat = stats[(w.sequence * (a.q_starts.p ? 0 : a.q_starts.all) + token) * ((int64_t)a.kv * a.per_kv) + head];
  acc_t<T> gq[D / SIDE];
#pragma unroll
  for (int ct = 0; ct < D / SIDE; ++ct) gq[ct] = no_sum<T>();
  Range<T> range;
  const int hi_first = __builtin_amdgcn_readfirstlane(own.hi), hi_last = __builtin_amdgcn_readlane(own.hi, SIDE - 1), lo_first = __builtin_amdgcn_readfirstlane(own.lo),
            lo_last = __builtin_amdgcn_readlane(own.lo, SIDE - 1);
  const char *pk = a.k.base + w.sequence * a.k.batch + w.k.first * a.k.token + (int64_t)w.kv * a.k.head, *pv = a.v.base + w.sequence * a.v.batch + w.k.first * a.v.token + (int64_t)w.kv * a.v.head;
  Pair<T, D, SIDE, WAVES * kWave> next;
  const auto load = [&](int at) {
    next.template load<VEC>(
        [&](int row, const char **x, const char **y) {
          const bool in = at + row < w.k.count;
          *x = pk + (int64_t)(in ? at + row : 0) * a.k.token;
          *y = pv + (int64_t)(in ? at + row : 0) * a.v.token;
          return in;
        },
        a.k.channel, a.v.channel, a.channels, threadIdx.x);
  };
  int at = all.lo / SIDE * SIDE, turn = 0;
  if (at < all.hi) {
    load(at);
    next.store(held, held + SIDE * PITCH, threadIdx.x);
    __syncthreads();
  }
  for (; at < all.hi; at += SIDE, turn ^= 1) {
    const bool more = at + SIDE < all.hi;
    if (more) load(at + SIDE);
    const char *const k = held + turn * 2 * SIDE * PITCH, *const v = k + SIDE * PITCH;
    if (at < hi_last && at + SIDE > lo_first) {
      acc_t<T> p = no_sum<T>(), s[1] = {no_sum<T>()};
#pragma unroll
      for (int c = 0; c < D / 16; ++c) p = product(rows_fragment<T, D>(k, 0, c, n, h), q[c], p);
#pragma unroll
      for (int c = 0; c < D / 16; ++c) s[0] = product(rows_fragment<T, D>(v, 0, c, n, h), g[c], s[0]);
      weights_of<T>(p, s[0], a.scale, [&](int) { return stat; });
      if (at + SIDE > hi_first || at < lo_last) {
#pragma unroll
        for (int i = 0; i < OWN; ++i) {
          const int j = at + own_index<T>(i) + 4 * h;
          if (j < own.lo || j >= own.hi) s[0][i] = 0.0f;
        }
      }
      in_range<T, 1>(s, range, gq, D / SIDE);
#pragma unroll
      for (int x = 0; x < Tile<T>::kSteps; ++x) {
        const frag_t<T> f = as_fragment<T>(s[0], x);
#pragma unroll
        for (int ct = 0; ct < D / SIDE; ++ct) gq[ct] = product(columns_fragment<T, D>(k, 16 * x, ct, lane), f, gq[ct]);
      }
    }
    if (more) next.store(held + (turn ^ 1) * 2 * SIDE * PITCH, held + ((turn ^ 1) * 2 + 1) * SIDE * PITCH, threadIdx.x);
    __syncthreads();
  }
  if (!place.in) return;
  const float weight = kWeightTop<T> > 0.0f ? 0x1p-12f : 1.0f;
  store_columns<T, D, VEC>(gq, a.gq.base + w.sequence * a.gq.batch + token * a.gq.token + head * a.gq.head, a.gq.channel, h, a.channels, a.true_scale * weight * range.back());
}

// ---------------------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------------------

template <class Launch> int in_launches(int64_t blocks, Launch launch) {
  for (int64_t at = 0; at < blocks; at += max_launch_blocks()) {
    launch((uint32_t)std::min<int64_t>(blocks - at, max_launch_blocks()), (uint32_t)at);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) {
      record_hip_error((int)e);
      return OCN_ERR_LAUNCH;
    }
  }
  return OCN_OK;
}

template <class T, int D, bool VEC> int run_grad(AttentionArgs &a, const AttentionSizes &sizes, const AttentionGrad &p, f32x2 *stats, hipStream_t stream) {
  const int side = Tile<T>::kSide;
  int rc = OCN_OK;
  const uint32_t rows = (uint32_t)p.rows;
  if (rows) {
    const FastDiv heads = make_fastdiv((uint32_t)(a.kv * a.per_kv)), queries = make_fastdiv((uint32_t)std::max<int64_t>(1, sizes.packed ? sizes.queries : a.q_starts.all));
    hipLaunchKernelGGL((attention_along_kernel<T, VEC>), dim3(std::min<uint32_t>((rows + 15) / 16, 8192)), dim3(kBlock), 0, stream, a, rows, heads, queries, stats);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) {
      record_hip_error((int)e);
      return OCN_ERR_LAUNCH;
    }
  }
  if (p.keys) {
    if (!set_key_blocks(a, sizes, side * kGradWaves)) return OCN_ERR_SHAPE;
    rc = in_launches(key_units_of(sizes, side * kGradWaves), [&](uint32_t grid, uint32_t first) {
      hipLaunchKernelGGL((attention_keys_kernel<T, D, VEC, kGradWaves>), dim3(grid), dim3(kGradWaves * kWave), 0, stream, a, first, stats);
    });
    if (rc != OCN_OK) return rc;
  }
  if (p.queries) {
    if (!set_blocks(a, sizes, side * kGradWaves, 1)) return OCN_ERR_SHAPE;
    rc = in_launches(units_of(sizes, side * kGradWaves), [&](uint32_t grid, uint32_t first) {
      hipLaunchKernelGGL((attention_queries_kernel<T, D, VEC, kGradWaves>), dim3(grid), dim3(kGradWaves * kWave), 0, stream, a, first, stats);
    });
  }
  return rc;
}

template <class T> int run_grad_type(AttentionArgs &a, const AttentionSizes &sizes, const AttentionGrad &p, bool vec, void *workspace, hipStream_t stream) {
#define OCN_RUN(T, D, VEC) return run_grad<T, D, VEC>(a, sizes, p, (f32x2 *)workspace, stream)
  OCN_BY_PADDED(T, a.channels, vec, OCN_RUN);
#undef OCN_RUN
}

}  // namespace
}  // namespace ocn
