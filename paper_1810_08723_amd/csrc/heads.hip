// Operators over the heads of a layer's queries, keys and values: rotary positions, the norm of every head with the
// rotation in the same pass, its gradient, and the cache of 4-bit values: appending to it and reading it back.
//
// All of them read each row (one head of one token) once and write it once: memory bounds them, or, for a few tokens, the
// launch.  Eight channels of a row have a lane, so that a row of 128 channels takes 16 lanes and one 16-byte access each for 16-bit
// types; the lanes of a row lie in one wavefront, and what they need of each other (sums, maxima) goes over it in shuffles.  A channel's
// partner in a rotated pair is loaded a second time, by the lane that needs it: the row's lines are in the vector cache then.
//
// A workgroup takes some tokens with some or all of their heads.  The cosines and sines of a token's pairs are the same
// for all of its heads: the workgroup forms them once in LDS, in double precision (angles of far positions lose everything in
// single: 2^24 radians have a spacing of 2), while its first rows are on their way.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstring>

#include "dev_types.hpp"
#include "head_types.hpp"
#include "heads.hpp"

namespace ocn {
namespace {

constexpr int kTable = 2048;           // channels, of all its tokens, that a workgroup holds factors of
constexpr int kPasses = 4;              // of a workgroup's lanes over its rows, at most
constexpr int kFoldBlocks = 1024;      // workgroups that sum a gradient of weights, at most

// Where the pairs of a lane's eight channels lie.  kPairsInside: among the eight; kPairsEight: the partners of all eight are eight more
// channels in a row; kPairsFour: of each half of them; kPairsOne: anywhere.
enum { kPairsNone = 0, kPairsInside, kPairsEight, kPairsFour, kPairsOne };

// ---------------------------------------------------------------------------------------
// arguments
// ---------------------------------------------------------------------------------------

struct HeadJob {                       // one tensor of heads
  const char *x, *g, *weight;          // input; gradient of the output (backward); weights of the norm
  char *out;
  float *partial;                      // backward: sums for the weights' gradient, [workgroups][channels]; null: not wanted
  int64_t xh, xe, gh, ge, oh, oe;      // strides of heads and channels
  int64_t xl[kMaxLead], gl[kMaxLead], ol[kMaxLead];
  int64_t weight_stride;
  int32_t weight_type;
  bool stream;                         // the output is too large to stay cached
  int32_t heads, per, per_tokens;      // heads of a token; heads and tokens of an item
  FastDiv per_div, blocks_div;         // by `per`; by items along the heads
  uint32_t items;
  int32_t workers;                     // backward: workgroups
};

struct HeadArgs {
  HeadJob job[2];
  Lead lead;
  const char *pos;
  const char *freq;
  int64_t pos_l[kMaxLead], freq_stride;
  int64_t pos_axis, freq_axis;         // strides from axis to axis
  double magnitude;
  float sign;                          // -1: turned back
  float eps, over_d;
  int32_t pos_wide, axes;
  int32_t half, row;                   // pairs of a head; floats of a token in the table
  FastDiv half_div;
  int32_t d, lanes_log2;               // channels; lanes of a row
  int32_t small;                       // one leading dimension, strides and what an item spans in 24 and 31 bits
  uint32_t items, first_item;          // of all launches; of this one
  // the cache
  const char *slots;
  int64_t slot_l[kMaxLead], page_stride, head_stride, slot_count;
  char *cache;
  int32_t slots_wide, page, small_cache;   // the cache's strides in 32 bits
  FastDiv page_div;
};

// The address of head h of a workgroup's token t (from `token` on, which all lanes share).  Products of 64 bits are some twenty times the work
// of one of 24; where strides are small (a.small) only the shared part takes them, in scalar registers.
__device__ __forceinline__ const char *address(const HeadArgs &a, const char *base, const int64_t *stride, uint32_t token, int t, int64_t head_stride, int h) {
  if (a.small) return base + (int64_t)token * stride[0] + (__mul24(t, (int)stride[0]) + __mul24(h, (int)head_stride));
  uint32_t i = token + t;
  int64_t o = h * head_stride;
#pragma nounroll
  for (int d = a.lead.n - 1; d > 0; --d) {
    const uint32_t q = fast_quotient(i, a.lead.div[d]);
    o += (int64_t)(i - q * a.lead.div[d].d) * stride[d];
    i = q;
  }
  return base + (o + (int64_t)i * stride[0]);
}

// ---------------------------------------------------------------------------------------
// cosines and sines
// ---------------------------------------------------------------------------------------

// sin and cos of t: t less a multiple of pi/2 (in two parts, the first 53 bits and the next 53), then the Taylor series up to
// x^15 and x^16, whose remainders on [-pi/4, pi/4] are below 2^-54.
// (The coefficients are kept in scalar registers: the compiler puts them all in vector registers, 32 of them, and the kernels around this lose wavefronts.)
__device__ __forceinline__ double scalar(double x) {
  asm("" : "+s"(x));
  return x;
}
__device__ __forceinline__ void sine_cosine(double t, double *s, double *c) {
  const double n = __builtin_rint(t * scalar(0.63661977236758134308));
  double x = __builtin_fma(-n, scalar(1.57079632679489655800), t);
  x = __builtin_fma(-n, scalar(6.12323399573676603587e-17), x);
  const double z = x * x;
  double p = scalar(-1.0 / 1307674368000.0), q = scalar(1.0 / 20922789888000.0);
  p = __builtin_fma(p, z, scalar(1.0 / 6227020800.0));
  q = __builtin_fma(q, z, scalar(-1.0 / 87178291200.0));
  p = __builtin_fma(p, z, scalar(-1.0 / 39916800.0));
  q = __builtin_fma(q, z, scalar(1.0 / 479001600.0));
  p = __builtin_fma(p, z, scalar(1.0 / 362880.0));
  q = __builtin_fma(q, z, scalar(-1.0 / 3628800.0));
  p = __builtin_fma(p, z, scalar(-1.0 / 5040.0));
  q = __builtin_fma(q, z, scalar(1.0 / 40320.0));
  p = __builtin_fma(p, z, scalar(1.0 / 120.0));
  q = __builtin_fma(q, z, scalar(-1.0 / 720.0));
  p = __builtin_fma(p, z, scalar(-1.0 / 6.0));
  q = __builtin_fma(q, z, scalar(1.0 / 24.0));
  q = __builtin_fma(q, z, -0.5);
  p = __builtin_fma(p * z, x, x);
  q = __builtin_fma(q, z, 1.0);
  const int quarter = (int)(n - 4.0 * __builtin_floor(n * 0.25));
  const double a = quarter & 1 ? q : p, b = quarter & 1 ? p : q;
  *s = quarter & 2 ? -a : a;
  *c = (quarter + 1) & 2 ? -b : b;
}

// For each of the channels that rotate, of each token of an item: what the channel and its partner in the pair are multiplied by.  (Weights of a norm
// are in them already, and the signs: a channel takes two products and a sum.)
struct alignas(16) Table { float own[kTable], other[kTable]; };

template <int KIND> __device__ __forceinline__ void fill_table(const HeadArgs &a, const HeadJob &j, Table &tab, uint32_t token, int tokens, bool weights) {
#pragma nounroll
  for (int i = threadIdx.x; i < tokens * a.half; i += kBlock) {
    const int t = (int)fast_quotient((uint32_t)i, a.half_div), p = i - t * a.half;
    const char *pos = address(a, a.pos, a.pos_l, token, t, 0, 0), *freq = a.freq + p * a.freq_stride;
    double angle = (double)load_index(pos, a.pos_wide) * *(const double *)freq, s, c;
#pragma nounroll
    for (int k = 1; k < a.axes; ++k)
      angle = __builtin_fma((double)load_index(pos + k * a.pos_axis, a.pos_wide), *(const double *)(freq + k * a.freq_axis), angle);
    sine_cosine(angle, &s, &c);
    const float cc = (float)(c * a.magnitude), ss = (float)(s * a.magnitude) * a.sign;
    const int one = KIND == kPairsInside ? 2 * p : p, two = KIND == kPairsInside ? 2 * p + 1 : p + a.half;
    float w1 = 1.0f, w2 = 1.0f;
    if (weights && j.weight) {
      w1 = load_as_float(j.weight + one * j.weight_stride, j.weight_type);
      w2 = load_as_float(j.weight + two * j.weight_stride, j.weight_type);
    }
    tab.own[t * a.row + one] = cc * w1;
    tab.other[t * a.row + one] = -ss * w2;
    tab.own[t * a.row + two] = cc * w2;
    tab.other[t * a.row + two] = ss * w1;
  }
}

// ---------------------------------------------------------------------------------------
// rows
// ---------------------------------------------------------------------------------------

template <class T> struct Four { typedef T V __attribute__((ext_vector_type(4))); };

// the other channels of the pairs that channels e ... e + 7 belong to (channel i < half goes with i + half), where they lie apart
template <class T, int KIND> __device__ __forceinline__ eight_t<T> load_partners(const char *row, int64_t step, int e, int half) {
  eight_t<T> v = {};
  if constexpr (KIND == kPairsEight) {
    if (e < 2 * half) v = *(const eight_t<T> *)(row + (e < half ? e + half : e - half) * (int)sizeof(T));
  } else if constexpr (KIND == kPairsFour) {
#pragma unroll
    for (int k = 0; k < kEight; k += 4) {
      const int f = e + k;
      if (f < 2 * half) {
        const typename Four<T>::V w = *(const typename Four<T>::V *)(row + (f < half ? f + half : f - half) * (int)sizeof(T));
#pragma unroll
        for (int i = 0; i < 4; ++i) v[k + i] = w[i];
      }
    }
  } else if constexpr (KIND == kPairsOne) {
#pragma unroll
    for (int i = 0; i < kEight; ++i) {
      const int f = e + i;
      if (f < 2 * half) v[i] = *(const T *)(row + (f < half ? f + half : f - half) * step);
    }
  }
  return v;
}

// x turned, with the row's part of the table; p: the partners of pairs that lie apart
template <int KIND> __device__ __forceinline__ void turn(float *x, const float *p, const float *own, const float *other, int e, int half) {
  if constexpr (KIND == kPairsNone) return;
  if (e >= 2 * half) return;
  float q[kEight];
#pragma unroll
  for (int i = 0; i < kEight; ++i) q[i] = KIND == kPairsInside ? x[i ^ 1] : p[i];
  // (a token's part of the table is padded to eights)
  f32x4 a[2], b[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) a[k] = *(const f32x4 *)(own + e + 4 * k), b[k] = *(const f32x4 *)(other + e + 4 * k);
#pragma unroll
  for (int i = 0; i < kEight; ++i)
    if (KIND == kPairsEight || e + i < 2 * half) x[i] = x[i] * a[i / 4][i % 4] + q[i] * b[i / 4][i % 4];
}

struct Item { int which, tokens, head; uint32_t token; };

// a workgroup's tokens and heads
__device__ __forceinline__ Item item_of(const HeadArgs &a, uint32_t i) {
  Item r;
  r.which = i >= a.job[0].items;
  const HeadJob &j = a.job[r.which];
  if (r.which) i -= a.job[0].items;
  const uint32_t block = fast_quotient(i, j.blocks_div);
  r.head = (int)(i - block * j.blocks_div.d) * j.per;
  r.token = block * j.per_tokens;
  r.tokens = (int)min((uint32_t)j.per_tokens, a.lead.tokens - r.token);
  return r;
}

// Rotation, with the norm before it where NORM is set.  (No loop over items in the kernel: what their first instructions share would be kept in registers;
// launches take up to as many as a launch may have.)  Two prompts of 4096 tokens, 32 heads of 128 channels in bfloat16, rotated: 134 MB in 23.0 us; 8192 tokens of
// 40 heads with the norm: 168 MB in 46.7 us (a large copy: 32), as its workgroups wait for positions, sines and rows in turn.  Four rows of a lane at a time: 51.9.
template <class T, bool VEC, int KIND, bool NORM> __global__ __launch_bounds__(kBlock) void head_rows_kernel(const HeadArgs a) {
  warm_arguments<HeadArgs>();
  constexpr int U = 2;                  // rows of a lane at a time
  __shared__ Table tab;
  const int lanes = 1 << a.lanes_log2, e = (threadIdx.x & (lanes - 1)) * kEight, rows = kBlock >> a.lanes_log2, d = a.d;
  const Item item = item_of(a, a.first_item + blockIdx.x);
  const HeadJob &j = a.job[item.which];
  const int total = item.tokens * j.per;
  float w[kEight];                      // of channels that do not rotate
  for (int base = 0; base < total; base += U * rows) {
    eight_t<T> x[U], p[U];
    char *to[U];
    int tt[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = base + u * rows + (threadIdx.x >> a.lanes_log2), t = (int)fast_quotient((uint32_t)r, j.per_div), h = item.head + r - t * j.per;
      to[u] = nullptr;
      tt[u] = t;
      if (r < total && h < j.heads && e < d) {
        const char *row = address(a, j.x, j.xl, item.token, t, j.xh, h);
        x[u] = load_eight<T, VEC>(row, j.xe, e, d);
        p[u] = load_partners<T, KIND>(row, j.xe, e, a.half);
        to[u] = (char *)address(a, j.out, j.ol, item.token, t, j.oh, h);
      }
    }
    if (base == 0) {
      if constexpr (NORM) {
#pragma unroll
        for (int i = 0; i < kEight; ++i)
          w[i] = j.weight && e + i >= 2 * a.half && e + i < d ? load_as_float(j.weight + (e + i) * j.weight_stride, j.weight_type) : 1.0f;
      }
      if constexpr (KIND != kPairsNone) {
        fill_table<KIND>(a, j, tab, item.token, item.tokens, NORM);
        __syncthreads();
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float v[kEight], q[kEight], r = 1.0f;
      if constexpr (NORM) {
        float sum = 0.0f;
        if (to[u]) {
#pragma unroll
          for (int i = 0; i < kEight; ++i) sum = __builtin_fmaf((float)x[u][i], (float)x[u][i], sum);
        }
        r = __builtin_amdgcn_rsqf(sum_over_row(sum, lanes) * a.over_d + a.eps);
      }
      if (!to[u]) continue;
#pragma unroll
      for (int i = 0; i < kEight; ++i) {
        v[i] = (float)x[u][i];
        q[i] = (float)p[u][i];
        if constexpr (NORM) {
          v[i] = v[i] * r * w[i];
          q[i] = q[i] * r;
        }
      }
      turn<KIND>(v, q, tab.own + tt[u] * a.row, tab.other + tt[u] * a.row, e, a.half);
      store_eight<T, VEC>(to[u], j.oe, e, d, v, j.stream);
    }
  }
}

// Gradient of the norm with the rotation.  With h = the gradient turned back, u = x r, r = 1 / sqrt(mean(x^2) + eps):
//     gradient of x = r (h w - u mean(h w u)),    gradient of w = the sum of h u over all rows.
// A lane keeps its channels' sums over all rows of its workgroup; workgroups leave theirs in the workspace, and a second launch
// adds those up in a fixed order: no atomics, the same bits every time.  8002 tokens of 24 heads (147 MB): 43.7 us, 4.6 of them the second launch.
template <class T, bool VEC, int KIND> __global__ __launch_bounds__(kBlock) void head_grad_kernel(const HeadArgs a) {
  warm_arguments<HeadArgs>();
  __shared__ Table tab;
  static_assert(kTable >= kBlock * kEight, "the sums take the table's place");
  float *const sums = tab.own;
  const int lanes = 1 << a.lanes_log2, e = (threadIdx.x & (lanes - 1)) * kEight, rows = kBlock >> a.lanes_log2, d = a.d;
  // a workgroup's items are of one job: blockIdx.y
  const HeadJob &j = a.job[blockIdx.y];
  if (blockIdx.x >= (uint32_t)j.workers) return;
  float w[kEight], gw[kEight];
#pragma unroll
  for (int i = 0; i < kEight; ++i) {
    gw[i] = 0.0f;
    w[i] = j.weight && e + i < d ? load_as_float(j.weight + (e + i) * j.weight_stride, j.weight_type) : 1.0f;
  }
  for (uint32_t it = blockIdx.x; it < j.items; it += j.workers) {
    const Item item = item_of(a, it + (blockIdx.y ? a.job[0].items : 0));
    const int total = item.tokens * j.per;
    // two rows of a lane are on their way while it works on one
    eight_t<T> x[2], g[2], p[2];
    const auto load = [&](int base, int u) {
      const int r = base + (threadIdx.x >> a.lanes_log2), t = (int)fast_quotient((uint32_t)r, j.per_div), n = item.head + r - t * j.per;
      if (r < total && n < j.heads && e < d) {
        const char *row = address(a, j.g, j.gl, item.token, t, j.gh, n);
        x[u] = load_eight<T, VEC>(address(a, j.x, j.xl, item.token, t, j.xh, n), j.xe, e, d);
        g[u] = load_eight<T, VEC>(row, j.ge, e, d);
        p[u] = load_partners<T, KIND>(row, j.ge, e, a.half);
      }
    };
    load(0, 0);
    load(rows, 1);
    if constexpr (KIND != kPairsNone) {
      fill_table<KIND>(a, j, tab, item.token, item.tokens, false);
      __syncthreads();
    }
    for (int both = 0; both < total; both += 2 * rows) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int base = both + u * rows, r = base + (threadIdx.x >> a.lanes_log2), t = (int)fast_quotient((uint32_t)r, j.per_div), n = item.head + r - t * j.per;
        const bool mine = r < total && n < j.heads && e < d;
        float v[kEight], h[kEight], square = 0.0f, cross = 0.0f;
        if (mine) {
          float q[kEight];
#pragma unroll
          for (int i = 0; i < kEight; ++i) v[i] = (float)x[u][i], h[i] = (float)g[u][i], q[i] = (float)p[u][i];
          turn<KIND>(h, q, tab.own + t * a.row, tab.other + t * a.row, e, a.half);
#pragma unroll
          for (int i = 0; i < kEight; ++i) {
            square = __builtin_fmaf(v[i], v[i], square);
            cross = __builtin_fmaf(h[i] * w[i], v[i], cross);
          }
        }
        load(base + 2 * rows, u);
        square = sum_over_row(square, lanes);
        cross = sum_over_row(cross, lanes);
        if (mine) {
          const float over = __builtin_amdgcn_rsqf(square * a.over_d + a.eps), mean = cross * over * a.over_d;
#pragma unroll
          for (int i = 0; i < kEight; ++i) {
            const float unit = v[i] * over;
            gw[i] = __builtin_fmaf(h[i], unit, gw[i]);
            v[i] = over * (h[i] * w[i] - unit * mean);
          }
          store_eight<T, VEC>((char *)address(a, j.out, j.ol, item.token, t, j.oh, n), j.oe, e, d, v, j.stream);
        }
      }
    }
    __syncthreads();
  }
  if (!j.partial) return;
#pragma unroll
  for (int i = 0; i < kEight; ++i) sums[threadIdx.x * kEight + i] = gw[i];
  __syncthreads();
  for (int c = threadIdx.x; c < d; c += kBlock) {
    float s = 0.0f;
    for (int r = 0; r < rows; ++r) s += sums[r * lanes * kEight + c];
    j.partial[(int64_t)blockIdx.x * d + c] = s;
  }
}

constexpr int kFoldLanes = 1024;

struct FoldArgs {
  const float *partial[2];
  char *out[2];
  int64_t stride[2];
  int32_t type[2], d, count[2];
};

// eight channels of a job have a workgroup; sums of sums in double precision
__global__ __launch_bounds__(kFoldLanes) void head_fold_kernel(const FoldArgs a) {
  __shared__ double part[kFoldLanes / 8][8];
  const int which = blockIdx.y, lane = threadIdx.x & 7, row = threadIdx.x >> 3, c = blockIdx.x * 8 + lane;
  if (!a.out[which]) return;
  double s = 0.0;
  if (c < a.d) {
#pragma unroll 8
    for (int i = row; i < a.count[which]; i += kFoldLanes / 8) s += a.partial[which][(int64_t)i * a.d + c];
  }
  part[row][lane] = s;
  for (int half = kFoldLanes / 16; half > 0; half /= 2) {
    __syncthreads();
    if (row < half) part[row][lane] += part[row + half][lane];
  }
  if (row == 0 && c < a.d) store_from_float(a.out[which] + c * a.stride[which], a.type[which], (float)part[0][lane]);
}

// ---------------------------------------------------------------------------------------
// the cache
// ---------------------------------------------------------------------------------------

struct Slot { int64_t page; int place; };
// (slots within 2^31 are divided in 32 bits)
__device__ __forceinline__ Slot slot_of(const HeadArgs &a, int64_t slot) {
  Slot s;
  s.page = slot < 0x7fffffff ? (int64_t)fast_quotient((uint32_t)slot, a.page_div) : slot / a.page;
  s.place = (int)(slot - s.page * a.page);
  return s;
}

__device__ __forceinline__ char *block_of(const HeadArgs &a, int64_t page, int h) {
  if (a.small_cache) return a.cache + ((uint64_t)(uint32_t)page * (uint32_t)a.page_stride + (uint64_t)(uint32_t)h * (uint32_t)a.head_stride);
  return a.cache + page * a.page_stride + h * a.head_stride;
}

// nine significant bits of a float, ties to even, as a half
__device__ __forceinline__ f16 nine_bits(float m) {
  const uint32_t b = __builtin_bit_cast(uint32_t, m);
  return (f16)__builtin_bit_cast(float, (b + 0x3fff + ((b >> 15) & 1)) & 0xffff8000u);
}

// Keys and values into the cache: job 0 the keys, job 1 the values.  A group's 32 channels are four lanes'.  Each lane's eight codes are four
// bytes of a token's row; the conversion of two floats to two codes is one instruction and rounds to nearest even.  8331 tokens of 8 heads of 64 channels:
// 13 us (17 MB in, 5 MB out): V's codes go out in pieces of two bytes; reading them back takes 9.
template <class T, bool VEC, int KIND> __global__ __launch_bounds__(kBlock) void cache_append_kernel(const HeadArgs a) {
  warm_arguments<HeadArgs>();
  __shared__ Table tab;
  const int lanes = 1 << a.lanes_log2, e = (threadIdx.x & (lanes - 1)) * kEight, rows = kBlock >> a.lanes_log2, d = a.d;
  const Item item = item_of(a, a.first_item + blockIdx.x);
  const HeadJob &j = a.job[item.which];
  const int total = item.tokens * j.per;
  constexpr int U = 2;                   // rows of a lane at a time
  for (int base = 0; base < total; base += U * rows) {
    eight_t<T> x[U], p[U];
    int64_t slots[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = base + u * rows + (threadIdx.x >> a.lanes_log2), t = (int)fast_quotient((uint32_t)r, j.per_div), h = item.head + r - t * j.per;
      slots[u] = -1;
      if (r < total && h < j.heads) {
        const char *row = address(a, j.x, j.xl, item.token, t, j.xh, h);
        slots[u] = load_index(address(a, a.slots, a.slot_l, item.token, t, 0, 0), a.slots_wide);
        x[u] = load_eight<T, VEC>(row, j.xe, e, d);
        if (!item.which) p[u] = load_partners<T, KIND>(row, j.xe, e, a.half);
      }
    }
    if (KIND != kPairsNone && base == 0 && !item.which) {
      fill_table<KIND>(a, j, tab, item.token, item.tokens, false);
      __syncthreads();
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = base + u * rows + (threadIdx.x >> a.lanes_log2), t = (int)fast_quotient((uint32_t)r, j.per_div), h = item.head + r - t * j.per;
      const int64_t slot = slots[u];
      float v[kEight];
      uint32_t bits = 0;                     // of the largest magnitude: as whole numbers, infinities are above all others and NaNs above them
      const bool mine = slot >= 0 && slot < a.slot_count;
      if (mine) {
#pragma unroll
        for (int i = 0; i < kEight; ++i) v[i] = (float)x[u][i];
        if (!item.which) {
          float q[kEight];
#pragma unroll
          for (int i = 0; i < kEight; ++i) q[i] = (float)p[u][i];
          turn<KIND>(v, q, tab.own + t * a.row, tab.other + t * a.row, e, a.half);
        }
#pragma unroll
        for (int i = 0; i < kEight; ++i) bits = max(bits, __builtin_bit_cast(uint32_t, v[i]) & 0x7fffffffu);
      }
      bits = max(bits, other_lane_bits<0xb1>(bits));
      bits = max(bits, other_lane_bits<0x4e>(bits));
      if (!mine) continue;
      const f16 scale = bits >= 0x7f800000u ? (f16)__builtin_nanf("") : nine_bits(fminf(__builtin_bit_cast(float, bits) * (float)(1.0 / 12.0), 5456.0f));
      // x / scale, correctly rounded: the reciprocal's quotient and one step with the exact remainder.  (Zeros get their signs back; beyond +-12
      // the conversion saturates.)
      const float s = (float)scale, inverse = s > 0.0f ? 1.0f / s : 0.0f;
      uint32_t codes = 0;
      float y[kEight];
#pragma unroll
      for (int i = 0; i < kEight; ++i) {
        const float y0 = v[i] * inverse;
        y[i] = __builtin_copysignf(__builtin_fmaf(__builtin_fmaf(-y0, s, v[i]), inverse, y0), v[i]);
      }
      codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, y[0], y[1], 2.0f, 0);
      codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, y[2], y[3], 2.0f, 1);
      codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, y[4], y[5], 2.0f, 2);
      codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, y[6], y[7], 2.0f, 3);
      const Slot at = slot_of(a, slot);
      char *block = block_of(a, at.page, h);
      if (!item.which) {
        *(uint32_t *)(block + block_k_codes(a.page, d, at.place, e)) = codes;
      } else if (d == 64) {      // (four channels of a token lie together)
        *(uint16_t *)(block + block_v_codes(a.page, d, at.place, e)) = (uint16_t)codes;
        *(uint16_t *)(block + block_v_codes(a.page, d, at.place, e + 4)) = (uint16_t)(codes >> 16);
      } else {
        *(uint32_t *)(block + block_v_codes(a.page, d, at.place, e)) = codes;
      }
      if (e % 32 == 0) *(f16 *)(block + block_scale(a.page, d, item.which != 0, e / 32, at.place)) = scale;
    }
  }
}

// The values at slots: job 0 the keys, job 1 the values.
template <class T, bool VEC> __global__ __launch_bounds__(kBlock) void cache_read_kernel(const HeadArgs a) {
  warm_arguments<HeadArgs>();
  const int lanes = 1 << a.lanes_log2, e = (threadIdx.x & (lanes - 1)) * kEight, rows = kBlock >> a.lanes_log2, d = a.d;
  const Item item = item_of(a, a.first_item + blockIdx.x);
  const HeadJob &j = a.job[item.which];
  const int total = item.tokens * j.per;
  for (int r = threadIdx.x >> a.lanes_log2; r < total; r += rows) {
    const int t = (int)fast_quotient((uint32_t)r, j.per_div), h = item.head + r - t * j.per;
    if (h >= j.heads) continue;
    const int64_t slot = load_index(address(a, a.slots, a.slot_l, item.token, t, 0, 0), a.slots_wide);
    if (slot < 0 || slot >= a.slot_count) continue;
    const Slot at = slot_of(a, slot);
    const char *block = block_of(a, at.page, h);
    uint32_t codes;
    if (!item.which)
      codes = *(const uint32_t *)(block + block_k_codes(a.page, d, at.place, e));
    else if (d == 64)
      codes = *(const uint16_t *)(block + block_v_codes(a.page, d, at.place, e)) |
              (uint32_t)*(const uint16_t *)(block + block_v_codes(a.page, d, at.place, e + 4)) << 16;
    else
      codes = *(const uint32_t *)(block + block_v_codes(a.page, d, at.place, e));
    const float s = (float)*(const f16 *)(block + block_scale(a.page, d, item.which != 0, e / 32, at.place));
    const f16x2 c0 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, 2.0f, 0), c1 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, 2.0f, 1);
    const f16x2 c2 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, 2.0f, 2), c3 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, 2.0f, 3);
    const float v[kEight] = {(float)c0.x * s, (float)c0.y * s, (float)c1.x * s, (float)c1.y * s,
                             (float)c2.x * s, (float)c2.y * s, (float)c3.x * s, (float)c3.y * s};
    store_eight<T, VEC>((char *)address(a, j.out, j.ol, item.token, t, j.oh, h), j.oe, e, d, v, j.stream);
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

int64_t channels_of(const ocn_tensor *t) { return t->size[t->ndim - 1]; }
int64_t heads_of(const ocn_tensor *t) { return t->size[t->ndim - 2]; }

int64_t tokens_of(const ocn_tensor *t) {
  int64_t n = 1;
  for (int d = 0; d + 2 < t->ndim; ++d) n = t->size[d] > 0 && n > ((int64_t)1 << 31) / t->size[d] ? (int64_t)1 << 31 : n * t->size[d];
  return n;
}

int check_heads(const ocn_tensor *t) {
  const int rc = check_operand(t, kHeadTypes);
  if (rc != OCN_OK) return rc;
  if (t->ndim < 2) return OCN_ERR_NDIM;
  if (channels_of(t) > OCN_MAX_CHANNELS) return OCN_ERR_SHAPE;
  if (heads_of(t) >= ((int64_t)1 << 24)) return OCN_ERR_SHAPE;
  return OCN_OK;
}

bool same_shape(const ocn_tensor *a, const ocn_tensor *b) {
  if (a->ndim != b->ndim) return false;
  for (int d = 0; d < a->ndim; ++d)
    if (a->size[d] != b->size[d]) return false;
  return true;
}


// whole vectors of eight channels, each at a multiple of its size (or of 16 bytes)
bool whole_vectors(const ocn_tensor *t) {
  const int64_t size = head_type_size(t->dtype);
  if (channels_of(t) % kEight != 0 || (channels_of(t) > 1 && t->stride[t->ndim - 1] != size)) return false;
  if (((intptr_t)t->base + t->offset) % 16 != 0) return false;
  for (int d = 0; d + 1 < t->ndim; ++d)
    if (t->size[d] > 1 && t->stride[d] % 16 != 0) return false;
  return true;
}

int kind_of_pairs(const ocn_rotation *r, bool vec) {
  if (!r) return kPairsNone;
  if (r->layout == OCN_ROTARY_INTERLEAVED) return kPairsInside;
  const int half = r->rotary_dim / 2;
  return !vec ? kPairsOne : half % 8 == 0 ? kPairsEight : half % 4 == 0 ? kPairsFour : kPairsOne;
}

// the positions on one axis, as they broadcast
ocn_tensor one_axis(const ocn_rotation *r) {
  ocn_tensor t;
  std::memset(&t, 0, sizeof t);
  if (!r) return t;
  t = *r->positions;
  if (r->frequencies->ndim == 1) return t;
  --t.ndim;
  for (int d = 0; d < t.ndim; ++d) t.size[d] = r->positions->size[d + 1], t.stride[d] = r->positions->stride[d + 1];
  return t;
}

// what does not hang on the tensors' addresses: rotation, lanes, and how the tokens and heads go to items
// (false where there are too many items for the kernels' 31 bits)
bool shape_of_launch(HeadArgs &a, const ocn_rotation *r, int64_t d, int jobs) {
  a.d = (int32_t)d;
  a.over_d = 1.0f / (float)d;
  a.lanes_log2 = 0;
  while ((kEight << a.lanes_log2) < d) ++a.lanes_log2;
  a.half = r ? r->rotary_dim / 2 : 0;
  a.row = (2 * a.half + 7) & ~7;
  a.half_div = make_fastdiv((uint32_t)std::max(a.half, 1));
  if (r) {
    a.magnitude = r->magnitude;
    a.pos = (const char *)r->positions->base + r->positions->offset;
    a.pos_wide = r->positions->dtype == OCN_INT64;
    a.freq = (const char *)r->frequencies->base + r->frequencies->offset;
    a.axes = rotation_axes(r);
    a.freq_stride = r->frequencies->stride[r->frequencies->ndim - 1];
    if (a.axes > 1) a.pos_axis = r->positions->stride[0], a.freq_axis = r->frequencies->stride[0];
  }
  // Rows of an item: up to kPasses passes of the workgroup's lanes share the cosines, fewer where that leaves CUs without work.
  const int rows = kBlock >> a.lanes_log2;
  int64_t all = 0, want = kPasses * rows, items = 0;
  for (int i = 0; i < jobs; ++i) all += (int64_t)a.lead.tokens * a.job[i].heads;
  while (want > rows && all / want < 4 * kNumCUs) want /= 2;
  const int64_t most_tokens = r ? std::max<int64_t>(1, kTable / a.row) : 64;
  for (int i = 0; i < jobs; ++i) {
    HeadJob &j = a.job[i];
    const int64_t parts = std::max<int64_t>(1, (j.heads + want - 1) / want);
    j.per = (int32_t)std::max<int64_t>(1, (j.heads + parts - 1) / parts);
    j.per_tokens = (int32_t)std::min<int64_t>(most_tokens, std::max<int64_t>(1, (want + j.per / 2) / j.per));
    const int64_t blocks = ((int64_t)a.lead.tokens + j.per_tokens - 1) / j.per_tokens, across = j.heads ? (j.heads + j.per - 1) / j.per : 0;
    j.per_div = make_fastdiv((uint32_t)j.per);
    j.blocks_div = make_fastdiv((uint32_t)std::max<int64_t>(across, 1));
    j.items = (uint32_t)(blocks * across);
    items += blocks * across;
  }
  // 24-bit products: counts and strides below 2^23, and what an item's tokens and a token's heads span below 2^30 each
  const auto fits = [](int64_t stride, int64_t count) {
    const int64_t s = stride < 0 ? -stride : stride;
    return s < (1 << 23) && count < (1 << 23) && s * count < (1 << 30);
  };
  a.small = a.lead.n == 1;
  for (int i = 0; i < jobs; ++i) {
    const HeadJob &j = a.job[i];
    a.small = a.small && fits(a.pos_l[0], j.per_tokens) && fits(a.slot_l[0], j.per_tokens) && fits(j.xl[0], j.per_tokens) && fits(j.gl[0], j.per_tokens) && fits(j.ol[0], j.per_tokens) && fits(j.xh, j.heads) &&
              fits(j.gh, j.heads) && fits(j.oh, j.heads);
  }
  a.items = (uint32_t)items;
  return items < ((int64_t)1 << 31);
}

void set_rows(HeadJob &j, const ocn_tensor *x, const ocn_tensor *g, const ocn_tensor *out) {
  if (x) { j.x = (const char *)x->base + x->offset; j.xh = x->stride[x->ndim - 2]; j.xe = x->stride[x->ndim - 1]; }
  if (g) { j.g = (const char *)g->base + g->offset; j.gh = g->stride[g->ndim - 2]; j.ge = g->stride[g->ndim - 1]; }
  if (out) j.stream = (int64_t)tokens_of(out) * heads_of(out) * channels_of(out) * head_type_size(out->dtype) >= kStreamBytes;
  if (out) { j.out = (char *)out->base + out->offset; j.oh = out->stride[out->ndim - 2]; j.oe = out->stride[out->ndim - 1]; }
}

int check_weight(const ocn_tensor *w, int64_t channels) {
  if (!w) return OCN_OK;
  const int rc = check_operand(w, kHeadTypes);
  if (rc != OCN_OK) return rc;
  return w->ndim != 1 || w->size[0] != channels ? OCN_ERR_SHAPE : OCN_OK;
}

// CALL(type, whole vectors, kind of pairs) for a launch's
#define OCN_BY_KIND(T, vec, k, CALL)                        \
  do {                                                      \
    if (vec) {                                              \
      if ((k) == kPairsNone) CALL(T, true, kPairsNone);  \
      else if ((k) == kPairsInside) CALL(T, true, kPairsInside); \
      else if ((k) == kPairsEight) CALL(T, true, kPairsEight);   \
      else if ((k) == kPairsFour) CALL(T, true, kPairsFour);     \
      else CALL(T, true, kPairsOne);                        \
    } else {                                                \
      if ((k) == kPairsNone) CALL(T, false, kPairsNone); \
      else if ((k) == kPairsInside) CALL(T, false, kPairsInside); \
      else CALL(T, false, kPairsOne);                       \
    }                                                       \
  } while (0)
#define OCN_BY_TYPE(dtype, vec, kind, CALL)                             \
  do {                                                                  \
    const int pairs_ = (kind);                                          \
    if ((dtype) == OCN_HALF) OCN_BY_KIND(f16, vec, pairs_, CALL);       \
    else if ((dtype) == OCN_BFLOAT16) OCN_BY_KIND(bf16, vec, pairs_, CALL); \
    else OCN_BY_KIND(float, vec, pairs_, CALL);                         \
  } while (0)

// `launch` for all items, as many at a time as a launch may have
template <class Launch> int for_all_items(HeadArgs &a, Launch launch) {
  for (int64_t at = 0; at < a.items; at += max_launch_blocks()) {
    a.first_item = (uint32_t)at;
    launch((uint32_t)std::min<int64_t>(a.items - at, max_launch_blocks()));
    const int rc = done(hipGetLastError());
    if (rc != OCN_OK) return rc;
  }
  return OCN_OK;
}

int run_rows(bool norm, const ocn_tensor *const *x, const ocn_tensor *const *w, const ocn_tensor *const *out, int jobs, double eps,
             const ocn_rotation *r, bool back, hipStream_t stream) {
  HeadOperand ops[8];
  int n = 0, rc;
  for (int i = 0; i < jobs; ++i) {
    if ((rc = check_heads(x[i])) != OCN_OK || (rc = check_heads(out[i])) != OCN_OK) return rc;
    if (out[i]->dtype != x[i]->dtype || x[i]->dtype != x[0]->dtype) return OCN_ERR_DTYPE;
    if (!same_shape(x[i], out[i]) || channels_of(x[i]) != channels_of(x[0])) return OCN_ERR_SHAPE;
    if (norm && (rc = check_weight(w[i], channels_of(x[i]))) != OCN_OK) return rc;
  }
  if ((rc = check_rotation(r, channels_of(x[0]), x[0]->device)) != OCN_OK) return rc;
  for (int i = 0; i < jobs; ++i) {
    ops[n++] = {x[i], false};
    ops[n] = {out[i], true, n - 1};
    ++n;
    if (norm && w[i]) ops[n++] = {w[i], false};
  }
  if (r) {
    ops[n++] = {r->positions, false};
    ops[n++] = {r->frequencies, false};
  }
  if ((rc = check_operands(ops, n)) != OCN_OK) return rc;
  HeadArgs a;
  std::memset(&a, 0, sizeof a);
  const ocn_tensor of_axis = one_axis(r);
  const ocn_tensor *with[5] = {x[0], out[0], jobs > 1 ? x[1] : nullptr, jobs > 1 ? out[1] : nullptr, r ? &of_axis : nullptr};
  const int inner[5] = {2, 2, 2, 2, 0};
  int64_t strides[5][kMaxLead];
  if (jobs > 1) {
    if (x[1]->ndim != x[0]->ndim) return OCN_ERR_SHAPE;
    for (int d = 0; d + 2 < x[0]->ndim; ++d)
      if (x[0]->size[d] != x[1]->size[d]) return OCN_ERR_SHAPE;
  }
  if ((rc = merge_lead(x[0], 2, with, inner, 5, &a.lead, strides)) != OCN_OK) return rc;
  bool vec = true;
  for (int i = 0; i < jobs; ++i) {
    HeadJob &j = a.job[i];
    set_rows(j, x[i], nullptr, out[i]);
    std::memcpy(j.xl, strides[2 * i], sizeof j.xl);
    std::memcpy(j.ol, strides[2 * i + 1], sizeof j.ol);
    j.heads = (int32_t)heads_of(x[i]);
    if (norm && w[i]) {
      j.weight = (const char *)w[i]->base + w[i]->offset;
      j.weight_stride = w[i]->stride[0];
      j.weight_type = w[i]->dtype;
    }
    vec = vec && whole_vectors(x[i]) && whole_vectors(out[i]);
  }
  std::memcpy(a.pos_l, strides[4], sizeof a.pos_l);
  if (channels_of(x[0]) == 0 || a.lead.tokens == 0) return OCN_OK;
  if (!shape_of_launch(a, r, channels_of(x[0]), jobs)) return OCN_ERR_SHAPE;
  if (a.items == 0) return OCN_OK;
  a.eps = (float)eps;
  a.sign = back ? -1.0f : 1.0f;
  const int kind = kind_of_pairs(r, vec);
  return for_all_items(a, [&](uint32_t grid) {
#define OCN_ROWS(T, VEC, KIND)                                                                                           \
  do {                                                                                                                   \
    if (norm) hipLaunchKernelGGL((head_rows_kernel<T, VEC, KIND, true>), dim3(grid), dim3(kBlock), 0, stream, a);         \
    else if constexpr (KIND != kPairsNone) hipLaunchKernelGGL((head_rows_kernel<T, VEC, KIND, false>), dim3(grid), dim3(kBlock), 0, stream, a); \
  } while (0)
    OCN_BY_TYPE(x[0]->dtype, vec, kind, OCN_ROWS);
#undef OCN_ROWS
  });
}

// k, v, slots and cache of ocn_cache_append (out: false) and ocn_cache_read (true); either of k and v may be null in the latter
int run_cache(const ocn_tensor *k, const ocn_tensor *v, const ocn_rotation *r, const ocn_tensor *slots, const ocn_tensor *cache, bool out,
              hipStream_t stream) {
  const ocn_tensor *x[2] = {k, v};
  int rc;
  if ((rc = check_operand(slots, kIndexTypes)) != OCN_OK) return rc;
  HeadOperand ops[8];
  int n = 0;
  const ocn_tensor *first = nullptr;
  for (int i = 0; i < 2; ++i) {
    if (out && !x[i]) continue;
    if ((rc = check_heads(x[i])) != OCN_OK) return rc;
    if (!first) first = x[i];
    if (x[i]->dtype != first->dtype) return OCN_ERR_DTYPE;
    if (!same_shape(x[i], first)) return OCN_ERR_SHAPE;
    ops[n++] = {x[i], out};
  }
  if (!first) return OCN_ERR_NULLPTR;
  const int64_t d = channels_of(first);
  int64_t page;
  if ((rc = check_cache(cache, d, heads_of(first), &page)) != OCN_OK) return rc;
  if ((rc = check_rotation(r, d, first->device)) != OCN_OK) return rc;
  if (slots->ndim != first->ndim - 2) return OCN_ERR_SHAPE;
  for (int i = 0; i < slots->ndim; ++i)
    if (slots->size[i] != first->size[i]) return OCN_ERR_SHAPE;
  ops[n++] = {slots, false};
  ops[n++] = {cache, !out};
  if (r) {
    ops[n++] = {r->positions, false};
    ops[n++] = {r->frequencies, false};
  }
  if ((rc = check_operands(ops, n)) != OCN_OK) return rc;
  HeadArgs a;
  std::memset(&a, 0, sizeof a);
  const ocn_tensor of_axis = one_axis(r);
  const ocn_tensor *with[4] = {k, v, slots, r ? &of_axis : nullptr};
  const int inner[4] = {2, 2, 0, 0};
  int64_t strides[4][kMaxLead];
  if ((rc = merge_lead(first, 2, with, inner, 4, &a.lead, strides)) != OCN_OK) return rc;
  bool vec = true;
  for (int i = 0; i < 2; ++i) {
    if (!x[i]) continue;
    HeadJob &j = a.job[i];
    set_rows(j, out ? nullptr : x[i], nullptr, out ? x[i] : nullptr);
    std::memcpy(out ? j.ol : j.xl, strides[i], sizeof j.xl);
    j.heads = (int32_t)heads_of(x[i]);
    vec = vec && whole_vectors(x[i]);
  }
  std::memcpy(a.slot_l, strides[2], sizeof a.slot_l);
  std::memcpy(a.pos_l, strides[3], sizeof a.pos_l);
  a.slots = (const char *)slots->base + slots->offset;
  a.slots_wide = slots->dtype == OCN_INT64;
  a.cache = (char *)cache->base + cache->offset;
  a.page_stride = cache->stride[0];
  a.head_stride = cache->stride[1];
  a.small_cache = a.page_stride >= 0 && a.page_stride < ((int64_t)1 << 32) && a.head_stride >= 0 && a.head_stride < ((int64_t)1 << 32);
  a.page = (int32_t)page;
  a.page_div = make_fastdiv((uint32_t)page);
  a.slot_count = cache->size[0] * page;
  if (!shape_of_launch(a, r, d, 2)) return OCN_ERR_SHAPE;
  if (a.items == 0 || a.slot_count == 0) return OCN_OK;
  a.sign = 1.0f;
  const int kind = kind_of_pairs(r, vec);
  return for_all_items(a, [&](uint32_t grid) {
#define OCN_READ(T, VEC, KIND) hipLaunchKernelGGL((cache_read_kernel<T, VEC>), dim3(grid), dim3(kBlock), 0, stream, a)
#define OCN_APPEND(T, VEC, KIND) hipLaunchKernelGGL((cache_append_kernel<T, VEC, KIND>), dim3(grid), dim3(kBlock), 0, stream, a)
    if (out) OCN_BY_TYPE(first->dtype, vec, kPairsNone, OCN_READ);
    else OCN_BY_TYPE(first->dtype, vec, kind, OCN_APPEND);
#undef OCN_READ
#undef OCN_APPEND
  });
}

// workgroups that sum a gradient of weights, of `heads` of all heads of a token
int grad_blocks(int64_t tokens, int64_t heads, int64_t all) {
  const int64_t share = all > 0 ? kFoldBlocks * heads / all : 0;
  return (int)std::max<int64_t>(1, std::min<int64_t>(share, tokens * heads / 16));
}

}  // namespace
}  // namespace ocn

using namespace ocn;

extern "C" {

int ocn_rotary(const ocn_tensor *x, const ocn_rotation *rotation, const ocn_tensor *out, uint32_t flags, void *stream) {
  if (!rotation) return OCN_ERR_NULLPTR;
  if (flags & ~OCN_ROTATE_BACK) return OCN_ERR_OP;
  const ocn_tensor *none = nullptr;
  return run_rows(false, &x, &none, &out, 1, 0.0, rotation, (flags & OCN_ROTATE_BACK) != 0, (hipStream_t)stream);
}

int ocn_norm_rotary(const ocn_tensor *q, const ocn_tensor *q_weight, const ocn_tensor *q_out, const ocn_tensor *k,
                    const ocn_tensor *k_weight, const ocn_tensor *k_out, double eps, const ocn_rotation *rotation, void *stream) {
  if ((!k) != (!k_out)) return OCN_ERR_NULLPTR;
  const ocn_tensor *x[2] = {q, k}, *w[2] = {q_weight, k_weight}, *out[2] = {q_out, k_out};
  return run_rows(true, x, w, out, k ? 2 : 1, eps, rotation, false, (hipStream_t)stream);
}

size_t ocn_norm_rotary_grad_workspace_bytes(const ocn_tensor *q, const ocn_tensor *k) {
  if (check_heads(q) != OCN_OK || (k && check_heads(k) != OCN_OK)) return 0;
  const int64_t all = heads_of(q) + (k ? heads_of(k) : 0);
  size_t n = (size_t)grad_blocks(tokens_of(q), heads_of(q), all) * channels_of(q);
  if (k) n += (size_t)grad_blocks(tokens_of(k), heads_of(k), all) * channels_of(k);
  return n * sizeof(float);
}

int ocn_norm_rotary_grad(const ocn_tensor *q_gout, const ocn_tensor *q, const ocn_tensor *q_weight, const ocn_tensor *q_gin, const ocn_tensor *q_gweight,
                         const ocn_tensor *k_gout, const ocn_tensor *k, const ocn_tensor *k_weight, const ocn_tensor *k_gin, const ocn_tensor *k_gweight,
                         double eps, const ocn_rotation *rotation, void *workspace, size_t workspace_bytes, void *stream) {
  if ((!k) != (!k_gin) || (!k) != (!k_gout)) return OCN_ERR_NULLPTR;
  const int jobs = k ? 2 : 1;
  const ocn_tensor *x[2] = {q, k}, *g[2] = {q_gout, k_gout}, *w[2] = {q_weight, k_weight}, *out[2] = {q_gin, k_gin}, *gw[2] = {q_gweight, k_gweight};
  HeadOperand ops[12];
  int n = 0, rc;
  for (int i = 0; i < jobs; ++i) {
    if ((rc = check_heads(x[i])) != OCN_OK || (rc = check_heads(g[i])) != OCN_OK || (rc = check_heads(out[i])) != OCN_OK) return rc;
    if (g[i]->dtype != x[0]->dtype || out[i]->dtype != x[0]->dtype || x[i]->dtype != x[0]->dtype) return OCN_ERR_DTYPE;
    if (!same_shape(x[i], out[i]) || !same_shape(x[i], g[i]) || channels_of(x[i]) != channels_of(x[0])) return OCN_ERR_SHAPE;
    if ((rc = check_weight(w[i], channels_of(x[i]))) != OCN_OK || (rc = check_weight(gw[i], channels_of(x[i]))) != OCN_OK) return rc;
    if (gw[i] && !w[i]) return OCN_ERR_NULLPTR;
  }
  if ((rc = check_rotation(rotation, channels_of(x[0]), x[0]->device)) != OCN_OK) return rc;
  for (int i = 0; i < jobs; ++i) {
    ops[n++] = {x[i], false};
    ops[n++] = {g[i], false};
    ops[n] = {out[i], true, n - 2, n - 1};
    ++n;
    if (w[i]) ops[n++] = {w[i], false};
    if (gw[i]) ops[n++] = {gw[i], true};
  }
  if (rotation) {
    ops[n++] = {rotation->positions, false};
    ops[n++] = {rotation->frequencies, false};
  }
  if ((rc = check_operands(ops, n)) != OCN_OK) return rc;
  HeadArgs a;
  std::memset(&a, 0, sizeof a);
  const ocn_tensor of_axis = one_axis(rotation);
  const ocn_tensor *with[7] = {x[0], g[0], out[0], x[1], g[1], out[1], rotation ? &of_axis : nullptr};
  const int inner[7] = {2, 2, 2, 2, 2, 2, 0};
  int64_t strides[7][kMaxLead];
  if (k) {
    if (k->ndim != q->ndim) return OCN_ERR_SHAPE;
    for (int d = 0; d + 2 < q->ndim; ++d)
      if (q->size[d] != k->size[d]) return OCN_ERR_SHAPE;
  }
  if ((rc = merge_lead(q, 2, with, inner, 7, &a.lead, strides)) != OCN_OK) return rc;
  const int64_t d = channels_of(q);
  bool vec = true;
  FoldArgs f;
  std::memset(&f, 0, sizeof f);
  size_t need = 0;
  bool sums = false;
  for (int i = 0; i < jobs; ++i) {
    HeadJob &j = a.job[i];
    set_rows(j, x[i], g[i], out[i]);
    std::memcpy(j.xl, strides[3 * i], sizeof j.xl);
    std::memcpy(j.gl, strides[3 * i + 1], sizeof j.gl);
    std::memcpy(j.ol, strides[3 * i + 2], sizeof j.ol);
    j.heads = (int32_t)heads_of(x[i]);
    if (w[i]) {
      j.weight = (const char *)w[i]->base + w[i]->offset;
      j.weight_stride = w[i]->stride[0];
      j.weight_type = w[i]->dtype;
    }
    vec = vec && whole_vectors(x[i]) && whole_vectors(g[i]) && whole_vectors(out[i]);
    j.workers = grad_blocks(a.lead.tokens, j.heads, heads_of(q) + (k ? heads_of(k) : 0));
    if (gw[i]) {
      sums = true;
      f.partial[i] = j.partial = (float *)workspace + need;
      f.out[i] = (char *)gw[i]->base + gw[i]->offset;
      f.stride[i] = gw[i]->stride[0];
      f.type[i] = gw[i]->dtype;
    }
    need += (size_t)j.workers * d;
  }
  if (sums) {
    if (!workspace || workspace_bytes < need * sizeof(float)) return OCN_ERR_WORKSPACE;
    if ((uintptr_t)workspace % 256 != 0) return OCN_ERR_ALIGN;
  }
  std::memcpy(a.pos_l, strides[6], sizeof a.pos_l);
  if (d == 0) return OCN_OK;
  if (!shape_of_launch(a, rotation, d, jobs)) return OCN_ERR_SHAPE;
  for (int i = 0; i < jobs; ++i) {     // as many items for each, or one fewer for some
    HeadJob &j = a.job[i];
    const uint32_t rounds = std::max<uint32_t>(1, (j.items + j.workers - 1) / j.workers);
    f.count[i] = j.workers = (int32_t)std::max<uint32_t>(1, (j.items + rounds - 1) / rounds);
  }
  a.eps = (float)eps;
  a.sign = -1.0f;
  const int kind = kind_of_pairs(rotation, vec), across = std::max(f.count[0], f.count[1]);
  const hipStream_t s = (hipStream_t)stream;
#define OCN_GRAD(T, VEC, KIND) hipLaunchKernelGGL((head_grad_kernel<T, VEC, KIND>), dim3(across, jobs), dim3(kBlock), 0, s, a)
  OCN_BY_TYPE(q->dtype, vec, kind, OCN_GRAD);
#undef OCN_GRAD
  rc = done(hipGetLastError());
  if (rc != OCN_OK || !sums) return rc;
  f.d = (int32_t)d;
  hipLaunchKernelGGL(head_fold_kernel, dim3((uint32_t)((d + 7) / 8), jobs), dim3(kFoldLanes), 0, s, f);
  return done(hipGetLastError());
}

size_t ocn_cache_block_bytes(int64_t page_tokens, int32_t channels) {
  if (page_tokens < 16 || page_tokens % 16 != 0 || page_tokens > kMaxPage || !cache_channels(channels)) return 0;
  return (size_t)page_tokens * channels * 9 / 8;
}

int ocn_cache_append(const ocn_tensor *k, const ocn_tensor *v, const ocn_rotation *rotation, const ocn_tensor *slots,
                     const ocn_tensor *cache, void *stream) {
  if (!k || !v) return OCN_ERR_NULLPTR;
  return run_cache(k, v, rotation, slots, cache, false, (hipStream_t)stream);
}

int ocn_cache_read(const ocn_tensor *cache, const ocn_tensor *slots, const ocn_tensor *k, const ocn_tensor *v, void *stream) {
  return run_cache(k, v, nullptr, slots, cache, true, (hipStream_t)stream);
}

}  // extern "C"
