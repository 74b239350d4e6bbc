// The layer norm and its gradient.
//
//     out = (x - m) r w + b,     m = mean(x),  r = 1 / sqrt(mean((x - m)^2) + eps)
//
// and, with u = (x - m) r and h = w times the gradient of out,
//
//     gradient of x = r (h - mean(h) - u mean(h u)),     of w: the sum over all rows of u times the gradient of out,     of b: of that gradient.
//
// A row is read once and stays in registers: its mean, then the deviations from it, whose squares are summed (two passes over registers: sums of
// x and x^2 lose the variance of rows far from zero).  A mean that is off by its own rounding is as far from a constant row as that row's deviations would be, and 1 / sqrt(eps) makes
// results of the difference: means are of exact sums where values are alike, and divided exactly.  Memory bounds both directions, or, for a few rows, the launch: 24705 rows of 1280 halves (127 MB) in 27.4 us,
// 48 rows of 4096 in 4.8; the gradient of 16384 rows of 4096 bfloat16 (403 MB) in 82.8 us, of which a large copy would take 80.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstring>
#include <type_traits>

#include "dev_types.hpp"
#include "head_types.hpp"
#include "heads.hpp"

namespace ocn {
namespace {

struct LayerArgs {
  const char *x, *g, *weight, *bias;   // g: the gradient of out (backward)
  char *out;
  float *partial;                      // backward: [workgroups][2][width], sums for the gradients of weight and bias; null: not wanted
  Lead lead;
  int64_t xl[kMaxLead], gl[kMaxLead], ol[kMaxLead];
  int64_t xe, ge, oe, weight_stride, bias_stride;
  int32_t weight_type, bias_type;
  int32_t weight_whole, bias_whole;    // their channels lie together
  int32_t width, lanes_log2;           // lanes of a row, where they lie in one wavefront
  int32_t stream;
  float eps, over, wide;               // over: 1 / wide
  double count, one_over;              // the same
};

__device__ __forceinline__ int64_t row_offset(const Lead &lead, const int64_t *stride, uint32_t row) {
  int64_t o = 0;
#pragma nounroll
  for (int d = lead.n - 1; d > 0; --d) {
    const uint32_t q = fast_quotient(row, lead.div[d]);
    o += (int64_t)(row - q * lead.div[d].d) * stride[d];
    row = q;
  }
  return o + (int64_t)row * stride[0];
}

// Where a lane's chunks of eight channels lie.  Where channels lie together (VEC) a chunk is eight of them in a row, which may begin at any element: loads of 16 bytes need no
// alignment.  Else lanes have neighbouring channels, so that a load of theirs is of neighbouring bytes, or nearly.
template <class T> struct Anywhere { typedef eight_t<T> V __attribute__((aligned(2))); };
template <> struct Anywhere<float> { typedef f32x8 V __attribute__((aligned(4))); };

template <bool VEC> struct Place {
  int first, step, chunk;              // of chunk 0; from channel to channel; from chunk to chunk
  __device__ __forceinline__ Place(int lane, int lanes) : first(VEC ? lane * kEight : lane), step(VEC ? 1 : lanes), chunk(lanes * kEight) {}
  __device__ __forceinline__ int at(int c, int i) const { return first + c * chunk + i * step; }
};

template <class T, bool VEC> __device__ __forceinline__ eight_t<T> load_chunk(const char *row, int64_t step, const Place<VEC> &p, int c, int width) {
  eight_t<T> v = {};
  if constexpr (VEC) {
    const char *from = row + p.at(c, 0) * (int)sizeof(T);
    if (p.at(c, 0) + kEight <= width) {
      v = *(const typename Anywhere<T>::V *)from;
    } else if (p.at(c, 0) < width) {      // the row's last ones
#pragma unroll
      for (int i = 0; i < kEight - 1; ++i)
        if (p.at(c, i) < width) v[i] = *(const T *)(from + i * (int)sizeof(T));
    }
  } else {
#pragma unroll
    for (int i = 0; i < kEight; ++i)
      if (p.at(c, i) < width) v[i] = *(const T *)(row + p.at(c, i) * step);
  }
  return v;
}
template <class T, bool VEC> __device__ __forceinline__ void store_chunk(char *row, int64_t step, const Place<VEC> &p, int c, int width, const float *v, bool stream) {
  if constexpr (VEC) {
    char *to = row + p.at(c, 0) * (int)sizeof(T);
    if (p.at(c, 0) + kEight <= width) {
      eight_t<T> o;
#pragma unroll
      for (int i = 0; i < kEight; ++i) o[i] = (T)v[i];
      if (stream) {
        asm volatile("");     // (these keep the two apart: made into one store, they would be an ordinary one)
        __builtin_nontemporal_store(o, (typename Anywhere<T>::V *)to);
        asm volatile("");
      } else {
        *(typename Anywhere<T>::V *)to = o;
      }
    } else if (p.at(c, 0) < width) {
#pragma unroll
      for (int i = 0; i < kEight - 1; ++i)
        if (p.at(c, i) < width) *(T *)(to + i * (int)sizeof(T)) = (T)v[i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < kEight; ++i)
      if (p.at(c, i) < width) *(T *)(row + p.at(c, i) * step) = (T)v[i];
  }
}
// a chunk of weights or biases, which have a type of their own; `none` where there are none
template <bool VEC> __device__ __forceinline__ void load_factors(const char *p, int64_t stride, int type, int whole, const Place<VEC> &at, int c, int width, float none, float *v) {
#pragma unroll
  for (int i = 0; i < kEight; ++i) v[i] = none;
  if (!p) return;
  if (VEC && whole && at.at(c, 0) + kEight <= width) {
    if (type == OCN_FLOAT) {
      const f32x8 w = *(const typename Anywhere<float>::V *)(p + at.at(c, 0) * 4);
#pragma unroll
      for (int i = 0; i < kEight; ++i) v[i] = w[i];
    } else {
      typedef u32x4 Any __attribute__((aligned(2)));
      const u32x4 w = *(const Any *)(p + at.at(c, 0) * 2);
#pragma unroll
      for (int i = 0; i < kEight; ++i) {
        const uint16_t half = (uint16_t)(i % 2 ? w[i / 2] >> 16 : w[i / 2]);
        v[i] = type == OCN_HALF ? (float)__builtin_bit_cast(f16, half) : __builtin_bit_cast(float, (uint32_t)half << 16);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < kEight; ++i)
      if (at.at(c, i) < width) v[i] = load_as_float(p + at.at(c, i) * stride, type);
  }
}

// Sums over the lanes of a row: of one wavefront's, or (WIDE) of a whole workgroup's wavefronts, through LDS.  `slots` is not used again before another call's barrier.
constexpr int kMostWaves = 16;
template <bool WIDE, int N> __device__ __forceinline__ void sums_over_row(float *v, int lanes, float (*slots)[N]) {
#pragma unroll
  for (int n = 0; n < N; ++n) v[n] = sum_over_row(v[n], WIDE ? kWave : lanes);
  if constexpr (WIDE) {
    if (threadIdx.x % kWave == 0) {
#pragma unroll
      for (int n = 0; n < N; ++n) slots[threadIdx.x / kWave][n] = v[n];
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] = 0.0f;
    for (int w = 0; w < lanes / kWave; ++w) {
#pragma unroll
      for (int n = 0; n < N; ++n) v[n] += slots[w][n];
    }
  }
}

// Rows of up to 64 lanes have 256 lanes' workgroups together; longer ones a workgroup of as many wavefronts as they need.
template <bool WIDE> constexpr int kMostLanes = WIDE ? kMostWaves * kWave : kBlock;

template <int CTRL> __device__ __forceinline__ double other_lane(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  return __builtin_bit_cast(double, (uint64_t)other_lane_bits<CTRL>((uint32_t)(u >> 32)) << 32 | other_lane_bits<CTRL>((uint32_t)u));
}
__device__ __forceinline__ double sum_over_row(double v, int lanes) {
  if (lanes > 1) v += other_lane<0xb1>(v);
  if (lanes > 2) v += other_lane<0x4e>(v);
  if (lanes > 4) v += other_lane<0x141>(v);
  if (lanes > 8) v += other_lane<0x140>(v);
  if (lanes > 16) v += __shfl_xor(v, 16);
  if (lanes > 32) v += __shfl_xor(v, 32);
  return v;
}

// A row's mean: rounded to single precision, and what it is more than that (single precision only; of the other types values have fewer bits than that rounding leaves).  Values of
// single precision are summed in double.  Those of 11 bits and fewer that are alike have exact sums of 64 x 16 in single precision; wavefronts' sums are added in double.
template <class T> constexpr bool kWhole = sizeof(T) == 4;
struct Mean { float near, rest; };
// s / n: where that is a number of the type, exactly that
__device__ __forceinline__ double quotient(double s, double n, double over) {
  const double q = s * over;
  return __builtin_fma(__builtin_fma(-q, n, s), over, q);
}
__device__ __forceinline__ float quotient(float s, float n, float over) {
  const float q = s * over;
  return __builtin_fmaf(__builtin_fmaf(-q, n, s), over, q);
}
template <class T, bool WIDE, int C> __device__ __forceinline__ Mean mean_of_row(const LayerArgs &a, const eight_t<T> *x, int lanes, double *slots) {
  typedef std::conditional_t<kWhole<T>, double, float> Sum;
  Sum own = 0;
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int i = 0; i < kEight; ++i) own += (Sum)x[c][i];
  own = sum_over_row(own, WIDE ? kWave : lanes);
  if constexpr (WIDE) {
    if (threadIdx.x % kWave == 0) slots[threadIdx.x / kWave] = (double)own;
    __syncthreads();
    double all = 0.0;
    for (int w = 0; w < lanes / kWave; ++w) all += slots[w];
    const double mean = quotient(all, a.count, a.one_over);
    return {(float)mean, kWhole<T> ? (float)(mean - (double)(float)mean) : 0.0f};
  } else if constexpr (kWhole<T>) {
    const double mean = quotient(own, a.count, a.one_over);
    return {(float)mean, (float)(mean - (double)(float)mean)};
  } else {
    return {quotient(own, a.wide, a.over), 0.0f};
  }
}
template <class T> __device__ __forceinline__ float deviation(float x, const Mean &m) { return kWhole<T> ? (x - m.near) - m.rest : x - m.near; }

// (wavefronts that a SIMD is to hold: two registers more of three chunks are one less, 29.6 for 27.3 us of 24705 rows of 1280 halves)
template <class T, bool WIDE, int C> constexpr int kNormWaves = WIDE ? 8 : C == 4 ? 4 : C == 3 ? (sizeof(T) == 2 ? 6 : 5) : 8;

template <class T, bool VEC, bool WIDE, int C>
__global__ __launch_bounds__(kMostLanes<WIDE>) __attribute__((amdgpu_waves_per_eu(kNormWaves<T, WIDE, C>))) void layer_norm_kernel(const LayerArgs a, uint32_t first) {
  warm_arguments<LayerArgs>();
  __shared__ double means[WIDE ? kMostWaves : 1];
  __shared__ float squares[WIDE ? kMostWaves : 1][1];
  const int lanes = WIDE ? (int)blockDim.x : 1 << a.lanes_log2, lane = WIDE ? (int)threadIdx.x : (int)threadIdx.x & (lanes - 1), width = a.width;
  const Place<VEC> p(lane, lanes);
  const uint32_t row = WIDE ? first + blockIdx.x : (first + blockIdx.x) * (kBlock >> a.lanes_log2) + (threadIdx.x >> a.lanes_log2);
  const bool mine = row < a.lead.tokens;
  const char *from = a.x + row_offset(a.lead, a.xl, mine ? row : 0);
  eight_t<T> x[C];
#pragma unroll
  for (int c = 0; c < C; ++c) x[c] = load_chunk<T, VEC>(from, a.xe, p, c, mine ? width : 0);
  char *to = a.out + row_offset(a.lead, a.ol, mine ? row : 0);
  const Mean mean = mean_of_row<T, WIDE, C>(a, x, lanes, means);
  float s[1] = {0.0f};
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int i = 0; i < kEight; ++i) {
      const float d = p.at(c, i) < width ? deviation<T>((float)x[c][i], mean) : 0.0f;
      s[0] = __builtin_fmaf(d, d, s[0]);
    }
  sums_over_row<WIDE, 1>(s, lanes, squares);
  const float r = __builtin_amdgcn_rsqf(s[0] * a.over + a.eps);
  if (!mine) return;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    float w[kEight], b[kEight], v[kEight];
    load_factors<VEC>(a.weight, a.weight_stride, a.weight_type, a.weight_whole, p, c, width, 1.0f, w);
    load_factors<VEC>(a.bias, a.bias_stride, a.bias_type, a.bias_whole, p, c, width, 0.0f, b);
#pragma unroll
    for (int i = 0; i < kEight; ++i) {
      v[i] = __builtin_fmaf(deviation<T>((float)x[c][i], mean) * r, w[i], b[i]);
    }
    store_chunk<T, VEC>(to, a.oe, p, c, width, v, a.stream);
  }
}

// The gradient.  A lane keeps the sums of its channels over all rows of its workgroup, workgroups leave theirs in the workspace, and a second launch adds them
// up in a fixed order: no atomics, the same bits every time.  The next rows are on their way while one is worked on, as far as there are registers for them (16384 rows of 4096
// channels: 115 us for 137 with none).
template <bool WIDE, int C> constexpr int kRowsAhead = C == 1 ? 2 : WIDE ? 0 : 1;

template <class T, bool VEC, bool WIDE, int C> __global__ __launch_bounds__(kMostLanes<WIDE>) void layer_grad_kernel(const LayerArgs a) {
  warm_arguments<LayerArgs>();
  __shared__ double means[WIDE ? kMostWaves : 1];
  __shared__ float squares[WIDE ? kMostWaves : 1][3];
  const int lanes = WIDE ? (int)blockDim.x : 1 << a.lanes_log2, lane = WIDE ? (int)threadIdx.x : (int)threadIdx.x & (lanes - 1), width = a.width;
  const Place<VEC> p(lane, lanes);
  const uint32_t rows = WIDE ? 1 : kBlock >> a.lanes_log2, mine = WIDE ? 0 : threadIdx.x >> a.lanes_log2;
  float gw[C * kEight], gb[C * kEight], w[C][kEight];       // (weights stay: loads of theirs, which arrive in order, would wait for the rows ahead)
#pragma unroll
  for (int i = 0; i < C * kEight; ++i) gw[i] = gb[i] = 0.0f;
#pragma unroll
  for (int c = 0; c < C; ++c) load_factors<VEC>(a.weight, a.weight_stride, a.weight_type, a.weight_whole, p, c, width, 1.0f, w[c]);
  constexpr int AHEAD = kRowsAhead<WIDE, C>;
  eight_t<T> x[AHEAD + 1][C], g[AHEAD + 1][C];       // this row and the next ones
  const auto load = [&](uint64_t base, int u) {
    const uint64_t row = base + mine;
    const bool in = row < a.lead.tokens;
    const char *px = a.x + row_offset(a.lead, a.xl, in ? (uint32_t)row : 0), *pg = a.g + row_offset(a.lead, a.gl, in ? (uint32_t)row : 0);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      x[u][c] = load_chunk<T, VEC>(px, a.xe, p, c, in ? width : 0);
      g[u][c] = load_chunk<T, VEC>(pg, a.ge, p, c, in ? width : 0);
    }
  };
  const uint64_t step = (uint64_t)gridDim.x * rows;       // (rows past the last may pass 32 bits)
#pragma unroll
  for (int u = 0; u < AHEAD; ++u) load((uint64_t)blockIdx.x * rows + u * step, u);
  for (uint64_t base = (uint64_t)blockIdx.x * rows; base < a.lead.tokens; base += step) {
    const uint32_t row = (uint32_t)base + mine;
    const bool in = row < a.lead.tokens;
    load(base + AHEAD * step, AHEAD);
    const eight_t<T> *const x0 = x[0], *const g0 = g[0];
    const Mean mean = mean_of_row<T, WIDE, C>(a, x0, lanes, means);
    float s[3] = {0.0f, 0.0f, 0.0f};       // of d^2, h, h d
#pragma unroll
    for (int c = 0; c < C; ++c) {
#pragma unroll
      for (int i = 0; i < kEight; ++i) {
        const float d = p.at(c, i) < width ? deviation<T>((float)x0[c][i], mean) : 0.0f, h = (float)g0[c][i] * w[c][i];
        s[0] = __builtin_fmaf(d, d, s[0]);
        s[1] += h;
        s[2] = __builtin_fmaf(h, d, s[2]);
      }
    }
    sums_over_row<WIDE, 3>(s, lanes, squares);
    const float r = __builtin_amdgcn_rsqf(s[0] * a.over + a.eps);
    const float all = s[1] * a.over, along = s[2] * a.over * r;
    if (in) {
      char *to = a.out + row_offset(a.lead, a.ol, row);
#pragma unroll
      for (int c = 0; c < C; ++c) {
        float v[kEight];
#pragma unroll
        for (int i = 0; i < kEight; ++i) {
          const float u = deviation<T>((float)x0[c][i], mean) * r, gg = (float)g0[c][i];
          gw[c * kEight + i] = __builtin_fmaf(gg, u, gw[c * kEight + i]);
          gb[c * kEight + i] += gg;
          v[i] = r * (__builtin_fmaf(gg, w[c][i], -all) - u * along);
        }
        store_chunk<T, VEC>(to, a.oe, p, c, width, v, a.stream);
      }
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
#pragma unroll
      for (int c = 0; c < C; ++c) x[u][c] = x[u + 1][c], g[u][c] = g[u + 1][c];
  }
  if (!a.partial) return;
  float *const partial = a.partial + (int64_t)blockIdx.x * 2 * width;
  if constexpr (WIDE) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      store_chunk<float, VEC>((char *)partial, 4, p, c, width, gw + c * kEight, false);
      store_chunk<float, VEC>((char *)(partial + width), 4, p, c, width, gb + c * kEight, false);
    }
  } else {      // the rows that the workgroup's lanes took side by side
    __shared__ float sums[kBlock * C * kEight];
    const int wide = lanes * C * kEight;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      __syncthreads();
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < kEight; ++i) sums[mine * wide + p.at(c, i)] = which ? gb[c * kEight + i] : gw[c * kEight + i];
      __syncthreads();
      for (int e = threadIdx.x; e < width; e += kBlock) {
        float s = 0.0f;
        for (uint32_t r = 0; r < rows; ++r) s += sums[r * wide + e];
        partial[which * width + e] = s;
      }
    }
  }
}

constexpr int kFoldColumns = 32, kFoldRows = 32;

struct LayerFoldArgs {
  const float *partial;
  char *out[2];
  int64_t stride[2];
  int32_t type[2], width, count;
};

// 32 channels have a workgroup of 32 rows of lanes; sums of sums in double precision
__global__ __launch_bounds__(kFoldColumns *kFoldRows) void layer_fold_kernel(const LayerFoldArgs a) {
  __shared__ double part[kFoldRows][kFoldColumns];
  const int which = blockIdx.y, lane = threadIdx.x % kFoldColumns, row = threadIdx.x / kFoldColumns, c = blockIdx.x * kFoldColumns + lane;
  if (!a.out[which]) return;
  double s = 0.0;
  if (c < a.width) {
#pragma unroll 8
    for (int i = row; i < a.count; i += kFoldRows) s += a.partial[((int64_t)i * 2 + which) * a.width + c];
  }
  part[row][lane] = s;
  for (int half = kFoldRows / 2; half > 0; half /= 2) {
    __syncthreads();
    if (row < half) part[row][lane] += part[row + half][lane];
  }
  if (row == 0 && c < a.width) store_from_float(a.out[which] + c * a.stride[which], a.type[which], (float)part[0][lane]);
}

// ---------------------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------------------

int done(hipError_t e) {
  if (e == hipSuccess) return OCN_OK;
  record_hip_error((int)e);
  return OCN_ERR_LAUNCH;
}

// How rows go to lanes: wavefronts of a row (1: a row has 2^lanes_log2 lanes of one), and chunks of eight channels of a lane.  Forward a lane has two chunks of a long row, so that enough
// is on its way (16384 rows of 4096 channels: 49 us, 80 with one); backward, where it keeps sums of its channels and the next rows, one up to eight wavefronts (86 us, 102 with two), and two of
// longer rows, which sixteen wavefronts would wait for one another over (16384 rows of 8192: 162 us for 199).
struct Shape { int waves, chunks, lanes_log2; };
Shape shape_of(int64_t width, bool grad) {
  int64_t lanes = 1;
  int log2 = 0;
  while (lanes * kEight < width && lanes < kWave) lanes *= 2, ++log2;
  if (width <= lanes * kEight) return {1, 1, log2};
  const int64_t chunk = kWave * kEight;
  if (width <= (grad ? 2 : 4) * chunk) return {1, (int)((width + chunk - 1) / chunk), 6};
  const int chunks = grad && width <= 8 * chunk ? 1 : 2;
  return {(int)((width + chunks * chunk - 1) / (chunks * chunk)), chunks, 6};
}

int64_t rows_of(const ocn_tensor *t) {
  int64_t n = 1;
  for (int d = 0; d + 1 < t->ndim; ++d) n = t->size[d] > 0 && n > ((int64_t)1 << 31) / t->size[d] ? (int64_t)1 << 31 : n * t->size[d];
  return n;
}
int64_t width_of(const ocn_tensor *t) { return t->size[t->ndim - 1]; }

// Workgroups of the gradient: as many as leave their sums a small part of what is read, twice as many where a lane has one chunk and a row four wavefronts or fewer (bfloat16: 16384 rows of
// 2048 channels 46 us for 56 with 512, 65536 of 512 channels 45 for 56; but 16384 of 4096 channels 94 for 86, of 1024 channels, two chunks to a lane, 38 for 32).
int64_t workers_of(int64_t rows, int64_t width) {
  const Shape s = shape_of(width, true);
  const int64_t at_once = s.waves > 1 ? 1 : kBlock >> s.lanes_log2, most = s.waves <= 4 && s.chunks == 1 ? 1024 : 512;
  const int64_t want = (rows + at_once - 1) / at_once, rounds = std::max<int64_t>(1, (want + most - 1) / most);
  return std::max<int64_t>(1, (want + rounds - 1) / rounds);
}

// channels that lie together
bool whole(const ocn_tensor *t) { return width_of(t) <= 1 || t->stride[t->ndim - 1] == head_type_size(t->dtype); }

int check_rows(const ocn_tensor *t) {
  const int rc = check_operand(t, kHeadTypes);
  if (rc != OCN_OK) return rc;
  if (t->ndim < 1) return OCN_ERR_NDIM;
  return width_of(t) > OCN_MAX_WIDTH ? OCN_ERR_SHAPE : OCN_OK;
}

int check_same(const ocn_tensor *t, const ocn_tensor *x) {
  const int rc = check_rows(t);
  if (rc != OCN_OK) return rc;
  if (t->dtype != x->dtype) return OCN_ERR_DTYPE;
  if (t->ndim != x->ndim) return OCN_ERR_SHAPE;
  for (int d = 0; d < t->ndim; ++d)
    if (t->size[d] != x->size[d]) return OCN_ERR_SHAPE;
  return OCN_OK;
}

int check_factors(const ocn_tensor *t, const ocn_tensor *x) {
  if (!t) return OCN_OK;
  const int rc = check_operand(t, kHeadTypes);
  if (rc != OCN_OK) return rc;
  return t->ndim != 1 || t->size[0] != width_of(x) ? OCN_ERR_SHAPE : OCN_OK;
}

const char *start_of(const ocn_tensor *t) { return (const char *)t->base + t->offset; }

int fill(LayerArgs &a, const ocn_tensor *x, const ocn_tensor *g, const ocn_tensor *weight, const ocn_tensor *bias, const ocn_tensor *out, double eps) {
  std::memset(&a, 0, sizeof a);
  const ocn_tensor *with[3] = {x, g, out};
  const int inner[3] = {1, 1, 1};
  int64_t strides[3][kMaxLead];
  const int rc = merge_lead(x, 1, with, inner, 3, &a.lead, strides);
  if (rc != OCN_OK) return rc;
  std::memcpy(a.xl, strides[0], sizeof a.xl);
  std::memcpy(a.gl, strides[1], sizeof a.gl);
  std::memcpy(a.ol, strides[2], sizeof a.ol);
  const int last = x->ndim - 1;
  a.x = start_of(x), a.xe = x->stride[last];
  if (g) a.g = start_of(g), a.ge = g->stride[last];
  a.out = (char *)start_of(out), a.oe = out->stride[last];
  if (weight) a.weight = start_of(weight), a.weight_stride = weight->stride[0], a.weight_type = weight->dtype, a.weight_whole = whole(weight);
  if (bias) a.bias = start_of(bias), a.bias_stride = bias->stride[0], a.bias_type = bias->dtype, a.bias_whole = whole(bias);
  a.width = (int32_t)width_of(x);
  a.lanes_log2 = shape_of(a.width, g != nullptr).lanes_log2;
  a.over = a.width ? 1.0f / (float)a.width : 0.0f;
  a.wide = (float)a.width;
  a.count = (double)a.width;
  a.one_over = a.width ? 1.0 / a.count : 0.0;
  a.eps = (float)eps;
  a.stream = (int64_t)a.lead.tokens * a.width * head_type_size(out->dtype) >= kStreamBytes;
  return OCN_OK;
}

// CALL(type, channels that lie together, whether a row has several wavefronts, chunks of a lane)
#define OCN_NORM_SHAPES(T, VEC, s, CALL)                     \
  do {                                                       \
    if ((s).waves > 1) CALL(T, VEC, true, 2);                \
    else if ((s).chunks == 4) CALL(T, VEC, false, 4);        \
    else if ((s).chunks == 3) CALL(T, VEC, false, 3);        \
    else if ((s).chunks == 2) CALL(T, VEC, false, 2);        \
    else CALL(T, VEC, false, 1);                             \
  } while (0)
#define OCN_GRAD_SHAPES(T, VEC, s, CALL)                     \
  do {                                                       \
    if ((s).waves > 1 && (s).chunks == 1) CALL(T, VEC, true, 1); \
    else if ((s).waves > 1) CALL(T, VEC, true, 2);           \
    else if ((s).chunks == 2) CALL(T, VEC, false, 2);        \
    else CALL(T, VEC, false, 1);                             \
  } while (0)
#define OCN_LAYER_TYPES(SHAPES, dtype, vec, s, CALL)                                       \
  do {                                                                             \
    if ((dtype) == OCN_HALF) { if (vec) SHAPES(f16, true, s, CALL); else SHAPES(f16, false, s, CALL); } \
    else if ((dtype) == OCN_BFLOAT16) { if (vec) SHAPES(bf16, true, s, CALL); else SHAPES(bf16, false, s, CALL); } \
    else { if (vec) SHAPES(float, true, s, CALL); else SHAPES(float, false, s, CALL); } \
  } while (0)

}  // namespace
}  // namespace ocn

using namespace ocn;

extern "C" {

int ocn_layer_norm(const ocn_tensor *x, const ocn_tensor *weight, const ocn_tensor *bias, const ocn_tensor *out, double eps, void *stream) {
  int rc;
  if ((rc = check_rows(x)) != OCN_OK || !out) return rc != OCN_OK ? rc : OCN_ERR_NULLPTR;
  if ((rc = check_same(out, x)) != OCN_OK || (rc = check_factors(weight, x)) != OCN_OK || (rc = check_factors(bias, x)) != OCN_OK) return rc;
  const HeadOperand ops[4] = {{x, false}, {out, true, 0}, {weight, false}, {bias, false}};
  if ((rc = check_operands(ops, 4)) != OCN_OK) return rc;
  LayerArgs a;
  if ((rc = fill(a, x, nullptr, weight, bias, out, eps)) != OCN_OK) return rc;
  if (a.width == 0 || a.lead.tokens == 0) return OCN_OK;
  const Shape s = shape_of(a.width, false);
  const uint32_t at_once = s.waves > 1 ? 1 : kBlock >> s.lanes_log2;
  const int64_t blocks = ((int64_t)a.lead.tokens + at_once - 1) / at_once;
  const bool vec = whole(x) && whole(out);
  for (int64_t at = 0; at < blocks; at += max_launch_blocks()) {
    const uint32_t grid = (uint32_t)std::min<int64_t>(blocks - at, max_launch_blocks()), first = (uint32_t)at;
#define OCN_LAYER(T, VEC, WIDE, C) \
  hipLaunchKernelGGL((layer_norm_kernel<T, VEC, WIDE, C>), dim3(grid), dim3(WIDE ? s.waves * kWave : kBlock), 0, (hipStream_t)stream, a, first)
    OCN_LAYER_TYPES(OCN_NORM_SHAPES, x->dtype, vec, s, OCN_LAYER);
#undef OCN_LAYER
    if ((rc = done(hipGetLastError())) != OCN_OK) return rc;
  }
  return OCN_OK;
}

size_t ocn_layer_norm_grad_workspace_bytes(const ocn_tensor *x) {
  if (check_rows(x) != OCN_OK) return 0;
  return (size_t)workers_of(rows_of(x), width_of(x)) * 2 * width_of(x) * sizeof(float);
}

int ocn_layer_norm_grad(const ocn_tensor *gout, const ocn_tensor *x, const ocn_tensor *weight, const ocn_tensor *gin, const ocn_tensor *gweight,
                        const ocn_tensor *gbias, double eps, void *workspace, size_t workspace_bytes, void *stream) {
  int rc;
  if ((rc = check_rows(x)) != OCN_OK) return rc;
  if (!gout || !gin) return OCN_ERR_NULLPTR;
  if ((rc = check_same(gout, x)) != OCN_OK || (rc = check_same(gin, x)) != OCN_OK || (rc = check_factors(weight, x)) != OCN_OK ||
      (rc = check_factors(gweight, x)) != OCN_OK || (rc = check_factors(gbias, x)) != OCN_OK)
    return rc;
  if (gweight && !weight) return OCN_ERR_NULLPTR;
  const HeadOperand ops[6] = {{x, false}, {gout, false}, {gin, true, 0, 1}, {weight, false}, {gweight, true}, {gbias, true}};
  if ((rc = check_operands(ops, 6)) != OCN_OK) return rc;
  LayerArgs a;
  if ((rc = fill(a, x, gout, weight, nullptr, gin, eps)) != OCN_OK) return rc;
  if (a.width == 0) return OCN_OK;
  const int64_t workers = workers_of(a.lead.tokens, a.width);
  const bool sums = gweight || gbias;
  if (sums) {
    if (!workspace || workspace_bytes < (size_t)workers * 2 * a.width * sizeof(float)) return OCN_ERR_WORKSPACE;
    if ((uintptr_t)workspace % 256 != 0) return OCN_ERR_ALIGN;
    a.partial = (float *)workspace;
  } else if (a.lead.tokens == 0) {
    return OCN_OK;
  }
  const Shape s = shape_of(a.width, true);
  const bool vec = whole(x) && whole(gout) && whole(gin);
#define OCN_LAYER(T, VEC, WIDE, C) \
  hipLaunchKernelGGL((layer_grad_kernel<T, VEC, WIDE, C>), dim3((uint32_t)workers), dim3(WIDE ? s.waves * kWave : kBlock), 0, (hipStream_t)stream, a)
  OCN_LAYER_TYPES(OCN_GRAD_SHAPES, x->dtype, vec, s, OCN_LAYER);
#undef OCN_LAYER
  if ((rc = done(hipGetLastError())) != OCN_OK || !sums) return rc;
  LayerFoldArgs f;
  std::memset(&f, 0, sizeof f);
  f.partial = a.partial;
  f.width = a.width;
  f.count = (int32_t)workers;
  if (gweight) f.out[0] = (char *)start_of(gweight), f.stride[0] = gweight->stride[0], f.type[0] = gweight->dtype;
  if (gbias) f.out[1] = (char *)start_of(gbias), f.stride[1] = gbias->stride[0], f.type[1] = gbias->dtype;
  hipLaunchKernelGGL(layer_fold_kernel, dim3((uint32_t)((a.width + kFoldColumns - 1) / kFoldColumns), 2), dim3(kFoldColumns * kFoldRows), 0, (hipStream_t)stream, f);
  return done(hipGetLastError());
}

}  // extern "C"
