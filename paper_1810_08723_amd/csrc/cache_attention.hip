// Attention over the paged cache of 4-bit values.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>

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
  int64_t pages, columns, window;
  int32_t batch, queries, heads, per_kv;       // query heads to a head of the cache
  int32_t page, type, table_wide, seen_wide;
  FastDiv page_div;
  float scale;                                 // of the scores, times log2(e)
};

// A workgroup has one query head of one query.  Each wavefront goes over tiles of 64 tokens with a running maximum and
// sum: a lane has a token's score, then its channels of the weighted values.
template <int D> __global__ __launch_bounds__(kBlock) void attention_kernel(const AttentionArgs a) {
  constexpr int W = kBlock / kWave, C = D / kWave;
  __shared__ float query[D];
  __shared__ float weight[W][kWave];
  __shared__ int64_t place[W][kWave];
  __shared__ float sums[W][D], top_of[W], total_of[W];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  for (int64_t unit = blockIdx.x; unit < (int64_t)a.batch * a.queries * a.heads; unit += gridDim.x) {
    const int h = (int)(unit % a.heads), t = (int)(unit / a.heads % a.queries), b = (int)(unit / a.heads / a.queries);
    for (int c = threadIdx.x; c < D; c += kBlock)
      query[c] = load_as_float(a.q + b * a.qb + t * a.qt + h * a.qh + c * a.qe, a.type) * a.scale;
    __syncthreads();
    const int64_t n = min(load_index(a.seen + b * a.sb + t * a.st, a.seen_wide), a.columns * a.page);
    const int64_t first = a.window > 0 ? max(n - a.window, (int64_t)0) : 0;
    float top = -__builtin_inff(), total = 0.0f, acc[C];
#pragma unroll
    for (int c = 0; c < C; ++c) acc[c] = 0.0f;
    for (int64_t base = first / kWave * kWave + wave * kWave; base < n; base += W * kWave) {
      const int64_t j = base + lane;
      float score = -__builtin_inff();
      place[wave][lane] = -1;
      if (j >= first && j < n) {
        const int64_t column = j / a.page, page = load_index(a.table + b * a.tb + column * a.tc, a.table_wide);
        const int at = (int)(j - column * a.page);
        if (page >= 0 && page < a.pages) {
          const int64_t block = page * a.page_stride + (h / a.per_kv) * a.head_stride;
          place[wave][lane] = block * 2 * kMaxPage + at;
          score = 0.0f;
          for (int g = 0; g < D / 32; ++g) {
            float part = 0.0f;
            for (int c = 0; c < 32; c += 8) {
              const uint32_t codes = *(const uint32_t *)(a.cache + block + block_k_codes(a.page, D, at, g * 32 + c));
              const f16x2 c0 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, 2.0f, 0), c1 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, 2.0f, 1);
              const f16x2 c2 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, 2.0f, 2), c3 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, 2.0f, 3);
              const float *q = query + g * 32 + c;
              part += (float)c0.x * q[0] + (float)c0.y * q[1] + (float)c1.x * q[2] + (float)c1.y * q[3] + (float)c2.x * q[4] +
                      (float)c2.y * q[5] + (float)c3.x * q[6] + (float)c3.y * q[7];
            }
            score += part * (float)*(const f16 *)(a.cache + block + block_scale(a.page, D, false, g, at));
          }
        }
      }
      float most = score;
      for (int m = 1; m < kWave; m <<= 1) most = fmaxf(most, __shfl_xor(most, m));
      const float now = fmaxf(top, most), shift = now == -__builtin_inff() ? 0.0f : now;
      const float p = __builtin_amdgcn_exp2f(score - shift), keep = __builtin_amdgcn_exp2f(top - shift);
      top = now;
      float add = p;
      for (int m = 1; m < kWave; m <<= 1) add += __shfl_xor(add, m);
      total = total * keep + add;
      weight[wave][lane] = p;
#pragma unroll
      for (int c = 0; c < C; ++c) acc[c] *= keep;
      for (int i = 0; i < kWave; ++i) {
        const int64_t where = place[wave][i];
        if (where < 0) continue;
        const int at = (int)(where & (2 * kMaxPage - 1));
        const char *block = a.cache + where / (2 * kMaxPage);
#pragma unroll
        for (int c = 0; c < C; ++c) {
          const int channel = lane * C + c;
          const uint32_t codes = *(const uint8_t *)(block + block_v_codes(a.page, D, at, channel));
          const f16x2 v = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, 2.0f, 0);
          const float s = (float)*(const f16 *)(block + block_scale(a.page, D, true, channel / 32, at));
          acc[c] += weight[wave][i] * ((float)(channel & 1 ? v.y : v.x) * s);
        }
      }
    }
#pragma unroll
    for (int c = 0; c < C; ++c) sums[wave][lane * C + c] = acc[c];
    if (lane == 0) {
      top_of[wave] = top;
      total_of[wave] = total;
    }
    __syncthreads();
    float all = -__builtin_inff(), sum = 0.0f;
    for (int w = 0; w < W; ++w) all = fmaxf(all, top_of[w]);
    const float shift = all == -__builtin_inff() ? 0.0f : all;
    for (int w = 0; w < W; ++w) sum += total_of[w] * __builtin_amdgcn_exp2f(top_of[w] - shift);
    for (int c = threadIdx.x; c < D; c += kBlock) {
      float v = 0.0f;
      for (int w = 0; w < W; ++w) v += sums[w][c] * __builtin_amdgcn_exp2f(top_of[w] - shift);
      store_from_float(a.out + b * a.ob + t * a.ot + h * a.oh + c * a.oe, a.type, sum == 0.0f ? 0.0f : v / sum);
    }
    if (a.log_sum && threadIdx.x == 0)
      *(float *)(a.log_sum + b * a.lb + t * a.lt + h * a.lh) = sum == 0.0f ? -__builtin_inff() : 0.69314718f * (all + __builtin_log2f(sum));
    __syncthreads();
  }
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
  if (table->size[1] > most / *page) return OCN_ERR_SHAPE;        // (tokens of a sequence)
  int64_t units = 1;
  for (int d = 0; d < 3; ++d) {
    if (q->size[d] != 0 && units > (most - 1) / q->size[d]) return OCN_ERR_SHAPE;
    units *= q->size[d];
  }
  return OCN_OK;
}

}  // namespace
}  // namespace ocn

using namespace ocn;

extern "C" {

size_t ocn_cache_attention_workspace_bytes(const ocn_tensor *q, const ocn_tensor *cache, const ocn_tensor *table) {
  int64_t page;
  if (check_shapes(q, cache, table, &page) != OCN_OK) return 0;
  return 0;
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
  if (!std::isfinite(scale) || window < 0) return OCN_ERR_DOMAIN;
  const HeadOperand ops[6] = {{q, false, nullptr, nullptr}, {cache, false, nullptr, nullptr}, {table, false, nullptr, nullptr},
                              {visible, false, nullptr, nullptr}, {out, true, q, nullptr}, {log_sum, true, nullptr, nullptr}};
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
  a.columns = table->size[1];
  a.window = window;
  a.batch = (int32_t)q->size[0], a.queries = (int32_t)q->size[1], a.heads = (int32_t)q->size[2];
  const int64_t units = (int64_t)a.batch * a.queries * a.heads, d = q->size[3];
  if (units == 0) return OCN_OK;
  a.per_kv = a.heads / (int32_t)cache->size[1];
  a.page = (int32_t)page;
  a.page_div = make_fastdiv((uint32_t)page);
  a.type = q->dtype;
  a.table_wide = table->dtype == OCN_INT64;
  a.seen_wide = visible->dtype == OCN_INT64;
  a.scale = (float)(scale * 1.4426950408889634074);
  const uint32_t grid = (uint32_t)std::min<int64_t>(units, max_launch_blocks());
  const hipStream_t s = (hipStream_t)stream;
  if (d == 64) hipLaunchKernelGGL((attention_kernel<64>), dim3(grid), dim3(kBlock), 0, s, a);
  else if (d == 128) hipLaunchKernelGGL((attention_kernel<128>), dim3(grid), dim3(kBlock), 0, s, a);
  else hipLaunchKernelGGL((attention_kernel<256>), dim3(grid), dim3(kBlock), 0, s, a);
  return done(hipGetLastError());
}

}  // extern "C"
