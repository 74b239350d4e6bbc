// What attention's kernels over whole sequences and their gradients share: tiles of the matrix units, operands in LDS, and which sequence a workgroup has.
//
// Rows are the queries of a sequence with the query heads that share a head of keys and values: row r is query r / per_kv, head r % per_kv of the group.
// A tile is kSide keys by kSide rows.  Products are formed so that a lane holds one column of the result and the sixteen (four) other indices that are
// its own come in runs of four:
//
//     16-bit types   32x32x16 products: lane (n = lane % 32, h = lane / 32), element i of the result: column n, index 8 (i / 4) + 4 h + i % 4
//     float          16x16x4 products:  lane (n = lane % 16, h = lane / 16), element i: column n, index 4 h + i
//
// A fragment is 16 bytes of a lane, an operand's share of 16 steps of a sum.  Which of the 16 a lane has is free as long as both operands agree: where a result
// is the next product's operand, its own order is taken, so that nothing crosses lanes, and the other operand, transposed, is read from LDS in that order.
#pragma once

#include <hip/hip_runtime.h>

#include <type_traits>

#include "attention.hpp"
#include "dev_types.hpp"
#include "head_types.hpp"

namespace ocn {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

template <class T> struct Tile {
  static constexpr int kSide = sizeof(T) == 2 ? 32 : 16;
  static constexpr int kOwn = sizeof(T) == 2 ? 16 : 4;            // elements of a result in a lane
  static constexpr int kGroups = kWave / kSide;                   // h
  static constexpr int kFrag = 16 / (int)sizeof(T);               // elements of a fragment in a lane
  static constexpr int kSteps = kSide / 16;                       // fragments along a tile's side
  typedef T Frag __attribute__((ext_vector_type(16 / sizeof(T))));
  typedef float Acc __attribute__((ext_vector_type(sizeof(T) == 2 ? 16 : 4)));
};
template <class T> using frag_t = typename Tile<T>::Frag;
template <class T> using acc_t = typename Tile<T>::Acc;

__device__ __forceinline__ f32x16 product(f16x8 a, f16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 product(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 product(f32x4 a, f32x4 b, f32x4 c) {
#pragma unroll
  for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
  return c;
}

// index of element i of a result (of which 4 h is the lane's own part)
template <class T> __device__ __forceinline__ constexpr int own_index(int i) { return 8 * (i / 4) + i % 4; }

// Elements 16 s ... of a result as a fragment, rounded to the type: weights, and differences times weights in the gradient, are off by half a step at most.  The matrix units take operands of one type, and two
// parts of each, which would hold twice the bits, would be twice the products that take them; results are rounded as much again.  Scores, sums and the weights' exponents stay in single precision.
template <class T> __device__ __forceinline__ frag_t<T> as_fragment(const acc_t<T> &a, int s) {
  frag_t<T> f;
  constexpr int N = Tile<T>::kFrag;
#pragma unroll
  for (int e = 0; e < N; ++e) f[e] = (T)a[s * N + e];
  return f;
}

// tiles of channels of a result, which may have more than operands do, and channels of those
template <class TILE, int D> constexpr int kTilesOf = (D + TILE::kSide - 1) / TILE::kSide;
template <class T, int D> constexpr int kWidth = kTilesOf<Tile<T>, D> * Tile<T>::kSide;

// over the lanes that hold a column
template <class T> __device__ __forceinline__ float column_max(float x) {
  const auto a = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
  const uint32_t a0 = a[0], a1 = a[1];
  x = fmaxf(__builtin_bit_cast(float, a0), __builtin_bit_cast(float, a1));
  if constexpr (Tile<T>::kSide == 16) {
    const auto b = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
    const uint32_t b0 = b[0], b1 = b[1];
    x = fmaxf(__builtin_bit_cast(float, b0), __builtin_bit_cast(float, b1));
  }
  return x;
}
template <class T> __device__ __forceinline__ float column_sum(float x) {
  const auto a = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
  const uint32_t a0 = a[0], a1 = a[1];
  x = __builtin_bit_cast(float, a0) + __builtin_bit_cast(float, a1);
  if constexpr (Tile<T>::kSide == 16) {
    const auto b = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
    const uint32_t b0 = b[0], b1 = b[1];
    x = __builtin_bit_cast(float, b0) + __builtin_bit_cast(float, b1);
  }
  return x;
}

// ---- operands in LDS ---------------------------------------------------------------------------
//
// Rows of D channels, each at a power of two of bytes, in pieces of 16 bytes.  Piece c of row r lies at place c ^ turn(r), so that
// neither sixteen rows' same piece nor four rows' pieces of sixteen channels (a transposed read) meet in a bank.
template <class T, int D> struct Held {
  static constexpr int kPitch = (D * (int)sizeof(T) <= 128 ? 128 : D * (int)sizeof(T) <= 256 ? 256 : D * (int)sizeof(T) <= 512 ? 512 : 1024);
  static constexpr int kPieces = D * (int)sizeof(T) / 16;
  __device__ __forceinline__ static int turn(int row) {
    if constexpr (sizeof(T) == 4) return row & 15;
    else if constexpr (kPitch == 128) return (2 * ((row >> 1) & 3)) | ((row >> 3) & 1);
    else return (2 * (row & 7)) | ((row >> 3) & 1);
  }
  __device__ __forceinline__ static int at(int row, int piece) { return row * kPitch + ((piece ^ turn(row)) << 4); }
};

// Where a lane finds its fragments: step 0 of a row-wise one and tile 0 of a transposed one.  Those of other steps and tiles differ in bits that
// no sum carries into.
struct LanePlaces { int row, column; };
template <class T, int D> __device__ __forceinline__ LanePlaces lane_places(int lane) {
  const int n = lane & (Tile<T>::kSide - 1), h = lane / Tile<T>::kSide, j = lane & 15;
  LanePlaces p;
  p.row = Held<T, D>::at(n, h);
  if constexpr (sizeof(T) == 2) p.column = Held<T, D>::at(4 * h + (j >> 2), ((lane & 16) + 4 * (j & 3)) >> 3) + 8 * (j & 1);
  else p.column = 4 * h * Held<T, D>::kPitch + 4 * (j & 3) + ((j >> 2) << 4);
  return p;
}

// A fragment of 16 channels (16 step ...) of rows `row` + n
template <class T, int D> __device__ __forceinline__ frag_t<T> rows_fragment(const char *held, int row, int step, const LanePlaces &p) {
  return *(const frag_t<T> *)(held + ((p.row ^ step * 16 * (int)sizeof(T)) + row * Held<T, D>::kPitch));
}

// Its transpose: lane n has channel side * tile + n of the 16 rows row ... row + 15 (a multiple of 16), in a result's order
template <class T, int D> __device__ __forceinline__ frag_t<T> columns_fragment(const char *held, int row, int tile, const LanePlaces &p) {
  constexpr int PITCH = Held<T, D>::kPitch;
  frag_t<T> f;
  if constexpr (sizeof(T) == 2) {
    typedef __attribute__((address_space(3))) s16x4 *Lds;
    union { s16x4 s[2]; frag_t<T> f; } u;
#pragma unroll
    for (int k = 0; k < 2; ++k)       // (eight rows further a row's turn differs in its last bit)
      u.s[k] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(held + ((p.column ^ (tile * 64 + 16 * k)) + (row + 8 * k) * PITCH)));
    f = u.f;
  } else {
    const int h = threadIdx.x / 16 % 4;
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = *(const float *)(held + ((p.column ^ ((tile * 4 ^ Held<T, D>::turn(4 * h + e)) << 4)) + (row + e) * PITCH));
  }
  return f;
}

// 16 bytes of a row in memory, from channel e on; what lies outside of the row's d channels is zero.  VEC: whole, aligned rows.  Others whose channels lie
// together are loaded in pieces as well, which may begin at any element; the last one, where it is not whole, ends with the row and is shifted.
template <class T, bool VEC> __device__ __forceinline__ u32x4 load_piece(const char *row, int64_t step, int e, int d) {
  constexpr int EACH = 16 / (int)sizeof(T);
  u32x4 v = {0, 0, 0, 0};
  if constexpr (VEC) {
    if (e < d) v = *(const u32x4 *)(row + e * (int)sizeof(T));
  } else if (step == (int)sizeof(T) && d >= EACH) {
    typedef u32x4 Any __attribute__((aligned(2)));
    if (e < d) {
      const int past = e + EACH > d ? e + EACH - d : 0;        // channels of the piece that are none
      v = *(const Any *)(row + (e - past) * (int)sizeof(T));
      if (past) {
        const int bytes = past * (int)sizeof(T);
        if (bytes & 8) v = u32x4{v[2], v[3], 0, 0};
        if (bytes & 4) v = u32x4{v[1], v[2], v[3], 0};
        if (bytes & 2) v = u32x4{v[0] >> 16 | v[1] << 16, v[1] >> 16 | v[2] << 16, v[2] >> 16 | v[3] << 16, v[3] >> 16};
      }
    }
  } else {
    union { T t[EACH]; u32x4 v; } u;
    u.v = v;
#pragma unroll
    for (int i = 0; i < EACH; ++i)
      if (e + i < d) u.t[i] = *(const T *)(row + (e + i) * step);
    v = u.v;
  }
  return v;
}

// four neighbouring channels of a row, rounded
template <class T, bool VEC> __device__ __forceinline__ void store_four(char *row, int64_t step, int e, int d, const float *v) {
  typedef T Four __attribute__((ext_vector_type(4)));
  typedef Four Any __attribute__((aligned(2)));
  Four o;
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = (T)v[i];
  if constexpr (VEC) {
    if (e < d) *(Four *)(row + e * (int)sizeof(T)) = o;
  } else if (step == (int)sizeof(T) && e + 4 <= d) {
    *(Any *)(row + e * (int)sizeof(T)) = o;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (e + i < d) *(T *)(row + (e + i) * step) = o[i];
  }
}

// Wavefronts that a SIMD is to hold: two have 256 registers each, which all are operands of any instruction; a single one has half of its 512 beside the others, reached by copies.
template <class T, int D> constexpr int kWavesAtOnce = sizeof(T) == 2 && D <= 128 ? 2 : 1;

// ---- from memory to LDS ------------------------------------------------------------------------
//
// Whole rows go there without passing through registers: a wavefront's load writes 64 pieces one behind the other, so that a lane loads the piece that
// belongs at its place.  The compiler does not see these loads (it would wait for all of them before any read of LDS): arrived() has to be between them and the reads.  (Their place in LDS is in m0, which scalar instructions write: one wait.)
__device__ __forceinline__ void load_to_lds(uint32_t lds, const char *from) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"{m0}"(lds), "v"(from) : "memory");
}
__device__ __forceinline__ void load_word_to_lds(uint32_t lds, const char *from) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dword %1, off" ::"{m0}"(lds), "v"(from) : "memory");
}
// Every load of the wavefront's has arrived.  Kernels call it behind their loops as well: no path through them ends with a copy into LDS on its way.
__device__ __forceinline__ void arrived() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
__device__ __forceinline__ uint32_t lds_address(const char *p) { return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char *)p; }

// ROWS rows of a tensor into LDS by WAVES wavefronts.  DIRECT: past registers (rows are whole); else put() loads, and store() writes what it loaded.
template <class T, int D, int ROWS, int WAVES, bool DIRECT> struct Carrier {
  static constexpr int kPitch = Held<T, D>::kPitch, kSlots = kPitch / 16;            // places of a row
  static constexpr int kAll = DIRECT ? ROWS * kSlots : ROWS * Held<T, D>::kPieces, kLanes = WAVES * kWave, kEach = (kAll + kLanes - 1) / kLanes;
  u32x4 x[DIRECT ? 1 : kEach];
  __device__ __forceinline__ static int row_of(int i) { return DIRECT ? (i * kLanes + (int)threadIdx.x) / kSlots : (i * kLanes + (int)threadIdx.x) / Held<T, D>::kPieces; }
  // row(i): the address of row i; step: from channel to channel; d: channels
  template <class Row> __device__ __forceinline__ void load(char *held, const Row &row, int64_t step, int d) {
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int at = i * kLanes + (int)threadIdx.x, r = row_of(i);
      if constexpr (DIRECT) {
        if (kAll % kLanes != 0 && i * kLanes + (int)(threadIdx.x & ~(kWave - 1)) >= kAll) continue;
        const int piece = at % kSlots ^ Held<T, D>::turn(r);
        const char *from = row(r) + piece * 16;
        const uint32_t to = __builtin_amdgcn_readfirstlane(lds_address(held) + (at & ~(kWave - 1)) * 16);
        if (d == kSlots * 16 / (int)sizeof(T)) load_to_lds(to, from);
        else if (piece * 16 < d * (int)sizeof(T)) load_to_lds(to, from);
      } else {
        const bool in = kAll % kLanes == 0 || at < kAll;
        x[i] = load_piece<T, false>(row(in ? r : 0), step, at % Held<T, D>::kPieces * (16 / (int)sizeof(T)), in ? d : 0);
      }
    }
  }
  __device__ __forceinline__ void store(char *held) const {
    if constexpr (!DIRECT) {
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const int at = i * kLanes + (int)threadIdx.x;
        if (kAll % kLanes == 0 || at < kAll) *(u32x4 *)(held + Held<T, D>::at(row_of(i), at % Held<T, D>::kPieces)) = x[i];
      }
    }
  }
};
// what lies outside of the rows' channels has to be zero before the first load
template <int LANES> __device__ __forceinline__ void clear_lds(char *held, int bytes) {
  for (int i = threadIdx.x * 16; i < bytes; i += LANES * 16) *(u32x4 *)(held + i) = u32x4{0, 0, 0, 0};
}

// ---- products with operands in LDS ----------------------------------------------------------------
//
// The compiler reads an operand right before the product that takes it, to save registers, and waits for LDS there.  Here N operands (or sets of them) are read AHEAD of
// their turn, and nothing moves from one turn to another: read(i) gives operand i, use(i, operand) takes it.
__device__ __forceinline__ void in_order() { __builtin_amdgcn_sched_barrier(0); }

template <int N, int AHEAD, class Operand, class Read, class Use> __device__ __forceinline__ void pipelined(const Read &read, const Use &use) {
  Operand held[AHEAD + 1];
#pragma unroll
  for (int i = 0; i < AHEAD && i < N; ++i) held[i] = read(i);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if (i + AHEAD < N) held[(i + AHEAD) % (AHEAD + 1)] = read(i + AHEAD);
    in_order();
    use(i, held[i % (AHEAD + 1)]);
    in_order();
  }
  // The last results are not written before eleven or more cycles of waiting, which the compiler does not put where their reader is in another basic block:
  // behind a loop whose last product this is it read a result's last element too early.
  asm volatile("s_nop 15\n\ts_nop 3");
  in_order();
}

// ---- sequences ---------------------------------------------------------------------------------

struct Span { int64_t first; int32_t count; };      // tokens of a sequence

__device__ __forceinline__ int64_t start_at(const Starts &s, int i) {
  const int64_t at = load_index(s.p + i * s.stride, s.wide);
  return at < 0 ? 0 : at > s.all ? s.all : at;
}
__device__ __forceinline__ Span span_of(const Starts &s, int i) {
  if (!s.p) return {0, (int32_t)s.all};
  const int64_t first = start_at(s, i), end = start_at(s, i + 1);
  return {first, (int32_t)(end > first ? end - first : 0)};
}

// Blocks of `size` tokens: a packed sequence has the slots start / size + its number up to the next one's, one for each of its blocks at least, as
// a sequence that begins inside of a block's size may have one more than its length makes.  `own`, the starts that blocks go by, and `other` give the sequence's tokens.
__device__ __forceinline__ bool find_slot(const Starts &own, const Starts &other, const FastDiv &size, uint32_t slot, int *sequence, uint32_t *block, Span *own_span, Span *other_span) {
  // the last sequence whose first slot is not behind this one; all lanes of a wavefront look at once, in the end with all that there is to know of a sequence each
  int lo = 0, hi = own.sequences;      // in [lo, hi)
  const int lane = threadIdx.x & (kWave - 1);
  while (hi - lo > kWave) {
    const int step = (hi - lo + kWave - 1) / kWave, at = lo + lane * step;
    const bool fits = at < hi && fast_quotient((uint32_t)start_at(own, at), size) + (uint32_t)at <= slot;
    const uint64_t all = __ballot(fits);
    const int last = all ? 63 - __builtin_clzll(all) : 0;
    lo += last * step;
    hi = lo + step < hi ? lo + step : hi;
  }
  const int at = lo + lane < hi ? lo + lane : hi - 1;
  const uint32_t own_start = (uint32_t)start_at(own, at), own_end = (uint32_t)start_at(own, at + 1), other_start = (uint32_t)start_at(other, at), other_end = (uint32_t)start_at(other, at + 1);
  const uint32_t first = fast_quotient(own_start, size) + (uint32_t)at;
  const uint64_t all = __ballot(lo + lane < hi && first <= slot);
  const int last = all ? 63 - __builtin_clzll(all) : 0;
  const auto of_last = [&](uint32_t x) { return (uint32_t)__builtin_amdgcn_readlane((int)x, last); };
  *sequence = lo + last;
  *block = slot - of_last(first);
  const uint32_t a = of_last(own_start), b = of_last(own_end), c = of_last(other_start), d = of_last(other_end);
  *own_span = {(int64_t)a, (int32_t)(b > a ? b - a : 0)};
  *other_span = {(int64_t)c, (int32_t)(d > c ? d - c : 0)};
  return all != 0;
}

// What a workgroup has: a block of a sequence's queries (or keys), with some heads that share a head of keys and values
struct Work {
  uint32_t unit, block;
  int split, sequence, kv, head_block;
  Span q, k;
};

// KEYS: blocks are of keys.  False: there is no such block.
template <bool KEYS> __device__ __forceinline__ bool find_work_of(const AttentionArgs &a, uint32_t index, Work *w) {
  w->unit = fast_quotient(index, a.splits_div);
  w->split = (int)(index - w->unit * (uint32_t)a.splits);
  const uint32_t down = fast_quotient(w->unit, a.across_div), across = w->unit - down * a.across_div.d;
  if (down >= a.slots) return false;
  w->kv = (int)fast_quotient(across, a.head_blocks_div);
  w->head_block = (int)(across - (uint32_t)w->kv * (uint32_t)a.head_blocks);
  const Starts &s = KEYS ? a.k_starts : a.q_starts;
  // With a causal mask the first blocks of keys and the last ones of queries have most to do.
  if (s.p) {
    const uint32_t slot = KEYS ? (a.order ? a.order[down] : down) : a.slots - 1 - down;
    if (!find_slot(s, KEYS ? a.q_starts : a.k_starts, a.tokens_div, slot, &w->sequence, &w->block, KEYS ? &w->k : &w->q, KEYS ? &w->q : &w->k)) return false;
  } else {
    const uint32_t turn = fast_quotient(down, a.sequences_div);
    w->sequence = (int)(down - turn * a.sequences_div.d);
    w->block = KEYS ? turn : a.per_sequence - 1 - turn;
  }
  if (!s.p) {
    w->q = span_of(a.q_starts, w->sequence);
    w->k = span_of(a.k_starts, w->sequence);
  }
  return (int64_t)w->block * a.tokens < (KEYS ? w->k.count : w->q.count);
}
__device__ __forceinline__ bool find_work(const AttentionArgs &a, uint32_t index, Work *w) { return find_work_of<false>(a, index, w); }

// Row `row` of a block: its query (of the sequence) and head (of the group); those past the end are taken as the last ones
struct RowPlace { int query, head; bool in; };
__device__ __forceinline__ RowPlace row_place(const AttentionArgs &a, const Work &w, int row) {
  const int t = (int)fast_quotient((uint32_t)row, a.heads_div);
  RowPlace p;
  p.head = w.head_block * a.heads + row - t * a.heads;
  const int64_t query = (int64_t)w.block * a.tokens + t;
  p.in = t < a.tokens && query < w.q.count && p.head < a.per_kv;
  p.query = (int)(query < w.q.count ? query : w.q.count - 1);
  if (p.head >= a.per_kv) p.head = a.per_kv - 1;
  return p;
}

struct Limits { int lo, hi; };       // keys lo <= j < hi of the sequence
__device__ __forceinline__ Limits limits_of(const AttentionArgs &a, const Work &w, int query) {
  Limits l = {0, w.k.count};
  if (a.causal) {
    const int end = query - w.q.count + w.k.count + 1;
    l.hi = end < 0 ? 0 : end;
    if (a.window && end > a.window) l.lo = end - a.window;
  }
  return l;
}
// what some row of a block of queries sees
__device__ __forceinline__ Limits limits_of_block(const AttentionArgs &a, const Work &w) {
  const int64_t first = (int64_t)w.block * a.tokens, end = first + a.tokens < w.q.count ? first + a.tokens : w.q.count;
  const Limits one = limits_of(a, w, (int)first), last = limits_of(a, w, (int)end - 1);
  return {one.lo, last.hi};
}

// ... and what all of them see
__device__ __forceinline__ Limits limits_of_all(const AttentionArgs &a, const Work &w) {
  const int64_t first = (int64_t)w.block * a.tokens, end = first + a.tokens < w.q.count ? first + a.tokens : w.q.count;
  const Limits one = limits_of(a, w, (int)first), last = limits_of(a, w, (int)end - 1);
  return {last.lo, one.hi};
}

// ---- parts -------------------------------------------------------------------------------------
//
// Where blocks leave CUs without work, what a block goes over (`tiles` of them) is cut into parts, a workgroup each, of `least` tiles or more.
struct Part { int first, end, parts; bool alone, mine; };      // its tiles; parts in all, one at least; whether it is the only one; whether there is it
__device__ __forceinline__ Part part_of(int tiles, int splits, int least, int split) {
  int per = (tiles + splits - 1) / splits;
  if (per < least) per = least;
  Part p;
  p.parts = tiles <= per ? 1 : (tiles + per - 1) / per;
  p.alone = p.parts == 1;
  p.mine = split < p.parts;
  p.first = split * per;
  p.end = split * per + per < tiles ? split * per + per : tiles;
  return p;
}

constexpr int kJoinRows = 8;       // rows of a workgroup that joins parts, two of each wavefront
constexpr int kJoinAtOnce = 8;     // parts of a row that are on their way from memory at once: one after the other, 64 of them took 23 us

// ---- the order of blocks -----------------------------------------------------------------------
//
// Packed sequences may be of any lengths, which only the GPU knows.  A workgroup that takes long and is started last is waited for by all the others: where there are more of them
// than CUs, those with most to do go first.  One workgroup sorts all blocks by what they have to do, to a sixteenth of it.
static __global__ __launch_bounds__(kOrderLanes) void attention_order_kernel(const AttentionArgs a) {
  constexpr int kSizes = 512;
  __shared__ uint32_t places[kSizes];
  const Starts &s = a.k_starts;
  const auto size_of = [&](uint32_t slot) {
    int lo = 0, hi = s.sequences;
    while (hi - lo > 1) {
      const int middle = lo + (hi - lo) / 2;
      if (fast_quotient((uint32_t)start_at(s, middle), a.tokens_div) + (uint32_t)middle <= slot) lo = middle; else hi = middle;
    }
    const Span q = span_of(a.q_starts, lo), k = span_of(a.k_starts, lo);
    const int64_t block = (int64_t)slot - (fast_quotient((uint32_t)start_at(s, lo), a.tokens_div) + (uint32_t)lo), first = block * a.tokens;
    if (block < 0 || first >= k.count) return 0;
    const int64_t end = first + a.tokens < k.count ? first + a.tokens : k.count;
    int64_t most = q.count;       // queries that see some key of the block
    if (a.causal) {
      const int64_t ahead = (int64_t)q.count - k.count;
      const int64_t from = first + ahead > 0 ? first + ahead : 0;
      const int64_t to = a.window && end - 1 + a.window + ahead < q.count ? end - 1 + a.window + ahead : q.count;
      most = to > from ? to - from : 0;
    }
    const int size = (int)(__builtin_bit_cast(uint32_t, (float)most) >> 19) - (126 << 4);       // four bits behind the first
    return size < 1 ? 1 : size < kSizes ? size : kSizes - 1;
  };
  for (int i = threadIdx.x; i < kSizes; i += blockDim.x) places[i] = 0;
  __syncthreads();
  for (uint32_t i = threadIdx.x; i < a.slots; i += blockDim.x) atomicAdd(&places[size_of(i)], 1u);
  __syncthreads();
  if (threadIdx.x < kWave) {      // blocks that are larger
    constexpr int kEach = kSizes / kWave;
    const int lane = threadIdx.x;
    uint32_t own[kEach], sum = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {      // from the largest down
      own[i] = sum;
      sum += places[kSizes - 1 - lane * kEach - i];
    }
    uint32_t before = sum;
    for (int o = 1; o < kWave; o *= 2) {
      const uint32_t x = __shfl_up(before, o);
      if (lane >= o) before += x;
    }
    before -= sum;
#pragma unroll
    for (int i = 0; i < kEach; ++i) places[kSizes - 1 - lane * kEach - i] = before + own[i];
  }
  __syncthreads();
  for (uint32_t i = threadIdx.x; i < a.slots; i += blockDim.x) a.order[atomicAdd(&places[size_of(i)], 1u)] = i;      // (those of the same size as they come: results do not depend on it)
}

}  // namespace ocn
