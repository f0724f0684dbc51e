// What the kernels of attention over gaps of time share (gap.hip: forward, gap_back.hip: gradients,
// gap_step.hip: one token of each beam): the rows of tokens, the buckets of gaps, and fragments of
// queries that lie in global memory.
#pragma once

#include <type_traits>

#include "tiles.h"

namespace als {

using i32x4 = int32_t __attribute__((ext_vector_type(4)));

// The keys [first, i] that a token i reads as a query, and the queries [i, end) that read it as a key.
// Of a token that no row holds: neither.
struct Span2 {
  int32_t first, end;
};
constexpr int32_t kNoRow = 0x7fffffff;  // first of a token without a row

// Up to as many rows a block counts those that begin at its tokens or before; for more there is a
// table, whose launch costs about as much as 64 rows' counting in each block.
constexpr int64_t kCountedRows = 64;

__device__ __forceinline__ Span2 span_from(const int64_t *row_ptr, int64_t n_rows, int64_t n_tokens,
                                           int64_t row, int64_t t) {
  Span2 s = {kNoRow, 0};
  if (row >= 0 && row < n_rows) {
    const int64_t first = clamped(row_ptr[row], 0, n_tokens), end = clamped(row_ptr[row + 1], first, n_tokens);
    if (t >= first && t < end) {
      s.first = (int32_t)first;
      s.end = (int32_t)end;
    }
  }
  return s;
}
__device__ __forceinline__ Span2 span_of(const GapShape &G, const Span2 *spans, int64_t t) {
  if (t >= G.n_tokens) return {kNoRow, 0};
  if (spans) return spans[t];
  int64_t row = -1;
  for (int64_t r = 0; r < G.n_rows; ++r) row += G.row_ptr[r] <= t ? 1 : 0;
  return span_from(G.row_ptr, G.n_rows, G.n_tokens, row, t);
}

// Zeros at token t, if there is one, of `rows` packed rows of a width: row `row` of each token.
template <typename T>
__device__ __forceinline__ void clear_row(const GapShape &G, void *out, int64_t t, int rows, int row, int c0) {
  if (!G.clear_unheld || t >= G.n_tokens) return;
  T *to = (T *)out + (t * rows + row) * G.width;
  for (int c = c0; c < G.width; c += 4) to[c] = (T)0.f;
}

// a - b, at the ends of the range where it does not fit
__device__ __forceinline__ int32_t gap_of(int32_t a, int32_t b) { return __builtin_elementwise_sub_sat(a, b); }

// ---- buckets --------------------------------------------------------------------------------------
// The bucket of a gap is the number of bounds at it or below. Where the last bound is below kTableGaps a table
// in LDS holds for each gap the bias itself (Entry float: one read a score) or the bucket (uint8_t, times four: a
// quarter of the LDS, and a second read for the bias, whose 64 places are 64 banks); larger bounds are searched
// (Entry void), and such calls stage rows of any alignment. With a last bound of 7679 and of 7680, which no gap
// reached, us a call: reading 134 219 tokens of 512 rows, 590 and 880; training on 1 075 431, 19 300 and 25 600.
constexpr int kTableGaps = 7680;
constexpr float kLargest = 3.402823466e38f;

// A bias as scores take it: times log2 e, finite where it was.
__device__ __forceinline__ float bias2(float b) {
  const float x = b * kLog2e;
  return fabsf(b) <= kLargest ? fminf(fmaxf(x, -kLargest), kLargest) : x;
}

// The number of 63 ascending bounds at the gap or below.
__device__ __forceinline__ int bucket_of(const int32_t *bounds, int buckets, int32_t gap) {
  int n = 0;
#pragma unroll
  for (int step = 32; step > 0; step >>= 1) n += bounds[n + step - 1] <= gap ? step : 0;
  return n < buckets - 1 ? n : buckets - 1;
}

template <typename Entry> struct Table { Entry of[kTableGaps]; };
template <> struct Table<void> {};

template <typename Entry> struct Buckets : Table<Entry> {
  static constexpr bool SEARCHED = std::is_void<Entry>::value, DIRECT = std::is_same<Entry, float>::value;
  int32_t bounds[64];
  float bias[64];

  // by the first 64 threads, with a barrier before anything else
  __device__ __forceinline__ void start(const GapShape &G, int head, int tid) {
    if (tid < 64) {
      bias[tid] = bias2(tid < G.buckets ? G.bias[(int64_t)head * G.buckets + tid] : 0.f);
      bounds[tid] = tid < G.buckets - 1 ? G.bounds[tid] : 0x7fffffff;
    }
  }
  // a wave a bucket in turn
  __device__ __forceinline__ void fill(const GapShape &G, int wave, int lane) {
    if constexpr (!SEARCHED) {
      for (int b = wave; b < G.buckets; b += 4) {
        const int lo = b ? bounds[b - 1] : 0, hi = b < G.buckets - 1 ? bounds[b] : G.last_bound + 1;
        if constexpr (DIRECT) {
          const float x = bias[b];
          for (int g = lo + lane; g < hi; g += 64) this->of[g] = x;
        } else {
          for (int g = lo + lane; g < hi; g += 64) this->of[g] = (uint8_t)(b * 4);
        }
      }
    }
  }
  // within [0, last_bound], in one instruction
  __device__ __forceinline__ int clipped(const GapShape &G, int32_t gap) const {
    int g;
    asm("v_med3_i32 %0, %1, 0, %2" : "=v"(g) : "v"(gap), "s"(G.last_bound));
    return g;
  }
  // four times the bucket (not of a DIRECT table, whose biases come without it), and its bias
  __device__ __forceinline__ int kind4(const GapShape &G, int32_t gap) const {
    static_assert(!DIRECT, "a table of biases");
    if constexpr (SEARCHED)
      return 4 * bucket_of(bounds, G.buckets, gap);
    else
      return this->of[clipped(G, gap)];
  }
  __device__ __forceinline__ float bias4(int kind4) const { return *(const float *)((const char *)bias + kind4); }
  __device__ __forceinline__ float bias_of(const GapShape &G, int32_t gap) const {
    if constexpr (DIRECT)
      return this->of[clipped(G, gap)];
    else
      return bias4(kind4(G, gap));
  }
};
// Up to this bias a score's largest is as good as the score itself: exponents may take their
// difference first.
constexpr float kPlainBias = 16777216.f;

// Lane l's bound and bias: whether two gaps have one bucket takes two comparisons over the wave.
struct BucketLanes {
  int32_t bound;
  float bias;
  uint64_t plain;  // buckets whose bias is below kPlainBias
  int last;        // bucket
  template <typename B> __device__ __forceinline__ void read(const B &b, const GapShape &G, int lane) {
    bound = b.bounds[lane];
    bias = b.bias[lane];
    plain = __ballot(fabsf(bias) < kPlainBias);
    last = G.buckets - 1;
  }
  // of the gaps low <= high; -1: more than one. The same in all lanes.
  __device__ __forceinline__ int kind(int32_t low, int32_t high) const {
    const int at = __popcll(__ballot(bound <= low)), to = __popcll(__ballot(bound <= high));
    return at == to ? (at < last ? at : last) : -1;
  }
  __device__ __forceinline__ bool is_plain(int kind) const { return kind >= 0 && (plain >> kind & 1); }
  __device__ __forceinline__ float bias_of(int kind) const {
    return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(bias), kind < 0 ? 0 : kind));
  }
};
// ---- tiles on their way to LDS ----------------------------------------------------------------
// Tile (tiles.h) for rows that are whole pieces of 16 bytes: rows past `size` are taken as the last one, since
// masks leave them out anyway, so that no load has a condition and no register is cleared.
template <typename T, int C, int WP, bool VEC> struct Staged : Tile<T, C, WP, 256, VEC> {
  using Base = Tile<T, C, WP, 256, VEC>;
  using Rows = typename Base::Rows;
  using Piece = typename Base::Piece;
  __device__ __forceinline__ void fetch(const Rows &x, int tid) {
    if constexpr (!VEC) {
      Base::fetch(x, tid);
    } else {
      const int r0 = tid / Base::ROW, c = tid % Base::ROW * Base::E, col = c < x.width ? c : 0;
#pragma unroll
      for (int i = 0; i < Base::N; ++i) {
        const int r = r0 + i * Base::ROWS;
        this->held[i] = *(const Piece *)x.at(r < x.size ? r : x.size - 1, col);
      }
    }
  }
  __device__ __forceinline__ void put_parts(bf16 *lds, int ld, const Rows &x, int tid) {
    if constexpr (VEC) {
      if (x.width < WP) {
        asm volatile("");  // a branch: selected by condition, the pieces would cost every tile their selects
        if (tid % Base::ROW * Base::E >= x.width) {
#pragma unroll
          for (int i = 0; i < Base::N; ++i) this->held[i] = Piece{};
        }
      }
    }
    Base::put_parts(lds, ld, x, tid);
  }
  // Whether what is held has infinities or NaN (columns past the width may be anything).
  __device__ __forceinline__ bool nonfinite(const Rows &x, int tid) const {
    if (!VEC && x.width < Base::E) {  // too narrow for a piece: read as they go to LDS
      bool any = false;
      for (int r = tid / Base::ROW; r < x.size && r < C; r += Base::ROWS)
        for (int e = 0; e < x.width; ++e) any = any || !((float)((const T *)x.at(r, 0))[e] * 0.f == 0.f);
      return any;
    }
    constexpr uint32_t mask = sizeof(T) == 4 ? 0x7f800000u : 0x7f807f80u;  // exponents; all ones carry
    constexpr uint32_t one = sizeof(T) == 4 ? 0x00800000u : 0x00800080u;
    constexpr uint32_t carry = sizeof(T) == 4 ? 0x80000000u : 0x80008000u;
    uint32_t any = 0;
#pragma unroll
    for (int i = 0; i < Base::N; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) any |= (__builtin_bit_cast(u32x4, this->held[i])[e] & mask) + one;
    return (any & carry) != 0;
  }
};

// ---- fragments of a row in global memory ---------------------------------------------------------
// 8 values from column c of the row at p as they lie there, zero past `width`.
template <typename T> struct Raw8 {
  T v[8];
};
template <typename T>
__device__ __forceinline__ Raw8<T> load8(const T *p, int c, int width, bool vec) {
  Raw8<T> x;
#pragma unroll
  for (int e = 0; e < 8; ++e) x.v[e] = (T)0;
  if (vec) {
    constexpr int E = 16 / sizeof(T);
    struct alignas(16) Piece { T v[E]; };
#pragma unroll
    for (int n = 0; n < 8; n += E)
      if (c + n < width) __builtin_memcpy(x.v + n, (const Piece *)(p + c + n), 16);
  } else if (c + 8 <= width) {  // at any alignment of the type
    __builtin_memcpy(x.v, p + c, 8 * sizeof(T));
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (c + e < width) x.v[e] = p[c + e];
  }
  return x;
}
template <typename T> __device__ __forceinline__ f32x4 low4(const Raw8<T> &x) {
  return f32x4{(float)x.v[0], (float)x.v[1], (float)x.v[2], (float)x.v[3]};
}
template <typename T> __device__ __forceinline__ f32x4 high4(const Raw8<T> &x) {
  return f32x4{(float)x.v[4], (float)x.v[5], (float)x.v[6], (float)x.v[7]};
}
// as operands: bf16 values as they are, fp32 ones in three parts
template <typename T> __device__ __forceinline__ Frag<kParts<T>> operand(const Raw8<T> &x) {
  if constexpr (sizeof(T) == 4) {
    return as_frag<3>(low4(x), high4(x));
  } else {
    return Frag<1>{{__builtin_bit_cast(bf16x8, x)}};
  }
}
template <int NP> __device__ __forceinline__ Frag<NP> negated(Frag<NP> f) {
#pragma unroll
  for (int n = 0; n < NP; ++n) f.p[n] = -f.p[n];
  return f;
}
template <typename T, int D>
__device__ __forceinline__ void load_row(const T *p, int width, bool vec, int lane,
                                         Frag<kParts<T>> *f) {
#pragma unroll
  for (int d = 0; d < D / 32; ++d) f[d] = operand(load8(p, d * 32 + (lane >> 4) * 8, width, vec));
}

// Sums of products. Of parts, the products of first parts have a sum of their own: beside it the others' would be
// rounded to its last bits, six times a step.
template <int NP> struct Acc {
  f32x4 sum;
  __device__ __forceinline__ void start(f32x4 x) { sum = x; }
  __device__ __forceinline__ void add(const Frag<NP> &a, const Frag<NP> &b) { sum = mma(a, b, sum); }
  __device__ __forceinline__ f32x4 value() const { return sum; }
};
template <> struct Acc<3> {
  f32x4 sum, rest;
  __device__ __forceinline__ void start(f32x4 x) {
    sum = x;
    rest = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  __device__ __forceinline__ void add(const Frag<3> &a, const Frag<3> &b) {
    rest = mma(a.p[0], b.p[2], rest);
    rest = mma(a.p[2], b.p[0], rest);
    rest = mma(a.p[1], b.p[1], rest);
    rest = mma(a.p[0], b.p[1], rest);
    rest = mma(a.p[1], b.p[0], rest);
    sum = mma(a.p[0], b.p[0], sum);
  }
  __device__ __forceinline__ f32x4 value() const { return sum + rest; }
};
__device__ __forceinline__ f32x4 mma(const Frag<1> &a, const Frag<3> &b, f32x4 c) {
  c = mma(a.p[0], b.p[2], c);
  c = mma(a.p[0], b.p[1], c);
  return mma(a.p[0], b.p[0], c);
}

// Four values at p, at any alignment of the type, of which `n` belong to the row.
template <typename T> __device__ __forceinline__ void store4(T *p, f32x4 x, int n) {
  using V4 = typename Vec4<T>::type;
  const V4 r = __builtin_convertvector(x, V4);
  if (n >= 4) {
    __builtin_memcpy(p, &r, sizeof r);
  } else {
#pragma unroll
    for (int e = 0; e < 3; ++e)
      if (e < n) p[e] = (T)x[e];
  }
}

// What rounding to bf16 leaves out, as the distance of the bit patterns: 16 more bits, so that value and rest
// together are the fp32 value (one bit short of it where a tie went down).
__device__ __forceinline__ void store_rest(int16_t *p, f32x4 x, int n) {
  using s16x4 = int16_t __attribute__((ext_vector_type(4)));
  s16x4 r;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int32_t far = (int32_t)(__float_as_uint(x[e]) -
                                  ((uint32_t)__builtin_bit_cast(uint16_t, (bf16)x[e]) << 16));
    r[e] = (int16_t)(far > 32767 ? 32767 : far < -32768 ? -32768 : far);
  }
  if (n >= 4) {
    __builtin_memcpy(p, &r, sizeof r);
  } else {
#pragma unroll
    for (int e = 0; e < 3; ++e)
      if (e < n) p[e] = r[e];
  }
}
__device__ __forceinline__ float with_rest(bf16 x, int16_t rest) {
  return __uint_as_float(((uint32_t)__builtin_bit_cast(uint16_t, x) << 16) + (uint32_t)(int32_t)rest);
}

// Over the lanes of a column (lane & 15): the sum or the largest. The swaps give each lane both halves of a
// pair of rows of lanes, then of the wave, without a way through LDS.
__device__ __forceinline__ float larger(uint32_t a, uint32_t b) {  // without a first pass for signalling NaNs
  float x;
  asm("v_max_f32 %0, %1, %2" : "=v"(x) : "v"(a), "v"(b));
  return x;
}
__device__ __forceinline__ float column_max(float x) {
  const uint32_t a = __float_as_uint(x);
  const auto y = __builtin_amdgcn_permlane16_swap(a, a, false, false);
  const uint32_t b = __float_as_uint(larger(y[0], y[1]));
  const auto z = __builtin_amdgcn_permlane32_swap(b, b, false, false);
  return larger(z[0], z[1]);
}
__device__ __forceinline__ float column_sum(float x) {
  const uint32_t a = __float_as_uint(x);
  const auto y = __builtin_amdgcn_permlane16_swap(a, a, false, false);
  const uint32_t b = __float_as_uint(__uint_as_float(y[0]) + __uint_as_float(y[1]));
  const auto z = __builtin_amdgcn_permlane32_swap(b, b, false, false);
  return __uint_as_float(z[0]) + __uint_as_float(z[1]);
}
// Over the wave: rotations within rows of 16 lanes, then the swaps. (By six ds_bpermute, each of which waits for
// LDS, 2000 histories of 25 took 118 us forward, 111 so.)
template <typename F> __device__ __forceinline__ int wave_reduced(int x, F of) {
  x = of(x, __builtin_amdgcn_update_dpp(x, x, 0x128, 0xf, 0xf, false));  // row_ror:8
  x = of(x, __builtin_amdgcn_update_dpp(x, x, 0x124, 0xf, 0xf, false));
  x = of(x, __builtin_amdgcn_update_dpp(x, x, 0x122, 0xf, 0xf, false));
  x = of(x, __builtin_amdgcn_update_dpp(x, x, 0x121, 0xf, 0xf, false));
  const auto y = __builtin_amdgcn_permlane16_swap((uint32_t)x, (uint32_t)x, false, false);
  x = of((int)y[0], (int)y[1]);
  const auto z = __builtin_amdgcn_permlane32_swap((uint32_t)x, (uint32_t)x, false, false);
  return of((int)z[0], (int)z[1]);
}
__device__ __forceinline__ int wave_min(int x) {
  return wave_reduced(x, [](int a, int b) { return a < b ? a : b; });
}
__device__ __forceinline__ int wave_max(int x) {
  return wave_reduced(x, [](int a, int b) { return a > b ? a : b; });
}

// A tile of which a mask leaves some places has weights of zero in the others, which an infinity or NaN there
// would turn into NaN. Where such a tile's rows have any, they are summed by weight without those values, and
// the sums that do read them become NaN at the end.
template <int NP> __device__ __forceinline__ Frag<NP> cleaned(Frag<NP> f) {
#pragma unroll
  for (int n = 0; n < NP; ++n) {
    u32x4 x = __builtin_bit_cast(u32x4, f.p[n]);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      x[e] &= ~(((((x[e] & 0x7f807f80u) + 0x00800080u) & 0x80008000u) >> 15) * 0xffffu);
    f.p[n] = __builtin_bit_cast(bf16x8, x);
  }
  return f;
}
// x: rows `lo` to `hi` are looked at, `ok(row)` tells what the lane's column reads. to[c]: columns 16 c + 4 g
// onwards, g the lane's group.
template <typename T, int C, typename OK>
__device__ __forceinline__ void mark_read(const T *x, int64_t stride, int width, int lo, int hi, int lane, OK ok,
                                          f32x4 *to) {
#pragma unroll 1
  for (int r = lo; r < hi; ++r) {
    const T *p = x + r * stride + (lane >> 4) * 4;
    if (!ok(r)) continue;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (c * 16 + (lane >> 4) * 4 + e < width && (float)p[c * 16 + e] * 0.f != 0.f)
          to[c][e] = __builtin_nanf("");
  }
}

}  // namespace als
