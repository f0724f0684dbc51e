// What the attentions over packed rows share: fragments of matrix products on MFMA, the places of the
// rows' segments, and tiles of tokens on their way to LDS.
#pragma once

#include <type_traits>

#include "sequence.h"

namespace als {

using u32x4 = uint32_t __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.44269504088896340736f;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// ---- fragments: 8 values of a contraction of 32 per lane ---------------------------------------
// Lane l holds 8 of 32 places for row (or column) m = l & 15, in one of two orders (a sum's terms may
// come in any, provided both operands use the same). With g = l >> 4:
//   along a row of LDS, places 8 g .. 8 g + 7, one 16-byte read;
//   down the tokens, places 4 g .. 4 g + 3 and 16 + 4 g .. 16 + 4 g + 3.
// Two result tiles of an MFMA hold their rows 4 g .. 4 g + 3 in a lane, which is the second order, so
// that weights are operands of the next product as they are. The state's tiles take the columns of k
// in such an order (frag_col's STEP 8) that a pair of them is an operand of the first order.
//
// bf16 values are held as they are. fp32 values are held in three bf16 parts, whose sum they are, and
// a product is the sum of six products of parts, which leaves out 2^-22 of it at most, in either
// direction: six MFMAs of 16 cycles where the fp32 MFMAs of the same tile take 256.
template <typename T> constexpr int kParts = sizeof(T) == 2 ? 1 : 3;
// Of the weights, and of the state where a query reads it. Their second part costs bf16 a second MFMA,
// 14 of 57 in a wave's chunk at 64 wide.
template <typename T> constexpr int kReadParts = sizeof(T) == 2 ? 2 : 3;
template <int NP> struct Frag { bf16x8 p[NP]; };

template <typename T> struct Vec4;
template <> struct Vec4<float> { using type = f32x4; };
template <> struct Vec4<bf16> { using type = bf16x4; };

__device__ __forceinline__ bf16x8 joined(bf16x4 lo, bf16x4 hi) {
  return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}

__device__ __forceinline__ f32x4 mma(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma(const Frag<1> &a, const Frag<1> &b, f32x4 c) {
  return mma(a.p[0], b.p[0], c);
}
__device__ __forceinline__ f32x4 mma(const Frag<1> &a, const Frag<2> &b, f32x4 c) {
  c = mma(a.p[0], b.p[1], c);
  return mma(a.p[0], b.p[0], c);
}
__device__ __forceinline__ f32x4 mma(const Frag<3> &a, const Frag<3> &b, f32x4 c) {
  c = mma(a.p[0], b.p[2], c);
  c = mma(a.p[2], b.p[0], c);
  c = mma(a.p[1], b.p[1], c);
  c = mma(a.p[0], b.p[1], c);
  c = mma(a.p[1], b.p[0], c);
  return mma(a.p[0], b.p[0], c);
}

// Row m of a 16-row tile at x (row length ld, parts `part` apart), contraction along the row from
// column 0.
template <int NP>
__device__ __forceinline__ Frag<NP> frag_row(const bf16 *x, int ld, int part, int lane) {
  const bf16 *p = x + (lane & 15) * ld + (lane >> 4) * 8;
  Frag<NP> f;
#pragma unroll
  for (int n = 0; n < NP; ++n) f.p[n] = *(const bf16x8 *)(p + n * part);
  return f;
}
// Column STEP * (m / 4) + m % 4 from x, contraction down 32 rows. The transposing LDS read: 16 lanes
// name the 16 8-byte pieces of a 4 x 16 block, and lane i of them gets column i.
template <int NP, int STEP>
__device__ __forceinline__ Frag<NP> frag_col(const bf16 *x, int ld, int part, int lane) {
  using L = __attribute__((address_space(3))) bf16x4 *;
  const bf16 *p = x + (lane >> 2) * ld + (lane & 3) * STEP;
  Frag<NP> f;
#pragma unroll
  for (int n = 0; n < NP; ++n)
    f.p[n] = joined(__builtin_amdgcn_ds_read_tr16_b64_v4bf16((L)(p + n * part)),
                    __builtin_amdgcn_ds_read_tr16_b64_v4bf16((L)(p + n * part + 16 * ld)));
  return f;
}

// Four values in two or three bf16 parts of 8 bits. The first is cut off, so that the largest finite values
// stay finite. The second is rounded (of three by an integer sum, which takes less time than the
// conversion), so that what it leaves, 2^-16 of the value at most, leans to neither side: with a second part
// cut off as well, fp32 products were all short, by 2^-24 on average. A third takes exactly what is left of
// fp32's 24 bits. Where the other operand is one part (ONE), nothing is left out and all are cut off.
template <int NP, bool ONE = false> __device__ __forceinline__ void as_parts(f32x4 x, bf16x4 *part) {
  using u32x2 = uint32_t __attribute__((ext_vector_type(2)));
#pragma unroll
  for (int n = 0; n < NP; ++n) {
    if (NP == 2 && n == 1) {
      part[1] = __builtin_convertvector(x, bf16x4);
      return;
    }
    uint32_t bits[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) bits[e] = __float_as_uint(x[e]) + (n == 1 && !ONE ? 0x8000u : 0u);
    // the upper halves
    const u32x2 out = {__builtin_amdgcn_perm(bits[1], bits[0], 0x07060302),
                       __builtin_amdgcn_perm(bits[3], bits[2], 0x07060302)};
    part[n] = __builtin_bit_cast(bf16x4, out);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] -= __uint_as_float(bits[e] & 0xffff0000u);
  }
}
template <int NP, bool ONE = false>
__device__ __forceinline__ Frag<NP> as_frag(f32x4 lo, f32x4 hi) {
  bf16x4 a[NP], b[NP];
  as_parts<NP, ONE>(lo, a);
  as_parts<NP, ONE>(hi, b);
  Frag<NP> f;
#pragma unroll
  for (int n = 0; n < NP; ++n) f.p[n] = joined(a[n], b[n]);
  return f;
}

// ---- packed rows --------------------------------------------------------------------------------
// Rows are cut into segments of L = 2^shift tokens, which run side by side. Row b's segments have the
// slots row_ptr[b] / L + b onwards: at least as many as it has segments, one for an empty row, and
// never another row's. The segments that are not their row's last have the entries row_ptr[b] / L
// onwards, again never another row's.
struct Place {
  int64_t first;    // of the row's tokens
  int32_t len;      // tokens of the row
  int32_t row;
  int64_t segment;  // of the row; none where it is not below the number of segments
};

// Values of row_ptr outside [0, n_tokens] are taken as the nearest inside, so that nothing outside
// the tensors is touched whatever it holds.
__device__ __forceinline__ int64_t clamped(int64_t x, int64_t lo, int64_t hi) {
  return x < lo ? lo : (x > hi ? hi : x);
}
__device__ __forceinline__ int64_t segments_of(int64_t len, int shift) {
  return (len + (1LL << shift) - 1) >> shift;
}
// The last row whose slots (or entries) begin at `index` or before, 64 rows at a time.
template <bool ENTRY>
__device__ __forceinline__ Place find_place(const int64_t *__restrict__ row_ptr, int64_t n_rows,
                                            int64_t n_tokens, int shift, int64_t index, int lane) {
  int64_t lo = 0, hi = n_rows;
  while (hi - lo > 1) {
    const int64_t step = (hi - lo + 63) / 64, at = lo + lane * step;
    const bool before =
        at < hi && (clamped(row_ptr[at], 0, n_tokens) >> shift) + (ENTRY ? 0 : at) <= index;
    const int n = __popcll(__ballot(before));
    lo += (n > 0 ? n - 1 : 0) * step;
    hi = lo + step < hi ? lo + step : hi;
  }
  Place p;
  p.row = (int32_t)lo;
  p.first = clamped(row_ptr[lo], 0, n_tokens);
  p.len = (int32_t)(clamped(row_ptr[lo + 1], p.first, n_tokens) - p.first);
  p.segment = index - ((p.first >> shift) + (ENTRY ? 0 : lo));
  return p;
}

// A chunk's tokens of one head of x on their way to LDS, zero past `size` tokens and past `width`: 16
// bytes at a time, fetched into registers while the chunk before is worked on. Without VEC the pieces
// lie at any alignment of their type, and a row's last one is read so that it ends with the row and is
// shifted into place on its way out (read value by value, such rows took three times as long).
// Place r of the chunk is row r ^ flip from `base`, the chunk's lowest token: flip is C - 1 in a pass
// from the last token to the first, and 0 otherwise. Offsets from there are below 2^31
// (kMaxTokenStride).
template <typename T, int C, int WP, int THREADS, bool VEC> struct Tile {
  static constexpr int E = 16 / sizeof(T), ROW = WP / E;
  static constexpr int ROWS = THREADS / ROW, N = (C + ROWS - 1) / ROWS;
  static_assert(THREADS % ROW == 0 && (ROWS >= C || C % ROWS == 0), "whole rows a pass");
  // E values: of bf16 as four words, since the compiler takes halves apart where a read has a condition, and
  // waits for the read to do so
  struct alignas(16) Values { T v[E]; };
  using Piece = typename std::conditional<sizeof(T) == 4, Values, u32x4>::type;
  struct Rows {  // of one chunk
    const char *base;
    uint32_t bytes;  // from row to row
    int flip, size, width;
    __device__ __forceinline__ const char *at(int r, int c) const {
      return base + ((uint32_t)(r ^ flip) * bytes + c * (int)sizeof(T));
    }
  };
  Piece held[N];

  __device__ __forceinline__ void fetch(const Rows &x, int tid) {
    const int r0 = tid / ROW, c = tid % ROW * E;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int r = r0 + i * ROWS;
      if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < E; ++e) held[i].v[e] = (T)0.f;
      } else {
        held[i] = Piece{};
      }
      if (r < x.size && c < x.width) {
        if (VEC)
          held[i] = *(const Piece *)x.at(r, c);
        else if (x.width >= E)
          __builtin_memcpy(&held[i], x.at(r, c < x.width - E ? c : x.width - E), 16);
      }
    }
  }
  // piece i of this lane, as it goes to column c
  __device__ __forceinline__ Piece piece(const Rows &x, int i, int r, int c) const {
    if (VEC) return held[i];
    if (x.width < E) {  // too narrow for any whole piece
      Values p;
#pragma unroll
      for (int e = 0; e < E; ++e)
        p.v[e] = r < x.size && c + e < x.width ? ((const T *)x.at(r, 0))[e] : (T)0.f;
      return __builtin_bit_cast(Piece, p);
    }
    int bits = (c + E > x.width ? c + E - x.width : 0) * (int)sizeof(T) * 8;
    uint64_t w[2];
    __builtin_memcpy(w, &held[i], 16);
    if (bits >= 64) {
      w[0] = w[1];
      w[1] = 0;
      bits -= 64;
    }
    if (bits >= 64) bits = 0;  // past the row: nothing was fetched
    const uint64_t out[2] = {w[0] >> bits | w[1] << 1 << (63 - bits), w[1] >> bits};
    Piece p;
    __builtin_memcpy(&p, out, 16);
    return p;
  }
  __device__ __forceinline__ void put(T *lds, int ld, const Rows &x, int tid) const {
    const int r0 = tid / ROW, c = tid % ROW * E;
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (ROWS <= C || r0 < C)
        *(Piece *)(lds + (r0 + i * ROWS) * ld + c) = piece(x, i, r0 + i * ROWS, c);
  }
  // as operands of products: fp32 in parts
  __device__ __forceinline__ void put_parts(bf16 *lds, int ld, const Rows &x, int tid) const {
    if constexpr (sizeof(T) == 2) {
      put(lds, ld, x, tid);
    } else {
      const int r0 = tid / ROW, c = tid % ROW * E;
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (ROWS <= C || r0 < C) {
          const Piece p = piece(x, i, r0 + i * ROWS, c);
          bf16x4 part[3];
          as_parts<3>(f32x4{p.v[0], p.v[1], p.v[2], p.v[3]}, part);
#pragma unroll
          for (int n = 0; n < 3; ++n)
            *(bf16x4 *)(lds + n * C * ld + (r0 + i * ROWS) * ld + c) = part[n];
        }
    }
  }
};

}  // namespace als
