// Linear attention with a decay for each head: over the tokens t of a row (a user's ratings in
// the order of time), with e^a the head's decay,
//   S_t = e^a S_{t-1} + k_t v_t^T,   o_t = scale S_t^T q_t.
//
// A row is read in chunks of C tokens. With S the state before the chunk and i, j the places of
// its tokens,
//   o_i = scale (e^{a (i + 1)} S^T q_i + sum_{j <= i} e^{a (i - j)} (q_i . k_j) v_j),
//   S  <- e^{a C} S + sum_j e^{a (C - 1 - j)} k_j v_j^T,
// four matrix products on MFMA. A block holds one head of one row (or of a segment of it): wave w
// owns the columns 16 w .. 16 w + 15 of v, and of the state, which stays in its registers in fp32
// from chunk to chunk; the weights e^{a (i - j)} (q_i . k_j) are computed once per block and shared
// through LDS.
//
// The gradients are passes of the same form. With X the gradient that reaches the state from later
// tokens,
//   dq_t = scale S_t do_t: the pass over (q, k, v) := (do, v, k), with S transposed;
//   X <- e^a (X + scale q_t do_t^T) from the last token to the first, and with X before that step,
//   dv_t = (X + scale q_t do_t^T)^T k_t: the reversed pass over (k, q, do);
//   dk_t = (X + scale q_t do_t^T) v_t: the reversed pass over (v, do, q), with X transposed;
//   X after the first token is the gradient of the entering state.
// A reversed pass reads its state one step nearer and adds to it one step further
// (read e^{a i}, add e^{a (C - j)}).
//
// Rounding. Products have sums in fp32. bf16 inputs: the weights and the state enter a product in two
// bf16 parts, which are off by 2^-16 at most, so that an output is rounded once, on its way out (as one
// bf16 value they would cost as much again as that rounding); what a token adds to the state is split
// into three parts (24 bits), so that the state, an output in fp32, has no bf16 rounding in it. fp32
// inputs: all operands are split so.
#include <type_traits>

#include "internal.h"
#include "sequence.h"

namespace als {

namespace {

constexpr float kLog2e = 1.44269504088896340736f;
// Decays below e^-10000 a token are the same as none left; keeps -inf * 0 out of the exponents.
constexpr float kMinLogDecay = -1e4f;

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

// A lane's 8 values down 32 rows of column m from x, as they lie in LDS.
template <typename T> struct Column;
template <> struct Column<bf16> {
  Frag<1> f;
  __device__ __forceinline__ void read(const bf16 *x, int ld, int lane) {
    f = frag_col<1, 4>(x, ld, 0, lane);
  }
  __device__ __forceinline__ float get(int e) const { return (float)f.p[0][e]; }
  __device__ __forceinline__ void clear(int e) { f.p[0][e] = (bf16)0.f; }
  __device__ __forceinline__ Frag<1> frag() const { return f; }
  __device__ __forceinline__ bool finite() const {
    using u32x4 = uint32_t __attribute__((ext_vector_type(4)));
    const u32x4 bits = __builtin_bit_cast(u32x4, f.p[0]);
    uint32_t carry = 0;  // into either half's sign: its exponent was all ones
#pragma unroll
    for (int e = 0; e < 4; ++e) carry |= (bits[e] & 0x7fff7fffu) + 0x00800080u;
    return (carry & 0x80008000u) == 0;
  }
};
template <> struct Column<float> {
  f32x4 lo, hi;
  __device__ __forceinline__ void read(const float *x, int ld, int lane) {
    const float *p = x + (lane >> 4) * 4 * ld + (lane & 15);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      lo[e] = p[e * ld];
      hi[e] = p[(16 + e) * ld];
    }
  }
  __device__ __forceinline__ float get(int e) const { return e < 4 ? lo[e] : hi[e - 4]; }
  __device__ __forceinline__ void clear(int e) {
    if (e < 4) lo[e] = 0.f; else hi[e - 4] = 0.f;
  }
  __device__ __forceinline__ Frag<3> frag() const { return as_frag<3>(lo, hi); }
  __device__ __forceinline__ bool finite() const {
    float x = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) x = fmaf(lo[e], 0.f, fmaf(hi[e], 0.f, x));
    return x == 0.f;
  }
};

// Row of the state that element e of lane group g holds in tile kt.
__device__ __forceinline__ constexpr int state_row(int kt, int g, int e) {
  return kt / 2 * 32 + g * 8 + kt % 2 * 4 + e;
}

// Padding of a staged row: with it the four lane groups and the rows of one LDS read fall on
// different banks.
template <typename T> constexpr int padded(int width) { return width + (sizeof(T) == 2 ? 16 : 4); }
// Of rows of q and k. Three parts of them at up to 64 wide leave a CU a fourth block with half the
// padding, which is worth more than the conflicts cost: 2000 rows of 25 at 33 x 50 174 -> 156 us, forward
// and backward of 400 rows of 250 at 32 x 32 474 -> 452 us; at 128 wide it frees nothing (2290 -> 2400 us for
// 100 rows of 1000, 8 heads).
template <typename T> constexpr int key_row(int KP, int VP) {
  return KP + (sizeof(T) == 4 && KP < 128 && VP < 128 ? 8 : 16);
}

template <typename T> constexpr int chunk_tokens() { return sizeof(T) == 2 ? 64 : 32; }

// Rows are cut into segments of L = 2^shift tokens, which run side by side. Row b's segments have the
// slots row_ptr[b] / L + b onwards: at least as many as it has segments, one for an empty row, and
// never another row's. The segments that are not their row's last, whose states the later ones need,
// have the entries row_ptr[b] / L onwards, again never another row's. States are kept by entry (a batch of
// short rows has few): at first of the entry's segment alone, then before the segment after it.
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

// The places of all slots and the slots of all entries (-1: none), one wave a row. Where there are
// more rows than one step of the search covers, a block's search took about 4 us of a few chunks'
// work (35 000 blocks of 4096 rows: 170 us), and this table one launch of 5 us for all of them.
constexpr int64_t kSearchedRows = 64;
__global__ __launch_bounds__(256) void k_places(const int64_t *__restrict__ row_ptr, int64_t row0,
                                                int64_t n_rows, int64_t n_tokens, int shift, int64_t n_slots,
                                                int64_t n_entries, Place *__restrict__ places,
                                                int32_t *__restrict__ entries) {
  const int64_t row = row0 + (int64_t)blockIdx.x * 4 + threadIdx.x / 64;
  if (row >= n_rows) return;
  const int lane = (int)threadIdx.x & 63;
  Place p;
  p.row = (int32_t)row;
  p.first = clamped(row_ptr[row], 0, n_tokens);
  p.len = (int32_t)(clamped(row_ptr[row + 1], p.first, n_tokens) - p.first);
  const int64_t e0 = p.first >> shift, s0 = e0 + row, n = segments_of(p.len, shift);
  const int64_t e1 = row + 1 == n_rows ? n_entries : (p.first + p.len) >> shift;
  const int64_t s1 = row + 1 == n_rows ? n_slots : e1 + row + 1;
  for (int64_t s = (row ? s0 : 0) + lane; s < s1 && s < n_slots; s += 64) {
    p.segment = s - s0;
    places[s] = p;
  }
  for (int64_t e = (row ? e0 : 0) + lane; e < e1 && e < n_entries; e += 64)
    entries[e] = e >= e0 && e - e0 + 1 < n ? (int32_t)(s0 + e - e0) : -1;
}

// Passes of one launch, whose blocks alternate: those that read the same tensors run side by side.
struct Args {
  AttentionPass p[3];
  int n;
  int kp, vp;       // widths of the state that all of them are compiled for
  int shift;        // log2 of the tokens a segment
  int64_t slot0;    // first slot (or entry) of this launch
  int64_t n_slots;
  const Place *places;     // nullable: searched for
  const int32_t *entries;
};

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

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
  struct alignas(16) Piece { T v[E]; };
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
#pragma unroll
      for (int e = 0; e < E; ++e) held[i].v[e] = (T)0.f;
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
      Piece p;
#pragma unroll
      for (int e = 0; e < E; ++e)
        p.v[e] = r < x.size && c + e < x.width ? ((const T *)x.at(r, 0))[e] : (T)0.f;
      return p;
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

// Waves a SIMD to compile for: four (128 registers), two where few threads hold the pieces of a chunk,
// and never more than LDS has room for.
template <typename T> constexpr int waves_for(int KP, int VP) {
  constexpr int C = chunk_tokens<T>(), NT = C / 16;
  const int bytes = kParts<T> * 4 * C * key_row<T>(KP, VP) + kReadParts<T> * NT * (NT + 1) * 256 +
                    C * padded<T>(VP) * (int)sizeof(T);
  const int room = (160 * 1024 / bytes * (VP / 16) + 3) / 4;
  const int most = VP == 32 ? 2 : 4;
  return room < most ? room : most;
}

// One block: one head of one segment. STATES: only the state after the segment, for all segments of
// a row but its last.
//
// What bounds it: vector instructions above all, and the chain of a wave's chunk (LDS writes, barrier,
// weights, barrier, products, update) that the other blocks of its CU have to cover: four of four waves for
// bf16 at 64 wide. Measured there, 4096 rows of 263 tokens, 8 heads: 1350 us forward (q, k, v and o move at
// 3.3 TB/s of a copy's 4.8), 2910 us for the three passes backward (the seven tensors at 2.6 TB/s); vector
// instructions issue in 72 and 82 % of the SIMDs' cycles, MFMA is busy in 25 and 29 %. The passes backward
// read past L2 what each of them needs (9.9 GB), since a row's three blocks lie on three XCDs. One row of
// 62496: 63 us after 27 us of states. f32 at 128 wide, 100 rows of 1000, 8 heads to 2 key heads: 570 us
// forward, 1480 us backward (issue 69 and 70 %, MFMA 42 %) at two blocks a CU, which LDS allows. One chunk
// a row (2000 f32 rows of 25 at 33 x 50): 119 us, the latency of a block from its first load to its last
// store, four blocks a CU.
template <typename T, int KP, int VP, bool STATES, bool VEC>
__global__ __launch_bounds__(VP * 4, waves_for<T>(KP, VP)) void k_attention(Args A) {
  constexpr int C = chunk_tokens<T>(), NT = C / 16, NW = VP / 16, THREADS = NW * 64;
  constexpr int KT = KP / 16, KF = KP / 32, SF = C / 32, LK = key_row<T>(KP, VP), LV = padded<T>(VP);
  constexpr int PT = NT * (NT + 1) / 2, NP = kParts<T>, RP = kReadParts<T>, KPART = C * LK;
  using V4 = typename Vec4<T>::type;
  using TK = Tile<T, C, KP, THREADS, VEC>;
  using TV = Tile<T, C, VP, THREADS, VEC>;
  __shared__ __align__(16) bf16 lq[STATES ? 1 : NP * KPART];
  __shared__ __align__(16) bf16 lk[NP * KPART];
  __shared__ __align__(16) T lv[C * LV];
  __shared__ __align__(16) bf16 lp[STATES ? 1 : PT * RP * 256];  // by tile, part, lane

  const AttentionPass &P = A.p[blockIdx.x % (unsigned)A.n];
  const unsigned block = blockIdx.x / (unsigned)A.n;
  const int lane0 = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
  const int lane = lane0, g = lane >> 4, m = lane & 15;
  const int64_t index = A.slot0 + block / P.heads;
  const int head = (int)(block % P.heads);
  Place at;
  if (STATES) {
    if (A.places) {
      const int32_t slot = A.entries[index];
      if (slot < 0 || slot >= A.n_slots) return;
      at = A.places[slot];
    } else {
      at = find_place<true>(P.row_ptr, P.n_rows, P.n_tokens, A.shift, index, lane);
    }
  } else {
    at = A.places ? A.places[index]
                  : find_place<false>(P.row_ptr, P.n_rows, P.n_tokens, A.shift, index, lane);
  }
  // where row_ptr decreases, two rows write a place, in any mixture: nothing is taken from it unchecked
  if (at.row < 0 || at.row >= P.n_rows || at.first < 0 || at.len < 0 ||
      at.first + at.len > P.n_tokens)
    return;
  const int64_t L = 1LL << A.shift, n_segments = segments_of(at.len, A.shift);
  const bool last = at.segment == (n_segments > 0 ? n_segments - 1 : 0);
  if (at.segment < 0 || at.segment >= (n_segments > 0 ? n_segments : 1) || (STATES && last)) return;

  const float raw = P.log_decay[head];
  // a decay above one (or NaN) has no meaning here: its head becomes NaN
  const float a2 = (raw <= 0.f ? fmaxf(raw, kMinLogDecay) : __builtin_nanf("")) * kLog2e;
  const int read_off = P.reverse ? 0 : 1, add_off = P.reverse ? 1 : 0;

  const int64_t begin = at.segment << A.shift;
  const int count = (int)(begin + L < at.len ? L : at.len - begin);  // tokens
  const int flip = P.reverse ? C - 1 : 0;
  const int64_t token0 = P.reverse ? at.first + at.len - begin - C : at.first + begin;
  const int64_t q_row = P.q.token_stride * (int)sizeof(T), k_row = P.k.token_stride * (int)sizeof(T),
                v_row = P.v.token_stride * (int)sizeof(T),
                out_row = (int64_t)P.heads * P.v_width * (P.out_f32 ? 4 : (int)sizeof(T));
  const char *q = (const char *)((const T *)P.q.data + head / P.q_group * P.q.head_stride);
  const char *k = (const char *)((const T *)P.k.data + head / P.group * P.k.head_stride);
  const char *v = (const char *)((const T *)P.v.data + head / P.v_group * P.v.head_stride);

  TK hq, hk;
  TV hv;
  const auto rows_of = [&](auto &tile, const char *x, int64_t bytes, int width, int c) {
    using Rows = typename std::remove_reference<decltype(tile)>::type::Rows;
    return Rows{x + (token0 + (P.reverse ? -c : c)) * bytes, (uint32_t)bytes, flip,
                count - c < C ? count - c : C, width};
  };
  const auto fetch = [&](int c, int tid) {
    if (!STATES) hq.fetch(rows_of(hq, q, q_row, P.k_width, c), tid);
    hk.fetch(rows_of(hk, k, k_row, P.k_width, c), tid);
    hv.fetch(rows_of(hv, v, v_row, P.v_width, c), tid);
  };
  if (count > 0) fetch(0, (int)threadIdx.x);

  // the state: tile kt holds rows state_row(kt, g, e) of its column 16 wave + m
  f32x4 S[KT];
  const int64_t state = ((int64_t)at.row * P.heads + head) * (int64_t)P.k_width * P.v_width;
  const int col = wave * 16 + m;
  // an entry's: row r, column c at r * segment_ld[0] + c * segment_ld[1]. This segment's own or, for
  // outputs, the one before it; at.first + at.len <= n_tokens keeps it below n_tokens >> shift.
  const int64_t entry = (at.first >> A.shift) + at.segment - (STATES ? 0 : 1);
  float *entry_state = P.segments + (entry * P.heads + head) * (int64_t)(KP * VP);
  const auto in_entry = [&](int kt, int e) {
    return (unsigned)(state_row(kt, g, e) * P.segment_ld[0] + col * P.segment_ld[1]);
  };
#pragma unroll
  for (int kt = 0; kt < KT; ++kt) S[kt] = f32x4{0.f, 0.f, 0.f, 0.f};
  if (at.segment > 0 && !STATES) {
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int e = 0; e < 4; ++e) S[kt][e] = entry_state[in_entry(kt, e)];
  } else if (at.segment == 0 && P.first_state) {
    const float *from = P.first_state + state;
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int r = state_row(kt, g, e);
        if (r < P.k_width && col < P.v_width)
          S[kt][e] = from[(unsigned)(r * P.first_ld[0] + col * P.first_ld[1])];
      }
  }

  // Powers of the decay. Exponents are split into parts that are never negative, so that no factor
  // exceeds one: e^{a n} may be zero while e^{-a n} is infinite.
  float near[4], diag[4];  // e^{a (3 - e)}; weight_scale e^{a (m - 4 g - e)}
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    near[e] = exp2_fast(a2 * (float)(3 - e));
    diag[e] = P.weight_scale * exp2_fast(a2 * (float)(m >= g * 4 + e ? m - g * 4 - e : 0));
  }

  // of the tokens 16 n + 4 g + e of a chunk of `size` in the state's update. A full chunk's are held,
  // where the state leaves the registers for it.
  constexpr bool HELD = KP < 128 && NP == 1;
  const auto for_update = [&](int n, int size, int g) {
    f32x4 w;
    if (size == C) {
      const float far = P.update_scale * exp2_fast(a2 * (float)(C - 4 - n * 16 - g * 4 + add_off));
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = far * near[e];
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int left = size - 1 - n * 16 - g * 4 - e;  // below 0: no token, v is zero
        w[e] = P.update_scale * exp2_fast(a2 * (float)((left > 0 ? left : 0) + add_off));
      }
    }
    return w;
  };
  f32x4 add[HELD ? 2 * SF : 1];
  if constexpr (HELD) {
#pragma unroll
    for (int n = 0; n < 2 * SF; ++n) add[n] = for_update(n, C, g);
  }

  for (int c = 0; c < count; c += C) {
    const int size = count - c < C ? count - c : C;
    const int64_t low = token0 + (P.reverse ? -c : c);
    // addresses are formed anew in each chunk: held across chunks, as the compiler would by itself,
    // they cost a wave its place on the SIMD (53 registers spilled at four waves)
    int lane = lane0, tid = (int)threadIdx.x;
    asm volatile("" : "+v"(lane), "+v"(tid));
    const int g = lane >> 4, m = lane & 15;
    __syncthreads();
    if (!STATES) hq.put_parts(lq, LK, rows_of(hq, q, q_row, P.k_width, c), tid);
    hk.put_parts(lk, LK, rows_of(hk, k, k_row, P.k_width, c), tid);
    hv.put(lv, LV, rows_of(hv, v, v_row, P.v_width, c), tid);
    __syncthreads();
    if (c + C < count) fetch(c + C, tid);

    if (!STATES) {
      // weights of places i (columns) and j (rows) <= i, one 16 x 16 tile at a time
#pragma unroll 1
      for (int tile = wave; tile < PT; tile += NW) {
        const int i = tile < 1 ? 0 : tile < 3 ? 1 : tile < 6 ? 2 : 3, j = tile - i * (i + 1) / 2;
        f32x4 w = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int d = 0; d < KF; ++d)
          w = mma(frag_row<NP>(lk + j * 16 * LK + d * 32, LK, KPART, lane),
                  frag_row<NP>(lq + i * 16 * LK + d * 32, LK, KPART, lane), w);
        if (i == j) {
#pragma unroll
          for (int e = 0; e < 4; ++e) w[e] = m >= g * 4 + e ? w[e] * diag[e] : 0.f;
        } else {
          const float far = P.weight_scale * exp2_fast(a2 * (float)(16 * (i - j) + m - g * 4 - 3));
#pragma unroll
          for (int e = 0; e < 4; ++e) w[e] *= far * near[e];
        }
        bf16x4 part[RP];
        as_parts<RP>(w, part);
#pragma unroll
        for (int n = 0; n < RP; ++n) *(bf16x4 *)(lp + (tile * RP + n) * 256 + lane * 4) = part[n];
      }
      __syncthreads();
    }
    Column<T> vc[SF];  // column `col` of v
#pragma unroll
    for (int s = 0; s < SF; ++s) vc[s].read(lv + s * 32 * LV + wave * 16, LV, lane);
    if (!STATES) {
      // 0 * inf and 0 * NaN are NaN: values of v that are neither enter the products as zeros, and
      // are added to their own and later places alone
      bool mine = true;
#pragma unroll
      for (int s = 0; s < SF; ++s) mine = mine && vc[s].finite();
      const bool all_finite = !__any(!mine);
      if (!all_finite) {
#pragma unroll
        for (int s = 0; s < SF; ++s)
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (vc[s].get(e) * 0.f != 0.f) vc[s].clear(e);
      }
      const bf16x4 zero = {(bf16)0.f, (bf16)0.f, (bf16)0.f, (bf16)0.f};
      const int c0 = wave * 16 + g * 4;
      // rows c0 + e of v, column 16 i + m: what the state before the chunk gives, 32 rows of the state at
      // a time
      Frag<NP> vf[SF];
      f32x4 all[NT];
#pragma unroll
      for (int i = 0; i < NT; ++i) all[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int d = 0; d < KF; ++d) {
        const Frag<RP> sf = as_frag<RP>(S[2 * d], S[2 * d + 1]);
        const auto q_of = [&](int i) { return frag_row<NP>(lq + i * 16 * LK + d * 32, LK, KPART, lane); };
        if constexpr (NP == 1) {  // two tiles side by side: a product waits for the one before it of its tile
#pragma unroll
          for (int i = 0; i < NT; i += 2) {
            const Frag<NP> q0 = q_of(i), q1 = q_of(i + 1);
#pragma unroll
            for (int n = RP - 1; n >= 0; --n) {
              all[i] = mma(sf.p[n], q0.p[0], all[i]);
              all[i + 1] = mma(sf.p[n], q1.p[0], all[i + 1]);
            }
          }
        } else {
#pragma unroll
          for (int i = 0; i < NT; ++i) all[i] = mma(sf, q_of(i), all[i]);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int s = 0; s < SF; ++s) vf[s] = vc[s].frag();
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        f32x4 o = all[i];
        o *= P.read_scale * exp2_fast(a2 * (float)(16 * i + m + read_off));
#pragma unroll
        for (int s = 0; s <= i / 2; ++s) {
          const bf16 *t = lp + (i * (i + 1) / 2 + 2 * s) * RP * 256 + lane * 4;
          Frag<RP> pf;
#pragma unroll
          for (int n = 0; n < RP; ++n)
            pf.p[n] = joined(*(const bf16x4 *)(t + n * 256),
                             2 * s + 1 <= i ? *(const bf16x4 *)(t + (RP + n) * 256) : zero);
          o = mma(vf[s], pf, o);
        }
        const int place = 16 * i + m;
        if (!all_finite) {
#pragma unroll 1
          for (int j = 0; j <= place; ++j) {
            const bf16 *t = lp + (i * (i + 1) / 2 + j / 16) * RP * 256 + (m + j % 16 / 4 * 16) * 4 + j % 4;
            float w = 0.f;
#pragma unroll
            for (int n = RP - 1; n >= 0; --n) w += (float)t[n * 256];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float x = (float)lv[j * LV + c0 + e];
              if (x * 0.f != 0.f) o[e] = fmaf(w, x, o[e]);
            }
          }
        }
        if (place < size && c0 < P.v_width) {
          char *to = (char *)P.out + low * out_row + (int64_t)head * P.v_width * (P.out_f32 ? 4 : (int)sizeof(T));
          to += (uint32_t)(place ^ flip) * (uint32_t)out_row + c0 * (P.out_f32 ? 4 : (int)sizeof(T));
          if (c0 + 4 <= P.v_width) {  // at any alignment of the type
            const V4 r = __builtin_convertvector(o, V4);
            if (P.out_f32) __builtin_memcpy(to, &o, 16);
            else __builtin_memcpy(to, &r, sizeof r);
          } else {
#pragma unroll
            for (int e = 0; e < 3; ++e)
              if (c0 + e < P.v_width) {
                if (P.out_f32) ((float *)to)[e] = o[e];
                else ((T *)to)[e] = (T)o[e];
              }
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      if (!all_finite) {
#pragma unroll
        for (int s = 0; s < SF; ++s) vc[s].read(lv + s * 32 * LV + wave * 16, LV, lane);
      }
    }

    // S <- e^{a size} S + sum_j k_j (e^{a (size - 1 - j + add_off)} update_scale v_j)^T
    const float whole = exp2_fast(a2 * (float)size);
    if constexpr (HELD) {
      if (size < C) {
#pragma unroll
        for (int n = 0; n < 2 * SF; ++n) add[n] = for_update(n, size, g);
      }
    }
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) S[kt] *= whole;
#pragma unroll
    for (int s = 0; s < SF; ++s) {
      f32x4 w[2];
      if constexpr (HELD) {
        w[0] = add[2 * s];
        w[1] = add[2 * s + 1];
      } else {
        w[0] = for_update(2 * s, size, g);
        w[1] = for_update(2 * s + 1, size, g);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        w[0][e] *= vc[s].get(e);
        w[1][e] *= vc[s].get(4 + e);
      }
      const Frag<3> x = as_frag<3, NP == 1>(w[0], w[1]);
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) {
        const Frag<NP> kf =
            frag_col<NP, 8>(lk + s * 32 * LK + kt / 2 * 32 + kt % 2 * 4, LK, KPART, lane);
        if constexpr (NP == 3) {
          S[kt] = mma(kf, x, S[kt]);
        } else {
#pragma unroll
          for (int n = 2; n >= 0; --n) S[kt] = mma(kf.p[0], x.p[n], S[kt]);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  }

  if (STATES) {
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int e = 0; e < 4; ++e) entry_state[in_entry(kt, e)] = S[kt][e];
  } else if (last && P.last_state) {
    float *to = P.last_state + state;
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int r = state_row(kt, g, e);
        if (r < P.k_width && col < P.v_width)
          to[(unsigned)(r * P.last_ld[0] + col * P.last_ld[1])] = S[kt][e];
      }
  }
}

// States after each segment alone -> states before each segment: one block (of blockIdx.y parts) a
// head of a row, one thread four values of the state. Bound by the latency of a long row's reads, 16 at
// a time: 14 us for 8 heads' 121 states of 64 x 64 (32 MB moved); where rows are many, by HBM.
__global__ __launch_bounds__(256) void k_join_segments(float *first_pass, float *second_pass,
                                                       const int64_t *row_ptr, int64_t n_rows,
                                                       int64_t index0, int64_t n_tokens,
                                                       int64_t n_slots, int shift, int heads,
                                                       const float *log_decay, int64_t floats,
                                                       const Place *places, const int32_t *entries) {
  float *segments = blockIdx.z ? second_pass : first_pass;
  int64_t row = index0 + blockIdx.x / heads;
  const int head = (int)(blockIdx.x % heads);
  if (entries) {  // of a row's, the first one's block
    const int32_t at = entries[row];
    if (at < 0 || at >= n_slots || places[at].segment != 0) return;
    row = places[at].row;
    if (row < 0 || row >= n_rows) return;
  }
  const int64_t first = clamped(row_ptr[row], 0, n_tokens);
  const int64_t len = clamped(row_ptr[row + 1], first, n_tokens) - first;
  const int64_t entry = first >> shift, n = segments_of(len, shift) - 1;  // the row's entries
  if (n < 2 || entry + n > n_tokens >> shift) return;
  const float raw = log_decay[head];
  const float a2 = (raw <= 0.f ? fmaxf(raw, kMinLogDecay) : __builtin_nanf("")) * kLog2e;
  const float whole = exp2_fast(a2 * (float)(1 << shift));
  const int64_t stride = heads * floats;
  for (int64_t x = ((int64_t)blockIdx.y * 256 + threadIdx.x) * 4; x < floats;
       x += (int64_t)gridDim.y * 1024) {
    float *p = segments + (entry * heads + head) * floats + x;
    f32x4 state = *(const f32x4 *)p;
    constexpr int kAhead = 16;  // states on their way: the sums wait for each other, the reads need not
    for (int64_t j = 1; j < n; j += kAhead) {
      f32x4 own[kAhead];
#pragma unroll
      for (int i = 0; i < kAhead; ++i)
        own[i] = j + i < n ? *(const f32x4 *)(p + (j + i) * stride) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < kAhead; ++i)
        if (j + i < n) {
          state = state * whole + own[i];
          *(f32x4 *)(p + (j + i) * stride) = state;
        }
    }
  }
}

// The gradients of shared heads: blockIdx.y: of k, of v. A group's heads are other blocks of the pass,
// with decays of their own, so each leaves its part in fp32 and they are added here in their order
// (atomics would change the result from run to run). Bound by HBM: 189 us for 8 heads to 2 of 100 003
// tokens at 128 wide in f32, 5.4 TB/s (a value a thread: 217).
// A thread holds VW neighbouring values of its heads (four or, of widths not a multiple of it, one).
template <typename T, int VW>
__global__ __launch_bounds__(256) void k_sum_groups(const float *__restrict__ of_k,
                                                    const float *__restrict__ of_v, int64_t n_heads,
                                                    int group, int k_width, int v_width,
                                                    T *__restrict__ dk, T *__restrict__ dv) {
  const float *x = blockIdx.y ? of_v : of_k;
  T *out = blockIdx.y ? dv : dk;
  const int width = blockIdx.y ? v_width : k_width;
  using F = float __attribute__((ext_vector_type(VW)));
  using O = T __attribute__((ext_vector_type(VW)));
  const int pieces = width / VW, heads = 256 / pieces;  // of a block
  const int tid = (int)threadIdx.x, mine = tid / pieces, c = tid % pieces * VW;
  if (mine >= heads) return;
  for (int64_t head = (int64_t)blockIdx.x * heads + mine; head < n_heads;
       head += (int64_t)gridDim.x * heads) {
    const float *p = x + head * group * width + c;
    F sum = *(const F *)p;
#pragma unroll 4
    for (int j = 1; j < group; ++j) sum += *(const F *)(p + j * width);
    *(O *)(out + head * width + c) = __builtin_convertvector(sum, O);
  }
}

// One token: S' = e^a S + k v^T, o = scale S'^T q. One block a head of a row; the state is read and
// written once. Thread: VW neighbouring columns, every (256 / lanes)-th row. Bound by HBM: 188 us for
// 4096 rows of 8 heads of 64 x 64, 5.7 TB/s; 4.7 us, a launch, for 8 rows.
template <typename T, int VW>
__global__ __launch_bounds__(256) void k_step(int64_t row0, int heads, int group, int K, int V, als_heads q,
                                              als_heads k, als_heads v,
                                              const float *__restrict__ log_decay, float scale,
                                              const float *state, const int32_t *__restrict__ source,
                                              int64_t n_sources, float *state_out, T *out) {
  __shared__ float lk[128], lq[128], sums[256 * VW];
  const int64_t row = row0 + blockIdx.x / heads;
  const int head = (int)(blockIdx.x % heads), tid = (int)threadIdx.x;
  const T *qp = (const T *)q.data + row * q.token_stride + head * q.head_stride;
  const T *kp = (const T *)k.data + row * k.token_stride + head / group * k.head_stride;
  const T *vp = (const T *)v.data + row * v.token_stride + head / group * v.head_stride;
  if (tid < K) {
    lk[tid] = (float)kp[tid];
    lq[tid] = (float)qp[tid] * scale;
  }
  const int64_t from = source ? source[row] : row;
  const bool ok = from >= 0 && from < n_sources;
  const float raw = log_decay[head];
  const float decay = raw <= 0.f ? exp2_fast(fmaxf(raw, kMinLogDecay) * kLog2e) : __builtin_nanf("");
  const int lanes = (V + VW - 1) / VW, rows = 256 / lanes, c = tid % lanes * VW, r0 = tid / lanes;
  const int64_t size = (int64_t)K * V;
  const float *in = state + ((ok ? from : 0) * heads + head) * size;
  float *to = state_out + (row * heads + head) * size;
  float vv[VW], acc[VW];
#pragma unroll
  for (int e = 0; e < VW; ++e) {
    vv[e] = c + e < V ? (float)vp[c + e] : 0.f;
    acc[e] = 0.f;
  }
  __syncthreads();
  if (r0 < rows) {
    for (int r = r0; r < K; r += rows) {
      float s[VW];
      if constexpr (VW == 4) {
        const f32x4 x = ok ? *(const f32x4 *)(in + r * V + c) : f32x4{} + __builtin_nanf("");
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] = x[e];
      } else {
        s[0] = ok ? in[r * V + c] : __builtin_nanf("");
      }
#pragma unroll
      for (int e = 0; e < VW; ++e) {
        s[e] = fmaf(decay, s[e], lk[r] * vv[e]);
        acc[e] = fmaf(lq[r], s[e], acc[e]);
      }
      if constexpr (VW == 4)
        *(f32x4 *)(to + r * V + c) = f32x4{s[0], s[1], s[2], s[3]};
      else
        to[r * V + c] = s[0];
    }
#pragma unroll
    for (int e = 0; e < VW; ++e) sums[r0 * lanes * VW + c + e] = acc[e];
  }
  __syncthreads();
  if (tid < V) {
    float sum = 0.f;
    for (int r = 0; r < rows; ++r) sum += sums[r * lanes * VW + tid];
    out[(row * heads + head) * V + tid] = (T)sum;
  }
}

int padded_width3(int width) { return width <= 32 ? 32 : width <= 64 ? 64 : 128; }

template <typename T, int KP, int VP> hipError_t launch_kv(Args A, bool split, hipStream_t s) {
  const int heads = A.p[0].heads;
  bool vec = true;
  for (int i = 0; i < A.n; ++i) vec = vec && A.p[i].vec_in;
  const auto each = [&](auto kernel, const Args &all, int64_t places) {
    Args a = all;
    const int64_t per = max_blocks(VP * 4) / (heads * a.n);  // a launch
    for (a.slot0 = 0; a.slot0 < places; a.slot0 += per) {
      const int64_t n = places - a.slot0 < per ? places - a.slot0 : per;
      hipLaunchKernelGGL(kernel, dim3((unsigned)(n * heads * a.n)), dim3(VP * 4), 0, s, a);
    }
  };
  const auto states = [&](const Args &a) {
    each(vec ? k_attention<T, KP, VP, true, true> : k_attention<T, KP, VP, true, false>, a,
         a.p[0].n_tokens >> a.shift);
  };
  const auto outputs = [&](const Args &a) {
    each(vec ? k_attention<T, KP, VP, false, true> : k_attention<T, KP, VP, false, false>, a,
         a.n_slots);
  };
  if (split) {  // the states of those passes that do not take another's
    Args own = A;
    own.n = 0;
    for (int i = 0; i < A.n; ++i)
      if (!A.p[i].shares_segments) own.p[own.n++] = A.p[i];
    states(own);  // of one pass, or two
    const AttentionPass &P = own.p[0];
    const int64_t floats = (int64_t)KP * VP, per = max_blocks(256) / heads;
    // over the rows or, where those are fewer and known, the entries: most rows may be one segment
    const int64_t n_entries = P.n_tokens >> A.shift;
    const bool of_entries = A.places && n_entries < P.n_rows;
    const int64_t count = of_entries ? n_entries : P.n_rows;
    for (int64_t r = 0; r < count; r += per) {
      const int64_t n = count - r < per ? count - r : per;
      // parts of a state: as many as fill the chip, where rows and heads alone do not
      const int64_t parts = n * heads >= 4096 ? 1 : (floats + 1023) / 1024;
      hipLaunchKernelGGL(k_join_segments,
                         dim3((unsigned)(n * heads), (unsigned)parts, (unsigned)own.n), dim3(256), 0, s,
                         P.segments, own.n > 1 ? own.p[1].segments : nullptr, P.row_ptr, P.n_rows, r,
                         P.n_tokens, A.n_slots, A.shift, heads, P.log_decay, floats,
                         of_entries ? A.places : nullptr, of_entries ? A.entries : nullptr);
    }
  }
  outputs(A);
  return hipGetLastError();
}

template <typename T, int KP>
hipError_t launch_k(const Args &A, bool split, hipStream_t s) {
  switch (A.vp) {
    case 32: return launch_kv<T, KP, 32>(A, split, s);
    case 64: return launch_kv<T, KP, 64>(A, split, s);
    default: return launch_kv<T, KP, 128>(A, split, s);
  }
}

template <typename T> hipError_t launch_t(const Args &A, bool split, hipStream_t s) {
  switch (A.kp) {
    case 32: return launch_k<T, 32>(A, split, s);
    case 64: return launch_k<T, 64>(A, split, s);
    default: return launch_k<T, 128>(A, split, s);
  }
}

}  // namespace

// Short segments fill the chip where tokens are few; each costs a pass over its k and v and a state
// written and read. From four chunks up, as many as leave 1024 blocks (bf16: what the chip holds at
// a time) or 2048 (f32, whose chunks are half as long), at most 2048 tokens. Us with segments of 256,
// 512, 1024 and 2048 tokens: one row of 62496 bf16 tokens, 8 heads of 64: 138, 126, 125, 163; forward
// and backward of 4096 such rows of 263: 5700, 4990, 4570, 4430; of 100 f32 rows of 1000, 8 heads of 128
// to 2: 2860, 2630, 2660, 2890, of 1000 f32 rows of 262, 8 heads of 64: 2400, 2200, 2110, 2270; forward
// of 8 bf16 rows of 250: 32, 49, 79, 85.
int attention_shift(als_dtype dtype, int64_t n_tokens, int32_t heads) {
  int shift = dtype == ALS_F32 ? 7 : 8;
  while (shift < 11 && (n_tokens >> shift) * heads > (dtype == ALS_F32 ? 2048 : 1024)) ++shift;
  return shift;
}

AttentionSpace attention_space(als_dtype dtype, int64_t n_tokens, int64_t n_rows, int32_t heads,
                               int k_width, int v_width) {
  const int shift = attention_shift(dtype, n_tokens, heads);
  const int64_t entries = n_tokens >> shift, slots = entries + n_rows;
  AttentionSpace x{};
  if (n_rows > kSearchedRows) {
    x.places = (slots * (int64_t)sizeof(Place) + 15) / 16 * 16;
    x.entries = (entries * 4 + 15) / 16 * 16;
  }
  if (n_tokens > 1LL << shift)  // else no row is longer than a segment
    x.states = entries * heads * padded_width3(k_width) * padded_width3(v_width) * 4;
  return x;
}

hipError_t launch_places(als_dtype dtype, const AttentionPass &p, hipStream_t s) {
  if (!p.places) return hipSuccess;
  const int shift = attention_shift(dtype, p.n_tokens, p.heads);
  const int64_t entries = p.n_tokens >> shift;
  const int64_t per = max_blocks(256) * 4;  // rows a launch
  for (int64_t r = 0; r < p.n_rows; r += per) {
    const int64_t n = p.n_rows - r < per ? p.n_rows - r : per;
    hipLaunchKernelGGL(k_places, dim3((unsigned)((n + 3) / 4)), dim3(256), 0, s, p.row_ptr, r, p.n_rows,
                       p.n_tokens, shift, entries + p.n_rows, entries, (Place *)p.places, p.entries);
  }
  return hipGetLastError();
}

hipError_t launch_attention(als_dtype dtype, const AttentionPass *p, int n, hipStream_t s) {
  if (p[0].n_rows == 0) return hipSuccess;
  Args A{};
  A.shift = attention_shift(dtype, p[0].n_tokens, p[0].heads);
  A.n_slots = (p[0].n_tokens >> A.shift) + p[0].n_rows;
  A.places = (const Place *)p[0].places;
  A.entries = p[0].entries;
  const bool split = p[0].n_tokens > 1LL << A.shift;
  const int size = dtype == ALS_F32 ? 4 : 2;
  // passes over a state and over its transpose share launches at the wider of its widths
  int k = 0, v = 0;
  for (int i = 0; i < n; ++i) {
    k = p[i].k_width > k ? p[i].k_width : k;
    v = p[i].v_width > v ? p[i].v_width : v;
  }
  A.kp = padded_width3(k);
  A.vp = padded_width3(v);
  A.n = n;
  for (int i = 0; i < n; ++i) {
    AttentionPass &x = A.p[i] = p[i];
    const auto vec = [&](const als_heads &h, int width) {
      return aligned16(h.data, h.token_stride, h.head_stride, width, size);
    };
    x.vec_in = vec(x.q, x.k_width) && vec(x.k, x.k_width) && vec(x.v, x.v_width);
    // row-major as the pass that forms them has them, its rows padded
    x.segment_ld[0] = x.shares_segments ? 1 : A.vp;
    x.segment_ld[1] = x.shares_segments ? A.kp : 1;
  }
  return dtype == ALS_F32 ? launch_t<float>(A, split, s) : launch_t<bf16>(A, split, s);
}

hipError_t launch_sum_groups(als_dtype dtype, const float *of_k, const float *of_v, int64_t n_tokens,
                             int32_t heads, int32_t group, int32_t k_width, int32_t v_width, void *dk,
                             void *dv, hipStream_t s) {
  const int64_t n_heads = n_tokens * (heads / group);
  if (n_heads == 0) return hipSuccess;
  const bool vec = (k_width | v_width) % 4 == 0 &&
                   (((uintptr_t)of_k | (uintptr_t)of_v | (uintptr_t)dk | (uintptr_t)dv) % 16 == 0);
  const int wide = (k_width > v_width ? k_width : v_width) / (vec ? 4 : 1);
  const int64_t blocks = (n_heads + 256 / wide - 1) / (256 / wide);
  const dim3 grid((unsigned)(blocks < 8192 ? blocks : 8192), 2);
  const auto sum = [&](auto kernel, auto *k, auto *v) {
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, of_k, of_v, n_heads, group, k_width, v_width, k, v);
  };
  if (dtype == ALS_F32)
    sum(vec ? k_sum_groups<float, 4> : k_sum_groups<float, 1>, (float *)dk, (float *)dv);
  else
    sum(vec ? k_sum_groups<bf16, 4> : k_sum_groups<bf16, 1>, (bf16 *)dk, (bf16 *)dv);
  return hipGetLastError();
}

hipError_t launch_attention_step(als_dtype dtype, int64_t n_rows, int32_t heads, int32_t group,
                                 int32_t k_width, int32_t v_width, const als_heads &q,
                                 const als_heads &k, const als_heads &v, const float *log_decay,
                                 float scale, const float *state, const int32_t *source,
                                 int64_t n_sources, float *state_out, void *out, hipStream_t s) {
  if (n_rows == 0) return hipSuccess;
  const bool vec = v_width % 4 == 0 && ((uintptr_t)state | (uintptr_t)state_out) % 16 == 0;
  const int64_t per = max_blocks(256) / heads;
  for (int64_t r = 0; r < n_rows; r += per) {
    const dim3 grid((unsigned)((n_rows - r < per ? n_rows - r : per) * heads));
    const auto step = [&](auto kernel, auto *to) {
      hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, r, heads, group, k_width, v_width, q, k, v,
                         log_decay, scale, state, source, n_sources, state_out, to);
    };
    if (dtype == ALS_F32)
      step(vec ? k_step<float, 4> : k_step<float, 1>, (float *)out);
    else
      step(vec ? k_step<bf16, 4> : k_step<bf16, 1>, (bf16 *)out);
  }
  return hipGetLastError();
}

}  // namespace als
