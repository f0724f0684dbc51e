// Gradients of the attention over gaps of time (gap.hip). With do the gradient of the outputs, p_ij the
// weights, formed anew from the saved largest scores and sums, and delta_i = do_i . o_i,
//   ds_ij = p_ij (do_i . v_j - delta_i),
//   dq_i = scale sum_j ds_ij k_j,   dk_j = scale sum_i ds_ij q_i,   dv_j = sum_i p_ij do_i,
//   dbias[b] = sum of ds_ij over the pairs whose gap is in bucket b.
//
// Two kernels, each with sums that stay in the registers of the block that owns them, so that no result
// depends on an order of atomics: one over the keys of a block's queries (dq, dbias; it also leaves delta for
// the other), one over the queries of a block's keys and, in turn, of the query heads that share them
// (dk, dv). Scores and do . v are formed in both.
//
// Rounding. Weights and ds enter products in two bf16 parts where the inputs are bf16. delta takes what the
// outputs' rounding left out as well, so that dbias, fp32 whatever the inputs, does not hold it.
#include "gap.h"
#include "internal.h"

namespace als {

namespace {

struct BackArgs {
  GapShape G;
  als_heads q, k, v, d_out;
  const Span2 *spans;
  const void *out;         // packed
  const int16_t *rest;     // nullable
  const float *stats;
  float *delta;            // [heads, n_tokens]
  float *dbias_parts;      // [heads, buckets, n_tiles]
  void *dq, *dk, *dv;      // packed
  float *dk_parts, *dv_parts;  // of each query head [n_tokens, heads, width]; nullable
  int64_t tile0, n_tiles;
  bool vec_rows, vec_out;  // rows read from global memory as operands; out and rest
};

template <typename T> constexpr int tile_tokens() { return sizeof(T) == 2 ? 64 : 32; }
// ---- over keys: dq and dbias ---------------------------------------------------------------------

// Sums by bucket: a column each lane, so that no two lanes add to the same place and the order of a sum's
// terms is that of the program; or, where that would leave a CU one block, a column each two lanes, which add
// one after the other. LDS adds floats by itself at 3 cycles a lane (194 a wave's instruction, where a read and
// a write take 8), so a lane reads, adds and writes: four places at a time, each with what the ones before it
// give the same place, so that the last write to a place has all of them.
template <int COLUMNS> struct BucketSums {
  float *column;
  int lane;
  __device__ __forceinline__ float *at(int kind4) const { return column + kind4 * (COLUMNS / 4); }
  __device__ __forceinline__ void add_now(const i32x4 &kind4, f32x4 x) const {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] += *at(kind4[e]);
#pragma unroll
    for (int e = 0; e < 4; ++e) *at(kind4[e]) = x[e];
  }
  __device__ __forceinline__ void add(const i32x4 &kind4, f32x4 x) const {
    x[1] += kind4[1] == kind4[0] ? x[0] : 0.f;
    x[2] += kind4[2] == kind4[1] ? x[1] : kind4[2] == kind4[0] ? x[0] : 0.f;
    x[3] += kind4[3] == kind4[2] ? x[2] : kind4[3] == kind4[1] ? x[1] : kind4[3] == kind4[0] ? x[0] : 0.f;
    if constexpr (COLUMNS == 64) {
      add_now(kind4, x);
    } else {
      if (lane < 32) add_now(kind4, x);
      asm volatile("" ::: "memory");  // one half of the wave after the other
      if (lane >= 32) add_now(kind4, x);
    }
  }
  __device__ __forceinline__ void add(int kind, float x) const {
    if (COLUMNS == 64 || lane < 32) *at(kind * 4) += x;
    asm volatile("" ::: "memory");
    if (COLUMNS == 32 && lane >= 32) *at(kind * 4) += x;
  }
};

// One block: 64 queries of a head.
//
// What bounds it: vector instructions (about 20 a score where a tile has several buckets, 9 where it has one) and
// waits, at two barriers a tile and at the reads before each write of dbias's sums, with the three blocks a CU (two
// at 128 wide) that registers and LDS allow. Measured: 1 075 431 bf16 tokens of 4096 rows, 8 heads of 64, 7.1 ms
// (issue 56 %, MFMA 16 %; 128 queries a block, two blocks a CU, took 7.5); four rows of 8000 at 128 wide with 64
// buckets 1.8 ms; fp32 at 128 wide, 25 003 tokens of 100 rows, 670 us, of which its longest row, 3013 tokens, takes
// 405 alone (gap.hip: a block goes through its keys one tile after the other).
template <typename T, int D, bool VEC, typename Entry, int COLUMNS>
__global__ __launch_bounds__(256, D == 128 ? 2 : 3) void k_gap_dq(BackArgs A) {
  constexpr int KN = tile_tokens<T>(), LD = D + 16, PART = KN * LD;
  constexpr int NP = kParts<T>, RP = kReadParts<T>, KS = KN / 32, DF = D / 32, DT = D / 16;
  using Tiles = Staged<T, KN, D, VEC>;
  __shared__ __align__(16) bf16 lk[NP * PART];
  __shared__ __align__(16) bf16 lv[NP * PART];
  __shared__ __align__(16) int32_t lpos[KN];
  __shared__ int32_t lrange[2], lbad;
  __shared__ Buckets<Entry> lb;
  extern __shared__ float lsums[];  // [waves, buckets, columns]

  const GapShape &G = A.G;
  int tid = (int)threadIdx.x, lane = tid & 63, g = lane >> 4, m = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int head = (int)(blockIdx.x % (unsigned)G.heads);
  const int64_t tile = A.n_tiles - 1 - (A.tile0 + blockIdx.x / (unsigned)G.heads);
  const int64_t t0 = tile * 64;

  lb.start(G, head, tid);
  if (tid == 0) lbad = -1;
  for (int n = tid; n < 4 * G.buckets * COLUMNS; n += 256) lsums[n] = 0.f;
  const int span_first = span_of(G, A.spans, t0 + lane).first;
  const int block_first = __builtin_amdgcn_readfirstlane(wave_min(span_first));
  const int block_last = __builtin_amdgcn_readfirstlane(wave_max(span_first != kNoRow ? (int)t0 + lane : -1));
  const int rows_first = __builtin_amdgcn_readfirstlane(wave_max(span_first));
  float *parts = A.dbias_parts + (int64_t)head * G.buckets * A.n_tiles + tile;
  const int i0 = (int)t0 + wave * 16, at = i0 + m, first = __shfl(span_first, wave * 16 + m);
  if (first == kNoRow) clear_row<T>(G, A.dq, at, G.heads, head, g);
  if (block_last < 0) {
    if (tid < G.buckets) parts[tid * A.n_tiles] = 0.f;
    return;
  }

  // this wave's queries, one a lane
  const bool real = first != kNoRow;
  const unsigned before = real ? (unsigned)(at - first) : 0u;
  const int64_t t = real ? at : block_last;
  const int pos = G.positions[t];
  // The matrix cores round down (not to nearest), which leaves all do . v a little short. That is nothing to
  // one of them, but dbias sums them over all tokens, where their own signs nearly cancel (1 075 431 tokens: off
  // by 3e-6 of its norm). So every other query's do is negated, and what comes of it once more at the end.
  const float sign = m & 1 ? -1.f : 1.f;
  Frag<NP> qf[DF], of[DF];
  load_row<T, D>((const T *)A.q.data + t * A.q.token_stride + head * A.q.head_stride, G.width, A.vec_rows,
                 lane, qf);
  const float *stats = A.stats + (int64_t)head * G.n_tokens + t;
  float top = stats[0], inv = stats[(int64_t)G.heads * G.n_tokens];
  // delta, and do as operands
  float x = 0.f;
  const int64_t row = (t * G.heads + head) * G.width;
#pragma unroll
  for (int d = 0; d < DF; ++d) {
    const int c = d * 32 + g * 8;
    const Raw8<T> y = load8((const T *)A.d_out.data + t * A.d_out.token_stride + head * A.d_out.head_stride,
                            c, G.width, A.vec_rows);
    const Raw8<T> z = load8((const T *)A.out + row, c, G.width, A.vec_out);
    f32x4 o[2] = {low4(z), high4(z)};
    if constexpr (sizeof(T) == 2) {
      if (A.rest) {
        const Raw8<int16_t> r = load8(A.rest + row, c, G.width, A.vec_out);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          o[0][e] = with_rest(z.v[e], r.v[e]);
          o[1][e] = with_rest(z.v[4 + e], r.v[4 + e]);
        }
      }
    }
    const f32x4 lo = low4(y), hi = high4(y);
#pragma unroll
    for (int e = 0; e < 4; ++e) x = fmaf(lo[e], o[0][e], fmaf(hi[e], o[1][e], x));
    of[d] = operand(y);
    if (m & 1) of[d] = negated(of[d]);
    if (G.scale < 0.f) qf[d] = negated(qf[d]);
  }
  float delta = column_sum(x);
  if (g == 0 && real) A.delta[(int64_t)head * G.n_tokens + t] = delta;
  // A sum that is no number would make a masked pair's zero one as well, on its way to dbias: the weights are
  // formed as NaN instead, before the mask.
  if (!(fabsf(inv) <= kLargest)) {
    top = __builtin_nanf("");
    inv = 1.f;
  }
  delta *= sign;
  inv *= sign;  // with the factor of a query's sums
  const int first_min = __builtin_amdgcn_readfirstlane(wave_min(first));
  const int first_max = __builtin_amdgcn_readfirstlane(wave_max(first));
  const int last = __builtin_amdgcn_readfirstlane(wave_max(real ? at : -1));
  const int pos_min = __builtin_amdgcn_readfirstlane(wave_min(pos));
  const int pos_max = __builtin_amdgcn_readfirstlane(wave_max(pos));
  const float scale = fabsf(G.scale) * kLog2e;

  const char *k = (const char *)((const T *)A.k.data + head / G.group * A.k.head_stride);
  const char *v = (const char *)((const T *)A.v.data + head / G.group * A.v.head_stride);
  const int64_t k_row = A.k.token_stride * (int)sizeof(T), v_row = A.v.token_stride * (int)sizeof(T);
  Tiles hk, hv;
  int hpos = 0;
  const auto rows_of = [&](const char *x, int64_t bytes, int k0) {
    return typename Tiles::Rows{x + k0 * bytes, (uint32_t)bytes, 0,
                                 block_last + 1 - k0 < KN ? block_last + 1 - k0 : KN, G.width};
  };
  const auto fetch = [&](int k0) {
    hk.fetch(rows_of(k, k_row, k0), tid);
    hv.fetch(rows_of(v, v_row, k0), tid);
    if (wave == 0) hpos = G.positions[min(k0 + (lane & (KN - 1)), block_last)];
  };
  fetch(block_first);
  __syncthreads();
  lb.fill(G, wave, lane);
  BucketLanes bl;
  bl.read(lb, G, lane);

  f32x4 dq[DT];
#pragma unroll
  for (int c = 0; c < DT; ++c) dq[c] = f32x4{0.f, 0.f, 0.f, 0.f};
  const BucketSums<COLUMNS> sums{lsums + wave * G.buckets * COLUMNS + (lane & (COLUMNS - 1)), lane};
  // of the tiles so far whose gaps were all in bucket run_kind, before the query's own factor
  float run = 0.f;
  int run_kind = 0;
  int bad_lo = 0, bad_hi = 0;  // keys among which some values were left out
  const auto end_run = [&]() {
    sums.add(run_kind, fmaf(run, inv, 0.f));  // one rounding before the sum's own
    run = 0.f;
  };

  for (int k0 = block_first; k0 <= block_last; k0 += KN) {
    // addresses are formed anew in each tile: held across tiles they cost registers
    asm volatile("" : "+v"(tid));
    tid &= 255;
    lane = tid & 63;
    g = lane >> 4;
    __syncthreads();
    const bool masked = k0 + KN - 1 > (int)t0 || k0 < rows_first;
    if (masked && hk.nonfinite(rows_of(k, k_row, k0), tid)) lbad = k0;
    hk.put_parts(lk, LD, rows_of(k, k_row, k0), tid);
    hv.put_parts(lv, LD, rows_of(v, v_row, k0), tid);
    if (wave == 0) {
      const int lo = wave_min(hpos), hi = wave_max(hpos);
      if (lane < KN) lpos[lane] = hpos;
      if (lane == 0) {
        lrange[0] = lo;
        lrange[1] = hi;
      }
    }
    __syncthreads();
    const bool bad = masked && __builtin_amdgcn_readfirstlane(lbad) == k0;
    if (bad) {
      bad_lo = bad_hi ? bad_lo : k0;
      bad_hi = min(k0 + KN, block_last + 1);
    }
    if (k0 + KN <= block_last) fetch(k0 + KN);
    if (k0 > last || k0 + KN <= first_min) continue;

    const bool partial = k0 + KN - 1 > i0 || k0 < first_max;
    const int one = bl.kind(gap_of(pos_min, lrange[1]), gap_of(pos_max, lrange[0]));
    const float b = bl.bias_of(one);
    const bool plain = bl.is_plain(one) && !partial;
    if (plain && one != run_kind) {
      end_run();
      run_kind = one;
    }
#pragma unroll 1
    for (int w = 0; w < KS; ++w) {  // 32 keys at a time
      const bf16 *wk = lk + w * 32 * LD, *wv = lv + w * 32 * LD;
      f32x4 s[2], dp[2];  // do . v - delta
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        Acc<NP> qk, ov;
        qk.start(f32x4{0.f, 0.f, 0.f, 0.f});
        ov.start(f32x4{0.f, 0.f, 0.f, 0.f} - delta);
#pragma unroll
        for (int d = 0; d < DF; ++d) {
          const Frag<NP> kf = frag_row<NP>(wk + t * 16 * LD + d * 32, LD, PART, lane);
          const Frag<NP> vf = frag_row<NP>(wv + t * 16 * LD + d * 32, LD, PART, lane);
          qk.add(kf, qf[d]);
          ov.add(vf, of[d]);
        }
        s[t] = qk.value();
        dp[t] = ov.value();
      }
      if (plain) {
        const float shift = b - top;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float p = exp2_fast(fmaf(s[t][e], scale, shift));
            s[t][e] = p * dp[t][e];
            run += s[t][e];
          }
      } else {
        i32x4 kind[2];
        f32x4 add[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const i32x4 kpos = *(const i32x4 *)(lpos + w * 32 + t * 16 + g * 4);
#pragma unroll
          for (int e = 0; e < 4; ++e) kind[t][e] = lb.kind4(G, gap_of(pos, kpos[e]));
        }
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) add[t][e] = lb.bias4(kind[t][e]);
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float p = exp2_fast(fmaf(s[t][e], scale, add[t][e]) - top);
            const bool kept = (unsigned)(k0 + w * 32 + t * 16 + g * 4 + e - first) <= before;
            s[t][e] = kept ? p * dp[t][e] : 0.f;
          }
#pragma unroll
        for (int t = 0; t < 2; ++t) sums.add(kind[t], s[t] * inv);
      }
      const Frag<RP> df = as_frag<RP>(s[0], s[1]);
#pragma unroll
      for (int c = 0; c < DT; ++c) {
        Frag<NP> kf = frag_col<NP, 4>(wk + c * 16, LD, PART, lane);
        if (bad) kf = cleaned(kf);
        dq[c] = mma(kf, df, dq[c]);
      }
    }
  }

  if (real) {
    if (bad_hi)
      mark_read<T, DT>((const T *)k, A.k.token_stride, G.width, bad_lo, bad_hi, lane,
                       [&](int j) { return (unsigned)(j - first) <= before; }, dq);
    T *to = (T *)A.dq + ((int64_t)at * G.heads + head) * G.width;
#pragma unroll
    for (int c = 0; c < DT; ++c) {
      const int d = c * 16 + g * 4;
      if (d < G.width) store4(to + d, dq[c] * (G.scale * inv), G.width - d);
    }
  }
  end_run();
  __syncthreads();
  // four threads a bucket, a wave's columns each
  for (int n = tid; n < 4 * G.buckets; n += 256) {
    const float *x = lsums + ((n & 3) * G.buckets + n / 4) * COLUMNS;
    double sum = 0.0;
    for (int c = 0; c < COLUMNS; ++c) sum += (double)x[(c + n) & (COLUMNS - 1)];
    sum += __shfl_xor(sum, 1);
    sum += __shfl_xor(sum, 2);
    if ((n & 3) == 0) parts[n / 4 * A.n_tiles] = (float)sum;
  }
}

// dbias[h, b]: the blocks' parts, in fp64. One block a head and bucket. 27 us for 16 804 parts of 8 heads and
// 32 buckets (17 MB): the latency of 66 reads a thread.
__global__ __launch_bounds__(256) void k_gap_dbias(const float *__restrict__ parts, int64_t n_tiles,
                                                   float *__restrict__ dbias) {
  __shared__ double sums[4];
  const float *x = parts + blockIdx.x * n_tiles;
  double sum = 0.0;
  for (int64_t t = threadIdx.x; t < n_tiles; t += 256) sum += (double)x[t];
#pragma unroll
  for (int n = 1; n < 64; n <<= 1) sum += __shfl_xor(sum, n);
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x / 64] = sum;
  __syncthreads();
  if (threadIdx.x == 0) dbias[blockIdx.x] = (float)(sums[0] + sums[1] + (sums[2] + sums[3]));
}

// ---- over queries: dk and dv ---------------------------------------------------------------------

// One block: 64 keys of a key head, or of one of its query heads.
//
// What bounds it: vector instructions (13 a score where a tile has one bucket) with four products on MFMA, two of
// them of two parts. Measured: 1 075 431 bf16 tokens of 4096 rows, 8 heads of 64, 7.0 ms (issue 63 %, MFMA 26 %,
// three blocks a CU; 128 keys a block took 8.6); four rows of 8000 at 128 wide 2.0 ms; fp32 at 128 wide, 25 003
// tokens of 100 rows, 8 heads to 2, 720 us (MFMA 40 %, issue 41 %; 16 registers spilled).
template <typename T, int D, bool VEC, typename Entry>
__global__ __launch_bounds__(256, 2) void k_gap_dkv(BackArgs A) {
  constexpr int QN = tile_tokens<T>(), BK = 64, LD = D + 16, PART = QN * LD;
  constexpr int NP = kParts<T>, RP = kReadParts<T>, QS = QN / 32, DF = D / 32, DT = D / 16;
  // A query's factor of the weights goes into the exponent, a product less a weight: off by 2^-24 of the exponent's
  // parts, the largest score (as the score is itself) and the logarithm of the sum, which bf16 does not see.
  constexpr bool LOG = sizeof(T) == 2;
  using Tiles = Staged<T, QN, D, VEC>;
  __shared__ __align__(16) bf16 lq[NP * PART];
  __shared__ __align__(16) bf16 lo[NP * PART];
  __shared__ __align__(16) int32_t lpos[QN];
  __shared__ __align__(16) float ltop[QN], linv[QN], ldelta[QN];
  __shared__ int32_t lrange[2], lbad;
  __shared__ Buckets<Entry> lb;

  const GapShape &G = A.G;
  int tid = (int)threadIdx.x, lane = tid & 63, g = lane >> 4, m = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // a key head and its query heads in turn, or one query head
  const int k_heads = G.heads / G.group, owners = A.dk_parts ? G.heads : k_heads;
  const int owner = (int)(blockIdx.x % (unsigned)owners);
  const int k_head = A.dk_parts ? owner / G.group : owner;
  const int head0 = A.dk_parts ? owner : k_head * G.group, head1 = A.dk_parts ? owner + 1 : head0 + G.group;
  const int64_t t0 = (A.tile0 + blockIdx.x / (unsigned)owners) * BK;

  // the block's queries: from its first token that has a row to its last row's end
  const int span_end = span_of(G, A.spans, t0 + lane).end;
  const int block_first = __builtin_amdgcn_readfirstlane(wave_min(span_end > 0 ? (int)t0 + lane : kNoRow));
  const int block_end = __builtin_amdgcn_readfirstlane(wave_max(span_end));
  const int rows_end = __builtin_amdgcn_readfirstlane(wave_min(span_end));  // the first row's
  const int j0 = (int)t0 + wave * 16, at = j0 + m, end = __shfl(span_end, wave * 16 + m);
  if (end == 0 && !A.dk_parts) {
    clear_row<T>(G, A.dk, at, owners, owner, g);
    clear_row<T>(G, A.dv, at, owners, owner, g);
  }
  if (block_end == 0) return;

  // this wave's keys, one a lane
  const unsigned after = end > 0 ? (unsigned)(end - at) : 0u;  // queries from the key on
  const int64_t t = end > 0 ? at : block_first;
  const int pos = G.positions[t];
  Frag<NP> kf[DF], vf[DF];
  load_row<T, D>((const T *)A.k.data + t * A.k.token_stride + k_head * A.k.head_stride, G.width, A.vec_rows,
                 lane, kf);
  load_row<T, D>((const T *)A.v.data + t * A.v.token_stride + k_head * A.v.head_stride, G.width, A.vec_rows,
                 lane, vf);
  if (G.scale < 0.f) {
#pragma unroll
    for (int d = 0; d < DF; ++d) kf[d] = negated(kf[d]);
  }
  const int end_min = __builtin_amdgcn_readfirstlane(wave_min(end));
  const int end_max = __builtin_amdgcn_readfirstlane(wave_max(end));
  const int pos_min = __builtin_amdgcn_readfirstlane(wave_min(pos));
  const int pos_max = __builtin_amdgcn_readfirstlane(wave_max(pos));
  const float scale = fabsf(G.scale) * kLog2e;
  const int64_t q_row = A.q.token_stride * (int)sizeof(T), o_row = A.d_out.token_stride * (int)sizeof(T);

  f32x4 dk[DT], dv[DT];
#pragma unroll
  for (int c = 0; c < DT; ++c) dk[c] = dv[c] = f32x4{0.f, 0.f, 0.f, 0.f};

  for (int head = head0; head < head1; ++head) {
    __syncthreads();
    if (tid == 0) lbad = -1;
    int bad_lo = 0, bad_hi = 0;  // queries among which some values were left out
    lb.start(G, head, tid);
    __syncthreads();
    if (Buckets<Entry>::DIRECT || head == head0) lb.fill(G, wave, lane);
    BucketLanes bl;
    bl.read(lb, G, lane);
    const char *q = (const char *)((const T *)A.q.data + head * A.q.head_stride);
    const char *o = (const char *)((const T *)A.d_out.data + head * A.d_out.head_stride);
    const float *stats = A.stats + (int64_t)head * G.n_tokens;
    const float *inv_stats = stats + (int64_t)G.heads * G.n_tokens;
    const float *deltas = A.delta + (int64_t)head * G.n_tokens;
    Tiles hq, ho;
    int hpos = 0;
    float hstat = 0.f;
    const auto rows_of = [&](const char *x, int64_t bytes, int q0) {
      return typename Tiles::Rows{x + q0 * bytes, (uint32_t)bytes, 0,
                                   block_end - q0 < QN ? block_end - q0 : QN, G.width};
    };
    const auto fetch = [&](int q0) {
      hq.fetch(rows_of(q, q_row, q0), tid);
      ho.fetch(rows_of(o, o_row, q0), tid);
      const int t = min(q0 + (lane & (QN - 1)), block_end - 1);
      if (wave == 0) hpos = G.positions[t];
      if (wave == 1) hstat = stats[t];
      if (wave == 2) hstat = LOG ? __log2f(inv_stats[t]) : inv_stats[t];
      if (wave == 3) hstat = -deltas[t];
    };
    fetch(block_first);

    for (int q0 = block_first; q0 < block_end; q0 += QN) {
      asm volatile("" : "+v"(tid));  // as above
      tid &= 255;
      lane = tid & 63;
      g = lane >> 4;
      __syncthreads();
      const bool masked = q0 < (int)t0 + BK - 1 || q0 + QN > rows_end;  // for some key of the block
      if (masked && (hq.nonfinite(rows_of(q, q_row, q0), tid) || ho.nonfinite(rows_of(o, o_row, q0), tid))) lbad = q0;
      hq.put_parts(lq, LD, rows_of(q, q_row, q0), tid);
      ho.put_parts(lo, LD, rows_of(o, o_row, q0), tid);
      if (wave == 0) {
        const int low = wave_min(hpos), high = wave_max(hpos);
        if (lane < QN) lpos[lane] = hpos;
        if (lane == 0) {
          lrange[0] = low;
          lrange[1] = high;
        }
      } else if (lane < QN) {
        (wave == 1 ? ltop : wave == 2 ? linv : ldelta)[lane] = hstat;
      }
      __syncthreads();
      const bool bad = masked && __builtin_amdgcn_readfirstlane(lbad) == q0;
      if (bad) {
        bad_lo = bad_hi ? bad_lo : q0;
        bad_hi = min(q0 + QN, block_end);
      }
      if (q0 + QN < block_end) fetch(q0 + QN);
      if (q0 + QN <= j0 || q0 >= end_max) continue;

      const bool partial = q0 < j0 + 15 || q0 + QN > end_min;
      const int one = bl.kind(gap_of(lrange[0], pos_max), gap_of(lrange[1], pos_min));
      const float b = bl.bias_of(one);
      const bool plain = bl.is_plain(one) && !partial;
#pragma unroll 1
      for (int w = 0; w < QS; ++w) {  // 32 queries at a time
        const bf16 *wq = lq + w * 32 * LD, *wo = lo + w * 32 * LD;
        f32x4 s[2], dp[2];  // do . v - delta
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          Acc<NP> qk, ov;
          qk.start(f32x4{0.f, 0.f, 0.f, 0.f});
          ov.start(*(const f32x4 *)(ldelta + w * 32 + t * 16 + g * 4));  // -delta
#pragma unroll
          for (int d = 0; d < DF; ++d) {
            const Frag<NP> qf = frag_row<NP>(wq + t * 16 * LD + d * 32, LD, PART, lane);
            const Frag<NP> of = frag_row<NP>(wo + t * 16 * LD + d * 32, LD, PART, lane);
            qk.add(qf, kf[d]);
            ov.add(of, vf[d]);
          }
          s[t] = qk.value();
          dp[t] = ov.value();
        }
        // s, dp -> p, ds
        if (plain) {
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            const int r = w * 32 + t * 16 + g * 4;
            const f32x4 top = *(const f32x4 *)(ltop + r), inv = *(const f32x4 *)(linv + r);
            const f32x4 shift = LOG ? b - top + inv : b - top;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float x = exp2_fast(fmaf(s[t][e], scale, shift[e])), p = LOG ? x : x * inv[e];
              s[t][e] = p;
              dp[t][e] = p * dp[t][e];
            }
          }
        } else {
          f32x4 add[2];
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            const i32x4 qpos = *(const i32x4 *)(lpos + w * 32 + t * 16 + g * 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) add[t][e] = lb.bias_of(G, gap_of(qpos[e], pos));
          }
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            const int r = w * 32 + t * 16 + g * 4;
            const f32x4 top = *(const f32x4 *)(ltop + r), inv = *(const f32x4 *)(linv + r);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float x = fmaf(s[t][e], scale, add[t][e]) - top[e];
              const float p = LOG ? exp2_fast(x + inv[e]) : exp2_fast(x) * inv[e];
              const bool kept = (unsigned)(q0 + r + e - at) < after;
              s[t][e] = kept ? p : 0.f;
              dp[t][e] = kept ? p * dp[t][e] : 0.f;
            }
          }
        }
        const Frag<RP> pf = as_frag<RP>(s[0], s[1]), df = as_frag<RP>(dp[0], dp[1]);
#pragma unroll
        for (int c = 0; c < DT; ++c) {
          Frag<NP> of = frag_col<NP, 4>(wo + c * 16, LD, PART, lane);
          Frag<NP> qf = frag_col<NP, 4>(wq + c * 16, LD, PART, lane);
          if (bad) {
            of = cleaned(of);
            qf = cleaned(qf);
          }
          dv[c] = mma(of, pf, dv[c]);
          dk[c] = mma(qf, df, dk[c]);
        }
      }
    }
    if (bad_hi) {
      const auto ok = [&](int i) { return (unsigned)(i - at) < after; };
      mark_read<T, DT>((const T *)o, A.d_out.token_stride, G.width, bad_lo, bad_hi, lane, ok, dv);
      mark_read<T, DT>((const T *)q, A.q.token_stride, G.width, bad_lo, bad_hi, lane, ok, dk);
    }
  }

  if (after == 0) return;
  const int64_t row = ((int64_t)at * owners + owner) * G.width;
#pragma unroll
  for (int c = 0; c < DT; ++c) {
    const int d = c * 16 + g * 4;
    if (d >= G.width) continue;
    if (A.dk_parts) {
      store4(A.dk_parts + row + d, dk[c] * G.scale, G.width - d);
      store4(A.dv_parts + row + d, dv[c], G.width - d);
    } else {
      store4((T *)A.dk + row + d, dk[c] * G.scale, G.width - d);
      store4((T *)A.dv + row + d, dv[c], G.width - d);
    }
  }
}

// dk and dv of key heads from their query heads' parts, in their order, for the tokens that rows hold (and zeros for
// the others, where they are asked for). Bound by
// HBM: 76 us for 25 003 tokens of 8 heads of 128 to 2, 5.4 TB/s.
template <typename T> __global__ __launch_bounds__(256) void k_gap_sum_heads(BackArgs A) {
  const GapShape &G = A.G;
  const int pieces = (G.width + 3) / 4, k_heads = G.heads / G.group;
  const int64_t values = (int64_t)k_heads * pieces;
  for (int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x; x < G.n_tokens * values; x += (int64_t)gridDim.x * 256) {
    const int64_t t = x / values;
    const int k_head = (int)(x % values) / pieces, c = (int)(x % values) % pieces * 4;
    const bool held = span_of(G, A.spans, t).end != 0;
    if (!held && !G.clear_unheld) continue;
    const int64_t from = (t * G.heads + k_head * G.group) * G.width + c;
    f32x4 k = {0.f, 0.f, 0.f, 0.f}, v = k;
    for (int h = 0; h < (held ? G.group : 0); ++h)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (c + e < G.width) {
          k[e] += A.dk_parts[from + h * G.width + e];
          v[e] += A.dv_parts[from + h * G.width + e];
        }
    const int64_t to = (t * k_heads + k_head) * G.width + c;
    store4((T *)A.dk + to, k, G.width - c);
    store4((T *)A.dv + to, v, G.width - c);
  }
}

// Whether each query head's dk and dv are formed by themselves: a block that goes through a key head's query
// heads takes as many times longer, which the longest rows' blocks show where there are few others. Training on
// 25 003 ratings, 8 heads of 128 to 2: 2020 us in the kernel over queries, the longest row's time.
bool splits_heads(int64_t n_tokens, int32_t heads, int32_t k_heads) {
  return heads > k_heads && (n_tokens + 63) / 64 * k_heads < 2048;
}

template <typename T, int D> hipError_t launch_back(BackArgs A, bool vec, float *dbias, hipStream_t s) {
  A.n_tiles = (A.G.n_tokens + 63) / 64;
  const auto each = [&](auto kernel, int heads, size_t lds) {
    const int64_t per = max_blocks(256) / heads;
    for (A.tile0 = 0; A.tile0 < A.n_tiles; A.tile0 += per) {
      const int64_t n = A.n_tiles - A.tile0 < per ? A.n_tiles - A.tile0 : per;
      hipLaunchKernelGGL(kernel, dim3((unsigned)(n * heads)), dim3(256), lds, s, A);
    }
  };
  // tables of biases, where they leave a CU two blocks
  using Entry = typename std::conditional<D == 128 && sizeof(T) == 4, uint8_t, float>::type;
  const bool searched = A.G.last_bound >= kTableGaps;
  // 64 columns of dbias's sums where there are few blocks and they leave a CU two, beside the tiles of k and v and
  // the table; else 32, with which a CU takes three. Us in this kernel with 64 and 32: training on 2001 ratings,
  // 8 heads of 64, 32 buckets, 44 and 47; on 1 075 431, 7600 and 7100; at 128 wide with 64 buckets 3090 and 1820,
  // in fp32 with 32 buckets 1020 and 700.
  constexpr int tiles = 2 * kParts<T> * tile_tokens<T>() * (D + 16) * (int)sizeof(bf16) + 8704;
  const bool all =
      !searched && A.G.n_tokens * A.G.heads < 512 * 128 && tiles + 1024 * A.G.buckets <= 80 * 1024;
  const auto dq = searched ? k_gap_dq<T, D, false, void, 32>
                  : vec    ? all ? k_gap_dq<T, D, true, uint8_t, 64> : k_gap_dq<T, D, true, uint8_t, 32>
                  : all    ? k_gap_dq<T, D, false, uint8_t, 64>
                           : k_gap_dq<T, D, false, uint8_t, 32>;
  each(dq, A.G.heads, (size_t)(4 * A.G.buckets * (all ? 64 : 32)) * sizeof(float));
  hipLaunchKernelGGL(k_gap_dbias, dim3((unsigned)(A.G.heads * A.G.buckets)), dim3(256), 0, s, A.dbias_parts,
                     A.n_tiles, dbias);
  each(searched ? k_gap_dkv<T, D, false, void>
       : vec    ? k_gap_dkv<T, D, true, Entry>
                : k_gap_dkv<T, D, false, Entry>,
       A.dk_parts ? A.G.heads : A.G.heads / A.G.group, 0);
  if (A.dk_parts) {
    const int64_t values = A.G.n_tokens * (A.G.heads / A.G.group) * ((A.G.width + 3) / 4);
    const int64_t blocks = (values + 255) / 256;
    if (blocks > 0)
      hipLaunchKernelGGL((k_gap_sum_heads<T>), dim3((unsigned)(blocks < 65536 ? blocks : 65536)), dim3(256), 0, s,
                         A);
  }
  return hipGetLastError();
}
template <typename T> hipError_t launch_back(const BackArgs &A, bool vec, float *dbias, hipStream_t s) {
  return A.G.width <= 32   ? launch_back<T, 32>(A, vec, dbias, s)
         : A.G.width <= 64 ? launch_back<T, 64>(A, vec, dbias, s)
                           : launch_back<T, 128>(A, vec, dbias, s);
}

int64_t rounded(int64_t x) { return (x + 15) / 16 * 16; }

}  // namespace

GapBackSpace gap_back_space(int64_t n_tokens, int64_t n_rows, int32_t heads, int32_t k_heads, int32_t width,
                            int32_t buckets) {
  // tiles of 64 tokens
  return {gap_spans_bytes(n_tokens, n_rows), rounded(4 * n_tokens * heads),
          rounded(4 * ((n_tokens + 63) / 64) * heads * buckets),
          splits_heads(n_tokens, heads, k_heads) ? rounded(4 * n_tokens * heads * width) : 0};
}

hipError_t launch_gap_back(als_dtype dtype, const GapShape &G, const als_heads &d_out, const als_heads &q,
                           const als_heads &k, const als_heads &v, const void *out, const float *stats,
                           const int16_t *rest, void *dq, void *dk, void *dv, float *dbias, void *workspace,
                           hipStream_t s) {
  const GapBackSpace x = gap_back_space(G.n_tokens, G.n_rows, G.heads, G.heads / G.group, G.width, G.buckets);
  char *w = (char *)workspace;
  BackArgs A{};
  A.G = G;
  A.q = q;
  A.k = k;
  A.v = v;
  A.d_out = d_out;
  A.spans = x.spans ? (const Span2 *)w : nullptr;
  A.out = out;
  A.rest = rest;
  A.stats = stats;
  A.delta = (float *)(w + x.spans);
  A.dbias_parts = (float *)(w + x.spans + x.delta);
  if (x.heads) {
    A.dk_parts = (float *)(w + x.spans + x.delta + x.dbias);
    A.dv_parts = (float *)(w + x.spans + x.delta + x.dbias + x.heads);
  }
  A.dq = dq;
  A.dk = dk;
  A.dv = dv;
  const int size = dtype == ALS_F32 ? 4 : 2;
  const auto vec = [&](const als_heads &h) {
    return aligned16(h.data, h.token_stride, h.head_stride, G.width, size);
  };
  A.vec_rows = vec(q) && vec(k) && vec(v) && vec(d_out);
  A.vec_out = ((uintptr_t)out | (uintptr_t)rest | (uint64_t)(G.width * size)) % 16 == 0;
  hipError_t e = launch_gap_spans(G, x.spans ? w : nullptr, s);
  if (e != hipSuccess) return e;
  return dtype == ALS_F32 ? launch_back<float>(A, A.vec_rows, dbias, s)
                          : launch_back<bf16>(A, A.vec_rows, dbias, s);
}

}  // namespace als
