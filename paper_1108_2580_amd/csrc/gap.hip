// Softmax attention over packed rows of tokens (a user's ratings in the order of time), with a bias that
// each head learns for each bucket of the gap of time between two tokens: for the tokens j <= i of a row,
//   s_ij = scale q_i . k_j + bias[bucket(t_i - t_j)],  p_ij = exp(s_ij) / sum_j exp(s_ij),
//   o_i = sum_j p_ij v_j.
//
// One pass over the keys: a block holds 64 queries of a head, reads keys and values in tiles through
// LDS, and keeps the largest score and the sum of the exponentials so far. Both products are on MFMA with
// the queries as columns, so that the weights are operands of the second as they lie in registers. A block's
// queries are neighbours in the packed order, of one row or of several: a token's row says which keys it
// reads, so that short rows share tiles.
//
// Rounding. Scores, weights, sums and outputs are fp32; weights of bf16 values enter their product in two bf16
// parts, off by 2^-16 at most (one would cost an output as much again as its own rounding), or in three where
// the gradients are to follow: they take the outputs in 32 bits, and dbias, which sums terms that nearly cancel,
// was off by 2.3e-6 of its norm with two and is by 1e-7.
#include "gap.h"
#include "internal.h"

namespace als {

namespace {

// The table of the tokens' rows: a search each, 14 us for 1 075 431 tokens of 4096 rows.
__global__ __launch_bounds__(256) void k_gap_spans(GapShape G, Span2 *__restrict__ spans) {
  const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (t >= G.n_tokens) return;
  int64_t lo = 0, hi = G.n_rows + 1;  // rows that begin at t or before
  while (lo < hi) {
    const int64_t mid = (lo + hi) / 2;
    if (G.row_ptr[mid] <= t) lo = mid + 1; else hi = mid;
  }
  spans[t] = span_from(G.row_ptr, G.n_rows, G.n_tokens, lo - 1, t);
}

struct ReadArgs {
  GapShape G;
  als_heads q, k, v;
  const Span2 *spans;  // nullable: counted
  void *out;
  int16_t *rest;       // nullable
  float *stats;        // nullable
  int64_t tile0, n_tiles;
  bool vec_q;
};

template <typename T> constexpr int tile_keys() { return sizeof(T) == 2 ? 64 : 32; }

// One block: 64 queries of a head, 16 a wave. RP: parts of a weight. Twice the queries would halve what a score reads
// from LDS, at twice the registers: two blocks of 128 a CU took 730 us for 134 219 bf16 tokens of 512 rows, 8 heads
// of 64, where four of 64 take 570 (one row of 62 496: 7.8 and 7.9 ms).
//
// What bounds it: vector instructions, of which a score takes 7 where a tile has one bucket (three for the two
// parts of its weight) and about 7 more where it has several, and about 70 a tile and wave. Measured, 8 heads of
// 64 in bf16: one row of 62 496 tokens 7.9 ms, 500 TFLOP/s of a large product's 1235 (issue 83 %, MFMA 35 %, four
// blocks a CU, with which the waves' MFMAs and exponentials overlap: three took 8.5); 134 219 tokens of 512 rows
// 570 us (q, k, v and o at 1 TB/s of a copy's 5.1). fp32 at 128 wide, 25 003 tokens of 100 rows, 8 heads to 2:
// 500 us (MFMA 31 %, issue 50 %, two blocks, which LDS and registers allow). A block goes through its keys one tile
// after the other, so a batch takes at least the time of its longest row's last block: of 2000 fp32 rows of 25 on
// average at 50 wide, 111 us, the row of 1060 alone takes 95 (34 tiles; a block has 4.2 on average); of 8 bf16 rows,
// 36 us, the row of 827 takes 33; of the 100 above, the row of 3013 takes 315. A byte a gap in LDS (two reads a
// score) leaves four blocks a CU where the bias itself, 30 KB, leaves two.
template <typename T, int D, bool VEC, typename Entry, int RP>
__global__ __launch_bounds__(256, D == 128 ? 2 : D == 64 && sizeof(T) == 4 ? 3 : 4) void k_gap_read(ReadArgs A) {
  constexpr int KN = tile_keys<T>(), LD = D + 16, PART = KN * LD;
  constexpr int NP = kParts<T>, KT = KN / 16, KS = KN / 32, DF = D / 32, DT = D / 16;
  using Tiles = Staged<T, KN, D, VEC>;
  __shared__ __align__(16) bf16 lk[NP * PART];
  __shared__ __align__(16) bf16 lv[NP * PART];
  __shared__ __align__(16) int32_t lpos[KN];
  __shared__ int32_t lrange[2], lbad;
  __shared__ Buckets<Entry> lb;

  const GapShape &G = A.G;
  int tid = (int)threadIdx.x, lane = tid & 63, g = lane >> 4, m = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int head = (int)(blockIdx.x % (unsigned)G.heads);
  // a row's last tokens have the most keys: they go first
  const int64_t tile = A.n_tiles - 1 - (A.tile0 + blockIdx.x / (unsigned)G.heads);
  const int64_t t0 = tile * 64;

  lb.start(G, head, tid);
  if (tid == 0) lbad = -1;
  // the block's keys: from its first row's first token to its last token that has a row
  const int span_first = span_of(G, A.spans, t0 + lane).first;
  const int block_first = __builtin_amdgcn_readfirstlane(wave_min(span_first));
  const int block_last = __builtin_amdgcn_readfirstlane(wave_max(span_first != kNoRow ? (int)t0 + lane : -1));
  const int rows_first = __builtin_amdgcn_readfirstlane(wave_max(span_first));  // the last row's
  const int i0 = (int)t0 + wave * 16, at = i0 + m, first = __shfl(span_first, wave * 16 + m);
  if (first == kNoRow) clear_row<T>(G, A.out, at, G.heads, head, g);
  if (block_last < 0) return;

  // this wave's queries, one a lane
  const bool real = first != kNoRow;
  const unsigned before = real ? (unsigned)(at - first) : 0u;
  const int64_t t = real ? at : block_last;
  const int pos = G.positions[t];
  Frag<NP> qf[DF];
  load_row<T, D>((const T *)A.q.data + t * A.q.token_stride + head * A.q.head_stride, G.width, A.vec_q,
                 lane, qf);
  if (G.scale < 0.f) {
#pragma unroll
    for (int d = 0; d < DF; ++d) qf[d] = negated(qf[d]);
  }
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

  f32x4 o[DT];
  int bad_lo = 0, bad_hi = 0;  // keys among which some values were left out
  float top = -__builtin_inff(), base = 0.f, sum = 0.f;
#pragma unroll
  for (int c = 0; c < DT; ++c) o[c] = f32x4{0.f, 0.f, 0.f, 0.f};

  for (int k0 = block_first; k0 <= block_last; k0 += KN) {
    // addresses are formed anew in each tile: held across tiles they would cost a block its place on the CU
    asm volatile("" : "+v"(tid));
    tid &= 255;
    lane = tid & 63;
    g = lane >> 4;
    __syncthreads();
    hk.put_parts(lk, LD, rows_of(k, k_row, k0), tid);
    const bool masked = k0 + KN - 1 > (int)t0 || k0 < rows_first;  // for some query of the block
    if (masked && hv.nonfinite(rows_of(v, v_row, k0), tid)) lbad = k0;
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
    __builtin_amdgcn_sched_barrier(0);

    const bool partial = k0 + KN - 1 > i0 || k0 < first_max;
    f32x4 s[KT];
#pragma unroll
    for (int t = 0; t < KT; ++t) {
      Acc<NP> qk;
      qk.start(f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
      for (int d = 0; d < DF; ++d) {
        const Frag<NP> kf = frag_row<NP>(lk + t * 16 * LD + d * 32, LD, PART, lane);
        qk.add(kf, qf[d]);
      }
      s[t] = qk.value();
    }

    // one bucket for the tile's gaps, or one for each
    const int kind = bl.kind(gap_of(pos_min, lrange[1]), gap_of(pos_max, lrange[0]));
    const float b = bl.bias_of(kind);
    const bool plain = bl.is_plain(kind) && !partial;

    // The largest score so far is followed only where it has grown by 8: exponentials up to 2^8 keep
    // their precision, and most tiles leave the sums as they are.
    const auto follow = [&](float most) {
      most = column_max(most);
      if (__any(most > top + 8.f)) {
        const bool none = top == -__builtin_inff();  // so far: there is nothing to scale
        top = fmaxf(top, most);
        const float next = top == -__builtin_inff() ? 0.f : top;
        const float factor = none ? 0.f : exp2_fast(base - next);
        base = next;
        sum *= factor;
#pragma unroll
        for (int c = 0; c < DT; ++c) o[c] *= factor;
      }
    };
    // s -> 2^(by s + shift), of 32 keys, as operands
    const auto weigh = [&](int w, float by, float shift) {
#pragma unroll
      for (int t = 2 * w; t < 2 * w + 2; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float x = exp2_fast(fmaf(s[t][e], by, shift));
          s[t][e] = x;
          sum += x;
        }
      asm("" : "+v"(sum));  // now: put off, the sums would hold the weights' registers
      return as_frag<RP>(s[2 * w], s[2 * w + 1]);
    };
    const auto add_values = [&](int w, bool bad, const Frag<RP> &pf) {
#pragma unroll
      for (int c = 0; c < DT; ++c) {
        Frag<NP> vf = frag_col<NP, 4>(lv + w * 32 * LD + c * 16, LD, PART, lane);
        if (bad) vf = cleaned(vf);
        o[c] = mma(vf, pf, o[c]);
      }
    };
    if (plain) {
      float most = s[0][0];
#pragma unroll
      for (int t = 0; t < KT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) most = fmaxf(most, s[t][e]);
      most = fmaf(most, scale, b);
      follow(most);
      const float shift = b - base;
#pragma unroll
      for (int w = 0; w < KS; ++w) {
        add_values(w, false, weigh(w, scale, shift));
        __builtin_amdgcn_sched_barrier(0);
      }
    } else {
      float most = -__builtin_inff();
#pragma unroll
      for (int t = 0; t < KT; ++t) {
        const i32x4 kpos = *(const i32x4 *)(lpos + t * 16 + g * 4);
        f32x4 add;
#pragma unroll
        for (int e = 0; e < 4; ++e) add[e] = lb.bias_of(G, gap_of(pos, kpos[e]));
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const bool kept = (unsigned)(k0 + t * 16 + g * 4 + e - first) <= before;
          const float x = kept ? fmaf(s[t][e], scale, add[e]) : -__builtin_inff();
          s[t][e] = x;
          most = fmaxf(most, x);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      follow(most);
#pragma unroll
      for (int w = 0; w < KS; ++w) {
        add_values(w, bad, weigh(w, 1.f, -base));
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }

  const float total = column_sum(sum);
  if (first == kNoRow) return;
  if (bad_hi)
    mark_read<T, DT>((const T *)v, A.v.token_stride, G.width, bad_lo, bad_hi, lane,
                     [&](int j) { return (unsigned)(j - first) <= before; }, o);
  const float inv = total == 0.f ? 0.f : 1.f / total;
  const int64_t row = ((int64_t)at * G.heads + head) * G.width;
#pragma unroll
  for (int c = 0; c < DT; ++c) {
    const int d = c * 16 + g * 4;
    if (d >= G.width) continue;
    const f32x4 x = o[c] * inv;
    store4((T *)A.out + row + d, x, G.width - d);
    if constexpr (sizeof(T) == 2) {
      if (A.rest) store_rest(A.rest + row + d, x, G.width - d);
    }
  }
  if (A.stats && g == 0) {
    float *to = A.stats + (int64_t)head * G.n_tokens + at;
    to[0] = base;
    to[(int64_t)G.heads * G.n_tokens] = inv;
  }
}

template <typename T, int D> hipError_t launch_read(ReadArgs A, bool vec, hipStream_t s) {
  using Entry = uint8_t;
  A.n_tiles = (A.G.n_tokens + 63) / 64;
  const int64_t per = max_blocks(256) / A.G.heads;
  for (A.tile0 = 0; A.tile0 < A.n_tiles; A.tile0 += per) {
    const int64_t n = A.n_tiles - A.tile0 < per ? A.n_tiles - A.tile0 : per;
    const dim3 grid((unsigned)(n * A.G.heads));
    // for gradients, with three parts of a weight
    constexpr int RP = kReadParts<T>;
    const auto kernel = A.G.last_bound >= kTableGaps ? A.stats ? k_gap_read<T, D, false, void, 3>
                                                               : k_gap_read<T, D, false, void, RP>
                        : vec                        ? A.stats ? k_gap_read<T, D, true, Entry, 3>
                                                               : k_gap_read<T, D, true, Entry, RP>
                        : A.stats                    ? k_gap_read<T, D, false, Entry, 3>
                                                     : k_gap_read<T, D, false, Entry, RP>;
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, A);
  }
  return hipGetLastError();
}
template <typename T> hipError_t launch_read(const ReadArgs &A, bool vec, hipStream_t s) {
  return A.G.width <= 32   ? launch_read<T, 32>(A, vec, s)
         : A.G.width <= 64 ? launch_read<T, 64>(A, vec, s)
                           : launch_read<T, 128>(A, vec, s);
}

}  // namespace

int64_t gap_spans_bytes(int64_t n_tokens, int64_t n_rows) {
  return n_rows > kCountedRows ? (n_tokens * (int64_t)sizeof(Span2) + 15) / 16 * 16 : 0;
}

hipError_t launch_gap_spans(const GapShape &G, void *spans, hipStream_t s) {
  if (!spans || G.n_tokens == 0) return hipSuccess;
  hipLaunchKernelGGL(k_gap_spans, dim3((unsigned)((G.n_tokens + 255) / 256)), dim3(256), 0, s, G,
                     (Span2 *)spans);
  return hipGetLastError();
}

hipError_t launch_gap_read(als_dtype dtype, const GapShape &G, const als_heads &q, const als_heads &k,
                           const als_heads &v, const void *spans, void *out, float *stats, int16_t *rest,
                           hipStream_t s) {
  if (G.n_tokens == 0) return hipSuccess;
  const int size = dtype == ALS_F32 ? 4 : 2;
  const auto vec = [&](const als_heads &x) {
    return aligned16(x.data, x.token_stride, x.head_stride, G.width, size);
  };
  ReadArgs A{G, q, k, v, (const Span2 *)spans, out, rest, stats, 0, 0, vec(q)};
  const bool all = vec(k) && vec(v);
  return dtype == ALS_F32 ? launch_read<float>(A, all, s) : launch_read<bf16>(A, all, s);
}

}  // namespace als
