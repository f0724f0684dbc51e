// One token of each beam of each list, over the list's row of the history (gap.hip's scores) and the
// tokens that the beam has chosen itself: those lie by step and beam, and a table says which beam holds
// each step of a beam's path, so that nothing is copied where beams fork.
//
// The history is read once for all beams of a list and all query heads that share a key head: they are the
// columns of the products. Rows are cut into segments that run side by side; a second kernel joins a beam's
// segments with its path. Bound by HBM: every key and value is read once.
#include "gap.h"
#include "internal.h"

namespace als {

namespace {

struct StepArgs {
  GapShape G;
  GapPath P;
  als_heads q, k, v;
  void *out;
  float *parts;   // [slots, heads, beams, width]
  float *stats;   // [slots, heads, beams, 2]: the largest score (-inf: none) and the sum
  const Place *places;  // of the slots; nullable: searched for
  int64_t slot0, row0;
  int shift, passes;
  bool vec, vec_path;
};

// Partials of slot, head, beam.
__device__ __forceinline__ int64_t part_index(const StepArgs &A, int64_t slot, int head, int beam) {
  return (slot * A.G.heads + head) * A.P.beams + beam;
}

// The places of the segments, a search each: 5 us for 2074.
__global__ __launch_bounds__(256) void k_gap_places(GapShape G, int shift, int64_t n_slots, Place *places) {
  const int64_t slot = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (slot >= n_slots) return;
  int64_t lo = 0, hi = G.n_rows;  // the last row whose slots begin at this one or before
  while (hi - lo > 1) {
    const int64_t mid = (lo + hi) / 2;
    if ((clamped(G.row_ptr[mid], 0, G.n_tokens) >> shift) + mid <= slot) lo = mid; else hi = mid;
  }
  Place p;
  p.row = (int32_t)lo;
  p.first = clamped(G.row_ptr[lo], 0, G.n_tokens);
  p.len = (int32_t)(clamped(G.row_ptr[lo + 1], p.first, G.n_tokens) - p.first);
  p.segment = slot - ((p.first >> shift) + lo);
  places[slot] = p;
}

// One block: a segment, a key head and up to 16 CT of its columns (beams and the head's query heads). A wave
// takes every fourth 32 keys; the next are on their way while it works.
//
// What bounds it: a block's chain of reads (its place, the first keys, the next), at the four blocks a CU that
// 124 registers allow. Measured in bf16, 8 key heads of 64: one list of 62 496 tokens, 8 beams, 33 us (3.9 TB/s);
// 1024 lists of 262 tokens, 16 beams, 195 us (2.8 TB/s; waves wait 77 % of their time). Two tiles ahead took 40 and
// 236: their registers leave three blocks.
template <typename T, int D, int CT>
__global__ __launch_bounds__(256, D == 128 && sizeof(T) == 4 ? 1 : 2) void k_gap_history(StepArgs A) {
  constexpr int LD = D + 16, PART = 32 * LD, NP = kParts<T>, RP = kReadParts<T>, DF = D / 32, DT = D / 16;
  constexpr int COLS = 16 * CT, V8 = D / 8, ROWS = 64 / V8, VN = 32 / ROWS, LB = 65;
  // values of the waves' tiles, and at the end their sums: of all four side by side where they fit
  constexpr int TILES = 4 * NP * PART * (int)sizeof(bf16), SUMS = COLS * D * (int)sizeof(float);
  constexpr int SIDE = 4 * SUMS <= 32768 || 4 * SUMS <= TILES ? 4 : 1;
  __shared__ __align__(16) char lmem[TILES > SIDE * SUMS ? TILES : SIDE * SUMS];
  bf16(*lv)[NP * PART] = (bf16(*)[NP * PART])lmem;
  float *lout = (float *)lmem;
  __shared__ __align__(16) int32_t lkind[4][32];
  __shared__ int32_t lbounds[64];
  __shared__ float lbias[COLS * LB];
  __shared__ float ltop[4][COLS], lsum[4][COLS];

  const GapShape &G = A.G;
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6, g = lane >> 4, m = lane & 15;
  const int k_heads = G.heads / G.group, columns = A.P.beams * G.group;
  unsigned block = blockIdx.x;
  const int col0 = (int)(block % (unsigned)A.passes) * COLS;
  block /= (unsigned)A.passes;
  const int k_head = (int)(block % (unsigned)k_heads);
  const int64_t slot = A.slot0 + block / (unsigned)k_heads;
  const Place at = A.places ? A.places[slot]
                            : find_place<false>(G.row_ptr, G.n_rows, G.n_tokens, A.shift, slot, lane);
  const int64_t begin = at.segment << A.shift;
  if (at.segment < 0 || begin >= at.len) return;
  const int count = (int)(at.len - begin < 1LL << A.shift ? at.len - begin : 1LL << A.shift);
  const int64_t token0 = at.first + begin;
  const T *k = (const T *)A.k.data + token0 * A.k.token_stride + k_head * A.k.head_stride;
  const T *v = (const T *)A.v.data + token0 * A.v.token_stride + k_head * A.v.head_stride;

  // 32 keys: rows m and 16 + m as operands; rows of v eight values a lane
  Raw8<T> hk[2][DF], hv[VN];
  int hpos = 0;
  const auto fetch = [&](int j0) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int j = min(j0 + 16 * t + m, count - 1);
#pragma unroll
      for (int d = 0; d < DF; ++d)
        hk[t][d] = load8(k + j * A.k.token_stride, d * 32 + g * 8, G.width, A.vec);
    }
#pragma unroll
    for (int i = 0; i < VN; ++i) {
      const int j = j0 + i * ROWS + lane / V8;
      hv[i] = load8(v + min(j, count - 1) * A.v.token_stride, lane % V8 * 8, j < count ? G.width : 0, A.vec);
    }
    hpos = G.positions[token0 + min(j0 + (lane & 31), count - 1)];
  };
  if (wave * 32 < count) fetch(wave * 32);

  if (tid < 64) lbounds[tid] = tid < G.buckets - 1 ? G.bounds[tid] : 0x7fffffff;
  {
    const int c = tid % COLS, col = min(col0 + c, columns - 1);
    const float *from = G.bias + (int64_t)(k_head * G.group + col % G.group) * G.buckets;
#pragma unroll 4
    for (int n = tid / COLS; n < G.buckets; n += 256 / COLS) lbias[c * LB + n] = bias2(from[n]);
  }
  Frag<NP> qf[CT][DF];
  int pos[CT];
  bool alike = true;
  const int64_t rows = (int64_t)at.row * A.P.beams;
  const int pos0 = A.P.q_positions[rows];
#pragma unroll
  for (int n = 0; n < CT; ++n) {
    const int col = min(col0 + n * 16 + m, columns - 1);
    const int64_t row = rows + col / G.group;
    pos[n] = A.P.q_positions[row];
    alike = alike && pos[n] == pos0;
    load_row<T, D>((const T *)A.q.data + row * A.q.token_stride +
                       (k_head * G.group + col % G.group) * A.q.head_stride,
                   G.width, A.vec, lane, qf[n]);
    if (G.scale < 0.f) {
#pragma unroll
      for (int d = 0; d < DF; ++d) qf[n][d] = negated(qf[n][d]);
    }
  }
  alike = __all(alike);
  const float scale = fabsf(G.scale) * kLog2e;

  f32x4 o[CT][DT];
  float top[CT], base[CT], sum[CT];
#pragma unroll
  for (int n = 0; n < CT; ++n) {
    top[n] = -__builtin_inff();
    base[n] = sum[n] = 0.f;
#pragma unroll
    for (int c = 0; c < DT; ++c) o[n][c] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  __syncthreads();

  for (int j0 = wave * 32; j0 < count; j0 += 128) {
    Frag<NP> kf[2][DF];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int d = 0; d < DF; ++d) kf[t][d] = operand(hk[t][d]);
    bf16 *mine = lv[wave];
#pragma unroll
    for (int i = 0; i < VN; ++i) {
      const Frag<NP> x = operand(hv[i]);
      bf16 *to = mine + (i * ROWS + lane / V8) * LD + lane % V8 * 8;
#pragma unroll
      for (int n = 0; n < NP; ++n) *(bf16x8 *)(to + n * PART) = x.p[n];
    }
    // where the beams' positions are alike, a lane finds the bucket of one key, for all columns
    if (lane < 32) lkind[wave][lane] = alike ? bucket_of(lbounds, G.buckets, gap_of(pos0, hpos)) : hpos;
    if (j0 + 128 < count) fetch(j0 + 128);
    __builtin_amdgcn_wave_barrier();

    f32x4 s[CT][2];
    float most[CT];
    i32x4 near[2];  // buckets of the lane's keys, or, where positions differ, the keys' positions
#pragma unroll
    for (int t = 0; t < 2; ++t) near[t] = *(const i32x4 *)(lkind[wave] + t * 16 + g * 4);
#pragma unroll
    for (int n = 0; n < CT; ++n) {
      i32x4 kind[2] = {near[0], near[1]};
      if (!alike) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) kind[t][e] = bucket_of(lbounds, G.buckets, gap_of(pos[n], near[t][e]));
      }
      f32x4 add[2];
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) add[t][e] = lbias[(n * 16 + m) * LB + kind[t][e]];
      most[n] = -__builtin_inff();
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        s[n][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int d = 0; d < DF; ++d) s[n][t] = mma(kf[t][d], qf[n][d], s[n][t]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int r = t * 16 + g * 4 + e;
          const float y = j0 + r < count ? fmaf(s[n][t][e], scale, add[t][e]) : -__builtin_inff();
          s[n][t][e] = y;
          most[n] = fmaxf(most[n], y);
        }
      }
    }
    bool grown = false;
#pragma unroll
    for (int n = 0; n < CT; ++n) {
      most[n] = column_max(most[n]);
      grown = grown || most[n] > top[n] + 8.f;
    }
    if (__any(grown)) {
#pragma unroll
      for (int n = 0; n < CT; ++n) {
        const bool none = top[n] == -__builtin_inff();
        top[n] = fmaxf(top[n], most[n]);
        const float next = top[n] == -__builtin_inff() ? 0.f : top[n];
        const float factor = none ? 0.f : exp2_fast(base[n] - next);
        base[n] = next;
        sum[n] *= factor;
#pragma unroll
        for (int c = 0; c < DT; ++c) o[n][c] *= factor;
      }
    }
    Frag<RP> pf[CT];
#pragma unroll
    for (int n = 0; n < CT; ++n) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s[n][t][e] = exp2_fast(s[n][t][e] - base[n]);
          sum[n] += s[n][t][e];
        }
      pf[n] = as_frag<RP>(s[n][0], s[n][1]);
    }
#pragma unroll
    for (int c = 0; c < DT; ++c) {
      const Frag<NP> vf = frag_col<NP, 4>(mine + c * 16, LD, PART, lane);
#pragma unroll
      for (int n = 0; n < CT; ++n) o[n][c] = mma(vf, pf[n], o[n][c]);
    }
    __builtin_amdgcn_wave_barrier();
  }

  // the waves' parts on one base, added in their order
#pragma unroll
  for (int n = 0; n < CT; ++n) {
    sum[n] = column_sum(sum[n]);
    if (g == 0) {
      ltop[wave][n * 16 + m] = top[n] == -__builtin_inff() && sum[n] == 0.f ? -__builtin_inff() : base[n];
      lsum[wave][n * 16 + m] = sum[n];
    }
  }
  __syncthreads();
  float total[CT], highest[CT];
#pragma unroll
  for (int n = 0; n < CT; ++n) {
    const int c = n * 16 + m;
    highest[n] = fmaxf(fmaxf(ltop[0][c], ltop[1][c]), fmaxf(ltop[2][c], ltop[3][c]));
    const float to = highest[n] == -__builtin_inff() ? 0.f : highest[n];
    total[n] = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) total[n] += lsum[w][c] * exp2_fast(ltop[w][c] - to);
    const float factor = exp2_fast(ltop[wave][c] - to);
#pragma unroll
    for (int d = 0; d < DT; ++d) o[n][d] *= factor;
  }
  if (wave == 0 && g == 0) {
#pragma unroll
    for (int n = 0; n < CT; ++n) {
      const int col = col0 + n * 16 + m;
      if (col < columns) {
        float *to = A.stats + 2 * part_index(A, slot, k_head * G.group + col % G.group, col / G.group);
        to[0] = highest[n];
        to[1] = total[n];
      }
    }
  }
  // the waves are past their tiles: the barrier above
#pragma unroll 1
  for (int w = 0; w < 4; ++w) {
    if (SIDE == 4 ? w == 0 : wave == w) {
#pragma unroll
      for (int n = 0; n < CT; ++n)
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          f32x4 *to = (f32x4 *)(lout + (SIDE == 4 ? wave * COLS * D : 0) + (n * 16 + m) * D + d * 16 + g * 4);
          *to = SIDE == 4 || w == 0 ? o[n][d] : *to + o[n][d];
        }
    }
    if (SIDE == 4) break;
    __syncthreads();
  }
  if (SIDE == 4) __syncthreads();
  for (int x = tid * 4; x < COLS * D; x += 1024) {
    const int col = col0 + x / D, d = x % D;
    f32x4 y = *(const f32x4 *)(lout + x);
#pragma unroll
    for (int w = 1; w < SIDE; ++w) y += *(const f32x4 *)(lout + w * COLS * D + x);
    if (col < columns && d < G.width)
      store4(A.parts + part_index(A, slot, k_head * G.group + col % G.group, col / G.group) * G.width + d, y,
             G.width - d);
  }
}

// What a lane has of a head's softmax so far: eight features.
struct Sums {
  float top, sum;
  f32x4 o[2];
  __device__ __forceinline__ void clear() {
    top = -__builtin_inff();
    sum = 0.f;
    o[0] = o[1] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  // takes a part whose weights are `by` at the largest score `score`
  __device__ __forceinline__ void take(float score, float by, f32x4 lo, f32x4 hi) {
    const float next = fmaxf(top, score), to = next == -__builtin_inff() ? 0.f : next;
    const float mine = top == next ? 1.f : exp2_fast(top - to), its = exp2_fast(score - to);
    top = next;
    sum = sum * mine + by * its;
    o[0] = o[0] * mine + lo * its;
    o[1] = o[1] * mine + hi * its;
  }
  __device__ __forceinline__ void take_lane(int n) {  // of the lane n apart
    const float score = __shfl_xor(top, n), by = __shfl_xor(sum, n);
    f32x4 x[2];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[0][e] = __shfl_xor(o[0][e], n);
      x[1][e] = __shfl_xor(o[1][e], n);
    }
    take(score, by, x[0], x[1]);
  }
  template <typename T> __device__ __forceinline__ void store(T *to, int n) const {
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    store4(to, o[0] * inv, n);
    if (n > 4) store4(to + 4, o[1] * inv, n - 4);
  }
};

// A token of a beam's path as a lane reads it.
template <typename T> struct PathToken {
  Raw8<T> k, v;
  int32_t position;
  bool ok;
  __device__ __forceinline__ void read(const StepArgs &A, int64_t list, int holder, int64_t step, int k_head,
                                       int c) {
    ok = holder >= 0 && holder < A.P.beams;
    const int64_t from = list * A.P.beams + (ok ? holder : 0);
    k = load8((const T *)A.P.k.data + step * A.P.k_step + from * A.P.k.token_stride + k_head * A.P.k.head_stride,
              c, A.G.width, A.vec_path);
    v = load8((const T *)A.P.v.data + step * A.P.v_step + from * A.P.v.token_stride + k_head * A.P.v.head_stride,
              c, A.G.width, A.vec_path);
    position = A.P.positions[step * (A.G.n_rows * A.P.beams) + from];
  }
  // q . k over the L lanes of a head, with its bias
  template <int L>
  __device__ __forceinline__ float score(const GapShape &G, const int32_t *bounds, const f32x4 *q, int32_t at,
                                         int head) const {
    const f32x4 a = low4(k), b = high4(k);
    float x = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) x = fmaf(q[0][e], a[e], fmaf(q[1][e], b[e], x));
#pragma unroll
    for (int n = 1; n < L; n <<= 1) x += __shfl_xor(x, n);
    const float bias = G.bias[(int64_t)head * G.buckets + bucket_of(bounds, G.buckets, gap_of(at, position))];
    return ok ? fmaf(x, G.scale * kLog2e, bias2(bias)) : __builtin_nanf("");
  }
};

// The path and the segments' parts of many beams: a wave takes 512 / D heads of one, eight features a lane, so
// that a step's keys and values are one read each of neighbouring heads; four steps are on their way at a
// time. 104 us for 16 384 beams of 9 steps, 8 heads of 64 (3.9 TB/s with the segments' parts).
template <typename T, int D> __global__ __launch_bounds__(256) void k_gap_path(StepArgs A) {
  constexpr int L = D / 8, HEADS = 64 / L, AHEAD = 4;
  __shared__ int32_t lbounds[64];
  const GapShape &G = A.G;
  const int tid = (int)threadIdx.x, lane = tid & 63, c = lane % L * 8;
  if (tid < 64) lbounds[tid] = tid < G.buckets - 1 ? G.bounds[tid] : 0x7fffffff;
  __syncthreads();
  const unsigned per_row = (unsigned)((G.heads + HEADS - 1) / HEADS);
  const unsigned index = blockIdx.x * 4 + (unsigned)__builtin_amdgcn_readfirstlane(tid / 64);
  const int64_t row = A.row0 + index / per_row;
  if (row >= G.n_rows * A.P.beams) return;
  const int head0 = (int)(index % per_row) * HEADS + lane / L, head = min(head0, G.heads - 1);
  const int64_t list = row / A.P.beams;
  const int beam = (int)(row - list * A.P.beams), k_head = head / G.group;
  const int32_t *path = A.P.path + row * A.P.path_stride;

  const Raw8<T> raw = load8((const T *)A.q.data + row * A.q.token_stride + head * A.q.head_stride, c, G.width,
                            A.vec);
  const int32_t at = A.P.q_positions[row];
  const f32x4 q[2] = {low4(raw), high4(raw)};
  Sums s;
  s.clear();
  for (int t0 = 0; t0 < A.P.steps; t0 += AHEAD) {
    PathToken<T> x[AHEAD];
    const int n = min(A.P.steps - t0, AHEAD);
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
      if (i < n) x[i].read(A, list, path[t0 + i], t0 + i, k_head, c);
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
      if (i < n) s.take(x[i].template score<L>(G, lbounds, q, at, head), 1.f, low4(x[i].v), high4(x[i].v));
  }
  const int64_t first = clamped(G.row_ptr[list], 0, G.n_tokens);
  const int64_t len = clamped(G.row_ptr[list + 1], first, G.n_tokens) - first;
  const int64_t slot = (first >> A.shift) + list, n_slots = segments_of(len, A.shift);
  for (int64_t n = 0; n < n_slots; ++n) {
    const int64_t part = part_index(A, slot + n, head, beam);
    const Raw8<float> x = load8(A.parts + part * G.width, c, G.width, G.width % 4 == 0);
    s.take(A.stats[2 * part], A.stats[2 * part + 1], low4(x), high4(x));
  }
  if (head0 < G.heads && c < G.width) s.store((T *)A.out + (row * G.heads + head) * G.width + c, G.width - c);
}

// Of fewer beams: WAVES waves take one head, L = D / 8 lanes a segment or a step.
template <typename T, int D, int WAVES> __global__ __launch_bounds__(256) void k_gap_path_wide(StepArgs A) {
  constexpr int L = D / 8, KEYS = 64 * WAVES / L;
  __shared__ int32_t lbounds[64];
  __shared__ float lparts[WAVES > 1 ? 3 : 1][L][10];
  const GapShape &G = A.G;
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid / 64, c = lane % L * 8;
  const int sub = (WAVES == 1 ? lane : tid) / L;
  if (tid < 64) lbounds[tid] = tid < G.buckets - 1 ? G.bounds[tid] : 0x7fffffff;
  if (WAVES == 1) __syncthreads();
  const unsigned index = WAVES == 1 ? blockIdx.x * 4 + (unsigned)wave : blockIdx.x;
  const int64_t row = A.row0 + index / (unsigned)G.heads;
  if (row >= G.n_rows * A.P.beams) return;
  const int head = (int)(index % (unsigned)G.heads);
  const int64_t list = row / A.P.beams;
  const int beam = (int)(row - list * A.P.beams);
  const Raw8<T> raw = load8((const T *)A.q.data + row * A.q.token_stride + head * A.q.head_stride, c, G.width,
                            A.vec);
  const int32_t at = A.P.q_positions[row];
  const int64_t first = clamped(G.row_ptr[list], 0, G.n_tokens);
  const int64_t len = clamped(G.row_ptr[list + 1], first, G.n_tokens) - first;
  const int64_t slot = (first >> A.shift) + list, n_slots = segments_of(len, A.shift);
  const f32x4 q[2] = {low4(raw), high4(raw)};
  Sums s;
  s.clear();
  if (WAVES > 1) __syncthreads();
  for (int t = sub; t < A.P.steps; t += KEYS) {
    PathToken<T> x;
    x.read(A, list, A.P.path[row * A.P.path_stride + t], t, head / G.group, c);
    s.take(x.template score<L>(G, lbounds, q, at, head), 1.f, low4(x.v), high4(x.v));
  }
  for (int64_t n0 = sub; n0 < n_slots; n0 += 2 * KEYS) {
    Raw8<float> x[2];
    float score[2], by[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int64_t n = n0 + i * KEYS, part = part_index(A, slot + (n < n_slots ? n : n0), head, beam);
      x[i] = load8(A.parts + part * G.width, c, G.width, G.width % 4 == 0);
      score[i] = A.stats[2 * part];
      by[i] = A.stats[2 * part + 1];
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (n0 + i * KEYS < n_slots) s.take(score[i], by[i], low4(x[i]), high4(x[i]));
  }
#pragma unroll
  for (int n = L; n < 64; n <<= 1) s.take_lane(n);
  if constexpr (WAVES > 1) {
    if (wave > 0 && lane < L) {
      float *to = lparts[wave - 1][lane];
      to[0] = s.top;
      to[1] = s.sum;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        to[2 + e] = s.o[0][e];
        to[6 + e] = s.o[1][e];
      }
    }
    __syncthreads();
    if (wave > 0) return;
    for (int w = 0; w < 3; ++w) {
      const float *x = lparts[w][lane % L];
      s.take(x[0], x[1], f32x4{x[2], x[3], x[4], x[5]}, f32x4{x[6], x[7], x[8], x[9]});
    }
  }
  if (lane < L && c < G.width)
    s.store((T *)A.out + (row * G.heads + head) * G.width + c, G.width - c);
}

// Short segments fill the chip where tokens are few, long ones leave fewer parts of every beam's and head's sums:
// 128 tokens up to 2048 blocks, then as few above 256 as leave 8192. History and join, us, at 2048, 4096, 8192
// and 16 384 blocks: one list of 62 496 tokens, 8 key heads of 64: 44, 56, 56, 56 (segments of 256, then 128);
// 1024 lists of 262: 336, 309, 306, 320 (of 2048, 1024, 512, 256).
int step_shift(int64_t n_tokens, int32_t k_heads) {
  int shift = (n_tokens >> 7) * k_heads > 2048 ? 8 : 7;
  while (shift < 12 && (n_tokens >> shift) * k_heads > 8192) ++shift;
  return shift;
}

template <typename T, int D, int CT> void launch_history(StepArgs A, hipStream_t s) {
  const int k_heads = A.G.heads / A.G.group, columns = A.P.beams * A.G.group;
  A.passes = (columns + 16 * CT - 1) / (16 * CT);
  const int64_t slots = (A.G.n_tokens >> A.shift) + A.G.n_rows;
  const int64_t per = max_blocks(256) / ((int64_t)k_heads * A.passes);
  for (A.slot0 = 0; A.slot0 < slots; A.slot0 += per) {
    const int64_t n = slots - A.slot0 < per ? slots - A.slot0 : per;
    hipLaunchKernelGGL((k_gap_history<T, D, CT>), dim3((unsigned)(n * k_heads * A.passes)), dim3(256), 0, s, A);
  }
}
template <typename T, int D> hipError_t launch_step(StepArgs A, hipStream_t s) {
  const int columns = A.P.beams * A.G.group;
  if (A.G.n_tokens > 0) {
    // as many columns as fit the registers beside a tile of keys and one of values
    constexpr int MOST = D == 128 ? (sizeof(T) == 4 ? 1 : 2) : (sizeof(T) == 4 ? 2 : 4);
    if (columns <= 16 || MOST == 1)
      launch_history<T, D, 1>(A, s);
    else if (columns <= 32 || MOST == 2)
      launch_history<T, D, MOST < 2 ? 1 : 2>(A, s);
    else
      launch_history<T, D, MOST>(A, s);
  }
  // Waves a beam: four a head where those are few, one, or one for 512 / D heads. 4, 1 and 1/8 a head, us:
  // 64 heads of beams with 245 segments 9.6, 19.6, -; 4000 with 3 steps at 50 wide 20, 10, 23; 131 072 with 9
  // steps at 64 wide -, 178, 100.
  constexpr int HEADS = 512 / D;
  const int64_t rows = A.G.n_rows * A.P.beams, heads = rows * A.G.heads;
  const int64_t waves = heads <= 1024    ? 4 * A.G.heads
                        : heads <= 16384 ? A.G.heads
                                         : (A.G.heads + HEADS - 1) / HEADS;
  const auto kernel = heads <= 1024    ? k_gap_path_wide<T, D, 4>
                      : heads <= 16384 ? k_gap_path_wide<T, D, 1>
                                       : k_gap_path<T, D>;
  const int64_t per = max_blocks(256) / A.G.heads;
  for (A.row0 = 0; A.row0 < rows; A.row0 += per) {
    const int64_t n = rows - A.row0 < per ? rows - A.row0 : per;
    hipLaunchKernelGGL(kernel, dim3((unsigned)((n * waves + 3) / 4)), dim3(256), 0, s, A);
  }
  return hipGetLastError();
}
template <typename T> hipError_t launch_step(const StepArgs &A, hipStream_t s) {
  return A.G.width <= 32   ? launch_step<T, 32>(A, s)
         : A.G.width <= 64 ? launch_step<T, 64>(A, s)
                           : launch_step<T, 128>(A, s);
}

int64_t part_bytes(int64_t n_tokens, int64_t n_lists, int32_t heads, int32_t k_heads, int32_t beams,
                   int64_t values) {
  const int64_t slots = (n_tokens >> step_shift(n_tokens, k_heads)) + n_lists;
  return n_tokens > 0 ? (slots * heads * beams * values * 4 + 15) / 16 * 16 : 0;
}

// Of the slots' places, for more rows than a search looks at together.
int64_t place_bytes(int64_t n_tokens, int64_t n_lists, int32_t k_heads) {
  const int64_t slots = (n_tokens >> step_shift(n_tokens, k_heads)) + n_lists;
  return n_tokens > 0 && n_lists > 64 ? (slots * (int64_t)sizeof(Place) + 15) / 16 * 16 : 0;
}

}  // namespace

int64_t gap_step_space(int64_t n_tokens, int64_t n_lists, int32_t heads, int32_t k_heads, int32_t beams,
                       int32_t width) {
  return part_bytes(n_tokens, n_lists, heads, k_heads, beams, width) +
         part_bytes(n_tokens, n_lists, heads, k_heads, beams, 2) + place_bytes(n_tokens, n_lists, k_heads);
}

hipError_t launch_gap_step(als_dtype dtype, const GapShape &G, const GapPath &P, const als_heads &q,
                           const als_heads &k, const als_heads &v, void *out, void *workspace, hipStream_t s) {
  if (G.n_rows == 0) return hipSuccess;
  const int32_t k_heads = G.heads / G.group;
  StepArgs A{};
  A.G = G;
  A.P = P;
  A.q = q;
  A.k = k;
  A.v = v;
  A.out = out;
  A.parts = (float *)workspace;
  A.stats = (float *)((char *)workspace + part_bytes(G.n_tokens, G.n_rows, G.heads, k_heads, P.beams, G.width));
  A.shift = step_shift(G.n_tokens, k_heads);
  if (place_bytes(G.n_tokens, G.n_rows, k_heads)) {
    Place *places =
        (Place *)((char *)A.stats + part_bytes(G.n_tokens, G.n_rows, G.heads, k_heads, P.beams, 2));
    A.places = places;
    const int64_t slots = (G.n_tokens >> A.shift) + G.n_rows;  // below 2^31
    hipLaunchKernelGGL(k_gap_places, dim3((unsigned)((slots + 255) / 256)), dim3(256), 0, s, G, A.shift, slots,
                       places);
  }
  const int size = dtype == ALS_F32 ? 4 : 2;
  const auto vec = [&](const als_heads &h) {
    return aligned16(h.data, h.token_stride, h.head_stride, G.width, size);
  };
  A.vec = vec(q) && vec(k) && vec(v);
  A.vec_path = vec(P.k) && vec(P.v) && (P.k_step * size) % 16 == 0 && (P.v_step * size) % 16 == 0;
  return dtype == ALS_F32 ? launch_step<float>(A, s) : launch_step<bf16>(A, s);
}

}  // namespace als
