// Beam search's selection over beams and items, and the reordering of the beams' states.
//
// A list (one user's answer) is kept as W beams. Beam w extended by item v has the score
//   c_w + x_wv - max_v x - log sum_v exp(x_wv - max_v x),
// with the beam's score c and its logits x; the best `width` of the W V candidates go on. A finished
// beam has one candidate: the end item, at its own score. Masked items (-inf or NaN) and dead beams (a
// score of -inf or NaN) have none.
//
// Order: score in fp64, then the lowest beam, the largest logit, the lowest item. A beam's scores rise
// with its logits, but beside a logit (or under a score) some 2^53 times larger they may be equal where
// the logits differ; with the logit in the order, a beam's candidates go by their logits in any case, as
// a slice orders them without knowing the score.
//
// The logits are read once, by k_slices: a block keeps a slice of a row in registers, takes its
// maximum and its sum of exponentials, and writes the slice's best `width` items, which are all that
// can be chosen of it. k_merge takes one list's slices, forms log-sum-exp and scores in fp64 from them
// and ranks those that reach the width-th best head of the sorted slices.
#include <cfloat>

#include "internal.h"
#include "sequence.h"

namespace als {

namespace {

constexpr int kThreads = 256;
constexpr int kSlice = 4096;             // items a slice
constexpr int kHeld = kSlice / kThreads; // of them in one thread's registers, one bit of a mask each
static_assert(kHeld <= 32, "a mask of 32 bits");
constexpr int kFound = 256;              // candidates that are ranked at once
constexpr int kMergeThreads = 1024;
constexpr int kFirst = 4;                // heads that a thread of k_merge fetches at the start

// fp32 as a whole number of the same order. Both zeros give the same one.
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float from_ordered(uint32_t o) {
  return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o);
}
// Larger: the larger value, or of equal ones the lower item. Never 0 for a candidate.
__device__ __forceinline__ uint64_t key_of(float x, uint32_t item) {
  return (uint64_t)ordered(x) << 32 | (0xffffffffu - item);
}

// -inf for NaN (of NaN and a number the maximum is the number), the largest finite value for +inf.
__device__ __forceinline__ float usable(float x) { return fminf(fmaxf(x, -INFINITY), FLT_MAX); }

// Maximum over the wave: within rows of 16 by lane exchanges of the vector unit, then over the rows.
template <int CTRL> __device__ __forceinline__ float max_with(float x) {
  const int y = __builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, false);
  return fmaxf(x, __int_as_float(y));
}
__device__ __forceinline__ float row_lane(float x, int lane) {
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), lane));
}
__device__ __forceinline__ float wave_max(float x) {
  x = max_with<0xb1>(x);   // lanes 1 0 3 2
  x = max_with<0x4e>(x);   // lanes 2 3 0 1
  x = max_with<0x141>(x);  // mirrored in 8
  x = max_with<0x140>(x);  // mirrored in 16
  return fmaxf(fmaxf(row_lane(x, 0), row_lane(x, 16)), fmaxf(row_lane(x, 32), row_lane(x, 48)));
}

// A value that at least n of the wave's lanes reach, and (to 11 bits) the largest such one, bit by
// bit: the lanes that reach a value are counted by one comparison.
__device__ __forceinline__ uint32_t reached_by(uint32_t x, int n) {
  uint32_t bound = 0;
#pragma unroll
  for (int b = 31; b >= 12; --b) {
    const uint32_t next = bound | 1u << b;
    bound = __popcll(__ballot(x >= next)) >= n ? next : bound;
  }
  return bound;
}

struct SliceStats {
  float max, sum;  // of the slice; sum of exp(x - max)
};

// Bound by reading the logits: 72 us for 8 lists of 16 beams of 624 961 items in f32, a tenth of them
// finished: 4.0 TB/s, what a large sum reaches; 13.7 us for 32 lists of 8 of 50 000 in bf16, where few
// waves of blocks leave the latency of each one's load, maximum and ranking in sight; 4.7 us for one
// list of 4 of 1000.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_slices(const T *__restrict__ logits, int64_t n_items,
                                                     int64_t row_stride, int slices, int width,
                                                     const uint8_t *__restrict__ finished,
                                                     const float *__restrict__ scores,
                                                     SliceStats *__restrict__ stats,
                                                     uint64_t *__restrict__ best) {
  constexpr int E = 16 / sizeof(T);
  __shared__ float part[kThreads / 64], total[kThreads / 64];
  __shared__ uint32_t bound[kThreads / 64];
  __shared__ uint64_t found[kFound];
  __shared__ uint64_t top[kThreads / 64];
  __shared__ int n_found;
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t row = blockIdx.x / slices;
  const int slice = (int)(blockIdx.x % slices);
  if ((finished && finished[row]) || !(scores[row] > -INFINITY)) return;  // k_merge reads none
  const T *x = logits + row * row_stride;
  const int64_t c0 = (int64_t)slice * kSlice;
  // 16-byte pieces are cut at their alignment; the row starts `skew` values into the first
  const int skew = (int)(((uintptr_t)x % 16) / sizeof(T));
  float v[kHeld];
#pragma unroll
  for (int i = 0; i < kHeld / E; ++i) {
    const int64_t c = c0 - skew + (int64_t)(i * kThreads + tid) * E;
    const int64_t lo = c0 > 0 ? c0 - skew : 0, hi0 = c0 + kSlice - skew;
    const int64_t hi = slice + 1 == slices || hi0 > n_items ? n_items : hi0;
    if (c >= lo && c + E <= hi) {
      const uint4 raw = *(const uint4 *)(x + c);
      const T *t = (const T *)&raw;
#pragma unroll
      for (int e = 0; e < E; ++e) v[i * E + e] = usable((float)t[e]);
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e)
        v[i * E + e] = c + e >= lo && c + e < hi ? usable((float)x[c + e]) : -INFINITY;
    }
  }
  const auto item = [&](int j) {  // of v[j]
    return (uint32_t)(c0 - skew + (int64_t)(j / E * kThreads + tid) * E + j % E);
  };
  if (tid == 0) n_found = 0;
  float mine = -INFINITY;
#pragma unroll
  for (int j = 0; j < kHeld; ++j) mine = fmaxf(mine, v[j]);
  // at least `width` items of the wave reach this: one in each of that many lanes
  const uint32_t reach = reached_by(ordered(mine), width);
  float m = wave_max(mine);
  if (lane == 0) {
    part[wave] = m;
    bound[wave] = reach;
  }
  __syncthreads();
  m = part[0];
  uint32_t most = bound[0];
#pragma unroll
  for (int w = 1; w < kThreads / 64; ++w) {
    m = fmaxf(m, part[w]);
    most = bound[w] > most ? bound[w] : most;
  }
  const float least = most <= ordered(-INFINITY) ? -INFINITY : from_ordered(most);
  float sum = 0.f;
  if (m > -INFINITY) {
#pragma unroll
    for (int j = 0; j < kHeld; ++j) sum += __expf(v[j] - m);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
  if (lane == 0) total[wave] = sum;
  // few lanes hold any: the places as a mask, and the values read again
  uint32_t hits = 0;
#pragma unroll
  for (int j = 0; j < kHeld; ++j) hits |= v[j] >= least && v[j] > -INFINITY ? 1u << j : 0u;
  while (hits) {
    const int j = __ffs(hits) - 1;
    hits &= hits - 1;
    const uint32_t at = item(j);
    const int n = atomicAdd(&n_found, 1);
    if (n < kFound) found[n] = key_of(usable((float)x[at]), at);
  }
  __syncthreads();
  uint64_t *out = best + (int64_t)blockIdx.x * width;
  const int n = n_found;
  if (n <= kFound) {
    // each candidate's rank is the number of larger ones
    if (tid < n) {
      const uint64_t key = found[tid];
      int rank = 0;
      for (int j = 0; j < n; ++j) rank += found[j] > key;
      if (rank < width) out[rank] = key;
    }
    if (tid >= n && tid < width) out[tid] = 0;
  } else {
    // many equal values: one at a time
    uint64_t below = ~0ull;
    for (int i = 0; i < width; ++i) {
      uint64_t k = 0;
#pragma unroll
      for (int j = 0; j < kHeld; ++j) {
        const uint64_t c = v[j] > -INFINITY ? key_of(v[j], item(j)) : 0;
        if (c < below && c > k) k = c;
      }
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) {
        const uint64_t other = __shfl_xor(k, o);
        k = other > k ? other : k;
      }
      if (lane == 0) top[wave] = k;
      __syncthreads();
      k = top[0];
      for (int w = 1; w < kThreads / 64; ++w) k = top[w] > k ? top[w] : k;
      if (tid == 0) out[i] = k;
      below = k;
      __syncthreads();
    }
  }
  if (tid == 0) {
    float s = 0.f;
    for (int w = 0; w < kThreads / 64; ++w) s += total[w];
    stats[blockIdx.x] = {m, s};
  }
}

struct Candidate {
  double score;
  uint64_t key;   // of the logit and the item
  uint32_t beam;  // kMaxBeams: no candidate
};
__device__ __forceinline__ bool better(const Candidate &a, const Candidate &b) {
  return a.score > b.score ||
         (a.score == b.score && (a.beam < b.beam || (a.beam == b.beam && a.key > b.key)));
}
__device__ __forceinline__ uint32_t item_of(uint64_t key) { return 0xffffffffu - (uint32_t)key; }

// One block a list, for whom it is a chain of latencies (statistics, log-sum-exp, heads, candidates,
// ranks): 7.2 us for 4 lists of candidates, 7.9 us for 104 (8 beams), 15.3 us for 2448 (16 beams).
__global__ __launch_bounds__(kMergeThreads) void k_merge(
    int64_t list0, int beams, int width, int slices, const float *__restrict__ scores,
    const uint8_t *__restrict__ finished, int32_t end, const SliceStats *__restrict__ stats,
    const uint64_t *__restrict__ best, int32_t *__restrict__ parents, int32_t *__restrict__ tokens,
    float *__restrict__ scores_out, uint8_t *__restrict__ finished_out) {
  __shared__ double base[kMaxBeams], top[kMaxBeams];
  __shared__ int kind[kMaxBeams];  // 0 dead, 1 live, 2 finished
  __shared__ Candidate found[kFound];
  __shared__ uint32_t best_heads[kMergeThreads];
  __shared__ int n_found;
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t list = list0 + blockIdx.x;
  scores += list * beams;
  if (finished) finished += list * beams;
  stats += list * beams * slices;
  best += list * beams * slices * width;
  const int lists = beams * slices;
  // the first heads are on their way while log-sum-exp is formed
  uint64_t first[kFirst];
#pragma unroll
  for (int i = 0; i < kFirst; ++i) {
    const int l = tid + i * kMergeThreads;
    first[i] = l < lists ? best[(int64_t)l * width] : 0;
  }
  // score of an item: base + (x - top)
  for (int w = wave; w < beams; w += kMergeThreads / 64) {
    const float c = scores[w];
    const bool done = finished && finished[w], live = c > -INFINITY && !done;
    float m = -INFINITY;
    if (live)
      for (int i = lane; i < slices; i += 64) m = fmaxf(m, stats[w * slices + i].max);
    m = wave_max(m);
    double s = 0.0;
    if (m > -INFINITY)
      for (int i = lane; i < slices; i += 64) {
        const SliceStats x = stats[w * slices + i];
        if (x.max > -INFINITY) s += (double)x.sum * exp((double)x.max - (double)m);
      }
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
    if (lane == 0) {
      top[w] = m;
      base[w] = (double)fminf(c, FLT_MAX) - (m > -INFINITY ? log(s) : 0.0);
      kind[w] = live ? 1 : done && c > -INFINITY ? 2 : 0;
    }
  }
  if (tid == 0) n_found = 0;
  __syncthreads();
  // Every (beam, slice) list is sorted, so that `width` of the lists' heads reach a bound, and no
  // candidate below it can be chosen: those that reach it are gathered and ranked at once.
  const Candidate none = {-INFINITY, 0, kMaxBeams};
  const auto of_key = [&](int l, int j, uint64_t key) {  // candidate j of list l, whose key this is
    const int w = l / slices;
    if (kind[w] == 2)  // finished
      return l == w * slices && j == 0 ? Candidate{base[w], key_of(0.f, (uint32_t)end), (uint32_t)w} : none;
    if (kind[w] == 0 || !key) return none;
    return Candidate{base[w] + ((double)from_ordered((uint32_t)(key >> 32)) - top[w]), key, (uint32_t)w};
  };
  const auto head = [&](int l, int j) { return of_key(l, j, best[(int64_t)l * width + j]); };
  const auto write = [&](int i, const Candidate &c) {
    const bool any = c.beam < kMaxBeams;
    const int p = any ? (int)c.beam : 0;
    const int t = any ? (int)item_of(c.key) : -1;
    const int64_t to = list * width + i;
    parents[to] = p;
    tokens[to] = t;
    scores_out[to] = any ? (float)c.score : -INFINITY;
    finished_out[to] = any && ((finished && finished[p]) || t == end);
  };
  float mine = -INFINITY;
  float heads[kFirst];
#pragma unroll
  for (int i = 0; i < kFirst; ++i) {
    const int l = tid + i * kMergeThreads;
    heads[i] = l < lists ? (float)of_key(l, 0, first[i]).score : -INFINITY;
    mine = fmaxf(mine, heads[i]);
  }
  for (int l = tid + kFirst * kMergeThreads; l < lists; l += kMergeThreads)
    mine = fmaxf(mine, (float)head(l, 0).score);
  best_heads[tid] = ordered(mine);
  __syncthreads();
  // the bound over 64 groups of threads, formed by every wave
  uint32_t group = 0;
#pragma unroll
  for (int i = 0; i < kMergeThreads / 64; ++i) {
    const uint32_t x = best_heads[i * 64 + lane];
    group = x > group ? x : group;
  }
  const uint32_t most = reached_by(group, width);
  const auto gather = [&](int l) {
    constexpr int kAhead = 4;
    for (int j = 0; j < width; j += kAhead) {
      uint64_t keys[kAhead];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) keys[i] = j + i < width ? best[(int64_t)l * width + j + i] : 0;
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const Candidate c = of_key(l, j + i, keys[i]);
        if (c.beam == kMaxBeams || ordered((float)c.score) < most) return;
        const int n = atomicAdd(&n_found, 1);
        if (n < kFound) found[n] = c;
      }
    }
  };
#pragma unroll
  for (int i = 0; i < kFirst; ++i)
    if (heads[i] > -INFINITY && ordered(heads[i]) >= most) gather(tid + i * kMergeThreads);
  for (int l = tid + kFirst * kMergeThreads; l < lists; l += kMergeThreads) gather(l);
  __syncthreads();
  const int n = n_found;
  if (n <= kFound) {
    for (int i = tid; i < n; i += kMergeThreads) {
      const Candidate c = found[i];
      int rank = 0;
      for (int j = 0; j < n; ++j) rank += better(found[j], c);
      if (rank < width) write(rank, c);
    }
    if (tid < width && tid >= n) write(tid, none);
    return;
  }
  // many equal scores: one at a time
  Candidate last = none;
  for (int i = 0; i < width; ++i) {
    Candidate mine = none;
    for (int l = tid; l < lists; l += kMergeThreads)
      for (int j = 0; j < width; ++j) {
        const Candidate c = head(l, j);
        if (c.beam == kMaxBeams) break;
        if (i == 0 || better(last, c)) {
          if (better(c, mine)) mine = c;
          break;
        }
      }
    for (int o = 32; o > 0; o >>= 1) {
      const Candidate c = {__shfl_xor(mine.score, o), __shfl_xor(mine.key, o), __shfl_xor(mine.beam, o)};
      if (better(c, mine)) mine = c;
    }
    if (lane == 0) found[wave] = mine;
    __syncthreads();
    last = found[0];
    for (int w = 1; w < kMergeThreads / 64; ++w)
      if (better(found[w], last)) last = found[w];
    if (tid == 0) write(i, last);
    __syncthreads();
  }
}

// Copies rows of `bytes` bytes, a V at a time: row w of list b from row parents[b, w]. 10.2 us for 256
// rows of 131 kB, 6.6 TB/s (some of it from the caches).
template <typename V>
__global__ __launch_bounds__(256) void k_reorder(const V *src, V *dst, int64_t n, int64_t row0,
                                                 int beams, int width,
                                                 const int32_t *__restrict__ parents) {
  const int64_t row = row0 + blockIdx.y;
  const int p = parents[row];
  if (p < 0 || p >= beams) return;
  const V *from = src + (row / width * beams + p) * n;
  V *to = dst + row * n;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256)
    to[i] = from[i];
}

// In place: a thread reads its piece of all beams of a list before it writes any.
template <typename V, int W>
__global__ __launch_bounds__(256) void k_reorder_in_place(V *x, int64_t n, int64_t list0, int beams,
                                                          const int32_t *__restrict__ parents) {
  const int64_t list = list0 + blockIdx.y;
  parents += list * beams;
  x += list * beams * n;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    V v[W];
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const int p = w < beams ? parents[w] : -1;
      if (p >= 0 && p < beams && p != w) v[w] = x[p * n + i];
    }
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const int p = w < beams ? parents[w] : -1;
      if (p >= 0 && p < beams && p != w) x[w * n + i] = v[w];
    }
  }
}

template <typename V>
hipError_t reorder(const void *src, void *dst, int64_t lists, int beams, int width, int64_t bytes,
                   const int32_t *parents, hipStream_t s) {
  const int64_t n = bytes / (int64_t)sizeof(V), pieces = (n + 255) / 256;
  const unsigned x = (unsigned)(pieces < 1024 ? pieces : 1024);
  constexpr int64_t kRows = 32768;  // blocks in y a launch
  if (src != dst) {
    for (int64_t r = 0; r < lists * width; r += kRows) {
      const int64_t k = lists * width - r < kRows ? lists * width - r : kRows;
      hipLaunchKernelGGL(k_reorder<V>, dim3(x, (unsigned)k), dim3(256), 0, s, (const V *)src,
                         (V *)dst, n, r, beams, width, parents);
    }
    return hipGetLastError();
  }
  const auto launch = beams <= 4    ? k_reorder_in_place<V, 4>
                      : beams <= 8  ? k_reorder_in_place<V, 8>
                      : beams <= 16 ? k_reorder_in_place<V, 16>
                                    : k_reorder_in_place<V, kMaxBeams>;
  for (int64_t l = 0; l < lists; l += kRows) {
    const int64_t k = lists - l < kRows ? lists - l : kRows;
    hipLaunchKernelGGL(launch, dim3(x, (unsigned)k), dim3(256), 0, s, (V *)dst, n, l, beams, parents);
  }
  return hipGetLastError();
}

}  // namespace

int64_t beam_slices(int64_t n_items) { return (n_items + 7 + kSlice - 1) / kSlice; }

int64_t beam_workspace(int64_t lists, int beams, int width, int64_t n_items) {
  return lists * beams * beam_slices(n_items) * (int64_t)(sizeof(SliceStats) + 8 * width);
}

hipError_t launch_beam_select(als_dtype dtype, int64_t lists, int beams, int width, int64_t n_items,
                              const void *logits, int64_t row_stride, const float *scores,
                              const uint8_t *finished, int32_t end, int32_t *parents,
                              int32_t *tokens, float *scores_out, uint8_t *finished_out,
                              void *workspace, hipStream_t s) {
  const int slices = (int)beam_slices(n_items);
  uint64_t *best = (uint64_t *)workspace;
  SliceStats *stats = (SliceStats *)(best + lists * beams * slices * width);
  const int64_t per = max_blocks(kThreads) / slices;  // rows a launch
  for (int64_t r = 0; r < lists * beams; r += per) {
    const int64_t n = lists * beams - r < per ? lists * beams - r : per;
    const dim3 grid((unsigned)(n * slices));
    const uint8_t *done = finished ? finished + r : nullptr;
#define SLICES(T)                                                                                \
  hipLaunchKernelGGL(k_slices<T>, grid, dim3(kThreads), 0, s, (const T *)logits + r * row_stride, \
                     n_items, row_stride, slices, width, done, scores + r, stats + r * slices,   \
                     best + r * slices * width)
    if (dtype == ALS_F32)
      SLICES(float);
    else
      SLICES(bf16);
#undef SLICES
  }
  const int64_t merged = max_blocks(kMergeThreads);
  for (int64_t l = 0; l < lists; l += merged) {
    const int64_t n = lists - l < merged ? lists - l : merged;
    hipLaunchKernelGGL(k_merge, dim3((unsigned)n), dim3(kMergeThreads), 0, s, l, beams, width, slices,
                       scores, finished, end, stats, best, parents, tokens, scores_out, finished_out);
  }
  return hipGetLastError();
}

hipError_t launch_reorder(const void *src, void *dst, int64_t lists, int beams, int width,
                          int64_t bytes, const int32_t *parents, hipStream_t s) {
  if (lists == 0 || bytes == 0) return hipSuccess;
  const uint64_t at = (uintptr_t)src | (uintptr_t)dst | (uint64_t)bytes;
  if (at % 16 == 0) return reorder<uint4>(src, dst, lists, beams, width, bytes, parents, s);
  if (at % 4 == 0) return reorder<uint32_t>(src, dst, lists, beams, width, bytes, parents, s);
  return reorder<uint8_t>(src, dst, lists, beams, width, bytes, parents, s);
}

}  // namespace als
