// Beam search's selection over beams and items, and the reordering of the beams' states.
//
// A list (one user's answer) is kept as W beams. Beam w extended by item v has the score
//   c_w + x_wv - max_v x - log sum_v exp(x_wv - max_v x),
// with the beam's score c and its logits x; the best `width` of the W V candidates go on, equal
// scores by the lowest (w, v). A finished beam has one candidate: the end item, at its own score.
// Masked items (-inf or NaN) and dead beams (a score of -inf or NaN) have none.
//
// The logits are read once, by k_slices: a block keeps a slice of a row in registers, takes its
// maximum and its sum of exponentials, and writes the slice's best `width` items. Within a row
// scores order as logits do, so those are all that can be chosen. k_merge takes one list's slices,
// forms log-sum-exp and scores in fp64 from them (so that two candidates tie only where their
// logits do) and picks the best `width`, one at a time, from the heads of the sorted slices.
#include <cfloat>

#include "internal.h"
#include "sequence.h"

namespace als {

namespace {

constexpr int kThreads = 256;
constexpr int kSlice = 8192;             // items a slice
constexpr int kHeld = kSlice / kThreads; // of them in one thread's registers
constexpr int kFound = 256;              // candidates that k_slices ranks at once
constexpr int kMergeThreads = 256;

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

__device__ __forceinline__ float usable(float x) {
  return x > -INFINITY ? fminf(x, FLT_MAX) : -INFINITY;  // NaN compares false
}

struct SliceStats {
  float max, sum;  // of the slice; sum of exp(x - max)
};

template <typename T>
__global__ __launch_bounds__(kThreads) void k_slices(const T *__restrict__ logits, int64_t n_items,
                                                     int64_t row_stride, int slices, int width,
                                                     const uint8_t *__restrict__ finished,
                                                     const float *__restrict__ scores,
                                                     SliceStats *__restrict__ stats,
                                                     uint64_t *__restrict__ best) {
  constexpr int E = 16 / sizeof(T);
  __shared__ float part[kThreads / 64], total[kThreads / 64], bound[kThreads / 64];
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
  float m = mine;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
  // the width-th largest of the lanes' maxima: at least `width` items of the wave reach it
  float sorted = mine;
#pragma unroll
  for (int size = 2; size <= 64; size *= 2)
#pragma unroll
    for (int o = size / 2; o > 0; o >>= 1) {
      const float other = __shfl_xor(sorted, o);
      const bool larger = ((lane & o) == 0) == ((lane & size) == 0);  // descending at the end
      sorted = larger ? fmaxf(sorted, other) : fminf(sorted, other);
    }
  const float reach = __shfl(sorted, width - 1);
  if (lane == 0) {
    part[wave] = m;
    bound[wave] = reach;
  }
  __syncthreads();
  m = part[0];
  float least = bound[0];
#pragma unroll
  for (int w = 1; w < kThreads / 64; ++w) {
    m = fmaxf(m, part[w]);
    least = fmaxf(least, bound[w]);
  }
  float sum = 0.f;
  if (m > -INFINITY) {
#pragma unroll
    for (int j = 0; j < kHeld; ++j) sum += __expf(v[j] - m);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
  if (lane == 0) total[wave] = sum;
#pragma unroll
  for (int j = 0; j < kHeld; ++j)
    if (v[j] >= least && v[j] > -INFINITY) {
      const int n = atomicAdd(&n_found, 1);
      if (n < kFound) found[n] = key_of(v[j], item(j));
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
  uint64_t place;  // beam << 32 | item
};
__device__ __forceinline__ bool better(const Candidate &a, const Candidate &b) {
  return a.score > b.score || (a.score == b.score && a.place < b.place);
}

__global__ __launch_bounds__(kMergeThreads) void k_merge(
    int beams, int width, int slices, const float *__restrict__ scores,
    const uint8_t *__restrict__ finished, int32_t end, const SliceStats *__restrict__ stats,
    const uint64_t *__restrict__ best, int32_t *__restrict__ parents, int32_t *__restrict__ tokens,
    float *__restrict__ scores_out, uint8_t *__restrict__ finished_out) {
  __shared__ double base[kMaxBeams], top[kMaxBeams];
  __shared__ Candidate wave_best[kMergeThreads / 64];
  __shared__ Candidate chosen;
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t list = blockIdx.x;
  scores += list * beams;
  if (finished) finished += list * beams;
  stats += list * beams * slices;
  best += list * beams * slices * width;
  // score of an item: base + (x - top)
  for (int w = wave; w < beams; w += kMergeThreads / 64) {
    const float c = scores[w];
    const bool live = c > -INFINITY && !(finished && finished[w]);
    float m = -INFINITY;
    if (live)
      for (int i = lane; i < slices; i += 64) m = fmaxf(m, stats[w * slices + i].max);
    for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
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
    }
  }
  __syncthreads();
  // each thread keeps the best unused head of its (beam, slice) lists
  const int lists = beams * slices;
  Candidate last = {INFINITY, 0};
  for (int i = 0; i < width; ++i) {
    Candidate mine = {-INFINITY, ~0ull};
    for (int l = tid; l < lists; l += kMergeThreads) {
      const int w = l / slices;
      if (!(scores[w] > -INFINITY)) continue;
      if (finished && finished[w]) {
        const Candidate c = {base[w], (uint64_t)w << 32 | (uint32_t)end};
        if (l == w * slices && (i == 0 || better(last, c)) && better(c, mine)) mine = c;
        continue;
      }
      for (int j = 0; j < width; ++j) {
        const uint64_t key = best[(int64_t)l * width + j];
        if (!key) break;
        const Candidate c = {base[w] + ((double)from_ordered((uint32_t)(key >> 32)) - top[w]),
                             (uint64_t)w << 32 | (0xffffffffu - (uint32_t)key)};
        if (i == 0 || better(last, c)) {
          if (better(c, mine)) mine = c;
          break;
        }
      }
    }
    for (int o = 32; o > 0; o >>= 1) {
      const Candidate c = {__shfl_xor(mine.score, o), __shfl_xor(mine.place, o)};
      if (better(c, mine)) mine = c;
    }
    if (lane == 0) wave_best[wave] = mine;
    __syncthreads();
    if (tid == 0) {
      for (int w = 1; w < kMergeThreads / 64; ++w)
        if (better(wave_best[w], mine)) mine = wave_best[w];
      chosen = mine;
      const bool any = mine.place != ~0ull;
      const int p = any ? (int)(mine.place >> 32) : 0;
      const int t = any ? (int)(uint32_t)mine.place : -1;
      const int64_t to = list * width + i;
      parents[to] = p;
      tokens[to] = t;
      scores_out[to] = any ? (float)mine.score : -INFINITY;
      finished_out[to] = any && ((finished && finished[p]) || t == end);
    }
    __syncthreads();
    last = chosen;
  }
}

// Copies rows of `bytes` bytes, a V at a time: row w of list b from row parents[b, w].
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
  hipLaunchKernelGGL(k_merge, dim3((unsigned)lists), dim3(kMergeThreads), 0, s, beams, width, slices,
                     scores, finished, end, stats, best, parents, tokens, scores_out, finished_out);
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
