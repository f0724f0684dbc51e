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
// Rounding. Products run in the inputs' type with sums in fp32. bf16: the weights and the state are
// rounded once more where they enter a product, which is as much again as the output's own rounding.
// What a token adds to the state is split into three bf16 parts (24 bits), so that the state, an
// output in fp32, has no bf16 rounding in it.
#include "internal.h"
#include "sequence.h"

namespace als {

namespace {

constexpr float kLog2e = 1.44269504088896340736f;
// Decays below e^-10000 a token are the same as none left; keeps -inf * 0 out of the exponents.
constexpr float kMinLogDecay = -1e4f;

// ---- fragments: 8 values of a contraction of 32 per lane ---------------------------------------
// Lane l holds, for row (or column) l & 15, the places 4 g .. 4 g + 3 and 16 + 4 g .. 16 + 4 g + 3
// with g = l >> 4: the order in which two result tiles of an MFMA hold their rows, so that results
// are operands of the next product as they are. (A sum's terms may come in any order, provided both
// operands use the same.)
template <typename T> struct Frag;
template <> struct Frag<float> {
  f32x4 lo, hi;
  __device__ __forceinline__ float get(int e) const { return e < 4 ? lo[e] : hi[e - 4]; }
  __device__ __forceinline__ void set(int e, float v) {
    if (e < 4) lo[e] = v; else hi[e - 4] = v;
  }
};
template <> struct Frag<bf16> {
  bf16x8 x;
  __device__ __forceinline__ bf16 get(int e) const { return x[e]; }
  __device__ __forceinline__ void set(int e, bf16 v) { x[e] = v; }
};

template <typename T> struct Vec4;
template <> struct Vec4<float> { using type = f32x4; };
template <> struct Vec4<bf16> { using type = bf16x4; };

__device__ __forceinline__ Frag<float> joined(f32x4 lo, f32x4 hi) { return {lo, hi}; }
__device__ __forceinline__ Frag<bf16> joined(bf16x4 lo, bf16x4 hi) {
  return {__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7)};
}

__device__ __forceinline__ f32x4 mma(const Frag<bf16> &a, const Frag<bf16> &b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.x, b.x, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma(const Frag<float> &a, const Frag<float> &b, f32x4 c) {
#pragma unroll
  for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.lo[e], b.lo[e], c, 0, 0, 0);
#pragma unroll
  for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.hi[e], b.hi[e], c, 0, 0, 0);
  return c;
}

// Row l & 15 of a 16-row tile at x (row length ld), contraction along the row from column 0.
template <typename T>
__device__ __forceinline__ Frag<T> frag_row(const T *x, int ld, int lane) {
  using V = typename Vec4<T>::type;
  const T *p = x + (lane & 15) * ld + (lane >> 4) * 4;
  return joined(*(const V *)p, *(const V *)(p + 16));
}
// Column l & 15 of a 16-column tile at x, contraction down 32 rows.
__device__ __forceinline__ Frag<float> frag_col(const float *x, int ld, int lane) {
  const float *p = x + (lane >> 4) * 4 * ld + (lane & 15);
  Frag<float> f;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    f.lo[e] = p[e * ld];
    f.hi[e] = p[(16 + e) * ld];
  }
  return f;
}
// The transposing LDS read: 16 lanes name the 16 8-byte pieces of a 4 x 16 block, and lane i of
// them gets column i.
__device__ __forceinline__ Frag<bf16> frag_col(const bf16 *x, int ld, int lane) {
  using L = __attribute__((address_space(3))) bf16x4 *;
  const bf16 *p = x + (lane >> 2) * ld + (lane & 3) * 4;
  return joined(__builtin_amdgcn_ds_read_tr16_b64_v4bf16((L)p),
                __builtin_amdgcn_ds_read_tr16_b64_v4bf16((L)(p + 16 * ld)));
}

template <typename T> __device__ __forceinline__ typename Vec4<T>::type rounded(f32x4 x) {
  return __builtin_convertvector(x, typename Vec4<T>::type);
}

// Padding of a staged row: with it the four lane groups and the rows of one LDS read fall on
// different banks.
template <typename T> constexpr int padded(int width) { return width + (sizeof(T) == 2 ? 16 : 4); }

template <typename T> constexpr int chunk_tokens() { return sizeof(T) == 2 ? 64 : 32; }

// Row and place of a slot. Row b's segments have the slots row_ptr[b] / L + b onwards: at least as
// many as it has segments, one for an empty row, and never another row's.
struct Place {
  int64_t row, first, len;  // the row, its first token and length
  int64_t segment;          // of the row
};

// One wave searches 64 rows at a time. Values of row_ptr outside [0, n_tokens] are taken as the
// nearest inside, so that nothing outside the tensors is touched whatever it holds.
__device__ __forceinline__ int64_t clamped(int64_t x, int64_t lo, int64_t hi) {
  return x < lo ? lo : (x > hi ? hi : x);
}
__device__ __forceinline__ Place find_place(const int64_t *__restrict__ row_ptr, int64_t n_rows,
                                            int64_t n_tokens, int64_t L, int64_t slot, int lane) {
  int64_t lo = 0, hi = n_rows;
  while (hi - lo > 1) {
    const int64_t step = (hi - lo + 63) / 64, at = lo + lane * step;
    const bool before = at < hi && clamped(row_ptr[at], 0, n_tokens) / L + at <= slot;
    const int n = __popcll(__ballot(before));
    lo += (n > 0 ? n - 1 : 0) * step;
    hi = lo + step < hi ? lo + step : hi;
  }
  Place p;
  p.row = lo;
  p.first = clamped(row_ptr[lo], 0, n_tokens);
  p.len = clamped(row_ptr[lo + 1], p.first, n_tokens) - p.first;
  p.segment = slot - (p.first / L + lo);
  return p;
}

struct Args {
  AttentionPass p;
  int64_t segment;  // tokens a segment
  int64_t slot0;    // first slot of this launch
  int vec;          // bit 0: q, 1: k, 2: v read 16 bytes at a time, 3: out written 4 values at a time
};

// Stages `size` tokens of one head of x, zero past them and past `width`, into rows of LD elements.
template <typename T, int C, int WP, int THREADS>
__device__ __forceinline__ void stage(T *lds, const T *__restrict__ x, int64_t token_stride,
                                      int64_t first, int64_t step, int size, int width, bool vec) {
  constexpr int LD = padded<T>(WP), E = 16 / sizeof(T), PIECES = C * WP / E;
#pragma unroll
  for (int i = 0; i < (PIECES + THREADS - 1) / THREADS; ++i) {
    const int n = i * THREADS + (int)threadIdx.x;
    if (PIECES % THREADS != 0 && n >= PIECES) break;
    const int r = n / (WP / E), c = n % (WP / E) * E;
    T v[E];
    if (vec) {
      uint4 raw = make_uint4(0, 0, 0, 0);
      if (r < size && c < width) raw = *(const uint4 *)(x + (first + r * step) * token_stride + c);
      *(uint4 *)(lds + r * LD + c) = raw;
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e)
        v[e] = r < size && c + e < width ? x[(first + r * step) * token_stride + c + e] : (T)0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) lds[r * LD + c + e] = v[e];
    }
  }
}

__device__ __forceinline__ void split3(f32x4 x, bf16x4 *part) {
#pragma unroll
  for (int n = 0; n < 3; ++n) {
    part[n] = rounded<bf16>(x);
    x -= __builtin_convertvector(part[n], f32x4);
  }
}

// One block: one head of one segment. STATES: only the state after the segment, for all segments of
// a row but its last.
template <typename T, int KP, int VP, bool STATES>
__global__ __launch_bounds__(VP * 4) void k_attention(Args A) {
  constexpr int C = chunk_tokens<T>(), NT = C / 16, NW = VP / 16, THREADS = NW * 64;
  constexpr int KT = KP / 16, KF = KP / 32, SF = C / 32, LK = padded<T>(KP), LV = padded<T>(VP);
  constexpr int PT = NT * (NT + 1) / 2;
  using V4 = typename Vec4<T>::type;
  __shared__ __align__(16) T lq[STATES ? 1 : C * LK];
  __shared__ __align__(16) T lk[C * LK];
  __shared__ __align__(16) T lv[C * LV];
  __shared__ __align__(16) T lp[STATES ? 1 : PT * 256];

  const AttentionPass &P = A.p;
  const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6, g = lane >> 4, m = lane & 15;
  const int64_t slot = A.slot0 + blockIdx.x / P.heads;
  const int head = (int)(blockIdx.x % P.heads);
  const Place at = find_place(P.row_ptr, P.n_rows, P.n_tokens, A.segment, slot, lane);
  const int64_t n_segments = (at.len + A.segment - 1) / A.segment;
  const bool last = at.segment == (n_segments > 0 ? n_segments - 1 : 0);
  if (at.segment < 0 || at.segment >= (n_segments > 0 ? n_segments : 1) || (STATES && last)) return;

  const float raw = P.log_decay[head];
  // a decay above one (or NaN) has no meaning here: its head becomes NaN
  const float a2 = (raw <= 0.f ? fmaxf(raw, kMinLogDecay) : __builtin_nanf("")) * kLog2e;
  const int read_off = P.reverse ? 0 : 1, add_off = P.reverse ? 1 : 0;

  // the state: tile kt holds rows 16 kt + 4 g + e of its column 16 wave + m
  f32x4 S[KT];
  const int64_t state = (at.row * P.heads + head) * (int64_t)P.k_width * P.v_width;
  const int col = wave * 16 + m;
  float *slot_state = P.segments + ((slot * P.heads + head) * (int64_t)(KT * NW) + wave * KT) * 256 +
                      lane * 4;
#pragma unroll
  for (int kt = 0; kt < KT; ++kt) {
    S[kt] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (at.segment > 0 && !STATES) {
      S[kt] = *(const f32x4 *)(slot_state + kt * 256);
    } else if (at.segment == 0 && P.first_state) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int r = kt * 16 + g * 4 + e;
        if (r < P.k_width && col < P.v_width)
          S[kt][e] = P.first_state[state + r * P.first_ld[0] + col * P.first_ld[1]];
      }
    }
  }

  const int64_t begin = at.segment * A.segment;
  const int64_t end = begin + A.segment < at.len ? begin + A.segment : at.len;
  const T *q = (const T *)P.q.data + head / P.q_group * P.q.head_stride;
  const T *k = (const T *)P.k.data + head / P.group * P.k.head_stride;
  const T *v = (const T *)P.v.data + head / P.v_group * P.v.head_stride;
  const int64_t step = P.reverse ? -1 : 1;

  float read[NT];  // of place 16 i + m
#pragma unroll
  for (int i = 0; i < NT; ++i) read[i] = P.read_scale * exp2f(a2 * (float)(16 * i + m + read_off));

  for (int64_t c = begin; c < end; c += C) {
    const int size = (int)(end - c < C ? end - c : C);
    const int64_t first = P.reverse ? at.first + at.len - 1 - c : at.first + c;
    __syncthreads();
    if (!STATES)
      stage<T, C, KP, THREADS>(lq, q, P.q.token_stride, first, step, size, P.k_width, A.vec & 1);
    stage<T, C, KP, THREADS>(lk, k, P.k.token_stride, first, step, size, P.k_width, A.vec & 2);
    stage<T, C, VP, THREADS>(lv, v, P.v.token_stride, first, step, size, P.v_width, A.vec & 4);
    __syncthreads();

    Frag<T> vf[SF];  // column `col` of v
#pragma unroll
    for (int s = 0; s < SF; ++s) vf[s] = frag_col(lv + s * 32 * LV + wave * 16, LV, lane);

    if (!STATES) {
      // weights of places i (columns) and j (rows) <= i, one 16 x 16 tile at a time
#pragma unroll
      for (int n = 0; n < (PT + NW - 1) / NW; ++n) {
        const int tile = n * NW + wave;
        if (tile < PT) {
          int i = 0;
          while ((i + 1) * (i + 2) / 2 <= tile) ++i;
          const int j = tile - i * (i + 1) / 2;
          f32x4 w = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int d = 0; d < KF; ++d)
            w = mma(frag_row(lk + j * 16 * LK + d * 32, LK, lane),
                    frag_row(lq + i * 16 * LK + d * 32, LK, lane), w);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int gap = 16 * (i - j) + m - g * 4 - e;
            w[e] = gap >= 0 ? w[e] * (P.weight_scale * exp2f(a2 * (float)gap)) : 0.f;
          }
          *(V4 *)(lp + tile * 256 + lane * 4) = rounded<T>(w);
        }
      }
      // what the state before the chunk gives: rows 16 wave + 4 g + e of v, column 16 i + m
      f32x4 o[NT];
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int d = 0; d < KF; ++d)
          o[i] = mma(joined(rounded<T>(S[2 * d]), rounded<T>(S[2 * d + 1])),
                     frag_row(lq + i * 16 * LK + d * 32, LK, lane), o[i]);
        o[i] *= read[i];
      }
      __syncthreads();
      // 0 * inf and 0 * NaN are NaN: values of v that are neither enter the products as zeros, and
      // are added to their own and later places alone
      float finite = 0.f;
#pragma unroll
      for (int s = 0; s < SF; ++s)
#pragma unroll
        for (int e = 0; e < 8; ++e) finite = fmaf((float)vf[s].get(e), 0.f, finite);
      const bool all_finite = !__any(finite != 0.f);
      Frag<T> vc[SF];
#pragma unroll
      for (int s = 0; s < SF; ++s) vc[s] = vf[s];
      if (!all_finite) {
#pragma unroll
        for (int s = 0; s < SF; ++s)
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if ((float)vf[s].get(e) * 0.f != 0.f) vc[s].set(e, (T)0.f);
      }
#pragma unroll
      for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int s = 0; s <= i / 2; ++s) {
          const T *t = lp + (i * (i + 1) / 2 + 2 * s) * 256 + lane * 4;
          const V4 zero = {(T)0.f, (T)0.f, (T)0.f, (T)0.f};
          o[i] = mma(vc[s], joined(*(const V4 *)t, 2 * s + 1 <= i ? *(const V4 *)(t + 256) : zero),
                     o[i]);
        }
      if (!all_finite) {
        for (int i = 0; i < NT; ++i) {
          f32x4 add = {0.f, 0.f, 0.f, 0.f};
          for (int j = 0; j <= 16 * i + m; ++j) {
            const float w = (float)lp[(i * (i + 1) / 2 + j / 16) * 256 + (m + j % 16 / 4 * 16) * 4 + j % 4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float x = (float)lv[j * LV + wave * 16 + g * 4 + e];
              if (x * 0.f != 0.f) add[e] = fmaf(w, x, add[e]);
            }
          }
#pragma unroll
          for (int n = 0; n < NT; ++n)
            if (n == i) o[n] += add;
        }
      }
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        const int place = 16 * i + m, c0 = wave * 16 + g * 4;
        if (place < size && c0 < P.v_width) {
          const int64_t to = ((first + place * step) * P.heads + head) * (int64_t)P.v_width + c0;
          if (P.out_f32) {
            float *x = (float *)P.out + to;
            if (A.vec & 8) {
              *(f32x4 *)x = o[i];
            } else {
              for (int e = 0; e < 4; ++e)
                if (c0 + e < P.v_width) x[e] = o[i][e];
            }
          } else {
            T *x = (T *)P.out + to;
            const V4 r = rounded<T>(o[i]);
            if (A.vec & 8) {
              *(V4 *)x = r;
            } else {
              for (int e = 0; e < 4; ++e)
                if (c0 + e < P.v_width) x[e] = r[e];
            }
          }
        }
      }
    }

    // S <- e^{a size} S + sum_j k_j (e^{a (size - 1 - j + add_off)} update_scale v_j)^T
    const float whole = exp2f(a2 * (float)size);
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) S[kt] *= whole;
#pragma unroll
    for (int s = 0; s < SF; ++s) {
      f32x4 w[2];
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int left = size - 1 - (s * 32 + h * 16 + g * 4 + e);
          w[h][e] = left >= 0 ? P.update_scale * exp2f(a2 * (float)(left + add_off)) : 0.f;
        }
      if constexpr (sizeof(T) == 2) {
        bf16x4 part[2][3];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          f32x4 x;
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = w[h][e] * (float)vf[s].x[h * 4 + e];
          split3(x, part[h]);
        }
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) {
          const Frag<bf16> kf = frag_col(lk + s * 32 * LK + kt * 16, LK, lane);
#pragma unroll
          for (int n = 0; n < 3; ++n) S[kt] = mma(kf, joined(part[0][n], part[1][n]), S[kt]);
        }
      } else {
        const Frag<float> x = {vf[s].lo * w[0], vf[s].hi * w[1]};
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
          S[kt] = mma(frag_col(lk + s * 32 * LK + kt * 16, LK, lane), x, S[kt]);
      }
    }
  }

  if (STATES) {
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) *(f32x4 *)(slot_state + kt * 256) = S[kt];
  } else if (last && P.last_state) {
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int r = kt * 16 + g * 4 + e;
        if (r < P.k_width && col < P.v_width)
          P.last_state[state + r * P.last_ld[0] + col * P.last_ld[1]] = S[kt][e];
      }
  }
}

// States after each segment alone -> states before each segment. One thread a value of the state,
// one block a part of one head of one row.
__global__ __launch_bounds__(256) void k_join_segments(float *segments, const int64_t *row_ptr,
                                                       int64_t row0, int64_t n_tokens,
                                                       int64_t n_slots, int64_t L, int heads,
                                                       const float *log_decay, int64_t floats) {
  const int64_t row = row0 + blockIdx.x / heads;
  const int head = (int)(blockIdx.x % heads);
  const int64_t first = clamped(row_ptr[row], 0, n_tokens);
  const int64_t len = clamped(row_ptr[row + 1], first, n_tokens) - first;
  const int64_t slot = first / L + row;
  const int64_t n = (len + L - 1) / L;
  const int64_t x = (int64_t)blockIdx.y * 256 + threadIdx.x;
  if (n < 2 || x >= floats || slot + n > n_slots) return;
  const float raw = log_decay[head];
  const float a2 = (raw <= 0.f ? fmaxf(raw, kMinLogDecay) : __builtin_nanf("")) * kLog2e;
  const float whole = exp2f(a2 * (float)L);
  float *p = segments + (slot * heads + head) * floats + x;
  const int64_t stride = heads * floats;
  float state = p[0];
  for (int64_t j = 1; j < n; ++j) {
    const float own = j + 1 < n ? p[j * stride] : 0.f;
    p[j * stride] = state;
    state = fmaf(whole, state, own);
  }
}

template <typename T>
__global__ __launch_bounds__(256) void k_sum_groups(const float *__restrict__ x, int64_t n, int group,
                                                    int width, T *__restrict__ out) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int64_t head = i / width;
    const float *p = x + head * group * width + (i - head * width);
    float sum = p[0];
    for (int j = 1; j < group; ++j) sum += p[(int64_t)j * width];
    out[i] = (T)sum;
  }
}

// One token: S' = e^a S + k v^T, o = scale S'^T q. One block a head of a row; the state is read and
// written once. Thread: VW neighbouring columns, every (256 / lanes)-th row.
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
  const float decay = raw <= 0.f ? exp2f(fmaxf(raw, kMinLogDecay) * kLog2e) : __builtin_nanf("");
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

template <typename T, int KP, int VP>
hipError_t launch_kv(Args A, int64_t slots, bool split, hipStream_t s) {
  const AttentionPass &P = A.p;
  const auto each = [&](auto kernel) {
    const int64_t per = max_blocks(VP * 4) / P.heads;  // slots a launch
    for (A.slot0 = 0; A.slot0 < slots; A.slot0 += per) {
      const int64_t n = slots - A.slot0 < per ? slots - A.slot0 : per;
      hipLaunchKernelGGL(kernel, dim3((unsigned)(n * P.heads)), dim3(VP * 4), 0, s, A);
    }
  };
  if (split) {
    each(k_attention<T, KP, VP, true>);
    const int64_t floats = (int64_t)KP * VP, per = max_blocks(256) / P.heads;
    for (int64_t r = 0; r < P.n_rows; r += per) {
      const int64_t n = P.n_rows - r < per ? P.n_rows - r : per;
      hipLaunchKernelGGL(k_join_segments, dim3((unsigned)(n * P.heads), (unsigned)(floats / 256)),
                         dim3(256), 0, s, P.segments, P.row_ptr, r, P.n_tokens, slots, A.segment,
                         P.heads, P.log_decay, floats);
    }
  }
  each(k_attention<T, KP, VP, false>);
  return hipGetLastError();
}

template <typename T, int KP>
hipError_t launch_k(const Args &A, int64_t slots, bool split, hipStream_t s) {
  switch (padded_width3(A.p.v_width)) {
    case 32: return launch_kv<T, KP, 32>(A, slots, split, s);
    case 64: return launch_kv<T, KP, 64>(A, slots, split, s);
    default: return launch_kv<T, KP, 128>(A, slots, split, s);
  }
}

template <typename T> hipError_t launch_t(const Args &A, int64_t slots, bool split, hipStream_t s) {
  switch (padded_width3(A.p.k_width)) {
    case 32: return launch_k<T, 32>(A, slots, split, s);
    case 64: return launch_k<T, 64>(A, slots, split, s);
    default: return launch_k<T, 128>(A, slots, split, s);
  }
}

}  // namespace

int64_t attention_segment(int64_t n_tokens, int32_t heads) {
  int64_t L = 512;
  while (L < 4096 && n_tokens / L * heads > 2048) L *= 2;
  return L;
}

int64_t attention_segment_floats(int64_t n_tokens, int64_t n_rows, int32_t heads, int k_width,
                                 int v_width) {
  const int64_t L = attention_segment(n_tokens, heads);
  if (n_tokens <= L) return 0;  // no row is longer than a segment
  return (n_tokens / L + n_rows) * heads * padded_width3(k_width) * padded_width3(v_width);
}

hipError_t launch_attention(als_dtype dtype, const AttentionPass &p, hipStream_t s) {
  if (p.n_rows == 0) return hipSuccess;
  Args A{p, attention_segment(p.n_tokens, p.heads), 0};
  const int size = dtype == ALS_F32 ? 4 : 2, out = p.out_f32 ? 4 : size;
  A.vec = (aligned16(p.q.data, p.q.token_stride, p.q.head_stride, p.k_width, size) ? 1 : 0) |
          (aligned16(p.k.data, p.k.token_stride, p.k.head_stride, p.k_width, size) ? 2 : 0) |
          (aligned16(p.v.data, p.v.token_stride, p.v.head_stride, p.v_width, size) ? 4 : 0) |
          (p.v_width % 4 == 0 && (uintptr_t)p.out % (4 * out) == 0 ? 8 : 0);
  const int64_t slots = p.n_tokens / A.segment + p.n_rows;
  const bool split = p.n_tokens > A.segment;
  return dtype == ALS_F32 ? launch_t<float>(A, slots, split, s) : launch_t<bf16>(A, slots, split, s);
}

hipError_t launch_sum_groups(als_dtype dtype, const float *x, int64_t n_tokens, int32_t heads,
                             int32_t group, int32_t width, void *out, hipStream_t s) {
  const int64_t n = n_tokens * (heads / group) * width;
  if (n == 0) return hipSuccess;
  const dim3 grid((unsigned)((n + 255) / 256 < 8192 ? (n + 255) / 256 : 8192));
  if (dtype == ALS_F32)
    hipLaunchKernelGGL(k_sum_groups<float>, grid, dim3(256), 0, s, x, n, group, width, (float *)out);
  else
    hipLaunchKernelGGL(k_sum_groups<bf16>, grid, dim3(256), 0, s, x, n, group, width, (bf16 *)out);
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
