// Norm of queries and keys for each head, with the rotation by position in the same pass:
//   r = 1 / sqrt(mean x^2 + eps),  y = x r w,
// and the first R features of y in pairs (a, b), turned by the angle of the token's position:
//   a' = a cos - b sin,  b' = b cos + a sin.
// Backward, with g = dy turned back: dw = sum g x r,
//   dx = r (g w - n mean(g w n)),  n = x r
// (formed from n, of unit size at any scale of x: r^3 alone leaves fp32's range from about 1e13 and 1e-13 on).
//
// Every byte is read and written once; the arithmetic is small, so memory bounds it. A group of G
// lanes shares a row (one head of one token), and a lane holds whole pairs: VW values of each half
// (or two runs of VW neighbours), so that the rotation needs no exchange and the norm one sum over the group.
// Sums and products run in fp32, rounded once on the way out. The weights' gradient is summed per
// lane over the rows that it meets, then per block, then over the blocks in fp64, always in one
// order.
#include "internal.h"
#include "sequence.h"

namespace als {

namespace {

constexpr int kBlock = 256;

struct Side {
  als_heads x, dy, out;  // forward: x -> out; backward: x, dy -> out
  const float *weight;
  float *partial;        // backward: [blocks, width] sums of the weight's gradient
  float *dweight;
  int32_t heads;
};

struct Rotate {
  Side side[2];
  int64_t n_tokens, n_positions;
  const float *cos, *sin;
  const int32_t *positions;
  int32_t width, half;
  int64_t tokens_per_block;
  float eps;
};

// VW values in one access at any alignment of their type.
template <typename T, int VW> struct Run {
  using V = T __attribute__((ext_vector_type(VW)));
  using U = V __attribute__((aligned(sizeof(T))));
};
// VW values from p, zero past `left` of them. Without CUT there are VW or none.
template <typename T, int VW, bool CUT>
__device__ __forceinline__ void load(const T *p, int left, float (&x)[VW]) {
  if (left >= VW) {
    const typename Run<T, VW>::V v = *(const typename Run<T, VW>::U *)p;
#pragma unroll
    for (int e = 0; e < VW; ++e) x[e] = (float)v[e];
  } else {
#pragma unroll
    for (int e = 0; e < VW; ++e) x[e] = CUT && e < VW - 1 && e < left ? (float)p[e] : 0.f;
  }
}
template <typename T, int VW, bool CUT>
__device__ __forceinline__ void store(T *p, int left, const float (&x)[VW]) {
  if (left >= VW) {
    typename Run<T, VW>::V v;
#pragma unroll
    for (int e = 0; e < VW; ++e) v[e] = (T)x[e];
    *(typename Run<T, VW>::U *)p = v;
  } else if (CUT) {
#pragma unroll
    for (int e = 0; e < VW - 1; ++e)
      if (e < left) p[e] = (T)x[e];
  }
}

// How a row's runs of VW values meet its end, and a half's:
enum Ends {
  kWhole,   // they end with it
  kOver,    // the last one starts early, over values of the run before it, which both lanes form and
            // write alike; `skip` of them count in the other lane's sums alone
  kCut,     // the last one is short and goes value by value: rows and halves shorter than a run
};

// Where a lane's unit lies in a row: two runs of VW values. Of a lane group, runs a lie side by side,
// and so do runs b, so that each load and store of the group is one piece of memory. Turned pairs lie
// across the two runs (halves) or within each run (neighbours).
struct Unit {
  int a, b;            // first features of the runs
  int left_a, left_b;  // values there, at most VW count
  int skip_a, skip_b;
  bool turned;
};
template <int VW, bool NEXT, Ends ENDS, int G>
__device__ __forceinline__ Unit unit_of(int lane, int width, int half) {
  Unit x;
  x.skip_a = x.skip_b = 0;
  const auto run = [&](int from, int end, int &at, int &left, int &skip) {
    at = from;
    left = end - from;
    if (ENDS == kOver && left > 0 && left < VW) {
      skip = VW - left;
      at = end - VW;
      left = VW;
    }
  };
  const int pairs = (half + VW - 1) / VW;
  x.turned = NEXT || lane < pairs;
  if (NEXT) {
    run(lane * VW, width, x.a, x.left_a, x.skip_a);
    run(lane * VW + G * VW, width, x.b, x.left_b, x.skip_b);
  } else if (x.turned) {
    run(lane * VW, half, x.a, x.left_a, x.skip_a);
    x.b = half + x.a;
    x.left_b = x.left_a;
    x.skip_b = x.skip_a;
  } else {
    const int from = 2 * half + (lane - pairs) * 2 * VW;
    run(from, width, x.a, x.left_a, x.skip_a);
    run(from + VW, width, x.b, x.left_b, x.skip_b);
  }
  return x;
}
template <int VW, bool NEXT> inline int units_in(int width, int half) {
  return NEXT ? (width + 2 * VW - 1) / (2 * VW)
              : (half + VW - 1) / VW + (width - 2 * half + 2 * VW - 1) / (2 * VW);
}

// N angles from pair p of a table of `half`, of which those past its end turn nothing.
template <int N> struct Angles {
  float c[N], s[N];
  __device__ __forceinline__ Angles(const float *cs, const float *sn, int p, int half) {
    if (p + N <= half) {
      __builtin_memcpy(c, cs + p, sizeof c);
      __builtin_memcpy(s, sn + p, sizeof s);
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e) {
        c[e] = p + e < half ? cs[p + e] : 1.f;
        s[e] = p + e < half ? sn[p + e] : 0.f;
      }
    }
  }
  template <int SIGN> __device__ __forceinline__ void turn(int e, float &x, float &y) const {
    const float was = x;
    x = was * c[e] - y * (SIGN * s[e]);
    y = y * c[e] + was * (SIGN * s[e]);
  }
};
// Turns a unit's pairs by the angles of cs and sn, or back with SIGN -1.
template <int VW, bool NEXT, int SIGN>
__device__ __forceinline__ void turn(const Unit &u, float (&a)[VW], float (&b)[VW], const float *cs,
                                     const float *sn, int half) {
  if constexpr (NEXT) {
    const Angles<VW / 2> x(cs, sn, u.a / 2, half), y(cs, sn, u.b / 2, half);
#pragma unroll
    for (int e = 0; e < VW / 2; ++e) {
      x.template turn<SIGN>(e, a[2 * e], a[2 * e + 1]);
      y.template turn<SIGN>(e, b[2 * e], b[2 * e + 1]);
    }
  } else if (u.turned) {
    const Angles<VW> x(cs, sn, u.a, half);
#pragma unroll
    for (int e = 0; e < VW; ++e) x.template turn<SIGN>(e, a[e], b[e]);
  }
}

template <int G> __device__ __forceinline__ float group_sum(float x) {
#pragma unroll
  for (int o = G / 2; o > 0; o >>= 1) x += __shfl_xor(x, o);
  return x;
}

// blockIdx.y: queries or keys; blockIdx.x: a run of tokens. G lanes a row, a unit a lane. Measured: 8 and
// 2 heads of 128 in bf16, 1 000 990 tokens, neighbours: 1053 us forward, 1633 us backward, 4.9 and 4.7
// TB/s of the bytes it has to move; 4 and 4 heads of 100 in f32, 200 003 tokens: 277 and 391 us, 4.6 and
// 4.9 TB/s (a large copy reaches 4.8); 64 tokens: 4.8 us, a launch.
template <typename T, int VW, bool NEXT, Ends ENDS, int G, bool BACK>
__global__ __launch_bounds__(kBlock) void k_rotate(Rotate R) {
  const Side &S = R.side[blockIdx.y];
  const int tid = (int)threadIdx.x, lane = tid % G;
  const int64_t t0 = (int64_t)blockIdx.x * R.tokens_per_block;
  const int64_t t1 = t0 + R.tokens_per_block < R.n_tokens ? t0 + R.tokens_per_block : R.n_tokens;
  const int rows = (int)(t1 > t0 ? t1 - t0 : 0) * S.heads;
  const Unit u = unit_of<VW, NEXT, ENDS, G>(lane, R.width, R.half);
  float wa[VW], wb[VW], ga[VW], gb[VW];
#pragma unroll
  for (int e = 0; e < VW; ++e) {
    wa[e] = e < u.left_a ? S.weight[u.a + e] : 0.f;
    wb[e] = e < u.left_b ? S.weight[u.b + e] : 0.f;
    ga[e] = gb[e] = 0.f;
  }
  constexpr int kStep = kBlock / G;
  const int token_step = kStep / S.heads, head_step = kStep % S.heads;
  int head = tid / G % S.heads;
  int64_t token = t0 + tid / G / S.heads;
  for (int row = tid / G; row < rows; row += kStep) {
    const T *x = (const T *)S.x.data + token * S.x.token_stride + head * S.x.head_stride;
    T *out = (T *)S.out.data + token * S.out.token_stride + head * S.out.head_stride;
    const T *dy = BACK ? (const T *)S.dy.data + token * S.dy.token_stride + head * S.dy.head_stride
                       : nullptr;
    const int64_t at = R.positions[token];
    const bool ok = at >= 0 && at < R.n_positions;
    const float *cs = R.cos + (ok ? at : 0) * R.half, *sn = R.sin + (ok ? at : 0) * R.half;
    float xa[VW], xb[VW], da[VW], db[VW];
    load<T, VW, ENDS == kCut>(x + u.a, u.left_a, xa);
    load<T, VW, ENDS == kCut>(x + u.b, u.left_b, xb);
    if (BACK) {
      load<T, VW, ENDS == kCut>(dy + u.a, u.left_a, da);
      load<T, VW, ENDS == kCut>(dy + u.b, u.left_b, db);
    }
    float squares = 0.f, along = 0.f;
#pragma unroll
    for (int e = 0; e < VW; ++e) {
      if (e >= u.skip_a) squares = fmaf(xa[e], xa[e], squares);
      if (e >= u.skip_b) squares = fmaf(xb[e], xb[e], squares);
    }
    squares = group_sum<G>(squares);
    // a position outside the tables makes its rows NaN
    const float r = ok ? 1.f / sqrtf(squares / (float)R.width + R.eps) : __builtin_nanf("");
    if (!BACK) {
#pragma unroll
      for (int e = 0; e < VW; ++e) {
        xa[e] *= r * wa[e];
        xb[e] *= r * wb[e];
      }
      turn<VW, NEXT, 1>(u, xa, xb, cs, sn, R.half);
    } else {
      turn<VW, NEXT, -1>(u, da, db, cs, sn, R.half);
#pragma unroll
      for (int e = 0; e < VW; ++e) {
        xa[e] *= r;
        xb[e] *= r;
        ga[e] = fmaf(da[e], xa[e], ga[e]);
        gb[e] = fmaf(db[e], xb[e], gb[e]);
        da[e] *= wa[e];
        db[e] *= wb[e];
        if (e >= u.skip_a) along = fmaf(da[e], xa[e], along);
        if (e >= u.skip_b) along = fmaf(db[e], xb[e], along);
      }
      along = group_sum<G>(along);
      const float mean = along / (float)R.width;
#pragma unroll
      for (int e = 0; e < VW; ++e) {
        xa[e] = r * (da[e] - xa[e] * mean);
        xb[e] = r * (db[e] - xb[e] * mean);
      }
    }
    store<T, VW, ENDS == kCut>(out + u.a, u.left_a, xa);
    store<T, VW, ENDS == kCut>(out + u.b, u.left_b, xb);
    token += token_step;
    head += head_step;
    if (head >= S.heads) {
      head -= S.heads;
      ++token;
    }
  }
  if (BACK) {
    __shared__ float sums[kBlock / G][G * 2 * VW];
#pragma unroll
    for (int e = 0; e < VW; ++e) {
      sums[tid / G][lane * 2 * VW + e] = ga[e];
      sums[tid / G][lane * 2 * VW + VW + e] = gb[e];
    }
    __syncthreads();
    for (int i = tid; i < G * 2 * VW; i += kBlock) {
      const Unit v = unit_of<VW, NEXT, ENDS, G>(i / (2 * VW), R.width, R.half);
      const int run = i / VW % 2, e = i % VW;
      if (e >= (run ? v.left_b : v.left_a) || e < (run ? v.skip_b : v.skip_a)) continue;
      float sum = 0.f;
      for (int j = 0; j < kBlock / G; ++j) sum += sums[j][i];
      S.partial[(int64_t)blockIdx.x * R.width + (run ? v.b : v.a) + e] = sum;
    }
  }
}

// One feature a block: the blocks' sums in fp64, in order within each thread and then over them. 22 us
// for 8192 blocks' sums of 128 features: strided reads of what the caches still hold. (16 features a
// block, so that reads are whole lines, leave too few blocks: 61 us.)
__global__ __launch_bounds__(256) void k_sum_partials(Rotate R, int blocks) {
  const Side &S = R.side[blockIdx.y];
  __shared__ double sums[256];
  double x = 0.0;
  for (int i = threadIdx.x; i < blocks; i += 256) x += (double)S.partial[(int64_t)i * R.width + blockIdx.x];
  sums[threadIdx.x] = x;
  __syncthreads();
  for (int o = 128; o > 0; o >>= 1) {
    if ((int)threadIdx.x < o) sums[threadIdx.x] += sums[threadIdx.x + o];
    __syncthreads();
  }
  if (threadIdx.x == 0) S.dweight[blockIdx.x] = (float)sums[0];
}

template <typename T, int VW, bool NEXT, Ends ENDS, bool BACK>
hipError_t launch_vw(const Rotate &R, int blocks, hipStream_t s) {
  const int units = units_in<VW, NEXT>(R.width, R.half);
  const dim3 grid((unsigned)blocks, 2);
#define ROTATE(G) hipLaunchKernelGGL((k_rotate<T, VW, NEXT, ENDS, G, BACK>), grid, dim3(kBlock), 0, s, R)
  if (units <= 4) ROTATE(4);
  else if (units <= 8) ROTATE(8);
  else if (units <= 16) ROTATE(16);
  else if (units <= 32) ROTATE(32);
  else ROTATE(64);
#undef ROTATE
  if (BACK)
    hipLaunchKernelGGL(k_sum_partials, dim3((unsigned)R.width, 2), dim3(256), 0, s, R, blocks);
  return hipGetLastError();
}

// Whether every run is whole and aligned at 16 bytes.
bool whole_runs(const Rotate &R, bool next, bool back, int size) {
  const int vw = 16 / size;
  bool fits = R.width % vw == 0 && (next || R.half % vw == 0);
  for (const Side &S : R.side)
    for (const als_heads *x : {&S.x, &S.out, back ? &S.dy : &S.x})
      fits = fits && (uintptr_t)x->data % 16 == 0 && x->token_stride % vw == 0 && x->head_stride % vw == 0;
  return fits;
}
// Whether the last run of the row and of each half can start early.
bool over_runs(const Rotate &R, bool next, int vw) {
  const int rest = R.width - 2 * R.half;
  return next ? R.width >= vw && R.width % 2 == 0
              : (R.half == 0 || R.half >= vw) && (rest == 0 || rest >= vw);
}

template <typename T, bool NEXT, bool BACK>
hipError_t launch_next(const Rotate &R, int blocks, hipStream_t s) {
  constexpr int VW = 16 / sizeof(T);
  if (whole_runs(R, NEXT, BACK, sizeof(T))) return launch_vw<T, VW, NEXT, kWhole, BACK>(R, blocks, s);
  if (over_runs(R, NEXT, VW)) return launch_vw<T, VW, NEXT, kOver, BACK>(R, blocks, s);
  // cut runs of eight would take seven loads each
  return launch_vw<T, 4, NEXT, kCut, BACK>(R, blocks, s);
}

}  // namespace

// Eight tokens a block, up to 8192 blocks; forward and backward in us with at most 2048, 4096 and 8192
// blocks: 200 003 tokens of 8 heads of 100 in f32 702, 691, 676; 1 000 990 of 10 of 128 in bf16 2800,
// 2679, 2676; 400 000 of 16 of 64 in bf16 916, 919, 941.
int64_t rotate_blocks(int64_t n_tokens) {
  const int64_t n = (n_tokens + 7) / 8;
  return n < 8192 ? (n > 0 ? n : 1) : 8192;
}

hipError_t launch_rotate(als_dtype dtype, bool back, const als_rotation &shape, const als_heads *x,
                         const als_heads *dy, const als_heads *out, const float *const *weight,
                         float *const *dweight, float *partial, hipStream_t s) {
  Rotate R{};
  const int64_t blocks = rotate_blocks(shape.n_tokens);
  for (int i = 0; i < 2; ++i) {
    R.side[i].x = x[i];
    R.side[i].out = out[i];
    if (back) R.side[i].dy = dy[i];
    R.side[i].weight = weight[i];
    R.side[i].heads = i ? shape.k_heads : shape.q_heads;
    R.side[i].partial = partial + i * blocks * shape.width;
    R.side[i].dweight = back ? dweight[i] : nullptr;
  }
  R.n_tokens = shape.n_tokens;
  R.n_positions = shape.n_positions;
  R.cos = shape.cos_table;
  R.sin = shape.sin_table;
  R.positions = shape.positions;
  R.width = shape.width;
  R.half = shape.rotated / 2;
  R.tokens_per_block = (shape.n_tokens + blocks - 1) / blocks;
  R.eps = shape.eps;
  const auto launch = dtype == ALS_F32
      ? (shape.neighbours ? (back ? launch_next<float, true, true> : launch_next<float, true, false>)
                          : (back ? launch_next<float, false, true> : launch_next<float, false, false>))
      : (shape.neighbours ? (back ? launch_next<bf16, true, true> : launch_next<bf16, true, false>)
                          : (back ? launch_next<bf16, false, true> : launch_next<bf16, false, false>));
  return launch(R, (int)blocks, s);
}

}  // namespace als
