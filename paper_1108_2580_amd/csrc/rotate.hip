// Norm of queries and keys for each head, with the rotation by position in the same pass:
//   r = 1 / sqrt(mean x^2 + eps),  y = x r w,
// and the first R features of y in pairs (a, b), turned by the angle of the token's position:
//   a' = a cos - b sin,  b' = b cos + a sin.
// Backward, with g = dy turned back: dw = sum g x r,
//   dx = r g w - x r^3 mean(g w x).
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

template <typename T, int N> struct alignas(sizeof(T) * N) Pack { T v[N]; };

// VW values from p, zero past `left` of them; whole where VW of them are left.
template <typename T, int VW>
__device__ __forceinline__ void load(const T *p, int left, float *x) {
  Pack<T, VW> v;
  if (left >= VW) {
    v = *(const Pack<T, VW> *)p;
#pragma unroll
    for (int e = 0; e < VW; ++e) x[e] = (float)v.v[e];
  } else {
#pragma unroll
    for (int e = 0; e < VW; ++e) x[e] = e < left ? (float)p[e] : 0.f;
  }
}
template <typename T, int VW>
__device__ __forceinline__ void store(T *p, int left, const float *x) {
  if (left >= VW) {
    Pack<T, VW> v;
#pragma unroll
    for (int e = 0; e < VW; ++e) v.v[e] = (T)x[e];
    *(Pack<T, VW> *)p = v;
  } else {
#pragma unroll
    for (int e = 0; e < VW; ++e)
      if (e < left) p[e] = (T)x[e];
  }
}

// Where unit n of a lane lies in a row: two runs of VW values. A lane group's runs lie side by side, so
// that each load and store of the group is one piece of memory. Turned pairs lie across the two runs
// (halves, and neighbours one by one), or within each run (neighbours otherwise).
struct Unit {
  int a, b;            // first features of the runs
  int left_a, left_b;  // values there, at most VW count
  bool turned_a, turned_b;
};
template <int VW, bool NEXT, int G>
__device__ __forceinline__ Unit unit_of(int lane, int n, int width, int half) {
  Unit x;
  if (NEXT && VW > 1) {
    x.a = (2 * n * G + lane) * VW;
    x.b = x.a + G * VW;
    x.turned_a = x.a < 2 * half;
    x.turned_b = x.b < 2 * half;
  } else {
    const int u = n * G + lane, pairs = half / VW;
    x.turned_a = x.turned_b = u < pairs;
    if (u < pairs) {
      x.a = NEXT ? 2 * u : u * VW;
      x.b = NEXT ? 2 * u + 1 : half + u * VW;
    } else {
      x.a = 2 * half + (u - pairs) * 2 * VW;
      x.b = x.a + VW;
    }
  }
  x.left_a = width - x.a;
  x.left_b = width - x.b;
  return x;
}
// Units in a row, for halves and for neighbours.
template <int VW, bool NEXT> __host__ __device__ inline int units_in(int width, int half) {
  return NEXT && VW > 1 ? (width + 2 * VW - 1) / (2 * VW)
                        : half / VW + (width - 2 * half + 2 * VW - 1) / (2 * VW);
}

// Turns a unit's pairs by the angles of cs and sn, or back with SIGN -1.
template <int VW, bool NEXT, int SIGN>
__device__ __forceinline__ void turn(const Unit &u, float *a, float *b, const float *cs, const float *sn) {
  const auto pair = [&](float &x, float &y, int p) {
    const float c = cs[p], s = SIGN * sn[p], was = x;
    x = was * c - y * s;
    y = y * c + was * s;
  };
  if constexpr (NEXT && VW > 1) {
    if (u.turned_a) {
#pragma unroll
      for (int e = 0; e < VW; e += 2) pair(a[e], a[e + 1], (u.a + e) / 2);
    }
    if (u.turned_b) {
#pragma unroll
      for (int e = 0; e < VW; e += 2) pair(b[e], b[e + 1], (u.b + e) / 2);
    }
  } else if (u.turned_a) {
#pragma unroll
    for (int e = 0; e < VW; ++e) pair(a[e], b[e], (NEXT ? u.a / 2 : u.a) + e);
  }
}

template <int G> __device__ __forceinline__ float group_sum(float x) {
#pragma unroll
  for (int o = G / 2; o > 0; o >>= 1) x += __shfl_xor(x, o);
  return x;
}

// blockIdx.y: queries or keys; blockIdx.x: a run of tokens. G lanes a row, UN units a lane.
template <typename T, int VW, bool NEXT, int G, int UN, bool BACK>
__global__ __launch_bounds__(kBlock) void k_rotate(Rotate R) {
  const Side &S = R.side[blockIdx.y];
  const int tid = (int)threadIdx.x, lane = tid % G;
  const int64_t t0 = (int64_t)blockIdx.x * R.tokens_per_block;
  const int64_t t1 = t0 + R.tokens_per_block < R.n_tokens ? t0 + R.tokens_per_block : R.n_tokens;
  const int rows = (int)(t1 > t0 ? t1 - t0 : 0) * S.heads;
  float wa[UN][VW], wb[UN][VW], ga[UN][VW], gb[UN][VW];
#pragma unroll
  for (int n = 0; n < UN; ++n) {
    const Unit u = unit_of<VW, NEXT, G>(lane, n, R.width, R.half);
#pragma unroll
    for (int e = 0; e < VW; ++e) {
      wa[n][e] = e < u.left_a ? S.weight[u.a + e] : 0.f;
      wb[n][e] = e < u.left_b ? S.weight[u.b + e] : 0.f;
      ga[n][e] = gb[n][e] = 0.f;
    }
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
    float xa[UN][VW], xb[UN][VW], da[UN][VW], db[UN][VW];
    float squares = 0.f, along = 0.f;
#pragma unroll
    for (int n = 0; n < UN; ++n) {
      const Unit u = unit_of<VW, NEXT, G>(lane, n, R.width, R.half);
      load<T, VW>(x + u.a, u.left_a, xa[n]);
      load<T, VW>(x + u.b, u.left_b, xb[n]);
      if (BACK) {
        load<T, VW>(dy + u.a, u.left_a, da[n]);
        load<T, VW>(dy + u.b, u.left_b, db[n]);
      }
#pragma unroll
      for (int e = 0; e < VW; ++e) squares = fmaf(xa[n][e], xa[n][e], fmaf(xb[n][e], xb[n][e], squares));
    }
    squares = group_sum<G>(squares);
    // a position outside the tables makes its rows NaN
    const float r = ok ? 1.f / sqrtf(squares / (float)R.width + R.eps) : __builtin_nanf("");
#pragma unroll
    for (int n = 0; n < UN; ++n) {
      const Unit u = unit_of<VW, NEXT, G>(lane, n, R.width, R.half);
      float *a = BACK ? da[n] : xa[n], *b = BACK ? db[n] : xb[n];
      if (!BACK) {
#pragma unroll
        for (int e = 0; e < VW; ++e) {
          a[e] *= r * wa[n][e];
          b[e] *= r * wb[n][e];
        }
      }
      turn<VW, NEXT, BACK ? -1 : 1>(u, a, b, cs, sn);
      if (BACK) {
#pragma unroll
        for (int e = 0; e < VW; ++e) {
          ga[n][e] = fmaf(a[e], xa[n][e] * r, ga[n][e]);
          gb[n][e] = fmaf(b[e], xb[n][e] * r, gb[n][e]);
          a[e] *= wa[n][e];
          b[e] *= wb[n][e];
          along = fmaf(a[e], xa[n][e], fmaf(b[e], xb[n][e], along));
        }
      }
    }
    if (BACK) {
      along = group_sum<G>(along);
      const float f = r * r * r * (along / (float)R.width);
#pragma unroll
      for (int n = 0; n < UN; ++n)
#pragma unroll
        for (int e = 0; e < VW; ++e) {
          xa[n][e] = da[n][e] * r - xa[n][e] * f;
          xb[n][e] = db[n][e] * r - xb[n][e] * f;
        }
    }
#pragma unroll
    for (int n = 0; n < UN; ++n) {
      const Unit u = unit_of<VW, NEXT, G>(lane, n, R.width, R.half);
      store<T, VW>(out + u.a, u.left_a, xa[n]);
      store<T, VW>(out + u.b, u.left_b, xb[n]);
    }
    token += token_step;
    head += head_step;
    if (head >= S.heads) {
      head -= S.heads;
      ++token;
    }
  }
  if (BACK) {
    __shared__ float sums[kBlock / G][G * UN * 2 * VW];
#pragma unroll
    for (int n = 0; n < UN; ++n)
#pragma unroll
      for (int e = 0; e < VW; ++e) {
        sums[tid / G][((lane + n * G) * 2) * VW + e] = ga[n][e];
        sums[tid / G][((lane + n * G) * 2 + 1) * VW + e] = gb[n][e];
      }
    __syncthreads();
    for (int i = tid; i < G * UN * 2 * VW; i += kBlock) {
      const Unit u = unit_of<VW, NEXT, G>(i / (2 * VW) % G, i / (2 * VW) / G, R.width, R.half);
      const int run = i / VW % 2, d = (run ? u.b : u.a) + i % VW;
      if (d >= R.width) continue;
      float sum = 0.f;
      for (int j = 0; j < kBlock / G; ++j) sum += sums[j][i];
      S.partial[(int64_t)blockIdx.x * R.width + d] = sum;
    }
  }
}

// One feature a block: the blocks' sums in fp64, in order within each thread and then over them.
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

template <typename T, int VW, bool NEXT, bool BACK>
hipError_t launch_vw(const Rotate &R, int blocks, hipStream_t s) {
  const int units = units_in<VW, NEXT>(R.width, R.half);
  const dim3 grid((unsigned)blocks, 2);
#define ROTATE(G, UN) \
  hipLaunchKernelGGL((k_rotate<T, VW, NEXT, G, UN, BACK>), grid, dim3(kBlock), 0, s, R)
  if (units <= 4) ROTATE(4, 1);
  else if (units <= 8) ROTATE(8, 1);
  else if (units <= 16) ROTATE(16, 1);
  else if (units <= 32) ROTATE(32, 1);
  else if (units <= 64) ROTATE(64, 1);
  else ROTATE(64, 2);
#undef ROTATE
  if (BACK)
    hipLaunchKernelGGL(k_sum_partials, dim3((unsigned)R.width, 2), dim3(256), 0, s, R, blocks);
  return hipGetLastError();
}

// Values per load: the widest (16 bytes, two values, one) that every run's alignment allows.
int run_width(const Rotate &R, bool next, bool back, int size) {
  for (int vw : {16 / size, 2, 1}) {
    // halves: the second starts at `half`; neighbours: a run is turned as a whole or not at all
    bool fits = (next ? 2 * R.half : R.half) % vw == 0;
    for (const Side &S : R.side)
      for (const als_heads *x : {&S.x, &S.out, back ? &S.dy : &S.x})
        fits = fits && ((uintptr_t)x->data % (vw * size) == 0) && x->token_stride % vw == 0 &&
               x->head_stride % vw == 0;
    if (fits) return vw;
  }
  return 1;
}

template <typename T, bool NEXT, bool BACK>
hipError_t launch_next(const Rotate &R, int blocks, hipStream_t s) {
  const int vw = run_width(R, NEXT, BACK, sizeof(T));
  if (vw == 1) return launch_vw<T, 1, NEXT, BACK>(R, blocks, s);
  if (vw == 2) return launch_vw<T, 2, NEXT, BACK>(R, blocks, s);
  return launch_vw<T, 16 / sizeof(T), NEXT, BACK>(R, blocks, s);
}

}  // namespace

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
