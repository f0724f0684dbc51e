// Zeros at the tokens that no row holds: those before the first row and behind the last. The decayed attention works
// on rows and leaves such places as they are; where its results go on into sums over all tokens (the gradient of a
// projection), they have to count as nothing.
//
// Bound by the launch where there are no such tokens: each block reads the two ends of the rows.
#include "internal.h"
#include "sequence.h"

namespace als {

namespace {

using u32x4 = uint32_t __attribute__((ext_vector_type(4)));

// bytes [from, to) of p, by all threads of the grid: 16 at a time, and the ends one by one
__device__ __forceinline__ void clear(char *p, int64_t from, int64_t to, int64_t thread, int64_t threads) {
  if (from >= to) return;
  char *const first = p + from, *const last = p + to;
  char *lo = first + (16 - (uintptr_t)first % 16) % 16, *hi = last - (uintptr_t)last % 16;
  if (lo >= hi) lo = hi = last;  // no whole piece
  for (int64_t n = thread; n < (lo - first) + (last - hi); n += threads)
    (n < lo - first ? first[n] : hi[n - (lo - first)]) = 0;
  for (int64_t n = thread; n < (hi - lo) / 16; n += threads) ((u32x4 *)lo)[n] = u32x4{0, 0, 0, 0};
}

__global__ __launch_bounds__(256) void k_clear_unheld(int64_t n_tokens, int64_t n_rows,
                                                      const int64_t *__restrict__ row_ptr, Unheld u) {
  const auto within = [&](int64_t x, int64_t lo) { return x < lo ? lo : x > n_tokens ? n_tokens : x; };
  const int64_t first = within(row_ptr[0], 0), end = within(row_ptr[n_rows], first);
  const int64_t thread = (int64_t)blockIdx.x * 256 + threadIdx.x, threads = (int64_t)gridDim.x * 256;
  for (int i = 0; i < u.n; ++i) {
    clear(u.data[i], 0, first * u.token_bytes[i], thread, threads);
    clear(u.data[i], end * u.token_bytes[i], n_tokens * u.token_bytes[i], thread, threads);
  }
}

}  // namespace

hipError_t launch_clear_unheld(int64_t n_tokens, int64_t n_rows, const int64_t *row_ptr, const Unheld &u,
                               hipStream_t s) {
  int64_t bytes = 0;
  for (int i = 0; i < u.n; ++i) bytes += n_tokens * u.token_bytes[i];
  if (bytes == 0) return hipSuccess;
  const int64_t blocks = (bytes + 65535) / 65536;
  hipLaunchKernelGGL(k_clear_unheld, dim3((unsigned)(blocks < 1024 ? blocks : 1024)), dim3(256), 0, s, n_tokens,
                     n_rows, row_ptr, u);
  return hipGetLastError();
}

}  // namespace als
