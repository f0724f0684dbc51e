/* Stands in for HIP's launch calls and prints every launch: its blocks, then the kernel's first argument as
 * RECORDED_WORDS 64-bit words (no more than the shortest such argument holds). Nothing runs. */
#include <stddef.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

typedef struct {
  uint32_t x, y, z;
} dim3;

static dim3 grid, block;
static size_t shared;
static void *stream;

int __hipPushCallConfiguration(dim3 g, dim3 b, size_t lds, void *s) {
  grid = g;
  block = b;
  shared = lds;
  stream = s;
  return 0;
}

int __hipPopCallConfiguration(dim3 *g, dim3 *b, size_t *lds, void **s) {
  *g = grid;
  *b = block;
  *lds = shared;
  *s = stream;
  return 0;
}

int hipLaunchKernel(const void *f, dim3 g, dim3 b, void **args, size_t lds, void *s) {
  (void)f;
  (void)b;
  (void)lds;
  (void)s;
  printf("%u", g.x);
  const int n = atoi(getenv("RECORDED_WORDS"));
  for (int i = 0; i < n; ++i) {
    uint64_t word = 0;
    memcpy(&word, (const char *)args[0] + 8 * i, 8);
    printf(" %llu", (unsigned long long)word);
  }
  printf("\n");
  fflush(stdout);
  return 0;
}

int hipGetLastError(void) { return 0; }
