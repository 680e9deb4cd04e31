// Host-side exercise of the index rules that the kernels over a cache of keys share (csrc/attention.h), for a build of host code alone.
#include <stdio.h>

#include "attention.h"

using namespace moespec;

static int failures = 0;

#define EXPECT(cond)                                                           \
  do {                                                                         \
    if (!(cond)) {                                                             \
      fprintf(stderr, "%s:%d: check failed: %s\n", __FILE__, __LINE__, #cond); \
      ++failures;                                                              \
    }                                                                          \
  } while (0)

// n keys lie in stages of `stage` places.  The last key has a value that is not finite, so the places behind it, which repeat it, are
// marked as it is: the keys whose values are read from memory again are keys, all those that are marked, whatever else is marked.
static void marked_keys(int n, int stage) {
  for (int base0 = 0; base0 < n; base0 += stage)
    for (int base = base0; base < base0 + stage; base += 32) {
      uint32_t marked = 0;
      for (int j = 0; j < 32; ++j)
        if (base + j >= n - 1 || (base + j) % 7 == 3) marked |= 1u << j;
      for (const uint32_t bits : {marked, marked | 0xffff0000u, ~0u}) {
        const uint32_t there = keys_there(bits, n - base);
        for (int j = 0; j < 32; ++j) EXPECT(((there >> j) & 1u) == (base + j < n ? (bits >> j) & 1u : 0u));
      }
    }
}

int main() {
  for (int n = 1; n <= 300; ++n)
    for (const int stage : {32, 64, 128}) marked_keys(n, stage);
  if (failures) {
    fprintf(stderr, "%d host checks failed\n", failures);
    return 1;
  }
  printf("host checks passed\n");
  return 0;
}
