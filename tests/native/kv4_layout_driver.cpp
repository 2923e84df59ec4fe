// Prints csrc/kv4_layout.h: for each head dim, token and dim the key's and the
// value's byte, nibble and scale byte; then the scale bytes of the magnitudes
// given on stdin (fp32 bits).
#include <cstdio>
#define __host__
#define __device__
#define __forceinline__ inline
#include "kv4_layout.h"

int main() {
  using namespace spec;
  for (int hd = 64; hd <= 128; hd += 64)
    for (int t = 0; t < 16; ++t)
      for (int d = 0; d < hd; ++d)
        printf("%d %d %d %d %d %d %d %d %d\n", hd, t, d, kv4_k_unit(t, d / 32, d / 8 % 4, hd) + d % 8 / 2, d % 2,
               kv4_k_scale(t, d / 32, hd), kv4_v_byte(t, d / 32, d % 16), d % 32 / 16, kv4_v_scale(t, d / 32, hd));
  unsigned bits;
  while (scanf("%u", &bits) == 1) printf("%u\n", kv4_scale_of(bits));
  return 0;
}
