// Which kernel takes a product of an expert layer (csrc/moe_choice.h, compiled alone), for test_moe_choice.py.  Reads lines
//   "forward|dx n_rows n_experts routed n_j n_r f32 words gated"  or  "dw n_rows n_experts d_in d_z f32 words"
// and prints "few wide fragments parts" of each; or "tiles lo hi rows", and prints their number.
#include <stdio.h>
#include <string.h>

#include "moe_choice.h"

int main() {
  char op[16];
  while (scanf("%15s", op) == 1) {
    long long n_rows;
    int experts, f32, words;
    if (!strcmp(op, "tiles")) {
      int lo, hi, rows;
      if (scanf("%d %d %d", &lo, &hi, &rows) != 3) return 1;
      printf("%d\n", sptir::moe_tiles_of(lo, hi, rows));
    } else if (!strcmp(op, "dw")) {
      int d_in, d_z;
      if (scanf("%lld %d %d %d %d %d", &n_rows, &experts, &d_in, &d_z, &f32, &words) != 6) return 1;
      const int parts = sptir::moe_dw_parts(n_rows, experts, d_in, d_z);
      const bool wide = sptir::moe_dw_wide_pays(n_rows, experts, d_in, d_z, parts, f32 != 0, words != 0);
      printf("0 %d 1 %d\n", wide, wide ? 1 : parts);
    } else {
      int routed, n_j, n_r, gated;
      if (scanf("%lld %d %d %d %d %d %d %d", &n_rows, &experts, &routed, &n_j, &n_r, &f32, &words, &gated) != 8) return 1;
      const sptir::MoeSizes s = {n_rows, experts, routed != 0, n_j, n_r, f32 != 0, words != 0, gated != 0};
      const sptir::MoeChoice c = !strcmp(op, "dx") ? sptir::moe_choose_dx(s) : sptir::moe_choose_forward(s);
      printf("%d %d %d 1\n", c.few, c.wide, c.fragments);
    }
  }
  return 0;
}
