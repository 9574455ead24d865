// The rules of the 8-bit integer product (radial_product_i8_rule.h) on the host.  Input lines:
//   form M N groups    -> index, rows, columns, parts of the tiles chosen; rows of M in them, index of the form of the rest
//   small M N          -> 1 where pieces of 16 x 16 are taken
//   tiles TM TN        -> "m n" of every workgroup
#include <stdio.h>
#include <string.h>

#include "radial_product_i8_rule.h"

using namespace radial;

int main() {
  char what[16];
  int a, b, c;
  while (scanf("%15s", what) == 1) {
    if (!strcmp(what, "form") && scanf("%d %d %d", &a, &b, &c) == 3) {
      const ProductPlan plan = plan_product_i8(a, b, c);
      const TileForm& f = kTileFormsI8[plan.form];
      printf("%d %d %d %d %d %d\n", plan.form, f.rows, f.columns, f.split, plan.rows, plan.rest);
    } else if (!strcmp(what, "small") && scanf("%d %d", &a, &b) == 2) {
      printf("%d\n", takes_pieces_i8(a, b));
    } else if (!strcmp(what, "tiles") && scanf("%d %d", &a, &b) == 2) {
      for (uint32_t id = 0; id < (uint32_t)a * b; ++id) {
        int32_t m, n;
        tile_of<kBandI8>(id, a, b, m, n);
        printf("%d %d ", m, n);
      }
      printf("\n");
    } else {
      return 1;
    }
  }
  return 0;
}
