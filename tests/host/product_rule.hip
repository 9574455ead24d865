// The rules of the 8-bit product (radial_product_rule.h) on the host.  Input lines:
//   form M N groups    -> index, rows, columns, parts of the tiles chosen; rows of M in them, index of the form of the rest
//   small M N          -> 1 where pieces of 16 x 16 are taken
//   tiles TM TN        -> "m n" of every workgroup
//   pieces B           -> byte offset of piece p of row r, r below 256, p below 8, of operand A (0) or B (1), and whether 16 lanes that read one piece meet 16 banks
#include <stdio.h>
#include <string.h>

#include "radial_product_rule.h"

using namespace radial;

template <bool kB>
void pieces() {
  for (int r = 0; r < 256; ++r)
    for (int p = 0; p < 8; ++p) printf("%d ", code_piece<kB>(r, p));
  printf("\n");
  // a wave's read of fragment t: lane l takes piece (l >> 4) + 4 h of the row of l & 15; 16 lanes at a time
  const int first[] = {0, 1, 2, 3, 12, 13, 14, 15, 20, 21, 22, 23, 24, 25, 26, 27}, second[] = {4, 5, 6, 7, 8, 9, 10, 11, 16, 17, 18, 19, 28, 29, 30, 31};
  int meets = 0;
  for (int t = 0; t < 4; ++t)
    for (int h = 0; h < 2; ++h)
      for (int half = 0; half < 2; ++half)
        for (const int* lanes : {first, second}) {
          uint32_t banks = 0;
          for (int i = 0; i < 16; ++i) {
            const int lane = lanes[i] + 32 * half, l16 = lane & 15;
            const int row = kB ? (l16 >> 2) * 16 + t * 4 + (l16 & 3) : t * 16 + l16;
            banks |= 1u << (code_piece<kB>(row, (lane >> 4) + 4 * h) >> 4 & 15);
          }
          meets += banks != 0xffffu;
        }
  printf("%d\n", meets);
}

int main() {
  char what[16];
  int a, b, c;
  while (scanf("%15s", what) == 1) {
    if (!strcmp(what, "form") && scanf("%d %d %d", &a, &b, &c) == 3) {
      const ProductPlan plan = plan_product(a, b, c);
      const TileForm& f = kTileForms[plan.form];
      printf("%d %d %d %d %d %d\n", plan.form, f.rows, f.columns, f.split, plan.rows, plan.rest);
    } else if (!strcmp(what, "small") && scanf("%d %d", &a, &b) == 2) {
      printf("%d\n", takes_pieces(a, b));
    } else if (!strcmp(what, "tiles") && scanf("%d %d", &a, &b) == 2) {
      for (uint32_t id = 0; id < (uint32_t)a * b; ++id) {
        int32_t m, n;
        tile_of(id, a, b, m, n);
        printf("%d %d ", m, n);
      }
      printf("\n");
    } else if (!strcmp(what, "pieces") && scanf("%d", &a) == 1) {
      a ? pieces<true>() : pieces<false>();
    } else {
      return 1;
    }
  }
  return 0;
}
