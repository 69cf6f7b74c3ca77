// Prints what csrc/mm_plan.h plans.  stdin, a line each:
//   i8 m n k                            -> kind slices
//   ortho batch rows cols split         -> kind slices of the Gram product, kind of the polynomial, kind of the step,
//                                          grouped
#include <cstdio>
#include <cstring>

#include "mm_plan.h"

int main() {
  char what[8];
  long long a, b, c;
  while (std::scanf("%7s %lld %lld %lld", what, &a, &b, &c) == 4) {
    if (!std::strcmp(what, "i8")) {
      const dfp::I8Plan p = dfp::plan_gemm_i8(a, b, c);
      std::printf("%d %d\n", p.kind, p.slices);
    } else {
      int split;
      if (std::scanf("%d", &split) != 1) return 1;
      const dfp::OrthoPlan p = dfp::plan_ortho(a, b, c, split != 0);
      std::printf("%d %d %d %d %d\n", p.gram.kind, p.gram.slices, p.poly.kind, p.step.kind, (int)p.grouped);
    }
  }
}
