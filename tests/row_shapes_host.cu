// Host program around the rules that give rows their kernels: lines "rows vocab n tail" (n elements in 16 bytes) give the
// loss's kernel with its pieces or warps and CTAs, and the draws' warps, CTAs and whether a row is one round.
#include <cstdio>

#include "mca_row_shapes.h"

int main() {
  static const char* const by[] = {"registers", "shared", "staying", "team"};
  long long rows, vocab;
  int n, tail;
  while (std::scanf("%lld %lld %d %d", &rows, &vocab, &n, &tail) == 4) {
    const mca::DistillShape d = mca::distill_shape(rows, vocab, n, tail != 0);
    const mca::DrawShape s(rows, vocab, n);
    std::printf("%s %d %d %d %d %d\n", by[(int)d.by], d.n, d.split, s.warps, s.split, s.round ? 1 : 0);
  }
  return 0;
}
