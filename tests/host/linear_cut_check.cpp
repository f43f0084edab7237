// Prints how products are cut: lines of rows, columns, length of the sum, bytes of an element and whether both operands' rows run along
// the sum come in; tile, parts and their length go out.
#include <cstdio>

#include "../../paper_2503_04424_amd/csrc/linear_cut.h"

int main() {
  long long rows, cols, k, size, inner;
  while (std::scanf("%lld %lld %lld %lld %lld", &rows, &cols, &k, &size, &inner) == 5) {
    const mdet::Cut c = mdet::cut_of(rows, cols, k, size, inner != 0);
    std::printf("%d %d %lld\n", c.tile, c.splits, (long long)c.kpart);
  }
}
