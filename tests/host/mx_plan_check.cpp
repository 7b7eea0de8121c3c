// Which kernel, tile and split the microscaled 4-bit operators take (mx_plan.h), for lines "m n k matrices terms" on
// standard input: "<kernel of the product> <dx's tile> <its splits> <dW's tile> <its splits>".  Built with g++ and the
// address and undefined-behaviour sanitizers by tests/test_mx_plan.py.
#include <stdio.h>

#include "mx_plan.h"

int main() {
  using namespace polyq::mx;
  int m, n, k, mats, terms;
  while (scanf("%d %d %d %d %d", &m, &n, &k, &mats, &terms) == 5) {
    const Choice c = choose(m, n, k, mats);
    const int m_steps = (m + kStep - 1) / kStep, n_steps = (n + kStep - 1) / kStep;
    const Shape dx = grad_shape(false, k, m, 1, mats * n_steps, terms), dw = grad_shape(true, n, k, mats, m_steps, terms);
    printf("%s %d %dx%d %d %dx%d %d\n", c.split ? "split" : "gemm", c.tm, dx.l, dx.s, dx.splits, dw.l, dw.s, dw.splits);
  }
  return 0;
}
