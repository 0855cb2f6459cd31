// Prints, for each line "n N ldq K lead" of its input, the kernel that the 8-bit
// product uses and whether rows of q are ragged.
#include <stdio.h>

#include "qlinear_plan.h"

int main() {
  int n, m, k, lead;
  long long ldq;
  while (scanf("%d %d %lld %d %d", &n, &m, &ldq, &k, &lead) == 5)
    printf("%d %d\n", (int)bmlp::qlinear_kernel(n, m, ldq), (int)bmlp::qlinear_ragged((uintptr_t)lead, n, ldq, k));
  return 0;
}
