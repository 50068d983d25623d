// Reads "m n steps" lines and prints what a product of 8-bit rows with 4-bit rows chooses:
// the form, and for few rows whether groups are shared out and a is held in LDS.
#include <cstdio>

#include "mx4_choice.h"

int main() {
  long long m, n;
  int steps;
  while (std::scanf("%lld %lld %d", &m, &n, &steps) == 3)
    std::printf("%d %d %d\n", int(rslm::score8_form(m, n, steps)), int(rslm::few8_split(n, steps)),
                int(rslm::few8_held(m, steps)));
  return 0;
}
