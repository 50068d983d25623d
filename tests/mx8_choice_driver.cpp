// Reads "m n steps exact" lines and prints what a product of 8-bit rows with 4-bit rows chooses:
// the form, and for few rows whether groups are shared out and a is held in LDS.
#include <cstdio>

#include "mx4_choice.h"

int main() {
  long long m, n;
  int steps, exact;
  while (std::scanf("%lld %lld %d %d", &m, &n, &steps, &exact) == 4)
    std::printf("%d %d %d\n", int(rslm::score8_form(m, n, steps, exact != 0)), int(rslm::few8_split(n, steps)),
                int(rslm::few8_held(m, steps)));
  return 0;
}
