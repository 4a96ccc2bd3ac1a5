// Steps of the fragments that heads of rows of 4 bits are cut into, for test_fragment_math.py.
#include "common.h"
#include "fragments.h"

extern "C" int fragment_steps(const int *steps, int heads, int rows, int units, int apart) {
  int total = 0, longest = 0;
  for (int h = 0; h < heads; ++h) {
    total += steps[h];
    longest = steps[h] > longest ? steps[h] : longest;
  }
  return cmp::bits4_fragment_rule(total, longest, heads, rows, cmp::bits4_fragment_target(heads, longest, rows, units, apart != 0), apart != 0).per;
}
