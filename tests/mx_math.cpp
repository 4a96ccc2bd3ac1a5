// The rule that cuts heads of rows of 4 bits into fragments, for test_mx_math.py.
#include "common.h"
#include "fragments.h"

extern "C" {
int fragments_launched(int heads, int steps, int rows, int units, int apart) {
  return cmp::fragments_most(heads, cmp::bits4_fragment_target(heads, steps, rows, units, apart != 0));
}
int fragments_made(const int *steps, int heads, int promised, int rows, int units, int apart) {
  int total = 0, longest = 0, made = 0;
  for (int h = 0; h < heads; ++h) {
    total += steps[h];
    longest = steps[h] > longest ? steps[h] : longest;
  }
  const cmp::FragmentRule r = cmp::bits4_fragment_rule(total, longest, heads, rows, cmp::bits4_fragment_target(heads, promised, rows, units, apart != 0), apart != 0);
  for (int h = 0; h < heads; ++h) made += cmp::fragments_of(steps[h], r);
  return made;
}
int fragments_of(int steps, int per) { return cmp::fragments_of(steps, cmp::FragmentRule{0, per, 1.f / (float)per}); }
}
