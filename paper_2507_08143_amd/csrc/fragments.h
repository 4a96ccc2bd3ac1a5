// How attention to a paged cache cuts heads into fragments: the rule, which every workgroup carries out for itself on the lengths that the device
// finds, and the room that the host makes for what comes out of it.  The two have to agree whatever the device and the lengths are.
#pragma once

#include <algorithm>

#include "common.h"

namespace cmp {

constexpr int ATT_LEAST_LOG = 2;             // fewest steps of a fragment where there are many, log 2
constexpr int SCAN_HEADS = 512, SCAN_ROUNDS = 6;        // heads that a wave looks through, and fragments for every workgroup that
                                             // there is room for on the chip
constexpr int ATT_EVEN = 256, EVEN_PARTS = 4;          // units that have equal parts of heads of one length, and most parts of a head then

// Steps of a fragment: 1 << log, or `per` where that is not 0.
struct FragmentRule { int log, per; };
// total: steps of all heads; rows: query rows of a head; target: fragments that there are to be, beside the last of each head
__host__ __device__ __forceinline__ FragmentRule fragment_rule(int total, int longest, int heads, int rows, int target) {
  // More than 16 query rows make a step dearer and a start too, and more than 32 leave room for one workgroup a unit: fewer steps where all
  // find room at once (16 heads of 500 to 1411, 40 rows: 24 us with 4 steps, 19 with 1; one of 20000, 64 rows, 30 and 28; up to 16 rows
  // the join costs as much), and twice as many where there is enough for all (24 heads of 18000, 40 rows: 80 us with 4 steps, 62 with 8,
  // with weights 100 and 87; 96 heads of 18000 or of 900 to 9800: the same within 1 %).
  const bool many_rows = rows > 16;
  FragmentRule r{many_rows ? 0 : ATT_LEAST_LOG, 0};
  while (r.log < ATT_LEAST_LOG && total >> r.log > ATT_EVEN) ++r.log;
  while ((total - 1) >> r.log >= target) ++r.log;
  if (many_rows && r.log == ATT_LEAST_LOG && total >> (r.log + 1) >= ATT_EVEN) ++r.log;
  if (10ll * total >= 9ll * longest * heads)
    for (int parts = 1; parts <= EVEN_PARTS && r.per == 0; ++parts) {
      const int wgs = heads * parts, over = wgs % ATT_EVEN;
      if (wgs <= 2 * ATT_EVEN && (over == 0 || 10 * over >= 9 * ATT_EVEN)) {
        const int even = (int)((unsigned)(longest + parts - 1) / (unsigned)parts);
        r.per = even > 1 << ATT_LEAST_LOG ? even : 1 << ATT_LEAST_LOG;
      }
    }
  return r;
}
// Fragments of a head of that many steps.
__host__ __device__ __forceinline__ int fragments_of(int steps, const FragmentRule &r) {
  if (r.per == 0) return (steps + (1 << r.log) - 1) >> r.log;
  int parts = 0;
#pragma unroll
  for (int k = 0; k < EVEN_PARTS; ++k) parts += steps > k * r.per;
  return parts;
}

// The host's side, for heads of up to `steps` steps: the target, and room for all fragments that a device of `units` compute units
// makes of them or of longer ones.  (An even cut makes no more than 2 * ATT_EVEN, however few the units.)
inline int fragment_target(long long heads, long long steps, int rows, int units) {
  return (int)std::min((long long)SCAN_ROUNDS * (rows <= 32 ? 2 : 1) * units, std::max(((heads * steps - 1) >> ATT_LEAST_LOG) + 1, 2ll * ATT_EVEN));
}
inline int fragments_most(int heads, int target) { return std::max(target + heads, 2 * ATT_EVEN); }

}  // namespace cmp
