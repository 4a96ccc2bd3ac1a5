// How attention to a paged cache cuts heads into fragments: the rule, which every workgroup carries out for itself on the lengths that the device
// finds, and the room that the host makes for what comes out of it.  The two have to agree whatever the device and the lengths are.
#pragma once

#include <algorithm>
#include <cmath>

#include "common.h"

namespace cmp {

constexpr int ATT_LEAST_LOG = 2;             // fewest steps of a fragment where there are many, log 2
constexpr int SCAN_HEADS = 512, SCAN_ROUNDS = 6;        // heads that a wave looks through, and fragments for every workgroup that
                                             // there is room for on the chip
constexpr int ATT_EVEN = 256, EVEN_PARTS = 4;          // units that have equal parts of heads of one length, and most parts of a head then

// Steps of a fragment: 1 << log, or `per` where that is not 0.  inv: 1 / per, or 0 where heads have EVEN_PARTS at most.
struct FragmentRule { int log, per; float inv; };
// total: steps of all heads; rows: query rows of a head; target: fragments that there are to be, beside the last of each head
__host__ __device__ __forceinline__ FragmentRule fragment_rule(int total, int longest, int heads, int rows, int target) {
  // More than 16 query rows make a step dearer and a start too, and more than 32 leave room for one workgroup a unit: fewer steps where all
  // find room at once (16 heads of 500 to 1411, 40 rows: 24 us with 4 steps, 19 with 1; one of 20000, 64 rows, 30 and 28; up to 16 rows
  // the join costs as much), and twice as many where there is enough for all (24 heads of 18000, 40 rows: 80 us with 4 steps, 62 with 8,
  // with weights 100 and 87; 96 heads of 18000 or of 900 to 9800: the same within 1 %).
  const bool many_rows = rows > 16;
  FragmentRule r{many_rows ? 0 : ATT_LEAST_LOG, 0, 0.f};
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
// The same for rows of 4 bits, which are so little to read that starts, ends and joins count for more, and a step waits for itself as much as for memory.
// Whole rounds of the workgroups that run at a time (slots), with steps of any number: as few rounds as leave fragments of 32 steps (a head's last
// one counts for five eighths of nothing), or where heads are of (nearly) one length of 64, of 24 where slots of a head lie apart and there are up to 16
// rows, and no more than the target has room for (us with 64 and 24: 384 heads of 16000, 4 rows, slots apart 199 and 185, together 164 and 167; 96 of 32000 105 and 102, 87
// and 90; 96 of 16000, 20 rows with their mass, apart 110 and 117).
// us with powers of two of steps and so: 128 heads of 2000 to 9000, 4 rows with their mass, 38.8 and 33.6, in pages of 7 slots 46.7 and 39.0; 96 of 900 to
// 9831, 4 rows, 25.6 and 23.5, 40 rows 81 and 66; 192 of 8192 to 32000, 40 capped rows, 325 and 280; 384 of 4000, 4 rows, 57 and 44; but 96 of 32000, 20
// rows with their mass, 191 and 200.
// Few heads: a fragment more costs their join what a step costs a fragment, nearly, so that most fragments of a head go with the root of its steps, in whole
// numbers of fragments for every unit (8 heads, 7 rows, of 8000 15.5 with one step each and 13.3 with two, of 16000 17.8 with two and 15.8 with four).
// What the ends of hundreds of short heads take must not leave a long one among them in one piece (us of 512 heads, one of 131072 and the others of 100 or 500, 4 rows,
// 4 with their mass, 20 with it, 40, with one part at least 791, 1030, 2156, 1520; 772, 1005, 2181, 1529; with 64 43, 45, 87, 57; 57, 65, 144, 108; with 96 43, 45, 82, 50; 46, 51,
// 112, 86; with ends taken off the rounds only 55, 58, 82, 56; 50, 51, 90, 66, but then of 256 heads, the others of 100, 45, 48, 72, 53 instead of 30, 32, 62, 44).
constexpr int LEAST_PARTS = 96;
__host__ __device__ __forceinline__ int bits4_slots(int rows) { return rows <= 16 ? 3 * ATT_EVEN : rows <= 48 ? 2 * ATT_EVEN : ATT_EVEN; }
__host__ __device__ __forceinline__ long long bits4_rounds(long long total, long long longest, long long heads, int rows, bool apart, bool even) {
  const int slots = bits4_slots(rows), even_steps = rows <= 16 && apart ? 24 : 64;
  return even ? (heads * ((longest + even_steps - 1) / even_steps) + slots - 1) / slots : ((total >> 5) + (5 * heads >> 3)) / slots + 1;
}
__host__ __device__ __forceinline__ FragmentRule bits4_fragment_rule(int total, int longest, int heads, int rows, int target, bool apart) {
  const int slots = bits4_slots(rows);
  const bool even = 10ll * total >= 9ll * longest * heads;
  const int ends = even ? 0 : 5 * heads >> 3, room = std::max(target / slots, 1), rounds = (int)bits4_rounds(total, longest, heads, rows, apart, even);
  const int joined = total / ((int)(0.375f * sqrtf((float)longest)) + 1) / ATT_EVEN + 1;
  const int parts = std::max(std::min(std::min(rounds, room) * slots, joined * ATT_EVEN) - ends, LEAST_PARTS);
  const int all = even ? longest : total, cut = even ? std::max(parts / heads, 1) : parts;
  int per = (int)((unsigned)(all + cut - 1) / (unsigned)cut);
  if ((long long)per * target < total) per = (int)((unsigned)(total + target - 1) / (unsigned)target);
  return FragmentRule{0, per, 1.f / (float)per};
}
// Fragments of a head of that many steps.
__host__ __device__ __forceinline__ int fragments_of(int steps, const FragmentRule &r) {
  if (r.per == 0) return (steps + (1 << r.log) - 1) >> r.log;
  if (r.inv > 0.f) {             // below 2^24, where a quotient by way of fp32 is off by one at most
    int parts = (int)((float)(steps + r.per - 1) * r.inv);
    const int rest = steps + r.per - 1 - parts * r.per;
    return parts + (rest >= r.per) - (rest < 0);
  }
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
// Workgroups that find no fragment cost their start, so no more rounds than the rule can want where heads hold no more than `steps` (us with a round or
// more to spare and so: 384 heads of 4000, 4 rows, 46.2 and 42.3, of 2000 32.1 and 29.3).
inline int bits4_fragment_target(long long heads, long long steps, int rows, int units, bool apart) {
  const long long joined = (heads * std::min(steps, (long long)(sqrtf((float)steps) / 0.375f)) / ATT_EVEN + 1) * ATT_EVEN;
  const long long rounds = std::max(bits4_rounds(heads * steps, steps, heads, rows, apart, true), bits4_rounds(heads * steps, steps, heads, rows, apart, false));
  return (int)std::min(std::min((long long)SCAN_ROUNDS * (rows <= 32 ? 2 : 1) * units, rounds * bits4_slots(rows)), joined);
}
inline int fragments_most(int heads, int target) { return std::max(target + heads, 2 * ATT_EVEN); }

}  // namespace cmp
