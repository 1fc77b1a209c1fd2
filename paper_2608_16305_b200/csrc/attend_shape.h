// How attention over the row cache is launched: plain C++, so that the rule can be run without a device.
#pragma once
#include <stdint.h>

namespace tgnn_history {

constexpr int kAttendWarps = 4;            // warps of a block

// Warps on one unit: by warp, or a block, or a cluster of `ranks` blocks.  By warp, a warp takes `take` neighbouring units.
struct AttendShape {
  bool by_block;
  int ranks, take;
};

// By warp where a unit has too few tiles to share, or where there are units enough.  A warp per unit works in waves of as many warps as are resident (8 to 20
// per SM, by the kernel's registers), a block per unit spreads evenly but meets at its end, which costs the more the shorter the windows are.  The two
// sides cross near 12 units per SM for windows of up to 16 tiles, near 24 beyond (by warp and by block, us; 2 heads of 50 in 8 bits over 66 entries: 1200 units
// 10.0 and 10.4, 2400 11.7 and 16.7, 3400 16.5 and 22.7; one of 128 in 8 bits over 250: 888 25.4 and 20.9, 1776 29.0 and 38.9, 2200 49.3 and 46.8,
// 3400 53.8 and 69.8; over 1000: 888 76.5 and 55.8, 1776 88.8 and 104.9, 2200 154 and 127, 3400 171 and 193; 8 heads over 2 of 64 in 4 bits over 1000: 888
// 44.5 and 32.8, 1776 52.0 and 51.0, 2700 71.5 and 75.5, 3400 97.7 and 90.3).
// By warp, a warp takes all units of a root where they have a single tile and the roots alone make 12 warps per SM: the units of a root share its
// set-up (14 400 roots of 21 entries, 2 heads: 39 us, 45 by single units; 1776 roots 8.4 and 10.3, 1000 roots 8.3 and 7.6; with more tiles single units
// balance better, 289 and 299 us for 12 000 roots of 516).
// A cluster above the portable size of 8 blocks is taken where fits(ranks) says that the device holds one.
template <typename Fits>
AttendShape choose_attend_shape(int64_t roots, int per_root, int64_t tiles, int sms, const Fits& fits) {
  const int64_t units = roots * per_root;
  const int64_t machine = (int64_t)sms * 12;
  AttendShape s = {false, 1, tiles <= 1 && roots >= machine ? per_root : 1};
  if (tiles <= 2 || units >= (tiles <= 16 ? machine : 2 * machine)) return s;
  s.by_block = true;
  while (s.ranks < 16 && units * kAttendWarps * s.ranks * 2 <= machine && tiles >= 2 * kAttendWarps * s.ranks * 2) s.ranks *= 2;
  if (s.ranks > 8 && !fits(s.ranks)) s.ranks = 8;
  return s;
}

}  // namespace tgnn_history
