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

// By warp, unless the units leave most of the machine's warps without work and a unit has more tiles than
// a warp should walk alone.  By warp, a warp takes all units of a root where they have a single tile and the roots alone fill the
// machine (14 400 roots of 21 entries: 51 against 55 us; with more tiles single units balance better, 278 against 315 us for 12 000
// roots of 520).
// A cluster above the portable size of 8 blocks is taken where fits(ranks) says that the device holds one.
template <typename Fits>
AttendShape choose_attend_shape(int64_t roots, int per_root, int64_t tiles, int sms, const Fits& fits) {
  const int64_t units = roots * per_root;
  const int64_t machine = (int64_t)sms * 12;                         // warps that are resident together
  AttendShape s = {false, 1, tiles <= 1 && roots >= machine ? per_root : 1};
  if (tiles <= 2 || units >= 2 * machine) return s;
  s.by_block = true;
  while (s.ranks < 16 && units * kAttendWarps * s.ranks * 2 <= machine && tiles >= 2 * kAttendWarps * s.ranks * 2) s.ranks *= 2;
  if (s.ranks > 8 && !fits(s.ranks)) s.ranks = 8;
  return s;
}

}  // namespace tgnn_history
