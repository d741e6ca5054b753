// Which columns a lane of the adapters' outer products has, and how many of them a row holds.  Plain C++, shared by the kernel that makes their sums, the one that joins
// them and a host program that walks both.
#pragma once
#include "split_index.hpp"

namespace cprune {

// A work-group has 16 V of a side's c columns, lanes of a row number V of them from `column` on.  A lane past the last V has the last V again, and stores what their lanes do; of a
// side of fewer than V, whatever the other has, the row holds `there` (none where that is not above 0).
struct OuterLane {
  int column, there;
};
CPRUNE_HD OuterLane outer_lane(int c, int v, int group, int lane_row) {
  const int from = (group * 16 + lane_row) * v, column = c < v || from < c - v ? from : c - v;
  return OuterLane{column, c - column};
}

}  // namespace cprune
