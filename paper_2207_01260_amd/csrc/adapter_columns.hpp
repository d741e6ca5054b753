// Which columns a lane of the adapters' outer products has, and how many of them a row holds.  Plain C++, for the kernel and a host program that walks every lane.
#pragma once
#include "split_index.hpp"

namespace cprune {

// A work-group has 16 V of a side's c columns, lanes of a row number V of them from `column` on; the row holds `there` of those (none where that is not above 0).
// thin: columns are read one by one.  Otherwise there are V, and a lane past the last V has the last V again.
struct OuterLane {
  int column, there;
};
CPRUNE_HD OuterLane outer_lane(int c, int v, int group, int lane_row, bool thin) {
  const int from = (group * 16 + lane_row) * v, column = thin || from < c - v ? from : c - v;
  return OuterLane{column, c - column};
}

}  // namespace cprune
