// Host build of the dQ kernel's grid: row workgroups that fit a launch by themselves (at most 2^32 - 1 threads, 256 each)
// have the split blocks' sums behind them exactly where both fit.  Prints "ok" and exits 0, or names the first failure.
#include <cstdio>

#include "kvs_launch.h"

int main() {
  const long long most = 0xffffffffll / 256;   // workgroups of a launch
  for (long long rows = most - 2 * kvs::kReduceGrid; rows <= most; ++rows)
    if (!kvs::row_blocks_fit(rows) || kvs::row_blocks_fit(rows + 2 * kvs::kReduceGrid + 1) ||
        kvs::sums_fit_dq(rows) != (rows + kvs::kReduceGrid <= most)) {
      std::printf("%lld row workgroups\n", rows);
      return 1;
    }
  if (!kvs::sums_fit_dq(1)) return 1;
  std::printf("ok\n");
  return 0;
}
