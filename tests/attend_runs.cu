// How the attention's steps are cut into runs, on the host: every run's start, and the run of its first and last step, against 64 bits.
#include <cstdio>

#include "spd_attend.cuh"

int main() {
  const int runs[] = {1, 2, 3, 147, 296, 592, 1184, 1776, 2047, 2048, 2049, 2368, 4736};
  const int sums[] = {1, 5, 2367, 2368, 4096, 906876, 1 << 20, 1813753, 1813754, 1813755, 1867776, 2064384, (1 << 21) - 1, 1 << 21, (1 << 21) + 1, 2129920, 1 << 26, 2147483647};
  int bad = 0;
  for (int n : runs)
    for (int steps : sums) {
      if (n > steps) continue;   // no run is empty
      for (int i = 0; i <= n; ++i) {
        const long long from = (long long)i * steps / n, to = (long long)(i + 1) * steps / n - 1;
        if (spd::run_start(i, n, steps) != from) ++bad;
        if (i < n && (spd::run_of((int)from, n, steps) != i || spd::run_of((int)to, n, steps) != i)) ++bad;
        if (bad == 1) std::printf("run %d of %d over %d steps\n", i, n, steps);
      }
    }
  std::printf("%d wrong\n", bad);
  return bad != 0;
}
