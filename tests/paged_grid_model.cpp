// What in_launches() of bc_paged_grid.h makes of every line "groups threads" of the input: launches, workgroups in all, the most threads of one, whether each starts where the last
// one ended.
#include <cstdio>

#include "bc_paged_grid.h"

int main() {
  long long groups;
  int threads;
  while (std::scanf("%lld %d", &groups, &threads) == 2) {
    long long launches = 0, all = 0, most = 0;
    bool joined = true;
    bc::in_launches(groups, threads, [&](uint32_t first, unsigned n) {
      ++launches;
      joined = joined && first == all && n > 0;
      all += n;
      most = (long long)n * threads > most ? (long long)n * threads : most;
    });
    std::printf("launches=%lld all=%lld most=%lld joined=%d\n", launches, all, most, joined);
  }
}
