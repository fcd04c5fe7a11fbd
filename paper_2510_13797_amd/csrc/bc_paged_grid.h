// Grids of more threads than one launch takes.  HIP launches fewer than 2^32 threads at once, 2^24 workgroups of 256; the paged cache's
// calls may have up to 2^31 - 1 workgroups (each sequence may have all of a call's rows, as far as the host knows).  Those go out in
// several launches, each of which is told its first workgroup.  No HIP here: a host test plays it through.
#pragma once
#include <cstdint>

namespace bc {

constexpr int64_t kLaunchThreads = 1LL << 31;

// launch(first workgroup, workgroups) until all `groups` of `threads` each are out
template <typename F>
void in_launches(int64_t groups, int threads, F launch) {
  const int64_t most = kLaunchThreads / threads;
  for (int64_t first = 0; first < groups; first += most) launch((uint32_t)first, (unsigned)(groups - first < most ? groups - first : most));
}

}  // namespace bc
