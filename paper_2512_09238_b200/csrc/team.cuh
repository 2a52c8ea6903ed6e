// A decision that all threads of a team take alike.
#pragma once

namespace tca {

// One answer for a team to a question whose answer may change while it is asked (an abort flag that another role of the
// CTA sets, a status word that another CTA writes): the leader asks, everybody hears what it was told at the team's
// barrier `meet`.  Needed wherever a branch holds barriers of the team: threads that asked for themselves could differ, and
// would then wait at different barriers, which have no limit.  The team meets again before it calls this with the
// same `said` the next time.
template <typename Ask, typename Meet>
__host__ __device__ __forceinline__ bool team_agrees(bool leader, volatile int* said, Ask ask, Meet meet) {
  if (leader) *said = ask() ? 1 : 0;
  meet();
  return *said != 0;
}

}  // namespace tca
