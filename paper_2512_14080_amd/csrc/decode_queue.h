// What a workgroup of the work queue (decode.hip) makes of the numbers that it reads from the
// workspace.  A call that shares its workspace with another one in flight, which is an error,
// may find counters that were set back, a selection of other experts, or partial logits that change
// between two waves of a token (whose places may then stay open): its results are then
// any, but its items and experts are its own ones all the same, and it ends.
#pragma once
#include <cstdint>
#ifndef __HIP__
#define __host__
#define __device__
#endif

namespace smoe {

// the item after `after`: the ticket's, or where the counter fell back the next one, so that a
// workgroup's items increase and are not below zero (first: after = -1)
__host__ __device__ inline int next_item(int after, int ticket) { return ticket > after ? ticket : after + 1; }

// an expert's number as read
__host__ __device__ inline int expert_within(uint32_t e, int E) { return e < (uint32_t)E ? (int)e : E - 1; }

}  // namespace smoe
