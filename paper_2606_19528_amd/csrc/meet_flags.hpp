// meet_flags.hpp -- the flags of meet.hpp's meetings in device memory.
#pragma once

#include <hip/hip_runtime.h>

#include "meet.hpp"

namespace lora {

// The flags of a meeting of n <= 64 workgroups (meet.hpp) as one wave reads and
// writes them, a word a lane.  (A counter instead of flags serialised the
// arrivals, 1.1 us each; only those that see all flags up meet in the exchange.)
struct MeetFlags {
  meet_word *w;
  int lane;
  __device__ void raise(int i, meet_word tag) {
    if (lane == 0) __hip_atomic_store(w + i, tag, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __device__ void settle() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
  __device__ bool all_up(int n, meet_word tag) {
    const meet_word f = lane < n ? __hip_atomic_load(w + lane, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : tag;
    return __ballot(f != tag) == 0;
  }
  // (the return value is lane 0's)
  __device__ meet_word lower(int n) {
    if (lane == 0) return __hip_atomic_exchange(w, meet_word(0), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (lane < n) __hip_atomic_store(w + lane, meet_word(0), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return 0;
  }
};

}  // namespace lora
