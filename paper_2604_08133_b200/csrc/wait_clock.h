// The clock of a bounded wait on something that is reached only after work of any length.  Plain C++ so that it can be
// unit-tested without a GPU.
#pragma once

#include <stdint.h>

#ifdef __CUDACC__
#define ALLOCMOE_HD __host__ __device__ __forceinline__
#else
#define ALLOCMOE_HD inline
#endif

namespace allocmoe {

// Runs out once `limit` clocks have gone by in which `progress` stayed the same.  A wait whose limit counted all the time
// until its event would give up on a long launch with nothing stuck; one that restarts without end would never give up.
// Each restart needs the counter to move, so a wait ends whenever whoever moves it does.
struct WaitClock {
  long long start = 0;
  uint32_t seen = 0;
  bool running = false;

  ALLOCMOE_HD bool ran_out(long long now, uint32_t progress, long long limit) {
    if (!running || progress != seen) {
      running = true;
      seen = progress;
      start = now;
      return false;
    }
    return now - start > limit;
  }
};

}  // namespace allocmoe
