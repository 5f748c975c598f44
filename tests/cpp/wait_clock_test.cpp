// Host-only check of the clock behind waits that span work of any length (csrc/wait_clock.h).
#include <cstdio>

#include "wait_clock.h"

using namespace allocmoe;

static int fails = 0;
#define CHECK(c) do { if (!(c)) { std::printf("FAIL line %d: %s\n", __LINE__, #c); ++fails; } } while (0)

int main() {
  {   // nothing moves: over after the limit, whatever the first reading of the clock and of the counter
    WaitClock w;
    CHECK(!w.ran_out(5000000000000ll, 17u, 100));
    CHECK(!w.ran_out(5000000000100ll, 17u, 100));
    CHECK(w.ran_out(5000000000101ll, 17u, 100));
  }
  {   // a counter that starts at zero and stays there is no progress
    WaitClock w;
    CHECK(!w.ran_out(10, 0u, 100));
    CHECK(w.ran_out(111, 0u, 100));
  }
  {   // work goes on: a thousand limits later the wait still holds, and it ends when the work does
    WaitClock w;
    long long now = 0;
    for (uint32_t k = 0; k < 2000; ++k, now += 50) CHECK(!w.ran_out(now, k, 100));
    now -= 50;
    CHECK(!w.ran_out(now + 100, 1999u, 100));
    CHECK(w.ran_out(now + 101, 1999u, 100));
  }
  {   // progress seen late restarts the clock at the time it is seen; a counter that wraps is progress too
    WaitClock w;
    CHECK(!w.ran_out(0, 0xFFFFFFFFu, 100));
    CHECK(!w.ran_out(1000, 0u, 100));
    CHECK(!w.ran_out(1100, 0u, 100));
    CHECK(w.ran_out(1101, 0u, 100));
  }
  std::printf(fails ? "FAILED\n" : "ok\n");
  return fails ? 1 : 0;
}
