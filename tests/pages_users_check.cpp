// How the kernels of the pages step over users, on the host, under UndefinedBehaviorSanitizer: every user once and in order, up to the last of
// 2^31 - 1 and for every step that the launchers take. Built and run by tests/test_pages_users_cpu.py.
#include <climits>
#include <cstdio>
#include <cstdlib>

#include "pages.h"

int main() {
  long long looked = 0;
  for (int U : {1, 1023, 1024, 1025, 70000, INT_MAX - 65536, INT_MAX - 65535, INT_MAX - 1024, INT_MAX - 1, INT_MAX})
    for (unsigned step : {1024u, 4096u, 65536u})
      for (unsigned first : {0u, 1u, 1022u, 1023u, step - 2, step - 1}) {
        if (first >= step) continue;
        long long next = first;
        laser::for_users(first, step, U, [&](int u) {
          if (u != next) {
            std::printf("user %lld of %d by steps of %u: %d\n", next, U, step, u);
            std::exit(1);
          }
          next += step;
        });
        if (next < U) return 1;
        ++looked;
      }
  std::printf("%lld ways, every user in order\n", looked);
  return 0;
}
