// An entry point that has no memory for its message returns a status: no exception
// leaves it.
#include <cstdio>
#include <cstdlib>
#include <new>

#include "simsd.h"

static bool refuse = false;
void* operator new(std::size_t n) {
  if (refuse) throw std::bad_alloc();
  void* p = std::malloc(n ? n : 1);
  if (!p) throw std::bad_alloc();
  return p;
}
void operator delete(void* p) noexcept { std::free(p); }
void operator delete(void* p, std::size_t) noexcept { std::free(p); }

int main() {
  double freq[32];
  float factor;
  refuse = true;
  simsd_status st[3];
  st[0] = simsd_rope_frequencies(64, 10000.0, SIMSD_ROPE_NONE, 1.0, 0, 1.0, 1.0, nullptr, &factor);
  st[1] = simsd_rope_frequencies(63, 10000.0, SIMSD_ROPE_NONE, 1.0, 0, 1.0, 1.0, freq, &factor);
  st[2] = simsd_rope_frequencies(64, 10000.0, SIMSD_ROPE_NONE, 1.0, 0, 1.0, 1.0, freq, &factor);
  refuse = false;
  std::printf("%d %d %d\n", st[0], st[1], st[2]);
  return st[0] != SIMSD_OK && st[1] != SIMSD_OK && st[2] == SIMSD_OK ? 0 : 1;
}
