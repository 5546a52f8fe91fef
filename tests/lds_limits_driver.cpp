// Host check of csrc/lds_limits.h: whatever sizes calls ask for one after another, a kernel's limit
// on a device is never below what the call needs.
#include <cstdio>
#include <cstdlib>
#include <map>
#include <random>
#include <utility>

#include "lds_limits.h"

#define CHECK(c)                                  \
  do {                                            \
    if (!(c)) {                                   \
      std::printf("line %d: %s\n", __LINE__, #c); \
      std::exit(1);                               \
    }                                             \
  } while (0)

int main() {
  int kernels[3];
  std::map<std::pair<const void*, int>, int> limit;  // what a device would hold: the last value set
  aqlm::LdsLimits limits;
  int sets = 0;
  auto call = [&](int k, int dev, int bytes) {
    CHECK(limits.allow(&kernels[k], dev, bytes, [&] {
      limit[{&kernels[k], dev}] = bytes;
      ++sets;
      return 0;
    }) == 0);
    CHECK((limit[{&kernels[k], dev}]) >= bytes);
  };
  for (int bytes : {73728, 2304, 73728, 1000, 73728}) call(0, 0, bytes);  // long lists, short ones, long ones again
  CHECK(sets == 1);
  call(0, 1, 2304);  // another device, another kernel: limits of their own
  call(1, 0, 2304);
  CHECK(sets == 3);
  std::mt19937 gen(3);
  for (int i = 0; i < 100000; ++i) call(gen() % 3, gen() % 4, 1 + gen() % 163840);
  // a refused size is not remembered
  CHECK(limits.allow(&kernels[0], 9, 500, [] { return 7; }) == 7);
  CHECK(limits.allow(&kernels[0], 9, 500, [] { return 0; }) == 0);
  std::printf("lds limits ok\n");
  return 0;
}
