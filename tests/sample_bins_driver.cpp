// Host check of csrc/sample_bins.h: a bin has the numbers between its ends, and the ends of bins beside one
// another meet, whatever the size of the numbers.
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <random>

#include "sample_bins.h"

using aqlm::Bins;

#define CHECK(c)                                                                \
  do {                                                                          \
    if (!(c)) {                                                                 \
      std::printf("line %d: %s (f %.9g, bin %d)\n", __LINE__, #c, at_f, at_bin); \
      std::exit(1);                                                             \
    }                                                                           \
  } while (0)
static float at_f = 0.f;
static int at_bin = 0;

static void whole(float f, int depth) {
  const Bins b{(int)std::floor(f) + depth, false, 0.f};
  at_f = f;
  at_bin = b.at(f);
  CHECK(at_bin == depth);
  CHECK(b.lower(at_bin) <= f && f < b.upper(at_bin));
}

static void part(float low, float f) {
  if (!(low <= f && f < low + 1.f)) return;
  const Bins b{0, true, low};
  at_f = f;
  at_bin = b.at(f);
  CHECK(at_bin >= 0 && at_bin < 512);
  CHECK(b.lower(at_bin) <= f && f < b.upper(at_bin));
}

int main() {
  std::mt19937 gen(5);
  std::uniform_real_distribution<float> unit(0.f, 1.f);
  for (int round = 0; round < 2000000; ++round) {
    float f = std::ldexp(unit(gen) - 0.5f, (int)(gen() % 31));  // up to 2^29
    switch (gen() % 4) {
      case 0: f = std::floor(f); break;
      case 1: f = std::nextafter(std::floor(f), -INFINITY); break;
      case 2: f = std::nextafter(std::floor(f), INFINITY); break;
    }
    whole(f, gen() % 511);
  }
  for (int e = 0; e <= 29; ++e)
    for (int sign = -1; sign <= 1; sign += 2) {
      const Bins b{sign * (1 << e) + (int)(gen() % 100), false, 0.f};
      for (at_bin = 0; at_bin < 510; ++at_bin) {
        CHECK(b.upper(at_bin + 1) == b.lower(at_bin));
        CHECK((double)b.lower(at_bin) >= b.top - at_bin);
        CHECK((double)std::nextafter(b.lower(at_bin), -INFINITY) < b.top - at_bin);
      }
    }
  for (int e = 0; e < 14; ++e)
    for (int sign = -1; sign <= 1; sign += 2) {
      const float low = (float)(e == 0 ? (sign < 0 ? -1 : 0) : sign * ((1 << e) - (int)(gen() % 2)));
      for (int round = 0; round < 100000; ++round) {
        float f = low + unit(gen);
        if (round % 2) f = low + (float)(gen() % 513) / 512.f;
        part(low, f);
        part(low, std::nextafter(f, -INFINITY));
        part(low, std::nextafter(f, INFINITY));
      }
    }
  for (float f : {-1e-9f, -1e-30f, -1e-45f, -2e-8f, -6e-8f, -1.f / 512, -1.f / 512 - 1e-9f, -0.25f - 1e-8f}) part(-1.f, f);
  std::printf("sample bins ok\n");
  return 0;
}
