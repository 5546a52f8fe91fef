// Host check of csrc/attention_rows.h: what sequences hold, from offsets and lengths of
// any value, and that the costs of a call's sequences add up in 32 bits.
#include <climits>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "attention_rows.h"

using aqlm::AttnSeq;

#define CHECK(c)                                               \
  do {                                                         \
    if (!(c)) {                                                \
      std::printf("line %d: %s\n", __LINE__, #c);              \
      std::exit(1);                                            \
    }                                                          \
  } while (0)

static std::vector<AttnSeq> apart(const std::vector<int>& cu, const std::vector<int>& lens, int tokens, int64_t room,
                                  bool after = true) {
  std::vector<AttnSeq> s;
  int end = 0;
  for (size_t b = 0; b < lens.size(); ++b) {
    const AttnSeq own = aqlm::attn_cut(cu[b], cu[b + 1], lens[b], tokens, room);
    s.push_back(after ? aqlm::attn_after(own, end) : own);
    if (own.first + own.count > end) end = own.first + own.count;
  }
  return s;
}

// The largest cost that sequences can have: every unit of `rows` rows reads all keys.
static int64_t cost(const std::vector<AttnSeq>& s, int group, int rows, int64_t tiles) {
  int64_t sum = 0;
  for (const AttnSeq& x : s) sum += ((int64_t)x.count * group + rows - 1) / rows * tiles;
  return sum;
}

int main() {
  std::mt19937 gen(7);
  for (int round = 0; round < 20000; ++round) {
    const int seqs = 1 + gen() % 70, tokens = 1 + gen() % 200;
    const int64_t room = 1 + gen() % 1000;
    auto any = [&](int most) {
      const int odd[] = {INT_MIN, INT_MIN + 1, -1, 0, most, most + 1, INT_MAX - 1, INT_MAX};
      return gen() % 3 ? (int)(gen() % (most + 1)) : odd[gen() % 8];
    };
    std::vector<int> cu(seqs + 1), lens(seqs);
    for (int& x : cu) x = any(tokens);
    for (int& x : lens) x = any((int)room);
    const std::vector<AttnSeq> s = apart(cu, lens, tokens, room);
    std::vector<int> held(tokens, 0);
    int at = s[0].first;
    for (const AttnSeq& x : s) {
      CHECK(x.first == at && x.count >= 0 && x.count <= tokens - x.first);  // one after another, no token twice
      CHECK(x.keys >= 0 && x.keys <= room);
      at = x.first + x.count;
    }
    // offsets that ascend: every sequence is what they say
    for (int& x : cu) x = gen() % (tokens + 1);
    std::vector<int> up = cu;
    for (size_t i = 1; i < up.size(); ++i) up[i] = up[i] < up[i - 1] ? up[i - 1] : up[i];
    const std::vector<AttnSeq> t = apart(up, lens, tokens, room);
    for (int b = 0; b < seqs; ++b) CHECK(t[b].first == up[b] && t[b].first + t[b].count == up[b + 1]);
  }

  // A call at the limit that the entry point sets, (rows / 16 + sequences) * tiles below
  // 2^31, whose offsets give all tokens to every second sequence.
  const int seqs = 2032, tokens = 16384, group = 8;
  const int64_t tiles = ((int64_t(1) << 31) - 1) / (tokens * group / 16 + seqs);
  std::vector<int> cu(seqs + 1), lens(seqs, INT_MAX);
  for (int b = 0; b <= seqs; ++b) cu[b] = b % 2 ? tokens : 0;
  CHECK(cost(apart(cu, lens, tokens, tiles * 64), group, 16, tiles) <= INT_MAX);
  CHECK(cost(apart(cu, lens, tokens, tiles * 64, false), group, 16, tiles) > INT_MAX);  // each by itself: it would wrap
  std::printf("attention rows ok\n");
  return 0;
}
