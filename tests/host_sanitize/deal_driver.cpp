// Every head of every token of a rows call is dealt to exactly one wave, and every launch takes at least one group of tokens:
// the dealing as the library makes it, over head counts from none to the most that a call may have.  Host arithmetic.
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "rows_deal.h"

using namespace tl;

static long n_waves_seen = 0;

static void check(bool ok, const char* what, const int32_t (&heads)[3]) {
  if (ok) return;
  std::fprintf(stderr, "deal_driver: %d / %d / %d heads: %s\n", heads[0], heads[1], heads[2], what);
  std::exit(1);
}

static void deal(int32_t q, int32_t k, int32_t v) {
  const int32_t heads[3] = {q, k, v};
  const Dealing a = deal_heads(heads);
  const int64_t waves = a.group_waves.d, most = most_groups(a);
  check(waves >= 1, "no waves", heads);
  check(most >= 1, "a launch takes no group", heads);
  check(most * waves <= (int64_t)1 << 25, "threads of a launch beyond 2^31", heads);
  check((uint64_t)(most * waves) * (uint64_t)waves < (uint64_t)1 << 32, "a quotient that is not exact", heads);
  // the first, the second and the last groups of a launch, every wave
  const int64_t tokens = (int64_t)1 << a.group_log2;
  std::vector<uint8_t> seen((size_t)(q + k + v) * tokens);
  for (int64_t g : {(int64_t)0, (int64_t)1, most - 1}) {
    if (g >= most) continue;
    seen.assign(seen.size(), 0);
    for (int64_t w = g * waves; w < (g + 1) * waves; ++w) {
      const Place p = place_of(a.kind, a.group_log2, a.group_waves, (uint32_t)w);
      check(p.kind >= 0 && p.kind < 3 && heads[p.kind] > 0, "a wave of a kind that is not there", heads);
      const Deal& d = a.kind[p.kind];
      const int at_once = kWaveHeads >> d.tokens_log2;
      check(p.token >= g * tokens && p.token + (1 << d.tokens_log2) <= (g + 1) * tokens, "a token of another group", heads);
      check(p.head >= 0 && p.head < d.heads, "a head that is not there", heads);
      const int64_t first = p.kind == 0 ? 0 : p.kind == 1 ? q : q + k;
      for (int t = 0; t < 1 << d.tokens_log2; ++t)
        for (int h = p.head; h < p.head + at_once && h < d.heads; ++h) {
          uint8_t& s = seen[(size_t)((p.token - g * tokens + t) * (q + k + v) + first + h)];
          check(s == 0, "a head of a token is dealt twice", heads);
          s = 1;
        }
      ++n_waves_seen;
    }
    for (uint8_t s : seen) check(s == 1, "a head of a token is not dealt", heads);
  }
}

int main() {
  const int32_t counts[] = {0, 1, 2, 3, 4, 5, 8, 9, 28, 64, 1000, 8191, 16384, 23169, 23176, 23184, 32768, 46336, 46337, 46344, 50000, 65535, kMostHeads};
  for (int32_t q : counts)
    for (int32_t kv : counts) {
      if (q || kv) deal(q, kv, kv);            // queries, keys and values
      if (q || kv) deal(q, kv, 0);             // without values
      if (kv) deal(0, kv, kv);                 // keys and values, as moves have them
    }
  deal(0, 0, 1);
  deal(0, 0, kMostHeads);
  std::printf("%ld waves, every head dealt once\n", n_waves_seen);
  return 0;
}
