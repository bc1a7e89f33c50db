// Host-only exercise of the calls that bring rows to the pool, for a build with AddressSanitizer and UndefinedBehaviorSanitizer on
// the host pass: reservations over random chains, and every refusal of the calls that would launch.  Device pointers are
// fake and never dereferenced; no call here enqueues work.
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cmath>
#include <random>
#include <vector>

#include "tokenlake.h"

#define CHECK(cond)                                                                                                   \
  do {                                                                                                                \
    if (!(cond)) {                                                                                                    \
      std::fprintf(stderr, "rows_driver: line %d: %s failed (%s)\n", __LINE__, #cond, tl_last_error());              \
      std::exit(1);                                                                                                   \
    }                                                                                                                 \
  } while (0)

static void* at(uintptr_t x) { return (void*)x; }

int main() {
  std::mt19937_64 rng(2024);
  auto pick = [&](int lo, int hi) { return (int)(lo + rng() % (uint64_t)(hi - lo + 1)); };
  long n_rows_seen = 0;
  for (int round = 0; round < 60; ++round) {
    const int C = 64 << pick(0, 2), n_slots = pick(3, 40), n_chains = pick(1, 6);
    tl_pool* pool = nullptr;
    CHECK(tl_pool_create(&pool, n_slots, C, 1 << pick(0, 3), 128, at(1 << 28), at(1u << 30)) == TL_OK);
    std::vector<std::vector<uint64_t>> chain(n_chains);
    std::vector<int> total(n_chains, 0);
    std::vector<int> owner(n_slots * C, 0);        // which row of the pool has been given out
    uint64_t next = 1;
    for (int step = 0; step < 8; ++step) {
      std::vector<int32_t> has(n_chains), new_ptr(1, 0), row_ptr(1, 0);
      std::vector<uint64_t> tails(n_chains, 0), ids;
      for (int c = 0; c < n_chains; ++c) {
        const int n = pick(0, 4) == 0 ? 0 : pick(1, 2 * C);
        has[c] = total[c] % C != 0;
        if (has[c]) tails[c] = chain[c].back();
        const int room = has[c] ? C - total[c] % C : 0, rest = n > room ? n - room : 0;
        for (int i = 0; i < (rest + C - 1) / C; ++i) ids.push_back(next + ids.size() + 1000 * step);
        new_ptr.push_back((int32_t)ids.size());
        row_ptr.push_back(row_ptr.back() + n);
      }
      next += ids.size();
      std::vector<int32_t> slots(ids.size(), -1), rows(row_ptr.back(), -1);
      int32_t used = 0, after = 0;
      CHECK(tl_pool_used(pool, &used) == TL_OK);
      const tl_status s = tl_pool_reserve_batch(pool, n_chains, has.data(), tails.data(), new_ptr.data(), ids.empty() ? nullptr : ids.data(),
                                                row_ptr.data(), slots.empty() ? nullptr : slots.data(), rows.empty() ? nullptr : rows.data());
      CHECK(tl_pool_used(pool, &after) == TL_OK);
      if (used + (int)ids.size() > n_slots) {
        CHECK(s == TL_EFULL && after == used);
        break;
      }
      CHECK(s == TL_OK && after == used + (int)ids.size());
      for (int c = 0; c < n_chains; ++c) {
        for (int i = row_ptr[c]; i < row_ptr[c + 1]; ++i) {
          CHECK(rows[i] >= 0 && rows[i] < n_slots * C && owner[rows[i]]++ == 0);
          CHECK(rows[i] % C == (total[c] + i - row_ptr[c]) % C);
          ++n_rows_seen;
        }
        total[c] += row_ptr[c + 1] - row_ptr[c];
        chain[c].insert(chain[c].end(), ids.begin() + new_ptr[c], ids.begin() + new_ptr[c + 1]);
      }
    }
    CHECK(tl_pool_destroy(pool) == TL_OK);
  }

  std::vector<double> freq = {1.0, 0.5, -3.0, 1e300, 1e-300, 0.0, 7.0, 6.283185307179586};
  std::vector<uint64_t> steps(freq.size());
  CHECK(tl_rope_steps(freq.data(), (int32_t)freq.size(), steps.data()) == TL_OK && steps[5] == 0);
  freq[3] = INFINITY;
  CHECK(tl_rope_steps(freq.data(), (int32_t)freq.size(), steps.data()) == TL_EINVAL);

  // refused calls: nothing here may reach a launch (random strides and addresses, always one thing wrong)
  tl_pool* pool = nullptr;
  CHECK(tl_pool_create(&pool, 8, 64, 2, 128, at(1 << 28), at(1u << 30)) == TL_OK);
  for (int round = 0; round < 4000; ++round) {
    tl_rope rope = {(const uint64_t*)at(0x5000), 16 * pick(1, 8), pick(0, 1), 1.f};
    tl_qkv d = {};
    d.q = at(0x100000), d.k = at(0x200000), d.v = at(0x300000);
    auto stride = [&]() { return (int64_t)(rng() >> pick(0, 63)) * (pick(0, 1) ? 1 : -1); };
    d.q_row_stride = stride(), d.q_head_stride = stride(), d.k_row_stride = stride(), d.k_head_stride = stride(), d.v_row_stride = stride(), d.v_head_stride = stride();
    d.q_heads = pick(1, 70), d.kv_heads = 2, d.is_bf16 = pick(0, 1), d.eps = 1e-6f;
    d.q_out = at(0x400000), d.k_out = at(0x500000), d.v_out = at(0x600000);
    int32_t n = pick(1, 5);
    const void *pos = at(0x7000), *rows = at(0x8000);
    switch (pick(0, 6)) {
      case 0: rope.rot_dim = pick(0, 1) ? 8 : 256; break;
      case 1: rope.factor = NAN; break;
      case 2: n = -pick(1, 1 << 30); break;
      case 3: d.q_out = nullptr; break;
      case 4: d.kv_heads = -1; break;
      case 5: pos = nullptr; break;
      case 6: d.k_out = d.v_out; break;
    }
    CHECK(tl_rotate_rows(&rope, &d, (const int32_t*)pos, n, nullptr) == TL_EINVAL);
    CHECK(tl_pool_write_rows(pool, &rope, &d, (const int32_t*)pos, (const int32_t*)rows, n, nullptr) == TL_EINVAL);
  }
  CHECK(tl_pool_destroy(pool) == TL_OK);
  std::printf("%ld rows reserved, all statuses as expected\n", n_rows_seen);
  return 0;
}
