// Host memory that runs out while ids are entered into the pool or leave it: every call says TL_ENOMEM, nothing throws across the C boundary and nothing is
// registered.  operator new fails at the n-th call for every n until the call gets through.  Device pointers are fake; no call here enqueues work.
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <new>
#include <vector>

#include "tl_internal.h"
#include "tokenlake.h"

static long g_left = -1;       // allocations until one fails; -1: none does

void* operator new(std::size_t n) {
  if (g_left == 0) throw std::bad_alloc();
  if (g_left > 0) --g_left;
  void* p = std::malloc(n ? n : 1);
  if (!p) throw std::bad_alloc();
  return p;
}
void operator delete(void* p) noexcept { std::free(p); }
void operator delete(void* p, std::size_t) noexcept { std::free(p); }

#define CHECK(cond)                                                                                                   \
  do {                                                                                                                \
    if (!(cond)) {                                                                                                    \
      g_left = -1;                                                                                                    \
      std::fprintf(stderr, "memory_driver: line %d: %s failed (%s)\n", __LINE__, #cond, tl_last_error());            \
      std::exit(1);                                                                                                   \
    }                                                                                                                 \
  } while (0)

static void* at(uintptr_t x) { return (void*)x; }

static tl_pool* new_pool() {
  tl_pool* pool = nullptr;
  CHECK(tl_pool_create(&pool, 64, 64, 1, 128, at(1 << 28), at(1u << 30)) == TL_OK);
  return pool;
}

// `used` slots are taken and none of the ids is resident.
static void check_unchanged(tl_pool* pool, int32_t used, const std::vector<uint64_t>& ids) {
  int32_t n = -1;
  CHECK(tl_pool_used(pool, &n) == TL_OK && n == used);
  std::vector<int32_t> slots(ids.size(), 7);
  CHECK(tl_pool_lookup(pool, ids.data(), (int32_t)ids.size(), slots.data()) == TL_OK);
  for (int32_t s : slots) CHECK(s == -1);
}

int main() {
  std::vector<uint64_t> ids;
  std::vector<int32_t> slots, fills;
  for (int i = 0; i < 40; ++i) ids.push_back(1000 + i), slots.push_back(i), fills.push_back(1 + i);
  long failures = 0;

  // adopt
  for (long n = 0;; ++n) {
    tl_pool* pool = new_pool();
    g_left = n;
    const tl_status s = tl_pool_adopt(pool, ids.data(), slots.data(), fills.data(), 40, nullptr);
    g_left = -1;
    if (s == TL_OK) {
      int32_t used = 0;
      CHECK(tl_pool_used(pool, &used) == TL_OK && used == 40);
      CHECK(tl_pool_destroy(pool) == TL_OK);
      break;
    }
    CHECK(s == TL_ENOMEM);
    check_unchanged(pool, 0, ids);
    CHECK(tl_pool_adopt(pool, ids.data(), slots.data(), fills.data(), 40, nullptr) == TL_OK);      // and the same call works once there is memory
    CHECK(tl_pool_destroy(pool) == TL_OK);
    ++failures;
  }

  // reserve: a tail and new segments
  for (long n = 0;; ++n) {
    tl_pool* pool = new_pool();
    const uint64_t tail = 1;
    const int32_t slot = 3, fill = 60, has = 1, new_ptr[2] = {0, 40}, row_ptr[2] = {0, 4 + 40 * 64};
    CHECK(tl_pool_adopt(pool, &tail, &slot, &fill, 1, nullptr) == TL_OK);
    std::vector<int32_t> rows(row_ptr[1]);
    g_left = n;
    const tl_status s = tl_pool_reserve_batch(pool, 1, &has, &tail, new_ptr, ids.data(), row_ptr, nullptr, rows.data());
    g_left = -1;
    if (s == TL_OK) {
      CHECK(tl_pool_destroy(pool) == TL_OK);
      break;
    }
    int32_t now = 0;
    CHECK(s == TL_ENOMEM);
    check_unchanged(pool, 1, ids);
    CHECK(tl_pool_fills(pool, &slot, 1, &now) == TL_OK && now == fill);
    CHECK(tl_pool_destroy(pool) == TL_OK);
    ++failures;
  }

  // prefix tree and eviction: paths 1000, 1001, ... under the root and the same ids under 1005, so that slots have nodes with and without children
  for (long n = 0;; ++n) {
    tl_pool* pool = new_pool();
    CHECK(tl_pool_adopt(pool, ids.data(), slots.data(), fills.data(), 40, nullptr) == TL_OK);
    for (uint64_t id : ids) CHECK(tl_pool_release(pool, id) == TL_OK);
    bool threw = false;
    int32_t at = 0, made = 0;
    g_left = n;
    try {
      for (int i = 0; i < 40; ++i) at = pool->tree.child(i % 8 ? at : 0, ids[i], slots[i]), ++made;
      for (int i = 0; i < 40; ++i)
        if (i != 5) pool->tree.child(i % 3 ? at : pool->tree.child(0, ids[5], slots[5]), ids[i], slots[i]);
    } catch (const std::bad_alloc&) {
      threw = true;
    }
    g_left = -1;
    const int32_t before = pool->tree.size();
    // every node is reached from the root and from its parent by its id
    std::vector<int32_t> order;
    pool->tree.level_order(1 << 20, order);
    CHECK((int32_t)order.size() == before && before >= made);
    for (int32_t x : order) CHECK(pool->tree.child(pool->tree.at(x).parent, pool->tree.at(x).id, pool->tree.at(x).slot) == x);
    // evictions with one failure each, until all is gone
    uint64_t gone = 0;
    int32_t used = 40;
    while (used > 0) {
      g_left = n % 3;
      tl_status s = tl_pool_evict_lru(pool, &gone);
      g_left = -1;
      int32_t now = 0;
      CHECK(tl_pool_used(pool, &now) == TL_OK);
      if (s == TL_ENOMEM) {
        CHECK(now == used);
        ++failures;
        s = tl_pool_evict_lru(pool, &gone);
        CHECK(tl_pool_used(pool, &now) == TL_OK);
      }
      CHECK(s == TL_OK && now == used - 1);
      used = now;
      order.clear();
      pool->tree.level_order(1 << 20, order);
      CHECK((int32_t)order.size() == pool->tree.size());
    }
    CHECK(pool->tree.size() == 0);
    CHECK(tl_pool_destroy(pool) == TL_OK);
    if (!threw) break;
    ++failures;
  }

  // put: its one entry, before anything is enqueued
  tl_pool* pool = new_pool();
  int32_t got = -1;
  g_left = 0;
  const tl_status s = tl_pool_put(pool, 1000, at(0x1000), at(0x2000), 5, -1, &got, nullptr);
  g_left = -1;
  CHECK(s == TL_ENOMEM && got == -1);
  check_unchanged(pool, 0, ids);
  CHECK(tl_pool_destroy(pool) == TL_OK);
  std::printf("%ld failures, nothing registered\n", failures + 1);
  return 0;
}
