// Host-side checker of the plans of the 4-bit attention and of eviction (plan.cpp), over random calls: the
// workspace's regions hold what the kernels put there and follow each other, and the order in which
// an eviction's tasks are moved is a permutation from the longest to the shortest.  Prints "ok <calls>", or
// what is wrong.
#include <stdio.h>
#include <stdlib.h>

#include <random>
#include <vector>

#include "plan.h"

using namespace tide;

static int g_call = 0;

#define CHECK(x)                                                             \
  do {                                                                       \
    if (!(x)) {                                                              \
      printf("line %d: %s (call %d)\n", __LINE__, #x, g_call);               \
      exit(1);                                                               \
    }                                                                        \
  } while (0)

static void check_units(int op, const std::vector<int32_t>& a, const std::vector<int32_t>& e, const tide_dims& d) {
  Plan p;
  CHECK(make_plan_kv4_units(op, (int)a.size(), a.data(), e.data(), d, -1, true, &p) == TIDE_OK);
  if (p.num_items == 0) return;
  const int group = d.num_q_heads / d.num_kv_heads;
  const StreamSlots slots = {p.num_runs, p.num_tasks, kv4_waves(p.num_items)};
  const size_t parts = (size_t)slots.count() * d.num_kv_heads, rows = parts * p.tokens_per_item * group;
  CHECK(p.tasks_off >= sizeof(WsHeader));
  CHECK(p.tasks_off + p.num_tasks * sizeof(TaskDesc) <= p.items_off);
  CHECK(p.items_off + p.num_runs * sizeof(Kv4Run) <= p.tickets_off);
  CHECK(p.tickets_off + parts * sizeof(uint64_t) <= p.upload_bytes && p.upload_bytes == p.part_o_off);
  CHECK(p.part_o_off + rows * d.head_dim * sizeof(float) <= p.part_ml_off);
  CHECK(p.part_ml_off + rows * 4 * sizeof(float) <= p.total_bytes);
  CHECK(p.tasks_off % 16 == 0 && p.items_off % 16 == 0 && p.tickets_off % 16 == 0 && p.part_o_off % 16 == 0 &&
        p.part_ml_off % 16 == 0);
}

static void check_evict(const std::vector<int32_t>& n, const std::vector<int32_t>& keep, const tide_dims& d) {
  Plan p;
  CHECK(make_plan_evict((int)n.size(), n.data(), keep.data(), nullptr, d, -1, -1, true, &p) == TIDE_OK);
  const EvictTask* t = reinterpret_cast<const EvictTask*>(p.blob.data() + p.tasks_off);
  std::vector<bool> seen(p.num_tasks);
  for (int i = 0; i < p.num_tasks; ++i) {
    const int x = t[i].nth;
    CHECK(x >= 0 && x < p.num_tasks && !seen[x]);
    seen[x] = true;
    if (i > 0) {
      const int y = t[i - 1].nth;
      CHECK(t[y].keep > t[x].keep || (t[y].keep == t[x].keep && y < x));
    }
  }
  int32_t longest = 0;
  for (int32_t k : keep) longest = std::max(longest, k);
  CHECK(p.chunk == longest);
  CHECK(p.tasks_off + p.num_tasks * sizeof(EvictTask) <= p.upload_bytes && p.upload_bytes <= p.part_o_off);
}

int main(int argc, char** argv) {
  const int calls = argc > 1 ? atoi(argv[1]) : 300;
  std::mt19937 rng(11);
  auto pick = [&](int lo, int hi) { return (int)std::uniform_int_distribution<int>(lo, hi)(rng); };
  const int heads[][2] = {{1, 1}, {28, 4}, {32, 8}, {16, 1}, {5, 5}, {2500, 2500}, {64, 8}, {32, 2}};
  for (g_call = 0; g_call < calls; ++g_call) {
    const auto& h = heads[pick(0, 7)];
    const tide_dims d = {h[0], h[1], pick(0, 1) ? 64 : 128, kPage, 0.1f};
    const int n = pick(0, 3) ? pick(1, 20) : pick(100, 700);
    const int longest = pick(0, 2) ? 300 : 9000;
    std::vector<int32_t> p(n), few(n), kv(n), keep(n);
    for (int b = 0; b < n; ++b) {
      p[b] = pick(0, 4) ? pick(0, longest) : 0;
      few[b] = pick(0, pick(0, 1) ? 9 : 70);
      kv[b] = pick(1, longest);
      keep[b] = pick(0, 1) ? pick(0, kv[b]) : std::min(kv[b], pick(0, 3));
    }
    check_units(TIDE_OP_KV4_DECODE, kv, kv, d);
    check_units(TIDE_OP_KV4_EXTEND, p, few, d);
    check_evict(kv, keep, d);
  }
  printf("ok %d\n", calls);
  return 0;
}
