// Host-side checker of the plans of the 4-bit cache, attention mass and eviction (plan.cpp): over random
// calls, the work lists cover every position once, stay inside their regions and describe each unit.
// Prints "ok <calls>", or what is wrong.
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <map>
#include <random>
#include <vector>

#include "plan.h"

using namespace tide;

#define CHECK(x)                                                             \
  do {                                                                       \
    if (!(x)) {                                                              \
      printf("line %d: %s (call %d)\n", __LINE__, #x, g_call);                \
      exit(1);                                                               \
    }                                                                        \
  } while (0)

static int g_call = 0;

static void check_store(const std::vector<int32_t>& p, const std::vector<int32_t>& e, const tide_dims& d) {
  Plan plan;
  CHECK(make_plan_kv4_store((int)p.size(), p.data(), e.data(), d, -1, true, &plan) == TIDE_OK);
  Plan sized;
  CHECK(make_plan_kv4_store((int)p.size(), p.data(), e.data(), d, -1, false, &sized) == TIDE_OK);
  CHECK(sized.total_bytes == plan.total_bytes && sized.num_items == plan.num_items);
  CHECK(plan.blob.size() == plan.upload_bytes);
  const Kv4StoreItem* it = reinterpret_cast<const Kv4StoreItem*>(plan.blob.data() + plan.items_off);
  int64_t row = 0;
  int k = 0;
  for (size_t b = 0; b < p.size(); ++b)
    for (int32_t pos = p[b]; pos < p[b] + e[b]; ++k) {
      CHECK(k < plan.num_items);
      const int s0 = it[k].span & 31, n = it[k].span >> 5;
      CHECK(it[k].task == (int)b && it[k].lpage == pos / kPage && s0 == pos % kPage && it[k].row0 == row);
      CHECK(n >= 1 && s0 + n <= kPage && pos + n <= p[b] + e[b]);
      pos += n;
      row += n;
    }
  CHECK(k == plan.num_items && row == plan.total_rows);
}

static void check_units(int op, const std::vector<int32_t>& a, const std::vector<int32_t>& e, const tide_dims& d) {
  Plan plan, sized;
  const int n = (int)a.size();
  CHECK(make_plan_kv4_units(op, n, a.data(), e.data(), d, -1, true, &plan) == TIDE_OK);
  CHECK(make_plan_kv4_units(op, n, a.data(), e.data(), d, -1, false, &sized) == TIDE_OK);
  CHECK(sized.total_bytes == plan.total_bytes);
  if (plan.num_items == 0) return;
  CHECK(plan.blob.size() == plan.upload_bytes && plan.tickets_off <= plan.upload_bytes);
  const int group = d.num_q_heads / d.num_kv_heads;
  const TaskDesc* u = reinterpret_cast<const TaskDesc*>(plan.blob.data() + plan.tasks_off);
  const Kv4Run* r = reinterpret_cast<const Kv4Run*>(plan.blob.data() + plan.items_off);
  // units: the query rows in order, their positions and block-table rows
  int k = 0;
  int64_t row = 0;
  std::vector<int64_t> first(plan.num_tasks);  // step before the unit
  int64_t steps = 0;
  for (int b = 0; b < n; ++b) {
    const int prefix = op == TIDE_OP_KV4_DECODE ? a[b] - 1 : a[b], ext = op == TIDE_OP_KV4_DECODE ? 1 : e[b];
    for (int t = 0; t < ext; ++k) {
      CHECK(k < plan.num_tasks);
      CHECK(u[k].row_start == row && u[k].prefix == prefix + t && u[k].aux == b && u[k].extend >= 1);
      CHECK(u[k].extend * group <= kKv4Cols && u[k].extend <= plan.tokens_per_item && t + u[k].extend <= ext);
      if (u[k].extend < ext) CHECK(plan.reread);
      first[k] = steps;
      steps += (u[k].prefix + u[k].extend + kDecodeStep - 1) / kDecodeStep;
      t += u[k].extend;
      row += u[k].extend;
    }
  }
  CHECK(k == plan.num_tasks);
  // runs: equal, in order, the last one shorter
  CHECK((int64_t)(plan.num_runs - 1) * plan.steps + plan.last_steps == steps);
  CHECK(plan.last_steps >= 1 && plan.last_steps <= plan.steps);
  for (int i = 0; i < plan.num_runs; ++i) {
    const int64_t at = (int64_t)i * plan.steps;
    const int x = r[i].unit;
    CHECK(x >= 0 && x < plan.num_tasks && r[i].step >= 0 && first[x] + r[i].step == at);
    CHECK(at < (x + 1 < plan.num_tasks ? first[x + 1] : steps));
    CHECK(memcmp(&r[i].desc, &u[x], sizeof(TaskDesc)) == 0);
  }
  // partial slots: distinct for the parts of different units, inside the region
  const StreamSlots slots = {plan.num_runs, plan.num_tasks, kv4_waves(plan.num_items)};
  std::map<int32_t, int> owner;
  for (int x = 0; x < plan.num_tasks; ++x) {
    const int64_t end = x + 1 < plan.num_tasks ? first[x + 1] : steps;
    const int32_t total = (int32_t)(end - first[x]);
    const int32_t w = (int32_t)(first[x] / plan.steps);
    const int64_t run_end = std::min<int64_t>(steps, (int64_t)(w + 1) * plan.steps);
    if (end <= run_end && total < plan.steps) continue;  // inside one run
    const StreamUnit unit = stream_unit(w, 0, (int32_t)(std::min(end, run_end) - first[x]), total, plan.steps);
    for (int32_t p = 0; p < stream_parts(unit, slots.per); ++p) {
      const int32_t s = stream_slot(unit, slots, x, p);
      if (stream_parts(unit, slots.per) == 1) break;  // combined inside a workgroup
      CHECK(s >= 0 && s < slots.count());
      CHECK(owner.emplace(s, x).second);
    }
  }
  const int64_t bytes = (int64_t)slots.count() * d.num_kv_heads * plan.tokens_per_item * group * (d.head_dim + 4) * 4;
  CHECK((int64_t)plan.part_o_off + bytes <= (int64_t)plan.total_bytes + 512);
}

static void check_extend(const std::vector<int32_t>& p, const std::vector<int32_t>& e, const tide_dims& d) {
  Kv4ExtendPlan plan, sized;
  const int n = (int)p.size();
  CHECK(make_plan_kv4_extend(n, p.data(), e.data(), d, -1, true, &plan) == TIDE_OK);
  CHECK(make_plan_kv4_extend(n, p.data(), e.data(), d, -1, false, &sized) == TIDE_OK);
  CHECK(sized.total_bytes == plan.total_bytes && sized.by_units == plan.by_units);
  if (plan.by_units) return;
  int next = 0;
  int64_t row = 0;
  for (const Kv4Round& r : plan.rounds) {
    for (; next < r.first; ++next) CHECK(e[next] == 0);
    CHECK(r.row0 == row);
    const Kv4StageItem* it = reinterpret_cast<const Kv4StageItem*>(r.stage.blob.data() + r.stage.items_off);
    int k = 0;
    int64_t to = 0;
    for (int b = r.first; b < r.first + r.tasks; ++b) {
      const int pages = e[b] ? (p[b] + e[b] + kPage - 1) / kPage : 0;
      CHECK(pages <= r.stride);
      for (int lp = 0; lp < pages; ++k) {
        CHECK(k < r.stage.num_items);
        CHECK(it[k].row == b && it[k].task == b - r.first && it[k].lpage == lp && it[k].to == to);
        CHECK(it[k].pages >= 1 && it[k].pages <= 16 && lp + it[k].pages <= pages);
        lp += it[k].pages;
        to += it[k].pages;
      }
      row += e[b];
    }
    CHECK(k == r.stage.num_items && to == r.pages);
    CHECK(r.extend.total_bytes <= plan.table_off - plan.extend_off);
    CHECK(r.stage.total_bytes <= plan.extend_off - plan.stage_off);
    CHECK((size_t)r.tasks * r.stride * 4 <= plan.pool_off - plan.table_off);
    CHECK(plan.pool_off + (size_t)r.pages * d.num_kv_heads * kPage * d.head_dim * 4 <= plan.total_bytes);
    next = r.first + r.tasks;
  }
  for (; next < n; ++next) CHECK(e[next] == 0);
}

static void check_mass(const std::vector<int32_t>& p, const std::vector<int32_t>& e, const tide_dims& d) {
  Plan plan, sized;
  const int n = (int)p.size();
  CHECK(make_plan_mass(n, p.data(), e.data(), nullptr, d, -1, true, &plan) == TIDE_OK);
  CHECK(make_plan_mass(n, p.data(), e.data(), nullptr, d, -1, false, &sized) == TIDE_OK);
  CHECK(sized.total_bytes == plan.total_bytes && plan.blob.size() == plan.upload_bytes);
  const MassRun* r = reinterpret_cast<const MassRun*>(plan.blob.data() + plan.items_off);
  int b = 0, k = 0, i = 0;
  int64_t inside = 0;
  auto blocks = [&](int x) { return e[x] ? (p[x] + e[x] + kMassKeys - 1) / kMassKeys : 0; };
  for (; b < n; ++b)
    for (k = 0; k < blocks(b); ++k) {
      if (inside == 0) {
        CHECK(i < plan.num_runs && r[i].task == b && r[i].block == k && r[i].blocks >= 1);
        inside = r[i++].blocks;
      }
      --inside;
    }
  CHECK(inside == 0 && i == plan.num_runs);
  CHECK((int64_t)plan.num_runs <= std::max<int64_t>(1, 4096 / d.num_kv_heads));
}

static void check_evict(const std::vector<int32_t>& n, const std::vector<int32_t>& keep, const std::vector<int32_t>& rec,
                        const tide_dims& d) {
  Plan plan;
  CHECK(make_plan_evict((int)n.size(), n.data(), keep.data(), rec.data(), d, -1, -1, true, &plan) == TIDE_OK);
  const EvictTask* t = reinterpret_cast<const EvictTask*>(plan.blob.data() + plan.tasks_off);
  int64_t rows = 0;
  int k = 0;
  for (size_t b = 0; b < n.size(); ++b) {
    if (keep[b]) {
      CHECK(t[k].task == (int)b && t[k].kv_len == n[b] && t[k].keep == keep[b] && t[k].recent == rec[b] && t[k].first == rows);
      ++k;
    }
    rows += keep[b];
  }
  CHECK(k == plan.num_tasks);
  CHECK(plan.items_off + (size_t)rows * d.num_kv_heads * sizeof(EvictIndex) <= plan.total_bytes);
  CHECK(plan.part_o_off + plan.num_tasks * sizeof(EvictTask) <= plan.items_off);
}

int main(int argc, char** argv) {
  const int calls = argc > 1 ? atoi(argv[1]) : 300;
  std::mt19937 rng(7);
  auto pick = [&](int lo, int hi) { return (int)std::uniform_int_distribution<int>(lo, hi)(rng); };
  const int heads[][2] = {{1, 1}, {28, 4}, {32, 8}, {16, 1}, {5, 5}, {2500, 2500}, {64, 8}};
  for (g_call = 0; g_call < calls; ++g_call) {
    const auto& h = heads[pick(0, 6)];
    const tide_dims d = {h[0], h[1], pick(0, 1) ? 64 : 128, kPage, 0.1f};
    const int n = pick(0, 3) ? pick(1, 20) : pick(100, 700);
    const int longest = pick(0, 2) ? 300 : 9000;
    std::vector<int32_t> p(n), e(n), few(n), kv(n), keep(n), rec(n);
    for (int b = 0; b < n; ++b) {
      p[b] = pick(0, 4) ? pick(0, longest) : 0;
      e[b] = pick(0, 4) ? pick(0, pick(0, 1) ? 40 : 700) : 0;
      few[b] = pick(0, 9);
      kv[b] = pick(1, longest);
      keep[b] = pick(0, kv[b]);
      rec[b] = pick(0, keep[b]);
    }
    check_store(p, e, d);
    check_units(TIDE_OP_KV4_DECODE, kv, kv, d);
    check_units(TIDE_OP_KV4_EXTEND, p, few, d);
    check_extend(p, e, d);
    check_extend(p, few, d);
    check_mass(p, e, d);
    check_evict(kv, keep, rec, d);
  }
  printf("ok %d\n", calls);
  return 0;
}
