// The extern "C" entry points of the 4-bit cache, of attention mass and of eviction
// (include/tide.h): checks, plans (plan.cpp), staging (staging.h) and launches.
#include <hip/hip_runtime.h>

#include "kernels.h"
#include "staging.h"
#include "tide.h"

namespace tide {
namespace {

// Device buffers are read and written 16 bytes at a time.
bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// Checks that every entry point starts with.  *go: there is something to do.
int start(const tide_dims* dims, int32_t num_tasks, int64_t num_pages, int32_t bt_stride, bool* go) {
  *go = false;
  const int rc = check_dims(dims);
  if (rc != TIDE_OK) return rc;
  if (num_tasks < 0) return TIDE_ERR_INVALID_ARG;
  if (num_tasks == 0) return TIDE_OK;
  if (num_pages <= 0 || bt_stride <= 0) return TIDE_ERR_INVALID_ARG;
  *go = true;
  return TIDE_OK;
}

int store(bool append, const void* k, const void* v, void* pool, int64_t num_pages, const int32_t* block_table,
          int32_t bt_stride, int32_t num_tasks, const int32_t* prefix_lens, const int32_t* extend_lens,
          const tide_dims* dims, void* workspace, size_t workspace_bytes, void* stream) {
  bool go;
  int rc = start(dims, num_tasks, num_pages, bt_stride, &go);
  if (rc != TIDE_OK || !go) return rc;
  Plan plan;
  rc = make_plan_kv4_store(num_tasks, prefix_lens, extend_lens, *dims, bt_stride, true, &plan);
  if (rc != TIDE_OK) return rc;
  if (plan.num_items == 0) return TIDE_OK;
  if (!k || !v || !pool || !block_table || !workspace) return TIDE_ERR_INVALID_ARG;
  if (!aligned16(k) || !aligned16(v) || !aligned16(pool) || !aligned16(workspace)) return TIDE_ERR_INVALID_ARG;
  if (workspace_bytes < plan.total_bytes) return TIDE_ERR_CAPACITY;
  hipStream_t s = static_cast<hipStream_t>(stream);
  Staged st;
  const int64_t groups = (int64_t)plan.num_items * kv4_store_groups(dims->num_kv_heads);
  rc = upload(plan, workspace, s, groups <= kInPlaceGroups ? (uint32_t)groups : 0, &st);
  if (rc != TIDE_OK) return rc;
  Kv4StoreArgs a = {};
  a.reads = st.reads;
  if (append) {
    a.k_new = static_cast<const uint16_t*>(k);
    a.v_new = static_cast<const uint16_t*>(v);
  } else {
    a.k_out = static_cast<uint16_t*>(const_cast<void*>(k));
    a.v_out = static_cast<uint16_t*>(const_cast<void*>(v));
  }
  a.pool = static_cast<uint8_t*>(pool);
  a.block_table = block_table;
  a.num_pages = num_pages;
  a.bt_stride = bt_stride;
  a.num_kv_heads = dims->num_kv_heads;
  a.head_dim = dims->head_dim;
  a.num_items = plan.num_items;
  a.items = at<Kv4StoreItem>(st.plan, plan.items_off);
  a.error_flags = at_mut<int32_t>(workspace, 0);
  return finish(launch_kv4_store(a, s), st, workspace, s);
}

// Attention of a plan of units (decode, with the append of one token a task where k_new is set, and
// extends of a few tokens).
int attend_units(const Plan& plan, const void* q, const void* k_new, const void* v_new, void* pool,
                 int64_t num_pages, const int32_t* block_table, int32_t bt_stride, const tide_dims& dims, void* out,
                 float* lse, void* workspace, hipStream_t s) {
  Staged st;
  // a wave reads the units again where its run crosses into the next one, so a call with more
  // units than runs keeps the copy
  const uint32_t readers =
      plan.num_tasks <= plan.num_runs ? kv4_groups(plan.num_runs, dims.num_kv_heads) : 0;
  const int rc = upload(plan, workspace, s, readers, &st);
  if (rc != TIDE_OK) return rc;
  Kv4AttnArgs a = {};
  a.q = static_cast<const uint16_t*>(q);
  a.pool = static_cast<uint8_t*>(pool);
  a.block_table = block_table;
  a.num_pages = num_pages;
  a.bt_stride = bt_stride;
  a.num_q_heads = dims.num_q_heads;
  a.num_kv_heads = dims.num_kv_heads;
  a.group = dims.num_q_heads / dims.num_kv_heads;
  a.cols = plan.tokens_per_item * a.group;
  a.scale_log2 = dims.sm_scale * 1.44269504088896340736f;
  a.num_runs = plan.num_runs;
  a.steps = plan.steps;
  a.last_steps = plan.last_steps;
  a.units = at<TaskDesc>(st.plan, plan.tasks_off);
  a.runs = at<Kv4Run>(st.plan, plan.items_off);
  a.num_units = plan.num_tasks;
  a.reread = plan.reread;
  a.part_o = at_mut<float>(workspace, plan.part_o_off);
  a.part_ml = at_mut<float>(workspace, plan.part_ml_off);
  a.flags = at_mut<uint64_t>(workspace, plan.tickets_off);
  a.call = next_call();
  a.out = static_cast<uint16_t*>(out);
  a.lse = lse;
  a.error_flags = at_mut<int32_t>(workspace, 0);
  a.k_new = static_cast<const uint16_t*>(k_new);
  a.v_new = static_cast<const uint16_t*>(v_new);
  a.reads = st.reads;
  return finish(launch_kv4_decode(a, dims.head_dim, s), st, workspace, s);
}

int decode(const void* q, const void* k_new, const void* v_new, bool append, void* pool, int64_t num_pages,
           const int32_t* block_table, int32_t bt_stride, int32_t num_tasks, const int32_t* kv_lens,
           const tide_dims* dims, void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  bool go;
  int rc = start(dims, num_tasks, num_pages, bt_stride, &go);
  if (rc != TIDE_OK || !go) return rc;
  Plan plan;
  rc = make_plan_kv4_units(TIDE_OP_KV4_DECODE, num_tasks, kv_lens, nullptr, *dims, bt_stride, true, &plan);
  if (rc != TIDE_OK) return rc;
  if (!q || !pool || !block_table || !out || !workspace) return TIDE_ERR_INVALID_ARG;
  if (append && (!k_new || !v_new)) return TIDE_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(pool) || !aligned16(out) || !aligned16(workspace) || !aligned16(k_new) ||
      !aligned16(v_new))
    return TIDE_ERR_INVALID_ARG;
  if (workspace_bytes < plan.total_bytes) return TIDE_ERR_CAPACITY;
  return attend_units(plan, q, append ? k_new : nullptr, append ? v_new : nullptr, pool, num_pages, block_table,
                      bt_stride, *dims, out, lse, workspace, static_cast<hipStream_t>(stream));
}

int mass(const void* q, const float* lse, const void* pool, bool kv4, int64_t num_pages, const int32_t* block_table,
         int32_t bt_stride, int32_t num_tasks, const int32_t* prefix_lens, const int32_t* extend_lens,
         const int32_t* counted_lens, const tide_dims* dims, float* sums, void* workspace, size_t workspace_bytes,
         void* stream) {
  bool go;
  int rc = start(dims, num_tasks, num_pages, bt_stride, &go);
  if (rc != TIDE_OK || !go) return rc;
  Plan plan;
  rc = make_plan_mass(num_tasks, prefix_lens, extend_lens, counted_lens, *dims, bt_stride, true, &plan);
  if (rc != TIDE_OK) return rc;
  if (plan.num_items == 0) return TIDE_OK;
  if (!q || !lse || !pool || !block_table || !sums || !workspace) return TIDE_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(pool) || !aligned16(sums) || !aligned16(workspace)) return TIDE_ERR_INVALID_ARG;
  if (workspace_bytes < plan.total_bytes) return TIDE_ERR_CAPACITY;
  hipStream_t s = static_cast<hipStream_t>(stream);
  Staged st;
  const uint32_t readers =
      num_tasks <= plan.num_runs ? mass_groups(plan.num_runs, dims->num_kv_heads, plan.one_trip) : 0;
  rc = upload(plan, workspace, s, readers, &st);
  if (rc != TIDE_OK) return rc;
  MassArgs a = {};
  a.q = static_cast<const uint16_t*>(q);
  a.lse = lse;
  a.pool = pool;
  a.block_table = block_table;
  a.num_pages = num_pages;
  a.bt_stride = bt_stride;
  a.num_q_heads = dims->num_q_heads;
  a.num_kv_heads = dims->num_kv_heads;
  a.group = dims->num_q_heads / dims->num_kv_heads;
  a.scale_log2 = dims->sm_scale * 1.44269504088896340736f;
  a.num_runs = plan.num_runs;
  a.one_trip = plan.one_trip;
  a.tasks = at<TaskDesc>(st.plan, plan.tasks_off);
  a.runs = at<MassRun>(st.plan, plan.items_off);
  a.mass = sums;
  a.error_flags = at_mut<int32_t>(workspace, 0);
  a.reads = st.reads;
  return finish(launch_attn_mass(a, dims->head_dim, kv4, s), st, workspace, s);
}

int evict(void* k_pool, void* v_pool, bool kv4, float* sums, int64_t num_pages, const int32_t* block_table,
          int32_t bt_stride, const int32_t* new_table, int32_t new_stride, int32_t num_tasks, const int32_t* kv_lens,
          const int32_t* keep_lens, const int32_t* recent_lens, const tide_dims* dims, int32_t* kept, void* workspace,
          size_t workspace_bytes, void* stream) {
  bool go;
  int rc = start(dims, num_tasks, num_pages, bt_stride, &go);
  if (rc != TIDE_OK || !go) return rc;
  if (new_table && new_stride <= 0) return TIDE_ERR_INVALID_ARG;
  if (!new_table) new_table = block_table, new_stride = bt_stride;
  Plan plan;
  rc = make_plan_evict(num_tasks, kv_lens, keep_lens, recent_lens, *dims, bt_stride, new_stride, true, &plan);
  if (rc != TIDE_OK) return rc;
  if (plan.num_items == 0) return TIDE_OK;
  if (!k_pool || (!kv4 && !v_pool) || !sums || !block_table || !workspace) return TIDE_ERR_INVALID_ARG;
  if (!aligned16(k_pool) || !aligned16(v_pool) || !aligned16(sums) || !aligned16(workspace))
    return TIDE_ERR_INVALID_ARG;
  if (workspace_bytes < plan.total_bytes) return TIDE_ERR_CAPACITY;
  hipStream_t s = static_cast<hipStream_t>(stream);
  Staged st;
  const int64_t readers = (int64_t)plan.num_tasks * dims->num_kv_heads;
  rc = upload(plan, workspace, s, readers <= kInPlaceGroups ? (uint32_t)readers : 0, &st);
  if (rc != TIDE_OK) return rc;
  EvictArgs a = {};
  a.k_pool = static_cast<uint8_t*>(k_pool);
  a.v_pool = static_cast<uint8_t*>(v_pool);
  a.mass = sums;
  a.block_table = block_table;
  a.new_table = new_table;
  a.num_pages = num_pages;
  a.bt_stride = bt_stride;
  a.new_stride = new_stride;
  a.num_kv_heads = dims->num_kv_heads;
  a.num_tasks = plan.num_tasks;
  a.longest_keep = plan.chunk;
  a.tasks = at<EvictTask>(st.plan, plan.tasks_off);
  a.move_tasks = at_mut<EvictTask>(workspace, plan.part_o_off);
  a.reads = st.reads;
  a.index = at_mut<EvictIndex>(workspace, plan.items_off);
  a.kept = kept;
  a.error_flags = at_mut<int32_t>(workspace, 0);
  return finish(launch_evict(a, dims->head_dim, kv4, s), st, workspace, s);
}

}  // namespace
}  // namespace tide

using namespace tide;

extern "C" {

TIDE_API int tide_kv4_append(const void* k_new, const void* v_new, void* kv4_pool, int64_t num_pages,
                             const int32_t* block_table, int32_t bt_stride, int32_t num_tasks,
                             const int32_t* prefix_lens, const int32_t* extend_lens, const tide_dims* dims,
                             void* workspace, size_t workspace_bytes, void* stream) {
  try {
    return store(true, k_new, v_new, kv4_pool, num_pages, block_table, bt_stride, num_tasks, prefix_lens,
                 extend_lens, dims, workspace, workspace_bytes, stream);
  } catch (...) {
    return TIDE_ERR_HIP;
  }
}

TIDE_API int tide_kv4_unpack(const void* kv4_pool, int64_t num_pages, const int32_t* block_table, int32_t bt_stride,
                             int32_t num_tasks, const int32_t* prefix_lens, const int32_t* extend_lens,
                             const tide_dims* dims, void* k_out, void* v_out, void* workspace,
                             size_t workspace_bytes, void* stream) {
  try {
    return store(false, k_out, v_out, const_cast<void*>(kv4_pool), num_pages, block_table, bt_stride, num_tasks,
                 prefix_lens, extend_lens, dims, workspace, workspace_bytes, stream);
  } catch (...) {
    return TIDE_ERR_HIP;
  }
}

TIDE_API int tide_kv4_decode_attn(const void* q, const void* kv4_pool, int64_t num_pages, const int32_t* block_table,
                                  int32_t bt_stride, int32_t num_tasks, const int32_t* kv_lens,
                                  const tide_dims* dims, void* out, float* lse, void* workspace,
                                  size_t workspace_bytes, void* stream) {
  try {
    return decode(q, nullptr, nullptr, false, const_cast<void*>(kv4_pool), num_pages, block_table, bt_stride,
                  num_tasks, kv_lens, dims, out, lse, workspace, workspace_bytes, stream);
  } catch (...) {
    return TIDE_ERR_HIP;
  }
}

TIDE_API int tide_kv4_decode_append_attn(const void* q, const void* k_new, const void* v_new, void* kv4_pool,
                                         int64_t num_pages, const int32_t* block_table, int32_t bt_stride,
                                         int32_t num_tasks, const int32_t* kv_lens, const tide_dims* dims, void* out,
                                         float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  try {
    return decode(q, k_new, v_new, true, kv4_pool, num_pages, block_table, bt_stride, num_tasks, kv_lens, dims, out,
                  lse, workspace, workspace_bytes, stream);
  } catch (...) {
    return TIDE_ERR_HIP;
  }
}

TIDE_API int tide_kv4_extend_attn(const void* q, const void* kv4_pool, int64_t num_pages, const int32_t* block_table,
                                  int32_t bt_stride, int32_t num_tasks, const int32_t* prefix_lens,
                                  const int32_t* extend_lens, const tide_dims* dims, void* out, float* lse,
                                  void* workspace, size_t workspace_bytes, void* stream) {
  try {
    bool go;
    int rc = start(dims, num_tasks, num_pages, bt_stride, &go);
    if (rc != TIDE_OK || !go) return rc;
    Kv4ExtendPlan plan;
    rc = make_plan_kv4_extend(num_tasks, prefix_lens, extend_lens, *dims, bt_stride, true, &plan);
    if (rc != TIDE_OK) return rc;
    if (plan.by_units ? plan.units.num_items == 0 : plan.rounds.empty()) return TIDE_OK;
    if (!q || !kv4_pool || !block_table || !out || !workspace) return TIDE_ERR_INVALID_ARG;
    if (!aligned16(q) || !aligned16(kv4_pool) || !aligned16(out) || !aligned16(workspace)) return TIDE_ERR_INVALID_ARG;
    if (workspace_bytes < plan.total_bytes) return TIDE_ERR_CAPACITY;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (plan.by_units)
      return attend_units(plan.units, q, nullptr, nullptr, const_cast<void*>(kv4_pool), num_pages, block_table,
                          bt_stride, *dims, out, lse, workspace, s);
    for (const Kv4Round& r : plan.rounds) {
      const int64_t pool_elems = r.pages * dims->num_kv_heads * kPage * dims->head_dim;
      uint16_t* k_stage = at_mut<uint16_t>(workspace, plan.pool_off);
      uint16_t* v_stage = k_stage + pool_elems;
      int32_t* table = at_mut<int32_t>(workspace, plan.table_off);
      void* stage_ws = at_mut<uint8_t>(workspace, plan.stage_off);
      {
        Staged st;
        rc = upload(r.stage, stage_ws, s, (uint32_t)r.stage.num_items, &st);
        if (rc != TIDE_OK) return rc;
        Kv4StageArgs a = {};
        a.reads = st.reads;
        a.pool = static_cast<const uint8_t*>(kv4_pool);
        a.block_table = block_table;
        a.num_pages = num_pages;
        a.bt_stride = bt_stride;
        a.num_kv_heads = dims->num_kv_heads;
        a.head_dim = dims->head_dim;
        a.num_items = r.stage.num_items;
        a.items = at<Kv4StageItem>(st.plan, r.stage.items_off);
        a.k_stage = k_stage;
        a.v_stage = v_stage;
        a.stage_table = table;
        a.stage_stride = r.stride;
        a.error_flags = at_mut<int32_t>(stage_ws, 0);
        rc = finish(launch_kv4_stage(a, s), st, stage_ws, s);
        if (rc != TIDE_OK) return rc;
      }
      const int64_t row = r.row0 * dims->num_q_heads;
      rc = run_extend_plan(r.extend, static_cast<const uint16_t*>(q) + row * dims->head_dim, k_stage, v_stage,
                           r.pages, table, r.stride, *dims, static_cast<uint16_t*>(out) + row * dims->head_dim,
                           lse ? lse + row : nullptr, at_mut<uint8_t>(workspace, plan.extend_off), s, nullptr, nullptr);
      if (rc != TIDE_OK) return rc;
    }
    return TIDE_OK;
  } catch (...) {
    return TIDE_ERR_HIP;
  }
}

TIDE_API int tide_attn_mass(const void* q, const float* lse, const void* k_pool, int64_t num_pages,
                            const int32_t* block_table, int32_t bt_stride, int32_t num_tasks,
                            const int32_t* prefix_lens, const int32_t* extend_lens, const int32_t* counted_lens,
                            const tide_dims* dims, float* mass_pool, void* workspace, size_t workspace_bytes,
                            void* stream) {
  try {
    return mass(q, lse, k_pool, false, num_pages, block_table, bt_stride, num_tasks, prefix_lens, extend_lens,
                counted_lens, dims, mass_pool, workspace, workspace_bytes, stream);
  } catch (...) {
    return TIDE_ERR_HIP;
  }
}

TIDE_API int tide_kv4_attn_mass(const void* q, const float* lse, const void* kv4_pool, int64_t num_pages,
                                const int32_t* block_table, int32_t bt_stride, int32_t num_tasks,
                                const int32_t* prefix_lens, const int32_t* extend_lens, const int32_t* counted_lens,
                                const tide_dims* dims, float* mass_pool, void* workspace, size_t workspace_bytes,
                                void* stream) {
  try {
    return mass(q, lse, kv4_pool, true, num_pages, block_table, bt_stride, num_tasks, prefix_lens, extend_lens,
                counted_lens, dims, mass_pool, workspace, workspace_bytes, stream);
  } catch (...) {
    return TIDE_ERR_HIP;
  }
}

TIDE_API int tide_kv_evict(void* k_pool, void* v_pool, float* mass_pool, int64_t num_pages,
                           const int32_t* block_table, int32_t bt_stride, const int32_t* new_block_table,
                           int32_t new_bt_stride, int32_t num_tasks, const int32_t* kv_lens,
                           const int32_t* keep_lens, const int32_t* recent_lens, const tide_dims* dims, int32_t* kept,
                           void* workspace, size_t workspace_bytes, void* stream) {
  try {
    return evict(k_pool, v_pool, false, mass_pool, num_pages, block_table, bt_stride, new_block_table, new_bt_stride,
                 num_tasks, kv_lens, keep_lens, recent_lens, dims, kept, workspace, workspace_bytes, stream);
  } catch (...) {
    return TIDE_ERR_HIP;
  }
}

TIDE_API int tide_kv4_evict(void* kv4_pool, float* mass_pool, int64_t num_pages, const int32_t* block_table,
                            int32_t bt_stride, const int32_t* new_block_table, int32_t new_bt_stride,
                            int32_t num_tasks, const int32_t* kv_lens, const int32_t* keep_lens,
                            const int32_t* recent_lens, const tide_dims* dims, int32_t* kept, void* workspace,
                            size_t workspace_bytes, void* stream) {
  try {
    return evict(kv4_pool, nullptr, true, mass_pool, num_pages, block_table, bt_stride, new_block_table,
                 new_bt_stride, num_tasks, kv_lens, keep_lens, recent_lens, dims, kept, workspace, workspace_bytes,
                 stream);
  } catch (...) {
    return TIDE_ERR_HIP;
  }
}

}  // extern "C"
