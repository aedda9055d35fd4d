// Host-side planning for the entry points: argument validation, workspace layout and the
// per-call work lists.  Plain C++ (no HIP); the entry points in tide_api.hip stage the blob
// it builds.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include <vector>

#include "tide.h"
#include "tide_common.h"

namespace tide {

// Where each region lives inside the caller's workspace (byte offsets).
struct Plan {
  int op = 0;
  int32_t num_tasks = 0;
  // upload region [0, upload_bytes): header, task table, items
  size_t tasks_off = 0;
  size_t items_off = 0;
  size_t upload_bytes = 0;
  // extend split-KV plan: per-row merge descriptors (uploaded after the items)
  bool split = false;
  size_t merge_rows_off = 0;
  // decode, at the blob's end, zeros in it.  Chunks: arrival counters per (task, kv head), used
  // when the split kernel merges (fold_merge: few splits per task) instead of a merge kernel.
  // Runs (`stream`): a flag per partial slot, set to the call's own number, so the zeros do not
  // matter where the plan is read in place and never copied.
  size_t tickets_off = 0;
  bool fold_merge = false;
  // decode with the library's own split (make_plan_decode): StreamItems, one per run
  bool stream = false;
  int32_t num_runs = 0;
  int32_t steps = 0;       // key steps per run
  int32_t last_steps = 0;  // of the last run
  int64_t row_slots = 0;  // partial row slots (each holds every query head)
  // the planner's run-time estimates (microseconds) of the plain and chosen extend plans;
  // 0 when the call was too large to consider splitting
  double est_plain_us = 0.0;
  double est_us = 0.0;
  // decode and split-extend partials (not uploaded)
  size_t part_o_off = 0;
  size_t part_ml_off = 0;
  size_t total_bytes = 0;
  int32_t num_items = 0;
  // extend: tokens per work item and waves per workgroup
  int32_t tokens_per_item = 0;
  int32_t waves = 0;
  bool reread = false;    // 4-bit attention: some task has several units
  bool one_trip = false;  // attention mass: no task has over 16 query rows a kv head
  // extend: passes over the blocks that the search for the chunk length made
  int32_t search_passes = 0;
  int32_t chunk = 0;  // decode: keys per chunk or run; split extend: most key tiles per chunk
  // decode
  int32_t max_splits = 0;
  int32_t total_rows = 0;
  std::vector<uint8_t> blob;  // bytes to upload (header + tasks + items)
};

// Shape validation shared by every entry point.
int check_dims(const tide_dims* dims);

// Validates lengths and builds the plan.  When `build_blob` is false only the sizes are
// computed (tide_workspace_size).  `bt_stride` < 0 skips the block-table capacity check.
int make_plan(int op, int32_t num_tasks, const int32_t* lens_a, const int32_t* lens_b,
              const tide_dims& dims, int32_t num_splits, int32_t bt_stride, bool build_blob,
              Plan* plan);

// Decode: runs of equal length when the library chooses the split (num_splits == 0) and the call's
// steps can be counted in 32 bits, else the chunk plan of make_plan.
int make_plan_decode(int32_t num_tasks, const int32_t* kv_lens, const tide_dims& dims,
                     int32_t num_splits, int32_t bt_stride, bool build_blob, Plan* plan);

// The runs of a decode plan as one int32 each, the task a run starts in, in place of the
// StreamItems; the task table then holds each task's first step (aux), from which the rest
// follows.  Returns the bytes of the blob up to their end.
size_t compact_runs(Plan* plan);

// Shared-prefix decode: groups are consecutive task ranges [group_start[g],
// group_start[g+1]); the first shared_lens[g] keys (a multiple of the page size, below
// every member's kv_len) live in pages every member's block table shares.
constexpr int kOpDecodeShared = 100;  // internal op code of the plan
int make_plan_shared(int32_t num_tasks, const int32_t* kv_lens, int32_t num_groups,
                     const int32_t* group_start, const int32_t* shared_lens,
                     const tide_dims& dims, int32_t num_splits, int32_t bt_stride,
                     bool build_blob, Plan* plan);

// ---- the 4-bit cache, attention mass, eviction ----------------------------------------------
// Append and unpack: Kv4StoreItems.
int make_plan_kv4_store(int32_t num_tasks, const int32_t* prefix_lens, const int32_t* extend_lens,
                        const tide_dims& dims, int32_t bt_stride, bool build_blob, Plan* plan);

// Runs of steps over units of up to kKv4Cols / G query tokens each (Kv4AttnArgs).  lens_a, lens_b as
// TIDE_OP_KV4_DECODE or TIDE_OP_KV4_EXTEND take them.
int make_plan_kv4_units(int op, int32_t num_tasks, const int32_t* lens_a, const int32_t* lens_b,
                        const tide_dims& dims, int32_t bt_stride, bool build_blob, Plan* plan);

// An extend over the 4-bit cache: by units, or by rounds of consecutive tasks whose pages are
// unpacked into a staging area of the workspace that the bf16 extend kernel reads.
struct Kv4Round {
  int32_t first = 0, tasks = 0;  // consecutive tasks
  int64_t row0 = 0;              // the first one's packed row
  Plan stage;                    // Kv4StageItems
  Plan extend;
  int32_t stride = 0;            // of the staging block table
  int64_t pages = 0;             // staged
};

struct Kv4ExtendPlan {
  bool by_units = false;
  Plan units;
  std::vector<Kv4Round> rounds;
  // byte offsets of a round's parts (the rounds follow each other in the same bytes)
  size_t stage_off = 0, extend_off = 0, table_off = 0, pool_off = 0;
  size_t total_bytes = 0;
};

int make_plan_kv4_extend(int32_t num_tasks, const int32_t* prefix_lens, const int32_t* extend_lens,
                         const tide_dims& dims, int32_t bt_stride, bool build_blob, Kv4ExtendPlan* plan);

// Attention mass: MassRuns.  counted: positions per task whose sums are carried on (null: prefix).
int make_plan_mass(int32_t num_tasks, const int32_t* prefix_lens, const int32_t* extend_lens,
                   const int32_t* counted, const tide_dims& dims, int32_t bt_stride, bool build_blob, Plan* plan);

// Eviction: EvictTasks (at tasks_off, room for a copy at part_o_off); the index at items_off.  recent may be
// null (0 everywhere); new_stride < 0: the new pages' capacity is not checked.
int make_plan_evict(int32_t num_tasks, const int32_t* kv_lens, const int32_t* keep_lens, const int32_t* recent,
                    const tide_dims& dims, int32_t bt_stride, int32_t new_stride, bool build_blob, Plan* plan);

// Waves per workgroup of the extend kernel for a head size and GQA group.
int32_t extend_waves(int32_t head_dim, int32_t group);

inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

}  // namespace tide
