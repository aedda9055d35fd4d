// Definitions shared by the host planner and the gfx950 kernels: the work-item records
// uploaded into the caller's workspace, and the kernel argument blocks.
#pragma once

#include <stdint.h>

#ifdef __HIPCC__
#define TIDE_HD __host__ __device__
#else
#define TIDE_HD
#endif

namespace tide {

constexpr int kPage = 16;         // tokens per page
constexpr int kMaxGroup = 16;     // largest supported Hq / Hkv
// Largest supported Hkv: a pool page (Hkv blocks of kPage rows of head_dim bf16) then
// spans at most 2^28 bytes, which the extend kernel's 32-bit page stride holds.
constexpr int kMaxKvHeads = 65536;
constexpr int kExtendKeyTile = 64;  // keys per extend-kernel iteration (4 pages)
constexpr int kDecodeStep = 32;   // keys per decode-kernel iteration (2 pages)
constexpr int kWsAlign = 256;
constexpr int kXcds = 8;          // MI355X: 8 accelerator dies, one L2 each

// One task as the kernels see it.  `row_start` indexes the packed token rows of Q/O
// (extend, prefill) or the task itself (decode); tokens at positions
// [prefix, prefix + extend) are the ones this call processes.
struct TaskDesc {
  int32_t row_start;
  int32_t prefix;
  int32_t extend;
  int32_t aux;  // decode: number of splits of this task; append: first new-row index
};

// Extend / prefill work item: tokens [tok0, tok0 + ntok) of `task` (relative to its
// prefix) for every query head that reads kv head `kv_head`.
struct ExtendItem {
  int32_t task;
  int32_t kv_head;
  int32_t tok0;
  int32_t ntok;
};

// Extend / prefill work item of the split-KV plan, used when a call has too few items
// to fill the chip: key tiles [t_begin, t_end) of the item (64 keys each, counted from
// key 0).  split >= 0: one of the item's chunks; its unnormalised partial for row slot
// s = pbase + split * ntok + tk (tk = token inside the item) and query head h goes to
// part_o[(s * Hq + h) * d] and part_ml[(s * Hq + h) * 4], and a merge combines the
// chunks.  split == -1: the item is not split and writes its output directly.
struct ExtendChunkItem {
  int32_t task;
  int32_t kv_head;
  int32_t tok0;
  int32_t ntok;
  int32_t t_begin;
  int32_t t_end;
  int32_t split;
  int32_t pbase;
};

// Merge descriptor of one packed extend row: its partials sit in row slots base,
// base + stride, ..., base + (nsplit - 1) * stride; nsplit == 0 means the row was
// written directly and has nothing to merge.
struct MergeRow {
  int32_t base;
  int32_t stride;
  int32_t nsplit;
  int32_t pad;
};

// Decode split-K item: keys [k_begin, min(kv_len, k_begin + chunk)) of one (task, kv head).
struct DecodeItem {
  int32_t task;
  int32_t kv_head;
  int32_t split;
  int32_t k_begin;
};

// Decode work of one run when the split count is left to the library: the tasks' 32-key
// steps, laid end to end, are cut into equal runs, and one wave per kv head takes the run
// that starts at `step` of `task` and may cross into the next tasks.
struct StreamItem {
  int32_t task;
  int32_t step;
  int32_t kv_len;  // of `task`, so that a wave's first loads wait for one record only
  int32_t pad;
};

// A task cut by the ends of runs: run w0 + i holds part i of n (of every kv head).
struct StreamUnit {
  int32_t w0, n;
  bool ends_inside;  // the last part ends before its run does
};

// The cut task that run w has steps begin .. begin + part - 1 of, in runs of `run` steps.
TIDE_HD inline StreamUnit stream_unit(int32_t w, int32_t begin, int32_t part, int32_t steps,
                                      int32_t run) {
  StreamUnit u;
  const int32_t i = begin / run + (begin % run ? 1 : 0);        // this run's part
  const int32_t first = i == 0 ? part : begin - (i - 1) * run;  // steps of part 0
  const int32_t rest = steps - first;
  u.w0 = w - i;
  u.n = 1 + rest / run + (rest % run ? 1 : 0);
  u.ends_inside = rest % run != 0;
  return u;
}

// Waves per workgroup of a call of `items` waves (runs x kv heads), each workgroup taking that
// many consecutive runs of one kv head: 8 combine more partials in LDS; a call of up to 256
// waves takes 4, so that it spreads over more CUs.
TIDE_HD inline int32_t stream_waves(int64_t items) { return items > 256 ? 8 : 4; }

// Workgroups of such a call.
TIDE_HD inline int32_t stream_groups(int32_t runs, int32_t num_kv_heads) {
  const int32_t waves = stream_waves((int64_t)runs * num_kv_heads);
  return (runs + waves - 1) / waves * num_kv_heads;
}

// Where the partials of one kv head's cut tasks go.  The parts that reach their run's end are
// combined per workgroup, into one slot for each (workgroup, task); a part that ends inside
// its run has a slot of its own, at most one for a task and one for a run.  Along the runs
// either the workgroup or the task grows from one such part to the next, so their sum is a
// slot index; where tasks outnumber runs, the (first) run is a smaller one.  A single run cuts
// no task, and with the over 1,024 kv heads that lead to one its slots would be large.
struct StreamSlots {
  int32_t runs, tasks, per;  // per: runs of a workgroup
  TIDE_HD int32_t groups() const { return (runs + per - 1) / per; }
  TIDE_HD int32_t open_slots() const {
    return (int64_t)groups() + tasks < runs ? groups() + tasks : runs;
  }
  TIDE_HD int32_t count() const {
    return runs == 1 ? 0 : open_slots() + (tasks < runs ? tasks : runs);
  }
  TIDE_HD int32_t open(int32_t run, int32_t task) const {
    return (int64_t)groups() + tasks < runs ? run / per + task : run;
  }
  TIDE_HD int32_t ended(int32_t run, int32_t task) const {
    return open_slots() + (tasks < runs ? task : run);
  }
};

// The number of a cut task's partials, and the slot of the e-th in key order.
TIDE_HD inline int32_t stream_parts(const StreamUnit& u, int32_t per) {
  const int32_t wf = u.w0 + u.n - (u.ends_inside ? 2 : 1);
  return wf / per - u.w0 / per + 1 + (u.ends_inside ? 1 : 0);
}

TIDE_HD inline int32_t stream_slot(const StreamUnit& u, const StreamSlots& s, int32_t task,
                                   int32_t e) {
  if (u.ends_inside && e == stream_parts(u, s.per) - 1) return s.ended(u.w0 + u.n - 1, task);
  const int32_t w = (u.w0 / s.per + e) * s.per;
  return s.open(w > u.w0 ? w : u.w0, task);
}

// Shared-prefix decode item: keys [k_begin, k_end) for tasks first_task ..
// first_task + ntasks - 1 and one kv head.  With ntasks > 1 the keys lie in the prefix
// the tasks share (the same physical pages, read through first_task's block table), and
// the item writes one split partial per task; ntasks * group <= 16.
struct SharedDecodeItem {
  int32_t first_task;
  int32_t ntasks;
  int32_t kv_head;
  int32_t split;
  int32_t k_begin;
  int32_t k_end;
  int32_t pad[2];
};

// Append item: positions [pos_begin, pos_end) of `task`, all inside logical page `lpage`.
struct AppendItem {
  int32_t task;
  int32_t lpage;
  int32_t pos_begin;
  int32_t pos_end;
};

// Layout of the per-call header at the start of the workspace.
struct WsHeader {
  int32_t error_flags;  // bit 0: a block-table page id was outside [0, num_pages)
  int32_t pad[63];
};

// A plan (tasks, items) that the kernel reads in place in a pinned staging slot: each workgroup
// sets done[its index] to seq once it has read all it will read of it, and the host then
// reuses the slot.  done == nullptr: the plan is in the workspace.
struct PlanReads {
  uint32_t* done;
  uint32_t seq;
};

struct AppendArgs {
  const uint16_t* k_new;
  const uint16_t* v_new;
  uint16_t* k_pool;
  uint16_t* v_pool;
  const int32_t* block_table;
  int64_t num_pages;
  int32_t bt_stride;
  int32_t num_kv_heads;
  int32_t head_dim;
  int32_t num_items;
  const TaskDesc* tasks;
  const AppendItem* items;
  int32_t* error_flags;
  PlanReads reads;
};

struct ExtendArgs {
  const uint16_t* q;
  const uint16_t* k_pool;
  const uint16_t* v_pool;
  const int32_t* block_table;
  int64_t num_pages;
  int32_t bt_stride;
  int32_t num_q_heads;
  int32_t num_kv_heads;
  int32_t group;
  float scale_log2;  // sm_scale * log2(e): scores are kept in base-2 units
  int32_t num_items;
  const TaskDesc* tasks;
  const ExtendItem* items;
  uint16_t* out;
  float* lse;
  int32_t* error_flags;
  // split-KV plan (chunk_items non-null): items, per-row merge descriptors and the
  // partial buffers [row slots][Hq][d] and [row slots][Hq][4] (max in base-2 units, sum of
  // the bf16-rounded weights, exact fp32 sum, unused)
  const ExtendChunkItem* chunk_items;
  const MergeRow* merge_rows;
  float* part_o;
  float* part_ml;
  int32_t total_rows;
  // fused append (non-null k_new): the new tokens' K/V rows, packed like q by extend_lens,
  // [rows][Hkv][d].  Keys at or past a task's prefix are read from them instead of the
  // pool, and each item writes its own tokens' rows into the pool.
  const uint16_t* k_new;
  const uint16_t* v_new;
  PlanReads reads;  // (plain plan)
};

struct DecodeArgs {
  const uint16_t* q;
  const uint16_t* k_pool;
  const uint16_t* v_pool;
  const int32_t* block_table;
  int64_t num_pages;
  int32_t bt_stride;
  int32_t num_q_heads;
  int32_t num_kv_heads;
  int32_t group;
  float scale_log2;
  int32_t num_tasks;
  int32_t num_items;
  int32_t chunk;       // keys per split (multiple of kDecodeStep)
  int32_t max_splits;  // split slots per (task, q head) in the partial buffers
  const TaskDesc* tasks;  // prefix + extend == kv_len, aux == number of splits
  const void* items;      // DecodeItem, or SharedDecodeItem for the shared-prefix variant
  float* part_o;   // [num_tasks][Hq][max_splits][d] unnormalised partial outputs
  float* part_ml;  // [num_tasks][Hq][max_splits][4]: max (base-2 units), sum of the
                   // bf16-rounded weights, exact fp32 sum, unused
  uint16_t* out;
  float* lse;
  int32_t* error_flags;
  // fused append: the K/V rows of each task's newest token (position kv_len - 1),
  // [num_tasks][Hkv][d]; the split that holds that position writes them into the pool
  // and uses them directly.  Null for a plain decode.
  const uint16_t* k_new;
  const uint16_t* v_new;
  // plain decode: one arrival counter per (task, kv head), zero at launch (uploaded with
  // the work list); the split that brings it to the task's split count merges that kv
  // head's rows.  Null for the shared-prefix variant, which merges in a second kernel.
  int32_t* tickets;
};

struct StreamArgs {
  const uint16_t* q;
  const uint16_t* k_pool;
  const uint16_t* v_pool;
  const int32_t* block_table;
  int64_t num_pages;
  int32_t bt_stride;
  int32_t num_q_heads;
  int32_t num_kv_heads;
  int32_t group;
  float scale_log2;
  int32_t num_runs;
  int32_t steps;       // steps per run
  int32_t last_steps;  // steps of the last run, 1 .. steps
  const TaskDesc* tasks;  // prefix + extend == kv_len
  const StreamItem* items;
  int32_t item_bytes;  // from one to the next: of a StreamItem, or 4 (compact_runs)
  int32_t num_tasks;
  // partials: per kv head the slots of StreamSlots
  float* part_o;     // [Hkv][slots][group][d] unnormalised outputs
  float* part_ml;    // [Hkv][slots][group][4]: max (base-2 units), sum of the bf16-rounded
                     // weights, exact fp32 sum, unused
  // one flag per partial slot: this call's number once the partial is complete (whatever an
  // earlier use of the workspace left there is another call's)
  uint64_t* flags;
  uint64_t call;
  uint16_t* out;
  float* lse;
  int32_t* error_flags;
  const uint16_t* k_new;  // fused append as in DecodeArgs
  const uint16_t* v_new;
  PlanReads reads;
};

// ---- the 4-bit cache ------------------------------------------------------------------------
// Bytes of one (page, kv head) block: K codes, V codes, K scales, V scales (kv4.h).
TIDE_HD constexpr int kv4_block_bytes(int head_dim) { return 17 * head_dim; }

// Query rows (tokens x heads of a kv head) of one attention unit: the columns of one 16-wide MFMA or
// two.
constexpr int kKv4Cols = 32;

// Waves per workgroup of such attention, and workgroups, as stream_waves and stream_groups.
TIDE_HD inline int32_t kv4_waves(int64_t items) { return items > 256 ? 8 : 4; }

TIDE_HD inline int32_t kv4_groups(int32_t runs, int32_t num_kv_heads) {
  const int32_t waves = kv4_waves((int64_t)runs * num_kv_heads);
  return (runs + waves - 1) / waves * num_kv_heads;
}

// Append and unpack item: slots [s0, s0 + n) of logical page `lpage` of block-table row `task`, packed
// rows row0 .. row0 + n - 1.  One record has it all: read where it was staged, a second one that
// depends on it cost another 1.5 us.
struct Kv4StoreItem {
  int32_t task;
  int32_t lpage;
  int32_t row0;
  int32_t span;  // s0 + 32 n: scalar loads have no 16-bit form
};

struct Kv4StoreArgs {
  const uint16_t* k_new;  // append
  const uint16_t* v_new;
  uint16_t* k_out;        // unpack: rows packed like k_new
  uint16_t* v_out;
  uint8_t* pool;
  const int32_t* block_table;
  int64_t num_pages;
  int32_t bt_stride;
  int32_t num_kv_heads;
  int32_t head_dim;
  int32_t num_items;
  const Kv4StoreItem* items;
  int32_t* error_flags;
  PlanReads reads;
};

// Unpacking whole pages for the extend kernel: pages [lpage, lpage + pages) of block-table row
// `row` go to pages [to, to + pages) of the bf16 staging pools, and those ids into row `task` of
// the staging block table.
struct Kv4StageItem {
  int32_t row;
  int32_t lpage;
  int32_t pages;
  int32_t to;
  int32_t task;
  int32_t pad[3];
};

struct Kv4StageArgs {
  const uint8_t* pool;
  const int32_t* block_table;
  int64_t num_pages;
  int32_t bt_stride;
  int32_t num_kv_heads;
  int32_t head_dim;
  int32_t num_items;
  const Kv4StageItem* items;
  uint16_t* k_stage;  // [staging pages][Hkv][kPage][d]
  uint16_t* v_stage;
  int32_t* stage_table;  // [tasks][stage_stride]
  int32_t stage_stride;
  int32_t* error_flags;
  PlanReads reads;
};

// A run of steps: it starts with step `step` of unit `unit`, whose description it repeats (as
// Kv4StoreItem does) and may cross into the next units.
struct Kv4Run {
  int32_t unit;
  int32_t step;
  TaskDesc desc;
  int32_t pad[2];
};

// Attention over the 4-bit cache in runs of steps, as StreamArgs.  A task of the plan is a unit:
// `extend` query tokens (packed rows row_start ..) at positions prefix .. prefix + extend - 1, read
// through block-table row `aux`; their extend x group rows are the columns of the MFMAs.
struct Kv4AttnArgs {
  const uint16_t* q;
  uint8_t* pool;
  const int32_t* block_table;
  int64_t num_pages;
  int32_t bt_stride;
  int32_t num_q_heads;
  int32_t num_kv_heads;
  int32_t group;
  int32_t cols;  // rows of a partial: the most tokens of a unit x group
  float scale_log2;
  int32_t num_runs;
  int32_t steps;
  int32_t last_steps;
  const TaskDesc* units;
  const Kv4Run* runs;
  int32_t num_units;
  bool reread;  // some task has several units
  float* part_o;   // [Hkv][slots][cols][d]
  float* part_ml;  // [Hkv][slots][cols][4]
  uint64_t* flags;
  uint64_t call;
  uint16_t* out;
  float* lse;
  int32_t* error_flags;
  const uint16_t* k_new;  // fused append: one token a unit, [units][Hkv][d]
  const uint16_t* v_new;
  PlanReads reads;
};

// ---- attention mass and eviction ---------------------------------------------------------------
constexpr int kMassKeys = 64;  // keys of a block
// Waves of a workgroup (consecutive runs of one kv head), by whether no task has over 16 query rows a
// kv head: registers let a CU hold 16 and 12 of them (with 6 in place of 4, which the 4 SIMDs do not
// share evenly, a call of 43 rows x 7 heads took 110 us instead of 74).
TIDE_HD constexpr int32_t mass_waves(bool one_trip) { return one_trip ? 8 : 4; }

// Mass work of one wave and kv head: `blocks` blocks from block `block` of `task` on, crossing into
// the next tasks (those without new tokens have no blocks).
struct MassRun {
  int32_t task;
  int32_t block;
  int32_t blocks;
  int32_t pad;
};

TIDE_HD inline int32_t mass_groups(int32_t runs, int32_t num_kv_heads, bool one_trip) {
  return (runs + mass_waves(one_trip) - 1) / mass_waves(one_trip) * num_kv_heads;
}

// aux of a task: the positions whose sums are carried on (later ones start at 0).
struct MassArgs {
  const uint16_t* q;
  const float* lse;
  const void* pool;  // K pages, or the 4-bit pool
  const int32_t* block_table;
  int64_t num_pages;
  int32_t bt_stride;
  int32_t num_q_heads;
  int32_t num_kv_heads;
  int32_t group;
  float scale_log2;
  int32_t num_runs;
  bool one_trip;  // no task has over 16 query rows a kv head
  const TaskDesc* tasks;
  const MassRun* runs;
  float* mass;
  int32_t* error_flags;
  PlanReads reads;
};

// One task of an eviction: `keep` of `kv_len` positions stay, the last `recent` of them always.
struct EvictTask {
  int32_t task;    // block-table row
  int32_t kv_len;
  int32_t keep;
  int32_t recent;
  int32_t first;   // packed row of `kept`: the sum of the earlier tasks' keep
  int32_t nth;     // of record i: the record of the task with the i-th largest `keep`
  int32_t pad[2];
};

// A kept position: its sum, and the pages that it leaves and that its rank lies in (leaves < 0: one of
// them is out of range, the position is not moved).
struct EvictIndex {
  int32_t pos;
  int32_t from;
  int32_t to;
  float mass;
};

struct EvictArgs {
  uint8_t* k_pool;  // K pages, or the 4-bit pool
  uint8_t* v_pool;
  float* mass;
  const int32_t* block_table;
  const int32_t* new_table;  // equal to block_table: in place
  int64_t num_pages;
  int32_t bt_stride;
  int32_t new_stride;
  int32_t num_kv_heads;
  int32_t num_tasks;
  int32_t first_pair;  // of the launch's (task, kv head) pairs
  int32_t longest_keep;
  const EvictTask* tasks;
  EvictTask* move_tasks;  // the same in the workspace, written by the first kernel for the second
  EvictIndex* index;  // [sum of keep x Hkv]: a task's from first x Hkv on, head after head, ascending
  int32_t* kept;      // [sum of keep][Hkv], may be null
  int32_t* error_flags;
  PlanReads reads;
};

// ---- steps whose rows, lengths and block lists are device data -------------------------------------
// A row is one query token: its task (block-table row) and its position in it; either negative, or out
// of range, marks a row that nothing is done for.
TIDE_HD inline bool live_row(int32_t task, int32_t pos, int32_t num_tasks, int64_t max_len) {
  return task >= 0 && task < num_tasks && pos >= 0 && pos < max_len;
}

struct PageMapArgs {
  const int32_t* lens;
  const int32_t* want;
  int32_t num_tasks;
  int32_t* block_table;
  int32_t bt_stride;
  int32_t* free_pages;  // a stack
  int32_t capacity;
  const int32_t* free_count;
  int32_t num_rows;
  int32_t* lens_out;
  int32_t* free_count_out;
  int32_t* row_start;  // [num_tasks + 1]
  int32_t* row_task;   // [num_rows] each
  int32_t* row_pos;
  int64_t* row_slot;
  bool rows_apart;     // the rows are written by a kernel of their own
  bool returns_apart;  // and the pages that go back are moved by one
};

// Key bounds: per (page, kv head) d upper and d lower bounds in whole units 2^units (kNoUnit: a key
// of the page is not finite).
constexpr int kLeastUnit = -120, kMostUnit = 122, kNoUnit = 127;

struct SlotAppendArgs {
  const uint16_t* k_new;
  const uint16_t* v_new;
  const int64_t* row_slot;
  uint16_t* k_pool;
  uint16_t* v_pool;
  int64_t num_pages;
  int32_t num_kv_heads;
  int32_t num_rows;
  int32_t first_row;  // of the launch
  int32_t window;     // rows of a workgroup
  int8_t* bounds;     // [num_pages][Hkv][2][d], may be null
  int8_t* units;      // [num_pages][Hkv]
  int32_t* error_flags;
};

struct KeyBoundsArgs {
  const uint16_t* k_pool;
  int64_t num_pages;
  const int32_t* block_table;
  int32_t bt_stride;
  int32_t num_kv_heads;
  const int32_t* lens;
  const int32_t* from;  // may be null: 0
  int32_t max_len;
  int32_t chunks;       // of a task: the pages of one wave
  int32_t first_task, first_chunk, units_here;  // (task, chunk) pairs of the launch
  int8_t* bounds;
  int8_t* units;
  int32_t* error_flags;
};

// Blocks that a wave of the score kernel takes at a time, one page id a lane.
constexpr int kScoreChunk = 64;

struct BlockSelectArgs {
  const uint16_t* q;
  const int32_t* row_task;
  const int32_t* row_pos;
  const int8_t* bounds;
  const int8_t* units;
  int64_t num_pages;
  const int32_t* block_table;
  int32_t bt_stride;
  int32_t num_tasks;
  int32_t num_q_heads;
  int32_t num_kv_heads;
  int32_t group;
  int32_t max_len;
  int32_t first_row, rows;  // of the launches
  int32_t tile_rows;        // rows of a unit of the score kernel
  int32_t splits;           // waves that share a (unit, kv head)
  int32_t* scores;          // [rows][Hkv][score_stride], integers that order like the scores
  int32_t score_stride;     // blocks, a multiple of kScoreChunk
  int32_t budget, sink, recent;
  int32_t* sel;             // [num_rows][Hkv][budget]
  int32_t* error_flags;
};

// Rows taken together by the shared kernel: entries of its packed list, and blocks of a context that it can mark.
constexpr int kSharedEntries = 1536, kSharedRows = 8;
template <int D>
constexpr int kSharedBlocks = 8 * kPage * D * 2;

// Workgroups of a call up to which each has a CU of its own.
constexpr uint32_t kSparseAlone = 256;

struct SparseArgs {
  const uint16_t* q;
  const uint16_t* k_pool;
  const uint16_t* v_pool;
  int64_t num_pages;
  const int32_t* block_table;
  int32_t bt_stride;
  int32_t num_tasks;
  int32_t num_q_heads;
  int32_t num_kv_heads;
  int32_t group;
  float scale_log2;
  const int32_t* row_task;
  const int32_t* row_pos;
  int32_t first_row, rows;  // of the launch
  const int32_t* sel;
  int32_t budget;
  int32_t splits;       // workgroups that share a (row, kv head)
  int32_t rows_at_once, padded_shift;  // shared kernel: rows of a workgroup, log2 of the columns of each
  float* part_o;        // [rows of a launch][Hkv][splits][group][d]
  float* part_ml;       // [..][splits][group][4]: max (base-2 units), sum of the bf16-rounded weights,
                        // exact sum, 1 if the part has a key
  uint16_t* out;
  float* lse;
  int32_t* error_flags;
};

}  // namespace tide
