// The extern "C" entry points of steps whose rows, lengths and block lists are device data
// (include/tide.h): checks, workspaces, launches.  Nothing is planned from lengths, so nothing is staged.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "kernels.h"
#include "plan.h"
#include "staging.h"
#include "tide.h"

namespace tide {
namespace {

constexpr size_t kHeader = sizeof(WsHeader);

bool on16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// Checks that the entry points of rows start with.  *go: there is something to do.
int begin(const tide_dims* dims, int32_t count, int64_t num_pages, bool* go) {
  *go = false;
  const int rc = check_dims(dims);
  if (rc != TIDE_OK) return rc;
  if (count < 0) return TIDE_ERR_INVALID_ARG;
  if (count == 0) return TIDE_OK;
  if (num_pages <= 0) return TIDE_ERR_INVALID_ARG;
  *go = true;
  return TIDE_OK;
}

// Whether the arrays that a page map writes overlap another of its arrays.  One workgroup writes while others still read,
// and rows are written from what was granted before: a refused task's length in the place of the wanted one would pass
// for a granted one, with rows in pages that it was not given.  lens_out may be lens itself (a task's length is replaced
// by the thread that read it, after its last use), also where lens is what is wanted, and free_count_out free_count.
bool arrays_overlap(const PageMapArgs& a) {
  struct Span {
    uintptr_t at;
    int64_t bytes;
  };
  auto span = [](const void* p, int64_t bytes) { return Span{reinterpret_cast<uintptr_t>(p), bytes}; };
  const int64_t tasks = 4 * (int64_t)a.num_tasks, rows = 4 * (int64_t)a.num_rows;
  const Span all[] = {span(a.lens, tasks), span(a.want, tasks), span(a.free_count, 4),
                      // written:
                      span(a.lens_out, tasks), span(a.free_count_out, 4),
                      span(a.block_table, tasks * a.bt_stride), span(a.free_pages, 4 * (int64_t)a.capacity),
                      span(a.row_start, tasks + 4), span(a.row_task, rows), span(a.row_pos, rows),
                      span(a.row_slot, 2 * rows)};
  constexpr int kRead = 3, kAll = sizeof(all) / sizeof(all[0]);
  for (int j = kRead; j < kAll; ++j)
    for (int i = 0; i < j; ++i) {
      const Span &x = all[i], &y = all[j];
      if (x.bytes == 0 || y.bytes == 0 || x.at >= y.at + y.bytes || y.at >= x.at + x.bytes) continue;
      const bool lens = j == 3 && i < 2 && x.at == y.at && all[0].at == y.at;
      const bool count = i == 2 && j == 4 && x.at == y.at;
      if (!lens && !count) return true;
    }
  return false;
}

// The longest context of a call: max_len, or (0) all that the block table holds.
int longest(int32_t max_len, int32_t bt_stride, int32_t* out) {
  const int64_t most = std::min<int64_t>((int64_t)bt_stride * kPage, INT32_MAX);
  if (max_len < 0) return TIDE_ERR_INVALID_ARG;
  if (max_len > most) return TIDE_ERR_CAPACITY;
  *out = max_len ? max_len : (int32_t)most;
  return TIDE_OK;
}

// Entries of a row's list: two rounds of them more still fit in 32 bits.
constexpr int32_t kMostBudget = 1 << 30;

// ---- selection: rows go in rounds of at most kScoreBytes of scores, which stay in the last-level cache
constexpr int64_t kScoreBytes = 256 << 20;
constexpr int32_t kRoundPairs = 1 << 20;  // (row, kv head) pairs of a round
// Waves of the score kernels: contexts differ, so rows are cut finer than the device needs to be full (by rows: 117 us with
// 8,192 waves, 126 with 4,096; by tasks: 221 with 4,096 for 1,761 rows over 32k-98k, 233 with 8,192).
constexpr int64_t kScoreRowWaves = 8192, kScoreChunkWaves = 4096;

// Whether rows go to the score kernel task by task.  Its workgroups bring a chunk of bounds for up to 256 rows, but walk
// these rows' tasks one after the other; the other kernel reads a task's bounds for each row.  (Contexts of 4k-16k, scores
// and choice, row by row and task by task: 28 / 4 heads, 64 x 4 rows 43 and 44 us, 64 x 8 64 and 52, 8 x 4 16 and 31, 8 x
// 16 30 and 19, 256 x 2 85 and 124, 256 x 4 154 and 102; 8 / 8 heads, whose products hold four times the rows, 64 x 4 61
// and 238, 64 x 8 111 and 130, 64 x 16 243 and 91, 256 x 4 298 and 284.)
// Launches may not depend on device data, so what counts is the table's height and the rows with their padding: in a table
// much taller than the tasks that have rows, or a batch that is mostly padding, this is the slower one of the two (32 / 8
// heads, contexts of 1k-16k: 256 single tokens of 256 tasks 66 us, with 1,792 rows of padding behind them 364; 8 x 128 rows
// of 4k-16k 55 in tables of 8-256 tasks, 133 of 1,056).  A table of the tasks that have rows avoids it.
bool score_by_task(int32_t num_rows, int32_t num_tasks, int32_t group) {
  const int64_t rows = num_rows, tasks = num_tasks;
  return rows >= (group > 2 ? 8 : 16) * tasks || (rows >= 4 * tasks && rows >= 1024);
}

struct SelectRounds {
  int32_t rows;         // of a round
  int32_t stride;       // scores of a (row, kv head)
  size_t bytes;
};

int32_t score_stride(int32_t max_len) {
  const int64_t blocks = ((int64_t)max_len + kPage - 1) / kPage;
  return (int32_t)((blocks + kScoreChunk - 1) / kScoreChunk * kScoreChunk);
}

SelectRounds select_rounds(int32_t num_rows, int32_t max_len, const tide_dims& dims) {
  SelectRounds r;
  r.stride = score_stride(max_len);
  const int64_t row = (int64_t)r.stride * dims.num_kv_heads * 4;
  const int64_t most = std::min<int64_t>(kScoreBytes / row, kRoundPairs / dims.num_kv_heads);
  r.rows = (int32_t)std::min<int64_t>(num_rows, std::max<int64_t>(1, most));
  r.bytes = kHeader + (size_t)((int64_t)r.rows * row);
  return r;
}

// At least select_rounds(n, m).bytes for every n <= num_rows and m <= max_len.  (Those fall where a row grows by so much that
// one fewer fits in a round.)
size_t select_bound(int32_t num_rows, int32_t max_len, const tide_dims& dims) {
  const int64_t row = (int64_t)score_stride(max_len) * dims.num_kv_heads * 4;
  if (row >= kScoreBytes) return kHeader + (size_t)row;
  return kHeader + (size_t)std::min<int64_t>(kScoreBytes, num_rows * row);
}

// ---- sparse attention: workgroups that share a (row, kv head) where there are few of them.  A part keeps 4 steps for
// each of its 4 waves, and there are none where the whole has fewer than 12: less does not pay for the second kernel,
// which joins the parts.  (4 rows of 4 kv heads: 64 blocks 12.4 us in one part, 15.2 in two; 128 blocks 22.0 in one,
// 16.7 in two, 14.6 in four; 256 blocks 40.1 in one, 26.1 in two, 15.2 in eight.)
constexpr int32_t kLeastPairs = 16, kSplitPairs = 48;
constexpr int32_t kSparseLaunch = 1 << 23; // workgroups of a launch (fewer than 2^32 threads)

int32_t sparse_splits(int64_t num_rows, int32_t budget, const tide_dims& dims) {
  const int64_t units = num_rows * dims.num_kv_heads;
  const int64_t pairs = ((int64_t)budget + 1) / 2;
  if (pairs < kSplitPairs) return 1;
  return (int32_t)std::max<int64_t>(1, std::min<int64_t>(kSparseAlone / units, pairs / kLeastPairs));
}

size_t sparse_bytes(int32_t num_rows, int32_t budget, const tide_dims& dims, size_t* ml_off) {
  const int64_t splits = sparse_splits(num_rows, budget, dims);
  if (splits == 1) return kHeader;
  const size_t rows = (size_t)num_rows * dims.num_q_heads * splits;  // at most 512 x 16
  *ml_off = kHeader + rows * dims.head_dim * 4;
  return *ml_off + rows * 16;
}

// At least sparse_bytes(n, b) for every n <= num_rows and b <= budget.  (Those fall where rows become so many that they are
// split into fewer parts or none: a (row, kv head) has at most pairs / kLeastPairs parts, and all have at most kSparseAlone.)
size_t sparse_bound(int32_t num_rows, int32_t budget, const tide_dims& dims) {
  const int64_t pairs = ((int64_t)budget + 1) / 2;
  if (pairs < kSplitPairs) return kHeader;
  const int64_t most = kSparseAlone;  // (each factor is cut there before they are multiplied)
  const int64_t units = std::min(most, (int64_t)num_rows * dims.num_kv_heads), parts = std::min(most, pairs / kLeastPairs);
  return kHeader + (size_t)(std::min(most, units * parts) * (dims.num_q_heads / dims.num_kv_heads) * (dims.head_dim * 4 + 16));
}

// Up to this many (row, kv head) pairs rows are taken one by one even where they share a task: a workgroup each, all at
// once (28 / 4 heads, 128 blocks, 64 rows of a task: 18 us, 31 together; 8 x 16 rows 31 and 35; 8 x 64 rows 103 and 52;
// 32 / 8 heads, 8 x 16 rows: 55 and 40).  Whether rows share tasks goes by the table's height, as above: 8 x 128 rows take
// 194 us in tables of 8-256 tasks, 650 of 1,056, and 256 single tokens 318, with 256 rows of padding 352.
constexpr int64_t kFewPairs = 512;

// Rows that a workgroup takes at once: 1 where rows have tasks of their own or are few, and where their lists or
// contexts are longer than a workgroup can mark.
void shared_rows(int32_t num_rows, int32_t num_tasks, int32_t budget, int32_t bt_stride, const tide_dims& dims,
                 int32_t splits, int32_t* rows, int32_t* shift) {
  const int32_t group = dims.num_q_heads / dims.num_kv_heads;
  *shift = 0;
  while ((1 << *shift) < group) ++*shift;
  *rows = 1;
  if (num_rows <= num_tasks || (int64_t)num_rows * dims.num_kv_heads <= kFewPairs || splits > 1) return;
  if (bt_stride > (dims.head_dim == 128 ? kSharedBlocks<128> : kSharedBlocks<64>)) return;
  *rows = std::max(1, std::min({kSharedRows, 32 >> *shift, kSharedEntries / budget}));
}

// bound: of every call with at most these rows, budget and longest context; else of this one.
int rows_workspace(int op, int32_t num_rows, int32_t budget, int32_t max_len, const tide_dims* dims, bool bound,
                   size_t* bytes_out) {
  try {
    const int rc = check_dims(dims);
    if (rc != TIDE_OK) return rc;
    if (!bytes_out || num_rows < 0) return TIDE_ERR_INVALID_ARG;
    size_t ml_off = 0;
    switch (op) {
      case TIDE_OP_SLOT_APPEND:
      case TIDE_OP_KEY_BOUNDS:
        *bytes_out = kHeader;
        return TIDE_OK;
      case TIDE_OP_BLOCK_SELECT:
        if (max_len <= 0) return TIDE_ERR_INVALID_ARG;
        *bytes_out = kHeader;
        if (num_rows > 0)
          *bytes_out = bound ? select_bound(num_rows, max_len, *dims) : select_rounds(num_rows, max_len, *dims).bytes;
        return TIDE_OK;
      case TIDE_OP_SPARSE_ATTN:
        if (budget <= 0) return TIDE_ERR_INVALID_ARG;
        if (budget > kMostBudget) return TIDE_ERR_UNSUPPORTED;
        *bytes_out = kHeader;
        if (num_rows > 0)
          *bytes_out = bound ? sparse_bound(num_rows, budget, *dims) : sparse_bytes(num_rows, budget, *dims, &ml_off);
        return TIDE_OK;
      default:
        return TIDE_ERR_INVALID_ARG;
    }
  } catch (...) {
    return TIDE_ERR_HIP;
  }
}

}  // namespace
}  // namespace tide

using namespace tide;

extern "C" {

TIDE_API int tide_rows_workspace_size(int op, int32_t num_rows, int32_t budget, int32_t max_len, const tide_dims* dims,
                                      size_t* bytes_out) {
  return rows_workspace(op, num_rows, budget, max_len, dims, false, bytes_out);
}

TIDE_API int tide_rows_workspace_bound(int op, int32_t num_rows, int32_t budget, int32_t max_len, const tide_dims* dims,
                                       size_t* bytes_out) {
  return rows_workspace(op, num_rows, budget, max_len, dims, true, bytes_out);
}

TIDE_API int tide_page_map(const int32_t* lens, const int32_t* want_lens, int32_t num_tasks, int32_t* block_table,
                           int32_t bt_stride, int32_t* free_pages, int32_t free_capacity, const int32_t* free_count,
                           int32_t num_rows, int32_t* lens_out, int32_t* free_count_out, int32_t* row_start,
                           int32_t* row_task, int32_t* row_pos, int64_t* row_slot, const tide_dims* dims, void* stream) {
  try {
    const int rc = check_dims(dims);
    if (rc != TIDE_OK) return rc;
    if (num_tasks < 0 || num_rows < 0 || free_capacity < 0) return TIDE_ERR_INVALID_ARG;
    if (num_tasks == 0) return TIDE_OK;
    if (bt_stride <= 0) return TIDE_ERR_INVALID_ARG;
    if ((int64_t)num_tasks * bt_stride > INT32_MAX || num_rows == INT32_MAX) return TIDE_ERR_UNSUPPORTED;
    if (!lens || !want_lens || !block_table || !free_count || !lens_out || !free_count_out || !row_start ||
        (free_capacity > 0 && !free_pages) || (num_rows > 0 && (!row_task || !row_pos || !row_slot)))
      return TIDE_ERR_INVALID_ARG;
    PageMapArgs a = {};
    a.lens = lens;
    a.want = want_lens;
    a.num_tasks = num_tasks;
    a.block_table = block_table;
    a.bt_stride = bt_stride;
    a.free_pages = free_pages;
    a.capacity = free_capacity;
    a.free_count = free_count;
    a.num_rows = num_rows;
    a.lens_out = lens_out;
    a.free_count_out = free_count_out;
    a.row_start = row_start;
    a.row_task = row_task;
    a.row_pos = row_pos;
    a.row_slot = row_slot;
    if (arrays_overlap(a)) return TIDE_ERR_INVALID_ARG;
    return launch_page_map(a, static_cast<hipStream_t>(stream)) == hipSuccess ? TIDE_OK : TIDE_ERR_HIP;
  } catch (...) {
    return TIDE_ERR_HIP;
  }
}

TIDE_API int tide_slot_append(const void* k_new, const void* v_new, const int64_t* row_slot, int32_t num_rows,
                              void* k_pool, void* v_pool, int64_t num_pages, int8_t* bounds, int8_t* units,
                              const tide_dims* dims, void* workspace, size_t workspace_bytes, void* stream) {
  try {
    bool go;
    int rc = begin(dims, num_rows, num_pages, &go);
    if (rc != TIDE_OK || !go) return rc;
    if (!k_new || !v_new || !row_slot || !k_pool || !v_pool || !workspace || !bounds != !units)
      return TIDE_ERR_INVALID_ARG;
    if (!on16(k_new) || !on16(v_new) || !on16(k_pool) || !on16(v_pool) || !on16(bounds) || !on16(workspace))
      return TIDE_ERR_INVALID_ARG;
    if (workspace_bytes < kHeader) return TIDE_ERR_CAPACITY;
    hipStream_t s = static_cast<hipStream_t>(stream);
    rc = clear_flags(workspace, s);
    if (rc != TIDE_OK) return rc;
    SlotAppendArgs a = {};
    a.k_new = static_cast<const uint16_t*>(k_new);
    a.v_new = static_cast<const uint16_t*>(v_new);
    a.row_slot = row_slot;
    a.k_pool = static_cast<uint16_t*>(k_pool);
    a.v_pool = static_cast<uint16_t*>(v_pool);
    a.num_pages = num_pages;
    a.num_kv_heads = dims->num_kv_heads;
    a.num_rows = num_rows;
    a.bounds = bounds;
    a.units = units;
    a.error_flags = at_mut<int32_t>(workspace, 0);
    Staged none;
    return finish(launch_slot_append(a, dims->head_dim, s), none, workspace, s);
  } catch (...) {
    return TIDE_ERR_HIP;
  }
}

TIDE_API int tide_key_bounds(const void* k_pool, int64_t num_pages, const int32_t* block_table, int32_t bt_stride,
                             int32_t num_tasks, const int32_t* lens, const int32_t* from_lens, int32_t max_len,
                             int8_t* bounds, int8_t* units, const tide_dims* dims, void* workspace,
                             size_t workspace_bytes, void* stream) {
  try {
    bool go;
    int rc = begin(dims, num_tasks, num_pages, &go);
    if (rc != TIDE_OK || !go) return rc;
    if (bt_stride <= 0) return TIDE_ERR_INVALID_ARG;
    int32_t most;
    rc = longest(max_len, bt_stride, &most);
    if (rc != TIDE_OK) return rc;
    if (!k_pool || !block_table || !lens || !bounds || !units || !workspace) return TIDE_ERR_INVALID_ARG;
    if (!on16(k_pool) || !on16(bounds) || !on16(workspace)) return TIDE_ERR_INVALID_ARG;
    if (workspace_bytes < kHeader) return TIDE_ERR_CAPACITY;
    hipStream_t s = static_cast<hipStream_t>(stream);
    rc = clear_flags(workspace, s);
    if (rc != TIDE_OK) return rc;
    KeyBoundsArgs a = {};
    a.k_pool = static_cast<const uint16_t*>(k_pool);
    a.num_pages = num_pages;
    a.block_table = block_table;
    a.bt_stride = bt_stride;
    a.num_kv_heads = dims->num_kv_heads;
    a.lens = lens;
    a.from = from_lens;
    a.max_len = most;
    a.bounds = bounds;
    a.units = units;
    a.error_flags = at_mut<int32_t>(workspace, 0);
    Staged none;
    return finish(launch_key_bounds(a, dims->head_dim, num_tasks, s), none, workspace, s);
  } catch (...) {
    return TIDE_ERR_HIP;
  }
}

TIDE_API int tide_block_select(const void* q, const int32_t* row_task, const int32_t* row_pos, int32_t num_rows,
                               const int8_t* bounds, const int8_t* units, int64_t num_pages,
                               const int32_t* block_table, int32_t bt_stride, int32_t num_tasks, int32_t budget,
                               int32_t sink, int32_t recent, int32_t max_len, const tide_dims* dims, int32_t* sel,
                               void* workspace, size_t workspace_bytes, void* stream) {
  try {
    bool go;
    int rc = begin(dims, num_rows, num_pages, &go);
    if (rc != TIDE_OK) return rc;
    if (budget <= 0 || sink < 0 || recent < 0 || (int64_t)sink + recent > budget || num_tasks < 0)
      return TIDE_ERR_INVALID_ARG;
    if (budget > kMostBudget) return TIDE_ERR_UNSUPPORTED;
    if (!go || num_tasks == 0) return TIDE_OK;
    if (bt_stride <= 0) return TIDE_ERR_INVALID_ARG;
    int32_t most;
    rc = longest(max_len, bt_stride, &most);
    if (rc != TIDE_OK) return rc;
    if (!q || !row_task || !row_pos || !bounds || !units || !block_table || !sel || !workspace)
      return TIDE_ERR_INVALID_ARG;
    if (!on16(q) || !on16(bounds) || !on16(workspace)) return TIDE_ERR_INVALID_ARG;
    const SelectRounds rounds = select_rounds(num_rows, most, *dims);
    if (workspace_bytes < rounds.bytes) return TIDE_ERR_CAPACITY;
    hipStream_t s = static_cast<hipStream_t>(stream);
    rc = clear_flags(workspace, s);
    if (rc != TIDE_OK) return rc;
    BlockSelectArgs a = {};
    a.q = static_cast<const uint16_t*>(q);
    a.row_task = row_task;
    a.row_pos = row_pos;
    a.bounds = bounds;
    a.units = units;
    a.num_pages = num_pages;
    a.block_table = block_table;
    a.bt_stride = bt_stride;
    a.num_tasks = num_tasks;
    a.num_q_heads = dims->num_q_heads;
    a.num_kv_heads = dims->num_kv_heads;
    a.group = dims->num_q_heads / dims->num_kv_heads;
    a.max_len = most;
    a.scores = at_mut<int32_t>(workspace, kHeader);
    a.score_stride = rounds.stride;
    a.budget = budget;
    a.sink = sink;
    a.recent = recent;
    a.sel = sel;
    a.error_flags = at_mut<int32_t>(workspace, 0);
    a.tile_rows = select_tile_rows(a.group, score_by_task(num_rows, num_tasks, a.group));
    const int64_t target = a.tile_rows == 1 ? kScoreRowWaves : kScoreChunkWaves;
    hipError_t err = hipSuccess;
    for (int64_t first = 0; first < num_rows && err == hipSuccess; first += rounds.rows) {
      a.first_row = (int32_t)first;
      a.rows = (int32_t)std::min<int64_t>(rounds.rows, num_rows - first);
      const int64_t waves = (int64_t)((a.rows + a.tile_rows - 1) / a.tile_rows) * a.num_kv_heads;
      a.splits = (int32_t)std::max<int64_t>(1, std::min<int64_t>((target + waves - 1) / waves, rounds.stride / kScoreChunk));
      err = launch_block_select(a, dims->head_dim, s);
    }
    Staged none;
    return finish(err, none, workspace, s);
  } catch (...) {
    return TIDE_ERR_HIP;
  }
}

TIDE_API int tide_sparse_attn(const void* q, const void* k_pool, const void* v_pool, int64_t num_pages,
                              const int32_t* block_table, int32_t bt_stride, int32_t num_tasks,
                              const int32_t* row_task, const int32_t* row_pos, int32_t num_rows, const int32_t* sel,
                              int32_t budget, const tide_dims* dims, void* out, float* lse, void* workspace,
                              size_t workspace_bytes, void* stream) {
  try {
    bool go;
    int rc = begin(dims, num_rows, num_pages, &go);
    if (rc != TIDE_OK) return rc;
    if (budget <= 0 || num_tasks < 0) return TIDE_ERR_INVALID_ARG;
    if (budget > kMostBudget) return TIDE_ERR_UNSUPPORTED;
    if (!go || num_tasks == 0) return TIDE_OK;
    if (bt_stride <= 0) return TIDE_ERR_INVALID_ARG;
    if (!q || !k_pool || !v_pool || !block_table || !row_task || !row_pos || !sel || !out || !workspace)
      return TIDE_ERR_INVALID_ARG;
    if (!on16(q) || !on16(k_pool) || !on16(v_pool) || !on16(out) || !on16(workspace)) return TIDE_ERR_INVALID_ARG;
    size_t ml_off = 0;
    if (workspace_bytes < sparse_bytes(num_rows, budget, *dims, &ml_off)) return TIDE_ERR_CAPACITY;
    // (rows that are taken again read q after out was written)
    const uintptr_t q_at = reinterpret_cast<uintptr_t>(q), out_at = reinterpret_cast<uintptr_t>(out);
    if ((q_at < out_at ? out_at - q_at : q_at - out_at) < (uintptr_t)num_rows * dims->num_q_heads * dims->head_dim * 2)
      return TIDE_ERR_INVALID_ARG;
    hipStream_t s = static_cast<hipStream_t>(stream);
    rc = clear_flags(workspace, s);
    if (rc != TIDE_OK) return rc;
    SparseArgs a = {};
    a.q = static_cast<const uint16_t*>(q);
    a.k_pool = static_cast<const uint16_t*>(k_pool);
    a.v_pool = static_cast<const uint16_t*>(v_pool);
    a.num_pages = num_pages;
    a.block_table = block_table;
    a.bt_stride = bt_stride;
    a.num_tasks = num_tasks;
    a.num_q_heads = dims->num_q_heads;
    a.num_kv_heads = dims->num_kv_heads;
    a.group = dims->num_q_heads / dims->num_kv_heads;
    a.scale_log2 = dims->sm_scale * 1.44269504088896340736f;
    a.row_task = row_task;
    a.row_pos = row_pos;
    a.sel = sel;
    a.budget = budget;
    a.splits = sparse_splits(num_rows, budget, *dims);
    a.part_o = at_mut<float>(workspace, kHeader);
    a.part_ml = at_mut<float>(workspace, ml_off);
    a.out = static_cast<uint16_t*>(out);
    a.lse = lse;
    a.error_flags = at_mut<int32_t>(workspace, 0);
    // rows of one task share pages; a row of its own streams them
    const bool shared = num_rows > num_tasks;
    shared_rows(num_rows, num_tasks, budget, bt_stride, *dims, a.splits, &a.rows_at_once, &a.padded_shift);
    int64_t most = std::max<int64_t>(1, kSparseLaunch / ((int64_t)a.num_kv_heads * a.splits));
    most -= a.rows_at_once > 1 ? most % a.rows_at_once : 0;
    hipError_t err = hipSuccess;
    for (int64_t first = 0; first < num_rows && err == hipSuccess; first += most) {
      a.first_row = (int32_t)first;
      a.rows = (int32_t)std::min<int64_t>(most, num_rows - first);
      err = a.rows_at_once > 1 ? launch_sparse_shared(a, dims->head_dim, s) : launch_sparse(a, dims->head_dim, shared, s);
    }
    Staged none;
    return finish(err, none, workspace, s);
  } catch (...) {
    return TIDE_ERR_HIP;
  }
}

}  // extern "C"
