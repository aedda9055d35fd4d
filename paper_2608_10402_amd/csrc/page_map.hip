// Page map: block tables and slot maps from lengths that live on the device.
//
// lens[b] positions of task b are cached, want[b] are wanted.  A task that shrinks gives its last pages
// back to the free list, a stack; a task that grows by e tokens takes ceil(want / 16) - ceil(lens / 16)
// pages from its top and gets e rows, one a new token, packed in task order:
//     rows:   start_b = sum of the e before b            (refused where start_b + e > num_rows)
//     pages:  first_b = sum of the pages before b        (refused where first_b + pages > what is there)
//     page j of the call is free_pages[count - 1 - j], with the returned pages pushed first.
// Both sums only grow, so a refusal holds for every later task that needs one more, and what is
// granted is one run from the top: the result does not depend on the order of threads.
//
// One workgroup scans the tasks, 2,048 a round, and then writes pages and rows element by element: each
// finds its task by bisection of the sums in LDS, so one long task costs no more than many short ones.
// Above kRowsHere rows a second kernel writes the rows from the results of the first, and pages that go back to a large
// table are moved by a kernel before it, whose workgroups scan all lengths again.
//
// Latencies bound it: lengths, three scans with a barrier each, free pages, rows.  175 tasks of one token each take 7.2 us;
// 1,056 tasks of 1-450 tokens, a tenth of which end, take 23 us a call with their 69,946 rows: 24 with the 17,000 page ids
// through one CU, 32 with one task a thread and one element at a time.
#include <type_traits>

#include "kernels.h"
#include "tide_device.h"

namespace tide {
namespace kern {

constexpr int kMapThreads = 1024;
constexpr int kMapTasks = 2048;  // of a round
constexpr int kMany = 4;  // pages or rows of a thread whose bisections and loads are in flight together
constexpr int kRowThreads = 256;
constexpr int kRowTasks = 4096;  // tasks whose row starts the second kernel keeps in LDS

// a + b for 0 <= a, b <= 2^31 - 1, at most that: the new tokens of many tasks may sum to more
__device__ __forceinline__ uint32_t sat_add(uint32_t a, uint32_t b) { return min(a + b, 0x7FFFFFFFu); }

// Inclusive sums of x over the workgroup's threads, and their sum over all.  tmp: 16 words that no
// other call before the next barrier but one uses.
__device__ __forceinline__ uint32_t map_scan(uint32_t x, uint32_t* tmp, uint32_t* all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    const uint32_t y = __shfl_up((int)x, o, 64);
    if (lane >= o) x = sat_add(x, y);
  }
  if (lane == 63) tmp[wave] = x;
  __syncthreads();
  uint32_t before = 0, total = 0;
#pragma unroll
  for (int w = 0; w < kMapThreads / 64; ++w) {
    if (w == wave) before = total;
    total = sat_add(total, tmp[w]);
  }
  *all = total;
  return sat_add(before, x);
}

// The last of the n entries of ascending first[] that is at most j (first[0] <= j).
template <class T>
__device__ __forceinline__ int last_at_most(const T* first, int n, T j) {
  int lo = 0;
  while (n > 1) {
    const int half = n >> 1;
    if (first[lo + half] <= j) lo += half, n -= half;
    else n = half;
  }
  return lo;
}

// The same for several values, whose reads are in flight together.
template <int kAtOnce>
__device__ __forceinline__ void last_at_most(const uint32_t* first, int n, const uint32_t (&j)[kAtOnce], int (&at)[kAtOnce]) {
#pragma unroll
  for (int u = 0; u < kAtOnce; ++u) at[u] = 0;
  while (n > 1) {
    const int half = n >> 1;
    uint32_t x[kAtOnce];
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) x[u] = first[at[u] + half];
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) at[u] += x[u] <= j[u] ? half : 0;
    n -= half;
  }
}

__device__ __forceinline__ int32_t pages_of(int32_t len) { return (int32_t)(((int64_t)len + kPage - 1) / kPage); }

__device__ __forceinline__ void put_row(const PageMapArgs& a, int64_t r, int32_t task, int32_t pos, int64_t slot) {
  a.row_task[r] = task;
  a.row_pos[r] = pos;
  a.row_slot[r] = slot;
}

// Lengths of a thread's two neighbouring tasks of a round, from task b on; one whose lengths are no lengths stays as
// it is.
__device__ __forceinline__ void load_lengths(const PageMapArgs& a, int b, int32_t (&len)[2], int32_t (&want)[2]) {
  const int64_t most = (int64_t)a.bt_stride * kPage;
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    len[c] = want[c] = 0;
    if (b + c >= a.num_tasks) continue;
    len[c] = a.lens[b + c];
    want[c] = a.want[b + c];
    if (len[c] < 0 || len[c] > most || want[c] < 0 || want[c] > most) want[c] = len[c];
  }
}

// f(how many elements of `all` a thread takes at once)
template <class F>
__device__ __forceinline__ void by_width(uint32_t all, F&& f) {
  if (all > kMapThreads) f(std::integral_constant<int, kMany>());
  else f(std::integral_constant<int, 1>());
}

// Pages that go back, on top of a stack of `count`; returns how many.  Workgroup `part` of `parts` moves every parts-th
// run of them (none: part < 0).  first_page, keep: LDS, a word a task of a round; tmp: as map_scan's; len, want: of the
// last round on return.
__device__ __forceinline__ uint32_t give_back(const PageMapArgs& a, uint32_t count, int part, int parts, uint32_t* first_page,
                                              int32_t* keep, uint32_t* tmp, int32_t (&len)[2], int32_t (&want)[2]) {
  const int tid = threadIdx.x;
  uint32_t back = 0;
  for (int t0 = 0; t0 < a.num_tasks; t0 += kMapTasks) {
    load_lengths(a, t0 + 2 * tid, len, want);
    uint32_t n[2], all;
#pragma unroll
    for (int c = 0; c < 2; ++c) n[c] = want[c] < len[c] ? (uint32_t)(pages_of(len[c]) - pages_of(want[c])) : 0u;
    // (a table has fewer than 2^31 entries, so these sums are exact)
    const uint32_t before = map_scan(n[0] + n[1], tmp, &all) - (n[0] + n[1]);
    if (all > 0 && part >= 0) {
      first_page[2 * tid] = before;
      first_page[2 * tid + 1] = before + n[0];
      keep[2 * tid] = want[0];
      keep[2 * tid + 1] = want[1];
      __syncthreads();
      const int tasks = min(kMapTasks, a.num_tasks - t0);
      by_width(all, [&](auto at_once) {
        constexpr int kAtOnce = decltype(at_once)::value;
        for (uint32_t j0 = tid + part * kAtOnce * kMapThreads; j0 < all; j0 += parts * kAtOnce * kMapThreads) {
          uint32_t j[kAtOnce];
          int i[kAtOnce];
          int32_t page[kAtOnce];
#pragma unroll
          for (int u = 0; u < kAtOnce; ++u) j[u] = min(j0 + u * kMapThreads, all - 1);
          last_at_most(first_page, tasks, j, i);
#pragma unroll
          for (int u = 0; u < kAtOnce; ++u)
            page[u] = a.block_table[(int64_t)(t0 + i[u]) * a.bt_stride + pages_of(keep[i[u]]) +
                                    (int32_t)(j[u] - first_page[i[u]])];
#pragma unroll
          for (int u = 0; u < kAtOnce; ++u) {
            const uint32_t at = sat_add(sat_add(count, back), j[u]);
            if (j0 + u * kMapThreads < all && at < (uint32_t)a.capacity) a.free_pages[at] = page[u];
          }
        }
      });
    }
    back = sat_add(back, all);
    __syncthreads();
  }
  return back;
}

__device__ __forceinline__ uint32_t free_now(const PageMapArgs& a) { return (uint32_t)min(max(*a.free_count, 0), a.capacity); }

// The pages that go back alone, by many workgroups, each of which scans all lengths.
__global__ __launch_bounds__(kMapThreads) void give_back_kernel(PageMapArgs a) {
  __shared__ uint32_t tmp[kMapThreads / 64], first_page[kMapTasks];
  __shared__ int32_t keep[kMapTasks];
  int32_t len[2], want[2];
  give_back(a, free_now(a), blockIdx.x, gridDim.x, first_page, keep, tmp, len, want);
}

__global__ __launch_bounds__(kMapThreads) void page_map_kernel(PageMapArgs a) {
  __shared__ uint32_t tmp[4][kMapThreads / 64];
  __shared__ uint32_t first_page[kMapTasks], first_row[kMapTasks];
  __shared__ int32_t len_of[kMapTasks], want_of[kMapTasks];  // want: that of the call, or the length where refused
  __shared__ uint32_t used;
  const int tid = threadIdx.x;
  const uint32_t count = free_now(a);
  if (tid == 0) used = 0;

  int32_t len[2], want[2];
  // sums of x over the tasks before each of a thread's two
  auto sums_before = [&](const uint32_t (&x)[2], uint32_t* scratch, uint32_t (&before)[2], uint32_t* all) {
    const uint32_t both = sat_add(x[0], x[1]), upto = map_scan(both, scratch, all);
    before[0] = upto - both;  // (callers whose sums may be cut off use the sums up to a task instead)
    before[1] = sat_add(before[0], x[0]);
    return upto;
  };

  const bool one_round = a.num_tasks <= kMapTasks;
  const uint32_t back = give_back(a, count, a.returns_apart ? -1 : 0, 1, first_page, len_of, tmp[0], len, want);
  const uint32_t there = min(sat_add(count, back), (uint32_t)a.capacity);

  // rows and pages of the tasks that grow
  uint32_t asked = 0, rows = 0, pages = 0;
  for (int t0 = 0; t0 < a.num_tasks; t0 += kMapTasks) {
    const int b = t0 + 2 * tid, tasks = min(kMapTasks, a.num_tasks - t0);
    if (!one_round) load_lengths(a, b, len, want);
    uint32_t e[2], p[2], in_r[2], in_p[2], all_e, all_r, all_p;
#pragma unroll
    for (int c = 0; c < 2; ++c) e[c] = want[c] > len[c] ? (uint32_t)(want[c] - len[c]) : 0u;
    // (sums may be cut off here: the one up to the thread's first task is taken from those before the thread)
    const uint32_t both = sat_add(e[0], e[1]);
    uint32_t upto = map_scan(both, tmp[1], &all_e);
    const uint32_t upto_prev = (uint32_t)__shfl_up((int)upto, 1, 64);
    uint32_t start = (tid & 63) ? upto_prev : 0;
    if ((tid & 63) == 0) {
#pragma unroll
      for (int w = 0; w < kMapThreads / 64; ++w) start = w < (tid >> 6) ? sat_add(start, tmp[1][w]) : start;
    }
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      start = sat_add(start, e[c]);
      if (sat_add(asked, start) > (uint32_t)a.num_rows) {  // no rows left: refused
        if (e[c]) want[c] = len[c];
        e[c] = 0;
      }
      p[c] = e[c] ? (uint32_t)(pages_of(want[c]) - pages_of(len[c])) : 0u;
    }
    sums_before(e, tmp[2], in_r, &all_r);  // (at most num_rows)
    sums_before(p, tmp[3], in_p, &all_p);
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const uint32_t end_p = sat_add(pages, in_p[c] + p[c]);
      const bool short_of = p[c] > 0 && end_p > there;
      if (p[c] > 0 && !short_of) atomicMax(&used, end_p);
      const int32_t to = short_of ? len[c] : want[c];
      first_row[2 * tid + c] = in_r[c];
      first_page[2 * tid + c] = in_p[c];
      len_of[2 * tid + c] = len[c];
      want_of[2 * tid + c] = to;
      if (b + c < a.num_tasks) {
        a.row_start[b + c] = (int32_t)(rows + in_r[c]);
        a.lens_out[b + c] = to;
      }
    }
    __syncthreads();
    const uint32_t granted = min(all_p, there - min(there, pages));  // pages this round may take, some refused
    auto take = [&](auto at_once) {
      constexpr int kAtOnce = decltype(at_once)::value;
      for (uint32_t j0 = tid; j0 < granted; j0 += kAtOnce * kMapThreads) {
        uint32_t j[kAtOnce];
        int i[kAtOnce];
        int32_t page[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
          j[u] = min(j0 + u * kMapThreads, granted - 1);
          page[u] = a.free_pages[there - 1 - pages - j[u]];
        }
        last_at_most(first_page, tasks, j, i);
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
          const int32_t lp = pages_of(len_of[i[u]]) + (int32_t)(j[u] - first_page[i[u]]);
          if (j0 + u * kMapThreads < granted && lp < pages_of(want_of[i[u]]))
            a.block_table[(int64_t)(t0 + i[u]) * a.bt_stride + lp] = page[u];
        }
      }
    };
    by_width(granted, take);
    auto write_rows = [&](auto at_once) {
      constexpr int kAtOnce = decltype(at_once)::value;
      for (uint32_t r0 = tid; r0 < all_r; r0 += kAtOnce * kMapThreads) {
        uint32_t r[kAtOnce];
        int i[kAtOnce];
        int32_t pos[kAtOnce], page[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) r[u] = min(r0 + u * kMapThreads, all_r - 1);
        last_at_most(first_row, tasks, r, i);
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
          const int32_t l = len_of[i[u]];
          pos[u] = l + (int32_t)(r[u] - first_row[i[u]]);
          // pages before `own` are the table's, the others new
          const int32_t lp = pos[u] / kPage, own = pages_of(l);
          page[u] = -1;
          if (pos[u] < want_of[i[u]])
            page[u] = lp < own ? a.block_table[(int64_t)(t0 + i[u]) * a.bt_stride + lp]
                               : a.free_pages[there - 1 - pages - first_page[i[u]] - (uint32_t)(lp - own)];
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
          if (r0 + u * kMapThreads >= all_r) continue;
          const bool ok = pos[u] < want_of[i[u]];
          put_row(a, rows + r[u], ok ? t0 + i[u] : -1, ok ? pos[u] : -1,
                  page[u] < 0 ? -1 : (int64_t)page[u] * kPage + pos[u] % kPage);
        }
      }
    };
    if (!a.rows_apart) by_width(all_r, write_rows);
    asked = sat_add(asked, all_e);
    rows += all_r;
    pages = sat_add(pages, all_p);
    __syncthreads();
  }
  if (tid == 0) {
    a.row_start[a.num_tasks] = (int32_t)rows;
    *a.free_count_out = (int32_t)(there - used);
  }
  if (!a.rows_apart)
    for (int64_t r = rows + tid; r < a.num_rows; r += kMapThreads) put_row(a, r, -1, -1, -1);
}

// The rows alone, from what the first kernel wrote: a granted task has lens_out == want and its new
// tokens end there.
__global__ __launch_bounds__(kRowThreads) void map_rows_kernel(PageMapArgs a) {
  __shared__ int32_t start[kRowTasks];
  const bool held = a.num_tasks <= kRowTasks;
  if (held) {
    for (int i = threadIdx.x; i < a.num_tasks; i += kRowThreads) start[i] = a.row_start[i];
    __syncthreads();
  }
  const int64_t r = (int64_t)blockIdx.x * kRowThreads + threadIdx.x;
  if (r >= a.num_rows) return;
  if (r >= a.row_start[a.num_tasks]) {
    put_row(a, r, -1, -1, -1);
    return;
  }
  const int b = held ? last_at_most(start, a.num_tasks, (int32_t)r)
                     : last_at_most((const int32_t*)a.row_start, a.num_tasks, (int32_t)r);
  const int32_t want = a.want[b], pos = want - (a.row_start[b + 1] - (int32_t)r);
  if (a.lens_out[b] != want) {
    put_row(a, r, -1, -1, -1);
    return;
  }
  const int32_t page = a.block_table[(int64_t)b * a.bt_stride + pos / kPage];
  put_row(a, r, b, pos, page < 0 ? -1 : (int64_t)page * kPage + pos % kPage);
}

}  // namespace kern

// Tables of this many entries have their returned pages moved by workgroups of their own, before the others: 2.8 us more
// where none return (1,056 tasks of 4k-8k: 13.4 and 16.2 us), less where some do (a tenth of 4k-8k 33 and 19, four tenths
// 95 and 16; a tenth of 16k-32k 92 and 19, four tenths 362 and 19).
constexpr int64_t kTableHere = 1 << 16;
constexpr uint32_t kReturnGroups = 128;

// One workgroup writes this many rows itself (256 tasks of 16, 32 and 64 rows each: 14.7, 17.3 and 22.9 us by it alone,
// 16.1 us each with the second kernel).
constexpr int32_t kRowsHere = 4096;

hipError_t launch_page_map(const PageMapArgs& args, hipStream_t stream) {
  PageMapArgs a = args;
  a.rows_apart = a.num_rows > kRowsHere;
  a.returns_apart = (int64_t)a.num_tasks * a.bt_stride >= kTableHere;
  if (a.returns_apart)
    hipLaunchKernelGGL(kern::give_back_kernel, dim3(kReturnGroups), dim3(kern::kMapThreads), 0, stream, a);
  hipLaunchKernelGGL(kern::page_map_kernel, dim3(1), dim3(kern::kMapThreads), 0, stream, a);
  hipError_t rc = hipGetLastError();
  if (rc != hipSuccess || !a.rows_apart) return rc;
  const int64_t blocks = ((int64_t)a.num_rows + kern::kRowThreads - 1) / kern::kRowThreads;
  hipLaunchKernelGGL(kern::map_rows_kernel, dim3((uint32_t)blocks), dim3(kern::kRowThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace tide
