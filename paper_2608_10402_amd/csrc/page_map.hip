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
// One workgroup scans the tasks, 1,024 a round, and then writes pages and rows element by element: each
// finds its task by bisection of the sums in LDS, so one long task costs no more than many short ones.
// Above kRowsHere rows a second kernel writes the rows from the results of the first.
#include "kernels.h"
#include "tide_device.h"

namespace tide {
namespace kern {

constexpr int kMapThreads = 1024;
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

__device__ __forceinline__ int32_t pages_of(int32_t len) { return (int32_t)(((int64_t)len + kPage - 1) / kPage); }

__device__ __forceinline__ void put_row(const PageMapArgs& a, int64_t r, int32_t task, int32_t pos, int64_t slot) {
  a.row_task[r] = task;
  a.row_pos[r] = pos;
  a.row_slot[r] = slot;
}

__global__ __launch_bounds__(kMapThreads) void page_map_kernel(PageMapArgs a) {
  __shared__ uint32_t tmp[4][kMapThreads / 64];
  __shared__ uint32_t first_page[kMapThreads], first_row[kMapThreads];
  __shared__ int32_t len_of[kMapThreads], want_of[kMapThreads];  // want: that of the call, or the length where refused
  __shared__ uint32_t used;
  const int tid = threadIdx.x;
  const uint32_t count = (uint32_t)min(max(*a.free_count, 0), a.capacity);
  const int64_t most = (int64_t)a.bt_stride * kPage;
  if (tid == 0) used = 0;

  auto load = [&](int b, int32_t* len, int32_t* want) {  // a task whose lengths are no lengths stays as it is
    *len = *want = 0;
    if (b >= a.num_tasks) return;
    *len = a.lens[b];
    *want = a.want[b];
    if (*len < 0 || *len > most || *want < 0 || *want > most) *want = *len;
  };

  // pages that go back, on top of the stack
  uint32_t back = 0;
  for (int t0 = 0; t0 < a.num_tasks; t0 += kMapThreads) {
    int32_t len, want;
    load(t0 + tid, &len, &want);
    const uint32_t n = want < len ? (uint32_t)(pages_of(len) - pages_of(want)) : 0u;
    uint32_t all;
    const uint32_t in = map_scan(n, tmp[0], &all);
    first_page[tid] = in - n;  // (a table has fewer than 2^31 entries, so these sums are exact)
    len_of[tid] = want;
    __syncthreads();
    const int tasks = min(kMapThreads, a.num_tasks - t0);
    for (uint32_t j = tid; j < all; j += kMapThreads) {
      const int i = last_at_most(first_page, tasks, j);
      const uint32_t at = sat_add(sat_add(count, back), j);
      if (at < (uint32_t)a.capacity)
        a.free_pages[at] = a.block_table[(int64_t)(t0 + i) * a.bt_stride + pages_of(len_of[i]) + (int32_t)(j - first_page[i])];
    }
    back = sat_add(back, all);
    __syncthreads();
  }
  const uint32_t there = min(sat_add(count, back), (uint32_t)a.capacity);

  // rows and pages of the tasks that grow
  uint32_t asked = 0, rows = 0, pages = 0;
  for (int t0 = 0; t0 < a.num_tasks; t0 += kMapThreads) {
    const int b = t0 + tid, tasks = min(kMapThreads, a.num_tasks - t0);
    int32_t len, want;
    load(b, &len, &want);
    uint32_t e = want > len ? (uint32_t)(want - len) : 0u, all_e, all_r, all_p;
    const uint32_t end_e = sat_add(asked, map_scan(e, tmp[1], &all_e));
    if (end_e > (uint32_t)a.num_rows) {  // no rows left: refused
      if (e) want = len;
      e = 0;
    }
    const uint32_t p = e ? (uint32_t)(pages_of(want) - pages_of(len)) : 0u;
    const uint32_t in_r = map_scan(e, tmp[2], &all_r), in_p = map_scan(p, tmp[3], &all_p);
    const uint32_t end_p = sat_add(pages, in_p);
    const bool short_of = p > 0 && end_p > there;
    if (p > 0 && !short_of) atomicMax(&used, end_p);
    first_row[tid] = in_r - e;
    first_page[tid] = in_p - p;
    len_of[tid] = len;
    want_of[tid] = short_of ? len : want;
    if (b < a.num_tasks) {
      a.row_start[b] = (int32_t)(rows + in_r - e);
      a.lens_out[b] = short_of ? len : want;
    }
    __syncthreads();
    const uint32_t granted = min(all_p, there - min(there, pages));  // pages this round may take, some refused
    for (uint32_t j = tid; j < granted; j += kMapThreads) {
      const int i = last_at_most(first_page, tasks, j);
      const int32_t lp = pages_of(len_of[i]) + (int32_t)(j - first_page[i]);
      if (lp < pages_of(want_of[i]))
        a.block_table[(int64_t)(t0 + i) * a.bt_stride + lp] = a.free_pages[there - 1 - pages - j];
    }
    if (!a.rows_apart)
      for (uint32_t r = tid; r < all_r; r += kMapThreads) {
        const int i = last_at_most(first_row, tasks, r);
        const int32_t l = len_of[i], pos = l + (int32_t)(r - first_row[i]);
        if (pos >= want_of[i]) {
          put_row(a, rows + r, -1, -1, -1);
          continue;
        }
        const int32_t lp = pos / kPage, own = pages_of(l);  // pages before `own` are the table's, the others new
        const int32_t page = lp < own ? a.block_table[(int64_t)(t0 + i) * a.bt_stride + lp]
                                      : a.free_pages[there - 1 - pages - first_page[i] - (uint32_t)(lp - own)];
        put_row(a, rows + r, t0 + i, pos, page < 0 ? -1 : (int64_t)page * kPage + pos % kPage);
      }
    asked = sat_add(asked, all_e);
    rows += all_r;  // (at most num_rows)
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

// One workgroup writes this many rows itself.
constexpr int32_t kRowsHere = 4096;

hipError_t launch_page_map(const PageMapArgs& args, hipStream_t stream) {
  PageMapArgs a = args;
  a.rows_apart = a.num_rows > kRowsHere;
  hipLaunchKernelGGL(kern::page_map_kernel, dim3(1), dim3(kern::kMapThreads), 0, stream, a);
  hipError_t rc = hipGetLastError();
  if (rc != hipSuccess || !a.rows_apart) return rc;
  const int64_t blocks = ((int64_t)a.num_rows + kern::kRowThreads - 1) / kern::kRowThreads;
  hipLaunchKernelGGL(kern::map_rows_kernel, dim3((uint32_t)blocks), dim3(kern::kRowThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace tide
