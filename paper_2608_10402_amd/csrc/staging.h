// staging.h -- how an entry point hands its plan to its kernels and ends (tide_api.hip).
#pragma once

#include <hip/hip_runtime.h>

#include <mutex>

#include "plan.h"

namespace tide {

struct StagingSlot;

// Where a call's kernel finds its plan.
struct Staged {
  const uint8_t* plan = nullptr;  // the workspace, or a staging slot
  PlanReads reads = {nullptr, 0};
  StagingSlot* slot = nullptr;    // set with reads.done
  // the ring's, held with a slot until its reader is launched: until then another call that
  // came round to the slot would wait for flags that no kernel is there to set
  std::unique_lock<std::mutex> lock;
};

// A plan that at most this many workgroups read, once each, is read where it was staged: a
// record costs each a read of host memory (about 2 us), which is less than the copy kernel,
// its launch and the gap behind it (3-5 us on the GPU and 3 on the host): a four-task decode
// step went from 16.0 to 13.5 us, the smallest append + extend from 31 to 25.  Each workgroup
// pays for its own read, so the gain ends where an extend's workgroups come in rounds of the
// CUs: copied and in place, us a call (28 / 4 heads, d = 128), extends of 64 workgroups 18.5 and
// 16.5, 256 23.5 and 20.9, 512 38.3 and 38.9, 1,024 69.5 and 79, 2,000 134 and 145; appends of 512
// 20.8 and 18.3, 1,024 21.4 and 18.4; decodes (up to 256 workgroups at 4 kv heads) 2 us less.
constexpr uint32_t kInPlaceGroups = 512;

// Stages the plan.  readers: the workgroups of the one kernel that reads it, if it may be read
// in place (0: not).  Under debug checks the kernel needs the zeroed header, which keeps the
// copy into the workspace; under capture no staging slot is used.
int upload(const Plan& plan, void* workspace, hipStream_t stream, uint32_t readers, Staged* out);

// Ends a call whose kernels were launched with `launch_status`: releases the ring; under debug
// checks waits for the stream and reads the workspace's error flags.
int finish(hipError_t launch_status, Staged& st, void* workspace, hipStream_t stream);

// An extend of a plan made with its work lists: everything behind the arguments' checks.
int run_extend_plan(const Plan& plan, const void* q, const void* k_pool, const void* v_pool, int64_t num_pages,
                    const int32_t* block_table, int32_t bt_stride, const tide_dims& dims, void* out, float* lse,
                    void* workspace, hipStream_t stream, const void* k_new, const void* v_new);

// A number no other call of the process has, and no chance contents of a workspace: the count
// starts at a random 64-bit number.
uint64_t next_call();

template <class T>
const T* at(const void* ws, size_t off) {
  return reinterpret_cast<const T*>(static_cast<const uint8_t*>(ws) + off);
}

template <class T>
T* at_mut(void* ws, size_t off) {
  return reinterpret_cast<T*>(static_cast<uint8_t*>(ws) + off);
}

}  // namespace tide
