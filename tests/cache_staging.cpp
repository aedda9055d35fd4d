// Launches that report an error although a kernel that reads a staging slot is queued, on the CPU:
// the host halves of tide_api.hip and cache_api.hip, linked with the HIP calls that they make and the
// kernel launches replaced by the functions below.
//
// A queued kernel runs when its stream is waited for, or else at the very end.  Whenever it runs it has
// to find the plan of its own call.  An eviction whose second launch fails has queued the first, which
// reads the plan in its slot; a copy whose launch is said to have failed (an error that an earlier call
// of the program left behind) is queued all the same.  Either way more calls than the ring has slots
// follow.  Prints "ok", or what went wrong.
#include <hip/hip_runtime_api.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <functional>
#include <vector>

#include "kernels.h"
#include "tide.h"

static std::vector<std::function<void()>> queued;
static bool fail_second = false, stale_error = false;
static int bad = 0;

static void run_queued() {
  std::vector<std::function<void()>> now;
  now.swap(queued);
  for (auto& f : now) f();
}

// ---- HIP, as far as the two files call it -------------------------------------------------
extern "C" {
void** __hipRegisterFatBinary(const void*) { static void* h; return &h; }
void __hipUnregisterFatBinary(void**) {}
void __hipRegisterFunction(void**, const void*, char*, const char*, unsigned, uint3*, uint3*, dim3*, dim3*, int*) {}
void __hipRegisterVar(void**, void*, char*, char*, int, size_t, int, int) {}
static dim3 g_grid;
hipError_t __hipPushCallConfiguration(dim3 grid, dim3, size_t, hipStream_t) { g_grid = grid; return hipSuccess; }
hipError_t __hipPopCallConfiguration(dim3* g, dim3* b, size_t* n, hipStream_t* s) {
  *g = g_grid, *b = dim3(256), *n = 0, *s = nullptr;
  return hipSuccess;
}
// the one kernel launched here is the copy: dst, src, 16-byte pieces, flags, use count
hipError_t hipLaunchKernel(const void*, dim3 grid, dim3, void** args, size_t, hipStream_t) {
  void* dst = *(void**)args[0];
  const void* src = *(const void**)args[1];
  const size_t bytes = *(size_t*)args[2] * 16;
  uint32_t* done = *(uint32_t**)args[3];
  const uint32_t seq = *(uint32_t*)args[4];
  const std::vector<uint8_t> sent((const uint8_t*)src, (const uint8_t*)src + bytes);
  auto copy = [=] {
    memcpy(dst, src, bytes);
    if (memcmp(dst, sent.data(), bytes)) printf("a queued copy read another call's plan\n"), ++bad;
    for (unsigned b = 0; b < grid.x; ++b) done[b] = seq;
  };
  if (stale_error) queued.push_back(copy);
  else copy();
  return hipSuccess;
}
hipError_t hipDeviceSynchronize() { run_queued(); return hipSuccess; }
hipError_t hipStreamSynchronize(hipStream_t) { run_queued(); return hipSuccess; }
hipError_t hipGetDevice(int* d) { *d = 0; return hipSuccess; }
hipError_t hipGetLastError() {
  const bool e = stale_error;
  stale_error = false;
  return e ? hipErrorUnknown : hipSuccess;
}
hipError_t hipGetSymbolAddress(void**, const void*) { return hipErrorUnknown; }
hipError_t hipHostMalloc(void** p, size_t n, unsigned) { *p = malloc(n); return hipSuccess; }
hipError_t hipHostFree(void* p) { free(p); return hipSuccess; }
hipError_t hipHostGetDevicePointer(void** d, void* h, unsigned) { *d = h; return hipSuccess; }
hipError_t hipMemcpy(void*, const void*, size_t, hipMemcpyKind) { return hipErrorUnknown; }
hipError_t hipMemcpyAsync(void*, const void*, size_t, hipMemcpyKind, hipStream_t) { return hipErrorUnknown; }
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus* s) {
  *s = hipStreamCaptureStatusNone;
  return hipSuccess;
}
}

// ---- launches -------------------------------------------------------------------------------
namespace tide {
int append_groups(int32_t num_kv_heads) { return (num_kv_heads + 3) / 4; }
int append_waves() { return 4; }
int decode_waves(int32_t) { return 4; }
int kv4_store_groups(int32_t num_kv_heads) { return (num_kv_heads + 3) / 4; }
hipError_t launch_extend(const ExtendArgs&, int, int, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_decode(const DecodeArgs&, int, bool, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_decode_stream(const StreamArgs&, int, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_kv4_store(const Kv4StoreArgs&, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_kv4_stage(const Kv4StageArgs&, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_kv4_decode(const Kv4AttnArgs&, int, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_attn_mass(const MassArgs&, int, bool, hipStream_t) { return hipErrorUnknown; }
// (a call here is read in place where it is small, else from the workspace)
hipError_t launch_kv_append(const AppendArgs& a, hipStream_t) {
  if (a.reads.done)
    for (int i = 0; i < a.num_items * append_groups(a.num_kv_heads); ++i) a.reads.done[i] = a.reads.seq;
  return hipSuccess;
}
hipError_t launch_evict(const EvictArgs& a, int, bool, hipStream_t) {
  const EvictTask sent = a.tasks[0];
  queued.push_back([=] {
    if (memcmp(a.tasks, &sent, sizeof(sent))) printf("a queued select read another call's plan\n"), ++bad;
    if (a.reads.done)
      for (int i = 0; i < a.num_tasks * a.num_kv_heads; ++i) a.reads.done[i] = a.reads.seq;
  });
  if (fail_second) return hipErrorInvalidConfiguration;  // of the move's launch
  run_queued();
  return hipSuccess;
}
}  // namespace tide

alignas(16) static uint8_t mem[1 << 20], ws[1 << 20];
static const tide_dims dims = {4, 4, 64, 16, 0.125f};

static int append(int tasks) {
  const std::vector<int32_t> prefix(tasks, 0), extend(tasks, 3);
  return tide_kv_append(mem, mem, mem, mem, 64, reinterpret_cast<const int32_t*>(mem), 64, tasks, prefix.data(),
                        extend.data(), &dims, ws, sizeof(ws), nullptr);
}

static int evict() {
  const int32_t len[1] = {40}, keep[1] = {20};
  return tide_kv_evict(mem, mem, reinterpret_cast<float*>(mem), 64, reinterpret_cast<const int32_t*>(mem), 64, nullptr,
                       0, 1, len, keep, nullptr, &dims, nullptr, ws, sizeof(ws), nullptr);
}

static void others(const char* after) {
  for (int i = 0; i < 40 && !bad; ++i)
    if (append(1) != TIDE_OK) printf("call %d after %s failed\n", i, after), ++bad;
  run_queued();
}

int main() {
  setenv("TIDE_STAGING_WAIT_US", "0", 1);
  unsetenv("TIDE_DEBUG_CHECKS");
  if (evict() != TIDE_OK) printf("an eviction failed\n"), ++bad;
  fail_second = true;
  if (evict() != TIDE_ERR_HIP) printf("a failed second launch was not reported\n"), ++bad;
  fail_second = false;
  others("a failed second launch");
  // 600 workgroups: their plan is copied
  if (append(600) != TIDE_OK) printf("a copied call failed\n"), ++bad;
  stale_error = true;
  if (append(600) != TIDE_ERR_HIP) printf("the error behind a copy was not reported\n"), ++bad;
  others("a copy with an error");
  tide_shutdown();
  if (!bad) printf("ok\n");
  return bad != 0;
}
