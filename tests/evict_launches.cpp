// The launches of an eviction (the host half of kv_evict.hip, linked with the HIP calls that it makes) for
// few and for very many (task, kv head) pairs: each has less than 2^32 threads, and together they
// cover every pair once with either kernel.  Prints "ok", or what went wrong.
#include <hip/hip_runtime_api.h>
#include <stdio.h>
#include <string.h>

#include <map>
#include <string>
#include <vector>

#include "kernels.h"

static std::map<const void*, std::string> names;
struct Launch {
  std::string name;
  dim3 grid, block;
  tide::EvictArgs args;
};
static std::vector<Launch> launches;
static dim3 g_grid, g_block;

extern "C" {
void** __hipRegisterFatBinary(const void*) { static void* h; return &h; }
void __hipUnregisterFatBinary(void**) {}
void __hipRegisterFunction(void**, const void* f, char*, const char* name, unsigned, uint3*, uint3*, dim3*, dim3*, int*) {
  names[f] = name;
}
void __hipRegisterVar(void**, void*, char*, char*, int, size_t, int, int) {}
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t, hipStream_t) {
  g_grid = grid, g_block = block;
  return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3* g, dim3* b, size_t* n, hipStream_t* s) {
  *g = g_grid, *b = g_block, *n = 0, *s = nullptr;
  return hipSuccess;
}
hipError_t hipLaunchKernel(const void* f, dim3 grid, dim3 block, void** args, size_t, hipStream_t) {
  Launch l = {names[f], grid, block, {}};
  memcpy(&l.args, args[0], sizeof(l.args));
  launches.push_back(l);
  return hipSuccess;
}
hipError_t hipGetLastError() { return hipSuccess; }
}

int main() {
  int bad = 0;
  const int shapes[][2] = {{1, 1}, {64, 4}, {16, 65536}, {700, 2500}, {1 << 20, 1}, {4000, 512}, {(1 << 29) - 1, 1}};
  static int32_t table[2];
  for (const auto& sh : shapes)
    for (int d : {64, 128})
      for (int kv4 = 0; kv4 < 2; ++kv4)
        for (int in_place = 0; in_place < 2; ++in_place) {
          launches.clear();
          tide::EvictArgs a = {};
          a.num_tasks = sh[0], a.num_kv_heads = sh[1], a.longest_keep = 5000;
          a.block_table = table, a.new_table = in_place ? table : table + 1;
          if (tide::launch_evict(a, d, kv4, nullptr) != hipSuccess) printf("not launched\n"), ++bad;
          int64_t pairs[2] = {0, 0};
          for (const Launch& l : launches) {
            const bool move = l.name.find("evict_move_kernel") != std::string::npos;
            if (!move && l.name.find("evict_select_kernel") == std::string::npos) printf("%s?\n", l.name.c_str()), ++bad;
            if ((uint64_t)l.grid.x * l.block.x >> 32 || l.grid.y > 65535 || l.grid.z != 1)
              printf("%d tasks x %d heads: %u x %u threads\n", sh[0], sh[1], l.grid.x, l.block.x), ++bad;
            const unsigned per = !move ? 1 : in_place && (kv4 || d == 128) ? 4 : 2;  // workgroups of a pair
            if (!move && pairs[1]) printf("a select behind a move\n"), ++bad;
            if (l.grid.x % per || l.args.first_pair != pairs[move]) printf("pairs are left out\n"), ++bad;
            pairs[move] += l.grid.x / per;
          }
          const int64_t all = (int64_t)sh[0] * sh[1];
          if (pairs[0] != all || pairs[1] != all) printf("%lld, %lld pairs of %lld\n", (long long)pairs[0], (long long)pairs[1], (long long)all), ++bad;
          if (bad > 9) return 1;
        }
  if (!bad) printf("ok\n");
  return bad != 0;
}
