// Eviction by accumulated attention weight: per task and kv head, which cached positions stay (the
// last `recent` and the heaviest of the others, equal sums by position), and their move to the
// front of the task's pages, or of new ones, in order.
//
// Select: one workgroup per (task, kv head).  Sums become 32-bit keys that order like them (NaN
// lowest); three passes over the task's keys count 11, 11 and 10 bits of those that match the
// digits found so far and so find the smallest key that stays, and how many of its equals; a last
// pass ranks what stays by prefix sums and writes an EvictIndex for each, in order.
//
// Move: K and V rows go from their position to their rank.  Ranks never exceed positions, so in
// place a workgroup that loads a chunk of rows, waits for all of them (a barrier) and only then
// stores them is right if it takes its chunks in order: later chunks read positions beyond every
// slot written so far, which also lets it load the next chunk before it stores one.  Into new pages
// the chunks are independent and go to workgroups of their own.  The largest tasks come first.
#include "kernels.h"
#include "kv4.h"

namespace tide {
namespace kern {

constexpr int kSelect = 1024;  // threads
constexpr int kBins = 2048;
constexpr int kHeld = 5;  // chunks of 4 kSelect keys that the threads hold: contexts of up to 20,480 are read once to count

__device__ __forceinline__ uint32_t order_key(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x + 0.0f);  // -0 counts as 0
  if ((u & 0x7FFFFFFFu) > 0x7F800000u) return 0;
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ uint32_t wave_scan(uint32_t x, int lane) {  // inclusive
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    const uint32_t y = __shfl_up((int)x, o, 64);
    if (lane >= o) x += y;
  }
  return x;
}

// Sum of x over the threads before this one; *all: over all.  tmp: 16 words, free again after the
// next barrier.
__device__ __forceinline__ uint32_t block_scan(uint32_t x, uint32_t* tmp, uint32_t* all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t in = wave_scan(x, lane);
  if (lane == 63) tmp[wave] = in;
  __syncthreads();
  uint32_t before = 0, total = 0;
#pragma unroll
  for (int w = 0; w < kSelect / 64; ++w) {
    const uint32_t t = tmp[w];
    if (w < wave) before += t;
    total += t;
  }
  *all = total;
  return before + in - x;
}

__global__ __launch_bounds__(kSelect) void evict_select_kernel(EvictArgs a) {
  __shared__ uint32_t hist[kBins];
  __shared__ uint32_t tmp[2][kSelect / 64];
  __shared__ uint32_t found[3];  // digit, keys above it, keys with it
  const int tid = threadIdx.x;
  const int pair = a.first_pair + blockIdx.x, unit = pair / a.num_kv_heads, head = pair - unit * a.num_kv_heads;
  __shared__ EvictTask task;
  if (tid == 0) task = a.tasks[unit];
  __syncthreads();
  const EvictTask t = task;
  if (tid == 0) {
    if (a.reads.done) plan_read(a.reads, pair);
    if (head == 0) a.move_tasks[unit] = t;  // for the move, which comes after the slot's release
  }
  const int32_t* row = a.block_table + (int64_t)t.task * a.bt_stride;
  const int n = t.kv_len, cand = n - t.recent, want = t.keep - t.recent;

  // the keys of positions p .. p + 3 (p a multiple of 4, below n)
  auto load4 = [&](int p, uint32_t (&key)[4], float (&m)[4], int32_t* page) {
    const int32_t g = row[p / kPage];
    const bool ok = g >= 0 && g < a.num_pages;
    f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
    if (ok) x = *reinterpret_cast<const f32x4*>(a.mass + ((int64_t)g * a.num_kv_heads + head) * kPage + p % kPage);
    else atomicOr(a.error_flags, 1);
#pragma unroll
    for (int i = 0; i < 4; ++i) m[i] = x[i], key[i] = ok ? order_key(x[i]) : 0;
    *page = ok ? g : -1;
  };

  // the `want` largest keys of the candidates: those above `least`, and the first `equal` equals
  uint32_t least = 0, equal = 0;
  if (want > 0 && want < cand) {
    uint32_t held[kHeld][4];
#pragma unroll
    for (int c = 0; c < kHeld; ++c) {
      const int p = 4 * (tid + c * kSelect);
      float m[4];
      int32_t page;
      if (p < cand) load4(p, held[c], m, &page);
    }
    uint32_t prefix = 0, mask = 0, rest = want;
    constexpr int kShift[3] = {21, 10, 0}, kWidth[3] = {11, 11, 10};
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
      for (int i = tid; i < kBins; i += kSelect) hist[i] = 0;
      __syncthreads();
      const uint32_t digits = (1u << kWidth[pass]) - 1;
      auto count = [&](const uint32_t (&key)[4], int p) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (p + i < cand && (key[i] & mask) == prefix) atomicAdd(&hist[(key[i] >> kShift[pass]) & digits], 1u);
      };
#pragma unroll
      for (int c = 0; c < kHeld; ++c) count(held[c], 4 * (tid + c * kSelect));
      for (int p = 4 * (tid + kHeld * kSelect); p < cand; p += 4 * kSelect) {
        uint32_t key[4];
        float m[4];
        int32_t page;
        load4(p, key, m, &page);
        count(key, p);
      }
      __syncthreads();
      // bins from the largest digit down, two a thread
      const uint32_t hi = hist[kBins - 1 - 2 * tid], lo = hist[kBins - 2 - 2 * tid];
      uint32_t all;
      const uint32_t before = block_scan(hi + lo, tmp[0], &all);
      if (before < rest && before + hi >= rest)
        found[0] = kBins - 1 - 2 * tid, found[1] = before, found[2] = hi;
      else if (before + hi < rest && before + hi + lo >= rest)
        found[0] = kBins - 2 - 2 * tid, found[1] = before + hi, found[2] = lo;
      __syncthreads();
      prefix |= found[0] << kShift[pass];
      mask |= digits << kShift[pass];
      rest -= found[1];
      if (rest == found[2]) {  // every key that begins with these digits stays
        rest = 0;
        --prefix;  // (not 0: some candidate does not stay)
        break;
      }
      __syncthreads();  // (before found is written again)
    }
    least = prefix;
    equal = rest;
  }
  const bool all_stay = want == cand;

  const int64_t out0 = (int64_t)t.first * a.num_kv_heads + (int64_t)head * t.keep;
  const int32_t* to_row = a.new_table + (int64_t)t.task * a.new_stride;
  uint32_t above = 0, equals = 0;  // positions before the chunk
  int flip = 0;
  for (int p0 = 0; p0 < n; p0 += 4 * kSelect, flip ^= 1) {
    const int p = p0 + 4 * tid;
    uint32_t key[4] = {0, 0, 0, 0};
    float m[4];
    int32_t page = -1;
    if (p < n) load4(p, key, m, &page);
    uint32_t gt = 0, eq = 0;  // bit i: position p + i
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool c = p + i < cand, late = !c && p + i < n;
      if (late || (c && want > 0 && (all_stay || key[i] > least))) gt |= 1u << i;
      else if (c && want > 0 && key[i] == least) eq |= 1u << i;
    }
    uint32_t all;
    const uint32_t before = block_scan(__popc(gt) | (__popc(eq) << 16), tmp[flip], &all);
    uint32_t g = above + (before & 0xFFFFu), e = equals + (before >> 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool is_eq = eq >> i & 1;
      if ((gt >> i & 1) || (is_eq && e < equal)) {
        const int rank = (int)(g + min(e, equal));
        const int32_t to = to_row[rank / kPage];
        const bool ok = to >= 0 && to < a.num_pages;
        if (!ok) atomicOr(a.error_flags, 1);
        a.index[out0 + rank] = EvictIndex{p + i, ok ? page : -1, to, m[i]};
        if (a.kept) a.kept[((int64_t)t.first + rank) * a.num_kv_heads + head] = p + i;
      }
      g += gt >> i & 1;
      e += is_eq;
    }
    above += all & 0xFFFFu;
    equals += all >> 16;
  }
}

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

constexpr int kMove = 1024;  // threads
// Workgroups that share a (task, kv head)'s K or V rows, and the rows that a thread has under way in each
// of two chunks.  In place chunks follow each other, so the longest tasks are the call's end and a lone
// task is a chain of latencies: two workgroups take half of each row (one line of 128 bytes).  Into new
// pages the chunks themselves are spread.  Call us on fresh sums, half of the positions kept (64 tasks of
// 2k-16k, 28 / 4 heads, d = 128, bf16, in place | the same into new pages | one task of 30k in place | 64
// tasks, 32 / 8 heads, 4 bits, in place with 260 for reading the rows back):
//   whole rows, 4 under way         335 | 309 | 171 | 690
//   half rows, 4                    297 | 348 | 112 | 681
//   half rows, 2                    306 | 311 | 125 | 656
//   whole rows, 2                         295
// 512 threads are 4-15% slower than 1024 in place.  The first takes 42 us to select and 255 to move 1.2 GB,
// the rate of a large copy (4.8 TB/s).  4-bit rows are pieces of 16 and 4 bytes all over their pages, so every
// line of a page is read for the half of it that stays, and lines are read and written in parts: without the
// reading back 356 us in place and 425 into new pages, of 135 for the bytes that stay.  Few long tasks leave
// most of the device idle, a chain of chunks per workgroup: the one of 30k takes 112 us of 13 for its bytes.
template <int D, bool kKv4, bool kInPlace>
constexpr int move_parts = kInPlace && (kKv4 || D == 128) ? 2 : 1;
template <bool kKv4, bool kInPlace>
constexpr int move_in_flight = kInPlace && !kKv4 ? 4 : 2;

// The pieces of one token's K or V row: kLanes of kBytes each.
// Pieces of kRun slots lie next to each other.
template <int D, bool kKv4, bool kV>
struct MoveRow {
  static constexpr int kLanes = kKv4 ? (kV ? 16 : 4) : D / 8;
  static constexpr int kBytes = kKv4 ? (kV ? D / 32 : D / 8) : 16;
  static constexpr int kRun = kKv4 ? (kV ? 4 : 16) : 1;
};

template <int kBytes>
struct MovePiece {
  uint32_t w[kBytes < 4 ? 1 : kBytes / 4];
  __device__ __forceinline__ void load(const uint8_t* p) {
    if constexpr (kBytes == 16) {
      const u32x4 x = load_u32x4(p);
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = x[i];
    } else if constexpr (kBytes == 8) {
      const uint2 x = *reinterpret_cast<const uint2*>(p);
      w[0] = x.x, w[1] = x.y;
    } else if constexpr (kBytes == 4) {
      w[0] = *reinterpret_cast<const uint32_t*>(p);
    } else {
      w[0] = *reinterpret_cast<const uint16_t*>(p);
    }
  }
  __device__ __forceinline__ void store(uint8_t* p) const {
    if constexpr (kBytes == 16) store_u32x4(p, u32x4{w[0], w[1], w[2], w[3]});
    else if constexpr (kBytes == 8) *reinterpret_cast<uint2*>(p) = uint2{w[0], w[1]};
    else if constexpr (kBytes == 4) *reinterpret_cast<uint32_t*>(p) = w[0];
    else *reinterpret_cast<uint16_t*>(p) = (uint16_t)w[0];
  }
};

template <int D, bool kKv4, bool kV, bool kInPlace>
__device__ __forceinline__ void move_rows(const EvictArgs& a, const EvictTask& t, int head, int part, int chunk_first,
                                          int chunk_step) {
  using M = MoveRow<D, kKv4, kV>;
  using F = Kv4<D>;
  constexpr int kInFlight = move_in_flight<kKv4, kInPlace>;
  constexpr int kLanes = M::kLanes / move_parts<D, kKv4, kInPlace>, kRun = M::kRun;
  constexpr int kRows = kMove / kLanes;  // rows a load
  constexpr int kChunk = kRows * kInFlight;
  const int lane = part * kLanes + threadIdx.x / kRun % kLanes;  // piece
  const int r0 = threadIdx.x / (kRun * kLanes) * kRun + threadIdx.x % kRun;
  const int64_t out0 = (int64_t)t.first * a.num_kv_heads + (int64_t)head * t.keep;
  uint8_t* pool = kV && !kKv4 ? a.v_pool : a.k_pool;
  constexpr int64_t kBlk = kKv4 ? F::kBlock : (int64_t)kPage * D * 2;
  auto piece_at = [&](int32_t page, int slot) {
    uint8_t* blk = pool + ((int64_t)page * a.num_kv_heads + head) * kBlk;
    if constexpr (!kKv4) return blk + slot * D * 2 + 16 * lane;
    else if constexpr (kV) return blk + F::v_word(lane, slot);
    else return blk + (16 * lane + slot) * F::kLane;
  };
  // the scale byte that goes with this lane's piece, where it is the lane that moves it
  const bool scale_lane = kKv4 && (kV ? lane % F::kVLanes == 0 : D == 128 || lane % 2 == 0);
  auto scale_at = [&](int32_t page, int slot) {
    uint8_t* blk = pool + ((int64_t)page * a.num_kv_heads + head) * kBlk;
    if constexpr (kV) return blk + F::v_scale(16 * (slot >> 2) + lane) + (slot & 3);
    else return blk + F::k_scale(16 * lane + slot);
  };
  struct Chunk {
    MovePiece<M::kBytes> x[kInFlight];
    uint32_t scale[kInFlight];
    int32_t to[kInFlight];  // page, or -1: not moved
  };
  i32x4 rec[kInFlight];  // EvictIndex of the next chunk's rows
  auto fetch = [&](int c0) {
#pragma unroll
    for (int i = 0; i < kInFlight; ++i) {
      const int r = c0 + i * kRows + r0;
      rec[i] = *reinterpret_cast<const i32x4*>(a.index + out0 + min(r, t.keep - 1));
    }
  };
  auto load = [&](Chunk& c, int c0) {
#pragma unroll
    for (int i = 0; i < kInFlight; ++i) {
      const int r = c0 + i * kRows + r0, pos = rec[i][0], from = rec[i][1], to = rec[i][2];
      c.to[i] = -1;
      if (r < t.keep && from >= 0 && (from != to || pos % kPage != r % kPage)) {
        c.to[i] = to;
        c.x[i].load(piece_at(from, pos % kPage));
        if (scale_lane) c.scale[i] = *scale_at(from, pos % kPage);
      }
    }
    fetch(c0 + chunk_step * kChunk);
  };
  auto store = [&](const Chunk& c, int c0) {
#pragma unroll
    for (int i = 0; i < kInFlight; ++i) {
      const int slot = (c0 + i * kRows + r0) % kPage;
      if (c.to[i] < 0) continue;
      c.x[i].store(piece_at(c.to[i], slot));
      if (scale_lane) *scale_at(c.to[i], slot) = (uint8_t)c.scale[i];
    }
  };
  // this thread's rows of the chunk are in registers
  auto arrive = [](Chunk& c) {
#pragma unroll
    for (int i = 0; i < kInFlight; ++i) {
      asm volatile("" : "+v"(c.scale[i])::"memory");
#pragma unroll
      for (int w = 0; w < (int)(sizeof(c.x[0].w) / 4); ++w) asm volatile("" : "+v"(c.x[i].w[w])::"memory");
    }
  };
  const int step = chunk_step * kChunk;
  if (chunk_first * kChunk >= t.keep) return;
  Chunk even, odd;
  fetch(chunk_first * kChunk);
  load(even, chunk_first * kChunk);
  for (int c0 = chunk_first * kChunk; c0 < t.keep; c0 += 2 * step) {
    load(odd, c0 + step);
    arrive(even);
    __syncthreads();
    store(even, c0);
    if (c0 + step >= t.keep) break;
    load(even, c0 + 2 * step);
    arrive(odd);
    __syncthreads();
    store(odd, c0 + step);
  }
}

// The kept positions' sums, to the slots of their ranks (read from the index: no order needed).
__device__ __forceinline__ void move_mass(const EvictArgs& a, const EvictTask& t, int head, int first, int step) {
  const int64_t out0 = (int64_t)t.first * a.num_kv_heads + (int64_t)head * t.keep;
  for (int r = first; r < t.keep; r += step) {
    const EvictIndex x = a.index[out0 + r];
    if (x.from >= 0) a.mass[((int64_t)x.to * a.num_kv_heads + head) * kPage + r % kPage] = x.mass;
  }
}

// grid: (task, from the largest, kv head, part of the rows, K or V with the sums) x chunk groups
template <int D, bool kKv4, bool kInPlace>
__global__ __launch_bounds__(kMove) void evict_move_kernel(EvictArgs a) {
  constexpr int kParts = move_parts<D, kKv4, kInPlace>;
  const int x = a.first_pair + blockIdx.x / (2 * kParts), part = blockIdx.x / 2 % kParts;
  const int nth = x / a.num_kv_heads, head = x - nth * a.num_kv_heads;
  const EvictTask t = a.move_tasks[a.move_tasks[nth].nth];
  if (blockIdx.x % 2 == 0) {
    move_rows<D, kKv4, false, kInPlace>(a, t, head, part, blockIdx.y, gridDim.y);
  } else {
    move_rows<D, kKv4, true, kInPlace>(a, t, head, part, blockIdx.y, gridDim.y);
    if (part == 0) move_mass(a, t, head, blockIdx.y * kMove + threadIdx.x, gridDim.y * kMove);
  }
}

// Both kernels over all pairs, as many a launch as leave it less than 2^32 threads.
template <int D, bool kKv4>
hipError_t launch(EvictArgs a, hipStream_t stream) {
  const bool in_place = a.new_table == a.block_table;
  const int64_t pairs = (int64_t)a.num_tasks * a.num_kv_heads;
  auto in_turn = [&](int groups, int threads, auto&& kernel) {  // groups: workgroups of a pair
    const int64_t most = (((int64_t)1 << 32) - 1) / (groups * threads);
    for (int64_t at = 0; at < pairs; at += most) {
      a.first_pair = (int32_t)at;
      kernel((unsigned)(min(most, pairs - at) * groups));
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    return hipSuccess;
  };
  const hipError_t e = in_turn(1, kSelect, [&](unsigned n) {
    hipLaunchKernelGGL(evict_select_kernel, dim3(n), dim3(kSelect), 0, stream, a);
  });
  if (e != hipSuccess) return e;
  if (in_place)
    return in_turn(2 * move_parts<D, kKv4, true>, kMove, [&](unsigned n) {
      hipLaunchKernelGGL((evict_move_kernel<D, kKv4, true>), dim3(n), dim3(kMove), 0, stream, a);
    });
  return in_turn(2, kMove, [&](unsigned n) {
    hipLaunchKernelGGL((evict_move_kernel<D, kKv4, false>), dim3(n, (unsigned)min(64, (a.longest_keep + 255) / 256)),
                       dim3(kMove), 0, stream, a);
  });
}

// Every variant is instantiated explicitly (see attn_decode.hip).
template __global__ void evict_move_kernel<128, false, false>(EvictArgs);
template __global__ void evict_move_kernel<128, false, true>(EvictArgs);
template __global__ void evict_move_kernel<128, true, false>(EvictArgs);
template __global__ void evict_move_kernel<128, true, true>(EvictArgs);
template __global__ void evict_move_kernel<64, false, false>(EvictArgs);
template __global__ void evict_move_kernel<64, false, true>(EvictArgs);
template __global__ void evict_move_kernel<64, true, false>(EvictArgs);
template __global__ void evict_move_kernel<64, true, true>(EvictArgs);

}  // namespace kern

hipError_t launch_evict(const EvictArgs& a, int head_dim, bool kv4, hipStream_t stream) {
  if (a.num_tasks == 0) return hipSuccess;
  if (head_dim == 128) return kv4 ? kern::launch<128, true>(a, stream) : kern::launch<128, false>(a, stream);
  if (head_dim == 64) return kv4 ? kern::launch<64, true>(a, stream) : kern::launch<64, false>(a, stream);
  return hipErrorInvalidValue;
}

}  // namespace tide
