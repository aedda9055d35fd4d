// Eviction by accumulated attention weight: per task and kv head, which cached positions stay (the
// last `recent` and the heaviest of the others, equal sums by position), and their move to the
// front of the task's pages, or of new ones, in order.
//
// Select: one workgroup per (task, kv head).  Sums become 32-bit keys that order like them (NaN
// lowest); three passes over the task's keys count 11, 11 and 10 bits of those that match the
// digits found so far and so find the smallest key that stays, and how many of its equals; a last
// pass ranks what stays by prefix sums and writes (position, page) and the sum, in order.
//
// Move: K and V rows go from their position to their rank.  Ranks never exceed positions, so in
// place a workgroup that loads a chunk of rows, waits for all of them (a barrier) and only then
// stores them is right if it takes its chunks in order: later chunks read positions beyond every
// slot written so far.  A workgroup does so for one 128-byte column of K's or V's rows; into new
// pages the chunks are independent and go to workgroups of their own.
#include "kernels.h"
#include "kv4.h"

namespace tide {
namespace kern {

constexpr int kSelect = 1024;  // threads
constexpr int kBins = 2048;

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
  __shared__ uint32_t found[2];  // digit, keys above it
  const int tid = threadIdx.x;
  const int unit = blockIdx.x / a.num_kv_heads, head = blockIdx.x - unit * a.num_kv_heads;
  const EvictTask t = a.tasks[unit];
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
    uint32_t prefix = 0, mask = 0, rest = want;
    constexpr int kShift[3] = {21, 10, 0}, kWidth[3] = {11, 11, 10};
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
      for (int i = tid; i < kBins; i += kSelect) hist[i] = 0;
      __syncthreads();
      const uint32_t digits = (1u << kWidth[pass]) - 1;
      for (int p = 4 * tid; p < cand; p += 4 * kSelect) {
        uint32_t key[4];
        float m[4];
        int32_t page;
        load4(p, key, m, &page);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (p + i < cand && (key[i] & mask) == prefix) atomicAdd(&hist[(key[i] >> kShift[pass]) & digits], 1u);
      }
      __syncthreads();
      // bins from the largest digit down, two a thread
      const uint32_t hi = hist[kBins - 1 - 2 * tid], lo = hist[kBins - 2 - 2 * tid];
      uint32_t all;
      const uint32_t before = block_scan(hi + lo, tmp[0], &all);
      if (before < rest && before + hi >= rest) found[0] = kBins - 1 - 2 * tid, found[1] = before;
      else if (before + hi < rest && before + hi + lo >= rest) found[0] = kBins - 2 - 2 * tid, found[1] = before + hi;
      __syncthreads();
      prefix |= found[0] << kShift[pass];
      mask |= digits << kShift[pass];
      rest -= found[1];
    }
    least = prefix;
    equal = rest;
  }
  const bool all_stay = want == cand;

  const int64_t out0 = (int64_t)t.first * a.num_kv_heads + (int64_t)head * t.keep;
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
        a.index[out0 + rank] = EvictIndex{p + i, page};
        a.index_mass[out0 + rank] = m[i];
        if (a.kept) a.kept[((int64_t)t.first + rank) * a.num_kv_heads + head] = p + i;
      }
      g += gt >> i & 1;
      e += is_eq;
    }
    above += all & 0xFFFFu;
    equals += all >> 16;
  }
}

constexpr int kMove = 256;  // threads
constexpr int kInFlight = 8;

// The pieces of one token's row that a part of the move takes: kLanes lanes of kBytes each.
//   bf16   128-byte columns of K, then of V
//   4 bit  K codes with their scales, V codes with theirs
template <int D, bool kKv4, bool kV>
struct MoveRow {
  static constexpr int kLanes = kKv4 ? (kV ? 16 : 4) : 8;
  static constexpr int kBytes = kKv4 ? (kV ? D / 32 : D / 8) : 16;
};

template <int kBytes>
struct Piece {
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

template <int D, bool kKv4, bool kV>
__device__ __forceinline__ void move_rows(const EvictArgs& a, const EvictTask& t, int head, int column,
                                          int chunk_first, int chunk_step) {
  using M = MoveRow<D, kKv4, kV>;
  using F = Kv4<D>;
  constexpr int kRows = kMove / M::kLanes;  // rows a load
  constexpr int kChunk = kRows * kInFlight;
  const int lane = threadIdx.x % M::kLanes, r0 = threadIdx.x / M::kLanes;
  const int64_t out0 = (int64_t)t.first * a.num_kv_heads + (int64_t)head * t.keep;
  const int32_t* to_row = a.new_table + (int64_t)t.task * a.new_stride;
  uint8_t* pool = kV && !kKv4 ? a.v_pool : a.k_pool;
  constexpr int64_t kBlk = kKv4 ? F::kBlock : (int64_t)kPage * D * 2;
  auto piece_at = [&](int32_t page, int slot) {
    uint8_t* blk = pool + ((int64_t)page * a.num_kv_heads + head) * kBlk;
    if constexpr (!kKv4) return blk + slot * D * 2 + 128 * column + 16 * lane;
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
  for (int c0 = chunk_first * kChunk; c0 < t.keep; c0 += chunk_step * kChunk) {
    Piece<M::kBytes> x[kInFlight];
    uint8_t scale[kInFlight];
    int32_t to[kInFlight];  // page, or -1: not moved
#pragma unroll
    for (int i = 0; i < kInFlight; ++i) {
      const int r = c0 + i * kRows + r0;
      to[i] = -1;
      if (r < t.keep) {
        const EvictIndex from = a.index[out0 + r];
        const int32_t g = to_row[r / kPage];
        const bool ok = g >= 0 && g < a.num_pages;
        if (!ok && lane == 0) atomicOr(a.error_flags, 1);
        if (ok && from.page >= 0 && (from.page != g || from.pos % kPage != r % kPage)) {
          to[i] = g;
          x[i].load(piece_at(from.page, from.pos % kPage));
          if (scale_lane) scale[i] = *scale_at(from.page, from.pos % kPage);
        }
      }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this thread's rows are here; after the barrier, all of the chunk's
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kInFlight; ++i) {
      const int slot = (c0 + i * kRows + r0) % kPage;
      if (to[i] < 0) continue;
      x[i].store(piece_at(to[i], slot));
      if (scale_lane) *scale_at(to[i], slot) = scale[i];
    }
  }
}

// The kept positions' sums, to the slots of their ranks (read from the index: no order needed).
__device__ __forceinline__ void move_mass(const EvictArgs& a, const EvictTask& t, int head, int first, int step) {
  const int64_t out0 = (int64_t)t.first * a.num_kv_heads + (int64_t)head * t.keep;
  const int32_t* to_row = a.new_table + (int64_t)t.task * a.new_stride;
  for (int r = first; r < t.keep; r += step) {
    const int32_t g = to_row[r / kPage];
    if (g >= 0 && g < a.num_pages && a.index[out0 + r].page >= 0)
      a.mass[((int64_t)g * a.num_kv_heads + head) * kPage + r % kPage] = a.index_mass[out0 + r];
  }
}

// grid: (task, kv head) x parts (K columns, V columns, sums) x chunk groups
template <int D, bool kKv4>
__global__ __launch_bounds__(kMove) void evict_move_kernel(EvictArgs a) {
  constexpr int kCols = kKv4 ? 1 : D / 64;
  const int unit = blockIdx.x / a.num_kv_heads, head = blockIdx.x - unit * a.num_kv_heads;
  const EvictTask t = a.tasks[unit];
  const int part = blockIdx.y;
  if (part < kCols) move_rows<D, kKv4, false>(a, t, head, part, blockIdx.z, gridDim.z);
  else if (part < 2 * kCols) move_rows<D, kKv4, true>(a, t, head, part - kCols, blockIdx.z, gridDim.z);
  else move_mass(a, t, head, blockIdx.z * kMove + threadIdx.x, gridDim.z * kMove);
}

template <int D, bool kKv4>
hipError_t launch(const EvictArgs& a, hipStream_t stream) {
  const unsigned units = (unsigned)a.num_tasks * a.num_kv_heads;
  hipLaunchKernelGGL(evict_select_kernel, dim3(units), dim3(kSelect), 0, stream, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  constexpr int kParts = 2 * (kKv4 ? 1 : D / 64) + 1;
  // in place one workgroup takes a column's chunks in order
  const unsigned chunks = a.new_table == a.block_table ? 1u : (unsigned)min(64, (a.longest_keep + 255) / 256);
  hipLaunchKernelGGL((evict_move_kernel<D, kKv4>), dim3(units, kParts, chunks), dim3(kMove), 0, stream, a);
  return hipGetLastError();
}

// Every variant is instantiated explicitly (see attn_decode.hip).
template __global__ void evict_move_kernel<128, false>(EvictArgs);
template __global__ void evict_move_kernel<128, true>(EvictArgs);
template __global__ void evict_move_kernel<64, false>(EvictArgs);
template __global__ void evict_move_kernel<64, true>(EvictArgs);

}  // namespace kern

hipError_t launch_evict(const EvictArgs& a, int head_dim, bool kv4, hipStream_t stream) {
  if (a.num_tasks == 0) return hipSuccess;
  if (head_dim == 128) return kv4 ? kern::launch<128, true>(a, stream) : kern::launch<128, false>(a, stream);
  if (head_dim == 64) return kv4 ? kern::launch<64, true>(a, stream) : kern::launch<64, false>(a, stream);
  return hipErrorInvalidValue;
}

}  // namespace tide
