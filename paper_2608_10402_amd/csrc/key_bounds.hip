// Key bounds, and the append by slots that keeps them.
//
// The bounds of a (page, kv head) stand for its keys where blocks are chosen (block_select.hip): with
// s the least unit in [-120, 122] such that max|k| <= 127 * 2^s over the page's positions and entries,
//     hi_i = ceil(max_t k_ti / 2^s),  lo_i = floor(min_t k_ti / 2^s),  i < d,
// whole numbers of 8 bits, rounded outwards so that lo_i 2^s <= k_ti <= hi_i 2^s holds for every key.
// They are 1/16 of the keys' bytes, and sums of their products with whole-number queries are exact in
// 32 bits.  The unit is a power of two so that it can be applied without a rounding.  A page with a
// key that is not finite has unit 127 and zeros.  Bounds are a function of the keys that the page holds
// up to its last position: an append takes the page's older keys from the pool, not from older bounds
// (rounded bounds of bounds would depend on how the tokens came in).
//
// One wave takes one page of one kv head.  Its 16 rows are d/8 pieces of 16 bytes each; a lane holds
// pieces of 4 (d = 128) or 2 (d = 64) rows at the same entries.  bf16 values become 16-bit integers
// of the same order, so maxima and minima are two entries an instruction, in the lane first and then
// across the 4 or 8 lanes that share its entries.
#include <algorithm>

#include "kernels.h"
#include "tide_device.h"

namespace tide {
namespace kern {

typedef int16_t i16x2 __attribute__((ext_vector_type(2)));

constexpr int kBoundWaves = 4;

// One page's rows as its wave loads them: lane l has piece l % kG of rows l / kG + kRows i.
template <int D>
struct PageRows {
  static constexpr int kG = D / 8;         // 16-byte pieces of a row
  static constexpr int kRows = 64 / kG;    // rows of a load
  static constexpr int kLoads = kPage / kRows;
  u32x4 x[kLoads];
};

// bf16 pairs as integers that order like them (-0 next below 0, infinities and NaN outermost), and back.
__device__ __forceinline__ i16x2 ordered(uint32_t pair) {
  const i16x2 v = __builtin_bit_cast(i16x2, pair);
  return v ^ ((v >> 15) & (int16_t)0x7FFF);
}

__device__ __forceinline__ float value_of(int16_t o) {
  const uint16_t b = (uint16_t)(o ^ ((o >> 15) & 0x7FFF));
  return __builtin_bit_cast(float, (uint32_t)b << 16);
}

__device__ __forceinline__ i16x2 shfl_i16x2(i16x2 v, int mask) {
  return __builtin_bit_cast(i16x2, __shfl_xor(__builtin_bit_cast(int, v), mask, 64));
}

// Bounds of the first n (1 .. 16) rows, stored for (page, head) = block `at` of the pools.
template <int D>
__device__ __forceinline__ void put_bounds(const PageRows<D>& rows, int n, int8_t* bounds, int8_t* units, int64_t at) {
  using R = PageRows<D>;
  const int lane = threadIdx.x & 63, part = lane % R::kG, row = lane / R::kG;
  constexpr int16_t kInf = 0x7F80;
  i16x2 hi[4], lo[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    hi[j] = i16x2{INT16_MIN, INT16_MIN};
    lo[j] = i16x2{INT16_MAX, INT16_MAX};
  }
#pragma unroll
  for (int i = 0; i < R::kLoads; ++i) {
    const bool in = row + R::kRows * i < n;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const i16x2 v = ordered(rows.x[i][j]);
      hi[j] = in ? __builtin_elementwise_max(hi[j], v) : hi[j];
      lo[j] = in ? __builtin_elementwise_min(lo[j], v) : lo[j];
    }
  }
#pragma unroll
  for (int m = R::kG; m < 64; m *= 2)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      hi[j] = __builtin_elementwise_max(hi[j], shfl_i16x2(hi[j], m));
      lo[j] = __builtin_elementwise_min(lo[j], shfl_i16x2(lo[j], m));
    }
  // the largest magnitude over the entries, as an ordered integer; at least kInf where one is not finite
  int top = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int e = 0; e < 2; ++e) top = max(top, max((int)hi[j][e], ~(int)lo[j][e]));  // ~: a negative's magnitude
#pragma unroll
  for (int m = 1; m < R::kG; m *= 2) top = max(top, __shfl_xor(top, m, 64));
  const bool finite = top < kInf;
  // top = 1.f 2^e with 7 bits of f: 127 2^(e - 6) = 1.1111110b 2^e is at least that for f < 0x7F
  const int e = (top >> 7) - 127;
  const int unit = max(kLeastUnit, e - 6 + ((top & 0x7F) == 0x7F ? 1 : 0));
  const float scale = __builtin_bit_cast(float, (uint32_t)(127 - unit) << 23);
  // lanes of the first rows store the upper bounds, those of the next the lower ones
  const bool up = row == 0;
  uint32_t packed[2] = {0, 0};
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int16_t o = up ? hi[j][c] : lo[j][c];
      const float y = value_of(o) * scale;  // exact, but for values below 2^-149, which are 1 or -1 then
      int v = (int)(up ? ceilf(y) : floorf(y));
      if (up && o > 0) v = max(v, 1);
      if (!up && o < -1) v = min(v, -1);
      packed[j >> 1] |= (uint32_t)(v & 0xFF) << (16 * (j & 1) + 8 * c);
    }
  if (!finite) packed[0] = packed[1] = 0;
  if (row < 2)
    *reinterpret_cast<uint2*>(bounds + at * (2 * D) + (up ? 0 : D) + 8 * part) = uint2{packed[0], packed[1]};
  if (lane == 0) units[at] = (int8_t)(finite ? unit : kNoUnit);
}

// One wave per (row, kv head); it works if the row is the first of its page's, and takes the rows behind
// it that follow in the same page.
template <int D, bool kBounds>
__global__ __launch_bounds__(kBoundWaves * 64) void slot_append_kernel(SlotAppendArgs a) {
  using R = PageRows<D>;
  const int lane = threadIdx.x & 63;
  const uint32_t id = blockIdx.x * kBoundWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int32_t nth = (int32_t)(id / (uint32_t)a.num_kv_heads), head = (int32_t)id - nth * a.num_kv_heads;
  if (nth >= a.rows) return;
  const int32_t row = a.first_row + nth;
  // lane 0 the row before, lane 1 + i row + i
  const int64_t r = (int64_t)row - 1 + lane;
  const int64_t slot = lane <= kPage && r >= 0 && r < a.num_rows ? a.row_slot[r] : -1;
  const int64_t slot0 = __shfl(slot, 1, 64), before = __shfl(slot, 0, 64);
  if (slot0 < 0) return;
  if (slot0 >= a.num_pages * kPage) {
    if (lane == 1) atomicOr(a.error_flags, 1);
    return;
  }
  const int s0 = (int)(slot0 % kPage);
  if (s0 > 0 && before == slot0 - 1) return;
  const uint64_t follow = __builtin_amdgcn_ballot_w64(lane > 0 && lane <= kPage - s0 && slot == slot0 + (lane - 1));
  const int n = __builtin_ctzll(~(follow >> 1));  // rows of this page, 1 .. 16 - s0
  const int64_t at = slot0 / kPage * a.num_kv_heads + head;
  const int part = lane % R::kG, first = lane / R::kG;
  PageRows<D> k, v;
#pragma unroll
  for (int i = 0; i < R::kLoads; ++i) {
    const int s = first + R::kRows * i;
    k.x[i] = v.x[i] = zero_u32x4();
    if (s >= s0 && s < s0 + n) {
      const int64_t src = (((int64_t)row + s - s0) * a.num_kv_heads + head) * D + 8 * part;
      k.x[i] = load_u32x4(a.k_new + src);
      v.x[i] = load_u32x4(a.v_new + src);
    } else if (kBounds && s < s0) {
      k.x[i] = load_u32x4(a.k_pool + (at * kPage + s) * D + 8 * part);
    }
  }
#pragma unroll
  for (int i = 0; i < R::kLoads; ++i) {
    const int s = first + R::kRows * i;
    if (s >= s0 && s < s0 + n) {
      store_u32x4(a.k_pool + (at * kPage + s) * D + 8 * part, k.x[i]);
      store_u32x4(a.v_pool + (at * kPage + s) * D + 8 * part, v.x[i]);
    }
  }
  if constexpr (kBounds) put_bounds<D>(k, s0 + n, a.bounds, a.units, at);
}

// One wave per (task, kBoundPages pages, kv head): all of them in flight at once.
constexpr int kBoundPages = 4;

template <int D>
__global__ __launch_bounds__(kBoundWaves * 64) void key_bounds_kernel(KeyBoundsArgs a) {
  using R = PageRows<D>;
  const int lane = threadIdx.x & 63;
  const uint32_t id = blockIdx.x * kBoundWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t nth = id / (uint32_t)a.num_kv_heads;
  const int head = (int)(id - nth * (uint32_t)a.num_kv_heads);
  if (nth >= (uint32_t)a.units_here) return;
  const uint32_t chunk = (uint32_t)a.first_chunk + nth, tasks = chunk / (uint32_t)a.chunks;
  const int task = a.first_task + (int)tasks;
  const int p0 = (int)(chunk - tasks * (uint32_t)a.chunks) * kBoundPages;
  const int len = min(a.lens[task], a.max_len), from = a.from ? max(0, a.from[task]) : 0;
  if ((int64_t)p0 * kPage >= len || from >= len || (int64_t)(p0 + kBoundPages) * kPage <= from) return;
  const int32_t* table = a.block_table + (int64_t)task * a.bt_stride;
  PageRows<D> k[kBoundPages];
  int64_t at[kBoundPages];
  int n[kBoundPages];
#pragma unroll
  for (int i = 0; i < kBoundPages; ++i) {
    const int64_t pos = (int64_t)(p0 + i) * kPage;
    n[i] = pos < len && pos + kPage > from ? (int)min((int64_t)kPage, len - pos) : 0;
    at[i] = -1;
    if (n[i] > 0) {
      const int32_t page = load_page_id(table, p0 + i);
      if (page >= 0 && page < a.num_pages) at[i] = (int64_t)page * a.num_kv_heads + head;
      else if (lane == 0) atomicOr(a.error_flags, 1);
    }
  }
#pragma unroll
  for (int i = 0; i < kBoundPages; ++i)
#pragma unroll
    for (int j = 0; j < R::kLoads; ++j) {
      k[i].x[j] = zero_u32x4();
      if (at[i] >= 0 && lane / R::kG + R::kRows * j < n[i])
        k[i].x[j] = load_u32x4(a.k_pool + at[i] * kPage * D + 8 * (lane + 64 * j));
    }
#pragma unroll
  for (int i = 0; i < kBoundPages; ++i)
    if (at[i] >= 0) put_bounds<D>(k[i], n[i], a.bounds, a.units, at[i]);
}

template <int D>
hipError_t append_slots(const SlotAppendArgs& args, hipStream_t stream) {
  SlotAppendArgs a = args;
  // a launch holds fewer than 2^32 threads
  const int32_t most = std::max(1, (1 << 25) / a.num_kv_heads);
  for (a.first_row = 0; a.first_row < a.num_rows; a.first_row += a.rows) {
    a.rows = std::min(most, a.num_rows - a.first_row);
    const uint32_t blocks = (uint32_t)(((int64_t)a.rows * a.num_kv_heads + kBoundWaves - 1) / kBoundWaves);
    if (a.bounds)
      hipLaunchKernelGGL((slot_append_kernel<D, true>), dim3(blocks), dim3(kBoundWaves * 64), 0, stream, a);
    else
      hipLaunchKernelGGL((slot_append_kernel<D, false>), dim3(blocks), dim3(kBoundWaves * 64), 0, stream, a);
    const hipError_t rc = hipGetLastError();
    if (rc != hipSuccess) return rc;
  }
  return hipSuccess;
}

template <int D>
hipError_t make_bounds(const KeyBoundsArgs& args, int32_t num_tasks, hipStream_t stream) {
  KeyBoundsArgs a = args;
  constexpr int kPer = kBoundPages * kPage;
  a.chunks = (a.max_len - 1) / kPer + 1;
  const int64_t units = (int64_t)num_tasks * a.chunks, most = std::max(1, (1 << 25) / a.num_kv_heads);
  for (int64_t first = 0; first < units; first += most) {
    a.first_task = (int32_t)(first / a.chunks);
    a.first_chunk = (int32_t)(first % a.chunks);
    a.units_here = (int32_t)std::min(most, units - first);
    const uint32_t blocks = (uint32_t)(((int64_t)a.units_here * a.num_kv_heads + kBoundWaves - 1) / kBoundWaves);
    hipLaunchKernelGGL((key_bounds_kernel<D>), dim3(blocks), dim3(kBoundWaves * 64), 0, stream, a);
    const hipError_t rc = hipGetLastError();
    if (rc != hipSuccess) return rc;
  }
  return hipSuccess;
}

}  // namespace kern

hipError_t launch_slot_append(const SlotAppendArgs& a, int head_dim, hipStream_t stream) {
  return head_dim == 128 ? kern::append_slots<128>(a, stream) : kern::append_slots<64>(a, stream);
}

hipError_t launch_key_bounds(const KeyBoundsArgs& a, int head_dim, int32_t num_tasks, hipStream_t stream) {
  return head_dim == 128 ? kern::make_bounds<128>(a, num_tasks, stream) : kern::make_bounds<64>(a, num_tasks, stream);
}

}  // namespace tide
