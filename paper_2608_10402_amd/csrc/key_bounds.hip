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

// Lane groups of 16 (or halves): the larger of a's pair of groups in one, of b's in the other (max_groups, max_halves
// of block_select.hip, two entries at a time); kMin: the smaller.
template <bool kMin>
__device__ __forceinline__ uint32_t pick(uint32_t a, uint32_t b) {
  const i16x2 x = __builtin_bit_cast(i16x2, a), y = __builtin_bit_cast(i16x2, b);
  return __builtin_bit_cast(uint32_t, kMin ? __builtin_elementwise_min(x, y) : __builtin_elementwise_max(x, y));
}

template <bool kMin>
__device__ __forceinline__ uint32_t join16(uint32_t a, uint32_t b) {
  const auto s = __builtin_amdgcn_permlane16_swap(a, b, false, false);
  return pick<kMin>((uint32_t)s[0], (uint32_t)s[1]);
}

template <bool kMin>
__device__ __forceinline__ uint32_t join32(uint32_t a, uint32_t b) {
  const auto s = __builtin_amdgcn_permlane32_swap(a, b, false, false);
  return pick<kMin>((uint32_t)s[0], (uint32_t)s[1]);
}

// Over the wave's row groups: lane l gets the word of entries 8 (l % kG) + 2 (l / 16) of x[0 .. 3].
template <int D, bool kMin>
__device__ __forceinline__ uint32_t over_rows(const uint32_t (&x)[4]) {
  uint32_t y = join32<kMin>(join16<kMin>(x[0], x[1]), join16<kMin>(x[2], x[3]));
  if (D == 64) y = pick<kMin>(y, (uint32_t)__builtin_amdgcn_mov_dpp((int)y, 0x128, 0xF, 0xF, true));  // row_ror:8
  return y;
}

// The largest of the wave's x.
__device__ __forceinline__ int wave_max(int x) {
  x = max(x, __builtin_amdgcn_mov_dpp(x, 0x121, 0xF, 0xF, true));  // row_ror 1, 2, 4, 8: over 16 lanes
  x = max(x, __builtin_amdgcn_mov_dpp(x, 0x122, 0xF, 0xF, true));
  x = max(x, __builtin_amdgcn_mov_dpp(x, 0x124, 0xF, 0xF, true));
  x = max(x, __builtin_amdgcn_mov_dpp(x, 0x128, 0xF, 0xF, true));
  const auto r = __builtin_amdgcn_permlane16_swap((uint32_t)x, (uint32_t)x, false, false);
  x = max((int)r[0], (int)r[1]);
  const auto h = __builtin_amdgcn_permlane32_swap((uint32_t)x, (uint32_t)x, false, false);
  return max((int)h[0], (int)h[1]);
}

// Bounds of a page's rows, stored for (page, head) = block `at` of the pools.  Rows past the last position repeat
// one that counts.
template <int D>
__device__ __forceinline__ void put_bounds(const PageRows<D>& rows, int8_t* bounds, int8_t* units, int64_t at) {
  using R = PageRows<D>;
  const int lane = threadIdx.x & 63, part = lane % R::kG;
  constexpr int kInf = 0x7F80;
  uint32_t hi[4], lo[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    hi[j] = lo[j] = __builtin_bit_cast(uint32_t, ordered(rows.x[0][j]));
#pragma unroll
    for (int i = 1; i < R::kLoads; ++i) {
      const uint32_t v = __builtin_bit_cast(uint32_t, ordered(rows.x[i][j]));
      hi[j] = pick<false>(hi[j], v);
      lo[j] = pick<true>(lo[j], v);
    }
  }
  const i16x2 most = __builtin_bit_cast(i16x2, over_rows<D, false>(hi));
  const i16x2 least = __builtin_bit_cast(i16x2, over_rows<D, true>(lo));
  // the largest magnitude over the entries, as an ordered integer; at least kInf where one is not finite
  int top = max(max((int)most[0], (int)most[1]), max(~(int)least[0], ~(int)least[1]));  // ~: a negative's magnitude
  top = wave_max(max(top, 0));
  const bool finite = top < kInf;
  // top = 1.f 2^e with 7 bits of f: 127 2^(e - 6) = 1.1111110b 2^e is at least that for f < 0x7F
  const int e = (top >> 7) - 127;
  const int unit = max(kLeastUnit, e - 6 + ((top & 0x7F) == 0x7F ? 1 : 0));
  const float scale = finite ? __builtin_bit_cast(float, (uint32_t)(127 - unit) << 23) : 0.0f;
  uint32_t upper = 0, lower = 0;
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    // the product is exact, but for values below 2^-149, which are 1 or -1 then
    int u = (int)ceilf(value_of(most[c]) * scale), l = (int)floorf(value_of(least[c]) * scale);
    u = most[c] > 0 ? max(u, 1) : u;
    l = least[c] < -1 ? min(l, -1) : l;  // (-1 is -0)
    upper |= (uint32_t)(u & 0xFF) << (8 * c);
    lower |= (uint32_t)(l & 0xFF) << (8 * c);
  }
  if (!finite) upper = lower = 0;
  if (D == 128 || (lane & 8) == 0) {
    int8_t* to = bounds + at * (2 * D) + 8 * part + 2 * (lane >> 4);
    *reinterpret_cast<uint16_t*>(to) = (uint16_t)upper;
    *reinterpret_cast<uint16_t*>(to + D) = (uint16_t)lower;
  }
  if (lane == 0) units[at] = (int8_t)(finite ? unit : kNoUnit);
}

// A workgroup looks at a.window rows (append_window) for the first rows of pages.  Such a row, with those behind it that
// follow in the same page, is an item for each kv head, and the items go round the workgroups of the window
// (gridDim.y) and their waves.
template <int D, bool kBounds>
__global__ __launch_bounds__(kBoundWaves * 64) void slot_append_kernel(SlotAppendArgs a) {
  using R = PageRows<D>;
  const int lane = threadIdx.x & 63, Hkv = a.num_kv_heads;
  const int wave = blockIdx.y * kBoundWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = gridDim.y * kBoundWaves;
  // lane 0 the row before the window, lane 1 + i row i of it and the 15 behind it
  const int64_t row0 = a.first_row + (int64_t)blockIdx.x * a.window, r = row0 - 1 + lane;
  const bool there = lane <= a.window + kPage - 1 && r >= 0 && r < a.num_rows;
  const int64_t slot = there ? a.row_slot[r] : -1;
  const int64_t before = __shfl_up(slot, 1, 64);
  const bool follows = slot > 0 && slot % kPage != 0 && slot == before + 1;  // the row before it in the same page
  const bool in_window = lane > 0 && lane <= a.window && slot >= 0;
  const bool outside = slot >= a.num_pages * kPage;
  if (in_window && outside && wave == 0) atomicOr(a.error_flags, 1);
  const uint64_t chain = __builtin_amdgcn_ballot_w64(follows);
  uint64_t firsts = __builtin_amdgcn_ballot_w64(in_window && !outside && (!follows || before < 0));
  const int part = lane % R::kG, first = lane / R::kG;
  for (int turn = wave; firsts; firsts &= firsts - 1, turn -= Hkv) {  // item `turn` of this row's kv heads is this wave's
    if (turn >= Hkv) continue;
    const int at_lane = __builtin_ctzll(firsts);
    const int64_t slot0 = ((int64_t)__builtin_amdgcn_readlane((int)(slot >> 32), at_lane) << 32) |
                          (uint32_t)__builtin_amdgcn_readlane((int)slot, at_lane);
    const int s0 = (int)(slot0 % kPage);
    const int n = __builtin_ctzll(~(chain >> at_lane >> 1)) + 1;  // rows of this page, 1 .. 16 - s0
    const int64_t row = row0 - 1 + at_lane;
    for (; turn < Hkv; turn += waves) {
      const int64_t at = slot0 / kPage * Hkv + turn;
      PageRows<D> k, v;
#pragma unroll
      for (int i = 0; i < R::kLoads; ++i) {
        // slots past the new rows: the last of them again, for the bounds
        const int s = first + R::kRows * i, from = max(0, min(s - s0, n - 1));
        const int64_t src = ((row + from) * Hkv + turn) * D + 8 * part;
        if (kBounds) {
          k.x[i] = load_u32x4(s < s0 ? a.k_pool + (at * kPage + s) * D + 8 * part : a.k_new + src);
          v.x[i] = load_u32x4(a.v_new + src);
        } else if (s >= s0 && s < s0 + n) {
          k.x[i] = load_u32x4(a.k_new + src);
          v.x[i] = load_u32x4(a.v_new + src);
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
      if constexpr (kBounds) put_bounds<D>(k, a.bounds, a.units, at);
    }
  }
}

// One wave per (task, kBoundPages pages, kv head): all of them in flight at once, read past the caches (687 MB of keys:
// 144 us with ordinary loads, 130 without; 125 with two entries an instruction, 5.5 TB/s).
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
      const int s = max(0, min(lane / R::kG + R::kRows * j, n[i] - 1));
      if (at[i] >= 0)
        k[i].x[j] = __builtin_nontemporal_load(
            reinterpret_cast<const u32x4*>(a.k_pool + (at[i] * kPage + s) * D + 8 * (lane % R::kG)));
    }
#pragma unroll
  for (int i = 0; i < kBoundPages; ++i)
    if (at[i] >= 0) put_bounds<D>(k[i], a.bounds, a.units, at[i]);
}

// Few (row, kv head) pairs: a workgroup for 4 kv heads of each row, so that the call ends soon.  More than the device
// holds waves: one for several rows, since 15 of 16 rows of an observation are not the first of a page, and a wave that
// only finds that out costs a third of one that works; single tokens, which all are, want short windows.  (A call by
// windows of 1, 4, 8 and 16 rows: 1,024 x 1 rows of 8 heads 9.3, 10.9, 18.6 and 33 us; 4,096 x 1 of 8 heads 25, 20, 25,
// 37; 8,192 x 1 of 8 heads 46, 38, 38, 49; 64 x 512 of 4 heads 36, 24, 24, 24; 64 x 64-2,048 of 4 heads by the last three
// 38, 35, 34; 64 x 1,024 of 8 heads 195, 118, 118, 119.)
int32_t append_window(int64_t pairs) { return pairs <= 8192 ? 1 : pairs < 65536 ? 4 : 8; }

template <int D>
hipError_t append_slots(const SlotAppendArgs& args, hipStream_t stream) {
  SlotAppendArgs a = args;
  a.window = append_window((int64_t)a.num_rows * a.num_kv_heads);
  const uint32_t parts = a.window > 1 ? 1 : (uint32_t)((a.num_kv_heads + kBoundWaves - 1) / kBoundWaves);
  // a launch holds fewer than 2^32 threads
  const int32_t most = (int32_t)((1 << 23) / parts) * a.window;
  for (int64_t row = 0; row < a.num_rows; row += most) {
    a.first_row = (int32_t)row;
    const dim3 blocks((uint32_t)((std::min<int64_t>(most, a.num_rows - row) + a.window - 1) / a.window), parts);
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
