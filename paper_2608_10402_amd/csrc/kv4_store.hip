// The 4-bit cache's plain data movement: append (bf16 rows into codes and scales), unpack (the
// reverse) and the unpacking of whole pages that the extend call reads.
//
// One wave per (task, logical page, kv head), like the bf16 append.  A lane holds exactly the
// codes that the attention kernels will read with it (kv4.h), so K needs the maximum of a lane's own
// entries (d = 128) and V that of 4 neighbouring lanes, and every store of a whole page is one
// contiguous piece of d / 8 bytes a lane.  A page that is appended in part takes exactly its new
// slots' bytes.
#include "kernels.h"
#include "kv4.h"

namespace tide {
namespace kern {

constexpr int kStoreWaves = 4;

// N 32-bit words of packed bf16 pairs, in loads of up to 16 bytes
template <int N>
__device__ __forceinline__ void load_words(uint32_t (&to)[N], const uint16_t* from) {
  if constexpr (N >= 4) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const u32x4 x = load_u32x4(from + 2 * i);
#pragma unroll
      for (int j = 0; j < 4; ++j) to[i + j] = x[j];
    }
  } else {
    const uint2 x = *reinterpret_cast<const uint2*>(from);
    to[0] = x.x;
    to[1] = x.y;
  }
}

template <int D>
__device__ __forceinline__ void append_page(const Kv4StoreArgs& a, uint8_t* blk, int64_t row0, int head,
                                            int s0, int n) {
  using F = Kv4<D>;
  const int lane = threadIdx.x & 63, lo = lane & 15, hi = lane >> 4;
  // K: slot lo, entries [D/4 hi, + D/4)
  {
    const bool in = lo >= s0 && lo < s0 + n;
    uint32_t x[D / 8];
    if (in) {
      load_words(x, a.k_new + ((row0 + lo - s0) * a.num_kv_heads + head) * D + (D / 4) * hi);
    } else {
#pragma unroll
      for (int i = 0; i < D / 8; ++i) x[i] = 0;
    }
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < D / 8; ++i) m = kv4_max(m, x[i]);
    if constexpr (D == 64) m = max(m, (uint32_t)__shfl_xor((int)m, 16, 64));  // a block: two lanes
    const uint32_t byte = kv4_scale_byte(m);
    const float f = kv4_factor(byte);
    uint32_t c[F::kWords];
#pragma unroll
    for (int w = 0; w < F::kWords; ++w)
      c[w] = kv4_codes(u32x4{x[4 * w], x[4 * w + 1], x[4 * w + 2], x[4 * w + 3]}, f);
    if (in) {
      uint32_t* to = reinterpret_cast<uint32_t*>(blk + lane * F::kLane);
      if constexpr (D == 128) store_u32x4(to, u32x4{c[0], c[1], c[2], c[3]});
      else *reinterpret_cast<uint2*>(to) = uint2{c[0], c[1]};
      if (D == 128 || (hi & 1) == 0) blk[F::k_scale(lane)] = (uint8_t)byte;
    }
  }
  // V: slots 4 hi .. + 3, entries [D/16 lo, + D/16)
  constexpr int kW = F::kSpan / 2;  // words of bf16 pairs of a slot
  uint32_t x[4][kW];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int slot = 4 * hi + i;
    if (slot >= s0 && slot < s0 + n) {
      load_words(x[i], a.v_new + ((row0 + slot - s0) * a.num_kv_heads + head) * D + F::kSpan * lo);
    } else {
#pragma unroll
      for (int w = 0; w < kW; ++w) x[i][w] = 0;
    }
  }
  uint32_t bytes = 0, c[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t m = 0;
#pragma unroll
    for (int w = 0; w < kW; ++w) m = kv4_max(m, x[i][w]);
#pragma unroll
    for (int o = 1; o < F::kVLanes; o *= 2) m = max(m, (uint32_t)__shfl_xor((int)m, o, 64));
    const uint32_t byte = kv4_scale_byte(m);
    u32x4 p = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int w = 0; w < kW; ++w) p[w] = x[i][w];
    c[i] = kv4_codes(p, kv4_factor(byte));
    bytes |= byte << (8 * i);
  }
  const bool scale_lane = lo % F::kVLanes == 0;
  if (n == kPage) {
    uint8_t* to = blk + F::kVCodes + lane * F::kLane;
    if constexpr (D == 128) store_u32x4(to, u32x4{c[0], c[1], c[2], c[3]});
    else *reinterpret_cast<uint2*>(to) = uint2{(c[0] & 0xFFFFu) | (c[1] << 16), (c[2] & 0xFFFFu) | (c[3] << 16)};
    if (scale_lane) *reinterpret_cast<uint32_t*>(blk + F::v_scale(lane)) = bytes;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int slot = 4 * hi + i;
      if (slot < s0 || slot >= s0 + n) continue;
      if constexpr (D == 128) *reinterpret_cast<uint32_t*>(blk + F::v_word(lo, slot)) = c[i];
      else *reinterpret_cast<uint16_t*>(blk + F::v_word(lo, slot)) = (uint16_t)c[i];
      if (scale_lane) blk[F::v_scale(lane) + i] = (uint8_t)(bytes >> (8 * i));
    }
  }
}

// Rows [s0, s0 + n) of a page to bf16: slot s of K and V to k_out / v_out + (s - s0) * stride.
// blk == null (a page id out of range): zeros.
template <int D>
__device__ __forceinline__ void unpack_page(const uint8_t* blk, uint16_t* k_out, uint16_t* v_out, int64_t stride,
                                            int s0, int n) {
  using F = Kv4<D>;
  const int lane = threadIdx.x & 63, lo = lane & 15, hi = lane >> 4;
  uint32_t kc[F::kWords] = {}, vc[F::kWords] = {}, kb = 127, vb = 0x7F7F7F7Fu;
  if (blk) {
    const uint32_t* kp = reinterpret_cast<const uint32_t*>(blk + lane * F::kLane);
    const uint32_t* vp = reinterpret_cast<const uint32_t*>(blk + F::kVCodes + lane * F::kLane);
    if constexpr (D == 128) {
      const u32x4 k = load_u32x4(kp), v = load_u32x4(vp);
#pragma unroll
      for (int w = 0; w < 4; ++w) kc[w] = k[w], vc[w] = v[w];
    } else {
      const uint2 k = *reinterpret_cast<const uint2*>(kp), v = *reinterpret_cast<const uint2*>(vp);
      kc[0] = k.x, kc[1] = k.y, vc[0] = v.x, vc[1] = v.y;
    }
    kb = blk[F::k_scale(lane)];
    vb = *reinterpret_cast<const uint32_t*>(blk + F::v_scale(lane));
  }
  if (lo >= s0 && lo < s0 + n) {
    uint16_t* to = k_out + (lo - s0) * stride + (D / 4) * hi;
    const float f = kv4_factor(kb);
#pragma unroll
    for (int w = 0; w < F::kWords; ++w)
      store_u32x4(to + 8 * w, __builtin_bit_cast(u32x4, kv4_octet(kc[w], f)));
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int slot = 4 * hi + i;
    if (slot < s0 || slot >= s0 + n) continue;
    uint16_t* to = v_out + (slot - s0) * stride + F::kSpan * lo;
    const float f = kv4_factor((vb >> (8 * i)) & 255u);
    if constexpr (D == 128) {
      store_u32x4(to, __builtin_bit_cast(u32x4, kv4_octet(vc[i], f)));
    } else {
      const uint32_t c = vc[i >> 1] >> (16 * (i & 1));
      *reinterpret_cast<uint2*>(to) = uint2{kv4_pair<0>(c, f), kv4_pair<1>(c, f)};
    }
  }
}

template <int D, bool kAppend>
__global__ __launch_bounds__(kStoreWaves * 64) void kv4_store_kernel(Kv4StoreArgs a) {
  const int wave = threadIdx.x >> 6;
  const int head = blockIdx.y * kStoreWaves + wave;
  const AppendItem it = a.items[blockIdx.x];
  const TaskDesc td = a.tasks[it.task];
  const int32_t phys = a.block_table[(int64_t)it.task * a.bt_stride + it.lpage];
  if (a.reads.done) {
    asm volatile("" ::"v"(it.pos_end), "v"(td.extend));  // both records have arrived
    __syncthreads();
    if (threadIdx.x == 0) plan_read(a.reads, blockIdx.y * gridDim.x + blockIdx.x);
  }
  const bool page_ok = phys >= 0 && phys < a.num_pages;
  if (!page_ok && threadIdx.x == 0) atomicOr(a.error_flags, 1);
  if (head >= a.num_kv_heads || (kAppend && !page_ok)) return;
  const int s0 = it.pos_begin % kPage, n = it.pos_end - it.pos_begin;
  const int64_t row0 = (int64_t)td.row_start + (it.pos_begin - td.prefix);
  uint8_t* blk = a.pool + ((int64_t)(page_ok ? phys : 0) * a.num_kv_heads + head) * kv4_block_bytes(D);
  if constexpr (kAppend) {
    append_page<D>(a, blk, row0, head, s0, n);
  } else {
    const int64_t at = (row0 * a.num_kv_heads + head) * D;
    unpack_page<D>(page_ok ? blk : nullptr, a.k_out + at, a.v_out + at, (int64_t)a.num_kv_heads * D, s0, n);
  }
}

template <int D>
__global__ __launch_bounds__(kStoreWaves * 64) void kv4_stage_kernel(Kv4StageArgs a) {
  const Kv4StageItem it = a.items[blockIdx.x];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (a.reads.done) {
    asm volatile("" ::"v"(it.task));  // the record has arrived
    __syncthreads();
    if (threadIdx.x == 0) plan_read(a.reads, blockIdx.x);
  }
  const int32_t* row = a.block_table + (int64_t)it.row * a.bt_stride + it.lpage;
  if ((int)threadIdx.x < it.pages)
    a.stage_table[(int64_t)it.task * a.stage_stride + it.lpage + threadIdx.x] = it.to + threadIdx.x;
  for (int i = wave; i < it.pages * a.num_kv_heads; i += kStoreWaves) {
    const int page = i / a.num_kv_heads, head = i - page * a.num_kv_heads;
    const int32_t phys = row[page];
    const bool ok = phys >= 0 && phys < a.num_pages;
    if (!ok && (threadIdx.x & 63) == 0) atomicOr(a.error_flags, 1);
    const uint8_t* blk = a.pool + ((int64_t)(ok ? phys : 0) * a.num_kv_heads + head) * kv4_block_bytes(D);
    const int64_t at = ((int64_t)(it.to + page) * a.num_kv_heads + head) * (kPage * D);
    unpack_page<D>(ok ? blk : nullptr, a.k_stage + at, a.v_stage + at, D, 0, kPage);
  }
}

// Every variant is instantiated explicitly (see attn_decode.hip).
template __global__ void kv4_store_kernel<128, false>(Kv4StoreArgs);
template __global__ void kv4_store_kernel<128, true>(Kv4StoreArgs);
template __global__ void kv4_store_kernel<64, false>(Kv4StoreArgs);
template __global__ void kv4_store_kernel<64, true>(Kv4StoreArgs);
template __global__ void kv4_stage_kernel<128>(Kv4StageArgs);
template __global__ void kv4_stage_kernel<64>(Kv4StageArgs);

}  // namespace kern

int kv4_store_groups(int32_t num_kv_heads) {
  return (num_kv_heads + kern::kStoreWaves - 1) / kern::kStoreWaves;
}

hipError_t launch_kv4_store(const Kv4StoreArgs& a, hipStream_t stream) {
  if (a.num_items == 0) return hipSuccess;
  const dim3 grid(a.num_items, kv4_store_groups(a.num_kv_heads)), block(kern::kStoreWaves * 64);
  const bool append = a.k_new != nullptr;
  if (a.head_dim == 128) {
    if (append) hipLaunchKernelGGL((kern::kv4_store_kernel<128, true>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((kern::kv4_store_kernel<128, false>), grid, block, 0, stream, a);
  } else if (a.head_dim == 64) {
    if (append) hipLaunchKernelGGL((kern::kv4_store_kernel<64, true>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((kern::kv4_store_kernel<64, false>), grid, block, 0, stream, a);
  } else {
    return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

hipError_t launch_kv4_stage(const Kv4StageArgs& a, hipStream_t stream) {
  if (a.num_items == 0) return hipSuccess;
  const dim3 grid(a.num_items), block(kern::kStoreWaves * 64);
  if (a.head_dim == 128) hipLaunchKernelGGL((kern::kv4_stage_kernel<128>), grid, block, 0, stream, a);
  else if (a.head_dim == 64) hipLaunchKernelGGL((kern::kv4_stage_kernel<64>), grid, block, 0, stream, a);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace tide
