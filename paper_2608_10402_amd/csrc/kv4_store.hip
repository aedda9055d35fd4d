// The 4-bit cache's plain data movement: append (bf16 rows into codes and scales), unpack (the
// reverse) and the unpacking of whole pages that the extend call reads.
//
// One wave per (task, logical page, kv head), like the bf16 append.  Lane (quad l / 16, piece l % 16)
// takes d / 16 entries of 4 slots' rows, so that 16 lanes read (or write) a whole bf16 row, and a
// scale block is 4 neighbouring lanes' (8 at d = 64).  With the attention kernels' mapping, where a
// lane holds d / 4 entries of one K row, 64 lanes touched 64 separate pieces: appending 36k tokens
// and reading them back (4 heads, d = 128) took 55 us, and 44 so (4.2 TB/s; a large copy reaches
// 4.8), unpacking the pages of 590k tokens 0.45 ms, and 0.30 so (5.0 TB/s).  Bound by memory; a
// conversion is one instruction per two values.
#include "kernels.h"
#include "kv4.h"

namespace tide {
namespace kern {

constexpr int kStoreWaves = 4;

// The kSpan bf16 entries of a lane's piece of a row: 16 bytes (d = 128) or 8.
template <int D>
struct Piece {
  u32x4 x;  // (8 bytes: the first two words)
  __device__ __forceinline__ void load(const uint16_t* from) {
    if constexpr (D == 128) {
      x = load_u32x4(from);
    } else {
      const uint2 y = *reinterpret_cast<const uint2*>(from);
      x = u32x4{y.x, y.y, 0u, 0u};
    }
  }
  __device__ __forceinline__ void store(uint16_t* to) const {
    if constexpr (D == 128) store_u32x4(to, x);
    else *reinterpret_cast<uint2*>(to) = uint2{x[0], x[1]};
  }
  // Its codes (d = 64: the lower half), with the scale byte of the block that it shares with the
  // neighbouring lanes.
  __device__ __forceinline__ uint32_t encode(uint32_t* byte) const {
    uint32_t m = kv4_max(kv4_max(kv4_max(kv4_max(0u, x[0]), x[1]), x[2]), x[3]);
#pragma unroll
    for (int o = 1; o < Kv4<D>::kVLanes; o *= 2) m = max(m, (uint32_t)__shfl_xor((int)m, o, 64));
    *byte = kv4_scale_byte(m);
    return kv4_codes(x, kv4_factor(*byte));
  }
  __device__ __forceinline__ void decode(uint32_t codes, uint32_t byte) {
    const float f = kv4_factor(byte);
    x = u32x4{kv4_pair<0>(codes, f), kv4_pair<1>(codes, f), 0u, 0u};
    if constexpr (D == 128) x[2] = kv4_pair<2>(codes, f), x[3] = kv4_pair<3>(codes, f);
  }
};

template <int D>
__device__ __forceinline__ void put_codes(uint8_t* to, uint32_t codes) {
  if constexpr (D == 128) *reinterpret_cast<uint32_t*>(to) = codes;
  else *reinterpret_cast<uint16_t*>(to) = (uint16_t)codes;
}

template <int D>
__device__ __forceinline__ uint32_t get_codes(const uint8_t* from) {
  if constexpr (D == 128) return *reinterpret_cast<const uint32_t*>(from);
  else return *reinterpret_cast<const uint16_t*>(from);
}

template <int D>
__device__ __forceinline__ void append_page(const Kv4StoreArgs& a, uint8_t* blk, int64_t row0, int head,
                                            int s0, int n) {
  using F = Kv4<D>;
  const int lane = threadIdx.x & 63, r = lane & 15, quad = lane >> 4;
  Piece<D> k[4], v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int slot = 4 * quad + i;
    k[i].x = v[i].x = zero_u32x4();
    if (slot >= s0 && slot < s0 + n) {
      const int64_t at = ((row0 + slot - s0) * a.num_kv_heads + head) * D + F::kSpan * r;
      k[i].load(a.k_new + at);
      v[i].load(a.v_new + at);
    }
  }
  const bool scale_lane = r % F::kVLanes == 0;
  uint32_t codes[4], bytes = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int slot = 4 * quad + i;
    const bool in = slot >= s0 && slot < s0 + n;
    uint32_t byte;
    const uint32_t c = k[i].encode(&byte);
    if (in) {
      put_codes<D>(blk + F::k_word(r, slot), c);
      if (scale_lane) blk[F::k_byte(r, slot)] = (uint8_t)byte;
    }
    codes[i] = v[i].encode(&byte);
    bytes |= byte << (8 * i);
  }
  if (n == kPage) {
    uint8_t* to = blk + F::kVCodes + lane * F::kLane;
    if constexpr (D == 128) store_u32x4(to, u32x4{codes[0], codes[1], codes[2], codes[3]});
    else
      *reinterpret_cast<uint2*>(to) =
          uint2{(codes[0] & 0xFFFFu) | (codes[1] << 16), (codes[2] & 0xFFFFu) | (codes[3] << 16)};
    if (scale_lane) *reinterpret_cast<uint32_t*>(blk + F::v_scale(lane)) = bytes;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int slot = 4 * quad + i;
      if (slot < s0 || slot >= s0 + n) continue;
      put_codes<D>(blk + F::v_word(r, slot), codes[i]);
      if (scale_lane) blk[F::v_scale(lane) + i] = (uint8_t)(bytes >> (8 * i));
    }
  }
}

// A page's codes and scales in a lane: piece r of slots 4 quad .. + 3.
template <int D>
struct PageCodes {
  uint32_t k[4], kb[4], v[4], vb;
  // blk == null (a page id out of range): zeros
  __device__ __forceinline__ void load(const uint8_t* blk, int s0, int n) {
    using F = Kv4<D>;
    const int lane = threadIdx.x & 63, r = lane & 15, quad = lane >> 4;
    vb = 0x7F7F7F7Fu;
#pragma unroll
    for (int i = 0; i < 4; ++i) k[i] = v[i] = 0, kb[i] = 127;
    if (!blk || 4 * quad + 4 <= s0 || 4 * quad >= s0 + n) return;
    if constexpr (D == 128) {
      const u32x4 x = load_u32x4(blk + F::kVCodes + lane * F::kLane);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = x[i];
    } else {
      const uint2 x = *reinterpret_cast<const uint2*>(blk + F::kVCodes + lane * F::kLane);
      v[0] = x.x, v[1] = x.x >> 16, v[2] = x.y, v[3] = x.y >> 16;
    }
    vb = *reinterpret_cast<const uint32_t*>(blk + F::v_scale(lane));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      k[i] = get_codes<D>(blk + F::k_word(r, 4 * quad + i));
      kb[i] = blk[F::k_byte(r, 4 * quad + i)];
    }
  }
  // Rows of slots [s0, s0 + n): slot s of K and V to k_out / v_out + (s - s0) * stride.
  __device__ __forceinline__ void store(uint16_t* k_out, uint16_t* v_out, int64_t stride, int s0, int n) const {
    const int lane = threadIdx.x & 63, r = lane & 15, quad = lane >> 4;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int slot = 4 * quad + i;
      if (slot < s0 || slot >= s0 + n) continue;
      const int64_t at = (slot - s0) * stride + Kv4<D>::kSpan * r;
      Piece<D> x;
      x.decode(k[i], kb[i]);
      x.store(k_out + at);
      x.decode(v[i], (vb >> (8 * i)) & 255u);
      x.store(v_out + at);
    }
  }
};

template <int D, bool kAppend>
__global__ __launch_bounds__(kStoreWaves * 64) void kv4_store_kernel(Kv4StoreArgs a) {
  const int wave = threadIdx.x >> 6;
  const int head = blockIdx.y * kStoreWaves + wave;
  const Kv4StoreItem it = a.items[blockIdx.x];
  if (a.reads.done) {
    asm volatile("" ::"v"(it.row0));  // the record has arrived
    __syncthreads();
    if (threadIdx.x == 0) plan_read(a.reads, blockIdx.y * gridDim.x + blockIdx.x);
  }
  const int32_t phys = a.block_table[(int64_t)it.task * a.bt_stride + it.lpage];
  const bool page_ok = phys >= 0 && phys < a.num_pages;
  if (!page_ok && threadIdx.x == 0) atomicOr(a.error_flags, 1);
  if (head >= a.num_kv_heads || (kAppend && !page_ok)) return;
  const int s0 = it.span & 31, n = it.span >> 5;
  const int64_t row0 = it.row0;
  uint8_t* blk = a.pool + ((int64_t)(page_ok ? phys : 0) * a.num_kv_heads + head) * kv4_block_bytes(D);
  if constexpr (kAppend) {
    append_page<D>(a, blk, row0, head, s0, n);
  } else {
    const int64_t at = (row0 * a.num_kv_heads + head) * D;
    PageCodes<D> x;
    x.load(page_ok ? blk : nullptr, s0, n);
    x.store(a.k_out + at, a.v_out + at, (int64_t)a.num_kv_heads * D, s0, n);
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
  // the next block's codes are loaded before one's rows are stored
  const int blocks = it.pages * a.num_kv_heads;
  auto load = [&](PageCodes<D>& x, int i) {
    const int page = i / a.num_kv_heads, head = i - page * a.num_kv_heads;
    const int32_t phys = row[page];
    const bool ok = phys >= 0 && phys < a.num_pages;
    if (!ok && (threadIdx.x & 63) == 0) atomicOr(a.error_flags, 1);
    const uint8_t* blk = a.pool + ((int64_t)(ok ? phys : 0) * a.num_kv_heads + head) * kv4_block_bytes(D);
    x.load(ok ? blk : nullptr, 0, kPage);
  };
  PageCodes<D> next;
  if (wave < blocks) load(next, wave);
  for (int i = wave; i < blocks; i += kStoreWaves) {
    const PageCodes<D> x = next;
    if (i + kStoreWaves < blocks) load(next, i + kStoreWaves);
    // (the staging pages of an item follow each other, like the heads of a page)
    const int64_t at = ((int64_t)it.to * a.num_kv_heads + i) * (kPage * D);
    x.store(a.k_stage + at, a.v_stage + at, D, 0, kPage);
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
