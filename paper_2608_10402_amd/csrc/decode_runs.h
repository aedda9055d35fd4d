// decode_runs.h -- how the waves of a decode in runs put the parts of a cut task together: the
// parts of a workgroup's consecutive runs in LDS, those of several workgroups through the
// workspace, with a flag per part (attn_decode_stream.hip, kv4_decode.hip).
#pragma once

#include "attn_decode.h"

namespace tide {
namespace kern {

// Rows of one unit being merged by a wave: lanes L j .. L j + L - 1 hold head j0 + j (64 / L
// heads a pass), each lane D / L consecutive head-dim entries.  With M the largest m seen, acc
// = sum 2^(m_s - M) o_s, l and lx the same sums of the bf16-rounded and the exact weights.
template <int D, int L>
struct RowMerge {
  static constexpr int kPer = D / L, kV = kPer / 4;
  f32x4 acc[kV];
  float mx, l, lx;
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int k = 0; k < kV; ++k) acc[k] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    mx = kNoMax;
    l = lx = 0.0f;
  }
  // makes `m` part of the running maximum
  __device__ __forceinline__ void raise(float m) {
    const float mn = fmaxf(mx, m), w = fast_exp2(mx - mn);
#pragma unroll
    for (int k = 0; k < kV; ++k) acc[k] *= w;
    l *= w;
    lx *= w;
    mx = mn;
  }
  // adds a part whose maximum is included in mx already
  __device__ __forceinline__ void add(f32x4 ml, const f32x4 (&o)[kV]) {
    const float w = fast_exp2(ml[0] - mx);
    l += w * ml[1];
    lx += w * ml[2];
#pragma unroll
    for (int k = 0; k < kV; ++k) acc[k] += w * o[k];
  }
};

// The parts of one kv head.  A part has `cols` rows (one per query row of the unit); Rows(task,
// j) is the packed output row of row j, or negative where the unit has no row j.
template <int D, int kWaves, class Rows>
struct RunParts {
  float* part_o;   // [slots][cols][D], from slot0 this head's
  float* part_ml;  // [slots][cols][4]
  uint64_t* flags;
  uint64_t call;
  uint16_t* out;
  float* lse;
  StreamSlots slots;
  int64_t slot0;
  int cols;
  Rows row_of;

  template <int L>
  __device__ __forceinline__ void write_row(const RowMerge<D, L>& rm, int64_t row, int sub) const {
    using RM = RowMerge<D, L>;
    const float inv = 1.0f / rm.l;
    uint16_t* orow = out + row * D + RM::kPer * sub;
#pragma unroll
    for (int k = 0; k < RM::kV; ++k) {
      const uint2 x = {pack_bf16x2(rm.acc[k][0] * inv, rm.acc[k][1] * inv),
                       pack_bf16x2(rm.acc[k][2] * inv, rm.acc[k][3] * inv)};
      *reinterpret_cast<uint2*>(orow + 4 * k) = x;
    }
    if (lse && sub == 0) lse[row] = (rm.mx + __log2f(rm.lx)) * kLn2;
  }

  // Merges every part of a task in key order and writes this head's rows.
  template <int L>
  __device__ __forceinline__ void merge(const StreamUnit& u, int task) const {
    using RM = RowMerge<D, L>;
    constexpr int kB = 16 / RM::kV;  // parts loaded together
    const int lane = threadIdx.x & 63;
    const int sub = lane % L;
    const int np = stream_parts(u, kWaves);
    for (int j0 = 0; j0 < cols; j0 += 64 / L) {
      const int j = j0 + lane / L;
      RM rm;
      rm.clear();
      for (int e0 = 0; e0 < np; e0 += kB) {
        f32x4 ml[kB], po[kB][RM::kV];
#pragma unroll
        for (int i = 0; i < kB; ++i) {
          const int e = e0 + i;
          const bool in = e < np;
          const int64_t slot = slot0 + stream_slot(u, slots, task, in ? e : 0);
          const auto rml = __builtin_amdgcn_make_buffer_rsrc(
              part_ml + slot * cols * 4, 0, in ? cols * 16 : 0, 0x00020000);
          const auto rpo = __builtin_amdgcn_make_buffer_rsrc(
              part_o + slot * cols * D, 0, in ? cols * D * 4 : 0, 0x00020000);
          ml[i] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rml, 16 * j, 0, kDeviceScope));
#pragma unroll
          for (int k = 0; k < RM::kV; ++k)
            po[i][k] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(
                                                     rpo, 4 * (j * D + RM::kPer * sub + 4 * k), 0, kDeviceScope));
        }
        float m = kNoMax;
#pragma unroll
        for (int i = 0; i < kB; ++i) {
          if (e0 + i >= np) ml[i][0] = kNoMax;
          m = fmaxf(m, ml[i][0]);
        }
        rm.raise(m);
#pragma unroll
        for (int i = 0; i < kB; ++i) rm.add(ml[i], po[i]);
      }
      const int64_t row = j < cols ? row_of(task, j) : -1;
      if (row >= 0) write_row<L>(rm, row, sub);
    }
  }

  // Flags the part in `slot` complete; a part that then finds all of the task's flags set merges.
  // Each flag is written (device scope, acknowledged) after the part's own stores and before
  // it looks, so the part whose flag lands last finds them all; should two find them, both
  // write the same rows.  Unlike a counter, the flags need no zeros to start from.
  __device__ __forceinline__ void arrive(const StreamUnit& u, int task, int64_t slot) const {
    const int lane = threadIdx.x & 63;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    if (lane == 0)
      __hip_atomic_store(flags + slot, call, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    const int np = stream_parts(u, kWaves);
    for (int e = lane; e - lane < np; e += 64) {
      const int64_t other = slot0 + stream_slot(u, slots, task, min(e, np - 1));
      if (__any(__hip_atomic_load(flags + other, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) != call))
        return;
    }
    asm volatile("" ::: "memory");
    if (cols > 4) merge<8>(u, task);
    else merge<16>(u, task);
  }

  // Combines the `len` consecutive waves' partials of one task that lie in LDS from lds_o (outputs,
  // row j at 4 D j, its 16-byte granule g at g ^ (j % 16)) and lds_s (statistics, 16 bytes a row), a
  // wave's `stride` and `stride_s` bytes behind the last one's; whole: the unit lies inside this workgroup.
  template <int L>
  __device__ __forceinline__ void combine(const uint8_t* lds_o, const uint8_t* lds_s, int stride, int stride_s, int len,
                                          bool whole, int run, int task) const {
    using RM = RowMerge<D, L>;
    const int lane = threadIdx.x & 63;
    const int sub = lane % L;
    for (int j0 = 0; j0 < cols; j0 += 64 / L) {
      const int j = j0 + lane / L;
      const int jr = j < cols ? j : 0;
      RM rm;
      rm.clear();
      for (int x = 0; x < len; ++x) {
        const uint8_t* xo = lds_o + x * stride + 4 * D * jr;
        const f32x4 ml = *reinterpret_cast<const f32x4*>(lds_s + x * stride_s + 16 * jr);
        f32x4 po[RM::kV];
#pragma unroll
        for (int k = 0; k < RM::kV; ++k)
          po[k] = *reinterpret_cast<const f32x4*>(xo + 16 * ((RM::kV * sub + k) ^ (jr & 15)));
        rm.raise(ml[0]);
        rm.add(ml, po);
      }
      if (j >= cols) continue;
      if (whole) {
        const int64_t row = row_of(task, j);
        if (row >= 0) write_row<L>(rm, row, sub);
      } else {
        const int64_t slot = slot0 + slots.open(run, task);
        float* po = part_o + slot * cols * D;
#pragma unroll
        for (int k = 0; k < RM::kV; ++k)
          store_f32x4_device(po, cols * D * 4, 4 * (j * D + RM::kPer * sub + 4 * k), rm.acc[k]);
        if (sub == 0)
          store_f32x4_device(part_ml + slot * cols * 4, cols * 16, 16 * j,
                             f32x4{rm.mx, rm.l, rm.lx, 0.0f});
      }
    }
  }

  __device__ __forceinline__ void close(const uint8_t* lds_o, const uint8_t* lds_s, int stride, int stride_s, int len,
                                        bool whole, const StreamUnit& u, int run, int task) const {
    if (cols > 4) combine<8>(lds_o, lds_s, stride, stride_s, len, whole, run, task);
    else combine<16>(lds_o, lds_s, stride, stride_s, len, whole, run, task);
    if (!whole) arrive(u, task, slot0 + slots.open(run, task));
  }
};

}  // namespace kern
}  // namespace tide
