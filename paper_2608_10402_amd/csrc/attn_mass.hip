// Attention mass: adds, to a running sum per cached key and kv head, the softmax weights that the
// key gets from the new tokens' query rows,
//     mass[p] += sum over tokens j with P + j >= p, query heads h of the group: exp(s_jhp - lse_jh),
// with the scores s recomputed from the cache and the log-sum-exps that the attention returned.
//
// A wave takes 64 keys (4 pages) of one (task, kv head), holds their K in registers as the A
// operands of S^T = K Q^T and walks the query rows 16 at a time: a lane then owns one row's scores
// of 16 keys and adds exp2(s - lse) to 16 sums, which are added across the 16 rows' lanes once, at
// the end, in a fixed order.  Every sum has one writer: no atomics, and repeated calls give the
// same bits.  Scores, weights and sums are fp32.
//
// The blocks of all tasks, laid end to end, are cut into runs of near equal cost (rows and reads; whole
// blocks, so that runs of few differ much), and one wave takes a run of one kv head, the next block's
// loads behind the last rows of one.
// Query rows pass through a wave's own 4 KB of LDS, whole rows at a time, the next 16 on their way
// while 16 are used: as operands straight from memory, 64 lanes read 64 separate pieces, which
// kept the L1 busy for 73% of a call of 43 rows x 7 heads.  Where 16 rows are all of every task's
// (kOneTrip: decode steps), they are read as operands, once a task, since the compiler lets every
// read of LDS wait for the K loads in flight, too.
//
// Decode steps are bound by reading: 64 tasks of 1k-16k keys (32 / 8 heads, d = 128, 4 bits) 69 us for
// 0.33 GB of codes and sums, the rate of a large copy; over bf16 keys 233 us for 1.13 GB.
// The votes of 32-64 tokens a task are far from it: 16 tasks of 2k-16k keys (28 / 4) 76 us over bf16
// and 70 over 4 bits, of 27 for the bytes or the FLOPs.  A trip issues 88 vector instructions beside
// its MFMAs, of which the scores' exponential, multiply-add and sum are 48, and 88 scalar ones: the
// others find the next rows (descriptors, divisions by the group).  Runs there are 2 or 3 blocks (the
// mean costs 0.68 of the longest), so 1.8 of 3 waves a SIMD live over the kernel, vector instructions
// issue in 35% of the SIMDs' cycles and MFMAs run in 18%.  32 rows a trip took 1% more, blocks of
// 32 keys 2% more, 6 waves a workgroup 45% more, rows staged two trips ahead 8% more.
#include "attn_decode.h"
#include "kv4.h"

namespace tide {
namespace kern {

typedef const __attribute__((address_space(4))) MassRun const_run;

// 16 rows of Q into LDS, laid out like the 16 rows of a K page (KLds), and their log-sum-exps.  A lane
// loads pieces of rows lane / 8 and lane / 8 + 8, whose byte offsets are at_lo and at_hi.
template <int D>
__device__ __forceinline__ void rows_to_lds(__amdgpu_buffer_rsrc_t q, uint8_t* qbuf, uint32_t at_lo, uint32_t at_hi,
                                            __amdgpu_buffer_rsrc_t lse, float* lbuf, uint32_t at_lse) {
  using L = KLds<D>;
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int i = 0; i < L::kDma; ++i) {
    const int r = 8 * (i / L::kHalves) + (lane >> 3);  // as L::src_offset, without the row's own offset
    const uint32_t in_row = L::src_offset(i, lane) - (uint32_t)(r * 2 * D);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(q, (lds_void*)(qbuf + 1024 * i), 16,
                                             (i < L::kHalves ? at_lo : at_hi) + in_row, 0, 0, 0);
  }
  __builtin_amdgcn_raw_ptr_buffer_load_lds(lse, (lds_void*)lbuf, 4, at_lse, 0, 0, 0);
}

// Adds the first 2 kHalf sums of lanes whose columns differ by kHalf: the lane keeps the half that its
// column's bit names.
template <int kHalf>
__device__ __forceinline__ void fold(float (&acc)[16], int col) {
  const bool up = (col & kHalf) != 0;
#pragma unroll
  for (int i = 0; i < kHalf; ++i) {
    const float send = up ? acc[i] : acc[i + kHalf], keep = up ? acc[i + kHalf] : acc[i];
    acc[i] = keep + xor_shfl(send, kHalf);
  }
}

template <int D, bool kKv4, bool kOneTrip>
__global__ __launch_bounds__(mass_waves(kOneTrip) * 64)
    __attribute__((amdgpu_waves_per_eu(kOneTrip ? 4 : 3, kOneTrip ? 4 : 3)))
void attn_mass_kernel(MassArgs a) {
  using F = Kv4<D>;
  constexpr int kC = D / 32, kWaves = mass_waves(kOneTrip);
  constexpr int kBlk = kKv4 ? F::kBlock : kPage * D * 2;
  const int lane = threadIdx.x & 63, col = lane & 15, grp = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // workgroup b runs on die b % 8: each die takes neighbouring runs, whose query rows then stay in its L2
  const int groups = mass_groups(a.num_runs, a.num_kv_heads, kOneTrip), per = (groups + kXcds - 1) / kXcds;
  const int wg = (blockIdx.x % kXcds) * per + blockIdx.x / kXcds;
  const int Hkv = a.num_kv_heads, rg = wg / Hkv, head = wg - rg * Hkv;
  const int run = rg * kWaves + wave;
  const bool live = wg < groups && run < a.num_runs;
  const const_run* it = (const const_run*)(a.runs + (live ? run : 0));
  const int n = live ? it->blocks : 0;
  using L = KLds<D>;  // 16 rows of Q lie in LDS like the rows of a K page
  __shared__ __attribute__((aligned(1024))) uint8_t q_lds[kOneTrip ? 16 : kWaves * L::kPageBytes];
  __shared__ __attribute__((aligned(16))) float lse_lds[kOneTrip ? 4 : kWaves * 64];
  uint8_t* const qbuf = q_lds + (kOneTrip ? 0 : wave * L::kPageBytes);
  float* const lbuf = lse_lds + (kOneTrip ? 0 : wave * 64);
  // this lane's key of a block once the rows' lanes are summed: page col / 4, slot
  const int my_page = col >> 2, my_slot = 4 * grp + (col & 3);

  // Position in the sequence of the tasks' blocks; all wave-uniform.
  struct Cursor {
    int task, block, blocks, row_start, prefix, extend, counted;
  };
  auto load_task = [&](Cursor& c) {
    const const_i32* t = (const const_i32*)(a.tasks + c.task);
    c.row_start = t[0];
    c.prefix = t[1];
    c.extend = t[2];
    c.counted = t[3];
    c.blocks = c.extend > 0 ? (c.prefix + c.extend - 1) / kMassKeys + 1 : 0;
  };
  auto next_block = [&](Cursor& c, bool more) {  // more: there is one (it is not looked for otherwise)
    if (++c.block < c.blocks || !more) return;
    c.block = 0;
    do {
      ++c.task;
      load_task(c);
    } while (c.blocks == 0);
  };
  Cursor cu = {it->task, it->block, 0, 0, 0, 0, 0};
  load_task(cu);

  // Rows: 16 a trip, numbered token by token and in a token by query head of the group, from the first
  // token that sees one of the block's keys.
  const int G = a.group, dt = 16 / G, dh = 16 - dt * G;
  const uint32_t per_group = 65536u / (uint32_t)G + 1;  // x / G for the x < 32 below
  int first = 0, first_h = 0;  // token and query head of the trip's first row
  auto restart = [&]() {
    first = max(0, kMassKeys * cu.block - cu.prefix);
    first_h = 0;
  };
  auto advance = [&]() {  // the next 16 rows
    first += dt;
    first_h += dh;
    if (first_h >= G) first_h -= G, ++first;
  };
  auto token_of = [&](int r) { return (int)(__umul24(first_h + r, per_group) >> 16); };  // of row r, from `first`
  // Row r's place behind the first token's first query head, in rows.  In place of rows past the task's last
  // that one is read: zeros would make NaN of a key that holds infinities, whose scores with the task's
  // own rows may all be -inf.
  auto place_of = [&](int r) {
    const int i = min(first_h + r, G * min(cu.extend - first, 32) - 1);
    return __umul24(__umul24(i, per_group) >> 16, a.num_q_heads - G) + (uint32_t)i;
  };
  bf16x8 q[kC];
  float lse = 0.0f;
  auto load_rows = [&]() {
    const int64_t row = ((int64_t)cu.row_start + first) * a.num_q_heads + head * G;
    const int64_t rows = (int64_t)(cu.extend - first - 1) * a.num_q_heads + G;  // from there to the task's end
    const auto q_rows = block_rsrc(reinterpret_cast<const uint8_t*>(a.q + row * D),
                              (int)min((int64_t)INT32_MAX, rows * (D * 2)));
    const auto l_rows = block_rsrc(reinterpret_cast<const uint8_t*>(a.lse + row), (int)min((int64_t)INT32_MAX, rows * 4));
    if constexpr (kOneTrip) {
      const uint32_t at = place_of(col);
#pragma unroll
      for (int c = 0; c < kC; ++c)
        q[c] = __builtin_bit_cast(bf16x8, __builtin_amdgcn_raw_buffer_load_b128(
                                              q_rows, at * (D * 2) + (kKv4 ? (D / 2) * grp + 16 * c : 64 * c + 16 * grp), 0, 0));
      lse = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(l_rows, at * 4, 0, 0)) * kLog2e;
      return;
    }
    const uint32_t at_lo = place_of(lane >> 3) * (D * 2), at_hi = place_of(8 + (lane >> 3)) * (D * 2);
    rows_to_lds<D>(q_rows, qbuf, at_lo, at_hi, l_rows, lbuf, lane < 16 ? place_of(col) * 4 : 0x7FFFFFFCu);
  };
  const uint32_t q_even = L::lds_offset(col, grp), q_odd = L::lds_offset(col, 4 + grp);

  // Loads of the load cursor's block: K as the operand of MFMA c of page t, entries (bf16) 32 c + 8 grp
  // of slot col, or (4 bit) D/4 grp + 8 c, Q below in the same order; the old sum of this lane's key and
  // its page (-1: not written).  Past the run's end, a context and for invalid page ids through
  // zero-length buffers.  Page ids are scalar loads, fetched one block ahead.
  bool flag_error = false;
  Cursor ld = cu;
  int left = n;
  int32_t pg[4];
  u32x4 raw[4][kKv4 ? 1 : kC];
  uint32_t scale[4];
  float old;
  int32_t page;
  auto fetch_pages = [&]() {
    const const_i32* table = (const const_i32*)(a.block_table + (int64_t)ld.task * a.bt_stride);
    const int last = max(0, (ld.prefix + ld.extend - 1) / kPage);
#pragma unroll
    for (int t = 0; t < 4; ++t) pg[t] = table[left > 0 ? min(4 * ld.block + t, last) : 0];
  };
  auto issue = [&]() {
    const int kv_len = ld.prefix + ld.extend, kb = kMassKeys * ld.block;
    page = -1;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const bool in = left > 0 && kb + 16 * t < kv_len;
      const bool ok = in && pg[t] >= 0 && pg[t] < a.num_pages;
      flag_error |= in && !ok;
      const auto blk = block_rsrc(static_cast<const uint8_t*>(a.pool) + ((int64_t)(ok ? pg[t] : 0) * Hkv + head) * kBlk,
                                  ok ? kBlk : 0);
      if constexpr (kKv4) {
        if constexpr (D == 128) {
          raw[t][0] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(blk, 16 * lane, 0, kStreamPolicy));
        } else {
          const uint2 x =
              __builtin_bit_cast(uint2, __builtin_amdgcn_raw_buffer_load_b64(blk, 8 * lane, 0, kStreamPolicy));
          raw[t][0] = u32x4{x.x, x.y, 0u, 0u};
        }
        scale[t] = __builtin_amdgcn_raw_buffer_load_b8(blk, F::k_scale(lane), 0, kStreamPolicy);
      } else {
#pragma unroll
        for (int c = 0; c < kC; ++c)
          raw[t][c] = __builtin_bit_cast(
              u32x4, __builtin_amdgcn_raw_buffer_load_b128(blk, col * D * 2 + 64 * c + 16 * grp, 0, kStreamPolicy));
      }
      if (ok && my_page == t && kb + 16 * t + my_slot < kv_len) page = pg[t];
    }
    old = page >= 0 && kb + 16 * my_page + my_slot < ld.counted
              ? a.mass[((int64_t)page * Hkv + head) * kPage + my_slot]
              : 0.0f;
    if (left > 0) {
      --left;
      next_block(ld, left > 0);
    }
    fetch_pages();
  };

  bool fresh = true;  // the rows in LDS were loaded since they were last used
  if (n > 0) {
    fetch_pages();
    issue();
    restart();
    load_rows();
  }
  for (int done = 0; done < n;) {
    const int kb = kMassKeys * cu.block;
    bf16x8 kk[4][kC];
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int c = 0; c < kC; ++c) {
        if constexpr (kKv4) kk[t][c] = kv4_octet(raw[t][0][c], kv4_factor(scale[t]));
        else kk[t][c] = as_bf16x8(raw[t][c]);
      }
    const float was_sum = old;
    float* const sum = page >= 0 ? a.mass + ((int64_t)page * Hkv + head) * kPage + my_slot : nullptr;
    float acc[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[i] = 0.0f;
    ++done;
    bool more = true;
    auto next_rows = [&]() {
      advance();
      more = !kOneTrip && first < cu.extend;
      fresh = more;
      if (!more) {  // the next block's first; those of a task with one trip of rows serve all its blocks
        const int task = cu.task;
        const bool one = cu.extend * G <= 16;
        next_block(cu, done < n);
        restart();
        fresh = done < n && !(one && cu.task == task && first == 0);
      }
      if (fresh) load_rows();
    };
    do {
      if constexpr (!kOneTrip) {
        if (fresh) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the rows are in LDS
#pragma unroll
        for (int c = 0; c < kC; ++c) {
          // granule of entries 32 c + 8 grp, or D/4 grp + 8 c
          const uint32_t at = kKv4 ? L::lds_offset(col, (D / 32) * grp + c) : 1024 * (c >> 1) + (c & 1 ? q_odd : q_even);
          q[c] = as_bf16x8(*reinterpret_cast<const u32x4*>(qbuf + at));
        }
        lse = lbuf[col] * kLog2e;
        // (the reads are done before the next rows' loads write there)
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      }
      const int row_tok = first + token_of(col);
      float bias = row_tok < cu.extend ? lse : INFINITY;  // no row: no weight
      const int seen = cu.prefix + row_tok + 1 - kb - 4 * grp;  // keys that the row sees, from this lane's first
      const bool partial = kb > cu.prefix + first + 1 - kMassKeys;
      if constexpr (!kOneTrip) next_rows();
      f32x4 s[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        s[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int c = 0; c < kC; ++c) s[t] = mfma16(kk[t][c], q[c], s[t]);
      }
      if (partial) {
        auto hidden = [&](int i) { return 16 * (i >> 2) + (i & 3) >= seen; };
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (hidden(i)) s[i >> 2][i & 3] = -INFINITY;
        // a log-sum-exp that would turn hidden keys' weights into NaN goes into the others' scores
        const bool odd = !(bias > -INFINITY);
        if (__any(odd)) {
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (odd && !hidden(i)) s[i >> 2][i & 3] -= bias;
          bias = odd ? 0.0f : bias;
        }
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[i] += fast_exp2(s[i >> 2][i & 3] * a.scale_log2 - bias);
      if constexpr (kOneTrip) next_rows();
    } while (!kOneTrip && more);
    issue();
    // across the 16 lanes of a row: lane `col` ends with sum `col`
    fold<8>(acc, col);
    fold<4>(acc, col);
    fold<2>(acc, col);
    fold<1>(acc, col);
    if (sum) *sum = was_sum + acc[0];
  }
  if (flag_error && lane == 0) atomicOr(a.error_flags, 1);
  if (a.reads.done) {
    __syncthreads();
    if (threadIdx.x == 0 && wg < groups) plan_read(a.reads, wg);
  }
}

template <int D, bool kKv4>
hipError_t launch_mass(const MassArgs& a, hipStream_t stream) {
  const dim3 grid((mass_groups(a.num_runs, a.num_kv_heads, a.one_trip) + kXcds - 1) / kXcds * kXcds);
  const dim3 block(mass_waves(a.one_trip) * 64);
  if (a.one_trip) hipLaunchKernelGGL((attn_mass_kernel<D, kKv4, true>), grid, block, 0, stream, a);
  else hipLaunchKernelGGL((attn_mass_kernel<D, kKv4, false>), grid, block, 0, stream, a);
  return hipGetLastError();
}

// Every variant is instantiated explicitly (see attn_decode.hip).
template __global__ void attn_mass_kernel<128, false, false>(MassArgs);
template __global__ void attn_mass_kernel<128, false, true>(MassArgs);
template __global__ void attn_mass_kernel<128, true, false>(MassArgs);
template __global__ void attn_mass_kernel<128, true, true>(MassArgs);
template __global__ void attn_mass_kernel<64, false, false>(MassArgs);
template __global__ void attn_mass_kernel<64, false, true>(MassArgs);
template __global__ void attn_mass_kernel<64, true, false>(MassArgs);
template __global__ void attn_mass_kernel<64, true, true>(MassArgs);

}  // namespace kern

hipError_t launch_attn_mass(const MassArgs& a, int head_dim, bool kv4, hipStream_t stream) {
  if (head_dim == 128) return kv4 ? kern::launch_mass<128, true>(a, stream) : kern::launch_mass<128, false>(a, stream);
  if (head_dim == 64) return kv4 ? kern::launch_mass<64, true>(a, stream) : kern::launch_mass<64, false>(a, stream);
  return hipErrorInvalidValue;
}

}  // namespace tide
