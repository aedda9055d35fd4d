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
#include "kernels.h"
#include "kv4.h"

namespace tide {
namespace kern {

constexpr int kMassWaves = 4;
static_assert(kMassKeys == kMassWaves * 64, "a wave takes 64 keys");

template <int D, bool kKv4>
__global__ __launch_bounds__(kMassWaves * 64) void attn_mass_kernel(MassArgs a) {
  using F = Kv4<D>;
  constexpr int kC = D / 32;
  const int lane = threadIdx.x & 63, col = lane & 15, grp = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int item = blockIdx.x / a.num_kv_heads, head = blockIdx.x - item * a.num_kv_heads;
  const MassItem it = a.items[item];
  const TaskDesc td = a.tasks[it.task];
  const int kv_len = td.prefix + td.extend;
  const int kb = it.key0 + 64 * wave;
  if (a.reads.done) {
    asm volatile("" ::"v"(it.key0), "v"(td.aux));  // both records have arrived
    __syncthreads();
    if (threadIdx.x == 0) plan_read(a.reads, blockIdx.x);
  }
  if (kb >= kv_len) return;
  const int32_t* row = a.block_table + (int64_t)it.task * a.bt_stride + kb / kPage;
  const int npages = min(4, (kv_len - kb + kPage - 1) / kPage);
  int32_t pg[4];
  bool ok[4];
#pragma unroll
  for (int t = 0; t < 4; ++t) pg[t] = load_page_id(row, t < npages ? t : 0);
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    const bool in = pg[t] >= 0 && pg[t] < a.num_pages;
    ok[t] = in && t < npages;
    if (!in && lane == 0) atomicOr(a.error_flags, 1);
  }
  bf16x8 kk[4][kC];
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    const int64_t b = (int64_t)(ok[t] ? pg[t] : 0) * a.num_kv_heads + head;
    if constexpr (kKv4) {
      const uint8_t* blk = static_cast<const uint8_t*>(a.pool) + b * F::kBlock;
      uint32_t w[kC] = {};
      uint32_t byte = 127;
      if (ok[t]) {
        if constexpr (D == 128) {
          const u32x4 x = load_u32x4(blk + lane * 16);
#pragma unroll
          for (int c = 0; c < 4; ++c) w[c] = x[c];
        } else {
          const uint2 x = *reinterpret_cast<const uint2*>(blk + lane * 8);
          w[0] = x.x, w[1] = x.y;
        }
        byte = blk[F::k_scale(lane)];
      }
#pragma unroll
      for (int c = 0; c < kC; ++c) kk[t][c] = kv4_octet(w[c], kv4_factor(byte));
    } else {
      const uint16_t* blk = static_cast<const uint16_t*>(a.pool) + b * (kPage * D) + col * D + (D / 4) * grp;
#pragma unroll
      for (int c = 0; c < kC; ++c) kk[t][c] = as_bf16x8(ok[t] ? load_u32x4(blk + 8 * c) : zero_u32x4());
    }
  }
  // this lane's key after the sum across lanes
  const int my_page = col >> 2, my_slot = 4 * grp + (col & 3);
  const int key = kb + 16 * my_page + my_slot;
  int32_t page = pg[0];
  bool mine = ok[0];
#pragma unroll
  for (int t = 1; t < 4; ++t)
    if (my_page == t) page = pg[t], mine = ok[t];
  mine = mine && key < kv_len;
  float* sum = a.mass + ((int64_t)(mine ? page : 0) * a.num_kv_heads + head) * kPage + my_slot;
  const float old = mine && key < td.aux ? *sum : 0.0f;

  float acc[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) acc[i] = 0.0f;
  // rows: token `tok`, query head `h` of the group; 16 of them a trip, from the first token that
  // sees a key of the block
  const int G = a.group, dt = 16 / G, dh = 16 - dt * G;
  const int tok0 = max(0, kb - td.prefix);
  int tok = tok0 + col / G, h = col % G;
  bf16x8 qf[kC], qn[kC];
  float lse, lse_n;
  auto load_row = [&](bf16x8 (&q)[kC], float& l) {
    const bool in = tok < td.extend;
    const int64_t r = ((int64_t)td.row_start + (in ? tok : 0)) * a.num_q_heads + head * G + h;
    const uint16_t* from = a.q + r * D + (D / 4) * grp;
#pragma unroll
    for (int c = 0; c < kC; ++c) q[c] = as_bf16x8(load_u32x4(from + 8 * c));
    l = in ? a.lse[r] * kLog2e : INFINITY;
  };
  load_row(qf, lse);
  for (;;) {
    const int cur_tok = tok;
    const bool row_ok = tok < td.extend;
    const int first = __builtin_amdgcn_readfirstlane(tok);  // lane 0 holds the trip's first row
    tok += dt;
    h += dh;
    if (h >= G) h -= G, ++tok;
    const bool more = __builtin_amdgcn_readfirstlane(tok) < td.extend;
    if (more) load_row(qn, lse_n);
    f32x4 s[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      s[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int c = 0; c < kC; ++c) s[t] = mfma16(kk[t][c], qf[c], s[t]);
    }
    const bool partial = kb + 63 > td.prefix + first || !row_ok;
    if (__any(partial)) {
      const int keys = row_ok ? td.prefix + cur_tok + 1 - kb - 4 * grp : 0;  // that the row sees, from this lane's first
#pragma unroll
      for (int i = 0; i < 16; ++i)
        acc[i] += 16 * (i >> 2) + (i & 3) < keys ? fast_exp2(s[i >> 2][i & 3] * a.scale_log2 - lse) : 0.0f;
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[i] += fast_exp2(s[i >> 2][i & 3] * a.scale_log2 - lse);
    }
    if (!more) break;
#pragma unroll
    for (int c = 0; c < kC; ++c) qf[c] = qn[c];
    lse = lse_n;
  }
  // across the 16 lanes of a row: lane `col` ends with sum `col`
#pragma unroll
  for (int half = 8; half > 0; half /= 2) {
    const bool up = (col & half) != 0;
#pragma unroll
    for (int i = 0; i < half; ++i) {
      const float send = up ? acc[i] : acc[i + half], keep = up ? acc[i + half] : acc[i];
      acc[i] = keep + xor_shfl(send, half);
    }
  }
  if (mine) *sum = old + acc[0];
}

template <int D, bool kKv4>
hipError_t launch_mass(const MassArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL((attn_mass_kernel<D, kKv4>), dim3((unsigned)a.num_items * a.num_kv_heads), dim3(kMassWaves * 64), 0,
                     stream, a);
  return hipGetLastError();
}

}  // namespace kern

hipError_t launch_attn_mass(const MassArgs& a, int head_dim, bool kv4, hipStream_t stream) {
  if (head_dim == 128) return kv4 ? kern::launch_mass<128, true>(a, stream) : kern::launch_mass<128, false>(a, stream);
  if (head_dim == 64) return kv4 ? kern::launch_mass<64, true>(a, stream) : kern::launch_mass<64, false>(a, stream);
  return hipErrorInvalidValue;
}

}  // namespace tide
