// Attention of rows over the blocks that a list names for each (row, kv head).
//
// A row is one query token at position t of its task; its list holds logical blocks (pages of 16
// positions).  For the G query heads of the kv head, as in decode,
//     o = sum_p softmax(s)_p v_p,  s_p = sm_scale <q, k_p>,  p <= t in the listed blocks,
// so a row costs its list and not its context, and neither the length nor the position has to be known
// to the host.
//
// One workgroup takes a (row, kv head), or a part of its list where there are few (splits): wave w of 4
// takes the pairs of entries w, w + 4, ...: 32 keys a step, the G heads as MFMA columns.  Its lanes hold
// the page ids of 64 entries at a time and entries that name nothing (negative, beyond the row's
// position, a page id out of range) are left out of them, so a step always has a page to read.  The step
// is that of the decode kernels (K through LDS, V transposed in LDS; attn_decode.h), with the next step
// in flight while one is used.  The waves' parts are joined in LDS, in wave order.
//
// A decode batch reads its lists' pages once and is bound by HBM: 256 rows of 128 blocks (32 / 8 heads, d = 128), 2.1 GB
// in 320 us, 6.6 TB/s.  Few rows are bound by the chain list entry, page id, K and V, join: 4 rows of 64 blocks
// (28 / 4 heads) 11 us.
#include <algorithm>

#include "attn_decode.h"

namespace tide {
namespace kern {

// Running maximum of no keys: finite, so that differences of two of them are numbers, and below every
// score but -inf.
constexpr float kNoKeys = -3.0e38f;

// Waves of a workgroup.  (8 for calls that leave CUs idle: 4 rows of 64 blocks 10.7 us instead of 11.1, 16 rows of 256
// 30.6 instead of 29.7.)
constexpr int kWaves = 4;

template <int D, int kPolicy>
__global__ __launch_bounds__(kWaves * 64) __attribute__((amdgpu_waves_per_eu(2, 2)))
void sparse_attn_kernel(SparseArgs a) {
  using KL = KLds<D>;
  using VL = VLds<D>;
  constexpr int kC = D / 32, kT = D / 16;
  const int lane = threadIdx.x & 63, col = lane & 15, grp = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int Hkv = a.num_kv_heads, G = a.group;
  const int unit = blockIdx.x / a.splits, split = blockIdx.x - unit * a.splits;
  const int nth = unit / Hkv, head = unit - nth * Hkv;
  const int64_t row = (int64_t)a.first_row + nth;
  const int task = ((const const_i32*)a.row_task)[row], pos = ((const const_i32*)a.row_pos)[row];
  if (!live_row(task, pos, a.num_tasks, (int64_t)a.bt_stride * kPage)) return;
  // K pages of the two steps in flight; at the end outputs in k_lds0, statistics in k_lds1
  __shared__ __attribute__((aligned(1024))) uint8_t k_lds0[kWaves * 2 * KL::kPageBytes];
  __shared__ __attribute__((aligned(1024))) uint8_t k_lds1[kWaves * 2 * KL::kPageBytes];
  uint8_t* const ka = k_lds0 + wave * 2 * KL::kPageBytes;
  uint8_t* const kb = k_lds1 + wave * 2 * KL::kPageBytes;
  const bool col_ok = col < G;
  const uint8_t* kpool = reinterpret_cast<const uint8_t*>(a.k_pool);
  const uint8_t* vpool = reinterpret_cast<const uint8_t*>(a.v_pool);
  constexpr int64_t kBlk = (int64_t)kPage * D * 2;

  uint32_t k_src[KL::kDma];
#pragma unroll
  for (int i = 0; i < KL::kDma; ++i) k_src[i] = KL::src_offset(i, lane);
  const uint32_t k_rd_even = KL::lds_offset(col, grp), k_rd_odd = KL::lds_offset(col, 4 + grp);
  const uint32_t v_off = (uint32_t)(16 * lane);
  constexpr int kRpl = 1024 / (2 * D);
  uint32_t v_wr[DecodeRegs<D>::kLoads];
#pragma unroll
  for (int i = 0; i < DecodeRegs<D>::kLoads; ++i)
    v_wr[i] = VL::offset(i * kRpl + lane / VL::kNG, lane % VL::kNG);
  const int vr = 4 * grp + (col >> 2);
  uint32_t v_rd[kT];
#pragma unroll
  for (int t = 0; t < kT; ++t) v_rd[t] = (uint32_t)(vr * 2 * D + 32 * (t ^ VL::vsw(vr)) + 8 * (col & 3));

  const int32_t* list = a.sel + (row * Hkv + head) * a.budget;
  const int32_t* table = a.block_table + (int64_t)task * a.bt_stride;
  // this workgroup's pairs of entries, and this wave's
  const int pairs = (a.budget + 1) / 2, per = (pairs + a.splits - 1) / a.splits;
  const int end = min(pairs, (split + 1) * per);
  int next_pair = split * per + wave;  // of the batch that is fetched next

  // A batch: lane l holds entry l % 2 of pair next_pair + kWaves (l / 2).  open: the entries that name
  // something, not yet used.
  bool flag_error = false;
  int32_t page = 0, keys = 0;  // keys: of the block, up to the row's position
  uint64_t open = 0;
  auto fetch = [&]() {
    while (open == 0 && next_pair < end) {
      const int pair = next_pair + kWaves * (lane >> 1), at = 2 * pair + (lane & 1);
      next_pair += 32 * kWaves;
      const int32_t b = pair < end && at < a.budget ? list[at] : -1;
      const bool in = b >= 0 && b <= pos / kPage;
      page = in ? table[b] : -1;
      const bool ok = in && page >= 0 && page < a.num_pages;
      flag_error |= in && !ok;
      keys = in ? min(kPage, pos + 1 - b * kPage) : 0;
      open = __builtin_amdgcn_ballot_w64(ok);
    }
  };
  // The next step: up to two entries.
  struct Step {
    int n0, n1;  // keys of each; 0, 0: no step
  };
  auto issue = [&](DecodeRegs<D>& r, uint8_t* kbuf) {
    fetch();
    int64_t b0 = 0, b1 = 0;
    Step s = {0, 0};
    if (open) {
      const int i = __builtin_ctzll(open);
      open &= open - 1;
      s.n0 = __builtin_amdgcn_readlane(keys, i);
      b0 = ((int64_t)__builtin_amdgcn_readlane(page, i) * Hkv + head) * kBlk;
    }
    if (open) {
      const int i = __builtin_ctzll(open);
      open &= open - 1;
      s.n1 = __builtin_amdgcn_readlane(keys, i);
      b1 = ((int64_t)__builtin_amdgcn_readlane(page, i) * Hkv + head) * kBlk;
    }
    const int z0 = s.n0 ? (int)kBlk : 0, z1 = s.n1 ? (int)kBlk : 0;
    load_step<D, kPolicy>(r, kbuf, block_rsrc(kpool + b0, z0), block_rsrc(kpool + b1, z1), block_rsrc(vpool + b0, z0),
                          block_rsrc(vpool + b1, z1), k_src, v_off);
    return s;
  };

  f32x4 o[kT];
#pragma unroll
  for (int t = 0; t < kT; ++t) o[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  float m_ref = kNoKeys, l_part = 0.0f, l_exact = 0.0f;
  bf16x8 qf[kC];
  {
    const int64_t at = (row * a.num_q_heads + head * G + (col_ok ? col : 0)) * D;
#pragma unroll
    for (int c = 0; c < kC; ++c) {
      const u32x4 x = load_u32x4(a.q + at + 32 * c + 8 * grp);
      qf[c] = as_bf16x8(col_ok ? x : zero_u32x4());
    }
  }

  auto compute = [&](DecodeRegs<D>& cur, const uint8_t* kbuf, Step st) {
    u32x4 kk[2][kC];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int c = 0; c < kC; ++c)
        kk[t][c] = *reinterpret_cast<const u32x4*>(kbuf + t * KL::kPageBytes + 1024 * (c >> 1) +
                                                   ((c & 1) ? k_rd_odd : k_rd_even));
    if (st.n0 + st.n1 < 2 * kPage) {
      // V rows past the position must not reach the MFMA (NaN * 0 = NaN)
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < DecodeRegs<D>::kLoads; ++i)
          if (i * kRpl + lane / VL::kNG >= (t ? st.n1 : st.n0)) cur.v[t][i] = zero_u32x4();
    }
    f32x4 s[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      s[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int c = 0; c < kC; ++c) s[t] = mfma16(as_bf16x8(kk[t][c]), qf[c], s[t]);
    }
    if (st.n0 + st.n1 < 2 * kPage) {  // keys past the position
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s[0][e] = 4 * grp + e < st.n0 ? s[0][e] : -INFINITY;
        s[1][e] = 4 * grp + e < st.n1 ? s[1][e] : -INFINITY;
      }
    }
    float mt = a.scale_log2 * fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])),
                                    fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
    if (__any(mt > m_ref + kRescaleSlack)) {  // only then is the column's maximum worked out
      mt = fmaxf(mt, xor_shfl(mt, 16));
      mt = fmaxf(mt, xor_shfl(mt, 32));
      const float m_new = fmaxf(m_ref, mt);
      const float alpha = fast_exp2(m_ref - m_new);
      l_part *= alpha;
      l_exact *= alpha;
#pragma unroll
      for (int t = 0; t < kT; ++t) o[t] *= alpha;
      m_ref = m_new;
    }
    u32x4 wp;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float p0 = fast_exp2(fmaf(s[t][2 * e], a.scale_log2, -m_ref));
        const float p1 = fast_exp2(fmaf(s[t][2 * e + 1], a.scale_log2, -m_ref));
        // Weights go to the P V product in bf16, as in decode and extend: operands of more bits run at a fraction of
        // its rate, or as two products.  Each is off by at most half a step, 2^-8 of it; the sum that divides them is
        // of the rounded ones, so that they add to one, and an output is off by at most 2 * 2^-8 sum w |v| beside its
        // own rounding (off from 64 bits by 0.0023 of the outputs' norm; weights of 32 bits leave 0.0017).  Sums have 32 bits,
        // and the one that lse takes is of the weights before they are rounded.
        wp[2 * t + e] = pack_bf16x2(p0, p1);
        l_part = add_bf16x2(wp[2 * t + e], l_part);
        l_exact += p0 + p1;
      }
    const bf16x8 pb = as_bf16x8(wp);
    uint8_t* vbuf = const_cast<uint8_t*>(kbuf);  // V over the K copy, which is done with
#pragma unroll
    for (int hp = 0; hp < 2; ++hp)
#pragma unroll
      for (int i = 0; i < DecodeRegs<D>::kLoads; ++i)
        *reinterpret_cast<u32x4*>(vbuf + hp * KL::kPageBytes + v_wr[i]) = cur.v[hp][i];
    u32x4 vv[kT];
#pragma unroll
    for (int t = 0; t < kT; ++t) {
      const uint2 v0 = read_tr(vbuf + v_rd[t]), v1 = read_tr(vbuf + KL::kPageBytes + v_rd[t]);
      vv[t] = u32x4{v0.x, v0.y, v1.x, v1.y};
    }
#pragma unroll
    for (int t = 0; t < kT; ++t) o[t] = mfma16(as_bf16x8(vv[t]), pb, o[t]);
  };

  bool any = false;
  {
    DecodeRegs<D> ra, rb;
    Step sa = issue(ra, ka), sb;
    while (sa.n0) {
      any = true;
      sb = issue(rb, kb);
      __builtin_amdgcn_sched_barrier(0);
      compute(ra, ka, sa);
      if (!sb.n0) break;
      sa = issue(ra, ka);
      __builtin_amdgcn_sched_barrier(0);
      compute(rb, kb, sb);
    }
  }
  if (flag_error) atomicOr(a.error_flags, 1);

  // ---- the waves' parts ----
  // every load into LDS, the zero-length ones too, is done before LDS takes the parts
  __atomic_signal_fence(__ATOMIC_SEQ_CST);
  __builtin_amdgcn_s_waitcnt(0);
  __atomic_signal_fence(__ATOMIC_SEQ_CST);
  auto sum_cols = [&](float v) {
    v += xor_shfl(v, 16);
    return v + xor_shfl(v, 32);
  };
  const float l = sum_cols(l_part), lx = sum_cols(l_exact);
  if (col_ok) {
#pragma unroll
    for (int t = 0; t < kT; ++t)
      *reinterpret_cast<f32x4*>(ka + 4 * D * col + 16 * ((4 * t + grp) ^ col)) = o[t];
    if (grp == 0) *reinterpret_cast<f32x4*>(kb + 16 * col) = f32x4{m_ref, l, lx, any ? 1.0f : 0.0f};
  }
  __syncthreads();
  constexpr int kPiece = D / 4;  // 16-byte pieces of a head's output
  for (int i = threadIdx.x; i < G * kPiece; i += kWaves * 64) {
    const int j = i / kPiece, p = i % kPiece;
    f32x4 st[kWaves];
    float m = kNoKeys;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      st[w] = *reinterpret_cast<const f32x4*>(k_lds1 + w * 2 * KL::kPageBytes + 16 * j);
      m = fmaxf(m, st[w][0]);
    }
    f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
    float ls = 0.0f, lxs = 0.0f, has = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float f = fast_exp2(st[w][0] - m);
      acc += f * *reinterpret_cast<const f32x4*>(k_lds0 + w * 2 * KL::kPageBytes + 4 * D * j + 16 * (p ^ j));
      ls += f * st[w][1];
      lxs += f * st[w][2];
      has = fmaxf(has, st[w][3]);
    }
    if (a.splits > 1) {
      const int64_t at = ((int64_t)blockIdx.x) * G + j;
      *reinterpret_cast<f32x4*>(a.part_o + at * D + 4 * p) = acc;
      if (p == 0) *reinterpret_cast<f32x4*>(a.part_ml + at * 4) = f32x4{m, ls, lxs, has};
      continue;
    }
    // a row whose list names nothing: zeros, and no weight at all
    const float inv = has > 0.0f ? 1.0f / ls : 0.0f;
    const int64_t h = row * a.num_q_heads + head * G + j;
    const uint2 x = {pack_bf16x2(acc[0] * inv, acc[1] * inv), pack_bf16x2(acc[2] * inv, acc[3] * inv)};
    *reinterpret_cast<uint2*>(a.out + h * D + 4 * p) = x;
    if (a.lse && p == 0) a.lse[h] = has > 0.0f ? (m + __log2f(lxs)) * kLn2 : -INFINITY;
  }
}

// Joins the parts of split rows, in order: D / 4 lanes a (row, query head).
template <int D>
__global__ __launch_bounds__(256) void sparse_merge_kernel(SparseArgs a) {
  constexpr int kPiece = D / 4;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int p = (int)(i % kPiece);
  const int64_t hq = i / kPiece;
  const int64_t nth = hq / a.num_q_heads;
  if (nth >= a.rows) return;
  const int h = (int)(hq - nth * a.num_q_heads), head = h / a.group, j = h - head * a.group;
  const int64_t row = a.first_row + nth;
  if (!live_row(a.row_task[row], a.row_pos[row], a.num_tasks, (int64_t)a.bt_stride * kPage)) return;
  const int64_t first = (nth * a.num_kv_heads + head) * a.splits * a.group + j;
  f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
  float m = kNoKeys, l = 0.0f, lx = 0.0f, has = 0.0f;
  for (int s = 0; s < a.splits; ++s) {
    const f32x4 st = *reinterpret_cast<const f32x4*>(a.part_ml + (first + (int64_t)s * a.group) * 4);
    const f32x4 x = *reinterpret_cast<const f32x4*>(a.part_o + (first + (int64_t)s * a.group) * D + 4 * p);
    const float to = fmaxf(m, st[0]), f0 = fast_exp2(m - to), f1 = fast_exp2(st[0] - to);
    m = to;
    acc = f0 * acc + f1 * x;
    l = f0 * l + f1 * st[1];
    lx = f0 * lx + f1 * st[2];
    has = fmaxf(has, st[3]);
  }
  const float inv = has > 0.0f ? 1.0f / l : 0.0f;
  const int64_t at = row * a.num_q_heads + h;
  const uint2 x = {pack_bf16x2(acc[0] * inv, acc[1] * inv), pack_bf16x2(acc[2] * inv, acc[3] * inv)};
  *reinterpret_cast<uint2*>(a.out + at * D + 4 * p) = x;
  if (a.lse && p == 0) a.lse[at] = has > 0.0f ? (m + __log2f(lx)) * kLn2 : -INFINITY;
}

template <int D, int kPolicy>
void launch_lists(const SparseArgs& a, hipStream_t stream) {
  const uint32_t groups = (uint32_t)a.rows * (uint32_t)a.num_kv_heads * (uint32_t)a.splits;
  hipLaunchKernelGGL((sparse_attn_kernel<D, kPolicy>), dim3(groups), dim3(kWaves * 64), 0, stream, a);
}

template <int D>
hipError_t launch_sparse_d(const SparseArgs& a, bool shared, hipStream_t stream) {
  if (shared) launch_lists<D, kSharedPolicy>(a, stream);
  else launch_lists<D, kStreamPolicy>(a, stream);
  const hipError_t rc = hipGetLastError();
  if (rc != hipSuccess || a.splits == 1) return rc;
  const int64_t threads = (int64_t)a.rows * a.num_q_heads * (D / 4);
  hipLaunchKernelGGL((sparse_merge_kernel<D>), dim3((uint32_t)((threads + 255) / 256)), dim3(256), 0, stream, a);
  return hipGetLastError();
}

// Every variant is instantiated explicitly (see attn_decode.hip).
template __global__ void sparse_attn_kernel<128, kSharedPolicy>(SparseArgs);
template __global__ void sparse_attn_kernel<128, kStreamPolicy>(SparseArgs);
template __global__ void sparse_attn_kernel<64, kSharedPolicy>(SparseArgs);
template __global__ void sparse_attn_kernel<64, kStreamPolicy>(SparseArgs);

}  // namespace kern

hipError_t launch_sparse(const SparseArgs& a, int head_dim, bool shared, hipStream_t stream) {
  return head_dim == 128 ? kern::launch_sparse_d<128>(a, shared, stream) : kern::launch_sparse_d<64>(a, shared, stream);
}

}  // namespace tide
