// Attention of a few query tokens a task over the 4-bit cache: decode, and the extends that read the
// codes themselves (kKv4DirectUnits in plan.cpp).
//
// A unit is 1 .. 32 / G consecutive query tokens of a task (one, of decode); their (token, query head)
// rows of one kv head are the columns of one or two 16x16x32 MFMAs, a step is 32 keys (2 pages).  As in
// attn_decode_stream.hip the units' steps are laid end to end and cut into equal runs, one wave
// takes a run of one kv head, and cut units are put together at the end (decode_runs.h).
//
// The step never touches LDS: codes arrive in the lanes that feed them to the MFMAs (kv4.h).  With
// S^T = K Q^T a lane's A operand is its slot's codes, 8 entries a word, converted with their one
// scale; the lane then holds the probabilities of keys 4 (l/16) + e of both pages as the B operand
// of O^T += V^T P^T, whose A operand is converted from the codes of those very keys, 2 entries
// of one key at a time, and paired key by key with byte permutations.  Both products take bf16
// operands, which hold code times scale exactly; sums, scores and softmax statistics are fp32,
// and probabilities are rounded to bf16 for the second product as in the bf16 decode (its row sums
// add the rounded ones, the log-sum-exp the exact ones).  The MFMA that takes 4-bit operands was not
// used for S^T: it adds products in groups with about 16 bits, 2^-14.7 of their sum of magnitudes
// off, and the conversions are not what bounds the call.
//
// Bound by reading: 256 tasks of 1k-16k keys (32 / 8 heads, d = 128) take 384 us for 2.3 GB, 6.0
// TB/s, against 367 us for the same loads with nothing done to them.  Two steps are in flight a
// wave, at 2 waves a SIMD: three to five steps take the same time, 3 waves a SIMD 3-12% more, 4 spill.
// A fifth fewer vector instructions changed nothing.  Short contexts add the merge of cut units to that:
// 32 tasks with 2-8 tokens each 86 us, of which 19 after the last step (flags and partials through
// memory; merged by whole workgroups 122 us).  Its other 67 us, of 41 to read the codes, have no one
// bound: over the whole kernel 1.3 of 2 waves a SIMD live, a third of their time waits for memory,
// vector instructions issue in 36% of the SIMDs' cycles and MFMAs run in 15%.
#include "attn_decode.h"
#include "decode_runs.h"
#include "kv4.h"

namespace tide {
namespace kern {

constexpr int kKv4Big = 8, kKv4Small = 4;  // waves per workgroup (kv4_waves)

typedef const __attribute__((address_space(4))) Kv4Run const_run;

// One step's codes and scales: [page][word], and a page's scale byte of K and 4 of V.
template <int D>
struct Kv4Regs {
  uint32_t k[2][Kv4<D>::kWords], v[2][Kv4<D>::kWords], ks[2], vs[2];
};

template <int D, int kPolicy>
__device__ __forceinline__ void kv4_load_page(Kv4Regs<D>& r, int t, __amdgpu_buffer_rsrc_t blk, int lane) {
  using F = Kv4<D>;
  if constexpr (D == 128) {
    const u32x4 k = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(blk, lane * 16, 0, kPolicy));
    const u32x4 v = __builtin_bit_cast(
        u32x4, __builtin_amdgcn_raw_buffer_load_b128(blk, F::kVCodes + lane * 16, 0, kPolicy));
#pragma unroll
    for (int w = 0; w < 4; ++w) r.k[t][w] = k[w], r.v[t][w] = v[w];
  } else {
    const uint2 k = __builtin_bit_cast(uint2, __builtin_amdgcn_raw_buffer_load_b64(blk, lane * 8, 0, kPolicy));
    const uint2 v = __builtin_bit_cast(
        uint2, __builtin_amdgcn_raw_buffer_load_b64(blk, F::kVCodes + lane * 8, 0, kPolicy));
    r.k[t][0] = k.x, r.k[t][1] = k.y, r.v[t][0] = v.x, r.v[t][1] = v.y;
  }
  r.ks[t] = __builtin_amdgcn_raw_buffer_load_b8(blk, F::k_scale(lane), 0, kPolicy);
  r.vs[t] = __builtin_amdgcn_raw_buffer_load_b32(blk, F::v_scale(lane), 0, kPolicy);
}

__device__ __forceinline__ uint32_t lo_halves(uint32_t a, uint32_t b) {
  return __builtin_amdgcn_perm(b, a, 0x05040100u);
}
__device__ __forceinline__ uint32_t hi_halves(uint32_t a, uint32_t b) {
  return __builtin_amdgcn_perm(b, a, 0x07060302u);
}

// The entry pair 2 s, 2 s + 1 of key i of a lane's V codes.
template <int D, int kS>
__device__ __forceinline__ uint32_t v_pair(const uint32_t (&v)[Kv4<D>::kWords], int i, float f) {
  if constexpr (D == 128) return kv4_pair<kS>(v[i], f);
  else return i & 1 ? kv4_pair<2 + (kS & 1)>(v[i >> 1], f) : kv4_pair<(kS & 1)>(v[i >> 1], f);
}

template <int D, bool kAppend, int kWaves, int kSets, int kPolicy>
__global__ __launch_bounds__(kWaves * 64) __attribute__((amdgpu_waves_per_eu(2, 2)))
void kv4_decode_kernel(Kv4AttnArgs a) {
  using F = Kv4<D>;
  constexpr int kC = D / 32;      // MFMAs of S^T a page, words of a lane's K codes
  constexpr int kJ = F::kSpan;    // MFMAs of O^T, entries of a V slot in a lane
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int R = a.num_runs, rg = blockIdx.x / a.num_kv_heads;
  const int head = blockIdx.x - rg * a.num_kv_heads;
  const int run = rg * kWaves + wave;
  // the waves' partials at the end: outputs, statistics
  __shared__ __attribute__((aligned(16))) uint8_t lds_o[kWaves * kSets * 16 * 4 * D];
  __shared__ __attribute__((aligned(16))) uint8_t lds_s[kWaves * kSets * 16 * 16];
  __shared__ int open_unit[kWaves];  // the unit each wave leaves unfinished, or -1

  const bool live = run < R;
  const int n = !live ? 0 : run == R - 1 ? a.last_steps : a.steps;
  const StreamSlots slots = {R, a.num_units, kWaves};
  const int64_t slot0 = (int64_t)head * slots.count();
  const int G = a.group, Hkv = a.num_kv_heads;
  const int col = lane & 15, grp = lane >> 4;
  // column `col` of set x is row 16 x + col of the unit: token tok[x], query head row - tok G of the group
  int tok[kSets];
#pragma unroll
  for (int x = 0; x < kSets; ++x) tok[x] = (16 * x + col) / G;

  // Position in the sequence of the units' steps; all wave-uniform.
  struct Cursor {
    int unit, step, steps, prefix, tokens, row_start;
    const int32_t* table;
  };
  auto load_unit = [&](Cursor& c) {
    const const_i32* u = (const const_i32*)(a.units + c.unit);
    c.row_start = u[0];
    c.prefix = u[1];
    c.tokens = u[2];
    c.table = a.block_table + (int64_t)u[3] * a.bt_stride;
    c.steps = (c.prefix + c.tokens - 1) / kDecodeStep + 1;
  };
  const const_run* it = (const const_run*)(a.runs + (live ? run : 0));
  Cursor ld = {it->unit, it->step, 0, it->desc.prefix, it->desc.extend, it->desc.row_start,
               a.block_table + (int64_t)it->desc.aux * a.bt_stride};
  ld.steps = (ld.prefix + ld.tokens - 1) / kDecodeStep + 1;
  Cursor cu = ld;

  // Loads of the load cursor's step, through zero-length buffers (zeros, no memory access) past
  // the run's end, past a context and for invalid page ids.  Page ids are scalar loads, fetched one
  // step ahead.
  bool flag_error = false;
  int left = n;
  int32_t pg[2];
  auto fetch_pages = [&]() {
    const const_i32* row = (const const_i32*)ld.table;
    const int last = (ld.prefix + ld.tokens - 1) / kPage;
    pg[0] = row[left > 0 ? 2 * ld.step : 0];
    pg[1] = row[left > 0 ? min(2 * ld.step + 1, last) : 0];
  };
  // the newest token's rows (kAppend), loaded with the step that holds its slot: V in lanes 0 ..
  // 15 (entries D/16 lane ..), K in lanes 16 .. 31
  struct NewRow {
    uint32_t x[kJ / 2];
    int page;  // its pool page, or -1
  };
  auto issue = [&](Kv4Regs<D>& r, NewRow& nw) {
    const bool in = left > 0;
    const bool second = in && (2 * ld.step + 1) * kPage < ld.prefix + ld.tokens;
    const bool ok0 = in && pg[0] >= 0 && pg[0] < a.num_pages;
    const bool ok1 = second && pg[1] >= 0 && pg[1] < a.num_pages;
    flag_error |= (in && !ok0) || (second && !ok1);
    const int64_t b0 = ((int64_t)(ok0 ? pg[0] : 0) * Hkv + head) * F::kBlock;
    const int64_t b1 = ((int64_t)(ok1 ? pg[1] : 0) * Hkv + head) * F::kBlock;
    kv4_load_page<D, kPolicy>(r, 0, block_rsrc(a.pool + b0, ok0 ? F::kBlock : 0), lane);
    kv4_load_page<D, kPolicy>(r, 1, block_rsrc(a.pool + b1, ok1 ? F::kBlock : 0), lane);
    if constexpr (kAppend) {
      nw.page = -1;
      if (in && ld.step == ld.steps - 1) {
        const bool hi = (ld.prefix & (kDecodeStep - 1)) >= kPage;
        if (hi ? ok1 : ok0) {
          nw.page = hi ? pg[1] : pg[0];
          const int64_t row = ((int64_t)ld.row_start * Hkv + head) * D + kJ * col;
          const uint16_t* from = (lane < 16 ? a.v_new : a.k_new) + row;
#pragma unroll
          for (int w = 0; w < kJ / 2; ++w) nw.x[w] = reinterpret_cast<const uint32_t*>(from)[w];
        }
      }
    }
    if (in) {
      --left;
      if (++ld.step == ld.steps) {
        ld.step = 0;
        ++ld.unit;
        if (left > 0) load_unit(ld);
      }
    }
    fetch_pages();
  };

  bf16x8 qf[kSets][kC];
  auto row_ok = [&](int x) { return 16 * x + col < cu.tokens * G; };
  auto out_row = [&](int x) {
    return ((int64_t)cu.row_start + tok[x]) * a.num_q_heads + head * G + (16 * x + col - tok[x] * G);
  };
  auto load_q = [&]() {
#pragma unroll
    for (int x = 0; x < kSets; ++x) {
      const uint16_t* from = a.q + out_row(x) * D + (D / 4) * grp;
#pragma unroll
      for (int c = 0; c < kC; ++c) qf[x][c] = as_bf16x8(row_ok(x) ? load_u32x4(from + 8 * c) : zero_u32x4());
    }
  };
  // The accumulators of a new unit are cleared where its first step raises the reference: set to zero
  // at the last one's end they would be copied on every step, where that path joins the others.
  f32x4 o[kSets][kJ];
#pragma unroll
  for (int x = 0; x < kSets; ++x)
#pragma unroll
    for (int j = 0; j < kJ; ++j) o[x][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  float m_ref[kSets], l_part[kSets], l_exact[kSets];
  bool fresh;
  auto reset = [&]() {
    fresh = true;
#pragma unroll
    for (int x = 0; x < kSets; ++x) {
      m_ref[x] = kNoMax;
      l_part[x] = l_exact[x] = 0.0f;
    }
  };

  // The newest token takes the place of its slot in the operands (whatever the pool holds there)
  // and goes to the pool; nothing in this call reads the slot afterwards.
  auto put_new = [&](Kv4Regs<D>& cur, const NewRow& nw) {
    const int pos = cu.prefix, slot = pos & (kPage - 1), half = (pos / kPage) & 1;
    uint32_t m = 0;
#pragma unroll
    for (int w = 0; w < kJ / 2; ++w) m = kv4_max(m, nw.x[w]);
#pragma unroll
    for (int s = 1; s < F::kVLanes; s *= 2) m = max(m, (uint32_t)__shfl_xor((int)m, s, 64));
    const uint32_t byte = kv4_scale_byte(m);
    u32x4 p = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int w = 0; w < kJ / 2; ++w) p[w] = nw.x[w];
    const uint32_t codes = kv4_codes(p, kv4_factor(byte));  // D = 64: the lower half
    // K: lane (slot, grp) needs its D / 4 entries from lanes 16 + 4 grp .. + 3
    uint32_t kc[kC];
#pragma unroll
    for (int w = 0; w < kC; ++w) {
      if constexpr (D == 128) {
        kc[w] = (uint32_t)__shfl((int)codes, 16 + 4 * grp + w, 64);
      } else {
        const uint32_t c0 = (uint32_t)__shfl((int)codes, 16 + 4 * grp + 2 * w, 64);
        const uint32_t c1 = (uint32_t)__shfl((int)codes, 16 + 4 * grp + 2 * w + 1, 64);
        kc[w] = (c0 & 0xFFFFu) | (c1 << 16);
      }
    }
    const uint32_t kb = (uint32_t)__shfl((int)byte, 16 + 4 * grp, 64);
    const uint32_t vc = (uint32_t)__shfl((int)codes, col, 64), vb = (uint32_t)__shfl((int)byte, col, 64);
    uint8_t* blk = a.pool + ((int64_t)nw.page * Hkv + head) * F::kBlock;
    const bool k_lane = col == slot, v_lane = grp == slot >> 2;
    const int i = slot & 3;
    auto take = [](uint32_t& x, uint32_t value, uint32_t mask) { x = (x & ~mask) | (value & mask); };
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const uint32_t in_k = t == half && k_lane ? ~0u : 0u, in_v = t == half && v_lane ? ~0u : 0u;
#pragma unroll
      for (int w = 0; w < kC; ++w) take(cur.k[t][w], kc[w], in_k);
      take(cur.ks[t], kb, in_k);
      take(cur.vs[t], vb << (8 * i), in_v & (255u << (8 * i)));
#pragma unroll
      for (int w = 0; w < F::kWords; ++w) {
        if constexpr (D == 128) take(cur.v[t][w], vc, w == i ? in_v : 0u);
        else take(cur.v[t][w], vc << (16 * (i & 1)), w == i >> 1 ? in_v & (0xFFFFu << (16 * (i & 1))) : 0u);
      }
    }
    if (k_lane) {
      uint32_t* to = reinterpret_cast<uint32_t*>(blk + lane * F::kLane);
#pragma unroll
      for (int w = 0; w < kC; ++w) to[w] = kc[w];
      if (D == 128 || (grp & 1) == 0) blk[F::k_scale(lane)] = (uint8_t)kb;
    }
    if (v_lane) {
      if constexpr (D == 128) *reinterpret_cast<uint32_t*>(blk + F::v_word(col, slot)) = vc;
      else *reinterpret_cast<uint16_t*>(blk + F::v_word(col, slot)) = (uint16_t)vc;
      if (col % F::kVLanes == 0) blk[F::v_scale(lane) + i] = (uint8_t)vb;
    }
  };

  auto compute = [&](Kv4Regs<D>& cur, NewRow& nw) {
    const int k = cu.step * kDecodeStep;
    const int kv_len = cu.prefix + cu.tokens;
    if (cu.step == cu.steps - 1) {  // the only one with slots past the context or the newest token's
      if constexpr (kAppend) {
        if (nw.page >= 0) put_new(cur, nw);
      }
      // V past the context must not reach the MFMA (NaN * 0 = NaN)
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (k + 16 * t + 4 * grp + i < kv_len) continue;
          cur.vs[t] = (cur.vs[t] & ~(255u << (8 * i))) | (127u << (8 * i));
          if constexpr (D == 128) cur.v[t][i] = 0;
          else cur.v[t][i >> 1] &= i & 1 ? 0x0000FFFFu : 0xFFFF0000u;
        }
    }
    f32x4 s[kSets][2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const float f = kv4_factor(cur.ks[t]);
#pragma unroll
      for (int c = 0; c < kC; ++c) {
        const bf16x8 kk = kv4_octet(cur.k[t][c], f);
#pragma unroll
        for (int x = 0; x < kSets; ++x)
          s[x][t] = mfma16(kk, qf[x][c], c == 0 ? f32x4{0.0f, 0.0f, 0.0f, 0.0f} : s[x][t]);
      }
    }
    if (k > cu.prefix + 1 - kDecodeStep) {  // keys that some token of the unit does not see
#pragma unroll
      for (int x = 0; x < kSets; ++x) {
        const int keys = cu.prefix + 1 + tok[x] - k - 4 * grp;  // of this lane's, counted from its first
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[x][t][e] = 16 * t + e < keys ? s[x][t][e] : -INFINITY;
      }
    }
    float mt[kSets];
    bool raise = false;
#pragma unroll
    for (int x = 0; x < kSets; ++x) {
      float m = -INFINITY;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) m = fmaxf(m, s[x][t][e]);
      m = fmaxf(m, xor_shfl(m, 16));
      mt[x] = fmaxf(m, xor_shfl(m, 32)) * a.scale_log2;
      raise |= mt[x] > m_ref[x] + kRescaleSlack;
    }
    if (fresh || __any(raise)) {
#pragma unroll
      for (int x = 0; x < kSets; ++x) {
        const float m_new = fmaxf(m_ref[x], mt[x]);
        const float alpha = fast_exp2(m_ref[x] - m_new);
        l_part[x] *= alpha;
        l_exact[x] *= alpha;
#pragma unroll
        for (int j = 0; j < kJ; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[x][j][i] = fresh ? 0.0f : o[x][j][i] * alpha;
        m_ref[x] = m_new;
      }
      fresh = false;
    }
    bf16x8 pb[kSets];
#pragma unroll
    for (int x = 0; x < kSets; ++x) {
      u32x4 wp;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float p0 = fast_exp2(s[x][t][2 * e] * a.scale_log2 - m_ref[x]);
          const float p1 = fast_exp2(s[x][t][2 * e + 1] * a.scale_log2 - m_ref[x]);
          wp[2 * t + e] = pack_bf16x2(p0, p1);
          l_part[x] = add_bf16x2(wp[2 * t + e], l_part[x]);
          if (a.lse) l_exact[x] += p0 + p1;
        }
      pb[x] = as_bf16x8(wp);
    }
    float vf[2][4];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) vf[t][i] = kv4_factor((cur.vs[t] >> (8 * i)) & 255u);
    auto product = [&](auto tag) {
      constexpr int kS = decltype(tag)::value;
      if constexpr (kS < kJ / 2) {
        uint32_t y[2][4];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) y[t][i] = v_pair<D, kS>(cur.v[t], i, vf[t][i]);
        const u32x4 even = {lo_halves(y[0][0], y[0][1]), lo_halves(y[0][2], y[0][3]),
                            lo_halves(y[1][0], y[1][1]), lo_halves(y[1][2], y[1][3])};
        const u32x4 odd = {hi_halves(y[0][0], y[0][1]), hi_halves(y[0][2], y[0][3]),
                           hi_halves(y[1][0], y[1][1]), hi_halves(y[1][2], y[1][3])};
#pragma unroll
        for (int x = 0; x < kSets; ++x) {
          o[x][2 * kS] = mfma16(as_bf16x8(even), pb[x], o[x][2 * kS]);
          o[x][2 * kS + 1] = mfma16(as_bf16x8(odd), pb[x], o[x][2 * kS + 1]);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    product(std::integral_constant<int, 0>());
    product(std::integral_constant<int, 1>());
    product(std::integral_constant<int, 2>());
    product(std::integral_constant<int, 3>());
  };

  auto sum_cols = [&](float v) {
    v += xor_shfl(v, 16);
    return v + xor_shfl(v, 32);
  };
  // Lane (col, grp) holds entries (D/4) grp + kJ i + j of its row of set x as o[x][j][i]; four at a
  // time: quad y is entries (D/4) grp + 4 y.
  auto quad = [&](int x, int y) {
    const int i = 4 * y / kJ, j = 4 * y % kJ;
    return f32x4{o[x][j][i], o[x][j + 1][i], o[x][j + 2][i], o[x][j + 3][i]};
  };
  constexpr int kQuads = D / 16;

  int begin = cu.step;  // steps of the current unit before this wave
  bool has_final = false, has_flush = false;
  StreamUnit flush = {0, 0, false};
  int flush_unit = 0, flush_row = 0, flush_tokens = 0, done = 0;
  // The unit whose last step was just computed.
  auto unit_end = [&]() {
    if (begin == 0) {  // all of it in this wave: its rows are final
#pragma unroll
      for (int x = 0; x < kSets; ++x) {
        const float inv = 1.0f / sum_cols(l_part[x]), lx = sum_cols(l_exact[x]);
        if (!row_ok(x)) continue;
        const int64_t row = out_row(x);
        uint16_t* to = a.out + row * D + (D / 4) * grp;
#pragma unroll
        for (int y = 0; y < kQuads; y += 2) {
          const f32x4 q0 = quad(x, y), q1 = quad(x, y + 1);
          store_u32x4(to + 4 * y, u32x4{pack_bf16x2(q0[0] * inv, q0[1] * inv), pack_bf16x2(q0[2] * inv, q0[3] * inv),
                                        pack_bf16x2(q1[0] * inv, q1[1] * inv), pack_bf16x2(q1[2] * inv, q1[3] * inv)});
        }
        if (a.lse && grp == 0) a.lse[row] = (m_ref[x] + __log2f(lx)) * kLn2;
      }
    } else if (cu.steps - begin == a.steps) {  // it took the whole run: like an unfinished one
      has_final = true;
      return;
    } else {
      has_flush = true;
      flush_unit = cu.unit, flush_row = cu.row_start, flush_tokens = cu.tokens;
      flush = stream_unit(run, begin, cu.steps - begin, cu.steps, a.steps);
      const int64_t slot = slot0 + slots.ended(run, cu.unit);
      float* po = a.part_o + slot * a.cols * D;
#pragma unroll
      for (int x = 0; x < kSets; ++x) {
        const float l = sum_cols(l_part[x]), lx = sum_cols(l_exact[x]);
        const int row = 16 * x + col;
        if (row >= a.cols) continue;
#pragma unroll
        for (int y = 0; y < kQuads; ++y)
          store_f32x4_device(po, a.cols * D * 4, 4 * (row * D + (D / 4) * grp + 4 * y), quad(x, y));
        if (grp == 0)
          store_f32x4_device(a.part_ml + slot * a.cols * 4, a.cols * 16, 16 * row, f32x4{m_ref[x], l, lx, 0.0f});
      }
    }
    begin = 0;
    reset();
  };
  auto process = [&](Kv4Regs<D>& r, NewRow& nw) {
    const bool last = cu.step == cu.steps - 1;
    compute(r, nw);
    ++done;
    ++cu.step;
    if (last) {
      unit_end();
      if (!has_final) {
        cu.step = 0;
        ++cu.unit;
        if (done < n) {
          load_unit(cu);
          load_q();
        }
      }
    }
  };

  reset();
  fetch_pages();
  if (n > 0) {
    Kv4Regs<D> r0, r1;
    NewRow n0, n1;
    load_q();
    // every load is issued on straight-line code (past the run's end, loads of nothing), so that a
    // step's wait leaves the next in flight.  The loop has one exit: with one behind each
    // step the accumulators got registers of their own per copy of the step (60 more a copy).
    auto trip = [&](Kv4Regs<D>& next, NewRow& next_new, Kv4Regs<D>& r, NewRow& nw) {
      issue(next, next_new);
      __builtin_amdgcn_sched_barrier(0);
      if (done < n) process(r, nw);
    };
    issue(r0, n0);
    do {
      trip(r1, n1, r0, n0);
      trip(r0, n0, r1, n1);
    } while (done < n);
    has_final |= cu.step > 0 && cu.step < cu.steps;
  }
  if (flag_error && lane == 0) atomicOr(a.error_flags, 1);

  // ---- parts of cut units (decode_runs.h) ---------------------------------------------------
  constexpr int kStrideO = kSets * 64 * D, kStrideS = kSets * 256;  // a wave's rows and statistics
  uint8_t* const my_o = lds_o + wave * kStrideO;
  uint8_t* const my_s = lds_s + wave * kStrideS;
  if (has_final) {
#pragma unroll
    for (int x = 0; x < kSets; ++x) {
      const float l = sum_cols(l_part[x]), lx = sum_cols(l_exact[x]);
      // row 16 x + col of the wave's partial: 16-byte granule g at g ^ col
#pragma unroll
      for (int y = 0; y < kQuads; ++y)
        *reinterpret_cast<f32x4*>(my_o + 4 * D * (16 * x + col) + 16 * (((D / 16) * grp + y) ^ col)) = quad(x, y);
      if (grp == 0) *reinterpret_cast<f32x4*>(my_s + 16 * (16 * x + col)) = f32x4{m_ref[x], l, lx, 0.0f};
    }
  }
  if (lane == 0) open_unit[wave] = has_final ? cu.unit : -1;
  __syncthreads();
  if (a.reads.done && threadIdx.x == 0) plan_read(a.reads, blockIdx.x);
  // (the units are not read here: a plan in a staging slot may be gone by now)
  struct Rows {
    int64_t first;  // output row of the kv head's first query head of the unit's first token
    int rows, group, heads;
    __device__ __forceinline__ int64_t operator()(int, int j) const {
      const int t = j / group;
      return j < rows ? first + (int64_t)t * heads + (j - t * group) : -1;
    }
  };
  auto parts_of = [&](int row_start, int tokens) {
    const Rows rows = {(int64_t)row_start * a.num_q_heads + head * G, tokens * G, G, a.num_q_heads};
    return RunParts<D, kWaves, Rows>{a.part_o, a.part_ml, a.flags, a.call, a.out, a.lse, slots, slot0, a.cols, rows};
  };
  if (has_flush)
    parts_of(flush_row, flush_tokens).arrive(flush, flush_unit, slot0 + slots.ended(run, flush_unit));
  if (!has_final) return;
  auto left_open = [&](int x) { return __builtin_amdgcn_readfirstlane(open_unit[x]); };
  if (wave > 0 && left_open(wave - 1) == cu.unit) return;  // the first of these waves goes on
  int len = 1;
  while (wave + len < kWaves && left_open(wave + len) == cu.unit) ++len;
  const StreamUnit u = stream_unit(run, begin, cu.step - begin, cu.steps, a.steps);
  const bool whole = !u.ends_inside && u.n == len;  // the unit lies inside this workgroup
  parts_of(cu.row_start, cu.tokens).close(my_o, my_s, kStrideO, kStrideS, len, whole, u, run, cu.unit);
}

template <int D, bool kAppend, int kSets, int kPolicy>
hipError_t launch_kv4(const Kv4AttnArgs& a, hipStream_t stream) {
  const int waves = kv4_waves((int64_t)a.num_runs * a.num_kv_heads);
  const dim3 blocks(kv4_groups(a.num_runs, a.num_kv_heads));
  if (waves == kKv4Big)
    hipLaunchKernelGGL((kv4_decode_kernel<D, kAppend, kKv4Big, kSets, kPolicy>), blocks, dim3(kKv4Big * 64), 0, stream,
                       a);
  else
    hipLaunchKernelGGL((kv4_decode_kernel<D, kAppend, kKv4Small, kSets, kPolicy>), blocks, dim3(kKv4Small * 64), 0,
                       stream, a);
  return hipGetLastError();
}

// Every variant is instantiated explicitly (see attn_decode.hip).
template __global__ void kv4_decode_kernel<128, false, kKv4Big, 1, kStreamPolicy>(Kv4AttnArgs);
template __global__ void kv4_decode_kernel<128, false, kKv4Small, 1, kStreamPolicy>(Kv4AttnArgs);
template __global__ void kv4_decode_kernel<128, true, kKv4Big, 1, kStreamPolicy>(Kv4AttnArgs);
template __global__ void kv4_decode_kernel<128, true, kKv4Small, 1, kStreamPolicy>(Kv4AttnArgs);
template __global__ void kv4_decode_kernel<128, false, kKv4Big, 2, kStreamPolicy>(Kv4AttnArgs);
template __global__ void kv4_decode_kernel<128, false, kKv4Small, 2, kStreamPolicy>(Kv4AttnArgs);
template __global__ void kv4_decode_kernel<128, false, kKv4Big, 2, kSharedPolicy>(Kv4AttnArgs);
template __global__ void kv4_decode_kernel<128, false, kKv4Small, 2, kSharedPolicy>(Kv4AttnArgs);
template __global__ void kv4_decode_kernel<64, false, kKv4Big, 1, kStreamPolicy>(Kv4AttnArgs);
template __global__ void kv4_decode_kernel<64, false, kKv4Small, 1, kStreamPolicy>(Kv4AttnArgs);
template __global__ void kv4_decode_kernel<64, true, kKv4Big, 1, kStreamPolicy>(Kv4AttnArgs);
template __global__ void kv4_decode_kernel<64, true, kKv4Small, 1, kStreamPolicy>(Kv4AttnArgs);
template __global__ void kv4_decode_kernel<64, false, kKv4Big, 2, kStreamPolicy>(Kv4AttnArgs);
template __global__ void kv4_decode_kernel<64, false, kKv4Small, 2, kStreamPolicy>(Kv4AttnArgs);
template __global__ void kv4_decode_kernel<64, false, kKv4Big, 2, kSharedPolicy>(Kv4AttnArgs);
template __global__ void kv4_decode_kernel<64, false, kKv4Small, 2, kSharedPolicy>(Kv4AttnArgs);

// One set of columns where every unit has at most 16 rows.  Codes that one unit alone reads are streamed
// past the caches (256 tasks' decode 384 us, 429 without); those that the next unit of their task reads
// again are not.
template <int D>
hipError_t launch_kv4(const Kv4AttnArgs& a, hipStream_t stream) {
  if (a.k_new) return launch_kv4<D, true, 1, kStreamPolicy>(a, stream);
  if (a.cols <= 16) return launch_kv4<D, false, 1, kStreamPolicy>(a, stream);
  return a.reread ? launch_kv4<D, false, 2, kSharedPolicy>(a, stream) : launch_kv4<D, false, 2, kStreamPolicy>(a, stream);
}

}  // namespace kern

hipError_t launch_kv4_decode(const Kv4AttnArgs& a, int head_dim, hipStream_t stream) {
  if (head_dim == 128) return kern::launch_kv4<128>(a, stream);
  if (head_dim == 64) return kern::launch_kv4<64>(a, stream);
  return hipErrorInvalidValue;
}

}  // namespace tide
