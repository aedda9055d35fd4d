// Attention of rows over block lists (sparse_attn.hip), several rows of one task at a time.
//
// Neighbouring rows of a task list mostly the same blocks, and a step of one row fills G of the 16 columns of an
// MFMA.  One workgroup here takes up to 8 rows of a kv head, 32 / P of them, where P is the least power of two of
// at least G: it marks which row lists which block (a byte a block in LDS), packs the marked blocks, and walks
// them as the one-row kernel walks a list, with the rows' heads as the columns of one or two products that share
// every K and V operand.  A column takes part where its row's mark is set and the key is not past its position.
// Its traffic is the union of the lists, not their sum: 1,761 rows of 128 blocks each over 8 contexts of 32k-98k
// (64 / 8 heads, d = 128), whose fours list 227-263 different blocks, take 675 us by single rows, which is what the L1s
// deliver (16 KB a step of 32 keys), and 410 here (16 TB/s out of L2, 91% hits; registers and LDS hold two waves a
// SIMD).  Leaving out a product whose rows list neither block costs more than it saves: branches between products made
// the accumulators be copied and each read of V be waited for by itself (470 us).
//
// What rows do not share must not reach them: a weight of zero times a V that is not finite is NaN.  The outputs
// of rows taken together are looked at, and rows with one that is not finite are taken again, one by one; so are
// rows that list a block twice, which a mark does not count.
#include <algorithm>
#include <type_traits>

#include "attn_decode.h"

namespace tide {
namespace kern {

constexpr float kNoKeysYet = -3.0e38f;  // as kNoKeys of sparse_attn.hip
constexpr int kSharedWaves = 4, kSharedThreads = kSharedWaves * 64;

// The lane, worked out where it is used: offsets made from a lane that is known from the start are kept from one turn
// of the loop over tasks to the next, and cost more registers than there are.
__device__ __forceinline__ int lane_now() {
  int x;
  asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=&v"(x));
  return x;
}

// f over the four lane groups of 16, in every lane.
template <class F>
__device__ __forceinline__ float over_groups(float x, F&& f) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  const auto s = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  const uint32_t y = __builtin_bit_cast(uint32_t, f(__builtin_bit_cast(float, (uint32_t)s[0]), __builtin_bit_cast(float, (uint32_t)s[1])));
  const auto t = __builtin_amdgcn_permlane32_swap(y, y, false, false);
  return f(__builtin_bit_cast(float, (uint32_t)t[0]), __builtin_bit_cast(float, (uint32_t)t[1]));
}

// An entry of the packed list: its page, and its block in the upper 24 bits of the other word, the rows that list it in
// the lower 8 (none where there is no page to read).
struct SharedStep {
  bool there;
  uint32_t what0, what1;
};

template <int D, int kTiles>
__global__ __launch_bounds__(kSharedThreads) __attribute__((amdgpu_waves_per_eu(2, 2)))
void sparse_shared_kernel(SparseArgs a) {
  using KL = KLds<D>;
  using VL = VLds<D>;
  constexpr int kC = D / 32, kT = D / 16, kWaves = kSharedWaves;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int Hkv = a.num_kv_heads, G = a.group, R = a.rows_at_once, shift = a.padded_shift;
  const int nth = blockIdx.x / Hkv, head = blockIdx.x - nth * Hkv;
  const int64_t row0 = (int64_t)a.first_row + (int64_t)nth * R;
  // K pages of the two steps in flight; marks before them, outputs after them
  __shared__ __attribute__((aligned(1024))) uint8_t k_lds0[kWaves * 2 * KL::kPageBytes];
  __shared__ __attribute__((aligned(1024))) uint8_t k_lds1[kWaves * 2 * KL::kPageBytes];
  __shared__ __attribute__((aligned(16))) uint2 list_of[kSharedEntries + 1];
  __shared__ f32x4 stats[kWaves][16 * kTiles];
  __shared__ int32_t row_task[kSharedRows], row_pos[kSharedRows], used;
  __shared__ uint32_t sums[kWaves], flags;  // flags: rows that have to be taken again
  static_assert(sizeof(k_lds0) >= kSharedBlocks<D>, "a mark a block");
  uint8_t* const ka = k_lds0 + wave * 2 * KL::kPageBytes;
  uint8_t* const kb = k_lds1 + wave * 2 * KL::kPageBytes;
  uint32_t* const marks = reinterpret_cast<uint32_t*>(k_lds0);
  const uint8_t* kpool = reinterpret_cast<const uint8_t*>(a.k_pool);
  const uint8_t* vpool = reinterpret_cast<const uint8_t*>(a.v_pool);
  constexpr uint32_t kMine = 2 * KL::kPageBytes;  // of a wave in either
  constexpr int64_t kBlk = (int64_t)kPage * D * 2;

  // lane r: row r.  (In LDS, not in registers, while attention runs; every wave writes the same.)
  auto load_rows = [&](int& task, int& pos) {
    const int l = lane_now();
    task = pos = -1;
    if (l < R) task = row_task[l], pos = row_pos[l];
  };
  uint32_t left = 0, solo = 0;
  {
    const int l = lane_now();
    int task = -1, pos = -1;
    if (l < R && (int64_t)nth * R + l < a.rows) {
      task = a.row_task[row0 + l];
      pos = a.row_pos[row0 + l];
      if (!live_row(task, pos, a.num_tasks, (int64_t)a.bt_stride * kPage)) task = -1;
    }
    if (l < R) row_task[l] = task, row_pos[l] = pos;
    left = (uint32_t)__builtin_amdgcn_ballot_w64(task >= 0);
  }
  bool flag_error = false;
  while (left) {
    int my_task, my_pos;
    load_rows(my_task, my_pos);
    const int r0 = __builtin_ctz(left), task = __builtin_amdgcn_readlane(my_task, r0);
    const uint32_t same = (uint32_t)__builtin_amdgcn_ballot_w64(my_task == task) & left & ~solo;
    const uint32_t subset = (solo >> r0) & 1 ? 1u << r0 : same;
    const bool alone = (subset & (subset - 1)) == 0;
    const int32_t* table = a.block_table + (int64_t)task * a.bt_stride;
    int least = INT32_MAX, last = -1;  // positions
    for (uint32_t rows = subset; rows; rows &= rows - 1) {
      const int pos = __builtin_amdgcn_readlane(my_pos, __builtin_ctz(rows));
      least = min(least, pos);
      last = max(last, pos);
    }
    auto entry = [&](int b, uint32_t rows) {
      const int32_t page = table[b];
      const bool ok = page >= 0 && page < a.num_pages;
      flag_error |= !ok;
      return ok ? uint2{(uint32_t)page, (uint32_t)b << 8 | rows} : uint2{0u, 0u};
    };

    // ---- the packed list ----
    int entries;
    const int me = 64 * wave + lane_now();
    if (me == 0) flags = 0, used = 0;
    if (alone) {
      const int32_t* list = a.sel + ((row0 + r0) * Hkv + head) * a.budget;
      __syncthreads();
      for (int i = me; i < a.budget; i += kSharedThreads) {
        const int32_t b = list[i];
        const bool in = b >= 0 && b <= last / kPage;
        list_of[i] = in ? entry(b, subset) : uint2{0u, 0u};
        if (in) atomicMax(&used, i + 1);
      }
      __syncthreads();
      entries = __builtin_amdgcn_readfirstlane(used);
    } else {
      const int words = (last / kPage + 4) / 4;
      for (int i = me; i < words; i += kSharedThreads) marks[i] = 0;
      __syncthreads();
      for (int r = wave; r < R; r += kWaves) {  // a row a wave, four entries of a lane on their way
        if (!((subset >> r) & 1)) continue;
        const int blocks = __builtin_amdgcn_readlane(my_pos, r) / kPage + 1;
        const int32_t* list = a.sel + ((row0 + r) * Hkv + head) * a.budget;
        for (int i = me & 63; i < a.budget; i += 256) {
          int32_t b[4];
#pragma unroll
          for (int u = 0; u < 4; ++u) b[u] = list[min(i + 64 * u, a.budget - 1)];
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            if (i + 64 * u >= a.budget || b[u] < 0 || b[u] >= blocks) continue;
            const uint32_t bit = 1u << (8 * (b[u] & 3) + r);
            if (atomicOr(&marks[b[u] >> 2], bit) & bit) flags = 1u;  // (any thread that finds it writes the same)
          }
        }
      }
      __syncthreads();
      const bool twice = flags != 0;
      __syncthreads();
      if (twice) {
        solo |= subset;
        continue;
      }
      // a thread packs `per` words
      const int per = (words + kSharedThreads - 1) / kSharedThreads, w0 = min(words, me * per), w1 = min(words, w0 + per);
      uint32_t count = 0;
      for (int w = w0; w < w1; ++w) {
        const uint32_t m = marks[w];
        count += ((m & 0xFF) != 0) + ((m & 0xFF00) != 0) + ((m & 0xFF0000) != 0) + ((m >> 24) != 0);
      }
      // sums over the lanes before this one, bit by bit (a shuffle's lane addresses would be kept in registers)
      uint32_t to = 0, all = 0;
      for (int k = 0; (4 * per) >> k; ++k) {
        const uint64_t who = __builtin_amdgcn_ballot_w64((count >> k) & 1);
        to += __builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0)) << k;
        all += (uint32_t)__popcll(who) << k;
      }
      if ((me & 63) == 0) sums[wave] = all;
      __syncthreads();
      entries = 0;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        to += w < wave ? sums[w] : 0u;
        entries += (int)sums[w];
      }
      entries = __builtin_amdgcn_readfirstlane(entries);
      for (int w = w0; w < w1; ++w) {
        const uint32_t m = marks[w];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t rows = (m >> (8 * i)) & 0xFF;
          if (rows) list_of[to++] = uint2{(uint32_t)(4 * w + i), rows};
        }
      }
      __syncthreads();
      for (int i = me; i < entries; i += kSharedThreads) list_of[i] = entry((int)list_of[i].x, list_of[i].y);
    }
    if (me == 0) list_of[entries] = uint2{0u, 0u};  // (the other of the last pair)
    __syncthreads();

    // ---- its attention ----
    const int l0 = lane_now(), col = l0 & 15, grp = l0 >> 4;
    uint32_t k_src[KL::kDma];
#pragma unroll
    for (int i = 0; i < KL::kDma; ++i) k_src[i] = KL::src_offset(i, l0);
    const uint32_t k_rd = kMine * wave + KL::lds_offset(col, grp);  // odd pieces: ^ 64
    const uint32_t v_off = (uint32_t)(16 * l0);
    constexpr int kRpl = 1024 / (2 * D);
    // (of load i: 1024 i + (v_wr ^ what i changes of the row's swizzle))
    const uint32_t v_wr = kMine * wave + VL::offset(l0 / VL::kNG, l0 % VL::kNG);
    auto v_place = [&](int i) { return (v_wr ^ (32u * VL::vsw(i * kRpl))) + 1024 * i; };
    const int vr = 4 * grp + (col >> 2);
    // (of piece t: v_rd ^ 32 t, since a row's swizzle is an exclusive or of the same bits; registers are scarce here)
    const uint32_t v_rd = kMine * wave + (uint32_t)(vr * 2 * D + 32 * VL::vsw(vr) + 8 * (l0 & 3));
    const int pairs = (entries + 1) / 2;
    int next_pair = wave;
    auto issue = [&](DecodeRegs<D>& r, uint8_t* kbuf) {
      SharedStep s = {next_pair < pairs, 0u, 0u};
      uint32_t page0 = 0, page1 = 0;
      if (s.there) {
        const u32x4 x = *reinterpret_cast<const u32x4*>(&list_of[2 * next_pair]);
        page0 = (uint32_t)__builtin_amdgcn_readfirstlane((int)x[0]);
        s.what0 = (uint32_t)__builtin_amdgcn_readfirstlane((int)x[1]);
        page1 = (uint32_t)__builtin_amdgcn_readfirstlane((int)x[2]);
        s.what1 = (uint32_t)__builtin_amdgcn_readfirstlane((int)x[3]);
        next_pair += kWaves;
      }
      const int64_t b0 = ((int64_t)page0 * Hkv + head) * kBlk, b1 = ((int64_t)page1 * Hkv + head) * kBlk;
      const int z0 = (s.what0 & 0xFF) ? (int)kBlk : 0, z1 = (s.what1 & 0xFF) ? (int)kBlk : 0;
      load_step<D, kSharedPolicy>(r, kbuf, block_rsrc(kpool + b0, z0), block_rsrc(kpool + b1, z1),
                                  block_rsrc(vpool + b0, z0), block_rsrc(vpool + b1, z1), k_src, v_off);
      return s;
    };

    // column `col` of product t: row and head, its bit, its position
    uint32_t bit[kTiles];
    bf16x8 qf[kTiles][kC];
    f32x4 o[kTiles][kT];
    float m_ref[kTiles], l_part[kTiles], l_exact[kTiles];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      const int r = (16 * t + col) >> shift, h = (16 * t + col) & ((1 << shift) - 1);
      const bool on = h < G && r < R && (subset >> r) & 1;
      bit[t] = on ? 1u << r : 0;
      const int64_t at = ((row0 + (on ? r : r0)) * a.num_q_heads + head * G + (on ? h : 0)) * D;
#pragma unroll
      for (int c = 0; c < kC; ++c) {
        const u32x4 x = load_u32x4(a.q + at + 32 * c + 8 * grp);
        qf[t][c] = as_bf16x8(on ? x : zero_u32x4());
      }
#pragma unroll
      for (int i = 0; i < kT; ++i) o[t][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      m_ref[t] = kNoKeysYet;
      l_part[t] = l_exact[t] = 0.0f;
    }

    auto compute = [&](DecodeRegs<D>& cur, uint8_t* lds, const SharedStep& st) {  // lds: k_lds0 or k_lds1
      const int p0 = (int)(st.what0 >> 8) * kPage, p1 = (int)(st.what1 >> 8) * kPage;  // first positions
      const bool tail = max(p0, p1) + kPage - 1 > least;  // some key may be past some row's position
      if (tail) {
        // V rows past every position must not reach the MFMA (NaN * 0 = NaN)
        const int l2 = lane_now();
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int i = 0; i < DecodeRegs<D>::kLoads; ++i)
            if ((t ? p1 : p0) + i * kRpl + l2 / VL::kNG > last) cur.v[t][i] = zero_u32x4();
      }
      f32x4 s[kTiles][2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        u32x4 kk[kC];
#pragma unroll
        for (int c = 0; c < kC; ++c)
          kk[c] = *reinterpret_cast<const u32x4*>(lds + (k_rd ^ (64 * (c & 1))) + t * KL::kPageBytes + 1024 * (c >> 1));
#pragma unroll
        for (int u = 0; u < kTiles; ++u) {
          s[u][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
          for (int c = 0; c < kC; ++c) s[u][t] = mfma16(as_bf16x8(kk[c]), qf[u][c], s[u][t]);
        }
      }
      // V over the K copy, which is done with
#pragma unroll
      for (int hp = 0; hp < 2; ++hp)
#pragma unroll
        for (int i = 0; i < DecodeRegs<D>::kLoads; ++i)
          *reinterpret_cast<u32x4*>(lds + v_place(i) + hp * KL::kPageBytes) = cur.v[hp][i];
      bf16x8 pb[kTiles];
#pragma unroll
      for (int u = 0; u < kTiles; ++u) {
        const bool in0 = (st.what0 & bit[u]) != 0, in1 = (st.what1 & bit[u]) != 0;
        if (tail) {  // keys past the row's position
          const int l2 = lane_now(), r = (16 * u + (l2 & 15)) >> shift;
          const int n0 = row_pos[min(r, kSharedRows - 1)] + 1 - 4 * (l2 >> 4) - p0, n1 = n0 + p0 - p1;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            s[u][0][e] = e < n0 ? s[u][0][e] : -INFINITY;
            s[u][1][e] = e < n1 ? s[u][1][e] : -INFINITY;
          }
        }
        const float top0 = fmaxf(fmaxf(s[u][0][0], s[u][0][1]), fmaxf(s[u][0][2], s[u][0][3]));
        const float top1 = fmaxf(fmaxf(s[u][1][0], s[u][1][1]), fmaxf(s[u][1][2], s[u][1][3]));
        float mt = a.scale_log2 * fmaxf(in0 ? top0 : -INFINITY, in1 ? top1 : -INFINITY);
        if (__any(mt > m_ref[u] + kRescaleSlack)) {  // only then is the column's maximum worked out
          mt = over_groups(mt, [](float x, float y) { return fmaxf(x, y); });
          const float m_new = fmaxf(m_ref[u], mt);
          const float alpha = fast_exp2(m_ref[u] - m_new);
          l_part[u] *= alpha;
          l_exact[u] *= alpha;
#pragma unroll
          for (int t = 0; t < kT; ++t) o[u][t] *= alpha;
          m_ref[u] = m_new;
        }
        // a row that does not list the block has weights of 2^-inf
        const float off0 = in0 ? -m_ref[u] : -INFINITY, off1 = in1 ? -m_ref[u] : -INFINITY;
        u32x4 wp;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float x0 = fast_exp2(fmaf(s[u][t][2 * e], a.scale_log2, t ? off1 : off0));
            const float x1 = fast_exp2(fmaf(s[u][t][2 * e + 1], a.scale_log2, t ? off1 : off0));
            // weights go to the P V product in bf16; the sum that divides it is of the rounded ones (sparse_attn.hip)
            wp[2 * t + e] = pack_bf16x2(x0, x1);
            l_part[u] = add_bf16x2(wp[2 * t + e], l_part[u]);
            l_exact[u] += x0 + x1;
          }
        pb[u] = as_bf16x8(wp);
      }
      constexpr int kAtOnce = 4;
#pragma unroll
      for (int t0 = 0; t0 < kT; t0 += kAtOnce) {
        bf16x8 vv[kAtOnce];
#pragma unroll
        for (int t = 0; t < kAtOnce; ++t) {
          const uint32_t at = v_rd ^ (32 * (t0 + t));
          const uint2 v0 = read_tr(lds + at), v1 = read_tr(lds + at + KL::kPageBytes);
          vv[t] = as_bf16x8(u32x4{v0.x, v0.y, v1.x, v1.y});
        }
#pragma unroll
        for (int t = 0; t < kAtOnce; ++t)
#pragma unroll
          for (int u = 0; u < kTiles; ++u) o[u][t0 + t] = mfma16(vv[t], pb[u], o[u][t0 + t]);
      }
    };

    {
      DecodeRegs<D> ra, rb;
      SharedStep sa = issue(ra, ka), sb;
      // no wave reads marks any more, which the loads overwrite
      while (sa.there) {
        sb = issue(rb, kb);
        __builtin_amdgcn_sched_barrier(0);
        compute(ra, k_lds0, sa);
        if (!sb.there) break;
        sa = issue(ra, ka);
        __builtin_amdgcn_sched_barrier(0);
        compute(rb, k_lds1, sb);
      }
    }

    // ---- the waves' parts ----
    // every load into LDS, the zero-length ones too, is done before LDS takes the parts
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    __builtin_amdgcn_s_waitcnt(0);
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    auto add = [](float x, float y) { return x + y; };
    const int l1 = lane_now(), c1 = l1 & 15, g1 = l1 >> 4;
#pragma unroll
    for (int u = 0; u < kTiles; ++u) {
      const float l = over_groups(l_part[u], add), lx = over_groups(l_exact[u], add);
      uint8_t* to = u ? kb : ka;
#pragma unroll
      for (int t = 0; t < kT; ++t)
        *reinterpret_cast<f32x4*>(to + 4 * D * c1 + 16 * ((4 * t + g1) ^ c1)) = o[u][t];
      if (g1 == 0) stats[wave][16 * u + c1] = f32x4{m_ref[u], l, lx, 0.0f};
    }
    __syncthreads();
    const int it = 64 * wave + lane_now(), il = it & 63;
    // whether a row has a key at all: it lists a block of the pool (every listed block has one)
    uint32_t listed = 0, with_keys = 0;
    for (int i = il; i < entries; i += 64) listed |= list_of[i].y & 0xFF;
#pragma unroll
    for (int r = 0; r < kSharedRows; ++r) with_keys |= __any((listed >> r) & 1) ? 1u << r : 0u;
    constexpr int kPiece = D / 4;  // 16-byte pieces of a head's output
    uint32_t again = 0;
    for (int i = it; i < (R << shift) * kPiece; i += kSharedThreads) {
      const int c = i / kPiece, p = i % kPiece, r = c >> shift, h = c & ((1 << shift) - 1), j = c & 15;
      if (h >= G || !((subset >> r) & 1)) continue;
      const uint8_t* from = (c < 16 ? k_lds0 : k_lds1) + 4 * D * j + 16 * (p ^ j);
      f32x4 st[kWaves];
      float m = kNoKeysYet;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        st[w] = stats[w][c];
        m = fmaxf(m, st[w][0]);
      }
      f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
      float ls = 0.0f, lxs = 0.0f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float f = fast_exp2(st[w][0] - m);
        acc += f * *reinterpret_cast<const f32x4*>(from + w * 2 * KL::kPageBytes);
        ls += f * st[w][1];
        lxs += f * st[w][2];
      }
      const bool has = (with_keys >> r) & 1;
      const float inv = has ? 1.0f / ls : 0.0f;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (!(fabsf(acc[e] * inv) < INFINITY)) again |= 1u << r;
      }
      const int64_t at = (row0 + r) * a.num_q_heads + head * G + h;
      const uint2 x = {pack_bf16x2(acc[0] * inv, acc[1] * inv), pack_bf16x2(acc[2] * inv, acc[3] * inv)};
      *reinterpret_cast<uint2*>(a.out + at * D + 4 * p) = has ? x : uint2{0u, 0u};
      if (a.lse && p == 0) a.lse[at] = has ? (m + __log2f(lxs)) * kLn2 : -INFINITY;
    }
    if (again && !alone) atomicOr(&flags, again);
    __syncthreads();
    const uint32_t redo = alone ? 0u : (uint32_t)__builtin_amdgcn_readfirstlane((int)flags);
    left &= ~subset | redo;
    solo |= redo;
    __syncthreads();  // flags, marks and parts have been read
  }
  if (flag_error) atomicOr(a.error_flags, 1);
}

template <int D>
hipError_t launch_shared(const SparseArgs& a, hipStream_t stream) {
  const uint32_t groups = (uint32_t)((a.rows + a.rows_at_once - 1) / a.rows_at_once);
  const dim3 grid(groups * (uint32_t)a.num_kv_heads);
  if ((a.rows_at_once << a.padded_shift) > 16)
    hipLaunchKernelGGL((sparse_shared_kernel<D, 2>), grid, dim3(kSharedThreads), 0, stream, a);
  else
    hipLaunchKernelGGL((sparse_shared_kernel<D, 1>), grid, dim3(kSharedThreads), 0, stream, a);
  return hipGetLastError();
}

// Every variant is instantiated explicitly (see attn_decode.hip).
template __global__ void sparse_shared_kernel<128, 1>(SparseArgs);
template __global__ void sparse_shared_kernel<128, 2>(SparseArgs);
template __global__ void sparse_shared_kernel<64, 1>(SparseArgs);
template __global__ void sparse_shared_kernel<64, 2>(SparseArgs);

}  // namespace kern

hipError_t launch_sparse_shared(const SparseArgs& a, int head_dim, hipStream_t stream) {
  return head_dim == 128 ? kern::launch_shared<128>(a, stream) : kern::launch_shared<64>(a, stream);
}

}  // namespace tide
