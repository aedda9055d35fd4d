// Choice of the blocks (pages of 16 positions) that a row attends to, by the bounds of their keys.
//
// For every entry i a key of the block lies between lo_i 2^s and hi_i 2^s (key_bounds.hip), so a query's
// product with any of its keys is at most sum_i max(q_i hi_i, q_i lo_i) 2^s.  With the query itself in whole
// units, c = q / 2^t rounded, |c| <= 127, the score of a block is the largest of that bound over the kv
// head's query heads:
//     score = max_h 2^clamp(s + t_h, -100, 100) I_h,   I_h = sum_i max(c_hi hi_i, c_hi lo_i).
// max(c hi, c lo) = max(c, 0) hi + min(c, 0) lo, so I_h is one product of length 2 d over 8-bit whole
// numbers, for the matrix instructions; |I_h| <= d 127^2 < 2^24, so float(I_h) and its scaling are exact and
// the choice does not depend on the order of any sum.
//
// Scores (score_kernel): a wave takes 64 blocks of one (unit, kv head) at a time, their bounds as B
// operands straight from memory (16 columns = blocks) and 16 query rows a product as A operands: the heads
// of a row then lie in the registers of a lane and in 1, 2 or 4 lane groups, and their maximum costs 3 to 5
// instructions.  A unit is one row (decode steps: each row has a task of its own), or the rows of a few
// products, which share the bounds they read where they are of one task.
// Choice (choose_kernel): one workgroup per (row, kv head) finds the smallest score that is taken, by
// counting scores in bins that narrow around it, and packs what is taken in order by prefix sums.
#include <algorithm>

#include "kernels.h"
#include "tide_device.h"

namespace tide {
namespace kern {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

constexpr int kScoreWaves = 4;
constexpr int kChunkTiles = 4;  // products of 16 query rows of a unit that is not one row
constexpr int kSteps = 4;       // groups of 16 blocks that a wave has in flight

template <int D>
struct QueryTile {
  i32x4 a[D / 32];  // chunk c: entries 64 c .. of max(c, 0) for c < D / 64, of min(c, 0) behind them
  int unit[4];      // t of query rows 4 (lane / 16) + r
};

// Query rows of a tile: row p of 16 is head min(p % P, G - 1) of token `token[p / P]`.
template <int D>
__device__ __forceinline__ void load_tile(const BlockSelectArgs& a, QueryTile<D>& out, int64_t row, int head, int h) {
  constexpr int kC = D / 64;
  const int lane = threadIdx.x & 63, grp = lane >> 4;
  const uint16_t* q = a.q + ((row * a.num_q_heads) + head * a.group + h) * D;
  u32x4 x[kC][2];
#pragma unroll
  for (int c = 0; c < kC; ++c)
#pragma unroll
    for (int i = 0; i < 2; ++i) x[c][i] = load_u32x4(q + 64 * c + 16 * grp + 8 * i);
  uint32_t top = 0;
#pragma unroll
  for (int c = 0; c < kC; ++c)
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) top = max(top, max(x[c][i][j] & 0x7FFFu, (x[c][i][j] >> 16) & 0x7FFFu));
  top = max(top, (uint32_t)__shfl_xor((int)top, 16, 64));
  top = max(top, (uint32_t)__shfl_xor((int)top, 32, 64));
  // (as the units of key bounds)
  const int unit = max(kLeastUnit, (int)(top >> 7) - 133 + ((top & 0x7F) == 0x7F ? 1 : 0));
  const bool finite = top < 0x7F80u;
  const float scale = finite ? __builtin_bit_cast(float, (uint32_t)(127 - unit) << 23) : 0.0f;
#pragma unroll
  for (int c = 0; c < kC; ++c) {
    i32x4 plus = {0, 0, 0, 0}, minus = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const uint32_t pair = x[c][e >> 3][(e >> 1) & 3];
      const float v = __builtin_bit_cast(float, (e & 1) ? pair & 0xFFFF0000u : pair << 16);
      const int code = finite ? (int)rintf(v * scale) : 0;  // a query that is not finite counts as zeros
      plus[e >> 2] |= (max(code, 0) & 0xFF) << (8 * (e & 3));
      minus[e >> 2] |= (min(code, 0) & 0xFF) << (8 * (e & 3));
    }
    out.a[c] = plus;
    out.a[kC + c] = minus;
  }
#pragma unroll
  for (int r = 0; r < 4; ++r) out.unit[r] = __shfl(finite ? unit : 0, 4 * grp + r, 64);
}

template <int D, int kTiles>
__global__ __launch_bounds__(kScoreWaves * 64) void score_kernel(BlockSelectArgs a) {
  constexpr int kC = D / 32;
  const int lane = threadIdx.x & 63, col = lane & 15, grp = lane >> 4;
  const uint32_t id = blockIdx.x * kScoreWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int Hkv = a.num_kv_heads, G = a.group;
  const int rest = (int)(id / (uint32_t)Hkv), head = (int)id - rest * Hkv;
  const int unit = rest / a.splits, split = rest - unit * a.splits;
  const int row0 = unit * a.tile_rows;  // from first_row
  if (row0 >= a.rows) return;
  // heads of a token are padded to P rows of a product (the last one again), 16 / P tokens a product
  const int shift = 32 - __builtin_clz(2 * G - 1) - 1, P = 1 << shift, tokens = 16 >> shift;

  // lane i: row i of the unit
  int my_task = -1, my_pos = -1;
  if (lane < a.tile_rows && row0 + lane < a.rows) {
    my_task = a.row_task[a.first_row + row0 + lane];
    my_pos = a.row_pos[a.first_row + row0 + lane];
    if (!live_row(my_task, my_pos, a.num_tasks, a.max_len)) my_task = -1;
  }
  uint64_t left = __builtin_amdgcn_ballot_w64(my_task >= 0);
  bool flag_error = false;
  bool loaded = false;
  QueryTile<D> q[kTiles];
  while (left) {
    const int task = __builtin_amdgcn_readlane(my_task, __builtin_ctzll(left));
    const uint64_t mine = __builtin_amdgcn_ballot_w64(my_task == task) & left;
    left &= ~mine;
    int last = (mine >> lane) & 1 ? my_pos : 0;
#pragma unroll
    for (int m = 1; m < 64; m *= 2) last = max(last, __shfl_xor(last, m, 64));
    const int blocks = __builtin_amdgcn_readfirstlane(last) / kPage + 1;
    const int32_t* table = a.block_table + (int64_t)task * a.bt_stride;
    constexpr int kPer = 16 * kSteps;
    for (int b0 = split * kPer; b0 < blocks; b0 += a.splits * kPer) {
      const int mb = b0 + lane;
      int32_t page = mb < blocks ? table[mb] : 0;
      const bool bad = mb < blocks && (page < 0 || page >= a.num_pages);
      flag_error |= bad;
      if (bad) page = 0;  // read in its place; its score is -inf
      const int64_t block = (int64_t)page * Hkv + head;
      int s = a.units[block];
      if (bad) s = -128;
      i32x4 b[kSteps][kC];
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        const int64_t from = (int64_t)__shfl(page, 16 * i + col, 64) * Hkv + head;
        const int8_t* p = a.bounds + from * (2 * D) + 16 * grp;
        if (b0 + 16 * i < blocks) {
#pragma unroll
          for (int c = 0; c < kC; ++c) b[i][c] = *reinterpret_cast<const i32x4*>(p + 64 * c);
        }
      }
      if (!loaded) {
        loaded = true;
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
          const int token = min(row0 + t * tokens + (col >> shift), a.rows - 1);
          load_tile<D>(a, q[t], (int64_t)a.first_row + token, head, min(col & (P - 1), G - 1));
        }
      }
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        if (b0 + 16 * i >= blocks) break;
        const int us = __shfl(s, 16 * i + col, 64);
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
          i32x4 acc = {0, 0, 0, 0};
#pragma unroll
          for (int c = 0; c < kC; ++c) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(q[t].a[c], b[i][c], acc, 0, 0, 0);
          float x[4];
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int e = min(max(us + q[t].unit[r], -100), 100);
            x[r] = __builtin_amdgcn_ldexpf((float)acc[r], e);
            if (us == kNoUnit) x[r] = INFINITY;
            if (us == -128) x[r] = -INFINITY;
          }
          // query row 4 grp + r is head (4 grp + r) % P of token (4 grp + r) / P of the product
          auto put = [&](float v, int token) {
            const int u = t * tokens + token;
            if (u < a.tile_rows && ((mine >> u) & 1))
              a.scores[((int64_t)(row0 + u) * Hkv + head) * a.score_stride + b0 + 16 * i + col] = v;
          };
          if (shift == 0) {
#pragma unroll
            for (int r = 0; r < 4; ++r) put(x[r], 4 * grp + r);
          } else if (shift == 1) {
            put(fmaxf(x[0], x[1]), 2 * grp);
            put(fmaxf(x[2], x[3]), 2 * grp + 1);
          } else {
            float m = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
            if (shift > 2) m = fmaxf(m, xor_shfl(m, 16));
            if (shift > 3) m = fmaxf(m, xor_shfl(m, 32));
            if ((grp & ((P >> 2) - 1)) == 0) put(m, (4 * grp) >> shift);
          }
        }
      }
    }
  }
  if (flag_error) atomicOr(a.error_flags, 1);
}

// ---- the choice ----------------------------------------------------------------------------------
constexpr int kChoose = 256;     // threads
constexpr int kChooseBins = 1024;
constexpr int kChooseHeld = 8;   // chunks of 4 kChoose scores that the threads hold: contexts of 131,072

__device__ __forceinline__ uint32_t score_key(float x) {  // orders as scores do
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Sum of x over the threads before this one; *all: over all.  tmp: 4 words, free again after the
// next barrier.
__device__ __forceinline__ uint32_t choose_scan(uint32_t x, uint32_t* tmp, uint32_t* all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t in = x;
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    const uint32_t y = __shfl_up((int)in, o, 64);
    if (lane >= o) in += y;
  }
  if (lane == 63) tmp[wave] = in;
  __syncthreads();
  uint32_t before = 0, total = 0;
#pragma unroll
  for (int w = 0; w < kChoose / 64; ++w) {
    if (w == wave) before = total;
    total += tmp[w];
  }
  *all = total;
  return before + in - x;
}

__global__ __launch_bounds__(kChoose) void choose_kernel(BlockSelectArgs a) {
  __shared__ uint32_t hist[kChooseBins];
  __shared__ uint32_t tmp[2][kChoose / 64];
  __shared__ uint32_t found[3];  // bin, scores above it, scores in it
  __shared__ uint32_t range[2];  // least and largest key
  const int tid = threadIdx.x;
  const int nth = blockIdx.x / a.num_kv_heads, head = blockIdx.x - nth * a.num_kv_heads;
  const int64_t row = (int64_t)a.first_row + nth;
  const int32_t task = a.row_task[row], pos = a.row_pos[row];
  if (!live_row(task, pos, a.num_tasks, a.max_len)) return;
  int32_t* sel = a.sel + (row * a.num_kv_heads + head) * a.budget;
  const int blocks = pos / kPage + 1;
  if (blocks <= a.budget) {
    for (int i = tid; i < a.budget; i += kChoose) sel[i] = i < blocks ? i : -1;
    return;
  }
  const int want = a.budget - a.sink - a.recent, n = blocks - a.sink - a.recent;  // n > want >= 0
  for (int i = tid; i < a.sink; i += kChoose) sel[i] = i;
  for (int i = tid; i < a.recent; i += kChoose) sel[a.sink + want + i] = blocks - a.recent + i;
  if (want == 0) return;
  const float* score = a.scores + ((int64_t)nth * a.num_kv_heads + head) * a.score_stride + a.sink;

  // scores 4 p .. 4 p + 3 of the n; those past them count nowhere
  auto load4 = [&](int p, uint32_t (&key)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) key[i] = p + i < n ? score_key(score[p + i]) : 0;
  };
  uint32_t held[kChooseHeld][4];
#pragma unroll
  for (int c = 0; c < kChooseHeld; ++c)
    if (4 * c * kChoose < n) load4(4 * (tid + c * kChoose), held[c]);
  auto each = [&](auto&& f) {  // f(keys, first index) over this thread's scores, in order
#pragma unroll
    for (int c = 0; c < kChooseHeld; ++c)
      if (4 * c * kChoose < n) f(held[c], 4 * (tid + c * kChoose));
    for (int c = kChooseHeld; 4 * c * kChoose < n; ++c) {
      uint32_t key[4];
      load4(4 * (tid + c * kChoose), key);
      f(key, 4 * (tid + c * kChoose));
    }
  };

  // The want-th largest key: bins over [low, high] in which it lies, `rest` of them to take from there.
  // Taken in the end: keys >= from, and the first `equal` of those == from - 1.
  uint32_t low = 0, high = 0xFFFFFFFFu, rest = want, from = 0, equal = 0;
  for (;;) {
    // the range that the keys in question cover
    if (tid == 0) range[0] = 0xFFFFFFFFu, range[1] = 0;
    for (int i = tid; i < kChooseBins; i += kChoose) hist[i] = 0;
    __syncthreads();
    uint32_t mn = 0xFFFFFFFFu, mx = 0;
    each([&](const uint32_t (&key)[4], int p) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (p + i < n && key[i] >= low && key[i] <= high) mn = min(mn, key[i]), mx = max(mx, key[i]);
    });
#pragma unroll
    for (int m = 1; m < 64; m *= 2) {
      mn = min(mn, (uint32_t)__shfl_xor((int)mn, m, 64));
      mx = max(mx, (uint32_t)__shfl_xor((int)mx, m, 64));
    }
    if ((tid & 63) == 0) {
      atomicMin(&range[0], mn);
      atomicMax(&range[1], mx);
    }
    __syncthreads();
    low = range[0], high = range[1];
    if (low == high) {  // equal scores
      from = low + 1;
      equal = rest;
      break;
    }
    const int shift = max(0, 32 - __builtin_clz(high - low) - 10);  // bins of 2^shift keys
    each([&](const uint32_t (&key)[4], int p) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (p + i < n && key[i] >= low && key[i] <= high) atomicAdd(&hist[(key[i] - low) >> shift], 1u);
    });
    __syncthreads();
    // bins from the largest down, four a thread
    uint32_t in[4], sum = 0, all;
#pragma unroll
    for (int i = 0; i < 4; ++i) sum += in[i] = hist[kChooseBins - 1 - 4 * tid - i];
    uint32_t before = choose_scan(sum, tmp[0], &all);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (before < rest && before + in[i] >= rest)
        found[0] = kChooseBins - 1 - 4 * tid - i, found[1] = before, found[2] = in[i];
      before += in[i];
    }
    __syncthreads();
    const uint32_t bin = found[0], above = found[1], inside = found[2];
    rest -= above;
    low += bin << shift;
    if (inside == rest) {  // all of the bin
      from = low;
      break;
    }
    high = min(high, low + ((1u << shift) - 1));
    __syncthreads();
  }

  // what is taken, in order
  uint32_t placed = 0, met = 0;  // taken by `from`, and equal to from - 1, in the chunks before
  int round = 0;
  each([&](const uint32_t (&key)[4], int p) {
    uint32_t flags = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (p + i < n) flags += key[i] >= from ? 1u : equal && key[i] == from - 1 ? 0x10000u : 0u;
    uint32_t all;
    const uint32_t before = choose_scan(flags, tmp[round & 1], &all);
    ++round;
    uint32_t ge = placed + (before & 0xFFFF), eq = met + (before >> 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (p + i >= n) continue;
      const bool is_ge = key[i] >= from, is_eq = !is_ge && equal && key[i] == from - 1;
      if (is_ge || (is_eq && eq < equal)) sel[a.sink + ge + min(eq, equal)] = a.sink + p + i;
      ge += is_ge;
      eq += is_eq;
    }
    placed += all & 0xFFFF;
    met += all >> 16;
  });
}

template <int D>
hipError_t launch_scores(const BlockSelectArgs& a, hipStream_t stream) {
  const int64_t units = (a.rows + a.tile_rows - 1) / a.tile_rows;
  const uint32_t blocks = (uint32_t)((units * a.splits * a.num_kv_heads + kScoreWaves - 1) / kScoreWaves);
  if (a.tile_rows == 1)
    hipLaunchKernelGGL((score_kernel<D, 1>), dim3(blocks), dim3(kScoreWaves * 64), 0, stream, a);
  else
    hipLaunchKernelGGL((score_kernel<D, kChunkTiles>), dim3(blocks), dim3(kScoreWaves * 64), 0, stream, a);
  return hipGetLastError();
}

}  // namespace kern

int select_tile_rows(int32_t group, bool chunk) {
  int padded = 1;
  while (padded < group) padded *= 2;
  return chunk ? kern::kChunkTiles * 16 / padded : 1;
}

hipError_t launch_block_select(const BlockSelectArgs& a, int head_dim, hipStream_t stream) {
  // (a context within the budget has nothing to choose: no scores are read)
  hipError_t rc = hipSuccess;
  if ((a.max_len - 1) / kPage + 1 > a.budget && a.budget > a.sink + a.recent)
    rc = head_dim == 128 ? kern::launch_scores<128>(a, stream) : kern::launch_scores<64>(a, stream);
  if (rc != hipSuccess) return rc;
  hipLaunchKernelGGL(kern::choose_kernel, dim3((uint32_t)(a.rows * a.num_kv_heads)), dim3(kern::kChoose), 0, stream, a);
  return hipGetLastError();
}

}  // namespace tide
