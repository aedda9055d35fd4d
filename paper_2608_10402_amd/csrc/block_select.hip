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
// Scores (score_kernel): a wave holds 16 query rows a product as A operands and walks the blocks 16 at a
// time, their bounds as B operands straight from memory, the next 16 on their way while 16 are used.  With
// blocks as columns the heads of a token lie in the registers of a lane and in 1, 2 or 4 groups of 16 lanes,
// so their maximum is mostly in the lane; where it crosses groups, two products' groups are swapped into one
// register, and every lane ends with a score of its own to store.  The units are applied as products of
// floats, which is exact where no exponent leaves the normal range: t in [-60, 60], s in [-40, 40]; others
// take the clamped exponents one by one.  A unit of work is one row (decode steps: each row has a task of its
// own), or the rows of kChunkTiles products, which share the bounds that they read where they are of one task.
// Choice (choose_kernel): one workgroup per (row, kv head) finds the smallest score that is taken, by
// counting scores in bins that narrow around it, and packs what is taken in order by prefix sums.
#include <algorithm>

#include "attn_decode.h"

namespace tide {
namespace kern {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

constexpr int kChunkTiles = 4;  // products of 16 query rows of a unit that is not one row

// Scores are kept as 32-bit integers that order like them, both ways:
__device__ __forceinline__ int score_order(float x) {
  const int u = __builtin_bit_cast(int, x);
  return u ^ ((u >> 31) & 0x7FFFFFFF);
}

__device__ __forceinline__ float score_of(int key) {
  return __builtin_bit_cast(float, key ^ ((key >> 31) & 0x7FFFFFFF));
}

template <int D>
struct QueryTile {
  i32x4 a[D / 32];  // chunk c: entries 64 c .. of max(c, 0) for c < D / 64, of min(c, 0) behind them
  float two[4];     // 2^t of query rows 4 (lane / 16) + r
};

// Lane l's query row is l % 16 of the tile: head h of the row at `q`.  Returns whether t is in [-60, 60].
template <int D>
__device__ __forceinline__ bool load_tile(QueryTile<D>& out, const uint16_t* q) {
  constexpr int kC = D / 64;
  const int lane = threadIdx.x & 63, grp = lane >> 4;
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
  // (as the units of key bounds); a query that is not finite counts as zeros
  const bool finite = top < 0x7F80u;
  const int unit = finite ? max(kLeastUnit, (int)(top >> 7) - 133 + ((top & 0x7F) == 0x7F ? 1 : 0)) : 0;
  const float scale = __builtin_bit_cast(float, (uint32_t)(127 - unit) << 23);
#pragma unroll
  for (int c = 0; c < kC; ++c) {
    i32x4 plus = {0, 0, 0, 0}, minus = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const uint32_t pair = x[c][e >> 3][(e >> 1) & 3];
      const float v = __builtin_bit_cast(float, (e & 1) ? pair & 0xFFFF0000u : pair << 16);
      const int code = finite ? (int)rintf(v * scale) : 0;
      plus[e >> 2] |= (max(code, 0) & 0xFF) << (8 * (e & 3));
      minus[e >> 2] |= (min(code, 0) & 0xFF) << (8 * (e & 3));
    }
    out.a[c] = plus;
    out.a[kC + c] = minus;
  }
#pragma unroll
  for (int r = 0; r < 4; ++r)
    out.two[r] = __builtin_bit_cast(float, (uint32_t)(127 + __shfl(unit, 4 * grp + r, 64)) << 23);
  return unit >= -60 && unit <= 60;
}

// Lane groups g = 0 .. 3 of 16 lanes: max(a.g, a.g+1) for even g in group g, the same of b in group g + 1.
__device__ __forceinline__ float max_groups(float a, float b) {
  const auto s = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b),
                                                  false, false);
  return fmaxf(__builtin_bit_cast(float, (uint32_t)s[0]), __builtin_bit_cast(float, (uint32_t)s[1]));
}

// max of a's halves in the lower half, of b's in the upper one.
__device__ __forceinline__ float max_halves(float a, float b) {
  const auto s = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b),
                                                  false, false);
  return fmaxf(__builtin_bit_cast(float, (uint32_t)s[0]), __builtin_bit_cast(float, (uint32_t)s[1]));
}

// The bounds of 16 blocks in LDS.  A load brings whole blocks, neighbouring lanes neighbouring 16-byte pieces
// of one (read as operands straight from memory, neighbouring lanes would be in different blocks: 64 separate
// pieces a load, which kept the L1 busy for the whole kernel), and places them in lane order; which piece a
// lane brings is swizzled by the block, so that the 16 columns of an operand read distinct banks.
template <int D>
struct BoundsLds {
  static constexpr int kBlock = 2 * D;              // bytes
  static constexpr int kPieces = kBlock / 16;       // 16 or 8
  static constexpr int kPerLoad = 64 / kPieces;     // blocks
  static constexpr int kLoads = 16 / kPerLoad;      // of 1 KB
  static constexpr int kBytes = 16 * kBlock;
  // lane l of load i: block kPerLoad i + l / kPieces and its piece
  static __device__ __forceinline__ int block(int i) { return kPerLoad * i + (threadIdx.x & 63) / kPieces; }
  static __device__ __forceinline__ uint32_t piece(int i) {
    return 16u * (uint32_t)(((int)threadIdx.x & (kPieces - 1)) ^ (block(i) & (kPieces - 1)));
  }
  // byte offset of piece p of block `col`
  static __device__ __forceinline__ uint32_t offset(int col, int p) {
    return (uint32_t)(kBlock * col + 16 * (p ^ (col & (kPieces - 1))));
  }
};

typedef __attribute__((address_space(1))) const void global_void;

// kShift: the heads of a token are padded to P = 2^kShift rows of a product (the last head again), so a
// product holds 16 / P tokens.
template <int kTiles, int kShift>
struct ScoreOut {
  static constexpr int kTokens = 16 >> kShift;  // of a product
  // scores of a lane: one for each token and block of 16 x kTiles query rows and 16 blocks, 64 at a time
  static constexpr int kOut = kTiles * kTokens >= 4 ? kTiles * kTokens / 4 : 1;
  // score o of lane group grp is of token_of(o, grp) and block lane % 16
  static __device__ __forceinline__ int token_of(int o, int grp) {
    if (kShift == 0) return (o >> 2) * 16 + 4 * grp + (o & 3);
    if (kShift == 1) return (o >> 1) * 8 + 2 * grp + (o & 1);
    if (kShift == 2) return o * 4 + grp;
    if (kShift == 3) return kTiles > 1 ? (2 * o + (grp & 1)) * 2 + (grp >> 1) : grp >> 1;
    return kTiles > 1 ? 4 * o + grp : 0;
  }
  // a lane group that repeats another's scores
  static __device__ __forceinline__ bool repeats(int grp) {
    return kTiles == 1 && ((kShift == 3 && (grp & 1)) || (kShift == 4 && grp));
  }
};

// What a lane knows of a block: 2^s (1 where exponents go one by one; 0 where the score does not depend on
// the keys), and what is added to the score then.
struct BlockScale {
  int s;
  float two, more;
};

__device__ __forceinline__ BlockScale block_scale(bool ok, int s, bool odd_rows, bool* odd) {
  const bool none = !ok | (s == kNoUnit);
  *odd = odd_rows | (__builtin_amdgcn_ballot_w64(!none & ((uint32_t)(s + 40) > 80u)) != 0);
  uint32_t two = *odd ? 0x3F800000u : (uint32_t)(127 + s) << 23;
  two = none ? 0u : two;
  float more = s == kNoUnit ? INFINITY : 0.0f;
  more = ok ? more : -INFINITY;
  return BlockScale{s, __builtin_bit_cast(float, two), more};
}

// Scores of 16 blocks (their bounds as operands b; what lane 16 step + i of `sc` knows is of block i) and the query
// rows of q; stored 4 * block bytes behind put[], past the buffer's end where there is none to store.
template <int D, int kTiles, int kShift, bool kOdd>
__device__ __forceinline__ void score_step(const QueryTile<D> (&q)[kTiles], const i32x4 (&b)[D / 32], const BlockScale& sc,
                                           int step, __amdgpu_buffer_rsrc_t scores,
                                           const uint32_t (&put)[ScoreOut<kTiles, kShift>::kOut], int block) {
  constexpr int kC = D / 32;
  const int lane = threadIdx.x & 63, col = lane & 15, grp = lane >> 4;
  const float two = __shfl(sc.two, 16 * step + col, 64), more = __shfl(sc.more, 16 * step + col, 64);
  i32x4 acc[kTiles];
#pragma unroll
  for (int t = 0; t < kTiles; ++t) acc[t] = i32x4{0, 0, 0, 0};
#pragma unroll
  for (int c = 0; c < kC; ++c)
#pragma unroll
    for (int t = 0; t < kTiles; ++t) acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(q[t].a[c], b[c], acc[t], 0, 0, 0);
  const int us = kOdd ? __shfl(sc.s, 16 * step + col, 64) : 0;
  float x[kTiles][4];
#pragma unroll
  for (int t = 0; t < kTiles; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      if (kOdd) {
        const int e = us + (int)(__builtin_bit_cast(uint32_t, q[t].two[r]) >> 23) - 127;
        x[t][r] = __builtin_amdgcn_ldexpf((float)acc[t][r], min(max(e, -100), 100));
      } else {
        x[t][r] = (float)acc[t][r] * q[t].two[r];
      }
    }
  auto top4 = [&](int t) { return fmaxf(fmaxf(x[t][0], x[t][1]), fmaxf(x[t][2], x[t][3])); };
#pragma unroll
  for (int o = 0; o < ScoreOut<kTiles, kShift>::kOut; ++o) {
    float y;
    if (kShift == 0) y = x[o >> 2][o & 3];
    if (kShift == 1) y = fmaxf(x[o >> 1][2 * (o & 1)], x[o >> 1][2 * (o & 1) + 1]);
    if (kShift == 2) y = top4(o);
    if (kShift == 3) y = kTiles > 1 ? max_groups(top4(2 * o), top4(2 * o + 1)) : max_groups(top4(0), top4(0));
    if (kShift == 4) {
      const float lo = kTiles > 1 ? max_groups(top4(4 * o), top4(4 * o + 1)) : max_groups(top4(0), top4(0));
      y = kTiles > 1 ? max_halves(lo, max_groups(top4(4 * o + 2), top4(4 * o + 3))) : max_halves(lo, lo);
    }
    __builtin_amdgcn_raw_buffer_store_b32((uint32_t)score_order(fmaf(y, two, more)), scores, put[o], 4 * block, 0);
  }
}

// stores past the buffer's end are dropped: a lane with no score to store has such an offset
constexpr uint32_t kNowhere = 0x80000000u;

__device__ __forceinline__ __amdgpu_buffer_rsrc_t score_rsrc(const BlockSelectArgs& a, int row0, int head) {
  return __builtin_amdgcn_make_buffer_rsrc(a.scores + ((int64_t)row0 * a.num_kv_heads + head) * a.score_stride, 0,
                                           0x7FFFFFFF, 0x00020000);
}

// Decode steps: one wave a (row, kv head, every splits-th chunk of 64 blocks); the waves of a workgroup take
// neighbouring kv heads, whose bounds and units lie side by side.  A wave's bounds go through a ring of four
// steps of 16 blocks in LDS, three of them on their way while one is used, across its chunks; page ids and
// units come through LDS too, a chunk ahead (page ids: two).  Scores of blocks past the last are stored and
// never read (a row's scores have room for whole chunks).  HBM bounds it: 256 rows of 8 kv heads over contexts of
// 1k-32k, 582 MB of bounds, in 117 us, 5.0 TB/s.
// All waits in the loop are counted by hand, since the compiler waits for every load into LDS before a read of
// any: a step's read waits until at most kWait newer vector-memory operations are unfinished.  A chunk issues
//     U P F3 S0 F0 S1 F1 S2 F2 S3
// with U, P the units of the next chunk and the page ids of the one after it, F3 the last step's bounds, F0 ..
// F2 those of the next chunk's first steps (kLoads each) and S the steps' stores (kOut each); before the first
// chunk come U F0 F1 F2.  So what is issued behind F0 before its step is at least F1 F2 U P F3 (later chunks have
// stores between them); behind F1, F2 U P F3 S0 F0; behind F2, U P F3 S0 F0 S1 F1; behind F3, S0 F0 S1 F1 S2 F2;
// behind U and P before the next chunk begins, F0 F1 F2.  The order of an S and the F beside it is free.
// (256 rows of 8 heads, contexts of 1k-32k: 117 us with 4 waves a workgroup, 131 with 8, 120 with 2.)
constexpr int kRowWaves = 4;

// The operands of one step, read once all but kWait of the wave's vector-memory operations are done.
template <int kWait, int kOffset>
__device__ __forceinline__ void read_step(i32x4 (&b)[4], const uint32_t (&at)[4]) {
  asm volatile(
      "s_waitcnt vmcnt(%8)\n\t"
      "ds_read_b128 %0, %4 offset:%9\n\t"
      "ds_read_b128 %1, %5 offset:%9\n\t"
      "ds_read_b128 %2, %6 offset:%9\n\t"
      "ds_read_b128 %3, %7 offset:%9\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(b[0]), "=&v"(b[1]), "=&v"(b[2]), "=&v"(b[3])
      : "v"(at[0]), "v"(at[1]), "v"(at[2]), "v"(at[3]), "n"(kWait), "n"(kOffset)
      : "memory");
}

template <int kWait, int kOffset>
__device__ __forceinline__ void read_step(i32x4 (&b)[2], const uint32_t (&at)[2]) {
  asm volatile(
      "s_waitcnt vmcnt(%4)\n\t"
      "ds_read_b128 %0, %2 offset:%5\n\t"
      "ds_read_b128 %1, %3 offset:%5\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(b[0]), "=&v"(b[1])
      : "v"(at[0]), "v"(at[1]), "n"(kWait), "n"(kOffset)
      : "memory");
}

// Two words of the wave's page ids and units.
template <int kWait>
__device__ __forceinline__ void read_words(int32_t& x, int32_t& y, uint32_t at_x, uint32_t at_y) {
  asm volatile(
      "s_waitcnt vmcnt(%4)\n\t"
      "ds_read_b32 %0, %2\n\t"
      "ds_read_b32 %1, %3\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(x), "=&v"(y)
      : "v"(at_x), "v"(at_y), "n"(kWait)
      : "memory");
}

__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p;
}

template <int D, int kShift>
__global__ __launch_bounds__(kRowWaves * 64) __attribute__((amdgpu_waves_per_eu(2)))
void score_rows_kernel(BlockSelectArgs a) {
  using L = BoundsLds<D>;
  using O = ScoreOut<1, kShift>;
  constexpr int kC = D / 32, kRing = L::kBytes;  // from one step of a wave's ring to the next
  __shared__ __attribute__((aligned(1024))) uint8_t ring[kRowWaves * 4 * kRing];
  __shared__ __attribute__((aligned(1024))) int32_t words[2][2][kRowWaves][64];  // page ids, units; by the chunk's parity
  const int lane = threadIdx.x & 63, col = lane & 15, grp = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int Hkv = a.num_kv_heads;
  const uint32_t id = blockIdx.x * kRowWaves + wave;
  const int rest = (int)(id / (uint32_t)Hkv), head = (int)id - rest * Hkv;
  const int row = rest / a.splits, split = rest - row * a.splits;  // from first_row
  if (row >= a.rows) return;
  const int task = ((const const_i32*)a.row_task)[a.first_row + row], pos = ((const const_i32*)a.row_pos)[a.first_row + row];
  const int blocks = pos / kPage + 1, jump = a.splits * kScoreChunk;
  int b0 = split * kScoreChunk;
  // (a context within the budget is taken whole)
  if (!live_row(task, pos, a.num_tasks, a.max_len) || b0 >= blocks || blocks <= a.budget) return;
  const int32_t* table = a.block_table + (int64_t)task * a.bt_stride;
  const uint32_t pages = (uint32_t)min(a.num_pages, (int64_t)1 << 31);
  const uint32_t block_bytes = (uint32_t)Hkv * (2 * D);
  const int8_t* bounds = a.bounds + (int64_t)head * (2 * D);
  const int8_t* units = a.units + head;
  // lane i's page of block first + i, past the last block that one's again
  auto fetch_pages = [&](int first, int parity) {
    __builtin_amdgcn_global_load_lds((global_void*)(table + min(first + lane, blocks - 1)),
                                     (lds_void*)words[0][parity][wave], 4, 0, 0);
  };
  auto fetch_units = [&](int32_t page, int parity) {
    __builtin_amdgcn_global_load_lds((global_void*)(units + (int64_t)page * Hkv), (lds_void*)words[1][parity][wave], 1, 0, 0);
  };
  // bounds of blocks 16 step .. of a chunk; a bad page's are those of page 0, on which its score does not depend
  auto fetch = [&](int32_t page, int step) {
    uint8_t* to = ring + (4 * wave + step) * kRing;
#pragma unroll
    for (int i = 0; i < L::kLoads; ++i) {
      const uint32_t p = (uint32_t)__shfl(page, 16 * step + L::block(i), 64);
      __builtin_amdgcn_global_load_lds((global_void*)(bounds + (uint64_t)p * block_bytes + L::piece(i)),
                                       (lds_void*)(to + 1024 * i), 16, 0, kStreamPolicy);
    }
  };
  uint32_t at[kC], word_at[2];  // of words[0]; words[1] lies behind it
#pragma unroll
  for (int c = 0; c < kC; ++c) at[c] = lds_address(ring) + wave * 4 * kRing + L::offset(col, 4 * c + grp);
#pragma unroll
  for (int i = 0; i < 2; ++i) word_at[i] = lds_address(&words[0][i][wave][lane]);
  constexpr uint32_t kUnitsAt = sizeof(words[0]);

  fetch_pages(b0, 0);
  fetch_pages(b0 + jump, 1);
  QueryTile<D> q[1];
  const bool odd_rows = __any(!load_tile<D>(
      q[0], a.q + (((int64_t)a.first_row + row) * a.num_q_heads + head * a.group + min(col & ((1 << kShift) - 1), a.group - 1)) * D));
  const auto scores = score_rsrc(a, row, head);
  uint32_t put[O::kOut];
#pragma unroll
  for (int o = 0; o < O::kOut; ++o) put[o] = O::token_of(o, grp) == 0 && !O::repeats(grp) ? 4u * (uint32_t)col : kNowhere;

  bool flag_error = false;
  int32_t raw, other;
  read_words<0>(raw, other, word_at[0], word_at[0]);
  bool ok = (uint32_t)raw < pages;
  int32_t page = ok ? raw : 0;
  fetch_units(page, 0);
  fetch(page, 0);
  fetch(page, 1);
  fetch(page, 2);
  constexpr int kF = L::kLoads, kS = O::kOut;
  int parity = 0;
  for (; b0 < blocks; b0 += jump) {
    int32_t raw_next, s;
    read_words<3 * kF>(raw_next, s, parity ? word_at[0] : word_at[1], (parity ? word_at[1] : word_at[0]) + kUnitsAt);
    s = (int8_t)s;
    const bool ok_next = (uint32_t)raw_next < pages;
    const int32_t page_next = ok_next ? raw_next : 0;
    fetch_units(page_next, parity ^ 1);
    fetch_pages(b0 + 2 * jump, parity);
    flag_error |= !ok;
    bool odd;
    const BlockScale sc = block_scale(ok, s, odd_rows, &odd);
    i32x4 b[kC];
    auto step = [&](int i) {
      if (__builtin_expect(odd, 0)) score_step<D, 1, kShift, true>(q, b, sc, i, scores, put, b0 + 16 * i);
      else score_step<D, 1, kShift, false>(q, b, sc, i, scores, put, b0 + 16 * i);
    };
    fetch(page, 3);
    read_step<3 * kF + 2, 0>(b, at);
    step(0);
    fetch(page_next, 0);
    read_step<3 * kF + 2 + kS, kRing>(b, at);
    step(1);
    fetch(page_next, 1);
    read_step<3 * kF + 2 + 2 * kS, 2 * kRing>(b, at);
    step(2);
    fetch(page_next, 2);
    read_step<3 * kF + 3 * kS, 3 * kRing>(b, at);
    step(3);
    page = page_next;
    ok = ok_next;
    parity ^= 1;
  }
  if (flag_error) atomicOr(a.error_flags, 1);
  // the last loads into LDS are done before it is another workgroup's
  __atomic_signal_fence(__ATOMIC_SEQ_CST);
  __builtin_amdgcn_s_waitcnt(0);
}

// Several rows of most tasks: a workgroup takes the tile_rows rows of each of its waves, task by task (mostly one), and
// all of its waves use the chunk of 64 blocks that they bring into LDS together, the next one on its way.  A kv
// head's workgroups run on the same dies (workgroup b on die b % 8) where the number of kv heads lets them.
// Vector instructions (41% of SIMD cycles) and products (27%) bound it, while long tasks' workgroups last longest: 1,761 rows of 64 / 8 heads over 8 contexts of 32k-98k
// in 167 + 54 us, two rounds.  (302 us a call with the choice; 1,053 when each wave read operands of its own straight
// from memory and choices were made by the general way.)
constexpr int kChunkWaves = 4;

template <int D, int kShift>
__global__ __launch_bounds__(kChunkWaves * 64) __attribute__((amdgpu_waves_per_eu(2)))
void score_chunk_kernel(BlockSelectArgs a) {
  using L = BoundsLds<D>;
  using O = ScoreOut<kChunkTiles, kShift>;
  __shared__ __attribute__((aligned(1024))) uint8_t lds0[4 * L::kBytes];
  __shared__ __attribute__((aligned(1024))) uint8_t lds1[4 * L::kBytes];
  const int lane = threadIdx.x & 63, col = lane & 15, grp = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int Hkv = a.num_kv_heads;
  const int rest = blockIdx.x / Hkv, head = blockIdx.x - rest * Hkv;
  const int group = rest / a.splits, split = rest - group * a.splits;
  const int rows = a.tile_rows, first = group * kChunkWaves * rows;  // rows of a wave; of the workgroup, from first_row
  const int row0 = first + wave * rows;
  if (first >= a.rows) return;

  // lane i: row i of each wave's
  int their_task[kChunkWaves], their_pos[kChunkWaves];
  uint64_t left[kChunkWaves];
#pragma unroll
  for (int w = 0; w < kChunkWaves; ++w) {
    const int r = first + w * rows + lane;
    their_task[w] = -1, their_pos[w] = -1;
    if (lane < rows && r < a.rows) {
      their_task[w] = a.row_task[a.first_row + r];
      their_pos[w] = a.row_pos[a.first_row + r];
    }
    left[w] = __builtin_amdgcn_ballot_w64(live_row(their_task[w], their_pos[w], a.num_tasks, a.max_len));
  }
  QueryTile<D> q[kChunkTiles];
  bool near_one = true;
#pragma unroll
  for (int t = 0; t < kChunkTiles; ++t) {
    const int token = min(row0 + t * O::kTokens + (col >> kShift), a.rows - 1);
    const int h = min(col & ((1 << kShift) - 1), a.group - 1);
    near_one &= load_tile<D>(q[t], a.q + (((int64_t)a.first_row + token) * a.num_q_heads + head * a.group + h) * D);
  }
  const bool odd_rows = __any(!near_one);
  const auto scores = score_rsrc(a, min(row0, a.rows - 1), head);
  const uint32_t pages = (uint32_t)min(a.num_pages, (int64_t)1 << 31);
  const uint32_t block_bytes = (uint32_t)Hkv * (2 * D);
  const int8_t* bounds = a.bounds + (int64_t)head * (2 * D);
  bool flag_error = false;
  for (;;) {
    // the next task: that of the first row left; the same in every wave
    int task = -1;
#pragma unroll
    for (int w = kChunkWaves - 1; w >= 0; --w)
      if (left[w]) task = __builtin_amdgcn_readlane(their_task[w], __builtin_ctzll(left[w]));
    if (task < 0) break;
    uint64_t mine = 0;
    int last = 0, my_last = -1;
#pragma unroll
    for (int w = 0; w < kChunkWaves; ++w) {
      const uint64_t of = __builtin_amdgcn_ballot_w64(their_task[w] == task) & left[w];
      left[w] &= ~of;
      int top = (of >> lane) & 1 ? their_pos[w] : -1;
#pragma unroll
      for (int m = 1; m < 64; m *= 2) top = max(top, __shfl_xor(top, m, 64));
      last = max(last, top);
      if (w == wave) mine = of, my_last = top;
    }
    const int blocks = __builtin_amdgcn_readfirstlane(last) / kPage + 1;
    const int my_blocks = my_last < 0 ? 0 : __builtin_amdgcn_readfirstlane(my_last) / kPage + 1;
    uint32_t put[O::kOut];
#pragma unroll
    for (int o = 0; o < O::kOut; ++o) {
      const int u = O::token_of(o, grp);
      put[o] = u < rows && ((mine >> u) & 1)
                   ? 4u * ((uint32_t)u * (uint32_t)Hkv * (uint32_t)a.score_stride + (uint32_t)col) : kNowhere;
    }
    const int32_t* table = a.block_table + (int64_t)task * a.bt_stride;
    auto table_page = [&](int b) { return table[min(b + lane, blocks - 1)]; };
    // this wave's 16 blocks of a chunk
    auto fetch = [&](uint8_t* lds, int32_t page) {
      uint8_t* to = lds + wave * L::kBytes;
#pragma unroll
      for (int i = 0; i < L::kLoads; ++i) {
        const uint32_t p = (uint32_t)__shfl(page, 16 * wave + L::block(i), 64);
        __builtin_amdgcn_global_load_lds((global_void*)(bounds + (uint64_t)p * block_bytes + L::piece(i)),
                                         (lds_void*)(to + 1024 * i), 16, 0, kSharedPolicy);
      }
    };
    const int jump = a.splits * kScoreChunk;
    int b0 = split * kScoreChunk;
    if (b0 >= blocks) continue;
    int32_t raw = table_page(b0), raw_next = table_page(b0 + jump);
    bool ok = (uint32_t)raw < pages;
    int32_t page = ok ? raw : 0;
    int s = a.units[(int64_t)page * Hkv + head];
    fetch(lds0, page);
    auto round = [&](const uint8_t* now, uint8_t* next) {
      // every wave's part of `now` is there, and `next` has been read
      __atomic_signal_fence(__ATOMIC_SEQ_CST);
      __builtin_amdgcn_s_waitcnt(0);
      __builtin_amdgcn_s_barrier();
      __atomic_signal_fence(__ATOMIC_SEQ_CST);
      const bool ok_next = (uint32_t)raw_next < pages;
      const int32_t page_next = ok_next ? raw_next : 0;
      fetch(next, page_next);
      const int s_next = a.units[(int64_t)page_next * Hkv + head];
      raw_next = table_page(b0 + 2 * jump);
      flag_error |= !ok;
      bool odd;
      const BlockScale sc = block_scale(ok, s, odd_rows, &odd);
      if (b0 < my_blocks) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          i32x4 b[D / 32];
#pragma unroll
          for (int c = 0; c < D / 32; ++c)
            b[c] = *reinterpret_cast<const i32x4*>(now + i * L::kBytes + L::offset(col, 4 * c + grp));
          if (__builtin_expect(odd, 0))
            score_step<D, kChunkTiles, kShift, true>(q, b, sc, i, scores, put, b0 + 16 * i);
          else
            score_step<D, kChunkTiles, kShift, false>(q, b, sc, i, scores, put, b0 + 16 * i);
        }
      }
      page = page_next;
      ok = ok_next;
      s = s_next;
      b0 += jump;
    };
    for (;;) {
      round(lds0, lds1);
      if (b0 >= blocks) break;
      round(lds1, lds0);
      if (b0 >= blocks) break;
    }
    // the last load is done, and both buffers have been read
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    __builtin_amdgcn_s_waitcnt(0);
    __builtin_amdgcn_s_barrier();
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
  }
  if (flag_error) atomicOr(a.error_flags, 1);
}

// The least s with 2^s >= group.
int padded_shift(int32_t group) {
  int s = 0;
  while ((1 << s) < group) ++s;
  return s;
}

// ---- the choice ----------------------------------------------------------------------------------
// One workgroup of kT threads a (row, kv head).  The want-th largest of the maxima of four neighbours (quads) is
// at most the want-th largest score, so the quads that reach it hold all that is taken, and are few more than
// `want`: the others are looked at once.  Bins of equal width find it, and then the want-th largest score of the
// listed quads, with equal scores ranked by position; what is taken becomes bits, which are packed in order.
// Where the budget is above a quarter of the context all quads are listed.  What this does not fit (more than 256
// quads to list, infinite scores, more than 64 scores in the border's bin, contexts above 262,144) takes a way that
// any can go: bins of keys that narrow to the last key taken, and prefix sums over all.
constexpr int kChooseBins = 512;
constexpr int kChooseQuads = 256;  // of the list
constexpr int kChooseWords = 512;  // of bits
constexpr int kChooseSame = 64;    // scores of one bin that are ranked against each other
constexpr int kNoScore = INT32_MIN;  // in the place of a block that is not to be chosen from

template <int kT>
constexpr int kChooseHeld = kT == 128 ? 12 : 8;  // quads that a thread holds: contexts of 98,304 or 131,072

__device__ __forceinline__ uint32_t wave_sums(uint32_t x) {  // inclusive
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    const uint32_t y = __shfl_up((int)x, o, 64);
    if (lane >= o) x += y;
  }
  return x;
}

// Bins of equal width from `least` on, both finite.  (Rounded differences and products do not change the order.)
struct ScoreBins {
  float least, width;
  __device__ __forceinline__ ScoreBins(int low, int high)
      : least(score_of(low)), width(high > low ? (kChooseBins - 1) / (score_of(high) - score_of(low)) : 0.0f) {}
  __device__ __forceinline__ int operator()(int key) const {
    return min((int)fmaxf((score_of(key) - least) * width, 0.0f), kChooseBins - 1);
  }
  // a key that is at most every key of bin b: the bin's edge, less what the roundings of operator() are worth
  __device__ __forceinline__ int edge(int b) const {
    if (b == 0) return score_order(least);
    const float off = (float)b / width;
    return score_order(least + off - 0x1p-20f * (fabsf(least) + off));
  }
};

template <int kT>
__global__ __launch_bounds__(kT) __attribute__((amdgpu_waves_per_eu(4))) void choose_kernel(BlockSelectArgs a) {
  constexpr int kHeld = kChooseHeld<kT>, kWaves = kT / 64;
  __shared__ uint32_t hist[kChooseBins];
  __shared__ uint32_t bits[kChooseWords];
  __shared__ __attribute__((aligned(16))) i32x4 quad[kChooseQuads];
  __shared__ int quad_at[kChooseQuads];
  __shared__ int same_key[kChooseSame], same_at[kChooseSame], sames, quads;
  __shared__ uint32_t sums[4][kWaves];
  __shared__ int extreme[2][kWaves];
  __shared__ uint32_t found[3];  // bin, scores above it, scores in it
  __shared__ uint32_t range[2];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int nth = blockIdx.x / a.num_kv_heads, head = blockIdx.x - nth * a.num_kv_heads;
  const int64_t row = (int64_t)a.first_row + nth;
  const int32_t task = ((const const_i32*)a.row_task)[row], pos = ((const const_i32*)a.row_pos)[row];
  if (!live_row(task, pos, a.num_tasks, a.max_len)) return;
  int32_t* sel = a.sel + (row * a.num_kv_heads + head) * a.budget;
  const int blocks = pos / kPage + 1;
  if (blocks <= a.budget) {
    for (int i = tid; i < a.budget; i += kT) sel[i] = i < blocks ? i : -1;
    return;
  }
  const int want = a.budget - a.sink - a.recent, end = blocks - a.recent, n = end - a.sink;  // n > want >= 0
  for (int i = tid; i < a.sink; i += kT) sel[i] = i;
  for (int i = tid; i < a.recent; i += kT) sel[a.sink + want + i] = end + i;
  if (want == 0) return;
  const int32_t* score = a.scores + ((int64_t)nth * a.num_kv_heads + head) * a.score_stride;

  // the quad of blocks p .. p + 3  (a row's scores have room for whole chunks of 64)
  auto load4 = [&](int p) {
    i32x4 x = *reinterpret_cast<const i32x4*>(score + p);
    if (p < a.sink || p + 4 > end) {
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = p + i >= a.sink && p + i < end ? x[i] : kNoScore;
    }
    return x;
  };
  i32x4 held[kHeld];
#pragma unroll
  for (int c = 0; c < kHeld; ++c) {
    const int p = 4 * (tid + c * kT);
    held[c] = i32x4{kNoScore, kNoScore, kNoScore, kNoScore};
    if (4 * c * kT < end && p < end) held[c] = load4(p);
  }
  auto each4 = [&](auto&& f) {  // f(quad, first block), by all threads of the workgroup at once
#pragma unroll
    for (int c = 0; c < kHeld; ++c)
      if (4 * c * kT < end) f(held[c], 4 * (tid + c * kT));
    for (int c = kHeld; 4 * c * kT < end; ++c) {
      const int p = 4 * (tid + c * kT);
      f(p < end ? load4(p) : i32x4{kNoScore, kNoScore, kNoScore, kNoScore}, p);
    }
  };
  auto max4 = [](const i32x4& x) { return max(max(x[0], x[1]), max(x[2], x[3])); };
  auto clear_bins = [&]() {
#pragma unroll
    for (int i = 0; i < kChooseBins / kT; ++i) hist[tid + i * kT] = 0;
  };
  // exclusive sums over the workgroup's threads (one barrier; `sums` row k)
  auto block_sums = [&](uint32_t x, int k, uint32_t* all) {
    const uint32_t upto = wave_sums(x);
    if (lane == 63) sums[k][wave] = upto;
    __syncthreads();
    uint32_t before = upto - x, total = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      before += w < wave ? sums[k][w] : 0u;
      total += sums[k][w];
    }
    *all = total;
    return before;
  };
  // of the bins counted in hist the one that the rest-th largest lies in, to `found`
  auto find_bin = [&](uint32_t rest) __attribute__((always_inline)) {
    constexpr int kPer = kChooseBins / kT;
    uint32_t in[kPer], sum = 0, all;
#pragma unroll
    for (int i = 0; i < kPer; ++i) sum += in[i] = hist[kChooseBins - 1 - kPer * tid - i];
    uint32_t before = block_sums(sum, 0, &all);
    if (before < rest && before + sum >= rest) {
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        if (before < rest && before + in[i] >= rest)
          found[0] = kChooseBins - 1 - kPer * tid - i, found[1] = before, found[2] = in[i];
        before += in[i];
      }
    }
    __syncthreads();
  };

  clear_bins();
  const bool all_quads = n < 4 * want;  // then every quad is listed
  if (end <= 32 * kChooseWords && (!all_quads || end <= 4 * kChooseQuads)) {
    int low = INT32_MAX, high = INT32_MIN;  // of the quads' maxima, or of all scores
    each4([&](const i32x4& x, int) {
      const int m = max4(x);
      high = max(high, m);
      low = min(low, m == kNoScore ? INT32_MAX : m);
    });
    if (all_quads) {
      each4([&](const i32x4& x, int) {
#pragma unroll
        for (int i = 0; i < 4; ++i) low = min(low, x[i] == kNoScore ? INT32_MAX : x[i]);
      });
    }
#pragma unroll
    for (int m = 1; m < 64; m *= 2) {
      low = min(low, __shfl_xor(low, m, 64));
      high = max(high, __shfl_xor(high, m, 64));
    }
#pragma unroll
    for (int i = 0; i < kChooseWords / kT; ++i) bits[tid + i * kT] = 0;
    if (tid == 0) sames = quads = 0;
    if (lane == 0) extreme[0][wave] = low, extreme[1][wave] = high;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      low = min(low, extreme[0][w]);
      high = max(high, extreme[1][w]);
    }
    if (low > score_order(-INFINITY) && high < score_order(INFINITY)) {
      int least = low;
      if (!all_quads) {
        const ScoreBins coarse(low, high);
        each4([&](const i32x4& x, int) {
          const int m = max4(x);
          if (m != kNoScore) atomicAdd(&hist[coarse(m)], 1u);
        });
        __syncthreads();
        find_bin(want);
        least = coarse.edge((int)found[0]);
        clear_bins();
      }
      // the quads that reach it
      each4([&](const i32x4& x, int p) {
        const bool in = max4(x) >= least;
        const uint64_t who = __builtin_amdgcn_ballot_w64(in);
        int base = 0;
        if (lane == 0) base = atomicAdd(&quads, (int)__popcll(who));
        base = __builtin_amdgcn_readfirstlane(base);
        const int to = base + (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0));
        if (in && to < kChooseQuads) quad[to] = x, quad_at[to] = p;
      });
      __syncthreads();
      const int listed = quads;
      if (listed <= kChooseQuads) {
        const ScoreBins bin(least, high);
        const int* key_of = reinterpret_cast<const int*>(quad);
        for (int i = tid; i < 4 * listed; i += kT)
          if (key_of[i] >= least) atomicAdd(&hist[bin(key_of[i])], 1u);
        __syncthreads();
        find_bin(want);
        const int border = (int)found[0];
        const uint32_t rest = want - found[1], inside = found[2];
        const bool few = inside <= kChooseSame;
        if (few || inside == rest) {
          auto take = [&](int at) { atomicOr(&bits[at >> 5], 1u << (at & 31)); };
          for (int i = tid; i < 4 * listed; i += kT) {
            const int key = key_of[i], at = quad_at[i >> 2] + (i & 3);
            if (key < least) continue;
            const int b = bin(key);
            if (b > border || (b == border && inside == rest)) {
              take(at);
            } else if (b == border) {
              const int k = atomicAdd(&sames, 1);
              same_key[k] = key;
              same_at[k] = at;
            }
          }
          __syncthreads();
          if (inside > rest) {
            if (tid < (int)inside) {
              const int key = same_key[tid], at = same_at[tid];
              uint32_t before = 0;  // larger scores, and equal ones of earlier blocks
              for (uint32_t i = 0; i < inside; ++i)
                before += (same_key[i] > key) | ((same_key[i] == key) & (same_at[i] < at));
              if (before < rest) take(at);
            }
            __syncthreads();
          }
          const int words = (end + 31) / 32, per = (words + kT - 1) / kT, w0 = tid * per;
          uint32_t count = 0, all;
          for (int w = w0; w < min(words, w0 + per); ++w) count += __popc(bits[w]);
          int32_t* out = sel + a.sink + block_sums(count, 1, &all);
          for (int w = w0; w < min(words, w0 + per); ++w)
            for (uint32_t left = bits[w]; left; left &= left - 1) *out++ = 32 * w + __builtin_ctz(left);
          return;
        }
      }
    }
    __syncthreads();
  }

  // Bins of keys over the range that the keys in question cover, until one key is left: `rest` of it are taken.
  int low = INT32_MIN + 1, high = INT32_MAX;  // (kNoScore is below)
  uint32_t rest = want;
  auto each_key = [&](auto&& f) {
    each4([&](const i32x4& x, int) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (x[i] >= low && x[i] <= high) f(x[i]);
    });
  };
  auto up = [](int key) { return (uint32_t)key ^ 0x80000000u; };
  for (;;) {
    if (tid == 0) range[0] = 0xFFFFFFFFu, range[1] = 0;
    clear_bins();
    __syncthreads();
    int kmin = INT32_MAX, kmax = INT32_MIN;
    each_key([&](int key) { kmin = min(kmin, key), kmax = max(kmax, key); });
    atomicMin(&range[0], up(kmin));
    atomicMax(&range[1], up(kmax));
    __syncthreads();
    low = (int)up((int)range[0]), high = (int)up((int)range[1]);
    if (low == high) break;
    const uint32_t span = (uint32_t)high - (uint32_t)low;
    const int shift = max(0, 32 - __builtin_clz(span) - 9);  // bins of 2^shift keys
    each_key([&](int key) { atomicAdd(&hist[((uint32_t)key - (uint32_t)low) >> shift], 1u); });
    __syncthreads();
    find_bin(rest);
    rest -= found[1];
    const uint32_t first = found[0] << shift;  // from `low` on
    high = (int)((uint32_t)low + min(span, first + ((1u << shift) - 1)));
    low = (int)((uint32_t)low + first);
    __syncthreads();
  }
  // What is taken, in order: larger keys, and the first `rest` equal ones.
  uint32_t placed = 0, met = 0;
  for (int c = 0; 4 * c * kT < end; ++c) {
    const int p = 4 * (tid + c * kT);
    i32x4 x = {kNoScore, kNoScore, kNoScore, kNoScore};
    if (p < end) x = load4(p);
    uint32_t flags = 0, all;  // larger keys in the lower half, equal ones in the upper
#pragma unroll
    for (int i = 0; i < 4; ++i) flags += x[i] > low ? 1u : x[i] == low ? 0x10000u : 0u;
    const uint32_t before = block_sums(flags, c & 3, &all);
    uint32_t ge = placed + (before & 0xFFFF), eq = met + (before >> 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (x[i] > low || (x[i] == low && eq < rest)) sel[a.sink + ge + min(eq, rest)] = p + i;
      ge += x[i] > low;
      eq += x[i] == low;
    }
    placed += all & 0xFFFF;
    met += all >> 16;
  }
}

template <int D, int kShift>
void launch_scores(const BlockSelectArgs& a, hipStream_t stream) {
  const int64_t heads = (int64_t)a.splits * a.num_kv_heads;
  if (a.tile_rows == 1) {
    const uint32_t blocks = (uint32_t)((a.rows * heads + kRowWaves - 1) / kRowWaves);
    hipLaunchKernelGGL((score_rows_kernel<D, kShift>), dim3(blocks), dim3(kRowWaves * 64), 0, stream, a);
  } else {
    const int per = kChunkWaves * a.tile_rows;
    const uint32_t blocks = (uint32_t)((a.rows + per - 1) / per * heads);
    hipLaunchKernelGGL((score_chunk_kernel<D, kShift>), dim3(blocks), dim3(kChunkWaves * 64), 0, stream, a);
  }
}

template <int D>
hipError_t launch_scores(const BlockSelectArgs& a, hipStream_t stream) {
  switch (padded_shift(a.group)) {
    case 0: launch_scores<D, 0>(a, stream); break;
    case 1: launch_scores<D, 1>(a, stream); break;
    case 2: launch_scores<D, 2>(a, stream); break;
    case 3: launch_scores<D, 3>(a, stream); break;
    default: launch_scores<D, 4>(a, stream); break;
  }
  return hipGetLastError();
}

}  // namespace kern

int select_tile_rows(int32_t group, bool chunk) {
  return chunk ? kern::kChunkTiles * (16 >> kern::padded_shift(group)) : 1;
}

// Up to this many (row, kv head) pairs take four waves each, more two: 16 pairs, contexts of 2k-16k, 5.6 us with four
// waves, 7.2 with two, 9.5 with one; 14,000 pairs, contexts of 32k-98k, 175, 78 and 86 us; calls of 1,024 pairs, scores and
// choice, 48.4 and 48.5 us with four and two, of 2,048 pairs 85.6 and 82.3.
constexpr uint32_t kChooseWide = 1024;

hipError_t launch_block_select(const BlockSelectArgs& a, int head_dim, hipStream_t stream) {
  // (a context within the budget has nothing to choose: no scores are read)
  hipError_t rc = hipSuccess;
  if ((a.max_len - 1) / kPage + 1 > a.budget && a.budget > a.sink + a.recent)
    rc = head_dim == 128 ? kern::launch_scores<128>(a, stream) : kern::launch_scores<64>(a, stream);
  if (rc != hipSuccess) return rc;
  const uint32_t pairs = (uint32_t)(a.rows * a.num_kv_heads);
  if (pairs > kChooseWide)
    hipLaunchKernelGGL((kern::choose_kernel<128>), dim3(pairs), dim3(128), 0, stream, a);
  else
    hipLaunchKernelGGL((kern::choose_kernel<256>), dim3(pairs), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace tide
