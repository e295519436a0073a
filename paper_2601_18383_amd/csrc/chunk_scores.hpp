// The attention weight that every cached slot receives from a chunk's queries (Eq. importance-score for a block of queries that are part of
// the cache): S_j += sum over the rows r that see slot j of 2^(x_rj - L_r), with the logits of chunk_attend.hpp and their
// log-sum-exp L_r.
//
// Keys are the stationary operand (B: 64 slots a wave), query rows stream through LDS 32 at a time (A), so that a lane holds 16
// rows of one slot, adds them up by itself, and joins the other half once, at the end: no atomics, one order.  What a row sees, and its L, are
// looked up a group of 256 rows ahead, one row a thread.  Chunks of rows that all see all of a wave's keys skip the comparisons,
// those that see none skip the products.
//
// Bound by instruction issue (one exponential a 256 operations, twice the density of the attention) and the clock: 512 tokens of 32 sequences on 2464
// slots, 28 heads on 4 of 128, 320 GFLOP in 347 us; the matrix cores are busy 43 % of the cycles, the vector units 59 %.  Two chunks a
// barrier: 343 us instead of 353 with one; with a bias, where registers are short, 263 with one instead of 278 (16 of these sequences).  Rows' addresses
// stepped instead of computed: 1 % faster for 6 registers, left out.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "chunk_attend.hpp"

namespace dynts {

struct ChunkScoreParams {
  ChunkCache c;
  const uint16_t *q;     // [Nb][T][Hq][D]
  const int32_t *n_new;  // [Nb] or null: T
  const float *lse;      // [Nb][T][Hq]
  float *dst;            // [Nb][Hkv][cap]
  ChunkShape shape;
  int T;
  int skip_question;     // slots below n_prompt are left alone
  int accumulate;
  float scale_log2;
  uint32_t g_magic;      // as in ChunkAttendParams
};

constexpr int kCsKeys = kSbRowsPerWg;  // slots a workgroup
constexpr int kCsGroup = kSbLRows, kCsPer = kCsGroup / kSbChunk;  // rows looked up at a time; chunks of them

// of a group's rows: minus their L, and what they see: the last slot, or shaped the lowest position, the distance to the highest, their own, their slope
template <bool SHAPED, bool BIASED, int ROWS>
struct ChunkRows {
  float minus_l[ROWS];
  int lo[ROWS];
  uint32_t span[SHAPED ? ROWS : 1];
  int own[BIASED ? ROWS : 1];
  float slope[BIASED ? ROWS : 1];
  // by chunk, shaped: what all of its rows see, what any does
  int all_lo[ROWS / kSbChunk], all_hi[ROWS / kSbChunk], any_lo[ROWS / kSbChunk], any_hi[ROWS / kSbChunk];
};

// What a row adds to its logits: minus its lse, in log2 units.  A row that has seen a NaN, whose lse is one, gives NaN to all slots that it sees and nothing to the
// others: hidden logits are -inf, which a NaN added to them would not leave, so it adds what takes every other weight to infinity (v_min_f32 of a NaN and a number is
// the number), and a sum that is infinite, of weights of 1 at most, is NaN.  (A row without a key it sees, whose lse is -inf, adds the same to nothing but -inf.)
constexpr float kNanRow = 3e38f;
__device__ __forceinline__ float row_addend(float lse) { return fminf(lse * -1.4426950408889634f, kNanRow); }
// (by its bits, and the number out of the compiler's sight: to it floats are never NaN)
__device__ __forceinline__ float received(float sum) {
  uint32_t nan = 0x7fc00000u;
  asm("" : "+v"(nan));
  return __uint_as_float(__float_as_uint(sum) == 0x7f800000u ? nan : __float_as_uint(sum));
}

// One row of a unit a thread: fetched, then put among the others' (32 neighbouring threads have a chunk).
template <bool SHAPED>
struct ChunkRow {
  float l;
  int own, first, last, r;
};
template <bool SHAPED>
__device__ __forceinline__ void chunk_fetch_row(ChunkRow<SHAPED> &row, const ChunkScoreParams &p, const int32_t *pos, int b, int h, int R, int base, int r) {
  row.r = r;
  r = r < R ? r : R - 1;
  const int i = chunk_token(r, p.g_magic);
  const size_t at = (size_t)b * p.T + i;
  row.l = p.lse[at * p.c.Hq + (size_t)h * p.c.G + (r - i * p.c.G)];
  if (SHAPED) {
    row.own = pos[base + i];
    if (p.shape.first) row.first = p.shape.first[at];
    if (p.shape.last) row.last = p.shape.last[at];
  }
}
template <bool SHAPED, bool BIASED, int ROWS>
__device__ __forceinline__ void chunk_put_row(ChunkRows<SHAPED, BIASED, ROWS> &rows, const ChunkRow<SHAPED> &row, const ChunkScoreParams &p, int h, int R,
                                              int base, int at) {
  const bool real = row.r < R;
  const int r = real ? row.r : R - 1, i = chunk_token(r, p.g_magic);
  rows.minus_l[at] = row_addend(row.l);  // (rows behind the last see nothing)
  if (SHAPED) {
    int lo;
    uint32_t span;
    chunk_bounds(p.shape, row.first, row.last, row.own, lo, span);
    if (!real) {
      lo = kNowhere;
      span = 0;
    }
    rows.lo[at] = lo;
    rows.span[at] = span;
    if (BIASED) {
      rows.own[at] = row.own;
      rows.slope[at] = p.shape.slope[h * p.c.G + (r - i * p.c.G)] * 1.4426950408889634f;
    }
    const int hi = lo == kNowhere ? -1 : (int)(lo + span);
    int all_lo = lo, all_hi = hi, any_lo = lo, any_hi = hi;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const int al = __shfl_xor(all_lo, d), ah = __shfl_xor(all_hi, d), nl = __shfl_xor(any_lo, d), nh = __shfl_xor(any_hi, d);
      all_lo = al > all_lo ? al : all_lo;
      all_hi = ah < all_hi ? ah : all_hi;
      any_lo = nl < any_lo ? nl : any_lo;
      any_hi = nh > any_hi ? nh : any_hi;
    }
    if (at % kSbChunk == 0) {
      rows.all_lo[at / kSbChunk] = all_lo;
      rows.all_hi[at / kSbChunk] = all_hi;
      rows.any_lo[at / kSbChunk] = any_lo;
      rows.any_hi[at / kSbChunk] = any_hi;
    }
  } else {
    rows.lo[at] = real ? base + i : -1;
  }
}

// Whether some, and whether all of the rows of chunk `ch` (from row r0 of `rows` on) see keys k_first to k_last.
template <bool SHAPED, bool BIASED, int ROWS>
__device__ __forceinline__ void chunk_sees(const ChunkRows<SHAPED, BIASED, ROWS> &rows, const ChunkScoreParams &p, int ch, int part, int R, int base, int k_first,
                                           int k_last, bool &any, bool &all) {
  if (SHAPED) {
    any = __builtin_amdgcn_readfirstlane(rows.any_lo[part]) <= k_last && __builtin_amdgcn_readfirstlane(rows.any_hi[part]) >= k_first;
    all = __builtin_amdgcn_readfirstlane(rows.all_lo[part]) <= k_first && __builtin_amdgcn_readfirstlane(rows.all_hi[part]) >= k_last;
  } else {
    const int last = (ch + 1) * kSbChunk - 1;
    any = base + chunk_token(last < R ? last : R - 1, p.g_magic) >= k_first;
    all = last < R && base + chunk_token(ch * kSbChunk, p.g_magic) >= k_last;
  }
}

// The weights of a chunk's products, added to the lane's sums.  r0: the chunk's first row among `rows`.  FAR: as in soft_caps.
template <bool FAR, bool SHAPED, bool BIASED, int ROWS>
__device__ __forceinline__ void chunk_add(float (&sum)[kSbTiles], f32x16 (&acc)[kSbTiles], const ChunkRows<SHAPED, BIASED, ROWS> &rows, const ChunkScoreParams &p,
                                          const int (&kpos)[kSbTiles], int r0, bool all, int hf) {
  f32x4 ml[4];  // of the rows 8 j + 4 hf .. +3 that this lane's products belong to
#pragma unroll
  for (int j = 0; j < 4; ++j) ml[j] = *reinterpret_cast<const f32x4 *>(&rows.minus_l[r0 + 8 * j + 4 * hf]);
  float scale = p.scale_log2;
  if (SHAPED && p.shape.cap > 0.f) {
    scale = 1.f;
#pragma unroll
    for (int kt = 0; kt < kSbTiles; ++kt) soft_caps<FAR>(acc[kt], p.scale_log2, p.shape);
  }
  if (BIASED) {
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int r = r0 + 8 * (e >> 2) + 4 * hf + (e & 3), own = rows.own[BIASED ? r : 0];
      const float slope = rows.slope[BIASED ? r : 0];
#pragma unroll
      for (int kt = 0; kt < kSbTiles; ++kt) acc[kt][e] = fmaf(-slope, fabsf((float)(own - kpos[kt])), acc[kt][e] * scale);
    }
    scale = 1.f;
  }
  if (!all) {
    asm volatile("; some keys are hidden");  // (a branch: the compiler would compare every key of every chunk)
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int r = r0 + 8 * (e >> 2) + 4 * hf + (e & 3), lo = rows.lo[r];
#pragma unroll
      for (int kt = 0; kt < kSbTiles; ++kt) {
        const bool seen = SHAPED ? (uint32_t)(kpos[kt] - lo) <= rows.span[SHAPED ? r : 0] : kpos[kt] <= lo;
        if (!seen) acc[kt][e] = -INFINITY;
      }
    }
  }
#pragma unroll
  for (int kt = 0; kt < kSbTiles; ++kt) sum[kt] += sb_exp_sum(acc[kt], scale, [&](int e) { return ml[e >> 2][e & 3]; });
}

// A wave's keys, 64 from key0 on, as stationary operands.
template <int D, bool SHAPED, int CODE>
__device__ __forceinline__ void chunk_keys(bf16x8 (&kf)[kSbTiles][D / 16], int (&kpos)[kSbTiles], const ChunkCache &c, const int32_t *pos, int unit, int n,
                                           int key0, int col, int hf) {
#pragma unroll
  for (int kt = 0; kt < kSbTiles; ++kt) {
    int slot = key0 + 32 * kt + col;
    slot = slot < n ? slot : n - 1;
    const size_t row = c.block_table ? paged_row<D>(c.block_table + (size_t)unit * c.max_pages, slot, c.max_pages, c.n_pages)
                                     : ((size_t)unit * c.cap + slot) * D;
    if (CODE) decode_row_frags<D, CODE>(kf[kt], reinterpret_cast<const uint8_t *>(c.K) + row, c.K_scale + row / kCodeBlock, hf);
    else load_row_frags<D>(kf[kt], reinterpret_cast<const char *>(c.K + row), hf);
    kpos[kt] = SHAPED ? pos[slot] : slot;
  }
}

// 1-D grid of ceil(cap / 256) * round_up(units, 8) workgroups, 256 threads.
// SHAPED, BIASED as in chunk_attend_kernel.
// CODE: the cache holds codes, which become bf16 as the keys are loaded.
template <int D, bool SHAPED, bool BIASED, int CODE>
__device__ __forceinline__ void chunk_scores(const ChunkScoreParams &p) {
  using St = SbStage<D>;
  const ChunkCache &c = p.c;
  constexpr int kCsStage = BIASED && D == 128 ? 1 : 2;  // chunks staged at a time, one barrier for all
  __shared__ __attribute__((aligned(16))) char sm_q[2][kCsStage * St::kBufBytes];
  __shared__ __attribute__((aligned(16))) ChunkRows<SHAPED, BIASED, kCsGroup> sm_rows[2];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 31, hf = lane >> 5;
  int unit, blk;
  if (!chunk_map(kAllUnits, (c.cap + kCsKeys - 1) / kCsKeys, c.Nb * c.Hkv, unit, blk)) return;
  const int b = unit / c.Hkv, h = unit - b * c.Hkv;
  int n;
  const int m = chunk_tokens(c, p.n_new, p.T, b, n);
  if (m == 0) return;
  int skip = p.skip_question ? c.n_prompt[b] : 0;
  skip = skip < 0 ? 0 : skip;
  if (blk * kCsKeys >= n || (blk + 1) * kCsKeys <= skip) return;
  const int R = m * c.G, base = n - m;
  const int key0 = blk * kCsKeys + wave * kSbRowsPerWave;
  const int32_t *pos = c.pos + (size_t)unit * c.cap;

  bf16x8 kf[kSbTiles][D / 16];
  int kpos[kSbTiles];  // of the lane's keys: slot, or shaped position
  float sum[kSbTiles] = {};
  chunk_keys<D, SHAPED, CODE>(kf, kpos, c, pos, unit, n, key0, col, hf);
  const bool has_keys = key0 < n && key0 + kSbRowsPerWave > skip;  // else: staging and barriers only
  const int k_first = __builtin_amdgcn_readfirstlane(kpos[0]), k_last = __shfl(kpos[kSbTiles - 1], 31);

  // staging: eight threads a row, 128 bytes apart
  const int st_row = tid >> 3;
  const uint32_t st_piece = 16u * (uint32_t)(tid & 7);
  char *const park = sm_q[0] + st_row * St::LROW + st_piece;
  u32x4 stage[kCsStage][St::NL];
  auto row_of = [&](int r) {
    r = r < R ? r : R - 1;
    const int i = chunk_token(r, p.g_magic);
    return ((size_t)b * p.T + i) * c.Hq + (size_t)h * c.G + (r - i * c.G);
  };
  auto fetch = [&](int ch) {
#pragma unroll
    for (int x = 0; x < kCsStage; ++x) {
      const char *src = reinterpret_cast<const char *>(p.q + row_of((ch + x) * kSbChunk + st_row) * D) + st_piece;
#pragma unroll
      for (int k = 0; k < St::NL; ++k) stage[x][k] = *reinterpret_cast<const u32x4 *>(src + 128 * k);
    }
  };
  auto put = [&](int buf) {
#pragma unroll
    for (int x = 0; x < kCsStage; ++x)
#pragma unroll
      for (int k = 0; k < St::NL; ++k) *reinterpret_cast<u32x4 *>(park + (buf * kCsStage + x) * St::kBufBytes + 128 * k) = stage[x][k];
  };
  // one row a thread, of the group that begins with row r0
  ChunkRow<SHAPED> mine{};
  auto fetch_rows = [&](int r0) { chunk_fetch_row(mine, p, pos, b, h, R, base, r0 + tid); };
  auto put_rows = [&](int buf) { chunk_put_row(sm_rows[buf], mine, p, h, R, base, tid); };

  // (plain, and shaped without `last`: rows whose own slot lies before all of these keys see none of them)
  const int i0 = (SHAPED && p.shape.last) || blk * kCsKeys <= base ? 0 : blk * kCsKeys - base;
  const int first = i0 * c.G / kCsGroup * kCsPer, chunks = (R + kSbChunk - 1) / kSbChunk;  // (from a whole group on)
  if (first < chunks) {
    fetch_rows(first * kSbChunk);
    fetch(first);
    put(0);
    put_rows(0);
    if (first + kCsStage < chunks) fetch(first + kCsStage);
  }
  // a chunk whose rows are in `q`, and what is known of them from row r0 of `rows` on
  auto chunk = [&](int ch, const char *q, const ChunkRows<SHAPED, BIASED, kCsGroup> &rows) {
    const int in_group = (ch - first) % kCsPer;
    bool any, all;
    chunk_sees(rows, p, ch, in_group, R, base, k_first, k_last, any, all);
    if (__builtin_amdgcn_readfirstlane((int)(any && has_keys))) {
      f32x16 acc[kSbTiles];
      sb_multiply<D>(acc, q, kf, col, hf);
      chunk_add<false>(sum, acc, rows, p, kpos, in_group * kSbChunk, __builtin_amdgcn_readfirstlane((int)all), hf);
    }
  };
  int buf = 0;
  for (int ch = first; ch < chunks; ch += kCsStage) {
    __syncthreads();
    if (ch + kCsStage < chunks) put(buf ^ 1);
    if (ch + 2 * kCsStage < chunks) fetch(ch + 2 * kCsStage);
    const int in_group = (ch - first) % kCsPer, group = (ch - first) / kCsPer;
    if (in_group == 0 && ch + kCsPer < chunks) fetch_rows((ch + kCsPer) * kSbChunk);
    if (in_group == kCsPer - kCsStage && ch + kCsStage < chunks) put_rows((group + 1) & 1);
#pragma unroll
    for (int x = 0; x < kCsStage; ++x)
      if (ch + x < chunks) chunk(ch + x, sm_q[buf] + x * St::kBufBytes, sm_rows[group & 1]);
    buf ^= 1;
  }
  if (!has_keys) return;
  float tot[kSbTiles];
#pragma unroll
  for (int kt = 0; kt < kSbTiles; ++kt) tot[kt] = sum[kt] + __shfl_xor(sum[kt], 32);
  const float v = received(hf == 0 ? tot[0] : tot[1]);
  const int slot = key0 + 32 * hf + col;
  if (slot < n && slot >= skip) {
    float *d = p.dst + (size_t)unit * c.cap + slot;
    *d = p.accumulate ? *d + v : v;
  }
}

template <int D, bool SHAPED, bool BIASED>
__global__ __launch_bounds__(kSbWaves * 64, D == 128 || SHAPED ? 3 : 4) void chunk_scores_kernel(const ChunkScoreParams p) {
  chunk_scores<D, SHAPED, BIASED, 0>(p);
}
template <int D, bool SHAPED, bool BIASED, int CODE>
__global__ __launch_bounds__(kSbWaves * 64, D == 128 || SHAPED ? 3 : 4) void coded_scores_kernel(const ChunkScoreParams p) {
  chunk_scores<D, SHAPED, BIASED, CODE>(p);
}

// ---- few keys: 64 of them a workgroup, its eight waves share out the rows ----------------------------------------------------
// For few units on short caches, where workgroups of 256 slots would leave compute units without work and every wave with all of the rows.  A wave takes
// every eighth chunk straight from global memory, the next one's on its way while it works on one, no barrier before the end; there the waves' sums
// are added up in their order.  Bound by the latency of a wave's chain, 1 to 2 us a chunk: 328 tokens of 13 sequences, 16 heads on 1 of 64, 23 us (the kernel
// above 128).
constexpr int kCfWaves = 8, kCfKeys = 64;
template <int D, bool SHAPED, bool BIASED, int CODE>
__device__ __forceinline__ void chunk_scores_few(const ChunkScoreParams &p) {
  const ChunkCache &c = p.c;
  __shared__ __attribute__((aligned(16))) ChunkRows<SHAPED, BIASED, kSbChunk> sm_rows[kCfWaves];
  __shared__ float sm_sum[kCfWaves][kCfKeys];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 31, hf = lane >> 5;
  int unit, blk;
  if (!chunk_map(1, (c.cap + kCfKeys - 1) / kCfKeys, c.Nb * c.Hkv, unit, blk)) return;
  const int b = unit / c.Hkv, h = unit - b * c.Hkv;
  int n;
  const int m = chunk_tokens(c, p.n_new, p.T, b, n);
  if (m == 0) return;
  int skip = p.skip_question ? c.n_prompt[b] : 0;
  skip = skip < 0 ? 0 : skip;
  const int key0 = blk * kCfKeys;
  if (key0 >= n || key0 + kCfKeys <= skip) return;
  const int R = m * c.G, base = n - m;
  const int32_t *pos = c.pos + (size_t)unit * c.cap;

  bf16x8 kf[kSbTiles][D / 16];
  int kpos[kSbTiles];
  float sum[kSbTiles] = {};
  chunk_keys<D, SHAPED, CODE>(kf, kpos, c, pos, unit, n, key0, col, hf);
  const int k_first = __builtin_amdgcn_readfirstlane(kpos[0]), k_last = __shfl(kpos[kSbTiles - 1], 31);

  const int i0 = (SHAPED && p.shape.last) || key0 <= base ? 0 : key0 - base;  // (as above)
  const int chunks = (R + kSbChunk - 1) / kSbChunk;
  ChunkRow<SHAPED> mine{};
  auto fetch = [&](int ch, bf16x8 (&a)[D / 16]) {
    int r = ch * kSbChunk + col;
    r = r < R ? r : R - 1;
    const int i = chunk_token(r, p.g_magic);
    load_row_frags<D>(a, reinterpret_cast<const char *>(p.q + (((size_t)b * p.T + i) * c.Hq + (size_t)h * c.G + (r - i * c.G)) * D), hf);
  };
  ChunkRows<SHAPED, BIASED, kSbChunk> &rows = sm_rows[wave];
  // the chunk in `a`; the one after it goes to `next`
  auto chunk = [&](int ch, const bf16x8 (&a)[D / 16], bf16x8 (&next)[D / 16]) {
    chunk_put_row(rows, mine, p, h, R, base, col);
    if (ch + kCfWaves < chunks) {
      fetch(ch + kCfWaves, next);
      chunk_fetch_row(mine, p, pos, b, h, R, base, (ch + kCfWaves) * kSbChunk + col);
    }
    wave_lds_fence();
    bool any, all;
    chunk_sees(rows, p, ch, 0, R, base, k_first, k_last, any, all);
    if (__builtin_amdgcn_readfirstlane((int)any)) {
      f32x16 acc[kSbTiles];
#pragma unroll
      for (int kt = 0; kt < kSbTiles; ++kt)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[kt][e] = 0.f;
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
        for (int kt = 0; kt < kSbTiles; ++kt) acc[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[ks], kf[kt][ks], acc[kt], 0, 0, 0);
      chunk_add<true>(sum, acc, rows, p, kpos, 0, __builtin_amdgcn_readfirstlane((int)all), hf);
    }
    wave_lds_fence();
  };
  bf16x8 a0[D / 16], a1[D / 16];
  int ch = i0 * c.G / kSbChunk + wave;
  if (ch < chunks) {
    fetch(ch, a0);
    chunk_fetch_row(mine, p, pos, b, h, R, base, ch * kSbChunk + col);
  }
  for (; ch < chunks; ch += 2 * kCfWaves) {
    chunk(ch, a0, a1);
    if (ch + kCfWaves < chunks) chunk(ch + kCfWaves, a1, a0);
  }
  float tot[kSbTiles];
#pragma unroll
  for (int kt = 0; kt < kSbTiles; ++kt) tot[kt] = sum[kt] + __shfl_xor(sum[kt], 32);
  sm_sum[wave][lane] = hf == 0 ? tot[0] : tot[1];
  __syncthreads();
  const int slot = key0 + lane;
  if (wave == 0 && slot < n && slot >= skip) {
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < kCfWaves; ++w) v += sm_sum[w][lane];
    v = received(v);
    float *d = p.dst + (size_t)unit * c.cap + slot;
    *d = p.accumulate ? *d + v : v;
  }
}

template <int D, bool SHAPED, bool BIASED>
__global__ __launch_bounds__(kCfWaves * 64, 2) void chunk_scores_few_kernel(const ChunkScoreParams p) {
  chunk_scores_few<D, SHAPED, BIASED, 0>(p);
}
template <int D, bool SHAPED, bool BIASED, int CODE>
__global__ __launch_bounds__(kCfWaves * 64, 2) void coded_scores_few_kernel(const ChunkScoreParams p) {
  chunk_scores_few<D, SHAPED, BIASED, CODE>(p);
}

}  // namespace dynts
