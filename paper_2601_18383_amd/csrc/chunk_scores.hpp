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
// slots, 28 heads on 4 of 128, 320 GFLOP in 347 us; the matrix cores are busy 37 % of the cycles, the vector units 51 %.  Two chunks a
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
template <bool SHAPED, bool BIASED>
struct ChunkRows {
  float minus_l[kCsGroup];
  int lo[kCsGroup];
  uint32_t span[SHAPED ? kCsGroup : 1];
  int own[BIASED ? kCsGroup : 1];
  float slope[BIASED ? kCsGroup : 1];
  // by chunk, shaped: what all of its rows see, what any does
  int all_lo[kCsPer], all_hi[kCsPer], any_lo[kCsPer], any_hi[kCsPer];
};

// 1-D grid of ceil(cap / 256) * round_up(units, 8) workgroups, 256 threads.
// SHAPED, BIASED as in chunk_attend_kernel.
template <int D, bool SHAPED, bool BIASED>
__global__ __launch_bounds__(kSbWaves * 64, D == 128 || SHAPED ? 3 : 4) void chunk_scores_kernel(const ChunkScoreParams p) {
  using St = SbStage<D>;
  const ChunkCache &c = p.c;
  constexpr int kCsStage = BIASED && D == 128 ? 1 : 2;  // chunks staged at a time, one barrier for all
  __shared__ __attribute__((aligned(16))) char sm_q[2][kCsStage * St::kBufBytes];
  __shared__ __attribute__((aligned(16))) ChunkRows<SHAPED, BIASED> sm_rows[2];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 31, hf = lane >> 5;
  int unit, blk;
  if (!sb_map((c.cap + kCsKeys - 1) / kCsKeys, c.Nb * c.Hkv, unit, blk)) return;
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
  float sum[kSbTiles];
#pragma unroll
  for (int kt = 0; kt < kSbTiles; ++kt) {
    int slot = key0 + 32 * kt + col;
    slot = slot < n ? slot : n - 1;
    const size_t row = c.block_table ? paged_row<D>(c.block_table + (size_t)unit * c.max_pages, slot, c.max_pages, c.n_pages)
                                     : ((size_t)unit * c.cap + slot) * D;
    load_row_frags<D>(kf[kt], reinterpret_cast<const char *>(c.K + row), hf);
    kpos[kt] = SHAPED ? pos[slot] : slot;
    sum[kt] = 0.f;
  }
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
  float row_l = 0.f;
  int row_own = 0, row_first = 0, row_last = 0, row_r = 0;
  auto fetch_rows = [&](int r0) {
    row_r = r0 + tid;
    row_l = p.lse[row_of(row_r)];
    if (SHAPED) {
      const int i = chunk_token(row_r < R ? row_r : R - 1, p.g_magic);
      const size_t at = (size_t)b * p.T + i;
      row_own = pos[base + i];
      if (p.shape.first) row_first = p.shape.first[at];
      if (p.shape.last) row_last = p.shape.last[at];
    }
  };
  auto put_rows = [&](int buf) {
    ChunkRows<SHAPED, BIASED> &rows = sm_rows[buf];
    const bool real = row_r < R;
    const int r = real ? row_r : R - 1, i = chunk_token(r, p.g_magic);
    // (a row without a key it sees has no weights: its comparisons say so.  Rows behind the last see nothing)
    rows.minus_l[tid] = row_l == -INFINITY ? 0.f : row_l * -1.4426950408889634f;
    if (SHAPED) {
      int lo;
      uint32_t span;
      chunk_bounds(p.shape, row_first, row_last, row_own, lo, span);
      if (!real) {
        lo = kNowhere;
        span = 0;
      }
      rows.lo[tid] = lo;
      rows.span[tid] = span;
      if (BIASED) {
        rows.own[tid] = row_own;
        rows.slope[tid] = p.shape.slope[h * c.G + (r - i * c.G)] * 1.4426950408889634f;
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
      if (col == 0) {
        rows.all_lo[tid >> 5] = all_lo;
        rows.all_hi[tid >> 5] = all_hi;
        rows.any_lo[tid >> 5] = any_lo;
        rows.any_hi[tid >> 5] = any_hi;
      }
    } else {
      rows.lo[tid] = real ? base + i : -1;
    }
  };

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
  auto chunk = [&](int ch, const char *q, const ChunkRows<SHAPED, BIASED> &rows) {
    const int in_group = (ch - first) % kCsPer;
    const int r0 = in_group * kSbChunk;
    bool any = has_keys, all;
    if (SHAPED) {
      any = any && __builtin_amdgcn_readfirstlane(rows.any_lo[in_group]) <= k_last && __builtin_amdgcn_readfirstlane(rows.any_hi[in_group]) >= k_first;
      all = __builtin_amdgcn_readfirstlane(rows.all_lo[in_group]) <= k_first && __builtin_amdgcn_readfirstlane(rows.all_hi[in_group]) >= k_last;
    } else {
      const int last = (ch + 1) * kSbChunk - 1;
      any = any && base + chunk_token(last < R ? last : R - 1, p.g_magic) >= k_first;
      all = last < R && base + chunk_token(ch * kSbChunk, p.g_magic) >= k_last;
    }
    if (__builtin_amdgcn_readfirstlane((int)any)) {
      f32x16 acc[kSbTiles];
      sb_multiply<D>(acc, q, kf, col, hf);
      f32x4 ml[4];  // of the rows 8 j + 4 hf .. +3 that this lane's products belong to
#pragma unroll
      for (int j = 0; j < 4; ++j) ml[j] = *reinterpret_cast<const f32x4 *>(&rows.minus_l[r0 + 8 * j + 4 * hf]);
      float scale = p.scale_log2;
      if (SHAPED && p.shape.cap > 0.f) {
        scale = 1.f;
#pragma unroll
        for (int kt = 0; kt < kSbTiles; ++kt)
#pragma unroll
          for (int e = 0; e < 16; ++e) acc[kt][e] = soft_cap(acc[kt][e], p.shape);
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
      if (!__builtin_amdgcn_readfirstlane((int)all)) {
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
  const float v = hf == 0 ? tot[0] : tot[1];
  const int slot = key0 + 32 * hf + col;
  if (slot < n && slot >= skip) {
    float *d = p.dst + (size_t)unit * c.cap + slot;
    *d = p.accumulate ? *d + v : v;
  }
}

}  // namespace dynts
