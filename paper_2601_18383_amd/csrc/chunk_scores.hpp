// The attention weight that every cached slot receives from a chunk's queries (Eq. importance-score for a block of queries that are part of
// the cache): S_j += sum over the rows r that see slot j of 2^(x_rj - L_r), with the logits of chunk_attend.hpp and their
// log-sum-exp L_r.
//
// Keys are the stationary operand (B: 64 slots a wave), query rows stream through LDS 32 at a time (A), so that a lane holds 16
// rows of one slot, adds them up by itself, and joins the other half once, at the end: no atomics, one order.
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
};

constexpr int kCsKeys = kSbRowsPerWg;  // slots a workgroup

// 1-D grid of ceil(cap / 256) * round_up(units, 8) workgroups, 256 threads.
template <int D, bool SHAPED>
__global__ __launch_bounds__(kSbWaves * 64) void chunk_scores_kernel(const ChunkScoreParams p) {
  using St = SbStage<D>;
  const ChunkCache &c = p.c;
  __shared__ __attribute__((aligned(16))) char sm_q[St::kBufBytes];
  struct Row {
    float L;      // log2 of the denominator, +inf: the row does not count
    int lo;       // plain: the last slot it sees; shaped: the lowest position
    uint32_t span;
    float at, slope;
  };
  __shared__ Row sm_row[kSbChunk];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 31, hf = lane >> 5;
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
  const int ref = SHAPED ? __builtin_amdgcn_readfirstlane(pos[base]) : 0;

  bf16x8 kf[kSbTiles][D / 16];
  int kpos[kSbTiles];
  float kat[kSbTiles], sum[kSbTiles];
#pragma unroll
  for (int kt = 0; kt < kSbTiles; ++kt) {
    int slot = key0 + 32 * kt + col;
    slot = slot < n ? slot : n - 1;
    const size_t row = c.block_table ? paged_row<D>(c.block_table + (size_t)unit * c.max_pages, slot, c.max_pages, c.n_pages)
                                     : ((size_t)unit * c.cap + slot) * D;
    load_row_frags<D>(kf[kt], reinterpret_cast<const char *>(c.K + row), hf);
    kpos[kt] = SHAPED ? pos[slot] : slot;
    kat[kt] = SHAPED ? (float)(kpos[kt] - ref) : 0.f;
    sum[kt] = 0.f;
  }
  // (plain: rows whose own slot lies before all of these keys see none of them)
  const int i0 = SHAPED ? 0 : (blk * kCsKeys > base ? blk * kCsKeys - base : 0);
  for (int ch = i0 * c.G / kSbChunk; ch * kSbChunk < R; ++ch) {
    __syncthreads();
    {
      const int at = tid >> 3, r = ch * kSbChunk + at < R ? ch * kSbChunk + at : R - 1, i = r / c.G, g = r - i * c.G;
      const size_t qrow = ((size_t)b * p.T + i) * c.Hq + (size_t)h * c.G + g;
      const char *src = reinterpret_cast<const char *>(p.q + qrow * D) + 16 * (tid & 7);
#pragma unroll
      for (int k = 0; k < St::NL; ++k)
        *reinterpret_cast<u32x4 *>(sm_q + at * St::LROW + 16 * (tid & 7) + 128 * k) = *reinterpret_cast<const u32x4 *>(src + 128 * k);
      if ((tid & 7) == 0) {
        Row row;
        const float l = p.lse[qrow];
        row.L = ch * kSbChunk + at < R && l != -INFINITY ? l * 1.4426950408889634f : INFINITY;
        row.lo = base + i;
        row.span = 0;
        row.at = row.slope = 0.f;
        if (SHAPED) {
          const int own = pos[base + i];
          chunk_interval(p.shape, (size_t)b * p.T + i, own, row.lo, row.span);
          row.at = (float)(own - ref);
          if (p.shape.slope) row.slope = p.shape.slope[h * c.G + g] * 1.4426950408889634f;
        }
        sm_row[at] = row;
      }
    }
    __syncthreads();
    f32x16 acc[kSbTiles];
    sb_multiply<D>(acc, sm_q, kf, col, hf);
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const Row row = sm_row[8 * (e >> 2) + 4 * hf + (e & 3)];
#pragma unroll
      for (int kt = 0; kt < kSbTiles; ++kt) {
        float x;
        bool seen;
        if (SHAPED) {
          x = p.shape.cap > 0.f ? soft_cap(acc[kt][e], p.shape) : acc[kt][e] * p.scale_log2;
          x -= row.slope * fabsf(row.at - kat[kt]);
          seen = (uint32_t)(kpos[kt] - row.lo) <= row.span;
        } else {
          x = acc[kt][e] * p.scale_log2;
          seen = kpos[kt] <= row.lo;
        }
        sum[kt] += seen ? fast_exp2(x - row.L) : 0.f;
      }
    }
  }
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
