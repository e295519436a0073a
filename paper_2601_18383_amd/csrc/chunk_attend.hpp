// Attention of a chunk of new tokens over the cache (Eq. attn-score, Eq. attn-o for a block of queries at once).
//
// The m new tokens of a sequence are the last m slots of its cache.  Query row r = i * G + g of a (sequence, KV head) unit is head g of the
// group and token i; a unit's rows all read the same K and V.  A row sees the slots up to its own, or, with a shaping, the
// positions of an interval:
//   x_rj = c * q_r . k_j               (log2 units: c = scale * log2 e)
//   x_rj = cap * tanh(x_rj / cap)      softcap
//   x_rj -= slope_g * |p_i - p_j|      bias by distance (positions, not slots: evictions leave gaps)
//   x_rj = -inf unless max(first_i, p_i - window + 1) <= p_j <= last_i
//   out_r = sum_j 2^(x_rj - L_r) v_j,  L_r = log2 sum_j 2^x_rj
// in one pass over the keys, with a shift per row in place of the maximum (see fold) that is only ever raised.
//
// Operands: K tile (A, 32 keys x 16) times query rows (B, 16 x 32 rows) gives a lane 16 keys, 8 (i / 4) + 4 hf + i % 4, of one row
// (lane (col, hf) = (lane % 32, lane / 32)).  Those are the elements that lane has to give as B operand of V^T P, if V^T's columns
// are taken in the same order: the weights never change lanes.  V^T comes out of LDS by ds_read_b64_tr_b16.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "attend.hpp"
#include "chunk.hpp"
#include "score_block.hpp"

namespace dynts {

// dynts_shaping in log2 units
struct ChunkShape {
  float cap, cap_in;      // softcap * log2 e, or 0; 2 * log2 e * scale / softcap
  int window;             // 0: none
  const float *slope;     // [Hq] or null
  const int32_t *first, *last;  // [Nb][T] or null
};

struct ChunkAttendParams {
  ChunkCache c;
  const uint16_t *q;      // [Nb][T][Hq][D]
  const int32_t *n_new;   // [Nb] or null: T
  uint16_t *out;          // [Nb][T][Hq][D]
  float *lse;             // [Nb][T][Hq] or null
  ChunkShape shape;
  int T;
  float scale_log2;
  // Keys of a row block cut into n_split shares, a workgroup each: unnormalised outputs and (shift, sum) of unit u, share s and row r in row
  // (u * n_split + s) * Rpad + r
  int n_split, Rpad;
  float *part_o, *part_ml;  // [..][D], [..][2]
};

constexpr int kChWaves = 4, kChThreads = kChWaves * 64;
constexpr int kChRows = 32 * kChWaves;  // query rows a workgroup
constexpr int kChTile = 64;             // slots staged at a time
constexpr int kNowhere = 0x7fffffff;    // a position that no key has

// New tokens of sequence b that are queries, and its length.
__device__ __forceinline__ int chunk_tokens(const ChunkCache &c, const int32_t *n_new, int T, int b, int &n) {
  n = c.seq_len[b];
  n = n < 0 ? 0 : (n > c.cap ? c.cap : n);
  int m = n_new ? n_new[b] : T;
  m = m < 0 ? 0 : (m > T ? T : m);
  return m < n ? m : n;
}

// Where slot t (a multiple of kChTile, and of a page's rows) of a unit begins, in elements.
template <int D>
__device__ __forceinline__ size_t chunk_tile(const ChunkCache &c, size_t unit, int t) {
  return c.block_table ? paged_row<D>(c.block_table + unit * c.max_pages, t, c.max_pages, c.n_pages) : (unit * (size_t)c.cap + t) * D;
}

// Byte of LDS at which 16-byte piece `piece` of row `row` of a tile lies.  The pieces of a row are permuted so that what is read together lies in
// different banks: 16 rows of one piece (K operands), and 4 rows of 4 neighbouring pieces (V operands).
template <int D>
__device__ __forceinline__ int chunk_lds(int row, int piece) {
  const int f = D == 128 ? (row & 3) << 2 | ((row >> 2) & 3) : ((row >> 1) & 1) << 2 | ((row >> 2) & 3);
  return row * (2 * D) + 16 * (piece ^ f);
}

// The interval of positions that token i sees, as its lower end and the distance to its upper one; own: the token's position.
__device__ __forceinline__ void chunk_interval(const ChunkShape &s, size_t at, int own, int &lo, uint32_t &span) {
  int low = 0, high = own;
  if (s.window > 0) low = own - s.window + 1;
  if (s.first) {
    const int f = s.first[at];
    low = f > low ? f : low;
  }
  if (s.last) high = s.last[at];
  low = low < 0 ? 0 : low;
  high = high >= kNowhere ? kNowhere - 1 : high;
  if (high < low) low = high = kNowhere;
  lo = low;
  span = (uint32_t)high - (uint32_t)low;
}

// Slots of [0, n) whose position is below `target` (positions ascend along the cache): 64 of them looked at a time, by one wave.
__device__ __forceinline__ int slots_below(const int32_t *pos, int n, int target, int lane) {
  int lo = 0, hi = n;  // the answer lies in [lo, hi]
  while (lo < hi) {
    const int step = (hi - lo + 63) / 64, at = lo + lane * step;
    const int below = __popcll(__ballot(at < hi && pos[at < hi ? at : lo] < target));
    if (below == 0) return lo;
    const int from = lo + (below - 1) * step + 1, to = lo + below * step;
    lo = from;
    hi = to < hi ? to : hi;
  }
  return lo;
}

// cap * tanh(dot * scale / softcap) in log2 units: (1 - u) / (1 + u) with u = 2^(-2 |z| log2 e) is off by 2^-25 of the cap where its argument is small.
__device__ __forceinline__ float soft_cap(float dot, const ChunkShape &s) {
  const float u = fast_exp2(-fabsf(dot * s.cap_in));
  return copysignf(s.cap * (1.f - u) * __builtin_amdgcn_rcpf(1.f + u), dot);
}

// Eight neighbouring elements of an output row, and its lse, from their unnormalised values, shift and sum.
template <int D>
__device__ __forceinline__ void chunk_write(const ChunkAttendParams &p, size_t row, int d0, const float (&o)[8], float top, float sum) {
  const float inv = sum > 0.f ? 1.f / sum : 0.f;  // (a row that sees nothing: zeros, and -inf)
  store_u32x4(p.out + row * D + d0, u32x4{bf16_pack(o[0] * inv, o[1] * inv), bf16_pack(o[2] * inv, o[3] * inv), bf16_pack(o[4] * inv, o[5] * inv),
                                          bf16_pack(o[6] * inv, o[7] * inv)});
  if (p.lse && d0 == 0) p.lse[row] = sum > 0.f ? (top + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f : -INFINITY;
}

template <int D, bool SHAPED>
__global__ __launch_bounds__(kChThreads) void chunk_attend_kernel(const ChunkAttendParams p) {
  const ChunkCache &c = p.c;
  constexpr int kTileBytes = kChTile * 2 * D;
  __shared__ __attribute__((aligned(16))) char sm_k[kTileBytes], sm_v[kTileBytes];
  __shared__ __attribute__((aligned(16))) int sm_pos[kChTile];
  __shared__ int sm_range[2];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, hf = lane >> 5, r16 = lane & 15;
  int unit, blk;
  const int n_blk = (p.T * c.G + kChRows - 1) / kChRows;
  if (!sb_map(n_blk, c.Nb * c.Hkv, unit, blk)) return;
  const int b = unit / c.Hkv, h = unit - b * c.Hkv;
  int n;
  const int m = chunk_tokens(c, p.n_new, p.T, b, n);
  const int R = m * c.G;
  blk = n_blk - 1 - blk;  // (the last rows see most)
  if (blk * kChRows >= R) return;
  const int base = n - m;  // the chunk's first slot

  const int row0 = blk * kChRows + wave * 32;
  const int r = row0 + col < R ? row0 + col : R - 1;
  const int i = r / c.G, g = r - i * c.G;
  const size_t qrow = ((size_t)b * p.T + i) * c.Hq + (size_t)h * c.G + g;
  bf16x8 qf[D / 16];
  load_row_frags<D>(qf, reinterpret_cast<const char *>(p.q + qrow * D), hf);

  // what the row sees; in the plain form slots [0, lim], else positions [lo, lo + span]
  const int32_t *pos = c.pos + (size_t)unit * c.cap;
  const int lim = base + i;
  int lo = 0, ref = 0;
  uint32_t span = 0;
  float at = 0.f, slope = 0.f;
  int t_lo = 0, t_hi;
  if (SHAPED) {
    const int own = pos[base + i];
    chunk_interval(p.shape, (size_t)b * p.T + i, own, lo, span);
    ref = __builtin_amdgcn_readfirstlane(pos[base]);
    at = (float)(own - ref);
    if (p.shape.slope) slope = p.shape.slope[h * c.G + g] * 1.4426950408889634f;
    // the slots that some row of the workgroup sees
    if (tid == 0) {
      sm_range[0] = kNowhere;
      sm_range[1] = -1;
    }
    __syncthreads();
    if (lo != kNowhere) {
      atomicMin(&sm_range[0], lo);
      atomicMax(&sm_range[1], (int)(lo + span));
    }
    __syncthreads();
    t_lo = slots_below(pos, n, sm_range[0], lane) / kChTile * kChTile;
    t_hi = slots_below(pos, n, sm_range[1] + 1, lane);
  } else {
    int last = blk * kChRows + kChRows - 1;
    last = last < R ? last : R - 1;
    t_hi = base + last / c.G + 1;
  }
  t_lo = __builtin_amdgcn_readfirstlane(t_lo);
  t_hi = __builtin_amdgcn_readfirstlane(t_hi);

  f32x16 acc[D / 32];
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[dt][e] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;

  constexpr int PPR = D / 8, PIECES = kChTile * PPR / kChThreads;
  for (int t = t_lo; t < t_hi; t += kChTile) {
    const size_t from = chunk_tile<D>(c, unit, t);
    const int rows = n - t < kChTile ? n - t : kChTile;
    const RowBuffer kb = row_buffer<D>(c.K + from, rows), vb = row_buffer<D>(c.V + from, rows);
    __syncthreads();
#pragma unroll
    for (int k = 0; k < PIECES; ++k) {
      const int at_piece = tid + kChThreads * k, dst = chunk_lds<D>(at_piece / PPR, at_piece % PPR);
      *reinterpret_cast<u32x4 *>(sm_k + dst) = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(kb, 16 * at_piece, 0, 0));
      *reinterpret_cast<u32x4 *>(sm_v + dst) = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(vb, 16 * at_piece, 0, 0));
    }
    if (SHAPED && tid < kChTile) sm_pos[tid] = tid < rows ? pos[t + tid] : -1;
    __syncthreads();
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      f32x16 s;
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = 0.f;
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks) {
        const bf16x8 kf = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(sm_k + chunk_lds<D>(32 * half + col, 2 * ks + hf)));
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[ks], s, 0, 0, 0);
      }
      float mx = -INFINITY;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int key = 32 * half + 8 * (e >> 2) + 4 * hf + (e & 3);
        if (SHAPED) {
          float x = p.shape.cap > 0.f ? soft_cap(s[e], p.shape) : s[e] * p.scale_log2;
          const int kp = sm_pos[key];
          x -= slope * fabsf(at - (float)(kp - ref));
          s[e] = (uint32_t)(kp - lo) <= span ? x : -INFINITY;
        } else {
          s[e] = t + key <= lim ? s[e] * p.scale_log2 : -INFINITY;
        }
        mx = fmaxf(mx, s[e]);
      }
      mx = fmaxf(mx, __shfl_xor(mx, 32));
      const float m_next = fmaxf(m_run, mx), m_use = m_next == -INFINITY ? 0.f : m_next;
      const float corr = fast_exp2(m_run - m_use);
      m_run = m_next;
      float sum = 0.f;
      bf16x8 pf[2];  // (the weights are rounded to bf16 for the product with V: half a step of 2^-8 relative each, as the output is)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float w = fast_exp2(s[e] - m_use);
        sum += w;
        pf[e >> 3][e & 7] = (__bf16)w;
      }
      l_run = l_run * corr + sum;
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt) {
        acc[dt] *= corr;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
          // lane (r16 of its 16, ...) points at row r16 / 4 and columns 4 (r16 % 4) .. +3, and gets column r16 of the four rows
          const int vrow = 32 * half + 16 * ks + 4 * hf + (r16 >> 2), piece = 4 * dt + 2 * ((lane >> 4) & 1) + ((r16 >> 1) & 1);
          const i16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4 *)(sm_v + chunk_lds<D>(vrow, piece) + 8 * (r16 & 1)));
          const i16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4 *)(sm_v + chunk_lds<D>(vrow + 8, piece) + 8 * (r16 & 1)));
          acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7)), pf[ks],
                                                            acc[dt], 0, 0, 0);
        }
      }
    }
  }

  const float l = l_run + __shfl_xor(l_run, 32);
  if (row0 + col >= R) return;
  const float inv = l > 0.f ? 1.f / l : 0.f;  // (a row that sees nothing: zeros, and -inf)
  uint16_t *out = p.out + qrow * D;
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int e = 0; e < 16; e += 4) {
      const uint2 w = {bf16_pack(acc[dt][e] * inv, acc[dt][e + 1] * inv), bf16_pack(acc[dt][e + 2] * inv, acc[dt][e + 3] * inv)};
      *reinterpret_cast<uint2 *>(out + 32 * dt + 2 * e + 4 * hf) = w;
    }
  if (p.lse && hf == 0) p.lse[qrow] = l > 0.f ? (m_run + __builtin_amdgcn_logf(l)) * 0.6931471805599453f : -INFINITY;
}

// ---- few rows: 32 of them a workgroup, its eight waves share out the keys --------------------------------------------------
// Bound by HBM (or the memory-side cache): every wave streams 32 slots at a time through registers and a part of LDS of its own, the next
// tile's loads in flight while it works on one, no barrier before the end.  There the waves' outputs are joined through LDS.
constexpr int kFewWaves = 8, kFewThreads = kFewWaves * 64, kFewRows = 32, kFewTile = 32;
template <int D>
struct FewLds {
  static constexpr int kTileBytes = kFewTile * 2 * D;             // K's, and V's
  static constexpr int kJoin = D / 2 * 65 * (int)sizeof(float);   // a wave's output: 64 lanes by D / 2 registers, a row of 64 padded by one
  static constexpr int kWave = 2 * kTileBytes > kJoin ? 2 * kTileBytes : kJoin;
};

template <int D, bool SHAPED>
__global__ __launch_bounds__(kFewThreads, 2) void chunk_attend_few_kernel(const ChunkAttendParams p) {
  using Lds = FewLds<D>;
  const ChunkCache &c = p.c;
  __shared__ __attribute__((aligned(16))) char sm[kFewWaves][Lds::kWave];
  __shared__ __attribute__((aligned(16))) int sm_pos[kFewWaves][kFewTile];
  __shared__ float sm_m[kFewWaves][kFewRows], sm_l[kFewWaves][kFewRows];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, hf = lane >> 5, r16 = lane & 15;
  int unit, blk;
  const int n_blk = (p.T * c.G + kFewRows - 1) / kFewRows;
  if (!sb_map(n_blk * p.n_split, c.Nb * c.Hkv, unit, blk)) return;
  const int split = blk / n_blk;  // (the blocks of one share side by side: they read the same keys)
  blk -= split * n_blk;
  const int b = unit / c.Hkv, h = unit - b * c.Hkv;
  int n;
  const int m = chunk_tokens(c, p.n_new, p.T, b, n);
  const int R = m * c.G, row0 = blk * kFewRows;
  if (row0 >= R) return;
  const int base = n - m;

  const int r = row0 + col < R ? row0 + col : R - 1;
  const int i = r / c.G, g = r - i * c.G;
  const size_t qrow = ((size_t)b * p.T + i) * c.Hq + (size_t)h * c.G + g;
  bf16x8 qf[D / 16];
  load_row_frags<D>(qf, reinterpret_cast<const char *>(p.q + qrow * D), hf);

  const int32_t *pos = c.pos + (size_t)unit * c.cap;
  const int lim = base + i;
  int lo = 0, ref = 0;
  uint32_t span = 0;
  float at = 0.f, slope = 0.f;
  int t_lo = 0, t_hi;
  if (SHAPED) {
    const int own = pos[base + i];
    chunk_interval(p.shape, (size_t)b * p.T + i, own, lo, span);
    ref = __builtin_amdgcn_readfirstlane(pos[base]);
    at = (float)(own - ref);
    if (p.shape.slope) slope = p.shape.slope[h * c.G + g] * 1.4426950408889634f;
    // the slots that some row sees (every wave has all rows)
    int first = lo, last = lo == kNowhere ? -1 : (int)(lo + span);
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const int f = __shfl_xor(first, d), l = __shfl_xor(last, d);
      first = f < first ? f : first;
      last = l > last ? l : last;
    }
    t_lo = slots_below(pos, n, first, lane) / kFewTile * kFewTile;
    t_hi = slots_below(pos, n, last + 1, lane);
  } else {
    const int last = row0 + kFewRows - 1 < R ? row0 + kFewRows - 1 : R - 1;
    t_hi = base + last / c.G + 1;
  }
  // this share's tiles, every kFewWaves'th of them this wave's
  const int tiles = t_hi > t_lo ? (t_hi - t_lo + kFewTile - 1) / kFewTile : 0;
  const int from = (int)((long long)tiles * split / p.n_split), to = (int)((long long)tiles * (split + 1) / p.n_split);
  const int t_end = __builtin_amdgcn_readfirstlane(t_lo + to * kFewTile);
  int t = __builtin_amdgcn_readfirstlane(t_lo + (from + wave) * kFewTile);

  f32x16 acc[D / 32];
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[dt][e] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;

  char *const sk = sm[wave], *const sv = sm[wave] + Lds::kTileBytes;
  constexpr int PPR = D / 8, PIECES = kFewTile * PPR / 64;  // 16-byte pieces a row, and of K or V a lane
  u32x4 kr[PIECES], vr[PIECES];
  int pr = 0;
  auto fetch = [&](int tile, u32x4 (&x)[PIECES], const uint16_t *pool) {
    // (past the share's end: a buffer of no rows, nothing is fetched)
    const int rows = tile < t_end ? (n - tile < kFewTile ? n - tile : kFewTile) : 0;
    const RowBuffer buf = row_buffer<D>(pool + (rows > 0 ? chunk_tile<D>(c, unit, tile) : 0), rows);
#pragma unroll
    for (int k = 0; k < PIECES; ++k) x[k] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(buf, 16 * (lane + 64 * k), 0, 0));
  };
  auto park = [&](char *dst, const u32x4 (&x)[PIECES]) {
#pragma unroll
    for (int k = 0; k < PIECES; ++k) *reinterpret_cast<u32x4 *>(dst + chunk_lds<D>((lane + 64 * k) / PPR, (lane + 64 * k) % PPR)) = x[k];
  };
  auto fetch_pos = [&](int tile) { pr = tile < t_end && tile + col < n ? pos[tile + col] : -1; };
  fetch(t, kr, c.K);
  if (SHAPED) fetch_pos(t);
  fetch(t, vr, c.V);
  for (; t < t_end; t += kFewWaves * kFewTile) {
    const int next = t + kFewWaves * kFewTile;
    park(sk, kr);
    if (SHAPED && hf == 0) sm_pos[wave][col] = pr;
    fetch(next, kr, c.K);
    if (SHAPED) fetch_pos(next);
    wave_lds_fence();
    f32x16 s;
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = 0.f;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
      const bf16x8 kf = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(sk + chunk_lds<D>(col, 2 * ks + hf)));
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[ks], s, 0, 0, 0);
    }
    float mx = -INFINITY;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int key = 8 * (e >> 2) + 4 * hf + (e & 3);
      if (SHAPED) {
        float x = p.shape.cap > 0.f ? soft_cap(s[e], p.shape) : s[e] * p.scale_log2;
        const int kp = sm_pos[wave][key];
        x -= slope * fabsf(at - (float)(kp - ref));
        s[e] = (uint32_t)(kp - lo) <= span ? x : -INFINITY;
      } else {
        s[e] = t + key <= lim ? s[e] * p.scale_log2 : -INFINITY;
      }
      mx = fmaxf(mx, s[e]);
    }
    mx = fmaxf(mx, __shfl_xor(mx, 32));
    const float m_next = fmaxf(m_run, mx), m_use = m_next == -INFINITY ? 0.f : m_next;
    const float corr = fast_exp2(m_run - m_use);
    m_run = m_next;
    float sum = 0.f;
    bf16x8 pf[2];
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float w = fast_exp2(s[e] - m_use);
      sum += w;
      pf[e >> 3][e & 7] = (__bf16)w;
    }
    l_run = l_run * corr + sum;
    park(sv, vr);
    fetch(next, vr, c.V);
    wave_lds_fence();
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt) {
      acc[dt] *= corr;
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        const int vrow = 16 * ks + 4 * hf + (r16 >> 2), piece = 4 * dt + 2 * ((lane >> 4) & 1) + ((r16 >> 1) & 1);
        const i16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4 *)(sv + chunk_lds<D>(vrow, piece) + 8 * (r16 & 1)));
        const i16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4 *)(sv + chunk_lds<D>(vrow + 8, piece) + 8 * (r16 & 1)));
        acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7)), pf[ks],
                                                          acc[dt], 0, 0, 0);
      }
    }
    wave_lds_fence();
  }

  // the waves' outputs together: eight neighbouring elements of a row a thread
  const float l = l_run + __shfl_xor(l_run, 32);
  if (hf == 0) {
    sm_m[wave][col] = m_run;
    sm_l[wave][col] = l;
  }
  float *const own_part = reinterpret_cast<float *>(sm[wave]);
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int e = 0; e < 16; ++e) own_part[(16 * dt + e) * 65 + lane] = acc[dt][e];
  __syncthreads();
  const int row = tid / (D / 8), d0 = 8 * (tid % (D / 8));
  if (row >= kFewRows || row0 + row >= R) return;  // (D = 64: 256 threads have none)
  float top = -INFINITY;
#pragma unroll
  for (int w = 0; w < kFewWaves; ++w) top = fmaxf(top, sm_m[w][row]);
  const float use = top == -INFINITY ? 0.f : top;
  float o[8] = {}, sum = 0.f;
#pragma unroll
  for (int w = 0; w < kFewWaves; ++w) {
    const float f = fast_exp2(sm_m[w][row] - use);
    const float *part = reinterpret_cast<const float *>(sm[w]) + (16 * (d0 / 32) + 4 * (d0 % 32 / 8)) * 65 + row;
    sum += f * sm_l[w][row];
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] += f * part[(j & 3) * 65 + 32 * (j >> 2)];
  }
  const int rr = row0 + row;
  if (p.n_split == 1) {
    const int ri = rr / c.G;
    const size_t orow = ((size_t)b * p.T + ri) * c.Hq + (size_t)h * c.G + (rr - ri * c.G);
    chunk_write<D>(p, orow, d0, o, use, sum);
  } else {
    const size_t prow = ((size_t)unit * p.n_split + split) * p.Rpad + rr;
    *reinterpret_cast<f32x4 *>(p.part_o + prow * D + d0) = f32x4{o[0], o[1], o[2], o[3]};
    *reinterpret_cast<f32x4 *>(p.part_o + prow * D + d0 + 4) = f32x4{o[4], o[5], o[6], o[7]};
    if (d0 == 0) *reinterpret_cast<float2 *>(p.part_ml + 2 * prow) = float2{use, sum};
  }
}

// The shares of a row together.  grid (ceil(T * G / kMergeRows), units), D / 8 threads a row.
constexpr int kMergeThreads = 256;
template <int D>
__global__ __launch_bounds__(kMergeThreads) void chunk_merge_kernel(const ChunkAttendParams p) {
  const ChunkCache &c = p.c;
  const int unit = blockIdx.y, b = unit / c.Hkv, h = unit - b * c.Hkv;
  int n;
  const int m = chunk_tokens(c, p.n_new, p.T, b, n);
  const int r = blockIdx.x * (kMergeThreads / (D / 8)) + threadIdx.x / (D / 8), d0 = 8 * (threadIdx.x % (D / 8));
  if (r >= m * c.G) return;
  const size_t first = (size_t)unit * p.n_split * p.Rpad + r;
  float top = -INFINITY, sum = 0.f, o[8] = {};
  for (int s0 = 0; s0 < p.n_split; s0 += 4) {  // four shares' loads at a time
    float2 ml[4];
    f32x4 a[4], z[4];
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const size_t prow = first + (size_t)(s0 + s < p.n_split ? s0 + s : s0) * p.Rpad;
      ml[s] = *reinterpret_cast<const float2 *>(p.part_ml + 2 * prow);
      a[s] = *reinterpret_cast<const f32x4 *>(p.part_o + prow * D + d0);
      z[s] = *reinterpret_cast<const f32x4 *>(p.part_o + prow * D + d0 + 4);
    }
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      if (s0 + s >= p.n_split || !(ml[s].y > 0.f)) continue;  // (a share without a key that the row sees)
      const float next = fmaxf(top, ml[s].x), f = fast_exp2(top - next), w = fast_exp2(ml[s].x - next);
      top = next;
      sum = sum * f + ml[s].y * w;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        o[j] = o[j] * f + a[s][j] * w;
        o[4 + j] = o[4 + j] * f + z[s][j] * w;
      }
    }
  }
  const int i = r / c.G;
  chunk_write<D>(p, ((size_t)b * p.T + i) * c.Hq + (size_t)h * c.G + (r - i * c.G), d0, o, top, sum);
}

}  // namespace dynts
