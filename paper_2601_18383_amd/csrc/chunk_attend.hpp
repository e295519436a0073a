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

}  // namespace dynts
