// Single tokens (and chunks of up to 16 query rows of a unit) on caches of codes: attention and the weights that slots receive.  The formulas are those of
// chunk_attend.hpp and chunk_scores.hpp; bound by HBM.
//
// With products of 16 keys by 16 rows a lane (col, quad) = (lane % 16, lane / 16) gives 8 neighbouring elements of key `col`, and which 8 of the row they are is
// free as long as the queries take the same: 16-byte pieces `quad` and, with head_dim 128, `4 + quad` of the row, so that K's codes come from memory in the
// order in which the products want them, 64 bytes of 16 rows a load, and are decoded in registers.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "chunk_attend.hpp"
#include "chunk_scores.hpp"
#include "codes.hpp"

namespace dynts {

constexpr int kTokRows = 16, kTokTile = 32, kTokWaves = 8;
typedef float tok_f32x4 __attribute__((ext_vector_type(4)));

// Query row r of a unit as an operand: elements 64 j + 16 quad + 8 h .. +7 in place 2 j + h.
template <int D>
__device__ __forceinline__ void token_query(bf16x8 (&f)[D / 32], const uint16_t *row, int quad) {
#pragma unroll
  for (int j = 0; j < D / 64; ++j)
#pragma unroll
    for (int h = 0; h < 2; ++h) f[2 * j + h] = __builtin_bit_cast(bf16x8, load_u32x4(row + 64 * j + 16 * quad + 8 * h));
}
// Codes of a key, as fetched, as the other operand.  scales: the row's, D / 32 bytes.
template <int D, int CODE>
__device__ __forceinline__ void token_key(bf16x8 (&f)[D / 32], const u32x4 (&x)[D / 64], uint32_t scales, int quad) {
#pragma unroll
  for (int j = 0; j < D / 64; ++j) {
    u32x4 lo, hi;
    decode16<CODE>(x[j], scales >> (8 * (2 * j + (quad >> 1))) & 255u, lo, hi);
    f[2 * j] = __builtin_bit_cast(bf16x8, lo);
    f[2 * j + 1] = __builtin_bit_cast(bf16x8, hi);
  }
}
template <int D>
__device__ __forceinline__ uint32_t scales_of_row(RowBuffer buf, int row) {
  if (D == 128) return (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(buf, 4 * row, 0, 0);
  return (uint32_t)__builtin_amdgcn_raw_buffer_load_b16(buf, 2 * row, 0, 0);
}

// Byte of LDS of 16-byte piece `piece` (8 elements) of V's row `row`: 8 rows of two neighbouring pieces lie in different banks.
template <int D>
__device__ __forceinline__ int token_lds(int row, int piece) {
  return row * (2 * D) + 16 * (piece ^ (D == 128 ? 2 * (row & 7) : 2 * ((row >> 1) & 3)));
}

template <int D>
struct TokenLds {
  static constexpr int kPitch = D + 4;                                        // of a wave's output rows, in floats
  static constexpr int kTile = kTokTile * 2 * D, kJoin = kTokRows * kPitch * 4;
  static constexpr int kWave = kTile > kJoin ? kTile : kJoin;
  static_assert(kWave % (2 * D) == 0, "a row of V's tile is changed by its address's low bits alone");
};

// A share of a unit's keys a workgroup, every WAVES'th tile of 32 a wave; V through a part of LDS of the wave's own, the next tile's loads in flight, no
// barrier before the end, where the waves' outputs are joined.  Two workgroups a compute unit, but one where shaped rows of 128 need the registers (158; with 128 and spills
// 512 slots of 128 units 12.4 us instead of 9.5, 16000 140 instead of 99).
// us with eight waves / sixteen / chunk_attend_few's 32 rows (e4m3, head_dim 128): 8 units of 16000 slots 15.9 / 16.9 / 17.3, 128 of 500 7.8 / 9.4 / 9.2, of 2464 19.8 /
// 20.3 / 22.2, 512 of 500 14.5 / 18.9 / - , of 2464 60 / 63 / 68: 333 MB, 5.5 TB/s (a large copy reaches 5.1, these caches lie in the memory-side cache in part).
template <int D, int MASK, int CODE, int WAVES>
__global__ __launch_bounds__(WAVES * 64, MASK == kShaped && D == 128 ? 2 : 4) void coded_token_kernel(const ChunkAttendParams p) {
  using Lds = TokenLds<D>;
  constexpr bool SHAPED = MASK == kShaped;
  const ChunkCache &c = p.c;
  __shared__ __attribute__((aligned(256))) char sm[WAVES][Lds::kWave];
  __shared__ float sm_m[WAVES][kTokRows], sm_l[WAVES][kTokRows];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, quad = lane >> 4;
  int unit, split;
  if (!chunk_map(1, p.n_split, c.Nb * c.Hkv, unit, split)) return;
  const int b = unit / c.Hkv, h = unit - b * c.Hkv;
  int n;
  const int m = chunk_tokens(c, p.n_new, p.T, b, n);
  const int R = m * c.G;
  if (R == 0) return;
  const int base = n - m;
  const int r = col < R ? col : R - 1;
  const int i = chunk_token(r, p.g_magic), g = r - i * c.G;
  bf16x8 qf[D / 32];
  token_query<D>(qf, p.q + (((size_t)b * p.T + i) * c.Hq + (size_t)h * c.G + g) * D, quad);

  const int32_t *pos = c.pos + (size_t)unit * c.cap;
  const int lim = base + i;
  int lo = 0, own = 0;
  uint32_t span = 0;
  float slope = 0.f;
  int t_lo = 0, t_hi = n;
  if (SHAPED) {
    const int head = pos[0], tail = pos[n - 1];
    own = pos[base + i];
    chunk_interval(p.shape, (size_t)b * p.T + i, own, lo, span);
    if (p.shape.slope) slope = p.shape.slope[h * c.G + g] * 1.4426950408889634f;
    int first = lo, last = lo == kNowhere ? -1 : (int)(lo + span);
#pragma unroll
    for (int d = 1; d < 16; d *= 2) {
      const int f = __shfl_xor(first, d), l = __shfl_xor(last, d);
      first = f < first ? f : first;
      last = l > last ? l : last;
    }
    chunk_range(p.shape, pos, n, base, 0, m - 1, __builtin_amdgcn_readfirstlane(first), __builtin_amdgcn_readfirstlane(last),
                __builtin_amdgcn_readfirstlane(head), __builtin_amdgcn_readfirstlane(tail), lane, t_lo, t_hi);
    t_lo = t_lo / kTokTile * kTokTile;
  }
  const int tiles = t_hi > t_lo ? (t_hi - t_lo + kTokTile - 1) / kTokTile : 0;
  int shares, from, to;
  if (!chunk_share(p, tiles, split, unit, shares, from, to)) return;
  const int t_end = __builtin_amdgcn_readfirstlane(t_lo + to * kTokTile);
  int t = __builtin_amdgcn_readfirstlane(t_lo + (from + wave) * kTokTile);

  tok_f32x4 acc[D / 16];
#pragma unroll
  for (int dt = 0; dt < D / 16; ++dt) acc[dt] = tok_f32x4{0.f, 0.f, 0.f, 0.f};
  float nm = 1e30f, l_run = 0.f;  // the exponents' addend (minus the shift, a whole number of log2 units); the lane's share of the sum of weights

  constexpr int PPR = D / 16, PIECES = kTokTile * PPR / 64;  // pieces of 16 codes a row, and of V a lane
  u32x4 kr[2][D / 64], vr[PIECES], pr[2];
  uint32_t ks[2], vs[PIECES];
  auto row_at = [&](int tile) { return chunk_tile<1>(c, unit, tile, c.block_table ? chunk_page(c, unit, tile) : 0); };
  auto rows_of = [&](int tile) { return tile < t_end ? (n - tile < kTokTile ? n - tile : kTokTile) : 0; };  // (past the end: nothing is fetched)
  auto fetch_k = [&](int tile, size_t row) {
    const int rows = rows_of(tile);
    const RowBuffer buf = row_buffer<D / 2>(c.K + row * (D / 2), rows), sb = scale_buffer<D>(c.K_scale + row * (D / kCodeBlock), rows);
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
#pragma unroll
      for (int j = 0; j < D / 64; ++j)
        kr[kt][j] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(buf, (16 * kt + col) * D + 64 * j + 16 * quad, 0, 0));
      ks[kt] = scales_of_row<D>(sb, 16 * kt + col);
    }
    if (SHAPED) {
      const RowBuffer pb = row_buffer<2>(reinterpret_cast<const uint16_t *>(pos + (rows > 0 ? tile : 0)), rows);
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) pr[kt] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(pb, 4 * (16 * kt + 4 * quad), 0, 0));
    }
  };
  auto fetch_v = [&](int tile, size_t row) {
    const int rows = rows_of(tile);
    const RowBuffer buf = row_buffer<D / 2>(c.V + row * (D / 2), rows), sb = scale_buffer<D>(c.V_scale + row * (D / kCodeBlock), rows);
#pragma unroll
    for (int k = 0; k < PIECES; ++k) {
      vr[k] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(buf, 16 * (lane + 64 * k), 0, 0));
      vs[k] = __builtin_amdgcn_raw_buffer_load_b8(sb, (lane + 64 * k) / 2, 0, 0);
    }
  };
  char *const sv = sm[wave];
  // columns 16 dt + col of V's rows 4 quad .. +3: byte v_at ^ 32 dt
  const uint32_t v_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)sv + token_lds<D>(4 * quad + (col >> 2), (col >> 1) & 1) + 8 * (col & 1);
  const bool capped = SHAPED && p.shape.cap > 0.f;
  const float scale = SHAPED ? 1.f : p.scale_log2;
  size_t row = t < t_end ? row_at(t) : 0;
  fetch_k(t, row);
  fetch_v(t, row);
  for (; t < t_end; t += WAVES * kTokTile) {
    const int next = t + WAVES * kTokTile;
    row = next < t_end ? row_at(next) : 0;
    tok_f32x4 s[2];
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      bf16x8 kf[D / 32];
      token_key<D, CODE>(kf, kr[kt], ks[kt], quad);
      s[kt] = tok_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < D / 32; ++k) s[kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[k], qf[k], s[kt], 0, 0, 0);
    }
    u32x4 kp[2];
    if (SHAPED) {
      kp[0] = pr[0];
      kp[1] = pr[1];
    }
    fetch_k(next, row);
    // logits, keys t + 16 kt + 4 quad + e of row `col`: shaped, and hidden keys' at -inf
    if (SHAPED) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int at = (int)kp[e >> 2][e & 3];
        float v = s[e >> 2][e & 3];
        v = !capped ? v * p.scale_log2 : p.shape.far_in == 0.f ? soft_cap(v, p.shape) : soft_cap_far(v, p.scale_log2, p.shape);
        v -= slope * fabsf((float)(own - at));
        s[e >> 2][e & 3] = t + 16 * (e >> 2) + 4 * quad + (e & 3) < n && (uint32_t)(at - lo) <= span ? v : -INFINITY;
      }
    } else if (t + kTokTile > base) {
      asm volatile("; some keys are hidden");
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (t + 16 * (e >> 2) + 4 * quad + (e & 3) > lim) s[e >> 2][e & 3] = -INFINITY;
    }
    // weights with the shift at hand, raised where the tile's logits lie far above it, or are the first (as in chunk_attend_rows)
    bf16x8 pf;
    auto fold = [&]() {
      float w[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        w[e] = fast_exp2(fmaf(s[e >> 2][e & 3], scale, nm));
        pf[e] = (__bf16)w[e];  // (half a step of 2^-8, as the output's rounding)
      }
      return ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
    };
    float sum = fold();
    if (__any(!(sum < kChLimit))) {
      float mx = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
      mx = fmaxf(mx, __shfl_xor(mx, 16));
      mx = fmaxf(mx, __shfl_xor(mx, 32));
      const float next_nm = fminf(floorf(-mx * scale), nm), f = fast_exp2(next_nm - nm);
      l_run *= f;
#pragma unroll
      for (int dt = 0; dt < D / 16; ++dt) acc[dt] *= f;
      nm = next_nm;
      sum = fold();
    }
    l_run += sum;
#pragma unroll
    for (int k = 0; k < PIECES; ++k) {
      u32x4 a, z;
      const int at = lane + 64 * k;
      decode16<CODE>(vr[k], vs[k], a, z);
      *reinterpret_cast<u32x4 *>(sv + token_lds<D>(at / PPR, 2 * (at % PPR))) = a;
      *reinterpret_cast<u32x4 *>(sv + token_lds<D>(at / PPR, 2 * (at % PPR) + 1)) = z;
    }
    fetch_v(next, row);
    wave_lds_fence();
    // (the weights are of keys 4 quad .. +3 and 16 + 4 quad .. +3: so are these columns of V)
    uint32_t vo = v_at;
    asm volatile("" : "+v"(vo));  // (the addresses of the columns are made again for every tile: kept, they would cost eight registers)
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) acc[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(lds_columns(vo ^ 32 * dt, 16 * 2 * D), pf, acc[dt], 0, 0, 0);
    wave_lds_fence();
  }

  // the waves' outputs together: eight neighbouring elements of a row a thread
  l_run += __shfl_xor(l_run, 16);
  l_run += __shfl_xor(l_run, 32);
  if (quad == 0) {
    sm_m[wave][col] = -nm;
    sm_l[wave][col] = l_run;
  }
  float *const mine = reinterpret_cast<float *>(sm[wave]) + col * Lds::kPitch + 4 * quad;
#pragma unroll
  for (int dt = 0; dt < D / 16; ++dt) *reinterpret_cast<tok_f32x4 *>(mine + 16 * dt) = acc[dt];
  __syncthreads();
  const int orow = tid / (D / 8), d0 = 8 * (tid % (D / 8));
  if (orow >= R) return;
  float use = sm_m[0][orow];
#pragma unroll
  for (int w = 1; w < WAVES; ++w) use = fmaxf(use, sm_m[w][orow]);
  float o[8] = {}, sum = 0.f;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    const float f = fast_exp2(sm_m[w][orow] - use);
    const float *part = reinterpret_cast<const float *>(sm[w]) + orow * Lds::kPitch + d0;
    const tok_f32x4 a = *reinterpret_cast<const tok_f32x4 *>(part), z = *reinterpret_cast<const tok_f32x4 *>(part + 4);
    sum += f * sm_l[w][orow];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      o[j] += f * a[j];
      o[4 + j] += f * z[j];
    }
  }
  if (shares == 1) {
    const int oi = chunk_token(orow, p.g_magic);
    chunk_write<D>(p, ((size_t)b * p.T + oi) * c.Hq + (size_t)h * c.G + (orow - oi * c.G), d0, o, use, sum);
  } else {
    const size_t prow = ((size_t)unit * p.n_split + split) * p.Rpad + orow;
    *reinterpret_cast<f32x4 *>(p.part_o + prow * D + d0) = f32x4{o[0], o[1], o[2], o[3]};
    *reinterpret_cast<f32x4 *>(p.part_o + prow * D + d0 + 4) = f32x4{o[4], o[5], o[6], o[7]};
    if (d0 == 0) *reinterpret_cast<float2 *>(p.part_ml + 2 * prow) = float2{use, sum};
  }
}

// The weight that slots receive from up to 16 rows: 64 of them a wave, all asked for at once, rows in the registers of the quads.  grid as chunk_scores_kernel's:
// ceil(cap / 256) workgroups a unit.  Bound by HBM: 512 units of 2657 slots, 180 MB, 32 us, 5.6 TB/s.
constexpr int kTsWaves = 4, kTsKeys = 64 * kTsWaves;
template <int D, bool SHAPED, int CODE>
__global__ __launch_bounds__(kTsWaves * 64) void coded_token_scores_kernel(const ChunkScoreParams p) {
  const ChunkCache &c = p.c;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, quad = lane >> 4;
  int unit, blk;
  if (!chunk_map(kAllUnits, (c.cap + kTsKeys - 1) / kTsKeys, c.Nb * c.Hkv, unit, blk)) return;
  const int b = unit / c.Hkv, h = unit - b * c.Hkv;
  int n;
  const int m = chunk_tokens(c, p.n_new, p.T, b, n);
  if (m == 0) return;
  int skip = p.skip_question ? c.n_prompt[b] : 0;
  skip = skip < 0 ? 0 : skip;
  const int key0 = __builtin_amdgcn_readfirstlane(blk * kTsKeys + 64 * wave);
  if (key0 >= n || key0 + 64 <= skip) return;
  const int R = m * c.G, base = n - m;
  const int32_t *pos = c.pos + (size_t)unit * c.cap;

  const size_t row = chunk_tile<1>(c, unit, key0, c.block_table ? chunk_page(c, unit, key0) : 0);  // (64 slots: of one page)
  const int rows = n - key0 < 64 ? n - key0 : 64;
  const RowBuffer buf = row_buffer<D / 2>(c.K + row * (D / 2), rows), sb = scale_buffer<D>(c.K_scale + row * (D / kCodeBlock), rows);
  u32x4 kr[4][D / 64];
  uint32_t ks[4];
  int kpos[4];
#pragma unroll
  for (int kt = 0; kt < 4; ++kt) {
#pragma unroll
    for (int j = 0; j < D / 64; ++j)
      kr[kt][j] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(buf, (16 * kt + col) * D + 64 * j + 16 * quad, 0, 0));
    ks[kt] = scales_of_row<D>(sb, 16 * kt + col);
    const int slot = key0 + 16 * kt + col;
    kpos[kt] = SHAPED ? pos[slot < n ? slot : n - 1] : slot;
  }
  bf16x8 qf[D / 32];
  {
    const int r = col < R ? col : R - 1, i = chunk_token(r, p.g_magic);
    token_query<D>(qf, p.q + (((size_t)b * p.T + i) * c.Hq + (size_t)h * c.G + (r - i * c.G)) * D, quad);
  }
  // this lane's rows, 4 quad + e: minus their L, and what they see
  float minus_l[4], slope[4];
  int lo[4], own[4];
  uint32_t span[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int r = 4 * quad + e, at = r < R ? r : R - 1, i = chunk_token(at, p.g_magic);
    const size_t token = (size_t)b * p.T + i;
    minus_l[e] = row_addend(p.lse[token * c.Hq + (size_t)h * c.G + (at - i * c.G)]);
    if (SHAPED) {
      own[e] = pos[base + i];
      chunk_interval(p.shape, token, own[e], lo[e], span[e]);
      slope[e] = p.shape.slope ? p.shape.slope[h * c.G + (at - i * c.G)] * 1.4426950408889634f : 0.f;
      if (r >= R) {
        lo[e] = kNowhere;
        span[e] = 0;
      }
    } else {
      lo[e] = r < R ? base + i : -1;
    }
  }
  float got = 0.f;
#pragma unroll
  for (int kt = 0; kt < 4; ++kt) {
    bf16x8 kf[D / 32];
    token_key<D, CODE>(kf, kr[kt], ks[kt], quad);
    tok_f32x4 s = tok_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < D / 32; ++k) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(qf[k], kf[k], s, 0, 0, 0);
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float x = s[e];
      bool seen;
      if (SHAPED) {
        x = !(p.shape.cap > 0.f) ? x * p.scale_log2 : p.shape.far_in == 0.f ? soft_cap(x, p.shape) : soft_cap_far(x, p.scale_log2, p.shape);
        x -= slope[e] * fabsf((float)(own[e] - kpos[kt]));
        seen = (uint32_t)(kpos[kt] - lo[e]) <= span[e];
      } else {
        x *= p.scale_log2;
        seen = kpos[kt] <= lo[e];
      }
      sum += seen ? fast_exp2(x + minus_l[e]) : 0.f;
    }
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    if (quad == kt) got = sum;
  }
  const int slot = key0 + lane;
  if (slot < n && slot >= skip) {
    float *d = p.dst + (size_t)unit * c.cap + slot;
    got = received(got);
    *d = p.accumulate ? *d + got : got;
  }
}

}  // namespace dynts
