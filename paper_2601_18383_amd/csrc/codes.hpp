// Caches of 8-bit codes.  A block of 32 neighbouring elements of a row shares a scale, a power of two:
//   value = code * 2^(s - 127),   s the block's scale byte, the least (27 at least) with   max |x| <= top * 2^(s - 127),
// top 448 for e4m3 (a float of 4 bits of exponent and 3 of mantissa), 127 for whole numbers; codes are rounded to nearest, ties to even: off by
// 2^-4 of the value at most, small ones by 2^-10 of 2^(s - 127) (e4m3), or by half of 2^(s - 127) (whole numbers).  A block that holds an infinity, a NaN or 2^126 and more has s = 255, and reads as NaN.
//
// A code has at most eight significant bits and the scale none: every value is exact in bf16, so the kernels that read a cache
// of codes are those of bf16 caches with the codes turned into bf16 on the way, and nothing about their arithmetic changes.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "attend.hpp"
#include "chunk.hpp"
#include "compact.hpp"

namespace dynts {

constexpr int kCodeBlock = 32;  // elements of a scale
constexpr int kLeastScale = 27, kNoScale = 255;

template <int CODE>
__device__ __forceinline__ uint32_t code_scale(uint32_t most) {  // most: the largest of a block, as bf16 without its sign
  const int e = (int)(most >> 7), m = (int)(most & 127u);
  int s = CODE == DYNTS_CODE_E4M3 ? e - 8 + (m > 96) : e - 6 + (m > 126);  // (448 = 1.75 * 2^8, 127 = 1.984375 * 2^6)
  s = s < kLeastScale ? kLeastScale : s;
  return most >= 0x7e80u ? (uint32_t)kNoScale : (uint32_t)s;
}

// Eight neighbouring elements, x, to `codes + at`, and their block's scale, by four neighbouring lanes that have a block between them; piece: which eighth of
// elements of the row.  (512 tokens of 64 sequences, 8 heads of 128, 203 MB read and written: 37 us, 5.5 TB/s; a large copy reaches 5.1.)
template <int CODE>
__device__ __forceinline__ void encode8(u32x4 x, uint8_t *codes, uint8_t *scales, size_t at, int piece) {
  uint32_t most = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const uint32_t lo = x[k] & 0x7fffu, hi = x[k] >> 16 & 0x7fffu;
    most = lo > most ? lo : most;
    most = hi > most ? hi : most;
  }
#pragma unroll
  for (int d = 1; d < 4; d *= 2) {
    const uint32_t other = (uint32_t)__shfl_xor((int)most, d);
    most = other > most ? other : most;
  }
  const uint32_t s = code_scale<CODE>(most);
  const float inv = __uint_as_float((254u - s) << 23);  // (exact: a power of two)
  uint32_t out[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const float a = bf16_low(x[2 * k]) * inv, b = bf16_high(x[2 * k]) * inv, c = bf16_low(x[2 * k + 1]) * inv, d = bf16_high(x[2 * k + 1]) * inv;
    if (CODE == DYNTS_CODE_E4M3) {
      int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
      out[k] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
      if (s == kNoScale) out[k] = 0x7f7f7f7fu;
    } else {
      auto whole = [](float v) { return (uint32_t)(int)__builtin_rintf(v) & 255u; };
      out[k] = s == kNoScale ? 0u : whole(a) | whole(b) << 8 | whole(c) << 16 | whole(d) << 24;  // (0 times infinity)
    }
  }
  *reinterpret_cast<uint2 *>(codes + at) = uint2{out[0], out[1]};
  if (piece % 4 == 0) scales[at / kCodeBlock] = (uint8_t)s;
}

// Four codes of a word as bf16.  scale: 2^(s - 127).
template <int CODE>
__device__ __forceinline__ void decode4(uint32_t w, float scale, uint32_t &lo, uint32_t &hi) {
  if (CODE == DYNTS_CODE_E4M3) {
    lo = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false));
    hi = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true));
  } else {
    lo = bf16_pack((float)(int8_t)w * scale, (float)(int8_t)(w >> 8) * scale);
    hi = bf16_pack((float)(int8_t)(w >> 16) * scale, (float)(int8_t)(w >> 24) * scale);
  }
}
// Sixteen neighbouring codes of one block as two pieces of eight bf16.
template <int CODE>
__device__ __forceinline__ void decode16(u32x4 x, uint32_t s, u32x4 &lo, u32x4 &hi) {
  const float scale = __uint_as_float(s << 23);
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    uint32_t a, b;
    decode4<CODE>(x[k], scale, a, b);
    lo[2 * k] = a;
    lo[2 * k + 1] = b;
    decode4<CODE>(x[k + 2], scale, a, b);
    hi[2 * k] = a;
    hi[2 * k + 1] = b;
  }
}

// load_row_frags for a row of codes: 16 bytes a lane, the halves of the wave then change what the other's operands want.  (Scores of 35 rows of 128 units on 2464
// slots 15.5 us instead of 16.9 with eight bytes a lane.  With head_dim 64 eight bytes are taken: 10.2 instead of 11.4, 40 rows of 128 units on 2500.)
template <int D, int CODE>
__device__ __forceinline__ void decode_row_frags(bf16x8 (&f)[D / 16], const uint8_t *row, const uint8_t *scales, int hf) {
  u32x4 x[D / 32];
#pragma unroll
  for (int j = 0; j < D / 32; ++j) {
    if (D == 128) {
      x[j] = *reinterpret_cast<const u32x4 *>(row + 32 * j + 16 * hf);
    } else {
      const uint2 a = *reinterpret_cast<const uint2 *>(row + 32 * j + 8 * hf), z = *reinterpret_cast<const uint2 *>(row + 32 * j + 16 + 8 * hf);
      x[j] = u32x4{a.x, a.y, z.x, z.y};
    }
  }
  uint32_t s;
  if (D == 128) s = *reinterpret_cast<const uint32_t *>(scales);
  else s = *reinterpret_cast<const uint16_t *>(scales);
#pragma unroll
  for (int j = 0; j < D / 32; ++j) {
    const float scale = __uint_as_float((s >> (8 * j) & 255u) << 23);
    u32x4 w[2];  // elements 32 j + 8 hf .. +7 and 32 j + 16 + 8 hf .. +7
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      uint32_t y[2] = {x[j][k], x[j][2 + k]};
      if (D == 128) {
        const auto swapped = __builtin_amdgcn_permlane32_swap(y[0], y[1], false, false);
        y[0] = swapped[0];
        y[1] = swapped[1];
      }
#pragma unroll
      for (int o = 0; o < 2; ++o) {
        uint32_t lo, hi;
        decode4<CODE>(y[o], scale, lo, hi);
        w[o][2 * k] = lo;
        w[o][2 * k + 1] = hi;
      }
    }
    f[2 * j] = __builtin_bit_cast(bf16x8, w[0]);
    f[2 * j + 1] = __builtin_bit_cast(bf16x8, w[1]);
  }
}

// The scales of the first `rows` rows from `base` on, as row_buffer has rows.
template <int D>
__device__ __forceinline__ RowBuffer scale_buffer(const uint8_t *base, int rows) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(base), 0, __builtin_amdgcn_readfirstlane((rows > 0 ? rows : 0) * (D / kCodeBlock)), 0x00027000);
}

// ---- rows of a cache as bf16 -------------------------------------------------------------------------------------------
struct ReadParams {
  ChunkCache c;
  const int32_t *first;  // [Nb] or null: 0
  uint16_t *K, *V;       // [Nb][Hkv][n_rows][D]
  int n_rows;
};

constexpr int kReadThreads = 256;

// Slots first[b] + i of every unit to row i, those that the sequence has; a copy, bound by HBM.  grid (ceil(n_rows * D / 8 / 256 / 2), Hkv, Nb), eight elements of
// K and V a thread, so that a wave's stores are whole lines, and twice.  PAST: stores go past the caches, for a reader that comes later.  (1900 rows of 128 units, 189 MB: 28 us,
// 6.7 TB/s, part of it from the memory-side cache; before a long chunk, 2764 rows of them, 274 MB, 44 us.)
constexpr int kReadAtOnce = 2;
template <int D, int CODE, bool PAST>
__global__ __launch_bounds__(kReadThreads) void read_rows_kernel(const ReadParams p) {
  const ChunkCache &c = p.c;
  constexpr int LPR = D / 8, ROWS = kReadThreads / LPR;
  const int h = blockIdx.y, b = blockIdx.z, piece = threadIdx.x % LPR;
  int n = c.seq_len[b];
  n = n < c.cap ? n : c.cap;
  const long long first = p.first ? p.first[b] : 0;
  const int i0 = (int)blockIdx.x * (ROWS * kReadAtOnce) + threadIdx.x / LPR;
  const size_t unit = (size_t)b * c.Hkv + h;
  u32x4 x[kReadAtOnce][2];
  uint32_t s[kReadAtOnce][2];
  bool has[kReadAtOnce];
#pragma unroll
  for (int u = 0; u < kReadAtOnce; ++u) {
    const int i = i0 + u * ROWS;
    const long long slot = first + i;
    has[u] = i < p.n_rows && slot >= 0 && slot < n;
    if (!has[u]) continue;
    const size_t row = c.block_table ? paged_row<1>(c.block_table + unit * c.max_pages, (int)slot, c.max_pages, c.n_pages) : unit * (size_t)c.cap + (size_t)slot;
    const size_t src = row * D + 8 * piece;
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      const uint16_t *from = kv ? c.V : c.K;
      if (CODE) {
        const uint2 w = *reinterpret_cast<const uint2 *>(reinterpret_cast<const uint8_t *>(from) + src);
        x[u][kv][0] = w.x;
        x[u][kv][1] = w.y;
        s[u][kv] = (kv ? c.V_scale : c.K_scale)[src / kCodeBlock];
      } else {
        x[u][kv] = load_u32x4(from + src);
      }
    }
  }
#pragma unroll
  for (int u = 0; u < kReadAtOnce; ++u) {
    if (!has[u]) continue;
    const size_t dst = (unit * (size_t)p.n_rows + (i0 + u * ROWS)) * D + 8 * piece;
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      u32x4 y = x[u][kv];
      if (CODE) {
        const float scale = __uint_as_float(s[u][kv] << 23);
        uint32_t lo, hi;
        decode4<CODE>(x[u][kv][0], scale, lo, hi);
        y[0] = lo;
        y[1] = hi;
        decode4<CODE>(x[u][kv][1], scale, lo, hi);
        y[2] = lo;
        y[3] = hi;
      }
      u32x4 *to = reinterpret_cast<u32x4 *>((kv ? p.V : p.K) + dst);
      if (PAST) __builtin_nontemporal_store(y, to);
      else *to = y;
    }
  }
}

// ---- eviction: as compact_kernel, rows of D bytes and their scales --------------------------------------------------------
// grid (6, Hkv, Nb): K's codes, V's, K's scales, V's, S, pos.  PAGED leaves seq_len to paged_trim_kernel.  Bound by HBM: 128 units, 1920 of 2432 rows kept, 130 MB, 22.5 us
// (compact_kernel on the same rows in bf16 46).
template <int D, bool PAGED, int THREADS>
__global__ __launch_bounds__(THREADS) void coded_compact_kernel(const CompactParams p, const ChunkCache c) {
  const int tid = threadIdx.x, what = blockIdx.x, h = blockIdx.y, b = blockIdx.z;
  __shared__ int32_t sm_keep[compact_keep(THREADS)], sm_first[THREADS / 64];
  if (p.trigger && !p.trigger[b]) return;
  const size_t unit = (size_t)b * p.Hkv + h;
  const int32_t *tb = PAGED ? c.block_table + unit * c.max_pages : nullptr;
  const auto keep = take_keep_list<THREADS>(p, (int)unit, b, sm_keep, sm_first);
  const int m = keep.m, first = keep.first;
  auto row_of = [&](int slot) { return PAGED ? paged_row<1>(tb, slot, c.max_pages, c.n_pages) : unit * (size_t)p.cap + (size_t)slot; };

  // elements of type T, `per` of them a row, kUnroll rows a thread and pass; the in-place argument is compact_kernel's
  auto move = [&](auto *base, auto row, auto PER, auto UNROLL) {
    using T = typename std::remove_reference<decltype(*base)>::type;
    constexpr int per = decltype(PER)::value, kUnroll = decltype(UNROLL)::value, ROWS = THREADS / per, TILE = ROWS * kUnroll;
    const int r = tid / per, piece = tid % per;
    T cur[kUnroll], nxt[kUnroll];
    // (rows past the end read slot 0 and are never stored)
    auto fetch = [&](T (&x)[kUnroll], int i0) {
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const int i = i0 + u * ROWS + r;
        x[u] = base[row(i < m ? keep.source(i) : 0) * per + piece];
      }
    };
    if (first < m) fetch(cur, first);
    for (int i0 = first; i0 < m; i0 += TILE) {
      fetch(nxt, i0 + TILE);
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) arrived(cur[u]);
      __syncthreads();
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const int i = i0 + u * ROWS + r;
        if (i < m) base[row(i) * per + piece] = cur[u];
      }
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) cur[u] = nxt[u];
    }
  };
  using Scales = std::conditional_t<D == 128, uint32_t, uint16_t>;
  auto flat = [&](int slot) { return unit * (size_t)p.cap + (size_t)slot; };
  constexpr std::integral_constant<int, 1> kOne{};
  constexpr std::integral_constant<int, 2048 / THREADS> kMany{};
  constexpr std::integral_constant<int, kCompactUnroll> kRows{};
  if (what < 2) move(reinterpret_cast<u32x4 *>(what ? c.V : c.K), row_of, std::integral_constant<int, D / 16>{}, kRows);
  else if (what < 4) move(reinterpret_cast<Scales *>(what == 3 ? c.V_scale : c.K_scale), row_of, kOne, kMany);
  else move(what == 4 ? reinterpret_cast<uint32_t *>(p.S) : reinterpret_cast<uint32_t *>(p.pos), flat, kOne, kMany);
  if (!PAGED && what == 4 && h == 0 && tid == 0) p.seq_len[b] = m;
}

}  // namespace dynts
