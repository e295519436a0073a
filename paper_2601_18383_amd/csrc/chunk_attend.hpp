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
#include "chunk_append.hpp"
#include "score_block.hpp"

namespace dynts {

// dynts_shaping in log2 units
struct ChunkShape {
  float cap, cap_in;      // softcap * log2 e, or 0; 2 * log2 e * scale / softcap
  float far_in;           // scale / softcap where the cap lies above kCapNear, else 0
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
  uint32_t g_magic;       // ceil(2^32 / G), 0 for G = 1
  // Keys of a row block cut into shares, a workgroup each, as many as there are kShareTiles tiles for, n_split at most: unnormalised outputs
  // and (shift, sum) of unit u, share s and row r in row (u * n_split + s) * Rpad + r; how many shares there are, in part_n[u * blocks + block].
  // (The host does not know the lengths: a short cache has one share, and its output is written straight away.)
  int n_split, Rpad;
  float *part_o, *part_ml;  // [..][D], [..][2]
  int32_t *part_n;
  // the chunk's rows, where they are still to be appended (as in ChunkAppendParams)
  const uint16_t *k_new, *v_new;
  const float *s_new;
  int question;
};

constexpr int kShareTiles = 16;  // least tiles of 32 slots in a share

// Workgroup to unit and block: a unit's blocks on one XCD (four units and fewer: on 8 / units of them, or XCDs would be idle; 256 rows of 2 units on 16000 slots
// 23 us instead of 56), block by block through `group` units at a time, so that those that have least
// to do (the first rows, the last slots) come last and fill what the others leave.  Attention, 4 units: 1024 tokens of 8 sequences, 32 heads on 8, 73 us
// instead of 82, 512 of 8 25 instead of 32, of 64 198 instead of 206.  (8 units 74, 29 and 206; all of them 74, 29 and 243: then the blocks that wait for HBM no longer
// run beside those that compute.)  Scores, all units: 2000 tokens of 16 sequences 297 us instead of 425, 1024 of 16 (28 on 4) on 2464 slots 380 instead of 474, 512 of
// 64 676 instead of 661.
__device__ __forceinline__ bool chunk_map(int group, int n_blk, int n_units, int &unit, int &blk) {
  const int id = blockIdx.x, xcd = id & 7, slot = id >> 3, per_xcd = (n_units + 7) >> 3;
  if (n_units <= 4) {
    const int bits = n_units > 2 ? 2 : n_units - 1;
    unit = xcd & ((1 << bits) - 1);
    blk = (slot << (3 - bits)) + (xcd >> bits);
    return unit < n_units && blk < n_blk;
  }
  group = group < per_xcd ? group : per_xcd;
  const int first = slot / (group * n_blk) * group, left = per_xcd - first, size = left < group ? left : group, rem = slot - first * n_blk;
  blk = rem / size;
  unit = (first + rem - blk * size) * 8 + xcd;
  return unit < n_units;
}
constexpr int kAllUnits = 0x7fffffff;

// This workgroup's share of the tiles of its rows, as [from, to); false: it has none.
__device__ __forceinline__ bool chunk_share(const ChunkAttendParams &p, int tiles, int split, int place, int &shares, int &from, int &to) {
  shares = 1;
  from = 0;
  to = tiles;
  if (p.n_split == 1) return true;
  shares = tiles / kShareTiles;
  shares = shares < 1 ? 1 : (shares < p.n_split ? shares : p.n_split);
  if (split == 0 && threadIdx.x == 0) p.part_n[place] = shares;
  if (split >= shares) return false;
  from = tiles * split / shares;  // (tiles below 2^18, shares 32 at most)
  to = tiles * (split + 1) / shares;
  return true;
}

constexpr int kChWaves = 4, kChThreads = kChWaves * 64;
constexpr int kChRows = 32 * kChWaves;  // query rows a workgroup
constexpr int kChTile = 32;             // slots staged at a time
constexpr float kChLimit = 1e18f;       // a lane's weights of a tile that sum to this or more raise the shift
constexpr int kNowhere = 0x7fffffff;    // a position that no key has
static_assert(kPageSlots % kChTile == 0, "a tile lies inside a page");

// New tokens of sequence b that are queries, and its length.
__device__ __forceinline__ int chunk_tokens(const ChunkCache &c, const int32_t *n_new, int T, int b, int &n) {
  n = c.seq_len[b];
  n = n < 0 ? 0 : (n > c.cap ? c.cap : n);
  int m = n_new ? n_new[b] : T;
  m = m < 0 ? 0 : (m > T ? T : m);
  return m < n ? m : n;
}

// The page that the table has for slot t (the same in every lane) of a unit.  The number comes by the scalar cache: by the vector caches it would be
// waited for behind every load in flight.
__device__ __forceinline__ int chunk_page(const ChunkCache &c, size_t unit, int t) {
  int pi = t / kPageSlots;
  pi = pi < c.max_pages ? pi : c.max_pages - 1;
  return *(const __attribute__((address_space(4))) int32_t *)(uintptr_t)(c.block_table + unit * c.max_pages + pi);
}
// Where slot t begins, in elements; page: chunk_page's, if there are pages.
template <int D>
__device__ __forceinline__ size_t chunk_tile(const ChunkCache &c, size_t unit, int t, int page) {
  return c.block_table ? ((size_t)safe_page(page, c.n_pages) * kPageSlots + t % kPageSlots) * D : (unit * (size_t)c.cap + t) * D;
}

// Byte of LDS at which 16-byte piece `piece` of row `row` of a tile lies.  The pieces of a row are permuted so that what is read together lies in
// different banks: 16 rows of one piece (K operands), and 4 rows of 4 neighbouring pieces (V operands).
template <int D>
__device__ __forceinline__ int chunk_lds(int row, int piece) {
  const int f = D == 128 ? (row & 3) << 2 | ((row >> 2) & 3) : ((row >> 1) & 1) << 2 | ((row >> 2) & 3);
  return row * (2 * D) + 16 * (piece ^ f);
}

// LDS by its address, so that what differs between a lane's reads is a constant in the instruction.
typedef __attribute__((address_space(3))) const u32x4 LdsPiece;
typedef __attribute__((address_space(3))) i16x4 LdsQuad;
__device__ __forceinline__ bf16x8 lds_piece(uint32_t at) { return __builtin_bit_cast(bf16x8, *(LdsPiece *)(uintptr_t)at); }
__device__ __forceinline__ bf16x8 lds_columns(uint32_t at, uint32_t further) {
  const i16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsQuad *)(uintptr_t)at), b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsQuad *)(uintptr_t)(at + further));
  return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

// 16 (or 4) bytes a lane from a buffer straight to LDS, lane after lane from `to` on (`to` and `further` the same in every lane).  The compiler does not know of these loads:
// who reads what they bring waits for them by s_waitcnt vmcnt, and whoever else reads it, behind a barrier.
__device__ __forceinline__ void lds_bring16(RowBuffer buf, uint32_t offset, uint32_t further, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(to), "v"(offset), "s"(buf), "s"(further) : "memory");
}
__device__ __forceinline__ void lds_bring4(RowBuffer buf, uint32_t offset, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(to), "v"(offset), "s"(buf) : "memory");
}

// The interval of positions that a token at position `own` sees, as its lower end and the distance to its upper one; first, last: its own, where given.
__device__ __forceinline__ void chunk_bounds(const ChunkShape &s, int first, int last, int own, int &lo, uint32_t &span) {
  int low = 0, high = own;
  if (s.window > 0) low = own - s.window + 1;
  if (s.first) low = first > low ? first : low;
  if (s.last) high = last;
  low = low < 0 ? 0 : low;
  high = high >= kNowhere ? kNowhere - 1 : high;
  if (high < low) low = high = kNowhere;
  lo = low;
  span = (uint32_t)high - (uint32_t)low;
}
__device__ __forceinline__ void chunk_interval(const ChunkShape &s, size_t at, int own, int &lo, uint32_t &span) {
  const int first = s.first ? s.first[at] : 0, last = s.last ? s.last[at] : 0;
  chunk_bounds(s, first, last, own, lo, span);
}

// The token a row belongs to (rows below 2^28).
__device__ __forceinline__ int chunk_token(int r, uint32_t magic) { return magic ? (int)__umulhi((uint32_t)r, magic) : r; }

// The first slot of [lo, hi) whose position is not below `target`, or hi (positions ascend along the cache): 64 of them looked at a time, by one wave.
__device__ __forceinline__ int slot_from(const int32_t *pos, int lo, int hi, int target, int lane) {
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

// The slots that rows of tokens [i0, i1] see, as [lo, hi), given the lowest and the highest position that one of them sees (kNowhere and -1: none) and
// the positions of slots 0 and n - 1.
__device__ __forceinline__ void chunk_range(const ChunkShape &s, const int32_t *pos, int n, int base, int i0, int i1, int first, int last, int head, int tail,
                                            int lane, int &lo, int &hi) {
  lo = 0;
  hi = base + i1 + 1;
  if (tail - head == n - 1) {  // (no gaps: nothing to look up)
    if (s.first || s.window > 0) lo = first <= head ? 0 : ((uint32_t)first - (uint32_t)head < (uint32_t)n ? first - head : n);
    if (s.last) hi = last < head ? 0 : ((uint32_t)last - (uint32_t)head < (uint32_t)n ? last - head + 1 : n);
    return;
  }
  if (s.first || s.window > 0) {
    // (two slots lie no further apart than their positions)
    const int slot = base + i0, d = pos[slot] - first;
    lo = d >= 0 ? slot_from(pos, d < slot ? slot - d : 0, slot, first, lane) : slot_from(pos, slot, n, first, lane);
  }
  if (s.last) hi = slot_from(pos, 0, n, last + 1, lane);
}

// cap * tanh(z), z = dot * scale / softcap, in log2 units, as cap - 2 cap / (1 + e^(2 z)): five operations, off by 6 half steps of the cap at most, wherever it lies
// (cap (1 - u) / (1 + u) with u = e^(-2 |z|): seven, off by 3; attention of 2048 tokens of 8 sequences, 32 heads on 8, 372 us and so 346, scores of 512
// tokens of 16 on 2464 slots, 28 on 4, 346 and so 307).
__device__ __forceinline__ float soft_cap(float dot, const ChunkShape &s) {
  return fmaf(-2.f * s.cap, __builtin_amdgcn_rcpf(1.f + fast_exp2(dot * s.cap_in)), s.cap);
}
// The same for a cap that may lie far above the logits, whose bits that form loses: where |z| < 0.3 the logit times the series of tanh(z) / z, to z^8 (the next
// term is half a step of 2^-24), elsewhere cap * (1 - 2 / (1 + e^(2 z))); off by 24 half steps of the logit at most.
__device__ __forceinline__ float soft_cap_far(float dot, float scale_log2, const ChunkShape &s) {
  const float z = dot * s.far_in, t = z * z;
  const float series = fmaf(t, fmaf(t, fmaf(t, fmaf(t, 62.f / 2835.f, -17.f / 315.f), 2.f / 15.f), -1.f / 3.f), 1.f);
  const float whole = s.cap * fmaf(-2.f, __builtin_amdgcn_rcpf(1.f + fast_exp2(dot * s.cap_in)), 1.f);
  return fabsf(z) < 0.3f ? dot * scale_log2 * series : whole;
}
// Caps up to here (log2 units: a softcap of 128) take the short form, whose error is 2^-14 then; above, a logit costs fifteen operations.  FAR: a kernel that
// knows both; those for few rows and few slots do, which far caps take at every size.  (Code for both cost the others registers: with a window scores 160 us
// instead of 149, capped 319 instead of 309, attention 336 instead of 332; in the forms with a bias alone, scores 263 instead of 253, attention 90.7 instead of 89.0.  A far cap takes attention of 2048 tokens of 8 sequences, 32 heads
// on 8, 1070 us, scores of 512 of 16 on 2464 slots, 28 on 4, 590.)
constexpr float kCapNear = 128.f * 1.4426950408889634f;
template <bool FAR>
__device__ __forceinline__ void soft_caps(f32x16 &x, float scale_log2, const ChunkShape &s) {
  if (!FAR || s.far_in == 0.f) {
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = soft_cap(x[e], s);
  } else {
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = soft_cap_far(x[e], scale_log2, s);
  }
}

// Eight neighbouring elements of an output row, and its lse, from their unnormalised values, shift and sum.
template <int D>
__device__ __forceinline__ void chunk_write(const ChunkAttendParams &p, size_t row, int d0, const float (&o)[8], float top, float sum) {
  const float inv = sum > 0.f ? 1.f / sum : 0.f;  // (a row that sees nothing: zeros, and -inf)
  store_u32x4(p.out + row * D + d0, u32x4{bf16_pack(o[0] * inv, o[1] * inv), bf16_pack(o[2] * inv, o[3] * inv), bf16_pack(o[4] * inv, o[5] * inv),
                                          bf16_pack(o[6] * inv, o[7] * inv)});
  if (p.lse && d0 == 0) p.lse[row] = sum > 0.f ? (top + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f : -INFINITY;
}

// ---- many rows: 32 of them a wave, four waves, which share the keys through LDS ----------------------------------------
template <int D>
struct ChunkLds {
  static constexpr int kTileBytes = kChTile * 2 * D;
  static constexpr int kPlace = 2 * kTileBytes + kChTile * 4;  // K, V and positions of a tile
  static constexpr int kPlaces = 3;
};
// Byte of LDS at which piece `piece` of V's row `row` lies (its operands are read four rows by four pieces; K's as chunk_lds has it).
template <int D>
__device__ __forceinline__ int chunk_lds_v(int row, int piece) {
  return row * (2 * D) + 16 * (piece ^ (D == 128 ? (row & 3) << 2 : ((row >> 1) & 1) << 2));
}

// Bound by instruction issue and by the clock that the matrix cores leave: 2048 queries on 16384 slots, 32 heads on 8 of 128, 584 GFLOP in 517 us, 1.13
// PFLOP/s (a product of 8192 x 8192 x 8192 reaches 1.27); the matrix cores are busy 57 % of the cycles, at 1.8 GHz.  Short prompts by HBM: 512
// tokens of 64 sequences into an empty cache move 0.8 GB in 235 us.
//   Three workgroups a compute unit (168 registers): with two and twice the rows a wave 640 us, with the next tile's products among a tile's weights 551.
//   Tiles by loads straight to LDS: through registers there is no room for three workgroups (1610 us, spilled).
//
// SHAPED: positions count, not slots.  BIASED: with a bias by distance (a form of its own: its operations cost the others registers).  APPEND (plain
// form): the chunk's own rows are not in the cache yet; they are read where the caller has them, and every workgroup copies those of its tokens at its
// end.  (Copied by a launch of their own before, 512 tokens of 64 sequences, 32 heads on 8: 244 us a step instead of 236, heads of 64 134 instead of
// 123, 28 on 4 of 32 sequences, 600 tokens, 122 instead of 123.)
template <int D, bool SHAPED, bool BIASED, bool APPEND>
__global__ __launch_bounds__(kChThreads, D == 128 ? 3 : 4) void chunk_attend_kernel(const ChunkAttendParams p) {
  using Lds = ChunkLds<D>;
  const ChunkCache &c = p.c;
  // Three tiles' places: one is worked on, one is on its way, one is being asked for.
  __shared__ __attribute__((aligned(1024))) char sm[Lds::kPlaces * Lds::kPlace];
  __shared__ int sm_range[2 * kChWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, hf = lane >> 5, r16 = lane & 15;
  int unit, blk;
  const int n_blk = (p.T * c.G + kChRows - 1) / kChRows;
  // (documents: which rows see most is not known, and units at once cost: means of eight draws, 470 tokens of 21 sequences on 1571 slots, 28 heads on 4, in
  // documents 71 us unit by unit, 90 four at a time, 75 two; 4096 of 2, 32 on 8, 102 / 102 / 101; first rows first 76 and 110)
  if (!chunk_map(SHAPED && p.shape.first ? 1 : 4, n_blk * p.n_split, c.Nb * c.Hkv, unit, blk)) return;
  const int split = blk / n_blk;
  blk -= split * n_blk;
  const int b = unit / c.Hkv, h = unit - b * c.Hkv;
  int n;
  const int m = chunk_tokens(c, p.n_new, p.T, b, n);
  const int R = m * c.G;
  blk = n_blk - 1 - blk;  // (the last rows see most)
  if (blk * kChRows >= R) return;
  const int base = n - m;  // the chunk's first slot

  const int row0 = blk * kChRows + wave * 32;
  const int r = row0 + col < R ? row0 + col : R - 1;
  const int tok = chunk_token(r, p.g_magic), g = r - tok * c.G;
  bf16x8 qf[D / 16];
  load_row_frags<D>(qf, reinterpret_cast<const char *>(p.q + (((size_t)b * p.T + tok) * c.Hq + (size_t)h * c.G + g) * D), hf);
  float slope = 0.f;
  if (BIASED) slope = p.shape.slope[h * c.G + g] * 1.4426950408889634f;

  // what the rows see: plain, slots [0, lim]; shaped, positions [lo, lo + span].  all_lo, all_hi: what all of the wave's rows see
  const int32_t *pos = c.pos + (size_t)unit * c.cap;
  int lim, own = 0, t_lo = 0, t_hi, all_lo = 0, all_hi, own_lo = 0;  // (own_lo: of the wave's first row)
  uint32_t span = 0;
  const int r1 = blk * kChRows + kChRows - 1;
  const int i0 = chunk_token(blk * kChRows, p.g_magic), i1 = chunk_token(r1 < R ? r1 : R - 1, p.g_magic);
  if (SHAPED) {
    own = pos[base + tok];
    const int head = pos[0], tail = pos[n - 1];
    chunk_interval(p.shape, (size_t)b * p.T + tok, own, lim, span);
    int first = lim, last = lim == kNowhere ? -1 : (int)(lim + span);
    all_lo = first;
    all_hi = last;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const int f = __shfl_xor(first, d), l = __shfl_xor(last, d), al = __shfl_xor(all_lo, d), ah = __shfl_xor(all_hi, d);
      first = f < first ? f : first;
      last = l > last ? l : last;
      all_lo = al > all_lo ? al : all_lo;
      all_hi = ah < all_hi ? ah : all_hi;
    }
    if (lane == 0) {
      sm_range[wave] = first;
      sm_range[kChWaves + wave] = last;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kChWaves; ++w) {
      first = sm_range[w] < first ? sm_range[w] : first;
      last = sm_range[kChWaves + w] > last ? sm_range[kChWaves + w] : last;
    }
    chunk_range(p.shape, pos, n, base, i0, i1, __builtin_amdgcn_readfirstlane(first), __builtin_amdgcn_readfirstlane(last), __builtin_amdgcn_readfirstlane(head),
                __builtin_amdgcn_readfirstlane(tail), lane, t_lo, t_hi);
    t_lo = t_lo / kChTile * kChTile;
    all_lo = __builtin_amdgcn_readfirstlane(all_lo);
    if (BIASED) own_lo = __builtin_amdgcn_readlane(own, 0);
  } else {
    lim = base + tok;
    t_hi = base + i1 + 1;
    all_hi = base + chunk_token(row0 < R ? row0 : R - 1, p.g_magic);
  }
  all_hi = __builtin_amdgcn_readfirstlane(all_hi);
  const int tiles = t_hi > t_lo ? (t_hi - t_lo + kChTile - 1) / kChTile : 0;
  int shares, from, to;
  if (!chunk_share(p, tiles, split, unit * n_blk + blk, shares, from, to)) return;
  const int t0 = __builtin_amdgcn_readfirstlane(t_lo + from * kChTile), t1 = __builtin_amdgcn_readfirstlane(t_lo + to * kChTile);

  f32x16 acc[D / 32];
  float nm = 1e30f, l = 0.f;  // the exponents' addend (minus the shift, a whole number of log2 units); the lane's share of the sum of weights
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[dt][e] = 0.f;

  // Staging, past the registers: a wave brings kInstr parts of 1 KB of either operand.  A lane's piece of a part is the one that belongs at byte
  // 16 * lane of it; its place in the row is the same for all of a lane's parts.  Rows past the cache's end repeat the last one.
  constexpr int PPR = D / 8, kInstr = Lds::kTileBytes / 1024 / kChWaves, kRowsPart = 1024 / (2 * D);
  const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)sm;
  const int my_row = wave * kRowsPart + lane / PPR;
  const uint32_t k_off = chunk_lds<D>(my_row, lane % PPR), v_off = chunk_lds_v<D>(my_row, lane % PPR);
  constexpr int kNext = kRowsPart * kChWaves;  // rows from a lane's part to its next one
  // rows `cached` and on of a tile: from k_new and v_new, where a token's heads lie side by side
  auto bring_fresh = [&](int t, int rows, int cached, uint32_t place) {
    const uint32_t pitch = (uint32_t)c.Hkv * 2 * D;
    const long long at = ((long long)b * p.T + t - base) * c.Hkv * D + (long long)h * D;
    const int bytes = __builtin_amdgcn_readfirstlane((int)(rows * pitch));
    const RowBuffer kb = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t *>(p.k_new + at), 0, bytes, 0x00027000);
    const RowBuffer vb = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t *>(p.v_new + at), 0, bytes, 0x00027000);
#pragma unroll
    for (int i = 0; i < kInstr; ++i) {
      const int row = my_row + i * kNext;
      if (row < cached) continue;
      const uint32_t off = (row < rows ? row : rows - 1) * pitch - my_row * (2 * D), to = place + 1024 * (wave + i * kChWaves);
      lds_bring16(kb, off + k_off, 0, to);
      lds_bring16(vb, off + v_off, 0, to + Lds::kTileBytes);
    }
  };
  // (the page of the next tile to bring: looked up a tile ahead)
  int page = c.block_table ? chunk_page(c, unit, t0) : 0;
  auto bring = [&](int t, uint32_t place) {
    if (t >= t1) return;
    const int this_page = page;
    int rows = n - t < kChTile ? n - t : kChTile, cached = kChTile;
    if (APPEND) {
      cached = base - t;
      if (cached < rows) bring_fresh(t, rows, cached, place);
      if (cached <= 0) return;
      rows = cached < rows ? cached : rows;
    }
    const size_t at = chunk_tile<D>(c, unit, t, this_page);
    if (c.block_table) page = chunk_page(c, unit, t + kChTile);
    const RowBuffer kb = row_buffer<D>(c.K + at, rows), vb = row_buffer<D>(c.V + at, rows);
#pragma unroll
    for (int i = 0; i < kInstr; ++i) {
      const uint32_t to = place + 1024 * (wave + i * kChWaves);
      if (rows == kChTile) {
        lds_bring16(kb, k_off, i * kNext * 2 * D, to);
        lds_bring16(vb, v_off, i * kNext * 2 * D, to + Lds::kTileBytes);
      } else {
        const int over = my_row + i * kNext - (rows - 1);
        if (APPEND && over > 0) continue;
        const uint32_t back = (over > 0 ? over : 0) * (2 * D);
        lds_bring16(kb, k_off + i * kNext * 2 * D - back, 0, to);
        lds_bring16(vb, v_off + i * kNext * 2 * D - back, 0, to + Lds::kTileBytes);
      }
    }
    if (SHAPED && wave == 0 && lane < kChTile) {
      const RowBuffer pb = row_buffer<2>(reinterpret_cast<const uint16_t *>(pos + t), rows);
      lds_bring4(pb, 4 * (lane < rows ? lane : rows - 1), place + 2 * Lds::kTileBytes);
    }
  };

  // this lane's operands in a place: K's row `col`, piece 2 ks + hf; V's rows r16 / 4 + 4 hf + .., columns 4 (r16 % 4) .. +3 of 16 (of which it then gets
  // column r16, of four rows)
  uint32_t k_at[D / 16], v_at[D / 32];
#pragma unroll
  for (int ks = 0; ks < D / 16; ++ks) k_at[ks] = lds + chunk_lds<D>(col, 2 * ks + hf);
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
    v_at[dt] = lds + Lds::kTileBytes + chunk_lds_v<D>(4 * hf + (r16 >> 2), 4 * dt + 2 * ((lane >> 4) & 1) + ((r16 >> 1) & 1)) + 8 * (r16 & 1);

  // Operands are read a few products ahead, in this order: left to itself the compiler reads one ahead, and every product waits for LDS (2048 queries on
  // 16384 slots, 32 heads on 8: 515 us instead of 541; half of the weights among the products of the other half: 549).
  constexpr int kAheadK = 3, kAheadV = 4;
  // raw products of the tile in a place
  auto products = [&](f32x16 &s, uint32_t place) {
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = 0.f;
    bf16x8 kf[kAheadK];
#pragma unroll
    for (int ks = 0; ks < kAheadK; ++ks) kf[ks] = lds_piece(k_at[ks] + place);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[ks % kAheadK], qf[ks], s, 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
      if (ks + kAheadK < D / 16) {
        kf[ks % kAheadK] = lds_piece(k_at[ks + kAheadK < D / 16 ? ks + kAheadK : 0] + place);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };
  // Logits of tile t from its products: shaped, and hidden keys' at -inf.  `scale` is still to be multiplied with them, 1 if they are log2 units already.
  const bool capped = SHAPED && p.shape.cap > 0.f;
  const float scale = capped || BIASED ? 1.f : p.scale_log2;
  auto shape = [&](f32x16 &s, int t, const int *tp) {
    if (SHAPED) {
      if (capped) soft_caps<false>(s, p.scale_log2, p.shape);
      const int first = __builtin_amdgcn_readfirstlane(tp[0]), last = __builtin_amdgcn_readfirstlane(tp[kChTile - 1]);
      if (BIASED) {
        const float c = capped ? 1.f : p.scale_log2;
        if (t + kChTile <= n && last - first == kChTile - 1 && last <= own_lo) {  // 32 positions without gaps, none behind a row's own
          const float bias = -slope * (float)(own - first - 4 * hf);
#pragma unroll
          for (int e = 0; e < 16; ++e) s[e] = fmaf(s[e], c, fmaf(slope, (float)(8 * (e >> 2) + (e & 3)), bias));
        } else {
#pragma unroll
          for (int e = 0; e < 16; ++e) s[e] = fmaf(-slope, fabsf((float)(own - tp[8 * (e >> 2) + 4 * hf + (e & 3)])), s[e] * c);
        }
      }
      if (first < all_lo || last > all_hi || t + kChTile > n) {
        asm volatile("; some keys are hidden");  // (a branch: the compiler would compare every key of every tile)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int key = 8 * (e >> 2) + 4 * hf + (e & 3), kp = t + key < n ? tp[key] : -1;
          if ((uint32_t)(kp - lim) > span) s[e] = -INFINITY;
        }
      }
    } else if (t + kChTile - 1 > all_hi) {
      asm volatile("; some keys are hidden");
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (t + 8 * (e >> 2) + 4 * hf + (e & 3) > lim) s[e] = -INFINITY;
    }
  };
  // weights of a tile from its logits, with the shift at hand, and their sum
  auto fold = [&](const f32x16 &s, bf16x8 (&pf)[2]) {
    float q[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      float w[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        w[e] = fast_exp2(fmaf(s[4 * k + e], scale, nm));
        pf[k >> 1][4 * (k & 1) + e] = (__bf16)w[e];  // (half a step of 2^-8, as the output's rounding)
      }
      q[k] = (w[0] + w[1]) + (w[2] + w[3]);
    }
    return (q[0] + q[1]) + (q[2] + q[3]);
  };
  // the shift that takes the weight of the tile's largest logit to between 1/2 and 1, if it is above the one at hand
  auto above = [&](const f32x16 &s) {
    float mx = s[0];
#pragma unroll
    for (int e = 1; e < 16; ++e) mx = fmaxf(mx, s[e]);
    mx = fmaxf(mx, __shfl_xor(mx, 32));
    return fminf(floorf(-mx * scale), nm);
  };
  // the weights with the shift raised where the tile's logits lie far above it, or are the first
  auto weigh = [&](const f32x16 &s, bf16x8 (&pf)[2], auto FIRST) {
    if (decltype(FIRST)::value) {
      nm = above(s);
      l = fold(s, pf);
      return;
    }
    float sum = fold(s, pf);
    if (__any(!(sum < kChLimit))) {
      const float next = above(s), f = fast_exp2(next - nm);
      l *= f;
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt) acc[dt] *= f;
      nm = next;
      sum = fold(s, pf);
    }
    l += sum;
  };
  auto add_values = [&](const bf16x8 (&pf)[2], uint32_t place) {
    constexpr int N = 2 * (D / 32);
    auto columns = [&](int x) { return lds_columns(v_at[x % (D / 32)] + place + 16 * (x / (D / 32)) * (2 * D), 8 * (2 * D)); };
    bf16x8 vt[kAheadV];
#pragma unroll
    for (int x = 0; x < kAheadV; ++x) vt[x] = columns(x);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int x = 0; x < N; ++x) {
      acc[x % (D / 32)] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vt[x % kAheadV], pf[x / (D / 32)], acc[x % (D / 32)], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
      if (x + kAheadV < N) {
        vt[x % kAheadV] = columns(x + kAheadV);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };

  // One tile out of its place, while the tile after the next goes to the place that the last one has left.  Before the barrier a wave waits for
  // its own parts of the tile alone, those of the next one stay on their way (a __syncthreads would wait for all).
  constexpr int kWait = 0x0070;  // s_waitcnt of lgkmcnt(0) and vmcnt(0)
  auto tile = [&](int t, auto PLACE, auto FREE, auto FIRST) {
    constexpr uint32_t place = decltype(PLACE)::value * Lds::kPlace, free = decltype(FREE)::value * Lds::kPlace;
    if (t + kChTile >= t1) __builtin_amdgcn_s_waitcnt(kWait);
    else if (SHAPED && wave == 0) __builtin_amdgcn_s_waitcnt(kWait + 2 * kInstr + 1);
    else __builtin_amdgcn_s_waitcnt(kWait + 2 * kInstr);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    bring(t + 2 * kChTile, lds + free);
    f32x16 s;
    products(s, place);
    const int *tp = reinterpret_cast<const int *>(sm + place + 2 * Lds::kTileBytes);
    shape(s, t, tp);
    bf16x8 pf[2];
    weigh(s, pf, FIRST);
    add_values(pf, place);
  };
  bring(t0, lds);
  bring(t0 + kChTile, lds + Lds::kPlace);
  // (the queries are waited for here: in the loop, every third tile would wait for all loads)
#pragma unroll
  for (int ks = 0; ks < D / 16; ++ks) asm volatile("" : "+v"(qf[ks]));
  constexpr std::integral_constant<int, 0> kA{};
  constexpr std::integral_constant<int, 1> kB{};
  constexpr std::integral_constant<int, 2> kC{};
  if (t0 < t1) tile(t0, kA, kC, std::true_type{});
  for (int t = t0 + kChTile; t < t1; t += 3 * kChTile) {
    tile(t, kB, kA, std::false_type{});
    if (t + kChTile < t1) tile(t + kChTile, kC, kB, std::false_type{});
    if (t + 2 * kChTile < t1) tile(t + 2 * kChTile, kA, kC, std::false_type{});
  }

  if (APPEND && split == 0) {  // the tokens whose first row is one of this workgroup's
    const int first = (blk * kChRows + c.G - 1) / c.G, last = (blk * kChRows + kChRows + c.G - 1) / c.G;
    chunk_copy_head<D>(c, p.k_new, p.v_new, p.s_new, p.T, p.question, b, h, base, first, last < m ? last : m, c.next_pos[b] - m, tid, kChThreads);
  }

  // sums of the two halves' keys; outputs row by row through LDS
  __syncthreads();
  const float sum = l + __shfl_xor(l, 32);
  if (shares > 1) {
    if (row0 + col >= R) return;
    const size_t prow = ((size_t)unit * p.n_split + split) * p.Rpad + row0 + col;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
      for (int e = 0; e < 16; e += 4)
        *reinterpret_cast<f32x4 *>(p.part_o + prow * D + 32 * dt + 2 * e + 4 * hf) =
            f32x4{acc[dt][e], acc[dt][e + 1], acc[dt][e + 2], acc[dt][e + 3]};
    if (hf == 0) *reinterpret_cast<float2 *>(p.part_ml + 2 * prow) = float2{-nm, sum};
    return;
  }
  const float inv = sum > 0.f ? 1.f / sum : 0.f;  // (a row that sees nothing: zeros, and -inf)
  char *const turn = sm + wave * (32 * 2 * D);
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int e = 0; e < 16; e += 4)
      *reinterpret_cast<uint2 *>(turn + chunk_lds<D>(col, 4 * dt + (e >> 2)) + 8 * hf) =
          uint2{bf16_pack(acc[dt][e] * inv, acc[dt][e + 1] * inv), bf16_pack(acc[dt][e + 2] * inv, acc[dt][e + 3] * inv)};
  // rows by their distance from the workgroup's first token: 32 bits
  const size_t first_row = ((size_t)b * p.T + i0) * c.Hq + (size_t)h * c.G;
  auto row_from = [&](int rr) {
    const int ri = chunk_token(rr, p.g_magic);
    return (uint32_t)((ri - i0) * c.Hq + (rr - ri * c.G));
  };
  if (p.lse && hf == 0 && row0 + col < R)
    (p.lse + first_row)[row_from(row0 + col)] = sum > 0.f ? (__builtin_amdgcn_logf(sum) - nm) * 0.6931471805599453f : -INFINITY;
  wave_lds_fence();
  uint16_t *const out = p.out + first_row * D;
#pragma unroll
  for (int k = 0; k < 32 * PPR / 64; ++k) {
    const int row = lane / PPR + k * (64 / PPR), piece = lane % PPR, rr = row0 + row;
    // (past the caches, which hold the keys: 512 tokens of 64 sequences, 32 heads on 8, 238 us instead of 243, 600 of 32, 28 on 4, 123 instead of 136)
    if (rr < R)
      __builtin_nontemporal_store(*reinterpret_cast<const u32x4 *>(turn + chunk_lds<D>(row, piece)),
                                  reinterpret_cast<u32x4 *>(out + (row_from(rr) * D + 8 * piece)));
  }
}

// ---- few rows: 32 of them a workgroup, its eight waves share out the keys --------------------------------------------------
// Bound by HBM (or the memory-side cache): every wave streams 32 slots at a time through registers and a part of LDS of its own, the next
// tile's loads in flight while it works on one, no barrier before the end.  There the waves' outputs are joined through LDS.  Four tokens of 32
// sequences on 2464 slots, 28 heads on 4 of 128: 161 MB in 35 us from HBM, 28 from the memory-side cache.
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
  if (!chunk_map(1, n_blk * p.n_split, c.Nb * c.Hkv, unit, blk)) return;
  const int split = blk / n_blk;  // (the blocks of one share side by side: they read the same keys)
  blk -= split * n_blk;
  const int b = unit / c.Hkv, h = unit - b * c.Hkv;
  int n;
  const int m = chunk_tokens(c, p.n_new, p.T, b, n);
  const int R = m * c.G, row0 = blk * kFewRows;
  if (row0 >= R) return;
  const int base = n - m;

  const int r = row0 + col < R ? row0 + col : R - 1;
  const int i = chunk_token(r, p.g_magic), g = r - i * c.G;
  const size_t qrow = ((size_t)b * p.T + i) * c.Hq + (size_t)h * c.G + g;
  bf16x8 qf[D / 16];
  load_row_frags<D>(qf, reinterpret_cast<const char *>(p.q + qrow * D), hf);

  const int32_t *pos = c.pos + (size_t)unit * c.cap;
  const int lim = base + i;
  int lo = 0, own = 0;
  uint32_t span = 0;
  float slope = 0.f;
  int t_lo = 0, t_hi;
  const int i0 = chunk_token(row0, p.g_magic), i1 = chunk_token(row0 + kFewRows - 1 < R ? row0 + kFewRows - 1 : R - 1, p.g_magic);
  if (SHAPED) {
    const int head = pos[0], tail = pos[n - 1];
    own = pos[base + i];
    chunk_interval(p.shape, (size_t)b * p.T + i, own, lo, span);
    if (p.shape.slope) slope = p.shape.slope[h * c.G + g] * 1.4426950408889634f;
    // the slots that some row sees (every wave has all rows)
    int first = lo, last = lo == kNowhere ? -1 : (int)(lo + span);
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const int f = __shfl_xor(first, d), l = __shfl_xor(last, d);
      first = f < first ? f : first;
      last = l > last ? l : last;
    }
    chunk_range(p.shape, pos, n, base, i0, i1, __builtin_amdgcn_readfirstlane(first), __builtin_amdgcn_readfirstlane(last), __builtin_amdgcn_readfirstlane(head),
                __builtin_amdgcn_readfirstlane(tail), lane, t_lo, t_hi);
    t_lo = t_lo / kFewTile * kFewTile;
  } else {
    t_hi = base + i1 + 1;
  }
  // this share's tiles, every kFewWaves'th of them this wave's
  const int tiles = t_hi > t_lo ? (t_hi - t_lo + kFewTile - 1) / kFewTile : 0;
  int shares, from, to;
  if (!chunk_share(p, tiles, split, unit * n_blk + blk, shares, from, to)) return;
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
    const RowBuffer buf = row_buffer<D>(pool + (rows > 0 ? chunk_tile<D>(c, unit, tile, c.block_table ? chunk_page(c, unit, tile) : 0) : 0), rows);
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
    const bool capped = SHAPED && p.shape.cap > 0.f;
    if (capped) soft_caps<true>(s, p.scale_log2, p.shape);
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int key = 8 * (e >> 2) + 4 * hf + (e & 3);
      if (SHAPED) {
        float x = capped ? s[e] : s[e] * p.scale_log2;
        const int kp = sm_pos[wave][key];
        x -= slope * fabsf((float)(own - kp));
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
      pf[e >> 3][e & 7] = (__bf16)w;  // (half a step of 2^-8, as the output's rounding; with the low part as well, as single steps have it, drafts of four
                                      // tokens 29.5 us instead of 28.4, 175 rows of 4 units on 16000 slots 27.2 instead of 24.8)
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
  if (shares == 1) {
    const int ri = chunk_token(rr, p.g_magic);
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
__global__ __launch_bounds__(kMergeThreads) void chunk_merge_kernel(const ChunkAttendParams p, int block_rows) {
  const ChunkCache &c = p.c;
  const int unit = blockIdx.y, b = unit / c.Hkv, h = unit - b * c.Hkv;
  int n;
  const int m = chunk_tokens(c, p.n_new, p.T, b, n);
  const int r = blockIdx.x * (kMergeThreads / (D / 8)) + threadIdx.x / (D / 8), d0 = 8 * (threadIdx.x % (D / 8));
  if (r >= m * c.G) return;
  const int shares = p.part_n[unit * (p.Rpad / block_rows) + r / block_rows];
  if (shares == 1) return;
  const size_t first = (size_t)unit * p.n_split * p.Rpad + r;
  float top = -INFINITY, sum = 0.f, o[8] = {};
  for (int s0 = 0; s0 < shares; s0 += 4) {  // four shares' loads at a time
    float2 ml[4];
    f32x4 a[4], z[4];
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const size_t prow = first + (size_t)(s0 + s < shares ? s0 + s : s0) * p.Rpad;
      ml[s] = *reinterpret_cast<const float2 *>(p.part_ml + 2 * prow);
      a[s] = *reinterpret_cast<const f32x4 *>(p.part_o + prow * D + d0);
      z[s] = *reinterpret_cast<const f32x4 *>(p.part_o + prow * D + d0 + 4);
    }
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      if (s0 + s >= shares || !(ml[s].y > 0.f)) continue;  // (a share without a key that the row sees)
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
  const int i = chunk_token(r, p.g_magic);
  chunk_write<D>(p, ((size_t)b * p.T + i) * c.Hq + (size_t)h * c.G + (r - i * c.G), d0, o, top, sum);
}

}  // namespace dynts
