// A chunk's rows into the cache.  Two launches: one workgroup per sequence decides whether the chunk fits, takes the pages it needs and moves the
// lengths on; then one thread per 16 bytes copies (a copy, bound by HBM: 512 rows of 64 sequences, 8 heads of 128, 268 MB read and written, 48 us both).
// Small chunks are copied by the first launch.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "attend.hpp"
#include "chunk.hpp"
#include "codes.hpp"

namespace dynts {

struct ChunkAppendParams {
  ChunkCache c;
  const uint16_t *k_new, *v_new;  // [Nb][T][Hkv][D]
  const float *s_new;             // [Nb][T][Hkv] or null
  const int32_t *n_new;           // [Nb] or null: T
  int32_t *taken;                 // [Nb], out: tokens of each sequence that were appended
  int T;
  int question;                   // the tokens are question slots
  uint64_t hkv_magic;             // ceil(2^36 / Hkv)
};

constexpr int kAppendThreads = 256;
// Pieces of 16 bytes, K's, that the first launch copies itself: a workgroup has 16 a thread then.
constexpr int kAppendSmall = 16 * kAppendThreads;

// Pieces [from, ...) of sequence b, `step` apart: piece p is part p % (D / 8) of head (p / (D / 8)) % Hkv of token p / (D / 8) / Hkv.  AT_ONCE: four of them are asked for at a
// time where one workgroup has all: behind the stores of one the next would wait for a trip to memory (16 tokens of 32 sequences, 4 heads of 128, by one workgroup a sequence 5.0 us instead
// of 7.9).  CODE: the cache holds codes (codes.hpp).
constexpr int kAppendAtOnce = 4;
// Row `src` of a sequence's [T][Hkv]: its token.  (Below 2^27 rows, 2^20 tokens of 128 heads: the magic number is off by less than 2^7 / 2^36 of the quotient's step a row.)
__device__ __forceinline__ int append_token(int src, uint64_t magic) { return (int)((uint64_t)(uint32_t)src * magic >> 36); }
template <int D, int CODE, int AT_ONCE>
__device__ __forceinline__ void chunk_copy(const ChunkAppendParams &p, int b, int n, int m, int pos0, int from, int step) {
  constexpr int LPR = D / 8;
  const ChunkCache &c = p.c;
  const int end = m * c.Hkv * LPR;
  const size_t row0 = (size_t)b * p.T * c.Hkv;
  for (int first = from; first < end; first += AT_ONCE * step) {
    u32x4 k[AT_ONCE], v[AT_ONCE];
    float score[AT_ONCE];
    size_t row[AT_ONCE];  // in the cache
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
      const int at = first + u * step < end ? first + u * step : first;
      const int piece = at % LPR, src = at / LPR, i = append_token(src, p.hkv_magic), h = src - i * c.Hkv;
      k[u] = load_u32x4(p.k_new + (row0 + src) * D + 8 * piece);
      v[u] = load_u32x4(p.v_new + (row0 + src) * D + 8 * piece);
      score[u] = p.question ? INFINITY : 0.f;
      if (p.s_new && !p.question) score[u] = p.s_new[row0 + src];
      const size_t unit = (size_t)b * c.Hkv + h;
      row[u] = c.block_table ? paged_row<1>(c.block_table + unit * c.max_pages, n + i, c.max_pages, c.n_pages) : unit * (size_t)c.cap + (n + i);
    }
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
      const int at = first + u * step;
      if (at >= end) break;
      const int piece = at % LPR, src = at / LPR, i = append_token(src, p.hkv_magic), h = src - i * c.Hkv;
      const size_t dst = row[u] * D + 8 * piece;
      if (CODE) {
        encode8<CODE>(k[u], reinterpret_cast<uint8_t *>(c.K), c.K_scale, dst, piece);
        encode8<CODE>(v[u], reinterpret_cast<uint8_t *>(c.V), c.V_scale, dst, piece);
      } else {
        store_u32x4(c.K + dst, k[u]);
        store_u32x4(c.V + dst, v[u]);
      }
      if (piece == 0) {
        const size_t e = ((size_t)b * c.Hkv + h) * (size_t)c.cap + (n + i);
        c.S[e] = score[u];
        c.pos[e] = pos0 + i;
      }
    }
  }
}

// The same for tokens [i0, i1) of one head, by `threads` threads.
template <int D>
__device__ __forceinline__ void chunk_copy_head(const ChunkCache &c, const uint16_t *k_new, const uint16_t *v_new, const float *s_new, int T, int question,
                                                int b, int h, int n, int i0, int i1, int pos0, int tid, int threads) {
  constexpr int LPR = D / 8;
  const size_t unit = (size_t)b * c.Hkv + h;
  for (int at = i0 * LPR + tid; at < i1 * LPR; at += threads) {
    const int piece = at % LPR, i = at / LPR, slot = n + i;
    const size_t row = ((size_t)b * T + i) * c.Hkv + h, src = row * D + 8 * piece;
    size_t dst;
    if (c.block_table) dst = paged_row<D>(c.block_table + unit * c.max_pages, slot, c.max_pages, c.n_pages) + 8 * piece;
    else dst = (unit * (size_t)c.cap + slot) * D + 8 * piece;
    // (past the caches, as the outputs beside them: 512 tokens of 64 sequences, 8 heads of 64, 121 us a step instead of 126)
    __builtin_nontemporal_store(load_u32x4(k_new + src), reinterpret_cast<u32x4 *>(c.K + dst));
    __builtin_nontemporal_store(load_u32x4(v_new + src), reinterpret_cast<u32x4 *>(c.V + dst));
    if (piece == 0) {
      const size_t e = unit * (size_t)c.cap + slot;
      c.S[e] = question ? INFINITY : s_new ? s_new[row] : 0.f;
      c.pos[e] = pos0 + i;
    }
  }
}

// grid (Nb).  A chunk that does not fit leaves its sequence alone: status bit 0 (no room), 2 (no pages), 3 (a question behind thinking tokens).
template <int D, bool COPY, int CODE>
__device__ __forceinline__ void chunk_reserve(const ChunkAppendParams &p) {
  const ChunkCache &c = p.c;
  const int b = blockIdx.x, tid = threadIdx.x;
  __shared__ int sm_m, sm_top;
  const int n = c.seq_len[b], pos0 = c.next_pos[b];
  int m = p.n_new ? p.n_new[b] : p.T;
  m = m < 0 ? 0 : (m > p.T ? p.T : m);
  int refused = 0;
  if (n < 0 || n > c.cap || m > c.cap - n) refused = 1;
  else if (p.question && n > c.n_prompt[b]) refused = 8;
  if (m == 0) refused = 0;
  if (refused || n < 0 || n > c.cap) m = 0;
  const int have = (n + kPageSlots - 1) / kPageSlots;
  const int more = m > 0 && c.block_table ? (n + m + kPageSlots - 1) / kPageSlots - have : 0;  // pages per head
  if (tid == 0) {
    int top = 0;
    if (more > 0) {
      const int need = more * c.Hkv;
      top = __hip_atomic_load(c.free_top, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      // (taken all at once or not at all; a failed exchange means that another sequence has got its pages)
      while (top >= need && !__hip_atomic_compare_exchange_strong(c.free_top, &top, top - need, __ATOMIC_RELAXED, __ATOMIC_RELAXED,
                                                                  __HIP_MEMORY_SCOPE_AGENT)) {
      }
      if (top < need) refused = 4;
    }
    sm_m = refused ? 0 : m;
    sm_top = top;
    if (refused) atomicOr(c.status, refused);
  }
  __syncthreads();
  m = sm_m;
  if (m > 0 && more > 0) {
    const int top = sm_top;
    for (int at = tid; at < more * c.Hkv; at += kAppendThreads) {
      const int h = at / more, j = at - h * more;
      c.block_table[((size_t)b * c.Hkv + h) * c.max_pages + have + j] = c.free_stack[top - 1 - at];
    }
  }
  if (tid == 0) {
    p.taken[b] = m;
    if (m > 0) {
      c.seq_len[b] = n + m;
      c.next_pos[b] = pos0 + m;
      if (p.question) c.n_prompt[b] = n + m;
    }
  }
  if (COPY) {
    __syncthreads();  // (the pages above)
    chunk_copy<D, CODE, kAppendAtOnce>(p, b, n, m, pos0, tid, kAppendThreads);
  }
}
template <int D, bool COPY>
__global__ __launch_bounds__(kAppendThreads) void chunk_reserve_kernel(const ChunkAppendParams p) {
  chunk_reserve<D, COPY, 0>(p);
}
template <int D, int CODE>
__global__ __launch_bounds__(kAppendThreads) void coded_reserve_kernel(const ChunkAppendParams p) {
  chunk_reserve<D, true, CODE>(p);
}

// grid (ceil(T * Hkv * D / 8 / 256), Nb), behind chunk_reserve_kernel
template <int D>
__global__ __launch_bounds__(kAppendThreads) void chunk_copy_kernel(const ChunkAppendParams p) {
  const int b = blockIdx.y, m = p.taken[b];
  chunk_copy<D, 0, 1>(p, b, p.c.seq_len[b] - m, m, p.c.next_pos[b] - m, blockIdx.x * kAppendThreads + threadIdx.x, gridDim.x * kAppendThreads);
}
// The same for a cache of codes, a workgroup for kCodedTokens neighbouring tokens of one head: scales, scores and positions of 32 rows share a line, and are to leave
// from one L2 (token by token over the heads, as above, 512 of 64 sequences, 8 heads of 128, 54 us instead of 43, on other arrays in turn).
// grid (ceil(T / kCodedTokens) * Hkv, Nb).
template <int D>
constexpr int kCodedTokens = kAppendAtOnce * kAppendThreads / (D / 8);
template <int D, int CODE>
__global__ __launch_bounds__(kAppendThreads) void coded_copy_kernel(const ChunkAppendParams p) {
  constexpr int LPR = D / 8, TOKENS = kCodedTokens<D>, kStep = kAppendThreads / LPR;
  const ChunkCache &c = p.c;
  const int blocks = (int)gridDim.x / c.Hkv, h = (int)blockIdx.x / blocks, b = blockIdx.y, tid = threadIdx.x;
  const int i0 = ((int)blockIdx.x - h * blocks) * TOKENS, m = p.taken[b];
  if (i0 >= m) return;
  const int n = c.seq_len[b] - m, pos0 = c.next_pos[b] - m, piece = tid % LPR;
  const size_t unit = (size_t)b * c.Hkv + h;
  u32x4 k[kAppendAtOnce], v[kAppendAtOnce];
  size_t row[kAppendAtOnce];
#pragma unroll
  for (int u = 0; u < kAppendAtOnce; ++u) {
    int i = i0 + u * kStep + tid / LPR;
    i = i < m ? i : i0;
    const size_t src = (((size_t)b * p.T + i) * c.Hkv + h) * D + 8 * piece;
    k[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p.k_new + src));
    v[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p.v_new + src));
    row[u] = c.block_table ? paged_row<1>(c.block_table + unit * c.max_pages, n + i, c.max_pages, c.n_pages) : unit * (size_t)c.cap + (n + i);
  }
  for (int t = tid; t < TOKENS && i0 + t < m; t += kAppendThreads) {
    const size_t e = unit * (size_t)c.cap + (n + i0 + t);
    c.S[e] = p.question ? INFINITY : p.s_new ? p.s_new[((size_t)b * p.T + i0 + t) * c.Hkv + h] : 0.f;
    c.pos[e] = pos0 + i0 + t;
  }
#pragma unroll
  for (int u = 0; u < kAppendAtOnce; ++u) {
    if (i0 + u * kStep + tid / LPR >= m) break;
    encode8<CODE>(k[u], reinterpret_cast<uint8_t *>(c.K), c.K_scale, row[u] * D + 8 * piece, piece);
    encode8<CODE>(v[u], reinterpret_cast<uint8_t *>(c.V), c.V_scale, row[u] * D + 8 * piece, piece);
  }
}

}  // namespace dynts
