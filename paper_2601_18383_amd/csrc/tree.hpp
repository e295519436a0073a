// Drafts whose tokens branch: who sees whom, and the accepted path's way back into the cache.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "chunk.hpp"
#include "codes.hpp"
#include "compact.hpp"
#include "forms.hpp"

namespace dynts {

constexpr int kTreeThreads = 256;

struct TreeBuildParams {
  const int32_t *parents;  // [Nb][T]
  const int32_t *n_new;    // [Nb] or null: T
  uint32_t *seen;          // [Nb][T][words]
  int32_t *depth;          // [Nb][T] or null
  int T, words;
};

// A token's ancestors and itself as bits: seen_i = {i} + seen_parent(i), followed upwards from every token by a thread of its own (parents lie before their
// children, so a token's words are complete from the last to the first).  grid (ceil(T / 256), Nb), LDS for T words.  Once a draft, for all layers: 3.0 us for 16 tokens of
// 32 sequences, which is a launch; a chain of T tokens is T steps of its last thread.
__global__ __launch_bounds__(kTreeThreads) void tree_build_kernel(const TreeBuildParams p) {
  extern __shared__ int32_t sm_parent[];
  const int b = blockIdx.y, tid = threadIdx.x;
  const int32_t *parents = p.parents + (size_t)b * p.T;
  const int last = (int)(blockIdx.x + 1) * kTreeThreads < p.T ? (int)(blockIdx.x + 1) * kTreeThreads : p.T;
  for (int i = tid; i < last; i += kTreeThreads) {
    const int q = parents[i];
    sm_parent[i] = q < i ? q : -1;  // (one that is not before its child, or negative: the cache)
  }
  __syncthreads();
  const int i = blockIdx.x * kTreeThreads + tid;
  if (i >= p.T) return;
  int m = p.n_new ? p.n_new[b] : p.T;
  m = m < p.T ? m : p.T;
  uint32_t *row = p.seen + ((size_t)b * p.T + i) * p.words;
  int at = i < m ? i : -1, depth = -1;
  for (int w = p.words - 1; w >= 0; --w) {
    uint32_t bits = 0;
    while (at >= 32 * w) {
      bits |= 1u << (at - 32 * w);
      at = sm_parent[at];
      ++depth;
    }
    row[w] = bits;
  }
  if (p.depth) p.depth[(size_t)b * p.T + i] = depth < 0 ? 0 : depth;
}

struct TreeKeepParams {
  ChunkCache c;
  const uint32_t *seen;    // [Nb][T][words]
  const int32_t *leaf;     // [Nb]
  const int32_t *n_taken;  // [Nb] or null: T
  int32_t *n_kept;         // [Nb]
  const uint16_t *q;       // [Nb][T][Hq][D] or null
  const float *lse;        // [Nb][T][Hq] or null
  uint16_t *q_kept;
  float *lse_kept;
  int T, words;
};

constexpr int kKeepThreads = 512, kKeepUnroll = 2;

// Tokens that stay, the set bits of the leaf's words in order: their number, and which they are, in LDS (T words).  Called by all threads.
__device__ __forceinline__ int tree_path(const TreeKeepParams &p, int b, int m, int leaf, int32_t *source, uint32_t *words, int *count) {
  const int tid = threadIdx.x;
  const uint32_t *row = p.seen + ((size_t)b * p.T + leaf) * p.words;
  for (int w = tid; w < p.words; w += kKeepThreads) {
    const uint32_t bits = row[w];
    words[w] = m - 32 * w >= 32 ? bits : m - 32 * w > 0 ? bits & ((1u << (m - 32 * w)) - 1u) : 0u;
  }
  __syncthreads();
  for (int w = tid; w < p.words; w += kKeepThreads) {
    int before = 0;
    for (int v = 0; v < w; ++v) before += __popc(words[v]);
    uint32_t bits = words[w];
    while (bits) {
      source[before++] = 32 * w + __builtin_ctz(bits);
      bits &= bits - 1;
    }
    if (w == p.words - 1) *count = before;
  }
  __syncthreads();
  return *count;
}

// grid (1 + gathering workgroups, Nb).  Workgroup 0 of a sequence moves its rows: destinations in ascending order, a batch's sources read before its
// destinations are written; a kept token's source lies at or behind its destination, so no later batch's source is overwritten (as in compact_kernel).
// Positions stay: the slot of the k-th kept token had the k-th position already.  The others gather q and lse.  Bound by the chain leaf, words, rows: 5.2 us for 16 tokens of
// 32 sequences, 4 heads of 128, any of them the last that stays.
template <int D>
__global__ __launch_bounds__(kKeepThreads) void tree_keep_kernel(const TreeKeepParams p) {
  const ChunkCache &c = p.c;
  __shared__ int32_t source[kTreeMost];
  __shared__ uint32_t words[kTreeMost / 32];
  __shared__ int count;
  const int b = blockIdx.y, tid = threadIdx.x;
  int m = p.n_taken ? p.n_taken[b] : p.T;
  m = m < 0 ? 0 : (m > p.T ? p.T : m);
  const int leaf = p.leaf[b];
  const bool some = leaf >= 0 && leaf < m;

  if (blockIdx.x > 0) {
    if (!some) return;
    const int kept = tree_path(p, b, m, leaf, source, words, &count), threads = ((int)gridDim.x - 1) * kKeepThreads;
    const int from = ((int)blockIdx.x - 1) * kKeepThreads + tid, LPT = c.Hq * (D / 8);
    const size_t token0 = (size_t)b * p.T;
    if (p.q_kept)
      for (long long at = from; at < (long long)kept * LPT; at += threads) {
        const int k = (int)(at / LPT), piece = (int)(at - (long long)k * LPT);
        store_u32x4(p.q_kept + ((token0 + k) * LPT + piece) * 8, load_u32x4(p.q + ((token0 + source[k]) * LPT + piece) * 8));
      }
    if (p.lse_kept)
      for (long long at = from; at < (long long)kept * c.Hq; at += threads) {
        const int k = (int)(at / c.Hq), hq = (int)(at - (long long)k * c.Hq);
        p.lse_kept[(token0 + k) * c.Hq + hq] = p.lse[(token0 + source[k]) * c.Hq + hq];
      }
    return;
  }

  int n = c.seq_len[b];
  n = n < 0 ? 0 : (n > c.cap ? c.cap : n);
  const int pos = c.next_pos[b];
  m = m < n ? m : n;
  const int base = n - m;
  const bool keeps = some && leaf < m;
  const int kept = keeps ? tree_path(p, b, m, leaf, source, words, &count) : 0;
  int first = 0;  // (the tokens up to the first that is dropped stay where they are)
  for (int hi = kept; first < hi;) {
    const int mid = (first + hi) / 2;
    if (source[mid] == mid) first = mid + 1;
    else hi = mid;
  }

  // where slot j of head h lies, in rows
  auto row_of = [&](int h, int j) {
    const size_t unit = (size_t)b * c.Hkv + h;
    return c.block_table ? paged_row<1>(c.block_table + unit * c.max_pages, j, c.max_pages, c.n_pages) : unit * (size_t)c.cap + (size_t)j;
  };
  // item `at` of a pass: piece at % per of head (at / per) % Hkv of kept token first + at / per / Hkv
  auto move = [&](auto *K, auto *V, int per, bool flat) {
    using T = typename std::remove_reference<decltype(*K)>::type;
    const int items = (kept - first) * c.Hkv * per;  // (below 2^12 * 2^7 * 2^4)
    for (int i0 = 0; i0 < items; i0 += kKeepThreads * kKeepUnroll) {
      T k[kKeepUnroll], v[kKeepUnroll];
      size_t to[kKeepUnroll];
#pragma unroll
      for (int u = 0; u < kKeepUnroll; ++u) {
        int at = i0 + u * kKeepThreads + tid;
        at = at < items ? at : items - 1;
        const int piece = at % per, rest = at / per, h = rest % c.Hkv, i = first + rest / c.Hkv;
        const size_t unit = (size_t)b * c.Hkv + h;
        const size_t from = (flat ? unit * (size_t)c.cap + base + source[i] : row_of(h, base + source[i])) * per + piece;
        to[u] = (flat ? unit * (size_t)c.cap + base + i : row_of(h, base + i)) * per + piece;
        k[u] = K[from];
        v[u] = V[from];
      }
#pragma unroll
      for (int u = 0; u < kKeepUnroll; ++u) {
        arrived(k[u]);
        arrived(v[u]);
      }
      __syncthreads();
#pragma unroll
      for (int u = 0; u < kKeepUnroll; ++u)
        if (i0 + u * kKeepThreads + tid < items) {
          K[to[u]] = k[u];
          V[to[u]] = v[u];
        }
    }
  };
  if (c.code) {
    move(reinterpret_cast<u32x4 *>(c.K), reinterpret_cast<u32x4 *>(c.V), D / 16, false);
    using Scales = std::conditional_t<D == 128, uint32_t, uint16_t>;
    move(reinterpret_cast<Scales *>(c.K_scale), reinterpret_cast<Scales *>(c.V_scale), 1, false);
  } else {
    move(reinterpret_cast<u32x4 *>(c.K), reinterpret_cast<u32x4 *>(c.V), D / 8, false);
  }
  move(c.S, c.S, 1, true);

  // pages past the new length go back, all of a sequence's at once
  const int end = base + kept, keep_pages = (end + kPageSlots - 1) / kPageSlots;
  int old_pages = (n + kPageSlots - 1) / kPageSlots;
  old_pages = old_pages < c.max_pages ? old_pages : c.max_pages;
  const int less = c.block_table ? old_pages - keep_pages : 0;
  if (less > 0) {
    __syncthreads();
    if (tid == 0) count = atomicAdd(c.free_top, less * c.Hkv);
    __syncthreads();
    const int top = count;
    for (int at = tid; at < less * c.Hkv; at += kKeepThreads) {
      const int h = at / less, j = at - h * less;
      c.free_stack[top + at] = c.block_table[((size_t)b * c.Hkv + h) * c.max_pages + keep_pages + j];
    }
  }
  if (tid == 0) {
    c.seq_len[b] = end;
    c.next_pos[b] = pos - m + kept;
    p.n_kept[b] = kept;
    if (leaf < -1 || (leaf >= 0 && !keeps)) atomicOr(c.status, 16);
  }
}

}  // namespace dynts
