// Host side of the entry points for chunks of new tokens and rotary positions: argument checks, scratch layout and launches.
// Nothing here allocates device memory or synchronises the host.
#include "chunk.hpp"

#include <cmath>

#include "chunk_append.hpp"
#include "chunk_attend.hpp"
#include "chunk_scores.hpp"
#include "rotate.hpp"

namespace {

using dynts::ChunkCache;

constexpr size_t kAlign = 256;
constexpr int kMostTokens = 1 << 20;
constexpr float kLog2E = 1.4426950408889634f;

size_t align_up(size_t v) { return (v + kAlign - 1) / kAlign * kAlign; }
bool misaligned(const void *p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to != 0; }
int launch_status() { return hipGetLastError() == hipSuccess ? DYNTS_OK : DYNTS_EHIP; }

// scratch of a chunk's calls
struct ChunkPlan {
  bool few;          // chunk_attend_few_kernel
  int blocks, n_split, Rpad;
  size_t off_lse = 0, off_ml = 0, off_o = 0, bytes = 0;
};

// At most this many workgroups take a share of a row block's keys.
constexpr int kMostShares = 512;

ChunkPlan chunk_plan(const dynts_config &c, int n_tokens) {
  ChunkPlan pl;
  const long long R = (long long)n_tokens * (c.n_q_heads / c.n_kv_heads), units = (long long)c.batch * c.n_kv_heads;
  pl.few = R <= 64;
  const int rows = pl.few ? dynts::kFewRows : dynts::kChRows;
  pl.blocks = (int)((R + rows - 1) / rows);
  pl.Rpad = pl.blocks * rows;
  pl.n_split = 1;
  if (pl.few) {
    const long long want = 256 / (units * pl.blocks), most = (c.capacity + 255) / 256;
    pl.n_split = (int)(want < most ? want : most);
    pl.n_split = pl.n_split < 1 ? 1 : pl.n_split;
  }
  size_t off = align_up((size_t)c.batch * sizeof(int32_t));
  pl.off_lse = off;
  off += align_up((size_t)c.batch * n_tokens * c.n_q_heads * sizeof(float));
  // (room for the shares of any shorter chunk, too)
  const long long most = (long long)kMostShares * dynts::kFewRows;
  pl.off_ml = off;
  off += align_up((size_t)most * 2 * sizeof(float));
  pl.off_o = off;
  off += align_up((size_t)most * c.head_dim * sizeof(float));
  pl.bytes = off;
  return pl;
}

ChunkPlan chunk_plan(const ChunkCache &c, int n_tokens) {
  dynts_config cfg{};
  cfg.batch = c.Nb; cfg.n_q_heads = c.Hq; cfg.n_kv_heads = c.Hkv; cfg.head_dim = c.D; cfg.capacity = c.cap;
  return chunk_plan(cfg, n_tokens);
}

int check_shaping(const dynts_shaping *s) {
  if (!s) return DYNTS_OK;
  if (!(s->softcap >= 0.f) || std::isinf(s->softcap) || s->window < 0) return DYNTS_EINVAL;
  if (misaligned(s->slope, 4) || misaligned(s->first, 4) || misaligned(s->last, 4)) return DYNTS_EINVAL;
  return DYNTS_OK;
}

uint32_t group_magic(int G) { return G == 1 ? 0u : (uint32_t)(((1ull << 32) + G - 1) / G); }

bool shaped(const dynts_shaping *s) { return s && (s->softcap > 0.f || s->window > 0 || s->slope || s->first || s->last); }

dynts::ChunkShape chunk_shape(const dynts_shaping *s, float scale) {
  dynts::ChunkShape out{};
  if (!s) return out;
  if (s->softcap > 0.f) {
    out.cap = s->softcap * kLog2E;
    out.cap_in = 2.f * kLog2E * scale / s->softcap;
  }
  out.window = s->window;
  out.slope = s->slope;
  out.first = s->first;
  out.last = s->last;
  return out;
}

int check_scratch(const void *scratch, size_t bytes, size_t need) {
  if (!scratch) return DYNTS_ENULL;
  return bytes < need || misaligned(scratch, kAlign) ? DYNTS_EWORKSPACE : DYNTS_OK;
}

int check_append(const ChunkCache &c, const uint16_t *k_new, const uint16_t *v_new, const float *s_new, int question) {
  if (!k_new || !v_new) return DYNTS_ENULL;
  if (c.score_mode == DYNTS_SCORE_EXTERNAL && !question && !s_new) return DYNTS_ENULL;
  if (misaligned(k_new, 16) || misaligned(v_new, 16)) return DYNTS_EINVAL;
  return DYNTS_OK;
}

int launch_append(const ChunkCache &c, const uint16_t *k_new, const uint16_t *v_new, const float *s_new, int n_tokens,
                  const int32_t *n_new, int question, int32_t *taken, hipStream_t st) {
  const dynts::ChunkAppendParams p{c, k_new, v_new, c.score_mode == DYNTS_SCORE_EXTERNAL ? s_new : nullptr, n_new, taken, n_tokens, question ? 1 : 0};
  const long long pieces = (long long)n_tokens * c.Hkv * (c.D / 8);
  const dim3 block(dynts::kAppendThreads);
  if (pieces <= dynts::kAppendSmall) {
    if (c.D == 128) hipLaunchKernelGGL((dynts::chunk_reserve_kernel<128, true>), dim3(c.Nb), block, 0, st, p);
    else hipLaunchKernelGGL((dynts::chunk_reserve_kernel<64, true>), dim3(c.Nb), block, 0, st, p);
    return launch_status();
  }
  const dim3 grid((unsigned)((pieces + dynts::kAppendThreads - 1) / dynts::kAppendThreads), c.Nb);
  if (c.D == 128) {
    hipLaunchKernelGGL((dynts::chunk_reserve_kernel<128, false>), dim3(c.Nb), block, 0, st, p);
    hipLaunchKernelGGL((dynts::chunk_copy_kernel<128>), grid, block, 0, st, p);
  } else {
    hipLaunchKernelGGL((dynts::chunk_reserve_kernel<64, false>), dim3(c.Nb), block, 0, st, p);
    hipLaunchKernelGGL((dynts::chunk_copy_kernel<64>), grid, block, 0, st, p);
  }
  return launch_status();
}

// workgroups of `blocks` a unit, units rounded up to the 8 XCDs; 0 if a grid cannot hold them (2^32 threads)
unsigned chunk_grid(const ChunkCache &c, long long blocks) {
  const long long wgs = blocks * (((long long)c.Nb * c.Hkv + 7) / 8 * 8);
  return wgs >= (1LL << 32) / 256 ? 0u : (unsigned)wgs;
}
unsigned attend_grid(const ChunkCache &c, const ChunkPlan &pl) { return chunk_grid(c, (long long)pl.blocks * pl.n_split); }
unsigned scores_grid(const ChunkCache &c) { return chunk_grid(c, (c.cap + dynts::kCsKeys - 1) / dynts::kCsKeys); }

template <int D, bool SHAPED>
void launch_attend_d(const dynts::ChunkAttendParams &p, const ChunkPlan &pl, unsigned grid, hipStream_t st) {
  if (pl.few) hipLaunchKernelGGL((dynts::chunk_attend_few_kernel<D, SHAPED>), dim3(grid), dim3(dynts::kFewThreads), 0, st, p);
  else hipLaunchKernelGGL((dynts::chunk_attend_kernel<D, SHAPED>), dim3(grid), dim3(dynts::kChThreads), 0, st, p);
  if (p.n_split > 1) {
    constexpr int rows = dynts::kMergeThreads / (D / 8);
    hipLaunchKernelGGL(dynts::chunk_merge_kernel<D>, dim3((p.T * p.c.G + rows - 1) / rows, p.c.Nb * p.c.Hkv), dim3(dynts::kMergeThreads), 0, st, p);
  }
}

int launch_attend(const ChunkCache &c, const uint16_t *q, int n_tokens, const int32_t *n_new, const dynts_shaping *shaping, uint16_t *out,
                  float *lse, void *scratch, hipStream_t st) {
  const ChunkPlan pl = chunk_plan(c, n_tokens);
  char *const base = static_cast<char *>(scratch);
  const dynts::ChunkAttendParams p{c, q, n_new, out, lse, chunk_shape(shaping, c.scale), n_tokens, c.scale * kLog2E, group_magic(c.G), pl.n_split, pl.Rpad,
                                   reinterpret_cast<float *>(base + pl.off_o), reinterpret_cast<float *>(base + pl.off_ml)};
  const unsigned grid = attend_grid(c, pl);
  if (!grid) return DYNTS_EINVAL;
  if (c.D == 128) {
    if (shaped(shaping)) launch_attend_d<128, true>(p, pl, grid, st);
    else launch_attend_d<128, false>(p, pl, grid, st);
  } else {
    if (shaped(shaping)) launch_attend_d<64, true>(p, pl, grid, st);
    else launch_attend_d<64, false>(p, pl, grid, st);
  }
  return launch_status();
}

int launch_scores(const ChunkCache &c, const uint16_t *q, int n_tokens, const int32_t *n_new, const dynts_shaping *shaping, const float *lse,
                  float *dst, int accumulate, hipStream_t st) {
  const dynts::ChunkScoreParams p{c, q, n_new, lse, dst ? dst : c.S, chunk_shape(shaping, c.scale), n_tokens, dst ? 0 : 1, accumulate ? 1 : 0,
                                  c.scale * kLog2E, group_magic(c.G)};
  const unsigned grid = scores_grid(c);
  if (!grid) return DYNTS_EINVAL;
  const dim3 block(dynts::kSbWaves * 64);
  if (c.D == 128) {
    if (shaped(shaping)) hipLaunchKernelGGL((dynts::chunk_scores_kernel<128, true>), dim3(grid), block, 0, st, p);
    else hipLaunchKernelGGL((dynts::chunk_scores_kernel<128, false>), dim3(grid), block, 0, st, p);
  } else {
    if (shaped(shaping)) hipLaunchKernelGGL((dynts::chunk_scores_kernel<64, true>), dim3(grid), block, 0, st, p);
    else hipLaunchKernelGGL((dynts::chunk_scores_kernel<64, false>), dim3(grid), block, 0, st, p);
  }
  return launch_status();
}

int check_tokens(int32_t n_tokens) { return n_tokens <= 0 || n_tokens > kMostTokens ? DYNTS_EINVAL : DYNTS_OK; }

}  // namespace

extern "C" {

size_t dynts_chunk_scratch_bytes(const dynts_config *cfg, int32_t n_tokens) {
  if (dynts::chunk_check_config(cfg) != DYNTS_OK || check_tokens(n_tokens) != DYNTS_OK) return 0;
  return chunk_plan(*cfg, n_tokens).bytes;
}

int dynts_chunk_append(dynts_ctx *ctx, int32_t layer, const uint16_t *k_new, const uint16_t *v_new, const float *s_new, int32_t n_tokens,
                       const int32_t *n_new, int32_t question, void *scratch, size_t scratch_bytes, void *stream) {
  ChunkCache c;
  int rc = dynts::chunk_cache(ctx, layer, &c);
  if (rc == DYNTS_OK) rc = check_tokens(n_tokens);
  if (rc == DYNTS_OK) rc = check_append(c, k_new, v_new, s_new, question);
  if (rc == DYNTS_OK) rc = check_scratch(scratch, scratch_bytes, chunk_plan(c, n_tokens).bytes);
  if (rc != DYNTS_OK) return rc;
  return launch_append(c, k_new, v_new, s_new, n_tokens, n_new, question, static_cast<int32_t *>(scratch), static_cast<hipStream_t>(stream));
}

int dynts_chunk_attend(dynts_ctx *ctx, int32_t layer, const uint16_t *q, int32_t n_tokens, const int32_t *n_new, const dynts_shaping *shaping,
                       uint16_t *out, float *lse, void *scratch, size_t scratch_bytes, void *stream) {
  ChunkCache c;
  int rc = dynts::chunk_cache(ctx, layer, &c);
  if (rc == DYNTS_OK) rc = check_tokens(n_tokens);
  if (rc == DYNTS_OK) rc = check_shaping(shaping);
  if (rc != DYNTS_OK) return rc;
  if (!q || !out) return DYNTS_ENULL;
  if (misaligned(q, 16) || misaligned(out, 16)) return DYNTS_EINVAL;
  rc = check_scratch(scratch, scratch_bytes, chunk_plan(c, n_tokens).bytes);
  if (rc != DYNTS_OK) return rc;
  return launch_attend(c, q, n_tokens, n_new, shaping, out, lse, scratch, static_cast<hipStream_t>(stream));
}

int dynts_chunk_scores(dynts_ctx *ctx, int32_t layer, const uint16_t *q, int32_t n_tokens, const int32_t *n_new, const dynts_shaping *shaping,
                       const float *lse, float *dst, int32_t accumulate, void *stream) {
  ChunkCache c;
  int rc = dynts::chunk_cache(ctx, layer, &c);
  if (rc == DYNTS_OK) rc = check_tokens(n_tokens);
  if (rc == DYNTS_OK) rc = check_shaping(shaping);
  if (rc != DYNTS_OK) return rc;
  if (!q || !lse) return DYNTS_ENULL;
  if (misaligned(q, 16)) return DYNTS_EINVAL;
  return launch_scores(c, q, n_tokens, n_new, shaping, lse, dst, accumulate, static_cast<hipStream_t>(stream));
}

int dynts_chunk_step(dynts_ctx *ctx, int32_t layer, const uint16_t *q, const uint16_t *k_new, const uint16_t *v_new, const float *s_new,
                     int32_t n_tokens, const int32_t *n_new, int32_t question, const dynts_shaping *shaping, uint16_t *out, float *lse,
                     void *scratch, size_t scratch_bytes, void *stream) {
  ChunkCache c;
  int rc = dynts::chunk_cache(ctx, layer, &c);
  if (rc == DYNTS_OK) rc = check_tokens(n_tokens);
  if (rc == DYNTS_OK) rc = check_shaping(shaping);
  if (rc == DYNTS_OK) rc = check_append(c, k_new, v_new, s_new, question);
  if (rc != DYNTS_OK) return rc;
  if (!q || !out) return DYNTS_ENULL;
  if (misaligned(q, 16) || misaligned(out, 16)) return DYNTS_EINVAL;
  const ChunkPlan pl = chunk_plan(c, n_tokens);
  rc = check_scratch(scratch, scratch_bytes, pl.bytes);
  if (rc != DYNTS_OK) return rc;
  hipStream_t st = static_cast<hipStream_t>(stream);
  int32_t *taken = static_cast<int32_t *>(scratch);
  const bool scores = c.score_mode == DYNTS_SCORE_ACCUMULATE && !question;
  if (!attend_grid(c, pl) || (scores && !scores_grid(c))) return DYNTS_EINVAL;  // (before the append)
  if (scores && !lse) lse = reinterpret_cast<float *>(static_cast<char *>(scratch) + pl.off_lse);
  rc = launch_append(c, k_new, v_new, s_new, n_tokens, n_new, question, taken, st);
  if (rc == DYNTS_OK) rc = launch_attend(c, q, n_tokens, taken, shaping, out, lse, scratch, st);
  if (rc == DYNTS_OK && scores) rc = launch_scores(c, q, n_tokens, taken, shaping, lse, nullptr, 1, st);
  return rc;
}

int dynts_rotate(const dynts_rotary *r, const uint16_t *q, int32_t q_heads, const uint16_t *k, int32_t k_heads, const int32_t *positions,
                 int32_t n_tokens, int32_t inverse, uint16_t *q_out, uint16_t *k_out, void *stream) {
  if (!r) return DYNTS_ENULL;
  if (r->pairing != DYNTS_PAIR_HALVES && r->pairing != DYNTS_PAIR_ADJACENT) return DYNTS_EINVAL;
  if (r->n_axes < 1 || r->n_pairs <= 0 || n_tokens < 0) return DYNTS_EINVAL;
  if (r->head_dim <= 0 || r->head_dim % 8 || r->n_pairs % 8 || r->head_dim < 2 * (long long)r->n_pairs || r->n_pairs > dynts::kRotMaxPairs)
    return DYNTS_ESHAPE;
  if (n_tokens == 0) return DYNTS_OK;
  if (!r->freq || !positions || !q || !q_out || (k && !k_out)) return DYNTS_ENULL;
  if (q_heads <= 0 || (k && k_heads <= 0)) return DYNTS_EINVAL;
  if (((long long)q_heads + (k ? k_heads : 0)) * r->head_dim > (1 << 28)) return DYNTS_ESHAPE;
  if (misaligned(q, 16) || misaligned(q_out, 16) || (k && (misaligned(k, 16) || misaligned(k_out, 16)))) return DYNTS_EINVAL;
  const dynts::RotateParams p{q, k, q_out, k_out, positions, r->freq, r->axis, n_tokens, q_heads, k ? k_heads : 0, r->head_dim, r->n_pairs,
                              r->n_axes, inverse ? -1.f : 1.f};
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (r->pairing == DYNTS_PAIR_ADJACENT) hipLaunchKernelGGL((dynts::rotate_kernel<true>), dim3(n_tokens), dim3(dynts::kRotThreads), 0, st, p);
  else hipLaunchKernelGGL((dynts::rotate_kernel<false>), dim3(n_tokens), dim3(dynts::kRotThreads), 0, st, p);
  return launch_status();
}

}  // extern "C"
