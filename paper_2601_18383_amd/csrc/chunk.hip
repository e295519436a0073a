// Host side of the entry points for chunks of new tokens and rotary positions: argument checks, scratch layout and launches.
// Nothing here allocates device memory or synchronises the host.
#include "chunk.hpp"

#include <cfloat>
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
bool overlap(const void *a, size_t a_bytes, const void *b, size_t b_bytes) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + b_bytes && y < x + a_bytes;
}
int launch_status() { return hipGetLastError() == hipSuccess ? DYNTS_OK : DYNTS_EHIP; }

// scratch of a chunk's calls
struct ChunkPlan {
  bool few;          // chunk_attend_few_kernel
  int rows, blocks;  // query rows of a workgroup, row blocks of a unit
  int n_split, Rpad;
  size_t off_lse = 0, off_n = 0, off_ml = 0, off_o = 0, bytes = 0;
};

// Rows of partials that the shares of one call may leave.
constexpr long long kMostPartials = 65536;

// Which kernel, and into how many shares the keys of a row block are cut at most.  slots: how many a token can see; far_cap: only the one for few rows knows it.
//
// Few rows, F row blocks of 32, one workgroup a compute unit (two with head_dim 64): a row block is done in 5 + 5.8 us per 1000 slots; many rows, W
// of 128, three or four a compute unit: 4 + 21 us per 1000 slots.  us, few / many, each with its shares:
//   head_dim 128, 2 units: 16000 slots R = 256 23.1 / 27.9, R = 1024 39.4 / 37.6; 8 units: 1000 slots R = 4 10.9 / 24.1, R = 1024 14.2 / 25.6; 4500 slots R = 64
//     15.2 / 20.8, R = 512 27.2 / 29.5, R = 1024 36.8 / 36.8; 16000 slots R = 128 25.1 / 29.0, R = 256 37.7 / 36.1, R = 512 64.4 / 47.9
//   32 units: 200 slots R = 256 8.0 / 9.0, R = 512 14.4 / 9.3; 4500 slots R = 128 26.6 / 26.5, R = 256 37.8 / 35.5; 16000 slots R = 64 50.0 / 52.3, R = 128
//     68.4 / 58.4
//   128 units: R = 64 200 slots 8.0 / 8.8, 4500 52.3 / 58.7, 16000 184 / 197; R = 128 200 slots 14.5 / 9.2, 1000 26.3 / 26.1, 4500 89.7 / 68.8
//   512 units: R = 16 300 slots 19.1 / 17.2, 2600 120 / 124; R = 64 300 slots 32.3 / 18.2, 2600 140 / 126
//   head_dim 64: 2 units of 6000 slots R = 1024 15.1 / 20.4, R = 2048 20.9 / 25.2; 8 of 400 R = 304 6.3 / 9.9; 32 of 2000 R = 512 20.2 / 26.8, of 8000 R = 128
//     24.6 / 24.2; 128 of 400 R = 128 8.8 / 10.1, R = 256 14.9 / 10.8, of 2000 R = 128 21.0 / 24.6
// Shares, at least 512 slots each, until the chip is full; none on short caches, where joining them costs more, nor two of few rows of many units, which are
// bound by HBM.  us by their number:
//   few rows, head_dim 128: 8 units of 1000 slots 1 / 2 / 4: 12.6 / 13.0 / 12.9, of 4500 1 / 4 / 8 / 16: 33.0 / 16.7 / 14.6 / 14.4, of 16000 8 / 16 / 31: 24.0 /
//     21.7 / 24.2; R = 128, 32 units of 4500 1 / 2: 34.6 / 26.8; 64 units of 4000 1 / 2 / 4: 30.9 / 27.8 / 27.6; 128 units of 1200 1 / 2: 17.2 / 20.4, of 2464 28.1 /
//     32.0, of 4000 42.9 / 47.5; head_dim 64, 128 units of 6000 1 / 2: 30.8 / 35.2, 10 of 1500 9.9 / 10.4
//   many rows, W = 64, 4500 slots 1 / 4 / 8 / 16: 94.9 / 41.6 / 37.3 / 37.1, 1000 1 / 2: 24.8 / 28.1; W = 128 of 1000 1 / 2 / 4: 25.4 / 30.5 / 31.4; W = 256 of 4500
//     1 / 2 / 4: 97.8 / 84.7 / 84.4, of 1000 25.6 / 33.2 / 33.2; W = 16 of 16000 8 / 16 / 31: 50.9 / 35.4 / 36.4
ChunkPlan chunk_plan(const dynts_config &c, int n_tokens, int slots, bool far_cap = false) {
  ChunkPlan pl;
  const long long R = (long long)n_tokens * (c.n_q_heads / c.n_kv_heads), units = (long long)c.batch * c.n_kv_heads;
  const long long F = units * ((R + dynts::kFewRows - 1) / dynts::kFewRows), W = units * ((R + dynts::kChRows - 1) / dynts::kChRows);
  pl.few = far_cap || R <= dynts::kFewRows || (F <= (c.head_dim == 128 ? 256 : 512) && (R <= 2 * dynts::kFewRows || F * slots <= 1 << 20));
  pl.rows = pl.few ? dynts::kFewRows : dynts::kChRows;
  pl.blocks = (int)((R + pl.rows - 1) / pl.rows);
  pl.Rpad = pl.blocks * pl.rows;
  long long shares = slots / (32 * dynts::kShareTiles);
  if (pl.few) {
    shares = shares < 16 ? shares : 16;
    shares = shares < 256 / F ? shares : 256 / F;
    if (shares < 3 && units > 64) shares = 1;
  } else {
    shares = shares < 32 ? shares : 32;
    shares = shares < 512 / W ? shares : 512 / W;
  }
  if (slots < 1536) shares = 1;
  while (shares > 1 && units * pl.Rpad * shares > kMostPartials) --shares;
  pl.n_split = shares < 1 ? 1 : (int)shares;
  size_t off = align_up((size_t)c.batch * sizeof(int32_t));
  pl.off_lse = off;
  off += align_up((size_t)c.batch * n_tokens * c.n_q_heads * sizeof(float));
  // room for the shares of this and of every shorter chunk: of rows padded to either kernel's, in as many shares as the slots allow
  const long long padded = (R + dynts::kChRows - 1) / dynts::kChRows * dynts::kChRows, all = units * padded * (c.capacity / (32 * dynts::kShareTiles));
  const long long most = all < kMostPartials ? all : kMostPartials;
  pl.off_n = off;
  off += align_up((size_t)(most / dynts::kFewRows + 1) * sizeof(int32_t));
  pl.off_ml = off;
  off += align_up((size_t)most * 2 * sizeof(float));
  pl.off_o = off;
  off += align_up((size_t)most * c.head_dim * sizeof(float));
  pl.bytes = off;
  return pl;
}

// a cap that takes the longer form of soft_caps
bool far_cap(const dynts_shaping *s) { return s && s->softcap * kLog2E > dynts::kCapNear; }

ChunkPlan chunk_plan(const ChunkCache &c, int n_tokens, const dynts_shaping *shaping = nullptr) {
  dynts_config cfg{};
  cfg.batch = c.Nb; cfg.n_q_heads = c.Hq; cfg.n_kv_heads = c.Hkv; cfg.head_dim = c.D; cfg.capacity = c.cap;
  // (slots of a window: no more than its positions, those of the chunk's other tokens beside them)
  const long long seen = shaping && shaping->window > 0 ? (long long)shaping->window + n_tokens : c.cap;
  return chunk_plan(cfg, n_tokens, (int)(seen < c.cap ? seen : c.cap), far_cap(shaping));
}

// the factor of a logit's exponent, 2 z log2 e; infinite for a softcap below the smallest normal numbers
float cap_in(float softcap, float scale) { return 2.f * kLog2E * scale / softcap; }

int check_shaping(const dynts_shaping *s, float scale) {
  if (!s) return DYNTS_OK;
  if (!(s->softcap >= 0.f) || std::isinf(s->softcap) || s->window < 0) return DYNTS_EINVAL;
  if (s->softcap > 0.f && std::isinf(cap_in(s->softcap, scale))) return DYNTS_EINVAL;
  if (misaligned(s->slope, 4) || misaligned(s->first, 4) || misaligned(s->last, 4)) return DYNTS_EINVAL;
  return DYNTS_OK;
}

uint32_t group_magic(int G) { return G == 1 ? 0u : (uint32_t)(((1ull << 32) + G - 1) / G); }

bool shaped(const dynts_shaping *s) { return s && (s->softcap > 0.f || s->window > 0 || s->slope || s->first || s->last); }
bool shaped(const dynts::ChunkShape &s) { return s.cap > 0.f || s.window > 0 || s.slope || s.first || s.last; }
dynts::ChunkShape chunk_shape(const dynts_shaping *s, float scale) {
  dynts::ChunkShape out{};
  if (!s) return out;
  if (s->softcap > 0.f) {
    out.cap = std::fmin(s->softcap * kLog2E, FLT_MAX);
    out.cap_in = cap_in(s->softcap, scale);
    // (scale / softcap, or what is still not 0: then z is, and the logit stays as it is)
    if (far_cap(s)) out.far_in = std::fmax(scale / s->softcap, FLT_MIN);
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

// copy: false leaves the rows to chunk_attend_kernel
int launch_append(const ChunkCache &c, const uint16_t *k_new, const uint16_t *v_new, const float *s_new, int n_tokens,
                  const int32_t *n_new, int question, int32_t *taken, bool copy, hipStream_t st) {
  const dynts::ChunkAppendParams p{c, k_new, v_new, s_new, n_new, taken, n_tokens, question};
  const long long pieces = (long long)n_tokens * c.Hkv * (c.D / 8);
  const dim3 block(dynts::kAppendThreads);
  if (copy && pieces <= dynts::kAppendSmall) {
    if (c.D == 128) hipLaunchKernelGGL((dynts::chunk_reserve_kernel<128, true>), dim3(c.Nb), block, 0, st, p);
    else hipLaunchKernelGGL((dynts::chunk_reserve_kernel<64, true>), dim3(c.Nb), block, 0, st, p);
    return launch_status();
  }
  const dim3 grid((unsigned)((pieces + dynts::kAppendThreads - 1) / dynts::kAppendThreads), c.Nb);
  if (c.D == 128) {
    hipLaunchKernelGGL((dynts::chunk_reserve_kernel<128, false>), dim3(c.Nb), block, 0, st, p);
    if (copy) hipLaunchKernelGGL((dynts::chunk_copy_kernel<128>), grid, block, 0, st, p);
  } else {
    hipLaunchKernelGGL((dynts::chunk_reserve_kernel<64, false>), dim3(c.Nb), block, 0, st, p);
    if (copy) hipLaunchKernelGGL((dynts::chunk_copy_kernel<64>), grid, block, 0, st, p);
  }
  return launch_status();
}

// workgroups of `blocks` a unit as chunk_map has them, units rounded up to the 8 XCDs; 0 if a grid cannot hold their threads (2^32)
unsigned chunk_grid(const ChunkCache &c, long long blocks, int threads) {
  const long long units = (long long)c.Nb * c.Hkv, share = units > 4 ? 1 : units > 2 ? 2 : 8 / units;  // XCDs of a unit
  const long long wgs = (blocks + share - 1) / share * ((units + 7) / 8 * 8);
  return wgs >= (1LL << 32) / threads ? 0u : (unsigned)wgs;
}
unsigned attend_grid(const ChunkCache &c, const ChunkPlan &pl) {
  return chunk_grid(c, (long long)pl.blocks * pl.n_split, pl.few ? dynts::kFewThreads : dynts::kChThreads);
}
// Which kernel of chunk_scores.hpp.  C: chunks of 32 rows of a unit, W: workgroups of 64 slots, one a compute unit.  Few slots: 7 + C / 4 us a round of 256 of
// them; many: 4 + 0.8 C us while its W / 4 workgroups have a compute unit each.  us, few / many:
//   head_dim 128: C = 66, W = 168 21.9 / 60.4, W = 672 60.9 / 61.5; C = 219, W = 152 57.0 / 170, W = 512 97.6 / 184; C = 389, W = 432 100 / 304; C = 112,
//     W = 752 93.1 / 92.2, W = 1504 183 / 122; C = 14, W = 640 26.3 / 16.8; C = 2, W = 568 14.5 / 5.9
//   head_dim 64: C = 164, W = 78 23.1 / 128; C = 10, W = 64 6.0 / 10.9; C = 38, W = 288 15.7 / 29.8, W = 1152 38.2 / 40.2
bool scores_few(const ChunkCache &c, int n_tokens, const dynts_shaping *shaping) {
  if (far_cap(shaping)) return true;  // (the other one does not know it)
  const long long W = (long long)c.Nb * c.Hkv * ((c.cap + dynts::kCfKeys - 1) / dynts::kCfKeys);
  const long long C = ((long long)n_tokens * c.G + dynts::kSbChunk - 1) / dynts::kSbChunk;
  return W <= 256 ? C >= 8 : W <= 512 && C >= 32;
}
unsigned scores_grid(const ChunkCache &c, bool few) {
  return few ? chunk_grid(c, (c.cap + dynts::kCfKeys - 1) / dynts::kCfKeys, dynts::kCfWaves * 64)
             : chunk_grid(c, (c.cap + dynts::kCsKeys - 1) / dynts::kCsKeys, dynts::kSbWaves * 64);
}

template <int D, bool SHAPED>
void launch_attend_d(const dynts::ChunkAttendParams &p, const ChunkPlan &pl, unsigned grid, hipStream_t st) {
  if (pl.few) hipLaunchKernelGGL((dynts::chunk_attend_few_kernel<D, SHAPED>), dim3(grid), dim3(dynts::kFewThreads), 0, st, p);
  else if (SHAPED && p.shape.slope) hipLaunchKernelGGL((dynts::chunk_attend_kernel<D, SHAPED, SHAPED, false>), dim3(grid), dim3(dynts::kChThreads), 0, st, p);
  else if (!SHAPED && p.k_new) hipLaunchKernelGGL((dynts::chunk_attend_kernel<D, false, false, !SHAPED>), dim3(grid), dim3(dynts::kChThreads), 0, st, p);
  else hipLaunchKernelGGL((dynts::chunk_attend_kernel<D, SHAPED, false, false>), dim3(grid), dim3(dynts::kChThreads), 0, st, p);
  if (p.n_split > 1) {
    constexpr int rows = dynts::kMergeThreads / (D / 8);
    hipLaunchKernelGGL(dynts::chunk_merge_kernel<D>, dim3((p.T * p.c.G + rows - 1) / rows, p.c.Nb * p.c.Hkv), dim3(dynts::kMergeThreads), 0, st, p,
                       pl.rows);
  }
}

// rows to append on the way, or none
struct Fresh {
  const uint16_t *k_new = nullptr, *v_new = nullptr;
  const float *s_new = nullptr;
  int question = 0;
};

int launch_attend(const ChunkCache &c, const uint16_t *q, int n_tokens, const int32_t *n_new, const dynts_shaping *shaping, uint16_t *out,
                  float *lse, void *scratch, const Fresh &fresh, hipStream_t st) {
  const ChunkPlan pl = chunk_plan(c, n_tokens, shaping);
  char *const base = static_cast<char *>(scratch);
  const dynts::ChunkAttendParams p{c, q, n_new, out, lse, chunk_shape(shaping, c.scale), n_tokens, c.scale * kLog2E, group_magic(c.G), pl.n_split, pl.Rpad,
                                   reinterpret_cast<float *>(base + pl.off_o), reinterpret_cast<float *>(base + pl.off_ml),
                                   reinterpret_cast<int32_t *>(base + pl.off_n), fresh.k_new, fresh.v_new, fresh.s_new, fresh.question};
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

template <int D, bool SHAPED, bool BIASED>
void launch_scores_form(const dynts::ChunkScoreParams &p, bool few, unsigned grid, hipStream_t st) {
  if (few) hipLaunchKernelGGL((dynts::chunk_scores_few_kernel<D, SHAPED, BIASED>), dim3(grid), dim3(dynts::kCfWaves * 64), 0, st, p);
  else hipLaunchKernelGGL((dynts::chunk_scores_kernel<D, SHAPED, BIASED>), dim3(grid), dim3(dynts::kSbWaves * 64), 0, st, p);
}
template <int D>
void launch_scores_d(const dynts::ChunkScoreParams &p, bool few, unsigned grid, hipStream_t st) {
  if (shaped(p.shape) && p.shape.slope) launch_scores_form<D, true, true>(p, few, grid, st);
  else if (shaped(p.shape)) launch_scores_form<D, true, false>(p, few, grid, st);
  else launch_scores_form<D, false, false>(p, few, grid, st);
}

int launch_scores(const ChunkCache &c, const uint16_t *q, int n_tokens, const int32_t *n_new, const dynts_shaping *shaping, const float *lse,
                  float *dst, int accumulate, hipStream_t st) {
  const dynts::ChunkScoreParams p{c, q, n_new, lse, dst ? dst : c.S, chunk_shape(shaping, c.scale), n_tokens, dst ? 0 : 1, accumulate ? 1 : 0,
                                  c.scale * kLog2E, group_magic(c.G)};
  const bool few = scores_few(c, n_tokens, shaping);
  const unsigned grid = scores_grid(c, few);
  if (!grid) return DYNTS_EINVAL;
  if (c.D == 128) launch_scores_d<128>(p, few, grid, st);
  else launch_scores_d<64>(p, few, grid, st);
  return launch_status();
}

int check_tokens(int32_t n_tokens) { return n_tokens <= 0 || n_tokens > kMostTokens ? DYNTS_EINVAL : DYNTS_OK; }

}  // namespace

extern "C" {

size_t dynts_chunk_scratch_bytes(const dynts_config *cfg, int32_t n_tokens) {
  if (dynts::chunk_check_config(cfg) != DYNTS_OK || check_tokens(n_tokens) != DYNTS_OK) return 0;
  return chunk_plan(*cfg, n_tokens, cfg->capacity).bytes;
}

int dynts_chunk_append(dynts_ctx *ctx, int32_t layer, const uint16_t *k_new, const uint16_t *v_new, const float *s_new, int32_t n_tokens,
                       const int32_t *n_new, int32_t question, void *scratch, size_t scratch_bytes, void *stream) {
  ChunkCache c;
  int rc = dynts::chunk_cache(ctx, layer, &c);
  if (rc == DYNTS_OK) rc = check_tokens(n_tokens);
  if (rc == DYNTS_OK) rc = check_append(c, k_new, v_new, s_new, question);
  if (rc == DYNTS_OK) rc = check_scratch(scratch, scratch_bytes, chunk_plan(c, n_tokens).bytes);
  if (rc != DYNTS_OK) return rc;
  if (c.score_mode != DYNTS_SCORE_EXTERNAL) s_new = nullptr;
  return launch_append(c, k_new, v_new, s_new, n_tokens, n_new, question ? 1 : 0, static_cast<int32_t *>(scratch), true, static_cast<hipStream_t>(stream));
}

int dynts_chunk_attend(dynts_ctx *ctx, int32_t layer, const uint16_t *q, int32_t n_tokens, const int32_t *n_new, const dynts_shaping *shaping,
                       uint16_t *out, float *lse, void *scratch, size_t scratch_bytes, void *stream) {
  ChunkCache c;
  int rc = dynts::chunk_cache(ctx, layer, &c);
  if (rc == DYNTS_OK) rc = check_tokens(n_tokens);
  if (rc == DYNTS_OK) rc = check_shaping(shaping, c.scale);
  if (rc != DYNTS_OK) return rc;
  if (!q || !out) return DYNTS_ENULL;
  if (misaligned(q, 16) || misaligned(out, 16)) return DYNTS_EINVAL;
  rc = check_scratch(scratch, scratch_bytes, chunk_plan(c, n_tokens).bytes);
  if (rc != DYNTS_OK) return rc;
  const size_t q_bytes = (size_t)c.Nb * n_tokens * c.Hq * c.D * 2;
  if (overlap(out, q_bytes, q, q_bytes)) return DYNTS_EINVAL;
  return launch_attend(c, q, n_tokens, n_new, shaping, out, lse, scratch, Fresh{}, static_cast<hipStream_t>(stream));
}

int dynts_chunk_scores(dynts_ctx *ctx, int32_t layer, const uint16_t *q, int32_t n_tokens, const int32_t *n_new, const dynts_shaping *shaping,
                       const float *lse, float *dst, int32_t accumulate, void *stream) {
  ChunkCache c;
  int rc = dynts::chunk_cache(ctx, layer, &c);
  if (rc == DYNTS_OK) rc = check_tokens(n_tokens);
  if (rc == DYNTS_OK) rc = check_shaping(shaping, c.scale);
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
  if (rc == DYNTS_OK) rc = check_shaping(shaping, c.scale);
  if (rc == DYNTS_OK) rc = check_append(c, k_new, v_new, s_new, question);
  if (rc != DYNTS_OK) return rc;
  if (!q || !out) return DYNTS_ENULL;
  if (misaligned(q, 16) || misaligned(out, 16)) return DYNTS_EINVAL;
  const ChunkPlan pl = chunk_plan(c, n_tokens, shaping);
  rc = check_scratch(scratch, scratch_bytes, pl.bytes);
  if (rc != DYNTS_OK) return rc;
  hipStream_t st = static_cast<hipStream_t>(stream);
  int32_t *taken = static_cast<int32_t *>(scratch);
  const bool scores = c.score_mode == DYNTS_SCORE_ACCUMULATE && !question;
  if (!attend_grid(c, pl) || (scores && !scores_grid(c, scores_few(c, n_tokens, shaping)))) return DYNTS_EINVAL;  // (before the append)
  const size_t row = (size_t)c.Nb * n_tokens * c.D * 2, q_bytes = row * c.Hq, k_bytes = row * c.Hkv;
  if (overlap(out, q_bytes, q, q_bytes) || overlap(out, q_bytes, k_new, k_bytes) || overlap(out, q_bytes, v_new, k_bytes)) return DYNTS_EINVAL;
  if (scores && !lse) lse = reinterpret_cast<float *>(static_cast<char *>(scratch) + pl.off_lse);
  if (c.score_mode != DYNTS_SCORE_EXTERNAL) s_new = nullptr;
  question = question ? 1 : 0;
  const bool on_the_way = !pl.few && !shaped(shaping);
  rc = launch_append(c, k_new, v_new, s_new, n_tokens, n_new, question, taken, !on_the_way, st);
  if (rc == DYNTS_OK)
    rc = launch_attend(c, q, n_tokens, taken, shaping, out, lse, scratch, on_the_way ? Fresh{k_new, v_new, s_new, question} : Fresh{}, st);
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
  if (((long long)q_heads + (k ? k_heads : 0)) * r->head_dim > (1 << 28) || n_tokens >= dynts::kRotMaxTokens) return DYNTS_ESHAPE;
  if (misaligned(q, 16) || misaligned(q_out, 16) || (k && (misaligned(k, 16) || misaligned(k_out, 16)))) return DYNTS_EINVAL;
  const dynts::RotateParams p{q, k, q_out, k_out, positions, r->freq, r->axis, n_tokens, q_heads, k ? k_heads : 0, r->head_dim, r->n_pairs,
                              r->n_axes, inverse ? -1.f : 1.f};
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (r->pairing == DYNTS_PAIR_ADJACENT) hipLaunchKernelGGL((dynts::rotate_kernel<true>), dim3(n_tokens), dim3(dynts::kRotThreads), 0, st, p);
  else hipLaunchKernelGGL((dynts::rotate_kernel<false>), dim3(n_tokens), dim3(dynts::kRotThreads), 0, st, p);
  return launch_status();
}

}  // extern "C"
