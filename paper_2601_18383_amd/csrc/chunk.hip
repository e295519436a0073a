// Host side of the entry points for chunks of new tokens and rotary positions: argument checks, scratch layout and launches.
// Nothing here allocates device memory or synchronises the host.
#include "chunk.hpp"

#include <cfloat>
#include <cmath>

#include "chunk_append.hpp"
#include "chunk_attend.hpp"
#include "chunk_scores.hpp"
#include "forms.hpp"
#include "rotate.hpp"

namespace {

using dynts::ChunkCache;

constexpr size_t kAlign = 256;
constexpr int kMostTokens = 1 << 20, kMostDraft = dynts::kTreeMost;
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
  bool token;        // coded_token_kernel
  bool groups;       // forms_attend_groups_kernel
  bool half;         // forms_attend_half_kernel
  bool unpack;       // codes are made bf16 in scratch beforehand
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
//
// Caches of codes by the same rule, which is wrong for 64 rows of very many units on long caches alone (512 units, below).  us, few / many (e4m3; whole numbers up to a
// fourth more):
//   head_dim 128, 8 units: 4500 slots R = 512 27.2 / 28.3, R = 1024 38.1 / 36.8; 16000 slots R = 128 25.9 / 28.8, R = 256 37.3 / 34.3; 32 units: 1500 slots R = 256 17.4 /
//     24.1, R = 512 32.8 / 30.3, 4500 R = 256 36.2 / 35.2, 16000 R = 64 39.8 / 50.6, R = 128 66.4 / 56.0; 128 units: 500 slots R = 64 10.9 / 16.2, R = 128 19.9 / 17.1, 4500
//     R = 64 42.5 / 54.2, R = 128 77.6 / 60.4; 512 units: 500 slots R = 64 37.1 / 26.8, 1500 70.5 / 69.4, 4500 163 / 185
//   head_dim 64, 8 units: 16000 slots R = 128 19.8 / 21.7, R = 256 27.3 / 24.5; 32 units: 1500 slots R = 512 18.8 / 22.3, 4500 43.2 / 38.3; 128 units: 1500 slots R = 96
//     17.6 / 23.6, 4500 41.4 / 36.8
// Groups of waves (drafts, chunks on codes): one workgroup a compute unit, and no two shares of many units, which are bound by HBM, before the slots pay for
// the joint.  us by the number of shares: W = 128, 32 units of 2500 slots 1 / 2: 39.1 / 35.1, 128 units 44.2 / 47.0, 64 units of 4500 71.4 / 55.2; W = 16, 8 units of
// 16400 8 / 16 / 32: 40.3 / 33.9 / 47.1; W = 64, 64 units of 9000 2 / 4 / 8: 81.7 / 70.1 / 83.6.
// Where they have no shares and half as many rows a workgroup, H of them, still have a compute unit each: half.  us, 128 rows / 64 (bf16 | e4m3 | whole numbers; on codes
// measured with one barrier for all groups: 64 rows have become up to 5 us faster since, 128 up to 2):
//   head_dim 128, 500 slots: 64 units R = 256 17.2 / 14.6 | 18.5 / 15.8 | 19.6 / 16.7, 128 of R = 128 16.1 / 14.6 | 18.0 / 15.2 | 18.9 / 16.0, 256 of R = 64 18.7 / 17.1 | 18.0 / 16.2 |
//     19.2 / 16.9; 2464 slots: 128 of R = 112 45.7 / 41.6 | 47.1 / 42.4 | 51.4 / 45.8, 256 of R = 64 63.5 / 61.1 | 56.1 / 50.1 | 61.4 / 52.3, H = 512 53.3 / 56.9 | 55.9 / 56.8 | 61.9 / 61.0
//   head_dim 64, 2464 slots: 128 of R = 128 27.8 / 25.1 | 35.4 / 29.1 | 37.1 / 30.9
//   instead of shares: 64 units of 4500 slots R = 128 45.8 / 47.2 | 38.5 / 44.1 | 40.7 / 48.1, 32 of 16000 R = 256 88.0 / 112 | 87.3 / 123 | 97.2 / 135
ChunkPlan chunk_plan(const dynts_config &c, int n_tokens, int slots, bool far_cap = false, int code = 0, bool tree = false, bool shaped = false) {
  ChunkPlan pl;
  const long long R = (long long)n_tokens * (c.n_q_heads / c.n_kv_heads), units = (long long)c.batch * c.n_kv_heads;
  const long long F = units * ((R + dynts::kFewRows - 1) / dynts::kFewRows), W = units * ((R + dynts::kChRows - 1) / dynts::kChRows);
  const int room = c.head_dim == 128 ? 256 : 512;  // workgroups of few rows that the chip holds
  pl.few = far_cap || R <= dynts::kFewRows || (F <= room && (R <= 2 * dynts::kFewRows || F * slots <= 1 << 20));
  // Codes become bf16 in every row block anew; shaped, or of more blocks than this, they are unpacked before.  us by the blocks of a unit, unpacked / not: e4m3, head_dim 128,
  // 128 units of 2500 slots 8 / 12 / 16 / 24: 217 291 374 554 / 186 273 361 556, 8 units of 16000 8 / 24 / 64: 98 238 523 / 80 243 578; whole numbers 128 units 8 / 12 / 16: 217
  // 293 376 / 201 295 396; head_dim 64, 32 units of 2500 8 / 12: 43.5 55.9 / 36.3 62.2, 128 of 1000 8 / 12 / 24: 54.9 77.4 140 / 49.5 75.4 143, whole numbers 55 79 141 / 55
  // 79 158.  Shaped, of two evils: the kernel of many rows with a shaping has no form for codes, and the layer is unpacked whole, also slots that a window hides from all
  // rows.  512 tokens, window 1024, 4 heads a group of 128, bf16 cache / codes: 8 units of 1536 slots 35.2 / 40.3, of 16384 34.3 / 48.6; 32 units 45.2 / 55.1, 44.6 / 118.5.
  const int most_blocks = c.head_dim == 128 ? (code == DYNTS_CODE_E4M3 ? 20 : 10) : code == DYNTS_CODE_E4M3 ? 10 : 8;
  pl.unpack = code && !pl.few && (shaped || W > units * most_blocks);
  pl.groups = !pl.few && W <= 256 && (tree || (code && !pl.unpack));
  pl.token = code && !tree && R <= dynts::kTokRows;
  pl.rows = pl.token ? dynts::kTokRows : pl.few ? dynts::kFewRows : dynts::kChRows;
  long long shares = slots / (32 * dynts::kShareTiles);
  if (pl.token) {
    shares = shares < 32 ? shares : 32;
    shares = shares < 256 / units ? shares : 256 / units;
  } else if (pl.few) {
    shares = shares < 16 ? shares : 16;
    shares = shares < 256 / F ? shares : 256 / F;
    if (shares < 3 && units > 64) shares = 1;
  } else {
    shares = shares < 32 ? shares : 32;
    shares = shares < 512 / W ? shares : 512 / W;
    if (pl.groups) {
      shares = shares < 256 / W ? shares : 256 / W;
      if (units > 64 && slots < 3500) shares = 1;
    }
  }
  if (slots < 1536) shares = 1;
  pl.half = pl.groups && shares < 2 && units * ((R + dynts::kHalfRows - 1) / dynts::kHalfRows) <= 256;
  if (pl.half) pl.rows = dynts::kHalfRows;
  pl.blocks = (int)((R + pl.rows - 1) / pl.rows);
  pl.Rpad = pl.blocks * pl.rows;
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

bool shaped(const dynts_shaping *s) { return s && (s->softcap > 0.f || s->window > 0 || s->slope || s->first || s->last); }
// a cap that takes the longer form of soft_caps
bool far_cap(const dynts_shaping *s) { return s && s->softcap * kLog2E > dynts::kCapNear; }

dynts_config config_of(const ChunkCache &c) {
  dynts_config cfg{};
  cfg.batch = c.Nb; cfg.n_q_heads = c.Hq; cfg.n_kv_heads = c.Hkv; cfg.head_dim = c.D; cfg.capacity = c.cap;
  return cfg;
}
// tree: for a draft
ChunkPlan chunk_plan(const ChunkCache &c, int n_tokens, const dynts_shaping *shaping, bool tree) {
  // (slots of a window: no more than its positions, those of the chunk's other tokens beside them)
  const long long seen = shaping && shaping->window > 0 ? (long long)shaping->window + n_tokens : c.cap;
  return chunk_plan(config_of(c), n_tokens, (int)(seen < c.cap ? seen : c.cap), far_cap(shaping), c.code, tree, shaped(shaping));
}

// Room behind a chunk's scratch where the layer's codes lie as bf16, for the kernel of many rows.
size_t unpacked_bytes(const dynts_config &c) { return align_up((size_t)c.batch * c.n_kv_heads * c.capacity * c.head_dim * 2); }
size_t scratch_bytes_of(const dynts_config &c, int n_tokens, bool codes) {
  // (which kernel a shorter chunk takes goes by its sizes: the room is there for all that may be of many rows)
  const bool many = (long long)n_tokens * (c.n_q_heads / c.n_kv_heads) > dynts::kFewRows;
  return chunk_plan(c, n_tokens, c.capacity).bytes + (codes && many ? 2 * unpacked_bytes(c) : 0);
}
size_t scratch_bytes_of(const ChunkCache &c, int n_tokens) { return scratch_bytes_of(config_of(c), n_tokens, c.code != 0); }

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
  const dynts::ChunkAppendParams p{c, k_new, v_new, s_new, n_new, taken, n_tokens, question,
                                  ((1ull << 36) + c.Hkv - 1) / c.Hkv};
  const long long pieces = (long long)n_tokens * c.Hkv * (c.D / 8);
  const dim3 block(dynts::kAppendThreads);
  if (c.code && pieces <= dynts::kAppendSmall) {
    dynts::launch_coded_append(p, true, st);
    return launch_status();
  }
  if (copy && pieces <= dynts::kAppendSmall) {
    if (c.D == 128) hipLaunchKernelGGL((dynts::chunk_reserve_kernel<128, true>), dim3(c.Nb), block, 0, st, p);
    else hipLaunchKernelGGL((dynts::chunk_reserve_kernel<64, true>), dim3(c.Nb), block, 0, st, p);
    return launch_status();
  }
  const dim3 grid((unsigned)((pieces + dynts::kAppendThreads - 1) / dynts::kAppendThreads), c.Nb);
  if (c.code) copy = false;
  if (c.D == 128) {
    hipLaunchKernelGGL((dynts::chunk_reserve_kernel<128, false>), dim3(c.Nb), block, 0, st, p);
    if (copy) hipLaunchKernelGGL((dynts::chunk_copy_kernel<128>), grid, block, 0, st, p);
  } else {
    hipLaunchKernelGGL((dynts::chunk_reserve_kernel<64, false>), dim3(c.Nb), block, 0, st, p);
    if (copy) hipLaunchKernelGGL((dynts::chunk_copy_kernel<64>), grid, block, 0, st, p);
  }
  if (c.code) dynts::launch_coded_append(p, false, st);
  return launch_status();
}

// workgroups of `blocks` a unit as chunk_map has them, units rounded up to the 8 XCDs; 0 if a grid cannot hold their threads (2^32)
unsigned chunk_grid(const ChunkCache &c, long long blocks, int threads) {
  const long long units = (long long)c.Nb * c.Hkv, share = units > 4 ? 1 : units > 2 ? 2 : 8 / units;  // XCDs of a unit
  const long long wgs = (blocks + share - 1) / share * ((units + 7) / 8 * 8);
  return wgs >= (1LL << 32) / threads ? 0u : (unsigned)wgs;
}
unsigned attend_grid(const ChunkCache &c, const ChunkPlan &pl) {
  return chunk_grid(c, (long long)pl.blocks * pl.n_split, pl.token ? dynts::kTokWaves * 64 : pl.few ? dynts::kFewThreads : pl.half ? dynts::kHalfGroups<1> * dynts::kHalfWaves * 64 : pl.groups ? dynts::kGroups * dynts::kChThreads : dynts::kChThreads);
}
// Which kernel of chunk_scores.hpp.  C: chunks of 32 rows of a unit, W: workgroups of 64 slots, one a compute unit.  Few slots: 7 + C / 4 us a round of 256 of
// them; many: 4 + 0.8 C us while its W / 4 workgroups have a compute unit each.  us, few / many:
//   head_dim 128: C = 66, W = 168 21.9 / 60.4, W = 672 60.9 / 61.5; C = 219, W = 152 57.0 / 170, W = 512 97.6 / 184; C = 389, W = 432 100 / 304; C = 112,
//     W = 752 93.1 / 92.2, W = 1504 183 / 122; C = 14, W = 640 26.3 / 16.8; C = 2, W = 568 14.5 / 5.9
//   head_dim 64: C = 164, W = 78 23.1 / 128; C = 10, W = 64 6.0 / 10.9; C = 38, W = 288 15.7 / 29.8, W = 1152 38.2 / 40.2
bool scores_token(const ChunkCache &c, int n_tokens);
bool scores_few(const ChunkCache &c, int n_tokens, const dynts_shaping *shaping) {
  if (scores_token(c, n_tokens)) return false;
  if (far_cap(shaping)) return true;  // (the other one does not know it)
  const long long W = (long long)c.Nb * c.Hkv * ((c.cap + dynts::kCfKeys - 1) / dynts::kCfKeys);
  const long long C = ((long long)n_tokens * c.G + dynts::kSbChunk - 1) / dynts::kSbChunk;
  return W <= 256 ? C >= 8 : W <= 512 && C >= 32;
}
// coded_token_scores_kernel
bool scores_token(const ChunkCache &c, int n_tokens) { return c.code && (long long)n_tokens * c.G <= dynts::kTokRows; }
static_assert(dynts::kTsKeys == dynts::kCsKeys, "one grid for both");
unsigned scores_grid(const ChunkCache &c, bool few) {
  return few ? chunk_grid(c, (c.cap + dynts::kCfKeys - 1) / dynts::kCfKeys, dynts::kCfWaves * 64)
             : chunk_grid(c, (c.cap + dynts::kCsKeys - 1) / dynts::kCsKeys, dynts::kSbWaves * 64);
}

template <int D, bool SHAPED>
void launch_attend_d(const dynts::ChunkAttendParams &p, const ChunkPlan &pl, unsigned grid, hipStream_t st) {
  if (pl.token) dynts::launch_coded_token(p, SHAPED, grid, st);
  else if (pl.few && (p.seen || p.c.code)) dynts::launch_few_form(p, p.seen ? dynts::kTree : SHAPED ? dynts::kShaped : dynts::kPlain, grid, st);
  else if (pl.half) dynts::launch_attend_half(p, p.seen ? dynts::kTree : dynts::kPlain, grid, st);
  else if (pl.groups) dynts::launch_attend_groups(p, p.seen ? dynts::kTree : dynts::kPlain, grid, st);
  else if (!pl.few && p.c.code) dynts::launch_coded_attend(p, p.seen ? dynts::kTree : dynts::kPlain, grid, st);
  else if (p.seen) dynts::launch_tree_attend(p, grid, st);
  else if (pl.few) hipLaunchKernelGGL((dynts::chunk_attend_few_kernel<D, SHAPED>), dim3(grid), dim3(dynts::kFewThreads), 0, st, p);
  else if (SHAPED && p.shape.slope) hipLaunchKernelGGL((dynts::chunk_attend_kernel<D, SHAPED, SHAPED, false>), dim3(grid), dim3(dynts::kChThreads), 0, st, p);
  else if (!SHAPED && p.k_new) hipLaunchKernelGGL((dynts::chunk_attend_kernel<D, false, false, !SHAPED>), dim3(grid), dim3(dynts::kChThreads), 0, st, p);
  else hipLaunchKernelGGL((dynts::chunk_attend_kernel<D, SHAPED, false, false>), dim3(grid), dim3(dynts::kChThreads), 0, st, p);
  if (p.n_split > 1 && (p.seen || p.c.code)) {
    dynts::launch_merge_form(p, pl.rows, st);
  } else if (p.n_split > 1) {
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

// seen: of a draft's tokens, or null
int launch_attend(ChunkCache c, const uint16_t *q, int n_tokens, const int32_t *n_new, const dynts_shaping *shaping, const uint32_t *seen, uint16_t *out,
                  float *lse, void *scratch, const Fresh &fresh, hipStream_t st) {
  const ChunkPlan pl = chunk_plan(c, n_tokens, shaping, seen != nullptr);
  char *const base = static_cast<char *>(scratch);
  if (pl.unpack) {  // in a dense cache
    uint16_t *const K = reinterpret_cast<uint16_t *>(base + pl.bytes), *const V = reinterpret_cast<uint16_t *>(base + pl.bytes + unpacked_bytes(config_of(c)));
    dynts::launch_read_rows(c, nullptr, c.cap, K, V, false, st);
    c.K = K;
    c.V = V;
    c.code = 0;
    c.block_table = nullptr;
  }
  const dynts::ChunkAttendParams p{c, q, n_new, out, lse, chunk_shape(shaping, c.scale), n_tokens, c.scale * kLog2E, group_magic(c.G), pl.n_split, pl.Rpad,
                                   reinterpret_cast<float *>(base + pl.off_o), reinterpret_cast<float *>(base + pl.off_ml),
                                   reinterpret_cast<int32_t *>(base + pl.off_n), fresh.k_new, fresh.v_new, fresh.s_new, fresh.question,
                                   seen, (n_tokens + 31) / 32};
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
  if (scores_token(c, n_tokens)) dynts::launch_coded_token_scores(p, shaped(p.shape), grid, st);
  else if (c.code) dynts::launch_coded_scores(p, few, shaped(p.shape), p.shape.slope != nullptr, grid, st);
  else if (c.D == 128) launch_scores_d<128>(p, few, grid, st);
  else launch_scores_d<64>(p, few, grid, st);
  return launch_status();
}

int check_tokens(int32_t n_tokens) { return n_tokens <= 0 || n_tokens > kMostTokens ? DYNTS_EINVAL : DYNTS_OK; }

int check_draft(const ChunkCache &c, const uint16_t *q, int n_tokens, const uint32_t *seen, const uint16_t *out) {
  if (n_tokens <= 0 || n_tokens > kMostDraft) return DYNTS_EINVAL;
  if (!q || !seen || !out) return DYNTS_ENULL;
  if (misaligned(q, 16) || misaligned(out, 16) || misaligned(seen, 4)) return DYNTS_EINVAL;
  const size_t q_bytes = (size_t)c.Nb * n_tokens * c.Hq * c.D * 2;
  if (overlap(out, q_bytes, q, q_bytes)) return DYNTS_EINVAL;
  return attend_grid(c, chunk_plan(c, n_tokens, nullptr, true)) ? DYNTS_OK : DYNTS_EINVAL;
}

}  // namespace

extern "C" {

size_t dynts_chunk_scratch_bytes(const dynts_config *cfg, int32_t n_tokens) {
  if (dynts::chunk_check_config(cfg) != DYNTS_OK || check_tokens(n_tokens) != DYNTS_OK) return 0;
  return chunk_plan(*cfg, n_tokens, cfg->capacity).bytes;
}

size_t dynts_codes_scratch_bytes(const dynts_config *cfg, int32_t n_tokens) {
  if (dynts::chunk_check_config(cfg) != DYNTS_OK || check_tokens(n_tokens) != DYNTS_OK) return 0;
  return scratch_bytes_of(*cfg, n_tokens, true);
}

int dynts_chunk_append(dynts_ctx *ctx, int32_t layer, const uint16_t *k_new, const uint16_t *v_new, const float *s_new, int32_t n_tokens,
                       const int32_t *n_new, int32_t question, void *scratch, size_t scratch_bytes, void *stream) {
  ChunkCache c;
  int rc = dynts::chunk_cache(ctx, layer, &c);
  if (rc == DYNTS_OK) rc = check_tokens(n_tokens);
  if (rc == DYNTS_OK) rc = check_append(c, k_new, v_new, s_new, question);
  if (rc == DYNTS_OK) rc = check_scratch(scratch, scratch_bytes, scratch_bytes_of(c, n_tokens));
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
  rc = check_scratch(scratch, scratch_bytes, scratch_bytes_of(c, n_tokens));
  if (rc != DYNTS_OK) return rc;
  const size_t q_bytes = (size_t)c.Nb * n_tokens * c.Hq * c.D * 2;
  if (overlap(out, q_bytes, q, q_bytes)) return DYNTS_EINVAL;
  return launch_attend(c, q, n_tokens, n_new, shaping, nullptr, out, lse, scratch, Fresh{}, static_cast<hipStream_t>(stream));
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
  const ChunkPlan pl = chunk_plan(c, n_tokens, shaping, false);
  rc = check_scratch(scratch, scratch_bytes, c.code ? scratch_bytes_of(c, n_tokens) : pl.bytes);
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
  const bool on_the_way = !pl.few && !shaped(shaping) && !c.code;
  rc = launch_append(c, k_new, v_new, s_new, n_tokens, n_new, question, taken, !on_the_way, st);
  if (rc == DYNTS_OK)
    rc = launch_attend(c, q, n_tokens, taken, shaping, nullptr, out, lse, scratch, on_the_way ? Fresh{k_new, v_new, s_new, question} : Fresh{}, st);
  if (rc == DYNTS_OK && scores) rc = launch_scores(c, q, n_tokens, taken, shaping, lse, nullptr, 1, st);
  return rc;
}

int dynts_tree_attend(dynts_ctx *ctx, int32_t layer, const uint16_t *q, int32_t n_tokens, const int32_t *n_new, const uint32_t *seen, uint16_t *out,
                      float *lse, void *scratch, size_t scratch_bytes, void *stream) {
  ChunkCache c;
  int rc = dynts::chunk_cache(ctx, layer, &c);
  if (rc == DYNTS_OK) rc = check_draft(c, q, n_tokens, seen, out);
  if (rc == DYNTS_OK) rc = check_scratch(scratch, scratch_bytes, scratch_bytes_of(c, n_tokens));
  if (rc != DYNTS_OK) return rc;
  return launch_attend(c, q, n_tokens, n_new, nullptr, seen, out, lse, scratch, Fresh{}, static_cast<hipStream_t>(stream));
}

int dynts_tree_step(dynts_ctx *ctx, int32_t layer, const uint16_t *q, const uint16_t *k_new, const uint16_t *v_new, const float *s_new, int32_t n_tokens,
                    const int32_t *n_new, const uint32_t *seen, int32_t *n_taken, uint16_t *out, float *lse, void *scratch, size_t scratch_bytes,
                    void *stream) {
  ChunkCache c;
  int rc = dynts::chunk_cache(ctx, layer, &c);
  if (rc == DYNTS_OK) rc = check_draft(c, q, n_tokens, seen, out);
  if (rc == DYNTS_OK) rc = check_append(c, k_new, v_new, s_new, 0);
  if (rc == DYNTS_OK && !n_taken) rc = DYNTS_ENULL;
  if (rc == DYNTS_OK) rc = check_scratch(scratch, scratch_bytes, scratch_bytes_of(c, n_tokens));
  if (rc != DYNTS_OK) return rc;
  const size_t row = (size_t)c.Nb * n_tokens * c.D * 2, q_bytes = row * c.Hq, k_bytes = row * c.Hkv;
  if (overlap(out, q_bytes, k_new, k_bytes) || overlap(out, q_bytes, v_new, k_bytes)) return DYNTS_EINVAL;
  if (c.score_mode != DYNTS_SCORE_EXTERNAL) s_new = nullptr;
  hipStream_t st = static_cast<hipStream_t>(stream);
  rc = launch_append(c, k_new, v_new, s_new, n_tokens, n_new, 0, n_taken, true, st);
  if (rc == DYNTS_OK) rc = launch_attend(c, q, n_tokens, n_taken, nullptr, seen, out, lse, scratch, Fresh{}, st);
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
