// Caches of codes and drafts that branch: launches of their kernels, and the entry points that are theirs alone.  Nothing here allocates device memory or
// synchronises the host.
#include "forms.hpp"

#include "codes.hpp"
#include "tree.hpp"

namespace dynts {

// (here and below: a cache that is not of codes comes with mask kTree)
template <int D, int CODE>
static void few_form(const ChunkAttendParams &p, int mask, unsigned grid, hipStream_t st) {
  auto *kernel = forms_attend_few_kernel<D, kTree, CODE>;
  if constexpr (CODE != 0) {
    if (mask == kShaped) kernel = forms_attend_few_kernel<D, kShaped, CODE>;
    else if (mask == kPlain) kernel = forms_attend_few_kernel<D, kPlain, CODE>;
  }
  hipLaunchKernelGGL(kernel, dim3(grid), dim3(kFewThreads), 0, st, p);
}
void launch_few_form(const ChunkAttendParams &p, int mask, unsigned grid, hipStream_t st) {
  if (p.c.D == 128) {
    if (p.c.code == DYNTS_CODE_E4M3) few_form<128, DYNTS_CODE_E4M3>(p, mask, grid, st);
    else if (p.c.code == DYNTS_CODE_INT8) few_form<128, DYNTS_CODE_INT8>(p, mask, grid, st);
    else few_form<128, 0>(p, mask, grid, st);
  } else {
    if (p.c.code == DYNTS_CODE_E4M3) few_form<64, DYNTS_CODE_E4M3>(p, mask, grid, st);
    else if (p.c.code == DYNTS_CODE_INT8) few_form<64, DYNTS_CODE_INT8>(p, mask, grid, st);
    else few_form<64, 0>(p, mask, grid, st);
  }
}

template <int D, int CODE>
static void coded_token(const ChunkAttendParams &p, bool shaped, unsigned grid, hipStream_t st) {
  if (shaped) hipLaunchKernelGGL((coded_token_kernel<D, kShaped, CODE, kTokWaves>), dim3(grid), dim3(kTokWaves * 64), 0, st, p);
  else hipLaunchKernelGGL((coded_token_kernel<D, kPlain, CODE, kTokWaves>), dim3(grid), dim3(kTokWaves * 64), 0, st, p);
}
void launch_coded_token(const ChunkAttendParams &p, bool shaped, unsigned grid, hipStream_t st) {
  if (p.c.D == 128) {
    if (p.c.code == DYNTS_CODE_E4M3) coded_token<128, DYNTS_CODE_E4M3>(p, shaped, grid, st);
    else coded_token<128, DYNTS_CODE_INT8>(p, shaped, grid, st);
  } else {
    if (p.c.code == DYNTS_CODE_E4M3) coded_token<64, DYNTS_CODE_E4M3>(p, shaped, grid, st);
    else coded_token<64, DYNTS_CODE_INT8>(p, shaped, grid, st);
  }
}
template <int D, int CODE>
static void coded_token_scores(const ChunkScoreParams &p, bool shaped, unsigned grid, hipStream_t st) {
  if (shaped) hipLaunchKernelGGL((coded_token_scores_kernel<D, true, CODE>), dim3(grid), dim3(kTsWaves * 64), 0, st, p);
  else hipLaunchKernelGGL((coded_token_scores_kernel<D, false, CODE>), dim3(grid), dim3(kTsWaves * 64), 0, st, p);
}
void launch_coded_token_scores(const ChunkScoreParams &p, bool shaped, unsigned grid, hipStream_t st) {
  if (p.c.D == 128) {
    if (p.c.code == DYNTS_CODE_E4M3) coded_token_scores<128, DYNTS_CODE_E4M3>(p, shaped, grid, st);
    else coded_token_scores<128, DYNTS_CODE_INT8>(p, shaped, grid, st);
  } else {
    if (p.c.code == DYNTS_CODE_E4M3) coded_token_scores<64, DYNTS_CODE_E4M3>(p, shaped, grid, st);
    else coded_token_scores<64, DYNTS_CODE_INT8>(p, shaped, grid, st);
  }
}

void launch_tree_attend(const ChunkAttendParams &p, unsigned grid, hipStream_t st) {
  if (p.c.D == 128) hipLaunchKernelGGL((tree_attend_kernel<128>), dim3(grid), dim3(kChThreads), 0, st, p);
  else hipLaunchKernelGGL((tree_attend_kernel<64>), dim3(grid), dim3(kChThreads), 0, st, p);
}
template <int D, int CODE>
static void attend_groups(const ChunkAttendParams &p, int mask, unsigned grid, hipStream_t st) {
  auto *kernel = forms_attend_groups_kernel<D, kTree, CODE>;
  if constexpr (CODE != 0) {
    if (mask == kPlain) kernel = forms_attend_groups_kernel<D, kPlain, CODE>;
  }
  hipLaunchKernelGGL(kernel, dim3(grid), dim3(kGroups * kChThreads), 0, st, p);
}
template <int D, int CODE>
static void attend_half(const ChunkAttendParams &p, int mask, unsigned grid, hipStream_t st) {
  auto *kernel = forms_attend_half_kernel<D, kTree, CODE>;
  if constexpr (CODE != 0) {
    if (mask == kPlain) kernel = forms_attend_half_kernel<D, kPlain, CODE>;
  }
  hipLaunchKernelGGL(kernel, dim3(grid), dim3(kHalfGroups<CODE> * kHalfWaves * 64), 0, st, p);
}
void launch_attend_half(const ChunkAttendParams &p, int mask, unsigned grid, hipStream_t st) {
  if (p.c.D == 128) {
    if (p.c.code == DYNTS_CODE_E4M3) attend_half<128, DYNTS_CODE_E4M3>(p, mask, grid, st);
    else if (p.c.code == DYNTS_CODE_INT8) attend_half<128, DYNTS_CODE_INT8>(p, mask, grid, st);
    else attend_half<128, 0>(p, mask, grid, st);
  } else {
    if (p.c.code == DYNTS_CODE_E4M3) attend_half<64, DYNTS_CODE_E4M3>(p, mask, grid, st);
    else if (p.c.code == DYNTS_CODE_INT8) attend_half<64, DYNTS_CODE_INT8>(p, mask, grid, st);
    else attend_half<64, 0>(p, mask, grid, st);
  }
}
void launch_attend_groups(const ChunkAttendParams &p, int mask, unsigned grid, hipStream_t st) {
  if (p.c.D == 128) {
    if (p.c.code == DYNTS_CODE_E4M3) attend_groups<128, DYNTS_CODE_E4M3>(p, mask, grid, st);
    else if (p.c.code == DYNTS_CODE_INT8) attend_groups<128, DYNTS_CODE_INT8>(p, mask, grid, st);
    else attend_groups<128, 0>(p, mask, grid, st);
  } else {
    if (p.c.code == DYNTS_CODE_E4M3) attend_groups<64, DYNTS_CODE_E4M3>(p, mask, grid, st);
    else if (p.c.code == DYNTS_CODE_INT8) attend_groups<64, DYNTS_CODE_INT8>(p, mask, grid, st);
    else attend_groups<64, 0>(p, mask, grid, st);
  }
}
template <int D>
static void merge_form(const ChunkAttendParams &p, int block_rows, hipStream_t st) {
  const int rows = p.n_split > 4 ? kMergeThreads / 64 : kMergeThreads / (D / 8);
  const dim3 grid((p.T * p.c.G + rows - 1) / rows, p.c.Nb * p.c.Hkv), block(kMergeThreads);
  if (p.n_split > 4) hipLaunchKernelGGL(forms_merge_kernel<D>, grid, block, 0, st, p, block_rows);
  else hipLaunchKernelGGL(forms_merge_few_kernel<D>, grid, block, 0, st, p, block_rows);
}
void launch_merge_form(const ChunkAttendParams &p, int block_rows, hipStream_t st) {
  if (p.c.D == 128) merge_form<128>(p, block_rows, st);
  else merge_form<64>(p, block_rows, st);
}
template <int D, int CODE>
static void coded_attend(const ChunkAttendParams &p, int mask, unsigned grid, hipStream_t st) {
  if (mask == kTree) hipLaunchKernelGGL((coded_attend_kernel<D, kTree, CODE>), dim3(grid), dim3(kChThreads), 0, st, p);
  else hipLaunchKernelGGL((coded_attend_kernel<D, kPlain, CODE>), dim3(grid), dim3(kChThreads), 0, st, p);
}
void launch_coded_attend(const ChunkAttendParams &p, int mask, unsigned grid, hipStream_t st) {
  if (p.c.D == 128) {
    if (p.c.code == DYNTS_CODE_E4M3) coded_attend<128, DYNTS_CODE_E4M3>(p, mask, grid, st);
    else coded_attend<128, DYNTS_CODE_INT8>(p, mask, grid, st);
  } else {
    if (p.c.code == DYNTS_CODE_E4M3) coded_attend<64, DYNTS_CODE_E4M3>(p, mask, grid, st);
    else coded_attend<64, DYNTS_CODE_INT8>(p, mask, grid, st);
  }
}

template <int D, int CODE, bool SHAPED, bool BIASED>
static void coded_scores_form(const ChunkScoreParams &p, bool few, unsigned grid, hipStream_t st) {
  if (few) hipLaunchKernelGGL((coded_scores_few_kernel<D, SHAPED, BIASED, CODE>), dim3(grid), dim3(kCfWaves * 64), 0, st, p);
  else hipLaunchKernelGGL((coded_scores_kernel<D, SHAPED, BIASED, CODE>), dim3(grid), dim3(kSbWaves * 64), 0, st, p);
}
template <int D, int CODE>
static void coded_scores(const ChunkScoreParams &p, bool few, bool shaped, bool biased, unsigned grid, hipStream_t st) {
  if (biased) coded_scores_form<D, CODE, true, true>(p, few, grid, st);
  else if (shaped) coded_scores_form<D, CODE, true, false>(p, few, grid, st);
  else coded_scores_form<D, CODE, false, false>(p, few, grid, st);
}
void launch_coded_scores(const ChunkScoreParams &p, bool few, bool shaped, bool biased, unsigned grid, hipStream_t st) {
  if (p.c.D == 128) {
    if (p.c.code == DYNTS_CODE_E4M3) coded_scores<128, DYNTS_CODE_E4M3>(p, few, shaped, biased, grid, st);
    else coded_scores<128, DYNTS_CODE_INT8>(p, few, shaped, biased, grid, st);
  } else {
    if (p.c.code == DYNTS_CODE_E4M3) coded_scores<64, DYNTS_CODE_E4M3>(p, few, shaped, biased, grid, st);
    else coded_scores<64, DYNTS_CODE_INT8>(p, few, shaped, biased, grid, st);
  }
}

template <int D, int CODE>
static void coded_append(const ChunkAppendParams &p, bool small, hipStream_t st) {
  const unsigned blocks = (unsigned)(p.T + kCodedTokens<D> - 1) / kCodedTokens<D> * p.c.Hkv;
  if (small) hipLaunchKernelGGL((coded_reserve_kernel<D, CODE>), dim3(p.c.Nb), dim3(kAppendThreads), 0, st, p);
  else hipLaunchKernelGGL((coded_copy_kernel<D, CODE>), dim3(blocks, p.c.Nb), dim3(kAppendThreads), 0, st, p);
}
void launch_coded_append(const ChunkAppendParams &p, bool small, hipStream_t st) {
  if (p.c.D == 128) {
    if (p.c.code == DYNTS_CODE_E4M3) coded_append<128, DYNTS_CODE_E4M3>(p, small, st);
    else coded_append<128, DYNTS_CODE_INT8>(p, small, st);
  } else {
    if (p.c.code == DYNTS_CODE_E4M3) coded_append<64, DYNTS_CODE_E4M3>(p, small, st);
    else coded_append<64, DYNTS_CODE_INT8>(p, small, st);
  }
}

template <int D, bool PAST>
static void read_rows(const ReadParams &p, hipStream_t st) {
  constexpr int kPer = kReadThreads * kReadAtOnce;
  const dim3 grid((unsigned)(((long long)p.n_rows * (D / 8) + kPer - 1) / kPer), p.c.Hkv, p.c.Nb), block(kReadThreads);
  if (p.c.code == DYNTS_CODE_E4M3) hipLaunchKernelGGL((read_rows_kernel<D, DYNTS_CODE_E4M3, PAST>), grid, block, 0, st, p);
  else if (p.c.code == DYNTS_CODE_INT8) hipLaunchKernelGGL((read_rows_kernel<D, DYNTS_CODE_INT8, PAST>), grid, block, 0, st, p);
  else if (PAST) hipLaunchKernelGGL((read_rows_kernel<D, 0, true>), grid, block, 0, st, p);
}
void launch_read_rows(const ChunkCache &c, const int32_t *first, int n_rows, uint16_t *K, uint16_t *V, bool past, hipStream_t st) {
  const ReadParams p{c, first, K, V, n_rows};
  if (c.D == 128) past ? read_rows<128, true>(p, st) : read_rows<128, false>(p, st);
  else past ? read_rows<64, true>(p, st) : read_rows<64, false>(p, st);
}

}  // namespace dynts

namespace {

bool misaligned(const void *p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to != 0; }
bool overlap(const void *a, size_t a_bytes, const void *b, size_t b_bytes) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + b_bytes && y < x + a_bytes;
}
int launch_status() { return hipGetLastError() == hipSuccess ? DYNTS_OK : DYNTS_EHIP; }

}  // namespace

extern "C" {

int dynts_read_rows(dynts_ctx *ctx, int32_t layer, const int32_t *first, int32_t n_rows, uint16_t *K_out, uint16_t *V_out, void *stream) {
  dynts::ChunkCache c;
  const int rc = dynts::chunk_cache(ctx, layer, &c);
  if (rc != DYNTS_OK) return rc;
  if (!K_out || !V_out) return DYNTS_ENULL;
  if (n_rows <= 0 || n_rows > c.cap) return DYNTS_EINVAL;
  if (misaligned(K_out, 16) || misaligned(V_out, 16) || misaligned(first, 4)) return DYNTS_EINVAL;
  const size_t bytes = (size_t)c.Nb * c.Hkv * n_rows * c.D * 2;
  if (overlap(K_out, bytes, V_out, bytes)) return DYNTS_EINVAL;
  dynts::launch_read_rows(c, first, n_rows, K_out, V_out, true, static_cast<hipStream_t>(stream));
  return launch_status();
}

int dynts_tree_build(const int32_t *parents, const int32_t *n_new, int32_t batch, int32_t n_tokens, uint32_t *seen, int32_t *depth, void *stream) {
  if (!parents || !seen) return DYNTS_ENULL;
  if (batch <= 0 || batch > 65535 || n_tokens <= 0 || n_tokens > dynts::kTreeMost) return DYNTS_EINVAL;
  if (misaligned(parents, 4) || misaligned(n_new, 4) || misaligned(seen, 4) || misaligned(depth, 4)) return DYNTS_EINVAL;
  const int words = (n_tokens + 31) / 32;
  const size_t tokens = (size_t)batch * n_tokens;
  if (overlap(seen, tokens * words * 4, parents, tokens * 4) ||
      (depth && (overlap(depth, tokens * 4, parents, tokens * 4) || overlap(depth, tokens * 4, seen, tokens * words * 4))))
    return DYNTS_EINVAL;
  const dynts::TreeBuildParams p{parents, n_new, seen, depth, n_tokens, words};
  hipLaunchKernelGGL(dynts::tree_build_kernel, dim3((n_tokens + dynts::kTreeThreads - 1) / dynts::kTreeThreads, batch), dim3(dynts::kTreeThreads),
                     n_tokens * sizeof(int32_t), static_cast<hipStream_t>(stream), p);
  return launch_status();
}

int dynts_tree_keep(dynts_ctx *ctx, int32_t layer, int32_t n_tokens, const int32_t *n_taken, const uint32_t *seen, const int32_t *leaf,
                    const uint16_t *q, const float *lse, uint16_t *q_kept, float *lse_kept, int32_t *n_kept, void *stream) {
  dynts::ChunkCache c;
  const int rc = dynts::chunk_cache(ctx, layer, &c);
  if (rc != DYNTS_OK) return rc;
  if (!seen || !leaf || !n_kept || (q_kept && !q) || (lse_kept && !lse)) return DYNTS_ENULL;
  if (n_tokens <= 0 || n_tokens > dynts::kTreeMost) return DYNTS_EINVAL;
  if (misaligned(q, 16) || misaligned(q_kept, 16) || misaligned(lse, 4) || misaligned(lse_kept, 4) || misaligned(seen, 4)) return DYNTS_EINVAL;
  const size_t each = (size_t)c.Nb * 4;  // (other workgroups read leaf and n_taken while n_kept is written)
  if (overlap(n_kept, each, leaf, each) || (n_taken && overlap(n_kept, each, n_taken, each))) return DYNTS_EINVAL;
  const size_t rows = (size_t)c.Nb * n_tokens * c.Hq;
  if ((q_kept && overlap(q_kept, rows * c.D * 2, q, rows * c.D * 2)) || (lse_kept && overlap(lse_kept, rows * 4, lse, rows * 4))) return DYNTS_EINVAL;
  // (an update owed by a single step counts slots that move now, if the draft, or its end, was appended by such steps)
  const int owed = dynts_update_scores(ctx, layer, stream);
  if (owed != DYNTS_OK) return owed;
  const dynts::TreeKeepParams p{c, seen, leaf, n_taken, n_kept, q, lse, q_kept, lse_kept, n_tokens, (n_tokens + 31) / 32};
  // (a gathering workgroup for eight kept tokens, four at most)
  const unsigned gather = q_kept || lse_kept ? (n_tokens > 24 ? 4 : (n_tokens + 7) / 8) : 0;
  const dim3 grid(1 + gather, c.Nb), block(dynts::kKeepThreads);
  if (c.D == 128) hipLaunchKernelGGL((dynts::tree_keep_kernel<128>), grid, block, 0, static_cast<hipStream_t>(stream), p);
  else hipLaunchKernelGGL((dynts::tree_keep_kernel<64>), grid, block, 0, static_cast<hipStream_t>(stream), p);
  return launch_status();
}

}  // extern "C"
