// Launches of the kernels for caches of codes and for drafts that branch (forms.hip).
#pragma once
#include "chunk_attend.hpp"
#include "chunk_scores.hpp"
#include "coded_token.hpp"

namespace dynts {

// tokens of a draft (tree_keep_kernel has them in LDS)
constexpr int kTreeMost = 4096;

// chunk_attend_few_kernel's other forms: mask kTree, or a cache of codes with any mask.
__attribute__((visibility("hidden"))) void launch_few_form(const ChunkAttendParams &p, int mask, unsigned grid, hipStream_t st);
// many rows on a cache of codes, mask kPlain or kTree
__attribute__((visibility("hidden"))) void launch_coded_attend(const ChunkAttendParams &p, int mask, unsigned grid, hipStream_t st);
// up to kTokRows rows on a cache of codes
__attribute__((visibility("hidden"))) void launch_coded_token(const ChunkAttendParams &p, bool shaped, unsigned grid, hipStream_t st);
__attribute__((visibility("hidden"))) void launch_coded_token_scores(const ChunkScoreParams &p, bool shaped, unsigned grid, hipStream_t st);
// many rows: a draft's tokens; groups of waves, with mask kPlain (caches of codes) or kTree, for kChRows rows a workgroup, or kHalfRows (unsplit)
__attribute__((visibility("hidden"))) void launch_tree_attend(const ChunkAttendParams &p, unsigned grid, hipStream_t st);
__attribute__((visibility("hidden"))) void launch_attend_half(const ChunkAttendParams &p, int mask, unsigned grid, hipStream_t st);
__attribute__((visibility("hidden"))) void launch_attend_groups(const ChunkAttendParams &p, int mask, unsigned grid, hipStream_t st);
// the shares of a draft's rows, or of rows on a cache of codes, together
__attribute__((visibility("hidden"))) void launch_merge_form(const ChunkAttendParams &p, int block_rows, hipStream_t st);
__attribute__((visibility("hidden"))) void launch_coded_scores(const ChunkScoreParams &p, bool few, bool shaped, bool biased, unsigned grid, hipStream_t st);
// small: one launch that makes room and writes; else one (behind chunk_reserve_kernel) that writes
__attribute__((visibility("hidden"))) void launch_coded_append(const ChunkAppendParams &p, bool small, hipStream_t st);
// rows of a cache as bf16; past: the caches, for who does not read them next (bf16 caches: always)
__attribute__((visibility("hidden"))) void launch_read_rows(const ChunkCache &c, const int32_t *first, int n_rows, uint16_t *K, uint16_t *V, bool past, hipStream_t st);

}  // namespace dynts
