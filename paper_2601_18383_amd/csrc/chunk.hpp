// Chunks of new tokens on the cache: what the host side of their entry points (chunk.hip) shares with the contexts (dynts.hip) and
// with the kernels (chunk_append.hpp, chunk_attend.hpp, chunk_scores.hpp).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/dynts.h"

namespace dynts {

// One layer of a bound context, as these kernels see it.  dense: K and V are the layer's [Nb][Hkv][cap][D]; paged: the pools, slot j of a unit
// in row j % 64 of page block_table[unit][j / 64].
struct ChunkCache {
  uint16_t *K, *V;
  float *S;
  int32_t *pos, *seq_len, *next_pos, *n_prompt, *status;
  int32_t *block_table, *free_stack, *free_top;  // paged layout, else null
  int max_pages, n_pages;
  int Nb, Hq, Hkv, G, D, cap;
  int score_mode;
  float scale;  // of the softmax
  // caches of codes (dynts_bind_codes; K and V then are theirs, one byte an element): DYNTS_CODE_*, else 0, and a byte for 32 elements
  int code;
  uint8_t *K_scale, *V_scale;
};

// Looks the layer up; DYNTS_OK or the error that a call on this context and layer has to return.
__attribute__((visibility("hidden"))) int chunk_cache(const dynts_ctx *ctx, int32_t layer, ChunkCache *out);
// DYNTS_OK if dynts_create would take it.
__attribute__((visibility("hidden"))) int chunk_check_config(const dynts_config *cfg);

// two bf16 in a word
__device__ __forceinline__ float bf16_low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_high(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ uint32_t bf16_pack(float lo, float hi) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)lo, (__bf16)hi});
}

}  // namespace dynts
