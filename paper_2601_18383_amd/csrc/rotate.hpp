// Rotary positions with several axes.  Pair p of a head (a, b) is turned by theta = positions[axis[p]][token] * freq[p]:
//   a' = a cos theta - b sin theta,   b' = b cos theta + a sin theta;
// the gradient with respect to the input is the turn back, by -theta.
//
// Bound by HBM: every element is read and written once.  8192 tokens of 40 heads of 128, 168 MB in 32 us (5.2 TB/s, a large copy's rate), on the same arrays
// again in 25 (part of it out of the memory-side cache).  A token a workgroup: its angles are computed once, in LDS, for all heads.  Small calls are a launch, 3 us.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "attend.hpp"
#include "chunk.hpp"

namespace dynts {

struct RotateParams {
  const uint16_t *q, *k;     // [tokens][q_heads][D], [tokens][k_heads][D] or null
  uint16_t *q_out, *k_out;
  const int32_t *positions;  // [n_axes][tokens]
  const float *freq;         // [pairs], radians a position
  const uint8_t *axis;       // [pairs] or null: axis 0
  int tokens, q_heads, k_heads, D, pairs, n_axes;
  float sign;                // -1: the gradient
};

constexpr int kRotThreads = 256;
constexpr int kRotMaxPairs = 128;
constexpr int kRotMaxTokens = 1 << 24;  // (a grid holds fewer than 2^32 threads)

// grid (tokens), one token a workgroup.
template <bool ADJACENT>
__global__ __launch_bounds__(kRotThreads) void rotate_kernel(const RotateParams p) {
  __shared__ float sm_cos[kRotMaxPairs], sm_sin[kRotMaxPairs];
  const int t = blockIdx.x, tid = threadIdx.x;
  for (int i = tid; i < p.pairs; i += kRotThreads) {
    int a = p.axis ? p.axis[i] : 0;
    a = a < p.n_axes ? a : p.n_axes - 1;
    // Whole turns leave in 64 bits: a position of 2^20 times a frequency has four bits behind the point in 32.
    const double turns = (double)p.positions[(size_t)a * p.tokens + t] * (double)p.freq[i] * 0.15915494309189533577;
    const float part = (float)(turns - rint(turns));
    float s, c;
    sincospif(2.f * part, &s, &c);
    sm_cos[i] = c;
    sm_sin[i] = p.sign * s;
  }
  __syncthreads();
  // Units of work: eight pairs of a head (HALVES: eight elements and their partners `pairs` further on; ADJACENT: sixteen in a row), or
  // eight elements behind the turned ones.
  const int turned = p.pairs / 8, units = turned + (p.D - 2 * p.pairs) / 8, heads = p.q_heads + p.k_heads;
  for (int w = tid; w < heads * units; w += kRotThreads) {
    const int h = w / units, u = w - h * units;
    const bool is_q = h < p.q_heads;
    const size_t row = is_q ? ((size_t)t * p.q_heads + h) * p.D : ((size_t)t * p.k_heads + (h - p.q_heads)) * p.D;
    const uint16_t *src = (is_q ? p.q : p.k) + row;
    uint16_t *dst = (is_q ? p.q_out : p.k_out) + row;
    if (u >= turned) {
      const int e = 2 * p.pairs + 8 * (u - turned);
      store_u32x4(dst + e, load_u32x4(src + e));
      continue;
    }
    const int e0 = ADJACENT ? 16 * u : 8 * u, e1 = ADJACENT ? 16 * u + 8 : p.pairs + 8 * u;
    u32x4 x = load_u32x4(src + e0), y = load_u32x4(src + e1);
    const float *c = sm_cos + 8 * u, *s = sm_sin + 8 * u;
    if (ADJACENT) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float a0 = bf16_low(x[j]), b0 = bf16_high(x[j]), a1 = bf16_low(y[j]), b1 = bf16_high(y[j]);
        x[j] = bf16_pack(a0 * c[j] - b0 * s[j], b0 * c[j] + a0 * s[j]);
        y[j] = bf16_pack(a1 * c[4 + j] - b1 * s[4 + j], b1 * c[4 + j] + a1 * s[4 + j]);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float a0 = bf16_low(x[j]), a1 = bf16_high(x[j]), b0 = bf16_low(y[j]), b1 = bf16_high(y[j]);
        x[j] = bf16_pack(a0 * c[2 * j] - b0 * s[2 * j], a1 * c[2 * j + 1] - b1 * s[2 * j + 1]);
        y[j] = bf16_pack(b0 * c[2 * j] + a0 * s[2 * j], b1 * c[2 * j + 1] + a1 * s[2 * j + 1]);
      }
    }
    store_u32x4(dst + e0, x);
    store_u32x4(dst + e1, y);
  }
}

}  // namespace dynts
