// AdamW over the tensors of all workers, moments in 32 or 8 bits (device code).
#pragma once

#include "choco_philox.h"
#include "choco_types.h"

namespace choco {

enum { STREAM_ADAMW = 3 };
constexpr int kMomentBlock = 256;   // entries of a tensor that share a scale
constexpr int kTileBlocks = 4;      // ... and how many such blocks of one tensor a wave takes
constexpr int kTile = kMomentBlock * kTileBlocks;

// A piece of a tensor: what a wave takes.
struct AdamwTile {
  int32_t start, len;    // in the row
  int32_t block;         // number of its first block; -1: entries of no tensor
  float lr_scale, weight_decay;
  int32_t pad[3];
};

struct AdamwArgs {
  float* x;
  const void* g;
  const float* grad_scale;   // per worker, or null
  void *m, *v;               // fp32 or bytes, laid out like x
  float *m_scale, *v_scale;  // 8 bits: per worker and block
  float *m_out, *v_out;      // read-back
  const AdamwTile* tiles;
  int32_t ntiles, nblocks;
  int64_t ld;
  float beta1, one_minus_beta1, beta2, one_minus_beta2;
  float lr, rate, root_scale, eps;   // rate = lr / (1 - beta1^t), root_scale = 1 / sqrt(1 - beta2^t)
  uint32_t seed_lo, seed_hi, t_lo, t_hi;
};

// The new x.  Square root and reciprocal to one unit in the last place each: they only scale the step, which is
// small against x.
__device__ __forceinline__ float adamw_x(const AdamwArgs& A, float x, float m, float v, float rate, float keep) {
  const float root = __builtin_amdgcn_sqrtf(v) * A.root_scale + A.eps;
  return x * keep - rate * m * __builtin_amdgcn_rcpf(root);
}

// The scale of a block: the power of two that brings the bits `most` of its largest magnitude into (0.9375, 1.875].
// A power of two, because the codes are then exact multiples of one another from step to step: a moment that moves by
// 0.1 % in a step changes its code in one step of a hundred, whereas a scale that follows the largest entry would put
// every entry between two codes in every step, and rounding noise of 4 % a step adds up over the 1 / (1 - beta2) steps
// that v remembers.  Zero for a block below the normal numbers (held as zero); infinite or NaN as `most` is.
__device__ __forceinline__ uint32_t scale_bits(uint32_t most) {
  const uint32_t up = (most & 0x7FFFFFu) > 0x700000u && most < 0x7F800000u ? 1u << 23 : 0u;
  return most >= 0x7F800000u ? most : (most & 0x7F800000u) == 0 ? 0u : (most & 0x7F800000u) + up;
}
// 2^-k of a scale 2^k; 0 for the scales that are no power of two.
__device__ __forceinline__ float inverse_scale(uint32_t scale) {
  return scale == 0u || scale >= 0x7F800000u ? 0.0f : scale == 254u << 23 ? 5.87747175e-39f : __uint_as_float((254u << 23) - scale);
}

// What a code of 3 mantissa bits under TOP exponents stands for relative to its scale, at most 1.875: its bits are those of a
// (denormal, below the lowest exponent) float, scaled up by a power of two.
template <int TOP>
__device__ __forceinline__ float code_value(uint32_t code) {
  return __uint_as_float(code << 20) * __uint_as_float((uint32_t)(127 - TOP + 127) << 23);
}
// ... and the code of |x| = y <= 1.875, r of 65536 deciding whether what is cut off is rounded up.
template <int TOP>
__device__ __forceinline__ uint32_t value_code(float y, uint32_t r) {
  const uint32_t bits = __float_as_uint(y * __uint_as_float((uint32_t)TOP << 23));
  const uint32_t code = (bits + (r << 4)) >> 20;
  return code < 8u * TOP + 7u ? code : 8u * TOP + 7u;
}

// Largest of a wave's values by their bits: these are non-negative floats (or NaN, which is above all).
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) {
    const uint32_t y = (uint32_t)__shfl_xor((int)x, off, 64);
    x = x > y ? x : y;
  }
  return x;
}

// An entry of a block for every lane and turn: entry lane + 64 j.
template <class G, int BITS>
__global__ __launch_bounds__(256) void k_adamw(AdamwArgs A) {
  const int lane = threadIdx.x & 63, w = blockIdx.y;
  const int ti = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (ti >= A.ntiles) return;
  const AdamwTile tile = A.tiles[ti];
  const float gs = A.grad_scale ? A.grad_scale[w] : 1.0f;
  if (!(fabsf(gs) <= 3.402823466e38f)) return;
  const int64_t row = (int64_t)w * A.ld;
  const float rate = A.rate * tile.lr_scale, keep = 1.0f - A.lr * tile.lr_scale * tile.weight_decay;
  for (int b = 0; b * kMomentBlock < tile.len; ++b) {
    const int64_t block = (int64_t)w * A.nblocks + tile.block + b;
    float m[4], v[4];
    uint32_t most_m = 0, most_v = 0;
    float old_m = 0.0f, old_v = 0.0f;
    if (BITS == 8) { old_m = A.m_scale[block]; old_v = A.v_scale[block]; }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int at = b * kMomentBlock + j * 64 + lane;
      m[j] = v[j] = 0.0f;
      if (at >= tile.len) continue;
      const int64_t e = row + tile.start + at;
      const float g = to_float(((const G*)A.g)[e]) * gs;
      if (BITS == 32) {
        m[j] = ((const float*)A.m)[e];
        v[j] = ((const float*)A.v)[e];
      } else {
        const uint32_t cm = ((const uint8_t*)A.m)[e], cv = ((const uint8_t*)A.v)[e];
        m[j] = code_value<15>(cm & 127u) * old_m;
        if (cm & 128u) m[j] = -m[j];
        v[j] = code_value<31>(cv) * old_v;
      }
      m[j] = m[j] * A.beta1 + g * A.one_minus_beta1;
      v[j] = v[j] * A.beta2 + (g * g) * A.one_minus_beta2;
      A.x[e] = adamw_x(A, A.x[e], m[j], v[j], rate, keep);
      if (BITS == 32) {
        ((float*)A.m)[e] = m[j];
        ((float*)A.v)[e] = v[j];
      } else {
        const uint32_t bm = __float_as_uint(m[j]) & 0x7FFFFFFFu, bv = __float_as_uint(v[j]) & 0x7FFFFFFFu;
        most_m = bm > most_m ? bm : most_m;
        most_v = bv > most_v ? bv : most_v;
      }
    }
    if (BITS == 32) continue;
    const uint32_t scale_m = scale_bits(wave_max(most_m)), scale_v = scale_bits(wave_max(most_v));
    const float up_m = inverse_scale(scale_m), up_v = inverse_scale(scale_v);
    if (lane == 0) {
      A.m_scale[block] = __uint_as_float(scale_m);
      A.v_scale[block] = __uint_as_float(scale_v);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int at = b * kMomentBlock + j * 64 + lane;
      if (at >= tile.len) continue;
      const int32_t e = tile.start + at;
      const uint4 words = philox4x32_10((uint32_t)e >> 2, (uint32_t)w, A.t_lo, STREAM_ADAMW | (A.t_hi << 8), A.seed_lo, A.seed_hi);
      const uint32_t word = (e & 3) == 0 ? words.x : (e & 3) == 1 ? words.y : (e & 3) == 2 ? words.z : words.w;
      uint32_t cm = value_code<15>(fabsf(m[j]) * up_m, word & 0xFFFFu);
      if (m[j] < 0.0f) cm |= 128u;
      uint32_t cv = value_code<31>(v[j] * up_v, word >> 16);
      if (cv == 0 && v[j] > 0.0f) cv = 1;
      ((uint8_t*)A.m)[row + e] = (uint8_t)cm;
      ((uint8_t*)A.v)[row + e] = (uint8_t)cv;
    }
  }
}

// The moments as floats.
template <int BITS>
__global__ __launch_bounds__(256) void k_adamw_moments(AdamwArgs A) {
  const int lane = threadIdx.x & 63, w = blockIdx.y;
  const int ti = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (ti >= A.ntiles) return;
  const AdamwTile tile = A.tiles[ti];
  for (int at = lane; at < tile.len; at += 64) {
    const int64_t e = (int64_t)w * A.ld + tile.start + at;
    float m = 0.0f, v = 0.0f;
    if (tile.block < 0) {
    } else if (BITS == 32) {
      m = ((const float*)A.m)[e];
      v = ((const float*)A.v)[e];
    } else {
      const int64_t block = (int64_t)w * A.nblocks + tile.block + at / kMomentBlock;
      const uint32_t cm = ((const uint8_t*)A.m)[e], cv = ((const uint8_t*)A.v)[e];
      m = code_value<15>(cm & 127u) * A.m_scale[block];
      if (cm & 128u) m = -m;
      v = code_value<31>(cv) * A.v_scale[block];
    }
    A.m_out[e] = m;
    A.v_out[e] = v;
  }
}

}  // namespace choco
