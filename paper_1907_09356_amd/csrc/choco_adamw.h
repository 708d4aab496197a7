// AdamW over the tensors of all workers, moments in 32 or 8 bits (device code).
//
// Bound by memory: 28 bytes an entry in 32 bits (x, m and v in and out, g in), 16 in 8 bits (14 with g in bf16).  The tensors of a row are
// cut into tiles of 1024 entries, a wave each, listed in a table, so one launch takes all tensors of all workers and no
// wave looks for its tensor; a tile's loads are all asked for before the first is used.  254 M entries in 32 bits 1,305 us (5.5 TB/s)
// and their read-back 732, 127 M in 8 bits 310 to 333 (5.5 to 5.9 TB/s) and their read-back 206; 2.2 M, out of the caches, 10.4 (6.0 TB/s).
// Entry by entry before: 2,273, and 790 with the read-back of 8 bits.  Tiles of 512 or 2048 entries: 0 to 4 % slower.
#pragma once

#include "choco_philox.h"
#include "choco_types.h"

namespace choco {

enum { STREAM_ADAMW = 3 };
constexpr int kMomentBlock = 256;   // entries of a tensor that share a scale
constexpr int kTileBlocks = 4;      // ... and how many such blocks of one tensor a wave takes
constexpr int kTile = kMomentBlock * kTileBlocks;
// eps is at least this / sqrt(1 - beta2).  A step rounds v by up to 2^-149 (two products below the normal numbers), and
// t steps' worth of that over 1 - beta2^t, the root taken, is 2^-74.5 / sqrt(1 - beta2): 2^-14 of eps at the most.
constexpr double kLeastEps = 0x1p-60;

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
// small against x.  The square root's instruction takes a v below the normal numbers for zero, so a small one is scaled up
// first; what then is lost of v are fp32's own roundings, which the least eps that a plan may have (kLeastEps) outweighs.  It
// is a normal number, as the reciprocal's instruction wants it.
__device__ __forceinline__ float adamw_x(const AdamwArgs& A, float x, float m, float v, float rate, float keep) {
  const bool low = v < 0x1p-100f;
  const float root = __builtin_amdgcn_sqrtf(low ? v * 0x1p32f : v) * (low ? A.root_scale * 0x1p-16f : A.root_scale) + A.eps;
  return x * keep - rate * m * __builtin_amdgcn_rcpf(root);
}

// The scale of a block is the power of two that brings the largest magnitude into (0.9375, 1.875]: its exponent field is that of
// the largest number with the cut-off bits below 1.875 carried up, so lanes compare exponent fields, those of m and v at once.
// A power of two, because the codes are then exact multiples of one another from step to step: a moment that moves by
// 0.1 % in a step changes its code in one step of a hundred, whereas a scale that follows the largest entry would put
// every entry between two codes in every step, and rounding noise of 4 % a step adds up over the 1 / (1 - beta2) steps
// that v remembers.  (Simulated over 4000 steps: v stays within 0.3 % of itself on average, with a spread of 20 %; m 9 %.)  A
// block whose largest lies below the normal numbers has the least normal scale, that of field 1; code 1 of v then stands for less than any
// number, so a positive v stays positive.  Fields of 255 and more: something in the block is infinite or NaN.
typedef uint16_t Fields __attribute__((ext_vector_type(2)));   // of m and of v
__device__ __forceinline__ uint32_t scale_field(float x) { return ((__float_as_uint(x) & 0x7FFFFFFFu) + 0xFFFFFu) >> 23; }
__device__ __forceinline__ float scale_of(uint32_t field) { return __uint_as_float(field >= 255u ? 0x7FC00000u : field << 23); }
// 2^-k of a scale 2^k, fields from 1; 0 for those of no power of two.
__device__ __forceinline__ float inverse_scale(uint32_t field) {
  return field >= 255u ? 0.0f : field == 254u ? 5.87747175e-39f : __uint_as_float((254u - field) << 23);
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

// Largest fields of a wave, in every lane: the halves and neighbouring rows of 16 lanes swapped, then rotations and permutations
// within a row, all by moves of the vector unit.
template <int CTRL>
__device__ __forceinline__ Fields moved_max(Fields x) {
  const Fields y = __builtin_bit_cast(Fields, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xF, 0xF, true));
  return __builtin_elementwise_max(x, y);
}
__device__ __forceinline__ Fields pair_max(uint32_t x, uint32_t y) {
  return __builtin_elementwise_max(__builtin_bit_cast(Fields, x), __builtin_bit_cast(Fields, y));
}
__device__ __forceinline__ Fields wave_max(Fields x) {
  const uint32_t b = __builtin_bit_cast(uint32_t, x);
  const auto halves = __builtin_amdgcn_permlane32_swap(b, b, false, false);
  x = pair_max(halves[0], halves[1]);
  const uint32_t c = __builtin_bit_cast(uint32_t, x);
  const auto rows = __builtin_amdgcn_permlane16_swap(c, c, false, false);
  x = pair_max(rows[0], rows[1]);
  x = moved_max<0x128>(x);    // row_ror 8
  x = moved_max<0x124>(x);    // row_ror 4
  x = moved_max<0x4E>(x);     // quad_perm [2,3,0,1]
  return moved_max<0xB1>(x);  // quad_perm [1,0,3,2]
}

// The four entries that a lane takes of a block: next to one another, from the first that the lane's number times four
// reaches, where the tensor starts on a multiple of four; every 64th otherwise.
template <bool ALIGNED>
__device__ __forceinline__ int entry_of(int lane, int i) { return ALIGNED ? lane * 4 + i : i * 64 + lane; }

// A lane's entries of those from p on; there are `left` of them (kMomentBlock or more: no lane has to look).
template <bool ALIGNED, bool STREAM, class T>
__device__ __forceinline__ void load_four(const T* p, int lane, int left, T (&x)[4]) {
  if (ALIGNED && (left >= kMomentBlock || lane * 4 + 4 <= left)) {
    typedef T Four __attribute__((ext_vector_type(4)));
    Four v;
    // (codes through the caches: asked for past them, 127 M entries take 570 us instead of 518)
    if constexpr (STREAM && sizeof(T) > 1) v = __builtin_nontemporal_load(reinterpret_cast<const Four*>(p + lane * 4));
    else v = *reinterpret_cast<const Four*>(p + lane * 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = v[i];
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = entry_of<ALIGNED>(lane, i) < left ? p[entry_of<ALIGNED>(lane, i)] : T(0);
  }
}
template <bool ALIGNED, bool STREAM, class T>
__device__ __forceinline__ void store_four(T* p, int lane, int left, const T (&x)[4]) {
  if (ALIGNED && (left >= kMomentBlock || lane * 4 + 4 <= left)) {
    typedef T Four __attribute__((ext_vector_type(4)));
    Four v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = x[i];
    if constexpr (STREAM) __builtin_nontemporal_store(v, reinterpret_cast<Four*>(p + lane * 4));
    else *reinterpret_cast<Four*>(p + lane * 4) = v;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (entry_of<ALIGNED>(lane, i) < left) p[entry_of<ALIGNED>(lane, i)] = x[i];
  }
}

// The words of a lane's entries in the BLOCKS blocks from entry e on.
template <bool ALIGNED, int BLOCKS>
__device__ __forceinline__ void entry_words(const AdamwArgs& A, int w, uint32_t e, int lane, uint32_t (&words)[BLOCKS][4]) {
  const uint32_t c3 = STREAM_ADAMW | (A.t_hi << 8);
  if (ALIGNED) {
    uint4 four[BLOCKS];
    philox_side_by_side<BLOCKS>((e >> 2) + lane, (uint32_t)w, A.t_lo, c3, A.seed_lo, A.seed_hi, four);
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) {
      words[b][0] = four[b].x;
      words[b][1] = four[b].y;
      words[b][2] = four[b].z;
      words[b][3] = four[b].w;
    }
  } else {
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t at = e + b * kMomentBlock + entry_of<false>(lane, i);
        const uint4 four = philox4x32_10(at >> 2, (uint32_t)w, A.t_lo, c3, A.seed_lo, A.seed_hi);
        words[b][i] = (at & 3) == 0 ? four.x : (at & 3) == 1 ? four.y : (at & 3) == 2 ? four.z : four.w;
      }
  }
}

// A wave takes a tile: loads everything of its blocks, then computes and writes them.  FULL: the blocks are whole.
template <class G, int BITS, bool STREAM, bool ALIGNED, bool FULL, int BLOCKS>
__device__ __forceinline__ void adamw_tile(const AdamwArgs& A, const AdamwTile& tile, int w, float gs, int first) {
  const int lane = threadIdx.x & 63;
  const int64_t at = (int64_t)w * A.ld + tile.start + first;
  const int64_t block = (int64_t)w * A.nblocks + tile.block + first / kMomentBlock;
  const float rate = A.rate * tile.lr_scale, keep = 1.0f - A.lr * tile.lr_scale * tile.weight_decay;
  float x[BLOCKS][4], m[BLOCKS][4], v[BLOCKS][4];
  G g[BLOCKS][4];
  uint8_t cm[BLOCKS][4], cv[BLOCKS][4];
  float old_m[BLOCKS], old_v[BLOCKS];
#pragma unroll
  for (int b = 0; b < BLOCKS; ++b) {
    const int64_t e = at + b * kMomentBlock;
    const int left = FULL ? kMomentBlock : tile.len - first - b * kMomentBlock;
    load_four<ALIGNED, STREAM>((const G*)A.g + e, lane, left, g[b]);
    if (BITS == 32) {
      load_four<ALIGNED, STREAM>((const float*)A.m + e, lane, left, m[b]);
      load_four<ALIGNED, STREAM>((const float*)A.v + e, lane, left, v[b]);
    } else {
      load_four<ALIGNED, STREAM>((const uint8_t*)A.m + e, lane, left, cm[b]);
      load_four<ALIGNED, STREAM>((const uint8_t*)A.v + e, lane, left, cv[b]);
      old_m[b] = left > 0 ? A.m_scale[block + b] : 0.0f;
      old_v[b] = left > 0 ? A.v_scale[block + b] : 0.0f;
    }
    load_four<ALIGNED, STREAM>(A.x + e, lane, left, x[b]);
  }
  uint32_t words[BLOCKS][4];
  if (BITS == 8) entry_words<ALIGNED, BLOCKS>(A, w, (uint32_t)(tile.start + first), lane, words);
#pragma unroll
  for (int b = 0; b < BLOCKS; ++b) {
    const int64_t e = at + b * kMomentBlock;
    const int left = FULL ? kMomentBlock : tile.len - first - b * kMomentBlock;
    Fields top = {1, 1};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (BITS == 8) {
        m[b][i] = code_value<15>(cm[b][i] & 127u) * old_m[b];
        if (cm[b][i] & 128u) m[b][i] = -m[b][i];
        v[b][i] = code_value<31>(cv[b][i]) * old_v[b];
      }
      const float gr = to_float(g[b][i]) * gs;
      m[b][i] = m[b][i] * A.beta1 + gr * A.one_minus_beta1;
      v[b][i] = v[b][i] * A.beta2 + (gr * gr) * A.one_minus_beta2;
      x[b][i] = adamw_x(A, x[b][i], m[b][i], v[b][i], rate, keep);
      if (BITS == 8 && entry_of<ALIGNED>(lane, i) < left)
        top = __builtin_elementwise_max(top, Fields{(uint16_t)scale_field(m[b][i]), (uint16_t)scale_field(v[b][i])});
    }
    store_four<ALIGNED, STREAM>(A.x + e, lane, left, x[b]);
    if (BITS == 32) {
      store_four<ALIGNED, STREAM>((float*)A.m + e, lane, left, m[b]);
      store_four<ALIGNED, STREAM>((float*)A.v + e, lane, left, v[b]);
      continue;
    }
    top = wave_max(top);
    const float up_m = inverse_scale(top[0]), up_v = inverse_scale(top[1]);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t code = value_code<15>(fabsf(m[b][i]) * up_m, words[b][i] & 0xFFFFu);
      cm[b][i] = (uint8_t)(m[b][i] < 0.0f ? code | 128u : code);
      const uint32_t code_v = value_code<31>(v[b][i] * up_v, words[b][i] >> 16);
      cv[b][i] = (uint8_t)(code_v == 0u && v[b][i] > 0.0f ? 1u : code_v);
    }
    store_four<ALIGNED, STREAM>((uint8_t*)A.m + e, lane, left, cm[b]);
    store_four<ALIGNED, STREAM>((uint8_t*)A.v + e, lane, left, cv[b]);
    if (lane == 0 && left > 0) {
      A.m_scale[block + b] = scale_of(top[0]);
      A.v_scale[block + b] = scale_of(top[1]);
    }
  }
}

// Tiles of whole blocks that start on a multiple of four entries - nearly all of a model's - go through at once, the others
// block by block.
template <class G, int BITS, bool STREAM>
__global__ __launch_bounds__(256) void k_adamw(AdamwArgs A) {
  const int w = blockIdx.y;
  const int ti = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (ti >= A.ntiles) return;
  const AdamwTile tile = A.tiles[ti];
  const float gs = A.grad_scale ? A.grad_scale[w] : 1.0f;
  if (!(fabsf(gs) <= 3.402823466e38f)) return;
  if ((tile.start & 3) == 0 && tile.len == kTile) {
    adamw_tile<G, BITS, STREAM, true, true, kTileBlocks>(A, tile, w, gs, 0);
  } else if ((tile.start & 3) == 0) {
    for (int first = 0; first < tile.len; first += kMomentBlock) adamw_tile<G, BITS, STREAM, true, false, 1>(A, tile, w, gs, first);
  } else {
    for (int first = 0; first < tile.len; first += kMomentBlock) adamw_tile<G, BITS, STREAM, false, false, 1>(A, tile, w, gs, first);
  }
}

// The moments as floats.
template <int BITS, bool ALIGNED, bool FULL, int BLOCKS>
__device__ __forceinline__ void adamw_moments_tile(const AdamwArgs& A, const AdamwTile& tile, int w, int first) {
  constexpr bool STREAM = true;
  const int lane = threadIdx.x & 63;
  const int64_t at = (int64_t)w * A.ld + tile.start + first;
  const int64_t block = (int64_t)w * A.nblocks + tile.block + first / kMomentBlock;
  float m[BLOCKS][4], v[BLOCKS][4], scale_m[BLOCKS], scale_v[BLOCKS];
  uint8_t cm[BLOCKS][4], cv[BLOCKS][4];
#pragma unroll
  for (int b = 0; b < BLOCKS; ++b) {
    const int64_t e = at + b * kMomentBlock;
    const int left = FULL ? kMomentBlock : tile.len - first - b * kMomentBlock;
    if (BITS == 32) {
      load_four<ALIGNED, STREAM>((const float*)A.m + e, lane, left, m[b]);
      load_four<ALIGNED, STREAM>((const float*)A.v + e, lane, left, v[b]);
    } else {
      load_four<ALIGNED, STREAM>((const uint8_t*)A.m + e, lane, left, cm[b]);
      load_four<ALIGNED, STREAM>((const uint8_t*)A.v + e, lane, left, cv[b]);
      scale_m[b] = tile.block >= 0 ? A.m_scale[block + b] : 0.0f;
      scale_v[b] = tile.block >= 0 ? A.v_scale[block + b] : 0.0f;
    }
  }
#pragma unroll
  for (int b = 0; b < BLOCKS; ++b) {
    const int64_t e = at + b * kMomentBlock;
    const int left = FULL ? kMomentBlock : tile.len - first - b * kMomentBlock;
    if (BITS == 8) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        m[b][i] = code_value<15>(cm[b][i] & 127u) * scale_m[b];
        if (cm[b][i] & 128u) m[b][i] = -m[b][i];
        v[b][i] = code_value<31>(cv[b][i]) * scale_v[b];
      }
    }
    store_four<ALIGNED, STREAM>(A.m_out + e, lane, left, m[b]);
    store_four<ALIGNED, STREAM>(A.v_out + e, lane, left, v[b]);
  }
}

// (Entries of no tensor hold zeros, codes and floats alike.)
template <int BITS>
__global__ __launch_bounds__(256) void k_adamw_moments(AdamwArgs A) {
  const int w = blockIdx.y;
  const int ti = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (ti >= A.ntiles) return;
  const AdamwTile tile = A.tiles[ti];
  if ((tile.start & 3) == 0 && tile.len == kTile) {
    adamw_moments_tile<BITS, true, true, kTileBlocks>(A, tile, w, 0);
  } else if ((tile.start & 3) == 0) {
    for (int first = 0; first < tile.len; first += kMomentBlock) adamw_moments_tile<BITS, true, false, 1>(A, tile, w, first);
  } else {
    for (int first = 0; first < tile.len; first += kMomentBlock) adamw_moments_tile<BITS, false, false, 1>(A, tile, w, first);
  }
}

}  // namespace choco
