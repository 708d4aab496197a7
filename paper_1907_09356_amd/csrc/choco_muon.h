// Newton-Schulz iterations X <- a X + (b P + c P^2) X, P = X X^T, on stacks of matrices, and an optimiser step along their
// result (device code).
//
// A matrix is taken with its shorter side first: a x b entries, a <= b.  Every product is of rows with rows, D[m][n] = sum over k of
// L[m][k] R[n][k]:  P from X and X,  Q = a I + b P + c P^2 from P and P (symmetric),  X' = Q X from Q and X^T.  So X is held both
// ways, X^T twice (a launch reads one and writes the other).
//
// Bound by matrix instructions: with symmetric products by half 5 (3 a^2 b + a^3) operations, three fp16 instructions each, against some 20 bytes
// an entry.  Measured, us: eight workers' six 2600 x 650 4,980 (2,230 at the rate of a large fp16 product by the library), 16 of 1024 x 640 720
// (317), 333 x 1000 alone 193, four of 64 x 192 37.  Before: products straight out of memory, a wave 32 x 32, 18,840, 2,460, 480 and 158; in tiles
// of 128 through LDS 6,620 and 1,030; neighbouring tiles on one XCD 6,000 and 760; a X by Q's diagonal 5,640; all matrices at once 4,980.
//
// Operands are two fp16 numbers for one fp32, 2^13 x = high + low.  No entry of X, P or Q is beyond 3.5 (their singular
// values are not), so high is below 2^15, and low keeps 11 bits more down to 2^-24: 22 bits of an entry above 2^-15, 2^-38 of a smaller
// one.  A product takes high high + high low + low high on the matrix cores, where sums are fp32; the last, low low, is 2^-22 of the
// first.
#pragma once

#include <type_traits>

#include "choco_types.h"

namespace choco {

constexpr float kMuonA = 3.4445f, kMuonB = -4.7750f, kMuonC = 2.0315f;
constexpr float kMuonUp = 8192.0f, kMuonDown = 1.0f / 8192.0f;
constexpr int kMuonPad = 32;      // rows of operands end on a multiple of so many entries, with zeros: a step along the inner index
constexpr int kMuonMost = 1 << 16;

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef float float4_t __attribute__((ext_vector_type(4)));

// Matrices of one shape: one of each of some workers from `first` on.
struct MuonShape {
  int64_t source, source_of;      // entries from the source's begin to the first worker's matrix, and from there to the next's
  int64_t target, target_of;      // of x or of the result
  int64_t moment;                 // of worker 0's momentum; the next is rows * cols behind
  int64_t source_ld, target_ld;
  int64_t scratch, scratch_of;    // bytes
  int64_t partials;               // sums of squares of the tiles, one matrix behind the other
  int32_t rows, cols, a, b, a_ld, b_ld, first;
  float decay, rate;
  uint32_t start_begin, gram_begin, apply_begin;    // tiles before these matrices'
  uint32_t start_tiles, gram_tiles, apply_tiles;    // of one of them
};

struct MuonArgs {
  MuonShape one;                  // without a table
  const MuonShape* table;
  int32_t count;
  const void* source;             // gradients or matrices
  float* target;                  // parameters or result
  float* moments;                 // null: matrices as they are
  const float* grad_scale;
  double* partials;
  char* scratch;
  float momentum, lr;
  int32_t nesterov;
  int32_t now;                    // which of the X^T is read
  bool last;
};

// The operands of a matrix, high planes with the low ones behind them.
struct MuonPlanes {
  f16_t *x, *xt[2], *p, *q;
  int64_t x_low, xt_low, p_low;
};
inline __host__ __device__ int64_t muon_scratch(int64_t a, int64_t b, int64_t a_ld, int64_t b_ld) {
  return 4 * (a * b_ld + 2 * b * a_ld + 2 * a * a_ld);
}
__device__ __forceinline__ MuonPlanes planes_of(const MuonArgs& A, const MuonShape& S, int i) {
  MuonPlanes P;
  P.x_low = (int64_t)S.a * S.b_ld;
  P.xt_low = (int64_t)S.b * S.a_ld;
  P.p_low = (int64_t)S.a * S.a_ld;
  P.x = (f16_t*)(A.scratch + S.scratch + i * S.scratch_of);
  P.xt[0] = P.x + 2 * P.x_low;
  P.xt[1] = P.xt[0] + 2 * P.xt_low;
  P.p = P.xt[1] + 2 * P.xt_low;
  P.q = P.p + 2 * P.p_low;
  return P;
}

// Which matrices a tile belongs to: the last whose tiles begin at or before it.  (The table is read as constant memory, so that what
// comes of it stays in scalar registers.)
typedef const __attribute__((address_space(4))) uint32_t ConstantWord;
static_assert(sizeof(MuonShape) % 4 == 0);
__device__ __forceinline__ MuonShape shape_at(const MuonArgs& A, int i) {
  struct Words { uint32_t w[sizeof(MuonShape) / 4]; } words;
  ConstantWord* from = (ConstantWord*)(uintptr_t)(A.table + i);
#pragma unroll
  for (size_t k = 0; k < sizeof(MuonShape) / 4; ++k) words.w[k] = from[k];
  return __builtin_bit_cast(MuonShape, words);
}
template <uint32_t MuonShape::*BEGIN>
__device__ __forceinline__ MuonShape shape_of(const MuonArgs& A, uint32_t tile) {
  if (!A.table) return A.one;
  int lo = 0, hi = A.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (shape_at(A, mid).*BEGIN <= tile) lo = mid;
    else hi = mid - 1;
  }
  return shape_at(A, lo);
}

__device__ __forceinline__ void split(float x, f16_t& high, f16_t& low) {
  high = (f16_t)x;
  low = (f16_t)(x - (float)high);
}

// ---- from gradients to the first X ----
// A tile of 64 x 64 entries of the matrix as it lies in memory; a thread takes 16 of a column.
struct MuonTile {
  int i;              // which of the shape's matrices
  int64_t row, col;
};
__device__ __forceinline__ MuonTile start_tile(const MuonShape& S) {
  const uint32_t at = blockIdx.x - S.start_begin, in = at % S.start_tiles, wide = (S.cols + 63) / 64;
  return {(int)(at / S.start_tiles), (int64_t)(in / wide) * 64, (int64_t)(in % wide) * 64};
}
template <class T>
__device__ __forceinline__ float source_entry(const MuonArgs& A, const MuonShape& S, int i, int64_t r, int64_t c) {
  return to_float(((const T*)A.source)[S.source + i * S.source_of + r * S.source_ld + c]);
}
// The momentum's update; the sum of squares of what is to be orthogonalised.
template <class T, bool STEP>
__global__ __launch_bounds__(256) void k_muon_squares(MuonArgs A) {
  __shared__ double part[4];
  const MuonShape S = shape_of<&MuonShape::start_begin>(A, blockIdx.x);
  const MuonTile M = start_tile(S);
  const int worker = S.first + M.i;
  const float scale = STEP && A.grad_scale ? A.grad_scale[worker] : 1.0f;
  const int64_t c = M.col + (threadIdx.x & 63);
  double sum = 0.0;
  if (c < S.cols)
    for (int j = threadIdx.x >> 6; j < 64; j += 4) {
      const int64_t r = M.row + j;
      if (r >= S.rows) break;
      float u = source_entry<T>(A, S, M.i, r, c);
      if (STEP) {
        float* m = A.moments + S.moment + ((int64_t)worker * S.rows + r) * S.cols + c;
        if (__builtin_isfinite(scale)) {
          const float g = u * scale, now = fmaf(A.momentum, *m, g);
          *m = now;
          u = A.nesterov ? fmaf(A.momentum, now, g) : now;
        } else {
          u = 0.0f;
        }
      }
      sum += (double)u * (double)u;
    }
  for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0) A.partials[S.partials + blockIdx.x - S.start_begin] = (part[0] + part[1]) + (part[2] + part[3]);
}
// X = u / |u|, both ways.
template <class T, bool STEP>
__global__ __launch_bounds__(256) void k_muon_start(MuonArgs A) {
  __shared__ float tile[64][65];
  __shared__ double part[4];
  const MuonShape S = shape_of<&MuonShape::start_begin>(A, blockIdx.x);
  const MuonTile M = start_tile(S);
  const int worker = S.first + M.i;
  const float scale = STEP && A.grad_scale ? A.grad_scale[worker] : 1.0f;
  double sum = 0.0;
  for (uint32_t t = threadIdx.x; t < S.start_tiles; t += 256) sum += A.partials[S.partials + (int64_t)M.i * S.start_tiles + t];
  for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
  __syncthreads();
  sum = (part[0] + part[1]) + (part[2] + part[3]);
  const double up = sum == 0.0 ? 0.0 : (double)kMuonUp / sqrt(sum);
  const int64_t c = M.col + (threadIdx.x & 63);
  for (int j = threadIdx.x >> 6; j < 64; j += 4) {
    const int64_t r = M.row + j;
    float u = 0.0f;
    if (c < S.cols && r < S.rows) {
      u = source_entry<T>(A, S, M.i, r, c);
      if (STEP) {
        const float g = u * scale, now = A.moments[S.moment + ((int64_t)worker * S.rows + r) * S.cols + c];
        u = A.nesterov ? fmaf(A.momentum, now, g) : now;
      }
      u = (float)((double)u * up);
    }
    tile[j][threadIdx.x & 63] = u;
  }
  __syncthreads();
  const MuonPlanes P = planes_of(A, S, M.i);
  const bool tall = S.rows > S.cols;
  // rows of X are rows of memory, or its columns
  f16_t *const along = tall ? P.xt[0] : P.x, *const across = tall ? P.x : P.xt[0];
  const int64_t along_low = tall ? P.xt_low : P.x_low, across_low = tall ? P.x_low : P.xt_low;
  const int64_t along_ld = tall ? S.a_ld : S.b_ld, across_ld = tall ? S.b_ld : S.a_ld;
  for (int j = threadIdx.x >> 6; j < 64; j += 4) {
    const int e = threadIdx.x & 63;
    f16_t high, low;
    if (M.row + j < S.rows && M.col + e < along_ld) {
      split(tile[j][e], high, low);
      f16_t* to = along + (M.row + j) * along_ld + M.col + e;
      to[0] = high;
      to[along_low] = low;
    }
    if (M.col + j < S.cols && M.row + e < across_ld) {
      split(tile[e][j], high, low);
      f16_t* to = across + (M.col + j) * across_ld + M.row + e;
      to[0] = high;
      to[across_low] = low;
    }
  }
}

// ---- small matrices ----
// A workgroup takes a whole matrix, whose operands stay in LDS from the first iteration to the last.  Bound by latency: a product, its reads and
// writes of LDS and a barrier, is some 2 us, four of 64 x 192 37 in all (eight waves 56; seventeen launches 115).  Rows end on a multiple of 32 entries
// and 8 more, which are 4 banks modulo 16, so that 16 lanes that read 16 bytes of 16 rows meet all banks.
constexpr int kWholeWaves = 16;
constexpr int64_t kWholeBytes = 160 * 1024 - 256;
constexpr int kWholeTiles = 4;       // most 16 x 16 tiles of X that a wave makes
inline __host__ __device__ int64_t whole_bytes(int64_t a, int64_t b) {
  const int64_t ra = (a + 31) / 32 * 32, rb = (b + 31) / 32 * 32;
  return 4 * (ra * (rb + 8) + rb * (ra + 8) + 2 * ra * (ra + 8));
}
// D tile of 16 x 16: rows m0 of one operand with rows n0 of another, both with their low planes so many entries behind.
__device__ __forceinline__ float4_t whole_product(const f16_t* left, int64_t left_low, int left_ld, const f16_t* right, int64_t right_low, int right_ld,
                                                  int m0, int n0, int inner, int l, int g) {
  float4_t acc[3] = {};       // (apart, so that the instructions of a step do not wait for each other)
  const f16_t *pl = left + (m0 + l) * left_ld + 8 * g, *pr = right + (n0 + l) * right_ld + 8 * g;
  for (int k = 0; k < inner; k += 32) {
    const half8 lh = *(const half8*)(pl + k), ll = *(const half8*)(pl + left_low + k);
    const half8 rh = *(const half8*)(pr + k), rl = *(const half8*)(pr + right_low + k);
    acc[0] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ll, rh, acc[0], 0, 0, 0);
    acc[1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(lh, rl, acc[1], 0, 0, 0);
    acc[2] = __builtin_amdgcn_mfma_f32_16x16x32_f16(lh, rh, acc[2], 0, 0, 0);
  }
  return (acc[0] + acc[1]) + acc[2];
}
typedef _Float16 half4 __attribute__((ext_vector_type(4)));
// Four entries that are next to one another.
__device__ __forceinline__ void whole_place(f16_t* to, int64_t low, const float4_t& x) {
  half4 high, less;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    high[r] = (f16_t)x[r];
    less[r] = (f16_t)(x[r] - (float)high[r]);
  }
  *(half4*)to = high;
  *(half4*)(to + low) = less;
}
__device__ __forceinline__ float4_t whole_entries(const f16_t* from, int64_t low) {
  const half4 high = *(const half4*)from, less = *(const half4*)(from + low);
  return float4_t{(float)high[0], (float)high[1], (float)high[2], (float)high[3]} + float4_t{(float)less[0], (float)less[1], (float)less[2], (float)less[3]};
}
__device__ __forceinline__ void whole_place(f16_t* to, int64_t low, float x) {
  f16_t high, less;
  split(x, high, less);
  to[0] = high;
  to[low] = less;
}

// Tile `at` of the lower triangle, row after row: its row and column.
__device__ __forceinline__ void triangle(uint32_t at, uint32_t& i, uint32_t& j) {
  i = (uint32_t)((sqrtf(8.0f * (float)at + 1.0f) - 1.0f) * 0.5f);
  while (i * (i + 1) / 2 > at) --i;
  while ((i + 1) * (i + 2) / 2 <= at) ++i;
  j = at - i * (i + 1) / 2;
}

template <class T, bool STEP>
__global__ __launch_bounds__(64 * kWholeWaves) void k_muon_whole(MuonArgs A, int iterations) {
  extern __shared__ __attribute__((aligned(16))) char whole_lds[];
  __shared__ double part[kWholeWaves];
  constexpr int kThreads = 64 * kWholeWaves;
  const MuonShape S = shape_of<&MuonShape::start_begin>(A, blockIdx.x);
  const int which = (int)(blockIdx.x - S.start_begin), worker = S.first + which;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, l = lane & 15, g = lane >> 4;
  const int ra = (S.a + 31) / 32 * 32, rb = (S.b + 31) / 32 * 32, a_ld = ra + 8, b_ld = rb + 8;
  f16_t* const x = (f16_t*)whole_lds;
  const int64_t x_low = (int64_t)ra * b_ld, xt_low = (int64_t)rb * a_ld, p_low = (int64_t)ra * a_ld;
  f16_t *const xt = x + 2 * x_low, *const p = xt + 2 * xt_low, *const q = p + 2 * p_low;
  const bool tall = S.rows > S.cols;
  const float scale = STEP && A.grad_scale ? A.grad_scale[worker] : 1.0f;
  if (STEP && !__builtin_isfinite(scale)) return;
  const int entries = S.rows * S.cols;
  float* const moment = A.moments + S.moment + (int64_t)worker * entries;
  // entry threadIdx.x and every kThreads-th from there, row and column counted on; all loads are under way together
  constexpr int kEach = 256 * kWholeTiles / 64;      // (as many as a wave's part of X has for a lane)
  const int step_rows = kThreads / S.cols, step_cols = kThreads % S.cols, r0 = (int)threadIdx.x / S.cols, c0 = (int)threadIdx.x % S.cols;
  const auto for_entries = [&](auto&& fn) {
    int r = r0, c = c0;
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      fn(k, (int)threadIdx.x + k * kThreads < entries, r, c);
      c += step_cols;
      r += step_rows;
      if (c >= S.cols) {
        c -= S.cols;
        ++r;
      }
    }
  };
  float u[kEach], before[kEach];
  for_entries([&](int k, bool there, int r, int c) {
    u[k] = there ? source_entry<T>(A, S, which, r, c) : 0.0f;
    if (STEP) before[k] = there ? moment[r * S.cols + c] : 0.0f;
  });
  for (int64_t e = threadIdx.x; e < (x_low + xt_low) / 4; e += kThreads) ((float4_t*)x)[e] = float4_t{};     // zeros behind the rows
  double sum = 0.0;
  for_entries([&](int k, bool there, int r, int c) {
    if (STEP) {
      const float grad = u[k] * scale, now = fmaf(A.momentum, before[k], grad);
      if (there) moment[r * S.cols + c] = now;
      u[k] = A.nesterov ? fmaf(A.momentum, now, grad) : now;
    }
    sum += (double)u[k] * (double)u[k];
  });
  for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
  if (lane == 0) part[wave] = sum;
  __syncthreads();
  sum = 0.0;
  for (int w = 0; w < kWholeWaves; ++w) sum += part[w];
  const double up = sum == 0.0 ? 0.0 : (double)kMuonUp / sqrt(sum);
  for_entries([&](int k, bool there, int r, int c) {
    if (!there) return;
    const int i = tall ? c : r, j = tall ? r : c;      // of the shorter side, of the longer
    const float value = (float)((double)u[k] * up);
    whole_place(x + i * b_ld + j, x_low, value);
    whole_place(xt + j * a_ld + i, xt_low, value);
  });
  __syncthreads();
  const int high = ra / 16, wide = rb / 16, triangles = high * (high + 1) / 2;
  for (int round = 0; round < iterations; ++round) {
    const bool last = round + 1 == iterations;
    // a tile of P or Q by its columns, which is its mirror image by rows, and by rows where the tile is not its own mirror image
    const auto mirrored = [&](f16_t* to, uint32_t i, uint32_t j, const float4_t& d) {
      const int m = 16 * i + 4 * g, n = 16 * j + l;
      whole_place(to + n * a_ld + m, p_low, d);
      if (i != j)
#pragma unroll
        for (int r = 0; r < 4; ++r) whole_place(to + (m + r) * a_ld + n, p_low, d[r]);
    };
    for (int t = wave; t < triangles; t += kWholeWaves) {
      uint32_t i, j;
      triangle(t, i, j);
      mirrored(p, i, j, whole_product(x, x_low, b_ld, x, x_low, b_ld, 16 * i, 16 * j, rb, l, g) * kMuonDown);
    }
    __syncthreads();
    for (int t = wave; t < triangles; t += kWholeWaves) {
      uint32_t i, j;
      triangle(t, i, j);
      const float4_t d = whole_product(p, p_low, a_ld, p, p_low, a_ld, 16 * i, 16 * j, ra, l, g);
      float4_t sum = d * (kMuonDown * kMuonC) + whole_entries(p + (16 * j + l) * a_ld + 16 * i + 4 * g, p_low) * kMuonB;
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (i == j && 4 * g + r == l) sum[r] += kMuonA * kMuonUp;
      mirrored(q, i, j, sum);
    }
    __syncthreads();
    float4_t made[kWholeTiles];
#pragma unroll
    for (int n = 0; n < kWholeTiles; ++n) {
      const int t = wave + n * kWholeWaves;
      if (t >= high * wide) continue;
      const int i = t % high, j = t / high;
      made[n] = whole_product(q, p_low, a_ld, xt, xt_low, a_ld, 16 * i, 16 * j, ra, l, g) * kMuonDown;
    }
    if (!last) __syncthreads();
#pragma unroll
    for (int n = 0; n < kWholeTiles; ++n) {
      const int t = wave + n * kWholeWaves;
      if (t >= high * wide) continue;
      const int i = t % high, j = t / high;
      if (!last) whole_place(xt + (16 * j + l) * a_ld + 16 * i + 4 * g, xt_low, made[n]);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int m = 16 * i + 4 * g + r, c = 16 * j + l;
        if (!last) {
          whole_place(x + m * b_ld + c, x_low, made[n][r]);
        } else if (m < S.a && c < S.b) {
          float* to = A.target + S.target + which * S.target_of + (int64_t)(tall ? c : m) * S.target_ld + (tall ? m : c);
          const float o = made[n][r] * kMuonDown;
          *to = STEP ? *to * (1.0f - A.lr * S.decay) - A.lr * S.rate * o : o;
        }
      }
    }
    __syncthreads();
  }
}

// ---- products ----
// One XCD's workgroups make neighbouring tiles, whose operands its L2 then holds.
__device__ __forceinline__ uint32_t by_xcd(uint32_t block, uint32_t blocks) {
  const uint32_t x = block & 7, each = blocks >> 3, more = blocks & 7;
  return x * each + min(x, more) + (block >> 3);
}
enum { kGram = 0, kSquare = 1, kApply = 2 };

// 16 bytes for each lane of a wave, straight into LDS, where the lanes' lie one behind the other.
__device__ __forceinline__ void to_lds(const void* from, void* to) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from, (__attribute__((address_space(3))) void*)to, 16, 0, 0);
}

// A workgroup makes a tile of TILE x TILE entries.  A step along the inner index takes 32 entries of TILE rows of both operands, high and
// low, into one of two buffers while the other one's are multiplied.  48 matrices of 2600 x 650: P 224 to 232 us, X' 570 to 617, 0.55 to 0.7 of the rate of a large
// product by the library on the tiles as they are (a wave reads 16 KB of LDS for 48 instructions: both are busy alike).  In a buffer a row's four 16-byte parts are exchanged by bits 2
// and 3 of its number, so that 16 lanes that read one part of 16 rows meet 16 different banks.
//   TILE 128: a wave makes a quarter of the tile, and loads one plane of the operands for all.
//   TILE 64, where the tiles are too few to fill the card: every wave makes the whole tile, of every fourth step, from buffers of its own,
// so that four steps are under way and nobody waits for anybody; the four sums are added up at the end.
template <int KIND, int TILE>
__global__ __launch_bounds__(256, TILE == 128 ? 2 : 1) void k_muon_product(MuonArgs A) {
  constexpr bool ALONE = TILE == 64;
  constexpr int W = 4;                                // 16-row parts of a wave's side
  constexpr int kLoads = TILE / 16 * (ALONE ? 4 : 1); // of a wave, a step
  __shared__ __attribute__((aligned(1024))) f16_t lds[2 * (ALONE ? 4 : 1)][4][TILE][32];    // left high, left low, right high, right low
  constexpr uint32_t MuonShape::*kBegin = KIND == kApply ? &MuonShape::apply_begin : &MuonShape::gram_begin;
  const uint32_t tile_at = by_xcd(blockIdx.x, gridDim.x);
  const MuonShape S = shape_of<kBegin>(A, tile_at);
  const uint32_t at = tile_at - S.*kBegin, tiles = KIND == kApply ? S.apply_tiles : S.gram_tiles, in = at % tiles;
  const int which = (int)(at / tiles);
  const MuonPlanes P = planes_of(A, S, which);
  uint32_t ti, tj;
  if (KIND == kApply) {
    const uint32_t high = (S.a + TILE - 1) / TILE;
    ti = in % high;
    tj = in / high;
  } else {
    triangle(in, ti, tj);
  }
  const f16_t *left = KIND == kGram ? P.x : KIND == kSquare ? P.p : P.q, *right = KIND == kApply ? P.xt[A.now] : left;
  const int64_t left_low = KIND == kGram ? P.x_low : P.p_low, right_low = KIND == kApply ? P.xt_low : left_low;
  const int64_t ld = KIND == kGram ? S.b_ld : S.a_ld;
  const int ms = S.a, ns = KIND == kApply ? S.b : S.a;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, l = lane & 15, g = lane >> 4;
  const int m0 = ti * TILE, n0 = tj * TILE, mw = ALONE ? 0 : (wave & 1) * (TILE / 2), nw = ALONE ? 0 : (wave >> 1) * (TILE / 2);

  // what a lane loads each step, 16 rows a load: of plane `wave`, or of all four
  const f16_t* source[kLoads];
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const int p = ALONE ? i / (TILE / 16) : wave, row = 16 * (i % (TILE / 16)) + (lane >> 2), part = (lane & 3) ^ ((row >> 2) & 3);
    const f16_t* from = (p < 2 ? left : right) + (p & 1) * (p < 2 ? left_low : right_low);
    source[i] = from + (int64_t)min((p < 2 ? m0 : n0) + row, (p < 2 ? ms : ns) - 1) * ld + 8 * part;
  }
  const int buffers = ALONE ? 2 * wave : 0;
  const auto load = [&](int64_t k, int buffer) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
      to_lds(source[i] + k, &lds[buffers + buffer][ALONE ? i / (TILE / 16) : wave][16 * (i % (TILE / 16))][0]);
  };
  const int swap = 8 * (g ^ ((l >> 2) & 3));
  constexpr int kStride = ALONE ? 128 : 32;
  float4_t acc[W][W] = {};
  int64_t k = ALONE ? 32 * wave : 0;
  if (k < ld) load(k, 0);
  // 16-row parts of the wave's sides that rows reach
  const int m_parts = max(0, min(W, (ms - m0 - mw + 15) / 16)), n_parts = max(0, min(W, (ns - n0 - nw + 15) / 16));
  const auto steps = [&](auto edges) {
    constexpr bool EDGES = decltype(edges)::value;
    for (int buffer = 0; k < ld; k += kStride, buffer ^= 1) {
      // this step's parts are there (for everybody), and (everybody is) done with the other buffer
      __builtin_amdgcn_s_waitcnt(0);
      if (ALONE) __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      else __syncthreads();
      half8 f[4][W];
#pragma unroll
      for (int p = 0; p < 4; ++p)
#pragma unroll
        for (int i = 0; i < W; ++i) f[p][i] = *(const half8*)&lds[buffers + buffer][p][(p < 2 ? mw : nw) + 16 * i + l][swap];
      if (k + kStride < ld) load(k + kStride, buffer ^ 1);
      if (m_parts == 0 || n_parts == 0) continue;
#pragma unroll
      for (int i = 0; i < W; ++i)
#pragma unroll
        for (int j = 0; j < W; ++j) {
          if (EDGES && (i >= m_parts || j >= n_parts)) continue;
          acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f[1][i], f[2][j], acc[i][j], 0, 0, 0);
          acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f[0][i], f[3][j], acc[i][j], 0, 0, 0);
          acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f[0][i], f[2][j], acc[i][j], 0, 0, 0);
        }
    }
  };
  if (ms - m0 >= TILE && ns - n0 >= TILE) steps(std::false_type{});
  else steps(std::true_type{});
  // The tile in LDS, fp32, columns exchanged by the rows' number so that reading down a column meets all banks, then out of it by
  // rows and by columns, 8 entries a lane.
  __syncthreads();
  float* const tile = (float*)&lds[0][0][0][0];
  static_assert(sizeof(lds) >= (ALONE ? 4 : 1) * TILE * TILE * sizeof(float));
  const auto place = [](int m, int n) { return m * TILE + (n ^ ((m >> 1) & (TILE / 2 - 4))); };
  constexpr float kScale = KIND == kSquare ? kMuonDown * kMuonC : kMuonDown;
#pragma unroll
  for (int i = 0; i < W; ++i)
#pragma unroll
    for (int j = 0; j < W; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) tile[(ALONE ? wave * TILE * TILE : 0) + place(mw + 16 * i + 4 * g + r, nw + 16 * j + l)] = acc[i][j][r] * kScale;
  __syncthreads();
  if (ALONE) {
    for (int e = threadIdx.x * 4; e < TILE * TILE; e += 1024) {
      float4_t* const sum = (float4_t*)(tile + e);
      *sum = (*sum + sum[TILE * TILE / 4]) + (sum[2 * (TILE * TILE / 4)] + sum[3 * (TILE * TILE / 4)]);
    }
    __syncthreads();
  }
  constexpr int kParts = TILE / 8;
  constexpr bool kAdds = KIND == kSquare;     // a I + b P
  const bool last = KIND == kApply && A.last;
  f16_t* const made = KIND == kApply ? P.x : KIND == kGram ? P.p : P.q;
  f16_t* const turned = KIND == kApply ? P.xt[A.now ^ 1] : made;
  const int64_t low = KIND == kApply ? P.x_low : P.p_low, turned_low = KIND == kApply ? P.xt_low : P.p_low;
  const int n_ld = KIND == kApply ? S.b_ld : S.a_ld;
  const int worker = S.first + which;
  const bool tall = S.rows > S.cols;
  const bool skip = last && A.moments && A.grad_scale && !__builtin_isfinite(A.grad_scale[worker]);
  const auto finish = [&](int m, int n, const float (&x)[8], int count) {      // `count` entries of a row of memory
    float* to = A.target + S.target + which * S.target_of + (int64_t)(tall ? n : m) * S.target_ld + (tall ? m : n);
    if (skip) return;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < count) {
        const float o = x[e] * kMuonDown;
        to[e] = A.moments ? to[e] * (1.0f - A.lr * S.decay) - A.lr * S.rate * o : o;
      }
  };
  if (!(last && tall))
  for (int u = threadIdx.x; u < TILE * kParts; u += 256) {
    const int i = u / kParts, j = u % kParts * 8, m = m0 + i, n = n0 + j;
    if (m >= ms || n >= n_ld) continue;
    float x[8];
    *(float4_t*)&x[0] = *(const float4_t*)&tile[place(i, j)];
    *(float4_t*)&x[4] = *(const float4_t*)&tile[place(i, j + 4)];
    if (KIND != kApply && ti == tj) {     // the lower triangle's mirror image here too: P and Q are symmetric to the bit
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (j + e > i) x[e] = tile[place(j + e, i)];
    }
    const int64_t at_row = (int64_t)m * n_ld + n;
    if (kAdds) {
      const half8 high = *(const half8*)(P.p + at_row), less = *(const half8*)(P.p + at_row + low);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] += kMuonB * ((float)high[e] + (float)less[e]) + (m == n + e ? kMuonA * kMuonUp : 0.0f);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (n + e >= ns) x[e] = 0.0f;
    if (last) {
      finish(m, n, x, ns - n);
      continue;
    }
    if (kAdds && ti != tj) {
      *(float4_t*)&tile[place(i, j)] = *(const float4_t*)&x[0];
      *(float4_t*)&tile[place(i, j + 4)] = *(const float4_t*)&x[4];
    }
    half8 high, less;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      high[e] = (f16_t)x[e];
      less[e] = (f16_t)(x[e] - (float)high[e]);
    }
    *(half8*)(made + at_row) = high;
    *(half8*)(made + at_row + low) = less;
  }
  if (KIND == kApply ? last && !tall : ti == tj) return;
  __syncthreads();
  for (int u = threadIdx.x; u < TILE * kParts; u += 256) {
    const int j = u / kParts, i = u % kParts * 8, m = m0 + i, n = n0 + j;
    if (n >= ns || m >= S.a_ld) continue;
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = m + e < ms ? tile[place(i + e, j)] : 0.0f;
    if (last) {
      finish(m, n, x, ms - m);
      continue;
    }
    half8 high, less;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      high[e] = (f16_t)x[e];
      less[e] = (f16_t)(x[e] - (float)high[e]);
    }
    f16_t* to = turned + (int64_t)n * S.a_ld + m;
    *(half8*)to = high;
    *(half8*)(to + turned_low) = less;
  }
}

}  // namespace choco
