// Linear attention with a decay for each head, S_t = e^g_t S_{t-1} + k_t v_t^T, y_t = S_t^T q_t, and its backward pass (device code).
//
// Every part of the work is one of four passes of one kind: for a sequence and head, through its steps forwards or backwards,
//   S <- w S + b c^T,   out = S^T a
//   y:  a, b, c = q, k, v              dq: dy, v, k     (the same states transposed)
//   dk: v, dy, q   backwards           dv: k, q, dy     backwards
// where w = e^g_t forwards, and backwards the next step's, 1 at a sequence's last.
//
// Measured, us a call (what it has to read and write at the rate of a large copy, 5.1 TB/s), three sets of inputs in turn: one token of 64 x 16 heads of
// 128 in bf16 28 (26), of 160 x 13 of 50 in fp32 12 (8); 160 x 35 x 13 x 50 in fp32 62 (17), backward 229 (25); 2 x 32,768 x 16 x 128 in bf16, lengths
// from a half on, 489 (172); 8 x 2000 x 20 x 64 in fp16, q and k shared by four, 95 (21); backward of 4 x 16,384 x 10 x 128 in bf16 1,200 (230).
// Before: step by step all of it, 69,800 and 131,900 for the long ones; chunks without loads ahead 1,320 and 2,840; every wave its own P, 780
// and 2,120; loads with branches, 710 and 2,030; four waves and 64 columns a workgroup 640 and 1,610; gates' gradients by differences of sums, which
// lose their places where a gate is nearly closed, 1,090 backward.
#pragma once

#include <type_traits>

#include "choco_types.h"

namespace choco {

constexpr int kLinearSave = 256;    // the forward pass keeps the state before every so many steps
constexpr int kLinearSlice = 64;    // columns of a pass' result that a workgroup takes
constexpr float kLinearLeast = -200.0f;     // a logarithm below counts as -infinity

struct LinearPass {
  const void *a, *b, *c;
  const void* x;            // multiplied with the result's rows to `dots`, or null
  void* out;
  int64_t a_seq, a_step, a_head, b_seq, b_step, b_head, c_seq, c_step, c_head, x_seq, x_step, x_head, out_seq, out_step, out_head;
  int32_t a_share, b_share, c_share, x_share;     // heads of the attention to one of these
  int32_t da, dc;           // entries of a and b; of c and out
  int32_t state_a, state_c; // strides of a state's entries in memory; a state has da * dc
  const float* first;       // state before a sequence's first step of the pass, or null: zero; `first_of` states from one head to the next
  float* last;              // state after its last step, backwards decayed by the first step's w: of S_0
  float* kept;              // forwards: states before every kLinearSave-th step and the last one, `kept_of` of each sequence and head
  int64_t kept_of, first_of;
  // What a pass in chunks adds to the gates' gradient, or null:
  float* dots;              // [slices][batch * heads][steps]
  const float* met;         // dq: states that the backwards passes have before their pieces; dk: what the forward pass kept
  const float* met_last;    // dq: the gradient of the last states, or null
  int64_t met_of;           // states of `met` from one head to the next
  bool back, wide;          // wide: out is fp32 whatever the inputs' type
};

struct LinearArgs {
  const float* g;
  const int32_t* lengths;
  int64_t batch, steps, g_seq, g_step, g_head;
  int32_t heads;
};

__device__ __forceinline__ int64_t steps_of(const LinearArgs& A, int64_t b) {
  if (!A.lengths) return A.steps;
  const int64_t n = A.lengths[b];
  return n < 0 ? 0 : n > A.steps ? A.steps : n;
}
// g of a step, by the caller inside its sequence.
__device__ __forceinline__ float log_gate(const LinearArgs& A, int64_t b, int64_t t, int h) {
  return A.g[b * A.g_seq + t * A.g_step + h * A.g_head];
}
__device__ __forceinline__ float linear_decay(float g) { return g < kLinearLeast ? 0.0f : expf(g); }

template <class T>
__device__ __forceinline__ void store_result(const LinearPass& P, int64_t at, float x) {
  if (P.wide) ((float*)P.out)[at] = x;
  else ((T*)P.out)[at] = from_float<T>(x);
}

// ---- step by step ----
// A workgroup takes a slice of columns and holds the state in registers, V columns of every 4 V-th row a lane (V as the state's rows divide;
// one that lies on no border of V is read and written by entries, with the same sums).  Bound by the state, in and out once: for a step of D x D,
// 8 D^2 bytes against 5 D^2 operations.  One token of 64 x 16 heads of 128 in bf16 28 us, 4.8 TB/s (25 and 5.4 where its 135 MB stay in the last-level
// cache; a column a lane, a quarter of the rows a wave: 33), of 160 x 13 of 50 in fp32 12 us, 3.6 TB/s (20).
constexpr int kLinearStage = 8;     // steps whose a and b are in LDS at a time

template <class T, int V, int D>
__global__ __launch_bounds__(256) void k_linear_steps(LinearArgs A, LinearPass P) {
  constexpr int kLanes = kLinearSlice / V, kRows = 256 / kLanes, R = D / kRows;
  __shared__ float sa[kLinearStage][D], sb[kLinearStage][D];
  __shared__ __attribute__((aligned(16))) float part[2][kRows][kLinearSlice];
  const int row = threadIdx.x / kLanes, at = threadIdx.x % kLanes * V;
  const int slices = (P.dc + kLinearSlice - 1) / kLinearSlice, slice = blockIdx.x % slices;
  const int64_t bh = blockIdx.x / slices, b = bh / A.heads;
  const int h = (int)(bh % A.heads), col = slice * kLinearSlice + at;
  const bool in = col < P.dc;      // (V divides the columns)
  const int64_t len = steps_of(A, b), state = (int64_t)P.da * P.dc;
  const T* pa = (const T*)P.a + b * P.a_seq + (h / P.a_share) * P.a_head;
  const T* pb = (const T*)P.b + b * P.b_seq + (h / P.b_share) * P.b_head;
  const T* pc = (const T*)P.c + b * P.c_seq + (h / P.c_share) * P.c_head + col;
  const int64_t out = b * P.out_seq + h * P.out_head + slice * kLinearSlice;
  float s[R][V];
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int v = 0; v < V; ++v) s[r][v] = 0.0f;
  const auto on_border = [](const float* p) { return V == 1 || ((uintptr_t)p & (4 * V - 1)) == 0; };
  if (P.first) {
    const float* p = P.first + bh * P.first_of * state + (int64_t)row * P.state_a + (int64_t)col * P.state_c;
    if (on_border(P.first)) {
#pragma unroll
      for (int r = 0; r < R; ++r)
        if (in && row + r * kRows < P.da) load_floats<float, V>(p + (int64_t)r * kRows * P.state_a, s[r]);
    } else {
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int v = 0; v < V; ++v)
          if (in && row + r * kRows < P.da) s[r][v] = p[(int64_t)r * kRows * P.state_a + v];
    }
  }
  const auto keep = [&](float* to, float w) {
    float* p = to + (int64_t)row * P.state_a + (int64_t)col * P.state_c;
    if (on_border(to)) {
#pragma unroll
      for (int r = 0; r < R; ++r) {
        float x[V];
#pragma unroll
        for (int v = 0; v < V; ++v) x[v] = s[r][v] * w;
        if (in && row + r * kRows < P.da) store_floats<float, V>(p + (int64_t)r * kRows * P.state_a, x);
      }
    } else {
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int v = 0; v < V; ++v)
          if (in && row + r * kRows < P.da) p[(int64_t)r * kRows * P.state_a + v] = s[r][v] * w;
    }
  };
  for (int64_t i0 = 0; i0 < len; i0 += kLinearStage) {
    const int n = len - i0 < kLinearStage ? (int)(len - i0) : kLinearStage;
    __syncthreads();
    for (int e = threadIdx.x; e < n * D; e += 256) {
      const int i = e / D, j = e % D;
      const int64_t t = P.back ? len - 1 - (i0 + i) : i0 + i;
      sa[i][j] = j < P.da ? to_float(pa[t * P.a_step + j]) : 0.0f;
      sb[i][j] = j < P.da ? to_float(pb[t * P.b_step + j]) : 0.0f;
    }
    __syncthreads();
    for (int i = 0; i < n; ++i) {
      const int64_t t = P.back ? len - 1 - (i0 + i) : i0 + i;
      if (P.kept && t % kLinearSave == 0) keep(P.kept + (bh * P.kept_of + t / kLinearSave) * state, 1.0f);
      float w = 1.0f;
      if (!P.back) w = linear_decay(log_gate(A, b, t, h));
      else if (t + 1 < len) w = linear_decay(log_gate(A, b, t + 1, h));
      float c[V], sum[V];
#pragma unroll
      for (int v = 0; v < V; ++v) {
        c[v] = in ? to_float(pc[t * P.c_step + v]) : 0.0f;
        sum[v] = 0.0f;
      }
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int v = 0; v < V; ++v) {
          s[r][v] = fmaf(sb[i][row + r * kRows], c[v], s[r][v] * w);
          sum[v] = fmaf(sa[i][row + r * kRows], s[r][v], sum[v]);
        }
      store_floats<float, V>(&part[i & 1][row][at], sum);
      __syncthreads();
      if (threadIdx.x < kLinearSlice) {
        const int mine = slice * kLinearSlice + (int)threadIdx.x;
        float y = 0.0f;
#pragma unroll
        for (int r = 0; r < kRows; ++r) y += part[i & 1][r][threadIdx.x];
        if (mine < P.dc) store_result<T>(P, out + t * P.out_step + threadIdx.x, y);
      }
    }
  }
  const int width = min(P.dc - slice * kLinearSlice, kLinearSlice);
  for (int64_t e = threadIdx.x; e < (A.steps - len) * width; e += 256) store_result<T>(P, out + (len + e / width) * P.out_step + e % width, 0.0f);
  if (P.kept) keep(P.kept + (bh * P.kept_of + (len + kLinearSave - 1) / kLinearSave) * state, 1.0f);
  if (P.last) keep(P.last + bh * state, P.back && len > 0 ? linear_decay(log_gate(A, b, 0, h)) : 1.0f);
}

// ---- in chunks ----
// With c_t the sum of the logarithms of w since the chunk began and S the state before it,
//   out_t = e^c_t S^T a_t + sum over s <= t of e^(c_t - c_s) (a_t b_s) c_s,   S <- e^c_end S + sum of e^(c_end - c_s) b_s c_s^T:
// four products of matrices, on the matrix cores, out^T = S^T a^T + c^T P^T with P^T = (b a^T) weighted.  A wave takes 16 columns of the result
// and holds the state's in registers as the matrix cores leave a product: a lane has a column's rows 4 g to 4 g + 3 of every 16.
// That is how the cores take a left operand whose inner index is the row, so S does not go through LDS; P^T does, a wave makes
// a quarter of it.  Differences of c are taken of c in two floats: a start-over leaves the steps behind it exact.
//
// Entries of 32 bits go to the fp32 matrix instruction.  Those of 16 bits are operands as they are; what is fp32 by nature (P, S, weighted c)
// enters as a sum of numbers of that type.  bf16: three of them (2^-25) for states, and for dq and dk, whose products with what comes of states go into the
// gates' gradient in fp32; two (2^-17) for y and dv, which are rounded to 16 bits next (dv of shared heads after their sum).  Which does not depend on
// what is asked for.  fp16: two (2^-22), after a power of two has brought the largest of a state's column, or of a step's P, to the top of fp16's range.
//
// What bounds it: of a chunk of 64 x 128 x 128 in bf16 a SIMD's four waves take some 10,000 cycles of vector instructions (half of them split
// fp32 numbers), 7,000 of matrix instructions, and LDS 5,000; memory 5,000 at the rate of a copy.  They overlap by half: 363 us for the
// results of 2 x 32,768 x 16 x 128, 2.5 TB/s.  A workgroup has eight waves in 128 registers, two of them a compute unit: with one of them
// (256 registers) 488 us, with four waves and 64 columns 527.
constexpr int kChunk = 64;
constexpr float kLog2Least = -300.0f;     // stands for -infinity: less than any difference that counts

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

template <int CONTROL>
__device__ __forceinline__ float moved_in_row(float x) {      // of 16 lanes; zero from beyond
  return __uint_as_float(__builtin_amdgcn_update_dpp(0u, __float_as_uint(x), CONTROL, 15, 15, false));
}
// Of 16 neighbouring lanes: sums from each on; the sum of all, everywhere.
__device__ __forceinline__ float row_sums_from(float x) {
  x += moved_in_row<0x101>(x);
  x += moved_in_row<0x102>(x);
  x += moved_in_row<0x104>(x);
  return x + moved_in_row<0x108>(x);
}
__device__ __forceinline__ float row_sum(float x) {
  x += moved_in_row<0x128>(x);
  x += moved_in_row<0x124>(x);
  x += moved_in_row<0x122>(x);
  return x + moved_in_row<0x121>(x);
}

// The four rows of 16 lanes added up, in all of them; of numbers that are a row's own, the sum of the rows before.
__device__ __forceinline__ float rows_summed(float x) {
  const auto two = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(two[0]) + __uint_as_float(two[1]);
  const auto four = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(four[0]) + __uint_as_float(four[1]);
}
template <int CONTROL, int ROWS>
__device__ __forceinline__ float last_lane_of(float x) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0u, __float_as_uint(x), CONTROL, ROWS, 15, false));
}
__device__ __forceinline__ float rows_before(float x) {
  x = last_lane_of<0x142, 14>(x);      // each row's, one row on; then the first's to the second's, the third's to the fourth's, the first half's
  x += last_lane_of<0x142, 10>(x);
  return x + last_lane_of<0x143, 12>(x);
}
// Sums over the lanes from each on, without its own where `own` is false.
__device__ __forceinline__ float sums_from(float x, bool own, int row) {
  x = row_sums_from(x);
  float behind = 0.0f;
#pragma unroll
  for (int k = 3; k > 0; --k) {
    const float sum = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), 16 * k));
    behind += row < k ? sum : 0.0f;
  }
  return behind + (own ? x : moved_in_row<0x101>(x));
}

template <class Core>
struct Operand;
template <>
struct Operand<float> {
  typedef f32x4 Frag;
  static constexpr int kInner = 16, kTiles = 1;     // entries of the inner index; tiles of a product that make an operand
  static __device__ __forceinline__ Frag load(const float* row, int j, int g) { return *(const f32x4*)(row + 16 * j + 4 * g); }
  static __device__ __forceinline__ f32x4 mma(Frag a, Frag b, f32x4 c) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
    return c;
  }
};
template <>
struct Operand<bf16_t> {
  typedef bf16x8 Frag;
  static constexpr int kInner = 32, kTiles = 2;
  static __device__ __forceinline__ Frag load(const bf16_t* row, int j, int g) {
    const bf16x4 lo = *(const bf16x4*)(row + 32 * j + 4 * g), hi = *(const bf16x4*)(row + 32 * j + 16 + 4 * g);
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  }
  static __device__ __forceinline__ f32x4 mma(Frag a, Frag b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <>
struct Operand<f16_t> {
  typedef f16x8 Frag;
  static constexpr int kInner = 32, kTiles = 2;
  static __device__ __forceinline__ Frag load(const f16_t* row, int j, int g) {
    const f16x4 lo = *(const f16x4*)(row + 32 * j + 4 * g), hi = *(const f16x4*)(row + 32 * j + 16 + 4 * g);
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  }
  static __device__ __forceinline__ f32x4 mma(Frag a, Frag b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};
// A power of two that brings numbers, the largest of them `most`, to the top of fp16's range, and back: below 2^15, so that what is 2^-39 of the
// largest still counts.
struct Range {
  float up, down;
  __device__ __forceinline__ explicit Range(float most) {
    const uint32_t e = max(__float_as_uint(most) >> 23, 15u);      // (not negative, not infinite)
    up = __uint_as_float((268u - e) << 23);
    down = __uint_as_float((e - 14u) << 23);
  }
};
// The largest magnitude of a column's numbers, which are in a lane of each row of 16 and which `each` hands out; where one is infinite, of the others,
// which then keep their places.
template <class Each>
__device__ __forceinline__ float largest_of_column(Each each) {
  constexpr float kInfinite = __builtin_inff();
  float most = 0.0f;
  each([&](float x) { most = fmaxf(most, fabsf(x)); });
  if (__any(most == kInfinite)) {
    most = 0.0f;
    each([&](float x) { most = fmaxf(most, fabsf(x) < kInfinite ? fabsf(x) : 0.0f); });
  }
  const auto two = __builtin_amdgcn_permlane16_swap(__float_as_uint(most), __float_as_uint(most), false, false);
  most = fmaxf(__uint_as_float(two[0]), __uint_as_float(two[1]));
  const auto four = __builtin_amdgcn_permlane32_swap(__float_as_uint(most), __float_as_uint(most), false, false);
  return fmaxf(__uint_as_float(four[0]), __uint_as_float(four[1]));
}
// fp32 numbers of an operand as so many operands that add up to it.
template <class Core, int N>
__device__ __forceinline__ void pieces_of(const f32x4 (&x)[Operand<Core>::kTiles], typename Operand<Core>::Frag (&p)[N]) {
  if constexpr (std::is_same_v<Core, float>) {
    static_assert(N == 1);
    p[0] = x[0];
  } else {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    typedef Core Two __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      f32x2 left = {x[e / 4][e % 4], x[e / 4][e % 4 + 1]};
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const Two two = __builtin_convertvector(left, Two);
        p[i][e] = two.x;
        p[i][e + 1] = two.y;
        const uint32_t word = __builtin_bit_cast(uint32_t, two);
        if (i + 1 < N) left = f32x2{left.x - entry<Core>(word, 0), left.y - entry<Core>(word, 1)};
      }
    }
  }
}

// How a launch goes through the chunks.
struct LinearChunks {
  float* states;        // before each segment, `states_of` of da * dc for each sequence and head; null: one segment, from P.first
  int64_t states_of;
  double* totals;       // STATE: sums of the segments' logarithms (base 2), [batch * heads][segments]
  int32_t segments, chunks;      // a segment has so many chunks
  int32_t slices;
  uint32_t blocks;
  int32_t way;          // how rows are read
  int32_t vec_out, vec_x;   // entries that a store, or a load of x, takes
};

// Workgroups go to the eight XCDs in turn: segments of a head one after the other, so that those a sequence does not reach are spread over all
// of them, and slices of one segment eight apart, so that they share their a and b in an L2.  (2 x 32,768 x 16 x 128 in bf16 541 us;
// neighbours on one XCD 540, but with lengths from a half on 496 | 494; heads one after the other 562 | 511.)
struct ChunkPlace {
  int64_t bh;
  int segment, slice;
  bool there;
};
__device__ __forceinline__ ChunkPlace chunk_place(const LinearArgs& A, const LinearChunks& C) {
  const uint32_t rows = (uint32_t)(A.batch * A.heads), each = 8 * C.slices, in = blockIdx.x % each;
  const uint32_t unit = blockIdx.x / each * 8 + (in & 7);
  return {unit / C.segments, (int)(unit % C.segments), (int)(in >> 3), unit < rows * (uint32_t)C.segments};
}

template <class Core, int DA, int WAVES>
struct ChunkShared {
  static constexpr int kPad = 16 / sizeof(Core), kSlice = 16 * WAVES;
  static constexpr bool kTurned = sizeof(Core) == 2;      // b by columns as well
  static constexpr int kTurnedRow = kChunk + 4, kScoreRow = kChunk + 4;
  // (P, in 16 bits three pieces of it, or two and x, lies over a, in 16 bits also over b, and what is missing)
  static constexpr int kTwo = 2 * kChunk * kScoreRow, kScores = kTwo + kChunk * (kScoreRow > kSlice + kPad ? kScoreRow : kSlice + kPad), kRows = 2 * kChunk * (DA + kPad);
  Core a[kChunk][DA + kPad], b[kChunk][DA + kPad];
  Core more[kTurned && kScores > kRows ? kScores - kRows : 1];
  alignas(16) Core c[kChunk][kSlice + kPad];
  alignas(16) Core turned[kTurned ? DA : 1][kTurned ? kTurnedRow : 1];
  alignas(16) float c_high[kChunk], c_low[kChunk], to_end[kChunk];
  // for the gates' gradient, by one pass or the other (so that three workgroups of 64 x 64 in fp32 fit a compute unit)
  union {
    struct {
      float dots[WAVES][kChunk], met[WAVES], ahead[WAVES], weights[kChunk], ahead_all;
    };
    struct {
      alignas(16) float behind[10][16], before[10][16];      // sums over pairs of steps, of ten tiles
    };
  };
  uint32_t most[std::is_same_v<Core, f16_t> ? kChunk : 1];
};

// How rows are read: parts of 16 bytes or words of 4 by offsets of 32 bits, where what is not there has one outside the buffer and comes
// back as zero, without a branch; or entry by entry by 64-bit addresses, for rows that are on no word's border or far apart.
enum { kEntries = 0, kWords = 4, kParts = 16 };
constexpr uint32_t kBufferBytes = 0x80000000u;

typedef uint32_t word2 __attribute__((ext_vector_type(2)));
typedef uint32_t word4 __attribute__((ext_vector_type(4)));

// Four entries of a row, of which those from `width` on are not there: `at` is their byte in the buffer, ~0 for none at all.
template <class T>
struct Four {
  uint32_t x[sizeof(T)];
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t buffer, uint32_t at, int width, bool whole) {
    if (whole) {
      const uint32_t from = width >= 4 ? at : ~0u;
      if constexpr (sizeof(T) == 4) {
        const word4 v = __builtin_amdgcn_raw_buffer_load_b128(buffer, from, 0, 0);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = v[i];
      } else {
        const word2 v = __builtin_amdgcn_raw_buffer_load_b64(buffer, from, 0, 0);
        x[0] = v.x;
        x[1] = v.y;
      }
      return;
    }
    const auto from = [&](int i) { return i < width && at != ~0u ? at + i * (uint32_t)sizeof(T) : ~0u; };
#pragma unroll
    for (int i = 0; i < (int)sizeof(T); ++i) {
      if constexpr (sizeof(T) == 4) x[i] = __builtin_amdgcn_raw_buffer_load_b32(buffer, from(i), 0, 0);
      else
        x[i] = __builtin_amdgcn_raw_buffer_load_b16(buffer, from(2 * i), 0, 0) |
               (uint32_t)__builtin_amdgcn_raw_buffer_load_b16(buffer, from(2 * i + 1), 0, 0) << 16;
    }
  }
  __device__ __forceinline__ void load(const T* p, int width) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T); ++i) {
      if constexpr (sizeof(T) == 4) x[i] = i < width ? *reinterpret_cast<const uint32_t*>(p + i) : 0u;
      else {
        const uint16_t* half = reinterpret_cast<const uint16_t*>(p);
        x[i] = (2 * i < width ? half[2 * i] : 0u) | (2 * i + 1 < width ? (uint32_t)half[2 * i + 1] << 16 : 0u);
      }
    }
  }
  __device__ __forceinline__ float operator[](int i) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(x[i]);
    else return entry<T>(x[i / 2], i & 1);
  }
};
template <class T>
__device__ __forceinline__ void store_four(__amdgpu_buffer_rsrc_t buffer, uint32_t at, int width, bool whole, const f32x4& x) {
  Pack<T, 4> v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v.e[i] = from_float<T>(x[i]);
  if (whole) {
    const uint32_t to = width >= 4 ? at : ~0u;
    if constexpr (sizeof(T) == 4) __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(word4, v), buffer, to, 0, 0);
    else __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(word2, v), buffer, to, 0, 0);
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t to = i < width && at != ~0u ? at + i * (uint32_t)sizeof(T) : ~0u;
    if constexpr (sizeof(T) == 4) __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, v.e[i]), buffer, to, 0, 0);
    else __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(uint16_t, v.e[i]), buffer, to, 0, 0);
  }
}

// A chunk's rows of one array on their way from memory to LDS, in the registers of WAVES waves: they are asked for while the chunk
// before is worked on.  A thread takes R rows of V entries at a time: one of eight, or, for rows that are also laid out by
// columns, four of four, 16 neighbouring lanes 4 x 4 of these, which meets all banks both ways.
template <class In, int W, int R, int WAVES, int WAY>
struct Staged {
  static constexpr int V = R == 1 ? 8 : 4;
  static constexpr int kWordsOf = V * sizeof(In) / 4;      // of V entries
  static constexpr int kThreads = 64 * WAVES, kAll = kChunk / R * (W / V), kUnits = (kAll + kThreads - 1) / kThreads;
  // words of rows of their own: neighbouring lanes' are next to one another, a thread's in rows apart
  static constexpr bool kByWords = WAY == kWords && R == 1;
  static constexpr int kRowWords = W * sizeof(In) / 4, kEach = 4 / sizeof(In);      // entries of a word
  static_assert(!kByWords || (kThreads % kRowWords == 0 && kUnits * kWordsOf * (kThreads / kRowWords) == kChunk));
  uint32_t x[kUnits][R][kWordsOf];

  static __device__ __forceinline__ void place(int i, int thread, int& row, int& col) {
    const int u = i * kThreads + thread;
    if constexpr (R == 1) {
      row = u / (W / V);
      col = u % (W / V) * V;
    } else {
      static_assert(kChunk / R == 16);
      row = ((u & 3) | (u >> 2 & 12)) * R;
      col = ((u >> 2 & 3) | (u >> 6) * 4) * V;
    }
  }
  static __device__ __forceinline__ bool mine(int row, int col) { return kAll % kThreads == 0 || (row < kChunk && col < W); }
  // Rows of the chunk from `lo` to `hi`, `width` entries each; `first` is the row of the chunk's earliest step, which backwards is the
  // last row.
  __device__ __forceinline__ void load(int thread, const In* first, int64_t step, bool back, int width, int lo, int hi) {
    const __amdgpu_buffer_rsrc_t buffer = __builtin_amdgcn_make_buffer_rsrc((void*)first, 0, kBufferBytes, 0x00027000);
    if constexpr (kByWords) {
      const int col = thread % kRowWords * kEach;
      const bool in = col < width;
#pragma unroll
      for (int i = 0; i < kUnits * kWordsOf; ++i) {
        const int row = thread / kRowWords + i * (kThreads / kRowWords), t = back ? kChunk - 1 - row : row;
        const uint32_t at = ((uint32_t)t * (uint32_t)step + (uint32_t)col) * (uint32_t)sizeof(In);
        x[i / kWordsOf][0][i % kWordsOf] = __builtin_amdgcn_raw_buffer_load_b32(buffer, in && row >= lo && row < hi ? at : ~0u, 0, 0);
      }
      return;
    }
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
      int row, col;
      place(i, thread, row, col);
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const bool there = row + r >= lo && row + r < hi && mine(row, col);
        const int t = back ? kChunk - 1 - row - r : row + r;
        const uint32_t at = ((uint32_t)t * (uint32_t)step + (uint32_t)col) * (uint32_t)sizeof(In);
        if constexpr (WAY == kParts) {
          if constexpr (kWordsOf == 2) {
            const word2 v = __builtin_amdgcn_raw_buffer_load_b64(buffer, there && col < width ? at : ~0u, 0, 0);
            x[i][r][0] = v.x;
            x[i][r][1] = v.y;
          } else {
#pragma unroll
            for (int w = 0; w < kWordsOf; w += 4) {
              const word4 v = __builtin_amdgcn_raw_buffer_load_b128(buffer, there && col + w * kEach < width ? at + 4 * w : ~0u, 0, 0);
#pragma unroll
              for (int e = 0; e < 4; ++e) x[i][r][w + e] = v[e];
            }
          }
        } else if constexpr (WAY == kWords) {
#pragma unroll
          for (int w = 0; w < kWordsOf; ++w)
            x[i][r][w] = __builtin_amdgcn_raw_buffer_load_b32(buffer, there && col + w * kEach < width ? at + 4 * w : ~0u, 0, 0);
        } else {
          const In* p = first + t * step + col;
#pragma unroll
          for (int w = 0; w < kWordsOf; ++w) {
            x[i][r][w] = 0;
            if constexpr (sizeof(In) == 4) {
              if (there && col + w < width) x[i][r][w] = *reinterpret_cast<const uint32_t*>(p + w);
            } else {
              const uint16_t* half = reinterpret_cast<const uint16_t*>(p);
              if (there && col + 2 * w < width) x[i][r][w] = half[2 * w];
              if (there && col + 2 * w + 1 < width) x[i][r][w] |= (uint32_t)half[2 * w + 1] << 16;
            }
          }
        }
      }
    }
  }
  template <int STRIDE>
  __device__ __forceinline__ void store(int thread, In (&to)[kChunk][STRIDE]) const {
    if constexpr (kByWords) {
#pragma unroll
      for (int i = 0; i < kUnits * kWordsOf; ++i) {
        In* p = &to[thread / kRowWords + i * (kThreads / kRowWords)][thread % kRowWords * kEach];
        *reinterpret_cast<uint32_t*>(p) = x[i / kWordsOf][0][i % kWordsOf];
      }
      return;
    }
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
      int row, col;
      place(i, thread, row, col);
      if (!mine(row, col)) continue;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        if constexpr (kWordsOf == 2) {
          *reinterpret_cast<uint2*>(&to[row + r][col]) = uint2{x[i][r][0], x[i][r][1]};
        } else {
#pragma unroll
          for (int w = 0; w < kWordsOf; w += 4)
            *reinterpret_cast<uint4*>(&to[row + r][col + w * kEach]) = uint4{x[i][r][w], x[i][r][w + 1], x[i][r][w + 2], x[i][r][w + 3]};
        }
      }
    }
  }
  // ... by columns: four steps of an entry are 8 bytes
  template <int STRIDE>
  __device__ __forceinline__ void store_turned(int thread, In (*to)[STRIDE]) const {
    static_assert(R == 4 && sizeof(In) == 2);
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
      int row, col;
      place(i, thread, row, col);
      if (!mine(row, col)) continue;
#pragma unroll
      for (int e = 0; e < V; e += 2) {
        const uint32_t w0 = x[i][0][e / 2], w1 = x[i][1][e / 2], w2 = x[i][2][e / 2], w3 = x[i][3][e / 2];
        *reinterpret_cast<uint2*>(&to[col + e][row]) = uint2{__builtin_amdgcn_perm(w1, w0, 0x05040100u), __builtin_amdgcn_perm(w3, w2, 0x05040100u)};
        *reinterpret_cast<uint2*>(&to[col + e + 1][row]) = uint2{__builtin_amdgcn_perm(w1, w0, 0x07060302u), __builtin_amdgcn_perm(w3, w2, 0x07060302u)};
      }
    }
  }
};

// Sums over the lanes up to each.
template <int CONTROL, int ROWS>
__device__ __forceinline__ double moved(double x) {
  const uint64_t bits = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0u, (uint32_t)bits, CONTROL, ROWS, 15, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0u, (uint32_t)(bits >> 32), CONTROL, ROWS, 15, false);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double sums_to(double x) {
  x += moved<0x111, 15>(x);       // of 16 lanes: from 1, 2, 4 and 8 before
  x += moved<0x112, 15>(x);
  x += moved<0x114, 15>(x);
  x += moved<0x118, 15>(x);
  x += moved<0x142, 10>(x);       // the first 16's to the second's, the third's to the fourth's
  x += moved<0x143, 12>(x);       // the first half's to the second's
  return x;
}

// What a launch is for: the segments' own contributions to the state and their logarithms' sums; the result; dq or dk, and dv, with their parts of the
// gates' gradient (dq and dk also without).
enum { kStates = 0, kResult = 1, kOfStates = 2, kOfPairs = 3 };
// numbers of 16 bits that stand for one of fp32 (one float otherwise)
template <class Core, int MODE>
constexpr int kPieces = std::is_same_v<Core, float> ? 1 : std::is_same_v<Core, f16_t> || MODE == kResult || MODE == kOfPairs ? 2 : 3;
// Waves of a SIMD: those of two workgroups where a compute unit's LDS holds two.
template <class Core, int DA, int WAVES>
constexpr int kChunkWaves = WAVES == 8 ? (sizeof(ChunkShared<Core, DA, WAVES>) * 2 > 163840 ? 2 : 4) : sizeof(ChunkShared<Core, DA, WAVES>) * 2 > 163840 ? 1 : 2;

template <class In, int DA, int WAVES, int MODE, int WAY>
__global__ __launch_bounds__(64 * WAVES, (kChunkWaves<In, DA, WAVES>)) void k_linear_chunks(LinearArgs A, LinearPass P, LinearChunks C) {
  typedef ChunkShared<In, DA, WAVES> Shared;
  constexpr bool STATE = MODE == kStates, DOTS = MODE == kOfStates, PAIRS = MODE == kOfPairs, X_IN_LDS = sizeof(In) == 2;
  constexpr bool RANGED = std::is_same_v<In, f16_t>;
  constexpr int N_OUT = kPieces<In, MODE>, N_STATE = kPieces<In, kStates>, kSlice = Shared::kSlice;
  typedef Operand<In> Op;
  typedef typename Op::Frag Frag;
  constexpr int kJ = DA / Op::kInner, kT = Op::kTiles, kS = kChunk / Op::kInner;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  Shared& S = *reinterpret_cast<Shared*>(lds);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, l = lane & 15, g = lane >> 4;
  const ChunkPlace place = chunk_place(A, C);
  if (!place.there) return;
  const int slice = place.slice, segment = place.segment;
  const int64_t bh = place.bh, b = bh / A.heads, entries = (int64_t)P.da * P.dc;
  const int64_t len = __builtin_amdgcn_readfirstlane((int)steps_of(A, b));      // (below 2^31)
  const int h = (int)(bh % A.heads), col = slice * kSlice + 16 * wave;     // the wave's first column
  const In* pa = (const In*)P.a + b * P.a_seq + (h / P.a_share) * P.a_head;
  const In* pb = (const In*)P.b + b * P.b_seq + (h / P.b_share) * P.b_head;
  const In* pc = (const In*)P.c + b * P.c_seq + (h / P.c_share) * P.c_head + slice * kSlice;
  const In* px = (const In*)P.x + b * P.x_seq + (h / P.x_share) * P.x_head;
  const int64_t out = b * P.out_seq + h * P.out_head;
  const int64_t begin = (int64_t)segment * C.chunks * kChunk;
  const int64_t end = segment + 1 == C.segments ? A.steps : begin + (int64_t)C.chunks * kChunk;
  const int in_slice = min(P.dc - slice * kSlice, kSlice);

  f32x4 state[kJ * kT];       // rows 16 j + 4 g + r of column `col + l`
  const float* from = STATE ? nullptr : C.states ? C.states + (bh * C.states_of + segment) * entries : P.first ? P.first + bh * P.first_of * entries : nullptr;
  const bool column = col + l < P.dc;
  if (P.state_a == 1 && P.da % 4 == 0 && ((uintptr_t)from & 15) == 0) {      // four rows are next to one another (and so are on their border)
#pragma unroll
    for (int j = 0; j < kJ * kT; ++j) {
      const int row = 16 * j + 4 * g;
      state[j] = from && column && row < P.da ? *(const f32x4*)(from + (int64_t)(col + l) * P.state_c + row) : f32x4{};
    }
  } else {
#pragma unroll
    for (int j = 0; j < kJ * kT; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = 16 * j + 4 * g + r;
        state[j][r] = from && column && row < P.da ? from[(int64_t)row * P.state_a + (int64_t)(col + l) * P.state_c] : 0.0f;
      }
  }
  const auto keep = [&](float* to, float w) {
    int mine = 4 * g;
    asm volatile("" : "+v"(mine));      // (or its addresses would be kept in registers over the chunks)
    to += (int64_t)(col + l) * P.state_c + (int64_t)mine * P.state_a;
#pragma unroll
    for (int j = 0; j < kJ * kT; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (column && 16 * j + r + mine < P.da) to[(16 * j + r) * P.state_a] = state[j][r] * w;
  };
  double total = 0.0;

  // The state's products with one of the other direction, <E, S>: the sum over a wave's columns.
  const auto meet = [&](const float* other, int thread) -> float {
    const int l = thread & 15, row = (thread & 63) >> 4 << 2;
    const float* p = other + (int64_t)(col + l) * P.state_c + (int64_t)row * P.state_a;
    const bool together = P.state_a == 1 && P.da % 4 == 0 && ((uintptr_t)other & 15) == 0, in = col + l < P.dc;
    float sum = 0.0f;
#pragma unroll
    for (int j = 0; j < kJ * kT; ++j) {
      f32x4 x = {};
      if (together) {
        if (in && row + 16 * j < P.da) x = *(const f32x4*)(p + 16 * j);
      } else {
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (in && row + 16 * j + r < P.da) x[r] = p[(16 * j + r) * P.state_a];
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) sum = fmaf(x[r], state[j][r], sum);
    }
    return rows_summed(row_sum(sum));
  };

  const int64_t inside = min(end, len);       // steps of the segment that are in the sequence end here
  const int chunks = inside > begin ? (int)((inside - begin + kChunk - 1) / kChunk) : 0;
  Staged<In, DA, 1, WAVES, WAY> next_a;
  Staged<In, DA, Shared::kTurned ? 4 : 1, WAVES, WAY> next_b;
  Staged<In, kSlice, 1, WAVES, WAY> next_c;
  float next_g = 0.0f;
  const int64_t dir = P.back ? -1 : 1;
  const auto begin_of = [&](int i) { return begin + (int64_t)(P.back ? chunks - 1 - i : i) * kChunk; };
  const auto ask = [&](int i, int thread) {
    const int64_t t0 = begin_of(i), first = t0 + (P.back ? kChunk - 1 : 0);      // the time of row 0
    const int there = (int)min((int64_t)kChunk, inside - t0), lo = P.back ? kChunk - there : 0, hi = P.back ? kChunk : there;
    if (!STATE) next_a.load(thread, pa + t0 * P.a_step, P.a_step, P.back, P.da, lo, hi);
    next_b.load(thread, pb + t0 * P.b_step, P.b_step, P.back, P.da, lo, hi);
    next_c.load(thread, pc + t0 * P.c_step, P.c_step, P.back, in_slice, lo, hi);
    if (wave == 0) {
      const int64_t t = first + dir * lane + (P.back ? 1 : 0);
      next_g = lane >= lo && lane < hi && t < len ? log_gate(A, b, t, h) : 0.0f;
    }
  };
  // P^T by tiles of 16 x 16: rows s, columns t, s <= t, and two of zeros that complete an operand of two tiles.  A wave's are the
  // pairs t, s in a word, three of them or two.
  constexpr int kTiles = WAVES == 4 ? 3 : 2;
  constexpr uint32_t kOfWaves[8] = {WAVES == 4 ? 0x300010u : 0x0010u, WAVES == 4 ? 0x311101u : 0x1101u, WAVES == 4 ? 0x322021u : 0x20FFu,
                                    WAVES == 4 ? 0x332223u : 0x21FFu, 0x2223u, 0x3031u, 0x32FFu, 0x33FFu};
  uint32_t tiles = kOfWaves[0];
#pragma unroll
  for (int w = 1; w < WAVES; ++w)
    if (wave == w) tiles = kOfWaves[w];
  // What a chunk's pairs put on its steps, those on either side of each, by one wave (backwards: a step's begin is its row's end).
  const auto gather = [&](int i) {
    const int64_t t0 = begin_of(i);
    const int row = kChunk - lane, m = row >> 4, e = row & 15;      // (the row from whose begin on pairs count)
    const auto tile = [](int t, int s) { return t * (t + 1) / 2 + s; };
    const auto of = [](bool there, float x) { return there ? x : 0.0f; };
    const int mine = m & 3;
    float sum = S.behind[tile(mine, mine)][e];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      sum += of(k < mine, S.behind[tile(mine, k < mine ? k : 0)][e]);
      sum += of(mine + k < 3, S.before[tile(mine + k < 3 ? mine + k + 1 : 3, mine + k < 3 ? mine : 0)][e]);
    }
    if (mine == 1) sum += S.behind[tile(2, 0)][0] + S.behind[tile(3, 0)][0];
    if (mine == 2) sum += S.behind[tile(3, 0)][0] + S.behind[tile(3, 1)][0];
    if (m > 3) sum = 0.0f;
    if (t0 + lane >= inside) return;
    P.dots[((int64_t)slice * A.batch * A.heads + bh) * A.steps + t0 + lane] = sum;
  };
  if (chunks > 0) ask(0, threadIdx.x);
  for (int i = 0; i < chunks; ++i) {
    // (threads' places are worked out anew for every chunk: kept over them, they would take more registers than there are)
    int thread = threadIdx.x;
    asm volatile("" : "+v"(thread));
    const int lane = thread & 63, l = lane & 15, g = lane >> 4;
    const int64_t t0 = begin_of(i), first_time = t0 + (P.back ? kChunk - 1 : 0);
    // rows of the chunk that are in the sequence: forwards its first ones, backwards its last
    const int there = (int)min((int64_t)kChunk, inside - t0), lo = P.back ? kChunk - there : 0, hi = P.back ? kChunk : there;
    if (MODE == kResult && P.kept && t0 % kLinearSave == 0) keep(P.kept + (bh * P.kept_of + t0 / kLinearSave) * entries, 1.0f);
    __syncthreads();
    if (PAIRS && i > 0 && wave == WAVES - 1) gather(i - 1);
    if (!STATE) next_a.store(thread, S.a);
    if constexpr (Shared::kTurned) next_b.store_turned(thread, S.turned);
    if (!STATE || !Shared::kTurned) next_b.store(thread, S.b);
    next_c.store(thread, S.c);
    const bool busy = 16 * wave < in_slice;      // (the others help with P only)
    // What goes through a whole chunk to the gates' gradient is <E, S> of its two ends.  In memory there are S at the begins and E at the ends of
    // pieces of four chunks: dk's pass, which has E, does the first two, dq's, which has S, the last two.  Of these each does one with the
    // next chunk "ahead": E reaches the piece's begin, or S its end, by way of that chunk's rows.
    const int in_piece = (int)(t0 / kChunk) % (kLinearSave / kChunk);
    const bool meets = DOTS && P.dots && (P.back ? in_piece < 2 : in_piece >= 2), ahead = meets && in_piece == (P.back ? 1 : 2) && i + 1 < chunks;
    // the step whose logarithm the chunks' sums lack
    const int64_t past = P.back ? t0 - (ahead ? kChunk : 0) : t0 + (ahead ? 2 : 1) * kChunk;
    const float past_gate = meets && past < len ? log_gate(A, b, past, h) : 0.0f;
    if constexpr (DOTS) {
      if (meets && busy) {
        const int64_t piece = t0 / kLinearSave;
        const bool within = P.back || (piece + 1) * kLinearSave < len;
        const float* other = within ? P.met + (bh * P.met_of + piece) * entries : P.met_last ? P.met_last + bh * entries : nullptr;
        S.met[wave] = other ? meet(other, thread) : 0.0f;
      }
    }
    if (!STATE && RANGED && wave == WAVES - 1) S.most[lane] = 0;
    if (wave == 0) {      // the logarithms' sums
      const double x = sums_to(next_g < kLinearLeast ? (double)kLog2Least : (double)next_g * 1.4426950408889634);
      const double all = __shfl(x, 63);
      S.c_high[lane] = (float)x;
      S.c_low[lane] = (float)(x - (double)(float)x);
      S.to_end[lane] = __builtin_amdgcn_exp2f((float)(all - x));
      total += all;
    }
    const int first = col + 4 * g;
    if (i + 1 < chunks) ask(i + 1, thread);
    // four entries of a row of x from column `at` on, of which `width` are there
    const auto entries_of_x = [&](int64_t t0, int lo, int hi, int row, int at, int width) {
      Four<In> x;
      const int when = P.back ? kChunk - 1 - row : row;
      const bool here = row >= lo && row < hi;
      if constexpr (WAY != kEntries) {
        const __amdgpu_buffer_rsrc_t from = __builtin_amdgcn_make_buffer_rsrc((void*)(px + t0 * P.x_step), 0, kBufferBytes, 0x00027000);
        x.load(from, here ? ((uint32_t)when * (uint32_t)P.x_step + (uint32_t)at) * (uint32_t)sizeof(In) : ~0u, width, C.vec_x == 4);
      } else {
        x.load(px + (t0 + when) * P.x_step + at, here ? width : 0);
      }
      return x;
    };
    constexpr int kXWide = X_IN_LDS || kSlice < DA ? kSlice : DA, kXParts = kSlice / kXWide;
    Staged<In, kXWide, 1, WAVES, WAY> now_x[kXParts];
    if constexpr (PAIRS)
#pragma unroll
      for (int k = 0; k < kXParts; ++k)
        now_x[k].load(thread, px + slice * kSlice + k * kXWide + t0 * P.x_step, P.x_step, P.back, in_slice - k * kXWide, lo, hi);
    __syncthreads();
    Frag cf[kS];       // column l's entries, a lane's steps
    const auto columns = [&](Frag (&cf)[kS]) {
#pragma unroll
      for (int s = 0; s < kS; ++s)
#pragma unroll
        for (int t = 0; t < kT; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r) cf[s][4 * t + r] = S.c[16 * (s * kT + t) + 4 * g + r][16 * wave + l];
    };
    if constexpr (!STATE) {
      // what comes of the state before the chunk
      f32x4 y[4] = {};
      // y += S^T a of the rows in LDS, in fp16 times powers of two for each column of S that are taken back by the result
      const auto by_state = [&](f32x4 (&y)[4]) -> f32x4 {
        float most = 0.0f;
        if constexpr (RANGED)
          most = largest_of_column([&](auto&& see) {
#pragma unroll
            for (int j = 0; j < kJ * kT; ++j)
#pragma unroll
              for (int r = 0; r < 4; ++r) see(state[j][r]);
          });
        const Range range(most);
#pragma unroll
        for (int j = 0; j < kJ; ++j) {
          Frag p[N_OUT];
          if constexpr (RANGED) {
            const f32x4 ranged[2] = {state[j * kT] * range.up, state[j * kT + 1] * range.up};
            pieces_of<In, N_OUT>(ranged, p);
          } else {
            pieces_of<In, N_OUT>(*(const f32x4(*)[kT])&state[j * kT], p);
          }
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            const Frag q = Op::load(&S.a[16 * t + l][0], j, g);
#pragma unroll
            for (int n = N_OUT - 1; n >= 0; --n) y[t] = Op::mma(p[n], q, y[t]);
          }
        }
        f32x4 down = {};      // of the columns that a lane has of y
        if constexpr (RANGED)
#pragma unroll
          for (int r = 0; r < 4; ++r) down[r] = __shfl(range.down, 4 * g + r);
        return down;
      };
      const auto products_with = [&](const f32x4& y, const Four<In>& x) {      // of a row of the wave's columns (what is not there is zero)
        float d = 0.0f;
#pragma unroll
        for (int r = 0; r < 4; ++r) d = fmaf(y[r], x[r], d);
        return rows_summed(d);
      };
      const auto from_state = [&] {
        if (!busy) return;
        Four<In> times[4];
        if constexpr (DOTS)
          if (P.dots)
#pragma unroll
            for (int t = 0; t < 4; ++t) times[t] = entries_of_x(t0, lo, hi, 16 * t + l, first, P.dc - first);
        const f32x4 down = by_state(y);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const float here = __builtin_amdgcn_exp2f(S.c_high[16 * t + l] + S.c_low[16 * t + l]);
#pragma unroll
          for (int r = 0; r < 4; ++r) y[t][r] *= RANGED ? here * down[r] : here;
          if constexpr (DOTS)
            if (P.dots) {
              const float d = products_with(y[t], times[t]);
              if (g == 0) S.dots[wave][16 * t + l] = d;
            }
        }
      };
      from_state();
      f32x4 score[kTiles];
      // x by rows: in 16 bits behind P's two pieces, in fp32 over P once that has been used, as many columns as there is room for
      typedef In XRows[kChunk][kXWide + Shared::kPad];
      XRows& x_rows = *reinterpret_cast<XRows*>(&S.a[0][0] + (X_IN_LDS ? Shared::kTwo : 0));
      const auto add_products_of_x = [&](f32x4& sum, int s, int t, int from) {      // of rows s of c with rows t of x
#pragma unroll
        for (int j = 0; j < kXWide / Op::kInner; ++j)
          sum = Op::mma(Op::load(&S.c[16 * s + l][from], j, g), Op::load(&x_rows[16 * t + l][0], j, g), sum);
      };
      // Pairs of a row of tile s (4 g + r of its tile) and one of tile t (column l).  Their sums over those on either side of a row's begin: in one tile
      // by row, of two tiles over t's rows from one on and over s's before it.
      const auto sums_of_pairs = [&](const f32x4& pairs, int t, int s) {
        const int tile = t * (t + 1) / 2 + s;
        float behind = 0.0f;
        if (s == t) {
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float from = row_sums_from(pairs[r]);
            behind += 4 * g + r < l ? from : 0.0f;
          }
        } else {
          behind = row_sums_from((pairs[0] + pairs[1]) + (pairs[2] + pairs[3]));
          f32x4 before;
          float sum = 0.0f;
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            before[r] = sum;
            sum += row_sum(pairs[r]);
          }
          const float rows = rows_before(sum);
          if (l == 0) *(f32x4*)&S.before[tile][4 * g] = before + rows;
        }
        behind = rows_summed(behind);
        if (g == 0) S.behind[tile][l] = behind;
      };
#pragma unroll
      for (int n = 0; n < kTiles; ++n) {
        const int pair = tiles >> (8 * (kTiles - 1 - n)) & 255, t = pair >> 4, s = pair & 15;
        score[n] = f32x4{};
        if (s > t || 16 * t >= hi || 16 * t + 15 < lo) continue;
#pragma unroll
        for (int j = 0; j < kJ; ++j) score[n] = Op::mma(Op::load(&S.b[16 * s + l][0], j, g), Op::load(&S.a[16 * t + l][0], j, g), score[n]);
        const float high = S.c_high[16 * t + l], low = S.c_low[16 * t + l];
        const f32x4 high_s = *(const f32x4*)&S.c_high[16 * s + 4 * g], low_s = *(const f32x4*)&S.c_low[16 * s + 4 * g];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float weighted = score[n][r] * __builtin_amdgcn_exp2f((high - high_s[r]) + (low - low_s[r]));
          score[n][r] = s < t || 4 * g + r <= l ? weighted : 0.0f;
        }
      }
      if constexpr (RANGED)
#pragma unroll
        for (int n = 0; n < kTiles; ++n) {
          const int pair = tiles >> (8 * (kTiles - 1 - n)) & 255, t = pair >> 4, s = pair & 15;
          if (s > t || t > 3) continue;
          const float most = largest_of_column([&](auto&& see) {
#pragma unroll
            for (int r = 0; r < 4; ++r) see(score[n][r]);
          });
          if (g == 0) atomicMax(&S.most[16 * t + l], __float_as_uint(most));      // (the order does not matter)
        }
      const auto range_of = [&](int t) { return Range(__uint_as_float(S.most[16 * t + l])); };      // of P's row
      __syncthreads();
      // P by rows, over a (and b, which in 16 bits is needed by columns only from here on)
      In (*const scores)[kChunk][Shared::kScoreRow] = reinterpret_cast<In (*)[kChunk][Shared::kScoreRow]>(&S.a[0][0]);
      static_assert(Shared::kTurned ? N_OUT <= 3 : kChunk * Shared::kScoreRow * sizeof(In) <= sizeof(S.a));
#pragma unroll
      for (int n = 0; n < kTiles; ++n) {
        const int pair = tiles >> (8 * (kTiles - 1 - n)) & 255, t = pair >> 4, s = pair & 15;
        if (t > 3) continue;
        float left[4] = {score[n][0], score[n][1], score[n][2], score[n][3]};
        if constexpr (RANGED) {
          const float up = range_of(t).up;
#pragma unroll
          for (int r = 0; r < 4; ++r) left[r] *= up;
        }
#pragma unroll
        for (int k = 0; k < N_OUT; ++k) {
          store_floats<In, 4>(&scores[k][16 * t + l][16 * s + 4 * g], left);
#pragma unroll
          for (int r = 0; r < 4; ++r) left[r] -= to_float((In)left[r]);
        }
      }
      if constexpr (PAIRS && X_IN_LDS) now_x[0].store(thread, x_rows);
      __syncthreads();
      const auto all_pairs = [&] {
        f32x4 sum[kTiles] = {};
#pragma unroll
        for (int k = 0; k < kXParts; ++k) {
          if (!X_IN_LDS) {
            __syncthreads();
            now_x[k].store(thread, x_rows);
            __syncthreads();
          }
#pragma unroll
          for (int n = 0; n < kTiles; ++n) {
            const int pair = tiles >> (8 * (kTiles - 1 - n)) & 255, t = pair >> 4, s = pair & 15;
            if (s > t || 16 * t >= hi || 16 * t + 15 < lo) continue;
            add_products_of_x(sum[n], s, t, k * kXWide);
            if (k + 1 == kXParts) sums_of_pairs(score[n] * sum[n], t, s);
          }
        }
      };
      if constexpr (PAIRS && X_IN_LDS) all_pairs();
      if (busy) {
        columns(cf);
        const uint32_t out_size = P.wide ? 4 : sizeof(In);
        char* const earliest = (char*)P.out + out_size * (out + t0 * P.out_step);
        const __amdgpu_buffer_rsrc_t to = __builtin_amdgcn_make_buffer_rsrc(earliest, 0, kBufferBytes, 0x00027000);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          if (16 * t >= hi || 16 * t + 15 < lo) continue;
          f32x4 sum = RANGED ? f32x4{} : y[t];
#pragma unroll
          for (int s = 0; s <= t / kT; ++s)
#pragma unroll
            for (int n = N_OUT - 1; n >= 0; --n) sum = Op::mma(cf[s], Op::load(&scores[n][16 * t + l][0], s, g), sum);
          if constexpr (RANGED) y[t] += sum * range_of(t).down;
          else y[t] = sum;
          // rows of the result: step 16 t + l, columns 4 g to 4 g + 3 of the wave's
          const int row = 16 * t + l, when = P.back ? kChunk - 1 - row : row;
          const bool here = row >= lo && row < hi;
          if constexpr (WAY != kEntries) {
            const uint32_t at = here ? ((uint32_t)when * (uint32_t)P.out_step + (uint32_t)first) * out_size : ~0u;
            if (P.wide) store_four<float>(to, at, P.dc - first, C.vec_out == 4, y[t]);
            else store_four<In>(to, at, P.dc - first, C.vec_out == 4, y[t]);
          } else if (here) {
#pragma unroll
            for (int r = 0; r < 4; ++r)
              if (first + r < P.dc) store_result<In>(P, out + (t0 + when) * P.out_step + first + r, y[t][r]);
          }
        }
      }
      if constexpr (DOTS) {
        if (ahead) {      // the next chunk's rows with this one's state
          int thread = threadIdx.x;      // (anew, for the registers)
          asm volatile("" : "+v"(thread));
          const int lane = thread & 63, l = lane & 15, g = lane >> 4, first = col + 4 * g;
          const int64_t t1 = begin_of(i + 1);
          const int there = (int)min((int64_t)kChunk, inside - t1), lo = P.back ? kChunk - there : 0, hi = P.back ? kChunk : there;
          __syncthreads();
          next_a.store(thread, S.a);
          if (wave == 0) {
            const double x = sums_to(next_g < kLinearLeast ? (double)kLog2Least : (double)next_g * 1.4426950408889634);
            S.weights[lane] = __builtin_amdgcn_exp2f((float)x);
            if (lane == 63) S.ahead_all = (float)x;
          }
          __syncthreads();
          if (busy) {
            f32x4 z[4] = {};
            const f32x4 down = by_state(z);
            Four<In> times[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) times[t] = entries_of_x(t1, lo, hi, 16 * t + l, first, P.dc - first);
            float sum = 0.0f;
#pragma unroll
            for (int t = 0; t < 4; ++t) {
              const int row = 16 * t + l;
              const float d = products_with(RANGED ? z[t] * down : z[t], times[t]);
              sum += row >= lo && row < hi ? d * S.weights[row] : 0.0f;
            }
            S.ahead[wave] = row_sum(sum);
          }
          __syncthreads();
        }
        if (P.dots && wave == WAVES - 1) {
          // of a step: later steps of the chunk with what was before the chunk, or earlier ones with what comes behind it, and what goes
          // through the whole chunk
          const bool here = lane >= lo && lane < hi;
          float d = 0.0f, met = 0.0f, beyond = 0.0f;
          for (int w = 0; w < (in_slice + 15) / 16; ++w) {
            d += S.dots[w][lane];
            if (meets) met += S.met[w];
            if (ahead) beyond += S.ahead[w];
          }
          d = sums_from(here ? d : 0.0f, !P.back, g);
          if (meets) {
            const float high = S.c_high[kChunk - 1], low = S.c_low[kChunk - 1], more = past_gate < kLinearLeast ? kLog2Least : past_gate * 1.44269504f;
            met *= __builtin_amdgcn_exp2f(high + (low + (more + (ahead ? S.ahead_all : 0.0f))));
            if (ahead) met = fmaf(beyond, __builtin_amdgcn_exp2f(high + low), met);
          }
          if (here) P.dots[((int64_t)slice * A.batch * A.heads + bh) * A.steps + first_time + dir * lane] = d + met;
        }
      }
      if constexpr (PAIRS && !X_IN_LDS) all_pairs();
      if (i + 1 == chunks && (C.states || !P.last) && !(MODE == kResult && P.kept)) break;      // nobody reads the state
    }
    if (!busy) continue;
    if constexpr (STATE) columns(cf);
    const float all = __builtin_amdgcn_exp2f(S.c_high[kChunk - 1] + S.c_low[kChunk - 1]);
    const auto weighted = [&](int s, f32x4 (&w)[kT]) {
#pragma unroll
      for (int t = 0; t < kT; ++t) {
        const f32x4 left = *(const f32x4*)&S.to_end[16 * (s * kT + t) + 4 * g];
#pragma unroll
        for (int r = 0; r < 4; ++r) w[t][r] = (float)cf[s][4 * t + r] * left[r];
      }
    };
    const auto rows_of_b = [&](int s, int j) {
      Frag rows;
      if constexpr (Shared::kTurned) {
        rows = Op::load(&S.turned[16 * j + l][0], s, g);
      } else {
#pragma unroll
        for (int r = 0; r < 4; ++r) rows[r] = S.b[16 * s + 4 * g + r][16 * j + l];
      }
      return rows;
    };
    if constexpr (RANGED) {
      f32x4 w[kS][kT];
#pragma unroll
      for (int s = 0; s < kS; ++s) weighted(s, w[s]);
      const Range range(largest_of_column([&](auto&& see) {
#pragma unroll
        for (int s = 0; s < kS; ++s)
#pragma unroll
          for (int t = 0; t < kT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) see(w[s][t][r]);
      }));
      Frag p[kS][N_STATE];
#pragma unroll
      for (int s = 0; s < kS; ++s) {
#pragma unroll
        for (int t = 0; t < kT; ++t) w[s][t] = w[s][t] * range.up;
        pieces_of<In, N_STATE>(w[s], p[s]);
      }
#pragma unroll
      for (int j = 0; j < kJ * kT; ++j) {
        f32x4 sum = {};
#pragma unroll
        for (int s = 0; s < kS; ++s) {
          const Frag rows = rows_of_b(s, j);
#pragma unroll
          for (int n = N_STATE - 1; n >= 0; --n) sum = Op::mma(rows, p[s][n], sum);
        }
        state[j] = state[j] * all + sum * range.down;
      }
    } else {
#pragma unroll
      for (int j = 0; j < kJ * kT; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) state[j][r] *= all;
#pragma unroll
      for (int s = 0; s < kS; ++s) {
        f32x4 w[kT];
        weighted(s, w);
        Frag p[N_STATE];
        pieces_of<In, N_STATE>(w, p);
#pragma unroll
        for (int j = 0; j < kJ * kT; ++j) {
          const Frag rows = rows_of_b(s, j);
#pragma unroll
          for (int n = N_STATE - 1; n >= 0; --n) state[j] = Op::mma(rows, p[n], state[j]);
        }
      }
    }
  }
  if constexpr (STATE) {
    keep(C.states + (bh * C.states_of + segment) * entries, 1.0f);
    if (slice == 0 && threadIdx.x == 0) C.totals[bh * C.segments + segment] = total;
    return;
  }
  if (PAIRS && chunks > 0) {
    __syncthreads();
    if (wave == WAVES - 1) gather(chunks - 1);
  }
  // zeros behind the sequence
  const int64_t zero = max(begin, len);
  const int width = in_slice;
  for (int64_t e = threadIdx.x; e < (end - zero) * width; e += 64 * WAVES)
    store_result<In>(P, out + (zero + e / width) * P.out_step + slice * kSlice + e % width, 0.0f);
  if (MODE == kResult && P.kept && (len == 0 ? segment == 0 : begin < len && len <= end))
    keep(P.kept + (bh * P.kept_of + (len + kLinearSave - 1) / kLinearSave) * entries, 1.0f);
  if (!DOTS && P.last && !C.states) keep(P.last + bh * entries, P.back && len > 0 ? linear_decay(log_gate(A, b, 0, h)) : 1.0f);
}

#ifndef CHOCO_LINEAR_TYPE      // (where only one type's chunks are compiled)
// From the segments' own contributions to the states before them, in place, and the last one.  Bound by memory: 40 heads of 128 x 128 in 64
// segments 64 us, 5.3 TB/s (one segment after the other, each waited for, 93).
__global__ __launch_bounds__(256) void k_linear_scan(LinearArgs A, float* states, const double* totals, int segments, int64_t entries, const float* first,
                                                     float* last, bool back) {
  const int64_t each = (entries + 255) / 256, count = A.batch * A.heads * each;
  for (int64_t block = blockIdx.x; block < count; block += gridDim.x) {
    const int64_t bh = block / each, b = bh / A.heads, e = block % each * 256 + threadIdx.x;
    if (e >= entries) continue;
    float s = first ? first[bh * entries + e] : 0.0f;
    float* p = states + bh * segments * entries + e;
    constexpr int kAhead = 16;      // (asked for together: a store may be of the next one's entry, for all that the compiler knows)
    for (int i = 0; i < segments; i += kAhead) {
      float own[kAhead], decay[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k)
        if (i + k < segments) {
          const int at = back ? segments - 1 - i - k : i + k;
          own[k] = p[at * entries];
          decay[k] = __builtin_amdgcn_exp2f((float)totals[bh * segments + at]);
        }
#pragma unroll
      for (int k = 0; k < kAhead; ++k)
        if (i + k < segments) {
          p[(back ? segments - 1 - i - k : i + k) * entries] = s;
          s = fmaf(s, decay[k], own[k]);
        }
    }
    if (last) last[bh * entries + e] = back && steps_of(A, b) > 0 ? s * linear_decay(log_gate(A, b, 0, (int)(bh % A.heads))) : s;
  }
}

// ---- the gates' gradient ----
// dg_t = e^g_t <E_t, S_{t-1}> = the sum over pairs of steps s >= t > r of e^(c_s - c_r) (q_s k_r) (dy_s v_r), where r may also stand for the first state
// and s for the last one's gradient: only what passes t is added up, so that a gate that hardly lets anything through has as many places right as
// any other.  (By differences, sums of q dq - k dk, a gate of -10 beside open ones has two, one of -20 none.)  In chunks, dv's pass has pairs
// within a chunk, as score times score, dq's and dk's those with what is before or behind it, by slices.  Bound as these passes are: of 4 x 16,384 x 10 x
// 128 in bf16 dq and dk take 395 us each (325 without their part: a state more to read for two of four chunks, a product with another chunk's rows),
// dv 297 (245: its x to read, a score more); in fp32, 160 x 35 x 13 x 50, 70 (65) and 91 (70).  What is left, the slices' sum, takes 7 us of the long one.
// Not kept: states between the chunks written by dq's pass and read by dk's, 1,680 to 1,420 us in all; pairs in dq's pass, whose registers do not hold them.
struct LinearGates {
  const float* dots;     // [slices of dq, dk and dv][batch * heads][steps]
  int32_t slices;
  float* dg;       // [batch][steps][heads], or the pieces' sums [heads][batch * pieces]
  int64_t pieces;
  bool sums;
};

__device__ __forceinline__ double wave_sum(double x) {
  for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o);
  return x;
}

__global__ __launch_bounds__(kLinearSave) void k_linear_gates(LinearArgs A, LinearGates G) {
  __shared__ double part[4];
  const int64_t bh = blockIdx.x / G.pieces, piece = blockIdx.x % G.pieces, b = bh / A.heads, t = piece * kLinearSave + threadIdx.x;
  const int h = (int)(bh % A.heads), wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  float dg = 0.0f;
  if (t < steps_of(A, b) && !(log_gate(A, b, t, h) < kLinearLeast))
    for (int s = 0; s < G.slices; ++s) dg += G.dots[(s * A.batch * A.heads + bh) * A.steps + t];
  if (!G.sums) {
    if (t < A.steps) G.dg[(b * A.steps + t) * A.heads + h] = dg;
    return;
  }
  const double sum = wave_sum((double)dg);
  if (lane == 0) part[wave] = sum;
  __syncthreads();
  if (threadIdx.x == 0) G.dg[h * A.batch * G.pieces + b * G.pieces + piece] = (float)((part[0] + part[1]) + (part[2] + part[3]));
}

// ... of up to N steps, by one workgroup for a sequence and head: products of steps' rows, and of rows with the first state and the last one's gradient, both read
// once.  Bound by latency: 8 steps of 160 x 10 heads of 64 in fp32 37 us, the two states 10 at the rate of a copy.  P is dv's pass (a, b, c = k, q, dy) with x = v; P.first and P.met_last are the two states.
constexpr int few_row(int n) { return 2 * n + 4; }       // floats of a row of LDS, of which four neighbours are read at a time
template <class T, int N>
__global__ __launch_bounds__(256) void k_linear_few_gates(LinearArgs A, LinearPass P, LinearGates G) {
  constexpr int kRow = few_row(N);
  extern __shared__ __attribute__((aligned(16))) char few_lds[];
  float (*const qk)[kRow] = reinterpret_cast<float (*)[kRow]>(few_lds), (*const yv)[kRow] = qk + P.da;     // [entry][step of q or dy, step of k or v]
  __shared__ float w[N], pairs[N][N], part[4][2 * N + 1];
  const int64_t bh = blockIdx.x, b = bh / A.heads;
  const int h = (int)(bh % A.heads), wave = threadIdx.x >> 6, lane = threadIdx.x & 63, n = (int)steps_of(A, b);
  const T* pk = (const T*)P.a + b * P.a_seq + (h / P.a_share) * P.a_head;
  const T* pq = (const T*)P.b + b * P.b_seq + (h / P.b_share) * P.b_head;
  const T* py = (const T*)P.c + b * P.c_seq + (h / P.c_share) * P.c_head;
  const T* pv = (const T*)P.x + b * P.x_seq + (h / P.x_share) * P.x_head;
  static_assert(2 * N % 4 == 0);
  const auto stage = [&](float (*to)[kRow], int dim, const T* x, int64_t x_step, const T* y, int64_t y_step) {
    const int e = threadIdx.x;      // (256 entries at most)
    if (e >= dim) return;
    float all[2 * N];
#pragma unroll
    for (int s = 0; s < N; ++s) {
      all[s] = s < n ? to_float(x[s * x_step + e]) : 0.0f;
      all[N + s] = s < n ? to_float(y[s * y_step + e]) : 0.0f;
    }
#pragma unroll
    for (int k = 0; k < 2 * N; k += 4) *(float4*)&to[e][k] = float4{all[k], all[k + 1], all[k + 2], all[k + 3]};
  };
  stage(qk, P.da, pq, P.b_step, pk, P.a_step);
  stage(yv, P.dc, py, P.c_step, pv, P.x_step);
  if (threadIdx.x < N) w[threadIdx.x] = (int)threadIdx.x < n ? linear_decay(log_gate(A, b, threadIdx.x, h)) : 1.0f;
  __syncthreads();
  {      // a pair of steps by so many threads
    constexpr int kEach = 256 / (N * N);
    const int s = threadIdx.x / (N * kEach), r = threadIdx.x / kEach % N;
    float x = 0.0f, y = 0.0f;
    if (r < s && s < n) {
      for (int e = threadIdx.x % kEach; e < P.da; e += kEach) x = fmaf(qk[e][s], qk[e][N + r], x);
      for (int e = threadIdx.x % kEach; e < P.dc; e += kEach) y = fmaf(yv[e][s], yv[e][N + r], y);
    }
    for (int o = kEach / 2; o; o >>= 1) {
      x += __shfl_xor(x, o);
      y += __shfl_xor(y, o);
    }
    x *= y;
    for (int u = r + 1; u <= s; ++u) x *= w[u];
    if (threadIdx.x % kEach == 0) pairs[s][r] = x;
  }
  float sums[2 * N + 1] = {};      // q_s S dy_s, k_r E v_r, <E, S>
  const int64_t state = (int64_t)P.da * P.dc;
  const float* first = P.first ? P.first + bh * P.first_of * state : nullptr;
  const float* last = P.met_last ? P.met_last + bh * state : nullptr;
  for (int col = lane; col < P.dc; col += 64) {
    float column[2 * N] = {};
    constexpr int kAhead = 8;      // rows under way
    for (int i0 = wave; i0 < P.da; i0 += 4 * kAhead) {
      float s[kAhead], e[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int i = i0 + 4 * u;
        s[u] = first && i < P.da ? first[(int64_t)i * P.dc + col] : 0.0f;
        e[u] = last && i < P.da ? last[(int64_t)i * P.dc + col] : 0.0f;
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const float* row = qk[min(i0 + 4 * u, P.da - 1)];      // (with zeros where there is none)
#pragma unroll
        for (int k = 0; k < 2 * N; ++k) column[k] = fmaf(row[k], k < N ? s[u] : e[u], column[k]);
        sums[2 * N] = fmaf(s[u], e[u], sums[2 * N]);
      }
    }
#pragma unroll
    for (int k = 0; k < 2 * N; ++k) sums[k] = fmaf(column[k], yv[col][k], sums[k]);
  }
#pragma unroll
  for (int k = 0; k <= 2 * N; ++k) {
    const float x = rows_summed(row_sum(sums[k]));
    if (lane == 0) part[wave][k] = x;
  }
  const int t = threadIdx.x;
  const bool counts = t < n && !(log_gate(A, b, t, h) < kLinearLeast);
  __syncthreads();
  if (wave > 0) return;
  float all[2 * N + 1];
  const float x = lane <= 2 * N ? (part[0][lane] + part[1][lane]) + (part[2][lane] + part[3][lane]) : 0.0f;
#pragma unroll
  for (int k = 0; k <= 2 * N; ++k) all[k] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), k));
  float dg = 0.0f;
  if (counts) {
    float left = 1.0f;      // from the first state to step s
#pragma unroll
    for (int s = 0; s < N; ++s) {      // (a step behind the sequence has a decay of one and rows of zeros)
      left *= w[s];
      dg += s >= t ? left * all[s] : 0.0f;
    }
    dg = last ? fmaf(left, all[2 * N], dg) : dg;
    left = 1.0f;      // from step r to the last
#pragma unroll
    for (int r = N - 1; r >= 0; --r) {
      dg += last && r < t ? left * all[N + r] : 0.0f;
      left *= w[r];
    }
#pragma unroll
    for (int s = 1; s < N; ++s)
#pragma unroll
      for (int r = 0; r < s; ++r) dg += r < t && t <= s && s < n ? pairs[s][r] : 0.0f;
  }
  if (!G.sums) {
    if (t < A.steps) G.dg[(b * A.steps + t) * A.heads + h] = dg;
    return;
  }
  const double sum = wave_sum((double)dg);
  if (lane == 0) G.dg[h * A.batch + b] = (float)sum;
}
// One head's sum over all sequences and pieces.
__global__ __launch_bounds__(256) void k_linear_gate_sums(const float* parts, int64_t count, float* dg) {
  __shared__ double part[4];
  double x = 0.0;
  for (int64_t i = threadIdx.x; i < count; i += 256) x += (double)parts[blockIdx.x * count + i];
  x = wave_sum(x);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
  __syncthreads();
  if (threadIdx.x == 0) dg[blockIdx.x] = (float)((part[0] + part[1]) + (part[2] + part[3]));
}

#endif

// A gradient of all heads, fp32 [batch][steps][heads][dim], added up over those that share one.
template <class T>
__global__ __launch_bounds__(256) void k_linear_share(const float* x, void* out, int64_t rows, int64_t steps, int shared, int share, int dim,
                                                      int64_t seq, int64_t step, int64_t head) {
  const int64_t count = rows * shared * dim;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < count; i += (int64_t)gridDim.x * 256) {
    const int64_t e = i % dim, at = i / dim, h = at % shared, row = at / shared;
    const float* p = x + (row * shared + h) * share * dim + e;
    float sum = 0.0f;
    for (int j = 0; j < share; ++j) sum += p[(int64_t)j * dim];
    ((T*)out)[row / steps * seq + row % steps * step + h * head + e] = from_float<T>(sum);
  }
}

}  // namespace choco
