// Linear attention with a decay for each head, S_t = e^g_t S_{t-1} + k_t v_t^T, y_t = S_t^T q_t, and its backward pass (device code).
//
// Every part of the work is one of four passes of one kind: for a sequence and head, through its steps forwards or backwards,
//   S <- w S + b c^T,   out = S^T a
//   y:  a, b, c = q, k, v              dq: dy, v, k     (the same states transposed)
//   dk: v, dy, q   backwards           dv: k, q, dy     backwards
// where w = e^g_t forwards, and backwards the next step's, 1 at a sequence's last.
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
  float* dots;              // [slices][batch * heads][steps]
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
// A workgroup takes a slice of columns, a lane a column, a wave a quarter of the state's rows.
constexpr int kLinearStage = 8;     // steps whose a and b are in LDS at a time

template <class T, int R>
__global__ __launch_bounds__(256) void k_linear_steps(LinearArgs A, LinearPass P) {
  __shared__ float sa[kLinearStage][4 * R], sb[kLinearStage][4 * R], part[2][4][64];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int slices = (P.dc + kLinearSlice - 1) / kLinearSlice, slice = blockIdx.x % slices;
  const int64_t bh = blockIdx.x / slices, b = bh / A.heads;
  const int h = (int)(bh % A.heads), col = slice * kLinearSlice + lane, row = wave * R;
  const bool in = col < P.dc;
  const int64_t len = steps_of(A, b), state = (int64_t)P.da * P.dc;
  const T* pa = (const T*)P.a + b * P.a_seq + (h / P.a_share) * P.a_head;
  const T* pb = (const T*)P.b + b * P.b_seq + (h / P.b_share) * P.b_head;
  const T* pc = (const T*)P.c + b * P.c_seq + (h / P.c_share) * P.c_head;
  const int64_t out = b * P.out_seq + h * P.out_head + col;
  float s[R];
#pragma unroll
  for (int r = 0; r < R; ++r)
    s[r] = P.first && in && row + r < P.da ? P.first[bh * P.first_of * state + (int64_t)(row + r) * P.state_a + (int64_t)col * P.state_c] : 0.0f;
  const auto keep = [&](float* to, float w) {
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (in && row + r < P.da) to[(int64_t)(row + r) * P.state_a + (int64_t)col * P.state_c] = s[r] * w;
  };
  for (int64_t i0 = 0; i0 < len; i0 += kLinearStage) {
    const int n = len - i0 < kLinearStage ? (int)(len - i0) : kLinearStage;
    __syncthreads();
    for (int e = threadIdx.x; e < n * P.da; e += 256) {
      const int i = e / P.da, j = e % P.da;
      const int64_t t = P.back ? len - 1 - (i0 + i) : i0 + i;
      sa[i][j] = to_float(pa[t * P.a_step + j]);
      sb[i][j] = to_float(pb[t * P.b_step + j]);
    }
    __syncthreads();
    for (int i = 0; i < n; ++i) {
      const int64_t t = P.back ? len - 1 - (i0 + i) : i0 + i;
      if (P.kept && t % kLinearSave == 0) keep(P.kept + (bh * P.kept_of + t / kLinearSave) * state, 1.0f);
      float w = 1.0f;
      if (!P.back) w = linear_decay(log_gate(A, b, t, h));
      else if (t + 1 < len) w = linear_decay(log_gate(A, b, t + 1, h));
      const float c = in ? to_float(pc[t * P.c_step + col]) : 0.0f;
      float sum = 0.0f;
#pragma unroll
      for (int r = 0; r < R; ++r)
        if (row + r < P.da) {
          s[r] = fmaf(sb[i][row + r], c, s[r] * w);
          sum = fmaf(sa[i][row + r], s[r], sum);
        }
      part[i & 1][wave][lane] = sum;
      __syncthreads();
      if (wave == (i & 3)) {
        const float y = (part[i & 1][0][lane] + part[i & 1][1][lane]) + (part[i & 1][2][lane] + part[i & 1][3][lane]);
        if (in) store_result<T>(P, out + t * P.out_step, y);
        if (P.dots) {
          float d = in ? y * to_float(((const T*)P.x)[b * P.x_seq + t * P.x_step + (h / P.x_share) * P.x_head + col]) : 0.0f;
          for (int o = 32; o; o >>= 1) d += __shfl_xor(d, o);
          if (lane == 0) P.dots[((int64_t)slice * A.batch * A.heads + bh) * A.steps + t] = d;
        }
      }
    }
  }
  if (in)
    for (int64_t t = len + wave; t < A.steps; t += 4) store_result<T>(P, out + t * P.out_step, 0.0f);
  if (P.kept) keep(P.kept + (bh * P.kept_of + (len + kLinearSave - 1) / kLinearSave) * state, 1.0f);
  if (P.last) keep(P.last + bh * state, P.back && len > 0 ? linear_decay(log_gate(A, b, 0, h)) : 1.0f);
}

// ---- in chunks ----
// With c_t the sum of the logarithms of w since the chunk began and S the state before it,
//   out_t = e^c_t S^T a_t + sum over s <= t of e^(c_t - c_s) (a_t b_s) c_s,   S <- e^c_end S + sum of e^(c_end - c_s) b_s c_s^T:
// four products of matrices, on the matrix cores, out^T = S^T a^T + c^T P^T with P^T = (b a^T) weighted.  A wave takes 16 columns of the result
// and holds the state's in registers as the matrix cores leave a product: a lane has a column's rows 4 g to 4 g + 3 of every 16.
// That is how the cores take a left operand whose inner index is the row, so neither S nor P^T goes through LDS; every wave makes
// P^T of its own.  Differences of c are taken of c in two floats: a start-over leaves the steps behind it exact.
//
// Entries of 32 bits (and of fp16, taken as 32 bits) go to the fp32 matrix instruction.  Those of bf16 are operands as they are; what is fp32
// by nature (P, S, weighted c) enters as a sum of bf16 numbers, two of them (2^-17) for a result of 16 bits, three (2^-25) for states
// and wherever the result also goes into fp32 sums.
constexpr int kChunk = 64;
constexpr float kLog2Least = -300.0f;     // stands for -infinity: less than any difference that counts

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

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
// fp32 numbers of an operand as so many operands that add up to it.
template <class Core, int N>
__device__ __forceinline__ void pieces_of(const f32x4 (&x)[Operand<Core>::kTiles], typename Operand<Core>::Frag (&p)[N]) {
  if constexpr (std::is_same_v<Core, float>) {
    static_assert(N == 1);
    p[0] = x[0];
  } else {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float left = x[t][r];
#pragma unroll
        for (int i = 0; i < N; ++i) {
          p[i][4 * t + r] = (bf16_t)left;
          if (i + 1 < N) left -= (float)p[i][4 * t + r];
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
  int32_t vec_a, vec_b, vec_c, vec_out;   // entries that a load or store takes
};

// One XCD's workgroups take neighbouring parts of the work: slices of the same head share their a and b in its L2.
__device__ __forceinline__ uint32_t by_xcd(uint32_t block, uint32_t blocks) {
  const uint32_t x = block & 7, each = blocks >> 3, more = blocks & 7;
  return x * each + min(x, more) + (block >> 3);
}

template <class Core, int DA>
struct ChunkShared {
  static constexpr int kPad = 16 / sizeof(Core);
  static constexpr bool kTurned = sizeof(Core) == 2;      // b by columns as well
  static constexpr int kTurnedRow = kChunk + 4;
  Core a[kChunk][DA + kPad], b[kChunk][DA + kPad];
  Core c[kChunk][kLinearSlice + kPad];
  Core turned[kTurned ? DA : 1][kTurned ? kTurnedRow : 1];
  float c_high[kChunk], c_low[kChunk], to_end[kChunk], dots[4][kChunk];
};

// A chunk's rows of one array on their way from memory to LDS, in a thread's registers: they are asked for while the chunk before is
// worked on.  A thread takes R rows of 8 entries at a time.  R = 4, for rows that are also laid out by columns: 16 neighbouring lanes take
// 4 x 4 of these, which meets all banks both ways.
template <class In, class Core, int W, int R>
struct Staged {
  static constexpr int kWords = 8 * sizeof(In) / 4;      // of 8 entries
  static constexpr int kAll = kChunk / R * (W / 8), kUnits = (kAll + 255) / 256;
  uint32_t x[kUnits][R][kWords];

  static __device__ __forceinline__ void place(int i, int& row, int& col) {
    const int u = i * 256 + (int)threadIdx.x;
    if constexpr (R == 1) {
      row = u / (W / 8);
      col = u % (W / 8) * 8;
    } else {
      static_assert(kChunk / R == 16);
      row = ((u & 3) | (u >> 2 & 12)) * R;
      col = ((u >> 2 & 3) | (u >> 6) * 4) * 8;
    }
  }
  // `width` entries of a row are there; of rows that `time` says -1, none.  vec: entries that a load takes, 16 bytes, or 2 or 1.
  template <class Time>
  __device__ __forceinline__ void load(const In* from, int64_t step, int width, int vec, Time time) {
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
      int row, col;
      place(i, row, col);
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const int64_t t = row + r < kChunk && col < W ? time(row + r) : -1;
        const In* p = from + t * step + col;
        const int have = t < 0 ? 0 : width - col;
#pragma unroll
        for (int w = 0; w < kWords; ++w) x[i][r][w] = 0;
        if (vec * sizeof(In) == 16) {
#pragma unroll
          for (int w = 0; w < kWords; w += 4)
            if (have > w * (int)(4 / sizeof(In))) {
              const uint4 v = *reinterpret_cast<const uint4*>(p + w * (4 / sizeof(In)));
              x[i][r][w] = v.x; x[i][r][w + 1] = v.y; x[i][r][w + 2] = v.z; x[i][r][w + 3] = v.w;
            }
        } else if (sizeof(In) == 4 || vec == 2) {
#pragma unroll
          for (int w = 0; w < kWords; ++w)
            if (have > w * (int)(4 / sizeof(In))) x[i][r][w] = *reinterpret_cast<const uint32_t*>(p + w * (4 / sizeof(In)));
        } else {
#pragma unroll
          for (int w = 0; w < kWords; ++w) {
            const uint16_t* half = reinterpret_cast<const uint16_t*>(p);
            if (have > 2 * w) x[i][r][w] = half[2 * w];
            if (have > 2 * w + 1) x[i][r][w] |= (uint32_t)half[2 * w + 1] << 16;
          }
        }
      }
    }
  }
  __device__ __forceinline__ float at(int i, int r, int e) const {
    if constexpr (sizeof(In) == 4) return __uint_as_float(x[i][r][e]);
    else return entry<In>(x[i][r][e / 2], e & 1);
  }
  template <int STRIDE>
  __device__ __forceinline__ void store(Core (&to)[kChunk][STRIDE]) const {
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
      int row, col;
      place(i, row, col);
      if (row >= kChunk || col >= W) continue;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        if constexpr (sizeof(Core) == 2) {
          *reinterpret_cast<uint4*>(&to[row + r][col]) = uint4{x[i][r][0], x[i][r][1], x[i][r][2], x[i][r][3]};
        } else {
          *reinterpret_cast<f32x4*>(&to[row + r][col]) = f32x4{at(i, r, 0), at(i, r, 1), at(i, r, 2), at(i, r, 3)};
          *reinterpret_cast<f32x4*>(&to[row + r][col + 4]) = f32x4{at(i, r, 4), at(i, r, 5), at(i, r, 6), at(i, r, 7)};
        }
      }
    }
  }
  // ... by columns: four steps of an entry are 8 bytes
  template <int STRIDE>
  __device__ __forceinline__ void store_turned(Core (*to)[STRIDE]) const {
    static_assert(R == 4 && sizeof(Core) == 2);
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
      int row, col;
      place(i, row, col);
      if (col >= W) continue;
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
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

// STATE: only the segments' own contributions to the state, and their logarithms' sums.
// (workgroups of a compute unit: as its LDS holds, two at least where it holds them)
template <class Core, int DA>
constexpr int kChunkGroups = sizeof(ChunkShared<Core, DA>) * 2 > 163840 ? 1 : 2;
template <class In, class Core, int DA, int N_OUT, int N_STATE, bool STATE>
__global__ __launch_bounds__(256, (kChunkGroups<Core, DA>)) void k_linear_chunks(LinearArgs A, LinearPass P, LinearChunks C) {
  typedef Operand<Core> Op;
  typedef typename Op::Frag Frag;
  constexpr int kJ = DA / Op::kInner, kT = Op::kTiles, kS = kChunk / Op::kInner;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  ChunkShared<Core, DA>& S = *reinterpret_cast<ChunkShared<Core, DA>*>(lds);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, l = lane & 15, g = lane >> 4;
  const uint32_t at = by_xcd(blockIdx.x, C.blocks);
  const int slice = at % C.slices, segment = at / C.slices % C.segments;
  const int64_t bh = at / C.slices / C.segments, b = bh / A.heads, len = steps_of(A, b), entries = (int64_t)P.da * P.dc;
  const int h = (int)(bh % A.heads), col = slice * kLinearSlice + 16 * wave;     // the wave's first column
  const In* pa = (const In*)P.a + b * P.a_seq + (h / P.a_share) * P.a_head;
  const In* pb = (const In*)P.b + b * P.b_seq + (h / P.b_share) * P.b_head;
  const In* pc = (const In*)P.c + b * P.c_seq + (h / P.c_share) * P.c_head + slice * kLinearSlice;
  const In* px = (const In*)P.x + b * P.x_seq + (h / P.x_share) * P.x_head;
  const int64_t out = b * P.out_seq + h * P.out_head;
  const int64_t begin = (int64_t)segment * C.chunks * kChunk;
  const int64_t end = segment + 1 == C.segments ? A.steps : begin + (int64_t)C.chunks * kChunk;
  const int in_slice = min(P.dc - slice * kLinearSlice, kLinearSlice);

  f32x4 state[kJ * kT];       // rows 16 j + 4 g + r of column `col + l`
  const float* from = STATE ? nullptr : C.states ? C.states + (bh * C.states_of + segment) * entries : P.first ? P.first + bh * P.first_of * entries : nullptr;
  const bool column = col + l < P.dc;
#pragma unroll
  for (int j = 0; j < kJ * kT; ++j)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int row = 16 * j + 4 * g + r;
      state[j][r] = from && column && row < P.da ? from[(int64_t)row * P.state_a + (int64_t)(col + l) * P.state_c] : 0.0f;
    }
  const auto keep = [&](float* to, float w) {
#pragma unroll
    for (int j = 0; j < kJ * kT; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = 16 * j + 4 * g + r;
        if (column && row < P.da) to[(int64_t)row * P.state_a + (int64_t)(col + l) * P.state_c] = state[j][r] * w;
      }
  };
  double total = 0.0;

  const int64_t inside = min(end, len);       // steps of the segment that are in the sequence end here
  const int chunks = inside > begin ? (int)((inside - begin + kChunk - 1) / kChunk) : 0;
  typedef ChunkShared<Core, DA> Shared;
  Staged<In, Core, DA, 1> next_a;
  Staged<In, Core, DA, Shared::kTurned ? 4 : 1> next_b;
  Staged<In, Core, kLinearSlice, 1> next_c;
  float next_g = 0.0f;
  const auto begin_of = [&](int i) { return begin + (int64_t)(P.back ? chunks - 1 - i : i) * kChunk; };
  // the step of a row of a chunk, -1 behind the sequence
  const auto step_of = [&](int64_t t0, int row) -> int64_t {
    const int64_t t = t0 + (P.back ? kChunk - 1 - row : row);
    return t < inside ? t : -1;
  };
  const auto ask = [&](int i) {
    const int64_t t0 = begin_of(i);
    const auto time = [&](int row) { return step_of(t0, row); };
    if (!STATE) next_a.load(pa, P.a_step, P.da, C.vec_a, time);
    next_b.load(pb, P.b_step, P.da, C.vec_b, time);
    next_c.load(pc, P.c_step, in_slice, C.vec_c, time);
    if (wave == 0) {
      const int64_t t = step_of(t0, lane) + (P.back ? 1 : 0);
      next_g = step_of(t0, lane) >= 0 && t < len ? log_gate(A, b, t, h) : 0.0f;
    }
  };
  if (chunks > 0) ask(0);
  for (int i = 0; i < chunks; ++i) {
    const int64_t t0 = begin_of(i);
    const auto time = [&](int row) { return step_of(t0, row); };
    if (!STATE && P.kept && t0 % kLinearSave == 0) keep(P.kept + (bh * P.kept_of + t0 / kLinearSave) * entries, 1.0f);
    __syncthreads();
    if (!STATE) next_a.store(S.a);
    if constexpr (Shared::kTurned) next_b.store_turned(S.turned);
    if (!STATE || !Shared::kTurned) next_b.store(S.b);
    next_c.store(S.c);
    if (wave == 0) {      // the logarithms' sums
      const double x = sums_to(next_g < kLinearLeast ? (double)kLog2Least : (double)next_g * 1.4426950408889634);
      const double all = __shfl(x, 63);
      S.c_high[lane] = (float)x;
      S.c_low[lane] = (float)(x - (double)(float)x);
      S.to_end[lane] = __builtin_amdgcn_exp2f((float)(all - x));
      total += all;
    }
    if (i + 1 < chunks) ask(i + 1);
    __syncthreads();
    const bool busy = 16 * wave < in_slice;
    if (busy) [&] {
    Frag cf[kS];       // column l's entries, a lane's steps
#pragma unroll
    for (int s = 0; s < kS; ++s)
#pragma unroll
      for (int t = 0; t < kT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) cf[s][4 * t + r] = S.c[16 * (s * kT + t) + 4 * g + r][16 * wave + l];
    if constexpr (!STATE) {
      Frag before[kJ][N_OUT];
#pragma unroll
      for (int j = 0; j < kJ; ++j) pieces_of<Core, N_OUT>(*(const f32x4(*)[kT])&state[j * kT], before[j]);
      // (steps behind the sequence are its first rows backwards, its last ones forwards)
      const int there = (int)min((int64_t)kChunk, inside - t0), t_first = P.back ? (kChunk - there) / 16 : 0, t_end = P.back ? 4 : (there + 15) / 16;
#pragma unroll 1
      for (int t = t_first; t < t_end; ++t) {
        const float high = S.c_high[16 * t + l], low = S.c_low[16 * t + l];
        const float here = __builtin_amdgcn_exp2f(high + low);
        Frag q[kJ];
        f32x4 y = {};
#pragma unroll
        for (int j = 0; j < kJ; ++j) {
          q[j] = Op::load(&S.a[16 * t + l][0], j, g);
#pragma unroll
          for (int n = N_OUT - 1; n >= 0; --n) y = Op::mma(before[j][n], q[j], y);
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) y[r] *= here;
#pragma unroll
        for (int s = 0; s < kS; ++s) {
          if (s * kT > t) continue;
          f32x4 w[kT];
#pragma unroll
          for (int u = 0; u < kT; ++u) {
            const int from = s * kT + u;      // steps 16 from + 4 g + r
            w[u] = f32x4{};
            if (from > t) continue;
#pragma unroll
            for (int j = 0; j < kJ; ++j) w[u] = Op::mma(Op::load(&S.b[16 * from + l][0], j, g), q[j], w[u]);
            const f32x4 high_s = *(const f32x4*)&S.c_high[16 * from + 4 * g], low_s = *(const f32x4*)&S.c_low[16 * from + 4 * g];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const float weighted = w[u][r] * __builtin_amdgcn_exp2f((high - high_s[r]) + (low - low_s[r]));
              w[u][r] = from < t || 4 * g + r <= l ? weighted : 0.0f;
            }
          }
          Frag p[N_OUT];
          pieces_of<Core, N_OUT>(w, p);
#pragma unroll
          for (int n = N_OUT - 1; n >= 0; --n) y = Op::mma(cf[s], p[n], y);
        }
        // rows of the result: step 16 t + l, columns 4 g to 4 g + 3 of the wave's
        const int64_t when = time(16 * t + l);
        const int first = col + 4 * g;
        if (when >= 0) {
          const int64_t to = out + when * P.out_step + first;
          if (C.vec_out == 4 && first < P.dc) {
            const float x[4] = {y[0], y[1], y[2], y[3]};
            if (P.wide) store_floats<float, 4>((float*)P.out + to, x);
            else store_floats<In, 4>((In*)P.out + to, x);
          } else {
#pragma unroll
            for (int r = 0; r < 4; ++r)
              if (first + r < P.dc) store_result<In>(P, to + r, y[r]);
          }
        }
        if (P.dots) {
          float d = 0.0f;
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (when >= 0 && first + r < P.dc) d = fmaf(y[r], to_float(px[when * P.x_step + first + r]), d);
          d += __shfl_xor(d, 16);
          d += __shfl_xor(d, 32);
          if (g == 0) S.dots[wave][16 * t + l] = d;
        }
      }
      if (i + 1 == chunks && (C.states || !P.last) && !P.kept) return;      // nobody reads the state
    }
    const float all = __builtin_amdgcn_exp2f(S.c_high[kChunk - 1] + S.c_low[kChunk - 1]);
#pragma unroll
    for (int j = 0; j < kJ * kT; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) state[j][r] *= all;
#pragma unroll
    for (int s = 0; s < kS; ++s) {
      f32x4 w[kT];
#pragma unroll
      for (int t = 0; t < kT; ++t) {
        const f32x4 left = *(const f32x4*)&S.to_end[16 * (s * kT + t) + 4 * g];
#pragma unroll
        for (int r = 0; r < 4; ++r) w[t][r] = (float)cf[s][4 * t + r] * left[r];
      }
      Frag p[N_STATE];
      pieces_of<Core, N_STATE>(w, p);
#pragma unroll
      for (int j = 0; j < kJ * kT; ++j) {
        Frag rows;
        if constexpr (ChunkShared<Core, DA>::kTurned) {
          rows = Op::load(&S.turned[16 * j + l][0], s, g);
        } else {
#pragma unroll
          for (int r = 0; r < 4; ++r) rows[r] = S.b[16 * s + 4 * g + r][16 * j + l];
        }
#pragma unroll
        for (int n = N_STATE - 1; n >= 0; --n) state[j] = Op::mma(rows, p[n], state[j]);
      }
    }
    }();
    if (!STATE && P.dots) {
      __syncthreads();
      if (wave == 0 && time(lane) >= 0) {
        float d = S.dots[0][lane];
        for (int w = 1; w < (in_slice + 15) / 16; ++w) d += S.dots[w][lane];
        P.dots[((int64_t)slice * A.batch * A.heads + bh) * A.steps + time(lane)] = d;
      }
    }
  }
  if constexpr (STATE) {
    keep(C.states + (bh * C.states_of + segment) * entries, 1.0f);
    if (slice == 0 && threadIdx.x == 0) C.totals[bh * C.segments + segment] = total;
    return;
  }
  // zeros behind the sequence
  const int64_t zero = max(begin, len);
  const int width = in_slice;
  for (int64_t e = threadIdx.x; e < (end - zero) * width; e += 256)
    store_result<In>(P, out + (zero + e / width) * P.out_step + slice * kLinearSlice + e % width, 0.0f);
  if (P.kept && (len == 0 ? segment == 0 : begin < len && len <= end))
    keep(P.kept + (bh * P.kept_of + (len + kLinearSave - 1) / kLinearSave) * entries, 1.0f);
  if (P.last && !C.states) keep(P.last + bh * entries, P.back && len > 0 ? linear_decay(log_gate(A, b, 0, h)) : 1.0f);
}

// From the segments' own contributions to the states before them, in place, and the last one.
__global__ __launch_bounds__(256) void k_linear_scan(LinearArgs A, float* states, const double* totals, int segments, int64_t entries, const float* first,
                                                     float* last, bool back) {
  const int64_t each = (entries + 255) / 256, count = A.batch * A.heads * each;
  for (int64_t block = blockIdx.x; block < count; block += gridDim.x) {
    const int64_t bh = block / each, b = bh / A.heads, e = block % each * 256 + threadIdx.x;
    if (e >= entries) continue;
    float s = first ? first[bh * entries + e] : 0.0f;
    float* p = states + bh * segments * entries + e;
    for (int i = 0; i < segments; ++i) {
      const int at = back ? segments - 1 - i : i;
      const float own = p[at * entries];
      p[at * entries] = s;
      s = fmaf(s, __builtin_amdgcn_exp2f((float)totals[bh * segments + at]), own);
    }
    if (last) last[bh * entries + e] = back && steps_of(A, b) > 0 ? s * linear_decay(log_gate(A, b, 0, (int)(bh % A.heads))) : s;
  }
}

// ---- the gates' gradient ----
// dg_t = sum over s >= t of (q_s dq_s - k_s dk_s) up to any later step u, and what goes from before u past it, <E_u, S_u>: pieces of
// kLinearSave steps, each with the states at its end, so that the differences' errors do not add up over a sequence.
struct LinearGates {
  const float *q_dots, *k_dots, *saved, *later, *dlast;   // later: states that the backwards passes have before their pieces
  int64_t saved_of, later_of;
  int32_t q_slices, k_slices, state;
  float* dg;       // [batch][steps][heads], or the pieces' sums [heads][batch * pieces]
  int64_t pieces;
  bool sums;
};

__device__ __forceinline__ double wave_sum(double x) {
  for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o);
  return x;
}

__global__ __launch_bounds__(kLinearSave) void k_linear_gates(LinearArgs A, LinearGates G) {
  __shared__ double part[8];
  const int64_t bh = blockIdx.x / G.pieces, piece = blockIdx.x % G.pieces, b = bh / A.heads;
  const int h = (int)(bh % A.heads), wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t len = steps_of(A, b), t = piece * kLinearSave + threadIdx.x, end = (piece + 1) * kLinearSave;
  const bool in = t < len;
  double x = 0.0;
  if (in) {
    const int64_t all = A.batch * A.heads;
    for (int s = 0; s < G.q_slices; ++s) x += (double)G.q_dots[(s * all + bh) * A.steps + t];
    for (int s = 0; s < G.k_slices; ++s) x -= (double)G.k_dots[(s * all + bh) * A.steps + t];
  }
  for (int o = 1; o < 64; o <<= 1) {      // from this step to the wave's last
    const double y = __shfl_down(x, o);
    if (lane + o < 64) x += y;
  }
  // what goes past the piece's end
  double past = 0.0;
  const bool whole = end < len;
  const float* later = whole ? G.later + (bh * G.later_of + piece) * G.state : G.dlast ? G.dlast + bh * G.state : nullptr;
  if (later && piece * kLinearSave < len) {
    const float* s = G.saved + (bh * G.saved_of + piece + 1) * G.state;
    for (int i = threadIdx.x; i < G.state; i += kLinearSave) past += (double)later[i] * (double)s[i];
    if (whole) past *= (double)linear_decay(log_gate(A, b, end, h));
  }
  past = wave_sum(past);
  if (lane == 0) {
    part[wave] = x;
    part[4 + wave] = past;
  }
  __syncthreads();
  x += (part[4] + part[5]) + (part[6] + part[7]);
  for (int w = wave + 1; w < 4; ++w) x += part[w];
  float dg = (float)x;
  if (!in || log_gate(A, b, t, h) < kLinearLeast) dg = 0.0f;
  if (!G.sums) {
    if (t < A.steps) G.dg[(b * A.steps + t) * A.heads + h] = dg;
    return;
  }
  __syncthreads();
  const double sum = wave_sum((double)dg);
  if (lane == 0) part[wave] = sum;
  __syncthreads();
  if (threadIdx.x == 0) G.dg[h * A.batch * G.pieces + b * G.pieces + piece] = (float)((part[0] + part[1]) + (part[2] + part[3]));
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
