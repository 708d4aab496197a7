// Linear attention with a decay for each head, S_t = e^g_t S_{t-1} + k_t v_t^T, y_t = S_t^T q_t, and its backward pass (device code).
//
// Every part of the work is one of four passes of one kind: for a sequence and head, through its steps forwards or backwards,
//   S <- w S + b c^T,   out = S^T a
//   y:  a, b, c = q, k, v              dq: dy, v, k     (the same states transposed)
//   dk: v, dy, q   backwards           dv: k, q, dy     backwards
// where w = e^g_t forwards, and backwards the next step's, 1 at a sequence's last.
#pragma once

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
  float* kept;              // states before the pass' pieces of kLinearSave steps, of each sequence and head `kept_of`; forwards and the last
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
      if (P.kept && (P.back ? t == len - 1 || t % kLinearSave == kLinearSave - 1 : t % kLinearSave == 0))
        keep(P.kept + (bh * P.kept_of + t / kLinearSave) * state, 1.0f);
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
  if (P.kept && !P.back) keep(P.kept + (bh * P.kept_of + (len + kLinearSave - 1) / kLinearSave) * state, 1.0f);
  if (P.last) keep(P.last + bh * state, P.back && len > 0 ? linear_decay(log_gate(A, b, 0, h)) : 1.0f);
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
