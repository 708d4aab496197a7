// Gated linear recurrence h_t = a_t h_{t-1} + (1 - a_t) u_t, a = sigmoid(f), y = sigmoid(o) h, and its backward
// pass (device code).
#pragma once

#include "choco_types.h"

namespace choco {

constexpr int kSaveSteps = 16;   // the forward pass keeps the state before every so many steps

struct RecurArgs {
  const void *f, *u, *o, *dy;
  void *y, *df, *du, *dout;
  const float *h0, *dlast;
  float *h_last, *dh0;
  float* saved;             // [ceil(steps / kSaveSteps)][batch][dim]
  const int32_t* lengths;
  int64_t batch, steps, dim;
  int64_t f_seq, f_step, u_seq, u_step, o_seq, o_step, y_seq, y_step;
  int64_t df_seq, df_step, du_seq, du_step, do_seq, do_step;
};

// sigmoid(x) and sigmoid(-x) = 1 - sigmoid(x), neither by a difference: exp(-|x|) <= 1 cannot overflow and the
// smaller of the two keeps its relative accuracy (about 2^-22).
__device__ __forceinline__ void gate(float x, float& up, float& down) {
  const float e = __expf(-fabsf(x));
  const float r = __builtin_amdgcn_rcpf(1.0f + e);
  up = x >= 0.0f ? r : e * r;
  down = x >= 0.0f ? e * r : r;
  if (x != x) up = down = x;
}

__device__ __forceinline__ int64_t steps_of(const RecurArgs& A, int64_t b) {
  if (!A.lengths) return A.steps;
  const int64_t n = A.lengths[b];
  return n < 0 ? 0 : n > A.steps ? A.steps : n;
}

// A lane per channel, step after step.
template <class T, bool GATED>
__global__ __launch_bounds__(256) void k_recur(RecurArgs A) {
  const uint32_t strips = (uint32_t)((A.dim + 255) / 256);
  const int64_t b = blockIdx.x / strips, c = (int64_t)(blockIdx.x % strips) * 256 + threadIdx.x;
  if (c >= A.dim) return;
  const int64_t len = steps_of(A, b);
  const T* f = (const T*)A.f + b * A.f_seq + c;
  const T* u = (const T*)A.u + b * A.u_seq + c;
  const T* o = GATED ? (const T*)A.o + b * A.o_seq + c : nullptr;
  T* y = (T*)A.y + b * A.y_seq + c;
  float h = A.h0 ? A.h0[b * A.dim + c] : 0.0f;
  for (int64_t t = 0; t < A.steps; ++t) {
    if (A.saved && t % kSaveSteps == 0) A.saved[((t / kSaveSteps) * A.batch + b) * A.dim + c] = h;
    float out = 0.0f;
    if (t < len) {
      float a, i;
      gate(to_float(f[t * A.f_step]), a, i);
      h = a * h + i * to_float(u[t * A.u_step]);
      out = h;
      if (GATED) {
        float s, r;
        gate(to_float(o[t * A.o_step]), s, r);
        out = s * h;
      }
    }
    y[t * A.y_step] = from_float<T>(out);
  }
  if (A.h_last) A.h_last[b * A.dim + c] = h;
}

// A lane per channel; from the last steps back, kSaveSteps at a time, whose states are computed again.
template <class T, bool GATED>
__global__ __launch_bounds__(256) void k_recur_back(RecurArgs A) {
  const uint32_t strips = (uint32_t)((A.dim + 255) / 256);
  const int64_t b = blockIdx.x / strips, c = (int64_t)(blockIdx.x % strips) * 256 + threadIdx.x;
  if (c >= A.dim) return;
  const int64_t len = steps_of(A, b);
  const T* f = (const T*)A.f + b * A.f_seq + c;
  const T* u = (const T*)A.u + b * A.u_seq + c;
  const T* o = GATED ? (const T*)A.o + b * A.o_seq + c : nullptr;
  const T* dy = (const T*)A.dy + b * A.y_seq + c;
  T* df = (T*)A.df + b * A.df_seq + c;
  T* du = (T*)A.du + b * A.du_seq + c;
  T* dout = GATED ? (T*)A.dout + b * A.do_seq + c : nullptr;
  float e = A.dlast ? A.dlast[b * A.dim + c] : 0.0f;   // a_{t+1} e_{t+1}
  for (int64_t k = (A.steps + kSaveSteps - 1) / kSaveSteps - 1; k >= 0; --k) {
    const int64_t t0 = k * kSaveSteps;
    float h[kSaveSteps + 1];
    h[0] = A.saved[(k * A.batch + b) * A.dim + c];
#pragma unroll
    for (int j = 0; j < kSaveSteps; ++j) {
      h[j + 1] = h[j];
      if (t0 + j < len) {
        float a, i;
        gate(to_float(f[(t0 + j) * A.f_step]), a, i);
        h[j + 1] = a * h[j] + i * to_float(u[(t0 + j) * A.u_step]);
      }
    }
#pragma unroll
    for (int j = kSaveSteps - 1; j >= 0; --j) {
      const int64_t t = t0 + j;
      if (t >= A.steps) continue;
      float gf = 0.0f, gu = 0.0f, go = 0.0f;
      if (t < len) {
        float a, i, s = 1.0f, r = 0.0f;
        gate(to_float(f[t * A.f_step]), a, i);
        const float d = to_float(dy[t * A.y_step]);
        if (GATED) gate(to_float(o[t * A.o_step]), s, r);
        e += d * s;
        go = d * h[j + 1] * s * r;
        gu = e * i;
        gf = e * (h[j] - to_float(u[t * A.u_step])) * a * i;
        e *= a;
      }
      df[t * A.df_step] = from_float<T>(gf);
      du[t * A.du_step] = from_float<T>(gu);
      if (GATED) dout[t * A.do_step] = from_float<T>(go);
    }
  }
  if (A.dh0) A.dh0[b * A.dim + c] = e;
}

}  // namespace choco
