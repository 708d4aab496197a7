// Gated linear recurrence h_t = a_t h_{t-1} + (1 - a_t) u_t, a = sigmoid(f), y = sigmoid(o) h, and its backward
// pass (device code).
#pragma once

#include <type_traits>

#include "choco_types.h"

namespace choco {

constexpr int kSaveSteps = 16;   // the forward pass keeps the state before every so many steps

#ifndef RW
#define RW 8
#endif
constexpr int kRecurWaves = RW;   // most waves of a workgroup
constexpr int kMaxSegments = 64; // most pieces that a sequence is split into

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
  float2* parts;            // [segments][batch][dim], see k_recur_part; null: one segment
  int64_t segment_steps;    // a multiple of kSaveSteps * (waves of a workgroup)
  uint32_t strips, segments;
};

// sigmoid(x) and 1 - sigmoid(x), the smaller of the two not by a difference: the exponential's argument is rounded to
// |x| 2^-24, the rest is good to a few 2^-24.  exp(-x) may overflow: up is then 0 and down 1.
__device__ __forceinline__ void gate(float x, float& up, float& down) {
  const float e = __builtin_amdgcn_exp2f(x * -1.44269504f);
  up = __builtin_amdgcn_rcpf(1.0f + e);
  down = x >= 0.0f ? e * up : 1.0f - up;
}
__device__ __forceinline__ float gate(float x) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x * -1.44269504f));
}

__device__ __forceinline__ int64_t steps_of(const RecurArgs& A, int64_t b) {
  if (!A.lengths) return A.steps;
  const int64_t n = A.lengths[b];
  return n < 0 ? 0 : n > A.steps ? A.steps : n;
}

// How the work is split.  A strip is 64 * V channels of one sequence, V channels a lane.  A workgroup takes a strip (of
// one segment of the sequence) and goes through its steps in rounds, kSaveSteps of a round for each wave: a wave loads
// its steps at once, reduces them to the map h -> A h + H, the waves exchange these maps through LDS, and each applies
// the maps before its own to the state and goes through its steps, which are still in registers, once more.  Everything
// is read once, and the chain from step to step is as long as a round has waves, not steps.
// Sequences with too few strips to fill the chip are split into segments, whose maps a first kernel (k_recur_part)
// computes: f and u (backward: f, o and dy) are then read twice.
struct RecurPlace {
  int64_t b, strip, len, begin, end;   // sequence, first channel of the strip, its length, the segment's steps
  uint32_t segment;
  int lane;                        // first channel of the lane in the strip (of one that has none: 0, and it writes nothing)
  bool in;                         // the lane has channels
};

template <int V>
__device__ __forceinline__ RecurPlace recur_place(const RecurArgs& A) {
  RecurPlace P;
  const uint32_t rest = blockIdx.x / A.strips, strip = blockIdx.x % A.strips;
  P.segment = rest / (uint32_t)A.batch;
  P.b = rest % (uint32_t)A.batch;
  P.strip = (int64_t)strip * (64 * V);
  P.lane = (threadIdx.x & 63) * V;
  P.in = P.strip + P.lane < A.dim;
  if (!P.in) P.lane = 0;
  P.len = steps_of(A, P.b);
  P.begin = P.segment * A.segment_steps;
  P.end = P.begin + A.segment_steps < A.steps ? P.begin + A.segment_steps : A.steps;
  return P;
}

// What a lane holds of a step, in one register: an entry of 32 bits, or two or one of 16.
template <class T, int V>
__device__ __forceinline__ uint32_t load_word(const T* p) {
  static_assert(V * sizeof(T) <= 4, "one register");
  if constexpr (V * sizeof(T) == 4) return *reinterpret_cast<const uint32_t*>(p);
  else return *reinterpret_cast<const uint16_t*>(p);
}
template <class T>
__device__ __forceinline__ float entry(uint32_t word, int i) {
  if constexpr (sizeof(T) == 4) return __uint_as_float(word);
  else if constexpr (std::is_same_v<T, bf16_t>) return __uint_as_float(i ? word & 0xFFFF0000u : word << 16);
  else return (float)__builtin_bit_cast(f16_t, (uint16_t)(i ? word >> 16 : word));
}

// Rows t .. t + n - 1 of a lane's channels, n >= 1; the rest of the wave's steps repeat the last row.
template <class T, int V>
__device__ __forceinline__ void load_steps(const void* base, int64_t seq, int64_t step, const RecurPlace& P, int64_t t, int n,
                                           uint32_t (&x)[kSaveSteps]) {
  const T* p = (const T*)base + P.b * seq + t * step + P.strip;
#pragma unroll
  for (int j = 0; j < kSaveSteps; ++j) {
    x[j] = load_word<T, V>(p + P.lane);
    p += j + 1 < n ? step : 0;
  }
}

template <class T, int V>
__device__ __forceinline__ void store_step(void* base, int64_t seq, int64_t step, const RecurPlace& P, int64_t t, const float (&x)[V]) {
  store_floats<T, V>((T*)base + P.b * seq + t * step + P.strip + P.lane, x);
}

__device__ __forceinline__ int steps_left(int64_t end, int64_t t) {
  return __builtin_amdgcn_readfirstlane(end <= t ? 0 : end - t < kSaveSteps ? (int)(end - t) : kSaveSteps);
}

// (a, b) of the steps of a wave, and all of them in one map after (ma, mh); steps that are not in the sequence pass the state on.
template <class T, int V>
__device__ __forceinline__ void step_maps(const uint32_t (&f)[kSaveSteps], const uint32_t (&u)[kSaveSteps], int n,
                                          float (&a)[kSaveSteps][V], float (&b)[kSaveSteps][V], float (&ma)[V], float (&mh)[V]) {
#pragma unroll
  for (int j = 0; j < kSaveSteps; ++j)
#pragma unroll
    for (int i = 0; i < V; ++i) {
      float down;
      gate(entry<T>(f[j], i), a[j][i], down);
      b[j][i] = down * entry<T>(u[j], i);
      if (j >= n) {
        a[j][i] = 1.0f;
        b[j][i] = 0.0f;
      }
      mh[i] = fmaf(a[j][i], mh[i], b[j][i]);
      ma[i] *= a[j][i];
    }
}

// The waves' maps in LDS, two rounds in turn (so that one barrier a round is enough).
template <int V>
struct RecurMaps {
  float a[2][kRecurWaves][64][V], h[2][kRecurWaves][64][V];
};

template <class T, int V, bool GATED>
__global__ __launch_bounds__(64 * kRecurWaves) void k_recur(RecurArgs A) {
  __shared__ RecurMaps<V> S;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const RecurPlace P = recur_place<V>(A);
  float h[V];
#pragma unroll
  for (int i = 0; i < V; ++i) h[i] = A.parts || !A.h0 ? 0.0f : A.h0[P.b * A.dim + P.strip + P.lane + i];
  if (A.parts)
    for (uint32_t s = 0; s <= P.segment; ++s)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float2 m = A.parts[((int64_t)s * A.batch + P.b) * A.dim + P.strip + P.lane + i];
        h[i] = fmaf(m.x, h[i], m.y);
      }
  int turn = 0;
  for (int64_t t = P.begin; t < P.end; t += kSaveSteps * waves, turn ^= 1) {
    const int64_t t0 = t + kSaveSteps * wave;
    const int n = steps_left(P.len, t0), all = steps_left(P.end, t0);
    float a[kSaveSteps][V], b[kSaveSteps][V];
    uint32_t o[kSaveSteps];
    float ma[V], mh[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      ma[i] = 1.0f;
      mh[i] = 0.0f;
    }
    if (n > 0) {
      uint32_t f[kSaveSteps], u[kSaveSteps];
      load_steps<T, V>(A.f, A.f_seq, A.f_step, P, t0, n, f);
      load_steps<T, V>(A.u, A.u_seq, A.u_step, P, t0, n, u);
      if (GATED) load_steps<T, V>(A.o, A.o_seq, A.o_step, P, t0, n, o);
      step_maps<T, V>(f, u, n, a, b, ma, mh);
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
      S.a[turn][wave][lane][i] = ma[i];
      S.h[turn][wave][lane][i] = mh[i];
    }
    __syncthreads();
    float g[V];
    for (int w = 0; w < waves; ++w)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        if (w == wave) g[i] = h[i];
        h[i] = fmaf(S.a[turn][w][lane][i], h[i], S.h[turn][w][lane][i]);
      }
    if (!P.in || all == 0) continue;
    if (A.saved) {
#pragma unroll
      for (int i = 0; i < V; ++i) A.saved[((t0 / kSaveSteps) * A.batch + P.b) * A.dim + P.strip + P.lane + i] = g[i];
    }
#pragma unroll
    for (int j = 0; j < kSaveSteps; ++j) {
      float out[V];
      if (j >= all) break;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        out[i] = 0.0f;
        if (j < n) {
          g[i] = fmaf(a[j][i], g[i], b[j][i]);
          out[i] = GATED ? gate(entry<T>(o[j], i)) * g[i] : g[i];
        }
      }
      store_step<T, V>(A.y, A.y_seq, A.y_step, P, t0 + j, out);
    }
  }
  if (A.h_last && P.in && wave == 0 && P.segment + 1 == A.segments)
#pragma unroll
    for (int i = 0; i < V; ++i) A.h_last[P.b * A.dim + P.strip + P.lane + i] = h[i];
}

// The maps of the segments: parts[0] = (0, h0), parts[s + 1] = that of segment s; the last one's is not needed.  A wave
// takes a piece of the segment in one go.
template <class T, int V>
__global__ __launch_bounds__(64 * kRecurWaves) void k_recur_part(RecurArgs A) {
  __shared__ RecurMaps<V> S;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const RecurPlace P = recur_place<V>(A);
  const int64_t piece = A.segment_steps / waves;
  float ma[V], mh[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    ma[i] = 1.0f;
    mh[i] = 0.0f;
  }
  for (int64_t t0 = P.begin + wave * piece; t0 < P.begin + (wave + 1) * piece; t0 += kSaveSteps) {
    const int n = steps_left(P.len, t0);
    if (n == 0) break;
    uint32_t f[kSaveSteps], u[kSaveSteps];
    load_steps<T, V>(A.f, A.f_seq, A.f_step, P, t0, n, f);
    load_steps<T, V>(A.u, A.u_seq, A.u_step, P, t0, n, u);
    float a[kSaveSteps][V], b[kSaveSteps][V];
    step_maps<T, V>(f, u, n, a, b, ma, mh);
  }
#pragma unroll
  for (int i = 0; i < V; ++i) {
    S.a[0][wave][lane][i] = ma[i];
    S.h[0][wave][lane][i] = mh[i];
  }
  __syncthreads();
  if (wave != 0 || !P.in) return;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    for (int w = 1; w < waves; ++w) {
      mh[i] = fmaf(S.a[0][w][lane][i], mh[i], S.h[0][w][lane][i]);
      ma[i] *= S.a[0][w][lane][i];
    }
    const int64_t at = P.b * A.dim + P.strip + P.lane + i;
    A.parts[(int64_t)(P.segment + 1) * A.batch * A.dim + at] = make_float2(ma[i], mh[i]);
    if (P.segment == 0) A.parts[at] = make_float2(0.0f, A.h0 ? A.h0[at] : 0.0f);
  }
}

// Backward: the same from the last steps back, with the map of a step on a_{t+1} e_{t+1}: e -> a (e + dy s).  The states
// before each wave's steps are those that the forward pass kept.
template <class T, int V, bool GATED>
__global__ __launch_bounds__(64 * kRecurWaves) void k_recur_back(RecurArgs A) {
  __shared__ RecurMaps<V> S;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const RecurPlace P = recur_place<V>(A);
  float e[V];
#pragma unroll
  for (int i = 0; i < V; ++i) e[i] = A.dlast ? A.dlast[P.b * A.dim + P.strip + P.lane + i] : 0.0f;
  if (A.parts)
    for (uint32_t s = A.segments - 1; s > P.segment; --s)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float2 m = A.parts[((int64_t)s * A.batch + P.b) * A.dim + P.strip + P.lane + i];
        e[i] = fmaf(m.x, e[i], m.y);
      }
  const int64_t round = kSaveSteps * waves;
  int turn = 0;
  for (int64_t t = P.begin + (P.end - P.begin + round - 1) / round * round - round; t >= P.begin; t -= round, turn ^= 1) {
    const int64_t t0 = t + kSaveSteps * wave;
    const int n = steps_left(P.len, t0), all = steps_left(P.end, t0);
    // of each step: a, dy s, 1 - a, (h_{t-1} - u) a
    float a[kSaveSteps][V], into[kSaveSteps][V], down[kSaveSteps][V], off[kSaveSteps][V];
    float ma[V], me[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      ma[i] = 1.0f;
      me[i] = 0.0f;
    }
    if (n > 0) {
      uint32_t f[kSaveSteps], u[kSaveSteps], o[kSaveSteps], d[kSaveSteps];
      load_steps<T, V>(A.f, A.f_seq, A.f_step, P, t0, n, f);
      load_steps<T, V>(A.u, A.u_seq, A.u_step, P, t0, n, u);
      load_steps<T, V>(A.dy, A.y_seq, A.y_step, P, t0, n, d);
      if (GATED) load_steps<T, V>(A.o, A.o_seq, A.o_step, P, t0, n, o);
      float h[V];
#pragma unroll
      for (int i = 0; i < V; ++i) h[i] = A.saved[((t0 / kSaveSteps) * A.batch + P.b) * A.dim + P.strip + P.lane + i];
#pragma unroll
      for (int j = 0; j < kSaveSteps; ++j) {
        float go[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const float x = entry<T>(u[j], i), dy = entry<T>(d[j], i);
          gate(entry<T>(f[j], i), a[j][i], down[j][i]);
          off[j][i] = (h[i] - x) * a[j][i];
          h[i] = fmaf(a[j][i], h[i], down[j][i] * x);
          into[j][i] = dy;
          if (GATED) {
            float s, r;
            gate(entry<T>(o[j], i), s, r);
            into[j][i] = dy * s;
            go[i] = dy * h[i] * s * r;
          }
          if (j >= n) {
            a[j][i] = 1.0f;
            into[j][i] = 0.0f;
          }
        }
        if (GATED && P.in && j < n) store_step<T, V>(A.dout, A.do_seq, A.do_step, P, t0 + j, go);
      }
#pragma unroll
      for (int j = kSaveSteps - 1; j >= 0; --j) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
          me[i] = (me[i] + into[j][i]) * a[j][i];
          ma[i] *= a[j][i];
        }
      }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
      S.a[turn][wave][lane][i] = ma[i];
      S.h[turn][wave][lane][i] = me[i];
    }
    __syncthreads();
    float g[V];
    for (int w = waves - 1; w >= 0; --w)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        if (w == wave) g[i] = e[i];
        e[i] = fmaf(S.a[turn][w][lane][i], e[i], S.h[turn][w][lane][i]);
      }
    if (!P.in || all == 0) continue;
#pragma unroll
    for (int j = kSaveSteps - 1; j >= 0; --j) {
      if (j >= all) continue;
      float gf[V], gu[V];
#pragma unroll
      for (int i = 0; i < V; ++i) {
        gf[i] = gu[i] = 0.0f;
        if (j < n) {
          g[i] += into[j][i];
          gu[i] = g[i] * down[j][i];
          gf[i] = gu[i] * off[j][i];
          g[i] *= a[j][i];
        }
      }
      store_step<T, V>(A.df, A.df_seq, A.df_step, P, t0 + j, gf);
      store_step<T, V>(A.du, A.du_seq, A.du_step, P, t0 + j, gu);
      if (GATED && j >= n) {
        const float zero[V] = {};
        store_step<T, V>(A.dout, A.do_seq, A.do_step, P, t0 + j, zero);
      }
    }
  }
  if (A.dh0 && P.in && wave == 0 && P.segment == 0)
#pragma unroll
    for (int i = 0; i < V; ++i) A.dh0[P.b * A.dim + P.strip + P.lane + i] = e[i];
}

// parts[s] = the map of segment s; the first one's is not needed.
template <class T, int V, bool GATED>
__global__ __launch_bounds__(64 * kRecurWaves) void k_recur_back_part(RecurArgs A) {
  __shared__ RecurMaps<V> S;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  RecurPlace P = recur_place<V>(A);
  P.begin += A.segment_steps;     // from the second segment on
  const int64_t piece = A.segment_steps / waves;
  float ma[V], me[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    ma[i] = 1.0f;
    me[i] = 0.0f;
  }
  for (int64_t t0 = P.begin + (wave + 1) * piece - kSaveSteps; t0 >= P.begin + wave * piece; t0 -= kSaveSteps) {
    const int n = steps_left(P.len, t0);
    if (n == 0) continue;
    uint32_t f[kSaveSteps], o[kSaveSteps], d[kSaveSteps];
    load_steps<T, V>(A.f, A.f_seq, A.f_step, P, t0, n, f);
    load_steps<T, V>(A.dy, A.y_seq, A.y_step, P, t0, n, d);
    if (GATED) load_steps<T, V>(A.o, A.o_seq, A.o_step, P, t0, n, o);
#pragma unroll
    for (int j = kSaveSteps - 1; j >= 0; --j) {
      if (j >= n) continue;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float a = gate(entry<T>(f[j], i));
        float into = entry<T>(d[j], i);
        if (GATED) into *= gate(entry<T>(o[j], i));
        me[i] = (me[i] + into) * a;
        ma[i] *= a;
      }
    }
  }
#pragma unroll
  for (int i = 0; i < V; ++i) {
    S.a[0][wave][lane][i] = ma[i];
    S.h[0][wave][lane][i] = me[i];
  }
  __syncthreads();
  if (wave != waves - 1 || !P.in) return;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    for (int w = waves - 2; w >= 0; --w) {
      me[i] = fmaf(S.a[0][w][lane][i], me[i], S.h[0][w][lane][i]);
      ma[i] *= S.a[0][w][lane][i];
    }
    A.parts[((int64_t)(P.segment + 1) * A.batch + P.b) * A.dim + P.strip + P.lane + i] = make_float2(ma[i], me[i]);
  }
}

}  // namespace choco
