// Gated linear recurrence h_t = a_t h_{t-1} + (1 - a_t) u_t, a = sigmoid(f), y = sigmoid(o) h, and its backward
// pass (device code).
//
// Bound by memory: 25 operations an entry against 4 to 14 bytes.
//
// How the work is split.  A strip is 64 * V channels of one sequence, V channels a lane (two of 16 bits where everything is
// aligned to that).  A workgroup takes a tile: the steps of a strip that its waves hold in registers, 8 or 16 each.  A wave loads
// its steps at once and reduces them to the map h -> A h + H; the waves exchange these maps through LDS, and each applies those
// before its own to the state before the tile and goes through its steps, which are still in registers, once more.  So
// everything is read once, and the chain from step to step is as long as a tile has waves.
//
// Sequences longer than a tile are chains of tiles.  A tile publishes its map as soon as it has it; kChainTiles of them in a row
// form a link: each applies to the state before the link the maps of the tiles before it in the link, and the last one
// publishes the state after it.  Which values are combined, and in which order, is fixed, so the bits of a result do not depend on
// timing.  A published value is one 64-bit word with the map's A in its lower half, all ones until it is there, stored and
// loaded by relaxed atomics of the device's scope: a word carries its own readiness and nothing else has to be ordered
// with it.  A workgroup takes its place in a chain from the chain's counter when it starts.  What it waits for are tiles that have
// taken theirs before, so they are running or done; their maps do not wait for anything, and the state before a link waits for
// earlier links only: whatever the order in which workgroups are started, every wait ends.  (A wait gives up after kMostPolls
// all the same; what it waited for is then NaN.)
//
// Measured, us (GB/s of what cannot be done without): 160 sequences of 35 steps x 650 in fp32 14 (3,450), backward 22 to 23.5 (3,750 to
// 4,000); 2 of 32,768 x 2048 in bf16 197 to 208 (4,200 to 4,400), with the states kept 213; backward of 4 of 16,384 x 1280 without o 200 to
// 202 (4,200); 64 of 512 x 1280 73 and 125 (4,600 to 4,700); a large copy reaches 4,700.  1 of 8192 x 512 in fp32 without o 18 and 22,
// of which 3 start the chains (50 MB and 84 MB, 8.5 and 14 us at the rate of two reads and a write): every tile is under way at once,
// and the last of 64 waits for three links.
// Before: two passes over segments of a sequence, the first for their maps, 324 and 280; eight steps a wave 310 and 228;
// one lane a channel, step by step, 14,059 and 20,573.  Workgroups that stay and ask for their next tile's steps ahead hold
// places in the chain that others wait for: 302 to 790.
#pragma once

#include <type_traits>

#include "choco_types.h"

namespace choco {

constexpr int kSaveSteps = 8;       // the forward pass keeps the state before every so many
constexpr int kRecurWaves = 16;     // most waves of a workgroup
// A sequence of one tile: steps of a wave, up to kRecurWaves of them.  160 x 35 x 650 in fp32, 8 | 16 steps: 14.0 | 14.9 us, back
// 22.0 | 25.3.
constexpr int kAloneSteps = 8;
// Chains: waves of a tile, steps of a wave - as many as leave two workgroups for a compute unit (backward holds four numbers a step
// and channel) - and tiles of a link.  2 of 32,768 x 2048, 4 of 16,384 x 1280 back, 1 of 8192 x 512: 8 waves 207 | 202 | 18 us,
// 4 waves and links of 32 tiles 250 | 243 | 20, 16 waves 234 | 204 | 19; 8 steps forward 272 | - | 24; links of 5, 8, 24 tiles
// 211 | 206 | 26, 208 | 207 | 22, 210 | 201 | 18.
constexpr int kChainWaves = 8;
constexpr int kForwardSteps = 16;
constexpr int back_steps(int v) { return v == 1 ? 16 : 8; }
constexpr int kChainTiles = 16;
// (a kept state has one wave that writes it and one that starts from it; what does not fit one tile fills more than one of a chain)
static_assert(kAloneSteps % kSaveSteps == 0 && kForwardSteps % kSaveSteps == 0 && back_steps(1) % kSaveSteps == 0 && back_steps(2) % kSaveSteps == 0);
static_assert(kAloneSteps * kRecurWaves >= kChainWaves * kForwardSteps && kForwardSteps >= back_steps(1) && kForwardSteps >= back_steps(2));
constexpr int kMostPolls = 1 << 20;
constexpr int kTakenWords = 64;     // from one chain's counter to the next: additions to one line wait for each other, 11 ns each

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
  // chains (strips of all sequences): words of their tiles' maps [chains][tiles][64 * V], of the states before their links
  // [chains][links][64 * V], and how many tiles have been taken [chains][kTakenWords]
  uint64_t *maps, *states;
  uint32_t* taken;
  uint32_t strips, chains, tiles, links;
};

// exp(-x) for an x of type T.  The instruction takes a power of two: its argument is a product rounded to |x| 2^-24, and what that
// leaves is put back as a factor (without it 1 - sigmoid(60) is off by 29 2^-24 on average, with it by less than one).  Infinite
// arguments leave nothing.  An x of 16 bits is itself rounded to |x| 2^-9 or 2^-12, against which the product's rounding is
// nothing, and goes without: 2 of 32,768 x 2048 in bf16 208 us, with it 220.
template <class T>
__device__ __forceinline__ float exp_minus(float x) {
  constexpr float kHigh = -1.44269502f, kLow = -1.92596299e-8f;     // together -log2(e)
  const float p = x * kHigh;
  if constexpr (sizeof(T) == 2) return __builtin_amdgcn_exp2f(p);
  const float left = fmaf(x, kLow, fmaf(x, kHigh, -p));
  return __builtin_amdgcn_exp2f(p) * (fabsf(p) < 256.0f ? fmaf(left, 0.693147182f, 1.0f) : 1.0f);
}
// sigmoid(x) and 1 - sigmoid(x), the smaller of the two not by a difference: in fp32 good to 10 2^-24 each.  exp(-x) may overflow: up
// is then 0 and down 1.
template <class T>
__device__ __forceinline__ void gate(float x, float& up, float& down) {
  const float e = exp_minus<T>(x);
  up = __builtin_amdgcn_rcpf(1.0f + e);
  down = x >= 0.0f ? e * up : 1.0f - up;
}
template <class T>
__device__ __forceinline__ float gate(float x) { return __builtin_amdgcn_rcpf(1.0f + exp_minus<T>(x)); }

__device__ __forceinline__ int64_t steps_of(const RecurArgs& A, int64_t b) {
  if (!A.lengths) return A.steps;
  const int64_t n = A.lengths[b];
  return n < 0 ? 0 : n > A.steps ? A.steps : n;
}

// ---- words of a chain ----
constexpr uint64_t kNotThere = ~(uint64_t)0;
__device__ __forceinline__ void publish(uint64_t* word, float a, float h) {
  uint32_t low = __float_as_uint(a);
  if (low == 0xFFFFFFFFu) low = 0x7FC00000u;     // any other NaN
  __hip_atomic_store(word, (uint64_t)__float_as_uint(h) << 32 | low, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
template <int V>
__device__ __forceinline__ void await(uint64_t* words, float (&a)[V], float (&h)[V]) {
  uint64_t x[V];
  for (int polls = 0; polls < kMostPolls; ++polls) {
    bool there = true;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      x[i] = __hip_atomic_load(words + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      there = there && (uint32_t)x[i] != 0xFFFFFFFFu;
    }
    if (__all(there)) break;
    __builtin_amdgcn_s_sleep(1);
  }
#pragma unroll
  for (int i = 0; i < V; ++i) {
    a[i] = __uint_as_float((uint32_t)x[i]);
    h[i] = __uint_as_float((uint32_t)(x[i] >> 32));
  }
}

// Before the chains start: no word is there but the states before the first links (`first`, batch x dim, or zero), nothing is
// taken.
__global__ __launch_bounds__(256) void k_recur_chains(RecurArgs A, const float* first, int width) {
  const int64_t maps = (int64_t)A.chains * A.tiles * width, states = (int64_t)A.chains * A.links * width;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < maps + states + A.chains; i += (int64_t)gridDim.x * 256) {
    if (i < maps) {
      A.maps[i] = kNotThere;
    } else if (i < maps + states) {
      const int64_t j = i - maps, chain = j / ((int64_t)A.links * width);
      uint64_t word = kNotThere;
      if (j % ((int64_t)A.links * width) < width) {
        const int64_t b = chain / A.strips;
        int64_t c = chain % A.strips * width + j % width;
        if (c >= A.dim) c = chain % A.strips * width;
        word = first ? (uint64_t)__float_as_uint(first[b * A.dim + c]) << 32 : 0;
      }
      A.states[j] = word;
    } else {
      A.taken[(i - maps - states) * kTakenWords] = 0;
    }
  }
}

// ---- a workgroup's tile ----
struct RecurPlace {
  int64_t b, strip, len, begin;    // sequence, first channel of the strip, its length, the tile's first step
  uint32_t chain, tile, turn;      // turn: the tile's place in its chain (backward: counted from the last)
  int lane;                        // first channel of the lane in the strip (of one that has none: 0, and it writes nothing)
  bool in;                         // the lane has channels
};

template <int V, bool CHAIN, bool BACK>
__device__ __forceinline__ RecurPlace recur_place(const RecurArgs& A, int tile_steps, uint32_t* taken) {
  RecurPlace P;
  P.chain = CHAIN ? blockIdx.x % A.chains : blockIdx.x;
  P.turn = 0;
  if (CHAIN) {
    if (threadIdx.x == 0) *taken = atomicAdd(A.taken + (int64_t)P.chain * kTakenWords, 1u);
    __syncthreads();
    P.turn = __builtin_amdgcn_readfirstlane(*taken);
  }
  P.tile = BACK ? A.tiles - 1 - P.turn : P.turn;
  P.b = P.chain / A.strips;
  P.strip = (int64_t)(P.chain % A.strips) * (64 * V);
  P.lane = (threadIdx.x & 63) * V;
  P.in = P.strip + P.lane < A.dim;
  if (!P.in) P.lane = 0;
  P.len = steps_of(A, P.b);
  P.begin = (int64_t)P.tile * tile_steps;
  return P;
}

// A sequence of one tile; chains through the caches, with their results written past them, or read past them as well.
enum { kAlone = 0, kThrough = 1, kPastOut = 2, kPast = 3 };

// What a lane holds of a step, in one register: an entry of 32 bits, or two or one of 16.
template <class T, int V, bool PAST>
__device__ __forceinline__ uint32_t load_word(const T* p) {
  static_assert(V * sizeof(T) <= 4, "one register");
  using Word = std::conditional_t<V * sizeof(T) == 4, uint32_t, uint16_t>;
  if constexpr (PAST) return __builtin_nontemporal_load(reinterpret_cast<const Word*>(p));
  else return *reinterpret_cast<const Word*>(p);
}
// Rows t .. t + n - 1 of a lane's channels, n >= 1; the rest of the wave's steps repeat the last row.
template <class T, int V, bool PAST, int K>
__device__ __forceinline__ void load_steps(const void* base, int64_t seq, int64_t step, const RecurPlace& P, int64_t t, int n,
                                           uint32_t (&x)[K]) {
  const T* p = (const T*)base + P.b * seq + t * step + P.strip;
#pragma unroll
  for (int j = 0; j < K; ++j) {
    x[j] = load_word<T, V, PAST>(p + P.lane);
    p += j + 1 < n ? step : 0;
  }
}

template <class T, int V, bool PAST>
__device__ __forceinline__ void store_step(void* base, int64_t seq, int64_t step, const RecurPlace& P, int64_t t, const float (&x)[V]) {
  T* p = (T*)base + P.b * seq + t * step + P.strip + P.lane;
  if constexpr (PAST) store_floats_past<T, V>(p, x);
  else store_floats<T, V>(p, x);
}

template <int K>
__device__ __forceinline__ int steps_left(int64_t end, int64_t t) {
  return __builtin_amdgcn_readfirstlane(end <= t ? 0 : end - t < K ? (int)(end - t) : K);
}

template <int V, int W, bool CHAIN>
struct RecurShared {
  static constexpr int kLink = CHAIN ? kChainTiles : 1;
  float a[W][64][V], h[W][64][V];               // the waves' maps, in the order of the recurrence
  float link_a[kLink][64][V], link_h[kLink][64][V];     // those of the tiles before in the link; last: the state before it
  uint32_t taken;
};

// From the waves' maps (m_a, m_h; `turn`: a wave's place in the order of the recurrence) and the state `h` before the tile
// (outside chains: given) to the state before the wave's own steps; the last wave's ends as the one after the tile.
template <int V, bool CHAIN, int W>
__device__ __forceinline__ void recur_carry(const RecurArgs& A, const RecurPlace& P, RecurShared<V, W, CHAIN>& S, int turn, int waves,
                                            const float (&ma)[V], const float (&mh)[V], float (&h)[V], float (&after)[V]) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    S.a[turn][lane][i] = ma[i];
    S.h[turn][lane][i] = mh[i];
  }
  __syncthreads();
  if (CHAIN) {
    const uint32_t link = P.turn / kChainTiles, before = P.turn % kChainTiles;
    if (turn == waves - 1 && before + 1 < kChainTiles && P.turn + 1 < A.tiles) {
      float ta[V], th[V];
#pragma unroll
      for (int i = 0; i < V; ++i) {
        ta[i] = 1.0f;
        th[i] = 0.0f;
      }
      for (int w = 0; w < waves; ++w)
#pragma unroll
        for (int i = 0; i < V; ++i) {
          th[i] = fmaf(S.a[w][lane][i], th[i], S.h[w][lane][i]);
          ta[i] *= S.a[w][lane][i];
        }
#pragma unroll
      for (int i = 0; i < V; ++i) publish(A.maps + ((int64_t)P.chain * A.tiles + P.turn) * (64 * V) + lane * V + i, ta[i], th[i]);
    }
    for (uint32_t k = turn; k <= before; k += waves) {     // the maps before, and the state before them
      float la[V], lh[V];
      await<V>((k < before ? A.maps + ((int64_t)P.chain * A.tiles + P.turn - before + k) * (64 * V)
                           : A.states + ((int64_t)P.chain * A.links + link) * (64 * V)) + lane * V, la, lh);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        S.link_a[k][lane][i] = la[i];
        S.link_h[k][lane][i] = lh[i];
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < V; ++i) h[i] = S.link_h[before][lane][i];
    for (uint32_t w = 0; w < before; ++w)
#pragma unroll
      for (int i = 0; i < V; ++i) h[i] = fmaf(S.link_a[w][lane][i], h[i], S.link_h[w][lane][i]);
  }
  for (int w = 0; w < turn; ++w)
#pragma unroll
    for (int i = 0; i < V; ++i) h[i] = fmaf(S.a[w][lane][i], h[i], S.h[w][lane][i]);
  if (turn != waves - 1) return;
#pragma unroll
  for (int i = 0; i < V; ++i) after[i] = fmaf(ma[i], h[i], mh[i]);
  if (CHAIN && P.turn % kChainTiles + 1 == kChainTiles && P.turn + 1 < A.tiles)
#pragma unroll
    for (int i = 0; i < V; ++i)
      publish(A.states + ((int64_t)P.chain * A.links + P.turn / kChainTiles + 1) * (64 * V) + lane * V + i, 0.0f, after[i]);
}

template <class T, int V, bool GATED, int MODE>
__global__ __launch_bounds__(64 * (MODE != kAlone ? kChainWaves : kRecurWaves)) void k_recur(RecurArgs A) {
  constexpr bool CHAIN = MODE != kAlone;
  constexpr int K = CHAIN ? kForwardSteps : kAloneSteps, W = CHAIN ? kChainWaves : kRecurWaves;
  __shared__ RecurShared<V, W, CHAIN> S;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  const RecurPlace P = recur_place<V, CHAIN, false>(A, K * W, &S.taken);
  const int64_t state = P.b * A.dim + P.strip + P.lane, t0 = P.begin + K * wave;
  const int n = steps_left<K>(P.len, t0), all = steps_left<K>(A.steps, t0);
  float h[V], a[K][V], b[K][V], ma[V], mh[V], after[V];
  uint32_t o[K];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    h[i] = CHAIN || !A.h0 ? 0.0f : A.h0[state + i];
    ma[i] = 1.0f;
    mh[i] = 0.0f;
  }
  if (n > 0) {
    uint32_t f[K], u[K];
    load_steps<T, V, MODE == kPast, K>(A.f, A.f_seq, A.f_step, P, t0, n, f);
    load_steps<T, V, MODE == kPast, K>(A.u, A.u_seq, A.u_step, P, t0, n, u);
    if (GATED) load_steps<T, V, MODE == kPast, K>(A.o, A.o_seq, A.o_step, P, t0, n, o);
#pragma unroll
    for (int j = 0; j < K; ++j)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        float down;
        gate<T>(entry<T>(f[j], i), a[j][i], down);
        b[j][i] = down * entry<T>(u[j], i);
        if (j >= n) {     // not in the sequence: the state is passed on
          a[j][i] = 1.0f;
          b[j][i] = 0.0f;
        }
        mh[i] = fmaf(a[j][i], mh[i], b[j][i]);
        ma[i] *= a[j][i];
      }
  }
  recur_carry<V, CHAIN, W>(A, P, S, wave, waves, ma, mh, h, after);
  if (!P.in) return;
  if (A.h_last && P.tile + 1 == A.tiles && wave == waves - 1)
#pragma unroll
    for (int i = 0; i < V; ++i) A.h_last[state + i] = after[i];
  if (all == 0) return;
#pragma unroll
  for (int j = 0; j < K; ++j) {
    if (j < all) {
      if (j % kSaveSteps == 0 && A.saved)
#pragma unroll
        for (int i = 0; i < V; ++i) A.saved[((t0 + j) / kSaveSteps) * A.batch * A.dim + state + i] = h[i];
      float out[V];
#pragma unroll
      for (int i = 0; i < V; ++i) {
        out[i] = 0.0f;
        if (j < n) {
          h[i] = fmaf(a[j][i], h[i], b[j][i]);
          out[i] = GATED ? gate<T>(entry<T>(o[j], i)) * h[i] : h[i];
        }
      }
      store_step<T, V, MODE != kAlone && MODE != kThrough>(A.y, A.y_seq, A.y_step, P, t0 + j, out);
    }
  }
}

// Backward: the same from the last steps back, with the map of a step on a_{t+1} e_{t+1}: e -> a (e + dy s).  The states
// before each wave's steps are those that the forward pass kept.
template <class T, int V, bool GATED, int MODE>
__global__ __launch_bounds__(64 * (MODE != kAlone ? kChainWaves : kRecurWaves)) void k_recur_back(RecurArgs A) {
  constexpr bool CHAIN = MODE != kAlone;
  constexpr int K = CHAIN ? back_steps(V) : kAloneSteps, W = CHAIN ? kChainWaves : kRecurWaves;
  __shared__ RecurShared<V, W, CHAIN> S;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  const RecurPlace P = recur_place<V, CHAIN, true>(A, K * W, &S.taken);
  const int64_t state = P.b * A.dim + P.strip + P.lane, t0 = P.begin + K * wave;
  const int n = steps_left<K>(P.len, t0), all = steps_left<K>(A.steps, t0);
  // of each step: a, dy s, 1 - a, (h_{t-1} - u) a
  float e[V], a[K][V], into[K][V], down[K][V], off[K][V], ma[V], me[V], after[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    e[i] = CHAIN || !A.dlast ? 0.0f : A.dlast[state + i];
    ma[i] = 1.0f;
    me[i] = 0.0f;
  }
  if (n > 0) {
    uint32_t f[K], u[K], o[K], d[K];
    load_steps<T, V, MODE == kPast, K>(A.f, A.f_seq, A.f_step, P, t0, n, f);
    load_steps<T, V, MODE == kPast, K>(A.u, A.u_seq, A.u_step, P, t0, n, u);
    load_steps<T, V, MODE == kPast, K>(A.dy, A.y_seq, A.y_step, P, t0, n, d);
    if (GATED) load_steps<T, V, MODE == kPast, K>(A.o, A.o_seq, A.o_step, P, t0, n, o);
    float h[V];
#pragma unroll
    for (int i = 0; i < V; ++i) h[i] = A.saved[(t0 / kSaveSteps) * A.batch * A.dim + state + i];
#pragma unroll
    for (int j = 0; j < K; ++j) {
      float go[V];
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float x = entry<T>(u[j], i), dy = entry<T>(d[j], i);
        gate<T>(entry<T>(f[j], i), a[j][i], down[j][i]);
        off[j][i] = (h[i] - x) * a[j][i];
        h[i] = fmaf(a[j][i], h[i], down[j][i] * x);
        into[j][i] = dy;
        if (GATED) {
          float s, r;
          gate<T>(entry<T>(o[j], i), s, r);
          into[j][i] = dy * s;
          go[i] = dy * h[i] * s * r;
        }
        if (j >= n) {
          a[j][i] = 1.0f;
          into[j][i] = 0.0f;
        }
      }
      if (GATED && P.in && j < n) store_step<T, V, MODE != kAlone && MODE != kThrough>(A.dout, A.do_seq, A.do_step, P, t0 + j, go);
    }
#pragma unroll
    for (int j = K - 1; j >= 0; --j)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        me[i] = (me[i] + into[j][i]) * a[j][i];
        ma[i] *= a[j][i];
      }
  }
  recur_carry<V, CHAIN, W>(A, P, S, waves - 1 - wave, waves, ma, me, e, after);
  if (!P.in) return;
  if (A.dh0 && P.tile == 0 && wave == 0)
#pragma unroll
    for (int i = 0; i < V; ++i) A.dh0[state + i] = after[i];
#pragma unroll
  for (int j = K - 1; j >= 0; --j) {
    if (j < all) {
      float gf[V], gu[V];
#pragma unroll
      for (int i = 0; i < V; ++i) {
        gf[i] = gu[i] = 0.0f;
        if (j < n) {
          e[i] += into[j][i];
          gu[i] = e[i] * down[j][i];
          gf[i] = gu[i] * off[j][i];
          e[i] *= a[j][i];
        }
      }
      store_step<T, V, MODE != kAlone && MODE != kThrough>(A.df, A.df_seq, A.df_step, P, t0 + j, gf);
      store_step<T, V, MODE != kAlone && MODE != kThrough>(A.du, A.du_seq, A.du_step, P, t0 + j, gu);
      if (GATED && j >= n) {
        const float zero[V] = {};
        store_step<T, V, MODE != kAlone && MODE != kThrough>(A.dout, A.do_seq, A.do_step, P, t0 + j, zero);
      }
    }
  }
}

}  // namespace choco
