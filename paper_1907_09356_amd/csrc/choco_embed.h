// Embedding lookup with scaling, and its gradient summed by token (device code).
#pragma once

#include "choco_types.h"

namespace choco {

struct EmbedArgs {
  const void* tokens;
  const void* table;   // forward: the tables
  const void* rows;    // y (written) or dy (read)
  float* dtable;
  int64_t ntokens, vocab, dim;
  int64_t token_stride, table_stride, row_stride, row_ld;
  float scale;
  // the gradient's workspace, per worker
  uint32_t *keys, *places;           // tokens in ascending order and where each stood; [workers][ntokens]
  uint32_t *keys_next, *places_next; // the same again, where the order takes several passes through memory
  uint32_t* counts;                  // [workers][chunks][1 << digit_bits]
  float* partial;                    // [workers][pieces][2][partial_ld]
  int64_t partial_ld, pieces, column_chunks;
  uint32_t chunks, zero_blocks;      // zero_blocks: per worker, of kZeroFloats each
  int digit_bits, passes, accumulate;
};

constexpr int kSortThreads = 1024;                     // a workgroup that orders all of a worker's tokens in LDS ...
constexpr int kSortRounds = 8;
constexpr int kSortOne = kSortThreads * kSortRounds;   // ... of which there are no more than this
constexpr int kSortDigit = 9;                          // bits of the key in one pass, at most
constexpr int kChunkThreads = 256;                     // otherwise: a workgroup for each so many tokens
constexpr int kChunkRounds = 16;
constexpr int kChunkTokens = kChunkThreads * kChunkRounds;
constexpr int kChunkDigit = 10;
constexpr int kPiece = 32;                             // ordered tokens that a wave adds up
constexpr int kZeroFloats = 1 << 16;                   // floats that a workgroup clears
constexpr int kJoinWaves = 8;

// A token, or -1 for one outside the table.
template <class Tok>
__device__ __forceinline__ int32_t token_at(const EmbedArgs& A, int worker, int64_t r) {
  const int64_t t = (int64_t)((const Tok*)A.tokens)[(int64_t)worker * A.token_stride + r];
  return t >= 0 && t < A.vocab ? (int32_t)t : -1;
}

// y[w, r, :] = scale * table[w, token, :].  A group of 2^LANES_LOG2 lanes takes a row, V entries a lane at a time, and
// asks for kRowAhead such pieces before it writes the first.
constexpr int kRowAhead = 4;
template <class Tok, class Tab, class Row, int V>
__global__ __launch_bounds__(256) void k_embed(EmbedArgs A, int lanes_log2) {
  const int lane = threadIdx.x & ((1 << lanes_log2) - 1);
  const int64_t r = (int64_t)blockIdx.x * (256 >> lanes_log2) + (threadIdx.x >> lanes_log2);
  const int w = blockIdx.y;
  if (r >= A.ntokens) return;
  const int32_t t = token_at<Tok>(A, w, r);
  const Tab* from = (const Tab*)A.table + (int64_t)w * A.table_stride + (int64_t)(t < 0 ? 0 : t) * A.dim;
  Row* to = (Row*)A.rows + (int64_t)w * A.row_stride + r * A.row_ld;
  const int64_t step = (int64_t)V << lanes_log2;
  for (int64_t c = (int64_t)lane * V; c < A.dim; c += kRowAhead * step) {
    Pack<Tab, V> x[kRowAhead];
#pragma unroll
    for (int j = 0; j < kRowAhead; ++j)
      if (t >= 0 && c + j * step < A.dim) x[j] = *reinterpret_cast<const Pack<Tab, V>*>(from + c + j * step);
#pragma unroll
    for (int j = 0; j < kRowAhead; ++j) {
      if (c + j * step >= A.dim) break;
      float y[V];
#pragma unroll
      for (int i = 0; i < V; ++i) y[i] = t >= 0 ? to_float(x[j].e[i]) * A.scale : 0.0f;
      store_floats<Row, V>(to + c + j * step, y);
    }
  }
}

// ---- gradient ----
// 1. The tokens are put in order, stably, by counting on a few bits at a time (key: the token, or vocab for one outside the table);
//    the same launch clears the gradient, which takes longer than the order of an ordinary batch.
// 2. A wave adds up the rows of kPiece consecutive ordered tokens, for 64 * V columns: sums of tokens that lie in the piece
//    as a whole go to the gradient, those that reach over its ends to `partial`.
// 3. The partial sums of a token that spans pieces are added in their order.
// So work is split evenly whatever the tokens are (one word in a sixteenth of the places is ordinary), nothing is added by
// atomics, and every row of the gradient is written by one wave.

// Part `block` of the gradient's clearing, by a whole workgroup.
__device__ __forceinline__ void zero_part(const EmbedArgs& A, int64_t worker, int64_t block) {
  float* base = A.dtable + worker * A.table_stride;
  const int64_t size = A.vocab * A.dim;
  int64_t from = block * kZeroFloats, to = from + kZeroFloats < size ? from + kZeroFloats : size;
  // whole 16-byte vectors of memory between a few single floats at the ends
  const int64_t lead = (4 - (int64_t)(((uintptr_t)(base + from) >> 2) & 3)) & 3;
  const int64_t first = from + lead < to ? from + lead : to, last = first + (to - first) / 4 * 4;
  for (int64_t i = from + threadIdx.x; i < first; i += blockDim.x) base[i] = 0.0f;
  for (int64_t i = first + 4 * (int64_t)threadIdx.x; i < last; i += 4 * (int64_t)blockDim.x)
    *reinterpret_cast<Pack<float, 4>*>(base + i) = Pack<float, 4>{};
  for (int64_t i = last + threadIdx.x; i < to; i += blockDim.x) base[i] = 0.0f;
}

template <class Tok>
__device__ __forceinline__ uint32_t key_at(const EmbedArgs& A, int worker, int64_t r) {
  const int32_t t = token_at<Tok>(A, worker, r);
  return t < 0 ? (uint32_t)A.vocab : (uint32_t)t;
}

// Ranks of a wave's keys among those of the wave that hold the same digit, in the order (round, lane); `count`, the wave's
// counters in LDS, starts at zero and ends as the digits' numbers.  Lanes of one digit find each other by a ballot for each of its bits.
template <int ROUNDS>
__device__ __forceinline__ void rank_digits(volatile uint32_t* count, const uint32_t (&key)[ROUNDS], const bool (&there)[ROUNDS],
                                            int shift, int bits, uint32_t (&rank)[ROUNDS]) {
  const uint64_t before = ((uint64_t)1 << (threadIdx.x & 63)) - 1;
#pragma unroll
  for (int j = 0; j < ROUNDS; ++j) {
    const uint32_t digit = (key[j] >> shift) & ((1u << bits) - 1u);
    uint64_t same = __ballot(there[j]);
    for (int b = 0; b < bits; ++b) {
      const bool one = (digit >> b) & 1u;
      const uint64_t ones = __ballot(one);
      same &= one ? ones : ~ones;
    }
    const uint32_t below = (uint32_t)__popcll(same & before), all = (uint32_t)__popcll(same);
    uint32_t base = 0;
    if (there[j]) base = count[digit];
    rank[j] = base + below;
    if (there[j] && below + 1 == all) count[digit] = base + all;
  }
}

// Exclusive sums over the workgroup's threads, in their order.
template <int THREADS>
__device__ __forceinline__ uint32_t sum_before(uint32_t x, uint32_t* waves) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t sum = x;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const uint32_t y = (uint32_t)__shfl_up((int)sum, off, 64);
    if (lane >= off) sum += y;
  }
  if (lane == 63) waves[wave] = sum;
  __syncthreads();
  uint32_t base = 0;
  for (int w = 0; w < wave; ++w) base += waves[w];
  __syncthreads();
  return base + sum - x;
}

// All of a worker's tokens (no more than kSortOne) in order, in LDS.  Workgroups from the n-th on clear the gradient.
template <class Tok>
__global__ __launch_bounds__(kSortThreads) void k_embed_sort(EmbedArgs A, int workers) {
  constexpr int kWaves = kSortThreads / 64, kBins = 1 << kSortDigit;
  __shared__ uint32_t count[kWaves][kBins], base[kBins], sums[kWaves];
  __shared__ uint32_t keys[kSortOne], places[kSortOne];
  if ((int)blockIdx.x >= workers) {
    const uint32_t z = blockIdx.x - workers;
    zero_part(A, z / A.zero_blocks, z % A.zero_blocks);
    return;
  }
  const int w = blockIdx.x, wave = threadIdx.x >> 6, lane = threadIdx.x & 63, total = (int)A.ntokens;
  uint32_t key[kSortRounds], place[kSortRounds], rank[kSortRounds];
  bool there[kSortRounds];
#pragma unroll
  for (int j = 0; j < kSortRounds; ++j) {
    const int r = (wave * kSortRounds + j) * 64 + lane;
    there[j] = r < total;
    key[j] = there[j] ? key_at<Tok>(A, w, r) : 0u;
    place[j] = (uint32_t)r;
  }
  const uint32_t bins = 1u << A.digit_bits;
  for (int pass = 0; pass < A.passes; ++pass) {
    const int shift = pass * A.digit_bits;
    for (uint32_t d = lane; d < bins; d += 64) count[wave][d] = 0;
    rank_digits<kSortRounds>(count[wave], key, there, shift, A.digit_bits, rank);
    __syncthreads();
    // counters of a wave -> tokens of that digit in the waves before it; base -> tokens of lower digits
    uint32_t sum = 0;
    if (threadIdx.x < bins)
      for (int v = 0; v < kWaves; ++v) {
        const uint32_t c = count[v][threadIdx.x];
        count[v][threadIdx.x] = sum;
        sum += c;
      }
    const uint32_t lower = sum_before<kSortThreads>(sum, sums);
    if (threadIdx.x < bins) base[threadIdx.x] = lower;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kSortRounds; ++j)
      if (there[j]) {
        const uint32_t digit = (key[j] >> shift) & (bins - 1u), at = base[digit] + count[wave][digit] + rank[j];
        keys[at] = key[j];
        places[at] = place[j];
      }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kSortRounds; ++j) {
      const int r = (wave * kSortRounds + j) * 64 + lane;
      if (there[j]) {
        key[j] = keys[r];
        place[j] = places[r];
      }
    }
    __syncthreads();
  }
#pragma unroll
  for (int j = 0; j < kSortRounds; ++j) {
    const int r = (wave * kSortRounds + j) * 64 + lane;
    if (there[j]) {
      A.keys[(int64_t)w * A.ntokens + r] = key[j];
      A.places[(int64_t)w * A.ntokens + r] = place[j];
    }
  }
}

// One pass over longer lists, first half: how many tokens of a chunk hold each digit.  Workgroups from the last chunk's on clear
// the gradient.  The first pass reads the tokens, later ones what the one before wrote.
template <class Tok, bool FIRST>
__global__ __launch_bounds__(kChunkThreads) void k_embed_count(EmbedArgs A, int shift) {
  __shared__ uint32_t count[1 << kChunkDigit];
  const int w = blockIdx.y;
  if (blockIdx.x >= A.chunks) {
    zero_part(A, w, blockIdx.x - A.chunks);
    return;
  }
  const uint32_t bins = 1u << A.digit_bits;
  for (uint32_t d = threadIdx.x; d < bins; d += kChunkThreads) count[d] = 0;
  __syncthreads();
#pragma unroll
  for (int j = 0; j < kChunkRounds; ++j) {
    const int64_t r = (int64_t)blockIdx.x * kChunkTokens + j * kChunkThreads + threadIdx.x;
    if (r < A.ntokens) {
      const uint32_t key = FIRST ? key_at<Tok>(A, w, r) : A.keys[(int64_t)w * A.ntokens + r];
      atomicAdd(&count[(key >> shift) & (bins - 1u)], 1u);
    }
  }
  __syncthreads();
  uint32_t* out = A.counts + ((int64_t)w * A.chunks + blockIdx.x) * bins;
  for (uint32_t d = threadIdx.x; d < bins; d += kChunkThreads) out[d] = count[d];
}

// ... second half: the chunk's tokens to their places of the pass.
template <class Tok, bool FIRST>
__global__ __launch_bounds__(kChunkThreads) void k_embed_scatter(EmbedArgs A, int shift) {
  constexpr int kWaves = kChunkThreads / 64, kBins = 1 << kChunkDigit, kEach = kBins / kChunkThreads;
  __shared__ uint32_t count[kWaves][kBins], sums[kWaves];
  const int w = blockIdx.y, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const uint32_t bins = 1u << A.digit_bits, chunk = blockIdx.x;
  const int64_t row = (int64_t)w * A.ntokens;
  uint32_t key[kChunkRounds], place[kChunkRounds], rank[kChunkRounds];
  bool there[kChunkRounds];
#pragma unroll
  for (int j = 0; j < kChunkRounds; ++j) {
    const int64_t r = (int64_t)chunk * kChunkTokens + (wave * kChunkRounds + j) * 64 + lane;
    there[j] = r < A.ntokens;
    key[j] = !there[j] ? 0u : FIRST ? key_at<Tok>(A, w, r) : A.keys[row + r];
    place[j] = FIRST ? (uint32_t)r : there[j] ? A.places[row + r] : 0u;
  }
  for (uint32_t d = lane; d < bins; d += 64) count[wave][d] = 0;
  rank_digits<kChunkRounds>(count[wave], key, there, shift, A.digit_bits, rank);
  // of a thread's digits (next to one another): tokens in all chunks, and in those before this one
  const uint32_t* counts = A.counts + (int64_t)w * A.chunks * bins;
  const uint32_t each = bins >= (uint32_t)kChunkThreads ? bins / kChunkThreads : 1u;
  uint32_t all[kEach] = {}, before[kEach] = {};
  if (threadIdx.x * each < bins)
    for (uint32_t c = 0; c < A.chunks; ++c)
#pragma unroll
      for (int i = 0; i < kEach; ++i)
        if ((uint32_t)i < each) {
          const uint32_t x = counts[(int64_t)c * bins + threadIdx.x * each + i];
          all[i] += x;
          before[i] += c < chunk ? x : 0u;
        }
  uint32_t sum = 0;
#pragma unroll
  for (int i = 0; i < kEach; ++i) sum += all[i];
  uint32_t lower = sum_before<kChunkThreads>(sum, sums);   // (its barriers also close the ranking)
  if (threadIdx.x * each < bins)
#pragma unroll
    for (int i = 0; i < kEach; ++i)
      if ((uint32_t)i < each) {
        uint32_t at = lower + before[i];
        lower += all[i];
        for (int v = 0; v < kWaves; ++v) {
          const uint32_t c = count[v][threadIdx.x * each + i];
          count[v][threadIdx.x * each + i] = at;
          at += c;
        }
      }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < kChunkRounds; ++j)
    if (there[j]) {
      const int64_t at = row + count[wave][(key[j] >> shift) & (bins - 1u)] + rank[j];
      A.keys_next[at] = key[j];
      A.places_next[at] = place[j];
    }
}

// V floats in vectors of at most 16 bytes.
template <int V>
__device__ __forceinline__ void load_sums(const float* p, float (&x)[V]) {
  constexpr int S = V < 4 ? V : 4;
#pragma unroll
  for (int i = 0; i < V; i += S) {
    const Pack<float, S> v = *reinterpret_cast<const Pack<float, S>*>(p + i);
#pragma unroll
    for (int k = 0; k < S; ++k) x[i + k] = v.e[k];
  }
}
template <int V>
__device__ __forceinline__ void store_sums(float* p, const float (&x)[V]) {
  constexpr int S = V < 4 ? V : 4;
#pragma unroll
  for (int i = 0; i < V; i += S) {
    Pack<float, S> v;
#pragma unroll
    for (int k = 0; k < S; ++k) v.e[k] = x[i + k];
    *reinterpret_cast<Pack<float, S>*>(p + i) = v;
  }
}
// scale * sum to (or onto) the gradient.
template <int V>
__device__ __forceinline__ void put_sums(const EmbedArgs& A, int w, uint32_t token, int64_t c, const float (&sum)[V]) {
  float* p = A.dtable + (int64_t)w * A.table_stride + (int64_t)token * A.dim + c;
  float x[V];
#pragma unroll
  for (int i = 0; i < V; ++i) x[i] = sum[i] * A.scale;
  if (A.accumulate) {
    float old[V];
    load_sums<V>(p, old);
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] += old[i];
  }
  store_sums<V>(p, x);
}

// A wave adds up the rows of a piece, for 64 * V columns.  Partial sums: slot 0 of a piece, its first token, where that is also the
// last of the piece before; slot 1, its last token, where that goes on in the next piece (and is not in slot 0).
template <class Row, int V>
__global__ __launch_bounds__(256) void k_embed_sum(EmbedArgs A) {
  const int lane = threadIdx.x & 63, w = blockIdx.y;
  const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int64_t piece = unit / A.column_chunks, c = (unit % A.column_chunks * 64 + lane) * V;
  if (piece >= A.pieces) return;
  const uint32_t* keys = A.keys + (int64_t)w * A.ntokens;
  const int64_t first = piece * kPiece;
  const int count = __builtin_amdgcn_readfirstlane((int)(A.ntokens - first < kPiece ? A.ntokens - first : kPiece));
  // lane l: the l-th token of the piece; lanes kPiece and kPiece + 1: the tokens around it
  const uint32_t none = 0xFFFFFFFFu, vocab = (uint32_t)A.vocab;
  uint32_t key = none, place = 0;
  if (lane < count) {
    key = keys[first + lane];
    place = A.places[(int64_t)w * A.ntokens + first + lane];
  } else if (lane == kPiece && first > 0) {
    key = keys[first - 1];
  } else if (lane == kPiece + 1 && first + count < A.ntokens) {
    key = keys[first + count];
  }
  const uint32_t left = (uint32_t)__builtin_amdgcn_readlane((int)key, kPiece), right = (uint32_t)__builtin_amdgcn_readlane((int)key, kPiece + 1);
  const bool in = c < A.dim;
  const Row* rows = (const Row*)A.rows + (int64_t)w * A.row_stride + (in ? c : 0);
  float* partial = A.partial + ((int64_t)w * A.pieces + piece) * 2 * A.partial_ld + c;
  float sum[V];
#pragma unroll
  for (int i = 0; i < V; ++i) sum[i] = 0.0f;
  uint32_t begun = (uint32_t)__builtin_amdgcn_readlane((int)key, 0);   // the token that `sum` is of
  bool inside = begun != left;                                         // ... and whether it began in this piece
  constexpr int kAhead = 8;
  for (int s = 0; s < count; s += kAhead) {
    Pack<Row, V> x[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int at = s + j < count ? s + j : count - 1;
      const int64_t r = (uint32_t)__builtin_amdgcn_readlane((int)place, at);
      x[j] = *reinterpret_cast<const Pack<Row, V>*>(rows + r * A.row_ld);
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      if (s + j >= count) break;
      const uint32_t k = (uint32_t)__builtin_amdgcn_readlane((int)key, s + j);
      if (k != begun) {
        if (in && begun != vocab) {
          if (inside) put_sums<V>(A, w, begun, c, sum);
          else store_sums<V>(partial, sum);
        }
        begun = k;
        inside = true;
#pragma unroll
        for (int i = 0; i < V; ++i) sum[i] = 0.0f;
      }
#pragma unroll
      for (int i = 0; i < V; ++i) sum[i] += to_float(x[j].e[i]);
    }
    if (begun == vocab) return;   // outside the table, and so are all that follow
  }
  if (!in) return;
  if (inside && begun != right) put_sums<V>(A, w, begun, c, sum);
  else store_sums<V>(inside ? partial + A.partial_ld : partial, sum);
}

// Adds up the partial sums of a token that begins in `piece` and goes on in the next one: a workgroup for 64 * V columns, each wave
// a share of the pieces.
template <int V>
__global__ __launch_bounds__(64 * kJoinWaves) void k_embed_join(EmbedArgs A) {
  __shared__ float sums[kJoinWaves][64][V];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, w = blockIdx.y;
  const int64_t piece = blockIdx.x / A.column_chunks, c = (blockIdx.x % A.column_chunks * 64 + lane) * V;
  const uint32_t* keys = A.keys + (int64_t)w * A.ntokens;
  const int64_t next = (piece + 1) * kPiece;
  if (next >= A.ntokens) return;
  const uint32_t token = keys[next - 1];
  if (token != keys[next] || token == (uint32_t)A.vocab) return;
  const int64_t before = piece * kPiece - 1;
  if (before >= 0 && keys[before] == token) return;     // began earlier
  // pieces that begin with the token
  int64_t reach = 0;
  for (int64_t p = piece + 1;; p += 64) {
    const bool on = (p + lane) * kPiece < A.ntokens && keys[(p + lane) * kPiece] == token;
    const uint64_t all = __ballot(on);
    if (~all) {
      reach += __builtin_ctzll(~all);
      break;
    }
    reach += 64;
  }
  const bool in = c < A.dim;
  const float* partial = A.partial + ((int64_t)w * A.pieces + piece) * 2 * A.partial_ld + (in ? c : 0);
  const int64_t share = reach < 16 ? reach : (reach + kJoinWaves - 1) / kJoinWaves;
  const int64_t from = share * wave < reach ? share * wave : reach, to = from + share < reach ? from + share : reach;
  float sum[V];
#pragma unroll
  for (int i = 0; i < V; ++i) sum[i] = 0.0f;
  if (wave == 0) load_sums<V>(partial + A.partial_ld, sum);
#pragma unroll 4
  for (int64_t p = from; p < to; ++p) {
    float x[V];
    load_sums<V>(partial + (p + 1) * 2 * A.partial_ld, x);
#pragma unroll
    for (int i = 0; i < V; ++i) sum[i] += x[i];
  }
  if (share < reach) {
#pragma unroll
    for (int i = 0; i < V; ++i) sums[wave][lane][i] = sum[i];
    __syncthreads();
    if (wave != 0) return;
    for (int v = 1; v < kJoinWaves; ++v)
#pragma unroll
      for (int i = 0; i < V; ++i) sum[i] += sums[v][lane][i];
  }
  if (wave == 0 && in) put_sums<V>(A, w, token, c, sum);
}

}  // namespace choco
