// Embedding lookup with scaling, and its gradient summed by token (device code).
#pragma once

#include <type_traits>

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
  int digit_bits, passes;
  bool zero_past;                    // cleared past the caches
};

constexpr int kFew = 128;                              // so many tokens are compared with each other instead of ordered
constexpr int kSortThreads = 1024;                     // a workgroup that orders all of a worker's tokens in LDS ...
constexpr int kSortRounds = 8;
constexpr int kSortOne = kSortThreads * kSortRounds;   // ... of which there are no more than this
constexpr int kSortDigit = 9;                          // bits of the key in one pass, at most
constexpr int kChunkThreads = 256;                     // otherwise: a workgroup for each so many tokens ...
// ... times this: more workgroups, but each reads the counts of all chunks, so kLongRounds from kLongLists tokens on.  us, 4 | 16, rows
// of 64 in bf16 added, vocabulary 50,257, one worker: 64 K tokens 36 | 58, 128 K 44 | 63, 256 K 59 | 74, 512 K 94 | 100, 1 M 189 | 144;
// 4 workers: 128 K 75 | 93, 256 K 122 | 122, 512 K 238 | 192; 16: 64 K 114 | 126, 128 K 198 | 197, 256 K 375 | 333; vocabulary 1000, one
// worker: 128 K 38 | 45, 256 K 60 | 60, 512 K 105 | 86; of 1 M words: 60 | 72, 92 | 89, 167 | 126.
constexpr int kShortRounds = 4, kLongRounds = 16;
constexpr int64_t kLongLists = 1 << 18;
constexpr int kChunkDigit = 10;
constexpr int kPiece = 32;                             // ordered tokens that a wave adds up ... (16, 48: within 2 %)
constexpr int kAhead = 8;                              // ... asking for so many rows at once (16: the same)
constexpr int kZeroFloats = 1 << 16;                   // floats that a workgroup clears
constexpr int kJoinWaves = 4;
constexpr int64_t kJoinAlone = 16;                     // partial sums that a wave adds up by itself

// A token, or -1 for one outside the table.
template <class Tok>
__device__ __forceinline__ int32_t token_at(const EmbedArgs& A, int worker, int64_t r) {
  const int64_t t = (int64_t)((const Tok*)A.tokens)[(int64_t)worker * A.token_stride + r];
  return t >= 0 && t < A.vocab ? (int32_t)t : -1;
}

// y[w, r, :] = scale * table[w, token, :].  A group of 2^LANES_LOG2 lanes takes a row, V entries (16 bytes of the wider type, as
// far as rows are aligned) a lane at a time, and asks for kRowAhead such pieces before it writes the first.  Bound by memory: 49,153
// rows of 2048 in bf16 44.3 us (5.9 TB/s), entry by entry 142.
constexpr int kRowAhead = 4;
template <class Tok, class Tab, class Row, int V, bool PAST>
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
      if constexpr (PAST) store_floats_past<Row, V>(to + c + j * step, y);
      else store_floats<Row, V>(to + c + j * step, y);
    }
  }
}

// ---- gradient ----
// 1. The tokens are put in order, stably, by counting on a few bits at a time (key: the token, or vocab for one outside the table);
//    the same launch clears the gradient, which takes longer than the order of an ordinary batch.
// 2. A wave adds up the rows of kPiece consecutive ordered tokens, for 64 * V columns: sums of tokens that lie in the piece
//    as a whole go to the gradient, those that reach over its ends to `partial`.
// 3. The partial sums of a token that spans pieces are added in their order.
// So the rows are split evenly whatever the tokens are (one word in a sixteenth of the places is ordinary), no float is added by
// atomics, and every row of the gradient is written by one wave.
// Bound by memory where the gradient is cleared: 8 x 1120 tokens into 8 x 33,278 x 650 138 us, of which 117 clear 692 MB (5.9 TB/s)
// and hide the order, 12 to 18 add up and 5 join.  Added to what is there: 65,536 tokens of 1024 in bf16 83 us, 26 for
// the order, 49 to add up (5.6 TB/s), 9 to join; 8 x 1120 tokens 26.  A wave per token that looks for its like: 565 and 25,657.
// What does not scale: the partial sums of one token are joined by one workgroup for 64 * V columns, so a token that fills the list
// takes time in proportion (rows of 128 in bf16, all of one token: 64 K 63 us, 1 M 625, 4 M 2,508; 1 M of 1024 1,149 against 708 for
// frequent words); and every chunk of a long list reads the counts of all of them (rows of 64 in bf16, vocabulary 50,257: 1 M
// tokens 144 us, 4 M 467, 16 M 2,770, where reading the rows takes some 450).

// Part `block` of the gradient's clearing, by a whole workgroup.
__device__ __forceinline__ void zero_part(const EmbedArgs& A, int64_t worker, int64_t block) {
  float* base = A.dtable + worker * A.table_stride;
  const float zeros[4] = {};
  const int64_t size = A.vocab * A.dim;
  int64_t from = block * kZeroFloats, to = from + kZeroFloats < size ? from + kZeroFloats : size;
  // whole 16-byte vectors of memory between a few single floats at the ends
  const int64_t lead = (4 - (int64_t)(((uintptr_t)(base + from) >> 2) & 3)) & 3;
  const int64_t first = from + lead < to ? from + lead : to, last = first + (to - first) / 4 * 4;
  for (int64_t i = from + threadIdx.x; i < first; i += blockDim.x) base[i] = 0.0f;
  if (A.zero_past) {
    for (int64_t i = first + 4 * (int64_t)threadIdx.x; i < last; i += 4 * (int64_t)blockDim.x) store_floats_past<float, 4>(base + i, zeros);
  } else {
    for (int64_t i = first + 4 * (int64_t)threadIdx.x; i < last; i += 4 * (int64_t)blockDim.x) store_floats<float, 4>(base + i, zeros);
  }
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
                                            int rounds, int shift, int bits, uint32_t (&rank)[ROUNDS]) {
  const uint64_t before = ((uint64_t)1 << (threadIdx.x & 63)) - 1;
#pragma unroll
  for (int j = 0; j < ROUNDS; ++j) {
    if (j >= rounds) break;
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

inline size_t sort_lds(int64_t tokens, int digit_bits) {
  const size_t rounds = (size_t)((tokens + kSortThreads - 1) / kSortThreads), waves = kSortThreads / 64;
  return (2 * rounds * kSortThreads + waves + ((1 + waves) << digit_bits)) * sizeof(uint32_t);
}

// All of a worker's tokens (no more than kSortOne) in order, in LDS.  Workgroups from the n-th on clear the gradient.
template <class Tok>
__global__ __launch_bounds__(kSortThreads) void k_embed_sort(EmbedArgs A, int workers) {
  constexpr int kWaves = kSortThreads / 64;
  extern __shared__ uint32_t lds[];     // as much as sort_lds says
  if ((int)blockIdx.x >= workers) {
    const uint32_t z = blockIdx.x - workers;
    zero_part(A, z / A.zero_blocks, z % A.zero_blocks);
    return;
  }
  const int w = blockIdx.x, wave = threadIdx.x >> 6, lane = threadIdx.x & 63, total = (int)A.ntokens;
  const int rounds = (total + kSortThreads - 1) / kSortThreads;
  const uint32_t bins = 1u << A.digit_bits;
  uint32_t *keys = lds, *places = keys + rounds * kSortThreads, *base = places + rounds * kSortThreads, *sums = base + bins,
           *counts = sums + kWaves, *count = counts + wave * bins;
  uint32_t key[kSortRounds], place[kSortRounds], rank[kSortRounds];
  bool there[kSortRounds];
#pragma unroll
  for (int j = 0; j < kSortRounds; ++j) {
    const int r = (wave * rounds + j) * 64 + lane;
    there[j] = j < rounds && r < total;
    key[j] = there[j] ? key_at<Tok>(A, w, r) : 0u;
    place[j] = (uint32_t)r;
  }
  for (int pass = 0; pass < A.passes; ++pass) {
    const int shift = pass * A.digit_bits;
    for (uint32_t d = lane; d < bins; d += 64) count[d] = 0;
    rank_digits<kSortRounds>(count, key, there, rounds, shift, A.digit_bits, rank);
    __syncthreads();
    // counters of a wave -> tokens of that digit in the waves before it; base -> tokens of lower digits
    uint32_t sum = 0;
    if (threadIdx.x < bins)
      for (int v = 0; v < kWaves; ++v) {
        const uint32_t c = counts[v * bins + threadIdx.x];
        counts[v * bins + threadIdx.x] = sum;
        sum += c;
      }
    const uint32_t lower = sum_before<kSortThreads>(sum, sums);
    if (threadIdx.x < bins) base[threadIdx.x] = lower;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kSortRounds; ++j)
      if (there[j]) {
        const uint32_t digit = (key[j] >> shift) & (bins - 1u), at = base[digit] + count[digit] + rank[j];
        keys[at] = key[j];
        places[at] = place[j];
      }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kSortRounds; ++j) {
      const int r = (wave * rounds + j) * 64 + lane;
      if (there[j]) {
        key[j] = keys[r];
        place[j] = places[r];
      }
    }
    __syncthreads();
  }
#pragma unroll
  for (int j = 0; j < kSortRounds; ++j) {
    const int r = (wave * rounds + j) * 64 + lane;
    if (there[j]) {
      A.keys[(int64_t)w * A.ntokens + r] = key[j];
      A.places[(int64_t)w * A.ntokens + r] = place[j];
    }
  }
}

// One pass over longer lists, first half: how many tokens of a chunk hold each digit.  Workgroups from the last chunk's on clear
// the gradient.  The first pass reads the tokens, later ones what the one before wrote.
template <class Tok, bool FIRST, int ROUNDS>
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
  for (int j = 0; j < ROUNDS; ++j) {
    const int64_t r = ((int64_t)blockIdx.x * ROUNDS + j) * kChunkThreads + threadIdx.x;
    if (r < A.ntokens) {
      const uint32_t key = FIRST ? key_at<Tok>(A, w, r) : A.keys[(int64_t)w * A.ntokens + r];
      atomicAdd(&count[(key >> shift) & (bins - 1u)], 1u);
    }
  }
  __syncthreads();
  uint32_t* out = A.counts + ((int64_t)w * A.chunks + blockIdx.x) * bins;
  for (uint32_t d = threadIdx.x; d < bins; d += kChunkThreads) out[d] = count[d];
}

// ... second half: the tokens of a chunk to their places.  Each workgroup adds up the counts of all chunks for itself, four digits a
// thread and eight chunks at once, where the threads are more than a quarter of the digits groups of them a share of the chunks.
template <class Tok, bool FIRST, int ROUNDS>
__global__ __launch_bounds__(kChunkThreads) void k_embed_scatter(EmbedArgs A, int shift) {
  constexpr int kWaves = kChunkThreads / 64, kBins = 1 << kChunkDigit, kAtOnce = 8;
  static_assert(kBins == 4 * kChunkThreads, "four digits a thread");
  __shared__ uint32_t count[kWaves][kBins], sums[kWaves];
  __shared__ uint4 all[kChunkThreads], before[kChunkThreads];
  const int w = blockIdx.y, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const uint32_t bins = 1u << A.digit_bits, chunk = blockIdx.x, quads = bins / 4;
  const int64_t row = (int64_t)w * A.ntokens;
  uint32_t key[ROUNDS], place[ROUNDS], rank[ROUNDS];
  bool there[ROUNDS];
#pragma unroll
  for (int j = 0; j < ROUNDS; ++j) {
    const int64_t r = (int64_t)chunk * (ROUNDS * kChunkThreads) + (wave * ROUNDS + j) * 64 + lane;
    there[j] = r < A.ntokens;
    key[j] = !there[j] ? 0u : FIRST ? key_at<Tok>(A, w, r) : A.keys[row + r];
    place[j] = FIRST ? (uint32_t)r : there[j] ? A.places[row + r] : 0u;
  }
  const uint32_t group = threadIdx.x / quads, groups = kChunkThreads / quads;
  const uint4* counts = reinterpret_cast<const uint4*>(A.counts + (int64_t)w * A.chunks * bins) + threadIdx.x % quads;
  uint4 sum_all = make_uint4(0, 0, 0, 0), sum_earlier = sum_all;
  for (uint32_t c = group; c < A.chunks; c += kAtOnce * groups) {
    uint4 x[kAtOnce];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const uint32_t from = c + k * groups;
      x[k] = counts[(int64_t)(from < A.chunks ? from : A.chunks - 1) * quads];
    }
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const uint32_t from = c + k * groups;
      const uint32_t mask = from < A.chunks ? 0xFFFFFFFFu : 0u, mask_before = from < chunk ? 0xFFFFFFFFu : 0u;
      sum_all.x += x[k].x & mask;
      sum_all.y += x[k].y & mask;
      sum_all.z += x[k].z & mask;
      sum_all.w += x[k].w & mask;
      sum_earlier.x += x[k].x & mask_before;
      sum_earlier.y += x[k].y & mask_before;
      sum_earlier.z += x[k].z & mask_before;
      sum_earlier.w += x[k].w & mask_before;
    }
  }
  all[threadIdx.x] = sum_all;
  before[threadIdx.x] = sum_earlier;
  for (uint32_t d = lane; d < bins; d += 64) count[wave][d] = 0;
  rank_digits<ROUNDS>(count[wave], key, there, ROUNDS, shift, A.digit_bits, rank);
  __syncthreads();
  uint32_t mine[4] = {}, earlier[4] = {};     // of digits 4 t ... 4 t + 3
  if (threadIdx.x < quads)
    for (uint32_t g = 0; g < groups; ++g) {
      const uint4 a = all[g * quads + threadIdx.x], b = before[g * quads + threadIdx.x];
      mine[0] += a.x, mine[1] += a.y, mine[2] += a.z, mine[3] += a.w;
      earlier[0] += b.x, earlier[1] += b.y, earlier[2] += b.z, earlier[3] += b.w;
    }
  uint32_t lower = sum_before<kChunkThreads>(mine[0] + mine[1] + mine[2] + mine[3], sums);
  if (threadIdx.x < quads)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t at = lower + earlier[i];
      lower += mine[i];
#pragma unroll
      for (int v = 0; v < kWaves; ++v) {
        const uint32_t c = count[v][threadIdx.x * 4 + i];
        count[v][threadIdx.x * 4 + i] = at;
        at += c;
      }
    }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < ROUNDS; ++j)
    if (there[j]) {
      const int64_t at = row + count[wave][(key[j] >> shift) & (bins - 1u)] + rank[j];
      A.keys_next[at] = key[j];
      A.places_next[at] = place[j];
    }
}

// A lane's columns of a row: registers of one entry of 32 bits, or two or one of 16.  (The words are taken apart where they are used:
// a load of 16-bit floats would lose its way past the caches in the compiler.)
template <class Row, int V>
struct RowWords {
  static constexpr int kWords = sizeof(Row) == 4 ? V : 1;
  using Word = std::conditional_t<V * sizeof(Row) == 2, uint16_t, uint32_t>;
  typedef Word Words __attribute__((ext_vector_type(kWords)));
  Words words;
  template <bool PAST>
  __device__ __forceinline__ void load(const Row* p) {
    if constexpr (PAST) words = __builtin_nontemporal_load(reinterpret_cast<const Words*>(p));
    else words = *reinterpret_cast<const Words*>(p);
  }
  __device__ __forceinline__ float at(int i) const { return sizeof(Row) == 4 ? entry<Row>(words[i], 0) : entry<Row>(words[0], i); }
};
__device__ __forceinline__ float* sums_of(const EmbedArgs& A, int w, uint32_t token, int64_t c) {
  return A.dtable + (int64_t)w * A.table_stride + (int64_t)token * A.dim + c;
}
// scale * sum to (ADD: onto `old`, what is there) the gradient.
template <bool ADD, bool PAST, int V>
__device__ __forceinline__ void put_sums(const EmbedArgs& A, float* p, const float (&sum)[V], const float (&old)[V]) {
  float x[V];
#pragma unroll
  for (int i = 0; i < V; ++i) x[i] = ADD ? sum[i] * A.scale + old[i] : sum[i] * A.scale;
  if constexpr (PAST) store_floats_past<float, V>(p, x);
  else store_floats<float, V>(p, x);
}

// A wave adds up the rows of a piece, for 64 * V columns.  Partial sums: slot 0 of a piece, its first token, where that is also the
// last of the piece before; slot 1, its last token, where that goes on in the next piece (and is not in slot 0).
template <class Row, int V, bool ADD, bool PAST>
__global__ __launch_bounds__(256) void k_embed_sum(EmbedArgs A) {
  const int lane = threadIdx.x & 63, w = blockIdx.y;
  const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int64_t piece = unit / A.column_chunks, c = (unit % A.column_chunks * 64 + lane) * V;
  if (piece >= A.pieces) return;
  const uint32_t* keys = A.keys + (int64_t)w * A.ntokens;
  const int64_t first = piece * kPiece;
  const int count = __builtin_amdgcn_readfirstlane((int)(A.ntokens - first < kPiece ? A.ntokens - first : kPiece));
  // lane l: the (l - 1)-th token of the piece; lanes 0 and count + 1: those around it
  const uint32_t none = 0xFFFFFFFFu, vocab = (uint32_t)A.vocab;
  const int64_t r = first + lane - 1;
  const uint32_t key = lane <= count + 1 && r >= 0 && r < A.ntokens ? keys[r] : none;
  const uint32_t place = lane >= 1 && lane <= count ? A.places[(int64_t)w * A.ntokens + r] : 0u;
  const uint32_t after = (uint32_t)__shfl_down((int)key, 1, 64), ahead = (uint32_t)__shfl_up((int)key, 1, 64);
  // tokens after which another one begins (or the piece ends); those, of these, whose sum is complete
  const uint64_t ends = __ballot(lane >= 1 && lane <= count && (key != after || lane == count));
  const uint64_t starts = __ballot(lane >= 1 && lane <= count && key != ahead);
  const int here = __builtin_amdgcn_readfirstlane(__popcll(__ballot(lane >= 1 && lane <= count && key != vocab)));   // in the table
  if (here == 0) return;
  const bool in = c < A.dim;
  const int64_t column = in ? c : 0;
  const Row* rows = (const Row*)A.rows + (int64_t)w * A.row_stride + column;
  float* partial = A.partial + ((int64_t)w * A.pieces + piece) * 2 * A.partial_ld + column;
  const uint32_t right = (uint32_t)__builtin_amdgcn_readlane((int)key, count + 1);
  float sum[V];
#pragma unroll
  for (int i = 0; i < V; ++i) sum[i] = 0.0f;
  bool inside = starts >> 1 & 1;     // the token that `sum` is of began in this piece
  for (int s = 0; s < here; s += kAhead) {
    RowWords<Row, V> x[kAhead];
    float old[kAhead][V];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int at = (s + j < here ? s + j : here - 1) + 1;
      const int64_t p = (uint32_t)__builtin_amdgcn_readlane((int)place, at);
      x[j].template load<PAST>(rows + p * A.row_ld);
      if (ADD && (ends >> at & 1)) load_floats<float, V>(sums_of(A, w, (uint32_t)__builtin_amdgcn_readlane((int)key, at), column), old[j]);
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      if (s + j >= here) break;
      const int at = s + j + 1;
#pragma unroll
      for (int i = 0; i < V; ++i) sum[i] += x[j].at(i);
      if (!(ends >> at & 1)) continue;
      const uint32_t token = (uint32_t)__builtin_amdgcn_readlane((int)key, at);
      const bool goes_on = at == count && token == right;
      if (in) {
        if (inside && !goes_on) put_sums<ADD, PAST, V>(A, sums_of(A, w, token, column), sum, old[j]);
        else store_floats<float, V>(inside ? partial + A.partial_ld : partial, sum);
      }
      inside = true;
#pragma unroll
      for (int i = 0; i < V; ++i) sum[i] = 0.0f;
    }
  }
}

// A few tokens (no more than kFew): a wave for each of them and 64 * V columns.  The first of its kind adds up the rows of all of
// its kind, in their order.  One launch instead of three: 64 tokens of 512 added 17.3 -> 6.0 us, 8 x 128 19.2 -> 5.9; of 128 tokens that are all the
// same one wave adds up 128 rows, eight at a time (13.5 -> 10.4).
template <class Tok, class Row, int V, bool ADD>
__global__ __launch_bounds__(256) void k_embed_few(EmbedArgs A) {
  const int lane = threadIdx.x & 63, w = blockIdx.y;
  const int64_t unit = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (unit >= A.ntokens * A.column_chunks) return;
  const int r = (int)(unit / A.column_chunks);
  const int64_t c = (unit % A.column_chunks * 64 + lane) * V;
  const int32_t low = lane < A.ntokens ? token_at<Tok>(A, w, lane) : -1, high = lane + 64 < A.ntokens ? token_at<Tok>(A, w, lane + 64) : -1;
  const int32_t token = r < 64 ? __builtin_amdgcn_readlane(low, r) : __builtin_amdgcn_readlane(high, r - 64);
  if (token < 0) return;
  uint64_t same_low = __ballot(low == token), same_high = __ballot(high == token);
  if (r < 64 ? (same_low & (((uint64_t)1 << r) - 1)) != 0 : (same_low | (same_high & (((uint64_t)1 << (r - 64)) - 1))) != 0) return;
  const bool in = c < A.dim;
  const int64_t column = in ? c : 0;
  const Row* rows = (const Row*)A.rows + (int64_t)w * A.row_stride + column;
  float sum[V], old[V];
  if (ADD) load_floats<float, V>(sums_of(A, w, (uint32_t)token, column), old);
#pragma unroll
  for (int i = 0; i < V; ++i) sum[i] = 0.0f;
  int left = __popcll(same_low) + __popcll(same_high), at = r;
  for (; left > 0; left -= kAhead) {
    RowWords<Row, V> x[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {     // (where none is left: the last one again)
      if (same_low) {
        at = __builtin_ctzll(same_low);
        same_low &= same_low - 1;
      } else if (same_high) {
        at = 64 + __builtin_ctzll(same_high);
        same_high &= same_high - 1;
      }
      x[j].template load<false>(rows + at * A.row_ld);
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
#pragma unroll
      for (int i = 0; i < V; ++i) sum[i] += j < left ? x[j].at(i) : 0.0f;
  }
  if (in) put_sums<ADD, false, V>(A, sums_of(A, w, (uint32_t)token, column), sum, old);
}

// The sum of V columns of partial sums (slot 0) from piece `from` to before `to`, onto `sum`.
template <int V>
__device__ __forceinline__ void add_pieces(const float* partial, int64_t partial_ld, int64_t from, int64_t to, float (&sum)[V]) {
#pragma unroll 8
  for (int64_t p = from; p < to; ++p) {
    float x[V];
    load_floats<float, V>(partial + p * 2 * partial_ld, x);
#pragma unroll
    for (int i = 0; i < V; ++i) sum[i] += x[i];
  }
}

// Adds up the partial sums of the tokens that span pieces.  A wave looks at a piece (for 64 * V columns): if a token begins there and
// goes on in the next one, it adds up its partial sums, unless there are many; those the workgroup's waves share.  (Its waves look at
// neighbouring pieces, of which few begin a token with many.)
template <int V, bool ADD>
__global__ __launch_bounds__(64 * kJoinWaves) void k_embed_join(EmbedArgs A) {
  __shared__ float sums[kJoinWaves][64][V];
  __shared__ int64_t many[kJoinWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, w = blockIdx.y;
  const uint32_t* keys = A.keys + (int64_t)w * A.ntokens;
  const float* partial = A.partial + (int64_t)w * A.pieces * 2 * A.partial_ld;
  const int64_t units = A.pieces * A.column_chunks, first = (int64_t)blockIdx.x * kJoinWaves;
  {
    const int64_t piece = (first + wave) % A.pieces, next = (piece + 1) * kPiece, before = piece * kPiece - 1;
    const int64_t c = ((first + wave) / A.pieces * 64 + lane) * V;
    int64_t reach = 0;     // pieces after this one that begin with the token
    uint32_t token = 0;
    if (first + wave < units && next < A.ntokens) {
      const uint32_t after = keys[next], left = before >= 0 ? keys[before] : 0xFFFFFFFFu;
      token = keys[next - 1];
      if (token == after && token != left && token != (uint32_t)A.vocab)
        for (int64_t p = piece + 1;; p += 64) {
          const bool on = (p + lane) * kPiece < A.ntokens && keys[(p + lane) * kPiece] == token;
          const uint64_t all = __ballot(on);
          if (~all) {
            reach += __builtin_ctzll(~all);
            break;
          }
          reach += 64;
        }
    }
    if (lane == 0) many[wave] = reach >= kJoinAlone ? reach : 0;
    if (reach > 0 && reach < kJoinAlone && c < A.dim) {
      float sum[V], old[V];
      if (ADD) load_floats<float, V>(sums_of(A, w, token, c), old);
      load_floats<float, V>(partial + (piece * 2 + 1) * A.partial_ld + c, sum);
      add_pieces<V>(partial + c, A.partial_ld, piece + 1, piece + 1 + reach, sum);
      put_sums<ADD, false, V>(A, sums_of(A, w, token, c), sum, old);
    }
  }
  __syncthreads();
  for (int v = 0; v < kJoinWaves; ++v) {
    const int64_t reach = many[v];
    if (reach == 0) continue;
    const int64_t piece = (first + v) % A.pieces, share = (reach + kJoinWaves - 1) / kJoinWaves;
    const int64_t c = ((first + v) / A.pieces * 64 + lane) * V, column = c < A.dim ? c : 0;
    const int64_t from = share * wave < reach ? share * wave : reach, to = from + share < reach ? from + share : reach;
    float sum[V];
#pragma unroll
    for (int i = 0; i < V; ++i) sum[i] = 0.0f;
    if (wave == 0) load_floats<float, V>(partial + (piece * 2 + 1) * A.partial_ld + column, sum);
    add_pieces<V>(partial + column, A.partial_ld, piece + 1 + from, piece + 1 + to, sum);
#pragma unroll
    for (int i = 0; i < V; ++i) sums[wave][lane][i] = sum[i];
    __syncthreads();
    if (wave == 0 && c < A.dim) {
      float old[V];
      float* to_row = sums_of(A, w, keys[(piece + 1) * kPiece], c);
      if (ADD) load_floats<float, V>(to_row, old);
#pragma unroll
      for (int u = 1; u < kJoinWaves; ++u)
#pragma unroll
        for (int i = 0; i < V; ++i) sum[i] += sums[u][lane][i];
      put_sums<ADD, false, V>(A, to_row, sum, old);
    }
    __syncthreads();
  }
}

}  // namespace choco
