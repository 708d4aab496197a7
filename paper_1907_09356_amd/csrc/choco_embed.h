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
};

// A token, or -1 for one outside the table.
template <class Tok>
__device__ __forceinline__ int32_t token_at(const EmbedArgs& A, int worker, int64_t r) {
  const int64_t t = (int64_t)((const Tok*)A.tokens)[(int64_t)worker * A.token_stride + r];
  return t >= 0 && t < A.vocab ? (int32_t)t : -1;
}

// y[w, r, :] = scale * table[w, token, :].  A group of 2^LANES_LOG2 lanes takes a row, V entries a lane at a time.
template <class Tok, class Tab, class Row, int V>
__global__ __launch_bounds__(256) void k_embed(EmbedArgs A, int lanes_log2) {
  const int lane = threadIdx.x & ((1 << lanes_log2) - 1);
  const int64_t r = (int64_t)blockIdx.x * (256 >> lanes_log2) + (threadIdx.x >> lanes_log2);
  const int w = blockIdx.y;
  if (r >= A.ntokens) return;
  const int32_t t = token_at<Tok>(A, w, r);
  const Tab* from = (const Tab*)A.table + (int64_t)w * A.table_stride + (int64_t)(t < 0 ? 0 : t) * A.dim;
  Row* to = (Row*)A.rows + (int64_t)w * A.row_stride + r * A.row_ld;
  for (int64_t c = (int64_t)lane * V; c < A.dim; c += (int64_t)V << lanes_log2) {
    float x[V];
    if (t >= 0) {
      load_floats<Tab, V>(from + c, x);
#pragma unroll
      for (int i = 0; i < V; ++i) x[i] *= A.scale;
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) x[i] = 0.0f;
    }
    store_floats<Row, V>(to + c, x);
  }
}

// dtable = 0.
__global__ __launch_bounds__(256) void k_embed_zero(EmbedArgs A) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i < A.vocab * A.dim) A.dtable[(int64_t)blockIdx.y * A.table_stride + i] = 0.0f;
}

// A wave per token: the first of its kind adds up the rows of all of its kind, in their order.
template <class Tok, class Row>
__global__ __launch_bounds__(64) void k_embed_sum(EmbedArgs A) {
  const int w = blockIdx.y, lane = threadIdx.x;
  const int64_t r = blockIdx.x;
  const int32_t t = token_at<Tok>(A, w, r);
  if (t < 0) return;
  for (int64_t at = 0; at < r; at += 64) {
    const bool same = at + lane < r && token_at<Tok>(A, w, at + lane) == t;
    if (__ballot(same)) return;
  }
  const Row* rows = (const Row*)A.rows + (int64_t)w * A.row_stride;
  float* to = A.dtable + (int64_t)w * A.table_stride + (int64_t)t * A.dim;
  for (int64_t c = 0; c < A.dim; c += 64) {
    const bool in = c + lane < A.dim;
    float sum = 0.0f;
    for (int64_t at = r; at < A.ntokens; at += 64) {
      uint64_t same = __ballot(at + lane < A.ntokens && token_at<Tok>(A, w, at + lane) == t);
      while (same) {
        const int64_t s = at + __builtin_ctzll(same);
        same &= same - 1;
        if (in) sum += to_float(rows[s * A.row_ld + c + lane]);
      }
    }
    if (in) to[c + lane] += sum * A.scale;
  }
}

}  // namespace choco
