// Host side of the C ABI declared in include/choco_train.h: argument checks, workspace layout, kernel
// launches.  No device memory is allocated here; only choco_adamw_init waits for the device.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <initializer_list>
#include <new>
#include <type_traits>
#include <utility>
#include <vector>

#include "choco_train.h"
#include "choco_host.h"
#include "choco_adamw.h"
#include "choco_embed.h"
#include "choco_recur.h"

using namespace choco;

namespace {

// ---- embedding ----

int check_embed(const choco_embed_config* c) {
  if (!c) return CHOCO_E_INVAL;
  if (c->n < 0 || c->n > 65535 || c->tokens < 0 || c->tokens >= kMaxIndex || c->vocab < 1 || c->vocab >= kMaxIndex ||
      c->dim < 0 || c->dim >= kMaxIndex)
    return CHOCO_E_INVAL;
  if ((c->token_type != CHOCO_I32 && c->token_type != CHOCO_I64) || !type_bytes(c->table_type) || !type_bytes(c->row_type))
    return CHOCO_E_INVAL;
  if (c->token_stride < c->tokens || c->row_ld < c->dim || c->row_ld >= kMaxIndex || c->table_stride < c->vocab * c->dim ||
      c->row_stride < c->tokens * c->row_ld)
    return CHOCO_E_INVAL;
  const int64_t most = kMaxExtent / (c->n > 0 ? c->n : 1);
  if (c->token_stride > most || c->table_stride > most || c->row_stride > most) return CHOCO_E_INVAL;
  return CHOCO_OK;
}

// The gradient's partial sums take a sixteenth of the rows' entries in fp32: below 2^50 bytes with any number of workers.
bool embed_fits(const choco_embed_config& c) {
  return (double)c.n * ((double)c.tokens + kPiece) * ((double)c.dim + 8.0) < 1125899906842624.0;
}

EmbedArgs embed_args(const choco_embed_config& c, const void* tokens) {
  EmbedArgs A{};
  A.tokens = tokens;
  A.ntokens = c.tokens;
  A.vocab = c.vocab;
  A.dim = c.dim;
  A.token_stride = c.token_stride;
  A.table_stride = c.table_stride;
  A.row_stride = c.row_stride;
  A.row_ld = c.row_ld;
  A.scale = c.scale;
  return A;
}

// How the gradient's tokens are put in order, and where its workspace lies.
struct EmbedLayout {
  size_t keys, places, keys_next, places_next, counts, partial, total;
  int64_t pieces, partial_ld;
  uint32_t chunks;
  int digit_bits, passes, rounds;
  bool one;    // a workgroup orders all of a worker's tokens
};

EmbedLayout embed_layout(const choco_embed_config& c) {
  EmbedLayout L{};
  if (c.n == 0 || c.tokens <= kFew || c.dim == 0) return L;
  L.one = c.tokens <= kSortOne;
  int bits = 1;
  while (c.vocab >> bits) ++bits;    // keys go up to vocab itself
  const int most = L.one ? kSortDigit : kChunkDigit;
  L.passes = (bits + most - 1) / most;
  L.digit_bits = std::max(2, (bits + L.passes - 1) / L.passes);
  L.rounds = c.tokens < kLongLists ? kShortRounds : kLongRounds;
  L.chunks = blocks_of(c.tokens, kChunkThreads * L.rounds);
  L.pieces = (c.tokens + kPiece - 1) / kPiece;
  L.partial_ld = (c.dim + 7) / 8 * 8;
  size_t at = 0;
  const auto take = [&](size_t bytes) {
    const size_t here = at;
    at = (at + bytes + 255) / 256 * 256;
    return here;
  };
  const size_t list = (size_t)c.n * (size_t)c.tokens * sizeof(uint32_t);
  L.keys = take(list);
  L.places = take(list);
  if (!L.one) {
    L.keys_next = take(list);
    L.places_next = take(list);
    L.counts = take(((size_t)c.n * L.chunks << L.digit_bits) * sizeof(uint32_t));
  }
  L.partial = take((size_t)c.n * (size_t)L.pieces * 2 * (size_t)L.partial_ld * sizeof(float));
  L.total = at;
  return L;
}

// Entries that a lane moves at once: most, most / 2, ... or 1, as rows and strides are aligned.
int embed_width(int most, int64_t dim, std::initializer_list<std::pair<const void*, size_t>> pointers,
                std::initializer_list<std::pair<int64_t, size_t>> strides) {
  for (int v = most; v > 1; v /= 2) {
    bool ok = dim % v == 0;
    for (const auto& p : pointers) ok = ok && aligned_to(p.first, std::min<size_t>(v * p.second, 16));
    for (const auto& s : strides) ok = ok && (size_t)s.first * s.second % std::min<size_t>(v * s.second, 16) == 0;
    if (ok) return v;
  }
  return 1;
}

// calls fn with the width as a type's value
template <class Fn>
void with_vector(int v, Fn&& fn) {
  if (v == 8) fn(std::integral_constant<int, 8>{});
  else if (v == 4) fn(std::integral_constant<int, 4>{});
  else if (v == 2) fn(std::integral_constant<int, 2>{});
  else fn(std::integral_constant<int, 1>{});
}

// ---- recurrence ----

bool strides_ok(const choco_recur_config& c, const int64_t s[2], bool output) {
  if (s[0] < 0 || s[1] < 0 || s[0] > kMaxExtent || s[1] > kMaxExtent) return false;
  const double extent = (double)s[0] * (double)(c.batch - 1) + (double)s[1] * (double)(c.steps - 1) + (double)c.dim;
  if (extent > (double)kMaxExtent) return false;
  if (!output) return true;
  // entries of an output apart: sequence after sequence, or step after step
  const bool one_seq = c.batch <= 1, one_step = c.steps <= 1;
  const bool by_seq = (one_step || s[1] >= c.dim) && (one_seq || (double)s[0] >= (double)s[1] * (double)(c.steps - 1) + (double)c.dim);
  const bool by_step = (one_seq || s[0] >= c.dim) && (one_step || (double)s[1] >= (double)s[0] * (double)(c.batch - 1) + (double)c.dim);
  return by_seq || by_step;
}

int check_recur(const choco_recur_config* c) {
  if (!c) return CHOCO_E_INVAL;
  if (c->batch < 0 || c->steps < 0 || c->dim < 0 || c->batch >= kMaxIndex || c->steps >= kMaxIndex || c->dim >= kMaxIndex)
    return CHOCO_E_INVAL;
  const int64_t most = (int64_t)1 << 40;
  if (c->batch * c->dim >= most || c->batch * c->steps >= most) return CHOCO_E_INVAL;
  if (!type_bytes(c->type)) return CHOCO_E_INVAL;
  return CHOCO_OK;
}

RecurArgs recur_args(const choco_recur_config& c, const void* f, const void* u, const void* o, const int32_t* lengths) {
  RecurArgs A{};
  A.f = f; A.u = u; A.o = o;
  A.lengths = lengths;
  A.batch = c.batch; A.steps = c.steps; A.dim = c.dim;
  A.f_seq = c.f_stride[0]; A.f_step = c.f_stride[1];
  A.u_seq = c.u_stride[0]; A.u_step = c.u_stride[1];
  A.o_seq = c.o_stride[0]; A.o_step = c.o_stride[1];
  A.y_seq = c.y_stride[0]; A.y_step = c.y_stride[1];
  A.df_seq = c.df_stride[0]; A.df_step = c.df_stride[1];
  A.du_seq = c.du_stride[0]; A.du_step = c.du_stride[1];
  A.do_seq = c.do_stride[0]; A.do_step = c.do_stride[1];
  return A;
}

// Channels a lane takes at once: two of 16 bits where everything is aligned to that.
bool recur_pairs(const choco_recur_config& c, bool gated, bool back, std::initializer_list<const void*> pointers) {
  if (c.type == CHOCO_F32 || c.dim % 2) return false;
  uint64_t all = (uint64_t)(c.f_stride[0] | c.f_stride[1] | c.u_stride[0] | c.u_stride[1] | c.y_stride[0] | c.y_stride[1]);
  if (gated) all |= (uint64_t)(c.o_stride[0] | c.o_stride[1]);
  if (back) all |= (uint64_t)(c.df_stride[0] | c.df_stride[1] | c.du_stride[0] | c.du_stride[1]);
  if (back && gated) all |= (uint64_t)(c.do_stride[0] | c.do_stride[1]);
  if (all & 1) return false;
  for (const void* p : pointers)
    if (!aligned_to(p, 4)) return false;
  return true;
}

// Chains of tiles (see choco_recur.h) for strips of `width` channels, a wave of a chain taking so many steps.
struct RecurPlan {
  int64_t strips, chains, tiles, links;
  int waves;
};

RecurPlan plan_recur(const choco_recur_config& c, int width, int steps) {
  RecurPlan P{};
  P.strips = (c.dim + width - 1) / width;
  P.chains = P.strips * c.batch;
  P.waves = (int)std::max<int64_t>(1, (c.steps + kAloneSteps - 1) / kAloneSteps);
  P.tiles = 1;
  if (c.steps > kAloneSteps * kRecurWaves) {
    P.waves = kChainWaves;
    const int64_t tile = (int64_t)P.waves * steps;
    P.tiles = (c.steps + tile - 1) / tile;
  }
  P.links = (P.tiles + kChainTiles - 1) / kChainTiles;
  return P;
}

// Words of a chain's maps and states, and of the whole workspace with the counters.
double chain_words(const RecurPlan& P, int width) { return P.tiles > 1 ? (double)P.chains * (double)(P.tiles + P.links) * width : 0.0; }

// A call's launches hold it, whichever way it is split.
bool recur_fits(const choco_recur_config& c) {
  for (int v : {1, 2})
    for (int steps : {kForwardSteps, back_steps(v)}) {
      const RecurPlan P = plan_recur(c, 64 * v, steps);
      if (!launch_fits((double)P.chains * (double)P.tiles, 64 * P.waves)) return false;
    }
  return true;
}

size_t recur_workspace(const choco_recur_config& c) {
  // (a call takes the wide strips or the narrow ones, whatever its pointers allow: room for either, and for both passes)
  size_t most = 0;
  for (int v : {1, 2})
    for (int steps : {kForwardSteps, back_steps(v)}) {
      const RecurPlan P = plan_recur(c, 64 * v, steps);
      if (P.tiles > 1) most = std::max(most, (size_t)chain_words(P, 64 * v) * sizeof(uint64_t) + (size_t)P.chains * kTakenWords * sizeof(uint32_t));
    }
  return most;
}

// The launch of a call.
void place_recur(const choco_recur_config& c, int width, int steps, void* workspace, RecurArgs& A, dim3& grid, int& threads) {
  const RecurPlan P = plan_recur(c, width, steps);
  threads = 64 * P.waves;
  A.strips = (uint32_t)P.strips;
  A.chains = (uint32_t)P.chains;
  A.tiles = (uint32_t)P.tiles;
  A.links = (uint32_t)P.links;
  A.maps = (uint64_t*)workspace;
  A.states = A.maps + P.chains * P.tiles * width;
  A.taken = (uint32_t*)(A.states + P.chains * P.links * width);
  grid = dim3((uint32_t)(P.chains * P.tiles));
}

// Launches what starts the chains (`first`: the states before them) of a call that has any.
void start_chains(const RecurArgs& A, int width, const float* first, hipStream_t stream) {
  const double words = (double)A.chains * (A.tiles + A.links) * width + A.chains;
  k_recur_chains<<<dim3((uint32_t)std::min(2048.0, words / 256 + 1)), 256, 0, stream>>>(A, first, width);
}

// Past the caches?  A call moves `arrays` arrays of batch x steps x dim.  Small results are left in the caches for what reads them
// next.  us, through the caches | results past them | all past them: forward, MB moved 134 33.5 | 32.6 | 34.5, 335 77 | 61 | 69,
// 872 232 | 224 | 210; backward 235 52.0 | 51.1 | 58.6, 587 137 | 129 | 124, 839 228 | 214 | 202.  Tiles alone: 100 22 | 27 | 33.
int recur_mode(const choco_recur_config& c, const RecurArgs& A, int arrays) {
  if (A.tiles <= 1) return kAlone;
  const double mib = (double)c.batch * (double)c.steps * (double)c.dim * type_bytes(c.type) * arrays / 1048576.0;
  return mib > 384.0 ? kPast : mib > 128.0 ? kPastOut : kThrough;
}
template <class Fn>
void with_mode(int mode, Fn&& fn) {
  if (mode == kAlone) fn(std::integral_constant<int, kAlone>{});
  else if (mode == kThrough) fn(std::integral_constant<int, kThrough>{});
  else if (mode == kPastOut) fn(std::integral_constant<int, kPastOut>{});
  else fn(std::integral_constant<int, kPast>{});
}

// calls fn with the channels a lane takes (a type's only where it can be two)
template <class T, class Fn>
void with_width(bool pairs, Fn&& fn) {
  if constexpr (sizeof(T) == 2) {
    if (pairs) return fn(std::integral_constant<int, 2>{});
  }
  fn(std::integral_constant<int, 1>{});
}

static_assert(kSaveSteps == CHOCO_RECUR_SAVE_STEPS, "the header says what is kept");

// (of a call that its launches hold: far from 64 bits)
int64_t saved_floats(const choco_recur_config& c) {
  return (c.steps + CHOCO_RECUR_SAVE_STEPS - 1) / CHOCO_RECUR_SAVE_STEPS * c.batch * c.dim;
}

// ---- AdamW ----

struct AdamwLayout {
  size_t state, m, v, m_scale, v_scale, state_end, tiles, total;
  int64_t ntiles, nblocks, ngaps;
};

int64_t resolve_adamw_ld(const choco_adamw_config& c) { return c.ld == 0 ? (c.d + 3) / 4 * 4 : c.ld; }

int check_adamw(const choco_adamw_config* c) {
  if (!c) return CHOCO_E_INVAL;
  if (c->n < 1 || c->n > 65535 || c->d < 1 || c->d > CHOCO_MAX_D) return CHOCO_E_INVAL;
  const int64_t ld = resolve_adamw_ld(*c);
  if (ld < c->d || (ld & 3) != 0 || ld > kMaxIndex) return CHOCO_E_INVAL;
  if (!(c->beta1 >= 0.0 && c->beta1 < 1.0) || !(c->beta2 >= 0.0 && c->beta2 < 1.0)) return CHOCO_E_INVAL;
  if ((float)c->beta1 >= 1.0f || (float)c->beta2 >= 1.0f) return CHOCO_E_INVAL;
  if (!(c->eps >= kLeastEps / std::sqrt(1.0 - c->beta2)) || !std::isfinite((float)c->eps)) return CHOCO_E_INVAL;
  if (c->state_bits != 32 && c->state_bits != 8) return CHOCO_E_INVAL;
  if (c->ntensors < 0 || (c->ntensors > 0 && (!c->start_host || !c->len_host))) return CHOCO_E_INVAL;
  const int32_t rows = c->ntensors > 0 ? c->ntensors : 1;
  int64_t end = 0;
  for (int32_t t = 0; t < c->ntensors; ++t) {
    const int64_t start = c->start_host[t], len = c->len_host[t];
    if (start < end || len < 0 || start > c->d || len > c->d - start) return CHOCO_E_INVAL;
    end = start + len;
  }
  for (int32_t t = 0; t < rows; ++t) {
    if (c->weight_decay_host && !(c->weight_decay_host[t] >= 0.0f && std::isfinite(c->weight_decay_host[t]))) return CHOCO_E_INVAL;
    if (c->lr_scale_host && !std::isfinite(c->lr_scale_host[t])) return CHOCO_E_INVAL;
  }
  return CHOCO_OK;
}

// Loads and stores past the caches?  Where x, g, m and v do not stay in the 256 MB of the last-level cache until the next step.
// us a step, through | past the caches: 32 bits, entries 2.2 M 15 | 16, 4 M 21 | 25, 8 M 37 | 42, 16 M 68 | 78, 32 M 172 | 152,
// 254 M 1379 | 1319; 8 bits, with the moments read back, 2.2 M 17 | 19, 16 M 69 | 70, 32 M 125 | 128, 127 M 607 | 486.
bool adamw_streams(const choco_adamw_config& c) {
  return (double)c.n * (double)resolve_adamw_ld(c) * (8 + c.state_bits / 4) > 320.0 * 1048576.0;
}

// calls fn(tensor, start, len) for every tensor
template <class Fn>
void for_tensors(const choco_adamw_config& c, Fn&& fn) {
  if (c.ntensors == 0) fn(0, (int64_t)0, c.d);
  for (int32_t t = 0; t < c.ntensors; ++t) fn(t, c.start_host[t], c.len_host[t]);
}

AdamwLayout adamw_layout(const choco_adamw_config& c) {
  AdamwLayout L{};
  int64_t end = 0;
  for_tensors(c, [&](int32_t, int64_t start, int64_t len) {
    L.ntiles += (len + kTile - 1) / kTile;
    L.nblocks += (len + kMomentBlock - 1) / kMomentBlock;
    L.ngaps += (start - end + kTile - 1) / kTile;
    end = start + len;
  });
  L.ngaps += (resolve_adamw_ld(c) - end + kTile - 1) / kTile;
  const size_t entries = (size_t)c.n * (size_t)resolve_adamw_ld(c);
  size_t at = 0;
  const auto take = [&](size_t bytes) {
    const size_t here = at;
    at = (at + bytes + 255) / 256 * 256;
    return here;
  };
  L.m = take(entries * (c.state_bits / 8));
  L.v = take(entries * (c.state_bits / 8));
  if (c.state_bits == 8) {
    L.m_scale = take((size_t)c.n * L.nblocks * sizeof(float));
    L.v_scale = take((size_t)c.n * L.nblocks * sizeof(float));
  }
  L.state_end = at;
  L.tiles = take((size_t)(L.ntiles + L.ngaps) * sizeof(AdamwTile));
  L.total = at;
  return L;
}

// A launch holds a step, and a read-back with its tiles of no tensor.
bool adamw_fits(const AdamwLayout& L) { return launch_fits((double)((L.ntiles + L.ngaps + 3) / 4), 256); }

}  // namespace

struct choco_adamw {
  AdamwArgs args;
  AdamwLayout layout;
  char* workspace;
  hipStream_t stream;
  double beta1, beta2;
  int32_t n, state_bits;
  bool streamed;
  uint64_t t;
};

extern "C" {

int choco_train_last_hip_error(void) { return g_last_hip_error; }

int choco_embed_workspace_bytes(const choco_embed_config* cfg, size_t* bytes_host) {
  if (!bytes_host) return CHOCO_E_INVAL;
  if (const int rc = check_embed(cfg)) return rc;
  if (!embed_fits(*cfg)) return CHOCO_E_UNSUPPORTED;
  *bytes_host = embed_layout(*cfg).total;
  return CHOCO_OK;
}

int choco_embed_forward(const choco_embed_config* cfg, const void* tokens_dev, const void* table_dev, void* y_dev) {
  if (const int rc = check_embed(cfg)) return rc;
  const choco_embed_config& c = *cfg;
  if (c.n == 0 || c.tokens == 0 || c.dim == 0) return CHOCO_OK;
  if (!tokens_dev || !table_dev || !y_dev) return CHOCO_E_INVAL;
  if (!aligned_to(tokens_dev, c.token_type == CHOCO_I32 ? 4 : 8) || !aligned_to(table_dev, type_bytes(c.table_type)) ||
      !aligned_to(y_dev, type_bytes(c.row_type)))
    return CHOCO_E_INVAL;
  EmbedArgs A = embed_args(c, tokens_dev);
  A.table = table_dev;
  A.rows = y_dev;
  const size_t tab_size = type_bytes(c.table_type), row_size = type_bytes(c.row_type);
  const int v = embed_width((int)(16 / std::max(tab_size, row_size)), c.dim, {{table_dev, tab_size}, {y_dev, row_size}},
                            {{c.table_stride, tab_size}, {c.row_ld, row_size}, {c.row_stride, row_size}});
  int lanes_log2 = 2;
  while (lanes_log2 < 6 && ((int64_t)v << lanes_log2) < c.dim) ++lanes_log2;
  const int64_t blocks = (c.tokens + (256 >> lanes_log2) - 1) / (256 >> lanes_log2);
  if (!launch_fits(blocks, 256)) return CHOCO_E_UNSUPPORTED;
  const dim3 grid((uint32_t)blocks, (uint32_t)c.n);
  // Rows past the caches where they do not stay there until they are read.  us, through | past: 16 MB written 7.7 | 7.8, 64 MB
  // 18.0 | 17.0, 134 MB 36.6 | 31.4, 201 MB 57.0 | 44.6, 268 MB 86 | 60.
  const bool past = (double)c.n * (double)c.tokens * (double)c.dim * row_size > 96.0 * 1048576.0;
  with_type(c.table_type, [&](auto tab) {
    with_type(c.row_type, [&](auto row) {
      with_vector(v, [&](auto width) {
        using Tab = decltype(tab);
        using Row = decltype(row);
        constexpr int V = decltype(width)::value;
        if constexpr (V * std::max(sizeof(Tab), sizeof(Row)) <= 16) {
          const auto launch = [&](auto token) {
            if (past) k_embed<decltype(token), Tab, Row, V, true><<<grid, 256, 0, (hipStream_t)c.stream>>>(A, lanes_log2);
            else k_embed<decltype(token), Tab, Row, V, false><<<grid, 256, 0, (hipStream_t)c.stream>>>(A, lanes_log2);
          };
          if (c.token_type == CHOCO_I32) launch(int32_t{});
          else launch(int64_t{});
        }
      });
    });
  });
  TRY_HIP(hipGetLastError());
  return CHOCO_OK;
}

int choco_embed_backward(const choco_embed_config* cfg, const void* tokens_dev, const void* dy_dev, float* dtable_dev,
                         int accumulate, void* workspace_dev, size_t workspace_bytes) {
  if (const int rc = check_embed(cfg)) return rc;
  const choco_embed_config& c = *cfg;
  if (c.n == 0 || c.dim == 0 || (c.tokens == 0 && accumulate)) return CHOCO_OK;
  if (!dtable_dev || (c.tokens > 0 && (!tokens_dev || !dy_dev))) return CHOCO_E_INVAL;
  if (!aligned_to(tokens_dev, c.token_type == CHOCO_I32 ? 4 : 8) || !aligned_to(dtable_dev, 4) || !aligned_to(dy_dev, type_bytes(c.row_type)))
    return CHOCO_E_INVAL;
  if (!embed_fits(c)) return CHOCO_E_UNSUPPORTED;
  const EmbedLayout L = embed_layout(c);
  if (L.total > 0 && (!workspace_dev || !aligned_to(workspace_dev, 16))) return CHOCO_E_INVAL;
  if (L.total > workspace_bytes) return CHOCO_E_NOMEM;
  EmbedArgs A = embed_args(c, tokens_dev);
  A.rows = dy_dev;
  A.dtable = dtable_dev;
  const hipStream_t stream = (hipStream_t)c.stream;
  const int64_t zero_blocks = accumulate ? 0 : (c.vocab * c.dim + kZeroFloats - 1) / kZeroFloats;
  if (!launch_fits((double)zero_blocks * c.n + c.n, kSortThreads)) return CHOCO_E_UNSUPPORTED;
  A.zero_blocks = (uint32_t)zero_blocks;
  // Cleared past the caches where what is cleared would push the rows out that are added up afterwards, but up to 64 MB left there for
  // what reads the gradient next.  us, through | past, rows of 640 in fp32, of 1120 tokens cleared 64 MB 23 | 23, 128 MB 36 | 34, 692 MB
  // 134 | 135; 8192 tokens 64 MB 39 | 39, 86 MB 53 | 39, 128 MB 53 | 39, 256 MB 64 | 61; 32,768 tokens 16 MB 51 | 50, 64 MB 67 | 60,
  // 96 MB 74 | 67, 256 MB 108 | 101; but 100 tokens, with a launch that only clears, 128 MB 28 | 27, 256 MB 49 | 51, 692 MB 123 | 132.
  A.zero_past = c.tokens > kFew && (double)c.n * (double)c.vocab * (double)c.dim * 4 > 64.0 * 1048576.0;
  const size_t size = type_bytes(c.row_type);
  // Two columns a lane: with eight (or four) a wave holds so many rows of sums and old values that too few waves fit to keep the
  // memory busy (65,536 rows of 1024 in bf16: eight 111 us, four 101, two 99).
  int v = embed_width(2, c.dim, {{dy_dev, size}, {dtable_dev, 4}}, {{c.row_ld, size}, {c.row_stride, size}, {c.table_stride, 4}});
  if (c.dim <= 64) v = 1;     // (no lane without columns)
  // Rows and sums past the caches where the rows, other ones with every step, would push too much else out of them.  us, through | past,
  // rows of 1024 added: fp32 16 MB 28 | 28, 32 MB 40 | 42, 64 MB 51 | 50, 96 MB 69 | 60, 256 MB 125 | 106, 512 MB 228 | 209; bf16
  // 16 MB 39 | 40, 32 MB 42 | 44, 64 MB 65 | 58, 96 MB 83 | 71, 256 MB 170 | 156, 512 MB 261 | 235.
  const bool past = (double)c.n * (double)c.tokens * (double)c.dim * size > 48.0 * 1048576.0;
  A.column_chunks = (c.dim + 64 * v - 1) / (64 * v);
  if (c.tokens <= kFew) {
    if (!launch_fits((double)c.tokens * (double)A.column_chunks, 64)) return CHOCO_E_UNSUPPORTED;
    if (!accumulate) {   // zeros first
      k_embed_count<int32_t, true, kShortRounds><<<dim3(A.zero_blocks, (uint32_t)c.n), kChunkThreads, 0, stream>>>(A, 0);
      TRY_HIP(hipGetLastError());
    }
    if (c.tokens == 0) return CHOCO_OK;
    with_type(c.row_type, [&](auto row) {
      const auto launch = [&](auto token, auto width, auto add) {
        k_embed_few<decltype(token), decltype(row), decltype(width)::value, decltype(add)::value>
            <<<dim3(blocks_of(c.tokens * A.column_chunks, 4), (uint32_t)c.n), 256, 0, stream>>>(A);
      };
      const auto with_add = [&](auto token, auto width) {
        if (accumulate) launch(token, width, std::true_type{});
        else launch(token, width, std::false_type{});
      };
      const auto with_lanes = [&](auto token) {
        if (v == 2) with_add(token, std::integral_constant<int, 2>{});
        else with_add(token, std::integral_constant<int, 1>{});
      };
      if (c.token_type == CHOCO_I32) with_lanes(int32_t{});
      else with_lanes(int64_t{});
    });
    TRY_HIP(hipGetLastError());
    return CHOCO_OK;
  }
  char* ws = (char*)workspace_dev;
  A.keys = (uint32_t*)(ws + L.keys);
  A.places = (uint32_t*)(ws + L.places);
  A.partial = (float*)(ws + L.partial);
  A.partial_ld = L.partial_ld;
  A.pieces = L.pieces;
  A.digit_bits = L.digit_bits;
  A.passes = L.passes;
  if (!launch_fits((double)A.pieces * (double)A.column_chunks, 64) || !launch_fits((double)L.chunks + zero_blocks, kChunkThreads))
    return CHOCO_E_UNSUPPORTED;
  const auto order = [&](auto token) {
    using Tok = decltype(token);
    if (L.one) {
      k_embed_sort<Tok><<<dim3((uint32_t)(c.n + zero_blocks * c.n)), kSortThreads, sort_lds(c.tokens, L.digit_bits), stream>>>(A, c.n);
      return;
    }
    A.counts = (uint32_t*)(ws + L.counts);
    A.keys_next = (uint32_t*)(ws + L.keys_next);
    A.places_next = (uint32_t*)(ws + L.places_next);
    A.chunks = L.chunks;
    const auto passes = [&](auto length) {
      constexpr int ROUNDS = decltype(length)::value;
      const dim3 grid(L.chunks, (uint32_t)c.n), grid_and_zeros(L.chunks + A.zero_blocks, (uint32_t)c.n);
      for (int pass = 0; pass < L.passes; ++pass) {
        const int shift = pass * L.digit_bits;
        if (pass == 0) {
          k_embed_count<Tok, true, ROUNDS><<<grid_and_zeros, kChunkThreads, 0, stream>>>(A, shift);
          k_embed_scatter<Tok, true, ROUNDS><<<grid, kChunkThreads, 0, stream>>>(A, shift);
        } else {
          k_embed_count<Tok, false, ROUNDS><<<grid, kChunkThreads, 0, stream>>>(A, shift);
          k_embed_scatter<Tok, false, ROUNDS><<<grid, kChunkThreads, 0, stream>>>(A, shift);
        }
        std::swap(A.keys, A.keys_next);
        std::swap(A.places, A.places_next);
      }
    };
    if (L.rounds == kShortRounds) passes(std::integral_constant<int, kShortRounds>{});
    else passes(std::integral_constant<int, kLongRounds>{});
  };
  if (c.token_type == CHOCO_I32) order(int32_t{});
  else order(int64_t{});
  TRY_HIP(hipGetLastError());
  const int64_t units = A.pieces * A.column_chunks;
  with_type(c.row_type, [&](auto row) {
    const auto sums = [&](auto width, auto add) {
      using Row = decltype(row);
      constexpr int V = decltype(width)::value;
      constexpr bool ADD = decltype(add)::value;
      const dim3 grid(blocks_of(units, 4), (uint32_t)c.n);
      if (past) k_embed_sum<Row, V, ADD, true><<<grid, 256, 0, stream>>>(A);
      else k_embed_sum<Row, V, ADD, false><<<grid, 256, 0, stream>>>(A);
      if (A.pieces > 1) k_embed_join<V, ADD><<<dim3(blocks_of(units, kJoinWaves), (uint32_t)c.n), 64 * kJoinWaves, 0, stream>>>(A);
    };
    const auto with_add = [&](auto width) {
      if (accumulate) sums(width, std::true_type{});
      else sums(width, std::false_type{});
    };
    if (v == 2) with_add(std::integral_constant<int, 2>{});
    else with_add(std::integral_constant<int, 1>{});
  });
  TRY_HIP(hipGetLastError());
  return CHOCO_OK;
}

int choco_recur_saved_bytes(const choco_recur_config* cfg, size_t* bytes_host) {
  if (!bytes_host) return CHOCO_E_INVAL;
  if (const int rc = check_recur(cfg)) return rc;
  if (!recur_fits(*cfg)) return CHOCO_E_UNSUPPORTED;
  *bytes_host = (size_t)saved_floats(*cfg) * sizeof(float);
  return CHOCO_OK;
}

int choco_recur_workspace_bytes(const choco_recur_config* cfg, size_t* bytes_host) {
  if (!bytes_host) return CHOCO_E_INVAL;
  if (const int rc = check_recur(cfg)) return rc;
  if (!recur_fits(*cfg)) return CHOCO_E_UNSUPPORTED;
  *bytes_host = recur_workspace(*cfg);
  return CHOCO_OK;
}

int choco_recur_forward(const choco_recur_config* cfg, const void* f_dev, const void* u_dev, const void* o_dev,
                        const float* h0_dev, const int32_t* lengths_dev, void* y_dev, float* h_last_dev, float* saved_dev,
                        void* workspace_dev, size_t workspace_bytes) {
  if (const int rc = check_recur(cfg)) return rc;
  const choco_recur_config& c = *cfg;
  if (c.batch == 0 || c.dim == 0) return CHOCO_OK;
  const size_t size = type_bytes(c.type);
  if (c.steps > 0) {
    if (!f_dev || !u_dev || !y_dev) return CHOCO_E_INVAL;
    if (!strides_ok(c, c.f_stride, false) || !strides_ok(c, c.u_stride, false) || (o_dev && !strides_ok(c, c.o_stride, false)) ||
        !strides_ok(c, c.y_stride, true))
      return CHOCO_E_INVAL;
  }
  if (!aligned_to(f_dev, size) || !aligned_to(u_dev, size) || !aligned_to(o_dev, size) || !aligned_to(y_dev, size) ||
      !aligned_to(h0_dev, 4) || !aligned_to(lengths_dev, 4) || !aligned_to(h_last_dev, 4) || !aligned_to(saved_dev, 4))
    return CHOCO_E_INVAL;
  if (!recur_fits(c)) return CHOCO_E_UNSUPPORTED;
  const size_t need = recur_workspace(c);
  if (need > 0 && (!workspace_dev || !aligned_to(workspace_dev, 16))) return CHOCO_E_INVAL;
  if (need > workspace_bytes) return CHOCO_E_NOMEM;
  RecurArgs A = recur_args(c, f_dev, u_dev, o_dev, lengths_dev);
  A.h0 = h0_dev;
  A.y = y_dev;
  A.h_last = h_last_dev;
  A.saved = saved_dev;
  const bool pairs = recur_pairs(c, o_dev, false, {f_dev, u_dev, o_dev, y_dev});
  const int width = pairs ? 128 : 64;
  dim3 grid;
  int threads;
  place_recur(c, width, kForwardSteps, workspace_dev, A, grid, threads);
  const hipStream_t stream = (hipStream_t)c.stream;
  if (A.tiles > 1) start_chains(A, width, h0_dev, stream);
  with_type(c.type, [&](auto x) {
    using T = decltype(x);
    with_width<T>(pairs, [&](auto each) {
      constexpr int V = decltype(each)::value;
      const auto launch = [&](auto gated) {
        with_mode(recur_mode(c, A, o_dev ? 4 : 3), [&](auto mode) {
          k_recur<T, V, decltype(gated)::value, decltype(mode)::value><<<grid, threads, 0, stream>>>(A);
        });
      };
      if (o_dev) launch(std::true_type{});
      else launch(std::false_type{});
    });
  });
  TRY_HIP(hipGetLastError());
  return CHOCO_OK;
}

int choco_recur_backward(const choco_recur_config* cfg, const void* f_dev, const void* u_dev, const void* o_dev,
                         const int32_t* lengths_dev, const float* saved_dev, const void* dy_dev, const float* dlast_dev,
                         void* df_dev, void* du_dev, void* do_dev, float* dh0_dev, void* workspace_dev, size_t workspace_bytes) {
  if (const int rc = check_recur(cfg)) return rc;
  const choco_recur_config& c = *cfg;
  if (c.batch == 0 || c.dim == 0) return CHOCO_OK;
  const size_t size = type_bytes(c.type);
  if (c.steps > 0) {
    if (!f_dev || !u_dev || !saved_dev || !dy_dev || !df_dev || !du_dev || (o_dev && !do_dev)) return CHOCO_E_INVAL;
    if (!strides_ok(c, c.f_stride, false) || !strides_ok(c, c.u_stride, false) || (o_dev && !strides_ok(c, c.o_stride, false)) ||
        !strides_ok(c, c.y_stride, false) || !strides_ok(c, c.df_stride, true) || !strides_ok(c, c.du_stride, true) ||
        (o_dev && !strides_ok(c, c.do_stride, true)))
      return CHOCO_E_INVAL;
  }
  if (!aligned_to(f_dev, size) || !aligned_to(u_dev, size) || !aligned_to(o_dev, size) || !aligned_to(dy_dev, size) ||
      !aligned_to(df_dev, size) || !aligned_to(du_dev, size) || !aligned_to(do_dev, size) || !aligned_to(lengths_dev, 4) ||
      !aligned_to(saved_dev, 4) || !aligned_to(dlast_dev, 4) || !aligned_to(dh0_dev, 4))
    return CHOCO_E_INVAL;
  if (!recur_fits(c)) return CHOCO_E_UNSUPPORTED;
  const size_t need = recur_workspace(c);
  if (need > 0 && (!workspace_dev || !aligned_to(workspace_dev, 16))) return CHOCO_E_INVAL;
  if (need > workspace_bytes) return CHOCO_E_NOMEM;
  RecurArgs A = recur_args(c, f_dev, u_dev, o_dev, lengths_dev);
  A.saved = const_cast<float*>(saved_dev);
  A.dy = dy_dev;
  A.dlast = dlast_dev;
  A.df = df_dev;
  A.du = du_dev;
  A.dout = do_dev;
  A.dh0 = dh0_dev;
  const bool pairs = recur_pairs(c, o_dev, true, {f_dev, u_dev, o_dev, dy_dev, df_dev, du_dev, do_dev});
  const int width = pairs ? 128 : 64;
  dim3 grid;
  int threads;
  place_recur(c, width, back_steps(width / 64), workspace_dev, A, grid, threads);
  const hipStream_t stream = (hipStream_t)c.stream;
  if (A.tiles > 1) start_chains(A, width, dlast_dev, stream);
  with_type(c.type, [&](auto x) {
    using T = decltype(x);
    with_width<T>(pairs, [&](auto each) {
      constexpr int V = decltype(each)::value;
      const auto launch = [&](auto gated) {
        with_mode(recur_mode(c, A, o_dev ? 7 : 5), [&](auto mode) {
          k_recur_back<T, V, decltype(gated)::value, decltype(mode)::value><<<grid, threads, 0, stream>>>(A);
        });
      };
      if (o_dev) launch(std::true_type{});
      else launch(std::false_type{});
    });
  });
  TRY_HIP(hipGetLastError());
  return CHOCO_OK;
}

int choco_adamw_workspace_bytes(const choco_adamw_config* cfg, size_t* bytes_host) {
  if (!bytes_host) return CHOCO_E_INVAL;
  if (const int rc = check_adamw(cfg)) return rc;
  const AdamwLayout L = adamw_layout(*cfg);
  if (!adamw_fits(L)) return CHOCO_E_UNSUPPORTED;
  *bytes_host = L.total;
  return CHOCO_OK;
}

int choco_adamw_init(const choco_adamw_config* cfg, float* x_dev, void* workspace_dev, size_t workspace_bytes,
                     choco_adamw** out) {
  if (!out) return CHOCO_E_INVAL;
  *out = nullptr;
  if (const int rc = check_adamw(cfg)) return rc;
  if (!x_dev || !workspace_dev || !aligned_to(x_dev, 16) || !aligned_to(workspace_dev, 256)) return CHOCO_E_INVAL;
  const choco_adamw_config& c = *cfg;
  const AdamwLayout L = adamw_layout(c);
  if (!adamw_fits(L)) return CHOCO_E_UNSUPPORTED;
  if (workspace_bytes < L.total) return CHOCO_E_NOMEM;
  try {
    std::vector<AdamwTile> tiles;
    tiles.reserve((size_t)(L.ntiles + L.ngaps));
    const auto gap = [&](int64_t at, int64_t end) {   // entries of no tensor, behind the tensors' tiles
      for (; at < end; at += kTile) {
        AdamwTile tile{};
        tile.start = (int32_t)at;
        tile.len = (int32_t)(end - at < kTile ? end - at : kTile);
        tile.block = -1;
        tiles.push_back(tile);
      }
    };
    int32_t block = 0;
    for_tensors(c, [&](int32_t t, int64_t start, int64_t len) {
      for (int64_t at = 0; at < len; at += kTile) {
        AdamwTile tile{};
        tile.start = (int32_t)(start + at);
        tile.len = (int32_t)(len - at < kTile ? len - at : kTile);
        tile.block = block;
        tile.lr_scale = c.lr_scale_host ? c.lr_scale_host[t] : 1.0f;
        tile.weight_decay = c.weight_decay_host ? c.weight_decay_host[t] : 0.0f;
        block += (tile.len + kMomentBlock - 1) / kMomentBlock;
        tiles.push_back(tile);
      }
    });
    int64_t end = 0;
    for_tensors(c, [&](int32_t, int64_t start, int64_t len) {
      gap(end, start);
      end = start + len;
    });
    gap(end, resolve_adamw_ld(c));
    char* ws = (char*)workspace_dev;
    const hipStream_t stream = (hipStream_t)c.stream;
    TRY_HIP(hipMemsetAsync(ws, 0, L.state_end, stream));
    if (!tiles.empty())
      TRY_HIP(hipMemcpyAsync(ws + L.tiles, tiles.data(), tiles.size() * sizeof(AdamwTile), hipMemcpyHostToDevice, stream));
    TRY_HIP(hipStreamSynchronize(stream));   // `tiles` goes
    choco_adamw* a = new choco_adamw{};
    a->layout = L;
    a->workspace = ws;
    a->stream = stream;
    a->beta1 = c.beta1;
    a->beta2 = c.beta2;
    a->n = c.n;
    a->state_bits = c.state_bits;
    a->streamed = adamw_streams(c);
    AdamwArgs& A = a->args;
    A.x = x_dev;
    A.m = ws + L.m;
    A.v = ws + L.v;
    A.m_scale = (float*)(ws + L.m_scale);
    A.v_scale = (float*)(ws + L.v_scale);
    A.tiles = (const AdamwTile*)(ws + L.tiles);
    A.ntiles = (int32_t)L.ntiles;      // (a launch holds them)
    A.nblocks = (int32_t)L.nblocks;
    A.ld = resolve_adamw_ld(c);
    A.beta1 = (float)c.beta1;
    A.one_minus_beta1 = (float)(1.0 - c.beta1);
    A.beta2 = (float)c.beta2;
    A.one_minus_beta2 = (float)(1.0 - c.beta2);
    A.eps = (float)c.eps;
    A.seed_lo = (uint32_t)c.seed;
    A.seed_hi = (uint32_t)(c.seed >> 32);
    *out = a;
  } catch (const std::bad_alloc&) {
    return CHOCO_E_NOMEM;
  }
  return CHOCO_OK;
}

int choco_adamw_step(choco_adamw* a, const void* g_dev, int32_t grad_type, float lr, const float* grad_scale_dev) {
  if (!a || !g_dev || !aligned_to(g_dev, 16) || !aligned_to(grad_scale_dev, 4)) return CHOCO_E_INVAL;
  if ((grad_type != CHOCO_F32 && grad_type != CHOCO_BF16) || !std::isfinite(lr)) return CHOCO_E_INVAL;
  AdamwArgs A = a->args;
  A.g = g_dev;
  A.grad_scale = grad_scale_dev;
  // the words of step t are keyed by the steps before it; its corrections are those of the (t + 1)-th
  A.t_lo = (uint32_t)a->t;
  A.t_hi = (uint32_t)(a->t >> 32);
  const double t = (double)a->t + 1.0;
  A.lr = lr;
  A.rate = (float)((double)lr / (1.0 - std::pow(a->beta1, t)));
  A.root_scale = (float)(1.0 / std::sqrt(1.0 - std::pow(a->beta2, t)));
  if (A.ntiles > 0) {
    const dim3 grid(blocks_of(A.ntiles, 4), (uint32_t)a->n);
    const auto launch = [&](auto g, auto bits, auto stream) {
      k_adamw<decltype(g), decltype(bits)::value, decltype(stream)::value><<<grid, 256, 0, a->stream>>>(A);
    };
    const auto with_stream = [&](auto g, auto bits) {
      if (a->streamed) launch(g, bits, std::true_type{});
      else launch(g, bits, std::false_type{});
    };
    const auto with_bits = [&](auto g) {
      if (a->state_bits == 32) with_stream(g, std::integral_constant<int, 32>{});
      else with_stream(g, std::integral_constant<int, 8>{});
    };
    if (grad_type == CHOCO_F32) with_bits(float{});
    else with_bits(bf16_t{});
    TRY_HIP(hipGetLastError());
  }
  ++a->t;
  return CHOCO_OK;
}

int choco_adamw_moments(choco_adamw* a, float* m_dev, float* v_dev) {
  if (!a || !m_dev || !v_dev || !aligned_to(m_dev, 16) || !aligned_to(v_dev, 16)) return CHOCO_E_INVAL;
  AdamwArgs A = a->args;
  A.m_out = m_dev;
  A.v_out = v_dev;
  A.ntiles += (int32_t)a->layout.ngaps;
  const dim3 grid(blocks_of(A.ntiles, 4), (uint32_t)a->n);
  if (a->state_bits == 32) k_adamw_moments<32><<<grid, 256, 0, a->stream>>>(A);
  else k_adamw_moments<8><<<grid, 256, 0, a->stream>>>(A);
  TRY_HIP(hipGetLastError());
  return CHOCO_OK;
}

int choco_adamw_state(choco_adamw* a, void** state_dev, size_t* bytes_host) {
  if (!a || !state_dev || !bytes_host) return CHOCO_E_INVAL;
  *state_dev = a->workspace;
  *bytes_host = a->layout.state_end;
  return CHOCO_OK;
}

int choco_adamw_set_stream(choco_adamw* a, void* stream) {
  if (!a) return CHOCO_E_INVAL;
  a->stream = (hipStream_t)stream;
  return CHOCO_OK;
}

int choco_adamw_get_step(choco_adamw* a, uint64_t* t_host) {
  if (!a || !t_host) return CHOCO_E_INVAL;
  *t_host = a->t;
  return CHOCO_OK;
}

int choco_adamw_set_step(choco_adamw* a, uint64_t t) {
  if (!a) return CHOCO_E_INVAL;
  a->t = t;
  return CHOCO_OK;
}

int choco_adamw_destroy(choco_adamw* a) {
  delete a;
  return CHOCO_OK;
}

}  // extern "C"
