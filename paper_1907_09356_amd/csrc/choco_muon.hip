// Host side of choco_train.h's orthogonalised matrices and of the optimiser that steps along them: argument checks, workspace
// layout, kernel launches.  No device memory is allocated here; only choco_muon_init waits for the device.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <new>
#include <type_traits>
#include <vector>

#include "choco_host.h"
#include "choco_muon.h"

using namespace choco;

namespace {

constexpr int kMostIterations = 32;
// Tiles of 128 x 128 entries where there are at least so many to fill the card with, of X' or of the lower triangles of P and Q, else of
// 64 x 64.  us, all products in tiles of 64 | of 128 (so many of X', of a triangle): 333 x 1000 194 | 383 (24, 6); four of 650 x 650 373 | 490 (144,
// 84), eight 518 | 478 (288, 168); two of 650 x 2600 462 | 768 (252, 42), four 753 | 816 (504, 84); 2048 x 2048 1198 | 1084 (256, 136); 64 of 256 x 256
// 424 | 332 (256, 192); eight of 1024 x 1024 1201 | 798 (512, 288).
constexpr double kFewTiles = 200, kFewOfTriangle = 128;
struct Tiles {
  int apply = 128, gram = 128;      // sides
  double applies = 0.0, grams = 0.0;
  void add(int64_t rows, int64_t cols, double count);
  void choose() {
    if (applies < kFewTiles) apply = 64;
    if (grams < kFewOfTriangle) gram = 64;
  }
};
// Matrices that a step takes at once: operands of at most so many bytes, or one matrix.  (48 of 2600 x 650, whose operands are 1.2 GB: at once
// 4.97 ms; in rounds of 1 GB 5.61, of 512 MB 5.69, of 256 MB, which stay in the last-level cache, 6.19.)
constexpr int64_t kRoundBytes = (int64_t)1 << 31;

int64_t padded(int64_t n) { return (n + kMuonPad - 1) / kMuonPad * kMuonPad; }
int64_t tiles_of(int64_t n, int tile) { return (n + tile - 1) / tile; }

// A matrix that a workgroup takes whole: what it holds fits LDS, and a wave's part of X its registers.
bool whole(int64_t rows, int64_t cols) {
  const int64_t a = std::min(rows, cols), b = std::max(rows, cols), ra = (a + 31) / 32 * 32, rb = (b + 31) / 32 * 32;
  return whole_bytes(a, b) <= kWholeBytes && ra * rb <= 256 * kWholeTiles * kWholeWaves;
}

// Threads of a workgroup, of matrices taken whole and of the others.
constexpr int kTileThreads = 256;
int threads_of(bool whole) { return whole ? 64 * kWholeWaves : kTileThreads; }

// A shape's sides, operands and tiles (null: taken whole); where it lies and what is behind the begins are the caller's.
MuonShape shape_from(int64_t rows, int64_t cols, const Tiles* tiles) {
  MuonShape S{};
  S.rows = (int32_t)rows;
  S.cols = (int32_t)cols;
  S.a = std::min(S.rows, S.cols);
  S.b = std::max(S.rows, S.cols);
  S.a_ld = (int32_t)padded(S.a);
  S.b_ld = (int32_t)padded(S.b);
  S.scratch_of = (muon_scratch(S.a, S.b, S.a_ld, S.b_ld) + 255) / 256 * 256;
  S.start_tiles = (uint32_t)(((rows + 63) / 64) * ((cols + 63) / 64));
  if (!tiles) {      // a workgroup takes all of it
    S.start_tiles = 1;
    S.scratch_of = 0;
    return S;
  }
  const int64_t high = tiles_of(S.a, tiles->gram);
  S.gram_tiles = (uint32_t)(high * (high + 1) / 2);
  S.apply_tiles = (uint32_t)(tiles_of(S.a, tiles->apply) * tiles_of(S.b, tiles->apply));
  return S;
}
void Tiles::add(int64_t rows, int64_t cols, double count) {
  const Tiles large;
  const MuonShape S = shape_from(rows, cols, &large);
  applies += S.apply_tiles * count;
  grams += S.gram_tiles * count;
}

// Matrices that one set of launches takes.
struct Round {
  int32_t first, count;     // entries of the table
  uint32_t start_tiles, gram_tiles, apply_tiles;
  int64_t lds;              // of matrices taken whole: the most that one needs
};

template <int KIND>
void launch_product(const MuonArgs& A, uint32_t tiles, int side, hipStream_t stream) {
  if (side == 128) k_muon_product<KIND, 128><<<dim3(tiles), kTileThreads, 0, stream>>>(A);
  else k_muon_product<KIND, 64><<<dim3(tiles), kTileThreads, 0, stream>>>(A);
}

template <class T, bool STEP>
int run_tiles(MuonArgs A, const Round& R, int iterations, const Tiles& tiles, hipStream_t stream) {
  k_muon_squares<T, STEP><<<dim3(R.start_tiles), kTileThreads, 0, stream>>>(A);
  TRY_HIP(hipGetLastError());
  k_muon_start<T, STEP><<<dim3(R.start_tiles), kTileThreads, 0, stream>>>(A);
  TRY_HIP(hipGetLastError());
  for (int i = 0; i < iterations; ++i) {
    A.now = i & 1;
    A.last = i + 1 == iterations;
    launch_product<kGram>(A, R.gram_tiles, tiles.gram, stream);
    TRY_HIP(hipGetLastError());
    launch_product<kSquare>(A, R.gram_tiles, tiles.gram, stream);
    TRY_HIP(hipGetLastError());
    launch_product<kApply>(A, R.apply_tiles, tiles.apply, stream);
    TRY_HIP(hipGetLastError());
  }
  return CHOCO_OK;
}
template <class T, bool STEP>
int run_round(const MuonArgs& A, const Round& R, int iterations, const Tiles& tiles, hipStream_t stream) {
  if (R.lds > 0) {
    static std::atomic<uint64_t> done{0};
    TRY_HIP(allow_lds((const void*)k_muon_whole<T, STEP>, kWholeBytes, done));
    k_muon_whole<T, STEP><<<dim3(R.start_tiles), 64 * kWholeWaves, (size_t)R.lds, stream>>>(A, iterations);
    TRY_HIP(hipGetLastError());
    return CHOCO_OK;
  }
  return run_tiles<T, STEP>(A, R, iterations, tiles, stream);
}

// ---- a stack of matrices ----

int check_orthogonalize(const choco_orthogonalize_config* c) {
  if (!c) return CHOCO_E_INVAL;
  if (c->batch < 0 || c->batch >= kMaxIndex || c->rows < 0 || c->rows > kMuonMost || c->cols < 0 || c->cols > kMuonMost) return CHOCO_E_INVAL;
  if (!type_bytes(c->type) || c->iterations < 1 || c->iterations > kMostIterations) return CHOCO_E_INVAL;
  if (c->batch == 0 || c->rows == 0 || c->cols == 0) return CHOCO_OK;
  for (const int64_t* s : {c->x_stride, c->y_stride}) {
    if (s[0] < 0 || s[1] < 0 || s[0] > kMaxExtent || s[1] > kMaxExtent) return CHOCO_E_INVAL;
    if ((double)s[0] * (double)(c->batch - 1) + (double)s[1] * (double)(c->rows - 1) + (double)c->cols > (double)kMaxExtent) return CHOCO_E_INVAL;
  }
  const int64_t* s = c->y_stride;    // entries apart: matrix after matrix, or row after row
  const bool one = c->batch <= 1, one_row = c->rows <= 1;
  const bool by_matrix = (one_row || s[1] >= c->cols) && (one || (double)s[0] >= (double)s[1] * (double)(c->rows - 1) + (double)c->cols);
  const bool by_row = (one || s[0] >= c->cols) && (one_row || (double)s[1] >= (double)s[0] * (double)(c->batch - 1) + (double)c->cols);
  return by_matrix || by_row ? CHOCO_OK : CHOCO_E_INVAL;
}

struct StackLayout {
  MuonShape shape;
  Tiles tiles;
  bool whole;
  int64_t each;       // matrices taken at once
  size_t partials, scratch, total;
};
int stack_layout(const choco_orthogonalize_config& c, StackLayout& L) {
  L = {};
  if (c.batch == 0 || c.rows == 0 || c.cols == 0) return CHOCO_OK;
  L.whole = whole(c.rows, c.cols);
  L.tiles.add(c.rows, c.cols, (double)c.batch);
  L.tiles.choose();
  L.shape = shape_from(c.rows, c.cols, L.whole ? nullptr : &L.tiles);
  const double most = std::max<double>(L.shape.start_tiles, std::max(L.shape.gram_tiles, L.shape.apply_tiles));
  const int threads = threads_of(L.whole);
  if (!launch_fits(most, threads)) return CHOCO_E_UNSUPPORTED;
  L.each = L.whole ? c.batch : std::min<int64_t>(c.batch, std::max<int64_t>(1, kRoundBytes / L.shape.scratch_of));
  while (L.each > 1 && !launch_fits(most * (double)L.each, threads)) L.each /= 2;
  const int64_t times = (c.batch + L.each - 1) / L.each;      // of like sizes
  L.each = (c.batch + times - 1) / times;
  Parts parts;
  if (!L.whole) L.partials = parts.take((size_t)L.each * L.shape.start_tiles * sizeof(double));
  L.scratch = parts.take((size_t)L.each * (size_t)L.shape.scratch_of);
  L.total = parts.at;
  return CHOCO_OK;
}

// ---- the optimiser ----

int64_t resolve_ld(const choco_muon_config& c) { return c.ld == 0 ? (c.d + 3) / 4 * 4 : c.ld; }

int check_muon(const choco_muon_config* c) {
  if (!c) return CHOCO_E_INVAL;
  if (c->n < 1 || c->n > 65535 || c->d < 1 || c->d > CHOCO_MAX_D) return CHOCO_E_INVAL;
  const int64_t ld = resolve_ld(*c);
  if (ld < c->d || (ld & 3) != 0 || ld > kMaxIndex) return CHOCO_E_INVAL;
  if (c->ntensors < 1 || !c->start_host || !c->rows_host || !c->cols_host) return CHOCO_E_INVAL;
  if (!(c->momentum >= 0.0 && c->momentum < 1.0) || (float)c->momentum >= 1.0f) return CHOCO_E_INVAL;
  if ((c->nesterov != 0 && c->nesterov != 1) || c->iterations < 1 || c->iterations > kMostIterations) return CHOCO_E_INVAL;
  int64_t end = 0;
  for (int32_t t = 0; t < c->ntensors; ++t) {
    const int64_t start = c->start_host[t], rows = c->rows_host[t], cols = c->cols_host[t];
    if (rows < 0 || rows > kMuonMost || cols < 0 || cols > kMuonMost) return CHOCO_E_INVAL;
    if (start < end || start > c->d || rows * cols > c->d - start) return CHOCO_E_INVAL;
    end = start + rows * cols;
    if (c->weight_decay_host && !(c->weight_decay_host[t] >= 0.0f && std::isfinite(c->weight_decay_host[t]))) return CHOCO_E_INVAL;
    if (c->lr_scale_host && !std::isfinite(c->lr_scale_host[t])) return CHOCO_E_INVAL;
  }
  return CHOCO_OK;
}

struct MuonLayout {
  Tiles tiles;
  size_t state_end, table, partials, scratch, total;
};
// The matrices in rounds, and the workspace.  CHOCO_E_UNSUPPORTED: one that no launch holds.
int muon_layout(const choco_muon_config& c, std::vector<MuonShape>& table, std::vector<Round>& rounds, MuonLayout& L) {
  const int64_t ld = resolve_ld(c);
  int64_t moment = 0, most_scratch = 0, most_partials = 0, scratch = 0, partials = 0;
  Round now{};
  for (int32_t t = 0; t < c.ntensors; ++t)
    if (c.rows_host[t] > 0 && c.cols_host[t] > 0 && !whole(c.rows_host[t], c.cols_host[t])) L.tiles.add(c.rows_host[t], c.cols_host[t], (double)c.n);
  L.tiles.choose();
  // rounds of like sizes, as many as it takes (a little more than their share each, as matrices are not divided)
  double all = 0.0;
  for (int32_t t = 0; t < c.ntensors; ++t)
    if (c.rows_host[t] > 0 && c.cols_host[t] > 0 && !whole(c.rows_host[t], c.cols_host[t]))
      all += (double)c.n * (double)shape_from(c.rows_host[t], c.cols_host[t], &L.tiles).scratch_of;
  const int64_t most = (int64_t)std::min<double>(kRoundBytes, 1.02 * all / std::max(1.0, std::ceil(all / (double)kRoundBytes)));
  const auto close = [&] {
    if (now.count > 0) rounds.push_back(now);
    now = {};
    now.first = (int32_t)table.size();
    scratch = partials = 0;
  };
  std::vector<int64_t> moments((size_t)c.ntensors);
  for (int32_t t = 0; t < c.ntensors; ++t) {
    moments[t] = moment;
    moment += c.n * c.rows_host[t] * c.cols_host[t];
  }
  for (int32_t i = 0; i < 2 * c.ntensors; ++i) {      // those taken whole, then the others
    const int32_t t = i % c.ntensors;
    const int64_t rows = c.rows_host[t], cols = c.cols_host[t], start = c.start_host[t];
    if (rows == 0 || cols == 0 || whole(rows, cols) != (i < c.ntensors)) continue;
    const bool alone = i < c.ntensors;
    if (!alone && now.lds > 0) close();
    MuonShape S = shape_from(rows, cols, alone ? nullptr : &L.tiles);
    S.source = S.target = start;
    S.source_of = S.target_of = ld;
    S.source_ld = S.target_ld = cols;
    S.moment = moments[t];
    S.decay = c.weight_decay_host ? c.weight_decay_host[t] : 0.0f;
    S.rate = c.lr_scale_host ? c.lr_scale_host[t] : std::sqrt(std::max(1.0f, (float)rows / (float)cols));
    const double tiles = std::max<double>(S.start_tiles, std::max(S.gram_tiles, S.apply_tiles));
    if (!launch_fits(tiles, threads_of(alone))) return CHOCO_E_UNSUPPORTED;
    if (alone) now.lds = std::max(now.lds, whole_bytes(S.a, S.b));
    for (int32_t w = 0; w < c.n;) {
      const double taken = std::max<double>(now.start_tiles, std::max(now.gram_tiles, now.apply_tiles));
      int64_t count = alone ? c.n - w : std::min<int64_t>(c.n - w, (most - scratch) / S.scratch_of);
      while (count > 0 && !launch_fits(taken + tiles * (double)count, threads_of(alone))) count /= 2;
      if (count < 1) {
        if (now.count > 0) {
          close();
          if (alone) now.lds = whole_bytes(S.a, S.b);
          continue;
        }
        count = 1;
      }
      S.first = w;
      S.source = start + w * ld;
      S.target = S.source;
      S.scratch = scratch;
      S.partials = partials;
      S.start_begin = now.start_tiles;
      S.gram_begin = now.gram_tiles;
      S.apply_begin = now.apply_tiles;
      scratch += count * S.scratch_of;
      partials += alone ? 0 : count * S.start_tiles;
      now.start_tiles += (uint32_t)count * S.start_tiles;
      now.gram_tiles += (uint32_t)count * S.gram_tiles;
      now.apply_tiles += (uint32_t)count * S.apply_tiles;
      ++now.count;
      table.push_back(S);
      most_scratch = std::max(most_scratch, scratch);
      most_partials = std::max(most_partials, partials);
      w += (int32_t)count;
    }
  }
  close();
  Parts parts;
  parts.take((size_t)moment * sizeof(float));
  L.state_end = (size_t)moment * sizeof(float);
  L.table = parts.take(table.size() * sizeof(MuonShape));
  L.partials = parts.take((size_t)most_partials * sizeof(double));
  L.scratch = parts.take((size_t)most_scratch);
  L.total = parts.at;
  return CHOCO_OK;
}

}  // namespace

struct choco_muon {
  MuonArgs args;
  MuonLayout layout;
  std::vector<Round> rounds;
  char* workspace;
  hipStream_t stream;
  int32_t iterations;
};

extern "C" {

int choco_orthogonalize_workspace_bytes(const choco_orthogonalize_config* cfg, size_t* bytes_host) {
  if (!bytes_host) return CHOCO_E_INVAL;
  if (const int rc = check_orthogonalize(cfg)) return rc;
  StackLayout L;
  if (const int rc = stack_layout(*cfg, L)) return rc;
  *bytes_host = L.total;
  return CHOCO_OK;
}

int choco_orthogonalize(const choco_orthogonalize_config* cfg, const void* x_dev, float* y_dev, void* workspace_dev,
                        size_t workspace_bytes) {
  if (const int rc = check_orthogonalize(cfg)) return rc;
  const choco_orthogonalize_config& c = *cfg;
  if (c.batch == 0 || c.rows == 0 || c.cols == 0) return CHOCO_OK;
  if (!x_dev || !y_dev || !aligned_to(x_dev, type_bytes(c.type)) || !aligned_to(y_dev, 4)) return CHOCO_E_INVAL;
  StackLayout L;
  if (const int rc = stack_layout(c, L)) return rc;
  if (L.total > 0 && (!workspace_dev || !aligned_to(workspace_dev, 256))) return CHOCO_E_INVAL;
  if (L.total > workspace_bytes) return CHOCO_E_NOMEM;
  for (int64_t first = 0; first < c.batch; first += L.each) {
    MuonArgs A{};
    A.one = L.shape;
    A.one.source = first * c.x_stride[0];
    A.one.source_of = c.x_stride[0];
    A.one.source_ld = c.x_stride[1];
    A.one.target = first * c.y_stride[0];
    A.one.target_of = c.y_stride[0];
    A.one.target_ld = c.y_stride[1];
    A.source = x_dev;
    A.target = y_dev;
    A.partials = (double*)((char*)workspace_dev + L.partials);
    A.scratch = (char*)workspace_dev + L.scratch;
    const uint32_t count = (uint32_t)std::min(L.each, c.batch - first);
    const Round R{0, 1, count * L.shape.start_tiles, count * L.shape.gram_tiles, count * L.shape.apply_tiles, L.whole ? whole_bytes(L.shape.a, L.shape.b) : 0};
    int rc = CHOCO_OK;
    with_type(c.type, [&](auto x) { rc = run_round<decltype(x), false>(A, R, c.iterations, L.tiles, (hipStream_t)c.stream); });
    if (rc) return rc;
  }
  return CHOCO_OK;
}

int choco_muon_workspace_bytes(const choco_muon_config* cfg, size_t* bytes_host) {
  if (!bytes_host) return CHOCO_E_INVAL;
  if (const int rc = check_muon(cfg)) return rc;
  try {
    std::vector<MuonShape> table;
    std::vector<Round> rounds;
    MuonLayout L{};
    if (const int rc = muon_layout(*cfg, table, rounds, L)) return rc;
    *bytes_host = L.total;
  } catch (const std::bad_alloc&) {
    return CHOCO_E_NOMEM;
  }
  return CHOCO_OK;
}

int choco_muon_init(const choco_muon_config* cfg, float* x_dev, void* workspace_dev, size_t workspace_bytes, choco_muon** out) {
  if (!out) return CHOCO_E_INVAL;
  *out = nullptr;
  if (const int rc = check_muon(cfg)) return rc;
  if (!x_dev || !workspace_dev || !aligned_to(x_dev, 4) || !aligned_to(workspace_dev, 256)) return CHOCO_E_INVAL;
  const choco_muon_config& c = *cfg;
  choco_muon* a = nullptr;
  try {
    std::vector<MuonShape> table;
    std::vector<Round> rounds;
    MuonLayout L{};
    if (const int rc = muon_layout(c, table, rounds, L)) return rc;
    if (workspace_bytes < L.total) return CHOCO_E_NOMEM;
    char* ws = (char*)workspace_dev;
    const hipStream_t stream = (hipStream_t)c.stream;
    if (L.state_end > 0) TRY_HIP(hipMemsetAsync(ws, 0, L.state_end, stream));
    if (!table.empty()) TRY_HIP(hipMemcpyAsync(ws + L.table, table.data(), table.size() * sizeof(MuonShape), hipMemcpyHostToDevice, stream));
    TRY_HIP(hipStreamSynchronize(stream));   // `table` goes
    a = new choco_muon{};
    a->layout = L;
    a->rounds = std::move(rounds);
    a->workspace = ws;
    a->stream = stream;
    a->iterations = c.iterations;
    MuonArgs& A = a->args;
    A.table = (const MuonShape*)(ws + L.table);
    A.target = x_dev;
    A.moments = (float*)ws;
    A.partials = (double*)(ws + L.partials);
    A.scratch = ws + L.scratch;
    A.momentum = (float)c.momentum;
    A.nesterov = c.nesterov;
    *out = a;
  } catch (const std::bad_alloc&) {
    return CHOCO_E_NOMEM;
  }
  return CHOCO_OK;
}

int choco_muon_step(choco_muon* a, const void* g_dev, int32_t grad_type, float lr, const float* grad_scale_dev) {
  if (!a || !g_dev || !aligned_to(grad_scale_dev, 4)) return CHOCO_E_INVAL;
  if ((grad_type != CHOCO_F32 && grad_type != CHOCO_BF16) || !std::isfinite(lr) || !aligned_to(g_dev, type_bytes(grad_type))) return CHOCO_E_INVAL;
  for (const Round& R : a->rounds) {
    MuonArgs A = a->args;
    A.table += R.first;
    A.count = R.count;
    A.source = g_dev;
    A.grad_scale = grad_scale_dev;
    A.lr = lr;
    const int rc = grad_type == CHOCO_F32 ? run_round<float, true>(A, R, a->iterations, a->layout.tiles, a->stream)
                                          : run_round<bf16_t, true>(A, R, a->iterations, a->layout.tiles, a->stream);
    if (rc) return rc;
  }
  return CHOCO_OK;
}

int choco_muon_state(choco_muon* a, void** state_dev, size_t* bytes_host) {
  if (!a || !state_dev || !bytes_host) return CHOCO_E_INVAL;
  *state_dev = a->workspace;
  *bytes_host = a->layout.state_end;
  return CHOCO_OK;
}

int choco_muon_set_stream(choco_muon* a, void* stream) {
  if (!a) return CHOCO_E_INVAL;
  a->stream = (hipStream_t)stream;
  return CHOCO_OK;
}

int choco_muon_destroy(choco_muon* a) {
  delete a;
  return CHOCO_OK;
}

}  // extern "C"
