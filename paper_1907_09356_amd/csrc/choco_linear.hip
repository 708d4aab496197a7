// Host side of choco_train.h's linear attention: argument checks, workspace layout, kernel launches.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <initializer_list>
#include <type_traits>
#include <utility>

#include "choco_host.h"
#include "choco_linear.h"
#include "choco_linear_chunks.h"

using namespace choco;

namespace {

static_assert(kLinearSave == CHOCO_LINEAR_SAVE_STEPS, "the header says what is kept");

int check_linear(const choco_linear_config* c) {
  if (!c) return CHOCO_E_INVAL;
  if (c->batch < 0 || c->steps < 0 || c->heads < 0 || c->batch >= kMaxIndex || c->steps >= kMaxIndex) return CHOCO_E_INVAL;
  if (c->heads > 0 && c->batch >= ((int64_t)1 << 24) / c->heads + (((int64_t)1 << 24) % c->heads != 0)) return CHOCO_E_INVAL;
  for (int32_t heads : {c->q_heads, c->k_heads, c->v_heads})
    if (heads < 1 || c->heads % heads != 0) return CHOCO_E_INVAL;
  for (int32_t dim : {c->dim_k, c->dim_v})
    if (dim < 1 || dim > CHOCO_LINEAR_MAX_DIM) return CHOCO_E_INVAL;
  if (!type_bytes(c->type) || (c->gate_steps != 0 && c->gate_steps != 1)) return CHOCO_E_INVAL;
  return CHOCO_OK;
}

// Strides of an array of batch x steps x heads rows of dim entries.
bool strides_ok(const choco_linear_config& c, const int64_t s[3], int64_t heads, int64_t dim, bool output) {
  std::pair<int64_t, int64_t> by[3] = {{s[0], c.batch}, {s[1], c.steps}, {s[2], heads}};
  double extent = (double)dim;
  for (const auto& p : by) {
    if (p.first < 0 || p.first > kMaxExtent) return false;
    extent += (double)p.first * (double)(p.second - 1);
  }
  if (extent > (double)kMaxExtent) return false;
  if (!output) return true;
  // entries of an output apart: from the shortest stride on, each beyond what the ones before it reach
  std::sort(by, by + 3);
  double reach = (double)dim;
  for (const auto& p : by) {
    if (p.second <= 1) continue;
    if ((double)p.first < reach) return false;
    reach += (double)p.first * (double)(p.second - 1);
  }
  return true;
}

int64_t pieces_of(const choco_linear_config& c) { return (c.steps + kLinearSave - 1) / kLinearSave; }

// Every launch of a call fits, and what it keeps stays far from 64 bits.
bool linear_fits(const choco_linear_config& c) {
  const double rows = (double)rows_of(c), pieces = (double)pieces_of(c) + 1.0;
  if (rows * pieces * c.dim_k * c.dim_v > 1125899906842624.0 || rows * (double)c.steps * 512.0 > 1125899906842624.0) return false;
  return launch_fits((rows * pieces + 8.0) * slices_of(CHOCO_LINEAR_MAX_DIM), 512);
}

// Slices of the passes in chunks of dq and dk, and of dv.
int slices_by_k(const choco_linear_config& c) { return slices_of(c.dim_k, slice_of(c, c.dim_v, c.dim_k)); }
int slices_by_v(const choco_linear_config& c) { return slices_of(c.dim_v, slice_of(c, c.dim_k, c.dim_v)); }

struct LinearLayout {
  size_t later, totals, dots, sums, wide, total;
};
void segments_of(const choco_linear_config& c, int32_t& segments, int32_t& chunks);
int64_t step_by_step(const choco_linear_config& c);
LinearLayout linear_layout(const choco_linear_config& c, bool back) {
  LinearLayout L{};
  Parts parts;
  if (c.batch == 0 || c.heads == 0) return L;
  const size_t rows = (size_t)rows_of(c), state = (size_t)c.dim_k * c.dim_v, steps = (size_t)c.steps;
  size_t segments = (size_t)pieces_of(c);
  if (!back) {
    int32_t count, each;
    segments_of(c, count, each);
    segments = (size_t)count;
  }
  if (segments > 1) {
    L.later = parts.take(rows * segments * state * sizeof(float));
    L.totals = parts.take(rows * segments * sizeof(double));
  }
  if (back) {
    if (c.steps > step_by_step(c)) L.dots = parts.take(rows * steps * (2 * slices_by_k(c) + slices_by_v(c)) * sizeof(float));
    L.sums = parts.take(rows * (size_t)pieces_of(c) * sizeof(float));
    size_t most = 0;
    if (c.q_heads != c.heads || c.k_heads != c.heads) most = c.dim_k;
    if (c.v_heads != c.heads) most = std::max(most, (size_t)c.dim_v);
    L.wide = parts.take(rows * steps * most * sizeof(float));
  }
  L.total = parts.at;
  return L;
}

// One of the arrays that a pass reads or writes.
struct Rows {
  const void* p;
  const int64_t* stride;
  int32_t heads, dim;
};
LinearPass pass_of(const choco_linear_config& c, const Rows& a, const Rows& b, const Rows& v, void* out, const int64_t out_stride[3]) {
  LinearPass P{};
  P.a = a.p; P.a_seq = a.stride[0]; P.a_step = a.stride[1]; P.a_head = a.stride[2]; P.a_share = c.heads / a.heads;
  P.b = b.p; P.b_seq = b.stride[0]; P.b_step = b.stride[1]; P.b_head = b.stride[2]; P.b_share = c.heads / b.heads;
  P.c = v.p; P.c_seq = v.stride[0]; P.c_step = v.stride[1]; P.c_head = v.stride[2]; P.c_share = c.heads / v.heads;
  P.out = out; P.out_seq = out_stride[0]; P.out_step = out_stride[1]; P.out_head = out_stride[2];
  P.x_share = 1;
  P.da = a.dim;
  P.dc = v.dim;
  return P;
}
// The state of y's pass and of dv's is one of dim_k x dim_v entries, row after row; the others have it transposed.
void state_of(const choco_linear_config& c, bool transposed, LinearPass& P) {
  P.state_a = transposed ? 1 : c.dim_v;
  P.state_c = transposed ? c.dim_v : 1;
}

LinearArgs linear_args(const choco_linear_config& c, const float* g, const int32_t* lengths) {
  LinearArgs A{};
  A.g = g;
  A.lengths = lengths;
  A.batch = c.batch;
  A.steps = c.steps;
  A.heads = c.heads;
  A.g_seq = c.gate_steps ? c.g_stride[0] : 0;
  A.g_step = c.gate_steps ? c.g_stride[1] : 0;
  A.g_head = c.g_stride[2];
  return A;
}

// Entries of rows that a load or store takes: `most`, a power of two, or fewer, as the rows are aligned.
int width_of(const Rows& r, size_t size, int most, const choco_linear_config& c) {
  for (int v = most; v > 1; v /= 2) {
    const size_t bytes = v * size;
    bool ok = r.dim % v == 0 && aligned_to(r.p, bytes);
    const int64_t count[3] = {c.batch, c.steps, r.heads};
    for (int i = 0; i < 3; ++i) ok = ok && (count[i] <= 1 || (size_t)r.stride[i] * size % bytes == 0);
    if (ok) return v;
  }
  return 1;
}

// Up to so many steps are taken one by one.  us, one by one | in chunks, forward and backward, three sets of inputs in turn: 160 x 10 heads of 64 in fp32, 4
// steps 22 and 81 | 41 and 123, 8 steps 33 and 125 | 40 and 124; 64 x 16 heads of 128 in bf16, 2 steps 31 and 140 | 39 and 114, 3 steps 35 and 150 | 39 and
// 120, 4 steps 38 and 157 | 38 and 115, 8 steps 53 and 223 | 38 and 117.
constexpr int kFewOf32 = 8, kFewOf16 = 3;
int64_t step_by_step(const choco_linear_config& c) { return c.type == CHOCO_F32 ? kFewOf32 : kFewOf16; }

template <class T>
int run_steps(const choco_linear_config& c, const LinearArgs& A, const LinearPass& P) {
  const dim3 grid((uint32_t)(rows_of(c) * slices_of(P.dc)));
  const auto launch = [&](auto v, auto d) {
    k_linear_steps<T, decltype(v)::value, decltype(d)::value><<<grid, 256, 0, (hipStream_t)c.stream>>>(A, P);
  };
  const auto with_dim = [&](auto v) {
    if (P.da <= 64) launch(v, std::integral_constant<int, 64>{});
    else if (P.da <= 128) launch(v, std::integral_constant<int, 128>{});
    else launch(v, std::integral_constant<int, 256>{});
  };
  // columns of a state next to one another: by sizes alone, as it sets the order of sums (the kernel looks at the addresses)
  const auto wide = [&](int v) { return P.state_c == 1 && P.dc % v == 0; };
  if (wide(4)) with_dim(std::integral_constant<int, 4>{});
  else if (wide(2)) with_dim(std::integral_constant<int, 2>{});
  else with_dim(std::integral_constant<int, 1>{});
  TRY_HIP(hipGetLastError());
  return CHOCO_OK;
}

// (x: what the result is multiplied with, or null)
LinearChunks chunks_of(const choco_linear_config& c, const LinearPass& P, const Rows& a, const Rows& b, const Rows& v, const Rows& out, const Rows* x) {
  LinearChunks C{};
  const size_t size = type_bytes(c.type), out_size = P.wide ? 4 : size;
  const auto far = [&](const Rows& r, size_t bytes) {
    return (double)r.stride[1] * bytes * kChunk + 16.0 * CHOCO_LINEAR_MAX_DIM >= (double)kBufferBytes;
  };
  C.segments = 1;
  C.chunks = (int32_t)((c.steps + kChunk - 1) / kChunk);
  C.way = far(out, out_size) ? kEntries : kParts;
  for (const Rows* r : {&a, &b, &v, x}) {
    if (!r) continue;
    const int v16 = (int)(16 / size), v4 = (int)(4 / size);
    if (width_of(*r, size, v16, c) != v16) C.way = std::min(C.way, (int)kWords);
    if (far(*r, size) || (v4 > 1 && width_of(*r, size, v4, c) != v4)) C.way = kEntries;
  }
  C.vec_out = width_of(out, out_size, 4, c);
  C.vec_x = x ? width_of(*x, size, 4, c) : 1;
  return C;
}

// The states before all segments.
template <class T>
int run_states(const choco_linear_config& c, const LinearArgs& A, const LinearPass& P, const LinearChunks& C, const float* first, float* last) {
  if (const int rc = run_chunks<T, kStates>(c, A, P, C)) return rc;
  const int64_t entries = (int64_t)P.da * P.dc;
  const dim3 grid((uint32_t)std::min<int64_t>(65536, rows_of(c) * ((entries + 255) / 256)));
  k_linear_scan<<<grid, 256, 0, (hipStream_t)c.stream>>>(A, C.states, C.totals, C.segments, entries, first, last, P.back);
  TRY_HIP(hipGetLastError());
  return CHOCO_OK;
}

// Segments of a forward pass in chunks: as many as give so many workgroups, none shorter than kLinearSave steps.  (2 x 32,768 x 16 x 128
// in bf16, us, with lengths from a half on: 512 580 | 519, 1024 572 | 519, 2048 594 | 551, 4096 680 | 611.)
constexpr int64_t kWorkgroups = 1024;
void segments_of(const choco_linear_config& c, int32_t& segments, int32_t& chunks) {
  const int64_t all = (c.steps + kChunk - 1) / kChunk, alone = rows_of(c) * slices_of(c.dim_v, 128), least = kLinearSave / kChunk;
  int64_t each = std::max(all, least);
  if (alone < kWorkgroups / 2 && all > least) each = std::max(least, (all * alone + kWorkgroups - 1) / kWorkgroups);
  each = (each + least - 1) / least * least;
  chunks = (int32_t)each;
  segments = (int32_t)std::max<int64_t>(1, (all + each - 1) / each);
}

template <class T>
int run_forward(const choco_linear_config& c, const LinearArgs& A, LinearPass P, const Rows& q, const Rows& k, const Rows& v, const Rows& y, char* ws) {
  if (c.steps <= step_by_step(c)) return run_steps<T>(c, A, P);
  LinearChunks C = chunks_of(c, P, q, k, v, y, nullptr);
  segments_of(c, C.segments, C.chunks);
  if (C.segments > 1) {
    const LinearLayout L = linear_layout(c, false);
    C.states = (float*)(ws + L.later);
    C.totals = (double*)(ws + L.totals);
    C.states_of = C.segments;
    if (const int rc = run_states<T>(c, A, P, C, P.first, P.last)) return rc;
  }
  return run_chunks<T, kResult>(c, A, P, C);
}

template <class T>
int run_backward(const choco_linear_config& c, const LinearArgs& A, const void* q, const void* k, const void* v, const float* saved,
                 const void* dy, const float* dlast, void* dq, void* dk, void* dv, float* dg, float* dh0, char* ws) {
  const hipStream_t stream = (hipStream_t)c.stream;
  const LinearLayout L = linear_layout(c, true);
  const Rows Q{q, c.q_stride, c.q_heads, c.dim_k}, K{k, c.k_stride, c.k_heads, c.dim_k}, V{v, c.v_stride, c.v_heads, c.dim_v},
      Y{dy, c.y_stride, c.heads, c.dim_v};
  const int64_t rows = rows_of(c), pieces = pieces_of(c);
  float* const later = (float*)(ws + L.later);
  float* const q_dots = (float*)(ws + L.dots);
  float* const k_dots = q_dots + rows * c.steps * slices_by_k(c);
  float* const v_dots = k_dots + rows * c.steps * slices_by_k(c);
  const bool stepwise = c.steps <= step_by_step(c), several = pieces > 1;
  // a pass on its own arrays; a gradient of heads that share one: of every head to the workspace, then added up
  const auto through = [&](LinearPass P, const Rows& ra, const Rows& rb, const Rows& rc_, Rows out, const Rows* x, const float* states,
                           int64_t states_of, int mode) -> int {
    const LinearPass given = P;
    const int32_t heads = out.heads, dim = out.dim;
    const int64_t wide_stride[3] = {(int64_t)c.heads * dim * c.steps, (int64_t)c.heads * dim, dim};
    if (heads != c.heads) {
      P.out = ws + L.wide;
      P.wide = true;
      P.out_seq = wide_stride[0];
      P.out_step = wide_stride[1];
      P.out_head = wide_stride[2];
      out = Rows{P.out, wide_stride, c.heads, dim};
    }
    if (stepwise) {
      if (const int rc = run_steps<T>(c, A, P)) return rc;
    } else {
      LinearChunks C = chunks_of(c, P, ra, rb, rc_, out, x);
      C.segments = (int32_t)pieces;
      C.chunks = kLinearSave / kChunk;
      if (several) {
        C.states = const_cast<float*>(states);
        C.states_of = states_of;
      }
      const int rc = mode == kOfStates ? run_chunks<T, kOfStates>(c, A, P, C) : mode == kOfPairs ? run_chunks<T, kOfPairs>(c, A, P, C) : run_chunks<T, kResult>(c, A, P, C);
      if (rc) return rc;
    }
    if (heads == c.heads) return CHOCO_OK;
    const int64_t count = c.batch * c.steps * heads * dim;
    if (count == 0) return CHOCO_OK;
    k_linear_share<T><<<dim3((uint32_t)std::min<int64_t>(4096, (count + 255) / 256)), 256, 0, stream>>>(
        (const float*)P.out, given.out, c.batch * c.steps, c.steps, heads, c.heads / heads, dim, given.out_seq, given.out_step, given.out_head);
    TRY_HIP(hipGetLastError());
    return CHOCO_OK;
  };
  const Rows DQ{dq, c.dq_stride, c.q_heads, c.dim_k}, DK{dk, c.dk_stride, c.k_heads, c.dim_k}, DV{dv, c.dv_stride, c.v_heads, c.dim_v};
  LinearPass last = pass_of(c, K, Q, Y, dv, c.dv_stride);
  state_of(c, false, last);
  last.back = true;
  last.first = dlast;
  last.first_of = 1;
  last.last = dh0;
  if (!stepwise && several) {
    LinearChunks C = chunks_of(c, last, K, Q, Y, DV, nullptr);
    C.segments = (int32_t)pieces;
    C.chunks = kLinearSave / kChunk;
    C.states = later;
    C.states_of = pieces;
    C.totals = (double*)(ws + L.totals);
    if (const int rc = run_states<T>(c, A, last, C, dlast, dh0)) return rc;
  }
  const bool parts = dg && !stepwise;      // of the gates' gradient, by dq's pass and dk's
  LinearPass P = pass_of(c, Y, V, K, dq, c.dq_stride);
  state_of(c, true, P);
  P.first = saved;
  P.first_of = pieces + 1;
  if (parts) {
    P.x = q; P.x_seq = c.q_stride[0]; P.x_step = c.q_stride[1]; P.x_head = c.q_stride[2]; P.x_share = c.heads / c.q_heads;
    P.dots = q_dots;
    P.met = later;
    P.met_of = pieces;
    P.met_last = dlast;
  }
  if (const int rc = through(P, Y, V, K, DQ, parts ? &Q : nullptr, saved, pieces + 1, kOfStates)) return rc;
  P = pass_of(c, V, Y, Q, dk, c.dk_stride);
  state_of(c, true, P);
  P.back = true;
  P.first = dlast;
  P.first_of = 1;
  if (parts) {
    P.x = k; P.x_seq = c.k_stride[0]; P.x_step = c.k_stride[1]; P.x_head = c.k_stride[2]; P.x_share = c.heads / c.k_heads;
    P.dots = k_dots;
    P.met = saved;
    P.met_of = pieces + 1;
  }
  if (const int rc = through(P, V, Y, Q, DK, parts ? &K : nullptr, later, pieces, kOfStates)) return rc;
  if (parts) {
    last.x = v; last.x_seq = c.v_stride[0]; last.x_step = c.v_stride[1]; last.x_head = c.v_stride[2]; last.x_share = c.heads / c.v_heads;
    last.dots = v_dots;
  }
  if (const int rc = through(last, K, Q, Y, DV, parts ? &V : nullptr, later, pieces, parts ? kOfPairs : kResult)) return rc;
  if (!dg) return CHOCO_OK;
  LinearGates G{};
  G.dots = q_dots;
  G.slices = 2 * slices_by_k(c) + slices_by_v(c);
  G.pieces = pieces;
  G.sums = !c.gate_steps;
  G.dg = G.sums ? (float*)(ws + L.sums) : dg;
  if (pieces > 0 && stepwise) {
    LinearPass few = pass_of(c, K, Q, Y, nullptr, c.dv_stride);
    few.x = v; few.x_seq = c.v_stride[0]; few.x_step = c.v_stride[1]; few.x_head = c.v_stride[2]; few.x_share = c.heads / c.v_heads;
    few.first = saved;
    few.first_of = pieces + 1;
    few.met_last = dlast;
    constexpr int kFew = std::is_same_v<T, float> ? kFewOf32 : kFewOf16;
    const auto lds = [&](int n) { return (size_t)(c.dim_k + c.dim_v) * few_row(n) * sizeof(float); };
    if (c.steps <= 4) k_linear_few_gates<T, 4><<<dim3((uint32_t)rows), 256, lds(4), stream>>>(A, few, G);
    else if constexpr (kFew > 4) k_linear_few_gates<T, kFew><<<dim3((uint32_t)rows), 256, lds(kFew), stream>>>(A, few, G);
    TRY_HIP(hipGetLastError());
  } else if (pieces > 0) {
    k_linear_gates<<<dim3((uint32_t)(rows * pieces)), kLinearSave, 0, stream>>>(A, G);
    TRY_HIP(hipGetLastError());
  }
  if (G.sums) {
    k_linear_gate_sums<<<dim3((uint32_t)c.heads), 256, 0, stream>>>(G.dg, c.batch * pieces, dg);
    TRY_HIP(hipGetLastError());
  }
  return CHOCO_OK;
}

}  // namespace

extern "C" {

int choco_linear_saved_bytes(const choco_linear_config* cfg, size_t* bytes_host) {
  if (!bytes_host) return CHOCO_E_INVAL;
  if (const int rc = check_linear(cfg)) return rc;
  if (!linear_fits(*cfg)) return CHOCO_E_UNSUPPORTED;
  *bytes_host = (size_t)rows_of(*cfg) * (size_t)(pieces_of(*cfg) + 1) * cfg->dim_k * cfg->dim_v * sizeof(float);
  return CHOCO_OK;
}

int choco_linear_workspace_bytes(const choco_linear_config* cfg, int backward, size_t* bytes_host) {
  if (!bytes_host) return CHOCO_E_INVAL;
  if (const int rc = check_linear(cfg)) return rc;
  if (!linear_fits(*cfg)) return CHOCO_E_UNSUPPORTED;
  *bytes_host = linear_layout(*cfg, backward != 0).total;
  return CHOCO_OK;
}

int choco_linear_forward(const choco_linear_config* cfg, const void* q_dev, const void* k_dev, const void* v_dev, const float* g_dev,
                         const float* h0_dev, const int32_t* lengths_dev, void* y_dev, float* h_last_dev, float* saved_dev,
                         void* workspace_dev, size_t workspace_bytes) {
  if (const int rc = check_linear(cfg)) return rc;
  const choco_linear_config& c = *cfg;
  if (c.batch == 0 || c.heads == 0) return CHOCO_OK;
  const size_t size = type_bytes(c.type);
  if (c.steps > 0) {
    if (!q_dev || !k_dev || !v_dev || !g_dev || !y_dev) return CHOCO_E_INVAL;
    if (!strides_ok(c, c.q_stride, c.q_heads, c.dim_k, false) || !strides_ok(c, c.k_stride, c.k_heads, c.dim_k, false) ||
        !strides_ok(c, c.v_stride, c.v_heads, c.dim_v, false) || !strides_ok(c, c.y_stride, c.heads, c.dim_v, true) ||
        !strides_ok(c, c.g_stride, c.heads, 1, false))
      return CHOCO_E_INVAL;
  }
  if (!aligned_to(q_dev, size) || !aligned_to(k_dev, size) || !aligned_to(v_dev, size) || !aligned_to(y_dev, size) || !aligned_to(g_dev, 4) ||
      !aligned_to(h0_dev, 4) || !aligned_to(lengths_dev, 4) || !aligned_to(h_last_dev, 4) || !aligned_to(saved_dev, 4))
    return CHOCO_E_INVAL;
  if (!linear_fits(c)) return CHOCO_E_UNSUPPORTED;
  const LinearLayout L = linear_layout(c, false);
  if (L.total > 0 && (!workspace_dev || !aligned_to(workspace_dev, 16))) return CHOCO_E_INVAL;
  if (L.total > workspace_bytes) return CHOCO_E_NOMEM;
  const LinearArgs A = linear_args(c, g_dev, lengths_dev);
  const Rows q{q_dev, c.q_stride, c.q_heads, c.dim_k}, k{k_dev, c.k_stride, c.k_heads, c.dim_k}, v{v_dev, c.v_stride, c.v_heads, c.dim_v},
      y{y_dev, c.y_stride, c.heads, c.dim_v};
  LinearPass P = pass_of(c, q, k, v, y_dev, c.y_stride);
  state_of(c, false, P);
  P.first = h0_dev;
  P.first_of = 1;
  P.last = h_last_dev;
  P.kept = saved_dev;
  P.kept_of = pieces_of(c) + 1;
  int rc = CHOCO_OK;
  with_type(c.type, [&](auto x) { rc = run_forward<decltype(x)>(c, A, P, q, k, v, y, (char*)workspace_dev); });
  return rc;
}

int choco_linear_backward(const choco_linear_config* cfg, const void* q_dev, const void* k_dev, const void* v_dev, const float* g_dev,
                          const int32_t* lengths_dev, const float* saved_dev, const void* dy_dev, const float* dlast_dev, void* dq_dev,
                          void* dk_dev, void* dv_dev, float* dg_dev, float* dh0_dev, void* workspace_dev, size_t workspace_bytes) {
  if (const int rc = check_linear(cfg)) return rc;
  const choco_linear_config& c = *cfg;
  if (c.batch == 0 || c.heads == 0) {
    if (c.heads == 0 || c.gate_steps || !dg_dev) return CHOCO_OK;
    if (!aligned_to(dg_dev, 4)) return CHOCO_E_INVAL;
    k_linear_gate_sums<<<dim3((uint32_t)c.heads), 256, 0, (hipStream_t)c.stream>>>(nullptr, 0, dg_dev);    // sums over nothing
    TRY_HIP(hipGetLastError());
    return CHOCO_OK;
  }
  const size_t size = type_bytes(c.type);
  if (c.steps > 0) {
    if (!q_dev || !k_dev || !v_dev || !g_dev || !saved_dev || !dy_dev || !dq_dev || !dk_dev || !dv_dev) return CHOCO_E_INVAL;
    if (!strides_ok(c, c.q_stride, c.q_heads, c.dim_k, false) || !strides_ok(c, c.k_stride, c.k_heads, c.dim_k, false) ||
        !strides_ok(c, c.v_stride, c.v_heads, c.dim_v, false) || !strides_ok(c, c.y_stride, c.heads, c.dim_v, false) ||
        !strides_ok(c, c.g_stride, c.heads, 1, false) || !strides_ok(c, c.dq_stride, c.q_heads, c.dim_k, true) ||
        !strides_ok(c, c.dk_stride, c.k_heads, c.dim_k, true) || !strides_ok(c, c.dv_stride, c.v_heads, c.dim_v, true))
      return CHOCO_E_INVAL;
  }
  if (!aligned_to(q_dev, size) || !aligned_to(k_dev, size) || !aligned_to(v_dev, size) || !aligned_to(dy_dev, size) ||
      !aligned_to(dq_dev, size) || !aligned_to(dk_dev, size) || !aligned_to(dv_dev, size) || !aligned_to(g_dev, 4) ||
      !aligned_to(lengths_dev, 4) || !aligned_to(saved_dev, 4) || !aligned_to(dlast_dev, 4) || !aligned_to(dg_dev, 4) || !aligned_to(dh0_dev, 4))
    return CHOCO_E_INVAL;
  if (!linear_fits(c)) return CHOCO_E_UNSUPPORTED;
  const LinearLayout L = linear_layout(c, true);
  if (L.total > 0 && (!workspace_dev || !aligned_to(workspace_dev, 16))) return CHOCO_E_INVAL;
  if (L.total > workspace_bytes) return CHOCO_E_NOMEM;
  const LinearArgs A = linear_args(c, g_dev, lengths_dev);
  int rc = CHOCO_OK;
  with_type(c.type, [&](auto x) {
    rc = run_backward<decltype(x)>(c, A, q_dev, k_dev, v_dev, saved_dev, dy_dev, dlast_dev, dq_dev, dk_dev, dv_dev, dg_dev, dh0_dev,
                                   (char*)workspace_dev);
  });
  return rc;
}

}  // extern "C"
