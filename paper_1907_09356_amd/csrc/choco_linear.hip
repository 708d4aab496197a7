// Host side of choco_train.h's linear attention: argument checks, workspace layout, kernel launches.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <initializer_list>
#include <type_traits>
#include <utility>

#include "choco_host.h"
#include "choco_linear.h"

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
int slices_of(int dim) { return (dim + kLinearSlice - 1) / kLinearSlice; }
int64_t rows_of(const choco_linear_config& c) { return c.batch * c.heads; }

// Every launch of a call fits, and what it keeps stays far from 64 bits.
bool linear_fits(const choco_linear_config& c) {
  const double rows = (double)rows_of(c), pieces = (double)pieces_of(c) + 1.0;
  if (rows * pieces * c.dim_k * c.dim_v > 1125899906842624.0 || rows * (double)c.steps * 512.0 > 1125899906842624.0) return false;
  return launch_fits(rows * pieces * slices_of(CHOCO_LINEAR_MAX_DIM), 256);
}

struct LinearLayout {
  size_t later, dots, sums, wide, total;
};
LinearLayout linear_layout(const choco_linear_config& c, bool back) {
  LinearLayout L{};
  Parts parts;
  if (c.batch == 0 || c.heads == 0 || !back) return L;
  const size_t rows = (size_t)rows_of(c), state = (size_t)c.dim_k * c.dim_v, steps = (size_t)c.steps;
  L.later = parts.take(rows * (size_t)pieces_of(c) * state * sizeof(float));
  L.dots = parts.take(rows * steps * 2 * slices_of(c.dim_k) * sizeof(float));
  L.sums = parts.take(rows * (size_t)pieces_of(c) * sizeof(float));
  size_t most = 0;
  if (c.q_heads != c.heads || c.k_heads != c.heads) most = c.dim_k;
  if (c.v_heads != c.heads) most = std::max(most, (size_t)c.dim_v);
  L.wide = parts.take(rows * steps * most * sizeof(float));
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

template <class T>
int run_pass(const choco_linear_config& c, const LinearArgs& A, const LinearPass& P) {
  const dim3 grid((uint32_t)(rows_of(c) * slices_of(P.dc)));
  const hipStream_t stream = (hipStream_t)c.stream;
  if (P.da <= 64) k_linear_steps<T, 16><<<grid, 256, 0, stream>>>(A, P);
  else if (P.da <= 128) k_linear_steps<T, 32><<<grid, 256, 0, stream>>>(A, P);
  else k_linear_steps<T, 64><<<grid, 256, 0, stream>>>(A, P);
  TRY_HIP(hipGetLastError());
  return CHOCO_OK;
}

template <class T>
int run_backward(const choco_linear_config& c, const LinearArgs& A, const void* q, const void* k, const void* v, const float* saved,
                 const void* dy, const float* dlast, void* dq, void* dk, void* dv, float* dg, float* dh0, char* ws) {
  const hipStream_t stream = (hipStream_t)c.stream;
  const LinearLayout L = linear_layout(c, true);
  const Rows Q{q, c.q_stride, c.q_heads, c.dim_k}, K{k, c.k_stride, c.k_heads, c.dim_k}, V{v, c.v_stride, c.v_heads, c.dim_v},
      Y{dy, c.y_stride, c.heads, c.dim_v};
  const int64_t rows = rows_of(c), pieces = pieces_of(c), state = (int64_t)c.dim_k * c.dim_v;
  float* const later = (float*)(ws + L.later);
  float* const q_dots = (float*)(ws + L.dots);
  float* const k_dots = q_dots + rows * c.steps * slices_of(c.dim_k);
  // a gradient of heads that share one: of every head to the workspace, then added up
  const auto through = [&](LinearPass P, int32_t heads, int32_t dim) -> int {
    if (heads == c.heads) return run_pass<T>(c, A, P);
    LinearPass W = P;
    W.out = ws + L.wide;
    W.wide = true;
    W.out_head = dim;
    W.out_step = (int64_t)c.heads * dim;
    W.out_seq = W.out_step * c.steps;
    if (const int rc = run_pass<T>(c, A, W)) return rc;
    const int64_t count = c.batch * c.steps * heads * dim;
    if (count == 0) return CHOCO_OK;
    k_linear_share<T><<<dim3((uint32_t)std::min<int64_t>(4096, (count + 255) / 256)), 256, 0, stream>>>(
        (const float*)W.out, P.out, c.batch * c.steps, c.steps, heads, c.heads / heads, dim, P.out_seq, P.out_step, P.out_head);
    TRY_HIP(hipGetLastError());
    return CHOCO_OK;
  };
  LinearPass P = pass_of(c, Y, V, K, dq, c.dq_stride);
  state_of(c, true, P);
  P.first = saved;      // (with its own distance from one sequence's to the next)
  P.x = q; P.x_seq = c.q_stride[0]; P.x_step = c.q_stride[1]; P.x_head = c.q_stride[2]; P.x_share = c.heads / c.q_heads;
  P.dots = dg ? q_dots : nullptr;
  P.first_of = pieces + 1;
  if (const int rc = through(P, c.q_heads, c.dim_k)) return rc;
  P = pass_of(c, V, Y, Q, dk, c.dk_stride);
  state_of(c, true, P);
  P.back = true;
  P.first = dlast;
  P.first_of = 1;
  P.x = k; P.x_seq = c.k_stride[0]; P.x_step = c.k_stride[1]; P.x_head = c.k_stride[2]; P.x_share = c.heads / c.k_heads;
  P.dots = dg ? k_dots : nullptr;
  if (const int rc = through(P, c.k_heads, c.dim_k)) return rc;
  P = pass_of(c, K, Q, Y, dv, c.dv_stride);
  state_of(c, false, P);
  P.back = true;
  P.first = dlast;
  P.first_of = 1;
  P.last = dh0;
  P.kept = dg ? later : nullptr;
  P.kept_of = pieces;
  if (const int rc = through(P, c.v_heads, c.dim_v)) return rc;
  if (!dg) return CHOCO_OK;
  LinearGates G{};
  G.q_dots = q_dots; G.k_dots = k_dots;
  G.saved = saved; G.later = later; G.dlast = dlast;
  G.saved_of = pieces + 1; G.later_of = pieces;
  G.q_slices = G.k_slices = slices_of(c.dim_k);
  G.state = (int32_t)state;
  G.pieces = pieces;
  G.sums = !c.gate_steps;
  G.dg = G.sums ? (float*)(ws + L.sums) : dg;
  if (pieces > 0) {
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
  LinearPass P = pass_of(c, {q_dev, c.q_stride, c.q_heads, c.dim_k}, {k_dev, c.k_stride, c.k_heads, c.dim_k},
                         {v_dev, c.v_stride, c.v_heads, c.dim_v}, y_dev, c.y_stride);
  state_of(c, false, P);
  P.first = h0_dev;
  P.first_of = 1;
  P.last = h_last_dev;
  P.kept = saved_dev;
  P.kept_of = pieces_of(c) + 1;
  int rc = CHOCO_OK;
  with_type(c.type, [&](auto x) { rc = run_pass<decltype(x)>(c, A, P); });
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
