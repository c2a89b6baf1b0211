// extern "C" entry points of the parts around the layer: the embedding, the norms before and after a block, orthogonalised updates.  Arguments are
// checked before any HIP call; declarations and contracts are in include/moe.h.
#include <cmath>
#include <initializer_list>

#include "block.h"
#include "newton_schulz.h"

namespace moe {
namespace {

bool at_elements(const void* p, size_t es) { return (reinterpret_cast<uintptr_t>(p) & (es - 1)) == 0; }

// (a product with an infinity or no number would leave something in the rows of zeros)
bool scale_ok(double scale) { return std::isfinite((float)scale); }
bool embedding_sizes_ok(int T, int d, int V) { return T >= 0 && d > 0 && V > 0; }
// (the sort's keys are words, a launch holds less than 2^32 threads)
bool embedding_takes(int T, int d, int V) {
  return d % 16 == 0 && d <= MOE_VOCAB_MAX_WIDTH && V <= MOE_VOCAB_MAX && T <= MOE_VOCAB_MAX_ROWS && (long)T * d < 1L << 36;
}
bool grad_types_ok(moe_dtype dt, moe_dtype grad_dt) {
  return (dt == MOE_F32 && grad_dt == MOE_F32) || (dt == MOE_BF16 && (grad_dt == MOE_F32 || grad_dt == MOE_BF16));
}

struct Range { const void* p; size_t bytes; };
// no output shares a byte with an input or another output (NULL: none), but for the pairs that `same` allows to be one buffer
bool outputs_apart(std::initializer_list<Range> outputs, std::initializer_list<Range> inputs, std::initializer_list<const void*> same_out,
                   std::initializer_list<const void*> same_in) {
  auto allowed = [&](const void* o, const void* i) {
    if (o != i) return false;
    bool a = false, b = false;
    for (const void* p : same_out) a = a || p == o;
    for (const void* p : same_in) b = b || p == i;
    return a && b;
  };
  for (const Range* o = outputs.begin(); o != outputs.end(); ++o) {
    if (!o->p) continue;
    for (const Range& i : inputs)
      if (i.p && !allowed(o->p, i.p) && !apart(o->p, o->bytes, i.p, i.bytes)) return false;
    for (const Range* q = o + 1; q != outputs.end(); ++q)
      if (q->p && !apart(o->p, o->bytes, q->p, q->bytes)) return false;
  }
  return true;
}

// sizes, steps and workspace of a batch of matrices; fills in the problem and how it is taken
int orthogonal_problem(int batch, int rows, int cols, int steps, const double* coefficients, int piece, const void* workspace, size_t ws_bytes, MuonProblem* q,
                       OrthPlan* plan) {
  if (batch < 0 || rows < 1 || cols < 1 || piece < 0 || steps < 1 || steps > MOE_ORTH_MAX_STEPS) return MOE_ERR_INVALID;
  if (!orth_takes(batch, rows, cols, piece)) return MOE_ERR_UNSUPPORTED;
  for (int k = 0; k < steps; ++k)
    q->coef[k] = coefficients ? OrthCoef{coefficients[3 * k], coefficients[3 * k + 1], coefficients[3 * k + 2]} : kDefaultCoef;
  if (!orth_coefficients_ok(q->coef, steps, rows, cols)) return MOE_ERR_UNSUPPORTED;
  q->batch = batch; q->rows = rows; q->cols = cols; q->steps = steps;
  *plan = orth_plan(batch, rows, cols, piece);
  if (batch > 0 && (!workspace || !aligned16(workspace) || ws_bytes < plan->bytes)) return MOE_ERR_WORKSPACE;
  return MOE_OK;
}

}  // namespace
}  // namespace moe

using namespace moe;

extern "C" {

size_t moe_embedding_workspace_bytes(int T, int d, int V) {
  return embedding_sizes_ok(T, d, V) && embedding_takes(T, d, V) ? embedding_plan(T, d, V).bytes : 0;
}

int moe_embedding_fwd(const void* table, const int32_t* tokens, moe_dtype dt, int T, int d, int V, double scale, void* out, void* stream) {
  if (!embedding_sizes_ok(T, d, V) || !scale_ok(scale)) return MOE_ERR_INVALID;
  if (!embedding_takes(T, d, V) || !grad_types_ok(dt, dt)) return MOE_ERR_UNSUPPORTED;
  if (T == 0) return MOE_OK;
  if (!table || !tokens || !out) return MOE_ERR_INVALID;
  if (!aligned16(table) || !aligned16(out) || !at_elements(tokens, 4)) return MOE_ERR_UNSUPPORTED;
  const size_t es = dtype_size(dt);
  if (!outputs_apart({{out, (size_t)T * d * es}}, {{table, (size_t)V * d * es}, {tokens, (size_t)T * 4}}, {}, {})) return MOE_ERR_INVALID;
  return launch_embedding_fwd(table, tokens, dt, T, d, V, (float)scale, out, as_stream(stream));
}

int moe_embedding_bwd(const int32_t* tokens, const void* dy, moe_dtype dt, int T, int d, int V, double scale, void* d_table, moe_dtype grad_dt,
                      int accumulate, void* workspace, size_t ws_bytes, void* stream) {
  if (!embedding_sizes_ok(T, d, V) || !scale_ok(scale)) return MOE_ERR_INVALID;
  if (!embedding_takes(T, d, V) || !grad_types_ok(dt, grad_dt)) return MOE_ERR_UNSUPPORTED;
  if (T == 0 && accumulate) return MOE_OK;
  if (!d_table || (T > 0 && (!tokens || !dy))) return MOE_ERR_INVALID;
  if (!aligned16(d_table) || !aligned16(dy) || !at_elements(tokens, 4)) return MOE_ERR_UNSUPPORTED;
  const EmbeddingPlan p = embedding_plan(T, d, V);
  if (!workspace || !aligned16(workspace) || ws_bytes < p.bytes) return MOE_ERR_WORKSPACE;
  if (T > 0 && !outputs_apart({{d_table, (size_t)V * d * dtype_size(grad_dt)}}, {{dy, (size_t)T * d * dtype_size(dt)}, {tokens, (size_t)T * 4}}, {}, {}))
    return MOE_ERR_INVALID;
  return launch_embedding_bwd(tokens, dy, dt, T, d, V, (float)scale, d_table, grad_dt, accumulate != 0, p, static_cast<char*>(workspace),
                              as_stream(stream));
}

// (an empty batch's rows may be NULL whatever is asked for; places of rows, to the end of the last team's share, are counted in 31 bits)
static int norm_arguments(const void* y, const float* w_after, const float* gate, moe_dtype dt, int T, int d, int gate_rows, double alpha, double eps) {
  if (T < 0 || d <= 0 || !(eps >= 0) || alpha != alpha || (gate && gate_rows < 1)) return MOE_ERR_INVALID;
  if ((dt != MOE_F32 && dt != MOE_BF16) || d % 16 != 0 || d > MOE_NORM_MAX_WIDTH || T > MOE_NORM_MAX_ROWS) return MOE_ERR_UNSUPPORTED;
  return T > 0 && !y && (w_after || gate || alpha != 1.0) ? MOE_ERR_INVALID : MOE_OK;
}

int moe_block_norm_fwd(const void* x, const void* y, const float* w_after, const float* gate, const float* w_before, moe_dtype dt, int T, int d,
                       int gate_rows, double alpha, double eps, void* out, void* h, void* stream) {
  if (const int rc = norm_arguments(y, w_after, gate, dt, T, d, gate_rows, alpha, eps)) return rc;
  if (T == 0) return MOE_OK;
  if (!x || (y == nullptr) != (out == nullptr) || (w_before == nullptr) != (h == nullptr) || (!y && !w_before)) return MOE_ERR_INVALID;
  for (const void* p : {x, y, (const void*)out, (const void*)h, (const void*)w_after, (const void*)gate, (const void*)w_before})
    if (!aligned16(p)) return MOE_ERR_UNSUPPORTED;
  const size_t rows = (size_t)T * d * dtype_size(dt), vec = (size_t)d * 4, gates = gate ? ((size_t)T + gate_rows - 1) / gate_rows * vec : 0;
  if (!outputs_apart({{out, rows}, {h, rows}}, {{x, rows}, {y, rows}, {w_after, vec}, {gate, gates}, {w_before, vec}}, {out}, {x, y})) return MOE_ERR_INVALID;
  NormProblem q{};
  q.x = x; q.y = y; q.w_after = w_after; q.gate = gate; q.w_before = w_before; q.dt = dt; q.T = T; q.d = d; q.gate_rows = gate ? gate_rows : 1;
  q.alpha = (float)alpha; q.eps = (float)eps; q.out = out; q.h = h;
  return launch_norm_fwd(q, as_stream(stream));
}

size_t moe_block_norm_workspace_bytes(int T, int d, moe_dtype dt, int after, int gate, int before) {
  if (T < 0 || T > MOE_NORM_MAX_ROWS || d <= 0 || d % 16 != 0 || d > MOE_NORM_MAX_WIDTH || (dt != MOE_F32 && dt != MOE_BF16)) return 0;
  return norm_bwd_plan(T, d, dt, after != 0, gate != 0, before != 0).bytes;
}

int moe_block_norm_bwd(const void* out, const void* y, const float* w_after, const float* gate, const float* w_before, const void* d_out, const void* d_h,
                       moe_dtype dt, int T, int d, int gate_rows, double alpha, double eps, void* dx, void* dy, float* d_w_after, float* d_gate,
                       float* d_w_before, int accumulate, void* workspace, size_t ws_bytes, void* stream) {
  // (without a norm behind the block or a gate y is not read: dy says whether a block ends here)
  if (const int rc = norm_arguments(dy, w_after, gate, dt, T, d, gate_rows, alpha, eps)) return rc;
  if (T == 0) return MOE_OK;
  if ((w_after == nullptr) != (d_w_after == nullptr) || (gate == nullptr) != (d_gate == nullptr) || (w_before == nullptr) != (d_w_before == nullptr) ||
      (w_before == nullptr) != (d_h == nullptr))
    return MOE_ERR_INVALID;
  if (!dx || (w_before && !out) || ((w_after || gate) && !y) || (!d_out && !d_h)) return MOE_ERR_INVALID;
  for (const void* p : {out, y, d_out, d_h, (const void*)dx, (const void*)dy, (const void*)w_after, (const void*)gate, (const void*)w_before,
                        (const void*)d_w_after, (const void*)d_gate, (const void*)d_w_before})
    if (!aligned16(p)) return MOE_ERR_UNSUPPORTED;
  const NormPlan p = norm_bwd_plan(T, d, dt, w_after, gate, w_before);
  if (!workspace || !aligned16(workspace) || ws_bytes < p.bytes) return MOE_ERR_WORKSPACE;
  const size_t rows = (size_t)T * d * dtype_size(dt), vec = (size_t)d * 4, gates = gate ? ((size_t)T + gate_rows - 1) / gate_rows * vec : 0;
  const void* read_out = w_before ? out : nullptr;
  const void* read_y = w_after || gate ? y : nullptr;
  if (!outputs_apart({{dx, rows}, {dy, rows}, {d_w_after, vec}, {d_gate, gates}, {d_w_before, vec}},
                     {{read_out, rows}, {read_y, rows}, {d_out, rows}, {d_h, rows}, {w_after, vec}, {gate, gates}, {w_before, vec}}, {dx, dy}, {d_out, d_h, read_y}) ||
      (dx == read_y && dx != d_out && dx != d_h))
    return MOE_ERR_INVALID;
  NormProblem q{};
  q.x = read_out; q.y = read_y; q.w_after = w_after; q.gate = gate; q.w_before = w_before; q.dt = dt; q.T = T; q.d = d; q.gate_rows = gate ? gate_rows : 1;
  q.alpha = (float)alpha; q.eps = (float)eps; q.d_out = d_out; q.d_h = d_h; q.dx = dx; q.dy = dy;
  q.d_w_after = d_w_after; q.d_gate = d_gate; q.d_w_before = d_w_before; q.accumulate = accumulate != 0;
  return launch_norm_bwd(q, p, static_cast<float*>(workspace), as_stream(stream));
}

size_t moe_orthogonal_workspace_bytes(int batch, int rows, int cols, int piece) {
  if (batch < 0 || rows < 1 || cols < 1 || piece < 0 || !orth_takes(batch, rows, cols, piece)) return 0;
  return orth_plan(batch, rows, cols, piece).bytes;
}

int moe_orthogonalize(const void* x, moe_dtype dt, int batch, int rows, int cols, int steps, const double* coefficients, int piece, void* out,
                      moe_dtype out_dt, void* workspace, size_t ws_bytes, void* stream) {
  MuonProblem q{};
  OrthPlan plan{};
  const int rc = orthogonal_problem(batch, rows, cols, steps, coefficients, piece, workspace, ws_bytes, &q, &plan);
  if (rc != MOE_OK && rc != MOE_ERR_WORKSPACE) return rc;
  if ((dt != MOE_F32 && dt != MOE_BF16) || (out_dt != MOE_F32 && out_dt != MOE_BF16)) return MOE_ERR_UNSUPPORTED;
  if (batch == 0) return MOE_OK;
  if (!x || !out) return MOE_ERR_INVALID;
  if (!at_elements(x, dtype_size(dt)) || !at_elements(out, dtype_size(out_dt))) return MOE_ERR_UNSUPPORTED;
  const size_t n = (size_t)batch * rows * cols;
  // (in place a piece is read before it is written; with two types the pieces would lie elsewhere)
  if (!(out == x && dt == out_dt) && !apart(out, n * dtype_size(out_dt), x, n * dtype_size(dt))) return MOE_ERR_INVALID;
  if (rc != MOE_OK) return rc;
  q.u = x; q.u_dt = dt; q.out = out; q.out_dt = out_dt;
  return launch_orth(q, plan, static_cast<char*>(workspace), as_stream(stream));
}

int moe_muon(float* p, const void* grad, moe_dtype grad_dt, float* m, void* weights, int batch, int rows, int cols, const float* lr, const float* coef,
             double momentum, int nesterov, double weight_decay, double scale, int steps, const double* coefficients, int piece, void* workspace,
             size_t ws_bytes, void* stream) {
  return moe_muon_eps(p, grad, grad_dt, m, weights, batch, rows, cols, lr, coef, momentum, nesterov, weight_decay, scale, MOE_MUON_EPS, steps, coefficients,
                      piece, workspace, ws_bytes, stream);
}

int moe_muon_eps(float* p, const void* grad, moe_dtype grad_dt, float* m, void* weights, int batch, int rows, int cols, const float* lr, const float* coef,
                 double momentum, int nesterov, double weight_decay, double scale, double eps, int steps, const double* coefficients, int piece,
                 void* workspace, size_t ws_bytes, void* stream) {
  MuonProblem q{};
  OrthPlan plan{};
  const int rc = orthogonal_problem(batch, rows, cols, steps, coefficients, piece, workspace, ws_bytes, &q, &plan);
  if (rc != MOE_OK && rc != MOE_ERR_WORKSPACE) return rc;
  if (!(momentum >= 0 && momentum < 1) || !(weight_decay >= 0) || !(scale >= 0) || !(eps >= 0)) return MOE_ERR_INVALID;
  if (grad_dt != MOE_F32 && grad_dt != MOE_BF16) return MOE_ERR_UNSUPPORTED;
  if (batch == 0) return MOE_OK;
  if (!p || !grad || !m || !lr) return MOE_ERR_INVALID;
  if (!at_elements(p, 4) || !at_elements(grad, dtype_size(grad_dt)) || !at_elements(m, 4) || !at_elements(weights, 2) || !at_elements(lr, 4) ||
      !at_elements(coef, 4))
    return MOE_ERR_UNSUPPORTED;
  const size_t n = (size_t)batch * rows * cols;
  if (!outputs_apart({{p, n * 4}, {m, n * 4}, {weights, n * 2}}, {{grad, n * dtype_size(grad_dt)}, {lr, 4}, {coef, 4}}, {}, {})) return MOE_ERR_INVALID;
  if (rc != MOE_OK) return rc;
  q.u = grad; q.u_dt = grad_dt; q.p = p; q.m = m; q.w = weights; q.lr = lr; q.factor = coef;
  q.momentum = (float)momentum; q.nesterov = nesterov != 0; q.decay = weight_decay; q.scale = (float)scale; q.eps = eps;
  return launch_orth(q, plan, static_cast<char*>(workspace), as_stream(stream));
}

}  // extern "C"
