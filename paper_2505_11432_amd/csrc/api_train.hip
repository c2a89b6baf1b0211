// extern "C" entry points of what follows the layer in a training step: the vocabulary loss, clipping and the AdamW update.  Arguments are
// checked before any HIP call; declarations and contracts are in include/moe.h.
#include <type_traits>

#include "optim.h"
#include "vocab_loss.h"

namespace moe {
namespace {

bool vocab_sizes_ok(int T, int d, int V) { return T >= 0 && d > 0 && V > 0; }
bool vocab_types_ok(int T, int d, int V, moe_dtype dt, moe_dtype grad_dt, bool grad) {
  if (dt != MOE_F32 && dt != MOE_BF16) return false;
  if (dt == MOE_F32 ? grad_dt != MOE_F32 : grad_dt != MOE_F32 && grad_dt != MOE_BF16) return false;
  // (tiles are counted in 32 bits)
  const long tiles = ((long)T / 64 + 1) * ((long)V / 128 + 1);
  if (grad && dt == MOE_BF16 && !vocab_dx_takes(128, (long)align_up((size_t)V, 64))) return false;
  return d % 16 == 0 && d <= MOE_VOCAB_MAX_WIDTH && V <= MOE_VOCAB_MAX && T <= MOE_VOCAB_MAX_ROWS && tiles <= 0x3fffffffL;
}

int vocab_call(const VocabProblem& q, int piece_rows, void* workspace, size_t ws_bytes, void* stream) {
  const VocabPlan p = vocab_plan(q.T, q.d, q.V, q.dt, q.grad_dt, piece_rows, q.grad);
  if (!workspace || !aligned16(workspace) || ws_bytes < p.bytes) return MOE_ERR_WORKSPACE;
  if (q.grad) {
    // d_w's product reads x after dx is written
    const size_t es = dtype_size(q.dt), x = (size_t)q.T * q.d * es, w = (size_t)q.V * q.d * es, d_w = (size_t)q.V * q.d * dtype_size(q.grad_dt);
    if (!apart(q.dx, x, q.x, x) || !apart(q.dx, x, q.w, w) || !apart(q.d_w, d_w, q.x, x) || !apart(q.d_w, d_w, q.w, w) || !apart(q.dx, x, q.d_w, d_w))
      return MOE_ERR_INVALID;
  }
  return launch_vocab_loss(q, p, static_cast<char*>(workspace), as_stream(stream));
}

// sums of elements and chunks into the entries, whose types are set
template <typename Entry> bool number_entries(const int64_t* numel, int n, Entry* table) {
  int64_t at = 0, chunk = 0;
  for (int i = 0; i <= n; ++i) {
    if (i == n) table[i] = Entry{};
    table[i].first = at;
    if constexpr (std::is_same_v<Entry, ClipEntry>) table[i].chunk = (int32_t)chunk;
    if (i == n) break;
    if (numel[i] < 0 || numel[i] > INT64_MAX / 16 - at) return false;
    at += numel[i];
    chunk += (numel[i] + chunk_elements(table[i]) - 1) / chunk_elements(table[i]) + 1;
    if (chunk > INT32_MAX / 2) return false;
  }
  return true;
}

bool at_elements(const void* p, size_t es) { return (reinterpret_cast<uintptr_t>(p) & (es - 1)) == 0; }

bool adamw_lists_ok(int n, void* const* params, const void* const* grads, void* const* m, void* const* v, const int64_t* numel, const void* table) {
  return n >= 0 && table && (n == 0 || (params && grads && m && v && numel));
}
// type(i): of gradient i; bf16_mark: what is set in the addresses of those in bf16
template <typename Type>
int adamw_table(int n, void* const* params, const void* const* grads, Type type, void* const* m, void* const* v, void* const* weights, const int64_t* numel,
                uintptr_t bf16_mark, void* table) {
  AdamwEntry* e = static_cast<AdamwEntry*>(table);
  for (int i = 0; i < n; ++i) {
    const moe_dtype dt = type(i);
    if (dt != MOE_F32 && dt != MOE_BF16) return MOE_ERR_UNSUPPORTED;
    if (numel[i] > 0 && (!params[i] || !grads[i] || !m[i] || !v[i])) return MOE_ERR_INVALID;
    void* w = weights ? weights[i] : nullptr;
    if (!at_elements(params[i], 4) || !at_elements(m[i], 4) || !at_elements(v[i], 4) || !at_elements(grads[i], dtype_size(dt)) || !at_elements(w, 2))
      return MOE_ERR_UNSUPPORTED;
    const uintptr_t g = reinterpret_cast<uintptr_t>(grads[i]) | (dt == MOE_BF16 ? bf16_mark : 0);
    e[i] = AdamwEntry{params[i], reinterpret_cast<const void*>(g), m[i], v[i], w, 0};
  }
  return number_entries(numel, n, e) ? MOE_OK : MOE_ERR_INVALID;
}

}  // namespace
}  // namespace moe

using namespace moe;

extern "C" {

size_t moe_vocab_workspace_bytes(int T, int d, int V, moe_dtype dt, moe_dtype grad_dt, int piece_rows, int gradients) {
  if (!vocab_sizes_ok(T, d, V) || piece_rows < 0 || !vocab_types_ok(T, d, V, dt, gradients ? grad_dt : dt, gradients != 0)) return 0;
  return T == 0 ? 256 : vocab_plan(T, d, V, dt, gradients ? grad_dt : dt, piece_rows, gradients != 0).bytes;
}

int moe_vocab_score(const void* x, const void* w, const int32_t* target, moe_dtype dt, int T, int d, int V, int piece_rows, float* loss, float* lse,
                    void* workspace, size_t ws_bytes, void* stream) {
  if (!vocab_sizes_ok(T, d, V) || piece_rows < 0) return MOE_ERR_INVALID;
  if (!vocab_types_ok(T, d, V, dt, dt, false)) return MOE_ERR_UNSUPPORTED;
  if (T == 0) return MOE_OK;
  if (!x || !w || !target || !loss || !lse) return MOE_ERR_INVALID;
  if (!aligned16(x) || !aligned16(w) || !at_elements(target, 4) || !at_elements(loss, 4) || !at_elements(lse, 4)) return MOE_ERR_UNSUPPORTED;
  VocabProblem q{};
  q.x = x; q.w = w; q.target = target; q.T = T; q.d = d; q.V = V; q.dt = dt; q.grad_dt = dt; q.loss = loss; q.lse = lse;
  return vocab_call(q, piece_rows, workspace, ws_bytes, stream);
}

int moe_vocab_loss(const void* x, const void* w, const int32_t* target, const float* token_w, moe_dtype dt, int T, int d, int V, int piece_rows,
                   float* total, float* loss, float* lse, void* dx, void* d_w, moe_dtype grad_dt, int accumulate, void* workspace, size_t ws_bytes,
                   void* stream) {
  if (!vocab_sizes_ok(T, d, V) || piece_rows < 0) return MOE_ERR_INVALID;
  if (!vocab_types_ok(T, d, V, dt, grad_dt, true)) return MOE_ERR_UNSUPPORTED;
  if (T == 0) return MOE_OK;
  if (!x || !w || !target || !total || !loss || !lse || !dx || !d_w) return MOE_ERR_INVALID;
  if (!aligned16(x) || !aligned16(w) || !aligned16(dx) || !aligned16(d_w) || !at_elements(target, 4) || !at_elements(token_w, 4) ||
      !at_elements(total, 4) || !at_elements(loss, 4) || !at_elements(lse, 4))
    return MOE_ERR_UNSUPPORTED;
  VocabProblem q{};
  q.x = x; q.w = w; q.target = target; q.token_w = token_w; q.T = T; q.d = d; q.V = V; q.dt = dt;
  q.loss = loss; q.lse = lse; q.grad = true; q.total = total; q.dx = dx; q.d_w = d_w; q.grad_dt = grad_dt; q.accumulate = accumulate != 0;
  return vocab_call(q, piece_rows, workspace, ws_bytes, stream);
}

size_t moe_grad_clip_table_bytes(int n) { return n < 0 ? 0 : ((size_t)n + 1) * sizeof(ClipEntry); }

int moe_grad_clip_table(int n, const void* const* grads, void* const* outs, const int64_t* numel, const int32_t* dtypes, void* table) {
  if (n < 0 || !table || (n > 0 && (!grads || !numel || !dtypes))) return MOE_ERR_INVALID;
  ClipEntry* e = static_cast<ClipEntry*>(table);
  for (int i = 0; i < n; ++i) {
    if (dtypes[i] != MOE_F32 && dtypes[i] != MOE_BF16) return MOE_ERR_UNSUPPORTED;
    const size_t es = dtype_size((moe_dtype)dtypes[i]);
    if (numel[i] > 0 && !grads[i]) return MOE_ERR_INVALID;
    if (!at_elements(grads[i], es) || (outs && !at_elements(outs[i], es))) return MOE_ERR_UNSUPPORTED;
    e[i] = ClipEntry{grads[i], outs ? outs[i] : nullptr, 0, dtypes[i], 0};
  }
  return number_entries(numel, n, e) ? MOE_OK : MOE_ERR_INVALID;
}

size_t moe_grad_clip_workspace_bytes(void) { return kNormParts * sizeof(double); }

int moe_grad_clip(const void* table, int n, int64_t total, double max_norm, int write, float* norm, float* coef, void* workspace, size_t ws_bytes,
                  void* stream) {
  if (n < 0 || total < 0 || !(max_norm >= 0)) return MOE_ERR_INVALID;
  if (!table || !norm || !coef) return MOE_ERR_INVALID;
  if (!at_elements(table, 8) || !at_elements(norm, 4) || !at_elements(coef, 4)) return MOE_ERR_UNSUPPORTED;
  if (!workspace || !aligned16(workspace) || ws_bytes < moe_grad_clip_workspace_bytes()) return MOE_ERR_WORKSPACE;
  return launch_grad_clip(static_cast<const ClipEntry*>(table), n, total, max_norm, write, norm, coef, static_cast<double*>(workspace), as_stream(stream));
}

size_t moe_adamw_table_bytes(int n) { return n < 0 ? 0 : ((size_t)n + 1) * sizeof(AdamwEntry); }

int moe_adamw_table(int n, void* const* params, const void* const* grads, void* const* m, void* const* v, void* const* weights, const int64_t* numel,
                    moe_dtype grad_dt, void* table) {
  if (!adamw_lists_ok(n, params, grads, m, v, numel, table)) return MOE_ERR_INVALID;
  if (grad_dt != MOE_F32 && grad_dt != MOE_BF16) return MOE_ERR_UNSUPPORTED;
  return adamw_table(n, params, grads, [=](int) { return grad_dt; }, m, v, weights, numel, 0, table);
}

int moe_adamw_table_mixed(int n, void* const* params, const void* const* grads, const int32_t* grad_dtypes, void* const* m, void* const* v,
                          void* const* weights, const int64_t* numel, void* table) {
  if (!adamw_lists_ok(n, params, grads, m, v, numel, table) || (n > 0 && !grad_dtypes)) return MOE_ERR_INVALID;
  return adamw_table(n, params, grads, [=](int i) { return (moe_dtype)grad_dtypes[i]; }, m, v, weights, numel, kBf16Gradient, table);
}

int moe_adamw(const void* table, int n, int64_t total, moe_dtype grad_dt, const float* lr, int32_t* step, const float* coef, double beta1, double beta2,
              double eps, double weight_decay, void* workspace, size_t ws_bytes, void* stream) {
  if (n < 0 || total < 0 || !table || !lr || !step) return MOE_ERR_INVALID;
  if (!(beta1 >= 0 && beta1 < 1) || !(beta2 >= 0 && beta2 < 1) || !(eps >= 0) || !(weight_decay >= 0)) return MOE_ERR_INVALID;
  if (grad_dt != MOE_F32 && grad_dt != MOE_BF16 && grad_dt != MOE_GRADS_MIXED) return MOE_ERR_UNSUPPORTED;
  if (!at_elements(table, 8) || !at_elements(lr, 4) || !at_elements(step, 4) || !at_elements(coef, 4)) return MOE_ERR_UNSUPPORTED;
  if (!workspace || !at_elements(workspace, 4) || ws_bytes < MOE_ADAMW_WS_BYTES) return MOE_ERR_WORKSPACE;
  return launch_adamw(static_cast<const AdamwEntry*>(table), n, total, grad_dt, lr, step, coef, AdamwHyper{beta1, beta2, eps, weight_decay},
                      static_cast<unsigned*>(workspace), as_stream(stream));
}

}  // extern "C"
