// What the entry points (api_block.hip) and the kernels (embedding.hip, norm.hip) of the parts around the layer share.
#pragma once
#include "moe_common.h"

namespace moe {

// ---- embedding -----------------------------------------------------------------------------
constexpr int kSortTile = 4096;             // tokens that a workgroup sorts at a time (twice as many where one workgroup sorts all)
constexpr int kSortOne = 2 * kSortTile;
constexpr int kOneBits = 19;                // bits of a word where one workgroup sorts all
constexpr int kMaxDigit = 9;                // bits of a sorting pass
constexpr int kFewTokens = 2048;            // up to so many are not sorted, if the workgroups that look through them
constexpr long kFewLooks = 1L << 24;        // look at no more than so many
struct EmbeddingPlan {
  bool few, zero_first;                     // no sort; the gradient is zeroed beside the sort
  int chunk, chunks;                        // sorted tokens that one wave adds up
  int tiles, passes, bits;                  // of the sort: workgroups, passes and bits of each
  size_t pairs, counts, parts, bytes;       // offsets in the workspace; what it takes
};
EmbeddingPlan embedding_plan(int T, int d, int V);
int launch_embedding_fwd(const void* table, const int32_t* tokens, moe_dtype dt, int T, int d, int V, float scale, void* out, hipStream_t s);
int launch_embedding_bwd(const int32_t* tokens, const void* dy, moe_dtype dt, int T, int d, int V, float scale, void* d_table, moe_dtype grad_dt,
                         int accumulate, const EmbeddingPlan& p, char* ws, hipStream_t s);

// ---- norms around a block --------------------------------------------------------------------
struct NormProblem {
  const void* x; const void* y;             // forward: stream and block output (or NULL); backward: x is the stream that h was made from
  const float* w_after; const float* gate; const float* w_before;
  moe_dtype dt;
  int T, d, gate_rows;                      // gate_rows tokens share a row of the gate
  float alpha, eps;
  void* out; void* h;                       // forward
  const void* d_out; const void* d_h;       // backward
  void* dx; void* dy;
  float* d_w_after; float* d_gate; float* d_w_before;
  int accumulate;
};
struct NormPlan { int teams, rows; size_t bytes; };      // teams of threads, each with so many rows one after another
NormPlan norm_bwd_plan(int T, int d, moe_dtype dt, bool after, bool gate, bool before);
int launch_norm_fwd(const NormProblem& q, hipStream_t s);
int launch_norm_bwd(const NormProblem& q, const NormPlan& p, float* ws, hipStream_t s);

}  // namespace moe
