// What the entry points (api_train.hip) and the kernels (vocab_loss.hip) of the vocabulary loss share.
#pragma once
#include "moe_common.h"

namespace moe {

struct VocabCounts { int n; float mean; };          // rows that count, 1 / n (0 without any)

// Layout of a workspace (offsets in bytes) and the choices that follow from sizes alone
struct VocabPlan {
  int R, pieces;                 // rows of a piece
  long ld;                       // elements of a row of G (whole 128-byte lines); fp32: of a row of a panel
  int panels;                    // fp32: panels of `ld` words, one after another ([panel][row][ld]); else 1
  bool gather;                   // the rows that count are gathered first
  bool twice;                    // d_w's contraction holds what the rounding of G left as further rows
  bool dw_sum_used;              // several pieces add up d_w in fp32 before it is rounded to bf16
  VocabTiles tiles;              // bf16: statistics per row
  struct Products { F32Plan z, dx, dw; };
  Products whole, last;          // fp32: parts of the products of a whole panel and of the last one
  size_t counts, ranges, token, target_of, xc, G, stats, z_target, weighted, rest, dxc, parts, dw_sum, bytes;
};
VocabPlan vocab_plan(int T, int d, int V, moe_dtype dt, moe_dtype grad_dt, int piece_rows, bool grad);

struct VocabProblem {
  const void* x; const void* w; const int32_t* target; const float* token_w;
  int T, d, V; moe_dtype dt;
  float* loss; float* lse;
  bool grad;
  float* total; void* dx; void* d_w; moe_dtype grad_dt; int accumulate;
};
int launch_vocab_loss(const VocabProblem& q, const VocabPlan& p, char* ws, hipStream_t s);

}  // namespace moe
