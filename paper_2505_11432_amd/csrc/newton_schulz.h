// What the entry points (api_block.hip) and the kernels (newton_schulz.hip) of orthogonalised updates share.
#pragma once
#include "moe_common.h"

namespace moe {

constexpr int kOrthPad = 128;                // rows and columns of a matrix in the workspace are multiples of this
constexpr int kNormBlocks = 1024;             // sums of squares per matrix, at most
constexpr int kSmallSide = 64, kSmallTile = 128;
struct OrthCoef { double a, b, c; };
constexpr OrthCoef kDefaultCoef{3.4445, -4.7750, 2.0315};

struct MuonProblem {
  const void* u; moe_dtype u_dt;             // matrices to orthogonalise; Muon: their gradients
  int batch, rows, cols;
  OrthCoef coef[MOE_ORTH_MAX_STEPS]; int steps;
  void* out; moe_dtype out_dt;               // orthogonalised matrices, or NULL: Muon
  float* p; float* m; void* w;
  const float* lr; const float* factor;
  float momentum, scale; bool nesterov;
  double decay;
  double eps;                                // least norm that a matrix is divided by
};
struct OrthPlan {
  int R, C, S;                               // padded rows, columns, and the smaller of them
  int count;                                 // matrices at a time
  int norm_blocks;
  bool pairs;                                // steps taken two at a time
  bool small;                                // the smaller side within kSmallSide: see newton_schulz_small.hip
  int slabs, tiles_per_slab;                 // of the longer side there
  size_t hi, lo, t, other, gram, parts, sums;      // offsets of a piece's buffers
  size_t gram_one;                           // bytes of one list of Gram matrices
  size_t bytes;
};
bool orth_takes(int batch, int rows, int cols, int piece);
OrthPlan orth_plan(int batch, int rows, int cols, int piece);
int orth_configure();                        // per-device set-up (moe_init)
bool orth_is_default(const OrthCoef* c, int steps);
bool orth_coefficients_ok(const OrthCoef* c, int steps, int rows, int cols);      // every matrix that is kept fits 16 bits, and what it leaves out stays small
int orth_small_configure();
int launch_orth_small(const MuonProblem& q, const OrthPlan& p, int first, int count, char* ws, hipStream_t s);
int launch_orth(const MuonProblem& q, const OrthPlan& p, char* ws, hipStream_t s);

}  // namespace moe
