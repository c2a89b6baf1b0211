// What the entry points (api_train.hip) and the kernels (optim.hip) of clipping and the update share.
#pragma once
#include "moe_common.h"

namespace moe {

// Tables of n + 1 entries; `first` counts the elements of the tensors before, and the last entry holds the sum alone.
struct ClipEntry { const void* g; void* out; int64_t first; int32_t dt, reserved; };
struct AdamwEntry { void* p; const void* g; void* m; void* v; void* w; int64_t first; };
struct AdamwHyper { double beta1, beta2, eps, weight_decay; };

constexpr int kNormParts = 2048;        // most workgroups of a launch: 64-bit sums of the norm

int launch_grad_clip(const ClipEntry* table, int n, long total, double max_norm, int write, float* norm, float* coef, double* parts, hipStream_t s);
int launch_adamw(const AdamwEntry* table, int n, long total, moe_dtype grad_dt, const float* lr, int32_t* step, const float* coef, const AdamwHyper& h,
                 unsigned* done, hipStream_t s);

}  // namespace moe
