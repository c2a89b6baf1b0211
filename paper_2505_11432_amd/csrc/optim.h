// What the entry points (api_train.hip) and the kernels (optim.hip) of clipping and the update share.
#pragma once
#include "moe_common.h"

namespace moe {

// Tables of n + 1 entries; `first` counts the elements of the tensors before, `chunk` their chunks, and the last entry holds the sums alone.
constexpr int kChunkBytes = 2048, kAdamwChunk = 512;
struct ClipEntry { const void* g; void* out; int64_t first; int32_t dt, chunk; };
struct AdamwEntry { void* p; const void* g; void* m; void* v; void* w; int64_t first; };
// In a list of both types bit 0 of g, which an address of either has clear, says that its gradient is bf16.
constexpr uintptr_t kBf16Gradient = 1;
__host__ __device__ inline long chunk_elements(const ClipEntry& e) { return kChunkBytes / (e.dt == MOE_F32 ? 4 : 2); }
__host__ __device__ inline long chunk_elements(const AdamwEntry&) { return kAdamwChunk; }
// first chunk of entry i (AdamW, whose lists have one type: at least one chunk more than a tensor fills)
__host__ __device__ inline int first_chunk(const ClipEntry* table, int i) { return table[i].chunk; }
__host__ __device__ inline int first_chunk(const AdamwEntry* table, int i) { return (int)(table[i].first / kAdamwChunk) + 2 * i; }
struct AdamwHyper { double beta1, beta2, eps, weight_decay; };

constexpr int kNormParts = 2048;        // most workgroups of a launch: 64-bit sums of the norm

int launch_grad_clip(const ClipEntry* table, int n, long total, double max_norm, int write, float* norm, float* coef, double* parts, hipStream_t s);
int launch_adamw(const AdamwEntry* table, int n, long total, moe_dtype grad_dt, const float* lr, int32_t* step, const float* coef, const AdamwHyper& h,
                 unsigned* done, hipStream_t s);

}  // namespace moe
