// What the kernels of orthogonalised updates share (newton_schulz.hip, newton_schulz_small.hip).
#pragma once
#include "gemm_mfma_dma.h"
#include "newton_schulz.h"

namespace moe {
namespace orth {

using mfma::KTile;
using mfma::dma16s;
using mfma::f32x4;
using mfma::uniform_ptr;
using mfma::wait_vmcnt;

typedef _Float16 half;
typedef __attribute__((ext_vector_type(4))) _Float16 f16x4;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef f32x4 f32x4_u __attribute__((aligned(4)));
typedef bf16x4 bf16x4_u __attribute__((aligned(2)));

constexpr float kScale = 4096.f;                        // what is kept is times 2^12
constexpr float kLow = 2048.f;                          // lo is times 2^11 more

// What a matrix is multiplied by: 2^12 over its norm, or over eps where that is larger.  (No number stays none, zeros stay zeros.)
__device__ __forceinline__ double scale_of_norm(double sum, double eps) { return sum > 0 ? (double)kScale / fmax(sqrt(sum), eps) : sum; }

__device__ __forceinline__ float factor_of(const float* f) { return f ? *f : 1.0f; }

// four elements, the last ones of a row one by one
template <typename T> __device__ __forceinline__ f32x4 load4(const T* p, int n) {
  f32x4 v = {};
  if (n >= 4) {
    if constexpr (sizeof(T) == 4) v = *reinterpret_cast<const f32x4_u*>(p);
    else v = __builtin_convertvector(*reinterpret_cast<const bf16x4_u*>(p), f32x4);
  } else {
#pragma unroll
    for (int i = 0; i < 3; ++i)
      if (i < n) v[i] = to_f32(p[i]);
  }
  return v;
}
template <typename T> __device__ __forceinline__ void store4(T* p, int n, f32x4 v) {
  if (n >= 4) {
    if constexpr (sizeof(T) == 4) *reinterpret_cast<f32x4_u*>(p) = v;
    else *reinterpret_cast<bf16x4_u*>(p) = __builtin_convertvector(v, bf16x4);
  } else {
#pragma unroll
    for (int i = 0; i < 3; ++i)
      if (i < n) p[i] = from_f32<T>(v[i]);
  }
}

__device__ __forceinline__ f32x4 momentum_of(f32x4 g, f32x4 m, float factor, float momentum) { return m * momentum + g * factor; }
__device__ __forceinline__ f32x4 update_of(f32x4 g, f32x4 m, float factor, float momentum, bool nesterov) { return nesterov ? g * factor + m * momentum : m; }

__device__ __forceinline__ double block_sum(double s, double* lds) {      // of 256 threads
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) s += __shfl_xor(s, off);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
  __syncthreads();
  return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

// Four elements of the outcome: new parameters and weights, or the orthogonalised matrix.  v: the result, of which n elements exist; old: the parameters.
enum Result { SYMMETRIC, KEPT, MUON_UPDATE, OUT_F32, OUT_BF16 };
template <Result RES> __device__ __forceinline__ void write_result(const MuonProblem& mu, long o, int n, f32x4 v, f32x4 old) {
  if constexpr (RES == MUON_UPDATE) {
    const float factor = factor_of(mu.factor), lr_now = *mu.lr;
    if (factor == factor) {
      const float keep = (float)(1.0 - (double)lr_now * mu.decay), step = lr_now * mu.scale;
      const f32x4 x = old * keep - v * step;
      store4(mu.p + o, n, x);
      if (mu.w) store4(static_cast<bf16*>(mu.w) + o, n, x);
    }
  } else if constexpr (RES == OUT_F32) {
    store4(static_cast<float*>(mu.out) + o, n, v);
  } else {
    store4(static_cast<bf16*>(mu.out) + o, n, v);
  }
}

}  // namespace orth
}  // namespace moe
