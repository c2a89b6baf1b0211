// Orthogonalised updates of matrices with a side of at most 128: all steps on the Gram matrix alone, which fits one workgroup.
//   A = X X^T (S x S, X over its norm),  each step  R = b A + c A^2,  Q <- (a I + R) Q,  A <- (a I + R) A (a I + R),  in the end  O = Q X
// Where both sides are small the general way is a row of launches that each take longer to start than to run: here it is four (the norm, parts of A by slabs of
// the longer side, the steps, Q X), and X is read twice and never written.
//
// Numbers: A's eigenvalues are squares of singular values, so what a step rounds off is multiplied by a^2 = 12 in every later one, 20000 in five.  All matrices are
// therefore pairs of fp16, hi + 2^-11 lo (22 bits), and a product is hi hi + hi lo + lo hi, summed in fp32; Q is kept over the largest value that its polynomial
// can have.  Relative error of 64 x 2048 matrices with singular values falling as i^0, i^-0.5, i^-1.5: 1.4e-4, 3e-4, 1.8e-3.
//
// 64 x 2048: 38 us, of which the steps 21 (the general way 216); 16 of 256 x 128: 81, the steps 50 (191).
#include <math.h>

#include <atomic>

#include "newton_schulz_device.h"

namespace moe {
namespace {

using namespace orth;

struct SmallSteps { float a[MOE_ORTH_MAX_STEPS], b[MOE_ORTH_MAX_STEPS], c[MOE_ORTH_MAX_STEPS], unit[MOE_ORTH_MAX_STEPS]; int steps; };      // unit: one over the largest |a + R|

template <int SP> constexpr int threads_of() { return SP == 64 ? 256 : 512; }

// A matrix in LDS: hi, then lo, K-major rows of K elements
template <int ROWS, int K> struct Split {
  typedef KTile<ROWS, K> T;
  static constexpr int BYTES = 2 * T::BYTES;
  // four elements of a row
  __device__ static __forceinline__ void put(char* at, int row, int col, f32x4 v) {
    const f16x4 h = __builtin_convertvector(v, f16x4);
    char* to = at + T::offset(row, col >> 3) + (col & 7) * 2;
    *reinterpret_cast<f16x4*>(to) = h;
    *reinterpret_cast<f16x4*>(to + T::BYTES) = __builtin_convertvector((v - __builtin_convertvector(h, f32x4)) * kLow, f16x4);
  }
  // four elements of a column
  __device__ static __forceinline__ void put_turned(char* at, int row, int col, f32x4 v) {
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const half h = (half)v[c];
      char* to = at + T::offset(row + c, col >> 3) + (col & 7) * 2;
      *reinterpret_cast<half*>(to) = h;
      *reinterpret_cast<half*>(to + T::BYTES) = (half)((v[c] - (float)h) * kLow);
    }
  }
};

// sums += L R^T over K, of a wave's FM x FN parts from rows row0 and col0 on; `low`: those with one lo, to be taken times 2^-11
template <int LROWS, int RROWS, int K, int FM, int FN>
__device__ __forceinline__ void multiply(unsigned l, unsigned r, int row0, int col0, f32x4 (&sums)[FM][FN], f32x4 (&low)[FM][FN]) {
  const int lane = threadIdx.x & 63;
  const unsigned fl = l + mfma::frag_origin<mfma::KMAJOR, LROWS, K>(row0, lane), fr = r + mfma::frag_origin<mfma::KMAJOR, RROWS, K>(col0, lane);
  constexpr unsigned LB = KTile<LROWS, K>::BYTES, RB = KTile<RROWS, K>::BYTES;
#pragma unroll
  for (int kk = 0; kk < K / 32; ++kk) {
    f16x8 lh[FM], ll[FM], rh[FN], rl[FN];
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      lh[i] = __builtin_bit_cast(f16x8, mfma::read_frag_dma<mfma::KMAJOR, LROWS, K>(fl, i, kk));
      ll[i] = __builtin_bit_cast(f16x8, mfma::read_frag_dma<mfma::KMAJOR, LROWS, K>(fl + LB, i, kk));
    }
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      rh[j] = __builtin_bit_cast(f16x8, mfma::read_frag_dma<mfma::KMAJOR, RROWS, K>(fr, j, kk));
      rl[j] = __builtin_bit_cast(f16x8, mfma::read_frag_dma<mfma::KMAJOR, RROWS, K>(fr + RB, j, kk));
    }
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) {
        sums[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(rh[j], lh[i], sums[i][j], 0, 0, 0);
        low[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(rh[j], ll[i], low[i][j], 0, 0, 0);
        low[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(rl[j], lh[i], low[i][j], 0, 0, 0);
      }
  }
}
template <int FM, int FN> __device__ __forceinline__ void clear(f32x4 (&v)[FM][FN]) {
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) v[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
}

// 2^12 over the norm of the matrix
template <int THREADS> __device__ __forceinline__ double scale_of(const double* sums, int n, double* lds) {
  double s = 0;
  for (int i = threadIdx.x; i < n; i += THREADS) s += sums[i];
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) s += __shfl_xor(s, off);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
  __syncthreads();
  s = 0;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) s += lds[w];
  return s > 0 ? (double)kScale / sqrt(s) : s;
}

// A tile of X, 128 of the longer side, to LDS: [SP][128] (along the longer side) or [128][SP]; zeros outside.
template <typename TG, bool MUON, int SP, bool LONG_ROWS>
__device__ __forceinline__ void load_tile(const MuonProblem& q, long base, int tile, double scale, char* at) {
  const TG* g = static_cast<const TG*>(q.u) + base;
  const float* m = MUON ? q.m + base : nullptr;
  const float factor = MUON ? factor_of(q.factor) : 1.0f;
  const bool tall = q.rows > q.cols;
  const int r0 = tall ? tile * kSmallTile : 0, c0 = tall ? 0 : tile * kSmallTile, height = tall ? kSmallTile : SP, quads = (tall ? SP : kSmallTile) / 4;
  for (int unit = threadIdx.x; unit < height * quads; unit += threads_of<SP>()) {
    const int r = unit / quads, c = (unit - r * quads) * 4;
    f32x4 v = {};
    const int n = r0 + r < q.rows ? max(min(q.cols - c0 - c, 4), 0) : 0;
    if (n > 0) {
      const long o = (long)(r0 + r) * q.cols + c0 + c;
      v = load4(g + o, n);
      if constexpr (MUON) v = update_of(v, load4(m + o, n), factor, q.momentum, q.nesterov);
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = (float)((double)v[k] * scale);
    }
    if constexpr (LONG_ROWS) {                       // [SP][128]
      if (tall) Split<SP, kSmallTile>::put_turned(at, c, r, v);
      else Split<SP, kSmallTile>::put(at, r, c, v);
    } else {                                         // [128][SP]
      if (tall) Split<kSmallTile, SP>::put(at, r, c, v);
      else Split<kSmallTile, SP>::put_turned(at, c, r, v);
    }
  }
}

// parts[matrix][slab]: X X^T over a slab of the longer side, in units of 2^12
template <typename TG, bool MUON, int SP>
__global__ void __launch_bounds__(threads_of<SP>()) small_gram_kernel(MuonProblem q, OrthPlan p, int first, const double* __restrict__ sums, float* __restrict__ parts) {
  constexpr int FM = 2, FN = SP / 32;
  __shared__ __attribute__((aligned(256))) char tile[Split<SP, kSmallTile>::BYTES];
  const unsigned at = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)tile;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row0 = (wave >> 1) * 32, col0 = (wave & 1) * (SP / 2);
  const int which = blockIdx.y, long_side = q.rows > q.cols ? q.rows : q.cols;
  const long base = (first + (long)which) * q.rows * q.cols;
  const double scale = scale_of<threads_of<SP>()>(sums + (long)which * p.norm_blocks, p.norm_blocks, reinterpret_cast<double*>(tile));
  f32x4 acc[FM][FN], low[FM][FN];
  clear(acc);
  clear(low);
  const int t1 = min(((int)blockIdx.x + 1) * p.tiles_per_slab, (long_side + kSmallTile - 1) / kSmallTile);
  for (int t = blockIdx.x * p.tiles_per_slab; t < t1; ++t) {
    __syncthreads();
    load_tile<TG, MUON, SP, true>(q, base, t, scale, tile);
    __syncthreads();
    multiply<SP, SP, kSmallTile, FM, FN>(at, at, row0, col0, acc, low);
  }
  float* to = parts + ((long)which * gridDim.x + blockIdx.x) * SP * SP;
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j)
      *reinterpret_cast<f32x4*>(to + (row0 + i * 16 + (lane & 15)) * SP + col0 + j * 16 + (lane >> 4) * 4) = (acc[i][j] + low[i][j] * (1.0f / kLow)) * (1.0f / kScale);
}

// All steps of a matrix: Q, hi and lo
template <int SP>
__global__ void __launch_bounds__(threads_of<SP>(), 2) small_steps_kernel(SmallSteps c, int slabs, const float* __restrict__ parts, half* __restrict__ out) {
  constexpr int FM = 2, FN = SP / 32, BYTES = Split<SP, SP>::BYTES;
  extern __shared__ __attribute__((aligned(256))) char smem[];
  char* const buf0 = smem;
  char* const buf1 = smem + BYTES;
  const unsigned at0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)smem, at1 = at0 + BYTES;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row0 = (wave >> 1) * 32 + (lane & 15), col0 = (wave & 1) * (SP / 2) + (lane >> 4) * 4;
  f32x4 a[FM][FN], r[FM][FN], q[FM][FN];
  clear(a);
  for (int n = 0; n < slabs; ++n) {
    const float* from = parts + ((long)blockIdx.x * slabs + n) * SP * SP;
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) a[i][j] += *reinterpret_cast<const f32x4*>(from + (row0 + i * 16) * SP + col0 + j * 16);
  }
  auto put = [&](char* buf, const f32x4 (&v)[FM][FN]) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) Split<SP, SP>::put(buf, row0 + i * 16, col0 + j * 16, v[i][j]);
  };
  // v <- (e v + f L R) * unit, all in units of 2^12
  auto product = [&](unsigned l, unsigned rr, float e, float f, float unit, const f32x4 (&from)[FM][FN], f32x4 (&to)[FM][FN]) __attribute__((always_inline)) {
    f32x4 acc[FM][FN], low[FM][FN];
    clear(acc);
    clear(low);
    multiply<SP, SP, SP, FM, FN>(l, rr, (wave >> 1) * 32, (wave & 1) * (SP / 2), acc, low);
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) to[i][j] = (from[i][j] * e + (acc[i][j] + low[i][j] * (1.0f / kLow)) * (f / kScale)) * unit;
  };
  put(buf0, a);
  __syncthreads();
  for (int k = 0; k < c.steps; ++k) {
    const bool more = k + 1 < c.steps;
    product(at0, at0, c.b[k], c.c[k], 1.0f, a, r);
    put(buf1, r);
    __syncthreads();
    if (more) {
      f32x4 t[FM][FN];
      product(at1, at0, c.a[k], 1.0f, 1.0f, a, t);
      __syncthreads();
      put(buf0, t);
      __syncthreads();
      product(at1, at0, c.a[k], 1.0f, 1.0f, t, a);
      __syncthreads();
    }
    if (k == 0) {
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
          for (int n = 0; n < 4; ++n)
            q[i][j][n] = (r[i][j][n] + (row0 + i * 16 == col0 + j * 16 + n ? c.a[0] * kScale : 0.f)) * c.unit[0];
    } else {
      put(buf0, q);
      __syncthreads();
      product(at1, at0, c.a[k], 1.0f, c.unit[k], q, q);
      __syncthreads();
    }
    if (more) {
      put(buf0, a);
      __syncthreads();
    }
  }
  half* hi = out + (long)blockIdx.x * 2 * SP * SP;
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      const f16x4 h = __builtin_convertvector(q[i][j], f16x4);
      const int at = (row0 + i * 16) * SP + col0 + j * 16;
      *reinterpret_cast<f16x4*>(hi + at) = h;
      *reinterpret_cast<f16x4*>(hi + SP * SP + at) = __builtin_convertvector((q[i][j] - __builtin_convertvector(h, f32x4)) * kLow, f16x4);
    }
}

// O = Q X of 128 of the longer side
template <Result RES, typename TG, int SP>
__global__ void __launch_bounds__(threads_of<SP>(), 2) small_apply_kernel(MuonProblem mu, OrthPlan p, int first, const double* __restrict__ sums,
                                                                        const half* __restrict__ qs, float unit) {
  constexpr bool MUON = RES == MUON_UPDATE;
  constexpr int FM = 2, FN = 4;
  extern __shared__ __attribute__((aligned(256))) char smem[];
  char* const xs = smem + Split<SP, SP>::BYTES;
  const unsigned at_q = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)smem, at_x = at_q + Split<SP, SP>::BYTES;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, which = blockIdx.y;
  const long base = (first + (long)which) * mu.rows * mu.cols;
  const half* hi = qs + (long)which * 2 * SP * SP;
  for (int unit8 = threadIdx.x; unit8 < SP * SP / 8; unit8 += threads_of<SP>()) {
    const int row = unit8 / (SP / 8), chunk = unit8 % (SP / 8);
    char* to = smem + KTile<SP, SP>::offset(row, chunk);
    *reinterpret_cast<f16x8*>(to) = *reinterpret_cast<const f16x8*>(hi + row * SP + chunk * 8);
    *reinterpret_cast<f16x8*>(to + KTile<SP, SP>::BYTES) = *reinterpret_cast<const f16x8*>(hi + SP * SP + row * SP + chunk * 8);
  }
  const double scale = scale_of<threads_of<SP>()>(sums + (long)which * p.norm_blocks, p.norm_blocks, reinterpret_cast<double*>(xs));
  __syncthreads();
  load_tile<TG, MUON, SP, false>(mu, base, blockIdx.x, scale, xs);
  __syncthreads();
  f32x4 acc[FM][FN], low[FM][FN];
  clear(acc);
  clear(low);
  const bool tall = mu.rows > mu.cols;
  int row0, col0, r0, c0;                            // of the wave in the tile, of the tile in the matrix
  if (tall) {                                        // 128 rows of X, SP columns
    row0 = (SP == 64 ? wave : wave >> 1) * 32;
    col0 = SP == 64 ? 0 : (wave & 1) * 64;
    r0 = blockIdx.x * kSmallTile;
    c0 = 0;
    multiply<kSmallTile, SP, SP, FM, FN>(at_x, at_q, row0, col0, acc, low);
  } else {                                           // SP rows, 128 columns
    row0 = (wave >> 1) * 32;
    col0 = (wave & 1) * 64;
    r0 = 0;
    c0 = blockIdx.x * kSmallTile;
    multiply<SP, kSmallTile, SP, FM, FN>(at_q, at_x, row0, col0, acc, low);
  }
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      const int row = r0 + row0 + i * 16 + (lane & 15), col = c0 + col0 + j * 16 + (lane >> 4) * 4, n = min(mu.cols - col, 4);
      if (row < mu.rows && n > 0) {
        const long o = base + (long)row * mu.cols + col;
        f32x4 old = {};
        if constexpr (MUON) old = load4(mu.p + o, n);
        write_result<RES>(mu, o, n, (acc[i][j] + low[i][j] * (1.0f / kLow)) * (unit / (kScale * kScale)), old);
      }
    }
}

template <int SP> constexpr int steps_lds() { return 2 * Split<SP, SP>::BYTES; }
template <int SP> constexpr int apply_lds() { return Split<SP, SP>::BYTES + Split<kSmallTile, SP>::BYTES; }

template <Result RES, typename TG, int SP> int run(const MuonProblem& mu, const OrthPlan& p, int first, int count, char* ws, hipStream_t s) {
  const double* sums = reinterpret_cast<const double*>(ws + p.sums);
  float* parts = reinterpret_cast<float*>(ws + p.gram);
  half* q = reinterpret_cast<half*>(ws + p.t);
  SmallSteps c{};
  c.steps = mu.steps;
  const bool usual = orth_is_default(mu.coef, mu.steps);          // a + b l + c l^2 is largest at 0 then
  double top = 1.0, whole = 1.0;                     // largest singular value; largest value that Q's polynomial can have
  for (int k = 0; k < mu.steps; ++k) {
    const OrthCoef& o = mu.coef[k];
    double most = usual ? o.a : 1e-6, next = 0;
    for (int i = 0; !usual && i <= 128; ++i) {
      const double x = top * 1.01 * i / 128, v = fabs(o.a + (o.b + o.c * x * x) * x * x);
      most = fmax(most, v);
      next = fmax(next, v * x);
    }
    c.a[k] = (float)o.a;
    c.b[k] = (float)o.b;
    c.c[k] = (float)o.c;
    c.unit[k] = (float)(1.0 / most);
    whole *= most;
    top = next;
  }
  small_gram_kernel<TG, RES == MUON_UPDATE, SP><<<dim3(p.slabs, count), dim3(threads_of<SP>()), 0, s>>>(mu, p, first, sums, parts);
  MOE_LAUNCH_CHECK();
  small_steps_kernel<SP><<<dim3(count), dim3(threads_of<SP>()), steps_lds<SP>(), s>>>(c, p.slabs, parts, q);
  MOE_LAUNCH_CHECK();
  const int tiles = cdiv(mu.rows > mu.cols ? mu.rows : mu.cols, kSmallTile);
  small_apply_kernel<RES, TG, SP><<<dim3(tiles, count), dim3(threads_of<SP>()), apply_lds<SP>(), s>>>(mu, p, first, sums, q, (float)whole);
  MOE_LAUNCH_CHECK();
  return MOE_OK;
}

template <Result RES, typename TG> int sized(const MuonProblem& mu, const OrthPlan& p, int first, int count, char* ws, hipStream_t s) {
  return p.S == 64 ? run<RES, TG, 64>(mu, p, first, count, ws, s) : run<RES, TG, 128>(mu, p, first, count, ws, s);
}
template <Result RES> int typed(const MuonProblem& mu, const OrthPlan& p, int first, int count, char* ws, hipStream_t s) {
  return mu.u_dt == MOE_F32 ? sized<RES, float>(mu, p, first, count, ws, s) : sized<RES, bf16>(mu, p, first, count, ws, s);
}

}  // namespace

// (raised limits of dynamic LDS: see orth_configure)
int orth_small_configure() {
  for (const void* k : {(const void*)small_apply_kernel<MUON_UPDATE, float, 128>, (const void*)small_apply_kernel<MUON_UPDATE, bf16, 128>,
                        (const void*)small_apply_kernel<OUT_F32, float, 128>, (const void*)small_apply_kernel<OUT_F32, bf16, 128>,
                        (const void*)small_apply_kernel<OUT_BF16, float, 128>, (const void*)small_apply_kernel<OUT_BF16, bf16, 128>})
    MOE_HIP_TRY(hipFuncSetAttribute(k, hipFuncAttributeMaxDynamicSharedMemorySize, apply_lds<128>()));
  MOE_HIP_TRY(hipFuncSetAttribute((const void*)small_steps_kernel<128>, hipFuncAttributeMaxDynamicSharedMemorySize, steps_lds<128>()));
  return MOE_OK;
}

int launch_orth_small(const MuonProblem& mu, const OrthPlan& p, int first, int count, char* ws, hipStream_t s) {
  if (!mu.out) return typed<MUON_UPDATE>(mu, p, first, count, ws, s);
  return mu.out_dt == MOE_F32 ? typed<OUT_F32>(mu, p, first, count, ws, s) : typed<OUT_BF16>(mu, p, first, count, ws, s);
}

}  // namespace moe
