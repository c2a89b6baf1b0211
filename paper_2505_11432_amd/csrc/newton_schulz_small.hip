// Orthogonalised updates of matrices with a side of at most 64: all steps on the Gram matrix alone, which fits one workgroup.
//   A = X X^T (64 x 64, X over its norm or eps),  each step  R = b A + c A^2,  Q <- (a I + R) Q,  A <- (a I + R) A (a I + R),  in the end  O = Q X
// Where both sides are small the general way is a row of launches that each take longer to start than to run: here it is four (the norm, parts of A by slabs of
// the longer side, the steps, Q X), and X is read twice and never written.  64 x 2048 71 us (5 the norm, 10 the parts of A, 50 the steps, a chain of products on one
// CU, 9 Q X), 64 times 64 x 512 72, 16 times 32 x 4096 90; the general way 87, 116, 172, and 62 and 66 for a single 64 x 64.
//
// Numbers: A's eigenvalues are squares of singular values, so what a step rounds off is multiplied by a^2 = 12 in every later one, 20000 in five: in fp32 the
// outcome of steep spectra is off by 4e-3.  A and the steps are therefore in 64 bits, on the matrix cores (a product of 64 x 64 takes 1.7 us of a CU), and the
// outcome is off by 1e-6 (flat spectra, full rank) to 5e-6 (steep ones).  Q, over the
// largest value that its polynomial can have, and X are pairs of fp16 in the last product (hi + 2^-11 lo, 22 bits, summed in fp32).  No later step multiplies their
// roundings, but Q itself does: by 485 in directions that X does not have.  Of rank 8, 2 and 1 the outcome is off by 1.3e-5, 3e-5 and 7e-5.
#include <math.h>

#include <atomic>

#include "newton_schulz_device.h"

namespace moe {
namespace {

using namespace orth;

struct SmallSteps { double a[MOE_ORTH_MAX_STEPS], b[MOE_ORTH_MAX_STEPS], c[MOE_ORTH_MAX_STEPS], unit[MOE_ORTH_MAX_STEPS]; int steps; };      // unit: one over the largest |a + R|

constexpr int SP = 64, kThreads = 256;
typedef __attribute__((ext_vector_type(4))) double f64x4;

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

// of 2^12 over the norm of the matrix
__device__ __forceinline__ double scale_of(const double* sums, int n, double eps, double* lds) {
  double s = 0;
  for (int i = threadIdx.x; i < n; i += kThreads) s += sums[i];
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) s += __shfl_xor(s, off);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
  __syncthreads();
  s = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) s += lds[w];
  return scale_of_norm(s, eps);
}

// f(row, column, four elements) for a tile of X, 128 of the longer side and 64 of the other; zeros outside.
template <typename TG, bool MUON, typename F> __device__ __forceinline__ void for_tile(const MuonProblem& q, long base, int tile, double scale, F f) {
  const TG* g = static_cast<const TG*>(q.u) + base;
  const float* m = MUON ? q.m + base : nullptr;
  const float factor = MUON ? factor_of(q.factor) : 1.0f;
  const bool tall = q.rows > q.cols;
  const int r0 = tall ? tile * kSmallTile : 0, c0 = tall ? 0 : tile * kSmallTile, quads = (tall ? SP : kSmallTile) / 4;
#pragma unroll 4
  for (int unit = threadIdx.x; unit < SP * kSmallTile / 4; unit += kThreads) {
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
    f(r, c, v);
  }
}

// sums += L R^T of a wave's 32 x 16 M (2 x M of 16 x 16): the fp64 matrix instruction takes four of k at a time, lane l has row (column) l % 16 and k = l / 16, and
// of the sums column l % 16 and rows l / 16 + 4 i.
template <int K, int PITCH, int M, typename T> __device__ __forceinline__ void multiply64(const T* l, const T* r, f64x4 (&sums)[2][M]) {
  const int lane = threadIdx.x & 63, i = lane & 15, k0 = lane >> 4;
#pragma unroll 8
  for (int k = 0; k < K; k += 4) {
    double a[2], b[M];
#pragma unroll
    for (int n = 0; n < 2; ++n) a[n] = (double)l[(n * 16 + i) * PITCH + k + k0];
#pragma unroll
    for (int m = 0; m < M; ++m) b[m] = (double)r[(m * 16 + i) * PITCH + k + k0];
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int m = 0; m < M; ++m) sums[n][m] = __builtin_amdgcn_mfma_f64_16x16x4f64(a[n], b[m], sums[n][m], 0, 0, 0);
  }
}
// f(row, column, which of the sums) for a wave's sums; row0, col0: where they begin
template <int M, typename F> __device__ __forceinline__ void each64(int row0, int col0, F f) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int n = 0; n < 2; ++n)
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
      for (int i = 0; i < 4; ++i) f(row0 + n * 16 + (lane >> 4) + 4 * i, col0 + m * 16 + (lane & 15), n, m, i);
}

constexpr int kTilePitch = kSmallTile + 4, kGramPitch = SP + 2;      // (rows in different banks)

// parts[matrix][slab]: X X^T over a slab of the longer side
template <typename TG, bool MUON>
__global__ void __launch_bounds__(kThreads) small_gram_kernel(MuonProblem q, OrthPlan p, int first, const double* __restrict__ sums, double* __restrict__ parts) {
  __shared__ __attribute__((aligned(16))) float tile[SP * kTilePitch];
  __shared__ double lds[kThreads / 64];
  const int wave = threadIdx.x >> 6, row0 = (wave >> 1) * 32, col0 = (wave & 1) * 32;
  const int which = blockIdx.y, long_side = q.rows > q.cols ? q.rows : q.cols;
  const long base = (first + (long)which) * q.rows * q.cols;
  const double scale = scale_of(sums + (long)which * p.norm_blocks, p.norm_blocks, q.eps, lds);
  f64x4 acc[2][2] = {};
  const int t1 = min(((int)blockIdx.x + 1) * p.tiles_per_slab, (long_side + kSmallTile - 1) / kSmallTile);
  for (int t = blockIdx.x * p.tiles_per_slab; t < t1; ++t) {
    __syncthreads();
    const bool tall = q.rows > q.cols;
    for_tile<TG, MUON>(q, base, t, scale, [&](int r, int c, f32x4 v) __attribute__((always_inline)) {
#pragma unroll
      for (int k = 0; k < 4; ++k) tile[tall ? (c + k) * kTilePitch + r : r * kTilePitch + c + k] = v[k];
    });
    __syncthreads();
    multiply64<kSmallTile, kTilePitch, 2>(tile + row0 * kTilePitch, tile + col0 * kTilePitch, acc);
  }
  double* to = parts + ((long)which * gridDim.x + blockIdx.x) * SP * SP;
  each64<2>(row0, col0, [&](int r, int c, int n, int m, int i) __attribute__((always_inline)) { to[r * SP + c] = acc[n][m][i] * (1.0 / ((double)kScale * kScale)); });
}

// All steps of a matrix: Q, hi and lo, in units of 2^12.  Two matrices in LDS, the others in the registers of the threads that made them.
__global__ void __launch_bounds__(2 * kThreads) small_steps_kernel(SmallSteps c, int slabs, const double* __restrict__ parts, half* __restrict__ out) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  double* const buf0 = reinterpret_cast<double*>(smem);
  double* const buf1 = buf0 + SP * kGramPitch;
  const int wave = threadIdx.x >> 6, row0 = (wave >> 2) * 32, col0 = (wave & 3) * 16;
  f64x4 a[2][1] = {}, r[2][1], q[2][1];
  for (int s = 0; s < slabs; ++s) {
    const double* from = parts + ((long)blockIdx.x * slabs + s) * SP * SP;
    each64<1>(row0, col0, [&](int y, int x, int n, int m, int i) __attribute__((always_inline)) { a[n][m][i] += from[y * SP + x]; });
  }
  auto put = [&](double* buf, const f64x4 (&v)[2][1]) __attribute__((always_inline)) {
    each64<1>(row0, col0, [&](int y, int x, int n, int m, int i) __attribute__((always_inline)) { buf[y * kGramPitch + x] = v[n][m][i]; });
  };
  // to = (e from + f L R) unit of symmetric matrices
  auto product = [&](const double* l, const double* rr, double e, double f, double unit, const f64x4 (&from)[2][1], f64x4 (&to)[2][1]) __attribute__((always_inline)) {
    f64x4 acc[2][1] = {};
    multiply64<SP, kGramPitch, 1>(l + row0 * kGramPitch, rr + col0 * kGramPitch, acc);
#pragma unroll
    for (int n = 0; n < 2; ++n) to[n][0] = (from[n][0] * e + acc[n][0] * f) * unit;
  };
  put(buf0, a);
  __syncthreads();
  for (int k = 0; k < c.steps; ++k) {
    const bool more = k + 1 < c.steps;
    product(buf0, buf0, c.b[k], c.c[k], 1.0, a, r);
    put(buf1, r);
    __syncthreads();
    if (more) {
      f64x4 t[2][1];
      product(buf1, buf0, c.a[k], 1.0, 1.0, a, t);
      __syncthreads();
      put(buf0, t);
      __syncthreads();
      product(buf1, buf0, c.a[k], 1.0, 1.0, t, a);
      __syncthreads();
    }
    if (k == 0) {
      each64<1>(row0, col0, [&](int y, int x, int n, int m, int i) __attribute__((always_inline)) { q[n][m][i] = (r[n][m][i] + (y == x ? c.a[0] : 0.0)) * c.unit[0]; });
    } else {
      put(buf0, q);
      __syncthreads();
      product(buf1, buf0, c.a[k], 1.0, c.unit[k], q, q);
      __syncthreads();
    }
    if (more) {
      put(buf0, a);
      __syncthreads();
    }
  }
  half* hi = out + (long)blockIdx.x * 2 * SP * SP;
  each64<1>(row0, col0, [&](int y, int x, int n, int m, int i) __attribute__((always_inline)) {
    const double v = q[n][m][i] * (double)kScale;
    const half h = (half)(float)v;
    hi[y * SP + x] = h;
    hi[SP * SP + y * SP + x] = (half)(float)((v - (double)(float)h) * (double)kLow);
  });
}

// O = Q X of 128 of the longer side
template <Result RES, typename TG>
__global__ void __launch_bounds__(kThreads) small_apply_kernel(MuonProblem mu, OrthPlan p, int first, const double* __restrict__ sums, const half* __restrict__ qs, float unit) {
  constexpr bool MUON = RES == MUON_UPDATE;
  constexpr int FM = 2, FN = 4;
  __shared__ __attribute__((aligned(256))) char smem[Split<SP, SP>::BYTES + Split<kSmallTile, SP>::BYTES];
  char* const xs = smem + Split<SP, SP>::BYTES;
  const unsigned at_q = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)smem, at_x = at_q + Split<SP, SP>::BYTES;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, which = blockIdx.y;
  const long base = (first + (long)which) * mu.rows * mu.cols;
  const half* hi = qs + (long)which * 2 * SP * SP;
  for (int unit8 = threadIdx.x; unit8 < SP * SP / 8; unit8 += kThreads) {
    const int row = unit8 / (SP / 8), chunk = unit8 % (SP / 8);
    char* to = smem + KTile<SP, SP>::offset(row, chunk);
    *reinterpret_cast<f16x8*>(to) = *reinterpret_cast<const f16x8*>(hi + row * SP + chunk * 8);
    *reinterpret_cast<f16x8*>(to + KTile<SP, SP>::BYTES) = *reinterpret_cast<const f16x8*>(hi + SP * SP + row * SP + chunk * 8);
  }
  const bool tall = mu.rows > mu.cols;
  const double scale = scale_of(sums + (long)which * p.norm_blocks, p.norm_blocks, mu.eps, reinterpret_cast<double*>(xs));
  __syncthreads();
  for_tile<TG, MUON>(mu, base, blockIdx.x, scale, [&](int r, int c, f32x4 v) __attribute__((always_inline)) {
    if (tall) Split<kSmallTile, SP>::put(xs, r, c, v);
    else Split<kSmallTile, SP>::put_turned(xs, c, r, v);
  });
  __syncthreads();
  f32x4 acc[FM][FN], low[FM][FN];
  clear(acc);
  clear(low);
  int row0, col0, r0, c0;                            // of the wave in the tile, of the tile in the matrix
  if (tall) {                                        // 128 rows of X, 64 columns
    row0 = wave * 32;
    col0 = 0;
    r0 = blockIdx.x * kSmallTile;
    c0 = 0;
    multiply<kSmallTile, SP, SP, FM, FN>(at_x, at_q, row0, col0, acc, low);
  } else {                                           // 64 rows, 128 columns
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

constexpr int kStepsLds = 2 * SP * kGramPitch * 8;

template <Result RES, typename TG> int run(const MuonProblem& mu, const OrthPlan& p, int first, int count, char* ws, hipStream_t s) {
  const double* sums = reinterpret_cast<const double*>(ws + p.sums);
  double* parts = reinterpret_cast<double*>(ws + p.gram);
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
    c.a[k] = o.a;
    c.b[k] = o.b;
    c.c[k] = o.c;
    c.unit[k] = 1.0 / most;
    whole *= most;
    top = next;
  }
  small_gram_kernel<TG, RES == MUON_UPDATE><<<dim3(p.slabs, count), dim3(kThreads), 0, s>>>(mu, p, first, sums, parts);
  MOE_LAUNCH_CHECK();
  small_steps_kernel<<<dim3(count), dim3(2 * kThreads), kStepsLds, s>>>(c, p.slabs, parts, q);
  MOE_LAUNCH_CHECK();
  const int tiles = cdiv(mu.rows > mu.cols ? mu.rows : mu.cols, kSmallTile);
  small_apply_kernel<RES, TG><<<dim3(tiles, count), dim3(kThreads), 0, s>>>(mu, p, first, sums, q, (float)whole);
  MOE_LAUNCH_CHECK();
  return MOE_OK;
}

template <Result RES> int typed(const MuonProblem& mu, const OrthPlan& p, int first, int count, char* ws, hipStream_t s) {
  return mu.u_dt == MOE_F32 ? run<RES, float>(mu, p, first, count, ws, s) : run<RES, bf16>(mu, p, first, count, ws, s);
}

}  // namespace

// (a raised limit of dynamic LDS: see orth_configure)
int orth_small_configure() {
  MOE_HIP_TRY(hipFuncSetAttribute((const void*)small_steps_kernel, hipFuncAttributeMaxDynamicSharedMemorySize, kStepsLds));
  return MOE_OK;
}

int launch_orth_small(const MuonProblem& mu, const OrthPlan& p, int first, int count, char* ws, hipStream_t s) {
  if (!mu.out) return typed<MUON_UPDATE>(mu, p, first, count, ws, s);
  return mu.out_dt == MOE_F32 ? typed<OUT_F32>(mu, p, first, count, ws, s) : typed<OUT_BF16>(mu, p, first, count, ws, s);
}

}  // namespace moe
