// Orthogonalised updates (Muon): u / |u| through Newton-Schulz steps, a batch of matrices at a time.
//   m = mu m + f g,  u = f g + mu m (or m),  X = u / |u|_F,  steps X <- (a I + b A + c A^2) X with A = X X^T,  p = p (1 - lr wd) - lr s X
// For matrices with more rows than columns A = X^T X, on the smaller side, and the steps multiply from the right.
// Bound by the matrix cores: a step multiplies m^2 (3 n + m) times per m x n matrix, m <= n, with A and R = b A + c A^2 symmetric and half of their tiles
// computed (the other half is mirrored).
//
// Numbers: operands are fp16, products are summed in fp32 (bf16 operands, eight bits instead of eleven, leave an error eight times as large).  What a step
// multiplies is bounded: the singular values of X by the steps' polynomials, so all entries of X, A and R lie within 2^4 (the entry points check that for the
// coefficients) and are kept times 2^12, where entries down to 1.5e-8 have all their bits.  A rounding of X enters directions of small singular values
// like a singular value of its own size and is multiplied by up to a = 3.4 in every later step, 485 in five.  X is therefore carried as two fp16, hi + 2^-11 lo
// (22 bits), a step adds R X, whose operand is hi, to a (hi + lo): what is left out, R lo, has no part in directions that A does not have.  Relative error
// (2-norm) of 512 x 1024 matrices with singular values falling as i^0, i^-0.5, i^-1, i^-1.5: 1.5e-3, 1.0e-3, 5e-4, 5e-4; with X in one fp16 1.2e-3,
// 2.4e-3, 4.9e-3, 1.2e-2, in bf16 eight times that.
//
// Every product reads both operands along the contraction (rows of 128 bytes per step of 64), so X is kept in both orientations: as it lies (hi, lo) and
// transposed (hi).  Matrices are padded with zeros to multiples of 128 in the workspace, which changes no value.
#include <math.h>

#include <atomic>

#include "gemm_mfma_dma.h"
#include "newton_schulz.h"

namespace moe {
namespace {

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

constexpr float kScale = 4096.f, kLimit = 15.5f;        // what is kept is times 2^12
constexpr float kLow = 2048.f;                          // lo is times 2^11 more

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

// New momentum, and sums of squares of u: gridDim.x parts of every matrix.
template <typename TG, bool MUON>
__global__ void __launch_bounds__(256) norm_kernel(MuonProblem q, int first, double* __restrict__ sums) {
  __shared__ double lds[4];
  const long size = (long)q.rows * q.cols, base = (first + (long)blockIdx.y) * size;
  const TG* g = static_cast<const TG*>(q.u) + base;
  float* m = MUON ? q.m + base : nullptr;
  const float factor = MUON ? factor_of(q.factor) : 1.0f;
  if (factor != factor) return;                         // (the update is left out)
  double s = 0;
  for (long i = ((long)blockIdx.x * 256 + threadIdx.x) * 4; i < size; i += (long)gridDim.x * 1024) {
    const int n = (int)min(size - i, 4L);
    f32x4 v = load4(g + i, n);
    if constexpr (MUON) {
      const f32x4 mv = momentum_of(v, load4(m + i, n), factor, q.momentum);
      store4(m + i, n, mv);
      v = update_of(v, mv, factor, q.momentum, q.nesterov);
    }
#pragma unroll
    for (int c = 0; c < 4; ++c) s = fma((double)v[c], (double)v[c], s);
  }
  s = block_sum(s, lds);
  if (threadIdx.x == 0) sums[(long)blockIdx.y * gridDim.x + blockIdx.x] = s;
}

// X = u / |u| in both orientations, 64 x 64 elements per workgroup; padding is zeros.
template <typename TG, bool MUON>
__global__ void __launch_bounds__(256) start_kernel(MuonProblem q, OrthPlan p, int first, const double* __restrict__ sums, half* __restrict__ hi,
                                                    half* __restrict__ lo, half* __restrict__ t) {
  __shared__ half tile[64][72];
  const long size = (long)q.rows * q.cols, base = (first + (long)blockIdx.z) * size, padded = (long)p.R * p.C * blockIdx.z;
  const TG* g = static_cast<const TG*>(q.u) + base;
  const float* m = MUON ? q.m + base : nullptr;
  const float factor = MUON ? factor_of(q.factor) : 1.0f;
  __shared__ double lds[4];
  double sum = 0;
  for (int i = threadIdx.x; i < p.norm_blocks; i += 256) sum += sums[(long)blockIdx.z * p.norm_blocks + i];
  sum = block_sum(sum, lds);
  const double scale = sum > 0 ? (double)kScale / sqrt(sum) : sum;      // (no number stays none)
  const int r0 = blockIdx.y * 64, c0 = blockIdx.x * 64;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int unit = threadIdx.x + i * 256, r = unit >> 4, c = (unit & 15) * 4;
    f32x4 v = {};
    const int n = r0 + r < q.rows ? max(min(q.cols - c0 - c, 4), 0) : 0;
    if (n > 0) {
      const long at = (long)(r0 + r) * q.cols + c0 + c;
      v = load4(g + at, n);
      if constexpr (MUON) v = update_of(v, load4(m + at, n), factor, q.momentum, q.nesterov);
    }
    f16x4 h, l;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float x = (float)((double)v[k] * scale);
      h[k] = (half)x;
      l[k] = (half)((x - (float)h[k]) * kLow);
    }
    const long to = padded + (long)(r0 + r) * p.C + c0 + c;
    *reinterpret_cast<f16x4*>(hi + to) = h;
    *reinterpret_cast<f16x4*>(lo + to) = l;
    *reinterpret_cast<f16x4*>(&tile[r][c]) = h;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int unit = threadIdx.x + i * 256, c = unit >> 3, r = (unit & 7) * 8;
    f16x8 v;
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = tile[r + k][c];
    *reinterpret_cast<f16x8*>(t + padded + (long)(c0 + c) * p.R + r0 + r) = v;
  }
}

// ---- products --------------------------------------------------------------------------------
// C = e1 E1 + e2 E2 + f L R^T, both operands [rows][K] of fp16; a list of matrices, `one` elements from each to the next.
struct Product {
  const half* l; const half* r; long l_one, r_one;
  int ldl, ldr, K;
  int tiles_m, tiles_n;                     // SYMMETRIC: tiles_m of both, the lower ones are computed
  const half* e1; const half* e2; float f1, f2, f;
  half* c; half* c_lo; half* ct; long c_one; int ldc, ldt;      // ct: the transposed result
};
enum Result { SYMMETRIC, KEPT, MUON_UPDATE, OUT_F32, OUT_BF16 };

constexpr int BM = 128, BN = 128, BK = 64, NW = 4;
typedef KTile<BM, BK> Tile;
constexpr int kStage = 2 * Tile::BYTES;
constexpr int kPitch = BM + 8;              // of the transposed tile in LDS, elements
static_assert(BN * kPitch * 2 <= 2 * kStage, "the transposed tile takes the place of the operands");

template <Result RES>
__global__ void __launch_bounds__(NW * 64, 2) product_kernel(Product q, MuonProblem mu, int first) {
  __shared__ __attribute__((aligned(256))) char smem[2 * kStage];
  const unsigned lds = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int wm = wave >> 1, wn = wave & 1;
  const int per = RES == SYMMETRIC ? q.tiles_m * (q.tiles_m + 1) / 2 : q.tiles_m * q.tiles_n;
  const int which = blockIdx.x / per;
  int at = blockIdx.x - which * per, mt, nt;
  if constexpr (RES == SYMMETRIC) {
    mt = (int)((sqrtf(8.f * (float)at + 1.f) - 1.f) * 0.5f);
    while ((mt + 1) * (mt + 2) / 2 <= at) ++mt;
    while (mt * (mt + 1) / 2 > at) --mt;
    nt = at - mt * (mt + 1) / 2;
  } else {
    mt = at / q.tiles_n;
    nt = at - mt * q.tiles_n;
  }
  const char* l = uniform_ptr(reinterpret_cast<const char*>(q.l + which * q.l_one + (long)mt * BM * q.ldl));
  const char* r = uniform_ptr(reinterpret_cast<const char*>(q.r + which * q.r_one + (long)nt * BN * q.ldr));
  // loads: 16 slots of 1 KB per operand tile, four per wave
  constexpr int SLOTS = Tile::BYTES / 1024 / NW;
  unsigned offl[SLOTS], offr[SLOTS];
#pragma unroll
  for (int j = 0; j < SLOTS; ++j) {
    const int row = (wave + j * NW) * Tile::ROWS_PER_DMA + lane / Tile::CPR, chunk = (lane % Tile::CPR) ^ Tile::swz(row);
    offl[j] = (unsigned)row * (unsigned)q.ldl * 2u + (unsigned)chunk * 16u;
    offr[j] = (unsigned)row * (unsigned)q.ldr * 2u + (unsigned)chunk * 16u;
  }
  auto issue = [&](int s) __attribute__((always_inline)) {
    const unsigned to = lds + (unsigned)(s & 1) * kStage + (unsigned)wave * 1024u;
#pragma unroll
    for (int j = 0; j < SLOTS; ++j) {
      dma16s(l + (long)s * BK * 2, offl[j], to + (unsigned)j * NW * 1024u);
      dma16s(r + (long)s * BK * 2, offr[j], to + Tile::BYTES + (unsigned)j * NW * 1024u);
    }
  };
  f32x4 acc[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int steps = q.K / BK;
  const unsigned fa = mfma::frag_origin<mfma::KMAJOR, BM, BK>(wm * 64, lane), fb = Tile::BYTES + mfma::frag_origin<mfma::KMAJOR, BN, BK>(wn * 64, lane);
  issue(0);
  for (int s = 0; s < steps; ++s) {
    wait_vmcnt<0>();
    __syncthreads();
    if (s + 1 < steps) issue(s + 1);
    const unsigned base = lds + (unsigned)(s & 1) * kStage;
#pragma unroll
    for (int kk = 0; kk < BK / 32; ++kk) {
      f16x8 a[4], b[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) a[i] = __builtin_bit_cast(f16x8, mfma::read_frag_dma<mfma::KMAJOR, BM, BK>(base + fa, i, kk));
#pragma unroll
      for (int j = 0; j < 4; ++j) b[j] = __builtin_bit_cast(f16x8, mfma::read_frag_dma<mfma::KMAJOR, BN, BK>(base + fb, j, kk));
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(b[j], a[i], acc[i][j], 0, 0, 0);
    }
  }
  __syncthreads();                          // the operands' LDS is free
  // a lane holds row lane % 16 and columns 4 (lane / 16) .. + 3 of every 16 x 16 part
  half* turned = reinterpret_cast<half*>(smem);
  const int row0 = mt * BM, col0 = nt * BN;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int lr = wm * 64 + i * 16 + (lane & 15), lc = wn * 64 + j * 16 + (lane >> 4) * 4;
      const long to = which * q.c_one + (long)(row0 + lr) * q.ldc + col0 + lc;
      f32x4 v = acc[i][j] * q.f;
      if (q.e1) v += __builtin_convertvector(*reinterpret_cast<const f16x4*>(q.e1 + to), f32x4) * q.f1;
      if (q.e2) v += __builtin_convertvector(*reinterpret_cast<const f16x4*>(q.e2 + to), f32x4) * q.f2;
      if constexpr (RES == SYMMETRIC || RES == KEPT) {
        const f16x4 h = __builtin_convertvector(v, f16x4);
        *reinterpret_cast<f16x4*>(q.c + to) = h;
        if constexpr (RES == KEPT) {
          const f16x4 low = __builtin_convertvector((v - __builtin_convertvector(h, f32x4)) * kLow, f16x4);
          *reinterpret_cast<f16x4*>(q.c_lo + to) = low;
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) turned[(lc + k) * kPitch + lr] = h[k];
      } else {
        const int row = row0 + lr, n = min(mu.cols - col0 - lc, 4);
        if (row < mu.rows && n > 0) {
          const long o = ((first + (long)which) * mu.rows + row) * mu.cols + col0 + lc;
          if constexpr (RES == MUON_UPDATE) {
            const float factor = factor_of(mu.factor), lr_now = *mu.lr;
            if (factor == factor) {
              const float keep = (float)(1.0 - (double)lr_now * mu.decay), step = lr_now * mu.scale * (1.0f / kScale);
              const f32x4 x = load4(mu.p + o, n) * keep - v * step;
              store4(mu.p + o, n, x);
              if (mu.w) store4(static_cast<bf16*>(mu.w) + o, n, x);
            }
          } else {
            v *= 1.0f / kScale;
            if constexpr (RES == OUT_F32) store4(static_cast<float*>(mu.out) + o, n, v);
            else store4(static_cast<bf16*>(mu.out) + o, n, v);
          }
        }
      }
    }
  if constexpr (RES == SYMMETRIC || RES == KEPT) {
    half* t = RES == SYMMETRIC ? q.c : q.ct;
    const int ldt = RES == SYMMETRIC ? q.ldc : q.ldt;
    if (RES == SYMMETRIC && mt == nt) return;          // (the tile holds both halves)
    __syncthreads();
#pragma unroll
    for (int i = 0; i < BM * BN / 8 / (NW * 64); ++i) {
      const int unit = threadIdx.x + i * NW * 64, c = unit / (BM / 8), x = unit % (BM / 8) * 8;
      *reinterpret_cast<f16x8*>(t + which * q.c_one + (long)(col0 + c) * ldt + row0 + x) = *reinterpret_cast<const f16x8*>(&turned[c * kPitch + x]);
    }
  }
}

template <Result RES> int product(const Product& q, const MuonProblem& mu, int first, int count, hipStream_t s) {
  const long per = RES == SYMMETRIC ? (long)q.tiles_m * (q.tiles_m + 1) / 2 : (long)q.tiles_m * q.tiles_n;
  product_kernel<RES><<<dim3((unsigned)(per * count)), dim3(NW * 64), 0, s>>>(q, mu, first);
  MOE_LAUNCH_CHECK();
  return MOE_OK;
}

// the products of the steps on `count` matrices from `first` on, whose X is in the workspace
int run_steps(const MuonProblem& mu, const OrthPlan& p, int first, int count, char* ws, hipStream_t s) {
  half* hi = reinterpret_cast<half*>(ws + p.hi);
  half* t = reinterpret_cast<half*>(ws + p.t);
  half* lo = reinterpret_cast<half*>(ws + p.lo);
  half* other = reinterpret_cast<half*>(ws + p.other);          // the next one of the orientation that a step reads
  half* gram[2] = {reinterpret_cast<half*>(ws + p.gram), reinterpret_cast<half*>(ws + p.gram + p.gram_one)};
  const bool tall = mu.rows > mu.cols;
  const long one = (long)p.R * p.C, gram_size = (long)p.S * p.S;
  for (int k = 0; k < mu.steps; ++k) {
    const OrthCoef c = mu.coef[k];
    Product a{};
    a.l = a.r = tall ? t : hi;
    a.l_one = a.r_one = one;
    a.ldl = a.ldr = a.K = tall ? p.R : p.C;
    a.tiles_m = a.tiles_n = p.S / BM;
    a.f = 1.0f / kScale;
    a.c = gram[0]; a.c_one = gram_size; a.ldc = p.S;
    if (const int rc = product<SYMMETRIC>(a, mu, first, count, s)) return rc;
    Product b = a;
    b.l = b.r = gram[0];
    b.l_one = b.r_one = gram_size;
    b.ldl = b.ldr = b.K = p.S;
    b.e1 = gram[0]; b.f1 = (float)c.b;
    b.f = (float)c.c / kScale;
    b.c = gram[1];
    if (const int rc = product<SYMMETRIC>(b, mu, first, count, s)) return rc;
    Product x{};
    x.l = tall ? hi : gram[1];
    x.l_one = tall ? one : gram_size;
    x.r = tall ? gram[1] : t;
    x.r_one = tall ? gram_size : one;
    x.ldl = x.ldr = x.K = p.S;
    x.tiles_m = p.R / BM; x.tiles_n = p.C / BN;
    x.e1 = hi; x.f1 = (float)c.a;
    x.e2 = lo; x.f2 = (float)c.a / kLow;
    x.f = 1.0f / kScale;
    x.c_one = one; x.ldc = p.C; x.ldt = p.R;
    if (k + 1 < mu.steps) {
      x.c = tall ? other : hi;
      x.c_lo = lo;
      x.ct = tall ? t : other;
      if (const int rc = product<KEPT>(x, mu, first, count, s)) return rc;
      half*& read = tall ? hi : t;
      half* was = read;
      read = other;
      other = was;
    } else {
      const int rc = !mu.out ? product<MUON_UPDATE>(x, mu, first, count, s)
                             : mu.out_dt == MOE_F32 ? product<OUT_F32>(x, mu, first, count, s) : product<OUT_BF16>(x, mu, first, count, s);
      if (rc) return rc;
    }
  }
  return MOE_OK;
}

template <typename TG, bool MUON> int start(const MuonProblem& mu, const OrthPlan& p, int first, int count, char* ws, hipStream_t s) {
  double* sums = reinterpret_cast<double*>(ws + p.sums);
  norm_kernel<TG, MUON><<<dim3(p.norm_blocks, count), dim3(256), 0, s>>>(mu, first, sums);
  MOE_LAUNCH_CHECK();
  start_kernel<TG, MUON><<<dim3(p.C / 64, p.R / 64, count), dim3(256), 0, s>>>(mu, p, first, sums, reinterpret_cast<half*>(ws + p.hi),
                                                                              reinterpret_cast<half*>(ws + p.lo), reinterpret_cast<half*>(ws + p.t));
  MOE_LAUNCH_CHECK();
  return MOE_OK;
}

}  // namespace

// matrices at a time: a launch has at most 65535 of them along a side of its grid
int matrices_at_a_time(int batch, int piece) {
  const int most = 32768, n = piece > 0 && piece < batch ? piece : batch;
  return n < most ? n : most;
}

// (a launch holds less than 2^32 threads, and the tiles of a piece are counted in 31 bits)
bool orth_takes(int batch, int rows, int cols, int piece) {
  if (rows > MOE_ORTH_MAX_SIDE || cols > MOE_ORTH_MAX_SIDE) return false;
  const long R = (long)align_up(rows, kOrthPad), C = (long)align_up(cols, kOrthPad), S = R < C ? R : C;
  const long tiles = (R / 64) * (C / 64) > (S / 64) * (S / 64) ? (R / 64) * (C / 64) : (S / 64) * (S / 64);
  return tiles * matrices_at_a_time(batch, piece) < 1L << 24 && C / 64 < 65536 && R / 64 < 65536;
}

OrthPlan orth_plan(int batch, int rows, int cols, int piece) {
  OrthPlan p{};
  const int count = matrices_at_a_time(batch, piece) < 1 ? 1 : matrices_at_a_time(batch, piece);
  p.count = count;
  p.R = (int)align_up(rows, kOrthPad);
  p.C = (int)align_up(cols, kOrthPad);
  p.S = p.R < p.C ? p.R : p.C;
  const long size = (long)rows * cols;
  long blocks = (size + 4095) / 4096;
  const long share = 4096 / count + 1;
  if (blocks > share) blocks = share;
  p.norm_blocks = (int)(blocks < kNormBlocks ? blocks : kNormBlocks);
  const size_t x = (size_t)count * p.R * p.C * 2;
  p.gram_one = (size_t)count * p.S * p.S * 2;
  p.hi = 0;
  p.lo = x;
  p.t = 2 * x;
  p.other = 3 * x;
  p.gram = 4 * x;
  p.sums = p.gram + 2 * p.gram_one;
  p.bytes = p.sums + (size_t)count * p.norm_blocks * 8 + 256;
  return p;
}

bool orth_coefficients_ok(const OrthCoef* c, int steps) {
  // singular values from 0 to `top` go to the polynomial's values there; what is kept on the way are values of polynomials in them
  double top = 1.0;
  for (int k = 0; k < steps; ++k) {
    double next = 0;
    if (!(fabs(c[k].a) <= 1e3 && fabs(c[k].b) <= 1e3 && fabs(c[k].c) <= 1e3)) return false;
    for (int i = 0; i <= 4096; ++i) {
      const double x = top * 1.01 * i / 4096, l = x * x, r = c[k].b * l + c[k].c * l * l, v = fabs(x * (c[k].a + r));
      if (l > kLimit || fabs(r) > kLimit || v > kLimit) return false;
      if (v > next) next = v;
    }
    top = next;
  }
  return true;
}

int launch_orth(const MuonProblem& mu, const OrthPlan& p, char* ws, hipStream_t s) {
  for (int first = 0; first < mu.batch; first += p.count) {
    const int count = mu.batch - first < p.count ? mu.batch - first : p.count;
    int rc;
    if (mu.out) rc = mu.u_dt == MOE_F32 ? start<float, false>(mu, p, first, count, ws, s) : start<bf16, false>(mu, p, first, count, ws, s);
    else rc = mu.u_dt == MOE_F32 ? start<float, true>(mu, p, first, count, ws, s) : start<bf16, true>(mu, p, first, count, ws, s);
    if (rc != MOE_OK) return rc;
    if (const int rc2 = run_steps(mu, p, first, count, ws, s)) return rc2;
  }
  return MOE_OK;
}

}  // namespace moe
