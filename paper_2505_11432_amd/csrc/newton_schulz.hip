// Orthogonalised updates (Muon): u / |u| through Newton-Schulz steps, a batch of matrices at a time.
//   m = mu m + f g,  u = f g + mu m (or m),  X = u / max(|u|_F, eps),  steps X <- (a I + b A + c A^2) X with A = X X^T,  p = p (1 - lr wd) - lr s X
// For matrices with more rows than columns A = X^T X, on the smaller side, and the steps multiply from the right.
// Bound by the matrix cores: a step multiplies m^2 (3 n + m) times per m x n matrix, m <= n, with A and R = b A + c A^2 symmetric and half of their tiles
// computed (the other half is mirrored).
//
// Numbers: operands are fp16, products are summed in fp32 (bf16 operands, eight bits instead of eleven, leave an error eight times as large).  What a step
// multiplies is bounded: the singular values of X by the steps' polynomials, so all entries of X, A and R lie within 2^4 (the entry points check that for the
// coefficients) and are kept times 2^12, where entries down to 1.5e-8 have all their bits.  A rounding of X enters directions of small singular values
// like a singular value of its own size and is multiplied by up to a = 3.4 in every later step, 485 in five.  X is therefore carried as two fp16, hi + 2^-11 lo
// (22 bits), a step adds R X, whose operand is hi, to a (hi + lo): what is left out, R lo, has no part in directions that A does not have.  Relative error
// (2-norm) of matrices with singular values flat, falling as i^-0.5, as i^-1.5, and 64 of 512: 6e-4, 6e-4, 9e-4, 1.7e-3 measured (of rank 1 1.9e-3, of small full ones,
// 65 x 512, 1.2e-3); 9e-4, 8e-4, 1.1e-3, 2.3e-3 by a model of these roundings in 64 bits, which gives 2.6e-3, 3.2e-3, 1.6e-2, 3.0e-2 for X in one fp16 and
// 2.1e-2, 2.6e-2, 0.13, 0.24 for bf16 throughout.
//
// Every product reads both operands along the contraction (rows of 128 bytes per step of 64), so X is kept in both orientations: as it lies (hi, lo) and
// transposed (hi).  Matrices are padded with zeros to multiples of 128 in the workspace, which changes no value.
#include <math.h>

#include <algorithm>
#include <atomic>

#include "newton_schulz_device.h"
#include "orth_tiles.h"

namespace moe {
namespace {

using namespace orth;

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
  const double scale = scale_of_norm(sum, q.eps);
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
// C = e1 E1 + e2 E2 + f L R^T + diagonal I, both operands [rows][K] of fp16; a list of matrices, `one` elements from each to the next.
struct Product {
  const half* l; const half* r; long l_one, r_one;
  int ldl, ldr, K;
  int M, N;                                 // multiples of 128; SYMMETRIC: M of both
  const half* e1; const half* e2; float f1, f2, f, diagonal;
  half* c; half* c_lo; half* ct; long c_one; int ldc, ldt;      // c_lo: what c leaves of the result; ct: the transposed result
  int full, split, items;                   // the tiles from `full` on are cut into `split` parts along K, which go to
  float* parts;
};

// Tiles of 256 x 256 by eight waves, 128 x 64 each, one workgroup per CU that walks a list of tiles.  Operands go from memory to an LDS ring of two steps of
// 64 directly; the lower four waves, one per SIMD, issue the loads while the others multiply.  The loads of a tile's first step are issued before the results
// of the tile in front are stored.  Two 4096 x 14336: the Gram matrices 411 us, 1.24 PFLOP/s of the tiles computed, R X with X rewritten 936 us, 1.03 PFLOP/s, matrix
// cores 50 % busy at 1.96 GHz; of 64 times 2048 x 1408 789 us, 0.66 PFLOP/s: 22 steps of some 1.1 us and 40 us of results, 0.75 MB of memory per tile, which all CUs
// move at once (half of the CUs begun half a tile later: 2 % slower).  128 x 256 by two workgroups per CU took 8.2 ms for that update, this 6.75.
constexpr int BM = 256, BN = 256, BK = 64, NW = 8, LOADERS = 4;
constexpr int WTM = 128, WTN = 64, FM = WTM / 16, FN = WTN / 16, TM = WTM / 32, TN = WTN / 32;
typedef KTile<BM, BK> Tile;
constexpr int kStage = 2 * Tile::BYTES;
constexpr int kRing = 2 * kStage;
constexpr int kProductLds = kRing + NW * mfma::STG_BYTES;
static_assert(kProductLds <= 160 * 1024, "LDS of a CU");
constexpr int kPartFloats = BM * BN;
static_assert(kPartFloats == kOrthPartFloats && BM == kOrthTile && BK == kOrthStep, "what the choice of tiles goes by");

// A wave's rows and columns in the tile.  Waves w and w + 4 share a SIMD: they lie in opposite halves along both sides, so that of a tile that is half
// outside each SIMD has one wave to multiply for (the others skip their products).
__device__ __forceinline__ int wave_row(int wave) { return (wave >> 2) * WTM; }
__device__ __forceinline__ int wave_col(int wave) { return ((wave & 3) ^ (wave >> 2) * 2) * WTN; }

// Which tile: matrix, row and column.  Squares of the lower triangle (SYMMETRIC), or bands of four rows of tiles, column by column.
struct Place { int which, mt, nt; };
template <Result RES> __host__ __device__ __forceinline__ int tiles_of(const Product& q) {
  const int tm = (q.M + BM - 1) / BM, tn = (q.N + BN - 1) / BN;
  return RES == SYMMETRIC ? tm * (tm + 1) / 2 : tm * tn;
}
template <Result RES> __device__ __forceinline__ Place place_of(const Product& q, int item) {
  const int per = tiles_of<RES>(q), which = item / per;
  int at = item - which * per;
  if constexpr (RES == SYMMETRIC) {
    int p = (int)((sqrtf(8.f * (float)at + 1.f) - 1.f) * 0.5f);
    while ((p + 1) * (p + 2) / 2 <= at) ++p;
    while (p * (p + 1) / 2 > at) --p;
    p = __builtin_amdgcn_readfirstlane(p);
    return {which, p, at - p * (p + 1) / 2};
  } else {
    const int tm = (q.M + BM - 1) / BM, tn = (q.N + BN - 1) / BN, band = at / (4 * tn), rows = min(4, tm - band * 4);
    at -= band * 4 * tn;
    return {which, band * 4 + at % rows, at / rows};
  }
}

// Blocks of 32 x 32 fp16 in memory: the block's place is the same for the wave and goes into a buffer descriptor, a lane has 8 columns of rows l / 4 and
// 16 + l / 4, at an offset that is the same in every block.
__device__ __forceinline__ int lane_offset(int ld, int lane) { return ((lane >> 2) * ld + (lane & 3) * 8) * 2; }
struct Fetch { mfma::u32x4v v[2]; };
__device__ __forceinline__ Fetch fetch_block(const half* g, int ld, int off) {
  const __amdgpu_buffer_rsrc_t rs = mfma::block_rsrc(g);
  Fetch f;
#pragma unroll
  for (int pass = 0; pass < 2; ++pass) f.v[pass] = __builtin_amdgcn_raw_buffer_load_b128(rs, off, pass * 32 * ld, 0);
  return f;
}
// to the lanes that hold the sums: group q of a lane is row 16 (q / 2) + lane % 16, columns 16 (q % 2) + 4 (lane / 16) .. + 3
__device__ __forceinline__ void unpack_block(char* stg, const Fetch& f, f16x4 (&v)[4], int lane) {
#pragma unroll
  for (int pass = 0; pass < 2; ++pass)
    *reinterpret_cast<mfma::u32x4v*>(stg + (pass * 16 + (lane >> 2)) * mfma::STG_STRIDE + (lane & 3) * 16) = f.v[pass];
#pragma unroll
  for (int q = 0; q < 4; ++q) v[q] = *reinterpret_cast<const f16x4*>(stg + mfma::patch_row(q, lane) * mfma::STG_STRIDE + mfma::patch_col(q, lane) * 2);
}
// (The offset of the second half is added to the lane's.  With it in the store's scalar offset the compiler puts no wait state between the store and a write of
// its data registers, and the last of a lane's four words has been stored as what was written behind it.)
__device__ __forceinline__ void store_patch(const char* stg, half* g, int ld, int off, int lane) {
  const __amdgpu_buffer_rsrc_t rs = mfma::block_rsrc(g);
#pragma unroll
  for (int pass = 0; pass < 2; ++pass)
    __builtin_amdgcn_raw_buffer_store_b128(*reinterpret_cast<const mfma::u32x4v*>(stg + (pass * 16 + (lane >> 2)) * mfma::STG_STRIDE + (lane & 3) * 16), rs,
                                           off + pass * 32 * ld, 0, 0);
}
__device__ __forceinline__ void store_block(char* stg, const f16x4 (&v)[4], half* g, int ld, int off, int lane) {
#pragma unroll
  for (int q = 0; q < 4; ++q) *reinterpret_cast<f16x4*>(stg + mfma::patch_row(q, lane) * mfma::STG_STRIDE + mfma::patch_col(q, lane) * 2) = v[q];
  store_patch(stg, g, ld, off, lane);
}
__device__ __forceinline__ void store_turned(char* stg, const f16x4 (&v)[4], half* g, int ld, int off, int lane) {
#pragma unroll
  for (int q = 0; q < 4; ++q)
#pragma unroll
    for (int c = 0; c < 4; ++c)
      *reinterpret_cast<half*>(stg + (mfma::patch_col(q, lane) + c) * mfma::STG_STRIDE + mfma::patch_row(q, lane) * 2) = v[q][c];
  store_patch(stg, g, ld, off, lane);
}

// The results of TI x TJ blocks of 32 x 32 of a wave, which begin at row0 and col0 of matrix `which`; mirrored: the transposed ones as well (SYMMETRIC, off the
// diagonal tiles, which hold both halves).
template <Result RES, int TI, int TJ>
__device__ __forceinline__ void finish(const Product& q, const MuonProblem& mu, int first, int which, int row0, int col0, bool mirrored, const f32x4 (&acc)[2 * TI][2 * TJ], char* stg) {
  const int lane = threadIdx.x & 63;
  constexpr int NB = TI * TJ;
  auto origin = [&](int b) __attribute__((always_inline)) -> long {
    return which * q.c_one + (long)(row0 + b / TJ * 32) * q.ldc + col0 + b % TJ * 32;
  };
  // What is read lies AHEAD blocks ahead of what is stored: a block takes a fraction of the time that a read does.
  constexpr int AHEAD = NB < 2 ? NB : 2;
  const int off = lane_offset(q.ldc, lane), off_t = lane_offset(q.ldt, lane);
  Fetch f1[AHEAD], f2[AHEAD];
  f32x4 old[4];
  auto ask = [&](int b) __attribute__((always_inline)) {
    if (q.e1) f1[b % AHEAD] = fetch_block(q.e1 + origin(b), q.ldc, off);
    if (q.e2) f2[b % AHEAD] = fetch_block(q.e2 + origin(b), q.ldc, off);
  };
  auto place = [&](int b, int n4, int& n) __attribute__((always_inline)) -> long {      // four elements of the result: where, and how many there are
    const int row = row0 + b / TJ * 32 + mfma::patch_row(n4, lane), col = col0 + b % TJ * 32 + mfma::patch_col(n4, lane);
    n = row < mu.rows ? min(mu.cols - col, 4) : 0;
    return ((first + (long)which) * mu.rows + row) * mu.cols + col;
  };
  auto ask_old = [&](int b) __attribute__((always_inline)) {
    if constexpr (RES == MUON_UPDATE) {
#pragma unroll
      for (int n4 = 0; n4 < 4; ++n4) {
        int n;
        const long o = place(b, n4, n);
        old[n4] = n > 0 ? load4(mu.p + o, n) : f32x4{};
      }
    }
  };
#pragma unroll
  for (int b = 0; b < AHEAD; ++b) ask(b);
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    const int i = b / TJ, j = b % TJ;
    ask_old(b);
    f32x4 v[4] = {acc[2 * i][2 * j] * q.f, acc[2 * i][2 * j + 1] * q.f, acc[2 * i + 1][2 * j] * q.f, acc[2 * i + 1][2 * j + 1] * q.f};
    f16x4 h[4];
    if (q.e1) {
      unpack_block(stg, f1[b % AHEAD], h, lane);
#pragma unroll
      for (int n = 0; n < 4; ++n) v[n] += __builtin_convertvector(h[n], f32x4) * q.f1;
    }
    if (q.e2) {
      unpack_block(stg, f2[b % AHEAD], h, lane);
#pragma unroll
      for (int n = 0; n < 4; ++n) v[n] += __builtin_convertvector(h[n], f32x4) * q.f2;
    }
    if (b + AHEAD < NB) ask(b + AHEAD);
    const int br = row0 + i * 32, bc = col0 + j * 32;
    if constexpr (RES == SYMMETRIC) {
      if (br == bc && q.diagonal != 0.f) {
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
          for (int c = 0; c < 4; ++c) v[n][c] += mfma::patch_row(n, lane) == mfma::patch_col(n, lane) + c ? q.diagonal : 0.f;
      }
    }
    if constexpr (RES == SYMMETRIC || RES == KEPT) {
      const long o = which * q.c_one;
#pragma unroll
      for (int n = 0; n < 4; ++n) h[n] = __builtin_convertvector(v[n], f16x4);
      store_block(stg, h, q.c + origin(b), q.ldc, off, lane);
      if (RES == KEPT) store_turned(stg, h, q.ct + o + (long)bc * q.ldt + br, q.ldt, off_t, lane);
      else if (mirrored) store_turned(stg, h, q.c + o + (long)bc * q.ldc + br, q.ldc, off, lane);
      if constexpr (RES == KEPT) {
#pragma unroll
        for (int n = 0; n < 4; ++n) h[n] = __builtin_convertvector((v[n] - __builtin_convertvector(h[n], f32x4)) * kLow, f16x4);
        store_block(stg, h, q.c_lo + origin(b), q.ldc, off, lane);
      }
    } else {
#pragma unroll
      for (int n4 = 0; n4 < 4; ++n4) {
        int n;
        const long o = place(b, n4, n);
        if (n > 0) write_result<RES>(mu, o, n, v[n4] * (1.0f / kScale), old[n4]);
      }
    }
  }
}

template <Result RES>
__global__ void __launch_bounds__(NW * 64, 2) product_kernel(Product q, MuonProblem mu, int first) {
  extern __shared__ __attribute__((aligned(256))) char smem[];
  const unsigned lds = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const bool is_loader = wave < LOADERS;
  char* stg = smem + kRing + wave * mfma::STG_BYTES;
  const unsigned fa = mfma::frag_origin<mfma::KMAJOR, BM, BK>(wave_row(wave), lane), fb = Tile::BYTES + mfma::frag_origin<mfma::KMAJOR, BN, BK>(wave_col(wave), lane);
  // a tile, or a part of one
  Place at{};
  int part = -1, steps = 0;
  const char* l = nullptr;
  const char* r = nullptr;
  unsigned offl[8], offr[8];
  auto open_tile = [&](int slot) __attribute__((always_inline)) -> bool {
    // Workgroup b runs on XCD b % 8: neighbouring tiles, which share operands, go to the CUs of one XCD.
    const int round = slot * kGroups, size = min(kGroups, q.items - round), share = size / 8, b = blockIdx.x;
    if (b >= size) return false;
    int item = round + (b < share * 8 ? b % 8 * share + b / 8 : b);
    part = -1;
    int step0 = 0;
    steps = q.K / BK;
    if (item >= q.full) {
      part = item - q.full;
      item = q.full + part / q.split;
      const int n = part % q.split, all = steps;
      step0 = n * all / q.split;
      steps = (n + 1) * all / q.split - step0;
    }
    at = place_of<RES>(q, item);
    l = uniform_ptr(reinterpret_cast<const char*>(q.l + at.which * q.l_one + (long)at.mt * BM * q.ldl + (long)step0 * BK));
    r = uniform_ptr(reinterpret_cast<const char*>(q.r + at.which * q.r_one + (long)at.nt * BN * q.ldr + (long)step0 * BK));
    if (is_loader) {
      // slot j of a loader: 1 KB, eight rows of the tile; rows past the last one repeat it
      const int left_l = q.M - at.mt * BM - 1, left_r = (RES == SYMMETRIC ? q.M : q.N) - at.nt * BN - 1;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int row = (wave + j * LOADERS) * Tile::ROWS_PER_DMA + lane / Tile::CPR, chunk = (lane % Tile::CPR) ^ Tile::swz(row);
        offl[j] = (unsigned)min(row, left_l) * (unsigned)q.ldl * 2u + (unsigned)chunk * 16u;
        offr[j] = (unsigned)min(row, left_r) * (unsigned)q.ldr * 2u + (unsigned)chunk * 16u;
      }
    }
    return true;
  };
  static_assert(Tile::BYTES / 1024 / LOADERS == 8 && Tile::BYTES == 0x8000, "sixteen loads per loader and step, an operand after the other");
  auto issue = [&](int s) __attribute__((always_inline)) {
    if (is_loader) mfma::dma16s_x16(l + (long)s * BK * 2, r + (long)s * BK * 2, offl, offr, lds + (unsigned)(s & 1) * kStage + (unsigned)wave * 1024u);
  };
  int slot = 0;
  if (!open_tile(slot)) return;
  issue(0);
  for (;;) {
    f32x4 acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    // A step has four phases, two for each half of its 64: the wave's right fragments are held for two, the left ones pass through four at a time, and the
    // fragments of each phase are read while the one before multiplies.  The barrier that opens step s + 1, whose loads have landed then, lies before the
    // last phase of step s, whose fragments are in registers: the slot of s is free for the loads of s + 2.
    f16x8 held[2][FN], strm[2][FM / 2];
    auto read_phase = [&](unsigned base, int p) __attribute__((always_inline)) {
      const int kk = p >> 1, ph = p & 1;
      if (ph == 0) {
#pragma unroll
        for (int j = 0; j < FN; ++j) held[kk][j] = __builtin_bit_cast(f16x8, mfma::read_frag_dma<mfma::KMAJOR, BN, BK>(base + fb, j, kk));
      }
#pragma unroll
      for (int i = 0; i < FM / 2; ++i) strm[p & 1][i] = __builtin_bit_cast(f16x8, mfma::read_frag_dma<mfma::KMAJOR, BM, BK>(base + fa, ph * (FM / 2) + i, kk));
    };
    auto open_step = [&](int s) __attribute__((always_inline)) {
      if (is_loader) wait_vmcnt<0>();
      __syncthreads();
      if (s + 1 < steps) issue(s + 1);
    };
    const bool active = at.mt * BM + wave_row(wave) < q.M && at.nt * BN + wave_col(wave) < (RES == SYMMETRIC ? q.M : q.N);
    open_step(0);
    if (!active) {
      for (int s = 1; s < steps; ++s) open_step(s);
    } else {
      read_phase(lds, 0);
      for (int s = 0; s < steps; ++s) {
        const unsigned base = lds + (unsigned)(s & 1) * kStage;
#pragma unroll
        for (int p = 0; p < 4; ++p) {
          if (p < 3) {
            read_phase(base, p + 1);
          } else {
            mfma::wait_lgkmcnt0();
            if (s + 1 < steps) {
              open_step(s + 1);
              read_phase(lds + (unsigned)((s + 1) & 1) * kStage, 0);
            }
          }
          __builtin_amdgcn_sched_barrier(0);        // (the compiler would move the reads behind the products, to where they are used)
          const int kk = p >> 1, ph = p & 1;
#pragma unroll
          for (int i = 0; i < FM / 2; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j)
              acc[ph * (FM / 2) + i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(held[kk][j], strm[p & 1][i], acc[ph * (FM / 2) + i][j], 0, 0, 0);
        }
      }
    }
    const Place was = at;
    const int was_part = part;
    ++slot;
    __syncthreads();                        // every wave has read its last fragments: the ring is free
    const bool more = open_tile(slot);
    if (more) issue(0);
    if (was_part >= 0) {
      f32x4* to = reinterpret_cast<f32x4*>(q.parts + (long)was_part * kPartFloats) + threadIdx.x;
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) to[(i * FN + j) * (NW * 64)] = acc[i][j];
    } else {
      const int row0 = was.mt * BM + wave_row(wave), col0 = was.nt * BN + wave_col(wave);
      if (active) finish<RES, TM, TN>(q, mu, first, was.which, row0, col0, was.mt != was.nt, acc, stg);
    }
    if (!more) break;
  }
}

// Adds the parts of the cut tiles and finishes them: eight workgroups per tile, a block of each wave each.
template <Result RES>
__global__ void __launch_bounds__(NW * 64) join_kernel(Product q, MuonProblem mu, int first) {
  __shared__ __attribute__((aligned(16))) char smem[NW * mfma::STG_BYTES];
  const int cut = blockIdx.x / (TM * TN), b0 = blockIdx.x / TN % TM, j0 = blockIdx.x % TN, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const Place at = place_of<RES>(q, q.full + cut);
  f32x4 acc[2][2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  const f32x4* from = reinterpret_cast<const f32x4*>(q.parts + (long)cut * q.split * kPartFloats) + threadIdx.x + (2 * b0 * FN + 2 * j0) * (NW * 64);
#pragma unroll 4
  for (int n = 0; n < q.split; ++n, from += kPartFloats / 4)
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) acc[i][j] += from[(i * FN + j) * (NW * 64)];
  const int row0 = at.mt * BM + wave_row(wave), col0 = at.nt * BN + wave_col(wave);
  if (row0 < q.M && col0 < (RES == SYMMETRIC ? q.M : q.N))
    finish<RES, 1, 1>(q, mu, first, at.which, row0 + b0 * 32, col0 + j0 * 32, at.mt != at.nt, acc, smem + wave * mfma::STG_BYTES);
}

// The same on tiles of 64 x 64 by four waves, 32 x 32 each, a workgroup per tile: where there are too few large tiles to fill the CUs, a product is
// bound by how long a tile takes from start to end.  (Sides are multiples of 128: no tile lies half outside.)  Four steps of operands are in LDS or on the way.
constexpr int SB = kOrthSmallTile, STAGES = 4, SNW = 4;
typedef KTile<SB, BK> SmallTile;
constexpr int kSmallStage = 2 * SmallTile::BYTES;
constexpr int kSmallLds = STAGES * kSmallStage + SNW * mfma::STG_BYTES;
static_assert(2 * kSmallLds <= 160 * 1024, "two workgroups share a CU's LDS");

template <Result RES>
__global__ void __launch_bounds__(SNW * 64, 2) small_product_kernel(Product q, MuonProblem mu, int first) {
  extern __shared__ __attribute__((aligned(256))) char smem[];
  const unsigned lds = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int wrow = (wave >> 1) * 32, wcol = (wave & 1) * 32;
  const int tm = q.M / SB, tn = q.N / SB, per = RES == SYMMETRIC ? tm * (tm + 1) / 2 : tm * tn, which = blockIdx.x / per;
  int at = blockIdx.x - which * per, mt, nt;
  if constexpr (RES == SYMMETRIC) {
    mt = (int)((sqrtf(8.f * (float)at + 1.f) - 1.f) * 0.5f);
    while ((mt + 1) * (mt + 2) / 2 <= at) ++mt;
    while (mt * (mt + 1) / 2 > at) --mt;
    mt = __builtin_amdgcn_readfirstlane(mt);
    nt = at - mt * (mt + 1) / 2;
  } else {
    mt = at / tn;
    nt = at - mt * tn;
  }
  const char* l = uniform_ptr(reinterpret_cast<const char*>(q.l + which * q.l_one + (long)mt * SB * q.ldl));
  const char* r = uniform_ptr(reinterpret_cast<const char*>(q.r + which * q.r_one + (long)nt * SB * q.ldr));
  constexpr int SLOTS = SmallTile::BYTES / 1024 / SNW;
  unsigned offl[SLOTS], offr[SLOTS];
#pragma unroll
  for (int j = 0; j < SLOTS; ++j) {
    const int row = (wave + j * SNW) * SmallTile::ROWS_PER_DMA + lane / SmallTile::CPR, chunk = (lane % SmallTile::CPR) ^ SmallTile::swz(row);
    offl[j] = (unsigned)row * (unsigned)q.ldl * 2u + (unsigned)chunk * 16u;
    offr[j] = (unsigned)row * (unsigned)q.ldr * 2u + (unsigned)chunk * 16u;
  }
  auto issue = [&](int s) __attribute__((always_inline)) {
    const unsigned to = lds + (unsigned)(s % STAGES) * kSmallStage + (unsigned)wave * 1024u;
#pragma unroll
    for (int j = 0; j < SLOTS; ++j) {
      dma16s(l + (long)s * BK * 2, offl[j], to + (unsigned)j * SNW * 1024u);
      dma16s(r + (long)s * BK * 2, offr[j], to + SmallTile::BYTES + (unsigned)j * SNW * 1024u);
    }
  };
  constexpr int LOADS = 2 * SLOTS;
  const unsigned fa = mfma::frag_origin<mfma::KMAJOR, SB, BK>(wrow, lane), fb = SmallTile::BYTES + mfma::frag_origin<mfma::KMAJOR, SB, BK>(wcol, lane);
  f32x4 acc[2][2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int steps = q.K / BK;
#pragma unroll
  for (int s = 0; s < STAGES - 1; ++s)
    if (s < steps) issue(s);
  for (int s = 0; s < steps; ++s) {
    // at most the loads of the steps behind this one are on their way
    if (s + 2 < steps) wait_vmcnt<2 * LOADS>();
    else if (s + 1 < steps) wait_vmcnt<LOADS>();
    else wait_vmcnt<0>();
    __syncthreads();                        // ... and every wave has read step s - 1, whose slot is filled next
    if (s + STAGES - 1 < steps) issue(s + STAGES - 1);
    const unsigned base = lds + (unsigned)(s % STAGES) * kSmallStage;
    f16x8 a[2][2], b[2][2];
#pragma unroll
    for (int kk = 0; kk < 2; ++kk)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        a[kk][i] = __builtin_bit_cast(f16x8, mfma::read_frag_dma<mfma::KMAJOR, SB, BK>(base + fa, i, kk));
        b[kk][i] = __builtin_bit_cast(f16x8, mfma::read_frag_dma<mfma::KMAJOR, SB, BK>(base + fb, i, kk));
      }
#pragma unroll
    for (int kk = 0; kk < 2; ++kk)
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(b[kk][j], a[kk][i], acc[i][j], 0, 0, 0);
  }
  finish<RES, 1, 1>(q, mu, first, which, mt * SB + wrow, nt * SB + wcol, mt != nt, acc, smem + STAGES * kSmallStage + wave * mfma::STG_BYTES);
}

template <Result RES> int product(Product q, const MuonProblem& mu, int first, int count, float* parts, hipStream_t s) {
  const OrthTiles t = orth_tiles(RES == SYMMETRIC, q.M, q.N);
  const long tiles = t.large * count, small_tiles = t.small * count;
  const Cut cut = cut_of(tiles, q.K / BK);
  if (small_tiles_time(small_tiles, q.K / BK) < cut.time) {
    small_product_kernel<RES><<<dim3((unsigned)small_tiles), dim3(SNW * 64), kSmallLds, s>>>(q, mu, first);
    MOE_LAUNCH_CHECK();
    return MOE_OK;
  }
  const int rem = (int)(tiles - cut.full);
  q.full = cut.full;
  q.split = cut.split;
  q.items = cut.full + rem * cut.split;
  q.parts = parts;
  product_kernel<RES><<<dim3(q.items < kGroups ? q.items : kGroups), dim3(NW * 64), kProductLds, s>>>(q, mu, first);
  MOE_LAUNCH_CHECK();
  if (rem > 0) {
    join_kernel<RES><<<dim3((unsigned)rem * TM * TN), dim3(NW * 64), 0, s>>>(q, mu, first);
    MOE_LAUNCH_CHECK();
  }
  return MOE_OK;
}

// Every product's dynamic-LDS limit is raised once per device; moe_init does it ahead of a graph capture.
}  // namespace
int orth_configure() {
  static std::atomic<unsigned long long> done{0};
  int dev = 0;
  MOE_HIP_TRY(hipGetDevice(&dev));
  if (dev < 0 || dev >= 64) return MOE_ERR_UNSUPPORTED;
  if (done.load(std::memory_order_acquire) >> dev & 1) return MOE_OK;
  for (const void* k : {(const void*)product_kernel<SYMMETRIC>, (const void*)product_kernel<KEPT>, (const void*)product_kernel<MUON_UPDATE>,
                        (const void*)product_kernel<OUT_F32>, (const void*)product_kernel<OUT_BF16>})
    MOE_HIP_TRY(hipFuncSetAttribute(k, hipFuncAttributeMaxDynamicSharedMemorySize, kProductLds));
  for (const void* k : {(const void*)small_product_kernel<SYMMETRIC>, (const void*)small_product_kernel<KEPT>, (const void*)small_product_kernel<MUON_UPDATE>,
                        (const void*)small_product_kernel<OUT_F32>, (const void*)small_product_kernel<OUT_BF16>})
    MOE_HIP_TRY(hipFuncSetAttribute(k, hipFuncAttributeMaxDynamicSharedMemorySize, kSmallLds));
  if (const int rc = orth_small_configure()) return rc;
  done.fetch_or(1ull << dev, std::memory_order_release);
  return MOE_OK;
}
namespace {

// The steps of a piece, each alone or two on the powers of one A.  With A' = A - c I a step's polynomial is
//   p(A) = s I + R,  s = p(c),  R = (b + 2 c2 c) A' + c2 A'^2
// The centre c is 0 at first and near the singular values' squares in late steps, where what is kept of A and R is then small (512 x 512, flat
// spectrum: error 1.5e-3 -> 8e-4).  Two steps may share one A and one product with X; A of the second one is
//   A2' = (s I + R)^2 (c I + A') - c' I,  made as  T = s A' + c R + R A',  A2' = s T + s c R + R T + (s^2 c - c') I
// and both together multiply X with s s' I + (s R' + s' R + R' R).  The first two and the last two are taken so: an error of A2' passes through one
// polynomial more, which matters least there (steps 0 1, 2, 3 4: errors of 2.1e-3 to 2.6e-3, and 6e-3 of matrices of an eighth of their rank).
double centre_of(int k, int steps) { return k < 3 ? 0.0 : k + 1 == steps ? 0.8 : 0.5; }
bool pair_at(int k, int steps) { return k + 1 < steps && (k == 0 || k + 2 == steps); }

int run_steps(const MuonProblem& mu, const OrthPlan& p, int first, int count, char* ws, hipStream_t stream) {
  half* hi = reinterpret_cast<half*>(ws + p.hi);
  half* t = reinterpret_cast<half*>(ws + p.t);
  half* lo = reinterpret_cast<half*>(ws + p.lo);
  half* other = reinterpret_cast<half*>(ws + p.other);          // the next one of the orientation that a step reads
  half* gram[4];
  for (int i = 0; i < 4; ++i) gram[i] = reinterpret_cast<half*>(ws + p.gram + i * p.gram_one);
  float* parts = reinterpret_cast<float*>(ws + p.parts);
  const bool tall = mu.rows > mu.cols;
  const long one = (long)p.R * p.C, gram_size = (long)p.S * p.S;
  // C = f1 E1 + f2 E2 + f L R + diagonal I of symmetric matrices, in units of what is kept
  auto symmetric = [&](int to, int l, int r, double f, int e1, double f1, int e2, double f2, double diagonal) -> int {
    Product q{};
    q.l = gram[l]; q.r = gram[r];
    q.l_one = q.r_one = q.c_one = gram_size;
    q.ldl = q.ldr = q.K = q.ldc = q.M = q.N = p.S;
    q.f = (float)(f / kScale);
    if (e1 >= 0) { q.e1 = gram[e1]; q.f1 = (float)f1; }
    if (e2 >= 0) { q.e2 = gram[e2]; q.f2 = (float)f2; }
    q.diagonal = (float)(diagonal * kScale);
    q.c = gram[to];
    return product<SYMMETRIC>(q, mu, first, count, parts, stream);
  };
  for (int k = 0; k < mu.steps; ++k) {
    OrthCoef c = mu.coef[k];
    double mid = centre_of(k, mu.steps), s = c.a + c.b * mid + c.c * mid * mid;
    Product a{};
    a.l = a.r = tall ? t : hi;
    a.l_one = a.r_one = one;
    a.ldl = a.ldr = a.K = tall ? p.R : p.C;
    a.M = a.N = p.S;
    a.f = 1.0f / kScale;
    a.diagonal = (float)(-mid * kScale);
    a.c = gram[0]; a.c_one = gram_size; a.ldc = p.S;
    if (const int rc = product<SYMMETRIC>(a, mu, first, count, parts, stream)) return rc;
    if (const int rc = symmetric(1, 0, 0, c.c, 0, c.b + 2 * c.c * mid, -1, 0, 0)) return rc;
    int r = 1;
    if (p.pairs && pair_at(k, mu.steps)) {
      const double mid2 = centre_of(++k, mu.steps);
      if (const int rc = symmetric(2, 1, 0, 1, 0, s, mid != 0 ? 1 : -1, mid, 0)) return rc;
      if (const int rc = symmetric(3, 1, 2, 1, 2, s, mid != 0 ? 1 : -1, s * mid, s * s * mid - mid2)) return rc;
      c = mu.coef[k];
      const double s2 = c.a + c.b * mid2 + c.c * mid2 * mid2;
      if (const int rc = symmetric(2, 3, 3, c.c, 3, c.b + 2 * c.c * mid2, -1, 0, 0)) return rc;
      if (const int rc = symmetric(0, 2, 1, 1, 2, s, 1, s2, 0)) return rc;
      s *= s2;
      r = 0;
    }
    Product x{};
    x.l = tall ? hi : gram[r];
    x.l_one = tall ? one : gram_size;
    x.r = tall ? gram[r] : t;
    x.r_one = tall ? gram_size : one;
    x.ldl = x.ldr = x.K = p.S;
    x.M = p.R; x.N = p.C;
    x.e1 = hi; x.f1 = (float)s;
    x.e2 = lo; x.f2 = (float)(s / kLow);
    x.f = 1.0f / kScale;
    x.c_one = one; x.ldc = p.C; x.ldt = p.R;
    if (k + 1 < mu.steps) {
      x.c = tall ? other : hi;
      x.c_lo = lo;
      x.ct = tall ? t : other;
      if (const int rc = product<KEPT>(x, mu, first, count, parts, stream)) return rc;
      half*& read = tall ? hi : t;
      half* was = read;
      read = other;
      other = was;
    } else {
      const int rc = !mu.out ? product<MUON_UPDATE>(x, mu, first, count, parts, stream)
                             : mu.out_dt == MOE_F32 ? product<OUT_F32>(x, mu, first, count, parts, stream) : product<OUT_BF16>(x, mu, first, count, parts, stream);
      if (rc) return rc;
    }
  }
  return MOE_OK;
}

template <typename TG, bool MUON> int start(const MuonProblem& mu, const OrthPlan& p, int first, int count, char* ws, hipStream_t s) {
  double* sums = reinterpret_cast<double*>(ws + p.sums);
  norm_kernel<TG, MUON><<<dim3(p.norm_blocks, count), dim3(256), 0, s>>>(mu, first, sums);
  MOE_LAUNCH_CHECK();
  if (p.small) return MOE_OK;
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
  const int least = rows < cols ? rows : cols, most = rows < cols ? cols : rows;
  const long size = (long)rows * cols;
  long blocks = (size + 4095) / 4096;
  const long share = 4096 / count + 1;
  if (blocks > share) blocks = share;
  p.norm_blocks = (int)(blocks < kNormBlocks ? blocks : kNormBlocks);
  p.small = least <= kSmallSide;
  if (p.small) {
    p.S = kSmallSide;
    const int tiles = cdiv(most, kSmallTile);
    p.tiles_per_slab = cdiv(tiles, 32);
    p.slabs = cdiv(tiles, p.tiles_per_slab);
    p.gram = 0;
    p.gram_one = (size_t)count * p.slabs * p.S * p.S * 8;
    p.t = p.gram_one;
    p.sums = p.t + (size_t)count * p.S * p.S * 4;
    p.bytes = p.sums + (size_t)count * p.norm_blocks * 8 + 256;
    return p;
  }
  p.R = (int)align_up(rows, kOrthPad);
  p.C = (int)align_up(cols, kOrthPad);
  p.S = p.R < p.C ? p.R : p.C;
  const size_t x = (size_t)count * p.R * p.C * 2;
  p.gram_one = (size_t)count * p.S * p.S * 2;
  p.hi = 0;
  p.lo = x;
  p.t = 2 * x;
  p.other = 3 * x;
  p.gram = 4 * x;
  // Steps in pairs leave out 6 (n - m) m^2 of a matrix's products and two of four rewritings of X, for two launches more and twice the error: where what they leave
  // out is long (us, in pairs and alone: 64 of 2048 x 1408 6740, 7150; two 4096 x 6144 3460, 3730; 8 of 2048 x 4096 2750, 3070; 2048 x 6144 683, 738; 1536 x 8192
  // 535, 651; below: 8 of 1024 x 2048 722, 704; 8 of 1024 x 1536 645, 586; 16 of 1024 x 1024 652, 610; 2048 x 2048 500, 441; 1024 x 4096 202, 229).
  p.pairs = (double)count * p.S * p.S * ((p.R < p.C ? p.C : p.R) - p.S) > 1.2e10;
  p.parts = p.gram + (p.pairs ? 4 : 2) * p.gram_one;
  const int contracted = p.R < p.C ? p.C : p.R;
  const long gram_parts = orth_most_parts(true, p.S, p.S, contracted, count), square_parts = orth_most_parts(true, p.S, p.S, p.S, count),
             x_parts = orth_most_parts(false, p.R, p.C, p.S, count);
  p.sums = p.parts + (size_t)std::max(gram_parts, std::max(square_parts, x_parts)) * kOrthPartFloats * 4;
  p.bytes = p.sums + (size_t)count * p.norm_blocks * 8 + 256;
  return p;
}

bool orth_is_default(const OrthCoef* c, int steps) {
  for (int k = 0; k < steps; ++k)
    if (c[k].a != kDefaultCoef.a || c[k].b != kDefaultCoef.b || c[k].c != kDefaultCoef.c) return false;
  return true;
}

constexpr double kLimit = 15.0;             // (and a little for what lies between the places that are looked at)
constexpr int kLook = 128;

// The largest factor by which steps one after another multiply a small singular value, and with it what an earlier step rounded off in a direction that a matrix
// of low rank does not have.  By a model of the roundings the relative error (2-norm) of such matrices is this gain times 4e-6 to 6e-6 for default steps and 3.2e-5 for
// the worst of 30 other lists; with a side of at most 64 it is 2e-7 to 3.5e-7.  Up to kMostGain it stays within the 0.24 that bf16 operands throughout leave after
// five default steps, whose gain is 485; seven of them have 5753, eight 19800.
constexpr double kMostGain = 8192, kMostGainSmall = 262144;
double gain_of(const OrthCoef* c, int steps) {
  double run = 1, most = 1;
  for (int k = 0; k < steps; ++k) {
    run = fmax(run, 1.0) * fabs(c[k].a);
    most = fmax(most, run);
  }
  return most;
}

bool orth_coefficients_ok(const OrthCoef* c, int steps, int rows, int cols) {
  if (!(gain_of(c, steps) <= ((rows < cols ? rows : cols) <= kSmallSide ? kMostGainSmall : kMostGain))) return false;
  // The default ones keep singular values within 1.21, and what is kept within 12: the looking alone takes longer than a small update.
  if (orth_is_default(c, steps)) return true;
  for (int k = 0; k < steps; ++k)
    if (!(fabs(c[k].a) <= 1e3 && fabs(c[k].b) <= 1e3 && fabs(c[k].c) <= 1e3)) return false;
  // singular values from 0 to `top` go to the polynomial's values there; what is kept on the way, with steps alone and in pairs, are values of
  // polynomials in them
  double top = 1.0;
  for (int k = 0; k < steps; ++k) {
    double next = 0;
    const double mid = centre_of(k, steps), s = c[k].a + c[k].b * mid + c[k].c * mid * mid;
    for (int i = 0; i <= kLook; ++i) {
      const double x = top * 1.01 * i / kLook, a = x * x - mid, r = (c[k].b + 2 * c[k].c * mid) * a + c[k].c * a * a, v = fabs(x * (s + r));
      double most = fmax(fmax(fabs(a), fabs(r)), v);
      if (pair_at(k, steps)) {
        const OrthCoef d = c[k + 1];
        const double mid2 = centre_of(k + 1, steps), s2 = d.a + d.b * mid2 + d.c * mid2 * mid2, t = s * a + mid * r + r * a,
                     a2 = s * t + s * mid * r + r * t + s * s * mid - mid2, r2 = (d.b + 2 * d.c * mid2) * a2 + d.c * a2 * a2, both = s * r2 + s2 * r + r2 * r;
        most = fmax(fmax(fmax(most, fabs(t)), fmax(fabs(a2), fabs(r2))), fabs(both));
      }
      most = fmax(most, fabs(x * x * (c[k].a + (c[k].b + c[k].c * x * x) * x * x)));      // (A times its polynomial, of small matrices)
      if (!(most <= kLimit)) return false;
      if (v > next) next = v;
    }
    top = next;
  }
  return true;
}

int launch_orth(const MuonProblem& mu, const OrthPlan& p, char* ws, hipStream_t s) {
  if (const int rc = orth_configure()) return rc;
  for (int first = 0; first < mu.batch; first += p.count) {
    const int count = mu.batch - first < p.count ? mu.batch - first : p.count;
    int rc;
    if (mu.out) rc = mu.u_dt == MOE_F32 ? start<float, false>(mu, p, first, count, ws, s) : start<bf16, false>(mu, p, first, count, ws, s);
    else rc = mu.u_dt == MOE_F32 ? start<float, true>(mu, p, first, count, ws, s) : start<bf16, true>(mu, p, first, count, ws, s);
    if (rc == MOE_OK) rc = p.small ? launch_orth_small(mu, p, first, count, ws, s) : run_steps(mu, p, first, count, ws, s);
    if (rc != MOE_OK) return rc;
  }
  return MOE_OK;
}

}  // namespace moe
