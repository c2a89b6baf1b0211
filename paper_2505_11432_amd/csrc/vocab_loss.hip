// Loss over a vocabulary: softmax cross entropy of hidden rows x [T, d] against a vocabulary matrix w [V, d], and its gradients.
//   z = x w^T,  lse_t = log sum_v exp z_tv,  loss_t = lse_t - z_t,target(t),  total = sum_t c_t loss_t
//   G = c (softmax(z) - onehot(target)),  dx = G w,  d_w = G^T x
// The products are those of gemm_mfma_dma.h (bf16) and gemm_f32*.hip (fp32); here are the passes between them.
//
// bf16: the logits never reach memory.  The first product leaves, per row and per 64 or 128 columns, the maximum and the sum of
// exp(z - maximum), and for a gradient exp(z - maximum) itself in 16 bits (unit16.h).  One pass per row joins the statistics and scales what was kept to G in
// bf16, in place.  G exists for one piece of rows at a time.  (To keep nothing and multiply x w^T again for the gradient would be 8 T V d
// operations instead of 6 T V d: a third more of a step that the matrix cores bound.)
// Rows whose target is left out are not computed: the rows that count are gathered to the front first, so that they cost nothing and whatever
// they hold, NaN included, reaches no result.
//
// Rounding.  G is rounded to bf16 once, 2^-8 of an element at most.  Where every token has the same weight G is kept without it and the products
// take it as a factor: most rows then hold nearly -1 in the column of the target, where numbers lie closest for their size.  That element is nearly
// the whole row, and the results of few tokens would carry its rounding error undivided, so what the rounding took off (`rest`) is kept in fp32:
// dx gets rest * w[target] when its parts are added, d_w one more row per token with rest in the target's column where the tokens are few
// (kFewRows) and that is free.
#include <algorithm>
#include <type_traits>

#include "dense_plan.h"
#include "moe_common.h"
#include "unit16.h"
#include "vocab_loss.h"

namespace moe {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(4))) unsigned u32x4;

constexpr float kLog2e = 1.44269504088896341f, kLowest = -3.402823466e38f;

__device__ __forceinline__ float exp_f32(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

// Joins (m, s) with another maximum and sum of exp(z - maximum).  A part without columns is (lowest, 0).
__device__ __forceinline__ void join(float& m, float& s, float m2, float s2) {
  const float top = fmaxf(m, m2);
  s = s * exp_f32(m - top) + s2 * exp_f32(m2 - top);
  m = top;
}
__device__ __forceinline__ void join_wave(float& m, float& s) {
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) join(m, s, __shfl_xor(m, off), __shfl_xor(s, off));
}
// over the WAVES waves of a workgroup; every thread gets the result
template <int WAVES> __device__ __forceinline__ void join_block(float& m, float& s, f32x2 (&lds)[WAVES]) {
  join_wave(m, s);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = f32x2{m, s};
  __syncthreads();
  m = lds[0][0];
  s = lds[0][1];
#pragma unroll
  for (int i = 1; i < WAVES; ++i) join(m, s, lds[i][0], lds[i][1]);
}

// A row's loss from its target's logit and the other words' maximum m and sum s of exp(z - m): 1 - p keeps its precision where p is near 1.
// A target's logit of +inf leaves no number, as the row's lse and gradient have none: log1p of the others alone would be 0.
struct RowLoss { float loss, lse, top, log_sum, miss; };          // lse = top + log_sum, miss = 1 - p
__device__ __forceinline__ RowLoss row_loss(float zt, float m, float s) {
  RowLoss r;
  r.top = fmaxf(m, zt);
  const float others = s * exp_f32(m - r.top), all = others + exp_f32(zt - r.top);
  r.log_sum = logf(all);
  r.lse = r.top + r.log_sum;
  r.loss = zt >= m && zt < __builtin_inff() ? log1pf(others) : (m - zt) + r.log_sum;
  r.miss = others / all;
  return r;
}

// Rows that count, in their order: token[i] = t, target_of[i] = its target; n; the pieces' numbers of rows.
// One workgroup: 8192 targets at a time, eight per thread.  (For lists that are too long for vocab_compact_few_kernel.)
__global__ void __launch_bounds__(1024) vocab_compact_kernel(const int32_t* __restrict__ target, int T, int V, int R, int pieces,
                                                             int32_t* __restrict__ token, int32_t* __restrict__ target_of,
                                                             VocabCounts* __restrict__ counts, int32_t* __restrict__ ranges) {
  __shared__ int wave_sum[16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int base = 0;
  for (int t0 = 0; t0 < T; t0 += 8192) {
    const int t = t0 + threadIdx.x * 8;
    int tg[8], mine = 0;
    if (t + 8 <= T) {
      typedef __attribute__((ext_vector_type(4))) int i32x4;
      typedef i32x4 i32x4_u __attribute__((aligned(4)));
      const i32x4 a = *reinterpret_cast<const i32x4_u*>(target + t), b = *reinterpret_cast<const i32x4_u*>(target + t + 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        tg[i] = a[i];
        tg[4 + i] = b[i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) tg[i] = t + i < T ? target[t + i] : -1;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) mine += tg[i] >= 0 && tg[i] < V;
    int incl = mine;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const int o = __shfl_up(incl, off);
      if (lane >= off) incl += o;
    }
    if (lane == 63) wave_sum[wave] = incl;
    __syncthreads();
    int at = base + incl - mine;
    for (int w = 0; w < 16; ++w) {
      if (w < wave) at += wave_sum[w];
      base += wave_sum[w];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (tg[i] >= 0 && tg[i] < V) {
        token[at] = t + i;
        target_of[at] = tg[i];
        ++at;
      }
    __syncthreads();
  }
  if (threadIdx.x == 0) *counts = VocabCounts{base, base ? 1.0f / (float)base : 0.f};
  for (int p = threadIdx.x; p < pieces; p += 1024) {
    const long left = (long)base - (long)p * R;
    const int n = left < 0 ? 0 : left < R ? (int)left : R;
    ranges[2 * p] = 0;
    ranges[2 * p + 1] = n;
  }
  if (threadIdx.x == 0) {                   // behind the pieces: the rows of d_w's contraction where every row comes twice
    ranges[2 * pieces] = 0;
    ranges[2 * pieces + 1] = 2 * base;
  }
}

// The same by a workgroup per 1024 tokens, each of which counts all targets in front of its own (16384 tokens: one workgroup 17 us).
__global__ void __launch_bounds__(256) vocab_compact_few_kernel(const int32_t* __restrict__ target, int T, int V, int R, int pieces, int32_t* __restrict__ token,
                                                                int32_t* __restrict__ target_of, VocabCounts* __restrict__ counts, int32_t* __restrict__ ranges) {
  __shared__ int sums[2][4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, first = blockIdx.x * 1024;
  auto keeps = [&](int tg) __attribute__((always_inline)) { return tg >= 0 && tg < V ? 1 : 0; };
  typedef __attribute__((ext_vector_type(4))) int i32x4;
  typedef i32x4 i32x4_u __attribute__((aligned(4)));
  int lower = 0;
#pragma unroll 4
  for (int t = threadIdx.x * 4; t < first; t += 1024) {             // (whole quads: `first` is a multiple of 1024)
    const i32x4 tg = *reinterpret_cast<const i32x4_u*>(target + t);
    lower += keeps(tg[0]) + keeps(tg[1]) + keeps(tg[2]) + keeps(tg[3]);
  }
  const int t0 = first + threadIdx.x * 4;
  int tg[4], mine = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    tg[i] = t0 + i < T ? target[t0 + i] : -1;
    mine += keeps(tg[i]);
  }
  int incl = mine;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const int o = __shfl_up(incl, off);
    if (lane >= off) incl += o;
    lower += __shfl_xor(lower, off);
  }
  if (lane == 63) {
    sums[0][wave] = lower;
    sums[1][wave] = incl;
  }
  __syncthreads();
  int at = incl - mine, base = 0;
  for (int w = 0; w < 4; ++w) {
    base += sums[0][w];
    if (w < wave) at += sums[1][w];
  }
  at += base;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (keeps(tg[i])) {
      token[at] = t0 + i;
      target_of[at] = tg[i];
      ++at;
    }
  if (blockIdx.x + 1 == gridDim.x) {                      // the last one has them all
    const int n = base + sums[1][0] + sums[1][1] + sums[1][2] + sums[1][3];
    if (threadIdx.x == 0) {
      *counts = VocabCounts{n, n ? 1.0f / (float)n : 0.f};
      ranges[2 * pieces] = 0;
      ranges[2 * pieces + 1] = 2 * n;
    }
    for (int p = threadIdx.x; p < pieces; p += 256) {
      const long left = (long)n - (long)p * R;
      ranges[2 * p] = 0;
      ranges[2 * p + 1] = left < 0 ? 0 : left < R ? (int)left : R;
    }
  }
}

template <typename T_> struct Row16 { static constexpr int N = 16 / (int)sizeof(T_); };

// The zeros of a token that is left out, by a wave
template <typename TX> __device__ __forceinline__ void clear_token(int t, int d, float* loss, float* lse, TX* dx) {
  const int lane = threadIdx.x & 63;
  if (lane == 0) loss[t] = lse[t] = 0.f;
  if (!dx) return;
  u32x4* dst = reinterpret_cast<u32x4*>(dx + (long)t * d);
  for (int i = lane; i < d / Row16<TX>::N; i += 64) dst[i] = u32x4{0u, 0u, 0u, 0u};
}

// Few tokens, one piece: compacting and gathering in one launch.  Every workgroup counts all targets and moves the rows of four tokens, a wave
// each.  (131 tokens, 1040 wide, fp32: 9.4 us in two launches.)
template <typename TX>
__global__ void __launch_bounds__(256) vocab_prepare_kernel(const TX* __restrict__ x, const int32_t* __restrict__ target, int T, int V, int d, int twice,
                                                            int32_t* __restrict__ token, int32_t* __restrict__ target_of, VocabCounts* __restrict__ counts,
                                                            int32_t* __restrict__ ranges, TX* __restrict__ xc, float* __restrict__ loss,
                                                            float* __restrict__ lse, TX* __restrict__ dx) {
  __shared__ int before[4], all[4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, first = blockIdx.x * 4;
  int lower = 0, kept = 0;                  // tokens that count: before this workgroup's, and all
  for (int t = threadIdx.x; t < T; t += 256) {
    const int tg = target[t], keeps = tg >= 0 && tg < V;
    kept += keeps;
    lower += keeps && t < first;
  }
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    lower += __shfl_xor(lower, off);
    kept += __shfl_xor(kept, off);
  }
  if (lane == 0) {
    before[wave] = lower;
    all[wave] = kept;
  }
  __syncthreads();
  const int n = all[0] + all[1] + all[2] + all[3];
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    *counts = VocabCounts{n, n ? 1.0f / (float)n : 0.f};
    ranges[0] = ranges[2] = 0;
    ranges[1] = n;
    ranges[3] = 2 * n;
  }
  const int t = first + wave;
  if (t >= T) return;
  const int tg = target[t];
  if (tg < 0 || tg >= V) {
    clear_token(t, d, loss, lse, dx);
    return;
  }
  int r = before[0] + before[1] + before[2] + before[3];
  for (int i = first; i < t; ++i) r += target[i] >= 0 && target[i] < V;
  if (lane == 0) {
    token[r] = t;
    target_of[r] = tg;
  }
  const u32x4* src = reinterpret_cast<const u32x4*>(x + (long)t * d);
  u32x4* dst = reinterpret_cast<u32x4*>(xc + (long)r * d);
  u32x4* again = reinterpret_cast<u32x4*>(xc + (long)(n + r) * d);
  for (int i = lane; i < d / Row16<TX>::N; i += 64) {
    const u32x4 v = src[i];
    dst[i] = v;
    if (twice) again[i] = v;
  }
}

// The rows of a piece to the front of xc, a wave per row; with the first piece also the zeros of the tokens left out.  Nothing where every token
// counts and there is one piece (`all`): the products then read x itself.
template <typename TX>
__global__ void __launch_bounds__(256) vocab_gather_kernel(const TX* __restrict__ x, const int32_t* __restrict__ target, const int32_t* __restrict__ token,
                                                           const int32_t* __restrict__ range, int all, int T, int V, int d, int row0, TX* __restrict__ xc,
                                                           float* __restrict__ loss, float* __restrict__ lse, TX* __restrict__ dx) {
  const int lane = threadIdx.x & 63, r = blockIdx.x * 4 + (threadIdx.x >> 6), n = range[1];
  if (all && n == T) return;
  if (r < n) {
    const u32x4* src = reinterpret_cast<const u32x4*>(x + (long)token[row0 + r] * d);
    u32x4* dst = reinterpret_cast<u32x4*>(xc + (long)r * d);
    for (int i = lane; i < d / Row16<TX>::N; i += 64) dst[i] = src[i];
  }
  if (row0 == 0 && r < T) {
    const int tg = target[r];
    if (tg < 0 || tg >= V) clear_token(r, d, loss, lse, dx);
  }
}

// loss and lse of a row from its parts, WAVES waves per row (forward only).  token: the row's token (NULL: rows are tokens).
template <int WAVES>
__global__ void __launch_bounds__(256) vocab_score_kernel(const f32x2* __restrict__ stats, int parts, const float* __restrict__ z_target,
                                                          const int32_t* __restrict__ target, const int32_t* __restrict__ token,
                                                          const int32_t* __restrict__ range, int R, int V, float* __restrict__ loss, float* __restrict__ lse) {
  __shared__ f32x2 lds[4];
  const int r = WAVES == 4 ? (int)blockIdx.x : (int)blockIdx.x * 4 + (int)(threadIdx.x >> 6), in_row = threadIdx.x & (64 * WAVES - 1);
  if (r >= (range ? min(range[1], R) : R)) return;
  const int t = token ? token[r] : r;
  if (!token && (target[r] < 0 || target[r] >= V)) {
    if (in_row == 0) loss[t] = lse[t] = 0.f;
    return;
  }
  const float zt = z_target[r];
  float m = kLowest, s = 0.f;
  for (int i = in_row; i < parts; i += 64 * WAVES) {
    const f32x2 p = stats[(long)r * parts + i];
    join(m, s, p[0], p[1]);
  }
  if constexpr (WAVES == 4) join_block(m, s, lds);
  else join_wave(m, s);
  if (in_row == 0) {
    const RowLoss l = row_loss(zt, m, s);
    loss[t] = l.loss;
    lse[t] = l.lse;
  }
}

struct RowOut {
  const int32_t* token;          // of the piece's rows
  const int32_t* target_of;
  const int32_t* range;          // [1]: rows of the piece
  const VocabCounts* counts;
  const float* token_w;          // [T] or NULL
  float* loss; float* lse;       // [T]
  float* weighted;               // c * loss of the piece's rows
  float* rest;                   // what rounding took off G in the target's column
};

__device__ __forceinline__ float row_weight(const RowOut& o, int t) { return o.token_w ? o.token_w[t] : o.counts->mean; }

// exp(z - maximum of its part) in 16 bits (unit16.h) -> G in bf16, in place, a workgroup per row.  Bound by memory: 4 bytes per element (8192 rows
// of 32000 words 197 us, 5.3 TB/s).  Threads by the row's length, so that each has some pieces of it, and 1024 where rows are few.  Whole steps of
// 16384 tokens, 256 wide (us; 64, 128, 256, 1024 threads): 1200 words 126, 131, 143, -; 2500 182, 185, 197, 334; 5000 282, 279, 286, -; 10000 529, 520,
// 514, 616; 2000 tokens, 512 wide, 102400 words -, -, 867, 845.
template <int THREADS>
__global__ void __launch_bounds__(THREADS) vocab_grad_rows_kernel(const f32x2* __restrict__ stats, int parts, int part_shift, const float* __restrict__ z_target,
                                                              int V, long ld, int twice, char* __restrict__ G, RowOut o) {
  __shared__ f32x2 lds[THREADS / 64];
  const int r = blockIdx.x, n = o.range[1];
  if (r >= n) return;
  const f32x2* row_stats = stats + (long)r * parts;
  float m = kLowest, s = 0.f;
  for (int i = threadIdx.x; i < parts; i += THREADS) join(m, s, row_stats[i][0], row_stats[i][1]);
  join_block(m, s, lds);
  const int t = o.token[r], tg = o.target_of[r];
  const RowLoss l = row_loss(z_target[r], m, s);
  const float weight = row_weight(o, t), c = o.token_w ? weight : 1.0f, g_target = -c * l.miss;
  const bf16 g_rounded = static_cast<bf16>(g_target);
  const float rest = g_target - static_cast<float>(g_rounded);
  if (threadIdx.x == 0) {
    o.loss[t] = l.loss;
    o.lse[t] = l.lse;
    o.weighted[r] = weight * l.loss;
    o.rest[r] = o.token_w ? rest : weight * rest;
  }
  char* row = G + (long)r * ld * 2;
  for (int v = threadIdx.x * 8; v < ld; v += THREADS * 8) {
    const u32x4 p = *reinterpret_cast<const u32x4*>(row + (long)v * 2);
    bf16x8 g;
    // eight columns lie in one part; past the width nothing was written
    const float f = v < V ? c * exp_f32((row_stats[v >> part_shift][0] - l.top) - l.log_sum) : 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) g[i] = v + i < V ? static_cast<bf16>((i & 1 ? unit16_high(p[i / 2]) : unit16_low(p[i / 2])) * f) : static_cast<bf16>(0.f);
    const unsigned at = (unsigned)(tg - v);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (at == (unsigned)i) g[i] = g_rounded;
    *reinterpret_cast<bf16x8*>(row + (long)v * 2) = g;
    if (twice) {
      bf16x8 q;
#pragma unroll
      for (int i = 0; i < 8; ++i) q[i] = static_cast<bf16>(at == (unsigned)i ? rest : 0.f);
      *reinterpret_cast<bf16x8*>(G + (long)(n + r) * ld * 2 + (long)v * 2) = q;
    }
  }
}

// fp32: the logits of a piece are in Z, in n_parts parts; loss and lse, and with GRAD G in the place of the first part.  PANELS: each panel of kF32Panel
// words has its rows together (then one part).
template <bool GRAD, int THREADS, bool PANELS>
__global__ void __launch_bounds__(THREADS) vocab_rows_f32_kernel(float* __restrict__ Z, int n_parts, long part_stride, int V, long ld, RowOut o) {
  __shared__ f32x2 lds[THREADS / 64];
  const int r = blockIdx.x;
  if (r >= o.range[1]) return;
  float* row = Z + (long)r * ld;
  auto at = [&](int v) __attribute__((always_inline)) { return PANELS ? row + (v / kF32Panel * part_stride + v % kF32Panel) : row + v; };
  const int t = o.token[r], tg = o.target_of[r], width = (V + 63) / 64 * 64;
  float zt = *at(tg);
  if constexpr (!PANELS)
    for (int p = 1; p < n_parts; ++p) zt += row[p * part_stride + tg];
  if (!PANELS && n_parts > 1) __syncthreads();        // (the sums go over the first part)
  float m = kLowest, s = 0.f;
  for (int v = threadIdx.x * 4; v < V; v += THREADS * 4) {
    f32x4 z = *reinterpret_cast<const f32x4*>(at(v));
    if (!PANELS && n_parts > 1) {
      for (int p = 1; p < n_parts; ++p) z += *reinterpret_cast<const f32x4*>(row + p * part_stride + v);
      if (GRAD) *reinterpret_cast<f32x4*>(row + v) = z;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (v + i >= V || v + i == tg) z[i] = -__builtin_inff();
    const float top = fmaxf(fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3])), m);
    s = s * exp_f32(m - top) + ((exp_f32(z[0] - top) + exp_f32(z[1] - top)) + (exp_f32(z[2] - top) + exp_f32(z[3] - top)));
    m = top;
  }
  join_block(m, s, lds);
  const RowLoss l = row_loss(zt, m, s);
  if (threadIdx.x == 0) {
    o.loss[t] = l.loss;
    o.lse[t] = l.lse;
  }
  if constexpr (GRAD) {                    // (every thread has read the target's logit and its share of the row: join_block waits for all)
    const float c = row_weight(o, t), g_target = -c * l.miss;
    if (threadIdx.x == 0) o.weighted[r] = c * l.loss;
    for (int v = threadIdx.x * 4; v < width; v += THREADS * 4) {
      f32x4 z = *reinterpret_cast<const f32x4*>(at(v));
#pragma unroll
      for (int i = 0; i < 4; ++i) z[i] = v + i >= V ? 0.f : v + i == tg ? g_target : c * exp_f32((z[i] - l.top) - l.log_sum);
      *reinterpret_cast<f32x4*>(at(v)) = z;
    }
  }
}

// total = sum of the weighted losses, in a fixed order, in 64 bits, by one workgroup of 256
__device__ __forceinline__ void sum_total(const float* __restrict__ weighted, int n, float* __restrict__ total) {
  __shared__ double lds[4];
  double s[4] = {0.0, 0.0, 0.0, 0.0};
  for (int i = threadIdx.x; i < n; i += 1024)
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (i + q * 256 < n) s[q] += (double)weighted[i + q * 256];
  double all = (s[0] + s[1]) + (s[2] + s[3]);
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) all += __shfl_xor(all, off);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = all;
  __syncthreads();
  if (threadIdx.x == 0) *total = (float)((lds[0] + lds[1]) + (lds[2] + lds[3]));
}

// dx of the piece's rows: the product's whole tiles, or the sum of a cut tile's parts, with what the rounding of G took off in the target's
// column, rounded once; `each` pieces of 16 bytes per thread.  With the last piece a further workgroup makes the total.
template <int TILE>
__global__ void __launch_bounds__(256) vocab_dx_kernel(int each, const float* __restrict__ whole, const float* __restrict__ parts, int groups, CutCost cost,
                                                       const bf16* __restrict__ w, int d, int V, const RowOut o, bf16* __restrict__ dx,
                                                       const float* __restrict__ weighted, float* __restrict__ total) {
  if (total && blockIdx.x == gridDim.x - 1) {
    sum_total(weighted, o.counts->n, total);
    return;
  }
  const int n = o.range[1], vecs = d / 8, tiles_m = (n + TILE - 1) / TILE, tiles_n = (d + TILE - 1) / TILE;
  const long first = (long)blockIdx.x * each * 256, left = (long)n * vecs - first;
  if (left <= 0) return;
  const int row0 = (int)(first / vecs), in_row0 = (int)(first - (long)row0 * vecs), items = (int)min(left, each * 256L);
  const DensePlan cut = dense_plan(tiles_m * tiles_n, groups, (V + 63) / 64, cost, true);
  for (int i = threadIdx.x; i < items; i += 256) {
    const int q = (in_row0 + i) / vecs, r = row0 + q, c = (in_row0 + i - q * vecs) * 8;
    const int l = dense_tile_index(r / TILE, c / TILE, tiles_m, tiles_n);
    f32x4 a, b;
    if (l < cut.full_tiles) {
      const float* src = whole + (long)r * d + c;
      a = *reinterpret_cast<const f32x4*>(src);
      b = *reinterpret_cast<const f32x4*>(src + 4);
    } else {
      const float* src = parts + (long)(l - cut.full_tiles) * cut.split * (TILE * TILE) + (r % TILE) * TILE + c % TILE;
      a = b = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
      for (int p = 0; p < cut.split; ++p, src += TILE * TILE) {
        a += *reinterpret_cast<const f32x4*>(src);
        b += *reinterpret_cast<const f32x4*>(src + 4);
      }
    }
    const bf16x8 wt = *reinterpret_cast<const bf16x8*>(w + (long)o.target_of[r] * d + c);
    const float rest = o.rest[r];
    bf16x8 out;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      out[q] = static_cast<bf16>(a[q] + rest * (float)wt[q]);
      out[4 + q] = static_cast<bf16>(b[q] + rest * (float)wt[4 + q]);
    }
    *reinterpret_cast<bf16x8*>(dx + (long)o.token[r] * d + c) = out;
  }
}
__global__ void __launch_bounds__(256) vocab_dx_f32_kernel(const float* __restrict__ parts, int n_parts, long part_stride, int d, const RowOut o,
                                                           float* __restrict__ dx, const float* __restrict__ weighted, float* __restrict__ total) {
  if (total && blockIdx.x == gridDim.x - 1) {
    sum_total(weighted, o.counts->n, total);
    return;
  }
  const int vecs = d / 4;
  const long items = (long)o.range[1] * vecs, blocks = gridDim.x - (total ? 1 : 0);
  for (long i = blockIdx.x * 256L + threadIdx.x; i < items; i += blocks * 256L) {
    const int r = (int)(i / vecs), c = (int)(i - (long)r * vecs) * 4;
    const float* src = parts + (long)r * d + c;
    f32x4 a = *reinterpret_cast<const f32x4*>(src);
    for (int p = 1; p < n_parts; ++p) a += *reinterpret_cast<const f32x4*>(src + p * part_stride);
    *reinterpret_cast<f32x4*>(dx + (long)o.token[r] * d + c) = a;
  }
}
// out (+)= the sum of its parts
__global__ void __launch_bounds__(256) vocab_add_f32_kernel(const float* __restrict__ parts, int n_parts, long part_stride, long vecs, int accumulate,
                                                            float* __restrict__ out) {
  for (long i = blockIdx.x * 256L + threadIdx.x; i < vecs; i += gridDim.x * 256L) {
    f32x4 a = *reinterpret_cast<const f32x4*>(parts + 4 * i);
    for (int p = 1; p < n_parts; ++p) a += *reinterpret_cast<const f32x4*>(parts + p * part_stride + 4 * i);
    f32x4* dst = reinterpret_cast<f32x4*>(out + 4 * i);
    *dst = accumulate ? a + *dst : a;
  }
}

// The vocabulary gradient that several pieces have added up in fp32, to bf16 (plus what was there)
__global__ void __launch_bounds__(256) vocab_dw_round_kernel(const float* __restrict__ src, long vecs, int accumulate, bf16* __restrict__ d_w) {
  for (long i = blockIdx.x * 256L + threadIdx.x; i < vecs; i += gridDim.x * 256L) {
    const f32x4 a = *reinterpret_cast<const f32x4*>(src + 8 * i), b = *reinterpret_cast<const f32x4*>(src + 8 * i + 4);
    bf16x8 out, old;
    if (accumulate) old = *reinterpret_cast<const bf16x8*>(d_w + 8 * i);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      out[q] = static_cast<bf16>(accumulate ? a[q] + (float)old[q] : a[q]);
      out[4 + q] = static_cast<bf16>(accumulate ? b[q] + (float)old[4 + q] : b[q]);
    }
    *reinterpret_cast<bf16x8*>(d_w + 8 * i) = out;
  }
}

unsigned blocks_for(long items) { return (unsigned)(items < 256L * 4096 ? (items + 255) / 256 : 4096); }

size_t take(size_t& at, size_t bytes) {
  const size_t here = at;
  at += align_up(bytes, 256);
  return here;
}

// Up to so many rows d_w takes a second row per token with what the rounding of G left (its product then waits for the gradient to be written,
// V * d elements, not for the matrix cores).
constexpr int kFewRows = 128;
// Forward only: up to so many rows nothing is gathered.  They are one row of tiles whether they count or not, and rows do not mix.
constexpr int kScoreAsIs = 256;
// and so many rows at a time, which bounds the statistics (128 k words: 0.5 GB)
constexpr int kScorePiece = 65536;
// Up to so many tokens every workgroup of the gathering counts them itself.
constexpr int kPrepareTokens = 2048;
// Up to so many tokens every workgroup that compacts a part of them counts the ones before it.
constexpr int kCompactFew = 65536;
// Up to so many rows a row's pass has 1024 threads instead of 256: the CUs hold no more workgroups anyway.
constexpr int kFewGroups = 512;
// fp32 products in parts: floats that all parts may take
constexpr size_t kPartFloats = (size_t)64 << 20;

GemmProblem f32_logits(const VocabPlan& p, const void* x, const void* w, const int32_t* range, int d, int V, float* Z) {
  GemmProblem g{};
  g.offsets = range; g.E = 1; g.mode = 0; g.M = p.R;
  g.A = x; g.a_rs = d; g.a_cs = 1;
  g.B = w; g.b_rs = 1; g.b_cs = d;
  g.C = Z; g.ldc = p.ld; g.N = (int)align_up((size_t)V, 16); g.K = d; g.b_rows = V;
  return g;
}
GemmProblem f32_dx(const VocabPlan& p, const float* G, const void* w, const int32_t* range, int d, int V, float* out) {
  GemmProblem g{};
  g.offsets = range; g.E = 1; g.mode = 0; g.M = p.R;
  g.A = G; g.a_rs = p.ld; g.a_cs = 1;
  g.B = w; g.b_rs = d; g.b_cs = 1;
  g.C = out; g.ldc = d; g.N = d; g.K = V;
  return g;
}
GemmProblem f32_dw(const VocabPlan& p, const float* G, const void* x, const int32_t* range, int d, int V, float* out) {
  GemmProblem g{};
  g.offsets = range; g.E = 1; g.mode = 1; g.M = (int)align_up((size_t)V, 64); g.c_rows = V;
  g.A = G; g.a_rs = 1; g.a_cs = p.ld;
  g.B = x; g.b_rs = d; g.b_cs = 1;
  g.C = out; g.ldc = d; g.N = d; g.K = p.R;
  return g;
}
// as one product, whichever way is the faster one, or in the plan's parts
int launch_f32(const GemmProblem& g, F32Plan plan, hipStream_t s) {
  return plan.parts > 1 ? launch_gemm_f32_cut(g, plan, s) : launch_gemm_f32(g, s);
}
F32Plan plan_f32(const GemmProblem& g) {
  const F32Product q{g.mode == 0, g.M, g.N, g.K, 1};
  const long room = (long)(kPartFloats / ((size_t)g.M * g.ldc));
  if (!gemm_f32_cuts(g)) return F32Plan{F32_64, 1};
  return g.mode == 0 && g.b_rs == 1 ? f32_logit_parts(q, room) : f32_parts(q, room);
}

}  // namespace

VocabPlan vocab_plan(int T, int d, int V, moe_dtype dt, moe_dtype grad_dt, int piece_rows, bool grad) {
  VocabPlan p{};
  const bool f32 = dt == MOE_F32;
  const size_t es = dtype_size(dt);
  p.R = piece_rows > 0 && piece_rows < T ? piece_rows : T;
  if (!grad && !f32) p.R = T < kScorePiece ? T : kScorePiece;          // nothing is kept per element
  if (f32) p.R = vocab_f32_rows(p.R, V, d);
  p.pieces = (T + p.R - 1) / p.R;
  const long ld = (long)align_up((size_t)V, 64);
  p.ld = f32 ? vocab_f32_panel(ld) : ld;
  p.panels = (int)((ld + p.ld - 1) / p.ld);
  p.gather = grad || f32 || T > kScoreAsIs;
  p.twice = grad && !f32 && T <= kFewRows && p.pieces == 1;
  const size_t R = (size_t)p.R, rows = R * p.pieces, copies = p.twice ? 2 : 1;
  size_t at = 0;
  p.counts = take(at, sizeof(VocabCounts));
  p.ranges = take(at, ((size_t)p.pieces + 1) * 8);
  if (p.gather) {
    p.token = take(at, rows * 4);
    p.target_of = take(at, rows * 4);
    p.xc = take(at, copies * R * d * es);
  }
  if (f32) {
    auto products = [&](int words) {
      VocabPlan::Products q{};
      q.z = plan_f32(f32_logits(p, nullptr, nullptr, nullptr, d, words, nullptr));
      if (p.panels > 1) q.z.parts = 1;                  // (the row pass knows panels or parts)
      q.dx = plan_f32(f32_dx(p, nullptr, nullptr, nullptr, d, words, nullptr));
      q.dw = plan_f32(f32_dw(p, nullptr, nullptr, nullptr, d, words, nullptr));
      return q;
    };
    p.last = products(V - (p.panels - 1) * (int)p.ld);
    p.whole = p.panels > 1 ? products((int)p.ld) : p.last;
    p.G = take(at, (size_t)p.whole.z.parts * p.panels * R * p.ld * 4);
  } else {
    p.tiles = mfma_vocab_tiles(p.R, V, d, grad);
    p.stats = take(at, R * p.tiles.parts * 8);
    p.z_target = take(at, R * 4);
    if (grad) p.G = take(at, copies * R * p.ld * 2);
  }
  if (grad) {
    p.weighted = take(at, rows * 4);
    p.rest = take(at, R * 4);
    size_t part_floats;
    if (f32) {
      // dx's parts are added where its rows are placed, or panel by panel into the sum of those before; d_w's into d_w
      p.dxc = take(at, (size_t)(p.panels > 1 ? 1 : p.last.dx.parts) * R * d * 4);
      part_floats = 0;
      for (const VocabPlan::Products* q : {&p.whole, &p.last}) {
        const size_t words = q == &p.last ? (size_t)V - (p.panels - 1) * p.ld : (size_t)p.ld;
        const size_t dx_floats = p.panels > 1 && q->dx.parts > 1 ? (size_t)q->dx.parts * R * d : 0;
        const size_t dw_floats = q->dw.parts > 1 ? (size_t)q->dw.parts * align_up(words, 64) * d : 0;
        part_floats = std::max({part_floats, dx_floats, dw_floats});
      }
    } else {
      const size_t dx_floats = mfma_vocab_dx_plan(p.R, V, d).part_floats, dw_floats = mfma_vocab_dw_part_floats(p.twice ? 2 * p.R : p.R, V, d);
      p.dxc = take(at, R * d * 4);
      part_floats = dx_floats > dw_floats ? dx_floats : dw_floats;
      p.dw_sum_used = p.pieces > 1 && grad_dt == MOE_BF16;
      if (p.dw_sum_used) p.dw_sum = take(at, (size_t)V * d * 4);
    }
    p.parts = take(at, part_floats * 4);
  }
  p.bytes = at;
  return p;
}

namespace {

template <typename TX> int gather_rows(const VocabProblem& q, const VocabPlan& p, char* ws, int piece, hipStream_t s) {
  int32_t* token = reinterpret_cast<int32_t*>(ws + p.token);
  int32_t* target_of = reinterpret_cast<int32_t*>(ws + p.target_of);
  int32_t* ranges = reinterpret_cast<int32_t*>(ws + p.ranges);
  VocabCounts* counts = reinterpret_cast<VocabCounts*>(ws + p.counts);
  TX* xc = reinterpret_cast<TX*>(ws + p.xc);
  const TX* x = static_cast<const TX*>(q.x);
  TX* dx = static_cast<TX*>(q.grad ? q.dx : nullptr);
  if (p.pieces == 1 && q.T <= kPrepareTokens) {
    vocab_prepare_kernel<TX><<<dim3(cdiv(q.T, 4)), dim3(256), 0, s>>>(x, q.target, q.T, q.V, q.d, p.twice, token, target_of, counts, ranges, xc, q.loss, q.lse, dx);
    MOE_LAUNCH_CHECK();
    return MOE_OK;
  }
  if (piece == 0) {
    if (q.T <= kCompactFew)
      vocab_compact_few_kernel<<<dim3(cdiv(q.T, 1024)), dim3(256), 0, s>>>(q.target, q.T, q.V, p.R, p.pieces, token, target_of, counts, ranges);
    else
      vocab_compact_kernel<<<dim3(1), dim3(1024), 0, s>>>(q.target, q.T, q.V, p.R, p.pieces, token, target_of, counts, ranges);
    MOE_LAUNCH_CHECK();
  }
  vocab_gather_kernel<TX><<<dim3(cdiv(piece == 0 ? q.T : p.R, 4)), dim3(256), 0, s>>>(x, q.target, token, ranges + 2 * piece, p.pieces == 1 && q.dt == MOE_BF16, q.T, q.V, q.d, piece * p.R, xc,
                                                                                    q.loss, q.lse, dx);
  MOE_LAUNCH_CHECK();
  return MOE_OK;
}

// loss and lse of rows from their statistics: a workgroup per row where rows are few
int score_rows(const VocabProblem& q, const VocabPlan& p, const float* stats, const float* z_target, const int32_t* target, const int32_t* token,
               const int32_t* range, hipStream_t s) {
  const f32x2* st = reinterpret_cast<const f32x2*>(stats);
  if (p.R <= 1024) vocab_score_kernel<4><<<dim3(p.R), dim3(256), 0, s>>>(st, p.tiles.parts, z_target, target, token, range, p.R, q.V, q.loss, q.lse);
  else vocab_score_kernel<1><<<dim3(cdiv(p.R, 4)), dim3(256), 0, s>>>(st, p.tiles.parts, z_target, target, token, range, p.R, q.V, q.loss, q.lse);
  MOE_LAUNCH_CHECK();
  return MOE_OK;
}

int f32_piece(const VocabProblem& q, const VocabPlan& p, char* ws, int piece, const RowOut& o, hipStream_t s) {
  const int R = p.R, d = q.d, V = q.V;
  float* Z = reinterpret_cast<float*>(ws + p.G);
  float* parts = reinterpret_cast<float*>(ws + p.parts);
  const float* w = static_cast<const float*>(q.w);
  const void* xc = ws + p.xc;
  const long panel_floats = (long)R * p.ld;
  // f(words of the panel, its first word, its logits, its products)
  auto each_panel = [&](auto f) {
    for (int i = 0; i < p.panels; ++i) {
      const bool last = i + 1 == p.panels;
      const long v0 = i * p.ld;
      const int rc = f(last ? V - (int)v0 : (int)p.ld, v0, Z + i * panel_floats, last ? p.last : p.whole);
      if (rc != MOE_OK) return rc;
    }
    return (int)MOE_OK;
  };
  auto add = [&](int n, long stride, long floats, int accumulate, float* out) {
    vocab_add_f32_kernel<<<dim3(blocks_for(floats / 4)), dim3(256), 0, s>>>(parts, n, stride, floats / 4, accumulate, out);
    MOE_LAUNCH_CHECK();
    return (int)MOE_OK;
  };
  int rc = each_panel([&](int words, long v0, float* z, const VocabPlan::Products& plan) {
    return launch_f32(f32_logits(p, xc, w + v0 * d, o.range, d, words, z), plan.z, s);
  });
  if (rc != MOE_OK) return rc;
  const int n_parts = p.last.z.parts;
  auto rows = [&](auto grad, auto threads, auto panels) {
    constexpr int N = decltype(threads)::value;
    vocab_rows_f32_kernel<decltype(grad)::value, N, decltype(panels)::value><<<dim3(R), dim3(N), 0, s>>>(Z, n_parts, panel_floats, V, p.ld, o);
  };
  auto rows_in = [&](auto grad, auto panels) {
    if (R <= kFewGroups) rows(grad, std::integral_constant<int, 1024>(), panels);
    else rows(grad, std::integral_constant<int, 256>(), panels);
  };
  if (q.grad && p.panels > 1) rows_in(std::true_type(), std::true_type());
  else if (q.grad) rows_in(std::true_type(), std::false_type());
  else if (p.panels > 1) rows_in(std::false_type(), std::true_type());
  else rows_in(std::false_type(), std::false_type());
  MOE_LAUNCH_CHECK();
  if (!q.grad) return MOE_OK;
  float* dxc = reinterpret_cast<float*>(ws + p.dxc);
  rc = each_panel([&](int words, long v0, float* g, const VocabPlan::Products& plan) {
    if (p.panels == 1) return launch_f32(f32_dx(p, g, w, o.range, d, words, dxc), plan.dx, s);
    const int accumulate = v0 > 0, cut = plan.dx.parts > 1;
    GemmProblem product = f32_dx(p, g, w + v0 * d, o.range, d, words, cut ? parts : dxc);
    product.accumulate = cut ? 0 : accumulate;
    const int made = launch_f32(product, plan.dx, s);
    return made != MOE_OK || !cut ? made : add(plan.dx.parts, (long)R * d, (long)R * d, accumulate, dxc);
  });
  if (rc != MOE_OK) return rc;
  const bool last = piece + 1 == p.pieces;
  vocab_dx_f32_kernel<<<dim3(blocks_for((long)R * d / 4) + last), dim3(256), 0, s>>>(dxc, p.panels > 1 ? 1 : p.last.dx.parts, (long)R * d, d, o,
                                                                                    static_cast<float*>(q.dx), reinterpret_cast<float*>(ws + p.weighted),
                                                                                    last ? q.total : nullptr);
  MOE_LAUNCH_CHECK();
  const int accumulate = q.accumulate || piece > 0;
  return each_panel([&](int words, long v0, float* g, const VocabPlan::Products& plan) {
    float* d_w = static_cast<float*>(q.d_w) + v0 * d;
    const int cut = plan.dw.parts > 1;
    GemmProblem product = f32_dw(p, g, xc, o.range, d, words, cut ? parts : d_w);
    product.accumulate = cut ? 0 : accumulate;
    const int made = launch_f32(product, plan.dw, s);
    return made != MOE_OK || !cut ? made : add(plan.dw.parts, (long)product.M * d, (long)words * d, accumulate, d_w);
  });
}

int bf16_piece(const VocabProblem& q, const VocabPlan& p, char* ws, int piece, const RowOut& o, hipStream_t s) {
  const int R = p.R, d = q.d, V = q.V;
  float* z_target = reinterpret_cast<float*>(ws + p.z_target);
  float* stats = reinterpret_cast<float*>(ws + p.stats);
  const void* xc = ws + p.xc;
  const VocabRows x{xc, p.pieces == 1 && q.T > kPrepareTokens ? q.x : nullptr, o.range + 1, q.T};
  int rc = mfma_vocab_softmax(x, q.w, o.range + 1, o.target_of, R, V, d, q.grad ? ws + p.G : nullptr, p.ld, stats, z_target, s);
  if (rc != MOE_OK) return rc;
  if (!q.grad) return score_rows(q, p, stats, z_target, o.target_of, o.token, o.range, s);
  const f32x2* st = reinterpret_cast<const f32x2*>(stats);
  auto rows = [&](auto threads) {
    constexpr int N = decltype(threads)::value;
    vocab_grad_rows_kernel<N><<<dim3(R), dim3(N), 0, s>>>(st, p.tiles.parts, p.tiles.shift, z_target, V, p.ld, p.twice, ws + p.G, o);
  };
  const bool few = R <= kFewGroups && V > 1024;
  if (!few && V <= 4096) rows(std::integral_constant<int, 64>());
  else if (!few && V <= 8192) rows(std::integral_constant<int, 128>());
  else if (!few && V <= 65536) rows(std::integral_constant<int, 256>());
  else rows(std::integral_constant<int, 1024>());
  MOE_LAUNCH_CHECK();
  float* dxc = reinterpret_cast<float*>(ws + p.dxc);
  float* parts = reinterpret_cast<float*>(ws + p.parts);
  const VocabDxPlan plan = mfma_vocab_dx_plan(R, V, d);
  const float* scale = q.token_w ? nullptr : &o.counts->mean;
  int groups = 0;
  rc = mfma_vocab_dx(ws + p.G, p.ld, q.w, o.range + 1, scale, R, V, d, plan, dxc, parts, &groups, s);
  if (rc != MOE_OK) return rc;
  const bool last = piece + 1 == p.pieces;
  const long pieces = (long)R * d / 8;
  const int each = pieces < 256 * 2048 ? 1 : 4;           // (a workgroup works out the plan of the cut tiles first)
  const dim3 grid((unsigned)((pieces + each * 256 - 1) / (each * 256)) + last);
  float* total = last ? q.total : nullptr;
  const float* weighted = reinterpret_cast<float*>(ws + p.weighted);
  const bf16* w = static_cast<const bf16*>(q.w);
  if (plan.tile == 256) vocab_dx_kernel<256><<<grid, dim3(256), 0, s>>>(each, dxc, parts, groups, plan.cost, w, d, V, o, static_cast<bf16*>(q.dx), weighted, total);
  else vocab_dx_kernel<128><<<grid, dim3(256), 0, s>>>(each, dxc, parts, groups, plan.cost, w, d, V, o, static_cast<bf16*>(q.dx), weighted, total);
  MOE_LAUNCH_CHECK();
  const int32_t* n_dw = p.twice ? o.range + 3 : o.range + 1;
  if (p.dw_sum_used) return mfma_vocab_dw(ws + p.G, p.ld, x, n_dw, scale, R, V, d, ws + p.dw_sum, MOE_F32, piece > 0, parts, s);
  return mfma_vocab_dw(ws + p.G, p.ld, x, n_dw, scale, p.twice ? 2 * R : R, V, d, q.d_w, q.grad_dt, q.accumulate || piece > 0, parts, s);
}

}  // namespace

int launch_vocab_loss(const VocabProblem& q, const VocabPlan& p, char* ws, hipStream_t s) {
  if (!p.gather) {
    float* z_target = reinterpret_cast<float*>(ws + p.z_target);
    float* stats = reinterpret_cast<float*>(ws + p.stats);
    const int rc = mfma_vocab_softmax(VocabRows{q.x, nullptr, nullptr, 0}, q.w, nullptr, q.target, q.T, q.V, q.d, nullptr, 0, stats, z_target, s);
    return rc != MOE_OK ? rc : score_rows(q, p, stats, z_target, q.target, nullptr, nullptr, s);
  }
  for (int piece = 0; piece < p.pieces; ++piece) {
    int rc = q.dt == MOE_F32 ? gather_rows<float>(q, p, ws, piece, s) : gather_rows<bf16>(q, p, ws, piece, s);
    if (rc != MOE_OK) return rc;
    const long row0 = (long)piece * p.R;
    const RowOut o{reinterpret_cast<int32_t*>(ws + p.token) + row0, reinterpret_cast<int32_t*>(ws + p.target_of) + row0,
                   reinterpret_cast<int32_t*>(ws + p.ranges) + 2 * piece, reinterpret_cast<VocabCounts*>(ws + p.counts), q.token_w, q.loss, q.lse,
                   reinterpret_cast<float*>(ws + p.weighted) + row0, reinterpret_cast<float*>(ws + p.rest)};
    rc = q.dt == MOE_F32 ? f32_piece(q, p, ws, piece, o, s) : bf16_piece(q, p, ws, piece, o, s);
    if (rc != MOE_OK) return rc;
  }
  if (p.dw_sum_used) {
    const long vecs = (long)q.V * q.d / 8;
    vocab_dw_round_kernel<<<dim3(blocks_for(vecs)), dim3(256), 0, s>>>(reinterpret_cast<const float*>(ws + p.dw_sum), vecs, q.accumulate, (bf16*)q.d_w);
    MOE_LAUNCH_CHECK();
  }
  return MOE_OK;
}

}  // namespace moe
