// Loss over a vocabulary: softmax cross entropy of hidden rows x [T, d] against a vocabulary matrix w [V, d], and its gradients.
//   z = x w^T,  lse_t = log sum_v exp z_tv,  loss_t = lse_t - z_t,target(t),  total = sum_t c_t loss_t
//   G = c (softmax(z) - onehot(target)),  dx = G w,  d_w = G^T x
// The products are those of gemm_mfma_dma.h (bf16) and gemm_f32*.hip (fp32); here are the passes between them.
//
// bf16: the logits never reach memory.  The first product leaves, per row and per 64 or 128 columns, the maximum and the sum of
// exp(z - maximum), and for a gradient exp(z - maximum) itself in fp16.  One pass per row joins the statistics and scales what was kept to G in
// bf16, in place.  G exists for one piece of rows at a time.  (To keep nothing and multiply x w^T again for the gradient would be 8 T V d
// operations instead of 6 T V d: a third more of a step that the matrix cores bound.)
// Rows whose target is left out are not computed: the rows that count are gathered to the front first, so that they cost nothing and whatever
// they hold, NaN included, reaches no result.
//
// Rounding.  G is rounded to bf16 once, 2^-8 of an element at most.  In the column of the target it is nearly the whole row, and the rows of
// few tokens would carry its rounding error undivided, so what the rounding took off (`rest`) is kept in fp32: dx gets rest * w[target] when its
// parts are added, d_w one more row per token with rest in the target's column where the tokens are few (kFewRows), where that is free.
#include "moe_common.h"
#include "vocab_loss.h"

namespace moe {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
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
// over the 256 threads of a workgroup; every thread gets the result
__device__ __forceinline__ void join_block(float& m, float& s, f32x2 (&lds)[4]) {
  join_wave(m, s);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = f32x2{m, s};
  __syncthreads();
  m = lds[0][0];
  s = lds[0][1];
#pragma unroll
  for (int i = 1; i < 4; ++i) join(m, s, lds[i][0], lds[i][1]);
}

// A row's loss from its target's logit and the other words' maximum m and sum s of exp(z - m): 1 - p keeps its precision where p is near 1.
struct RowLoss { float loss, lse, top, log_sum, miss; };          // lse = top + log_sum, miss = 1 - p
__device__ __forceinline__ RowLoss row_loss(float zt, float m, float s) {
  RowLoss r;
  r.top = fmaxf(m, zt);
  const float others = s * exp_f32(m - r.top), all = others + exp_f32(zt - r.top);
  r.log_sum = logf(all);
  r.lse = r.top + r.log_sum;
  r.loss = zt >= m ? log1pf(others) : (m - zt) + r.log_sum;
  r.miss = others / all;
  return r;
}

// Rows that count, in their order: token[i] = t, target_of[i] = its target; n; the pieces' numbers of rows.
// One workgroup: 8192 targets at a time, eight per thread.
__global__ void __launch_bounds__(1024) vocab_compact_kernel(const int32_t* __restrict__ target, int T, int V, int R, int pieces,
                                                             int32_t* __restrict__ token, int32_t* __restrict__ target_of,
                                                             VocabCounts* __restrict__ counts, int32_t* __restrict__ ranges) {
  __shared__ int wave_sum[16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int base = 0;
  for (int t0 = 0; t0 < T; t0 += 8192) {
    const int t = t0 + threadIdx.x * 8;
    int tg[8], mine = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      tg[i] = t + i < T ? target[t + i] : -1;
      mine += tg[i] >= 0 && tg[i] < V;
    }
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
  if (threadIdx.x == 0) counts->n = base;
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

// The rows of a piece to the front of xc (a second time behind them for `twice`), a wave per row; with the first piece also the zeros of the
// tokens left out.
template <typename T_> struct Row16 { static constexpr int N = 16 / (int)sizeof(T_); };
template <typename TX>
__global__ void __launch_bounds__(256) vocab_gather_kernel(const TX* __restrict__ x, const int32_t* __restrict__ target, const int32_t* __restrict__ token,
                                                           const int32_t* __restrict__ range, int T, int V, int d, int row0, int twice,
                                                           TX* __restrict__ xc, float* __restrict__ loss, float* __restrict__ lse, TX* __restrict__ dx) {
  const int lane = threadIdx.x & 63, r = blockIdx.x * 4 + (threadIdx.x >> 6);
  const int vecs = d / Row16<TX>::N, n = range[1];
  if (r < n) {
    const u32x4* src = reinterpret_cast<const u32x4*>(x + (long)token[row0 + r] * d);
    u32x4* dst = reinterpret_cast<u32x4*>(xc + (long)r * d);
    u32x4* again = reinterpret_cast<u32x4*>(xc + (long)(n + r) * d);
    for (int i = lane; i < vecs; i += 64) {
      const u32x4 v = src[i];
      dst[i] = v;
      if (twice) again[i] = v;
    }
  }
  if (row0 == 0 && r < T) {
    const int tg = target[r];
    if (tg < 0 || tg >= V) {
      if (lane == 0) loss[r] = lse[r] = 0.f;
      if (dx) {
        u32x4* dst = reinterpret_cast<u32x4*>(dx + (long)r * d);
        for (int i = lane; i < vecs; i += 64) dst[i] = u32x4{0u, 0u, 0u, 0u};
      }
    }
  }
}

// loss and lse of a row from its parts, a wave per row (forward only).  token: the row's token (NULL: rows are tokens).
__global__ void __launch_bounds__(256) vocab_score_kernel(const f32x2* __restrict__ stats, int parts, const float* __restrict__ z_target,
                                                          const int32_t* __restrict__ target, const int32_t* __restrict__ token,
                                                          const int32_t* __restrict__ range, int R, int V, float* __restrict__ loss, float* __restrict__ lse) {
  const int lane = threadIdx.x & 63, r = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (r >= (range ? min(range[1], R) : R)) return;
  const int t = token ? token[r] : r;
  if (!token && (target[r] < 0 || target[r] >= V)) {
    if (lane == 0) loss[t] = lse[t] = 0.f;
    return;
  }
  float m = kLowest, s = 0.f;
  for (int i = lane; i < parts; i += 64) {
    const f32x2 p = stats[(long)r * parts + i];
    join(m, s, p[0], p[1]);
  }
  join_wave(m, s);
  if (lane == 0) {
    const RowLoss l = row_loss(z_target[r], m, s);
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

__device__ __forceinline__ float row_weight(const RowOut& o, int t) { return o.token_w ? o.token_w[t] : 1.0f / (float)o.counts->n; }

// exp(z - maximum of its part) in fp16 -> G in bf16, in place, a workgroup per row.  Bound by memory: 4 bytes per element.
__global__ void __launch_bounds__(256) vocab_grad_rows_kernel(const f32x2* __restrict__ stats, int parts, int part_shift, const float* __restrict__ z_target,
                                                              int V, long ld, int twice, char* __restrict__ G, RowOut o) {
  __shared__ f32x2 lds[4];
  const int r = blockIdx.x, n = o.range[1];
  if (r >= n) return;
  const f32x2* row_stats = stats + (long)r * parts;
  float m = kLowest, s = 0.f;
  for (int i = threadIdx.x; i < parts; i += 256) join(m, s, row_stats[i][0], row_stats[i][1]);
  join_block(m, s, lds);
  const int t = o.token[r], tg = o.target_of[r];
  const RowLoss l = row_loss(z_target[r], m, s);
  const float c = row_weight(o, t), g_target = -c * l.miss;
  const bf16 g_rounded = static_cast<bf16>(g_target);
  const float rest = g_target - static_cast<float>(g_rounded);
  if (threadIdx.x == 0) {
    o.loss[t] = l.loss;
    o.lse[t] = l.lse;
    o.weighted[r] = c * l.loss;
    o.rest[r] = rest;
  }
  char* row = G + (long)r * ld * 2;
  for (int v = threadIdx.x * 8; v < ld; v += 256 * 8) {
    const f16x8 p = *reinterpret_cast<const f16x8*>(row + (long)v * 2);
    bf16x8 g;
    // eight columns lie in one part; past the width nothing was written
    const float f = v < V ? c * exp_f32((row_stats[v >> part_shift][0] - l.top) - l.log_sum) : 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) g[i] = v + i < V ? static_cast<bf16>((float)p[i] * f) : static_cast<bf16>(0.f);
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

// fp32: the logits of a piece are in Z; loss and lse, and with GRAD G in their place.
template <bool GRAD>
__global__ void __launch_bounds__(256) vocab_rows_f32_kernel(float* __restrict__ Z, int V, long ld, RowOut o) {
  __shared__ f32x2 lds[4];
  const int r = blockIdx.x;
  if (r >= o.range[1]) return;
  float* row = Z + (long)r * ld;
  const int t = o.token[r], tg = o.target_of[r];
  const float zt = row[tg];
  float m = kLowest, s = 0.f;
  for (int v = threadIdx.x * 4; v < V; v += 1024) {
    f32x4 z = *reinterpret_cast<const f32x4*>(row + v);
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
    for (int v = threadIdx.x * 4; v < ld; v += 1024) {
      f32x4 z = *reinterpret_cast<const f32x4*>(row + v);
#pragma unroll
      for (int i = 0; i < 4; ++i) z[i] = v + i >= V ? 0.f : v + i == tg ? g_target : c * exp_f32((z[i] - l.top) - l.log_sum);
      *reinterpret_cast<f32x4*>(row + v) = z;
    }
  }
}

// dx of the piece's rows: the sum of the product's parts, with what the rounding of G took off in the target's column, rounded once.
__global__ void __launch_bounds__(256) vocab_dx_kernel(const float* __restrict__ parts, int n_parts, long part_stride, const bf16* __restrict__ w, int d,
                                                       const RowOut o, bf16* __restrict__ dx) {
  const int vecs = d / 8;
  const long total = (long)o.range[1] * vecs;
  for (long i = blockIdx.x * 256L + threadIdx.x; i < total; i += gridDim.x * 256L) {
    const int r = (int)(i / vecs), c = (int)(i - (long)r * vecs) * 8;
    const float* src = parts + (long)r * d + c;
    f32x4 a = *reinterpret_cast<const f32x4*>(src), b = *reinterpret_cast<const f32x4*>(src + 4);
    for (int p = 1; p < n_parts; ++p) {
      src += part_stride;
      a += *reinterpret_cast<const f32x4*>(src);
      b += *reinterpret_cast<const f32x4*>(src + 4);
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
__global__ void __launch_bounds__(256) vocab_dx_f32_kernel(const float* __restrict__ src, int d, const RowOut o, float* __restrict__ dx) {
  const int vecs = d / 4;
  const long total = (long)o.range[1] * vecs;
  for (long i = blockIdx.x * 256L + threadIdx.x; i < total; i += gridDim.x * 256L) {
    const int r = (int)(i / vecs), c = (int)(i - (long)r * vecs) * 4;
    *reinterpret_cast<f32x4*>(dx + (long)o.token[r] * d + c) = *reinterpret_cast<const f32x4*>(src + (long)r * d + c);
  }
}

// total = sum of the weighted losses, in a fixed order, in 64 bits
__global__ void __launch_bounds__(1024) vocab_total_kernel(const float* __restrict__ weighted, const VocabCounts* __restrict__ counts, float* __restrict__ total) {
  __shared__ double lds[16];
  double s = 0.0;
  for (int i = threadIdx.x; i < counts->n; i += 1024) s += (double)weighted[i];
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) s += __shfl_xor(s, off);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < 16; ++w) s += lds[w];
    *total = (float)s;
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

}  // namespace

// Up to so many rows d_w takes a second row per token with what the rounding of G left (its product then waits for the gradient to be written,
// V * d elements, not for the matrix cores).
constexpr int kFewRows = 128;
// Forward only: up to so many rows nothing is gathered.  They are one row of tiles whether they count or not, and rows do not mix.
constexpr int kScoreAsIs = 256;

VocabPlan vocab_plan(int T, int d, int V, moe_dtype dt, moe_dtype grad_dt, int piece_rows, bool grad) {
  VocabPlan p{};
  const bool f32 = dt == MOE_F32;
  const size_t es = dtype_size(dt);
  p.R = piece_rows > 0 && piece_rows < T ? piece_rows : T;
  if (!grad && !f32) p.R = T;                              // nothing is kept per element
  p.pieces = (T + p.R - 1) / p.R;
  p.ld = (long)align_up((size_t)V, 64);
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
    p.G = take(at, R * p.ld * 4);
  } else {
    p.tiles = mfma_vocab_tiles(p.R, V, d);
    p.stats = take(at, R * p.tiles.parts * 8);
    p.z_target = take(at, R * 4);
    if (grad) p.G = take(at, copies * R * p.ld * 2);
  }
  if (grad) {
    p.weighted = take(at, rows * 4);
    p.rest = take(at, R * 4);
    if (f32) {
      const size_t one = R * d, most = (size_t)64 << 20;
      p.dx_floats = one * 6 < most ? one * 6 : one < most ? most / one * one : 0;
      p.dxc = take(at, one * 4);
      p.dx_parts = take(at, p.dx_floats * 4);
    } else {
      p.dx_floats = (size_t)mfma_vocab_dx_plan(p.R, V, d).parts * R * d;
      p.dx_parts = take(at, p.dx_floats * 4);
      p.dw_sum_used = p.pieces > 1 && grad_dt == MOE_BF16;
      if (p.dw_sum_used) p.dw_sum = take(at, (size_t)V * d * 4);
    }
  }
  p.bytes = at;
  return p;
}

int launch_vocab_loss(const VocabProblem& q, const VocabPlan& p, char* ws, hipStream_t s) {
  const bool f32 = q.dt == MOE_F32, grad = q.grad;
  const int T = q.T, d = q.d, V = q.V;
  VocabCounts* counts = reinterpret_cast<VocabCounts*>(ws + p.counts);
  int32_t* ranges = reinterpret_cast<int32_t*>(ws + p.ranges);
  int32_t* token = p.gather ? reinterpret_cast<int32_t*>(ws + p.token) : nullptr;
  int32_t* target_of = reinterpret_cast<int32_t*>(ws + p.target_of);
  float* z_target = reinterpret_cast<float*>(ws + p.z_target);
  float* stats = reinterpret_cast<float*>(ws + p.stats);
  if (!p.gather) {
    int rc = mfma_vocab_softmax(q.x, q.w, nullptr, q.target, T, V, d, nullptr, 0, stats, z_target, s);
    if (rc != MOE_OK) return rc;
    vocab_score_kernel<<<dim3(cdiv(T, 4)), dim3(256), 0, s>>>(reinterpret_cast<const f32x2*>(stats), p.tiles.parts, z_target, q.target, nullptr, nullptr, T, V,
                                                             q.loss, q.lse);
    MOE_LAUNCH_CHECK();
    return MOE_OK;
  }
  vocab_compact_kernel<<<dim3(1), dim3(1024), 0, s>>>(q.target, T, V, p.R, p.pieces, token, target_of, counts, ranges);
  MOE_LAUNCH_CHECK();
  for (int piece = 0; piece < p.pieces; ++piece) {
    const int row0 = piece * p.R, R = p.R;          // (rows past the last one: none, as the device knows)
    const int32_t* range = ranges + 2 * piece;
    const dim3 gather_grid(cdiv(piece == 0 ? T : R, 4));
    if (f32)
      vocab_gather_kernel<float><<<gather_grid, dim3(256), 0, s>>>((const float*)q.x, q.target, token, range, T, V, d, row0, 0, (float*)(ws + p.xc), q.loss,
                                                                   q.lse, (float*)(grad ? q.dx : nullptr));
    else
      vocab_gather_kernel<bf16><<<gather_grid, dim3(256), 0, s>>>((const bf16*)q.x, q.target, token, range, T, V, d, row0, p.twice, (bf16*)(ws + p.xc),
                                                                  q.loss, q.lse, (bf16*)(grad ? q.dx : nullptr));
    MOE_LAUNCH_CHECK();
    RowOut o{token + row0, target_of + row0, range, counts, q.token_w, q.loss, q.lse, reinterpret_cast<float*>(ws + p.weighted) + row0,
             reinterpret_cast<float*>(ws + p.rest)};
    const void* xc = ws + p.xc;
    const int first = piece == 0;
    int rc;
    if (f32) {
      GemmProblem g{};
      float* Z = reinterpret_cast<float*>(ws + p.G);
      g.offsets = range; g.E = 1; g.mode = 0; g.M = R;
      g.A = xc; g.a_rs = d; g.a_cs = 1;
      g.B = q.w; g.b_rs = 1; g.b_cs = d;
      g.C = Z; g.ldc = p.ld; g.N = (int)align_up((size_t)V, 16); g.K = d; g.b_rows = V;
      rc = launch_gemm_f32(g, s);
      if (rc != MOE_OK) return rc;
      if (!grad) {
        vocab_rows_f32_kernel<false><<<dim3(R), dim3(256), 0, s>>>(Z, V, p.ld, o);
        MOE_LAUNCH_CHECK();
        continue;
      }
      vocab_rows_f32_kernel<true><<<dim3(R), dim3(256), 0, s>>>(Z, V, p.ld, o);
      MOE_LAUNCH_CHECK();
      GemmProblem h{};
      float* dxc = reinterpret_cast<float*>(ws + p.dxc);
      h.offsets = range; h.E = 1; h.mode = 0; h.M = R;
      h.A = Z; h.a_rs = p.ld; h.a_cs = 1;
      h.B = q.w; h.b_rs = d; h.b_cs = 1;
      h.C = dxc; h.ldc = d; h.N = d; h.K = V;
      h.scratch = reinterpret_cast<float*>(ws + p.dx_parts); h.scratch_floats = p.dx_floats;
      rc = launch_gemm_f32(h, s);
      if (rc != MOE_OK) return rc;
      vocab_dx_f32_kernel<<<dim3(blocks_for((long)R * d / 4)), dim3(256), 0, s>>>(dxc, d, o, static_cast<float*>(q.dx));
      MOE_LAUNCH_CHECK();
      GemmProblem k{};
      k.offsets = range; k.E = 1; k.mode = 1; k.M = (int)p.ld; k.c_rows = V;
      k.A = Z; k.a_rs = 1; k.a_cs = p.ld;
      k.B = xc; k.b_rs = d; k.b_cs = 1;
      k.C = q.d_w; k.ldc = d; k.N = d; k.K = R;
      k.accumulate = q.accumulate || !first;
      rc = launch_gemm_f32(k, s);
      if (rc != MOE_OK) return rc;
      continue;
    }
    rc = mfma_vocab_softmax(xc, q.w, range + 1, target_of + row0, R, V, d, grad ? ws + p.G : nullptr, p.ld, stats, z_target, s);
    if (rc != MOE_OK) return rc;
    if (!grad) {
      vocab_score_kernel<<<dim3(cdiv(R, 4)), dim3(256), 0, s>>>(reinterpret_cast<const f32x2*>(stats), p.tiles.parts, z_target, target_of + row0, token + row0, range, R,
                                                               V, q.loss, q.lse);
      MOE_LAUNCH_CHECK();
      continue;
    }
    vocab_grad_rows_kernel<<<dim3(R), dim3(256), 0, s>>>(reinterpret_cast<const f32x2*>(stats), p.tiles.parts, p.tiles.shift, z_target, V, p.ld,
                                                         p.twice, ws + p.G, o);
    MOE_LAUNCH_CHECK();
    float* dx_parts = reinterpret_cast<float*>(ws + p.dx_parts);
    rc = mfma_vocab_dx(ws + p.G, p.ld, q.w, range + 1, R, V, d, dx_parts, s);
    if (rc != MOE_OK) return rc;
    vocab_dx_kernel<<<dim3(blocks_for((long)R * d / 8)), dim3(256), 0, s>>>(dx_parts, mfma_vocab_dx_plan(R, V, d).parts, (long)R * d, (const bf16*)q.w, d, o,
                                                                           (bf16*)q.dx);
    MOE_LAUNCH_CHECK();
    if (p.dw_sum_used)
      rc = mfma_vocab_dw(ws + p.G, p.ld, xc, range, R, V, d, ws + p.dw_sum, MOE_F32, !first, s);
    else
      rc = mfma_vocab_dw(ws + p.G, p.ld, xc, p.twice ? ranges + 2 : range, p.twice ? 2 * R : R, V, d, q.d_w, q.grad_dt, q.accumulate || !first, s);
    if (rc != MOE_OK) return rc;
  }
  if (!grad) return MOE_OK;
  if (p.dw_sum_used) {
    const long vecs = (long)V * d / 8;
    vocab_dw_round_kernel<<<dim3(blocks_for(vecs)), dim3(256), 0, s>>>(reinterpret_cast<const float*>(ws + p.dw_sum), vecs, q.accumulate, (bf16*)q.d_w);
    MOE_LAUNCH_CHECK();
  }
  vocab_total_kernel<<<dim3(1), dim3(1024), 0, s>>>(reinterpret_cast<const float*>(ws + p.weighted), counts, q.total);
  MOE_LAUNCH_CHECK();
  return MOE_OK;
}

}  // namespace moe
