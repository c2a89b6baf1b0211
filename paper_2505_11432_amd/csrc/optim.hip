// Gradient norm, clipping and the AdamW update over a list of tensors in one launch each (the norm and the clipped gradients two).
//   norm = sqrt(sum g^2),  coef = min(1, max_norm / (norm + 1e-6)),  out = coef g
//   g' = coef g,  m = b1 m + (1 - b1) g',  v = b2 v + (1 - b2) g'^2,
//   p = p (1 - lr wd) - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps)
// All of it is bound by memory (3 and 15 operations per element).  The tensors are one sequence of elements, cut into equal ranges for the
// workgroups: one search in the table per workgroup, and tensors of any size fill the chip alike.
//
// Alignment: a tensor may begin at any element.  A range is walked four elements at a time from the first one that is a multiple of four from
// the tensor's 16-byte aligned element on; loads and stores of the other lists may then be unaligned, which the hardware takes.
//
// The norm is summed in 64 bits (squares of single-precision numbers neither overflow nor vanish there; the conversion and the sum hide behind
// the loads) and in a fixed order: a sum per workgroup, and every workgroup of the second launch adds those up in the same order.  The second
// launch walks each range backwards: what the first one read last is still in the Infinity Cache (256 MB).
#include "moe_common.h"
#include "optim.h"

namespace moe {
namespace {

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef f32x4 f32x4_u __attribute__((aligned(4)));
typedef bf16x4 bf16x4_u __attribute__((aligned(2)));

template <typename T> struct Quad;
template <> struct Quad<float> {
  __device__ static __forceinline__ f32x4 load(const float* p) { return *reinterpret_cast<const f32x4_u*>(p); }
  __device__ static __forceinline__ void store(float* p, f32x4 v) { *reinterpret_cast<f32x4_u*>(p) = v; }
};
template <> struct Quad<bf16> {
  __device__ static __forceinline__ f32x4 load(const bf16* p) { return __builtin_convertvector(*reinterpret_cast<const bf16x4_u*>(p), f32x4); }
  __device__ static __forceinline__ void store(bf16* p, f32x4 v) { *reinterpret_cast<bf16x4_u*>(p) = __builtin_convertvector(v, bf16x4); }
};

// elements in front of the first whole group of four
template <typename T> __device__ __forceinline__ long misfit(const T* p) {
  return (long)((4 - (reinterpret_cast<uintptr_t>(p) / sizeof(T) & 3)) & 3);
}

// last entry whose first element is at or before `at`
template <typename Entry> __device__ __forceinline__ int find(const Entry* __restrict__ table, int n, long at) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (table[mid].first <= at) lo = mid; else hi = mid;
  }
  return lo;
}

constexpr int kThreads = 256;

template <typename T> __device__ __forceinline__ double square_sum(const T* __restrict__ g, long n) {
  double s0 = 0, s1 = 0;
  const long head = min(misfit(g), n), quads = (n - head) >> 2;
  if (threadIdx.x < head) {
    const double v = (double)to_f32(g[threadIdx.x]);
    s0 += v * v;
  }
  const T* q = g + head;
  constexpr int U = 4;
  long i = threadIdx.x;
  for (; i + (U - 1) * kThreads < quads; i += U * kThreads) {
    f32x4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = Quad<T>::load(q + 4 * (i + u * kThreads));
#pragma unroll
    for (int u = 0; u < U; ++u) {
      s0 = fma((double)v[u][0], (double)v[u][0], s0);
      s1 = fma((double)v[u][1], (double)v[u][1], s1);
      s0 = fma((double)v[u][2], (double)v[u][2], s0);
      s1 = fma((double)v[u][3], (double)v[u][3], s1);
    }
  }
  for (; i < quads; i += kThreads) {
    const f32x4 v = Quad<T>::load(q + 4 * i);
#pragma unroll
    for (int c = 0; c < 4; ++c) s1 = fma((double)v[c], (double)v[c], s1);
  }
  const long tail = head + 4 * quads + threadIdx.x;
  if (tail < n) {
    const double v = (double)to_f32(g[tail]);
    s0 += v * v;
  }
  return s0 + s1;
}

__device__ __forceinline__ double block_sum(double s, double (&lds)[4]) {
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) s += __shfl_xor(s, off);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
  __syncthreads();
  return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

__global__ void __launch_bounds__(kThreads) norm_parts_kernel(const ClipEntry* __restrict__ table, int n, long total, long per, double* __restrict__ parts) {
  __shared__ double lds[4];
  long at = blockIdx.x * per;
  const long end = min(at + per, total);
  double s = 0;
  for (int e = at < end ? find(table, n, at) : n; at < end; ++e) {
    const ClipEntry t = table[e];
    const long stop = min(end, table[e + 1].first), k = stop - at;
    if (k <= 0) continue;
    if (t.dt == MOE_F32) s += square_sum(static_cast<const float*>(t.g) + (at - t.first), k);
    else s += square_sum(static_cast<const bf16*>(t.g) + (at - t.first), k);
    at = stop;
  }
  s = block_sum(s, lds);
  if (threadIdx.x == 0) parts[blockIdx.x] = s;
}

// the same sum, in the same order, by every workgroup that asks
__device__ __forceinline__ double norm_of(const double* __restrict__ parts, int n_parts, double (&lds)[4]) {
  double s = 0;
  for (int i = threadIdx.x; i < n_parts; i += kThreads) s += parts[i];
  return sqrt(block_sum(s, lds));
}
__device__ __forceinline__ float clip_coef(double norm, double max_norm) {
  const double c = max_norm / (norm + 1e-6);
  return c < 1.0 ? (float)c : c == c ? 1.0f : (float)c;          // (a norm that is no number gives a factor that is none)
}

// four elements at a time, the last ones first
template <typename T> __device__ __forceinline__ void scale_range(const T* g, T* out, long n, float c) {
  const long head = min(misfit(g), n), quads = (n - head) >> 2, tail = head + 4 * quads + threadIdx.x;
  if (tail < n) out[tail] = from_f32<T>(c * to_f32(g[tail]));
  const T* q = g + head;
  T* o = out + head;
  constexpr int U = 4;
  long i = quads - 1 - threadIdx.x;
  for (; i - (U - 1) * kThreads >= 0; i -= U * kThreads) {
    f32x4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = Quad<T>::load(q + 4 * (i - u * kThreads));
#pragma unroll
    for (int u = 0; u < U; ++u) Quad<T>::store(o + 4 * (i - u * kThreads), v[u] * c);
  }
  for (; i >= 0; i -= kThreads) Quad<T>::store(o + 4 * i, Quad<T>::load(q + 4 * i) * c);
  if (threadIdx.x < head) out[threadIdx.x] = from_f32<T>(c * to_f32(g[threadIdx.x]));
}

__global__ void __launch_bounds__(kThreads) clip_kernel(const ClipEntry* __restrict__ table, int n, long total, long per, const double* __restrict__ parts,
                                                        int n_parts, double max_norm, int write, float* __restrict__ norm, float* __restrict__ coef) {
  __shared__ double lds[4];
  const double full = norm_of(parts, n_parts, lds);
  const float c = clip_coef(full, max_norm);
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    *norm = (float)full;
    *coef = c;
  }
  if (!write) return;
  const long begin = blockIdx.x * per;
  long end = min(begin + per, total);
  for (int e = begin < end ? find(table, n, end - 1) : 0; begin < end; --e) {
    const ClipEntry t = table[e];
    const long start = max(begin, (long)t.first), k = end - start;
    if (k <= 0) continue;
    const long off = start - t.first;
    // gradients in place that are within the limit stay as they are
    if (t.out && !(t.out == t.g && c == 1.0f)) {
      if (t.dt == MOE_F32) scale_range(static_cast<const float*>(t.g) + off, static_cast<float*>(t.out) + off, k, c);
      else scale_range(static_cast<const bf16*>(t.g) + off, static_cast<bf16*>(t.out) + off, k, c);
    }
    end = start;
  }
}

struct AdamwScalars { float coef, b1, g1, b2, g2, keep, lr, r1, r2, eps; };

__device__ __forceinline__ void adamw_one(float& p, float g, float& m, float& v, const AdamwScalars& a) {
  g *= a.coef;
  m = m * a.b1 + g * a.g1;
  v = v * a.b2 + g * g * a.g2;
  p = p * a.keep - a.lr * (m * a.r1) / (sqrtf(v * a.r2) + a.eps);
}

template <typename TG>
__device__ __forceinline__ void adamw_range(float* __restrict__ p, const TG* __restrict__ g, float* __restrict__ m, float* __restrict__ v, bf16* __restrict__ w,
                                            long n, const AdamwScalars& a) {
  const long head = min(misfit(p), n), quads = (n - head) >> 2;
  auto single = [&](long i) __attribute__((always_inline)) {
    float pi = p[i], mi = m[i], vi = v[i];
    adamw_one(pi, to_f32(g[i]), mi, vi, a);
    p[i] = pi;
    m[i] = mi;
    v[i] = vi;
    if (w) w[i] = from_f32<bf16>(pi);
  };
  if (threadIdx.x < head) single(threadIdx.x);
  constexpr int U = 2;
  long i = threadIdx.x;
  auto group = [&](auto count) __attribute__((always_inline)) {
    constexpr int N = decltype(count)::value;
    f32x4 pv[N], gv[N], mv[N], vv[N];
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const long at = head + 4 * (i + u * kThreads);
      gv[u] = Quad<TG>::load(g + at);
      mv[u] = Quad<float>::load(m + at);
      vv[u] = Quad<float>::load(v + at);
      pv[u] = Quad<float>::load(p + at);
    }
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const long at = head + 4 * (i + u * kThreads);
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        float pi = pv[u][c], mi = mv[u][c], vi = vv[u][c];
        adamw_one(pi, gv[u][c], mi, vi, a);
        pv[u][c] = pi;
        mv[u][c] = mi;
        vv[u][c] = vi;
      }
      Quad<float>::store(p + at, pv[u]);
      Quad<float>::store(m + at, mv[u]);
      Quad<float>::store(v + at, vv[u]);
      if (w) Quad<bf16>::store(w + at, pv[u]);
    }
  };
  for (; i + (U - 1) * kThreads < quads; i += U * kThreads) group(std::integral_constant<int, U>());
  for (; i < quads; i += kThreads) group(std::integral_constant<int, 1>());
  const long tail = head + 4 * quads + threadIdx.x;
  if (tail < n) single(tail);
}

// base^t in 64 bits by squaring
__device__ __forceinline__ double power(double base, unsigned t) {
  double r = 1.0;
  for (; t; t >>= 1, base *= base)
    if (t & 1) r *= base;
  return r;
}

// Every workgroup reads the step count before any has changed it: the last one to finish writes the new one.
template <typename TG>
__global__ void __launch_bounds__(kThreads) adamw_kernel(const AdamwEntry* __restrict__ table, int n, long total, long per, const float* __restrict__ lr,
                                                         int32_t* step, const float* __restrict__ coef, AdamwHyper h, unsigned* done) {
  const int t = *step + 1;
  AdamwScalars a;
  a.coef = coef ? *coef : 1.0f;
  a.b1 = (float)h.beta1;
  a.g1 = (float)(1.0 - h.beta1);
  a.b2 = (float)h.beta2;
  a.g2 = (float)(1.0 - h.beta2);
  a.lr = *lr;
  a.keep = (float)(1.0 - (double)a.lr * h.weight_decay);
  a.r1 = (float)(1.0 / (1.0 - power(h.beta1, (unsigned)t)));
  a.r2 = (float)(1.0 / (1.0 - power(h.beta2, (unsigned)t)));
  a.eps = (float)h.eps;
  long at = blockIdx.x * per;
  const long end = min(at + per, total);
  for (int e = at < end ? find(table, n, at) : n; at < end; ++e) {
    const AdamwEntry q = table[e];
    const long stop = min(end, table[e + 1].first), k = stop - at, off = at - q.first;
    if (k <= 0) continue;
    adamw_range(static_cast<float*>(q.p) + off, static_cast<const TG*>(q.g) + off, static_cast<float*>(q.m) + off, static_cast<float*>(q.v) + off,
                q.w ? static_cast<bf16*>(q.w) + off : nullptr, k, a);
    at = stop;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    __threadfence();
    if (atomicAdd(done, 1u) == gridDim.x - 1) {
      *step = t;
      *done = 0;
    }
  }
}

// Workgroups and elements of a range: ranges of whole groups, up to 2048 of them (eight per CU).
struct Cut { int blocks; long per; };
Cut cut(long total, long least) {
  long per = (total + 2047) / 2048;
  per = per < least ? least : (per + 1023) / 1024 * 1024;
  const long blocks = (total + per - 1) / per;
  return {blocks < 1 ? 1 : (int)blocks, per};
}

}  // namespace

int launch_grad_clip(const ClipEntry* table, int n, long total, double max_norm, int write, float* norm, float* coef, double* parts, hipStream_t s) {
  const Cut c = cut(total, 2048);
  norm_parts_kernel<<<dim3(c.blocks), dim3(kThreads), 0, s>>>(table, n, total, c.per, parts);
  MOE_LAUNCH_CHECK();
  clip_kernel<<<dim3(write ? c.blocks : 1), dim3(kThreads), 0, s>>>(table, n, total, c.per, parts, c.blocks, max_norm, write, norm, coef);
  MOE_LAUNCH_CHECK();
  return MOE_OK;
}

int launch_adamw(const AdamwEntry* table, int n, long total, moe_dtype grad_dt, const float* lr, int32_t* step, const float* coef, const AdamwHyper& h,
                 unsigned* done, hipStream_t s) {
  const Cut c = cut(total, 2048);
  if (grad_dt == MOE_F32) adamw_kernel<float><<<dim3(c.blocks), dim3(kThreads), 0, s>>>(table, n, total, c.per, lr, step, coef, h, done);
  else adamw_kernel<bf16><<<dim3(c.blocks), dim3(kThreads), 0, s>>>(table, n, total, c.per, lr, step, coef, h, done);
  MOE_LAUNCH_CHECK();
  return MOE_OK;
}

}  // namespace moe
