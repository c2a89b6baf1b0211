// Gradient norm, clipping and the AdamW update over a list of tensors in one launch each (the norm and the clipped gradients two).
//   norm = sqrt(sum g^2),  coef = min(1, max_norm / (norm + 1e-6)),  out = coef g
//   g' = coef g,  m = b1 m + (1 - b1) g',  v = b2 v + (1 - b2) g'^2,
//   p = p (1 - lr wd) - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps)
// All of it is bound by memory (3 and 15 operations per element).
//
// The tensors are one sequence of chunks, 2 KB each (AdamW: 512 elements), which the workgroups take in turn, a few at a time, so that all of
// them stay near one another in memory.  A tensor takes one chunk more than it fills, for what its entry and its ends cost.  Probe of the
// access patterns on 1.7 GB per list (TB/s; a contiguous range per workgroup, in turn; 2048 workgroups, 32768): read 6.0, 6.3; read and write 5.05,
// 5.57; AdamW's streams 5.02, 5.22.
// What is not read again is read and written past the caches (nontemporal): read 7.0, read and write 6.0, AdamW's streams 5.4.
//
// Alignment: a tensor may begin at any element.  Its elements in front of the first whole 128-byte line go one by one; chunks begin at lines.  The
// other lists of an update may then be unaligned, which the hardware takes.
//
// The norm is summed in 64 bits (squares of single-precision numbers neither overflow nor vanish there; the conversion and the sum hide behind
// the loads) and in a fixed order: a sum per workgroup, and every workgroup of the second launch adds those up in the same order.  (The second launch
// from the last chunk on, which the Infinity Cache might still hold, is slower: 20 M elements 37.6 us, from the first on 32.4; 300 M 357, 345.)
#include <type_traits>

#include "moe_common.h"
#include "optim.h"

namespace moe {
namespace {

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(8))) float f32x8;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef f32x4 f32x4_u __attribute__((aligned(4)));
typedef bf16x4 bf16x4_u __attribute__((aligned(2)));
typedef bf16x8 bf16x8_u __attribute__((aligned(2)));

// N elements as floats
template <typename T, int N> struct Piece;
template <> struct Piece<float, 4> {
  typedef f32x4 values;
  __device__ static __forceinline__ f32x4 load(const float* p) { return __builtin_nontemporal_load(reinterpret_cast<const f32x4_u*>(p)); }
  __device__ static __forceinline__ f32x4 load_kept(const float* p) { return *reinterpret_cast<const f32x4_u*>(p); }
  __device__ static __forceinline__ void store(float* p, f32x4 v) { __builtin_nontemporal_store(v, reinterpret_cast<f32x4_u*>(p)); }
};
template <> struct Piece<bf16, 4> {
  typedef f32x4 values;
  __device__ static __forceinline__ f32x4 load(const bf16* p) {
    return __builtin_convertvector(__builtin_nontemporal_load(reinterpret_cast<const bf16x4_u*>(p)), f32x4);
  }
  __device__ static __forceinline__ void store(bf16* p, f32x4 v) {
    __builtin_nontemporal_store(__builtin_convertvector(v, bf16x4), reinterpret_cast<bf16x4_u*>(p));
  }
};
template <> struct Piece<bf16, 8> {
  typedef f32x8 values;
  __device__ static __forceinline__ f32x8 load(const bf16* p) {
    return __builtin_convertvector(__builtin_nontemporal_load(reinterpret_cast<const bf16x8_u*>(p)), f32x8);
  }
  __device__ static __forceinline__ f32x8 load_kept(const bf16* p) { return __builtin_convertvector(*reinterpret_cast<const bf16x8_u*>(p), f32x8); }
  __device__ static __forceinline__ void store(bf16* p, f32x8 v) {
    __builtin_nontemporal_store(__builtin_convertvector(v, bf16x8), reinterpret_cast<bf16x8_u*>(p));
  }
};
template <typename T> using Wide = Piece<T, 16 / (int)sizeof(T)>;

// elements in front of the first whole line
template <typename T> __device__ __forceinline__ long misfit(const T* p) {
  constexpr int LINE = 128 / sizeof(T);
  return (long)((LINE - (reinterpret_cast<uintptr_t>(p) / sizeof(T) & (LINE - 1))) & (LINE - 1));
}
__device__ __forceinline__ long misfit(const ClipEntry& e) {
  return e.dt == MOE_F32 ? misfit(static_cast<const float*>(e.g)) : misfit(static_cast<const bf16*>(e.g));
}
__device__ __forceinline__ long misfit(const AdamwEntry& e) { return misfit(static_cast<const float*>(e.p)); }

// The tensor that holds chunk `at`: 64 entries at a time, a lane each.
template <typename Entry> __device__ __forceinline__ int find(const Entry* __restrict__ table, int n, int at) {
  const int lane = threadIdx.x & 63;
  int lo = 0, len = n;
  while (len > 1) {
    const int step = (len + 63) / 64;
    const unsigned long long before = __ballot(lane * step < len && first_chunk(table, lo + lane * step) <= at);
    const int k = __popcll(before) - 1;
    lo += k * step;
    len = min(step, len - k * step);
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

// Takes groups of `per` chunks in turn with the other workgroups and calls body(entry, first element, number
// of elements) for the part of every tensor that lies in them.  Only the first part of a tensor begins in front of a line, and only the last one
// ends anywhere.
template <typename Entry, typename Body> __device__ __forceinline__ void for_parts(const Entry* __restrict__ table, int n, int per, Body body) {
  const int chunks = first_chunk(table, n), groups = (chunks + per - 1) / per;
  int e = 0, chunk = 0, next = 0;          // the open tensor and its chunks
  Entry t{};
  long numel = 0, head = 0;
  for (int g = blockIdx.x; g < groups; g += gridDim.x) {
    int at = g * per;
    const int end = min(at + per, chunks);
    while (at < end) {
      if (at < chunk || at >= next) {
        e = at == next && next != 0 ? e + 1 : find(table, n, at);
        chunk = first_chunk(table, e);
        next = first_chunk(table, e + 1);
        t = table[e];
        numel = table[e + 1].first - t.first;
        head = misfit(t);
      }
      const long size = chunk_elements(t);
      const int stop = min(end, next);
      const long lo = at == chunk ? 0 : min((at - chunk) * size + head, numel), hi = min((stop - chunk) * size + head, numel);
      if (lo < hi) body(t, lo, hi - lo);
      at = stop;
    }
  }
}

constexpr int kThreads = 256;

// f(first element) for pieces of N elements from the first line on, U of them in flight per thread, and single(element) for the others
template <int N, int U, typename T, typename Single, typename Pieces>
__device__ __forceinline__ void walk(const T* p, long n, Single single, Pieces pieces) {
  const long head = min(misfit(p), n), count = (n - head) / N, tail = head + N * count + threadIdx.x;
  if (threadIdx.x < head) single((long)threadIdx.x);
  for (long i = threadIdx.x; i < count; i += U * kThreads) pieces(head + N * i, (int)min((count - i + kThreads - 1) / kThreads, (long)U));
  if (tail < n) single(tail);
}

template <bool KEEP, typename T> __device__ __forceinline__ double square_sum(const T* __restrict__ g, long n) {
  typedef Wide<T> P;
  constexpr int N = 16 / (int)sizeof(T), U = 4;
  double sum[2] = {0, 0};
  walk<N, U>(g, n,
             [&](long i) __attribute__((always_inline)) {
               const double v = (double)to_f32(g[i]);
               sum[0] = fma(v, v, sum[0]);
             },
             [&](long at, int count) __attribute__((always_inline)) {
               typename P::values v[U];
#pragma unroll
               for (int u = 0; u < U; ++u) {
                 v[u] = typename P::values{};
                 if (u < count) v[u] = KEEP ? P::load_kept(g + at + N * u * kThreads) : P::load(g + at + N * u * kThreads);
               }
#pragma unroll
               for (int u = 0; u < U; ++u)
#pragma unroll
                 for (int c = 0; c < N; ++c) sum[c & 1] = fma((double)v[u][c], (double)v[u][c], sum[c & 1]);
             });
  return sum[0] + sum[1];
}

__device__ __forceinline__ double block_sum(double s, double (&lds)[4]) {
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) s += __shfl_xor(s, off);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
  __syncthreads();
  return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

// (eight workgroups of every CU at a time, as many as are launched).  KEEP: the second launch finds them in the Infinity Cache.
template <bool KEEP>
__global__ void __launch_bounds__(kThreads, 8) norm_parts_kernel(const ClipEntry* __restrict__ table, int n, int per, double* __restrict__ parts) {
  __shared__ double lds[4];
  double s = 0;
  for_parts(table, n, per, [&](const ClipEntry& t, long first, long k) __attribute__((always_inline)) {
    if (t.dt == MOE_F32) s += square_sum<KEEP>(static_cast<const float*>(t.g) + first, k);
    else s += square_sum<KEEP>(static_cast<const bf16*>(t.g) + first, k);
  });
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

template <typename T> __device__ __forceinline__ void scale_range(const T* g, T* out, long n, float c) {
  typedef Wide<T> P;
  constexpr int N = 16 / (int)sizeof(T), U = 4;
  walk<N, U>(g, n, [&](long i) __attribute__((always_inline)) { out[i] = from_f32<T>(c * to_f32(g[i])); },
             [&](long at, int count) __attribute__((always_inline)) {
               typename P::values v[U];
#pragma unroll
               for (int u = 0; u < U; ++u)
                 if (u < count) v[u] = P::load(g + at + N * u * kThreads);
#pragma unroll
               for (int u = 0; u < U; ++u)
                 if (u < count) P::store(out + at + N * u * kThreads, v[u] * c);
             });
}

__global__ void __launch_bounds__(kThreads, 8) clip_kernel(const ClipEntry* __restrict__ table, int n, int per, const double* __restrict__ parts, int n_parts,
                                                           double max_norm, int write, float* __restrict__ norm, float* __restrict__ coef) {
  __shared__ double lds[4];
  const double full = norm_of(parts, n_parts, lds);
  const float c = clip_coef(full, max_norm);
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    *norm = (float)full;
    *coef = c;
  }
  if (!write) return;
  for_parts(table, n, per, [&](const ClipEntry& t, long first, long k) __attribute__((always_inline)) {
    // gradients in place that are within the limit stay as they are
    if (!t.out || (t.out == t.g && c == 1.0f)) return;
    if (t.dt == MOE_F32) scale_range(static_cast<const float*>(t.g) + first, static_cast<float*>(t.out) + first, k, c);
    else scale_range(static_cast<const bf16*>(t.g) + first, static_cast<bf16*>(t.out) + first, k, c);
  });
}

struct AdamwScalars { float coef, b1, g1, b2, g2, keep, lr, r1, r2, eps; };

// Which products are fused is written out, so that an element's bits do not depend on whether it is taken alone or with its neighbours (that is, on where its
// tensor begins).
__device__ __forceinline__ void adamw_one(float& p, float g, float& m, float& v, const AdamwScalars& a) {
#pragma clang fp contract(off)
  g *= a.coef;
  m = __builtin_fmaf(g, a.g1, m * a.b1);
  v = __builtin_fmaf(v, a.b2, g * g * a.g2);
  p = __builtin_fmaf(p, a.keep, -(a.lr * (m * a.r1) / (sqrtf(v * a.r2) + a.eps)));
}

template <typename TG>
__device__ __forceinline__ void adamw_range(float* __restrict__ p, const TG* __restrict__ g, float* __restrict__ m, float* __restrict__ v, bf16* __restrict__ w,
                                            long n, const AdamwScalars& a) {
  typedef Piece<float, 4> P;
  constexpr int U = 2;
  walk<4, U>(p, n,
             [&](long i) __attribute__((always_inline)) {
               float pi = p[i], mi = m[i], vi = v[i];
               adamw_one(pi, to_f32(g[i]), mi, vi, a);
               p[i] = pi;
               m[i] = mi;
               v[i] = vi;
               if (w) w[i] = from_f32<bf16>(pi);
             },
             [&](long at, int count) __attribute__((always_inline)) {
               f32x4 pv[U], gv[U], mv[U], vv[U];
#pragma unroll
               for (int u = 0; u < U; ++u)
                 if (u < count) {
                   const long i = at + 4 * u * kThreads;
                   gv[u] = Piece<TG, 4>::load(g + i);
                   mv[u] = P::load(m + i);
                   vv[u] = P::load(v + i);
                   pv[u] = P::load(p + i);
                 }
#pragma unroll
               for (int u = 0; u < U; ++u)
                 if (u < count) {
                   const long i = at + 4 * u * kThreads;
#pragma unroll
                   for (int c = 0; c < 4; ++c) {
                     float pi = pv[u][c], mi = mv[u][c], vi = vv[u][c];
                     adamw_one(pi, gv[u][c], mi, vi, a);
                     pv[u][c] = pi;
                     mv[u][c] = mi;
                     vv[u][c] = vi;
                   }
                   P::store(p + i, pv[u]);
                   P::store(m + i, mv[u]);
                   P::store(v + i, vv[u]);
                   if (w) Piece<bf16, 4>::store(w + i, pv[u]);
                 }
             });
}

// base^t in 64 bits by squaring
__device__ __forceinline__ double power(double base, unsigned t) {
  double r = 1.0;
  for (; t; t >>= 1, base *= base)
    if (t & 1) r *= base;
  return r;
}

constexpr int kShards = 16, kShardWords = 32;              // a line each
static_assert((kShards + 1) * kShardWords * 4 <= MOE_ADAMW_WS_BYTES, "the workspace holds the counters");

struct Mixed {};                         // gradients of both types (optim.h)

// Every workgroup reads the step count before any has changed it: the last one to finish writes the new one.
template <typename TG>
__global__ void __launch_bounds__(kThreads) adamw_kernel(const AdamwEntry* __restrict__ table, int n, int per, const float* __restrict__ lr, int32_t* step,
                                                         const float* __restrict__ coef, AdamwHyper h, unsigned* done) {
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
  const bool left_out = a.coef != a.coef;      // (looked at behind the table, whose reads do not wait for the factor then)
  for_parts(table, n, per, [&](const AdamwEntry& q, long first, long k) __attribute__((always_inline)) {
    if (left_out) return;
    auto range = [&](auto* g) __attribute__((always_inline)) {
      adamw_range(static_cast<float*>(q.p) + first, g + first, static_cast<float*>(q.m) + first, static_cast<float*>(q.v) + first,
                  q.w ? static_cast<bf16*>(q.w) + first : nullptr, k, a);
    };
    if constexpr (std::is_same_v<TG, Mixed>) {
      const uintptr_t at = reinterpret_cast<uintptr_t>(q.g);
      if (at & kBf16Gradient) range(reinterpret_cast<const bf16*>(at - kBf16Gradient));
      else range(static_cast<const float*>(q.g));
    } else {
      range(static_cast<const TG*>(q.g));
    }
  });
  if (left_out) return;                        // (every workgroup: the counters stay cleared)
  __syncthreads();
  if (threadIdx.x == 0) {
    // (no fence: what counts is that this workgroup has read the step, which the values above have needed; a fence would write back its L2)
    // Counters on one address take a workgroup's turn each, 10 ns: every 16th workgroup shares one, and who fills it counts in the last.
    const unsigned shard = blockIdx.x % kShards, members = (gridDim.x + kShards - 1 - shard) / kShards, shards = min(gridDim.x, (unsigned)kShards);
    if (atomicAdd(done + shard * kShardWords, 1u) == members - 1) {
      done[shard * kShardWords] = 0;
      if (atomicAdd(done + kShards * kShardWords, 1u) == shards - 1) {
        done[kShards * kShardWords] = 0;
        *step = t;
      }
    }
  }
}

// How many chunks a workgroup takes at a time, and how many workgroups: about so many chunks are there, at most `most` workgroups run.
struct Cut { unsigned blocks; int per; };
Cut cut(long chunks, int per, long most) {
  // small lists: four each (460 thousand elements of AdamW in 1, 2, 4, 8: 7.3, 6.35, 6.4, 7.5 us)
  if (chunks < 1024) per = 4;
  else if (chunks < 2048L * per) per = (int)((chunks + 2047) / 2048);
  const long blocks = (chunks + per - 1) / per;
  return {(unsigned)(blocks < 1 ? 1 : blocks < most ? blocks : most), per};
}

}  // namespace

int launch_grad_clip(const ClipEntry* table, int n, long total, double max_norm, int write, float* norm, float* coef, double* parts, hipStream_t s) {
  // The host does not know the types: chunks as if all were single precision.  Eight at a time, 64 in the longest lists: 300 M elements by 4, 8, 16 chunks
  // 374, 329, 334 us, 20 M 34.8, 32.3, 32.4; 1.4 G by 32, 64, 128 2985, 2925, 2915.
  const long chunks = total / (kChunkBytes / 4) + n;
  const Cut c = cut(chunks, chunks < (2 << 20) ? 8 : 64, kNormParts);
  // Where the second launch may find some of them in the Infinity Cache, reads are not made past the caches: 60 M elements 124 -> 115 us, 300 M (660 MB)
  // 354 -> 340; but 1.4 G (5.6 GB) 2926 -> 3000.
  if (write && total <= (512L << 20)) norm_parts_kernel<true><<<dim3(c.blocks), dim3(kThreads), 0, s>>>(table, n, c.per, parts);
  else norm_parts_kernel<false><<<dim3(c.blocks), dim3(kThreads), 0, s>>>(table, n, c.per, parts);
  MOE_LAUNCH_CHECK();
  clip_kernel<<<dim3(write ? c.blocks : 1), dim3(kThreads), 0, s>>>(table, n, c.per, parts, (int)c.blocks, max_norm, write, norm, coef);
  MOE_LAUNCH_CHECK();
  return MOE_OK;
}

int launch_adamw(const AdamwEntry* table, int n, long total, moe_dtype grad_dt, const float* lr, int32_t* step, const float* coef, const AdamwHyper& h,
                 unsigned* done, hipStream_t s) {
  // four chunks, 2048 elements, at a time, two pieces per thread: 400 M elements by 2, 4, 8, 16 chunks 1965, 1925, 2045, 2130 us, 20 M 102, 102, 112, 120
  const Cut c = cut(total / kAdamwChunk + 2L * n, 4, 1L << 20);
  if (grad_dt == MOE_F32) adamw_kernel<float><<<dim3(c.blocks), dim3(kThreads), 0, s>>>(table, n, c.per, lr, step, coef, h, done);
  else if (grad_dt == MOE_BF16) adamw_kernel<bf16><<<dim3(c.blocks), dim3(kThreads), 0, s>>>(table, n, c.per, lr, step, coef, h, done);
  else adamw_kernel<Mixed><<<dim3(c.blocks), dim3(kThreads), 0, s>>>(table, n, c.per, lr, step, coef, h, done);
  MOE_LAUNCH_CHECK();
  return MOE_OK;
}

}  // namespace moe
