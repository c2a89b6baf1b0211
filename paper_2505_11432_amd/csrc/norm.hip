// The end of one block and the start of the next on the residual stream, and their gradients, each row in one piece.
//   n = y / rms(y) * w_after  (or y),  out = alpha x + gate * n  (or + n),  h = out / rms(out) * w_before
//   rms(v) = sqrt(mean v^2 + eps);  h is made from `out` as it is kept (rounded), which is what the backward pass reads again.
// Backward, with unit(v) = v / rms(v) and back(v, u) = (u - unit(v) mean(u unit(v))) / rms(v):
//   g = d_out + back(out, d_h w_before),  d_w_before = sum d_h unit(out),  dx = alpha g
//   d_gate = sum over its tokens of g n,  u = gate g,  d_w_after = sum u unit(y),  dy = back(y, u w_after)
// Bound by memory: a row is read once into registers, its statistics are made again in the backward pass from the row that it needs
// anyway (a sum more in a round of sums that is made anyway, instead of kept numbers).
//
// A team of 64, 256 or 1024 threads has a row, eight elements of it per thread and step; sums in fp32.  In the backward pass a team takes rows one
// after another and keeps its share of the weights' gradients in registers; they go to memory once per team and a second launch adds
// them up in order.  A row of the gate whose tokens lie with one team is written at once.
#include "block.h"

namespace moe {
namespace {

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(8))) float f32x8;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;

template <typename T> struct Row8;                  // eight elements as they lie in memory
template <> struct Row8<float> {
  f32x8 v;
  __device__ __forceinline__ void load(const float* p) { v = *reinterpret_cast<const f32x8 __attribute__((aligned(16)))*>(p); }
  __device__ __forceinline__ f32x8 get() const { return v; }
};
template <> struct Row8<bf16> {
  bf16x8 v;
  __device__ __forceinline__ void load(const bf16* p) { v = *reinterpret_cast<const bf16x8*>(p); }
  __device__ __forceinline__ f32x8 get() const { return __builtin_convertvector(v, f32x8); }
};
__device__ __forceinline__ f32x8 load8(const float* p) { return *reinterpret_cast<const f32x8 __attribute__((aligned(16)))*>(p); }
__device__ __forceinline__ void store8(float* p, f32x8 v) {
  *reinterpret_cast<f32x4*>(p) = __builtin_shufflevector(v, v, 0, 1, 2, 3);
  *(reinterpret_cast<f32x4*>(p) + 1) = __builtin_shufflevector(v, v, 4, 5, 6, 7);
}
__device__ __forceinline__ void store8(bf16* p, f32x8 v) { *reinterpret_cast<bf16x8*>(p) = __builtin_convertvector(v, bf16x8); }
// v as T keeps it
template <typename T> __device__ __forceinline__ f32x8 rounded(f32x8 v);
template <> __device__ __forceinline__ f32x8 rounded<float>(f32x8 v) { return v; }
template <> __device__ __forceinline__ f32x8 rounded<bf16>(f32x8 v) { return __builtin_convertvector(__builtin_convertvector(v, bf16x8), f32x8); }

__device__ __forceinline__ float sum8(f32x8 v) { return ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7])); }

// Sums of N values over a team, the same in every thread; `lds` holds two rounds, told apart by `turn`, so one barrier a round is enough.
template <int TS, int N> __device__ __forceinline__ void team_sum(float (&v)[N], float* lds, int& turn) {
#pragma unroll
  for (int off = 1; off < 64; off <<= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor(v[i], off);
  if constexpr (TS > 64) {
    constexpr int WAVES = TS / 64;
    float* at = lds + turn * (2 * WAVES);
    turn ^= 1;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) at[(threadIdx.x >> 6) * N + i] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float s = 0.f;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) s += at[w * N + i];
      v[i] = s;
    }
  }
}

constexpr int block_threads(int ts) { return ts < 256 ? 256 : ts; }

template <typename T, int TS, int K>
__global__ void __launch_bounds__(block_threads(TS)) norm_fwd_kernel(NormProblem q, int teams) {
  __shared__ float lds[2 * 2 * (TS / 64)];
  const int lane = threadIdx.x % TS, team = blockIdx.x * (block_threads(TS) / TS) + threadIdx.x / TS;
  if (team >= teams) return;                        // (whole waves; teams of more than one wave are blocks of their own)
  const T* x = static_cast<const T*>(q.x);
  const T* y = static_cast<const T*>(q.y);
  T* out = static_cast<T*>(q.out);
  T* h = static_cast<T*>(q.h);
  const float inv_d = 1.0f / (float)q.d;
  int turn = 0;
  f32x8 wa[K], wb[K], gate[K];
  int col[K];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    col[k] = (k * TS + lane) * 8;
    wa[k] = wb[k] = gate[k] = f32x8{};
    if (col[k] < q.d) {
      if (q.w_after) wa[k] = load8(q.w_after + col[k]);
      if (q.w_before) wb[k] = load8(q.w_before + col[k]);
    }
  }
  int open = -1;
  for (int t = team; t < q.T; t += teams) {
    const long row = (long)t * q.d;
    Row8<T> xr[K], yr[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      xr[k].v = {};
      yr[k].v = {};
      if (col[k] < q.d) {
        xr[k].load(x + row + col[k]);
        if (y) yr[k].load(y + row + col[k]);
      }
    }
    if (q.gate) {
      const int group = t / q.gate_rows;
      if (group != open) {
        open = group;
#pragma unroll
        for (int k = 0; k < K; ++k)
          if (col[k] < q.d) gate[k] = load8(q.gate + (long)group * q.d + col[k]);
      }
    }
    f32x8 o[K];
    if (y) {
      float r = 1.f;
      if (q.w_after) {
        float s[1] = {0.f};
#pragma unroll
        for (int k = 0; k < K; ++k) {
          const f32x8 v = yr[k].get();
          s[0] += sum8(v * v);
        }
        team_sum<TS>(s, lds, turn);
        r = 1.0f / sqrtf(s[0] * inv_d + q.eps);
      }
#pragma unroll
      for (int k = 0; k < K; ++k) {
        f32x8 n = yr[k].get();
        if (q.w_after) n = n * r * wa[k];
        if (q.gate) n = n * gate[k];
        o[k] = rounded<T>(xr[k].get() * q.alpha + n);
        if (col[k] < q.d) store8(out + row + col[k], o[k]);
      }
    } else {
#pragma unroll
      for (int k = 0; k < K; ++k) o[k] = xr[k].get();
    }
    if (q.w_before) {
      float s[1] = {0.f};
#pragma unroll
      for (int k = 0; k < K; ++k) s[0] += sum8(o[k] * o[k]);
      team_sum<TS>(s, lds, turn);
      const float r = 1.0f / sqrtf(s[0] * inv_d + q.eps);
#pragma unroll
      for (int k = 0; k < K; ++k)
        if (col[k] < q.d) store8(h + row + col[k], o[k] * r * wb[k]);
    }
  }
}

// Where the parts of a team's sums lie: [team][list][d], lists: w_before, w_after, and the gate's first and last row (tokens of other teams
// share them).
struct Parts { int lists, wb, wa, gate; };
__host__ __device__ inline Parts parts_of(bool after, bool gate, bool before) {
  Parts p{0, 0, 0, 0};
  if (before) p.wb = p.lists++;
  if (after) p.wa = p.lists++;
  if (gate) { p.gate = p.lists; p.lists += 2; }
  return p;
}

template <typename T, int TS, int K>
__global__ void __launch_bounds__(block_threads(TS)) norm_bwd_kernel(NormProblem q, int teams, int rows, float* __restrict__ parts) {
  __shared__ float lds[2 * 2 * (TS / 64)];
  const int lane = threadIdx.x % TS, team = blockIdx.x * (block_threads(TS) / TS) + threadIdx.x / TS;
  if (team >= teams) return;
  const T* x = static_cast<const T*>(q.x);
  const T* y = static_cast<const T*>(q.y);
  const T* d_out = static_cast<const T*>(q.d_out);
  const T* d_h = static_cast<const T*>(q.d_h);
  T* dx = static_cast<T*>(q.dx);
  T* dy = static_cast<T*>(q.dy);
  const Parts lists = parts_of(q.w_after, q.gate, q.w_before);
  float* mine = parts + (long)team * lists.lists * q.d;
  const float inv_d = 1.0f / (float)q.d;
  int turn = 0;
  f32x8 wa[K], wb[K], gate[K], sum_wa[K], sum_wb[K], sum_gate[K];
  int col[K];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    col[k] = (k * TS + lane) * 8;
    wa[k] = wb[k] = gate[k] = sum_wa[k] = sum_wb[k] = sum_gate[k] = f32x8{};
    if (col[k] < q.d) {
      if (q.w_after) wa[k] = load8(q.w_after + col[k]);
      if (q.w_before) wb[k] = load8(q.w_before + col[k]);
    }
  }
  const bool needs_y = q.dy && (q.w_after || q.gate);
  const int t0 = team * rows, t1 = min(t0 + rows, q.T);
  int open = -1;
  auto close_gate = [&](int group) __attribute__((always_inline)) {
    const long begin = (long)group * q.gate_rows;
    const bool begins = begin >= t0, ends = min(begin + q.gate_rows, (long)q.T) <= t1;
    float* to = begins && ends ? q.d_gate + (long)group * q.d : mine + (long)(lists.gate + (begins ? 1 : 0)) * q.d;
    const bool add = begins && ends && q.accumulate;
#pragma unroll
    for (int k = 0; k < K; ++k)
      if (col[k] < q.d) {
        store8(to + col[k], add ? sum_gate[k] + load8(to + col[k]) : sum_gate[k]);
        sum_gate[k] = f32x8{};
      }
  };
  for (int t = t0; t < t1; ++t) {
    const long row = (long)t * q.d;
    Row8<T> xr[K], yr[K], gr[K], hr[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      xr[k].v = {};
      yr[k].v = {};
      gr[k].v = {};
      hr[k].v = {};
      if (col[k] < q.d) {
        if (q.w_before) {
          xr[k].load(x + row + col[k]);
          hr[k].load(d_h + row + col[k]);
        }
        if (d_out) gr[k].load(d_out + row + col[k]);
        if (needs_y) yr[k].load(y + row + col[k]);
      }
    }
    if (q.gate) {
      const int group = t / q.gate_rows;
      if (group != open) {
        if (open >= 0) close_gate(open);
        open = group;
#pragma unroll
        for (int k = 0; k < K; ++k)
          if (col[k] < q.d) gate[k] = load8(q.gate + (long)group * q.d + col[k]);
      }
    }
    f32x8 g[K];
#pragma unroll
    for (int k = 0; k < K; ++k) g[k] = gr[k].get();
    if (q.w_before) {
      float s[2] = {0.f, 0.f};
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const f32x8 v = xr[k].get();
        s[0] += sum8(v * v);
        s[1] += sum8(hr[k].get() * wb[k] * v);
      }
      team_sum<TS>(s, lds, turn);
      const float r = 1.0f / sqrtf(s[0] * inv_d + q.eps), mean = s[1] * r * inv_d;
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const f32x8 unit = xr[k].get() * r, dh = hr[k].get();
        sum_wb[k] += dh * unit;
        g[k] += (dh * wb[k] - unit * mean) * r;
      }
    }
#pragma unroll
    for (int k = 0; k < K; ++k)
      if (col[k] < q.d) store8(dx + row + col[k], g[k] * q.alpha);
    if (!q.dy) continue;
    float r = 1.f, mean = 0.f;
    if (q.w_after) {
      float s[2] = {0.f, 0.f};
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const f32x8 v = yr[k].get();
        s[0] += sum8(v * v);
        s[1] += sum8((q.gate ? g[k] * gate[k] : g[k]) * wa[k] * v);
      }
      team_sum<TS>(s, lds, turn);
      r = 1.0f / sqrtf(s[0] * inv_d + q.eps);
      mean = s[1] * r * inv_d;
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const f32x8 unit = yr[k].get() * r;
      f32x8 u = g[k];
      if (q.gate) {
        sum_gate[k] += q.w_after ? u * unit * wa[k] : u * unit;
        u = u * gate[k];
      }
      if (q.w_after) {
        sum_wa[k] += u * unit;
        u = (u * wa[k] - unit * mean) * r;
      }
      if (col[k] < q.d) store8(dy + row + col[k], u);
    }
  }
  if (q.gate && open >= 0) close_gate(open);
#pragma unroll
  for (int k = 0; k < K; ++k)
    if (col[k] < q.d) {
      if (q.w_before) store8(mine + (long)lists.wb * q.d + col[k], sum_wb[k]);
      if (q.w_after) store8(mine + (long)lists.wa * q.d + col[k], sum_wa[k]);
    }
}

// Sums over the teams: 64 columns of one list (a weight, or a row of the gate that several teams share) per workgroup, four columns and every 64th team
// per thread.  blockIdx.y: the weights, then the gate's rows, or where those are more than the teams, the ends of teams.
__global__ void __launch_bounds__(1024) norm_join_kernel(NormProblem q, int teams, int rows, int gates, const float* __restrict__ parts) {
  __shared__ f32x4 lds[64][17];
  const Parts lists = parts_of(q.w_after, q.gate, q.w_before);
  const int part = threadIdx.x >> 4, col = blockIdx.x * 64 + (threadIdx.x & 15) * 4;
  const long team_stride = (long)lists.lists * q.d;
  int first = 0, last = teams - 1;
  const int weights = (q.w_before ? 1 : 0) + (q.w_after ? 1 : 0), list = blockIdx.y;
  const bool is_gate = list >= weights;
  float* to;
  const float* from;
  if (!is_gate) {
    const bool is_before = q.w_before && list == 0;
    to = is_before ? q.d_w_before : q.d_w_after;
    from = parts + (long)(is_before ? lists.wb : lists.wa) * q.d;
  } else {
    const int n = list - weights;
    const int group = gates < teams ? n : (int)(((long)(n + 1) * rows - 1) / q.gate_rows);       // the row of the gate that is open where team n ends
    const long begin = (long)group * q.gate_rows, end = min(begin + q.gate_rows, (long)q.T);
    first = (int)(begin / rows);
    last = (int)((end - 1) / rows);
    if (first == last || (gates >= teams && first != n)) return;          // written by its team, or another workgroup's
    to = q.d_gate + (long)group * q.d;
    from = parts + (long)lists.gate * q.d;
  }
  f32x4 sum = {};
  if (col < q.d) {
    // (a row of the gate begins in its first team's second list)
#pragma unroll 4
    for (int t = first + part; t <= last; t += 64) sum += *reinterpret_cast<const f32x4*>(from + (long)t * team_stride + (is_gate && t == first ? q.d : 0) + col);
  }
  lds[part][threadIdx.x & 15] = sum;
  __syncthreads();
  if (part < 16) {                                  // (a quarter each, then all of them)
    sum = lds[part][threadIdx.x & 15] + lds[part + 16][threadIdx.x & 15] + lds[part + 32][threadIdx.x & 15] + lds[part + 48][threadIdx.x & 15];
  }
  __syncthreads();
  if (part < 16) lds[part][threadIdx.x & 15] = sum;
  __syncthreads();
  if (part == 0 && col < q.d) {
    for (int w = 1; w < 16; ++w) sum += lds[w][threadIdx.x & 15];
    f32x4* at = reinterpret_cast<f32x4*>(to + col);
    *at = q.accumulate ? *at + sum : sum;
  }
}

// (threads of a team, steps of each)
template <typename F> int with_team(int d, F f) {
  if (d <= 512) return f(std::integral_constant<int, 64>(), std::integral_constant<int, 1>());
  if (d <= 1024) return f(std::integral_constant<int, 64>(), std::integral_constant<int, 2>());
  if (d <= 2048) return f(std::integral_constant<int, 256>(), std::integral_constant<int, 1>());
  if (d <= 4096) return f(std::integral_constant<int, 256>(), std::integral_constant<int, 2>());
  if (d <= 8192) return f(std::integral_constant<int, 1024>(), std::integral_constant<int, 1>());
  return f(std::integral_constant<int, 1024>(), std::integral_constant<int, 2>());
}

}  // namespace

NormPlan norm_bwd_plan(int T, int d, moe_dtype dt, bool after, bool gate, bool before) {
  NormPlan p{};
  const int most = d <= 1024 ? 2048 : 512;
  p.rows = cdiv(T, most);
  if (p.rows < 4) p.rows = T < 4 ? (T < 1 ? 1 : T) : 4;
  p.teams = cdiv(T, p.rows);
  p.bytes = (size_t)p.teams * parts_of(after, gate, before).lists * d * 4 + 256;
  return p;
}

int launch_norm_fwd(const NormProblem& q, hipStream_t s) {
  return with_team(q.d, [&](auto ts, auto k) {
    constexpr int TS = decltype(ts)::value, K = decltype(k)::value, per = block_threads(TS) / TS;
    const int most = 256 * 2048 / TS;
    const int teams = q.T < most ? q.T : most;
    const dim3 grid((unsigned)cdiv(teams, per)), block(block_threads(TS));
    if (q.dt == MOE_F32) norm_fwd_kernel<float, TS, K><<<grid, block, 0, s>>>(q, teams);
    else norm_fwd_kernel<bf16, TS, K><<<grid, block, 0, s>>>(q, teams);
    MOE_LAUNCH_CHECK();
    return (int)MOE_OK;
  });
}

int launch_norm_bwd(const NormProblem& q, const NormPlan& p, float* ws, hipStream_t s) {
  const int rc = with_team(q.d, [&](auto ts, auto k) {
    constexpr int TS = decltype(ts)::value, K = decltype(k)::value, per = block_threads(TS) / TS;
    const dim3 grid((unsigned)cdiv(p.teams, per)), block(block_threads(TS));
    if (q.dt == MOE_F32) norm_bwd_kernel<float, TS, K><<<grid, block, 0, s>>>(q, p.teams, p.rows, ws);
    else norm_bwd_kernel<bf16, TS, K><<<grid, block, 0, s>>>(q, p.teams, p.rows, ws);
    MOE_LAUNCH_CHECK();
    return (int)MOE_OK;
  });
  if (rc != MOE_OK) return rc;
  const int weights = (q.w_before ? 1 : 0) + (q.w_after ? 1 : 0);
  const int gates = q.gate ? (int)(((long)q.T + q.gate_rows - 1) / q.gate_rows) : 0;
  const int spans = !q.gate || q.gate_rows == 1 || p.teams == 1 ? 0 : gates < p.teams ? gates : p.teams - 1;      // (a token's own row never spans teams)
  if (weights + spans > 0) {
    norm_join_kernel<<<dim3((unsigned)cdiv(q.d, 64), (unsigned)(weights + spans)), dim3(1024), 0, s>>>(q, p.teams, p.rows, gates, ws);
    MOE_LAUNCH_CHECK();
  }
  return MOE_OK;
}

}  // namespace moe
