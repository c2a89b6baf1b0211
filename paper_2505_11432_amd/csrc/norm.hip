// The end of one block and the start of the next on the residual stream, and their gradients, each row in one piece.
//   n = y / rms(y) * w_after  (or y),  out = alpha x + gate * n  (or + n),  h = out / rms(out) * w_before
//   rms(v) = sqrt(mean v^2 + eps);  h is made from `out` as it is kept (rounded), which is what the backward pass reads again.
// Backward, with unit(v) = v / rms(v) and back(v, u) = (u - unit(v) mean(u unit(v))) / rms(v):
//   g = d_out + back(out, d_h w_before),  d_w_before = sum d_h unit(out),  dx = alpha g
//   d_gate = sum over its tokens of g n,  u = gate g,  d_w_after = sum u unit(y),  dy = back(y, u w_after)
// Bound by memory: a row is read once into registers, its statistics are made again in the backward pass from the row that it needs
// anyway (a sum more in a round of sums that is made anyway, instead of kept numbers).
//
// A team of 64 to 1024 threads has a row, eight elements of it per thread and step.  In the forward pass the rows in flight are those of the teams that share a
// CU.  In the backward pass what a team holds per column (weights, gate, sums of gradients) is most of its registers, few teams fit a CU, and a team loads the next
// row while it works on one.  Sums in fp32.  In the backward pass a team's rows lie one after another; its share
// of the weights' gradients goes to memory once and a second launch adds the teams up in order.  A row of the gate whose tokens lie with one team is
// written at once.
#include "block.h"

namespace moe {
namespace {

typedef __attribute__((ext_vector_type(4))) float f32x4;

constexpr int W = 8;                        // elements of a thread's piece of a row
typedef float vec __attribute__((ext_vector_type(W)));

// A piece as it lies in memory, read and written past the caches (a row is used once)
template <typename T> struct Piece;
template <> struct Piece<float> {
  vec v;
  __device__ __forceinline__ void load(const float* p) {
    const f32x4 a = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(p));
    v = __builtin_shufflevector(a, __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(p) + 1), 0, 1, 2, 3, 4, 5, 6, 7);
  }
  __device__ __forceinline__ vec get() const { return v; }
};
template <> struct Piece<bf16> {
  typedef __bf16 raw __attribute__((ext_vector_type(W)));
  raw v;
  __device__ __forceinline__ void load(const bf16* p) { v = __builtin_nontemporal_load(reinterpret_cast<const raw*>(p)); }
  __device__ __forceinline__ vec get() const { return __builtin_convertvector(v, vec); }
};
__device__ __forceinline__ vec load_f32(const float* p) {
  return __builtin_shufflevector(*reinterpret_cast<const f32x4*>(p), *(reinterpret_cast<const f32x4*>(p) + 1), 0, 1, 2, 3, 4, 5, 6, 7);
}
__device__ __forceinline__ void store(float* p, vec v) {
  *reinterpret_cast<f32x4*>(p) = __builtin_shufflevector(v, v, 0, 1, 2, 3);
  *(reinterpret_cast<f32x4*>(p) + 1) = __builtin_shufflevector(v, v, 4, 5, 6, 7);
}
__device__ __forceinline__ void store(bf16* p, vec v) {
  typedef __bf16 raw __attribute__((ext_vector_type(W)));
  __builtin_nontemporal_store(__builtin_convertvector(v, raw), reinterpret_cast<raw*>(p));
}
// v as T keeps it
template <typename T> __device__ __forceinline__ vec rounded(vec v) {
  typedef T raw __attribute__((ext_vector_type(W)));
  return __builtin_convertvector(__builtin_convertvector(v, raw), vec);
}
__device__ __forceinline__ float sum_of(vec v) {
  const float s = (v[0] + v[1]) + (v[2] + v[3]);
  return s + ((v[4] + v[5]) + (v[6] + v[7]));
}

// Sums of N values over a team, the same in every thread; `lds` holds two rounds, told apart by `turn`, so one barrier a round is enough.
constexpr int kMostSums = 2;
template <int TS, int N> __device__ __forceinline__ void team_sum(float (&v)[N], float* lds, int& turn) {
  static_assert(N <= kMostSums, "the sums of a round");
#pragma unroll
  for (int off = 1; off < 64; off <<= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor(v[i], off);
  if constexpr (TS > 64) {
    constexpr int WAVES = TS / 64;
    float* at = lds + turn * (kMostSums * WAVES);
    turn ^= 1;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) at[i * WAVES + (threadIdx.x >> 6)] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float s = 0.f;
#pragma unroll
      for (int w = 0; w < WAVES; w += 4) {
        const f32x4 four = *reinterpret_cast<const f32x4*>(at + i * WAVES + w);
        s += (four[0] + four[1]) + (four[2] + four[3]);
      }
      v[i] = s;
    }
  }
}

constexpr int block_threads(int ts) { return ts < 256 ? 256 : ts; }
template <int TS> constexpr int lds_floats() { return 2 * kMostSums * (TS / 64); }

// Teams of the forward pass take rows in turn.
template <typename T, int TS, int K>
__global__ void __launch_bounds__(block_threads(TS)) norm_fwd_kernel(NormProblem q, int teams) {
  __shared__ __attribute__((aligned(16))) float lds[lds_floats<TS>()];
  const int lane = threadIdx.x % TS, team = blockIdx.x * (block_threads(TS) / TS) + threadIdx.x / TS;
  if (team >= teams) return;                        // (whole waves; teams of more than one wave are blocks of their own)
  const T* x = static_cast<const T*>(q.x);
  const T* y = static_cast<const T*>(q.y);
  T* out = static_cast<T*>(q.out);
  T* h = static_cast<T*>(q.h);
  const float inv_d = 1.0f / (float)q.d;
  int turn = 0;
  vec wa[K], wb[K], gate[K];
  int col[K];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    col[k] = (k * TS + lane) * W;
    wa[k] = wb[k] = gate[k] = vec{};
    if (col[k] < q.d) {
      if (q.w_after) wa[k] = load_f32(q.w_after + col[k]);
      if (q.w_before) wb[k] = load_f32(q.w_before + col[k]);
    }
  }
  int open = -1;                                    // row of the gate in registers
  for (long t = team; t < q.T; t += teams) {
    Piece<T> xr[K], yr[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      xr[k].v = {};
      yr[k].v = {};
      if (col[k] < q.d) {
        xr[k].load(x + t * q.d + col[k]);
        if (y) yr[k].load(y + t * q.d + col[k]);
      }
    }
    float sum[1];
    vec o[K];
    if (y) {
      float inv = 1.f;
      if (q.w_after) {
        sum[0] = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
          const vec v = yr[k].get();
          sum[0] += sum_of(v * v);
        }
        team_sum<TS>(sum, lds, turn);
        inv = 1.0f / sqrtf(sum[0] * inv_d + q.eps);
      }
      if (q.gate) {
        const int group = (int)(t / q.gate_rows);
        if (group != open) {
          open = group;
#pragma unroll
          for (int k = 0; k < K; ++k)
            if (col[k] < q.d) gate[k] = load_f32(q.gate + (long)group * q.d + col[k]);
        }
      }
#pragma unroll
      for (int k = 0; k < K; ++k) {
        vec n = yr[k].get();
        if (q.w_after) n = n * inv * wa[k];
        if (q.gate) n = n * gate[k];
        o[k] = rounded<T>(xr[k].get() * q.alpha + n);
        if (col[k] < q.d) store(out + t * q.d + col[k], o[k]);
      }
    } else {
#pragma unroll
      for (int k = 0; k < K; ++k) o[k] = xr[k].get();
    }
    if (q.w_before) {
      sum[0] = 0.f;
#pragma unroll
      for (int k = 0; k < K; ++k) sum[0] += sum_of(o[k] * o[k]);
      team_sum<TS>(sum, lds, turn);
      const float inv = 1.0f / sqrtf(sum[0] * inv_d + q.eps);
#pragma unroll
      for (int k = 0; k < K; ++k)
        if (col[k] < q.d) store(h + t * q.d + col[k], o[k] * inv * wb[k]);
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

// TOKEN: every token has its own row of the gate.  HOLD: the weights stay in registers (the widest rows leave no room for them).  AHEAD: the next row is
// on its way while one is worked on.
template <typename T, int TS, int K, bool HOLD, bool TOKEN, bool AHEAD>
__global__ void __launch_bounds__(block_threads(TS)) norm_bwd_kernel(NormProblem q, int teams, int rows, float* __restrict__ parts) {
  __shared__ __attribute__((aligned(16))) float lds[lds_floats<TS>()];
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
  const bool grouped = q.gate && !TOKEN;
  int turn = 0;
  vec wa_held[HOLD ? K : 1], wb_held[HOLD ? K : 1], gate_held[HOLD && !TOKEN ? K : 1], sum_wa[K], sum_wb[K], sum_gate[TOKEN ? 1 : K];
  int col[K];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    col[k] = (k * TS + lane) * W;
    sum_wa[k] = sum_wb[k] = vec{};
    if constexpr (!TOKEN) sum_gate[k] = vec{};
    if constexpr (HOLD && !TOKEN) gate_held[k] = vec{};
    if constexpr (HOLD) {
      wa_held[k] = wb_held[k] = vec{};
      if (col[k] < q.d) {
        if (q.w_after) wa_held[k] = load_f32(q.w_after + col[k]);
        if (q.w_before) wb_held[k] = load_f32(q.w_before + col[k]);
      }
    }
  }
  const bool needs_y = q.dy && (q.w_after || q.gate);
  const int t_begin = team * rows, t_end = min(t_begin + rows, q.T);
  int open = -1;
  auto at_col = [&](const float* w, int k) __attribute__((always_inline)) -> vec { return col[k] < q.d ? load_f32(w + col[k]) : vec{}; };
  auto wa = [&](int k) __attribute__((always_inline)) -> vec { if constexpr (HOLD) return wa_held[k]; else return at_col(q.w_after, k); };
  auto wb = [&](int k) __attribute__((always_inline)) -> vec { if constexpr (HOLD) return wb_held[k]; else return at_col(q.w_before, k); };
  auto close_gate = [&](int group) __attribute__((always_inline)) {
    if constexpr (!TOKEN) {
      const long begin = (long)group * q.gate_rows;
      const bool begins = begin >= t_begin, ends = min(begin + q.gate_rows, (long)q.T) <= t_end;
      float* to = begins && ends ? q.d_gate + (long)group * q.d : mine + (long)(lists.gate + (begins ? 1 : 0)) * q.d;
      const bool add = begins && ends && q.accumulate;
#pragma unroll
      for (int k = 0; k < K; ++k)
        if (col[k] < q.d) {
          store(to + col[k], add ? sum_gate[k] + load_f32(to + col[k]) : sum_gate[k]);
          sum_gate[k] = vec{};
        }
    }
  };
  struct Row { Piece<T> x[K], y[K], g[K], h[K]; } now, next;
  auto fetch = [&](Row& to, int t) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const long at = (long)t * q.d + col[k];
      to.x[k].v = {};
      to.y[k].v = {};
      to.g[k].v = {};
      to.h[k].v = {};
      if (col[k] < q.d) {
        if (q.w_before) {
          to.x[k].load(x + at);
          to.h[k].load(d_h + at);
        }
        if (d_out) to.g[k].load(d_out + at);
        if (needs_y) to.y[k].load(y + at);
      }
    }
  };
  if constexpr (AHEAD) {
    if (t_begin < t_end) fetch(next, t_begin);
  }
  for (int t = t_begin; t < t_end; ++t) {
    if (grouped) {
      const int group = t / q.gate_rows;
      if (group != open) {
        if (open >= 0) close_gate(open);
        open = group;
        if constexpr (HOLD && !TOKEN) {
#pragma unroll
          for (int k = 0; k < K; ++k) gate_held[k] = at_col(q.gate + (long)group * q.d, k);
        }
      }
    }
    const long row = (long)t * q.d;
    if constexpr (AHEAD) {
      now = next;
      if (t + 1 < t_end) fetch(next, t + 1);
    } else {
      fetch(now, t);
    }
    vec token_gate[TOKEN ? K : 1];
    if constexpr (TOKEN) {
#pragma unroll
      for (int k = 0; k < K; ++k) token_gate[k] = at_col(q.gate + row, k);
    }
    auto gate = [&](int k) __attribute__((always_inline)) -> vec {
      if constexpr (TOKEN) return token_gate[k];
      else if constexpr (HOLD) return gate_held[k];
      else return at_col(q.gate + (long)open * q.d, k);
    };
    vec g[K];
#pragma unroll
    for (int k = 0; k < K; ++k) g[k] = now.g[k].get();
    if (q.w_before) {
      float s[2] = {0.f, 0.f};
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const vec v = now.x[k].get();
        s[0] += sum_of(v * v);
        s[1] += sum_of(now.h[k].get() * wb(k) * v);
      }
      team_sum<TS>(s, lds, turn);
      const float i = 1.0f / sqrtf(s[0] * inv_d + q.eps), mean = s[1] * i * inv_d;
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const vec unit = now.x[k].get() * i, dh = now.h[k].get();
        sum_wb[k] += dh * unit;
        g[k] += (dh * wb(k) - unit * mean) * i;
      }
    }
#pragma unroll
    for (int k = 0; k < K; ++k)
      if (col[k] < q.d) store(dx + row + col[k], g[k] * q.alpha);
    if (!q.dy) continue;
    float i = 1.f, mean = 0.f;
    if (q.w_after) {
      float s[2] = {0.f, 0.f};
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const vec v = now.y[k].get();
        s[0] += sum_of(v * v);
        s[1] += sum_of((q.gate ? g[k] * gate(k) : g[k]) * wa(k) * v);
      }
      team_sum<TS>(s, lds, turn);
      i = 1.0f / sqrtf(s[0] * inv_d + q.eps);
      mean = s[1] * i * inv_d;
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const vec unit = now.y[k].get() * i;
      vec u = g[k];
      if (q.gate) {
        const vec d_gate = q.w_after ? u * unit * wa(k) : u * unit;
        if constexpr (TOKEN) {
          float* to = q.d_gate + row + col[k];
          if (col[k] < q.d) store(to, q.accumulate ? d_gate + load_f32(to) : d_gate);
        } else {
          sum_gate[k] += d_gate;
        }
        u = u * gate(k);
      }
      if (q.w_after) {
        sum_wa[k] += u * unit;
        u = (u * wa(k) - unit * mean) * i;
      }
      if (col[k] < q.d) store(dy + row + col[k], u);
    }
  }
  if (grouped && open >= 0) close_gate(open);
#pragma unroll
  for (int k = 0; k < K; ++k)
    if (col[k] < q.d) {
      if (q.w_before) store(mine + (long)lists.wb * q.d + col[k], sum_wb[k]);
      if (q.w_after) store(mine + (long)lists.wa * q.d + col[k], sum_wa[k]);
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

// Threads of a team and pieces of each; HOLD: see the backward pass.
template <int TS_, int K_, bool HOLD_ = true> struct Team { static constexpr int TS = TS_, K = K_; static constexpr bool HOLD = HOLD_; };
// Forward (bf16, all parts, us): a row at a time 16384 x 2048 50 (5.4 TB/s), 8192 x 4096 49, 4096 x 8192 52; two or four rows at a time, which leave room for fewer
// teams, 53 and 56, 56 and 64, 60; 32768 x 1024 by one wave with two steps 59, by 256 threads of four elements 66.
template <typename F> int with_fwd_team(int d, F f) {
  if (d <= 512) return f(Team<64, 1>());
  if (d <= 1024) return f(Team<64, 2>());
  if (d <= 2048) return f(Team<256, 1>());
  if (d <= 4096) return f(Team<512, 1>());
  if (d <= 8192) return f(Team<1024, 1>());
  return f(Team<1024, 2>());
}
// Backward (8192 x 4096, bf16, all parts, 256 or 512 teams, us): 256 threads, 16 elements each 91, with the next row ahead 84; 512 threads, 8 elements, a row
// ahead 82 (4.9 TB/s, what a copy takes); 1024 threads 109 to 127; two to four rows at a time instead of one ahead 103 to 141.  Wider rows have 1024 threads all the
// same: 4096 x 8192 99, 6144 x 5120 110, 2048 x 16384, which keeps no weights in registers, 292.
template <typename F> int with_bwd_team(int d, F f) {
  if (d <= 512) return f(Team<64, 1>());
  if (d <= 1024) return f(Team<64, 2>());
  if (d <= 2048) return f(Team<256, 1>());
  if (d <= 4096) return f(Team<512, 1>());
  if (d <= 8192) return f(Team<1024, 1>());
  return f(Team<1024, 2, false>());
}

}  // namespace

NormPlan norm_bwd_plan(int T, int d, moe_dtype dt, bool after, bool gate, bool before) {
  NormPlan p{};
  // as many teams as run at a time; of few rows two each (777 x 1040, fp32, with 1, 2, 3, 4, 6: 19.8, 15.4, 15.6, 16.6, 19.8 us; other sizes of few rows were not
  // tried with other teams, whose sums weigh more the wider the rows: 1024 x 4096, bf16, 28.6, 1025 x 4096 23.0)
  const int most = d <= 1024 ? 2048 : d <= 2048 ? 512 : 256;
  p.rows = T <= 1024 ? cdiv(T, 512) : cdiv(T, most);
  if (p.rows < 1) p.rows = 1;
  p.teams = cdiv(T, p.rows);
  p.bytes = (size_t)p.teams * parts_of(after, gate, before).lists * d * 4 + 256;
  return p;
}

int launch_norm_fwd(const NormProblem& q, hipStream_t s) {
  return with_fwd_team(q.d, [&](auto team) {
    typedef decltype(team) C;
    constexpr int per = block_threads(C::TS) / C::TS;
    const int most = 256 * 2048 / C::TS, teams = q.T < most ? q.T : most;
    const dim3 grid((unsigned)cdiv(teams, per)), block(block_threads(C::TS));
    if (q.dt == MOE_F32) norm_fwd_kernel<float, C::TS, C::K><<<grid, block, 0, s>>>(q, teams);
    else norm_fwd_kernel<bf16, C::TS, C::K><<<grid, block, 0, s>>>(q, teams);
    MOE_LAUNCH_CHECK();
    return (int)MOE_OK;
  });
}

int launch_norm_bwd(const NormProblem& q, const NormPlan& p, float* ws, hipStream_t s) {
  const int rc = with_bwd_team(q.d, [&](auto team) {
    typedef decltype(team) C;
    constexpr int per = block_threads(C::TS) / C::TS;
    // (a row ahead takes registers: twice as many in fp32)
    constexpr bool AHEAD16 = C::TS < 1024, AHEAD32 = AHEAD16 && C::K == 1;
    const dim3 grid((unsigned)cdiv(p.teams, per)), block(block_threads(C::TS));
    const bool token = q.gate && q.gate_rows == 1;
    if (q.dt == MOE_F32 && !token) norm_bwd_kernel<float, C::TS, C::K, C::HOLD, false, AHEAD32><<<grid, block, 0, s>>>(q, p.teams, p.rows, ws);
    else if (q.dt == MOE_F32) norm_bwd_kernel<float, C::TS, C::K, C::HOLD, true, AHEAD32><<<grid, block, 0, s>>>(q, p.teams, p.rows, ws);
    else if (!token) norm_bwd_kernel<bf16, C::TS, C::K, C::HOLD, false, AHEAD16><<<grid, block, 0, s>>>(q, p.teams, p.rows, ws);
    else norm_bwd_kernel<bf16, C::TS, C::K, C::HOLD, true, AHEAD16><<<grid, block, 0, s>>>(q, p.teams, p.rows, ws);
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
