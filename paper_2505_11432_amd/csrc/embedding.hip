// Embedding rows of a batch of tokens, and the gradient of the embedding by sorted tokens.
//   out[t] = scale * table[token t]  (zeros where the token is outside 0..V-1)
//   d_table[v] (+)= scale * sum of dy[t] over the tokens t that are v
// Both are bound by memory; of few tokens by the launches.
//
// The gradient: the tokens are sorted by word, those of one word in the order of the batch (counting sort by digits, stable), and cut into
// chunks of the sorted order.  A wave adds up one chunk over 512 columns in fp32, run by run of equal words; a run that lies inside a chunk is
// written to its row at once, the first and last run of a chunk may go on in the next one and leave a partial sum, which a second launch
// adds up in order.  No atomic addition: the bits depend on the tokens and the sizes alone.  Rows without a token are zeroed by
// other workgroups of the same launch, which find them by binary search, a lane per row, or all rows are zeroed beside the sort.  Of few tokens nothing is
// sorted.
//
// Measured (fp32 gradients): 16384 rows of 2048 in bf16 looked up 16.4 us (20 MB read, 67 MB written: 5.3 TB/s); the gradient of 8192 x 4096, 32000 words 137 us, of them
// 81 the sort with 524 MB of zeros beside it (6.5 TB/s) and 42 the sums; of 65536 x 4096 266 us (1.06 GB, 4.0 TB/s).
#include "block.h"

namespace moe {
namespace {

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(8))) float f32x8;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) unsigned u32x4;

// eight elements as floats, from and to memory that is 16-byte aligned
__device__ __forceinline__ f32x8 load8(const float* p) { return *reinterpret_cast<const f32x8 __attribute__((aligned(16)))*>(p); }
__device__ __forceinline__ f32x8 load8(const bf16* p) { return __builtin_convertvector(*reinterpret_cast<const bf16x8*>(p), f32x8); }
// (eight fp32 lie in two stores that fill a line together: they are left to the L2)
__device__ __forceinline__ void store8(float* p, f32x8 v) {
  *reinterpret_cast<f32x4*>(p) = __builtin_shufflevector(v, v, 0, 1, 2, 3);
  *(reinterpret_cast<f32x4*>(p) + 1) = __builtin_shufflevector(v, v, 4, 5, 6, 7);
}
__device__ __forceinline__ void store8(bf16* p, f32x8 v) { __builtin_nontemporal_store(__builtin_convertvector(v, bf16x8), reinterpret_cast<bf16x8*>(p)); }

// ---- lookup ------------------------------------------------------------------------------------
// Units of eight elements, four at a time per thread.
template <typename T>
__global__ void __launch_bounds__(256) lookup_kernel(const T* __restrict__ table, const int32_t* __restrict__ tokens, long units, int per_row, int V, float scale,
                                                     T* __restrict__ out) {
  constexpr int U = 4;
  const long first = (long)blockIdx.x * (256 * U) + threadIdx.x;
  f32x8 v[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const long at = first + u * 256;
    v[u] = f32x8{};
    if (at < units) {
      const long row = at / per_row;
      const int col = (int)(at - row * per_row), token = tokens[row];
      if ((unsigned)token < (unsigned)V) v[u] = load8(table + ((long)token * per_row + col) * 8);
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const long at = first + u * 256;
    if (at < units) store8(out + at * 8, v[u] * scale);
  }
}

// ---- sort ----------------------------------------------------------------------------------------
// One pass over BITS bits of the keys of a tile, the items of a wave lying one after another: wave w of NW, round r, lane l holds item
// (w * ROUNDS + r) * 64 + l.  rank: how many items with the same digit lie in front of it in its wave; counts[digit][wave].
template <int ROUNDS, typename Count>
__device__ __forceinline__ void rank_items(const unsigned (&digit)[ROUNDS], const bool (&there)[ROUNDS], int bits, Count* counts, unsigned (&rank)[ROUNDS]) {
  const int lane = threadIdx.x & 63;
  const unsigned long long below = (1ull << lane) - 1;
#pragma unroll
  for (int r = 0; r < ROUNDS; ++r) {
    unsigned long long same = __ballot(there[r]);
    for (int b = 0; b < bits; ++b) {
      const unsigned long long set = __ballot(digit[r] >> b & 1);
      same &= digit[r] >> b & 1 ? set : ~set;
    }
    rank[r] = 0;
    if (there[r]) {
      // (a wave's counts are its own: the lane in front reads and writes for its digit, the others take what it read)
      const unsigned before = counts[digit[r]];
      rank[r] = before + (unsigned)__popcll(same & below);
    }
    __builtin_amdgcn_wave_barrier();
    if (there[r] && (same & below) == 0) counts[digit[r]] += (Count)__popcll(same);
    __builtin_amdgcn_wave_barrier();
  }
}

// exclusive sums over bins of 1024 threads' values, thread by thread
__device__ __forceinline__ unsigned block_scan(unsigned v, unsigned (&sums)[16]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  unsigned incl = v;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const unsigned o = __shfl_up(incl, off);
    if (lane >= off) incl += o;
  }
  if (lane == 63) sums[wave] = incl;
  __syncthreads();
  unsigned base = 0;
  for (int w = 0; w < wave; ++w) base += sums[w];
  __syncthreads();
  return base + incl - v;
}

__device__ __forceinline__ unsigned key_of(int32_t token, int V) { return (unsigned)token < (unsigned)V ? (unsigned)token : (unsigned)V; }

constexpr int kBins = 1 << kMaxDigit, kWaves = 16;
constexpr int kStride = kBins + 1;      // (counts of the waves in different banks)

// All passes over at most kSortOne tokens in one workgroup, word and place packed into one number in LDS (the words take at most kOneBits bits).  The
// other workgroups zero `zero_units` pieces of 16 bytes.
__global__ void __launch_bounds__(1024) sort_one_kernel(const int32_t* __restrict__ tokens, int T, int V, int passes, int bits, uint2* __restrict__ pairs,
                                                        u32x4* __restrict__ zero, long zero_units) {
  constexpr int ROUNDS = kSortOne / 1024, PLACE = 32 - kOneBits;
  static_assert(kSortOne <= 1 << PLACE, "a place fits beside the word");
  __shared__ unsigned items[kSortOne];
  __shared__ unsigned short counts[kWaves * kStride];
  __shared__ unsigned sums[16];
  if (blockIdx.x > 0) {
    const long step = ((long)gridDim.x - 1) * 1024;
    long i = ((long)blockIdx.x - 1) * 1024 + threadIdx.x;
    for (; i + 3 * step < zero_units; i += 4 * step)
#pragma unroll
      for (int u = 0; u < 4; ++u) zero[i + u * step] = u32x4{0, 0, 0, 0};
    for (; i < zero_units; i += step) zero[i] = u32x4{0, 0, 0, 0};
    return;
  }
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, rounds = (T + 1023) / 1024;
  unsigned item[ROUNDS];
  bool there[ROUNDS];
#pragma unroll
  for (int r = 0; r < ROUNDS; ++r) {
    const int i = (wave * rounds + r) * 64 + lane;
    there[r] = r < rounds && i < T;
    item[r] = there[r] ? key_of(tokens[i], V) << PLACE | (unsigned)i : 0u;
  }
  for (int pass = 0; pass < passes; ++pass) {
    for (int i = tid; i < kWaves * kStride; i += 1024) counts[i] = 0;
    __syncthreads();
    unsigned digit[ROUNDS], rank[ROUNDS];
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) digit[r] = item[r] >> (PLACE + pass * bits) & ((1u << bits) - 1);
    rank_items<ROUNDS>(digit, there, bits, counts + wave * kStride, rank);
    __syncthreads();
    // thread t: digit t; its counts become where each wave's items begin
    unsigned total = 0;
    if (tid < kBins)
      for (int w = 0; w < kWaves; ++w) total += counts[w * kStride + tid];
    unsigned at = block_scan(total, sums);
    if (tid < kBins)
      for (int w = 0; w < kWaves; ++w) {
        const unsigned n = counts[w * kStride + tid];
        counts[w * kStride + tid] = (unsigned short)at;
        at += n;
      }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r)
      if (there[r]) {
        const unsigned to = counts[wave * kStride + digit[r]] + rank[r];
        if (pass + 1 < passes) items[to] = item[r];
        else pairs[to] = uint2{item[r] >> PLACE, item[r] & ((1u << PLACE) - 1)};
      }
    __syncthreads();
    if (pass + 1 < passes) {
#pragma unroll
      for (int r = 0; r < ROUNDS; ++r)
        if (there[r]) item[r] = items[(wave * rounds + r) * 64 + lane];
      __syncthreads();
    }
  }
}

constexpr int kTileRounds = kSortTile / 1024;
__device__ __forceinline__ void tile_items(const int32_t* tokens, const uint2* from, int T, int V, uint2 (&item)[kTileRounds], bool (&there)[kTileRounds]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int r = 0; r < kTileRounds; ++r) {
    const int i = blockIdx.x * kSortTile + (wave * kTileRounds + r) * 64 + lane;
    there[r] = i < T;
    item[r] = !there[r] ? uint2{0, 0} : from ? from[i] : uint2{key_of(tokens[i], V), (unsigned)i};
  }
}

// counts[tile][digit] of a pass; from == NULL: the first pass
__global__ void __launch_bounds__(1024) sort_count_kernel(const int32_t* __restrict__ tokens, const uint2* __restrict__ from, int T, int V, int shift, int bits,
                                                          unsigned* __restrict__ tile_counts) {
  __shared__ unsigned counts[kBins];
  for (int i = threadIdx.x; i < kBins; i += 1024) counts[i] = 0;
  __syncthreads();
  uint2 item[kTileRounds];
  bool there[kTileRounds];
  tile_items(tokens, from, T, V, item, there);
#pragma unroll
  for (int r = 0; r < kTileRounds; ++r)
    if (there[r]) atomicAdd(&counts[item[r].x >> shift & ((1u << bits) - 1)], 1u);      // (integers: the order does not matter)
  __syncthreads();
  for (int i = threadIdx.x; i < kBins; i += 1024) tile_counts[(long)blockIdx.x * kBins + i] = counts[i];
}

__global__ void __launch_bounds__(1024) sort_place_kernel(const int32_t* __restrict__ tokens, const uint2* __restrict__ from, int T, int V, int shift, int bits,
                                                          const unsigned* __restrict__ tile_counts, uint2* __restrict__ to) {
  __shared__ unsigned counts[kWaves * kStride];
  __shared__ unsigned halves[2][2 * kBins];
  __shared__ unsigned sums[16];
  const int tid = threadIdx.x, wave = tid >> 6;
  for (int i = tid; i < kWaves * kStride; i += 1024) counts[i] = 0;
  uint2 item[kTileRounds];
  bool there[kTileRounds];
  tile_items(tokens, from, T, V, item, there);
  // this tile's first place for every digit: the items of smaller digits, and those of this digit in the tiles in front
  {
    const int bin = tid & (kBins - 1), half = tid / kBins;
    unsigned all = 0, before = 0;
    for (int t = half; t < (int)gridDim.x; t += 2) {
      const unsigned n = tile_counts[(long)t * kBins + bin];
      all += n;
      before += t < (int)blockIdx.x ? n : 0;
    }
    halves[half][bin] = all;
    halves[half][kBins + bin] = before;
  }
  __syncthreads();
  unsigned digit[kTileRounds], rank[kTileRounds];
#pragma unroll
  for (int r = 0; r < kTileRounds; ++r) digit[r] = item[r].x >> shift & ((1u << bits) - 1);
  rank_items<kTileRounds>(digit, there, bits, counts + wave * kStride, rank);
  __syncthreads();
  const unsigned total = tid < kBins ? halves[0][tid] + halves[1][tid] : 0;
  unsigned at = block_scan(total, sums);
  if (tid < kBins) {
    at += halves[0][kBins + tid] + halves[1][kBins + tid];
    for (int w = 0; w < kWaves; ++w) {
      const unsigned n = counts[w * kStride + tid];
      counts[w * kStride + tid] = at;
      at += n;
    }
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < kTileRounds; ++r)
    if (there[r]) to[counts[wave * kStride + digit[r]] + rank[r]] = item[r];
}

// ---- sums ----------------------------------------------------------------------------------------
constexpr int kSlab = 512;                  // columns of a wave
constexpr int kZeroRows = 16;               // rows that a zeroing workgroup looks at

// first place whose key is >= key
__device__ __forceinline__ int lower_bound(const uint2* __restrict__ pairs, int T, unsigned key) {
  int lo = 0, hi = T;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (pairs[mid].x < key) lo = mid + 1; else hi = mid;
  }
  return lo;
}

template <typename TG> __device__ __forceinline__ void write_sum(TG* p, f32x8 sum, float scale, int accumulate) {
  sum *= scale;
  if (accumulate) sum += load8(p);
  store8(p, sum);
}

// zeros, by 256 threads
template <typename TG> __device__ __forceinline__ void zero_row(TG* row, int d) {
  constexpr int N = 16 / sizeof(TG);
  for (int c = threadIdx.x * N; c < d; c += 256 * N) *reinterpret_cast<u32x4*>(row + c) = u32x4{0, 0, 0, 0};
}

// Few tokens: the whole gradient in one launch, without a sort.  A workgroup per token and slab of columns looks through all tokens; if its own is the
// first of its word it adds them up, wave w the w-th quarter of the batch, in order.
template <typename T, typename TG>
__global__ void __launch_bounds__(256) few_kernel(const int32_t* __restrict__ tokens, const T* __restrict__ dy, int n, int d, int V, float scale,
                                                  TG* __restrict__ d_table, int accumulate, int slabs, int sum_groups) {
  constexpr int B = 8;                      // rows in flight
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  if ((int)blockIdx.x >= sum_groups) {      // rows without a token
    __shared__ unsigned seen[kZeroRows];
    const int row0 = ((int)blockIdx.x - sum_groups) * kZeroRows, rows = min(kZeroRows, V - row0);
    if (threadIdx.x < kZeroRows) seen[threadIdx.x] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += 256) {
      const unsigned r = (unsigned)tokens[i] - (unsigned)row0;
      if (r < (unsigned)rows) seen[r] = 1;
    }
    __syncthreads();
    for (int r = 0; r < rows; ++r)
      if (!seen[r]) zero_row(d_table + (long)(row0 + r) * d, d);
    return;
  }
  __shared__ f32x8 others[3][64];
  const int t = blockIdx.x / slabs, slab = blockIdx.x - t * slabs, col = slab * kSlab + lane * 8;
  const int token = tokens[t];
  if ((unsigned)token >= (unsigned)V) return;
  int found = 0;
  for (int i = threadIdx.x; i < t; i += 256) found |= tokens[i] == token;
  if (__syncthreads_or(found)) return;
  // places of the word in this wave's quarter of what is left, in order
  constexpr int ROUNDS = kFewTokens / 4 / 64;
  __shared__ unsigned short list[4][ROUNDS * 64];
  const int quarter = (n - t + 3) / 4, begin = t + wave * quarter, end = min(begin + quarter, n);
  int count = 0;
  bool same[ROUNDS];
#pragma unroll
  for (int r = 0; r < ROUNDS; ++r) {
    const int i = begin + r * 64 + lane;
    same[r] = i < end && tokens[min(i, n - 1)] == token;
  }
#pragma unroll
  for (int r = 0; r < ROUNDS; ++r) {
    const unsigned long long mask = __ballot(same[r]);
    if (same[r]) list[wave][count + __popcll(mask & ((1ull << lane) - 1))] = (unsigned short)(begin + r * 64 + lane);
    count += __popcll(mask);
  }
  __builtin_amdgcn_wave_barrier();
  const T* src = dy + min(col, d - 8);
  f32x8 sum = {};
  for (int k = 0; k < count; k += B) {
    f32x8 v[B];
#pragma unroll
    for (int b = 0; b < B; ++b) {
      v[b] = f32x8{};
      if (k + b < count) v[b] = load8(src + (long)list[wave][k + b] * d);
    }
#pragma unroll
    for (int b = 0; b < B; ++b) sum += v[b];
  }
  if (wave > 0) others[wave - 1][lane] = sum;
  __syncthreads();
  if (wave == 0 && col < d) {
    sum = sum + others[0][lane] + others[1][lane] + others[2][lane];
    write_sum(d_table + (long)token * d + col, sum, scale, accumulate);
  }
}

template <typename T, typename TG>
__global__ void __launch_bounds__(256) sum_kernel(const uint2* __restrict__ pairs, const T* __restrict__ dy, int n, int d, int V, float scale, TG* __restrict__ d_table,
                                                  int accumulate, int chunk, int chunks, int slabs, int sum_groups, float* __restrict__ parts) {
  constexpr int B = 8;                      // rows in flight
  const int lane = threadIdx.x & 63;
  if ((int)blockIdx.x >= sum_groups) {      // rows without a token
    __shared__ unsigned empty;
    const int row0 = ((int)blockIdx.x - sum_groups) * kZeroRows, rows = min(kZeroRows, V - row0);
    if (threadIdx.x < 64) {
      bool none = false;
      if (lane < rows) {
        const int at = lower_bound(pairs, n, (unsigned)(row0 + lane));
        none = at == n || pairs[at].x != (unsigned)(row0 + lane);
      }
      const unsigned mask = (unsigned)__ballot(none);
      if (lane == 0) empty = mask;
    }
    __syncthreads();
    for (int r = 0; r < rows; ++r)
      if (empty >> r & 1) zero_row(d_table + (long)(row0 + r) * d, d);
    return;
  }
  const long task = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + (threadIdx.x >> 6)));
  const int c = (int)(task / slabs), slab = (int)(task - (long)c * slabs);
  if (c >= chunks) return;
  const int first = c * chunk, count = min(chunk, n - first), col = slab * kSlab + lane * 8;
  const bool live = col < d;
  if (pairs[first].x >= (unsigned)V) return;                             // padding, to the end
  // (lanes past the width go along with the last columns and write nothing)
  const T* src = dy + min(col, d - 8);
  const uint2 mine = pairs[first + min(lane, count - 1)];
  const unsigned key_before = first > 0 ? pairs[first - 1].x : ~0u, key_after = first + count < n ? pairs[first + count].x : ~0u;
  f32x8 sum = {};
  int begin = 0;                            // of the open run
  for (int i0 = 0; i0 < count; i0 += B) {
    f32x8 v[B];
#pragma unroll
    for (int b = 0; b < B; ++b) {
      const int i = min(i0 + b, count - 1);
      const unsigned at = (unsigned)__builtin_amdgcn_readlane((int)mine.y, i);
      v[b] = load8(src + (long)at * d);
    }
#pragma unroll
    for (int b = 0; b < B; ++b) {
      const int i = i0 + b;
      if (i >= count) break;
      const unsigned key = (unsigned)__builtin_amdgcn_readlane((int)mine.x, i);
      sum += v[b];
      const bool last = i + 1 == count;
      const unsigned next = last ? key_after : (unsigned)__builtin_amdgcn_readlane((int)mine.x, min(i + 1, 63));
      if (next == key && !last) continue;
      const bool begins = begin > 0 || key_before != key, ends = next != key;
      if (key < (unsigned)V && live) {
        if (begins && ends) write_sum(d_table + (long)key * d + col, sum, scale, accumulate);
        else {
          float* p = parts + ((long)c * 2 + (begins ? 1 : 0)) * d + col;
          *reinterpret_cast<f32x8 __attribute__((aligned(16)))*>(p) = sum;
        }
      }
      sum = f32x8{};
      begin = i + 1;
    }
  }
}

// Adds the parts of a run that goes over several chunks: the workgroup of the chunk where it begins, four waves in turn.
template <typename TG>
__global__ void __launch_bounds__(256) join_kernel(const uint2* __restrict__ pairs, int n, int d, int V, float scale, TG* __restrict__ d_table, int accumulate, int chunk,
                                                   int slabs, const float* __restrict__ parts) {
  __shared__ f32x8 others[3][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int c = blockIdx.x / slabs, slab = blockIdx.x - c * slabs;
  const int last = (c + 1) * chunk - 1;
  if (last + 1 >= n) return;
  const unsigned key = pairs[last].x;
  if (key >= (unsigned)V || pairs[last + 1].x != key) return;
  if (pairs[c * chunk].x == key && c > 0 && pairs[c * chunk - 1].x == key) return;      // it began in front
  const int end = (lower_bound(pairs, n, key + 1) - 1) / chunk;                          // the chunk where it ends
  const int col = slab * kSlab + lane * 8;
  f32x8 sum = {};
  if (col < d) {
    if (wave == 0) sum = load8(parts + ((long)c * 2 + 1) * d + col);
    const float* head = parts + (long)(c + 1) * 2 * d + col;
#pragma unroll 4
    for (int j = wave; j < end - c; j += 4) sum += load8(head + (long)j * 2 * d);
  }
  if (wave > 0) others[wave - 1][lane] = sum;
  __syncthreads();
  if (wave == 0 && col < d) {
    sum += others[0][lane] + others[1][lane] + others[2][lane];
    write_sum(d_table + (long)key * d + col, sum, scale, accumulate);
  }
}

template <typename T, typename TG>
int sums(const int32_t* tokens, const T* dy, int n, int d, int V, float scale, TG* d_table, int accumulate, const EmbeddingPlan& p, char* ws, hipStream_t s) {
  const int slabs = cdiv(d, kSlab);
  if (p.few) {
    const int sum_groups = n * slabs, zero_groups = accumulate ? 0 : cdiv(V, kZeroRows);
    if (sum_groups + zero_groups > 0) {
      few_kernel<T, TG><<<dim3(sum_groups + zero_groups), dim3(256), 0, s>>>(tokens, dy, n, d, V, scale, d_table, accumulate, slabs, sum_groups);
      MOE_LAUNCH_CHECK();
    }
    return MOE_OK;
  }
  const uint2* pairs = reinterpret_cast<const uint2*>(ws + p.pairs);
  float* parts = reinterpret_cast<float*>(ws + p.parts);
  const int sum_groups = cdiv(p.chunks * slabs, 4), zero_groups = accumulate || p.zero_first ? 0 : cdiv(V, kZeroRows);
  if (sum_groups + zero_groups > 0) {
    sum_kernel<T, TG><<<dim3(sum_groups + zero_groups), dim3(256), 0, s>>>(pairs, dy, n, d, V, scale, d_table, accumulate, p.chunk, p.chunks, slabs, sum_groups, parts);
    MOE_LAUNCH_CHECK();
  }
  if (p.chunks > 1) {
    join_kernel<TG><<<dim3((p.chunks - 1) * slabs), dim3(256), 0, s>>>(pairs, n, d, V, scale, d_table, accumulate, p.chunk, slabs, parts);
    MOE_LAUNCH_CHECK();
  }
  return MOE_OK;
}

}  // namespace

// How each gradient is taken (us, bf16 rows, fp32 gradient, T x d, V words all alike):
//   few tokens without a sort, or sorted: 16 x 4096, 32000 92, 108; 1024 x 1024, 5000 8.2, 24.8; 2048 x 1024, 5000 12.4, 26.6; 1024 x 4096, 32000, added to what is
//   there 17, 27; 2048 x 4096 40, 34 and 4096 x 1024 28, 28: every workgroup looks at every token, so workgroups times tokens are bounded
//   the sort by one workgroup, or by one per tile: 2500 x 512, 5000 25, 39; 4096 x 4096, 32000 117, 145; 8192 x 4096 137, 145
//   all rows zeroed beside that sort, whose CU leaves the others idle, or those without a token behind it: 4096 x 4096, 32000 117, 127; 8192 x 4096 137, 142 to 147;
//   of words that are used twice on average it writes too much twice
//   chunks of 64, or of 8: 65536 x 4096 266, 335 and 65536 x 1024 85, 107; of few tokens they do not fill the chip (4096 x 1024, 5000 44 with the tiled sort, 28)
EmbeddingPlan embedding_plan(int T, int d, int V) {
  EmbeddingPlan p{};
  const int slabs = cdiv(d, kSlab);
  p.chunk = 64;
  while (p.chunk > 8 && (long)cdiv(T, p.chunk) * slabs < 2048) p.chunk /= 2;
  p.chunks = cdiv(T, p.chunk);
  int key_bits = 1;
  while (key_bits < 31 && (V >> key_bits) != 0) ++key_bits;      // keys 0..V
  p.passes = cdiv(key_bits, kMaxDigit);
  p.bits = cdiv(key_bits, p.passes);
  p.tiles = T <= kSortOne && key_bits <= kOneBits ? 0 : cdiv(T, kSortTile);
  p.few = T <= kFewTokens && (long)T * T * slabs <= kFewLooks;
  p.zero_first = p.tiles == 0 && T <= V / 2;
  const size_t list = align_up((size_t)T * sizeof(uint2), 256);
  p.pairs = 0;
  p.counts = p.tiles ? 2 * list : list;
  p.parts = p.counts + align_up((size_t)p.tiles * kBins * 4, 256);
  p.bytes = p.parts + (p.chunks > 1 ? (size_t)p.chunks * 2 * d * 4 : 0) + 256;
  return p;
}

int launch_embedding_fwd(const void* table, const int32_t* tokens, moe_dtype dt, int T, int d, int V, float scale, void* out, hipStream_t s) {
  const long units = (long)T * (d / 8);
  const dim3 grid((unsigned)((units + 1023) / 1024));
  if (dt == MOE_F32) lookup_kernel<float><<<grid, dim3(256), 0, s>>>(static_cast<const float*>(table), tokens, units, d / 8, V, scale, static_cast<float*>(out));
  else lookup_kernel<bf16><<<grid, dim3(256), 0, s>>>(static_cast<const bf16*>(table), tokens, units, d / 8, V, scale, static_cast<bf16*>(out));
  MOE_LAUNCH_CHECK();
  return MOE_OK;
}

int launch_embedding_bwd(const int32_t* tokens, const void* dy, moe_dtype dt, int T, int d, int V, float scale, void* d_table, moe_dtype grad_dt,
                         int accumulate, const EmbeddingPlan& p, char* ws, hipStream_t s) {
  uint2* pairs = reinterpret_cast<uint2*>(ws + p.pairs);
  if (!p.few && p.tiles == 0) {
    const long units = accumulate || !p.zero_first ? 0 : (long)V * d * (long)dtype_size(grad_dt) / 16;
    const long groups = (units + 4095) / 4096;
    sort_one_kernel<<<dim3((unsigned)(1 + (groups < 2048 ? groups : 2048))), dim3(1024), 0, s>>>(tokens, T, V, p.passes, p.bits, pairs,
                                                                                              static_cast<u32x4*>(d_table), units);
    MOE_LAUNCH_CHECK();
  } else if (!p.few) {
    uint2* lists[2] = {pairs, reinterpret_cast<uint2*>(ws + p.counts / 2)};
    unsigned* counts = reinterpret_cast<unsigned*>(ws + p.counts);
    const uint2* from = nullptr;
    for (int pass = 0; pass < p.passes; ++pass) {
      uint2* to = lists[(p.passes - 1 - pass) & 1];              // the last pass ends in the first list
      sort_count_kernel<<<dim3(p.tiles), dim3(1024), 0, s>>>(tokens, from, T, V, pass * p.bits, p.bits, counts);
      MOE_LAUNCH_CHECK();
      sort_place_kernel<<<dim3(p.tiles), dim3(1024), 0, s>>>(tokens, from, T, V, pass * p.bits, p.bits, counts, to);
      MOE_LAUNCH_CHECK();
      from = to;
    }
  }
  if (dt == MOE_F32) return sums(tokens, static_cast<const float*>(dy), T, d, V, scale, static_cast<float*>(d_table), accumulate, p, ws, s);
  if (grad_dt == MOE_F32) return sums(tokens, static_cast<const bf16*>(dy), T, d, V, scale, static_cast<float*>(d_table), accumulate, p, ws, s);
  return sums(tokens, static_cast<const bf16*>(dy), T, d, V, scale, static_cast<bf16*>(d_table), accumulate, p, ws, s);
}

}  // namespace moe
