// Embedding lookup y_t = scale E[id_t] and its gradient dE_v = scale sum of dy_t over the
// tokens t with id_t = v, in ascending order (no atomics on floats). Ids outside the table
// have no row: zeros forward, no gradient.
//
// Both are bound by HBM: the lookup of 16384 rows of 4096 bf16 (179 MB) takes 33 us, 5.5 TB/s. The
// gradient needs a row's tokens side by side: a stable radix sort of (id, t) by 8 bits a pass, then
// sums of equally many tokens a wave, so that an id of thousands of tokens holds no wave up (a
// wave a few rows of the table, each walking its tokens: 32768 x 2048 of 50021 rows 442 us; so
// 139, the sums 38, the rows without tokens and the joins 66, the sort's four launches 20).
#include <algorithm>

#include "common.hpp"

namespace flowmoe {
namespace {

struct EmbedArgs {
  const int32_t* ids;  // forward: T; backward: sorted
  const int32_t* tok;  // backward: their tokens
  const void* table;
  const void* dy;
  void* y;
  float* dtable;
  float* part;  // the runs' parts
  int T, M, V, rows, groups;
  int zero;  // the launch clears the rows without tokens
  float scale;
};

// Lookup: L lanes a token, four tokens a thread in flight.
template <typename T, int L, bool NT>
__global__ __launch_bounds__(256) void embed_kernel(EmbedArgs a) {
  constexpr int P = 256 / L, K = 4;
  const long t0 = (long)blockIdx.x * (P * K) + threadIdx.x / L;
  long row[K];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int id = t0 + k * P < a.T ? a.ids[t0 + k * P] : -1;
    row[k] = id >= 0 && id < a.V ? (long)id * a.M : -1;
  }
  for (int c = 8 * (threadIdx.x % L); c < a.M; c += 8 * L) {
    float v[K][8] = {};
#pragma unroll
    for (int k = 0; k < K; ++k)
      if (row[k] >= 0) load8(static_cast<const T*>(a.table) + row[k] + c, v[k]);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (t0 + k * P >= a.T) break;
#pragma unroll
      for (int i = 0; i < 8; ++i) v[k][i] *= a.scale;
      store8_t<NT>(static_cast<T*>(a.y) + (t0 + k * P) * a.M + c, v[k]);
    }
  }
}

// ---- the sort ------------------------------------------------------------------------
// Keys are ids, V for those outside the table. A block has `per` items in order (a multiple
// of 1024, at most 256 blocks), 1024 at a time, an item a thread.
struct SortArgs {
  const int32_t *key_in, *val_in;  // val_in null: the first pass (val = index, raw ids)
  int32_t *key, *val;
  int32_t* hist;  // blocks x 256
  int T, V, per, shift;
};

__device__ __forceinline__ int sort_key(const SortArgs& a, int i) {
  const int k = a.key_in[i];
  return a.val_in == nullptr && (k < 0 || k >= a.V) ? a.V : k;
}

__global__ __launch_bounds__(1024) void embed_hist_kernel(SortArgs a) {
  __shared__ int cnt[256];
  const int tid = threadIdx.x;
  if (tid < 256) cnt[tid] = 0;
  __syncthreads();
  const int i1 = min((long)a.T, ((long)blockIdx.x + 1) * a.per);
  for (int i = blockIdx.x * a.per + tid; i < i1; i += 1024)
    atomicAdd(&cnt[(sort_key(a, i) >> a.shift) & 255], 1);
  __syncthreads();
  if (tid < 256) a.hist[blockIdx.x * 256 + tid] = cnt[tid];
}

// where this block's items of digit d go from (thread d < 256): the smaller digits' items
// of all blocks, then d's of the blocks before; `tot` d's items of all blocks
__device__ __forceinline__ void digit_bases(int* base, int tot, int before) {
  // an exclusive scan of tot over the first four waves
  __shared__ int sums[4];
  const int tid = threadIdx.x, lane = tid & 63;
  int run = tot;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int v = __shfl_up(run, o);
    if (lane >= o) run += v;
  }
  if (tid < 256 && lane == 63) sums[tid >> 6] = run;
  __syncthreads();
  if (tid < 256) {
    for (int k = 0; k < tid >> 6; ++k) run += sums[k];
    base[tid] = run - tot + before;
  }
  __syncthreads();
}

// items i0 .. i1 - 1, 1024 at a time, to their places from base on, in order
__device__ __forceinline__ void place_items(const SortArgs& a, int i0, int i1, int* base,
                                            int (*cnt)[256]) {
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  for (int t0 = i0; t0 < i1; t0 += 1024) {
    for (int j = tid; j < 16 * 256; j += 1024) cnt[j >> 8][j & 255] = 0;
    __syncthreads();
    const int i = t0 + tid;
    const bool on = i < i1;
    const int key = on ? sort_key(a, i) : 0, val = !on ? 0 : a.val_in ? a.val_in[i] : i;
    const int d = (key >> a.shift) & 255;
    unsigned long same = __ballot(on);  // the wave's items of this digit
#pragma unroll
    for (int b = 0; b < 8; ++b) {
      const unsigned long m = __ballot((d >> b) & 1);
      same &= (d >> b) & 1 ? m : ~m;
    }
    const int rank = __popcll(same & ((1ul << lane) - 1));
    if (on && rank == 0) cnt[w][d] = __popcll(same);
    __syncthreads();
    if (tid < 256) {
      int s = base[tid];
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        const int n = cnt[k][tid];
        cnt[k][tid] = s;
        s += n;
      }
      base[tid] = s;
    }
    __syncthreads();
    if (on) {
      const int p = cnt[w][d] + rank;
      a.key[p] = key;
      a.val[p] = val;
    }
    __syncthreads();
  }
}

__global__ __launch_bounds__(1024) void embed_place_kernel(SortArgs a) {
  __shared__ int base[256];
  __shared__ int cnt[16][256];
  const int tid = threadIdx.x, i0 = blockIdx.x * a.per;
  int tot = 0, before = 0;
  if (tid < 256) {
#pragma unroll 8
    for (int b = 0; b < (int)gridDim.x; ++b) {
      const int n = a.hist[b * 256 + tid];
      tot += n;
      if (b < (int)blockIdx.x) before += n;
    }
  }
  digit_bases(base, tot, before);
  place_items(a, i0, (int)min((long)a.T, (long)i0 + a.per), base, cnt);
}

// Few tokens, in one launch: an item's place is the number of items that sort before it.
// A block finds those of B items, whose keys are scalars: its 16 waves compare them with every
// 16th 64 of all items each, a vector comparison and a scalar count of its mask for 64 pairs.
constexpr int kRankItems = 32;
__global__ __launch_bounds__(1024) void embed_rank_kernel(const int32_t* ids, int32_t* key,
                                                          int32_t* val, int T, int V) {
  constexpr int B = kRankItems, kNone = 0x7FFFFFFE;
  __shared__ int part[16][B];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int b0 = blockIdx.x * B, own = b0 & ~63;
  // (an id of no row sorts as V, a place behind the items before all)
  auto in = [&](int j) { return j < T ? (int)min((unsigned)ids[j], (unsigned)V) : kNone; };
  int k[B], cnt[B];
#pragma unroll
  for (int u = 0; u < B; ++u) {
    k[u] = in(b0 + u);
    cnt[u] = 0;
  }
  int next = in(64 * w + lane);
  for (int j = 64 * w; j < T; j += 1024) {
    const int q = next + (j > own ? 1 : 0);  // (equal ones behind the block sort behind it)
    next = in(j + 1024 + lane);
    if (j == own) {
#pragma unroll
      for (int u = 0; u < B; ++u)
        cnt[u] += __popcll(__ballot(q + (j + lane >= b0 + u ? 1 : 0) <= k[u]));
    } else {
#pragma unroll
      for (int u = 0; u < B; ++u) cnt[u] += __popcll(__ballot(q <= k[u]));
    }
  }
  int n = 0;
#pragma unroll
  for (int u = 0; u < B; ++u) n = lane == u ? cnt[u] : n;
  if (lane < B) part[w][lane] = n;
  __syncthreads();
  const int i = b0 + lane;
  if (w != 0 || lane >= B || i >= T) return;
  n = 0;
#pragma unroll
  for (int u = 0; u < 16; ++u) n += part[u][lane];
  key[n] = in(i);
  val[n] = i;
}

// ---- sums of rows -----------------------------------------------------------------------
// The sorted tokens in chunks of C, a wave a chunk and 512 columns (8 a lane): whatever runs
// of one id it holds, a wave reads the same rows, eight in flight. A run inside a chunk is
// written by its wave; of one that crosses chunks each leaves its part, and the join adds them
// up in order. part: chunks x [a run that began before | a run that goes on] x M.

template <typename T, int C, bool ADD, bool NT>
__device__ __forceinline__ void sum_chunk(const EmbedArgs& a, int ch, int c, int lane) {
  constexpr int B = ADD ? 4 : 8;  // rows in flight (ADD: and what they are added to)
  const bool on = c < a.M;
  // lane l has position ch * C + l - 1: one before the chunk, the chunk, one behind it
  const int p = ch * C + lane - 1;
  const bool there = p >= 0 && p < a.T && lane < C + 2;
  const int id = there ? a.ids[p] : p < 0 ? -1 : 0x7FFFFFFF, tok = there ? a.tok[p] : 0;
  const int before = __shfl_up(id, 1);
  const bool mine = lane >= 1 && lane <= C && id < a.V;
  const int n = __popcll(__ballot(mine));
  // bit k: token k begins, ends a run (the last one: or its part of one)
  const unsigned head = (unsigned)(__ballot(mine && id != before) >> 1);
  const unsigned end = (head >> 1) | (n > 0 ? 1u << (n - 1) : 0u);
  const bool goes_on = n == C && __builtin_amdgcn_readlane(id, C + 1) ==
                                          __builtin_amdgcn_readlane(id, C);
  float acc[8] = {};
  for (int k = 0; k < n; k += B) {
    float v[B][8] = {}, old[ADD ? B : 1][8] = {};
#pragma unroll
    for (int u = 0; u < B; ++u) {
      const int i = min(k + u, n - 1);
      const long t = __builtin_amdgcn_readlane(tok, i + 1);
      if (on) load8(static_cast<const T*>(a.dy) + t * a.M + c, v[u]);
      if constexpr (ADD) {
        const long r = __builtin_amdgcn_readlane(id, i + 1);
        if (on && (end >> i & 1)) load8(a.dtable + r * a.M + c, old[u]);
      }
    }
#pragma unroll
    for (int u = 0; u < B; ++u) {
      const int i = k + u;
      if (i >= n) break;
      const bool first = head >> i & 1;
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] = (first ? 0.0f : acc[e]) + v[u][e];
      if (!(end >> i & 1) || !on) continue;
      const bool began = (head & ((2u << i) - 1)) == 0, open = i == n - 1 && goes_on;
      if (began || open) {
        store8(a.part + (2L * ch + (began ? 0 : 1)) * a.M + c, acc);
      } else {
        const long r = __builtin_amdgcn_readlane(id, i + 1);
        float o[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = ADD ? old[ADD ? u : 0][e] + a.scale * acc[e] : a.scale * acc[e];
        store8_t<NT>(a.dtable + r * a.M + c, o);
      }
    }
  }
}

// the first sorted position whose id is at least v, a wave's search of 64 at a time
__device__ __forceinline__ int first_of(const EmbedArgs& a, int v, int lane) {
  int lo = 0, hi = a.T;  // in lo .. hi
  while (lo < hi) {
    const int step = (hi - lo + 63) / 64, i = lo + lane * step;
    const int n = __popcll(__ballot(i < hi && a.ids[i] < v));
    if (n == 0) return lo;
    hi = min(hi, lo + n * step);
    lo += (n - 1) * step + 1;
  }
  return lo;
}

// zeros in the rows v0 .. v0 + rows - 1 (at most 64) that have no tokens: 16 contiguous bytes a
// lane (32 a lane in two stores: 198 us of the case above, so 150)
template <bool NT>
__device__ __forceinline__ void zero_absent(const EmbedArgs& a, long v0, int lane) {
  const int v1 = (int)min((long)a.V, v0 + a.rows), v = (int)v0 + lane;
  int lo = first_of(a, (int)v0, lane);
  bool absent = v < v1;
  const int q = lo + lane < a.T ? a.ids[lo + lane] : 0x7FFFFFFF;
  if (__builtin_amdgcn_readlane(q, 63) >= v1) {  // the rows' tokens are at most these
    for (int u = 0; u < 64; ++u) {
      const int o = __builtin_amdgcn_readlane(q, u);
      if (o >= v1) break;
      absent = absent && o != v;
    }
  } else {  // each lane searches its own row's first
    const int end = first_of(a, v1, lane);
    int hi = end;
    while (__any(lo < hi)) {
      const int mid = (lo + hi) >> 1;
      const bool less = lo < hi && a.ids[mid] < v;
      if (lo < hi) {
        if (less) lo = mid + 1;
        else hi = mid;
      }
    }
    absent = absent && !(lo < end && a.ids[lo] == v);
  }
  unsigned long m = __ballot(absent);
  if (a.M < 256) {  // narrow rows: the wave's rows as one run of 16-byte vectors
    const int per = a.M / 4, n = (v1 - (int)v0) * per;
    for (int u = lane; u < n; u += 64)
      if (m >> (u / per) & 1)
        st16<NT>(reinterpret_cast<u32x4v_t*>(a.dtable + v0 * a.M + 4 * u), u32x4v_t{0, 0, 0, 0});
    return;
  }
  while (m) {
    const long r = v0 + __builtin_ctzll(m);
    m &= m - 1;
#pragma unroll 4
    for (int c = 4 * lane; c < a.M; c += 256)
      st16<NT>(reinterpret_cast<u32x4v_t*>(a.dtable + r * a.M + c), u32x4v_t{0, 0, 0, 0});
  }
}

// Waves 0 .. chunks * slabs - 1: the chunks' sums, and in the next launch the joins. The waves behind
// them clear the rows without tokens, in one of the two: beside the joins, whose latencies they
// hide, where rows are wide (us beside the sums and so: 16384 tokens of one id, 32000 rows of 1024
// 111, 104; 40000 of 2048, 50021 rows 150, 143), beside the sums where narrow ones take longer for
// their searches than the joins (16384 of 264, 70000 rows 50, 57; of 64, 200000 48, 54).
template <typename T, int C, bool ADD, bool NT>
__global__ __launch_bounds__(256) void embed_bwd_kernel(EmbedArgs a) {
  const int lane = threadIdx.x & 63, slabs = (a.M + 511) / 512;
  const long u = (long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const long sums = ((long)a.T + C - 1) / C * slabs;
  if (u < sums) {
    sum_chunk<T, C, ADD, NT>(a, (int)(u / slabs), (int)(u % slabs) * 512 + 8 * lane, lane);
  } else if constexpr (!ADD) {
    const long v0 = (u - sums) * a.rows;
    if (a.zero && v0 < a.V) zero_absent<NT>(a, v0, lane);
  }
}

// a run that crosses chunks: the wave of the chunk ch where it begins adds up its parts
template <int C, bool ADD>
__device__ __forceinline__ void join_chunk(const EmbedArgs& a, int ch, int c, int lane) {
  const long p = (long)ch * C;
  if (p + C >= a.T) return;
  const int id = a.ids[p + C - 1];
  if (id >= a.V || a.ids[p + C] != id) return;
  if (a.ids[p] == id && p > 0 && a.ids[p - 1] == id) return;  // began before
  const bool on = c < a.M;
  float acc[8] = {}, old[8] = {};
  if (on) load8(a.part + (2L * ch + 1) * a.M + c, acc);
  if (ADD && on) load8(a.dtable + (long)id * a.M + c, old);
  for (int j = ch + 1;; j += 64) {
    const long q = (long)(j + lane) * C;
    const int n = __popcll(__ballot(q < a.T && a.ids[q] == id));
    for (int k = 0; k < n; k += 16) {
      float v[16][8] = {};
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (on) load8(a.part + 2L * (j + min(k + e, n - 1)) * a.M + c, v[e]);
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (k + e < n)
#pragma unroll
          for (int i = 0; i < 8; ++i) acc[i] += v[e][i];
    }
    if (n < 64) break;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) acc[i] = ADD ? old[i] + a.scale * acc[i] : a.scale * acc[i];
  if (on) store8(a.dtable + (long)id * a.M + c, acc);
}

template <int C, bool ADD, bool NT>
__global__ __launch_bounds__(256) void embed_join_kernel(EmbedArgs a) {
  const int lane = threadIdx.x & 63, slabs = (a.M + 511) / 512;
  const long u = (long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const long sums = ((long)a.T + C - 1) / C * slabs;
  if (u < sums) {
    join_chunk<C, ADD>(a, (int)(u / slabs), (int)(u % slabs) * 512 + 8 * lane, lane);
  } else if constexpr (!ADD) {
    const long v0 = (u - sums) * a.rows;
    if (a.zero && v0 < a.V) zero_absent<NT>(a, v0, lane);
  }
}

// ---- very few tokens ----------------------------------------------------------------------
// In one launch, without a sort: `groups` blocks a token look, by all ids (I a thread), whether it
// is the first of its id and sum its id's rows if so, the columns shared out among them: 512 a
// wave, eight rows in flight; of a long run waves sum parts, which are added up in order. The
// other blocks clear the rows without tokens, `rows` of them each. us of 1000 f32 tokens of 264,
// 5003 rows: 6.6 (launches of a sort, the sums and the joins: 15), five of them a launch's least.
constexpr int kFewWaves = 8;  // (1000 tokens of 264, 4, 8 and 16 waves: 8.4, 7.5, 12.9 us)
template <typename T, int I, bool ADD, bool NT>
__global__ __launch_bounds__(64 * kFewWaves) void embed_few_kernel(EmbedArgs a) {
  constexpr int W = kFewWaves, B = 8;
  __shared__ int list[64 * W * I];  // the id's tokens, or which rows have tokens
  __shared__ int cnt[W * I];
  __shared__ __attribute__((aligned(16))) float part[W][512];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int t = blockIdx.x / a.groups, s0 = blockIdx.x % a.groups;
  int ids[I];
#pragma unroll
  for (int k = 0; k < I; ++k) ids[k] = tid + 64 * W * k < a.T ? a.ids[tid + 64 * W * k] : -1;
  if (t >= a.T) {
    if constexpr (!ADD) {
      const long v0 = (blockIdx.x - (long)a.T * a.groups) * a.rows;
      const int n = (int)min((long)a.rows, a.V - v0), per = a.M / 4;
      for (int u = tid; u < n; u += 64 * W) list[u] = 0;
      __syncthreads();
#pragma unroll
      for (int k = 0; k < I; ++k)
        if (ids[k] >= v0 && ids[k] < v0 + n) list[ids[k] - v0] = 1;
      __syncthreads();
      for (int u = tid; u < n * per; u += 64 * W)
        if (list[u / per] == 0)
          st16<NT>(reinterpret_cast<u32x4v_t*>(a.dtable + v0 * a.M + 4L * u), u32x4v_t{0, 0, 0, 0});
    }
    return;
  }
  const int id = a.ids[t];
  if (id < 0 || id >= a.V) return;
  unsigned long same[I];
  bool before = false;
#pragma unroll
  for (int k = 0; k < I; ++k) {
    same[k] = __ballot(ids[k] == id);
    before = before || (ids[k] == id && tid + 64 * W * k < t);
    if (lane == 0) cnt[W * k + w] = __popcll(same[k]);
  }
  if (__syncthreads_or(before)) return;
  int n = 0;
#pragma unroll
  for (int k = 0; k < I; ++k)
#pragma unroll
    for (int u = 0; u < W; ++u) {
      if (u == w && ids[k] == id) list[n + __popcll(same[k] & ((1ul << lane) - 1))] = tid + 64 * W * k;
      n += cnt[W * k + u];
    }
  n = __builtin_amdgcn_readfirstlane(n);
  __syncthreads();
  int P = 1;
  while (P < W && n > 8 * P) P *= 2;
  const int p = w & (P - 1);
  const int k0 = (int)((long)n * p / P), k1 = (int)((long)n * (p + 1) / P);
  for (int c0 = 512 * (W / P) * s0; c0 < a.M; c0 += 512 * (W / P) * a.groups) {
    const int c = c0 + 512 * (w / P) + 8 * lane;
    const bool on = c < a.M;
    float acc[8] = {}, old[8] = {};
    float* const row = a.dtable + (long)id * a.M + c;
    if (ADD && on && p == 0) load8(row, old);
    for (int k = k0; k < k1; k += B) {
      float v[B][8] = {};
#pragma unroll
      for (int u = 0; u < B; ++u) {
        const long j = __builtin_amdgcn_readfirstlane(list[min(k + u, k1 - 1)]);
        if (on && k + u < k1) load8(static_cast<const T*>(a.dy) + j * a.M + c, v[u]);
      }
#pragma unroll
      for (int u = 0; u < B; ++u)
        if (k + u < k1)
#pragma unroll
          for (int i = 0; i < 8; ++i) acc[i] += v[u][i];
    }
    if (P > 1) {
      if (p > 0) store8(part[w] + 8 * lane, acc);
      __syncthreads();
      if (p == 0)
        for (int e = 1; e < P; ++e) {
          float v[8];
          load8(part[w + e] + 8 * lane, v);
#pragma unroll
          for (int i = 0; i < 8; ++i) acc[i] += v[i];
        }
      __syncthreads();
    }
    if (p > 0 || !on) continue;
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i] = ADD ? old[i] + a.scale * acc[i] : a.scale * acc[i];
    store8_t<NT>(row, acc);
  }
}

// ---- host -------------------------------------------------------------------------------
// us so and with a sort: 512 tokens of 1024, 1000 rows 7, 13, 1000 of 2048, 5003 rows 15, 20, of
// 1024, 32000 rows 26, 33. Only a run of most of the tokens is slow, as one or two CUs read it:
// 512 tokens of one id, 32000 rows of 1024 34, 35, 1000 60, 43, added to the gradient 29, 26;
// 2000 lose with ids of any spread (of 4096, 32000 rows 169, 125).
constexpr int kVeryFew = 128 * kFewWaves;
constexpr int kFew = 8192;
int key_passes(int V) {  // keys 0 .. V
  int p = 1;
  while (p < 4 && ((unsigned)V >> (8 * p)) != 0) ++p;
  return p;
}
// Tokens a chunk: few tokens are better served by more waves, many by fewer parts of runs. us
// with 8 and 32: 4096 x 1024, 32000 rows 46,
// 55; 16384 65, 69, all of one id 248, 114; 32768 x 2048, 50021 rows 169, 135.
int embed_chunk(int T) { return T <= kFew ? 8 : 32; }

// Ranked, in one launch, or sorted in two a pass? us of the whole gradient ranked and sorted, rows of
// 264, two passes (5003 rows) and three (70000): 2048 tokens 18, 24 and 28, 40; 4096 22, 26 and
// 31, 44; 8192 29, 31 and 36, 44; 12000 54, 38 and 68, 58. One pass is half of two's.
bool ranked(int T, int V) { return T <= (key_passes(V) > 1 ? 8192 : 2048); }
int sort_per(int T) { return std::max(1, (int)(((long)T + 262143) / 262144)) * 1024; }
int sort_blocks(int T) { return (int)(((long)T + sort_per(T) - 1) / sort_per(T)); }

struct EmbedWs {
  size_t a, b, hist, part, bytes;
};
EmbedWs embed_ws(int T, int M, int V) {
  EmbedWs w;
  const size_t items = align256((size_t)T * 8);
  w.a = 0;
  w.b = items;
  w.hist = 2 * items;
  w.part = w.hist + align256(ranked(T, V) ? 0 : (size_t)sort_blocks(T) * 1024);
  w.bytes = w.part + align256(((size_t)T + embed_chunk(T) - 1) / embed_chunk(T) * 2 * M * sizeof(float));
  return w;
}

hipError_t sort_tokens(int T, int V, const int32_t* ids, const EmbedWs& w, char* ws, hipStream_t st) {
  const int passes = key_passes(V);
  int32_t* x = reinterpret_cast<int32_t*>(ws + w.b);
  int32_t* y = reinterpret_cast<int32_t*>(ws + w.a);
  if (ranked(T, V))
    return traced(FLOWMOE_K_EMBED_SORT, st, [&] {
      hipLaunchKernelGGL(embed_rank_kernel, dim3((T + kRankItems - 1) / kRankItems), dim3(1024), 0, st, ids, y, y + T, T, V);
    });
  SortArgs a = {ids, nullptr, nullptr, nullptr, reinterpret_cast<int32_t*>(ws + w.hist), T, V,
                sort_per(T), 0};
  for (int p = 0; p < passes; ++p) {
    int32_t* out = (passes - 1 - p) % 2 ? x : y;
    a.key = out;
    a.val = out + T;
    a.shift = 8 * p;
    const dim3 g(sort_blocks(T)), b(1024);
    const hipError_t e = traced(FLOWMOE_K_EMBED_SORT, st, [&] {
      hipLaunchKernelGGL(embed_hist_kernel, g, b, 0, st, a);
      hipLaunchKernelGGL(embed_place_kernel, g, b, 0, st, a);
    });
    if (e != hipSuccess) return e;
    a.key_in = out;
    a.val_in = out + T;
  }
  return hipSuccess;
}

int embed_lanes(int M) {
  int l = 8;
  while (l < 256 && 8 * l < M) l *= 2;
  return l;
}

}  // namespace

// Rows of the table that a wave looks at for those without tokens: 1024 waves or more (1500 tokens
// of 264, 5003 rows: 64 rows a wave 22 us, 4 18).
static int embed_rows(int M, int V) {
  return std::max(4, std::min(M >= 512 ? 16 : 64, V / 1024));
}
static long embed_waves(int T, int M, int V, bool add) {
  const long slabs = (M + 511) / 512;
  return ((long)T + embed_chunk(T) - 1) / embed_chunk(T) * slabs +
         (add ? 0 : (V + embed_rows(M, V) - 1L) / embed_rows(M, V));
}

bool embed_fits(int T, int M, int V) {
  const long f = 4 * (256 / embed_lanes(M));
  return (T + f - 1) / f <= kMaxBlocks && (embed_waves(T, M, V, false) + 3) / 4 <= kMaxBlocks;
}

size_t embed_ws_bytes(int T, int M, int V) {
  return T <= kVeryFew ? 0 : embed_ws(T, M, V).bytes;
}

hipError_t launch_embed_fwd(int dtype, int T, int M, int V, float scale, const int32_t* ids,
                            const void* table, void* y, hipStream_t st) {
  if (T == 0) return hipSuccess;
  EmbedArgs a = {};
  a.ids = ids;
  a.table = table;
  a.y = y;
  a.T = T;
  a.M = M;
  a.V = V;
  a.scale = scale;
  const int L = embed_lanes(M), per = 4 * (256 / L);
  const dim3 g((unsigned)((T + (long)per - 1) / per)), b(256);
  const bool nt = 2L * T * M * (long)esize(dtype) >= (256L << 20);
#define FLOWMOE_EMBED_CASE(T, L)                                                \
  if (nt) hipLaunchKernelGGL((embed_kernel<T, L, true>), g, b, 0, st, a);       \
  else hipLaunchKernelGGL((embed_kernel<T, L, false>), g, b, 0, st, a);         \
  break
#define FLOWMOE_EMBED_LAUNCH(T)                 \
  switch (L) {                                  \
    case 8: FLOWMOE_EMBED_CASE(T, 8);           \
    case 16: FLOWMOE_EMBED_CASE(T, 16);         \
    case 32: FLOWMOE_EMBED_CASE(T, 32);         \
    case 64: FLOWMOE_EMBED_CASE(T, 64);         \
    case 128: FLOWMOE_EMBED_CASE(T, 128);       \
    default: FLOWMOE_EMBED_CASE(T, 256);        \
  }
  return traced(FLOWMOE_K_EMBED, st, [&] {
    if (dtype == FLOWMOE_BF16) FLOWMOE_EMBED_LAUNCH(bf16_t)
    else FLOWMOE_EMBED_LAUNCH(float)
  });
}

hipError_t launch_embed_bwd(int dtype, int T, int M, int V, float scale, const int32_t* ids,
                            const void* dy, float* dtable, int accumulate, void* ws,
                            hipStream_t st) {
  if (T == 0 && accumulate) return hipSuccess;
  const EmbedWs w = embed_ws(T, M, V);
  char* base = static_cast<char*>(ws);
  EmbedArgs a = {};
  a.dy = dy;
  a.dtable = dtable;
  a.T = T;
  a.M = M;
  a.V = V;
  a.scale = scale;
  const bool nt = (long)V * M * 4 >= (256L << 20), few = embed_chunk(T) == 8;
  if (T <= kVeryFew) {
    a.ids = ids;
    // (two blocks a token where there are columns for them: 512 tokens of 2048, 5003 rows 16, 12)
    a.groups = M > 512 ? 2 : 1;
    a.rows = std::max({1, std::min({512, V / 256, 8192 / M}), V >> 21});
    const long zero = accumulate ? 0 : (V + (long)a.rows - 1) / a.rows;
    const dim3 g((unsigned)((long)T * a.groups + zero)), b(64 * kFewWaves);
    return traced(FLOWMOE_K_EMBED_BWD, st, [&] {
#define FLOWMOE_EMBED_FEW(T, I)                                                               \
  if (accumulate) hipLaunchKernelGGL((embed_few_kernel<T, I, true, false>), g, b, 0, st, a);  \
  else if (nt) hipLaunchKernelGGL((embed_few_kernel<T, I, false, true>), g, b, 0, st, a);     \
  else hipLaunchKernelGGL((embed_few_kernel<T, I, false, false>), g, b, 0, st, a)
      if (T <= 64 * kFewWaves && dtype == FLOWMOE_BF16) {
        FLOWMOE_EMBED_FEW(bf16_t, 1);
      } else if (T <= 64 * kFewWaves) {
        FLOWMOE_EMBED_FEW(float, 1);
      } else if (dtype == FLOWMOE_BF16) {
        FLOWMOE_EMBED_FEW(bf16_t, 2);
      } else {
        FLOWMOE_EMBED_FEW(float, 2);
      }
    });
  }
  const hipError_t se = sort_tokens(T, V, ids, w, base, st);
  if (se != hipSuccess) return se;
  a.ids = reinterpret_cast<const int32_t*>(base + w.a);
  a.tok = a.ids + T;
  a.part = reinterpret_cast<float*>(base + w.part);
  a.rows = embed_rows(M, V);
  const bool late = M >= 512;  // (clearing beside the joins)
  const dim3 g((unsigned)((embed_waves(T, M, V, accumulate || late) + 3) / 4)), b(256);
  const dim3 gj((unsigned)((embed_waves(T, M, V, accumulate || !late) + 3) / 4));
  a.zero = !late;
  const hipError_t e = traced(FLOWMOE_K_EMBED_BWD, st, [&] {
#define FLOWMOE_EMBED_BWD(T, C)                                                                 \
  if (accumulate) hipLaunchKernelGGL((embed_bwd_kernel<T, C, true, false>), g, b, 0, st, a);    \
  else if (nt) hipLaunchKernelGGL((embed_bwd_kernel<T, C, false, true>), g, b, 0, st, a);       \
  else hipLaunchKernelGGL((embed_bwd_kernel<T, C, false, false>), g, b, 0, st, a)
    if (few && dtype == FLOWMOE_BF16) {
      FLOWMOE_EMBED_BWD(bf16_t, 8);
    } else if (few) {
      FLOWMOE_EMBED_BWD(float, 8);
    } else if (dtype == FLOWMOE_BF16) {
      FLOWMOE_EMBED_BWD(bf16_t, 32);
    } else {
      FLOWMOE_EMBED_BWD(float, 32);
    }
  });
  if (e != hipSuccess) return e;
  a.zero = late;
  return traced(FLOWMOE_K_EMBED_BWD, st, [&] {
#define FLOWMOE_EMBED_JOIN(C)                                                                \
  if (accumulate) hipLaunchKernelGGL((embed_join_kernel<C, true, false>), gj, b, 0, st, a);  \
  else if (nt) hipLaunchKernelGGL((embed_join_kernel<C, false, true>), gj, b, 0, st, a);     \
  else hipLaunchKernelGGL((embed_join_kernel<C, false, false>), gj, b, 0, st, a)
    if (few) {
      FLOWMOE_EMBED_JOIN(8);
    } else {
      FLOWMOE_EMBED_JOIN(32);
    }
  });
}

}  // namespace flowmoe
