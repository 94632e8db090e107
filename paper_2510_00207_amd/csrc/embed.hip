// Embedding lookup y_t = scale E[id_t] and its gradient dE_v = scale sum of dy_t over the
// tokens t with id_t = v, in ascending order (no atomics on floats). Ids outside the table
// have no row: zeros forward, no gradient.
//
// Both are bound by HBM. The gradient needs a row's tokens side by side: a stable radix sort
// of (id, t) by 8 bits a pass, then a wave walks the tokens of its table rows.
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
  float* part;  // sums of chunks of 64 sorted tokens of one id, or null
  int T, M, V, rows;
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
  // an exclusive scan of tot over 256 threads, through LDS
  const int tid = threadIdx.x;
  if (tid < 256) base[tid] = tot;
  __syncthreads();
  for (int o = 1; o < 256; o <<= 1) {
    const int v = tid < 256 && tid >= o ? base[tid - o] : 0;
    __syncthreads();
    if (tid < 256) base[tid] += v;
    __syncthreads();
  }
  if (tid < 256) base[tid] += before - tot;
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
  const int tid = threadIdx.x;
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
  place_items(a, blockIdx.x * a.per, (int)min((long)a.T, ((long)blockIdx.x + 1) * a.per), base, cnt);
}

// every pass in one block, from `in` through x and y in turn; the last pass writes y
__global__ __launch_bounds__(1024) void embed_sort_kernel(const int32_t* in, int32_t* x, int32_t* y,
                                                          int T, int V, int passes) {
  __shared__ int base[256];
  __shared__ int cnt[16][256];
  const int tid = threadIdx.x;
  SortArgs a = {in, nullptr, nullptr, nullptr, nullptr, T, V, T, 0};
  for (int p = 0; p < passes; ++p) {
    int32_t* out = (passes - 1 - p) % 2 ? x : y;
    a.key = out;
    a.val = out + T;
    a.shift = 8 * p;
    if (tid < 256) cnt[0][tid] = 0;
    __syncthreads();
    for (int i = tid; i < T; i += 1024) atomicAdd(&cnt[0][(sort_key(a, i) >> a.shift) & 255], 1);
    __syncthreads();
    const int tot = tid < 256 ? cnt[0][tid] : 0;
    digit_bases(base, tot, 0);
    place_items(a, 0, T, base, cnt);
    __threadfence_block();
    __syncthreads();
    a.key_in = out;
    a.val_in = out + T;
  }
}

// ---- sums of rows -----------------------------------------------------------------------
// 8 columns a lane from c on; `on`: the lane has columns
struct Cols {
  int c;
  bool on;
};

__device__ __forceinline__ void add8(float acc[8], const float v[8], bool on) {
#pragma unroll
  for (int i = 0; i < 8; ++i) acc[i] += on ? v[i] : 0.0f;
}

// acc += dy of the tokens that lanes i0 .. i1 - 1 hold, four rows in flight
template <typename T>
__device__ __forceinline__ void add_tokens(const EmbedArgs& a, Cols s, int tok, int i0, int i1,
                                           float acc[8]) {
  for (int k = i0; k < i1; k += 4) {
    float v[4][8] = {};
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const long t = __builtin_amdgcn_readlane(tok, min(k + u, i1 - 1));
      if (s.on) load8(static_cast<const T*>(a.dy) + t * a.M + s.c, v[u]);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) add8(acc, v[u], k + u < i1);
  }
}

// The sorted tokens 64 at a time: ids and tokens of window `wb`, a lane each (past the last:
// no id's)
struct Window {
  int wb, id, tok;
  __device__ __forceinline__ void load(const EmbedArgs& a, int base, int lane) {
    wb = base;
    const bool there = base + lane < a.T;
    id = there ? a.ids[base + lane] : 0x7FFFFFFF;
    tok = there ? a.tok[base + lane] : 0;
  }
};

// acc = the sum of id v's tokens, the first of which is at or past pos (in window w); pos is
// then behind the last
template <typename T>
__device__ __forceinline__ void sum_id(const EmbedArgs& a, Cols s, int lane, int v, int& pos,
                                       Window& w, float acc[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) acc[i] = 0.0f;
  for (;;) {
    const unsigned long m = __ballot(w.id == v && w.wb + lane >= pos);
    const int n = __popcll(m), i0 = pos - w.wb;
    if (n == 64 && a.part != nullptr) {
      float t[8] = {};
      if (s.on) load8(a.part + (long)(w.wb / 64) * a.M + s.c, t);
      add8(acc, t, true);
    } else {
      add_tokens<T>(a, s, w.tok, i0, i0 + n, acc);
    }
    pos += n;
    if (i0 + n < 64) return;
    w.load(a, w.wb + 64, lane);
  }
}

// the sums of the chunks of 64 sorted tokens that are one id's, a wave a chunk and 512 columns
template <typename T>
__global__ __launch_bounds__(256) void embed_chunk_kernel(EmbedArgs a) {
  const int lane = threadIdx.x & 63, slabs = (a.M + 511) / 512;
  const long u = (long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int ch = (int)(u / slabs), c = (int)(u % slabs) * 512 + 8 * lane;
  if (ch >= a.T / 64) return;
  const int first = a.ids[ch * 64];
  if (first >= a.V || first != a.ids[ch * 64 + 63]) return;
  Window w;
  w.load(a, ch * 64, lane);
  float acc[8] = {};
  const Cols s = {c, c < a.M};
  add_tokens<T>(a, s, w.tok, 0, 64, acc);
  if (s.on) store8(a.part + (long)ch * a.M + c, acc);
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

// The whole table: a wave has `rows` rows of it, 512 columns
template <typename T, bool NT>
__global__ __launch_bounds__(256) void embed_bwd_kernel(EmbedArgs a) {
  const int lane = threadIdx.x & 63, slabs = (a.M + 511) / 512;
  const long u = (long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = (int)(u % slabs) * 512 + 8 * lane;
  const long v0 = u / slabs * a.rows;
  if (v0 >= a.V) return;
  const int v1 = (int)min((long)a.V, v0 + a.rows);
  const Cols s = {c, c < a.M};
  int pos = first_of(a, (int)v0, lane);
  Window w;
  w.load(a, pos & ~63, lane);
  for (int v = (int)v0; v < v1; ++v) {
    float acc[8];
    sum_id<T>(a, s, lane, v, pos, w, acc);
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i] *= a.scale;
    if (s.on) store8_t<NT>(a.dtable + (long)v * a.M + c, acc);
  }
}

// Added to the rows that have tokens: a wave has `rows` sorted positions (a divisor of 64),
// and of them the ids that begin there
template <typename T>
__global__ __launch_bounds__(256) void embed_bwd_add_kernel(EmbedArgs a) {
  const int lane = threadIdx.x & 63, slabs = (a.M + 511) / 512;
  const long u = (long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = (int)(u % slabs) * 512 + 8 * lane;
  const long p0 = u / slabs * a.rows;
  if (p0 >= a.T) return;
  const int p1 = (int)min((long)a.T, p0 + a.rows);
  const Cols s = {c, c < a.M};
  int pos = (int)p0;
  Window w;
  w.load(a, pos & ~63, lane);
  if (pos > 0) {  // an id that began before
    const int v = a.ids[pos - 1];
    const unsigned long m = __ballot(w.id == v && w.wb + lane >= pos);
    pos += __popcll(m);  // (past the window: its last position is past p1 as well)
  }
  while (pos < p1) {
    const int v = __builtin_amdgcn_readlane(w.id, pos - w.wb);
    if (v >= a.V) return;
    float* d = a.dtable + (long)v * a.M + c;
    float acc[8], old[8] = {};
    if (s.on) load8(d, old);
    sum_id<T>(a, s, lane, v, pos, w, acc);
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i] = old[i] + a.scale * acc[i];
    if (s.on) store8(d, acc);
  }
}

// ---- host -------------------------------------------------------------------------------
int key_passes(int V) {  // keys 0 .. V
  int p = 1;
  while (p < 4 && ((unsigned)V >> (8 * p)) != 0) ++p;
  return p;
}
// a block sorts up to 4096 items alone
constexpr int kSortOne = 4096;
int sort_per(int T) {
  return T <= kSortOne ? T : std::max(1, (int)(((long)T + 262143) / 262144)) * 1024;
}
int sort_blocks(int T) { return (int)(((long)T + sort_per(T) - 1) / sort_per(T)); }

struct EmbedWs {
  size_t a, b, hist, part, bytes;
};
EmbedWs embed_ws(int T, int M) {
  EmbedWs w;
  const size_t items = align256((size_t)T * 8);
  w.a = 0;
  w.b = items;
  w.hist = 2 * items;
  w.part = w.hist + align256(T <= kSortOne ? 0 : (size_t)sort_blocks(T) * 1024);
  w.bytes = w.part + align256((size_t)(T / 64) * M * sizeof(float));
  return w;
}

hipError_t sort_tokens(int T, int V, const int32_t* ids, const EmbedWs& w, char* ws, hipStream_t st) {
  const int passes = key_passes(V);
  int32_t* x = reinterpret_cast<int32_t*>(ws + w.b);
  int32_t* y = reinterpret_cast<int32_t*>(ws + w.a);
  if (T <= kSortOne)
    return traced(FLOWMOE_K_EMBED_SORT, st, [&] {
      hipLaunchKernelGGL(embed_sort_kernel, dim3(1), dim3(1024), 0, st, ids, x, y, T, V, passes);
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

// rows of the table that a wave of the gradient has
static int embed_rows(int M) { return M >= 512 ? 8 : 16; }
static constexpr int kAddRows = 8;

bool embed_fits(int T, int M, int V) {
  const long slabs = (M + 511) / 512, f = 4 * (256 / embed_lanes(M));
  const long n = std::max(((V + embed_rows(M) - 1L) / embed_rows(M)), (T + kAddRows - 1L) / kAddRows);
  return (T + f - 1) / f <= kMaxBlocks && (n * slabs + 3) / 4 <= kMaxBlocks;
}

size_t embed_ws_bytes(int T, int M) { return T == 0 ? 0 : embed_ws(T, M).bytes; }

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
  const EmbedWs w = embed_ws(T, M);
  char* base = static_cast<char*>(ws);
  const long slabs = (M + 511) / 512;
  EmbedArgs a = {};
  a.dy = dy;
  a.dtable = dtable;
  a.T = T;
  a.M = M;
  a.V = V;
  a.scale = scale;
  if (T > 0) {
    const hipError_t e = sort_tokens(T, V, ids, w, base, st);
    if (e != hipSuccess) return e;
    a.ids = reinterpret_cast<const int32_t*>(base + w.a);
    a.tok = a.ids + T;
    if (T >= 256) {
      a.part = reinterpret_cast<float*>(base + w.part);
      const dim3 g((unsigned)((T / 64 * slabs + 3) / 4)), b(256);
      const hipError_t e2 = traced(FLOWMOE_K_EMBED_BWD, st, [&] {
        if (dtype == FLOWMOE_BF16) hipLaunchKernelGGL(embed_chunk_kernel<bf16_t>, g, b, 0, st, a);
        else hipLaunchKernelGGL(embed_chunk_kernel<float>, g, b, 0, st, a);
      });
      if (e2 != hipSuccess) return e2;
    }
  }
  a.rows = accumulate ? kAddRows : embed_rows(M);
  const long n = ((accumulate ? T : V) + (long)a.rows - 1) / a.rows;
  const dim3 g((unsigned)((n * slabs + 3) / 4)), b(256);
  const bool nt = (long)V * M * 4 >= (256L << 20);
  return traced(FLOWMOE_K_EMBED_BWD, st, [&] {
    if (accumulate) {
      if (dtype == FLOWMOE_BF16) hipLaunchKernelGGL(embed_bwd_add_kernel<bf16_t>, g, b, 0, st, a);
      else hipLaunchKernelGGL(embed_bwd_add_kernel<float>, g, b, 0, st, a);
    } else if (dtype == FLOWMOE_BF16) {
      if (nt) hipLaunchKernelGGL((embed_bwd_kernel<bf16_t, true>), g, b, 0, st, a);
      else hipLaunchKernelGGL((embed_bwd_kernel<bf16_t, false>), g, b, 0, st, a);
    } else {
      if (nt) hipLaunchKernelGGL((embed_bwd_kernel<float, true>), g, b, 0, st, a);
      else hipLaunchKernelGGL((embed_bwd_kernel<float, false>), g, b, 0, st, a);
    }
  });
}

}  // namespace flowmoe
