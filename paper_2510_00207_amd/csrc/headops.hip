// Operators on the heads of a row: rotary positions (arXiv 2104.09864) and the RMS norm
// of each head, forward and backward. Both are bound by memory: every element is read
// once and written once, in 16-byte vectors.
#include <math.h>

#include "common.hpp"

namespace flowmoe {
namespace {

// Non-temporal stores, for calls that move at least 256 MB: their lines would evict, from
// the Infinity Cache, input that is still to be read. us, cached and non-temporal, with new
// inputs each pass: 537 MB of rotary positions 110, 107; 403 MB of the norm's backward 77.2,
// 75.8; 268 MB of its forward 50.3, 48.8; 50 MB of positions 10.5, 11.4. (Copies of the large
// ones' bytes, new buffers each pass, take 99, 74 and 51 us, 5.2-5.4 TB/s.)
bool stream_past_caches(long bytes) { return bytes >= (256L << 20); }

// ---------------------------------------------------------------------------
// rotary positions
// ---------------------------------------------------------------------------
struct RopeArgs {
  const void* x;
  void* y;
  const int32_t* pos;  // T, or null: token t stands at t % seq_len
  int T, heads, D, rot, seq_len;
  long ld;
  int copy;            // the columns past rot are copied (y is not x)
  int bands;
  double step;         // log2(base) * 2 / rot: pair i turns base^(-2 i / rot) a token
  double scale;        // of every angle (linear: 1 / factor)
  double inv_factor;   // bands: the scale of the slow pairs
  double orig, low, high;  // bands: turns over the original length, the ramp's ends
  float mscale, sign;  // of cos and sin; -1 for the backward
};

// Turns per token of pair i. In 64 bits: at position 2^20 an angle in 32 bits is off
// by up to 0.06.
__device__ __forceinline__ double pair_turns(const RopeArgs& a, int i) {
  double f = exp2(-a.step * i) * 0.15915494309189533577;
  if (a.bands) {
    const double g = fmin(fmax((a.orig * f - a.low) / (a.high - a.low), 0.0), 1.0);
    f *= g + (1.0 - g) * a.inv_factor;
  }
  return f * a.scale;
}

// Of 8 columns the first n turned (p), the others as they came, bit for bit: a computed
// copy would spread infinities and NaN and lose the sign of zeros. (n is even.)
template <bool NT>
__device__ __forceinline__ void store_turned(bf16_t* y, const float p[8], const Raw8b& r, int n) {
  u32x4v_t q;
#pragma unroll
  for (int w = 0; w < 4; ++w) q[w] = 2 * w < n ? pack_bf16x2(p[2 * w], p[2 * w + 1]) : r.a[w];
  st16<NT>(reinterpret_cast<u32x4v_t*>(y), q);
}
template <bool NT>
__device__ __forceinline__ void store_turned(float* y, const float p[8], const Raw8f& r, int n) {
  u32x4v_t lo, hi;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    lo[i] = i < n ? __float_as_uint(p[i]) : r.a[i];
    hi[i] = 4 + i < n ? __float_as_uint(p[4 + i]) : r.b[i];
  }
  st16<NT>(reinterpret_cast<u32x4v_t*>(y), lo);
  st16<NT>(reinterpret_cast<u32x4v_t*>(y + 4), hi);
}

// A block's place: n threads hold the vectors (8 columns) of a head, `per` heads are held
// at once, of `tps` tokens; a block has `tokens` tokens.
struct RopeTile {
  int n, per, tps, tokens;
};
__host__ __device__ __forceinline__ RopeTile rope_tile(int D, int heads, int T) {
  RopeTile r;
  r.n = D / 8;
  r.per = 256 / r.n;
  r.tps = heads < r.per ? r.per / heads : 1;
  // (tokens of a block one after the other: one a block while they are few; us of 1 and 4: 64
  // tokens 4.5, 6.7; 1024 of 32 heads of 64 6.2, 7.2; 2048 8.8, 8.4; 1500 of 64 of 128 13.9, 10.6)
  const int few = T <= 1024 ? 1 : 4;
  r.tokens = r.tps > few ? r.tps : few;
  return r;
}

// The cosines and sines of a block's tokens come first, once for all heads. Then a thread
// holds the same 8 columns of one head after another. With pairs (2 i, 2 i + 1) a column's
// partner is its neighbour; with halves (HALF) it is half a rotation away, anywhere in
// another thread's vector, and taken from LDS: element i of thread k lies at i * 256 + k
// there, and the cosines likewise, so that a wave's reads, which all have one distance,
// touch every bank once. 16384 tokens of 64 heads of 128, bf16: 537 MB in 107 us, 5.0 TB/s
// (a copy 5.4); with 122 columns turned the same (409 us with 16-byte accesses to either
// half where it starts, a thread both).
template <typename T, bool HALF, bool NT>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a) {
  extern __shared__ float2 table[];  // tokens x 8 x (pairs / 8, rounded up)
  __shared__ float stage[HALF ? 2 : 1][HALF ? 8 * 256 : 1];
  const RopeTile r = rope_tile(a.D, a.heads, a.T);
  const int half = a.rot / 2, tw = (half + 7) / 8, t0 = blockIdx.x * r.tokens,
            nt = min(r.tokens, a.T - t0), tid = threadIdx.x;
  for (int k = tid; k < half * nt; k += 256) {
    const int i = k % half, t = k / half;
    const int p = a.pos ? a.pos[t0 + t] : (t0 + t) % a.seq_len;
    const double turns = (double)p * pair_turns(a, i);
    float s, c;
    sincospif(2.0f * (float)(turns - rint(turns)), &s, &c);
    table[(t * 8 + i % 8) * tw + i / 8] = make_float2(c * a.mscale, s * a.mscale * a.sign);
  }
  __syncthreads();
  const int c = tid % r.n, h = tid / r.n;
  const int h0 = r.tps > 1 ? h % a.heads : h, tk = r.tps > 1 ? h / a.heads : 0;
  // (threads past the heads, and with y = x those of columns that stay as they are)
  const bool mine = h < r.per && tk < r.tps && (a.copy || 8 * c < a.rot);
  int from[8];  // where the partners lie
  if constexpr (HALF) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int e = 8 * c + i, q = e < half ? e + half : e - half;
      from[i] = h < r.per && e < a.rot ? (q % 8) * 256 + tid - c + q / 8 : i * 256 + tid;
    }
  }
  int step = 0;
  for (int tb = 0; tb < nt; tb += r.tps) {
    const int t = tb + tk;
    const bool live = mine && t < nt;
    float2 cs[8];  // by which the thread's columns and their partners are multiplied
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int e = 8 * c + i, pair = HALF ? (e < half ? e : e - half) : e / 2;
      const bool turn = live && e < a.rot;
      cs[i] = turn ? table[(t * 8 + pair % 8) * tw + pair / 8] : make_float2(1.0f, 0.0f);
      if (HALF ? e < half : i % 2 == 0) cs[i].y = -cs[i].y;
    }
    for (int g = 0; g < a.heads; g += r.tps > 1 ? a.heads : r.per, ++step) {
      const bool in = live && g + h0 < a.heads;
      const long at = (long)(t0 + t) * a.ld + (long)(g + h0) * a.D + 8 * c;
      float u[8], p[8];
      decltype(raw8_load(static_cast<const T*>(nullptr))) x = {};
      if (in) x = raw8_load(static_cast<const T*>(a.x) + at);
      raw8_f32(x, u);
      if constexpr (HALF) {
        float* s = stage[step & 1];
#pragma unroll
        for (int i = 0; i < 8; ++i) s[i * 256 + tid] = u[i];
        __syncthreads();  // (and the reads of the other stage, a step ago, are done)
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = u[i] * cs[i].x + s[from[i]] * cs[i].y;
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = u[i] * cs[i].x + u[i ^ 1] * cs[i].y;
      }
      if (in) store_turned<NT>(static_cast<T*>(a.y) + at, p, x, a.rot - 8 * c);
    }
  }
}

template <typename T>
void run_rope(const RopeArgs& a, bool half_layout, hipStream_t st) {
  const RopeTile r = rope_tile(a.D, a.heads, a.T);
  const dim3 g((unsigned)((a.T + (long)r.tokens - 1) / r.tokens)), b(256);
  const size_t lds = (size_t)r.tokens * 8 * ((a.rot / 2 + 7) / 8) * sizeof(float2);
  const bool nt = stream_past_caches(2L * a.T * a.heads * a.D * (long)sizeof(T));
  if (half_layout) {
    if (nt) hipLaunchKernelGGL((rope_kernel<T, true, true>), g, b, lds, st, a);
    else hipLaunchKernelGGL((rope_kernel<T, true, false>), g, b, lds, st, a);
  } else {
    if (nt) hipLaunchKernelGGL((rope_kernel<T, false, true>), g, b, lds, st, a);
    else hipLaunchKernelGGL((rope_kernel<T, false, false>), g, b, lds, st, a);
  }
}

// ---------------------------------------------------------------------------
// head norm
// ---------------------------------------------------------------------------
struct NormArgs {
  const void *x, *dy;
  const float* gain;  // D, or null (ones)
  void* y;            // dx in the backward
  float* part;        // backward: blocks x D partial sums of dgain, or null
  float* dgain;       // backward of one block: dgain itself, or null
  int accumulate;     // add to it
  long rows;          // tokens x heads
  int D;
  float eps, scale;
};

template <int L>
__device__ __forceinline__ float group_sum(float v) {
#pragma unroll
  for (int m = L / 2; m > 0; m >>= 1) v += __shfl_xor(v, m);
  return v;
}

// L lanes (a power of two) hold a head's D <= 8 L elements, 8 each; a block's groups walk
// the rows. 16384 tokens of 32 heads of 128, bf16: 268 MB in 49 us, 5.5 TB/s (a copy of as
// many bytes 51 us).
template <typename T, int L, bool NT>
__global__ __launch_bounds__(256) void head_norm_kernel(NormArgs a) {
  const int c = 8 * (threadIdx.x % L);
  const bool in = c < a.D;
  float g[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) g[i] = in ? a.scale * (a.gain ? a.gain[c + i] : 1.0f) : 0.0f;
  const long step = (long)gridDim.x * (256 / L);
  const float rd = 1.0f / a.D;
  for (long r = (long)blockIdx.x * (256 / L) + threadIdx.x / L; r < a.rows; r += step) {
    float v[8] = {}, s = 0.0f;
    if (in) load8(static_cast<const T*>(a.x) + r * a.D + c, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) s += v[i] * v[i];
    s = rsqrtf(group_sum<L>(s) * rd + a.eps);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] *= s * g[i];
    if (in) store8_t<NT>(static_cast<T*>(a.y) + r * a.D + c, v);
  }
}

// dx = r (u - x r^2 mean(u x)), u = scale gain dy; dgain's sums over the block's rows go
// to `part`, in a fixed order. As above 403 MB in 76 us, 5.3 TB/s, with the join's 5 us; 512,
// 1024 and 2048 blocks (with an older join of 7) 111, 82 and 91.
template <typename T, int L, bool NT>
__global__ __launch_bounds__(256) void head_norm_bwd_kernel(NormArgs a) {
  __shared__ float sums[256 * 8];
  const int c = 8 * (threadIdx.x % L);
  const bool in = c < a.D;
  float g[8], dg[8] = {};
#pragma unroll
  for (int i = 0; i < 8; ++i) g[i] = in ? a.scale * (a.gain ? a.gain[c + i] : 1.0f) : 0.0f;
  const long step = (long)gridDim.x * (256 / L);
  const float rd = 1.0f / a.D;
  for (long r = (long)blockIdx.x * (256 / L) + threadIdx.x / L; r < a.rows; r += step) {
    float v[8] = {}, d[8] = {}, s = 0.0f, p = 0.0f;
    if (in) {
      load8(static_cast<const T*>(a.x) + r * a.D + c, v);
      load8(static_cast<const T*>(a.dy) + r * a.D + c, d);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      s += v[i] * v[i];
      p += v[i] * d[i] * g[i];
    }
    s = rsqrtf(group_sum<L>(s) * rd + a.eps);
    p = group_sum<L>(p) * rd * s * s;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      dg[i] += d[i] * (v[i] * s);
      v[i] = s * (d[i] * g[i] - v[i] * p);
    }
    if (in) store8_t<NT>(static_cast<T*>(a.y) + r * a.D + c, v);
  }
  if (a.part == nullptr && a.dgain == nullptr) return;
#pragma unroll
  for (int i = 0; i < 8; ++i) sums[threadIdx.x * 8 + i] = dg[i];
  __syncthreads();
  for (int i = threadIdx.x; i < a.D; i += 256) {
    float s = 0.0f;
    for (int k = 0; k < 256 / L; ++k) s += sums[k * 8 * L + i];
    if (a.dgain == nullptr) a.part[(long)blockIdx.x * a.D + i] = s;
    else a.dgain[i] = (a.accumulate ? a.dgain[i] : 0.0f) + a.scale * s;
  }
}

// dgain = (or +=) scale x the sum of n partial rows: a block a column (a wave a column took
// 7 us for 1024 rows)
__global__ __launch_bounds__(256) void head_norm_join_kernel(const float* part, int n, int D,
                                                             float scale, float* dgain,
                                                             int accumulate) {
  __shared__ float sums[4];
  const int c = blockIdx.x;
  float s = 0.0f;
#pragma unroll 4
  for (int k = threadIdx.x; k < n; k += 256) s += part[(long)k * D + c];
  s = group_sum<64>(s);
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    s = scale * ((sums[0] + sums[1]) + (sums[2] + sums[3]));
    dgain[c] = accumulate ? dgain[c] + s : s;
  }
}

int norm_lanes(int D) {
  int l = 4;
  while (8 * l < D) l *= 2;
  return l;
}

// blocks of the norm kernels: up to four to a CU, each walking the rows
int norm_blocks(long rows, int D) {
  const long per = 256 / norm_lanes(D), need = (rows + per - 1) / per;
  return (int)(need < 1024 ? need : 1024);
}
// and of the backward with dgain: one for up to eight steps, which then needs no join (a
// launch; 10.3 us a call with it, 6.9 without)
int norm_bwd_blocks(long rows, int D) {
  const int n = norm_blocks(rows, D);
  return n <= 8 ? 1 : n;
}

#define FLOWMOE_NORM_CASE(KERNEL, T, L)                                          \
  if (nt) hipLaunchKernelGGL((KERNEL<T, L, true>), g, b, 0, st, a);              \
  else hipLaunchKernelGGL((KERNEL<T, L, false>), g, b, 0, st, a);                \
  break
#define FLOWMOE_NORM_LAUNCH(KERNEL, T)                                           \
  switch (norm_lanes(a.D)) {                                                     \
    case 4: FLOWMOE_NORM_CASE(KERNEL, T, 4);                                     \
    case 8: FLOWMOE_NORM_CASE(KERNEL, T, 8);                                     \
    case 16: FLOWMOE_NORM_CASE(KERNEL, T, 16);                                   \
    case 32: FLOWMOE_NORM_CASE(KERNEL, T, 32);                                   \
    default: FLOWMOE_NORM_CASE(KERNEL, T, 64);                                   \
  }

}  // namespace

bool rope_fits(const RopeShape& m, int T) {
  const int tokens = rope_tile(m.D, m.heads, T).tokens;
  return (T + (long)tokens - 1) / tokens <= kMaxBlocks;
}

hipError_t launch_rope(const RopeShape& m, int dtype, int T, long ld, bool back, const void* x,
                       const int32_t* pos, void* y, hipStream_t st) {
  if (T == 0) return hipSuccess;
  if (!rope_fits(m, T)) return hipErrorInvalidConfiguration;
  RopeArgs a = {};
  a.x = x;
  a.y = y;
  a.pos = pos;
  a.T = T;
  a.heads = m.heads;
  a.D = m.D;
  a.rot = m.rot;
  a.seq_len = m.seq_len;
  a.ld = ld;
  a.copy = x != y;
  a.step = log2(m.base) * 2.0 / m.rot;
  a.scale = m.linear;
  a.bands = m.bands;
  a.inv_factor = m.inv_factor;
  a.orig = m.orig;
  a.low = m.low;
  a.high = m.high;
  a.mscale = m.mscale;
  a.sign = back ? -1.0f : 1.0f;
  return traced(FLOWMOE_K_ROPE, st, [&] {
    if (dtype == FLOWMOE_BF16) run_rope<bf16_t>(a, m.half_layout, st);
    else run_rope<float>(a, m.half_layout, st);
  });
}

size_t head_norm_ws_bytes(int T, int heads, int D) {
  const int n = norm_bwd_blocks((long)T * heads, D);
  return T == 0 || n == 1 ? 0 : align256((size_t)n * D * sizeof(float));
}

hipError_t launch_head_norm_fwd(const NormShape& m, int dtype, int T, const void* x,
                                const float* gain, void* y, hipStream_t st) {
  if (T == 0) return hipSuccess;
  NormArgs a = {};
  a.x = x;
  a.gain = gain;
  a.y = y;
  a.rows = (long)T * m.heads;
  a.D = m.D;
  a.eps = m.eps;
  a.scale = m.scale;
  const dim3 g(norm_blocks(a.rows, a.D)), b(256);
  const bool nt = stream_past_caches(2 * a.rows * a.D * (long)esize(dtype));
  return traced(FLOWMOE_K_HEAD_NORM, st, [&] {
    if (dtype == FLOWMOE_BF16) FLOWMOE_NORM_LAUNCH(head_norm_kernel, bf16_t)
    else FLOWMOE_NORM_LAUNCH(head_norm_kernel, float)
  });
}

hipError_t launch_head_norm_bwd(const NormShape& m, int dtype, int T, const void* x,
                                const float* gain, const void* dy, void* dx, float* dgain,
                                int accumulate, void* ws, hipStream_t st) {
  NormArgs a = {};
  a.x = x;
  a.dy = dy;
  a.gain = gain;
  a.y = dx;
  a.rows = (long)T * m.heads;
  a.D = m.D;
  a.eps = m.eps;
  a.scale = m.scale;
  // (without tokens dgain is a sum of no partial rows)
  const int n = T == 0 ? 0 : dgain != nullptr ? norm_bwd_blocks(a.rows, a.D) : norm_blocks(a.rows, a.D);
  const bool one = n == 1;
  a.dgain = one ? dgain : nullptr;
  a.accumulate = accumulate;
  a.part = dgain != nullptr && !one ? static_cast<float*>(ws) : nullptr;
  if (T > 0) {
    const dim3 g(n), b(256);
    const bool nt = stream_past_caches(3 * a.rows * a.D * (long)esize(dtype));
    const hipError_t e = traced(FLOWMOE_K_HEAD_NORM_BWD, st, [&] {
      if (dtype == FLOWMOE_BF16) FLOWMOE_NORM_LAUNCH(head_norm_bwd_kernel, bf16_t)
      else FLOWMOE_NORM_LAUNCH(head_norm_bwd_kernel, float)
    });
    if (e != hipSuccess) return e;
  }
  if (dgain == nullptr || one) return hipSuccess;
  return traced(FLOWMOE_K_HEAD_NORM_BWD, st, [&] {
    hipLaunchKernelGGL(head_norm_join_kernel, dim3(a.D), dim3(256), 0, st, a.part, n, a.D, a.scale,
                       dgain, accumulate);
  });
}

}  // namespace flowmoe
