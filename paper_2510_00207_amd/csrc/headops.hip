// Operators on the heads of a row: rotary positions (arXiv 2104.09864) and the RMS norm
// of each head, forward and backward. Both are bound by memory: every element is read
// once and written once, in 16-byte vectors.
#include <math.h>

#include "common.hpp"

namespace flowmoe {
namespace {

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

constexpr int kRopeTokens = 4;  // tokens of a block

// 8 elements at any element's address (half of rot_dim need be no multiple of a vector;
// global memory takes 16-byte accesses there)
template <typename T>
struct __attribute__((packed, aligned(sizeof(T)))) Any8 {
  u32x4v_t v[sizeof(T) / 2];
};
__device__ __forceinline__ void load8_any(const bf16_t* p, float v[8]) {
  raw8_f32(Raw8b{reinterpret_cast<const Any8<bf16_t>*>(p)->v[0]}, v);
}
__device__ __forceinline__ void load8_any(const float* p, float v[8]) {
  const Any8<float>* q = reinterpret_cast<const Any8<float>*>(p);
  raw8_f32(Raw8f{q->v[0], q->v[1]}, v);
}
__device__ __forceinline__ void store8_any(bf16_t* p, const float v[8]) {
  reinterpret_cast<Any8<bf16_t>*>(p)->v[0] =
      u32x4v_t{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]),
               pack_bf16x2(v[6], v[7])};
}
__device__ __forceinline__ void store8_any(float* p, const float v[8]) {
  Any8<float>* q = reinterpret_cast<Any8<float>*>(p);
#pragma unroll
  for (int i = 0; i < 2; ++i)
    q->v[i] = u32x4v_t{__float_as_uint(v[4 * i]), __float_as_uint(v[4 * i + 1]),
                       __float_as_uint(v[4 * i + 2]), __float_as_uint(v[4 * i + 3])};
}

// A block's threads first make the cosines and sines of its tokens, once for all heads,
// then walk the heads in pieces. HALF: 8 pairs, 8 columns of each half of rot_dim, and
// then the copied columns by eights; the last piece of either may be short. Pairs: 8
// columns, of which those past rot_dim turn by nothing.
template <typename T, bool HALF>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a) {
  extern __shared__ float2 table[];  // kRopeTokens x (rot / 2, rounded up to 4)
  const int half = a.rot / 2, tw = (half + 3) & ~3, t0 = blockIdx.x * kRopeTokens,
            nt = min(kRopeTokens, a.T - t0);
  for (int i = threadIdx.x; i < tw; i += 256) {
    const double f = pair_turns(a, i);
    for (int t = 0; t < nt; ++t) {
      const int p = a.pos ? a.pos[t0 + t] : (t0 + t) % a.seq_len;
      const double turns = (double)p * f;
      float s, c;
      sincospif(2.0f * (float)(turns - rint(turns)), &s, &c);
      table[t * tw + i] = i < half ? make_float2(c * a.mscale, s * a.mscale * a.sign)
                                   : make_float2(1.0f, 0.0f);
    }
  }
  __syncthreads();
  // a head's pieces: np of turned columns, the others copied
  const int np = HALF ? (half + 7) / 8 : (a.rot + 7) / 8;
  const int rest = HALF ? a.rot : 8 * np;  // the first column that is only copied
  const int n = np + (a.copy ? (a.D - rest + 7) / 8 : 0);
  for (int k = threadIdx.x; k < n * a.heads * nt; k += 256) {
    const int c = k % n, r = k / n, hd = r % a.heads, t = r / a.heads;
    const long at = (long)(t0 + t) * a.ld + (long)hd * a.D;
    const T* x = static_cast<const T*>(a.x) + at;
    T* y = static_cast<T*>(a.y) + at;
    float u[8], p[8];
    if (c >= np) {
      const int e = rest + 8 * (c - np);
      if (e + 8 <= a.D) {
        load8_any(x + e, u);
        store8_any(y + e, u);
      } else {
        for (int i = e; i < a.D; ++i) y[i] = x[i];
      }
      continue;
    }
    const float2* cs = table + t * tw + c * (HALF ? 8 : 4);
    if constexpr (HALF) {
      if (8 * c + 8 <= half) {
        float v[8], q[8];
        load8(x + 8 * c, u);
        load8_any(x + half + 8 * c, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          p[i] = u[i] * cs[i].x - v[i] * cs[i].y;
          q[i] = u[i] * cs[i].y + v[i] * cs[i].x;
        }
        store8(y + 8 * c, p);
        store8_any(y + half + 8 * c, q);
      } else {
        for (int i = 8 * c; i < half; ++i, ++cs) {
          const float v = Elem<T>::load(x + i), w = Elem<T>::load(x + half + i);
          Elem<T>::store(y + i, v * cs->x - w * cs->y);
          Elem<T>::store(y + half + i, v * cs->y + w * cs->x);
        }
      }
    } else {
      load8(x + 8 * c, u);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        p[2 * i] = u[2 * i] * cs[i].x - u[2 * i + 1] * cs[i].y;
        p[2 * i + 1] = u[2 * i] * cs[i].y + u[2 * i + 1] * cs[i].x;
      }
      store8(y + 8 * c, p);
    }
  }
}

template <typename T>
void run_rope(const RopeArgs& a, bool half_layout, hipStream_t st) {
  const dim3 g((unsigned)((a.T + kRopeTokens - 1) / kRopeTokens)), b(256);
  const size_t lds = (size_t)kRopeTokens * ((a.rot / 2 + 3) & ~3) * sizeof(float2);
  if (half_layout) hipLaunchKernelGGL((rope_kernel<T, true>), g, b, lds, st, a);
  else hipLaunchKernelGGL((rope_kernel<T, false>), g, b, lds, st, a);
}

// ---------------------------------------------------------------------------
// head norm
// ---------------------------------------------------------------------------
struct NormArgs {
  const void *x, *dy;
  const float* gain;  // D, or null (ones)
  void* y;            // dx in the backward
  float* part;        // backward: blocks x D partial sums of dgain, or null
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

// L lanes (a power of two) hold a head's D <= 8 L elements, 8 each
template <typename T, int L>
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
    if (in) store8(static_cast<T*>(a.y) + r * a.D + c, v);
  }
}

// dx = r (u - x r^2 mean(u x)), u = scale gain dy; dgain's sums over the block's rows go
// to `part`, in a fixed order
template <typename T, int L>
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
    if (in) store8(static_cast<T*>(a.y) + r * a.D + c, v);
  }
  if (a.part == nullptr) return;
#pragma unroll
  for (int i = 0; i < 8; ++i) sums[threadIdx.x * 8 + i] = dg[i];
  __syncthreads();
  for (int i = threadIdx.x; i < a.D; i += 256) {
    float s = 0.0f;
    for (int k = 0; k < 256 / L; ++k) s += sums[k * 8 * L + i];
    a.part[(long)blockIdx.x * a.D + i] = s;
  }
}

// dgain = (or +=) scale x the sum of n partial rows: a wave a column
__global__ __launch_bounds__(64) void head_norm_join_kernel(const float* part, int n, int D,
                                                            float scale, float* dgain,
                                                            int accumulate) {
  const int c = blockIdx.x;
  float s = 0.0f;
  for (int k = threadIdx.x; k < n; k += 64) s += part[(long)k * D + c];
  s = scale * group_sum<64>(s);
  if (threadIdx.x == 0) dgain[c] = accumulate ? dgain[c] + s : s;
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

#define FLOWMOE_NORM_LAUNCH(KERNEL, T)                                                    \
  switch (norm_lanes(a.D)) {                                                               \
    case 4: hipLaunchKernelGGL((KERNEL<T, 4>), g, b, 0, st, a); break;                     \
    case 8: hipLaunchKernelGGL((KERNEL<T, 8>), g, b, 0, st, a); break;                     \
    case 16: hipLaunchKernelGGL((KERNEL<T, 16>), g, b, 0, st, a); break;                   \
    case 32: hipLaunchKernelGGL((KERNEL<T, 32>), g, b, 0, st, a); break;                   \
    default: hipLaunchKernelGGL((KERNEL<T, 64>), g, b, 0, st, a); break;                   \
  }

}  // namespace

hipError_t launch_rope(const RopeShape& m, int dtype, int T, long ld, bool back, const void* x,
                       const int32_t* pos, void* y, hipStream_t st) {
  if (T == 0) return hipSuccess;
  if ((T + kRopeTokens - 1) / kRopeTokens > kMaxBlocks) return hipErrorInvalidConfiguration;
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
  return T == 0 ? 0 : align256((size_t)norm_blocks((long)T * heads, D) * D * sizeof(float));
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
  a.part = dgain != nullptr ? static_cast<float*>(ws) : nullptr;
  a.rows = (long)T * m.heads;
  a.D = m.D;
  a.eps = m.eps;
  a.scale = m.scale;
  const int n = norm_blocks(a.rows, a.D);
  if (T > 0) {
    const dim3 g(n), b(256);
    const hipError_t e = traced(FLOWMOE_K_HEAD_NORM_BWD, st, [&] {
      if (dtype == FLOWMOE_BF16) FLOWMOE_NORM_LAUNCH(head_norm_bwd_kernel, bf16_t)
      else FLOWMOE_NORM_LAUNCH(head_norm_bwd_kernel, float)
    });
    if (e != hipSuccess) return e;
  }
  if (dgain == nullptr) return hipSuccess;
  return traced(FLOWMOE_K_HEAD_NORM_BWD, st, [&] {
    hipLaunchKernelGGL(head_norm_join_kernel, dim3(a.D), dim3(64), 0, st, a.part, n, a.D, a.scale,
                       dgain, accumulate);
  });
}

}  // namespace flowmoe
