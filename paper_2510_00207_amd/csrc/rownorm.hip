// Layer norm of rows of M, with the residual's addition in front of it:
//   h = x (+ res), mu = mean(h), r = 1 / sqrt(mean((h - mu)^2) + eps), n = (h - mu) r,
//   y = n gain + bias,
// and its gradients, with u = dy gain:
//   dh = r (u - mean(u) - n mean(u n)) (+ d_sum), dgain = sum of dy n, dbias = sum of dy.
// HBM bounds both: about ten operations an element. 16384 rows of 4096 bf16 with a residual (537
// MB): forward 93 us, 5.8 TB/s, backward 100, 5.4, with the join's 5.
//
// A row is W waves, V vectors of 8 elements a thread, all in registers, so that every
// element is read once and the squares are of deviations from the mean. The waves of a row
// share their sums in one exchange: each finds its own part's mean and the sums of
// deviations from that, and the parts' sums combine to the row's (the parallel form of
// the variance: M2 = sum of M2_w + n_w (mu_w - mu)^2).
#include <algorithm>

#include "common.hpp"

namespace flowmoe {
namespace {

struct LnArgs {
  const void* x;
  const void* res;    // forward: added to x; nullable
  const void* dy;     // backward
  const void* d_sum;  // backward: added to dx; nullable
  const float* gain;  // nullable
  const float* bias;  // nullable
  void* sum;          // forward: x + res; nullable
  void* y;            // forward y, backward dx
  float* part;        // backward: gridDim.x rows of [dgain | dbias], or null
  float *dgain, *dbias;  // backward: where one block runs, or null
  long rows;
  int M;
  float eps, rm;  // rm = 1 / M
  int accumulate;
};

// the sum over the L lanes of a row (its part)
template <int L>
__device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
  for (int o = L / 2; o > 0; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

// 8 floats of a gain or bias, which may be aligned to 4 bytes only
__device__ __forceinline__ bool aligned16(const void* p) { return (reinterpret_cast<unsigned long>(p) & 15) == 0; }
__device__ __forceinline__ void load_param(const float* p, int c, bool on, float other, float v[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = other;
  if (p == nullptr || !on) return;
  if (aligned16(p)) {
    load8(p + c, v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = p[c + i];
  }
}
// d = v, or d += v
__device__ __forceinline__ void store_grad(float* d, int c, const float v[8], bool add) {
  if (d == nullptr) return;
  float o[8];
  if (aligned16(d)) {
    if (add) load8(d + c, o);
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = add ? o[i] + v[i] : v[i];
    store8(d + c, o);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) d[c + i] = add ? d[c + i] + v[i] : v[i];
  }
}

// a row's vectors as stored, loaded a row ahead of their use (the forward above 125 -> 101 us, the
// backward 155 -> 102)
template <typename T>
using Raw8 = decltype(raw8_load(static_cast<const T*>(nullptr)));
template <typename T, int V>
__device__ __forceinline__ void load_row(Raw8<T> (&q)[V], const void* x, long r, bool row, int M,
                                         const int (&c)[V], const bool (&in)[V]) {
#pragma unroll
  for (int v = 0; v < V; ++v) {
    q[v] = Raw8<T>{};
    if (row && in[v]) q[v] = raw8_load(static_cast<const T*>(x) + r * M + c[v]);
  }
}

// threads of a block, and the rows it works on side by side
template <int L, int W>
constexpr int kThreads = W < 4 ? 256 : 64 * W;
template <int L, int W>
constexpr int kRows = kThreads<L, W> / (L * W);

// elements of a row in part w of its W waves (of L lanes), V vectors a thread
template <int L, int W, int V>
__device__ __forceinline__ int part_count(int M, int w) {
  int n = 0;
#pragma unroll
  for (int v = 0; v < V; ++v) n += min(max(M - 8 * L * (w + W * v), 0), 8 * L);
  return n;
}

template <typename T, int L, int W, int V, bool NT>
__global__ __launch_bounds__((kThreads<L, W>)) void layer_norm_kernel(LnArgs a) {
  constexpr int G = kRows<L, W>;
  __shared__ float red[2][W > 1 ? G * W : 1][2];
  const int lane = threadIdx.x % L, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6),
            w = W > 1 ? wv % W : 0, g = W > 1 ? wv / W : threadIdx.x / L;
  int c[V];
  bool in[V];
  float gn[V][8], bs[V][8];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    c[v] = 8 * (lane + L * (w + W * v));
    in[v] = c[v] < a.M;
    load_param(a.gain, c[v], in[v], 1.0f, gn[v]);
    load_param(a.bias, c[v], in[v], 0.0f, bs[v]);
  }
  const int nw = part_count<L, W, V>(a.M, w);
  const float rn = nw > 0 ? 1.0f / nw : 0.0f;
  int ph = 0;
  const long step = (long)gridDim.x * G;
  Raw8<T> qx[V], qr[V];
  load_row<T>(qx, a.x, (long)blockIdx.x * G + g, (long)blockIdx.x * G + g < a.rows, a.M, c, in);
  load_row<T>(qr, a.res, (long)blockIdx.x * G + g,
              a.res && (long)blockIdx.x * G + g < a.rows, a.M, c, in);
  for (long r0 = (long)blockIdx.x * G; r0 < a.rows; r0 += step, ph ^= 1) {
    const long r = r0 + g;
    const bool row = r < a.rows, next = r + step < a.rows;
    float h[V][8], t[V][8], s = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      raw8_f32(qx[v], h[v]);
      raw8_f32(qr[v], t[v]);
    }
    load_row<T>(qx, a.x, r + step, next, a.M, c, in);
    load_row<T>(qr, a.res, r + step, a.res && next, a.M, c, in);
#pragma unroll
    for (int v = 0; v < V; ++v) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        h[v][i] += t[v][i];
        s += h[v][i];
      }
    }
    float mu = lanes_sum<L>(s) * rn, m2 = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float d = in[v] ? h[v][i] - mu : 0.0f;
        m2 += d * d;
      }
    m2 = lanes_sum<L>(m2);
    if constexpr (W > 1) {
      if (lane == 0) {
        red[ph][wv][0] = mu;
        red[ph][wv][1] = m2;
      }
      __syncthreads();
      // (a lane a part)
      const int k = lane % W, nk = part_count<L, W, V>(a.M, k);
      const float* p = red[ph][g * W + k];
      mu = lanes_sum<W>(nk * p[0]) * a.rm;
      m2 = lanes_sum<W>(p[1] + nk * (p[0] - mu) * (p[0] - mu));
    }
    const float rs = rsqrtf(m2 * a.rm + a.eps);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if (!(row && in[v])) continue;
      if (a.sum) store8_t<NT>(static_cast<T*>(a.sum) + r * a.M + c[v], h[v]);
#pragma unroll
      for (int i = 0; i < 8; ++i) h[v][i] = (h[v][i] - mu) * rs * gn[v][i] + bs[v][i];
      store8_t<NT>(static_cast<T*>(a.y) + r * a.M + c[v], h[v]);
    }
  }
}

template <typename T, int L, int W, int V, bool NT>
__global__ __launch_bounds__((kThreads<L, W>)) void layer_norm_bwd_kernel(LnArgs a) {
  constexpr int G = kRows<L, W>;
  __shared__ float red[2][W > 1 ? G * W : 1][4];
  __shared__ float cols[G > 1 ? 2 * 8 * L * W * V : 1];
  // (rows of 16 waves leave no registers for a row ahead, nor for the gains)
  constexpr bool AHEAD = W < 16;
  __shared__ __attribute__((aligned(16))) float gains[AHEAD ? 4 : 8 * L * W * V];
  const int lane = threadIdx.x % L, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6),
            w = W > 1 ? wv % W : 0, g = W > 1 ? wv / W : threadIdx.x / L;
  int c[V];
  bool in[V];
  float gn[AHEAD ? V : 1][8], dg[V][8], db[V][8];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    c[v] = 8 * (lane + L * (w + W * v));
    in[v] = c[v] < a.M;
    if constexpr (AHEAD) {
      load_param(a.gain, c[v], in[v], 1.0f, gn[v]);
    } else {
      float t[8];
      load_param(a.gain, c[v], in[v], 1.0f, t);
      store8(gains + c[v], t);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) dg[v][i] = db[v][i] = 0.0f;
  }
  const int nw = part_count<L, W, V>(a.M, w);
  const float rn = nw > 0 ? 1.0f / nw : 0.0f;
  int ph = 0;
  const long step = (long)gridDim.x * G;
  Raw8<T> qx[V], qd[V], qs[V];
  if constexpr (AHEAD) {
    const long r = (long)blockIdx.x * G + g;
    load_row<T>(qx, a.x, r, r < a.rows, a.M, c, in);
    load_row<T>(qd, a.dy, r, r < a.rows, a.M, c, in);
    load_row<T>(qs, a.d_sum, r, a.d_sum && r < a.rows, a.M, c, in);
  }
  for (long r0 = (long)blockIdx.x * G; r0 < a.rows; r0 += step, ph ^= 1) {
    const long r = r0 + g;
    const bool row = r < a.rows, next = r + step < a.rows;
    float h[V][8], d[V][8], t[V][8], s = 0.0f;
    if constexpr (!AHEAD) {
      load_row<T>(qx, a.x, r, row, a.M, c, in);
      load_row<T>(qd, a.dy, r, row, a.M, c, in);
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
      raw8_f32(qx[v], h[v]);
      raw8_f32(qd[v], d[v]);
      if constexpr (AHEAD) raw8_f32(qs[v], t[v]);
#pragma unroll
      for (int i = 0; i < 8; ++i) s += h[v][i];
    }
    if constexpr (AHEAD) {
      load_row<T>(qx, a.x, r + step, next, a.M, c, in);
      load_row<T>(qd, a.dy, r + step, next, a.M, c, in);
      load_row<T>(qs, a.d_sum, r + step, a.d_sum && next, a.M, c, in);
    } else {
      load_row<T>(qs, a.d_sum, r, a.d_sum && row, a.M, c, in);
    }
    float mu = lanes_sum<L>(s) * rn, m2 = 0.0f, su = 0.0f, sx = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float e = in[v] ? h[v][i] - mu : 0.0f, u = d[v][i] * (AHEAD ? gn[AHEAD ? v : 0][i] : gains[c[v] + i]);
        m2 += e * e;
        su += u;
        sx += u * e;
      }
    m2 = lanes_sum<L>(m2);
    su = lanes_sum<L>(su);
    sx = lanes_sum<L>(sx);
    if constexpr (W > 1) {
      if (lane == 0) {
        red[ph][wv][0] = mu;
        red[ph][wv][1] = m2;
        red[ph][wv][2] = su;
        red[ph][wv][3] = sx;
      }
      __syncthreads();
      // (a lane a part)
      const int k = lane % W, nk = part_count<L, W, V>(a.M, k);
      const float* p = red[ph][g * W + k];
      mu = lanes_sum<W>(nk * p[0]) * a.rm;
      const float e = p[0] - mu;
      m2 = lanes_sum<W>(p[1] + nk * e * e);
      su = lanes_sum<W>(p[2]);
      sx = lanes_sum<W>(p[3] + e * p[2]);  // u (h - mu) = u (h - mu_w) + u (mu_w - mu)
    }
    const float rs = rsqrtf(m2 * a.rm + a.eps);
    const float c1 = su * a.rm, c2 = sx * a.rm * rs;  // mean(u), mean(u n)
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if (!(row && in[v])) continue;
      if constexpr (!AHEAD) raw8_f32(qs[v], t[v]);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float n = (h[v][i] - mu) * rs, dd = d[v][i];
        dg[v][i] += dd * n;
        db[v][i] += dd;
        t[v][i] += rs * (dd * (AHEAD ? gn[AHEAD ? v : 0][i] : gains[c[v] + i]) - c1 - n * c2);
      }
      store8_t<NT>(static_cast<T*>(a.y) + r * a.M + c[v], t[v]);
    }
  }
  if (a.part == nullptr && a.dgain == nullptr && a.dbias == nullptr) return;
  // the block's rows side by side, in order
  if constexpr (G > 1) {
    const int groups = (int)min((long)G, a.rows);  // (the others have no rows)
    for (int k = 1; k < groups; ++k) {
      __syncthreads();
      if (g == k)
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            cols[c[v] + i] = dg[v][i];
            cols[8 * L * W * V + c[v] + i] = db[v][i];
          }
      __syncthreads();
      if (g == 0)
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            dg[v][i] += cols[c[v] + i];
            db[v][i] += cols[8 * L * W * V + c[v] + i];
          }
    }
    if (g != 0) return;
  }
#pragma unroll
  for (int v = 0; v < V; ++v) {
    if (!in[v]) continue;
    if (a.part != nullptr) {
      float* p = a.part + (long)blockIdx.x * 2 * a.M + c[v];
      store8(p, dg[v]);
      store8(p + a.M, db[v]);
    } else {
      store_grad(a.dgain, c[v], dg[v], a.accumulate != 0);
      store_grad(a.dbias, c[v], db[v], a.accumulate != 0);
    }
  }
}

// dgain and dbias = (or +=) the sums of n partial rows [dgain | dbias]: blocks of 64
// columns, whose 16 waves take every 16th row each, added in order
__global__ __launch_bounds__(1024) void layer_norm_join_kernel(const float* part, int n, int M,
                                                               float* dgain, float* dbias,
                                                               int accumulate) {
  __shared__ float sums[16][64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
  float s = 0.0f;
  if (c < 2 * M) {
#pragma unroll 8
    for (int k = w; k < n; k += 16) s += part[(long)k * 2 * M + c];
  }
  sums[w][lane] = s;
  __syncthreads();
  if (w != 0 || c >= 2 * M) return;
  s = 0.0f;
#pragma unroll
  for (int k = 0; k < 16; ++k) s += sums[k][lane];
  float* d = c < M ? dgain : dbias;
  if (d == nullptr) return;
  const int i = c < M ? c : c - M;
  d[i] = accumulate ? d[i] + s : s;
}

// lanes (of one wave) and waves a row
int ln_lanes(int M) {
  int l = 8;
  while (l < 64 && 8 * l < M) l *= 2;
  return l;
}
int ln_waves(int M) {
  int w = 1;
  while (1024 * w < M) w *= 2;
  return w;
}

// Blocks: as many as have 4 MB of rows in flight (each a row or a few, and the next), at least
// one to a CU. us of the forward and backward with 256, 512, 1024 and 2048 blocks: 16384 x 4096
// bf16 131, 102, 110, 109 and 146, 103, 120, 127; f32 208, 259, 253, 233 and 211, 221, 224, 230;
// 65536 x 256 bf16 82, 48, 32, 33 and 88, 52, 39, 44.
int ln_blocks(long rows, int M, int es, int most) {
  const int lw = ln_lanes(M) * ln_waves(M);
  const long per = std::max(256 / lw, 1), need = (rows + per - 1) / per;
  const long fill = std::min(std::max((4L << 20) / (per * M * es), 256L), (long)most);
  return (int)std::min(need, fill);
}
// (up to four steps of one block need no join: a launch)
int ln_bwd_blocks(long rows, int M, int es) {
  const int n = ln_blocks(rows, M, es, 1024);
  return n <= 4 ? 1 : n;
}

#define FLOWMOE_LN_CASE(KERNEL, T, L, W, V)                                                    \
  {                                                                                            \
    const dim3 g(n), b(kThreads<L, W>);                                                        \
    if (nt) hipLaunchKernelGGL((KERNEL<T, L, W, V, true>), g, b, 0, st, a);                    \
    else hipLaunchKernelGGL((KERNEL<T, L, W, V, false>), g, b, 0, st, a);                      \
    break;                                                                                     \
  }
#define FLOWMOE_LN_LAUNCH(KERNEL, T)                                        \
  switch (a.M <= 512 ? -ln_lanes(a.M) : ln_waves(a.M)) {                    \
    case -8: FLOWMOE_LN_CASE(KERNEL, T, 8, 1, 1)                            \
    case -16: FLOWMOE_LN_CASE(KERNEL, T, 16, 1, 1)                          \
    case -32: FLOWMOE_LN_CASE(KERNEL, T, 32, 1, 1)                          \
    case -64: FLOWMOE_LN_CASE(KERNEL, T, 64, 1, 1)                          \
    case 1: FLOWMOE_LN_CASE(KERNEL, T, 64, 1, 2)                            \
    case 2: FLOWMOE_LN_CASE(KERNEL, T, 64, 2, 2)                            \
    case 4: FLOWMOE_LN_CASE(KERNEL, T, 64, 4, 2)                            \
    case 8: FLOWMOE_LN_CASE(KERNEL, T, 64, 8, 2)                            \
    default: FLOWMOE_LN_CASE(KERNEL, T, 64, 16, 2)                          \
  }

}  // namespace

size_t layer_norm_ws_bytes(int T, int M, int dtype) {
  const int n = ln_bwd_blocks(T, M, (int)esize(dtype));
  return T == 0 || n == 1 ? 0 : align256((size_t)n * 2 * M * sizeof(float));
}

hipError_t launch_layer_norm_fwd(int dtype, int T, int M, float eps, const void* x,
                                 const void* res, const float* gain, const float* bias, void* sum,
                                 void* y, hipStream_t st) {
  if (T == 0) return hipSuccess;
  LnArgs a = {};
  a.x = x;
  a.res = res;
  a.gain = gain;
  a.bias = bias;
  a.sum = sum;
  a.y = y;
  a.rows = T;
  a.M = M;
  a.eps = eps;
  a.rm = 1.0f / M;
  const int n = ln_blocks(T, M, (int)esize(dtype), 2048);
  const bool nt = (2 + (res != nullptr) + (sum != nullptr)) * (long)T * M * (long)esize(dtype) >= (256L << 20);
  return traced(FLOWMOE_K_LAYER_NORM, st, [&] {
    if (dtype == FLOWMOE_BF16) FLOWMOE_LN_LAUNCH(layer_norm_kernel, bf16_t)
    else FLOWMOE_LN_LAUNCH(layer_norm_kernel, float)
  });
}

hipError_t launch_layer_norm_bwd(int dtype, int T, int M, float eps, const void* x,
                                 const float* gain, const void* dy, const void* d_sum, void* dx,
                                 float* dgain, float* dbias, int accumulate, void* ws,
                                 hipStream_t st) {
  LnArgs a = {};
  a.x = x;
  a.dy = dy;
  a.d_sum = d_sum;
  a.gain = gain;
  a.y = dx;
  a.rows = T;
  a.M = M;
  a.eps = eps;
  a.rm = 1.0f / M;
  a.accumulate = accumulate;
  const bool sums = dgain != nullptr || dbias != nullptr;
  // (without tokens they are sums of no partial rows)
  const int n = T == 0 ? 0 : ln_bwd_blocks(T, M, (int)esize(dtype));
  if (n == 1) {
    a.dgain = dgain;
    a.dbias = dbias;
  } else if (sums) {
    a.part = static_cast<float*>(ws);
  }
  if (T > 0) {
    const bool nt = (3 + (d_sum != nullptr)) * (long)T * M * (long)esize(dtype) >= (256L << 20);
    const hipError_t e = traced(FLOWMOE_K_LAYER_NORM_BWD, st, [&] {
      if (dtype == FLOWMOE_BF16) FLOWMOE_LN_LAUNCH(layer_norm_bwd_kernel, bf16_t)
      else FLOWMOE_LN_LAUNCH(layer_norm_bwd_kernel, float)
    });
    if (e != hipSuccess) return e;
  }
  if (!sums || n == 1) return hipSuccess;
  return traced(FLOWMOE_K_LAYER_NORM_BWD, st, [&] {
    hipLaunchKernelGGL(layer_norm_join_kernel, dim3((2 * M + 63) / 64), dim3(1024), 0, st, a.part,
                       n, M, dgain, dbias, accumulate);
  });
}

}  // namespace flowmoe
