// Layer norm of rows of M, with the residual's addition in front of it:
//   h = x (+ res), mu = mean(h), r = 1 / sqrt(mean((h - mu)^2) + eps), n = (h - mu) r,
//   y = n gain + bias,
// and its gradients, with u = dy gain:
//   dh = r (u - mean(u) - n mean(u n)) (+ d_sum), dgain = sum of dy n, dbias = sum of dy.
// HBM bounds both: about ten operations an element.
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

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

// rows a block works on side by side, and its threads
template <int W>
constexpr int kRows = W < 4 ? 4 / W : 1;
template <int W>
constexpr int kThreads = W < 4 ? 256 : 64 * W;

// elements of a row in wave w of its W waves, V vectors a thread
template <int W, int V>
__device__ __forceinline__ int wave_count(int M, int w) {
  int n = 0;
#pragma unroll
  for (int v = 0; v < V; ++v) n += min(max(M - 512 * (w + W * v), 0), 512);
  return n;
}

template <typename T, int W, int V, bool NT>
__global__ __launch_bounds__(kThreads<W>) void layer_norm_kernel(LnArgs a) {
  constexpr int G = kRows<W>;
  __shared__ float red[2][G * W][2];
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6),
            w = wv % W, g = wv / W;
  int c[V];
  bool in[V];
  float gn[V][8], bs[V][8];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    c[v] = 8 * (lane + 64 * (w + W * v));
    in[v] = c[v] < a.M;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      gn[v][i] = in[v] && a.gain ? a.gain[c[v] + i] : 1.0f;
      bs[v][i] = in[v] && a.bias ? a.bias[c[v] + i] : 0.0f;
    }
  }
  const int nw = wave_count<W, V>(a.M, w);
  const float rn = nw > 0 ? 1.0f / nw : 0.0f;
  int ph = 0;
  for (long r0 = (long)blockIdx.x * G; r0 < a.rows; r0 += (long)gridDim.x * G, ph ^= 1) {
    const long r = r0 + g;
    const bool row = r < a.rows;
    float h[V][8], s = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const bool on = row && in[v];
      float t[8] = {};
#pragma unroll
      for (int i = 0; i < 8; ++i) h[v][i] = 0.0f;
      if (on) load8(static_cast<const T*>(a.x) + r * a.M + c[v], h[v]);
      if (on && a.res) load8(static_cast<const T*>(a.res) + r * a.M + c[v], t);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        h[v][i] += t[i];
        s += h[v][i];
      }
    }
    float mu = wave_sum(s) * rn, m2 = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float d = in[v] ? h[v][i] - mu : 0.0f;
        m2 += d * d;
      }
    m2 = wave_sum(m2);
    if constexpr (W > 1) {
      if (lane == 0) {
        red[ph][wv][0] = mu;
        red[ph][wv][1] = m2;
      }
      __syncthreads();
      float t = 0.0f;
#pragma unroll
      for (int k = 0; k < W; ++k) t += wave_count<W, V>(a.M, k) * red[ph][g * W + k][0];
      mu = t * a.rm;
      m2 = 0.0f;
#pragma unroll
      for (int k = 0; k < W; ++k) {
        const float d = red[ph][g * W + k][0] - mu;
        m2 += red[ph][g * W + k][1] + wave_count<W, V>(a.M, k) * d * d;
      }
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

template <typename T, int W, int V, bool NT>
__global__ __launch_bounds__(kThreads<W>) void layer_norm_bwd_kernel(LnArgs a) {
  constexpr int G = kRows<W>, NTH = kThreads<W>;
  __shared__ float red[2][G * W][4];
  __shared__ float cols[G > 1 ? 2 * 512 * W * V : 1];
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6),
            w = wv % W, g = wv / W;
  int c[V];
  bool in[V];
  float gn[V][8], dg[V][8], db[V][8];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    c[v] = 8 * (lane + 64 * (w + W * v));
    in[v] = c[v] < a.M;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      gn[v][i] = in[v] && a.gain ? a.gain[c[v] + i] : 1.0f;
      dg[v][i] = db[v][i] = 0.0f;
    }
  }
  const int nw = wave_count<W, V>(a.M, w);
  const float rn = nw > 0 ? 1.0f / nw : 0.0f;
  int ph = 0;
  for (long r0 = (long)blockIdx.x * G; r0 < a.rows; r0 += (long)gridDim.x * G, ph ^= 1) {
    const long r = r0 + g;
    const bool row = r < a.rows;
    float h[V][8], d[V][8], s = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
#pragma unroll
      for (int i = 0; i < 8; ++i) h[v][i] = d[v][i] = 0.0f;
      if (row && in[v]) {
        load8(static_cast<const T*>(a.x) + r * a.M + c[v], h[v]);
        load8(static_cast<const T*>(a.dy) + r * a.M + c[v], d[v]);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) s += h[v][i];
    }
    float mu = wave_sum(s) * rn, m2 = 0.0f, su = 0.0f, sx = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float e = in[v] ? h[v][i] - mu : 0.0f, u = d[v][i] * gn[v][i];
        m2 += e * e;
        su += u;
        sx += u * e;
      }
    m2 = wave_sum(m2);
    su = wave_sum(su);
    sx = wave_sum(sx);
    if constexpr (W > 1) {
      if (lane == 0) {
        red[ph][wv][0] = mu;
        red[ph][wv][1] = m2;
        red[ph][wv][2] = su;
        red[ph][wv][3] = sx;
      }
      __syncthreads();
      float t = 0.0f;
#pragma unroll
      for (int k = 0; k < W; ++k) t += wave_count<W, V>(a.M, k) * red[ph][g * W + k][0];
      mu = t * a.rm;
      m2 = su = sx = 0.0f;
#pragma unroll
      for (int k = 0; k < W; ++k) {
        const float* p = red[ph][g * W + k];
        const float e = p[0] - mu;
        m2 += p[1] + wave_count<W, V>(a.M, k) * e * e;
        su += p[2];
        sx += p[3] + e * p[2];  // u (h - mu) = u (h - mu_w) + u (mu_w - mu)
      }
    }
    const float rs = rsqrtf(m2 * a.rm + a.eps);
    const float c1 = su * a.rm, c2 = sx * a.rm * rs;  // mean(u), mean(u n)
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if (!(row && in[v])) continue;
      float t[8] = {};
      if (a.d_sum) load8(static_cast<const T*>(a.d_sum) + r * a.M + c[v], t);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float n = (h[v][i] - mu) * rs, dd = d[v][i];
        dg[v][i] += dd * n;
        db[v][i] += dd;
        t[i] += rs * (dd * gn[v][i] - c1 - n * c2);
      }
      store8_t<NT>(static_cast<T*>(a.y) + r * a.M + c[v], t);
    }
  }
  if (a.part == nullptr && a.dgain == nullptr && a.dbias == nullptr) return;
  // the block's rows side by side, in order
  if constexpr (G > 1) {
    for (int k = 1; k < G; ++k) {
      __syncthreads();
      if (g == k)
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            cols[c[v] + i] = dg[v][i];
            cols[512 * W * V + c[v] + i] = db[v][i];
          }
      __syncthreads();
      if (g == 0)
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            dg[v][i] += cols[c[v] + i];
            db[v][i] += cols[512 * W * V + c[v] + i];
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
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (a.dgain) a.dgain[c[v] + i] = (a.accumulate ? a.dgain[c[v] + i] : 0.0f) + dg[v][i];
        if (a.dbias) a.dbias[c[v] + i] = (a.accumulate ? a.dbias[c[v] + i] : 0.0f) + db[v][i];
      }
    }
  }
  (void)NTH;
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

// waves a row
int ln_waves(int M) {
  int w = 1;
  while (1024 * w < M) w *= 2;
  return w;
}

int ln_blocks(long rows, int M, int most) {
  const long per = std::max(4 / ln_waves(M), 1), need = (rows + per - 1) / per;
  return (int)std::min(need, (long)most);
}
int ln_bwd_blocks(long rows, int M) {
  const int n = ln_blocks(rows, M, 512);
  return n <= 4 ? 1 : n;
}

#define FLOWMOE_LN_CASE(KERNEL, T, W, V)                                                        \
  if (nt) hipLaunchKernelGGL((KERNEL<T, W, V, true>), dim3(n), dim3(kThreads<W>), 0, st, a);    \
  else hipLaunchKernelGGL((KERNEL<T, W, V, false>), dim3(n), dim3(kThreads<W>), 0, st, a);      \
  break
#define FLOWMOE_LN_LAUNCH(KERNEL, T)                                \
  switch (ln_waves(a.M)) {                                          \
    case 1:                                                         \
      if (a.M <= 512) {                                             \
        FLOWMOE_LN_CASE(KERNEL, T, 1, 1);                           \
      } else {                                                      \
        FLOWMOE_LN_CASE(KERNEL, T, 1, 2);                           \
      }                                                             \
    case 2: FLOWMOE_LN_CASE(KERNEL, T, 2, 2);                       \
    case 4: FLOWMOE_LN_CASE(KERNEL, T, 4, 2);                       \
    case 8: FLOWMOE_LN_CASE(KERNEL, T, 8, 2);                       \
    default: FLOWMOE_LN_CASE(KERNEL, T, 16, 2);                     \
  }

}  // namespace

size_t layer_norm_ws_bytes(int T, int M) {
  const int n = ln_bwd_blocks(T, M);
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
  const int n = ln_blocks(T, M, 2048);
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
  const int n = T == 0 ? 0 : ln_bwd_blocks(T, M);
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
