// Attention over packed sequences that are short: a tile of 32 rows is one wave's, so that
// a document of a few tokens takes a wave and not a block of four, and many are in flight (LDS:
// two tiles of 32 rows forward, four backward). Longer sequences loop over their tiles,
// one after the other. The tiles, operand forms and softmax are those of attn.hip.
//
// Backward: one kernel. A wave has the keys and the queries of a tile for every query head of a
// key head: dQ^T += K^T dS^T over the key tiles, then dV^T += dO^T P and dK^T += Q^T dS over
// the query tiles; of a sequence of one tile K, V, Q and dO are loaded once for both.
//
// Latency bounds it: a wave waits for its loads, its scores, its softmax, its products in turn. 5000
// tokens in 840 sequences of 1 to 12, 16 heads on 4 of 128: forward 40 us (185 in blocks of 128
// rows), backward 136 (351); 259 in 26 of up to 71, 4 on 2 of 64: 5 and 11.
#include <math.h>

#include "attn_tiles.hpp"
#include "common.hpp"
#include "packed.hpp"

namespace flowmoe {
namespace {

template <int D, bool CAUSAL>
__global__ __launch_bounds__(64, D == 128 ? 3 : 4) void short_fwd_kernel(AttnArgs a) {
  constexpr int KS = D / 16, DB = D / 32;
  using Dma = TileDma<D, 32, 1>;
  constexpr int TB = Dma::TB;
  __shared__ __attribute__((aligned(1024))) char lds[2 * TB];  // K, V
  const int lane = threadIdx.x, h2 = lane >> 5, lq = lane & 31;
  Span sp;
  int unit;
  if (!packed_span(a, a.heads, CAUSAL, 32, 1, lane, blockIdx.x, gridDim.x, sp, unit)) return;
  const long tok0 = sp.tok0, ld = (long)(a.heads + 2 * a.kv) * D;
  const int hd = sp.hd, N = sp.N, q0 = 32 * sp.tile, qw = q0 + lq, g = hd / (a.heads / a.kv);
  if (sp.none) {
    const int n = min(32, N - q0);
    zero_rows(a.out + (long)hd * D, a.M, tok0 + q0, n, D, lane, 64);
    if (lane < n) a.lse[(long)hd * a.T + tok0 + q0 + lane] = 0.0f;
    return;
  }
  const bf16_t* Qg = a.qkv + tok0 * ld + (long)hd * D;
  const bf16_t* Kg = a.qkv + tok0 * ld + (long)(a.heads + g) * D;
  const bf16_t* Vg = Kg + (long)a.kv * D;
  const int kend = CAUSAL ? min(N, q0 + 32) : N;
  const Dma dma(lds_base(lds), 0, lane, ld);
  bf16x8 qf[KS];
#pragma unroll
  for (int i = 0; i < KS; ++i)
    qf[i] = qw < N ? *reinterpret_cast<const bf16x8*>(Qg + qw * ld + 16 * i + 8 * h2) : zero8();
  floatx16 o[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) o[db] = zero16();
  float m = -INFINITY, l = 0.0f;
  const int rbase = row_base<D>(lq, h2), tb0 = tr_base<D>(lane, 0), tb1 = tr_base<D>(lane, 1);
  for (int kb = 0; kb < kend; kb += 32) {
    lds_barrier();  // the last tile's reads are done
    dma.load(Kg + kb * ld, kend - kb, 0);
    dma.load(Vg + kb * ld, kend - kb, TB);
    wait_vm<0>();
    lds_barrier();
    floatx16 s = zero16();
#pragma unroll
    for (int i = 0; i < KS; ++i) s = mfma(frag_row_x<D>(lds, rbase, 0, i), qf[i], s);
    if (kb + 32 > N || (CAUSAL && kb + 31 > q0)) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int key = kb + 8 * (r >> 2) + 4 * h2 + (r & 3);
        if (key >= N || (CAUSAL && key > qw)) s[r] = -INFINITY;
      }
    }
    float mx = s[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) mx = fmaxf(mx, s[r]);
    // (every query sees key 0 in the first tile: m is finite from then on)
    mx = fmaxf(m, pair_max(mx) * a.c2);
    const float al = exp2_fast(m - mx);
    m = mx;
    unsigned pw[8];
    float sum = 0.0f;
#pragma unroll
    for (int r = 0; r < 16; r += 2) {
      const float p0 = exp2_fast(fmaf(s[r], a.c2, -m)), p1 = exp2_fast(fmaf(s[r + 1], a.c2, -m));
      sum += p0;
      sum += p1;
      pw[r >> 1] = pack_bf16x2(p0, p1);
    }
    l = l * al + pair_sum(sum);
    if (kb > 0) {
#pragma unroll
      for (int db = 0; db < DB; ++db) o[db] *= al;
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const bf16x8 pb = __builtin_bit_cast(bf16x8, u32x4{pw[4 * k], pw[4 * k + 1], pw[4 * k + 2], pw[4 * k + 3]});
#pragma unroll
      for (int db = 0; db < DB; ++db)
        o[db] = mfma(frag_tr_x<D>(lds + TB, tb0, tb1, 16 * k, 32 * db), pb, o[db]);
    }
  }
  if (qw < N) {
    const float inv = 1.0f / l;
    bf16_t* Og = a.out + (tok0 + qw) * a.M + (long)hd * D;
#pragma unroll
    for (int db = 0; db < DB; ++db) store_cols(Og + 32 * db, o[db], h2, inv);
    if (h2 == 0) a.lse[(long)hd * a.T + tok0 + qw] = (m + log2f(l)) * kLn2;
  }
}

template <int D, bool CAUSAL, int W>
__global__ __launch_bounds__(64 * W, D == 128 ? 1 : 2) void short_bwd_kernel(AttnArgs a) {
  constexpr int KS = D / 16, DB = D / 32;
  using Dma = TileDma<D, 32, 1>;
  constexpr int TB = Dma::TB, VT = TB, QT = 2 * TB, GT = 3 * TB, ST = 4 * TB;
  // a wave: K, V, Q, dO; 32 lse2, 32 delta
  constexpr int LW = (ST + 256 + 1023) / 1024 * 1024;
  __shared__ __attribute__((aligned(1024))) char all[W * LW];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h2 = lane >> 5,
            lq = lane & 31;
  char* const lds = all + w * LW;
  Span sp;
  int unit;
  if (!packed_span(a, a.kv, false, 32, 1, lane, blockIdx.x, gridDim.x, sp, unit)) return;
  const int nh = a.heads / a.kv, g = sp.hd, N = sp.N, r0 = 32 * sp.tile, rw = r0 + lq;
  const long tok0 = sp.tok0, ld = (long)(a.heads + 2 * a.kv) * D;
  const long kcol = (long)(a.heads + g) * D, vcol = kcol + (long)a.kv * D;
  if (sp.none) {
    if (w > 0) return;
    const int n = min(32, N - r0);
    zero_rows(a.d_qkv + (long)g * nh * D, ld, tok0 + r0, n, nh * D, lane, 64);
    zero_rows(a.d_qkv + kcol, ld, tok0 + r0, n, D, lane, 64);
    zero_rows(a.d_qkv + vcol, ld, tok0 + r0, n, D, lane, 64);
    for (int h = g * nh; h < g * nh + nh; ++h)
      if (lane < n) a.delta[(long)h * a.T + tok0 + r0 + lane] = 0.0f;
    return;
  }
  const bf16_t* X = a.qkv + tok0 * ld;
  const bf16_t* G = a.d_o + tok0 * a.M;
  const bf16_t* O = a.o + tok0 * a.M;
  const Dma dma(lds_base(all) + w * LW, 0, lane, ld), dmag(lds_base(all) + w * LW, 0, lane, a.M);
  const int rbase = row_base<D>(lq, h2), tb0 = tr_base<D>(lane, 0), tb1 = tr_base<D>(lane, 1);
  const bool one = N <= 32;
  // (loads of a tile whose place in LDS is still being read wait for that first)
  auto load_kv = [&](int kb) {
    dma.load(X + kb * ld + kcol, N - kb, 0);
    dma.load(X + kb * ld + vcol, N - kb, VT);
  };
  auto load_qg = [&](int h, int qb) {
    dma.load(X + qb * ld + (long)h * D, N - qb, QT);
    dmag.load(G + (long)qb * a.M + (long)h * D, N - qb, GT);
  };
  // this lane's query of a tile: its delta and base-2 log-sum-exp
  auto stats = [&](int h, int qb, float& dl, float& l2) {
    const int q = qb + lq;
    dl = l2 = 0.0f;
    if (q < N) {
#pragma unroll
      for (int i = 0; i < KS; ++i) {
        const long off = (long)q * a.M + (long)h * D + 16 * i + 8 * h2;
        const bf16x8 gv = *reinterpret_cast<const bf16x8*>(G + off), ov = *reinterpret_cast<const bf16x8*>(O + off);
#pragma unroll
        for (int e = 0; e < 8; ++e) dl += (float)gv[e] * (float)ov[e];
      }
      l2 = a.lse[(long)h * a.T + tok0 + q] * kLog2e;
    }
    dl += __shfl_xor(dl, 32);
  };
  floatx16 dk[DB], dv[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) dk[db] = dv[db] = zero16();

  // dQ of the tile (its queries the accumulators' columns) from the keys kb .. kb + 31
  auto dq_tile = [&](floatx16 (&dq)[DB], int kb, float dl, float l2) {
    floatx16 s = zero16(), dp = zero16();
#pragma unroll
    for (int i = 0; i < KS; ++i) {
      s = mfma(frag_row_x<D>(lds, rbase, 0, i), frag_row_x<D>(lds + QT, rbase, 0, i), s);
      dp = mfma(frag_row_x<D>(lds + VT, rbase, 0, i), frag_row_x<D>(lds + GT, rbase, 0, i), dp);
    }
    unsigned pw[8];
#pragma unroll
    for (int r = 0; r < 16; r += 2) {
      float d[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int key = kb + 8 * (r >> 2) + 4 * h2 + (r & 3) + e;
        const bool on = key < N && (!CAUSAL || key <= rw);
        d[e] = on ? exp2_fast(fmaf(s[r + e], a.c2, -l2)) * (dp[r + e] - dl) : 0.0f;
      }
      pw[r >> 1] = pack_bf16x2(d[0], d[1]);
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const bf16x8 pb = __builtin_bit_cast(bf16x8, u32x4{pw[4 * k], pw[4 * k + 1], pw[4 * k + 2], pw[4 * k + 3]});
#pragma unroll
      for (int db = 0; db < DB; ++db)
        dq[db] = mfma(frag_tr_x<D>(lds, tb0, tb1, 16 * k, 32 * db), pb, dq[db]);
    }
  };
  // dK and dV of the tile (its keys the columns) from the queries qb .. qb + 31
  auto dkdv_tile = [&](int qb) {
    floatx16 s = zero16(), dp = zero16();
#pragma unroll
    for (int i = 0; i < KS; ++i) {
      s = mfma(frag_row_x<D>(lds + QT, rbase, 0, i), frag_row_x<D>(lds, rbase, 0, i), s);
      dp = mfma(frag_row_x<D>(lds + GT, rbase, 0, i), frag_row_x<D>(lds + VT, rbase, 0, i), dp);
    }
    unsigned pp[8], pd[8];
    const float* st = reinterpret_cast<const float*>(lds + ST);
#pragma unroll
    for (int J = 0; J < 4; ++J) {
      const float4 lv = *reinterpret_cast<const float4*>(st + 8 * J + 4 * h2);
      const float4 ev = *reinterpret_cast<const float4*>(st + 32 + 8 * J + 4 * h2);
      const float lr[4] = {lv.x, lv.y, lv.z, lv.w}, er[4] = {ev.x, ev.y, ev.z, ev.w};
      float p[4], d[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int q = qb + 8 * J + 4 * h2 + j;
        const bool on = q < N && (!CAUSAL || q >= rw);
        p[j] = on ? exp2_fast(fmaf(s[4 * J + j], a.c2, -lr[j])) : 0.0f;
        d[j] = on ? p[j] * (dp[4 * J + j] - er[j]) : 0.0f;
      }
#pragma unroll
      for (int j = 0; j < 4; j += 2) {
        pp[2 * J + j / 2] = pack_bf16x2(p[j], p[j + 1]);
        pd[2 * J + j / 2] = pack_bf16x2(d[j], d[j + 1]);
      }
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const bf16x8 bp = __builtin_bit_cast(bf16x8, u32x4{pp[4 * k], pp[4 * k + 1], pp[4 * k + 2], pp[4 * k + 3]});
      const bf16x8 bd = __builtin_bit_cast(bf16x8, u32x4{pd[4 * k], pd[4 * k + 1], pd[4 * k + 2], pd[4 * k + 3]});
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        dv[db] = mfma(frag_tr_x<D>(lds + GT, tb0, tb1, 16 * k, 32 * db), bp, dv[db]);
        dk[db] = mfma(frag_tr_x<D>(lds + QT, tb0, tb1, 16 * k, 32 * db), bd, dk[db]);
      }
    }
  };
  auto keep_stats = [&](float dl, float l2) {
    float* st = reinterpret_cast<float*>(lds + ST);
    st[lane] = h2 ? dl : l2;  // (both lanes of a query have both)
  };

  // (a wave has LDS of its own: no barriers, its reads done before a load's writes, and its loads
  // and writes before the reads)
  auto own_reads = [&] {
    wait_lgkm0();
    asm volatile("" ::: "memory");
  };
  auto own_loads = [&] {
    wait_vm<0>();
    wait_lgkm0();
    asm volatile("" ::: "memory");
  };
  if (one) load_kv(0);
  for (int h = g * nh + w; h < g * nh + nh; h += W) {
    float dl, l2;
    own_reads();
    load_qg(h, r0);
    stats(h, r0, dl, l2);
    if (h2 == 0 && rw < N) a.delta[(long)h * a.T + tok0 + rw] = dl;
    floatx16 dq[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db) dq[db] = zero16();
    if (one) {
      keep_stats(dl, l2);
      own_loads();
      dq_tile(dq, 0, dl, l2);
      dkdv_tile(0);
    } else {
      const int kend = CAUSAL ? min(N, r0 + 32) : N;
      for (int kb = 0; kb < kend; kb += 32) {
        own_reads();
        load_kv(kb);
        own_loads();
        dq_tile(dq, kb, dl, l2);
      }
    }
    if (rw < N) {
      bf16_t* dst = a.d_qkv + (tok0 + rw) * ld + (long)h * D;
#pragma unroll
      for (int db = 0; db < DB; ++db) store_cols(dst + 32 * db, dq[db], h2, a.rs);
    }
  }
  if (!one) {
    own_reads();
    load_kv(r0);
    for (int h = g * nh + w; h < g * nh + nh; h += W)
      for (int qb = CAUSAL ? r0 : 0; qb < N; qb += 32) {
        float dl, l2;
        own_reads();
        load_qg(h, qb);
        stats(h, qb, dl, l2);
        keep_stats(dl, l2);
        own_loads();
        dkdv_tile(qb);
      }
  }
  if constexpr (W > 1) {
    // the waves' sums, in order
    static_assert(2 * DB * 16 * 256 <= LW, "the sums fit a wave's LDS");
    own_loads();
    if (w > 0) {
      float* p = reinterpret_cast<float*>(lds) + lane;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          p[(16 * db + r) * 64] = dk[db][r];
          p[(16 * (DB + db) + r) * 64] = dv[db][r];
        }
    }
    lds_barrier();
    if (w > 0) return;
#pragma unroll 1
    for (int e = 1; e < W; ++e) {
      const float* p = reinterpret_cast<const float*>(all + e * LW) + lane;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          dk[db][r] += p[(16 * db + r) * 64];
          dv[db][r] += p[(16 * (DB + db) + r) * 64];
        }
    }
  }
  if (rw < N) {
    bf16_t* dst = a.d_qkv + (tok0 + rw) * ld;
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      store_cols(dst + kcol + 32 * db, dk[db], h2, a.rs);
      store_cols(dst + vcol + 32 * db, dv[db], h2, 1.0f);
    }
  }
}

unsigned short_blocks(const PackedShape& m, int T, int per) {
  return (unsigned)((T / 32 + (long)m.nseq + 1) * per);
}

// Few tiles of a key head leave room for a wave each of up to four of a group's query heads. us of
// the backward with one wave a block and so: 20 tokens in 2 sequences, 16 heads on 2 of 128 35, 18,
// on 4 of 64 12, 8; 1000 in 98, 16 on 2 of 128 (258 tiles) 40, 34; 2500 in 252 (650) 51, 68.
constexpr unsigned kFewTiles = 512;
template <int D>
void run_short_fwd(const PackedShape& m, const AttnArgs& a, hipStream_t st) {
  const dim3 g(short_blocks(m, a.T, m.heads)), b(64);
  if (m.causal) hipLaunchKernelGGL((short_fwd_kernel<D, true>), g, b, 0, st, a);
  else hipLaunchKernelGGL((short_fwd_kernel<D, false>), g, b, 0, st, a);
}
template <int D, int W>
void run_short_bwd(const PackedShape& m, const AttnArgs& a, hipStream_t st) {
  const dim3 g(short_blocks(m, a.T, m.kv)), b(64 * W);
  if (m.causal) hipLaunchKernelGGL((short_bwd_kernel<D, true, W>), g, b, 0, st, a);
  else hipLaunchKernelGGL((short_bwd_kernel<D, false, W>), g, b, 0, st, a);
}
template <int D>
void run_short_bwd(const PackedShape& m, const AttnArgs& a, hipStream_t st) {
  // (few tiles: waves for the heads of a group)
  const int nh = short_blocks(m, a.T, m.kv) > kFewTiles ? 1 : m.heads / m.kv;
  if (nh > 2) run_short_bwd<D, 4>(m, a, st);
  else if (nh > 1) run_short_bwd<D, 2>(m, a, st);
  else run_short_bwd<D, 1>(m, a, st);
}

}  // namespace

hipError_t launch_short_attn_fwd(const PackedShape& m, int T, const void* qkv,
                                 const int32_t* starts, void* o, float* lse, hipStream_t st) {
  AttnArgs a = packed_args(m, T, qkv, starts);
  a.out = static_cast<bf16_t*>(o);
  a.lse = lse;
  return traced(FLOWMOE_K_ATTN_FWD, st, [&] {
    if (m.D == 128) run_short_fwd<128>(m, a, st);
    else run_short_fwd<64>(m, a, st);
  });
}

hipError_t launch_short_attn_bwd(const PackedShape& m, int T, const void* qkv,
                                 const int32_t* starts, const void* o, const float* lse,
                                 const void* d_o, void* d_qkv, float* delta, hipStream_t st) {
  AttnArgs a = packed_args(m, T, qkv, starts);
  a.o = static_cast<const bf16_t*>(o);
  a.d_o = static_cast<const bf16_t*>(d_o);
  a.d_qkv = static_cast<bf16_t*>(d_qkv);
  a.lse = const_cast<float*>(lse);
  a.delta = delta;
  return traced(FLOWMOE_K_ATTN_BWD_DKDV, st, [&] {
    if (m.D == 128) run_short_bwd<128>(m, a, st);
    else run_short_bwd<64>(m, a, st);
  });
}

}  // namespace flowmoe
