// The multi-head attention of AT_r (Sec. 2.1): per sequence and head,
// A = softmax(Q K^T / sqrt(d)) V with Q, K, V the head's columns of
// I [W^Q | W^K | W^V], then I' = A W^O. The projections run on the grouped
// GEMM as one dense expert; the attention runs in the kernels below, which
// stream K and V tiles through LDS and never store the N x N scores.
//
// Forward (one block: 128 queries of one sequence and head, 4 waves of 32):
// each wave computes S^T = K Q^T for a 64-key tile with
// v_mfma_f32_32x32x16_bf16, so that a lane's accumulator column is one query
// and the online-softmax statistics (running max and sum, base-2 exponents)
// live in the lane pair (l, l + 32) that holds that query's 64 scores. The
// bf16 probabilities P^T are then the second MFMA's column operand straight
// from the registers, and O^T += V^T P^T takes V^T from LDS by transposing
// reads (ds_read_b64_tr_b16). The log-sum-exp of each row is kept for the
// backward.
//
// Backward (no atomics; every sum in a fixed order):
//   dq kernel (blocks of 128 queries, loop over 32-key tiles): recomputes P
//     from S and the log-sum-exp, dP^T = V dO^T, dS = P (dP - delta) with
//     delta = rowsum(dO * O) (computed here and stored for the next kernel),
//     dQ^T += K^T dS^T;
//   dkdv kernel (blocks of 128 keys, loop over 32-query steps): S and dP with
//     the key as the accumulator column, dV^T += dO^T P, dK^T += Q^T dS.
//
// Packed sequences (flowmoe_packed_attention_*) run in the same loops: a block finds its sequence
// by a search of their starts (packed.hpp), keys and values are those of a query head's group, and
// dK and dV walk the group's heads one after the other. 16384 tokens in 12 sequences of 46 to
// 8021, 32 heads on 8 of 128, causal (676 GF of 4 D a pair): forward 660-670 us, 1.01 PFLOP/s, the
// matrix pipes and LDS busy for 52 % of the cycles at 1.6 GHz; backward 2300 us with delta's 49 and
// the join, 735 TFLOP/s of its 10 D, pipes 55 % and LDS 79 % busy at 1.8 GHz. Waves of 64 keys for
// dK and dV (48 reads of LDS for 64 products, not 80) were 13 % slower: the accumulators fill half of
// the registers, the compiler moves scores between its halves, and a SIMD has one wave.
#include <math.h>

#include <algorithm>

#include "attn_tiles.hpp"
#include "common.hpp"
#include "packed.hpp"

namespace flowmoe {
namespace {

// Units of the packed backward's long key tiles: a launch's steps are cut into about kUnits, of
// at least 16 steps, or of 8 where it has few. us of the whole backward with 500, 850, 1300 and
// 2000 units (uncut, of an earlier version, in brackets): one sequence of 2031, 16 heads on 2 of 128,
// causal 107, 103, 104, 104 (696); one of 4096, 16 on 16 277, 294, 298, 321 (342); of 16384, 8 on 1
// 1881, 1893, 1892, 1886 (6340); 16384 tokens in 12 of 46 to 8021, 32 on 8 2314, 2340, 2300, 2310
// (2725), in 18 of 76 to 5801 1545, 1556, 1605, 1599 (1809). Of at least 8, 16 and 32 steps: the
// first 112, 103, 124; 1000 tokens in 5, 8 on 2 of 64 23, 35, 39; one of 512, 16 on 4 24, 30, 44;
// of 1024, 32 on 8 of 128 74, 71, 74.
constexpr int kUnits = 850, kMinSteps = 8;

// block -> (query or key tile, head, sequence). Blocks are dispatched in
// order; u = blockIdx / (heads x sequences) ranks the tiles by their causal
// work, longest first (`rev`: tiles in descending order, the query tiles of
// the forward and of dQ; else ascending, the key tiles of dK/dV). With
// `a.pair` (every block resident at once, two to a CU: the second half of
// the grid lands on the CUs of the first half) the second half runs the
// shortest tiles first, so that a CU's two blocks have complementary work
// (ranks u and nt - 1 - u) instead of ranks u and u + nt / 2.
//
// `shared` (query tiles; shared_order): the tiles of a head one after the other on
// one XCD (blocks go to the 8 XCDs round-robin), so that its K and V are read
// through that L2 once. In the order above they are per blocks apart, and a launch
// whose K and V exceed the caches reads them from HBM for every tile.
__device__ __forceinline__ void decode(const AttnArgs& a, bool rev, bool shared, int& tile, int& hd,
                                       int& sq, int rows) {
  const int per = a.heads * a.nseq, nt = (a.N + rows - 1) / rows;
  if (shared && per % 8 == 0) {
    const int i = blockIdx.x >> 3, rest = i / nt * 8 + (blockIdx.x & 7);
    tile = rev ? nt - 1 - i % nt : i % nt;
    hd = rest % a.heads;
    sq = rest / a.heads;
    return;
  }
  const int u = (int)(blockIdx.x / per), rest = (int)(blockIdx.x % per);
  const int h = (nt + 1) / 2;
  const int r = a.pair && u >= h ? nt - 1 - (u - h) : u;  // rank in work order
  tile = rev ? nt - 1 - r : r;
  hd = rest % a.heads;
  sq = rest / a.heads;
}

// Steps of a key tile of 128 rows in the backward, 32 queries a step: the group's heads one
// after the other.
__device__ __forceinline__ int key_steps(int N, int tile, int heads, bool causal) {
  return heads * ((N - (causal ? 128 * tile : 0) + 31) / 32);
}
// The steps of a launch's unit, from the sum over its sequences, a lane each (a wave's 64 at
// a time).
__device__ __forceinline__ int unit_steps(const AttnArgs& a, bool causal, int lane) {
  long sum = 0;
  for (int i = lane; i < a.nseq; i += 64) {
    const long n = max(packed_start(a, i + 1) - packed_start(a, i), 0), q = (n + 31) / 32,
               nt = (n + 127) / 128;
    sum += nt * q - (causal ? 2 * nt * (nt - 1) : 0);  // of q - 4 t over the tiles t
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
  sum *= a.heads;  // (kv heads, of heads / kv query heads each)
  // (uniform, and known to be: the loops' bounds come from it)
  return __builtin_amdgcn_readfirstlane(
      sum <= 2 * kUnits ? kMinSteps : (int)max(2L * kMinSteps, min((sum + kUnits - 1) / kUnits, 1L << 30)));
}
// Units of a tile of `steps` steps (at most `most`), and the steps of each
__device__ __forceinline__ int tile_units(int steps, int unit, int most, int& len) {
  const int n = min(most, (steps + unit - 1) / unit);
  len = n > 1 ? (steps + n - 1) / n : steps;
  return n > 1 ? (steps + len - 1) / len : 1;  // (none of them empty)
}

// The sums of unit u of the 32-row tile t32 of a sequence, of a key head's K (kv = 0) or V:
// 32 x D values as the lanes hold them, 16 bytes a lane side by side
__device__ __forceinline__ float* unit_part(const AttnArgs& a, const Span& s, int u, int t32,
                                            int g, int kv, int D) {
  const long tile = s.tok0 / 32 + s.seq + t32;
  return a.part + ((((long)u * a.rows32 + tile) * a.kv + g) * 2 + kv) * 32 * D;
}
template <int DB>
__device__ __forceinline__ void store_part(float* p, const floatx16 (&x)[DB], int lane, float scale) {
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int J = 0; J < 4; ++J)
      *reinterpret_cast<float4*>(p + ((db * 4 + J) * 64 + lane) * 4) =
          make_float4(x[db][4 * J] * scale, x[db][4 * J + 1] * scale, x[db][4 * J + 2] * scale,
                      x[db][4 * J + 3] * scale);
}

// Query tiles: the block's span, with or without packing; false: no rows
template <bool PACKED>
__device__ __forceinline__ bool query_span(const AttnArgs& a, int D, bool causal, int rows,
                                           int lane, unsigned block, unsigned blocks, Span& s) {
  if constexpr (PACKED) {
    int unit;
    const bool any = packed_span(a, a.heads, causal, rows, 1, lane, block, blocks, s, unit);
    s.ld = (long)(a.heads + 2 * a.kv) * D;
    const int g = s.hd / (a.heads / a.kv);
    s.k = (long)(a.heads + g - s.hd) * D;
    s.v = s.k + (long)a.kv * D;
    return any;
  } else {
    int sq;
    decode(a, causal, a.shared != 0, s.tile, s.hd, sq, rows);
    s.N = a.N;
    s.tok0 = (long)sq * a.N;
    s.ld = 3L * a.M;
    s.k = a.M;
    s.v = 2L * a.M;
    s.seq = 0;
    s.none = false;
    return true;
  }
}

// Forward: blocks of 4 waves of 32 queries (8 in some launches of heads of 64), two to
// four to a CU.
//
// The matrix pipes should bound it, but a tile's softmax takes about as many issue
// cycles as its 32 products take matrix cycles, and products that wait for their
// own LDS read or a softmax after them leave both idle (pipes busy 0.39 of the
// cycles). So a step runs one tile ahead: the products S(t + 1) = K Q are issued
// between the exponentials of S(t), the products with V(t) between the maxima of
// S(t + 1), and every LDS read two groups of products before its use. K and V
// tiles come by LDS-DMA into two slots each: step t reads K(t + 1) and V(t), and
// refills K(t)'s and V(t - 1)'s slots. Measured, before -> now: 4 x 4096 tokens, 32
// heads of 128, causal 635 -> 590 us; one sequence of 4096, 16 heads 112 -> 93; 4 x
// 2048, 32 heads, bidirectional 326 -> 297. Blocks of 8 waves (half the staging)
// are 0-4% slower, and 12% on short causal sequences; four slots instead of two,
// raised priority around the V products, and timing copies without the barrier
// or the wait for the loads change 0-2%, without the exponentials 7%, without the
// DMA 17% (less switching): two independent blocks a CU hide what there is.
//
// Heads of 64 have half the products for the same softmax, and room for four waves
// on a SIMD (128 registers) if a step does not run ahead: then the other waves
// hide a wave's softmax, and K(t), V(t) are used in turn. The one-tile-ahead loop
// with two waves a SIMD had made them up to 13 % slower than the loop before it,
// where a launch is several rounds. us of the loop before, ahead, in turn: 32
// sequences of 512, 16 heads, bidirectional 56, 62, 51 (8 waves); 4 x 4096, 24 heads,
// causal 252, 266, 229; 8 x 512 20, 19, 18; 1 x 4096, 8 heads 64, 54, 55.
template <int D, bool CAUSAL, int NW, bool PACKED, int SPLIT>
__global__ __launch_bounds__(64 * NW * SPLIT, D == 128 ? 2 : 4) void attn_fwd_kernel(AttnArgs a) {
  constexpr bool AHEAD = D == 128;
  constexpr int KS = D / 16, DB = D / 32, QB = 32 * NW;
  using Dma = TileDma<D, 64, NW>;
  constexpr int TB = Dma::TB;
  __shared__ __attribute__((aligned(1024))) char all[SPLIT * 4 * TB];  // a group: K slots 0, 1, then V slots 0, 1
  // the wave index through readfirstlane: the compiler then knows it is
  // wave-uniform, and the branches on a wave's query or key range are
  // scalar branches instead of exec-mask ones (backward 7-10% faster)
  const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6),
            h2 = lane >> 5, lq = lane & 31;
  // (group grp of NW waves has the key tiles grp, grp + SPLIT, ...)
  const int grp = SPLIT > 1 ? wv / NW : 0, w = SPLIT > 1 ? wv % NW : wv, ko = 64 * grp;
  constexpr int KT = 64 * SPLIT;
  char* const lds = all + grp * 4 * TB;
  Span sp;
  if (!query_span<PACKED>(a, D, CAUSAL, QB, lane, blockIdx.x, gridDim.x, sp)) return;
  const long tok0 = sp.tok0, ld = sp.ld;
  const int hd = sp.hd, N = sp.N, q0 = sp.tile * QB, qw = q0 + 32 * w + lq;
  if constexpr (PACKED) {
    if (sp.none) {
      const int n = min(QB, N - q0);
      zero_rows(a.out + (long)hd * D, a.M, tok0 + q0, n, D, tid, 64 * NW * SPLIT);
      for (int i = tid; i < n; i += 64 * NW * SPLIT) a.lse[(long)hd * a.T + tok0 + q0 + i] = 0.0f;
      return;
    }
  }
  const bf16_t* Qg = a.qkv + tok0 * ld + (long)hd * D;
  const bf16_t* Kg = Qg + sp.k + ko * ld;
  const bf16_t* Vg = Qg + sp.v + ko * ld;

  const int kend = CAUSAL ? min(N, q0 + QB) : N;
  const int nkt = (kend + 63) / 64, nk = (nkt + SPLIT - 1) / SPLIT;
  // (causal: a wave whose queries all precede a tile has nothing in it; packed: nor one
  // without queries)
  const int nkc = CAUSAL ? min(nkt, (q0 + 32 * w + 31) / 64 + 1) : nkt;
  const int nkw = PACKED && q0 + 32 * w >= N ? 0 : (nkc + SPLIT - 1 - grp) / SPLIT;
  const Dma dma(lds_base(all) + grp * 4 * TB, w, lane, ld);
  const long kstep = KT * ld;
  dma.load(Kg, kend - ko, 0);
  dma.load(Vg, kend - ko, 2 * TB);
  if constexpr (AHEAD) dma.load(Kg + kstep, kend - ko - KT, TB);  // (past the last tile: no traffic)

  bf16x8 qf[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks)
    qf[ks] = qw < N ? *reinterpret_cast<const bf16x8*>(Qg + qw * ld + 16 * ks + 8 * h2) : zero8();
  floatx16 o[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) o[db] = zero16();
  float m = -INFINITY, l = 0.0f;

  int rbase = row_base<D>(lq, h2), tb0 = tr_base<D>(lane, 0), tb1 = tr_base<D>(lane, 1);
  auto mask = [&](floatx16 (&s)[2], int kb0) {
    if (kb0 + 64 > N || (CAUSAL && kb0 + 63 > q0 + 32 * w)) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int key = kb0 + 32 * kb + 8 * (r >> 2) + 4 * h2 + (r & 3);
          if (key >= N || (CAUSAL && key > qw)) s[kb][r] = -INFINITY;
        }
    }
  };
  auto row_max = [&](const floatx16 (&s)[2]) {
    float mx = s[0][0];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[kb][r]);
    return mx;
  };
  // The reference m of the exponents moves only when a score exceeds it
  // by more than 2^8 (then the sum and the accumulators are rescaled):
  // probabilities up to 256 stay exact in float and in bf16's exponent
  // range, and the final lse = m + log2(l) is the same. Every query sees
  // key 0 in the first tile, so m is finite from then on.
  auto move_ref = [&](float mx) {
    mx = pair_max(mx) * a.c2;
    const bool up = mx > m + 8.0f;
    if (__any(up)) {
      const float mn = up ? mx : m;
      const float al = exp2_fast(m - mn);
      l *= al;
#pragma unroll
      for (int db = 0; db < DB; ++db) o[db] *= al;
      m = mn;
    }
  };

  // The LDS reads of a step in groups of two fragments, each read two groups ahead
  // of its products (a product that waits for its own read waits a whole LDS
  // latency): groups 0 .. KS - 1, both key blocks of K(t + 1) at k step i; then 2 DB
  // groups of V(t), 16 keys by 64 columns each
  constexpr int VG = 2 * DB, NG = KS + VG;
  bf16x8 fr[3][2];
  auto read_group = [&](const char* tk, const char* tv, int i) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      if (i < KS) fr[i % 3][u] = frag_row_x<D>(tk, rbase, 32 * u, i);
      else if (i < NG)
        fr[i % 3][u] = frag_tr_x<D>(tv, tb0, tb1, 16 * ((i - KS) / (DB / 2)),
                                    32 * (2 * ((i - KS) % (DB / 2)) + u));
    }
  };
  auto mul_k = [&](floatx16 (&s)[2], int i) {
#pragma unroll
    for (int u = 0; u < 2; ++u) s[u] = mfma(fr[i % 3][u], qf[i], i == 0 ? zero16() : s[u]);
  };

  // heads of 64: K(t) and V(t) in slots t % 2; the scores, the softmax and the value
  // products one after the other
  auto step_in_turn = [&](const int t, auto stc) {
    constexpr int st = decltype(stc)::value;
    opaque(rbase, tb0, tb1);
    wait_vm<0>();  // K(t) and V(t): loaded a step ago
    lds_barrier();  // and every wave's reads of the slots refilled now are done
    const char* tk = lds + st * TB;
    const char* tv = lds + (2 + st) * TB;
    const bool live = t < nkw;
    if (live) {
      read_group(tk, tv, 0);
      read_group(tk, tv, 1);
    }
    Kg += kstep;  // K(t + 1), V(t + 1)
    Vg += kstep;
    dma.load(Kg, kend - ko - KT * (t + 1), (st ^ 1) * TB);
    dma.load(Vg, kend - ko - KT * (t + 1), (2 + (st ^ 1)) * TB);
    if (!live) return;
    floatx16 sc[2];
#pragma unroll
    for (int i = 0; i < KS; ++i) {
      read_group(tk, tv, i + 2);
      __builtin_amdgcn_sched_barrier(0);
      mul_k(sc, i);
      __builtin_amdgcn_sched_barrier(0);
    }
    mask(sc, ko + KT * t);
    move_ref(row_max(sc));
    unsigned pw[16];
    float rsum = 0.0f;
#pragma unroll
    for (int q = 0; q < 32; q += 2) {
      const float p0 = exp2_fast(fmaf(sc[q >> 4][q & 15], a.c2, -m));
      const float p1 = exp2_fast(fmaf(sc[q >> 4][(q & 15) + 1], a.c2, -m));
      rsum += p0;
      rsum += p1;
      pw[q >> 1] = pack_bf16x2(p0, p1);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int j = 0; j < VG; ++j) {
      read_group(tk, tv, KS + j + 2);
      __builtin_amdgcn_sched_barrier(0);
      const int g = j / (DB / 2);
      const bf16x8 pb = __builtin_bit_cast(bf16x8, u32x4{pw[4 * g], pw[4 * g + 1], pw[4 * g + 2], pw[4 * g + 3]});
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int db = 2 * (j % (DB / 2)) + u;
        o[db] = mfma(fr[(KS + j) % 3][u], pb, o[db]);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    l += pair_sum(rsum);
  };

  floatx16 s[2][2];  // [tile parity][32-key block]
  if constexpr (AHEAD) {
    wait_vm<0>();
    lds_barrier();
    read_group(lds, lds, 0);
    read_group(lds, lds, 1);
#pragma unroll
    for (int i = 0; i < KS; ++i) {
      if (i + 2 < KS) read_group(lds, lds, i + 2);
      __builtin_amdgcn_sched_barrier(0);
      mul_k(s[0], i);
    }
    mask(s[0], ko);
    move_ref(row_max(s[0]));
  }

  auto step_ahead = [&](const int t, auto stc) {
    constexpr int st = decltype(stc)::value;
    opaque(rbase, tb0, tb1);
    wait_vm<0>();  // K(t + 1) and V(t): loaded a step ago
    lds_barrier();  // and every wave's reads of the slots refilled now are done
    const char* tk = lds + (st ^ 1) * TB;
    const char* tv = lds + (2 + st) * TB;
    floatx16(&sc)[2] = s[st];
    floatx16(&sn)[2] = s[st ^ 1];
    const bool live = t < nkw, next = t + 1 < nkw;
    if (next) {
      read_group(tk, tv, 0);
      read_group(tk, tv, 1);
    }
    Kg += kstep;  // K(t + 1), V(t + 1)
    Vg += kstep;
    dma.load(Kg + kstep, kend - ko - KT * (t + 2), st * TB);
    dma.load(Vg, kend - ko - KT * (t + 1), (2 + (st ^ 1)) * TB);
    if (!live) return;
    unsigned pw[16];  // the 32 probabilities of this lane, bf16 pairs
    // (the sum in key order, then the lane pair's two halves, tile by tile: results do
    // not depend on how the step is scheduled)
    float rsum = 0.0f;
    auto exps = [&](int q0s, int q1s) {  // scores q0s .. q1s - 1: exponentials, sum, bf16
#pragma unroll
      for (int q = q0s; q < q1s; q += 2) {
        const float p0 = exp2_fast(fmaf(sc[q >> 4][q & 15], a.c2, -m));
        const float p1 = exp2_fast(fmaf(sc[q >> 4][(q & 15) + 1], a.c2, -m));
        rsum += p0;
        rsum += p1;
        pw[q >> 1] = pack_bf16x2(p0, p1);
        // (computed here, not where they are used)
        asm volatile("" : "+v"(pw[q >> 1]), "+v"(rsum));
      }
    };
    __builtin_amdgcn_sched_barrier(0);
    if (next) {
      constexpr int CH = 32 / KS;  // scores exponentiated beside a group's two products
#pragma unroll
      for (int i = 0; i < KS; ++i) {
        read_group(tk, tv, i + 2);
        __builtin_amdgcn_sched_barrier(0);
        exps(i * CH, (i + 1) * CH);
        mul_k(sn, i);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
          __builtin_amdgcn_sched_group_barrier(0x402, 7 * CH / 4, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      mask(sn, ko + KT * (t + 1));
    } else {
      read_group(tk, tv, KS);
      read_group(tk, tv, KS + 1);
      exps(0, 32);
    }
    __builtin_amdgcn_sched_barrier(0);
    float mx = sn[0][0];
#pragma unroll
    for (int j = 0; j < VG; ++j) {
      read_group(tk, tv, KS + j + 2);
      __builtin_amdgcn_sched_barrier(0);
      const int g = j / (DB / 2);
      const bf16x8 pb = __builtin_bit_cast(bf16x8, u32x4{pw[4 * g], pw[4 * g + 1], pw[4 * g + 2], pw[4 * g + 3]});
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int db = 2 * (j % (DB / 2)) + u;
        o[db] = mfma(fr[(KS + j) % 3][u], pb, o[db]);
      }
      constexpr int CH = 32 / VG;
#pragma unroll
      for (int q = j * CH; q < (j + 1) * CH; ++q) mx = fmaxf(mx, sn[q >> 4][q & 15]);
      asm volatile("" : "+v"(mx));
      __builtin_amdgcn_sched_barrier(0);
    }
    l += pair_sum(rsum);
    if (next) move_ref(mx);
  };
  auto step = [&](const int t, auto stc) {
    if constexpr (AHEAD) step_ahead(t, stc);
    else step_in_turn(t, stc);
  };
  for (int t = 0; t < nk; t += 2) {
    step(t, Stage<0>{});
    if (t + 1 < nk) step(t + 1, Stage<1>{});
  }
  if constexpr (SPLIT > 1) {
    // the groups' sums, in order. (Of a live tile every query sees the first key, so that a
    // group's m is finite or, with no tile, its sums are zeros; the first group has key 0.)
    float* part = reinterpret_cast<float*>(all);
    constexpr int NF = 16 * DB + 2;
    static_assert((SPLIT - 1) * NW * NF * 256 <= SPLIT * 4 * TB, "the sums fit the tiles' LDS");
    wait_vm<0>();  // (loads past the last tile write zeros)
    lds_barrier();
    if (grp > 0) {
      float* p = part + ((grp - 1) * NW + w) * NF * 64 + lane;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) p[(16 * db + r) * 64] = o[db][r];
      p[16 * DB * 64] = m;
      p[(16 * DB + 1) * 64] = l;
    }
    lds_barrier();
    if (grp > 0) return;
#pragma unroll 1
    for (int e = 0; e < SPLIT - 1; ++e) {
      const float* p = part + (e * NW + w) * NF * 64 + lane;
      const float m1 = p[16 * DB * 64], mn = fmaxf(m, m1);
      const float a0 = exp2_fast(m - mn), a1 = exp2_fast(m1 - mn);
      l = l * a0 + p[(16 * DB + 1) * 64] * a1;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[db][r] = o[db][r] * a0 + p[(16 * db + r) * 64] * a1;
      m = mn;
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

// dQ and delta: blocks of 4 waves of 32 queries, two to a CU, over 32-key tiles.
//
// As the forward it runs one tile ahead: S(t + 1) = K Q and dP(t + 1) = V dO are
// issued between the elementwise work of tile t, dQ += K^T dS(t) follows, and each
// LDS read is one (D = 64: two) groups of products ahead of its use. K(t) is read in
// two steps (rows, then transposed), so K has three slots and V two; the block's dO
// rows are read from LDS (registers hold Q). Before -> now: 4 x 4096 tokens, 32 heads
// of 128, causal 970 -> 850 us; one sequence of 4096, 16 heads 171 -> 135; 4 x 1500, 20
// heads of 64, bidirectional 112 -> 102.
//
// DELTA: computed here; else read (attn_delta_kernel's).
template <int D>
constexpr int kDqLds = 5 * 64 * D + 256 * D;
template <int D, bool CAUSAL, bool PACKED, bool DELTA>
__device__ __forceinline__ void dq_rows(const AttnArgs& a, char* lds, unsigned block, unsigned blocks) {
  constexpr int KS = D / 16, DB = D / 32, NW = 4, QB = 32 * NW;
  using Dma = TileDma<D, 32, NW>;
  constexpr int TB = Dma::TB, VB = 3 * TB, GB = 5 * TB;  // K slots, V slots, the dO rows
  static_assert(GB + QB * D * 2 == kDqLds<D>, "the block's LDS");
  // the wave index through readfirstlane: the compiler then knows it is
  // wave-uniform, and the branches on a wave's query or key range are
  // scalar branches instead of exec-mask ones (backward 7-10% faster)
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6),
            h2 = lane >> 5, lq = lane & 31;
  Span sp;
  if (!query_span<PACKED>(a, D, CAUSAL, QB, lane, block, blocks, sp)) return;
  const long tok0 = sp.tok0, ld = sp.ld;
  const int hd = sp.hd, N = sp.N, q0 = sp.tile * QB, qw = q0 + 32 * w + lq;
  if constexpr (PACKED) {
    if (sp.none) {
      const int n = min(QB, N - q0);
      zero_rows(a.d_qkv + (long)hd * D, ld, tok0 + q0, n, D, tid, 64 * NW);
      for (int i = tid; i < n; i += 64 * NW) a.delta[(long)hd * a.T + tok0 + q0 + i] = 0.0f;
      return;
    }
  }
  const bf16_t* Qg = a.qkv + tok0 * ld + (long)hd * D;
  const bf16_t* Kg = Qg + sp.k;
  const bf16_t* Vg = Qg + sp.v;
  const bf16_t* Gg = a.d_o + tok0 * a.M + (long)hd * D;
  const bf16_t* Og = a.o + tok0 * a.M + (long)hd * D;
  const bool live = qw < N;

  const int kend = CAUSAL ? min(N, q0 + QB) : N;
  const int nk = (kend + 31) / 32;
  // (causal: a wave whose queries all precede a tile has nothing in it; packed: nor one
  // without queries)
  const int nkc = CAUSAL ? min(nk, (q0 + 32 * w + 31) / 32 + 1) : nk;
  const int nkw = PACKED && q0 + 32 * w >= N ? 0 : nkc;
  const long kstep = 32 * ld;
  const Dma dma(lds_base(lds), w, lane, ld);
  {
    const Dma dmag(lds_base(lds), w, lane, a.M);
#pragma unroll
    for (int i = 0; i < NW; ++i)
      dmag.load(Gg + (long)(q0 + 32 * i) * a.M, N - q0 - 32 * i, GB + i * TB);
  }
  dma.load(Kg, kend, 0);
  dma.load(Vg, kend, VB);
  dma.load(Kg + kstep, kend - 32, TB);  // (past the last tile: no traffic)
  dma.load(Vg + kstep, kend - 32, VB + TB);
  bf16x8 qf[KS];
  float dl = 0.0f;
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    qf[ks] = live ? *reinterpret_cast<const bf16x8*>(Qg + qw * ld + 16 * ks + 8 * h2) : zero8();
    if constexpr (DELTA) {
      const bf16x8 gv = live ? *reinterpret_cast<const bf16x8*>(Gg + (long)qw * a.M + 16 * ks + 8 * h2) : zero8();
      const bf16x8 ov = live ? *reinterpret_cast<const bf16x8*>(Og + (long)qw * a.M + 16 * ks + 8 * h2) : zero8();
#pragma unroll
      for (int t = 0; t < 8; ++t) dl += (float)gv[t] * (float)ov[t];
    }
  }
  const long srow = (long)hd * a.T + tok0 + qw;
  if constexpr (DELTA) dl += __shfl_xor(dl, 32);
  else dl = live ? a.delta[srow] : 0.0f;
  if (DELTA && live && h2 == 0) a.delta[srow] = dl;
  const float l2 = live ? a.lse[srow] * kLog2e : 0.0f;
  floatx16 dq[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) dq[db] = zero16();

  int rbase = row_base<D>(lq, h2), tb0 = tr_base<D>(lane, 0), tb1 = tr_base<D>(lane, 1);
  // read groups: 0 .. KS - 1, the K, V and dO rows at k step i of tile t + 1; then DB
  // groups of tile t's K transposed, 16 keys by 64 columns each
  constexpr int NG = KS + DB;
  constexpr int RS = D == 128 ? 2 : 3;  // groups in registers (128: three spill)
  bf16x8 fr[RS][3];
  auto read_group = [&](const char* tk, const char* tv, const char* tkt, int i) {
    if (i < KS) {
      fr[i % RS][0] = frag_row_x<D>(tk, rbase, 0, i);
      fr[i % RS][1] = frag_row_x<D>(tv, rbase, 0, i);
      fr[i % RS][2] = frag_row_x<D>(lds + GB, rbase, 32 * w, i);
    } else if (i < NG) {
#pragma unroll
      for (int u = 0; u < 2; ++u)
        fr[i % RS][u] = frag_tr_x<D>(tkt, tb0, tb1, 16 * ((i - KS) / (DB / 2)),
                                    32 * (2 * ((i - KS) % (DB / 2)) + u));
    }
  };
  floatx16 s[2], dp[2];  // [tile parity]
  auto mul = [&](floatx16& x, floatx16& y, int i) {
    x = mfma(fr[i % RS][0], qf[i], i == 0 ? zero16() : x);
    y = mfma(fr[i % RS][1], fr[i % RS][2], i == 0 ? zero16() : y);
  };
  auto mask = [&](floatx16& x, int kb0) {
    if (kb0 + 32 > N || (CAUSAL && kb0 + 31 > q0 + 32 * w)) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int key = kb0 + 8 * (r >> 2) + 4 * h2 + (r & 3);
        if (key >= N || (CAUSAL && key > qw)) x[r] = -INFINITY;
      }
    }
  };

  wait_vm<0>();
  lds_barrier();
  read_group(lds, lds + VB, lds, 0);
  if constexpr (RS > 2) read_group(lds, lds + VB, lds, 1);
#pragma unroll
  for (int i = 0; i < KS; ++i) {
    if (i + RS - 1 < KS) read_group(lds, lds + VB, lds, i + RS - 1);
    __builtin_amdgcn_sched_barrier(0);
    mul(s[0], dp[0], i);
  }
  mask(s[0], 0);

  int k0s = 0;  // tile t's K slot
  auto step = [&](const int t, auto stc) {
    constexpr int st = decltype(stc)::value;
    opaque(rbase, tb0, tb1);
    wait_vm<0>();   // K(t + 1) and V(t + 1)
    lds_barrier();  // and every wave's reads of the slots refilled now are done
    const int k1s = k0s == 2 ? 0 : k0s + 1, k2s = k1s == 2 ? 0 : k1s + 1;
    const char* tk = lds + k1s * TB;
    const char* tv = lds + VB + (st ^ 1) * TB;
    const char* tkt = lds + k0s * TB;
    const bool next = t + 1 < nkw;
    if (next) {
      read_group(tk, tv, tkt, 0);
      if constexpr (RS > 2) read_group(tk, tv, tkt, 1);
    }
    Kg += kstep;  // K(t + 1), V(t + 1)
    Vg += kstep;
    dma.load(Kg + kstep, kend - 32 * (t + 2), k2s * TB);
    dma.load(Vg + kstep, kend - 32 * (t + 2), VB + st * TB);
    k0s = k1s;
    if (t >= nkw) return;
    unsigned pw[8];  // dS^T of this lane, bf16 pairs
    auto elem = [&](int r0, int r1) {
#pragma unroll
      for (int r = r0; r < r1; r += 2) {
        const float d0 = exp2_fast(fmaf(s[st][r], a.c2, -l2)) * (dp[st][r] - dl);
        const float d1 = exp2_fast(fmaf(s[st][r + 1], a.c2, -l2)) * (dp[st][r + 1] - dl);
        pw[r >> 1] = pack_bf16x2(d0, d1);
        asm volatile("" : "+v"(pw[r >> 1]));  // (computed here, not where it is used)
      }
    };
    __builtin_amdgcn_sched_barrier(0);
    if (next) {
      constexpr int CH = 16 / KS;  // scores beside a group's two products
#pragma unroll
      for (int i = 0; i < KS; ++i) {
        read_group(tk, tv, tkt, i + RS - 1);
        __builtin_amdgcn_sched_barrier(0);
        elem(i * CH, (i + 1) * CH);
        mul(s[st ^ 1], dp[st ^ 1], i);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
          __builtin_amdgcn_sched_group_barrier(0x402, 9 * CH / 4, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      mask(s[st ^ 1], 32 * (t + 1));
    } else {
      read_group(tk, tv, tkt, KS);
      if constexpr (RS > 2) read_group(tk, tv, tkt, KS + 1);
      elem(0, 16);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int j = 0; j < DB; ++j) {
      read_group(tk, tv, tkt, KS + j + RS - 1);
      __builtin_amdgcn_sched_barrier(0);
      const int g = j / (DB / 2);
      const bf16x8 pb = __builtin_bit_cast(bf16x8, u32x4{pw[4 * g], pw[4 * g + 1], pw[4 * g + 2], pw[4 * g + 3]});
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int db = 2 * (j % (DB / 2)) + u;
        dq[db] = mfma(fr[(KS + j) % RS][u], pb, dq[db]);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  for (int t = 0; t < nk; t += 2) {
    step(t, Stage<0>{});
    if (t + 1 < nk) step(t + 1, Stage<1>{});
  }
  if (live) {
    bf16_t* dst = a.d_qkv + (tok0 + qw) * ld + (long)hd * D;
#pragma unroll
    for (int db = 0; db < DB; ++db) store_cols(dst + 32 * db, dq[db], h2, a.rs);
  }
}

template <int D, bool CAUSAL>
__global__ __launch_bounds__(256, 2) void attn_dq_kernel(AttnArgs a) {
  __shared__ __attribute__((aligned(1024))) char lds[kDqLds<D>];
  dq_rows<D, CAUSAL, false, true>(a, lds, blockIdx.x, gridDim.x);
}

// dK and dV: blocks of 4 waves of 32 keys, two to a CU, over 32-query tiles. The
// accumulators leave no registers for a tile ahead; within a tile every LDS read
// (Q, dO and the block's V rows, then dO and Q transposed) is one (D = 64: two)
// groups of products ahead of its use, S and dP alternate, and the other block of
// the CU fills the elementwise part (half of it beside the first products of
// dV and dK was 2-4% slower at D = 128). Before -> now, as above: 1258 -> 1120, 256 ->
// 182 and 163 -> 127 us.
template <int D>
constexpr int kDkdvLds = 4 * 64 * D + 256 * D + 512;
template <int D, bool CAUSAL, bool PACKED>
__device__ __forceinline__ void dkdv_rows(const AttnArgs& a, char* lds, unsigned block, unsigned blocks) {
  constexpr int KS = D / 16, DB = D / 32, NW = 4, KB = 32 * NW;
  using Dma = TileDma<D, 32, NW>;
  constexpr int TQ = Dma::TB;           // one 32-row tile
  constexpr int VT = 4 * TQ;            // two slots of Q and dO, then the block's V rows,
  constexpr int ST = VT + KB * D * 2;   // then two slots of 32 lse2 and 32 delta
  static_assert(ST + 2 * 256 == kDkdvLds<D>, "the block's LDS");
  // the wave index through readfirstlane: the compiler then knows it is
  // wave-uniform, and the branches on a wave's query or key range are
  // scalar branches instead of exec-mask ones (backward 7-10% faster)
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6),
            h2 = lane >> 5, lq = lane & 31;
  Span sp;
  int nh = 1;  // query heads from hd on
  int unit = 0, units = 1, it0 = 0, it1 = 0;  // the block's steps
  if constexpr (PACKED) {
    const bool any = packed_span(a, a.kv, false, KB, a.units, lane, block, blocks, sp, unit);
    if (!any) return;
    const int g = sp.hd;
    nh = a.heads / a.kv;
    sp.hd = g * nh;
    sp.ld = (long)(a.heads + 2 * a.kv) * D;
    sp.k = (long)(a.heads + g - sp.hd) * D;
    sp.v = sp.k + (long)a.kv * D;
  } else {
    int sq;
    decode(a, false, false, sp.tile, sp.hd, sq, KB);
    sp.N = a.N;
    sp.tok0 = (long)sq * a.N;
    sp.ld = 3L * a.M;
    sp.k = a.M;
    sp.v = 2L * a.M;
    sp.seq = 0;
    sp.none = false;
  }
  const long tok0 = sp.tok0, ld = sp.ld;
  const int hd = sp.hd, N = sp.N, k0 = sp.tile * KB, kw = k0 + 32 * w + lq;
  if constexpr (PACKED) {
    if (sp.none) {
      if (unit > 0) return;
      const int n = min(KB, N - k0);
      zero_rows(a.d_qkv + hd * D + sp.k, ld, tok0 + k0, n, D, tid, 64 * NW);
      zero_rows(a.d_qkv + hd * D + sp.v, ld, tok0 + k0, n, D, tid, 64 * NW);
      return;
    }
    const int steps = key_steps(N, sp.tile, nh, CAUSAL);
    it1 = steps;
    if (a.units > 1 && steps > kMinSteps) {
      int len;
      units = tile_units(steps, unit_steps(a, CAUSAL, lane), a.units, len);
      it0 = unit * len;
      it1 = min(steps, it0 + len);
    }
    if (unit >= units) return;
  }
  const bf16_t* Qg = a.qkv + tok0 * ld + (long)hd * D;
  const bf16_t* Gg = a.d_o + tok0 * a.M + (long)hd * D;
  const long srow0 = (long)hd * a.T + tok0;
  const bool live = kw < N;
  // query steps of 32: causal keys k0.. are seen by queries >= k0 only
  const int qs0 = CAUSAL ? k0 : 0;
  const int nqs = (N - qs0 + 31) / 32;
  // packed: the group's query heads one after the other, nqs steps each, of which the block
  // has it0 .. it1 - 1, from step qi of head g0 on
  const int steps = PACKED ? it1 - it0 : nqs;
  const int g0 = PACKED ? it0 / nqs : 0;
  int qi = PACKED ? it0 - g0 * nqs : 0;

  const Dma dma(lds_base(lds), w, lane, ld), dmag(lds_base(lds), w, lane, a.M);
#pragma unroll
  for (int i = 0; i < NW; ++i)
    dma.load(Qg + sp.v + (long)(k0 + 32 * i) * ld, N - k0 - 32 * i, VT + i * TQ);
  bf16x8 kf[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks)
    kf[ks] = live ? *reinterpret_cast<const bf16x8*>(Qg + sp.k + kw * ld + 16 * ks + 8 * h2) : zero8();
  float rstat = 0.0f;  // (the block's first 64 threads)
  const float* sp_stat = (tid < 32 ? a.lse : a.delta) + srow0 + (PACKED ? (long)g0 * a.T : 0) + (tid & 31);
  auto load_stat = [&](int qb) {
    if (tid < 64) rstat = qb + (tid & 31) < N ? sp_stat[qb] * (tid < 32 ? kLog2e : 1.0f) : 0.0f;
  };
  auto store_stat = [&](int slot) {
    if (tid < 64) reinterpret_cast<float*>(lds + ST + 256 * slot)[tid] = rstat;
  };
  const int qf0 = PACKED ? qs0 + 32 * qi : qs0;
  const bf16_t* Qt = Qg + qf0 * ld + (PACKED ? g0 * D : 0);
  const bf16_t* Gt = Gg + (long)qf0 * a.M + (PACKED ? g0 * D : 0);
  dma.load(Qt, N - qf0, 0);
  dmag.load(Gt, N - qf0, TQ);
  load_stat(qf0);
  store_stat(0);
  floatx16 dv[DB], dk[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) {
    dv[db] = zero16();
    dk[db] = zero16();
  }
  int rbase = row_base<D>(lq, h2), tb0 = tr_base<D>(lane, 0), tb1 = tr_base<D>(lane, 1);
  // read groups: 0 .. KS - 1, the Q, dO and V rows at k step i; then 2 DB groups of dO
  // and Q transposed, 16 queries by 32 columns each
  constexpr int NG = KS + 2 * DB;
  constexpr int RS = D == 128 ? 2 : 3;  // groups in registers (128: three spill)
  bf16x8 fr[RS][3];
  auto read_group = [&](const char* tq, int i) {
    const char* tg = tq + TQ;
    if (i < KS) {
      fr[i % RS][0] = frag_row_x<D>(tq, rbase, 0, i);
      fr[i % RS][1] = frag_row_x<D>(tg, rbase, 0, i);
      fr[i % RS][2] = frag_row_x<D>(lds + VT, rbase, 32 * w, i);
    } else if (i < NG) {
      fr[i % RS][0] = frag_tr_x<D>(tg, tb0, tb1, 16 * ((i - KS) / DB), 32 * ((i - KS) % DB));
      fr[i % RS][1] = frag_tr_x<D>(tq, tb0, tb1, 16 * ((i - KS) / DB), 32 * ((i - KS) % DB));
    }
  };
  auto step = [&](const int it, auto stc) {
    constexpr int st = decltype(stc)::value;
    opaque(rbase, tb0, tb1);
    const int qb = qs0 + 32 * (PACKED ? qi : it);
    wait_vm<0>();   // this tile's loads
    lds_barrier();  // and every wave's reads of the other slot are done
    const char* tq = lds + st * 2 * TQ;
    const float* l2 = reinterpret_cast<const float*>(lds + ST + 256 * st);
    // (packed: nor for a wave without keys)
    const bool mine = (!CAUSAL || qb + 31 >= k0 + 32 * w) && !(PACKED && k0 + 32 * w >= N);
    if (mine) {
      read_group(tq, 0);
      if constexpr (RS > 2) read_group(tq, 1);
    }
    int qn = qb + 32;
    Qt += 32 * ld;
    Gt += 32L * a.M;
    if constexpr (PACKED) {
      if (++qi == nqs) {  // the next head's first step
        qi = 0;
        qn = qs0;
        Qt += D - 32 * nqs * ld;
        Gt += D - 32L * nqs * a.M;
        sp_stat += a.T;
      }
    }
    // (after the last step: its head's rows end, or there is no further head)
    const int left = !PACKED || it + 1 < steps ? N - qn : 0;
    dma.load(Qt, left, (st ^ 1) * 2 * TQ);
    dmag.load(Gt, left, (st ^ 1) * 2 * TQ + TQ);
    if (it + 1 < steps) load_stat(qn);
    if (mine) {
      floatx16 s, dp;
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < KS; ++i) {
        read_group(tq, i + RS - 1);
        __builtin_amdgcn_sched_barrier(0);
        s = mfma(fr[i % RS][0], kf[i], i == 0 ? zero16() : s);
        dp = mfma(fr[i % RS][1], fr[i % RS][2], i == 0 ? zero16() : dp);
        __builtin_amdgcn_sched_barrier(0);
      }
      if (qb + 32 > N || (CAUSAL && k0 + 32 * w + 31 > qb)) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int q = qb + 8 * (r >> 2) + 4 * h2 + (r & 3);
          if (q >= N || (CAUSAL && kw > q)) s[r] = -INFINITY;
        }
      }
      unsigned pp[8], pd[8];  // P and dS of this lane, bf16 pairs
#pragma unroll
      for (int J = 0; J < 4; ++J) {
        const float4 lv = *reinterpret_cast<const float4*>(l2 + 8 * J + 4 * h2);
        const float4 dv4 = *reinterpret_cast<const float4*>(l2 + 32 + 8 * J + 4 * h2);
        const float lr[4] = {lv.x, lv.y, lv.z, lv.w}, dr[4] = {dv4.x, dv4.y, dv4.z, dv4.w};
        float pv[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          pv[j] = exp2_fast(fmaf(s[4 * J + j], a.c2, -lr[j]));
          dp[4 * J + j] = pv[j] * (dp[4 * J + j] - dr[j]);
        }
#pragma unroll
        for (int j = 0; j < 4; j += 2) {
          pp[2 * J + j / 2] = pack_bf16x2(pv[j], pv[j + 1]);
          pd[2 * J + j / 2] = pack_bf16x2(dp[4 * J + j], dp[4 * J + j + 1]);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int j = 0; j < 2 * DB; ++j) {
        read_group(tq, KS + j + RS - 1);
        __builtin_amdgcn_sched_barrier(0);
        const int g = j / DB, db = j % DB, c = (KS + j) % RS;
        dv[db] = mfma(fr[c][0], __builtin_bit_cast(bf16x8, u32x4{pp[4 * g], pp[4 * g + 1], pp[4 * g + 2], pp[4 * g + 3]}), dv[db]);
        dk[db] = mfma(fr[c][1], __builtin_bit_cast(bf16x8, u32x4{pd[4 * g], pd[4 * g + 1], pd[4 * g + 2], pd[4 * g + 3]}), dk[db]);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    if (it + 1 < steps) store_stat(st ^ 1);
  };
  for (int it = 0; it < steps; it += 2) {
    step(it, Stage<0>{});
    if (it + 1 < steps) step(it + 1, Stage<1>{});
  }
  if constexpr (PACKED) {
    if (units > 1) {
      if (k0 + 32 * w < N) {
        store_part<DB>(unit_part(a, sp, unit, sp.tile * NW + w, hd / nh, 0, D), dk, lane, a.rs);
        store_part<DB>(unit_part(a, sp, unit, sp.tile * NW + w, hd / nh, 1, D), dv, lane, 1.0f);
      }
      return;
    }
  }
  if (live) {
    bf16_t* dst = a.d_qkv + (tok0 + kw) * ld + (long)hd * D;
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      store_cols(dst + sp.k + 32 * db, dk[db], h2, a.rs);
      store_cols(dst + sp.v + 32 * db, dv[db], h2, 1.0f);
    }
  }
}

template <int D, bool CAUSAL>
__global__ __launch_bounds__(256, 2) void attn_dkdv_kernel(AttnArgs a) {
  __shared__ __attribute__((aligned(1024))) char lds[kDkdvLds<D>];
  dkdv_rows<D, CAUSAL, false>(a, lds, blockIdx.x, gridDim.x);
}

// The packed backward: kblocks blocks of dK and dV, from block k0 on, and the blocks of dQ
// before (k0 > 0) or behind them, in one launch, so that neither waits for the other's last
// blocks; delta is attn_delta_kernel's. The whole backward in us, two launches (dQ's with
// delta) and so: one sequence of 512, 8 heads of 128, causal 48, 29; 1024, 16 on 4 of 64 50, 35;
// 2031, 16 on 2 of 128 133, 103; 16384 tokens in 12 of 46 to 8021, 32 on 8 2500, 2233, in 18 of 76
// to 5801 1646, 1508. Where dQ's blocks are few they go first, as a block's walk over
// its keys takes longer than a unit of dK and dV: 4096 tokens, 4 heads on 4 of 64 125, 94, 16 on
// 16 of 128 304, 290; many go last: the 12 sequences 2490, 2233; 16384, 8 on 1 2027, 1791.
template <int D, bool CAUSAL>
__global__ __launch_bounds__(256, 2) void attn_packed_bwd_kernel(AttnArgs a, unsigned kblocks,
                                                                 unsigned k0) {
  constexpr int n = kDqLds<D> > kDkdvLds<D> ? kDqLds<D> : kDkdvLds<D>;
  __shared__ __attribute__((aligned(1024))) char lds[n];
  // (unsigned: blocks before k0 are not below kblocks)
  if (blockIdx.x - k0 < kblocks) dkdv_rows<D, CAUSAL, true>(a, lds, blockIdx.x - k0, kblocks);
  else dq_rows<D, CAUSAL, true, false>(a, lds, k0 > 0 ? blockIdx.x : blockIdx.x - kblocks, gridDim.x - kblocks);
}

// delta = rowsum(dO * O) per head and row, D / 8 lanes each (of the rows of no sequence
// whatever they hold: dQ's blocks clear it)
template <int D>
__global__ __launch_bounds__(256) void attn_delta_kernel(AttnArgs a) {
  constexpr int L = D / 8;
  const long n = (long)a.T * a.heads, step = (long)gridDim.x * (256 / L);
  for (long i = (long)blockIdx.x * (256 / L) + threadIdx.x / L; i < n; i += step) {
    const long off = i * D + 8 * (threadIdx.x % L);
    float g[8], o[8], s = 0.0f;
    load8(a.d_o + off, g);
    load8(a.o + off, o);
#pragma unroll
    for (int e = 0; e < 8; ++e) s += g[e] * o[e];
#pragma unroll
    for (int m = L / 2; m > 0; m >>= 1) s += __shfl_xor(s, m);
    if (threadIdx.x % L == 0) a.delta[i % a.heads * a.T + i / a.heads] = s;
  }
}

// dK and dV of the tiles that were cut, their units' sums added in order: a block a tile of
// 128 rows of a key head and 32 columns of K (blockIdx.y < D / 32) or V. B units in flight.
template <int D, bool CAUSAL, int B>
__global__ __launch_bounds__(256) void attn_join_kernel(AttnArgs a) {
  constexpr int DB = D / 32;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6),
            h2 = lane >> 5, lq = lane & 31;
  const int kv = blockIdx.y / DB, db = blockIdx.y % DB, g = (int)(blockIdx.x % a.kv);
  Span sp;
  if (!locate(a, (int)(blockIdx.x / a.kv), 128, false, lane, sp) || sp.none) return;
  const int steps = key_steps(sp.N, sp.tile, a.heads / a.kv, CAUSAL);
  if (steps <= kMinSteps) return;
  int len;
  const int units = tile_units(steps, unit_steps(a, CAUSAL, lane), a.units, len);
  const int row = 128 * sp.tile + 32 * w;
  if (units == 1 || row >= sp.N) return;
  const float* p = unit_part(a, sp, 0, row / 32, g, kv, D);
  const long next = (long)a.rows32 * a.kv * 64 * D;
  floatx16 x = zero16();
  for (int u = 0; u < units; u += B) {
    float4 v[B][4];
#pragma unroll
    for (int e = 0; e < B; ++e)
#pragma unroll
      for (int J = 0; J < 4; ++J)
        v[e][J] = *reinterpret_cast<const float4*>(p + min(u + e, units - 1) * next +
                                                   ((db * 4 + J) * 64 + lane) * 4);
#pragma unroll
    for (int e = 0; e < B; ++e)
      if (u + e < units)
#pragma unroll
        for (int J = 0; J < 4; ++J) {
          x[4 * J] += v[e][J].x;
          x[4 * J + 1] += v[e][J].y;
          x[4 * J + 2] += v[e][J].z;
          x[4 * J + 3] += v[e][J].w;
        }
  }
  if (row + lq >= sp.N) return;
  const int col = (a.heads + kv * a.kv + g) * D + 32 * db;
  store_cols(a.d_qkv + (sp.tok0 + row + lq) * ((long)(a.heads + 2 * a.kv) * D) + col, x, h2, 1.0f);
}

AttnArgs attn_args(const AttnShape& m, int T, int M) {
  AttnArgs a = {};
  a.T = T;
  a.M = M;
  a.N = m.N;
  a.heads = m.heads;
  a.nseq = m.N > 0 ? T / m.N : 0;
  a.c2 = kLog2e / sqrtf((float)m.D);
  a.rs = 1.0f / sqrtf((float)m.D);
  return a;
}

unsigned attn_blocks(const AttnArgs& a, int rows = 128) {
  return (unsigned)(((a.N + rows - 1) / rows) * a.heads * a.nseq);
}

// pair long and short causal tiles (decode) when the grid (two blocks per CU) is
// resident all at once: then the makespan is a CU's two blocks together, not
// the longest-first order's
int attn_pair(const AttnShape& m, const AttnArgs& a) {
  return m.causal && attn_blocks(a) <= 2u * 256u ? 1 : 0;
}

// Forward of heads of 64 in blocks of 8 waves, which read K and V half as often:
// where they are two rounds of two to a CU at least, and leave no half of a block
// without queries. 4 and 8 waves, us: 32 and 64 sequences of 512, 16 heads,
// bidirectional 58 and 51, 110 and 95; 16 sequences (one round), causal 21.8 and 23.0;
// 128 of 128 (half empty) 29 and 33; 4 of 700, 48 heads (576 blocks) 41 and 45.
bool fwd_wide(const AttnArgs& a) {
  return attn_blocks(a, 256) >= 4u * 256u && 2 * attn_blocks(a, 256) == attn_blocks(a);
}

// Query tiles of a head side by side (decode)? Bidirectional ones have equal work and
// lose nothing by it: 64 sequences of 512, 16 heads of 128, forward 263 -> 198 us (227
// with the 8-wave blocks before the one-tile-ahead loop, which read K and V half as
// often), dQ 378 -> 301; 4 x 4096, 32 heads 1110 -> 1013 and 1646 -> 1521; one sequence
// of 4096 the same. Causal tiles then no longer run longest first over the whole launch,
// which costs up to 40 % where K and V stay in the 256 MB Infinity Cache; the forward
// takes it where they do not (kv: their bytes) and the tiles of a head are few, or far
// past it (T = 65536, heads of 128, width 2048: N = 512 421 -> 349 us, 1024 632 -> 447, 2048
// 1004 -> 717, 4096 1345 -> 1208; half of that 199 -> 182, 261 -> 227, 375 -> 351, and
// 580 -> 592 for 4096; N = 300, 189 MB, heads of 128 and 64, 143 -> 120 and 163 -> 129).
// 8-wave blocks have half as many tiles and gain little (2-4 %) or lose up to 12 %.
// The key tiles of dK and dV gain 11 % and lose 8 % on the bidirectional shapes, and
// keep their order.
bool shared_order(const AttnShape& m, const AttnArgs& a) {
  if (!m.causal) return true;
  if (m.D == 64 && fwd_wide(a)) return false;
  const long mb = 1L << 20, kv = 4L * a.T * a.M, nt = (a.N + 127) / 128;
  return kv >= 448 * mb || (kv >= 176 * mb && nt <= 3) ||
         (kv >= 240 * mb && m.D == 128 && nt <= 16);
}

template <int D, int NW>
void launch_fwd(const AttnShape& m, const AttnArgs& a, hipStream_t st) {
  const dim3 g(attn_blocks(a, 32 * NW)), b(64 * NW);
  if (m.causal) hipLaunchKernelGGL((attn_fwd_kernel<D, true, NW, false, 1>), g, b, 0, st, a);
  else hipLaunchKernelGGL((attn_fwd_kernel<D, false, NW, false, 1>), g, b, 0, st, a);
}

#define FLOWMOE_ATTN_LAUNCH(KERNEL, a, st)                                     \
  do {                                                                            \
    const dim3 g(attn_blocks(a)), b(256);                                         \
    if (m.D == 128) {                                                             \
      if (m.causal) hipLaunchKernelGGL((KERNEL<128, true>), g, b, 0, st, a);      \
      else hipLaunchKernelGGL((KERNEL<128, false>), g, b, 0, st, a);              \
    } else {                                                                      \
      if (m.causal) hipLaunchKernelGGL((KERNEL<64, true>), g, b, 0, st, a);       \
      else hipLaunchKernelGGL((KERNEL<64, false>), g, b, 0, st, a);               \
    }                                                                             \
  } while (0)

}  // namespace

hipError_t launch_attn_fwd(const AttnShape& m, int T, int M, const void* qkv, void* o, float* lse,
                           hipStream_t st) {
  AttnArgs a = attn_args(m, T, M);
  if (attn_blocks(a) == 0) return hipSuccess;
  a.qkv = static_cast<const bf16_t*>(qkv);
  a.out = static_cast<bf16_t*>(o);
  a.lse = lse;
  a.pair = attn_pair(m, a);
  a.shared = shared_order(m, a);
  return traced(FLOWMOE_K_ATTN_FWD, st, [&] {
    if (m.D == 128) launch_fwd<128, 4>(m, a, st);
    else if (fwd_wide(a)) launch_fwd<64, 8>(m, a, st);
    else launch_fwd<64, 4>(m, a, st);
  });
}

hipError_t launch_attn_bwd(const AttnShape& m, int T, int M, const void* qkv, const void* o,
                           const float* lse, const void* d_o, void* d_qkv, float* delta,
                           hipStream_t st) {
  AttnArgs a = attn_args(m, T, M);
  if (attn_blocks(a) == 0) return hipSuccess;
  a.qkv = static_cast<const bf16_t*>(qkv);
  a.o = static_cast<const bf16_t*>(o);
  a.d_o = static_cast<const bf16_t*>(d_o);
  a.d_qkv = static_cast<bf16_t*>(d_qkv);
  a.lse = const_cast<float*>(lse);
  a.delta = delta;
  a.pair = attn_pair(m, a);
  a.shared = !m.causal;
  hipError_t e = traced(FLOWMOE_K_ATTN_BWD_DQ, st, [&] { FLOWMOE_ATTN_LAUNCH(attn_dq_kernel, a, st); });
  if (e != hipSuccess) return e;
  return traced(FLOWMOE_K_ATTN_BWD_DKDV, st,
                [&] { FLOWMOE_ATTN_LAUNCH(attn_dkdv_kernel, a, st); });
}

// ---------------------------------------------------------------------------
// packed sequences
// ---------------------------------------------------------------------------
namespace {

// Sequences so short on average that a wave a tile of 32 rows serves them best (packed_short.hip)?
// Up to 96 rows forward, 48 backward, 24 where a wave there walks more than two heads. The host
// knows the average alone, and a wave's walk over a long sequence is slow. us in blocks of 128
// rows and so, causal, 8 heads on 4 of 64, 16 on 16 and 32 on 4 of 128: forward of 8000 tokens in
// sequences of 32 13, 11; 50, 40; 93, 40; of 64 11, 8; 35, 28; 59, 41; of 128 11, 9; 47, 31; 50, 44; 6000
// in sequences of 1 to 500 13, 14; 35, 32; 57, 47; of 4000 and 100 of 20 54, 79; 96, 151; 164, 189.
// Backward of 8000 of 24 81, 19; 132, 80; 201, 150; of 32 68, 27; 157, 123; 167, 179; of 64 52, 24; 122,
// 90; 145, 140; 6000 of 40 to 120 49, 29; 105, 84; 142, 163; of 1 to 500 56, 62; 113, 114; 165, 376; of
// 4000 and 100 of 20 (59 on average) 170, 437; 313, 598; 534, 2723.
// The average counts empty entries of a list too, which send long sequences to the waves: in blocks
// and so, 2 of 2048 beside 254 empty ones forward 25, 45; 60, 80; 84, 112; backward 72, 227; 183, 327;
// 302, 772; with 16 heads on 2 of 128 179, 1268.
bool packed_short_fwd(const PackedShape& m, int T) { return T <= 96L * m.nseq; }
bool packed_short_bwd(const PackedShape& m, int T) {
  return T <= (m.heads / m.kv <= 2 ? 48L : 24L) * m.nseq;
}

// blocks of a packed grid: its slots (locate) times `per` heads
unsigned packed_blocks(const AttnArgs& a, int rows, int per) {
  return (unsigned)((a.T / rows + a.nseq + 1) * (long)per);
}

// The most units of a tile: as many as bring the units' sums to 256 MiB (K and V in float: 8 D bytes
// a row and unit), rounded up, so that they are below 512; few rows are cut the most. None where no
// tile has the steps, or so many sequences that a block's sum over them would take as long as it
// saves.
void packed_units(const PackedShape& m, int T, AttnArgs& a) {
  const long rows32 = T / 32 + (long)m.nseq + 1, steps = (T + 31) / 32 * (m.heads / m.kv);
  const long most = (262144L * 128 / m.D + rows32 * 32 * m.kv - 1) / (rows32 * 32 * m.kv);
  a.rows32 = (int)rows32;
  a.units = m.nseq > 4096 || steps <= 2 * kMinSteps ? 1 : (int)std::min(most, 32L);
}
size_t part_bytes(const PackedShape& m, const AttnArgs& a) {
  return a.units > 1 ? (size_t)a.units * a.rows32 * m.kv * 64 * m.D * sizeof(float) : 0;
}

}  // namespace

size_t packed_attn_ws_bytes(const PackedShape& m, int T) {
  AttnArgs a = {};
  packed_units(m, T, a);
  return T == 0 || packed_short_bwd(m, T) ? 0 : part_bytes(m, a);
}

template <int D, int S>
void run_packed_fwd(const PackedShape& m, const AttnArgs& a, hipStream_t st) {
  const dim3 g(packed_blocks(a, 128, m.heads)), b(256 * S);
  if (m.causal) hipLaunchKernelGGL((attn_fwd_kernel<D, true, 4, true, S>), g, b, 0, st, a);
  else hipLaunchKernelGGL((attn_fwd_kernel<D, false, 4, true, S>), g, b, 0, st, a);
}
// The forward's waves in two groups that share a block's queries, each with every other key tile?
// Where the launch's blocks are two to a CU at most and sequences are long. us of one sequence,
// causal, one group and two: 2048 tokens, 8 heads of 128 40, 37; 16 on 4 of 64 29, 25; 1024 23, 23
// and 17, 15; 512 15, 16 and 11, 10; 2031, 16 on 2 of 128 42, 38; 544 blocks (2048, 32 on 8) 51,
// 53. Four groups are no better.
bool packed_split(const PackedShape& m, const AttnArgs& a) {
  return packed_blocks(a, 128, m.heads) <= 512 && a.T >= (m.D == 128 ? 1024L : 512L) * m.nseq;
}

hipError_t launch_packed_attn_fwd(const PackedShape& m, int T, const void* qkv,
                                  const int32_t* starts, void* o, float* lse, hipStream_t st) {
  if (T == 0) return hipSuccess;
  if (packed_short_fwd(m, T)) return launch_short_attn_fwd(m, T, qkv, starts, o, lse, st);
  AttnArgs a = packed_args(m, T, qkv, starts);
  a.out = static_cast<bf16_t*>(o);
  a.lse = lse;
  return traced(FLOWMOE_K_ATTN_FWD, st, [&] {
    const bool split = packed_split(m, a);
    if (m.D == 128 && split) run_packed_fwd<128, 2>(m, a, st);
    else if (m.D == 128) run_packed_fwd<128, 1>(m, a, st);
    else if (split) run_packed_fwd<64, 2>(m, a, st);
    else run_packed_fwd<64, 1>(m, a, st);
  });
}

namespace {

template <int B>
void run_join(const PackedShape& m, const AttnArgs& a, hipStream_t st) {
  const dim3 g(packed_blocks(a, 128, m.kv), 2 * m.D / 32), b(256);
  if (m.D == 128) {
    if (m.causal) hipLaunchKernelGGL((attn_join_kernel<128, true, B>), g, b, 0, st, a);
    else hipLaunchKernelGGL((attn_join_kernel<128, false, B>), g, b, 0, st, a);
  } else {
    if (m.causal) hipLaunchKernelGGL((attn_join_kernel<64, true, B>), g, b, 0, st, a);
    else hipLaunchKernelGGL((attn_join_kernel<64, false, B>), g, b, 0, st, a);
  }
}
hipError_t join_packed(const PackedShape& m, const AttnArgs& a, hipStream_t st) {
  return traced(FLOWMOE_K_PACKED_JOIN, st, [&] {
    if (a.units <= 2) run_join<2>(m, a, st);
    else run_join<8>(m, a, st);
  });
}

}  // namespace

hipError_t launch_packed_attn_bwd(const PackedShape& m, int T, const void* qkv,
                                  const int32_t* starts, const void* o, const float* lse,
                                  const void* d_o, void* d_qkv, float* delta, void* ws,
                                  hipStream_t st) {
  if (T == 0) return hipSuccess;
  if (packed_short_bwd(m, T))
    return launch_short_attn_bwd(m, T, qkv, starts, o, lse, d_o, d_qkv, delta, st);
  AttnArgs a = packed_args(m, T, qkv, starts);
  a.o = static_cast<const bf16_t*>(o);
  a.d_o = static_cast<const bf16_t*>(d_o);
  a.d_qkv = static_cast<bf16_t*>(d_qkv);
  a.lse = const_cast<float*>(lse);
  a.delta = delta;
  packed_units(m, T, a);
  a.part = static_cast<float*>(ws);
  hipError_t e = traced(FLOWMOE_K_ATTN_BWD_DQ, st, [&] {
    const dim3 g((unsigned)std::min(((long)T * a.M / 8 + 255) / 256, 1L << 20)), b(256);
    if (m.D == 128) hipLaunchKernelGGL(attn_delta_kernel<128>, g, b, 0, st, a);
    else hipLaunchKernelGGL(attn_delta_kernel<64>, g, b, 0, st, a);
  });
  if (e != hipSuccess) return e;
  e = traced(FLOWMOE_K_ATTN_BWD_DKDV, st, [&] {
    const unsigned k = packed_blocks(a, 128, m.kv * a.units), q = packed_blocks(a, 128, m.heads),
                   k0 = q <= 1024 ? q : 0;
    const dim3 g(k + q), b(256);
    if (m.D == 128) {
      if (m.causal) hipLaunchKernelGGL((attn_packed_bwd_kernel<128, true>), g, b, 0, st, a, k, k0);
      else hipLaunchKernelGGL((attn_packed_bwd_kernel<128, false>), g, b, 0, st, a, k, k0);
    } else {
      if (m.causal) hipLaunchKernelGGL((attn_packed_bwd_kernel<64, true>), g, b, 0, st, a, k, k0);
      else hipLaunchKernelGGL((attn_packed_bwd_kernel<64, false>), g, b, 0, st, a, k, k0);
    }
  });
  return e != hipSuccess || a.units == 1 ? e : join_packed(m, a, st);
}

size_t packed_mha_ws_bytes(const PackedShape& m, int T) {
  const int M = m.heads * m.D, W = M + 2 * m.kv * m.D;
  return align256(std::max(packed_attn_ws_bytes(m, T),
                           std::max(wgrad_part_bytes(M, W, T), wgrad_part_bytes(M, M, T))));
}

hipError_t launch_packed_mha_fwd(const PackedShape& m, const RopeShape* r, int T,
                                 const flowmoe_packed_mha_bufs_t& b, hipStream_t st) {
  if (T == 0) return hipSuccess;
  if (r != nullptr && !rope_fits(*r, T)) return hipErrorInvalidConfiguration;  // (before any launch)
  const int M = m.heads * m.D, W = M + 2 * m.kv * m.D;
  hipError_t e = launch_dense_gemm(FLOWMOE_K_ATTN_QKV, T, b.in, M, M, b.w_qkv, W, false, W, b.qkv, W, st);
  if (e == hipSuccess && r != nullptr)
    e = launch_rope(*r, FLOWMOE_BF16, T, W, false, b.qkv, b.positions, b.qkv, st);
  if (e == hipSuccess) e = launch_packed_attn_fwd(m, T, b.qkv, b.starts, b.attn, b.lse, st);
  if (e != hipSuccess) return e;
  return launch_dense_gemm(FLOWMOE_K_ATTN_OUT, T, b.attn, M, M, b.w_o, M, false, M, b.out, M, st);
}

hipError_t launch_packed_mha_bwd(const PackedShape& m, const RopeShape* r, int T,
                                 const flowmoe_packed_mha_bufs_t& b, int accumulate,
                                 hipStream_t st) {
  if (r != nullptr && !rope_fits(*r, T)) return hipErrorInvalidConfiguration;
  const int M = m.heads * m.D, W = M + 2 * m.kv * m.D;
  hipError_t e = hipSuccess;
  if (T > 0) {
    e = launch_dense_gemm(FLOWMOE_K_ATTN_DGRAD, T, b.d_out, M, M, b.w_o, M, true, M, b.d_attn, M, st);
    if (e == hipSuccess)
      e = launch_packed_attn_bwd(m, T, b.qkv, b.starts, b.attn, b.lse, b.d_attn, b.d_qkv, b.delta,
                                 b.ws, st);
    if (e == hipSuccess && r != nullptr)
      e = launch_rope(*r, FLOWMOE_BF16, T, W, true, b.d_qkv, b.positions, b.d_qkv, st);
    if (e == hipSuccess)
      e = launch_dense_gemm(FLOWMOE_K_ATTN_DGRAD, T, b.d_qkv, W, W, b.w_qkv, W, true, M, b.d_in, M, st);
  }
  float* part = static_cast<float*>(b.ws);
  if (e == hipSuccess)
    e = launch_dense_wgrad(FLOWMOE_K_ATTN_WGRAD, T, 1, b.attn, M, 0, M, b.d_out, M, 0, M, b.dw_o, M,
                           accumulate, wgrad_part_bytes(M, M, T) ? part : nullptr, st);
  if (e == hipSuccess)
    e = launch_dense_wgrad(FLOWMOE_K_ATTN_WGRAD, T, 1, b.in, M, 0, M, b.d_qkv, W, 0, W, b.dw_qkv, W,
                           accumulate, wgrad_part_bytes(M, W, T) ? part : nullptr, st);
  return e;
}

hipError_t launch_mha_fwd(const AttnShape& m, int T, int M, const void* in, const void* w_qkv,
                          const void* w_o, void* qkv, void* attn, float* lse, void* out,
                          hipStream_t st) {
  if (T == 0) return hipSuccess;
  hipError_t e = launch_dense_gemm(FLOWMOE_K_ATTN_QKV, T, in, M, M, w_qkv, 3L * M, false, 3 * M,
                                   qkv, 3L * M, st);
  if (e != hipSuccess) return e;
  e = launch_attn_fwd(m, T, M, qkv, attn, lse, st);
  if (e != hipSuccess) return e;
  return launch_dense_gemm(FLOWMOE_K_ATTN_OUT, T, attn, M, M, w_o, M, false, M, out, M, st);
}

hipError_t launch_mha_bwd_data(const AttnShape& m, int T, int M, const void* w_qkv,
                               const void* w_o, const void* qkv, const void* attn,
                               const float* lse, const void* d_out, void* d_attn, void* d_qkv,
                               float* delta, void* d_in, hipStream_t st) {
  if (T == 0) return hipSuccess;
  // d_attn = d_out W^O^T: B[k][n] = W^O[n][k] (K-contiguous)
  hipError_t e = launch_dense_gemm(FLOWMOE_K_ATTN_DGRAD, T, d_out, M, M, w_o, M, true, M, d_attn,
                                   M, st);
  if (e != hipSuccess) return e;
  e = launch_attn_bwd(m, T, M, qkv, attn, lse, d_attn, d_qkv, delta, st);
  if (e != hipSuccess) return e;
  // d_in = d_qkv [W^Q | W^K | W^V]^T: B[k][n] = W_qkv[n][k] (K-contiguous)
  return launch_dense_gemm(FLOWMOE_K_ATTN_DGRAD, T, d_qkv, 3L * M, 3 * M, w_qkv, 3L * M, true, M,
                           d_in, M, st);
}

hipError_t launch_mha_wgrad(int T, int M, int R, const void* in, const void* attn,
                            const void* d_out, const void* d_qkv, float* dw_qkv, float* dw_o,
                            int accumulate, void* ws, hipStream_t st) {
  // dW^O = attn^T d_out and dW_qkv = in^T d_qkv, each summed over the R
  // chunks' rows in chunk order (through partial sums in ws when their
  // output tiles are too few for the CUs)
  float* part = static_cast<float*>(ws);
  hipError_t e = launch_dense_wgrad(FLOWMOE_K_ATTN_WGRAD, T, R, attn, M, (long)T * M, M, d_out, M,
                                    (long)T * M, M, dw_o, M, accumulate, part, st);
  if (e != hipSuccess) return e;
  return launch_dense_wgrad(FLOWMOE_K_ATTN_WGRAD, T, R, in, M, (long)T * M, M, d_qkv, 3L * M,
                            (long)T * 3 * M, 3 * M, dw_qkv, 3L * M, accumulate, part, st);
}

}  // namespace flowmoe
