// Differential attention (arXiv 2410.05258, Sec. 2.1) in the place of AT_r's softmax
// attention: head h has two query/key pairs of width d = D / 2, one value of width D,
// and a learned weight lambda_h,
//   P_i = softmax(Q_i K_i^T / sqrt(d)),   A = P_1 V - lambda_h P_2 V.
// Q_1 | Q_2 and K_1 | K_2 lie side by side in the head's D columns, so that a tile of
// K rows in LDS holds both maps' keys: k steps 0 .. KS/2 - 1 of a row read are the
// first map's, the others the second's. Query heads share key/value heads in groups.
//
// The tiles, operand forms and softmax are those of attn.hip. A padded batch gives
// each sequence's number of valid tokens: later tokens are no one's keys, their
// K, V, Q and dO rows are never used (tile loads past a sequence's length give
// zeros, without traffic, so that whatever they hold cannot reach a sum), and their
// outputs and gradients are zeros.
//
// Forward: a wave runs the online softmax of one map for 32 queries and its own P_i V;
// the second map's hands P_2 V to the first's through LDS at the end. P_2 V is kept for
// the backward as well.
//
// Backward (no atomics; every sum in a fixed order), with dP = dA V^T, which both
// maps share, d2 = rowsum(dA * P_2 V) and d1 = rowsum(dA * A) + lambda d2:
//   dS_1 = P_1 (dP - d1), dS_2 = -lambda P_2 (dP - d2),
//   dQ_i = dS_i K_i / sqrt(d), dK_i = dS_i^T Q_i / sqrt(d),
//   dV = (P_1 - lambda P_2)^T dA (one product), dlambda_h = -sum of d2 over the rows.
// A key/value head's gradients are sums over the query heads of its group, in order.
//
// Rounded to bf16: probabilities before P_i V, and dS_i and P_1 - lambda P_2 before their
// products, as matrix operands of one type with the bf16 tensors they multiply; sums, softmax
// statistics and row sums are fp32. Against fp64, in the 2-norm, A is 2.2e-3 to 2.6e-3 off
// (the output's own rounding is 1.7e-3; the maps' common part cancels in A, their errors do
// not) and the gradients 2.3e-3. Probabilities in two bf16 parts, a product each, leave the
// output's rounding alone (1.7e-3), for 1378 us in place of 879 (4 x 4096 tokens, 32 heads of
// 128, causal), 38.6 of 31.1 (16 x 500, 16 heads of 64, padded). (fp16, 2^-11, would need V in
// fp16 too, whose range bf16 values exceed.) The row sum is of the unrounded ones, so that lse
// is exact to fp32.
//
// Times in this file are of calls on the same inputs; new inputs each pass add 1-3 % to long
// ones.
#include <math.h>

#include <algorithm>

#include "attn_tiles.hpp"
#include "common.hpp"

namespace flowmoe {
namespace {

struct DiffArgs {
  const bf16_t* qkv;     // T x W = [Q | K | V], W = (heads + 2 kv) D
  const float* lambda;   // heads
  const int32_t* lens;   // valid tokens of each sequence, or null
  const bf16_t* o;       // T x M: A (backward)
  const bf16_t* o2;      // T x M: P_2 V (backward)
  const bf16_t* d_o;     // T x M: dA (backward)
  bf16_t* out;           // forward: A
  bf16_t* out2;          // forward: P_2 V, or null
  bf16_t* d_qkv;         // backward: T x W
  float* lse;            // 2 x heads x T: log-sum-exp of each map's rows (forward: or null)
  float* delta;          // 2 x heads x T: d1, d2
  float* d_lambda;       // heads
  int T, N, heads, kv, nseq;
  int sub;               // N holds N / sub short sequences (tile_rows)
  int accumulate;        // add to d_lambda
  long M, W;             // columns of a row of A, of qkv
  float *part, *qpart;   // sums of units: dK and dV, dQ
  int unit, units;       // steps of a unit (0: uncut), units of a key head of a sequence
  int qunit, qunits;     // the same of dQ and a query head
  int kblocks;           // blocks of the join of dK and dV
  int shared, pair;      // order of the blocks (diff_decode)
  float c2;              // log2(e) / sqrt(d)
  float rs;              // 1 / sqrt(d)
};

// the valid tokens of sequence sq
__device__ __forceinline__ int seq_end(const DiffArgs& a, int sq) {
  return a.lens == nullptr ? a.N : min(max(a.lens[sq], 0), a.N);
}

// Sequences of at most 16 tokens: a tile holds as many whole ones as fit, N = 32 / sub * sub
// tokens (the last tile of a call fewer), so that its rows and products are not empty. A bit
// of `valid` is a row. us of one sequence a tile and of several: 3357 x 1 token, 16 heads of
// 128, forward 112, 19, backward 424, 54; 1339 x 3, 8 heads (4) of 64, causal, backward 45, 19;
// 452 x 10, 16 heads (8) of 128, causal 25, 22 and 65, 60.
struct TileRows {
  unsigned valid;
  int end, rows;  // past the last valid one; of the call
};
__device__ __forceinline__ TileRows tile_rows(const DiffArgs& a, int sq) {
  const int r = threadIdx.x & 31, rows = min(a.N, a.T - sq * a.N), s = r / a.sub;
  bool v = r < rows;
  if (v && a.lens != nullptr) v = r - s * a.sub < a.lens[sq * (a.N / a.sub) + s];
  const unsigned valid = (unsigned)__ballot(v);
  return {valid, 32 - __clz((int)valid), rows};
}
// the valid tokens that row r of them sees (causal), or is seen by
template <bool CAUSAL, bool BY>
__device__ __forceinline__ unsigned partners(const DiffArgs& a, unsigned valid, int r) {
  const unsigned own = (~0u >> (32 - a.sub)) << (r / a.sub * a.sub), upto = (2u << r) - 1u;
  const unsigned order = !CAUSAL ? ~0u : BY ? ~(upto >> 1) : upto;
  return valid >> r & 1 ? valid & own & order : 0u;
}
// zeros in the rows of a tile between valid ones that are not (those past the last are not
// loaded): what they hold must not reach a sum
template <int D, int THREADS>
__device__ __forceinline__ void clear_rows(char* tile, unsigned valid, int tid) {
  for (int i = tid; i < 4 * D; i += THREADS)
    if (!(valid >> (i / (D / 8)) & 1)) reinterpret_cast<float4*>(tile)[i] = make_float4(0.f, 0.f, 0.f, 0.f);
}
// A product multiplies another sequence's rows by zeros, which holds for finite ones only:
// a tile of several sequences where this finds an infinity or a NaN in a product's rows is
// run again a sequence at a time (the others' rows cleared).
template <int D>
__device__ __forceinline__ bool not_finite(const char* tile, int lane) {
  typedef unsigned short u16x8 __attribute__((ext_vector_type(8)));
  u16x8 top = 0;
#pragma unroll
  for (int i = 0; i < D / 16; ++i)
    top = __builtin_elementwise_max(top, reinterpret_cast<const u16x8*>(tile)[64 * i + lane] & (unsigned short)0x7FFF);
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 8; ++i) bad = bad || top[i] >= 0x7F80;
  return __any(bad);
}
// x, or `other` where bit i of `seen` is not set
__device__ __forceinline__ float where_bit(unsigned seen, int i, float x, float other) {
  const unsigned m = (unsigned)__builtin_amdgcn_sbfe((int)seen, i, 1);
  return __uint_as_float((__float_as_uint(x) & m) | (__float_as_uint(other) & ~m));
}

// block -> (tile, head, sequence): tiles of the most causal work first (`rev`: the
// last query tiles), all heads of a tile side by side. `pair` (every block resident at
// once): the second half of the grid, which lands on the CUs of the first, runs the
// least work first, so that a CU's blocks have complementary work. `shared`: the tiles
// of a head one after the other on one XCD, so that its K and V are read through that
// L2 once.
__device__ __forceinline__ void diff_decode(const DiffArgs& a, int heads, bool rev, int rows,
                                            int& tile, int& hd, int& sq) {
  const int per = heads * a.nseq, nt = (a.N + rows - 1) / rows;
  if (a.shared && per % 8 == 0) {
    const int i = blockIdx.x >> 3, rest = i / nt * 8 + (blockIdx.x & 7);
    tile = rev ? nt - 1 - i % nt : i % nt;
    hd = rest % heads;
    sq = rest / heads;
    return;
  }
  const int u = (int)(blockIdx.x / per), rest = (int)(blockIdx.x % per), h = (nt + 1) / 2;
  const int r = a.pair && u >= h ? nt - 1 - (u - h) : u;
  tile = rev ? nt - 1 - r : r;
  hd = rest % heads;
  sq = rest / heads;
}

// Forward: NW waves, two (one a map) for each 32 queries and each of S parts of a key
// tile: with S > 1 a block has fewer queries and its waves share their keys.
//
// A wave has one map, not both: both maps' P_i V of 32 queries would take 128 of a
// lane's registers at D = 128, one map's take 64, and four waves fit a SIMD (128
// registers), whose softmaxes and products overlap. The 32 keys' scores, their softmax
// and their products follow each other in a wave. 4 x 4096 tokens, 32 heads of 128,
// causal: two waves a SIMD, 64 keys at a time 1030 us; the same one tile ahead of itself
// 973; four waves 897, 32 keys at a time 879 (938 TFLOP/s, 0.59 of what a large matrix
// product reaches here). A timing copy without the exponentials takes 817. Matrix pipes and
// LDS are busy for half of the cycles each, at a clock of 1.4-1.6 GHz: power, and the waits
// of one for the other.
template <int NW, int S>
struct FwdTile {
  static constexpr int G = NW / (2 * S), QB = 32 * G;  // groups of 32 queries, queries
  static constexpr int KB = S == 1 && NW == 8 ? 2 : 1, KT = 32 * KB * S;  // keys of a wave / 32, of a tile
};
// The tile's rows in `own` are written; false: none, its sequences have to run one by one.
template <int D, bool CAUSAL, int NW, int S, int ONE>
__device__ __forceinline__ bool diff_fwd_tile(const DiffArgs& a, char* lds, float2* stat,
                                              const TileRows& tr, unsigned own, int qt, int hd, int sq) {
  using Tile = FwdTile<NW, S>;
  // slots: ONE for sequences of one tile (1) or less (2) (more blocks to a CU)
  constexpr int SL = ONE ? 1 : 2;
  constexpr bool PACK = ONE == 2;  // several to a tile
  constexpr int KS = D / 32, DB = D / 32, QB = Tile::QB, KT = Tile::KT;  // KS: k steps of one map
  using Dma = TileDma<D, KT, NW>;
  constexpr int TB = Dma::TB;
  static_assert(2 * SL * TB >= (S > 1 ? NW : NW / 2) * 32 * D * 4, "the outputs fit the tiles' place");
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6),
            h2 = lane >> 5, lq = lane & 31;
  const int map = w & 1, grp = (w >> 1) % Tile::G, part = (w >> 1) / Tile::G;
  const int end = tr.end;
  const long tok0 = (long)sq * a.N, ld = a.W;
  const int q0 = qt * QB, qw = q0 + 32 * grp + lq;
  const unsigned seen = PACK ? partners<CAUSAL, false>(a, tr.valid, lq) : 0u;
  const bool live = PACK ? seen != 0u : qw < end;

  floatx16 o[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) o[db] = zero16();
  float m = -INFINITY, l = 1.0f;
  if (q0 < end) {  // (else padding only)
    const int kh = hd / (a.heads / a.kv);
    const bf16_t* Qg = a.qkv + tok0 * ld + (long)hd * D;
    const bf16_t* Kg = a.qkv + tok0 * ld + a.M + (long)kh * D;
    const bf16_t* Vg = Kg + (long)a.kv * D;
    const int kend = CAUSAL ? min(end, q0 + QB) : end;
    const int nk = (kend + KT - 1) / KT;
    const Dma dma(lds_base(lds), w, lane, ld);
    const long kstep = KT * ld;
    dma.load(Kg, kend, 0);
    dma.load(Vg, kend, SL * TB);
    bf16x8 qf[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
      qf[ks] = live ? *reinterpret_cast<const bf16x8*>(Qg + qw * ld + 16 * (KS * map + ks) + 8 * h2)
                    : zero8();
    l = 0.0f;
    int rbase = row_base<D>(lq, h2), tb0 = tr_base<D>(lane, 0), tb1 = tr_base<D>(lane, 1);

    auto step = [&](const int t, auto stc) __attribute__((always_inline)) {
      constexpr int st = decltype(stc)::value;
      opaque(rbase, tb0, tb1);
      wait_vm<0>();   // K(t) and V(t): loaded a step ago
      lds_barrier();  // and every wave's reads of the slots refilled now are done
      const char* tk = lds + st * TB;
      const char* tv = lds + (SL + st) * TB;
      if constexpr (!ONE) {
        Kg += kstep;  // K(t + 1), V(t + 1)
        Vg += kstep;
        dma.load(Kg, kend - KT * (t + 1), (st ^ 1) * TB);
        dma.load(Vg, kend - KT * (t + 1), (SL + (st ^ 1)) * TB);
      }
#pragma unroll
      for (int j = 0; j < Tile::KB; ++j) {
        const int kb = Tile::KB * part + j, kb0 = KT * t + 32 * kb;
        // (causal: nothing for a wave whose queries all precede these keys)
        if (CAUSAL && kb0 > q0 + 32 * grp + 31) return;
        floatx16 s;
#pragma unroll
        for (int i = 0; i < KS; ++i)
          s = mfma(frag_row_x<D>(tk, rbase, 32 * kb, KS * map + i), qf[i], i == 0 ? zero16() : s);
        if constexpr (PACK) {
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] = where_bit(seen >> 4 * h2, 8 * (r >> 2) + (r & 3), s[r], -INFINITY);
        } else if (kb0 + 32 > end || (CAUSAL && kb0 + 31 > q0 + 32 * grp)) {
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int key = kb0 + 8 * (r >> 2) + 4 * h2 + (r & 3);
            if (key >= end || (CAUSAL && key > qw)) s[r] = -INFINITY;
          }
        }
        float mx = s[0];
#pragma unroll
        for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[r]);
        // the reference moves only when a score exceeds it by more than 2^8 (attn.hip).
        // Every query sees key 0, so it is finite from its first tile on, but in the
        // waves that key 0 is not given to a row may see no key yet
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
        const float ref = S > 1 && m == -INFINITY ? 0.0f : m;
        unsigned pw[8];  // this lane's 16 probabilities, rounded to bf16 for the product
        float rsum = 0.0f;
#pragma unroll
        for (int q = 0; q < 16; q += 2) {
          const float p0 = exp2_fast(fmaf(s[q], a.c2, -ref));
          const float p1 = exp2_fast(fmaf(s[q + 1], a.c2, -ref));
          rsum += p0;
          rsum += p1;
          pw[q >> 1] = pack_bf16x2(p0, p1);
        }
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          const bf16x8 pb = __builtin_bit_cast(bf16x8, u32x4{pw[4 * g], pw[4 * g + 1], pw[4 * g + 2], pw[4 * g + 3]});
#pragma unroll
          for (int db = 0; db < DB; ++db)
            o[db] = mfma(frag_tr_x<D>(tv, tb0, tb1, 32 * kb + 16 * g, 32 * db), pb, o[db]);
        }
        l += pair_sum(rsum);
      }
    };
    if constexpr (ONE) {
      if constexpr (PACK) {
        wait_vm<0>();
        lds_barrier();
        if (tr.valid & (tr.valid + 1)) {
          clear_rows<D, 64 * NW>(lds + TB, tr.valid, tid);
          lds_barrier();
        }
        if (own == ~0u && not_finite<D>(lds + TB, lane)) return false;
      }
      step(0, Stage<0>{});
    } else {
      for (int t = 0; t < nk; t += 2) {
        step(t, Stage<0>{});
        if (t + 1 < nk) step(t + 1, Stage<1>{});
      }
    }
    // The waves of a part own the 32-column blocks db = part (mod S) of their rows: each hands
    // the others theirs, lane by lane, and adds up its own; then the second map's hand
    // theirs to the first's (in slots that the first exchange left free)
    auto slot = [&](int mp, int p, int db) {
      const int owner = S > 1 ? (grp * 2 + mp) * S + p : grp;
      return reinterpret_cast<float4*>(lds) + (long)(owner * DB + db) * 256 + lane;
    };
    auto put = [&](float4* x, const floatx16& v) {
#pragma unroll
      for (int J = 0; J < 4; ++J) x[J * 64] = make_float4(v[4 * J], v[4 * J + 1], v[4 * J + 2], v[4 * J + 3]);
    };
    wait_vm<0>();  // (the loads past the last tile write zeros)
    lds_barrier();
    if constexpr (S > 1) {
#pragma unroll
      for (int db = 0; db < DB; ++db)
        if (db % S != part) put(slot(map, part, db), o[db]);
      stat[w * 64 + lane] = make_float2(m, l);
      lds_barrier();
      float f[S], mn = -INFINITY;
#pragma unroll
      for (int p = 0; p < S; ++p) mn = fmaxf(mn, stat[(((p * Tile::G + grp) << 1) | map) * 64 + lane].x);
      const float ref = mn == -INFINITY ? 0.0f : mn;  // (part 0 has key 0: finite where the row is live)
      l = 0.0f;
#pragma unroll
      for (int p = 0; p < S; ++p) {
        const float2 x = stat[(((p * Tile::G + grp) << 1) | map) * 64 + lane];
        f[p] = exp2_fast(x.x - ref);
        l += x.y * f[p];
      }
      const float fo = exp2_fast(m - ref);
      m = mn;
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        if (db % S != part) continue;
        floatx16 s = o[db] * fo;
#pragma unroll
        for (int p = 0; p < S; ++p) {
          if (p == part) continue;
          const float4* x = slot(map, p, db);
#pragma unroll
          for (int J = 0; J < 4; ++J) {
            const float4 v = x[J * 64];
            s[4 * J] += v.x * f[p]; s[4 * J + 1] += v.y * f[p];
            s[4 * J + 2] += v.z * f[p]; s[4 * J + 3] += v.w * f[p];
          }
        }
        o[db] = s;
      }
    }
    const float inv = live ? 1.0f / l : 0.0f;
    const float lam = live ? a.lambda[hd] : 0.0f;
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      if (S > 1 && db % S != part) continue;
      if (PACK && !live) o[db] = zero16();  // (it saw no key: NaN)
      o[db] *= inv;
      if (map == 1) put(slot(1, part, db), o[db]);
    }
    lds_barrier();
    if (map == 0) {
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        if (S > 1 && db % S != part) continue;
        const float4* x = slot(1, part, db);
#pragma unroll
        for (int J = 0; J < 4; ++J) {
          const float4 v = x[J * 64];
          o[db][4 * J] -= lam * v.x; o[db][4 * J + 1] -= lam * v.y;
          o[db][4 * J + 2] -= lam * v.z; o[db][4 * J + 3] -= lam * v.w;
        }
      }
    }
  }
  if (qw >= tr.rows || (PACK && !(own >> lq & 1))) return true;
  bf16_t* out = map == 0 ? a.out : a.out2;
  if (out != nullptr) {
    bf16_t* Og = out + (tok0 + qw) * a.M + (long)hd * D;
#pragma unroll
    for (int db = 0; db < DB; ++db)
      if (S == 1 || db % S == part) store_cols(Og + 32 * db, o[db], h2, 1.0f);
  }
  if (h2 == 0 && part == 0 && a.lse != nullptr)
    a.lse[((long)map * a.heads + hd) * a.T + tok0 + qw] = live ? (m + log2f(l)) * kLn2 : 0.0f;
  return true;
}

// run(rows, own) for a tile of short sequences, or (it gives false) for each of them
template <class F>
__device__ __forceinline__ void run_short(const DiffArgs& a, int sq, F&& run) {
  const TileRows tr = tile_rows(a, sq);
  TileRows part = tr;
  unsigned own = ~0u;
  for (int r = 0;; r += a.sub) {
    if (run(part, own) && own == ~0u) return;
    if (own == ~0u) r = -a.sub;  // (from here on one by one)
    if (r + a.sub >= tr.rows) return;
    own = (~0u >> (32 - a.sub)) << (r + a.sub);
    part.valid = tr.valid & own;
    part.end = 32 - __clz((int)part.valid);
    wait_vm<0>();
    lds_barrier();
  }
}

template <int D, bool CAUSAL, int NW, int S, int ONE>
__global__ __launch_bounds__(64 * NW, S == 1 ? 4 : 2) void diff_fwd_kernel(DiffArgs a) {
  using Tile = FwdTile<NW, S>;
  // K slots, then V slots; at the end the waves' outputs (float)
  __shared__ __attribute__((aligned(1024))) char lds[(ONE ? 2 : 4) * TileDma<D, Tile::KT, NW>::TB];
  __shared__ float2 stat[S > 1 ? NW * 64 : 1];  // and their references and sums
  int qt, hd, sq;
  diff_decode(a, a.heads, CAUSAL, Tile::QB, qt, hd, sq);
  auto run = [&](const TileRows& tr, unsigned own) __attribute__((always_inline)) {
    return diff_fwd_tile<D, CAUSAL, NW, S, ONE>(a, lds, stat, tr, own, qt, hd, sq);
  };
  if constexpr (ONE == 2) run_short(a, sq, run);
  else run(TileRows{0u, seq_end(a, sq), a.N}, ~0u);
}

// S waves (the parts of a group) that hold sums of the same NB 32-row blocks: each hands
// the others theirs, lane by lane, and adds up its own, those with index = part (mod S),
// in the order of the parts. Every wave's reads of LDS are done. (One part after the
// other handing all to the first took 3.3 us of a dQ block of four waves at D = 128.)
template <int S, int NB>
__device__ __forceinline__ void add_parts(floatx16 (&v)[NB], char* lds, int grp, int part, int lane) {
  auto slot = [&](int p, int b) {
    return reinterpret_cast<float4*>(lds) + (long)((grp * S + p) * NB + b) * 256 + lane;
  };
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    if (b % S == part) continue;
    float4* x = slot(part, b);
#pragma unroll
    for (int J = 0; J < 4; ++J)
      x[J * 64] = make_float4(v[b][4 * J], v[b][4 * J + 1], v[b][4 * J + 2], v[b][4 * J + 3]);
  }
  lds_barrier();
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    if (b % S != part) continue;
    floatx16 s = zero16();
#pragma unroll
    for (int p = 0; p < S; ++p) {
      if (p == part) {
        s += v[b];
        continue;
      }
      const float4* x = slot(p, b);
#pragma unroll
      for (int J = 0; J < 4; ++J) {
        const float4 e = x[J * 64];
        s[4 * J] += e.x; s[4 * J + 1] += e.y; s[4 * J + 2] += e.z; s[4 * J + 3] += e.w;
      }
    }
    v[b] = s;
  }
}

// Steps of QT queries that see key tile kt of KB rows, and steps of KT keys that query
// tile qt of QB rows sees. A (tile, head, sequence) is cut into units of `a.unit` steps (key
// tiles; the group's heads one after the other) or `a.qunit` (query tiles); 0: uncut.
template <bool CAUSAL, int KB, int QT>
__host__ __device__ __forceinline__ int key_steps(int N, int kt) {
  return (N - (CAUSAL ? kt * KB : 0) + QT - 1) / QT;
}
template <bool CAUSAL, int QB, int KT>
__host__ __device__ __forceinline__ int query_steps(int N, int qt) {
  return ((CAUSAL && QB * (qt + 1) < N ? QB * (qt + 1) : N) + KT - 1) / KT;
}

// Of nt tiles of steps(tile) steps each in units of `unit`: unit u's tile, the tile's units,
// and its place among them; or (u < 0) the units before tile kt. A lane a tile, as a loop
// over the tiles with a division each took microseconds.
struct UnitAt {
  int kt, units, chunk;
};
template <class F>
__device__ __forceinline__ UnitAt find_unit(int nt, int unit, F&& steps, int u, int kt) {
  const int lane = threadIdx.x & 63;
  int before = 0;
  for (int k0 = 0;; k0 += 64) {
    const int k = k0 + lane;
    const int n = k < nt ? (steps(k) + unit - 1) / unit : 0;
    int upto = n;  // the units of tiles k0 .. k
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int v = __shfl_up(upto, d);
      if (lane >= d) upto += v;
    }
    const unsigned long long here = __ballot(u >= 0 ? before + upto > u : k == kt);
    if (here != 0) {
      const int f = __ffsll(here) - 1;
      const int units = __builtin_amdgcn_readlane(n, f);
      const int first = before + __builtin_amdgcn_readlane(upto, f) - units;
      return {k0 + f, units, u >= 0 ? u - first : first};
    }
    before += __builtin_amdgcn_readlane(upto, 63);
  }
}

// dQ, and d1 and d2: NW waves over 32-key tiles, both maps in a wave (they share dP). S
// waves share 32 queries, each with every S-th key tile, and add up at the end: blocks
// of few queries, for launches that leave CUs idle.
//
// 24 matrix products and 32 exponentials a lane for 32 x 32 pairs; the accumulators of dP
// start at -d1, so that a map's factor is there without a subtraction. Every LDS read is a
// group of products ahead of its use, which takes 4 % off (935 us of a kernel trace at 4 x 4096 tokens, 32 heads
// of 128, causal: 882 TFLOP/s of its 6 D flops a pair). The matrix pipes are busy for 43 % of
// the cycles, LDS for 57 %, at 1.9 GHz. Running dP and the first map's scores a tile ahead,
// beside the elementwise work, measured 2 % slower (18 % with heads of 64).
template <int D, bool CAUSAL, int NW, int S, int ONE>
__device__ __forceinline__ bool diff_dq_tile(const DiffArgs& a, char* lds, const TileRows& tr,
                                             unsigned own, int qt, int hd, int sq, int units, int chunk) {
  constexpr int SL = ONE ? 1 : 2;  // slots: ONE for sequences of one tile (1) or less (2)
  constexpr bool PACK = ONE == 2;
  constexpr int KS = D / 16, DB = D / 32, G = NW / S, QB = 32 * G, KT = 32 * S;
  using Dma = TileDma<D, KT, NW>;
  using DmaG = TileDma<D, QB, NW>;
  constexpr int TB = Dma::TB, VB = SL * TB, GB = 2 * VB;  // K slots, V slots, the dO rows
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6),
            h2 = lane >> 5, lq = lane & 31;
  const int grp = w % G, part = w / G;
  const int end = tr.end;
  const long tok0 = (long)sq * a.N, ld = a.W;
  const int q0 = qt * QB, qw = q0 + 32 * grp + lq;
  const unsigned seen = PACK ? partners<CAUSAL, false>(a, tr.valid, lq) : 0u;
  const bool live = PACK ? seen != 0u : qw < end;
  const long srow = (long)hd * a.T + tok0 + qw, smap = (long)a.heads * a.T;
  const float lam = a.lambda[hd];

  floatx16 dq[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) dq[db] = zero16();
  float d1 = 0.0f, d2 = 0.0f;
  if (q0 < end) {  // (else padding only)
    const int kh = hd / (a.heads / a.kv);
    const bf16_t* Qg = a.qkv + tok0 * ld + (long)hd * D;
    const bf16_t* Kg = a.qkv + tok0 * ld + a.M + (long)kh * D;
    const bf16_t* Vg = Kg + (long)a.kv * D;
    const long go = tok0 * a.M + (long)hd * D;
    const int kend = CAUSAL ? min(end, q0 + QB) : end;
    const int nk0 = (kend + KT - 1) / KT, t0 = chunk * a.qunit;
    const int nk = a.qunit > 0 ? min(nk0, t0 + a.qunit) : nk0;
    const long kstep = KT * ld;
    const Dma dma(lds_base(lds), w, lane, ld);
    bf16x8 qf[KS];
    {
      bf16x8 gv[KS], ov[KS], pv[KS];
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const long c = go + (long)qw * a.M + 16 * ks + 8 * h2;
        gv[ks] = live ? *reinterpret_cast<const bf16x8*>(a.d_o + c) : zero8();
        ov[ks] = live ? *reinterpret_cast<const bf16x8*>(a.o + c) : zero8();
        pv[ks] = live ? *reinterpret_cast<const bf16x8*>(a.o2 + c) : zero8();
        qf[ks] = live ? *reinterpret_cast<const bf16x8*>(Qg + qw * ld + 16 * ks + 8 * h2) : zero8();
      }
      // (after the rows above, which would else wait for the tiles too: loads return in order)
      DmaG(lds_base(lds), w, lane, a.M).load(a.d_o + go + (long)q0 * a.M, end - q0, GB);
      Kg += t0 * kstep;
      Vg += t0 * kstep;
      dma.load(Kg, kend - KT * t0, 0);
      dma.load(Vg, kend - KT * t0, VB);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int t = 0; t < 8; ++t) {
          d1 += (float)gv[ks][t] * (float)ov[ks][t];
          d2 += (float)gv[ks][t] * (float)pv[ks][t];
        }
    }
    d1 = pair_sum(d1);
    d2 = pair_sum(d2);
    d1 += lam * d2;
    const float l1 = live ? a.lse[srow] * kLog2e : 0.0f, l2 = live ? a.lse[srow + smap] * kLog2e : 0.0f;
    int rbase = row_base<D>(lq, h2), tb0 = tr_base<D>(lane, 0), tb1 = tr_base<D>(lane, 1);
    // read groups, each read one ahead of its products: 0 .. KS - 1, the K, V and dO rows
    // at k step i; then DB groups of K transposed, 16 keys by 64 columns each
    constexpr int NG = KS + DB, RS = 2;
    bf16x8 fr[RS][3];
    auto read_group = [&](const char* tk, const char* tv, int i) __attribute__((always_inline)) {
      if (i < KS) {
        fr[i % RS][0] = frag_row_x<D>(tk, rbase, 0, i);
        fr[i % RS][1] = frag_row_x<D>(tv, rbase, 0, i);
        fr[i % RS][2] = frag_row_x<D>(lds + GB, rbase, 32 * grp, i);
      } else if (i < NG) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
          fr[i % RS][u] = frag_tr_x<D>(tk, tb0, tb1, 16 * ((i - KS) / (DB / 2)),
                                      32 * (2 * ((i - KS) % (DB / 2)) + u));
      }
    };
    auto step = [&](const int t, auto stc) __attribute__((always_inline)) {
      constexpr int st = decltype(stc)::value;
      opaque(rbase, tb0, tb1);
      wait_vm<0>();   // K(t) and V(t): loaded a step ago
      lds_barrier();  // and every wave's reads of the slots refilled now are done
      const char* tk = lds + st * TB + part * (32 * 2 * D);
      const char* tv = tk + VB;
      if constexpr (!ONE) {
        Kg += kstep;
        Vg += kstep;
        dma.load(Kg, kend - KT * (t + 1), (st ^ 1) * TB);
        dma.load(Vg, kend - KT * (t + 1), VB + (st ^ 1) * TB);
      }
      const int kb0 = KT * t + 32 * part;
      // (causal: nothing for a wave whose queries all precede these keys)
      if (kb0 >= kend || (CAUSAL && kb0 > q0 + 32 * grp + 31)) return;
      floatx16 s[2], dp;
#pragma unroll
      for (int r = 0; r < 16; ++r) dp[r] = -d1;  // dP - d1
      read_group(tk, tv, 0);
#pragma unroll
      for (int i = 0; i < KS; ++i) {
        read_group(tk, tv, i + 1);
        __builtin_amdgcn_sched_barrier(0);
        floatx16& x = s[i >= KS / 2];
        x = mfma(fr[i % RS][0], qf[i], i % (KS / 2) == 0 ? zero16() : x);
        dp = mfma(fr[i % RS][1], fr[i % RS][2], dp);
        __builtin_amdgcn_sched_barrier(0);
      }
      if (!PACK && (kb0 + 32 > end || (CAUSAL && kb0 + 31 > q0 + 32 * grp))) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int key = kb0 + 8 * (r >> 2) + 4 * h2 + (r & 3);
          if (key >= end || (CAUSAL && key > qw)) s[0][r] = s[1][r] = -INFINITY;
        }
      }
      unsigned pw[2][8];  // dS^T of each map in this lane, rounded to bf16 for the product
      const float dd = d1 - d2;
#pragma unroll
      for (int r = 0; r < 16; r += 2) {
        float e[2], f[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          e[j] = exp2_fast(fmaf(s[0][r + j], a.c2, -l1)) * dp[r + j];
          f[j] = exp2_fast(fmaf(s[1][r + j], a.c2, -l2)) * (dp[r + j] + dd);
          if constexpr (PACK) {
            const int k = 8 * (r >> 2) + (r & 3) + j;
            e[j] = where_bit(seen >> 4 * h2, k, e[j], 0.0f);
            f[j] = where_bit(seen >> 4 * h2, k, f[j], 0.0f);
          }
        }
        pw[0][r >> 1] = pack_bf16x2(e[0], e[1]);
        pw[1][r >> 1] = pack_bf16x2(f[0], f[1]);  // (times -lambda at the end)
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int j = 0; j < DB; ++j) {
        read_group(tk, tv, KS + j + 1);
        __builtin_amdgcn_sched_barrier(0);
        const int g = j / (DB / 2);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int db = 2 * (j % (DB / 2)) + u;
          const unsigned* p = pw[db >= DB / 2 ? 1 : 0] + 4 * g;
          dq[db] = mfma(fr[(KS + j) % RS][u],
                        __builtin_bit_cast(bf16x8, u32x4{p[0], p[1], p[2], p[3]}), dq[db]);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    if constexpr (ONE) {
      if constexpr (PACK) {
        wait_vm<0>();
        lds_barrier();
        if (tr.valid & (tr.valid + 1)) {
          clear_rows<D, 64 * NW>(lds, tr.valid, tid);
          lds_barrier();
        }
        if (own == ~0u && not_finite<D>(lds, lane)) return false;
      }
      step(0, Stage<0>{});
    } else {
      for (int t = t0; t < nk; t += 2) {
        step(t, Stage<0>{});
        if (t + 1 < nk) step(t + 1, Stage<1>{});
      }
    }
    wait_vm<0>();           // (the loads past the last tile write zeros)
    if constexpr (S > 1) {
      lds_barrier();
      add_parts<S>(dq, lds, grp, part, lane);
    }
  }
  const bool lead = part == 0 && h2 == 0;
  if (units > 1) {
    if (q0 < end) {
      float4* x = reinterpret_cast<float4*>(a.qpart) +
                  ((long)(blockIdx.x % (a.heads * a.nseq)) * a.qunits + blockIdx.x / (a.heads * a.nseq)) *
                      (4 * DB * 64 * G) + 64 * grp + lane;
#pragma unroll
      for (int i = 0; i < 4 * DB; ++i) {
        const floatx16& v = dq[i / 4];
        const int r = 4 * (i % 4);
        if (i / 4 % S == part) x[i * 64 * G] = make_float4(v[r], v[r + 1], v[r + 2], v[r + 3]);
      }
    }
    if (chunk > 0) return true;  // (the first unit writes the rows' d1 and d2)
  }
  if (qw >= tr.rows || (PACK && !(own >> lq & 1))) return true;
  if (lead) {
    a.delta[srow] = d1;
    a.delta[srow + smap] = d2;
  }
  if (units > 1) return true;
  bf16_t* dst = a.d_qkv + (tok0 + qw) * ld + (long)hd * D;
#pragma unroll
  for (int db = 0; db < DB; ++db) {
    if (db % S != part) continue;
    if (!live) dq[db] = zero16();
    store_cols(dst + 32 * db, dq[db], h2, db >= DB / 2 ? -lam * a.rs : a.rs);
  }
  return true;
}

template <int D, bool CAUSAL, int NW, int S, int ONE>
__global__ __launch_bounds__(64 * NW, 2) void diff_dq_kernel(DiffArgs a) {
  constexpr int QB = 32 * NW / S, KT = 32 * S;
  __shared__ __attribute__((aligned(1024))) char lds[(ONE ? 2 : 4) * TileDma<D, KT, NW>::TB + QB * D * 2];
  int qt, hd, sq, units = 1, chunk = 0;
  if (a.qunit > 0) {
    const int per = a.heads * a.nseq, rest = (int)(blockIdx.x % per);
    const UnitAt at = find_unit((a.N + QB - 1) / QB, a.qunit,
                                [&](int k) { return query_steps<CAUSAL, QB, KT>(a.N, k); },
                                blockIdx.x / per, 0);
    qt = at.kt;
    units = at.units;
    chunk = at.chunk;
    hd = rest % a.heads;
    sq = rest / a.heads;
  } else {
    diff_decode(a, a.heads, CAUSAL, QB, qt, hd, sq);
  }
  auto run = [&](const TileRows& tr, unsigned own) __attribute__((always_inline)) {
    return diff_dq_tile<D, CAUSAL, NW, S, ONE>(a, lds, tr, own, qt, hd, sq, units, chunk);
  };
  if constexpr (ONE == 2) run_short(a, sq, run);
  else run(TileRows{0u, seq_end(a, sq), a.N}, ~0u);
}

// dlambda_h = -sum of d2 over all rows, by a block, of one wave where sequences are short: of
// very many this sum outlasts the other blocks (2^20 of one token, 1 head of 64: dQ 230 us, dK
// and dV with the sum 1098; 16384, 8 heads: 29 and 35)
__device__ __forceinline__ void sum_d_lambda(const DiffArgs& a, int hd, float* part) {
  const float* d2 = a.delta + ((long)a.heads + hd) * a.T;
  float s8[8] = {};
  const int n = blockDim.x;
  int t = threadIdx.x;
  for (; t + 7 * n < a.T; t += 8 * n) {  // (eight loads in flight)
#pragma unroll
    for (int i = 0; i < 8; ++i) s8[i] += d2[t + i * n];
  }
  for (; t < a.T; t += n) s8[0] += d2[t];
  float s = ((s8[0] + s8[1]) + (s8[2] + s8[3])) + ((s8[4] + s8[5]) + (s8[6] + s8[7]));
#pragma unroll
  for (int x = 32; x > 0; x >>= 1) s += __shfl_xor(s, x);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    s = 0.0f;
    for (int i = 0; i < (int)blockDim.x / 64; ++i) s += part[i];
    a.d_lambda[hd] = (a.accumulate ? a.d_lambda[hd] : 0.0f) - s;
  }
}

// dK and dV: waves of 32 keys over the 32-query tiles of every query head of the group, or
// over a unit of them, whose sums diff_join_kernel adds. With S > 1, S of the NW waves
// share 32 keys, each with every S-th query tile, and add up at the end. The last `heads`
// blocks sum dlambda.
//
// 32 matrix products and 32 exponentials a lane for 32 x 32 pairs; both accumulators (128
// registers at D = 128) and the K fragments leave none to read ahead of the products: with
// read groups as in dQ 1570 us, the plain order 1340 (4 x 4096 tokens, 32 heads of 128,
// causal: 820 TFLOP/s of its 8 D flops a pair; the matrix pipes busy for 38 % of the cycles,
// LDS for 68 %, at 2.0 GHz).
template <int D, bool CAUSAL, int NW, int S, int ONE>
__global__ __launch_bounds__(64 * NW, ONE == 2 && D == 128 ? 1 : 2) void diff_dkdv_kernel(DiffArgs a) {
  constexpr int SL = ONE ? 1 : 2;  // slots: ONE for sequences of one tile (1) or less (2)
  constexpr bool PACK = ONE == 2;
  constexpr int KS = D / 16, DB = D / 32, G = NW / S, KB = 32 * G, QT = 32 * S;
  using Dma = TileDma<D, QT, NW>;
  using DmaV = TileDma<D, KB, NW>;
  constexpr int TQ = Dma::TB;          // one query tile
  constexpr int VT = 2 * SL * TQ;      // slots of Q and dO, then the block's V rows,
  constexpr int ST = VT + KB * D * 2;  // then slots of 32 S x 4 row statistics
  constexpr int SB = 512 * S;
  __shared__ __attribute__((aligned(1024))) char lds[ST + SL * SB];
  static_assert(S == 1 || NW * DB * 4096 <= ST + SL * SB, "the parts' sums fit");
  const int per = a.kv * a.nseq, nblocks = (int)gridDim.x - a.heads;
  if ((int)blockIdx.x >= nblocks) {
    sum_d_lambda(a, blockIdx.x - nblocks, reinterpret_cast<float*>(lds));
    return;
  }
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6),
            h2 = lane >> 5, lq = lane & 31;
  const int grp = w % G, part = w / G;
  const int rest = (int)(blockIdx.x % per), kh = rest % a.kv, sq = rest / a.kv;
  const int group = a.heads / a.kv;
  int kt = (int)(blockIdx.x / per), units = 1, chunk = 0;
  if (a.unit > 0) {
    const UnitAt at = find_unit((a.N + KB - 1) / KB, a.unit,
                                [&](int k) { return group * key_steps<CAUSAL, KB, QT>(a.N, k); }, kt, 0);
    kt = at.kt;
    units = at.units;
    chunk = at.chunk;
  }
  TileRows tr = PACK ? tile_rows(a, sq) : TileRows{0u, seq_end(a, sq), a.N};
  const unsigned all = tr.valid;
  unsigned own = ~0u;  // (as in run_short, which as a function cost this kernel its registers)
one:
  const int end = tr.end;
  const long tok0 = (long)sq * a.N, ld = a.W;
  const int k0 = kt * KB, kw = k0 + 32 * grp + lq;
  const unsigned seen = PACK ? partners<CAUSAL, true>(a, tr.valid, lq) : 0u;
  const bool live = PACK ? seen != 0u : kw < end;
  const long kcol = a.M + (long)kh * D, vcol = kcol + (long)a.kv * D;
  floatx16 dv[DB], dk[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) {
    dv[db] = zero16();
    dk[db] = zero16();
  }
  if (k0 < end) {
    const bf16_t* rows = a.qkv + tok0 * ld;
    const Dma dma(lds_base(lds), w, lane, ld), dmag(lds_base(lds), w, lane, a.M);
    DmaV(lds_base(lds), w, lane, ld).load(rows + vcol + (long)k0 * ld, end - k0, VT);
    bf16x8 kf[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
      kf[ks] = live ? *reinterpret_cast<const bf16x8*>(rows + kcol + kw * ld + 16 * ks + 8 * h2) : zero8();
    // query steps of QT: causal keys k0.. are seen by queries >= k0 only
    const int qs0 = CAUSAL ? k0 : 0;
    const int steps = key_steps<CAUSAL, KB, QT>(a.N, kt), valid = (end - qs0 + QT - 1) / QT;
    const int lo = chunk * a.unit, hi = a.unit > 0 ? min(lo + a.unit, group * steps) : group * steps;
    int rbase = row_base<D>(lq, h2), tb0 = tr_base<D>(lane, 0), tb1 = tr_base<D>(lane, 1);

    bool more_heads = false;
    for (int gh = lo / steps; gh * steps < hi; ++gh) {
      const int it0 = max(lo - gh * steps, 0), it1 = min(hi - gh * steps, valid);
      if (it0 >= it1) continue;
      const int hd = kh * group + gh;
      // |lambda| goes into the second map's exponent (lambda = 0: -inf, and P_2 is 0), its sign
      // into the sums
      const float lam = a.lambda[hd], sgn = lam < 0.0f ? -1.0f : 1.0f, llam = log2f(fabsf(lam));
      const int qf0 = qs0 + QT * it0;
      const bf16_t* Qt = rows + (long)hd * D + qf0 * ld;
      const bf16_t* Gt = a.d_o + (tok0 + qf0) * a.M + (long)hd * D;
      // the statistics of a step's rows, two a thread: lse of map 1, of map 2 less log2 |lambda|
      // (base 2); -d1, +-(d2 - d1)
      float2 rstat = make_float2(0.0f, 0.0f);
      const bool isd = (tid & 32) != 0;
      const int srow = 32 * (tid >> 6) + lq;
      const float* sp = (isd ? a.delta : a.lse) + (long)hd * a.T + tok0 + srow;
      const long smap = (long)a.heads * a.T;
      auto load_stat = [&](int qb) __attribute__((always_inline)) {
        if (tid < 64 * S) {
          const bool in = qb + srow < end;
          const float x = in ? sp[qb] : 0.0f, y = in ? sp[qb + smap] : 0.0f;
          rstat = isd ? make_float2(-x, sgn * (y - x)) : make_float2(x * kLog2e, y * kLog2e - llam);
        }
      };
      auto store_stat = [&](int slot) __attribute__((always_inline)) {
        if (tid < 64 * S) {
          float* s = reinterpret_cast<float*>(lds + ST + SB * slot) + 128 * (tid >> 6) + (isd ? 64 : 0) + lq;
          s[0] = rstat.x;
          s[32] = rstat.y;
        }
      };
      if (more_heads) {  // (the last head's loads have landed and its reads are done)
        wait_vm<0>();
        lds_barrier();
      }
      more_heads = true;
      dma.load(Qt, end - qf0, 0);
      dmag.load(Gt, end - qf0, TQ);
      load_stat(qf0);
      store_stat(0);

      constexpr int H = KS / 2;
      auto step = [&](const int it, auto stc) __attribute__((always_inline)) {
        constexpr int st = decltype(stc)::value;
        opaque(rbase, tb0, tb1);
        const int qt0 = qs0 + QT * it, qb = qt0 + 32 * part;
        wait_vm<0>();   // this tile's loads
        lds_barrier();  // and every wave's reads of the other slot are done
        const char* tq = lds + st * 2 * TQ + part * (32 * 2 * D);
        const float* stat = reinterpret_cast<const float*>(lds + ST + SB * st) + 128 * part + 4 * h2;
        if constexpr (!ONE) {
          Qt += QT * ld;
          Gt += QT * a.M;
          const int more = it + 1 < it1 ? end - qt0 - QT : 0;
          dma.load(Qt, more, (st ^ 1) * 2 * TQ);
          dmag.load(Gt, more, (st ^ 1) * 2 * TQ + TQ);
          if (it + 1 < it1) load_stat(qt0 + QT);
        }
        // (a condition less in the loop of causal blocks that share nothing: it cost a spill of
        // a K fragment, whose reload waits for the loads under way, 8 % of the time)
        if (((S == 1 && CAUSAL) || qb < end) && (!CAUSAL || qb + 31 >= k0 + 32 * grp)) {
          const bool edge = qb + 32 > end || (CAUSAL && k0 + 32 * grp + 31 > qb);
          auto mask = [&](floatx16& s) __attribute__((always_inline)) {
            if (!PACK && edge) {
#pragma unroll
              for (int r = 0; r < 16; ++r) {
                const int q = qb + 8 * (r >> 2) + 4 * h2 + (r & 3);
                if (q >= end || (CAUSAL && kw > q)) s[r] = -INFINITY;
              }
            }
          };
          auto row4 = [&](int k, int J) __attribute__((always_inline)) { return *reinterpret_cast<const float4*>(stat + 32 * k + 8 * J); };
          floatx16 s1, s2, dp;
          unsigned pp[8], pd[2][8];  // P_1 - lambda P_2 and dS of each map, bf16 pairs
          const char* tg = tq + TQ;
#pragma unroll
          for (int J = 0; J < 4; ++J) {  // dP - d1
            const float4 v = row4(2, J);
            dp[4 * J] = v.x; dp[4 * J + 1] = v.y; dp[4 * J + 2] = v.z; dp[4 * J + 3] = v.w;
          }
#pragma unroll
          for (int i = 0; i < H; ++i) {
            s1 = mfma(frag_row_x<D>(tq, rbase, 0, i), kf[i], i == 0 ? zero16() : s1);
            s2 = mfma(frag_row_x<D>(tq, rbase, 0, H + i), kf[H + i], i == 0 ? zero16() : s2);
          }
#pragma unroll
          for (int i = 0; i < KS; ++i)
            dp = mfma(frag_row_x<D>(tg, rbase, 0, i), frag_row_x<D>(lds + VT, rbase, 32 * grp, i), dp);
          mask(s1);
          mask(s2);
#pragma unroll
          for (int J = 0; J < 4; ++J) {
            const float4 t = row4(0, J), v = row4(1, J), u = row4(3, J);
            const float l1[4] = {t.x, t.y, t.z, t.w}, l2[4] = {v.x, v.y, v.z, v.w}, dd[4] = {u.x, u.y, u.z, u.w};
            float p[4], e[4], f[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const int r = 4 * J + j;
              const float p1 = exp2_fast(fmaf(s1[r], a.c2, -l1[j]));
              const float p2 = exp2_fast(fmaf(s2[r], a.c2, -l2[j]));
              p[j] = fmaf(-sgn, p2, p1);
              e[j] = p1 * dp[r];
              f[j] = p2 * fmaf(-sgn, dp[r], dd[j]);
              if constexpr (PACK) {
                p[j] = where_bit(seen >> 4 * h2, 8 * J + j, p[j], 0.0f);
                e[j] = where_bit(seen >> 4 * h2, 8 * J + j, e[j], 0.0f);
                f[j] = where_bit(seen >> 4 * h2, 8 * J + j, f[j], 0.0f);
              }
            }
#pragma unroll
            for (int j = 0; j < 4; j += 2) {
              pp[2 * J + j / 2] = pack_bf16x2(p[j], p[j + 1]);
              pd[0][2 * J + j / 2] = pack_bf16x2(e[j], e[j + 1]);
              pd[1][2 * J + j / 2] = pack_bf16x2(f[j], f[j + 1]);
            }
          }
#pragma unroll
          for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int db = 0; db < DB; ++db) {
              const unsigned* d = pd[db >= DB / 2 ? 1 : 0] + 4 * g;
              dv[db] = mfma(frag_tr_x<D>(tg, tb0, tb1, 16 * g, 32 * db),
                            __builtin_bit_cast(bf16x8, u32x4{pp[4 * g], pp[4 * g + 1], pp[4 * g + 2], pp[4 * g + 3]}), dv[db]);
              dk[db] = mfma(frag_tr_x<D>(tq, tb0, tb1, 16 * g, 32 * db),
                            __builtin_bit_cast(bf16x8, u32x4{d[0], d[1], d[2], d[3]}), dk[db]);
            }
        }
        if (!ONE && it + 1 < it1) store_stat(st ^ 1);
      };
      if constexpr (ONE) {
        if constexpr (PACK) {
          wait_vm<0>();
          lds_barrier();
          if (tr.valid & (tr.valid + 1)) {
            clear_rows<D, 64 * NW>(lds, tr.valid, tid);
            clear_rows<D, 64 * NW>(lds + TQ, tr.valid, tid);
            lds_barrier();
          }
          if (own == ~0u && (not_finite<D>(lds, lane) || not_finite<D>(lds + TQ, lane)))
          {
            own = ~0u >> (32 - a.sub);
            tr.valid = all & own;
            tr.end = 32 - __clz((int)tr.valid);
            lds_barrier();
            goto one;
          }
        }
        step(it0, Stage<0>{});
      } else {
        for (int it = it0; it < it1; it += 2) {
          step(it, Stage<0>{});
          if (it + 1 < it1) step(it + 1, Stage<1>{});
        }
      }
    }
  }
  wait_vm<0>();           // (the loads past the last tile write zeros)
  if constexpr (S > 1) {
    lds_barrier();
    add_parts<S>(dk, lds, grp, part, lane);
    lds_barrier();
    add_parts<S>(dv, lds, grp, part, lane);
  }
  if (units > 1) {
    if (!PACK && k0 >= end) return;
    float4* x = reinterpret_cast<float4*>(a.part) +
                ((long)rest * a.units + blockIdx.x / per) * (8 * DB * 64 * G) + 64 * grp + lane;
#pragma unroll
    for (int i = 0; i < 8 * DB; ++i) {
      const floatx16& v = i < 4 * DB ? dk[i / 4] : dv[i / 4 - DB];
      const int r = 4 * (i % 4);
      if (i / 4 % DB % S == part && (!PACK || (own >> lq & 1)))
        x[i * 64 * G] = make_float4(v[r], v[r + 1], v[r + 2], v[r + 3]);
    }
  } else if (kw < tr.rows && (!PACK || (own >> lq & 1))) {  // (rows past the end: their accumulators hold only masked zeros)
    bf16_t* dst = a.d_qkv + (tok0 + kw) * ld;
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      if (db % S != part) continue;
      if (!live) dk[db] = dv[db] = zero16();
      store_cols(dst + kcol + 32 * db, dk[db], h2, a.rs);
      store_cols(dst + vcol + 32 * db, dv[db], h2, 1.0f);
    }
  }
  if constexpr (PACK) {
    if (own == ~0u) return;
    own <<= a.sub;
    if ((own & (~0u >> (32 - tr.rows))) == 0u) return;
    tr.valid = all & own;
    tr.end = 32 - __clz((int)tr.valid);
    wait_vm<0>();
    lds_barrier();
    goto one;
  }
}

// dK and dV of key tiles that were cut into units, their sums added in unit order: a block
// a key tile of 32 G and 32 columns of K or V, with the lanes as they were. Blocks past
// a.kblocks: dQ of query tiles that were, in the blocks that go with these of dK and dV.
template <int D, bool CAUSAL, int G, int S>
__global__ __launch_bounds__(64 * G) void diff_join_kernel(DiffArgs a) {
  constexpr int DB = D / 32, KB = 32 * G, QT = 32 * S;
  constexpr int GQ = S == 4 ? 1 : 2, SQ = S == 4 ? 4 : 2;
  const bool q = (int)blockIdx.x >= a.kblocks;
  const int b = (int)blockIdx.x - (q ? a.kblocks : 0), cols = q ? DB : 2 * DB, g = q ? GQ : G;
  const int heads = q ? a.heads : a.kv, per = heads * a.nseq, tid = threadIdx.x, lane = tid & 63;
  if (tid >= 64 * g) return;
  const int rest = b % per, hd = rest % heads, sq = rest / heads;
  const int u = b / per, col = u % cols, tile = u / cols;
  const int group = a.heads / a.kv, nt = (a.N + 32 * g - 1) / (32 * g);
  const UnitAt at =
      q ? find_unit(nt, a.qunit, [&](int k) { return query_steps<CAUSAL, 32 * GQ, 32 * SQ>(a.N, k); }, -1, tile)
        : find_unit(nt, a.unit, [&](int k) { return group * key_steps<CAUSAL, KB, QT>(a.N, k); }, -1, tile);
  if (at.units == 1) return;
  const int rw = tile * 32 * g + 32 * (tid >> 6) + (lane & 31);
  const TileRows tr = G * S == 1 ? tile_rows(a, sq) : TileRows{0u, seq_end(a, sq), a.N};
  floatx16 s = zero16();
  if (G * S == 1 ? tr.valid >> rw & 1 : rw < tr.end) {
    const int U = 4 * cols * 64 * g;  // float4s of a unit
    const float4* x = reinterpret_cast<const float4*>(q ? a.qpart : a.part) +
                      ((long)rest * (q ? a.qunits : a.units) + at.chunk) * U + 4 * col * 64 * g + tid;
    for (int n = 0; n < at.units; ++n, x += U) {
#pragma unroll
      for (int J = 0; J < 4; ++J) {
        const float4 v = x[J * 64 * g];
        s[4 * J] += v.x; s[4 * J + 1] += v.y; s[4 * J + 2] += v.z; s[4 * J + 3] += v.w;
      }
    }
  }
  if (rw >= tr.rows) return;
  bf16_t* row = a.d_qkv + ((long)sq * a.N + rw) * a.W;
  if (q) {
    store_cols(row + (long)hd * D + 32 * col, s, lane >> 5, col >= DB / 2 ? -a.lambda[hd] * a.rs : a.rs);
  } else {
    const long c = a.M + (long)(col < DB ? hd : a.kv + hd) * D + 32 * (col % DB);
    store_cols(row + c, s, lane >> 5, col < DB ? a.rs : 1.0f);
  }
}

DiffArgs diff_args(const DiffShape& m, int T) {
  DiffArgs a = {};
  a.T = T;
  a.N = m.N;
  a.heads = m.heads;
  a.kv = m.kv;
  a.nseq = T / m.N;
  a.sub = m.N;
  if (m.N <= 16) {
    const int n = 32 / m.N;
    a.N = n * m.N;
    a.nseq = (a.nseq + n - 1) / n;
  }
  a.M = (long)m.heads * m.D;
  a.W = a.M + 2L * m.kv * m.D;
  a.c2 = kLog2e / sqrtf((float)(m.D / 2));
  a.rs = 1.0f / sqrtf((float)(m.D / 2));
  return a;
}

long tiles(const DiffArgs& a, int heads, int rows) {
  return (long)((a.N + rows - 1) / rows) * heads * a.nseq;
}

template <int D, int NW, int S, int ONE = 0>
void launch_fwd(const DiffShape& m, const DiffArgs& a, hipStream_t st) {
  const dim3 g((unsigned)tiles(a, a.heads, FwdTile<NW, S>::QB)), b(64 * NW);
  if (m.causal) hipLaunchKernelGGL((diff_fwd_kernel<D, true, NW, S, ONE>), g, b, 0, st, a);
  else hipLaunchKernelGGL((diff_fwd_kernel<D, false, NW, S, ONE>), g, b, 0, st, a);
}

// Forward blocks by the launch: 0: 32 queries, 8 waves, four parts of the keys; 1: 32
// queries, 4 waves, two parts; 2: 64 queries, 4 waves; 3: 128 queries, 8 waves; 4: below.
// Few queries leave CUs idle and a block's walk over the keys is the time of the call, so
// its waves share the keys; many are better served by blocks that read K and V less
// often. us of variants 0, 1, 2, 3: 1 sequence of 2048, heads of 128, causal, 4 heads 23,
// 26, 43, 55; 8 heads 30, 28, 44, 55; 16 heads 58, 44, 47, 56; 32 heads 116, 81, 67, 73;
// 4 x 4096, 32 heads 1719, 1648, 904, 885; 8 x 2048, 16 heads, bidirectional 803, 736,
// 424, 413; 50 x 300 -, 155, 78, 90; 32 x 512, 32 heads -, 443, 241, 246. Heads of 64 leave
// room for more blocks of variant 1: 1 x 4485, 8 heads, variant 1 53, 2 86. 4: sequences of
// one tile or less, 32 queries by 2 waves: 407 x 1, 8 heads of 128 5, variant 2 19; 452 x 10,
// 16 heads 22, 38.
int fwd_variant(const DiffShape& m, const DiffArgs& a) {
  const long b32 = tiles(a, a.heads, 32), b128 = tiles(a, a.heads, 128);
  if (m.N <= 32) return 4;
  if (b32 <= 256) return 0;
  if (b32 <= (m.D == 64 ? 2048 : 1024)) return 1;
  return m.N >= 1024 && (b128 >= 1024 || !m.causal) ? 3 : 2;
}
long fwd_blocks(const DiffArgs& a, int v) {
  return tiles(a, a.heads, v == 2 ? 64 : v == 3 ? 128 : 32);
}

// Tiles of a head side by side? Bidirectional ones have equal work and lose nothing by
// it. Causal ones then no longer run longest first over the launch; it pays where they
// are few to a head, or K and V far exceed the 256 MB Infinity Cache. us, not shared and
// shared: bidirectional 8 x 2048, 16 heads of 128 430, 413; 16 x 500, 16 heads of 64 37,
// 31; causal 50 x 300, 16 heads of 128 98, 78; 32 x 512, 32 heads 289, 241; 32 x 2048, 16
// heads (537 MB) 1190, 1031; 4 x 4096, 32 heads (268 MB) 885, 899; 4 x 4096, 24 heads of
// 64 412, 439.
int fwd_shared(const DiffShape& m, const DiffArgs& a) {
  return !m.causal || m.N <= 512 || 4L * a.T * m.kv * m.D >= (400L << 20);
}

template <int D>
void launch_fwd_variant(int v, const DiffShape& m, const DiffArgs& a, hipStream_t st) {
  if (v == 0) launch_fwd<D, 8, 4>(m, a, st);
  else if (v == 1) launch_fwd<D, 4, 2>(m, a, st);
  else if (v == 2) launch_fwd<D, 4, 1>(m, a, st);
  else if (v == 3) launch_fwd<D, 8, 1>(m, a, st);
  else if (m.N > 16) launch_fwd<D, 2, 1, 1>(m, a, st);
  else launch_fwd<D, 2, 1, 2>(m, a, st);
}

template <int D, int NW, int S, int ONE = 0>
void launch_dq(const DiffShape& m, const DiffArgs& a, hipStream_t st) {
  const long n = a.qunit > 0 ? (long)a.qunits * a.heads * a.nseq : tiles(a, a.heads, 32 * NW / S);
  const dim3 g((unsigned)n), b(64 * NW);
  if (m.causal) hipLaunchKernelGGL((diff_dq_kernel<D, true, NW, S, ONE>), g, b, 0, st, a);
  else hipLaunchKernelGGL((diff_dq_kernel<D, false, NW, S, ONE>), g, b, 0, st, a);
}

// A backward of few queries: blocks of 32, whose waves share each other's keys or queries.
// Long sequences have so many steps that larger tiles cut into units read less: us of the
// whole backward with such blocks and without: heads of 128, 1 x 459, 1 head 29, 36 (its
// walk is the time); 2 x 300, 8 heads, causal 26, 28; 3 x 770, 3 heads 42, 53; 1 x 2000, 2 on 1
// 52, 60; 2 x 1024, 4 on 1, causal 47, 46; 1 x 2048, 4 heads, causal 69, 58; 1 x 2859, 2 heads,
// causal 69, 58; 1 x 6000, 1 head, causal 126, 75; heads of 64, 1 x 1000, 8 on 2, causal 32,
// 36; 1 x 1500, 4 heads, causal 29, 32; 1 x 3000, 1 head 35, 38; 1 x 8000, 1 head, causal 74, 65.
bool few_queries(const DiffShape& m, const DiffArgs& a) {
  const long b32 = tiles(a, a.heads, 32);
  return b32 <= 256 && b32 * m.N <= 256 * 1536;
}

// dQ blocks by the launch: 0: one wave of 32 queries (sequences of at most 32); 4: two of
// 64 (at most 64); four waves that share 1: 32 queries, 2: 64, 3: 128. us of the whole
// backward with 1, 2, 3: 2 x 512, 8 heads of 64, causal 34, 36, 42; 1 x 2048, heads of 128,
// causal, 4 heads 71, 75, 100; 16 on 4 heads 176, 139, 158; 32 heads 301, 208, 209; 16 x 500,
// 16 on 8 heads of 64 119, 95, 91; 4 x 4096, 32 heads of 128, causal 3610, 2460, 2270. 700 x
// 16, 4 heads of 64, variants 0, 3: 42, 50.
int dq_variant(const DiffShape& m, const DiffArgs& a) {
  if (m.N <= 32) return 0;
  const long b32 = tiles(a, a.heads, 32);
  return few_queries(m, a) ? 1 : m.N <= 64 ? 4 : b32 <= 2048 ? 2 : 3;
}

template <int D>
void launch_dq_variant(const DiffShape& m, const DiffArgs& a, hipStream_t st) {
  const int v = dq_variant(m, a);
  if (v == 0 && m.N > 16) launch_dq<D, 1, 1, 1>(m, a, st);
  else if (v == 0) launch_dq<D, 1, 1, 2>(m, a, st);
  else if (v == 4) launch_dq<D, 2, 1>(m, a, st);
  else if (v == 1) launch_dq<D, 4, 4>(m, a, st);
  else if (v == 2) launch_dq<D, 4, 2>(m, a, st);
  else launch_dq<D, 4, 1>(m, a, st);
}

// dK and dV by the launch: blocks of 32 G keys and 32 S queries a step. A block's walk over
// the queries (a step is about 1 us for a wave alone on its SIMD) is the time of a small
// call, so its waves share the queries there; large ones are better served by tiles that
// more keys share. Sequences of at most 32 and 64 take blocks of one and two waves. Query
// tiles of 64 and 128 rows of heads of 128 leave a CU one block, so those keep {4, 1}
// earlier and are cut into units instead. us of {1, 4}, {2, 2}, {4, 1}: heads of 64: 2 x 512,
// 8 heads, causal 19, 23, 32; 4 x 1024, 8 heads 59, 53, 78; 16 x 500, 16 heads (8) 95, 86,
// 92; 4 x 4096, 24 heads, causal 1170, 1042, 1012; heads of 128: 1 x 2048, 4 heads, causal
// 72, 79, 74; 8 x 256, 8 heads 38, 28, 35; 20 x 200, 8 heads (4) 78, 68, 61; 1 x 2048, 16
// heads (4), causal 173, 153, 134.
struct KeyTile {
  int G, S;
};
KeyTile key_tile(const DiffShape& m, const DiffArgs& a) {
  if (m.N <= 32) return {1, 1};
  if (few_queries(m, a)) return {1, 4};
  if (m.N <= 64) return {2, 1};
  if (m.D == 64) return tiles(a, a.kv, 128) < 1024 ? KeyTile{2, 2} : KeyTile{4, 1};
  // 128 keys by 32 queries: up to three such steps for each of 512 resident blocks
  const long n = (m.N + 31) / 32, steps = tiles(a, a.heads, 128) * (m.causal ? (n + 1) / 2 : n);
  return steps <= 3 * 512 ? KeyTile{2, 2} : KeyTile{4, 1};
}

// The unit that nt tiles of steps(tile) steps, `per` times over, are cut into: the smallest
// (at least 2) whose blocks run in one round of `slots` (dlambda's, a head each and last in
// the grid of dK and dV, are not counted and may wait for one that ends); 0 (uncut): no such
// unit, or the longest tile is less than the worth of the join longer (about 16 / S steps). A
// round that is not full costs as much as a full one: the whole backward of 2 x 2031 tokens,
// 16 heads on 4 of 128, causal, 512 slots: uncut 457 us; units of 34, 37, 40, 44, 51 steps
// (576, 536, 488, 456, 408 blocks) 221, 203, 184, 188, 197; of 20 (920 blocks, two rounds) 198.
template <class F>
int cut(int nt, long per, long slots, int S, F&& steps, int& units) {
  units = 0;
  if (per == 0 || nt * per > slots) return 0;
  long all = 0;
  int longest = 0;
  for (int i = 0; i < nt; ++i) {
    all += steps(i);
    longest = std::max(longest, steps(i));
  }
  auto count = [&](int unit) {
    int n = 0;
    for (int i = 0; i < nt; ++i) n += (steps(i) + unit - 1) / unit;
    return n;
  };
  int lo = (int)std::max<long>((all * per + slots - 1) / slots, 2), hi = longest;
  if (longest < lo + 16 / S) return 0;
  while (lo < hi) {
    const int mid = lo + (hi - lo) / 2;
    if (count(mid) * per <= slots) hi = mid;
    else lo = mid + 1;
  }
  if (longest < lo + 16 / S) return 0;
  units = count(lo);
  return lo;
}

// Units of dK and dV: a.unit, a.units. Two blocks to a CU, or one where 64 or 128 query rows
// of heads of 128 fill its LDS. The whole backward uncut and cut: 2 x 1024, 4 heads on 1 of
// 128, causal 92, 46 us; 1 x 2000, 2 on 1 of 128 100, 60; 1 x 3000, 1 head of 64 60, 44; 4 x
// 1024, 8 on 2 of 128 249, 98; 2 x 1500, 16 on 2 of 64, causal 253, 82.
void cut_units(const DiffShape& m, DiffArgs& a) {
  const KeyTile k = key_tile(m, a);
  const int group = m.heads / m.kv, KB = 32 * k.G, QT = 32 * k.S;
  a.unit = cut((m.N + KB - 1) / KB, (long)m.kv * a.nseq, m.D == 128 && k.S > 1 ? 256 : 512, k.S,
               [&](int kt) { return group * ((m.N - (m.causal ? KB * kt : 0) + QT - 1) / QT); }, a.units);
}
// And of dQ, in the blocks of its variants 1 and 2 (of 1 and heads of 128 one fills a CU):
// a.qunit, a.qunits. The whole backward uncut and cut: 1 x 2859, 2 heads of 128, causal 92,
// 84 us; 1 x 3000, 1 head of 64 60, 56; 1 x 773, 2 heads of 128 39, 36.
void cut_query_units(const DiffShape& m, DiffArgs& a) {
  const int v = dq_variant(m, a), QB = v == 1 ? 32 : 64, KT = v == 1 ? 128 : 64;
  a.qunit = a.qunits = 0;
  if (v != 1 && v != 2) return;
  a.qunit = cut((m.N + QB - 1) / QB, (long)m.heads * a.nseq, m.D == 128 && v == 1 ? 256 : 512, KT / 32,
                [&](int qt) { return ((m.causal ? std::min(QB * (qt + 1), m.N) : m.N) + KT - 1) / KT; },
                a.qunits);
}
size_t part_bytes(const DiffShape& m, const DiffArgs& a) {
  return align256((size_t)a.units * m.kv * a.nseq * 32 * key_tile(m, a).G * 2 * m.D * sizeof(float));
}

template <int D, int G, int S, int ONE = 0>
hipError_t launch_dkdv(const DiffShape& m, const DiffArgs& a, hipStream_t st) {
  const long n = a.unit > 0 ? (long)a.units * a.kv * a.nseq : tiles(a, a.kv, 32 * G);
  const hipError_t e = traced(FLOWMOE_K_DIFF_BWD_DKDV, st, [&] {
    const dim3 g((unsigned)(n + a.heads)), b(64 * G * S);
    if (m.causal) hipLaunchKernelGGL((diff_dkdv_kernel<D, true, G * S, S, ONE>), g, b, 0, st, a);
    else hipLaunchKernelGGL((diff_dkdv_kernel<D, false, G * S, S, ONE>), g, b, 0, st, a);
  });
  if (e != hipSuccess || (a.unit == 0 && a.qunit == 0)) return e;
  DiffArgs j = a;
  j.kblocks = a.unit > 0 ? (int)(tiles(a, a.kv, 32 * G) * (2 * D / 32)) : 0;
  const long nq = a.qunit > 0 ? tiles(a, a.heads, S == 4 ? 32 : 64) * (D / 32) : 0;
  return traced(FLOWMOE_K_DIFF_JOIN, st, [&] {
    const dim3 g((unsigned)(j.kblocks + nq)), b(64 * G);
    if (m.causal) hipLaunchKernelGGL((diff_join_kernel<D, true, G, S>), g, b, 0, st, j);
    else hipLaunchKernelGGL((diff_join_kernel<D, false, G, S>), g, b, 0, st, j);
  });
}

template <int D>
hipError_t launch_dkdv_variant(const DiffShape& m, const DiffArgs& a, hipStream_t st) {
  const KeyTile k = key_tile(m, a);
  if (k.G == 4) return launch_dkdv<D, 4, 1>(m, a, st);
  if (k.G == 2) return k.S == 2 ? launch_dkdv<D, 2, 2>(m, a, st) : launch_dkdv<D, 2, 1>(m, a, st);
  if (k.S == 4) return launch_dkdv<D, 1, 4>(m, a, st);
  return m.N > 16 ? launch_dkdv<D, 1, 1, 1>(m, a, st) : launch_dkdv<D, 1, 1, 2>(m, a, st);
}

}  // namespace

size_t diff_attn_ws_bytes(const DiffShape& m, int T) {
  DiffArgs a = diff_args(m, T);
  cut_units(m, a);
  cut_query_units(m, a);
  return part_bytes(m, a) + align256((size_t)a.qunits * m.heads * a.nseq * (dq_variant(m, a) == 1 ? 32 : 64) * m.D * sizeof(float));
}

hipError_t launch_diff_attn_fwd(const DiffShape& m, int T, const void* qkv, const float* lambda,
                                const int32_t* lens, void* out, void* out2, float* lse,
                                hipStream_t st) {
  if (T == 0) return hipSuccess;
  DiffArgs a = diff_args(m, T);
  a.qkv = static_cast<const bf16_t*>(qkv);
  a.lambda = lambda;
  a.lens = lens;
  a.out = static_cast<bf16_t*>(out);
  a.out2 = static_cast<bf16_t*>(out2);
  a.lse = lse;
  a.shared = fwd_shared(m, a);
  const int v = fwd_variant(m, a);
  // (every block resident at once: two to a CU, four of variant 2; 1 x 4096, 8 heads,
  // causal, 1024 blocks of variant 1: 87 us with, 78 without; 1 x 2048, 32 heads, of
  // variant 2: 67 and 69)
  a.pair = m.causal && fwd_blocks(a, v) <= (v == 2 ? 1024 : 512);
  return traced(FLOWMOE_K_DIFF_FWD, st, [&] {
    if (m.D == 128) launch_fwd_variant<128>(v, m, a, st);
    else launch_fwd_variant<64>(v, m, a, st);
  });
}

hipError_t launch_diff_attn_bwd(const DiffShape& m, int T, const void* qkv, const float* lambda,
                                const int32_t* lens, const void* o, const void* o2,
                                const float* lse, const void* d_o, void* d_qkv, float* delta,
                                float* d_lambda, int accumulate, void* ws, hipStream_t st) {
  DiffArgs a = diff_args(m, T);
  a.qkv = static_cast<const bf16_t*>(qkv);
  a.lambda = lambda;
  a.lens = lens;
  a.o = static_cast<const bf16_t*>(o);
  a.o2 = static_cast<const bf16_t*>(o2);
  a.d_o = static_cast<const bf16_t*>(d_o);
  a.lse = const_cast<float*>(lse);
  a.d_qkv = static_cast<bf16_t*>(d_qkv);
  a.delta = delta;
  a.d_lambda = d_lambda;
  a.accumulate = accumulate;
  cut_units(m, a);
  cut_query_units(m, a);
  a.part = static_cast<float*>(ws);
  a.qpart = a.qunit > 0 ? reinterpret_cast<float*>(static_cast<char*>(ws) + part_bytes(m, a)) : nullptr;
  if (T > 0) {
    const hipError_t e = traced(FLOWMOE_K_DIFF_BWD_DQ, st, [&] {
      if (m.D == 128) launch_dq_variant<128>(m, a, st);
      else launch_dq_variant<64>(m, a, st);
    });
    if (e != hipSuccess) return e;
  }
  // (without tokens: dlambda alone)
  return m.D == 128 ? launch_dkdv_variant<128>(m, a, st) : launch_dkdv_variant<64>(m, a, st);
}

// ---------------------------------------------------------------------------
// the block's attention: projections, positions, differential attention, head norm
// ---------------------------------------------------------------------------
size_t diff_mha_ws_bytes(const DiffShape& m, const NormShape& n, int T) {
  const int M = m.heads * m.D, W = M + 2 * m.kv * m.D;
  return align256(std::max(std::max(diff_attn_ws_bytes(m, T), head_norm_ws_bytes(T, n.heads, n.D)),
                           std::max(wgrad_part_bytes(M, W, T), wgrad_part_bytes(M, M, T))));
}

hipError_t launch_diff_mha_fwd(const DiffShape& m, const RopeShape* r, const NormShape& n, int T,
                               const flowmoe_diff_mha_bufs_t& b, hipStream_t st) {
  if (T == 0) return hipSuccess;
  if (r != nullptr && !rope_fits(*r, T)) return hipErrorInvalidConfiguration;  // (before any launch)
  const int M = m.heads * m.D, W = M + 2 * m.kv * m.D;
  hipError_t e = launch_dense_gemm(FLOWMOE_K_ATTN_QKV, T, b.in, M, M, b.w_qkv, W, false, W, b.qkv, W, st);
  if (e == hipSuccess && r != nullptr)
    e = launch_rope(*r, FLOWMOE_BF16, T, W, false, b.qkv, b.positions, b.qkv, st);
  if (e == hipSuccess)
    e = launch_diff_attn_fwd(m, T, b.qkv, b.lambda, b.lens, b.attn, b.attn2, b.lse, st);
  if (e == hipSuccess) e = launch_head_norm_fwd(n, FLOWMOE_BF16, T, b.attn, b.gain, b.normed, st);
  if (e != hipSuccess) return e;
  return launch_dense_gemm(FLOWMOE_K_ATTN_OUT, T, b.normed, M, M, b.w_o, M, false, M, b.out, M, st);
}

hipError_t launch_diff_mha_bwd(const DiffShape& m, const RopeShape* r, const NormShape& n, int T,
                               const flowmoe_diff_mha_bufs_t& b, int accumulate, hipStream_t st) {
  if (r != nullptr && !rope_fits(*r, T)) return hipErrorInvalidConfiguration;
  const int M = m.heads * m.D, W = M + 2 * m.kv * m.D;
  hipError_t e = hipSuccess;
  // the gradient of the norm's output, B[k][n] = W^O[n][k]; the norm's backward in its place
  if (T > 0)
    e = launch_dense_gemm(FLOWMOE_K_ATTN_DGRAD, T, b.d_out, M, M, b.w_o, M, true, M, b.d_attn, M, st);
  if (e == hipSuccess)
    e = launch_head_norm_bwd(n, FLOWMOE_BF16, T, b.attn, b.gain, b.d_attn, b.d_attn, b.dgain,
                             accumulate, b.ws, st);
  if (e == hipSuccess)
    e = launch_diff_attn_bwd(m, T, b.qkv, b.lambda, b.lens, b.attn, b.attn2, b.lse, b.d_attn, b.d_qkv,
                             b.delta, b.d_lambda, accumulate, b.ws, st);
  if (e == hipSuccess && r != nullptr)
    e = launch_rope(*r, FLOWMOE_BF16, T, W, true, b.d_qkv, b.positions, b.d_qkv, st);
  if (e == hipSuccess && T > 0)
    e = launch_dense_gemm(FLOWMOE_K_ATTN_DGRAD, T, b.d_qkv, W, W, b.w_qkv, W, true, M, b.d_in, M, st);
  float* part = static_cast<float*>(b.ws);
  if (e == hipSuccess)
    e = launch_dense_wgrad(FLOWMOE_K_ATTN_WGRAD, T, 1, b.normed, M, 0, M, b.d_out, M, 0, M, b.dw_o, M,
                           accumulate, wgrad_part_bytes(M, M, T) ? part : nullptr, st);
  if (e == hipSuccess)
    e = launch_dense_wgrad(FLOWMOE_K_ATTN_WGRAD, T, 1, b.in, M, 0, M, b.d_qkv, W, 0, W, b.dw_qkv, W,
                           accumulate, wgrad_part_bytes(M, W, T) ? part : nullptr, st);
  return e;
}

}  // namespace flowmoe
