// Backward of the attention over expanded keys and values.
//
//   P = exp(S - lse), D = rowsum(dO (.) O), dS = P (.) (dO V^T - D)
//   dV = P^T dO, dK = scale dS^T Q_n, dK_rope = scale sum over heads dS^T Q_r, dQ = scale dS [K | K_rope]
//
// P and dS enter the keys' products as one value of the call's type: each has the relative
// rounding of the results themselves, so a gradient is off by about sqrt(2) of its own rounding
// (measured 1.41 to 1.45).  dQ adds what D has from the rounded O (up to 1.5), so its dS enters in two
// terms (1.00 to 1.03 then) for heads up to 128 wide; wider ones (1.45 at 192) have no registers
// left and would pay 17% of their kernel (of 2 x 2048 tokens of 7B heads).
//
// Two kernels (queries, then keys), each forming S and dO V^T anew, so that every gradient is summed by
// one owner in a fixed order (no atomics on values): one owns 128 keys of a key head,
// holds their K and V as B operands in registers and walks the queries of all heads
// that share it; the other owns 128 queries and walks their keys.  The shared rotary
// key's gradient is summed over the key heads from fp32 partial results.
//
// Bound by the matrix cores (4 dk + 4 dv operations a pair of query and key in the keys' kernel,
// 4 dk + 2 dv in the queries') and by what a wave does between them.  Measured (two sequences of
// 2048 tokens, 7B heads, 128 + 64 wide keys, bf16, medians after 20 calls): queries 184 us, keys 278 us; with
// the forward (115 us) 553 TFLOP/s of the least work.  (The first calls on a card at rest are slower:
// 211, 341 and 133 us.)  The matrix cores are busy
// 48 and 30% of the CUs' cycles: the keys' wave holds so many operands and sums that one fits
// a SIMD, and nothing runs beside its loads and exponentials (of 7600 cycles of a step 2200
// issue loads, 2700 are scores and exponentials, 1900 the last products).  Two waves a
// SIMD that share the keys and pass P and dS through LDS were no faster (358 us).
#include "attn.h"
#include "attn_common.h"

namespace lb {

namespace {

constexpr int kThreads = 256;
constexpr int kWideRows = 128;  // rows a workgroup owns

struct BwdArgs {
  AttnArgs a;
  int vec, ovec;        // rows (those of o) may be read 16 bytes at a time
  int qvec, kvec, vvec;  // dq, dk, dv rows may be written four elements at a time
};

// f16: dS (|dO| |V| times a probability: anything from 2^-60 to 2^40) enters its products times a
// power of two, kept for each column of the accumulators (a query in one kernel, a key in the
// other) and lowered once the column's largest value passes 2^15, which brings it to 2^11 .. 2^12; the
// column's sums follow.  A value then keeps its 11 bits down to 2^-25 of the column's largest, whatever other
// columns, sequences or rows behind the last sequence hold.
constexpr float kDsMost = 32768.0f;
constexpr float kDsStart = 1.152921504606846976e18f;  // 2^60: what it leaves too small is far below f16's results
template <int DT, int T>
__device__ __forceinline__ void scale_ds(floatx16& ds, float& fac, floatx16 (&acc)[T]) {
  if constexpr (DT == kDtF16) {
    float m = 0.0f;
#pragma unroll
    for (int e = 0; e < 16; ++e) m = fmaxf(m, fabsf(ds[e]));
    m = fmaxf(m, __shfl_xor(m, 32));
    if (__any(m * fac > kDsMost)) {
      float to = fac;
      if (m * fac > kDsMost) {
        int ex;
        frexpf(fminf(m, 1e30f), &ex);
        to = ldexpf(1.0f, 12 - ex);
      }
      const float r = to / fac;
      fac = to;
#pragma unroll
      for (int t = 0; t < T; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[t][e] *= r;
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) ds[e] *= fac;
  }
}
// f16: P enters dV's product times 2^14, so that it keeps its 11 bits down to 2^-28 (a key that every
// query gives little has its gradient from nothing else); dS has the factor too
template <int DT>
constexpr float p_bits() {
  return DT == kDtF16 ? 14.0f : 0.0f;
}
template <int DT>
constexpr float p_factor() {
  return DT == kDtF16 ? 1.0f / 16384.0f : 1.0f;
}
template <int DT>
constexpr float ds_start() {
  return DT == kDtF16 ? kDsStart : 1.0f;
}

// S and dO V^T of a 32 x 32 block: A operands from rows of the tiles t0 (KC slices) and
// t1 (2 VT slices), B operands in registers; groups of GK fragments, each read while the
// one before is multiplied; tick(g) stands before group g's products.
template <int DT, int KC, int VC, int R, int GK, typename TICK>
__device__ __forceinline__ void scores(const char* t0, const char* t1, int row0, int lane, const Frag<DT> (&b0)[KC],
                                       const Frag<DT> (&b1)[VC], floatx16& s, floatx16& dp, TICK&& tick) {
  constexpr int N = KC + VC, NG = (N + GK - 1) / GK;
#pragma unroll
  for (int e = 0; e < 16; ++e) s[e] = 0.0f, dp[e] = 0.0f;
  Frag<DT> f[2][GK];
#pragma unroll
  for (int g = -1; g < NG; ++g) {
#pragma unroll
    for (int n = 0; n < GK; ++n) {
      const int c = (g + 1) * GK + n;
      if (c < KC)
        f[(g + 1) & 1][n] = frag_rows<DT, R>(t0, row0, 16 * c, lane);
      else if (c < N)
        f[(g + 1) & 1][n] = frag_rows<DT, R>(t1, row0, 16 * (c - KC), lane);
    }
    keep_order();
    if (g >= 0) {
      tick(g);
#pragma unroll
      for (int n = 0; n < GK; ++n) {
        const int c = g * GK + n;
        if (c < KC)
          s = mma32<DT>(f[g & 1][n], b0[c < KC ? c : 0], s);
        else if (c < N)
          dp = mma32<DT>(f[g & 1][n], b1[c >= KC && c < N ? c - KC : 0], dp);
      }
    }
  }
}
// acc[t] += (columns 32 t .. of the tile's rows row0 .. row0 + 31)^T x, x the block's
// accumulator as B operand, in TERMS terms of the type
template <int DT, int T, int R, int MOST = 4, int TERMS = 1>
__device__ __forceinline__ void add_products(const char* tile, int row0, int lane, const floatx16& x, floatx16 (&acc)[T]) {
  constexpr int GK = DT == kDtF32 ? 1 : T % 4 == 0 && MOST >= 4 ? 4 : T % 3 == 0 && MOST >= 3 ? 3 : 2, NG = 2 * T / GK;
  Frag<DT> f[2][GK], xf[TERMS][2];
#pragma unroll
  for (int sl = 0; sl < 2; ++sl) {
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = x[8 * sl + e];
    xf[0][sl] = frag_from<DT>(v);
    if constexpr (TERMS > 1) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] -= frag_elem<DT>(xf[0][sl], e);
      xf[1][sl] = frag_from<DT>(v);
    }
  }
#pragma unroll
  for (int g = -1; g < NG; ++g) {
    if (g + 1 < NG) {
#pragma unroll
      for (int n = 0; n < GK; ++n) {
        const int c = (g + 1) * GK + n;
        f[(g + 1) & 1][n] = frag_cols<DT, R>(tile, row0 + 16 * (c / T), 32 * (c % T), lane);
      }
    }
    keep_order();
    if (g >= 0) {
#pragma unroll
      for (int n = 0; n < GK; ++n) {
        const int c = g * GK + n;
        acc[c % T] = mma32<DT>(f[g & 1][n], xf[0][c / T], acc[c % T]);
      }
      if constexpr (TERMS > 1) {
#pragma unroll
        for (int n = 0; n < GK; ++n) {
          const int c = g * GK + n;
          acc[c % T] = mma32<DT>(f[g & 1][n], xf[1][c / T], acc[c % T]);
        }
      }
    }
  }
}

// Four waves' parts of an accumulator added, in their order: wave w gets rows 8 w + 4 (lane /
// 32) + q of its column in v[q].  buf: 16 KB.
__device__ __forceinline__ void join_waves(float* buf, const floatx16& x, int wave, int lane, float (&v)[4]) {
  lds_barrier();
#pragma unroll
  for (int e = 0; e < 16; ++e) buf[(wave * 16 + e) * 64 + lane] = x[e];
  lds_barrier();
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    v[q] = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w) v[q] += buf[(w * 16 + 4 * wave + q) * 64 + lane];
  }
}

// rows of a step: two tiles of 192 + 128 columns fill half of a CU's LDS; one tile that
// four waves split (32 rows each) where they share the workgroup's rows
template <int DT, bool WIDE>
constexpr int step_of() {
  return !WIDE ? 128 : DT == kDtF32 ? 32 : 64;
}
template <int DT, int KC, int VT, bool WIDE>
constexpr size_t lds_of(bool stats) {  // stats: 8 bytes a row (the keys' kernel)
  constexpr int B = step_of<DT, WIDE>();
  return (WIDE ? 2 : 1) * static_cast<size_t>(tile_bytes<DT, B, 16 * KC + 32 * VT>() + (stats ? 8 * B : 0));
}
constexpr size_t kLdsMax = 163840;

// queries: dQ.  For queries with few keys D is formed anew as sum_j P (dO V^T): the one
// from the rounded O is off by up to half a step of it, which where few keys share the
// weight is as large as the rounding of dS and the result together (at 20 keys 1.6 times
// the result's own rounding, at 600 1.1 times).
constexpr int kExactKeys = 512;
// WIDE and its other form: as in the forward.
template <int DT, int KC, int VT, bool WIDE>
__global__ void __launch_bounds__(kThreads, DT == kDtF32 || !WIDE ? 1 : 2) attn_bwd_queries(BwdArgs f) {
  constexpr int BN = step_of<DT, WIDE>(), kBM = WIDE ? kWideRows : 32, NB = WIDE ? BN / 32 : 1;
  constexpr bool SPREAD = WIDE && DT != kDtF32;  // as in the forward
  constexpr int KW = 16 * KC, VW = 32 * VT, KT = KC / 2;
  constexpr int DST = DT == kDtF32 || KC > 8 ? 1 : 2;  // terms of dS
  constexpr int SG = DT == kDtF32 ? 1 : KC > 8 ? 2 : 4;  // fragments read ahead: two waves a SIMD leave 256 registers
  constexpr int KB = tile_bytes<DT, BN, KW>(), TB = KB + tile_bytes<DT, BN, VW>(), ES = esize<DT>();
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const AttnArgs& a = f.a;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hh = lane >> 5, col = lane & 31;
  const int id = blockIdx.x, hi_ = id % a.H, G = a.H / a.Hk;
  const int kvh = hi_ % a.Hk, h = kvh * G + hi_ / a.Hk;
  int seq, tile;
  if (!find_tile(a.cu_q, a.n_seq, a.Tq, kBM, id / a.H, lane, seq, tile)) return;
  seq = __builtin_amdgcn_readfirstlane(seq), tile = __builtin_amdgcn_readfirstlane(tile);
  int q_lo, q_hi, k_lo, k_hi;
  seq_range(a.cu_q, seq, a.Tq, q_lo, q_hi);
  seq_range(a.cu_k, seq, a.Tk, k_lo, k_hi);
  const int nq = q_hi - q_lo, nk = k_hi - k_lo, off = nk - nq;
  tile = (nq + kBM - 1) / kBM - 1 - tile;  // the longest first
  const int w0 = WIDE ? 32 * wave : 0, rb = WIDE ? 0 : 32 * wave;  // the wave's first query and key in the tiles
  const int i0 = tile * kBM, i = i0 + w0 + col;
  const int dk = a.d_nope + a.d_rope, dv = a.d_v;
  const int lim = a.causal ? min(nk - 1, i + off) : nk - 1;
  const int lim_lo = a.causal ? min(nk - 1, i0 + w0 + off) : nk - 1;
  const int n_end = a.causal ? min(nk, min(i0 + kBM, nq) + off) : nk;
  const int w_end = a.causal ? min(n_end, i0 + w0 + 32 + off) : n_end;
  const float sc = a.scale * kLog2e;

  const char* kp = static_cast<const char*>(a.k) + (k_lo * a.k_t + kvh * a.k_h) * ES;
  const char* vp = static_cast<const char*>(a.v) + (k_lo * a.v_t + kvh * a.v_h) * ES;
  const char* rp = static_cast<const char*>(a.k_rope) + k_lo * a.kr_t * ES;
  auto issue = [&](int j0, char* t) __attribute__((always_inline)) {
    tile_load<DT, BN, KW, kThreads>(t, kp + j0 * a.k_t * ES, a.k_t, a.d_nope, rp + j0 * a.kr_t * ES, a.kr_t, a.d_rope,
                                    nk - j0, f.vec, tid);
    tile_load<DT, BN, VW, kThreads>(t + KB, vp + j0 * a.v_t * ES, a.v_t, dv, nullptr, 0, 0, nk - j0, f.vec, tid);
  };
  constexpr int R4 = 256 / pieces<DT>();  // (BN where SPREAD)
  TileLoads<DT, R4, KW, kThreads> kl;
  TileLoads<DT, R4, VW, kThreads> vl;
  constexpr int LOADS = SPREAD ? kl.LOADS + vl.LOADS : 0;
  auto tick = [&](int n) __attribute__((always_inline)) {
    if constexpr (SPREAD) {
      if (n < kl.LOADS)
        kl.load(n);
      else if (n < LOADS)
        vl.load(n - kl.LOADS);
    }
  };
  if (n_end > 0) issue(0, smem);
  const int64_t row = static_cast<int64_t>(q_lo + min(i, nq - 1)) * a.H + h;
  Frag<DT> qf[KC], df[2 * VT];
  {
    const char* qp = static_cast<const char*>(a.q) + ((q_lo + min(i, nq - 1)) * a.q_t + h * a.q_h) * ES;
    const char* dp = static_cast<const char*>(a.d_o) + row * dv * ES;
#pragma unroll
    for (int c = 0; c < KC; ++c) qf[c] = load8<DT>(qp, 16 * c + 8 * hh, dk, f.vec);
#pragma unroll
    for (int c = 0; c < 2 * VT; ++c) df[c] = load8<DT>(dp, 16 * c + 8 * hh, dv, f.vec);
  }
  const float l = a.lse[row];
  const float l2 = l == -INFINITY ? INFINITY : l * kLog2e;
  // D of the given O: in the row's two lanes, half of the columns each
  float del = 0.0f;
  {
    const char* op = static_cast<const char*>(a.o) + row * dv * ES;
#pragma unroll
    for (int c = 0; c < 2 * VT; ++c) {
      const Frag<DT> x = load8<DT>(op, 16 * c + 8 * hh, dv, f.ovec);
#pragma unroll
      for (int e = 0; e < 8; ++e) del += frag_elem<DT>(x, e) * frag_elem<DT>(df[c], e);
    }
    del += __shfl_xor(del, 32);
  }
  // P in s, from S; the mask where the block reaches past a query's last key
  auto probabilities = [&](int j, floatx16& s) __attribute__((always_inline)) {
    const bool mask = j + 31 > lim_lo;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      s[e] = exp2_fast(s[e] * sc - l2);
      if (mask && j + 8 * (e >> 2) + 4 * hh + (e & 3) > lim) s[e] = 0.0f;
    }
  };
  int at = 0;  // the tile that is read (the other form: whether it has been read)
  // the keys' tiles in turn; the last step issues the first tile again if `more`
  // (inlined by force: in the fp32 kernels the compiler made calls of these, through scratch)
  auto walk = [&](bool more, auto&& block) __attribute__((always_inline)) {
    for (int j0 = 0; j0 < n_end; j0 += BN) {
      char* kt = smem + (WIDE ? at * TB : 0);
      if constexpr (WIDE) {
        at ^= 1;
        wait_loads();
        lds_barrier();
        char* to = smem + at * TB;
        if constexpr (SPREAD) {
          // (after the last tile, the first: no branch between the products)
          const int jn = j0 + BN < n_end ? j0 + BN : 0;
          kl.start(to, kp + jn * a.k_t * ES, a.k_t, a.d_nope, rp + jn * a.kr_t * ES, a.kr_t, a.d_rope, nk - jn, tid);
          vl.start(to + KB, vp + jn * a.v_t * ES, a.v_t, dv, nullptr, 0, 0, nk - jn, tid);
        } else if (j0 + BN < n_end) {
          issue(j0 + BN, to);
        } else if (more) {
          issue(0, to);
        }
      } else {
        if (at > 0) {
          lds_barrier();
          issue(j0, smem);
        }
        at = 1;
        wait_loads();
        lds_barrier();
      }
      if (j0 + rb >= w_end) {
#pragma unroll
        for (int n = 0; n < LOADS; ++n) tick(n);
        continue;
      }
      // (the loads between the score products of the blocks: NG groups each)
      constexpr int NG = (KC + 2 * VT + SG - 1) / SG;
      static_assert(!SPREAD || NB * NG >= LOADS, "a place for every load");
#pragma unroll
      for (int b = 0; b < NB; ++b)
        block(kt, kt + KB, rb + 32 * b, j0 + rb + 32 * b, [&](int g) { tick(b * NG + g); });
    }
  };
  if (n_end <= kExactKeys) {
    float d = 0.0f;
    walk(true, [&](const char* kt, const char* vt, int r0, int j, auto&& between) __attribute__((always_inline)) {
      floatx16 s, dp;
      scores<DT, KC, 2 * VT, BN, SG>(kt, vt, r0, lane, qf, df, s, dp, between);
      probabilities(j, s);
#pragma unroll
      for (int e = 0; e < 16; ++e) d += s[e] == 0.0f ? 0.0f : s[e] * dp[e];
    });
    del = d + __shfl_xor(d, 32);
    if constexpr (!WIDE) {
      float* part = reinterpret_cast<float*>(smem);
      lds_barrier();
      if (hh == 0) part[wave * 32 + col] = del;
      lds_barrier();
      del = (part[col] + part[32 + col]) + (part[64 + col] + part[96 + col]);
    }
  }
  if (hh == 0 && i < nq && (WIDE || wave == 0)) a.delta[row] = del;  // (read by the keys' kernel, which runs after this one)
  floatx16 gq[KT];
#pragma unroll
  for (int t = 0; t < KT; ++t)
#pragma unroll
    for (int e = 0; e < 16; ++e) gq[t][e] = 0.0f;
  float fac = ds_start<DT>();
  walk(false, [&](const char* kt, const char* vt, int r0, int j, auto&& between) __attribute__((always_inline)) {
    floatx16 s, dp;
    scores<DT, KC, 2 * VT, BN, SG>(kt, vt, r0, lane, qf, df, s, dp, between);
    probabilities(j, s);
#pragma unroll
    for (int e = 0; e < 16; ++e) dp[e] = s[e] == 0.0f ? 0.0f : s[e] * (dp[e] - del);
    scale_ds<DT>(dp, fac, gq);
    add_products<DT, KT, BN, SG, DST>(kt, r0, lane, dp, gq);
  });
  if constexpr (SPREAD) wait_loads();  // none may arrive after the workgroup's end
  // (the waves' parts have factors of their own)
  const float inv = 1.0f / fac, qs = WIDE ? a.scale * inv : a.scale;
  char* gp = static_cast<char*>(a.dq) + row * dk * ES;
#pragma unroll
  for (int n = 0; n < KT; ++n) {
    if constexpr (WIDE) {
      if (i < nq) {
#pragma unroll
        for (int e = 0; e < 16; e += 4)
          store4<DT>(gp, 32 * n + 2 * e + 4 * hh, dk, f.qvec, gq[n][e] * qs, gq[n][e + 1] * qs, gq[n][e + 2] * qs,
                     gq[n][e + 3] * qs);
      }
    } else {
      float v[4];
      if constexpr (DT == kDtF16) gq[n] *= inv;
      join_waves(reinterpret_cast<float*>(smem), gq[n], wave, lane, v);
      if (i < nq) store4<DT>(gp, 32 * n + 8 * wave + 4 * hh, dk, f.qvec, v[0] * qs, v[1] * qs, v[2] * qs, v[3] * qs);
    }
  }
}

// keys: dK, dV.  (The loads of a step all at once: one at a time between the products, as for
// the queries, they take registers that the accumulators and operands do not leave.)
// Not WIDE: the four waves share 32 keys and split the queries.
template <int DT, int KC, int VT, bool WIDE>
__global__ void __launch_bounds__(kThreads, 1) attn_bwd_keys(BwdArgs f) {
  constexpr int BQ = step_of<DT, WIDE>(), kBM = WIDE ? kWideRows : 32, NB = WIDE ? BQ / 32 : 1, KW = 16 * KC, VW = 32 * VT, KT = KC / 2;
  constexpr int KB = tile_bytes<DT, BQ, KW>(), TB = KB + tile_bytes<DT, BQ, VW>() + 8 * BQ, ES = esize<DT>();
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const AttnArgs& a = f.a;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hh = lane >> 5, col = lane & 31;
  const int kvh = blockIdx.x % a.Hk, G = a.H / a.Hk;
  int seq, tile;
  if (!find_tile(a.cu_k, a.n_seq, a.Tk, kBM, blockIdx.x / a.Hk, lane, seq, tile)) return;
  seq = __builtin_amdgcn_readfirstlane(seq), tile = __builtin_amdgcn_readfirstlane(tile);
  int q_lo, q_hi, k_lo, k_hi;
  seq_range(a.cu_q, seq, a.Tq, q_lo, q_hi);
  seq_range(a.cu_k, seq, a.Tk, k_lo, k_hi);
  const int nq = q_hi - q_lo, nk = k_hi - k_lo, off = nk - nq;
  const int w0 = WIDE ? 32 * wave : 0, rb = WIDE ? 0 : 32 * wave;  // the wave's first key and query in the tiles
  const int j0 = tile * kBM, j = j0 + w0 + col;                    // this lane's key
  const int dk = a.d_nope + a.d_rope, dv = a.d_v;
  const float sc = a.scale * kLog2e;

  const int i_begin = a.causal ? max(0, j0 - off) / BQ * BQ : 0;
  const int n_it = max(0, (nq - i_begin + BQ - 1) / BQ), total = G * n_it;
  // a step: the queries i0 .. of head g of the group
  float lr = 0.0f, de = 0.0f;
  auto issue = [&](int i0, int g, char* t) {
    const int h = kvh * G + g;
    tile_load<DT, BQ, KW, kThreads>(t, static_cast<const char*>(a.q) + ((q_lo + i0) * a.q_t + h * a.q_h) * ES, a.q_t, dk,
                                    nullptr, 0, 0, nq - i0, f.vec, tid);
    tile_load<DT, BQ, VW, kThreads>(
        t + KB, static_cast<const char*>(a.d_o) + (static_cast<int64_t>(q_lo + i0) * a.H + h) * dv * ES,
        static_cast<int64_t>(a.H) * dv, dv, nullptr, 0, 0, nq - i0, f.vec, tid);
  };
  // statistics of a step's queries: into registers, and a step later (when the loads have
  // been waited for) into LDS
  auto fetch_stats = [&](int i0, int g) {
    if (tid < BQ) {
      const int64_t r = static_cast<int64_t>(q_lo + min(i0 + tid, nq - 1)) * a.H + kvh * G + min(g, G - 1);
      lr = a.lse[r], de = a.delta[r];
    }
  };
  auto put_stats = [&](int i0, char* t) {
    if (tid < BQ) {
      // rows past the end and rows that see no key get probability 0
      const bool ok = i0 + tid < nq && lr != -INFINITY;
      float* st = reinterpret_cast<float*>(t + TB - 8 * BQ);
      st[tid] = ok ? lr * kLog2e - p_bits<DT>() : INFINITY, st[BQ + tid] = ok ? de : 0.0f;
    }
  };
  auto next = [&](int& i0, int& g) {
    i0 += BQ;
    if (i0 >= nq) i0 = i_begin, ++g;
  };
  int i1 = i_begin, g1 = 0;  // the step behind the current one
  if (total > 0) {
    fetch_stats(i1, g1);
    put_stats(i1, smem);
    issue(i1, g1, smem);
    next(i1, g1);
    fetch_stats(i1, g1);
  }
  Frag<DT> kf[KC], vf[2 * VT];
  {
    const int64_t t = k_lo + min(j, nk - 1);
    const char* kp = static_cast<const char*>(a.k) + (t * a.k_t + kvh * a.k_h) * ES;
    const char* rp = static_cast<const char*>(a.k_rope) + t * a.kr_t * ES;
    const char* vp = static_cast<const char*>(a.v) + (t * a.v_t + kvh * a.v_h) * ES;
#pragma unroll
    for (int c = 0; c < KC; ++c) kf[c] = load8_joined<DT>(kp, a.d_nope, rp, a.d_rope, 16 * c + 8 * hh, f.vec);
#pragma unroll
    for (int c = 0; c < 2 * VT; ++c) vf[c] = load8<DT>(vp, 16 * c + 8 * hh, dv, f.vec);
  }
  floatx16 gk[KT], gv[VT];
#pragma unroll
  for (int t = 0; t < KT; ++t)
#pragma unroll
    for (int e = 0; e < 16; ++e) gk[t][e] = 0.0f;
#pragma unroll
  for (int t = 0; t < VT; ++t)
#pragma unroll
    for (int e = 0; e < 16; ++e) gv[t][e] = 0.0f;

  float fac = ds_start<DT>();
  int i_now = i_begin, g_now = 0;
  for (int it = 0; it < total; ++it) {
    char* qt = smem + (WIDE ? (it & 1) * TB : 0);
    const char* dt = qt + KB;
    const float* st = reinterpret_cast<const float*>(qt + TB - 8 * BQ);
    if (!WIDE && it > 0) {
      lds_barrier();
      put_stats(i_now, qt);  // (this step's: fetched during the one before)
      fetch_stats(i1, g1);
      issue(i_now, g_now, qt);
    }
    wait_loads();
    lds_barrier();
    const int i_here = i_now + rb;
    i_now = i1, g_now = g1;
    if (it + 1 < total) {
      next(i1, g1);
      if constexpr (WIDE) {
        char* t = smem + (~it & 1) * TB;
        put_stats(i_now, t);
        fetch_stats(i1, g1);
        issue(i_now, g_now, t);
      }
    }
    if (a.causal && i_here + 32 * NB - 1 + off < j0 + w0) continue;  // every query before the wave's first key
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      floatx16 s, dp;
      scores<DT, KC, 2 * VT, BQ, DT == kDtF32 ? 1 : 4>(qt, dt, rb + 32 * b, lane, kf, vf, s, dp, [](int) {});
      const bool mask = a.causal && i_here + 32 * b + off < j0 + w0 + 31;
#pragma unroll
      for (int e = 0; e < 16; e += 4) {
        const int row = 32 * b + 2 * e + 4 * hh;
        const float4 l4 = *reinterpret_cast<const float4*>(st + rb + row);
        const float4 d4 = *reinterpret_cast<const float4*>(st + BQ + rb + row);
        const float lv[4] = {l4.x, l4.y, l4.z, l4.w}, dl[4] = {d4.x, d4.y, d4.z, d4.w};
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          float p = exp2_fast(s[e + q] * sc - lv[q]);
          if (mask && i_here + row + q + off < j) p = 0.0f;
          s[e + q] = p;
          dp[e + q] = p == 0.0f ? 0.0f : p * (dp[e + q] - dl[q]);
        }
      }
      add_products<DT, VT, BQ>(dt, rb + 32 * b, lane, s, gv);
      scale_ds<DT>(dp, fac, gk);
      add_products<DT, KT, BQ>(qt, rb + 32 * b, lane, dp, gk);
    }
  }
  const int64_t t = k_lo + min(j, nk - 1);
  const float inv = p_factor<DT>() / fac, ks = WIDE ? a.scale * inv : a.scale;
  char* gkp = static_cast<char*>(a.dk) + (t * a.dk_t + kvh * a.dk_h) * ES;
  char* gvp = static_cast<char*>(a.dv) + (t * a.dv_t + kvh * a.dv_h) * ES;
  float* grp = a.dkr_part + (static_cast<int64_t>(kvh) * a.Tk + t) * a.d_rope;
  auto put_v = [&](int c, float v0, float v1, float v2, float v3) {
    constexpr float u = p_factor<DT>();
    if (j < nk) store4<DT>(gvp, c, dv, f.vvec, v0 * u, v1 * u, v2 * u, v3 * u);
  };
  auto put_k = [&](int c, float v0, float v1, float v2, float v3) {
    if (j >= nk) return;
    const float v[4] = {v0 * ks, v1 * ks, v2 * ks, v3 * ks};
    store4<DT>(gkp, c, a.d_nope, f.kvec, v[0], v[1], v[2], v[3]);
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (c + q >= a.d_nope && c + q < dk) grp[c + q - a.d_nope] = v[q];
  };
  float* buf = reinterpret_cast<float*>(smem);
#pragma unroll
  for (int n = 0; n < VT; ++n) {
    if constexpr (WIDE) {
#pragma unroll
      for (int e = 0; e < 16; e += 4) put_v(32 * n + 2 * e + 4 * hh, gv[n][e], gv[n][e + 1], gv[n][e + 2], gv[n][e + 3]);
    } else {
      float v[4];
      join_waves(buf, gv[n], wave, lane, v);
      put_v(32 * n + 8 * wave + 4 * hh, v[0], v[1], v[2], v[3]);
    }
  }
#pragma unroll
  for (int n = 0; n < KT; ++n) {
    if constexpr (WIDE) {
#pragma unroll
      for (int e = 0; e < 16; e += 4) put_k(32 * n + 2 * e + 4 * hh, gk[n][e], gk[n][e + 1], gk[n][e + 2], gk[n][e + 3]);
    } else {
      float v[4];
      if constexpr (DT == kDtF16) gk[n] *= inv;
      join_waves(buf, gk[n], wave, lane, v);
      put_k(32 * n + 8 * wave + 4 * hh, v[0], v[1], v[2], v[3]);
    }
  }
}

// the shared rotary key's gradient: the key heads' partial results in order
template <int DT>
__global__ void __launch_bounds__(kThreads) rope_sum(AttnArgs a) {
  const int64_t n = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
  const int64_t per = static_cast<int64_t>(a.Tk) * a.d_rope;
  if (n >= per) return;
  const int t = static_cast<int>(n / a.d_rope);
  if (a.cu_k != nullptr && (t < a.cu_k[0] || t >= a.cu_k[a.n_seq])) return;  // in no sequence
  float s = 0.0f;
#pragma unroll 4
  for (int h = 0; h < a.Hk; ++h) s += a.dkr_part[h * per + n];
  st<DT>(a.dkr, n, s);
}

// one of the two kernels in the form that fits the call
template <int DT, int KC, int VT, bool QUERIES, bool WIDE>
hipError_t bwd_one(const BwdArgs& f, int T, const int32_t* cu, int heads, hipStream_t stream) {
  constexpr size_t lds = lds_of<DT, KC, VT, WIDE>(!QUERIES);
  constexpr int rows = WIDE ? kWideRows : 32;
  const dim3 grid(static_cast<uint32_t>((T + rows - 1) / rows + (cu ? f.a.n_seq : 0)) * heads);
  static LdsLimit limit;
  if constexpr (QUERIES) {
    const hipError_t e = raise_lds(reinterpret_cast<const void*>(&attn_bwd_queries<DT, KC, VT, WIDE>), lds, limit);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((attn_bwd_queries<DT, KC, VT, WIDE>), grid, dim3(kThreads), lds, stream, f);
  } else {
    const hipError_t e = raise_lds(reinterpret_cast<const void*>(&attn_bwd_keys<DT, KC, VT, WIDE>), lds, limit);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((attn_bwd_keys<DT, KC, VT, WIDE>), grid, dim3(kThreads), lds, stream, f);
  }
  return hipGetLastError();
}
template <int DT, int KC, int VT, bool QUERIES>
hipError_t bwd_form(const BwdArgs& f, int T, const int32_t* cu, int heads, hipStream_t stream) {
  if (T == 0) return hipSuccess;
  // us, 128 rows a workgroup against the other form.  bf16, 7B heads, the queries' kernel: 160 workgroups (512 rows)
  // 41.2 against 29.8, 192 (4 x 128) 20.4 against 20.4, 224 (768) 41.3 against 41.7, 272 (2048) 79.6 against 75.0, 280 (4 x
  // 256) 28.4 against 42.4; the keys': 160 39.8 against 35.2, 192 24.4 against 27.7, 224 50.8 against 57.0, 280 31.2
  // against 52.9, four queries' heads a key head 264 362 against 377.  fp32, 64 wide, queries: 272 251 against 166, 408
  // 304 against 237, 544 327 against 302, 1056 520 against 594; keys: 272 305 against 191, 408 379 against 262, 544 408
  // against 340; 128 wide, queries: 272 423 against 336, 408 425 against 488; keys: 272 546 against 375, 408 553 against 558,
  // 544 601 against 734.  (Heads of up to 64 columns would cross later, above all the keys' with grouped heads: 16-bit 264 260
  // against 139.  The widest fp32 heads' 128 rows do not fit.  16-bit rows that fit no 16-byte loads
  // take the other form.)
  if constexpr (lds_of<DT, KC, VT, false>(!QUERIES) <= kLdsMax) {
    if (wide_groups(T, cu ? f.a.n_seq : 0, heads) < (DT == kDtF32 ? 400 : 210) || (DT != kDtF32 && !f.vec))
      return bwd_one<DT, KC, VT, QUERIES, false>(f, T, cu, heads, stream);
  }
  return bwd_one<DT, KC, VT, QUERIES, true>(f, T, cu, heads, stream);
}
template <int DT, int KC, int VT>
hipError_t bwd_launch(const BwdArgs& f, hipStream_t stream) {
  hipError_t e = bwd_form<DT, KC, VT, true>(f, f.a.Tq, f.a.cu_q, f.a.H, stream);
  if (e != hipSuccess) return e;
  e = bwd_form<DT, KC, VT, false>(f, f.a.Tk, f.a.cu_k, f.a.Hk, stream);
  if (e != hipSuccess) return e;
  if (f.a.d_rope > 0 && f.a.Tk > 0) {
    const int64_t n = static_cast<int64_t>(f.a.Tk) * f.a.d_rope;
    hipLaunchKernelGGL((rope_sum<DT>), dim3(static_cast<uint32_t>((n + kThreads - 1) / kThreads)), dim3(kThreads), 0,
                       stream, f.a);
    e = hipGetLastError();
  }
  return e;
}
template <int DT, int VT>
hipError_t bwd_kc(const BwdArgs& f, hipStream_t stream) {
  const int dk = f.a.d_nope + f.a.d_rope;
  if (dk <= 64) return bwd_launch<DT, 4, VT>(f, stream);
  if (dk <= 128) return bwd_launch<DT, 8, VT>(f, stream);
  return bwd_launch<DT, 12, VT>(f, stream);
}
template <int DT>
hipError_t bwd_dt(const BwdArgs& f, hipStream_t stream) {
  return f.a.d_v <= 64 ? bwd_kc<DT, 2>(f, stream) : bwd_kc<DT, 4>(f, stream);
}

}  // namespace

hipError_t launch_attn_backward(const AttnArgs& a, hipStream_t stream) {
  BwdArgs f{};
  f.a = a;
  f.vec = attn_vec(a, true);
  auto ok = [](const void* p, int64_t st, int64_t sh, int n) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && st % 4 == 0 && sh % 4 == 0 && n % 4 == 0;
  };
  f.qvec = ok(a.dq, 0, 0, a.d_nope + a.d_rope);
  f.kvec = ok(a.dk, a.dk_t, a.dk_h, a.d_nope);
  f.vvec = ok(a.dv, a.dv_t, a.dv_h, a.d_v);
  f.ovec = f.vec && reinterpret_cast<uintptr_t>(a.o) % 16 == 0;
  switch (a.dt) {
    case kDtF32: return bwd_dt<kDtF32>(f, stream);
    case kDtF16: return bwd_dt<kDtF16>(f, stream);
    default: return bwd_dt<kDtBF16>(f, stream);
  }
}

}  // namespace lb
