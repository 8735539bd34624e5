// Attention over expanded keys and values of packed sequences, forward.
//
//   S = scale (q_n k^T + q_r k_rope^T), O = softmax(S) V, lse = log sum exp S
//
// One pass over the keys with a running maximum and sum.  A wave owns 32 query rows as
// the columns of 32 x 32 tiles of S^T = K Q^T: a column's softmax then stays in two
// lanes, its factor is the lane's own for O^T = V^T P^T, and P goes from one product
// into the next in registers.  Bound by the matrix cores (2 (dk + dv) operations a
// pair of query and key) and, beside them, by the softmax's vector instructions: two
// waves a SIMD, so that one's run beside the other's products.
//
// Measured (7B heads, 128 + 64 wide keys, 128 wide values, bf16): four prompts of 8192 tokens 231 us a call
// (249 to 259 under the profiler), 780 TFLOP/s of the seen pairs (a large library product reaches 1120), the
// matrix cores busy 44% of the CUs' cycles (masked and padded pairs included); 777 tokens of 64
// grouped heads in f16 17.4 us.
#include "attn.h"
#include "attn_common.h"

namespace lb {

namespace {

constexpr int kThreads = 256;
constexpr int kWideRows = 128;   // query rows of a workgroup (4 waves x 32)
constexpr int kSplitKeys = 128;  // keys of a tile that four waves split
// keys of a step: two tiles of 192 + 128 columns fill half of a CU's LDS (fp32: all of it)
template <int DT>
constexpr int keys_of() {
  return DT == kDtF32 ? 32 : 64;
}

struct FwdArgs {
  AttnArgs a;
  int vec;      // rows may be read 16 bytes at a time
  int ovec;     // ... and o written four elements at a time
  int n_tiles;  // work items per head (an upper bound)
};

// KC: 16-wide slices of a key's width, VT: 32-wide tiles of a value's.
// WIDE: a wave has 32 queries of its own and all keys; two tiles of K and V, the next one's
// loads run during the products with this one.
// Otherwise the four waves share 32 queries and split the keys, a block of 32 each of one
// tile, and their sums are joined at the end: a quarter of the steps one after the other,
// for calls with too few queries and heads to fill the chip with 128-query workgroups.
template <int DT, int KC, int VT, bool WIDE>
__global__ void __launch_bounds__(kThreads, DT == kDtF32 || !WIDE ? 1 : 2) attn_fwd(FwdArgs f) {
  constexpr int KW = 16 * KC, VW = 32 * VT, BN = WIDE ? keys_of<DT>() : kSplitKeys, kBM = WIDE ? kWideRows : 32;
  constexpr int NB = WIDE ? BN / 32 : 1;  // blocks of 32 keys a wave takes of a tile
  constexpr bool SPREAD = WIDE && DT != kDtF32;  // the next tile's loads one at a time (rows fit 16-byte loads)
  constexpr int KB = tile_bytes<DT, BN, KW>(), TB = KB + tile_bytes<DT, BN, VW>();
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const AttnArgs& a = f.a;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hh = lane >> 5, col = lane & 31;
  // heads of one key head next to each other in turn, so that every XCD keeps few of them
  const int id = blockIdx.x, hi_ = id % a.H, G = a.H / a.Hk;
  const int kvh = hi_ % a.Hk, h = kvh * G + hi_ / a.Hk;
  int seq, tile;
  if (!find_tile(a.cu_q, a.n_seq, a.Tq, kBM, id / a.H, lane, seq, tile)) return;
  seq = __builtin_amdgcn_readfirstlane(seq), tile = __builtin_amdgcn_readfirstlane(tile);
  int q_lo, q_hi, k_lo, k_hi;
  seq_range(a.cu_q, seq, a.Tq, q_lo, q_hi);
  seq_range(a.cu_k, seq, a.Tk, k_lo, k_hi);
  const int nq = q_hi - q_lo, nk = k_hi - k_lo;
  // the last tiles first: with a causal mask they have the most keys
  tile = (nq + kBM - 1) / kBM - 1 - tile;
  const int i0 = tile * kBM, off = nk - nq;
  const int dk = a.d_nope + a.d_rope, dv = a.d_v;
  const int w0 = WIDE ? 32 * wave : 0, rb = WIDE ? 0 : 32 * wave;  // the wave's first query and key in the tiles
  const int i = i0 + w0 + col;                               // this lane's query
  const int lim = a.causal ? min(nk - 1, i + off) : nk - 1;  // its last key
  const int lim_lo = a.causal ? min(nk - 1, i0 + w0 + off) : nk - 1;
  const int n_end = a.causal ? min(nk, min(i0 + kBM, nq) + off) : nk;
  const int w_end = a.causal ? min(n_end, i0 + w0 + 32 + off) : n_end;  // this wave's last key, and one

  constexpr int ES = esize<DT>();
  const char* kp = static_cast<const char*>(a.k) + (k_lo * a.k_t + kvh * a.k_h) * ES;
  const char* vp = static_cast<const char*>(a.v) + (k_lo * a.v_t + kvh * a.v_h) * ES;
  const char* rp = static_cast<const char*>(a.k_rope) + k_lo * a.kr_t * ES;
  auto issue = [&](int j0, char* t) {
    tile_load<DT, BN, KW, kThreads>(t, kp + j0 * a.k_t * ES, a.k_t, a.d_nope, rp + j0 * a.kr_t * ES, a.kr_t, a.d_rope,
                                    nk - j0, f.vec, tid);
    tile_load<DT, BN, VW, kThreads>(t + KB, vp + j0 * a.v_t * ES, a.v_t, dv, nullptr, 0, 0, nk - j0, f.vec, tid);
  };
  constexpr int R4 = 256 / pieces<DT>();  // (BN where SPREAD)
  TileLoads<DT, R4, KW, kThreads> kl;
  TileLoads<DT, R4, VW, kThreads> vl;
  auto tick = [&](int n) {
    if constexpr (SPREAD) {
      if (n < kl.LOADS)
        kl.load(n);
      else if (n < kl.LOADS + vl.LOADS)
        vl.load(n - kl.LOADS);
    }
  };
  if (n_end > 0) issue(0, smem);
  const char* qp = static_cast<const char*>(a.q) + ((q_lo + min(i, nq - 1)) * a.q_t + h * a.q_h) * ES;
  Frag<DT> qf[KC];
#pragma unroll
  for (int c = 0; c < KC; ++c) qf[c] = load8<DT>(qp, 16 * c + 8 * hh, dk, f.vec);

  floatx16 o[VT];
#pragma unroll
  for (int t = 0; t < VT; ++t)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[t][e] = 0.0f;
  float mx = -INFINITY, sum = 0.0f;
  const float sc = a.scale * kLog2e;

  for (int j0 = 0; j0 < n_end; j0 += BN) {
    char* kt = smem + (WIDE ? (j0 / BN & 1) * TB : 0);
    const char* vt = kt + KB;
    if constexpr (WIDE) {
      wait_loads();
      lds_barrier();  // everyone's loads have arrived, and everyone is done with the other tile
      char* to = smem + (~(j0 / BN) & 1) * TB;
      if constexpr (SPREAD) {
        // (after the last tile, itself again: no branch between the products)
        const int jn = j0 + BN < n_end ? j0 + BN : j0;
        kl.start(to, kp + jn * a.k_t * ES, a.k_t, a.d_nope, rp + jn * a.kr_t * ES, a.kr_t, a.d_rope, nk - jn, tid);
        vl.start(to + KB, vp + jn * a.v_t * ES, a.v_t, dv, nullptr, 0, 0, nk - jn, tid);
      } else if (j0 + BN < n_end) {
        issue(j0 + BN, to);
      }
    } else {
      if (j0 > 0) {
        lds_barrier();
        issue(j0, smem);
      }
      wait_loads();
      lds_barrier();
    }
    const int jw = j0 + rb;  // the wave's first key of the tile
    if (jw >= w_end) {
#pragma unroll
      for (int n = 0; n < kl.LOADS + vl.LOADS; ++n) tick(n);
      continue;
    }

    // S^T: groups of GK fragments, each read while the one before is multiplied
    constexpr int GK = DT == kDtF32 ? 1 : 4, NG = NB * KC / GK;
    floatx16 s[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int e = 0; e < 16; ++e) s[b][e] = 0.0f;
    Frag<DT> kf[2][GK];
#pragma unroll
    for (int g = -1; g < NG; ++g) {
      if (g + 1 < NG) {
#pragma unroll
        for (int n = 0; n < GK; ++n) {
          const int c = (g + 1) * GK + n;
          kf[(g + 1) & 1][n] = frag_rows<DT, BN>(kt, rb + 32 * (c / KC), 16 * (c % KC), lane);
        }
      }
      keep_order();
      if (g >= 0) {
        tick(g);
#pragma unroll
        for (int n = 0; n < GK; ++n) {
          const int c = g * GK + n;
          s[c / KC] = mma32<DT>(kf[g & 1][n], qf[c % KC], s[c / KC]);
        }
      }
    }
    if (jw + 32 * NB - 1 > lim_lo) {
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (jw + 32 * b + 8 * (e >> 2) + 4 * hh + (e & 3) > lim) s[b][e] = -INFINITY;
    }
    float tm = s[0][0];
#pragma unroll
    for (int e = 1; e < 16 * NB; ++e) tm = fmaxf(tm, s[e >> 4][e & 15]);
    tm = fmaxf(tm, __shfl_xor(tm, 32));
    // sums are kept relative to mx, a maximum that follows once it is 2^kSlack behind
    if (__any((tm - mx) * sc > kSlack || (mx == -INFINITY && tm > mx))) {
      const float m2 = fmaxf(mx, tm);
      const float r = m2 == -INFINITY ? 1.0f : exp2_fast((mx - m2) * sc);
      mx = m2;
      sum *= r;
#pragma unroll
      for (int t = 0; t < VT; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[t][e] *= r;
    }
    const float mz = mx == -INFINITY ? 0.0f : mx * sc;
    // O^T: slices of 16 keys
    Frag<DT> vf[2][VT];
#pragma unroll
    for (int sl = -1; sl < 2 * NB; ++sl) {
      if (sl + 1 < 2 * NB) {
#pragma unroll
        for (int t = 0; t < VT; ++t) vf[(sl + 1) & 1][t] = frag_cols<DT, BN>(vt, rb + 16 * (sl + 1), 32 * t, lane);
      }
      keep_order();
      if (sl >= 0) {
        if (sl + 1 < 2 * NB)
          tick(NG + sl);
        else  // the rest
#pragma unroll
          for (int n = NG + sl; n < kl.LOADS + vl.LOADS; ++n) tick(n);
        // the probabilities in the operands' type: one rounding each (their sum keeps 32 bits)
        float pv[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          pv[e] = exp2_fast(s[sl >> 1][8 * (sl & 1) + e] * sc - mz);
          sum += pv[e];
        }
        const Frag<DT> pf = frag_from<DT>(pv);
#pragma unroll
        for (int t = 0; t < VT; ++t) o[t] = mma32<DT>(vf[sl & 1][t], pf, o[t]);
      }
    }
  }
  if constexpr (SPREAD) wait_loads();  // none may arrive after the workgroup's end
  sum += __shfl_xor(sum, 32);
  if constexpr (!WIDE) {
    // the waves' parts of the keys: each wave joins four rows of every accumulator
    float* part = reinterpret_cast<float*>(smem);  // [wave][VT 16][64]
    float* stat = part + 4 * VT * 1024;            // [wave][32][2]
    lds_barrier();
#pragma unroll
    for (int t = 0; t < VT; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e) part[(wave * VT * 16 + t * 16 + e) * 64 + lane] = o[t][e];
    if (hh == 0) stat[(wave * 32 + col) * 2] = mx, stat[(wave * 32 + col) * 2 + 1] = sum;
    lds_barrier();
    float r[4];
    mx = -INFINITY, sum = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w) mx = fmaxf(mx, stat[(w * 32 + col) * 2]);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float m = stat[(w * 32 + col) * 2];
      r[w] = m == -INFINITY ? 0.0f : exp2_fast((m - mx) * sc);
      sum += r[w] * stat[(w * 32 + col) * 2 + 1];
    }
#pragma unroll
    for (int t = 0; t < VT; ++t)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < 4; ++w) v += r[w] * part[(w * VT * 16 + t * 16 + 4 * wave + q) * 64 + lane];
        o[t][q] = v;
      }
  }
  if (i >= nq) return;
  const float inv = mx == -INFINITY ? 0.0f : 1.0f / sum;
  const int64_t row = static_cast<int64_t>(q_lo + i) * a.H + h;
  if (a.lse != nullptr && hh == 0 && (WIDE || wave == 0))
    a.lse[row] = mx * a.scale + log2f(sum) * kLn2;  // (no key: -infinity twice; scores all NaN: sum is)
  char* op = static_cast<char*>(a.o) + row * dv * ES;
#pragma unroll
  for (int t = 0; t < VT; ++t)
#pragma unroll
    for (int e = 0; e < (WIDE ? 16 : 4); e += 4)
      store4<DT>(op, 32 * t + (WIDE ? 2 * e : 8 * wave) + 4 * hh, dv, f.ovec, o[t][e] * inv, o[t][e + 1] * inv,
                 o[t][e + 2] * inv, o[t][e + 3] * inv);
}

template <int DT, int KC, int VT, bool WIDE>
hipError_t fwd_launch_form(const FwdArgs& f, hipStream_t stream) {
  static LdsLimit limit;
  constexpr size_t tiles = WIDE ? 2 * static_cast<size_t>(tile_bytes<DT, keys_of<DT>(), 16 * KC + 32 * VT>())
                                : static_cast<size_t>(tile_bytes<DT, kSplitKeys, 16 * KC + 32 * VT>());
  constexpr size_t parts = WIDE ? 0 : 4 * VT * 4096 + 1024;
  constexpr size_t lds = tiles > parts ? tiles : parts;
  const hipError_t e = raise_lds(reinterpret_cast<const void*>(&attn_fwd<DT, KC, VT, WIDE>), lds, limit);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((attn_fwd<DT, KC, VT, WIDE>), dim3(static_cast<uint32_t>(f.n_tiles) * f.a.H), dim3(kThreads), lds,
                     stream, f);
  return hipGetLastError();
}
template <int DT, int KC, int VT>
hipError_t fwd_launch(FwdArgs& f, hipStream_t stream) {
  const int seqs = f.a.cu_q ? f.a.n_seq : 0;
  f.n_tiles = (f.a.Tq + kWideRows - 1) / kWideRows + seqs;
  // (16-bit rows that fit no 16-byte loads take the other form, whose loads go through registers.)
  // us, this form against the other.  bf16, 7B heads: 96 workgroups (256 rows) 13.2 against 11.4, 160 (512) 19.9
  // against 23.7, 192 (4 x 128) 11.4 against 17.4; 64 wide: 160 13.0 against 10.3, 192 7.4 against 7.6, 280 9.6 against
  // 16.1.  fp32, 64 wide: 272 185 against 118, 408 132 against 101, 544 233 against 212, 1056 347 against 418; 128
  // wide: 272 314 against 240, 408 315 against 359 and 167 against 210, 600 (3 x 2048) 589 against 553.  (Heads of up to 64
  // columns would cross later: one limit for all widths costs them up to a quarter in between.)
  if (wide_groups(f.a.Tq, seqs, f.a.H) >= (DT == kDtF32 ? 400 : 128) && (f.vec || DT == kDtF32)) return fwd_launch_form<DT, KC, VT, true>(f, stream);
  f.n_tiles = (f.a.Tq + 31) / 32 + seqs;
  return fwd_launch_form<DT, KC, VT, false>(f, stream);
}
template <int DT, int VT>
hipError_t fwd_kc(FwdArgs& f, hipStream_t stream) {
  const int dk = f.a.d_nope + f.a.d_rope;
  if (dk <= 64) return fwd_launch<DT, 4, VT>(f, stream);
  if (dk <= 128) return fwd_launch<DT, 8, VT>(f, stream);
  return fwd_launch<DT, 12, VT>(f, stream);
}
template <int DT>
hipError_t fwd_dt(FwdArgs& f, hipStream_t stream) {
  return f.a.d_v <= 64 ? fwd_kc<DT, 2>(f, stream) : fwd_kc<DT, 4>(f, stream);
}

}  // namespace

// whether 16-byte reads fit every operand (both passes)
bool attn_vec(const AttnArgs& a, bool backward) {
  const int es = a.dt == kDtF32 ? 4 : 2, v = 16 / es;
  auto ok = [&](const void* p, int64_t st, int64_t sh) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && st % v == 0 && sh % v == 0;
  };
  bool r = a.d_nope % 8 == 0 && a.d_rope % 8 == 0 && a.d_v % 8 == 0 && ok(a.q, a.q_t, a.q_h) && ok(a.k, a.k_t, a.k_h) &&
           ok(a.v, a.v_t, a.v_h) && (a.d_rope == 0 || ok(a.k_rope, a.kr_t, 0));
  if (backward) r = r && ok(a.d_o, a.d_v, a.d_v);
  return r;
}

bool attn_supports(int64_t dk, int64_t dv) { return dk >= 1 && dk <= 192 && dv >= 1 && dv <= 128; }

hipError_t launch_attn_forward(const AttnArgs& a, hipStream_t stream) {
  FwdArgs f{a, attn_vec(a, false), reinterpret_cast<uintptr_t>(a.o) % 16 == 0 && a.d_v % 4 == 0, 0};
  switch (a.dt) {
    case kDtF32: return fwd_dt<kDtF32>(f, stream);
    case kDtF16: return fwd_dt<kDtF16>(f, stream);
    default: return fwd_dt<kDtBF16>(f, stream);
  }
}

}  // namespace lb
