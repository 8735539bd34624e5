// Backward of the attention over expanded keys and values.
//
//   P = exp(S - lse), D = rowsum(dO (.) O), dS = P (.) (dO V^T - D)
//   dV = P^T dO, dK = scale dS^T Q_n, dK_rope = scale sum over heads dS^T Q_r, dQ = scale dS [K | K_rope]
//
// Two kernels, each forming S and dO V^T anew, so that every gradient is summed by
// one owner in a fixed order (no atomics on values): one owns 128 keys of a key head,
// holds their K and V as B operands in registers and walks the queries of all heads
// that share it; the other owns 128 queries and walks their keys.  The shared rotary
// key's gradient is summed over the key heads from fp32 partial results.
#include "attn.h"
#include "attn_common.h"

namespace lb {

namespace {

constexpr int kThreads = 256;
constexpr int kBM = 128;  // rows a workgroup owns

struct BwdArgs {
  AttnArgs a;
  int vec;              // rows may be read 16 bytes at a time
  int qvec, kvec, vvec;  // dq, dk, dv rows may be written four elements at a time
  int tiles_q, tiles_k;  // work items per head (upper bounds)
};

// f16: dS is brought to f16's normal range by a power of two of the largest |dO|
// (products of small gradients and small probabilities would fall below it)
template <int DT>
__device__ __forceinline__ float ds_factor(const float* top) {
  if constexpr (DT != kDtF16) return 1.0f;
  const float t = *top;
  if (!(t > 0.0f) || t > 1e30f) return 1.0f;
  int ex;
  frexpf(t, &ex);
  return ldexpf(1.0f, 4 - ex);  // the largest |dO| to [8, 16)
}

// D, 16 lanes a row; with f16 also the largest |dO| (a maximum: its order does not matter)
template <int DT>
__global__ void __launch_bounds__(kThreads) delta_kernel(AttnArgs a, bool vec) {
  const int64_t row = static_cast<int64_t>(blockIdx.x) * (kThreads / 16) + threadIdx.x / 16;
  float s = 0.0f, top = 0.0f;
  if (row < static_cast<int64_t>(a.Tq) * a.H) {
    const char* o = static_cast<const char*>(a.o) + row * a.d_v * esize<DT>();
    const char* d = static_cast<const char*>(a.d_o) + row * a.d_v * esize<DT>();
    for (int c = 8 * (threadIdx.x & 15); c < a.d_v; c += 128) {
      const Frag<DT> x = load8<DT>(o, c, a.d_v, vec), y = load8<DT>(d, c, a.d_v, vec);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float v = frag_elem<DT>(y, e);
        s += frag_elem<DT>(x, e) * v;
        top = fmaxf(top, fabsf(v));
      }
    }
  }
#pragma unroll
  for (int m = 8; m > 0; m >>= 1) s += __shfl_xor(s, m);
  if ((threadIdx.x & 15) == 0 && row < static_cast<int64_t>(a.Tq) * a.H) a.delta[row] = s;
  if constexpr (DT == kDtF16) {
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) top = fmaxf(top, __shfl_xor(top, m));
    if ((threadIdx.x & 63) == 0 && top > 0.0f)
      __hip_atomic_fetch_max(reinterpret_cast<uint32_t*>(a.top), __float_as_uint(top), __ATOMIC_RELAXED,
                             __HIP_MEMORY_SCOPE_AGENT);
  }
}

// keys: dK, dV
template <int DT, int KC, int VT>
__global__ void __launch_bounds__(kThreads, 1) attn_bwd_keys(BwdArgs f) {
  constexpr int BQ = DT == kDtF32 ? 32 : 64;  // queries of a step
  constexpr int KW = 16 * KC, VW = 32 * VT, KT = KC / 2;
  constexpr int KS = tile_stride<DT>(KW), VS = tile_stride<DT>(VW);
  constexpr int ES = esize<DT>();
  extern __shared__ __attribute__((aligned(16))) char smem[];
  char* qt = smem;
  char* dt = smem + BQ * KS;
  float* st_lse = reinterpret_cast<float*>(smem + BQ * (KS + VS));
  float* st_del = st_lse + BQ;
  const AttnArgs& a = f.a;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hh = lane >> 5, col = lane & 31;
  const int kvh = blockIdx.x % a.Hk, G = a.H / a.Hk;
  int seq, tile;
  if (!find_tile(a.cu_k, a.n_seq, a.Tk, kBM, blockIdx.x / a.Hk, lane, seq, tile)) return;
  int q_lo, q_hi, k_lo, k_hi;
  seq_range(a.cu_q, seq, a.Tq, q_lo, q_hi);
  seq_range(a.cu_k, seq, a.Tk, k_lo, k_hi);
  const int nq = q_hi - q_lo, nk = k_hi - k_lo, off = nk - nq;
  const int j0 = tile * kBM, j = j0 + 32 * wave + col;  // this lane's key
  const int dk = a.d_nope + a.d_rope, dv = a.d_v;
  const float sc = a.scale * kLog2e;
  const float fac = ds_factor<DT>(a.top);

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

  const int i_begin = a.causal ? max(0, j0 - off) / BQ * BQ : 0;
  const int n_it = max(0, (nq - i_begin + BQ - 1) / BQ);
  constexpr int QL = BQ * KW / 8 / kThreads, OL = BQ * VW / 8 / kThreads;
  static_assert(QL * kThreads * 8 == BQ * KW && OL * kThreads * 8 == BQ * VW, "whole groups");
  Frag<DT> qr[QL], dr_[OL];
  float lr = 0.0f, de = 0.0f;
  auto fetch = [&](int it) {  // step it of G * n_it: head it / n_it of the group
    const int g = it / n_it, i0 = i_begin + (it - g * n_it) * BQ, h = kvh * G + g;
#pragma unroll
    for (int n = 0; n < QL; ++n) {
      const int u = tid + n * kThreads, row = u / (KW / 8), c = 8 * (u % (KW / 8));
      qr[n] = i0 + row < nq
                  ? load8<DT>(static_cast<const char*>(a.q) + ((q_lo + i0 + row) * a.q_t + h * a.q_h) * ES, c, dk, f.vec)
                  : frag_zero<DT>();
    }
#pragma unroll
    for (int n = 0; n < OL; ++n) {
      const int u = tid + n * kThreads, row = u / (VW / 8), c = 8 * (u % (VW / 8));
      dr_[n] = i0 + row < nq ? load8<DT>(static_cast<const char*>(a.d_o) +
                                             (static_cast<int64_t>(q_lo + i0 + row) * a.H + h) * dv * ES,
                                         c, dv, f.vec)
                             : frag_zero<DT>();
    }
    if (tid < BQ) {
      const bool ok = i0 + tid < nq;
      const int64_t r = static_cast<int64_t>(q_lo + min(i0 + tid, nq - 1)) * a.H + h;
      const float l = a.lse[r];
      // rows past the end and rows that see no key get probability 0
      lr = ok && l != -INFINITY ? l * kLog2e : INFINITY;
      de = ok ? a.delta[r] : 0.0f;
    }
  };
  const int total = G * n_it;
  if (total > 0) fetch(0);
  for (int it = 0; it < total; ++it) {
    __syncthreads();
#pragma unroll
    for (int n = 0; n < QL; ++n) {
      const int u = tid + n * kThreads;
      tile_put<DT>(qt, KS, u / (KW / 8), 8 * (u % (KW / 8)), qr[n]);
    }
#pragma unroll
    for (int n = 0; n < OL; ++n) {
      const int u = tid + n * kThreads;
      tile_put<DT>(dt, VS, u / (VW / 8), 8 * (u % (VW / 8)), dr_[n]);
    }
    if (tid < BQ) st_lse[tid] = lr, st_del[tid] = de;
    __syncthreads();
    const int i0 = i_begin + it % n_it * BQ;
    if (it + 1 < total) fetch(it + 1);
#pragma unroll
    for (int b = 0; b < BQ / 32; ++b) {
      floatx16 s, dp;
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = 0.0f, dp[e] = 0.0f;
#pragma unroll
      for (int c = 0; c < KC; ++c) s = mma32<DT>(frag_rows<DT>(qt, KS, 32 * b, 16 * c, lane), kf[c], s);
#pragma unroll
      for (int c = 0; c < 2 * VT; ++c) dp = mma32<DT>(frag_rows<DT>(dt, VS, 32 * b, 16 * c, lane), vf[c], dp);
      const bool mask = a.causal && i0 + 32 * b + off < j0 + 32 * wave + 31;
#pragma unroll
      for (int e = 0; e < 16; e += 4) {
        const int row = 32 * b + 2 * e + 4 * hh;
        const float4 l4 = *reinterpret_cast<const float4*>(st_lse + row);
        const float4 d4 = *reinterpret_cast<const float4*>(st_del + row);
        const float lv[4] = {l4.x, l4.y, l4.z, l4.w}, dl[4] = {d4.x, d4.y, d4.z, d4.w};
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          float p = exp2_fast(s[e + q] * sc - lv[q]);
          if (mask && i0 + row + q + off < j) p = 0.0f;
          s[e + q] = p;
          dp[e + q] = p == 0.0f ? 0.0f : p * (dp[e + q] - dl[q]) * fac;
        }
      }
#pragma unroll
      for (int sl = 0; sl < 2; ++sl) {
        float x[8], y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = s[8 * sl + e], y[e] = dp[8 * sl + e];
        const Frag<DT> pf = frag_from<DT>(x), df = frag_from<DT>(y);
#pragma unroll
        for (int t = 0; t < VT; ++t)
          gv[t] = mma32<DT>(frag_cols<DT>(dt, VS, 32 * b + 16 * sl, 32 * t, lane), pf, gv[t]);
#pragma unroll
        for (int t = 0; t < KT; ++t)
          gk[t] = mma32<DT>(frag_cols<DT>(qt, KS, 32 * b + 16 * sl, 32 * t, lane), df, gk[t]);
      }
    }
  }
  if (j >= nk) return;
  const int64_t t = k_lo + j;
  const float ks = a.scale / fac;
  char* gkp = static_cast<char*>(a.dk) + (t * a.dk_t + kvh * a.dk_h) * ES;
  char* gvp = static_cast<char*>(a.dv) + (t * a.dv_t + kvh * a.dv_h) * ES;
  float* grp = a.dkr_part + (static_cast<int64_t>(kvh) * a.Tk + t) * a.d_rope;
#pragma unroll
  for (int n = 0; n < VT; ++n)
#pragma unroll
    for (int e = 0; e < 16; e += 4)
      store4<DT>(gvp, 32 * n + 2 * e + 4 * hh, dv, f.vvec, gv[n][e], gv[n][e + 1], gv[n][e + 2], gv[n][e + 3]);
#pragma unroll
  for (int n = 0; n < KT; ++n)
#pragma unroll
    for (int e = 0; e < 16; e += 4) {
      const int c = 32 * n + 2 * e + 4 * hh;
      store4<DT>(gkp, c, a.d_nope, f.kvec, gk[n][e] * ks, gk[n][e + 1] * ks, gk[n][e + 2] * ks, gk[n][e + 3] * ks);
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (c + q >= a.d_nope && c + q < dk) grp[c + q - a.d_nope] = gk[n][e + q] * ks;
    }
}

// queries: dQ
template <int DT, int KC, int VT>
__global__ void __launch_bounds__(kThreads, 1) attn_bwd_queries(BwdArgs f) {
  constexpr int BN = DT == kDtF32 ? 32 : 64;  // keys of a step
  constexpr int KW = 16 * KC, VW = 32 * VT, KT = KC / 2;
  constexpr int KS = tile_stride<DT>(KW), VS = tile_stride<DT>(VW);
  constexpr int ES = esize<DT>();
  extern __shared__ __attribute__((aligned(16))) char smem[];
  char* kt = smem;
  char* vt = smem + BN * KS;
  const AttnArgs& a = f.a;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hh = lane >> 5, col = lane & 31;
  const int id = blockIdx.x, hi_ = id % a.H, G = a.H / a.Hk;
  const int kvh = hi_ % a.Hk, h = kvh * G + hi_ / a.Hk;
  int seq, tile;
  if (!find_tile(a.cu_q, a.n_seq, a.Tq, kBM, id / a.H, lane, seq, tile)) return;
  int q_lo, q_hi, k_lo, k_hi;
  seq_range(a.cu_q, seq, a.Tq, q_lo, q_hi);
  seq_range(a.cu_k, seq, a.Tk, k_lo, k_hi);
  const int nq = q_hi - q_lo, nk = k_hi - k_lo, off = nk - nq;
  tile = (nq + kBM - 1) / kBM - 1 - tile;  // the longest first
  const int i0 = tile * kBM, i = i0 + 32 * wave + col;
  const int dk = a.d_nope + a.d_rope, dv = a.d_v;
  const int lim = a.causal ? min(nk - 1, i + off) : nk - 1;
  const int lim_lo = a.causal ? min(nk - 1, i0 + 32 * wave + off) : nk - 1;
  const int n_end = a.causal ? min(nk, min(i0 + kBM, nq) + off) : nk;
  const float sc = a.scale * kLog2e;
  const float fac = ds_factor<DT>(a.top);

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
  const float l = a.lse[row], del = a.delta[row];
  const float l2 = l == -INFINITY ? INFINITY : l * kLog2e;
  floatx16 gq[KT];
#pragma unroll
  for (int t = 0; t < KT; ++t)
#pragma unroll
    for (int e = 0; e < 16; ++e) gq[t][e] = 0.0f;

  constexpr int KL = BN * KW / 8 / kThreads, VL = BN * VW / 8 / kThreads;
  static_assert(KL * kThreads * 8 == BN * KW && VL * kThreads * 8 == BN * VW, "whole groups");
  Frag<DT> kr[KL], vr[VL];
  const char* kp = static_cast<const char*>(a.k) + kvh * a.k_h * ES;
  const char* vp = static_cast<const char*>(a.v) + kvh * a.v_h * ES;
  const char* rp = static_cast<const char*>(a.k_rope);
  auto fetch = [&](int j0) {
#pragma unroll
    for (int n = 0; n < KL; ++n) {
      const int u = tid + n * kThreads, r = u / (KW / 8), c = 8 * (u % (KW / 8));
      const int64_t t = k_lo + j0 + r;
      kr[n] = j0 + r < nk ? load8_joined<DT>(kp + t * a.k_t * ES, a.d_nope, rp + t * a.kr_t * ES, a.d_rope, c, f.vec)
                          : frag_zero<DT>();
    }
#pragma unroll
    for (int n = 0; n < VL; ++n) {
      const int u = tid + n * kThreads, r = u / (VW / 8), c = 8 * (u % (VW / 8));
      vr[n] = j0 + r < nk ? load8<DT>(vp + (k_lo + j0 + r) * a.v_t * ES, c, dv, f.vec) : frag_zero<DT>();
    }
  };
  if (n_end > 0) fetch(0);
  for (int j0 = 0; j0 < n_end; j0 += BN) {
    __syncthreads();
#pragma unroll
    for (int n = 0; n < KL; ++n) {
      const int u = tid + n * kThreads;
      tile_put<DT>(kt, KS, u / (KW / 8), 8 * (u % (KW / 8)), kr[n]);
    }
#pragma unroll
    for (int n = 0; n < VL; ++n) {
      const int u = tid + n * kThreads;
      tile_put<DT>(vt, VS, u / (VW / 8), 8 * (u % (VW / 8)), vr[n]);
    }
    __syncthreads();
    if (j0 + BN < n_end) fetch(j0 + BN);
#pragma unroll
    for (int b = 0; b < BN / 32; ++b) {
      floatx16 s, dp;
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = 0.0f, dp[e] = 0.0f;
#pragma unroll
      for (int c = 0; c < KC; ++c) s = mma32<DT>(frag_rows<DT>(kt, KS, 32 * b, 16 * c, lane), qf[c], s);
#pragma unroll
      for (int c = 0; c < 2 * VT; ++c) dp = mma32<DT>(frag_rows<DT>(vt, VS, 32 * b, 16 * c, lane), df[c], dp);
      const bool mask = j0 + 32 * b + 31 > lim_lo;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        float p = exp2_fast(s[e] * sc - l2);
        if (mask && j0 + 32 * b + 8 * (e >> 2) + 4 * hh + (e & 3) > lim) p = 0.0f;
        dp[e] = p == 0.0f ? 0.0f : p * (dp[e] - del) * fac;
      }
#pragma unroll
      for (int sl = 0; sl < 2; ++sl) {
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = dp[8 * sl + e];
        const Frag<DT> sf = frag_from<DT>(y);
#pragma unroll
        for (int t = 0; t < KT; ++t)
          gq[t] = mma32<DT>(frag_cols<DT>(kt, KS, 32 * b + 16 * sl, 32 * t, lane), sf, gq[t]);
      }
    }
  }
  if (i >= nq) return;
  const float qs = a.scale / fac;
  char* gp = static_cast<char*>(a.dq) + row * dk * ES;
#pragma unroll
  for (int n = 0; n < KT; ++n)
#pragma unroll
    for (int e = 0; e < 16; e += 4)
      store4<DT>(gp, 32 * n + 2 * e + 4 * hh, dk, f.qvec, gq[n][e] * qs, gq[n][e + 1] * qs, gq[n][e + 2] * qs,
                 gq[n][e + 3] * qs);
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

template <int DT, int KC, int VT>
hipError_t bwd_launch(const BwdArgs& f, hipStream_t stream) {
  constexpr int B = DT == kDtF32 ? 32 : 64;
  constexpr size_t tiles = static_cast<size_t>(B) * (tile_stride<DT>(16 * KC) + tile_stride<DT>(32 * VT));
  static LdsLimit lk, lq;
  hipError_t e = raise_lds(reinterpret_cast<const void*>(&attn_bwd_keys<DT, KC, VT>), tiles + 8 * B, lk);
  if (e != hipSuccess) return e;
  e = raise_lds(reinterpret_cast<const void*>(&attn_bwd_queries<DT, KC, VT>), tiles, lq);
  if (e != hipSuccess) return e;
  if (f.tiles_k > 0) {
    hipLaunchKernelGGL((attn_bwd_keys<DT, KC, VT>), dim3(static_cast<uint32_t>(f.tiles_k) * f.a.Hk), dim3(kThreads),
                       tiles + 8 * B, stream, f);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (f.tiles_q > 0) {
    hipLaunchKernelGGL((attn_bwd_queries<DT, KC, VT>), dim3(static_cast<uint32_t>(f.tiles_q) * f.a.H), dim3(kThreads),
                       tiles, stream, f);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
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
  const AttnArgs& a = f.a;
  if constexpr (DT == kDtF16) {
    const hipError_t e = launch_zero_elems(a.top, 1, kDtF32, stream);
    if (e != hipSuccess) return e;
  }
  if (a.Tq > 0) {
    const bool vec = f.vec && reinterpret_cast<uintptr_t>(a.o) % 16 == 0;
    const int64_t rows = static_cast<int64_t>(a.Tq) * a.H;
    hipLaunchKernelGGL((delta_kernel<DT>), dim3(static_cast<uint32_t>((rows + 15) / 16)), dim3(kThreads), 0, stream, a,
                       vec);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return a.d_v <= 64 ? bwd_kc<DT, 2>(f, stream) : bwd_kc<DT, 4>(f, stream);
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
  f.tiles_q = a.Tq == 0 ? 0 : (a.Tq + kBM - 1) / kBM + (a.cu_q ? a.n_seq : 0);
  f.tiles_k = a.Tk == 0 ? 0 : (a.Tk + kBM - 1) / kBM + (a.cu_k ? a.n_seq : 0);
  switch (a.dt) {
    case kDtF32: return bwd_dt<kDtF32>(f, stream);
    case kDtF16: return bwd_dt<kDtF16>(f, stream);
    default: return bwd_dt<kDtBF16>(f, stream);
  }
}

}  // namespace lb
