// Attention read from the paged latent cache, the up-projection absorbed.
//
// A token's keys and values are K = U_k w and V = U_v w of its one latent w (2 r
// values), so with q' = U_k^T (h_k (.) q) the scores are q' . w + q_rope . k_rope and
// the output is h_v (.) U_v (sum_t a_t w_t): every query head reads the same cache
// rows, once, and nothing is expanded.  Three launches:
//
//   absorb   q' of every (token, head), with the rotated rotary part behind it and the
//            softmax scale folded into a factor per row, cut into terms of the cache's
//            type: TQ terms, so that q' (not a value of that type) enters the scores
//            with 16 bits or more.
//   split    the cache in one pass with a running maximum and sum.  A workgroup takes
//            an equal share of all sequences' tiles, whatever their lengths.
//   join     the partial results of a row joined, then h (.) U_v of the sum.
//
// split is bound by the cache's bytes: a row of 2 r + d_rope values serves 32 query
// rows (a model's heads) as the columns of 32 x 32 matrix-core tiles, where a column's
// statistics are two lanes' own and the probabilities go from one product into the next in
// their registers.  A token wave takes 32 tokens of a step for whole rows of up to 12 units
// (32 columns), with no wave waiting for another until the sums are added at the end;
// wider rows are cut into four waves' columns, whose scores are added through LDS each step.
//
// Measured (7B heads, 2 r + d_rope = 288, bf16, us of absorb + split + join): 32 sequences of 2048 to
// 16384 tokens 7.8 + 38.3 + 10.8 (129 MB: 3.3 TB/s over all of split, of which the first loads
// and the last sums are 11 us, and about what a large copy moves, 5.1, in between); one of 4096 tokens 5.8 + 12.0 + 7.0, a
// chain of dependent loads; 1440 columns, 8 sequences of 1000 to 4000: 9.0 + 36 + 17.8.
#include "attn.h"
#include "attn_common.h"
#include "latent_map.h"

namespace lb {

namespace {

constexpr size_t kLdsMax = 163840;

// ---------------------------------------------------------------------------
// plan (host)
// ---------------------------------------------------------------------------
struct LatPlan {
  int nu;      // units (32 columns) of a cache row
  int vu;      // units that hold latents
  int ncw;     // column waves: each holds nuw units of the row
  int ntw;     // token waves: each takes 32 tokens of a step
  int nuw;     // units a wave holds
  int upw;     // ... and the kernel's register class for them
  int stages;  // tiles in LDS per wave
  int tpt;     // tokens of a tile (32, or 16 where 32 do not fit)
  int step;    // tokens of a step: tpt ntw
  int tile_bytes, xchg_bytes;
  size_t lds;
};

// LDS of ntw waves' sums (rows padded by 16 bytes) and statistics
__host__ size_t sums_bytes(int ntw, int vu) { return static_cast<size_t>(ntw) * kCols * ((vu * 32 + 4) * 4 + 8); }

__host__ LatPlan lat_plan(int r, int d_rope, int es) {
  LatPlan p{};
  p.nu = latent_row(r, d_rope) / kRowUnit;
  p.vu = (2 * r + 31) / 32;
  // a wave's registers hold 12 units (q' and the sums); wider rows go to four waves
  p.ncw = p.nu <= 12 ? 1 : 4;
  p.nuw = (p.nu + p.ncw - 1) / p.ncw;
  p.upw = p.nuw <= 4 ? 4 : p.ncw == 1 ? p.nuw : (p.nuw + 1) / 2 * 2;
  p.tpt = 32;
  p.tile_bytes = p.nuw * 32 * 32 * es;
  if (p.ncw == 1) {
    // as many token waves as leave room for two tiles each, and for their sums
    p.ntw = 8 * static_cast<size_t>(p.tile_bytes) <= kLdsMax && sums_bytes(4, p.vu) <= kLdsMax ? 4 : 2;
    p.stages = 2 * static_cast<size_t>(p.ntw) * p.tile_bytes <= kLdsMax ? 2 : 1;
  } else {
    p.ntw = 1;
    p.xchg_bytes = 2 * p.ncw * 4096;  // partial scores, two buffers
    if (static_cast<size_t>(p.ncw) * p.tile_bytes + p.xchg_bytes > kLdsMax) p.tpt = 16, p.tile_bytes /= 2;
    p.stages = 2 * static_cast<size_t>(p.ncw) * p.tile_bytes + p.xchg_bytes <= kLdsMax ? 2 : 1;
  }
  p.step = p.tpt * p.ntw;
  const int nw = p.ncw * p.ntw;
  p.lds = static_cast<size_t>(nw) * p.stages * p.tile_bytes + p.xchg_bytes;
  if (p.ncw == 1) {
    // the token waves' sums are added through the same memory
    const size_t red = sums_bytes(p.ntw, p.vu);
    if (red > p.lds) p.lds = red;
  }
  return p;
}

// terms of q' and of the probabilities by the cache's type and the activations'
constexpr int terms_q(int cd, bool f32) { return cd == kDtF32 ? 1 : (cd == kDtBF16 && f32 ? 3 : 2); }
constexpr int terms_p(int cd, int act) {
  return cd == kDtF32 || act == kDtBF16 || (act == kDtF16 && cd == kDtF16) ? 1 : (cd == kDtBF16 && act == kDtF32 ? 3 : 2);
}

struct LatWs {
  size_t q_off, qs_off, ml_off, o_off, bytes;
};
// Sized for every type pair: three terms of 2 bytes cover two of 2 and one of 4.
__host__ LatWs lat_ws(int64_t T, int64_t n_seq, int64_t H, int r, int d_rope) {
  LatWs w{};
  const int64_t row = latent_row(r, d_rope), ow = (2 * r + 31) / 32 * 32;
  const int64_t slots = lat_slots(T, n_seq, H);
  auto up = [](size_t b) { return (b + 255) / 256 * 256; };
  w.qs_off = up(static_cast<size_t>((T * H + kCols - 1) / kCols * kCols * row) * 6);
  w.ml_off = w.qs_off + up(static_cast<size_t>(T * H) * 4);
  w.o_off = w.ml_off + up(static_cast<size_t>(slots) * kCols * 8);
  w.bytes = w.o_off + up(static_cast<size_t>(slots) * kCols * ow * 4);
  return w;
}

// ---------------------------------------------------------------------------
// work map: sequence b has ceil(nq_b H / 32) items of ceil(len_b / step) steps each;
// all W steps in a row are dealt to G workgroups (latent_map.h).
// ---------------------------------------------------------------------------
struct SeqWork {
  int q0, nq;       // first token, tokens
  int first;        // the first one's position (below 0: it has none)
  int len;          // cached tokens, within the page table
  int items, steps;  // items, steps of each
};
// sequence b, whose tokens are rows q0 .. q0 + nq - 1
__device__ __forceinline__ SeqWork seq_work(const CacheArgs& c, int b, int q0, int nq, int H, int step) {
  SeqWork s;
  s.q0 = q0, s.nq = nq;
  const int n = max(0, c.lens[b]);
  // as lb_latent_append places them: row t at lens[b] - (cu[b + 1] - t)
  s.first = nq > 0 ? n - (c.cu[b + 1] - q0) : 0;
  s.len = min(n, c.max_pages * c.page_size);
  s.items = (s.nq * H + kCols - 1) / kCols;
  // step is 16, 32, 64 or 128
  s.steps = (s.len + step - 1) >> (31 - __builtin_clz(step));
  return s;
}
__device__ __forceinline__ SeqWork seq_lane(const SeqWork& s, int k) {
  SeqWork r;
  r.q0 = __builtin_amdgcn_readlane(s.q0, k);
  r.nq = __builtin_amdgcn_readlane(s.nq, k);
  r.first = __builtin_amdgcn_readlane(s.first, k);
  r.len = __builtin_amdgcn_readlane(s.len, k);
  r.items = __builtin_amdgcn_readlane(s.items, k);
  r.steps = __builtin_amdgcn_readlane(s.steps, k);
  return r;
}

// The work map of a wave.  Its lanes hold 64 sequences at a time (the arrays are read
// once for batches of up to 64).
struct WorkMap {
  const CacheArgs& c;
  int T, H, step, lane;
  int block = -1;  // the 64 sequences held
  SeqWork s;
  int ws, is;      // inclusive sums of steps and items over them
  int end;         // the row behind the last of them
  // before: the row behind the sequences before b0 (of the first 64: what cu says)
  __device__ __forceinline__ void hold(int b0, int before) {
    if (b0 == block) return;
    block = b0;
    const int b = b0 + lane;
    if (b0 == 0) before = rows_end(0, c.cu[0], T);
    int hi = rows_end(before, b < c.n_seq ? c.cu[b + 1] : 0, T), lo = before;
    if (c.n_seq > 1) {
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) hi = max(hi, __shfl_up(hi, d));  // (a lane below d gets its own)
      lo = __shfl_up(hi, 1);
      if (lane == 0) lo = before;
    }
    end = __builtin_amdgcn_readlane(hi, 63);
    s = SeqWork{0, 0, 0, 0, 0, 0};
    if (b < c.n_seq) s = seq_work(c, b, lo, hi - lo, H, step);
    ws = s.items * s.steps, is = s.items;
    if (c.n_seq > 1) {
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(ws, d), q = __shfl_up(is, d);
        if (lane >= d) ws += o, is += q;
      }
    }
  }
  __device__ __forceinline__ int last() const { return min(63, c.n_seq - 1 - block); }
  __device__ __forceinline__ int total() {
    int w = 0, before = 0;
    for (int b0 = 0; b0 < c.n_seq; b0 += 64) {
      hold(b0, before);
      before = end;
      w += __builtin_amdgcn_readlane(ws, last());
    }
    return w;
  }
  // The sequence whose steps contain number x (by_step) or whose tokens contain row x:
  // its index (-1: none), its work, and the steps and items before it.
  __device__ __forceinline__ int find(bool by_step, int x, SeqWork& out, int& sb, int& ib) {
    sb = 0, ib = 0;
    int before = 0;
    for (int b0 = 0; b0 < c.n_seq; b0 += 64) {
      hold(b0, before);
      before = end;
      const uint64_t m = __ballot(b0 + lane < c.n_seq && (by_step ? sb + ws > x : s.q0 <= x && x < s.q0 + s.nq));
      if (m != 0) {
        const int k = __builtin_ctzll(m);
        out = seq_lane(s, k);
        sb += __builtin_amdgcn_readlane(ws, k) - out.items * out.steps;
        ib += __builtin_amdgcn_readlane(is, k) - out.items;
        return b0 + k;
      }
      sb += __builtin_amdgcn_readlane(ws, last());
      ib += __builtin_amdgcn_readlane(is, last());
    }
    return -1;
  }
};
// n / d for 0 <= n < 2^31 by a multiplication: m = ceil(2^(31 + l) / d), l = ceil(log2 d) (m = 0: d = 1)
struct Divisor {
  uint32_t m, shift;
  int d;
};
__host__ Divisor divisor(int d) {
  int l = 0;
  while ((int64_t(1) << l) < d) ++l;
  if (l == 0) return Divisor{0, 0, 1};
  return Divisor{static_cast<uint32_t>(((uint64_t(1) << (31 + l)) + d - 1) / d), static_cast<uint32_t>(l - 1), d};
}
__device__ __forceinline__ int quotient(int n, const Divisor& d) {
  return d.m == 0 ? n : static_cast<int>(__umulhi(static_cast<uint32_t>(n), d.m) >> d.shift);
}

// The words of one word column (latents 32 kb ..) of a packed matrix: full words, or
// the tail plane's 16- or 32-bit ones.
struct WordColumn {
  const char* p;
  bool half;  // 16-bit words
};
__device__ __forceinline__ WordColumn word_column(const void* U, int n_out, int r, int kb) {
  const int nb = r >> 5, w = r & 31;
  return WordColumn{static_cast<const char*>(U) + static_cast<int64_t>(4) * min(kb, nb) * n_out, kb >= nb && w <= 16};
}
__device__ __forceinline__ uint32_t word_at(const WordColumn& c, int o) {
  return c.half ? reinterpret_cast<const uint16_t*>(c.p)[o] : reinterpret_cast<const uint32_t*>(c.p)[o];
}

// x[8] as N terms of type CD, each the rounding of what the previous ones left
template <int CD, int N>
__device__ __forceinline__ void to_terms(float (&x)[8], Frag<CD> (&f)[N]) {
#pragma unroll
  for (int n = 0; n < N; ++n) {
    f[n] = frag_from<CD>(x);
    if (n + 1 < N) {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] -= frag_elem<CD>(f[n], e);
    }
  }
}

// x rounded to type CD, as fp32
template <int CD>
__device__ __forceinline__ float rounded(float x) {
  if constexpr (CD == kDtF32) return x;
  if constexpr (CD == kDtBF16) return bf16_bits_to_f32(f32_to_bf16_bits(x));
  asm volatile("" : "+v"(x));
  return __half2float(__float2half_rn(x));
}

// ---------------------------------------------------------------------------
// absorb
// ---------------------------------------------------------------------------
constexpr int kMaxHead = 256;    // widths of a head
constexpr int kRopeHeads = 8;    // heads of a rotary workgroup
constexpr int kAbsTokens = 32;   // tokens of a tile

// q' is kept as the B operands that split reads: for every 32 rows m = t H + h, term and
// 16-byte piece of the row's columns, the 32 rows' pieces next to each other.  Bytes from
// the start to column col of term n of row m:
template <int CD, int TQ>
__device__ __forceinline__ int64_t q_offset(int64_t m, int n, int col, int row) {
  constexpr int EP = 16 / esize<CD>();  // elements of a piece
  return (((m >> 5) * TQ + n) * (row / EP) + col / EP) * 512 + (m & 31) * 16 + col % EP * esize<CD>();
}

// With an f16 cache q' is brought into f16's range by a power of two per row, which takes a
// bound on the row's values (order-free maxima, so that every workgroup finds the same one) to
// 2^13 .. 2^14: two terms then hold 22 bits of values down to 2^-17 of the bound and 16 down to 2^-23, so
// that a small rotary part beside large latents keeps its digits.  top: the largest |h (.) q|, rope: of the rotary part.
__device__ __forceinline__ float row_factor(float top, float rope, int dn) {
  const float b = fmaxf(top * static_cast<float>(dn), 1.5f * rope);
  if (!(b > 0.0f) || b > 1e38f) return 1.0f;
  int ex;
  frexpf(b, &ex);
  return ldexpf(1.0f, max(-120, min(120, 14 - ex)));
}

// The first H 2 nkb tiles workgroups (a wave each) take 32 latents of a path (one packed
// word per output row) of one head for 32 tokens: q' = (h (.) q) U as 32 x 32 tiles,
// h (.) q cut into three bf16 terms, the signs as bf16 +-1, so every product is exact.
// The others take the rotary part (and the row's zeros) of one token and kRopeHeads heads.
template <int DT, int SC, int CD, int TQ>
__global__ void __launch_bounds__(64) absorb_kernel(LatentAttnArgs a, char* qout, float* qsc, int nkb, int n_mma,
                                                   bool vec) {
  const int lane = threadIdx.x, hh = lane >> 5;
  const CacheArgs& c = a.c;
  const int r = c.r, dn = a.d_nope, dr = c.d_rope, row = c.row, G = a.H / a.Hk;
  if (static_cast<int>(blockIdx.x) < n_mma) {
    const int u = blockIdx.x % (2 * nkb), hb = blockIdx.x / (2 * nkb), h = hb % a.H, t0 = hb / a.H * kAbsTokens;
    const int p = u >= nkb, kb = u - p * nkb, i0 = h / G * dn;
    const WordColumn v = word_column(a.U[p], a.Hk * (dn + a.d_v), r, kb);
    const int t = min(t0 + (lane & 31), a.T - 1), bit = lane & 31;
    const char* q = static_cast<const char*>(a.q) + (t * a.q_t + h * a.q_h) * esize<DT>();
    floatx16 acc;
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[e] = 0.0f;
    float top = 0.0f, rope = 0.0f;
    // 64 inputs at a time: all their loads first
    for (int c0 = 0; c0 < dn; c0 += 64) {
      uint32_t w[4][8];
      Frag<DT> qv[4];
      Frag<SC> hv[4], h2[4];
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        const int i = c0 + 16 * n + 8 * hh;
        qv[n] = load8<DT>(q, i, dn, vec);
        hv[n] = load8<SC>(static_cast<const char*>(a.h[p]) + i0 * esize<SC>(), i, dn, vec);
        if constexpr (CD == kDtF16)
          h2[n] = load8<SC>(static_cast<const char*>(a.h[1 - p]) + i0 * esize<SC>(), i, dn, vec);
      }
      if (v.half) {
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
          for (int e = 0; e < 8; ++e)
            w[n][e] = reinterpret_cast<const uint16_t*>(v.p)[i0 + min(c0 + 16 * n + 8 * hh + e, dn - 1)];
      } else if (c0 + 64 <= dn) {
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
          for (int e = 0; e < 8; ++e) w[n][e] = reinterpret_cast<const uint32_t*>(v.p)[i0 + c0 + 16 * n + 8 * hh + e];
      } else {
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
          for (int e = 0; e < 8; ++e)
            w[n][e] = reinterpret_cast<const uint32_t*>(v.p)[i0 + min(c0 + 16 * n + 8 * hh + e, dn - 1)];
      }
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        float x[8];
        u32x4 s;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float qe = frag_elem<DT>(qv[n], e);
          x[e] = qe * frag_elem<SC>(hv[n], e);
          if constexpr (CD == kDtF16) top = fmaxf(top, fmaxf(fabsf(x[e]), fabsf(qe * frag_elem<SC>(h2[n], e))));
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
          s[e] = 0x3f803f80u ^ (((w[n][2 * e] >> bit) & 1u) << 15) ^ ((w[n][2 * e + 1] >> bit) << 31);
        Frag<kDtBF16> sf, xf[3];
        sf.v[0] = s;
        to_terms<kDtBF16, 3>(x, xf);
#pragma unroll
        for (int m = 0; m < 3; ++m) acc = mma32<kDtBF16>(xf[m], sf, acc);
      }
    }
    float f = 1.0f;
    if constexpr (CD == kDtF16) {
      for (int i = hh; i < dr; i += 2) rope = fmaxf(rope, fabsf(ld<DT>(q, dn + i)));
      top = fmaxf(top, __shfl_xor(top, 32));
      rope = fmaxf(rope, __shfl_xor(rope, 32));
      f = row_factor(top, rope, dn);
    }
    const int k = 32 * kb + bit;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int tt = 8 * (e >> 2) + 4 * hh + (e & 3);
      float x = acc[e];
      if constexpr (CD == kDtF16) x *= __shfl(f, tt);
      if (t0 + tt < a.T && k < r) {
        const int64_t m = static_cast<int64_t>(t0 + tt) * a.H + h;
#pragma unroll
        for (int n = 0; n < TQ; ++n) {
          const float y = rounded<CD>(x);
          st<CD>(qout + q_offset<CD, TQ>(m, n, p * r + k, row), 0, y);
          x -= y;
        }
      }
    }
    return;
  }
  const int nh = (a.H + kRopeHeads - 1) / kRopeHeads, id = blockIdx.x - n_mma;
  const int t = id / nh, h0 = id % nh * kRopeHeads, h1 = min(a.H, h0 + kRopeHeads);
  int pos = 0;
  if (dr > 0 && a.freqs != nullptr) {
    WorkMap map{c, a.T, a.H, 32, lane};
    SeqWork s;
    int sb, ib;
    if (map.find(false, t, s, sb, ib) >= 0) pos = max(0, s.first + (t - s.q0));
  }
  float f = 1.0f;  // of head h0 + lane / 8
  if constexpr (CD == kDtF16) {
    const int h = min(h0 + lane / 8, a.H - 1), i0 = h / G * dn;
    const char* q = static_cast<const char*>(a.q) + (t * a.q_t + h * a.q_h) * esize<DT>();
    float top = 0.0f, rope = 0.0f;
    for (int i = 8 * (lane & 7); i < dn; i += 64) {
      const Frag<DT> x = load8<DT>(q, i, dn, vec);
      const Frag<SC> y = load8<SC>(static_cast<const char*>(a.h[0]) + i0 * esize<SC>(), i, dn, vec);
      const Frag<SC> z = load8<SC>(static_cast<const char*>(a.h[1]) + i0 * esize<SC>(), i, dn, vec);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float qe = frag_elem<DT>(x, e);
        top = fmaxf(top, fmaxf(fabsf(qe * frag_elem<SC>(y, e)), fabsf(qe * frag_elem<SC>(z, e))));
      }
    }
    for (int i = lane & 7; i < dr; i += 8) rope = fmaxf(rope, fabsf(ld<DT>(q, dn + i)));
#pragma unroll
    for (int s = 4; s > 0; s >>= 1) top = fmaxf(top, __shfl_xor(top, s)), rope = fmaxf(rope, __shfl_xor(rope, s));
    f = row_factor(top, rope, dn);
  }
  if ((lane & 7) == 0 && h0 + lane / 8 < h1) qsc[static_cast<int64_t>(t) * a.H + h0 + lane / 8] = a.scale * kLog2e / f;
  const int half = dr / 2;
  for (int i = lane; i < row - 2 * r; i += 64) {
    const bool in = i < dr, low = i < half;
    float cs = 1.0f, sn = 0.0f;
    if (in && a.freqs != nullptr) turn_of(pos, a.freqs[low ? i : i - half], cs, sn);
    if (low) sn = -sn;
#pragma unroll
    for (int n = 0; n < kRopeHeads; ++n) {
      if (h0 + n >= h1) continue;
      const char* q = static_cast<const char*>(a.q) + (t * a.q_t + (h0 + n) * a.q_h) * esize<DT>();
      float x = 0.0f;
      if (in) {
        x = ld<DT>(q, dn + i);
        if (a.freqs != nullptr) x = x * cs + ld<DT>(q, dn + (low ? i + half : i - half)) * sn;
      }
      if constexpr (CD == kDtF16) x *= __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f), 8 * n));
#pragma unroll
      for (int m = 0; m < TQ; ++m) {
        const float y = rounded<CD>(x);
        st<CD>(qout + q_offset<CD, TQ>(static_cast<int64_t>(t) * a.H + h0 + n, m, 2 * r + i, row), 0, y);
        x -= y;
      }
    }
  }
}

// ---------------------------------------------------------------------------
// split
// ---------------------------------------------------------------------------
struct SplitArgs {
  CacheArgs c;
  LatPlan p;
  int T, H;
  Divisor page, heads;
  const char* q;
  const float* qsc;
  float* ml;
  float* o;
};

// An LDS tile holds its tokens' columns of one wave, unit by unit as in attn_common.h (whose
// frag_rows and frag_cols read a unit as a tile of one): 32 rows, or 16.
// a cache row of zeros (the widest, 4 bytes a column)
__device__ const uint32_t kZeroRow[kMaxLatentRow] = {};

template <int CD, int TQ, int TP, int UPW, bool CSPLIT>
__global__ void __launch_bounds__(256, 1) split_kernel(SplitArgs a) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  constexpr int ES = esize<CD>(), PU = 2 * ES;
  // every wave holds UPW units (else up to UPW: absent ones meet a zero q' at the last one's place)
  constexpr bool EXACT = !CSPLIT && UPW > 4;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hh = lane >> 5, ml_ = lane & 31;
  const CacheArgs& c = a.c;
  const LatPlan& p = a.p;
  const int step = p.step;
  WorkMap map{c, a.T, a.H, step, lane};
  const int W = map.total();
  const int g = blockIdx.x;
  const int G = groups_of(W, step);
  if (W == 0 || g >= G) return;
  const int x_begin = first_step(W, g, G), x_end = first_step(W, g + 1, G);
  int x = x_begin;
  const int tw = CSPLIT ? 0 : wave, cw = CSPLIT ? wave : 0;
  const int u0 = cw * p.nuw;                                       // the wave's units of the row
  const int nu = EXACT ? UPW : min(p.nuw, p.nu - u0), vu = max(0, min(nu, p.vu - u0));
  char* tiles = smem + wave * p.stages * p.tile_bytes;
  float* xchg = reinterpret_cast<float*>(smem + (CSPLIT ? 4 : p.ntw) * p.stages * p.tile_bytes);
  const int64_t row_bytes = static_cast<int64_t>(c.row) * esize<CD>();
  const char* data = static_cast<const char*>(c.data) + u0 * 32 * esize<CD>();
  const char* zeros = reinterpret_cast<const char*>(kZeroRow) + u0 * 32 * esize<CD>();
  const int ow = p.vu * 32, unit_bytes = p.tpt * PU * 16;

  while (x < x_end) {
    SeqWork sw;
    int sb, ib;
    const int b = map.find(true, x, sw, sb, ib);
    if (b < 0) break;
    // (x - sb < items steps, the quotient of 32-bit integers in 64 bits: exact floor)
    const int item = static_cast<int>(static_cast<double>(x - sb) / static_cast<double>(sw.steps));
    const int s0 = x - sb - item * sw.steps;
    const int s1 = min(sw.steps, s0 + (x_end - x));
    const int64_t slot = g + ib + item;

    // a token's page; its row of the cache, where the page is one.  Tokens without a place
    // (and those past the end) read zeros, so that what the masked scores' zero probabilities
    // are multiplied with is no stranger's infinity.
    const int32_t* table = c.table + static_cast<int64_t>(b) * c.max_pages;
    auto page_of = [&](int tok) { return table[quotient(min(tok, sw.len - 1), a.page)]; };
    auto place = [&](int tok, int page, bool& ok) {
      ok = tok < sw.len && page >= 0 && page < c.n_pages;
      return page * c.page_size + (tok - quotient(tok, a.page) * c.page_size);
    };
    auto tile_at = [&](int s) { return (s * p.ntw + tw) * p.tpt; };
    int page = page_of(tile_at(s0) + ml_);

    // A tile's loads, 64 / PU tokens each: lane l takes piece l % PU of rows l / PU + n 64 / PU.
    // Returns which of the tile's tokens are seen.
    constexpr int TPL = 64 / PU, NL = 32 / TPL;  // tokens of a load, loads of a unit of 32 tokens
    auto issue = [&](int tok, int pg, char* dst) -> uint32_t {
      bool ok;
      const int at = place(tok, pg, ok);
      const int idx = ok ? at : -1;
      ok = ok && ml_ < p.tpt;
      const char* src[NL];
#pragma unroll
      for (int n = 0; n < NL; ++n) {
        const int t = lane / PU + n * TPL;
        const int of = __shfl(idx, t & (p.tpt - 1));
        src[n] = (of < 0 ? zeros : data + of * row_bytes) + 16 * ((lane & (PU - 1)) ^ swz<CD>(t));
      }
#pragma unroll
      for (int u = 0; u < UPW; ++u) {
        if (EXACT || u < nu) {
#pragma unroll
          for (int n = 0; n < NL; ++n) {
            if (n * TPL < p.tpt)
              load_lds16(src[n] + u * 32 * ES, dst + (u * p.tpt + n * TPL) * PU * 16);
          }
        }
      }
      return static_cast<uint32_t>(__ballot(ok));  // lanes 0 .. 31: the tile's tokens
    };

    uint32_t okm = 0, okn = 0;
    if (x > x_begin) lds_barrier();  // the previous item's readers of this memory are done
    x += s1 - s0;
    if (p.stages == 2) {
      okm = issue(tile_at(s0) + ml_, page, tiles);
      page = page_of(tile_at(s0 + 1) + ml_);
    }

    // the item's query rows: columns of the tiles
    const int rows = sw.nq * a.H;
    const int rr = min(ml_, rows - 1 - item * kCols);  // within the item
    const int64_t m0 = static_cast<int64_t>(sw.q0) * a.H + item * kCols;
    const int pos = sw.first + quotient(item * kCols + rr, a.heads);
    const int pos_min = sw.first + quotient(item * kCols, a.heads);
    const float qs = a.qsc[m0 + rr];
    // (piece of 16 bytes: slice k of 16 columns, the lane's half of it, part f of an fp32 eight)
    const char* qbase = a.q + q_offset<CD, TQ>(m0 + rr, 0, 32 * u0 + 8 * hh, c.row);
    const int term = c.row / (16 / ES) * 512;
    Frag<CD> qf[2 * UPW][TQ];
    constexpr int FP = ES / 2;  // pieces of a fragment a lane
    if (!CSPLIT && p.stages == 2 && p.ntw >= TQ) {
      // the token waves need the same fragments: each loads a part of them into the second
      // tiles (term n into wave n's), and all read them from there
      const int nf = 2 * nu * FP;
      for (int i = wave; i < TQ * nf; i += p.ntw) {
        const int n = i / nf, k = i - n * nf;
        load_lds16(qbase + n * term + (k / FP) * 1024 * FP + k % FP * 512, smem + (2 * n + 1) * p.tile_bytes + 1024 * k);
      }
      wait_loads();
      lds_barrier();
#pragma unroll
      for (int k = 0; k < 2 * UPW; ++k) {
#pragma unroll
        for (int n = 0; n < TQ; ++n) {
          qf[k][n] = frag_zero<CD>();
          if (EXACT || k < 2 * nu) {
            const char* src = smem + (2 * n + 1) * p.tile_bytes + 1024 * FP * k + 16 * lane;
            qf[k][n].v[0] = *reinterpret_cast<const u32x4*>(src);
            if constexpr (CD == kDtF32) qf[k][n].v[1] = *reinterpret_cast<const u32x4*>(src + 1024);
          }
        }
      }
      lds_barrier();
    } else {
#pragma unroll
      for (int k = 0; k < 2 * UPW; ++k) {
#pragma unroll
        for (int n = 0; n < TQ; ++n) {
          qf[k][n] = frag_zero<CD>();
          if (EXACT || k < 2 * nu) {
            const char* src = qbase + n * term + k * 1024 * FP;
            qf[k][n].v[0] = *reinterpret_cast<const u32x4*>(src);
            if constexpr (CD == kDtF32) qf[k][n].v[1] = *reinterpret_cast<const u32x4*>(src + 512);
          }
        }
      }
    }
    floatx16 o[UPW];
#pragma unroll
    for (int u = 0; u < UPW; ++u)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[u][e] = 0.0f;
    float mx = -INFINITY, sum = 0.0f;
    for (int s = s0; s < s1; ++s) {
      char* tile = tiles;
      if (p.stages == 2) {
        tile += ((s - s0) & 1) * p.tile_bytes;
        wait_loads();
        if (s + 1 < s1) {
          okn = issue(tile_at(s + 1) + ml_, page, tiles + ((s + 1 - s0) & 1) * p.tile_bytes);
          page = page_of(tile_at(s + 2) + ml_);
        }
      } else {
        okm = issue(tile_at(s) + ml_, page, tile);
        page = page_of(tile_at(s + 1) + ml_);
        wait_loads();
      }
      asm volatile("" ::: "memory");
      // scores: row (token) 8 (e / 4) + 4 hh + e % 4 of column (query row) lane % 32
      floatx16 acc;
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[e] = 0.0f;
#pragma unroll
      for (int u = 0; u < UPW; ++u) {
        const char* unit = tile + (EXACT ? u : min(u, nu - 1)) * unit_bytes;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const Frag<CD> kf = frag_rows<CD, 32>(unit, 0, 16 * k, lane, p.tpt - 1);
#pragma unroll
          for (int n = 0; n < TQ; ++n) acc = mma32<CD>(kf, qf[2 * u + k][n], acc);
        }
      }
      if constexpr (CSPLIT) {
        // the column waves' scores added, in the same order by each of them
        float* xb = xchg + ((s - s0) & 1) * 4096;
#pragma unroll
        for (int e = 0; e < 16; e += 4)
          *reinterpret_cast<float4*>(xb + wave * 1024 + (e >> 2) * 256 + lane * 4) =
              make_float4(acc[e], acc[e + 1], acc[e + 2], acc[e + 3]);
        lds_barrier();
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
          float4 t = *reinterpret_cast<const float4*>(xb + (e >> 2) * 256 + lane * 4);
#pragma unroll
          for (int w = 1; w < 4; ++w) {
            const float4 v = *reinterpret_cast<const float4*>(xb + w * 1024 + (e >> 2) * 256 + lane * 4);
            t.x += v.x, t.y += v.y, t.z += v.z, t.w += v.w;
          }
          acc[e] = t.x, acc[e + 1] = t.y, acc[e + 2] = t.z, acc[e + 3] = t.w;
        }
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[e] *= qs;
      const int base = tile_at(s);
      if (okm != 0xffffffffu || base + 31 > pos_min) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int t = 8 * (e >> 2) + 4 * hh + (e & 3);
          if (!((okm >> t) & 1u) || base + t > pos) acc[e] = -INFINITY;
        }
      }
      float tm = acc[0];
#pragma unroll
      for (int e = 1; e < 16; ++e) tm = fmaxf(tm, acc[e]);
      tm = fmaxf(tm, __shfl_xor(tm, 32));
      // sums are kept relative to mx, a maximum that follows once it is 2^kSlack behind: a
      // probability is then at most 2^kSlack, which neither type nor sum minds
      if (__any(tm > mx + kSlack)) {
        const float m2 = fmaxf(mx, tm);
        const float f = m2 == -INFINITY ? 1.0f : exp2_fast(mx - m2);
        mx = m2;
        sum *= f;
#pragma unroll
        for (int u = 0; u < UPW; ++u) {
#pragma unroll
          for (int e = 0; e < 16; ++e) o[u][e] *= f;
        }
      }
      const float mz = mx == -INFINITY ? 0.0f : mx;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        acc[e] = exp2_fast(acc[e] - mz);
        sum += acc[e];
      }
#pragma unroll
      for (int sl = 0; sl < 2; ++sl) {
        if (16 * sl >= p.tpt) break;
        // probabilities in terms of the cache's type: one rounding (relative half a step each,
        // of terms that the output averages) where the output's type is no finer, else TP terms
        float pv[8];
        Frag<CD> pf[TP];
#pragma unroll
        for (int e = 0; e < 8; ++e) pv[e] = acc[8 * sl + e];
        to_terms<CD, TP>(pv, pf);
        // (the rotary units too: their sums are not read)
#pragma unroll
        for (int u = 0; u < UPW; ++u) {
          const Frag<CD> vf = frag_cols<CD, 32>(tile + (EXACT ? u : min(u, nu - 1)) * unit_bytes, 16 * sl, 0, lane);
#pragma unroll
          for (int n = 0; n < TP; ++n) o[u] = mma32<CD>(vf, pf[n], o[u]);
        }
      }
      if (p.stages == 2) okm = okn;
      asm volatile("" ::: "memory");
    }

    // the item's partial result: sums of each column scaled by its maximum's exponential
    sum += __shfl_xor(sum, 32);
    float* po = a.o + slot * kCols * ow;
    float* pm = a.ml + slot * kCols * 2;
    if constexpr (CSPLIT) {
      // two units at a time through the wave's tile, so that rows are written 256 bytes at a time
      constexpr int st = 68;  // floats of a row there
      float* buf = reinterpret_cast<float*>(tiles);
      asm volatile("" ::: "memory");
#pragma unroll
      for (int u = 0; u < UPW; u += 2) {
        if (u < vu) {
#pragma unroll
          for (int v = 0; v < 2; ++v) {
            if (u + v < UPW) {
#pragma unroll
              for (int e = 0; e < 16; e += 4)
                *reinterpret_cast<float4*>(buf + ml_ * st + 32 * v + 2 * e + 4 * hh) =
                    make_float4(o[u + v][e], o[u + v][e + 1], o[u + v][e + 2], o[u + v][e + 3]);
            }
          }
          const int c4 = 4 * (lane & 15);
#pragma unroll
          for (int n = 0; n < 8; ++n) {
            const int m = 4 * n + (lane >> 4);
            if (32 * u + c4 < 32 * vu)
              *reinterpret_cast<float4*>(po + m * ow + 32 * (u0 + u) + c4) = *reinterpret_cast<const float4*>(buf + m * st + c4);
          }
        }
      }
      if (wave == 0 && hh == 0) pm[2 * ml_] = mx, pm[2 * ml_ + 1] = sum;
    } else {
      __syncthreads();  // every wave is done with its tiles
      const int st = ow + 4;
      float* red = reinterpret_cast<float*>(smem);
      float* rml = red + p.ntw * kCols * st;
#pragma unroll
      for (int u = 0; u < UPW; ++u) {
        if (u < vu) {
#pragma unroll
          for (int e = 0; e < 16; e += 4)
            *reinterpret_cast<float4*>(red + (wave * kCols + ml_) * st + 32 * u + 2 * e + 4 * hh) =
                make_float4(o[u][e], o[u][e + 1], o[u][e + 2], o[u][e + 3]);
        }
      }
      if (hh == 0) rml[(wave * kCols + ml_) * 2] = mx, rml[(wave * kCols + ml_) * 2 + 1] = sum;
      __syncthreads();
      // thread: query row m, every eighth (fourth with two waves) group of four columns
      const int tpr = 2 * p.ntw, m = tid / tpr, cq0 = tid - m * tpr;
      float top = -INFINITY, f[4], l = 0.0f;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        f[w] = w < p.ntw ? rml[(w * kCols + m) * 2] : -INFINITY;
        top = fmaxf(top, f[w]);
      }
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        f[w] = f[w] == -INFINITY ? 0.0f : exp2_fast(f[w] - top);
        if (w < p.ntw) l += f[w] * rml[(w * kCols + m) * 2 + 1];
      }
      if (cq0 == 0) *reinterpret_cast<float2*>(pm + 2 * m) = make_float2(top, l);
      const int ws = kCols * st;
      const float* rm = red + m * st;
#pragma unroll 2
      for (int cq = cq0; cq < ow / 4; cq += tpr) {
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          if (w < p.ntw) {
            const float4 t = *reinterpret_cast<const float4*>(rm + w * ws + 4 * cq);
            v.x += f[w] * t.x, v.y += f[w] * t.y, v.z += f[w] * t.z, v.w += f[w] * t.w;
          }
        }
        *reinterpret_cast<float4*>(po + m * ow + 4 * cq) = v;
      }
    }
  }
}

// ---------------------------------------------------------------------------
// join
// ---------------------------------------------------------------------------

struct JoinArgs {
  LatentAttnArgs a;
  LatPlan p;
  const float* ml;
  const float* o;
};

// A workgroup per (token, head): the partial sums of its row, in workgroup order,
// then its head's rows of U with h.
template <int DT, int SC, int KPARTS, int kMaxHalf, int kJThreads>
__global__ void __launch_bounds__(kJThreads) join_kernel(JoinArgs j) {
  __shared__ float wt[256];
  __shared__ __attribute__((aligned(16))) float ov[2][kMaxLatentRank];
  __shared__ float part[KPARTS][2][kMaxHead];
  const LatentAttnArgs& a = j.a;
  const CacheArgs& c = a.c;
  const int tid = threadIdx.x, lane = tid & 63;
  const int t = blockIdx.x / a.H, h = blockIdx.x - t * a.H;
  const int step = j.p.step, r = c.r, rp = (r + 31) & ~31;
  // the words of this thread's output, path and part of the path's words: they do not
  // depend on the sums
  const int n_out = a.Hk * (a.d_nope + a.d_v), row0 = a.Hk * a.d_nope + h / (a.H / a.Hk) * a.d_v;
  const int nb2 = (rp / 32 + KPARTS - 1) / KPARTS;
  uint32_t words[kMaxHalf];
  const int ph = tid / a.d_v, wp = ph & 1, wi = tid - ph * a.d_v, wk = (ph >> 1) * nb2;
#pragma unroll
  for (int n = 0; n < kMaxHalf; ++n) {
    // (the last one may be of 16 bits; absent ones read the first word again)
    const bool ok = ph < 2 * KPARTS && n < nb2 && wk + n < rp / 32;
    words[n] = word_at(word_column(a.U[wp], n_out, r, ok ? wk + n : 0), ok ? row0 + wi : 0);
  }
  WorkMap map{c, a.T, a.H, step, lane};
  const int W = map.total();
  SeqWork sw;
  int sb, ib;
  if (map.find(false, t, sw, sb, ib) < 0) return;  // a row behind the last sequence
#pragma unroll
  for (int n = 0; n < kMaxHalf; ++n) pin(words[n]);  // (loaded above, not where they are used)
  char* out = static_cast<char*>(a.out) + (static_cast<int64_t>(t) * a.H + h) * a.d_v * esize<DT>();
  if (sw.steps == 0) {
    for (int i = tid; i < a.d_v; i += kJThreads) st<DT>(out, i, 0.0f);
    return;
  }
  const int rr = (t - sw.q0) * a.H + h, item = rr / kCols, m = rr - item * kCols;
  const int x0 = sb + item * sw.steps, G = groups_of(W, step);
  const int g0 = group_of(W, x0, G), n = group_of(W, x0 + sw.steps - 1, G) - g0 + 1;  // n <= kG
  const int64_t slot0 = g0 + ib + item;
  const int ow = j.p.vu * 32;
  float top = -INFINITY;
  for (int i = lane; i < n; i += 64) top = fmaxf(top, j.ml[((slot0 + i) * kCols + m) * 2]);
#pragma unroll
  for (int s = 32; s > 0; s >>= 1) top = fmaxf(top, __shfl_xor(top, s));
  float l = 0.0f;
  for (int i = lane; i < n; i += 64) {
    const float* q = j.ml + ((slot0 + i) * kCols + m) * 2;
    const float f = top == -INFINITY ? 1.0f : exp2_fast(q[0] - top);
    l += f * q[1];  // (0: no token is seen)
    if (tid < 64) wt[i] = f;
  }
#pragma unroll
  for (int s = 32; s > 0; s >>= 1) l += __shfl_xor(l, s);
  const float inv = 1.0f / l;
  for (int i = tid; i < 2 * (rp - r); i += kJThreads) {
    const int p = i >= rp - r;
    ov[p][r + i - p * (rp - r)] = 0.0f;
  }
  __syncthreads();
  const float* po = j.o + (slot0 * kCols + m) * ow;
  for (int k = tid; k < 2 * r; k += kJThreads) {
    float v = 0.0f;
#pragma unroll 8
    for (int i = 0; i < n; ++i) v += wt[i] * po[static_cast<int64_t>(i) * kCols * ow + k];
    ov[k >= r][k >= r ? k - r : k] = l == 0.0f ? 0.0f : v * inv;
  }
  __syncthreads();
  if (ph < 2 * KPARTS) {
    float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int n = 0; n < kMaxHalf; ++n) {
      if (n >= nb2 || wk + n >= rp / 32) break;
#pragma unroll
      for (int k = 0; k < 32; k += 4) {
        const float4 v = *reinterpret_cast<const float4*>(&ov[wp][32 * (wk + n) + k]);
        const float vv[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int e = 0; e < 4; ++e)
          s[e] += __uint_as_float(__float_as_uint(vv[e]) ^ ((words[n] << (31 - k - e)) & 0x80000000u));
      }
    }
    part[ph >> 1][wp][wi] = (s[0] + s[1]) + (s[2] + s[3]);
  }
  __syncthreads();
  for (int i = tid; i < a.d_v; i += kJThreads) {
    float s0 = part[0][0][i], s1 = part[0][1][i];
#pragma unroll
    for (int n = 1; n < KPARTS; ++n) s0 += part[n][0][i], s1 += part[n][1][i];
    const float y0 = ld<SC>(a.h[0], row0 + i) * s0, y1 = ld<SC>(a.h[1], row0 + i) * s1;
    st<DT>(out, i, y0 + y1);
  }
}

// ---------------------------------------------------------------------------
// launches
// ---------------------------------------------------------------------------
template <int CD, int TQ, int TP, int UPW, bool CS>
hipError_t split_launch(const SplitArgs& s, hipStream_t stream) {
  static LdsLimit limit;
  const hipError_t e = raise_lds(reinterpret_cast<const void*>(&split_kernel<CD, TQ, TP, UPW, CS>), s.p.lds, limit);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((split_kernel<CD, TQ, TP, UPW, CS>), dim3(kG), dim3(64 * s.p.ncw * s.p.ntw), s.p.lds, stream, s);
  return hipGetLastError();
}
template <int CD, int TQ, int TP>
hipError_t split_cd(const SplitArgs& s, hipStream_t stream) {
  if (s.p.ncw == 1) {
    switch (s.p.upw) {
      case 4: return split_launch<CD, TQ, TP, 4, false>(s, stream);
      case 5: return split_launch<CD, TQ, TP, 5, false>(s, stream);
      case 6: return split_launch<CD, TQ, TP, 6, false>(s, stream);
      case 7: return split_launch<CD, TQ, TP, 7, false>(s, stream);
      case 8: return split_launch<CD, TQ, TP, 8, false>(s, stream);
      case 9: return split_launch<CD, TQ, TP, 9, false>(s, stream);
      case 10: return split_launch<CD, TQ, TP, 10, false>(s, stream);
      case 11: return split_launch<CD, TQ, TP, 11, false>(s, stream);
      default: return split_launch<CD, TQ, TP, 12, false>(s, stream);
    }
  }
  switch (s.p.upw) {
    case 4: return split_launch<CD, TQ, TP, 4, true>(s, stream);
    case 6: return split_launch<CD, TQ, TP, 6, true>(s, stream);
    case 8: return split_launch<CD, TQ, TP, 8, true>(s, stream);
    case 10: return split_launch<CD, TQ, TP, 10, true>(s, stream);
    default: return split_launch<CD, TQ, TP, 12, true>(s, stream);
  }
}

template <int DT, int SC, int KPARTS, int WORDS, int THREADS>
hipError_t join_launch(const JoinArgs& j, hipStream_t stream) {
  hipLaunchKernelGGL((join_kernel<DT, SC, KPARTS, WORDS, THREADS>), dim3(j.a.T * j.a.H), dim3(THREADS), 0, stream, j);
  return hipGetLastError();
}

template <int DT, int SC, int CD>
hipError_t run(const LatentAttnArgs& a, hipStream_t stream) {
  constexpr int TQ = terms_q(CD, DT == kDtF32), TP = terms_p(CD, DT);
  const LatPlan p = lat_plan(a.c.r, a.c.d_rope, esize<CD>());
  const LatWs w = lat_ws(a.T, a.c.n_seq, a.H, a.c.r, a.c.d_rope);
  char* ws = static_cast<char*>(a.ws);
  float* qsc = reinterpret_cast<float*>(ws + w.qs_off);
  const int nkb = (a.c.r + 31) / 32;
  const int n_mma = a.H * 2 * nkb * ((a.T + kAbsTokens - 1) / kAbsTokens);
  auto al = [](const void* q) { return reinterpret_cast<uintptr_t>(q) % 16 == 0; };
  const bool vec = a.d_nope % 8 == 0 && al(a.q) && al(a.h[0]) && al(a.h[1]) && a.q_t % 8 == 0 && a.q_h % 8 == 0;
  const int n_rope = a.T * ((a.H + kRopeHeads - 1) / kRopeHeads);
  hipLaunchKernelGGL((absorb_kernel<DT, SC, CD, TQ>), dim3(n_mma + n_rope), dim3(64), 0, stream, a, ws, qsc, nkb, n_mma,
                     vec);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  SplitArgs s{};
  s.c = a.c;
  s.p = p;
  s.T = a.T, s.H = a.H;
  s.page = divisor(a.c.page_size), s.heads = divisor(a.H);
  s.q = ws, s.qsc = qsc;
  s.ml = reinterpret_cast<float*>(ws + w.ml_off);
  s.o = reinterpret_cast<float*>(ws + w.o_off);
  e = split_cd<CD, TQ, TP>(s, stream);
  if (e != hipSuccess) return e;
  JoinArgs j{a, p, s.ml, s.o};
  // two threads an output; high ranks four, a path's words in halves
  const bool wide = a.d_v > 128, high = a.c.r > 256;
  if (high)
    return wide ? join_launch<DT, SC, 2, 12, 1024>(j, stream) : join_launch<DT, SC, 2, 12, 512>(j, stream);
  return wide ? join_launch<DT, SC, 1, 8, 512>(j, stream) : join_launch<DT, SC, 1, 8, 256>(j, stream);
}
template <int DT, int SC>
hipError_t run_sc(const LatentAttnArgs& a, hipStream_t stream) {
  switch (a.c.dt) {
    case kDtF32: return run<DT, SC, kDtF32>(a, stream);
    case kDtF16: return run<DT, SC, kDtF16>(a, stream);
    default: return run<DT, SC, kDtBF16>(a, stream);
  }
}
template <int DT>
hipError_t run_dt(const LatentAttnArgs& a, hipStream_t stream) {
  switch (a.sc_dt) {
    case kDtF32: return run_sc<DT, kDtF32>(a, stream);
    case kDtF16: return run_sc<DT, kDtF16>(a, stream);
    default: return run_sc<DT, kDtBF16>(a, stream);
  }
}

}  // namespace

size_t latent_attn_workspace_bytes(int T, int n_seq, int H, int r, int d_rope) {
  return lat_ws(T, n_seq, H, r, d_rope).bytes;
}

hipError_t launch_latent_attn(const LatentAttnArgs& a, hipStream_t stream) {
  switch (a.dt) {
    case kDtF32: return run_dt<kDtF32>(a, stream);
    case kDtF16: return run_dt<kDtF16>(a, stream);
    default: return run_dt<kDtBF16>(a, stream);
  }
}

}  // namespace lb
