// Position rotation of heads' rotary parts, and the append of new tokens to a
// paged latent cache with the rotation of their rotary key on the way.
//
//   y_i = x_i cos a - x_{i + d/2} sin a,   y_{i + d/2} = x_{i + d/2} cos a + x_i sin a,
//   a = position * freqs[i]   (the transposed map: a -> -a)
//
// Both are bound by the bytes they move, and small calls by their launch and the loads
// that follow one another (prefix sums, length, page, row).  Measured: 8192 tokens x 32 heads x
// 64 bf16 values 12.7 us, 5.3 TB/s, what a large copy reaches (5.1); 5 fp32 rows 1.7 us; the append of
// 64 single tokens 5.4 us, of 8 prompts with 7000 tokens (fp32 latents, r = 144, to f16) 10 us.
#include "attn.h"
#include "attn_common.h"

namespace lb {

namespace {

constexpr int kRThreads = 256;
constexpr int kRHeads = 4;  // heads per thread: they share a token's cosines and sines

// A thread owns VP pairs of one token in every nhg-th head: the angles (64-bit
// products, one sine and cosine a pair) are formed once for up to kRHeads heads.
template <int DT, int VP>
__global__ void __launch_bounds__(kRThreads) rotate_kernel(RotateArgs a, int niv, int nhg, uint32_t n) {
  const uint32_t id = blockIdx.x * kRThreads + threadIdx.x;
  if (id >= n) return;
  const int iv = id % niv;
  const int hg = (id / niv) % nhg;
  const int t = id / niv / nhg;
  const int half = a.d / 2;
  const int pos = a.positions[t];
  float c[VP], s[VP];
#pragma unroll
  for (int e = 0; e < VP; ++e) {
    turn_of(pos, a.freqs[iv * VP + e], c[e], s[e]);
    if (a.inverse) s[e] = -s[e];
  }
  const int es = esize<DT>();
#pragma unroll
  for (int q = 0; q < kRHeads; ++q) {
    const int h = hg + q * nhg;
    if (h >= a.H) break;
    const char* x = static_cast<const char*>(a.x) + (t * a.x_t + h * a.x_h + iv * VP) * es;
    char* y = static_cast<char*>(a.y) + (t * a.y_t + h * a.y_h + iv * VP) * es;
    if constexpr (VP == 1) {
      const float u = ld<DT>(x, 0), v = ld<DT>(x, half);
      st<DT>(y, 0, u * c[0] - v * s[0]);
      st<DT>(y, half, v * c[0] + u * s[0]);
    } else {
      // VP elements are 16 bytes (8 of 16 bits, 4 of 32)
      const u32x4 ub = *reinterpret_cast<const u32x4*>(x), vb = *reinterpret_cast<const u32x4*>(x + half * es);
      float lo[VP], hi[VP];
#pragma unroll
      for (int e = 0; e < VP; ++e) {
        float u, v;
        if constexpr (DT == kDtF32) {
          u = __uint_as_float(ub[e]), v = __uint_as_float(vb[e]);
        } else {
          u = bits_to_f32<DT>((ub[e >> 1] >> (16 * (e & 1))) & 0xffffu);
          v = bits_to_f32<DT>((vb[e >> 1] >> (16 * (e & 1))) & 0xffffu);
        }
        lo[e] = u * c[e] - v * s[e];
        hi[e] = v * c[e] + u * s[e];
      }
      u32x4 lob, hib;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if constexpr (DT == kDtF32) {
          lob[e] = __float_as_uint(lo[e]), hib[e] = __float_as_uint(hi[e]);
        } else {
          lob[e] = pack2<DT>(lo[2 * e], lo[2 * e + 1]);
          hib[e] = pack2<DT>(hi[2 * e], hi[2 * e + 1]);
        }
      }
      *reinterpret_cast<u32x4*>(y) = lob;
      *reinterpret_cast<u32x4*>(y + half * es) = hib;
    }
  }
}

template <int DT>
hipError_t rotate_dt(const RotateArgs& a, hipStream_t stream) {
  constexpr int VP = 16 / esize<DT>();
  const int half = a.d / 2;
  auto ok = [&](const void* p, int64_t st, int64_t sh) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && (a.T == 1 || st % VP == 0) && (a.H == 1 || sh % VP == 0);
  };
  const bool vec = half % VP == 0 && ok(a.x, a.x_t, a.x_h) && ok(a.y, a.y_t, a.y_h);
  const int niv = vec ? half / VP : half, nhg = (a.H + kRHeads - 1) / kRHeads;
  const uint32_t n = static_cast<uint32_t>(static_cast<int64_t>(a.T) * niv * nhg);
  const dim3 grid((n + kRThreads - 1) / kRThreads);
  if (vec)
    hipLaunchKernelGGL((rotate_kernel<DT, VP>), grid, dim3(kRThreads), 0, stream, a, niv, nhg, n);
  else
    hipLaunchKernelGGL((rotate_kernel<DT, 1>), grid, dim3(kRThreads), 0, stream, a, niv, nhg, n);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// append
// ---------------------------------------------------------------------------
// A wave writes one token's row, eight elements a lane and step (whole 16-byte
// stores: rows are multiples of 32 elements).  Its sequence is found from the prefix
// sums, 64 at a time; a token without a place (before position 0, past its page
// table, or on a page outside the cache) is not written.
template <int DT, int CD>
__global__ void __launch_bounds__(kRThreads) append_kernel(AppendArgs a, bool vec) {
  const int lane = threadIdx.x & 63;
  const int t = __builtin_amdgcn_readfirstlane(blockIdx.x * (blockDim.x >> 6) + (threadIdx.x >> 6));
  if (t >= a.T) return;
  const CacheArgs& c = a.c;
  int b = -1;
  for (int b0 = 0; b0 < c.n_seq; b0 += 64) {
    const uint64_t m = __ballot(b0 + lane < c.n_seq && c.cu[min(b0 + lane + 1, c.n_seq)] > t);
    if (m != 0) {
      b = b0 + __builtin_ctzll(m);
      break;
    }
  }
  if (b < 0 || c.cu[0] > t) return;
  const int64_t pos = static_cast<int64_t>(c.lens[b]) - (static_cast<int64_t>(c.cu[b + 1]) - t);
  if (pos < 0 || pos >= static_cast<int64_t>(c.max_pages) * c.page_size) return;
  const int pg = static_cast<int>(pos) / c.page_size, off = static_cast<int>(pos) - pg * c.page_size;
  const int page = c.table[static_cast<int64_t>(b) * c.max_pages + pg];
  if (page < 0 || page >= c.n_pages) return;
  char* row = static_cast<char*>(c.data) + (static_cast<int64_t>(page) * c.page_size + off) * c.row * esize<CD>();
  const int nw = 2 * c.r, dr = c.d_rope, half = dr / 2;
  const char* w = static_cast<const char*>(a.w) + static_cast<int64_t>(t) * nw * esize<DT>();
  const char* kr = static_cast<const char*>(a.k_rope) + t * a.kr_t * esize<DT>();
  for (int col = 8 * lane; col < c.row; col += 512) {
    Frag<DT> in = load8<DT>(w, col, nw, vec);
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = frag_elem<DT>(in, e);
    if (col + 8 > nw && col < nw + dr) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int i = col + e - nw;
        if (i < 0 || i >= dr) continue;
        float u = ld<DT>(kr, i);
        if (a.freqs != nullptr) {
          float cs, sn;
          const bool low = i < half;
          turn_of(static_cast<int>(pos), a.freqs[low ? i : i - half], cs, sn);
          const float o = ld<DT>(kr, low ? i + half : i - half);
          u = low ? u * cs - o * sn : u * cs + o * sn;
        }
        v[e] = u;
      }
    }
    const Frag<CD> out = frag_from<CD>(v);
    char* p = row + col * esize<CD>();
    *reinterpret_cast<u32x4*>(p) = out.v[0];
    if constexpr (CD == kDtF32) *reinterpret_cast<u32x4*>(p + 16) = out.v[1];
  }
}

template <int DT, int CD>
hipError_t append_dt(const AppendArgs& a, hipStream_t stream) {
  constexpr int V = 16 / esize<DT>();
  const bool vec = reinterpret_cast<uintptr_t>(a.w) % 16 == 0 && (2 * a.c.r) % V == 0;
  // few tokens: a wave a workgroup, so that they start on as many CUs
  const int waves = a.T <= 1024 ? 1 : kRThreads / 64;
  hipLaunchKernelGGL((append_kernel<DT, CD>), dim3((a.T + waves - 1) / waves), dim3(64 * waves), 0, stream, a, vec);
  return hipGetLastError();
}

template <int DT>
hipError_t append_cd(const AppendArgs& a, hipStream_t stream) {
  switch (a.c.dt) {
    case kDtF32: return append_dt<DT, kDtF32>(a, stream);
    case kDtF16: return append_dt<DT, kDtF16>(a, stream);
    default: return append_dt<DT, kDtBF16>(a, stream);
  }
}

}  // namespace

hipError_t launch_rotate(const RotateArgs& a, hipStream_t stream) {
  switch (a.dt) {
    case kDtF32: return rotate_dt<kDtF32>(a, stream);
    case kDtF16: return rotate_dt<kDtF16>(a, stream);
    default: return rotate_dt<kDtBF16>(a, stream);
  }
}

hipError_t launch_append(const AppendArgs& a, hipStream_t stream) {
  switch (a.dt) {
    case kDtF32: return append_cd<kDtF32>(a, stream);
    case kDtF16: return append_cd<kDtF16>(a, stream);
    default: return append_cd<kDtBF16>(a, stream);
  }
}

}  // namespace lb
