// Device helpers of the attention kernels: fragments of eight elements, matrix-
// core products on 32 x 32 tiles in the operands' own type, LDS tiles with rows
// that serve row-wise and transposed reads, and the work maps of packed sequences.
//
// Fragment convention (v_mfma_f32_32x32x16 and its fp32 form): lane l holds row
// (A) or column (B) l % 32 and the eight reduction slots 8 (l / 32) .. + 7 of a
// 16-wide slice; accumulator element e of lane l is row 8 (e / 4) + 4 (l / 32) +
// e % 4 of column l % 32.  An accumulator's elements 8 i .. 8 i + 7 are therefore a
// B operand over rows 16 i .. 16 i + 15 whose slot 4 a + b of lane half u stands for row
// 16 i + 8 a + 4 u + b; frag_cols() reads the A operand with the same relabelling, so
// probabilities go from one product into the next without leaving their registers.
#pragma once
#include "device_common.h"

namespace lb {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kSlack = 8.0f;  // log2 of what a running maximum may fall behind by

// 2^x by the hardware's instruction: values below 2^-126 become 0 (no probability
// that a sum of 32 bits would notice)
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

template <int DT>
constexpr int esize() {
  return DT == kDtF32 ? 4 : 2;
}

// eight elements in type DT
template <int DT>
struct Frag {
  u32x4 v[DT == kDtF32 ? 2 : 1];
};

template <int DT>
__device__ __forceinline__ Frag<DT> frag_zero() {
  Frag<DT> f;
#pragma unroll
  for (int i = 0; i < (DT == kDtF32 ? 2 : 1); ++i) f.v[i] = u32x4{0u, 0u, 0u, 0u};
  return f;
}

template <int DT>
__device__ __forceinline__ float frag_elem(const Frag<DT>& f, int e) {
  if constexpr (DT == kDtF32)
    return __uint_as_float(f.v[e >> 2][e & 3]);
  else
    return bits_to_f32<DT>((f.v[0][e >> 1] >> (16 * (e & 1))) & 0xffffu);
}

// two fp32 values as a pair of 16-bit ones, each rounded to nearest even
template <int DT>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  if constexpr (DT == kDtBF16) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){a, b}, bf16x2));
  } else {
    // the fp32 values are formed first (see st in device_common.h)
    asm volatile("" : "+v"(a), "+v"(b));
    return static_cast<uint32_t>(__half_as_ushort(__float2half_rn(a))) |
           (static_cast<uint32_t>(__half_as_ushort(__float2half_rn(b))) << 16);
  }
}

template <int DT>
__device__ __forceinline__ Frag<DT> frag_from(const float (&x)[8]) {
  Frag<DT> f;
  if constexpr (DT == kDtF32) {
#pragma unroll
    for (int e = 0; e < 8; ++e) f.v[e >> 2][e & 3] = __float_as_uint(x[e]);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) f.v[0][e] = pack2<DT>(x[2 * e], x[2 * e + 1]);
  }
  return f;
}

template <int DT>
__device__ __forceinline__ floatx16 mma32(const Frag<DT>& a, const Frag<DT>& b, floatx16 c) {
  if constexpr (DT == kDtBF16) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a.v[0]),
                                                   __builtin_bit_cast(bf16x8, b.v[0]), c, 0, 0, 0);
  } else if constexpr (DT == kDtF16) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a.v[0]),
                                                  __builtin_bit_cast(f16x8, b.v[0]), c, 0, 0, 0);
  } else {
    // fp32 operands: eight products of two slots each (slot j of both lane halves)
#pragma unroll
    for (int j = 0; j < 8; ++j)
      c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.v[j >> 2][j & 3]),
                                               __uint_as_float(b.v[j >> 2][j & 3]), c, 0, 0, 0);
    return c;
  }
}

// Eight elements at p[col .. col + 7] of a row with n elements; zero from n on.
// vec: the row starts on a 16-byte boundary and n is a multiple of a 16-byte group.
template <int DT>
__device__ __forceinline__ Frag<DT> load8(const void* row, int col, int n, bool vec) {
  Frag<DT> f = frag_zero<DT>();
  if (vec) {
    if constexpr (DT == kDtF32) {
      if (col < n) f.v[0] = *reinterpret_cast<const u32x4*>(static_cast<const float*>(row) + col);
      if (col + 4 < n) f.v[1] = *reinterpret_cast<const u32x4*>(static_cast<const float*>(row) + col + 4);
    } else {
      if (col < n) f.v[0] = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(row) + col);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (col + e < n) {
        const uint32_t u = ld_bits<DT>(row, col + e);
        if constexpr (DT == kDtF32)
          f.v[e >> 2][e & 3] = u;
        else
          f.v[0][e >> 1] |= u << (16 * (e & 1));
      }
    }
  }
  return f;
}
// the same over two joined parts: columns [0, n0) of r0, then [n0, n0 + n1) of r1
template <int DT>
__device__ __forceinline__ Frag<DT> load8_joined(const void* r0, int n0, const void* r1, int n1, int col, bool vec) {
  if (vec) return col < n0 ? load8<DT>(r0, col, n0, true) : load8<DT>(r1, col - n0, n1, true);
  if (col + 8 <= n0 || n1 == 0) return load8<DT>(r0, col, n0, false);
  if (col >= n0) return load8<DT>(r1, col - n0, n1, false);
  Frag<DT> f = load8<DT>(r0, col, n0, false);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int c = col + e - n0;
    if (c >= 0 && c < n1) {
      const uint32_t u = ld_bits<DT>(r1, c);
      if constexpr (DT == kDtF32)
        f.v[e >> 2][e & 3] = u;
      else
        f.v[0][e >> 1] |= u << (16 * (e & 1));
    }
  }
  return f;
}

// four values at row[col ..] of a row with n elements, rounded once; vec: as one store
// (col a multiple of 4, so is n, the row aligned to four elements)
template <int DT>
__device__ __forceinline__ void store4(void* row, int col, int n, bool vec, float v0, float v1, float v2, float v3) {
  char* p = static_cast<char*>(row) + col * esize<DT>();
  if (vec) {
    if (col >= n) return;
    if constexpr (DT == kDtF32)
      *reinterpret_cast<float4*>(p) = make_float4(v0, v1, v2, v3);
    else
      *reinterpret_cast<u32x2*>(p) = u32x2{pack2<DT>(v0, v1), pack2<DT>(v2, v3)};
  } else {
    if (col < n) st<DT>(p, 0, v0);
    if (col + 1 < n) st<DT>(p, 1, v1);
    if (col + 2 < n) st<DT>(p, 2, v2);
    if (col + 3 < n) st<DT>(p, 3, v3);
  }
}

// ---------------------------------------------------------------------------
// LDS tiles of R rows, by units of 32 columns: [unit][row][pieces of 16 bytes], PU pieces
// a row (4; fp32: 8), piece q of row t at q ^ swz(t).  Row-wise reads (16 rows at one
// piece) then meet 16 different slots of the 64 banks and transposed reads (8 rows of 4
// pieces) each slot twice, the least; and a load from memory into LDS (64 lanes' pieces
// in a row) takes the same pieces of 64 / PU rows in every unit.  (No bank conflicts counted
// in any kernel.  16-bit units of 64 columns, 8 rows a load, load no faster and their reads
// need twice the addresses: keys' gradient 330 -> 355 us.)
// ---------------------------------------------------------------------------

template <int DT>
constexpr int pieces() {
  return 2 * esize<DT>();
}
template <int DT>
__device__ __forceinline__ int swz(int t) {
  return DT == kDtF32 ? (t >> 1) & 7 : (t >> 2) & 3;
}
template <int DT, int R, int W>
constexpr int tile_bytes() {
  return R * W * esize<DT>();
}
// eight elements at row t, columns col .. col + 7
template <int DT, int R>
__device__ __forceinline__ void tile_put(char* tile, int t, int col, const Frag<DT>& f) {
  constexpr int PU = pieces<DT>();
  char* p = tile + ((col >> 5) * R + t) * PU * 16;
  const int q = (col & 31) * esize<DT>() / 16, s = swz<DT>(t);
  *reinterpret_cast<u32x4*>(p + 16 * (q ^ s)) = f.v[0];
  if constexpr (DT == kDtF32) *reinterpret_cast<u32x4*>(p + 16 * ((q + 1) ^ s)) = f.v[1];
}
// A or B operand from rows: lane l takes row row0 + l % 32, columns col + 8 (l / 32) .. + 7
// (row0 a multiple of 32, col of 16; a tile of 16 rows gives each twice: last_row 15)
template <int DT, int R>
__device__ __forceinline__ Frag<DT> frag_rows(const char* tile, int row0, int col, int lane, int last_row = 31) {
  constexpr int PU = pieces<DT>();
  const int t = lane & last_row, s = swz<DT>(t);
  const char* p = tile + t * PU * 16;
  const int o = ((col >> 5) * R + row0) * PU * 16;
  Frag<DT> f;
  if constexpr (DT == kDtF32) {
    const int q = 4 * ((col >> 4) & 1) + 2 * (lane >> 5);
    f.v[0] = *reinterpret_cast<const u32x4*>(p + 16 * (q ^ s) + o);
    f.v[1] = *reinterpret_cast<const u32x4*>(p + 16 * ((q + 1) ^ s) + o);
  } else {
    const int q = 2 * ((col >> 4) & 1) + (lane >> 5);
    f.v[0] = *reinterpret_cast<const u32x4*>(p + 16 * (q ^ s) + o);
  }
  return f;
}
// A operand from columns: lane l takes column col + l % 32 at rows row0 + 8 a + 4 (l / 32)
// + b (slot 4 a + b); row0 a multiple of 16, col of 32.  16-bit types: two transposed
// reads (each 16-lane group takes 4 rows x 16 columns).
template <int DT, int R>
__device__ __forceinline__ Frag<DT> frag_cols(const char* tile, int row0, int col, int lane) {
  constexpr int PU = pieces<DT>();
  const int u = lane >> 5, o = ((col >> 5) * R + row0) * PU * 16;
  Frag<DT> f;
  if constexpr (DT == kDtF32) {
    const int q = (lane & 31) >> 2;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int t = 8 * (k >> 2) + 4 * u + (k & 3);  // (16 rows on, swz is the same)
      f.v[k >> 2][k & 3] =
          *reinterpret_cast<const uint32_t*>(tile + t * PU * 16 + 16 * (q ^ swz<DT>(t)) + 4 * (lane & 3) + o);
    }
  } else {
    typedef __attribute__((address_space(3))) s16x4* lds4;
    const int i = lane & 15, q = 2 * ((lane >> 4) & 1) + ((i & 3) >> 1), t = 4 * u + (i >> 2);
    const char* p0 = tile + t * PU * 16 + 16 * (q ^ swz<DT>(t)) + 8 * (i & 1);
    const char* p1 = tile + (t + 8) * PU * 16 + 16 * (q ^ swz<DT>(t + 8)) + 8 * (i & 1);
    const u32x2 a = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(p0 + o)));
    const u32x2 b = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(p1 + o)));
    f.v[0] = u32x4{a[0], a[1], b[0], b[1]};
  }
  return f;
}

// 16 bytes of zeros that loads into LDS take for columns past a row's width
__device__ const uint32_t kZeros[4] = {0u, 0u, 0u, 0u};

// 64 lanes' 16 bytes each from memory into LDS at dst (the same for all lanes) + 16 lane.
// Written as assembly (it has no output register) so that the compiler does not wait for it
// before the next read of any LDS; wait_loads() does.  m0 is a reserved register, which a clobber
// list cannot name: the compiler keeps nothing in it, and the instructions for which it would set
// it (sends, global data share, indexed registers) do not occur here: in these kernels' assembly
// every m0 is this block's.
__device__ __forceinline__ void load_lds16(const void* src, char* dst) {
  const uint32_t off = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char*)dst));
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
               :
               : "s"(__builtin_amdgcn_readfirstlane(off)), "v"(src)
               : "memory");
}

// Memory and matrix instructions do not cross this point in the schedule (vector and
// scalar ones may): it keeps a group's LDS reads ahead of the products with the group before.
__device__ __forceinline__ void keep_order() { __builtin_amdgcn_sched_barrier(0x6); }

// A tile's rows of two joined parts (columns [0, n0) of p0 + row s0, then [n0, n0 + n1) of p1 +
// row s1; element strides; zeros behind) into LDS, by the waves of a workgroup.  Rows from
// n_rows (>= 1) on repeat the last one: their probabilities are 0.  vec: as loads straight into
// LDS (16-byte pieces; the caller waits for them), otherwise through registers.
template <int DT, int R, int W, int THREADS>
__device__ __forceinline__ void tile_load(char* tile, const char* p0, int64_t s0, int n0, const char* p1, int64_t s1, int n1,
                                          int n_rows, bool vec, int tid) {
  constexpr int ES = esize<DT>(), PU = pieces<DT>(), TPL = 64 / PU, NW = THREADS / 64;
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  if (vec) {
    static_assert(R / TPL % NW == 0, "whole rounds of the waves");
#pragma unroll
    for (int g = 0; g < R / TPL; g += NW) {
      const int gw = g + wave, t = gw * TPL + lane / PU;
      const int c = ((lane & (PU - 1)) ^ swz<DT>(t)) * (16 / ES);  // column within the unit
      const int64_t row = min(t, n_rows - 1);
      const char* a = p0 + row * s0 * ES + c * ES;
      const char* b = n1 > 0 ? p1 + row * s1 * ES + (c - n0) * ES : a;
#pragma unroll
      for (int u = 0; u < W / 32; ++u) {
        const int col = 32 * u + c;
        const char* src = (col < n0 ? a : b) + u * 32 * ES;
        src = col < n0 + n1 ? src : reinterpret_cast<const char*>(kZeros);
        load_lds16(src, tile + (u * R + gw * TPL) * PU * 16);
      }
    }
  } else {
    for (int u = tid; u < R * W / 8; u += THREADS) {
      const int t = u / (W / 8), c = 8 * (u % (W / 8));
      const int64_t row = min(t, n_rows - 1);
      tile_put<DT, R>(tile, t, c, load8_joined<DT>(p0 + row * s0 * ES, n0, p1 + row * s1 * ES, n1, c, false));
    }
  }
}

// The loads of such a tile one at a time (n = 0 .. LOADS - 1, known at compile time), so that they
// stand between products: all at once, a wave waits some 2000 cycles for the queue to take its ten.
// (Forward of 2 x 2048 tokens of 7B heads: 148 -> 130 us.)
template <int DT, int R, int W, int THREADS>
struct TileLoads {
  static constexpr int PU = pieces<DT>(), TPL = 64 / PU, LOADS = W / 32;
  static_assert(R == TPL * (THREADS / 64), "one round of the waves");
  const char *a, *b;
  int c, n0, n;
  char* tile;
  __device__ __forceinline__ void start(char* to, const char* p0, int64_t s0, int w0, const char* p1, int64_t s1, int w1,
                                        int n_rows, int tid) {
    constexpr int ES = esize<DT>();
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), t = wave * TPL + lane / PU;
    n0 = w0, n = w0 + w1;
    c = ((lane & (PU - 1)) ^ swz<DT>(t)) * (16 / ES);
    const int64_t row = min(t, n_rows - 1);
    a = p0 + row * s0 * ES + c * ES;
    b = w1 > 0 ? p1 + row * s1 * ES + (c - w0) * ES : a;
    tile = to + wave * TPL * PU * 16;
  }
  __device__ __forceinline__ void load(int u) const {
    constexpr int ES = esize<DT>();
    const int col = 32 * u + c;
    const char* src = (col < n0 ? a : b) + u * 32 * ES;
    src = col < n ? src : reinterpret_cast<const char*>(kZeros);
    load_lds16(src, tile + u * R * PU * 16);
  }
};

// a barrier for LDS: loads from memory stay in flight
__device__ __forceinline__ void lds_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}
// this wave's loads from memory (into LDS too) have arrived
__device__ __forceinline__ void wait_loads() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xf70);  // vmcnt(0); LDS and scalar counters left alone
  asm volatile("" ::: "memory");
}

// ---------------------------------------------------------------------------
// packed sequences
// ---------------------------------------------------------------------------
// Sequence b's rows [lo, hi) by its prefix sums, kept inside [0, T) whatever they hold
// (cu == nullptr: one sequence of all T rows).
__device__ __forceinline__ void seq_range(const int32_t* cu, int b, int T, int& lo, int& hi) {
  if (cu == nullptr) {
    lo = 0, hi = T;
    return;
  }
  lo = min(max(cu[b], 0), T);
  hi = min(max(cu[b + 1], lo), T);
}

// The sequence and the tile of `rows` rows in it that work item `item` stands for
// (every sequence has ceil(n / rows) tiles); false if there are fewer items.  Called by
// whole waves: 64 sequences a step.
__device__ __forceinline__ bool find_tile(const int32_t* cu, int n_seq, int T, int rows, int item, int lane, int& seq,
                                          int& tile) {
  if (cu == nullptr) {
    seq = 0, tile = item;
    return item < (T + rows - 1) / rows;
  }
  int before = 0;
  for (int b0 = 0; b0 < n_seq; b0 += 64) {
    const int b = b0 + lane;
    int n = 0;
    if (b < n_seq) {
      int lo, hi;
      seq_range(cu, b, T, lo, hi);
      n = (hi - lo + rows - 1) / rows;
    }
    int incl = n;
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
      const int o = __shfl_up(incl, s);
      if (lane >= s) incl += o;
    }
    const uint64_t m = __ballot(before + incl > item);
    if (m != 0) {
      const int w = __builtin_ctzll(m);
      seq = b0 + w;
      tile = item - before - (__shfl(incl, w) - __shfl(n, w));
      return true;
    }
    before += __shfl(incl, 63);
  }
  return false;
}

// ---------------------------------------------------------------------------
// position rotation
// ---------------------------------------------------------------------------
// cos and sin of position * frequency.  The angle is formed and brought to one turn in
// 64 bits: three roundings of 2^-53 of the number of turns, so off by 2^-44 of a turn near 160 turns (position 1000
// at frequency 1), by 2^-23 at the 3.4e8 turns of position 2^31.  The functions are taken in fp32 of the
// remaining half turn, whose rounding is up to 2^-26 of a turn.
__device__ __forceinline__ void turn_of(int position, float freq, float& c, float& s) {
  const double t = static_cast<double>(position) * static_cast<double>(freq) * 0.15915494309189533577;
  const float f = static_cast<float>(t - rint(t));  // turns, in [-1/2, 1/2]
  sincospif(2.0f * f, &s, &c);
}

}  // namespace lb
