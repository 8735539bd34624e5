// The arithmetic of the work map of the attention over the paged latent cache, for host and
// device: which rows a sequence has, which workgroup takes which steps, where the partial
// results stand.
//
// Sequence b's rows begin where the ones before it end, so that no row is in two sequences whatever the prefix
// sums hold, and all sequences together have at most ceil(T H / 32) + n_seq items of 32 rows.  All W steps
// in a row are dealt to G workgroups (G <= W), g taking [W g / G, W (g + 1) / G); its part of the
// item numbered i over all sequences goes to slot g + i: an item's slots are consecutive and no two
// meet.  Sums stay below 2^31 (the caller's sizes are checked for it).
#pragma once
#include <cstdint>

#ifdef __HIPCC__
#define LB_HOST_DEVICE __host__ __device__ __forceinline__
#else
#define LB_HOST_DEVICE inline
#endif

namespace lb {

constexpr int kCols = 32;  // query rows of an item (columns of the tiles)
constexpr int kG = 256;    // workgroups of split (one a CU)

// The row behind a sequence that begins at row `before` (0 .. T) and ends at prefix sum cu.
LB_HOST_DEVICE int rows_end(int before, int32_t cu, int T) {
  const int e = cu < T ? cu : T;
  return e > before ? e : before;
}

// Workgroups that W steps are dealt to: at least 128 tokens each, since a share's
// partial result (32 rows of 4-byte sums, written and read again) costs as much memory
// traffic as 128 tokens of a 16-bit cache.
LB_HOST_DEVICE int groups_of(int W, int step) {
  const int n = W / (step < 128 ? 128 / step : 1);
  return n < 1 ? 1 : n < kG ? n : kG;
}
// (quotients of integers below 2^40 in 64 bits: a floor is exact, the nearest wrong
// integer being 2^-31 or more away)
LB_HOST_DEVICE int first_step(int W, int g, int G) {
  return static_cast<int>(static_cast<double>(static_cast<int64_t>(W) * g) / static_cast<double>(G));
}
// the workgroup that step x belongs to
LB_HOST_DEVICE int group_of(int W, int x, int G) {
  return static_cast<int>(static_cast<double>((static_cast<int64_t>(x) + 1) * G - 1) / static_cast<double>(W));
}

// places for partial results
inline int64_t lat_slots(int64_t T, int64_t n_seq, int64_t H) { return kG + (T * H + kCols - 1) / kCols + n_seq; }

}  // namespace lb
