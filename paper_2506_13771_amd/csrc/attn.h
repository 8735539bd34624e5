// Internal declarations of the paged latent cache and the attention calls.
#pragma once
#include "lb_internal.h"

namespace lb {

constexpr int kMaxLatentRow = 1536;   // columns of a cache row
constexpr int kMaxLatentRank = kMaxLatentRow / 2;
constexpr int kMaxRope = 256;         // widths of a rotary part
constexpr int kRowUnit = 32;          // elements; cache rows are whole units

inline int latent_row(int64_t r, int64_t d_rope) {
  return static_cast<int>((2 * r + d_rope + kRowUnit - 1) / kRowUnit * kRowUnit);
}

struct RotateArgs {
  const void* x;
  void* y;
  int dt, T, H, d;
  int64_t x_t, x_h, y_t, y_h;  // strides in elements
  const int32_t* positions;
  const float* freqs;
  int inverse;
};

struct CacheArgs {
  void* data;
  int dt;
  int64_t n_pages;
  int page_size, r, d_rope, row;
  const int32_t* table;
  int n_seq, max_pages;
  const int32_t* lens;
  const int32_t* cu;
};

struct AppendArgs {
  CacheArgs c;
  const void* w;
  const void* k_rope;
  int64_t kr_t;
  int dt, T;
  const float* freqs;
};

struct LatentAttnArgs {
  CacheArgs c;
  const void* q;
  int dt, T, H, Hk, d_nope, d_v;
  int64_t q_t, q_h;
  const void* U[2];
  const void* h[2];
  int sc_dt;
  const float* freqs;
  float scale;
  void* out;
  void* ws;
};

struct AttnArgs {
  const void *q, *k, *v, *k_rope;
  int dt, Tq, Tk, H, Hk, d_nope, d_rope, d_v;
  int64_t q_t, q_h, k_t, k_h, v_t, v_h, kr_t;
  const int32_t *cu_q, *cu_k;
  int n_seq, causal;
  float scale;
  // outputs of the forward, inputs of the backward
  void* o;
  float* lse;
  // backward
  const void* d_o;
  void *dq, *dk, *dv, *dkr;
  int64_t dk_t, dk_h, dv_t, dv_h;
  float* delta;     // [Tq][H]: rowsum(dO (.) O)
  float* dkr_part;  // [Hk][Tk][d_rope]
};

// The number of 128-row workgroups (a wave 32 of the rows) that T rows of n_seq sequences and
// `heads` heads make, half of one counted for each sequence's last.  Below a kernel's
// limit the other form runs: 32 rows a workgroup, whose waves split the other axis.
inline int64_t wide_groups(int64_t T, int n_seq, int64_t heads) { return (T / 128 + (n_seq + 1) / 2) * heads; }

hipError_t launch_rotate(const RotateArgs& a, hipStream_t stream);
hipError_t launch_append(const AppendArgs& a, hipStream_t stream);
size_t latent_attn_workspace_bytes(int T, int n_seq, int H, int r, int d_rope);
hipError_t launch_latent_attn(const LatentAttnArgs& a, hipStream_t stream);
bool attn_vec(const AttnArgs& a, bool backward);
bool attn_supports(int64_t dk, int64_t dv);
hipError_t launch_attn_forward(const AttnArgs& a, hipStream_t stream);
hipError_t launch_attn_backward(const AttnArgs& a, hipStream_t stream);

}  // namespace lb
