// Host-side driver for the sanitizer build of the attention calls' boundary (csrc/attention_api.cpp).  The
// launches are stand-ins that note what reaches them, so calls that are accepted can be checked too: no GPU is
// used and no address is read.  Exits non-zero on the first unexpected result.
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <initializer_list>

#include "../../paper_2506_13771_amd/csrc/attn.h"

static int launches = 0;
static bool vec_fits = true;
namespace lb {
hipError_t launch_rotate(const RotateArgs&, hipStream_t) { return ++launches, hipSuccess; }
hipError_t launch_append(const AppendArgs&, hipStream_t) { return ++launches, hipSuccess; }
hipError_t launch_latent_attn(const LatentAttnArgs&, hipStream_t) { return ++launches, hipSuccess; }
hipError_t launch_attn_forward(const AttnArgs&, hipStream_t) { return ++launches, hipSuccess; }
hipError_t launch_attn_backward(const AttnArgs&, hipStream_t) { return ++launches, hipSuccess; }
size_t latent_attn_workspace_bytes(int T, int n_seq, int H, int r, int d_rope) {
  return 256 + 6 * static_cast<size_t>(T) * H * latent_row(r, d_rope) + n_seq;
}
bool attn_vec(const AttnArgs&, bool) { return vec_fits; }
bool attn_supports(int64_t dk, int64_t dv) { return dk >= 1 && dk <= 192 && dv >= 1 && dv <= 128; }
}  // namespace lb

static int failures = 0;
#define EXPECT(c)                                                              \
  do {                                                                         \
    if (!(c)) {                                                                \
      std::fprintf(stderr, "%s:%d: failed: %s\n", __FILE__, __LINE__, #c);     \
      ++failures;                                                              \
    }                                                                          \
  } while (0)
// the status, and whether anything was launched: only ever an accepted call
#define STATUS(call, want)                                                                        \
  do {                                                                                            \
    const int before = launches;                                                                  \
    const lb_status got = (call);                                                                 \
    if (got != (want)) std::fprintf(stderr, "%s:%d: status %d, not %d\n", __FILE__, __LINE__, got, want); \
    EXPECT(got == (want));                                                                        \
    EXPECT(got == LB_OK || launches == before);                                                   \
  } while (0)

// stand-ins for device addresses
static void* at(int64_t i) { return reinterpret_cast<void*>(i << 34); }
static constexpr int64_t kFar = int64_t(1) << 40, kMost = (int64_t(1) << 31) - 1;

static lb_latent_cache cache() {
  return lb_latent_cache{at(1), LB_BF16, 4, 16, 16, 8, static_cast<int32_t*>(at(2)), 2, 2, static_cast<int32_t*>(at(3)), static_cast<int32_t*>(at(4))};
}
static lb_attention attn() {
  lb_attention a{};
  a.q = at(10), a.k = at(12), a.v = at(14), a.k_rope = at(16);
  a.dtype = LB_BF16;
  a.Tq = 8, a.Tk = 9, a.H = 4, a.Hk = 2, a.d_nope = 32, a.d_rope = 16, a.d_v = 24;
  a.q_t = 192, a.q_h = 48, a.k_t = 64, a.k_h = 32, a.v_t = 48, a.v_h = 24, a.kr_t = 16;
  a.causal = 1, a.scale = 0.2f;
  return a;
}
static lb_attention_grads grads() {
  lb_attention_grads g{};
  g.dq = at(20), g.dk = at(22), g.dv = at(24), g.dk_rope = at(26);
  g.dk_t = 64, g.dk_h = 32, g.dv_t = 48, g.dv_h = 24;
  return g;
}
static lb_status forward(const lb_attention& a, void* o = at(30), void* lse = at(32)) {
  return lb_attention_forward(&a, o, static_cast<float*>(lse), nullptr);
}
static lb_status backward(const lb_attention& a, const lb_attention_grads& g, void* ws = at(40), size_t n = size_t(1) << 31) {
  return lb_attention_backward(&a, at(30), static_cast<const float*>(at(32)), at(34), &g, ws, n, nullptr);
}
static lb_status latent(const lb_latent_cache& c, int64_t T = 3, int64_t H = 4, int64_t Hk = 2, int64_t q_t = 160, int64_t q_h = 40,
                        void* out = at(50), void* ws = at(60), int64_t dn = 32, int64_t dv = 16) {
  static lb_path p[2];
  for (auto& x : p) x = lb_path{at(70), nullptr, at(72), nullptr, nullptr};
  return lb_latent_attention(at(74), LB_BF16, T, H, Hk, dn, dv, q_t, q_h, p, LB_F16, &c, static_cast<float*>(at(76)), 0.1f, out, ws,
                             size_t(1) << 40, nullptr);
}
static lb_status rotate(int64_t T, int64_t H, int64_t d, int64_t x_t, int64_t x_h, int64_t y_t, int64_t y_h) {
  return lb_rotate(at(80), LB_F32, T, H, d, x_t, x_h, static_cast<int32_t*>(at(2)), static_cast<float*>(at(3)), 0, at(4),
                   y_t, y_h, nullptr);
}

// Sizes and strides whose products pass 64 bits
static void offsets() {
  EXPECT(forward(attn()) == LB_OK && backward(attn(), grads()) == LB_OK && latent(cache()) == LB_OK && launches == 3);
  STATUS(rotate(2, 3, 8, 24, 8, 24, 8), LB_OK);
  // (an operand's last element may lie 2^59 elements behind its first)
  STATUS(rotate(1 << 19, 1, 8, kFar, 0, 8, 8), LB_OK);
  STATUS(rotate(1 << 28, 1, 2, kFar, 0, 8, 8), LB_ERR_SHAPE);
  STATUS(rotate(1, 1 << 28, 2, 8, kFar, 8, 8), LB_ERR_SHAPE);
  STATUS(rotate(1 << 28, 1, 2, 8, 8, kFar, 8), LB_ERR_SHAPE);
  STATUS(rotate(1, 1 << 28, 2, 8, 8, 8, kFar), LB_ERR_SHAPE);
  STATUS(rotate(1, 1, 2, kFar, kFar, kFar, kFar), LB_OK);
  for (int64_t T : {kMost / 32, int64_t(1) << 25}) {
    lb_attention a = attn();
    a.H = a.Hk = 1, a.d_nope = 8, a.d_rope = 0, a.d_v = 8, a.Tq = a.Tk = T;
    a.q_t = a.k_t = a.v_t = 8;
    lb_attention_grads g = grads();
    g.dk_t = g.dv_t = 8;
    STATUS(forward(a), LB_OK);
    STATUS(backward(a, g), LB_OK);
    for (int64_t lb_attention::*s : {&lb_attention::q_t, &lb_attention::k_t, &lb_attention::v_t}) {
      lb_attention b = a;
      b.*s = kFar;
      STATUS(forward(b), LB_ERR_SHAPE);
      STATUS(backward(b, g), LB_ERR_SHAPE);
    }
    lb_attention b = a;
    b.d_rope = 8, b.kr_t = kFar;
    STATUS(forward(b), LB_ERR_SHAPE);
    for (int64_t lb_attention_grads::*s : {&lb_attention_grads::dk_t, &lb_attention_grads::dv_t}) {
      lb_attention_grads h = g;
      h.*s = kFar;
      STATUS(backward(a, h), LB_ERR_SHAPE);
    }
    lb_latent_cache c = cache();
    STATUS(lb_latent_append(&c, at(90), at(1 << 20), kFar, LB_F32, T, nullptr, nullptr), LB_ERR_SHAPE);
  }
  lb_latent_cache c = cache();
  STATUS(latent(c, 1 << 20, 1, 1, kFar, 40), LB_ERR_SHAPE);
  STATUS(latent(c, 1, 1 << 20, 1, 40, kFar), LB_ERR_SHAPE);
  // no queries' heads: any number of key heads divides them
  for (int64_t n : {int64_t(3), int64_t(1) << 24}) {
    lb_attention a = attn();
    a.H = 0, a.Hk = int64_t(1) << 62, a.Tk = 0, a.n_seq = n;
    a.cu_q = a.cu_k = static_cast<int32_t*>(at(5));
    STATUS(forward(a), LB_ERR_SHAPE);
    STATUS(backward(a, grads()), LB_ERR_SHAPE);
  }
  for (int64_t n : {int64_t(0), int64_t(1), int64_t(33), kMost, int64_t(1) << 40, INT64_MAX}) {
    for (int64_t m : {int64_t(0), int64_t(1), kMost, INT64_MAX}) {
      (void)lb_latent_row(n, m), (void)lb_latent_attention_workspace_bytes(n, m, 1, 16, 8);
      (void)lb_latent_attention_workspace_bytes(n, 1, m, 16, 8), (void)lb_attention_backward_workspace_bytes(n, m, 1, 1, 64);
      (void)lb_attention_backward_workspace_bytes(n, 1, m, 1, 0), (void)lb_attention_backward_workspace_bytes(1, n, 0, m > 0 ? m : 1, 64);
    }
  }
}

// Calls whose launch would have 2^32 threads
static void launch_sizes() {
  for (const bool vec : {true, false}) {
    vec_fits = vec;
    for (const lb_dtype dt : {LB_F32, LB_F16, LB_BF16}) {
      const int64_t rows = dt == LB_F32 || vec ? 128 : 32;
      for (const int64_t H : {int64_t(1), int64_t(64), int64_t(4096)}) {
        lb_attention a = attn();
        a.dtype = dt, a.H = a.Hk = H, a.d_nope = 2, a.d_rope = 0, a.d_v = 2;
        a.q_t = a.k_t = a.v_t = 2 * H, a.q_h = a.k_h = a.v_h = 2;
        lb_attention_grads g = grads();
        g.dk_t = g.dv_t = 2 * H, g.dk_h = g.dv_h = 2;
        const int64_t most = ((int64_t(1) << 24) - 1) / H;  // T / rows + 1
        if ((most * rows) * H * 2 <= kMost) {
          a.Tq = a.Tk = (most - 1) * rows + rows - 1;
          STATUS(forward(a), LB_OK);
          STATUS(backward(a, g), LB_OK);
        }
        if ((most * rows + rows) * H * 2 > kMost) continue;
        a.Tq = most * rows, a.Tk = 1;
        STATUS(forward(a), LB_ERR_SHAPE);
        STATUS(backward(a, g), LB_ERR_SHAPE);
        a.Tq = 1, a.Tk = most * rows;
        STATUS(forward(a), LB_OK);
        STATUS(backward(a, g), LB_ERR_SHAPE);
      }
    }
  }
  vec_fits = true;
  lb_latent_cache c = cache();
  c.r = 704, c.d_rope = 0;
  // 44 waves a head, and one for eight heads
  STATUS(latent(c, 1, 1500000, 1, 40, 0, at(50), at(60), 1, 1), LB_OK);
  STATUS(latent(c, 1, 1524000, 1, 40, 0, at(50), at(60), 1, 1), LB_ERR_SHAPE);
}

// Operands that share bytes, and parts of one buffer that do not
static void overlaps() {
  const int64_t T = 9, H = 4, Hk = 2, dn = 32, dr = 16, dv = 24, es = 2;
  lb_attention a = attn();
  const lb_attention_grads far = grads();
  STATUS(backward(a, far), LB_OK);
  auto plus = [](const void* p, int64_t n) { return const_cast<char*>(static_cast<const char*>(p)) + n; };
  const void* in[] = {a.q, a.k, a.v, a.k_rope, at(30), at(32), at(34)};
  const int64_t in_bytes[] = {((a.Tq - 1) * a.q_t + (H - 1) * a.q_h + dn + dr) * es, ((T - 1) * a.k_t + (Hk - 1) * a.k_h + dn) * es,
                              ((T - 1) * a.v_t + (Hk - 1) * a.v_h + dv) * es, ((T - 1) * a.kr_t + dr) * es, a.Tq * H * dv * es,
                              a.Tq * H * 4, a.Tq * H * dv * es};
  const int64_t out_bytes[] = {a.Tq * H * (dn + dr) * es, ((T - 1) * far.dk_t + (Hk - 1) * far.dk_h + dn) * es,
                               ((T - 1) * far.dv_t + (Hk - 1) * far.dv_h + dv) * es, T * dr * es};
  auto put = [&](int o, void* p) {
    lb_attention_grads g = far;
    (o == 0 ? g.dq : o == 1 ? g.dk : o == 2 ? g.dv : g.dk_rope) = p;
    return backward(a, g);
  };
  for (int o = 0; o < 4; ++o) {
    for (int i = 0; i < 7; ++i) {
      STATUS(put(o, plus(in[i], 0)), LB_ERR_ARG);
      STATUS(put(o, plus(in[i], in_bytes[i] - 2)), LB_ERR_ARG);
      STATUS(put(o, plus(in[i], in_bytes[i])), LB_OK);
      STATUS(put(o, plus(in[i], 2 - out_bytes[o])), LB_ERR_ARG);
      STATUS(put(o, plus(in[i], -out_bytes[o])), LB_OK);
    }
    const void* out[] = {far.dq, far.dk, far.dv, far.dk_rope};
    for (int p = 0; p < 4; ++p) {
      if (p == o) continue;
      STATUS(put(o, plus(out[p], 0)), LB_ERR_ARG);
      STATUS(put(o, plus(out[p], out_bytes[p])), LB_OK);
    }
    STATUS(backward(a, far, plus(out[o], 0)), LB_ERR_ARG);
  }
  for (int i = 0; i < 7; ++i) STATUS(backward(a, far, plus(in[i], 0)), LB_ERR_ARG);
  // the two parts of the fused layer's dy, and heads that hold key and value next to each other
  lb_attention_grads g = far;
  g.dk_t = g.dv_t = Hk * (dn + dv), g.dv = plus(g.dk, Hk * dn * es);
  STATUS(backward(a, g), LB_OK);
  g.dv = plus(g.dk, (Hk * dn - 1) * es);
  STATUS(backward(a, g), LB_ERR_ARG);
  g.dv = plus(g.dk, (Hk * dn + 1) * es);  // the last value's end is the next token's first key
  STATUS(backward(a, g), LB_ERR_ARG);
  g.dk_h = g.dv_h = dn + dv, g.dv = plus(g.dk, dn * es);
  STATUS(backward(a, g), LB_OK);
  g.dv = plus(g.dk, dn * es - 2);
  STATUS(backward(a, g), LB_ERR_ARG);
  // tokens inside heads
  g.dk_t = dn, g.dv_t = dv, g.dk_h = g.dv_h = T * (dn + dv), g.dv = plus(g.dk, T * dn * es);
  STATUS(backward(a, g), LB_OK);
  g.dv = plus(g.dv, -2);
  STATUS(backward(a, g), LB_ERR_ARG);
  // gradients in the spare columns of the operands' own buffer
  lb_attention b = a;
  b.k_t = 2 * Hk * dn, g = far;
  g.dk = plus(b.k, Hk * dn * es), g.dk_t = b.k_t;
  STATUS(backward(b, g), LB_OK);
  g.dk = plus(g.dk, -2);
  STATUS(backward(b, g), LB_ERR_ARG);
  // one token: strides do not count
  b.Tk = 1, b.k_t = 0, g = far, g.dk = plus(b.k, (Hk * dn) * es), g.dk_t = 0;
  STATUS(backward(b, g), LB_OK);
  // the latent attention's workspace
  const lb_latent_cache c = cache();
  STATUS(latent(c, 3, 4, 2, 160, 40, at(50), at(74)), LB_ERR_ARG);
  STATUS(latent(c, 3, 4, 2, 160, 40, at(50), at(1)), LB_ERR_ARG);
  STATUS(latent(c, 3, 4, 2, 160, 40, at(50), at(50)), LB_ERR_ARG);
  const int64_t need = static_cast<int64_t>(lb_latent_attention_workspace_bytes(3, 2, 4, 16, 8));
  STATUS(latent(c, 3, 4, 2, 160, 40, plus(at(60), need - 2), at(60)), LB_ERR_ARG);
  STATUS(latent(c, 3, 4, 2, 160, 40, plus(at(60), need + need % 2), at(60)), LB_OK);
}

int main() {
  offsets();
  overlaps();
  launch_sizes();
  if (failures == 0) std::printf("sanitized attention checks passed\n");
  return failures == 0 ? 0 : 1;
}
