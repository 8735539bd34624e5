// C ABI of the paged latent cache and the attention calls: host-side validation
// and launch.  Nothing is enqueued unless every check has passed.
#include <cmath>
#include <cstring>
#include <numeric>

#include "attn.h"

namespace {

constexpr int64_t kMaxElems = (int64_t(1) << 31) - 1;

template <typename E>
int enum_value(const E& e) {
  static_assert(sizeof(E) == sizeof(int), "enums of the ABI are int-sized");
  int v;
  std::memcpy(&v, &e, sizeof v);
  return v;
}
bool dtype_ok(const lb_dtype& d) {
  const int v = enum_value(d);
  return v == LB_F32 || v == LB_F16 || v == LB_BF16;
}
int64_t dtype_size(lb_dtype d) { return d == LB_F32 ? 4 : 2; }
bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

// a launch's threads are counted in 32 bits: rows (token, head) with a workgroup of up to
// 1024 threads each, workgroups of 256, and single waves
constexpr int64_t kMaxRows = int64_t(1) << 22, kMaxGroups = int64_t(1) << 24, kMaxWaves = int64_t(1) << 26;

// a b (and a b c) below 2^31, all factors >= 0
bool fits(int64_t a, int64_t b) { return a == 0 || b <= kMaxElems / a; }
bool fits(int64_t a, int64_t b, int64_t c) { return fits(a, b) && fits(a * b, c); }

// A strided [T x H x d] operand: strides >= 0, its last row at most twice kMaxOffset elements behind its first
constexpr int64_t kMaxStride = int64_t(1) << 40, kMaxOffset = int64_t(1) << 59;
bool stride_ok(int64_t n, int64_t s) { return s >= 0 && s <= kMaxStride && (n <= 1 || s <= kMaxOffset / (n - 1)); }
bool strides_ok(int64_t T, int64_t H, int64_t st, int64_t sh) { return stride_ok(T, st) && stride_ok(H, sh); }
// elements from the first to one past the last
int64_t span(int64_t T, int64_t H, int64_t d, int64_t st, int64_t sh) { return (T - 1) * st + (H - 1) * sh + d; }
// rows of d elements that share no element: heads inside tokens, or tokens inside heads
bool rows_apart(int64_t T, int64_t H, int64_t d, int64_t st, int64_t sh) {
  if (T == 0 || H == 0 || d == 0) return true;
  const bool heads_in = (H == 1 || sh >= d) && (T == 1 || st >= (H - 1) * sh + d);
  const bool tokens_in = (T == 1 || st >= d) && (H == 1 || sh >= (T - 1) * st + d);
  return heads_in || tokens_in;
}
bool ranges_meet(const void* a, int64_t na, const void* b, int64_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return na > 0 && nb > 0 && x < y + static_cast<uintptr_t>(nb) && y < x + static_cast<uintptr_t>(na);
}

// Bytes of an operand: T x H rows of d at strides st, sh; or n bytes in a row.
struct Region {
  uintptr_t p;
  int64_t T, H, d, st, sh;
};
Region rows_of(const void* p, int64_t T, int64_t H, int64_t d, int64_t st, int64_t sh, int64_t es) {
  return Region{reinterpret_cast<uintptr_t>(p), T, H, d * es, T > 1 ? st * es : 0, H > 1 ? sh * es : 0};
}
Region bytes_of(const void* p, int64_t n) { return Region{reinterpret_cast<uintptr_t>(p), 1, 1, n, 0, 0}; }
// [p, p + e) and [q, q + f), both repeated every g bytes, apart?
bool repeats_apart(uintptr_t p, int64_t e, uintptr_t q, int64_t f, int64_t g) {
  if (g == 0 || e > g || f > g) return false;
  const int64_t m = q >= p ? static_cast<int64_t>((q - p) % g) : (g - static_cast<int64_t>((p - q) % g)) % g;
  return m >= e && m + f <= g;
}
// Whether two operands may share a byte.  Where their spans meet, parts of one buffer are still apart if
// their rows, whole tokens or whole heads keep to places of their own within a common period of the strides.
bool operands_meet(const Region& a, const Region& b) {
  if (a.T <= 0 || a.H <= 0 || a.d <= 0 || b.T <= 0 || b.H <= 0 || b.d <= 0) return false;
  const int64_t ea = (a.H - 1) * a.sh + a.d, eb = (b.H - 1) * b.sh + b.d;  // a token's bytes, all heads
  const int64_t fa = (a.T - 1) * a.st + a.d, fb = (b.T - 1) * b.st + b.d;  // a head's, all tokens
  const uintptr_t na = static_cast<uintptr_t>((a.T - 1) * a.st + ea), nb = static_cast<uintptr_t>((b.T - 1) * b.st + eb);
  if (a.p >= b.p + nb || b.p >= a.p + na) return false;
  const int64_t gt = std::gcd(a.st, b.st), gh = std::gcd(a.sh, b.sh);
  return !repeats_apart(a.p, a.d, b.p, b.d, std::gcd(gt, gh)) && !repeats_apart(a.p, ea, b.p, eb, gt) &&
         !repeats_apart(a.p, fa, b.p, fb, gh);
}

// (T / rows + n_seq + 1) heads workgroups: fewer than a launch may have
bool groups_ok(int64_t T, int rows, int64_t n_seq, int64_t heads) {
  return heads == 0 || T / rows + n_seq + 1 <= (kMaxGroups - 1) / heads;
}

bool cache_sizes_ok(int64_t r, int64_t d_rope) {
  return r >= 1 && d_rope >= 0 && d_rope % 2 == 0 && d_rope <= lb::kMaxRope && r <= lb::kMaxLatentRank &&
         2 * r + d_rope <= lb::kMaxLatentRow;
}

lb_status check_cache(const lb_latent_cache* c) {
  if (!c) return LB_ERR_NULL;
  if (!dtype_ok(c->dtype)) return LB_ERR_DTYPE;
  if (!cache_sizes_ok(c->r, c->d_rope) || c->n_pages < 0 || c->page_size < 1 || c->n_seq < 0 || c->max_pages < 0 ||
      c->n_seq > (1 << 24) || !fits(c->n_pages, c->page_size) || !fits(c->max_pages, c->page_size) ||
      c->max_pages * c->page_size > (1 << 30) || !fits(c->n_seq, c->max_pages))
    return LB_ERR_SHAPE;
  return LB_OK;
}
// the pointers of a cache that a call with work reads
lb_status check_cache_ptrs(const lb_latent_cache* c) {
  if ((c->n_pages > 0 && !c->data) || (c->max_pages > 0 && c->n_seq > 0 && !c->table) || !c->lens || !c->cu)
    return LB_ERR_NULL;
  if (!aligned(c->data, 16) || !aligned(c->table, 4) || !aligned(c->lens, 4) || !aligned(c->cu, 4)) return LB_ERR_ALIGN;
  return LB_OK;
}
lb::CacheArgs cache_args(const lb_latent_cache* c) {
  lb::CacheArgs a{};
  a.data = c->data;
  a.dt = c->dtype;
  a.n_pages = c->n_pages;
  a.page_size = static_cast<int>(c->page_size);
  a.r = static_cast<int>(c->r);
  a.d_rope = static_cast<int>(c->d_rope);
  a.row = lb::latent_row(c->r, c->d_rope);
  a.table = c->table;
  a.n_seq = static_cast<int>(c->n_seq);
  a.max_pages = c->n_pages == 0 ? 0 : static_cast<int>(c->max_pages);  // no page: no token has a place
  a.lens = c->lens;
  a.cu = c->cu;
  return a;
}

lb_status hip_status(hipError_t e) { return e == hipSuccess ? LB_OK : LB_ERR_HIP; }

bool scale_ok(float s) { return std::isfinite(s) && s > 0.0f; }

}  // namespace

extern "C" {

int64_t lb_latent_row(int64_t r, int64_t d_rope) { return cache_sizes_ok(r, d_rope) ? lb::latent_row(r, d_rope) : 0; }

lb_status lb_rotate(const void* x, lb_dtype dtype, int64_t T, int64_t H, int64_t d, int64_t x_t, int64_t x_h,
                    const int32_t* positions, const float* freqs, int inverse, void* y, int64_t y_t, int64_t y_h,
                    hipStream_t stream) {
  if (!dtype_ok(dtype)) return LB_ERR_DTYPE;
  if (T < 0 || H < 0 || d < 0 || d % 2 != 0 || d > lb::kMaxRope || !fits(T, H, d) || !strides_ok(T, H, x_t, x_h) ||
      !strides_ok(T, H, y_t, y_h))
    return LB_ERR_SHAPE;
  if (T == 0 || H == 0 || d == 0) return LB_OK;
  if (!x || !y || !positions || !freqs) return LB_ERR_NULL;
  const int64_t es = dtype_size(dtype);
  if (!aligned(x, es) || !aligned(y, es) || !aligned(positions, 4) || !aligned(freqs, 4)) return LB_ERR_ALIGN;
  if (!rows_apart(T, H, d, y_t, y_h)) return LB_ERR_ARG;
  const bool in_place = x == y && (T == 1 || x_t == y_t) && (H == 1 || x_h == y_h);
  if (!in_place && ranges_meet(x, span(T, H, d, x_t, x_h) * es, y, span(T, H, d, y_t, y_h) * es)) return LB_ERR_ARG;
  lb::RotateArgs a{};
  a.x = x, a.y = y;
  a.dt = dtype;
  a.T = static_cast<int>(T), a.H = static_cast<int>(H), a.d = static_cast<int>(d);
  a.x_t = x_t, a.x_h = x_h, a.y_t = y_t, a.y_h = y_h;
  a.positions = positions, a.freqs = freqs;
  a.inverse = inverse != 0;
  return hip_status(lb::launch_rotate(a, stream));
}

lb_status lb_latent_append(const lb_latent_cache* cache, const void* w, const void* k_rope, int64_t k_rope_t,
                           lb_dtype dtype, int64_t T, const float* freqs, hipStream_t stream) {
  if (!dtype_ok(dtype)) return LB_ERR_DTYPE;
  lb_status st = check_cache(cache);
  if (st != LB_OK) return st;
  if (T < 0 || !fits(T, lb::latent_row(cache->r, cache->d_rope)) || !stride_ok(T, k_rope_t)) return LB_ERR_SHAPE;
  if (T == 0 || cache->n_seq == 0) return LB_OK;
  if (!w || (cache->d_rope > 0 && !k_rope)) return LB_ERR_NULL;
  st = check_cache_ptrs(cache);
  if (st != LB_OK) return st;
  const int64_t es = dtype_size(dtype);
  if (!aligned(w, es) || !aligned(k_rope, es) || !aligned(freqs, 4)) return LB_ERR_ALIGN;
  const lb::CacheArgs c = cache_args(cache);
  const int64_t nc = cache->n_pages * cache->page_size * c.row * dtype_size(cache->dtype);
  if (ranges_meet(cache->data, nc, w, T * 2 * cache->r * es) ||
      (cache->d_rope > 0 && ranges_meet(cache->data, nc, k_rope, span(T, 1, cache->d_rope, k_rope_t, 0) * es)))
    return LB_ERR_ARG;
  lb::AppendArgs a{};
  a.c = c;
  a.w = w, a.k_rope = k_rope;
  a.kr_t = k_rope_t;
  a.dt = dtype;
  a.T = static_cast<int>(T);
  a.freqs = freqs;
  return hip_status(lb::launch_append(a, stream));
}

size_t lb_latent_attention_workspace_bytes(int64_t T, int64_t n_seq, int64_t H, int64_t r, int64_t d_rope) {
  if (T < 0 || n_seq < 0 || n_seq > (1 << 24) || H < 0 || !cache_sizes_ok(r, d_rope) ||
      !fits(T, H, lb::latent_row(r, d_rope)))
    return 0;
  return lb::latent_attn_workspace_bytes(static_cast<int>(T), static_cast<int>(n_seq), static_cast<int>(H),
                                         static_cast<int>(r), static_cast<int>(d_rope));
}

lb_status lb_latent_attention(const void* q, lb_dtype act_dtype, int64_t T, int64_t H, int64_t Hk, int64_t d_nope,
                              int64_t d_v, int64_t q_t, int64_t q_h, const lb_path* paths, lb_dtype scale_dtype,
                              const lb_latent_cache* cache, const float* freqs, float scale, void* out,
                              void* workspace, size_t workspace_bytes, hipStream_t stream) {
  if (!dtype_ok(act_dtype) || !dtype_ok(scale_dtype)) return LB_ERR_DTYPE;
  lb_status st = check_cache(cache);
  if (st != LB_OK) return st;
  if (T < 0 || H < 0 || Hk < 1 || H % Hk != 0 || d_nope < 0 || d_nope > 256 || d_v < 0 || d_v > 256 ||
      !strides_ok(T, H, q_t, q_h) || !fits(T, H, lb::latent_row(cache->r, cache->d_rope)) ||
      !fits(T, H, d_nope + cache->d_rope) || !fits(T, H, d_v) || !fits(Hk, d_nope + d_v, cache->r) || T * H >= kMaxRows)
    return LB_ERR_SHAPE;
  // single waves of absorb: 32 latents, 32 tokens and a head, or eight heads' rotary part
  const int64_t waves = 2 * ((cache->r + 31) / 32) * ((T + 31) / 32) * H + T * ((H + 7) / 8);
  if (waves >= kMaxWaves) return LB_ERR_SHAPE;
  // the kernels count steps of 16 tokens or more of items of 32 query rows in 31 bits
  if (!fits(T * H / 32 + cache->n_seq, cache->max_pages * cache->page_size / 16 + 1)) return LB_ERR_SHAPE;
  if (!scale_ok(scale)) return LB_ERR_ARG;
  if (T == 0 || H == 0 || d_v == 0 || cache->n_seq == 0) return LB_OK;
  if (!out || (d_nope + cache->d_rope > 0 && !q)) return LB_ERR_NULL;
  const int64_t es = dtype_size(act_dtype), ss = dtype_size(scale_dtype);
  if (!aligned(q, es) || !aligned(out, es) || !aligned(freqs, 4)) return LB_ERR_ALIGN;
  if (!paths) return LB_ERR_NULL;
  for (int p = 0; p < 2; ++p) {
    if (!paths[p].U || !paths[p].h) return LB_ERR_NULL;
    if (!aligned(paths[p].U, 4) || !aligned(paths[p].h, ss)) return LB_ERR_ALIGN;
  }
  st = check_cache_ptrs(cache);
  if (st != LB_OK) return st;
  const int64_t no = T * H * d_v * es;
  const int64_t nc = cache->n_pages * cache->page_size * lb::latent_row(cache->r, cache->d_rope) * dtype_size(cache->dtype);
  if (ranges_meet(out, no, q, span(T, H, d_nope + cache->d_rope, q_t, q_h) * es) || ranges_meet(out, no, cache->data, nc))
    return LB_ERR_ARG;
  const size_t need = lb_latent_attention_workspace_bytes(T, cache->n_seq, H, cache->r, cache->d_rope);
  if (!workspace) return LB_ERR_NULL;
  if (!aligned(workspace, 256)) return LB_ERR_ALIGN;
  if (workspace_bytes < need) return LB_ERR_WORKSPACE;
  const Region ws = bytes_of(workspace, static_cast<int64_t>(need));
  if (operands_meet(ws, bytes_of(out, no)) || operands_meet(ws, bytes_of(cache->data, nc)) ||
      operands_meet(ws, rows_of(q, T, H, d_nope + cache->d_rope, q_t, q_h, es)))
    return LB_ERR_ARG;
  lb::LatentAttnArgs a{};
  a.c = cache_args(cache);
  a.q = q;
  a.dt = act_dtype;
  a.T = static_cast<int>(T), a.H = static_cast<int>(H), a.Hk = static_cast<int>(Hk);
  a.d_nope = static_cast<int>(d_nope), a.d_v = static_cast<int>(d_v);
  a.q_t = q_t, a.q_h = q_h;
  for (int p = 0; p < 2; ++p) a.U[p] = paths[p].U, a.h[p] = paths[p].h;
  a.sc_dt = scale_dtype;
  a.freqs = freqs;
  a.scale = scale;
  a.out = out;
  a.ws = workspace;
  return hip_status(lb::launch_latent_attn(a, stream));
}

}  // extern "C"

namespace {

lb_status check_attention(const lb_attention* a) {
  if (!a) return LB_ERR_NULL;
  if (!dtype_ok(a->dtype)) return LB_ERR_DTYPE;
  if (a->Tq < 0 || a->Tk < 0 || a->H < 0 || a->Hk < 1 || a->H % a->Hk != 0 || a->d_nope < 0 || a->d_rope < 0 ||
      a->d_nope > 192 || a->d_rope > 192 || !lb::attn_supports(a->d_nope + a->d_rope, a->d_v) || a->n_seq < 0 ||
      a->n_seq > (1 << 24) || !strides_ok(a->Tq, a->H, a->q_t, a->q_h) || !strides_ok(a->Tk, a->Hk, a->k_t, a->k_h) ||
      !strides_ok(a->Tk, a->Hk, a->v_t, a->v_h) || !stride_ok(a->Tk, a->kr_t))
    return LB_ERR_SHAPE;
  const int64_t dk = a->d_nope + a->d_rope;
  if (!fits(a->Tq, a->H, dk) || !fits(a->Tq, a->H, a->d_v) || !fits(a->Tk, a->Hk, dk) || !fits(a->Tk, a->Hk, a->d_v) ||
      !fits(a->n_seq + 1, a->H) || !groups_ok(a->Tq, 128, a->n_seq, a->H) || !groups_ok(a->Tk, 128, a->n_seq, a->Hk))
    return LB_ERR_SHAPE;
  if ((a->cu_q == nullptr) != (a->cu_k == nullptr) || !scale_ok(a->scale)) return LB_ERR_ARG;
  return LB_OK;
}
lb_status check_attention_ptrs(const lb_attention* a) {
  if (a->Tq > 0 && a->H > 0 && !a->q) return LB_ERR_NULL;
  if (a->Tk > 0 && ((a->d_nope > 0 && !a->k) || !a->v || (a->d_rope > 0 && !a->k_rope))) return LB_ERR_NULL;
  const int64_t es = dtype_size(a->dtype);
  if (!aligned(a->q, es) || !aligned(a->k, es) || !aligned(a->v, es) || !aligned(a->k_rope, es) ||
      !aligned(a->cu_q, 4) || !aligned(a->cu_k, 4))
    return LB_ERR_ALIGN;
  return LB_OK;
}
// 16-bit operands that cannot be read 16 bytes at a time have 32 rows a workgroup (otherwise 32
// only where that makes few)
bool launch_ok(const lb::AttnArgs& a, bool backward) {
  const int rows = a.dt != LB_F32 && !lb::attn_vec(a, backward) ? 32 : 128;
  return groups_ok(a.Tq, rows, a.n_seq, a.H) && (!backward || groups_ok(a.Tk, rows, a.n_seq, a.Hk));
}
lb::AttnArgs attention_args(const lb_attention* a) {
  lb::AttnArgs r{};
  r.q = a->q, r.k = a->k, r.v = a->v, r.k_rope = a->k_rope;
  r.dt = a->dtype;
  r.Tq = static_cast<int>(a->Tq), r.Tk = static_cast<int>(a->Tk);
  r.H = static_cast<int>(a->H), r.Hk = static_cast<int>(a->Hk);
  r.d_nope = static_cast<int>(a->d_nope), r.d_rope = static_cast<int>(a->d_rope), r.d_v = static_cast<int>(a->d_v);
  r.q_t = a->q_t, r.q_h = a->q_h, r.k_t = a->k_t, r.k_h = a->k_h, r.v_t = a->v_t, r.v_h = a->v_h, r.kr_t = a->kr_t;
  r.cu_q = a->cu_q, r.cu_k = a->cu_k;
  r.n_seq = static_cast<int>(a->n_seq);
  r.causal = a->causal != 0;
  r.scale = a->scale;
  return r;
}

size_t up256(int64_t n) { return static_cast<size_t>((n + 255) / 256 * 256); }

}  // namespace

extern "C" {

lb_status lb_attention_forward(const lb_attention* a, void* o, float* lse, hipStream_t stream) {
  lb_status st = check_attention(a);
  if (st != LB_OK) return st;
  if (a->Tq == 0 || a->H == 0 || (a->cu_q && a->n_seq == 0)) return LB_OK;
  st = check_attention_ptrs(a);
  if (st != LB_OK) return st;
  if (!o) return LB_ERR_NULL;
  const int64_t es = dtype_size(a->dtype);
  if (!aligned(o, es) || !aligned(lse, 4)) return LB_ERR_ALIGN;
  const int64_t no = a->Tq * a->H * a->d_v * es, nl = lse ? a->Tq * a->H * 4 : 0;
  const int64_t dk = a->d_nope + a->d_rope;
  auto meets = [&](const void* p, int64_t n) { return ranges_meet(o, no, p, n) || ranges_meet(lse, nl, p, n); };
  if (ranges_meet(o, no, lse, nl) || meets(a->q, span(a->Tq, a->H, dk, a->q_t, a->q_h) * es) ||
      (a->Tk > 0 && (meets(a->k, a->d_nope ? span(a->Tk, a->Hk, a->d_nope, a->k_t, a->k_h) * es : 0) ||
                     meets(a->v, span(a->Tk, a->Hk, a->d_v, a->v_t, a->v_h) * es) ||
                     meets(a->k_rope, a->d_rope ? span(a->Tk, 1, a->d_rope, a->kr_t, 0) * es : 0))))
    return LB_ERR_ARG;
  lb::AttnArgs r = attention_args(a);
  r.o = o, r.lse = lse;
  if (!launch_ok(r, false)) return LB_ERR_SHAPE;
  return hip_status(lb::launch_attn_forward(r, stream));
}

size_t lb_attention_backward_workspace_bytes(int64_t Tq, int64_t Tk, int64_t H, int64_t Hk, int64_t d_rope) {
  if (Tq < 0 || Tk < 0 || H < 0 || Hk < 1 || H % Hk != 0 || d_rope < 0 || d_rope > 192 || !fits(Tq, H) ||
      !fits(Tk, Hk, d_rope))
    return 0;
  const size_t n = up256(Tq * H * 4) + up256(Tk * Hk * d_rope * 4);
  return n > 0 ? n : 256;
}

lb_status lb_attention_backward(const lb_attention* a, const void* o, const float* lse, const void* d_o,
                                const lb_attention_grads* grads, void* workspace, size_t workspace_bytes,
                                hipStream_t stream) {
  lb_status st = check_attention(a);
  if (st != LB_OK) return st;
  if (!grads) return LB_ERR_NULL;
  if (!strides_ok(a->Tk, a->Hk, grads->dk_t, grads->dk_h) || !strides_ok(a->Tk, a->Hk, grads->dv_t, grads->dv_h))
    return LB_ERR_SHAPE;
  if (a->H == 0 || (a->Tq == 0 && a->Tk == 0) || (a->cu_q && a->n_seq == 0)) return LB_OK;
  st = check_attention_ptrs(a);
  if (st != LB_OK) return st;
  if (a->Tq > 0 && (!o || !lse || !d_o || !grads->dq)) return LB_ERR_NULL;
  if (a->Tk > 0 && ((a->d_nope > 0 && !grads->dk) || !grads->dv || (a->d_rope > 0 && !grads->dk_rope)))
    return LB_ERR_NULL;
  const int64_t es = dtype_size(a->dtype);
  if (!aligned(o, es) || !aligned(lse, 4) || !aligned(d_o, es) || !aligned(grads->dq, es) || !aligned(grads->dk, es) ||
      !aligned(grads->dv, es) || !aligned(grads->dk_rope, es))
    return LB_ERR_ALIGN;
  if (!rows_apart(a->Tk, a->Hk, a->d_nope, grads->dk_t, grads->dk_h) ||
      !rows_apart(a->Tk, a->Hk, a->d_v, grads->dv_t, grads->dv_h))
    return LB_ERR_ARG;
  const size_t need = lb_attention_backward_workspace_bytes(a->Tq, a->Tk, a->H, a->Hk, a->d_rope);
  if (!workspace) return LB_ERR_NULL;
  if (!aligned(workspace, 256)) return LB_ERR_ALIGN;
  if (workspace_bytes < need) return LB_ERR_WORKSPACE;
  lb::AttnArgs r = attention_args(a);
  r.o = const_cast<void*>(o);
  r.lse = const_cast<float*>(lse);
  r.d_o = d_o;
  r.dq = grads->dq, r.dk = grads->dk, r.dv = grads->dv, r.dkr = grads->dk_rope;
  r.dk_t = grads->dk_t, r.dk_h = grads->dk_h, r.dv_t = grads->dv_t, r.dv_h = grads->dv_h;
  if (!launch_ok(r, true)) return LB_ERR_SHAPE;
  const int64_t dk = a->d_nope + a->d_rope, no = a->Tq * a->H * a->d_v * es;
  const Region in[] = {rows_of(a->q, a->Tq, a->H, dk, a->q_t, a->q_h, es), rows_of(a->k, a->Tk, a->Hk, a->d_nope, a->k_t, a->k_h, es),
                       rows_of(a->v, a->Tk, a->Hk, a->d_v, a->v_t, a->v_h, es), rows_of(a->k_rope, a->Tk, 1, a->d_rope, a->kr_t, 0, es),
                       bytes_of(o, no), bytes_of(lse, a->Tq * a->H * 4), bytes_of(d_o, no)};
  const Region out[] = {bytes_of(grads->dq, a->Tq * a->H * dk * es),
                        rows_of(grads->dk, a->Tk, a->Hk, a->d_nope, grads->dk_t, grads->dk_h, es),
                        rows_of(grads->dv, a->Tk, a->Hk, a->d_v, grads->dv_t, grads->dv_h, es),
                        bytes_of(grads->dk_rope, a->Tk * a->d_rope * es), bytes_of(workspace, static_cast<int64_t>(need))};
  constexpr int n_out = sizeof out / sizeof *out;
  for (int i = 0; i < n_out; ++i) {
    for (const Region& x : in)
      if (operands_meet(out[i], x)) return LB_ERR_ARG;
    for (int j = i + 1; j < n_out; ++j)
      if (operands_meet(out[i], out[j])) return LB_ERR_ARG;
  }
  char* ws = static_cast<char*>(workspace);
  r.delta = reinterpret_cast<float*>(ws);
  r.dkr_part = reinterpret_cast<float*>(ws + up256(a->Tq * a->H * 4));
  return hip_status(lb::launch_attn_backward(r, stream));
}

}  // extern "C"
