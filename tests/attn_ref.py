"""64-bit references of the paged latent cache and the attention calls, on the CPU, each with an element-wise bound
of how far a kernel's output may be from it.

Notation of the bounds: a rounding to a type is off by at most u = finfo(type).eps / 2 of the value (HALF below), fp32
operations by 2^-24.  A softmax weight is off by a factor within 1 +- 2 e_s (score and normaliser), where e_s bounds a
score's error: (terms + 4) 2^-24 of the absolute products' sum, 2^-22 of the largest score (its product with log2 e,
the subtraction of the maximum) and 2^-21 for the exponential.  An fp32 sum of n terms is off by n 2^-24 of its
absolute terms' sum.  Where 16-bit floats hold probabilities, those below fp16's normal range are off by up to 2^-25
absolutely."""
import math

import torch

HALF = {torch.float64: 2.0 ** -53, torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
E32 = 2.0 ** -24


def turn(x, positions, freqs, inverse=False):
    """x [T, ..., d] (fp64) turned by positions [T] and freqs [d / 2], pairs (i, i + d / 2)."""
    a = positions.double().view([-1] + [1] * (x.dim() - 1)) * freqs.double()
    if inverse:
        a = -a
    d = x.shape[-1] // 2
    u, v = x[..., :d], x[..., d:]
    return torch.cat([u * a.cos() - v * a.sin(), v * a.cos() + u * a.sin()], dim=-1)


def turn_bound(x, dtype):
    """Of turn's result y rounded to dtype: sin and cos within 2^-22, two products and a sum in fp32."""
    d = x.shape[-1] // 2
    m = x[..., :d].abs() + x[..., d:].abs()
    return torch.cat([m, m], dim=-1) * (HALF[dtype] + 2.0 ** -21) + 1e-30


def small(dtype):
    """The absolute error of a value of `dtype` below its normal range (bf16 and fp32: none that matters)."""
    return 2.0 ** -25 if dtype == torch.float16 else 0.0


class Head:
    """One sequence's one head: q [n, dk], k [m, dk], v [m, dv] in fp64; seen [n, m]."""

    def __init__(self, q, k, v, seen, scale, dtype, extra_score=None):
        self.q, self.k, self.v, self.scale, self.dtype = q, k, v, scale, dtype
        s = q @ k.T * scale
        s = s.masked_fill(~seen, -math.inf)
        self.lse = torch.logsumexp(s, dim=-1) if s.shape[1] else torch.full((q.shape[0],), -math.inf, dtype=torch.float64)
        empty = self.lse == -math.inf
        self.p = torch.exp(s - self.lse.masked_fill(empty, 0.0)[:, None]).masked_fill(~seen, 0.0)
        mag = (q.abs() @ k.abs().T * scale).masked_fill(~seen, 0.0)
        top = mag.amax(-1) if mag.shape[1] else torch.zeros(q.shape[0], dtype=torch.float64)
        big = s.masked_fill(~seen, 0.0).abs().amax(-1) if s.shape[1] else top
        self.es = (q.shape[-1] + 4) * E32 * top + 2.0 ** -22 * big + 2.0 ** -21
        if extra_score is not None:
            self.es = self.es + extra_score
        self.o = self.p @ v
        # a probability's relative error, and the absolute one below the normal range
        self.up = (0.0 if dtype in (torch.float32, torch.float64) else HALF[dtype]) + 2 * self.es + (seen.shape[1] + 4) * E32
        self.o_bound = HALF[dtype] * self.o.abs() + self.up[:, None] * (self.p @ v.abs()) + small(dtype) * (
            seen.double() @ v.abs()) + 1e-30
        self.lse_bound = 2 * self.es + (seen.shape[1] + 4) * E32 + 2.0 ** -22 * self.lse.abs().nan_to_num(posinf=0.0)

    def backward(self, do):
        """dq, dk, dv (fp64) and the bounds of their sums before the final rounding."""
        p, q, k, v, dt = self.p, self.q, self.k, self.v, self.dtype
        n, m = p.shape
        dp = do @ v.T
        d = (do * self.o).sum(-1, keepdim=True)
        ds = p * (dp - d)
        dv = p.T @ do
        e_p = p * self.up[:, None] + small(dt) * (p > 0)
        dv_b = e_p.T @ do.abs() + (n + 4) * E32 * (p.T @ do.abs())
        e_dp = (v.shape[1] + 4) * E32 * (do.abs() @ v.abs().T)
        e_d = (do.abs() * (self.o_bound + v.shape[1] * E32 * self.o.abs())).sum(-1, keepdim=True)
        # dS: its factors' errors and its own rounding; small values keep fp16's steps below the largest |dO| / 8
        u = 0.0 if dt in (torch.float32, torch.float64) else HALF[dt]
        e_ds = p * (e_dp + e_d) + ds.abs() * (u + 2 * self.es[:, None] + 8 * E32) + e_p * 0.0
        if dt == torch.float16:
            e_ds = e_ds + small(dt) * max(float(do.abs().max()), 1e-30) / 8 * (p > 0)
        dq, dk = ds @ k * self.scale, ds.T @ q * self.scale
        dq_b = (e_ds @ k.abs() + (m + 4) * E32 * (ds.abs() @ k.abs())) * self.scale
        dk_b = (e_ds.T @ q.abs() + (n + 4) * E32 * (ds.abs().T @ q.abs())) * self.scale
        return dq, dk, dv, dq_b, dk_b, dv_b


def seen_mask(n, m, causal):
    if not causal:
        return torch.ones((n, m), dtype=torch.bool)
    return torch.arange(m)[None, :] <= torch.arange(n)[:, None] + (m - n)


def attention(q, k, v, kr, lens_q, lens_k, causal, scale, do=None):
    """All sequences and heads: q [Tq, H, dk] ... as CPU tensors of the kernel's dtype.  A dict of results and bounds
    over the rows that belong to a sequence."""
    dt = q.dtype
    H, Hk, dn, dv = q.shape[1], k.shape[1], k.shape[2], v.shape[2]
    dr = 0 if kr is None else kr.shape[1]
    Tq, Tk = sum(lens_q), sum(lens_k)
    z = lambda *s: torch.zeros(s, dtype=torch.float64)  # noqa: E731
    r = dict(o=z(Tq, H, dv), o_b=z(Tq, H, dv), lse=z(Tq, H), lse_b=z(Tq, H))
    if do is not None:
        r.update(dq=z(Tq, H, dn + dr), dq_b=z(Tq, H, dn + dr), dk=z(Tk, Hk, dn), dk_b=z(Tk, Hk, dn), dv=z(Tk, Hk, dv),
                 dv_b=z(Tk, Hk, dv), dkr=z(Tk, dr), dkr_b=z(Tk, dr))
    a = b = 0
    for n, m in zip(lens_q, lens_k):
        seen = seen_mask(n, m, causal)
        for h in range(H):
            g = h // (H // Hk)
            kk = k[b:b + m, g].double()
            if dr:
                kk = torch.cat([kk, kr[b:b + m].double()], dim=-1)
            hd = Head(q[a:a + n, h].double(), kk, v[b:b + m, g].double(), seen, scale, dt)
            r["o"][a:a + n, h], r["o_b"][a:a + n, h] = hd.o, hd.o_bound
            r["lse"][a:a + n, h], r["lse_b"][a:a + n, h] = hd.lse, hd.lse_bound
            if do is not None and n and m:
                dq, dk, dvv, dqb, dkb, dvb = hd.backward(do[a:a + n, h].double())
                r["dq"][a:a + n, h], r["dq_b"][a:a + n, h] = dq, dqb
                r["dk"][b:b + m, g] += dk[:, :dn]
                r["dk_b"][b:b + m, g] += dkb[:, :dn] + E32 * dk[:, :dn].abs()
                r["dv"][b:b + m, g] += dvv
                r["dv_b"][b:b + m, g] += dvb + E32 * dvv.abs()
                r["dkr"][b:b + m] += dk[:, dn:]
                r["dkr_b"][b:b + m] += dkb[:, dn:] + E32 * H * dk[:, dn:].abs()
        a, b = a + n, b + m
    if do is not None:
        for name in ("dq", "dk", "dv", "dkr"):
            r[name + "_b"] += HALF[dt] * r[name].abs() + small(dt) + 1e-30
    return r


def unpack(words, n_out, r):
    """[n_out, r] of +-1 (fp64) from a packed matrix (role U), byte by byte."""
    import numpy as np
    raw = words.cpu().numpy().view("uint8")
    nb, w = divmod(r, 32)
    bits = np.unpackbits(raw[:4 * nb * n_out].reshape(nb, n_out, 4), axis=-1, bitorder="little")
    full = bits.transpose(1, 0, 2).reshape(n_out, 32 * nb)
    if w:
        size = 2 if w <= 16 else 4
        t = raw[4 * nb * n_out:4 * nb * n_out + size * n_out].reshape(n_out, size)
        full = np.concatenate([full, np.unpackbits(t, axis=-1, bitorder="little")[:, :w]], axis=1)
    return torch.from_numpy(np.where(full, -1.0, 1.0))


def latent_attention(q, rows, up, Hk, dv, lens, news, freqs, dr, scale, cache_dtype):
    """out [T, H, dv] and its bound.  rows: per sequence [len, 2 r + dr] fp64 cache contents; up [2 r, Hk (dn + dv)]
    fp64 (signs times h)."""
    dt = q.dtype
    T, H, dq = q.shape
    dn, r2 = dq - dr, up.shape[0]
    out, bound = torch.zeros((T, H, dv), dtype=torch.float64), torch.zeros((T, H, dv), dtype=torch.float64)
    f32 = dt == torch.float32
    # q' in terms of the cache's type: two terms leave u^2, three u^3, fp32 its half step
    u = HALF[cache_dtype]
    uq = u if cache_dtype == torch.float32 else (u ** 3 if cache_dtype == torch.bfloat16 and f32 else u ** 2)
    # ... and fp16's second term ends 2^-25 below the row's largest value
    uq += 2.0 ** -24 if cache_dtype == torch.float16 else 0.0
    up_p = 0.0 if cache_dtype == torch.float32 else ((u ** 3 if cache_dtype == torch.bfloat16 else u ** 2) if f32 else u)
    a = 0
    for m, n, w in zip(lens, news, rows):
        pos = torch.arange(m - n, m)
        seen = torch.arange(m)[None, :] <= pos[:, None]
        for h in range(H):
            g = h // (H // Hk)
            uk, uv = up[:, g * dn:(g + 1) * dn], up[:, Hk * dn + g * dv:Hk * dn + (g + 1) * dv]
            qh = q[a:a + n, h].double()
            qa, mag = qh[:, :dn] @ uk.T, qh[:, :dn].abs() @ uk.abs().T
            if dr:
                qr = qh[:, dn:] if freqs is None else turn(qh[:, dn:], pos, freqs)
                qa, mag = torch.cat([qa, qr], 1), torch.cat([mag, qh[:, dn:].abs().amax(-1, keepdim=True).expand(n, dr) * 2], 1)
            # q': dn sign flips and additions in fp32, then its terms (fp16's relative to the row's largest)
            top = qa.abs().amax(-1, keepdim=True) if cache_dtype == torch.float16 else qa.abs()
            e_q = (dn + 8) * E32 * mag + uq * torch.maximum(qa.abs(), top) + 2.0 ** -21 * mag * (1 if dr else 0)
            extra = scale * (e_q @ w.abs().T).amax(-1) if m else torch.zeros(n, dtype=torch.float64)
            v = w[:, :r2] @ uv
            hd = Head(qa, w, v, seen, scale, torch.float32, extra)
            out[a:a + n, h] = hd.o
            wide = hd.p @ w[:, :r2].abs() @ uv.abs()  # sums run over latents: their magnitude
            tiny = 2.0 ** -25 * (seen.double() @ v.abs()) if cache_dtype == torch.float16 else 0.0
            bound[a:a + n, h] = (HALF[dt] * hd.o.abs() + (up_p + 2 * hd.es + 8 * E32)[:, None] * (hd.p @ v.abs())
                                 + (m + r2 + 64) * E32 * wide + tiny + 1e-30)
        a += n
    return out, bound
