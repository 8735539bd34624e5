"""Operators of the paged latent cache and of the attention over it: what is measured, with plain forms, inputs, work and 64-bit results.

Each case is a dict of plain values.  `kind` picks the operator:
  rotate   lb_rotate: the position rotation of heads' rotary parts (and its transpose, for gradients)
  append   lb_latent_append: latents and a rotary key into a paged cache, rotated on the way
  latent   lb_latent_attention: attention read from the paged latent cache, the up-projection absorbed
  prompt   lb_attention_forward: attention over expanded keys and values of packed prompts
  train    lb_attention_forward and lb_attention_backward of packed sequences
A token's cache row is [w (2 r) | rotary key (d_rope) | zeros up to a multiple of 32].  The fused key/value projection is one
LittleBit linear with d_out = Hk (d_nope + d_v): the heads' keys first, then the heads' values.
Head counts and widths are those of the Llama-2 7B, 13B and 70B attention, ranks those of their fused K/V projection at 0.1 and
0.55 bits per weight, and generic ragged ones.
"""
import math

import numpy as np
import torch

own = False

_DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "f16": 2, "bf16": 2}
_BASE = 10000.0


def listed():
    return [
        # the rotary key of a few new tokens: the smallest call
        dict(name="rotate_key_f32_T5", kind="rotate", T=5, H=1, d=64, tail=64, pos=4096, inverse=False, act="f32"),
        # the rotary parts of a 7B model's queries (the last 64 of 192 values of a head), 8192 tokens of a training batch
        dict(name="rotate_7b_q_T8192", kind="rotate", T=8192, H=32, d=64, tail=192, pos=8192, inverse=False, act="bf16"),
        # one decoding step of 64 sequences: a token each into a bf16 cache
        dict(name="append_7b_decode_B64", kind="append", B=64, nq=1, lo=100, hi=4000, r=112, dr=64, page=64, act="bf16",
             cache="bf16"),
        # eight prompts of 100 to 2500 tokens, fp32 latents rounded into an f16 cache with pages of 100 tokens
        dict(name="append_13b_prompts", kind="append", B=8, nq=0, lo=100, hi=2500, r=144, dr=64, page=100, act="f32",
             cache="f16"),
        # one sequence of a 7B model decoding at 4096 tokens: latency, few rows, a long axis
        dict(name="latent_7b_B1_L4096", kind="latent", B=1, nq=1, lo=4096, hi=4096, H=32, Hk=32, dn=128, dv=128, r=112, dr=64,
             page=64, act="bf16", cache="bf16"),
        # a serving batch: 32 sequences of 2048 to 16384 tokens
        dict(name="latent_7b_B32_L16384", kind="latent", B=32, nq=1, lo=2048, hi=16384, H=32, Hk=32, dn=128, dv=128, r=112,
             dr=64, page=64, act="bf16", cache="bf16"),
        # a 70B model's grouped heads, four tokens a sequence (drafted tokens checked together), f16
        dict(name="latent_70b_B8_nq4", kind="latent", B=8, nq=4, lo=777, hi=6000, H=64, Hk=8, dn=128, dv=128, r=64, dr=64,
             page=48, act="f16", cache="f16"),
        # a wide latent: 7B at 0.55 bits per weight, no rotary key
        dict(name="latent_7b_055_B8", kind="latent", B=8, nq=1, lo=1000, hi=4000, H=32, Hk=32, dn=128, dv=128, r=720, dr=0,
             page=64, act="bf16", cache="bf16"),
        # packed prompts of a 7B model, 8192 tokens in all
        dict(name="prompt_7b_T8192", kind="prompt", B=4, total=8192, H=32, Hk=32, dn=128, dr=64, dv=128, causal=True, act="bf16"),
        # a short f16 prompt batch with grouped heads and odd lengths
        dict(name="prompt_70b_T777", kind="prompt", B=3, total=777, H=64, Hk=8, dn=128, dr=0, dv=128, causal=True, act="f16"),
        # attention of one training step on 2 x 2048 tokens, forward and backward
        dict(name="train_7b_T4096", kind="train", B=2, total=4096, H=32, Hk=32, dn=128, dr=64, dv=128, causal=True, act="bf16"),
        # a small fp32 model with odd head widths, ragged lengths, all keys seen
        dict(name="train_small_f32", kind="train", B=5, total=600, H=6, Hk=3, dn=40, dr=16, dv=56, causal=False, act="f32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotate", "append", "latent", "latent", "latent", "prompt", "prompt", "train", "train"])
    act = rng.choice(["bf16", "bf16", "f16", "f32"])
    if kind == "rotate":
        H, d = rng.choice([1, 8, 32, 40]), rng.choice([32, 64, 128, 2 * rng.randrange(5, 64)])
        return dict(kind=kind, T=_log(rng, 1, 6000), H=H, d=d, tail=d + rng.choice([0, 64, 128, 37]), pos=_log(rng, 100, 1000000),
                    inverse=rng.random() < 0.4, act=act)
    r, dr = _log(rng, 16, 256), rng.choice([0, 32, 64, 64])
    page = rng.choice([16, 48, 64, 64, 100, 256])
    if kind == "append":
        lo = _log(rng, 1, 1000)
        return dict(kind=kind, B=_log(rng, 1, 64), nq=rng.choice([0, 1, 1, 4]), lo=lo, hi=lo + _log(rng, 1, 1500), r=r, dr=dr,
                    page=page, act=act, cache=rng.choice(["bf16", "f16", "f32"]))
    H, Hk = rng.choice([(32, 32), (40, 40), (64, 8), (32, 8), (6, 2), (5, 5)])
    dn, dv = rng.choice([(128, 128), (128, 128), (64, 64), (96, 64), (40, 56)])
    if kind == "latent":
        if rng.random() < 0.2:
            r = _log(rng, 256, 800)
        hi = _log(rng, 16, 8192)
        return dict(kind=kind, B=_log(rng, 1, 24), nq=rng.choice([1, 1, 1, 2, 5, 8]), lo=max(8, hi // rng.choice([1, 2, 10])), hi=max(8, hi),
                    H=H, Hk=Hk, dn=dn, dv=dv, r=r, dr=dr, page=page, act=act, cache=act if rng.random() < 0.7 else "bf16")
    if act == "f32" and kind == "train":
        H, Hk = rng.choice([(8, 8), (6, 3), (16, 4)])
    B = _log(rng, 1, 8)
    return dict(kind=kind, B=B, total=max(4 * B, _log(rng, 64, 4096 if kind == "prompt" else 2500)), H=H, Hk=Hk, dn=dn, dr=dr, dv=dv,
                causal=rng.random() < 0.8, act=act)


# ----------------------------------------------------------------------------
# sizes of a case
# ----------------------------------------------------------------------------
def _lens(case):
    """Cached tokens of each sequence after the call: spread from lo to hi over their logarithm, in mixed order."""
    B, lo, hi = case["B"], case["lo"], case["hi"]
    v = [max(1, round(lo * (hi / lo) ** (i / max(1, B - 1)))) if B > 1 else hi for i in range(B)]
    return [v[(i * 7 + 3) % B] for i in range(B)] if B % 7 else v


def _news(case):
    """New tokens of each sequence: nq, or (nq = 0) all of them."""
    return [min(case["nq"], n) if case["nq"] else n for n in _lens(case)]


def _prompts(case):
    """Lengths of the packed sequences: uneven, summing to total."""
    B, total = case["B"], case["total"]
    cut = [round(total * (i / B) ** 1.3) for i in range(B + 1)]
    return [cut[i + 1] - cut[i] for i in range(B)]


def _row(case):
    return -(-(2 * case["r"] + case["dr"]) // 32) * 32


def _cum(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)


# ----------------------------------------------------------------------------
# inputs
# ----------------------------------------------------------------------------
def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 29)

    def normal(*shape, std=1.0):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * std

    def freqs(d):
        return torch.tensor([_BASE ** (-2.0 * i / d) for i in range(d // 2)], dtype=torch.float64).float().cuda()

    def ints(v):
        return torch.tensor([int(x) for x in v], dtype=torch.int32, device="cuda")

    kind, s = case["kind"], dict(case)
    if kind == "rotate":
        x = normal(case["T"], case["H"], case["tail"]).to(_DT[case["act"]])
        s["x"] = x[..., case["tail"] - case["d"]:]  # the last d values of each head
        s["positions"] = torch.randint(0, case["pos"], (case["T"],), generator=g, device="cuda", dtype=torch.int32)
        s["freqs"] = freqs(case["d"])
        return s
    if kind in ("append", "latent"):
        lens, news, row, page, r, dr = _lens(case), _news(case), _row(case), case["page"], case["r"], case["dr"]
        need = [-(-n // page) for n in lens]
        n_pages = sum(need) + 3
        order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
        starts = _cum(need)
        table = torch.full((case["B"], max(need)), -1, dtype=torch.int32, device="cuda")
        cells = np.concatenate([b * max(need) + np.arange(n) for b, n in enumerate(need)])
        table.view(-1)[torch.from_numpy(cells).cuda()] = order[:int(starts[-1])]
        cache = normal(n_pages, page, row).to(_DT[case["cache"]])
        cache[..., 2 * r + dr:] = 0
        s.update(cache=cache, table=table, lens=ints(lens), cu=ints(_cum(news)))
        T = sum(news)
        s["freqs"] = freqs(dr) if dr else None
        if kind == "append":
            s["w"] = normal(T, 2, r).to(_DT[case["act"]])
            s["k_rope"] = normal(T, dr).to(_DT[case["act"]]) if dr else None
            return s
        H, Hk, dn, dv = (case[k] for k in ("H", "Hk", "dn", "dv"))
        d_out = Hk * (dn + dv)
        s["q"] = normal(T, H, dn + dr, std=1.5).to(_DT[case["act"]])
        s["U"], s["h"] = [], []
        for p in range(2):
            nb, w = divmod(r, 32)
            a = torch.randint(0, 256, (4 * nb * d_out,), generator=g, device="cuda", dtype=torch.uint8)
            b = torch.randint(0, 1 << w, (d_out,), generator=g, device="cuda", dtype=torch.int64)
            b = b.to(torch.int16 if w <= 16 else torch.int32).view(torch.uint8)
            s["U"].append(torch.cat([a, b]) if w else a)
            # keys and values of standard deviation near 1
            s["h"].append((normal(d_out).abs() * 0.8 / math.sqrt(2 * r) + 0.1 / math.sqrt(2 * r)).to(torch.float16))
        return s
    lens, H, Hk, dn, dr, dv = _prompts(case), case["H"], case["Hk"], case["dn"], case["dr"], case["dv"]
    T, dt = sum(lens), _DT[case["act"]]
    s["cu"] = ints(_cum(lens))
    s["q"] = normal(T, H, dn + dr, std=1.5).to(dt)
    y = normal(T, Hk * (dn + dv)).to(dt)  # what the fused K/V projection gives: keys, then values
    s["k"], s["v"] = y[:, :Hk * dn].view(T, Hk, dn), y[:, Hk * dn:].view(T, Hk, dv)
    s["k_rope"] = normal(T, dr).to(dt) if dr else None
    if kind == "train":
        s["do"] = normal(T, H, dv).to(dt)
    return s


def _scale(case):
    return 1.0 / math.sqrt(case["dn"] + case["dr"])


# ----------------------------------------------------------------------------
# one pass
# ----------------------------------------------------------------------------
def run(s):
    if own:
        return _run_own(s)
    return {"rotate": _rotate, "append": _append, "latent": _latent, "prompt": _prompt, "train": _train}[s["kind"]](s)


def _run_own(s):
    import paper_2506_13771_amd as lb
    kind = s["kind"]
    if kind == "rotate":
        return lb.lb_rotate(s["x"], s["positions"], s["freqs"], inverse=s["inverse"])
    if kind == "append":
        c = s.setdefault("_cache", lb.LatentCache(s["cache"], s["r"], s["dr"]))
        lb.lb_latent_append(c, s["w"], s["k_rope"], s["freqs"], s["table"], s["lens"], s["cu"])
        return s["cache"]
    if kind == "latent":
        if "_plan" not in s:  # what a server keeps: the layer, the cache and a workspace
            layer = [lb.LittleBitPath(U=U, V=None, h=h, g=None, l=None) for U, h in zip(s["U"], s["h"])]
            c = lb.LatentCache(s["cache"], s["r"], s["dr"])
            n = lb.lb_latent_attention_workspace_bytes(s["q"].shape[0], s["B"], s["H"], s["r"], s["dr"])
            s["_plan"] = (c, layer, torch.empty(max(n, 256), dtype=torch.uint8, device="cuda"))
        c, layer, ws = s["_plan"]
        return lb.lb_latent_attention(s["q"], c, layer, s["Hk"], s["dv"], s["table"], s["lens"], s["cu"], s["freqs"],
                                      scale=_scale(s), workspace=ws)
    o, lse = lb.lb_attention_forward(s["q"], s["k"], s["v"], s["k_rope"], s["cu"], s["cu"], causal=s["causal"], scale=_scale(s))
    if kind == "prompt":
        return {"o": o, "lse": lse}
    dq, dk, dv, dkr = lb.lb_attention_backward(s["q"], s["k"], s["v"], s["k_rope"], o, lse, s["do"], s["cu"], s["cu"],
                                               causal=s["causal"], scale=_scale(s))
    return {"o": o, "lse": lse, "dq": dq, "dk": dk, "dv": dv, "dkr": dkr}


def _turn(x, positions, freqs, inverse=False):
    """x [T, H, d] fp32 rotated; the angles in 64 bits."""
    a = positions.double()[:, None] * freqs.double()[None, :]
    c, n = torch.cos(a).float()[:, None, :], torch.sin(a).float()[:, None, :]
    if inverse:
        n = -n
    d = x.shape[-1] // 2
    u, v = x[..., :d], x[..., d:]
    return torch.cat([u * c - v * n, v * c + u * n], dim=-1)


def _rotate(s):
    return _turn(s["x"].float(), s["positions"], s["freqs"], s["inverse"]).to(s["x"].dtype)


def _places(s, T):
    """(sequence, position) of each new token."""
    t = torch.arange(T, device="cuda")
    cu = s["cu"].long()
    b = torch.searchsorted(cu, t, right=True) - 1
    return b, s["lens"].long()[b] - (cu[b + 1] - t)


def _append(s):
    r, dr, page, cache = s["r"], s["dr"], s["page"], s["cache"]
    T = s["w"].shape[0]
    b, pos = _places(s, T)
    slot = s["table"].long()[b, pos // page] * page + pos % page
    rows = torch.zeros((T, cache.shape[-1]), dtype=torch.float32, device="cuda")
    rows[:, :2 * r] = s["w"].reshape(T, 2 * r).float()
    if dr:
        rows[:, 2 * r:2 * r + dr] = _turn(s["k_rope"].float()[:, None, :], pos, s["freqs"])[:, 0]
    cache.view(-1, cache.shape[-1])[slot] = rows.to(cache.dtype)
    return cache


def _signs(buf, n_out, r):
    """[r, n_out] signs of a packed matrix (fp32)."""
    nb, w = divmod(r, 32)
    words = buf[:4 * nb * n_out].view(torch.int32).view(nb, 1, n_out)
    bits = ((words >> torch.arange(32, device="cuda", dtype=torch.int32)[None, :, None]) & 1).reshape(32 * nb, n_out)
    if w:
        t = buf[4 * nb * n_out:].view(torch.int16 if w <= 16 else torch.int32).int()[None, :]
        bits = torch.cat([bits, (t >> torch.arange(w, device="cuda", dtype=torch.int32)[:, None]) & 1])
    return 1.0 - 2.0 * bits.float()


def _latent(s):
    H, Hk, dn, dv, r, dr, B, page = (s[k] for k in ("H", "Hk", "dn", "dv", "r", "dr", "B", "page"))
    d_out, T, G = Hk * (dn + dv), s["q"].shape[0], s["H"] // s["Hk"]
    up = torch.cat([_signs(s["U"][p], d_out, r) * s["h"][p].float() for p in range(2)])  # [2r, d_out]
    up_k = up[:, :Hk * dn].view(2 * r, Hk, dn).permute(1, 2, 0).contiguous()              # [Hk, dn, 2r]
    up_v = up[:, Hk * dn:].view(2 * r, Hk, dv).permute(1, 0, 2).contiguous()              # [Hk, 2r, dv]
    q = s["q"].float()
    b, pos = _places(s, T)
    qa = torch.matmul(q[..., :dn].reshape(T, Hk, G, dn).transpose(0, 1).reshape(Hk, T * G, dn), up_k)
    qa = qa.reshape(Hk, T, G, 2 * r).transpose(0, 1).reshape(T, H, 2 * r)
    if dr:
        qa = torch.cat([qa, _turn(q[..., dn:], pos, s["freqs"])], dim=-1)
    # every sequence has the same number of new tokens here
    nq, L = T // B, int(s["hi"])
    at = torch.arange(L, device="cuda")
    pages = s["table"].long()[:, at // page].clamp_min(0)
    rows = s["cache"].view(-1, s["cache"].shape[-1])[pages * page + at % page][..., :2 * r + dr].float()  # [B, L, 2r + dr]
    sc = torch.matmul(qa.reshape(B, nq * H, 2 * r + dr), rows.transpose(1, 2)) * _scale(s)
    seen = at[None, None, :] <= pos.view(B, nq, 1)
    sc = sc.reshape(B, nq, H, L).masked_fill(~seen[:, :, None, :], -math.inf)
    p = torch.exp(sc - sc.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True)
    ol = torch.matmul(p.reshape(B, nq * H, L), rows[..., :2 * r]).reshape(T, Hk, G, 2 * r)
    o = torch.matmul(ol.transpose(0, 1).reshape(Hk, T * G, 2 * r), up_v).reshape(Hk, T, G, dv)
    return o.transpose(0, 1).reshape(T, H, dv).to(s["q"].dtype)


def _seen(s, T):
    t = torch.arange(T, device="cuda")
    b = torch.searchsorted(s["cu"].long(), t, right=True)
    m = b[:, None] == b[None, :]
    return m & (t[:, None] >= t[None, :]) if s["causal"] else m


def _heads(s):
    """q, k, v in fp32 as [H, T, d], the shared rotary key and grouped heads repeated."""
    T, Hk, G = s["q"].shape[0], s["Hk"], s["H"] // s["Hk"]
    k = s["k"].float()
    if s["dr"]:
        k = torch.cat([k, s["k_rope"].float()[:, None, :].expand(T, Hk, s["dr"])], dim=-1)
    def rep(x):
        return x.transpose(0, 1).repeat_interleave(G, dim=0)
    return s["q"].float().transpose(0, 1), rep(k), rep(s["v"].float())


def _soft(s, q, k):
    sc = (torch.matmul(q, k.transpose(1, 2)) * _scale(s)).masked_fill(~_seen(s, q.shape[1])[None], -math.inf)
    m = sc.amax(-1, keepdim=True)
    p = torch.exp(sc - m)
    l = p.sum(-1, keepdim=True)
    return p / l, (m + torch.log(l))[..., 0]


def _prompt(s):
    q, k, v = _heads(s)
    p, lse = _soft(s, q, k)
    return {"o": torch.matmul(p, v).transpose(0, 1).to(s["q"].dtype), "lse": lse.transpose(0, 1).contiguous()}


def _train(s):
    q, k, v = _heads(s)
    T, H, Hk, dn, dr = q.shape[1], s["H"], s["Hk"], s["dn"], s["dr"]
    dt = s["q"].dtype
    p, lse = _soft(s, q, k)
    o = torch.matmul(p, v)
    do = s["do"].float().transpose(0, 1)
    dv = torch.matmul(p.transpose(1, 2), do)
    ds = p * (torch.matmul(do, v.transpose(1, 2)) - (do * o).sum(-1, keepdim=True)) * _scale(s)
    dq = torch.matmul(ds, k)
    dk = torch.matmul(ds.transpose(1, 2), q)
    def shared(x):
        return x.reshape(Hk, H // Hk, T, x.shape[-1]).sum(1).transpose(0, 1)
    return {"o": o.transpose(0, 1).to(dt), "lse": lse.transpose(0, 1).contiguous(), "dq": dq.transpose(0, 1).to(dt),
            "dk": shared(dk[..., :dn]).to(dt), "dv": shared(dv).to(dt),
            "dkr": dk[..., dn:].sum(0).to(dt) if dr else None}


# ----------------------------------------------------------------------------
# the least work of one pass
# ----------------------------------------------------------------------------
def _pairs(lens, causal):
    return sum(n * (n + 1) // 2 if causal else n * n for n in lens)


def work(case):
    kind, e = case["kind"], _BYTES[case["act"]]
    if kind == "rotate":
        n = case["T"] * case["H"] * case["d"]
        return {"bytes": 2 * n * e + 4 * case["T"], "flops": 3 * n}
    if kind == "append":
        T, n = sum(_news(case)), 2 * case["r"] + case["dr"]
        return {"bytes": T * (n * e + _row(case) * _BYTES[case["cache"]]), "flops": 3 * T * case["dr"]}
    H, Hk, dn, dv, dr = (case[k] for k in ("H", "Hk", "dn", "dv", "dr"))
    if kind == "latent":
        lens, news, r = _lens(case), _news(case), case["r"]
        T = sum(news)
        pairs = sum(q * n - q * (q - 1) // 2 for q, n in zip(news, lens)) * H
        d_out = Hk * (dn + dv)
        return {"bytes": sum(lens) * (2 * r + dr) * _BYTES[case["cache"]] + T * H * (dn + dr + dv) * e + 2 * d_out * (r / 8 + 2),
                "flops": pairs * 2 * (4 * r + dr) + 2 * T * H * (dn + dv) * 2 * r}
    lens, dk = _prompts(case), dn + dr
    T, pairs = sum(lens), _pairs(lens, case["causal"]) * H
    b = T * (H * (dk + dv) + Hk * (dn + dv) + dr) * e + 4 * T * H
    if kind == "prompt":
        return {"bytes": b, "flops": 2 * pairs * (dk + dv)}
    return {"bytes": b + T * (H * (dk + dv) + Hk * (dn + dv) + dr) * e, "flops": 2 * pairs * (4 * dk + 3 * dv)}


# ----------------------------------------------------------------------------
# 64-bit results, from the definitions, one sequence and head at a time
# ----------------------------------------------------------------------------
def _rot64(x, pos, freqs):
    d = x.shape[-1] // 2
    z = torch.complex(x[..., :d], x[..., d:])
    a = pos.double().reshape(-1, 1) * freqs.double().reshape(1, -1)
    z = z * torch.polar(torch.ones_like(a), a).reshape([a.shape[0]] + [1] * (x.dim() - 2) + [d])
    return torch.cat([z.real, z.imag], dim=-1)


def _dense64(buf, n_out, r):
    """The packed matrix as [n_out, r] of +-1, read byte by byte."""
    raw = buf.cpu().numpy()
    nb, w = divmod(r, 32)
    bits = np.unpackbits(raw[:4 * nb * n_out].reshape(nb, n_out, 4), axis=-1, bitorder="little")
    full = bits.transpose(1, 0, 2).reshape(n_out, 32 * nb)
    if w:
        tail = np.unpackbits(raw[4 * nb * n_out:].reshape(n_out, -1), axis=-1, bitorder="little")[:, :w]
        full = np.concatenate([full, tail], axis=1)
    return torch.from_numpy(np.where(full, -1.0, 1.0)).cuda()


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "rotate":
        return _rot64(s["x"].double(), -s["positions"] if case["inverse"] else s["positions"], s["freqs"])
    r, dr = case.get("r"), case["dr"] if "dr" in case else 0
    if kind in ("append", "latent"):
        lens, news, page = _lens(case), _news(case), case["page"]
        flat = s["cache"].double().view(-1, s["cache"].shape[-1])
        tab = s["table"].long()
    if kind == "append":
        t = 0
        for b, (n, q) in enumerate(zip(lens, news)):
            p = torch.arange(n - q, n, device="cuda")
            new = [s["w"][t:t + q].double().reshape(q, 2 * r)]
            if dr:
                new.append(_rot64(s["k_rope"][t:t + q].double(), p, s["freqs"]))
            flat[tab[b, p // page] * page + p % page, :2 * r + dr] = torch.cat(new, dim=-1)
            t += q
        return flat.view(s["cache"].shape)
    H, Hk, dn, dv = (case[k] for k in ("H", "Hk", "dn", "dv"))
    sc = _scale(case)
    if kind == "latent":
        d_out = Hk * (dn + dv)
        dense = torch.cat([s["h"][p].double()[:, None] * _dense64(s["U"][p], d_out, r) for p in range(2)], dim=1)
        out, t = [], 0
        for b, (n, nq) in enumerate(zip(lens, news)):
            at = torch.arange(n, device="cuda")
            rows = flat[tab[b, at // page] * page + at % page]
            kv = rows[:, :2 * r] @ dense.T  # the expanded keys and values of all heads
            pos = torch.arange(n - nq, n, device="cuda")
            q = s["q"][t:t + nq].double()
            qr = _rot64(q[..., dn:], pos, s["freqs"]) if dr else None
            hide = at[None, :] > pos[:, None]
            o = []
            for h in range(H):
                kh = h // (H // Hk)
                a = q[:, h, :dn] @ kv[:, kh * dn:(kh + 1) * dn].T
                if dr:
                    a = a + qr[:, h] @ rows[:, 2 * r:2 * r + dr].T
                a = torch.softmax((a * sc).masked_fill(hide, -math.inf), dim=-1)
                o.append(a @ kv[:, Hk * dn + kh * dv:Hk * dn + (kh + 1) * dv])
            out.append(torch.stack(o, dim=1))
            t += nq
        return torch.cat(out)
    lens, train = _prompts(case), kind == "train"
    T = sum(lens)
    z = lambda *n: torch.zeros(n, dtype=torch.float64, device="cuda")  # noqa: E731
    res = {"o": z(T, H, dv), "lse": z(T, H)}
    if train:
        res.update(dq=z(T, H, dn + dr), dk=z(T, Hk, dn), dv=z(T, Hk, dv), dkr=z(T, dr) if dr else None)
    t = 0
    for n in lens:
        w = slice(t, t + n)
        t += n
        hide = torch.ones((n, n), dtype=torch.bool, device="cuda").triu(1) if case["causal"] else None
        for h in range(H):
            kh = h // (H // Hk)
            q, k, v = s["q"][w, h].double(), s["k"][w, kh].double(), s["v"][w, kh].double()
            if dr:
                k = torch.cat([k, s["k_rope"][w].double()], dim=-1)
            a = q @ k.T * sc
            if hide is not None:
                a = a.masked_fill(hide, -math.inf)
            lse = torch.logsumexp(a, dim=-1)
            p = torch.exp(a - lse[:, None])
            o = p @ v
            res["o"][w, h], res["lse"][w, h] = o, lse
            if train:
                do = s["do"][w, h].double()
                ds = p * (do @ v.T - (do * o).sum(-1, keepdim=True)) * sc
                dk = ds.T @ q
                res["dq"][w, h] = ds @ k
                res["dk"][w, kh] += dk[:, :dn]
                res["dv"][w, kh] += p.T @ do
                if dr:
                    res["dkr"][w] += dk[:, dn:]
    return res
