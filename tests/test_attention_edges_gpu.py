"""GPU tests of the attention calls at the edges of what the header admits, against the 64-bit references and bounds
of attn_ref.py."""
import math

import pytest

import attn_ref as R
from conftest import gpu_available
from test_attention_gpu import Paged, _bits, _cum, _freqs, _gen, _ints, _layer, _normal, _split, _within

pytestmark = pytest.mark.gpu

if gpu_available():
    import torch
    import paper_2506_13771_amd as lb
    from test_attention_gpu import DT


# ----------------------------------------------------------------------------
# prefix sums that are none
# ----------------------------------------------------------------------------
def _latent_rows(case, cu, table=None, lens=None, guard=1 << 20, seed=0, f=True):
    """A call with these prefix sums; (out with one row more, P, up, q, freqs).  Bytes behind the workspace that the
    call asks for hold 0x5a before and after."""
    _, news, H, Hk, dn, dv, r, dr, page, act, cd, sc = case
    g = _gen(300 + seed)
    P = Paged(g, case[0], news, r, dr, page, cd)
    paths, up = _layer(g, r, Hk * (dn + dv), sc)
    T = sum(news)
    q = _normal(g, T, H, dn + dr, dtype=act)
    fr = _freqs(dr) if dr and f else None
    n = lb.lb_latent_attention_workspace_bytes(T, len(case[0]), H, r, dr)
    ws = torch.full((n + guard,), 0x5a, dtype=torch.uint8, device="cuda")
    out = torch.full((T, H, dv), 7.0, dtype=DT[act], device="cuda")
    lb.lb_latent_attention(q.cuda(), P.cache, paths, Hk, dv, P.meta[0] if table is None else table.cuda(),
                           P.meta[1] if lens is None else _ints(lens).cuda(), _ints(cu).cuda(),
                           None if fr is None else fr.cuda(), out=out, workspace=ws[:n])
    assert bool((ws[n:] == 0x5a).all())
    return out, P, up, q, fr


CUS = [  # lens, rows of the call, cu: the rows that it gives each sequence
    ([128] * 8, 64, [0, 64] * 4 + [0], [(0, 64)] + [(64, 64)] * 7),
    ([128, 90, 70, 64], 20, [0, 9, 4, 15, 12], [(0, 9), (9, 9), (9, 15), (15, 15)]),
    ([50, 90, 70], 12, [0, -5, 7, 12], [(0, 0), (0, 7), (7, 12)]),
    ([40] * 130, 30, [0, 20] * 64 + [0, 25, 30], [(0, 20)] + [(20, 20)] * 127 + [(20, 25), (25, 30)]),
]


@pytest.mark.parametrize("lens,T,cu,rows", CUS, ids=lambda c: None)
@pytest.mark.parametrize("act", ["f32", "bf16"])
def test_latent_attention_with_sums_that_fall(lens, T, cu, rows, act):
    # a sequence's rows begin where the ones before it end, whatever its prefix sum says
    H, dn, dv, r, dr = 8, 32, 32, 24, 16
    news = [0] * (len(lens) - 1) + [T]
    out, P, up, q, f = _latent_rows((lens, news, H, H, dn, dv, r, dr, 16, act, act, "f16"), cu)
    for b, (lo, hi) in enumerate(rows):
        if hi > lo:
            ref, bound = R.latent_attention(q[lo:hi], [P.rows[b]], up, H, dv, [lens[b]], [hi - lo], f, dr,
                                            (dn + dr) ** -0.5, DT[act])
            _within(out[lo:hi], ref, bound, (b, lo, hi))


# ----------------------------------------------------------------------------
# tokens without a place
# ----------------------------------------------------------------------------
def _free_page_0(P):
    """Page 0 of the pool belongs to no sequence and holds NaN."""
    used = (P.table == 0).nonzero()
    if len(used):
        taken = set(P.table.flatten().tolist())
        other = next(i for i in range(P.data.shape[0]) if i not in taken)
        P.data[other] = P.data[0]
        P.table[tuple(used[0])] = other
    P.data[0] = float("nan")
    P.cache.data.copy_(P.data)


MISSING = [  # lens, H, dn, dv, r, dr, page, act, cache
    ([40, 100, 9], 4, 32, 32, 24, 0, 8, "f32", "f32"),
    ([40, 100, 300], 32, 64, 64, 112, 64, 16, "bf16", "bf16"),
    ([70, 33, 20], 5, 32, 32, 64, 32, 7, "f16", "f16"),
    ([70, 130, 20], 3, 32, 32, 400, 64, 16, "bf16", "bf16"),   # four column waves
    ([70, 130, 20], 2, 32, 32, 700, 32, 16, "f32", "f32"),
]


@pytest.mark.parametrize("case", MISSING, ids=lambda c: f"r{c[4]}-{c[7]}-{c[8]}")
def test_first_pages_that_are_missing(case):
    # sequence 0 has lost its first page and a later one, sequence 1 its first three (a window that has moved on),
    # sequence 2 all of them
    lens, H, dn, dv, r, dr, page, act, cd = case
    g = _gen(r)
    P = Paged(g, lens, [1, 1, 1], r, dr, page, cd)
    _free_page_0(P)
    gone = {0: [0, 2], 1: [0, 1, 2], 2: list(range(P.table.shape[1]))}
    rows = []
    for b, pages in gone.items():
        keep = torch.ones(lens[b], dtype=torch.bool)
        for i in pages:
            P.table[b, i] = (-1, 0x7fffffff, P.data.shape[0], -(2 ** 31))[i % 4]
            keep[i * page:(i + 1) * page] = False
        keep[lens[b] - 1] &= True
        rows.append(P.rows[b][keep])
    paths, up = _layer(g, r, H * (dn + dv))
    q, f = _normal(g, 3, H, dn + dr, dtype=act), _freqs(dr) if dr else None
    out = lb.lb_latent_attention(q.cuda(), P.cache, paths, H, dv, P.table.cuda(), P.meta[1], P.meta[2],
                                 None if f is None else f.cuda())
    assert bool((out[2] == 0).all())
    for b in range(2):
        # (the query turned by its position among all tokens: the reference gets it turned)
        qb = q[b:b + 1].double()
        if dr:
            qb = torch.cat([qb[..., :dn], R.turn(qb[..., dn:], _ints([lens[b] - 1]), f)], -1)
        n = rows[b].shape[0]
        ref, bound = _turned_reference(qb, q[b:b + 1], rows[b], up, H, dv, n, dr, (dn + dr) ** -0.5, DT[cd])
        _within(out[b:b + 1], ref, bound, (b, n))


def _turned_reference(turned, q, rows, up, H, dv, n, dr, scale, cd):
    """attn_ref's reference of one query over n rows, its rotary part given turned (fp64)."""
    class Q:  # a tensor of q's type that reads as the turned values
        dtype, shape = q.dtype, q.shape

        def __getitem__(self, i):
            return turned[i]
    return R.latent_attention(Q(), [rows], up, H, dv, [n], [1], None, dr, scale, cd)


def test_queries_before_the_first_token_stay_0():
    # four new tokens of a sequence of two: the first two queries see nothing, whatever the cache's rows hold
    lens, H, dn, dv, r = [2], 4, 32, 32, 24
    g = _gen(77)
    P = Paged(g, lens, [4], r, 0, 8, "f32")
    P.cache.data[int(P.table[0, 0])] = float("inf")
    paths, _ = _layer(g, r, H * (dn + dv))
    out = lb.lb_latent_attention(_normal(g, 4, H, dn).cuda(), P.cache, paths, H, dv, *P.meta)
    assert bool((out[:2] == 0).all()) and bool(torch.isnan(out[2:]).all())


# ----------------------------------------------------------------------------
# lengths past the page table
# ----------------------------------------------------------------------------
@pytest.mark.parametrize("act,cd", [("f32", "f32"), ("bf16", "bf16")])
def test_append_and_attention_agree_past_the_table(act, cd):
    # sequence 0's length passes its table by 2 (three new tokens, one of which has a place), sequence 1 is full, the
    # third one's prefix sum passes the call's rows by 5
    H, dn, dv, r, dr, page, M = 4, 32, 32, 24, 16, 8, 6
    cap, news, g = M * page, [3, 2, 4], _gen(91)
    lens = [cap + 2, cap, 30]
    T, cu = sum(news), [0, 3, 5, 14]  # nine rows
    data = torch.zeros((3 * M, page, lb.lb_latent_row(r, dr)), dtype=DT[cd])
    table = torch.randperm(3 * M, generator=g).int().view(3, M)
    rows = _normal(g, 3, cap, 2 * r + dr, dtype=cd)
    for b in range(3):
        for t in range(cap):
            data[table[b, t // page], t % page, :2 * r + dr] = rows[b, t]
    f = _freqs(dr)
    w, kr = _normal(g, T, 2, r, dtype=act), _normal(g, T, dr, dtype=act)
    cache = lb.LatentCache(data.cuda(), r, dr)
    meta = (table.cuda(), _ints(lens).cuda(), _ints(cu).cuda())
    lb.lb_latent_append(cache, w.cuda(), kr.cuda(), f.cuda(), *meta)
    got = cache.data.cpu()
    place = []  # (sequence, position) of each row
    for b, (lo, hi) in enumerate(((0, 3), (3, 5), (5, 9))):
        place += [(b, lens[b] - (cu[b + 1] - t)) for t in range(lo, hi)]
    kept = torch.ones(got.shape[:2], dtype=torch.bool)
    for t, (b, pos) in enumerate(place):
        if pos < cap:
            at = (int(table[b, pos // page]), pos % page)
            kept[at] = False
            turned = R.turn(kr[t:t + 1].double(), _ints([pos]), f)
            _within(got[at][2 * r:2 * r + dr][None], turned, R.turn_bound(kr[t:t + 1].double(), DT[cd]) + R.small(DT[cd]), t)
            rows[b, pos] = got[at][:2 * r + dr]
    assert torch.equal(_bits(got[kept]), _bits(data[kept]))
    paths, up = _layer(g, r, H * (dn + dv))
    q = _normal(g, T, H, dn + dr, dtype=act)
    out = lb.lb_latent_attention(q.cuda(), cache, paths, H, dv, *meta, f.cuda())
    for t, (b, pos) in enumerate(place):
        qt = torch.cat([q[t:t + 1, :, :dn].double(), R.turn(q[t:t + 1, :, dn:].double(), _ints([pos]), f)], -1)
        n = min(pos + 1, cap)
        ref, bound = _turned_reference(qt, q[t:t + 1], rows[b, :n].double(), up, H, dv, n, dr, (dn + dr) ** -0.5, DT[cd])
        _within(out[t:t + 1], ref, bound, (t, b, pos))


def test_lengths_below_zero_and_at_the_end_of_32_bits():
    H, dn, dv, r, page = 2, 16, 16, 16, 8
    g = _gen(92)
    P = Paged(g, [20, 20, 20], [2, 2, 2], r, 0, page, "f32")
    P.table[2] = P.table[2, 0]  # every place has a page
    paths, up = _layer(g, r, H * (dn + dv))
    q = _normal(g, 6, H, dn)
    lens = [-(2 ** 31), 20, 2 ** 31 - 1]
    meta = (P.table.cuda(), _ints(lens).cuda(), P.meta[2])
    before = P.cache.data.clone()
    lb.lb_latent_append(P.cache, _normal(g, 6, 2, r).cuda(), None, None, *meta)
    changed = (_bits(P.cache.data) != _bits(before)).any(-1).cpu()
    assert int(changed.sum()) == 2 and all(bool(changed[int(P.table[1, t // page]), t % page]) for t in (18, 19))
    P.rows[1][18:] = torch.stack([P.cache.data[int(P.table[1, t // page]), t % page].cpu()[:2 * r] for t in (18, 19)]).double()
    out = lb.lb_latent_attention(q.cuda(), P.cache, paths, H, dv, *meta)
    assert bool((out[:2] == 0).all())
    ref, bound = R.latent_attention(q[2:4], [P.rows[1]], up, H, dv, [20], [2], None, 0, dn ** -0.5, torch.float32)
    _within(out[2:4], ref, bound, "the sequence between them")
    # all places are seen
    n = P.table.shape[1] * page
    one = P.cache.data[int(P.table[2, 0])].cpu()[:, :2 * r].double().repeat(P.table.shape[1], 1)
    for t in (4, 5):
        ref, bound = R.latent_attention(q[t:t + 1], [one], up, H, dv, [n], [1], None, 0, dn ** -0.5, torch.float32)
        _within(out[t:t + 1], ref, bound, "a length past every table")


# ----------------------------------------------------------------------------
# gradients of f16 heads
# ----------------------------------------------------------------------------
def _f16_gradients(q, k, v, lens_q, lens_k, causal, do, groups=1):
    """dq, dk, dv (fp64) with bounds, of attention without a rotary key.  As attn_ref's, but for dS's smallest step: a
    power of two brings each query's (for dq) and each key's (for dk) largest |dS| to 2^11 or more, so that what lies
    below f16's normal range is off by 2^-25 of 2^-11 of that largest value."""
    H, Hk, d, dv_ = q.shape[1], k.shape[1], q.shape[2], v.shape[2]
    z = lambda *s: torch.zeros(s, dtype=torch.float64)  # noqa: E731
    r = dict(dq=z(*q.shape), dk=z(*k.shape), dv=z(*v.shape))
    r.update({n + "_b": torch.zeros_like(x) for n, x in list(r.items())})
    u, e32, scale, step = R.HALF[torch.float16], R.E32, d ** -0.5, 2.0 ** -36
    a = b = 0
    for n, m in zip(lens_q, lens_k):
        seen = R.seen_mask(n, m, causal)
        for g in range(Hk):
            heads = range(g * H // Hk, (g + 1) * H // Hk)
            parts = []
            for h in heads:
                x = do[a:a + n, h].double()
                hd = R.Head(q[a:a + n, h].double(), k[b:b + m, g].double(), v[b:b + m, g].double(), seen, scale, torch.float16)
                dp = x @ hd.v.T
                dd = (x * hd.o).sum(-1, keepdim=True)
                ds = hd.p * (dp - dd)
                e_dp = (dv_ + 4) * e32 * (x.abs() @ hd.v.abs().T)
                e_d = (x.abs() * (hd.o_bound + dv_ * e32 * hd.o.abs())).sum(-1, keepdim=True)
                e_ds = hd.p * (e_dp + e_d) + ds.abs() * (u + 2 * hd.es[:, None] + 8 * e32)
                top = ds.abs().amax(1, keepdim=True)
                r["dq"][a:a + n, h] = ds @ hd.k * scale
                r["dq_b"][a:a + n, h] = ((e_ds + step * top) @ hd.k.abs() + (m + 4) * e32 * (ds.abs() @ hd.k.abs())) * scale
                r["dv"][b:b + m, g] += hd.p.T @ x
                r["dv_b"][b:b + m, g] += (hd.p * hd.up[:, None] + R.small(torch.float16) * (hd.p > 0)).T @ x.abs() + (
                    n + 4) * e32 * (hd.p.T @ x.abs())
                parts.append((hd.q, ds, e_ds))
            top = torch.stack([p[1].abs().amax(0) for p in parts]).amax(0)
            for qq, ds, e_ds in parts:
                r["dk"][b:b + m, g] += ds.T @ qq * scale
                r["dk_b"][b:b + m, g] += ((e_ds + step * top).T @ qq.abs() + (len(parts) * n + 4) * e32 * (ds.abs().T @ qq.abs())) * scale
        a, b = a + n, b + m
    for n in ("dq", "dk", "dv"):
        r[n + "_b"] += u * r[n].abs() + R.small(torch.float16)
    return r


def _run_f16(q, k, v, lens_q, lens_k, causal, do, pad=0, fill=0.0):
    """lb's gradients, with `pad` rows behind the last sequence that hold `fill`."""
    p = lambda x: torch.cat([x, torch.full((pad,) + x.shape[1:], fill, dtype=x.dtype)]).cuda()  # noqa: E731
    args = [p(x) for x in (q, k, v)] + [None]
    cu = (_cum(lens_q).cuda(), _cum(lens_k).cuda())
    o, lse = lb.lb_attention_forward(*args, *cu, causal=causal)
    o[sum(lens_q):], lse[sum(lens_q):] = fill, fill
    got = lb.lb_attention_backward(*args, o, lse, p(do), *cu, causal=causal)
    return dict(dq=got[0][:q.shape[0]], dk=got[1][:k.shape[0]], dv=got[2][:v.shape[0]])


def _agree(got, ref, what):
    for n in ("dq", "dk", "dv"):
        a, x, b = got[n].cpu().double(), ref[n], ref[n + "_b"]
        # (a value past f16's largest is an infinity of its sign; next to it, either)
        over, near = x.abs() - b >= 65520, x.abs() + b >= 65504
        assert bool((a[over] == x[over].sign() * math.inf).all()), (what, n)
        _within(torch.where(near, torch.zeros_like(a), a), torch.where(near, torch.zeros_like(x), x), b, (what, n))


@pytest.mark.parametrize("fill", [6e4, 100.0, math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("H", [2, 48])
def test_f16_gradients_beside_padding(fill, H):
    # rows behind the last sequence hold anything
    lens, d, g = [130, 470], 64, _gen(4)
    q, k, v = (_normal(g, 600, H, d, dtype="f16") for _ in range(3))
    do = _normal(g, 600, H, d, dtype="f16", std=1e-3)
    ref = _f16_gradients(q, k, v, lens, lens, False, do)
    _agree(_run_f16(q, k, v, lens, lens, False, do, 5, fill), ref, fill)


@pytest.mark.parametrize("d,dv", [(64, 128), (128, 64), (192, 128)])
@pytest.mark.parametrize("size,do_size", [(130.0, 1.0), (128.0, 1e-4), (60000.0, 4.0)])
@pytest.mark.parametrize("H", [1, 200])
def test_f16_gradients_of_large_values(d, dv, size, do_size, H):
    # equal scores of two keys with opposite values aligned with dO: dS reaches half of |dO| |V| dv
    n = 130 if H > 1 else 2
    g = _gen(5)
    q, k = _normal(g, n, H, d, dtype="f16", std=1e-3), _normal(g, 2, H, d, dtype="f16", std=1e-3)
    v = (torch.ones(2, H, dv) * torch.tensor([1.0, -1.0]).view(2, 1, 1) * size).half()
    do = torch.full((n, H, dv), do_size).half()
    ref = _f16_gradients(q, k, v, [n], [2], False, do)
    _agree(_run_f16(q, k, v, [n], [2], False, do), ref, (d, dv, size))


@pytest.mark.parametrize("H,Hk", [(2, 2), (4, 1), (64, 64)])
@pytest.mark.parametrize("causal", [True, False])
def test_f16_gradients_beside_one_large_one(H, Hk, causal):
    # one token's gradient 10^7 times the others': theirs keep their digits
    lens, d, g = [300, 200], 64, _gen(6)
    q, k, v = _normal(g, 500, H, d, dtype="f16"), _normal(g, 500, Hk, d, dtype="f16"), _normal(g, 500, Hk, d, dtype="f16")
    do = _normal(g, 500, H, d, dtype="f16", std=1e-3)
    do[7] *= 1e7
    assert bool(torch.isfinite(do).all())
    ref = _f16_gradients(q, k, v, lens, lens, causal, do)
    _agree(_run_f16(q, k, v, lens, lens, causal, do), ref, (H, Hk, causal))


# ----------------------------------------------------------------------------
# small probabilities in f16
# ----------------------------------------------------------------------------
@pytest.mark.parametrize("H", [2, 130])
@pytest.mark.parametrize("grad", [1.0, 1000.0])
def test_f16_values_gradient_of_little_seen_keys(H, grad):
    # keys that every query gives 2^-12 to 2^-27 of its weight; their dV comes from such probabilities alone
    n, m, d, dv, g = 600, 128, 8, 64, _gen(9)
    k = torch.zeros(m, H, d, dtype=torch.float16)
    k[1:, :, 0] = -torch.linspace(12.0, 27.0, m - 1)[:, None].half()
    q = torch.zeros(n, H, d, dtype=torch.float16)
    q[..., 0] = math.log(2.0)
    v = _normal(g, m, H, dv, dtype="f16")
    do = _normal(g, n, H, dv, dtype="f16", std=grad)
    args = [t.cuda() for t in (q, k, v)] + [None]
    o, lse = lb.lb_attention_forward(*args, causal=False, scale=1.0)
    got = lb.lb_attention_backward(*args, o, lse, do.cuda(), causal=False, scale=1.0)[2]
    for h in (0, H - 1):
        hd = R.Head(q[:, h].double(), k[:, h].double(), v[:, h].double(), R.seen_mask(n, m, False), 1.0, torch.float16)
        ref = hd.p.T @ do[:, h].double()
        # as attn_ref's bound, with f16's smallest step 2^-14 of what it is there
        bound = (hd.p * hd.up[:, None] + 2.0 ** -14 * R.small(torch.float16)).T @ do[:, h].double().abs() + (
            n + 4) * R.E32 * (hd.p.T @ do[:, h].double().abs()) + R.HALF[torch.float16] * ref.abs() + R.small(torch.float16)
        _within(got[:, h], ref, bound, (H, h))


# ----------------------------------------------------------------------------
# an f16 cache: parts of a query that differ much in size
# ----------------------------------------------------------------------------
@pytest.mark.parametrize("act", ["f32", "f16"])
@pytest.mark.parametrize("large", ["latents", "rotary"])
def test_f16_cache_keeps_the_smaller_part_of_a_query(act, large):
    # |h q| of thousands beside a rotary part near 1 (or the reverse), while the cache holds the smaller part's
    # counterparts some thousand times larger: both parts decide the scores
    n, H, dn, dv, r, dr, page, g = 200, 3, 128, 32, 64, 64, 16, _gen(61)
    w = _normal(g, n, 2 * r + dr)
    up_w, up_q = (2.0 ** -11, 2.0 ** 13) if large == "latents" else (16.0, 2.0 ** -5)
    w[:, :2 * r] *= up_w
    w[:, 2 * r:] *= 4.0 if large == "latents" else 2.0 ** -9
    w = w.half()
    q = _normal(g, 1, H, dn + dr)
    q[..., :dn] *= up_q
    q[..., dn:] *= 1.0 if large == "latents" else 2.0 ** 11
    q = q.to(DT[act])
    paths, up = _layer(g, r, H * (dn + dv))
    data = torch.zeros(-(-n // page), page, lb.lb_latent_row(r, dr), dtype=torch.float16)
    data.view(-1, data.shape[-1])[:n, :2 * r + dr] = w
    f, scale = _freqs(dr), (dn + dr) ** -0.5
    out = lb.lb_latent_attention(q.cuda(), lb.LatentCache(data.cuda(), r, dr), paths, H, dv,
                                 torch.arange(data.shape[0], dtype=torch.int32).view(1, -1).cuda(), _ints([n]).cuda(),
                                 _ints([0, 1]).cuda(), f.cuda())
    rows = w.double()
    ref, bound = R.latent_attention(q, [rows], up, H, dv, [n], [1], f, dr, scale, torch.float32)
    # attn_ref's bound with q' as fp32 holds it, and for the two f16 terms 2^-22 of every element (all are above 2^-17
    # of the row's bound but for those near 0: 2^-25 2^-13 of it), for a probability 2^-22, or 2^-11 (f16 activations)
    for h in range(H):
        uk, v = up[:, h * dn:(h + 1) * dn], rows[:, :2 * r] @ up[:, H * dn + h * dv:H * dn + (h + 1) * dv]
        x = q[0, h].double()
        qa = torch.cat([uk @ x[:dn], R.turn(x[None, dn:], _ints([n - 1]), f)[0]])
        top = max(dn * float((up.abs().amax() * x[:dn].abs()).max()), 1.5 * float(x[dn:].abs().max()))
        e = scale * float((rows.abs() @ (2.0 ** -22 * qa.abs() + 2.0 ** -38 * top)).max())
        p = torch.softmax(rows @ qa * scale, 0)
        bound[0, h] += (2 * e + (2.0 ** -22 if act == "f32" else 2.0 ** -11)) * (p @ v.abs()) + 2.0 ** -25 * v.abs().sum(0)
        assert 0.1 < float((rows[:, :2 * r] @ qa[:2 * r]).std() * scale) < 30 and 0.1 < float((rows[:, 2 * r:] @ qa[2 * r:]).std() * scale) < 30
    _within(out, ref, bound, (act, large))


# ----------------------------------------------------------------------------
# NaN
# ----------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("H", [2, 300])
def test_a_nan_query_is_not_taken_for_one_that_sees_nothing(dtype, H):
    # o, lse and the gradients of a NaN query are NaN; a query without keys has lse -infinity, o and dq 0
    lens_q, lens_k, d = [40, 30], [40, 28], 32
    g = _gen(71)
    q, k, v = _normal(g, 70, H, d, dtype=dtype), _normal(g, 68, H, d, dtype=dtype), _normal(g, 68, H, d, dtype=dtype)
    q[5, 0] = math.nan
    do = _normal(g, 70, H, d, dtype=dtype)
    args, cu = [t.cuda() for t in (q, k, v)] + [None], (_cum(lens_q).cuda(), _cum(lens_k).cuda())
    o, lse = lb.lb_attention_forward(*args, *cu)
    assert bool(torch.isnan(o[5, 0]).all()) and bool(torch.isnan(lse[5, 0]))
    assert bool((lse[40:42] == -math.inf).all()) and bool((o[40:42] == 0).all())
    dq, dk, _, _ = lb.lb_attention_backward(*args, o, lse, do.cuda(), *cu)
    assert bool(torch.isnan(dq[5, 0]).all()) and bool(torch.isnan(dk[:6, 0]).all()) and bool((dq[40:42] == 0).all())
    fine = torch.ones(70, H, dtype=torch.bool)
    fine[5, 0] = False
    assert bool(torch.isfinite(o.cpu()[fine]).all()) and bool(torch.isfinite(dq.cpu()[fine]).all())


# ----------------------------------------------------------------------------
# heads without a width
# ----------------------------------------------------------------------------
@pytest.mark.parametrize("act", ["f32", "bf16", "f16"])
def test_queries_of_width_0_average_the_values(act):
    # no columns to score with: every cached token counts alike (scale left out)
    lens, H, dv, r = [1, 50, 300], 3, 16, 20
    g = _gen(81)
    P = Paged(g, lens, [1, 1, 1], r, 0, 16, act)
    paths, up = _layer(g, r, H * dv)
    q = torch.zeros(3, H, 0, dtype=DT[act])
    out = lb.lb_latent_attention(q.cuda(), P.cache, paths, H, dv, *P.meta)
    ref, bound = R.latent_attention(q, P.rows, up, H, dv, lens, [1, 1, 1], None, 0, 1.0, DT[act])
    _within(out, ref, bound, act)


def test_expanded_queries_of_width_0_are_refused_by_the_library():
    q, k, v = (torch.zeros(4, 2, d, device="cuda") for d in (0, 0, 8))
    with pytest.raises(RuntimeError, match="lb_attention_forward"):
        lb.lb_attention_forward(q, k, v)
