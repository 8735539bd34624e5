"""GPU tests of the position rotation, the paged latent cache and the attention calls against 64-bit references, with
the element-wise bounds that attn_ref.py derives."""
import math

import numpy as np
import pytest

import attn_ref as R
from conftest import gpu_available

pytestmark = pytest.mark.gpu

if gpu_available():
    import torch
    import paper_2506_13771_amd as lb

    DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _normal(g, *shape, dtype="f32", std=1.0):
    return (torch.randn(shape, generator=g) * std).to(DT[dtype])


def _freqs(d, base=10000.0):
    return torch.tensor([base ** (-2.0 * i / d) for i in range(d // 2)], dtype=torch.float64).float()


def _ints(v):
    return torch.tensor(list(v), dtype=torch.int32)


def _cum(lens):
    return _ints(np.concatenate([[0], np.cumsum(lens)]))


def _within(got, ref, bound, what):
    got = got.detach().cpu().double()
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    assert torch.isfinite(got).all(), what
    bad = (got - ref).abs() > bound
    if bad.any():
        i = tuple(int(x) for x in bad.nonzero()[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} beyond the bound, first at {i}: "
                             f"{float(got[i])} against {float(ref[i])}, bound {float(bound[i])}; "
                             f"largest ratio {float(((got - ref).abs() / bound).max())}")


def _bits(t):
    return t.contiguous().view(torch.int16 if t.element_size() == 2 else torch.int32)


# ----------------------------------------------------------------------------
# rotation
# ----------------------------------------------------------------------------
@pytest.mark.parametrize("T,H,d,pos,dtype", [
    (1, 1, 2, 10, "f32"), (5, 1, 64, 4096, "f32"), (33, 7, 64, 2 ** 31 - 1, "bf16"), (300, 9, 128, 100000, "f16"),
    (17, 4, 6, 1000, "bf16"), (2, 40, 256, 500, "f32"), (65, 3, 32, 12345, "f16")])
@pytest.mark.parametrize("inverse", [False, True])
def test_rotate(T, H, d, pos, dtype, inverse):
    g = _gen(T * 31 + d)
    x = _normal(g, T, H, d, dtype=dtype)
    p = torch.randint(0, pos, (T,), generator=g, dtype=torch.int32)
    p[0] = pos - 1 if pos < 2 ** 31 - 1 else 2 ** 31 - 1
    f = _freqs(d)
    y = lb.lb_rotate(x.cuda(), p.cuda(), f.cuda(), inverse=inverse)
    _within(y, R.turn(x.double(), p, f, inverse), R.turn_bound(x.double(), DT[dtype]), (T, H, d, dtype))


@pytest.mark.parametrize("layout", ["tail", "odd_tail", "heads_first", "in_place", "in_place_tail", "shared_row"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rotate_layouts(layout, dtype):
    T, H, d = 37, 5, 32
    g = _gen(3)
    p, f = torch.randint(0, 9999, (T,), generator=g, dtype=torch.int32), _freqs(d)
    wide = _normal(g, T, H, 3 * d + 1, dtype=dtype).cuda()
    x = {"tail": wide[..., d:2 * d], "odd_tail": wide[..., d + 1:2 * d + 1], "in_place_tail": wide[..., 2 * d:3 * d],
         "heads_first": _normal(g, H, T, d, dtype=dtype).cuda().transpose(0, 1),
         "in_place": _normal(g, T, H, d, dtype=dtype).cuda(),
         "shared_row": _normal(g, T, 1, d, dtype=dtype).cuda().expand(T, H, d)}[layout]
    before, ref_x = wide.clone(), x.cpu().double()
    out = None
    if layout.startswith("in_place"):
        out = x
    elif layout == "heads_first":
        out = torch.empty(H, T, d, dtype=DT[dtype], device="cuda").transpose(0, 1)
    y = lb.lb_rotate(x, p.cuda(), f.cuda(), out=out)
    _within(y, R.turn(ref_x, p, f), R.turn_bound(ref_x, DT[dtype]), layout)
    keep = torch.ones_like(wide, dtype=torch.bool)
    if layout == "in_place_tail":
        keep[..., 2 * d:3 * d] = False
    assert torch.equal(_bits(wide[keep]), _bits(before[keep]))  # the other columns as they were


# ----------------------------------------------------------------------------
# the paged cache
# ----------------------------------------------------------------------------
class Paged:
    """A cache with shuffled pages for given lengths; everything that belongs to no token holds NaN."""

    def __init__(self, g, lens, news, r, dr, page, dtype, spare=2):
        need = [-(-n // page) for n in lens]
        self.lens, self.news, self.r, self.dr, self.page = lens, news, r, dr, page
        n_pages, most = sum(need) + spare, max(max(need), 1) + 1
        order = torch.randperm(n_pages, generator=g)
        self.table = torch.full((len(lens), most), -1, dtype=torch.int32)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[at:at + n].int()
            at += n
        row = lb.lb_latent_row(r, dr)
        self.data = torch.full((n_pages, page, row), float("nan"), dtype=DT[dtype])
        self.rows = []
        for b, n in enumerate(lens):
            w = _normal(g, n, 2 * r + dr, dtype=dtype)
            self.rows.append(w.double())
            for t in range(n):
                cell = self.data[self.table[b, t // page], t % page]
                cell[:2 * r + dr] = w[t]
                cell[2 * r + dr:] = 0
        self.cache = lb.LatentCache(self.data.cuda(), r, dr)
        self.meta = (self.table.cuda(), _ints(lens).cuda(), _cum(news).cuda())


APPENDS = [  # lens, news, r, dr, page, dtype, cache dtype
    ([1], [1], 1, 0, 1, "f32", "f32"),
    ([5, 40, 3], [5, 1, 0], 33, 6, 7, "f32", "bf16"),
    ([300, 64, 65, 1], [300, 1, 65, 1], 112, 64, 64, "bf16", "bf16"),
    ([17, 100], [4, 100], 17, 64, 16, "f16", "f16"),
    ([9] * 70, [1] * 70, 40, 32, 5, "bf16", "f32"),  # more sequences than lanes
    ([50, 1500], [50, 1200], 72, 16, 100, "f32", "f16"),
]


@pytest.mark.parametrize("case", APPENDS, ids=lambda c: f"B{len(c[0])}-r{c[2]}-d{c[3]}-p{c[4]}-{c[5]}-{c[6]}")
@pytest.mark.parametrize("turned", [True, False])
def test_append(case, turned):
    lens, news, r, dr, page, dtype, cd = case
    g = _gen(r)
    P = Paged(g, lens, news, r, dr, page, cd)
    T = sum(news)
    w, kr = _normal(g, T + 2, 2, r, dtype=dtype), _normal(g, T + 2, dr + 3, dtype=dtype)
    f = _freqs(dr) if dr and turned else None
    ref, bound = P.data.double(), torch.zeros(P.data.shape, dtype=torch.float64)
    t, touched = 0, torch.zeros(P.data.shape[:2], dtype=torch.bool)
    for b, (n, m) in enumerate(zip(news, lens)):
        for j in range(n):
            p = m - n + j
            pg, off = int(P.table[b, p // page]), p % page
            touched[pg, off] = True
            x = w[t].double().reshape(-1)
            k = kr[t:t + 1, 3:].double()
            kt = R.turn(k, _ints([p]), f) if f is not None else k
            kb = R.turn_bound(k, DT[cd]) if f is not None else R.HALF[DT[cd]] * k.abs()
            ref[pg, off] = torch.cat([x, kt[0], torch.zeros(P.data.shape[2] - 2 * r - dr, dtype=torch.float64)])
            bound[pg, off] = 0.0
            bound[pg, off, :2 * r] = R.HALF[DT[cd]] * x.abs() + R.small(DT[cd])
            bound[pg, off, 2 * r:2 * r + dr] = kb[0] + R.small(DT[cd])
            t += 1
    # two rows behind the last sequence are given and not written
    lb.lb_latent_append(P.cache, w.cuda(), kr.cuda()[:, 3:] if dr else None, None if f is None else f.cuda(), *P.meta)
    got = P.cache.data.cpu()
    assert torch.equal(_bits(got[~touched]), _bits(P.data[~touched]))  # every other row as it was
    _within(got[touched], ref[touched], bound[touched], case)


def test_append_skips_tokens_without_a_place():
    g = _gen(5)
    P = Paged(g, [20, 20, 20, 20], [3, 3, 3, 3], 16, 0, 8, "f32")
    P.table[0, 2] = -1                          # page missing
    P.table[1, 2] = P.data.shape[0]             # page past the cache
    lens = [20, 20, 2, 8 * P.table.shape[1] + 2]  # sequence 2: its first token before position 0; 3: two past the table
    w = _normal(g, 12, 2, 16)
    lb.lb_latent_append(P.cache, w.cuda(), None, None, P.table.cuda(), _ints(lens).cuda(), P.meta[2])
    want = P.data.clone()
    page = int(P.table[2, 0])
    want[page, 0, :32] = w[7].reshape(-1)
    want[page, 1, :32] = w[8].reshape(-1)
    # sequence 3's first token is the table's last place: its page there is -1, so none of the three is written
    assert torch.equal(_bits(P.cache.data.cpu()), _bits(want))


# ----------------------------------------------------------------------------
# attention from the latent cache
# ----------------------------------------------------------------------------
def _layer(g, r, n_out, scale_dtype="f16"):
    """(paths, up [2 r, n_out] fp64) of a fused layer with random signs."""
    paths, up = [], []
    for _ in range(2):
        u = torch.randn((n_out, r), generator=g)
        h = ((torch.randn(n_out, generator=g).abs() * 0.8 + 0.1) / math.sqrt(2 * r)).to(DT[scale_dtype])
        U = lb.lb_pack_signs(u.cuda(), lb.LB_ROLE_U)
        paths.append(lb.LittleBitPath(U=U, V=None, h=h.cuda(), g=None, l=None))
        s = R.unpack(U.cpu(), n_out, r)
        assert torch.equal(s, torch.where(u < 0, -1.0, 1.0).double())
        up.append((s * h.double()[:, None]).T)
    return paths, torch.cat(up)


LATENT = [  # lens, news, H, Hk, dn, dv, r, dr, page, act, cache, scales
    ([1], [1], 1, 1, 8, 8, 1, 0, 1, "f32", "f32", "f32"),
    ([37], [1], 5, 5, 40, 56, 33, 16, 7, "f32", "f32", "f16"),
    ([1, 300, 33, 32, 31], [1, 1, 1, 1, 1], 32, 32, 64, 64, 112, 64, 64, "bf16", "bf16", "f16"),
    ([200, 5, 129], [3, 5, 0], 12, 4, 96, 64, 64, 32, 16, "f16", "f16", "bf16"),
    ([90, 700], [1, 2], 8, 8, 128, 128, 80, 64, 100, "bf16", "bf16", "f16"),
    ([60, 257], [2, 1], 6, 2, 40, 56, 150, 64, 48, "bf16", "f32", "f32"),
    ([64, 100], [1, 4], 4, 2, 33, 17, 51, 10, 3, "f32", "bf16", "f16"),
    ([70, 40], [1, 1], 7, 7, 64, 32, 100, 64, 16, "f32", "f16", "f16"),
    ([300, 20], [1, 2], 4, 4, 64, 64, 400, 64, 64, "bf16", "bf16", "f16"),   # a row of four column waves
    ([130], [1], 3, 3, 32, 32, 768, 0, 16, "f16", "f16", "f16"),             # the widest row
    ([150, 33], [1, 1], 2, 1, 64, 64, 300, 32, 16, "f32", "f32", "f16"),
    ([100, 60], [1, 1], 4, 4, 64, 64, 176, 32, 64, "bf16", "bf16", "f16"),   # 12 units
    ([40] * 70, [1] * 70, 2, 2, 16, 16, 24, 0, 16, "bf16", "bf16", "f16"),   # more sequences than lanes
    ([65], [65], 8, 8, 64, 64, 48, 32, 16, "f16", "f16", "f16"),             # a prompt
    ([90], [1], 4, 4, 0, 32, 20, 64, 32, "bf16", "bf16", "f16"),             # scores from the rotary key alone
]


def _latent_id(c):
    return f"B{len(c[0])}L{max(c[0])}-H{c[2]}.{c[3]}-{c[4]}.{c[5]}-r{c[6]}.{c[7]}-p{c[8]}-{c[9]}-{c[10]}"


def _latent_call(case, seed=0, std=1.0, qlay="plain"):
    lens, news, H, Hk, dn, dv, r, dr, page, act, cd, sc = case
    g = _gen(100 + seed)
    P = Paged(g, lens, news, r, dr, page, cd)
    paths, up = _layer(g, r, Hk * (dn + dv), sc)
    T = sum(news)
    q = _normal(g, T + 1, H, dn + dr, dtype=act, std=std)
    f = _freqs(dr) if dr else None
    qd = q.cuda()
    if qlay == "heads_first":
        qd = qd.transpose(0, 1).contiguous().transpose(0, 1)
    elif qlay == "wide":
        qd = torch.cat([qd, qd, qd[..., :1]], dim=-1)[..., :dn + dr]
    return P, paths, up, q, qd, f


@pytest.mark.parametrize("case", LATENT, ids=_latent_id)
@pytest.mark.parametrize("std", [1.0, 6.0])
def test_latent_attention(case, std):
    lens, news, H, Hk, dn, dv, r, dr, page, act, cd, sc = case
    P, paths, up, q, qd, f = _latent_call(case, std=std)
    T, scale = sum(news), (dn + dr) ** -0.5
    out = torch.full((T + 1, H, dv), 7.0, dtype=DT[act], device="cuda")
    lb.lb_latent_attention(qd, P.cache, paths, Hk, dv, *P.meta, None if f is None else f.cuda(), out=out)
    ref, bound = R.latent_attention(q[:T], P.rows, up, Hk, dv, lens, news, f, dr, scale, DT[cd])
    assert bool((out[T] == 7.0).all())  # the row behind the last sequence
    _within(out[:T], ref, bound, case)
    again = torch.empty_like(out)
    ws = torch.full((lb.lb_latent_attention_workspace_bytes(T + 1, len(lens), H, r, dr),), 255, dtype=torch.uint8,
                    device="cuda")
    lb.lb_latent_attention(qd, P.cache, paths, Hk, dv, *P.meta, None if f is None else f.cuda(), out=again, workspace=ws)
    assert torch.equal(_bits(again[:T]), _bits(out[:T]))  # whatever the workspace held


@pytest.mark.parametrize("qlay", ["heads_first", "wide"])
def test_latent_attention_query_layouts(qlay):
    case = LATENT[3]
    P, paths, _, q, qd, f = _latent_call(case, qlay=qlay)
    a = lb.lb_latent_attention(qd, P.cache, paths, case[3], case[5], *P.meta, f.cuda())
    b = lb.lb_latent_attention(q.cuda(), P.cache, paths, case[3], case[5], *P.meta, f.cuda())
    T = sum(case[1])
    assert torch.equal(_bits(a[:T]), _bits(b[:T]))


def test_latent_attention_without_turning():
    case = ([50, 9], [2, 1], 4, 2, 32, 32, 20, 16, 16, "f32", "f32", "f16")
    P, paths, up, q, qd, _ = _latent_call(case)
    out = lb.lb_latent_attention(qd, P.cache, paths, 2, 32, *P.meta, None, scale=0.3)
    ref, bound = R.latent_attention(q[:3], P.rows, up, 2, 32, case[0], case[1], None, 16, 0.3, torch.float32)
    _within(out[:3], ref, bound, "no freqs")


def test_latent_attention_rows_that_see_nothing():
    # an empty sequence, a sequence shorter than its new tokens, and missing pages
    case = ([0, 2, 40, 40], [1, 4, 1, 1], 4, 4, 32, 32, 24, 0, 8, "f32", "f32", "f16")
    P, paths, up, q, qd, _ = _latent_call(case)
    P.table[3, :] = P.data.shape[0] + 5  # sequence 3: no page exists
    kept = P.table[2].clone()
    P.table[2, 1] = -7                   # sequence 2: tokens 8 .. 15 have no page
    out = lb.lb_latent_attention(qd, P.cache, paths, 4, 32, P.table.cuda(), P.meta[1], P.meta[2])
    got = out.cpu()
    assert bool((got[0] == 0).all()) and bool((got[1:3] == 0).all()) and bool((got[6] == 0).all())
    ref, bound = R.latent_attention(q[3:5], [P.rows[1]], up, 4, 32, [2], [2], None, 0, 32 ** -0.5, torch.float32)
    _within(got[3:5], ref, bound, "the tokens that have a position")
    rows = torch.cat([P.rows[2][:8], P.rows[2][16:]])
    ref, bound = R.latent_attention(q[5:6], [rows], up, 4, 32, [32], [1], None, 0, 32 ** -0.5, torch.float32)
    _within(got[5:6], ref, bound, "a missing page is not seen")
    assert kept.numel()


def test_latent_attention_scores_at_the_edges():
    # equal scores over a long axis, one score far above the rest, scores near fp32's and fp16's ends
    for act, cd in (("f32", "f32"), ("bf16", "bf16"), ("f16", "f16")):
        case = ([3000], [1], 2, 2, 32, 32, 16, 0, 64, act, cd, "f32")
        for std in (0.0, 200.0):
            P, paths, up, q, qd, _ = _latent_call(case, std=std)
            out = lb.lb_latent_attention(qd, P.cache, paths, 2, 32, *P.meta)
            ref, bound = R.latent_attention(q[:1], P.rows, up, 2, 32, [3000], [1], None, 0, 32 ** -0.5, DT[cd])
            _within(out[:1], ref, bound, (act, std))


def test_latent_attention_cache_beyond_32_bits():
    # rows past 2^31 elements and 2^32 bytes of the cache
    r, dr, page = 112, 64, 64
    row = lb.lb_latent_row(r, dr)
    n_pages = (1 << 32) // (page * row) + 40
    data = torch.zeros((n_pages, page, row), dtype=torch.bfloat16, device="cuda")
    g = _gen(11)
    table = _ints([n_pages - 1, 3, n_pages - 17]).view(1, 3)
    rows = _normal(g, 3 * page, 2 * r + dr, dtype="bf16")
    w, kr = rows[:, :2 * r].reshape(-1, 2, r).contiguous(), rows[:, 2 * r:].contiguous()
    cache = lb.LatentCache(data, r, dr)
    lens, f = [3 * page], _freqs(dr)
    lb.lb_latent_append(cache, w.cuda(), kr.cuda(), None, table.cuda(), _ints(lens).cuda(), _cum(lens).cuda())
    assert torch.equal(data[n_pages - 17, 5, :2 * r + dr].cpu(), rows[2 * page + 5])
    paths, up = _layer(g, r, 4 * 64)
    q = _normal(g, 1, 4, 32 + dr, dtype="bf16")
    out = lb.lb_latent_attention(q.cuda(), cache, paths, 4, 32, table.cuda(), _ints(lens).cuda(), _ints([0, 1]).cuda(),
                                 f.cuda())
    ref, bound = R.latent_attention(q, [rows.double()], up, 4, 32, lens, [1], f, dr, (32 + dr) ** -0.5, torch.bfloat16)
    _within(out, ref, bound, "long cache")


# ----------------------------------------------------------------------------
# attention over expanded keys and values
# ----------------------------------------------------------------------------
EXPANDED = [  # lens_q, lens_k, H, Hk, dn, dr, dv, causal, dtype
    ([1], [1], 1, 1, 8, 0, 8, True, "f32"),
    ([130], [130], 2, 2, 64, 0, 64, True, "f32"),
    ([130], [130], 2, 2, 128, 64, 128, True, "bf16"),
    ([1, 64, 65, 0, 200], [1, 64, 65, 3, 200], 4, 2, 128, 64, 128, True, "bf16"),
    ([33, 129, 7], [33, 129, 7], 6, 3, 40, 16, 56, False, "f16"),
    ([10, 3, 70], [4, 50, 300], 4, 4, 64, 32, 64, True, "f16"),     # queries before the first key; a longer past
    ([20, 5], [0, 260], 2, 1, 96, 0, 96, False, "bf16"),           # a sequence without keys
    ([77, 100], [150, 100], 3, 3, 33, 7, 17, True, "f32"),         # sizes that fit no vector
    ([50, 40], [50, 60], 2, 2, 21, 0, 128, True, "bf16"),
    ([300], [257], 2, 2, 0, 64, 128, False, "f32"),                # the rotary key alone
    ([128, 256], [128, 256], 8, 1, 64, 64, 128, True, "f16"),      # one key head
    ([60, 9], [60, 300], 2, 2, 128, 64, 128, True, "f32"),         # the widest fp32 heads
    # enough heads for workgroups of 128 rows
    ([200, 230], [200, 230], 64, 64, 64, 0, 64, True, "bf16"),
    ([150, 1, 170], [200, 5, 170], 64, 64, 128, 64, 128, True, "bf16"),
    ([260, 0, 33], [240, 9, 33], 64, 64, 64, 32, 128, True, "f16"),
    ([129, 100], [129, 100], 192, 192, 33, 7, 56, False, "f32"),
    ([290], [290], 128, 64, 96, 16, 40, True, "f16"),
    ([140, 140], [150, 140], 144, 144, 128, 0, 128, True, "f32"),
    ([130, 64], [130, 64], 208, 208, 120, 64, 128, False, "f32"),
]


def _expanded_id(c):
    return f"q{sum(c[0])}k{sum(c[1])}-H{c[2]}.{c[3]}-{c[4]}.{c[5]}.{c[6]}-{'c' if c[7] else 'f'}-{c[8]}"


def _expanded_inputs(case, seed=0, std=1.0, pad=2):
    lens_q, lens_k, H, Hk, dn, dr, dv, _, dtype = case
    g = _gen(200 + seed)
    Tq, Tk = sum(lens_q) + pad, sum(lens_k) + pad
    q = _normal(g, Tq, H, dn + dr, dtype=dtype, std=std)
    y = _normal(g, Tk, Hk * (dn + dv), dtype=dtype)
    kr = _normal(g, Tk, dr, dtype=dtype) if dr else None
    do = _normal(g, Tq, H, dv, dtype=dtype)
    return q, y, kr, do


def _split(y, Hk, dn, dv):
    T = y.shape[0]
    return y[:, :Hk * dn].view(T, Hk, dn), y[:, Hk * dn:].view(T, Hk, dv)


@pytest.mark.parametrize("case", EXPANDED, ids=_expanded_id)
@pytest.mark.parametrize("std", [1.0, 4.0])
def test_expanded_attention(case, std):
    lens_q, lens_k, H, Hk, dn, dr, dv, causal, dtype = case
    q, y, kr, do = _expanded_inputs(case, std=std)
    Tq, Tk, scale = sum(lens_q), sum(lens_k), (dn + dr) ** -0.5
    for t in (q, do):
        t[Tq:] = float("nan")
    y[Tk:] = float("nan")
    k, v = _split(y, Hk, dn, dv)
    ref = R.attention(q[:Tq], k[:Tk], v[:Tk], None if kr is None else kr[:Tk], lens_q, lens_k, causal, scale, do[:Tq])
    cu = (_cum(lens_q).cuda(), _cum(lens_k).cuda())
    qd, yd, krd, dod = q.cuda(), y.cuda(), None if kr is None else kr.cuda(), do.cuda()
    kd, vd = _split(yd, Hk, dn, dv)
    o = torch.full(do.shape, 3.0, dtype=DT[dtype], device="cuda")
    lse = torch.full(do.shape[:2], 3.0, device="cuda")
    lb.lb_attention_forward(qd, kd, vd, krd, *cu, causal=causal, o=o, lse=lse)
    assert bool((o[Tq:] == 3).all()) and bool((lse[Tq:] == 3).all())
    _within(o[:Tq], ref["o"], ref["o_b"], (case, "o"))
    none = ref["lse"] == -math.inf
    got = lse[:Tq].cpu().double()
    assert torch.equal(got == -math.inf, none)
    _within(got[~none], ref["lse"][~none], ref["lse_b"][~none], (case, "lse"))
    # gradients, into the two parts of one buffer
    dy = torch.full(y.shape, 5.0, dtype=DT[dtype], device="cuda")
    dk, dvv = _split(dy, Hk, dn, dv)
    dq = torch.full(q.shape, 5.0, dtype=DT[dtype], device="cuda")
    dkr = torch.full((y.shape[0], dr), 5.0, dtype=DT[dtype], device="cuda") if dr else None
    lb.lb_attention_backward(qd, kd, vd, krd, o, lse, dod, *cu, causal=causal, dq=dq, dk=dk, dv=dvv, dk_rope=dkr)
    assert bool((dy[Tk:] == 5).all()) and bool((dq[Tq:] == 5).all())
    _within(dq[:Tq], ref["dq"], ref["dq_b"], (case, "dq"))
    _within(dk[:Tk], ref["dk"], ref["dk_b"], (case, "dk"))
    _within(dvv[:Tk], ref["dv"], ref["dv_b"], (case, "dv"))
    if dr:
        assert bool((dkr[Tk:] == 5).all())
        _within(dkr[:Tk], ref["dkr"], ref["dkr_b"], (case, "dkr"))
    # the same bits again
    again = lb.lb_attention_backward(qd, kd, vd, krd, o, lse, dod, *cu, causal=causal)
    for a, b, n in zip(again, (dq, dk, dvv, dkr), (Tq, Tk, Tk, Tk)):
        if a is not None:
            assert torch.equal(_bits(a[:n]), _bits(b[:n]))


@pytest.mark.parametrize("layout", ["heads_first", "odd_offset", "one_sequence", "shared_kv"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_expanded_attention_layouts(layout, dtype):
    T, H, Hk, dn, dr, dv = 150, 4, 2, 32, 16, 48
    g = _gen(8)
    q, k, v = (_normal(g, T, h, d, dtype=dtype) for h, d in ((H, dn + dr), (Hk, dn), (Hk, dv)))
    kr, do = _normal(g, T, dr, dtype=dtype), _normal(g, T, H, dv, dtype=dtype)
    if layout == "shared_kv":
        k, v = k[:, :1].expand(T, Hk, dn), v[:, :1].expand(T, Hk, dv)
    ref = R.attention(q, k, v, kr, [T], [T], True, (dn + dr) ** -0.5, do)

    def put(x):
        if layout == "heads_first" and x.dim() == 3:
            return x.cuda().transpose(0, 1).contiguous().transpose(0, 1)
        if layout == "odd_offset":
            wide = torch.cat([x[..., :1], x, x[..., :2]], dim=-1).cuda()
            return wide[..., 1:-2]
        if layout == "shared_kv" and x.dim() == 3 and x.stride(1) == 0:
            return x[:, :1].contiguous().cuda().expand(x.shape)
        return x.cuda()

    args = [put(x) for x in (q, k, v, kr)]
    cu = () if layout == "one_sequence" else (_ints([0, T]).cuda(), _ints([0, T]).cuda())
    o, lse = lb.lb_attention_forward(*args, *cu)
    _within(o, ref["o"], ref["o_b"], layout)
    # (gradients of keys and values shared by expansion are the caller's to sum: one per key head comes back)
    grads = lb.lb_attention_backward(*args, o, lse, do.cuda(), *cu)
    for a, n in zip(grads, ("dq", "dk", "dv", "dkr")):
        _within(a, ref[n], ref[n + "_b"], (layout, n))


def test_expanded_gradient_against_differences():
    # directional derivatives of L = sum(o do) in fp32: central differences of 64-bit references
    T, H, Hk, dn, dr, dv = 40, 4, 2, 16, 8, 24
    g = _gen(21)
    q, k, v, kr = (_normal(g, *s) for s in ((T, H, dn + dr), (T, Hk, dn), (T, Hk, dv), (T, dr)))
    do = _normal(g, T, H, dv)
    o, lse = lb.lb_attention_forward(*(x.cuda() for x in (q, k, v, kr)))
    grads = lb.lb_attention_backward(*(x.cuda() for x in (q, k, v, kr)), o, lse, do.cuda())

    def loss(q, k, v, kr):
        return float((R.attention(q, k, v, kr, [T], [T], True, (dn + dr) ** -0.5)["o"] * do.double()).sum())

    for i, x in enumerate((q, k, v, kr)):
        d = _normal(g, *x.shape).double()
        e = 1e-4
        hi, lo = ([y.double() + (s * e * d if j == i else 0) for j, y in enumerate((q, k, v, kr))] for s in (1, -1))
        # (attention() takes the type of q for its bounds only)
        num = (loss(*hi) - loss(*lo)) / (2 * e)
        got = float((grads[i].cpu().double() * d).sum())
        # differences: third derivative times e^2 / 6 ~ 1e-8 of the terms' size, fp32 sums of the gradient
        size = float((grads[i].cpu().double().abs() * d.abs()).sum())
        assert abs(got - num) <= 1e-5 * size, (i, got, num, size)


def test_small_f16_gradients_keep_their_digits():
    # |dO| around 1e-3 over 600 keys: dS of about 1e-6 to 1e-9, below fp16's normal range
    T, H, d = 600, 2, 64
    g = _gen(4)
    q, k, v = (_normal(g, T, H, d, dtype="f16") for _ in range(3))
    do = _normal(g, T, H, d, dtype="f16", std=1e-3)
    ref = R.attention(q, k, v, None, [T], [T], False, d ** -0.5, do)
    args = [x.cuda() for x in (q, k, v)] + [None]
    o, lse = lb.lb_attention_forward(*args, causal=False)
    dq, dk, dv, _ = lb.lb_attention_backward(*args, o, lse, do.cuda(), causal=False)
    for got, n in ((dq, "dq"), (dk, "dk"), (dv, "dv")):
        _within(got, ref[n], ref[n + "_b"], n)


def test_infinite_and_nan_keys_behind_the_mask():
    # keys and values of other sequences, and keys (not values) that the causal mask hides, may hold anything
    T, H, d = 100, 2, 64
    g = _gen(6)
    q, k, v = (_normal(g, T, H, d, dtype="bf16") for _ in range(3))
    ref = R.attention(q[:60], k[:60], v[:60], None, [60], [60], True, d ** -0.5)
    k2, v2 = k.clone(), v.clone()
    k2[60:], v2[60:] = float("inf"), float("nan")
    k2[59] = float("nan")
    o, _ = lb.lb_attention_forward(q.cuda(), k2.cuda(), v2.cuda(), None, _ints([0, 60]).cuda(), _ints([0, 60]).cuda())
    _within(o[:59], ref["o"][:59], ref["o_b"][:59], "masked keys")
    assert bool(torch.isnan(o[59]).all())


# ----------------------------------------------------------------------------
# streams, graphs, and the operators together
# ----------------------------------------------------------------------------
def test_capture_and_replay():
    case = ([300, 64], [1, 1], 8, 8, 64, 64, 40, 32, 16, "bf16", "bf16", "f16")
    P, paths, _, q, qd, f = _latent_call(case)
    T, fd = 2, f.cuda()
    w, kr = torch.empty((T, 2, 40), dtype=torch.bfloat16, device="cuda"), torch.empty((T, 32), dtype=torch.bfloat16, device="cuda")
    tr = [x.cuda() for x in (_normal(_gen(1), 90, 4, 96, dtype="f16"), _normal(_gen(2), 90, 2, 64, dtype="f16"),
                             _normal(_gen(3), 90, 2, 64, dtype="f16"), _normal(_gen(4), 90, 32, dtype="f16"),
                             _normal(_gen(5), 90, 4, 64, dtype="f16"))]
    ws = torch.empty(lb.lb_latent_attention_workspace_bytes(3, 2, 8, 40, 32), dtype=torch.uint8, device="cuda")
    ws2 = torch.empty(lb.lb_attention_backward_workspace_bytes(90, 90, 4, 2, 32), dtype=torch.uint8, device="cuda")
    pos = torch.arange(90, dtype=torch.int32, device="cuda")

    def body(out):
        lb.lb_latent_append(P.cache, w, kr, fd, *P.meta)
        lb.lb_latent_attention(qd, P.cache, paths, 8, 64, *P.meta, fd, out=out["a"], workspace=ws)
        lb.lb_rotate(tr[0][..., 64:], pos, fd, out=out["rot"])
        lb.lb_attention_forward(*tr[:4], o=out["o"], lse=out["lse"])
        lb.lb_attention_backward(*tr[:4], out["o"], out["lse"], tr[4], dq=out["dq"], dk=out["dk"], dv=out["dv"],
                                 dk_rope=out["dkr"], workspace=ws2)

    def outs():
        e = lambda *s, **k: torch.zeros(s, dtype=k.get("dtype", torch.float16), device="cuda")  # noqa: E731
        return dict(a=e(3, 8, 64, dtype=torch.bfloat16), rot=e(90, 4, 32), o=e(90, 4, 64), lse=e(90, 4, dtype=torch.float32),
                    dq=e(90, 4, 96), dk=e(90, 2, 64), dv=e(90, 2, 64), dkr=e(90, 32))

    eager, graphed = outs(), outs()
    w.normal_(), kr.normal_()
    body(eager)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        body(graphed)
    for i in range(4):
        w.normal_(), kr.normal_()
        for t in tr:
            t.mul_(0.9)
        for t in graphed.values():
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        body(eager)
        torch.cuda.synchronize()
        for n in eager:
            rows = 2 if n == "a" else None
            assert torch.equal(_bits(eager[n][:rows]), _bits(graphed[n][:rows])), (i, n)


def test_on_another_stream():
    case = LATENT[2]
    P, paths, _, _, qd, f = _latent_call(case)
    a = lb.lb_latent_attention(qd, P.cache, paths, 32, 64, *P.meta, f.cuda())
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    fd = f.cuda()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        b = lb.lb_latent_attention(qd, P.cache, paths, 32, 64, *P.meta, fd)
    out = torch.empty_like(a)
    ws = torch.empty(lb.lb_latent_attention_workspace_bytes(qd.shape[0], 5, 32, 112, 64), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    lb.lb_latent_attention(qd, P.cache, paths, 32, 64, *P.meta, fd, out=out, workspace=ws, stream=s)
    s.synchronize()
    n = sum(case[1])
    assert torch.equal(_bits(a[:n]), _bits(b[:n])) and torch.equal(_bits(a[:n]), _bits(out[:n]))


def _fused(d_in, Hk, dn, dv, r, seed):
    """A fused key/value layer with all its parts, and its dense weight in 64 bits."""
    g = _gen(seed)
    d_out = Hk * (dn + dv)
    paths, train = [], []
    for _ in range(2):
        U, V = torch.randn((d_out, r), generator=g).cuda(), torch.randn((d_in, r), generator=g).cuda()
        sc = [((torch.randn(n, generator=g).abs() + 0.1) * s).to(torch.float32).cuda()
              for n, s in ((d_out, 1.0), (d_in, d_in ** -0.5), (r, (2 * r) ** -0.5))]
        paths.append(lb.LittleBitPath(U=lb.lb_pack_signs(U, lb.LB_ROLE_U), V=lb.lb_pack_signs(V, lb.LB_ROLE_V), h=sc[0],
                                      g=sc[1], l=sc[2]))
        train.append(lb.LittleBitPathTrain(U_latent=U, V_latent=V))
    W = sum((torch.where(t.U_latent < 0, -1.0, 1.0).double() * p.h.double()[:, None] * p.l.double()) @
            (torch.where(t.V_latent < 0, -1.0, 1.0).double() * p.g.double()[:, None]).T for p, t in zip(paths, train)).cpu()
    return paths, train, W


def test_prompt_then_decode_from_the_cache():
    # a fused layer serves: the prompt by the expanded form, then tokens one by one from the paged cache, each against
    # the 64-bit attention over all tokens so far
    d_in, H, Hk, dn, dv, r, dr, page, n0, n1 = 96, 4, 2, 32, 32, 24, 16, 16, 45, 6
    T, g = n0 + n1, _gen(31)
    paths, _, W = _fused(d_in, Hk, dn, dv, r, 32)
    x, q, kr = _normal(g, T, d_in), _normal(g, T, H, dn + dr), _normal(g, T, dr)
    f, pos = _freqs(dr), torch.arange(T, dtype=torch.int32)
    y = x.double() @ W.T
    k64, v64 = _split(y, Hk, dn, dv)
    q64 = torch.cat([q[..., :dn].double(), R.turn(q[..., dn:].double(), pos, f)], -1)
    kr64 = R.turn(kr.double(), pos, f)
    ref = R.attention(q64, k64, v64, kr64, [T], [T], True, (dn + dr) ** -0.5)["o"]
    cache = lb.LatentCache.empty(8, page, r, dr, torch.float32)
    table = _ints([5, 2, 7, 0]).view(1, 4).cuda()
    xd, qd, krd, fd, pd = x.cuda(), q.cuda(), kr.cuda(), f.cuda(), pos.cuda()
    w = lb.lb_linear_latent(xd[:n0], paths, r)
    lb.lb_latent_append(cache, w, krd[:n0], fd, table, _ints([n0]).cuda(), _ints([0, n0]).cuda())
    kv = lb.lb_linear_from_latent(w, paths)
    kd, vd = _split(kv, Hk, dn, dv)
    qt = qd[:n0].clone()
    lb.lb_rotate(qt[..., dn:], pd[:n0], fd, out=qt[..., dn:])
    krt = lb.lb_rotate(krd[:n0, None, :], pd[:n0], fd)[:, 0]
    got = [lb.lb_attention_forward(qt, kd, vd, krt)[0]]
    for t in range(n0, T):
        w = lb.lb_linear_latent(xd[t:t + 1], paths, r)
        meta = (table, _ints([t + 1]).cuda(), _ints([0, 1]).cuda())
        lb.lb_latent_append(cache, w, krd[t:t + 1], fd, *meta)
        got.append(lb.lb_latent_attention(qd[t:t + 1], cache, paths, Hk, dv, *meta, fd))
    got = torch.cat(got).cpu().double()
    # fp32 throughout: the layer's bar (1e-5 of its outputs' norm) carries into scores and sums
    assert float((got - ref).norm() / ref.norm()) <= 3e-5
    # and the cache alone gives the prompt's rows too
    meta = (table, _ints([T]).cuda(), _ints([0, T]).cuda())
    whole = lb.lb_latent_attention(qd, cache, paths, Hk, dv, *meta, fd).cpu().double()
    assert float((whole - ref).norm() / ref.norm()) <= 3e-5


def test_training_step_through_the_fused_layer():
    # y = layer(x), attention(rotate(q), k, v, rotate(kr)), L = sum(o do): gradients of x, q and kr against autograd in
    # 64 bits through the dense weight
    d_in, H, Hk, dn, dv, r, dr, lens = 64, 4, 2, 32, 24, 16, 8, [37, 60]
    T, g = sum(lens), _gen(41)
    paths, train, W = _fused(d_in, Hk, dn, dv, r, 42)
    x, q, kr, do = _normal(g, T, d_in), _normal(g, T, H, dn + dr), _normal(g, T, dr), _normal(g, T, H, dv)
    f = _freqs(dr)
    pos = torch.cat([torch.arange(n) for n in lens]).int()
    x64, q64, kr64 = (t.double().requires_grad_() for t in (x, q, kr))
    k64, v64 = _split(x64 @ W.T, Hk, dn, dv)
    qq = torch.cat([q64[..., :dn], R.turn(q64[..., dn:], pos, f)], -1)
    kk = torch.cat([k64, R.turn(kr64, pos, f)[:, None].expand(T, Hk, dr)], -1)
    seg = torch.repeat_interleave(torch.arange(2), torch.tensor(lens))
    seen = (seg[:, None] == seg[None]) & (torch.arange(T)[:, None] >= torch.arange(T)[None])
    rep = lambda t: t.transpose(0, 1).repeat_interleave(H // Hk, 0)  # noqa: E731
    a = (qq.transpose(0, 1) @ rep(kk).transpose(1, 2) * (dn + dr) ** -0.5).masked_fill(~seen, -math.inf)
    ((torch.softmax(a, -1) @ rep(v64)).transpose(0, 1) * do.double()).sum().backward()
    xd, qd, krd, fd, pd, cu = x.cuda(), q.cuda(), kr.cuda(), f.cuda(), pos.cuda(), _cum(lens).cuda()
    y = lb.lb_linear_forward(xd, paths, r)
    kd, vd = _split(y, Hk, dn, dv)
    qt = qd.clone()
    lb.lb_rotate(qt[..., dn:], pd, fd, out=qt[..., dn:])
    krt = lb.lb_rotate(krd[:, None], pd, fd)[:, 0]
    o, lse = lb.lb_attention_forward(qt, kd, vd, krt, cu, cu)
    dy = torch.empty_like(y)
    dk, dvv = _split(dy, Hk, dn, dv)
    dq, _, _, dkr = lb.lb_attention_backward(qt, kd, vd, krt, o, lse, do.cuda(), cu, cu, dk=dk, dv=dvv)
    lb.lb_rotate(dq[..., dn:], pd, fd, inverse=True, out=dq[..., dn:])
    dkr = lb.lb_rotate(dkr[:, None], pd, fd, inverse=True)[:, 0]
    dx = lb.lb_linear_backward(xd, dy, paths, train)
    for got, want in ((dx, x64.grad), (dq, q64.grad), (dkr, kr64.grad)):
        got = got.cpu().double()
        assert float((got - want).norm() / want.norm()) <= 3e-5
