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
