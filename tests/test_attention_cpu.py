"""CPU tests of the paged latent cache's and the attention calls' boundary: every refusal is returned before anything is
enqueued (no GPU is needed), and the pure size helpers."""
import ctypes

import pytest

import paper_2506_13771_amd as lb

P = 0x10000  # a stand-in for a device address: validation never reads it
OK, NULL, SHAPE, DTYPE, ALIGN, WORKSPACE, HIP, ARG = range(8)


@pytest.fixture(scope="module")
def lib():
    import os
    if not os.path.exists(lb.LIB_PATH):
        from paper_2506_13771_amd import _build
        _build.build()
    return lb.load_library()


def test_latent_row(lib):
    for r, dr in ((1, 0), (16, 0), (17, 0), (112, 64), (720, 0), (768, 0), (640, 256), (3, 2)):
        row = lb.lb_latent_row(r, dr)
        assert row % 32 == 0 and 2 * r + dr <= row < 2 * r + dr + 32
    for r, dr in ((0, 0), (-1, 0), (769, 0), (16, 3), (16, -2), (16, 258), (768, 2)):
        assert lb.lb_latent_row(r, dr) == 0


def test_workspace_bytes(lib):
    n = lb.lb_latent_attention_workspace_bytes
    assert n(1, 1, 1, 1, 0) > 0 and n(0, 0, 0, 16, 0) >= 0
    assert n(64, 64, 32, 112, 64) >= 64 * 32 * 288 * 6
    for bad in ((-1, 1, 1, 16, 0), (1, -1, 1, 16, 0), (1, 1, -1, 16, 0), (1, 1, 1, 0, 0), (1, 1, 1, 800, 0),
                (1, 1, 1, 16, 5), (1 << 31, 1, 64, 16, 0), (1, 1 << 25, 1, 16, 0)):
        assert n(*bad) == 0, bad
    m = lb.lb_attention_backward_workspace_bytes
    assert m(100, 50, 4, 2, 16) >= 100 * 4 * 4 + 50 * 2 * 16 * 4
    assert m(0, 0, 1, 1, 0) > 0
    for bad in ((-1, 1, 1, 1, 0), (1, -1, 1, 1, 0), (1, 1, 3, 2, 0), (1, 1, 1, 0, 0), (1, 1, 1, 1, -1), (1, 1, 1, 1, 193),
                (1 << 30, 1, 4, 4, 0)):
        assert m(*bad) == 0, bad


def _rotate(lib, **kw):
    a = dict(x=P, dt=lb.LB_F32, T=2, H=3, d=8, x_t=24, x_h=8, pos=P, freqs=P, inv=0, y=4 * P, y_t=24, y_h=8)
    a.update(kw)
    return lib.lb_rotate(a["x"], a["dt"], a["T"], a["H"], a["d"], a["x_t"], a["x_h"], a["pos"], a["freqs"], a["inv"],
                         a["y"], a["y_t"], a["y_h"], None)


@pytest.mark.parametrize("kw,want", [
    (dict(dt=3), DTYPE), (dict(dt=-1), DTYPE), (dict(T=-1), SHAPE), (dict(d=7), SHAPE), (dict(d=258), SHAPE),
    (dict(x_t=-1), SHAPE), (dict(y_h=1 << 41), SHAPE), (dict(T=1 << 30, H=4), SHAPE), (dict(x=0), NULL), (dict(y=0), NULL),
    (dict(pos=0), NULL), (dict(freqs=0), NULL), (dict(x=P + 1), ALIGN), (dict(y=4 * P + 2), ALIGN), (dict(pos=P + 2), ALIGN),
    (dict(y_h=7), ARG), (dict(y_t=23), ARG), (dict(y_t=0), ARG), (dict(y=P + 64), ARG), (dict(y=P, y_t=32), ARG),
    (dict(T=0), OK), (dict(H=0), OK), (dict(d=0), OK), (dict(T=0, x=0), OK)])
def test_rotate_refuses(lib, kw, want):
    assert _rotate(lib, **kw) == want


def _cache(**kw):
    a = dict(data=P, dtype=lb.LB_BF16, n_pages=4, page_size=16, r=16, d_rope=8, table=P, n_seq=2, max_pages=2, lens=P, cu=P)
    a.update(kw)
    return lb.lb_latent_cache(*[a[f] for f, _ in lb.lb_latent_cache._fields_])


CACHES = [
    (dict(dtype=9), DTYPE), (dict(n_pages=-1), SHAPE), (dict(page_size=0), SHAPE), (dict(r=0), SHAPE), (dict(r=769), SHAPE),
    (dict(d_rope=7), SHAPE), (dict(d_rope=258), SHAPE), (dict(r=768, d_rope=2), SHAPE), (dict(n_seq=-1), SHAPE),
    (dict(max_pages=-1), SHAPE), (dict(n_pages=1 << 27, page_size=16), SHAPE), (dict(max_pages=1 << 30, page_size=2), SHAPE), (dict(max_pages=(1 << 30) + 1, page_size=1, n_seq=1), SHAPE),
    (dict(data=0), NULL), (dict(table=0), NULL), (dict(lens=0), NULL), (dict(cu=0), NULL), (dict(data=P + 8), ALIGN),
    (dict(table=P + 2), ALIGN), (dict(cu=P + 1), ALIGN)]


def _append(lib, cache=None, null=False, **kw):
    a = dict(w=64 * P, kr=128 * P, kt=8, dt=lb.LB_F32, T=3, freqs=P)
    a.update(kw)
    c = _cache() if cache is None else cache
    return lib.lb_latent_append(None if null else ctypes.byref(c), a["w"], a["kr"], a["kt"], a["dt"], a["T"], a["freqs"], None)


@pytest.mark.parametrize("kw,want", CACHES)
def test_append_refuses_caches(lib, kw, want):
    assert _append(lib, _cache(**kw)) == want


@pytest.mark.parametrize("kw,want", [
    (dict(null=True), NULL), (dict(dt=5), DTYPE), (dict(T=-1), SHAPE), (dict(T=1 << 30), SHAPE), (dict(kt=-1), SHAPE),
    (dict(w=0), NULL), (dict(kr=0), NULL), (dict(w=64 * P + 2), ALIGN), (dict(kr=128 * P + 1), ALIGN), (dict(freqs=P + 1), ALIGN),
    (dict(w=P + 64), ARG), (dict(kr=P), ARG), (dict(T=0), OK), (dict(cache=_cache(n_seq=0)), OK)])
def test_append_refuses(lib, kw, want):
    assert _append(lib, **kw) == want


def _paths(**kw):
    a = dict(U=P, V=0, h=P, g=0, l=0)
    a.update(kw)
    return (lb.lb_path * 2)(*[lb.lb_path(a["U"], a["V"], a["h"], a["g"], a["l"]) for _ in range(2)])


def _latent(lib, cache=None, paths=None, nulls=(), **kw):
    a = dict(q=64 * P, act=lb.LB_BF16, T=3, H=4, Hk=2, dn=32, dv=16, q_t=160, q_h=40, sc=lb.LB_F16, freqs=P, scale=0.1,
             out=128 * P, ws=256 * P, n=1 << 30)
    a.update(kw)
    c, p = cache or _cache(), _paths() if paths is None else paths
    return lib.lb_latent_attention(a["q"], a["act"], a["T"], a["H"], a["Hk"], a["dn"], a["dv"], a["q_t"], a["q_h"],
                                   None if "paths" in nulls else p, a["sc"], None if "cache" in nulls else ctypes.byref(c),
                                   a["freqs"], a["scale"], a["out"], a["ws"], a["n"], None)


@pytest.mark.parametrize("kw,want", CACHES)
def test_latent_attention_refuses_caches(lib, kw, want):
    assert _latent(lib, _cache(**kw)) == want


@pytest.mark.parametrize("kw,want", [
    (dict(nulls=("cache",)), NULL), (dict(nulls=("paths",)), NULL), (dict(act=4), DTYPE), (dict(sc=-2), DTYPE),
    (dict(T=-1), SHAPE), (dict(H=3), SHAPE), (dict(Hk=0), SHAPE), (dict(dn=257), SHAPE), (dict(dv=257), SHAPE),
    (dict(dn=-1), SHAPE), (dict(q_t=-5), SHAPE), (dict(T=1 << 29), SHAPE), (dict(scale=0.0), ARG), (dict(scale=-1.0), ARG),
    (dict(scale=float("nan")), ARG), (dict(scale=float("inf")), ARG), (dict(q=0), NULL), (dict(out=0), NULL),
    (dict(ws=0), NULL), (dict(paths=_paths(U=0)), NULL), (dict(paths=_paths(h=0)), NULL), (dict(paths=_paths(U=P + 2)), ALIGN),
    (dict(paths=_paths(h=P + 1)), ALIGN), (dict(q=64 * P + 1), ALIGN), (dict(out=128 * P + 1), ALIGN),
    (dict(ws=256 * P + 128), ALIGN), (dict(n=1000), WORKSPACE), (dict(out=64 * P + 320), ARG), (dict(out=P + 64), ARG),
    (dict(T=1 << 20, cache=_cache(r=1, d_rope=0), dn=1, dv=1), SHAPE), (dict(T=0), OK),
    (dict(dv=0), OK), (dict(cache=_cache(n_seq=0)), OK)])
def test_latent_attention_refuses(lib, kw, want):
    assert _latent(lib, **kw) == want


def _attn(**kw):
    a = dict(q=P, k=16 * P, v=32 * P, k_rope=48 * P, dtype=lb.LB_BF16, Tq=8, Tk=9, H=4, Hk=2, d_nope=32, d_rope=16, d_v=24,
             q_t=192, q_h=48, k_t=64, k_h=32, v_t=48, v_h=24, kr_t=16, cu_q=0, cu_k=0, n_seq=0, causal=1, scale=0.2)
    a.update(kw)
    return lb.lb_attention(*[a[f] for f, _ in lb.lb_attention._fields_])


ATTNS = [
    (dict(dtype=7), DTYPE), (dict(Tq=-1), SHAPE), (dict(Tk=-1), SHAPE), (dict(H=5), SHAPE), (dict(Hk=0), SHAPE),
    (dict(d_nope=0, d_rope=0), SHAPE), (dict(d_nope=180, d_rope=13), SHAPE), (dict(d_nope=-8, d_rope=24), SHAPE),
    (dict(d_v=0), SHAPE), (dict(d_v=129), SHAPE), (dict(n_seq=-1), SHAPE), (dict(q_t=-1), SHAPE), (dict(v_h=-1), SHAPE),
    (dict(Tq=1 << 30), SHAPE), (dict(cu_q=P, cu_k=P, n_seq=1 << 22), SHAPE), (dict(cu_q=P), ARG), (dict(cu_k=P), ARG), (dict(scale=0.0), ARG),
    (dict(scale=float("nan")), ARG), (dict(q=0), NULL), (dict(k=0), NULL), (dict(v=0), NULL), (dict(k_rope=0), NULL),
    (dict(q=P + 1), ALIGN), (dict(k=16 * P + 1), ALIGN), (dict(v=32 * P + 1), ALIGN), (dict(k_rope=48 * P + 1), ALIGN),
    (dict(cu_q=P + 1, cu_k=P, n_seq=1), ALIGN)]


@pytest.mark.parametrize("kw,want", ATTNS + [(dict(Tq=0), OK), (dict(H=0), OK), (dict(cu_q=P, cu_k=P, n_seq=0), OK)])
def test_attention_forward_refuses(lib, kw, want):
    assert lib.lb_attention_forward(ctypes.byref(_attn(**kw)), 64 * P, 80 * P, None) == want


def test_attention_forward_refuses_outputs(lib):
    f = lambda o, lse: lib.lb_attention_forward(ctypes.byref(_attn()), o, lse, None)  # noqa: E731
    assert lib.lb_attention_forward(None, P, P, None) == NULL
    assert f(0, 80 * P) == NULL
    assert f(64 * P + 1, 80 * P) == ALIGN and f(64 * P, 80 * P + 2) == ALIGN
    assert f(P + 64, 80 * P) == ARG and f(64 * P, 16 * P) == ARG and f(64 * P, 64 * P) == ARG and f(48 * P, 80 * P) == ARG


def _grads(**kw):
    a = dict(dq=96 * P, dk=112 * P, dv=128 * P, dk_rope=144 * P, dk_t=64, dk_h=32, dv_t=48, dv_h=24)
    a.update(kw)
    return lb.lb_attention_grads(*[a[f] for f, _ in lb.lb_attention_grads._fields_])


def _backward(lib, attn=None, grads=None, **kw):
    a = dict(o=64 * P, lse=80 * P, do=160 * P, ws=256 * P, n=1 << 30)
    a.update(kw)
    return lib.lb_attention_backward(ctypes.byref(attn or _attn()), a["o"], a["lse"], a["do"],
                                     ctypes.byref(grads or _grads()), a["ws"], a["n"], None)


@pytest.mark.parametrize("kw,want", ATTNS + [(dict(H=0), OK), (dict(Tq=0, Tk=0), OK)])
def test_attention_backward_refuses_operands(lib, kw, want):
    assert _backward(lib, _attn(**kw)) == want


@pytest.mark.parametrize("kw,want", [
    (dict(o=0), NULL), (dict(lse=0), NULL), (dict(do=0), NULL), (dict(ws=0), NULL), (dict(grads=_grads(dq=0)), NULL),
    (dict(grads=_grads(dk=0)), NULL), (dict(grads=_grads(dv=0)), NULL), (dict(grads=_grads(dk_rope=0)), NULL),
    (dict(do=160 * P + 1), ALIGN), (dict(lse=80 * P + 1), ALIGN), (dict(ws=256 * P + 16), ALIGN),
    (dict(grads=_grads(dk=112 * P + 1)), ALIGN), (dict(n=64), WORKSPACE), (dict(grads=_grads(dk_t=63)), ARG),
    (dict(grads=_grads(dv_h=23)), ARG), (dict(grads=_grads(dk_t=-1)), SHAPE)])
def test_attention_backward_refuses(lib, kw, want):
    assert _backward(lib, **kw) == want
    assert lib.lb_attention_backward(None, P, P, P, None, P, 1, None) == NULL
    assert lib.lb_attention_backward(ctypes.byref(_attn()), P, P, P, None, P, 1, None) == NULL


def test_binding_refuses_cpu_tensors_and_wrong_shapes(lib):
    torch = pytest.importorskip("torch")
    if torch.cuda.is_available():
        dev = "cuda"
    else:
        dev = None
    x, pos, f = torch.zeros(2, 3, 8), torch.zeros(2, dtype=torch.int32), torch.zeros(4)
    with pytest.raises((ValueError, RuntimeError, AssertionError)):
        lb.lb_rotate(x, pos, f)  # CPU tensors never reach the library
    if dev is None:
        return
    x, pos, f = x.to(dev), pos.to(dev), f.to(dev)
    for bad in ((x, pos.long(), f), (x, pos[:1], f), (x, pos, f.double()), (x, pos, f[:3]), (x[..., ::2], pos, f[:2]),
                (x[0], pos, f)):
        with pytest.raises(ValueError):
            lb.lb_rotate(*bad)


def test_packed_structures_match_the_header(lib):
    import struct
    for pack, cls, n in (("@PiqqqqPqqPP", lb.lb_latent_cache, 11), ("@PPPPi14qPPqif", lb.lb_attention, 24),
                         ("@4P4q", lb.lb_attention_grads, 8), ("@10P", lb.lb_path * 2, 10)):
        vals = list(range(1, n + 1))
        raw = struct.pack(pack, *vals)
        assert len(raw) == ctypes.sizeof(cls)
        if hasattr(cls, "_fields_"):
            got = cls.from_buffer_copy(raw)
            assert [getattr(got, f) for f, _ in cls._fields_] == vals
