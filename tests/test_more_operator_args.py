"""Refusals of window attention, the paged cache and draft verification that need no device."""
import ctypes
import warnings

import pytest
import torch

from test_operator_args import attn, heads

INT_MAX = 2 ** 31 - 1


@pytest.fixture(scope="module")
def g():
    from paper_2608_01528_gb300 import build, gramspace
    build.build()
    gramspace.load_library()
    return gramspace


def test_window_arguments(g):
    L, ref = g.load_library(), ctypes.byref

    def forward(a, w, o=None):
        hs = [heads(g) for _ in range(3)] + [o or heads(g)]
        return L.gs_window_attention(ref(a), ref(w) if w else None, *map(ref, hs), None, None, 0, None)

    def back(a, w):
        h = [heads(g) for _ in range(8)]
        return L.gs_window_attention_backward(ref(a), ref(w) if w else None, *map(ref, h[:4]), None, *map(ref, h[4:]), None, 0, None)

    n = ctypes.c_longlong(7)
    for call in (forward, back, lambda a, w: L.gs_window_attention_workspace(ref(a), ref(w) if w else None, 0, ref(n))):
        for w in (None, g._Window(0, 0, 0, None), g._Window(-3, 0, 0, None), g._Window(4, -1, 0, None)):
            assert call(attn(g), w) == g.GS_ERR_INVALID_ARG
        assert call(attn(g), g._Window(4, 1, 0, 2)) == g.GS_ERR_ALIGNMENT
        ok = g._Window(4, 1, 0, None)
        assert call(attn(g, dtype=7), ok) == g.GS_ERR_INVALID_ARG
        assert call(attn(g, Hq=3), ok) == g.GS_ERR_SHAPE
        assert call(attn(g, dk=200), ok) == g.GS_ERR_UNSUPPORTED
    assert forward(attn(g), ok) == g.GS_ERR_INVALID_ARG  # null data
    assert forward(attn(g, B=0), ok) == g.GS_OK and forward(attn(g), ok, heads(g, row=0)) == g.GS_ERR_SHAPE


def test_window_wrapper(g):
    q, k, v = torch.zeros(2, 5, 4, 8), torch.zeros(2, 7, 2, 8), torch.zeros(2, 7, 2, 6)
    with pytest.raises(TypeError, match="CUDA"):
        g.window_attention(q, k, v, 3)
    for w in (0, -1):
        with pytest.raises((ValueError, TypeError)):
            g.window_attention(q, k, v, w)
    dev = q.device
    for bad in ((0, 0, 0), (3, -1, 0), (3, 0, 2 ** 31), (3, 0, torch.zeros(2)), (3, 0, torch.zeros(3, dtype=torch.int32))):
        with pytest.raises(ValueError):
            g._window(*bad, 2, dev)
    w = g._window(None, 2 ** 40, -5, 2, dev)
    assert (w.window, w.sinks, w.start) == (INT_MAX, INT_MAX, -5)
    a = [t.clone().requires_grad_() for t in (q, k, v)]
    with pytest.warns(UserWarning, match="window_attention_backward"), pytest.raises(TypeError, match="CUDA"):
        g.window_attention(*a, 3)
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        with torch.no_grad(), pytest.raises(TypeError, match="CUDA"):
            g.window_attention(*a, 3)


def paged(g, **kw):
    d = dict(dtype=0, B=1, Lq=1, Hq=4, Hkv=2, dk=8, dv=8, scale=1.0, pages=4, page_size=16, columns=3, table=16, ld_table=3, lens=16,
             q_lens=None, window=INT_MAX, sinks=0, flags=0)
    d.update(kw)
    return g._Paged(*(d[k] for k, _ in g._Paged._fields_))


def test_paged_arguments(g):
    L, ref = g.load_library(), ctypes.byref

    def call(a, q=None, k=None, v=None, o=None):
        hs = [x or heads(g) for x in (q, k, v, o)]
        return L.gs_paged_attention(ref(a), *map(ref, hs), None, None, 0, None)

    n = ctypes.c_longlong(7)
    space = lambda a: L.gs_paged_attention_workspace(ref(a), ref(n))  # noqa: E731
    for kw in (dict(dtype=2), dict(scale=0.0), dict(scale=float("nan")), dict(flags=3), dict(window=0), dict(window=-1), dict(sinks=-1)):
        assert call(paged(g, **kw)) == space(paged(g, **kw)) == g.GS_ERR_INVALID_ARG, kw
    for kw in (dict(B=-1), dict(Lq=-1), dict(Hq=3), dict(Hkv=0), dict(dk=0), dict(pages=-1), dict(page_size=0), dict(columns=-1),
               dict(ld_table=2), dict(pages=2 ** 20, page_size=2 ** 11), dict(columns=2 ** 20, page_size=2 ** 11, ld_table=2 ** 20),
               dict(Lq=2 ** 30), dict(B=2 ** 20, Lq=2 ** 12)):
        assert call(paged(g, **kw)) == space(paged(g, **kw)) == g.GS_ERR_SHAPE, kw
    for kw in (dict(dk=129), dict(dv=129)):
        assert call(paged(g, **kw)) == g.GS_ERR_UNSUPPORTED, kw
    for kw in (dict(table=18), dict(lens=17), dict(q_lens=2)):
        assert call(paged(g, **kw)) == g.GS_ERR_ALIGNMENT, kw
    assert n.value == 0
    assert call(paged(g), o=heads(g, head=0)) == g.GS_ERR_SHAPE and call(paged(g), k=heads(g, batch=-1)) == g.GS_ERR_SHAPE
    d = heads(g, data=16)
    for kw in (dict(lens=None), dict(table=None)):
        assert call(paged(g, **kw), d, d, d, d) == g.GS_ERR_INVALID_ARG, kw
    assert call(paged(g)) == g.GS_ERR_INVALID_ARG                        # null data
    assert call(paged(g), heads(g, data=18), d, d, d) == g.GS_ERR_ALIGNMENT
    assert call(paged(g, B=0)) == call(paged(g, Lq=0)) == g.GS_OK
    assert L.gs_paged_attention_workspace(None, ref(n)) == g.GS_ERR_INVALID_ARG
    assert L.gs_paged_attention_workspace(ref(paged(g)), None) == g.GS_ERR_INVALID_ARG


def test_slot_arguments(g):
    L = g.load_library()
    base = dict(lens=4096, added=8192, B=2, Lnew=3, page_size=16, pages=10, free=12288, n_free=5, frm=None, table=16384, ld=4, columns=4,
                slots=20480, new=24576, taken=28672)

    def call(**kw):
        d = dict(base, **kw)
        return L.gs_page_slots(*(d[k] for k in base), None)

    for kw in (dict(B=-1), dict(Lnew=-1), dict(page_size=0), dict(pages=-1), dict(n_free=-1), dict(columns=-1), dict(ld=3),
               dict(pages=2 ** 28), dict(columns=2 ** 27, ld=2 ** 27), dict(B=2 ** 30), dict(B=2 ** 20, Lnew=2 ** 12)):
        assert call(**kw) == g.GS_ERR_SHAPE, kw
    for kw in (dict(lens=None), dict(added=None), dict(free=None), dict(table=None), dict(slots=None)):
        assert call(**kw) == g.GS_ERR_INVALID_ARG, kw
    for kw in (dict(lens=4098), dict(slots=20481), dict(taken=28673), dict(frm=2)):
        assert call(**kw) == g.GS_ERR_ALIGNMENT, kw
    # outputs over inputs, or over one another
    for kw in (dict(new=4096), dict(new=4100), dict(slots=8180), dict(table=12300), dict(taken=12288), dict(frm=28672), dict(new=20480),
               dict(taken=16384 + 28), dict(slots=16384 - 20)):
        assert call(**kw) == g.GS_ERR_INVALID_ARG, kw
    assert call(B=0, taken=None) == g.GS_OK


def test_slot_wrapper(g):
    i = torch.zeros(3, dtype=torch.int32)
    t = torch.zeros(3, 4, dtype=torch.int32)
    with pytest.raises(TypeError, match="CUDA"):
        g.page_slots(i, i, t, i, 16, 2, 10)
    for bad in ((i[:2], i, t, i), (i, i.long(), t, i), (i, i, t.t(), i), (i, i, t.float(), i), (i, i, t[0], i), (i, i, t, t),
                (i, i, t, i[::2])):
        with pytest.raises(ValueError):
            g.page_slots(*bad, 16, 2, 10)
    for kw in (dict(free_from=i), dict(out={"slots": t}), dict(out={"taken": i}), dict(out={"lens": i.float()})):
        with pytest.raises(ValueError):
            g.page_slots(i, i, t, i, 16, 2, 10, **kw)
    with pytest.raises(ValueError):
        g.page_slots(i, i, t, i, 16, -1, 10)
    with pytest.raises(ValueError):
        g.page_slots(i, i, t, i, 2 ** 40, 1, 10)


def test_store(g):
    L, ref = g.load_library(), ctypes.byref

    def call(dtype=0, B=1, n=2, H=2, dk=8, dv=8, ld=2, pages=4, size=16, slots=16, k=None, v=None, kc=None, vc=None):
        hs = [x or heads(g, data=16) for x in (k, v, kc, vc)]
        return L.gs_page_store(dtype, B, n, H, dk, dv, ref(hs[0]), ref(hs[1]), slots, ld, pages, size, ref(hs[2]), ref(hs[3]), None)

    assert call(dtype=2) == call(slots=None) == call(k=heads(g)) == call(vc=heads(g)) == g.GS_ERR_INVALID_ARG
    for kw in (dict(B=-1), dict(n=-1), dict(H=0), dict(dk=0), dict(dv=0), dict(ld=1), dict(pages=-1), dict(size=0), dict(pages=2 ** 27),
               dict(B=2 ** 20, n=2 ** 12, ld=2 ** 12), dict(H=2 ** 28), dict(kc=heads(g, data=16, row=0)),
               dict(vc=heads(g, data=16, batch=0)), dict(k=heads(g, data=16, batch=-1))):
        assert call(**kw) == g.GS_ERR_SHAPE, kw
    assert call(k=heads(g, data=18)) == call(slots=18) == g.GS_ERR_ALIGNMENT
    assert call(B=0) == call(n=0, ld=0) == call(pages=0) == g.GS_OK
    k, c, s = torch.zeros(2, 3, 4, 8), torch.zeros(5, 16, 4, 8), torch.zeros(2, 3, dtype=torch.int32)
    with pytest.raises(TypeError, match="CUDA"):
        g.page_store(k, k, s, c, c)
    for bad in ((k[0], k, s, c, c), (k, k, s[:1], c, c), (k, k, s.long(), c, c), (k, k, s, c[:, :, :2], c), (k, k, s, c, c[..., :6]),
                (k, k, s, c[0], c), (k, k, s, c, c[:4])):
        with pytest.raises(ValueError):
            g.page_store(*bad)
    for bad in ((k, k.bfloat16(), s, c, c), (k, k, s, c.bfloat16(), c), (k.half(), k.half(), s, c.half(), c.half())):
        with pytest.raises(TypeError):
            g.page_store(*bad)


def test_paged_wrapper(g):
    q, c = torch.zeros(2, 1, 4, 8), torch.zeros(5, 16, 2, 8)
    t, n = torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(TypeError, match="CUDA"):
        g.paged_attention(q, c, c, t, n)
    for bad in ((q[0], c, c, t, n), (q, c[..., :6], c, t, n), (q, c, c[:4], t, n), (q, c, c, t[:1], n), (q, c, c, t.long(), n),
                (q, c, c, t, n[:1]), (q, c, c, t, n.float()), (q, c.transpose(2, 3), c, t, n)):
        with pytest.raises(ValueError):
            g.paged_attention(*bad)
    for kw in (dict(window=0), dict(sinks=-1), dict(q_lens=n[:1])):
        with pytest.raises(ValueError):
            g.paged_attention(q, c, c, t, n, **kw)
    with pytest.raises(TypeError):
        g.paged_attention(q, c.bfloat16(), c, t, n)


def test_verify_arguments(g):
    L = g.load_library()
    base = dict(P=16, D=16, dtype=0, B=2, K=3, M=100, pb=400, pr=100, db=300, dr=100, drafts=16, lens=None, U=16, accepted=16, tokens=16)

    def call(**kw):
        d = dict(base, **kw)
        return L.gs_verify_drafts(*(d[k] for k in base), None)

    for kw in (dict(P=None), dict(U=None), dict(drafts=None), dict(dtype=2), dict(accepted=None, tokens=None)):
        assert call(**kw) == g.GS_ERR_INVALID_ARG, kw
    for kw in (dict(B=-1), dict(K=-1), dict(M=0), dict(M=2 ** 19 + 1), dict(pb=-1), dict(pr=-1), dict(db=-1), dict(dr=-1),
               dict(B=2 ** 20, K=2 ** 12)):
        assert call(**kw) == g.GS_ERR_SHAPE, kw
    for kw in (dict(P=18), dict(D=18), dict(drafts=18), dict(lens=17), dict(U=18), dict(accepted=18), dict(tokens=18)):
        assert call(**kw) == g.GS_ERR_ALIGNMENT, kw
    assert call(B=0) == g.GS_OK
    P, D = torch.zeros(2, 4, 10), torch.zeros(2, 3, 10)
    x, u, n = torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, 4), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(TypeError, match="CUDA"):
        g.verify_drafts(P, D, x, u)
    for bad in ((P[0], D, x, u), (P, D[:1], x, u), (P, P, x, u), (P, D, x.long(), u), (P, D, x[:, :2], u), (P, D, x, u[:, :3]),
                (P, D, x, u.double()), (torch.zeros(2, 10, 4).transpose(1, 2), D, x, u), (P[:, :0], D, x, u)):
        with pytest.raises(ValueError):
            g.verify_drafts(*bad)
    with pytest.raises(TypeError):
        g.verify_drafts(P, D.bfloat16(), x, u)
    for kw in (dict(draft_lens=n.float()), dict(draft_lens=n[:1]), dict(out={"tokens": x}), dict(out={"accepted": x})):
        with pytest.raises(ValueError):
            g.verify_drafts(P, D, x, u, **kw)
