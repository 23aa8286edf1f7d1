"""Refusals of cross attention and sampling that need no device."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def g():
    from paper_2608_01528_gb300 import build, gramspace
    build.build()
    gramspace.load_library()
    return gramspace


def attn(g, **kw):
    d = dict(dtype=0, B=1, Lq=2, Lk=3, Hq=4, Hkv=2, dk=8, dv=8, scale=1.0, key_lens=None, key_mask=None, ld_mask=0, flags=0)
    d.update(kw)
    return g._Attn(*(d[k] for k, _ in g._Attn._fields_))


def heads(g, data=None, batch=1000, row=100, head=10):
    return g._Heads(data, batch, row, head)


def forward(g, a, q=None, k=None, v=None, o=None):
    hs = [x if x is not None else heads(g) for x in (q, k, v, o)]
    return g.load_library().gs_cross_attention(ctypes.byref(a), *map(ctypes.byref, hs), None, None, 0, None)


def test_attention_arguments(g):
    for kw in (dict(dtype=2), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(flags=3)):
        assert forward(g, attn(g, **kw)) == g.GS_ERR_INVALID_ARG, kw
    for kw in (dict(B=-1), dict(Lq=-1), dict(Lk=-1), dict(Hq=0), dict(Hkv=0), dict(Hq=3), dict(dk=0), dict(dv=0),
               dict(Lk=2 ** 31 - 1), dict(Lq=2 ** 30), dict(B=2 ** 20, Lq=2 ** 12), dict(B=2 ** 20, Lk=2 ** 12),
               dict(key_mask=16, ld_mask=2)):
        assert forward(g, attn(g, **kw)) == g.GS_ERR_SHAPE, kw
    for kw in (dict(dk=129), dict(dv=129)):
        assert forward(g, attn(g, **kw)) == g.GS_ERR_UNSUPPORTED, kw
    bad = heads(g, batch=-1)
    assert forward(g, attn(g), q=bad) == g.GS_ERR_SHAPE and forward(g, attn(g), o=bad) == g.GS_ERR_SHAPE
    assert forward(g, attn(g), o=heads(g, row=0)) == g.GS_ERR_SHAPE  # rows of the output on one another
    assert forward(g, attn(g)) == g.GS_ERR_INVALID_ARG               # null data
    assert forward(g, attn(g, B=0)) == g.GS_OK and forward(g, attn(g, Lq=0)) == g.GS_OK
    L = g.load_library()
    n = ctypes.c_longlong(7)
    assert L.gs_cross_attention_workspace(ctypes.byref(attn(g, dk=129)), 0, ctypes.byref(n)) == g.GS_ERR_UNSUPPORTED
    assert n.value == 0
    assert L.gs_cross_attention_workspace(None, 0, ctypes.byref(n)) == g.GS_ERR_INVALID_ARG
    assert L.gs_cross_attention_workspace(ctypes.byref(attn(g)), 0, None) == g.GS_ERR_INVALID_ARG
    h = [heads(g) for _ in range(8)]
    back = lambda a, hs, lse=None: L.gs_cross_attention_backward(  # noqa: E731
        ctypes.byref(a), *map(ctypes.byref, hs[:4]), lse, *map(ctypes.byref, hs[4:]), None, 0, None)
    assert back(attn(g), h) == g.GS_ERR_INVALID_ARG
    assert back(attn(g, B=0), h) == g.GS_OK
    assert back(attn(g), h[:5] + [heads(g, head=0)] + h[6:]) == g.GS_ERR_SHAPE


def test_attention_wrapper(g):
    q, k, v = torch.zeros(2, 5, 4, 8), torch.zeros(2, 7, 2, 8), torch.zeros(2, 7, 2, 6)
    for bad in ((q[0], k, v), (q, k[:1], v), (q, k, v[:, :3]), (q, torch.zeros(2, 7, 2, 9), v), (q, k, v[:, :, :1]),
                (q, torch.zeros(2, 7, 8, 2).transpose(2, 3), v)):
        with pytest.raises(ValueError):
            g.cross_attention(*bad)
    for bad in ((q.double(), k, v), (q, k.bfloat16(), v), (q.half(), k.half(), v.half())):
        with pytest.raises(TypeError):
            g.cross_attention(*bad)
    with pytest.raises(TypeError):  # host tensors
        g.cross_attention(q, k, v)
    for kw in (dict(key_lens=torch.zeros(2)), dict(key_lens=torch.zeros(3, dtype=torch.int32)),
               dict(key_mask=torch.zeros(2, 7)), dict(key_mask=torch.zeros(2, 6, dtype=torch.bool)),
               dict(key_mask=torch.zeros(7, 2, dtype=torch.bool).t())):
        with pytest.raises(ValueError):
            g.cross_attention(q, k, v, **kw)


def test_sampling_arguments(g):
    L = g.load_library()
    how = g._Sampling(1.0, 1.0, 0.0, 0)
    d = 16  # never dereferenced: every call below returns before touching memory

    def call(S=d, dt=0, N=4, M=10, ld=10, h=how, U=d, index=d, prob=d):
        return L.gs_sample_scores(S, dt, N, M, ld, ctypes.byref(h) if h is not None else None, U, index, prob, None)

    assert call(dt=2) == g.GS_ERR_INVALID_ARG and call(h=None) == g.GS_ERR_INVALID_ARG
    for kw in (dict(N=-1), dict(N=2 ** 31), dict(M=0), dict(M=2 ** 19 + 1, ld=2 ** 20), dict(ld=9)):
        assert call(**kw) == g.GS_ERR_SHAPE, kw
    for kw in (dict(S=None), dict(U=None), dict(index=None, prob=None)):
        assert call(**kw) == g.GS_ERR_INVALID_ARG, kw
    assert call(N=0, S=None, U=None) == g.GS_OK
    S, U = torch.zeros(3, 5), torch.zeros(3)
    for kw in (dict(U=torch.zeros(2)), dict(U=torch.zeros(3, dtype=torch.float64)), dict(temperature=torch.zeros(4)),
               dict(top_k=torch.zeros(3)), dict(out={"index": torch.zeros(3)}), dict(out={"prob": torch.zeros(2)})):
        with pytest.raises(ValueError):
            g.sample_scores(**{"S": S, "U": U, **kw})
    with pytest.raises(TypeError):
        g.sample_scores(S.double(), U)
    with pytest.raises(TypeError):
        g.sample_scores(S, U)
    with pytest.raises(ValueError):
        g.sample_scores(S.t(), torch.zeros(5))


def test_sizes_past_a_c_int(g):
    """Broadcast tensors reach sizes that a C int would cut to small ones."""
    big = 2 ** 32 + 1
    one = torch.zeros(1, 1, 1, 8)
    for q, k in ((one.expand(big, 1, 1, 8), one.expand(big, 1, 1, 8)), (one, one.expand(1, big, 1, 8)),
                 (one.expand(1, big, 1, 8), one)):
        with pytest.raises(ValueError, match="2\\^31"):
            g.cross_attention(q, k, k)
    with pytest.raises(ValueError):
        g.sample_scores(torch.zeros(big, dtype=torch.bfloat16, device="meta")[None], torch.zeros(1, device="meta"))


def test_top_k_past_a_c_int(g):
    """2^32 + 1 means all scores, not one."""
    seen = []

    class Library:
        def gs_sample_scores(self, S, code, N, M, ld, how, *rest):
            seen.append(how._obj.top_k)
            return g.GS_OK

    class Fake(torch.Tensor):  # a host tensor that says it is a CUDA one: the call goes as far as the library
        is_cuda = True

    S = torch.zeros(2, 6).as_subclass(Fake)
    load, on, stream = g.load_library, g._on_stream, g._stream
    g.load_library, g._on_stream, g._stream = Library, lambda *a: g._STAY, lambda *a: 0
    try:
        for k in (2 ** 32 + 1, 7, 6, 3, 0, -5, -2 ** 32 + 2):
            g.sample_scores(S, torch.zeros(2), top_k=k)
    finally:
        g.load_library, g._on_stream, g._stream = load, on, stream
    assert seen == [6, 6, 6, 3, 0, 0, 0]


def test_stream_of_another_device(g):
    class Stream:
        device = torch.device("cuda", 1)

    with pytest.raises(ValueError, match="cuda:0"):
        g._on_stream(torch.device("cuda", 0), Stream())


def test_arrays_off_their_elements(g):
    """A pointer between two elements would fault the kernels: refused before any device is asked for."""
    L = g.load_library()
    n = ctypes.c_longlong()
    for dt, off in ((0, 2), (0, 1), (1, 1)):
        good = [heads(g, 4096) for _ in range(8)]
        for i in range(4):
            hs = list(good[:4])
            hs[i] = heads(g, 4096 + off)
            assert forward(g, attn(g, dtype=dt), *hs) == g.GS_ERR_ALIGNMENT
        for i in range(8):
            hs = list(good)
            hs[i] = heads(g, 4096 + off)
            assert L.gs_cross_attention_backward(ctypes.byref(attn(g, dtype=dt)), *map(ctypes.byref, hs[:4]), 4096,
                                                 *map(ctypes.byref, hs[4:]), None, 0, None) == g.GS_ERR_ALIGNMENT
    for lse in (4097, 4098):
        assert L.gs_cross_attention(ctypes.byref(attn(g)), *map(ctypes.byref, good[:4]), lse, None, 0, None) == g.GS_ERR_ALIGNMENT
    assert L.gs_cross_attention_workspace(ctypes.byref(attn(g, key_lens=4098)), 0, ctypes.byref(n)) == g.GS_ERR_ALIGNMENT
    how = g._Sampling(1.0, 1.0, 0.0, 0)
    for i in range(4):
        p = [4096] * 4
        p[i] += 2
        assert L.gs_sample_scores(p[0], 0, 4, 10, 10, ctypes.byref(how), *p[1:], None) == g.GS_ERR_ALIGNMENT
    assert L.gs_sample_scores(4097, 1, 4, 10, 10, ctypes.byref(how), 4096, 4096, 4096, None) == g.GS_ERR_ALIGNMENT
    for name in ("temperature_rows", "top_p_rows", "min_p_rows", "top_k_rows"):
        how = g._Sampling(1.0, 1.0, 0.0, 0)
        setattr(how, name, 4098)
        assert L.gs_sample_scores(4096, 0, 4, 10, 10, ctypes.byref(how), 4096, 4096, 4096, None) == g.GS_ERR_ALIGNMENT


def test_scale_past_fp32(g):
    """scale * log2(e) has to be an fp32 number, else every logit of 0 would become NaN."""
    assert forward(g, attn(g, scale=3e38)) == g.GS_ERR_INVALID_ARG
    n = ctypes.c_longlong()
    assert g.load_library().gs_cross_attention_workspace(ctypes.byref(attn(g, scale=2.5e38)), 1, ctypes.byref(n)) == g.GS_ERR_INVALID_ARG
    assert forward(g, attn(g, scale=2e38, B=0)) == g.GS_OK
