"""Attention over a sliding window and its gradient through the public calls, against 64 bits."""
import math

import pytest
import torch

from attn_bounds import close
from window_bounds import SeenRef, sees

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def make(B, Lq, Lk, Hq, Hkv, dk, dv, dtype, seed=0, peak=1.5):
    g = torch.Generator().manual_seed(seed * 7919 + B + 31 * Lq + 101 * Lk + Hq + dk)
    t = [torch.randn(s, generator=g) * f for s, f in (((B, Lq, Hq, dk), peak), ((B, Lk, Hkv, dk), 1.0), ((B, Lk, Hkv, dv), 1.0),
                                                      ((B, Lq, Hq, dv), 1.0))]
    return [x.to(DT[dtype]).cuda() for x in t]


def masks(kind, B, Lk, seed=0):
    g = torch.Generator().manual_seed(seed + 5 * B + Lk)
    lens = mask = None
    if kind in ("lens", "both"):
        lens = torch.randint(0, Lk + 1, (B,), generator=g, dtype=torch.int32).cuda()
    if kind in ("holes", "both"):
        mask = (torch.rand(B, Lk, generator=g) < 0.6).cuda()
    return lens, mask


def check(gs, Q, K, V, dO, window, sinks, start, lens=None, mask=None, path="auto", tensor=None, grad=True, **kw):
    B, Lq, Hq, dk = Q.shape
    scale = 1.0 / math.sqrt(dk)
    if tensor is None:
        tensor = Q.dtype == torch.bfloat16 and path != "simt"
    w = 2 ** 40 if window is None else window  # (None: all keys up to a row, however far it stands)
    see = sees(B, Lq, K.shape[1], w, sinks, start, lens, mask)
    r = SeenRef(Q, K, V, scale, see, tensor)
    out = gs.window_attention(Q, K, V, window, sinks, start, scale, key_lens=lens, key_mask=mask, want_lse=True, path=path, **kw)
    gs.stream_status()
    tol, tol_lse = r.forward_tol()
    close(out["O"], r.o.permute(0, 2, 1, 3), tol, "O")
    none = r.lse == -math.inf
    lse = out["lse"].cpu().double()
    assert (lse[none] == -math.inf).all()
    assert (out["O"].cpu().permute(0, 2, 1, 3)[none] == 0).all()
    if K.shape[1]:
        close(lse[~none], r.lse[~none], tol_lse[~none], "lse")
    if not grad:
        return out
    O = r.o.permute(0, 2, 1, 3).to(Q.dtype).cuda()
    got = gs.window_attention_backward(Q, K, V, O, r.lse.float().cuda(), dO, window, sinks, start, scale, key_lens=lens,
                                       key_mask=mask, path=path, **kw)
    gs.stream_status()
    for name, (want, tol) in r.grad(dO).items():
        close(got[name], want, tol, name)
    off = ~r.ok
    assert (got["dK"].cpu()[off] == 0).all() and (got["dV"].cpu()[off] == 0).all()
    return out, got


# B, Lq, Lk, Hq, Hkv, dk, dv, window, sinks, start
SHAPES = [
    (1, 1, 1, 1, 1, 1, 1, 1, 0, 0),
    (2, 130, 130, 4, 2, 64, 64, 17, 0, 0),
    (2, 300, 300, 4, 4, 64, 64, 100, 4, 0),
    (1, 257, 400, 7, 1, 128, 128, 64, 3, 143),      # rows behind a cached prefix; 128 is no multiple of the group
    (3, 33, 64, 2, 2, 10, 5, 8, 20, 31),
    (1, 600, 600, 2, 1, 64, 128, 1, 0, 0),           # every row sees itself alone
    (1, 513, 513, 3, 3, 72, 8, 2, 1, 0),
    (2, 200, 200, 2, 2, 128, 64, 128, 130, 0),       # sinks of more than a tile
    (1, 700, 700, 2, 1, 64, 64, 5000, 0, 0),         # causal
    (2, 1, 900, 8, 2, 64, 64, 300, 4, 899),          # one row
    (2, 3, 900, 4, 2, 128, 128, 513, 1, 897),        # a few rows
    (1, 5, 3000, 2, 1, 40, 40, 2500, 16, 2995),      # a few rows, keys in parts
    (2, 100, 60, 2, 1, 32, 32, 30, 2, 0),            # rows past the last key see what the window leaves of it
    (1, 90, 50, 2, 2, 64, 64, 10, 0, -20),           # rows before the first key
    (1, 1100, 1100, 1, 1, 64, 64, 256, 0, 0),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["none", "lens", "holes", "both"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_cuda_cores(gs, shape, kind, dtype):
    Q, K, V, dO = make(*shape[:7], dtype)
    lens, mask = masks(kind, shape[0], shape[2])
    check(gs, Q, K, V, dO, *shape[7:], lens, mask, "simt")


@pytest.mark.parametrize("path", ["auto", "tensor"])
@pytest.mark.parametrize("kind", ["none", "lens", "holes", "both"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_tensor_cores(gs, shape, kind, path):
    """(Single rows of a narrow width may take CUDA cores: the bounds of rounded weights hold there as well.)"""
    Q, K, V, dO = make(*shape[:7], "bf16")
    lens, mask = masks(kind, shape[0], shape[2])
    check(gs, Q, K, V, dO, *shape[7:], lens, mask, path)


@pytest.mark.parametrize("shape", [(3, 1000, 1000, 8, 2, 128, 128, 200, 4, 0), (40, 300, 300, 16, 4, 64, 64, 77, 1, 0),
                                   (30, 512, 512, 8, 8, 128, 64, 3, 0, 0), (60, 257, 300, 12, 4, 64, 64, 129, 5, 43)],
                         ids=lambda s: "x".join(map(str, s)))
def test_pairs_of_row_tiles(gs, shape):
    """Enough rows for pairs of tiles in a CTA, and for CTAs that go on with another item; the same bits again."""
    Q, K, V, dO = make(*shape[:7], "bf16")
    lens, _ = masks("lens", shape[0], shape[2])
    a = check(gs, Q, K, V, dO, *shape[7:], lens)
    b = gs.window_attention(Q, K, V, *shape[7:], shape[5] ** -0.5, key_lens=lens, want_lse=True)
    assert torch.equal(a[0]["O"], b["O"]) and torch.equal(a[0]["lse"], b["lse"])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(4, 1200, 1200, 8, 8, 32, 24, 20, 5, 0), (2, 1100, 1300, 16, 8, 64, 64, 33, 130, 200),
                                   (1, 2000, 70, 32, 32, 40, 40, 9, 300, 0)], ids=lambda s: "x".join(map(str, s)))
def test_sinks_that_every_row_sees(gs, shape, dtype):
    """The gradients of the first tiles of keys come in parts, those of the others do not; the same bits again."""
    Q, K, V, dO = make(*shape[:7], dtype)
    lens, _ = masks("lens", shape[0], shape[2])
    for n in (None, lens):
        out, got = check(gs, Q, K, V, dO, *shape[7:], n)
        O = out["O"]
        a, b = (gs.window_attention_backward(Q, K, V, O, out["lse"], dO, *shape[7:], key_lens=n) for _ in range(2))
        assert all(torch.equal(a[k], b[k]) for k in a)


@pytest.mark.parametrize("shape", [(2, 300, 300, 4, 4, 64, 64, 60, 3, 0), (3, 120, 120, 8, 1, 128, 64, 2 ** 20, 0, 0),
                                   (1, 700, 700, 4, 2, 72, 40, 20, 0, 0), (1, 1, 250, 64, 1, 128, 128, 100, 130, 249)],
                         ids=lambda s: "x".join(map(str, s)))
def test_rows_of_few_keys_take_no_rounded_output(gs, shape):
    """Through a window of one or two tiles the gradient in bf16 does not go by O, which is rounded."""
    Q, K, V, dO = make(*shape[:7], "bf16")
    lens, mask = masks("both", shape[0], shape[2])
    for n, m in ((None, None), (lens, None), (None, mask)):
        out, got = check(gs, Q, K, V, dO, *shape[7:], n, m, "tensor")
        other = gs.window_attention_backward(Q, K, V, torch.zeros_like(out["O"]), out["lse"], dO, *shape[7:], key_lens=n, key_mask=m,
                                             path="tensor")
        same = gs.window_attention_backward(Q, K, V, out["O"], out["lse"], dO, *shape[7:], key_lens=n, key_mask=m, path="tensor")
        assert all(torch.equal(other[k], same[k]) for k in same)


@pytest.mark.parametrize("path", ["auto", "simt"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_row_of_one_key_has_no_gradient_but_its_value_s(gs, dtype, path):
    """Its weight is 1 whatever its logit: dQ and dK are 0, not a rounding's rest, also beside rows of more keys."""
    for Lq, window, sinks, start, n in ((400, 1, 0, 0, None), (300, 1, 0, 200, (1, 500)), (3, 5, 2, 0, (1, 1)), (200, 1000, 4, 0, (1, 1))):
        Q, K, V, dO = make(2, Lq, 500, 4, 2, 64, 64, dtype)
        lens = torch.tensor(n, dtype=torch.int32).cuda() if n else None
        out, got = check(gs, Q, K, V, dO, window, sinks, start, lens, path=path)
        assert (got["dQ"] == 0).all() and (got["dK"] == 0).all() and (got["dV"] != 0).any()
    Q, K, V, dO = make(2, 300, 300, 4, 2, 64, 64, dtype)
    out, got = check(gs, Q, K, V, dO, 150, 2, 0, path=path)
    assert (got["dQ"][:, 0] == 0).all() and (got["dQ"][:, 1] != 0).any()


@pytest.mark.parametrize("path", ["auto", "simt"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_starts_of_their_own(gs, dtype, path):
    Q, K, V, dO = make(5, 140, 400, 4, 2, 64, 64, dtype)
    start = torch.tensor([0, 260, -7, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32).cuda()
    check(gs, Q, K, V, dO, 50, 3, start, path=path)
    lens = torch.tensor([400, 300, 0, 9, 400], dtype=torch.int32).cuda()
    check(gs, Q, K, V, dO, 50, 3, start, lens, path=path)
    check(gs, Q, K, V, dO, None, 0, start, path=path)
    check(gs, Q, K, V, dO, 2 ** 31 - 1, 2 ** 31 - 1, start, path=path)


@pytest.mark.parametrize("path", ["auto", "simt"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Lq", [1, 3, 200])
def test_what_a_row_does_not_see_may_hold_anything(gs, dtype, path, Lq):
    """Keys and values from some position on, and one between the sinks and the window, are not finite: rows that do not see
    them are as if they were zero."""
    Lk, start = 400, 200
    for bad in (math.nan, math.inf, -torch.finfo(DT[dtype]).max):
        Q, K, V, dO = make(2, Lq, Lk, 4, 2, 64, 64, dtype)
        ref = gs.window_attention(Q, K, V, 90, 3, start, path=path, want_lse=True)
        x = start + Lq // 2 + 1
        K[:, x:], V[:, x:] = bad, bad
        K[:, 50], V[:, 50] = bad, bad
        out = gs.window_attention(Q, K, V, 90, 3, start, path=path, want_lse=True)
        gs.stream_status()
        n = x - start
        if path == "auto" and dtype == "bf16":  # (the tensor cores' rows are taken again, in fp32: other roundings of the weights)
            Q, K, V, dO = make(2, Lq, Lk, 4, 2, 64, 64, dtype)
            r = SeenRef(Q, K, V, 1 / 8, sees(2, Lq, Lk, 90, 3, start), True)
            close(out["O"][:, :n], r.o.permute(0, 2, 1, 3)[:, :n], r.forward_tol()[0][:, :n], "O")
        else:
            assert torch.equal(out["O"][:, :n], ref["O"][:, :n])
        assert torch.equal(out["lse"][:, :, :n], ref["lse"][:, :, :n])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_keys_that_no_row_sees_may_hold_anything(gs, dtype):
    for path in ("auto", "simt"):
        Q, K, V, dO = make(2, 200, 400, 4, 2, 64, 64, dtype)
        lens = torch.tensor([390, 150], dtype=torch.int32).cuda()
        mask = torch.ones(2, 400, dtype=torch.bool).cuda()
        mask[:, 120:130] = False
        for t in (K, V):
            t[0, 390:], t[1, 150:] = math.nan, math.inf
            t[:, 120:130] = math.nan
            t[:, 4:30] = math.inf  # between the sinks and the windows (the first row's from 31 on)
            t[:, 300:] = math.nan  # behind the last row
        K0, V0 = K.clone(), V.clone()
        dead = ~torch.isfinite(K0[:, :, :1, :1].float()).expand(K.shape)
        K0[dead], V0[dead] = 0, 0
        a = check(gs, Q, K, V, dO, 70, 4, 100, lens, mask, path)
        b = check(gs, Q, K0, V0, dO, 70, 4, 100, lens, mask, path)
        assert all(torch.equal(a[1][k], b[1][k]) for k in a[1])


@pytest.mark.parametrize("path", ["auto", "simt"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_an_infinite_value_goes_to_the_rows_that_see_it(gs, dtype, path):
    """In its column and nowhere else, also where its tile holds rows of both kinds (and where all rows of most tiles see it)."""
    for window, sinks, j in ((None, 0, 5), (100, 2, 300), (1, 6, 4), (40, 0, 511)):
        Q, K, V, _ = make(2, 700, 700, 8, 2, 64, 72, dtype)
        V[1, j, 1, 70] = math.inf
        O = gs.window_attention(Q, K, V, window, sinks, path=path)["O"].float().cpu()
        gs.stream_status()
        see = sees(1, 700, 700, window or 2 ** 40, sinks, 0)[0, :, j]
        hit = torch.zeros(2, 700, 8, 72, dtype=torch.bool)
        hit[1, :, 4:, 70] = see[:, None]
        assert (O[hit] == math.inf).all() and torch.isfinite(O[~hit]).all()


def test_gradient_against_differences(gs):
    Q, K, V, dO = make(1, 40, 60, 2, 1, 24, 16, "f32")
    args = (13, 2, 20)
    out = gs.window_attention(Q, K, V, *args, want_lse=True)
    got = gs.window_attention_backward(Q, K, V, out["O"], out["lse"], dO, *args)
    see = sees(1, 40, 60, *args)

    def loss(q, k, v):
        return float((SeenRef(q, k, v, 24 ** -0.5, see).o.permute(0, 2, 1, 3) * dO.cpu().double()).sum())

    g = torch.Generator().manual_seed(1)
    for name, i in (("dQ", 0), ("dK", 1), ("dV", 2)):
        t = [x.cpu().double() for x in (Q, K, V)]
        d = torch.randn(t[i].shape, generator=g, dtype=torch.float64)
        h = 1e-5
        up, down = list(t), list(t)
        up[i], down[i] = t[i] + h * d, t[i] - h * d
        want = (loss(*up) - loss(*down)) / (2 * h)
        have = float((got[name].cpu().double() * d).sum())
        # central differences are off by O(h^2), the fp32 gradient by 2^-24 times some hundred terms
        assert abs(want - have) <= 2e-5 * float((got[name].cpu().double().abs() * d.abs()).sum()), (name, want, have)


def test_a_window_of_everything_is_cross_attention(gs):
    """Rows behind the last key with a window over all keys see them all."""
    for dtype in ("f32", "bf16"):
        Q, K, V, dO = make(2, 100, 150, 4, 2, 64, 64, dtype)
        a = gs.window_attention(Q, K, V, None, 0, 150, want_lse=True, path="simt")
        b = gs.cross_attention(Q, K, V, want_lse=True, path="simt")
        assert torch.equal(a["O"], b["O"]) and torch.equal(a["lse"], b["lse"])


def test_empty(gs):
    for shape in ((0, 3, 4), (2, 0, 4), (2, 3, 0)):
        Q, K, V, dO = make(*shape, 2, 1, 8, 8, "f32")
        out = gs.window_attention(Q, K, V, 5, want_lse=True)
        assert (out["O"] == 0).all() and (out["lse"] == -math.inf).all()
        got = gs.window_attention_backward(Q, K, V, out["O"], out["lse"], dO, 5)
        assert all((t == 0).all() for t in got.values())
    gs.stream_status()
