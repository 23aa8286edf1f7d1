"""Cross attention and its gradient through the public calls, against 64 bits."""
import math

import pytest
import torch

from attn_bounds import Ref, close

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


def check_forward(gs, Q, K, V, scale, lens, mask, path, tensor, **kw):
    r = Ref(Q, K, V, scale, lens, mask, tensor)
    out = gs.cross_attention(Q, K, V, scale, key_lens=lens, key_mask=mask, want_lse=True, path=path, **kw)
    gs.stream_status()
    tol, tol_lse = r.forward_tol()
    close(out["O"], r.o.permute(0, 2, 1, 3), tol, "O")
    none = r.lse == -math.inf
    lse = out["lse"].cpu().double()
    assert (lse[none] == -math.inf).all()
    assert (out["O"].cpu().permute(0, 2, 1, 3)[none] == 0).all()
    close(lse[~none], r.lse[~none], tol_lse[~none] if torch.is_tensor(tol_lse) else tol_lse, "lse")
    return r, out


def check_grad(gs, Q, K, V, dO, scale, lens, mask, path, tensor, **kw):
    r = Ref(Q, K, V, scale, lens, mask, tensor)
    O = r.o.permute(0, 2, 1, 3).to(Q.dtype).cuda()
    lse = r.lse.float().cuda()
    got = gs.cross_attention_backward(Q, K, V, O, lse, dO, scale, key_lens=lens, key_mask=mask, path=path, **kw)
    gs.stream_status()
    for name, (want, tol) in r.grad(dO).items():
        close(got[name], want, tol, name)
    off = ~r.ok
    assert (got["dK"].cpu()[off] == 0).all() and (got["dV"].cpu()[off] == 0).all()
    return got


# B, Lq, Lk, Hq, Hkv, dk, dv
SHAPES = [
    (1, 1, 1, 1, 1, 1, 1),
    (2, 1, 197, 4, 4, 64, 64),
    (1, 3, 65, 2, 1, 40, 30),
    (2, 70, 129, 4, 2, 64, 128),
    (1, 130, 300, 7, 1, 128, 128),
    (3, 33, 64, 2, 2, 10, 5),
    (1, 1, 3000, 8, 2, 128, 64),
    (2, 257, 127, 6, 3, 72, 8),
    (1, 40, 2500, 2, 1, 64, 128),        # more rows than a few, keys in parts
    (3, 9, 700, 3, 1, 33, 20),           # a few rows, in chunks of four
    (2, 1, 9000, 1, 1, 24, 100),         # one row, keys in parts
    (1, 1, 500, 4, 4, 128, 128),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["none", "lens", "holes", "both"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_cuda_cores(gs, shape, kind, dtype):
    Q, K, V, dO = make(*shape, dtype)
    lens, mask = masks(kind, shape[0], shape[2])
    scale = 1.0 / math.sqrt(shape[5])
    check_forward(gs, Q, K, V, scale, lens, mask, "simt", False)
    check_grad(gs, Q, K, V, dO, scale, lens, mask, "simt", False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_invalid_keys_may_hold_anything(gs, dtype):
    """NaN, infinities and the type's lowest value in keys and values that are not read, for every path."""
    Q, K, V, dO = make(3, 40, 300, 4, 2, 64, 64, dtype)
    lens = torch.tensor([300, 131, 0], dtype=torch.int32).cuda()
    mask = torch.ones(3, 300, dtype=torch.bool)
    mask[0, 5:9] = False
    mask[0, 128:256] = False
    mask[1, 130] = False
    mask = mask.cuda()
    bad = torch.tensor([math.nan, math.inf, -math.inf, torch.finfo(DT[dtype]).min], dtype=DT[dtype]).cuda()
    ok = mask & (torch.arange(300).cuda()[None] < lens[:, None])
    for t in (K, V):
        n = int((~ok).sum())
        t[~ok] = bad[torch.arange(n).cuda() % 4][:, None, None].expand(n, 2, 64)
    for path in ("simt", "auto"):
        check_forward(gs, Q, K, V, 0.125, lens, mask, path, dtype == "bf16" and path == "auto")
        check_grad(gs, Q, K, V, dO, 0.125, lens, mask, path, dtype == "bf16" and path == "auto")


@pytest.mark.parametrize("path", ["simt", "auto"])
def test_lengths_outside_and_no_keys(gs, path):
    for dtype in ("f32", "bf16"):
        Q, K, V, dO = make(2, 9, 70, 2, 2, 64, 64, dtype)
        lens = torch.tensor([-5, 99], dtype=torch.int32).cuda()
        check_forward(gs, Q, K, V, 0.2, lens, None, path, dtype == "bf16")
        check_grad(gs, Q, K, V, dO, 0.2, lens, None, path, dtype == "bf16")
        out = gs.cross_attention(Q, K[:, :0], V[:, :0], 0.2, want_lse=True, path=path)
        assert (out["O"] == 0).all() and (out["lse"] == -math.inf).all()
        g = gs.cross_attention_backward(Q, K[:, :0], V[:, :0], out["O"], out["lse"], dO, 0.2, path=path)
        assert (g["dQ"] == 0).all() and g["dK"].shape[1] == 0
        g = gs.cross_attention_backward(Q[:, :0], K, V, out["O"][:, :0], out["lse"][:, :, :0].contiguous(), dO[:, :0], 0.2,
                                        path=path)
        assert (g["dK"] == 0).all() and (g["dV"] == 0).all()
        gs.stream_status()


@pytest.mark.parametrize("path", ["simt", "auto"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_not_finite_logits(gs, dtype, path):
    """A NaN or +inf logit makes its row NaN and no other; -inf logits weigh nothing; a row of them counts as empty."""
    Q, K, V, _ = make(1, 5, 150, 1, 1, 64, 64, dtype)
    K[0, 7, 0, 0], Q[0, :, 0, 0] = math.inf, 0.0
    Q[0, 1, 0, 0], Q[0, 2, 0, 0], Q[0, 3, 0, 0] = 1.0, -1.0, math.nan  # logit 7: +inf, -inf, NaN (0 inf: NaN in rows 0, 4)
    K2 = K.clone()
    K2[0, 7, 0, 0] = 0.0
    out = gs.cross_attention(Q, K, V, 0.125, want_lse=True, path=path)
    gs.stream_status()
    o, lse = out["O"][0, :, 0].float().cpu(), out["lse"][0, 0].cpu()
    for i in (0, 1, 3, 4):
        assert torch.isnan(o[i]).all() and torch.isnan(lse[i])
    mask = torch.ones(1, 150, dtype=torch.bool)
    mask[0, 7] = False
    r = Ref(Q[:, 2:3], K2, V, 0.125, None, mask.cuda(), dtype == "bf16" and path == "auto")
    tol, _ = r.forward_tol()
    close(out["O"][:, 2:3], r.o.permute(0, 2, 1, 3), tol, "O beside a logit of -inf")
    # every valid logit -inf
    K[0, :, 0, 0] = math.inf
    out = gs.cross_attention(Q[:, 2:3], K, V, 0.125, want_lse=True, path=path)
    assert (out["O"] == 0).all() and (out["lse"] == -math.inf).all()


def strided(t, how):
    """The same values in another layout."""
    B, L, H, w = t.shape
    if how == "heads first":
        return t.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)
    if how == "sliced":
        big = torch.full((B, L + 3, H + 1, w + 8), math.nan, dtype=t.dtype, device=t.device)
        big[:, 2:L + 2, 1:, 8:] = t
        return big[:, 2:L + 2, 1:, 8:]
    if how == "unaligned":
        big = torch.full((B, L, H, w + 3), math.nan, dtype=t.dtype, device=t.device)
        big[..., 1:w + 1] = t
        return big[..., 1:w + 1]
    return t.permute(1, 0, 2, 3).contiguous().permute(1, 0, 2, 3)  # length first


@pytest.mark.parametrize("path", ["simt", "auto"])
@pytest.mark.parametrize("how", ["heads first", "length first", "sliced", "unaligned"])
def test_strides(gs, how, path):
    for dtype in ("f32", "bf16"):
        Q, K, V, dO = make(2, 37, 140, 4, 2, 64, 64, dtype)
        lens, _ = masks("lens", 2, 140)
        tensor = dtype == "bf16" and path == "auto"
        a = [strided(t, how) for t in (Q, K, V, dO)]
        outs = {"O": strided(torch.zeros_like(Q), how)}
        _, out = check_forward(gs, a[0], a[1], a[2], 0.125, lens, None, path, tensor, out=outs)
        g = {n: strided(torch.zeros_like(t), how) for n, t in (("dQ", Q), ("dK", K), ("dV", V))}
        check_grad(gs, a[0], a[1], a[2], a[3], 0.125, lens, None, path, tensor, out=g)
        if how == "sliced":  # what lies around the outputs stays as it was
            for t in (outs["O"], g["dQ"], g["dK"], g["dV"]):
                base = t._base if t._base is not None else t
                assert torch.isnan(base[:, :2]).all() and torch.isnan(base[:, :, 0]).all() and torch.isnan(base[..., :8]).all()


@pytest.mark.parametrize("path", ["simt", "auto"])
def test_states_shared_by_all_sequences(gs, path):
    """K and V expanded over the batch (stride 0): gradients come one per sequence."""
    for dtype in ("f32", "bf16"):
        Q, K, V, dO = make(3, 20, 90, 4, 2, 64, 64, dtype)
        K, V = K[:1].expand(3, -1, -1, -1), V[:1].expand(3, -1, -1, -1)
        mask = (torch.rand(1, 90, generator=torch.Generator().manual_seed(1)) < 0.7).cuda().expand(3, -1)
        tensor = dtype == "bf16" and path == "auto"
        check_forward(gs, Q, K, V, 0.125, None, mask, path, tensor)
        check_grad(gs, Q, K, V, dO, 0.125, None, mask, path, tensor)


@pytest.mark.parametrize("path", ["simt", "auto"])
def test_offsets_beyond_32_bits(gs, path):
    """Sequences more than 2^32 bytes apart."""
    Q, K, V, _ = make(2, 2, 77, 2, 1, 64, 64, "bf16")
    gap = (1 << 31) + 64
    buf = torch.empty(gap + 2 * 77 * 64, dtype=torch.bfloat16, device="cuda")
    far = [buf[o:].as_strided((2, 77, 1, 64), (gap, 64, 64, 1)) for o in (0, 77 * 64)]
    far[0].copy_(K)
    far[1].copy_(V)
    check_forward(gs, Q, far[0], far[1], 0.125, None, None, path, path == "auto")


@pytest.mark.parametrize("path", ["simt", "auto"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradient_against_differences(gs, dtype, path):
    """<dX, E> against the change of <dO, O> along a random direction E, in 64 bits on the formula's side only
    for the step: the calls' own forward results are too coarse to be differenced."""
    Q, K, V, dO = make(1, 12, 50, 2, 1, 64, 64, dtype)
    mask = masks("holes", 1, 50)[1]
    out = gs.cross_attention(Q, K, V, 0.125, key_mask=mask, want_lse=True, path=path)
    got = gs.cross_attention_backward(Q, K, V, out["O"], out["lse"], dO, 0.125, key_mask=mask, path=path)
    f = lambda q, k, v: float((Ref(q, k, v, 0.125, None, mask).o.permute(0, 2, 1, 3) * dO.cpu().double()).sum())  # noqa: E731
    g = torch.Generator().manual_seed(3)
    base = [t.cpu().double() for t in (Q, K, V)]
    r = Ref(Q, K, V, 0.125, None, mask, dtype == "bf16" and path == "auto")
    tols = r.grad(dO)
    for i, name in enumerate(("dQ", "dK", "dV")):
        E = torch.randn(base[i].shape, generator=g, dtype=torch.float64)
        eps = 1e-5
        up, down = list(base), list(base)
        up[i], down[i] = base[i] + eps * E, base[i] - eps * E
        want = (f(*up) - f(*down)) / (2 * eps)
        have = float((got[name].cpu().double() * E).sum())
        # the elements' errors are independent of E: 7 standard deviations of their sum, and the difference quotient's own error
        tol = 7 * float((tols[name][1] * E).square().sum().sqrt()) + 1e-6 * abs(want) + 1e-6
        assert abs(have - want) <= tol, (name, have, want, tol)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_repeats_bit_for_bit(gs, dtype):
    Q, K, V, dO = make(2, 1, 5000, 4, 2, 64, 64, dtype)
    lens = torch.tensor([5000, 2100], dtype=torch.int32).cuda()
    a = gs.cross_attention(Q, K, V, key_lens=lens, want_lse=True)
    ga = gs.cross_attention_backward(Q, K, V, a["O"], a["lse"], dO, key_lens=lens)
    for _ in range(5):
        b = gs.cross_attention(Q, K, V, key_lens=lens, want_lse=True)
        gb = gs.cross_attention_backward(Q, K, V, a["O"], a["lse"], dO, key_lens=lens)
        assert all(torch.equal(a[k], b[k]) for k in a) and all(torch.equal(ga[k], gb[k]) for k in ga)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_side_stream_and_graphs(gs, dtype):
    """Another stream than the current one; two captured graphs, replayed in turn and at once on new inputs."""
    Q, K, V, dO = make(2, 3, 2500, 4, 2, 64, 64, dtype)
    want = gs.cross_attention(Q, K, V, want_lse=True)
    gwant = gs.cross_attention_backward(Q, K, V, want["O"], want["lse"], dO)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    out = gs.cross_attention(Q, K, V, want_lse=True, stream=side)
    g = gs.cross_attention_backward(Q, K, V, out["O"], out["lse"], dO, stream=side)
    side.synchronize()
    assert torch.equal(out["O"], want["O"]) and all(torch.equal(g[k], gwant[k]) for k in g)
    graphs = []
    for seed in (1, 2):
        t = [torch.empty_like(x) for x in (Q, K, V, dO)]
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            o = gs.cross_attention(t[0], t[1], t[2], want_lse=True)
            gg = gs.cross_attention_backward(t[0], t[1], t[2], o["O"], o["lse"], t[3])
        graphs.append((gr, t, o, gg, seed))
    for gr, t, o, gg, seed in graphs:
        for x, y in zip(t, make(2, 3, 2500, 4, 2, 64, 64, dtype, seed=seed)):
            x.copy_(y)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        for s, (gr, *_r) in zip(streams, graphs):
            with torch.cuda.stream(s):
                gr.replay()
    torch.cuda.synchronize()
    for gr, t, o, gg, seed in graphs:
        w = gs.cross_attention(t[0], t[1], t[2], want_lse=True)
        gw = gs.cross_attention_backward(t[0], t[1], t[2], w["O"], w["lse"], t[3])
        assert torch.equal(o["O"], w["O"]) and torch.equal(o["lse"], w["lse"])
        assert all(torch.equal(gg[k], gw[k]) for k in gg)
    gs.stream_status()


def test_decoding_step_end_to_end(gs):
    """Attention over a problem's context in coefficient space, its scores against the codebook, a draw."""
    g = torch.Generator().manual_seed(11)
    M, D, B, L = 40, 512, 6, 90
    C = (torch.randint(0, 2, (M, D), generator=g) * 2 - 1).float().cuda()
    b = gs.build_basis(C)
    P = torch.softmax(2 * torch.randn(B * L, M, generator=g), dim=1).cuda()
    ctx = gs.prob_vectorize(b, P).view(B, L, 1, b.r)
    lens = torch.randint(1, L + 1, (B,), generator=g, dtype=torch.int32).cuda()
    q = b.R[torch.randint(0, M, (B,), generator=g).cuda()].view(B, 1, 1, b.r).contiguous()
    o = gs.cross_attention(q, ctx, ctx, 1.0 / D, key_lens=lens)["O"]
    s = gs.similarity_coeffs(b, o.view(B, b.r), scale=8.0 / D, want_S=True)["S"]
    u = torch.rand(B, generator=g).cuda()
    d = gs.sample_scores(s, u, temperature=0.5, top_k=10)
    # in 64 bits, from the codebook itself
    Cd, Pd = C.cpu().double(), P.cpu().double().view(B, L, M)
    Rq = q.cpu().double().view(B, -1) @ b.Q.cpu().double()
    for i in range(B):
        X = Pd[i, :int(lens[i])] @ Cd
        w = torch.softmax(X @ Rq[i] / D, 0)
        sc = Cd @ (w @ X) * (8.0 / D)
        assert (s[i].cpu().double() - sc).abs().max() <= 1e-3
        v, idx = torch.sort(sc, descending=True)
        p = torch.zeros(M, dtype=torch.float64)
        p[idx[:10]] = torch.softmax(v[:10] / 0.5, 0)
        run = p.cumsum(0)
        j = int(d["index"][i])
        # a score off by 1e-3 moves a weight by 2e-3 of itself at this temperature: so far the borders may lie apart
        assert run[j] - p[j] - 5e-3 <= float(u[i]) <= run[j] + 5e-3


TENSOR_SHAPES = [
    (1, 1, 1, 1, 1, 8, 8),
    (1, 1, 128, 8, 8, 64, 64),
    (2, 1, 5000, 8, 2, 128, 64),
    (1, 5, 40000, 4, 1, 64, 128),        # keys in parts
    (1, 130, 1100, 1, 1, 72, 40),
    (3, 260, 517, 8, 2, 128, 128),
    (2, 3, 700, 128, 1, 64, 64),         # 128 query heads on one key head
    (4, 600, 300, 16, 16, 64, 64),       # pairs of row tiles
    (20, 129, 129, 8, 8, 40, 72),        # pairs, the second tile one row
    (8, 300, 200, 28, 4, 128, 128),      # pairs, groups of seven: 126 rows a tile
    (40, 128, 257, 4, 4, 128, 64),
]


@pytest.mark.parametrize("kind", ["none", "lens", "holes", "both"])
@pytest.mark.parametrize("shape", TENSOR_SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_tensor_cores(gs, shape, kind):
    Q, K, V, dO = make(*shape, "bf16")
    lens, mask = masks(kind, shape[0], shape[2])
    check_forward(gs, Q, K, V, 1.0 / math.sqrt(shape[5]), lens, mask, "tensor", True)


BACKWARD_SHAPES = TENSOR_SHAPES + [
    (1, 3000, 100, 2, 1, 64, 64),        # rows in parts
    (1, 700, 900, 2, 2, 128, 64),        # both in parts
    (2, 1, 300, 7, 1, 64, 128),
]


@pytest.mark.parametrize("kind", ["none", "lens", "holes", "both"])
@pytest.mark.parametrize("shape", BACKWARD_SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_tensor_cores_backward(gs, shape, kind):
    Q, K, V, dO = make(*shape, "bf16")
    lens, mask = masks(kind, shape[0], shape[2])
    check_grad(gs, Q, K, V, dO, 1.0 / math.sqrt(shape[5]), lens, mask, "tensor", True)


def test_growing_maxima(gs):
    """Keys whose logits grow along the sequence by far more than the running maximum lags, and fall again."""
    for B, H in ((1, 2), (16, 16)):
        Q, K, V, dO = make(B, 200, 1000, H, H, 64, 64, "bf16", peak=1.0)
        up = torch.cat([torch.linspace(0, 12, 700), torch.linspace(12, -12, 300)]).cuda()
        K[..., 0] = up[None, :, None].bfloat16()
        Q[..., 0] = (torch.arange(200) % 7 - 3).cuda()[None, :, None].bfloat16() * 4
        check_forward(gs, Q, K, V, 0.5, None, None, "tensor", True)


@pytest.mark.parametrize("path", ["simt", "auto"])
@pytest.mark.parametrize("Lk", [1, 2, 3, 8, 40, 64, 100, 128])
def test_gradient_over_few_keys(gs, Lk, path):
    """With few keys dP - D cancels: dS rounded to bf16 (the tensor cores) or not at all (CUDA cores) and the outputs'
    rounding are what may be off, not a bf16 O's 2^-9 of <dO, O>.  In the 2-norm over thousands of independent
    roundings of at most h, whose mean square is h^2 / 3 or less (1.2 of room for their spread)."""
    Q, K, V, dO = make(6, 50, Lk, 4, 2, 64, 64, "bf16")
    r = Ref(Q, K, V, 0.125)
    O, lse = r.o.permute(0, 2, 1, 3).bfloat16().cuda(), r.lse.float().cuda()
    got = gs.cross_attention_backward(Q, K, V, O, lse, dO, 0.125, path=path)
    gs.stream_status()
    n = 2 if path == "auto" else 1
    for name, (want, _) in r.grad(dO).items():
        off = (got[name].cpu().double() - want).norm()
        if Lk == 1 and name != "dV":  # P = 1: dS = 0, whatever fp32 leaves of it
            assert off <= 1e-5 * dO.float().norm().cpu() * 64
            continue
        assert off <= 1.2 * (n / 3) ** 0.5 * 2.0 ** -8 * want.norm(), (name, float(off / want.norm()))
