"""verify_drafts against the definition in whole numbers on the CPU."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def units(row):
    """rint(p 2^44) of each entry, as the definition has them."""
    p = np.nan_to_num(row.astype(np.float64), nan=0.0, posinf=1.0, neginf=0.0).clip(0.0, 1.0)
    return np.rint(p * 2.0 ** 44).astype(np.int64)


def unit(u):
    u = np.float32(u)
    return float(min(max(u, np.float32(0)), np.nextafter(np.float32(1), np.float32(0)))) if u == u else 0.0


def reference(P, D, x, U, n):
    K = len(x)
    n = min(max(n, 0), K)
    M = P.shape[1]
    a = 0
    while a < n and 0 <= x[a] < M:
        d = float(D[a, x[a]]) if D is not None else 1.0
        if not unit(U[a]) * d < float(P[a, x[a]]):
            break
        a += 1
    w = units(P[a])
    if a < n:
        if D is not None:
            rest = np.maximum(w - units(D[a]), 0)
        else:
            rest = w.copy()
            if 0 <= x[a] < M:
                rest[x[a]] = 0
        w = rest if rest.any() else w
    total = int(w.sum())
    if total == 0:
        drawn = -1
    else:
        # U total as a fraction: an fp32 number has a power of two below it
        u = unit(U[K])
        t = int(np.float64(u) * 2.0 ** 64) * total >> 64
        drawn = int(np.searchsorted(np.cumsum(w), t, side="right"))
    return a, list(x[:a]) + [drawn] + [-1] * (K - a)


def check(gs, P, D, x, U, n=None, **kw):
    out = gs.verify_drafts(P, D, x, U, draft_lens=n, **kw)
    gs.stream_status()
    p, d = P.float().cpu().numpy(), D.float().cpu().numpy() if D is not None else None
    B, K = x.shape
    for b in range(B):
        a, t = reference(p[b], d[b] if d is not None else None, x[b].tolist(), U[b].cpu().numpy(), int(n[b]) if n is not None else K)
        assert int(out["accepted"][b]) == a, b
        assert out["tokens"][b].tolist() == t, b
    return out


def make(B, K, M, dtype, seed=0, near=0.5):
    g = torch.Generator().manual_seed(seed + B + 7 * K + M)
    z = 2 * torch.randn(B, K + 1, M, generator=g)
    P = torch.softmax(z, dim=2).to(DT[dtype])
    D = torch.softmax(z[:, :K] + near * torch.randn(B, K, M, generator=g), dim=2)
    x = torch.multinomial(D.view(B * K, M).clamp(min=1e-30), 1, generator=g).view(B, K).int() if K else torch.zeros(B, 0).int()
    U = torch.rand(B, K + 1, generator=g)
    n = torch.randint(-1, K + 2, (B,), generator=g, dtype=torch.int32)
    return P.cuda(), D.to(DT[dtype]).cuda(), x.cuda(), U.cuda(), n.cuda()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,K,M", [(3, 1, 1), (5, 2, 7), (40, 4, 100), (7, 0, 33), (9, 5, 4099), (6, 3, 32000), (300, 2, 2048), (2, 40, 515),
                                   (3, 2, 131071), (1, 1, 524288)])
def test_draws(gs, B, K, M, dtype):
    P, D, x, U, n = make(B, K, M, dtype)
    check(gs, P, D, x, U)
    check(gs, P, D, x, U, n)
    check(gs, P, None, x, U, n)


def test_many_draws_are_the_targets(gs):
    """Over 200,000 drafts the tokens that come out are distributed as the target has them: each of 8 counts lies within 6 standard
    deviations (probability of a false alarm below 8 * 2e-9)."""
    g = torch.Generator().manual_seed(2)
    N = 200000
    p = torch.tensor([0.3, 0.05, 0.1, 0.2, 0.05, 0.02, 0.25, 0.03])
    d = torch.tensor([0.1, 0.3, 0.1, 0.1, 0.1, 0.1, 0.1, 0.1])
    x = torch.multinomial(d, N, replacement=True, generator=g).view(N, 1).int()
    P, D = p.cuda().expand(N, 2, 8), d.cuda().expand(N, 1, 8)  # rows that share memory
    out = gs.verify_drafts(P, D, x.cuda(), torch.rand(N, 2, generator=g).cuda())
    gs.stream_status()
    counts = torch.bincount(out["tokens"][:, 0].cpu(), minlength=8).double()
    want = p.double() / p.double().sum() * N
    assert ((counts - want).abs() <= 6 * (want * (1 - p.double())).sqrt()).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strides_and_alignment(gs, dtype):
    P, D, x, U, n = make(6, 3, 1000, dtype)
    big = torch.zeros(6, 4, 1013, dtype=P.dtype, device="cuda")
    for off in (0, 1, 5, 8):
        p, d = big[:, :, off:off + 1000], big.clone()[:, :3, off + 3:off + 1003]
        p.copy_(P)
        d.copy_(D)
        check(gs, p, d, x, U, n)
        check(gs, p, None, x, U, n)
    check(gs, P.transpose(0, 1).contiguous().transpose(0, 1), D, x, U, n)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_that_are_no_distributions(gs, dtype):
    """NaN, infinities, negative entries and entries above 1; the same row for both; nothing at all."""
    M, K = 3005, 2
    P, D, x, U, _ = make(8, K, M, dtype)
    P[0] = 0
    P[1, :, ::2], D[1, :, 1::3] = float("nan"), float("nan")
    P[2, :, 17], D[2, :, 18] = float("inf"), float("inf")
    P[3] = -P[3]
    P[4, :, 5:9] = 7.0
    D[5] = P[5, :K]                    # nothing is left: the target's row is drawn from
    U[5] = 0.999
    x[6] = torch.tensor([M, -1])       # no entries
    x[7] = torch.tensor([2 ** 31 - 1, -2 ** 31], dtype=torch.int64).int()
    check(gs, P, D, x, U)
    check(gs, P, None, x, U)
    for bad in (-1.0, float("nan"), 1.0, 5.0, 0.0, 1e-38, 1 - 2.0 ** -24):
        check(gs, P, D, x, torch.full_like(U, bad))


def test_single_outputs(gs):
    P, D, x, U, n = make(4, 2, 50, "f32")
    want = gs.verify_drafts(P, D, x, U)
    for drop, keep in (("tokens", "accepted"), ("accepted", "tokens")):
        out = gs.verify_drafts(P, D, x, U, out={drop: None})
        assert out[drop] is None and torch.equal(out[keep], want[keep])


def test_same_bits_in_a_graph_and_on_a_stream(gs):
    P, D, x, U, n = make(5, 3, 32000, "bf16")
    want = gs.verify_drafts(P, D, x, U, n)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = gs.verify_drafts(P, D, x, U, n, stream=s)
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        rec = gs.verify_drafts(P, D, x, U, n)
    g.replay()
    torch.cuda.synchronize()
    for k in want:
        assert torch.equal(want[k], got[k]) and torch.equal(want[k], rec[k])
