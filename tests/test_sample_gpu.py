"""sample_scores against the definition in extended precision on the CPU."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def reference(s, u, T, k, p, mp):
    """(the indices that exact arithmetic may draw, {index: probability}): two where u ends within 2^-35 of the kept
    weight from a border (weights exact to a relative e = 2^-34 move a share p by at most 2 p (1 - p) e <= 2^-35)."""
    s = np.asarray(s, dtype=np.longdouble)
    M = s.size
    live = ~np.isnan(s) & (s != -np.inf)
    if not live.any():
        return {-1}, {-1: 0.0}
    top = s[live].max()
    if not T > 0:
        i = int(np.nonzero(live & (s == top))[0][0])
        return {i}, {i: 1.0}
    w = np.zeros(M, dtype=np.longdouble)
    if np.isinf(top):
        w[live & (s == top)] = 1
    else:
        w[live] = np.exp((s[live] - top) / np.longdouble(np.float32(T)))
    order = np.argsort(np.where(live, -s, np.inf), kind="stable")
    keep = np.zeros(M, dtype=bool)
    n = int(live.sum())
    if 1 <= k < M:
        n = min(n, k)
    run = np.cumsum(w[order[:n]])
    if p < 1:
        need = np.longdouble(np.float32(max(p, 0))) * run[-1]
        n = min(n, max(1, 1 + int((run < need).sum())))
    keep[order[:n]] = True
    if mp > 0:
        keep &= (w >= np.longdouble(np.float32(min(mp, 1)))) | (w == 1)
    w[~keep] = 0
    run = np.cumsum(w)
    u = np.float32(u)
    u = min(max(u, np.float32(0)), np.nextafter(np.float32(1), np.float32(0))) if u == u else np.float32(0)
    t = np.longdouble(u) * run[-1]
    near = run[-1] * np.longdouble(2.0) ** -35
    cand = {int(np.searchsorted(run, x, side="right")) for x in (max(t - near, 0), t, min(t + near, run[-1] * (1 - 1e-15)))}
    if u == 0:
        cand = {int(np.nonzero(w)[0][0])}
    return cand, {i: float(w[i] / run[-1]) for i in cand}


def check(gs, S, U, T=1.0, k=0, p=1.0, mp=0.0, **kw):
    out = gs.sample_scores(S, U, temperature=T, top_k=k, top_p=p, min_p=mp, **kw)
    gs.stream_status()
    N = S.shape[0]
    cols = [x.cpu().numpy() if torch.is_tensor(x) else [x] * N for x in (U, T, k, p, mp)]
    idx, prob = out["index"].cpu().numpy(), out["prob"].cpu().numpy()
    s = S.float().cpu().numpy()
    for n in range(N):
        cand, pr = reference(s[n], *(c[n] for c in cols))
        assert int(idx[n]) in cand, (n, int(idx[n]), cand)
        # two conversions and one division in fp32, weights exact to 2^-34
        assert abs(prob[n] - pr[int(idx[n])]) <= 4 * 2.0 ** -24 * pr[int(idx[n])] + 2.0 ** -37, n
    return out


def scores(N, M, dtype, seed=0, spread=2.0):
    g = torch.Generator().manual_seed(seed * 1009 + N + 7 * M)
    S = (torch.randn(N, M, generator=g) * spread).to(DT[dtype]).cuda()
    return S, torch.rand(N, generator=g).cuda()


SETTINGS = [dict(), dict(T=0.7), dict(k=1), dict(k=3), dict(k=50), dict(p=0.9), dict(p=0.3), dict(mp=0.1), dict(T=0.0),
            dict(T=0.8, k=40, p=0.95, mp=0.02), dict(T=1.5, k=1000, p=0.5), dict(p=0.0), dict(mp=1.0), dict(T=2.0, p=0.999),
            dict(T=-1.0), dict(k=-3), dict(mp=2.0), dict(p=2.0)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M", [1, 2, 5, 31, 40, 257, 1000, 4099, 32000])
@pytest.mark.parametrize("how", SETTINGS, ids=str)
def test_settings(gs, how, M, dtype):
    S, U = scores(7 if M > 1000 else 33, M, dtype)
    check(gs, S, U, **how)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_vocabulary(gs, dtype):
    S, U = scores(3, 262144, dtype)
    for how in (dict(), dict(p=0.9), dict(k=50, p=0.9), dict(k=200000), dict(mp=0.01)):
        check(gs, S, U, **how)


def test_largest_rows(gs):
    S, U = scores(2, 1 << 19, "f32", spread=0.0)  # every weight the same: sums of 2^19 x 2^44
    check(gs, S, U)
    check(gs, S, U, p=0.75)
    check(gs, S, U, k=300000)


@pytest.mark.parametrize("M", [8, 64, 1000, 20000])
def test_ties_go_to_the_lowest_index(gs, M):
    g = torch.Generator().manual_seed(M)
    S = torch.randint(0, 3, (40, M), generator=g).float().cuda()
    S[0] = 0.0
    S[1] = -0.0
    S[2, ::2], S[2, 1::2] = 0.0, -0.0
    U = torch.rand(40, generator=g).cuda()
    for how in (dict(), dict(k=3), dict(k=M - 1), dict(p=0.5), dict(p=0.25, k=M // 2), dict(mp=1.0), dict(T=0.0)):
        check(gs, S, U, **how)
    assert (gs.sample_scores(S[:3], U[:3], temperature=0.0)["index"].cpu() == 0).all()


@pytest.mark.parametrize("M", [9, 3001])
def test_not_finite_scores(gs, M):
    S, U = scores(8, M, "f32")
    inf, nan = float("inf"), float("nan")
    S[0] = -inf                       # nothing to draw
    S[1] = nan
    S[2, 0], S[2, 1] = nan, -inf
    S[3, 2], S[3, 5] = inf, inf       # only these
    S[4] = -inf
    S[4, 6] = -3e38                   # one entry, the lowest that is finite
    S[5] = torch.finfo(torch.float32).min
    S[6, 0], S[6, 1] = 3e38, -3e38    # a difference beyond fp32
    for how in (dict(), dict(k=2), dict(p=0.8), dict(mp=0.5), dict(T=0.0), dict(T=inf), dict(T=1e-40), dict(T=1e38)):
        check(gs, S, U, **how)
    out = gs.sample_scores(S, U)
    assert out["index"][:2].tolist() == [-1, -1] and out["prob"][:2].tolist() == [0, 0]


def test_random_numbers_at_the_ends(gs):
    S, _ = scores(6, 500, "f32")
    U = torch.tensor([0.0, -1.0, float("nan"), 1.0, 7.0, 1 - 2.0 ** -24]).cuda()
    check(gs, S, U)
    check(gs, S, U, p=0.7)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M", [300, 5000])
def test_settings_per_row(gs, M, dtype):
    N = 48
    S, U = scores(N, M, dtype)
    g = torch.Generator().manual_seed(5)
    pick = lambda v, dt: torch.tensor(v, dtype=dt)[torch.randint(0, len(v), (N,), generator=g)].cuda()  # noqa: E731
    check(gs, S, U, T=pick([0.0, 0.5, 1.0, 2.0, float("nan")], torch.float32), k=pick([0, 1, 7, 100, 4000], torch.int32),
          p=pick([0.2, 0.9, 1.0, float("nan")], torch.float32), mp=pick([0.0, 0.3, 1.0, float("nan")], torch.float32))


@pytest.mark.parametrize("M", [40, 70000])
def test_probabilities(gs, M):
    """20,000 draws of one row land on each frequent entry as often as its probability says."""
    S, _ = scores(1, M, "f32", spread=3.0)
    N = 20000
    g = torch.Generator().manual_seed(2)
    U = torch.rand(N, generator=g).cuda()
    idx = gs.sample_scores(S.expand(N, M) if M > 1000 else S.repeat(N, 1), U, temperature=0.9, top_k=20)["index"].cpu()
    v, i = S[0].cpu().double().topk(20)
    p = torch.softmax(v / 0.9, 0)
    for q, j in zip(p.tolist(), i.tolist()):
        # binomial: 6 standard deviations and half a count
        assert abs(int((idx == j).sum()) - N * q) <= 6 * (N * q * (1 - q)) ** 0.5 + 1


def test_layouts_streams_graphs(gs):
    S, U = scores(30, 1501, "f32")
    want = check(gs, S, U, k=30)
    big = torch.full((30, 1600), 9e9, device="cuda")
    big[:, 7:1508] = S
    a = check(gs, big[:, 7:1508], U, k=30)
    assert torch.equal(a["index"], want["index"])
    b16 = torch.full((30, 1600), 9e9, device="cuda", dtype=torch.bfloat16)
    b16[:, 7:1508] = S.bfloat16()
    check(gs, b16[:, 7:1508], U, p=0.8)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    b = gs.sample_scores(S, U, top_k=30, stream=side)
    side.synchronize()
    assert torch.equal(b["index"], want["index"]) and torch.equal(b["prob"], want["prob"])
    s2, u2 = S.clone(), U.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c = gs.sample_scores(s2, u2, top_k=30)
    s2.copy_(S.flip(0))
    u2.copy_(U.flip(0))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(c["index"], want["index"].flip(0)) and torch.equal(c["prob"], want["prob"].flip(0))
    only = gs.sample_scores(S, U, top_k=30, want_prob=False)
    assert set(only) == {"index"} and torch.equal(only["index"], want["index"])
    assert gs.sample_scores(S[:0], U[:0])["index"].shape == (0,)


@pytest.mark.parametrize("N", [1, 20, 700])
def test_long_rows_of_few_and_many(gs, N):
    """Rows that one CTA, some or eight share."""
    S, U = scores(N, 9001, "f32", seed=3)
    for how in (dict(), dict(k=20, p=0.8), dict(p=0.95), dict(p=0.9999), dict(T=0.0), dict(mp=0.2)):
        out = gs.sample_scores(S, U, temperature=how.get("T", 1.0), top_k=how.get("k", 0), top_p=how.get("p", 1.0),
                               min_p=how.get("mp", 0.0))
        pick = torch.arange(0, N, max(1, N // 10)).cuda()
        part = check(gs, S[pick].contiguous(), U[pick].contiguous(), **how)
        assert torch.equal(part["index"], out["index"][pick]) and torch.equal(part["prob"], out["prob"][pick])


def test_long_rows_that_are_not_finite(gs):
    S, U = scores(7, 9000, "f32")
    inf = float("inf")
    S[0] = -inf
    S[1] = float("nan")
    S[2, ::3] = -inf
    S[3, 100], S[3, 8000], S[3, 8500] = inf, inf, inf
    S[4] = -inf
    S[4, 8999] = 1.0
    S[5] = 2.5
    S[6, ::2] = torch.finfo(torch.float32).min
    for how in (dict(), dict(k=2), dict(p=0.7), dict(k=5000, p=0.9), dict(mp=0.5), dict(T=0.0), dict(T=inf), dict(T=1e-40, k=3)):
        check(gs, S, U, **how)
