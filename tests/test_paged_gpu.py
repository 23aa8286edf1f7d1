"""The paged cache through the public calls: slots, stores and attention over it."""
import math

import pytest
import torch

from attn_bounds import close
from window_bounds import SeenRef

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


# ----------------------------------------------------------------- slots
def plain_slots(lens, added, table, free, page, max_new, pages, start):
    table = [list(r) for r in table]
    cols = len(table[0]) if table else 0
    nxt, slots, out = start, [], []
    for row, n, k in zip(table, lens, added):
        n, k = min(max(n, 0), cols * page), min(max(k, 0), max_new)
        end = min(n + k, cols * page)
        have, want = -(-n // page), -(-end // page)
        first = nxt
        for c in range(have, want):
            row[c] = free[nxt] if nxt < len(free) else -1
            nxt += 1
        end = min(end, (have + min(max(len(free) - first, 0), want - have)) * page)
        s = []
        for j in range(n, n + max_new):
            e = row[j // page] if j < end else -1
            s.append(e * page + j % page if 0 <= e < pages else -1)
        slots.append(s)
        out.append(end)
    return table, slots, out, nxt - start


@pytest.mark.parametrize("B,page,max_new,old,cols", [(1, 16, 1, 40, 8), (300, 16, 1, 90, 9), (700, 1, 3, 5, 8), (5, 7, 40, 30, 12),
                                                     (3, 64, 3000, 500, 60), (2000, 4, 2, 20, 7), (257, 5, 0, 20, 6), (4, 100, 9, 0, 1)])
@pytest.mark.parametrize("short", [False, True])
def test_slots(gs, B, page, max_new, old, cols, short):
    g = torch.Generator().manual_seed(B + page)
    pages = B * cols + 5
    lens = torch.randint(-2, old + 1, (B,), generator=g, dtype=torch.int32)
    added = torch.randint(-1, max_new + 2, (B,), generator=g, dtype=torch.int32)
    table = torch.randint(0, pages, (B, cols + 3), generator=g, dtype=torch.int32)
    table[torch.rand(B, cols + 3, generator=g) < 0.05] = -1
    table[torch.rand(B, cols + 3, generator=g) < 0.02] = pages
    free = torch.randperm(pages, generator=g).int()
    if short:
        free = free[:3 + B // 3]
    start = 3
    want = plain_slots(lens.tolist(), added.tolist(), table[:, 1:1 + cols].tolist(), free.tolist(), page, max_new, pages, start)
    dev = table.cuda()
    view = dev[:, 1:1 + cols]  # a table with columns of its own
    for _ in range(2):  # the same call again gives the same
        out = gs.page_slots(lens.cuda(), added.cuda(), view, free.cuda(), page, max_new, pages,
                            free_from=torch.tensor([start], dtype=torch.int32).cuda())
        gs.stream_status()
        assert view.tolist() == want[0]
        assert out["slots"].tolist() == want[1] and out["lens"].tolist() == want[2] and out["taken"].tolist() == [want[3]]
    assert torch.equal(dev[:, 0].cpu(), table[:, 0]) and torch.equal(dev[:, 1 + cols:].cpu(), table[:, 1 + cols:])


def test_slots_of_nobody(gs):
    e = torch.empty(0, dtype=torch.int32).cuda()
    out = gs.page_slots(e, e, e.view(0, 4), e, 16, 3, 10)
    assert out["slots"].shape == (0, 3) and out["taken"].tolist() == [0]
    one = torch.tensor([0], dtype=torch.int32).cuda()
    out = gs.page_slots(one, one + 2, one.view(1, 1)[:, :0], e, 16, 3, 10)  # a table without columns
    assert out["slots"].tolist() == [[-1, -1, -1]] and out["lens"].tolist() == [0] and out["taken"].tolist() == [0]


# ----------------------------------------------------------------- stores
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H,dk,dv,how", [(8, 128, 128, "dense"), (3, 40, 24, "dense"), (2, 5, 1, "dense"), (4, 64, 32, "heads first"),
                                         (2, 64, 64, "shifted"), (1, 16, 16, "dense")])
def test_store(gs, dtype, H, dk, dv, how):
    g = torch.Generator().manual_seed(H + dk)
    B, L, pages, page = 3, 50, 23, 9
    K, V = (torch.randn(B, L, H, w, generator=g).to(DT[dtype]).cuda() for w in (dk, dv))

    def cache(w):
        if how == "heads first":
            return torch.randn(pages, H, page, w, generator=g).to(DT[dtype]).cuda().permute(0, 2, 1, 3)
        if how == "shifted":
            return torch.randn(pages, page, H, w + 3, generator=g).to(DT[dtype]).cuda()[..., 1:1 + w]
        return torch.randn(pages, page, H, w, generator=g).to(DT[dtype]).cuda()

    Kc, Vc = cache(dk), cache(dv)
    slots = torch.randperm(pages * page, generator=g)[:B * L].view(B, L).int()
    slots[torch.rand(B, L, generator=g) < 0.2] = -1
    slots[0, 3], slots[1, 4] = pages * page, -2 ** 31
    want = [Kc.clone(), Vc.clone()]
    for b in range(B):
        for i in range(L):
            s = int(slots[b, i])
            if 0 <= s < pages * page:
                want[0][s // page, s % page], want[1][s // page, s % page] = K[b, i], V[b, i]
    gs.page_store(K, V, slots.cuda(), Kc, Vc)
    gs.stream_status()
    assert torch.equal(Kc, want[0]) and torch.equal(Vc, want[1])


# ----------------------------------------------------------------- attention
def make(B, Lq, Hq, Hkv, dk, dv, page, lens, dtype, seed=0, spare=2):
    g = torch.Generator().manual_seed(seed * 7919 + B + 31 * Lq + Hq + dk + page)
    cols = max(1, -(-max(lens) // page)) + spare
    pages = B * cols + 1
    Q = (torch.randn(B, Lq, Hq, dk, generator=g) * 1.5).to(DT[dtype]).cuda()
    Kc, Vc = (torch.randn(pages, page, Hkv, w, generator=g).to(DT[dtype]) for w in (dk, dv))
    table = torch.randperm(pages, generator=g)[:B * cols].view(B, cols).int()
    for b in range(B):  # what no request holds is not finite, and columns behind its pages are no pages
        used = -(-lens[b] // page)
        if lens[b] % page:
            last = int(table[b, used - 1])
            Kc[last, lens[b] % page:], Vc[last, lens[b] % page:] = math.nan, math.inf
        for c in range(used, cols):
            Kc[int(table[b, c])], Vc[int(table[b, c])] = math.inf, math.nan
        table[b, used + 1:] = -1
        table[b, cols - 1] = pages + 3 if used < cols else table[b, cols - 1]
    return Q, Kc.cuda(), Vc.cuda(), table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda()


def reference(Q, Kc, Vc, table, lens, q_lens, window, sinks, scale, tensor):
    B, Lq = Q.shape[:2]
    pages, page, Hkv, _ = Kc.shape
    n = int(lens.max().clamp(min=1))
    K = torch.zeros(B, n, Hkv, Kc.shape[3], dtype=Kc.dtype)
    V = torch.zeros(B, n, Hkv, Vc.shape[3], dtype=Vc.dtype)
    see = torch.zeros(B, Lq, n, dtype=torch.bool)
    kc, vc, t = Kc.cpu(), Vc.cpu(), table.cpu()
    for b in range(B):
        m = int(lens[b])
        ql = Lq if q_lens is None else min(max(int(q_lens[b]), 0), Lq)
        j = torch.arange(m)
        if m:
            e = t[b, j // page].long()
            there = (e >= 0) & (e < pages)
            K[b, :m][there], V[b, :m][there] = kc[e[there], j[there] % page], vc[e[there], j[there] % page]
        for i in range(ql):
            p = m - ql + i
            if m:
                see[b, i, :m] = there & (j <= p) & ((j > p - window) | (j < sinks))
    return SeenRef(Q, K, V, scale, see, tensor)


def attend(gs, Q, Kc, Vc, table, lens, q_lens=None, window=None, sinks=0, path="auto", tensor=None, **kw):
    scale = 1.0 / math.sqrt(Q.shape[3])
    if tensor is None:
        tensor = Q.dtype == torch.bfloat16 and path != "simt"
    r = reference(Q, Kc, Vc, table, lens, q_lens, window or 2 ** 40, sinks, scale, tensor)
    out = gs.paged_attention(Q, Kc, Vc, table, lens, scale, q_lens, window, sinks, want_lse=True, path=path, **kw)
    gs.stream_status()
    tol, tol_lse = r.forward_tol()
    close(out["O"], r.o.permute(0, 2, 1, 3), tol, "O")
    none = r.lse == -math.inf
    lse = out["lse"].cpu().double()
    assert (lse[none] == -math.inf).all() and (out["O"].cpu().permute(0, 2, 1, 3)[none] == 0).all()
    close(lse[~none], r.lse[~none], tol_lse[~none], "lse")
    return out


# Lq, Hq, Hkv, dk, dv, page, lens
CASES = [
    (1, 1, 1, 1, 1, 1, [1, 0, 5]),
    (1, 8, 8, 64, 64, 16, [197, 3, 16, 17]),
    (1, 32, 8, 128, 128, 16, [300, 1, 0, 1025]),
    (1, 8, 1, 64, 64, 64, [64, 65, 500]),
    (5, 8, 2, 128, 128, 32, [700, 5, 3, 33]),       # drafts: more rows than one request has keys
    (8, 16, 4, 64, 128, 24, [257, 100, 8]),         # 32 rows to a key head
    (3, 21, 3, 72, 40, 5, [90, 11]),                # 7 query heads to a key head
    (17, 4, 1, 128, 64, 16, [400, 20]),             # more rows than a tile
    (1, 4, 4, 40, 40, 32, [2000, 31, 513]),
    (2, 3, 3, 7, 33, 3, [40, 2]),
    (1, 128, 1, 128, 128, 128, [129, 900]),         # 128 query heads to a key head
    (1, 2, 2, 128, 128, 1, [77, 300]),              # pages of one position
    (4, 8, 8, 64, 64, 256, [3000, 255, 256]),
]


@pytest.mark.parametrize("path", ["auto", "simt"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("window,sinks", [(None, 0), (50, 0), (20, 4), (1, 0), (129, 130)])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "x".join(map(str, c[:6])))
def test_attention(gs, case, window, sinks, dtype, path):
    Lq, Hq, Hkv, dk, dv, page, lens = case
    t = make(len(lens), Lq, Hq, Hkv, dk, dv, page, lens, dtype)
    attend(gs, *t, window=window, sinks=sinks, path=path)
    if Lq > 1:
        q_lens = torch.tensor([(3 * b + 1) % (Lq + 2) - (b == 1) for b in range(len(lens))], dtype=torch.int32).cuda()
        attend(gs, *t, q_lens=q_lens, window=window, sinks=sinks, path=path)


@pytest.mark.parametrize("path", ["auto", "simt"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_requests_of_uneven_lengths(gs, dtype, path):
    """More work than CTAs run at once: parts of long requests beside short ones and empty ones."""
    g = torch.Generator().manual_seed(3)
    lens = [int(x) for x in torch.randint(0, 200, (150,), generator=g)] + [6000, 0, 1, 2, 2999]
    t = make(len(lens), 1, 8, 4, 64, 64, 16, lens, dtype)
    a = attend(gs, *t, path=path)
    b = attend(gs, *t, window=100, sinks=5, path=path)
    assert torch.equal(a["O"], gs.paged_attention(*t, path=path)["O"])
    assert torch.equal(b["O"], gs.paged_attention(*t, window=100, sinks=5, path=path)["O"])


@pytest.mark.parametrize("path", ["auto", "simt"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_holes_in_the_table(gs, dtype, path):
    t = make(3, 2, 8, 2, 128, 128, 16, [500, 90, 33], dtype)
    t[3][0, 3], t[3][0, 7], t[3][1, 0], t[3][2, :3] = -1, 2 ** 30, -5, -1
    attend(gs, *t, path=path)
    attend(gs, *t, window=150, sinks=60, path=path)


@pytest.mark.parametrize("path", ["auto", "simt"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_what_a_row_does_not_see(gs, dtype, path):
    """Later drafts' keys and values, and those that have left the window, are not finite."""
    for bad in (math.nan, math.inf, -torch.finfo(DT[dtype]).max):
        t = make(2, 6, 8, 2, 128, 128, 16, [300, 40], dtype)
        ref = gs.paged_attention(*t, window=32, sinks=2, want_lse=True, path=path)
        Kc, Vc, table = t[1], t[2], t[3]
        for b, n in ((0, 300), (1, 40)):
            for j in (n - 2, n - 1, n - 36, n - 35, n - 34, n - 33):  # seen by the last two rows; by no or the first rows
                if j >= 2:
                    Kc[table[b, j // 16], j % 16], Vc[table[b, j // 16], j % 16] = bad, bad
        out = gs.paged_attention(*t, window=32, sinks=2, want_lse=True, path=path)
        gs.stream_status()
        # row i stands at n - 6 + i and sees from n - 37 + i on: row 0 .. 3 see some of the old ones, none sees n - 2 but 4 and 5
        assert torch.equal(out["O"][0, 4:4], ref["O"][0, 4:4])
        clean = [i for i in range(6) if all(not (n - 37 + i <= j <= n - 6 + i) for n in (300,)
                                            for j in (n - 2, n - 1, n - 36, n - 35, n - 34, n - 33))]
        for i in clean:
            assert torch.equal(out["O"][0, i], ref["O"][0, i]) and torch.equal(out["lse"][0, :, i], ref["lse"][0, :, i])
        t = make(2, 6, 8, 2, 128, 128, 16, [300, 40], dtype)
        for b, n in ((0, 300), (1, 40)):
            for j in (n - 3, n - 2, n - 1):
                t[1][t[3][b, j // 16], j % 16], t[2][t[3][b, j // 16], j % 16] = bad, bad
        out = gs.paged_attention(*t, window=32, sinks=2, want_lse=True, path=path)
        gs.stream_status()
        assert torch.equal(out["O"][:, :3], ref["O"][:, :3]) and torch.equal(out["lse"][:, :, :3], ref["lse"][:, :, :3])


@pytest.mark.parametrize("how", ["heads first", "shifted", "one cache"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_layouts(gs, dtype, how):
    Q, Kc, Vc, table, lens = make(3, 2, 8, 4, 64, 64, 16, [300, 44, 1], dtype)
    if how == "heads first":
        Kc, Vc = (x.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3) for x in (Kc, Vc))
    elif how == "shifted":
        Kc, Vc = (torch.cat([x[..., :1], x, x[..., :2]], dim=3)[..., 1:65] for x in (Kc, Vc))
    else:  # keys and values of a page side by side
        both = torch.stack([Kc, Vc], dim=1)
        Kc, Vc = both[:, 0], both[:, 1]
    for path in ("auto", "simt"):
        attend(gs, Q, Kc, Vc, table, lens, path=path)
        attend(gs, Q, Kc, Vc, table, lens, window=33, sinks=3, path=path)


def test_decoding_steps(gs):
    """Slots, stores and attention together, step by step, against attention over the dense history."""
    g = torch.Generator().manual_seed(5)
    B, Hq, Hkv, w, page, cols, steps = 3, 4, 2, 64, 8, 12, (30, 1, 1, 3, 20, 1)
    pages = B * cols
    dt = torch.bfloat16
    Kc, Vc = (torch.full((pages, page, Hkv, w), math.nan, dtype=dt, device="cuda") for _ in range(2))
    table = torch.full((B, cols), -1, dtype=torch.int32, device="cuda")
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    free = torch.randperm(pages, generator=g).int().cuda()
    used = torch.zeros(1, dtype=torch.int32, device="cuda")
    past = [[torch.zeros(0, Hkv, w), torch.zeros(0, Hkv, w)] for _ in range(B)]
    for n in steps:
        added = torch.randint(0, n + 1, (B,), generator=g, dtype=torch.int32)
        Q, K, V = (torch.randn(B, n, h, w, generator=g).to(dt) for h in (Hq, Hkv, Hkv))
        s = gs.page_slots(lens, added.cuda(), table, free, page, n, pages, free_from=used)
        used += s["taken"]
        gs.page_store(K.cuda(), V.cuda(), s["slots"], Kc, Vc)
        lens = s["lens"]
        out = gs.paged_attention(Q.cuda(), Kc, Vc, table, lens, q_lens=added.cuda(), window=25, sinks=2)["O"]
        gs.stream_status()
        for b in range(B):
            k = int(added[b])
            past[b] = [torch.cat([x, y[b, :k].float()]) for x, y in zip(past[b], (K, V))]
            m = past[b][0].shape[0]
            assert int(lens[b]) == m
            if k:
                want = gs.window_attention(Q[b:b + 1, :k].cuda(), *(x.to(dt).cuda()[None] for x in past[b]), 25, 2, m - k)["O"]
                # two correct results: each is off by its rounding and that of its weights
                assert (out[b, :k].float() - want[0].float()).abs().max() <= 2 * 2.0 ** -8 * 4 * float(past[b][1].abs().max())
            assert (out[b, k:] == 0).all()
