"""Window attention, the paged cache and draft verification as programs call them: captured decoding steps, several streams and host
threads, layouts of other kinds, memory that held something else, nothing at all."""
import math
import threading

import pytest
import torch

from test_verify_gpu import make as drafts
from test_window_gpu import check, make, masks

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


class Decoder:
    """One step: slots for a token of each request, its keys and values stored, attention over the cache, new lengths."""

    def __init__(self, gs, dtype, B=5, Hq=8, Hkv=4, w=64, page=8, cols=20):
        g = torch.Generator().manual_seed(11)
        self.gs, self.page, self.pages = gs, page, B * cols
        self.Q, self.K, self.V = (torch.zeros(B, 1, h, w, dtype=DT[dtype], device="cuda") for h in (Hq, Hkv, Hkv))
        self.Kc, self.Vc = (torch.full((self.pages, page, Hkv, w), math.nan, dtype=DT[dtype], device="cuda") for _ in range(2))
        self.table = torch.full((B, cols), -1, dtype=torch.int32, device="cuda")
        self.lens = torch.zeros(B, dtype=torch.int32, device="cuda")
        self.one = torch.ones(B, dtype=torch.int32, device="cuda")
        self.free = torch.randperm(self.pages, generator=g).int().cuda()
        self.used = torch.zeros(1, dtype=torch.int32, device="cuda")

    def step(self):
        s = self.gs.page_slots(self.lens, self.one, self.table, self.free, self.page, 1, self.pages, free_from=self.used)
        self.used += s["taken"]
        self.gs.page_store(self.K, self.V, s["slots"], self.Kc, self.Vc)
        self.lens.copy_(s["lens"])
        return self.gs.paged_attention(self.Q, self.Kc, self.Vc, self.table, self.lens, window=30, sinks=2, want_lse=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_captured_decoding_steps(gs, dtype):
    """A captured step, replayed with new tokens, gives the bits of eager steps, while an eager decoder's own steps run between."""
    g = torch.Generator().manual_seed(3)
    a, b = Decoder(gs, dtype), Decoder(gs, dtype)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = b.step()
    past = []
    for i in range(45):
        new = [torch.randn(t.shape, generator=g).to(DT[dtype]).cuda() for t in (a.Q, a.K, a.V)]
        past.append(new[1:])
        for d in (a, b):
            for t, x in zip((d.Q, d.K, d.V), new):
                t.copy_(x)
        want = a.step()
        graph.replay()
        gs.stream_status()
        assert torch.equal(out["O"], want["O"]) and torch.equal(out["lse"], want["lse"])
        assert torch.equal(a.table, b.table) and torch.equal(a.lens, b.lens) and int(a.lens[0]) == i + 1
    K, V = (torch.cat([p[k] for p in past], dim=1) for k in range(2))
    dense = gs.window_attention(a.Q, K, V, 30, 2, 44, path="simt")["O"].float()
    # two results, each off by the output's rounding and (bf16) that of its weights, of values below 4
    tol = 2 * (2 * 2.0 ** -8 if dtype == "bf16" else 64 * 2.0 ** -24) * 4
    assert (out["O"].float() - dense).abs().max() <= tol


def calls(gs):
    """Calls with inputs of their own, each giving a list of tensors."""
    made = []
    for i, dtype in enumerate(("bf16", "f32", "bf16")):
        Q, K, V, dO = make(2, 150 + 10 * i, 300, 8, 2, 64, 64, dtype, seed=i)
        lens, _ = masks("lens", 2, 300, i)

        def window(Q=Q, K=K, V=V, dO=dO, lens=lens, **kw):
            o = gs.window_attention(Q, K, V, 70, 3, 120, key_lens=lens, want_lse=True, **kw)
            d = gs.window_attention_backward(Q, K, V, o["O"], o["lse"], dO, 70, 3, 120, key_lens=lens, **kw)
            return [*o.values(), *d.values()]

        made.append(window)
        P, D, x, U, n = drafts(9, 4, 5000 + i, dtype, seed=i)
        made.append(lambda P=P, D=D, x=x, U=U, n=n, **kw: list(gs.verify_drafts(P, D, x, U, n, **kw).values()))
        Kc, Vc = K.reshape(-1, 30, 2, 64).contiguous(), V.reshape(-1, 30, 2, 64).contiguous()
        table = torch.randperm(20, generator=torch.Generator().manual_seed(i)).int().view(2, 10).cuda()
        made.append(lambda Q=Q[:, :2].contiguous(), Kc=Kc, Vc=Vc, t=table, lens=lens, **kw: list(
            gs.paged_attention(Q, Kc, Vc, t, lens, want_lse=True, **kw).values()))
    return made


def test_threads_and_streams_at_once(gs):
    made = calls(gs)
    want = [f() for f in made]
    torch.cuda.synchronize()
    wrong = []

    def work(k):
        try:
            s = torch.cuda.Stream()
            for _ in range(8):
                for i in list(range(k, len(made))) + list(range(k)):
                    got = made[i](stream=s)
                    s.synchronize()
                    if not all(torch.equal(x, y) for x, y in zip(got, want[i])):
                        wrong.append(i)
        except Exception as e:  # noqa: BLE001
            wrong.append(repr(e))

    threads = [threading.Thread(target=work, args=(k,)) for k in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    gs.stream_status()
    assert not wrong, wrong


def test_memory_that_held_something_else(gs):
    """Outputs and workspaces over NaN give what they gave over zeros."""
    made = calls(gs)
    got = []
    for fill in (0.0, math.nan):
        torch.cuda.empty_cache()
        dirt = [torch.full((n,), fill, device="cuda") for n in (1 << 26, 1 << 20, 1 << 16, 1 << 12, 1 << 12, 1 << 8) * 2]
        torch.cuda.synchronize()
        del dirt
        got.append([[t.clone() for t in f()] for f in made])
    gs.stream_status()
    assert all(torch.equal(x, y) for a, b in zip(*got) for x, y in zip(a, b))


@pytest.mark.parametrize("how", ["interleaved", "heads first", "unaligned", "one for all", "one row's gradient"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_layouts(gs, dtype, how):
    Q, K, V, dO = make(2, 200, 260, 6, 3, 64, 64, dtype)
    if how == "interleaved":
        both = torch.stack([K, V], dim=2)
        K, V = both[:, :, 0], both[:, :, 1]
    elif how == "heads first":
        Q, K, V, dO = (t.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3) for t in (Q, K, V, dO))
    elif how == "unaligned":
        Q, K, V, dO = (torch.cat([t[..., :1], t, t[..., :2]], dim=3)[..., 1:65] for t in (Q, K, V, dO))
    elif how == "one for all":
        K = K[:1, :, :1].expand(2, 260, 3, 64)
        V = K
    else:
        dO = dO[:, :1].expand(2, 200, 6, 64)
    lens, _ = masks("lens", 2, 260)
    tensor = dtype == "bf16"
    for window, sinks in ((40, 3), (None, 0)):
        check(gs, Q, K, V, dO, window, sinks, 60, lens, tensor=tensor)
        check(gs, Q, K, V, dO, window, sinks, 60, lens, path="simt")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_nothing(gs, dtype):
    for B, Lq, Lk in ((0, 5, 6), (2, 0, 6), (2, 5, 0)):
        Q, K, V, dO = make(B, Lq, Lk, 4, 2, 64, 64, dtype)
        out = gs.window_attention(Q, K, V, 3, 1, want_lse=True)
        assert (out["O"] == 0).all() and (out["lse"] == -math.inf).all()
        d = gs.window_attention_backward(Q, K, V, out["O"], out["lse"], dO, 3, 1)
        assert all((t == 0).all() for t in d.values())
    Q = torch.randn(3, 2, 4, 64).to(DT[dtype]).cuda()
    cache = torch.zeros(4, 8, 2, 64, dtype=DT[dtype], device="cuda")
    lens = torch.tensor([0, 7, -3], dtype=torch.int32).cuda()
    none = torch.zeros(3, 0, dtype=torch.int32).cuda()
    for c, t in ((cache, none), (cache[:0], none), (cache[:0], torch.zeros(3, 2, dtype=torch.int32).cuda())):
        out = gs.paged_attention(Q, c, c, t, lens, want_lse=True)
        gs.stream_status()
        assert (out["O"] == 0).all() and (out["lse"] == -math.inf).all()
