"""Cross attention and sampling as programs call them: caches with room behind the sequences, interleaved states, broadcast
gradients, several streams and host threads, memory that held something else, a process whose first call is captured."""
import math
import pathlib
import subprocess
import sys
import threading

import pytest
import torch

from attn_bounds import Ref, close

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def rand(g, *shape, dtype="f32"):
    return torch.randn(*shape, generator=g).to(DT[dtype]).cuda()


def attend(gs, Q, K, V, lens=None, mask=None, path="auto", tensor=None, **kw):
    """One forward call against 64 bits."""
    scale = Q.shape[3] ** -0.5
    if tensor is None:
        tensor = Q.dtype == torch.bfloat16 and path != "simt"
    r = Ref(Q, K, V, scale, lens, mask, tensor)
    out = gs.cross_attention(Q, K, V, key_lens=lens, key_mask=mask, want_lse=True, path=path, **kw)
    gs.stream_status()
    tol, tol_lse = r.forward_tol()
    close(out["O"], r.o.permute(0, 2, 1, 3), tol, "O")
    none = r.lse == -math.inf
    lse = out["lse"].cpu().double()
    assert (lse[none] == -math.inf).all()
    close(lse[~none], r.lse[~none], tol_lse[~none], "lse")
    return out


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [(1, 1), (1, 2), (1, 5), (2, 1), (3, 4)], ids=str)
@pytest.mark.parametrize("width", [(64, 64), (128, 128), (40, 72), (128, 1)], ids=str)
def test_cache_with_room_behind(gs, width, rows, dtype):
    """A few rows over views of one cache: NaN behind the sequences and around the heads, lengths from 0 to all, holes."""
    (dk, dv), (Lq, G) = width, rows
    g = torch.Generator().manual_seed(dk + 10 * Lq + G)
    B, room, Lk, Hkv = 5, 900, 801, 3
    cache = torch.full((B, room, Hkv + 1, dk + dv + 8), math.nan, dtype=DT[dtype], device="cuda")
    K, V = cache[:, 3:3 + Lk, 1:, :dk], cache[:, 3:3 + Lk, 1:, dk:dk + dv]
    lens = torch.tensor([801, 0, 1, 259, 640], dtype=torch.int32)
    for b in range(B):
        n = int(lens[b])
        K[b, :n], V[b, :n] = rand(g, n, Hkv, dk, dtype=dtype), rand(g, n, Hkv, dv, dtype=dtype)
    mask = torch.rand(B, Lk, generator=g) < 0.7
    K[~mask.cuda()] = math.inf
    V[~mask.cuda()] = math.nan
    Q = rand(g, B, Lq, Hkv * G, dk, dtype=dtype)
    for path in ("auto", "simt"):
        attend(gs, Q, K, V, lens.cuda(), mask.cuda(), path)


@pytest.mark.parametrize("how", ["unaligned", "interleaved", "heads first", "one for all"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_layouts_of_a_few_rows(gs, dtype, how):
    g = torch.Generator().manual_seed(7)
    B, Lk, H, w = 3, 700, 4, 64
    if how == "interleaved":    # keys and values of one projection
        kv = rand(g, B, Lk, 2, H, w, dtype=dtype)
        K, V = kv[:, :, 0], kv[:, :, 1]
    elif how == "unaligned":
        kv = rand(g, B, Lk, H, 2 * w + 3, dtype=dtype)
        K, V = kv[..., 1:1 + w], kv[..., w + 2:2 * w + 2]
    elif how == "heads first":
        K, V = (rand(g, B, H, Lk, w, dtype=dtype).permute(0, 2, 1, 3) for _ in range(2))
    else:                       # one head and sequence of states, read by every head and sequence, keys as values
        K = V = rand(g, 1, Lk, 1, w, dtype=dtype).expand(B, Lk, H, w)
    for Lq in (1, 2, 3, 6):
        Q = rand(g, B, Lq, H, w, dtype=dtype)
        attend(gs, Q, K, V)
        attend(gs, Q, K, V, path="simt")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("width", [64, 128])
@pytest.mark.parametrize("Lq", [1, 2, 4])
def test_not_finite_logits_of_a_few_rows(gs, Lq, width, dtype):
    """A NaN or +inf among the valid logits makes its row NaN and no other; -inf weighs nothing."""
    g = torch.Generator().manual_seed(Lq)
    for path in ("auto", "simt"):
        for bad, at in ((math.inf, 3), (math.nan, 511), (-math.inf, 1299)):
            Q, K, V = rand(g, 2, Lq, 2, width, dtype=dtype), rand(g, 2, 1300, 2, width, dtype=dtype), rand(g, 2, 1300, 2, width, dtype=dtype)
            Q[..., 0] = 1.0
            clean = gs.cross_attention(Q, K, V, want_lse=True, path=path)
            keep = K.clone()
            K[0, at, 1, 0] = bad
            out = gs.cross_attention(Q, K, V, want_lse=True, path=path)
            gs.stream_status()
            hit = torch.zeros(2, Lq, 2, dtype=torch.bool)
            hit[0, :, 1] = True
            if bad != -math.inf:
                assert torch.isnan(out["O"][hit.cuda()]).all() and torch.isnan(out["lse"].permute(0, 2, 1)[hit.cuda()]).all()
            else:
                mask = torch.ones(2, 1300, dtype=torch.bool)
                mask[0, at] = False
                same = gs.cross_attention(Q, keep, V, want_lse=True, path=path, key_mask=mask.cuda())
                assert torch.equal(out["O"][hit.cuda()], same["O"][hit.cuda()])
            assert torch.equal(out["O"][~hit.cuda()], clean["O"][~hit.cuda()])
            assert torch.equal(out["lse"].permute(0, 2, 1)[~hit.cuda()], clean["lse"].permute(0, 2, 1)[~hit.cuda()])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_broadcast_gradient(gs, dtype):
    """dO of a sum: one number expanded over everything (all strides 0), as autograd hands it on."""
    g = torch.Generator().manual_seed(5)
    Q, K, V = rand(g, 2, 30, 4, 64, dtype=dtype), rand(g, 2, 170, 2, 64, dtype=dtype), rand(g, 2, 170, 2, 64, dtype=dtype)
    r = Ref(Q, K, V, 0.125)
    dO = torch.ones(1, 1, 1, 1, dtype=DT[dtype], device="cuda").expand(2, 30, 4, 64)
    O, lse = r.o.permute(0, 2, 1, 3).to(DT[dtype]).cuda(), r.lse.float().cuda()
    # the last axis has to be dense: the wrapper says so, and one row repeated along the others is taken
    with pytest.raises(ValueError):
        gs.cross_attention_backward(Q, K, V, O, lse, dO, 0.125)
    dO = torch.ones(64, dtype=DT[dtype], device="cuda").expand(2, 30, 4, 64)
    got = gs.cross_attention_backward(Q, K, V, O, lse, dO, 0.125)
    gs.stream_status()
    for name, (want, tol) in r.grad(dO).items():
        close(got[name], want, tol, name)


def test_outputs_that_repeat_memory(gs):
    g = torch.Generator().manual_seed(6)
    Q, K, V = (rand(g, 2, 3, 2, 8) for _ in range(3))
    for t in (torch.zeros(1, 3, 2, 8).cuda().expand(2, 3, 2, 8), torch.zeros(2, 1, 2, 8).cuda().expand(2, 3, 2, 8)):
        with pytest.raises(gs.GramSpaceError):
            gs.cross_attention(Q, K, V, out={"O": t})


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_memory_that_held_something_else(gs, dtype):
    """Outputs and workspaces on memory full of NaN; sequences that end in the first of many parts."""
    g = torch.Generator().manual_seed(8)
    Q, K, V, dO = (rand(g, 3, n, 4, 64, dtype=dtype) for n in (2, 6000, 6000, 2))
    lens = torch.tensor([6000, 5, 0], dtype=torch.int32).cuda()
    want = gs.cross_attention(Q, K, V, key_lens=lens, want_lse=True)
    gwant = gs.cross_attention_backward(Q, K, V, want["O"], want["lse"], dO, key_lens=lens)
    S, U = rand(g, 40, 9000, dtype=dtype), torch.rand(40, generator=g).cuda()
    swant = gs.sample_scores(S, U, top_p=0.9)
    torch.cuda.synchronize()
    for _ in range(3):
        torch.cuda.empty_cache()
        junk = [torch.full((n,), math.nan, device="cuda") for n in (1 << 24, 1 << 22, 1 << 20, 1 << 18, 1 << 16, 1 << 12, 128)
                for _ in range(4)]
        torch.cuda.synchronize()
        del junk
        a = gs.cross_attention(Q, K, V, key_lens=lens, want_lse=True)
        b = gs.cross_attention_backward(Q, K, V, a["O"], a["lse"], dO, key_lens=lens)
        c = gs.sample_scores(S, U, top_p=0.9)
        assert all(torch.equal(a[k], want[k]) for k in want) and all(torch.equal(b[k], gwant[k]) for k in gwant)
        assert all(torch.equal(c[k], swant[k]) for k in swant)


def test_threads_and_streams_at_once(gs):
    """Four host threads, each with a stream and a problem of its own, all operators in turn."""
    jobs = []
    for i, (dtype, Lq, Lk) in enumerate((("bf16", 1, 3000), ("f32", 4, 2000), ("bf16", 300, 500), ("f32", 90, 300))):
        g = torch.Generator().manual_seed(i)
        Q, K, V, dO = (rand(g, 2, n, 4, 64, dtype=dtype) for n in (Lq, Lk, Lk, Lq))
        S, U = rand(g, 30, 300 * 7 ** i, dtype=dtype), torch.rand(30, generator=g).cuda()

        def run(stream=None, Q=Q, K=K, V=V, dO=dO, S=S, U=U):
            a = gs.cross_attention(Q, K, V, want_lse=True, stream=stream)
            b = gs.cross_attention_backward(Q, K, V, a["O"], a["lse"], dO, stream=stream)
            return {**a, **b, **gs.sample_scores(S, U, top_k=50, top_p=0.9, stream=stream)}

        jobs.append((run, run()))
    torch.cuda.synchronize()
    wrong = []

    def work(run, want):
        try:
            s = torch.cuda.Stream()
            for _ in range(20):
                got = run(s)
                s.synchronize()
                if not all(torch.equal(got[k], want[k]) for k in want):
                    wrong.append("results differ")
        except Exception as e:  # a thread's exception would be lost
            wrong.append(repr(e))

    threads = [threading.Thread(target=work, args=j) for j in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong, wrong
    gs.stream_status()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_small_sequences(gs, dtype):
    """More (sequence, head) pairs than 2^16, of one to three rows and a few keys each."""
    g = torch.Generator().manual_seed(9)
    B = 23000
    for Lq, Lk, H, w in ((1, 3, 3, 8), (3, 5, 3, 8)):
        Q, K, V, dO = (rand(g, B, n, H, w, dtype=dtype) for n in (Lq, Lk, Lk, Lq))
        lens = torch.randint(0, Lk + 1, (B,), generator=g, dtype=torch.int32).cuda()
        out = attend(gs, Q, K, V, lens)
        got = gs.cross_attention_backward(Q, K, V, out["O"], out["lse"], dO, key_lens=lens)
        gs.stream_status()
        for i in (0, 1, 11500, B - 1):
            part = gs.cross_attention_backward(*(t[i:i + 1].contiguous() for t in (Q, K, V, out["O"], out["lse"], dO)),
                                               key_lens=lens[i:i + 1].contiguous())
            # alone the sequence may be cut into other parts: both lie within the bound
            r = Ref(Q[i:i + 1], K[i:i + 1], V[i:i + 1], w ** -0.5, lens[i:i + 1], None, dtype == "bf16")
            for name, (want, tol) in r.grad(dO[i:i + 1]).items():
                close(got[name][i:i + 1], want, tol, name)
                close(part[name], want, tol, name)


def test_draws_from_one_row(gs):
    """A row expanded over its draws: one pass each over the same scores."""
    g = torch.Generator().manual_seed(10)
    for M in (40, 3000, 20000):
        row = rand(g, 1, M)
        U = torch.rand(500, generator=g).cuda()
        a = gs.sample_scores(row.expand(500, M), U, top_p=0.7, top_k=20)
        b = gs.sample_scores(row.repeat(500, 1), U, top_p=0.7, top_k=20)
        assert torch.equal(a["index"], b["index"]) and torch.equal(a["prob"], b["prob"])


FIRST = """
import sys, torch
sys.path.insert(0, {root!r})
from paper_2608_01528_gb300 import gramspace as gs
torch.manual_seed(0)
Q, K, V = (torch.randn(2, n, 4, 64).bfloat16().cuda() for n in (40, 900, 900))
f = [t.float() for t in (Q, K, V)]
S, U = torch.randn(8, 9000).cuda(), torch.rand(8).cuda()
torch.cuda.synchronize()
def calls():
    out = []
    for q, k, v in ((Q, K, V), f, (Q[:, :1], K, V), [t[:, :2] for t in f]):
        a = gs.cross_attention(q, k, v, want_lse=True)
        b = gs.cross_attention_backward(q, k, v, a["O"], a["lse"], a["O"])
        out += [a["O"], a["lse"], b["dQ"], b["dK"], b["dV"]]
    for m in (9000, 2000, 100):
        c = gs.sample_scores(S[:, :m], U, top_p=0.9)
        out += [c["index"], c["prob"]]
    return out
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    got = calls()
graph.replay()
torch.cuda.synchronize()
assert all(torch.equal(x, y) for x, y in zip(got, calls()))
gs.stream_status()
print("same")
"""


def test_first_call_of_a_process_is_captured(gs):
    root = str(pathlib.Path(__file__).resolve().parent.parent)
    r = subprocess.run([sys.executable, "-c", FIRST.format(root=root)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "same" in r.stdout, r.stderr[-2000:]


@pytest.mark.parametrize("kind", ["none", "lens", "holes"])
@pytest.mark.parametrize("width", [(68, 64), (64, 87), (47, 128), (33, 33), (1, 127), (7, 1)], ids=str)
@pytest.mark.parametrize("shape", [(2, 40, 300, 4, 2), (3, 300, 70, 7, 1), (1, 17, 3000, 2, 2), (20, 129, 129, 8, 8)], ids=str)
def test_odd_widths_on_tensor_cores(gs, shape, width, kind):
    """bf16 widths that are no multiple of 8 are laid out again: dense, padded and broadcast inputs."""
    (B, Lq, Lk, Hq, Hkv), (dk, dv) = shape, width
    g = torch.Generator().manual_seed(dk + dv + Lk)
    Q, K, V, dO = (rand(g, *s, dtype="bf16") for s in ((B, Lq, Hq, dk), (B, Lk, Hkv, dk), (B, Lk, Hkv, dv), (B, Lq, Hq, dv)))
    lens = torch.randint(0, Lk + 1, (B,), generator=g, dtype=torch.int32).cuda() if kind == "lens" else None
    mask = (torch.rand(B, Lk, generator=g) < 0.6).cuda() if kind == "holes" else None
    ok = torch.ones(B, Lk, dtype=torch.bool)
    if lens is not None:
        ok &= torch.arange(Lk)[None] < lens.cpu()[:, None]
    if mask is not None:
        ok &= mask.cpu()
    K[~ok.cuda()], V[~ok.cuda()] = math.nan, math.inf
    scale = dk ** -0.5
    r = Ref(Q, K, V, scale, lens, mask, True)
    want = r.grad(dO)
    forms = [(Q, K, V, dO)]
    if kind == "none":  # rows padded to other lengths, heads first, one sequence's states for all
        pad = [torch.full((*t.shape[:3], t.shape[3] + 5), math.nan, dtype=t.dtype, device="cuda") for t in (Q, K, V, dO)]
        for p, t in zip(pad, (Q, K, V, dO)):
            p[..., 3:3 + t.shape[3]] = t
        forms.append(tuple(p[..., 3:3 + t.shape[3]] for p, t in zip(pad, (Q, K, V, dO))))
        forms.append(tuple(t.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3) for t in (Q, K, V, dO)))
    for q, k, v, d in forms:
        # only widths that are no multiple of 8 are laid out again: a forced path with others off their 16 bytes is refused
        off = any(t.shape[3] % 8 == 0 and t.data_ptr() % 16 for t in (q, k, v))
        if off:
            with pytest.raises(gs.GramSpaceError, match="ALIGNMENT"):
                gs.cross_attention(q, k, v, path="tensor")
        for path in ("auto",) if off else ("auto", "tensor"):
            out = attend(gs, q, k, v, lens, mask, path, True)
            O, lse = r.o.permute(0, 2, 1, 3).bfloat16().cuda(), r.lse.float().cuda()
            got = gs.cross_attention_backward(q, k, v, O, lse, d, scale, key_lens=lens, key_mask=mask, path=path)
            gs.stream_status()
            for name, (w, tol) in want.items():
                close(got[name], w, tol, name)
            assert out["O"].shape == O.shape


def test_odd_widths_broadcast_and_captured(gs):
    g = torch.Generator().manual_seed(12)
    Q, K, V, dO = rand(g, 3, 50, 4, 36, dtype="bf16"), rand(g, 1, 90, 1, 36, dtype="bf16"), rand(g, 1, 90, 1, 20, dtype="bf16"), \
        rand(g, 20, dtype="bf16")
    K, V, dO = K.expand(3, 90, 2, 36), V.expand(3, 90, 2, 20), dO.expand(3, 50, 4, 20)
    out = attend(gs, Q, K, V)
    got = gs.cross_attention_backward(Q, K, V, out["O"], out["lse"], dO)
    r = Ref(Q, K, V, 1 / 6, None, None, True)
    exact = gs.cross_attention_backward(Q, K, V, r.o.permute(0, 2, 1, 3).bfloat16().cuda(), r.lse.float().cuda(), dO)
    for name, (w, tol) in r.grad(dO).items():
        close(exact[name], w, tol, name)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o = gs.cross_attention(Q, K, V, want_lse=True)
        b = gs.cross_attention_backward(Q, K, V, o["O"], o["lse"], dO)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(o[k], out[k]) for k in out) and all(torch.equal(b[k], got[k]) for k in got)
    gs.stream_status()
