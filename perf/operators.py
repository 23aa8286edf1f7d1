"""Timed cases of cross attention, its gradient, and sampling from scores.

``cross_attention`` reads an encoder's states (keys and values of another length than the queries, padded, several heads,
key heads shared by groups of query heads), ``cross_attention_backward`` is its gradient, ``sample_scores`` draws one entry
of each score row from given random numbers.  ``run`` computes them in elementary torch operations, or through the library
where ``own`` is true; ``exact`` computes them in 64 bits, one sequence and head (or one row) at a time.
"""
import math

import torch

own = False


def listed():
    return [
        # one decoding step of a small batch against short memories: latency counts
        {"name": "step_small", "kind": "attend", "B": 4, "Lq": 1, "Lk": 197, "Hq": 8, "Hkv": 8, "dk": 64, "dv": 64,
         "dtype": "bf16", "mask": "none", "lse": False},
        # one decoding step of a full serving batch, memories padded to the longest
        {"name": "step_batch", "kind": "attend", "B": 64, "Lq": 1, "Lk": 1500, "Hq": 16, "Hkv": 16, "dk": 64, "dv": 64,
         "dtype": "bf16", "mask": "lens", "lse": False},
        # one decoding step against long memories, four query heads to a key head: bound by memory
        {"name": "step_long", "kind": "attend", "B": 8, "Lq": 1, "Lk": 65537, "Hq": 32, "Hkv": 8, "dk": 128, "dv": 128,
         "dtype": "bf16", "mask": "none", "lse": False},
        # the training forward pass of a decoder over padded encoder states (its backward pass is "train")
        {"name": "prompt", "kind": "attend", "B": 8, "Lq": 1024, "Lk": 1500, "Hq": 16, "Hkv": 16, "dk": 64, "dv": 64,
         "dtype": "bf16", "mask": "lens", "lse": True},
        # long prompts, shared key heads: the largest forward pass, bound by the tensor cores
        {"name": "prompt_large", "kind": "attend", "B": 4, "Lq": 4096, "Lk": 4096, "Hq": 32, "Hkv": 8, "dk": 128,
         "dv": 128, "dtype": "bf16", "mask": "none", "lse": False},
        # compressed vectors as the library returns them (fp32, one head as wide as a basis of 40 codewords): the 16
        # panels of each of 64 problems attend to a masked context of 1,024 vectors
        {"name": "panels_f32", "kind": "attend", "B": 64, "Lq": 16, "Lk": 1024, "Hq": 1, "Hkv": 1, "dk": 40, "dv": 40,
         "dtype": "f32", "mask": "holes", "lse": True},
        # the backward pass of "prompt"
        {"name": "train", "kind": "grad", "B": 8, "Lq": 1024, "Lk": 1500, "Hq": 16, "Hkv": 16, "dk": 64, "dv": 64,
         "dtype": "bf16", "mask": "lens"},
        # the largest backward pass
        {"name": "train_large", "kind": "grad", "B": 2, "Lq": 4096, "Lk": 4096, "Hq": 32, "Hkv": 8, "dk": 128, "dv": 128,
         "dtype": "bf16", "mask": "none"},
        # a small backward pass in 32 bits, odd lengths, keys and values of different widths
        {"name": "train_f32", "kind": "grad", "B": 16, "Lq": 100, "Lk": 257, "Hq": 4, "Hkv": 2, "dk": 40, "dv": 30,
         "dtype": "f32", "mask": "holes"},
        # drawing codebook entries for a batch of score rows (a codebook of 256 entries)
        {"name": "sample_codes", "kind": "sample", "N": 4096, "M": 256, "dtype": "f32", "temperature": 0.7, "top_k": 0,
         "top_p": 0.9, "min_p": 0.0, "per_row": False},
        # drawing tokens of a large vocabulary, every request with its own settings
        {"name": "sample_vocab", "kind": "sample", "N": 64, "M": 131071, "dtype": "bf16", "temperature": 0.8, "top_k": 50,
         "top_p": 0.95, "min_p": 0.02, "per_row": True},
        # the same for a large batch of 32-bit scores without top-k: the nucleus is cut out of the whole row
        {"name": "sample_nucleus", "kind": "sample", "N": 256, "M": 128000, "dtype": "f32", "temperature": 1.0, "top_k": 0,
         "top_p": 0.9, "min_p": 0.0, "per_row": False},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _near(rng, n, step):
    """n as it is, or rounded to a multiple of step: odd sizes and even ones."""
    return n if rng.random() < 0.5 else max(step, n // step * step)


def draw(rng):
    kind = rng.choice(["step", "step", "attend", "attend", "grad", "grad", "sample", "sample"])
    if kind == "sample":
        M = _near(rng, _log(rng, 5, 200000), 8)
        N = min(_log(rng, 1, 8192), (1 << 25) // M)
        return {"kind": kind, "N": max(1, N), "M": M, "dtype": rng.choice(["f32", "bf16"]),
                "temperature": rng.choice([0.0, 0.5, 0.8, 1.0, 1.5]), "top_k": rng.choice([0, 0, 1, 5, 50, 1000]),
                "top_p": rng.choice([1.0, 0.95, 0.9, 0.5]), "min_p": rng.choice([0.0, 0.0, 0.05, 0.2]),
                "per_row": rng.random() < 0.5}
    while True:
        Hkv = rng.choice([1, 2, 4, 8, 16])
        c = {"kind": "grad" if kind == "grad" else "attend", "B": _log(rng, 1, 64),
             "Lq": 1 if kind == "step" else _near(rng, _log(rng, 2, 4096), 64), "Lk": _near(rng, _log(rng, 1, 65536), 64),
             "Hq": Hkv * rng.choice([1, 1, 2, 4, 7, 8]), "Hkv": Hkv}
        c["dtype"] = rng.choice(["bf16", "bf16", "bf16", "f32"])
        c["dk"] = rng.choice([64, 128, 64, 128, 8 * rng.randint(1, 16), rng.randint(1, 128)])
        c["dv"] = rng.choice([c["dk"], c["dk"], 64, 128, rng.randint(1, 128)])
        c["mask"] = rng.choice(["none", "lens", "lens", "holes"])
        if c["kind"] == "attend":
            c["lse"] = rng.random() < 0.3
        w = work(c)
        scores = c["B"] * c["Hq"] * c["Lq"] * c["Lk"]
        if c["Lq"] * c["Lk"] >= 16 and w["bytes"] <= 1e9 and scores <= (1 << 30) and \
                w["flops"] <= (3e11 if c["dtype"] == "bf16" else 2e10):
            return c


# --------------------------------------------------------------------------- inputs
def _gen(seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1000003 + stream) & 0x7FFFFFFF)
    return g


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _inputs(case, seed):
    g = _gen(seed, 1)
    dt = _dtype(case)
    if case["kind"] == "sample":
        N, M = case["N"], case["M"]
        # scores as a trained model gives them: a normal bulk, and some entries that stand out
        S = torch.randn((N, M), generator=g, device="cuda") * 2.0
        top = torch.randint(0, M, (N, 8), generator=g, device="cuda")
        S.scatter_add_(1, top, 6.0 * torch.rand((N, 8), generator=g, device="cuda"))
        t = {"S": S.to(dt), "U": torch.rand(N, generator=g, device="cuda")}
        for name, default in (("temperature", 1.0), ("top_k", 0), ("top_p", 1.0), ("min_p", 0.0)):
            kind = torch.int32 if name == "top_k" else torch.float32
            v = torch.full((N,), case[name], dtype=kind, device="cuda")
            if case["per_row"]:  # some requests leave the setting at its default
                v = torch.where(torch.rand(N, generator=g, device="cuda") < 0.25, torch.full_like(v, default), v)
            t[name] = v
        return t
    B, Lq, Lk, Hq, Hkv, dk, dv = (case[k] for k in ("B", "Lq", "Lk", "Hq", "Hkv", "dk", "dv"))
    t = {"Q": (1.5 * torch.randn((B, Lq, Hq, dk), generator=g, device="cuda")).to(dt),
         "K": torch.randn((B, Lk, Hkv, dk), generator=g, device="cuda").to(dt),
         "V": torch.randn((B, Lk, Hkv, dv), generator=g, device="cuda").to(dt), "lens": None, "mask": None}
    if case["mask"] != "none":  # sequences of half the padded length to all of it
        t["lens"] = torch.randint((Lk + 1) // 2, Lk + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    if case["mask"] == "holes":  # and single positions that are not to be read
        t["mask"] = torch.rand((B, Lk), generator=g, device="cuda") < 0.8
    if case["kind"] == "grad":
        t["dO"] = torch.randn((B, Lq, Hq, dv), generator=g, device="cuda").to(dt)
    return t


def _scale(case):
    return 1.0 / math.sqrt(case["dk"])


def prepare(case, seed):
    state = {"case": case, **_inputs(case, seed)}
    if case["kind"] == "grad":  # the forward pass' results
        state["O"], state["lse"] = _attend(state, case)
    if case["kind"] == "sample" and not case["per_row"]:
        state["settings"] = {k: float(torch.tensor(case[k])) for k in ("temperature", "top_p", "min_p")}
    return state


# --------------------------------------------------------------------------- plain forms
def _valid(t, case):
    """B x 1 x 1 x Lk truth values: the keys that may be read."""
    pos = torch.arange(case["Lk"], device="cuda")
    ok = torch.ones((case["B"], case["Lk"]), dtype=torch.bool, device="cuda")
    if t["lens"] is not None:
        ok = pos < t["lens"][:, None]
    if t["mask"] is not None:
        ok = ok & t["mask"]
    return ok[:, None, None, :]


def _groups(x, Hkv):
    """B x L x Hq x d -> B x Hkv x (Hq / Hkv) L x d, in 32 bits."""
    B, L, Hq, d = x.shape
    return x.float().view(B, L, Hkv, Hq // Hkv, d).permute(0, 2, 3, 1, 4).reshape(B, Hkv, Hq // Hkv * L, d)


def _ungroup(x, Hq, L):
    """The way back."""
    B, Hkv, _, d = x.shape
    return x.view(B, Hkv, Hq // Hkv, L, d).permute(0, 3, 1, 2, 4).reshape(B, L, Hq, d)


def _logits(t, case):
    ok = _valid(t, case)
    q, k = _groups(t["Q"], case["Hkv"]), t["K"].float().permute(0, 2, 3, 1)
    return torch.where(ok, torch.matmul(q, k) * _scale(case), -math.inf), ok


def _values(x, ok):
    """B x Lk x Hkv x d keys or values -> B x Hkv x Lk x d in 32 bits, zero where they may not be read."""
    return torch.where(ok.permute(0, 1, 3, 2), x.float().permute(0, 2, 1, 3), 0.0)


def _attend(t, case):
    s, ok = _logits(t, case)
    m = s.amax(dim=-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    p = torch.exp(s - m)
    l = p.sum(dim=-1, keepdim=True)
    o = torch.matmul(p, _values(t["V"], ok)) / torch.where(l == 0, 1.0, l)
    o = _ungroup(o, case["Hq"], case["Lq"]).to(_dtype(case))
    return o, (m + torch.log(l)).view(case["B"], case["Hq"], case["Lq"])


def _grad(t, case):
    s, ok = _logits(t, case)
    lse = t["lse"].view(case["B"], case["Hkv"], -1, 1)
    p = torch.exp(s - torch.where(lse == -math.inf, 0.0, lse))
    del s
    do, q = _groups(t["dO"], case["Hkv"]), _groups(t["Q"], case["Hkv"])
    k, v = _values(t["K"], ok), _values(t["V"], ok)
    dv = torch.matmul(p.transpose(2, 3), do)
    dp = torch.matmul(do, v.transpose(2, 3))
    ds = p * (dp - (p * dp).sum(dim=-1, keepdim=True)) * _scale(case)
    del p, dp
    dq = _ungroup(torch.matmul(ds, k), case["Hq"], case["Lq"])
    dk = torch.matmul(ds.transpose(2, 3), q)
    dt = _dtype(case)
    return {"dQ": dq.to(dt), "dK": dk.permute(0, 2, 1, 3).to(dt), "dV": dv.permute(0, 2, 1, 3).to(dt)}


def _sample(t):
    """The kept entries' weights in sorted order decide what is kept, and in index order what is drawn: in 64 bits, as the
    running sums of many small weights end next to the drawn number."""
    s = t["S"].double()
    T = t["temperature"].double()[:, None]
    best = s.amax(dim=1, keepdim=True)
    w = torch.exp((s - best) / torch.where(T > 0, T, 1.0))
    order = torch.argsort(s, dim=1, descending=True, stable=True)
    ws = torch.gather(w, 1, order)
    rank = torch.arange(s.shape[1], device="cuda")[None, :]
    k = t["top_k"].long()[:, None]
    ws = torch.where((rank < k) | (k <= 0), ws, 0.0)
    cum = torch.cumsum(ws, dim=1)
    p = t["top_p"].double()[:, None]
    ws = torch.where((cum - ws < p * cum[:, -1:]) | (p >= 1) | (rank == 0), ws, 0.0)
    ws = torch.where((ws >= t["min_p"].double()[:, None]) & ((T > 0) | (rank == 0)), ws, 0.0)
    kept = torch.zeros_like(w).scatter_(1, order, ws)
    run = torch.cumsum(kept, dim=1)
    total = run[:, -1:]
    i = (run <= t["U"].double()[:, None] * total).sum(dim=1, keepdim=True)
    return {"index": i[:, 0].int(), "prob": (torch.gather(kept, 1, i) / total)[:, 0].float()}


def run(state):
    c = state["case"]
    if own:
        from paper_2608_01528_gb300 import gramspace as gs

        if c["kind"] == "attend":
            return gs.cross_attention(state["Q"], state["K"], state["V"], _scale(c), key_lens=state["lens"],
                                      key_mask=state["mask"], want_lse=c["lse"])
        if c["kind"] == "grad":
            return gs.cross_attention_backward(state["Q"], state["K"], state["V"], state["O"], state["lse"], state["dO"],
                                               _scale(c), key_lens=state["lens"], key_mask=state["mask"])
        if c["per_row"]:
            return gs.sample_scores(state["S"], state["U"], temperature=state["temperature"], top_k=state["top_k"],
                                    top_p=state["top_p"], min_p=state["min_p"])
        return gs.sample_scores(state["S"], state["U"], top_k=c["top_k"], **state["settings"])
    if c["kind"] == "attend":
        o, lse = _attend(state, c)
        return {"O": o, "lse": lse} if c["lse"] else {"O": o}
    return _grad(state, c) if c["kind"] == "grad" else _sample(state)


# --------------------------------------------------------------------------- work
def work(case):
    if case["kind"] == "sample":
        N, M = float(case["N"]), float(case["M"])
        e = 2 if case["dtype"] == "bf16" else 4
        return {"bytes": e * N * M + 12 * N + (16 * N if case["per_row"] else 0), "flops": 4 * N * M}
    B, Lq, Lk, Hq, Hkv, dk, dv = (float(case[k]) for k in ("B", "Lq", "Lk", "Hq", "Hkv", "dk", "dv"))
    e = 2 if case["dtype"] == "bf16" else 4
    read = 1.0 if case["mask"] == "none" else 0.75  # the mean length of padded sequences
    q, kv = B * Lq * Hq, B * Lk * read * Hkv
    bits = 0 if case["mask"] != "holes" else B * Lk * read
    if case["kind"] == "attend":
        return {"bytes": e * (q + kv) * (dk + dv) + bits + (4 * q if case["lse"] else 0),
                "flops": 2 * q * Lk * read * (dk + dv)}
    return {"bytes": e * (q * (2 * dk + 2 * dv) + (kv + B * Lk * Hkv) * (dk + dv)) + 4 * q + bits,
            "flops": 2 * q * Lk * read * (3 * dk + 2 * dv)}


# --------------------------------------------------------------------------- 64 bits
def _exact_head(t, case, b, h):
    """One sequence's query head: the keys that are read, and P, O, lse over them."""
    hk = h // (case["Hq"] // case["Hkv"])
    n = case["Lk"] if t["lens"] is None else int(t["lens"][b])
    read = torch.arange(n, device="cuda")
    if t["mask"] is not None:
        read = read[t["mask"][b, :n]]
    k, v = t["K"][b, read, hk].double(), t["V"][b, read, hk].double()
    q = t["Q"][b, :, h].double()
    if not len(read):
        return hk, read, q, k, v, None, None, None
    s = torch.einsum("id,jd->ij", q, k).mul_(_scale(case))
    lse = torch.logsumexp(s, dim=1)
    p = s.sub_(lse[:, None]).exp_()
    return hk, read, q, k, v, p, p @ v, lse


def _exact_row(s, u, T, k, p, mp):
    """One row of scores, entry by entry in the order of the definition."""
    M = s.numel()
    if T <= 0:
        return int((s == s.max()).nonzero()[0]), 1.0
    val, idx = torch.sort(s.double(), descending=True, stable=True)
    w = ((val - val[0]) / T).exp()
    n = k if 0 < k < M else M
    if p < 1:
        run = w[:n].cumsum(0)
        n = min(n, 1 + int((run < p * run[-1]).sum()))
    n = max(1, min(n, int((w[:n] >= mp).sum())))
    idx, order = idx[:n].sort()
    run = w[:n][order].cumsum(0)
    j = min(n - 1, int((run <= u * run[-1]).sum()))
    return int(idx[j]), float(w[:n][order][j] / run[-1])


def exact(case, seed):
    t = _inputs(case, seed)
    if case["kind"] == "sample":
        if case["N"] > 1024 and case["M"] > 1024:
            return None
        cols = [t[k].double().tolist() for k in ("U", "temperature", "top_k", "top_p", "min_p")]
        S = t["S"] if case["M"] > 4096 else t["S"].cpu()
        rows = [_exact_row(S[n], u, T, int(k), p, mp) for n, (u, T, k, p, mp) in enumerate(zip(*cols))]
        return {"index": torch.tensor([r[0] for r in rows], dtype=torch.int32),
                "prob": torch.tensor([r[1] for r in rows], dtype=torch.float64)}
    B, Lq, Lk, Hq, Hkv, dk, dv = (case[k] for k in ("B", "Lq", "Lk", "Hq", "Hkv", "dk", "dv"))

    def zeros(*shape):
        return torch.zeros(shape, dtype=torch.float64, device="cuda")

    O, lse = zeros(B, Lq, Hq, dv), zeros(B, Hq, Lq) - math.inf
    dQ, dK, dV = zeros(B, Lq, Hq, dk), zeros(B, Lk, Hkv, dk), zeros(B, Lk, Hkv, dv)
    for b in range(B):
        for h in range(Hq):
            hk, read, q, k, v, p, o, l = _exact_head(t, case, b, h)
            if p is None:
                continue
            O[b, :, h], lse[b, h] = o, l
            if case["kind"] == "grad":
                do = t["dO"][b, :, h].double()
                dV[b, read, hk] += p.T @ do
                ds = (do @ v.T).sub_((do * o).sum(1, keepdim=True)).mul_(p).mul_(_scale(case))
                dQ[b, :, h] = ds @ k
                dK[b, read, hk] += ds.T @ q
    if case["kind"] == "grad":
        return {"dQ": dQ, "dK": dK, "dV": dV}
    return {"O": O, "lse": lse} if case["lse"] else {"O": O}
