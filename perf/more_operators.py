"""Timed cases of a decoding program's operators: the paged cache (slots for new tokens, storing their keys and values,
attention over it), the verification of drafted tokens, and causal attention over a sliding window with its gradient.

``append`` gives new tokens their slots in the pages of a cache and stores their keys and values there; ``paged`` reads the cache with
the newest tokens of every request; ``verify`` accepts drafted tokens against the target's probabilities; ``window`` and ``grad`` are
attention over the last keys and a few first ones, as prompts and training have it.  ``run`` computes them in elementary torch
operations, or through the library where ``own`` is true; ``exact`` computes them in 64 bits, one sequence and head (or
one request) at a time.
"""
import math

import torch

own = False


def listed():
    return [
        # a decoding step of a serving batch: one token a request, most of them inside a page that is there already
        {"name": "append_step", "kind": "append", "B": 256, "Lnew": 1, "old": 1000, "page": 16, "Hkv": 8, "dk": 128, "dv": 128,
         "dtype": "bf16", "short": False},
        # prompts of uneven lengths enter the cache
        {"name": "append_prompt", "kind": "append", "B": 16, "Lnew": 4096, "old": 100, "page": 64, "Hkv": 8, "dk": 128,
         "dv": 128, "dtype": "bf16", "short": False},
        # one decoding step of four short requests: latency counts
        {"name": "decode_small", "kind": "paged", "B": 4, "Lq": 1, "lo": 90, "hi": 300, "page": 16, "Hq": 8, "Hkv": 8, "dk": 64,
         "dv": 64, "dtype": "bf16", "window": 0, "sinks": 0, "ragged": False},
        # one decoding step of a serving batch, requests of very different ages, four query heads to a key head
        {"name": "decode_batch", "kind": "paged", "B": 64, "Lq": 1, "lo": 1, "hi": 4096, "page": 16, "Hq": 32, "Hkv": 8, "dk": 128,
         "dv": 128, "dtype": "bf16", "window": 0, "sinks": 0, "ragged": False},
        # up to five drafted tokens and the last certain one over long histories: the largest step, bound by memory
        {"name": "drafts_long", "kind": "paged", "B": 8, "Lq": 6, "lo": 32769, "hi": 65537, "page": 64, "Hq": 32, "Hkv": 8,
         "dk": 128, "dv": 128, "dtype": "bf16", "window": 0, "sinks": 0, "ragged": True},
        # streams of compressed vectors as the library returns them (fp32, one head as wide as a basis of 40 codewords) that
        # read their last 512 and first 4 positions
        {"name": "stream_f32", "kind": "paged", "B": 256, "Lq": 1, "lo": 1, "hi": 2000, "page": 32, "Hq": 1, "Hkv": 1, "dk": 40,
         "dv": 40, "dtype": "f32", "window": 512, "sinks": 4, "ragged": False},
        # three drafts for each of a few requests: latency counts
        {"name": "verify_small", "kind": "verify", "B": 4, "K": 3, "M": 32000, "dtype": "f32", "given": True, "ragged": False},
        # a full serving batch, up to five drafts, a large vocabulary
        {"name": "verify_batch", "kind": "verify", "B": 256, "K": 5, "M": 131072, "dtype": "bf16", "given": True, "ragged": True},
        # prompts of padded length, shared key heads, the last 1,024 and the first 4 keys: the largest forward pass
        {"name": "prompt_window", "kind": "window", "B": 4, "Lq": 4096, "start": 0, "Hq": 32, "Hkv": 8, "dk": 128, "dv": 128,
         "dtype": "bf16", "window": 1024, "sinks": 4, "mask": "lens", "lse": True},
        # prompts that go on behind 57 cached positions, fp32, odd widths, single positions left out
        {"name": "window_f32", "kind": "window", "B": 16, "Lq": 200, "start": 57, "Hq": 4, "Hkv": 2, "dk": 40, "dv": 30,
         "dtype": "f32", "window": 64, "sinks": 2, "mask": "holes", "lse": False},
        # the backward pass of training on long sequences
        {"name": "train_window", "kind": "grad", "B": 2, "Lq": 4096, "start": 0, "Hq": 32, "Hkv": 8, "dk": 128, "dv": 128,
         "dtype": "bf16", "window": 1024, "sinks": 4, "mask": "none"},
        # a small backward pass in 32 bits, odd lengths, keys and values of different widths
        {"name": "train_window_f32", "kind": "grad", "B": 16, "Lq": 257, "start": 0, "Hq": 4, "Hkv": 2, "dk": 40, "dv": 30,
         "dtype": "f32", "window": 50, "sinks": 3, "mask": "holes"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _near(rng, n, step):
    """n as it is, or rounded to a multiple of step: odd sizes and even ones."""
    return n if rng.random() < 0.5 else max(step, n // step * step)


def _heads(rng):
    Hkv = rng.choice([1, 2, 4, 8, 16])
    c = {"Hq": Hkv * rng.choice([1, 1, 2, 4, 7, 8]), "Hkv": Hkv}
    c["dtype"] = rng.choice(["bf16", "bf16", "bf16", "f32"])
    c["dk"] = rng.choice([64, 128, 64, 128, 8 * rng.randint(1, 16), rng.randint(1, 128)])
    c["dv"] = rng.choice([c["dk"], c["dk"], c["dk"], 64, 128, rng.randint(1, 128)])
    return c


def draw(rng):
    kind = rng.choice(["append", "paged", "paged", "paged", "verify", "window", "window", "grad", "grad"])
    page = rng.choice([16, 16, 32, 64, 128, 24, 1, 256])
    if kind == "verify":
        M = _near(rng, _log(rng, 5, 200000), 8)
        K = rng.randint(1, 8)
        return {"kind": kind, "B": max(1, min(_log(rng, 1, 512), (1 << 27) // (M * (K + 1)))), "K": K, "M": M,
                "dtype": rng.choice(["f32", "bf16"]), "given": rng.random() < 0.75, "ragged": rng.random() < 0.5}
    if kind == "append":
        while True:
            c = {"kind": kind, "B": _log(rng, 1, 1024), "Lnew": rng.choice([1, 1, _log(rng, 2, 2048)]), "old": _log(rng, 1, 4096),
                 "page": page, **_heads(rng), "short": rng.random() < 0.2}
            del c["Hq"]
            e = 2 if c["dtype"] == "bf16" else 4
            if c["B"] * (c["old"] + c["Lnew"] + 2 * page) * c["Hkv"] * (c["dk"] + c["dv"]) * e <= 5e8:
                return c
    while True:
        c = {"kind": kind, "B": _log(rng, 1, 64), **_heads(rng)}
        if kind == "paged":
            c.update(Lq=rng.choice([1, 1, 1, rng.randint(2, 8)]), hi=_near(rng, _log(rng, 1, 65536), 64), page=page,
                     window=rng.choice([0, 0, _log(rng, 1, 8192)]), sinks=0, ragged=False)
            c["lo"] = rng.choice([1, max(1, c["hi"] // 2), c["hi"]])
            if c["window"]:
                c["sinks"] = rng.choice([0, 1, 4, 16, 130])
            if c["Lq"] > 1:
                c["ragged"] = rng.random() < 0.5
            e = 2 if c["dtype"] == "bf16" else 4
            if c["B"] * (c["hi"] + page) * c["Hkv"] * (c["dk"] + c["dv"]) * e <= 1e9:
                return c
            continue
        c.update(Lq=_near(rng, _log(rng, 1, 4096), 64), start=rng.choice([0, 0, _log(rng, 1, 1000)]),
                 window=rng.choice([_log(rng, 1, 4096), _log(rng, 1, 4096), 1 << 20]), sinks=rng.choice([0, 1, 4, 16, 130]),
                 mask=rng.choice(["none", "lens", "holes"]))
        if kind == "window":
            c["lse"] = rng.random() < 0.3
        w = work(c)
        if w["bytes"] <= 4e8 and c["B"] * c["Hq"] * c["Lq"] * (c["Lq"] + c["start"]) <= (1 << 30) and \
                w["flops"] <= (1.5e11 if c["dtype"] == "bf16" else 2e10):
            return c


# --------------------------------------------------------------------------- inputs
def _gen(seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1000003 + stream) & 0x7FFFFFFF)
    return g


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _randn(g, dt, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(dt)


def _ints(g, lo, hi, *shape):
    """lo to hi, both included."""
    return torch.randint(lo, hi + 1, shape, generator=g, device="cuda", dtype=torch.int32)


def _pages(case):
    """Columns of the block table, and pages of the cache."""
    longest = case["old"] + case["Lnew"] if case["kind"] == "append" else case["hi"]
    cols = -(-longest // case["page"])
    return cols, case["B"] * cols + 3


def _append_inputs(case, seed):
    g = _gen(seed, 2)
    dt, B, L, page = _dtype(case), case["B"], case["Lnew"], case["page"]
    cols, pages = _pages(case)
    t = {"lens": _ints(g, 0, case["old"], B), "new": _ints(g, (L + 1) // 2, L, B)}
    order = torch.randperm(pages, generator=g, device="cuda").int()
    have = (t["lens"] + page - 1) // page
    used = int(have.sum())
    t["table"] = torch.full((B, cols), -1, dtype=torch.int32, device="cuda")
    t["table"][torch.arange(cols, device="cuda")[None, :] < have[:, None]] = order[:used]
    # the free list of a program that has taken some pages of it already
    t["free"] = torch.cat([order[:2], order[used:]])
    t["from"] = torch.full((1,), 2, dtype=torch.int32, device="cuda")
    if case["short"]:  # fewer pages than tokens ask for
        t["free"] = t["free"][:2 + (len(t["free"]) - 2) // 3].clone()
    for name, w in (("K", case["dk"]), ("V", case["dv"])):
        t[name] = _randn(g, dt, B, L, case["Hkv"], w)
        t[name + "c"] = _randn(g, dt, pages, page, case["Hkv"], w)
    return t


def _paged_inputs(case, seed):
    g = _gen(seed, 3)
    dt, B, Lq, page = _dtype(case), case["B"], case["Lq"], case["page"]
    cols, pages = _pages(case)
    t = {"lens": _ints(g, case["lo"], case["hi"], B), "q_lens": None}
    t["Q"] = _randn(g, torch.float32, B, Lq, case["Hq"], case["dk"]).mul_(1.5).to(dt)
    t["Kc"] = _randn(g, dt, pages, page, case["Hkv"], case["dk"])
    t["Vc"] = _randn(g, dt, pages, page, case["Hkv"], case["dv"])
    order = torch.randperm(pages, generator=g, device="cuda").int()[:B * cols].view(B, cols)
    filled = torch.arange(cols, device="cuda")[None, :] * page < t["lens"][:, None]
    t["table"] = torch.where(filled, order, -1).int()
    if case["ragged"]:  # some requests have fewer drafted tokens
        t["q_lens"] = _ints(g, 1, Lq, B)
    return t


def _verify_inputs(case, seed):
    g = _gen(seed, 4)
    B, K, M, dt = case["B"], case["K"], case["M"], _dtype(case)
    # scores as a trained model gives them, a normal bulk and some entries that stand out; the drafting model is close to it
    z = torch.randn((B, K + 1, M), generator=g, device="cuda") * 2.0
    z.scatter_add_(2, torch.randint(0, M, (B, K + 1, 8), generator=g, device="cuda"),
                   8.0 * torch.rand((B, K + 1, 8), generator=g, device="cuda"))
    P = torch.softmax(z, dim=2).to(dt)
    z = z[:, :K] + 0.5 * torch.randn((B, K, M), generator=g, device="cuda")
    t = {"P": P, "D": None, "draft_lens": None}
    if case["given"]:
        t["D"] = torch.softmax(z, dim=2).to(dt)
        z -= torch.log(-torch.log(torch.rand(z.shape, generator=g, device="cuda").clamp_(1e-30, 1 - 1e-7)))
    t["drafts"] = z.argmax(dim=2).int()
    t["U"] = torch.rand((B, K + 1), generator=g, device="cuda")
    if case["ragged"]:
        t["draft_lens"] = _ints(g, 0, K, B)
    return t


def _inputs(case, seed):
    if case["kind"] == "append":
        return _append_inputs(case, seed)
    if case["kind"] == "paged":
        return _paged_inputs(case, seed)
    if case["kind"] == "verify":
        return _verify_inputs(case, seed)
    g = _gen(seed, 1)
    dt = _dtype(case)
    B, Lq, Hq, Hkv, dk, dv = (case[k] for k in ("B", "Lq", "Hq", "Hkv", "dk", "dv"))
    Lk = Lq + case["start"]
    t = {"Q": _randn(g, torch.float32, B, Lq, Hq, dk).mul_(1.5).to(dt), "K": _randn(g, dt, B, Lk, Hkv, dk),
         "V": _randn(g, dt, B, Lk, Hkv, dv), "lens": None, "mask": None}
    if case["mask"] != "none":  # sequences of half the padded length to all of it
        t["lens"] = _ints(g, (Lk + 1) // 2, Lk, B)
    if case["mask"] == "holes":  # and single positions that are not to be read
        t["mask"] = torch.rand((B, Lk), generator=g, device="cuda") < 0.8
    if case["kind"] == "grad":
        t["dO"] = _randn(g, dt, B, Lq, Hq, dv)
    return t


def _scale(case):
    return 1.0 / math.sqrt(case["dk"])


def prepare(case, seed):
    state = {"case": case, **_inputs(case, seed)}
    if case["kind"] == "grad":  # the forward pass' results
        state["O"], state["lse"] = _attend(state["Q"], state["K"], state["V"], _window_valid(state, case), case)
    return state


# --------------------------------------------------------------------------- plain forms
def _visible(pos, keys, window, sinks):
    """Which keys (their positions) a query at a position sees."""
    ok = keys <= pos
    return ok & ((keys > pos - window) | (keys < sinks)) if window else ok


def _window_valid(t, case):
    """B x 1 x Lq x Lk truth values."""
    Lk = case["Lq"] + case["start"]
    keys = torch.arange(Lk, device="cuda")
    pos = torch.arange(case["start"], Lk, device="cuda")
    ok = _visible(pos[:, None], keys[None, :], case["window"], case["sinks"])[None]
    if t["lens"] is not None:
        ok = ok & (keys < t["lens"][:, None])[:, None, :]
    if t["mask"] is not None:
        ok = ok & t["mask"][:, None, :]
    return ok[:, None]


def _groups(x, Hkv):
    """B x L x Hq x d -> B x Hkv x (Hq / Hkv) L x d, in 32 bits."""
    B, L, Hq, d = x.shape
    return x.float().view(B, L, Hkv, Hq // Hkv, d).permute(0, 2, 3, 1, 4).reshape(B, Hkv, Hq // Hkv * L, d)


def _ungroup(x, Hq, L):
    """The way back."""
    B, Hkv, _, d = x.shape
    return x.view(B, Hkv, Hq // Hkv, L, d).permute(0, 3, 1, 2, 4).reshape(B, L, Hq, d)


def _masked(s, ok, case, fill):
    """s (B x Hkv x G Lq x Lk), `fill` where the B x 1 x Lq x Lk truth values are false."""
    B, Hkv, R, Lk = s.shape
    v = s.view(B, Hkv, R // case["Lq"], case["Lq"], Lk)
    return torch.where(ok[:, :, None], v, fill).view(B, Hkv, R, Lk)


def _logits(Q, K, ok, case):
    return _masked(torch.matmul(_groups(Q, case["Hkv"]), K.float().permute(0, 2, 3, 1)) * _scale(case), ok, case, -math.inf)


def _read(x, ok):
    """B x Lk x Hkv x d keys or values -> B x Hkv x Lk x d in 32 bits, zero where no row reads them."""
    return torch.where(ok.any(dim=2)[:, :, :, None], x.float().permute(0, 2, 1, 3), 0.0)


def _attend(Q, K, V, ok, case):
    s = _logits(Q, K, ok, case)
    m = s.amax(dim=-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    p = torch.exp(s - m)
    del s
    l = p.sum(dim=-1, keepdim=True)
    o = torch.matmul(p, _read(V, ok)) / torch.where(l == 0, 1.0, l)
    o = _ungroup(o, case["Hq"], case["Lq"]).to(_dtype(case))
    return o, (m + torch.log(l)).view(case["B"], case["Hq"], case["Lq"])


def _grad(t, case):
    ok = _window_valid(t, case)
    s = _logits(t["Q"], t["K"], ok, case)
    lse = t["lse"].view(case["B"], case["Hkv"], -1, 1)
    p = torch.exp(s - torch.where(lse == -math.inf, 0.0, lse))
    del s
    do, q = _groups(t["dO"], case["Hkv"]), _groups(t["Q"], case["Hkv"])
    k, v = _read(t["K"], ok), _read(t["V"], ok)
    dv = torch.matmul(p.transpose(2, 3), do)
    dp = torch.matmul(do, v.transpose(2, 3))
    ds = p * (dp - (p * dp).sum(dim=-1, keepdim=True)) * _scale(case)
    del p, dp
    dq = _ungroup(torch.matmul(ds, k), case["Hq"], case["Lq"])
    dk = torch.matmul(ds.transpose(2, 3), q)
    dt = _dtype(case)
    return {"dQ": dq.to(dt), "dK": dk.permute(0, 2, 1, 3).to(dt), "dV": dv.permute(0, 2, 1, 3).to(dt)}


def _append(t, case):
    page, (B, cols) = case["page"], t["table"].shape
    lens, new, table = t["lens"], t["new"], t["table"]
    end = torch.minimum(lens + new, torch.full_like(lens, cols * page))
    have, want = (lens + page - 1) // page, (end + page - 1) // page
    need = want - have
    first = t["from"] + torch.cumsum(need, dim=0) - need
    got = torch.minimum((len(t["free"]) - first).clamp(min=0), need)
    col = torch.arange(cols, device="cuda")[None, :]
    at = first[:, None] + col - have[:, None]
    page_id = torch.where(col < (have + got)[:, None], t["free"][at.clamp(0, len(t["free"]) - 1).long()], -1)
    table.copy_(torch.where((col >= have[:, None]) & (col < want[:, None]), page_id, table))
    end = torch.minimum(end, (have + got) * page)
    pos = lens[:, None] + torch.arange(case["Lnew"], device="cuda")[None, :]
    entry = torch.gather(table, 1, (pos // page).clamp(max=cols - 1).long())
    ok = (pos < end[:, None]) & (entry >= 0)
    slots = torch.where(ok, entry * page + pos % page, -1).int()
    for name in ("K", "V"):
        cache = t[name + "c"]
        cache.view(-1, *cache.shape[2:])[slots[ok].long()] = t[name][ok]
    return {"table": table, "slots": slots, "lens": end, "taken": need.sum().int().view(1), "K": t["Kc"], "V": t["Vc"]}


def _paged(t, case):
    B, Lq = case["B"], case["Lq"]
    cols, _ = _pages(case)
    entry = t["table"].clamp(min=0).long()
    K, V = (t[n][entry].view(B, cols * case["page"], case["Hkv"], -1) for n in ("Kc", "Vc"))
    keys = torch.arange(cols * case["page"], device="cuda")
    i = torch.arange(Lq, device="cuda")[None, :]
    q = t["q_lens"] if t["q_lens"] is not None else torch.full_like(t["lens"], Lq)
    pos = torch.where(i < q[:, None], t["lens"][:, None] - q[:, None] + i, -1)
    ok = _visible(pos[:, :, None], keys, case["window"], case["sinks"])[:, None]
    return {"O": _attend(t["Q"], K, V, ok, case)[0]}


def _verify(t, case):
    """In 64 bits, as the running sums of many small weights end next to the drawn number."""
    P, D, x, U = t["P"], t["D"], t["drafts"].long(), t["U"].double()
    B, K = x.shape
    n = t["draft_lens"].long() if t["draft_lens"] is not None else torch.full((B,), K, device="cuda")
    p = torch.gather(P[:, :K], 2, x[:, :, None])[:, :, 0].double()
    d = torch.gather(D, 2, x[:, :, None])[:, :, 0].double() if D is not None else torch.ones_like(p)
    i = torch.arange(K, device="cuda")[None, :]
    accept = (U[:, :K] * d < p) & (i < n[:, None])
    a = torch.cumprod(accept.int(), dim=1).sum(dim=1)
    b = torch.arange(B, device="cuda")
    target = P[b, a].double()
    at = a.clamp(max=K - 1)
    if D is not None:
        other = D[b, at].double()
    else:
        other = torch.zeros_like(target).scatter_(1, x[b, at][:, None], 1.0)
    rest = (target - torch.where((a < n)[:, None], other, 0.0)).clamp(min=0)
    w = torch.where(rest.sum(dim=1, keepdim=True) > 0, rest, target)
    run = torch.cumsum(w, dim=1)
    drawn = (run <= U[:, K:] * run[:, -1:]).sum(dim=1, keepdim=True)
    i = torch.arange(K + 1, device="cuda")[None, :]
    tokens = torch.where(i < a[:, None], torch.cat([x, drawn], dim=1), torch.where(i == a[:, None], drawn, -1))
    return {"accepted": a.int(), "tokens": tokens.int()}


def run(state):
    c = state["case"]
    if own:
        from paper_2608_01528_gb300 import gramspace as gs

        if c["kind"] == "append":
            out = gs.page_slots(state["lens"], state["new"], state["table"], state["free"], c["page"], c["Lnew"],
                                state["Kc"].shape[0], free_from=state["from"])
            gs.page_store(state["K"], state["V"], out["slots"], state["Kc"], state["Vc"])
            return {"table": state["table"], "slots": out["slots"], "lens": out["lens"].long(), "taken": out["taken"],
                    "K": state["Kc"], "V": state["Vc"]}  # (lengths in 64 bits, as the plain form has them)
        if c["kind"] == "paged":
            return gs.paged_attention(state["Q"], state["Kc"], state["Vc"], state["table"], state["lens"], _scale(c),
                                      q_lens=state["q_lens"], window=c["window"] or None, sinks=c["sinks"])
        if c["kind"] == "verify":
            return gs.verify_drafts(state["P"], state["D"], state["drafts"], state["U"], draft_lens=state["draft_lens"])
        if c["kind"] == "window":
            return gs.window_attention(state["Q"], state["K"], state["V"], c["window"], c["sinks"], c["start"], _scale(c),
                                       key_lens=state["lens"], key_mask=state["mask"], want_lse=c["lse"])
        return gs.window_attention_backward(state["Q"], state["K"], state["V"], state["O"], state["lse"], state["dO"],
                                            c["window"], c["sinks"], c["start"], _scale(c), key_lens=state["lens"],
                                            key_mask=state["mask"])
    if c["kind"] == "append":
        return _append(state, c)
    if c["kind"] == "paged":
        return _paged(state, c)
    if c["kind"] == "verify":
        return _verify(state, c)
    if c["kind"] == "grad":
        return _grad(state, c)
    o, lse = _attend(state["Q"], state["K"], state["V"], _window_valid(state, c), c)
    return {"O": o, "lse": lse} if c["lse"] else {"O": o}


# --------------------------------------------------------------------------- work
def _pairs(case):
    """Pairs of a query and a key that it sees, a sequence of the full length, and the keys that some query sees."""
    Lq, s = case["Lq"], case["start"]
    w = min(case["window"], s + Lq)
    n = min(w + case["sinks"], s + Lq)
    pairs = sum(min(s + i + 1, n) for i in range(Lq))
    return float(pairs), float(min(s + Lq, w + Lq - 1 + case["sinks"]))


def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    B = float(case["B"])
    if case["kind"] == "verify":
        # one row of P, and one of D where a draft was rejected
        rows = 1 + (1 - 0.8 ** case["K"] if case["given"] else 0)
        return {"bytes": B * case["M"] * e * rows + B * (8 * case["K"] + 8), "flops": 4 * B * case["M"]}
    if case["kind"] == "append":
        tokens = B * 0.75 * case["Lnew"] if case["Lnew"] > 1 else B
        row = case["Hkv"] * (case["dk"] + case["dv"]) * e
        return {"bytes": 2 * tokens * row + 4 * B * case["Lnew"] + 8 * tokens / case["page"] + 12 * B, "flops": 0}
    Hq, Hkv, dk, dv, Lq = (float(case[k]) for k in ("Hq", "Hkv", "dk", "dv", "Lq"))
    if case["kind"] == "paged":
        keys = (case["lo"] + case["hi"]) / 2.0
        if case["window"]:
            keys = min(keys, case["window"] + Lq - 1 + case["sinks"])
        q = Lq * (0.5 + 0.5 / Lq if case["ragged"] else 1.0)
        return {"bytes": e * B * (keys * Hkv + q * Hq) * (dk + dv) + 4 * B * keys / case["page"],
                "flops": 2 * B * q * Hq * keys * (dk + dv)}
    read = 1.0 if case["mask"] == "none" else 0.75  # the mean length of padded sequences
    pairs, keys = _pairs(case)
    Lk = Lq + case["start"]
    q, kv = B * Lq * Hq, B * keys * read * Hkv
    bits = 0 if case["mask"] != "holes" else B * keys * read
    if case["kind"] == "window":
        return {"bytes": e * (q + kv) * (dk + dv) + bits + (4 * q if case["lse"] else 0),
                "flops": 2 * B * Hq * pairs * read * (dk + dv)}
    return {"bytes": e * (q * (2 * dk + 2 * dv) + (kv + B * Lk * Hkv) * (dk + dv)) + 4 * q + bits,
            "flops": 2 * B * Hq * pairs * read * (3 * dk + 2 * dv)}


# --------------------------------------------------------------------------- 64 bits
def _zeros(*shape):
    return torch.zeros(shape, dtype=torch.float64, device="cuda")


def _exact_append(t, case):
    page = case["page"]
    table, free = t["table"].tolist(), t["free"].tolist()
    cols = len(table[0])
    nxt, start = int(t["from"]), int(t["from"])
    slots, lens = [], []
    for row, old, new in zip(table, t["lens"].tolist(), t["new"].tolist()):
        have = -(-old // page)
        stop = -(-min(old + new, cols * page) // page)
        for c in range(have, stop):
            row[c] = free[nxt] if nxt < len(free) else -1
            nxt += 1
        mine, end = [], old
        for j in range(old, old + case["Lnew"]):
            inside = j < old + new and j < cols * page and row[j // page] >= 0
            mine.append(row[j // page] * page + j % page if inside else -1)
            end = j + 1 if inside else end
        slots.append(mine)
        lens.append(end)
    return {"table": torch.tensor(table, dtype=torch.int32), "slots": torch.tensor(slots, dtype=torch.int32),
            "lens": torch.tensor(lens, dtype=torch.int32), "taken": torch.tensor([nxt - start], dtype=torch.int32),
            "K": None, "V": None}


def _exact_paged(t, case):
    B, Lq, Hq, Hkv, dv = (case[k] for k in ("B", "Lq", "Hq", "Hkv", "dv"))
    G = Hq // Hkv
    O = _zeros(B, Lq, Hq, dv)
    lens = t["lens"].tolist()
    q_lens = t["q_lens"].tolist() if t["q_lens"] is not None else [Lq] * B
    for b in range(B):
        n = lens[b]
        j = torch.arange(n, device="cuda")
        page = t["table"][b, j // case["page"]].long()
        rows = [(i, n - q_lens[b] + i) for i in range(q_lens[b]) if n - q_lens[b] + i >= 0]
        if not rows:
            continue
        first = max(0, rows[0][1] - case["window"] + 1) if case["window"] else 0
        sel = torch.where((j >= first) | (j < case["sinks"]))[0]
        k, v = (t[name][page[sel], sel % case["page"]].double() for name in ("Kc", "Vc"))
        for i, p in rows:
            see = sel <= p
            if case["window"]:
                see &= (sel >= p - case["window"] + 1) | (sel < case["sinks"])
            q = t["Q"][b, i].double().view(Hkv, G, -1)
            s = torch.einsum("hgd,jhd->hgj", q, k).mul_(_scale(case))
            s[:, :, ~see] = -math.inf
            O[b, i] = torch.einsum("hgj,jhd->hgd", torch.softmax(s, dim=2), v).reshape(Hq, dv)
    return {"O": O}


def _exact_verify(t, case):
    K = case["K"]
    accepted, tokens = [], []
    n = t["draft_lens"].tolist() if t["draft_lens"] is not None else [K] * case["B"]
    U, drafts = t["U"].double().tolist(), t["drafts"].tolist()
    for b in range(case["B"]):
        a, row = 0, None
        while a < n[b]:
            x = drafts[b][a]
            if U[b][a] * (float(t["D"][b, a, x]) if t["D"] is not None else 1.0) < float(t["P"][b, a, x]):
                a += 1
                continue
            row = t["P"][b, a].double().cpu()
            if t["D"] is not None:
                row = row - t["D"][b, a].double().cpu()
            else:
                row[x] -= 1.0
            row.clamp_(min=0)
            break
        if row is None or not float(row.sum()) > 0:
            row = t["P"][b, a].double().cpu()
        cum = row.cumsum(0)
        i = int(torch.searchsorted(cum, torch.tensor(U[b][K] * float(cum[-1]), dtype=torch.float64), right=True))
        accepted.append(a)
        tokens.append(drafts[b][:a] + [i] + [-1] * (K - a))
    return {"accepted": torch.tensor(accepted, dtype=torch.int32), "tokens": torch.tensor(tokens, dtype=torch.int32)}


def exact(case, seed):
    t = _inputs(case, seed)
    if case["kind"] == "append":
        return _exact_append(t, case)
    if case["kind"] == "paged":
        return _exact_paged(t, case)
    if case["kind"] == "verify":
        return _exact_verify(t, case)
    B, Lq, Hq, Hkv, dk, dv = (case[k] for k in ("B", "Lq", "Hq", "Hkv", "dk", "dv"))
    Lk = Lq + case["start"]
    O, lse = _zeros(B, Lq, Hq, dv), _zeros(B, Hq, Lq) - math.inf
    dQ, dK, dV = _zeros(B, Lq, Hq, dk), _zeros(B, Lk, Hkv, dk), _zeros(B, Lk, Hkv, dv)
    back = torch.arange(case["start"], Lk, device="cuda")[:, None] - torch.arange(Lk, device="cuda")[None, :]
    near = (back >= 0) & ((back < case["window"]) | (torch.arange(Lk, device="cuda") < case["sinks"]))
    for b in range(B):
        see = near.clone()
        if t["lens"] is not None:
            see[:, int(t["lens"][b]):] = False
        if t["mask"] is not None:
            see &= t["mask"][b]
        some = see.any(dim=1)
        for h in range(Hq):
            hk = h // (Hq // Hkv)
            q, k, v = t["Q"][b, :, h].double(), t["K"][b, :, hk].double(), t["V"][b, :, hk].double()
            s = (q @ k.T).mul_(_scale(case)).masked_fill_(~see, -math.inf)
            lse[b, h] = torch.logsumexp(s, dim=1)
            p = s.sub_(torch.where(some, lse[b, h], 0.0)[:, None]).exp_()
            O[b, :, h] = p @ v
            if case["kind"] == "grad":
                do = t["dO"][b, :, h].double()
                dV[b, :, hk] += p.T @ do
                ds = (do @ v.T).sub_((do * O[b, :, h]).sum(1, keepdim=True)).mul_(p).mul_(_scale(case))
                dQ[b, :, h] = ds @ k
                dK[b, :, hk] += ds.T @ q
    if case["kind"] == "grad":
        return {"dQ": dQ, "dK": dK, "dV": dV}
    return {"O": O, "lse": lse} if case["lse"] else {"O": O}
