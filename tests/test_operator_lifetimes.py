"""Arguments that nobody else holds live until the library has been called."""
import gc
import weakref

import torch


class Fake(torch.Tensor):  # a host tensor that says it is a CUDA one: the call goes as far as the library
    is_cuda = True


class Library:
    def __init__(self):
        self.refs, self.calls = {}, []

    def workspace(self, a, backward, n):
        n._obj.value = 64
        return 0

    def call(self, name):
        gc.collect()
        self.calls.append(name)
        dead = [k for k, r in self.refs.items() if r() is None]
        assert not dead, f"{name}: freed before the call: {dead}"
        return 0

    gs_cross_attention_workspace = workspace

    def gs_cross_attention(self, *args):
        return self.call("gs_cross_attention")

    def gs_cross_attention_backward(self, *args):
        return self.call("gs_cross_attention_backward")

    def gs_sample_scores(self, *args):
        return self.call("gs_sample_scores")


def test_temporaries_outlive_their_call(monkeypatch):
    """An lse that was an expression of the call (lse.float(), lse.contiguous()) was freed before the kernels were
    launched, and the gradients or the workspace took its memory."""
    from paper_2608_01528_gb300 import gramspace as g
    lib = Library()
    monkeypatch.setattr(g, "load_library", lambda: lib)
    monkeypatch.setattr(g, "_on_stream", lambda *a: g._STAY)
    monkeypatch.setattr(g, "_stream", lambda *a: 0)

    def temporary(name, *shape, dtype=torch.float32):
        t = torch.zeros(*shape, dtype=dtype).as_subclass(Fake)
        lib.refs[name] = weakref.ref(t)
        return t

    q, k, v = (2, 5, 4, 8), (2, 7, 2, 8), (2, 7, 2, 6)

    def masks():
        return {"key_lens": temporary("key_lens", 2, dtype=torch.int32), "key_mask": temporary("key_mask", 2, 7, dtype=torch.bool)}

    g.cross_attention(temporary("Q", *q), temporary("K", *k), temporary("V", *v), **masks(),
                      out={"O": temporary("O", 2, 5, 4, 6), "lse": temporary("lse", 2, 4, 5)})
    lib.refs.clear()
    g.cross_attention_backward(temporary("Q", *q), temporary("K", *k), temporary("V", *v), temporary("O", 2, 5, 4, 6),
                               temporary("lse", 2, 4, 5), temporary("dO", 2, 5, 4, 6), **masks(),
                               out={"dQ": temporary("dQ", *q), "dK": temporary("dK", *k), "dV": temporary("dV", *v)})
    lib.refs.clear()
    row = {n: temporary(n, 3) for n in ("temperature", "top_p", "min_p")}
    g.sample_scores(temporary("S", 3, 6), temporary("U", 3), top_k=temporary("top_k", 3, dtype=torch.int32), **row,
                    out={"index": temporary("index", 3, dtype=torch.int32), "prob": temporary("prob", 3)})
    assert lib.calls == ["gs_cross_attention", "gs_cross_attention_backward", "gs_sample_scores"]
