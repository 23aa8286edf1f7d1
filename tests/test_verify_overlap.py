"""verify_drafts refuses outputs that lie on one of its dense inputs or on one another; needs no device."""
from test_operator_args import g  # noqa: F401


def test_overlaps(g):  # noqa: F811
    # 2 requests of 3 drafts: drafts of 24 bytes, draft_lens of 8, U and tokens of 32, accepted of 8
    base = dict(P=0x10000, D=0x20000, dtype=0, B=2, K=3, M=100, pb=400, pr=100, db=300, dr=100, drafts=0x30000, lens=0x40000, U=0x50000,
                accepted=0x60000, tokens=0x70000)

    def call(**kw):
        d = dict(base, **kw)
        return g.load_library().gs_verify_drafts(*(d[k] for k in base), None)

    for name, size in (("drafts", 24), ("lens", 8), ("U", 32)):
        at = base[name]
        for out, own in (("accepted", 8), ("tokens", 32)):
            for p in (at, at + size - 4, at - own + 4):
                assert call(**{out: p}) == g.GS_ERR_INVALID_ARG, (name, out, p - at)
    for p in (0x70000, 0x70000 + 28, 0x70000 - 4):
        assert call(accepted=p) == g.GS_ERR_INVALID_ARG
