"""A free list that ends, step after step, and gets pages again: as the calls' documentation has it, none is skipped or given twice."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("captured", [False, True])
def test_a_shortage_skips_no_page(gs, captured):
    page, cols, pages = 4, 8, 5
    lens = torch.zeros(2, dtype=torch.int32, device="cuda")
    one = torch.ones(2, dtype=torch.int32, device="cuda")
    table = torch.full((2, cols), -1, dtype=torch.int32, device="cuda")
    free = torch.tensor([3, 0, 4, 1, 2], dtype=torch.int32, device="cuda")
    used = torch.zeros(1, dtype=torch.int32, device="cuda")

    def step():
        s = gs.page_slots(lens, one, table, free, page, 1, pages, free_from=used)
        lens.copy_(s["lens"])
        used.add_(s["taken"]).clamp_(max=free.numel())
        return s["slots"]

    if captured:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            slots = step()

        def run():
            graph.replay()
            return slots.flatten().tolist()
    else:
        def run():
            return step().flatten().tolist()

    for i in range(8):
        got = run()
        assert min(got) >= 0 and lens.tolist() == [i + 1] * 2
    for i in range(4):  # one page is left: the first request's; the second asks again and again
        got = run()
        assert got[0] == 2 * page + i and got[1] == -1
        assert lens.tolist() == [9 + i, 8] and used.tolist() == [5]
    assert table[:, :3].tolist() == [[3, 4, 2], [0, 1, -1]]
    # the first request ends, its pages go back to the list
    used -= 3
    free[2:5] = table[0, :3]
    table[0], lens[0] = -1, 0
    seen = []
    for i in range(4):
        got = run()
        assert min(got) >= 0 and lens.tolist() == [1 + i, 9 + i]
        seen += got
    assert table[:, :3].tolist() == [[3, -1, -1], [0, 1, 4]] and used.tolist() == [4]
    assert sorted(seen) == [12, 13, 14, 15, 16, 17, 18, 19]
    gs.stream_status()
