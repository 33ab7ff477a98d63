"""Workspaces that reserve allocated stay while the context lives, since captured calls use them at every replay; a caller's own are the caller's."""
import gc
import weakref

import pytest
import torch

from paper_2603_11243_amd import binding


class _Lib:
    """The library's part in reserve, without a GPU."""

    def __init__(self):
        self.bytes, self.set = 0, []

    def ssd_workspace_bytes(self, h, *sizes):
        return self.bytes

    def ssd_set_workspace(self, h, p, n):
        self.set.append(n)
        return 0

    def ssd_destroy(self, h):
        pass


def _context(monkeypatch):
    monkeypatch.setattr(binding, "_ptr", lambda t: None if t is None else t.data_ptr())
    c = binding.Context.__new__(binding.Context)
    c._lib, c._h, c.device, c._ws, c._reserved = _Lib(), 1, torch.device("cpu"), None, []
    return c


def test_replaced_workspaces_live_as_long_as_the_context(monkeypatch):
    c = _context(monkeypatch)
    alive = []
    for c._lib.bytes in (1000, 3000, 2000, 3001):
        c.reserve()
        alive.append(weakref.ref(c._ws))
    assert c._lib.set == [1000, 3000, 3750]                  # one a quarter larger at least
    own = [torch.empty(10, dtype=torch.uint8) for _ in range(2)]
    gone = [weakref.ref(t) for t in own]
    for t in own + own + [None]:
        c.set_workspace(t)
    del own, t
    gc.collect()
    assert all(w() is not None for w in alive) and all(w() is None for w in gone)
    c._lib.bytes = 100
    c.reserve()
    assert c._lib.set[-1] == 3750 and c._ws is alive[-1]()      # (the last one is large enough)
    del c
    gc.collect()
    assert all(w() is None for w in alive)


@pytest.mark.gpu
def test_a_captured_call_uses_its_workspace_after_a_larger_one_is_reserved():
    """The pieces of a long context lie in the workspace: memory that torch gives out after the second reserve is not written by a replay."""
    from pages import Pool
    heads, n = (8, 2, 64), 9000
    side = torch.cuda.Stream()
    c = binding.Context(device="cuda:0", stream=side)
    c.reserve(paged_utts=1, paged_ctx=n, paged_heads=heads)
    pool = Pool("f16", heads[1:], [n], 64)
    q, graph = torch.randn(1, 8, 64, device="cuda").half(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        out = torch.empty_like(q)
        pages = pool.pages()
        want = c.paged_attention(q, pages, pool.table, pool.ctx_len)
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            c.paged_attention(q, pages, pool.table, pool.ctx_len, out=out)
        size = c._ws.numel()
        c.reserve(paged_utts=8, paged_ctx=4 * n, paged_heads=heads)
        assert c._ws.numel() > size
        others = [torch.zeros(size, dtype=torch.uint8, device="cuda") for _ in range(4)]
        for _ in range(3):
            out.zero_()
            graph.replay()
            again = c.paged_attention(q, pages, pool.table, pool.ctx_len)
            side.synchronize()
            assert torch.equal(out, want) and torch.equal(again, want) and not any(t.any() for t in others)
    c.close()
