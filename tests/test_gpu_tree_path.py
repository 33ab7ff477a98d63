"""tree_path against its definition."""
import numpy as np
import pytest
import torch

from paper_2603_11243_amd.binding import Context
from trees import accepted, cu, flat, tree

pytestmark = pytest.mark.gpu


def _check(trees, logp, tau, ctx=None):
    N = sum(len(t) for t in trees)
    if ctx is None:
        ctx = Context(device="cuda:0")
        ctx.reserve(tree_nodes=N, tree_utts=len(trees))
    got = ctx.tree_path(torch.from_numpy(logp).cuda(), cu(trees), flat(trees), tau)
    got = {k: v.cpu().numpy() for k, v in got.items()}
    at = cu(trees)
    for b, t in enumerate(trees):
        want = accepted(t, logp[at[b]:at[b + 1]], tau)
        assert got["accept_len"][b] == len(want)
        assert got["accept_node"][b] == (want[-1] if want else -1)
        assert got["path"][at[b]:at[b + 1]].tolist() == want + [-1] * (len(t) - len(want))


@pytest.mark.parametrize("shape", ["random", "chain", "star", "roots"])
@pytest.mark.parametrize("most", [1, 2, 63, 64, 65, 200, 256, 257, 1024])
def test_trees(shape, most):
    r = np.random.default_rng(most)
    trees = [tree(r, n, shape) for n in [most, 0, 1, most // 2, max(1, most - 1)]]
    logp = np.where(r.random(sum(map(len, trees))) < 0.93, -0.2, -4.0).astype(np.float32)
    _check(trees, logp, 0.1)


def test_thresholds():
    """Strictly above ln tau in fp32; tau <= 0 accepts everything; NaN does not pass."""
    edge = np.float32(np.log(np.float64(np.float32(0.2))))
    up, down = np.nextafter(edge, np.float32(0)), np.nextafter(edge, np.float32(-9))
    trees = [[-1, 0, 0, 1, 2], [-1, -1, 1]]
    logp = np.array([up, edge, up, 0, down, np.nan, up, -np.inf], dtype=np.float32)
    for tau in (0.2, 0.0, -1.0, 1.0, 5.0):
        _check(trees, logp, tau)
    _check(trees, np.full(8, -np.inf, dtype=np.float32), 0.0)


def test_many_trees_and_captured_calls():
    r = np.random.default_rng(3)
    trees = [tree(r, int(n), "random") for n in r.integers(0, 400, size=300)]
    logp = np.where(r.random(sum(map(len, trees))) < 0.95, -0.2, -4.0).astype(np.float32)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        ctx = Context(device="cuda:0", stream=s)
        ctx.reserve(tree_nodes=len(logp), tree_utts=len(trees))
        _check(trees, logp, 0.1, ctx)
        x = torch.from_numpy(logp).cuda()
        want = {k: v.clone() for k, v in ctx.tree_path(x, cu(trees), flat(trees), 0.1).items()}
        out = {k: torch.empty_like(v) for k, v in want.items()}
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            ctx.tree_path(x, cu(trees), flat(trees), 0.1, out=out)
        for _ in range(3):
            for v in out.values():
                v.fill_(7)
            ctx.tree_path(x, cu(trees[::-1]), flat(trees[::-1]), 0.1)
            s.synchronize()
            graph.replay()
            s.synchronize()
            assert all(torch.equal(out[k], want[k]) for k in want)
