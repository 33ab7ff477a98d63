"""tree_attention against 64 bits: lengths, trees, head layouts, strides, rows that must not count, weights, replays."""
import numpy as np
import pytest
import torch

from paper_2603_11243_amd.binding import Context
from trees import cu, flat, sees, tree

pytestmark = pytest.mark.gpu

DTYPE = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
# (query heads, K/V heads, head_dim)
HEADS_16 = [(16, 8, 128), (24, 8, 128), (4, 4, 64), (14, 2, 64), (5, 1, 128)]
HEADS_32 = [(4, 4, 64), (6, 2, 128), (3, 1, 4), (8, 2, 36)]


def _context(N, B, heads):
    ctx = Context(device="cuda:0")
    ctx.reserve(tree_nodes=N, tree_utts=B, tree_heads=heads)
    return ctx


class Call:
    """A batch: contexts of ctx_len rows and trees, their slots in some order with gaps; cache rows of nobody hold NaN."""

    def __init__(self, dtype, heads, ctx_len, trees, seed=0, layout="slots", q_gap=0, scale_q=1.5):
        hq, hkv, hd = heads
        t = DTYPE[dtype]
        g = torch.Generator().manual_seed(seed)
        r = np.random.default_rng(seed)
        self.heads, self.dtype, self.trees, self.ctx_len = heads, t, trees, np.array(ctx_len, dtype=np.int32)
        B = len(trees)
        at, start = 1, np.zeros(B, dtype=np.int32)
        for b in r.permutation(B):
            start[b] = at
            at += ctx_len[b] + len(trees[b]) + int(r.integers(0, 3))
        self.kv_start, self.slots = start, at + 1
        used = torch.zeros(self.slots, dtype=torch.bool)
        for b in range(B):
            used[start[b]:start[b] + ctx_len[b] + len(trees[b])] = True
        self.used = used

        def cache():
            x = torch.randn(self.slots, hkv, hd, generator=g).to(t)
            x[~used] = float("nan")
            if layout == "heads":
                return x.transpose(0, 1).contiguous().cuda().transpose(0, 1)
            if layout == "gaps":                             # rows with something else between them and between heads
                big = torch.full((self.slots, hkv + 1, 2 * hd), float("nan"), dtype=t)
                big[:, :hkv, :hd] = x
                return big.cuda()[:, :hkv, :hd]
            return x.cuda()

        self.k, self.v = cache(), cache()
        N = sum(len(x) for x in trees)
        self.q = torch.full((N, hq * hd + q_gap), float("nan"), dtype=t, device="cuda")
        self.q[:, :hq * hd] = (torch.randn(N, hq * hd, generator=g) * scale_q).to(t).cuda()
        self.q = self.q[:, :hq * hd].unflatten(1, (hq, hd))
        self.mass = torch.rand(hkv, self.slots, generator=g).cuda()
        self.lse = torch.full((N, hq), float("nan"), device="cuda")

    def run(self, ctx=None, mass=True, **more):
        ctx = ctx or _context(len(self.q), len(self.trees), self.heads)
        self.mass_out = self.mass.clone()
        out = ctx.tree_attention(self.q, self.k, self.v, self.kv_start, self.ctx_len, cu(self.trees), flat(self.trees), lse=self.lse,
                                 mass=self.mass_out if mass else None, **more)
        torch.cuda.synchronize()
        return out

    def exact(self, scale=None):
        """out, its error bound, lse, its bound, mass, its bound; all in 64 bits.
        u: half a step of the type.  A score is hd products added in fp32: off by at most (hd + 4) 2^-24 sum |q k| scale =: d (scaling and the
        factor to base 2 among the 4).  A probability: 2 d (its own score and the sum), rounded once to the type for the second product (u;
        of IEEE half nothing smaller than 2^-31 of the largest is left).  The sums over n keys in fp32: n 2^-24 of what is added; the joining of
        parts and the exponential a few more.  The output is rounded once."""
        hq, hkv, hd = self.heads
        scale = hd ** -0.5 if scale is None else scale
        f32 = self.dtype == torch.float32
        u = torch.finfo(self.dtype).eps / 2
        q, k, v = self.q.double().cpu().numpy(), self.k.double().cpu().numpy(), self.v.double().cpu().numpy()
        out, tol = np.zeros_like(q), np.zeros_like(q)
        lse, lse_tol = np.zeros(q.shape[:2]), np.zeros(q.shape[:2])
        mass = self.mass.double().cpu().numpy()
        mass_tol = np.zeros_like(mass)
        node0 = cu(self.trees)
        for b, t in enumerate(self.trees):
            n, N, s0 = int(self.ctx_len[b]), len(t), int(self.kv_start[b])
            seen = np.concatenate([np.ones((N, n), bool), sees(t)], 1)
            mass[:, s0 + n:s0 + n + N] = 0
            for h in range(hq):
                kv = h * hkv // hq
                kk, vv, qq = k[s0:s0 + n + N, kv], v[s0:s0 + n + N, kv], q[node0[b]:node0[b] + N, h]
                kk, vv = np.where(np.isfinite(kk), kk, 0), np.where(np.isfinite(vv), vv, 0)     # what is not finite is seen by nobody here
                s = np.where(seen, qq @ kk.T * scale, -np.inf)
                d = ((hd + 4) * 2.0 ** -24 * abs(scale) * (abs(qq) @ abs(kk).T) * seen).max(1, initial=0)[:, None] + 2.0 ** -22
                top = s.max(1, keepdims=True, initial=-np.inf)
                p = np.exp(s - top)
                l = p.sum(1, keepdims=True)
                p /= l
                at = slice(node0[b], node0[b] + N), h
                out[at] = p @ vv
                mag = p @ abs(vv)
                low = 0 if f32 else 2.0 ** -31 * (seen @ abs(vv)) / l
                tol[at] = u * abs(out[at]) + ((0 if f32 else u) + 2 * d + (n + N + 32) * 2.0 ** -24) * mag + low
                lse[at] = (top + np.log(l))[:, 0]
                lse_tol[at] = d[:, 0] + (n + N + 32) * 2.0 ** -24 + 2.0 ** -22 * abs(lse[at])
                mass[kv, s0:s0 + n + N] += p.sum(0)
                mass_tol[kv, s0:s0 + n + N] += ((2 * d + (n + N + 32) * 2.0 ** -24 + 2.0 ** -22 * abs(lse[at])[:, None]) * p).sum(0)
            mass_tol[:, s0:s0 + n + N] += (N * hq // hkv + 2) * 2.0 ** -24 * mass[:, s0:s0 + n + N]
        return out, tol, lse, lse_tol, mass, mass_tol

    def check(self, ctx=None, mass=True, **more):
        got = self.run(ctx, mass, **more).double().cpu().numpy()
        out, tol, lse, lse_tol, m, m_tol = self.exact(more.get("scale"))
        assert np.isfinite(got).all()
        assert (abs(got - out) <= tol).all(), (abs(got - out) / tol).max()
        assert (abs(self.lse.double().cpu().numpy() - lse) <= lse_tol).all()
        if mass:
            got_m = self.mass_out.double().cpu().numpy()
            used = self.used.numpy()
            assert np.array_equal(got_m[:, ~used], m[:, ~used])                  # slots of nobody are left alone
            assert (abs(got_m - m) <= m_tol)[:, used].all()


def _batch(seed, ctx_len, nodes, shapes=("random", "chain", "star", "roots")):
    r = np.random.default_rng(seed)
    return [tree(r, n, shapes[i % len(shapes)]) for i, n in enumerate(nodes)]


ALL = [(d, h) for d in ("f16", "bf16") for h in HEADS_16] + [("f32", h) for h in HEADS_32]


@pytest.mark.parametrize("dtype, heads", ALL)
def test_ragged_batches(dtype, heads):
    ctx_len = [0, 1, 5, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 0, 300]
    nodes = [1, 1, 2, 3, 7, 8, 9, 16, 17, 31, 33, 0, 5, 12, 1, 40, 70, 21]
    Call(dtype, heads, ctx_len, _batch(1, ctx_len, nodes), seed=2).check()


@pytest.mark.parametrize("dtype, heads", ALL)
@pytest.mark.parametrize("nodes", [1, 6, 20])
def test_long_contexts_that_are_cut_and_joined(dtype, heads, nodes):
    Call(dtype, heads, [5003, 17], _batch(3, None, [nodes, 2]), seed=4).check()


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("shape", ["chain", "random", "star"])
def test_largest_trees(dtype, shape):
    r = np.random.default_rng(5)
    heads = (2, 1, 128) if dtype != "f32" else (2, 1, 64)
    Call(dtype, heads, [70, 3], [tree(r, 1024, shape), tree(r, 333, shape)], seed=6).check()


@pytest.mark.parametrize("dtype, heads", [("f16", (16, 8, 128)), ("bf16", (8, 2, 64)), ("f32", (4, 2, 36))])
@pytest.mark.parametrize("layout", ["slots", "heads", "gaps"])
def test_strides(dtype, heads, layout):
    Call(dtype, heads, [40, 150, 1], _batch(7, None, [9, 20, 3]), seed=8, layout=layout, q_gap=32).check()


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
def test_one_token_of_one_utterance(dtype):
    for n in (0, 1, 2, 106, 257):
        Call(dtype, (16, 8, 128) if dtype != "f32" else (4, 4, 64), [n], [[-1]], seed=n).check()


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
def test_scale(dtype):
    c = Call(dtype, (4, 2, 64), [100, 40], _batch(9, None, [8, 18]), seed=10)
    c.check(scale=-0.37)
    c.check(scale=0.0)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_rows_that_are_not_seen_may_hold_anything(dtype, bad):
    """Two branches: whatever one holds, the other's nodes do not notice."""
    parent = [-1, 0, 1, 2, 0, 4, 5, -1]
    c = Call(dtype, (4, 2, 64), [33], [parent], seed=11)
    left, right = [1, 2, 3], [0, 4, 5, 6, 7]
    c.check()
    at = int(c.kv_start[0]) + 33 + torch.tensor(left)
    c.k[at], c.v[at] = bad, bad
    got = c.run(mass=False).double().cpu().numpy()
    out, tol, *_ = c.exact()
    assert (abs(got - out) <= tol)[right].all()
    assert not np.isfinite(got[left]).any()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_values_of_every_size(dtype):
    """Scores far apart (a later key beats all before it by more than the range of the type) and values near the end of the range."""
    c = Call(dtype, (4, 2, 128), [700, 90], _batch(12, None, [5, 40]), seed=13, scale_q=1.0)
    c.k[:] = (c.k.float() * torch.linspace(0.1, 12, c.slots, device="cuda")[:, None, None]).to(c.dtype)
    c.v[:] = (c.v.float().clamp(-3, 3) * (10000.0 if dtype == "f16" else 2.0 ** 100)).to(c.dtype)
    c.check()


def test_one_weight_of_one_and_many_small_ones():
    """A key with the value 0, and 4095 whose probabilities are 2^-20 of its own: each is rounded, none is lost."""
    c = Call("f16", (2, 1, 128), [4095], [[-1]], seed=14)
    c.q.zero_()
    c.q[..., 0] = 1.0
    c.k.zero_()
    c.v[:] = 1024.0
    first = int(c.kv_start[0])
    c.k[first, 0, 0], c.v[first] = 20.0 * np.log(2.0) / 1.0, 0.0
    c.check(scale=1.0)


def test_contexts_beyond_four_gib():
    """64 K/V heads: 16 KB a row, 2^18 rows are 4 GiB.  All keys are alike, only rows behind that point hold values."""
    rows, far = 2 ** 18, 64
    q = torch.ones(2, 64, 128, dtype=torch.float16, device="cuda")
    k = torch.zeros(rows + far + 2, 64, 128, dtype=torch.float16, device="cuda")
    v = torch.zeros_like(k)
    v[rows:] = 1024.0
    mass = torch.zeros(64, rows + far + 2, device="cuda")
    ctx = _context(2, 1, (64, 64, 128))
    got = ctx.tree_attention(q, k, v, [0], [rows + far], [0, 2], [-1, 0], mass=mass).double().cpu()
    want = torch.tensor([1024.0 * (far + 1) / (rows + far + 1), 1024.0 * (far + 2) / (rows + far + 2)]).double()
    # whole numbers times a probability that is one: sums exact, a division, the output's rounding
    assert (abs(got - want[:, None, None]) <= 2.0 ** -10 * want[:, None, None]).all()
    w = mass.double().cpu()
    p = 1 / (rows + far + 1) + 1 / (rows + far + 2)
    assert (abs(w[:, :rows + far + 1] - p) <= 2.0 ** -20 * p).all() and (abs(w[:, -1] * (rows + far + 2) - 1) <= 2.0 ** -20).all()


def test_utterances_may_share_their_rows_without_weights():
    c = Call("f16", (4, 2, 128), [90, 90], [[-1, 0, 0], [-1, 0, 0]], seed=15)
    c.kv_start[1] = c.kv_start[0]
    c.check(mass=False)
    with pytest.raises(RuntimeError, match="share slots"):
        c.run()


def test_results_do_not_depend_on_the_batch_and_repeat():
    """Utterances alone and together: the same bits, run after run."""
    trees = _batch(16, None, [6, 6, 6])
    c = Call("bf16", (16, 8, 128), [50, 70, 90], trees, seed=17)
    first = c.run().clone(), c.mass_out.clone()
    ctx = _context(18, 3, c.heads)
    for _ in range(3):
        assert torch.equal(c.run(ctx), first[0]) and torch.equal(c.mass_out, first[1])


@pytest.mark.parametrize("nodes", [[6, 3], [300, 700, 90, 400]])
def test_captured_calls(nodes):
    """Few and many nodes: replays after other calls of the same context with other trees give what the eager call gave."""
    trees = _batch(18, None, nodes, ("random",))
    c = Call("f16", (4, 2, 64), [100 + 37 * i for i in range(len(nodes))], trees, seed=19)
    other = Call("f16", (4, 2, 64), [80 + 11 * i for i in range(len(nodes))], _batch(20, None, nodes, ("chain",)), seed=21)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        ctx = Context(device="cuda:0", stream=s)
        ctx.reserve(tree_nodes=sum(nodes), tree_utts=len(nodes), tree_heads=c.heads)
        args = c.q, c.k, c.v, c.kv_start, c.ctx_len, cu(trees), flat(trees)
        want_mass = c.mass.clone()
        want = ctx.tree_attention(*args, mass=want_mass).clone()
        out, mass = torch.empty_like(want), c.mass.clone()
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            ctx.tree_attention(*args, out=out, mass=mass)
        for _ in range(3):
            out.zero_()
            mass.copy_(c.mass)
            other.run(ctx)
            s.synchronize()
            graph.replay()
            s.synchronize()
            assert torch.equal(out, want) and torch.equal(mass, want_mass)
